"""The operators around the SSD layer of a Mamba-2 block, as calls that can be timed and whose outputs can be compared.

  conv       `ssdi8_conv_fwd`       the short causal convolution of a prompt with its SiLU, ending in the int8 codes of
                                    x, B and C that the chunk scan takes (or in a tensor of the input's type, for calibration)
  cache      `ssdi8_cache_write`    states of finished prompts into slots of an 8-bit state cache, one step size per row
             `ssdi8_cache_read`     the states of slots back in fp32, with the tokens that wait in the slots' windows
  token      `ssdi8_token_step`     one token for every sequence: convolution, codes, time step and scan over the 8-bit cache
  norm       `ssdi8_norm_quantize`  RMS norm (with the block's gate) that ends in int8 codes for a projection
  linear     `ssdi8_linear`         int8 projection with step sizes, bias, activation and residual in its epilogue

Heads have 64 channels.  Int8 codes are whole numbers: a code is the nearest integer of the exact quotient of its
definition, and the plain forms compute what decides one in 64 bits.
"""
import math

import torch

own = False

P = 64        # head dimension (the only one the library takes)
WINDOW = 16   # tokens that wait beside a slot's state before they are folded into it

_SIZE = {"float32": 4, "float16": 2, "bfloat16": 2}


def listed():
    return [
        # one user's short prompt in a 130M-shaped bf16 model: latency and launches
        {"name": "conv 1x256x24", "op": "conv", "batch": 1, "seqlen": 256, "nheads": 24, "dstate": 128, "ngroups": 1,
         "dtype": "bfloat16", "width": 4, "codes": True, "ragged": False, "go_on": False},
        # the prefill batch of the 2.7B-shaped layer, read in place from the projection's rows
        {"name": "conv 8x2048x80", "op": "conv", "batch": 8, "seqlen": 2048, "nheads": 80, "dstate": 128, "ngroups": 1,
         "dtype": "bfloat16", "width": 4, "codes": True, "ragged": False, "go_on": False},
        # prompts of unequal lengths that go on from cached tails, two groups, fp16 out (a calibration run)
        {"name": "conv 5x1787x50 ragged", "op": "conv", "batch": 5, "seqlen": 1787, "nheads": 50, "dstate": 64, "ngroups": 2,
         "dtype": "float16", "width": 4, "codes": False, "ragged": True, "go_on": True},
        # the states of a prefill batch are put into the cache
        {"name": "cache write 8x80", "op": "cache", "write": True, "batch": 8, "nheads": 80, "dstate": 128, "ngroups": 1},
        # a large batch of conversations goes on: states with half-filled windows are read back
        {"name": "cache read 37x128", "op": "cache", "write": False, "batch": 37, "nheads": 128, "dstate": 128, "ngroups": 8},
        # decode of one sequence of the 130M shape: latency
        {"name": "token 1x24", "op": "token", "batch": 1, "nheads": 24, "dstate": 128, "ngroups": 1, "dtype": "bfloat16",
         "width": 4, "y": "bfloat16", "padded": 0},
        # decode of the 2.7B shape at batch 64 (the framework's decode workload)
        {"name": "token 64x80", "op": "token", "batch": 64, "nheads": 80, "dstate": 128, "ngroups": 1, "dtype": "bfloat16",
         "width": 4, "y": "bfloat16", "padded": 0},
        # decode of a large batch of the 8B shape with groups, a few rows of padding behind the last sequence
        {"name": "token 250x128", "op": "token", "batch": 250, "nheads": 128, "dstate": 128, "ngroups": 8, "dtype": "bfloat16",
         "width": 4, "y": "float32", "padded": 6},
        # the gated norm of a decode batch of the 2.7B shape
        {"name": "norm 64x5120 gated", "op": "norm", "rows": 64, "width": 5120, "groups": 1, "dtype": "bfloat16",
         "gate": "bfloat16", "static": False},
        # the gated norm of a prefill batch: the scan's fp32 y, the gate in place in the projection's rows
        {"name": "norm 16384x5120 gated", "op": "norm", "rows": 16384, "width": 5120, "groups": 1, "dtype": "float32",
         "gate": "bfloat16", "static": False},
        # the input projection of a decode batch: the weight is what is read
        {"name": "linear 64x10576x2560", "op": "linear", "rows": 64, "outs": 10576, "inner": 2560, "dtype": "bfloat16",
         "bias": False, "act": "none", "residual": False},
        # the output projection of a prefill batch, with the mean correction as its bias and the residual stream
        {"name": "linear 16384x2560x5120", "op": "linear", "rows": 16384, "outs": 2560, "inner": 5120, "dtype": "bfloat16",
         "bias": True, "act": "none", "residual": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng, most):
    G = rng.choice([1, 1, 1, 2, 4, 8])
    return G * max(1, _log_int(rng, 4, most) // G), G


def draw(rng):
    op = rng.choice(["conv", "conv", "cache", "token", "token", "norm", "linear", "linear"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    N = rng.choice([64, 128, 128])
    if op == "conv":
        H, G = _heads(rng, 128)
        b = _log_int(rng, 1, 16)
        L = max(1, min(_log_int(rng, 1, 8192), (8 * 2048 * 80) // (b * H)))
        return {"op": op, "batch": b, "seqlen": L, "nheads": H, "dstate": N, "ngroups": G, "dtype": dtype,
                "width": rng.choice([2, 3, 4, 4]), "codes": rng.random() < 0.7, "ragged": rng.random() < 0.5,
                "go_on": rng.random() < 0.5}
    if op == "cache":
        H, G = _heads(rng, 128)
        return {"op": op, "write": rng.random() < 0.5, "batch": min(_log_int(rng, 1, 128), max(1, 37 * 128 // H)), "nheads": H,
                "dstate": N, "ngroups": G}
    if op == "token":
        H, G = _heads(rng, 128)
        b = _log_int(rng, 1, 250)
        return {"op": op, "batch": b, "nheads": H, "dstate": N, "ngroups": G, "dtype": dtype, "width": rng.choice([2, 3, 4, 4]),
                "y": rng.choice(["bfloat16", "float16", "float32"]), "padded": rng.choice([0, 0, b // 8])}
    if op == "norm":
        groups = rng.choice([1, 1, 1, 2, 8])
        D = groups * 128 * max(1, _log_int(rng, 2, 64) // groups) if groups > 1 else 16 * _log_int(rng, 16, 512)
        return {"op": op, "rows": min(_log_int(rng, 1, 16384), 16384 * 5120 // D), "width": D, "groups": groups, "dtype": dtype,
                "gate": rng.choice(["none", "bfloat16", "float16", "float32"]), "static": rng.random() < 0.3}
    T, O, K = _log_int(rng, 1, 16384), _log_int(rng, 24, 18560), 16 * _log_int(rng, 16, 512)
    T = max(1, min(T, 16384 * 2560 * 5120 // (O * K)))
    return {"op": op, "rows": T, "outs": O, "inner": K, "dtype": dtype, "bias": rng.random() < 0.5,
            "act": rng.choice(["none", "none", "silu", "relu2"]), "residual": rng.random() < 0.5}


# ---------------------------------------------------------------------------------------------------------- inputs
class _Random:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, *shape, dtype=torch.float32):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=dtype)

    def uniform(self, lo, hi, *shape):
        return torch.rand(shape, generator=self.g, device="cuda") * (hi - lo) + lo

    def whole(self, lo, hi, *shape, dtype=torch.int32):
        return torch.randint(lo, hi, shape, generator=self.g, device="cuda", dtype=dtype)

    def codes(self, *shape, std=40.0):
        """int8 codes as Eq. 1 gives them for normal values: most are small, a few are at the ends"""
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float16).mul_(std).round_().clamp_(-127, 127).to(torch.int8)

    def order(self, n):
        return torch.randperm(n, generator=self.g, device="cuda").to(torch.int32)


def _dims(case):
    H, G, N = case["nheads"], case["ngroups"], case["dstate"]
    return H, G, N, H * P, H * P + 2 * G * N


def _conv_inputs(r, case, b, L):
    """Rows of the input projection [z | xBC | dt], the convolution's parameters and the static step sizes."""
    H, G, N, HP, Ch = _dims(case)
    W, dtype = case["width"], getattr(torch, case["dtype"])
    row = HP + Ch + H
    rows = r.normal(b, L, row, dtype=dtype)
    gain = torch.ones(Ch, device="cuda")
    gain[r.order(HP).long()[:math.ceil(0.01 * HP)]] = 50.0   # outlier channels of x
    weight, bias = r.uniform(-0.5, 0.5, Ch, W) * gain[:, None], 0.1 * r.normal(Ch)
    s = (3.5 / 127.0) * (weight.square().sum(1) + 0.01).sqrt()
    st = {"rows": rows, "xBC": rows[..., HP:HP + Ch], "dt_raw": rows[..., HP + Ch:], "weight": weight, "bias": bias,
          "s_x": s[:HP].contiguous(), "s_B": torch.full((G,), 2.0 / 127.0, device="cuda"),
          "s_C": torch.full((G,), 2.0 / 127.0, device="cuda"), "dt_bias": -3.0 + 0.25 * r.normal(H),
          "A": -torch.exp(r.uniform(0.0, math.log(16.0), H)), "D": r.normal(H), "corr": 0.01 * r.normal(HP)}
    return st


def _cache_tensors(r, case, nslots, ring):
    H, G, N, HP, Ch = _dims(case)
    c = {"codes": torch.empty(nslots, H, P, N, dtype=torch.int8, device="cuda"), "scales": r.uniform(0.005, 0.05, nslots, H, P),
         "xwin": r.codes(nslots, H, WINDOW, P), "Bwin": r.codes(nslots, G, WINDOW, N),
         "dtwin": torch.nn.functional.softplus(r.normal(nslots, H, WINDOW) - 3.0),
         "start": r.whole(0, 40, nslots), "ring": ring}
    c["codes"].copy_(r.codes(H, P, N)[None])
    for k in range(min(nslots, 8)):
        c["codes"][k::8] = r.codes(H, P, N)[None]
    return c


def prepare(case, seed):
    r, op = _Random(seed), case["op"]
    empty = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    if op == "conv":
        H, G, N, HP, Ch = _dims(case)
        b, L, W, dtype = case["batch"], case["seqlen"], case["width"], getattr(torch, case["dtype"])
        st = _conv_inputs(r, case, b, L)
        nslots = b + 3
        st["lens"] = r.whole(0, L + 1, b) if case["ragged"] else None
        st["pos"] = r.whole(0, 1000, b) if case["go_on"] else None
        st["slots"], st["ring"] = r.order(nslots)[:b].contiguous(), r.normal(nslots, W, Ch, dtype=dtype)
        st["dt"] = empty(b, L, H)
        if case["codes"]:
            st.update(xq=empty(b, L, HP, dtype=torch.int8), Bq=empty(b, L, G * N, dtype=torch.int8),
                      Cq=empty(b, L, G * N, dtype=torch.int8), out=None)
        else:
            st.update(xq=None, Bq=None, Cq=None, out=empty(b, L, Ch, dtype=dtype))
    elif op == "cache":
        H, G, N, HP, Ch = _dims(case)
        b = case["batch"]
        nslots = b + 5
        st = {"cache": _cache_tensors(r, case, nslots, r.normal(nslots, 4, Ch, dtype=torch.bfloat16)),
              "slots": r.order(nslots)[:b].contiguous(), "A": -torch.exp(r.uniform(0.0, math.log(16.0), H)),
              "s_x": r.uniform(0.01, 0.05, HP), "s_B": torch.full((G,), 2.0 / 127.0, device="cuda")}
        st["pos"] = r.whole(40, 5000, b)
        st["state"] = r.normal(b, H, P, N) * r.uniform(0.1, 3.0, 1, H, P, 1) if case["write"] else r.normal(b, H, P, N)
    elif op == "token":
        H, G, N, HP, Ch = _dims(case)
        b = case["batch"]
        nslots = b + b // 16 + 2
        st = _conv_inputs(r, case, b, 1)
        st.update(xBC=st["xBC"][:, 0], dt_raw=st["dt_raw"][:, 0])
        st["cache"] = _cache_tensors(r, case, nslots, r.normal(nslots, case["width"], Ch, dtype=getattr(torch, case["dtype"])))
        st["slots"] = r.order(nslots)[:b].contiguous()
        if case["padded"]:
            st["slots"][b - case["padded"]:] = -1
        st["pos"] = r.whole(40, 5000, b)
        st["y"] = r.normal(b, HP, dtype=getattr(torch, case["y"]))
    elif op == "norm":
        T, D, dtype = case["rows"], case["width"], getattr(torch, case["dtype"])
        st = {"x": r.normal(T, D, dtype=dtype), "weight": r.uniform(0.5, 1.5, D), "xq": empty(T, D, dtype=torch.int8),
              "scale": empty(T), "z": None, "static": None}
        st["x"] *= torch.where(torch.rand(D, generator=r.g, device="cuda") < 0.01, 20.0, 1.0).to(dtype)
        if case["gate"] != "none":
            st["z"] = r.normal(T, 2 * D + 272, dtype=getattr(torch, case["gate"]))[:, :D]   # (in place in the projection's rows)
        if case["static"]:
            st["static"] = torch.full((1,), 6.0 / 127.0, device="cuda")
    else:
        T, O, K, dtype = case["rows"], case["outs"], case["inner"], getattr(torch, case["dtype"])
        st = {"xq": r.codes(T, K), "wq": r.codes(O, K, std=30.0), "s_row": r.uniform(0.01, 0.05, T),
              "s_w": r.uniform(0.5, 1.5, O) / (40.0 * math.sqrt(K)), "bias": 0.1 * r.normal(O) if case["bias"] else None,
              "residual": r.normal(T, O, dtype=dtype) if case["residual"] else None, "out": empty(T, O, dtype=dtype)}
    st["case"] = case
    return st


# ---------------------------------------------------------------------------------------------------------- plain forms
def _silu(v):
    return v / (1.0 + torch.exp(-v))


def _round(v):
    return torch.round(v).clamp(-127, 127).to(torch.int8)


def _softplus(v):
    return torch.clamp(v, min=0.0) + torch.log1p(torch.exp(-v.abs()))


def _heads_of(t, H):
    """[.., G, ..] at dimension 1 -> [.., H, ..]"""
    return t.repeat_interleave(H // t.shape[1], dim=1)


def _plain_conv(st):
    c = st["case"]
    H, G, N, HP, Ch = _dims(c)
    b, L, W = c["batch"], c["seqlen"], c["width"]
    x, ring, slots = st["xBC"], st["ring"], st["slots"].long()
    zero = torch.zeros(b, dtype=torch.long, device="cuda")
    pos = zero if st["pos"] is None else st["pos"].long()
    lens = zero + L if st["lens"] is None else st["lens"].long()
    # the W - 1 tokens ahead of the call; those of negative positions are zeros
    before = pos[:, None] - (W - 1) + torch.arange(W - 1, device="cuda")
    past = ring[slots[:, None], before % W] * (before >= 0)[..., None]
    v = (torch.cat([past, x], 1).unfold(1, W, 1).double() * st["weight"].double()).sum(-1) + st["bias"].double()
    live = torch.arange(L, device="cuda") < lens[:, None]
    v = _silu(v) * live[..., None]
    # the last W tokens stay in the ring, token t in row t mod W
    rows = torch.arange(W, device="cuda")
    end = (pos + lens)[:, None]
    at = end - 1 - (end - 1 - rows) % W - pos[:, None]
    new = torch.gather(x, 1, at.clamp(min=0)[..., None].expand(b, W, Ch))
    ring[slots] = torch.where((at >= 0)[..., None], new, ring[slots])
    st["dt"].copy_(_softplus((st["dt_raw"].float() + st["dt_bias"]).double()) * live[..., None])
    out = {"dt": st["dt"], "ring": ring}
    if not c["codes"]:
        st["out"].copy_(v)
        return {**out, "out": st["out"]}
    st["xq"].copy_(_round(v[..., :HP] / st["s_x"].double()))
    st["Bq"].copy_(_round(v[..., HP:HP + G * N] / st["s_B"].double().repeat_interleave(N)))
    st["Cq"].copy_(_round(v[..., HP + G * N:] / st["s_C"].double().repeat_interleave(N)))
    return {**out, "xq": st["xq"], "Bq": st["Bq"], "Cq": st["Cq"]}


def _window(cache, slots, pos, A):
    """Time steps of the tokens that wait in the windows up to position `pos` (0 elsewhere), each one's decay from behind
    it up to `pos`, and the decay of the state ahead of the window.  64 bits."""
    first = pos // WINDOW * WINDOW
    at = first[:, None] + torch.arange(WINDOW, device="cuda")
    inside = (at >= torch.maximum(cache["start"][slots].long(), first)[:, None]) & (at <= pos[:, None])
    dt = cache["dtwin"][slots].double() * inside[:, None]
    behind = dt.sum(-1, keepdim=True) - dt.cumsum(-1)
    A = A.double()[None, :, None]
    return dt, torch.exp(A * behind), torch.exp(A * dt.sum(-1, keepdim=True))


def _folded(st, slots, pos):
    """fp64 states of slots with the tokens up to `pos`"""
    cache, H = st["cache"], st["case"]["nheads"]
    dt, decay, whole = _window(cache, slots, pos, st["A"])
    w = (dt * decay)[..., None] * cache["xwin"][slots].double()                       # [b, H, WINDOW, P]
    B = _heads_of(cache["Bwin"][slots].double() * st["s_B"].double()[:, None, None], H)
    new = torch.matmul(w.transpose(2, 3), B) * st["s_x"].double().view(H, P, 1)
    return whole[..., None] * cache["scales"][slots].double()[..., None] * cache["codes"][slots].double() + new


def _plain_cache(st):
    cache, slots, pos = st["cache"], st["slots"].long(), st["pos"].long()
    if not st["case"]["write"]:
        st["state"].copy_(_folded(st, slots, pos - 1))
        return {"state": st["state"]}
    most = st["state"].abs().amax(-1)
    step = torch.where(most > 0, most / torch.full_like(most, 127.0), torch.ones_like(most))
    cache["codes"][slots] = _round(st["state"] / step[..., None])
    cache["scales"][slots] = step
    cache["start"][slots] = st["pos"]
    return {k: cache[k] for k in ("codes", "scales", "start")}


def _plain_token(st):
    c, cache = st["case"], st["cache"]
    H, G, N, HP, Ch = _dims(c)
    W = c["width"]
    rows = (st["slots"] >= 0).nonzero().squeeze(1)
    slots, pos = st["slots"][rows].long(), st["pos"][rows].long()
    b = rows.numel()
    # convolution and codes
    before = pos[:, None] - (W - 1) + torch.arange(W - 1, device="cuda")
    past = cache["ring"][slots[:, None], before % W] * (before >= 0)[..., None]
    x = st["xBC"][rows]
    v = _silu((torch.cat([past, x[:, None]], 1).transpose(1, 2).double() * st["weight"].double()).sum(-1) + st["bias"].double())
    xq = _round(v[:, :HP] / st["s_x"].double()).view(b, H, P)
    Bq = _round(v[:, HP:HP + G * N].view(b, G, N) / st["s_B"].double()[:, None])
    Cq = _round(v[:, HP + G * N:].view(b, G, N) / st["s_C"].double()[:, None])
    cache["ring"][slots, pos % W] = x
    # into the window
    cache["xwin"][slots, :, pos % WINDOW] = xq
    cache["Bwin"][slots, :, pos % WINDOW] = Bq
    cache["dtwin"][slots, :, pos % WINDOW] = _softplus((st["dt_raw"][rows].float() + st["dt_bias"]).double()).float()
    # y from the state ahead of the window and the tokens inside it
    dt, decay, whole = _window(cache, slots, pos, st["A"])
    Cf = Cq.float()
    CB = _heads_of((Cf[:, :, None] * cache["Bwin"][slots].float()).sum(-1), H)
    sB, sC = st["s_B"].repeat_interleave(H // G)[:, None], st["s_C"].repeat_interleave(H // G)[:, None]
    s_x = st["s_x"].view(H, P)
    off = (cache["codes"][slots] * _heads_of(Cf, H)[:, :, None]).sum(-1)
    y = whole.float() * cache["scales"][slots] * off
    y = y + s_x * sB * ((dt * decay).float() * CB)[..., None].mul(cache["xwin"][slots]).sum(2)
    y = sC * y + st["D"][:, None] * s_x * xq + st["corr"].view(H, P)
    st["y"][rows] = y.reshape(b, HP).to(st["y"].dtype)
    # full windows are folded into the state
    full = (pos % WINDOW == WINDOW - 1).nonzero().squeeze(1)
    S = _folded(st, slots[full], pos[full])
    most = S.abs().amax(-1)
    step = torch.where(most > 0, most / torch.full_like(most, 127.0), torch.ones_like(most)).float()
    cache["codes"][slots[full]] = _round(S / step[..., None].double())
    cache["scales"][slots[full]] = step
    return {"y": st["y"], **{k: cache[k] for k in ("codes", "scales", "xwin", "Bwin", "dtwin", "ring")}}


def _plain_norm(st):
    c = st["case"]
    T, D, ng = c["rows"], c["width"], c["groups"]
    u = st["x"].double()
    if st["z"] is not None:
        u = u * _silu(st["z"].double())
    u = u.view(T, ng, D // ng)
    u = (u / torch.sqrt(u.square().mean(-1, keepdim=True) + 1e-5)).view(T, D) * st["weight"].double()
    if st["static"] is not None:
        st["xq"].copy_(_round(u / st["static"].double()))
        return {"xq": st["xq"]}
    most = u.abs().amax(-1, keepdim=True)
    step = torch.where(most > 0, most / torch.full_like(most, 127.0), torch.ones_like(most))
    st["xq"].copy_(_round(u / step))
    st["scale"].copy_(step[:, 0])
    return {"xq": st["xq"], "scale": st["scale"]}


def _plain_linear(st):
    v = torch.matmul(st["xq"].float(), st["wq"].float().t()) * st["s_row"][:, None] * st["s_w"]
    if st["bias"] is not None:
        v = v + st["bias"]
    if st["case"]["act"] == "silu":
        v = _silu(v)
    if st["case"]["act"] == "relu2":
        v = v.clamp(min=0.0).square()
    if st["residual"] is not None:
        v = v + st["residual"].float()
    st["out"].copy_(v)
    return {"out": st["out"]}


_PLAIN = {"conv": _plain_conv, "cache": _plain_cache, "token": _plain_token, "norm": _plain_norm, "linear": _plain_linear}


# ---------------------------------------------------------------------------------------------------------- the framework's calls
def _own(st):
    from paper_2608_21952_b200 import binding as bd
    c, op = st["case"], st["case"]["op"]
    if op == "norm":
        bd.ssdi8_norm_quantize(st["x"], st["xq"], weight=st["weight"], z=st["z"], groups=c["groups"], eps=1e-5,
                               scale=st["scale"] if st["static"] is None else None, static_scale=st["static"])
        return {"xq": st["xq"], "scale": st["scale"]} if st["static"] is None else {"xq": st["xq"]}
    if op == "linear":
        act = {"none": bd.ACT_NONE, "silu": bd.ACT_SILU, "relu2": bd.ACT_RELU2}[c["act"]]
        bd.ssdi8_linear(st["xq"], st["wq"], st["s_w"], st["out"], s_row=st["s_row"], bias=st["bias"], residual=st["residual"],
                        act=act)
        return {"out": st["out"]}
    if "dims" not in st:   # (the handles that a user's program makes once)
        st["dims"] = bd.Dims(c["batch"], c.get("seqlen", 1), c["nheads"], P, c["dstate"], c["ngroups"], 0)
        if op != "conv":
            st["handle"] = bd.cache_of(st["dims"], **st["cache"])
        if op == "cache":   # (a full window is read as it stands, with its 16 tokens beside the codes)
            st["first"] = torch.maximum(st["cache"]["start"][st["slots"].long()], (st["pos"] - 1) // WINDOW * WINDOW)
    if op == "conv":
        bd.ssdi8_conv_fwd(st["dims"], st["xBC"], st["weight"], st["bias"], s_x=st["s_x"], s_B=st["s_B"], s_C=st["s_C"],
                          xq=st["xq"], Bq=st["Bq"], Cq=st["Cq"], out=st["out"], dt_raw=st["dt_raw"], dt_bias=st["dt_bias"],
                          dt=st["dt"], lens=st["lens"], ring=st["ring"], slots=st["slots"], pos=st["pos"],
                          flags=bd.FLAG_DT_SOFTPLUS)
        return {k: st[k] for k in (("dt", "ring", "xq", "Bq", "Cq") if c["codes"] else ("dt", "ring", "out"))}
    cache = st["cache"]
    if op == "cache" and c["write"]:
        bd.ssdi8_cache_write(st["dims"], st["handle"], st["slots"], st["pos"], st["state"])
        return {k: cache[k] for k in ("codes", "scales", "start")}
    if op == "cache":
        bd.ssdi8_cache_read(st["dims"], st["handle"], st["slots"], st["pos"], st["A"], st["s_x"], st["s_B"], st["state"],
                            first=st["first"])
        return {"state": st["state"]}
    bd.ssdi8_token_step(st["dims"], st["handle"], st["xBC"], st["weight"], st["bias"], st["dt_raw"], st["dt_bias"], st["A"],
                        st["D"], st["corr"], st["s_x"], st["s_B"], st["s_C"], st["slots"], st["pos"], st["y"],
                        flags=bd.FLAG_DT_SOFTPLUS)
    return {"y": st["y"], **{k: cache[k] for k in ("codes", "scales", "xwin", "Bwin", "dtwin", "ring")}}


def run(st):
    if own:
        return _own(st)
    return _PLAIN[st["case"]["op"]](st)


# ---------------------------------------------------------------------------------------------------------- work
def work(case):
    """Inputs read once and outputs written once; two operations per multiply-accumulate, and what a plain reading of the
    formula takes elsewhere."""
    op = case["op"]
    if op == "norm":
        T, D = case["rows"], case["width"]
        gate = _SIZE.get(case["gate"], 0)
        return {"bytes": T * D * (_SIZE[case["dtype"]] + gate + 1) + 4 * D + 4 * T, "flops": 8.0 * T * D}
    if op == "linear":
        T, O, K, e = case["rows"], case["outs"], case["inner"], _SIZE[case["dtype"]]
        return {"bytes": T * K + O * K + T * O * e * (2 if case["residual"] else 1) + 4 * T + 8 * O, "flops": 2.0 * T * O * K}
    H, G, N, HP, Ch = _dims(case)
    b = case["batch"]
    state = b * H * P * N
    if op == "conv":
        T, e = b * case["seqlen"] / (2 if case["ragged"] else 1), _SIZE[case["dtype"]]
        out = b * case["seqlen"] * Ch * (1 if case["codes"] else e)   # (rows behind a short prompt are written too)
        return {"bytes": T * (Ch * e + H * e) + b * case["seqlen"] * H * 4 + out + Ch * 4 * (case["width"] + 2),
                "flops": T * Ch * (2.0 * case["width"] + 6)}
    if op == "cache":
        window = b * (H * WINDOW * (P + 4) + G * WINDOW * N) / 2
        if case["write"]:
            return {"bytes": 5 * state + 4 * b * H * P, "flops": 3.0 * state}
        return {"bytes": 5 * state + 4 * b * H * P + window, "flops": state * (2.0 + WINDOW)}
    b -= case["padded"]
    state, e = b * H * P * N, _SIZE[case["dtype"]]
    window = b * (H * (P + 4) + G * N) * (WINDOW / 2 + 1)
    fold = (state + 4 * b * H * P) / WINDOW
    return {"bytes": state + 4 * b * H * P + window + fold + b * (Ch * e * (case["width"] + 1) + H * e + HP * _SIZE[case["y"]])
            + Ch * 4 * (case["width"] + 2), "flops": state * (2.0 + 2.0) + 2.0 * WINDOW * b * H * (P + N)}


# ---------------------------------------------------------------------------------------------------------- 64 bits
def _exact_conv_values(st, x, past):
    """SiLU of the convolution of [.., tokens, channels], after W - 1 tokens `past`, in 64 bits"""
    full = torch.cat([past, x], 1).double().transpose(1, 2)
    v = torch.nn.functional.conv1d(full, st["weight"].double()[:, None], st["bias"].double(), groups=full.shape[1])
    return torch.nn.functional.silu(v).transpose(1, 2)


def _exact_past(ring, slot, pos, W):
    """the W - 1 tokens ahead of position `pos` of one sequence"""
    rows = [ring[slot, t % W] if t >= 0 else torch.zeros_like(ring[slot, 0]) for t in range(pos - W + 1, pos)]
    return torch.stack(rows)[None]


def _exact_step(v, most):
    return torch.where(most > 0, most / 127.0, torch.ones_like(most))


def exact(case, seed):
    st, op = prepare(case, seed), case["op"]
    if op == "linear":
        v = (st["xq"].double() @ st["wq"].double().t()) * (st["s_row"].double()[:, None] * st["s_w"].double())
        v = v if st["bias"] is None else v + st["bias"].double()
        v = torch.nn.functional.silu(v) if case["act"] == "silu" else torch.relu(v) ** 2 if case["act"] == "relu2" else v
        return {"out": v if st["residual"] is None else v + st["residual"].double()}
    if op == "norm":
        T, D, ng = case["rows"], case["width"], case["groups"]
        u = st["x"].double()
        u = u if st["z"] is None else u * torch.nn.functional.silu(st["z"].double())
        norm = torch.linalg.vector_norm(u.view(T, ng, -1), dim=-1, keepdim=True) ** 2 / (D // ng)
        u = (u.view(T, ng, -1) * torch.rsqrt(norm + 1e-5)).reshape(T, D) * st["weight"].double()
        if case["static"]:
            return {"xq": None}
        return {"xq": None, "scale": _exact_step(u, torch.linalg.vector_norm(u, ord=math.inf, dim=-1))}
    H, G, N, HP, Ch = _dims(case)
    b = case["batch"]
    if op == "conv":
        W, L = case["width"], case["seqlen"]
        pos = [0] * b if st["pos"] is None else st["pos"].tolist()
        lens = [L] * b if st["lens"] is None else st["lens"].tolist()
        slots, ring = st["slots"].tolist(), st["ring"].double()
        out, dt = torch.zeros(b, L, Ch, dtype=torch.float64, device="cuda"), torch.zeros(b, L, H, dtype=torch.float64, device="cuda")
        raw = (st["dt_raw"].float() + st["dt_bias"]).double()
        for i in range(b):
            n = lens[i]
            if not case["codes"] and n:
                out[i, :n] = _exact_conv_values(st, st["xBC"][i:i + 1, :n], _exact_past(st["ring"], slots[i], pos[i], W))[0]
            dt[i, :n] = torch.nn.functional.softplus(raw[i, :n], threshold=1000.0)
            for t in range(max(0, n - W), n):
                ring[slots[i], (pos[i] + t) % W] = st["xBC"][i, t].double()
        if case["codes"]:
            return {"dt": dt, "ring": ring, "xq": None, "Bq": None, "Cq": None}
        return {"dt": dt, "ring": ring, "out": out}
    cache, slots, pos = st["cache"], st["slots"].tolist(), st["pos"].tolist()
    A, s_x, s_B = st["A"].double(), st["s_x"].double().view(H, P), st["s_B"].double()
    group = torch.arange(H, device="cuda") // (H // G)
    start = cache["start"].tolist()

    def advance(h, slot, t):
        """the recurrence h = exp(dt A) h + dt x B of one waiting token, [H, P, N]"""
        dt = cache["dtwin"][slot, :, t % WINDOW].double()
        x = s_x * cache["xwin"][slot, :, t % WINDOW].double()
        B = (s_B[:, None] * cache["Bwin"][slot, :, t % WINDOW].double())[group]
        return torch.exp(dt * A)[:, None, None] * h + (dt[:, None] * x)[..., None] * B[:, None]

    if op == "cache":
        if case["write"]:
            scales = cache["scales"].double()
            scales[st["slots"].long()] = _exact_step(None, st["state"].double().abs().amax(-1))
            return {"codes": None, "scales": scales, "start": None}
        out = torch.empty(b, H, P, N, dtype=torch.float64, device="cuda")
        for i in range(b):
            h, last = cache["scales"][slots[i]].double()[..., None] * cache["codes"][slots[i]].double(), pos[i] - 1
            for t in range(max(start[slots[i]], last - last % WINDOW), last + 1):
                h = advance(h, slots[i], t)
            out[i] = h
        return {"state": out}
    W = case["width"]
    y, scales, dtwin, ring = st["y"].double(), cache["scales"].double(), cache["dtwin"].double(), cache["ring"].double()
    quant = lambda v, s: torch.round(v / s).clamp(-127, 127)  # noqa: E731
    for i in range(b):
        slot, p = slots[i], pos[i]
        if slot < 0:
            continue
        v = _exact_conv_values(st, st["xBC"][i:i + 1, None], _exact_past(cache["ring"], slot, p, W))[0, 0]
        xq = quant(v[:HP].view(H, P), s_x)
        Bq = quant(v[HP:HP + G * N].view(G, N), s_B[:, None])
        C = (st["s_C"].double()[:, None] * quant(v[HP + G * N:].view(G, N), st["s_C"].double()[:, None]))[group]
        dt = torch.nn.functional.softplus((st["dt_raw"][i].float() + st["dt_bias"]).double(), threshold=1000.0)
        ring[slot, p % W] = st["xBC"][i].double()
        dtwin[slot, :, p % WINDOW] = dt
        cache["xwin"][slot, :, p % WINDOW], cache["Bwin"][slot, :, p % WINDOW] = xq.to(torch.int8), Bq.to(torch.int8)
        cache["dtwin"][slot, :, p % WINDOW] = dt.float()
        h = scales[slot][..., None] * cache["codes"][slot].double()
        for t in range(max(start[slot], p - p % WINDOW), p + 1):
            h = advance(h, slot, t)
        y[i] = ((h * C[:, None]).sum(-1) + st["D"].double()[:, None] * s_x * xq + st["corr"].double().view(H, P)).view(HP)
        if p % WINDOW == WINDOW - 1:
            scales[slot] = _exact_step(None, h.abs().amax(-1))
    return {"y": y, "codes": None, "scales": scales, "xwin": None, "Bwin": None, "dtwin": dtwin, "ring": ring}
