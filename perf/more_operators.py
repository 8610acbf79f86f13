"""Projections in four bits and the norm ahead of them, as calls that can be timed and whose outputs can be compared.

  norm       `ssdi8_add_norm_quantize`   the residual stream's addition and the RMS norm behind it, ending in int8 codes with a step
                                         size per row (or a static one), or in four bits
  quantize   `ssdi8_fp4_quantize`        rows to four bits with a scale per block, and their values back
             `ssdi8_fp4_dequantize`
  linear     `ssdi8_fp4_linear`          the product of two matrices in four bits, with bias, activation and residual

Four bits: a code is one of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} (e2m1), two to a byte, the even column's in the low half.  A block is 16
columns with a scale in e4m3, or 32 with a power of two (e8m0); a row has a step size in binary32 beside them.  The scales stand in
tiles of 128 rows and 4 blocks: row 32 i + j of a tile has its four bytes at [j][i].
"""
import math

import torch

own = False

_SIZE = {"float32": 4, "float16": 2, "bfloat16": 2}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # one user's next token in a 130M-shaped model: the residual stream is fp32, latency is what counts
        {"name": "norm 1x768", "op": "norm", "rows": 1, "width": 768, "dtype": "bfloat16", "residual": "float32", "out": "int8"},
        # a decode batch of the 2.7B shape ahead of an input projection in four bits
        {"name": "norm 64x2560 fp4", "op": "norm", "rows": 64, "width": 2560, "dtype": "bfloat16", "residual": "float32", "out": "fp4 16"},
        # prompts of unequal lengths packed together, an fp16 model of an odd width
        {"name": "norm 3439x1248 fp4 32", "op": "norm", "rows": 3439, "width": 1248, "dtype": "float16", "residual": "float16", "out": "fp4 32"},
        # the prefill batch of the 2.7B shape
        {"name": "norm 16384x2560", "op": "norm", "rows": 16384, "width": 2560, "dtype": "bfloat16", "residual": "float32", "out": "int8"},
        # activations of a decode batch ahead of the output projection
        {"name": "quantize 64x5120", "op": "quantize", "rows": 64, "width": 5120, "dtype": "bfloat16", "block": 16},
        # a weight that is laid out, from fp32
        {"name": "quantize 10576x2560", "op": "quantize", "rows": 10576, "width": 2560, "dtype": "float32", "block": 32},
        # activations of the prefill batch
        {"name": "quantize 16384x5120", "op": "quantize", "rows": 16384, "width": 5120, "dtype": "bfloat16", "block": 16},
        # the input projection for one token: the weight is what is read
        {"name": "linear 1x10576x2560", "op": "linear", "rows": 1, "outs": 10576, "inner": 2560, "block": 16, "dtype": "bfloat16",
         "bias": False, "act": "none", "residual": False},
        # the same for a decode batch
        {"name": "linear 64x10576x2560", "op": "linear", "rows": 64, "outs": 10576, "inner": 2560, "block": 16, "dtype": "bfloat16",
         "bias": False, "act": "none", "residual": False},
        # a large decode batch of the 8B shape, powers of two as scales
        {"name": "linear 250x18560x4096", "op": "linear", "rows": 250, "outs": 18560, "inner": 4096, "block": 32, "dtype": "bfloat16",
         "bias": True, "act": "silu", "residual": False},
        # prompts of unequal lengths packed together, rows of out off 16-byte boundaries
        {"name": "linear 3439x16470x1248", "op": "linear", "rows": 3439, "outs": 16470, "inner": 1248, "block": 16, "dtype": "float16",
         "bias": False, "act": "none", "residual": True},
        # the output projection of the prefill batch, with the mean correction as its bias and the residual stream
        {"name": "linear 16384x2560x5120", "op": "linear", "rows": 16384, "outs": 2560, "inner": 5120, "block": 16, "dtype": "bfloat16",
         "bias": True, "act": "none", "residual": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "quantize", "linear", "linear", "linear"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    if op == "norm":
        out = rng.choice(["int8", "int8", "int8 static", "fp4 16", "fp4 16", "fp4 32"])
        D = 32 * _log_int(rng, 8, 512)
        return {"op": op, "rows": min(_log_int(rng, 1, 16384), 16384 * 2560 // D), "width": D, "dtype": dtype,
                "residual": rng.choice(["none", "float32", dtype]), "out": out}
    if op == "quantize":
        D = 32 * _log_int(rng, 8, 512)
        return {"op": op, "rows": min(_log_int(rng, 1, 18560), 16384 * 5120 // D), "width": D, "dtype": dtype, "block": rng.choice([16, 16, 32])}
    T, O, K = _log_int(rng, 1, 16384), _log_int(rng, 24, 18560), 32 * _log_int(rng, 8, 256)
    T = max(1, min(T, 16384 * 2560 * 5120 // (O * K)))
    return {"op": op, "rows": T, "outs": O, "inner": K, "block": rng.choice([16, 16, 32]), "dtype": dtype, "bias": rng.random() < 0.5,
            "act": rng.choice(["none", "none", "silu", "relu2"]), "residual": rng.random() < 0.5}


# ---------------------------------------------------------------------------------------------------------- inputs
class _Random:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, *shape, dtype=torch.float32):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=dtype)

    def uniform(self, lo, hi, *shape):
        return torch.rand(shape, generator=self.g, device="cuda") * (hi - lo) + lo

    def bytes(self, lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=self.g, device="cuda", dtype=torch.uint8)


def _fp4_empty(rows, width, block):
    """codes, scales in their tiles, step sizes of rows"""
    tiles = (-(-rows // 128), -(-(width // block) // 4), 32, 4, 4)
    return {"codes": torch.zeros(rows, width // 2, dtype=torch.uint8, device="cuda"),
            "scales": torch.zeros(tiles, dtype=torch.uint8, device="cuda"), "step": torch.ones(rows, device="cuda")}


def _fp4_codes(r, rows, width):
    """bytes of two codes each, as blocks of normal values have them whose largest is scaled to 6"""
    like = [int(min(range(8), key=lambda c: abs(E2M1[c] - v))) for v in (0.2, 0.6, 1.0, 1.4, 2.0, 2.6, 3.5, 5.2)]
    of = torch.tensor([c | 8 * s for s in (0, 1) for c in like], dtype=torch.uint8, device="cuda")
    b = r.bytes(0, 256, rows, width // 2)
    pair = of[torch.arange(256, device="cuda") & 15] | of[torch.arange(256, device="cuda") >> 4] << 4
    return pair[b.int()]


def prepare(case, seed):
    r, op = _Random(seed), case["op"]
    if op == "linear":
        T, O, K, block, dtype = case["rows"], case["outs"], case["inner"], case["block"], getattr(torch, case["dtype"])
        st = {"x": _fp4_empty(T, K, block), "w": _fp4_empty(O, K, block), "out": torch.empty(T, O, dtype=dtype, device="cuda")}
        lo, hi = (72, 127) if block == 16 else (121, 128)   # scales over a factor of about 100 (e4m3: 4 to 448; powers of two: 1/64 to 1)
        mean = 150.0 if block == 16 else 0.2
        for k, rows, size in (("x", T, 1.0), ("w", O, 1.0 / math.sqrt(K))):
            st[k]["codes"] = _fp4_codes(r, rows, K)
            live = _tiled(r.bytes(lo, hi, rows, K // block))
            st[k]["scales"].copy_(live)
            st[k]["step"].copy_(r.uniform(0.5, 1.5, rows) * (size / (3.0 * mean)))
        st["bias"] = 0.1 * r.normal(O) if case["bias"] else None
        st["residual"] = r.normal(T, O, dtype=dtype) if case["residual"] else None
        return {**st, "case": case}
    T, D, dtype = case["rows"], case["width"], getattr(torch, case["dtype"])
    st = {"x": r.normal(T, D, dtype=dtype)}
    st["x"] *= torch.where(torch.rand(D, generator=r.g, device="cuda") < 0.01, 20.0, 1.0).to(dtype)   # outlier channels
    block = case["block"] if op == "quantize" else int(case["out"][4:]) if case["out"][:3] == "fp4" else 0
    if block:
        st.update(q=_fp4_empty(T, D, block), block=block, values=torch.empty(T, D, dtype=dtype, device="cuda"))
    if op == "norm":
        st["weight"], st["residual"], st["stream"], st["static"] = r.uniform(0.5, 1.5, D), None, None, None
        if case["residual"] != "none":
            st["residual"] = r.normal(T, D, dtype=getattr(torch, case["residual"]))
            st["stream"] = torch.empty_like(st["residual"])
        if not block:
            st["xq"], st["scale"] = torch.empty(T, D, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
            if case["out"] == "int8 static":
                st["static"] = torch.full((1,), 6.0 / 127.0, device="cuda")
    return {**st, "case": case}


# ---------------------------------------------------------------------------------------------------------- plain forms
def _tiled(s):
    """bytes [rows, blocks] in tiles of 128 rows and 4 blocks, zeros behind the ends"""
    T, n = s.shape
    s = torch.nn.functional.pad(s, (0, -n % 4, 0, -T % 128))
    return s.view(-(-T // 128), 4, 32, -(-n // 4), 4).permute(0, 3, 2, 1, 4)


def _untiled(s, rows, blocks):
    return s.permute(0, 3, 2, 1, 4).reshape(s.shape[0] * 128, s.shape[1] * 4)[:rows, :blocks]


def _scale_values(b, block):
    if block == 16:
        return b.contiguous().view(torch.float8_e4m3fn).float()
    return torch.ldexp(torch.ones(b.shape, device=b.device), b.int() - 127)


def _values(q, block):
    """what a matrix in four bits stands for, in 32 bits"""
    T, half = q["codes"].shape
    e = torch.tensor(E2M1, device="cuda")
    e = torch.cat([e, -e])
    i = torch.arange(256, device="cuda")
    v = torch.stack([e[i & 15], e[i >> 4]], 1)[q["codes"].int()].view(T, 2 * half // block, block)
    v = v * _scale_values(_untiled(q["scales"], T, 2 * half // block), block)[..., None]
    return v.view(T, 2 * half) * q["step"][:, None]


def _e2m1(v):
    """the nearest code, ties to the even one, beyond 6 the largest"""
    a, c = v.abs(), torch.zeros(v.shape, dtype=torch.uint8, device=v.device)
    for k, (lo, hi) in enumerate(zip(E2M1[:-1], E2M1[1:])):
        c += (a > (lo + hi) / 2) if k % 2 == 0 else (a >= (lo + hi) / 2)
    return c | torch.signbit(v).to(torch.uint8) << 3


def _to_fp4(p, q, block):
    """rows p (32 bits) into q; returns the rows' step sizes"""
    T, D = p.shape
    p = p.view(T, D // block, block)
    most = p.abs().amax(-1)
    if block == 16:
        g = most.amax(-1, keepdim=True)
        g = g / torch.full_like(g, 2688.0)           # 6 x 448, the largest code times the largest scale
        g = (g.view(torch.int32) & -256).view(torch.float32)   # (16 bits, so that what lies between two codes has 24: ties are exact)
        g = torch.where(g > 0, g, torch.ones_like(g))
        s = (most / (6.0 * g)).clamp(min=2.0 ** -9).to(torch.float8_e4m3fn)
        step, bytes_, v = g, s.view(torch.uint8), p / (g * s.float())[..., None]
    else:
        f, e = torch.frexp(most)                     # most = f 2^e, 0.5 <= f < 1
        e = torch.where(f <= 0.75, e - 3, e - 2).clamp(-127, 127)
        e = torch.where(most > 0, e, torch.zeros_like(e))
        step, bytes_, v = torch.ones(T, 1, device="cuda"), (e + 127).to(torch.uint8), torch.ldexp(p, -e[..., None])
    c = _e2m1(v).view(T, D)
    q["codes"].copy_(c[:, 0::2] | c[:, 1::2] << 4)
    q["scales"].copy_(_tiled(bytes_))
    return step


def _plain_quantize(st):
    st["q"]["step"].copy_(_to_fp4(st["x"].float(), st["q"], st["block"])[:, 0])
    st["values"].copy_(_values(st["q"], st["block"]))
    return {"values": st["values"], "step": st["q"]["step"]}


def _plain_norm(st):
    h = st["x"]
    out = {}
    if st["residual"] is not None:
        st["stream"].copy_(st["x"].float() + st["residual"].float())
        h = out["stream"] = st["stream"]
    h = h.float()
    r = 1.0 / torch.sqrt(h.double().square().mean(-1, keepdim=True) + 1e-5)
    p = h * st["weight"]
    if "q" in st:
        step = _to_fp4(p, st["q"], st["block"])
        some = p.abs().amax(-1, keepdim=True) > 0
        st["q"]["step"].copy_(torch.where(some, step.double() * r, torch.ones_like(r))[:, 0])
        st["values"].copy_(_values(st["q"], st["block"]))
        return {**out, "values": st["values"], "step": st["q"]["step"]}
    if st["static"] is not None:
        st["xq"].copy_(torch.round(p * r.float() / st["static"]).clamp(-127, 127))
        return {**out, "xq": st["xq"]}
    a = p.abs().amax(-1, keepdim=True)
    a = a / torch.full_like(a, 127.0)
    some = a > 0
    a = torch.where(some, a, torch.ones_like(a))
    st["xq"].copy_(torch.round(p / a).clamp(-127, 127))
    st["scale"].copy_(torch.where(some, a.double() * r, torch.ones_like(r))[:, 0])
    return {**out, "xq": st["xq"], "scale": st["scale"]}


def _plain_linear(st):
    block = st["case"]["block"]
    v = torch.matmul(_values(st["x"], block), _values(st["w"], block).t())
    if st["bias"] is not None:
        v = v + st["bias"]
    if st["case"]["act"] == "silu":
        v = v / (1.0 + torch.exp(-v))
    if st["case"]["act"] == "relu2":
        v = v.clamp(min=0.0).square()
    if st["residual"] is not None:
        v = v + st["residual"].float()
    st["out"].copy_(v)
    return {"out": st["out"]}


_PLAIN = {"norm": _plain_norm, "quantize": _plain_quantize, "linear": _plain_linear}


# ---------------------------------------------------------------------------------------------------------- the framework's calls
def _own(st):
    from paper_2608_21952_b200 import binding as bd
    c, op = st["case"], st["case"]["op"]
    if "handles" not in st:   # (views of the tensors, which a user's program makes once with them)
        names = ("x", "w") if op == "linear" else ("q",) if "q" in st else ()
        st["handles"] = {k: bd.fp4_of(**st[k], block=c.get("block") or st["block"]) for k in names}
    h = st["handles"]
    if op == "linear":
        act = {"none": bd.ACT_NONE, "silu": bd.ACT_SILU, "relu2": bd.ACT_RELU2}[c["act"]]
        bd.ssdi8_fp4_linear(h["x"], h["w"], st["out"], bias=st["bias"], residual=st["residual"], act=act)
        return {"out": st["out"]}
    if op == "quantize":
        bd.ssdi8_fp4_quantize(st["x"], h["q"])
        bd.ssdi8_fp4_dequantize(h["q"], st["values"])
        return {"values": st["values"], "step": st["q"]["step"]}
    out = {"stream": st["stream"]} if st["residual"] is not None else {}
    if "q" in st:
        bd.ssdi8_add_norm_quantize(st["x"], residual=st["residual"], residual_out=st["stream"], weight=st["weight"], eps=1e-5, fp4=h["q"])
        bd.ssdi8_fp4_dequantize(h["q"], st["values"])
        return {**out, "values": st["values"], "step": st["q"]["step"]}
    bd.ssdi8_add_norm_quantize(st["x"], residual=st["residual"], residual_out=st["stream"], weight=st["weight"], eps=1e-5, xq=st["xq"],
                               scale=None if st["static"] is not None else st["scale"], static_scale=st["static"])
    return {**out, "xq": st["xq"]} if st["static"] is not None else {**out, "xq": st["xq"], "scale": st["scale"]}


def run(st):
    if own:
        return _own(st)
    return _PLAIN[st["case"]["op"]](st)


# ---------------------------------------------------------------------------------------------------------- work
def work(case):
    """Inputs read once and outputs written once (values in four bits, as what they stand for, where they are an output); two operations per
    multiply-accumulate, and what a plain reading of the formula takes elsewhere."""
    op, e = case["op"], _SIZE[case["dtype"]]
    T = case["rows"]
    if op == "linear":
        O, K = case["outs"], case["inner"]
        return {"bytes": (T + O) * (K / 2 + K / case["block"] + 4) + T * O * e * (2 if case["residual"] else 1) + (4 * O if case["bias"] else 0),
                "flops": 2.0 * T * O * K}
    D = case["width"]
    if op == "quantize":
        return {"bytes": T * D * 2 * e + 4 * T, "flops": 4.0 * T * D}
    stream = 2 * _SIZE.get(case["residual"], 0)
    return {"bytes": T * D * (e + stream + (e if case["out"][:3] == "fp4" else 1)) + 4 * D + 4 * T, "flops": 6.0 * T * D}


# ---------------------------------------------------------------------------------------------------------- 64 bits
def _exact_values(codes, scales, step, block):
    """[rows, width] in 64 bits, column by column of a byte, from the tiles' definition"""
    T, W = codes.shape[0], 2 * codes.shape[1]
    k, t = torch.arange(W // block, device="cuda"), torch.arange(T, device="cuda")[:, None]
    b = scales[t // 128, k // 4, t % 32, t % 128 // 32, k % 4].long()
    if block == 16:
        m, e = b & 7, b >> 3
        s = torch.where(e > 0, (8.0 + m.double()) * torch.exp2(e.double() - 10.0), m.double() * 2.0 ** -9)
    else:
        s = torch.exp2(b.double() - 127.0)
    out = torch.empty(T, W, dtype=torch.float64, device="cuda")
    for half in (0, 1):
        c = (codes >> 4 * half).to(torch.int64) & 15
        m, e = c & 1, c >> 1 & 3
        v = torch.where(e > 0, (2.0 + m) * torch.exp2(e.double() - 2.0), m * 0.5)
        out[:, half::2] = torch.where(c > 7, -v, v)
    return out.mul_(s.repeat_interleave(block, 1)).mul_(step.double()[:, None])


def _exact_fp4(p, block):
    """(values without a row's other factors, its step size) of rows p, in 64 bits"""
    T, D = p.shape
    top = p.abs().view(T, -1, block).max(-1).values
    if block == 16:
        most = p.abs().max(-1).values
        f, e = torch.frexp((most / torch.full_like(most, 2688.0)).float().double())
        g = torch.ldexp(torch.floor(torch.ldexp(f, e * 0 + 16)), e - 16)   # (binary32 by definition, and 16 bits of it)
        g[g == 0] = 1.0
        s = (top / (6.0 * g[:, None])).clamp(min=2.0 ** -9)
        quantum = torch.exp2(torch.floor(torch.log2(s)).clamp(min=-6.0) - 3.0)
        s = (s / quantum).round() * quantum
    else:
        g = torch.ones(T, dtype=torch.float64, device="cuda")
        k = torch.floor(torch.log2(top.clamp(min=1e-300)))
        s = torch.exp2(torch.where(top <= 1.5 * torch.exp2(k), k - 2.0, k - 1.0).clamp(-127.0, 127.0))
        s[top == 0] = 1.0
    v = p / (g[:, None] * s).repeat_interleave(block, 1)
    a = v.abs()
    quantum = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0)).to(a.dtype)
    v = torch.copysign(((a / quantum).round() * quantum).clamp(max=6.0), v)
    return v * s.repeat_interleave(block, 1), g


def exact(case, seed):
    st, op = prepare(case, seed), case["op"]
    if op == "linear":
        x, w = (_exact_values(**st[k], block=case["block"]) for k in ("x", "w"))
        v = x @ w.t()
        del x, w
        v = v if st["bias"] is None else v + st["bias"].double()
        v = torch.nn.functional.silu(v) if case["act"] == "silu" else torch.relu(v) ** 2 if case["act"] == "relu2" else v
        return {"out": v if st["residual"] is None else v + st["residual"].double()}
    if op == "quantize":
        v, g = _exact_fp4(st["x"].double(), st["block"])
        return {"values": v * g[:, None], "step": g}
    h, out = st["x"].double(), {}
    if st["residual"] is not None:
        out["stream"] = h + st["residual"].double()
        h = out["stream"].to(st["residual"].dtype).double()      # (the norm is that of the stream as it is kept)
    r = torch.rsqrt(torch.linalg.vector_norm(h, dim=-1) ** 2 / case["width"] + 1e-5)
    p = (h * st["weight"].double()).float().double()             # (in binary32 by definition)
    if "q" in st:
        v, g = _exact_fp4(p, st["block"])
        return {**out, "values": v * (g * r)[:, None], "step": g * r}
    if st["static"] is not None:
        return {**out, "xq": None}
    return {**out, "xq": None, "scale": torch.linalg.vector_norm(p, ord=math.inf, dim=-1) / 127.0 * r}
