"""The operators around the layer (ssdi8_conv_fwd, the 8-bit state cache, ssdi8_token_step, ssdi8_norm_quantize, ssdi8_linear)
against plain implementations in 64 bits, and what they refuse.

Int8 codes are compared for equality: they are defined by an exact quotient, which the reference forms in binary64 (1e-15), so a
difference would need a quotient within about 1e-13 of the middle of two integers.  Tolerances of the other outputs stand beside
their tests."""
import ctypes as C

import numpy as np
import pytest

import block_reference as ref

DTYPES = ("float32", "float16", "bfloat16")
SIZE = {"float32": 4, "float16": 2, "bfloat16": 2}
ADDR = 4096   # a well-aligned address that nothing dereferences: the call is refused first


def _lib():
    from paper_2608_21952_b200 import binding as bd
    return bd, bd._lib


def _dims(bd, batch=2, seqlen=8, nheads=4, headdim=64, dstate=64, ngroups=2):
    return bd.Dims(batch, seqlen, nheads, headdim, dstate, ngroups, 0)


def _t(a, dtype=None, device="cuda"):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).to(device)
    return t if dtype is None else t.to(getattr(torch, dtype))


def _np(t):
    """values of a tensor; bf16 as fp32 (exact)"""
    import torch
    t = t.detach()
    return (t.float() if t.dtype in (torch.bfloat16, torch.float16) else t).cpu().numpy()


# ------------------------------------------------------------------------------------------------ refusals, without a device
class ConvArgs(C.Structure):
    _fields_ = [("xBC", C.c_void_p), ("stride_b", C.c_int64), ("stride_t", C.c_int64), ("weight", C.c_void_p), ("bias", C.c_void_p),
                ("lens", C.c_void_p), ("slots", C.c_void_p), ("pos", C.c_void_p), ("ring", C.c_void_p), ("nslots", C.c_int32),
                ("s_x", C.c_void_p), ("s_B", C.c_void_p), ("s_C", C.c_void_p), ("xq", C.c_void_p), ("Bq", C.c_void_p),
                ("Cq", C.c_void_p), ("out", C.c_void_p), ("dt_raw", C.c_void_p), ("dt_stride_b", C.c_int64),
                ("dt_stride_t", C.c_int64), ("dt_bias", C.c_void_p), ("dt", C.c_void_p), ("status", C.c_void_p)]


def _conv_args(**kw):
    a = ConvArgs(xBC=ADDR, stride_b=8 * 512, stride_t=512, weight=ADDR, s_x=ADDR, s_B=ADDR, s_C=ADDR, xq=ADDR, Bq=ADDR, Cq=ADDR)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("want,dims,args,dtype,width,flags", [
    ("ERR_UNSUPPORTED", {}, {}, 3, 4, 0),
    ("ERR_UNSUPPORTED", {}, {}, 2, 4, 1 << 1),
    ("ERR_UNSUPPORTED", {}, {"out": ADDR}, 2, 4, 0),                 # codes or a tensor, not both
    ("ERR_SHAPE", {}, {}, 2, 1, 0),
    ("ERR_SHAPE", {}, {}, 2, 5, 0),
    ("ERR_SHAPE", {"headdim": 32}, {}, 2, 4, 0),
    ("ERR_SHAPE", {"nheads": 3}, {}, 2, 4, 0),
    ("ERR_SHAPE", {"batch": 0}, {}, 2, 4, 0),
    ("ERR_SHAPE", {"seqlen": -1}, {}, 2, 4, 0),
    ("ERR_SHAPE", {"nheads": 1 << 24}, {}, 2, 4, 0),
    ("ERR_SHAPE", {}, {"ring": ADDR, "nslots": 0}, 2, 4, 0),
    ("ERR_SHAPE", {}, {"ring": ADDR, "nslots": 1}, 2, 4, 0),         # slot b of two sequences
    ("ERR_NULL", {}, {"xBC": None}, 2, 4, 0),
    ("ERR_NULL", {}, {"weight": None}, 2, 4, 0),
    ("ERR_NULL", {}, {"s_B": None}, 2, 4, 0),
    ("ERR_NULL", {}, {"xq": None}, 2, 4, 0),                         # neither codes nor a tensor
    ("ERR_NULL", {}, {"dt": ADDR}, 2, 4, 0),
    ("ERR_ALIGN", {}, {"xBC": ADDR + 1}, 2, 4, 0),
    ("ERR_ALIGN", {}, {"xBC": ADDR + 2}, 0, 4, 0),
    ("ERR_ALIGN", {}, {"xq": ADDR + 4}, 2, 4, 0),
    ("ERR_ALIGN", {}, {"ring": ADDR + 8, "nslots": 2}, 2, 4, 0),
])
def test_conv_refuses(want, dims, args, dtype, width, flags):
    bd, lib = _lib()
    d = _dims(bd, **dims)
    a = _conv_args(**args)
    assert lib.ssdi8_conv_fwd(C.byref(d), C.byref(a), dtype, width, flags, None) == getattr(bd, want)


def test_conv_refuses_null_and_takes_no_tokens():
    bd, lib = _lib()
    d, a = _dims(bd), _conv_args()
    assert lib.ssdi8_conv_fwd(None, C.byref(a), 2, 4, 0, None) == bd.ERR_NULL
    assert lib.ssdi8_conv_fwd(C.byref(d), None, 2, 4, 0, None) == bd.ERR_NULL
    d, a = _dims(bd, seqlen=0), ConvArgs()
    assert lib.ssdi8_conv_fwd(C.byref(d), C.byref(a), 2, 4, 0, None) == bd.OK


# ------------------------------------------------------------------------------------------------ convolution
def _conv_case(seed, B, L, H, N, G, W, dtype, offset=0, gain=50.0):
    import torch
    rng = np.random.default_rng(seed)
    HP, Ch = 64 * H, 64 * H + 2 * G * N
    row = HP + Ch + H + offset
    rows = _t(rng.standard_normal((B, L, row)).astype(np.float32), dtype)
    x, raw = rows[..., HP + offset:HP + offset + Ch], rows[..., HP + offset + Ch:]
    w = rng.uniform(-0.5, 0.5, (Ch, W)).astype(np.float32)
    w[rng.permutation(HP)[:2]] *= gain
    bias = (0.1 * rng.standard_normal(Ch)).astype(np.float32)
    s_x = (3.0 / 127 * np.sqrt((w[:HP] ** 2).sum(1) + 0.01)).astype(np.float32)
    s_B, s_C = rng.uniform(0.01, 0.02, (2, G)).astype(np.float32)
    ring = _t(rng.standard_normal((B + 3, W, Ch)).astype(np.float32), dtype)
    return {"x": x, "raw": raw, "w": w, "bias": bias, "s_x": s_x, "s_B": s_B, "s_C": s_C, "ring": ring, "rng": rng,
            "dt_bias": (-3.0 + rng.standard_normal(H)).astype(np.float32), "dims": (B, L, H, N, G, W), "torch": torch}


def _conv_run(c, codes, bias=True, lens=None, slots=None, pos=None, ring=None, softplus=True, status=None, stream=None):
    from paper_2608_21952_b200 import binding as bd
    torch = c["torch"]
    B, L, H, N, G, W = c["dims"]
    new = lambda *s, dtype: torch.full(s, 77, dtype=dtype, device="cuda")  # noqa: E731
    o = {"dt": new(B, L, H, dtype=torch.float32)}
    if codes:
        o.update(xq=new(B, L, 64 * H, dtype=torch.int8), Bq=new(B, L, G * N, dtype=torch.int8), Cq=new(B, L, G * N, dtype=torch.int8))
    else:
        o.update(out=new(B, L, 64 * H + 2 * G * N, dtype=c["x"].dtype))
    dev = lambda a: None if a is None else _t(a)  # noqa: E731
    bd.ssdi8_conv_fwd(_dims(bd, B, L, H, 64, N, G), c["x"], _t(c["w"]), _t(c["bias"]) if bias else None, s_x=_t(c["s_x"]),
                      s_B=_t(c["s_B"]), s_C=_t(c["s_C"]), dt_raw=c["raw"], dt_bias=_t(c["dt_bias"]), lens=dev(lens), ring=ring,
                      slots=dev(slots), pos=dev(pos), status=status, flags=bd.FLAG_DT_SOFTPLUS if softplus else 0, stream=stream, **o)
    return o


def _conv_check(c, o, codes, bias=True, lens=None, slots=None, pos=None, ring=None, ring_before=None, softplus=True):
    B, L, H, N, G, W = c["dims"]
    HP, GN = 64 * H, G * N
    want_ring = None if ring is None else _np(ring_before).copy()
    u = ref.conv(_np(c["x"]), c["w"], c["bias"] if bias else None, lens, want_ring, slots, pos)
    if ring is not None:
        np.testing.assert_array_equal(_np(ring), want_ring)
    if codes:
        np.testing.assert_array_equal(_np(o["xq"]), ref.code(u[..., :HP] / c["s_x"].astype(np.float64)))
        np.testing.assert_array_equal(_np(o["Bq"]), ref.code(u[..., HP:HP + GN] / np.repeat(c["s_B"].astype(np.float64), N)))
        np.testing.assert_array_equal(_np(o["Cq"]), ref.code(u[..., HP + GN:] / np.repeat(c["s_C"].astype(np.float64), N)))
    else:
        # binary32 arithmetic: 1.1 * 4 eps of the sum of magnitudes and (10 + 1.5 |v|) eps of the value, and half a step of the type
        size = ref.conv(np.abs(_np(c["x"])), np.abs(c["w"]), None if not bias else np.abs(c["bias"]), lens,
                        None if ring is None else np.abs(_np(ring_before)), slots, pos) + 1.0   # (SiLU(m) > m - 1 for m > 0)
        half = {"torch.float32": 2.0 ** -24, "torch.float16": 2.0 ** -11, "torch.bfloat16": 2.0 ** -8}[str(c["x"].dtype)]
        tol = 2.0 ** -24 * (5 * size + 20 * np.abs(u) + 2 * np.abs(u) * size) + half * np.abs(u) + (2.0 ** -25 if half == 2.0 ** -11 else 0)
        assert np.all(np.abs(_np(o["out"]) - u) <= tol)
    raw = _np(c["raw"]).astype(np.float32)
    dt = ref.softplus((raw + c["dt_bias"]).astype(np.float64)) if softplus else raw.astype(np.float64)
    for b in range(B):
        s = b if slots is None else int(slots[b])
        dead = ring is not None and (s < 0 or s >= ring.shape[0] or (pos is not None and pos[b] < 0) or (slots is not None and s in slots[:b]))
        dt[b, 0 if dead else L if lens is None else int(np.clip(lens[b], 0, L)):] = 0
    np.testing.assert_allclose(_np(o["dt"]), dt, rtol=2.0 ** -23, atol=1e-38)   # (the binary64 value rounded once)


CONV = [  # B, L, H, N, G, W, dtype, element offset of the row (alignment)
    (1, 1, 1, 64, 1, 4, "bfloat16", 0), (1, 2, 2, 128, 1, 4, "float16", 1), (2, 3, 3, 64, 3, 3, "float32", 1),
    (2, 8, 4, 64, 2, 2, "bfloat16", 2), (1, 65, 5, 128, 1, 4, "bfloat16", 3), (3, 200, 2, 64, 1, 4, "float32", 0),
    (1, 517, 24, 128, 1, 4, "bfloat16", 0), (2, 131, 16, 128, 8, 3, "float16", 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("codes", [True, False])
@pytest.mark.parametrize("B,L,H,N,G,W,dtype,offset", CONV)
def test_conv_of_a_fresh_prompt(B, L, H, N, G, W, dtype, offset, codes):
    c = _conv_case(B + L + H, B, L, H, N, G, W, dtype, offset)
    _conv_check(c, _conv_run(c, codes), codes)
    _conv_check(c, _conv_run(c, codes, bias=False, softplus=False), codes, bias=False, softplus=False)


@pytest.mark.gpu
@pytest.mark.parametrize("codes", [True, False])
@pytest.mark.parametrize("B,L,H,N,G,W,dtype,offset", CONV)
def test_conv_goes_on_from_the_ring(B, L, H, N, G, W, dtype, offset, codes):
    """ragged lengths (none and all among them), positions from 0 on, padding and out-of-range slots, an already used one"""
    c = _conv_case(100 + B + L, B + 4, L, H, N, G, W, dtype, offset)
    n = B + 4
    slots = c["rng"].permutation(n + 3)[:n].astype(np.int32)
    slots[n - 1], slots[n - 2], slots[n - 3] = -1, n + 3, slots[0]
    pos = c["rng"].integers(0, 7, n).astype(np.int32)
    pos[1] = -5 if n > 5 else pos[1]
    lens = c["rng"].integers(0, L + 1, n).astype(np.int32)
    lens[0], lens[2 % n] = L, 0
    ring, before, status = c["ring"].clone(), c["ring"], c["torch"].zeros(1, dtype=c["torch"].int32, device="cuda")
    o = _conv_run(c, codes, lens=lens, slots=slots, pos=pos, ring=ring, status=status)
    _conv_check(c, o, codes, lens=lens, slots=slots, pos=pos, ring=ring, ring_before=before)
    assert int(status.item()) == -2


@pytest.mark.gpu
def test_conv_in_pieces_equals_the_whole():
    """a prompt of 300 tokens in one call, and in calls of 1, 2, 130, 0 and 167 tokens through the ring: the same codes"""
    torch = pytest.importorskip("torch")
    c = _conv_case(5, 1, 300, 4, 64, 2, 4, "bfloat16", 1)
    whole = _conv_run(c, True, ring=c["ring"].clone())
    ring, at, parts = c["ring"].clone(), 0, []
    for n in (1, 2, 130, 0, 167):
        piece = {**c, "x": c["x"][:, at:at + n], "raw": c["raw"][:, at:at + n], "dims": (1, n, 4, 64, 2, 4)}
        parts.append(_conv_run(piece, True, ring=ring, pos=np.array([at], np.int32)))
        at += n
    for k in ("xq", "Bq", "Cq", "dt"):
        assert torch.equal(torch.cat([p[k] for p in parts], 1), whole[k])


@pytest.mark.gpu
def test_conv_values_that_are_not_finite_and_step_sizes_at_the_ends():
    """an infinity or a NaN reaches the tokens under its taps only; step sizes far outside the normal range"""
    c = _conv_case(6, 2, 70, 2, 64, 1, 4, "float32", 0)
    c["x"][0, 9, 5], c["x"][0, 30, 6], c["x"][1, 33, 200], c["x"][1, 50, 7] = float("inf"), float("nan"), -float("inf"), 3e38
    c["s_x"][:6] = [1e-38, 1e-32, 1e31, 3e38, 0.02, 0.02]
    c["w"][3] = 0.0   # (no tap at all: the bias alone)
    with np.errstate(all="ignore"):
        _conv_check(c, _conv_run(c, True), True)


@pytest.mark.gpu
def test_conv_on_a_side_stream_and_in_a_graph():
    torch = pytest.importorskip("torch")
    from paper_2608_21952_b200 import binding as bd
    c = _conv_case(7, 2, 40, 2, 64, 1, 4, "bfloat16", 0)
    want = _conv_run(c, True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _conv_run(c, True)
    given = _conv_run(c, True, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    for k in want:
        assert torch.equal(got[k], want[k]) and torch.equal(given[k], want[k])
    # captured once, replayed on other tokens and positions: the ring goes on from replay to replay
    x, raw, ring, pos = c["x"].clone(), c["raw"].clone(), c["ring"].clone(), torch.zeros(2, dtype=torch.int32, device="cuda")
    p = {k: _t(c[k]) for k in ("w", "bias", "s_x", "s_B", "s_C", "dt_bias")}
    o = {k: torch.empty_like(v) for k, v in want.items()}
    call = lambda: bd.ssdi8_conv_fwd(_dims(bd, 2, 40, 2, 64, 64, 1), x, p["w"], p["bias"], s_x=p["s_x"], s_B=p["s_B"], s_C=p["s_C"],  # noqa: E731
                                     dt_raw=raw, dt_bias=p["dt_bias"], ring=ring, pos=pos, flags=bd.FLAG_DT_SOFTPLUS, **o)
    call()
    torch.cuda.synchronize()
    ring.copy_(c["ring"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    graph.replay()
    for k in want:
        assert torch.equal(o[k], want[k])
    pos += 40
    x.copy_(x.flip(1))
    before = ring.clone()
    graph.replay()
    again = {**c, "x": x}
    torch.cuda.synchronize()
    _conv_check(again, o, True, ring=ring, ring_before=before, pos=np.array([40, 40], np.int32))
