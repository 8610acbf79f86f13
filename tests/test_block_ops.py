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
    ("ERR_UNSUPPORTED", {}, {"xq": None, "out": ADDR}, 2, 4, 0),     # not in place: tokens ahead would be read behind their change
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
@pytest.mark.parametrize("dtype,H,L,W", [("bfloat16", 3, 150, 4), ("float32", 5, 64, 3), ("float16", 1, 9, 2)])
def test_conv_where_binary32_decides_next_to_nothing(dtype, H, L, W):
    """step sizes outside the normal range in most channels, and inputs far above the steps in others, going on from a ring"""
    c = _conv_case(8, 3, L, H, 64, 1, W, dtype, 0)
    c["s_x"][: 40 * H] = 1e-33
    c["s_x"][40 * H : 60 * H] = 1e-8
    lens, pos, slots = np.array([L, L - 1, 0], np.int32), np.array([5, 1, 2], np.int32), np.array([4, 0, 2], np.int32)
    ring = c["ring"].clone()
    _conv_check(c, _conv_run(c, True, lens=lens, slots=slots, pos=pos, ring=ring), True, lens=lens, slots=slots, pos=pos, ring=ring, ring_before=c["ring"])


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


# ------------------------------------------------------------------------------------------------ 8-bit state cache
class TokenArgs(C.Structure):
    _fields_ = [("xBC", C.c_void_p), ("stride_b", C.c_int64), ("weight", C.c_void_p), ("bias", C.c_void_p), ("dt_raw", C.c_void_p),
                ("dt_stride_b", C.c_int64)] + [(k, C.c_void_p) for k in ("dt_bias", "A", "D", "corr", "s_x", "s_B", "s_C", "slots",
                                                                         "pos", "y", "status")]


def _cache_struct(bd, **kw):
    c = bd.Cache(nslots=4, width=4, dtype=2)
    for k in ("codes", "scales", "xwin", "Bwin", "dtwin", "start", "ring"):
        setattr(c, k, ADDR)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


CACHE_REFUSALS = [
    ("ERR_SHAPE", {"headdim": 128}, {}), ("ERR_SHAPE", {"dstate": 32}, {}), ("ERR_SHAPE", {"nheads": 5}, {}), ("ERR_SHAPE", {"batch": 0}, {}),
    ("ERR_SHAPE", {}, {"nslots": 0}), ("ERR_SHAPE", {"batch": 5}, {}), ("ERR_NULL", {}, {"codes": None}), ("ERR_NULL", {}, {"scales": None}),
    ("ERR_NULL", {}, {"xwin": None}), ("ERR_NULL", {}, {"Bwin": None}), ("ERR_NULL", {}, {"dtwin": None}), ("ERR_NULL", {}, {"start": None}),
    ("ERR_ALIGN", {}, {"codes": ADDR + 8}), ("ERR_ALIGN", {}, {"xwin": ADDR + 4}),
]


@pytest.mark.parametrize("want,dims,cache", CACHE_REFUSALS)
def test_cache_refuses(want, dims, cache):
    bd, lib = _lib()
    d, c, want = _dims(bd, **dims), _cache_struct(bd, **cache), getattr(bd, want)
    a = TokenArgs(**{k: ADDR for k in ("xBC", "weight", "dt_raw", "A", "s_x", "s_B", "s_C", "pos", "y")})
    p = C.c_void_p(ADDR)
    assert lib.ssdi8_cache_write(C.byref(d), C.byref(c), None, p, p, None, None) == want
    assert lib.ssdi8_cache_read(C.byref(d), C.byref(c), None, None, p, p, p, p, p, None, None) == want
    assert lib.ssdi8_token_step(C.byref(d), C.byref(c), C.byref(a), 0, None) == want


def test_cache_refuses_what_one_entry_needs():
    bd, lib = _lib()
    d, c, p = _dims(bd), _cache_struct(bd), C.c_void_p(ADDR)
    assert lib.ssdi8_cache_write(C.byref(d), None, None, p, p, None, None) == bd.ERR_NULL
    assert lib.ssdi8_cache_write(C.byref(d), C.byref(c), None, p, C.c_void_p(ADDR + 4), None, None) == bd.ERR_ALIGN
    for k in range(4, 9):
        args = [C.byref(d), C.byref(c), None, None] + [p] * 5
        args[k] = None
        assert lib.ssdi8_cache_read(*args, None, None) == bd.ERR_NULL
    good = {k: ADDR for k in ("xBC", "weight", "dt_raw", "A", "s_x", "s_B", "s_C", "pos", "y")}
    call = lambda cc, flags=0, **kw: lib.ssdi8_token_step(C.byref(d), C.byref(cc), C.byref(TokenArgs(**{**good, **kw})), flags, None)  # noqa: E731
    for k in good:
        assert call(c, **{k: None}) == bd.ERR_NULL, k
    assert call(c, flags=bd.FLAG_Y_FP16 | bd.FLAG_Y_BF16) == bd.ERR_UNSUPPORTED
    assert call(c, flags=bd.FLAG_INT8_STATE) == bd.ERR_UNSUPPORTED
    assert call(c, y=ADDR + 2) == bd.ERR_ALIGN and call(c, xBC=ADDR + 1) == bd.ERR_ALIGN and call(c, weight=ADDR + 4) == bd.ERR_ALIGN
    assert call(_cache_struct(bd, ring=None)) == bd.ERR_NULL
    assert call(_cache_struct(bd, width=5)) == bd.ERR_SHAPE and call(_cache_struct(bd, width=1)) == bd.ERR_SHAPE
    assert call(_cache_struct(bd, dtype=3)) == bd.ERR_UNSUPPORTED


def _cache(rng, n, H, N, G, dtype="bfloat16", width=4, start=None):
    """a cache with random contents, and the same as arrays"""
    from paper_2608_21952_b200 import binding as bd
    import torch
    code = lambda *s: np.clip(np.rint(rng.standard_normal(s) * 40), -127, 127).astype(np.int8)  # noqa: E731
    a = {"codes": code(n, H, 64, N), "scales": rng.uniform(0.001, 0.05, (n, H, 64)).astype(np.float32), "xwin": code(n, H, 16, 64),
         "Bwin": code(n, G, 16, N), "dtwin": ref.softplus(rng.standard_normal((n, H, 16)) - 2).astype(np.float32),
         "start": np.zeros(n, np.int32) if start is None else np.asarray(start, np.int32)}
    ring = _t(rng.standard_normal((n, width, 64 * H + 2 * G * N)).astype(np.float32), dtype)
    c = bd.cache_of(_dims(bd, 1, 1, H, 64, N, G), ring=ring, **{k: _t(v) for k, v in a.items()})
    a["ring"] = _np(ring).copy()
    return c, a, torch


def _same(c, a, names=("codes", "scales", "xwin", "Bwin", "dtwin", "start", "ring")):
    for k in names:
        np.testing.assert_array_equal(_np(c.tensors[k]), a[k], err_msg=k)


@pytest.mark.gpu
@pytest.mark.parametrize("B,H,N,G", [(1, 1, 64, 1), (3, 5, 128, 1), (6, 4, 64, 2), (2, 24, 128, 1), (9, 16, 128, 8)])
def test_cache_write(B, H, N, G):
    from paper_2608_21952_b200 import binding as bd
    rng = np.random.default_rng(B * H)
    c, a, torch = _cache(rng, B + 3, H, N, G)
    d = _dims(bd, B, 1, H, 64, N, G)
    S = (rng.standard_normal((B, H, 64, N)) * 10.0 ** rng.uniform(-3, 3, (B, H, 64, 1))).astype(np.float32)
    S[0, 0, 0], S[0, 0, 1], S[0, 0, 2, 3], S[0, 0, 3, 5] = 0, 1e-44, np.nan, np.inf
    S[0, 0, 4] *= 1e-34
    S[0, 0, 5], S[0, 0, 6] = 0, np.nan
    S[0, 0, 5, 0] = 2.0 ** -149
    slots, pos = rng.permutation(B + 3)[:B].astype(np.int32), rng.integers(0, 99, B).astype(np.int32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    if B > 3:
        slots[-1], slots[-2], slots[-3], pos[1] = -1, slots[0], B + 3, -1
    s = ref.Slots(a, np.ones(H), np.ones(H * 64), np.ones(G))
    s.write(slots, pos, S)
    bd.ssdi8_cache_write(d, c, _t(slots), _t(pos), _t(S), status)
    _same(c, a)
    assert int(status.item()) == (-2 if B > 3 else 0)
    s.write(None, None, np.zeros_like(S))   # (no state: zeros, slot b, position 0)
    bd.ssdi8_cache_write(d, c, None, None, None)
    _same(c, a)


@pytest.mark.gpu
@pytest.mark.parametrize("B,H,N,G", [(1, 1, 64, 1), (3, 5, 128, 1), (20, 4, 64, 2), (18, 16, 128, 8)])
def test_cache_read(B, H, N, G):
    from paper_2608_21952_b200 import binding as bd
    rng = np.random.default_rng(B + H)
    n = B + 2
    pos = rng.integers(0, 64, B).astype(np.int32)
    pos[:min(B, 3)] = [48, 31, 17][:min(B, 3)]
    slots = rng.permutation(n)[:B].astype(np.int32)
    start = np.zeros(n, np.int32)
    start[slots] = np.maximum(0, pos - rng.integers(0, 12, B))
    if B > 3:
        slots[4], slots[5], pos[6] = -3, slots[0], -2
        start[slots[7]] = pos[7] + 1   # (written behind where it is read)
    c, a, torch = _cache(rng, n, H, N, G, start=start)
    A = -np.exp(rng.uniform(0, np.log(16), H)).astype(np.float32)
    A[0] = 0.05   # (a growing head)
    s_x, s_B = rng.uniform(0.01, 0.05, H * 64).astype(np.float32), rng.uniform(0.01, 0.02, G).astype(np.float32)
    s = ref.Slots(a, A, s_x, s_B)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for first in (None, np.maximum(0, pos - rng.integers(0, 17, B)).astype(np.int32)):
        if first is not None and B > 8:
            first[8], first[9] = pos[8] - 17, pos[9] + 1
        out = torch.full((B, H, 64, N), 7.0, device="cuda")
        bd.ssdi8_cache_read(_dims(bd, B, 1, H, 64, N, G), c, _t(slots), _t(pos), _t(A), _t(s_x), _t(s_B), out,
                            first=None if first is None else _t(first), status=status)
        got = _np(out)
        for b in range(B):
            ok = s.valid(slots, pos, b)
            f = 0 if not ok else max(int(start[slots[b]]), pos[b] - pos[b] % 16) if first is None else int(first[b])
            if not ok or f < 0 or not 0 <= pos[b] - f <= 16:
                assert np.all(got[b] == 7.0)
                continue
            S, size = s.state(int(slots[b]), list(range(f, pos[b])))
            # binary32: the exponential's and the factors' roundings, a product and up to 16 fused additions
            assert np.all(np.abs(got[b] - S) <= 24 * 2.0 ** -24 * size + 1e-38), b
        assert int(status.item()) == (-2 if B > 3 else 0)
    _same(c, a)   # (nothing is written)


# ------------------------------------------------------------------------------------------------ token step
def _token_params(rng, H, N, G, W):
    HP, Ch = 64 * H, 64 * H + 2 * G * N
    w = rng.uniform(-0.5, 0.5, (Ch, W)).astype(np.float32)
    w[rng.permutation(HP)[:2]] *= 50
    A = -np.exp(rng.uniform(0, np.log(16), H)).astype(np.float32)
    return {"w": w, "bias": (0.1 * rng.standard_normal(Ch)).astype(np.float32), "dt_bias": (-3 + rng.standard_normal(H)).astype(np.float32),
            "A": A, "D": rng.standard_normal(H).astype(np.float32), "corr": (0.1 * rng.standard_normal(HP)).astype(np.float32),
            "s_x": (3.0 / 127 * np.sqrt((w[:HP] ** 2).sum(1) + 0.01)).astype(np.float32),
            "s_B": rng.uniform(0.01, 0.02, G).astype(np.float32), "s_C": rng.uniform(0.01, 0.02, G).astype(np.float32)}


@pytest.mark.gpu
@pytest.mark.parametrize("B,H,N,G,W,dtype,ydt,steps", [
    (1, 1, 64, 1, 4, "bfloat16", "float32", 34), (1, 3, 128, 1, 3, "float16", "float16", 18), (5, 4, 64, 2, 2, "float32", "float32", 18),
    (3, 24, 128, 1, 4, "bfloat16", "bfloat16", 17), (150, 20, 64, 1, 4, "bfloat16", "float32", 3), (60, 60, 128, 4, 4, "float16", "float32", 2), (4, 9, 128, 3, 4, "bfloat16", "float32", 17), (2, 16, 64, 8, 4, "bfloat16", "bfloat16", 17),
])
def test_token_steps(B, H, N, G, W, dtype, ydt, steps):
    """sequences at different positions (0 among them, and one whose slot was written in the middle of a window), step after step:
    every tensor of the cache equal, y within binary32's error; a padding row and its slot stay as they are"""
    from paper_2608_21952_b200 import binding as bd
    rng = np.random.default_rng(10 * B + H)
    n = B + 3
    slots = rng.permutation(n)[:B].astype(np.int32)
    pos = rng.integers(0, 40, B).astype(np.int32)
    pos[0] = 0
    start = rng.integers(0, 1, n)
    start[slots] = np.maximum(0, pos - rng.integers(0, 9, B))
    if B > 2:
        slots[B - 1] = -1
    c, a, torch = _cache(rng, n, H, N, G, dtype, W, start)
    p = _token_params(rng, H, N, G, W)
    p["bias"] = None if W == 3 else p["bias"]
    p["corr"] = None if W == 2 else p["corr"]
    p["D"] = None if W == 2 else p["D"]
    s = ref.Slots(a, p["A"], p["s_x"], p["s_B"], p["s_C"], p["D"], p["corr"])
    dev = {k: None if v is None else _t(v) for k, v in p.items()}
    Ch, d = 64 * H + 2 * G * N, _dims(bd, B, 1, H, 64, N, G)
    y = torch.full((B, 64 * H), 5.0, device="cuda").to(getattr(torch, ydt))
    want = np.full((B, 64 * H), 5.0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    half = {"float32": 0.0, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}[ydt]
    live = slots >= 0
    for step in range(steps):
        rows = _t(rng.standard_normal((B, 3 + Ch + H)).astype(np.float32), dtype)
        x, raw = rows[:, 3:3 + Ch], rows[:, 3 + Ch:]
        u = ref.conv(_np(x)[:, None], p["w"], p["bias"], None, a["ring"].copy(), slots, pos)[:, 0]
        bd.ssdi8_token_step(d, c, x, dev["w"], dev["bias"], raw, dev["dt_bias"], dev["A"], dev["D"], dev["corr"], dev["s_x"], dev["s_B"],
                            dev["s_C"], _t(slots), _t(pos), y, status=status, flags=bd.FLAG_DT_SOFTPLUS)
        dt = ref.softplus((_np(raw) + p["dt_bias"]).astype(np.float64))
        got = np.stack([_np(c.tensors["dtwin"])[max(slots[b], 0), :, pos[b] % 16] for b in range(B)])
        np.testing.assert_allclose(got[live], dt[live], rtol=2.0 ** -23)
        bound = s.step(u, got, slots, pos, _np(x), want)
        _same(c, a)
        off = np.abs(_np(y) - want)
        assert np.all(off <= bound + half * (np.abs(want) + bound) + (2.0 ** -25 if ydt == "float16" else 0)), (step, off.max())
        pos = pos + 1
    assert int(status.item()) == 0


@pytest.mark.gpu
def test_token_step_takes_bad_rows_for_padding():
    """a slot out of range, one named twice, a negative position, a slot written behind the position: status set, the rows' y and
    slots as they were, the other rows right; without the softplus, without slots"""
    from paper_2608_21952_b200 import binding as bd
    rng = np.random.default_rng(3)
    B, H, N, G = 6, 2, 64, 1
    slots, pos = np.array([2, 7, 2, 0, 1, 3], np.int32), np.array([4, 4, 4, -1, 9, 20], np.int32)
    c, a, torch = _cache(rng, 6, H, N, G, start=[0, 10, 0, 0, 0, 0])
    p = _token_params(rng, H, N, G, 4)
    s = ref.Slots(a, p["A"], p["s_x"], p["s_B"], p["s_C"], p["D"], p["corr"])
    dev = {k: _t(v) for k, v in p.items()}
    x = _t(rng.standard_normal((B, 64 * H + 2 * N)).astype(np.float32), "bfloat16")
    raw = _t(rng.uniform(0.01, 0.1, (B, H)).astype(np.float32), "bfloat16")
    for sl in (slots, None):
        y = torch.full((B, 64 * H), 5.0, device="cuda")
        want, status = np.full((B, 64 * H), 5.0), torch.zeros(1, dtype=torch.int32, device="cuda")
        u = ref.conv(_np(x)[:, None], p["w"], p["bias"], None, a["ring"].copy(), sl, pos)[:, 0]
        bd.ssdi8_token_step(_dims(bd, B, 1, H, 64, N, G), c, x, dev["w"], dev["bias"], raw, dev["dt_bias"], dev["A"], dev["D"], dev["corr"],
                            dev["s_x"], dev["s_B"], dev["s_C"], None if sl is None else _t(sl), _t(pos), y, status=status)
        bound = s.step(u, _np(raw), sl, pos, _np(x), want)
        _same(c, a)
        assert np.all(np.abs(_np(y) - want) <= bound)
        assert int(status.item()) == -2
    assert np.all(want[3] == 5.0)


@pytest.mark.gpu
def test_token_steps_in_a_graph_equal_eager_ones():
    """one captured step, replayed 20 times with the position counted on the device, on two caches that share nothing"""
    from paper_2608_21952_b200 import binding as bd
    rng = np.random.default_rng(4)
    B, H, N, G = 3, 4, 128, 1
    c, a, torch = _cache(rng, B, H, N, G)
    other = bd.cache_of(_dims(bd, B, 1, H, 64, N, G), **{k: t.clone() for k, t in c.tensors.items()})
    dev = {k: _t(v) for k, v in _token_params(rng, H, N, G, 4).items()}
    tokens = _t(rng.standard_normal((20, B, 64 * H + 2 * N)).astype(np.float32), "bfloat16")
    raws = _t(rng.standard_normal((20, B, H)).astype(np.float32), "bfloat16")
    x, raw, pos, y = tokens[0].clone(), raws[0].clone(), torch.tensor([0, 5, 11], dtype=torch.int32, device="cuda"), torch.empty(B, 64 * H, device="cuda")

    def step(cache, out):
        bd.ssdi8_token_step(_dims(bd, B, 1, H, 64, N, G), cache, x, dev["w"], dev["bias"], raw, dev["dt_bias"], dev["A"], dev["D"], dev["corr"],
                            dev["s_x"], dev["s_B"], dev["s_C"], None, pos, out, flags=bd.FLAG_DT_SOFTPLUS)
    y2 = torch.empty_like(y)
    keep = {k: t.clone() for k, t in c.tensors.items()}
    step(c, y)   # (first use outside the capture)
    for k, t in keep.items():
        c.tensors[k].copy_(t)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(c, y)
        pos += 1
    pos.copy_(torch.tensor([0, 5, 11]))
    for i in range(20):
        x.copy_(tokens[i])
        raw.copy_(raws[i])
        step(other, y2)   # (before the replay counts the position on)
        graph.replay()
        assert torch.equal(y, y2), i
        for k in c.tensors:
            assert torch.equal(c.tensors[k], other.tensors[k]), (i, k)


# ------------------------------------------------------------------------------------------------ norm
class NormArgs(C.Structure):
    _fields_ = [("x", C.c_void_p), ("stride_x", C.c_int64), ("z", C.c_void_p), ("stride_z", C.c_int64), ("weight", C.c_void_p),
                ("xq", C.c_void_p), ("scale", C.c_void_p), ("static_scale", C.c_void_p), ("rows", C.c_int64), ("width", C.c_int32),
                ("groups", C.c_int32), ("eps", C.c_float)]


@pytest.mark.parametrize("want,args,dtype,zdtype", [
    ("ERR_UNSUPPORTED", {}, 3, 0), ("ERR_UNSUPPORTED", {"z": ADDR}, 0, 3), ("ERR_UNSUPPORTED", {}, -1, 0),
    ("ERR_SHAPE", {"rows": -1}, 0, 0), ("ERR_SHAPE", {"rows": 1 << 31}, 0, 0), ("ERR_SHAPE", {"width": 0}, 0, 0), ("ERR_SHAPE", {"width": 72}, 0, 0),
    ("ERR_SHAPE", {"width": 16400}, 0, 0), ("ERR_SHAPE", {"groups": 0}, 0, 0), ("ERR_SHAPE", {"groups": 3}, 0, 0),
    ("ERR_SHAPE", {"width": 128, "groups": 2}, 0, 0), ("ERR_SHAPE", {"eps": -1.0}, 0, 0), ("ERR_SHAPE", {"eps": float("nan")}, 0, 0),
    ("ERR_NULL", {"x": None}, 0, 0), ("ERR_NULL", {"xq": None}, 0, 0), ("ERR_ALIGN", {"xq": ADDR + 4}, 0, 0),
    ("ERR_ALIGN", {"weight": ADDR + 4}, 0, 0), ("ERR_ALIGN", {"x": ADDR + 2}, 0, 0), ("ERR_ALIGN", {"z": ADDR + 1}, 0, 1), ("OK", {"rows": 0, "x": None}, 0, 0),
])
def test_norm_refuses(want, args, dtype, zdtype):
    bd, lib = _lib()
    a = NormArgs(**{**dict(x=ADDR, stride_x=512, xq=ADDR, scale=ADDR, rows=4, width=512, groups=1, eps=1e-5), **args})
    assert lib.ssdi8_norm_quantize(C.byref(a), dtype, zdtype, None) == getattr(bd, want)
    assert lib.ssdi8_norm_quantize(None, 0, 0, None) == bd.ERR_NULL


def _norm_check(x, z, weight, groups, eps, static=None, scale=True):
    from paper_2608_21952_b200 import binding as bd
    import torch
    T, D = x.shape
    xq = torch.full((T, D), 99, dtype=torch.int8, device="cuda")
    sc = torch.full((T,), 7.0, device="cuda") if scale else None
    bd.ssdi8_norm_quantize(x, xq, weight=None if weight is None else _t(weight), z=z, groups=groups, eps=eps, scale=sc,
                           static_scale=None if static is None else _t(np.array([static], np.float32)))
    want, step = ref.norm_codes(_np(x), None if z is None else _np(z), weight, groups, eps, None if static is None else np.float32(static))
    np.testing.assert_array_equal(_np(xq), want)
    if scale and static is None:
        # binary32: 12 eps of u w, 24 of the norm, and the quotient
        np.testing.assert_allclose(_np(sc), step, rtol=40 * 2.0 ** -24, atol=1e-38)


NORM = [  # T, D, groups, dtype, gate, offset
    (1, 16, 1, "float32", None, 0), (3, 48, 1, "bfloat16", "bfloat16", 1), (5, 144, 1, "float16", "float32", 0), (130, 768, 1, "bfloat16", None, 2),
    (7, 1536, 2, "float32", "bfloat16", 0), (300, 2560, 1, "float32", "float16", 4), (33, 5120, 1, "bfloat16", "bfloat16", 3),
    (9, 8192, 8, "bfloat16", "bfloat16", 0), (2, 16384, 1, "float16", "float16", 0), (2, 16384, 4, "float32", None, 1), (40, 5120, 1, "float32", "bfloat16", 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("T,D,groups,dtype,gate,offset", NORM)
def test_norm(T, D, groups, dtype, gate, offset):
    rng = np.random.default_rng(T + D)
    x = rng.standard_normal((T, D + 2 * offset)).astype(np.float32)
    x[:, rng.permutation(D)[:max(1, D // 100)]] *= 20
    x = _t(x, dtype)[:, offset:offset + D]
    z = None if gate is None else _t((2 * rng.standard_normal((T, D + 7))).astype(np.float32), gate)[:, offset:offset + D]
    weight = rng.uniform(0.5, 1.5, D).astype(np.float32)
    _norm_check(x, z, weight, groups, 1e-5)
    _norm_check(x, z, weight, groups, 1e-5, static=0.04, scale=False)
    if gate:
        _norm_check(x, z, None if groups == 1 else weight, groups, 0.1)


@pytest.mark.gpu
@pytest.mark.parametrize("T,D,groups,dtype,gate,offset", [
    (1024, 2064, 1, "bfloat16", None, 0), (1025, 512, 1, "float32", "bfloat16", 0), (1025, 528, 1, "bfloat16", "float16", 1),
    (1030, 1024, 8, "float16", "bfloat16", 0), (1030, 2560, 2, "float32", None, 0), (1030, 4096, 1, "bfloat16", "float32", 0),
    (1030, 5136, 1, "bfloat16", "bfloat16", 0), (1030, 8192, 4, "bfloat16", None, 2),
])
def test_norm_of_many_rows(T, D, groups, dtype, gate, offset):
    """the widths and row counts at which a warp's share changes; rows of zeros, of one value and out of binary32's range among them"""
    test_norm(T, D, groups, dtype, gate, offset)
    rng = np.random.default_rng(D)
    x = rng.standard_normal((T, D)).astype(np.float32)
    x[5], x[T - 1], x[T - 2, 1:], x[17] = 0, 1, 0, x[17] * (1e-25 if dtype != "float16" else 1e-4)
    _norm_check(_t(x, dtype), None, None, groups, 1e-5)


@pytest.mark.gpu
@pytest.mark.parametrize("groups", [1, 2])
@pytest.mark.parametrize("gate", [None, "float32"])
def test_norm_of_extreme_rows(groups, gate):
    """rows of zeros, of one value, beyond binary32's squares on either side, with infinities and NaN, with gates that close"""
    rng = np.random.default_rng(8)
    D = 512
    x, z = rng.standard_normal((14, D)).astype(np.float32), rng.standard_normal((14, D)).astype(np.float32)
    weight = rng.uniform(0.5, 1.5, D).astype(np.float32)
    x[0], x[1, 1:], x[2], x[3] = 0, 0, x[2] * 1e25, x[3] * 1e-30
    x[4, 7], x[5, 9], x[6] = np.nan, np.inf, np.nan
    z[7], z[8, ::2], z[9, 3] = -95, -200, np.inf
    x[10, :256], x[11, 256:], x[12, 5] = 0, 1e-42, -np.inf
    z[13] = -60
    x[13] *= 1e3
    t = _t(x)
    zt = None if gate is None else _t(z)
    _norm_check(t, zt, weight, groups, 1e-5)
    _norm_check(t, zt, weight, groups, 1e-5, static=0.03)
    _norm_check(t[:1], None if zt is None else zt[:1], weight, groups, 0.0 if groups == 3 else 1e-12)


@pytest.mark.gpu
def test_norm_ties_go_to_the_even_code():
    """bf16 rows without gate or weight whose absmax is 127: every x of the form k + 1/2 is a tie of 127 x / absmax"""
    torch = pytest.importorskip("torch")
    x = np.zeros((2, 256), np.float32)
    x[:, :127] = np.arange(127) + 0.5
    x[:, 127], x[1] = 127, -x[1]
    x[1, 200] = -127
    _norm_check(torch.from_numpy(x).cuda(), None, None, 1, 1e-5)


@pytest.mark.gpu
@pytest.mark.parametrize("gate", [None, "float32"])
def test_norm_ties_in_the_group_of_the_absmax(gate):
    """rows of several groups: quotients of k + 1/2 in the group of the absmax, where the norm cancels, and beside groups of other norms"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    rng = np.random.default_rng(12)
    x = 0.01 * rng.standard_normal((254, 4, 128)).astype(np.float32)
    at, f = rng.integers(0, 4, 254), rng.uniform(0.5, 2, 254).astype(np.float32)
    k = rng.integers(-20, 20, (254, 127)).astype(np.float32)   # (the absmax is six times the root mean square and more; the others' is four)
    f = np.float32(2.0) ** -12 * np.round(f * 4096)   # (13 bits: products with k + 1/2 are exact)
    for t in range(254):
        x[t, at[t], 1:] = (k[t] + 0.5) * f[t]
        x[t, at[t], 0] = (-127.0 if t % 2 else 127.0) * f[t]
    z = None if gate is None else _t(np.full((254, 512), 40, np.float32))   # (SiLU(40) = 40 to 17 digits)
    rms = np.sqrt((x.astype(np.float64) ** 2).mean(-1))
    assert np.array_equal((np.abs(x).max(-1) / rms).argmax(-1), at)
    xq = torch.empty(254, 512, dtype=torch.int8, device="cuda")
    bd.ssdi8_norm_quantize(_t(x.reshape(254, 512)), xq, z=z, groups=4, eps=1e-5)
    got = _np(xq).reshape(254, 4, 128)
    for t in range(254):
        np.testing.assert_array_equal(got[t, at[t], 1:], np.rint(k[t] + 0.5))
        assert got[t, at[t], 0] == (-127 if t % 2 else 127)


# ------------------------------------------------------------------------------------------------ int8 projection
class LinearArgs(C.Structure):
    _fields_ = [("xq", C.c_void_p), ("wq", C.c_void_p), ("s_row", C.c_void_p), ("s_w", C.c_void_p), ("bias", C.c_void_p),
                ("residual", C.c_void_p), ("stride_residual", C.c_int64), ("out", C.c_void_p), ("stride_out", C.c_int64),
                ("rows", C.c_int32), ("outs", C.c_int32), ("inner", C.c_int32), ("act", C.c_int32), ("status", C.c_void_p)]


@pytest.mark.parametrize("want,args,dtype", [
    ("ERR_UNSUPPORTED", {}, 3), ("ERR_UNSUPPORTED", {"act": 3}, 0), ("ERR_UNSUPPORTED", {"act": -1}, 0), ("ERR_SHAPE", {"rows": -1}, 0),
    ("ERR_SHAPE", {"outs": 0}, 0), ("ERR_SHAPE", {"stride_out": 63}, 0), ("ERR_SHAPE", {"inner": 0}, 0), ("ERR_SHAPE", {"inner": 24}, 0), ("ERR_SHAPE", {"inner": 131088}, 0),
    ("ERR_NULL", {"xq": None}, 0), ("ERR_NULL", {"wq": None}, 0), ("ERR_NULL", {"s_w": None}, 0), ("ERR_NULL", {"out": None}, 0),
    ("ERR_ALIGN", {"xq": ADDR + 8}, 0), ("ERR_ALIGN", {"wq": ADDR + 1}, 0), ("ERR_ALIGN", {"out": ADDR + 2}, 0), ("ERR_ALIGN", {"residual": ADDR + 1}, 1),
    ("OK", {"rows": 0, "out": None}, 0),
])
def test_linear_refuses(want, args, dtype):
    bd, lib = _lib()
    a = LinearArgs(**{**dict(xq=ADDR, wq=ADDR, s_w=ADDR, out=ADDR, stride_out=64, rows=4, outs=64, inner=64), **args})
    assert lib.ssdi8_linear(C.byref(a), dtype, None) == getattr(bd, want)
    assert lib.ssdi8_linear(None, 0, None) == bd.ERR_NULL


def _linear_check(seed, T, O, K, dtype, act="none", bias=True, residual="own", s_row=True, pad=0, offset=0, extremes=False):
    from paper_2608_21952_b200 import binding as bd
    import torch
    rng = np.random.default_rng(seed)
    code = lambda *s: np.clip(np.rint(rng.standard_normal(s) * 40), -127, 127).astype(np.int8)  # noqa: E731
    x, w = code(T, K), code(O, K)
    if extremes:   # (the largest sums there are, of both signs)
        x[0], w[0], w[-1] = 127, 127, -127
    sr = rng.uniform(0.01, 0.05, T).astype(np.float32) if s_row else None
    sw = (rng.uniform(0.5, 1.5, O) / (40 * np.sqrt(K))).astype(np.float32)
    b = rng.standard_normal(O).astype(np.float32) if bias else None
    whole = torch.full((T, O + pad + offset), 3.0, device="cuda").to(getattr(torch, dtype))
    out = whole[:, offset:offset + O]
    res = None
    if residual == "own":
        res = _t(rng.standard_normal((T, O + 5)).astype(np.float32), dtype)[:, 2:2 + O]
    if residual == "out":
        out.copy_(_t(rng.standard_normal((T, O)).astype(np.float32), dtype))
        res = out
    before = None if res is None else _np(res).astype(np.float64).copy()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    bd.ssdi8_linear(_t(x), _t(w), _t(sw), out, s_row=None if sr is None else _t(sr), bias=None if b is None else _t(b), residual=res,
                    act={"none": bd.ACT_NONE, "silu": bd.ACT_SILU, "relu2": bd.ACT_RELU2}[act], status=status)
    acc = x.astype(np.float64) @ w.astype(np.float64).T   # (whole numbers below 2^53: exact)
    eps = 2.0 ** -24
    part = acc * (1.0 if sr is None else sr.astype(np.float64)[:, None]) * sw
    v = part + (0 if b is None else b.astype(np.float64))
    err = eps * (3 * np.abs(part) + np.abs(v) + 2 * 2 * eps)   # the sum as a float, the two products, the fused addition
    if act == "silu":
        u = ref.silu(v)
        err = 1.1 * err + eps * (10 + 1.5 * np.abs(v)) * np.abs(u)
    elif act == "relu2":
        u = np.maximum(v, 0) ** 2
        err = 2 * np.abs(v) * err + err * err + 2 * eps * u
    else:
        u = v
    if before is not None:
        u = u + before
        err = err + eps * np.abs(u)
    half = {"float32": 0.0, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}[dtype]
    got = _np(out)
    assert np.all(np.abs(got - u) <= err * 1.001 + half * (np.abs(u) + err) + (2.0 ** -25 if dtype == "float16" else 0)), np.abs(got - u).max()
    edge = _np(whole)
    assert np.all(edge[:, :offset] == 3.0) and np.all(edge[:, offset + O:] == 3.0)
    assert int(status.item()) == 0


LINEAR = [  # T, O, K, dtype, act, bias, residual, s_row, pad, offset
    (1, 1, 16, "float32", "none", False, None, False, 0, 0), (1, 8, 48, "bfloat16", "none", True, "own", True, 0, 0),
    (7, 100, 128, "float16", "silu", True, None, True, 4, 0), (64, 3352, 768, "bfloat16", "none", False, None, True, 0, 0),
    (129, 129, 640, "float32", "relu2", True, "own", True, 3, 1), (128, 256, 4096, "bfloat16", "none", True, "out", True, 0, 0),
    (300, 300, 144, "bfloat16", "silu", False, "out", False, 4, 4), (513, 2560, 272, "bfloat16", "none", True, "own", True, 0, 0),
    (2000, 1999, 96, "float16", "relu2", True, None, True, 1, 0), (257, 7000, 64, "float32", "none", True, "own", True, 8, 8),
    (2, 24, 8192, "float32", "none", True, None, True, 0, 0), (33, 515, 1040, "bfloat16", "none", True, "own", True, 0, 0),
    (200, 10576, 256, "bfloat16", "none", False, None, True, 0, 0),
    # few rows: K shared out among 2, 4 and 8 CTAs, parts of unequal length
    (17, 2000, 1296, "bfloat16", "silu", True, "own", True, 0, 0), (127, 1000, 2688, "float16", "none", True, "out", True, 1, 0),
    (128, 130, 5152, "float32", "relu2", True, None, True, 0, 0), (65, 2560, 5120, "bfloat16", "none", True, "own", True, 0, 0),
    # tiles of pairs of SMs: many tiles, ragged rows and columns, K of less than a block and of an odd number of blocks
    (4099, 1300, 16, "bfloat16", "none", True, "own", True, 0, 0), (3000, 2570, 656, "float16", "silu", True, "out", True, 6, 0),
    (5200, 2560, 1100 // 16 * 16, "bfloat16", "none", True, "own", True, 0, 0), (9000, 530, 2048, "float32", "relu2", False, None, False, 2, 2),
]


@pytest.mark.gpu
@pytest.mark.parametrize("T,O,K,dtype,act,bias,residual,s_row,pad,offset", LINEAR)
def test_linear(T, O, K, dtype, act, bias, residual, s_row, pad, offset):
    _linear_check(T + O + K, T, O, K, dtype, act, bias, residual, s_row, pad, offset)


@pytest.mark.gpu
def test_linear_of_the_longest_rows():
    """sums of 131072 products at the ends of the codes: 2.1e9 of either sign, in 32 bits"""
    _linear_check(1, 5, 40, 131072, "float32", residual=None, extremes=True)


@pytest.mark.gpu
def test_linear_on_two_streams_and_in_a_graph():
    torch = pytest.importorskip("torch")
    from paper_2608_21952_b200 import binding as bd
    rng = np.random.default_rng(2)
    x, w = (_t(rng.integers(-127, 128, s).astype(np.int8)) for s in ((150, 320), (700, 320)))
    sw = _t(rng.uniform(0.5, 1.5, 700).astype(np.float32))
    want, a, b, c = (torch.empty(150, 700, device="cuda") for _ in range(4))
    bd.ssdi8_linear(x, w, sw, want)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        bd.ssdi8_linear(x, w, sw, a, stream=s1)
        bd.ssdi8_linear(x, w, sw, b, stream=s2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bd.ssdi8_linear(x, w, sw, c)
        bd.ssdi8_linear(x, w, sw, c, residual=c)
    graph.replay()
    assert torch.equal(a, want) and torch.equal(b, want) and torch.equal(c, 2 * want)


# ------------------------------------------------------------------------------------------------ the binding's own checks
@pytest.mark.gpu
def test_binding_refuses_what_tensors_tell():
    """shapes are SSDi8Error(ERR_SHAPE), element types TypeError, host or strided tensors AssertionError, another device ValueError"""
    torch = pytest.importorskip("torch")
    from paper_2608_21952_b200 import binding as bd
    e = lambda *s, dtype=torch.int8, device="cuda": torch.empty(*s, dtype=dtype, device=device)  # noqa: E731
    x, w, sw, out = e(4, 64), e(32, 64), e(32, dtype=torch.float32), e(4, 32, dtype=torch.float32)
    for bad in (dict(wq=e(32, 48)), dict(s_w=e(31, dtype=torch.float32)), dict(out=e(5, 32, dtype=torch.float32)), dict(xq=e(4, 64, 1))):
        with pytest.raises(bd.SSDi8Error) as err:
            bd.ssdi8_linear(**{**dict(xq=x, wq=w, s_w=sw, out=out), **bad})
        assert err.value.code == bd.ERR_SHAPE
    for bad in (dict(xq=e(4, 64, dtype=torch.float32)), dict(out=e(4, 32)), dict(residual=e(4, 32, dtype=torch.bfloat16)), dict(s_w=None)):
        with pytest.raises(TypeError):
            bd.ssdi8_linear(**{**dict(xq=x, wq=w, s_w=sw, out=out), **bad})
    for bad in (dict(xq=e(4, 64, device="cpu")), dict(wq=e(64, 32).t()), dict(out=e(32, 4, dtype=torch.float32).t())):
        with pytest.raises(AssertionError):
            bd.ssdi8_linear(**{**dict(xq=x, wq=w, s_w=sw, out=out), **bad})
    dims = bd.Dims(1, 1, 2, 64, 64, 1, 0)
    cache = bd.make_cache(dims, 2)
    cache.device = 7
    with pytest.raises(ValueError):
        bd.ssdi8_cache_write(dims, cache, None, None, None)
    good = {k: t for k, t in cache.tensors.items()}
    for bad, kind in ((dict(codes=good["codes"][:1].contiguous()), bd.SSDi8Error), (dict(start=good["start"].float()), TypeError),
                      (dict(ring=good["ring"].to(torch.int16)), TypeError), (dict(xwin=good["xwin"].cpu()), ValueError)):
        with pytest.raises(kind):
            bd.cache_of(dims, **{**good, **bad})


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """a slot and a row whose elements lie more than 2^31 into their tensors"""
    torch = pytest.importorskip("torch")
    from paper_2608_21952_b200 import binding as bd
    H, N, n = 128, 128, 2100   # codes: 2100 x 1 MB
    dims = bd.Dims(2, 1, H, 64, N, 1, 0)
    cache = bd.make_cache(dims, n)
    assert cache.tensors["codes"].numel() > 2 ** 31
    slots, pos = torch.tensor([n - 1, 3], dtype=torch.int32, device="cuda"), torch.tensor([15, 15], dtype=torch.int32, device="cuda")
    S = torch.randn(1, H, 64, N, device="cuda").expand(2, -1, -1, -1).contiguous()
    bd.ssdi8_cache_write(dims, cache, slots, pos, S)
    rng = np.random.default_rng(1)
    p = {k: _t(v) for k, v in _token_params(rng, H, N, 1, 4).items()}
    x = _t(rng.standard_normal((1, 64 * H + 2 * N)).astype(np.float32), "bfloat16").expand(2, -1)
    raw, y = _t(rng.standard_normal((1, H)).astype(np.float32), "bfloat16").expand(2, -1), torch.empty(2, 64 * H, device="cuda")
    cache.tensors["ring"][n - 1].copy_(cache.tensors["ring"][3].normal_())
    bd.ssdi8_token_step(dims, cache, x, p["w"], p["bias"], raw, p["dt_bias"], p["A"], p["D"], p["corr"], p["s_x"], p["s_B"], p["s_C"], slots, pos, y,
                        flags=bd.FLAG_DT_SOFTPLUS)
    assert torch.equal(y[0], y[1]) and y.isfinite().all()
    for k in ("codes", "scales", "xwin", "Bwin", "dtwin", "ring"):   # (folded, too)
        assert torch.equal(cache.tensors[k][n - 1], cache.tensors[k][3]), k
    out = torch.empty(2, H, 64, N, device="cuda")
    bd.ssdi8_cache_read(dims, cache, slots, pos + 1, p["A"], p["s_x"], p["s_B"], out)
    assert torch.equal(out[0], out[1]) and (out[0] - cache.tensors["scales"][3][..., None] * cache.tensors["codes"][3]).abs().max() == 0
    del cache, out, S
    # rows of the projection and the norm: 2^31 elements apart and more
    T, O = 70000, 32768
    wide = torch.empty(T, O, dtype=torch.bfloat16, device="cuda")
    xq, wq, sw = torch.randint(-127, 128, (T, 64), dtype=torch.int8, device="cuda"), torch.randint(-127, 128, (O, 64), dtype=torch.int8, device="cuda"), torch.rand(O, device="cuda")
    xq[-300:] = xq[:300]
    bd.ssdi8_linear(xq, wq, sw, wide)
    assert torch.equal(wide[-300:], wide[:300])
    codes, sc = torch.empty(T, 16384, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    bd.ssdi8_norm_quantize(wide[:, 16384:], codes, z=wide[:, :16384], scale=sc)
    assert torch.equal(codes[-300:], codes[:300]) and torch.equal(sc[-300:], sc[:300])
