"""Matrices in four bits (quantiser, values, product) and the norm with the residual's addition, against plain implementations in 64 bits.
Codes, scales, values and the residual stream are compared for equality; tolerances elsewhere count roundings of 2^-24 (binary32)."""
import ctypes as C
import math

import numpy as np
import pytest

import fp4_reference as ref

EPS = 2.0 ** -24
HALF = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float32": 1e-37, "float16": 2.0 ** -24, "bfloat16": 1e-37}


def _np(t):
    import torch
    return (t.float() if t.dtype in (torch.bfloat16, torch.float16) else t).detach().cpu().numpy()


def _dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(getattr(torch, dtype))


def _rows(a, dtype, extra=0, offset=0):
    """`a` on the device as rows of a wider tensor: `extra` columns more, the first one at `offset`"""
    import torch
    T, D = a.shape
    if not extra:
        return _dev(a, dtype)
    w = torch.full((T, D + extra), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    w[:, offset:offset + D] = _dev(a, dtype)
    return w[:, offset:offset + D]


def _inputs(kind, T, D, seed, dtype):
    r = np.random.default_rng(seed)
    x = r.standard_normal((T, D)).astype(np.float32)
    if kind == "outliers":
        x *= np.where(r.random(D) < 0.02, 50, 1).astype(np.float32)
    elif kind == "grid":        # few bits, so that quotients lie on middles of codes and scales
        x = (r.integers(-12, 13, (T, D)) * 2.0 ** r.integers(-3, 4, (T, 1))).astype(np.float32)
    elif kind == "zeros":
        x[::2] = 0
        x[1::2, : D // 2] = 0
        x[1::2, -1] = -0.0
    elif kind == "bad":         # NaN and infinities in some rows, ends of the range in others
        x[0, :3] = np.nan
        x[0, 3] = -np.nan
        if T > 1:
            x[1, 5], x[1, D - 1] = np.inf, -np.inf
        if T > 2:
            x[2] *= 3e4
        if T > 3 and dtype != "float16":
            x[3] *= 1e37
        if T > 4 and dtype != "float16":
            x[4] *= 1e-27
    return ref.round_to(x, dtype)


def _check_fp4(q, codes, scales, step, block):
    import torch
    T = codes.shape[0]
    torch.cuda.synchronize()
    np.testing.assert_array_equal(ref.unpack(_np(q.tensors["codes"])), codes)
    np.testing.assert_array_equal(ref.untile(_np(q.tensors["scales"]), T, scales.shape[1]), scales)
    if step is not None:
        np.testing.assert_array_equal(_np(q.tensors["step"]), step)
    # bytes behind a row's last block are 0, rows behind the last one as they were
    whole = _np(q.tensors["scales"])
    n = 4 * whole.shape[1]
    if n > scales.shape[1]:
        assert not ref.untile(whole, T, n)[:, scales.shape[1]:].any()
    if T % 128:
        assert (ref.untile(whole, 128 * whole.shape[0], n)[T:] == 99).all()


def _marked(T, D, block):
    from paper_2608_21952_b200 import binding as bd
    q = bd.make_fp4(T, D, block)
    q.tensors["scales"].fill_(99)
    q.tensors["codes"].fill_(99)
    return q


# ---------------------------------------------------------------------------------------------------------- the reference itself
def test_reference_grids():
    import torch
    b = torch.arange(127, dtype=torch.uint8)
    np.testing.assert_array_equal(b.view(torch.float8_e4m3fn).float().numpy(), ref.E4M3)
    v = np.array([[0.25, 0.2500001, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 5.1, 9, 0.2499999, 0.7499999, 2.4999, 3.4999, 4.9999, 0]])
    assert ref.nearest(v, np.ones((1, 1)), ref.E2M1).tolist() == [[0, 1, 2, 2, 4, 4, 6, 6, 7, 7, 0, 1, 4, 5, 6, 0]]
    e = np.random.default_rng(0).uniform(0, 500, 4096)
    want = torch.from_numpy(np.minimum(e, 448)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(ref.nearest(e, np.ones(1), ref.E4M3), want)
    s = np.random.default_rng(1).integers(0, 255, (300, 18)).astype(np.uint8)
    np.testing.assert_array_equal(ref.untile(ref.tile(s), 300, 18), s)


@pytest.mark.parametrize("block", [16, 32])
def test_reference_quantiser_is_near(block):
    """a value is off by half of a code's distance at most: a sixth of the block's largest, and the scale's rounding (2^-4, or 2) on top"""
    p = np.random.default_rng(2).standard_normal((64, 256)).astype(np.float32)
    c, s, g = ref.quantize(p, block)
    v = ref.values(c, s, block) * g[:, None]
    top = np.abs(p).reshape(64, -1, block).max(-1)
    assert np.all(np.abs(v - p) <= np.repeat(top, block, 1) * (1.0 / 6 * (1 + 2.0 ** -4) if block == 16 else 1.0 / 3))


# ---------------------------------------------------------------------------------------------------------- refusals (no device)
def _q(bd, rows=4, width=64, block=16, codes=4096, scales=4096, step=4096):
    return bd.Fp4(rows=rows, width=width, block=block, codes=codes, scales=scales, step=step)


def test_scales_bytes():
    from paper_2608_21952_b200 import binding as bd
    assert bd.ssdi8_fp4_scales_bytes(1, 32, 16) == 512
    assert bd.ssdi8_fp4_scales_bytes(129, 2560, 16) == 2 * 40 * 512
    assert bd.ssdi8_fp4_scales_bytes(128, 1248, 32) == 10 * 512
    assert bd.ssdi8_fp4_scales_bytes(0, 64, 16) == 0
    for bad in ((4, 48, 16), (4, 0, 16), (4, 64, 8), (-1, 64, 16), (4, 131104, 16)):
        assert bd.ssdi8_fp4_scales_bytes(*bad) == 0


def test_refusals_of_the_library():
    from paper_2608_21952_b200 import binding as bd
    L = bd._lib
    for f, at in ((L.ssdi8_fp4_quantize, [C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]),
                  (L.ssdi8_fp4_dequantize, [C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p])):
        f.restype, f.argtypes = C.c_int32, at

    def quantize(q, x=4096, dtype=0):
        return L.ssdi8_fp4_quantize(x, 64, dtype, C.addressof(q) if q else None, None, None)

    def values(q, out=4096, stride=64, dtype=0):
        return L.ssdi8_fp4_dequantize(C.addressof(q) if q else None, out, stride, dtype, None)

    assert quantize(None) == bd.ERR_NULL and values(None) == bd.ERR_NULL
    for bad in (dict(width=48), dict(width=0), dict(block=8), dict(block=64), dict(rows=-1), dict(width=131104), dict(rows=0x7fffffff),
                dict(rows=0x7fffff00, width=131072)):
        assert quantize(_q(bd, **bad)) == bd.ERR_SHAPE, bad
        assert values(_q(bd, **bad), stride=1 << 20) == bd.ERR_SHAPE, bad
    assert quantize(_q(bd), dtype=3) == bd.ERR_UNSUPPORTED and values(_q(bd), dtype=-1) == bd.ERR_UNSUPPORTED
    assert quantize(_q(bd, step=0)) == bd.ERR_NULL and quantize(_q(bd, codes=0)) == bd.ERR_NULL and quantize(_q(bd), x=0) == bd.ERR_NULL
    assert quantize(_q(bd, codes=4097)) == bd.ERR_ALIGN and quantize(_q(bd, scales=4104)) == bd.ERR_ALIGN and quantize(_q(bd), x=4098) == bd.ERR_ALIGN
    assert values(_q(bd), stride=63) == bd.ERR_SHAPE and values(_q(bd), out=0) == bd.ERR_NULL and values(_q(bd), out=4097, dtype=1) == bd.ERR_ALIGN
    assert quantize(_q(bd, rows=0)) == bd.OK and values(_q(bd, rows=0)) == bd.OK


class _Norm(C.Structure):
    _fields_ = [("x", C.c_void_p), ("stride_x", C.c_int64), ("residual", C.c_void_p), ("stride_residual", C.c_int64), ("residual_out", C.c_void_p),
                ("stride_out", C.c_int64), ("weight", C.c_void_p), ("xq", C.c_void_p), ("scale", C.c_void_p), ("static_scale", C.c_void_p),
                ("fp4", C.c_void_p), ("rows", C.c_int64), ("width", C.c_int32), ("eps", C.c_float), ("status", C.c_void_p)]


class _Linear(C.Structure):
    _fields_ = [("x", C.c_void_p), ("w", C.c_void_p), ("bias", C.c_void_p), ("residual", C.c_void_p), ("stride_residual", C.c_int64),
                ("out", C.c_void_p), ("stride_out", C.c_int64), ("act", C.c_int32), ("status", C.c_void_p)]


def test_refusals_of_the_norm_and_the_product():
    from paper_2608_21952_b200 import binding as bd
    L = bd._lib
    L.ssdi8_add_norm_quantize.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p]
    L.ssdi8_fp4_linear.argtypes = [C.c_void_p, C.c_int32, C.c_void_p]

    def norm(dtype=2, rdtype=0, **kw):
        a = _Norm(**{**dict(x=4096, stride_x=64, xq=4096, rows=4, width=64, eps=1e-5, stride_out=64, stride_residual=64), **kw})
        return L.ssdi8_add_norm_quantize(C.addressof(a), dtype, rdtype, None)

    q = _q(bd)
    assert L.ssdi8_add_norm_quantize(None, 0, 0, None) == bd.ERR_NULL
    assert norm(xq=0) == bd.ERR_NULL and norm(fp4=C.addressof(q)) == bd.ERR_UNSUPPORTED
    assert norm(xq=0, fp4=C.addressof(q), static_scale=4096) == bd.ERR_UNSUPPORTED and norm(xq=0, fp4=C.addressof(q), scale=4096) == bd.ERR_UNSUPPORTED
    assert norm(dtype=3) == bd.ERR_UNSUPPORTED and norm(residual=4096, rdtype=1) == bd.ERR_UNSUPPORTED and norm(dtype=0, residual_out=4096, rdtype=2) == bd.ERR_UNSUPPORTED
    for bad in (dict(width=0), dict(width=72), dict(width=16400), dict(rows=-1), dict(rows=1 << 31), dict(eps=-1.0), dict(eps=float("nan")),
                dict(residual_out=4096, stride_out=63)):
        assert norm(**bad) == bd.ERR_SHAPE, bad
    for bad in (dict(rows=5), dict(width=32)):
        assert norm(**{**dict(xq=0, fp4=C.addressof(q)), **bad}) == bd.ERR_SHAPE
    bad = _q(bd, step=0)
    assert norm(xq=0, fp4=C.addressof(bad)) == bd.ERR_NULL and norm(x=0) == bd.ERR_NULL
    assert norm(weight=4100) == bd.ERR_ALIGN and norm(xq=4104) == bd.ERR_ALIGN and norm(x=4097) == bd.ERR_ALIGN
    assert norm(residual=4098) == bd.ERR_ALIGN and norm(residual_out=4098) == bd.ERR_ALIGN
    assert norm(rows=0) == bd.OK

    def linear(x=q, w=q, dtype=2, **kw):
        a = _Linear(**{**dict(x=C.addressof(x) if x else None, w=C.addressof(w) if w else None, out=4096, stride_out=64, stride_residual=64), **kw})
        return L.ssdi8_fp4_linear(C.addressof(a), dtype, None)

    assert linear(x=None) == bd.ERR_NULL and linear(w=None) == bd.ERR_NULL and linear(out=0) == bd.ERR_NULL
    assert linear(dtype=3) == bd.ERR_UNSUPPORTED and linear(act=3) == bd.ERR_UNSUPPORTED and linear(act=-1) == bd.ERR_UNSUPPORTED
    for x, w in ((_q(bd, width=96), q), (_q(bd, block=32), q), (q, _q(bd, rows=0)), (_q(bd, width=40), _q(bd, width=40)), (_q(bd, rows=-1), q),
                 (q, _q(bd, rows=0x7fffffff))):
        assert linear(x=x, w=w) == bd.ERR_SHAPE
    assert linear(stride_out=3) == bd.ERR_SHAPE
    assert linear(x=_q(bd, codes=0)) == bd.ERR_NULL and linear(w=_q(bd, scales=0)) == bd.ERR_NULL
    assert linear(x=_q(bd, codes=4100)) == bd.ERR_ALIGN and linear(out=4097) == bd.ERR_ALIGN and linear(residual=4097) == bd.ERR_ALIGN
    assert linear(x=_q(bd, rows=0)) == bd.OK


def test_refusals_of_the_handle():
    import torch
    from paper_2608_21952_b200 import binding as bd
    z = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    for codes, scales, kw in ((z(4, 20), z(1, 1, 32, 4, 4), {}), (z(4, 32), z(1, 2, 32, 4, 4), {}), (z(129, 32), z(1, 1, 32, 4, 4), {}),
                              (z(4, 32), z(1, 1, 32, 4, 4), dict(block=8)), (z(4, 32), z(512), {}),
                              (z(4, 32), z(1, 1, 32, 4, 4), dict(step=torch.ones(5)))):
        with pytest.raises(bd.SSDi8Error) as e:
            bd.fp4_of(codes, scales, **kw)
        assert e.value.code == bd.ERR_SHAPE
    with pytest.raises(TypeError):
        bd.fp4_of(z(4, 32).char(), z(1, 1, 32, 4, 4))
    for bad in ((4, 40, 16), (4, 64, 8), (4, 0, 16)):
        with pytest.raises(bd.SSDi8Error):
            bd.make_fp4(*bad)


# ---------------------------------------------------------------------------------------------------------- quantiser
QUANTIZE = [(1, 32, "float32", "normal", 0, 0), (1, 768, "bfloat16", "outliers", 0, 0), (127, 96, "float16", "grid", 0, 0), (128, 160, "float32", "grid", 0, 0),
            (129, 256, "bfloat16", "grid", 0, 0), (300, 288, "bfloat16", "zeros", 0, 0), (37, 1248, "float16", "outliers", 0, 0), (5, 5120, "float32", "bad", 0, 0),
            (5, 2112, "bfloat16", "bad", 0, 0), (3, 1056, "float16", "bad", 0, 0), (66, 2080, "float32", "normal", 24, 8), (66, 2080, "bfloat16", "outliers", 7, 3),
            (9, 416, "float32", "grid", 5, 1), (3, 16384, "bfloat16", "outliers", 0, 0), (2, 10240, "float32", "grid", 0, 0), (3, 16416, "float16", "outliers", 0, 0),
            (5, 40000, "bfloat16", "bad", 0, 0), (2, 131072, "float32", "normal", 0, 0), (130, 16448, "bfloat16", "grid", 9, 5)]


@pytest.mark.gpu
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("T,D,dtype,kind,extra,offset", QUANTIZE)
def test_quantize(T, D, dtype, kind, extra, offset, block):
    from paper_2608_21952_b200 import binding as bd
    x = _inputs(kind, T, D, T + D, dtype)
    q = _marked(T, D, block)
    bd.ssdi8_fp4_quantize(_rows(x, dtype, extra, offset), q)
    _check_fp4(q, *ref.quantize(x, block), block)


@pytest.mark.gpu
def test_quantize_next_to_the_middles():
    """values on, next above and next below every middle of two codes, under many row step sizes; the block's scale is made by a value of 6 d"""
    from paper_2608_21952_b200 import binding as bd
    r = np.random.default_rng(4)
    T, D = 512, 256
    x = np.zeros((T, D), np.float32)
    x[:, 0] = r.uniform(1, 2, T) * 2.0 ** r.integers(-40, 41, T)            # the row's absmax
    g = ref.row_step(x[:, 0]).astype(np.float64)
    mid = (ref.E2M1[:-1] + ref.E2M1[1:]) / 2
    for b in range(1, 16):
        d = g * ref.E4M3[r.integers(8, 126, T)]
        x[:, 16 * b] = np.minimum(6 * d, x[:, 0])
        for k in range(1, 16):
            v = (r.choice(mid, T) * d).astype(np.float32)
            v = np.where(k % 3 == 1, v, np.nextafter(v, np.float32(np.inf if k % 3 else -np.inf))).astype(np.float32)
            x[:, 16 * b + k] = v * r.choice([-1, 1], T)
    q = _marked(T, D, 16)
    bd.ssdi8_fp4_quantize(_dev(x), q)
    _check_fp4(q, *ref.quantize(x, 16), 16)


@pytest.mark.gpu
@pytest.mark.parametrize("block", [16, 32])
def test_quantize_subnormal_and_largest(block):
    """what binary32 holds at its ends (blocks of 16: only rows whose quotients are exact, absmax from 2e-32 on)"""
    from paper_2608_21952_b200 import binding as bd
    r = np.random.default_rng(5)
    x = r.standard_normal((64, 128)).astype(np.float32)
    x /= np.abs(x).max(-1, keepdims=True)
    top = np.float32(2.0) ** (np.linspace(-104, 127, 64) if block == 16 else np.linspace(-149, 127, 64)).astype(np.float32)
    x = (x.astype(np.float64) * np.minimum(top.astype(np.float64), 3.4e38)[:, None]).astype(np.float32)
    q = _marked(64, 128, block)
    bd.ssdi8_fp4_quantize(_dev(x), q)
    _check_fp4(q, *ref.quantize(x, block), block)


@pytest.mark.gpu
def test_quantize_block_32_without_step():
    from paper_2608_21952_b200 import binding as bd
    x = _inputs("normal", 40, 96, 1, "float32")
    q = _marked(40, 96, 32)
    h = bd.fp4_of(q.tensors["codes"], q.tensors["scales"], None, 32)
    bd.ssdi8_fp4_quantize(_dev(x), h)
    c, s, _ = ref.quantize(x, 32)
    _check_fp4(q, c, s, None, 32)


def _matrix(T, D, block, seed, lo=None, hi=None, step=True, spare=0):
    """(handle, codes, scale bytes, step sizes) of a matrix of random codes"""
    from paper_2608_21952_b200 import binding as bd
    r = np.random.default_rng(seed)
    lo, hi = (lo, hi) if lo is not None else (60, 127) if block == 16 else (120, 132)
    c, s = r.integers(0, 16, (T, D)).astype(np.uint8), r.integers(lo, hi, (T, D // block)).astype(np.uint8)
    g = r.uniform(0.5, 2, T).astype(np.float32) if step else None
    tiles = ref.tile(s)
    if spare:
        tiles = np.concatenate([tiles, np.full((spare,) + tiles.shape[1:], 255, np.uint8)])
    return bd.fp4_of(_dev(ref.pack(c)), _dev(tiles), None if g is None else _dev(g), block), c, s, np.ones(T, np.float32) if g is None else g


@pytest.mark.gpu
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("T,D,dtype,extra,offset,step", [(1, 32, "float32", 0, 0, True), (129, 96, "bfloat16", 0, 0, True), (300, 1248, "float16", 0, 0, False),
                                                         (17, 2080, "bfloat16", 7, 3, True), (5, 131072, "float32", 0, 0, True), (1000, 5120, "bfloat16", 8, 8, False)])
def test_dequantize(T, D, dtype, extra, offset, step, block):
    import torch
    from paper_2608_21952_b200 import binding as bd
    q, c, s, g = _matrix(T, D, block, T + D, 0 if block == 16 else 100, 127 if block == 16 else 140, step)
    wide = torch.full((T, D + extra), 77.0, dtype=getattr(torch, dtype), device="cuda")
    bd.ssdi8_fp4_dequantize(q, wide[:, offset:offset + D])
    want = ref.round_to((ref.values(c, s, block).astype(np.float32) * g[:, None]).astype(np.float32), dtype)
    got = _np(wide)
    np.testing.assert_array_equal(got[:, offset:offset + D], want)
    assert (got[:, :offset] == 77).all() and (got[:, offset + D:] == 77).all()


# ---------------------------------------------------------------------------------------------------------- norm
NORM = [(1, 16, "bfloat16", "float32", "normal", 0), (1, 768, "bfloat16", "float32", "outliers", 0), (3, 48, "float32", None, "normal", 0),
        (64, 2560, "bfloat16", "bfloat16", "outliers", 0), (37, 1248, "float16", "float16", "outliers", 0), (37, 1232, "float16", "float32", "grid", 0),
        (5, 5120, "float32", "float32", "zeros", 0), (129, 288, "bfloat16", "float32", "grid", 5), (9, 4112, "bfloat16", "bfloat16", "outliers", 3),
        (3, 16384, "bfloat16", "float32", "outliers", 0), (2, 8208, "float32", None, "normal", 8), (6, 2080, "bfloat16", "float32", "bad", 0)]


def _norm_case(T, D, dtype, rdtype, kind, extra, seed=0):
    x = _inputs(kind, T, D, T + D + seed, dtype)
    res = None if rdtype is None else _inputs("zeros" if kind == "zeros" else "outliers", T, D, T + D + 1 + seed, rdtype)
    if kind == "zeros" and res is not None:
        res = -x if rdtype == dtype else res
    with np.errstate(invalid="ignore"):
        h = x if res is None else ref.round_to((x + res).astype(np.float32), rdtype)
    w = np.random.default_rng(seed + 9).uniform(0.5, 1.5, D).astype(np.float32)
    with np.errstate(over="ignore"):
        return x, res, h, w, (h * w).astype(np.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["int8", "static", "fp4 16", "fp4 32"])
@pytest.mark.parametrize("T,D,dtype,rdtype,kind,extra", NORM)
def test_add_norm(T, D, dtype, rdtype, kind, extra, form):
    import torch
    from paper_2608_21952_b200 import binding as bd
    if form[:3] == "fp4":
        D = (D + 31) // 32 * 32
    x, res, h, w, p = _norm_case(T, D, dtype, rdtype, kind, extra)
    xd, off = _rows(x, dtype, extra, 1 if extra else 0), 1 if extra else 0
    kw = {}
    if rdtype is not None:
        wide = torch.full((T, D + extra), 77.0, dtype=getattr(torch, rdtype), device="cuda")
        kw = dict(residual=_rows(res, rdtype, extra, off), residual_out=wide[:, off:off + D])
    with np.errstate(invalid="ignore", over="ignore"):
        r = ref.factor(h, 1e-5)
    top = np.where(np.isnan(p), 0, np.abs(p)).max(-1)
    wd = _dev(w)
    if form[:3] == "fp4":
        q = _marked(T, D, int(form[4:]))
        bd.ssdi8_add_norm_quantize(xd, weight=wd, fp4=q, **kw)
        c, s, g = ref.quantize(p, q.block)
        _check_fp4(q, c, s, None, q.block)
        with np.errstate(invalid="ignore"):
            scale, want = _np(q.tensors["step"]), np.where(top > 0, g.astype(np.float64) * r, 1.0)
    else:
        xq, scale = torch.full((T, D), 99, dtype=torch.int8, device="cuda"), torch.full((T,), 77.0, device="cuda")
        if form == "static":
            s = np.float32(0.047)
            bd.ssdi8_add_norm_quantize(xd, weight=wd, xq=xq, scale=scale, static_scale=_dev(np.array([s])), **kw)
            with np.errstate(invalid="ignore", over="ignore"):
                codes = ref.int8_codes(p * r.astype(np.float32)[:, None], s)
            want = np.full(T, 77.0)
        else:
            bd.ssdi8_add_norm_quantize(xd, weight=wd, xq=xq, scale=scale, **kw)
            a = (top.astype(np.float32) / np.float32(127)).astype(np.float32)
            some = a > 0
            a = np.where(some, a, np.float32(1))
            codes = ref.int8_codes(p, a[:, None])
            with np.errstate(invalid="ignore"):
                want = np.where(some, a.astype(np.float64) * r, 1.0)
        np.testing.assert_array_equal(_np(xq), codes)
        scale = _np(scale)
    # one rounding to binary32; the sum's in binary64 are far below
    fine = np.isfinite(want)
    assert np.all(np.abs(scale[fine] - want[fine]) <= (EPS + 1e-14) * np.abs(want[fine]))
    np.testing.assert_array_equal(np.isnan(scale), np.isnan(want))
    if rdtype is not None:
        got = _np(wide)
        np.testing.assert_array_equal(got[:, off:off + D], h)
        assert (got[:, :off] == 77).all() and (got[:, off + D:] == 77).all()


# rows that a block walks through shared memory, several each; the last two are too wide for that, or on no 16-byte boundary
MANY = [(7300, 96, "bfloat16", "float32", "outliers", 0), (7300, 768, "float16", "float16", "grid", 0), (1900, 2560, "bfloat16", "float32", "outliers", 0),
        (1000, 5120, "float32", "float32", "zeros", 0), (1000, 8192, "bfloat16", "bfloat16", "normal", 0), (400, 16384, "bfloat16", "float32", "outliers", 0),
        (7300, 1248, "bfloat16", None, "normal", 0), (4000, 1264, "float16", "float32", "bad", 0), (310, 16384, "float32", "float32", "normal", 0),
        (2000, 2112, "bfloat16", "float32", "normal", 3)]


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["int8", "static", "fp4 16", "fp4 32"])
@pytest.mark.parametrize("T,D,dtype,rdtype,kind,extra", MANY)
def test_add_norm_many_rows(T, D, dtype, rdtype, kind, extra, form):
    test_add_norm(T, D, dtype, rdtype, kind, extra, form)


@pytest.mark.gpu
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("T,D,dtype,kind,extra,offset", [(7400, 32, "bfloat16", "normal", 0, 0), (6100, 2560, "bfloat16", "outliers", 0, 0), (1001, 5120, "float32", "grid", 0, 0),
                                                         (1000, 16384, "float16", "bad", 0, 0), (7300, 2112, "bfloat16", "bad", 16, 8), (2001, 2112, "bfloat16", "zeros", 3, 1)])
def test_quantize_many_rows(T, D, dtype, kind, extra, offset, block):
    test_quantize(T, D, dtype, kind, extra, offset, block)


@pytest.mark.gpu
@pytest.mark.parametrize("over", ["residual", "x"])
def test_add_norm_many_rows_in_place(over):
    import torch
    from paper_2608_21952_b200 import binding as bd
    T, D = 6100, 1280
    x, res, h, w, p = _norm_case(T, D, "bfloat16", "bfloat16", "outliers", 0)
    t = {"x": _dev(x, "bfloat16"), "residual": _dev(res, "bfloat16")}
    xq, status = torch.empty(T, D, dtype=torch.int8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    bd.ssdi8_add_norm_quantize(t["x"], residual=t["residual"], residual_out=t[over], weight=_dev(w), xq=xq, status=status)
    np.testing.assert_array_equal(_np(t[over]), h)
    np.testing.assert_array_equal(_np(xq), ref.int8_codes(p, (np.abs(p).max(-1).astype(np.float32) / np.float32(127))[:, None]))
    assert int(status.item()) == 0


@pytest.mark.gpu
def test_add_norm_in_place_first_layer_and_last():
    """residual_out over the residual, over x; without a residual (the stream begins); without residual_out (it ends)"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    T, D = 33, 2560
    x, res, h, w, p = _norm_case(T, D, "bfloat16", "bfloat16", "outliers", 0)
    a = np.abs(p).max(-1).astype(np.float32) / np.float32(127)
    codes = ref.int8_codes(p, a[:, None])
    xq, wd = torch.empty(T, D, dtype=torch.int8, device="cuda"), _dev(w)
    for over in ("residual", "x", None):
        t = {"x": _dev(x, "bfloat16"), "residual": _dev(res, "bfloat16")}
        bd.ssdi8_add_norm_quantize(t["x"], residual=t["residual"], residual_out=t.get(over), weight=wd, xq=xq)
        np.testing.assert_array_equal(_np(xq), codes)
        np.testing.assert_array_equal(_np(t["x"]), h if over == "x" else x)
        np.testing.assert_array_equal(_np(t["residual"]), h if over == "residual" else res)
    stream = torch.empty(T, D, device="cuda")
    bd.ssdi8_add_norm_quantize(_dev(x, "bfloat16"), residual_out=stream, xq=xq)     # no weight
    np.testing.assert_array_equal(_np(stream), x)
    np.testing.assert_array_equal(_np(xq), ref.int8_codes(x, (np.abs(x).max(-1).astype(np.float32) / np.float32(127))[:, None]))


@pytest.mark.gpu
def test_add_norm_binding_refusals():
    import torch
    from paper_2608_21952_b200 import binding as bd
    x, xq = torch.zeros(4, 64, device="cuda"), torch.zeros(4, 64, dtype=torch.int8, device="cuda")
    with pytest.raises(bd.SSDi8Error):
        bd.ssdi8_add_norm_quantize(x)
    with pytest.raises(bd.SSDi8Error):
        bd.ssdi8_add_norm_quantize(x, residual=x[:3], xq=xq)
    with pytest.raises(bd.SSDi8Error):
        bd.ssdi8_add_norm_quantize(x, residual=x.half(), xq=xq)
    with pytest.raises(TypeError):
        bd.ssdi8_add_norm_quantize(x, residual=x, residual_out=x.half(), xq=xq)
    with pytest.raises(bd.SSDi8Error):
        bd.ssdi8_add_norm_quantize(x, fp4=bd.make_fp4(5, 64))
    with pytest.raises(TypeError):
        bd.ssdi8_add_norm_quantize(x, fp4=x)
    q, w = bd.make_fp4(4, 64), bd.make_fp4(8, 96)
    with pytest.raises(bd.SSDi8Error):
        bd.ssdi8_fp4_linear(q, w, torch.zeros(4, 8, device="cuda"))
    with pytest.raises(bd.SSDi8Error):
        bd.ssdi8_fp4_linear(q, bd.make_fp4(8, 64), torch.zeros(4, 9, device="cuda"))
    with pytest.raises(bd.SSDi8Error):
        bd.ssdi8_fp4_quantize(x[:3], q)
    bd.ssdi8_fp4_linear(bd.make_fp4(0, 64), bd.make_fp4(8, 64), torch.zeros(0, 8, device="cuda"))
    bd.ssdi8_fp4_quantize(x[:0], bd.make_fp4(0, 64))
    bd.ssdi8_fp4_dequantize(bd.make_fp4(0, 64), x[:0])
    bd.ssdi8_add_norm_quantize(x[:0], xq=xq[:0])


# ---------------------------------------------------------------------------------------------------------- product
def _linear(T, O, K, block, dtype, bias=False, act=0, residual=False, extra=0, offset=0, seed=0, exact=False, steps=True, rextra=None):
    """runs a product and compares it; exact: scales and codes whose sums binary32 holds, so that only the epilogue rounds"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    lo, hi = ((56, 65, 2) if block == 16 else (126, 129, 1))[:2] if exact else (None, None)
    x, cx, sx, gx = _matrix(T, K, block, seed + 1, lo, hi, steps, spare=1)
    w, cw, sw, gw = _matrix(O, K, block, seed + 2, lo, hi, steps)
    r = np.random.default_rng(seed + 3)
    b = r.standard_normal(O).astype(np.float32) if bias else None
    res = ref.round_to(r.standard_normal((T, O)), dtype) if residual else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    wide = torch.full((T, O + extra), 77.0, dtype=getattr(torch, dtype), device="cuda")
    out = wide[:, offset:offset + O]
    bd.ssdi8_fp4_linear(x, w, out, bias=None if b is None else _dev(b), residual=None if res is None else _rows(res, dtype, *((extra, offset) if rextra is None else (rextra, rextra // 2))), act=act, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    vx, vw = ref.values(cx, sx, block), ref.values(cw, sw, block)
    s, size = vx @ vw.T, np.abs(vx) @ np.abs(vw).T
    g = gx.astype(np.float64)[:, None] * gw.astype(np.float64)
    v = s * g + (0 if b is None else b.astype(np.float64))
    want = ref.act(v, act) + (0 if res is None else res)
    # the sum: K roundings of its terms' magnitudes (none where it is exact); two products and a sum behind it; the activation's own error and its slope
    # (SiLU below 1.1, squared ReLU 2 |v|), the residual's addition, the result's rounding
    dv = (0 if exact else K * EPS) * size * g + 3 * EPS * (np.abs(s * g) + np.abs(v))
    da = dv if act == 0 else 1.1 * dv + (10 + 1.5 * np.abs(v)) * EPS * np.abs(ref.act(v, 1)) + 1e-37 if act == 1 else 2 * np.maximum(v, 0) * dv + dv * dv + 2 * EPS * want.clip(0)
    tol = da + EPS * np.abs(want)
    tol = tol + HALF[dtype] * (np.abs(want) + tol) + TINY[dtype]
    got = _np(wide)
    # (beyond the type's largest number by more than half a step the nearest is an infinity: fp16's 65504 and 65520)
    beyond = np.abs(want) - tol > 65520 if dtype == "float16" else np.zeros(want.shape, bool)
    near = np.abs(want) + tol >= 65520 if dtype == "float16" else beyond
    mine = got[:, offset:offset + O]
    assert np.all(mine[beyond] == np.sign(want[beyond]) * np.inf)
    off = np.where(near & (beyond | np.isinf(mine)), 0, np.abs(np.where(np.isinf(mine) & near, 0, mine) - want))
    assert np.all(off <= tol), (float((off / tol).max()), np.unravel_index(np.argmax(off / tol), off.shape))
    assert (got[:, :offset] == 77).all() and (got[:, offset + O:] == 77).all()


FEW = [(1, 128, 256, {}), (1, 8, 32, {}), (3, 24, 64, {}), (16, 300, 288, {}), (17, 129, 96, dict(bias=True)), (64, 1000, 2560, dict(residual=True)),
       (128, 256, 512, dict(act=1)), (33, 77, 1248, dict(act=2, bias=True)), (129, 130, 320, {}), (250, 400, 1024, dict(bias=True, act=1)),
       (256, 128, 4096, {}), (257, 384, 2112, dict(residual=True)), (300, 200, 768, {}), (64, 640, 8192, dict(residual=True, bias=True)), (700, 260, 160, {}),
       (5, 2570, 160, dict(steps=False))]


@pytest.mark.gpu
@pytest.mark.parametrize("exact", [True, False])
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("T,O,K,kw", FEW)
def test_linear_few_rows(T, O, K, kw, block, exact):
    _linear(T, O, K, block, "float32", exact=exact and K <= 2560, seed=T + O, **kw)


PAIR = [(2304, 2560, 256, {}), (4096, 4096, 512, dict(bias=True, residual=True)), (5000, 3001, 96, dict(residual=True)), (20000, 600, 352, dict(act=1)),
        (3500, 5130, 1248, {}), (16384, 1300, 64, dict(act=2))]


@pytest.mark.gpu
@pytest.mark.parametrize("exact", [True, False])
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("T,O,K,kw", PAIR)
def test_linear_many_rows(T, O, K, kw, block, exact):
    _linear(T, O, K, block, "float32", exact=exact, seed=T + O, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("T,O,K,extra,offset", [(1, 130, 256, 0, 0), (40, 264, 288, 6, 3), (40, 264, 288, 8, 8), (300, 200, 512, 5, 0), (4000, 4003, 160, 0, 0),
                                                (4000, 4000, 160, 16, 8), (4000, 4000, 160, 3, 1)])
def test_linear_types_and_strides(T, O, K, extra, offset, dtype):
    _linear(T, O, K, 16, dtype, bias=True, act=1, residual=True, extra=extra, offset=offset, seed=T + extra)


@pytest.mark.gpu
@pytest.mark.parametrize("T,O,extra,offset,rextra", [(4000, 4000, 3, 1, 0), (4000, 4000, 0, 0, 5), (4100, 4001, 0, 0, 3), (4000, 4002, 2, 1, 2), (4000, 4001, 3, 2, 1), (60, 203, 0, 0, 1),
                                                     (60, 204, 1, 1, 0), (300, 1003, 4, 3, 2)])
def test_linear_residual_on_other_boundaries(T, O, extra, offset, rextra):
    _linear(T, O, 160, 16, "bfloat16", residual=True, extra=extra, offset=offset, rextra=rextra, seed=T + O)


@pytest.mark.gpu
def test_linear_residual_in_place_and_again():
    """out over the residual; the same call again gives the same bits, captured too, on another stream"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    for T, O, K in ((64, 2560, 5120), (4096, 2560, 512), (64, 2563, 512), (4096, 2563, 512)):
        x, w = _matrix(T, K, 16, 1)[0], _matrix(O, K, 16, 2)[0]
        res = torch.randn(T, O, device="cuda").bfloat16()
        a, b = torch.empty_like(res), res.clone()
        bd.ssdi8_fp4_linear(x, w, a, residual=res)
        bd.ssdi8_fp4_linear(x, w, b, residual=b)
        assert torch.equal(a, b)
        side, c = torch.cuda.Stream(), torch.empty_like(res)
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            bd.ssdi8_fp4_linear(x, w, c, residual=res)
        for _ in range(3):
            c.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(a, c)
        d = torch.zeros_like(res)
        side.wait_stream(torch.cuda.current_stream())
        bd.ssdi8_fp4_linear(x, w, d, residual=res, stream=side)
        side.synchronize()
        assert torch.equal(a, d)


@pytest.mark.gpu
def test_linear_offsets_beyond_32_bits():
    """rows of out 12 million elements apart: the last ones lie beyond 2^31"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    for T, O in ((200, 260), (2304, 2560)):
        stride = (1 << 31) // T + 4096
        if T * stride * 2 > torch.cuda.mem_get_info()[0] // 2:
            pytest.skip("not enough memory")
        K = 256
        x, w = _matrix(T, K, 32, 1)[0], _matrix(O, K, 32, 2)[0]
        flat = torch.empty(T * stride, dtype=torch.bfloat16, device="cuda")
        out, want = flat.as_strided((T, O), (stride, 1)), torch.empty(T, O, dtype=torch.bfloat16, device="cuda")
        bd.ssdi8_fp4_linear(x, w, out)
        bd.ssdi8_fp4_linear(x, w, want)
        assert torch.equal(out, want)
        q, y = bd.make_fp4(T, O // 32 * 32), want[:, : O // 32 * 32]
        bd.ssdi8_fp4_quantize(y, q)
        again = bd.make_fp4(T, O // 32 * 32)
        bd.ssdi8_fp4_quantize(out[:, : O // 32 * 32], again)
        assert torch.equal(q.tensors["codes"], again.tensors["codes"]) and torch.equal(q.tensors["scales"], again.tensors["scales"])
        del flat, out


@pytest.mark.gpu
def test_two_streams_at_once():
    """quantiser, norm, values and products of every form on two streams beside one another: the results of calls alone"""
    import torch
    from paper_2608_21952_b200 import binding as bd

    class Work:
        def __init__(self, seed, T, O, K, block):
            g = torch.Generator(device="cuda").manual_seed(seed)
            self.x, self.res = (torch.randn(T, K, generator=g, device="cuda").bfloat16() for _ in range(2))
            self.q, self.w, self.block = bd.make_fp4(T, K, block), bd.make_fp4(O, K, block), block
            bd.ssdi8_fp4_quantize(torch.randn(O, K, generator=g, device="cuda"), self.w)
            self.stream, self.out = torch.empty_like(self.x), torch.empty(T, O, dtype=torch.float16, device="cuda")
            self.again, self.values = bd.make_fp4(T, O // 32 * 32, block), torch.empty(T, O // 32 * 32, device="cuda")

        def run(self, stream=None):
            bd.ssdi8_add_norm_quantize(self.x, residual=self.res, residual_out=self.stream, fp4=self.q, stream=stream)
            bd.ssdi8_fp4_linear(self.q, self.w, self.out, act=bd.ACT_SILU, stream=stream)
            bd.ssdi8_fp4_quantize(self.out[:, :self.values.shape[1]], self.again, stream=stream)
            bd.ssdi8_fp4_dequantize(self.again, self.values, stream=stream)

        def clear(self):
            for t in (self.stream, self.out, self.values):
                t.zero_()

    works = [[Work(10 * s + i, *c) for i, c in enumerate(((64, 2560, 1280, 16), (2304, 2561, 512, 32), (300, 640, 2048, 16), (1, 1000, 768, 32), (4000, 1280, 256, 16)))]
             for s in (0, 1)]
    want = []
    for side in works:
        for w in side:
            w.run()
            want.append([t.clone() for t in (w.stream, w.out, w.values)])
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for side in works:
            for w in side:
                w.clear()
        torch.cuda.synchronize()
        for i in range(len(works[0])):
            for side, st in zip(works, streams):
                side[i].run(st)
        torch.cuda.synchronize()
        for w, y in zip((w for side in works for w in side), want):
            for a, b in zip((w.stream, w.out, w.values), y):
                assert torch.equal(a, b)


@pytest.mark.gpu
def test_codes_and_rows_beyond_32_bits():
    """more than 2^32 codes, and a stream of more than 2^31 elements: the last rows are as of a call on them alone"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    T, D, n = 34000, 131072, 130
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("not enough memory")
    x = torch.empty(T, D, dtype=torch.bfloat16, device="cuda").fill_(1.5)
    x[-n:] = torch.randn(n, D, device="cuda").to(torch.bfloat16)
    big, small = bd.make_fp4(T, D), bd.make_fp4(n, D)
    bd.ssdi8_fp4_quantize(x, big)
    bd.ssdi8_fp4_quantize(x[-n:], small)
    assert torch.equal(big.tensors["codes"][-n:], small.tensors["codes"]) and torch.equal(big.tensors["step"][-n:], small.tensors["step"])
    want = torch.empty(n, D, dtype=torch.bfloat16, device="cuda")
    bd.ssdi8_fp4_dequantize(small, want)
    bd.ssdi8_fp4_dequantize(big, x)
    assert torch.equal(x[-n:], want)
    del big, small, want, x
    T, D = 135000, 16384
    x, res = (torch.empty(T, D, dtype=torch.bfloat16, device="cuda").fill_(0.5) for _ in range(2))
    x[-n:] = torch.randn(n, D, device="cuda").to(torch.bfloat16)
    last, xq, one = res[-n:].clone(), torch.empty(T, D, dtype=torch.int8, device="cuda"), torch.empty(n, D, dtype=torch.int8, device="cuda")
    bd.ssdi8_add_norm_quantize(x, residual=res, residual_out=res, xq=xq)
    bd.ssdi8_add_norm_quantize(x[-n:], residual=last, residual_out=last, xq=one)
    assert torch.equal(xq[-n:], one) and torch.equal(res[-n:], last)


@pytest.mark.gpu
def test_linear_in_a_row():
    """calls of all forms one behind the other without a wait, each scheduled while the one before drains; their results as of calls alone"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    shapes = [(1, 300, 512), (4096, 2560, 512), (250, 1000, 1024), (64, 2560, 2560), (5000, 1200, 256), (128, 256, 512)]
    ops = [(_matrix(T, K, b, 1)[0], _matrix(O, K, b, 2)[0], torch.empty(T, O, device="cuda")) for T, O, K in shapes for b in (16, 32)]
    want = []
    for x, w, out in ops:
        bd.ssdi8_fp4_linear(x, w, out)
        torch.cuda.synchronize()
        want.append(out.clone())
    for _ in range(20):
        for x, w, out in ops:
            out.fill_(0)
        for x, w, out in ops:
            bd.ssdi8_fp4_linear(x, w, out)
        torch.cuda.synchronize()
        for (x, w, out), y in zip(ops, want):
            assert torch.equal(out, y)
