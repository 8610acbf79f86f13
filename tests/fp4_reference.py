"""Matrices in four bits, the norm ahead of them and their product in numpy's binary64, from the definitions in include/ssdi8.h."""
import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
_e4 = [m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)]
E4M3 = np.array(_e4[:127])          # of the bytes 0 to 126 (127 is a NaN)


def nearest(v, unit, grid):
    """index of the number of `grid` (ascending) that v / unit is nearest to, ties to the even index, beyond the last one that;
    v >= 0 and unit broadcast together, their comparisons exact where grid's middles times unit have 53 bits"""
    mid = (grid[:-1] + grid[1:]) / 2
    out = np.zeros(np.broadcast_shapes(v.shape, unit.shape), np.int64)
    for k, m in enumerate(mid):
        out += (v > m * unit) if k % 2 == 0 else (v >= m * unit)
    return out


def row_step(m):
    """step size of a row with absmax m (binary32), blocks of 16"""
    with np.errstate(over="ignore"):
        g = (m.astype(np.float32) / np.float32(2688)).view(np.uint32) & np.uint32(0xffffff00)
    g = g.view(np.float32)
    return np.where(g > 0, g, np.float32(1))


def quantize(p, block):
    """rows p (binary32) -> (codes 0..15 [T, D], scale bytes [T, D / block], step [T] binary32)"""
    p = np.asarray(p, np.float32)
    T, D = p.shape
    a = np.abs(p.astype(np.float64)).reshape(T, D // block, block)
    nan = np.isnan(a)
    top = np.where(nan, 0.0, a).max(-1)
    if block == 16:
        g = row_step(top.max(-1).astype(np.float32))
        unit = 6.0 * g.astype(np.float64)[:, None]
        inf = np.isinf(unit)
        s = np.maximum(nearest(top, np.where(inf, 1.0, unit), E4M3), 1)       # at least 2^-9
        s = np.where(inf, 1, s)
        d = g.astype(np.float64)[:, None] * E4M3[s]
        step = g
    else:
        f, e = np.frexp(top)                        # top = f 2^e, 1/2 <= f < 1;  1.5 2^k is f = 3/4
        e = np.clip(np.where(f <= 0.75, e - 3, e - 2), -127, 127)
        e = np.where(top > 0, e, 0)
        s, d, step = e + 127, np.exp2(e.astype(np.float64)), np.ones(T, np.float32)
        inf = np.isinf(top)
        s = np.where(inf, 253, s)
        d = np.where(inf, 2.0 ** 126, d)
    d = d[..., None] + np.zeros_like(a)
    with np.errstate(invalid="ignore"):
        c = nearest(np.where(nan, 0.0, a), d, E2M1)
    if block == 16:
        c = np.where(np.isinf(d), np.where(np.isinf(a), 7, 0), c)
    c = np.where(nan, 7, c)
    neg = (p < 0).reshape(a.shape) & ~nan & ~np.isinf(d)   # (-0 is 0; in a row with an infinity: inf / inf is a NaN, +6, the rest 0)
    return (c + 8 * neg).reshape(T, D).astype(np.uint8), s.astype(np.uint8), step


def pack(c):
    return (c[:, 0::2] | c[:, 1::2] << 4).astype(np.uint8)


def unpack(b):
    out = np.empty((b.shape[0], 2 * b.shape[1]), np.uint8)
    out[:, 0::2], out[:, 1::2] = b & 15, b >> 4
    return out


def tile(s):
    """scale bytes [T, blocks] in tiles [ceil(T / 128), ceil(blocks / 4), 32, 4, 4]"""
    T, n = s.shape
    out = np.zeros((-(-T // 128), -(-n // 4), 32, 4, 4), np.uint8)
    t, b = np.meshgrid(np.arange(T), np.arange(n), indexing="ij")
    out[t // 128, b // 4, t % 32, t % 128 // 32, b % 4] = s
    return out


def untile(x, T, n):
    t, b = np.meshgrid(np.arange(T), np.arange(n), indexing="ij")
    return x[t // 128, b // 4, t % 32, t % 128 // 32, b % 4]


def scale_values(s, block):
    return E4M3[s] if block == 16 else np.exp2(s.astype(np.float64) - 127)


def values(codes, s, block):
    """[T, D] binary64, without the step sizes"""
    v = E2M1[codes & 7] * np.where(codes > 7, -1.0, 1.0)
    return v * np.repeat(scale_values(s, block), block, axis=1)


def round_to(v, dtype):
    """binary32 values rounded to a torch type by name, as binary32"""
    import torch
    return torch.from_numpy(np.ascontiguousarray(v, np.float32)).to(getattr(torch, dtype)).float().numpy()


def factor(h, eps):
    """1 / sqrt(mean of h^2 + eps) per row, binary64"""
    h = h.astype(np.float64)
    with np.errstate(divide="ignore"):
        return 1.0 / np.sqrt((h * h).sum(-1) / h.shape[1] + np.float64(np.float32(eps)))


def int8_codes(p, step):
    """rne(fdiv(p, step)) saturated, a NaN +127; binary32"""
    with np.errstate(invalid="ignore", over="ignore"):
        q = (p.astype(np.float32) / step.astype(np.float32)).astype(np.float32)
    return np.where(np.isnan(q), 127, np.clip(np.rint(np.where(np.isnan(q), 0, q)), -127, 127)).astype(np.int8)


def act(v, kind):
    if kind == 1:
        with np.errstate(over="ignore"):
            return v / (1 + np.exp(-v))
    return np.maximum(v, 0) ** 2 if kind == 2 else v
