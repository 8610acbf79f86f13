"""The operators around the layer at the edges of what they take: values that are not finite, rows and groups of zeros, step sizes
at the ends of the range, status words in use, arguments that contradict one another."""
import ctypes as C

import numpy as np
import pytest

import block_reference as ref
from test_block_ops import ADDR, LinearArgs, _cache, _dims, _lib, _np, _t, _token_params


# ------------------------------------------------------------------------------------------------ projection
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,O,K", [(3, 40, 64), (200, 72, 144), (3000, 2570, 656)])   # few rows, lone tiles, pairs of SMs
def test_squared_relu_of_values_that_are_not_finite(T, O, K, dtype):
    """max(v, 0)^2 is 0 for -inf (of a bias that closes an output, of a product that overflows), inf for inf and NaN for NaN alone"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    x, w = np.ones((T, K), np.int8), np.ones((O, K), np.int8)
    w[5] = -1
    sw, bias = np.full(O, 2.0 ** -10, np.float32), np.zeros(O, np.float32)
    bias[1], bias[2], bias[3], bias[4] = -np.inf, np.inf, np.nan, -3.0
    sw[5] = 3e38   # (K products of -1: beyond binary32)
    sw[6] = 3e38
    want = np.full(O, (K * 2.0 ** -10) ** 2)
    want[[1, 2, 3, 4, 5, 6]] = [0, np.inf, np.nan, 0, 0, np.inf]
    for residual in (None, 0.5):
        out = torch.full((T, O), 7.0, device="cuda").to(getattr(torch, dtype))
        res = None if residual is None else torch.full_like(out, residual)
        bd.ssdi8_linear(_t(x), _t(w), _t(sw), out, bias=_t(bias), residual=res, act=bd.ACT_RELU2)
        got = _np(out).astype(np.float64)
        exact = np.broadcast_to(want + (residual or 0), got.shape)
        np.testing.assert_array_equal(got[:, 1:7], exact[:, 1:7])
        assert residual is not None or not np.signbit(got[:, [1, 4, 5]]).any()
        # (K 2^-10, its square and the sum: one rounding each at most, and that of the type)
        half = 2.0 ** -24 if dtype == "float32" else 2.0 ** -8
        np.testing.assert_allclose(got[:, 7:], exact[:, 7:], rtol=half + 4 * 2.0 ** -24)


@pytest.mark.parametrize("args", [{"rows": 0x7fffff01}, {"rows": 0x7fffffff}, {"outs": 0x7fffff01, "stride_out": 1 << 31}])
def test_linear_refuses_counts_that_a_tile_would_carry_beyond_32_bits(args):
    bd, lib = _lib()
    a = LinearArgs(**{**dict(xq=ADDR, wq=ADDR, s_w=ADDR, out=ADDR, stride_out=64, rows=4, outs=64, inner=64), **args})
    assert lib.ssdi8_linear(C.byref(a), 0, None) == bd.ERR_SHAPE


# ------------------------------------------------------------------------------------------------ norm
def _norm(x, z, weight, groups, eps, static=None):
    import torch
    from paper_2608_21952_b200 import binding as bd
    T, D = x.shape
    xq, sc = torch.full((T, D), 99, dtype=torch.int8, device="cuda"), torch.full((T,), 7.0, device="cuda")
    bd.ssdi8_norm_quantize(_t(x), xq, weight=None if weight is None else _t(weight), z=None if z is None else _t(z), groups=groups, eps=eps,
                           scale=sc, static_scale=None if static is None else _t(np.array([static], np.float32)))
    return _np(xq), _np(sc)


@pytest.mark.gpu
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("static", [None, 0.03])
@pytest.mark.parametrize("groups,D", [(1, 512), (2, 512), (4, 8192)])
def test_norm_without_eps_of_rows_and_groups_of_zeros(groups, D, static, gate):
    """a group of zeros has o = 0: codes of 0, alone in its row and beside others alike; a whole row of them the step size 1"""
    rng = np.random.default_rng(D + groups)
    T = 7
    x, z = rng.standard_normal((T, D)).astype(np.float32), rng.standard_normal((T, D)).astype(np.float32)
    weight = rng.uniform(0.5, 1.5, D).astype(np.float32)
    w = D // groups
    x[0], x[2, :w], x[3, -w:], x[6, ::2] = 0, 0, 0, 0
    x[5] *= 1e-30   # (beyond binary32's squares, but no zeros)
    dead = np.repeat((x.reshape(T, groups, w) == 0).all(-1), w, -1)
    got, step = _norm(x, z if gate else None, weight, groups, 0.0, static)
    want, top = ref.norm_codes(x, z if gate else None, weight, groups, 0.0, None if static is None else np.float32(static))
    want[dead] = 0
    np.testing.assert_array_equal(got, want)
    if static is None:
        top[dead.all(-1)] = 1
        np.testing.assert_allclose(step, top, rtol=40 * 2.0 ** -24)
    else:
        assert np.all(step == 7.0)


@pytest.mark.gpu
@pytest.mark.parametrize("groups", [1, 2])
def test_norm_of_zeros_under_weights_and_steps_that_are_not_finite(groups):
    """0 times an infinite or missing weight is NaN, code +127, in a row of zeros as in any other; so is 0 over a step of 0 or NaN"""
    rng = np.random.default_rng(5)
    x = rng.standard_normal((4, 256)).astype(np.float32)
    x[0], x[1, :128] = 0, 0
    weight = rng.uniform(0.5, 1.5, 256).astype(np.float32)
    weight[7], weight[9] = np.nan, np.inf
    got, step = _norm(x[:2], None, weight, groups, 1e-5)
    want = np.zeros(256, np.int8)
    want[[7, 9]] = 127
    np.testing.assert_array_equal(got[0], want)
    assert step[0] == 1.0 and np.all(got[1, [7, 9]] == 127)
    got, _ = _norm(x, None, weight, groups, 1e-5, 0.03)
    with np.errstate(all="ignore"):
        np.testing.assert_array_equal(got, ref.norm_codes(x, None, weight, groups, 1e-5, np.float32(0.03))[0])
    for odd in (0.0, np.nan):
        got, _ = _norm(x, None, None, groups, 1e-5, odd)
        with np.errstate(all="ignore"):
            np.testing.assert_array_equal(got, ref.norm_codes(x, None, None, groups, 1e-5, np.float32(odd))[0])
        assert np.all(got[0] == 127)


@pytest.mark.gpu
@pytest.mark.parametrize("groups", [1, 2])
def test_norm_whose_factor_leaves_binary32(groups):
    """1 / (norm step) of 1e45: the small products are codes between the ends nevertheless"""
    rng = np.random.default_rng(6)
    x = (1e-15 * rng.uniform(0.5, 1.5, (3, 512)) * rng.choice([-1, 1], (3, 512))).astype(np.float32)
    weight = np.ones(512, np.float32)
    weight[::4] = 1e-28
    static = np.float32(1.5e-30)
    want, _ = ref.norm_codes(x, None, weight, groups, 0.0, static)
    assert np.abs(want[:, ::4]).max() < 127 and np.all(np.abs(want[:, 1::4]) == 127)
    got, _ = _norm(x, None, weight, groups, 0.0, static)
    np.testing.assert_array_equal(got, want)


# ------------------------------------------------------------------------------------------------ cache and token step
def _other_dims(bd):
    """other heads, other groups, another state size: what a cache of 4 heads of 64 x 64 in 2 groups was not laid out for"""
    return [_dims(bd, nheads=8), _dims(bd, nheads=2), _dims(bd, ngroups=4), _dims(bd, ngroups=1), _dims(bd, dstate=128)]


def test_calls_refuse_a_cache_of_other_dims(monkeypatch):
    """without a device: the cache is looked at ahead of every other argument (and never with the dims that it has)"""
    import torch
    bd, _ = _lib()
    monkeypatch.setattr(bd, "_ptr", lambda t: t.data_ptr())
    own = _dims(bd)
    z = lambda *s, dtype=torch.int8: torch.zeros(s, dtype=dtype)  # noqa: E731
    c = bd.cache_of(own, codes=z(4, 4, 64, 64), scales=z(4, 4, 64, dtype=torch.float32), xwin=z(4, 4, 16, 64), Bwin=z(4, 2, 16, 64),
                    dtwin=z(4, 4, 16, dtype=torch.float32), start=z(4, dtype=torch.int32), ring=z(4, 4, 512, dtype=torch.bfloat16))
    for d in _other_dims(bd):
        for call in (lambda: bd.ssdi8_cache_write(d, c, None, None, None), lambda: bd.ssdi8_cache_read(d, c, *[None] * 6),
                     lambda: bd.ssdi8_token_step(d, c, *[None] * 14)):
            with pytest.raises(bd.SSDi8Error) as err:
                call()
            assert err.value.code == bd.ERR_SHAPE


@pytest.mark.gpu
def test_a_cache_of_other_dims_stays_as_it_was():
    from paper_2608_21952_b200 import binding as bd
    import torch
    c, a, _ = _cache(np.random.default_rng(1), 4, 4, 64, 2)
    for d in _other_dims(bd):
        B, H, G, N = d.batch, d.nheads, d.ngroups, d.dstate
        state, f = torch.ones(B, H, 64, N, device="cuda"), lambda *s: torch.ones(s, device="cuda")  # noqa: E731
        pos = torch.zeros(B, dtype=torch.int32, device="cuda")
        with pytest.raises(bd.SSDi8Error):
            bd.ssdi8_cache_write(d, c, None, None, state)
        with pytest.raises(bd.SSDi8Error):
            bd.ssdi8_cache_read(d, c, None, pos, f(H), f(H * 64), f(G), state)
    for k, t in c.tensors.items():
        np.testing.assert_array_equal(_np(t), a[k])
    d = _dims(bd, batch=3, seqlen=77)   # (sequences and lengths are the call's own)
    bd.ssdi8_cache_write(d, c, None, None, torch.ones(3, 4, 64, 64, device="cuda"))
    assert np.all(_np(c.tensors["codes"])[:3] == 127)


def _token_case(seed, B, H, N, G, n=None, start=None):
    rng = np.random.default_rng(seed)
    c, a, torch = _cache(rng, n or B, H, N, G, start=start)
    p = _token_params(rng, H, N, G, 4)
    x = _t(rng.standard_normal((B, 64 * H + 2 * G * N)).astype(np.float32), "bfloat16")
    raw = _t(rng.standard_normal((B, H)).astype(np.float32), "bfloat16")
    return c, a, p, {k: _t(v) for k, v in p.items()}, x, raw, torch


def _token(bd, c, dev, x, raw, pos, y, dims, slots=None, status=None, flags=0):
    bd.ssdi8_token_step(dims, c, x, dev["w"], dev["bias"], raw, dev["dt_bias"], dev["A"], dev["D"], dev["corr"], dev["s_x"], dev["s_B"], dev["s_C"],
                        slots, pos, y, status=status, flags=bd.FLAG_DT_SOFTPLUS | flags)


@pytest.mark.gpu
def test_token_step_refuses_a_type_of_y_that_the_tensor_has_not():
    """an fp32 y with a flag of 16 bits would hold pairs of values; a flag that says what the tensor is passes"""
    from paper_2608_21952_b200 import binding as bd
    c, a, p, dev, x, raw, torch = _token_case(2, 2, 2, 64, 1)
    pos, d = torch.zeros(2, dtype=torch.int32, device="cuda"), _dims(bd, 2, 1, 2, 64, 64, 1)
    for t, flag in (("float32", bd.FLAG_Y_BF16), ("float32", bd.FLAG_Y_FP16), ("bfloat16", bd.FLAG_Y_FP16), ("float16", bd.FLAG_Y_BF16)):
        y = torch.full((2, 128), 5.0, device="cuda").to(getattr(torch, t))
        with pytest.raises(bd.SSDi8Error) as err:
            _token(bd, c, dev, x, raw, pos, y, d, flags=flag)
        assert err.value.code == bd.ERR_UNSUPPORTED and torch.all(y == 5.0)
    for k, t in c.tensors.items():
        np.testing.assert_array_equal(_np(t), a[k])
    same = [torch.empty(2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    _token(bd, c, dev, x, raw, pos, same[0], d, flags=bd.FLAG_Y_BF16)
    _token(bd, c, dev, x, raw, pos, same[1], d)
    assert torch.equal(*same)


@pytest.mark.gpu
@pytest.mark.parametrize("N,G,H", [(64, 2, 6), (128, 1, 9)])
def test_token_step_adds_a_rows_products_as_integers(N, G, H):
    """rows whose products cancel: y is off by binary32's error of the sum, not of the products (E scale sum_n C code is exact up to its factors)"""
    from paper_2608_21952_b200 import binding as bd
    B = 5
    c, a, p, dev, x, raw, torch = _token_case(3, B, H, N, G)
    p["D"][:], p["corr"][:], dev["D"], dev["corr"] = 0, 0, None, None
    pos = np.array([0, 16, 32, 48, 160], np.int32)   # (the token alone is in the window)
    u = ref.conv(_np(x)[:, None], p["w"], p["bias"], None, a["ring"].copy(), None, pos)[:, 0]
    HP, GN = 64 * H, G * N
    Cq = ref.code(u[:, HP + GN:].reshape(B, G, N) / p["s_C"].astype(np.float64)[:, None]).astype(np.int64)
    Bq = ref.code(u[:, HP:HP + GN].reshape(B, G, N) / p["s_B"].astype(np.float64)[:, None]).astype(np.int64)
    xq = ref.code(u[:, :HP] / p["s_x"].astype(np.float64)).reshape(B, H, 64).astype(np.int64)
    group = np.arange(H) // (H // G)
    # the code under the largest one of C is what brings a row's sum nearest to 0
    codes = a["codes"].astype(np.int64)
    at = np.abs(Cq).argmax(-1)   # [B, G]
    for b in range(B):
        for h in range(H):
            k = at[b, group[h]]
            big = Cq[b, group[h], k]
            if big:
                rest = codes[b, h] @ Cq[b, group[h]] - codes[b, h, :, k] * big
                codes[b, h, :, k] = np.clip(np.rint(-rest / big), -127, 127)
    c.tensors["codes"].copy_(_t(codes.astype(np.int8)))
    y = torch.empty(B, HP, device="cuda")
    _token(bd, c, dev, x, raw, _t(pos), y, _dims(bd, B, 1, H, 64, N, G))
    dt = np.stack([_np(c.tensors["dtwin"])[b, :, 0] for b in range(B)]).astype(np.float64)
    f = lambda k: p[k].astype(np.float64)  # noqa: E731
    exponent = np.abs(f("A")) * dt
    sums = np.einsum("bhpn,bhn->bhp", codes, Cq[:, group])
    off = np.exp(f("A") * dt)[..., None] * a["scales"].astype(np.float64) * sums
    own = f("s_x").reshape(H, 64) * f("s_B")[group][:, None] * (dt * (Cq * Bq).sum(-1)[:, group])[..., None] * xq
    sC = f("s_C")[group][:, None]
    want, size = sC * (off + own), sC * (np.abs(off) + np.abs(own))
    naive = sC * np.exp(f("A") * dt)[..., None] * a["scales"] * np.einsum("bhpn,bhn->bhp", np.abs(codes), np.abs(Cq[:, group]))
    bound = 2.0 ** -24 * (32 + exponent)[..., None] * size
    assert np.median(naive / np.maximum(np.abs(off * sC), 1e-30)) > 50   # (the case is what it says)
    assert np.all(np.abs(_np(y).reshape(B, H, 64) - want) <= bound)


# ------------------------------------------------------------------------------------------------ status words
def _us(torch, f, n=20, rounds=5):
    f()
    best = 1e9
    for _ in range(rounds):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        torch.cuda.synchronize()
        a.record()
        for _ in range(n):
            f()
        b.record()
        b.synchronize()
        best = min(best, 1000 * a.elapsed_time(b) / n)
    return best


@pytest.mark.gpu
@pytest.mark.parametrize("T,O,K", [(16, 256, 1024), (300, 300, 1024), (3000, 2570, 656)])
def test_linear_with_a_status_word_that_holds_another_calls_error(T, O, K):
    """SSDI8_ERR_SHAPE of a bad row elsewhere is no time-out: same outputs, no copies waited for at the end (50 us a block), the word kept"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    rng = np.random.default_rng(T)
    x, w = (_t(rng.integers(-127, 128, s).astype(np.int8)) for s in ((T, K), (O, K)))
    sw = _t(rng.uniform(0.5, 1.5, O).astype(np.float32))
    want, out = (torch.empty(T, O, device="cuda") for _ in range(2))
    clear, bad = (torch.tensor([v], dtype=torch.int32, device="cuda") for v in (0, bd.ERR_SHAPE))
    bd.ssdi8_linear(x, w, sw, want, status=clear)
    bd.ssdi8_linear(x, w, sw, out, status=bad)
    assert torch.equal(out, want) and int(bad.item()) == bd.ERR_SHAPE and int(clear.item()) == 0
    quick, slow = (_us(torch, lambda: bd.ssdi8_linear(x, w, sw, out, status=s)) for s in (clear, bad))
    assert slow < quick + 25, (quick, slow)


@pytest.mark.gpu
def test_bad_rows_do_not_hide_a_time_out():
    """a word that holds a time-out keeps it; one that holds nothing or another error becomes SSDI8_ERR_SHAPE"""
    from paper_2608_21952_b200 import binding as bd
    c, a, p, dev, x, raw, torch = _token_case(4, 2, 2, 64, 1)
    d, pos, slots = _dims(bd, 2, 1, 2, 64, 64, 1), torch.tensor([3, 0], dtype=torch.int32, device="cuda"), torch.tensor([0, 9], dtype=torch.int32, device="cuda")
    y, state = torch.empty(2, 128, device="cuda"), torch.zeros(2, 2, 64, 64, device="cuda")
    conv = lambda st: bd.ssdi8_conv_fwd(d, x[:, None], dev["w"], dev["bias"], out=torch.empty(2, 1, x.shape[1], dtype=torch.bfloat16, device="cuda"),  # noqa: E731
                                        ring=c.tensors["ring"], slots=slots, pos=pos, status=st)
    calls = {"conv": conv, "write": lambda st: bd.ssdi8_cache_write(d, c, slots, pos, state, status=st),
             "read": lambda st: bd.ssdi8_cache_read(d, c, slots, pos, dev["A"], dev["s_x"], dev["s_B"], state, status=st),
             "token": lambda st: _token(bd, c, dev, x, raw, pos, y, d, slots=slots, status=st)}
    for name, call in calls.items():
        for held, want in ((0, bd.ERR_SHAPE), (bd.ERR_SHAPE, bd.ERR_SHAPE), (bd.ERR_DEVICE_TIMEOUT, bd.ERR_DEVICE_TIMEOUT)):
            status = torch.tensor([held], dtype=torch.int32, device="cuda")
            call(status)
            assert int(status.item()) == want, (name, held)


# ------------------------------------------------------------------------------------------------ the binding
@pytest.mark.gpu
def test_numbers_beyond_32_bits_are_refused():
    """2^32 + 1 groups are not one, nor is a flag or an activation what is left of its low bits"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    x, xq = torch.ones(2, 256, device="cuda"), torch.full((2, 256), 9, dtype=torch.int8, device="cuda")
    sw, out = torch.ones(2, device="cuda"), torch.full((2, 2), 9.0, device="cuda")
    c, a, p, dev, t, raw, _ = _token_case(2, 2, 2, 64, 1)
    pos, y, d = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.full((2, 128), 9.0, device="cuda"), _dims(bd, 2, 1, 2, 64, 64, 1)
    for call in (lambda: bd.ssdi8_norm_quantize(x, xq, groups=2 ** 32 + 1), lambda: bd.ssdi8_linear(xq, xq, sw, out, act=2 ** 32),
                 lambda: _token(bd, c, dev, t, raw, pos, y, d, flags=1 << 32),
                 lambda: bd.ssdi8_conv_fwd(d, t[:, None], dev["w"], out=torch.empty_like(t)[:, None], flags=-(1 << 32))):
        with pytest.raises(OverflowError):
            call()
    assert torch.all(xq == 9) and torch.all(out == 9.0) and torch.all(y == 9.0)
