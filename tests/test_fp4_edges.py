"""Four bits at the edges: forms of the product that a cost decides between, operands that lie otherwise than usual, and numbers that are not finite."""
import pytest

from test_fp4 import _linear, _matrix


@pytest.mark.gpu
@pytest.mark.parametrize("T,O,K", [(1, 640, 8192), (2, 5709, 7488), (5, 300, 2560), (7, 1000, 2560), (33, 640, 8192), (134, 156, 3520)])
def test_parts_of_few_tokens(T, O, K):
    """K shared out among CTAs, each of which has one token of its last four or fewer: every part that is read is one of a token"""
    _linear(T, O, K, 16, "bfloat16", bias=True, residual=True, seed=T + O)


@pytest.mark.gpu
def test_parts_of_few_tokens_in_a_row():
    """the same without a wait between: CTAs that have left are followed by others in their shared memory"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    ops = [(_matrix(T, K, 16, 1)[0], _matrix(O, K, 16, 2)[0], torch.empty(T, O, device="cuda"))
           for T, O, K in ((1, 640, 8192), (64, 2560, 2560), (5, 300, 2560), (134, 156, 3520), (2, 5709, 7488))]
    want = []
    for x, w, out in ops:
        bd.ssdi8_fp4_linear(x, w, out)
        torch.cuda.synchronize()
        want.append(out.clone())
    for _ in range(50):
        for x, w, out in ops:
            bd.ssdi8_fp4_linear(x, w, out)
    torch.cuda.synchronize()
    for (x, w, out), y in zip(ops, want):
        assert torch.equal(out, y)


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["int8", "fp4 16", "fp4 32"])
@pytest.mark.parametrize("rdtype", [None, "float32"])
@pytest.mark.parametrize("T,D", [(5, 96), (7300, 768), (9, 4128)])
def test_norm_of_rows_with_nothing_beside_nan(T, D, rdtype, form):
    """rows of NaN alone, and of NaN and zeros: no absmax, but r is a NaN, and so is the row's step size; rows of zeros keep 1"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    x = torch.randn(T, D, device="cuda").bfloat16()
    x[0] = float("nan")
    x[1], x[1, D - 1] = 0, float("nan")
    x[2] = 0
    x[T - 1], x[T - 1, :32] = 0, float("nan")
    kw = {}
    if rdtype:
        res = torch.where(x.float() == 0, 0.0, torch.randn(T, D, device="cuda"))
        kw = dict(residual=res, residual_out=torch.empty_like(res))
    if form == "int8":
        xq, scale = torch.empty(T, D, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
        bd.ssdi8_add_norm_quantize(x, xq=xq, scale=scale, **kw)
        codes, most = xq, 127
    else:
        q = bd.make_fp4(T, D, int(form[4:]))
        bd.ssdi8_add_norm_quantize(x, fp4=q, **kw)
        b = q.tensors["codes"]
        codes, most, scale = torch.stack([b & 15, b >> 4], -1).view(T, D), 7, q.tensors["step"]
    bad = torch.tensor([0, 1, T - 1], device="cuda")
    assert torch.isnan(scale[bad]).all() and int(torch.isnan(scale).sum()) == 3 and float(scale[2]) == 1.0
    assert torch.equal(codes[bad] == most, torch.isnan(x[bad])) and (codes[bad].int().abs().amax(1) == most).all() and not codes[2].any()
    assert not codes[1, :D - 1].any()


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["static", "int8", "fp4 16", "fp4 32"])
@pytest.mark.parametrize("T,D", [(5, 96), (7300, 768)])
def test_norm_of_zeros_without_eps(T, D, form):
    """a row of zeros, and one whose sum with the residual is, has the codes 0 without an eps too; rows beside it are as ever"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    x = torch.randn(T, D, device="cuda").bfloat16()
    res = torch.randn(T, D, device="cuda").bfloat16()
    x[0], res[0] = 0, -0.0
    x[T - 1] = -res[T - 1]

    def run(eps):
        if form[:3] == "fp4":
            q = bd.make_fp4(T, D, int(form[4:]))
            bd.ssdi8_add_norm_quantize(x, residual=res, eps=eps, fp4=q)
            return q.tensors["codes"], q.tensors["step"]
        xq, scale = torch.empty(T, D, dtype=torch.int8, device="cuda"), torch.ones(T, device="cuda")
        bd.ssdi8_add_norm_quantize(x, residual=res, eps=eps, xq=xq, scale=scale, static_scale=torch.full((1,), 0.05, device="cuda") if form == "static" else None)
        return xq, scale

    (codes, step), (near, _) = run(0.0), run(1e-30)
    assert not codes[0].any() and not codes[T - 1].any() and float(step[0]) == float(step[T - 1]) == 1.0
    assert torch.equal(codes, near)   # (an eps that no other row's mean of squares sees)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("T,O,stride", [(2304, 2560, 0), (2304, 2560, 64), (2304, 2561, 0), (64, 2560, 0), (64, 2560, 8)])
def test_linear_residual_of_rows_that_overlap(T, O, stride, dtype):
    """any stride of the residual's rows: one row for all of them, and rows that begin inside the one before"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    x, w = _matrix(T, 256, 16, 1)[0], _matrix(O, 256, 16, 2)[0]
    flat = torch.randn(T * stride + O, device="cuda").to(getattr(torch, dtype))
    res = flat.as_strided((T, O), (stride, 1))
    out, want = (torch.empty(T, O, dtype=flat.dtype, device="cuda") for _ in range(2))
    bd.ssdi8_fp4_linear(x, w, out, residual=res)
    bd.ssdi8_fp4_linear(x, w, want, residual=res.contiguous())
    assert torch.equal(out, want)


@pytest.mark.gpu
@pytest.mark.parametrize("block,nan", [(16, 127), (32, 255)])
def test_scales_that_are_nan(block, nan):
    """the NaN of a scale's type makes its block's values NaN, and the products that they are in, those of others not"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    T, O, D = 5, 40, 128
    q = _matrix(T, D, block, 3)[0]
    w = _matrix(O, D, block, 4)[0]
    q.tensors["scales"][0, 0, 2, 0, 1] = nan   # row 2, block 1
    bad = torch.zeros(T, D, dtype=torch.bool, device="cuda")
    bad[2, block:2 * block] = True
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.zeros(T, D, dtype=dtype, device="cuda")
        bd.ssdi8_fp4_dequantize(q, out)
        assert torch.equal(torch.isnan(out), bad) and torch.isfinite(out[~bad]).all()
    y = torch.zeros(T, O, device="cuda")
    bd.ssdi8_fp4_linear(q, w, y)
    assert torch.equal(torch.isnan(y), bad.any(1)[:, None].expand(T, O)) and torch.isfinite(y[~bad.any(1)]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("block", [16, 32])
def test_every_scale(block):
    """values of every code under every scale that is a number"""
    import numpy as np
    import torch
    import fp4_reference as ref
    from paper_2608_21952_b200 import binding as bd
    T = 127 if block == 16 else 255
    codes = np.tile(np.arange(32, dtype=np.uint8) % 16, (T, 1))
    scales = np.repeat(np.arange(T, dtype=np.uint8)[:, None], 32 // block, 1)
    q = bd.fp4_of(torch.from_numpy(ref.pack(codes)).cuda(), torch.from_numpy(ref.tile(scales)).cuda(), None, block)
    out = torch.empty(T, 32, device="cuda")
    bd.ssdi8_fp4_dequantize(q, out)
    with np.errstate(over="ignore"):
        np.testing.assert_array_equal(out.cpu().numpy(), ref.values(codes, scales, block).astype(np.float32))


INFINITE = [float("inf"), 3e38, -1e38, 2.0 ** 125, 2.0 ** 124, -2.0 ** 124 * 1.01, 1.0, -float("inf"), 0.0, -0.0]


@pytest.mark.gpu
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("D", [64, 16416])
def test_infinities_beside_the_largest_numbers(block, D):
    """as the header has it.  Blocks of 16: every infinity +6, every number 0, the row's step size infinite.  Blocks of 32: the scale 2^126, an infinity
    6 with its sign, a number what 2^126 leaves of it; other blocks as ever"""
    import numpy as np
    import torch
    import fp4_reference as ref
    from paper_2608_21952_b200 import binding as bd
    x = torch.zeros(3, D, device="cuda")
    x[:, 32:] = torch.randn(3, D - 32, device="cuda")
    n = len(INFINITE)
    x[1, :n] = torch.tensor(INFINITE, device="cuda")
    x[2, :n] = -torch.tensor(INFINITE, device="cuda")
    q, out = bd.make_fp4(3, D, block), torch.empty(3, D, device="cuda")
    bd.ssdi8_fp4_quantize(x, q)
    bd.ssdi8_fp4_dequantize(q, out)
    codes = ref.unpack(q.tensors["codes"].cpu().numpy())
    scales = ref.untile(q.tensors["scales"].cpu().numpy(), 3, D // block)
    step = q.tensors["step"].cpu().numpy()
    got = out.cpu().numpy()
    c, s, g = ref.quantize(x.cpu().numpy(), block)
    np.testing.assert_array_equal(codes, c)
    np.testing.assert_array_equal(scales, s)
    np.testing.assert_array_equal(step, g)
    if block == 16:
        for t in (1, 2):
            inf = np.isinf(x[t].cpu().numpy())
            assert (codes[t][inf] == 7).all() and not codes[t][~inf].any() and (scales[t] == 1).all() and np.isinf(step[t])
            assert (got[t][inf] == np.inf).all() and np.isnan(got[t][~inf]).all()
    else:
        assert codes[1, :n].tolist() == [7, 6, 10, 1, 0, 9, 0, 15, 0, 0] and codes[2, :n].tolist() == [15, 14, 2, 9, 8, 1, 8, 7, 0, 0]
        assert (scales[1:, 0] == 253).all() and (step == 1).all()
        v = np.array([np.inf, np.inf, -2.0 ** 126, 2.0 ** 125, 0, -2.0 ** 125, 0, -np.inf, 0, 0], np.float32)   # (4 x 2^126 is beyond binary32)
        np.testing.assert_array_equal(got[1, :n], v)
        np.testing.assert_array_equal(got[2, :n], -v)
        assert np.isfinite(got[:, 32:]).all()
    assert np.isfinite(got[0]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["int8", "fp4 16", "fp4 32"])
def test_norm_of_rows_with_infinities(form):
    """an infinity in h: r is 0, and the row's values are NaN, or 0 where a step size of 0 meets a number"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    T, D = 4, 128
    x = torch.randn(T, D, device="cuda")
    x[1, 3] = float("inf")
    x[2, 5], x[2, 70] = -float("inf"), float("inf")
    if form == "int8":
        xq, scale = torch.empty(T, D, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
        bd.ssdi8_add_norm_quantize(x, xq=xq, scale=scale)
        inf = torch.isinf(x[1:3])
        assert (xq[1:3][inf] == 127).all() and not xq[1:3][~inf].any()
        assert torch.isnan(scale[1:3]).all() and torch.isfinite(scale[[0, 3]]).all()
        return
    q, out = bd.make_fp4(T, D, int(form[4:])), torch.empty(T, D, device="cuda")
    bd.ssdi8_add_norm_quantize(x, fp4=q)
    bd.ssdi8_fp4_dequantize(q, out)
    assert torch.isfinite(out[[0, 3]]).all() and torch.isnan(out[1:3][torch.isinf(x[1:3])]).all()
    step = q.tensors["step"][1:3]
    assert torch.isnan(step).all() if form == "fp4 16" else not step.any()
    assert torch.isnan(out[1:3]).all() if form == "fp4 16" else not out[1:3][~torch.isinf(x[1:3])].any()


def _device_check(T, O, K, block, rows=None, outs=None, dtype=None):
    """a product against binary64 on the device, some rows and outputs of it"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    g = torch.Generator(device="cuda").manual_seed(T + O)

    def matrix(n):
        q = bd.make_fp4(n, K, block)
        q.tensors["codes"].copy_(torch.randint(0, 256, (n, K // 2), generator=g, device="cuda", dtype=torch.uint8))
        lo, hi = (60, 127) if block == 16 else (120, 132)
        s = q.tensors["scales"]
        s.copy_(torch.randint(lo, hi, s.shape, generator=g, device="cuda", dtype=torch.uint8))
        return q
    x, w = matrix(T), matrix(O)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full((T + 1, O), 77.0, dtype=dtype or torch.float32, device="cuda")
    bd.ssdi8_fp4_linear(x, w, out[:T], status=status)
    assert int(status.item()) == 0 and (out[T] == 77).all()

    def values(q, n, at):
        v = torch.empty(n, K, device="cuda")
        bd.ssdi8_fp4_dequantize(q, v)
        return v[at].double()
    tr = torch.arange(T, device="cuda") if rows is None else torch.cat([torch.arange(rows, device="cuda"), torch.arange(T - rows, T, device="cuda")])
    oc = torch.arange(O, device="cuda") if outs is None else torch.cat([torch.arange(outs, device="cuda"), torch.arange(O - outs, O, device="cuda")])
    vx, vw = values(x, T, tr), values(w, O, oc)
    want, size = vx @ vw.T, vx.abs() @ vw.abs().T
    got = out[tr][:, oc].double()
    # K roundings of the sum of magnitudes, the result's own (bf16: half a step of 2^-7)
    tol = K * 2.0 ** -24 * size
    tol = tol + (2.0 ** -24 if dtype is None else 2.0 ** -8) * (want.abs() + tol)
    assert bool(((got - want).abs() <= tol).all())


@pytest.mark.gpu
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("T,O", [(3, 130), (300, 129), (600, 1000)])
def test_linear_of_the_widest_rows(T, O, block):
    _device_check(T, O, 131072, block)


@pytest.mark.gpu
@pytest.mark.parametrize("T,O,K", [(1, 1 << 21, 64), ((1 << 21) + 5, 9, 32), (2, (1 << 20) + 3, 96)])
def test_linear_of_one_long_side(T, O, K):
    """one token and millions of outputs, millions of tokens and a few outputs"""
    import torch
    _device_check(T, O, K, 16, rows=min(T, 700) if T > 700 else None, outs=700 if O > 700 else None, dtype=torch.bfloat16)


@pytest.mark.gpu
@pytest.mark.parametrize("block", [16, 32])
def test_linear_of_slices(block):
    """rows of a matrix from a multiple of 128 on are a matrix: a weight's shards, a batch's parts"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    T, O, K = 300, 700, 544
    x, w = _matrix(T, K, block, 1)[0], _matrix(O, K, block, 2)[0]

    def part(q, a, b):
        t = q.tensors
        return bd.fp4_of(t["codes"][a:b], t["scales"][a // 128:], t["step"][a:b], block)
    whole, out = torch.empty(T, O, device="cuda"), torch.full((T, O), 77.0, device="cuda")
    values = torch.empty(T, K, device="cuda")
    bd.ssdi8_fp4_linear(x, w, whole)
    for a, b in ((0, 128), (128, 300)):
        for c, d in ((0, 384), (384, 700)):
            bd.ssdi8_fp4_linear(part(x, a, b), part(w, c, d), out[a:b, c:d])
    # (forms differ, and with them the order of sums)
    vx, vw = torch.empty(T, K, device="cuda"), torch.empty(O, K, device="cuda")
    bd.ssdi8_fp4_dequantize(x, vx)
    bd.ssdi8_fp4_dequantize(w, vw)
    assert bool(((whole - out).abs() <= (2 * K + 8) * 2.0 ** -24 * (vx.abs() @ vw.abs().T)).all())
    for a, b in ((0, 128), (128, 300)):
        bd.ssdi8_fp4_dequantize(part(x, a, b), values[a:b])
    assert torch.equal(values, vx)


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["int8", "static"])
def test_norm_of_the_narrowest_rows(form):
    from test_fp4 import test_add_norm
    for T in (1, 9471, 9473, 20000):
        test_add_norm(T, 16, "bfloat16", "float32", "normal", 0, form)


@pytest.mark.gpu
def test_four_and_eight_bits_on_two_streams():
    """products of both kinds beside one another, whose tensor memory and clusters share the SMs"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    ops = [[], []]
    for i, (T, O, K) in enumerate(((64, 2560, 5120), (1, 640, 8192), (134, 156, 3520), (300, 1000, 1024), (2304, 2560, 512), (100, 600, 2560))):
        x, w, out = _matrix(T, K, 16, i)[0], _matrix(O, K, 16, i + 9)[0], torch.empty(T, O, device="cuda")
        ops[0].append((lambda st, x=x, w=w, out=out: bd.ssdi8_fp4_linear(x, w, out, stream=st), out))
        a, b = (torch.randint(-127, 128, s, dtype=torch.int8, device="cuda") for s in ((T, K), (O, K)))
        s, y = torch.rand(O, device="cuda"), torch.empty(T, O, device="cuda")
        ops[1].append((lambda st, a=a, b=b, s=s, y=y: bd.ssdi8_linear(a, b, s, y, stream=st), y))
    want = []
    for side in ops:
        for f, out in side:
            f(None)
            torch.cuda.synchronize()
            want.append(out.clone())
    streams = [torch.cuda.Stream() for _ in range(2)]
    for shift in range(12):
        for side in ops:
            for _, out in side:
                out.zero_()
        torch.cuda.synchronize()
        for i in range(len(ops[0])):
            ops[0][i][0](streams[0])
            ops[1][(i + shift) % len(ops[1])][0](streams[1])
        torch.cuda.synchronize()
        for (_, out), y in zip(ops[0] + ops[1], want):
            assert torch.equal(out, y)
