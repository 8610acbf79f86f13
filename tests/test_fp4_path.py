"""The input projection in four bits in a Mamba-2 block: the residual stream in fp32, its addition and norm ending in four bits, the product, and behind it
convolution, chunk scan, gated norm and int8 output projection; ragged prompts through two layers, then tokens, captured and not.  Every stage is
checked against its definition on what the stage before gave."""
import numpy as np
import pytest

import fp4_reference as f4
from test_block_path import CH, DM, H, HP, N, G, ROW, Block, _np


class Fp4Block(Block):
    def __init__(self, seed, block):
        super().__init__(seed)
        from paper_2608_21952_b200 import binding as bd
        self.block = block
        w = (self.rng.standard_normal((ROW, DM)) / np.sqrt(DM)).astype(np.float32)
        self.w4 = bd.make_fp4(ROW, DM, block)
        bd.ssdi8_fp4_quantize(self.t(w), self.w4)
        c, s, g = f4.quantize(w, block)
        np.testing.assert_array_equal(f4.unpack(_np(self.w4.tensors["codes"])), c)
        self.w4v = f4.values(c, s, block) * g[:, None].astype(np.float64)

    def project_in4(self, x, stream):
        """the block before's output x [T, DM] bf16 onto the stream (fp32, in place) -> rows [T, ROW] bf16"""
        from paper_2608_21952_b200 import binding as bd
        torch, T = self.torch, x.shape[0]
        q, rows = bd.make_fp4(T, DM, self.block), torch.empty(T, ROW, dtype=torch.bfloat16, device="cuda")
        h = (_np(x) + _np(stream)).astype(np.float32)
        bd.ssdi8_add_norm_quantize(x, residual=stream, residual_out=stream, weight=self.dev["n1"], fp4=q)
        bd.ssdi8_fp4_linear(q, self.w4, rows)
        np.testing.assert_array_equal(_np(stream), h)
        c, s, g = f4.quantize((h * self.n1).astype(np.float32), self.block)
        np.testing.assert_array_equal(f4.unpack(_np(q.tensors["codes"])), c)
        step = _np(q.tensors["step"]).astype(np.float64)
        np.testing.assert_allclose(step, g * f4.factor(h, 1e-5), rtol=2.0 ** -24 + 1e-14)
        v = f4.values(c, s, self.block) * step[:, None]
        want = v @ self.w4v.T
        # the sum's roundings, two products, the row's own rounding to bf16
        tol = (DM + 3) * 2.0 ** -24 * (np.abs(v) @ np.abs(self.w4v).T)
        assert np.all(np.abs(_np(rows) - want) <= tol + 2.0 ** -8 * (np.abs(want) + tol))
        return rows

    def project_out8(self, y, rows):
        """scan output and the gate in the rows -> the block's output, bf16 (the next one's norm adds it to the stream)"""
        from paper_2608_21952_b200 import binding as bd
        torch, T = self.torch, y.shape[0]
        yq, sc, out = torch.empty(T, HP, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, DM, dtype=torch.bfloat16, device="cuda")
        bd.ssdi8_norm_quantize(y, yq, weight=self.dev["n2"], z=rows[:, :HP], scale=sc)
        bd.ssdi8_linear(yq, self.dev["w_out"], self.dev["s_out"], out, s_row=sc, bias=self.dev["c_out"])
        want = (_np(yq).astype(np.float64) @ self.w_out.astype(np.float64).T) * _np(sc)[:, None] * self.s_out + self.c_out
        assert np.all(np.abs(_np(out) - want) <= 2.0 ** -8 * np.abs(want) + 1e-6)
        return out


@pytest.mark.gpu
@pytest.mark.parametrize("block", [16, 32])
def test_two_layers_on_ragged_prompts_and_their_tokens(block):
    torch = pytest.importorskip("torch")
    from paper_2608_21952_b200 import binding as bd
    layers = [Fp4Block(11, block), Fp4Block(12, block)]
    B, L, nslots = 3, 128, 5
    lens, slots = np.array([100, 128, 1], np.int32), np.array([3, 0, 2], np.int32)
    m = layers[0]
    one = bd.Dims(B, 1, H, 64, N, G, 0)
    caches = [bd.make_cache(one, nslots) for _ in layers]
    x = m.t(m.rng.standard_normal((B * L, DM)).astype(np.float32)).to(torch.bfloat16)
    stream = torch.zeros(B * L, DM, device="cuda")
    for m, cache in zip(layers, caches):
        rows = m.project_in4(x, stream)
        o = m.convolve(rows.view(B, L, ROW), lens, np.zeros(B, np.int32), slots, cache.tensors["ring"])
        m.calibrate(o)
        y, fin = m.scan(o)
        bd.ssdi8_cache_write(one, cache, m.t(slots), m.t(lens), fin)
        x = m.project_out8(y.view(B * L, HP), rows)
    pos = lens.copy()
    for step in range(3):
        x = m.t(m.rng.standard_normal((B, DM)).astype(np.float32)).to(torch.bfloat16)
        stream = torch.zeros(B, DM, device="cuda")
        for m, cache in zip(layers, caches):
            rows, d = m.project_in4(x, stream), m.dev
            y = torch.empty(B, HP, device="cuda")
            bd.ssdi8_token_step(one, cache, rows[:, HP:HP + CH], d["w"], d["bias"], rows[:, HP + CH:], d["dt_bias"], d["A"], d["D"], None, d["s_x"], d["s_B"],
                                d["s_C"], m.t(slots), m.t(pos), y, flags=bd.FLAG_DT_SOFTPLUS)
            x = m.project_out8(y, rows)
        pos = pos + 1
    # the last norm, ahead of a head: int8 codes, and the stream ends here
    h = (_np(x) + _np(stream)).astype(np.float32)
    xq, sc = torch.empty(B, DM, dtype=torch.int8, device="cuda"), torch.empty(B, device="cuda")
    bd.ssdi8_add_norm_quantize(x, residual=stream, weight=m.dev["n1"], xq=xq, scale=sc)
    p = (h * m.n1).astype(np.float32)
    np.testing.assert_array_equal(_np(xq), f4.int8_codes(p, (np.abs(p).max(-1) / np.float32(127))[:, None]))


@pytest.mark.gpu
def test_a_decode_step_with_four_bits_in_one_graph():
    """captured once and replayed: the same as called one by one"""
    torch = pytest.importorskip("torch")
    from paper_2608_21952_b200 import binding as bd
    m = Fp4Block(13, 16)
    B = 5
    dims, d = bd.Dims(B, 1, H, 64, N, G, 0), m.dev
    e = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    x0 = m.t(m.rng.standard_normal((20, B, DM)).astype(np.float32)).to(torch.bfloat16)

    class Run:
        def __init__(self):
            self.cache, self.pos = bd.make_cache(dims, B), torch.arange(B, dtype=torch.int32, device="cuda")
            self.x, self.stream, self.q = e(B, DM, dtype=torch.bfloat16), torch.zeros(B, DM, device="cuda"), bd.make_fp4(B, DM)
            self.rows, self.y, self.yq, self.sc = e(B, ROW, dtype=torch.bfloat16), e(B, HP, dtype=torch.bfloat16), e(B, HP, dtype=torch.int8), e(B)

        def step(self):
            bd.ssdi8_add_norm_quantize(self.x, residual=self.stream, residual_out=self.stream, weight=d["n1"], fp4=self.q)
            bd.ssdi8_fp4_linear(self.q, m.w4, self.rows)
            bd.ssdi8_token_step(dims, self.cache, self.rows[:, HP:HP + CH], d["w"], d["bias"], self.rows[:, HP + CH:], d["dt_bias"], d["A"], d["D"],
                                None, d["s_x"], d["s_B"], d["s_C"], None, self.pos, self.y, flags=bd.FLAG_DT_SOFTPLUS)
            bd.ssdi8_norm_quantize(self.y, self.yq, weight=d["n2"], z=self.rows[:, :HP], scale=self.sc)
            bd.ssdi8_linear(self.yq, d["w_out"], d["s_out"], self.x, s_row=self.sc, bias=d["c_out"])
            self.pos += 1

    eager, warm, captured = Run(), Run(), Run()
    warm.x.copy_(x0[0])
    warm.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.step()
    captured.pos.copy_(torch.arange(B))
    captured.stream.zero_()
    for i in range(20):
        eager.x.copy_(x0[i])
        captured.x.copy_(x0[i])
        graph.replay()
        eager.step()
        assert torch.equal(eager.x, captured.x) and torch.equal(eager.stream, captured.stream), i
    for k in eager.cache.tensors:
        assert torch.equal(eager.cache.tensors[k], captured.cache.tensors[k]), k
