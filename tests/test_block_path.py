"""The operators around the layer together, as a Mamba-2 block runs them: projection, convolution, chunk scan, norm and projection for
ragged prompts, states into the 8-bit cache, token steps on it, states back out for another prompt.  Every stage is checked against its
definition on what the stage before gave; the cache's own error is held to the half steps that its roundings can cost."""
import math

import numpy as np
import pytest

import block_reference as ref

H, N, G, W, DM, Q = 4, 64, 2, 4, 128, 64      # heads, state, groups, taps, model width, chunk
HP, GN = 64 * H, G * N
CH, ROW = HP + 2 * GN, 2 * HP + 2 * GN + H    # convolved channels; rows of the input projection: z, xBC, dt


def _np(t):
    import torch
    return (t.float() if t.dtype in (torch.bfloat16, torch.float16) else t).detach().cpu().numpy()


class Block:
    """weights and static step sizes of one block (the internal step sizes of the scan calibrated on the prompt)"""

    def __init__(self, seed):
        import torch
        self.torch, self.rng = torch, np.random.default_rng(seed)
        r = self.rng
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        f = lambda *s: r.standard_normal(s).astype(np.float32)  # noqa: E731
        code = lambda *s: np.clip(np.rint(r.standard_normal(s) * 40), -127, 127).astype(np.int8)  # noqa: E731
        self.n1, self.n2 = r.uniform(0.5, 1.5, DM).astype(np.float32), r.uniform(0.5, 1.5, HP).astype(np.float32)
        self.w_in, self.w_out = code(ROW, DM), code(DM, HP)
        self.s_in = (r.uniform(0.5, 1.5, ROW) / (40 * math.sqrt(DM))).astype(np.float32)
        self.s_out = (r.uniform(0.5, 1.5, DM) / (40 * math.sqrt(HP))).astype(np.float32)
        self.c_out = 0.1 * f(DM)      # mean correction at the output projection
        self.w, self.bias = r.uniform(-0.5, 0.5, (CH, W)).astype(np.float32), 0.1 * f(CH)
        self.dt_bias, self.D = (-3 + 0.25 * f(H)).astype(np.float32), f(H)
        self.A = -np.exp(r.uniform(0, math.log(16), H)).astype(np.float32)
        self.s_x = (3.0 / 127 * np.sqrt((self.w[:HP] ** 2).sum(1) + 0.01)).astype(np.float32)
        self.s_B, self.s_C = np.full(G, 2 / 127, np.float32), np.full(G, 2 / 127, np.float32)
        self.dev = {k: t(v) for k, v in self.__dict__.items() if isinstance(v, np.ndarray)}
        self.t = t

    def project_in(self, x):
        """residual stream [T, DM] bf16 -> rows [T, ROW] bf16; checks norm codes and the projection"""
        from paper_2608_21952_b200 import binding as bd
        torch, T = self.torch, x.shape[0]
        xq, sc = torch.empty(T, DM, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
        rows = torch.empty(T, ROW, dtype=torch.bfloat16, device="cuda")
        bd.ssdi8_norm_quantize(x, xq, weight=self.dev["n1"], scale=sc)
        bd.ssdi8_linear(xq, self.dev["w_in"], self.dev["s_in"], rows, s_row=sc)
        codes, _ = ref.norm_codes(_np(x), None, self.n1, 1, 1e-5)
        np.testing.assert_array_equal(_np(xq), codes)
        want = (codes.astype(np.float64) @ self.w_in.astype(np.float64).T) * _np(sc)[:, None] * self.s_in
        assert np.all(np.abs(_np(rows) - want) <= 2.0 ** -8 * np.abs(want) + 1e-6)
        return rows

    def project_out(self, y, rows, x):
        """scan output [T, HP] and the gate in the rows -> new residual stream, in place of x"""
        from paper_2608_21952_b200 import binding as bd
        torch, T = self.torch, x.shape[0]
        yq, sc, z = torch.empty(T, HP, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda"), rows[:, :HP]
        before = _np(x)
        bd.ssdi8_norm_quantize(y, yq, weight=self.dev["n2"], z=z, scale=sc)
        bd.ssdi8_linear(yq, self.dev["w_out"], self.dev["s_out"], x, s_row=sc, bias=self.dev["c_out"], residual=x)
        codes, _ = ref.norm_codes(_np(y), _np(z), self.n2, 1, 1e-5)
        np.testing.assert_array_equal(_np(yq), codes)
        want = (codes.astype(np.float64) @ self.w_out.astype(np.float64).T) * _np(sc)[:, None] * self.s_out + self.c_out + before
        assert np.all(np.abs(_np(x) - want) <= 2.0 ** -8 * np.abs(want) + 1e-6 * (1 + np.abs(before)))

    def convolve(self, rows, lens, pos, slots, ring):
        from paper_2608_21952_b200 import binding as bd
        torch, (B, L, _) = self.torch, rows.shape
        o = {k: torch.empty(B, L, n, dtype=torch.int8, device="cuda") for k, n in (("xq", HP), ("Bq", GN), ("Cq", GN))}
        o["dt"] = torch.empty(B, L, H, device="cuda")
        before = _np(ring).copy()
        d = self.dev
        bd.ssdi8_conv_fwd(bd.Dims(B, L, H, 64, N, G, Q), rows[..., HP:HP + CH], d["w"], d["bias"], s_x=d["s_x"], s_B=d["s_B"], s_C=d["s_C"],
                          dt_raw=rows[..., HP + CH:], dt_bias=d["dt_bias"], lens=self.t(lens), pos=self.t(pos), slots=self.t(slots), ring=ring,
                          flags=bd.FLAG_DT_SOFTPLUS, **o)
        u = ref.conv(_np(rows[..., HP:HP + CH]), self.w, self.bias, lens, before, slots, pos)
        np.testing.assert_array_equal(_np(ring), before)
        np.testing.assert_array_equal(_np(o["xq"]), ref.code(u[..., :HP] / self.s_x.astype(np.float64)))
        np.testing.assert_array_equal(_np(o["Cq"]), ref.code(u[..., HP + GN:] / np.repeat(self.s_C.astype(np.float64), N)))
        return o

    def calibrate(self, o):
        from paper_2608_21952_b200 import binding as bd
        torch, (B, L, _) = self.torch, o["xq"].shape
        d = bd.Dims(B, L, H, 64, N, G, Q)
        self.internal = {"s_xs": torch.empty(HP, device="cuda"), "s_cb": torch.empty(G, device="cuda"), "s_h": torch.empty(HP, device="cuda")}
        args = bd.make_fwd_args(A=self.dev["A"], s_x=self.dev["s_x"], s_B=self.dev["s_B"], s_C=self.dev["s_C"], **o)
        bd.ssdi8_calibrate(d, args, *(self.internal[k] for k in ("s_xs", "s_cb", "s_h")), bd.alloc_workspace(d))

    def scan(self, o, init=None):
        from paper_2608_21952_b200 import binding as bd
        torch, (B, L, _) = self.torch, o["xq"].shape
        d = bd.Dims(B, L, H, 64, N, G, Q)
        y, fin = torch.empty(B, L, HP, device="cuda"), torch.empty(B, H, 64, N, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        args = bd.make_fwd_args(y=y, final_state=fin, status=status, init_state=init, A=self.dev["A"], D=self.dev["D"], s_x=self.dev["s_x"],
                                s_B=self.dev["s_B"], s_C=self.dev["s_C"], **o, **self.internal)
        bd.ssdi8_chunk_scan_fwd(d, args, bd.alloc_workspace(d))
        assert int(status.item()) == 0
        return y, fin


@pytest.mark.gpu
def test_a_block_on_ragged_prompts_and_the_tokens_after_them():
    torch = pytest.importorskip("torch")
    from paper_2608_21952_b200 import binding as bd
    m = Block(1)
    B, L, nslots = 3, 192, 6
    lens, slots = np.array([150, 192, 1], np.int32), np.array([4, 0, 2], np.int32)
    x = m.t(m.rng.standard_normal((B * L, DM)).astype(np.float32)).to(torch.bfloat16)
    one = bd.Dims(B, 1, H, 64, N, G, 0)
    cache = bd.make_cache(one, nslots)
    # ---- the prompts
    rows = m.project_in(x)
    o = m.convolve(rows.view(B, L, ROW), lens, np.zeros(B, np.int32), slots, cache.tensors["ring"])
    m.calibrate(o)
    y, fin = m.scan(o)
    for b in range(B):   # tokens behind a prompt leave no trace
        assert torch.all(y[b, lens[b]:] == 0) and torch.all(o["dt"][b, lens[b]:] == 0)
    longer = {k: torch.cat([v, torch.zeros_like(v[:, :2 * Q])], 1) for k, v in o.items()}
    y2, fin2 = m.scan(longer)
    assert torch.equal(fin, fin2) and torch.equal(y, y2[:, :L])
    m.project_out(y.view(B * L, HP), rows, x)
    # ---- into the cache, and 40 tokens each
    bd.ssdi8_cache_write(one, cache, m.t(slots), m.t(lens), fin)
    t = {k: _np(v).copy() for k, v in cache.tensors.items()}
    s = ref.Slots(t, m.A, m.s_x, m.s_B, m.s_C, m.D)
    state, pos = fin.clone(), lens.copy()
    delta = t["scales"][slots].astype(np.float64) * 0.5   # [B, H, P]: how far the cache's state may be from the fp32 one
    d = m.dev
    for step in range(40):
        x = m.t(m.rng.standard_normal((B, DM)).astype(np.float32)).to(torch.bfloat16)
        rows = m.project_in(x)
        xBC, raw = rows[:, HP:HP + CH], rows[:, HP + CH:]
        u = ref.conv(_np(xBC)[:, None], m.w, m.bias, None, t["ring"].copy(), slots, pos)[:, 0]
        y = torch.empty(B, HP, device="cuda")
        bd.ssdi8_token_step(one, cache, xBC, d["w"], d["bias"], raw, d["dt_bias"], d["A"], d["D"], None, d["s_x"], d["s_B"], d["s_C"], m.t(slots),
                            m.t(pos), y, flags=bd.FLAG_DT_SOFTPLUS)
        dt = np.stack([_np(cache.tensors["dtwin"])[slots[b], :, pos[b] % 16] for b in range(B)])
        want = np.zeros((B, HP))
        bound = s.step(u, dt, slots, pos, _np(xBC), want)
        for k in ("codes", "scales", "xwin", "Bwin", "ring", "start"):
            np.testing.assert_array_equal(_np(cache.tensors[k]), t[k], err_msg=k)
        assert np.all(np.abs(_np(y) - want) <= bound)
        # against the recurrence on an fp32 state: what half a step of every code can do
        xq = m.t(ref.code(u[:, :HP] / m.s_x.astype(np.float64)))
        Bq, Cq = (ref.code(u[:, HP + i * GN:HP + (i + 1) * GN].reshape(B, G, N) / np.float64(np.float32(2 / 127))) for i in (0, 1))
        y32 = torch.empty(B, HP, device="cuda")
        bd.ssdi8_ssd_step(one, xq, d["s_x"], m.t(Bq), d["s_B"], m.t(Cq), d["s_C"], m.t(dt), d["A"], d["D"], None, state, y32)
        decay = np.exp(dt.astype(np.float64) * m.A)[..., None]
        delta = delta * decay
        reach = np.repeat(np.abs(Cq.astype(np.float64)).sum(-1) * m.s_C, H // G, 1)[..., None] * delta
        assert np.all(np.abs(_np(y) - _np(y32)) <= reach.reshape(B, HP) + bound + 1e-5 * (1 + np.abs(want)))
        for b in range(B):
            if pos[b] % 16 == 15:
                delta[b] += t["scales"][slots[b]].astype(np.float64) * 0.5
        m.project_out(y, rows, x)
        pos = pos + 1
    # ---- back out, for another prompt that goes on from there
    back = torch.empty_like(fin)
    bd.ssdi8_cache_read(one, cache, m.t(slots), m.t(pos), d["A"], d["s_x"], d["s_B"], back)
    assert np.all(np.abs(_np(back) - _np(state)) <= delta[..., None] + 1e-5 * (1 + np.abs(_np(state))))
    x = m.t(m.rng.standard_normal((B * Q, DM)).astype(np.float32)).to(torch.bfloat16)
    rows = m.project_in(x)
    o = m.convolve(rows.view(B, Q, ROW), np.full(B, Q, np.int32), pos, slots, cache.tensors["ring"])
    y, fin = m.scan(o, back)
    m.project_out(y.view(B * Q, HP), rows, x)
    # the scan went on from that state: the recurrence over the same codes, within what Q(X_scaled) loses at each token: half a step, or
    # what lies beyond the last code (its step sizes are those of the first prompts)
    S = _np(back).astype(np.float64)
    xh, Bh = _np(o["xq"]).reshape(B, Q, H, 64) * m.s_x.reshape(H, 64).astype(np.float64), _np(o["Bq"]).reshape(B, Q, G, N) * m.s_B[:, None].astype(np.float64)
    dt, s_xs = _np(o["dt"]).astype(np.float64), _np(m.internal["s_xs"]).reshape(1, H, 64).astype(np.float64)
    half = np.zeros_like(S)
    for i in range(Q):
        Bi = np.repeat(Bh[:, i], H // G, 1)[:, :, None]
        S = np.exp(dt[:, i] * m.A)[..., None, None] * S + (dt[:, i, :, None] * xh[:, i])[..., None] * Bi
        scaled = np.abs((dt[:, i] * np.exp(m.A * dt[:, i + 1:].sum(1)))[..., None] * xh[:, i])
        half += np.maximum(0.5 * s_xs, scaled - 127 * s_xs)[..., None] * np.abs(Bi)
    over = np.abs(_np(fin) - S) - half * 1.001 - 1e-4 * (1 + np.abs(S))
    assert over.max() <= 0


@pytest.mark.gpu
def test_a_decode_step_of_the_block_in_one_graph():
    """norm, projection, token step, norm and projection captured once and replayed: the same as called one by one"""
    torch = pytest.importorskip("torch")
    from paper_2608_21952_b200 import binding as bd
    m = Block(2)
    B = 5
    dims, d = bd.Dims(B, 1, H, 64, N, G, 0), m.dev
    e = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    x0 = m.t(m.rng.standard_normal((20, B, DM)).astype(np.float32)).to(torch.bfloat16)

    class Run:
        def __init__(self):
            self.cache, self.pos = bd.make_cache(dims, B), torch.arange(B, dtype=torch.int32, device="cuda")
            self.x, self.xq, self.sc, self.rows = e(B, DM, dtype=torch.bfloat16), e(B, DM, dtype=torch.int8), e(B), e(B, ROW, dtype=torch.bfloat16)
            self.y, self.yq = e(B, HP, dtype=torch.bfloat16), e(B, HP, dtype=torch.int8)

        def step(self):
            bd.ssdi8_norm_quantize(self.x, self.xq, weight=d["n1"], scale=self.sc)
            bd.ssdi8_linear(self.xq, d["w_in"], d["s_in"], self.rows, s_row=self.sc)
            bd.ssdi8_token_step(dims, self.cache, self.rows[:, HP:HP + CH], d["w"], d["bias"], self.rows[:, HP + CH:], d["dt_bias"], d["A"], d["D"],
                                None, d["s_x"], d["s_B"], d["s_C"], None, self.pos, self.y, flags=bd.FLAG_DT_SOFTPLUS)
            bd.ssdi8_norm_quantize(self.y, self.yq, weight=d["n2"], z=self.rows[:, :HP], scale=self.sc)
            bd.ssdi8_linear(self.yq, d["w_out"], d["s_out"], self.x, s_row=self.sc, bias=d["c_out"], residual=self.x)
            self.pos += 1

    eager, warm, captured = Run(), Run(), Run()
    warm.x.copy_(x0[0])
    warm.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.step()
    captured.pos.copy_(torch.arange(B))
    for i in range(20):
        eager.x.copy_(x0[i])
        captured.x.copy_(x0[i])
        eager.step()
        graph.replay()
        assert torch.equal(eager.x, captured.x), i
    for k in eager.cache.tensors:
        assert torch.equal(eager.cache.tensors[k], captured.cache.tensors[k]), k
