"""The operators around the layer from their definitions, in 64 bits and token by token (numpy, tests only)."""
import numpy as np

WINDOW = 16


def silu(v):
    with np.errstate(over="ignore", invalid="ignore"):
        return v / (1.0 + np.exp(-v))


def softplus(v):
    return np.logaddexp(0.0, v)


def code(q):
    """nearest integer, ties to even, saturated; NaN has the code +127"""
    q = np.where(np.isnan(q), 127.0, np.clip(q, -127, 127))
    return np.rint(q).astype(np.int8)


def conv(x, weight, bias, lens, ring, slots, pos):
    """x [B, L, Ch]; ring [nslots, W, Ch] is changed in place.  SiLU of the convolution (0 behind lens)."""
    B, L, Ch = x.shape
    W = weight.shape[1]
    w = weight.astype(np.float64)
    u = np.zeros((B, L, Ch))
    for b in range(B):
        n = L if lens is None else int(np.clip(lens[b], 0, L))
        p, s = (0 if pos is None else int(pos[b])), (b if slots is None else int(slots[b]))
        if ring is not None and (s < 0 or s >= ring.shape[0] or p < 0 or (slots is not None and s in slots[:b])):
            continue
        history = []
        for t in range(-(W - 1), 0):
            at = p + t
            history.append(ring[s, at % W].astype(np.float64) if ring is not None and at >= 0 else np.zeros(Ch))
        tokens = np.concatenate([np.stack(history), x[b, :n].astype(np.float64)])
        with np.errstate(invalid="ignore"):
            for t in range(n):
                v = (w.T * tokens[t:t + W]).sum(0)
                u[b, t] = silu(v if bias is None else v + bias)
        if ring is not None:
            for t in range(max(0, n - W), n):
                ring[s, (p + t) % W] = x[b, t]
    return u


class Slots:
    """The 8-bit state cache and the token step from their definitions, in 64 bits.  `t`: the cache's arrays by name."""

    def __init__(self, t, A, s_x, s_B, s_C=None, D=None, corr=None):
        f = lambda v: None if v is None else np.asarray(v, np.float64)  # noqa: E731
        self.t, self.A, self.s_x, self.s_B, self.s_C, self.D, self.corr = t, f(A), f(s_x), f(s_B), f(s_C), f(D), f(corr)
        self.n, self.H, self.P, self.N = t["codes"].shape
        self.G = t["Bwin"].shape[1]
        self.group = np.arange(self.H) // (self.H // self.G)

    def valid(self, slots, pos, b):
        s = b if slots is None else int(slots[b])
        return 0 <= s < self.n and pos[b] >= 0 and not (slots is not None and s in slots[:b])

    def terms(self, slot, tokens):
        """decay of the codes and the weight of each waiting token, per head; and the exponents' magnitudes"""
        dt = np.array([self.t["dtwin"][slot, :, j % WINDOW].astype(np.float64) for j in tokens]).reshape(len(tokens), self.H)
        behind = dt.sum(0) - np.cumsum(dt, 0)
        return np.exp(self.A * dt.sum(0)), dt * np.exp(self.A * behind), np.abs(self.A) * dt.sum(0)

    def state(self, slot, tokens):
        """[H, P, N] with the waiting tokens, and the sum of the magnitudes of its terms"""
        E, w, _ = self.terms(slot, tokens)
        base = E[:, None, None] * self.t["scales"][slot].astype(np.float64)[..., None] * self.t["codes"][slot]
        S, size = base, np.abs(base)
        for i, j in enumerate(tokens):
            x = self.s_x.reshape(self.H, self.P) * self.t["xwin"][slot, :, j % WINDOW]
            B = (self.s_B[:, None] * self.t["Bwin"][slot, :, j % WINDOW])[self.group]
            add = w[i][:, None, None] * x[..., None] * B[:, None]
            S, size = S + add, size + np.abs(add)
        return S, size

    def write(self, slots, pos, state):
        for b in range(state.shape[0]):
            p = np.zeros(state.shape[0], int) if pos is None else pos
            if not self.valid(slots, p, b):
                continue
            s = b if slots is None else int(slots[b])
            with np.errstate(all="ignore"):
                top = np.fmax.reduce(np.abs(state[b]), -1)
                top = np.where(np.isnan(top), np.float32(0), top)
                step = (top / np.float32(127)).astype(np.float32)
                step[step == 0] = 1
                q = (state[b] / step[..., None]).astype(np.float32)
            self.t["codes"][s], self.t["scales"][s], self.t["start"][s] = code(q), step, p[b]

    def step(self, u, dt, slots, pos, xBC, y):
        """u [B, Ch]: SiLU of the convolution (64 bits); dt [B, H] fp32; xBC raw rows.  y [B, H * P] (64 bits) is changed; returns
        the bound of binary32's error of y: the sum over the terms of (32 + |exponent|) 2^-24 of each (the exponential 4, its
        argument |exponent|, the products and sums below 16, the epilogue 4)."""
        bound = np.zeros_like(y)
        HP, GN = self.H * self.P, self.G * self.N
        sx = self.s_x.reshape(self.H, self.P)
        for b in range(u.shape[0]):
            s, p = (b if slots is None else int(slots[b])), int(pos[b])
            if not self.valid(slots, pos, b):
                continue
            first = max(int(self.t["start"][s]), p - p % WINDOW)
            if first > p:
                continue
            x = code(u[b, :HP] / self.s_x).reshape(self.H, self.P)
            B = code(u[b, HP:HP + GN].reshape(self.G, self.N) / self.s_B[:, None])
            Cq = code(u[b, HP + GN:].reshape(self.G, self.N) / self.s_C[:, None])
            self.t["ring"][s, p % self.t["ring"].shape[1]] = xBC[b]
            self.t["xwin"][s, :, p % WINDOW], self.t["Bwin"][s, :, p % WINDOW] = x, B
            self.t["dtwin"][s, :, p % WINDOW] = dt[b]
            tokens = list(range(first, p + 1))
            E, w, exponent = self.terms(s, tokens)
            Ch = Cq.astype(np.float64)[self.group]
            part = E[:, None] * self.t["scales"][s] * (self.t["codes"][s] * Ch[:, None]).sum(-1)
            v, size = part, np.abs(part)
            # (a row's integer sum is exact, but eight lanes add their parts of it in binary32, each with its factor)
            size = np.maximum(size, E[:, None] * self.t["scales"][s] * np.abs(self.t["codes"][s] * Ch[:, None]).sum(-1))
            for i, j in enumerate(tokens):
                cb = (Cq.astype(np.float64) * self.t["Bwin"][s, :, j % WINDOW]).sum(-1)[self.group]
                part = sx * self.s_B[self.group][:, None] * (w[i] * cb)[:, None] * self.t["xwin"][s, :, j % WINDOW]
                v, size = v + part, size + np.abs(part)
            sC = self.s_C[self.group][:, None]
            v, size = sC * v, sC * size
            if self.D is not None:
                v, size = v + self.D[:, None] * sx * x, size + np.abs(self.D[:, None] * sx * x)
            if self.corr is not None:
                v, size = v + self.corr.reshape(self.H, self.P), size + np.abs(self.corr.reshape(self.H, self.P))
            y[b] = v.reshape(-1)
            bound[b] = (2.0 ** -24 * (32 + exponent)[:, None] * size).reshape(-1)
            if p % WINDOW == WINDOW - 1:
                S, _ = self.state(s, tokens)
                step = (np.abs(S).max(-1) / 127.0).astype(np.float32)
                step[step == 0] = 1
                self.t["codes"][s], self.t["scales"][s] = code(S / step[..., None].astype(np.float64)), step
        return bound


def parts(x, z, weight, groups, eps):
    """u w, and each element's sqrt(mean + eps)"""
    T, D = x.shape
    u = x.astype(np.float64) if z is None else x.astype(np.float64) * silu(z.astype(np.float64))
    root = np.sqrt((u.reshape(T, groups, D // groups) ** 2).mean(-1) + eps)
    return u if weight is None else u * weight.astype(np.float64), np.repeat(root, D // groups, -1)


def norm(x, z, weight, groups, eps):
    """o of the gated RMS norm, and the same without the norm where the row is one group (it cancels out of 127 o / absmax)"""
    T, D = x.shape
    with np.errstate(all="ignore"):
        u = x.astype(np.float64) if z is None else x.astype(np.float64) * silu(z.astype(np.float64))
        g = u.reshape(T, groups, D // groups)
        w = np.ones(D) if weight is None else weight.astype(np.float64)
        root = np.sqrt((g * g).mean(-1, keepdims=True) + eps)
        o = (g / root).reshape(T, D) * w
        # (an infinite or missing norm does not cancel: o is then 0 or NaN)
        return o, np.where(np.isfinite(root[:, 0]), u * w, o) if groups == 1 else o


def norm_codes(x, z, weight, groups, eps, static=None):
    o, v = norm(x, z, weight, groups, eps)
    with np.errstate(all="ignore"):
        if static is not None:
            return code(o / np.float64(static)), None
        top, of = np.nan_to_num(np.fmax.reduce(np.abs(v), -1), nan=0.0, posinf=np.inf), np.nan_to_num(np.fmax.reduce(np.abs(o), -1), nan=0.0, posinf=np.inf)
        q = np.where(top[:, None] > 0, 127.0 * v / np.where(top > 0, top, 1)[:, None], v)
        if groups > 1:
            # the same with the ratio of the norms by itself, which is 1 in the group of the absmax: exact ties stay ties there
            v, root = parts(x, z, weight, groups, eps)
            at = np.where(np.isnan(o), -1.0, np.abs(o)).argmax(-1)[:, None]
            ratio = 127.0 * v / np.abs(np.take_along_axis(v, at, -1)) * (np.take_along_axis(root, at, -1) / root)
            q = np.where((top > 0)[:, None] & np.isfinite(root).all(-1, keepdims=True), ratio, q)
        return code(q), np.where(of > 0, of / 127.0, 1.0)
