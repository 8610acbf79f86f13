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
