"""Packed attention, the residual norm and AdamW, with their gradients, in float64 NumPy (test infrastructure only)."""
import numpy as np


def sequences(starts, lens, rows):
    """(first row, length) of every sequence, as the calls take them."""
    out = []
    for s in range(len(starts) - 1):
        a = min(max(int(starts[s]), 0), rows)
        b = max(a, min(int(starts[s + 1]), rows))
        out.append((a, b - a if lens is None else min(max(int(lens[s]), 0), b - a)))
    return out


def _attended(nq, nk, causal):
    if not causal:
        return np.ones((nq, nk), dtype=bool)
    return np.arange(nk)[None] <= (np.arange(nq) + nk - nq)[:, None]


def _probabilities(q, k, scale, seen):
    with np.errstate(invalid="ignore", divide="ignore"):
        s = np.where(seen, (q @ k.T) * scale, -np.inf)
        m = s.max(1, initial=-np.inf, keepdims=True)
        e = np.where(seen, np.exp(s - np.where(np.isfinite(m), m, 0.0)), 0.0)
        total = e.sum(1, keepdims=True)
        lse = np.where(total > 0, np.where(np.isfinite(m), m, 0.0) + np.log(np.where(total > 0, total, 1.0)), -np.inf)[:, 0]
        return s, np.where(total > 0, e / np.where(total > 0, total, 1.0), 0.0), lse


def attention(q, k, v, q_seqs, k_seqs, scale, causal):
    """q [n, heads, hd], k, v [m, kv heads, hd]; rows of no sequence stay NaN.  Returns (out, lse [heads, n])."""
    n, H, hd = q.shape
    G = H // k.shape[1]
    out, lse = np.full(q.shape, np.nan), np.full((H, n), np.nan)
    for (a, nq), (b, nk) in zip(q_seqs, k_seqs):
        seen = _attended(nq, nk, causal)
        for h in range(H):
            _, p, z = _probabilities(q[a:a + nq, h], k[b:b + nk, h // G], scale, seen)
            out[a:a + nq, h] = p @ v[b:b + nk, h // G]
            lse[h, a:a + nq] = z
    return out, lse


def attention_backward(q, k, v, out, lse, grad_out, q_seqs, k_seqs, scale, causal):
    """Gradients of q, k, v from the forward call's out and lse; rows of no sequence stay NaN."""
    H, G = q.shape[1], q.shape[1] // k.shape[1]
    dq, dk, dv = np.full(q.shape, np.nan), np.full(k.shape, np.nan), np.full(v.shape, np.nan)
    for (a, nq), (b, nk) in zip(q_seqs, k_seqs):
        A, B = slice(a, a + nq), slice(b, b + nk)
        dq[A], dk[B], dv[B] = 0.0, 0.0, 0.0
        seen = _attended(nq, nk, causal)
        for h in range(H):
            z = lse[h, A]
            p = np.where(seen, np.exp((q[A, h] @ k[B, h // G].T) * scale - np.where(np.isfinite(z), z, 0.0)[:, None]), 0.0)
            d = (grad_out[A, h] * out[A, h]).sum(1, keepdims=True)
            ds = p * (grad_out[A, h] @ v[B, h // G].T - d)
            dq[A, h] = scale * ds @ k[B, h // G]
            dk[B, h // G] += scale * ds.T @ q[A, h]
            dv[B, h // G] += p.T @ grad_out[A, h]
    return dq, dk, dv


def rms_norm(h, gain, eps):
    """(y, 1 / root mean square) of rows."""
    r = 1.0 / np.sqrt((h * h).mean(1) + eps)
    return h * r[:, None] * gain, r


def rms_norm_backward(dy, h, gain, rstd, inner):
    xhat, t = h * rstd[:, None], dy * gain
    return inner + rstd[:, None] * (t - xhat * (t * xhat).mean(1, keepdims=True)), (dy * xhat).sum(0)


# ---------------------------------------------------------------------------
# e4m3
# ---------------------------------------------------------------------------
def e4m3_values():
    """Value of every code; 0x7F and 0xFF are NaN."""
    c = np.arange(256)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


def power_scale(most):
    """Smallest power of two, 2^-126 at least, that brings `most` to at most 448."""
    f, e = np.frexp(most)
    return np.ldexp(1.0, np.where(np.asarray(most) > 0, np.maximum(e - 9 + (f > 0.875), -126), -126))


def spacing(a):
    """Distance of neighbouring e4m3 values at a >= 0."""
    return 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------
_M64, _GOLD = (1 << 64) - 1, 0x9E3779B97F4A7C15


def _finish64(x):
    x = ((x ^ (x >> 30)) * 0xBF58476D1CE4E5B9) & _M64
    x = ((x ^ (x >> 27)) * 0x94D049BB133111EB) & _M64
    return x ^ (x >> 31)


def _finish32(h):
    h = ((h ^ (h >> np.uint64(16))) * np.uint64(0x85EBCA6B)) & np.uint64(0xFFFFFFFF)
    h = ((h ^ (h >> np.uint64(13))) * np.uint64(0xC2B2AE35)) & np.uint64(0xFFFFFFFF)
    return h ^ (h >> np.uint64(16))


def adamw_bits(seed, step, tensor, index):
    """16 random bits each for the first moment, the second and the weight of elements `index` of a tensor."""
    index = np.asarray(index, dtype=np.uint64)
    first = _finish64((seed + _GOLD * step) & _M64)
    high = index >> np.uint64(32)
    keys = {int(r): _finish64((first + _GOLD * (tensor + (int(r) << 20) + 1)) & _M64) for r in np.unique(high)}
    pick = lambda f: np.array([f(keys[int(r)]) for r in np.unique(high)], dtype=np.uint64)[np.unique(high, return_inverse=True)[1]]  # noqa: E731
    low = np.uint64(0xFFFFFFFF)
    h = _finish32(((index & low) * np.uint64(0x9E3779B1) + pick(lambda k: k & 0xFFFFFFFF)) & low)
    w = _finish32((h + pick(lambda k: k >> 32)) & low)
    return (h & np.uint64(0xFFFF)).astype(np.int64), (h >> np.uint64(16)).astype(np.int64), (w & np.uint64(0xFFFF)).astype(np.int64)


def adamw(p, g, m, v, lr, beta1, beta2, eps, step, decay):
    """New weights and moments before any rounding."""
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    return p * (1 - lr * decay) - lr * m / (1 - beta1 ** step) / (np.sqrt(v / (1 - beta2 ** step)) + eps), m, v
