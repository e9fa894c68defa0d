"""Oracle of the update side of a GRPO step.

TEST INFRASTRUCTURE ONLY (see the package header).

The paper gives the update phase no arithmetic (section 3 names it), so these
are the plain definitions, in float64:

* token log probabilities under softmax(z / T), entropy, statistics (max z,
  log sum exp((z - max z) / T)) and the top ids by (logit descending, id
  ascending); and their gradient with respect to z;
* the clipped policy loss over groups with a k3 penalty towards a reference
  and an entropy term, and its gradients;
* embedding lookup with scaling, and its gradient.

Parity: pinned by torch's autograd in float64, finite differences and hand
cases in ``tests/test_oracle_update.py``.
"""
from __future__ import annotations

import numpy as np

NAN = float("nan")


def token_logprobs(z, temperature, tokens, top=0):
    """z [n, V] -> dict of logp [n], entropy [n], stats [n, 2], ids [n, top], top_logp [n, top]; tokens None: all rows,
    and no logp."""
    z = np.asarray(z, dtype=np.float64)
    n, V = z.shape
    out = {"logp": np.zeros(n), "entropy": np.zeros(n), "stats": np.zeros((n, 2)),
           "ids": np.full((n, top), -1, dtype=np.int64), "top_logp": np.zeros((n, top))}
    for r in range(n):
        t = 0 if tokens is None else int(tokens[r])
        if t < 0:
            continue
        row = z[r]
        if np.isnan(row).any() or np.isposinf(row).any():
            out["logp"][r] = out["entropy"][r] = NAN
            out["stats"][r] = NAN
            out["top_logp"][r] = NAN
            continue
        m = row.max()
        order = np.argsort(-row, kind="stable")[:top]  # -0.0 and 0.0 compare equal
        out["ids"][r] = order
        if np.isneginf(m):
            out["logp"][r] = -np.inf if t < V else NAN
            out["stats"][r] = -np.inf
            out["top_logp"][r] = -np.inf
            continue
        d = (row - m) / np.float64(np.float32(temperature))
        e = np.exp(d)
        log_s = np.log(e.sum())
        lp = d - log_s
        out["logp"][r] = lp[t] if t < V else NAN
        live = e > 0
        out["entropy"][r] = -(np.exp(lp[live]) * lp[live]).sum()
        out["stats"][r] = m, log_s
        out["top_logp"][r] = lp[order]
    return out


def token_logprobs_backward(z, temperature, tokens, stats, entropy, g, h=None):
    """dz [n, V] of sum_r g_r logp_r + h_r entropy_r, from the given statistics."""
    z = np.asarray(z, dtype=np.float64)
    n, V = z.shape
    T = np.float64(np.float32(temperature))
    dz = np.zeros((n, V))
    for r in range(n):
        t, gr = int(tokens[r]), float(g[r])
        hr, H = (0.0, 0.0) if h is None else (float(h[r]), float(entropy[r]))
        if t < 0 or (gr == 0 and hr == 0) or np.isneginf(stats[r, 0]):
            continue
        if t >= V:
            dz[r] = NAN
            continue
        lp = (z[r] - float(stats[r, 0])) / T - float(stats[r, 1])
        p = np.exp(lp)
        dz[r] = -gr * p
        live = p > 0
        dz[r, live] -= hr * p[live] * (lp[live] + H)
        dz[r, t] += gr
        dz[r] /= T
    return dz


MEAN_SEQUENCE, MEAN_TOKEN, MEAN_FIXED = 0, 1, 2


def policy_loss(logp, old, ref, entropy, adv, lengths, clip_low, clip_high, kl_coef, entropy_coef, mean):
    """logp, old, ref, entropy [S, N] (old, ref, entropy may be None), adv [S], lengths [S] or None ->
    (loss, stats [5], dlogp [S, N], dentropy [S, N])."""
    logp = np.asarray(logp, dtype=np.float64)
    S, N = logp.shape
    lengths = np.full(S, N) if lengths is None else np.clip(np.asarray(lengths, dtype=np.int64), 0, N)
    f = lambda x: float(np.float32(x))
    lo, hi, b, c = f(clip_low), f(clip_high), f(kl_coef), f(entropy_coef)
    total = int(lengths.sum())
    loss, sums = 0.0, np.zeros(5)
    dlogp, dent = np.zeros((S, N)), np.zeros((S, N))
    for s in range(S):
        A = float(adv[s])
        w = {MEAN_SEQUENCE: 1.0 / (S * max(1, lengths[s])), MEAN_TOKEN: 1.0 / max(1, total), MEAN_FIXED: 1.0 / (S * N)}[mean]
        for t in range(lengths[s]):
            r = np.exp(logp[s, t] - float(old[s, t])) if old is not None else 1.0
            low, high = A < 0 and r < 1.0 - lo, A > 0 and r > 1.0 + hi
            surr = (1.0 + hi) * A if high else (1.0 - lo) * A if low else r * A
            x = float(ref[s, t]) - logp[s, t] if ref is not None else 0.0
            kl = np.expm1(x) - x if x < np.inf else np.inf
            H = float(entropy[s, t]) if entropy is not None else 0.0
            loss += w * (-surr + (b * kl if b else 0.0) - (c * H if c else 0.0))
            sums += r, kl, low, high, H
            dlogp[s, t] = w * ((0.0 if low or high else -A * r) - (b * np.expm1(x) if b else 0.0))
            dent[s, t] = -c * w
    return loss, sums / max(1, total), dlogp, dent


def embedding(table, tokens, scale):
    table = np.asarray(table, dtype=np.float64)
    V, d = table.shape
    out = np.zeros((len(tokens), d))
    for n, t in enumerate(tokens):
        if t >= V:
            out[n] = NAN
        elif t >= 0:
            out[n] = np.float64(np.float32(scale)) * table[t]
    return out


def embedding_backward(grad, tokens, vocab, scale, base=None):
    """Gradient of the table, added to base if given."""
    grad = np.asarray(grad, dtype=np.float64)
    out = np.zeros((vocab, grad.shape[1]))
    tokens = np.asarray(tokens)
    live = (tokens >= 0) & (tokens < vocab)
    np.add.at(out, tokens[live], grad[live])
    out *= np.float64(np.float32(scale))
    return out if base is None else out + np.asarray(base, dtype=np.float64)
