"""Shared by the tests of the layers' operators on the GPU: calls with buffers of their own, and the bounds of their errors."""
import numpy as np
import torch

import paper_2608_11226_amd as R
from oracle import layers as L

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
CODE = {"fp32": R.DTYPE_FP32, "bf16": R.DTYPE_BF16, "e4m3": R.DTYPE_E4M3}
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}  # the largest relative error of a rounding
U = 2.0 ** -24
SENTINEL = 77.0


def wide(t):
    return t.detach().double().cpu().numpy()


class Attention:
    """Inputs of a call, its buffers, and what the definition gives."""

    def __init__(self, dtype, heads, kv, hd, q_lens, k_lens=None, causal=True, room=0, fused=False, scale=None, seed=0, spread=1.0,
                 give_lens=None, own_keys=None):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.dtype, self.H, self.K, self.hd, self.causal = dtype, heads, kv, hd, causal
        self.scale = float(np.float32(scale or hd ** -0.5))
        own_keys = k_lens is None if own_keys is None else own_keys
        k_lens = q_lens if k_lens is None else k_lens
        t = TYPES[dtype]

        def places(lens):
            starts = np.concatenate([[0], np.cumsum([n + room for n in lens])])
            return starts, max(1, int(starts[-1]) + 3)  # rows behind the last sequence

        (qs, self.n_q), (ks, self.n_k) = places(q_lens), places(k_lens)
        self.q_seqs = [(int(a), n) for a, n in zip(qs, q_lens)]
        self.k_seqs = [(int(a), n) for a, n in zip(ks, k_lens)]
        give_lens = room > 0 if give_lens is None else give_lens
        i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)  # noqa: E731
        self.q_starts, self.k_starts = i32(qs), None if own_keys else i32(ks)
        self.q_lens = i32(q_lens) if give_lens else None
        self.k_lens = i32(k_lens) if give_lens and not own_keys else None
        wq, wk = heads * hd, kv * hd
        rand = lambda n, w: (torch.randn((n, w), generator=g, device=DEV) * spread).to(t)  # noqa: E731
        if fused:
            x = rand(self.n_q, wq + 2 * wk + 16)
            self.q, self.k, self.v = x[:, :wq], x[:, wq:wq + wk], x[:, wq + wk:wq + 2 * wk]
        else:
            self.q, self.k, self.v = rand(self.n_q, wq), rand(self.n_k, wk), rand(self.n_k, wk)
        self.grad_out = rand(self.n_q, wq)
        # what belongs to no sequence is not read
        for x, seqs, n in ((self.q, self.q_seqs, self.n_q), (self.k, self.k_seqs, self.n_k), (self.v, self.k_seqs, self.n_k),
                           (self.grad_out, self.q_seqs, self.n_q)):
            x[self.unused(seqs, n)] = float("nan")
        self.shape = R.AttentionShape(dtype=CODE[dtype], n_heads=heads, n_kv_heads=kv, head_dim=hd, n_seqs=len(q_lens), n_q=self.n_q,
                                      n_k=self.n_k, causal=int(causal), scale=self.scale)
        self.fused, self.few = fused, False

    @staticmethod
    def unused(seqs, n):
        free = np.ones(n, dtype=bool)
        for a, k in seqs:
            free[a:a + k] = False
        return torch.tensor(free, device=DEV)

    def new(self, n, w, fill=SENTINEL):
        return torch.full((n, w), fill, dtype=TYPES[self.dtype], device=DEV)

    def inputs(self):
        return (self.q, self.q.stride(0), self.k, self.k.stride(0), self.v, self.v.stride(0), self.q_starts, self.q_lens,
                self.k_starts, self.k_lens)

    def forward(self, stream=None, out=None, lse=None, ws=None):
        out = self.new(self.n_q, self.H * self.hd) if out is None else out
        lse = torch.full((self.H, self.n_q), SENTINEL, device=DEV) if lse is None else lse
        need = R.rollout_attention_workspace(self.shape)
        ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV) if ws is None else ws
        R.rollout_attention(self.shape, *self.inputs(), out, out.stride(0), lse, ws, need,
                            torch.cuda.current_stream().cuda_stream if stream is None else stream)
        return out, lse

    def backward(self, out, lse, grads=None, ws=None, stream=None):
        wq, wk = self.H * self.hd, self.K * self.hd
        if grads is None:
            if self.fused:
                d = self.new(self.n_q, wq + 2 * wk + 8)
                grads = d[:, :wq], d[:, wq:wq + wk], d[:, wq + wk:wq + 2 * wk]
            else:
                grads = self.new(self.n_q, wq), self.new(self.n_k, wk), self.new(self.n_k, wk)
        need = R.rollout_attention_backward_workspace(self.shape)
        ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV) if ws is None else ws
        dq, dk, dv = grads
        R.rollout_attention_backward(self.shape, *self.inputs(), out, out.stride(0), lse, self.grad_out, self.grad_out.stride(0), dq,
                                     dq.stride(0), dk, dk.stride(0), dv, dv.stride(0), ws, need,
                                     torch.cuda.current_stream().cuda_stream if stream is None else stream)
        return grads

    def heads(self, x, n):
        return wide(x).reshape(x.shape[0], n, self.hd)

    def definition(self):
        q, k, v = self.heads(self.q, self.H), self.heads(self.k, self.K), self.heads(self.v, self.K)
        return q, k, v, L.attention(q, k, v, self.q_seqs, self.k_seqs, self.scale, self.causal)

    def check_forward(self, out, lse):
        q, k, v, (o, z) = self.definition()
        got, got_z = self.heads(out, self.H), wide(lse)
        G = self.H // self.K
        half = HALF[self.dtype]
        for (a, nq), (b, nk) in zip(self.q_seqs, self.k_seqs):
            for h in range(self.H):
                A, B = slice(a, a + nq), slice(b, b + nk)
                p, es = self.score_errors(q[A, h], k[B, h // G], nq, nk)
                # a probability: its score's error, the exponential's 2, a share of the running maximum's rescalings (2 each of
                # at most nk / 64), the sum's nk roundings; bf16 rounds it once more
                ep = es.max(1, initial=0.0)[:, None] * 2 + (nk + nk / 32 + 8) * U + self.second_rounding()
                bound = ep * (p @ np.abs(v[B, h // G])) * 1.01 + (half + 4 * U) * np.abs(o[A, h]) * 1.01 + 1e-37
                err = np.abs(got[A, h] - o[A, h])
                assert (err <= bound).all(), f"out: head {h} of the sequence at {a}: {np.nanmax(err / bound):.3g} of the bound"
                empty = np.isneginf(z[h, A])
                assert (np.isneginf(got_z[h, A]) == empty).all() and (got[A, h][empty] == 0).all()
                err = np.abs(got_z[h, A][~empty] - z[h, A][~empty])
                bound = (es.max(1, initial=0.0) + (nk + nk / 32 + 8) * U + 4 * U * np.abs(z[h, A]) + 2.0 ** -21)[~empty]
                assert (err <= bound).all(), f"lse: head {h} of the sequence at {a}"
        free = self.unused(self.q_seqs, self.n_q).cpu().numpy()
        assert (wide(out)[free] == SENTINEL).all() and (got_z[:, free] == SENTINEL).all(), "a row of no sequence was written"

    def second_rounding(self):
        """How far a probability may be off as an operand of the second product: half a step of bf16, and where what that lost is
        multiplied as well (calls of few pairs), half a step of the rest; nothing in fp32."""
        half = HALF["bf16"]
        return 0.0 if self.dtype == "fp32" else half * half if self.few else half

    def score_errors(self, q, k, nq, nk):
        """Probabilities, and how far the exponent of each may be off: hd + 4 roundings of the product's terms, and one of it
        times log2 e, twice (its own and the maximum's)."""
        seen = L._attended(nq, nk, self.causal)
        s, p, _ = L._probabilities(q, k, self.scale, seen)
        es = (self.hd + 4) * U * self.scale * (np.abs(q) @ np.abs(k).T) + 4 * U * np.abs(np.where(seen, s, 0.0))
        return p, np.where(seen, es, 0.0)

    def check_backward(self, grads, out, lse):
        q, k, v = self.heads(self.q, self.H), self.heads(self.k, self.K), self.heads(self.v, self.K)
        do, o, z = self.heads(self.grad_out, self.H), self.heads(out, self.H), wide(lse)
        want = L.attention_backward(q, k, v, o, z, do, self.q_seqs, self.k_seqs, self.scale, self.causal)
        got = [self.heads(x, n) for x, n in zip(grads, (self.H, self.K, self.K))]
        G, half = self.H // self.K, HALF[self.dtype]
        rounds = self.second_rounding()
        bounds = [np.zeros_like(w) for w in want]
        for (a, nq), (b, nk) in zip(self.q_seqs, self.k_seqs):
            A, B = slice(a, a + nq), slice(b, b + nk)
            for h in range(self.H):
                j = h // G
                p, es = self.score_errors(q[A, h], k[B, j], nq, nk)
                zz = np.where(np.isfinite(z[h, A]), z[h, A], 0.0)[:, None]
                # p = 2^(s log2 e - lse log2 e): the score's error, 4 roundings of lse, 2 of the exponential
                ep = es + 4 * U * np.abs(zz) + 4 * U + (self.hd * U * np.abs(zz) if self.few else 0.0)  # (products that start from lse)
                dp, d = do[A, h] @ v[B, j].T, (do[A, h] * o[A, h]).sum(1, keepdims=True)
                ds = np.abs(p * (dp - d))
                # both products' hd + 4 roundings
                eds = ds * (ep * 1.01 + 4 * U + rounds) + 1.01 * p * (self.hd + 4) * U * (
                    np.abs(do[A, h]) @ np.abs(v[B, j]).T + (np.abs(do[A, h]) * np.abs(o[A, h])).sum(1, keepdims=True))
                # sums of nq G (or nk) terms
                bounds[2][B, j] += (p * (ep * 1.01 + rounds + (nq * G + 2) * U)).T @ np.abs(do[A, h])
                bounds[1][B, j] += self.scale * (eds + ds * (nq * G + 3) * U).T @ np.abs(q[A, h])
                bounds[0][A, h] += self.scale * (eds + ds * (nk + 3) * U) @ np.abs(k[B, j])
        for name, g, w, b, seqs, n in zip("qkv", got, want, bounds, (self.q_seqs, self.k_seqs, self.k_seqs), (self.n_q, self.n_k, self.n_k)):
            free = self.unused(seqs, n).cpu().numpy()
            assert (g[free] == SENTINEL).all(), f"a row of no sequence was written in the gradient of {name}"
            err, b = np.abs(g - w)[~free], (b * 1.02 + half * np.abs(w) * 1.02 + 1e-37)[~free]
            assert (err <= b).all(), f"gradient of {name}: {np.nanmax(err / b):.3g} of the bound"
