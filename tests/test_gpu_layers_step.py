"""A training step through one layer, as its calls follow each other: embedding, norm, attention, norm behind the residual addition,
log probabilities, group loss, all the way back, and the optimiser's step; on a padded batch as the rollout leaves it, against
torch's autograd in float64, and against differences of the whole chain."""
import numpy as np
import pytest
import torch

import paper_2608_11226_amd as R
from layer_cases import CODE, DEV, TYPES, wide
from oracle import layers as L
from oracle import update as U

pytestmark = pytest.mark.gpu
S, G, N, V, D, H, K, HD = 6, 3, 37, 97, 64, 4, 2, 32
EPS, SCALE = 1e-6, HD ** -0.5
LENS = [37, 1, 20, 0, 36, 9]
NAMES = ("table", "gain1", "qkv", "o", "gain2", "head")


def weights(seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s, by=1.0: torch.randn(s, generator=g, device=DEV) * by  # noqa: E731
    return {"table": r(V, D), "gain1": 1 + r(D, by=0.1), "qkv": r((H + 2 * K) * HD, D, by=0.2), "o": r(D, H * HD, by=0.1),
            "gain2": 1 + r(D, by=0.1), "head": r(V, D, by=0.2)}


class Batch:
    def __init__(self, seed=1):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.lens = torch.tensor(LENS, dtype=torch.int32, device=DEV)
        live = torch.arange(N, device=DEV)[None] < self.lens[:, None]
        draw = lambda: torch.randint(0, V, (S, N), generator=g, device=DEV, dtype=torch.int32).masked_fill(~live, -1)  # noqa: E731
        self.tokens, self.targets, self.live = draw(), draw(), live
        self.starts = torch.arange(S + 1, dtype=torch.int32, device=DEV) * N
        self.rewards = torch.rand(S, generator=g, device=DEV)
        self.adv = torch.empty(S, device=DEV)
        R.grpo_advantages(self.rewards, S // G, G, 0.0, 1, self.adv, None, torch.cuda.current_stream().cuda_stream)
        self.old = None


def forward(w, b, dtype="fp32"):
    s, n = torch.cuda.current_stream().cuda_stream, S * N
    t, code = TYPES[dtype], CODE[dtype]
    new = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device=DEV)  # noqa: E731
    a = {"x": new(n, D), "y1": new(n, D, dtype=t), "r1": new(n), "h": new(n, D), "y2": new(n, D, dtype=t), "r2": new(n),
         "att": new(n, H * HD, dtype=t), "lse": new(H, n)}
    R.rollout_embedding(w["table"], 0, V, D, b.tokens, n, 1.0, a["x"], 0, s)
    R.rollout_rms_norm(a["x"], 0, None, 0, w["gain1"], n, D, EPS, None, a["y1"], code, None, a["r1"], s)
    a["qkv"] = a["y1"] @ w["qkv"].to(t).t()
    a["shape"] = R.AttentionShape(dtype=code, n_heads=H, n_kv_heads=K, head_dim=HD, n_seqs=S, n_q=n, n_k=n, causal=1, scale=SCALE)
    need = R.rollout_attention_workspace(a["shape"])
    width = (H + 2 * K) * HD
    a["views"] = (a["qkv"][:, :H * HD], width, a["qkv"][:, H * HD:(H + K) * HD], width, a["qkv"][:, (H + K) * HD:], width, b.starts, b.lens,
                  None, None)
    R.rollout_attention(a["shape"], *a["views"], a["att"], H * HD, a["lse"], new(need, dtype=torch.uint8), need, s)
    a["delta"] = a["att"] @ w["o"].to(t).t()
    R.rollout_rms_norm(a["x"], 0, a["delta"], code, w["gain2"], n, D, EPS, a["h"], a["y2"], code, None, a["r2"], s)
    a["logits"] = (a["y2"] @ w["head"].to(t).t()).float()
    a["logp"], a["H"], a["stats"] = new(S, N), new(S, N), new(S, N, 2)
    need = R.rollout_token_logprobs_workspace(n, V, 0)
    R.rollout_token_logprobs(a["logits"], 0, V, n, V, 1.0, b.targets, 0, a["logp"], a["H"], a["stats"], None, None,
                             new(max(need, 16), dtype=torch.uint8), need, s)
    a["loss"], a["dlogp"], a["dH"] = new(1), new(S, N), new(S, N)
    need = R.grpo_policy_loss_workspace(S, N)
    R.grpo_policy_loss(a["logp"], a["logp"] if b.old is None else b.old, None, a["H"], b.adv, b.lens, S, N, 0.2, 0.28, 0.0, 0.01,
                       R.MEAN_TOKEN, a["loss"], None, a["dlogp"], a["dH"], new(max(need, 16), dtype=torch.uint8), need, s)
    return a


def backward(w, b, a, dtype="fp32"):
    s, n = torch.cuda.current_stream().cuda_stream, S * N
    t, code = TYPES[dtype], CODE[dtype]
    new = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device=DEV)  # noqa: E731
    g = {k: new(*v.shape) for k, v in w.items()}
    dlogits = new(n, V)
    R.rollout_token_logprobs_backward(a["logits"], 0, V, n, V, 1.0, b.targets, a["stats"], a["H"], a["dlogp"], a["dH"], dlogits, V, s)
    dl = dlogits.to(t)
    g["head"] = (dl.t() @ a["y2"]).float()
    dy2 = dl @ w["head"].to(t)
    ws = new(max(R.rollout_rms_norm_backward_workspace(n, D), R.rollout_attention_backward_workspace(a["shape"]),
                 R.rollout_embedding_backward_workspace(n, V, D)), dtype=torch.uint8)
    dh = new(n, D)
    R.rollout_rms_norm_backward(dy2, code, a["h"], 0, w["gain2"], a["r2"], n, D, None, dh, 0, g["gain2"], 0, ws, ws.numel(), s)
    ddelta = dh.to(t)
    g["o"] = (ddelta.t() @ a["att"]).float()
    datt = ddelta @ w["o"].to(t)
    dqkv = new(n, (H + 2 * K) * HD, dtype=t)
    width = (H + 2 * K) * HD
    R.rollout_attention_backward(a["shape"], *a["views"], a["att"], H * HD, a["lse"], datt, H * HD, dqkv[:, :H * HD], width,
                                 dqkv[:, H * HD:(H + K) * HD], width, dqkv[:, (H + K) * HD:], width, ws, ws.numel(), s)
    g["qkv"] = (dqkv.t() @ a["y1"]).float()
    dy1 = dqkv @ w["qkv"].to(t)
    # on top of what came by the residual stream, in its place
    R.rollout_rms_norm_backward(dy1, code, a["x"], 0, w["gain1"], a["r1"], n, D, dh, dh, 0, g["gain1"], 0, ws, ws.numel(), s)
    R.rollout_embedding_backward(dh, 0, b.tokens, n, V, D, 1.0, 0, g["table"], 0, ws, ws.numel(), s)
    return g


def reference(w, b, old):
    """Loss and gradients by torch's autograd in float64 on the CPU, sequence by sequence without padding."""
    p = {k: v.double().cpu().requires_grad_() for k, v in w.items()}
    norm = lambda x, gain: x * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS) * gain  # noqa: E731
    total, count = 0.0, sum(LENS)
    for i, n in enumerate(LENS):
        if not n:
            continue
        ids, target = b.tokens[i, :n].long().cpu(), b.targets[i, :n].long().cpu()
        x = p["table"][ids]
        qkv = norm(x, p["gain1"]) @ p["qkv"].t()
        q, k, v = (z.view(n, -1, HD).transpose(0, 1) for z in qkv.split([H * HD, K * HD, K * HD], 1))
        sc = (q @ k.repeat_interleave(H // K, 0).transpose(1, 2)) * float(np.float32(SCALE))
        sc = sc.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -torch.inf)
        att = (torch.softmax(sc, 2) @ v.repeat_interleave(H // K, 0)).transpose(0, 1).reshape(n, -1)
        logp = torch.log_softmax(norm(x + att @ p["o"].t(), p["gain2"]) @ p["head"].t(), 1)
        ent = -(logp.exp() * logp).sum(1)
        lp = logp[torch.arange(n), target]
        adv, r = b.adv[i].double().cpu(), torch.exp(lp - old[i, :n].double().cpu())
        total = total + (-torch.minimum(r * adv, r.clamp(0.8, 1.28) * adv) - 0.01 * ent).sum() / count
    total.backward()
    return float(total.detach()), {k: v.grad for k, v in p.items()}


# the chain has 12 stages; fp32: sums of at most 1,024 terms, off by at most as many roundings of 2^-24 of their terms; bf16: one
# rounding of 2^-8 each, which largely cancel in a gradient's norm
@pytest.mark.parametrize("dtype,bound", [("fp32", 12 * 1024 * 2.0 ** -24), ("bf16", 12 * 2.0 ** -8)])
def test_gradients_of_a_step(dtype, bound):
    w, b = weights(), Batch()
    a = forward(w, b, dtype)
    g = backward(w, b, a, dtype)
    torch.cuda.synchronize()
    loss, want = reference(w, b, a["logp"])
    assert abs(float(a["loss"]) - loss) <= bound * max(1.0, abs(loss))
    for k in NAMES:
        assert torch.isfinite(g[k]).all()
        off = float((g[k].double().cpu() - want[k]).norm() / want[k].norm())
        assert off <= bound, (k, off)


def test_differences_of_the_chain():
    w, b = weights(2), Batch(3)
    a = forward(w, b)
    b.old = a["logp"].clone()
    g = backward(w, b, a)
    gen = torch.Generator(device=DEV).manual_seed(7)
    for k in NAMES:
        way = torch.randn(w[k].shape, generator=gen, device=DEV)
        way /= way.norm()
        slope, h = float((g[k].double() * way.double()).sum()), 2.0 ** -7
        ends = []
        for sign in (1, -1):
            moved = dict(w)
            moved[k] = w[k] + sign * h * way
            ends.append(float(forward(moved, b)["loss"]))
        # the loss is of size 1 and rounded to 2^-24 like every log probability in it; third order: h^2 = 2^-14 of derivatives of size 10
        assert abs((ends[0] - ends[1]) / (2 * h) - slope) <= 4 * 2.0 ** -24 / h * 8 + 10 * h * h, (k, slope)


def test_differences_along_the_gradients():
    """The same where it says most: along each weight's own gradient, where the slope is its norm, and half way from there to a random
    direction.  A gradient that is off by a tenth of its norm in either fails."""
    w, b = weights(8), Batch(9)
    a = forward(w, b)
    b.old = a["logp"].clone()
    g = backward(w, b, a)
    gen, h = torch.Generator(device=DEV).manual_seed(10), 2.0 ** -7
    # the loss is of size 1 and rounded to 2^-24 like every log probability in it; third order: h^2 of at most 4 (along the gradients
    # of six such chains in float64 at most 1.9)
    tol = 4 * 2.0 ** -24 / h * 8 + 4 * h * h
    for k in NAMES:
        along = g[k].double() / g[k].double().norm()
        other = torch.randn(w[k].shape, generator=gen, device=DEV, dtype=torch.float64)
        for way in (along, along + other / other.norm()):
            way = (way / way.norm()).float()
            slope = float((g[k].double() * way.double()).sum())
            assert slope >= 10 * tol, (k, slope)
            ends = [float(forward({**w, k: w[k] + sign * h * way}, b)["loss"]) for sign in (1, -1)]
            assert abs((ends[0] - ends[1]) / (2 * h) - slope) <= tol, (k, slope)


def test_steps_of_the_optimiser_follow():
    """Three steps with fp32 states against float64 on the same gradients, then with states in 8 bits: the loss of the tokens that
    are worth more than others is a number, and every weight has moved."""
    for state in ("fp32", "e4m3"):
        w, b = weights(4), Batch(5)
        s = torch.cuda.current_stream().cuda_stream
        grads = {k: torch.zeros_like(v) for k, v in w.items()}
        zeros = lambda k: torch.zeros(w[k].numel(), dtype=torch.float32 if state == "fp32" else torch.uint8, device=DEV)  # noqa: E731
        m, v = {k: zeros(k) for k in NAMES}, {k: zeros(k) for k in NAMES}
        sc = {k: [torch.zeros(-(-w[k].numel() // 128), device=DEV) for _ in range(2)] if state == "e4m3" else [None, None] for k in NAMES}
        copies = {k: torch.zeros(w[k].shape, dtype=torch.bfloat16, device=DEV) for k in NAMES}
        table, chunks = R.rollout_adamw_table([R.adamw_tensor(w[k], grads[k], m[k], v[k], 0.1, *sc[k], copy=copies[k]) for k in NAMES])
        table = table.to(DEV)
        exact = {k: (wide(w[k]), 0.0, 0.0) for k in NAMES}
        first = {k: x.clone() for k, x in w.items()}
        for step in (1, 2, 3):
            a = forward(w, b)
            for k, x in backward(w, b, a).items():
                grads[k].copy_(x)
            R.rollout_adamw(table, len(NAMES), chunks, 1e-3, 0.9, 0.95, 1e-8, step, 11, stream=s)
            exact = {k: L.adamw(exact[k][0], wide(grads[k]), exact[k][1], exact[k][2], 1e-3, 0.9, 0.95, 1e-8, step, 0.1) for k in NAMES}
            assert torch.isfinite(a["loss"]).all()
        for k in NAMES:
            assert torch.equal(copies[k], w[k].to(torch.bfloat16)) and not torch.equal(w[k], first[k])
            if state == "fp32":
                # three steps, each of at most 1e-3 / (1 - 0.9) sqrt(1 - 0.95) ... < 2e-2 and off by some 20 roundings of it
                assert (np.abs(wide(w[k]) - exact[k][0]) <= 3 * (20 * 2.0 ** -24 * 2e-2 + 4 * 2.0 ** -24 * np.abs(exact[k][0]))).all(), k


def test_the_step_in_a_graph():
    """Forward, backward and optimiser captured once and replayed: the same weights as calls one after the other."""
    def run(captured):
        w, b = weights(6), Batch(7)
        a = forward(w, b)
        b.old = a["logp"].clone()
        grads = {k: torch.zeros_like(x) for k, x in w.items()}
        m, v = ({k: torch.zeros(x.numel(), device=DEV) for k, x in w.items()} for _ in range(2))
        table, chunks = R.rollout_adamw_table([R.adamw_tensor(w[k], grads[k], m[k], v[k], 0.0) for k in NAMES])
        table, step = table.to(DEV), torch.zeros(1, dtype=torch.int64, device=DEV)

        def once():
            step.add_(1)
            a = forward(w, b)
            for k, x in backward(w, b, a).items():
                grads[k].copy_(x)
            R.rollout_adamw(table, len(NAMES), chunks, 1e-3, 0.9, 0.95, 1e-8, 1, 11, step_now=step, stream=torch.cuda.current_stream().cuda_stream)

        if not captured:
            for _ in range(4):
                once()
        else:
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                keep = {k: x.clone() for k, x in w.items()}
                once()  # (the products' library sets itself up outside the capture)
                for k, x in w.items():
                    x.copy_(keep[k]), m[k].zero_(), v[k].zero_()
                step.zero_()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=s):
                    once()
            torch.cuda.current_stream().wait_stream(s)
            for _ in range(4):
                graph.replay()
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return w

    a, b = run(False), run(True)
    for k in NAMES:
        assert torch.equal(a[k], b[k]), k
