"""A GRPO step from the rollout to the gradients of logits and embedding rows, as its calls follow each other: generate with
stop tokens, lengths, rewards, advantages, scoring of the drawn tokens, loss, and back; against the float64 definitions on
the same logits, and against differences of the whole chain."""
import numpy as np
import pytest

import paper_2608_11226_amd as R
import workload as W
from gpu_helpers import log, to_dev
from oracle import update as U

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, G, P, N, T = 3, 4, 16, 12, 0.9


@pytest.fixture(scope="module")
def step():
    """Tokens, lengths, advantages and the logits [S, N, V] that every token was drawn from."""
    cfg = R.model_config("tiny", R.DTYPE_FP32, P, N, B * G)
    eng = R.Engine(cfg, group_size=G)
    V, S, s = cfg.vocab, B * G, eng.stream_handle
    prompts = to_dev(W.prompts(B, P, V), torch)
    u = to_dev(W.uniforms(S, N), torch)
    stop = torch.arange(0, V, 9, dtype=torch.int32, device=DEV)
    tokens = torch.empty(S, N, dtype=torch.int32, device=DEV)
    lengths = torch.empty(S, dtype=torch.int32, device=DEV)
    rewards, adv = torch.empty(S, device=DEV), torch.empty(S, device=DEV)
    R.rollout_generate_eos(eng.ctx, prompts, B, P, G, S, N, T, 1.0, u, stop, stop.numel(), 1, 0, tokens, lengths)
    R.rollout_length_rewards(lengths, S, 6, rewards, None, s)
    R.grpo_advantages(rewards, B, G, 0.0, 1, adv, None, s)
    # the logits again, with the drawn tokens given (ended completions go on with token 0)
    logits = torch.empty(N, S, V, device=DEV)
    eng.synchronize()
    given = tokens.clamp(min=0).t().contiguous()
    torch.cuda.synchronize()
    R.rollout_prefill(eng.ctx, prompts, B, P, G, logits[0])
    for t in range(N - 1):
        R.rollout_decode_step(eng.ctx, given[t], logits[t + 1])
    table = torch.empty(V, cfg.d_model, device=DEV)
    R.rollout_export_weight(eng.ctx, 0, table)
    eng.synchronize()
    eng.close()
    return {"V": V, "S": S, "d": cfg.d_model, "tokens": tokens, "lengths": lengths, "adv": adv, "rewards": rewards,
            "logits": logits.transpose(0, 1).contiguous(), "prompts": prompts, "table": table}


def score(st, logits, dtype=R.DTYPE_FP32, top=0):
    S, V = st["S"], st["V"]
    out = {k: torch.empty(S, N, device=DEV) for k in ("logp", "entropy")}
    out["stats"] = torch.empty(S, N, 2, device=DEV)
    out["ids"], out["tops"] = torch.empty(S, N, max(1, top), dtype=torch.int32, device=DEV), torch.empty(S, N, max(1, top), device=DEV)
    need = R.rollout_token_logprobs_workspace(S * N, V, top)
    ws = torch.empty(max(16, need), dtype=torch.uint8, device=DEV)
    R.rollout_token_logprobs(logits, dtype, V, S * N, V, T, st["tokens"], top, out["logp"], out["entropy"], out["stats"],
                             out["ids"] if top else None, out["tops"] if top else None, ws, need)
    return out


COEF = (0.2, 0.28, 0.04, 0.01)


def loss_of(st, sc, old, ref, mean):
    S = st["S"]
    need = R.grpo_policy_loss_workspace(S, N)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    out = [torch.empty(1, device=DEV), torch.empty(5, device=DEV), torch.empty(S, N, device=DEV), torch.empty(S, N, device=DEV)]
    R.grpo_policy_loss(sc["logp"], old, ref, sc["entropy"], st["adv"], st["lengths"], S, N, *COEF, mean, *out, ws, need)
    return out


def back(st, logits, sc, loss, dtype=R.DTYPE_FP32):
    grad = torch.empty_like(logits)
    V = st["V"]
    R.rollout_token_logprobs_backward(logits, dtype, V, st["S"] * N, V, T, st["tokens"], sc["stats"], sc["entropy"], loss[2],
                                      loss[3], grad, V)
    return grad


def test_scores_agree_with_the_draws(step):
    """The alternatives of the first tokens hold the greedy ones, lengths and padding are those of the scores."""
    sc = score(step, step["logits"], top=4)
    lengths = step["lengths"].cpu().numpy()
    assert lengths.min() < N, "no completion ended early"
    live = torch.arange(N, device=DEV)[None] < step["lengths"][:, None]
    assert torch.equal(live, step["tokens"] >= 0)
    assert not sc["logp"][~live].any() and torch.all(sc["ids"][~live] == -1)
    assert torch.all(sc["logp"][live] < 0) and torch.all(sc["entropy"][live] > 0)
    greedy = torch.empty(step["S"], dtype=torch.int32, device=DEV)
    R.rollout_sample_noalloc(step["logits"][:, 0].contiguous(), step["S"], step["V"], 0.0, 1.0,
                             torch.zeros(step["S"], device=DEV), greedy)
    assert torch.equal(sc["ids"][:, 0, 0], greedy)


@pytest.mark.parametrize("mean", [0, 1, 2])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_step_matches_the_definitions(step, mean, dtype):
    S, V = step["S"], step["V"]
    kind = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
    code = {"fp32": R.DTYPE_FP32, "bf16": R.DTYPE_BF16}[dtype]
    gen = torch.Generator(device=DEV).manual_seed(1)
    noise = torch.randn(step["logits"].shape, generator=gen, device=DEV)
    now = (step["logits"] + 0.3 * noise).to(kind)  # the weights have moved on since the rollout
    old = score(step, step["logits"])["logp"]
    ref = score(step, (step["logits"] * 0.9).contiguous())["logp"]
    sc = score(step, now, code)
    out = loss_of(step, sc, old, ref, mean)
    grad = back(step, now, sc, out, code)
    # the same from the logits on, in 64 bits
    z = now.double().cpu().numpy().reshape(S * N, V)
    tok = step["tokens"].cpu().numpy().reshape(-1)
    o = U.token_logprobs(z, T, tok)
    lp = lambda x: U.token_logprobs(x.double().cpu().numpy().reshape(S * N, V), T, tok)["logp"].reshape(S, N)
    loss, stats, dlp, dH = U.policy_loss(o["logp"].reshape(S, N), lp(step["logits"]), lp(step["logits"] * 0.9),
                                         o["entropy"].reshape(S, N), step["adv"].cpu().numpy(), step["lengths"].cpu().numpy(),
                                         *COEF, mean)
    dz = U.token_logprobs_backward(z, T, tok, o["stats"], o["entropy"], dlp.reshape(-1), dH.reshape(-1)).reshape(S, N, V)
    log(f"loss {out[0].item():.6g} ({loss:.6g}), statistics {out[1].tolist()}")
    # log probabilities of some units are off by some 2^-22 (see their test), ratios by as much of themselves, and
    # everything behind follows from them linearly; bf16 gradients are rounded once more
    assert abs(out[0].item() - loss) <= 2.0 ** -18 * max(1.0, np.abs(step["adv"].cpu().numpy()).max())
    assert np.abs(out[1].double().cpu().numpy() - stats).max() <= 2.0 ** -18 * max(1.0, np.abs(stats).max())
    half = torch.finfo(kind).eps / 2
    size = np.abs(dlp).max() / T
    assert np.all(np.abs(grad.double().cpu().numpy() - dz) <= half * np.abs(dz) + 2.0 ** -17 * size)
    behind = (step["tokens"] < 0)
    assert not grad[behind].any()


def test_the_gradient_matches_differences_of_the_loss(step):
    gen = torch.Generator(device=DEV).manual_seed(2)
    now = step["logits"] + 0.05 * torch.randn(step["logits"].shape, generator=gen, device=DEV)
    old = score(step, step["logits"])["logp"]
    sc = score(step, now)
    out = loss_of(step, sc, old, old, 0)
    grad = back(step, now, sc, out)
    # along the gradient's own direction, with entries of size 1 at most, and along a random one
    for direction in (grad / grad.abs().max(), torch.randn(grad.shape, generator=gen, device=DEV)):
        step_ = 2.0 ** -6
        val = []
        for sgn in (1, -1):
            moved = now + sgn * step_ * direction
            val.append(loss_of(step, score(step, moved), old, old, 0)[0].item())
        want = (grad.double() * direction.double()).sum().item()
        scale = (grad.double().abs() * direction.double().abs()).sum().item()
        # tokens that cross a clipping border within the step change their slope: a step's share of the whole
        assert (val[0] - val[1]) / (2 * step_) == pytest.approx(want, abs=2.0 ** -20 / step_ + 0.02 * scale)


def test_embedding_rows_of_a_step(step):
    """Prompts and completions looked up in the exported table, and a gradient for each position sent back to its rows."""
    ids = torch.cat([step["prompts"].repeat_interleave(G, 0), step["tokens"]], 1).contiguous()
    n, V, d = ids.numel(), step["V"], step["d"]
    x = torch.empty(n, d, device=DEV)
    R.rollout_embedding(step["table"], R.DTYPE_FP32, V, d, ids, n, 1.0, x, R.DTYPE_FP32)
    flat = ids.flatten().long()
    assert torch.equal(x[flat >= 0], step["table"][flat[flat >= 0]]) and not x[flat < 0].any()
    g = torch.randn(n, d, device=DEV)
    need = R.rollout_embedding_backward_workspace(n, V, d)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    # two micro-batches into one gradient
    table = torch.empty(V, d, device=DEV)
    half = n // 2
    R.rollout_embedding_backward(g, 0, ids, half, V, d, 1.0, 0, table, 0, ws, need)
    R.rollout_embedding_backward(g[half:], 0, ids.flatten()[half:], n - half, V, d, 1.0, 1, table, 0, ws, need)
    want = U.embedding_backward(g.double().cpu().numpy(), ids.cpu().numpy().reshape(-1), V, 1.0)
    size = U.embedding_backward(g.double().abs().cpu().numpy(), ids.cpu().numpy().reshape(-1), V, 1.0)
    count = np.bincount(np.maximum(ids.cpu().numpy().reshape(-1), 0), minlength=V)[:, None]
    assert np.all(np.abs(table.double().cpu().numpy() - want) <= 2.0 ** -24 * (count + 3) * size)


def test_a_decode_step_scored_in_one_graph(step):
    """Draw and score of a decode step's logits captured together, replayed on other logits."""
    S, V = step["S"], step["V"]
    z = step["logits"][:, 0].contiguous()
    u = torch.rand(S, device=DEV)
    tok = torch.empty(S, dtype=torch.int32, device=DEV)
    logp, ent = torch.empty(S, device=DEV), torch.empty(S, device=DEV)
    ids, tops = torch.empty(S, 5, dtype=torch.int32, device=DEV), torch.empty(S, 5, device=DEV)
    need = R.rollout_token_logprobs_workspace(S, V, 5)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)

    def both(stream):
        R.rollout_sample_noalloc(z, S, V, T, 1.0, u, tok, stream)
        R.rollout_token_logprobs(z, 0, V, S, V, T, tok, 5, logp, ent, None, ids, tops, ws, need, stream)

    both(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(torch.cuda.current_stream().cuda_stream)
    for t in range(1, 4):
        z.copy_(step["logits"][:, t])
        u.copy_(torch.rand(S, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (tok, logp, ent, ids, tops)]
        both(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        for a, b in zip(got, (tok, logp, ent, ids, tops)):
            assert torch.equal(a, b)
        o = U.token_logprobs(z.double().cpu().numpy(), T, tok.cpu().numpy(), 5)
        assert np.array_equal(ids.cpu().numpy(), o["ids"])
        assert np.abs(logp.cpu().numpy() - o["logp"]).max() <= 2.0 ** -18
