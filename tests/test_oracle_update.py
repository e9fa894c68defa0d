"""The update side's float64 definitions against torch's autograd in float64, differences, and cases worked by hand."""
import math

import numpy as np
import pytest
import torch

from oracle import update as U


def _rows(n=5, V=23, seed=0):
    rng = np.random.default_rng(seed)
    return rng.standard_normal((n, V)) * 3, rng.integers(0, V, n), rng


@pytest.mark.parametrize("T", [1.0, 0.5, 1.25])
def test_logprobs_and_gradient_match_autograd(T):
    z, tok, rng = _rows()
    z[2, :7] = -np.inf
    tok[2] = 9
    g, h = rng.standard_normal(5), rng.standard_normal(5)
    zt = torch.tensor(z, requires_grad=True)
    lp = torch.log_softmax(zt / T, 1)
    logp = lp.gather(1, torch.tensor(tok)[:, None])[:, 0]
    p = lp.exp()
    H = -torch.where(p > 0, p * lp.clamp(min=-1e300), 0.0).sum(1)
    got = U.token_logprobs(z, T, tok, 4)
    np.testing.assert_allclose(got["logp"], logp.detach(), atol=1e-13)
    np.testing.assert_allclose(got["entropy"], H.detach(), atol=1e-13)
    np.testing.assert_allclose(got["stats"][:, 0] / T + got["stats"][:, 1], torch.logsumexp(zt / T, 1).detach(), atol=1e-13)
    want_ids = np.argsort(-z, axis=1, kind="stable")[:, :4]
    assert np.array_equal(got["ids"], want_ids)
    np.testing.assert_allclose(got["top_logp"], np.take_along_axis(lp.detach().numpy(), want_ids, 1), atol=1e-13)
    dz = U.token_logprobs_backward(z, T, tok, got["stats"], got["entropy"], g, h)
    # differences (autograd gives NaN through the masked entropy terms)
    f = lambda q: (lambda o: (g * o["logp"] + h * o["entropy"]).sum())(U.token_logprobs(q, T, tok))
    for r, i in [(0, 0), (1, int(tok[1])), (2, 9), (2, 20), (4, 5)]:
        up, dn = z.copy(), z.copy()
        up[r, i] += 1e-5
        dn[r, i] -= 1e-5
        assert dz[r, i] == pytest.approx((f(up) - f(dn)) / 2e-5, abs=1e-8)
    assert np.all(dz[2, :7] == 0)
    (torch.tensor(g) * logp).sum().backward()
    np.testing.assert_allclose(U.token_logprobs_backward(z, T, tok, got["stats"], got["entropy"], g), zt.grad, atol=1e-13)


def test_logprobs_by_hand():
    z = np.array([[0.0, math.log(3.0), -np.inf, 0.0], [-np.inf] * 4, [1, 2, np.nan, 0], [1, 2, np.inf, 0], [5, 5, 5, 5], [1, 2, 3, 4]])
    o = U.token_logprobs(z, 1.0, [1, 2, 0, 0, -1, 4], 3)
    assert o["logp"][0] == pytest.approx(math.log(0.6))
    assert o["entropy"][0] == pytest.approx(-(0.6 * math.log(0.6) + 0.4 * math.log(0.2)))
    assert o["ids"].tolist() == [[1, 0, 3], [0, 1, 2], [-1] * 3, [-1] * 3, [-1] * 3, [3, 2, 1]]
    assert o["logp"][1] == -np.inf and o["entropy"][1] == 0
    assert np.isnan(o["logp"][[2, 3, 5]]).all() and o["logp"][4] == 0 and not np.isnan(o["entropy"][5])


@pytest.mark.parametrize("mean", [0, 1, 2])
@pytest.mark.parametrize("parts", ["all", "no ref", "no old", "no entropy"])
def test_policy_loss_matches_autograd(mean, parts):
    rng = np.random.default_rng(7)
    S, N = 6, 9
    old = -rng.exponential(1.0, (S, N))
    lp = old + 0.4 * rng.standard_normal((S, N))
    ref = old + 0.3 * rng.standard_normal((S, N)) if parts != "no ref" else None
    H = rng.random((S, N)) if parts != "no entropy" else None
    adv = rng.standard_normal(S)
    lengths = np.array([0, 1, 9, 4, 20, 7])
    if parts == "no old":
        old = None
    args = (np.float32(0.2), np.float32(0.3), np.float32(0.05), np.float32(0.01))
    loss, stats, dlp, dH = U.policy_loss(lp, old, ref, H, adv, lengths, *args, mean)
    x = torch.tensor(lp, requires_grad=True)
    h = torch.tensor(H if H is not None else np.zeros((S, N)), requires_grad=True)
    A = torch.tensor(adv)[:, None]
    L = np.minimum(lengths, N)
    live = torch.arange(N)[None] < torch.tensor(L)[:, None]
    r = torch.exp(x - (torch.tensor(old) if old is not None else x.detach()))
    lo, hi, b, c = (float(a) for a in args)
    surr = torch.minimum(r * A, r.clamp(1 - lo, 1 + hi) * A)
    kl = torch.zeros_like(r)
    if ref is not None:
        y = torch.tensor(ref) - x
        kl = torch.exp(y) - y - 1
    tok = torch.where(live, -surr + b * kl - c * h, 0.0)
    if mean == 0:
        want = (tok.sum(1) / torch.tensor(np.maximum(L, 1))).mean()
    elif mean == 1:
        want = tok.sum() / L.sum()
    else:
        want = tok.sum() / (S * N)
    want.backward()
    assert loss == pytest.approx(want.item(), abs=1e-13)
    np.testing.assert_allclose(dlp, x.grad, atol=1e-14)
    np.testing.assert_allclose(dH, h.grad if H is not None else -c * (dH != 0) * np.abs(dH) / c, atol=1e-14)
    assert stats[0] == pytest.approx(r[live].mean().item())
    assert stats[1] == pytest.approx(kl[live].mean().item(), abs=1e-14)


def test_policy_loss_without_tokens():
    loss, stats, d, e = U.policy_loss(np.zeros((2, 3)), None, None, None, [1.0, 2.0], [0, 0], 0.2, 0.2, 0.0, 0.0, 1)
    assert loss == 0 and not stats.any() and not d.any() and not e.any()


def test_embedding_and_gradient_match_autograd():
    rng = np.random.default_rng(3)
    E = rng.standard_normal((11, 6))
    tok = np.array([3, 3, 0, 10, 3, -1, 7])
    w = torch.tensor(E, requires_grad=True)
    g = rng.standard_normal((7, 6))
    out = torch.nn.functional.embedding(torch.tensor(np.maximum(tok, 0)), w) * 1.5 * torch.tensor(tok >= 0)[:, None]
    np.testing.assert_allclose(U.embedding(E, tok, 1.5), out.detach(), atol=1e-15)
    (out * torch.tensor(g)).sum().backward()
    np.testing.assert_allclose(U.embedding_backward(g, tok, 11, 1.5), w.grad, atol=1e-14)
    np.testing.assert_allclose(U.embedding_backward(g, tok, 11, 1.5, E), w.grad.numpy() + E, atol=1e-14)
    assert np.isnan(U.embedding(E, [11], 1.0)).all() and not U.embedding_backward(g[:1], [11], 11, 1.0).any()


@pytest.mark.filterwarnings("ignore:overflow")
def test_policy_loss_terms_without_a_coefficient():
    lp, ref = np.array([[-np.inf, -1.0, -2.0]]), np.array([[-1.0, -np.inf, 800.0]])
    f = lambda r, b, e: U.policy_loss(lp, np.full((1, 3), -1.0), r, e, [0.5], None, 0.2, 0.2, b, 0.0, 0)
    want, (got, stats, dlp, _) = f(None, 0.0, None), f(ref, 0.0, np.full((1, 3), np.inf))
    assert got == want[0] and np.isfinite(got) and np.array_equal(dlp, want[2])
    assert np.isposinf(stats[1]) and np.isposinf(stats[4])
    loss, _, dlp, _ = f(ref, 0.1, None)
    assert np.isposinf(loss) and np.isneginf(dlp[0, 0])
