"""The clipped group loss and its gradients against the float64 definition.

Tolerances (eps = 2^-24): the ratio's exponent is rounded once, the exponential is good to two last bits, so r is off by
(|d| + 4) eps of itself; e^x - 1 by its two last bits and by x's rounding; what follows are four roundings more.  Sums
are fp64."""
import numpy as np
import pytest

import paper_2608_11226_amd as R
from gpu_helpers import log, to_dev
from oracle import update as U

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 2.0 ** -24


def inputs(S, N, seed):
    rng = np.random.default_rng(seed)
    f = np.float32
    old = -rng.exponential(1.0, (S, N)).astype(f)
    lp = (old + 0.3 * rng.standard_normal((S, N))).astype(f)
    ref = (old + 0.3 * rng.standard_normal((S, N))).astype(f)
    H = rng.random((S, N)).astype(f) * 3
    adv = rng.standard_normal(S).astype(f)
    lengths = rng.integers(0, N + 1, S).astype(np.int32)
    if S > 2:
        adv[1], lengths[0], lengths[2] = 0.0, 0, N
    return lp, old, ref, H, adv, lengths


def run(lp, old, ref, H, adv, lengths, lo, hi, kl, ent, mean, ws=None, stream=None, out=None):
    S, N = lp.shape
    need = R.grpo_policy_loss_workspace(S, N)
    ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV) if ws is None else ws
    out = out or [torch.full(k, 7.0, device=DEV) for k in ((1,), (5,), (S, N), (S, N))]
    R.grpo_policy_loss(lp, old, ref, H, adv, lengths, S, N, lo, hi, kl, ent, mean, out[0], out[1], out[2],
                       out[3] if H is not None else None, ws, need, stream)
    return out


def check(out, lp, old, ref, H, adv, lengths, lo, hi, kl, ent, mean):
    S, N = lp.shape
    loss, stats, dlp, dH = U.policy_loss(lp, old, ref, H, adv, lengths, lo, hi, kl, ent, mean)
    got = [x.cpu().numpy().astype(np.float64) for x in out]
    L = np.full(S, N) if lengths is None else np.clip(lengths, 0, N)
    live = np.arange(N)[None] < L[:, None]
    w = np.where(live, {0: 1.0 / (S * np.maximum(L, 1))[:, None], 1: 1.0 / max(1, L.sum()), 2: 1.0 / (S * N)}[mean], 0.0)
    A = np.abs(adv.astype(np.float64))[:, None]
    d = np.where(live, lp.astype(np.float64) - (old if old is not None else lp), 0.0)
    r = np.exp(d)
    x = np.where(live, ref.astype(np.float64) - lp, 0.0) if ref is not None else np.zeros((S, N))
    ex = np.expm1(x)
    e_r = EPS * r * (np.abs(d) + 4)
    e_ex = EPS * (np.abs(ex) * 3 + np.abs(x) * np.exp(x))
    e_kl = e_ex + EPS * (np.abs(ex - x) + np.abs(x))
    Hs = np.where(live, H, 0.0) if H is not None else 0.0
    size = A * np.maximum(r, 1 + hi) + abs(kl) * np.abs(ex - x) + abs(ent) * Hs
    e_tok = A * e_r + abs(kl) * e_kl + 4 * EPS * size
    assert abs(got[0][0] - loss) <= (w * (e_tok + EPS * size)).sum() + EPS * abs(loss)
    n = max(1, L.sum())
    for i, e in enumerate((e_r, e_kl, np.zeros((S, N)), np.zeros((S, N)), np.zeros((S, N)))):
        assert abs(got[1][i] - stats[i]) <= (e * live).sum() / n + EPS * abs(stats[i]), f"statistic {i}: {got[1][i]} {stats[i]}"
    e_g = w * (A * e_r + abs(kl) * e_ex + 4 * EPS * (A * r + abs(kl) * np.abs(ex))) + EPS * np.abs(dlp)
    assert np.all(np.abs(got[2] - dlp) <= e_g + 2.0 ** -140)
    assert not got[2][~live].any()
    if H is not None:
        assert np.all(np.abs(got[3] - dH) <= 3 * EPS * np.abs(dH) + 2.0 ** -140)


SIZES = [(1, 1), (1, 7), (3, 1), (5, 3), (4, 4), (64, 512), (7, 1023), (3, 2049), (1000, 2), (33, 130), (2, 9001), (20000, 3), (600000, 1)]


@pytest.mark.parametrize("S,N", SIZES)
def test_sizes_and_means(S, N):
    data = inputs(S, N, S * 1000 + N)
    dev = [to_dev(x, torch) for x in data]
    for mean in (0, 1, 2):
        log(f"policy loss {S} x {N} mean {mean}")
        k = (0.2, 0.28, 0.04, 0.01, mean)
        check(run(*dev, *k), *data, *k)


@pytest.mark.parametrize("S,N", [(1, 1024), (5, 205), (2, 2048), (1, 4095), (17, 241), (4096, 1), (4097, 1), (683, 6), (2, 2049)])
def test_as_many_places_as_one_workgroup_does_and_more(S, N):
    """All inputs, and without lengths, statistics and loss: gradients are the same bits."""
    data = inputs(S, N, S + N)
    dev = [to_dev(x, torch) for x in data]
    for mean in (0, 1, 2):
        log(f"policy loss {S} x {N} mean {mean}")
        k = (0.2, 0.28, 0.04, 0.01, mean)
        out = run(*dev, *k)
        check(out, *data, *k)
        none = run(*dev[:5], None, *k)
        check(none, *data[:5], None, *k)
        need = R.grpo_policy_loss_workspace(S, N)
        ws, grad = torch.empty(need, dtype=torch.uint8, device=DEV), torch.empty(S, N, device=DEV)
        R.grpo_policy_loss(*dev, S, N, *k, None, None, grad, None, ws, need)
        assert torch.equal(grad, out[2])


def test_absent_inputs_and_outputs():
    data = inputs(6, 77, 4)
    dev = [to_dev(x, torch) for x in data]
    for absent in ((1,), (2,), (3,), (5,), (1, 2, 3, 5)):
        d = [None if i in absent else x for i, x in enumerate(data)]
        t = [None if i in absent else x for i, x in enumerate(dev)]
        k = (0.1, 0.5, 0.0 if 2 in absent else 0.3, 0.0 if 3 in absent else -0.2, 0)
        check(run(*t, *k), *d, *k)
    whole = run(*dev, 0.2, 0.2, 0.1, 0.1, 1)
    need = R.grpo_policy_loss_workspace(6, 77)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    for i in range(4):
        out = [torch.full_like(x, 7.0) if j == i else None for j, x in enumerate(whole)]
        R.grpo_policy_loss(*dev, 6, 77, 0.2, 0.2, 0.1, 0.1, 1, *out, ws, need)
        assert torch.equal(out[i], whole[i])


def test_lengths_outside_their_range_and_empty_batches():
    data = list(inputs(5, 40, 8))
    data[5] = np.array([-3, 0, 41, 2**31 - 1, 7], dtype=np.int32)
    dev = [to_dev(x, torch) for x in data]
    for mean in (0, 1, 2):
        check(run(*dev, 0.2, 0.2, 0.1, 0.1, mean), *data, 0.2, 0.2, 0.1, 0.1, mean)
    dev[5] = torch.zeros(5, dtype=torch.int32, device=DEV)
    for mean in (0, 1, 2):
        out = run(*dev, 0.2, 0.2, 0.1, 0.1, mean)
        assert not any(x.any() for x in out)


def test_what_is_behind_the_completions_is_not_used():
    data = inputs(9, 50, 3)
    dev = [to_dev(x, torch) for x in data]
    behind = torch.arange(50, device=DEV)[None] >= dev[5][:, None]
    want = run(*dev, 0.2, 0.2, 0.1, 0.1, 0)
    for i in range(4):
        dev[i][behind] = float("nan")
    got = run(*dev, 0.2, 0.2, 0.1, 0.1, 0)
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_ratios_that_overflow_and_clipping_borders():
    lp = np.array([[0.0, 100.0, -100.0, 0.0, np.log(1.2), 0.0]], dtype=np.float32).repeat(3, 0)
    old = np.array([[0.0, 0.0, 0.0, 100.0, 0.0, np.log1p(0.25)]], dtype=np.float32).repeat(3, 0)
    adv = np.array([1.0, -1.0, 0.0], dtype=np.float32)
    out = run(*(to_dev(x, torch) if x is not None else None for x in (lp, old, None, None, adv, None)), 0.2, 0.25, 0.0, 0.0, 1)
    g = out[2].cpu().numpy()
    # A > 0: clipped above; A < 0: the unbounded side; A = 0: nothing, even where the ratio is infinite
    assert g[0, 1] == 0 and np.isposinf(g[1, 1]) and not g[2].any()
    assert np.isposinf(out[0].item()) and np.isposinf(out[1][0].item())
    # ratios of e^-100 have underflown towards zero; clipped where A < 0
    assert abs(g[0, 2]) <= 1e-40 and g[1, 2] == 0 and g[1, 3] == 0
    d = lp.astype(np.float64) - old
    high = (adv[:, None] > 0) & (np.exp(np.minimum(d, 700)) > 1.25)
    low = (adv[:, None] < 0) & (np.exp(np.minimum(d, 700)) < 1 - float(np.float32(0.2)))
    assert out[1][2].item() == np.float32(low.mean()) and out[1][3].item() == np.float32(high.mean())


def test_unaligned_buffers():
    data = inputs(5, 37, 11)
    dev = []
    for x in data:
        flat = torch.empty(x.size + 3, dtype=torch.from_numpy(x).dtype, device=DEV)
        flat[3:] = to_dev(x.reshape(-1), torch)
        dev.append(flat[3:].view(x.shape))
    S, N = 5, 37
    out = [torch.full((n + 5,), 7.0, device=DEV)[1:1 + n].view(k) for n, k in ((1, (1,)), (5, (5,)), (S * N, (S, N)), (S * N, (S, N)))]
    check(run(*dev, 0.2, 0.3, 0.1, 0.1, 1, out=out), *data, 0.2, 0.3, 0.1, 0.1, 1)


def test_gradient_matches_differences():
    """Differences of the kernel's own loss along each token, away from the borders."""
    S, N = 2, 3
    lp, old, ref, H, adv, _ = inputs(S, N, 21)
    lp = (old + np.array([[0.05, -0.1, 0.02], [0.1, 0.0, -0.05]])).astype(np.float32)
    dev = [to_dev(x, torch) for x in (lp, old, ref, H, adv)] + [None]
    out = run(*dev, 0.2, 0.2, 0.5, 0.1, 2)
    step = 2.0 ** -7
    for which, grad in ((0, out[2]), (3, out[3])):
        for s in range(S):
            for t in range(N):
                val = []
                for sgn in (1, -1):
                    moved = list(dev)
                    moved[which] = dev[which].clone()
                    moved[which][s, t] += sgn * step
                    val.append(run(*moved, 0.2, 0.2, 0.5, 0.1, 2)[0].item())
                # the loss is good to 2^-22 or so, its third derivative along a token below 4
                assert grad[s, t].item() == pytest.approx((val[0] - val[1]) / (2 * step), abs=2.0 ** -21 / step + 4 * step * step / 6)


def test_repeats_and_graphs():
    data = inputs(40, 3000, 5)
    dev = [to_dev(x, torch) for x in data]
    a, b = run(*dev, 0.2, 0.28, 0.04, 0.01, 1), run(*dev, 0.2, 0.28, 0.04, 0.01, 1)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    made = []
    for i in range(2):
        out = [torch.empty_like(x) for x in a]
        ws = torch.empty(R.grpo_policy_loss_workspace(40, 3000), dtype=torch.uint8, device=DEV)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(*dev, 0.2, 0.28, 0.04, 0.01, 1, ws=ws, stream=torch.cuda.current_stream().cuda_stream, out=out)
        made.append((graph, out))
    for replay in range(3):
        dev[0].add_(0.01 * torch.randn_like(dev[0]))
        dev[5].copy_(torch.randint(0, 3001, (40,), device=DEV, dtype=torch.int32))
        want = run(*dev, 0.2, 0.28, 0.04, 0.01, 1)
        for graph, out in made:
            graph.replay()
        torch.cuda.synchronize()
        for graph, out in made:
            assert all(torch.equal(x, y) for x, y in zip(want, out)), replay


@pytest.mark.parametrize("mean", [0, 1, 2])
def test_terms_without_a_coefficient_are_left_out(mean):
    """Penalties that overflow, masked ids (log p -inf) and entropies that are not finite, with coefficients of 0: loss and
    gradients are those of the call without them, the statistics are still theirs."""
    S, N = 4, 6
    lp, old, ref, H, adv, _ = inputs(S, N, 33)
    lp[0, 1], lp[2, 3] = -np.inf, -np.inf        # x = inf
    ref[1, 2] = lp[1, 2] + 90                    # e^x is past fp32
    ref[3, 0] = -np.inf                          # x = -inf
    dev = [to_dev(x, torch) for x in (lp, old, ref, H, adv)] + [None]
    want = run(dev[0], dev[1], None, None, dev[4], None, 0.2, 0.28, 0.0, 0.0, mean)
    assert torch.isfinite(want[0]).all() and torch.isfinite(want[2]).all()
    got = run(dev[0], dev[1], dev[2], dev[3], dev[4], None, 0.2, 0.28, 0.0, 0.0, mean)
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2]) and not got[3].any()
    assert torch.equal(got[1][[0, 2, 3]], want[1][[0, 2, 3]])
    assert got[1][1].item() == float("inf")      # every one of these penalties is infinite in fp32
    for bad in (float("inf"), float("nan")):
        dev[3][2, 2] = bad
        got = run(dev[0], dev[1], dev[2], dev[3], dev[4], None, 0.2, 0.28, 0.0, 0.0, mean)
        assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
        assert not torch.isfinite(got[1][4])


def test_penalty_of_a_masked_id():
    """log p = -inf under a reference that allows the id: the penalty's limit, and its gradient's."""
    lp = np.array([[-np.inf, -1.0]], dtype=np.float32)
    ref = np.array([[-2.0, -1.5]], dtype=np.float32)
    adv = np.array([0.5], dtype=np.float32)
    out = run(*(to_dev(x, torch) if x is not None else None for x in (lp, lp + 0, ref, None, adv, None)), 0.2, 0.28, 0.1, 0.0, 1)
    assert np.isnan(out[0].item())               # lp and old are both infinite: no ratio
    old = np.array([[-3.0, -1.0]], dtype=np.float32)
    out = run(*(to_dev(x, torch) if x is not None else None for x in (lp, old, ref, None, adv, None)), 0.2, 0.28, 0.1, 0.0, 1)
    loss, stats, dlp, _ = U.policy_loss(lp, old, ref, None, adv, None, 0.2, 0.28, 0.1, 0.0, 1)
    assert out[0].item() == loss == np.inf and out[1][1].item() == stats[1] == np.inf
    assert out[2][0, 0].item() == dlp[0, 0] == -np.inf and abs(out[2][0, 1].item() - dlp[0, 1]) <= 32 * EPS * abs(dlp[0, 1])


@pytest.mark.parametrize("spread", [1e-7, 1e-6, 1e-5, 1e-4, 1e-3, 1e-2, 0.1, 0.25, 0.49999, 0.5, 0.75, 1.0, 3.0])
@pytest.mark.parametrize("random", [True, False])
def test_penalty_of_a_policy_near_its_reference(spread, random):
    """The penalty relative to itself, as the statistic and as all of the loss.  It is about x^2 / 2.  x = ref - lp is rounded
    once (eps, no more than (2 + |x|) eps of the penalty); near zero a polynomial of which each step's rounding counts a third
    at most of the one after it and the coefficients' as much (3 eps), x^2 and the product (2 eps); further out e^x - 1 is off by
    2 eps, which is up to 4.4 times its size (9 eps), and the difference by 1.  The sum and the means: 2 eps.  In all under
    (16 + |x|) eps."""
    rng = np.random.default_rng(int(spread * 1e7))
    S, N = 3, 257
    lp = -rng.exponential(1.0, (S, N)).astype(np.float32) - 0.25
    x = rng.standard_normal((S, N)) if random else rng.choice([-1.0, 1.0], (S, N))
    ref = (lp + spread * x).astype(np.float32)
    x = ref.astype(np.float64) - lp
    exact = np.where(np.abs(x) < 0.01, x ** 2 * (1 / 2 + x / 6 + x ** 2 / 24 + x ** 3 / 120 + x ** 4 / 720), np.expm1(x) - x).mean()
    out = run(*(to_dev(v, torch) if v is not None else None
                for v in (lp, lp + 0, ref, None, np.zeros(S, dtype=np.float32), None)), 0.2, 0.28, 1.0, 0.0, 1)
    bound = (16 + np.abs(x).max()) * EPS * exact
    log(f"penalty near {spread}: {exact:.9g}, off by {abs(out[1][1].item() - exact) / exact / EPS:.2f} eps")
    assert abs(out[1][1].item() - exact) <= bound
    assert abs(out[0].item() - exact) <= bound
