"""Pins of oracle/layers.py: torch's autograd in float64, finite differences, and worked cases."""
import numpy as np
import pytest
import torch

from oracle import layers as L


def _case(seed, nq, nk, H=4, K=2, hd=8):
    r = np.random.default_rng(seed)
    return r.normal(size=(nq, H, hd)), r.normal(size=(nk, K, hd)), r.normal(size=(nk, K, hd)), r.normal(size=(nq, H, hd))


@pytest.mark.parametrize("nq,nk,causal", [(5, 5, True), (3, 7, True), (4, 6, False), (1, 9, True), (1, 1, True), (6, 6, False)])
def test_attention_is_torchs(nq, nk, causal):
    q, k, v, g = _case(nq * 10 + nk, nq, nk)
    out, lse = L.attention(q, k, v, [(0, nq)], [(0, nk)], 0.3, causal)
    tq, tk, tv = (torch.tensor(x, requires_grad=True) for x in (q, k, v))
    mask = torch.tensor(L._attended(nq, nk, causal))
    rep = lambda x: x.repeat_interleave(2, 1).transpose(0, 1)  # noqa: E731
    s = (tq.transpose(0, 1) @ rep(tk).transpose(1, 2)) * 0.3
    s = s.masked_fill(~mask, -torch.inf)
    o = (torch.softmax(s, 2) @ rep(tv)).transpose(0, 1)
    np.testing.assert_allclose(out, o.detach(), rtol=1e-12, atol=1e-13)
    np.testing.assert_allclose(lse, torch.logsumexp(s, 2).detach(), rtol=1e-12)
    o.backward(torch.tensor(g))
    for got, want in zip(L.attention_backward(q, k, v, out, lse, g, [(0, nq)], [(0, nk)], 0.3, causal), (tq, tk, tv)):
        np.testing.assert_allclose(got, want.grad, rtol=1e-11, atol=1e-12)


def test_queries_without_keys():
    q, k, v, g = _case(1, 5, 2)
    out, lse = L.attention(q, k, v, [(0, 5)], [(0, 2)], 1.0, True)  # query i attends keys 0 .. i - 3
    assert (out[:3] == 0).all() and np.isneginf(lse[:, :3]).all() and np.isfinite(lse[:, 3:]).all()
    np.testing.assert_allclose(out[3], v[0].repeat(2, 0))
    dq, dk, dv = L.attention_backward(q, k, v, out, lse, g, [(0, 5)], [(0, 2)], 1.0, True)
    assert (dq[:3] == 0).all() and np.isfinite(dk).all()
    np.testing.assert_allclose(dv.sum(0), g[3:].reshape(2, 2, 2, 8).sum((0, 2)))  # probabilities of a query sum to 1


def test_sequences_are_apart_and_padding_stays():
    q, k, v, _ = _case(2, 9, 9)
    seqs = L.sequences([0, 4, 9], [3, 5], 9)
    assert seqs == [(0, 3), (4, 5)]
    assert L.sequences([2, 100, 50], None, 9) == [(2, 7), (9, 0)]
    out, lse = L.attention(q, k, v, seqs, seqs, 1.0, True)
    assert np.isnan(out[3]).all() and np.isnan(lse[:, 3]).all()
    alone, _ = L.attention(q[4:], k[4:], v[4:], [(0, 5)], [(0, 5)], 1.0, True)
    np.testing.assert_array_equal(out[4:], alone)


def test_norm_is_torchs():
    r = np.random.default_rng(3)
    h, gain, dy, inner = r.normal(size=(4, 10)), r.normal(size=10), r.normal(size=(4, 10)), r.normal(size=(4, 10))
    y, rstd = L.rms_norm(h, gain, 1e-3)
    th, tg = torch.tensor(h, requires_grad=True), torch.tensor(gain, requires_grad=True)
    ty = torch.nn.functional.rms_norm(th, (10,), tg, 1e-3)
    np.testing.assert_allclose(y, ty.detach(), rtol=1e-12)
    ty.backward(torch.tensor(dy))
    dx, dgain = L.rms_norm_backward(dy, h, gain, rstd, inner)
    np.testing.assert_allclose(dx - inner, th.grad, rtol=1e-10, atol=1e-12)
    np.testing.assert_allclose(dgain, tg.grad, rtol=1e-10)


def test_norm_gradient_by_differences():
    r = np.random.default_rng(4)
    h, gain, dy = r.normal(size=(1, 6)), r.normal(size=6), r.normal(size=(1, 6))
    dx, _ = L.rms_norm_backward(dy, h, gain, L.rms_norm(h, gain, 1e-6)[1], 0.0)
    for i in range(6):
        d = np.zeros((1, 6))
        d[0, i] = 1e-6
        slope = ((L.rms_norm(h + d, gain, 1e-6)[0] - L.rms_norm(h - d, gain, 1e-6)[0]) * dy).sum() / 2e-6
        assert abs(slope - dx[0, i]) < 1e-8


def test_e4m3_values_are_torchs():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(L.e4m3_values(), want)
    assert L.power_scale(448.0) == 1.0 and L.power_scale(448.1) == 2.0 and L.power_scale(0.0) == 2.0 ** -126
    assert L.power_scale(1.75) == 2.0 ** -8 and L.power_scale(1.0) == 2.0 ** -8 and L.power_scale(0.875001) == 2.0 ** -8
    v = L.e4m3_values()[:127]
    np.testing.assert_array_equal(np.diff(v), L.spacing(v[:-1]))


def test_adamw_is_torchs():
    r = np.random.default_rng(5)
    p, m, v = r.normal(size=20), np.zeros(20), np.zeros(20)
    tp = torch.nn.Parameter(torch.tensor(p))
    opt = torch.optim.AdamW([tp], lr=1e-2, betas=(0.9, 0.97), eps=1e-8, weight_decay=0.1)
    for step in range(1, 6):
        g = r.normal(size=20)
        tp.grad = torch.tensor(g)
        opt.step()
        p, m, v = L.adamw(p, g, m, v, 1e-2, 0.9, 0.97, 1e-8, step, 0.1)
        np.testing.assert_allclose(p, tp.detach(), rtol=1e-12)


def test_random_bits():
    # finalisers at published points: SplitMix64's first output from state 0, MurmurHash3's of 1
    assert L._finish64(L._GOLD) == 0xE220A8397B1DCDAF
    assert int(L._finish32(np.uint64(1))) == 0x514E28B7 and int(L._finish32(np.uint64(0))) == 0
    a = L.adamw_bits(7, 3, 2, np.arange(1 << 16))
    for x in a:
        assert x.min() >= 0 and x.max() < 1 << 16
        # mean of 65,536 draws: sigma 74; eight of them
        assert abs(x.mean() - 32767.5) < 8 * 74
    assert abs(np.corrcoef(a)[0, 1]) < 8 / 256 and abs(np.corrcoef(a)[0, 2]) < 8 / 256
    assert any((x != y).any() for x, y in zip(a, L.adamw_bits(7, 4, 2, np.arange(1 << 16))))
