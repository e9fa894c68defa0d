"""Packed attention and its gradient against the definition in float64, with bounds from the roundings that the kernels make."""
import numpy as np
import pytest
import torch

import paper_2608_11226_amd as R
from layer_cases import DEV, SENTINEL, Attention, wide
from oracle import layers as L

pytestmark = pytest.mark.gpu

RAGGED = [1, 33, 0, 64, 129, 2, 200]
CASES = {
    "one token": dict(dtype="bf16", heads=4, kv=2, hd=64, q_lens=[1]),
    "single tokens": dict(dtype="fp32", heads=4, kv=4, hd=32, q_lens=[1] * 70),
    "tiny": dict(dtype="fp32", heads=4, kv=4, hd=32, q_lens=[32] * 8),
    "around tiles fp32": dict(dtype="fp32", heads=2, kv=1, hd=128, q_lens=[31, 32, 33, 63, 64, 65, 127, 128, 129]),
    "around tiles bf16": dict(dtype="bf16", heads=2, kv=1, hd=128, q_lens=[31, 32, 33, 63, 64, 65, 127, 128, 129]),
    "ragged 32": dict(dtype="bf16", heads=4, kv=4, hd=32, q_lens=RAGGED),
    "ragged 64": dict(dtype="bf16", heads=14, kv=2, hd=64, q_lens=RAGGED, fused=True),
    "ragged 128": dict(dtype="bf16", heads=7, kv=1, hd=128, q_lens=RAGGED, fused=True),
    "ragged 64 fp32": dict(dtype="fp32", heads=6, kv=2, hd=64, q_lens=RAGGED, fused=True),
    "places of equal size": dict(dtype="bf16", heads=4, kv=2, hd=128, q_lens=[50, 0, 130, 1], room=13),
    "lengths below the places": dict(dtype="fp32", heads=4, kv=2, hd=32, q_lens=[50, 0, 130, 1], room=13, fused=True),
    "not causal": dict(dtype="bf16", heads=4, kv=2, hd=128, q_lens=[70, 1, 130], causal=False),
    "not causal fp32": dict(dtype="fp32", heads=2, kv=2, hd=64, q_lens=[70, 1, 130], causal=False),
    "last queries": dict(dtype="bf16", heads=8, kv=1, hd=128, q_lens=[1, 3, 40, 130], k_lens=[300, 3, 65, 400]),
    "last queries fp32": dict(dtype="fp32", heads=4, kv=2, hd=128, q_lens=[1, 3, 40], k_lens=[300, 3, 65], room=4),
    "one token over many keys": dict(dtype="bf16", heads=16, kv=1, hd=128, q_lens=[1] * 5, k_lens=[1, 63, 64, 2000, 4097]),
    "one token over many keys fp32": dict(dtype="fp32", heads=4, kv=2, hd=64, q_lens=[1] * 3, k_lens=[1, 700, 2049]),
    "few tokens over many keys": dict(dtype="bf16", heads=4, kv=2, hd=64, q_lens=[5, 33], k_lens=[3001, 777], causal=False),
    "rows without keys": dict(dtype="bf16", heads=4, kv=2, hd=64, q_lens=[100, 40, 5, 0], k_lens=[30, 0, 5, 9]),
    "rows without keys fp32": dict(dtype="fp32", heads=4, kv=2, hd=128, q_lens=[100, 40, 5, 0], k_lens=[30, 0, 5, 9]),
    "no keys at all": dict(dtype="bf16", heads=2, kv=2, hd=128, q_lens=[20, 3], k_lens=[0, 0], causal=False),
    "no queries at all": dict(dtype="bf16", heads=2, kv=2, hd=128, q_lens=[0, 0], k_lens=[200, 3]),
    "more queries than keys, not causal": dict(dtype="bf16", heads=4, kv=1, hd=32, q_lens=[300], k_lens=[7], causal=False),
    "sharp": dict(dtype="bf16", heads=2, kv=1, hd=128, q_lens=[150], spread=2.0, scale=0.5),
    "sharp fp32": dict(dtype="fp32", heads=2, kv=1, hd=64, q_lens=[150], spread=2.0, scale=0.5),
    "long": dict(dtype="bf16", heads=2, kv=1, hd=128, q_lens=[1500, 700]),
    "many sequences": dict(dtype="bf16", heads=2, kv=1, hd=64, q_lens=[(7 * i) % 41 for i in range(300)]),
    "more heads than a multiple of dies": dict(dtype="bf16", heads=11, kv=11, hd=32, q_lens=[140]),
}


@pytest.mark.parametrize("name", CASES)
def test_attention(name):
    c = Attention(**CASES[name])
    out, lse = c.forward()
    torch.cuda.synchronize()
    c.check_forward(out, lse)


@pytest.mark.parametrize("name", CASES)
def test_attention_backward(name):
    c = Attention(**CASES[name])
    out, lse = c.forward()
    grads = c.backward(out, lse)
    torch.cuda.synchronize()
    c.check_backward(grads, out, lse)


@pytest.mark.parametrize("dtype,heads,kv,hd", [("bf16", 17, 1, 64), ("bf16", 66, 2, 128), ("fp32", 40, 1, 32), ("bf16", 64, 1, 32),
                                               ("fp32", 64, 1, 128), ("bf16", 128, 2, 64)])
def test_many_heads_to_a_keys(dtype, heads, kv, hd):
    """More than 16 query heads share a key's, and more than the rows of a tile: a tile lies within a token, or in two."""
    c = Attention(dtype, heads, kv, hd, [1, 19, 0, 66, 7], [40, 19, 3, 70, 2])
    out, lse = c.forward()
    c.check_forward(out, lse)
    c.check_backward(c.backward(out, lse), out, lse)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_the_same_bits_again(dtype):
    c = Attention(dtype, 8, 2, 128, [300, 65, 1, 130])
    first = [x.clone() for x in (*c.forward(), *c.backward(*c.forward()))]
    for _ in range(3):
        again = (*c.forward(), *c.backward(*c.forward()))
        assert all(torch.equal(a.view(torch.uint8), b.contiguous().view(torch.uint8)) for a, b in zip(first, map(torch.clone, again)))


@pytest.mark.parametrize("heads,kv,hd,q_lens,k_lens", [
    (4, 4, 32, [3, 3], [68, 68]), (14, 2, 64, [1, 2, 1], [60, 200, 1]), (28, 4, 128, [5, 1, 0, 7], None), (4, 1, 128, [1], [900])])
def test_few_pairs_lose_nothing_by_the_second_product(heads, kv, hd, q_lens, k_lens):
    """Up to 16,384 pairs of a query and a key: what bf16 rounds off the probabilities is multiplied as well."""
    c = Attention("bf16", heads, kv, hd, q_lens, k_lens)
    assert c.n_q * heads * c.n_k / len(q_lens) <= 16384
    c.few = True
    out, lse = c.forward()
    c.check_forward(out, lse)
    c.check_backward(c.backward(out, lse), out, lse)


def test_gradients_by_differences():
    """The loss sum(out * w) moves as the gradient says, along a random direction, by the kernel's own forward pass."""
    c = Attention("fp32", 4, 2, 64, [40, 70], [45, 70], scale=0.2)
    out, lse = c.forward()
    used = [~c.unused(s, n) for s, n in ((c.q_seqs, c.n_q), (c.k_seqs, c.n_k), (c.k_seqs, c.n_k))]
    dq, dk, dv = c.backward(out, lse)

    def loss():
        o, _ = c.forward()
        return float((o[used[0]].double() * c.grad_out[used[0]].double()).sum())

    for x, d, u in zip((c.q, c.k, c.v), (dq, dk, dv), used):
        way = torch.randn(x.shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(5))
        slope = float((d[u].double() * way[u].double()).sum())
        h = 2.0 ** -8
        keep = x.clone()
        x += h * way
        up = loss()
        x.copy_(keep)
        x -= h * way
        down = loss()
        x.copy_(keep)
        # third order: h^2 / 6 of a derivative of the size of the slope's; the outputs' roundings over 2 h: 2^-24 sqrt(28,160) / 2 h
        assert abs((up - down) / (2 * h) - slope) <= 1e-2 * abs(slope) + 0.05, (up, down, slope)


def test_a_sequence_of_nan_stays_alone():
    c = Attention("bf16", 4, 2, 64, [30, 40, 50])
    out, lse = c.forward()
    grads = [g.clone() for g in c.backward(out, lse)]
    want, z = out.clone(), lse.clone()
    c.k[30:70] = float("nan")
    c.v[30:70] = float("inf")
    got, got_z = c.forward()
    other = [g.clone() for g in c.backward(got, got_z)]
    for a, b in [(got, want), (got_z.t(), z.t()), *zip(other, grads)]:
        assert torch.equal(a[:30], b[:30]) and torch.equal(a[70:120], b[70:120])
    assert got[30:70].isnan().all()


def test_places_out_of_range_are_taken_into_it():
    c = Attention("bf16", 2, 1, 64, [40, 30])
    out, lse = c.forward()
    c.q_starts.copy_(torch.tensor([0, 40, 1 << 30], dtype=torch.int32))
    c.q_lens = torch.tensor([1 << 30, 30], dtype=torch.int32, device=DEV)
    got, got_z = c.forward()
    assert torch.equal(got, out) and torch.equal(got_z, lse)
    grads = c.backward(got, got_z)
    c.check_backward(grads, got, got_z)
    for starts in ([70, 0, 40], [-5, -3, -1], [73, 80, 90], [-(1 << 31), (1 << 31) - 1, 0]):
        c.q_starts.copy_(torch.tensor(starts, dtype=torch.int64).to(torch.int32))
        c.backward(*c.forward())
        torch.cuda.synchronize()


def test_on_another_stream_and_two_at_once():
    c = Attention("bf16", 8, 2, 128, [300, 65, 1, 130])
    d = Attention("bf16", 8, 2, 128, [200, 165, 10, 30], seed=1)
    wants = [[t.clone() for t in (*x.forward(), *x.backward(*x.forward()))] for x in (c, d)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for x, s in zip((c, d), streams):
        with torch.cuda.stream(s):
            o = x.forward()
            got.append((*o, *x.backward(*o)))
    torch.cuda.synchronize()
    for want, have in zip(wants, got):
        for a, b in zip(want, have):
            assert torch.equal(a, b)


def test_in_a_graph():
    c = Attention("bf16", 8, 2, 128, [300, 65, 1, 130], fused=True)
    out, lse = c.forward()
    grads = c.backward(out, lse)
    keep = [x.clone() for x in (out, lse, *grads)]
    ws = torch.empty(R.rollout_attention_backward_workspace(c.shape), dtype=torch.uint8, device=DEV)
    fw = torch.empty(max(1, R.rollout_attention_workspace(c.shape)), dtype=torch.uint8, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            c.forward(out=out, lse=lse, ws=fw)
            c.backward(out, lse, grads, ws)
    for i in range(4):
        for x in (out, lse, *grads):
            x.fill_(SENTINEL)
        ws.fill_(i)
        # the places are read at every replay
        if i == 2:
            c.q_starts.copy_(torch.tensor([0, 250, 365, 366, 496], dtype=torch.int32))
            eager = [x.clone() for x in (lambda o: (*o, *c.backward(*o)))(c.forward())]
            torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want = keep if i < 2 else eager
        for a, b in zip((out, lse, *grads), want):
            assert torch.equal(a, b), i


def test_large_values_of_masked_keys_do_not_matter():
    """Keys behind a query score higher than anything it attends."""
    c = Attention("bf16", 2, 2, 64, [130])
    c.k[65:] = 50.0
    c.q[:65] = c.q[:65].abs()
    out, lse = c.forward()
    c.check_forward(out, lse)
    c.check_backward(c.backward(out, lse), out, lse)


def test_rows_behind_4_gib():
    """Keys and queries whose places are more than 2^32 bytes behind the first, in rows far apart."""
    H, K, hd, stride, n = 4, 2, 128, 4096, 600000
    s = torch.cuda.current_stream().cuda_stream
    big, grads = (torch.zeros((n, stride), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    lens, first = [70, 1, 130], [10, 550000, 599000]
    c = Attention("bf16", H, K, hd, lens)
    wq, wk = H * hd, K * hd
    cols = [slice(0, wq), slice(wq, wq + wk), slice(wq + wk, wq + 2 * wk)]
    at = 0
    for f, m in zip(first, lens):
        for col, x in zip(cols, (c.q, c.k, c.v)):
            big[f:f + m, col] = x[at:at + m]
        at += m
    shape = R.AttentionShape(dtype=1, n_heads=H, n_kv_heads=K, head_dim=hd, n_seqs=3, n_q=n, n_k=n, causal=1, scale=c.scale)
    starts = torch.tensor(first + [n], dtype=torch.int32, device=DEV)
    n_lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
    out, dout = torch.zeros((n, wq), dtype=torch.bfloat16, device=DEV), torch.zeros((n, wq), dtype=torch.bfloat16, device=DEV)
    lse = torch.zeros((H, n), device=DEV)
    at = 0
    for f, m in zip(first, lens):
        dout[f:f + m] = c.grad_out[at:at + m]
        at += m
    need = max(R.rollout_attention_workspace(shape), R.rollout_attention_backward_workspace(shape))
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    views = [v for col in cols for v in (big[:, col], stride)]
    R.rollout_attention(shape, *views, starts, n_lens, None, None, out, wq, lse, ws, need, s)
    R.rollout_attention_backward(shape, *views, starts, n_lens, None, None, out, wq, lse, dout, wq,
                                 *[v for col in cols for v in (grads[:, col], stride)], ws, need, s)
    c_out, c_lse = c.forward()
    c_grads = c.backward(c_out, c_lse)
    c.check_forward(c_out, c_lse)
    c.check_backward(c_grads, c_out, c_lse)
    # (the two calls may cut walks into parts otherwise: within the bounds of both)
    pick = torch.cat([torch.arange(f, f + m, device=DEV) for f, m in zip(first, lens)])
    here = torch.full((c.n_q, wq), SENTINEL, dtype=torch.bfloat16, device=DEV)
    here[:len(pick)] = out[pick]
    z = torch.full((H, c.n_q), SENTINEL, device=DEV)
    z[:, :len(pick)] = lse[:, pick]
    c.check_forward(here, z)
    got = []
    for col in cols:
        x = torch.full((c.n_q, col.stop - col.start), SENTINEL, dtype=torch.bfloat16, device=DEV)
        x[:len(pick)] = grads[pick][:, col]
        got.append(x)
    c.check_backward(got, here, z)
    assert not grads[100:500000].any() and not out[100:500000].any()


def test_scores_of_minus_infinity():
    c = Attention("fp32", 2, 2, 32, [40])
    c.q[:, 0], c.k[:20, 0] = 1.0, -float("inf")
    c.q[:, 32], c.k[:20, 32] = 1.0, -float("inf")
    out, lse = c.forward()
    # the first 20 queries see nothing else, the others only the keys from 20 on
    assert (out[:20] == 0).all() and torch.isneginf(lse[:, :20]).all()
    q, k, v = (x[20:40] for x in (c.q, c.k, c.v))
    want, z = L.attention(*(wide(x).reshape(20, 2, 32) for x in (q, k, v)), [(0, 20)], [(0, 20)], c.scale, True)
    np.testing.assert_allclose(wide(out)[20:40], want.reshape(20, 64), rtol=1e-5, atol=1e-6)
    np.testing.assert_allclose(wide(lse)[:, 20:40], z, rtol=1e-5, atol=1e-5)
