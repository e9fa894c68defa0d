"""Embedding lookup and its gradient against the float64 definitions.

Lookup: one product in fp32 and one rounding to the output's type.  Gradient (eps = 2^-24): a row's k gradients are added
up in fp32 in at most min(k, 640 + k / 4096) steps, each off by eps of the sum of magnitudes at most, then scaled, added
to the old row, and rounded to the table's type."""
import numpy as np
import pytest

import paper_2608_11226_amd as R
from gpu_helpers import log, to_dev
from oracle import update as U

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 2.0 ** -24
TYPE = {"fp32": (torch.float32, R.DTYPE_FP32), "bf16": (torch.bfloat16, R.DTYPE_BF16)}
PAIRS = [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "fp32"), ("bf16", "bf16")]


def matrix(n, d, dtype, rng, offset=0):
    t = torch.empty(offset + n * d, dtype=TYPE[dtype][0], device=DEV)[offset:]
    t.copy_(to_dev(rng.standard_normal(n * d).astype(np.float32), torch))
    return t.view(n, d)


def half(dtype):
    return torch.finfo(TYPE[dtype][0]).eps / 2


@pytest.mark.parametrize("table,out", PAIRS)
@pytest.mark.parametrize("n,V,d", [(1, 1, 1), (3, 7, 5), (64, 50, 8), (65, 1024, 128), (9, 33, 2047), (300, 100, 3584), (2, 5, 8200)])
def test_lookup(n, V, d, table, out):
    rng = np.random.default_rng(n + V + d)
    for offset in (0, 1):
        log(f"lookup {table} -> {out}: {n} of {V} x {d} offset {offset}")
        E = matrix(V, d, table, rng, offset)
        tok = rng.integers(0, V, n).astype(np.int32)
        if n > 2:
            tok[0], tok[1], tok[2] = -1, V, V - 1
        y = torch.full((offset + n * d + 4,), 7.0, dtype=TYPE[out][0], device=DEV)
        R.rollout_embedding(E, TYPE[table][1], V, d, to_dev(tok, torch), n, 1.3, y[offset:offset + n * d], TYPE[out][1])
        got = y[offset:offset + n * d].view(n, d).double().cpu().numpy()
        want = U.embedding(E.double().cpu().numpy(), tok, 1.3)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        assert np.all((np.abs(got - want) <= (half(out) + EPS) * np.abs(want) + 2.0 ** -130) | np.isnan(want))
        assert torch.all(y[offset + n * d:] == 7.0) and torch.all(y[:offset] == 7.0)


def ids(kind, n, V, rng):
    if kind == "same":
        t = np.full(n, V - 1)
    elif kind == "text":
        t = np.minimum((np.exp(rng.random(n) * np.log(V + 1)) - 1).astype(np.int64), V - 1)
    elif kind == "none":
        t = np.full(n, -1)
    else:
        t = rng.integers(0, V, n)
    if n > 10 and kind != "none":
        t[rng.integers(0, n, n // 10)] = -1
        t[n // 2] = V
        t[n // 3] = np.iinfo(np.int32).min
    return t.astype(np.int32)


def grad(g, gdt, tok, V, scale, acc, table, tdt, stream=None, ws=None):
    n, d = g.shape
    need = R.rollout_embedding_backward_workspace(n, V, d)
    ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV) if ws is None else ws
    R.rollout_embedding_backward(g, TYPE[gdt][1], tok, n, V, d, scale, acc, table, TYPE[tdt][1], ws, need, stream)
    return ws


def check_grad(got, g, tok, V, scale, base, tdt):
    num = g.double().cpu().numpy()
    want = U.embedding_backward(num, tok, V, scale, base)
    size = U.embedding_backward(np.abs(num), tok, V, abs(scale))
    k = np.bincount(tok[(tok >= 0) & (tok < V)], minlength=V)[:, None]
    steps = np.minimum(k, 640 + k / 4096) + 2
    old = 0.0 if base is None else np.abs(base)
    assert np.all(np.abs(got - want) <= EPS * steps * size + EPS * old + half(tdt) * np.abs(want) + 2.0 ** -130)
    return k[:, 0]


@pytest.mark.parametrize("kind", ["uniform", "same", "text"])
@pytest.mark.parametrize("n,V,d", [(1, 1, 1), (2, 5, 3), (63, 40, 8), (64, 40, 9), (65, 3, 128), (1000, 600, 100), (4096, 1024, 128),
                                   (4097, 1024, 128), (4200, 511, 40), (9000, 512, 24), (70000, 300, 16), (140000, 40, 33), (3000, 300000, 8),
                                   (6000, 300000, 8), (200, 50, 3584), (5000, 2064, 2049), (6144, 1024, 128), (6145, 1024, 128),
                                   (6145, 300000, 8), (8000, 511, 40), (7000, 2064, 2049)])
def test_gradient(n, V, d, kind):
    rng = np.random.default_rng(n + V)
    tok = ids(kind, n, V, rng)
    td = to_dev(tok, torch)
    for i, (gdt, tdt) in enumerate(PAIRS):
        offset = i % 2
        log(f"gradient {gdt} -> {tdt}: {n} {kind} tokens, {V} x {d} offset {offset}")
        g = matrix(n, d, gdt, rng, offset)
        flat = torch.full((offset + V * d + 4,), 7.0, dtype=TYPE[tdt][0], device=DEV)
        table = flat[offset:offset + V * d].view(V, d)
        grad(g, gdt, td, V, 0.7, 0, table, tdt)
        k = check_grad(table.double().cpu().numpy(), g, tok, V, 0.7, None, tdt)
        assert torch.all(flat[offset + V * d:] == 7.0) and torch.all(flat[:offset] == 7.0)
        assert not table[to_dev(np.nonzero(k == 0)[0], torch)].any()
        table.copy_(to_dev(rng.standard_normal((V, d)).astype(np.float32), torch))
        base = table.clone()
        grad(g, gdt, td, V, 0.7, 1, table, tdt)
        check_grad(table.double().cpu().numpy(), g, tok, V, 0.7, base.double().cpu().numpy(), tdt)
        untouched = to_dev(np.nonzero(k == 0)[0], torch)
        assert torch.equal(table[untouched], base[untouched])


@pytest.mark.parametrize("kind", ["text", "same"])
@pytest.mark.parametrize("n,V,d", [(32767, 3, 8), (32768, 3, 8), (32767, 40, 512), (16384, 5, 1024), (16385, 5, 1024), (15, 2, 4),
                                   (16, 2, 4), (17, 2, 4), (31, 2, 4), (33, 2, 4), (399, 2, 4), (400, 2, 4)])
def test_gradient_where_pieces_change_their_length(n, V, d, kind):
    """Nothing behind the workspace is written, and the workspace of more tokens of more columns serves as well."""
    rng = np.random.default_rng(n + d)
    tok = ids(kind, n, V, rng)
    td = to_dev(tok, torch)
    log(f"{n} {kind} tokens, {V} x {d}")
    g = matrix(n, d, "fp32", rng)
    need, more = R.rollout_embedding_backward_workspace(n, V, d), R.rollout_embedding_backward_workspace(n + 1000, V, d + 100)
    assert more >= need
    ws = torch.full((more + 64,), 255, dtype=torch.uint8, device=DEV)
    table = torch.empty(V, d, device=DEV)
    R.rollout_embedding_backward(g, 0, td, n, V, d, 1.0, 0, table, 0, ws, need, None)
    check_grad(table.double().cpu().numpy(), g, tok, V, 1.0, None, "fp32")
    assert torch.all(ws[need:] == 255)
    again = torch.empty(V, d, device=DEV)
    R.rollout_embedding_backward(g, 0, td, n, V, d, 1.0, 0, again, 0, ws, more, None)
    assert torch.equal(table, again)


@pytest.mark.parametrize("kind", ["text", "same"])
def test_gradient_of_more_than_a_million_tokens(kind):
    """Tiles longer than what a lane holds on to, more tokens than a lookup's grid has workgroups, and, all of one id, sums of
    sums of pieces."""
    n, V, d = 1_100_000, 1000, 4
    rng = np.random.default_rng(3)
    tok = ids(kind, n, V, rng)
    td = to_dev(tok, torch)
    log(f"{n} tokens, {kind}")
    g = matrix(n, d, "fp32", rng)
    table = torch.empty(V, d, device=DEV)
    grad(g, "fp32", td, V, 1.0, 0, table, "fp32")
    check_grad(table.double().cpu().numpy(), g, tok, V, 1.0, None, "fp32")
    out = torch.empty(n, d, device=DEV)
    R.rollout_embedding(table, 0, V, d, td, n, 1.0, out, 0)
    live = (td >= 0) & (td < V)
    assert torch.equal(out[live], table[td[live].long()]) and not out[td < 0].any()
    assert torch.isnan(out[td >= V]).all()


def test_two_streams_at_once():
    rng = np.random.default_rng(9)
    n, V, d = 6000, 900, 64
    g = [matrix(n, d, "fp32", rng) for _ in range(2)]
    tok = to_dev(ids("text", n, V, rng), torch)
    want = [torch.empty(V, d, device=DEV) for _ in range(2)]
    for i in range(2):
        grad(g[i], "fp32", tok, V, 1.0, 0, want[i], "fp32")
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [torch.empty(V, d, device=DEV) for _ in range(2)]
    ws = [torch.empty(R.rollout_embedding_backward_workspace(n, V, d), dtype=torch.uint8, device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for i in range(2):
            grad(g[i], "fp32", tok, V, 1.0, 0, got[i], "fp32", streams[i].cuda_stream, ws[i])
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_gradient_without_tokens():
    rng = np.random.default_rng(0)
    g = matrix(100, 12, "fp32", rng)
    tok = to_dev(ids("none", 100, 9, rng), torch)
    table = torch.ones(9, 12, device=DEV)
    grad(g, "fp32", tok, 9, 1.0, 1, table, "fp32")
    assert torch.all(table == 1.0)
    grad(g, "fp32", tok, 9, 1.0, 0, table, "fp32")
    assert not table.any()


def test_the_order_of_addition_follows_from_the_positions():
    """Values whose fp32 sum depends on the order: the same bits whatever else is in the batch at other ids."""
    rng = np.random.default_rng(12)
    n, d = 100, 4
    vals = (rng.standard_normal((n, d)) * 2.0 ** rng.integers(-20, 20, (n, 1))).astype(np.float32)
    first = torch.empty(3, d, device=DEV)
    grad(to_dev(vals, torch), "fp32", torch.full((n,), 1, dtype=torch.int32, device=DEV), 3, 1.0, 0, first, "fp32")
    for _ in range(5):
        again = torch.empty(3, d, device=DEV)
        grad(to_dev(vals, torch), "fp32", torch.full((n,), 1, dtype=torch.int32, device=DEV), 3, 1.0, 0, again, "fp32")
        assert torch.equal(first, again)


@pytest.mark.parametrize("n", [300, 6000])
def test_gradients_of_padding_are_not_used(n):
    """NaN and infinities where the ids are padding or of no row; a token's own reach its row."""
    rng = np.random.default_rng(17)
    V, d = 70, 36
    tok = ids("text", n, V, rng)
    tok[::5] = -1
    tok[1::50] = V
    g = matrix(n, d, "fp32", rng)
    td = to_dev(tok, torch)
    want = torch.empty(V, d, device=DEV)
    grad(g, "fp32", td, V, 1.0, 0, want, "fp32")
    assert torch.isfinite(want).all()
    outside = (td < 0) | (td >= V)
    g[outside] = float("nan")
    g[outside.nonzero().flatten()[::2]] = float("inf")
    got = torch.empty(V, d, device=DEV)
    grad(g, "fp32", td, V, 1.0, 0, got, "fp32")
    assert torch.equal(want, got)
    first = int(np.nonzero((tok >= 0) & (tok < V))[0][0])
    g[first] = float("inf")
    grad(g, "fp32", td, V, 1.0, 0, got, "fp32")
    assert torch.all(got[tok[first]] == float("inf"))
    others = torch.arange(V, device=DEV) != tok[first]
    assert torch.equal(got[others], want[others])


def test_a_large_table_passes_32_bit_offsets():
    """More than 2^31 elements of table and more than 2^31 bytes of gradients: rows at both ends."""
    V, d, n = 300000, 8192, 40
    log("gradient of a table of 2.4e9 elements")
    table = torch.full((V, d), 7.0, dtype=torch.bfloat16, device=DEV)
    rng = np.random.default_rng(1)
    g = matrix(n, d, "bf16", rng)
    tok = np.array([0, V - 1, V - 2, 262144, 262145] * 8, dtype=np.int32)
    grad(g, "bf16", to_dev(tok, torch), V, 1.0, 0, table, "bf16")
    rows = np.unique(tok)
    got = table[to_dev(rows.astype(np.int64), torch)].double().cpu().numpy()
    want = U.embedding_backward(g.double().cpu().numpy(), np.searchsorted(rows, tok), len(rows), 1.0)
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 10 * EPS * 40)
    assert int((table != 0).sum()) <= len(rows) * d
    out = torch.empty(n, d, device=DEV)
    R.rollout_embedding(table, R.DTYPE_BF16, V, d, to_dev(tok, torch), n, 1.0, out, R.DTYPE_FP32)
    assert torch.equal(out, table[to_dev(tok.astype(np.int64), torch)].float())


def test_gradient_matches_differences():
    """Lookup and gradient are linear: <gradient, step> is the change of <g, lookup> along the step."""
    rng = np.random.default_rng(4)
    V, d, n = 20, 16, 50
    E, D, g = (matrix(k, d, "fp32", rng) for k in (V, V, n))
    tok = to_dev(rng.integers(-1, V, n).astype(np.int32), torch)
    table, y0, y1 = torch.empty(V, d, device=DEV), torch.empty(n, d, device=DEV), torch.empty(n, d, device=DEV)
    grad(g, "fp32", tok, V, 1.5, 0, table, "fp32")
    R.rollout_embedding(E, 0, V, d, tok, n, 1.5, y0, 0)
    R.rollout_embedding(E + D, 0, V, d, tok, n, 1.5, y1, 0)
    change = ((y1.double() - y0.double()) * g.double()).sum().item()
    size = (y1.double().abs() * g.double().abs()).sum().item()
    assert (table.double() * D.double()).sum().item() == pytest.approx(change, abs=4 * 20 * EPS * size)


@pytest.mark.parametrize("n", [500, 9000])
def test_repeats_and_graphs(n):
    rng = np.random.default_rng(6)
    V, d = 700, 200
    g = matrix(n, d, "bf16", rng)
    tok = to_dev(ids("text", n, V, rng), torch)
    first = torch.empty(V, d, device=DEV)
    grad(g, "bf16", tok, V, 1.0, 0, first, "fp32")
    for _ in range(3):
        again = torch.empty(V, d, device=DEV)
        grad(g, "bf16", tok, V, 1.0, 0, again, "fp32")
        assert torch.equal(first, again)
    made = []
    for i in range(2):
        table = torch.empty(V, d, device=DEV)
        ws = torch.empty(R.rollout_embedding_backward_workspace(n, V, d), dtype=torch.uint8, device=DEV)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            grad(g, "bf16", tok, V, 1.0, 0, table, "fp32", torch.cuda.current_stream().cuda_stream, ws)
        made.append((graph, table, ws))
    for replay in range(3):
        tok.copy_(to_dev(ids("text" if replay % 2 else "uniform", n, V, rng), torch))
        g.copy_(torch.randn(n, d, device=DEV))
        grad(g, "bf16", tok, V, 1.0, 0, first, "fp32")
        for graph, table, ws in made:
            graph.replay()
        torch.cuda.synchronize()
        for graph, table, ws in made:
            assert torch.equal(first, table), replay


def test_other_ids_in_the_batch_move_a_sum_by_roundings_only():
    """Where a run lies among the sorted ids decides where it is cut into pieces, and the batch's size how long they are: a
    row's sum is the same bits for the same batch, and within its bound whatever else is there."""
    rng = np.random.default_rng(13)
    n, d, V = 100, 4, 3
    vals = (rng.standard_normal((n, d)) * 2.0 ** rng.integers(-20, 20, (n, 1))).astype(np.float32)
    for before, behind in ((0, 0), (1, 0), (7, 0), (16, 3), (31, 500), (33, 33), (500, 5000), (9000, 1)):
        tok = np.repeat(np.array([0, 1, 2], dtype=np.int32), (before, n, behind))
        g = np.concatenate([rng.standard_normal((before, d)), vals, rng.standard_normal((behind, d))]).astype(np.float32)
        order = rng.permutation(len(tok))
        order[np.flatnonzero(tok[order] == 1)] = np.flatnonzero(tok == 1)  # this row's tokens in the same order
        tok, g = np.ascontiguousarray(tok[order]), np.ascontiguousarray(g[order])
        gd, td, table, again = to_dev(g, torch), to_dev(tok, torch), torch.empty(V, d, device=DEV), torch.empty(V, d, device=DEV)
        grad(gd, "fp32", td, V, 1.0, 0, table, "fp32")
        grad(gd, "fp32", td, V, 1.0, 0, again, "fp32")
        assert torch.equal(table, again)
        check_grad(table.double().cpu().numpy(), gd, tok, V, 1.0, None, "fp32")
