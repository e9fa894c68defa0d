"""Token log probabilities, their rows' entropy, statistics and alternatives, and the gradient, against the float64
definitions, at sizes from one id to the full vocabulary, strides, alignments and masks.

Tolerances are worst cases of fp32 arithmetic (eps = 2^-24, half a step).  With d_i = (z_i - m) / T: an exponent has
three roundings (the difference, the constant log2(e) / T, their product), so e_i is off by (3 |d_i| + 2) eps of itself
(2 for the exponential's own last bit); a sum of V of them, added up by at least 64 lanes, by V / 64 + 32 steps more.
"""
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


def forward(z, stride, V, T, tokens, top=0, dtype="fp32", stream=None, ws=None, want=("logp", "entropy", "stats")):
    n = (z.numel() - V) // stride + 1 if z.dim() == 1 else z.shape[0]
    out = {"logp": torch.full((n,), 7.0, device=DEV), "entropy": torch.full((n,), 7.0, device=DEV),
           "stats": torch.full((n, 2), 7.0, device=DEV), "ids": torch.full((n, max(1, top)), -7, dtype=torch.int32, device=DEV),
           "top_logp": torch.full((n, max(1, top)), 7.0, device=DEV)}
    need = R.rollout_token_logprobs_workspace(n, V, top)
    ws = torch.empty(max(16, need), dtype=torch.uint8, device=DEV) if ws is None else ws
    out["ws"] = ws
    pick = lambda k: out[k] if k in want else None
    R.rollout_token_logprobs(z, TYPE[dtype][1], stride, n, V, T, tokens, top, pick("logp"), pick("entropy"), pick("stats"),
                             out["ids"] if top else None, out["top_logp"] if top else None, ws, need, stream)
    return out


def check_forward(got, z, T, tokens, top=0):
    """z: float64 rows as the kernel saw them."""
    want = U.token_logprobs(z, T, tokens, top)
    V = z.shape[1]
    g = {k: v.cpu().numpy().astype(np.float64) for k, v in got.items() if k != "ws"}
    worst = 0.0
    for r in range(z.shape[0]):
        t = 0 if tokens is None else int(tokens[r])
        if t < 0 or not np.isfinite(want["stats"][r]).all():
            for k in ("logp", "entropy", "stats") + (("ids", "top_logp") if top else ()):
                if not (k == "logp" and tokens is None):
                    np.testing.assert_array_equal(g[k][r], want[k][r], err_msg=f"row {r} {k}")
            continue
        with np.errstate(over="ignore", invalid="ignore"):
            d = (z[r] - want["stats"][r, 0]) / T
            p = np.exp(d - want["stats"][r, 1])
            live = p > 0
            a1, a2 = (p[live] * -d[live]).sum(), (p[live] * d[live] ** 2).sum()
        steps = V / 64 + 32
        ln_s = want["stats"][r, 1]
        e_s = EPS * (3 * a1 + 2 + steps + 2 * abs(ln_s))
        assert g["stats"][r, 0] == want["stats"][r, 0], f"row {r}: maximum"
        assert abs(g["stats"][r, 1] - ln_s) <= e_s, f"row {r}: log sum {g['stats'][r, 1]} {ln_s}"
        e_H = e_s + EPS * (3 * a2 + (steps + 8) * a1) + a1 * e_s + EPS * abs(want["entropy"][r])
        # a masked id's exponent is taken as 2^-160 at least: nothing
        assert abs(g["entropy"][r] - want["entropy"][r]) <= e_H, f"row {r}: entropy"
        worst = max(worst, abs(g["entropy"][r] - want["entropy"][r]) / e_H)

        def near(name, x, y, dist):
            # below the largest fp32 value and half a step of it there is only the infinity
            if np.isneginf(y) or y < -(2.0 - 2.0 ** -24) * 2.0 ** 127 or np.isnan(y):
                assert (np.isneginf(x) if not np.isnan(y) else np.isnan(x)), f"row {r}: {name} {x} {y}"
            else:
                assert abs(x - y) <= e_s + EPS * (4 * abs(dist) + abs(y)), f"row {r}: {name} {x} {y}"

        if tokens is not None:
            near("log p", g["logp"][r], want["logp"][r], d[t] if t < V and np.isfinite(d[t]) else 0.0)
        if top:
            assert np.array_equal(g["ids"][r], want["ids"][r]), f"row {r}: {g['ids'][r]} {want['ids'][r]}"
            for j in range(top):
                dj = d[want["ids"][r, j]]
                near("alternative", g["top_logp"][r, j], want["top_logp"][r, j], dj if np.isfinite(dj) else 0.0)
    log(f"  worst entropy error {worst:.3f} of its bound")
    return want


def rows(n, V, dtype, seed, extra=0, offset=0, ties=False):
    """n rows of V logits, V + extra apart, starting offset elements into the allocation."""
    rng = np.random.default_rng(seed)
    z = (rng.standard_normal(n * (V + extra)) * 3).astype(np.float32)
    if ties:
        z = np.round(z)
    buf = torch.empty(offset + n * (V + extra), dtype=TYPE[dtype][0], device=DEV)
    buf[offset:] = torch.from_numpy(z).to(DEV).to(TYPE[dtype][0])
    flat = buf[offset:]
    seen = flat.view(n, V + extra)[:, :V].double().cpu().numpy()
    return flat.view(n, V + extra), seen, rng


SIZES = [(1, 1), (3, 2), (5, 7), (2, 64), (4, 255), (3, 256), (3, 257), (7, 511), (2, 513), (9, 1024), (3, 4099),
         (2, 8191), (130, 1000), (3, 32003), (2, 152064)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,V", SIZES)
def test_sizes(n, V, dtype):
    top = min(V, 20)
    for extra, offset, T, ties in ((0, 0, 1.0, False), (1, 1, 0.9, False), (5, 3, 1.7, True)):
        log(f"logprobs {dtype} {n} x {V} stride {V + extra} offset {offset} T {T}")
        z, seen, rng = rows(n, V, dtype, V + extra, extra, offset, ties)
        tok = rng.integers(0, V, n).astype(np.int32)
        tok[n // 2] = V - 1
        if n > 2:
            tok[1] = -1
        got = forward(z, V + extra, V, T, torch.from_numpy(tok).to(DEV), top, dtype)
        T = float(np.float32(T))
        check_forward(got, seen, T, tok, top)
        plain = forward(z, V + extra, V, T, torch.from_numpy(tok).to(DEV), 0, dtype)
        check_forward(plain, seen, T, tok)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [11, 700, 5000])
def test_masks_infinities_and_invalid_tokens(dtype, V):
    n, top = 12, min(V, 8)
    z, seen, rng = rows(n, V, dtype, V)
    low = torch.finfo(TYPE[dtype][0]).min
    tok = rng.integers(0, V, n).astype(np.int32)
    z[0] = -np.inf                         # nothing left
    z[1] = low                             # the type's lowest value everywhere: uniform
    z[2, :V - 1] = -np.inf                 # one id left, the last
    tok[2] = V - 1
    z[3, 1:] = low                         # one id left, the first
    tok[3] = V // 2
    z[4, V // 2] = float("nan")
    z[5, V // 2] = float("inf")
    z[6, : V // 2] = -np.inf
    tok[6] = 0                             # a masked token
    tok[7] = V                             # no such id
    tok[8] = np.iinfo(np.int32).min        # padding
    z[9] += 10000.0                        # far from zero
    z[10] = 3.0                            # all equal
    z[11] = float("nan")
    tok[11] = -1                           # padding is not looked at
    seen = z[:, :V].double().cpu().numpy()
    td = torch.from_numpy(tok).to(DEV)
    for T in (1.0, 0.5):
        log(f"logprobs masks {dtype} V {V} T {T}")
        want = check_forward(forward(z, V, V, T, td, top, dtype), seen, T, tok, top)
        check_forward(forward(z, V, V, T, td, 0, dtype), seen, T, tok)
    assert want["logp"][1] == pytest.approx(-np.log(V)) and np.isneginf(want["logp"][6]) and np.isnan(want["logp"][7])


@pytest.mark.parametrize("T", [0.01, 0.3, 7.5, 1000.0])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_temperatures(T, dtype):
    """From almost certain to almost uniform: both directions."""
    n, V = 6, 3001
    z, seen, rng = rows(n, V, dtype, 31)
    tok = rng.integers(0, V, n).astype(np.int32)
    tok[:3] = seen[:3].argmax(1)
    td = torch.from_numpy(tok).to(DEV)
    T32 = float(np.float32(T))
    log(f"temperature {T} {dtype}")
    fw = forward(z, V, V, T, td, 5, dtype)
    check_forward(fw, seen, T32, tok, 5)
    g = torch.from_numpy(rng.standard_normal(n).astype(np.float32)).to(DEV)
    h = torch.from_numpy(rng.standard_normal(n).astype(np.float32)).to(DEV)
    out = torch.empty_like(z)
    R.rollout_token_logprobs_backward(z, TYPE[dtype][1], V, n, V, T, td, fw["stats"], fw["entropy"], g, h, out, V)
    num = [x.double().cpu().numpy() for x in (fw["stats"], fw["entropy"], g, h)]
    want = U.token_logprobs_backward(seen, T32, tok, *num)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= backward_bound(seen, T32, tok, *num, want, dtype))


def test_alternatives_of_values_that_stand_together():
    """All alternatives in one unit of a row, in every unit's first and last id, and equal everywhere."""
    V = 9000
    for dtype in ("fp32", "bf16"):
        z, _, rng = rows(6, V, dtype, 5)
        z[0, 4097:4129] = torch.arange(32, device=DEV, dtype=z.dtype) + 32
        z[1, :] = 0.0
        z[1, 8990:] = -0.0
        z[2, ::256] = 40.0
        z[3, 255::256] = 40.0
        z[4] = torch.arange(V, device=DEV).to(z.dtype)     # ascending (bf16: runs of equal values)
        z[5] = -torch.arange(V, device=DEV).to(z.dtype)
        for top in (1, 2, 31, 32):
            log(f"alternatives {dtype} {top}")
            tok = np.zeros(6, dtype=np.int32)
            check_forward(forward(z, V, V, 1.0, torch.from_numpy(tok).to(DEV), top, dtype),
                          z.double().cpu().numpy(), 1.0, tok, top)


@pytest.mark.parametrize("V", [40, 70000])
def test_outputs_that_are_not_wanted(V):
    z, seen, rng = rows(4, V, "fp32", 9)
    tok = rng.integers(0, V, 4).astype(np.int32)
    td = torch.from_numpy(tok).to(DEV)
    whole = forward(z, V, V, 1.0, td, 3)
    for want in (("logp",), ("entropy",), ("stats",), ("logp", "stats")):
        got = forward(z, V, V, 1.0, td, 0, want=want)
        for k in ("logp", "entropy", "stats"):
            assert torch.equal(got[k], whole[k] if k in want else torch.full_like(got[k], 7.0)), (want, k)
    free = forward(z, V, V, 1.0, None, 3, want=("entropy", "stats"))
    for k in ("entropy", "stats", "ids", "top_logp"):
        assert torch.equal(free[k], whole[k])
    alone = forward(z, V, V, 1.0, None, 3, want=())
    assert torch.equal(alone["ids"], whole["ids"]) and torch.equal(alone["top_logp"], whole["top_logp"])


def test_far_rows_pass_32_bit_offsets():
    """Rows 2^22 elements apart: the last ones lie more than 2^31 elements (and 2^32 bytes) behind the first."""
    V, stride, n = 300, 1 << 22, 530
    buf = torch.empty((n - 1) * stride + V, dtype=torch.bfloat16, device=DEV)
    view = torch.as_strided(buf, (n, V), (stride, 1))
    view.copy_(torch.randn(n, V, device=DEV) * 2)
    tok = np.arange(n, dtype=np.int32) % V
    log(f"far rows: {buf.numel()} elements")
    seen = view.double().cpu().numpy()
    got = forward(buf, stride, V, 1.0, torch.from_numpy(tok).to(DEV), 2, "bf16")
    check_forward(got, seen, 1.0, tok, 2)
    g = torch.ones(n, device=DEV)
    R.rollout_token_logprobs_backward(buf, R.DTYPE_BF16, stride, n, V, 1.0, torch.from_numpy(tok).to(DEV), got["stats"], None, g,
                                      None, buf, stride)
    want = U.token_logprobs_backward(seen, 1.0, tok, got["stats"].cpu().numpy(), None, np.ones(n))
    assert np.abs(view.double().cpu().numpy() - want).max() <= 2.0 ** -8 * np.abs(want).max() + 1e-5


def backward_bound(z, T, tok, stats, H, g, h, want, dtype):
    """Half a step of the type, and of p's exponent: four roundings of size |d|, two of ln s, one of log p."""
    half = torch.finfo(TYPE[dtype][0]).eps / 2
    with np.errstate(over="ignore", invalid="ignore"):
        d = np.nan_to_num((z - stats[:, :1]) / T, neginf=0.0, posinf=0.0)
        lp = d - np.nan_to_num(stats[:, 1:], neginf=0.0)
        p = np.minimum(np.exp(np.minimum(lp, 0)), 1.0)
    rel = EPS * (4 * np.abs(d) + 2 * np.abs(stats[:, 1:]) + np.abs(lp) + 12)
    size = p * (np.abs(g)[:, None] + np.abs(h)[:, None] * (1 + np.abs(lp) + np.abs(H)[:, None]))
    hit = np.zeros_like(size)
    ok = (tok >= 0) & (tok < z.shape[1])
    hit[np.nonzero(ok)[0], tok[ok]] = np.abs(g)[ok]
    return half * np.abs(want) + (rel * size + 4 * EPS * hit) / T + 2.0 ** -120


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,V", SIZES)
def test_gradient(n, V, dtype):
    T = float(np.float32(0.8))
    for extra, offset, gextra, goffset, in_place, with_h in ((0, 0, 0, 0, False, True), (3, 1, 0, 0, False, True),
                                                             (1, 0, 8, 5, False, False), (2, 1, 2, 1, True, True)):
        log(f"gradient {dtype} {n} x {V} strides {V + extra} {V + gextra} in place {in_place}")
        z, seen, rng = rows(n, V, dtype, V + extra, extra, offset)
        if V > 8:
            z[:, 3] = -np.inf
            seen = z[:, :V].double().cpu().numpy()
        tok = rng.integers(0, V, n).astype(np.int32)
        tok[tok == 3] = 0
        if n > 2:
            tok[2] = -1
        td = torch.from_numpy(tok).to(DEV)
        fw = forward(z, V + extra, V, T, td, 0, dtype)
        g = torch.from_numpy(rng.standard_normal(n).astype(np.float32)).to(DEV)
        h = torch.from_numpy(rng.standard_normal(n).astype(np.float32)).to(DEV) if with_h else None
        if n > 3:
            g[3] = 0.0
            if with_h:
                h[3] = 0.0
                g[1] = 0.0  # the entropy's gradient alone
        if in_place:
            out = z
            before = z[:, V:].clone()
        else:
            out = torch.full((goffset + n * (V + gextra),), 7.0, dtype=z.dtype, device=DEV)[goffset:].view(n, V + gextra)
        R.rollout_token_logprobs_backward(z, TYPE[dtype][1], V + extra, n, V, T, td, fw["stats"], fw["entropy"], g, h, out,
                                          V + (extra if in_place else gextra))
        got = out[:, :V].double().cpu().numpy()
        rest = out[:, V:]
        assert torch.equal(rest, before if in_place else torch.full_like(rest, 7.0))
        num = [x.double().cpu().numpy() for x in (fw["stats"], fw["entropy"], g, h if with_h else torch.zeros_like(g))]
        want = U.token_logprobs_backward(seen, T, tok, num[0], num[1], num[2], num[3])
        assert np.all(np.abs(got - want) <= backward_bound(seen, T, tok, *num, want, dtype))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gradient_of_masked_and_invalid_rows(dtype):
    V, n = 600, 8
    z, _, rng = rows(n, V, dtype, 1)
    z[0] = -np.inf
    z[1] = torch.finfo(z.dtype).min
    z[2, 1:] = -np.inf
    z[3, 5] = float("nan")
    z[4] = float("nan")
    z[6] += 10000.0
    tok = np.array([0, 1, 0, 3, -1, V, 7, 9], dtype=np.int32)
    td = torch.from_numpy(tok).to(DEV)
    seen = z.double().cpu().numpy()
    fw = forward(z, V, V, 1.0, td, 0, dtype)
    g, h = torch.ones(n, device=DEV), torch.full((n,), 0.5, device=DEV)
    out = torch.full_like(z, 7.0)
    R.rollout_token_logprobs_backward(z, TYPE[dtype][1], V, n, V, 1.0, td, fw["stats"], fw["entropy"], g, h, out, V)
    got = out.double().cpu().numpy()
    assert not got[0].any() and not got[4].any() and not got[2].any()
    assert np.isnan(got[3]).all() and np.isnan(got[5]).all()
    num = [x.double().cpu().numpy() for x in (fw["stats"], fw["entropy"], g, h)]
    want = U.token_logprobs_backward(seen, 1.0, tok, *num)
    bound = backward_bound(seen, 1.0, tok, *num, want, dtype)
    for r in (1, 6, 7):
        assert np.all(np.abs(got[r] - want[r]) <= bound[r]), r
    # rows without a gradient are not read
    out.fill_(7.0)
    R.rollout_token_logprobs_backward(z, TYPE[dtype][1], V, n, V, 1.0, td, fw["stats"], None, torch.zeros_like(g), None, out, V)
    assert not out.any()


def test_gradient_matches_differences():
    """The kernel's gradient against differences of the kernel's own outputs, taken with steps that fp32 resolves."""
    V = 12
    rng = np.random.default_rng(2)
    z = torch.from_numpy(rng.standard_normal((1, V)).astype(np.float32)).to(DEV)
    tok = torch.tensor([4], dtype=torch.int32, device=DEV)
    fw = forward(z, V, V, 0.7, tok)
    out = torch.empty_like(z)
    R.rollout_token_logprobs_backward(z, 0, V, 1, V, 0.7, tok, fw["stats"], fw["entropy"], torch.tensor([1.5], device=DEV),
                                      torch.tensor([-0.5], device=DEV), out, V)
    step = 2.0 ** -6
    for i in range(V):
        val = []
        for sgn in (1, -1):
            q = z.clone()
            q[0, i] += sgn * step
            o = forward(q, V, V, 0.7, tok)
            val.append(1.5 * o["logp"].item() - 0.5 * o["entropy"].item())
        # a difference of outputs of a few units, each off by some 2^-22; the third derivative at most 2 / T^3
        assert out[0, i].item() == pytest.approx((val[0] - val[1]) / (2 * step), abs=2.0 ** -20 / step + step * step * 2 / 0.343)


def test_repeats_streams_and_graphs():
    """The same bits on every call, on another stream, and on replays of a graph with eager work between them."""
    n, V, top = 40, 20011, 5
    z, seen, rng = rows(n, V, "bf16", 3)
    tok = rng.integers(0, V, n).astype(np.int32)
    td = torch.from_numpy(tok).to(DEV)
    g = torch.randn(n, device=DEV)
    h = torch.randn(n, device=DEV)
    first = forward(z, V, V, 0.9, td, top, "bf16")
    check_forward(first, seen, float(np.float32(0.9)), tok, top)
    grad = torch.empty_like(z)
    back = lambda o, out, s=None: R.rollout_token_logprobs_backward(z, R.DTYPE_BF16, V, n, V, 0.9, td, o["stats"], o["entropy"],
                                                                    g, h, out, V, s)
    back(first, grad)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = forward(z, V, V, 0.9, td, top, "bf16", stream=side.cuda_stream)
    grad2 = torch.empty_like(z)
    back(other, grad2, side.cuda_stream)
    side.synchronize()
    for k in ("logp", "entropy", "stats", "ids", "top_logp"):
        assert torch.equal(first[k], other[k]), k
    assert torch.equal(grad, grad2)
    # two graphs, each with a workspace of its own
    need = R.rollout_token_logprobs_workspace(n, V, top)
    made = []
    for i in range(2):
        out = [torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.empty(n, 2, device=DEV),
               torch.empty(n, top, dtype=torch.int32, device=DEV), torch.empty(n, top, device=DEV), torch.empty_like(z)]
        ws = torch.empty(max(16, need), dtype=torch.uint8, device=DEV)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s = torch.cuda.current_stream().cuda_stream
            R.rollout_token_logprobs(z, R.DTYPE_BF16, V, n, V, 0.9, td, top, *out[:5], ws, need, s)
            R.rollout_token_logprobs_backward(z, R.DTYPE_BF16, V, n, V, 0.9, td, out[2], out[1], g, h, out[5], V, s)
        made.append((graph, out, ws))
    for replay in range(4):
        z.copy_(torch.randn(n, V, device=DEV) * (replay + 1))
        eager = forward(z, V, V, 0.9, td, top, "bf16")
        back(eager, grad)
        for graph, out, ws in made:
            graph.replay()
        torch.cuda.synchronize()
        for graph, out, ws in made:
            for k, x in zip(("logp", "entropy", "stats", "ids", "top_logp"), out):
                assert torch.equal(eager[k], x), (replay, k)
            assert torch.equal(grad, out[5])


def test_more_rows_than_a_launch_has_workgroups():
    """More rows than the grids hold: workgroups go on to further rows, with alternatives and without, and back."""
    for n, V, top in ((1100000, 5, 2), (70000, 4100, 0)):
        z = torch.randn(n, V, device=DEV, dtype=torch.bfloat16) * 3
        tok = torch.randint(-1, V, (n,), device=DEV, dtype=torch.int32)
        log(f"many rows: {n} x {V}")
        got = forward(z, V, V, 1.0, tok, top, "bf16")
        lp = torch.log_softmax(z.double(), 1)
        live = tok >= 0
        want = lp.gather(1, tok.clamp(min=0).long()[:, None])[:, 0] * live
        assert (got["logp"] - want).abs().max().item() <= EPS * (V / 64 + 200)  # distances of at most 27, entropies of at most 9
        if top:
            order = torch.sort(z.double(), dim=1, descending=True, stable=True)[1][:, :top].int()
            assert torch.equal(got["ids"], torch.where(live[:, None], order, -1))
        g = torch.randn(n, device=DEV)
        out = torch.empty_like(z)
        R.rollout_token_logprobs_backward(z, R.DTYPE_BF16, V, n, V, 1.0, tok, got["stats"], None, g, None, out, V)
        dz = -lp.exp() * (g * live)[:, None].double()
        dz.scatter_add_(1, tok.clamp(min=0).long()[:, None], (g * live).double()[:, None])
        assert ((out.double() - dz).abs() <= 2.0 ** -8 * dz.abs() + 200 * EPS * g.abs()[:, None]).all()


def test_two_streams_at_once():
    """Calls of two streams side by side, each with its own workspace."""
    n, V, top = 64, 50257, 8
    zs = [torch.randn(n, V, device=DEV) * 3 for _ in range(2)]
    tok = torch.randint(0, V, (n,), device=DEV, dtype=torch.int32)
    want = [forward(z, V, V, 1.0, tok, top) for z in zs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for _ in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i] = forward(zs[i], V, V, 1.0, tok, top, stream=streams[i].cuda_stream)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for k in ("logp", "entropy", "stats", "ids", "top_logp"):
            assert torch.equal(a[k], b[k])


def test_tensors_of_rows():
    """A view of wider rows is taken with its stride; tensors that do not fit the call are refused."""
    n, V = 6, 300
    wide = torch.randn(n, V + 20, device=DEV)
    tok = torch.zeros(n, dtype=torch.int32, device=DEV)
    part = wide[:, 7:7 + V]
    got = forward(part, V + 20, V, 1.0, tok)
    assert torch.equal(got["logp"], forward(part.contiguous(), V, V, 1.0, tok)["logp"])
    logp = torch.empty(n, device=DEV)
    no_ws = lambda z, stride, tokens=tok, out=logp: R.rollout_token_logprobs(z, 0, stride, n, V, 1.0, tokens, 0, out)
    no_ws(part, V + 20)
    assert torch.equal(logp, got["logp"])
    for bad in (lambda: no_ws(part, V + 21), lambda: no_ws(part.t(), V), lambda: no_ws(wide.half(), V + 20),
                lambda: no_ws(part, V + 20, tok[:-1]), lambda: no_ws(part, V + 20, tok.long()),
                lambda: no_ws(part, V + 20, tok, torch.empty(2 * n, device=DEV)[::2]), lambda: no_ws(part, V + 20, tok.cpu())):
        with pytest.raises(R.RolloutError) as e:
            bad()
        assert e.value.code == R.EINVAL


@pytest.mark.parametrize("top", [0, 20])
def test_the_workspace_of_a_large_call_serves_small_ones(top):
    """The same bits as with a workspace of the call's own, and nothing behind what its size asks for is written."""
    rng = np.random.default_rng(31)
    V, most = 20000, 3000
    big = torch.full((R.rollout_token_logprobs_workspace(most, V, top) + 64,), 255, dtype=torch.uint8, device=DEV)
    for n in (1, 7, 130, 1024):
        log(f"{n} rows of {V}, {top} alternatives")
        z = to_dev(rng.standard_normal((n, V)).astype(np.float32), torch)
        tokens = to_dev(rng.integers(0, V, n).astype(np.int32), torch)
        want = forward(z, V, V, 1.0, tokens, top)
        big.fill_(255)
        got = forward(z, V, V, 1.0, tokens, top, ws=big)
        for k in ("logp", "entropy", "stats", "ids", "top_logp"):
            assert torch.equal(want[k], got[k]), k
        assert torch.all(big[R.rollout_token_logprobs_workspace(n, V, top):] == 255)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,units", [(2, 19), (2, 20), (3, 21), (2, 31), (40, 32), (2, 33), (3, 47), (2, 48), (150, 63), (2, 64),
                                     (2, 65), (1024, 17), (2047, 5), (2048, 5), (2049, 17), (700, 40), (682, 69), (1024, 66),
                                     (409, 115), (1, 1100)])
def test_alternatives_of_rows_of_any_number_of_units(n, units, dtype):
    """Around as many units (1 KB) as alternatives, a split row or not, a wave or a workgroup a row; rows that end in a unit and
    with it, some with many equal values.  Nothing behind the workspace is written."""
    N = 4 if dtype == "fp32" else 8
    for V in (units * 64 * N, units * 64 * N - 3):
        log(f"alternatives {dtype} {n} x {V}")
        z, seen, rng = rows(n, V, dtype, V, 0, 0, n > 1)
        tok = rng.integers(0, V, n).astype(np.int32)
        tok[::7] = -1
        tok[0] = V - 1
        td = torch.from_numpy(tok).to(DEV)
        for top in (20, 0) if V <= 327680 else (0,):
            need = R.rollout_token_logprobs_workspace(n, V, top)
            ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)
            check_forward(forward(z, V, V, 1.0, td, top, dtype, ws=ws), seen, 1.0, tok, top)
            assert torch.all(ws[need:] == 255)


def test_views_are_read_and_written_at_their_own_stride():
    """The stride of a view has to be the call's: a smaller one would read, and write, what lies between its rows."""
    n, V = 5, 40
    wide = torch.randn(n, V + 24, device=DEV)
    part, tok = wide[:, 9:9 + V], torch.arange(n, dtype=torch.int32, device=DEV)
    for stride in (V, V + 1, V + 25, 2 * (V + 24)):
        for call in (lambda: forward(part, stride, V, 1.0, tok),
                     lambda: R.rollout_token_logprobs_backward(wide.clone(), 0, V + 24, n, V, 1.0, tok, torch.zeros(n, 2, device=DEV),
                                                               None, torch.ones(n, device=DEV), None, part, stride)):
            with pytest.raises(R.RolloutError) as e:
                call()
            assert e.value.code == R.EINVAL and "apart" in str(e.value)
    z, before = part.contiguous(), wide.clone()
    fw = forward(part, V + 24, V, 1.0, tok)
    R.rollout_token_logprobs_backward(part, 0, V + 24, n, V, 1.0, tok, fw["stats"], None, torch.ones(n, device=DEV), None, part, V + 24)
    want = torch.empty_like(z)
    R.rollout_token_logprobs_backward(z, 0, V, n, V, 1.0, tok, fw["stats"], None, torch.ones(n, device=DEV), None, want, V)
    assert torch.equal(part, want)
    assert torch.equal(wide[:, :9], before[:, :9]) and torch.equal(wide[:, 9 + V:], before[:, 9 + V:])


def test_waves_go_on_to_further_rows():
    """More rows than 2^20 workgroups of four waves take at once, without alternatives."""
    n, V = 4 * (1 << 20) + 4099, 5
    z = torch.randn(n, V, device=DEV, dtype=torch.bfloat16) * 3
    tok = torch.randint(-1, V, (n,), device=DEV, dtype=torch.int32)
    log(f"{n} x {V}")
    got = forward(z, V, V, 1.0, tok, 0, "bf16")
    lp = torch.log_softmax(z.double(), 1)
    live = tok >= 0
    want = lp.gather(1, tok.clamp(min=0).long()[:, None])[:, 0] * live
    assert (got["logp"] - want).abs().max().item() <= 200 * EPS  # distances of at most 27
    H = -(lp.exp() * lp).sum(1) * live
    assert (got["entropy"] - H).abs().max().item() <= 200 * EPS
    assert torch.equal(got["stats"][:, 0], torch.where(live, z.amax(1).float(), 0.0))


def test_workgroups_go_on_to_further_rows():
    """More than 2^20 rows that take a workgroup each (of 69 GB; nearly all are padding, which is not read, so only rows at both
    ends hold anything): a workgroup's second row follows a first one of its own, or a padded one, in the same LDS."""
    n, V, dtype = (1 << 20) + 24, 32769, "bf16"
    if torch.cuda.mem_get_info()[0] < 2 * n * V + (4 << 30):
        torch.cuda.empty_cache()
    z = torch.empty(n, V, dtype=torch.bfloat16, device=DEV)
    rows = torch.cat([torch.arange(16), (1 << 20) + torch.arange(24)]).to(DEV)
    z[rows] = (torch.randn(rows.numel(), V, device=DEV) * 3).to(z.dtype)
    tok = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    tok[rows] = torch.randint(0, V, (rows.numel(),), device=DEV, dtype=torch.int32)
    tok[rows[3::8]] = -1
    log(f"{n} x {V}")
    got = forward(z, V, V, 0.9, tok, 0, dtype)
    check_forward({k: got[k][rows] for k in ("logp", "entropy", "stats")}, z[rows].double().cpu().numpy(), float(np.float32(0.9)),
                  tok[rows].cpu().numpy())
    for k in ("logp", "entropy", "stats"):
        assert not got[k][tok < 0].any()
    del z
    torch.cuda.empty_cache()
