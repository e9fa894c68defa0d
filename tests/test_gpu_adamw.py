"""AdamW over many tensors against the definition in float64: sizes, types, rounding by the counter hash, replays."""
import numpy as np
import pytest
import torch

import paper_2608_11226_amd as R
from layer_cases import DEV, U, wide
from oracle import layers as L

pytestmark = pytest.mark.gpu

LR, B1, B2, EPS = 3e-3, 0.9, 0.97, 1e-8
E4M3 = torch.float8_e4m3fn
SIZES = [1, 7, 8, 127, 128, 129, 2047, 2048, 2049, 5000, 0, 70001]


class Tensor:
    def __init__(self, g, n, param="fp32", grad="fp32", state="fp32", copy=False, decay=0.1, offset=0, fresh=False):
        rand = lambda by: torch.randn(n, generator=g, device=DEV) * by  # noqa: E731
        at = lambda x: torch.cat([torch.zeros(offset, device=DEV, dtype=x.dtype), x])[offset:]  # noqa: E731
        T = {"fp32": torch.float32, "bf16": torch.bfloat16}
        self.n, self.param, self.state, self.decay = n, param, state, decay
        size = torch.exp(2.0 * rand(1.0)) * 1e-3
        self.p, self.g = at((0.05 * rand(1.0)).to(T[param])), at((rand(1.0) * size).to(T[grad]))
        m, v = (rand(0.4) * size, (0.3 + torch.rand(n, generator=g, device=DEV)) * size ** 2) if not fresh else (rand(0.0), rand(0.0))
        self.ms = self.vs = None
        if state == "e4m3":
            self.m, self.ms = self.encode(m)
            self.v, self.vs = self.encode(v.sqrt())
            self.m, self.v = at(self.m.view(torch.uint8)).view(E4M3), at(self.v.view(torch.uint8)).view(E4M3)
        else:
            self.m, self.v = at(m), at(v)
        self.copy = at(torch.zeros(n, dtype=torch.bfloat16, device=DEV)) if copy else None

    @staticmethod
    def encode(x):
        n = x.numel()
        y = torch.cat([x, torch.zeros(-n % 128, device=DEV)]).view(-1, 128)
        s = torch.tensor(L.power_scale(wide(y.abs().amax(1))), dtype=torch.float32, device=DEV) if n else torch.zeros(0, device=DEV)
        return (y / s[:, None]).to(E4M3).view(-1)[:n].clone(), s

    def entry(self):
        return R.adamw_tensor(self.p, self.g, self.m, self.v, self.decay, self.ms, self.vs, self.copy)

    def all(self):
        return [x for x in (self.p, self.m, self.v, self.ms, self.vs, self.copy) if x is not None]

    def moments(self):
        m, v = wide(self.m), wide(self.v)
        if self.state == "e4m3":
            b = np.arange(self.n) // 128
            m, v = m * wide(self.ms)[b], (v * wide(self.vs)[b]) ** 2
        return m, v


def table_of(tensors):
    table, chunks = R.rollout_adamw_table([t.entry() for t in tensors])
    return table.to(DEV), len(tensors), chunks


def check_step(tensors, step, seed, before, grad_scale=1.0, lr=LR):
    for i, (t, (p, m, v)) in enumerate(zip(tensors, before)):
        if not t.n:
            continue
        g = wide(t.g) * grad_scale
        # moments as fp32 holds them before the step (a product with a power of two, and its square)
        wp, wm, wv = L.adamw(p, g, m, v, lr, B1, B2, EPS, step, t.decay)
        # 4 roundings: factors, products, sum, the scaled gradient (twice in its square)
        em, ev = 5 * U * (np.abs(B1 * m) + np.abs((1 - B1) * g)), 7 * U * (B2 * v + (1 - B2) * g * g)
        root = np.sqrt(wv / (1 - B2 ** step)) + EPS
        eu = lr / (1 - B1 ** step) * (em / root + np.abs(wm) / root * (6 * U + ev / np.maximum(2 * wv, 1e-300) + 4 * U))
        ep = 4 * U * np.abs(wp) + 3 * U * np.abs(p) + 1.1 * eu
        rm, rv, rp = L.adamw_bits(seed, step, i, np.arange(t.n))
        if t.param == "fp32":
            assert (np.abs(wide(t.p) - wp) <= ep).all(), i
            if t.copy is not None:
                assert torch.equal(t.copy, t.p.to(torch.bfloat16))
        else:
            e = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(wp), 2.0 ** -126))) - 7)
            at = np.abs(wp) / e + rp / 2.0 ** 16
            settled = np.abs(at - np.round(at)) > ep / e * 2 + 2.0 ** -15
            got = np.abs(wide(t.p)) / e
            assert (got[settled] == np.floor(at)[settled]).all() and (np.abs(got - at) <= 1 + 2.0 ** -14 + ep / e).all(), i
            assert settled.mean() > 0.99 or t.n < 1000
        if t.state == "fp32":
            assert (np.abs(wide(t.m) - wm) <= em).all() and (np.abs(wide(t.v) - wv) <= ev + 1e-45).all(), i
            continue
        nb = (t.n + 127) // 128
        for got, scales, want, err, bits, root in ((t.m, t.ms, wm, em, rm, False), (t.v, t.vs, np.sqrt(wv), ev / np.maximum(2 * np.sqrt(wv), 1e-300), rv, True)):
            a = np.abs(want)
            pad = np.zeros(nb * 128)
            pad[:t.n] = a
            most = pad.reshape(nb, 128).max(1)
            s = wide(scales)
            assert ((s == L.power_scale(most * (1 - 2.0 ** -20))) | (s == L.power_scale(most * (1 + 2.0 ** -20)))).all(), i
            s = s[np.arange(t.n) // 128]
            e = L.spacing(a / s)
            at = a / s / e + (16 * bits + 8) / 2.0 ** 20
            slack = err / s / e * 2 + 2.0 ** -18
            settled = np.abs(at - np.round(at)) > slack
            code = np.abs(wide(got)) / e
            expect = np.floor(at)
            if root:
                expect = np.where((expect == 0) & (a > 0), 2.0 ** -9 / e, expect)
                assert (wide(got)[a > 0] > 0).all()
            assert (code[settled] == expect[settled]).all(), i
            assert (np.abs(code - at)[~settled] <= 1 + 2 * slack[~settled]).all(), i
            assert settled.mean() > 0.99 or t.n < 1000
            assert ((wide(got) == 0) | (np.sign(wide(got)) == np.sign(want))).all()


def step_of(handle, step, seed, stream=None, **kw):
    R.rollout_adamw(*handle, LR, B1, B2, EPS, step, seed, stream=stream or torch.cuda.current_stream().cuda_stream, **kw)


@pytest.mark.parametrize("param,grad,state,copy", [
    ("fp32", "fp32", "fp32", False), ("fp32", "bf16", "fp32", True), ("bf16", "bf16", "fp32", False), ("bf16", "fp32", "fp32", False),
    ("fp32", "fp32", "e4m3", True), ("fp32", "bf16", "e4m3", False), ("bf16", "bf16", "e4m3", False), ("bf16", "fp32", "e4m3", False)])
@pytest.mark.parametrize("offset", [0, 1])
def test_adamw(param, grad, state, copy, offset):
    g = torch.Generator(device=DEV).manual_seed(offset)
    tensors = [Tensor(g, n, param, grad, state, copy, 0.1 * (i % 2), offset) for i, n in enumerate(SIZES)]
    handle = table_of(tensors)
    for step in (1, 2, 9):
        before = [(wide(t.p), *t.moments()) for t in tensors]
        step_of(handle, step, 1234567890123, grad_scale=torch.full((1,), 0.5, device=DEV) if step == 2 else None)
        torch.cuda.synchronize()
        check_step(tensors, step, 1234567890123, before, 0.5 if step == 2 else 1.0)


def test_kinds_in_one_table_and_many_tensors():
    g = torch.Generator(device=DEV).manual_seed(3)
    kinds = [("fp32", "fp32", "fp32", False), ("bf16", "bf16", "e4m3", False), ("fp32", "bf16", "e4m3", True), ("bf16", "fp32", "fp32", False)]
    tensors = [Tensor(g, (37 * i) % 401 if i % 50 else 9000, *kinds[i % 4], decay=0.0) for i in range(700)]
    before = [(wide(t.p), *t.moments()) for t in tensors]
    step_of(table_of(tensors), 3, 5)
    torch.cuda.synchronize()
    check_step(tensors, 3, 5, before)


def test_chunks_of_four_steps():
    """As tables of more than 2^34 elements have them: a small table is given that chunk."""
    g = torch.Generator(device=DEV).manual_seed(4)
    tensors = [Tensor(g, n, "fp32", "bf16", "e4m3", True) for n in (3000001, 128, 2000003)]
    table, n, chunks = table_of(tensors)
    entries = table.cpu().view(torch.int64).view(n, -1)  # 7 addresses, n, first, chunk, ...
    assert entries[:, 9].tolist() == [2048] * n and entries[:, 8].tolist() == [0, 1465, 1466] and chunks == 2443
    entries[:, 9] = 8192
    entries[:, 8] = torch.tensor([0, 367, 368])
    handle = entries.view(torch.uint8).flatten().to(DEV), n, 613
    before = [(wide(t.p), *t.moments()) for t in tensors]
    step_of(handle, 2, 9)
    torch.cuda.synchronize()
    check_step(tensors, 2, 9, before)


def test_from_fresh_states():
    g = torch.Generator(device=DEV).manual_seed(5)
    for state in ("fp32", "e4m3"):
        t = Tensor(g, 1000, state=state, fresh=True)
        t.g[100:300] = 0.0  # a whole block without gradients among them
        before = [(wide(t.p), *t.moments())]
        step_of(table_of([t]), 1, 0)
        torch.cuda.synchronize()
        check_step([t], 1, 0, before)
        assert (t.m[100:300].float() == 0).all() and (t.v[100:300].float() == 0).all()


def test_expectation_of_rounded_states():
    """Over many seeds an 8-bit moment is on average what fp32 would hold."""
    g = torch.Generator(device=DEV).manual_seed(6)
    t = Tensor(g, 128, state="e4m3")
    first = [x.clone() for x in t.all()]
    _, m, v = L.adamw(wide(t.p), wide(t.g), *t.moments(), LR, B1, B2, EPS, 4, 0.1)
    handle, sums, n = table_of([t]), [0.0, 0.0], 4000
    for seed in range(n):
        for x, y in zip(t.all(), first):
            x.copy_(y)
        step_of(handle, 4, seed)
        sums[0] = sums[0] + t.m.double() * t.ms.double()
        sums[1] = sums[1] + t.v.double() * t.vs.double()
    for s, want, scale in zip(sums, (m, np.sqrt(v)), (t.ms, t.vs)):
        e = L.spacing(np.abs(want) / wide(scale)) * wide(scale)
        # a draw is off by at most one spacing with variance of at most a quarter of its square: six deviations of the mean
        assert (np.abs(wide(s) / n - want) <= 6 * 0.5 * e / np.sqrt(n) + 2.0 ** -16 * e).all()


def test_gradients_that_are_not_finite():
    g = torch.Generator(device=DEV).manual_seed(7)
    for state, param in (("fp32", "fp32"), ("e4m3", "bf16")):
        t = Tensor(g, 500, param, state=state)
        handle, first = table_of([t]), [x.clone() for x in t.all()]
        for bad in (float("nan"), float("inf"), -float("inf")):
            step_of(handle, 2, 0, grad_scale=torch.full((1,), bad, device=DEV))
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(t.all(), first))
        step_of(handle, 2, 0)
        clean = [x.clone() for x in t.all()]
        for x, y in zip(t.all(), first):
            x.copy_(y)
        # elements that are not the largest of their 128
        i, j = (int(t.v[k:k + 128].float().argmin()) + k for k in (0, 128))
        t.g[i], t.g[j] = float("nan"), float("inf")
        step_of(handle, 2, 0)
        # they stay where they are
        bad = torch.zeros(500, dtype=torch.bool, device=DEV)
        bad[i] = bad[j] = True
        assert t.p[bad].isnan().all() and t.m.float()[i].isnan() and not t.m.float()[j].isfinite()
        for x, y in zip(t.all(), clean):
            keep = ~bad if x.numel() == 500 else slice(None)
            assert torch.equal(x.float()[keep], y.float()[keep])


def test_a_step_that_changes_nothing():
    g = torch.Generator(device=DEV).manual_seed(8)
    t = Tensor(g, 300, decay=0.0)
    p = t.p.clone()
    R.rollout_adamw(*table_of([t]), 0.0, B1, B2, EPS, 1, 0, stream=torch.cuda.current_stream().cuda_stream)
    assert torch.equal(t.p, p)
    handle = table_of([Tensor(g, 0)])
    assert handle[2] == 0
    step_of(handle, 1, 0)


def test_rate_and_step_from_the_device_in_a_graph():
    g = torch.Generator(device=DEV).manual_seed(9)
    tensors = [Tensor(g, n, "fp32", "bf16", s, True) for n, s in ((5000, "e4m3"), (300, "fp32"))]
    handle, first = table_of(tensors), None
    lr, step = torch.full((1,), 1e-3, device=DEV), torch.ones(1, dtype=torch.int64, device=DEV)
    scale = torch.ones(1, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            R.rollout_adamw(*handle, 0.5, B1, B2, EPS, 99, 42, scale, lr, step, s.cuda_stream)
    for k in range(1, 5):
        step.fill_(k)
        lr.fill_(float(np.float32(LR / k)))
        scale.fill_(1.0 / k)
        torch.cuda.synchronize()
        before = [(wide(t.p), *t.moments()) for t in tensors]
        graph.replay()
        torch.cuda.synchronize()
        check_step(tensors, k, 42, before, float(np.float32(1.0 / k)), float(np.float32(LR / k)))


def test_elements_behind_the_first_2_to_the_32():
    n = (1 << 32) + 2000
    new = lambda t: torch.zeros(n, dtype=t, device=DEV)  # noqa: E731
    g = torch.Generator(device=DEV).manual_seed(11)
    p, grad, m, v = new(torch.bfloat16), new(torch.bfloat16), new(torch.uint8), new(torch.uint8)
    ms, vs = (torch.zeros((n + 127) // 128, device=DEV) for _ in range(2))
    at = torch.cat([torch.arange(1000), torch.arange(n - 2500, n)]).to(DEV)
    p[at] = torch.randn(3500, generator=g, device=DEV).bfloat16()
    grad[at] = torch.randn(3500, generator=g, device=DEV).bfloat16()
    before, gw = wide(p[at]), wide(grad[at])
    table, chunks = R.rollout_adamw_table([R.adamw_tensor(p, grad, m, v, 0.0, ms, vs)])
    step_of((table.to(DEV), 1, chunks), 1, 77)
    torch.cuda.synchronize()
    want, wm, _ = L.adamw(before, gw, 0.0, 0.0, LR, B1, B2, EPS, 1, 0.0)
    _, _, rp = L.adamw_bits(77, 1, 0, at.cpu().numpy())
    e = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(want), 2.0 ** -126))) - 7)
    pos = np.abs(want) / e + rp / 2.0 ** 16
    settled = np.abs(pos - np.round(pos)) > 2.0 ** -9  # (8 to 16 spacings of 2^-24 each, and a step of 2^-8 off by 20 of them)
    assert settled.mean() > 0.9 and (np.abs(wide(p[at]))[settled] == (np.floor(pos) * e)[settled]).all()
    mw = wide(m.view(E4M3)[at]) * wide(ms[at // 128])
    assert (np.abs(mw - wm) <= L.spacing(np.abs(wm) / wide(ms[at // 128])) * wide(ms[at // 128]) * 1.001).all()
    assert not m[1000:n - 2500].any() and not p[1000:n - 2500].any()


def test_on_another_stream():
    g = torch.Generator(device=DEV).manual_seed(10)
    t = Tensor(g, 40000, state="e4m3")
    before = [(wide(t.p), *t.moments())]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    step_of(table_of([t]), 5, 1, stream=s.cuda_stream)
    s.synchronize()
    check_step([t], 5, 1, before)


@pytest.mark.parametrize("grad,patterns", [("bf16", [0x7FFF, 0xFFFF, 0x7FF0, 0x7FC0, 0x7F81, 0xFF81]),
                                           ("fp32", [0x7FFFFFFF, 0xFFFFFFFF, 0x7FF00000, 0x7FC00000, 0x7F800001, 0xFF800001])])
def test_every_pattern_that_is_no_number_stays_one(grad, patterns):
    """Whatever the bits of a gradient that is not a number, both moments become NaN; nothing else changes by which it is."""
    g = torch.Generator(device=DEV).manual_seed(12)
    t = Tensor(g, 4096, "fp32", grad, "e4m3")
    handle, first, grads = table_of([t]), [x.clone() for x in t.all()], t.g.clone()
    bad = torch.arange(4096, device=DEV) % 3 == 1  # (many values of the hash)
    kind = torch.int16 if grad == "bf16" else torch.int32
    outs = []
    for u in patterns:
        for x, y in zip(t.all(), first):
            x.copy_(y)
        t.g.copy_(grads)
        t.g.view(kind)[bad] = u - (1 << 8 * kind.itemsize) if u >> (8 * kind.itemsize - 1) else u
        assert t.g[bad].isnan().all()
        step_of(handle, 2, 0)
        for x in (t.p, t.m.float(), t.v.float()):
            assert x[bad].isnan().all() and torch.isfinite(x[~bad]).all(), hex(u)
        outs.append([x.float()[~bad] if x.numel() == 4096 else x.clone() for x in t.all()])
        assert all(torch.equal(a, b) for a, b in zip(outs[0], outs[-1])), hex(u)


def test_states_that_are_no_numbers_stay_so():
    g = torch.Generator(device=DEV).manual_seed(13)
    t = Tensor(g, 2048, state="e4m3")
    for x, code in ((t.m, 0x7F), (t.m, 0xFF), (t.v, 0x7F)):
        keep = x.clone()
        x.view(torch.uint8)[::2] = code
        step_of(table_of([t]), 2, 0)
        assert x.float()[::2].isnan().all() and torch.isfinite(x.float()[1::2]).all()
        x.copy_(keep)


@pytest.mark.parametrize("binade", [-126, -125, -124, -122, -120, -117, -112, -107, -104, -96, -60, 0, 60, 126])
def test_roots_at_the_border_of_two_codes(binade):
    """Second moments down to 2^-126 whose roots, rounded to nearest, lie at the border that the hash's bits put between two codes, or
    one unit below it: a root that is off by a unit gives the other code."""
    n, beta2, seed, step = 8192, 0.5, 99, 1
    _, bits, _ = L.adamw_bits(seed, step, 0, np.arange(n))
    r = np.random.default_rng(binade + 200)
    # from fresh states v = g g / 2, each product rounded; v in [2^binade, 2^(binade + 1))
    g = np.sqrt(2.0 * r.uniform(1.001, 1.999, 1 << 22) * 2.0 ** binade).astype(np.float32)
    v = np.float32(0.5) * (g * g)
    assert (v >= np.float32(2.0 ** binade)).all()
    root = np.sqrt(v)  # (correctly rounded)
    low = root.view(np.uint32) & 0xFFFFF
    order = np.argsort(low, kind="stable")
    # (16 bits + 8) added to the mantissa's last 20 carries from `border` on
    border = (1 << 20) - (16 * bits + 8)
    wanted = border - (np.arange(n) & 1)
    at = np.searchsorted(low[order], wanted)
    found = (at < len(low)) & (low[order][np.minimum(at, len(low) - 1)] == wanted)
    assert found.mean() > 0.9
    pick = order[np.where(found, at, 0)]
    gn = torch.zeros(n, device=DEV)
    gn.copy_(torch.from_numpy(g[pick]))
    p, m, v8 = torch.zeros(n, device=DEV), torch.zeros(n, dtype=torch.uint8, device=DEV), torch.zeros(n, dtype=torch.uint8, device=DEV)
    ms, vs = torch.zeros(n // 128, device=DEV), torch.zeros(n // 128, device=DEV)
    table, chunks = R.rollout_adamw_table([R.adamw_tensor(p, gn, m, v8, 0.0, ms, vs)])
    R.rollout_adamw(table.to(DEV), 1, chunks, 0.0, 0.0, beta2, EPS, step, seed, stream=torch.cuda.current_stream().cuda_stream)
    most = root[pick].reshape(-1, 128).max(1).astype(np.float64)
    scale = L.power_scale(most)
    np.testing.assert_array_equal(wide(vs), scale)
    z = (root[pick].reshape(-1, 128) / scale[:, None]).astype(np.float32)  # (exact, and above 2^-6)
    want = ((z.view(np.uint32) + (16 * bits.reshape(-1, 128) + 8).astype(np.uint32)) & np.uint32(0xFFF00000)).view(np.float32)
    got = wide(v8.view(E4M3)).reshape(-1, 128)
    assert (got == want).all(), f"{(got != want).sum()} of {n} codes"
