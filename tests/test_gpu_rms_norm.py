"""The residual norm and its gradient against the definition in float64, with bounds from the roundings that the kernels make."""
import itertools

import numpy as np
import pytest
import torch

import paper_2608_11226_amd as R
from layer_cases import CODE, DEV, HALF, TYPES, U, wide
from oracle import layers as L

pytestmark = pytest.mark.gpu

EPS = float(np.float32(1e-6))
SIZES = [(1, 1), (3, 7), (5, 8), (9, 100), (64, 128), (130, 1000), (7, 2048), (6, 2049), (33, 3584), (4, 8192), (5, 8193), (3, 20001),
         (2, 32768)]
E4M3 = torch.float8_e4m3fn


def _rand(g, *shape, t=torch.float32, by=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * by).to(t)


def _sum_error(dim):
    """Relative, of a sum of dim terms of one sign: a thread adds up to 32, a wave 6 levels, a workgroup 16; each term is
    rounded itself."""
    return (min(dim, 32) + 6 + 16 + 2) * U


def forward(x, delta, gain, y_type, in_place=False, offset=0):
    n, d = x.shape
    new = lambda t: torch.empty(n * d + offset, dtype=t, device=DEV)[offset:].view(n, d)  # noqa: E731
    h = None if delta is None else x if in_place else new(x.dtype)
    y = new(E4M3 if y_type == "e4m3" else TYPES[y_type])
    scales = torch.full((n,), -1.0, device=DEV) if y_type == "e4m3" else None
    rstd = torch.full((n,), -1.0, device=DEV)
    code = {t: c for c, t in TYPES.items()}
    R.rollout_rms_norm(x, CODE[code[x.dtype]], delta, 0 if delta is None else CODE[code[delta.dtype]], gain, n, d, EPS, h, y, CODE[y_type],
                       scales, rstd, torch.cuda.current_stream().cuda_stream)
    return h, y, scales, rstd


def check_forward(x, delta, gain, y_type, got):
    h, y, scales, rstd = got
    d = x.shape[1]
    if delta is not None:
        assert torch.equal(h, (x.float() + delta.float()).to(x.dtype))
    hw = wide(x if delta is None else h)
    want, r = L.rms_norm(hw, np.ones(d) if gain is None else wide(gain), EPS)
    er = _sum_error(d) / 2 + 4 * U
    assert (np.abs(wide(rstd) - r) <= er * r).all()
    ey = er + 3 * U
    if y_type != "e4m3":
        assert (np.abs(wide(y) - want) <= (ey + HALF[y_type] * 1.01) * np.abs(want) + 1e-40).all()
        return
    most = np.abs(want).max(1)
    s = wide(scales)
    low, high = L.power_scale(most * (1 - ey)), L.power_scale(most * (1 + ey))
    assert ((s == low) | (s == high)).all()
    q, a = wide(y), np.abs(want) / s[:, None]
    assert np.isfinite(q).all() and (np.abs(q - want / s[:, None]) <= L.spacing(a * (1 + ey)) / 2 + ey * a).all()


@pytest.mark.parametrize("n,d", SIZES)
def test_rms_norm(n, d):
    g = torch.Generator(device=DEV).manual_seed(d)
    for i, (xt, dt, yt) in enumerate(itertools.product(("fp32", "bf16"), ("", "fp32", "bf16"), ("fp32", "bf16", "e4m3"))):
        x, delta = _rand(g, n, d, t=TYPES[xt], by=3.0), _rand(g, n, d, t=TYPES[dt]) if dt else None
        gain = None if i % 4 == 3 else 1.0 + _rand(g, d, by=0.1)
        got = forward(x, delta, gain, yt, offset=i % 3)
        check_forward(x, delta, gain, yt, got)


def test_in_place():
    g = torch.Generator(device=DEV).manual_seed(1)
    for t in ("fp32", "bf16"):
        x, delta, gain = _rand(g, 20, 1000, t=TYPES[t]), _rand(g, 20, 1000, t=torch.bfloat16), 1.0 + _rand(g, 1000, by=0.1)
        want = forward(x, delta, gain, "bf16")
        got = forward(x, delta, gain, "bf16", in_place=True)
        assert got[0] is x and all(torch.equal(a, b) for a, b in zip(want, got) if a is not None)


def test_rows_of_extremes():
    x = torch.zeros((9, 300), device=DEV)
    x[1], x[2], x[3, 5] = 1e-30, 1e18, 1.0  # x^2 underflows; large; one value alone
    x[4, 7], x[5, 8], x[6] = float("nan"), float("inf"), -2.5
    x[7] = torch.linspace(-1, 1, 300, device=DEV) * 1e-3
    x[8] = torch.linspace(1, 2, 300, device=DEV)
    for yt in ("fp32", "bf16", "e4m3"):
        got = forward(x, None, None, yt)
        keep = torch.tensor([0, 1, 2, 3, 6, 7, 8], device=DEV)
        check_forward(x[keep], None, None, yt, [None if a is None else a[keep] for a in got])
        y = wide(got[1])
        assert np.isnan(y[4]).all() and np.isnan(y[5, 8]) and (y[5, :8] == 0).all()
    codes, scales = got[1], got[2]
    assert (codes[0].view(torch.uint8) == 0).all() and scales[0] == 2.0 ** -126
    assert torch.isfinite(scales[4:6]).all()


def test_codes_are_the_nearest():
    """Rows whose norm and scale are exact: codes are torch's own conversion of y / scale."""
    g = torch.Generator(device=DEV).manual_seed(3)
    y = torch.cat([torch.arange(0, 2048, device=DEV) * 2.0 ** -13, _rand(g, 6 * 2048).abs() % 1.0]).view(-1, 2048)
    y = torch.where(torch.rand(y.shape, generator=g, device=DEV) < 0.5, -y, y)
    # x of ones and a gain that is y itself: rstd is 1 up to eps = 0
    one = torch.ones((1, 2048), device=DEV)
    for row in y:
        code = torch.empty((1, 2048), dtype=torch.uint8, device=DEV)
        scale = torch.empty(1, device=DEV)
        R.rollout_rms_norm(one, 0, None, 0, row.contiguous(), 1, 2048, 0.0, None, code, R.DTYPE_E4M3, scale, None,
                           torch.cuda.current_stream().cuda_stream)
        want = (row / scale).to(E4M3)
        assert torch.equal(code[0], want.view(torch.uint8))


def backward(dy, h, gain, rstd, inner, out_t, dgain=None, accumulate=0, in_place=False, stream=None):
    n, d = h.shape
    dx = inner if in_place else torch.empty((n, d), dtype=TYPES[out_t], device=DEV)
    code = {t: c for c, t in TYPES.items()}
    need = R.rollout_rms_norm_backward_workspace(n, d) if dgain is not None else 0
    ws = torch.full((max(need, 1),), 255, dtype=torch.uint8, device=DEV)
    R.rollout_rms_norm_backward(dy, CODE[code[dy.dtype]], h, CODE[code[h.dtype]], gain, rstd, n, d, inner, dx, CODE[out_t], dgain, accumulate,
                                ws, need, torch.cuda.current_stream().cuda_stream)
    return dx


@pytest.mark.parametrize("n,d", SIZES + [(5000, 64), (1500, 2500), (1100, 8200)])
def test_rms_norm_backward(n, d):
    g = torch.Generator(device=DEV).manual_seed(d + 1)
    for i, (ht, yt, ot) in enumerate(itertools.product(("fp32", "bf16"), ("fp32", "bf16"), ("fp32", "bf16"))):
        if n > 1000 and i not in (0, 3, 6):
            continue
        h, dy = _rand(g, n, d, t=TYPES[ht], by=3.0), _rand(g, n, d, t=TYPES[yt])
        gain = None if i % 4 == 3 else 1.0 + _rand(g, d, by=0.1)
        inner = None if i % 3 == 2 else _rand(g, n, d, t=TYPES[ot])
        rstd = torch.rsqrt(h.double().square().mean(1) + EPS).float()
        old = _rand(g, d)
        dgain, acc = old.clone(), i % 2
        dx = backward(dy, h, gain, rstd, inner, ot, dgain, acc)
        gw = np.ones(d) if gain is None else wide(gain)
        want, want_gain = L.rms_norm_backward(wide(dy), wide(h), gw, wide(rstd), 0.0 if inner is None else wide(inner))
        xhat, t = wide(h) * wide(rstd)[:, None], wide(dy) * gw
        terms = np.abs(t) + np.abs(xhat) * np.abs(t * xhat).mean(1, keepdims=True)
        bound = wide(rstd)[:, None] * terms * (_sum_error(d) + 8 * U) + (HALF[ot] * 1.01 + 2 * U) * np.abs(want)
        assert (np.abs(wide(dx) - want) <= bound + 1e-40).all(), (ht, yt, ot)
        # a worker adds its rows, the join the workers' sums: at most as many roundings as there are rows, and the old value's
        tol = (n + 4) * U * np.abs(wide(dy) * xhat).sum(0) + 2 * U * np.abs(wide(old)) * acc + 2 * U * np.abs(want_gain)
        assert (np.abs(wide(dgain) - want_gain - (wide(old) if acc else 0.0)) <= tol).all(), (ht, yt, ot)


def test_backward_in_place_and_without_gain_gradient():
    g = torch.Generator(device=DEV).manual_seed(8)
    h, dy, inner = _rand(g, 50, 777), _rand(g, 50, 777, t=torch.bfloat16), _rand(g, 50, 777)
    rstd = torch.rsqrt(h.square().mean(1) + EPS)
    want = backward(dy, h, None, rstd, inner, "fp32", torch.zeros(777, device=DEV))
    assert torch.equal(backward(dy, h, None, rstd, inner, "fp32"), want)
    assert torch.equal(backward(dy, h, None, rstd, inner.clone(), "fp32", in_place=True), want)


def test_gradients_by_differences():
    g = torch.Generator(device=DEV).manual_seed(9)
    x, gain, w = _rand(g, 3, 200), 1.0 + _rand(g, 200, by=0.1), _rand(g, 3, 200)
    _, y, _, rstd = forward(x, None, gain, "fp32")
    dgain = torch.zeros(200, device=DEV)
    dx = backward(w, x, gain, rstd, None, "fp32", dgain)

    def loss(a, b):
        return float((forward(a, None, b, "fp32")[1].double() * w.double()).sum())

    way, h = _rand(g, 3, 200), 2.0 ** -7
    slope = float((dx.double() * way.double()).sum())
    # third order: h^2 of a derivative of the slope's size; roundings of 600 outputs: 2^-24 sqrt(600) / h
    assert abs((loss(x + h * way, gain) - loss(x - h * way, gain)) / (2 * h) - slope) <= 1e-3 * abs(slope) + 1e-3
    way = _rand(g, 200)
    slope = float((dgain.double() * way.double()).sum())
    assert abs((loss(x, gain + h * way) - loss(x, gain - h * way)) / (2 * h) - slope) <= 1e-5 * abs(slope) + 1e-3


def test_more_than_2_to_the_32_elements():
    n, d = 540000, 8192
    at = torch.tensor([0, 1, 262143, 524287, 524288, n - 1], device=DEV)
    g = torch.Generator(device=DEV).manual_seed(12)
    x = torch.zeros((n, d), dtype=torch.bfloat16, device=DEV)
    x[at] = _rand(g, len(at), d, t=torch.bfloat16)
    y = torch.empty_like(x)
    rstd = torch.empty(n, device=DEV)
    s = torch.cuda.current_stream().cuda_stream
    R.rollout_rms_norm(x, 1, None, 0, None, n, d, EPS, None, y, 1, None, rstd, s)
    check_forward(x[at], None, None, "bf16", [None, y[at], None, rstd[at]])
    assert (y[2:262143] == 0).all()
    dgain = torch.empty(d, device=DEV)
    need = R.rollout_rms_norm_backward_workspace(n, d)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    dx = torch.empty_like(x)
    R.rollout_rms_norm_backward(x, 1, x, 1, None, rstd, n, d, None, dx, 1, dgain, 0, ws, need, s)
    few = [t[at].contiguous() for t in (x, rstd)]
    want = backward(few[0], few[0], None, few[1], None, "bf16", torch.empty(d, device=DEV))
    assert torch.equal(dx[at], want) and (dx[2:262143] == 0).all()
    w = wide(few[0])
    total = (w * w * wide(few[1])[:, None]).sum(0)
    assert (np.abs(wide(dgain) - total) <= 600 * U * total).all()  # a worker's 528 rows, most of them 0, and the join


def test_streams_and_graph():
    g = torch.Generator(device=DEV).manual_seed(10)
    x, delta, gain = _rand(g, 300, 1001), _rand(g, 300, 1001, t=torch.bfloat16), 1.0 + _rand(g, 1001, by=0.1)
    dy = _rand(g, 300, 1001, t=torch.bfloat16)
    h, y, scales, rstd = forward(x, delta, gain, "e4m3")
    dgain = torch.zeros(1001, device=DEV)
    dx = backward(dy, h, gain, rstd, x, "fp32", dgain)
    want = [t.clone().view(torch.uint8) for t in (h, y, scales, rstd, dx, dgain)]
    need = R.rollout_rms_norm_backward_workspace(300, 1001)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            R.rollout_rms_norm(x, 0, delta, 1, gain, 300, 1001, EPS, h, y, R.DTYPE_E4M3, scales, rstd, s.cuda_stream)
            R.rollout_rms_norm_backward(dy, 1, h, 0, gain, rstd, 300, 1001, x, dx, 0, dgain, 0, ws, need, s.cuda_stream)
    for i in range(3):
        for t in (h, y.view(torch.uint8), scales, rstd, dx, dgain, ws):
            t.fill_(i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((h, y, scales, rstd, dx, dgain), want):
            assert torch.equal(a.view(torch.uint8), b), i
