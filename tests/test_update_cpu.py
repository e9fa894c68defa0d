"""Refusals of the update side's entry points: every one is raised before the device is touched."""
import pytest

import paper_2608_11226_amd as R

A, B, C, D, E, F, G, H = ((i + 1) << 32 for i in range(8))  # addresses that are never dereferenced


def refuse(code, fn, *args, text=None):
    with pytest.raises(R.RolloutError) as e:
        fn(*args)
    assert e.value.code == code, e.value
    if text:
        assert text in str(e.value), e.value


def call(base, **change):
    k = dict(base)
    k.update(change)
    return tuple(k.values())


FORWARD = dict(z=A, dtype=0, stride=100, n=4, V=100, T=1.0, tokens=B, top=0, logp=C, entropy=D, stats=E, ids=None, tops=None,
               ws=F, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("code,change,text", [
    (R.EINVAL, dict(dtype=2), "dtype"), (R.EINVAL, dict(dtype=-1), "dtype"),
    (R.EINVAL, dict(n=0), "n_rows"), (R.EINVAL, dict(n=-3), "n_rows"), (R.EINVAL, dict(V=0), "vocab"),
    (R.EINVAL, dict(stride=99), "row_stride"), (R.EINVAL, dict(stride=1 << 62), "row_stride"),
    (R.EUNSUPPORTED, dict(V=(1 << 30) + 1, stride=1 << 31), "2^30"),
    (R.EINVAL, dict(z=None), "logits"), (R.EINVAL, dict(z=A + 2), "aligned"), (R.EINVAL, dict(z=A + 1, dtype=1), "aligned"),
    (R.EINVAL, dict(T=0.0), "temperature"), (R.EINVAL, dict(T=-1.0), "temperature"), (R.EINVAL, dict(T=float("inf")), "temperature"),
    (R.EINVAL, dict(T=float("nan")), "temperature"), (R.EINVAL, dict(T=1e-40), "temperature"),
    (R.EINVAL, dict(top=-1), "n_top"), (R.EINVAL, dict(top=33, ids=G, tops=H), "n_top"),
    (R.EINVAL, dict(V=3, top=4, ids=G, tops=H), "n_top"),
    (R.EUNSUPPORTED, dict(V=(1 << 20) + 1, stride=1 << 21, top=1, ids=G, tops=H), "2^20"),
    (R.EINVAL, dict(top=3), "alternatives"), (R.EINVAL, dict(top=3, ids=G), "alternatives"),
    (R.EINVAL, dict(tokens=None), "without tokens"), (R.EINVAL, dict(logp=None, entropy=None, stats=None), "no output"),
])
def test_logprobs_refusals(code, change, text):
    refuse(code, R.rollout_token_logprobs, *call(FORWARD, **change), text=text)


BACKWARD = dict(z=A, dtype=0, stride=100, n=4, V=100, T=1.0, tokens=B, stats=C, entropy=D, g=E, h=F, dz=G, dz_stride=100,
                stream=None)


@pytest.mark.parametrize("code,change,text", [
    (R.EINVAL, dict(dtype=2), "dtype"), (R.EINVAL, dict(n=0), "n_rows"), (R.EINVAL, dict(stride=99), "row_stride"),
    (R.EINVAL, dict(dz_stride=99), "grad_stride"), (R.EINVAL, dict(dz_stride=1 << 62), "grad_stride"),
    (R.EINVAL, dict(T=0.0), "temperature"),
    (R.EINVAL, dict(tokens=None), "NULL"), (R.EINVAL, dict(stats=None), "NULL"), (R.EINVAL, dict(g=None), "NULL"),
    (R.EINVAL, dict(dz=None), "NULL"), (R.EINVAL, dict(entropy=None), "entropies"), (R.EINVAL, dict(dz=G + 2), "aligned"),
    (R.EUNSUPPORTED, dict(V=(1 << 30) + 1, stride=1 << 31, dz_stride=1 << 31), "2^30"),
    # in place only at the same stride, and no other overlap
    (R.EINVAL, dict(dz=A, dz_stride=104), "overlap"), (R.EINVAL, dict(dz=A + 4), "overlap"),
    (R.EINVAL, dict(dz=A + 4 * 399), "overlap"), (R.EINVAL, dict(dz=A - 4 * 399), "overlap"),
])
def test_logprobs_backward_refusals(code, change, text):
    refuse(code, R.rollout_token_logprobs_backward, *call(BACKWARD, **change), text=text)


def test_logprobs_workspace():
    assert R.rollout_token_logprobs_workspace(1, 1) >= 0
    for args in ((0, 10, 0), (1, 0, 0), (1, 10, 11), (1, 100, 33), (1, 100, -1)):
        refuse(R.EINVAL, R.rollout_token_logprobs_workspace, *args)
    refuse(R.EUNSUPPORTED, R.rollout_token_logprobs_workspace, 1, (1 << 20) + 1, 1)
    assert R.lib.rollout_token_logprobs_workspace(1, 10, 0, None) == R.EINVAL


def test_tensors_are_checked():
    torch = pytest.importorskip("torch")
    host = torch.zeros(4, 100)
    refuse(R.EINVAL, R.rollout_token_logprobs, *call(FORWARD, z=host), text="current device")
    refuse(R.EINVAL, R.rollout_token_logprobs, *call(FORWARD, z=host.double()), text="float32")
    refuse(R.EINVAL, R.rollout_token_logprobs, *call(FORWARD, tokens=torch.zeros(4, dtype=torch.int64)), text="int32")
