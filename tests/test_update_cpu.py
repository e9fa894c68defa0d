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
    (R.EUNSUPPORTED, dict(n=(1 << 30) + 1), "2^30"),
    (R.EINVAL, dict(z=None), "logits"), (R.EINVAL, dict(z=A + 2), "aligned"), (R.EINVAL, dict(z=A + 1, dtype=1), "aligned"),
    (R.EINVAL, dict(T=0.0), "temperature"), (R.EINVAL, dict(T=-1.0), "temperature"), (R.EINVAL, dict(T=float("inf")), "temperature"),
    (R.EINVAL, dict(T=float("nan")), "temperature"), (R.EINVAL, dict(T=1e-40), "temperature"),
    (R.EINVAL, dict(top=-1), "n_top"), (R.EINVAL, dict(top=33, ids=G, tops=H), "n_top"),
    (R.EINVAL, dict(V=3, top=4, ids=G, tops=H), "n_top"),
    (R.EUNSUPPORTED, dict(V=327681, stride=1 << 21, top=1, ids=G, tops=H), "327,680"),
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
    refuse(R.EUNSUPPORTED, R.rollout_token_logprobs_workspace, 1, 327681, 1)
    assert R.lib.rollout_token_logprobs_workspace(1, 10, 0, None) == R.EINVAL


def test_tensors_are_checked():
    torch = pytest.importorskip("torch")
    host = torch.zeros(4, 100)
    refuse(R.EINVAL, R.rollout_token_logprobs, *call(FORWARD, z=host), text="current device")
    refuse(R.EINVAL, R.rollout_token_logprobs, *call(FORWARD, z=host.double()), text="float32")
    refuse(R.EINVAL, R.rollout_token_logprobs, *call(FORWARD, tokens=torch.zeros(4, dtype=torch.int64)), text="int32")
    refuse(R.EINVAL, R.rollout_token_logprobs, *call(FORWARD, z=host.bfloat16(), dtype=7), text="dtype must be 0")


LOSS = dict(lp=A, old=B, ref=C, H=D, adv=E, lengths=F, S=4, N=16, lo=0.2, hi=0.3, kl=0.1, ent=0.01, mean=0, loss=G, stats=G + 64,
            dlp=H, dH=H + (1 << 20), ws=H + (2 << 20), ws_bytes=1 << 20, stream=None)


@pytest.mark.parametrize("code,change,text", [
    (R.EINVAL, dict(S=0), "n_seqs"), (R.EINVAL, dict(N=0), "max_len"), (R.EUNSUPPORTED, dict(S=1 << 16, N=1 << 15), "2^31"),
    (R.EINVAL, dict(lp=None), "non-NULL"), (R.EINVAL, dict(adv=None), "non-NULL"),
    (R.EINVAL, dict(lo=-0.1), "clip_low"), (R.EINVAL, dict(lo=1.1), "clip_low"), (R.EINVAL, dict(lo=float("nan")), "clip_low"),
    (R.EINVAL, dict(hi=-0.1), "clip_high"), (R.EINVAL, dict(hi=float("inf")), "clip_high"),
    (R.EINVAL, dict(kl=float("nan")), "finite"), (R.EINVAL, dict(ent=float("inf")), "finite"),
    (R.EINVAL, dict(ref=None), "reference"), (R.EINVAL, dict(H=None), "entropies"), (R.EINVAL, dict(H=None, ent=0.0), "entropies"),
    (R.EINVAL, dict(mean=3), "mean"), (R.EINVAL, dict(mean=-1), "mean"),
    (R.EINVAL, dict(loss=None, stats=None, dlp=None, dH=None), "no output"),
    (R.EINVAL, dict(dlp=A), "overlaps an input"), (R.EINVAL, dict(dlp=B + 252), "overlaps an input"),
    (R.EINVAL, dict(dH=D - 252), "overlaps an input"), (R.EINVAL, dict(dH=H), "gradients overlap"),
    (R.ENOMEM, dict(ws_bytes=8), "workspace"), (R.EINVAL, dict(ws=None), "workspace"), (R.EINVAL, dict(ws=H + 8), "16 bytes"),
])
def test_policy_loss_refusals(code, change, text):
    refuse(code, R.grpo_policy_loss, *call(LOSS, **change), text=text)


LOOKUP = dict(table=A, tdt=0, V=100, dim=8, tokens=B, n=5, scale=1.0, out=C, odt=1, stream=None)


@pytest.mark.parametrize("code,change,text", [
    (R.EINVAL, dict(tdt=2), "dtype"), (R.EINVAL, dict(odt=-1), "dtype"), (R.EINVAL, dict(V=0), "vocab"),
    (R.EINVAL, dict(dim=0), "dim"), (R.EINVAL, dict(n=0), "n_tokens"), (R.EUNSUPPORTED, dict(V=(1 << 30) + 1), "2^30"),
    (R.EUNSUPPORTED, dict(n=(1 << 28) + 1), "2^28"), (R.EINVAL, dict(scale=float("nan")), "scale"),
    (R.EINVAL, dict(table=None), "NULL"), (R.EINVAL, dict(tokens=None), "NULL"), (R.EINVAL, dict(out=None), "NULL"),
    (R.EINVAL, dict(table=A + 2), "aligned"), (R.EINVAL, dict(out=C + 1), "aligned"),
    (R.EINVAL, dict(out=A + 3198), "overlaps"), (R.EINVAL, dict(out=A - 78), "overlaps"),
])
def test_embedding_refusals(code, change, text):
    refuse(code, R.rollout_embedding, *call(LOOKUP, **change), text=text)


GRAD = dict(g=A, gdt=1, tokens=B, n=5, V=100, dim=8, scale=1.0, acc=0, table=C, tdt=0, ws=D, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("code,change,text", [
    (R.EINVAL, dict(tdt=2), "dtype"), (R.EINVAL, dict(gdt=2), "dtype"), (R.EINVAL, dict(V=0), "vocab"), (R.EINVAL, dict(n=0), "n_tokens"),
    (R.EUNSUPPORTED, dict(n=(1 << 25) + 1), "2^25"), (R.EUNSUPPORTED, dict(n=(1 << 23) + 1, dim=3585), "2^25"),
    (R.EINVAL, dict(acc=2), "accumulate"), (R.EINVAL, dict(scale=float("inf")), "scale"),
    (R.EINVAL, dict(g=None), "NULL"), (R.EINVAL, dict(tokens=None), "NULL"), (R.EINVAL, dict(table=None), "NULL"),
    (R.EINVAL, dict(g=A + 1), "aligned"), (R.EINVAL, dict(table=C + 2), "aligned"),
    (R.EINVAL, dict(table=A + 76), "overlaps"), (R.EINVAL, dict(table=A - 3196), "overlaps"),
    (R.ENOMEM, dict(ws_bytes=100), "workspace"), (R.EINVAL, dict(ws=None), "NULL"), (R.EINVAL, dict(ws=D + 4), "16 bytes"),
])
def test_embedding_backward_refusals(code, change, text):
    refuse(code, R.rollout_embedding_backward, *call(GRAD, **change), text=text)


def test_workspaces_of_loss_and_embedding():
    assert R.grpo_policy_loss_workspace(1, 1) > 0
    assert R.rollout_embedding_backward_workspace(5, 100, 8) > 0
    refuse(R.EINVAL, R.grpo_policy_loss_workspace, 0, 4)
    refuse(R.EINVAL, R.rollout_embedding_backward_workspace, 0, 4, 4)
    assert R.lib.grpo_policy_loss_workspace(1, 1, None) == R.EINVAL
    assert R.lib.rollout_embedding_backward_workspace(1, 1, 1, None) == R.EINVAL


@pytest.mark.parametrize("dim", [1, 500, 513, 1024, 3584])
def test_the_embedding_workspace_of_more_serves_less(dim):
    sizes = [R.rollout_embedding_backward_workspace(n, 1000, dim) for n in (1, 31, 4096, 4097, 16384, 16385, 32767, 32768, 70000)]
    assert sizes == sorted(sizes)
    for n in (100, 16000, 32767, 40000):
        assert R.rollout_embedding_backward_workspace(n, 1000, dim) <= R.rollout_embedding_backward_workspace(n, 1000, dim + 1)
        assert R.rollout_embedding_backward_workspace(n, 1000, dim) <= R.rollout_embedding_backward_workspace(n, 1001, dim)


@pytest.mark.parametrize("top", [0, 1, 32])
def test_the_logprobs_workspace_of_more_serves_less(top):
    rows, vocabs = (1, 2, 33, 64, 1000, 1025, 2048, 2049, 4096, 70000), (32, 4096, 16384, 16385, 32003, 152064, 327680)
    for V in vocabs:
        sizes = [R.rollout_token_logprobs_workspace(n, V, top) for n in rows]
        assert sizes == sorted(sizes)
    for n in rows:
        sizes = [R.rollout_token_logprobs_workspace(n, V, top) for V in vocabs]
        assert sizes == sorted(sizes)
        assert sizes[0] >= R.rollout_token_logprobs_workspace(n, 32, 0)


def test_the_loss_workspace_of_more_serves_less():
    sizes = [R.grpo_policy_loss_workspace(n, 4096) for n in (1, 2, 7, 64, 700, 2048, 100000)]
    assert sizes == sorted(sizes)
    sizes = [R.grpo_policy_loss_workspace(64, n) for n in (1, 100, 511, 4096, 100000)]
    assert sizes == sorted(sizes)


# Matrices of 4 rows of 100 values, 128 apart, and small buffers beside them (as FORWARD, with room between the rows).
WIDE = dict(FORWARD, stride=128, top=3, ids=G, tops=H)


@pytest.mark.parametrize("change,text", [
    # outputs over inputs: logits (first and last element of a row), tokens
    (dict(logp=A), "overlaps an input, the logits"), (dict(entropy=A + 4 * (3 * 128 + 99)), "the logits"),
    (dict(stats=A + 4 * 128 - 28), "the logits"), (dict(logp=A - 12), "the logits"), (dict(ids=A + 4 * 128 - 44), "the logits"),
    (dict(tops=A + 4 * (128 + 99)), "the logits"), (dict(logp=A - (1 << 20) + 4, top=0, n=1 << 18), "the logits"),
    (dict(logp=B), "d_tokens"), (dict(stats=B - 28), "d_tokens"), (dict(ids=B + 12), "d_tokens"), (dict(tops=B), "d_tokens"),
    # outputs over each other
    (dict(entropy=C), "d_entropy overlaps d_logp"), (dict(stats=C + 12), "d_stats overlaps d_logp"),
    (dict(stats=D - 28), "d_stats overlaps d_entropy"), (dict(tops=G + 44), "d_top_logp overlaps d_top_ids"),
    # the workspace
    (dict(ws=A), "workspace overlaps an input, the logits"), (dict(ws=B - 16), "workspace overlaps an input, d_tokens"),
    (dict(ws=C), "workspace overlaps d_logp"), (dict(ws=H), "workspace overlaps d_top_logp"),
    # alignment of everything that is not a matrix
    (dict(tokens=B + 2), "aligned to 4"), (dict(logp=C + 1), "aligned to 4"), (dict(entropy=D + 2), "aligned to 4"),
    (dict(stats=E + 3), "aligned to 4"), (dict(ids=G + 2), "aligned to 4"), (dict(tops=H + 1), "aligned to 4"),
])
def test_logprobs_buffers_stand_apart(change, text):
    refuse(R.EINVAL, R.rollout_token_logprobs, *call(WIDE, **change), text=text)


BACK = dict(BACKWARD, stride=128, dz_stride=120)


@pytest.mark.parametrize("change,text", [
    (dict(dz=B), "d_tokens"), (dict(dz=C - 4 * (3 * 120 + 99)), "d_stats"), (dict(dz=C + 28), "d_stats"),
    (dict(dz=D + 12), "d_entropy"), (dict(dz=E), "d_grad_logp"), (dict(dz=F - 4 * 99), "d_grad_entropy"),
    (dict(tokens=B + 1), "aligned to 4"), (dict(stats=C + 2), "aligned to 4"), (dict(entropy=D + 2), "aligned to 4"),
    (dict(g=E + 2), "aligned to 4"), (dict(h=F + 3), "aligned to 4"),
])
def test_logprobs_backward_buffers_stand_apart(change, text):
    refuse(R.EINVAL, R.rollout_token_logprobs_backward, *call(BACK, **change), text=text)


@pytest.mark.parametrize("change,text", [
    (dict(dlp=E - 252), "d_adv"), (dict(dlp=F + 12), "d_lengths"), (dict(dH=E), "d_adv"), (dict(dH=F), "d_lengths"),
    (dict(loss=A + 252), "d_loss overlaps an input, d_logp"), (dict(loss=E), "d_adv"), (dict(stats=F - 16), "d_lengths"),
    (dict(stats=C), "d_ref_logp"), (dict(loss=G + 64 + 16), "overlaps d_loss"), (dict(loss=H + 252), "d_grad_logp overlaps d_loss"),
    (dict(stats=H + (1 << 20)), "d_grad_entropy overlaps d_stats"),
    (dict(ws=A - 16), "workspace overlaps an input, d_logp"), (dict(ws=E), "d_adv"), (dict(ws=F), "d_lengths"),
    (dict(ws=G), "workspace overlaps d_loss"), (dict(ws=H + 240), "workspace overlaps d_grad_logp"),
    (dict(lp=A + 2), "aligned to 4"), (dict(old=B + 1), "aligned to 4"), (dict(ref=C + 2), "aligned to 4"),
    (dict(H=D + 2), "aligned to 4"), (dict(adv=E + 2), "aligned to 4"), (dict(lengths=F + 2), "aligned to 4"),
    (dict(loss=G + 2), "aligned to 4"), (dict(stats=G + 66), "aligned to 4"), (dict(dlp=H + 1), "aligned to 4"),
    (dict(dH=H + (1 << 20) + 2), "aligned to 4"),
])
def test_policy_loss_buffers_stand_apart(change, text):
    refuse(R.EINVAL, R.grpo_policy_loss, *call(LOSS, **change), text=text)


@pytest.mark.parametrize("change,text", [(dict(out=B), "d_tokens"), (dict(out=B - 78), "d_tokens"), (dict(out=B + 18), "d_tokens"),
                                         (dict(tokens=B + 2), "aligned to 4")])
def test_embedding_buffers_stand_apart(change, text):
    refuse(R.EINVAL, R.rollout_embedding, *call(LOOKUP, **change), text=text)


@pytest.mark.parametrize("change,text", [
    (dict(table=B - 3196), "d_tokens"), (dict(table=B + 16), "d_tokens"), (dict(ws=A), "workspace overlaps an input, d_grad"),
    (dict(ws=B), "workspace overlaps an input, d_tokens"), (dict(ws=C), "workspace overlaps d_grad_table"),
    (dict(ws=C + 3184), "workspace overlaps d_grad_table"), (dict(tokens=B + 2), "aligned to 4"),
])
def test_embedding_backward_buffers_stand_apart(change, text):
    refuse(R.EINVAL, R.rollout_embedding_backward, *call(GRAD, **change), text=text)


def accepted(fn, *args):
    """The call passes every check of its buffers: without a device it is refused for that alone."""
    if R._torch.cuda.is_available():
        pytest.skip("addresses that are never dereferenced would be")
    refuse(R.EDEVICE, fn, *args)


def test_buffers_beside_each_other_are_taken():
    """Right before and behind one another, and between the rows of logits."""
    accepted(R.rollout_token_logprobs, *call(WIDE))
    accepted(R.rollout_token_logprobs, *call(WIDE, logp=A - 16, entropy=A + 4 * (3 * 128 + 100), stats=C, ids=A + 4 * 100,
                                             tops=A + 4 * (128 + 100)))
    accepted(R.rollout_token_logprobs, *call(WIDE, logp=A + 4 * (2 * 128 + 100), entropy=A + 4 * (2 * 128 + 104), tokens=A + 4 * 508))
    accepted(R.rollout_token_logprobs, *call(WIDE, ids=B, tops=B, top=0, entropy=C + 16, stats=C + 32))  # ids: not asked for
    accepted(R.rollout_token_logprobs_backward, *call(BACK))
    accepted(R.rollout_token_logprobs_backward, *call(BACK, dz=A, dz_stride=128))
    accepted(R.rollout_token_logprobs_backward, *call(BACK, dz=C - 400))
    accepted(R.rollout_token_logprobs_backward, *call(BACK, g=G + 4 * 100, tokens=G + 4 * (120 + 104), stats=G + 4 * (240 + 100)))
    accepted(R.rollout_token_logprobs_backward, *call(BACK, entropy=G + 2, h=None))  # not read
    accepted(R.grpo_policy_loss, *call(LOSS))
    accepted(R.grpo_policy_loss, *call(LOSS, loss=E + 16, stats=E + 20, dlp=A + 256, dH=A + 512))
    accepted(R.rollout_embedding, *call(LOOKUP, out=B + 20))
    accepted(R.rollout_embedding_backward, *call(GRAD, table=B + 20))


def _view_calls(monkeypatch):
    """Both directions on views of a host matrix that the binding takes for the device's: EDEVICE is what a call comes to that
    passes all checks."""
    if R._torch.cuda.is_available():
        pytest.skip("host tensors would reach the device")
    monkeypatch.setattr(R, "_device", lambda: -1)
    z, f = R._torch.zeros, lambda k, n, stride, V, **w: R.rollout_token_logprobs(k, 0, stride, n, V, 1.0, R._torch.zeros(64, dtype=R._torch.int32),
                                                                               0, R._torch.zeros(64))
    back = lambda k, n, stride, V: R.rollout_token_logprobs_backward(
        R._torch.zeros(64, 64), 0, 64, n, V, 1.0, R._torch.zeros(64, dtype=R._torch.int32), R._torch.zeros(128), None,
        R._torch.zeros(64), None, k, stride)
    return z, (f, back)


def test_rows_of_views_have_the_stride_of_the_call(monkeypatch):
    zeros, fns = _view_calls(monkeypatch)
    wide, deep = zeros(12, 50), zeros(4, 6, 50)
    for fn in fns:
        for x, n, stride, V in ((wide[:, 7:37], 12, 50, 30), (wide[:, 7:37], 5, 50, 30), (wide[:, 7:37], 12, 50, 20),
                                (wide[::2, :30], 6, 100, 30), (deep[:, :, :30], 24, 50, 30), (deep[:, :3, :30], 3, 50, 30),
                                (deep[:, 2:3, :30], 4, 300, 30), (wide[3:4, :30], 1, 30, 30), (wide[:, 7:37], 1, 30, 30),
                                (deep[:, :1, :30], 4, 300, 30), (wide, 20, 30, 30)):
            refuse(R.EDEVICE, fn, x, n, stride, V)
        for x, n, stride, V, text in ((wide[:, 7:37], 12, 30, 30, "apart"), (wide[:, 7:37], 12, 49, 30, "apart"),
                                      (wide[:, 7:37], 12, 51, 30, "apart"), (wide[:, 7:37], 13, 50, 30, "12 rows"),
                                      (wide[:, 7:37], 2, 30, 30, "apart"), (wide[::2, :30], 6, 50, 30, "apart"),
                                      (deep[:, :3, :30], 12, 50, 30, "apart"), (deep[:, :3, :30], 4, 50, 30, "apart"),
                                      (deep[::2, :, :30], 12, 50, 30, "apart"), (wide[:, :20], 11, 50, 30, "rows of 20"),
                                      (wide.t(), 50, 12, 12, "contiguous"), (wide[:1].expand(12, 50), 12, 50, 50, "apart"),
                                      (wide[:, 7:37], 12, 30, 31, "30 elements")):
            refuse(R.EINVAL, fn, x, n, stride, V, text=text)


BIG = 1 << 32  # its low 32 bits are 0


@pytest.mark.parametrize("code,fn,base,change", [
    (R.EUNSUPPORTED, R.rollout_token_logprobs, FORWARD, dict(n=BIG + 4)),
    (R.EUNSUPPORTED, R.rollout_token_logprobs, FORWARD, dict(V=BIG + 100, stride=BIG + 100)),
    (R.EUNSUPPORTED, R.rollout_token_logprobs, FORWARD, dict(stride=(1 << 64) + 100)),
    (R.EUNSUPPORTED, R.rollout_token_logprobs, FORWARD, dict(top=BIG)),
    (R.EINVAL, R.rollout_token_logprobs, FORWARD, dict(n=4 - BIG)),
    (R.EINVAL, R.rollout_token_logprobs, FORWARD, dict(ws_bytes=-1)),
    (R.EINVAL, R.rollout_token_logprobs, FORWARD, dict(ws_bytes=1 << 64)),
    (R.EUNSUPPORTED, R.rollout_token_logprobs_backward, BACKWARD, dict(n=BIG + 4)),
    (R.EUNSUPPORTED, R.rollout_token_logprobs_backward, BACKWARD, dict(V=BIG + 100, stride=BIG + 100, dz_stride=BIG + 100)),
    (R.EINVAL, R.rollout_token_logprobs_backward, BACKWARD, dict(stride=100 - (1 << 64))),
    (R.EUNSUPPORTED, R.rollout_token_logprobs_backward, BACKWARD, dict(dz_stride=(1 << 64) + 100)),
    (R.EUNSUPPORTED, R.grpo_policy_loss, LOSS, dict(S=BIG + 4)), (R.EUNSUPPORTED, R.grpo_policy_loss, LOSS, dict(N=BIG + 16)),
    (R.EUNSUPPORTED, R.grpo_policy_loss, LOSS, dict(mean=BIG + 1)), (R.EINVAL, R.grpo_policy_loss, LOSS, dict(ws_bytes=-1)),
    (R.EUNSUPPORTED, R.rollout_embedding, LOOKUP, dict(V=BIG + 100)), (R.EUNSUPPORTED, R.rollout_embedding, LOOKUP, dict(dim=BIG + 8)),
    (R.EUNSUPPORTED, R.rollout_embedding, LOOKUP, dict(n=BIG + 5)), (R.EINVAL, R.rollout_embedding, LOOKUP, dict(n=5 - BIG)),
    (R.EUNSUPPORTED, R.rollout_embedding_backward, GRAD, dict(n=BIG + 5)),
    (R.EUNSUPPORTED, R.rollout_embedding_backward, GRAD, dict(V=BIG + 100)),
    (R.EUNSUPPORTED, R.rollout_embedding_backward, GRAD, dict(dim=BIG + 8)),
    (R.EUNSUPPORTED, R.rollout_embedding_backward, GRAD, dict(acc=BIG)),
    (R.EINVAL, R.rollout_embedding_backward, GRAD, dict(ws_bytes=-1)),
    (R.EINVAL, R.rollout_embedding_backward, GRAD, dict(ws_bytes=1 << 64)),
])
def test_numbers_that_c_does_not_hold(code, fn, base, change):
    refuse(code, fn, *call(base, **change))


def test_sizes_of_workspaces_that_c_does_not_hold():
    for fn, args in ((R.rollout_token_logprobs_workspace, (4, 100, 2)), (R.grpo_policy_loss_workspace, (4, 16)),
                     (R.rollout_embedding_backward_workspace, (5, 100, 8))):
        for i in range(len(args)):
            refuse(R.EUNSUPPORTED, fn, *(x + BIG if j == i else x for j, x in enumerate(args)))
            refuse(R.EINVAL, fn, *(x - BIG if j == i else x for j, x in enumerate(args)))


def test_a_negative_workspace_size_does_not_pass_for_a_large_one(monkeypatch):
    """As a tensor's size every length is enough for -1, as an unsigned number -1 is enough for every call."""
    if R._torch.cuda.is_available():
        pytest.skip("host tensors would reach the device")
    monkeypatch.setattr(R, "_device", lambda: -1)
    refuse(R.EINVAL, R.rollout_embedding_backward, *call(GRAD, ws=R._torch.zeros(16, dtype=R._torch.uint8), ws_bytes=-1))
