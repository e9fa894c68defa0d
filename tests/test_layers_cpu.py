"""Refusals of attention's, the norm's and the optimiser's entry points: every one is raised before the device is touched."""
import ctypes

import pytest
import torch

import paper_2608_11226_amd as R
from test_update_cpu import accepted, call, refuse

A, B, C, D, E, F, G, H, I, J, K, L = ((i + 1) << 36 for i in range(12))  # addresses that are never dereferenced
BIG = 1 << 32  # its low 32 bits are 0


def shape(**change):
    k = dict(dtype=1, n_heads=8, n_kv_heads=2, head_dim=64, n_seqs=3, n_q=100, n_k=120, causal=1, scale=0.125)
    k.update(change)
    return R.AttentionShape(**k)


FORWARD = dict(shape=shape(), q=A, qs=512, k=B, ks=128, v=C, vs=128, q_starts=D, q_lens=E, k_starts=F, k_lens=G, out=H, os=512, lse=I,
               ws=J, ws_bytes=1 << 30, stream=None)
BACKWARD = dict(shape=shape(), q=A, qs=512, k=B, ks=128, v=C, vs=128, q_starts=D, q_lens=E, k_starts=F, k_lens=G, out=H, os=512, lse=I,
                dout=J, dos=512, dq=K, dqs=512, dk=L, dks=128, dv=L + (1 << 30), dvs=128, ws=L + (1 << 31), ws_bytes=1 << 30, stream=None)
SHAPES = [
    (R.EINVAL, dict(dtype=2), "dtype"), (R.EINVAL, dict(dtype=3), "dtype"), (R.EINVAL, dict(n_heads=0), "n_heads"),
    (R.EINVAL, dict(n_kv_heads=0), "n_heads"), (R.EINVAL, dict(n_heads=7), "multiple"), (R.EINVAL, dict(n_heads=-8), "n_heads"),
    (R.EUNSUPPORTED, dict(n_heads=130), "64 query heads"), (R.EUNSUPPORTED, dict(head_dim=96), "head_dim"),
    (R.EUNSUPPORTED, dict(head_dim=0), "head_dim"), (R.EUNSUPPORTED, dict(head_dim=256), "head_dim"),
    (R.EINVAL, dict(n_seqs=0), "n_seqs"), (R.EINVAL, dict(n_q=0), "n_q"), (R.EINVAL, dict(n_k=-1), "n_k"),
    (R.EINVAL, dict(causal=2), "causal"), (R.EINVAL, dict(scale=0.0), "scale"), (R.EINVAL, dict(scale=-1.0), "scale"),
    (R.EINVAL, dict(scale=float("nan")), "scale"), (R.EINVAL, dict(scale=float("inf")), "scale"), (R.EINVAL, dict(scale=3e38), "scale"),
    (R.EINVAL, dict(scale=1e-31), "scale"), (R.EINVAL, dict(scale=1.3e30), "scale"),
    (R.EUNSUPPORTED, dict(n_q=(1 << 23) + 1), "2^26"), (R.EUNSUPPORTED, dict(n_k=1 << 30), "2^26"),
    (R.EUNSUPPORTED, dict(n_seqs=1 << 22), "2^23"), (R.EUNSUPPORTED, dict(n_seqs=(1 << 20) + 1), "2^23"),
]


@pytest.mark.parametrize("code,change,text", SHAPES)
def test_shapes(code, change, text):
    refuse(code, R.rollout_attention, *call(FORWARD, shape=shape(**change)), text=text)
    refuse(code, R.rollout_attention_backward, *call(BACKWARD, shape=shape(**change)), text=text)
    refuse(code, R.rollout_attention_workspace, shape(**change), text=text)
    refuse(code, R.rollout_attention_backward_workspace, shape(**change), text=text)


def test_shapes_that_c_does_not_hold():
    for name in ("dtype", "n_heads", "n_kv_heads", "head_dim", "n_seqs", "n_q", "n_k", "causal"):
        refuse(R.EUNSUPPORTED, lambda: shape(**{name: BIG + 2}), text=name)
        refuse(R.EINVAL, lambda: shape(**{name: 2 - BIG}), text=name)
        s = shape()
        refuse(R.EUNSUPPORTED, lambda: setattr(s, name, 1 << 31), text=name)
    assert R.lib.rollout_attention_workspace(None, ctypes.byref(ctypes.c_uint64())) == R.EINVAL
    assert R.lib.rollout_attention_workspace(ctypes.byref(shape()), None) == R.EINVAL
    assert R.lib.rollout_attention_backward_workspace(ctypes.byref(shape()), None) == R.EINVAL


@pytest.mark.parametrize("code,change,text", [
    (R.EINVAL, dict(q=None), "d_q is NULL"), (R.EINVAL, dict(k=None), "d_k is NULL"), (R.EINVAL, dict(v=None), "d_v is NULL"),
    (R.EINVAL, dict(out=None), "d_out is NULL"), (R.EINVAL, dict(lse=None), "d_lse"), (R.EINVAL, dict(q_starts=None), "d_q_starts"),
    (R.EINVAL, dict(k_starts=None), "d_k_lens without"), (R.EINVAL, dict(k_starts=None, k_lens=None), "as many keys"),
    (R.EINVAL, dict(q=A + 8), "16 bytes"), (R.EINVAL, dict(out=H + 2), "16 bytes"), (R.EINVAL, dict(lse=I + 2), "4 bytes"),
    (R.EINVAL, dict(q_lens=E + 1), "4 bytes"), (R.EINVAL, dict(qs=511), "at least"), (R.EINVAL, dict(ks=127), "at least"),
    (R.EINVAL, dict(qs=516), "multiple of 16"), (R.EINVAL, dict(vs=132), "multiple of 16"), (R.EINVAL, dict(os=0), "at least"),
    (R.EUNSUPPORTED, dict(qs=1 << 25), "2^25"), (R.EUNSUPPORTED, dict(vs=1 << 62), "2^25"), (R.EUNSUPPORTED, dict(os=1 << 64), "int64"),
    (R.ENOMEM, dict(ws_bytes=16), "workspace"), (R.EINVAL, dict(ws=None), "workspace"), (R.EINVAL, dict(ws=J + 8), "workspace"),
    (R.EINVAL, dict(ws_bytes=-1), "workspace"), (R.EINVAL, dict(out=A), "overlaps"), (R.EINVAL, dict(out=A + 99 * 1024), "overlaps"),
    (R.EINVAL, dict(out=B + 1024, os=1024), "overlaps"), (R.EINVAL, dict(lse=D), "d_lse overlaps"), (R.EINVAL, dict(lse=H), "overlaps"),
    (R.EINVAL, dict(ws=G), "workspace overlaps"), (R.EINVAL, dict(ws=H + 4096), "workspace overlaps"),
])
def test_attention_refusals(code, change, text):
    refuse(code, R.rollout_attention, *call(FORWARD, **change), text=text)
    if set(change) <= {"q", "k", "v", "out", "lse", "q_starts", "k_starts", "k_lens", "q_lens", "qs", "ks", "vs", "os"} and "overlaps" not in text:
        refuse(code, R.rollout_attention_backward, *call(BACKWARD, **change), text=text)


@pytest.mark.parametrize("code,change,text", [
    (R.EINVAL, dict(dout=None), "d_grad_out is NULL"), (R.EINVAL, dict(dq=None), "d_grad_q"), (R.EINVAL, dict(dk=None), "d_grad_k"),
    (R.EINVAL, dict(dv=None), "d_grad_v"), (R.EINVAL, dict(dq=K + 4), "16 bytes"), (R.EINVAL, dict(dqs=100), "at least"),
    (R.EINVAL, dict(dvs=130), "multiple"), (R.EUNSUPPORTED, dict(dks=1 << 26), "2^25"), (R.ENOMEM, dict(ws_bytes=1000), "workspace"),
    (R.EINVAL, dict(dq=A), "d_grad_q overlaps"), (R.EINVAL, dict(dk=B), "d_grad_k overlaps"), (R.EINVAL, dict(dv=L), "overlaps"),
    (R.EINVAL, dict(dq=J), "overlaps an input, d_grad_out"), (R.EINVAL, dict(dk=I), "d_lse"), (R.EINVAL, dict(ws=L), "workspace overlaps"),
    # columns of one matrix that reach into each other
    (R.EINVAL, dict(dk=L, dks=256, dv=L + 2 * 127, dvs=256), "16 bytes"), (R.EINVAL, dict(dk=L, dks=256, dv=L + 2 * 120, dvs=256), "overlaps"),
    (R.EINVAL, dict(dk=L, dks=256, dv=L + 2 * 256 * 119, dvs=256), "overlaps"),
    (R.EINVAL, dict(dk=L, dks=256, dv=L + 2 * 128, dvs=264), "overlaps"),
])
def test_attention_backward_refusals(code, change, text):
    refuse(code, R.rollout_attention_backward, *call(BACKWARD, **change), text=text)


def test_attention_calls_that_are_taken():
    accepted(R.rollout_attention, *call(FORWARD))
    accepted(R.rollout_attention, *call(FORWARD, q_lens=None, k_lens=None))
    accepted(R.rollout_attention, *call(FORWARD, shape=shape(n_k=100), k_starts=None, k_lens=None))
    accepted(R.rollout_attention, *call(FORWARD, q=A, qs=768, k=A + 1024, ks=768, v=A + 1280, vs=768, shape=shape(n_k=100)))
    # queries, keys and out as columns of one matrix
    accepted(R.rollout_attention, *call(FORWARD, q=A, qs=1536, out=A + 1536, os=1536))
    accepted(R.rollout_attention_backward, *call(BACKWARD))
    accepted(R.rollout_attention_backward, *call(BACKWARD, shape=shape(n_k=100), dq=K, dqs=768, dk=K + 1024, dks=768, dv=K + 1280, dvs=768))
    # between the rows of the inputs
    accepted(R.rollout_attention_backward, *call(BACKWARD, q=A, qs=1024, dq=A + 1024, dqs=1024))
    # right behind the last row's end
    accepted(R.rollout_attention_backward, *call(BACKWARD, dk=B + 2 * 128 * 120))


def test_attention_workspaces_grow_with_the_call():
    """That of the largest call serves them all: in tokens, sequences and heads."""
    for ask in (R.rollout_attention_workspace, R.rollout_attention_backward_workspace):
        for dtype in (0, 1):
            last = 0
            for n in (1, 2, 17, 100, 1000, 4096, 10000, 100000, 1000000):
                here = [ask(shape(dtype=dtype, n_q=n, n_k=n, n_seqs=s)) for s in (1, 3, 64, 5000)]
                assert len(set(here)) == 1 and here[0] >= last
                assert ask(shape(dtype=dtype, n_q=n, n_k=2 * n)) >= here[0] and ask(shape(dtype=dtype, n_q=n, n_k=n, n_heads=16)) >= here[0]
                last = here[0]


def test_attention_tensors_are_checked(monkeypatch):
    if R._torch.cuda.is_available():
        pytest.skip("host tensors would reach the device")
    s = shape(n_k=100)
    qkv, i32 = torch.zeros(100, 768, dtype=torch.bfloat16), torch.zeros(10, dtype=torch.int32)
    base = call(FORWARD, shape=s, q=qkv[:, :512], qs=768, k=qkv[:, 512:640], ks=768, v=qkv[:, 640:], vs=768, q_starts=i32, q_lens=i32,
                k_starts=None, k_lens=None)
    refuse(R.EINVAL, R.rollout_attention, *base, text="current device")
    monkeypatch.setattr(R, "_device", lambda: -1)
    refuse(R.EDEVICE, R.rollout_attention, *base)

    def other(**change):
        names = list(FORWARD)
        return [change.get(n, x) for n, x in zip(names, base)]

    for change, text in ((dict(q=qkv[:, :512].float()), "bfloat16"), (dict(qs=776), "apart"), (dict(q=qkv[:99, :512]), "99 rows"),
                         (dict(q=qkv[:, :504]), "rows of 504"), (dict(q_starts=i32[:3]), "3 elements"), (dict(q_lens=i32.long()), "int32"),
                         (dict(lse=torch.zeros(700)), "700 elements"), (dict(k=qkv[:, 512:640].t()), "contiguous"),
                         (dict(out=torch.zeros(100, 511, dtype=torch.bfloat16)), "elements")):
        refuse(R.EINVAL, R.rollout_attention, *other(**change), text=text)


NORM = dict(x=A, xt=0, delta=B, dt=1, gain=C, n=4, dim=100, eps=1e-6, h=D, y=E, yt=1, scales=None, rstd=F, stream=None)
NORM_BACK = dict(dy=A, dyt=1, h=B, ht=0, gain=C, rstd=D, n=4, dim=100, inner=E, dx=F, dxt=0, dgain=G, acc=0, ws=H, ws_bytes=1 << 20,
                 stream=None)


@pytest.mark.parametrize("code,change,text", [
    (R.EINVAL, dict(n=0), "n_rows"), (R.EINVAL, dict(dim=0), "dim"), (R.EINVAL, dict(n=-4), "n_rows"), (R.EUNSUPPORTED, dict(dim=32769), "32,768"),
    (R.EUNSUPPORTED, dict(n=1 << 26), "rows"), (R.EUNSUPPORTED, dict(n=1 << 22, dim=5000), "rows"), (R.EUNSUPPORTED, dict(n=BIG + 4), "int32"),
    (R.EINVAL, dict(xt=2), "dtype"), (R.EINVAL, dict(xt=3), "dtype"), (R.EINVAL, dict(dt=3), "dtype"), (R.EINVAL, dict(yt=2), "dtype"),
    (R.EINVAL, dict(eps=-1e-6), "eps"), (R.EINVAL, dict(eps=float("nan")), "eps"), (R.EINVAL, dict(eps=float("inf")), "eps"),
    (R.EINVAL, dict(x=None), "NULL"), (R.EINVAL, dict(y=None), "NULL"), (R.EINVAL, dict(delta=None), "come together"),
    (R.EINVAL, dict(h=None), "come together"), (R.EINVAL, dict(yt=3), "d_scales"), (R.EINVAL, dict(scales=G), "d_scales"),
    (R.EINVAL, dict(x=A + 2), "aligned"), (R.EINVAL, dict(delta=B + 1), "aligned"), (R.EINVAL, dict(h=D + 2), "aligned"),
    (R.EINVAL, dict(y=E + 1), "aligned"), (R.EINVAL, dict(gain=C + 2), "4 bytes"), (R.EINVAL, dict(rstd=F + 1), "4 bytes"),
    (R.EINVAL, dict(y=A), "d_y overlaps an input, d_x"), (R.EINVAL, dict(y=B + 16), "d_delta"), (R.EINVAL, dict(h=A + 4), "d_h overlaps"),
    (R.EINVAL, dict(h=E), "d_y overlaps d_h"), (R.EINVAL, dict(rstd=C), "d_gain"), (R.EINVAL, dict(h=B), "d_h overlaps an input, d_delta"),
    (R.EINVAL, dict(x=D, h=D, y=D + 16), "overlaps"), (R.EINVAL, dict(x=C, h=C), "d_gain"), (R.EINVAL, dict(x=B - 16, h=B - 16), "d_delta"),
])
def test_norm_refusals(code, change, text):
    refuse(code, R.rollout_rms_norm, *call(NORM, **change), text=text)


@pytest.mark.parametrize("code,change,text", [
    (R.EINVAL, dict(n=0), "n_rows"), (R.EUNSUPPORTED, dict(dim=32769), "32,768"), (R.EINVAL, dict(dyt=3), "dtype"), (R.EINVAL, dict(ht=2), "dtype"),
    (R.EINVAL, dict(dxt=3), "dtype"), (R.EINVAL, dict(acc=2), "accumulate"), (R.EUNSUPPORTED, dict(acc=BIG), "int32"),
    (R.EINVAL, dict(dy=None), "NULL"), (R.EINVAL, dict(h=None), "NULL"), (R.EINVAL, dict(rstd=None), "NULL"), (R.EINVAL, dict(dx=None), "NULL"),
    (R.EINVAL, dict(dx=F + 2), "aligned"), (R.EINVAL, dict(inner=E + 2), "aligned"), (R.EINVAL, dict(dgain=G + 2), "4 bytes"),
    (R.ENOMEM, dict(ws_bytes=8), "workspace"), (R.EINVAL, dict(ws=None), "NULL"), (R.EINVAL, dict(ws_bytes=-1), "workspace"),
    (R.EINVAL, dict(dx=A), "overlaps"), (R.EINVAL, dict(dx=B), "overlaps"), (R.EINVAL, dict(dx=E + 4), "d_grad_h"),
    (R.EINVAL, dict(dgain=C), "d_gain"), (R.EINVAL, dict(ws=F), "workspace overlaps"), (R.EINVAL, dict(dgain=D), "d_rstd"),
])
def test_norm_backward_refusals(code, change, text):
    refuse(code, R.rollout_rms_norm_backward, *call(NORM_BACK, **change), text=text)


def test_norm_calls_that_are_taken():
    accepted(R.rollout_rms_norm, *call(NORM))
    accepted(R.rollout_rms_norm, *call(NORM, h=A))
    accepted(R.rollout_rms_norm, *call(NORM, delta=None, h=None, gain=None, rstd=None))
    accepted(R.rollout_rms_norm, *call(NORM, yt=3, y=E + 1, scales=G))
    accepted(R.rollout_rms_norm, *call(NORM, y=A + 1600))
    accepted(R.rollout_rms_norm_backward, *call(NORM_BACK))
    accepted(R.rollout_rms_norm_backward, *call(NORM_BACK, dx=E, gain=None))
    accepted(R.rollout_rms_norm_backward, *call(NORM_BACK, dgain=None, ws=None, ws_bytes=0, inner=None))
    with pytest.raises(R.RolloutError):
        R.rollout_rms_norm_backward_workspace(0, 5)


def test_norm_workspaces_grow_with_the_call():
    for n in (1, 100, 1024, 4096, 100000):
        last = 0
        for d in (1, 100, 1024, 1025, 2048, 2049, 4096, 8192, 8193, 32768):
            need = R.rollout_rms_norm_backward_workspace(n, d)
            assert need >= last and R.rollout_rms_norm_backward_workspace(n + 1, d) >= need, (n, d)
            last = need


def entry(**change):
    k = dict(d_param=A, d_grad=B, d_m=C, d_v=D, d_m_scales=None, d_v_scales=None, d_copy=None, n=1000, param_dtype=0, grad_dtype=1,
             state_dtype=0, weight_decay=0.1)
    k.update(change)
    return R.AdamwTensor(*k.values())


EIGHT = dict(state_dtype=3, d_m_scales=E, d_v_scales=F)


@pytest.mark.parametrize("code,tensors,text", [
    (R.EINVAL, [], "n_tensors"), (R.EINVAL, [entry(n=-1)], "n must be"), (R.EUNSUPPORTED, [entry(n=(1 << 36) + 1)], "2^36"),
    (R.EINVAL, [entry(param_dtype=2)], "dtype"), (R.EINVAL, [entry(grad_dtype=3)], "dtype"), (R.EINVAL, [entry(state_dtype=1)], "state_dtype"),
    (R.EINVAL, [entry(weight_decay=-0.1)], "weight_decay"), (R.EINVAL, [entry(weight_decay=float("nan"))], "weight_decay"),
    (R.EINVAL, [entry(param_dtype=1, d_copy=G)], "copy"), (R.EINVAL, [entry(d_param=None)], "NULL"), (R.EINVAL, [entry(d_grad=None)], "NULL"),
    (R.EINVAL, [entry(d_m=None)], "NULL"), (R.EINVAL, [entry(d_v=None)], "NULL"), (R.EINVAL, [entry(state_dtype=3)], "NULL"),
    (R.EINVAL, [entry(d_m_scales=E)], "8 bits"), (R.EINVAL, [entry(d_param=A + 2)], "aligned"), (R.EINVAL, [entry(d_grad=B + 1)], "aligned"),
    (R.EINVAL, [entry(**EIGHT | dict(d_m_scales=E + 2))], "aligned"), (R.EINVAL, [entry(d_copy=G + 1)], "aligned"),
    (R.EINVAL, [entry(d_grad=A)], "overlaps"), (R.EINVAL, [entry(d_m=A + 3996)], "overlaps"), (R.EINVAL, [entry(d_v=C)], "overlaps"),
    (R.EINVAL, [entry(**EIGHT | dict(d_v_scales=E + 28))], "overlaps"), (R.EINVAL, [entry(), entry()], "overlaps"),
    (R.EINVAL, [entry(), entry(d_param=G, d_grad=C + 8, d_m=H, d_v=I)], "tensor"),
    (R.EINVAL, [entry(n=0), entry(n=0, param_dtype=7)], "dtype"),
])
def test_adamw_tables(code, tensors, text):
    refuse(code, R.rollout_adamw_table, tensors, text=text)


def test_adamw_tables_that_are_taken():
    table, chunks = R.rollout_adamw_table([entry(), entry(n=0, d_param=None), entry(d_param=G, d_grad=B, d_m=H, d_v=I)])
    assert table.dtype == torch.uint8 and chunks == 2  # (gradients may be shared)
    table, chunks = R.rollout_adamw_table([entry(**EIGHT, d_copy=G, n=5000), entry(d_param=A + 20000, d_grad=B + 10000, d_m=C + 5000 + 3000,
                                                                                     d_v=D + 8000)])
    assert chunks == 4
    assert R.rollout_adamw_table([entry(n=1 << 30), entry(d_param=G, d_grad=H, d_m=I, d_v=J, n=1)])[1] == (1 << 19) + 1
    tight = [entry(d_param=A, d_grad=A + 4000, d_m=A + 6000, d_v=A + 10000)]
    assert R.rollout_adamw_table(tight)[1] == 1
    out, need = ctypes.c_int64(), ctypes.c_uint64()
    arr = (R.AdamwTensor * 2)(entry(), entry())
    assert R.lib.rollout_adamw_table_bytes(2, ctypes.byref(need)) == R.OK
    buf = ctypes.create_string_buffer(need.value)
    assert R.lib.rollout_adamw_table(arr, 2, buf, need.value - 1, ctypes.byref(out)) == R.ENOMEM
    for args in ((None, 2, buf, need.value, ctypes.byref(out)), (arr, 2, None, need.value, ctypes.byref(out)), (arr, 2, buf, need.value, None)):
        assert R.lib.rollout_adamw_table(*args) == R.EINVAL
    assert R.lib.rollout_adamw_table_bytes(2, None) == R.EINVAL
    assert R.lib.rollout_adamw_table_bytes((1 << 20) + 1, ctypes.byref(need)) == R.EUNSUPPORTED


STEP = dict(table=A, tensors=3, chunks=5, lr=1e-3, b1=0.9, b2=0.95, eps=1e-8, step=1, seed=7, scale=B, lr_now=C, step_now=None, stream=None)


@pytest.mark.parametrize("code,change,text", [
    (R.EINVAL, dict(table=None), "table"), (R.EINVAL, dict(table=A + 4), "aligned"), (R.EINVAL, dict(tensors=0), "n_tensors"),
    (R.EUNSUPPORTED, dict(tensors=BIG + 3), "int32"), (R.EUNSUPPORTED, dict(tensors=(1 << 20) + 1), "2^20"), (R.EINVAL, dict(chunks=-1), "n_chunks"),
    (R.EINVAL, dict(chunks=1 << 24), "n_chunks"), (R.EINVAL, dict(lr=float("nan")), "lr"), (R.EINVAL, dict(b1=1.0), "beta"),
    (R.EINVAL, dict(b1=-0.1), "beta"), (R.EINVAL, dict(b2=1.5), "beta"), (R.EINVAL, dict(b2=float("nan")), "beta"), (R.EINVAL, dict(eps=-1.0), "eps"),
    (R.EINVAL, dict(eps=1e-40), "2^-126"), (R.EINVAL, dict(eps=1e39), "eps"), (R.EINVAL, dict(lr=1e39), "lr"),
    (R.EINVAL, dict(eps=float("inf")), "eps"), (R.EINVAL, dict(step=0), "step"), (R.EINVAL, dict(step=-3), "step"),
    (R.EUNSUPPORTED, dict(step=1 << 64), "int64"), (R.EINVAL, dict(seed=-1), "seed"), (R.EINVAL, dict(seed=1 << 64), "seed"),
    (R.EINVAL, dict(scale=B + 2), "4 bytes"), (R.EINVAL, dict(step_now=D + 4), "8 bytes"),
])
def test_adamw_refusals(code, change, text):
    refuse(code, R.rollout_adamw, *call(STEP, **change), text=text)


def test_adamw_calls_that_are_taken():
    accepted(R.rollout_adamw, *call(STEP))
    accepted(R.rollout_adamw, *call(STEP, step=0, step_now=D, seed=(1 << 64) - 1, lr=0.0, b1=0.0, b2=0.0, eps=0.0))


def test_adamw_tensors_are_checked(monkeypatch):
    monkeypatch.setattr(R, "_device", lambda: -1)
    f, h, u = torch.zeros(300), torch.zeros(300, dtype=torch.bfloat16), torch.zeros(300, dtype=torch.uint8)
    s = torch.zeros(3)
    e = R.adamw_tensor(f, h, f, f, 0.1, copy=h)
    assert (e.n, e.param_dtype, e.grad_dtype, e.state_dtype, e.d_copy) == (300, 0, 1, 0, h.data_ptr())
    e = R.adamw_tensor(h, f, u.view(torch.float8_e4m3fn), u, 0.0, s, s)
    assert (e.param_dtype, e.grad_dtype, e.state_dtype, e.d_m_scales) == (1, 0, 3, s.data_ptr())
    for args, kw, text in (((f.double(), f, f, f, 0.0), {}, "float32"), ((f, u, f, f, 0.0), {}, "grad must"), ((f, f, h, f, 0.0), {}, "m must"),
                           ((f, f, f, u, 0.0), {}, "v must"), ((f, f[:299], f, f, 0.0), {}, "grad holds"), ((f, f, f[:9], f, 0.0), {}, "elements"),
                           ((f, f, u, u, 0.0, s[:2], s), {}, "m_scales holds"), ((f, f, f, f, 0.0), dict(copy=f), "copy must"),
                           ((f.view(20, 15).t(), f, f, f, 0.0), {}, "contiguous"), ((f, f.view(20, 15).t(), f, f, 0.0), {}, "contiguous")):
        refuse(R.EINVAL, R.adamw_tensor, *args, text=text, **kw) if not kw else refuse(R.EINVAL, lambda: R.adamw_tensor(*args, **kw), text=text)
    monkeypatch.undo()
    if not R._torch.cuda.is_available():
        refuse(R.EINVAL, R.adamw_tensor, f, f, f, f, 0.0, text="current device")
