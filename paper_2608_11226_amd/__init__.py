"""Python binding of librollout, the MI355X GRPO rollout library.

Argument marshalling only: every step of the rollout runs in the library's
HIP kernels.  The functions below carry the names of the C ABI in
``include/rollout.h`` and take device pointers as integers (or torch tensors,
whose ``data_ptr()`` is passed); PyTorch is used by ``Engine`` only to
allocate device memory and to provide the stream.

The library must have been built (``python paper_2608_11226_amd/build.py``);
importing this package fails loudly when it has not.
"""
from __future__ import annotations

import ctypes
import os

_PKG = os.path.dirname(os.path.abspath(__file__))
# ROLLOUT_LIBRARY may name another build of the same library (the host-sanitizer build of build.py --sanitize)
LIB_PATH = os.environ.get("ROLLOUT_LIBRARY") or os.path.join(_PKG, "librollout.so")

OK, EINVAL, ENOMEM, EDEVICE, ESTATE, EUNSUPPORTED = 0, -1, -2, -3, -4, -5
DTYPE_FP32, DTYPE_BF16, DTYPE_INT4, DTYPE_E4M3 = 0, 1, 2, 3
_NAMES = {EINVAL: "EINVAL", ENOMEM: "ENOMEM", EDEVICE: "EDEVICE", ESTATE: "ESTATE", EUNSUPPORTED: "EUNSUPPORTED"}

EXPORTED = (
    "rollout_plan", "rollout_init", "rollout_prefill", "rollout_decode_step", "rollout_sample",
    "grpo_advantages", "rollout_generate", "rollout_sync", "rollout_destroy", "rollout_last_error",
    "rollout_export_weight", "rollout_profile_decode_step", "rollout_generate_eos", "rollout_length_rewards",
    "rollout_sample_noalloc", "rollout_profile_projections",
    "rollout_token_logprobs_workspace", "rollout_token_logprobs", "rollout_token_logprobs_backward",
    "grpo_policy_loss_workspace", "grpo_policy_loss",
    "rollout_embedding", "rollout_embedding_backward_workspace", "rollout_embedding_backward",
    "rollout_attention_workspace", "rollout_attention", "rollout_attention_backward_workspace", "rollout_attention_backward",
    "rollout_rms_norm", "rollout_rms_norm_backward_workspace", "rollout_rms_norm_backward",
    "rollout_adamw_table_bytes", "rollout_adamw_table", "rollout_adamw",
)
MEAN_SEQUENCE, MEAN_TOKEN, MEAN_FIXED = 0, 1, 2  # ROLLOUT_MEAN_*
NOALLOC_SCRATCH_BYTES = 64 << 20  # ROLLOUT_SAMPLE_NOALLOC_SCRATCH_BYTES
# include/occupancy.h: power metrics and threshold policy of the occupancy controller (host code)
EXPORTED_OCC = (
    "occ_rolling_mean", "occ_violation", "occ_normalize_budget", "occ_hysteresis_step", "occ_monitor_create",
    "occ_monitor_push", "occ_monitor_read", "occ_monitor_state", "occ_monitor_destroy",
)


class RolloutError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{_NAMES.get(code, code)}: {msg}")
        self.code = code


class ModelConfig(ctypes.Structure):
    _fields_ = [
        ("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("d_ff", ctypes.c_int32),
        ("vocab", ctypes.c_int32), ("rms_eps", ctypes.c_float), ("rope_theta", ctypes.c_float),
        ("dtype", ctypes.c_int32), ("weight_seed", ctypes.c_uint64), ("weight_std", ctypes.c_double),
        ("kv_block_size", ctypes.c_int32), ("max_prompt_len", ctypes.c_int32),
        ("max_new_tokens", ctypes.c_int32), ("max_seqs_in_flight", ctypes.c_int32),
        ("hbm_budget_bytes", ctypes.c_uint64),
    ]


class Plan(ctypes.Structure):
    _fields_ = [
        ("seqs_in_flight_max", ctypes.c_int32), ("kv_blocks", ctypes.c_int32), ("arena_bytes", ctypes.c_uint64),
        ("weight_bytes", ctypes.c_uint64), ("kv_block_bytes", ctypes.c_uint64), ("kv_bytes", ctypes.c_uint64),
        ("work_bytes", ctypes.c_uint64),
    ]


class OccReading(ctypes.Structure):
    _fields_ = [
        ("n", ctypes.c_int64), ("p_now_w", ctypes.c_double), ("p_5s_ago_w", ctypes.c_double),
        ("p10_w", ctypes.c_double), ("p30_w", ctypes.c_double), ("violation_rate", ctypes.c_double),
        ("excess_ws", ctypes.c_double), ("peak30_w", ctypes.c_double),
    ]


class ProjectionProfile(ctypes.Structure):
    _fields_ = [
        ("launches", ctypes.c_int32), ("avg_us", ctypes.c_double), ("bytes_per_launch", ctypes.c_double),
        ("flops_per_launch", ctypes.c_double),
    ]


class StepProfile(ctypes.Structure):
    _fields_ = [
        ("ms", ctypes.c_double * 3), ("launches", ctypes.c_int32 * 3),
        ("bytes", ctypes.c_double * 3), ("flops", ctypes.c_double * 3),
    ]


class AttentionShape(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("n_seqs", ctypes.c_int32), ("n_q", ctypes.c_int32), ("n_k", ctypes.c_int32), ("causal", ctypes.c_int32),
        ("scale", ctypes.c_float),
    ]

    def __setattr__(self, name, value):  # (ctypes would keep the low bits of what an int32 does not hold)
        if name != "scale" and not -(1 << 31) <= value < 1 << 31:
            raise RolloutError(EINVAL if value < 0 else EUNSUPPORTED, f"{name}: {value} does not fit an int32")
        super().__setattr__(name, value)


class AdamwTensor(ctypes.Structure):
    _fields_ = [
        ("d_param", ctypes.c_void_p), ("d_grad", ctypes.c_void_p), ("d_m", ctypes.c_void_p), ("d_v", ctypes.c_void_p),
        ("d_m_scales", ctypes.c_void_p), ("d_v_scales", ctypes.c_void_p), ("d_copy", ctypes.c_void_p), ("n", ctypes.c_int64),
        ("param_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32), ("state_dtype", ctypes.c_int32),
        ("weight_decay", ctypes.c_float),
    ]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python paper_2608_11226_amd/build.py`")
    # torch's libraries link the HIP runtime it ships under an unversioned name;
    # loading torch first lets librollout's libamdhip64.so.7 / libhsa-runtime64.so.1
    # resolve to those same copies, so the process holds one HIP runtime.
    import torch  # noqa: F401

    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, f32, u64, f64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_uint64, ctypes.c_double
    i64, pu64 = ctypes.c_int64, ctypes.POINTER(u64)
    shape = ctypes.POINTER(AttentionShape)
    sig = {
        "rollout_plan": ([ctypes.POINTER(ModelConfig), i32, ctypes.POINTER(Plan)], i32),
        "rollout_init": ([ctypes.POINTER(ModelConfig), vp, u64, vp, ctypes.POINTER(vp)], i32),
        "rollout_prefill": ([vp, vp, i32, i32, i32, vp], i32),
        "rollout_decode_step": ([vp, vp, vp], i32),
        "rollout_sample": ([vp, vp, i32, f32, f32, vp, vp], i32),
        "grpo_advantages": ([vp, i32, i32, f32, i32, vp, vp, vp], i32),
        "rollout_generate": ([vp, vp, i32, i32, i32, i32, i32, f32, f32, vp, vp], i32),
        "rollout_sync": ([vp], i32),
        "rollout_destroy": ([vp], None),
        "rollout_last_error": ([vp], ctypes.c_char_p),
        "rollout_export_weight": ([vp, i32, vp], i32),
        "rollout_profile_decode_step": ([vp, vp, vp, ctypes.POINTER(StepProfile)], i32),
        "rollout_generate_eos": ([vp, vp, i32, i32, i32, i32, i32, f32, f32, vp, vp, i32, i32, i32, vp, vp, vp,
                                  ctypes.POINTER(i32)], i32),
        "rollout_length_rewards": ([vp, i32, i32, vp, vp, vp], i32),
        "rollout_sample_noalloc": ([vp, i32, i32, f32, f32, vp, vp, vp], i32),
        "rollout_profile_projections": ([vp, i32, vp, ctypes.POINTER(ProjectionProfile)], i32),
        "rollout_token_logprobs_workspace": ([i32, i32, i32, pu64], i32),
        "rollout_token_logprobs": ([vp, i32, i64, i32, i32, f32, vp, i32, vp, vp, vp, vp, vp, vp, u64, vp], i32),
        "rollout_token_logprobs_backward": ([vp, i32, i64, i32, i32, f32, vp, vp, vp, vp, vp, vp, i64, vp], i32),
        "grpo_policy_loss_workspace": ([i32, i32, pu64], i32),
        "grpo_policy_loss": ([vp, vp, vp, vp, vp, vp, i32, i32, f32, f32, f32, f32, i32, vp, vp, vp, vp, vp, u64, vp], i32),
        "rollout_embedding": ([vp, i32, i32, i32, vp, i32, f32, vp, i32, vp], i32),
        "rollout_embedding_backward_workspace": ([i32, i32, i32, pu64], i32),
        "rollout_embedding_backward": ([vp, i32, vp, i32, i32, i32, f32, i32, vp, i32, vp, u64, vp], i32),
        "rollout_attention_workspace": ([shape, pu64], i32),
        "rollout_attention": ([shape, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, i64, vp, vp, u64, vp], i32),
        "rollout_attention_backward_workspace": ([shape, pu64], i32),
        "rollout_attention_backward": ([shape, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, i64, vp, vp, i64, vp, i64, vp, i64,
                                        vp, i64, vp, u64, vp], i32),
        "rollout_rms_norm": ([vp, i32, vp, i32, vp, i32, i32, f32, vp, vp, i32, vp, vp, vp], i32),
        "rollout_rms_norm_backward_workspace": ([i32, i32, pu64], i32),
        "rollout_rms_norm_backward": ([vp, i32, vp, i32, vp, vp, i32, i32, vp, vp, i32, vp, i32, vp, u64, vp], i32),
        "rollout_adamw_table_bytes": ([i32, pu64], i32),
        "rollout_adamw_table": ([ctypes.POINTER(AdamwTensor), i32, vp, u64, ctypes.POINTER(i64)], i32),
        "rollout_adamw": ([vp, i32, i64, f64, f64, f64, f64, i64, u64, vp, vp, vp, vp], i32),
        "occ_rolling_mean": ([vp, ctypes.c_int64, f64, f64, vp], i32),
        "occ_violation": ([vp, ctypes.c_int64, f64, f64, ctypes.POINTER(f64), ctypes.POINTER(f64)], i32),
        "occ_normalize_budget": ([f64, f64, f64], f64),
        "occ_hysteresis_step": ([i32, i32, f64, f64, f64, f64, f64], i32),
        "occ_monitor_create": ([f64, f64], vp),
        "occ_monitor_push": ([vp, f64], i32),
        "occ_monitor_read": ([vp, ctypes.POINTER(OccReading)], i32),
        "occ_monitor_state": ([vp, i32, i32, f64, vp], i32),
        "occ_monitor_destroy": ([vp], None),
    }
    for name, (args, res) in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    return lib


lib = _load()

import torch as _torch  # noqa: E402  (loaded above)

_F, _I, _U8 = _torch.float32, _torch.int32, _torch.uint8
_TYPES = {DTYPE_FP32: _torch.float32, DTYPE_BF16: _torch.bfloat16}


def _ptr(x) -> int | None:
    """Device pointer of a tensor (data_ptr) or an integer address; None stays NULL."""
    if x is None:
        return None
    if hasattr(x, "data_ptr"):
        return x.data_ptr()
    return int(x)


def _check(code: int, ctx=None):
    if code != OK:
        raise RolloutError(code, lib.rollout_last_error(ctx).decode())


# ---------------------------------------------------------------------------
# C ABI, one wrapper per entry point
# ---------------------------------------------------------------------------
def rollout_plan(cfg: ModelConfig, group_size: int) -> Plan:
    out = Plan()
    _check(lib.rollout_plan(ctypes.byref(cfg), group_size, ctypes.byref(out)))
    return out


def rollout_init(cfg: ModelConfig, arena, arena_bytes: int, stream=None) -> int:
    ctx = ctypes.c_void_p()
    _check(lib.rollout_init(ctypes.byref(cfg), _ptr(arena), arena_bytes, _ptr(stream), ctypes.byref(ctx)))
    return ctx.value


def rollout_prefill(ctx, prompts, n_prompts: int, prompt_len: int, group_size: int, logits):
    _check(lib.rollout_prefill(ctx, _ptr(prompts), n_prompts, prompt_len, group_size, _ptr(logits)), ctx)


def rollout_decode_step(ctx, tokens, logits):
    _check(lib.rollout_decode_step(ctx, _ptr(tokens), _ptr(logits)), ctx)


def rollout_sample(ctx, logits, n_seqs: int, temperature: float, top_p: float, uniforms, tokens_out):
    _check(lib.rollout_sample(ctx, _ptr(logits), n_seqs, temperature, top_p, _ptr(uniforms), _ptr(tokens_out)), ctx)


def rollout_sample_noalloc(logits, n_seqs: int, vocab: int, temperature: float, top_p: float, uniforms, tokens_out,
                           stream=None):
    _check(lib.rollout_sample_noalloc(_ptr(logits), n_seqs, vocab, temperature, top_p, _ptr(uniforms),
                                      _ptr(tokens_out), _ptr(stream)))


def grpo_advantages(rewards, n_groups: int, group_size: int, eps: float, std_ddof: int, adv, zero_var=None,
                    stream=None):
    _check(lib.grpo_advantages(_ptr(rewards), n_groups, group_size, eps, std_ddof, _ptr(adv), _ptr(zero_var),
                               _ptr(stream)))


def rollout_generate(ctx, prompts, n_prompts: int, prompt_len: int, group_size: int, seqs_in_flight: int,
                     max_new_tokens: int, temperature: float, top_p: float, uniforms, tokens_out):
    _check(lib.rollout_generate(ctx, _ptr(prompts), n_prompts, prompt_len, group_size, seqs_in_flight,
                                max_new_tokens, temperature, top_p, _ptr(uniforms), _ptr(tokens_out)), ctx)


def rollout_generate_eos(ctx, prompts, n_prompts: int, prompt_len: int, group_size: int, seqs_in_flight: int,
                         max_new_tokens: int, temperature: float, top_p: float, uniforms, stop_ids, n_stop: int,
                         refill_interval: int, whole_groups: int, tokens_out, lengths_out,
                         admit_step_out=None) -> int:
    """Returns the number of decode steps run."""
    steps = ctypes.c_int32(0)
    _check(lib.rollout_generate_eos(ctx, _ptr(prompts), n_prompts, prompt_len, group_size, seqs_in_flight,
                                    max_new_tokens, temperature, top_p, _ptr(uniforms), _ptr(stop_ids), n_stop,
                                    refill_interval, whole_groups, _ptr(tokens_out), _ptr(lengths_out),
                                    _ptr(admit_step_out), ctypes.byref(steps)), ctx)
    return steps.value


def rollout_length_rewards(lengths, n: int, target: int, rewards, total_tokens=None, stream=None):
    _check(lib.rollout_length_rewards(_ptr(lengths), n, target, _ptr(rewards), _ptr(total_tokens), _ptr(stream)))


# The update side of a GRPO step: no context, caller-owned workspaces.  A tensor passed for a buffer has to be on the
# current device, of the buffer's type, contiguous (the rows of logits may be strided, by the row stride of the call) and
# large enough; a contiguous one is taken as so many elements in a row, whatever its shape, and an integer address is
# passed on as it is.  Workspaces are uint8 tensors.
def _buf(name: str, x, kind, n: int, device: int, rows=None) -> int | None:
    """Device pointer of a buffer of n elements of a torch type.  rows: (rows, stride, width) of a matrix whose rows may
    be apart."""
    if type(x) is _torch.Tensor:
        if x.dtype is kind and x.is_contiguous() and x.numel() >= n and x.get_device() == device:
            return x.data_ptr()
    elif x is None or type(x) is int:
        return x
    elif not hasattr(x, "is_contiguous"):
        return _ptr(x)
    elif x.dtype is kind and x.is_contiguous() and x.numel() >= n and x.get_device() == device:
        return x.data_ptr()
    if x.dtype is not kind:
        raise RolloutError(EINVAL, f"{name} must be {kind}, not {x.dtype}")
    if x.get_device() != device:
        raise RolloutError(EINVAL, f"{name} is on {x.device}, not on the current device")
    if not x.is_contiguous():
        if rows is None or x.stride(-1) != 1:
            raise RolloutError(EINVAL, f"{name} is not contiguous")
        _strided_rows(name, x, *rows)
    elif x.numel() < n:
        raise RolloutError(EINVAL, f"{name} holds {x.numel()} elements, the call needs {n}")
    return x.data_ptr()


def _strided_rows(name: str, x, n: int, stride: int, width: int):
    """Row r of the call is row r of x, for all n of them (dimensions before the last count rows)."""
    if x.shape[-1] < width:
        raise RolloutError(EINVAL, f"{name} has rows of {x.shape[-1]} elements, the call needs {width}")
    have = 1
    for size, step in zip(reversed(x.shape[:-1]), reversed(x.stride()[:-1])):
        if size > 1 and have < n:
            if step != stride * have:
                raise RolloutError(EINVAL, f"{name} has rows {step} elements apart, not {stride * have}")
            have *= size
    if have < n:
        raise RolloutError(EINVAL, f"{name} holds {have} rows, the call needs {n}")


def _sizes(ints, longs=(), size: int = 0):
    """Numbers that the library's int32, int64 and uint64 arguments hold.  ctypes would pass on the low bits of others.
    Called where one of them is negative or above 2^31 - 1, which is rare."""
    for x, bits in [(x, 31) for x in ints] + [(x, 63) for x in longs]:
        if not -(1 << bits) <= x < 1 << bits:
            raise RolloutError(EINVAL if x < 0 else EUNSUPPORTED, f"{x} does not fit an int{bits + 1}")
    if not 0 <= size < 1 << 64:
        raise RolloutError(EINVAL, f"a workspace of {size} bytes")


def _kind(dtype: int):
    kind = _TYPES.get(dtype)
    if kind is None:
        raise RolloutError(EINVAL, f"dtype must be 0 (fp32) or 1 (bf16), not {dtype}")
    return kind


def _device() -> int:
    return _torch.cuda.current_device() if _torch.cuda.is_initialized() else -2  # no tensor's


def rollout_token_logprobs_workspace(n_rows: int, vocab: int, n_top: int = 0) -> int:
    if (n_rows | vocab | n_top) >> 31:
        _sizes((n_rows, vocab, n_top))
    out = ctypes.c_uint64(0)
    _check(lib.rollout_token_logprobs_workspace(n_rows, vocab, n_top, ctypes.byref(out)))
    return out.value


def rollout_token_logprobs(logits, dtype: int, row_stride: int, n_rows: int, vocab: int, temperature: float, tokens,
                           n_top: int = 0, logp=None, entropy=None, stats=None, top_ids=None, top_logp=None,
                           workspace=None, workspace_bytes: int = 0, stream=None):
    if (n_rows | vocab | n_top | row_stride | workspace_bytes) >> 31:
        _sizes((n_rows, vocab, n_top), (row_stride,), workspace_bytes)
    dev = _device()
    _check(lib.rollout_token_logprobs(
        _buf("logits", logits, _kind(dtype), (n_rows - 1) * row_stride + vocab, dev, (n_rows, row_stride, vocab)),
        dtype, row_stride, n_rows, vocab, temperature,
        _buf("tokens", tokens, _I, n_rows, dev), n_top, _buf("logp", logp, _F, n_rows, dev),
        _buf("entropy", entropy, _F, n_rows, dev),
        _buf("stats", stats, _F, 2 * n_rows, dev), _buf("top_ids", top_ids, _I, n_rows * n_top, dev),
        _buf("top_logp", top_logp, _F, n_rows * n_top, dev), _buf("workspace", workspace, _U8, workspace_bytes, dev),
        workspace_bytes, _ptr(stream)))


def rollout_token_logprobs_backward(logits, dtype: int, row_stride: int, n_rows: int, vocab: int, temperature: float,
                                    tokens, stats, entropy, grad_logp, grad_entropy, grad_logits, grad_stride: int,
                                    stream=None):
    if (n_rows | vocab | row_stride | grad_stride) >> 31:
        _sizes((n_rows, vocab), (row_stride, grad_stride))
    dev = _device()
    _check(lib.rollout_token_logprobs_backward(
        _buf("logits", logits, _kind(dtype), (n_rows - 1) * row_stride + vocab, dev, (n_rows, row_stride, vocab)),
        dtype, row_stride, n_rows, vocab, temperature,
        _buf("tokens", tokens, _I, n_rows, dev), _buf("stats", stats, _F, 2 * n_rows, dev),
        _buf("entropy", entropy, _F, n_rows, dev),
        _buf("grad_logp", grad_logp, _F, n_rows, dev), _buf("grad_entropy", grad_entropy, _F, n_rows, dev),
        _buf("grad_logits", grad_logits, _kind(dtype), (n_rows - 1) * grad_stride + vocab, dev, (n_rows, grad_stride, vocab)),
        grad_stride, _ptr(stream)))


def grpo_policy_loss_workspace(n_seqs: int, max_len: int) -> int:
    if (n_seqs | max_len) >> 31:
        _sizes((n_seqs, max_len))
    out = ctypes.c_uint64(0)
    _check(lib.grpo_policy_loss_workspace(n_seqs, max_len, ctypes.byref(out)))
    return out.value


def grpo_policy_loss(logp, old_logp, ref_logp, entropy, adv, lengths, n_seqs: int, max_len: int, clip_low: float,
                     clip_high: float, kl_coef: float, entropy_coef: float, mean: int, loss=None, stats=None,
                     grad_logp=None, grad_entropy=None, workspace=None, workspace_bytes: int = 0, stream=None):
    if (n_seqs | max_len | mean | workspace_bytes) >> 31:
        _sizes((n_seqs, max_len, mean), (), workspace_bytes)
    dev = _device()
    n = n_seqs * max_len
    _check(lib.grpo_policy_loss(
        _buf("logp", logp, _F, n, dev), _buf("old_logp", old_logp, _F, n, dev), _buf("ref_logp", ref_logp, _F, n, dev),
        _buf("entropy", entropy, _F, n, dev), _buf("adv", adv, _F, n_seqs, dev),
        _buf("lengths", lengths, _I, n_seqs, dev), n_seqs,
        max_len, clip_low, clip_high, kl_coef, entropy_coef, mean, _buf("loss", loss, _F, 1, dev),
        _buf("stats", stats, _F, 5, dev),
        _buf("grad_logp", grad_logp, _F, n, dev), _buf("grad_entropy", grad_entropy, _F, n, dev),
        _buf("workspace", workspace, _U8, workspace_bytes, dev), workspace_bytes, _ptr(stream)))


def rollout_embedding(table, table_dtype: int, vocab: int, dim: int, tokens, n_tokens: int, scale: float, out,
                      out_dtype: int, stream=None):
    if (n_tokens | vocab | dim) >> 31:
        _sizes((n_tokens, vocab, dim))
    dev = _device()
    _check(lib.rollout_embedding(
        _buf("table", table, _kind(table_dtype), vocab * dim, dev), table_dtype, vocab, dim,
        _buf("tokens", tokens, _I, n_tokens, dev),
        n_tokens, scale, _buf("out", out, _kind(out_dtype), n_tokens * dim, dev), out_dtype, _ptr(stream)))


def rollout_embedding_backward_workspace(n_tokens: int, vocab: int, dim: int) -> int:
    if (n_tokens | vocab | dim) >> 31:
        _sizes((n_tokens, vocab, dim))
    out = ctypes.c_uint64(0)
    _check(lib.rollout_embedding_backward_workspace(n_tokens, vocab, dim, ctypes.byref(out)))
    return out.value


def rollout_embedding_backward(grad, grad_dtype: int, tokens, n_tokens: int, vocab: int, dim: int, scale: float,
                               accumulate: int, grad_table, table_dtype: int, workspace=None, workspace_bytes: int = 0,
                               stream=None):
    if (n_tokens | vocab | dim | accumulate | workspace_bytes) >> 31:
        _sizes((n_tokens, vocab, dim, accumulate), (), workspace_bytes)
    dev = _device()
    _check(lib.rollout_embedding_backward(
        _buf("grad", grad, _kind(grad_dtype), n_tokens * dim, dev), grad_dtype,
        _buf("tokens", tokens, _I, n_tokens, dev), n_tokens, vocab,
        dim, scale, accumulate, _buf("grad_table", grad_table, _kind(table_dtype), vocab * dim, dev), table_dtype,
        _buf("workspace", workspace, _U8, workspace_bytes, dev), workspace_bytes, _ptr(stream)))


def _matrix(name: str, x, kind, n: int, stride: int, width: int, device: int):
    """A matrix of n rows of width elements, stride apart."""
    if type(x) is _torch.Tensor and x.dtype is kind and x.get_device() == device and x.stride() == (stride, 1):
        have, wide = x.shape
        if have >= n and wide >= width:
            return x.data_ptr()
    return _buf(name, x, kind, (n - 1) * stride + width, device, (n, stride, width))


def rollout_attention_workspace(shape: AttentionShape) -> int:
    out = ctypes.c_uint64(0)
    _check(lib.rollout_attention_workspace(ctypes.byref(shape), ctypes.byref(out)))
    return out.value


def rollout_attention(shape: AttentionShape, q, q_stride: int, k, k_stride: int, v, v_stride: int, q_starts, q_lens, k_starts,
                      k_lens, out, out_stride: int, lse, workspace=None, workspace_bytes: int = 0, stream=None):
    if (q_stride | k_stride | v_stride | out_stride | workspace_bytes) >> 31:
        _sizes((), (q_stride, k_stride, v_stride, out_stride), workspace_bytes)
    dev, kind = _device(), _kind(shape.dtype)
    nq, nk, wq, wk, S = shape.n_q, shape.n_k, shape.n_heads * shape.head_dim, shape.n_kv_heads * shape.head_dim, shape.n_seqs
    _check(lib.rollout_attention(
        ctypes.byref(shape), _matrix("q", q, kind, nq, q_stride, wq, dev), q_stride, _matrix("k", k, kind, nk, k_stride, wk, dev),
        k_stride, _matrix("v", v, kind, nk, v_stride, wk, dev), v_stride, _buf("q_starts", q_starts, _I, S + 1, dev),
        _buf("q_lens", q_lens, _I, S, dev), _buf("k_starts", k_starts, _I, S + 1, dev), _buf("k_lens", k_lens, _I, S, dev),
        _matrix("out", out, kind, nq, out_stride, wq, dev), out_stride, _buf("lse", lse, _F, shape.n_heads * nq, dev),
        _buf("workspace", workspace, _U8, workspace_bytes, dev), workspace_bytes, _ptr(stream)))


def rollout_attention_backward_workspace(shape: AttentionShape) -> int:
    out = ctypes.c_uint64(0)
    _check(lib.rollout_attention_backward_workspace(ctypes.byref(shape), ctypes.byref(out)))
    return out.value


def rollout_attention_backward(shape: AttentionShape, q, q_stride: int, k, k_stride: int, v, v_stride: int, q_starts, q_lens,
                               k_starts, k_lens, out, out_stride: int, lse, grad_out, grad_out_stride: int, grad_q,
                               grad_q_stride: int, grad_k, grad_k_stride: int, grad_v, grad_v_stride: int, workspace=None,
                               workspace_bytes: int = 0, stream=None):
    strides = (q_stride, k_stride, v_stride, out_stride, grad_out_stride, grad_q_stride, grad_k_stride, grad_v_stride)
    if any(s >> 31 for s in strides) or workspace_bytes >> 31:
        _sizes((), strides, workspace_bytes)
    dev, kind = _device(), _kind(shape.dtype)
    nq, nk, wq, wk, S = shape.n_q, shape.n_k, shape.n_heads * shape.head_dim, shape.n_kv_heads * shape.head_dim, shape.n_seqs
    _check(lib.rollout_attention_backward(
        ctypes.byref(shape), _matrix("q", q, kind, nq, q_stride, wq, dev), q_stride, _matrix("k", k, kind, nk, k_stride, wk, dev),
        k_stride, _matrix("v", v, kind, nk, v_stride, wk, dev), v_stride, _buf("q_starts", q_starts, _I, S + 1, dev),
        _buf("q_lens", q_lens, _I, S, dev), _buf("k_starts", k_starts, _I, S + 1, dev), _buf("k_lens", k_lens, _I, S, dev),
        _matrix("out", out, kind, nq, out_stride, wq, dev), out_stride, _buf("lse", lse, _F, shape.n_heads * nq, dev),
        _matrix("grad_out", grad_out, kind, nq, grad_out_stride, wq, dev), grad_out_stride,
        _matrix("grad_q", grad_q, kind, nq, grad_q_stride, wq, dev), grad_q_stride,
        _matrix("grad_k", grad_k, kind, nk, grad_k_stride, wk, dev), grad_k_stride,
        _matrix("grad_v", grad_v, kind, nk, grad_v_stride, wk, dev), grad_v_stride,
        _buf("workspace", workspace, _U8, workspace_bytes, dev), workspace_bytes, _ptr(stream)))


def rollout_rms_norm(x, x_dtype: int, delta, delta_dtype: int, gain, n_rows: int, dim: int, eps: float, h, y, y_dtype: int,
                     scales=None, rstd=None, stream=None):
    if (n_rows | dim) >> 31:
        _sizes((n_rows, dim))
    dev, n = _device(), n_rows * dim
    _check(lib.rollout_rms_norm(
        _buf("x", x, _kind(x_dtype), n, dev), x_dtype, _buf("delta", delta, None if delta is None else _kind(delta_dtype), n, dev),
        delta_dtype, _buf("gain", gain, _F, dim, dev), n_rows, dim, eps, _buf("h", h, _kind(x_dtype), n, dev),
        _code_buf("y", y, n, dev) if y_dtype == DTYPE_E4M3 else _buf("y", y, _kind(y_dtype), n, dev), y_dtype,
        _buf("scales", scales, _F, n_rows, dev), _buf("rstd", rstd, _F, n_rows, dev), _ptr(stream)))


def rollout_rms_norm_backward_workspace(n_rows: int, dim: int) -> int:
    if (n_rows | dim) >> 31:
        _sizes((n_rows, dim))
    out = ctypes.c_uint64(0)
    _check(lib.rollout_rms_norm_backward_workspace(n_rows, dim, ctypes.byref(out)))
    return out.value


def rollout_rms_norm_backward(grad_y, grad_y_dtype: int, h, h_dtype: int, gain, rstd, n_rows: int, dim: int, grad_h, grad_x,
                              grad_x_dtype: int, grad_gain=None, accumulate: int = 0, workspace=None, workspace_bytes: int = 0,
                              stream=None):
    if (n_rows | dim | accumulate | workspace_bytes) >> 31:
        _sizes((n_rows, dim, accumulate), (), workspace_bytes)
    dev, n, kind = _device(), n_rows * dim, _kind(grad_x_dtype)
    _check(lib.rollout_rms_norm_backward(
        _buf("grad_y", grad_y, _kind(grad_y_dtype), n, dev), grad_y_dtype, _buf("h", h, _kind(h_dtype), n, dev), h_dtype,
        _buf("gain", gain, _F, dim, dev), _buf("rstd", rstd, _F, n_rows, dev), n_rows, dim, _buf("grad_h", grad_h, kind, n, dev),
        _buf("grad_x", grad_x, kind, n, dev), grad_x_dtype, _buf("grad_gain", grad_gain, _F, dim, dev), accumulate,
        _buf("workspace", workspace, _U8, workspace_bytes, dev), workspace_bytes, _ptr(stream)))


def _code_buf(name: str, x, n: int, device: int) -> int | None:
    """A buffer of e4m3 codes: torch's type of that name, or plain bytes."""
    return _buf(name, x, _U8 if getattr(x, "dtype", None) is _U8 else _torch.float8_e4m3fn, n, device)


def adamw_tensor(param, grad, m, v, weight_decay: float, m_scales=None, v_scales=None, copy=None) -> AdamwTensor:
    """A table entry from tensors on the current device: contiguous, as many elements each as param (scales: one for 128).
    Moments of torch.float8_e4m3fn or torch.uint8 are codes.  The entry keeps addresses only: the tensors have to live as
    long as the table is used."""
    dev, n = _device(), param.numel()
    codes = {t: c for c, t in _TYPES.items()}
    for name, x in (("param", param), ("grad", grad)):
        if x.dtype not in codes:
            raise RolloutError(EINVAL, f"{name} must be torch.float32 or torch.bfloat16, not {x.dtype}")
        if not x.is_contiguous():
            raise RolloutError(EINVAL, f"{name} is not contiguous")
    eight = m.dtype in (_U8, _torch.float8_e4m3fn)
    state = (lambda name, x: _code_buf(name, x, n, dev)) if eight else (lambda name, x: _buf(name, x, _F, n, dev))
    blocks = (n + 127) // 128
    for name, x in (("grad", grad), ("m", m), ("v", v), ("copy", copy)):
        if x is not None and x.numel() != n:
            raise RolloutError(EINVAL, f"{name} holds {x.numel()} elements, not {n}")
    return AdamwTensor(
        _buf("param", param, param.dtype, n, dev), _buf("grad", grad, grad.dtype, n, dev), state("m", m), state("v", v),
        _buf("m_scales", m_scales, _F, blocks, dev), _buf("v_scales", v_scales, _F, blocks, dev),
        _buf("copy", copy, _torch.bfloat16, n, dev), n, codes[param.dtype], codes[grad.dtype],
        DTYPE_E4M3 if eight else DTYPE_FP32, weight_decay)


def rollout_adamw_table(tensors):
    """(the table as a uint8 tensor in host memory, its number of chunks) of a list of AdamwTensor.  Copy the table to the
    device and pass that to rollout_adamw."""
    n, need, chunks = len(tensors), ctypes.c_uint64(0), ctypes.c_int64(0)
    _check(lib.rollout_adamw_table_bytes(n, ctypes.byref(need)))
    table = _torch.zeros(need.value, dtype=_U8)
    _check(lib.rollout_adamw_table((AdamwTensor * n)(*tensors), n, table.data_ptr(), need.value, ctypes.byref(chunks)))
    return table, chunks.value


def rollout_adamw(table, n_tensors: int, n_chunks: int, lr: float, beta1: float, beta2: float, eps: float, step: int, seed: int = 0,
                  grad_scale=None, lr_now=None, step_now=None, stream=None):
    """lr_now fp32 [1] and step_now int64 [1], on the device, replace lr and step."""
    if (n_tensors | n_chunks | step | seed) >> 31:
        _sizes((n_tensors,), (n_chunks, step))
        if not 0 <= seed < 1 << 64:
            raise RolloutError(EINVAL, f"the seed {seed} does not fit a uint64")
    dev = _device()
    need = ctypes.c_uint64(0)
    _check(lib.rollout_adamw_table_bytes(n_tensors, ctypes.byref(need)))
    _check(lib.rollout_adamw(
        _buf("table", table, _U8, need.value, dev), n_tensors, n_chunks, lr, beta1, beta2, eps, step, seed,
        _buf("grad_scale", grad_scale, _F, 1, dev), _buf("lr_now", lr_now, _F, 1, dev),
        _buf("step_now", step_now, _torch.int64, 1, dev), _ptr(stream)))


def rollout_sync(ctx):
    _check(lib.rollout_sync(ctx), ctx)


def rollout_destroy(ctx):
    lib.rollout_destroy(ctx)


def rollout_last_error(ctx=None) -> str:
    return lib.rollout_last_error(ctx).decode()


def rollout_export_weight(ctx, tensor_id: int, out):
    _check(lib.rollout_export_weight(ctx, tensor_id, _ptr(out)), ctx)


def rollout_profile_projections(ctx, reps: int, logits) -> ProjectionProfile:
    out = ProjectionProfile()
    _check(lib.rollout_profile_projections(ctx, reps, _ptr(logits), ctypes.byref(out)), ctx)
    return out


def rollout_profile_decode_step(ctx, tokens, logits) -> StepProfile:
    out = StepProfile()
    _check(lib.rollout_profile_decode_step(ctx, _ptr(tokens), _ptr(logits), ctypes.byref(out)), ctx)
    return out


# ---------------------------------------------------------------------------
# Model shapes of the synthetic workloads
# ---------------------------------------------------------------------------
SHAPES = {
    # n_layers, d_model, n_heads, n_kv_heads, head_dim, d_ff, vocab, rope_theta
    "tiny": (2, 128, 4, 4, 32, 512, 1024, 1e4),
    "7b": (28, 3584, 28, 4, 128, 18944, 152064, 1e6),
    "14b": (48, 5120, 40, 8, 128, 13824, 152064, 1e6),
    "72b": (80, 8192, 64, 8, 128, 29568, 152064, 1e6),
}


# ---------------------------------------------------------------------------
# include/occupancy.h (host code: arrays are float64 NumPy arrays)
# ---------------------------------------------------------------------------
def _f64(a):
    import numpy as np

    return np.ascontiguousarray(a, dtype=np.float64)


def occ_rolling_mean(p, dt_s: float, window_s: float):
    import numpy as np

    p = _f64(p)
    out = np.empty_like(p)
    _check(lib.occ_rolling_mean(p.ctypes.data, len(p), dt_s, window_s, out.ctypes.data))
    return out


def occ_violation(p30, budget_w: float, dt_s: float):
    p30 = _f64(p30)
    rate, excess = ctypes.c_double(), ctypes.c_double()
    _check(lib.occ_violation(p30.ctypes.data, len(p30), budget_w, dt_s, ctypes.byref(rate), ctypes.byref(excess)))
    return rate.value, excess.value


def occ_normalize_budget(budget_cal_w: float, p4_new_w: float, p4_cal_w: float) -> float:
    return lib.occ_normalize_budget(budget_cal_w, p4_new_w, p4_cal_w)


def occ_hysteresis_step(level_idx: int, n_levels: int, p30_w: float, p10_w: float, drop_w: float, climb30_w: float,
                        climb10_w: float) -> int:
    r = lib.occ_hysteresis_step(level_idx, n_levels, p30_w, p10_w, drop_w, climb30_w, climb10_w)
    if r < 0:
        raise RolloutError(EINVAL, "level index outside [0, n_levels)")
    return r


class OccMonitor:
    """occ_monitor_*: eq. (1) means and eqs. (2)-(3) accumulated over pushed power samples."""

    def __init__(self, dt_s: float, budget_w: float):
        self.h = lib.occ_monitor_create(dt_s, budget_w)
        if not self.h:
            raise RolloutError(EINVAL, "occ_monitor_create: dt_s must be > 0")
        self.dt_s, self.budget_w = dt_s, budget_w

    def push(self, power_w: float):
        _check(lib.occ_monitor_push(self.h, power_w))

    def read(self) -> OccReading:
        r = OccReading()
        _check(lib.occ_monitor_read(self.h, ctypes.byref(r)))
        return r

    def state(self, level: int, prev_level: int, prev_duration_s: float):
        import numpy as np

        out = np.empty(8, dtype=np.float64)
        _check(lib.occ_monitor_state(self.h, level, prev_level, prev_duration_s, out.ctypes.data))
        return out

    def close(self):
        if self.h:
            lib.occ_monitor_destroy(self.h)
            self.h = None

    def __del__(self):
        self.close()


def model_config(shape, dtype: int, max_prompt_len: int, max_new_tokens: int, max_seqs_in_flight: int,
                 n_layers: int | None = None, weight_seed: int = 0, weight_std: float = 0.02,
                 kv_block_size: int = 16, rms_eps: float = 1e-6, hbm_budget_bytes: int = 0) -> ModelConfig:
    """ModelConfig for a named shape (or a tuple in SHAPES order); n_layers overrides the depth."""
    t = SHAPES[shape] if isinstance(shape, str) else tuple(shape)
    return ModelConfig(
        n_layers=n_layers or t[0], d_model=t[1], n_heads=t[2], n_kv_heads=t[3], head_dim=t[4], d_ff=t[5],
        vocab=t[6], rms_eps=rms_eps, rope_theta=t[7], dtype=dtype, weight_seed=weight_seed,
        weight_std=weight_std, kv_block_size=kv_block_size, max_prompt_len=max_prompt_len,
        max_new_tokens=max_new_tokens, max_seqs_in_flight=max_seqs_in_flight,
        hbm_budget_bytes=hbm_budget_bytes)


class Engine:
    """A context plus the device arena it lives in (torch supplies memory and the stream)."""

    def __init__(self, cfg: ModelConfig, group_size: int = 1, device: str = "cuda:0", stream=None):
        import torch

        self.torch = torch
        self.device = torch.device(device)
        plan = rollout_plan(cfg, group_size)
        cfg.max_seqs_in_flight = plan.seqs_in_flight_max
        plan = rollout_plan(cfg, group_size)
        self.cfg, self.plan = cfg, plan
        self.arena = torch.empty(plan.arena_bytes, dtype=torch.uint8, device=self.device)
        self.stream = stream or torch.cuda.Stream(device=self.device)
        self.ctx = rollout_init(cfg, self.arena, plan.arena_bytes, self.stream.cuda_stream)

    @property
    def stream_handle(self) -> int:
        return self.stream.cuda_stream

    def synchronize(self):
        rollout_sync(self.ctx)

    def close(self):
        if self.ctx:
            rollout_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
