"""Thin Python binding of libgrpo's C ABI (see include/grpo.h).

Argument marshalling only: tensors become raw device pointers, sizes and the
current HIP stream; every step of the computation runs in the library's kernels.
There is no fallback: if the shared library cannot be loaded the call raises.

The small entry points take an ordinary call (plain tensors and numbers; no stream given, and no output but the
gradient's tensor) through _fastcall (csrc/fastcall.cpp), which does the same in native code: the two calls of a step
on 512 x 1024 logits took 28.8 us and take 19.5, the four of the shaping of a small rollout step 36.3 and 25.2.  It
declines every call that is not ordinary, and the Python below it, which checks and converts everything, takes it.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os
import threading
import warnings

import torch  # imported first so that the HIP runtime torch ships is the one in the process

from . import build as _build

GRPO_OK = 0
GRPO_F32, GRPO_BF16 = 0, 1
COUNT_NAMES = ("tokens", "clip_high", "clip_low", "delta", "out_of_band")

_lib = None
_lib_lock = threading.Lock()


class _NoFastcall:
    """In _fastcall's place before lib() has loaded it, or where it cannot be loaded: declines every call."""

    def __getattr__(self, name):
        return self._decline

    @staticmethod
    def _decline(*args):
        return None


_fast = _NoFastcall()


def _load_fastcall():
    """The binding's native part, built if there is none for these sources and this torch; None, with a warning, where it
    cannot be had (no compiler or headers): the general path can do every call."""
    try:
        path = _build.fastcall_path()
        if not os.path.exists(path):
            _build.build_fastcall()
        loader = importlib.machinery.ExtensionFileLoader("_fastcall", path)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_fastcall", loader))
        loader.exec_module(module)
        return module
    except (ImportError, OSError, RuntimeError) as e:
        warnings.warn("libgrpo's small calls take the general Python path, which is slower: the binding's native part cannot "
                      "be loaded (%s)" % e, RuntimeWarning, stacklevel=3)
        return None


class GrpoError(RuntimeError):
    def __init__(self, status, where):
        self.status = int(status)
        super().__init__("%s failed: %s (status %d)" % (where, status_string(status), status))


def lib():
    """The loaded C library with argument types declared, and with it the binding's native part.  Builds them only if absent."""
    if _lib is None:
        with _lib_lock:  # one thread builds and loads
            if _lib is None:
                _load_lib()
    return _lib


def _load_lib():
    global _lib, _fast
    path = _build.LIB_PATH
    if not os.path.exists(path):
        path = _build.build_library()
    L = ctypes.CDLL(path)
    vp, i64, i32, f32, f64, sz = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int,
                                  ctypes.c_float, ctypes.c_double, ctypes.c_size_t)
    L.grpo_status_string.restype = ctypes.c_char_p
    L.grpo_status_string.argtypes = [i32]
    L.grpo_workspace_bytes.restype = sz
    L.grpo_workspace_bytes.argtypes = [i64]
    L.grpo_row_kernel_plan.restype = i32
    L.grpo_row_kernel_plan.argtypes = [i32, i64, ctypes.POINTER(RowPlan)]
    L.grpo_group_advantages.restype = i32
    L.grpo_group_advantages.argtypes = [vp, i64, vp, i64, i64, f32, i32, vp, vp, i64, vp, vp]
    L.grpo_logprobs_fwd.restype = i32
    L.grpo_logprobs_fwd.argtypes = [vp, i32, i64, i64, i64, vp, vp, f32, vp, vp, sz, vp]
    L.grpo_loss_fwd_bwd.restype = i32
    L.grpo_loss_fwd_bwd.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, vp, f32, f32, f32, f32,
                                    f64, f32, vp, vp, vp, vp, vp, sz, vp]
    L.grpo_loss_fwd_bwd_noalloc.restype = i32
    L.grpo_loss_fwd_bwd_noalloc.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, vp, f32, f32, f32, f32,
                                            f64, f32, vp, vp, vp, vp, vp, vp]
    L.grpo_loss_aux_fwd_bwd.restype = i32
    L.grpo_loss_aux_fwd_bwd.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, vp, vp, vp, f32, f32, f32,
                                        f32, f32, f32, f64, f32, vp, vp, vp, vp, vp, vp, sz, vp]
    L.grpo_total_rewards.restype = i32
    L.grpo_total_rewards.argtypes = [vp, vp, vp, i64, f32, vp, vp]
    L.grpo_filter_groups.restype = i32
    L.grpo_filter_groups.argtypes = [vp, i64, vp, i64, i64, vp, vp, vp, vp, vp]
    L.grpo_packed_layout.restype = i32
    L.grpo_packed_layout.argtypes = [vp, i64, i64, i32, vp, vp, vp]
    L.grpo_workspace_error.restype = i32
    L.grpo_workspace_error.argtypes = [vp, vp, vp]
    L.grpo_lmhead_workspace_bytes.restype = sz
    L.grpo_lmhead_workspace_bytes.argtypes = [i64, i64, i64, i32]
    L.grpo_lmhead_workspace_bytes_for_chunk.restype = sz
    L.grpo_lmhead_workspace_bytes_for_chunk.argtypes = [i64, i64, i64, i64]
    L.grpo_lmhead_logprobs_fwd.restype = i32
    L.grpo_lmhead_logprobs_fwd.argtypes = [vp, i64, vp, i64, i64, i64, i64, vp, vp, f32, vp, vp, sz, vp]
    L.grpo_lmhead_loss_fwd_bwd.restype = i32
    L.grpo_lmhead_loss_fwd_bwd.argtypes = [vp, i64, vp, i64, i64, i64, i64, vp, vp, vp, vp, f32, f32,
                                           f32, f32, f64, f32, vp, vp, vp, vp, i64, vp, i64, i32,
                                           vp, sz, vp]
    L.grpo_lmhead_loss_aux_fwd_bwd.restype = i32
    L.grpo_lmhead_loss_aux_fwd_bwd.argtypes = [vp, i64, vp, i64, i64, i64, i64, vp, vp, vp, vp, vp, vp,
                                               f32, f32, f32, f32, f32, f32, f64, f32, vp, vp, vp, vp,
                                               vp, i64, vp, i64, i32, vp, sz, vp]
    L.grpo_verify_workspace_bytes.restype = sz
    L.grpo_verify_workspace_bytes.argtypes = [i64, i64, i64, i32]
    L.grpo_verify_drafts.restype = i32
    L.grpo_verify_drafts.argtypes = [vp, i64, i64, vp, i64, i64, i32, i64, i64, i64, vp, vp, vp, vp, f64, f64, vp, vp, vp, vp, sz, vp]
    L.grpo_block_norm_fwd.restype = i32
    L.grpo_block_norm_fwd.argtypes = [vp, i64, i32, vp, i64, vp, vp, i64, vp, i32, i64, i64, f64, f64, vp, i64, vp, i64, vp]
    L.grpo_block_norm_workspace_bytes.restype = sz
    L.grpo_block_norm_workspace_bytes.argtypes = [i64, i64]
    L.grpo_block_norm_bwd.restype = i32
    L.grpo_block_norm_bwd.argtypes = [vp, i64, i32, vp, i64, vp, vp, i64, vp, i32, i64, i64, f64, f64, vp, i64, vp, i64, vp, i64,
                                      vp, i64, vp, i64, vp, vp, i32, vp, sz, vp]
    L.grpo_optim_plan_bytes.restype = sz
    L.grpo_optim_plan_bytes.argtypes = [ctypes.POINTER(_OptimTensor), i64]
    L.grpo_optim_plan_build.restype = i32
    L.grpo_optim_plan_build.argtypes = [ctypes.POINTER(_OptimTensor), i64, vp, sz, ctypes.POINTER(_OptimPlan)]
    L.grpo_grad_norm_workspace_bytes.restype = sz
    L.grpo_grad_norm_workspace_bytes.argtypes = []
    L.grpo_grad_norm.restype = i32
    L.grpo_grad_norm.argtypes = [vp, vp, f64, vp, vp, sz, vp]
    L.grpo_adamw_step.restype = i32
    L.grpo_adamw_step.argtypes = [vp, vp, i64, vp, f64, vp, f64, f64, f64, vp, vp]
    fast = _load_fastcall()
    if fast is not None:
        fast.bind(*[ctypes.cast(f, vp).value for f in (
            L.grpo_workspace_bytes, L.grpo_group_advantages, L.grpo_logprobs_fwd, L.grpo_loss_fwd_bwd,
            L.grpo_loss_aux_fwd_bwd, L.grpo_total_rewards, L.grpo_filter_groups, L.grpo_packed_layout)])
        fast.bind_operators(*[ctypes.cast(f, vp).value for f in (
            L.grpo_verify_workspace_bytes, L.grpo_verify_drafts, L.grpo_block_norm_workspace_bytes, L.grpo_block_norm_fwd,
            L.grpo_block_norm_bwd, L.grpo_grad_norm_workspace_bytes, L.grpo_grad_norm, L.grpo_adamw_step)])
        _fast = fast
    _lib = L


def _fast_result(out, where):
    """What a function of _fastcall has returned: the outputs, or the status of a call the library refused."""
    if type(out) is int:
        raise GrpoError(out, where)
    return out


def status_string(status) -> str:
    return lib().grpo_status_string(int(status)).decode()


def grpo_workspace_bytes(n_tokens: int) -> int:
    return int(lib().grpo_workspace_bytes(int(n_tokens)))


class _OptimTensor(ctypes.Structure):
    """grpo_optim_tensor of grpo.h."""
    _fields_ = [(name, ctypes.c_void_p) for name in ("param", "master", "grad", "exp_avg", "exp_avg_sq", "exp_avg_scale",
                                                     "exp_avg_sq_scale")] + \
               [("n", ctypes.c_int64), ("weight_decay", ctypes.c_double), ("param_dtype", ctypes.c_int32),
                ("grad_dtype", ctypes.c_int32), ("state_bits", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class _OptimPlan(ctypes.Structure):
    """grpo_optim_plan of grpo.h."""
    _fields_ = [("n_tensors", ctypes.c_int64), ("n_chunks", ctypes.c_int64), ("has_params", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class RowPlan(ctypes.Structure):
    """grpo_row_plan of grpo.h."""
    _fields_ = [("vectors", ctypes.c_int64), ("resident_vectors", ctypes.c_int64), ("streaming", ctypes.c_int32),
                ("lanes", ctypes.c_int32), ("register_slots", ctypes.c_int32), ("lds_slots", ctypes.c_int32),
                ("workgroups_per_cu", ctypes.c_int32), ("ragged_tail_slot", ctypes.c_int32),
                ("streamed_remainder", ctypes.c_int32), ("reserved", ctypes.c_int32)]


def grpo_row_kernel_plan(dtype: int, vocab: int) -> dict:
    """Which row kernel serves rows of this width; see grpo_row_kernel_plan in grpo.h."""
    plan = RowPlan()
    rc = lib().grpo_row_kernel_plan(int(dtype), int(vocab), ctypes.byref(plan))
    if rc != 0:
        raise GrpoError(rc, "grpo_row_kernel_plan")
    return {name: int(getattr(plan, name)) for name, _ in RowPlan._fields_ if name != "reserved"}


def _ptr(t):
    return None if t is None else t.data_ptr()


def _raw_stream(stream, device_index=None):
    """The hipStream_t of `stream`, or of the current stream (of the given or the current device).  The current
    one is asked for as a number: making torch's Stream object around it takes 2.6 us, a third of what a
    small call spends on the host."""
    if stream is not None:
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if device_index is None else device_index)




def _check(t, dtype, n, name, device):
    if t.dtype != dtype or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of length %d" % (name, dtype, n))
    if t.device != device:
        raise ValueError("%s must live on %s" % (name, device))


def _logits_args(logits, vocab):
    if logits.dim() != 2 or logits.stride(1) != 1:
        raise ValueError("logits must be [n_tokens, vocab] with unit stride along the vocabulary")
    if not logits.is_cuda:
        raise ValueError("logits must be a device tensor: libgrpo has no CPU path")
    if logits.dtype == torch.bfloat16:
        dt = GRPO_BF16
    elif logits.dtype == torch.float32:
        dt = GRPO_F32
    else:
        raise ValueError("logits must be bfloat16 or float32")
    n = logits.shape[0]
    v = logits.shape[1] if vocab is None else int(vocab)
    stride = logits.stride(0) if n > 1 else max(logits.stride(0), v)
    return dt, n, v, stride


def grpo_group_advantages(rewards, group_size=None, group_offsets=None, eps_std=1e-6, ddof=0,
                          rollout_of_token=None, adv_out=None, adv_tok_out=None, stream=None):
    """Returns (adv [n_rollouts], adv_tok [n_tokens] or None); see grpo_group_advantages in grpo.h."""
    if group_offsets is None and adv_out is None and adv_tok_out is None and stream is None:
        out = _fast.group_advantages(rewards, group_size, eps_std, ddof, rollout_of_token)
        if out is not None:
            return _fast_result(out, "grpo_group_advantages")
    dev = rewards.device
    R = rewards.shape[0]
    _check(rewards, torch.float32, R, "rewards", dev)
    if group_offsets is not None:
        _check(group_offsets, torch.int32, group_offsets.shape[0], "group_offsets", dev)
        n_groups, gs = group_offsets.shape[0] - 1, 0
    else:
        gs = int(group_size)
        n_groups = R // gs if gs > 0 else 0
    if adv_out is None:
        adv_out = torch.empty(R, dtype=torch.float32, device=dev)
    n_tok = 0
    if rollout_of_token is not None:
        n_tok = rollout_of_token.shape[0]
        _check(rollout_of_token, torch.int32, n_tok, "rollout_of_token", dev)
        if adv_tok_out is None:
            adv_tok_out = torch.empty(n_tok, dtype=torch.float32, device=dev)
    rc = lib().grpo_group_advantages(_ptr(rewards), R, _ptr(group_offsets), n_groups, gs,
                                     float(eps_std), int(ddof), _ptr(adv_out),
                                     _ptr(rollout_of_token), n_tok, _ptr(adv_tok_out),
                                     _raw_stream(stream))
    if rc != GRPO_OK:
        raise GrpoError(rc, "grpo_group_advantages")
    return adv_out, adv_tok_out


_queue_workspaces = {}


def _queue_workspace(device, stream):
    """The small workspace grpo_logprobs_fwd's row queue lives in, one per device and stream, made
    on first use and kept: calls on one stream run one after the other, so they can share it, and
    the call does not allocate again (calls on different streams may overlap and must not)."""
    index = device.index if device.index is not None else torch.cuda.current_device()
    key = (index, _raw_stream(stream, index))
    ws = _queue_workspaces.get(key)
    if ws is None:
        ws = torch.empty(grpo_workspace_bytes(0), dtype=torch.uint8, device=device)
        if not torch.cuda.is_current_stream_capturing():   # memory made under capture belongs to that graph
            _queue_workspaces[key] = ws
    return ws


def grpo_logprobs_fwd(logits, tokens, mask=None, temperature=1.0, vocab=None, logprobs_out=None,
                      workspace=None, use_queue=True, stream=None):
    """log softmax(logits / T)[tokens] per row; see grpo_logprobs_fwd in grpo.h.
    Unless a workspace is passed or ``use_queue`` is False, the row queue uses a small
    workspace this module keeps per device and stream."""
    if vocab is None and logprobs_out is None and stream is None and use_queue and logits.is_cuda and logits.dim() == 2 and \
            logits.shape[0] > 0:
        out = _fast.logprobs_fwd(logits, tokens, mask, temperature,
                                 _queue_workspace(logits.device, None) if workspace is None else workspace)
        if out is not None:
            return _fast_result(out, "grpo_logprobs_fwd")
    dt, n, v, stride = _logits_args(logits, vocab)
    dev = logits.device
    _check(tokens, torch.int64, n, "tokens", dev)
    if mask is not None:
        _check(mask, torch.uint8, n, "mask", dev)
    if logprobs_out is None:
        logprobs_out = torch.empty(n, dtype=torch.float32, device=dev)
    if workspace is None and use_queue and n > 0:
        workspace = _queue_workspace(dev, stream)
    rc = lib().grpo_logprobs_fwd(_ptr(logits), dt, n, v, stride, _ptr(tokens), _ptr(mask),
                                 float(temperature), _ptr(logprobs_out), _ptr(workspace),
                                 0 if workspace is None else workspace.numel(), _raw_stream(stream))
    if rc != GRPO_OK:
        raise GrpoError(rc, "grpo_logprobs_fwd")
    return logprobs_out


def grpo_loss_fwd_bwd(logits, tokens, old_logprobs, advantages, mask=None, eps_low=0.2,
                      eps_high=0.2, delta=4.0, temperature=1.0, denom=0.0, grad_scale=1.0, *,
                      vocab=None, grad_logits=None, inplace=False, loss_out=None,
                      logprobs_out=None, counts_out=None, workspace=None, stream=None):
    """Objective forward + fused backward; see grpo_loss_fwd_bwd in grpo.h.

    Returns (loss [1] f32, logprobs [n] f32, counts [5] i64, grad_logits), all on the device and
    valid once the stream has run.  ``inplace=True`` writes the gradient over the logits.
    """
    if vocab is None and loss_out is None and logprobs_out is None and counts_out is None and stream is None:
        out = _fast.loss_fwd_bwd(logits, tokens, old_logprobs, advantages, mask, eps_low, eps_high, delta, temperature, denom,
                                 grad_scale, logits if inplace else grad_logits, workspace)
        if out is not None:
            return _fast_result(out, "grpo_loss_fwd_bwd")
    dt, n, v, stride = _logits_args(logits, vocab)
    dev = logits.device
    _check(tokens, torch.int64, n, "tokens", dev)
    _check(old_logprobs, torch.float32, n, "old_logprobs", dev)
    _check(advantages, torch.float32, n, "advantages", dev)
    if mask is not None:
        _check(mask, torch.uint8, n, "mask", dev)
    if inplace:
        grad_logits = logits
    elif grad_logits is None:
        grad_logits = torch.empty_strided(logits.shape, logits.stride(), dtype=logits.dtype, device=dev)
    elif grad_logits.dtype != logits.dtype or grad_logits.shape != logits.shape or \
            grad_logits.stride() != logits.stride():
        raise ValueError("grad_logits must match logits in dtype, shape and strides")
    if loss_out is None:
        loss_out = torch.empty(1, dtype=torch.float32, device=dev)
    if logprobs_out is None:
        logprobs_out = torch.empty(n, dtype=torch.float32, device=dev)
    if counts_out is None:
        counts_out = torch.empty(5, dtype=torch.int64, device=dev)
    need = grpo_workspace_bytes(n)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    rc = lib().grpo_loss_fwd_bwd(_ptr(logits), dt, n, v, stride, _ptr(tokens), _ptr(old_logprobs),
                                 _ptr(advantages), _ptr(mask), float(eps_low), float(eps_high),
                                 float(delta), float(temperature), float(denom), float(grad_scale),
                                 _ptr(loss_out), _ptr(logprobs_out), _ptr(counts_out),
                                 _ptr(grad_logits), _ptr(workspace), workspace.numel(),
                                 _raw_stream(stream))
    if rc != GRPO_OK:
        raise GrpoError(rc, "grpo_loss_fwd_bwd")
    return loss_out, logprobs_out, counts_out, grad_logits


NOALLOC_MAX_TOKENS = 524288  # GRPO_NOALLOC_MAX_TOKENS of grpo.h


def grpo_loss_fwd_bwd_noalloc(logits, tokens, old_logprobs, advantages, mask, eps_low, eps_high, delta,
                              temperature, denom, grad_scale, *, grad_logits, loss_out, logprobs_out=None,
                              counts_out=None, error_out=None, vocab=None, stream=None):
    """grpo_loss_fwd_bwd without a workspace; see grpo_loss_fwd_bwd_noalloc in grpo.h.  This wrapper
    allocates nothing either: every output tensor is the caller's (grad_logits may be the logits
    tensor itself).  Returns None; results are in the tensors passed."""
    dt, n, v, stride = _logits_args(logits, vocab)
    dev = logits.device
    _check(tokens, torch.int64, n, "tokens", dev)
    _check(old_logprobs, torch.float32, n, "old_logprobs", dev)
    _check(advantages, torch.float32, n, "advantages", dev)
    if mask is not None:
        _check(mask, torch.uint8, n, "mask", dev)
    if grad_logits.dtype != logits.dtype or grad_logits.shape != logits.shape or \
            grad_logits.stride() != logits.stride():
        raise ValueError("grad_logits must match logits in dtype, shape and strides")
    _check(loss_out, torch.float32, 1, "loss_out", dev)
    if logprobs_out is not None:
        _check(logprobs_out, torch.float32, n, "logprobs_out", dev)
    if counts_out is not None:
        _check(counts_out, torch.int64, 5, "counts_out", dev)
    if error_out is not None:
        _check(error_out, torch.int32, 1, "error_out", dev)
    rc = lib().grpo_loss_fwd_bwd_noalloc(_ptr(logits), dt, n, v, stride, _ptr(tokens), _ptr(old_logprobs),
                                         _ptr(advantages), _ptr(mask), float(eps_low), float(eps_high),
                                         float(delta), float(temperature), float(denom), float(grad_scale),
                                         _ptr(loss_out), _ptr(logprobs_out), _ptr(counts_out),
                                         _ptr(grad_logits), _ptr(error_out), _raw_stream(stream))
    if rc != GRPO_OK:
        raise GrpoError(rc, "grpo_loss_fwd_bwd_noalloc")


def grpo_loss_aux_fwd_bwd(logits, tokens, old_logprobs, ref_logprobs, advantages, mask=None,
                          eps_low=0.2, eps_high=0.2, delta=4.0, temperature=1.0, kl_coef=0.0,
                          entropy_coef=0.0, denom=0.0, grad_scale=1.0, *, token_weights=None,
                          vocab=None, grad_logits=None, inplace=False, loss_out=None, logprobs_out=None,
                          entropy_out=None, want_entropy=True, counts_out=None, workspace=None,
                          stream=None):
    """Objective with the KL and entropy terms fused in; see grpo_loss_aux_fwd_bwd in grpo.h.

    Returns (loss [4] f32: total, policy, mean kl, mean entropy; logprobs [n]; entropy [n] or
    None; counts [5] i64; grad_logits)."""
    if vocab is None and loss_out is None and logprobs_out is None and entropy_out is None and \
            counts_out is None and stream is None:
        out = _fast.loss_aux_fwd_bwd(logits, tokens, old_logprobs, ref_logprobs, advantages, mask, token_weights, eps_low,
                                     eps_high, delta, temperature, kl_coef, entropy_coef, denom, grad_scale,
                                     logits if inplace else grad_logits, workspace, want_entropy)
        if out is not None:
            return _fast_result(out, "grpo_loss_aux_fwd_bwd")
    dt, n, v, stride = _logits_args(logits, vocab)
    dev = logits.device
    _check(tokens, torch.int64, n, "tokens", dev)
    _check(old_logprobs, torch.float32, n, "old_logprobs", dev)
    _check(advantages, torch.float32, n, "advantages", dev)
    if ref_logprobs is not None:
        _check(ref_logprobs, torch.float32, n, "ref_logprobs", dev)
    if token_weights is not None:
        _check(token_weights, torch.float32, n, "token_weights", dev)
    if mask is not None:
        _check(mask, torch.uint8, n, "mask", dev)
    if inplace:
        grad_logits = logits
    elif grad_logits is None:
        grad_logits = torch.empty_strided(logits.shape, logits.stride(), dtype=logits.dtype, device=dev)
    elif grad_logits.dtype != logits.dtype or grad_logits.shape != logits.shape or \
            grad_logits.stride() != logits.stride():
        raise ValueError("grad_logits must match logits in dtype, shape and strides")
    if loss_out is None:
        loss_out = torch.empty(4, dtype=torch.float32, device=dev)
    if logprobs_out is None:
        logprobs_out = torch.empty(n, dtype=torch.float32, device=dev)
    if entropy_out is None and want_entropy:
        entropy_out = torch.empty(n, dtype=torch.float32, device=dev)
    if counts_out is None:
        counts_out = torch.empty(5, dtype=torch.int64, device=dev)
    if workspace is None:
        workspace = torch.empty(grpo_workspace_bytes(n), dtype=torch.uint8, device=dev)
    rc = lib().grpo_loss_aux_fwd_bwd(
        _ptr(logits), dt, n, v, stride, _ptr(tokens), _ptr(old_logprobs), _ptr(ref_logprobs),
        _ptr(advantages), _ptr(mask), _ptr(token_weights), float(eps_low), float(eps_high),
        float(delta), float(temperature), float(kl_coef), float(entropy_coef), float(denom),
        float(grad_scale),
        _ptr(loss_out), _ptr(logprobs_out), _ptr(entropy_out), _ptr(counts_out), _ptr(grad_logits),
        _ptr(workspace), workspace.numel(), _raw_stream(stream))
    if rc != GRPO_OK:
        raise GrpoError(rc, "grpo_loss_aux_fwd_bwd")
    return loss_out, logprobs_out, entropy_out, counts_out, grad_logits


def grpo_total_rewards(task_rewards, lengths, target_lengths, alpha, rewards_out=None, stream=None):
    """r_task - alpha |l_target - l_y| per rollout; see grpo_total_rewards in grpo.h."""
    if rewards_out is None and stream is None:
        out = _fast.total_rewards(task_rewards, lengths, target_lengths, alpha)
        if out is not None:
            return _fast_result(out, "grpo_total_rewards")
    dev = task_rewards.device
    R = task_rewards.shape[0]
    _check(task_rewards, torch.float32, R, "task_rewards", dev)
    _check(lengths, torch.int32, R, "lengths", dev)
    _check(target_lengths, torch.int32, R, "target_lengths", dev)
    if rewards_out is None:
        rewards_out = torch.empty(R, dtype=torch.float32, device=dev)
    rc = lib().grpo_total_rewards(_ptr(task_rewards), _ptr(lengths), _ptr(target_lengths), R,
                                  float(alpha), _ptr(rewards_out), _raw_stream(stream))
    if rc != GRPO_OK:
        raise GrpoError(rc, "grpo_total_rewards")
    return rewards_out


def grpo_filter_groups(rewards, group_size=None, group_offsets=None, stream=None):
    """Returns (keep u8 [n_groups], kept_groups i32 [n_groups], n_kept i32 [1], rollout_keep u8 [R]);
    see grpo_filter_groups in grpo.h."""
    if group_offsets is None and stream is None:
        out = _fast.filter_groups(rewards, group_size)
        if out is not None:
            return _fast_result(out, "grpo_filter_groups")
    dev = rewards.device
    R = rewards.shape[0]
    _check(rewards, torch.float32, R, "rewards", dev)
    if group_offsets is not None:
        _check(group_offsets, torch.int32, group_offsets.shape[0], "group_offsets", dev)
        n_groups, gs = group_offsets.shape[0] - 1, 0
    else:
        gs = int(group_size)
        n_groups = R // gs if gs > 0 else 0
    keep = torch.empty(n_groups, dtype=torch.uint8, device=dev)
    kept = torch.empty(n_groups, dtype=torch.int32, device=dev)
    n_kept = torch.empty(1, dtype=torch.int32, device=dev)
    # groups of one size own every rollout (the library refuses sizes that leave some over) unless there is
    # no group at all; with offsets some rollouts may belong to none: such a rollout keeps its 0
    owned = group_offsets is None and n_groups > 0
    rk = (torch.empty if owned else torch.zeros)(R, dtype=torch.uint8, device=dev)
    rc = lib().grpo_filter_groups(_ptr(rewards), R, _ptr(group_offsets), n_groups, gs, _ptr(keep),
                                  _ptr(kept), _ptr(n_kept), _ptr(rk), _raw_stream(stream))
    if rc != GRPO_OK:
        raise GrpoError(rc, "grpo_filter_groups")
    return keep, kept, n_kept, rk


def grpo_packed_layout(cu_seqlens, n_tokens, sample_level, weights_out=None, rollout_of_token_out=None,
                       stream=None):
    """(weights f32 [n_tokens], rollout_of_token i32 [n_tokens]) of a packed batch whose rollout i
    owns rows [cu_seqlens[i], cu_seqlens[i+1]); see grpo_packed_layout in grpo.h."""
    if weights_out is None and rollout_of_token_out is None and stream is None:
        out = _fast.packed_layout(cu_seqlens, n_tokens, sample_level)
        if out is not None:
            return _fast_result(out, "grpo_packed_layout")
    dev = cu_seqlens.device
    _check(cu_seqlens, torch.int64, cu_seqlens.shape[0], "cu_seqlens", dev)
    if weights_out is None:
        weights_out = torch.empty(n_tokens, dtype=torch.float32, device=dev)
    if rollout_of_token_out is None:
        rollout_of_token_out = torch.empty(n_tokens, dtype=torch.int32, device=dev)
    rc = lib().grpo_packed_layout(_ptr(cu_seqlens), cu_seqlens.shape[0] - 1, int(n_tokens),
                                  1 if sample_level else 0, _ptr(weights_out),
                                  _ptr(rollout_of_token_out), _raw_stream(stream))
    if rc != GRPO_OK:
        raise GrpoError(rc, "grpo_packed_layout")
    return weights_out, rollout_of_token_out


def grpo_workspace_error(workspace, stream=None) -> int:
    flag = ctypes.c_int32(0)
    rc = lib().grpo_workspace_error(_ptr(workspace), ctypes.byref(flag), _raw_stream(stream))
    if rc != GRPO_OK:
        raise GrpoError(rc, "grpo_workspace_error")
    return int(flag.value)


def grpo_lmhead_workspace_bytes(n_tokens: int, vocab: int, d_model: int, with_backward: bool) -> int:
    return int(lib().grpo_lmhead_workspace_bytes(int(n_tokens), int(vocab), int(d_model),
                                                 1 if with_backward else 0))


def grpo_lmhead_workspace_bytes_for_chunk(n_tokens: int, vocab: int, d_model: int, chunk_rows: int) -> int:
    """Workspace of the backward when it works through the rows in chunks of ``chunk_rows``."""
    return int(lib().grpo_lmhead_workspace_bytes_for_chunk(int(n_tokens), int(vocab), int(d_model),
                                                           int(chunk_rows)))


def _lmhead_args(hidden, weight):
    for name, t in (("hidden", hidden), ("weight", weight)):
        if t.dim() != 2 or t.stride(1) != 1 or t.dtype != torch.bfloat16 or not t.is_cuda:
            raise ValueError("%s must be a 2-D bfloat16 device tensor with unit stride along d_model" % name)
    n, d = hidden.shape
    v = weight.shape[0]
    if weight.shape[1] != d:
        raise ValueError("hidden is [n_tokens, d_model] and weight [vocab, d_model]: d_model differs")
    hs = hidden.stride(0) if n > 1 else max(hidden.stride(0), d)
    ws = weight.stride(0) if v > 1 else max(weight.stride(0), d)
    return n, v, d, hs, ws


def grpo_lmhead_logprobs_fwd(hidden, weight, tokens, mask=None, temperature=1.0, logprobs_out=None,
                             workspace=None, stream=None):
    """log softmax(hidden @ weight.T / T)[tokens] per row without materialising the logits; see
    grpo_lmhead_logprobs_fwd in grpo.h."""
    n, v, d, hs, ws = _lmhead_args(hidden, weight)
    dev = hidden.device
    _check(tokens, torch.int64, n, "tokens", dev)
    if mask is not None:
        _check(mask, torch.uint8, n, "mask", dev)
    if logprobs_out is None:
        logprobs_out = torch.empty(n, dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = torch.empty(grpo_lmhead_workspace_bytes(n, v, d, False), dtype=torch.uint8, device=dev)
    rc = lib().grpo_lmhead_logprobs_fwd(_ptr(hidden), hs, _ptr(weight), ws, n, v, d, _ptr(tokens),
                                        _ptr(mask), float(temperature), _ptr(logprobs_out),
                                        _ptr(workspace), workspace.numel(), _raw_stream(stream))
    if rc != GRPO_OK:
        raise GrpoError(rc, "grpo_lmhead_logprobs_fwd")
    return logprobs_out


def grpo_lmhead_loss_fwd_bwd(hidden, weight, tokens, old_logprobs, advantages, mask=None, eps_low=0.2,
                             eps_high=0.2, delta=4.0, temperature=1.0, denom=0.0, grad_scale=1.0, *,
                             grad_hidden=None, grad_weight=None, accumulate_grad_weight=False,
                             loss_out=None, logprobs_out=None, counts_out=None, workspace=None,
                             stream=None):
    """Objective on hidden @ weight.T with gradients for both operands; see
    grpo_lmhead_loss_fwd_bwd in grpo.h.  Returns (loss [1], logprobs [n], counts [5],
    grad_hidden bf16 [n, d], grad_weight f32 [vocab, d])."""
    n, v, d, hs, ws = _lmhead_args(hidden, weight)
    dev = hidden.device
    _check(tokens, torch.int64, n, "tokens", dev)
    _check(old_logprobs, torch.float32, n, "old_logprobs", dev)
    _check(advantages, torch.float32, n, "advantages", dev)
    if mask is not None:
        _check(mask, torch.uint8, n, "mask", dev)
    if grad_hidden is None:
        grad_hidden = torch.empty((n, d), dtype=torch.bfloat16, device=dev)
    if grad_weight is None:
        if accumulate_grad_weight:
            raise ValueError("accumulate_grad_weight needs the grad_weight tensor to add to")
        grad_weight = torch.empty((v, d), dtype=torch.float32, device=dev)
    if grad_hidden.dtype != torch.bfloat16 or grad_hidden.shape != (n, d) or grad_hidden.stride(1) != 1:
        raise ValueError("grad_hidden must be bfloat16 [n_tokens, d_model] with unit inner stride")
    if grad_weight.dtype != torch.float32 or grad_weight.shape != (v, d) or grad_weight.stride(1) != 1:
        raise ValueError("grad_weight must be float32 [vocab, d_model] with unit inner stride")
    if loss_out is None:
        loss_out = torch.empty(1, dtype=torch.float32, device=dev)
    if logprobs_out is None:
        logprobs_out = torch.empty(n, dtype=torch.float32, device=dev)
    if counts_out is None:
        counts_out = torch.empty(5, dtype=torch.int64, device=dev)
    if workspace is None:
        workspace = torch.empty(grpo_lmhead_workspace_bytes(n, v, d, True), dtype=torch.uint8, device=dev)
    ghs = grad_hidden.stride(0) if n > 1 else max(grad_hidden.stride(0), d)
    gws = grad_weight.stride(0) if v > 1 else max(grad_weight.stride(0), d)
    rc = lib().grpo_lmhead_loss_fwd_bwd(
        _ptr(hidden), hs, _ptr(weight), ws, n, v, d, _ptr(tokens), _ptr(old_logprobs), _ptr(advantages),
        _ptr(mask), float(eps_low), float(eps_high), float(delta), float(temperature), float(denom),
        float(grad_scale), _ptr(loss_out), _ptr(logprobs_out), _ptr(counts_out), _ptr(grad_hidden), ghs,
        _ptr(grad_weight), gws, 1 if accumulate_grad_weight else 0, _ptr(workspace), workspace.numel(),
        _raw_stream(stream))
    if rc != GRPO_OK:
        raise GrpoError(rc, "grpo_lmhead_loss_fwd_bwd")
    return loss_out, logprobs_out, counts_out, grad_hidden, grad_weight


def grpo_lmhead_loss_aux_fwd_bwd(hidden, weight, tokens, old_logprobs, ref_logprobs, advantages, mask=None,
                                 eps_low=0.2, eps_high=0.2, delta=4.0, temperature=1.0, kl_coef=0.0,
                                 entropy_coef=0.0, denom=0.0, grad_scale=1.0, *, token_weights=None,
                                 grad_hidden=None, grad_weight=None, accumulate_grad_weight=False,
                                 loss_out=None, logprobs_out=None, entropy_out=None, want_entropy=True,
                                 counts_out=None, workspace=None, stream=None):
    """Total objective (policy + KL - entropy bonus, per-token weights) on hidden @ weight.T with
    gradients for both operands; see grpo_lmhead_loss_aux_fwd_bwd in grpo.h.  Returns (loss [4]:
    total, policy, mean kl, mean entropy; logprobs [n]; entropy [n] or None; counts [5];
    grad_hidden bf16 [n, d]; grad_weight f32 [vocab, d])."""
    n, v, d, hs, ws = _lmhead_args(hidden, weight)
    dev = hidden.device
    _check(tokens, torch.int64, n, "tokens", dev)
    _check(old_logprobs, torch.float32, n, "old_logprobs", dev)
    _check(advantages, torch.float32, n, "advantages", dev)
    if ref_logprobs is not None:
        _check(ref_logprobs, torch.float32, n, "ref_logprobs", dev)
    if token_weights is not None:
        _check(token_weights, torch.float32, n, "token_weights", dev)
    if mask is not None:
        _check(mask, torch.uint8, n, "mask", dev)
    if grad_hidden is None:
        grad_hidden = torch.empty((n, d), dtype=torch.bfloat16, device=dev)
    if grad_weight is None:
        if accumulate_grad_weight:
            raise ValueError("accumulate_grad_weight needs the grad_weight tensor to add to")
        grad_weight = torch.empty((v, d), dtype=torch.float32, device=dev)
    if grad_hidden.dtype != torch.bfloat16 or grad_hidden.shape != (n, d) or grad_hidden.stride(1) != 1:
        raise ValueError("grad_hidden must be bfloat16 [n_tokens, d_model] with unit inner stride")
    if grad_weight.dtype != torch.float32 or grad_weight.shape != (v, d) or grad_weight.stride(1) != 1:
        raise ValueError("grad_weight must be float32 [vocab, d_model] with unit inner stride")
    if loss_out is None:
        loss_out = torch.empty(4, dtype=torch.float32, device=dev)
    if logprobs_out is None:
        logprobs_out = torch.empty(n, dtype=torch.float32, device=dev)
    if entropy_out is None and want_entropy:
        entropy_out = torch.empty(n, dtype=torch.float32, device=dev)
    if counts_out is None:
        counts_out = torch.empty(5, dtype=torch.int64, device=dev)
    if workspace is None:
        workspace = torch.empty(grpo_lmhead_workspace_bytes(n, v, d, True), dtype=torch.uint8, device=dev)
    ghs = grad_hidden.stride(0) if n > 1 else max(grad_hidden.stride(0), d)
    gws = grad_weight.stride(0) if v > 1 else max(grad_weight.stride(0), d)
    rc = lib().grpo_lmhead_loss_aux_fwd_bwd(
        _ptr(hidden), hs, _ptr(weight), ws, n, v, d, _ptr(tokens), _ptr(old_logprobs), _ptr(ref_logprobs),
        _ptr(advantages), _ptr(mask), _ptr(token_weights), float(eps_low), float(eps_high), float(delta),
        float(temperature), float(kl_coef), float(entropy_coef), float(denom), float(grad_scale),
        _ptr(loss_out), _ptr(logprobs_out), _ptr(entropy_out), _ptr(counts_out), _ptr(grad_hidden), ghs,
        _ptr(grad_weight), gws, 1 if accumulate_grad_weight else 0, _ptr(workspace), workspace.numel(),
        _raw_stream(stream))
    if rc != GRPO_OK:
        raise GrpoError(rc, "grpo_lmhead_loss_aux_fwd_bwd")
    return loss_out, logprobs_out, entropy_out, counts_out, grad_hidden, grad_weight


def _own_workspace(size, device, stream):
    """A workspace of a call's own.  On a stream that is given it may be freed, and the memory used again, before the call has run."""
    workspace = torch.empty(size, dtype=torch.uint8, device=device)
    if stream is not None:
        workspace.record_stream(stream)
    return workspace


def _call(where, device, f, *args):
    """Calls the library on a tensor's device, whichever is the current one."""
    if device.index == torch.cuda.current_device():
        rc = f(*args)
    else:
        with torch.cuda.device(device):
            rc = f(*args)
    if rc != GRPO_OK:
        raise GrpoError(rc, where)


def _verify_logits(t, name, batch, rows, vocab, dtype, device):
    """The strides of responses and of rows of [batch, rows, vocab] logits, in elements."""
    if t.dim() != 3 or t.dtype != dtype or tuple(t.shape) != (batch, rows, vocab) or (t.stride(2) != 1 and vocab > 1):
        raise ValueError("%s must be a %s tensor [%d, %d, %d] with unit stride along the vocabulary" % (name, dtype, batch, rows, vocab))
    if t.device != device:
        raise ValueError("%s must live on %s" % (name, device))
    # a stride that nothing is behind can be anything
    per16 = 8 if dtype == torch.bfloat16 else 4
    return (t.stride(0) if batch > 1 else 0), (t.stride(1) if rows > 1 else (vocab + per16 - 1) // per16 * per16)


def _check_2d(t, dtype, shape, name, device):
    if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor %s" % (name, dtype, list(shape)))
    if t.device != device:
        raise ValueError("%s must live on %s" % (name, device))


def grpo_verify_drafts(target_logits, draft_logits, draft_tokens, accept_u, sample_u, draft_lengths=None, temperature=1.0,
                       draft_temperature=1.0, *, tokens_out=None, n_accepted_out=None, logprobs_out=None, workspace=None, stream=None):
    """Verifies drafted tokens and samples the one behind them; see grpo_verify_drafts in grpo.h.

    target_logits [batch, drafts + 1, vocab] bf16 or f32; draft_logits [batch, drafts, vocab] of the same dtype, or None for
    tokens that no model drafted; draft_tokens [batch, drafts] i64 and accept_u [batch, drafts] f32 (either may be None without
    drafts); sample_u [batch] f64; draft_lengths [batch] i32 or None.  Returns (tokens [batch, drafts + 1] i64,
    n_accepted [batch] i32, logprobs [batch, drafts + 1] f32)."""
    if tokens_out is None and n_accepted_out is None and logprobs_out is None and workspace is None and stream is None:
        out = _fast.verify_drafts(target_logits, draft_logits, draft_tokens, accept_u, sample_u, draft_lengths, temperature, draft_temperature)
        if out is not None:
            return _fast_result(out, "grpo_verify_drafts")
    if not target_logits.is_cuda:
        raise ValueError("target_logits must be a device tensor: libgrpo has no CPU path")
    if target_logits.dim() != 3 or target_logits.dtype not in _DTYPE_CODES or target_logits.shape[1] < 1:
        raise ValueError("target_logits must be a bfloat16 or float32 tensor [batch, drafts + 1, vocab]")
    dev, dtype = target_logits.device, target_logits.dtype
    n, k, v = target_logits.shape[0], target_logits.shape[1] - 1, target_logits.shape[2]
    tb, tk = _verify_logits(target_logits, "target_logits", n, k + 1, v, dtype, dev)
    db = dk = 0
    if k == 0:
        draft_logits = None
    if draft_logits is not None:
        db, dk = _verify_logits(draft_logits, "draft_logits", n, k, v, dtype, dev)
    for t, dt, name in ((draft_tokens, torch.int64, "draft_tokens"), (accept_u, torch.float32, "accept_u")):
        if t is not None:
            _check_2d(t, dt, (n, k), name, dev)
        elif k > 0:
            raise ValueError("%s is needed where there are drafts" % name)
    _check(sample_u, torch.float64, n, "sample_u", dev)
    if draft_lengths is not None:
        _check(draft_lengths, torch.int32, n, "draft_lengths", dev)
    if tokens_out is None:
        tokens_out = torch.empty((n, k + 1), dtype=torch.int64, device=dev)
    else:
        _check_2d(tokens_out, torch.int64, (n, k + 1), "tokens_out", dev)
    if n_accepted_out is None:
        n_accepted_out = torch.empty(n, dtype=torch.int32, device=dev)
    else:
        _check(n_accepted_out, torch.int32, n, "n_accepted_out", dev)
    if logprobs_out is None:
        logprobs_out = torch.empty((n, k + 1), dtype=torch.float32, device=dev)
    else:
        _check_2d(logprobs_out, torch.float32, (n, k + 1), "logprobs_out", dev)
    L, code = lib(), _DTYPE_CODES[dtype]
    if workspace is None:
        workspace = _own_workspace(L.grpo_verify_workspace_bytes(n, k, v, code), dev, stream)
    _call("grpo_verify_drafts", dev, L.grpo_verify_drafts, _ptr(target_logits), tb, tk, _ptr(draft_logits), db, dk, code, n, k, v,
          _ptr(draft_tokens), _ptr(accept_u), _ptr(sample_u), _ptr(draft_lengths), float(temperature), float(draft_temperature),
          _ptr(tokens_out), _ptr(n_accepted_out), _ptr(logprobs_out), _ptr(workspace), workspace.numel(), _raw_stream(stream, dev.index))
    return tokens_out, n_accepted_out, logprobs_out


_DTYPE_CODES = {torch.float32: GRPO_F32, torch.bfloat16: GRPO_BF16}


def _block_norm_rows(t, name, dtype, n, d, device):
    """The pitch of an [n, d] tensor whose rows have unit stride."""
    if t.dtype != dtype or t.dim() != 2 or t.shape[0] != n or t.shape[1] != d or (t.stride(1) != 1 and d > 1):
        raise ValueError("%s must be a %s tensor [%d, %d] with unit stride along d_model" % (name, dtype, n, d))
    if t.device != device:
        raise ValueError("%s must live on %s" % (name, device))
    return t.stride(0) if n > 1 else max(t.stride(0), d)


def _block_norm_args(residual, block, post_weight, gate, pre_weight, dtype):
    """Device, sizes, dtype and the pitches of the residual stream, the block's output and the gate."""
    if not residual.is_cuda:
        raise ValueError("residual must be a device tensor: libgrpo has no CPU path")
    if residual.dim() != 2 or residual.dtype not in _DTYPE_CODES:
        raise ValueError("residual must be a float32 or bfloat16 tensor [n_tokens, d_model]")
    if dtype not in _DTYPE_CODES:
        raise ValueError("block, gate and weights must be float32 or bfloat16")
    dev = residual.device
    n, d = residual.shape
    rs = _block_norm_rows(residual, "residual", residual.dtype, n, d, dev)
    fs = gs = 0
    if block is not None:
        fs = _block_norm_rows(block, "block", dtype, n, d, dev)
    if post_weight is not None:
        _check(post_weight, dtype, d, "post_weight", dev)
    if pre_weight is not None:
        _check(pre_weight, dtype, d, "pre_weight", dev)
    if gate is not None and gate.dim() == 1:
        _check(gate, dtype, d, "gate", dev)
    elif gate is not None:
        gs = _block_norm_rows(gate, "gate", dtype, n, d, dev)
        if gs == 0 and n > 1:
            raise ValueError("a gate for all rows is a tensor [d_model]")
    return dev, n, d, rs, fs, gs


def _new_rows(n, d, dtype, device):
    """[n, d] with rows on 16-byte boundaries."""
    per16 = 8 if dtype == torch.bfloat16 else 4
    if d % per16 == 0:
        return torch.empty((n, d), dtype=dtype, device=device)
    return torch.empty((n, d + per16 - d % per16), dtype=dtype, device=device)[:, :d]


def grpo_block_norm_fwd(residual, block=None, post_weight=None, gate=None, pre_weight=None, residual_scale=1.0, eps=1e-6, *,
                        residual_out=None, hidden=None, inplace=False, stream=None):
    """Returns (residual_out, hidden): residual + residual_scale * gate * norm(block) * post_weight, and its norm times
    pre_weight (None without one); see grpo_block_norm_fwd in grpo.h.  ``gate`` is [n_tokens, d_model], or [d_model] for all
    rows.  Without a block residual_out is residual itself; ``inplace=True`` writes over it."""
    if residual_out is None and hidden is None and not inplace and stream is None:
        out = _fast.block_norm_fwd(residual, block, post_weight, gate, pre_weight, residual_scale, eps)
        if out is not None:
            return _fast_result(out, "grpo_block_norm_fwd")
    dtype = next((t.dtype for t in (block, pre_weight) if t is not None), residual.dtype)
    dev, n, d, rs, fs, gs = _block_norm_args(residual, block, post_weight, gate, pre_weight, dtype)
    os_ = hs = 0
    if block is not None:
        if inplace:
            residual_out = residual
        elif residual_out is None:
            residual_out = _new_rows(n, d, residual.dtype, dev)
        os_ = _block_norm_rows(residual_out, "residual_out", residual.dtype, n, d, dev)
    elif residual_out is not None:
        raise ValueError("residual_out is written only where there is a block")
    if pre_weight is not None:
        if hidden is None:
            hidden = _new_rows(n, d, dtype, dev)
        hs = _block_norm_rows(hidden, "hidden", dtype, n, d, dev)
    elif hidden is not None:
        raise ValueError("hidden is written only where there is a pre_weight")
    _call("grpo_block_norm_fwd", dev, lib().grpo_block_norm_fwd, _ptr(residual), rs, _DTYPE_CODES[residual.dtype], _ptr(block), fs,
          _ptr(post_weight), _ptr(gate), gs, _ptr(pre_weight), _DTYPE_CODES[dtype], n, d, float(residual_scale), float(eps),
          _ptr(residual_out), os_, _ptr(hidden), hs, _raw_stream(stream, dev.index))
    return (residual if block is None else residual_out), hidden


def grpo_block_norm_bwd(residual_out, block=None, post_weight=None, gate=None, pre_weight=None, grad_hidden=None,
                        grad_residual_out=None, residual_scale=1.0, eps=1e-6, *, grad_residual=None, grad_block=None, grad_gate=None,
                        grad_post_weight=None, grad_pre_weight=None, accumulate_grad_weights=False, workspace=None, stream=None):
    """Gradients of grpo_block_norm_fwd, whose residual_out this takes; see grpo_block_norm_bwd in grpo.h.

    Returns (grad_residual, grad_block, grad_gate, grad_post_weight, grad_pre_weight), None for what there is not.  The
    gradients of the weights, and of a gate for all rows, are f32 [d_model]."""
    if grad_residual is None and grad_block is None and grad_gate is None and grad_post_weight is None and grad_pre_weight is None and \
            not accumulate_grad_weights and workspace is None and stream is None:
        out = _fast.block_norm_bwd(residual_out, block, post_weight, gate, pre_weight, grad_hidden, grad_residual_out, residual_scale, eps)
        if out is not None:
            return _fast_result(out, "grpo_block_norm_bwd")
    dtype = next((t.dtype for t in (block, pre_weight) if t is not None), residual_out.dtype)
    dev, n, d, rs, fs, gs = _block_norm_args(residual_out, block, post_weight, gate, pre_weight, dtype)
    if (grad_hidden is None) != (pre_weight is None):
        raise ValueError("grad_hidden goes with pre_weight")
    hs = 0 if grad_hidden is None else _block_norm_rows(grad_hidden, "grad_hidden", dtype, n, d, dev)
    os_ = 0 if grad_residual_out is None else _block_norm_rows(grad_residual_out, "grad_residual_out", residual_out.dtype, n, d, dev)
    if grad_residual is None:
        grad_residual = _new_rows(n, d, residual_out.dtype, dev)
    dxs = _block_norm_rows(grad_residual, "grad_residual", residual_out.dtype, n, d, dev)
    dfs = dgs = 0
    if block is not None:
        if grad_block is None:
            grad_block = _new_rows(n, d, dtype, dev)
        dfs = _block_norm_rows(grad_block, "grad_block", dtype, n, d, dev)
    sums = [(grad_post_weight, post_weight, "grad_post_weight"), (grad_pre_weight, pre_weight, "grad_pre_weight")]
    if gate is not None and gate.dim() == 1:
        sums.append((grad_gate, gate, "grad_gate"))
    elif gate is not None:
        if grad_gate is None:
            grad_gate = _new_rows(n, d, dtype, dev)
        dgs = _block_norm_rows(grad_gate, "grad_gate", dtype, n, d, dev)
    made = []
    for grad, of, name in sums:
        if of is not None and grad is None:
            if accumulate_grad_weights:
                raise ValueError("accumulate_grad_weights needs the %s tensor to add to" % name)
            grad = torch.empty(d, dtype=torch.float32, device=dev)
        elif grad is not None:
            _check(grad, torch.float32, d, name, dev)
        made.append(grad)
    grad_post_weight, grad_pre_weight = made[:2]
    if len(made) > 2:
        grad_gate = made[2]
    L = lib()
    if workspace is None:
        workspace = _own_workspace(L.grpo_block_norm_workspace_bytes(n, d), dev, stream)
    _call("grpo_block_norm_bwd", dev, L.grpo_block_norm_bwd, _ptr(residual_out) if pre_weight is not None else None, rs,
          _DTYPE_CODES[residual_out.dtype], _ptr(block), fs, _ptr(post_weight), _ptr(gate), gs, _ptr(pre_weight), _DTYPE_CODES[dtype], n, d,
          float(residual_scale), float(eps), _ptr(grad_hidden), hs, _ptr(grad_residual_out), os_, _ptr(grad_residual), dxs,
          _ptr(grad_block), dfs, _ptr(grad_gate), dgs, _ptr(grad_post_weight), _ptr(grad_pre_weight), 1 if accumulate_grad_weights else 0,
          _ptr(workspace), workspace.numel(), _raw_stream(stream, dev.index))
    return grad_residual, grad_block, grad_gate, grad_post_weight, grad_pre_weight


class OptimPlan:
    """The tensors of a model as grpo_grad_norm and grpo_adamw_step take them: made by grpo_optim_plan, which see.  It
    keeps the tensors it was made from alive."""

    def __init__(self, plan, table, tensors):
        self._plan, self._table, self._tensors = plan, table, tensors
        self._address = ctypes.addressof(plan)

    @property
    def device(self):
        return self._table.device


def _optim_list(tensors, n, name, dtypes, device):
    """`tensors` as a list of n contiguous tensors of one of the dtypes on the device; n times None where there are none."""
    if tensors is None:
        return [None] * n
    tensors = list(tensors)
    if len(tensors) != n:
        raise ValueError("%s has %d tensors and grads %d" % (name, len(tensors), n))
    for t in tensors:
        if t is not None and (t.dtype not in dtypes or not t.is_contiguous() or t.device != device):
            raise ValueError("%s must be contiguous tensors of %s on %s" % (name, " or ".join(str(d) for d in dtypes), device))
    return tensors


def grpo_optim_plan(params, grads, exp_avgs=None, exp_avg_sqs=None, *, masters=None, exp_avg_scales=None, exp_avg_sq_scales=None,
                    weight_decay=0.0):
    """An OptimPlan of these tensors; see grpo_optim_tensor and grpo_optim_plan_build in grpo.h.

    Lists of equal length, a tensor's gradient, moments, ... at its own place: params f32 or bf16 (None: the plan is for
    grpo_grad_norm only), grads f32 or bf16, exp_avgs and exp_avg_sqs f32, or float8_e4m3fn with exp_avg_scales and
    exp_avg_sq_scales, one f32 for every 256 values; masters f32 or None, as a whole or in single places.  weight_decay: a
    number, or a list of them.  The plan holds the tensors' addresses: gradients are brought into the same tensors before
    every step, and moments and parameters are changed in them."""
    grads = list(grads)
    n = len(grads)
    if not grads:
        raise ValueError("there are no tensors")
    dev = grads[0].device
    if dev.type != "cuda":
        raise ValueError("grads must be device tensors: libgrpo has no CPU path")
    f32, bf16, e4m3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
    grads = _optim_list(grads, n, "grads", (f32, bf16), dev)
    params = _optim_list(params, n, "params", (f32, bf16), dev)
    masters = _optim_list(masters, n, "masters", (f32,), dev)
    m = _optim_list(exp_avgs, n, "exp_avgs", (f32, e4m3), dev)
    v = _optim_list(exp_avg_sqs, n, "exp_avg_sqs", (f32, e4m3), dev)
    ms = _optim_list(exp_avg_scales, n, "exp_avg_scales", (f32,), dev)
    vs = _optim_list(exp_avg_sq_scales, n, "exp_avg_sq_scales", (f32,), dev)
    decay = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else [float(w) for w in weight_decay]
    if len(decay) != n:
        raise ValueError("weight_decay has %d numbers and grads %d tensors" % (len(decay), n))
    table = (_OptimTensor * n)()
    for i, e in enumerate(table):
        count = grads[i].numel()
        for t, name in ((params[i], "param"), (masters[i], "master"), (m[i], "exp_avg"), (v[i], "exp_avg_sq")):
            if t is not None and t.numel() != count:
                raise ValueError("tensor %d: %s has %d values and its gradient %d" % (i, name, t.numel(), count))
        if m[i] is not None and v[i] is not None and m[i].dtype != v[i].dtype:
            raise ValueError("tensor %d: both moments must be of the same dtype" % i)
        for t, name in ((ms[i], "exp_avg_scale"), (vs[i], "exp_avg_sq_scale")):
            if t is not None and t.numel() != (count + 255) // 256:
                raise ValueError("tensor %d: %s must have one value for every 256" % (i, name))
        e.param, e.master, e.grad, e.exp_avg, e.exp_avg_sq = (_ptr(t) for t in (params[i], masters[i], grads[i], m[i], v[i]))
        e.exp_avg_scale, e.exp_avg_sq_scale = _ptr(ms[i]), _ptr(vs[i])
        e.n, e.weight_decay = count, decay[i]
        e.param_dtype = GRPO_BF16 if params[i] is not None and params[i].dtype == bf16 else GRPO_F32
        e.grad_dtype = GRPO_BF16 if grads[i].dtype == bf16 else GRPO_F32
        e.state_bits = 8 if m[i] is not None and m[i].dtype == e4m3 else 32
    host = torch.empty(int(lib().grpo_optim_plan_bytes(table, n)), dtype=torch.uint8)
    plan = _OptimPlan()
    rc = lib().grpo_optim_plan_build(table, n, _ptr(host), host.numel(), ctypes.byref(plan))
    if rc != GRPO_OK:
        raise GrpoError(rc, "grpo_optim_plan_build")
    return OptimPlan(plan, host.to(dev), [t for group in (params, masters, grads, m, v, ms, vs) for t in group if t is not None])


def grpo_grad_norm(plan, max_norm=0.0, *, norm_out=None, workspace=None, stream=None):
    """[2] f32: the norm of all the plan's gradients, and the coefficient that clips it at max_norm (1 where there is none);
    see grpo_grad_norm in grpo.h."""
    if norm_out is None and workspace is None and stream is None:
        out = _fast.grad_norm(plan._address, plan._table, max_norm)
        if out is not None:
            return _fast_result(out, "grpo_grad_norm")
    dev = plan.device
    if norm_out is None:
        norm_out = torch.empty(2, dtype=torch.float32, device=dev)
    else:
        _check(norm_out, torch.float32, 2, "norm_out", dev)
    L = lib()
    if workspace is None:
        workspace = _own_workspace(L.grpo_grad_norm_workspace_bytes(), dev, stream)
    _call("grpo_grad_norm", dev, L.grpo_grad_norm, plan._address, _ptr(plan._table), float(max_norm), _ptr(norm_out), _ptr(workspace),
          workspace.numel(), _raw_stream(stream, dev.index))
    return norm_out


def grpo_adamw_step(plan, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, *, clip=None, stream=None):
    """One AdamW step over the plan's tensors, in place; see grpo_adamw_step in grpo.h.

    ``step`` counts from 1; ``step`` (i64) and ``lr`` (f32) may be device tensors of one value, which a captured graph reads at
    every replay.  ``clip``: what grpo_grad_norm returned."""
    if stream is None:
        out = _fast.adamw_step(plan._address, plan._table, step, lr, beta1, beta2, eps, clip)
        if out is not None:
            _fast_result(out, "grpo_adamw_step")
            return
    dev = plan.device
    step_at = lr_at = None
    if isinstance(step, torch.Tensor):
        _check(step, torch.int64, 1, "step", dev)
        step, step_at = 0, _ptr(step)
    if isinstance(lr, torch.Tensor):
        _check(lr, torch.float32, 1, "lr", dev)
        lr, lr_at = 0.0, _ptr(lr)
    if clip is not None:
        _check(clip, torch.float32, 2, "clip", dev)
    _call("grpo_adamw_step", dev, lib().grpo_adamw_step, plan._address, _ptr(plan._table), int(step), step_at, float(lr), lr_at,
          float(beta1), float(beta2), float(eps), _ptr(clip), _raw_stream(stream, dev.index))
