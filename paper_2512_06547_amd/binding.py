"""ctypes binding of liba3po.so: same names as the C entry points, argument marshalling only.

Every function takes torch tensors that already live on the GPU, passes their device
pointers and the current HIP stream to the C ABI, and returns torch tensors.  There is no
fallback: if the shared library is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "liba3po.so")

A3PO_F32, A3PO_BF16 = 0, 1
A3PO_PROX_INTERP, A3PO_PROX_GIVEN, A3PO_PROX_BEHAV = 0, 1, 2
A3PO_WS_LOSS_FWD_BWD = 0
A3PO_WS_FUSED_LMHEAD = 1
A3PO_WS_FUSED_LMHEAD_LOSS = 2
A3PO_WS_NORM_BWD = 3
A3PO_WS_ADJUST_LOGITS = 4
A3PO_WS_W4_LINEAR = 5
A3PO_WS_SAMPLE = 6
A3PO_WS_GRAD_NORM = 7
A3PO_STATE_F32, A3PO_STATE_8BIT = 0, 1
A3PO_NORM_LAYER, A3PO_NORM_RMS = 0, 1
A3PO_NORM_ONE_LAUNCH_ROWS, A3PO_NORM_ONE_LAUNCH_ELEMENTS = 1024, 3 << 20

# layout of a3po_stats (include/a3po.h)
STATS_DTYPE = np.dtype([("n_tokens", "<i8"), ("n_clipped", "<i8"), ("n_bad_index", "<i8"),
                        ("n_negative_staleness", "<i8"), ("iw_min", "<f4"), ("iw_max", "<f4"),
                        ("entropy_mean", "<f4"), ("reserved", "<f4")])

_P, _I64, _I32, _F32, _SZ = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t



class LossOptions(ctypes.Structure):
    """a3po_loss_options (include/a3po.h)."""
    _fields_ = [("prox_mode", ctypes.c_int32), ("accumulate", ctypes.c_int32), ("logp_prox_in", ctypes.c_void_p),
                ("entropy_out", ctypes.c_void_p), ("iw_out", ctypes.c_void_p), ("clipped_out", ctypes.c_void_p),
                ("event_before_rows", ctypes.c_void_p), ("event_after_rows", ctypes.c_void_p),
                ("denom_dev", ctypes.c_void_p)]


class LogitAdjustments(ctypes.Structure):
    """a3po_logit_adjustments (include/a3po.h)."""
    _fields_ = [("history", ctypes.c_void_p), ("history_tokens", ctypes.c_int64), ("hist_start", ctypes.c_void_p),
                ("hist_len", ctypes.c_void_p), ("prompt_len", ctypes.c_void_p), ("repetition", ctypes.c_void_p),
                ("frequency", ctypes.c_void_p), ("presence", ctypes.c_void_p), ("temperature", ctypes.c_void_p),
                ("bias", ctypes.c_void_p), ("bias_ld", ctypes.c_int64), ("allowed", ctypes.c_void_p),
                ("allowed_ld", ctypes.c_int64)]


class Sampling(ctypes.Structure):
    """a3po_sampling (include/a3po.h)."""
    _fields_ = [("uniform", ctypes.c_void_p), ("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p),
                ("top_p", ctypes.c_void_p), ("min_p", ctypes.c_void_p)]


class AdamwTensor(ctypes.Structure):
    """a3po_adamw_tensor (include/a3po.h)."""
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("exp_avg", ctypes.c_void_p),
                ("exp_avg_sq", ctypes.c_void_p), ("exp_avg_scale", ctypes.c_void_p), ("exp_avg_sq_scale", ctypes.c_void_p),
                ("copy", ctypes.c_void_p), ("n", ctypes.c_int64)]


class AdamwOptions(ctypes.Structure):
    """a3po_adamw_options (include/a3po.h)."""
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("step", ctypes.c_int64), ("lr_dev", ctypes.c_void_p),
                ("step_dev", ctypes.c_void_p), ("norm", ctypes.c_void_p), ("max_norm", ctypes.c_double),
                ("seed", ctypes.c_uint32)]


_SIGNATURES = {
    "a3po_workspace_bytes": (_SZ, [ctypes.c_int, _I64, _I64, _I64]),
    "a3po_strerror": (ctypes.c_char_p, [ctypes.c_int]),
    "a3po_token_logprobs": (ctypes.c_int, [_P, ctypes.c_int, _I64, _I64, _I64, _P, _P, _P, _P, _P]),
    "a3po_proximal_interp": (ctypes.c_int, [_P, _P, _P, _I32, _I64, _P, _P, _P]),
    "a3po_grpo_advantages": (ctypes.c_int, [_P, _I64, _I32, _F32, _P, _I64, _P, _P]),
    "a3po_fused_lmhead_logprob": (ctypes.c_int, [_P, _P, _I64, _I64, _I64, _P, _P, _P, _P, _SZ, _P]),
    "a3po_fused_lmhead_loss_fwd_bwd": (ctypes.c_int, [_P, _P, _I64, _I64, _I64, _P, _P, _P, _I32, _P, _P, _F32, _F32,
                                                      _P, _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "a3po_loss_fwd_bwd": (ctypes.c_int, [_P, ctypes.c_int, _I64, _I64, _I64, _P, _P, _P, _I32, _P, _P, _F32, _F32,
                                         _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "a3po_loss_fwd_bwd_noalloc": (ctypes.c_int, [_P, ctypes.c_int, _I64, _I64, _I64, _P, _P, _P, _I32, _P, _P, _F32,
                                                 _F32, _P, _P, _P, _P, _P, _P]),
    "a3po_loss_fwd_bwd_ex": (ctypes.c_int, [_P, ctypes.c_int, _I64, _I64, _I64, _P, _P, _P, _I32, _P, _P, _F32,
                                            _F32, _P, _P, _P, _P, _P, _P, _SZ, _P, ctypes.POINTER(LossOptions)]),
    "a3po_count_tokens": (ctypes.c_int, [_P, _P, _I64, _I64, _P, _P, _P]),
    "a3po_histogram": (ctypes.c_int, [_P, _P, _I64, _P, _I32, _I32, _P, _P]),
    "a3po_plan_microbatches": (ctypes.c_int, [_P, _I64, _I32, _I64, _P, _P, _I64, _P]),
    "a3po_shard_partials": (ctypes.c_int, [_P, ctypes.c_int, _I64, _I64, _I64, _P, _I64, _P, _P]),
    "a3po_shard_combine": (ctypes.c_int, [_P, _I32, _I64, _P, _I64, _P, _P, _P, _P]),
    "a3po_shard_loss_bwd": (ctypes.c_int, [_P, ctypes.c_int, _I64, _I64, _I64, _I64, _I64, _P, _P, _P, _P, _P, _I32,
                                           _P, _P, _F32, _F32, _P, _P, _P, _P, _P, _SZ, _P,
                                           ctypes.POINTER(LossOptions)]),
    "a3po_token_logprobs_entropy": (ctypes.c_int, [_P, ctypes.c_int, _I64, _I64, _I64, _P, _P, _P, _P, _P, _P]),
    "a3po_norm_fwd": (ctypes.c_int, [_P, ctypes.c_int, _I64, _I64, _I64, _P, _P, ctypes.c_int, _F32, _I32, _P,
                                     ctypes.c_int, _I64, _P, _P, _P]),
    "a3po_norm_bwd": (ctypes.c_int, [_P, ctypes.c_int, _I64, _P, ctypes.c_int, _I64, _I64, _I64, _P, ctypes.c_int, _P, _P,
                                     _I32, _P, _I64, _P, _P, _I32, _P, _SZ, _P]),
    "a3po_adjust_logits": (ctypes.c_int, [_P, ctypes.c_int, _I64, _I64, _I64, ctypes.POINTER(LogitAdjustments), _P, _P,
                                          ctypes.c_int, _I64, _P, _P, _P, _SZ, _P]),
    "a3po_adjust_logits_bwd": (ctypes.c_int, [_P, ctypes.c_int, _I64, _P, ctypes.c_int, _I64, _I64, _I64,
                                              ctypes.POINTER(LogitAdjustments), _P, _I64, _P]),
    "a3po_w4_linear": (ctypes.c_int, [_P, _I64, _I64, _I64, _P, _P, ctypes.c_int, _P, _I32, _I64, _P, ctypes.c_int, _I64,
                                      _P, _SZ, _P]),
    "a3po_sample": (ctypes.c_int, [_P, ctypes.c_int, _I64, _I64, _I64, ctypes.POINTER(Sampling), _P, _P, _P, _P, _P, _I64, _P,
                                   _SZ, _P]),
    "a3po_grad_norm": (ctypes.c_int, [_P, _P, _I64, ctypes.c_int, _F32, _P, _P, _SZ, _P]),
    "a3po_adamw_step": (ctypes.c_int, [_P, _I64, ctypes.c_int, ctypes.c_int, _I32, ctypes.POINTER(AdamwOptions), _P]),
    "a3po_w4_quantize": (ctypes.c_int, [_P, ctypes.c_int, _I64, _I64, _I64, _I32, _P, _P, ctypes.c_int, _P, _P]),
}

_lib = None


class A3poError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} ({code})")


def lib_path() -> str:
    return _LIB_PATH


def lib() -> ctypes.CDLL:
    """The loaded shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise FileNotFoundError(
                f"{_LIB_PATH} is missing: build it with `python -m paper_2512_06547_amd.build` "
                "(there is no fallback path)")
        # PyTorch first: it brings its own copy of the HIP runtime, and the library must bind to that same copy (a
        # stream or pointer created by one copy of the runtime means nothing to another); once PyTorch's is in the
        # process, the library's dependency on the runtime resolves to it
        try:
            import torch  # noqa: F401
        except ImportError:
            pass
        handle = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype, fn.argtypes = res, args
        _lib = handle
    return _lib


def strerror(code: int) -> str:
    return lib().a3po_strerror(int(code)).decode()


def _check(rc: int, where: str) -> None:
    if rc != 0:
        raise A3poError(rc, where)


def _torch():
    import torch
    return torch


def _stream() -> int:
    # the raw handle of the current device's current stream.  torch.cuda.current_stream() builds a Stream object for it,
    # 3.0 us of the 10 us a short call takes on the host; asked for directly the handle costs 0.2 us
    c = _torch()._C
    if hasattr(c, "_cuda_getCurrentRawStream"):
        return c._cuda_getCurrentRawStream(c._cuda_getDevice())
    return _torch().cuda.current_stream().cuda_stream


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _logits_meta(logits, V):
    torch = _torch()
    assert logits.is_cuda and logits.dim() == 2 and logits.stride(1) == 1, "logits must be a row-major CUDA matrix"
    if logits.dtype == torch.float32:
        dt = A3PO_F32
    elif logits.dtype == torch.bfloat16:
        dt = A3PO_BF16
    else:
        raise TypeError("logits must be float32 or bfloat16")
    T = logits.shape[0]
    ld = logits.stride(0) if T > 1 else max(logits.stride(0), logits.shape[1])
    V = logits.shape[1] if V is None else int(V)
    return dt, T, V, ld


def _vec(t, dtype, n, name):
    assert t.is_cuda and t.dtype == dtype and t.is_contiguous() and t.numel() == n, f"{name}: need contiguous {dtype}[{n}] on GPU"
    return t


def workspace_bytes(T: int, V: int = 0, H: int = 0, which: int = A3PO_WS_LOSS_FWD_BWD) -> int:
    return int(lib().a3po_workspace_bytes(which, T, V, H))


def token_logprobs(logits, chosen, V=None, want_lse=True, want_chosen_logit=True, want_entropy=False):
    """a3po_token_logprobs -> (logp[T] f32, lse[T] f32 | None, chosen_logit[T] logits.dtype | None);
    with want_entropy, a3po_token_logprobs_entropy -> (..., entropy[T] f32)."""
    torch = _torch()
    dt, T, V, ld = _logits_meta(logits, V)
    _vec(chosen, torch.int32, T, "chosen")
    dev = logits.device
    logp = torch.empty(T, dtype=torch.float32, device=dev)
    lse = torch.empty(T, dtype=torch.float32, device=dev) if want_lse else None
    zy = torch.empty(T, dtype=logits.dtype, device=dev) if want_chosen_logit else None
    if not want_entropy:
        _check(lib().a3po_token_logprobs(_ptr(logits), dt, T, V, ld, _ptr(chosen), _ptr(logp), _ptr(lse), _ptr(zy),
                                         _stream()), "a3po_token_logprobs")
        return logp, lse, zy
    ent = torch.empty(T, dtype=torch.float32, device=dev)
    _check(lib().a3po_token_logprobs_entropy(_ptr(logits), dt, T, V, ld, _ptr(chosen), _ptr(logp), _ptr(lse),
                                             _ptr(zy), _ptr(ent), _stream()), "a3po_token_logprobs_entropy")
    return logp, lse, zy, ent


def proximal_interp(logp_behav, logp_theta, versions, current_version: int, want_alpha=True):
    """a3po_proximal_interp -> (logp_prox[T] f32, alpha[T] f32 | None)."""
    torch = _torch()
    T = versions.numel()
    _vec(logp_behav, torch.float32, T, "logp_behav")
    _vec(logp_theta, torch.float32, T, "logp_theta")
    _vec(versions, torch.int32, T, "versions")
    lp = torch.empty(T, dtype=torch.float32, device=versions.device)
    al = torch.empty(T, dtype=torch.float32, device=versions.device) if want_alpha else None
    _check(lib().a3po_proximal_interp(_ptr(logp_behav), _ptr(logp_theta), _ptr(versions), int(current_version), T,
                                      _ptr(lp), _ptr(al), _stream()), "a3po_proximal_interp")
    return lp, al


def grpo_advantages(rewards, G: int, seq_id, eps_adv: float = 1e-6, out=None):
    """a3po_grpo_advantages -> adv[T] f32 (advantage of each token's sequence)."""
    torch = _torch()
    S, T = rewards.numel(), seq_id.numel()
    _vec(rewards, torch.float32, S, "rewards")
    _vec(seq_id, torch.int32, T, "seq_id")
    adv = torch.empty(T, dtype=torch.float32, device=seq_id.device) if out is None else out
    _check(lib().a3po_grpo_advantages(_ptr(rewards), S, int(G), float(eps_adv), _ptr(seq_id), T, _ptr(adv),
                                      _stream()), "a3po_grpo_advantages")
    return adv


def loss_fwd_bwd(logits, chosen, logp_behav, versions, current_version: int, advantages, loss_mask,
                 clip_eps: float, denom: float = 0.0, V=None, dlogits=None, workspace=None, out=None,
                 events=None, prox_mode: int = A3PO_PROX_INTERP, logp_prox_in=None, want_entropy=False,
                 want_iw=False, want_clipped=False, denom_dev=None, accumulate=False):
    """a3po_loss_fwd_bwd, or a3po_loss_fwd_bwd_ex when any extra is asked for: ``events=(start, stop)`` raw
    hipEvent_t handles, ``prox_mode`` / ``logp_prox_in`` (the given-proximal and coupled variants; ``versions``
    may then be None), ``want_entropy`` / ``want_iw`` / ``want_clipped`` per-token outputs, ``denom_dev`` (a
    1-element float32 device tensor that replaces ``denom``) and ``accumulate`` (add to the loss / stats in ``out``).

    dlogits: None -> a new tensor like logits; or a tensor with the same dtype and strides (may be
    ``logits`` itself for the in-place form).  ``out`` may carry preallocated output tensors from an earlier
    call.  Returns a dict with dlogits, logp, logp_prox, loss (1-element tensor), stats (uint8 tensor, see
    STATS_DTYPE), the workspace, and entropy / iw / clipped when asked for.
    """
    torch = _torch()
    dt, T, V, ld = _logits_meta(logits, V)
    dev = logits.device
    _vec(chosen, torch.int32, T, "chosen")
    _vec(logp_behav, torch.float32, T, "logp_behav")
    if versions is not None:
        _vec(versions, torch.int32, T, "versions")
    _vec(advantages, torch.float32, T, "advantages")
    _vec(loss_mask, torch.uint8, T, "loss_mask")
    if logp_prox_in is not None:
        _vec(logp_prox_in, torch.float32, T, "logp_prox_in")
    if dlogits is None:
        dlogits = torch.empty_strided(logits.shape, logits.stride(), dtype=logits.dtype, device=dev)
    assert dlogits.dtype == logits.dtype and dlogits.shape == logits.shape and dlogits.stride() == logits.stride()
    need = workspace_bytes(T, V)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    out = {} if out is None else out

    def buf(name, dtype, n=T):
        t = out.get(name)
        return t if t is not None else torch.empty(n, dtype=dtype, device=dev)

    logp, prox = buf("logp", torch.float32), buf("logp_prox", torch.float32)
    loss, stats = buf("loss", torch.float32, 1), buf("stats", torch.uint8, STATS_DTYPE.itemsize)
    ent = buf("entropy", torch.float32) if want_entropy else None
    iw = buf("iw", torch.float32) if want_iw else None
    clipped = buf("clipped", torch.uint8) if want_clipped else None
    args = [_ptr(logits), dt, T, V, ld, _ptr(chosen), _ptr(logp_behav), _ptr(versions), int(current_version),
            _ptr(advantages), _ptr(loss_mask), float(clip_eps), float(denom), _ptr(dlogits), _ptr(logp), _ptr(prox),
            _ptr(loss), _ptr(stats), _ptr(workspace), workspace.numel(), _stream()]
    extras = (events is not None or prox_mode != A3PO_PROX_INTERP or logp_prox_in is not None or want_entropy
              or want_iw or want_clipped or denom_dev is not None or accumulate)
    if not extras:
        _check(lib().a3po_loss_fwd_bwd(*args), "a3po_loss_fwd_bwd")
    else:
        ev = events if events is not None else (None, None)
        opt = LossOptions(int(prox_mode), int(bool(accumulate)), _ptr(logp_prox_in), _ptr(ent), _ptr(iw),
                          _ptr(clipped), ev[0], ev[1], _ptr(denom_dev))
        _check(lib().a3po_loss_fwd_bwd_ex(*args, ctypes.byref(opt)), "a3po_loss_fwd_bwd_ex")
    res = dict(dlogits=dlogits, logp=logp, logp_prox=prox, loss=loss, stats=stats, workspace=workspace)
    if want_entropy:
        res["entropy"] = ent
    if want_iw:
        res["iw"] = iw
    if want_clipped:
        res["clipped"] = clipped
    return res


NOALLOC_MAX_TOKENS = 131072  # A3PO_NOALLOC_MAX_TOKENS


def loss_fwd_bwd_noalloc(logits, chosen, logp_behav, versions, current_version: int, advantages, loss_mask,
                         clip_eps: float, denom: float, dlogits, logp, logp_prox, loss, stats, V=None):
    """a3po_loss_fwd_bwd_noalloc: every output tensor is the caller's (dlogits like logits, logp / logp_prox
    float32[T], loss float32[1], stats uint8[sizeof a3po_stats]; logp_prox and stats may be None); the call
    itself allocates nothing, here or in the library."""
    torch = _torch()
    dt, T, V, ld = _logits_meta(logits, V)
    _vec(chosen, torch.int32, T, "chosen")
    _vec(logp_behav, torch.float32, T, "logp_behav")
    _vec(versions, torch.int32, T, "versions")
    _vec(advantages, torch.float32, T, "advantages")
    _vec(loss_mask, torch.uint8, T, "loss_mask")
    assert dlogits.dtype == logits.dtype and dlogits.shape == logits.shape and dlogits.stride() == logits.stride()
    _vec(logp, torch.float32, T, "logp")
    if logp_prox is not None:
        _vec(logp_prox, torch.float32, T, "logp_prox")
    _vec(loss, torch.float32, 1, "loss")
    if stats is not None:
        _vec(stats, torch.uint8, STATS_DTYPE.itemsize, "stats")
    _check(lib().a3po_loss_fwd_bwd_noalloc(_ptr(logits), dt, T, V, ld, _ptr(chosen), _ptr(logp_behav), _ptr(versions),
                                           int(current_version), _ptr(advantages), _ptr(loss_mask), float(clip_eps),
                                           float(denom), _ptr(dlogits), _ptr(logp), _ptr(logp_prox), _ptr(loss),
                                           _ptr(stats), _stream()), "a3po_loss_fwd_bwd_noalloc")


def count_tokens(chosen, loss_mask, V: int, want_count=False):
    """a3po_count_tokens -> denom (1-element f32 device tensor) [, count (1-element i64 device tensor)]."""
    torch = _torch()
    T = chosen.numel()
    _vec(chosen, torch.int32, T, "chosen")
    _vec(loss_mask, torch.uint8, T, "loss_mask")
    denom = torch.empty(1, dtype=torch.float32, device=chosen.device)
    cnt = torch.empty(1, dtype=torch.int64, device=chosen.device) if want_count else None
    _check(lib().a3po_count_tokens(_ptr(chosen), _ptr(loss_mask), T, int(V), _ptr(denom), _ptr(cnt), _stream()),
           "a3po_count_tokens")
    return (denom, cnt) if want_count else denom


def histogram(values, edges, select=None, accumulate=False, out=None):
    """a3po_histogram -> counts int64[nbins + 3] on the device (below, bins..., at-or-above, NaN)."""
    torch = _torch()
    T = values.numel()
    _vec(values, torch.float32, T, "values")
    if select is not None:
        _vec(select, torch.uint8, T, "select")
    nbins = edges.numel() - 1
    _vec(edges, torch.float32, nbins + 1, "edges")
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs the counts of the earlier calls in `out`")
        out = torch.empty(max(nbins, 0) + 3, dtype=torch.int64, device=values.device)
    else:
        _vec(out, torch.int64, nbins + 3, "out")
    _check(lib().a3po_histogram(_ptr(values), _ptr(select), T, _ptr(edges), nbins, int(bool(accumulate)), _ptr(out),
                                _stream()), "a3po_histogram")
    return out


def plan_microbatches(seq_len, n_minibatches: int, max_tokens: int, capacity=None):
    """a3po_plan_microbatches on a host int64 array -> (micro_first_seq[n+1], micro_minibatch[n]) NumPy arrays."""
    seq_len = np.ascontiguousarray(np.asarray(seq_len, dtype=np.int64))
    S = seq_len.shape[0]
    cap = S + int(max(n_minibatches, 0)) if capacity is None else int(capacity)
    first = np.zeros(max(cap, 0) + 1, dtype=np.int64)
    mb = np.zeros(max(cap, 1), dtype=np.int32)
    n = ctypes.c_int64(0)
    _check(lib().a3po_plan_microbatches(seq_len.ctypes.data, S, int(n_minibatches), int(max_tokens), first.ctypes.data,
                                        mb.ctypes.data, cap, ctypes.addressof(n)), "a3po_plan_microbatches")
    return first[:n.value + 1].copy(), mb[:n.value].copy()


def shard_partials(logits_shard, chosen, v0: int, Vs=None, out=None):
    """a3po_shard_partials -> partial[T, 4] f32 (max, sum_exp, chosen_logit, sum_exp_z) of one column shard."""
    torch = _torch()
    dt, T, Vs, ld = _logits_meta(logits_shard, Vs)
    _vec(chosen, torch.int32, T, "chosen")
    part = torch.empty((T, 4), dtype=torch.float32, device=logits_shard.device) if out is None else out
    assert part.is_contiguous() and part.dtype == torch.float32 and part.numel() == 4 * T
    _check(lib().a3po_shard_partials(_ptr(logits_shard), dt, T, Vs, ld, _ptr(chosen), int(v0), _ptr(part), _stream()),
           "a3po_shard_partials")
    return part


def shard_combine(partials, chosen, V: int, want_lse=True, want_entropy=False):
    """a3po_shard_combine on partials[P, T, 4] -> (logp[T], lse[T] | None, entropy[T] | None)."""
    torch = _torch()
    assert partials.is_cuda and partials.dtype == torch.float32 and partials.is_contiguous() and partials.dim() == 3
    P, T = partials.shape[0], partials.shape[1]
    _vec(chosen, torch.int32, T, "chosen")
    dev = partials.device
    logp = torch.empty(T, dtype=torch.float32, device=dev)
    lse = torch.empty(T, dtype=torch.float32, device=dev) if want_lse else None
    ent = torch.empty(T, dtype=torch.float32, device=dev) if want_entropy else None
    _check(lib().a3po_shard_combine(_ptr(partials), P, T, _ptr(chosen), int(V), _ptr(logp), _ptr(lse), _ptr(ent),
                                    _stream()), "a3po_shard_combine")
    return logp, lse, ent


def shard_loss_bwd(logits_shard, v0: int, V: int, chosen, logp_theta, lse, logp_behav, versions, current_version: int,
                   advantages, loss_mask, clip_eps: float, denom: float = 0.0, Vs=None, dlogits=None, workspace=None,
                   prox_mode: int = A3PO_PROX_INTERP, logp_prox_in=None, want_iw=False, want_clipped=False):
    """a3po_shard_loss_bwd -> dict(dlogits (the shard's slice), logp_prox, loss, stats, workspace[, iw, clipped])."""
    torch = _torch()
    dt, T, Vs, ld = _logits_meta(logits_shard, Vs)
    dev = logits_shard.device
    _vec(chosen, torch.int32, T, "chosen")
    for name, t in (("logp_theta", logp_theta), ("lse", lse), ("logp_behav", logp_behav), ("advantages", advantages)):
        _vec(t, torch.float32, T, name)
    if versions is not None:
        _vec(versions, torch.int32, T, "versions")
    _vec(loss_mask, torch.uint8, T, "loss_mask")
    if dlogits is None:
        dlogits = torch.empty_strided(logits_shard.shape, logits_shard.stride(), dtype=logits_shard.dtype, device=dev)
    assert dlogits.dtype == logits_shard.dtype and dlogits.shape == logits_shard.shape
    assert dlogits.stride() == logits_shard.stride()
    if workspace is None:
        workspace = torch.empty(workspace_bytes(T, V), dtype=torch.uint8, device=dev)
    prox = torch.empty(T, dtype=torch.float32, device=dev)
    loss = torch.empty(1, dtype=torch.float32, device=dev)
    stats = torch.empty(STATS_DTYPE.itemsize, dtype=torch.uint8, device=dev)
    iw = torch.empty(T, dtype=torch.float32, device=dev) if want_iw else None
    clipped = torch.empty(T, dtype=torch.uint8, device=dev) if want_clipped else None
    opt = LossOptions(int(prox_mode), 0, _ptr(logp_prox_in), None, _ptr(iw), _ptr(clipped), None, None, None)
    _check(lib().a3po_shard_loss_bwd(_ptr(logits_shard), dt, T, Vs, ld, int(v0), int(V), _ptr(chosen),
                                     _ptr(logp_theta), _ptr(lse), _ptr(logp_behav), _ptr(versions),
                                     int(current_version), _ptr(advantages), _ptr(loss_mask), float(clip_eps),
                                     float(denom), _ptr(dlogits), _ptr(prox), _ptr(loss), _ptr(stats), _ptr(workspace),
                                     workspace.numel(), _stream(), ctypes.byref(opt)), "a3po_shard_loss_bwd")
    res = dict(dlogits=dlogits, logp_prox=prox, loss=loss, stats=stats, workspace=workspace)
    if want_iw:
        res["iw"] = iw
    if want_clipped:
        res["clipped"] = clipped
    return res


def fused_lmhead_logprob(hidden, weight, chosen, want_lse=True, workspace=None):
    """a3po_fused_lmhead_logprob -> (logp[T] f32, lse[T] f32 | None); hidden [T,H], weight [V,H] bfloat16."""
    torch = _torch()
    assert hidden.is_cuda and weight.is_cuda and hidden.dtype == torch.bfloat16 and weight.dtype == torch.bfloat16
    assert hidden.is_contiguous() and weight.is_contiguous() and hidden.dim() == 2 and weight.dim() == 2
    T, H = hidden.shape
    V = weight.shape[0]
    assert weight.shape[1] == H
    _vec(chosen, torch.int32, T, "chosen")
    need = workspace_bytes(T, V, H, which=A3PO_WS_FUSED_LMHEAD)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=hidden.device)
    logp = torch.empty(T, dtype=torch.float32, device=hidden.device)
    lse = torch.empty(T, dtype=torch.float32, device=hidden.device) if want_lse else None
    _check(lib().a3po_fused_lmhead_logprob(_ptr(hidden), _ptr(weight), T, H, V, _ptr(chosen), _ptr(logp), _ptr(lse),
                                           _ptr(workspace), workspace.numel(), _stream()), "a3po_fused_lmhead_logprob")
    return logp, lse


def fused_lmhead_loss_fwd_bwd(hidden, weight, chosen, logp_behav, versions, current_version: int, advantages,
                              loss_mask, clip_eps: float, denom: float = 0.0, workspace=None):
    """a3po_fused_lmhead_loss_fwd_bwd -> dict(dhidden, dweight, logp, logp_prox, loss, stats, workspace)."""
    torch = _torch()
    assert hidden.is_cuda and weight.is_cuda and hidden.dtype == torch.bfloat16 and weight.dtype == torch.bfloat16
    assert hidden.is_contiguous() and weight.is_contiguous() and hidden.dim() == 2 and weight.dim() == 2
    T, H = hidden.shape
    V = weight.shape[0]
    assert weight.shape[1] == H
    dev = hidden.device
    _vec(chosen, torch.int32, T, "chosen")
    _vec(logp_behav, torch.float32, T, "logp_behav")
    _vec(versions, torch.int32, T, "versions")
    _vec(advantages, torch.float32, T, "advantages")
    _vec(loss_mask, torch.uint8, T, "loss_mask")
    need = workspace_bytes(T, V, H, which=A3PO_WS_FUSED_LMHEAD_LOSS)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    dh = torch.empty_like(hidden)
    dw = torch.empty_like(weight)
    logp = torch.empty(T, dtype=torch.float32, device=dev)
    prox = torch.empty(T, dtype=torch.float32, device=dev)
    loss = torch.empty(1, dtype=torch.float32, device=dev)
    stats = torch.empty(STATS_DTYPE.itemsize, dtype=torch.uint8, device=dev)
    _check(lib().a3po_fused_lmhead_loss_fwd_bwd(
        _ptr(hidden), _ptr(weight), T, H, V, _ptr(chosen), _ptr(logp_behav), _ptr(versions), int(current_version),
        _ptr(advantages), _ptr(loss_mask), float(clip_eps), float(denom), _ptr(dh), _ptr(dw), _ptr(logp), _ptr(prox),
        _ptr(loss), _ptr(stats), _ptr(workspace), workspace.numel(), _stream()), "a3po_fused_lmhead_loss_fwd_bwd")
    return dict(dhidden=dh, dweight=dw, logp=logp, logp_prox=prox, loss=loss, stats=stats, workspace=workspace)


# ---- operators around the log-probs ----------------------------------------------------------------------------------


_DTYPE_CODES: dict = {}


def _dtype_code(t, name):
    if not _DTYPE_CODES:
        torch = _torch()
        _DTYPE_CODES.update({torch.float32: A3PO_F32, torch.bfloat16: A3PO_BF16})
    code = _DTYPE_CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32 or bfloat16")
    return code


def _rows(t, name, shape=None):
    """(dtype code, row stride) of a row-major matrix on the GPU."""
    size = t.shape
    assert t.is_cuda and len(size) == 2, f"{name} must be a row-major CUDA matrix"
    ld, step = t.stride()
    assert step == 1 or size[1] == 1, f"{name} must be a row-major CUDA matrix"
    assert shape is None or size == shape, f"{name}: need shape {shape}"
    return _dtype_code(t, name), ld if size[0] > 1 else max(ld, size[1])


def _matrix(t, dtype, shape, name):
    """Arrays with a row for each of the weight's: by their number of elements a transposed one would pass too."""
    assert t.is_cuda and t.dtype == dtype and t.shape == shape and t.is_contiguous(), f"{name}: need contiguous {dtype}{list(shape)} on GPU"


def _params(weight, bias, H):
    """The dtype code that weight and bias share."""
    if bias is not None:
        _vec(bias, bias.dtype, H, "bias")
        assert weight is None or weight.dtype == bias.dtype, "weight and bias must have one dtype"
    if weight is not None:
        _vec(weight, weight.dtype, H, "weight")
        return _dtype_code(weight, "weight")
    return A3PO_F32 if bias is None else _dtype_code(bias, "bias")


def norm_fwd(x, weight=None, bias=None, eps: float = 1e-6, kind: int = A3PO_NORM_LAYER, out=None, out_dtype=None,
             want_stats=True):
    """a3po_norm_fwd -> (y[T, H], mean[T] f32 | None, rstd[T] f32 | None).  y goes to ``out`` (may be ``x`` itself), or to a
    new tensor of ``out_dtype`` (x's by default).  The statistics are what norm_bwd takes; mean is None for A3PO_NORM_RMS."""
    torch = _torch()
    xd, ldx = _rows(x, "x")
    T, H = x.shape
    if out is None:
        out = torch.empty((T, H), dtype=x.dtype if out_dtype is None else out_dtype, device=x.device)
    yd, ldy = _rows(out, "out", (T, H))
    mean = torch.empty(T, dtype=torch.float32, device=x.device) if want_stats and kind == A3PO_NORM_LAYER else None
    rstd = torch.empty(T, dtype=torch.float32, device=x.device) if want_stats else None
    _check(lib().a3po_norm_fwd(_ptr(x), xd, T, H, ldx, _ptr(weight), _ptr(bias), _params(weight, bias, H), float(eps),
                               int(kind), _ptr(out), yd, ldy, _ptr(mean), _ptr(rstd), _stream()), "a3po_norm_fwd")
    return out, mean, rstd


def norm_bwd(dy, x, weight, rstd, mean=None, kind: int = A3PO_NORM_LAYER, dx=None, want_dweight=True, want_dbias=False,
             dweight=None, dbias=None, accumulate=False, workspace=None):
    """a3po_norm_bwd -> dict(dx (x's dtype), dweight f32[H] | None, dbias f32[H] | None, workspace | None).  ``dx`` may be ``x``
    or ``dy`` itself; with ``accumulate`` the sums are added to the given ``dweight`` / ``dbias``."""
    torch = _torch()
    yd, lddy = _rows(dy, "dy")
    T, H = dy.shape
    xd, ldx = _rows(x, "x", (T, H))
    _vec(rstd, torch.float32, T, "rstd")
    if mean is not None:
        _vec(mean, torch.float32, T, "mean")
    dev = x.device
    if dx is None:
        dx = torch.empty((T, H), dtype=x.dtype, device=dev)
    assert dx.dtype == x.dtype, "dx must have x's dtype"
    lddx = _rows(dx, "dx", (T, H))[1]
    if accumulate and ((want_dweight and dweight is None) or (want_dbias and dbias is None)):
        raise ValueError("accumulate needs the sums of the earlier calls in `dweight` / `dbias`")
    if dweight is None and want_dweight:
        dweight = torch.empty(H, dtype=torch.float32, device=dev)
    if dbias is None and want_dbias:
        dbias = torch.empty(H, dtype=torch.float32, device=dev)
    for name, t in (("dweight", dweight), ("dbias", dbias)):
        if t is not None:
            _vec(t, torch.float32, H, name)
    if workspace is None and (dweight is not None or dbias is not None) and not (
            T <= A3PO_NORM_ONE_LAUNCH_ROWS and T * H <= A3PO_NORM_ONE_LAUNCH_ELEMENTS
            and dx.data_ptr() not in (x.data_ptr(), dy.data_ptr())):
        workspace = torch.empty(workspace_bytes(T, 0, H, which=A3PO_WS_NORM_BWD), dtype=torch.uint8, device=dev)
    _check(lib().a3po_norm_bwd(_ptr(dy), yd, lddy, _ptr(x), xd, T, H, ldx, _ptr(weight), _params(weight, None, H),
                               _ptr(mean), _ptr(rstd), int(kind), _ptr(dx), lddx, _ptr(dweight), _ptr(dbias),
                               int(bool(accumulate)), _ptr(workspace), 0 if workspace is None else workspace.numel(),
                               _stream()), "a3po_norm_bwd")
    return dict(dx=dx, dweight=dweight, dbias=dbias, workspace=workspace)


def _adjustments(T, V, history, hist_start, hist_len, prompt_len, repetition, frequency, presence, temperature, bias,
                 allowed):
    torch = _torch()
    adj = LogitAdjustments()
    if history is not None:
        adj.history, adj.history_tokens = _ptr(_vec(history, torch.int32, history.numel(), "history")), history.numel()
        if hist_start is None or hist_len is None:
            raise ValueError("history needs hist_start and hist_len")
        adj.hist_start = _ptr(_vec(hist_start, torch.int64, T, "hist_start"))
        adj.hist_len = _ptr(_vec(hist_len, torch.int32, T, "hist_len"))
        if prompt_len is not None:
            adj.prompt_len = _ptr(_vec(prompt_len, torch.int32, T, "prompt_len"))
    if repetition is not None:
        adj.repetition = _ptr(_vec(repetition, torch.float32, T, "repetition"))
    if frequency is not None:
        adj.frequency = _ptr(_vec(frequency, torch.float32, T, "frequency"))
    if presence is not None:
        adj.presence = _ptr(_vec(presence, torch.float32, T, "presence"))
    if temperature is not None:
        adj.temperature = _ptr(_vec(temperature, torch.float32, T, "temperature"))
    if bias is not None:
        adj.bias, adj.bias_ld = _shared_rows(bias, torch.float32, T, V, "bias")
    if allowed is not None:
        adj.allowed, adj.allowed_ld = _shared_rows(allowed, torch.int32, T, (V + 31) // 32, "allowed")
    return adj


def _shared_rows(t, dtype, T, width, name):
    """(pointer, row stride) of [T, width], or of one [width] row for all (stride 0; also a row expanded to [T, width])."""
    assert t.is_cuda and t.dtype == dtype and t.stride(-1) == 1 and t.shape[-1] == width, f"{name}: need {dtype}[..., {width}] on GPU"
    if t.dim() == 1:
        return t.data_ptr(), 0
    assert t.dim() == 2 and t.shape[0] == T, f"{name}: need one row, or one for each of the {T}"
    return t.data_ptr(), t.stride(0) if T > 1 else 0


def adjust_logits(logits, V=None, *, history=None, hist_start=None, hist_len=None, prompt_len=None, repetition=None,
                  frequency=None, presence=None, temperature=None, bias=None, allowed=None, chosen=None, out=None,
                  out_dtype=None, write=True, want_lse=True, workspace=None):
    """a3po_adjust_logits -> dict(out | None, lse[T] f32 | None, logp[T] f32 | None, workspace).

    history int32 [tokens], hist_start int64 [T], hist_len / prompt_len int32 [T]; repetition, frequency, presence,
    temperature float32 [T]; bias float32 [V] or [T, V]; allowed int32 [ceil(V/32)] or [T, ceil(V/32)] bits.  The adjusted
    logits go to ``out`` (may be ``logits`` itself) or to a new tensor of ``out_dtype`` (logits' by default); ``write=False``
    computes lse and, with ``chosen``, the log-probs alone."""
    torch = _torch()
    dt, T, V, ld = _logits_meta(logits, V)
    dev = logits.device
    adj = _adjustments(T, V, history, hist_start, hist_len, prompt_len, repetition, frequency, presence, temperature, bias,
                       allowed)
    od, ld_out = dt, 0
    if not write:
        out = None
    else:
        if out is None:
            out = torch.empty((T, V), dtype=logits.dtype if out_dtype is None else out_dtype, device=dev)
        od, ld_out = _rows(out, "out")
        assert out.shape[0] == T and out.shape[1] >= V, f"out: need [{T}, {V}]"
    lse = torch.empty(T, dtype=torch.float32, device=dev) if want_lse else None
    logp = None
    if chosen is not None:
        _vec(chosen, torch.int32, T, "chosen")
        logp = torch.empty(T, dtype=torch.float32, device=dev)
    if workspace is None and (lse is not None or logp is not None):
        workspace = torch.empty(workspace_bytes(T, V, which=A3PO_WS_ADJUST_LOGITS), dtype=torch.uint8, device=dev)
    _check(lib().a3po_adjust_logits(_ptr(logits), dt, T, V, ld, ctypes.byref(adj), _ptr(chosen), _ptr(out), od, ld_out,
                                    _ptr(lse), _ptr(logp), _ptr(workspace), 0 if workspace is None else workspace.numel(),
                                    _stream()), "a3po_adjust_logits")
    return dict(out=out, lse=lse, logp=logp, workspace=workspace)


def adjust_logits_bwd(dout, logits=None, V=None, *, history=None, hist_start=None, hist_len=None, prompt_len=None,
                      repetition=None, frequency=None, presence=None, temperature=None, bias=None, allowed=None,
                      dlogits=None, dtype=None):
    """a3po_adjust_logits_bwd -> dlogits: ``dlogits`` itself (may be ``dout``), or a new tensor of ``dtype`` (logits', or
    dout's without logits).  The adjustments are those of the forward call; logits are needed with history and repetition."""
    torch = _torch()
    od, T, V, ld_out = _logits_meta(dout, V)
    adj = _adjustments(T, V, history, hist_start, hist_len, prompt_len, repetition, frequency, presence, temperature, bias,
                       allowed)
    ld = V
    if logits is not None:
        zd, zT, _, ld = _logits_meta(logits, V)
        assert zT == T and logits.shape[1] >= V, f"logits: need [{T}, {V}]"
    if dlogits is None:
        dtype = dtype if dtype is not None else dout.dtype if logits is None else logits.dtype
        dlogits = torch.empty((T, V), dtype=dtype, device=dout.device)
    dd, ld_d = _rows(dlogits, "dlogits")
    assert dlogits.shape[0] == T and dlogits.shape[1] >= V, f"dlogits: need [{T}, {V}]"
    assert logits is None or dd == zd, "dlogits must have logits' dtype"
    _check(lib().a3po_adjust_logits_bwd(_ptr(dout), od, ld_out, _ptr(logits), dd, T, V, ld, ctypes.byref(adj), _ptr(dlogits),
                                        ld_d, _stream()), "a3po_adjust_logits_bwd")
    return dlogits


def w4_linear(x, codes, scales, zeros=None, group: int = 128, out=None, out_dtype=None, workspace=None):
    """a3po_w4_linear -> out[T, N] (``out``, or a new tensor of ``out_dtype``, bfloat16 by default).  x bfloat16 [T, H];
    codes uint8 [N, H/2] (low half: even k); scales bfloat16 or float32 [N, H/group]; zeros uint8 [N, H/group] or None (8)."""
    torch = _torch()
    assert x.dtype == torch.bfloat16, "x must be bfloat16"
    ldx = _rows(x, "x")[1]
    T, H = x.shape
    N = codes.shape[0]
    assert group in (32, 64, 128) and H % group == 0, "group must be 32, 64 or 128 and divide H"
    _matrix(codes, torch.uint8, (N, H // 2), "codes")
    _matrix(scales, scales.dtype, (N, H // group), "scales")
    if zeros is not None:
        _matrix(zeros, torch.uint8, (N, H // group), "zeros")
    if out is None:
        out = torch.empty((T, N), dtype=torch.bfloat16 if out_dtype is None else out_dtype, device=x.device)
    od, ld_out = _rows(out, "out", (T, N))
    if workspace is None:
        need = workspace_bytes(T, 0, H, which=A3PO_WS_W4_LINEAR)
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
    _check(lib().a3po_w4_linear(_ptr(x), T, H, ldx, _ptr(codes), _ptr(scales), _dtype_code(scales, "scales"), _ptr(zeros),
                                int(group), N, _ptr(out), od, ld_out, _ptr(workspace), 0 if workspace is None else workspace.numel(),
                                _stream()), "a3po_w4_linear")
    return out


# ---- operators that close the loop -----------------------------------------------------------------------------------


def _here(*tensors):
    """Calls go to the current device's current stream: tensors of another device are refused."""
    now = None
    for t in tensors:
        if t is None:
            continue
        at = t.get_device()  # (-1: none)
        if now is None and at >= 0:
            now = _torch()._C._cuda_getDevice()
        if at != now:
            raise ValueError(f"a tensor on {t.device}, but calls go to the current device" + ("" if now is None else f", cuda:{now}"))


def sample(logits, uniform, V=None, *, temperature=None, top_k=None, top_p=None, min_p=None, want_logp=True,
           want_logp_full=False, want_kept=False, want_allowed=False, workspace=None):
    """a3po_sample -> dict(token int32[T], logp, logp_full float32[T] | None, kept int32[T] | None, allowed int32[T, ceil(V/32)]
    | None, workspace | None).

    A token of each row, drawn by the row's number of ``uniform`` float32 [T] from what temperature, top_k, top_p and min_p
    ([T], float32 but for top_k, int32) leave of it; logp is the log-prob under that cut policy, logp_full under the uncut one.
    ``allowed`` holds the kept entries as adjust_logits takes them: training on the tokens then sees the policy they came from."""
    torch = _torch()
    dt, T, V, ld = _logits_meta(logits, V)
    dev = logits.device
    assert logits.shape[1] >= V, f"logits: need [{T}, {V}]"
    policy = Sampling()
    policy.uniform = _ptr(_vec(uniform, torch.float32, T, "uniform"))
    if temperature is not None:
        policy.temperature = _ptr(_vec(temperature, torch.float32, T, "temperature"))
    if top_k is not None:
        policy.top_k = _ptr(_vec(top_k, torch.int32, T, "top_k"))
    if top_p is not None:
        policy.top_p = _ptr(_vec(top_p, torch.float32, T, "top_p"))
    if min_p is not None:
        policy.min_p = _ptr(_vec(min_p, torch.float32, T, "min_p"))
    _here(logits, uniform, temperature, top_k, top_p, min_p, workspace)
    token = torch.empty(T, dtype=torch.int32, device=dev)
    logp = torch.empty(T, dtype=torch.float32, device=dev) if want_logp else None
    full = torch.empty(T, dtype=torch.float32, device=dev) if want_logp_full else None
    kept = torch.empty(T, dtype=torch.int32, device=dev) if want_kept else None
    words = (V + 31) // 32
    allowed = torch.empty((T, words), dtype=torch.int32, device=dev) if want_allowed else None
    if workspace is None:
        need = workspace_bytes(T, V, which=A3PO_WS_SAMPLE)
        workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _check(lib().a3po_sample(_ptr(logits), dt, T, V, ld, ctypes.byref(policy), _ptr(token), _ptr(logp), _ptr(full), _ptr(kept),
                             _ptr(allowed), words, _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream()),
           "a3po_sample")
    return dict(token=token, logp=logp, logp_full=full, kept=kept, allowed=allowed, workspace=workspace)


_tensor_list_fn = None


def _tensor_list():
    """a3po_tensor_list (csrc/a3po_tensors.cpp): it holds the interpreter's lock and reads Python's objects."""
    global _tensor_list_fn
    if _tensor_list_fn is None:
        _torch()
        path = os.path.join(_PKG, "a3po_tensors.so")
        if not os.path.exists(path):
            raise FileNotFoundError(f"{path} is missing: build it with `python -m paper_2512_06547_amd.build`")
        fn = ctypes.PyDLL(path).a3po_tensor_list
        fn.restype, fn.argtypes = _I64, [ctypes.py_object, _I64, _P, _P, _P]
        _tensor_list_fn = fn
    return _tensor_list_fn


def _device_of(t) -> int:
    _here(t)
    return t.get_device()


def _pointers(tensors, dtype, count, want, address, size, name, device):
    """Writes addresses (and sizes) of a list's tensors to int64 arrays, which are given by their own addresses: tensors that are all
    contiguous, of one dtype and the sizes ``want`` (0: any), on the GPU ``device``."""
    assert len(tensors) == count, f"{name}: need one for each parameter"
    right = _tensor_list()(tensors, device, want, address, size)
    if right == count and (not count or tensors[0].dtype == dtype):
        return
    right %= count
    t = tensors[0] if tensors[0].dtype != dtype else tensors[right]
    if isinstance(t, _torch().Tensor):
        _here(t)
    n = ctypes.c_int64.from_address(want + 8 * right).value if want else "n"
    raise AssertionError(f"{name}[{right}]: need contiguous {dtype}[{n}] on GPU")


def grad_norm(grads, scale: float = 1.0, out=None, workspace=None):
    """a3po_grad_norm -> norm float32 [1] (``out``, or a new tensor): the 2-norm of all gradients times ``scale`` together."""
    torch = _torch()
    grads = list(grads)
    count = len(grads)
    columns = (ctypes.c_int64 * (2 * count))()  # addresses, sizes
    at = ctypes.addressof(columns)
    dt = A3PO_F32
    if count:
        dt, device = _dtype_code(grads[0], "grads"), _device_of(grads[0])
        _pointers(grads, grads[0].dtype, count, 0, at, at + 8 * count, "grads", device)
    if out is None:
        out = torch.empty(1, dtype=torch.float32, device=grads[0].device if count else "cuda")
    else:
        _vec(out, torch.float32, 1, "out")
        _here(out)
    if workspace is None:
        if count:
            workspace = torch.empty(workspace_bytes(count, which=A3PO_WS_GRAD_NORM), dtype=torch.uint8, device=out.device)
    else:
        _here(workspace)
    _check(lib().a3po_grad_norm(at, at + 8 * count, count, dt, float(scale), _ptr(out), _ptr(workspace),
                                0 if workspace is None else workspace.numel(), _stream()), "a3po_grad_norm")
    return out


def adamw_state(param, bits: int = 32):
    """(exp_avg, exp_avg_sq, scales) of zeros for a parameter: float32 of its size and None, or with ``bits`` 8 float8_e4m3fn,
    float8_e5m2 and the pair of uint8 exponents that blocks of 32 elements share."""
    torch = _torch()
    if bits == 32:
        return torch.zeros_like(param, dtype=torch.float32), torch.zeros_like(param, dtype=torch.float32), None
    if bits != 8:
        raise ValueError("states have 32 bits or 8")
    zero = lambda n: torch.zeros(n, dtype=torch.uint8, device=param.device)
    return (zero(param.shape).view(torch.float8_e4m3fn), zero(param.shape).view(torch.float8_e5m2),
            (zero((param.numel() + 31) // 32), zero((param.numel() + 31) // 32)))


def adamw_state_values(state, scale):
    """The float32 values that an 8-bit state stands for (for checkpoints and inspection; elementary torch operations)."""
    torch = _torch()
    unit = (scale.to(torch.int32) << 23).view(torch.float32).repeat_interleave(32)[:state.numel()]
    return (state.float().view(-1) * unit).view(state.shape)


def adamw_step(params, grads, exp_avgs, exp_avg_sqs, *, step, lr, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
               weight_decay: float = 0.0, scales=None, copies=None, norm=None, max_norm: float = 1.0, seed: int | None = None):
    """a3po_adamw_step: one step for every tensor of the list ``params``, in place, with the states that adamw_state made
    (``scales``: their pairs, with 8-bit states) and, where ``copies`` are given, the updated parameters rounded to bfloat16.

    ``step`` (from 1 on) and ``lr`` are numbers, or CUDA tensors of one int64 and one float32 where a captured graph is to see
    them change.  ``norm``: what grad_norm left; gradients are scaled to ``max_norm`` at most, and a step whose norm is not
    finite changes nothing.  ``seed``: of the roundings by chance (bfloat16 parameters, 8-bit exp_avg_sq), another each step: with the
    same one, what a step takes from exp_avg_sq is lost at the same elements every time.  By default it is the step's number (a step
    on the device enters the random bits by itself)."""
    torch = _torch()
    params, grads = list(params), list(grads)
    count = len(params)
    columns = np.zeros((8, count), dtype=np.int64)  # of the fields of a3po_adamw_tensor
    at = columns.ctypes.data
    pd = gd = device = 0
    if count and grads:
        pd, gd, device = _dtype_code(params[0], "params"), _dtype_code(grads[0], "grads"), _device_of(params[0])
    field = lambda i: at + 8 * count * i
    sizes = field(7)
    put = lambda i, tensors, dtype, name, want=sizes: _pointers(tensors, dtype, count, want, field(i), 0, name, device)
    _pointers(params, params[0].dtype if count else None, count, 0, at, sizes, "params", device)
    put(1, grads, grads[0].dtype if grads else None, "grads")
    bytes_ = scales is not None
    put(2, list(exp_avgs), torch.float8_e4m3fn if bytes_ else torch.float32, "exp_avgs")
    put(3, list(exp_avg_sqs), torch.float8_e5m2 if bytes_ else torch.float32, "exp_avg_sqs")
    if bytes_:
        scales, blocks = list(scales), (columns[7] + 31) // 32
        for i in (0, 1):
            put(4 + i, [s[i] for s in scales], torch.uint8, "scales", blocks.ctypes.data)
    if copies is not None:
        copies = list(copies)
        put(6, copies, torch.bfloat16, "copies")
    table = np.ascontiguousarray(columns.T)
    if seed is None:
        seed = 0 if isinstance(step, torch.Tensor) else int(step)
    opt = AdamwOptions(beta1=beta1, beta2=beta2, eps=eps, weight_decay=weight_decay, max_norm=max_norm, seed=int(seed) & 0xFFFFFFFF)
    if isinstance(step, torch.Tensor):
        opt.step_dev = _ptr(_vec(step, torch.int64, 1, "step"))
        _here(step)
    else:
        opt.step = int(step)
    if isinstance(lr, torch.Tensor):
        opt.lr_dev = _ptr(_vec(lr, torch.float32, 1, "lr"))
        _here(lr)
    else:
        opt.lr = float(lr)
    if norm is not None:
        opt.norm = _ptr(_vec(norm, torch.float32, 1, "norm"))
        _here(norm)
    _check(lib().a3po_adamw_step(table.ctypes.data, count, pd, gd, A3PO_STATE_8BIT if bytes_ else A3PO_STATE_F32, ctypes.byref(opt), _stream()),
           "a3po_adamw_step")
    torch._C._increment_version(params if copies is None else params + copies)  # (autograd may have kept what these held)


def w4_quantize(weight, group: int = 128, scale_dtype=None, zeros: bool = False):
    """a3po_w4_quantize -> (codes uint8 [N, H/2], scales [N, H/group] of ``scale_dtype`` (float32 by default), zeros uint8
    [N, H/group] or None), as w4_linear takes them: the 4-bit layout of weight [N, H]."""
    torch = _torch()
    dt, ld = _rows(weight, "weight")
    N, H = weight.shape
    assert group in (32, 64, 128) and H % group == 0, "group must be 32, 64 or 128 and divide H"
    _here(weight)
    dev = weight.device
    codes = torch.empty((N, H // 2), dtype=torch.uint8, device=dev)
    scales = torch.empty((N, H // group), dtype=torch.float32 if scale_dtype is None else scale_dtype, device=dev)
    zero = torch.empty((N, H // group), dtype=torch.uint8, device=dev) if zeros else None
    _check(lib().a3po_w4_quantize(_ptr(weight), dt, N, H, ld, int(group), _ptr(codes), _ptr(scales),
                                  _dtype_code(scales, "scales"), _ptr(zero), _stream()), "a3po_w4_quantize")
    return codes, scales, zero



def stats_to_dict(stats_tensor) -> dict:
    """Copies a device a3po_stats to the host (synchronises) and decodes it."""
    rec = np.frombuffer(stats_tensor.cpu().numpy().tobytes(), dtype=STATS_DTYPE)[0]
    return {k: rec[k].item() for k in STATS_DTYPE.names}
