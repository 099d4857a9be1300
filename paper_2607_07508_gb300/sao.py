"""Thin Python binding of libsao (include/sao.h), argument marshalling only.

Every function here has the name of the C entry point it calls, takes torch
tensors that already live on the current CUDA device, checks their dtypes and
shapes, and passes raw device pointers and the current CUDA stream to the
library. All arithmetic happens in libsao's CUDA kernels; if the library is
missing the import of this module's functions raises, there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsao.so")

SAO_F32, SAO_BF16 = 0, 1
SAO_STEP_AVERAGE, SAO_STEP_LAST = 0, 1
SAO_NORM_TOKEN, SAO_NORM_SEQUENCE = 0, 1
SAO_SCORE_SOFTMAX, SAO_SCORE_SIGMOID = 0, 1
SAO_GROUP_MAX, SAO_GROUP_TOP2 = 0, 1
SAO_ROUTE_MAX_EXPERTS, SAO_ROUTE_MAX_K, SAO_ROUTE_MAX_GROUPS = 1024, 32, 32
SAO_SCALE_NONE, SAO_SCALE_ROW, SAO_SCALE_BLOCK128, SAO_SCALE_MX32 = 0, 1, 2, 3
SAO_NORM_MAX_H = 16384
SAO_DISTILL_MAX_K, SAO_BALANCE_MAX_EXPERTS = 1024, 1024
STATUS = {0: "SAO_OK", 1: "SAO_ERR_INVALID_ARG", 2: "SAO_ERR_SHAPE", 3: "SAO_ERR_WORKSPACE",
          4: "SAO_ERR_UNSUPPORTED", 5: "SAO_ERR_CUDA", 6: "SAO_ERR_DEVICE_CHECK"}
FLAG_IN, FLAG_LOW, FLAG_HIGH, FLAG_NONFINITE, FLAG_NOT_ACTION = 0, 1, 2, 3, 4
FLAG_MISMATCH_LOW, FLAG_MISMATCH_HIGH = 5, 6

EXPORTS = ("sao_version", "sao_last_error_string", "sao_set_checked", "sao_get_checked",
           "sao_set_dz_budget_bytes", "sao_get_dz_budget_bytes", "sao_set_cta_pairs", "sao_get_cta_pairs",
           "sao_debug_set_scan_hooks", "sao_workspace_bytes", "sao_token_logprobs_fwd",
           "sao_token_logprobs_bwd", "sao_advantages", "sao_advantages_noalloc", "sao_step_advantages",
           "sao_policy_loss_fwd", "sao_policy_loss_bwd", "sao_clip_loss_fwd", "sao_clip_loss_bwd",
           "sao_group_advantages", "sao_running_mean_advantages", "sao_decoupled_loss_fwd",
           "sao_decoupled_loss_bwd", "sao_logprob_cache_bytes", "sao_token_logprobs_fwd_cached",
           "sao_token_logprobs_bwd_cached",
           "sao_distill_workspace_bytes", "sao_distill_loss_fwd", "sao_distill_loss_bwd",
           "sao_balance_workspace_bytes", "sao_balance_loss_fwd", "sao_balance_loss_bwd",
           "sao_route_workspace_bytes", "sao_route_fwd", "sao_route_bwd",
           "sao_norm_workspace_bytes", "sao_rms_norm_fwd", "sao_rms_norm_bwd",
           "sao_grad_workspace_bytes", "sao_grad_sumsq", "sao_grad_clip",
           "sao_value_loss", "sao_profile_enable", "sao_profile_reset", "sao_profile_read")


class SaoError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


_lib = None


def load(path: Optional[str] = None):
    """Load libsao.so (building it first if absent) and declare its signatures."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or LIB_PATH
    if not os.path.exists(path):
        from . import build as _build
        _build.build()
    L = ctypes.CDLL(path)
    P, I64, I32, F, SZ = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
    sig = {
        "sao_version": (ctypes.c_int, []),
        "sao_last_error_string": (ctypes.c_char_p, []),
        "sao_set_checked": (None, [ctypes.c_int]),
        "sao_get_checked": (ctypes.c_int, []),
        "sao_set_dz_budget_bytes": (None, [SZ]),
        "sao_get_dz_budget_bytes": (SZ, []),
        "sao_set_cta_pairs": (None, [ctypes.c_int]),
        "sao_get_cta_pairs": (ctypes.c_int, []),
        "sao_debug_set_scan_hooks": (None, [ctypes.c_uint64, I32]),
        "sao_workspace_bytes": (SZ, [I64, I32, I32, ctypes.c_int]),
        "sao_logprob_cache_bytes": (SZ, [I64, I32]),
        "sao_token_logprobs_fwd_cached": (ctypes.c_int, [P, P, ctypes.c_int, P, P, I64, I32, I32, P, P, P, SZ, P,
                                                         SZ, P]),
        "sao_token_logprobs_bwd_cached": (ctypes.c_int, [P, P, ctypes.c_int, P, P, P, I64, I32, I32, P, P,
                                                         ctypes.c_int, P, SZ, P, SZ, P]),
        "sao_token_logprobs_fwd": (ctypes.c_int, [P, P, ctypes.c_int, P, P, I64, I32, I32, P, P, P, SZ, P]),
        "sao_token_logprobs_bwd": (ctypes.c_int, [P, P, ctypes.c_int, P, P, P, I64, I32, I32, P, P,
                                                  ctypes.c_int, P, SZ, P]),
        "sao_advantages": (ctypes.c_int, [P, P, P, P, I32, I64, F, F, F, F, P, P, P, SZ, P]),
        "sao_advantages_noalloc": (ctypes.c_int, [P, P, P, P, I32, I64, F, F, F, F, P, P, P]),
        "sao_step_advantages": (ctypes.c_int, [P, P, P, P, I32, I64, F, F, F, F, ctypes.c_int, P, P, P, P, SZ, P]),
        "sao_policy_loss_fwd": (ctypes.c_int, [P, P, P, P, I64, F, F, I64, P, P, P, P, P, SZ, P]),
        "sao_policy_loss_bwd": (ctypes.c_int, [P, P, P, P, I64, F, F, I64, P, P, P, SZ, P]),
        "sao_decoupled_loss_fwd": (ctypes.c_int, [P, P, P, P, P, I64, F, F, F, F, I64, P, P, P, P, P, SZ, P]),
        "sao_decoupled_loss_bwd": (ctypes.c_int, [P, P, P, P, P, I64, F, F, F, F, I64, P, P, P, SZ, P]),
        "sao_value_loss": (ctypes.c_int, [P, P, P, I64, I64, P, P, P, P, SZ, P]),
        "sao_clip_loss_fwd": (ctypes.c_int, [P, P, P, P, P, I32, I64, F, F, ctypes.c_int, P, P, P, P, P, SZ, P]),
        "sao_clip_loss_bwd": (ctypes.c_int, [P, P, P, P, P, I32, I64, F, F, ctypes.c_int, P, P, P, SZ, P]),
        "sao_group_advantages": (ctypes.c_int, [P, P, I32, P, P, I64, F, P, P, SZ, P]),
        "sao_running_mean_advantages": (ctypes.c_int, [P, P, I32, I32, P, P, I32, P, P, I64, P, P, SZ, P]),
        "sao_distill_workspace_bytes": (SZ, [I64, I32, I32, I32, ctypes.c_int]),
        "sao_distill_loss_fwd": (ctypes.c_int, [P, P, ctypes.c_int, P, P, ctypes.c_int, P, P, I64, I32, I32, I32, F, P,
                                                P, P, P, P, SZ, P]),
        "sao_distill_loss_bwd": (ctypes.c_int, [P, P, ctypes.c_int, P, P, ctypes.c_int, P, P, P, P, P, I64, I32, I32,
                                                I32, F, P, P, ctypes.c_int, ctypes.c_int, P, SZ, P]),
        "sao_balance_workspace_bytes": (SZ, [I64, I32, I32]),
        "sao_balance_loss_fwd": (ctypes.c_int, [P, ctypes.c_int, P, P, P, I32, I64, I32, I32, ctypes.c_int, P, P, P, P,
                                                P, SZ, P]),
        "sao_balance_loss_bwd": (ctypes.c_int, [P, ctypes.c_int, P, P, I32, I64, I32, I32, ctypes.c_int, P, P, P, P, P,
                                                SZ, P]),
        "sao_route_workspace_bytes": (SZ, [I64, I32]),
        "sao_route_fwd": (ctypes.c_int, [P, ctypes.c_int, P, P, I64, I32, I32, ctypes.c_int, I32, I32, ctypes.c_int,
                                         ctypes.c_int, F, ctypes.c_int, P, P, P, SZ, P]),
        "sao_route_bwd": (ctypes.c_int, [P, ctypes.c_int, P, I64, I32, I32, ctypes.c_int, ctypes.c_int, F, P, P, P, P,
                                         ctypes.c_int, P, SZ, P]),
        "sao_norm_workspace_bytes": (SZ, [I64, I32]),
        "sao_rms_norm_fwd": (ctypes.c_int, [P, P, ctypes.c_int, P, ctypes.c_int, F, I64, I32, P, P, P, P, P,
                                            ctypes.c_int, P, SZ, P]),
        "sao_rms_norm_bwd": (ctypes.c_int, [P, ctypes.c_int, P, ctypes.c_int, P, P, P, I64, I32, P, P, ctypes.c_int, P,
                                            SZ, P]),
        "sao_grad_workspace_bytes": (SZ, []),
        "sao_grad_sumsq": (ctypes.c_int, [P, I32, P, P, SZ, P]),
        "sao_grad_clip": (ctypes.c_int, [P, P, I32, P, F, P, P, P, SZ, P]),
        "sao_profile_enable": (None, [ctypes.c_int]),
        "sao_profile_reset": (None, []),
        "sao_profile_read": (ctypes.c_int, [P, P, P, ctypes.c_int]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


def _check(status: int):
    if status != 0:
        raise SaoError(status, load().sao_last_error_string().decode())


# A call on 65,536 tokens takes the GPU 6-14 us, and checking and converting ten
# arguments took the host about as long, so each tensor is looked at once, by one
# function, and pointers go to ctypes as plain integers.

def _ptr(t: torch.Tensor) -> int:
    """Device pointer of a tensor whose type and size the caller has looked at."""
    if not t.is_cuda:
        raise ValueError("libsao takes CUDA tensors")
    if not t.is_contiguous():
        raise ValueError("libsao takes contiguous tensors")
    return t.data_ptr()


def _arg(t: Optional[torch.Tensor], dtype, n: int, name: str) -> Optional[int]:
    """Device pointer of a tensor that has to hold n elements of `dtype` (None: NULL)."""
    if t is None:
        return None
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.numel() != n:
        raise ValueError(f"{name} must have {n} elements, got {t.numel()}")
    if not t.is_cuda:
        raise ValueError("libsao takes CUDA tensors")
    if n != 1 and not t.is_contiguous():
        raise ValueError("libsao takes contiguous tensors")
    return t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        return _raw_stream(_device())
    return stream.cuda_stream


def _current_device_stream(device: int) -> int:
    return torch.cuda.current_stream(device).cuda_stream


# the current device and its current stream's handle, without a Stream object
# (PyTorch builds without CUDA lack both names)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _current_device_stream)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype is _BF16:
        return SAO_BF16
    if t.dtype is _F32:
        return SAO_F32
    raise ValueError(f"bf16 or fp32 expected, got {t.dtype}")


_F32, _F64, _BF16 = torch.float32, torch.float64, torch.bfloat16
_U8, _I32, _I64 = torch.uint8, torch.int32, torch.int64
_E4M3, _E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


# ---------------------------------------------------------------------------
# process settings
# ---------------------------------------------------------------------------

def sao_version() -> int:
    return load().sao_version()


def sao_set_checked(on: bool):
    load().sao_set_checked(1 if on else 0)


def sao_get_checked() -> bool:
    return bool(load().sao_get_checked())


def sao_set_dz_budget_bytes(nbytes: int):
    load().sao_set_dz_budget_bytes(int(nbytes))


def sao_get_dz_budget_bytes() -> int:
    return int(load().sao_get_dz_budget_bytes())


def sao_set_cta_pairs(on: bool):
    load().sao_set_cta_pairs(1 if on else 0)


def sao_get_cta_pairs() -> bool:
    return bool(load().sao_get_cta_pairs())


def sao_debug_set_scan_hooks(wait_ns: int = 0, skip_chunks: int = 0):
    """Test hooks of the advantage scan; (0, 0) restores the defaults."""
    load().sao_debug_set_scan_hooks(int(wait_ns), int(skip_chunks))


def sao_workspace_bytes(N: int, h: int = 0, V: int = 0, dtype=torch.bfloat16) -> int:
    code = SAO_BF16 if dtype == torch.bfloat16 else SAO_F32
    return int(load().sao_workspace_bytes(int(N), int(h), int(V), code))


def workspace(N: int, h: int = 0, V: int = 0, dtype=torch.bfloat16, device=None) -> torch.Tensor:
    """Allocate a workspace tensor (torch owns the memory; 256-byte aligned)."""
    n = sao_workspace_bytes(N, h, V, dtype)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device or "cuda")


# ---------------------------------------------------------------------------
# entry points
# ---------------------------------------------------------------------------

def _head(H, W):
    """(N, h, V) of H [N, h] and W [V, h] of one dtype."""
    N, h = H.shape
    V = W.shape[0]
    if W.shape[1] != h or W.dtype is not H.dtype:
        raise ValueError("W must be [V, h] with the dtype of H")
    return N, h, V


def _head_grads(H, W, dH, dW):
    N, h = H.shape
    V = W.shape[0]
    if W.shape[1] != h or W.dtype is not H.dtype or dH.dtype is not H.dtype or tuple(dH.shape) != (N, h):
        raise ValueError("W [V,h] and dH [N,h] must share the dtype of H")
    if dW.dtype is not _F32 or tuple(dW.shape) != (V, h):
        raise ValueError("dW must be fp32 [V, h]")
    return N, h, V


def sao_token_logprobs_fwd(H, W, y, logp, lse, ws, row_mask=None, stream=None):
    N, h, V = _head(H, W)
    _check(load().sao_token_logprobs_fwd(_ptr(H), _ptr(W), _dtype_code(H), _arg(y, _I32, N, "y"),
                                         _arg(row_mask, _U8, N, "row_mask"), N, h, V, _arg(logp, _F32, N, "logp"),
                                         _arg(lse, _F32, N, "lse"), _ptr(ws), ws.numel(), _stream(stream)))


def sao_token_logprobs_bwd(H, W, y, lse, grad_logp, dH, dW, ws, accumulate_dW=False, stream=None):
    N, h, V = _head_grads(H, W, dH, dW)
    _check(load().sao_token_logprobs_bwd(_ptr(H), _ptr(W), _dtype_code(H), _arg(y, _I32, N, "y"),
                                         _arg(lse, _F32, N, "lse"), _arg(grad_logp, _F32, N, "grad_logp"), N, h, V,
                                         _ptr(dH), _ptr(dW), 1 if accumulate_dW else 0, _ptr(ws), ws.numel(),
                                         _stream(stream)))


def sao_logprob_cache_bytes(N: int, V: int) -> int:
    return int(load().sao_logprob_cache_bytes(int(N), int(V)))


def logprob_cache(N: int, V: int, device=None) -> torch.Tensor:
    """Allocate the forward's probability cache (about 2*N*V bytes)."""
    return torch.empty(max(sao_logprob_cache_bytes(N, V), 256), dtype=torch.uint8, device=device or "cuda")


def sao_token_logprobs_fwd_cached(H, W, y, logp, lse, cache, ws, row_mask=None, stream=None):
    N, h, V = _head(H, W)
    _check(load().sao_token_logprobs_fwd_cached(_ptr(H), _ptr(W), _dtype_code(H), _arg(y, _I32, N, "y"),
                                                _arg(row_mask, _U8, N, "row_mask"), N, h, V,
                                                _arg(logp, _F32, N, "logp"), _arg(lse, _F32, N, "lse"), _ptr(cache),
                                                cache.numel(), _ptr(ws), ws.numel(), _stream(stream)))


def sao_token_logprobs_bwd_cached(H, W, y, lse, grad_logp, dH, dW, cache, ws, accumulate_dW=False, stream=None):
    N, h, V = _head_grads(H, W, dH, dW)
    _check(load().sao_token_logprobs_bwd_cached(_ptr(H), _ptr(W), _dtype_code(H), _arg(y, _I32, N, "y"),
                                                _arg(lse, _F32, N, "lse"), _arg(grad_logp, _F32, N, "grad_logp"), N,
                                                h, V, _ptr(dH), _ptr(dW), 1 if accumulate_dW else 0, _ptr(cache),
                                                cache.numel(), _ptr(ws), ws.numel(), _stream(stream)))


def sao_advantages(values, rewards, loss_mask, cu_seqlens, gamma, lambda_policy, lambda_critic,
                   len_adaptive_alpha, adv, ret, ws, stream=None):
    N = values.numel()
    B = cu_seqlens.numel() - 1
    _check(load().sao_advantages(_arg(values, _F32, N, "values"), _arg(rewards, _F32, B, "rewards"),
                                 _arg(loss_mask, _U8, N, "loss_mask"), _arg(cu_seqlens, _I32, B + 1, "cu_seqlens"),
                                 B, N, float(gamma), float(lambda_policy), float(lambda_critic),
                                 float(len_adaptive_alpha), _arg(adv, _F32, N, "adv"), _arg(ret, _F32, N, "ret"),
                                 _ptr(ws), ws.numel(), _stream(stream)))


def sao_step_advantages(values, rewards, loss_mask, cu_seqlens, gamma, lambda_policy, lambda_critic,
                        len_adaptive_alpha, mode, adv, ret, ws, value_mask=None, stream=None):
    N = values.numel()
    B = cu_seqlens.numel() - 1
    _check(load().sao_step_advantages(_arg(values, _F32, N, "values"), _arg(rewards, _F32, B, "rewards"),
                                      _arg(loss_mask, _U8, N, "loss_mask"),
                                      _arg(cu_seqlens, _I32, B + 1, "cu_seqlens"), B, N, float(gamma),
                                      float(lambda_policy), float(lambda_critic), float(len_adaptive_alpha),
                                      int(mode), _arg(adv, _F32, N, "adv"),
                                      _arg(ret, _F32, N, "ret"), _arg(value_mask, _U8, N, "value_mask"), _ptr(ws),
                                      ws.numel(), _stream(stream)))


def sao_advantages_noalloc(values, rewards, loss_mask, cu_seqlens, gamma, lambda_policy, lambda_critic,
                           len_adaptive_alpha, adv, ret, stream=None):
    """sao_advantages with the library's fixed device scratch instead of a
    workspace, for callers that cannot allocate device memory."""
    N = values.numel()
    B = cu_seqlens.numel() - 1
    _check(load().sao_advantages_noalloc(_arg(values, _F32, N, "values"), _arg(rewards, _F32, B, "rewards"),
                                         _arg(loss_mask, _U8, N, "loss_mask"),
                                         _arg(cu_seqlens, _I32, B + 1, "cu_seqlens"), B, N, float(gamma),
                                         float(lambda_policy), float(lambda_critic), float(len_adaptive_alpha),
                                         _arg(adv, _F32, N, "adv"),
                                         _arg(ret, _F32, N, "ret"), _stream(stream)))


def sao_policy_loss_fwd(logp, old_logp, adv, loss_mask, eps_low, eps_high, loss, counts, ws, coef=None,
                        flags=None, n_norm=0, stream=None):
    N = logp.numel()
    _check(load().sao_policy_loss_fwd(_arg(logp, _F32, N, "logp"), _arg(old_logp, _F32, N, "old_logp"),
                                      _arg(adv, _F32, N, "adv"), _arg(loss_mask, _U8, N, "loss_mask"), N,
                                      float(eps_low), float(eps_high), int(n_norm), _arg(loss, _F32, 1, "loss"),
                                      _arg(coef, _F32, N, "coef"), _arg(flags, _U8, N, "flags"),
                                      _arg(counts, _I64, 4, "counts"), _ptr(ws), ws.numel(), _stream(stream)))


def sao_policy_loss_bwd(logp, old_logp, adv, loss_mask, eps_low, eps_high, grad_loss, grad_logp, ws, n_norm=0,
                        stream=None):
    N = logp.numel()
    _check(load().sao_policy_loss_bwd(_arg(logp, _F32, N, "logp"), _arg(old_logp, _F32, N, "old_logp"),
                                      _arg(adv, _F32, N, "adv"), _arg(loss_mask, _U8, N, "loss_mask"), N,
                                      float(eps_low), float(eps_high), int(n_norm),
                                      _arg(grad_loss, _F32, 1, "grad_loss"),
                                      _arg(grad_logp, _F32, N, "grad_logp"), _ptr(ws), ws.numel(), _stream(stream)))


def sao_decoupled_loss_fwd(logp, prox_logp, rollout_logp, adv, loss_mask, eps_low, eps_high, w_low, w_high, loss,
                           counts, ws, coef=None, flags=None, n_norm=0, stream=None):
    N = logp.numel()
    _check(load().sao_decoupled_loss_fwd(_arg(logp, _F32, N, "logp"), _arg(prox_logp, _F32, N, "prox_logp"),
                                         _arg(rollout_logp, _F32, N, "rollout_logp"), _arg(adv, _F32, N, "adv"),
                                         _arg(loss_mask, _U8, N, "loss_mask"), N, float(eps_low), float(eps_high),
                                         float(w_low), float(w_high), int(n_norm), _arg(loss, _F32, 1, "loss"),
                                         _arg(coef, _F32, N, "coef"),
                                         _arg(flags, _U8, N, "flags"), _arg(counts, _I64, 6, "counts"), _ptr(ws),
                                         ws.numel(), _stream(stream)))


def sao_decoupled_loss_bwd(logp, prox_logp, rollout_logp, adv, loss_mask, eps_low, eps_high, w_low, w_high,
                           grad_loss, grad_logp, ws, n_norm=0, stream=None):
    N = logp.numel()
    _check(load().sao_decoupled_loss_bwd(_arg(logp, _F32, N, "logp"), _arg(prox_logp, _F32, N, "prox_logp"),
                                         _arg(rollout_logp, _F32, N, "rollout_logp"), _arg(adv, _F32, N, "adv"),
                                         _arg(loss_mask, _U8, N, "loss_mask"), N, float(eps_low), float(eps_high),
                                         float(w_low), float(w_high), int(n_norm),
                                         _arg(grad_loss, _F32, 1, "grad_loss"),
                                         _arg(grad_logp, _F32, N, "grad_logp"), _ptr(ws), ws.numel(),
                                         _stream(stream)))


def sao_value_loss(values, ret, loss_mask, loss, grad_values, ws, ev_sums=None, n_norm=0, stream=None):
    N = values.numel()
    _check(load().sao_value_loss(_arg(values, _F32, N, "values"), _arg(ret, _F32, N, "ret"),
                                 _arg(loss_mask, _U8, N, "loss_mask"), N, int(n_norm), _arg(loss, _F32, 1, "loss"),
                                 _arg(grad_values, _F32, N, "grad_values"), _arg(ev_sums, _F64, 4, "ev_sums"),
                                 _ptr(ws), ws.numel(), _stream(stream)))


def sao_clip_loss_fwd(logp, old_logp, adv, loss_mask, cu_seqlens, eps_low, eps_high, norm, loss, counts, ws,
                      coef=None, flags=None, stream=None):
    N = logp.numel()
    B = cu_seqlens.numel() - 1
    _check(load().sao_clip_loss_fwd(_arg(logp, _F32, N, "logp"), _arg(old_logp, _F32, N, "old_logp"),
                                    _arg(adv, _F32, N, "adv"), _arg(loss_mask, _U8, N, "loss_mask"),
                                    _arg(cu_seqlens, _I32, B + 1, "cu_seqlens"), B, N, float(eps_low),
                                    float(eps_high), int(norm),
                                    _arg(loss, _F32, 1, "loss"), _arg(coef, _F32, N, "coef"),
                                    _arg(flags, _U8, N, "flags"), _arg(counts, _I64, 4, "counts"), _ptr(ws),
                                    ws.numel(), _stream(stream)))


def sao_clip_loss_bwd(logp, old_logp, adv, loss_mask, cu_seqlens, eps_low, eps_high, norm, grad_loss, grad_logp, ws,
                      stream=None):
    N = logp.numel()
    B = cu_seqlens.numel() - 1
    _check(load().sao_clip_loss_bwd(_arg(logp, _F32, N, "logp"), _arg(old_logp, _F32, N, "old_logp"),
                                    _arg(adv, _F32, N, "adv"), _arg(loss_mask, _U8, N, "loss_mask"),
                                    _arg(cu_seqlens, _I32, B + 1, "cu_seqlens"), B, N, float(eps_low),
                                    float(eps_high), int(norm),
                                    _arg(grad_loss, _F32, 1, "grad_loss"), _arg(grad_logp, _F32, N, "grad_logp"),
                                    _ptr(ws), ws.numel(), _stream(stream)))


def sao_group_advantages(rewards, group_ids, loss_mask, cu_seqlens, eps_stab, adv, ws, stream=None):
    N = loss_mask.numel()
    B = cu_seqlens.numel() - 1
    _check(load().sao_group_advantages(_arg(rewards, _F32, B, "rewards"), _arg(group_ids, _I32, B, "group_ids"), B,
                                       _arg(loss_mask, _U8, N, "loss_mask"),
                                       _arg(cu_seqlens, _I32, B + 1, "cu_seqlens"), N, float(eps_stab),
                                       _arg(adv, _F32, N, "adv"), _ptr(ws), ws.numel(), _stream(stream)))


def sao_running_mean_advantages(rewards, prompt_ids, history, seen, loss_mask, cu_seqlens, adv, ws, stream=None):
    """history [P, window] fp32 and seen [P] int64 are updated in place."""
    N = loss_mask.numel()
    B = cu_seqlens.numel() - 1
    P, window = history.shape
    if history.dtype is not _F32:
        raise ValueError("history must be fp32")
    _check(load().sao_running_mean_advantages(_arg(rewards, _F32, B, "rewards"),
                                              _arg(prompt_ids, _I32, B, "prompt_ids"), B, P, _ptr(history),
                                              _arg(seen, _I64, P, "seen"), window,
                                              _arg(loss_mask, _U8, N, "loss_mask"),
                                              _arg(cu_seqlens, _I32, B + 1, "cu_seqlens"), N,
                                              _arg(adv, _F32, N, "adv"), _ptr(ws), ws.numel(), _stream(stream)))


def sao_distill_workspace_bytes(N: int, h: int, V: int, K: int, dtype=torch.bfloat16) -> int:
    code = SAO_BF16 if dtype == torch.bfloat16 else SAO_F32
    return int(load().sao_distill_workspace_bytes(int(N), int(h), int(V), int(K), code))


def distill_workspace(N: int, h: int, V: int, K: int, dtype=torch.bfloat16, device=None) -> torch.Tensor:
    """Allocate the workspace of sao_distill_loss_fwd/bwd for up to N rows."""
    n = sao_distill_workspace_bytes(N, h, V, K, dtype)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device or "cuda")


def _entries(top_ids, top_logits, N):
    """K of the teacher's entries [N, K] and the code of their logits' dtype."""
    if top_ids.dim() != 2 or top_ids.shape[0] != N or top_logits.shape != top_ids.shape:
        raise ValueError("top_ids and top_logits must be [N, K]")
    if top_logits.dtype is not _F32 and top_logits.dtype is not _BF16:
        raise ValueError(f"top_logits must be bf16 or fp32, got {top_logits.dtype}")
    return top_ids.shape[1], _dtype_code(top_logits)


def sao_distill_loss_fwd(H, W, top_ids, top_logits, temperature, loss, lse, lse_rest, z_top, ws, teacher_lse=None,
                         row_mask=None, stream=None):
    N, h, V = _head(H, W)
    K, code = _entries(top_ids, top_logits, N)
    _check(load().sao_distill_loss_fwd(_ptr(H), _ptr(W), _dtype_code(H), _arg(top_ids, _I32, N * K, "top_ids"),
                                       _ptr(top_logits), code, _arg(teacher_lse, _F32, N, "teacher_lse"),
                                       _arg(row_mask, _U8, N, "row_mask"), N, h, V, K, float(temperature),
                                       _arg(loss, _F32, N, "loss"), _arg(lse, _F32, N, "lse"),
                                       _arg(lse_rest, _F32, N, "lse_rest"), _arg(z_top, _F32, N * K, "z_top"),
                                       _ptr(ws), ws.numel(), _stream(stream)))


def sao_distill_loss_bwd(H, W, top_ids, top_logits, temperature, lse, lse_rest, z_top, grad_loss, dH, dW, ws,
                         teacher_lse=None, accumulate_dW=False, stream=None):
    """dW fp32, or bf16 for a bf16 head (overwritten only)."""
    N, h, V = _head(H, W)
    K, code = _entries(top_ids, top_logits, N)
    if dH.dtype is not H.dtype or tuple(dH.shape) != (N, h):
        raise ValueError("dH must be [N, h] with the dtype of H")
    if tuple(dW.shape) != (V, h):
        raise ValueError("dW must be [V, h]")
    _check(load().sao_distill_loss_bwd(_ptr(H), _ptr(W), _dtype_code(H), _arg(top_ids, _I32, N * K, "top_ids"),
                                       _ptr(top_logits), code, _arg(teacher_lse, _F32, N, "teacher_lse"),
                                       _arg(lse, _F32, N, "lse"), _arg(lse_rest, _F32, N, "lse_rest"),
                                       _arg(z_top, _F32, N * K, "z_top"), _arg(grad_loss, _F32, N, "grad_loss"), N, h,
                                       V, K, float(temperature), _ptr(dH), _ptr(dW), _dtype_code(dW),
                                       1 if accumulate_dW else 0, _ptr(ws), ws.numel(), _stream(stream)))


def sao_balance_workspace_bytes(N: int, E: int, B: int = 1) -> int:
    return int(load().sao_balance_workspace_bytes(int(N), int(E), int(B)))


def balance_workspace(N: int, E: int, B: int = 1, device=None) -> torch.Tensor:
    """Allocate the workspace of sao_balance_loss_fwd/bwd (B trajectories, or 1 for the batch)."""
    return torch.empty(max(sao_balance_workspace_bytes(N, E, B), 256), dtype=torch.uint8, device=device or "cuda")


def sao_balance_loss_fwd(logits, expert_ids, score, loss, counts, prob_sums, rows, ws, row_mask=None, cu_seqlens=None,
                         stream=None):
    N, E = logits.shape
    if expert_ids.dim() != 2 or expert_ids.shape[0] != N:
        raise ValueError("expert_ids must be [N, k]")
    k = expert_ids.shape[1]
    B = 1 if cu_seqlens is None else cu_seqlens.numel() - 1
    _check(load().sao_balance_loss_fwd(_ptr(logits), _dtype_code(logits), _arg(expert_ids, _I32, N * k, "expert_ids"),
                                       _arg(row_mask, _U8, N, "row_mask"),
                                       _arg(cu_seqlens, _I32, B + 1, "cu_seqlens"), B, N, E, k, int(score),
                                       _arg(loss, _F32, 1, "loss"), _arg(counts, _I64, B * E, "counts"),
                                       _arg(prob_sums, _F32, B * E, "prob_sums"), _arg(rows, _I64, B, "rows"),
                                       _ptr(ws), ws.numel(), _stream(stream)))


def sao_balance_loss_bwd(logits, k, score, counts, rows, grad_loss, grad_logits, ws, row_mask=None, cu_seqlens=None,
                         stream=None):
    """k: the experts chosen per token, as in the forward's expert_ids [N, k]."""
    N, E = logits.shape
    B = 1 if cu_seqlens is None else cu_seqlens.numel() - 1
    _check(load().sao_balance_loss_bwd(_ptr(logits), _dtype_code(logits), _arg(row_mask, _U8, N, "row_mask"),
                                       _arg(cu_seqlens, _I32, B + 1, "cu_seqlens"), B, N, E, int(k), int(score),
                                       _arg(counts, _I64, B * E, "counts"), _arg(rows, _I64, B, "rows"),
                                       _arg(grad_loss, _F32, 1, "grad_loss"),
                                       _arg(grad_logits, logits.dtype, N * E, "grad_logits"), _ptr(ws), ws.numel(),
                                       _stream(stream)))


def _current(device) -> None:
    if device is not None and device != _device():
        raise ValueError(f"the tensors lie on device {device}, the current one is {_device()}")


def _on_current(t: torch.Tensor) -> None:
    device = t.get_device()
    if device >= 0:  # (others are refused where their pointers are taken)
        _current(device)


def sao_route_workspace_bytes(N: int, E: int) -> int:
    return int(load().sao_route_workspace_bytes(int(N), int(E)))


def route_workspace(N: int, E: int, device=None) -> torch.Tensor:
    """Allocate the workspace of sao_route_fwd/bwd for up to N tokens and E experts."""
    return torch.empty(max(sao_route_workspace_bytes(N, E), 256), dtype=torch.uint8, device=device or "cuda")


def _router(logits, expert_ids):
    """(N, E, k)"""
    N, E = logits.shape
    if expert_ids.dim() != 2 or expert_ids.shape[0] != N:
        raise ValueError("expert_ids must be [N, k]")
    _on_current(logits)
    return N, E, expert_ids.shape[1]


def sao_route_fwd(logits, score, expert_ids, weights, ws, bias=None, row_mask=None, groups=1, groups_kept=1,
                  group_score=SAO_GROUP_MAX, renormalise=True, scale=1.0, replay=False, stream=None):
    """expert_ids [N, k] int32: written, or read with `replay`."""
    N, E, k = _router(logits, expert_ids)
    _check(load().sao_route_fwd(_ptr(logits), _dtype_code(logits), _arg(bias, _F32, E, "bias"),
                                _arg(row_mask, _U8, N, "row_mask"), N, E, k, int(score), int(groups), int(groups_kept),
                                int(group_score), 1 if renormalise else 0, float(scale), 1 if replay else 0,
                                _arg(expert_ids, _I32, N * k, "expert_ids"), _arg(weights, _F32, N * k, "weights"),
                                _ptr(ws), ws.numel(), _stream(stream)))


def sao_route_bwd(logits, score, expert_ids, weights, grad_weights, grad_logits, ws, row_mask=None, renormalise=True,
                  scale=1.0, accumulate=False, stream=None):
    """accumulate: added to grad_logits, which holds another loss's gradient."""
    N, E, k = _router(logits, expert_ids)
    _check(load().sao_route_bwd(_ptr(logits), _dtype_code(logits), _arg(row_mask, _U8, N, "row_mask"), N, E, k,
                                int(score), 1 if renormalise else 0, float(scale),
                                _arg(expert_ids, _I32, N * k, "expert_ids"), _arg(weights, _F32, N * k, "weights"),
                                _arg(grad_weights, _F32, N * k, "grad_weights"),
                                _arg(grad_logits, logits.dtype, N * E, "grad_logits"), 1 if accumulate else 0, _ptr(ws),
                                ws.numel(), _stream(stream)))


def sao_norm_workspace_bytes(N: int, h: int) -> int:
    return int(load().sao_norm_workspace_bytes(int(N), int(h)))


def norm_workspace(N: int, h: int, device=None) -> torch.Tensor:
    """Allocate the workspace of sao_rms_norm_fwd/bwd for up to N rows of up to h columns."""
    return torch.empty(max(sao_norm_workspace_bytes(N, h), 256), dtype=torch.uint8, device=device or "cuda")


_SCALINGS = {"none": (0, 0, (None,)), "row": (1, 0, (_F32,)), "block": (2, 128, (_F32,)), "mx": (3, 32, (_E8M0, _U8))}
_BYTES = (_E4M3, _U8)


def _scales(scaling, h):
    """(code, scales to a row, their types) of a scaling's name."""
    if scaling not in _SCALINGS:
        raise ValueError(f"scaling is one of {', '.join(_SCALINGS)}, got {scaling!r}")
    code, size, dtypes = _SCALINGS[scaling]
    return code, 1 if size == 0 else -(-h // size), dtypes


def _arg_of(t: Optional[torch.Tensor], dtypes, n: int, name: str) -> Optional[int]:
    """_arg of a tensor of any of `dtypes`."""
    if t is None:
        return None
    if t.dtype not in dtypes:
        raise ValueError(f"{name} must be {dtypes[0]}, got {t.dtype}")
    return _arg(t, t.dtype, n, name)


def norm_out8(N: int, h: int, scaling: str, device=None):
    """Allocate the 8-bit rows [N, h] (e4m3) and their scales of sao_rms_norm_fwd: [N, 1] fp32 for "row", [N, ceil(h /
    128)] fp32 for "block", [N, ceil(h / 32)] e8m0 for "mx"."""
    code, n, dtypes = _scales(scaling, h)
    if code == 0:
        raise ValueError("no 8-bit rows without a scaling")
    return (torch.empty(N, h, dtype=_E4M3, device=device or "cuda"),
            torch.empty(N, n, dtype=dtypes[0], device=device or "cuda"))


def _norm(x, weight):
    """(N, h, code of x, code of the weight)"""
    N, h = x.shape
    if weight.numel() != h:
        raise ValueError("x must be [N, h], weight [h]")
    _on_current(x)
    return N, h, _dtype_code(x), _dtype_code(weight)


def sao_rms_norm_fwd(x, weight, eps, ws, residual=None, sum=None, y=None, rstd=None, y8=None, scales=None,
                     scaling="none", stream=None):
    """y8, scales: of norm_out8, or uint8 tensors of their sizes."""
    N, h, code, w_code = _norm(x, weight)
    scale_code, n, dtypes = _scales(scaling, h)
    _check(load().sao_rms_norm_fwd(_ptr(x), _arg(residual, x.dtype, N * h, "residual"), code, _ptr(weight), w_code,
                                   float(eps), N, h, _arg(sum, x.dtype, N * h, "sum"), _arg(y, x.dtype, N * h, "y"),
                                   _arg(rstd, _F32, N, "rstd"), _arg_of(y8, _BYTES, N * h, "y8"),
                                   _arg_of(scales, dtypes, N * n, "scales"), scale_code, _ptr(ws), ws.numel(),
                                   _stream(stream)))


def sao_rms_norm_bwd(sum, weight, rstd, dy, dx, dweight, ws, dsum=None, accumulate=False, stream=None):
    """sum: the forward's (x without a residual); dsum: the gradient that reaches it past the norm; dweight or None."""
    N, h, code, w_code = _norm(sum, weight)
    _check(load().sao_rms_norm_bwd(_ptr(sum), code, _ptr(weight), w_code, _arg(rstd, _F32, N, "rstd"),
                                   _arg(dy, sum.dtype, N * h, "dy"), _arg(dsum, sum.dtype, N * h, "dsum"), N, h,
                                   _arg(dx, sum.dtype, N * h, "dx"), _arg(dweight, _F32, h, "dweight"),
                                   1 if accumulate else 0, _ptr(ws), ws.numel(), _stream(stream)))


class _Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("n", ctypes.c_int64), ("dt", ctypes.c_int)]


class _Tensors:
    """A list of tensors for one call."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        self.device = self.tensors[0].get_device() if self.tensors else None
        for t in self.tensors:
            if t.get_device() != self.device:
                raise ValueError("the tensors of a list lie on one device")
        self.array = (_Tensor * len(self.tensors))(*[(_ptr(t), t.numel(), _dtype_code(t)) for t in self.tensors])

    def __len__(self):
        return len(self.tensors)


class TensorList(_Tensors):
    """Gradients, or their clipped copies, as the calls below take them: made once for tensors that stay where
    they are, which it keeps alive, and their memory. A list of which a tensor has since moved to other memory is refused
    (ValueError): make another one."""

    def __init__(self, tensors):
        super().__init__(tensors)
        # the memory that the addresses are of: while it is held, no other tensor can come to lie there
        self._held = [t.detach() for t in self.tensors]
        self._place_of = [t.data_ptr for t in self.tensors]
        self._places = [place() for place in self._place_of]

    def check(self):
        if [place() for place in self._place_of] != self._places:
            raise ValueError("a tensor of the list has moved since the list was made")


def _listed(tensors) -> _Tensors:
    if not isinstance(tensors, TensorList):
        return _Tensors(tensors)
    tensors.check()
    return tensors


def sao_grad_workspace_bytes() -> int:
    return int(load().sao_grad_workspace_bytes())


def grad_workspace(device=None) -> torch.Tensor:
    """Allocate the workspace of sao_grad_sumsq and sao_grad_clip, whatever their lists."""
    return torch.empty(sao_grad_workspace_bytes(), dtype=torch.uint8, device=device or "cuda")


def sao_grad_sumsq(grads, sumsq, ws, stream=None):
    """grads: a TensorList, or tensors; sumsq fp64."""
    grads = _listed(grads)
    _current(grads.device)
    _check(load().sao_grad_sumsq(grads.array, len(grads), _arg(sumsq, _F64, 1, "sumsq"), _ptr(ws), ws.numel(),
                                 _stream(stream)))


def sao_grad_clip(grads, sumsq, max_norm, norm, coef, ws, out=None, stream=None):
    """grads, out: TensorLists, or tensors; out None: in place."""
    grads = _listed(grads)
    out = None if out is None else _listed(out)
    if out is not None and (len(out) != len(grads) or out.device != grads.device):
        raise ValueError("out must have a tensor for each of grads, on their device")
    _current(grads.device)
    _check(load().sao_grad_clip(grads.array, None if out is None else out.array, len(grads),
                                _arg(sumsq, _F64, 1, "sumsq"), float(max_norm), _arg(norm, _F32, 1, "norm"),
                                _arg(coef, _F32, 1, "coef"), _ptr(ws), ws.numel(), _stream(stream)))


# ---------------------------------------------------------------------------
# kernel timing
# ---------------------------------------------------------------------------

def sao_profile_enable(on: bool):
    load().sao_profile_enable(1 if on else 0)


def sao_profile_reset():
    load().sao_profile_reset()


def sao_profile_read(cap: int = 64):
    """{kernel name: (launches, total ms)} since the last reset."""
    names = (ctypes.c_char_p * cap)()
    launches = (ctypes.c_int64 * cap)()
    ms = (ctypes.c_double * cap)()
    n = load().sao_profile_read(ctypes.cast(names, ctypes.c_void_p), ctypes.cast(launches, ctypes.c_void_p),
                                ctypes.cast(ms, ctypes.c_void_p), cap)
    return {names[i].decode(): (int(launches[i]), float(ms[i])) for i in range(n)}
