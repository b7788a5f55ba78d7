"""Thin ctypes binding of the C ABI declared in include/hilore.h (argument marshalling only).

Every function has the name and the argument order of its C entry point; tensors are torch
CUDA tensors of which only ``data_ptr()`` is passed on, and the current torch CUDA stream is
used unless ``stream`` is given.  Nothing here computes: every step of the path runs in the
library's CUDA kernels.  If the shared library is missing the import fails loudly; there is
no CPU or PyTorch fallback.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

from . import build as _build

OK, INVALID_ARG, SHAPE, ALIGN, ZERO_NORM, CUDA, WORKSPACE = range(7)
FMT_E4M3FN_RAW, FMT_E4M3FN_BLK, FMT_INT8_BLK = 0, 1, 2
ACT_R, ACT_H, ACT_L = 0, 1, 2
PHASE_DECIDE, PHASE_CAPTURE, PHASE_ENCODE, PHASE_RECOVER = 0, 1, 2, 3
BLOCK = 64
BF16, F32 = 0, 1
STATE_F32, STATE_E4M3FN = 0, 1
PARAM_TILE = 1024
RATIO_TOKEN, RATIO_SEQUENCE = 0, 1
MEAN_TOKENS, MEAN_SEQUENCES = 0, 1
KL_K1, KL_K2, KL_K3 = 1, 2, 3
PREF_SIGMOID, PREF_HINGE, PREF_SQUARE = 0, 1, 2

EXPORTS = ("hilore_status_string", "hilore_abi_version", "hilore_mask_count", "hilore_grpo_coeffs",
           "hilore_unit_exposure", "hilore_workspace_bytes", "hilore_compress", "hilore_recover",
           "hilore_plan_apply", "hilore_unit_exposure_static", "hilore_static_scratch_bytes",
           "hilore_allocate", "hilore_allocate_workspace_bytes", "hilore_risk_budget",
           "hilore_relative_error", "hilore_relative_error_workspace_bytes", "hilore_fit_kappa",
           "hilore_grpo_coeffs_variant", "hilore_omega_diagnostics", "hilore_omega_diagnostics_workspace_bytes",
           "hilore_grpo_coeffs_packed", "hilore_unit_exposure_packed", "hilore_codec_relative_error",
           "hilore_coeffs_exposure", "hilore_scores_plan", "hilore_scores_plan_workspace_bytes",
           "hilore_logits_apply", "hilore_logits_apply_backward", "hilore_token_logp", "hilore_token_logp_backward",
           "hilore_grad_norm", "hilore_grad_norm_workspace_bytes", "hilore_adamw_step",
           "hilore_advantages", "hilore_advantages_backward", "hilore_advantages_workspace_bytes", "hilore_policy_loss",
           "hilore_policy_loss_workspace_bytes", "hilore_preference_loss", "hilore_preference_loss_workspace_bytes")


class HiloreUnit(C.Structure):
    """Mirror of ``struct hilore_unit``."""
    _fields_ = [("x", C.c_void_p), ("codes", C.c_void_p), ("scales", C.c_void_p), ("out", C.c_void_p),
                ("row_rms", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64),
                ("fmt", C.c_int32), ("block", C.c_int32)]


class HiloreLogitRules(C.Structure):
    """Mirror of ``struct hilore_logit_rules``."""
    _fields_ = [("temperature", C.c_void_p), ("repetition", C.c_void_p), ("frequency", C.c_void_p), ("presence", C.c_void_p),
                ("tokens", C.c_void_p), ("n_tokens", C.c_int64), ("hist_begin", C.c_void_p), ("resp_begin", C.c_void_p),
                ("hist_end", C.c_void_p), ("bias_tokens", C.c_void_p), ("bias_values", C.c_void_p), ("n_bias", C.c_int64),
                ("bias_offsets", C.c_void_p), ("allow", C.c_void_p), ("allow_row", C.c_void_p), ("n_allow", C.c_int64),
                ("allow_ld", C.c_int64)]
    rows, on_host = None, ()  # rows that the tensors reach for and parts that a kernel cannot read, where make_logit_rules has seen them


class HiloreParam(C.Structure):
    """Mirror of ``struct hilore_param``."""
    _fields_ = [("p", C.c_void_p), ("master", C.c_void_p), ("g", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("m_scale", C.c_void_p), ("v_scale", C.c_void_p), ("n", C.c_int64), ("first", C.c_int64),
                ("p_dtype", C.c_int32), ("g_dtype", C.c_int32), ("state", C.c_int32), ("weight_decay", C.c_float)]


class HilorePolicyTerms(C.Structure):
    """Mirror of ``struct hilore_policy_terms``."""
    _fields_ = [("clip_low", C.c_double), ("clip_high", C.c_double), ("dual_clip", C.c_double), ("beta", C.c_double),
                ("rollout_cap", C.c_double), ("adv_eps", C.c_double), ("ratio", C.c_int32), ("mean", C.c_int32), ("kl", C.c_int32),
                ("adv_per_token", C.c_int32)]


class HilorePreferenceTerms(C.Structure):
    """Mirror of ``struct hilore_preference_terms``."""
    _fields_ = [("beta", C.c_double), ("margin", C.c_double), ("margin_reward", C.c_double), ("smoothing", C.c_double),
                ("nll", C.c_double), ("loss", C.c_int32), ("length_mean", C.c_int32)]


class HiloreError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status} ({status_string(status)})")


_lib = None


def library_path() -> str:
    return _build.LIB


def lib() -> C.CDLL:
    """Load libhilore_b200.so (built in-tree by paper_2609_33570_b200.build)."""
    global _lib
    if _lib is None:
        path = library_path()
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: run `python -m paper_2609_33570_b200.build` "
                              "(there is no fallback path)")
        _lib = C.CDLL(path)
        _lib.hilore_status_string.restype = C.c_char_p
        _lib.hilore_status_string.argtypes = [C.c_int]
        _lib.hilore_abi_version.restype = C.c_int
        _lib.hilore_workspace_bytes.restype = C.c_size_t
        _lib.hilore_workspace_bytes.argtypes = [C.c_int32, C.c_int64]
        vp, i64, i32, f32 = C.c_void_p, C.c_int64, C.c_int32, C.c_float
        _lib.hilore_mask_count.argtypes = [vp, i64, vp, vp]
        _lib.hilore_grpo_coeffs.argtypes = [vp, i64, i32, i64, i64, i64, vp, vp, vp, vp, i64, vp, f32, f32, f32,
                                            vp, vp, vp, vp, vp]
        _lib.hilore_unit_exposure.argtypes = [vp, vp, i64, i64, vp, i32, i64, i32, f32, vp, vp, vp, C.c_size_t, vp]
        _lib.hilore_unit_exposure_static.argtypes = [vp, vp, i64, i64, vp, i32, i64, i32, f32, vp, vp, vp]
        _lib.hilore_static_scratch_bytes.restype = C.c_size_t
        _lib.hilore_static_scratch_bytes.argtypes = []
        _lib.hilore_allocate.argtypes = [i32, vp, vp, vp, vp, C.c_double, C.c_double, i32, vp, vp, vp, vp, C.c_size_t, vp]
        _lib.hilore_allocate_workspace_bytes.restype = C.c_size_t
        _lib.hilore_allocate_workspace_bytes.argtypes = [i32, i32]
        _lib.hilore_risk_budget.restype = C.c_double
        _lib.hilore_risk_budget.argtypes = [C.c_double, i64, i64]
        _lib.hilore_relative_error.argtypes = [vp, vp, i64, i64, i64, i64, vp, vp, vp, C.c_size_t, vp]
        _lib.hilore_relative_error_workspace_bytes.restype = C.c_size_t
        _lib.hilore_relative_error_workspace_bytes.argtypes = []
        _lib.hilore_fit_kappa.restype = C.c_double
        _lib.hilore_fit_kappa.argtypes = [vp, vp, i64]
        _lib.hilore_grpo_coeffs_variant.argtypes = [vp, i64, i32, i64, i64, i64, vp, vp, vp, vp, i64, vp, f32, f32, f32, i32,
                                                    vp, vp, vp, vp, vp]
        _lib.hilore_grpo_coeffs_packed.argtypes = [vp, i64, i32, i64, i64, vp, i64, vp, vp, vp, vp, i64, vp, f32, f32, f32,
                                                   vp, vp, vp, vp, vp]
        _lib.hilore_unit_exposure_packed.argtypes = [vp, vp, i64, vp, i64, vp, i32, i64, i32, f32, vp, vp, vp, C.c_size_t, vp]
        _lib.hilore_coeffs_exposure.argtypes = [vp, i64, i32, i64, i64, i64, vp, vp, vp, vp, i64, vp, f32, f32, f32, vp, i32, i64,
                                                i32, f32, vp, vp, vp, vp, C.c_size_t, vp]
        _lib.hilore_scores_plan.argtypes = [vp, i64, i32, i64, i64, i64, vp, vp, vp, vp, i64, vp, f32, f32, f32, vp, i32, i64, i32,
                                            f32, vp, vp, vp, vp, vp, vp, f32, f32, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        _lib.hilore_scores_plan_workspace_bytes.restype = C.c_size_t
        _lib.hilore_scores_plan_workspace_bytes.argtypes = [i32, i64]
        _lib.hilore_codec_relative_error.argtypes = [vp, i64, i64, i64, i32, i32, vp, vp, vp, C.c_size_t, vp]
        _lib.hilore_omega_diagnostics.argtypes = [vp, vp, vp, vp, i64, i64, f32, vp, vp, vp, vp, C.c_size_t, vp]
        _lib.hilore_omega_diagnostics_workspace_bytes.restype = C.c_size_t
        _lib.hilore_omega_diagnostics_workspace_bytes.argtypes = []
        _lib.hilore_compress.argtypes = [vp, i64, i64, i64, i32, i32, vp, vp, vp, vp]
        _lib.hilore_recover.argtypes = [vp, vp, i64, i64, i32, i32, vp, i64, vp]
        _lib.hilore_plan_apply.argtypes = [vp, vp, i32, i32, vp, vp, vp, f32, f32, vp, vp, vp, vp, vp, vp]
        _lib.hilore_logits_apply.argtypes = [vp, i32, i64, i64, i64, vp, vp, i64, vp]
        _lib.hilore_logits_apply_backward.argtypes = [vp, i32, i64, i64, i64, vp, vp, i64, vp, i64, vp]
        _lib.hilore_token_logp.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, vp, vp, vp]
        _lib.hilore_token_logp_backward.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, vp, vp, i64, vp]
        _lib.hilore_grad_norm.argtypes = [vp, vp, i32, C.c_double, vp, vp, vp, C.c_size_t, vp]
        _lib.hilore_grad_norm_workspace_bytes.restype = C.c_size_t
        _lib.hilore_grad_norm_workspace_bytes.argtypes = []
        _lib.hilore_adamw_step.argtypes = [vp, vp, i32, C.c_double, vp, C.c_double, C.c_double, C.c_double, i64, vp, vp, vp]
        f64, sz = C.c_double, C.c_size_t
        _lib.hilore_advantages.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp, i64, i64, f64, f64, vp, vp, vp, vp, sz, vp]
        _lib.hilore_advantages_backward.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, f64, f64, vp, vp, vp, vp, vp, vp, sz, vp]
        _lib.hilore_policy_loss.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i64, i64, vp, i64, vp, vp, vp, vp, vp, sz, vp]
        _lib.hilore_preference_loss.argtypes = [vp, vp, vp, vp, i32, vp, i64, i64, vp, i64, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        _lib.hilore_advantages_workspace_bytes.argtypes = [i64]
        for name in ("hilore_policy_loss_workspace_bytes", "hilore_preference_loss_workspace_bytes"):
            getattr(_lib, name).argtypes = [i64, i64]
        for name in ("hilore_advantages_workspace_bytes", "hilore_policy_loss_workspace_bytes", "hilore_preference_loss_workspace_bytes"):
            getattr(_lib, name).restype = sz
        for name in EXPORTS:
            if name not in ("hilore_advantages_workspace_bytes", "hilore_policy_loss_workspace_bytes",
                            "hilore_preference_loss_workspace_bytes", "hilore_grad_norm_workspace_bytes", "hilore_status_string", "hilore_workspace_bytes", "hilore_static_scratch_bytes",
                            "hilore_allocate_workspace_bytes", "hilore_risk_budget",
                            "hilore_relative_error_workspace_bytes", "hilore_fit_kappa",
                            "hilore_omega_diagnostics_workspace_bytes", "hilore_scores_plan_workspace_bytes"):
                getattr(_lib, name).restype = C.c_int
    return _lib


def status_string(status: int) -> str:
    return lib().hilore_status_string(int(status)).decode()


def _ptr(t):
    """Device (or host) address of a tensor; None -> NULL; ints pass through as raw addresses."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


# the current stream's handle without building a Stream object (3.2 us -> 1.2 us per call where torch has these)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and _raw_device is not None:
            return _raw_stream(_raw_device())
        return torch.cuda.current_stream().cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


def _check(st, where, check):
    if check and st != OK:
        raise HiloreError(st, where)
    return st


def hilore_mask_count(mask, n, count, stream=None, check=True):
    return _check(lib().hilore_mask_count(_ptr(mask), n, _ptr(count), _stream(stream)), "hilore_mask_count", check)


def hilore_grpo_coeffs(rewards, n_resp_total, G, resp_offset, n_rows, T, logp_new, logp_old, logp_ref, mask,
                       N_norm, N_norm_dev, clip_eps, beta, adv_eps, adv_out, omega, ratio, clip_mask,
                       stream=None, check=True):
    st = lib().hilore_grpo_coeffs(_ptr(rewards), n_resp_total, G, resp_offset, n_rows, T, _ptr(logp_new),
                                  _ptr(logp_old), _ptr(logp_ref), _ptr(mask), N_norm, _ptr(N_norm_dev),
                                  clip_eps, beta, adv_eps, _ptr(adv_out), _ptr(omega), _ptr(ratio),
                                  _ptr(clip_mask), _stream(stream))
    return _check(st, "hilore_grpo_coeffs", check)


def hilore_grpo_coeffs_variant(rewards, n_resp_total, G, resp_offset, n_rows, T, logp_new, logp_old, logp_ref, mask,
                               N_norm, N_norm_dev, clip_eps, beta, adv_eps, variant, adv_out, omega, ratio, clip_mask,
                               stream=None, check=True):
    st = lib().hilore_grpo_coeffs_variant(_ptr(rewards), n_resp_total, G, resp_offset, n_rows, T, _ptr(logp_new),
                                          _ptr(logp_old), _ptr(logp_ref), _ptr(mask), N_norm, _ptr(N_norm_dev),
                                          clip_eps, beta, adv_eps, variant, _ptr(adv_out), _ptr(omega), _ptr(ratio),
                                          _ptr(clip_mask), _stream(stream))
    return _check(st, "hilore_grpo_coeffs_variant", check)


def hilore_grpo_coeffs_packed(rewards, n_resp_total, G, resp_offset, n_seq, cu_seqlens, n_tok, logp_new, logp_old,
                              logp_ref, mask, N_norm, N_norm_dev, clip_eps, beta, adv_eps, adv_out, omega, ratio,
                              clip_mask, stream=None, check=True):
    st = lib().hilore_grpo_coeffs_packed(_ptr(rewards), n_resp_total, G, resp_offset, n_seq, _ptr(cu_seqlens), n_tok,
                                         _ptr(logp_new), _ptr(logp_old), _ptr(logp_ref), _ptr(mask), N_norm,
                                         _ptr(N_norm_dev), clip_eps, beta, adv_eps, _ptr(adv_out), _ptr(omega),
                                         _ptr(ratio), _ptr(clip_mask), _stream(stream))
    return _check(st, "hilore_grpo_coeffs_packed", check)


def hilore_unit_exposure_packed(omega, mask, n_tok, cu_seqlens, n_seq, row_rms, U, rms_ld, row_shift, eps_alpha,
                                exposure, sum_abs_omega, workspace, workspace_bytes, stream=None, check=True):
    st = lib().hilore_unit_exposure_packed(_ptr(omega), _ptr(mask), n_tok, _ptr(cu_seqlens), n_seq, _ptr(row_rms), U,
                                           rms_ld, row_shift, eps_alpha, _ptr(exposure), _ptr(sum_abs_omega),
                                           _ptr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "hilore_unit_exposure_packed", check)


def hilore_coeffs_exposure(rewards, n_resp_total, G, resp_offset, n_rows, T, logp_new, logp_old, logp_ref, mask, N_norm,
                           N_norm_dev, clip_eps, beta, adv_eps, row_rms, U, rms_ld, row_shift, eps_alpha, omega, exposure,
                           sum_abs_omega, workspace, workspace_bytes, stream=None, check=True):
    st = lib().hilore_coeffs_exposure(_ptr(rewards), n_resp_total, G, resp_offset, n_rows, T, _ptr(logp_new), _ptr(logp_old),
                                      _ptr(logp_ref), _ptr(mask), N_norm, _ptr(N_norm_dev), clip_eps, beta, adv_eps,
                                      _ptr(row_rms), U, rms_ld, row_shift, eps_alpha, _ptr(omega), _ptr(exposure),
                                      _ptr(sum_abs_omega), _ptr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "hilore_coeffs_exposure", check)


def hilore_scores_plan_workspace_bytes(U, n_tok):
    return int(lib().hilore_scores_plan_workspace_bytes(U, n_tok))


def hilore_scores_plan(rewards, n_resp_total, G, resp_offset, n_rows, T, logp_new, logp_old, logp_ref, mask, N_norm, N_norm_dev,
                       clip_eps, beta, adv_eps, row_rms, U, rms_ld, row_shift, eps_alpha, omega, exposure, sum_abs_omega,
                       units_dev, kappa, ebar, tau_lo, tau_hi, avail, action_io, psi, recompute, retained_bytes, workspace,
                       workspace_bytes, stream=None, check=True):
    st = lib().hilore_scores_plan(_ptr(rewards), n_resp_total, G, resp_offset, n_rows, T, _ptr(logp_new), _ptr(logp_old),
                                  _ptr(logp_ref), _ptr(mask), N_norm, _ptr(N_norm_dev), clip_eps, beta, adv_eps, _ptr(row_rms), U,
                                  rms_ld, row_shift, eps_alpha, _ptr(omega), _ptr(exposure), _ptr(sum_abs_omega), _ptr(units_dev),
                                  _ptr(kappa), _ptr(ebar), tau_lo, tau_hi, _ptr(avail), _ptr(action_io), _ptr(psi),
                                  _ptr(recompute), _ptr(retained_bytes), _ptr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "hilore_scores_plan", check)


def hilore_codec_relative_error(x, rows, cols, ld, fmt, block, e_out, norms2, workspace, workspace_bytes, stream=None,
                                check=True):
    st = lib().hilore_codec_relative_error(_ptr(x), rows, cols, ld, fmt, block, _ptr(e_out), _ptr(norms2), _ptr(workspace),
                                           workspace_bytes, _stream(stream))
    return _check(st, "hilore_codec_relative_error", check)


def hilore_omega_diagnostics_workspace_bytes():
    return int(lib().hilore_omega_diagnostics_workspace_bytes())


def hilore_omega_diagnostics(adv, ratio, mask, omega, n_rows, T, clip_eps, counts, top_share, sum_abs, workspace,
                             workspace_bytes, stream=None, check=True):
    st = lib().hilore_omega_diagnostics(_ptr(adv), _ptr(ratio), _ptr(mask), _ptr(omega), n_rows, T, clip_eps,
                                        _ptr(counts), _ptr(top_share), _ptr(sum_abs), _ptr(workspace), workspace_bytes,
                                        _stream(stream))
    return _check(st, "hilore_omega_diagnostics", check)


def hilore_workspace_bytes(U, n_tok):
    return int(lib().hilore_workspace_bytes(U, n_tok))


def hilore_unit_exposure(omega, mask, n_rows, T, row_rms, U, rms_ld, row_shift, eps_alpha, exposure,
                         sum_abs_omega, workspace, workspace_bytes, stream=None, check=True):
    st = lib().hilore_unit_exposure(_ptr(omega), _ptr(mask), n_rows, T, _ptr(row_rms), U, rms_ld, row_shift,
                                    eps_alpha, _ptr(exposure), _ptr(sum_abs_omega), _ptr(workspace),
                                    workspace_bytes, _stream(stream))
    return _check(st, "hilore_unit_exposure", check)


def hilore_allocate_workspace_bytes(U, n_intervals=1024):
    return int(lib().hilore_allocate_workspace_bytes(U, n_intervals))


def hilore_risk_budget(delta, N_b, N_total):
    return float(lib().hilore_risk_budget(delta, N_b, N_total))


def hilore_allocate(U, psi, dtau, dmem, avail, M_res, delta_b, n_intervals, action, recompute, totals, workspace,
                    workspace_bytes, stream=None, check=True):
    st = lib().hilore_allocate(U, _ptr(psi), _ptr(dtau), _ptr(dmem), _ptr(avail), M_res, delta_b, n_intervals,
                               _ptr(action), _ptr(recompute), _ptr(totals), _ptr(workspace), workspace_bytes,
                               _stream(stream))
    return _check(st, "hilore_allocate", check)


def hilore_relative_error_workspace_bytes():
    return int(lib().hilore_relative_error_workspace_bytes())


def hilore_relative_error(x, xhat, rows, cols, ld, ld_hat, e_out, norms2, workspace, workspace_bytes, stream=None,
                          check=True):
    st = lib().hilore_relative_error(_ptr(x), _ptr(xhat), rows, cols, ld, ld_hat, _ptr(e_out), _ptr(norms2),
                                     _ptr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "hilore_relative_error", check)


def hilore_fit_kappa(x, y):
    """x, y: sequences of host floats (calibration pairs)."""
    n = len(x)
    ax = (C.c_double * n)(*[float(v) for v in x])
    ay = (C.c_double * n)(*[float(v) for v in y])
    return float(lib().hilore_fit_kappa(C.cast(ax, C.c_void_p), C.cast(ay, C.c_void_p), n))


def hilore_static_scratch_bytes():
    return int(lib().hilore_static_scratch_bytes())


def hilore_unit_exposure_static(omega, mask, n_rows, T, row_rms, U, rms_ld, row_shift, eps_alpha, exposure,
                                sum_abs_omega, stream=None, check=True):
    """hilore_unit_exposure without a workspace argument: the partial sums use the library's built-in
    1 MiB scratch array, so the call allocates nothing (see include/hilore.h for the limits)."""
    st = lib().hilore_unit_exposure_static(_ptr(omega), _ptr(mask), n_rows, T, _ptr(row_rms), U, rms_ld, row_shift,
                                           eps_alpha, _ptr(exposure), _ptr(sum_abs_omega), _stream(stream))
    return _check(st, "hilore_unit_exposure_static", check)


def hilore_compress(x, rows, cols, ld, fmt, block, codes, scales, row_rms, stream=None, check=True):
    st = lib().hilore_compress(_ptr(x), rows, cols, ld, fmt, block, _ptr(codes), _ptr(scales), _ptr(row_rms),
                               _stream(stream))
    return _check(st, "hilore_compress", check)


def hilore_recover(codes, scales, rows, cols, fmt, block, out, ld_out, stream=None, check=True):
    st = lib().hilore_recover(_ptr(codes), _ptr(scales), rows, cols, fmt, block, _ptr(out), ld_out,
                              _stream(stream))
    return _check(st, "hilore_recover", check)


def hilore_plan_apply(units_dev, units_host, U, phase, exposure, kappa, ebar, tau_lo, tau_hi, avail, action_io,
                      psi, recompute, retained_bytes, stream=None, check=True):
    """units_dev: device address (tensor or int) of the hilore_unit table; units_host: a ctypes array
    ``(HiloreUnit * U)`` holding the same table on the host."""
    host = C.cast(units_host, C.c_void_p) if units_host is not None else None
    st = lib().hilore_plan_apply(_ptr(units_dev), host, U, phase, _ptr(exposure), _ptr(kappa), _ptr(ebar),
                                 tau_lo, tau_hi, _ptr(avail), _ptr(action_io), _ptr(psi), _ptr(recompute),
                                 _ptr(retained_bytes), _stream(stream))
    return _check(st, "hilore_plan_apply", check)


def make_unit_table(units, device="cuda"):
    """Marshal a list of dicts (x, codes, scales, out, row_rms tensors or None; rows, cols, ld, fmt, block)
    into the host ctypes array and a device copy of it.  Returns (units_dev tensor, units_host array)."""
    arr = (HiloreUnit * len(units))()
    for i, u in enumerate(units):
        arr[i] = HiloreUnit(_ptr(u.get("x")), _ptr(u.get("codes")), _ptr(u.get("scales")), _ptr(u.get("out")),
                            _ptr(u.get("row_rms")), u["rows"], u["cols"], u.get("ld", u["cols"]), u["fmt"],
                            u["block"])
    raw = bytes(arr)
    host = torch.frombuffer(bytearray(raw), dtype=torch.uint8)
    dev = host.to(device)
    return dev, arr


def _rules(rules, n_rows):
    """Address of the rules, or None.  Those made from tensors have to reach for all rows, and from the device."""
    if rules is None:
        return None
    if rules.rows is not None and n_rows > rules.rows:
        raise ValueError(f"rules of {rules.rows} rows in a call of {n_rows}")
    if rules.on_host:
        raise ValueError(f"{', '.join(rules.on_host)}: expected device tensors")
    return C.addressof(rules)


def _table(params_host, n_params):
    """Address of the host half of a table, or None."""
    if params_host is None:
        return None
    if n_params > len(params_host):
        raise ValueError(f"a table of {len(params_host)} entries in a call of {n_params}")
    return C.addressof(params_host)


def hilore_logits_apply(logits, dtype, n_rows, V, ld, rules, out, ld_out, stream=None, check=True):
    """rules: a HiloreLogitRules on the host (make_logit_rules)."""
    st = lib().hilore_logits_apply(_ptr(logits), dtype, n_rows, V, ld, _rules(rules, n_rows), _ptr(out), ld_out, _stream(stream))
    return _check(st, "hilore_logits_apply", check)


def hilore_logits_apply_backward(logits, dtype, n_rows, V, ld, rules, grad_out, ld_grad_out, grad_in, ld_grad_in,
                                 stream=None, check=True):
    st = lib().hilore_logits_apply_backward(_ptr(logits), dtype, n_rows, V, ld, _rules(rules, n_rows), _ptr(grad_out), ld_grad_out,
                                            _ptr(grad_in), ld_grad_in, _stream(stream))
    return _check(st, "hilore_logits_apply_backward", check)


def hilore_token_logp(logits, dtype, n_rows, V, ld, rules, targets, logp, lse, entropy, stream=None, check=True):
    st = lib().hilore_token_logp(_ptr(logits), dtype, n_rows, V, ld, _rules(rules, n_rows), _ptr(targets), _ptr(logp), _ptr(lse),
                                 _ptr(entropy), _stream(stream))
    return _check(st, "hilore_token_logp", check)


def hilore_token_logp_backward(logits, dtype, n_rows, V, ld, rules, targets, lse, omega, grad, ld_grad, stream=None,
                               check=True):
    st = lib().hilore_token_logp_backward(_ptr(logits), dtype, n_rows, V, ld, _rules(rules, n_rows), _ptr(targets), _ptr(lse),
                                          _ptr(omega), _ptr(grad), ld_grad, _stream(stream))
    return _check(st, "hilore_token_logp_backward", check)


def hilore_grad_norm_workspace_bytes():
    return int(lib().hilore_grad_norm_workspace_bytes())


def hilore_grad_norm(params_dev, params_host, n_params, max_norm, norm, scale, workspace, workspace_bytes, stream=None,
                     check=True):
    """params_dev / params_host: the two halves of make_param_table."""
    st = lib().hilore_grad_norm(_ptr(params_dev), _table(params_host, n_params), n_params, max_norm, _ptr(norm), _ptr(scale),
                                _ptr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "hilore_grad_norm", check)


def hilore_adamw_step(params_dev, params_host, n_params, lr, lr_dev, beta1, beta2, eps, step, step_dev, grad_scale,
                      stream=None, check=True):
    st = lib().hilore_adamw_step(_ptr(params_dev), _table(params_host, n_params), n_params, lr, _ptr(lr_dev), beta1, beta2, eps, step,
                                 _ptr(step_dev), _ptr(grad_scale), _stream(stream))
    return _check(st, "hilore_adamw_step", check)


def hilore_advantages_workspace_bytes(n_tok):
    return int(lib().hilore_advantages_workspace_bytes(n_tok))


def hilore_advantages(rewards, outcome, values, values_dtype, bootstrap, trace, mask, cu_seqlens, n_seq, n_tok, gamma, lam, adv,
                      returns, moments, workspace, workspace_bytes, stream=None, check=True):
    st = lib().hilore_advantages(_ptr(rewards), _ptr(outcome), _ptr(values), values_dtype, _ptr(bootstrap), _ptr(trace), _ptr(mask),
                                 _ptr(cu_seqlens), n_seq, n_tok, gamma, lam, _ptr(adv), _ptr(returns), _ptr(moments),
                                 _ptr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "hilore_advantages", check)


def hilore_advantages_backward(grad_adv, grad_returns, adv, trace, mask, cu_seqlens, n_seq, n_tok, gamma, lam, grad_rewards,
                               grad_outcome, grad_values, grad_bootstrap, grad_trace, workspace, workspace_bytes, stream=None,
                               check=True):
    st = lib().hilore_advantages_backward(_ptr(grad_adv), _ptr(grad_returns), _ptr(adv), _ptr(trace), _ptr(mask), _ptr(cu_seqlens),
                                          n_seq, n_tok, gamma, lam, _ptr(grad_rewards), _ptr(grad_outcome), _ptr(grad_values),
                                          _ptr(grad_bootstrap), _ptr(grad_trace), _ptr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "hilore_advantages_backward", check)


def _terms(terms, kind):
    """Address of a struct of terms, or None."""
    if terms is None:
        return None
    if not isinstance(terms, kind):
        raise TypeError(f"terms: expected {kind.__name__}, got {type(terms).__name__}")
    return C.addressof(terms)


def make_policy_terms(clip_low=0.2, clip_high=0.2, dual_clip=0.0, beta=0.0, rollout_cap=float("inf"), adv_eps=1e-6,
                      ratio=RATIO_TOKEN, mean=MEAN_TOKENS, kl=KL_K3, adv_per_token=False):
    """The host struct that hilore_policy_loss reads."""
    return HilorePolicyTerms(clip_low, clip_high, dual_clip, beta, rollout_cap, adv_eps, ratio, mean, kl, int(adv_per_token))


def make_preference_terms(beta=0.1, margin=0.0, margin_reward=0.0, smoothing=0.0, nll=0.0, loss=PREF_SIGMOID, length_mean=False):
    """The host struct that hilore_preference_loss reads."""
    return HilorePreferenceTerms(beta, margin, margin_reward, smoothing, nll, loss, int(length_mean))


def hilore_policy_loss_workspace_bytes(n_seq, n_tok):
    return int(lib().hilore_policy_loss_workspace_bytes(n_seq, n_tok))


def hilore_policy_loss(logp, logp_old, logp_ref, logp_rollout, mask, adv, adv_moments, cu_seqlens, n_seq, n_tok, terms, N_norm,
                       N_norm_dev, grad_loss, stats, omega, workspace, workspace_bytes, stream=None, check=True):
    """terms: make_policy_terms."""
    st = lib().hilore_policy_loss(_ptr(logp), _ptr(logp_old), _ptr(logp_ref), _ptr(logp_rollout), _ptr(mask), _ptr(adv),
                                  _ptr(adv_moments), _ptr(cu_seqlens), n_seq, n_tok, _terms(terms, HilorePolicyTerms), N_norm,
                                  _ptr(N_norm_dev), _ptr(grad_loss), _ptr(stats), _ptr(omega), _ptr(workspace), workspace_bytes,
                                  _stream(stream))
    return _check(st, "hilore_policy_loss", check)


def hilore_preference_loss_workspace_bytes(n_seq, n_tok):
    return int(lib().hilore_preference_loss_workspace_bytes(n_seq, n_tok))


def hilore_preference_loss(logp, logp_ref, mask, rewards, G, cu_seqlens, n_seq, n_tok, terms, N_norm, N_norm_dev, grad_loss, scores,
                           pairs, stats, omega, workspace, workspace_bytes, stream=None, check=True):
    """terms: make_preference_terms."""
    st = lib().hilore_preference_loss(_ptr(logp), _ptr(logp_ref), _ptr(mask), _ptr(rewards), G, _ptr(cu_seqlens), n_seq, n_tok,
                                      _terms(terms, HilorePreferenceTerms), N_norm, _ptr(N_norm_dev), _ptr(grad_loss), _ptr(scores),
                                      _ptr(pairs), _ptr(stats), _ptr(omega), _ptr(workspace), workspace_bytes, _stream(stream))
    return _check(st, "hilore_preference_loss", check)


def _typed(t, name, *dtypes):
    """`t` if it is None or a contiguous tensor of one of `dtypes`: the structs below carry addresses only."""
    if t is not None and t.dtype not in dtypes:
        raise TypeError(f"{name}: expected {' or '.join(map(str, dtypes))}, got {t.dtype}")
    if t is not None and not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor")
    return t


def _on_host(t):
    """Whether `t` is a tensor in host memory that kernels cannot read."""
    return t is not None and not t.is_cuda and not (t.device.type == "cpu" and t.is_pinned())


def make_logit_rules(temperature=None, repetition=None, frequency=None, presence=None, tokens=None, hist_begin=None,
                     resp_begin=None, hist_end=None, bias_tokens=None, bias_values=None, bias_offsets=None, allow=None,
                     allow_row=None):
    """Marshal the tensors of ``struct hilore_logit_rules`` (fp32 levels, int32 tokens, int64 ranges, int32 mask words
    [n_allow, allow_ld]).  The struct holds addresses and keeps the tensors alive.  A call may have as many rows as the
    shortest of its tensors with an entry per row."""
    f, i, j = (torch.float32,), (torch.int32,), (torch.int64,)
    parts = dict(temperature=_typed(temperature, "temperature", *f), repetition=_typed(repetition, "repetition", *f),
                 frequency=_typed(frequency, "frequency", *f), presence=_typed(presence, "presence", *f),
                 tokens=_typed(tokens, "tokens", *i), hist_begin=_typed(hist_begin, "hist_begin", *j),
                 resp_begin=_typed(resp_begin, "resp_begin", *j), hist_end=_typed(hist_end, "hist_end", *j),
                 bias_tokens=_typed(bias_tokens, "bias_tokens", *i), bias_values=_typed(bias_values, "bias_values", *f),
                 bias_offsets=_typed(bias_offsets, "bias_offsets", *j), allow=_typed(allow, "allow", *i),
                 allow_row=_typed(allow_row, "allow_row", *i))
    needs = dict(hist_begin="tokens", resp_begin="tokens", hist_end="tokens", bias_offsets="bias_tokens", bias_values="bias_tokens",
                 allow_row="allow")  # parts that are read beside another one alone
    filled = {k: t for k, t in parts.items() if t is not None and t.numel()}
    read = {k: t for k, t in filled.items() if needs.get(k, k) in filled}
    per_row = {k: t.numel() - (k == "bias_offsets") for k, t in read.items()
               if k not in ("tokens", "bias_tokens", "bias_values", "allow")}
    if bias_tokens is not None and bias_values is not None and bias_values.numel() < bias_tokens.numel():
        raise ValueError(f"{bias_values.numel()} bias_values of {bias_tokens.numel()} bias_tokens")
    if allow is not None and allow.dim() != 2:
        raise ValueError(f"allow: expected [n_allow, allow_ld], got {tuple(allow.shape)}")
    r = HiloreLogitRules(**{k: _ptr(t) for k, t in parts.items()})
    r.n_tokens = 0 if tokens is None else tokens.numel()
    r.n_bias = 0 if bias_tokens is None else bias_tokens.numel()
    if allow is not None:
        r.n_allow, r.allow_ld = allow.shape
    r.rows = min(per_row.values(), default=None)
    r.on_host = tuple(k for k, t in read.items() if _on_host(t))
    r.keep = parts
    return r


def make_param_table(params, device="cuda"):
    """Marshal a list of dicts (p, g, m, v tensors; master, m_scale, v_scale tensors or None; weight_decay) into the
    host ctypes array and a device copy of it.  Types are taken from the tensors: one-byte m and v are codes.  Returns
    (params_dev tensor, params_host array); the array keeps the tensors alive."""
    kinds = {torch.bfloat16: BF16, torch.float32: F32}
    arr = (HiloreParam * len(params))()
    to_device = torch.device(device).type == "cuda"
    first = 0
    for i, e in enumerate(params):
        p, g, m, v = (_typed(e[k], k, *t) for k, t in (("p", tuple(kinds)), ("g", tuple(kinds)),
                                                       ("m", (torch.float32, torch.uint8, torch.float8_e4m3fn)),
                                                       ("v", (torch.float32, torch.uint8, torch.float8_e4m3fn))))
        n, coded = p.numel(), m.element_size() == 1
        master, ms, vs = (_typed(e.get(k), k, torch.float32) for k in ("master", "m_scale", "v_scale"))
        blocks = (n + BLOCK - 1) // BLOCK
        for name, t, want in (("p", p, n), ("g", g, n), ("m", m, n), ("v", v, n), ("master", master, n), ("m_scale", ms, blocks),
                              ("v_scale", vs, blocks)):
            if t is not None and t.numel() != want:
                raise ValueError(f"entry {i}: {name} has {t.numel()} elements, expected {want}")
            if to_device and _on_host(t):
                raise ValueError(f"entry {i}: {name} is on the host, the table on {device}")
        if (v.element_size() == 1) != coded or coded != (ms is not None) or coded != (vs is not None):
            raise ValueError(f"entry {i}: m and v are both fp32 without scales, or both codes with scales")
        arr[i] = HiloreParam(_ptr(p), _ptr(master), _ptr(g), _ptr(m), _ptr(v), _ptr(ms), _ptr(vs), n, first, kinds[p.dtype],
                             kinds[g.dtype], STATE_E4M3FN if coded else STATE_F32, e.get("weight_decay", 0.0))
        first += (n + PARAM_TILE - 1) // PARAM_TILE
    arr.keep = [dict(e) for e in params]
    dev = torch.frombuffer(bytearray(bytes(arr)), dtype=torch.uint8).to(device) if len(params) else None
    return dev, arr
