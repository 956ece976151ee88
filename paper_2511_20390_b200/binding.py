"""ctypes binding of libfree_b200.so: argument marshalling only.

Tensors are torch CUDA tensors (device memory owner); the library receives raw device pointers and
the current stream.  Nothing here computes any part of the method.
"""
import ctypes as C
import os
import struct
import threading
import typing
from operator import index

import numpy as np
import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libfree_b200.so")

FREE_FP32, FREE_BF16, FREE_E4M3 = 0, 1, 2
FREE_MAX_K = 64
EPI_BIAS, EPI_BIAS_GELU, EPI_BIAS_SILU, EPI_GATE_RESIDUAL = 0, 1, 2, 3


class FreeError(RuntimeError):
    def __init__(self, code, what):
        self.code = code
        super().__init__(f"{what}: error {code} ({lib().free_strerror(code).decode()})")


class BlockWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("ada_w", "ada_b", "qkv_w", "qkv_b", "proj_w", "proj_b",
                                          "fc1_w", "fc1_b", "fc2_w", "fc2_b")]


class ModelDesc(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("dtype", "C", "H", "W", "patch", "D", "depth", "heads",
                                          "n_classes", "c_out", "freq_dim", "mlp_ratio")]
                + [(n, C.c_void_p) for n in ("t_w1", "t_b1", "t_w2", "t_b2", "y_emb", "pe_w", "pe_b", "pos")]
                + [("blocks", BlockWeights)]
                + [(n, C.c_void_p) for n in ("fada_w", "fada_b", "fin_w", "fin_b")])


class DrafterDesc(C.Structure):
    _fields_ = ([("n_blocks", C.c_int32)] + [(n, C.c_void_p) for n in ("fc_w", "fc_b")]
                + [("blocks", BlockWeights)]
                + [(n, C.c_void_p) for n in ("fada_w", "fada_b", "fin_w", "fin_b")])


class ScheduleDesc(C.Structure):
    _fields_ = [("N", C.c_int32)] + [(n, C.c_void_p) for n in ("coef_x", "coef_eps", "sigma2", "t_embed_value")]


class SpecParams(C.Structure):
    _fields_ = [("K", C.c_int32), ("cfg_scale", C.c_float), ("lam", C.c_void_p), ("use_graph", C.c_int32)]


class ProfEntry(C.Structure):
    _fields_ = [("name", C.c_char * 48), ("launches", C.c_int64), ("ms", C.c_double), ("work", C.c_double)]


class TrajStats(C.Structure):
    _fields_ = [("rounds", C.c_int64), ("target_calls", C.c_int64), ("draft_calls", C.c_int64),
                ("accepted", C.c_int64), ("rejected", C.c_int64),
                ("accept_hist", C.c_int64 * (FREE_MAX_K + 1)), ("parallel_efficiency", C.c_double),
                ("graph_rounds", C.c_int64)]


_LIB = None


class _Int:
    """A C int argument.  C.c_int cuts larger numbers to 32 bits without a word (2^32 + 64 rows would be computed as 64);
    here they are an error (C.ArgumentError).  No slower than C.c_int, which makes an object per argument."""
    @staticmethod
    def from_param(v):
        n = index(v)
        if -0x80000000 <= n <= 0x7fffffff:
            return n
        raise ValueError(f"{n} does not fit a C int")


_SIGNATURES = {
    "free_strerror": (C.c_char_p, [_Int]),
    "free_create": (C.c_int, [C.POINTER(ModelDesc), C.POINTER(DrafterDesc), C.POINTER(C.c_void_p)]),
    "free_destroy": (C.c_int, [C.c_void_p]),
    "free_workspace_bytes": (C.c_size_t, [C.c_void_p, _Int]),
    "dit_verify_pass": (C.c_int, [C.c_void_p, _Int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float,
                                  C.POINTER(ScheduleDesc), C.c_void_p, C.c_void_p, C.c_void_p,
                                  C.c_void_p, C.c_size_t, C.c_void_p]),
    "dit_verify_pass_raw": (C.c_int, [C.c_void_p, _Int, C.c_void_p, C.c_void_p, C.c_void_p, _Int,
                                      C.POINTER(ScheduleDesc), C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "spec_verify": (C.c_int, [_Int, _Int, C.c_int64] + [C.c_void_p] * 11),
    "spec_verify_fused": (C.c_int, [_Int, _Int, C.c_int64, _Int, C.c_float] + [C.c_void_p] * 10 + [_Int] + [C.c_void_p] * 6),
    "draft_step": (C.c_int, [C.c_void_p, _Int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float,
                             C.POINTER(ScheduleDesc), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                             C.c_void_p, C.c_size_t, C.c_void_p]),
    "sample_trajectory": (C.c_int, [C.c_void_p, _Int, C.c_void_p, C.c_void_p, C.POINTER(ScheduleDesc),
                                    C.POINTER(SpecParams), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.POINTER(TrajStats), C.c_void_p, C.c_size_t, C.c_void_p]),
    "free_spec_round": (C.c_int, [C.c_void_p, _Int, C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(ScheduleDesc),
                                  C.POINTER(SpecParams), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                  C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "free_split_range": (C.c_int, [_Int, _Int, _Int, C.POINTER(C.c_int), C.POINTER(C.c_int)]),
    "free_spec_round_begin": (C.c_int, [C.c_void_p, _Int, C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(ScheduleDesc),
                                        C.POINTER(SpecParams), C.c_void_p, C.c_void_p, C.c_void_p, _Int, _Int, C.c_void_p,
                                        C.c_void_p, C.c_size_t, C.c_void_p]),
    "free_spec_round_finish": (C.c_int, [C.c_void_p, _Int, C.c_void_p, C.POINTER(ScheduleDesc), C.POINTER(SpecParams),
                                         C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                         C.c_void_p, C.c_size_t, C.c_void_p]),
    "free_uncertainty_profile": (C.c_int, [C.c_void_p, _Int, C.c_void_p, C.c_void_p, C.POINTER(ScheduleDesc),
                                           C.POINTER(SpecParams), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                           C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "free_schedule_linear": (C.c_int, [_Int, C.c_double, C.c_double, _Int, C.c_double, C.c_double] + [C.c_void_p] * 4),
    "free_schedule_respaced": (C.c_int, [_Int, _Int, C.c_double, C.c_double, _Int, C.c_double, C.c_double] + [C.c_void_p] * 4),
    "free_fit_lambda_profile": (C.c_int, [C.c_void_p, C.c_void_p, _Int, _Int, C.c_void_p]),
    "free_drafter_loss_workspace_bytes": (C.c_size_t, []),
    "free_drafter_loss": (C.c_int, [_Int] * 4 + [C.c_int64] + [C.c_void_p] * 4 + [C.c_float] * 4 +
                          [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "free_set_launch_overlap": (C.c_int, [_Int]),
    "free_device_error_code": (C.c_int, [C.c_uint32]),
    "free_selftest_bounded_wait": (C.c_int, [C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]),
    "free_profile_begin": (C.c_int, [C.c_void_p]),
    "free_profile_end": (C.c_int, [C.c_void_p, C.POINTER(ProfEntry), _Int, C.POINTER(C.c_int)]),
    "free_op_linear_workspace_bytes": (C.c_size_t, []),
    "free_op_linear": (C.c_int, [_Int] * 6 + [C.c_void_p] * 6 + [C.c_int64, _Int, C.c_void_p, C.c_size_t, C.c_void_p]),
    "free_op_ln_modulate": (C.c_int, [_Int] * 4 + [C.c_void_p] * 3 + [C.c_int64, C.c_void_p, C.c_void_p]),
    "free_op_gated_linear": (C.c_int, [_Int] * 5 + [C.c_void_p] * 7),
    "free_op_gated_linear_bwd_workspace_bytes": (C.c_size_t, [_Int] * 4),
    "free_op_gated_linear_bwd": (C.c_int, [_Int] * 5 + [C.c_void_p] * 8 + [C.c_size_t, C.c_void_p, C.c_void_p]),
    "free_op_layer_norm": (C.c_int, [_Int] * 5 + [C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_int64, _Int, C.c_float,
                                                     C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]),
    "free_op_layer_norm_bwd_workspace_bytes": (C.c_size_t, [_Int] * 3),
    "free_op_layer_norm_bwd": (C.c_int, [_Int] * 5 + [C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p,
                                                         C.c_int64, _Int, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64,
                                                         C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]),
    "free_op_rms_norm": (C.c_int, [_Int] * 7 + [C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p,
                                                C.c_int64, _Int, C.c_float, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_int64, _Int,
                                                C.c_void_p, C.c_void_p]),
    "free_op_rms_norm_bwd_workspace_bytes": (C.c_size_t, [_Int] * 3),
    "free_op_rms_norm_bwd": (C.c_int, [_Int] * 6 + [C.c_void_p, C.c_int64, C.c_int64] * 2 + [C.c_void_p, C.c_void_p, C.c_int64, _Int] +
                             [C.c_void_p, C.c_int64, C.c_int64] * 2 + [C.c_void_p, C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]),
    "free_op_rope_axes": (C.c_int, [_Int] * 9 + [C.c_void_p, C.c_double, C.c_void_p, C.c_int64] +
                          [C.c_void_p, C.c_int64, C.c_int64, C.c_int64] * 2 + [C.c_void_p]),
    "free_op_cross_attention_workspace_bytes": (C.c_size_t, [C.c_char_p]),
    "free_op_cross_attention": (C.c_int, [C.c_char_p, C.c_void_p] + [C.c_int64] * 3 + [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]),
    "free_op_cross_attention_bwd_workspace_bytes": (C.c_size_t, [C.c_char_p]),
    "free_op_cross_attention_bwd": (C.c_int, [C.c_char_p, C.c_void_p] + [C.c_int64] * 3 + [C.c_void_p] + ([C.c_void_p] + [C.c_int64] * 3) * 4 +
                                    [C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]),
    "free_op_attention": (C.c_int, [_Int] * 5 + [C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "free_op_attention_workspace_bytes": (C.c_size_t, [_Int] * 5),
    "free_op_attention_static": (C.c_int, [_Int] * 4 + [C.c_void_p] * 4),
}


def exported_symbols():
    return sorted(_SIGNATURES)


def lib():
    """The loaded shared library; raises if it has not been built (there is no fallback path)."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2511_20390_b200.build`")
        L = C.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(L, name)          # AttributeError if the library does not export it
            fn.restype, fn.argtypes = res, args
        _LIB = L
    return _LIB


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(code, what):
    if code != 0:
        raise FreeError(code, what)


def _dev(t, dtype):
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise ValueError("expected a contiguous CUDA tensor of dtype %s" % dtype)
    return t


# ------------------------------------------------------------------------------------------ verifier
def spec_verify(m, m_hat, x_hat, sigma2, u, lam=None, n_valid=None, want_logratio=False,
                x_out=None, n_accept=None):
    """Algorithm 2 over K drafts per sample with the first-rejection break (strict, or relaxed when
    `lam` is given).  m, m_hat, x_hat: CUDA fp32 [B,K,d...]; sigma2, u, lam: [B,K]; n_valid int32 [B].
    Returns (x_out [B,d...], n_accept int32 [B][, ell [B,K]])."""
    B, K = m.shape[:2]
    d = int(np.prod(m.shape[2:]))
    for t in (m, m_hat, x_hat, sigma2, u):
        _dev(t, torch.float32)
    if x_out is None:
        x_out = torch.zeros((B,) + tuple(m.shape[2:]), dtype=torch.float32, device=m.device)
    if n_accept is None:
        n_accept = torch.empty(B, dtype=torch.int32, device=m.device)
    ell = torch.empty((B, K), dtype=torch.float32, device=m.device) if want_logratio else None
    code = lib().spec_verify(B, K, d, _ptr(m), _ptr(m_hat), _ptr(x_hat), _ptr(sigma2),
                             _ptr(None if lam is None else _dev(lam, torch.float32)), _ptr(u),
                             _ptr(None if n_valid is None else _dev(n_valid, torch.int32)),
                             _ptr(x_out), _ptr(n_accept), _ptr(ell), _stream())
    _check(code, "spec_verify")
    return (x_out, n_accept, ell) if want_logratio else (x_out, n_accept)


def spec_verify_fused(eps, x_first, m_hat, x_hat, coef_x, coef_eps, sigma2, u, cfg_scale, lam=None,
                      n_valid=None, chunk=0, want_logratio=False, want_means=False, want_dist2=False, x_out=None, n_accept=None):
    """Verification straight from the packed pass's noise predictions (guidance, Eq. ddpm_update and Algorithm 2 in
    one kernel).  eps: CUDA fp32 [B,K,G,d...]; x_first [B,d...]; m_hat, x_hat [B,K,d...]; coef_x, coef_eps, sigma2, u,
    lam: [B,K]; chunk > 0 enables the early exit.  Returns (x_out, n_accept[, ell][, means][, dist2])."""
    B, K, G = eps.shape[:3]
    d = int(np.prod(eps.shape[3:]))
    for t in (eps, x_first, m_hat, x_hat, coef_x, coef_eps, sigma2, u):
        _dev(t, torch.float32)
    dev = eps.device
    if x_out is None:
        x_out = torch.zeros((B,) + tuple(eps.shape[3:]), dtype=torch.float32, device=dev)
    if n_accept is None:
        n_accept = torch.empty(B, dtype=torch.int32, device=dev)
    ell = torch.empty((B, K), dtype=torch.float32, device=dev) if want_logratio else None
    means = torch.zeros((B, K) + tuple(eps.shape[3:]), dtype=torch.float32, device=dev) if want_means else None
    dist2 = torch.empty((B, K), dtype=torch.float32, device=dev) if want_dist2 else None
    code = lib().spec_verify_fused(B, K, d, G, float(cfg_scale), _ptr(eps), _ptr(x_first),
                                   _ptr(m_hat), _ptr(x_hat), _ptr(coef_x), _ptr(coef_eps), _ptr(sigma2),
                                   _ptr(None if lam is None else _dev(lam, torch.float32)), _ptr(u),
                                   _ptr(None if n_valid is None else _dev(n_valid, torch.int32)), int(chunk),
                                   _ptr(x_out), _ptr(n_accept), _ptr(ell), _ptr(dist2), _ptr(means), _stream())
    _check(code, "spec_verify_fused")
    return ((x_out, n_accept) + ((ell,) if want_logratio else ()) + ((means,) if want_means else ())
            + ((dist2,) if want_dist2 else ()))


_LOSS_WS = {}


def drafter_loss(eps_pred, eps_ref, f_pred, f_ref, lambda_f, lambda_s, beta=1.0, eps_cos=1e-8, out=None):
    """Drafter training objectives (Sec. 3.2) in one fused reduction.  eps_*: CUDA fp32 [n, d...]; f_*: CUDA fp32 or
    bf16 [n, n_tok, D].  Returns a CUDA float64 tensor (L_noise, L_feat, L_smooth, L_total)."""
    n, n_tok, D = f_pred.shape
    _dev(eps_pred, torch.float32); _dev(eps_ref, torch.float32); _dev(f_ref, f_pred.dtype)
    dtype = {torch.float32: FREE_FP32, torch.bfloat16: FREE_BF16}[f_pred.dtype]
    _dev(f_pred, f_pred.dtype)
    if out is None:
        out = torch.empty(4, dtype=torch.float64, device=f_pred.device)
    ws = _LOSS_WS.get(f_pred.device)
    if ws is None:
        ws = _LOSS_WS[f_pred.device] = torch.empty(lib().free_drafter_loss_workspace_bytes(), dtype=torch.uint8, device=f_pred.device)
    _check(lib().free_drafter_loss(dtype, n, n_tok, D, eps_pred.numel() // n, _ptr(eps_pred), _ptr(eps_ref), _ptr(f_pred), _ptr(f_ref),
                                   float(lambda_f), float(lambda_s), float(beta), float(eps_cos), _ptr(out), _ptr(ws), ws.numel(),
                                   _stream()), "free_drafter_loss")
    return out


def fit_lambda_profile(eps_delta, count=None, window=0):
    """Relaxation table (Sec. 3.4) from per-transition prediction deviations: host-side fit inside the library.
    eps_delta: [N] (index n-1 for transition n); count: [N] measurements per transition or None.  Returns fp32 [N]."""
    e = np.ascontiguousarray(eps_delta, dtype=np.float64)
    c = None if count is None else np.ascontiguousarray(count, dtype=np.int64)
    out = np.empty(len(e), dtype=np.float32)
    code = lib().free_fit_lambda_profile(e.ctypes.data_as(C.c_void_p), None if c is None else c.ctypes.data_as(C.c_void_p),
                                         len(e), int(window), out.ctypes.data_as(C.c_void_p))
    _check(code, "free_fit_lambda_profile")
    return out


class HostVerifier:
    """spec_verify on HOST buffers: pinned staging, host->device copies, the kernel, device->host copies
    of the result, all on the current stream (the end-to-end path of the benchmark)."""

    def __init__(self, B, K, d, relaxed=False):
        self.shape = (B, K, d)
        pin = lambda *s, dt=torch.float32: torch.empty(*s, dtype=dt, pin_memory=True)
        dev = lambda *s, dt=torch.float32: torch.empty(*s, dtype=dt, device="cuda")
        self.h = {n: pin(B, K, d) for n in ("m", "m_hat", "x_hat")}
        self.h.update({n: pin(B, K) for n in ("sigma2", "u")})
        if relaxed:
            self.h["lam"] = pin(B, K)
        self.d = {n: dev(*t.shape) for n, t in self.h.items()}
        self.x_out, self.n_accept = dev(B, d), dev(B, dt=torch.int32)
        self.h_x_out, self.h_n_accept = pin(B, d), pin(B, dt=torch.int32)
        self.h2d_bytes = sum(t.numel() * t.element_size() for t in self.h.values())
        self.d2h_bytes = self.h_x_out.numel() * 4 + self.h_n_accept.numel() * 4

    def load(self, **arrays):
        for n, a in arrays.items():
            self.h[n].copy_(torch.from_numpy(np.ascontiguousarray(a)).reshape(self.h[n].shape))

    def run(self):
        for n, t in self.h.items():
            self.d[n].copy_(t, non_blocking=True)
        spec_verify(self.d["m"], self.d["m_hat"], self.d["x_hat"], self.d["sigma2"], self.d["u"],
                    lam=self.d.get("lam"), x_out=self.x_out, n_accept=self.n_accept)
        self.h_x_out.copy_(self.x_out, non_blocking=True)
        self.h_n_accept.copy_(self.n_accept, non_blocking=True)
        return self.h_x_out, self.h_n_accept


def spec_verify_host(m, m_hat, x_hat, sigma2, u, lam=None):
    """Convenience wrapper: numpy in, numpy out, through HostVerifier."""
    B, K = m.shape[:2]
    d = int(np.prod(m.shape[2:]))
    hv = HostVerifier(B, K, d, relaxed=lam is not None)
    args = dict(m=m, m_hat=m_hat, x_hat=x_hat, sigma2=sigma2, u=u)
    if lam is not None:
        args["lam"] = lam
    hv.load(**args)
    x, n = hv.run()
    torch.cuda.current_stream().synchronize()
    return x.numpy().reshape((B,) + tuple(m.shape[2:])).copy(), n.numpy().copy()


# ------------------------------------------------------------------------------------------ model
_ACT = {FREE_FP32: torch.float32, FREE_BF16: torch.bfloat16}
_MATRICES = ("t_w1", "t_w2", "ada_w", "qkv_w", "proj_w", "fc1_w", "fc2_w", "fada_w", "fc_w")


def split_range(n_states: int, world: int, rank: int):
    """The packed states [lo, hi) that `rank` of `world` owns (free_split_range)."""
    lo, hi = C.c_int(0), C.c_int(0)
    _check(lib().free_split_range(int(n_states), int(world), int(rank), C.byref(lo), C.byref(hi)), "free_split_range")
    return lo.value, hi.value


def selftest_bounded_wait(limit_cycles: int = 100_000):
    """Runs the pipelines' bounded wait once on a barrier nothing signals (free_selftest_bounded_wait).  Returns
    (error word, SM cycles waited, library return code the word maps to)."""
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    waited = torch.zeros(1, dtype=torch.int64, device="cuda")
    _check(lib().free_selftest_bounded_wait(_ptr(err), int(limit_cycles), _ptr(waited), _stream()), "free_selftest_bounded_wait")
    torch.cuda.current_stream().synchronize()
    word = int(err.item()) & 0xFFFFFFFF
    return word, int(waited.item()), int(lib().free_device_error_code(word))


class DeviceSchedule:
    """The four reverse-process tables (see paper_2511_20390_b200.schedule) as fp32 device arrays."""

    def __init__(self, tables: dict, device="cuda"):
        self.N = int(len(tables["sigma2"]))
        self.t = {k: torch.tensor(np.asarray(v, dtype=np.float32), device=device) for k, v in tables.items()}
        self.desc = ScheduleDesc(self.N, *(self.t[k].data_ptr() for k in ("coef_x", "coef_eps", "sigma2", "t_embed_value")))


def _upload(weights: dict, dtype: int, device):
    out = {}
    for k, v in weights.items():
        if isinstance(v, torch.Tensor):
            t = v.to(device)
            out[k] = (t.to(_ACT[dtype]) if k in _MATRICES else t.to(torch.float32)).contiguous()
            continue
        t = torch.from_numpy(np.ascontiguousarray(v, dtype=np.float32)).to(device)
        out[k] = t.to(_ACT[dtype]).contiguous() if k in _MATRICES else t
    return out


def _block_desc(w):
    return BlockWeights(*(w[k].data_ptr() for k in ("ada_w", "ada_b", "qkv_w", "qkv_b", "proj_w", "proj_b",
                                                    "fc1_w", "fc1_b", "fc2_w", "fc2_b")))


class Model:
    """A target DiT (and optionally a drafter) resident on the GPU, bound to a library context.

    `shape` carries the dimensions (fields C, H, W, patch, D, depth, heads, n_classes, c_out, freq_dim,
    mlp_ratio); `weights` / `drafter_weights` are dicts of host arrays laid out as the public header
    describes.  dtype "fp32" or "bf16" selects the compute mode.
    """

    def __init__(self, shape, weights: dict, drafter_weights: dict | None = None, dtype: str = "bf16",
                 n_draft_blocks: int = 1, device="cuda"):
        self.shape, self.dtype = shape, {"fp32": FREE_FP32, "bf16": FREE_BF16}[dtype]
        self.act = _ACT[self.dtype]
        self.device = torch.device(device)
        self.w = _upload(weights, self.dtype, self.device)
        w = self.w
        md = ModelDesc(self.dtype, shape.C, shape.H, shape.W, shape.patch, shape.D, shape.depth, shape.heads,
                       shape.n_classes, shape.c_out, shape.freq_dim, shape.mlp_ratio,
                       *(w[k].data_ptr() for k in ("t_w1", "t_b1", "t_w2", "t_b2", "y_emb", "pe_w", "pe_b", "pos")),
                       _block_desc(w), *(w[k].data_ptr() for k in ("fada_w", "fada_b", "fin_w", "fin_b")))
        dd = None
        self.wd = None
        if drafter_weights is not None:
            self.wd = _upload(drafter_weights, self.dtype, self.device)
            wd = self.wd
            dd = DrafterDesc(n_draft_blocks, wd["fc_w"].data_ptr(), wd["fc_b"].data_ptr(), _block_desc(wd),
                             *(wd[k].data_ptr() for k in ("fada_w", "fada_b", "fin_w", "fin_b")))
        self.ctx = C.c_void_p()
        _check(lib().free_create(C.byref(md), C.byref(dd) if dd is not None else None, C.byref(self.ctx)), "free_create")
        self._ws = None

    def __del__(self):
        try:
            if getattr(self, "ctx", None):
                lib().free_destroy(self.ctx)
                self.ctx = None
        except Exception:
            pass

    def workspace(self, n_states: int):
        need = lib().free_workspace_bytes(self.ctx, int(n_states))
        if self._ws is None or self._ws.numel() < need:
            self._ws = None
            self._ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        return self._ws

    @classmethod
    def random(cls, shape, seed: int, dtype: str = "bf16", with_drafter: bool = True, n_draft_blocks: int = 1,
               std: float = 0.02, device="cuda"):
        """Random-init model whose weights are drawn on the device (no host copy): for timing runs, where the
        values only need the right shapes and scale.  The fixed position table comes from `synth`."""
        import synth
        g = torch.Generator(device=device)
        g.manual_seed(int(seed))
        D, F = shape.D, shape.mlp_ratio * shape.D
        act = _ACT[{"fp32": FREE_FP32, "bf16": FREE_BF16}[dtype]]

        def mat(*s):
            return (torch.randn(*s, generator=g, device=device, dtype=torch.float32) * std).to(act)

        def vec(*s):
            return torch.randn(*s, generator=g, device=device, dtype=torch.float32) * std

        def blocks(n):
            return {"ada_w": mat(n, 6 * D, D), "ada_b": vec(n, 6 * D), "qkv_w": mat(n, 3 * D, D), "qkv_b": vec(n, 3 * D),
                    "proj_w": mat(n, D, D), "proj_b": vec(n, D), "fc1_w": mat(n, F, D), "fc1_b": vec(n, F),
                    "fc2_w": mat(n, D, F), "fc2_b": vec(n, D), "fada_w": mat(2 * D, D), "fada_b": vec(2 * D),
                    "fin_w": vec(shape.out_dim, D), "fin_b": vec(shape.out_dim)}
        w = {"t_w1": mat(D, shape.freq_dim), "t_b1": vec(D), "t_w2": mat(D, D), "t_b2": vec(D),
             "y_emb": vec(shape.n_classes + 1, D), "pe_w": vec(D, shape.patch_dim), "pe_b": vec(D),
             "pos": torch.from_numpy(synth.pos_embed_2d(shape)).to(device)}
        w.update(blocks(shape.depth))
        wd = None
        if with_drafter:
            wd = {"fc_w": mat(D, 2 * D), "fc_b": vec(D)}
            wd.update(blocks(n_draft_blocks))
        return cls(shape, w, wd, dtype=dtype, n_draft_blocks=n_draft_blocks, device=device)

    def device_error(self) -> int:
        """The device error word of the last call that used the workspace (0 = no bounded wait gave up).
        Synchronises the current stream."""
        if self._ws is None:
            return 0
        torch.cuda.current_stream().synchronize()
        return int(self._ws[:4].view(torch.int32).item())

    def profile_begin(self):
        _check(lib().free_profile_begin(self.ctx), "free_profile_begin")

    def profile_end(self):
        """Per-kernel-class totals since profile_begin(): list of dicts name / launches / ms / work."""
        buf = (ProfEntry * 32)()
        n = C.c_int(0)
        _check(lib().free_profile_end(self.ctx, buf, 32, C.byref(n)), "free_profile_end")
        return [{"name": buf[i].name.decode(), "launches": buf[i].launches, "ms": buf[i].ms, "work": buf[i].work}
                for i in range(n.value)]

    def spec_round(self, x_cur, cursor, labels, sched, K, cfg_scale, noise_target, noise_draft=None, uniforms=None,
                   lam=None, x_next=None, cursor_next=None, n_accept=None):
        """One round of Algorithm 1 (asynchronous).  Returns (x_next, cursor_next, n_accept)."""
        B = x_cur.shape[0]
        _dev(x_cur, torch.float32); _dev(cursor, torch.int32); _dev(labels, torch.int32)
        prm = SpecParams(int(K), float(cfg_scale), None if lam is None else _dev(lam, torch.float32).data_ptr())
        x_next = torch.empty_like(x_cur) if x_next is None else x_next
        cursor_next = torch.empty_like(cursor) if cursor_next is None else cursor_next
        n_accept = torch.zeros(B, dtype=torch.int32, device=x_cur.device) if n_accept is None else n_accept
        ws = self.workspace(B * max(int(K), 1))
        _check(lib().free_spec_round(self.ctx, B, _ptr(x_cur), _ptr(cursor), _ptr(labels), C.byref(sched.desc), C.byref(prm),
                                     _ptr(noise_target), _ptr(noise_draft), _ptr(uniforms), _ptr(x_next), _ptr(cursor_next),
                                     _ptr(n_accept), _ptr(ws), ws.numel(), _stream()), "free_spec_round")
        return x_next, cursor_next, n_accept

    def spec_round_begin(self, x_cur, cursor, labels, sched, K, cfg_scale, noise_target, noise_draft, uniforms, rank, world,
                         eps_all=None, lam=None):
        """First half of a round whose packed pass is partitioned over `world` ranks (free_spec_round_begin): target step,
        drafter steps, and the packed pass over this rank's states, written into eps_all [B*K, G, C, H, W] in place.
        Returns (eps_all, lo, hi)."""
        B, sh = x_cur.shape[0], self.shape
        _dev(x_cur, torch.float32); _dev(cursor, torch.int32); _dev(labels, torch.int32)
        prm = SpecParams(int(K), float(cfg_scale), None if lam is None else _dev(lam, torch.float32).data_ptr())
        lo, hi = split_range(B * int(K), world, rank)
        if eps_all is None:
            eps_all = torch.empty((B * int(K), self.guided(cfg_scale), sh.C, sh.H, sh.W), dtype=torch.float32, device=x_cur.device)
        ws = self.workspace(B * int(K))
        _check(lib().free_spec_round_begin(self.ctx, B, _ptr(x_cur), _ptr(cursor), _ptr(labels), C.byref(sched.desc), C.byref(prm),
                                           _ptr(noise_target), _ptr(noise_draft), _ptr(uniforms), int(rank), int(world), _ptr(eps_all),
                                           _ptr(ws), ws.numel(), _stream()), "free_spec_round_begin")
        return eps_all, lo, hi

    def spec_round_finish(self, eps_all, labels, sched, K, cfg_scale, noise_target, noise_draft, uniforms, like, lam=None,
                          x_next=None, cursor_next=None, n_accept=None):
        """Second half (free_spec_round_finish): verification and cursor update on the gathered predictions.  `like` is the
        round's x_cur (shape and device of the outputs).  Returns (x_next, cursor_next, n_accept)."""
        B = like.shape[0]
        prm = SpecParams(int(K), float(cfg_scale), None if lam is None else _dev(lam, torch.float32).data_ptr())
        x_next = torch.empty_like(like) if x_next is None else x_next
        cursor_next = torch.empty(B, dtype=torch.int32, device=like.device) if cursor_next is None else cursor_next
        n_accept = torch.zeros(B, dtype=torch.int32, device=like.device) if n_accept is None else n_accept
        ws = self.workspace(B * int(K))
        _check(lib().free_spec_round_finish(self.ctx, B, _ptr(labels), C.byref(sched.desc), C.byref(prm), _ptr(noise_target),
                                            _ptr(noise_draft), _ptr(uniforms), _ptr(eps_all), _ptr(x_next), _ptr(cursor_next),
                                            _ptr(n_accept), _ptr(ws), ws.numel(), _stream()), "free_spec_round_finish")
        return x_next, cursor_next, n_accept

    def spec_round_split(self, x_cur, cursor, labels, sched, K, cfg_scale, noise_target, noise_draft, uniforms, rank, world,
                         lam=None, eps_all=None, x_next=None, cursor_next=None, n_accept=None, group=None):
        """One round with the packed pass partitioned over the `world` ranks of a torch.distributed group: begin, an
        all-gather of the noise predictions (every rank contributes the slice it computed; NCCL on GPUs), finish.  Every
        rank must pass identical inputs.  Returns (x_next, cursor_next, n_accept), identical on all ranks."""
        eps_all, lo, hi = self.spec_round_begin(x_cur, cursor, labels, sched, K, cfg_scale, noise_target, noise_draft, uniforms,
                                                rank, world, eps_all=eps_all, lam=lam)
        if world > 1:
            import torch.distributed as dist
            # the rank's own slice is sent from a copy: not every backend takes an input that aliases the output
            dist.all_gather_into_tensor(eps_all, eps_all[lo:hi].clone(), group=group)
        return self.spec_round_finish(eps_all, labels, sched, K, cfg_scale, noise_target, noise_draft, uniforms, x_cur, lam=lam,
                                      x_next=x_next, cursor_next=cursor_next, n_accept=n_accept)

    @staticmethod
    def guided(cfg_scale: float) -> int:
        return 2 if (cfg_scale > 0 and cfg_scale != 1.0) else 1

    def dit_verify_pass(self, x, t_idx, labels, cfg_scale, sched: DeviceSchedule, want_eps=False, want_feat=False,
                        mean_out=None):
        """One packed target pass.  x: CUDA fp32 [n, C, H, W]; t_idx, labels: int32 [n].
        Returns mean [n,C,H,W] (+ eps, + feat [n,G,n_tok,D] when asked)."""
        sh = self.shape
        n = x.shape[0]
        _dev(x, torch.float32); _dev(t_idx, torch.int32); _dev(labels, torch.int32)
        mean = torch.empty_like(x) if mean_out is None else mean_out
        eps = torch.empty_like(x) if want_eps else None
        feat = (torch.empty((n, self.guided(cfg_scale), sh.n_tok, sh.D), dtype=self.act, device=x.device)
                if want_feat else None)
        ws = self.workspace(n)
        _check(lib().dit_verify_pass(self.ctx, n, _ptr(x), _ptr(t_idx), _ptr(labels), float(cfg_scale),
                                     C.byref(sched.desc), _ptr(mean), _ptr(eps), _ptr(feat),
                                     _ptr(ws), ws.numel(), _stream()), "dit_verify_pass")
        out = (mean,) + ((eps,) if want_eps else ()) + ((feat,) if want_feat else ())
        return out if len(out) > 1 else mean

    def dit_verify_pass_raw(self, x, t_idx, labels, guidance: bool, sched: DeviceSchedule, want_feat=False):
        """The packed target pass stopped at the network output: returns eps [n, G, C, H, W] (+ feat)."""
        sh = self.shape
        n, G = x.shape[0], 2 if guidance else 1
        _dev(x, torch.float32); _dev(t_idx, torch.int32); _dev(labels, torch.int32)
        head = torch.empty((n, G, sh.C, sh.H, sh.W), dtype=torch.float32, device=x.device)
        feat = torch.empty((n, G, sh.n_tok, sh.D), dtype=self.act, device=x.device) if want_feat else None
        ws = self.workspace(n)
        _check(lib().dit_verify_pass_raw(self.ctx, n, _ptr(x), _ptr(t_idx), _ptr(labels), int(bool(guidance)),
                                         C.byref(sched.desc), _ptr(head), _ptr(feat), _ptr(ws), ws.numel(), _stream()),
               "dit_verify_pass_raw")
        return (head, feat) if want_feat else head

    def draft_step(self, x_prev, f_prev, t_idx, labels, cfg_scale, sched: DeviceSchedule, noise):
        """One drafter step.  Returns (m_hat, x_hat, f_next)."""
        n = x_prev.shape[0]
        _dev(x_prev, torch.float32); _dev(f_prev, self.act); _dev(noise, torch.float32)
        m_hat, x_hat, f_next = torch.empty_like(x_prev), torch.empty_like(x_prev), torch.empty_like(f_prev)
        ws = self.workspace(n)
        _check(lib().draft_step(self.ctx, n, _ptr(x_prev), _ptr(f_prev), _ptr(_dev(t_idx, torch.int32)),
                                _ptr(_dev(labels, torch.int32)), float(cfg_scale), C.byref(sched.desc), _ptr(noise),
                                _ptr(m_hat), _ptr(x_hat), _ptr(f_next), _ptr(ws), ws.numel(), _stream()), "draft_step")
        return m_hat, x_hat, f_next

    def uncertainty_profile(self, x0, labels, sched: DeviceSchedule, K, cfg_scale, noise_target, noise_draft, uniforms, lam=None):
        """The offline run of Sec. 3.4.  Returns (eps_delta [N], accept_prob [N], count [N]) as numpy arrays."""
        B, N = x0.shape[0], sched.desc.N
        _dev(x0, torch.float32); _dev(labels, torch.int32); _dev(noise_target, torch.float32)
        prm = SpecParams(int(K), float(cfg_scale), None if lam is None else _dev(lam, torch.float32).data_ptr())
        dev, acc, cnt = np.zeros(N), np.zeros(N), np.zeros(N, np.int64)
        ws = self.workspace(B * max(int(K), 1))
        _check(lib().free_uncertainty_profile(self.ctx, B, _ptr(x0), _ptr(labels), C.byref(sched.desc), C.byref(prm),
                                              _ptr(noise_target), _ptr(noise_draft), _ptr(uniforms),
                                              dev.ctypes.data_as(C.c_void_p), acc.ctypes.data_as(C.c_void_p),
                                              cnt.ctypes.data_as(C.c_void_p), _ptr(ws), ws.numel(), _stream()),
               "free_uncertainty_profile")
        return dev, acc, cnt

    def sample_trajectory(self, x0, labels, sched: DeviceSchedule, K, cfg_scale, noise_target, noise_draft=None,
                          uniforms=None, lam=None, use_graph=False):
        """Algorithm 1 for a batch.  Returns (x_final, stats dict)."""
        B = x0.shape[0]
        _dev(x0, torch.float32); _dev(labels, torch.int32); _dev(noise_target, torch.float32)
        prm = SpecParams(int(K), float(cfg_scale), None if lam is None else _dev(lam, torch.float32).data_ptr(), int(bool(use_graph)))
        st = TrajStats()
        x_final = torch.empty_like(x0)
        ws = self.workspace(B * max(int(K), 1))
        _check(lib().sample_trajectory(self.ctx, B, _ptr(x0), _ptr(labels), C.byref(sched.desc), C.byref(prm),
                                       _ptr(noise_target), _ptr(noise_draft), _ptr(uniforms), _ptr(x_final),
                                       C.byref(st), _ptr(ws), ws.numel(), _stream()), "sample_trajectory")
        stats = {k: getattr(st, k) for k in ("rounds", "target_calls", "draft_calls", "accepted", "rejected",
                                             "parallel_efficiency", "graph_rounds")}
        stats["accept_hist"] = list(st.accept_hist)[:int(K) + 1]
        return x_final, stats


# ------------------------------------------------------------------------------------------ single ops
def op_linear(A, W, bias=None, epilogue=EPI_BIAS, out_dtype=None, resid=None, gate=None, rows_per_seq=1):
    """epilogue(A W^T + bias) with the library's linear-layer kernel (fp32: CUDA cores, bf16: tcgen05)."""
    dtype = FREE_FP32 if A.dtype == torch.float32 else FREE_BF16
    M, K = A.shape
    N = W.shape[0]
    od = dtype if out_dtype is None else out_dtype
    out = None if epilogue == EPI_GATE_RESIDUAL else torch.empty((M, N), dtype=_ACT[od], device=A.device)
    ws = torch.zeros(lib().free_op_linear_workspace_bytes(), dtype=torch.uint8, device=A.device)
    _check(lib().free_op_linear(dtype, epilogue, od, M, N, K, _ptr(A), _ptr(W), _ptr(bias), _ptr(out), _ptr(resid),
                                _ptr(gate), 0 if gate is None else gate.stride(0), rows_per_seq,
                                _ptr(ws), ws.numel(), _stream()), "free_op_linear")
    err = int(ws[:4].view(torch.int32).item())
    if err:
        raise FreeError(-8, f"free_op_linear (device error word {err:#x})")
    return resid if epilogue == EPI_GATE_RESIDUAL else out


def op_ln_modulate(x, shift, scale, rows_per_seq, out_dtype=FREE_FP32):
    M, D = x.shape
    y = torch.empty((M, D), dtype=_ACT[out_dtype], device=x.device)
    _check(lib().free_op_ln_modulate(out_dtype, M, D, rows_per_seq, _ptr(x), _ptr(shift), _ptr(scale),
                                     shift.stride(0), _ptr(y), _stream()), "free_op_ln_modulate")
    return y


_DTYPE = {torch.float32: FREE_FP32, torch.bfloat16: FREE_BF16}


def _code(dtype):
    """FREE_* code of a torch dtype (the codes themselves pass through)."""
    c = _DTYPE.get(dtype)
    if c is None:
        if dtype not in (FREE_FP32, FREE_BF16):
            raise ValueError(f"expected float32 or bfloat16, got {dtype}")
        c = dtype
    return c


# The calls below are short on the GPU (a few us for small batches), so the host's part is kept short: integers for
# pointers, device indices instead of device objects, the raw handle of the current stream.
def _device_of(first, *others):
    d = first.get_device()                                         # -1 on the host
    for t in others:
        if t is not None and t.get_device() != d:
            raise ValueError("expected CUDA tensors on one device")
    if d < 0:
        raise ValueError("expected CUDA tensors on one device")
    return d


def _like(t, dtype):
    """Uninitialised contiguous tensor of t's shape and device (the cheapest of torch's ways to make one)."""
    return torch.empty_like(t, dtype=dtype, memory_format=torch.contiguous_format)


def _adr(t):
    return None if t is None else t.data_ptr()


def _launch(what, device, *args):
    """Library call `what` with `device` current, on the stream that is current there (its last argument)."""
    fn = getattr(_LIB or lib(), what)
    if device == torch._C._cuda_getDevice():
        code = fn(*args, torch._C._cuda_getCurrentRawStream(device))
    else:
        with torch.cuda.device(device):
            code = fn(*args, torch._C._cuda_getCurrentRawStream(device))
    if code != 0:
        raise FreeError(code, what)


def _rows(t, M, D, what):
    """Row stride of a [M, D] matrix whose rows are dense."""
    if t.shape != (M, D) or (D > 1 and t.stride(1) != 1):
        raise ValueError(f"{what}: expected a [{M}, {D}] matrix with dense rows")
    return t.stride(0) if M > 1 else max(D, t.stride(0))


def _layout(t):
    """(size, stride) of the axes that a tensor's addresses depend on, and the elements from its first to behind its last."""
    axes = [(n, s) for n, s in zip(t.shape, t.stride()) if n > 1]
    return axes, 1 + sum((n - 1) * s for n, s in axes)


def _meet(a, b):
    """Whether two tensors share memory.  Exact where both fill their range or are laid out alike (nested strides, as views
    of a matrix have); False where the layouts cannot be compared."""
    if a.numel() == 0 or b.numel() == 0:
        return False
    (la, na), (lb, nb) = _layout(a), _layout(b)
    pa, pb, size = a.data_ptr(), b.data_ptr(), a.element_size()
    if pa + na * size <= pb or pb + nb * b.element_size() <= pa:
        return False
    if na == a.numel() and nb == b.numel():
        return True
    if la != lb or a.dtype != b.dtype:
        return False
    apart, rest = divmod(pb - pa, size)
    if rest:
        return True
    left = {apart}                                                 # the distance, less whole steps along one axis after the other
    for n, s in sorted(la, key=lambda v: -v[1]):
        if s > 0:
            left = {d - k * s for d in left for k in (d // s, d // s + 1) if abs(k) < n}
    return 0 in left


def _end(t):
    """Address behind a tensor's last element."""
    return t.data_ptr() + (t.nbytes if t.is_contiguous() else _layout(t)[1] * t.element_size())


def _apart(out, what, over, *others):
    """Refuses a result that the caller gave and that shares memory with an input; `over` are the inputs that it may replace
    element for element."""
    lo, hi = out.data_ptr(), None
    for i, t in enumerate(over + others):
        if t is None or (i < len(over) and (t is out or (t.data_ptr() == lo and t.dtype == out.dtype and t.shape == out.shape and t.stride() == out.stride()))):
            continue
        if hi is None:
            hi = _end(out)
        p = t.data_ptr()
        if p >= hi or (p < lo and _end(t) <= lo):                  # the usual case, found out cheaply
            continue
        if i < len(over) and p == lo and t.dtype == out.dtype and _layout(t) == _layout(out):      # strides of single entries differ
            continue
        if _meet(out, t):
            raise ValueError(f"{what}: overlaps an input")


def _group_rows(t, groups, D, what):
    """Group stride of a [D] or [groups, D] fp32 table (rows of an adaLN table may be far apart)."""
    n = t.dim()
    if t.dtype != torch.float32 or n > 2 or n < 1 or t.shape[n - 1] != D or (D > 1 and t.stride(n - 1) != 1):
        raise ValueError(f"{what}: expected fp32 [{groups}, {D}] with dense rows")
    if n == 1 or t.shape[0] == 1:
        return 0                                                   # one row for every group
    if t.shape[0] != groups:
        raise ValueError(f"{what}: expected fp32 [{groups}, {D}]")
    return t.stride(0)


def _groups(M, rows_per_group):
    rows = M if rows_per_group is None else int(rows_per_group)
    if rows < 0 or (rows == 0 and M > 0) or (rows > 0 and M % rows):
        raise ValueError(f"{M} rows are not whole groups of {rows}")
    return (1, 0) if rows == 0 else (M // rows, rows)


def op_layer_norm(x, weight=None, bias=None, rows_per_group=None, unit_offset=False, eps=1e-6, out_dtype=None, want_stats=False, out=None):
    """Layer norm of the rows of x (CUDA fp32 or bf16 [M, D], dense rows any distance apart) with a weight and bias (fp32 [D],
    or [groups, D] for groups of `rows_per_group` consecutive rows; unit_offset: the weight is stored as an offset from one, as
    adaLN's scale).  Returns y [M, D] in out_dtype (default: x's), and with want_stats also (mean, 1 / sqrt(var + eps)) as fp32
    [M, 2], what op_layer_norm_bwd needs.  x and out begin on 16 bytes; weight and bias rows of several groups lie the same distance
    apart; out may be x.  Like all operators here it records nothing for autograd."""
    if x.dim() != 2:
        raise ValueError("x: expected a matrix")
    M, D = x.shape
    groups, rows = _groups(M, rows_per_group)
    dev = _device_of(x, weight, bias, out)
    xc, xs = _code(x.dtype), _rows(x, M, D, "x")
    ms = 0 if weight is None else _group_rows(weight, groups, D, "weight")
    if bias is not None:
        bs = _group_rows(bias, groups, D, "bias")
        if weight is not None and bs != ms:
            raise ValueError("weight and bias need the same distance between groups")
        ms = bs
    if out is None:
        yc = xc if out_dtype is None else _code(out_dtype)
        out = _like(x, _ACT[yc])
        ys = D
    else:
        yc, ys = _code(out.dtype), _rows(out, M, D, "out")
        if out_dtype is not None and _code(out_dtype) != yc:
            raise ValueError("out_dtype: out has another type")
        _apart(out, "out", (x,), weight, bias)
    stats = x.new_empty((M, 2), dtype=torch.float32) if want_stats else None
    _launch("free_op_layer_norm", dev, xc, yc, groups, rows, D, x.data_ptr(), xs, _adr(weight), _adr(bias), ms, 1 if unit_offset else 0, eps,
            out.data_ptr(), ys, _adr(stats))
    return (out, stats) if want_stats else out


def op_layer_norm_bwd(x, dy, stats, weight=None, rows_per_group=None, unit_offset=False, dres=None, want_dweight=True, want_dbias=True,
                      dx=None):
    """Gradients of op_layer_norm from dy [M, D] and the stats it kept.  dres: gradient of x from another path, added to dx.
    Returns (dx in x's dtype, dweight, dbias), the last two fp32 [groups, D], or None where not wanted; a weight that all groups share
    has their sum as its gradient (or one group, of all rows).  dx may be x, dy or dres."""
    if x.dim() != 2:
        raise ValueError("x: expected a matrix")
    M, D = x.shape
    groups, rows = _groups(M, rows_per_group)
    dev = _device_of(x, dy, stats, weight, dres, dx)
    if stats.dtype != torch.float32 or stats.shape != (M, 2) or not stats.is_contiguous():
        raise ValueError("stats: expected the contiguous fp32 [M, 2] of the forward call")
    if (dres is not None and dres.dtype != x.dtype) or (dx is not None and dx.dtype != x.dtype):
        raise ValueError("dres, dx: expected x's dtype")
    if dx is None:
        dx = _like(x, x.dtype)
    else:
        _apart(dx, "dx", (x, dy, dres), stats, weight)
    dw = stats.new_empty((groups, D)) if want_dweight else None
    db = stats.new_empty((groups, D)) if want_dbias else None
    need = lib().free_op_layer_norm_bwd_workspace_bytes(groups, rows, D) if want_dweight or want_dbias else 0
    ws = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
    _launch("free_op_layer_norm_bwd", dev, _code(x.dtype), _code(dy.dtype), groups, rows, D, x.data_ptr(), _rows(x, M, D, "x"),
            dy.data_ptr(), _rows(dy, M, D, "dy"), stats.data_ptr(), _adr(weight),
            0 if weight is None else _group_rows(weight, groups, D, "weight"), 1 if unit_offset else 0,
            _adr(dres), 0 if dres is None else _rows(dres, M, D, "dres"), dx.data_ptr(), _rows(dx, M, D, "dx"),
            _adr(dw), _adr(db), D, _adr(ws), need)
    return dx, dw, db


class RmsNorm(typing.NamedTuple):
    """Results of op_rms_norm: y; the scales of an 8-bit y; the new residual stream; 1 / sqrt(mean square + eps).  None where there is none."""
    y: torch.Tensor
    scales: torch.Tensor | None
    residual: torch.Tensor | None
    rstd: torch.Tensor | None


def _tokens(t, shape, what):
    """(token stride, head stride) of a [tokens, D] or [tokens, heads, D] tensor whose rows are dense."""
    st, D = t.stride(), shape[-1]
    if t.shape != shape or (D > 1 and st[-1] != 1):
        raise ValueError(f"{what}: expected {list(shape)} with dense rows")
    if len(st) == 2:
        return (st[0] if shape[0] > 1 else max(D, st[0])), 0
    H = shape[1]
    head = st[1] if H > 1 else D
    return (st[0] if shape[0] > 1 else max(H * head, st[0])), head


def op_rms_norm(x, weight=None, residual=None, rows_per_group=None, unit_offset=False, eps=1e-6, out_dtype=None, scale_block=None,
                want_rstd=False, out=None, residual_out=None):
    """Root-mean-square norm of the rows of x (CUDA fp32 or bf16 [M, D] with dense rows any distance apart, or the heads [tokens, heads, D]
    of a packed projection), y = h / sqrt(mean(h^2) + eps) * weight with h = x + residual (fp32 or bf16 [M, D]; not for heads).  weight: fp32
    [D], or [groups, D] for groups of `rows_per_group` consecutive rows (of a head's: tokens times heads); unit_offset: stored as an
    offset from one.  out_dtype (default: x's) may be torch.float8_e4m3fn: y then is a value times its scale, fp32 [M, runs], one
    for every scale_block (128; None: the row's) columns.  Returns RmsNorm(y, scales, residual, rstd): residual is h in the residual's type,
    a new tensor unless residual_out is given (the residual itself: in place); rstd, fp32 with want_rstd, is what op_rms_norm_bwd
    needs.  out may be x."""
    shape = x.shape
    nd = len(shape)
    if nd not in (2, 3):
        raise ValueError("x: expected [rows, D] or [tokens, heads, D]")
    M, D, H = shape[0], shape[-1], 1
    if nd == 3:
        H = shape[1]
        M *= H
    groups, rows = (1, M) if rows_per_group is None else _groups(M, rows_per_group)
    dev = _device_of(x, weight, residual, out, residual_out)
    xc, (xt, xh) = _code(x.dtype), _tokens(x, shape, "x")
    ms = 0 if weight is None else _group_rows(weight, groups, D, "weight")
    if out is None:
        out = _like(x, x.dtype if out_dtype is None else _ACT.get(out_dtype, out_dtype))
        yt, yh = H * D, D
    else:
        if out_dtype is not None and _ACT.get(out_dtype, out_dtype) != out.dtype:
            raise ValueError("out_dtype: out has another type")
        _apart(out, "out", (x,), weight, residual)
        yt, yh = _tokens(out, shape, "out")
    scales = None
    if out.dtype == torch.float8_e4m3fn:
        yc, runs = FREE_E4M3, 1
        if nd == 3:
            raise ValueError("out_dtype: 8-bit results are of rows [M, D]")
        if scale_block not in (None, 128):
            raise ValueError("scale_block: expected 128, or None for a scale per row")
        if scale_block:
            runs = -(-D // 128)
        scales = x.new_empty((M, runs), dtype=torch.float32)
    else:
        yc, runs = _code(out.dtype), 0
        if scale_block is not None:
            raise ValueError("scale_block: only for 8-bit results")
    rc = rs = hs = 0
    if residual is not None:
        if nd == 3:
            raise ValueError("residual: expected rows, not heads")
        rc, rs = _code(residual.dtype), _rows(residual, M, D, "residual")
        if residual_out is None:
            residual_out, hs = _like(residual, residual.dtype), D
        elif residual_out.dtype != residual.dtype:
            raise ValueError("residual_out: expected the residual's dtype")
        else:
            _apart(residual_out, "residual_out", (residual,), x, weight)
            _apart(residual_out, "residual_out", (), out)
            hs = _rows(residual_out, M, D, "residual_out")
    elif residual_out is not None:
        raise ValueError("residual_out: there is no residual")
    rstd = x.new_empty(M, dtype=torch.float32) if want_rstd else None
    _launch("free_op_rms_norm", dev, xc, rc, yc, groups, rows, H, D, x.data_ptr(), xt, xh, _adr(residual), rs, _adr(residual_out), hs,
            _adr(weight), ms, 1 if unit_offset else 0, eps, out.data_ptr(), yt, yh, _adr(scales), runs, scale_block or 0, _adr(rstd))
    return RmsNorm(out, scales, residual_out, rstd)


def op_rms_norm_bwd(h, dy, rstd, weight=None, rows_per_group=None, unit_offset=False, dres=None, want_dweight=True, dx=None):
    """Gradients of op_rms_norm from dy (like h, fp32 or bf16), the h that it normed (its residual, or x where there was none) and the
    rstd it kept.  dres: gradient of h from another path, added to dx.  Returns (dx in h's dtype, which is the gradient of x and of the
    residual alike, dweight fp32 [groups, D] or None).  dx may be h, dy or dres.  Heads [tokens, heads, D] of more than 128 columns (256 where
    D is even) have to lie evenly apart."""
    nd = h.dim()
    if nd not in (2, 3):
        raise ValueError("h: expected [rows, D] or [tokens, heads, D]")
    shape = h.shape
    H, D = (shape[1] if nd == 3 else 1), shape[-1]
    M = shape[0] * H
    groups, rows = _groups(M, rows_per_group)
    dev = _device_of(h, dy, rstd, weight, dres, dx)
    if rstd.dtype != torch.float32 or rstd.shape != (M,) or not rstd.is_contiguous():
        raise ValueError("rstd: expected the contiguous fp32 [rows] of the forward call")
    if (dres is not None and dres.dtype != h.dtype) or (dx is not None and dx.dtype != h.dtype):
        raise ValueError("dres, dx: expected h's dtype")
    if dx is None:
        dx = _like(h, h.dtype)
    else:
        _apart(dx, "dx", (h, dy, dres), rstd, weight)
    dw = rstd.new_empty((groups, D)) if want_dweight else None
    need = lib().free_op_rms_norm_bwd_workspace_bytes(groups, rows, D) if want_dweight else 0
    ws = torch.empty(need, dtype=torch.uint8, device=h.device) if need else None
    _launch("free_op_rms_norm_bwd", dev, _code(h.dtype), _code(dy.dtype), groups, rows, H, D, h.data_ptr(), *_tokens(h, shape, "h"),
            dy.data_ptr(), *_tokens(dy, shape, "dy"), rstd.data_ptr(), _adr(weight), 0 if weight is None else _group_rows(weight, groups, D, "weight"),
            1 if unit_offset else 0, _adr(dres), *((0, 0) if dres is None else _tokens(dres, shape, "dres")), dx.data_ptr(),
            *_tokens(dx, shape, "dx"), _adr(dw), D, _adr(ws), need)
    return dx, dw


ROPE_PAIRING = {"interleaved": 0, "halves": 1}
_AXES = {n: C.c_int32 * n for n in range(1, 5)}


def op_rope_axes(x, pos, axis_dims, base=10000.0, pairing="interleaved", joint_freq=False, inverse=False, out=None):
    """Rotary positions with len(axis_dims) axes on x (CUDA fp32 or bf16 [n_seq, n_tok, heads, d_head], any strides with dense
    heads: q and k may be views into the packed projection); axis_dims[a] elements of a head follow axis a.  pos: fp32 [n_tok, n_axes], or
    [n_seq, n_tok, n_axes].  inverse turns back (the gradient of the forward call).  out=x rotates in place.  Returns the
    rotated heads, contiguous unless `out` is given."""
    if x.dim() != 4 or (x.shape[3] > 1 and x.stride(3) != 1):
        raise ValueError("x: expected [n_seq, n_tok, heads, d_head] with dense heads")
    if pairing not in ROPE_PAIRING:
        raise ValueError("pairing: expected 'interleaved' or 'halves'")
    n_axes = len(axis_dims)
    if n_axes not in _AXES:
        raise ValueError("axis_dims: expected one to four axes")
    if max(axis_dims) > 0x7fffffff or min(axis_dims) < -0x80000000:          # an array of C ints would cut them
        raise ValueError("axis_dims: expected even widths that fit into a head")
    shape = n_seq, n_tok, heads, d_head = x.shape
    dev = _device_of(x, pos, out)
    if pos.dtype != torch.float32 or not pos.is_contiguous() or (pos.shape != (n_tok, n_axes) and pos.shape != (n_seq, n_tok, n_axes)):
        raise ValueError("pos: expected contiguous fp32 [n_tok, n_axes] or [n_seq, n_tok, n_axes]")
    xs = x.stride()
    if out is None:
        out = _like(x, x.dtype)
        hs = heads * d_head
        ys = (n_tok * hs, hs, d_head)
    else:
        if out.shape != shape or out.dtype != x.dtype or (d_head > 1 and out.stride(3) != 1):
            raise ValueError("out: expected x's shape and dtype with dense heads")
        _apart(out, "out", (x,))
        ys = out.stride()
    _launch("free_op_rope_axes", dev, _code(x.dtype), ROPE_PAIRING[pairing], 1 if joint_freq else 0, 1 if inverse else 0, n_seq, n_tok, heads,
            d_head, n_axes, _AXES[n_axes](*axis_dims), base, pos.data_ptr(), n_tok * n_axes if pos.dim() == 3 else 0,
            x.data_ptr(), xs[0], xs[1], xs[2], out.data_ptr(), ys[0], ys[1], ys[2])
    return out


ACTIVATIONS = {"silu": 0, "gelu": 1}
_ERROR_WORDS = {}
_ERROR_WORDS_LOCK = threading.Lock()


def _error_word(device):
    """The device error word that the calls of the gated layer and of the attention to an encoder's states on a device share:
    zeroed once, OR-ed into by a kernel whose bounded wait gave up, never cleared in between (so calls on several streams and
    replays of captured graphs may share it)."""
    w = _ERROR_WORDS.get(device)
    if w is None:
        with _ERROR_WORDS_LOCK:                                    # threads that come first at once share one word
            w = _ERROR_WORDS.get(device)
            if w is None:
                with torch.cuda.device(device):
                    if torch.cuda.is_current_stream_capturing():
                        raise RuntimeError("call the operator once on this device before capturing it into a CUDA graph")
                    w = torch.zeros(1, dtype=torch.int32, device="cuda")
                    torch.cuda.current_stream().synchronize()      # zero before any other stream can use it
                _ERROR_WORDS[device] = w
    return w


def op_device_error(device=None):
    """Waits for `device` and returns the error word of the calls of the gated layer and of op_cross_attention on it so far (0: no bounded wait gave up)."""
    index = None if device is None else torch.device(device).index
    if index is None:
        index = torch.cuda.current_device()
    if index not in _ERROR_WORDS:
        return 0
    torch.cuda.synchronize(index)
    return int(_ERROR_WORDS[index].item()) & 0xFFFFFFFF


def _dense(t, dtype, shape, what):
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous {dtype} tensor of shape {list(shape)}")


def op_gated_linear(x, w, bias=None, act="silu", want_preact=False, out=None):
    """First half of a gated feed-forward layer, h = act(z[:, :F]) * z[:, F:] with z = x w^T + bias, in one kernel.  x: CUDA
    fp32 or bf16 [M, K]; w [2F, K], the gate rows and then the up rows; bias fp32 [2F]; act "silu" or "gelu" (tanh form).
    bf16 needs F and K to be multiples of 8.  Returns h [M, F], and with want_preact also z [M, 2F], what op_gated_linear_bwd
    needs.  Tensors are contiguous and begin on 16 bytes.  Asynchronous: op_device_error() tells whether a device-side wait gave
    up, in which case the outputs are invalid."""
    if x.dim() != 2 or w.dim() != 2 or w.shape[0] % 2:
        raise ValueError("x, w: expected matrices, w with an even number of rows")
    if act not in ACTIVATIONS:
        raise ValueError("act: expected 'silu' or 'gelu'")
    (M, K), F, dtype = x.shape, w.shape[0] // 2, x.dtype
    dev, code = _device_of(x, w, bias, out), _code(dtype)
    _dense(x, dtype, (M, K), "x"); _dense(w, dtype, (2 * F, K), "w")
    if bias is not None:
        _dense(bias, torch.float32, (2 * F,), "bias")
    if out is None:
        out = x.new_empty((M, F))
    else:
        _dense(out, dtype, (M, F), "out")
        _apart(out, "out", (), x, w, bias)
    pre = x.new_empty((M, 2 * F)) if want_preact else None
    _launch("free_op_gated_linear", dev, code, ACTIVATIONS[act], M, F, K, x.data_ptr(), w.data_ptr(), _adr(bias), out.data_ptr(), _adr(pre),
            _error_word(dev).data_ptr() if code == FREE_BF16 else None)
    return (out, pre) if want_preact else out


def op_gated_linear_bwd(x, w, preact, dh, act="silu", want_dx=True, want_dw=True, want_dbias=True):
    """Gradients of op_gated_linear from dh [M, F] and the preact it kept.  Returns (dx [M, K], dw [2F, K], both in x's dtype,
    dbias fp32 [2F]), None where not wanted.  Asynchronous as the forward call: op_device_error()."""
    if x.dim() != 2 or w.dim() != 2 or w.shape[0] % 2:
        raise ValueError("x, w: expected matrices, w with an even number of rows")
    if act not in ACTIVATIONS:
        raise ValueError("act: expected 'silu' or 'gelu'")
    (M, K), F, dtype = x.shape, w.shape[0] // 2, x.dtype
    dev, code = _device_of(x, w, preact, dh), _code(dtype)
    _dense(x, dtype, (M, K), "x"); _dense(w, dtype, (2 * F, K), "w")
    _dense(preact, dtype, (M, 2 * F), "preact"); _dense(dh, dtype, (M, F), "dh")
    dx = _like(x, dtype) if want_dx else None
    dw = _like(w, dtype) if want_dw else None
    db = x.new_empty(2 * F, dtype=torch.float32) if want_dbias else None
    need = lib().free_op_gated_linear_bwd_workspace_bytes(code, M, F, K)
    ws = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
    _launch("free_op_gated_linear_bwd", dev, code, ACTIVATIONS[act], M, F, K, x.data_ptr(), w.data_ptr(), preact.data_ptr(), dh.data_ptr(),
            _adr(dx), _adr(dw), _adr(db), _adr(ws), need, _error_word(dev).data_ptr() if code == FREE_BF16 else None)
    return dx, dw, db


def op_attention(qkv, heads):
    """qkv [n_seq, n_tok, 3*D] (split as 3, heads, d_head) -> [n_seq, n_tok, D]."""
    dtype = FREE_FP32 if qkv.dtype == torch.float32 else FREE_BF16
    n_seq, n_tok, D3 = qkv.shape
    D = D3 // 3
    out = torch.empty((n_seq, n_tok, D), dtype=qkv.dtype, device=qkv.device)
    need = lib().free_op_attention_workspace_bytes(dtype, n_seq, n_tok, heads, D // heads)
    ws = torch.zeros(need, dtype=torch.uint8, device=qkv.device)
    _check(lib().free_op_attention(dtype, n_seq, n_tok, heads, D // heads, _ptr(qkv), _ptr(out), _ptr(ws), need, _stream()),
           "free_op_attention")
    err = int(ws[:4].view(torch.int32).item())
    if err:
        raise FreeError(-8, f"free_op_attention (device error word {err:#x})")
    return out


# struct free_cross_attn of the public header
_CROSS = struct.Struct("<3Q9q4Q9if")


def _cross_shape(q, k, v, kv_lens, kv_mask, kv_seq, kv_offsets, max_kv, scale):
    """(device, packed free_cross_attn) of a call, after the checks that both directions share."""
    qshape, qs, kshape, ks, vs = q.shape, q.stride(), k.shape, k.stride(), v.stride()
    if len(qs) != 4 or (qshape[3] > 1 and qs[3] != 1):
        raise ValueError("q: expected [n_seq, n_q, heads, d_head] with dense heads")
    packed = kv_offsets is not None
    nd = 3 if packed else 4
    n_seq, n_q, heads, d = qshape
    if len(ks) != nd or kshape != v.shape or kshape[-1] != d or (d > 1 and (ks[-1] != 1 or vs[-1] != 1)):
        raise ValueError("k, v: expected [n_enc, n_kv, kv_heads, d_head] (with kv_offsets [rows, kv_heads, d_head]) with dense heads of q's size")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("k, v: expected q's dtype")
    kv_heads = kshape[-2]
    dev = _device_of(q, k, v, kv_lens, kv_mask, kv_seq, kv_offsets)
    if packed:
        if kv_lens is not None:
            raise ValueError("kv_lens: not with kv_offsets")
        _ints(kv_offsets, None, "kv_offsets")
        n_enc, rows = kv_offsets.shape[0] - 1, kshape[0]
        if n_enc < 0:
            raise ValueError("kv_offsets: expected n_enc + 1 numbers")
        n_kv = rows if max_kv is None else min(int(max_kv), rows)
        if n_kv < 0:
            raise ValueError("max_kv: expected a length")
        ks, vs = (0, *ks), (0, *vs)
    else:
        if max_kv is not None:
            raise ValueError("max_kv: only with kv_offsets")
        n_enc, n_kv = kshape[:2]
        rows = n_kv
        if kv_lens is not None:
            _ints(kv_lens, n_enc, "kv_lens")
    if kv_mask is not None and (kv_mask.dtype not in (torch.bool, torch.uint8) or kv_mask.shape != kshape[:nd - 2] or not kv_mask.is_contiguous()):
        raise ValueError("kv_mask: expected contiguous bool of the states' shape")
    if kv_seq is not None:
        _ints(kv_seq, n_seq, "kv_seq")
    elif n_seq % n_enc if n_enc else n_seq:
        raise ValueError(f"{n_seq} sequences do not share {n_enc} encoder sequences evenly: give kv_seq")
    try:
        return dev, _CROSS.pack(q.data_ptr(), k.data_ptr(), v.data_ptr(), qs[0], qs[1], qs[2], ks[0], ks[1], ks[2], vs[0], vs[1], vs[2],
                                _adr(kv_lens) or 0, _adr(kv_offsets) or 0, _adr(kv_seq) or 0, _adr(kv_mask) or 0, _code(q.dtype), n_seq, n_q, heads,
                                kv_heads, d, n_enc, n_kv, rows, d ** -0.5 if scale is None else scale)
    except (struct.error, OverflowError) as e:
        raise ValueError(f"sizes that do not fit a C int, or a scale that is no float: {e}") from None


def _ints(t, n, what):
    if t.dtype != torch.int32 or t.dim() != 1 or (n is not None and t.shape[0] != n) or not t.is_contiguous():
        raise ValueError(f"{what}: expected contiguous int32 [{'n_enc + 1' if n is None else n}]")


def op_cross_attention(q, k, v, kv_lens=None, kv_mask=None, kv_seq=None, kv_offsets=None, max_kv=None, scale=None, want_lse=False, out=None):
    """Attention of tokens q (CUDA fp32 or bf16 [n_seq, n_q, heads, d_head], any strides with dense heads, d_head up to 128) to an
    encoder's states k, v [n_enc, n_kv, kv_heads, d_head] (heads a multiple of kv_heads; views into a packed projection are fine).
    Encoder sequence e has kv_lens[e] states (int32, default n_kv); with kv_offsets (int32 [n_enc + 1]) the states are packed, k and v
    [rows, kv_heads, d_head], and sequence e has the rows kv_offsets[e] .. kv_offsets[e + 1] - 1, at most max_kv (default: all); offsets must
    not decrease, or dk and dv of the backward pass are undefined.  Give max_kv where it is known: few tokens' states are split by how long one
    sequence's may be (4 single tokens, 77 states each: 3.6 us of GPU time, 6 without it).  States whose kv_mask is False do not count either.  Sequence s reads encoder sequence kv_seq[s] (int32); by default n_seq / n_enc consecutive
    sequences share one.  scale defaults to d_head ** -0.5.  Returns out like q, zero for tokens without a state, and with want_lse also
    the log of the sums of exponentials, fp32 [n_seq, heads, n_q] (-inf for those), what op_cross_attention_bwd needs.  Asynchronous:
    op_device_error() tells whether a device-side wait gave up."""
    dev, shape = _cross_shape(q, k, v, kv_lens, kv_mask, kv_seq, kv_offsets, max_kv, scale)
    if out is None:
        out = _like(q, q.dtype)
    else:
        if out.shape != q.shape or out.dtype != q.dtype or (q.shape[3] > 1 and out.stride(3) != 1):
            raise ValueError("out: expected q's shape and dtype with dense heads")
        _device_of(q, out)
        _apart(out, "out", (), q, k, v)
    n_seq, n_q, heads, _ = q.shape
    lse = q.new_empty((n_seq, heads, n_q), dtype=torch.float32) if want_lse else None
    need = (_LIB or lib()).free_op_cross_attention_workspace_bytes(shape)
    ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    ys = out.stride()
    _launch("free_op_cross_attention", dev, shape, out.data_ptr(), ys[0], ys[1], ys[2], _adr(lse), _adr(ws), need,
            _error_word(dev).data_ptr() if q.dtype == torch.bfloat16 else None)
    return (out, lse) if want_lse else out


def op_cross_attention_bwd(q, k, v, out, lse, dout, kv_lens=None, kv_mask=None, kv_seq=None, kv_offsets=None, max_kv=None, scale=None,
                           want_dq=True, want_dkv=True):
    """Gradients of op_cross_attention from dout (like q) and the out and lse of the forward call; the other arguments as there.
    Returns (dq, dk, dv), contiguous and in q's dtype, None where not wanted; a state's gradients are summed over the tokens, heads and
    sequences that read it, zero where none does.  Asynchronous as the forward call: op_device_error()."""
    dev, shape = _cross_shape(q, k, v, kv_lens, kv_mask, kv_seq, kv_offsets, max_kv, scale)
    _device_of(q, out, lse, dout)
    for t, what in ((out, "out"), (dout, "dout")):
        if t.shape != q.shape or t.dtype != q.dtype or (q.shape[3] > 1 and t.stride(3) != 1):
            raise ValueError(f"{what}: expected q's shape and dtype with dense heads")
    if lse.dtype != torch.float32 or lse.shape != (q.shape[0], q.shape[2], q.shape[1]) or not lse.is_contiguous():
        raise ValueError("lse: expected the contiguous fp32 [n_seq, heads, n_q] of the forward call")
    dq = _like(q, q.dtype) if want_dq else None
    dk = dv = None
    if want_dkv:
        # packed rows that no sequence has are zeros: both cleared in one launch
        dk, dv = (_like(k, k.dtype), _like(v, k.dtype)) if kv_offsets is None else k.new_zeros((2, *k.shape)).unbind(0)
    need = lib().free_op_cross_attention_bwd_workspace_bytes(shape)
    ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    strides = lambda t: (0, 0, 0) if t is None else t.stride()[:3] if t.dim() == 4 else (0, *t.stride()[:2])
    _launch("free_op_cross_attention_bwd", dev, shape, out.data_ptr(), *strides(out), lse.data_ptr(), dout.data_ptr(), *strides(dout),
            _adr(dq), *strides(dq), _adr(dk), *strides(dk), _adr(dv), *strides(dv), _adr(ws), need,
            _error_word(dev).data_ptr() if q.dtype == torch.bfloat16 else None)
    return dq, dk, dv


STATIC_ATTN_MAX_ELEMS = 1 << 21


def op_attention_static(qkv, heads):
    """bf16 attention through the entry point that allocates nothing inside the library: its scratch is a fixed
    array in the library's device image (for callers that may not allocate).  qkv [n_seq, n_tok, 3*D] bf16.
    The output tensor and the 4-byte error word are the caller's (allocated here by torch, outside the call)."""
    n_seq, n_tok, D3 = qkv.shape
    D = D3 // 3
    _dev(qkv, torch.bfloat16)
    out = torch.empty((n_seq, n_tok, D), dtype=torch.bfloat16, device=qkv.device)
    err = torch.ones(1, dtype=torch.int32, device=qkv.device)
    _check(lib().free_op_attention_static(n_seq, n_tok, heads, D // heads, _ptr(qkv), _ptr(out), _ptr(err), _stream()),
           "free_op_attention_static")
    if int(err.item()):
        raise FreeError(-8, "free_op_attention_static (device error word set)")
    return out
