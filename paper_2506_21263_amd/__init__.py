"""Python binding of libdlcx_hip.so (see include/dlcx.h for the contract).

Argument marshalling only: every function below has the name of the C entry point it calls,
takes torch tensors that live on the GPU (PyTorch is used for device memory and streams and for
nothing else) and passes their addresses through.  There is no fallback: if the HIP library is
missing or a call fails, an exception is raised.
"""
import ctypes as C
import functools
import math
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdlcx_hip.so")

OK, EINVAL, EUNSUPPORTED, ELAUNCH, ETOOBIG = 0, -1, -2, -3, -4
PHASE_P, PHASE_Q = 0, 1
F32, BF16 = 0, 1
MMA_FMA, MMA_F32, MMA_BF16, MMA_F16 = 0, 1, 2, 3
MAX_RANK, MAX_WORKERS = 256, 16
MAX_ADAPTERS, MAX_TENSORS = 1024, 1 << 20
STATE_GROUP = 128  # elements of an 8-bit moment that share a scale


class DlcxError(RuntimeError):
    def __init__(self, code, what):
        self.code = code
        detail = lib().dlcx_last_hip_error().decode() if code == ELAUNCH else ""
        super().__init__("%s: %s (%d) %s" % (what, lib().dlcx_strerror(code).decode(), code, detail))


class Desc(C.Structure):
    _fields_ = [("m", C.c_int64), ("n", C.c_int64), ("r", C.c_int32), ("qbits", C.c_int32),
                ("group", C.c_int32), ("mma", C.c_int32)]


def desc(m, n, r, qbits, group, mma=MMA_FMA):
    return Desc(m, n, r, qbits, group, mma)


class AdapterDesc(C.Structure):
    _fields_ = [("m", C.c_int64), ("n", C.c_int64), ("r", C.c_int32), ("count", C.c_int32),
                ("dtype", C.c_int32)]


def adapter_desc(m, n, r, count, dtype=BF16):
    return AdapterDesc(m, n, r, count, dtype)


class Tensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("m_scale", C.c_void_p), ("v_scale", C.c_void_p), ("copy", C.c_void_p),
                ("numel", C.c_int64), ("lr_scale", C.c_float), ("weight_decay", C.c_float),
                ("param_dtype", C.c_int32), ("grad_dtype", C.c_int32), ("state_bits", C.c_int32),
                ("reserved", C.c_int32)]


class Table(C.Structure):
    """The caller's handle of a table of tensors; `held` keeps what it points to alive."""
    _fields_ = [("memory", C.c_void_p), ("blocks", C.c_int64), ("count", C.c_int32),
                ("steps", C.c_int32)]


class Fp8(C.Structure):
    """A matrix in 8 bits; `held` keeps the tensors behind it."""
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64),
                ("ld", C.c_int64), ("ldscale", C.c_int64)]


_lib = None
_vp, _i64, _i32, _int = C.c_void_p, C.c_int64, C.c_int32, C.c_int
_dp = C.POINTER(Desc)

SYMBOLS = {
    "dlcx_delta_ef": (_int, [_vp, _vp, _int, _vp, _i64, _vp]),
    "dlcx_compress": (_int, [_dp, _int, _vp, _vp, _vp, _vp, _vp, _vp]),
    "dlcx_compress_batched": (_int, [_dp, _int, _int, _vp, _vp, _vp, _vp, _vp, _vp]),
    "dlcx_compress_average": (_int, [_dp, _int, _int, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "dlcx_average": (_int, [_dp, _int, _int, _vp, _vp, _vp, _vp, _vp]),
    "dlcx_average_static": (_int, [_dp, _int, _int, _vp, _vp, _vp, _vp]),
    "dlcx_static_scratch_bytes": (C.c_size_t, []),
    "dlcx_static_scratch_need": (C.c_size_t, [_dp, _int]),
    "dlcx_decompress": (_int, [_dp, _vp, _vp, _vp, _int, _vp, _vp, _vp]),
    "dlcx_decompress_apply": (_int, [_dp, _vp, _vp, _int, _vp, _vp, _vp, C.c_float, C.c_float, _vp,
                                     _vp]),
    "dlcx_ef_delta_apply": (_int, [_dp, _vp, _vp, _int, _vp, _int, _vp, _vp, _vp, C.c_float,
                                   C.c_float, _vp, _vp]),
    "dlcx_ef_delta_apply_compress": (_int, [_dp, _i32, _vp, _vp, _int, _vp, _int, _vp, _vp, _vp,
                                            C.c_float, C.c_float, _vp, _vp, _vp, _vp, _vp]),
    "dlcx_ef_delta_apply_compress_average": (_int, [_dp, _i32, _vp, _vp, _int, _vp, _int, _vp, _vp,
                                                    _vp, C.c_float, C.c_float, _vp, _vp, _vp, _vp,
                                                    _vp, _vp]),
    "dlcx_outer_nesterov": (_int, [_vp, _vp, _vp, _i64, C.c_float, C.c_float, _vp]),
    "dlcx_quant_round": (_int, [_i64, _int, _int, _int, _vp, _int, _vp, _vp, _vp, C.c_double,
                                C.c_double, _vp, _vp, _int, _vp, _vp, _vp]),
    "dlcx_ef_update": (_int, [_int, _vp, _vp, _i64, _vp]),
    "dlcx_requantize": (_int, [_vp, _i64, _int, _int, _vp]),
    "dlcx_mfma_peak_probe": (_int, [_int, _int, _int, _vp, _vp]),
    "dlcx_traffic_probe": (_int, [_int, _vp, _int, _vp, _vp, _vp, _i64, _vp]),
    "dlcx_comm_seconds": (C.c_double, [C.c_double, _int, C.c_double]),
    "dlcx_plan_overlap": (_int, [_dp, _int, C.c_double, _int, _i32, _i32, _int, C.c_double,
                                 C.c_double, _i32, _vp, _vp, _vp]),
    "dlcx_select_rank": (_int, [_dp, _vp, _int, C.c_double, _vp, _i32, _i32, _i32, _i32, _i32,
                                _i32, _vp, _vp, _vp, _vp, _vp]),
    "dlcx_select_rank_from": (_int, [_vp, _int, _vp, _i32, _i32, _i32, _i32, _i32, _i32, _vp, _vp, _vp,
                                     _vp]),
    "dlcx_batched_workspace_bytes": (C.c_size_t, [_dp, _int]),
    "dlcx_orthonormalize_batched": (_int, [_dp, _vp, _int, _vp, _vp]),
    "dlcx_effective_rank_batched": (_int, [_dp, _vp, _int, C.c_double, _vp, _vp, _vp]),
    "dlcx_payload_bytes": (C.c_size_t, [_dp, _int, _vp, _vp]),
    "dlcx_workspace_bytes": (C.c_size_t, [_dp, _int]),
    "dlcx_select_rank_workspace_bytes": (C.c_size_t, [_dp, _int]),
    "dlcx_project": (_int, [_dp, _int, _int, _vp, _vp, _vp, _vp, _vp]),
    "dlcx_quantize": (_int, [_vp, _i64, _int, _int, _vp, _vp, _vp]),
    "dlcx_dequant_average": (_int, [_int, _vp, _vp, _i64, _int, _int, _vp, _vp]),
    "dlcx_orthonormalize": (_int, [_i64, _i32, _vp, _vp, _vp]),
    "dlcx_effective_rank": (_int, [_i64, _i32, _vp, C.c_double, _vp, _vp, _vp]),
    "dlcx_adapter_route_bytes": (C.c_size_t, [_i64, _i32]),
    "dlcx_adapter_route": (_int, [_i64, _vp, _i32, _vp, _vp]),
    "dlcx_adapter_workspace_bytes": (C.c_size_t, [_vp, _i64]),
    "dlcx_adapter_forward": (_int, [_vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64,
                                    _vp, _i64, _vp, _vp, _vp]),
    "dlcx_adapter_backward": (_int, [_vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp,
                                     _vp, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp]),
    "dlcx_tensor_table_bytes": (C.c_size_t, [_i32]),
    "dlcx_tensor_table": (_int, [_vp, _i32, _vp, _vp, _vp]),
    "dlcx_grad_norm": (_int, [_vp, C.c_double, _vp, _vp]),
    "dlcx_adamw": (_int, [_vp, C.c_double, C.c_double, C.c_double, C.c_double, _i64, C.c_double,
                          _vp, C.c_double, _vp]),
    "dlcx_state_decode": (_int, [_int, _vp, _vp, _i64, _vp, _int, _vp]),
    "dlcx_fp8_code_pitch": (_i64, [_i64]),
    "dlcx_fp8_scale_pitch": (_i64, [_i64]),
    "dlcx_fp8_quantize": (_int, [_i64, _i64, _vp, _i64, _int, _int, _vp, _vp, _vp]),
    "dlcx_fp8_decode": (_int, [_vp, _vp, _i64, _int, _vp]),
    "dlcx_fp8_product_workspace_bytes": (C.c_size_t, [_i64, _i64, _i64]),
    "dlcx_fp8_product_plan": (_int, [_i64, _i64, _i64, _int, _vp, _vp, _vp]),
    "dlcx_fp8_product": (_int, [_vp, _vp, _vp, _i64, _vp, _i64, _int, _vp, _vp]),
    "dlcx_rms_norm": (_int, [_i64, _i64, _int, _vp, _i64, _vp, _i64, _vp, C.c_float, _vp, _i64, _vp, _i64,
                             _vp, _vp, _vp]),
    "dlcx_rms_norm_workspace_bytes": (C.c_size_t, [_i64, _i64]),
    "dlcx_rms_norm_backward": (_int, [_i64, _i64, _int, _vp, _i64, _vp, _vp, _vp, _i64, _vp, _i64, _vp, _i64,
                                      _vp, _vp, _vp]),
    "dlcx_dropout": (_int, [_i64, _i64, _int, _vp, _i64, _vp, _i64, _vp, _i64, C.c_double, C.c_uint64,
                            C.c_uint64, _vp, _vp]),
    "dlcx_profile_enable": (_int, [_int]),
    "dlcx_profile_kernels": (_int, []),
    "dlcx_profile_name": (C.c_char_p, [_int]),
    "dlcx_profile_read": (_int, [_int, _vp, _vp]),
    "dlcx_strerror": (C.c_char_p, [_int]),
    "dlcx_last_hip_error": (C.c_char_p, []),
}


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("%s is missing: build it with `python paper_2506_21263_amd/build.py` "
                              "(there is no CPU fallback)" % LIB_PATH)
        L = C.CDLL(LIB_PATH)
        for name, (res, args) in SYMBOLS.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    assert t.is_cuda and t.is_contiguous(), "device-resident contiguous tensors only"
    return t.data_ptr()


def _ptr_array(ts):
    if ts is None:
        return None
    arr = (C.c_void_p * len(ts))(*[_ptr(t) for t in ts])
    return C.cast(arr, C.c_void_p), arr  # keep `arr` alive with the caller


# The handle of the current stream without the object around it (3 us of a call of 10), where torch has that; it is
# no documented name of torch, so no call depends on it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is None:
            return torch.cuda.current_stream().cuda_stream
        return _raw_stream(torch.cuda.current_device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(code, what):
    if code != OK:
        raise DlcxError(code, what)


def dlcx_payload_bytes(d, phase):
    cb, sb = C.c_size_t(0), C.c_size_t(0)
    total = lib().dlcx_payload_bytes(C.byref(d), phase, C.addressof(cb), C.addressof(sb))
    return total, cb.value, sb.value


def dlcx_workspace_bytes(d, K):
    return lib().dlcx_workspace_bytes(C.byref(d), K)


def dlcx_delta_ef(theta_g, theta_l, ef_inout, numel=None, stream=None):
    dt = BF16 if theta_l.dtype == torch.bfloat16 else F32
    n = theta_g.numel() if numel is None else numel
    _check(lib().dlcx_delta_ef(_ptr(theta_g), _ptr(theta_l), dt, _ptr(ef_inout), n,
                               _stream(stream)), "dlcx_delta_ef")


def dlcx_compress(d, phase, delta, basis, codes_out, scales_out, workspace, stream=None):
    _check(lib().dlcx_compress(C.byref(d), phase, _ptr(delta), _ptr(basis), _ptr(codes_out),
                               _ptr(scales_out), _ptr(workspace), _stream(stream)),
           "dlcx_compress")


def dlcx_compress_batched(d, phase, deltas, basis, codes_out, scales_out, workspace, stream=None):
    dp, k1 = _ptr_array(deltas)
    cp, k2 = _ptr_array(codes_out)
    sp, k3 = _ptr_array(scales_out)
    _check(lib().dlcx_compress_batched(C.byref(d), phase, len(deltas), dp, _ptr(basis), cp, sp,
                                       _ptr(workspace), _stream(stream)), "dlcx_compress_batched")


def dlcx_compress_average(d, phase, deltas, basis, codes_out, scales_out, mean_out, workspace,
                          stream=None):
    dp, k1 = _ptr_array(deltas)
    cp, k2 = _ptr_array(codes_out)
    sp, k3 = _ptr_array(scales_out)
    _check(lib().dlcx_compress_average(C.byref(d), phase, len(deltas), dp, _ptr(basis), cp, sp,
                                       _ptr(mean_out), _ptr(workspace), _stream(stream)),
           "dlcx_compress_average")


def dlcx_average(d, phase, codes, scales, factor_out, workspace, stream=None):
    cp, k1 = _ptr_array(codes)
    sp, k2 = _ptr_array(scales)
    _check(lib().dlcx_average(C.byref(d), phase, len(codes), cp, sp, _ptr(factor_out),
                              _ptr(workspace), _stream(stream)), "dlcx_average")


def dlcx_average_static(d, phase, codes, scales, factor_out, stream=None):
    cp, k1 = _ptr_array(codes)
    sp, k2 = _ptr_array(scales)
    _check(lib().dlcx_average_static(C.byref(d), phase, len(codes), cp, sp, _ptr(factor_out),
                                     _stream(stream)), "dlcx_average_static")


def dlcx_static_scratch_bytes():
    return lib().dlcx_static_scratch_bytes()


def dlcx_static_scratch_need(d, phase):
    return lib().dlcx_static_scratch_need(C.byref(d), phase)


def dlcx_decompress(d, p_hat, q_bar, delta_hat_out, ef_inout=(), workspace=None, stream=None):
    ep, keep = _ptr_array(list(ef_inout)) if len(ef_inout) else (None, None)
    _check(lib().dlcx_decompress(C.byref(d), _ptr(p_hat), _ptr(q_bar), _ptr(delta_hat_out),
                                 len(ef_inout), ep, _ptr(workspace), _stream(stream)),
           "dlcx_decompress")


def dlcx_decompress_apply(d, p_hat, q_bar, ef_inout, theta_g, v, lr, mu, workspace=None,
                          stream=None):
    ep, keep = _ptr_array(list(ef_inout)) if len(ef_inout) else (None, None)
    _check(lib().dlcx_decompress_apply(C.byref(d), _ptr(p_hat), _ptr(q_bar), len(ef_inout), ep,
                                       _ptr(theta_g), _ptr(v), lr, mu, _ptr(workspace),
                                       _stream(stream)), "dlcx_decompress_apply")


def dlcx_ef_delta_apply(d, p_hat, q_bar, theta_l, ef_inout, theta_g, v, lr, mu, workspace=None,
                        stream=None):
    dt = BF16 if theta_l[0].dtype == torch.bfloat16 else F32
    tp, k1 = _ptr_array(list(theta_l))
    ep, k2 = _ptr_array(list(ef_inout))
    _check(lib().dlcx_ef_delta_apply(C.byref(d), _ptr(p_hat), _ptr(q_bar), len(ef_inout), tp, dt,
                                     ep, _ptr(theta_g), _ptr(v), lr, mu, _ptr(workspace),
                                     _stream(stream)), "dlcx_ef_delta_apply")


def dlcx_ef_delta_apply_compress(d, r_prev, p_hat, q_bar, theta_l, ef_inout, theta_g, v, lr, mu,
                                 basis, codes_out, scales_out, workspace, stream=None):
    dt = BF16 if theta_l[0].dtype == torch.bfloat16 else F32
    tp, k1 = _ptr_array(list(theta_l))
    ep, k2 = _ptr_array(list(ef_inout))
    cp, k3 = _ptr_array(list(codes_out))
    sp, k4 = _ptr_array(list(scales_out))
    _check(lib().dlcx_ef_delta_apply_compress(
        C.byref(d), r_prev, _ptr(p_hat), _ptr(q_bar), len(ef_inout), tp, dt, ep, _ptr(theta_g),
        _ptr(v), lr, mu, _ptr(basis), cp, sp, _ptr(workspace), _stream(stream)),
        "dlcx_ef_delta_apply_compress")


def dlcx_ef_delta_apply_compress_average(d, r_prev, p_hat, q_bar, theta_l, ef_inout, theta_g, v, lr,
                                         mu, basis, codes_out, scales_out, mean_out, workspace,
                                         stream=None):
    dt = BF16 if theta_l[0].dtype == torch.bfloat16 else F32
    tp, k1 = _ptr_array(list(theta_l))
    ep, k2 = _ptr_array(list(ef_inout))
    cp, k3 = _ptr_array(list(codes_out))
    sp, k4 = _ptr_array(list(scales_out))
    _check(lib().dlcx_ef_delta_apply_compress_average(
        C.byref(d), r_prev, _ptr(p_hat), _ptr(q_bar), len(ef_inout), tp, dt, ep, _ptr(theta_g),
        _ptr(v), lr, mu, _ptr(basis), cp, sp, _ptr(mean_out), _ptr(workspace), _stream(stream)),
        "dlcx_ef_delta_apply_compress_average")


def dlcx_outer_nesterov(theta_g, v, delta_hat, lr, mu, numel=None, stream=None):
    n = theta_g.numel() if numel is None else numel
    _check(lib().dlcx_outer_nesterov(_ptr(theta_g), _ptr(v), _ptr(delta_hat), n, lr, mu,
                                     _stream(stream)), "dlcx_outer_nesterov")


def dlcx_quant_round(numel, qbits, group, theta_l, ef_inout, theta_g, v, lr, mu, prev_codes,
                     prev_scales, codes_out, scales_out, requant=False, stream=None):
    """prev_codes / prev_scales None: outer step 1."""
    dt = BF16 if theta_l[0].dtype == torch.bfloat16 else F32
    tp, k1 = _ptr_array(list(theta_l))
    ep, k2 = _ptr_array(list(ef_inout))
    pc, k3 = _ptr_array(list(prev_codes)) if prev_codes is not None else (None, None)
    ps, k4 = _ptr_array(list(prev_scales)) if prev_scales is not None else (None, None)
    cp, k5 = _ptr_array(list(codes_out))
    sp, k6 = _ptr_array(list(scales_out))
    _check(lib().dlcx_quant_round(numel, qbits, group, len(ef_inout), tp, dt, ep, _ptr(theta_g),
                                  _ptr(v), lr, mu, pc, ps, 1 if requant else 0, cp, sp,
                                  _stream(stream)), "dlcx_quant_round")


def dlcx_ef_update(ef_inout, delta_hat, numel=None, stream=None):
    n = delta_hat.numel() if numel is None else numel
    ep, keep = _ptr_array(list(ef_inout))
    _check(lib().dlcx_ef_update(len(ef_inout), ep, _ptr(delta_hat), n, _stream(stream)),
           "dlcx_ef_update")


def dlcx_mfma_peak_probe(workgroups, iters, out, random_operands=False, stream=None):
    _check(lib().dlcx_mfma_peak_probe(workgroups, iters, 1 if random_operands else 0, _ptr(out),
                                      _stream(stream)), "dlcx_mfma_peak_probe")


def dlcx_traffic_probe(theta_l, ef_inout, theta_g, v, numel=None, stream=None):
    dt = BF16 if theta_l[0].dtype == torch.bfloat16 else F32
    n = theta_g.numel() if numel is None else numel
    tp, k1 = _ptr_array(list(theta_l))
    ep, k2 = _ptr_array(list(ef_inout))
    _check(lib().dlcx_traffic_probe(len(ef_inout), tp, dt, ep, _ptr(theta_g), _ptr(v), n,
                                    _stream(stream)), "dlcx_traffic_probe")


def dlcx_requantize(x_inout, count, qbits, group, stream=None):
    _check(lib().dlcx_requantize(_ptr(x_inout), count, qbits, group, _stream(stream)),
           "dlcx_requantize")


def dlcx_comm_seconds(payload_bytes, clusters, bits_per_second):
    return lib().dlcx_comm_seconds(payload_bytes, clusters, bits_per_second)


def dlcx_plan_overlap(descs, extra_bytes, rmin, rmax, clusters, bits_per_second, step_seconds, H,
                      power_iters=1):
    """Returns (rank, H, seconds of the exchange at that rank).  Host only."""
    n = len(descs)
    arr = (Desc * max(n, 1))(*descs)
    r, h, t = _i32(0), _i32(0), C.c_double(0.0)
    _check(lib().dlcx_plan_overlap(arr, n, extra_bytes, power_iters, rmin, rmax, clusters,
                                   bits_per_second, step_seconds, H, C.addressof(r),
                                   C.addressof(h), C.addressof(t)), "dlcx_plan_overlap")
    return r.value, h.value, t.value


def dlcx_select_rank_workspace_bytes(descs):
    arr = (Desc * max(len(descs), 1))(*descs)
    return lib().dlcx_select_rank_workspace_bytes(arr, len(descs))


def dlcx_select_rank(descs, q_bars, tau, rprime_hist, t, c, r1, rmin, rmax, H1, workspace=None,
                     rprime=None, stream=None):
    """rprime_hist: ctypes int32 array of length c (the caller's ring).  Returns (r', r_t, H_t)."""
    n = len(descs)
    arr = (Desc * max(n, 1))(*descs)
    qp, keep = _ptr_array(list(q_bars)) if n else (None, None)
    rp = C.c_int32(0 if rprime is None else rprime)
    r_next, h_next = C.c_int32(0), C.c_int32(0)
    _check(lib().dlcx_select_rank(arr, qp, n, tau, C.addressof(rprime_hist), t, c, r1, rmin, rmax,
                                  H1, C.addressof(rp), C.addressof(r_next), C.addressof(h_next),
                                  _ptr(workspace), _stream(stream) if n else None),
           "dlcx_select_rank")
    return rp.value, r_next.value, h_next.value


def dlcx_select_rank_from(rprime_dev, n, rprime_hist, t, c, r1, rmin, rmax, H1, rprime=None,
                          stream=None):
    """Window rule on r' values already measured into the device int32 tensor rprime_dev."""
    rp = C.c_int32(0 if rprime is None else rprime)
    r_next, h_next = C.c_int32(0), C.c_int32(0)
    _check(lib().dlcx_select_rank_from(_ptr(rprime_dev) if n else None, n,
                                       C.addressof(rprime_hist), t, c, r1, rmin, rmax, H1,
                                       C.addressof(rp), C.addressof(r_next), C.addressof(h_next),
                                       _stream(stream) if n else None), "dlcx_select_rank_from")
    return rp.value, r_next.value, h_next.value


def dlcx_batched_workspace_bytes(descs):
    arr = (Desc * max(len(descs), 1))(*descs)
    return lib().dlcx_batched_workspace_bytes(arr, len(descs))


def dlcx_orthonormalize_batched(descs, p_inout, workspace, stream=None):
    arr = (Desc * max(len(descs), 1))(*descs)
    pp, keep = _ptr_array(list(p_inout))
    _check(lib().dlcx_orthonormalize_batched(arr, pp, len(descs), _ptr(workspace), _stream(stream)),
           "dlcx_orthonormalize_batched")


def dlcx_effective_rank_batched(descs, q_bars, tau, rprime_out_dev, workspace, stream=None):
    arr = (Desc * max(len(descs), 1))(*descs)
    qp, keep = _ptr_array(list(q_bars))
    _check(lib().dlcx_effective_rank_batched(arr, qp, len(descs), tau, _ptr(rprime_out_dev),
                                             _ptr(workspace), _stream(stream)),
           "dlcx_effective_rank_batched")


def dlcx_project(d, phase, deltas, basis, factors_out, workspace, stream=None):
    dp, k1 = _ptr_array(deltas)
    fp, k2 = _ptr_array(factors_out)
    _check(lib().dlcx_project(C.byref(d), phase, len(deltas), dp, _ptr(basis), fp, _ptr(workspace),
                              _stream(stream)), "dlcx_project")


def dlcx_quantize(x, qbits, group, codes_out, scales_out, count=None, stream=None):
    n = x.numel() if count is None else count
    _check(lib().dlcx_quantize(_ptr(x), n, qbits, group, _ptr(codes_out), _ptr(scales_out),
                               _stream(stream)), "dlcx_quantize")


def dlcx_dequant_average(codes, scales, count, qbits, group, mean_out, stream=None):
    cp, k1 = _ptr_array(codes)
    sp, k2 = _ptr_array(scales)
    _check(lib().dlcx_dequant_average(len(codes), cp, sp, count, qbits, group, _ptr(mean_out),
                                      _stream(stream)), "dlcx_dequant_average")


def dlcx_orthonormalize(L, r, p_inout, workspace, stream=None):
    _check(lib().dlcx_orthonormalize(L, r, _ptr(p_inout), _ptr(workspace), _stream(stream)),
           "dlcx_orthonormalize")


def dlcx_effective_rank(L, r, q_bar, tau, rprime_out_dev, workspace, stream=None):
    _check(lib().dlcx_effective_rank(L, r, _ptr(q_bar), tau, _ptr(rprime_out_dev),
                                     _ptr(workspace), _stream(stream)), "dlcx_effective_rank")


_CODE = {torch.float32: F32, torch.bfloat16: BF16}


def _typed(t, dtype, numel, what):
    """Address of a contiguous device tensor of that type with at least `numel` elements, or None."""
    if t is None:
        return None
    if not (t.is_cuda and t.dtype is dtype and t.numel() >= numel and t.is_contiguous()):
        raise ValueError("%s: a contiguous device tensor of %d elements of %s is wanted" % (what, numel, dtype))
    return t.data_ptr()


def _packed(t, dtype, shape, what):
    """Address of a packed device array of that shape: one with its last dimensions, or a flat one.  (Arrays of equal
    shapes, as P and Q of a square projection, cannot be told apart.)"""
    if t is not None and t.shape == shape and t.is_cuda and t.dtype == dtype and t.is_contiguous():
        return t.data_ptr()
    if t is not None and t.dim() > 1 and t.shape[-2:] != shape[-2:] and not (t.dim() == 2 and t.shape[1] == shape[-1]):
        raise ValueError("%s: an array of %s is wanted, not of %s" % (what, " x ".join(map(str, shape)), " x ".join(
            map(str, t.shape))))
    return _typed(t, dtype, math.prod(shape), what)


def _rows(t, rows, cols, dtype, what):
    """Address and row stride of a rows x cols device matrix whose rows are contiguous."""
    if t is None:
        return None, cols
    if t.is_cuda and t.dtype is dtype and t.shape == (rows, cols):  # the usual case, with few questions
        step, inner = t.stride()
        if inner == 1 and step >= cols:
            return t.data_ptr(), (step if rows > 1 else cols)
    if not (t.is_cuda and t.dtype == dtype and t.dim() == 2 and t.shape[0] == rows and t.shape[1] == cols):
        raise ValueError("%s: a %d x %d device matrix of %s is wanted" % (what, rows, cols, dtype))
    step, inner = t.stride()
    if (inner != 1 and cols > 1) or (step < cols and rows > 1):
        raise ValueError("%s: the elements of a row have to be consecutive, and rows apart" % what)
    return t.data_ptr(), (step if rows > 1 else cols)


def dlcx_adapter_route_bytes(rows, count):
    return lib().dlcx_adapter_route_bytes(rows, count)


def dlcx_adapter_route(ids, count, route, stream=None):
    """ids: int32 device tensor, one adapter (or a value outside [0, count)) per row."""
    rows = ids.numel()
    _typed(route, torch.uint8, dlcx_adapter_route_bytes(rows, count), "route")
    _check(lib().dlcx_adapter_route(rows, _typed(ids, torch.int32, rows, "ids"), count, _ptr(route),
                                    _stream(stream)), "dlcx_adapter_route")


def dlcx_adapter_workspace_bytes(d, rows):
    return lib().dlcx_adapter_workspace_bytes(C.byref(d), rows)


def _adapter_common(d, rows, ids, q, p, scale, ranks, route, workspace):
    dt = torch.bfloat16 if d.dtype == BF16 else torch.float32
    return (dt, _typed(ids, torch.int32, rows, "ids"), _packed(q, dt, (d.count, d.r, d.n), "q"),
            _packed(p, dt, (d.count, d.r, d.m), "p"), _typed(scale, torch.float32, d.count, "scale"),
            _typed(ranks, torch.int32, d.count, "ranks"),
            None if route is None else _typed(route, torch.uint8, dlcx_adapter_route_bytes(rows, d.count), "route"),
            _typed(workspace, torch.uint8, dlcx_adapter_workspace_bytes(d, rows), "workspace"))


def dlcx_adapter_forward(d, x, ids, q, p, y_in, y_out, h_out, workspace, scale=None, ranks=None,
                         route=None, stream=None):
    """x (rows x n), y_in (rows x m, None: zeros) and y_out may be views with a row stride."""
    rows = x.shape[0]
    dt, ids, q, p, scale, ranks, route, ws = _adapter_common(d, rows, ids, q, p, scale, ranks, route, workspace)
    x, ldx = _rows(x, rows, d.n, dt, "x")
    y_in, ldi = _rows(y_in, rows, d.m, dt, "y_in")
    y_out, ldo = _rows(y_out, rows, d.m, dt, "y_out")
    _check(lib().dlcx_adapter_forward(C.byref(d), rows, x, ldx, ids, q, p, scale, ranks, route, y_in, ldi,
                                      y_out, ldo, _packed(h_out, torch.float32, (rows, d.r), "h_out"), ws,
                                      _stream(stream)), "dlcx_adapter_forward")


def dlcx_adapter_backward(d, x, dy, ids, q, p, h, dx_in, dx_out, dq_out, dp_out, workspace,
                          scale=None, ranks=None, route=None, stream=None):
    """x, dy, dx_in (None: zeros) and dx_out may be views with a row stride; h is the forward call's."""
    rows = x.shape[0]
    dt, ids, q, p, scale, ranks, route, ws = _adapter_common(d, rows, ids, q, p, scale, ranks, route, workspace)
    x, ldx = _rows(x, rows, d.n, dt, "x")
    dy, lddy = _rows(dy, rows, d.m, dt, "dy")
    dx_in, ldi = _rows(dx_in, rows, d.n, dt, "dx_in")
    dx_out, ldo = _rows(dx_out, rows, d.n, dt, "dx_out")
    _check(lib().dlcx_adapter_backward(C.byref(d), rows, x, ldx, dy, lddy, ids, q, p, scale, ranks, route,
                                       _packed(h, torch.float32, (rows, d.r), "h"), dx_in, ldi, dx_out, ldo,
                                       _packed(dq_out, torch.float32, (d.count, d.r, d.n), "dq_out"),
                                       _packed(dp_out, torch.float32, (d.count, d.r, d.m), "dp_out"), ws,
                                       _stream(stream)), "dlcx_adapter_backward")


def tensor(grad, param=None, m=None, v=None, m_scale=None, v_scale=None, copy=None, weight_decay=0.0,
           lr_scale=1.0):
    """One tensor of a step (contiguous device tensors of equal lengths).  Moments: float32, or int8
    and uint8 codes with a float32 scale per STATE_GROUP elements.  Returns the structure and what it
    points to."""
    numel = grad.numel()
    if grad.dtype not in _CODE or (param is not None and param.dtype not in _CODE):
        raise ValueError("gradients and parameters are float32 or bfloat16")
    if param is not None and (m is None or v is None):
        raise ValueError("a parameter has both of its moments")
    t = Tensor(grad=_typed(grad, grad.dtype, numel, "grad"), numel=numel, lr_scale=lr_scale,
               weight_decay=weight_decay, grad_dtype=_CODE[grad.dtype], state_bits=32)
    if param is not None:
        eight = m.dtype != torch.float32
        if param.numel() != numel:
            raise ValueError("param and grad have different lengths")
        t.param, t.param_dtype = _typed(param, param.dtype, numel, "param"), _CODE[param.dtype]
        t.m = _typed(m, torch.int8 if eight else torch.float32, numel, "m")
        t.v = _typed(v, torch.uint8 if eight else torch.float32, numel, "v")
        t.copy = _typed(copy, torch.bfloat16, numel, "copy")
        if eight:
            groups = -(-numel // STATE_GROUP)
            t.state_bits = 8
            t.m_scale = _typed(m_scale, torch.float32, groups, "m_scale")
            t.v_scale = _typed(v_scale, torch.float32, groups, "v_scale")
    return t, (grad, param, m, v, m_scale, v_scale, copy)


def dlcx_tensor_table_bytes(count):
    return lib().dlcx_tensor_table_bytes(count)


def dlcx_tensor_table(tensors, memory, stream=None):
    """tensors: what `tensor` returned, one after the other.  The handle keeps them and `memory`."""
    table = Table()
    arr = (Tensor * max(len(tensors), 1))(*[t for t, _ in tensors])
    _typed(memory, torch.uint8, dlcx_tensor_table_bytes(len(tensors)), "memory")
    _check(lib().dlcx_tensor_table(arr, len(tensors), _ptr(memory), C.addressof(table), _stream(stream)),
           "dlcx_tensor_table")
    table.held = (memory, [held for _, held in tensors])
    return table


def dlcx_grad_norm(table, norm_out, grad_scale=1.0, stream=None):
    _check(lib().dlcx_grad_norm(C.addressof(table), grad_scale, _typed(norm_out, torch.float32, 1, "norm_out"),
                                _stream(stream)), "dlcx_grad_norm")


def dlcx_adamw(table, lr, beta1, beta2, eps, step, norm=None, max_norm=0.0, grad_scale=1.0, stream=None):
    _check(lib().dlcx_adamw(C.addressof(table), lr, beta1, beta2, eps, step, grad_scale,
                            _typed(norm, torch.float32, 1, "norm"), max_norm, _stream(stream)), "dlcx_adamw")


def dlcx_state_decode(codes, scales, out, stream=None):
    """int8 codes are a first moment's, uint8 codes a second one's; out: float32 or bfloat16."""
    if codes.dtype not in (torch.int8, torch.uint8) or out.dtype not in _CODE:
        raise ValueError("int8 or uint8 codes, float32 or bfloat16 values")
    n = codes.numel()
    _check(lib().dlcx_state_decode(int(codes.dtype == torch.uint8), _typed(codes, codes.dtype, n, "codes"),
                                   _typed(scales, torch.float32, -(-n // STATE_GROUP), "scales"), n,
                                   _typed(out, out.dtype, n, "out"), _CODE[out.dtype], _stream(stream)),
           "dlcx_state_decode")


def dlcx_fp8_code_pitch(cols):
    return lib().dlcx_fp8_code_pitch(cols)


def dlcx_fp8_scale_pitch(cols):
    return lib().dlcx_fp8_scale_pitch(cols)


def _bytes(t, kind, rows, pitch, what):
    """Address and row stride of `rows` rows of at least `pitch` bytes on the device."""
    if not (t.is_cuda and t.dtype in (kind, torch.uint8) and t.dim() == 2 and t.shape[0] == rows and t.shape[1] >= pitch):
        raise ValueError("%s: a device matrix of %d rows of %d bytes (%s or uint8) is wanted" % (what, rows, pitch, kind))
    step, inner = t.stride()
    if (inner != 1 and t.shape[1] > 1) or (step < t.shape[1] and rows > 1):
        raise ValueError("%s: the bytes of a row have to be consecutive, and rows apart" % what)
    return t.data_ptr(), (step if rows > 1 else pitch)  # (one row: its stride says nothing, and may be no multiple)


def fp8(codes, scales, cols):
    """A matrix in 8 bits of `cols` columns, from its codes (float8_e4m3fn or uint8, dlcx_fp8_code_pitch(cols) of them to a
    row, zeros from `cols` on) and its scales (uint8 or float8_e8m0fnu, dlcx_fp8_scale_pitch(cols) to a row)."""
    rows = codes.shape[0]
    c, ld = _bytes(codes, torch.float8_e4m3fn, rows, dlcx_fp8_code_pitch(cols), "codes")
    s, lds = _bytes(scales, torch.float8_e8m0fnu, rows, dlcx_fp8_scale_pitch(cols), "scales")
    a = Fp8(codes=c, scales=s, rows=rows, cols=cols, ld=ld, ldscale=lds)
    a.held = (codes, scales)
    return a


def fp8_empty(rows, cols, device="cuda"):
    """Memory for a matrix in 8 bits that dlcx_fp8_quantize or dlcx_rms_norm writes."""
    return fp8(torch.empty(rows, dlcx_fp8_code_pitch(cols), device=device, dtype=torch.float8_e4m3fn),
               torch.empty(rows, dlcx_fp8_scale_pitch(cols), device=device, dtype=torch.uint8), cols)


def _ref(a):
    return None if a is None else C.addressof(a)


def _type_of(t, what):
    dt = t.dtype
    if dt is torch.bfloat16 or dt is torch.float32:
        return dt
    raise ValueError("%s: float32 or bfloat16 is wanted" % what)


def dlcx_fp8_quantize(x, out=None, out_t=None, square=False, stream=None):
    """x (a matrix, its rows may be apart) to `out` and its transpose to `out_t` (what `fp8` or `fp8_empty` made, or None)."""
    dt = _type_of(x, "x")
    rows, cols = x.shape
    x, ldx = _rows(x, rows, cols, dt, "x")
    _check(lib().dlcx_fp8_quantize(rows, cols, x, ldx, _CODE[dt], int(square), _ref(out), _ref(out_t), _stream(stream)),
           "dlcx_fp8_quantize")


def dlcx_fp8_decode(a, out, stream=None):
    dt = _type_of(out, "out")
    out, ldo = _rows(out, a.rows, a.cols, dt, "out")
    _check(lib().dlcx_fp8_decode(C.addressof(a), out, ldo, _CODE[dt], _stream(stream)), "dlcx_fp8_decode")


@functools.lru_cache(maxsize=4096)  # (it looks at every smaller number of rows: up to 40 us, and every product asks)
def dlcx_fp8_product_workspace_bytes(rows, m, n):
    return lib().dlcx_fp8_product_workspace_bytes(rows, m, n)


def dlcx_fp8_product_plan(rows, m, n, dtype):
    """(form, tile, splits) of a product of these sizes with results of F32 or BF16."""
    out = [C.c_int32() for _ in range(3)]
    _check(lib().dlcx_fp8_product_plan(rows, m, n, dtype, *(C.addressof(k) for k in out)), "dlcx_fp8_product_plan")
    return tuple(k.value for k in out)


def dlcx_fp8_product(x, w, y_in, y_out, workspace, stream=None):
    """y_out = y_in (None: zeros) + x w^T; y may be views with a row stride."""
    dt = _type_of(y_out, "y_out")
    y_in, ldi = _rows(y_in, x.rows, w.rows, dt, "y_in")
    y_out, ldo = _rows(y_out, x.rows, w.rows, dt, "y_out")
    ws = _typed(workspace, torch.uint8, dlcx_fp8_product_workspace_bytes(x.rows, w.rows, x.cols), "workspace")
    _check(lib().dlcx_fp8_product(C.addressof(x), C.addressof(w), y_in, ldi, y_out, ldo, _CODE[dt], ws, _stream(stream)),
           "dlcx_fp8_product")


def dlcx_rms_norm(x, weight, eps, residual=None, sum_out=None, y_out=None, y8_out=None, rstd_out=None, stream=None):
    """y_out and y8_out (a matrix in 8 bits): one of them or both; sum_out where there is a residual."""
    dt = _type_of(x, "x")
    rows, n = x.shape
    x, ldx = _rows(x, rows, n, dt, "x")
    residual, ldr = _rows(residual, rows, n, dt, "residual")
    sum_out, lds = _rows(sum_out, rows, n, dt, "sum_out")
    y_out, ldy = _rows(y_out, rows, n, dt, "y_out")
    _check(lib().dlcx_rms_norm(rows, n, _CODE[dt], x, ldx, residual, ldr, _typed(weight, dt, n, "weight"), eps, sum_out,
                               lds, y_out, ldy, _ref(y8_out), _typed(rstd_out, torch.float32, rows, "rstd_out"),
                               _stream(stream)), "dlcx_rms_norm")


def dlcx_rms_norm_workspace_bytes(rows, n):
    return lib().dlcx_rms_norm_workspace_bytes(rows, n)


def dlcx_rms_norm_backward(x, weight, rstd, dy, dx_in, dx_out, dw_out, workspace, stream=None):
    """x: what was normalised (sum_out where there was a residual); dx_in None: zeros."""
    dt = _type_of(x, "x")
    rows, n = x.shape
    x, ldx = _rows(x, rows, n, dt, "x")
    dy, lddy = _rows(dy, rows, n, dt, "dy")
    dx_in, ldi = _rows(dx_in, rows, n, dt, "dx_in")
    dx_out, ldo = _rows(dx_out, rows, n, dt, "dx_out")
    _check(lib().dlcx_rms_norm_backward(rows, n, _CODE[dt], x, ldx, _typed(weight, dt, n, "weight"),
                                        _typed(rstd, torch.float32, rows, "rstd"), dy, lddy, dx_in, ldi, dx_out, ldo,
                                        _typed(dw_out, torch.float32, n, "dw_out"),
                                        _typed(workspace, torch.uint8, dlcx_rms_norm_workspace_bytes(rows, n), "workspace"),
                                        _stream(stream)), "dlcx_rms_norm_backward")


def dlcx_dropout(x, y_in, y_out, p, seed, offset=0, offset_more=None, stream=None):
    """y_out = y_in (None: zeros) + mask x / (1 - p).  seed and offset: 64 bits; offset_more: an int64 device tensor of one
    element that is added to offset when the call runs, or None."""
    dt = _type_of(x, "x")
    rows, cols = x.shape
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise ValueError("seed and offset: numbers of 64 bits are wanted")
    x, ldx = _rows(x, rows, cols, dt, "x")
    y_in, ldi = _rows(y_in, rows, cols, dt, "y_in")
    y_out, ldo = _rows(y_out, rows, cols, dt, "y_out")
    _check(lib().dlcx_dropout(rows, cols, _CODE[dt], x, ldx, y_in, ldi, y_out, ldo, p, seed, offset,
                              _typed(offset_more, torch.int64, 1, "offset_more"), _stream(stream)), "dlcx_dropout")


def dlcx_profile_enable(on):
    _check(lib().dlcx_profile_enable(1 if on else 0), "dlcx_profile_enable")


def dlcx_profile_read():
    """{kernel name: (total ms, launches)} of the launches recorded since dlcx_profile_enable(1)."""
    out = {}
    for kid in range(lib().dlcx_profile_kernels()):
        ms, cnt = C.c_double(0.0), C.c_int64(0)
        _check(lib().dlcx_profile_read(kid, C.addressof(ms), C.addressof(cnt)), "dlcx_profile_read")
        if cnt.value:
            out[lib().dlcx_profile_name(kid).decode()] = (ms.value, cnt.value)
    return out
