"""Python binding of libqnn.so: argument marshalling only.

Device tensors are torch tensors on a HIP device.  The device functions below name and document the
arguments; the compiled module ``_native`` (``csrc/binding.cpp``) checks the tensors, allocates the output and
calls the C ABI (``include/qnn.h``) on the current torch stream -- a Python-level ctypes call took longer than
a small layer runs.  Host helpers and the calibration calls go through ctypes.  No arithmetic of the method
happens in Python.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libqnn.so")
_lib = None

STATUS = {0: "QNN_OK", 1: "QNN_EINVAL", 2: "QNN_EUNSUPPORTED", 3: "QNN_ELAUNCH"}
B_COLUMNS_CONTIGUOUS, B_ROWS_CONTIGUOUS = 0, 1

EXPORTS = [
    "qnn_last_error", "qnn_version", "qnn_qgemm_plan", "qnn_quantize", "qnn_dequantize", "qnn_requantize", "qnn_qgemm", "qnn_pack_b",
    "qnn_qconv2d", "qnn_qdwconv2d", "qnn_qadd", "qnn_qgemm_add", "qnn_qconv2d_add", "qnn_rescale_u8", "qnn_qgemm_asym", "qnn_qconv2d_asym", "qnn_qdwconv2d_asym", "qnn_minmax", "qnn_quantize_with",
    "qnn_quantize_dynamic", "qnn_simquant", "qnn_simquant_backward", "qnn_choose_qparams", "qnn_quantize_multiplier", "qnn_act_range",
    "qnn_qadd_params", "qnn_quantize_weights", "qnn_pack_int4", "qnn_qgemm_workspace_bytes", "qnn_qconv2d_workspace_bytes",
    "qnn_tuning_set", "qnn_calibrate_mfma", "qnn_calibrate_copy", "qnn_qgemm_noalloc", "qnn_quantize_u16", "qnn_dequantize_u16", "qnn_calibrate_rescale",
    "qnn_w4_matmul", "qnn_w4_matmul_workspace_bytes", "qnn_w4_matmul_plan", "qnn_kv_append", "qnn_kv_gather", "qnn_kv_attention", "qnn_kv_attention_workspace_bytes",
    "qnn_quantize_weights_grouped", "qnn_f8_quantize", "qnn_f8_rmsnorm", "qnn_f8_matmul", "qnn_f8_matmul_workspace_bytes", "qnn_f8_matmul_plan", "qnn_f8_moe",
    "qnn_f8_moe_workspace_bytes", "qnn_quantize_weights_blocks",
]


class QnnError(RuntimeError):
    def __init__(self, name, code, detail=""):
        super().__init__(f"{name} failed with {STATUS.get(code, code)}{(': ' + detail) if detail else ''}")
        self.code = code


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libqnn.so.  There is no fallback: a missing library is an error."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(
            f"{_LIB_PATH} is missing: build it first (python -m paper_1806_08342_amd._build, or "
            "__graft_entry__.build()); there is no CPU fallback")
    lib = C.CDLL(_LIB_PATH)
    lib.qnn_last_error.restype = C.c_char_p
    lib.qnn_version.restype = C.c_char_p
    lib.qnn_qgemm_plan.restype = C.c_char_p
    lib.qnn_qgemm_plan.argtypes = [C.c_int64, C.c_int64, C.c_int64]
    vp, i32, i64, sz, f32, f64 = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_float, C.c_double
    ci = C.c_int
    sigs = {
        "qnn_quantize": [vp, vp, sz, f32, i32, i32, i32, vp],
        "qnn_dequantize": [vp, vp, sz, f32, i32, vp],
        "qnn_quantize_u16": [vp, vp, sz, f32, i32, i32, i32, vp],
        "qnn_dequantize_u16": [vp, vp, sz, f32, i32, vp],
        "qnn_requantize": [vp, vp, sz, sz, vp, vp, ci, i32, i32, i32, vp],
        "qnn_qgemm": [vp, i64, i32, vp, i64, ci, ci, i64, i64, i64, vp, vp, vp, i32, i32, i32, vp, i64, vp, sz, vp],
        "qnn_qgemm_noalloc": [vp, i64, i32, vp, i64, ci, ci, i64, i64, i64, vp, vp, vp, i32, i32, i32, vp, i64, vp],
        "qnn_pack_b": [vp, i64, i64, i64, vp, i64, vp],
        "qnn_qconv2d": [vp, ci, ci, ci, ci, i32, vp, ci, ci, ci, ci, ci, ci, ci, ci, vp, vp, vp, i32, i32, i32, vp, vp, sz, vp],
        "qnn_tuning_set": [C.c_char_p, C.c_char_p],
        "qnn_calibrate_mfma": [ci, ci, ci, vp, C.POINTER(f64), vp],
        "qnn_calibrate_rescale": [ci, ci, vp, C.POINTER(f64), vp],
        "qnn_calibrate_copy": [vp, vp, sz, vp],
        "qnn_minmax": [vp, sz, f32, ci, vp, vp],
        "qnn_quantize_with": [vp, vp, sz, vp, vp],
        "qnn_quantize_dynamic": [vp, vp, sz, vp, vp],
        "qnn_simquant": [vp, vp, sz, f32, i32, i32, i32, vp],
        "qnn_simquant_backward": [vp, vp, vp, sz, f32, i32, i32, i32, vp],
        "qnn_qdwconv2d_asym": [vp, ci, ci, ci, ci, i32, vp, ci, ci, vp, ci, ci, ci, ci, vp, vp, vp, i32, i32, i32, vp, vp],
        "qnn_qgemm_asym": [vp, i64, i32, vp, i64, ci, ci, vp, i64, i64, i64, vp, vp, vp, i32, i32, i32, vp, i64, vp, sz, vp],
        "qnn_qconv2d_asym": [vp, ci, ci, ci, ci, i32, vp, ci, ci, ci, ci, vp, ci, ci, ci, ci, vp, vp, vp, i32, i32, i32, vp, vp,
                             sz, vp],
        "qnn_rescale_u8": [vp, i64, i32, i32, i32, i32, i32, i32, vp, i64, i64, i64, vp],
        "qnn_qgemm_add": [vp, i64, i32, vp, i64, ci, ci, i64, i64, i64, vp, vp, vp, i32, i32, i32, vp, i64, vp, vp, i64, vp,
                          sz, vp],
        "qnn_qconv2d_add": [vp, ci, ci, ci, ci, i32, vp, ci, ci, ci, ci, ci, ci, ci, ci, vp, vp, vp, i32, i32, i32, vp, vp,
                            vp, vp, sz, vp],
        "qnn_qdwconv2d": [vp, ci, ci, ci, ci, i32, vp, ci, ci, ci, ci, ci, ci, vp, vp, vp, i32, i32, i32, vp, vp],
        "qnn_qadd": [vp, i32, i32, i32, vp, i32, i32, i32, i32, i32, i32, i32, i32, i32, vp, sz, vp],
        "qnn_choose_qparams": [f64, f64, ci, C.POINTER(f32), C.POINTER(i32)],
        "qnn_quantize_multiplier": [f64, C.POINTER(i32), C.POINTER(i32)],
        "qnn_act_range": [ci, f32, i32, C.POINTER(i32), C.POINTER(i32)],
        "qnn_qadd_params": [f64, f64, f64] + [C.POINTER(i32)] * 7,
        "qnn_quantize_weights": [vp, sz, sz, ci, ci, vp, vp],
        "qnn_pack_int4": [vp, sz, vp],
        "qnn_quantize_weights_grouped": [vp, sz, sz, sz, ci, vp, vp, vp],
        "qnn_w4_matmul": [vp, i64, vp, vp, vp, vp, i64, i64, i64, i64, ci, vp, i64, vp, sz, vp],
        "qnn_kv_append": [vp, vp, i64, i64, vp, i64, i64, ci, vp, vp, vp, i64, i64, i64, vp],
        "qnn_kv_gather": [vp, vp, vp, vp, i64, i64, i64, ci, vp, vp, vp],
        "qnn_kv_attention": [vp, vp, i64, i64, i32, ci, vp, vp, vp, i64, i64, i64, f32, i64, i64, vp, vp, vp, sz, vp],
        "qnn_quantize_weights_blocks": [vp, sz, sz, vp, vp],
        "qnn_f8_quantize": [vp, i64, i64, i64, ci, ci, vp, i64, vp, i64, vp],
        "qnn_f8_rmsnorm": [vp, i64, vp, i64, vp, f32, i64, i64, ci, vp, i64, vp, vp, i64, vp, i64, vp],
        "qnn_f8_matmul": [vp, i64, vp, i64, vp, vp, vp, i64, i64, i64, ci, vp, i64, vp, sz, vp],
        "qnn_f8_moe": [vp, i64, vp, i64, vp, i64, ci, vp, vp, vp, vp, i64, i64, i64, i64, i64, ci, ci, vp, i64, vp, vp, vp, sz, vp],
    }
    for name, args in sigs.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = C.c_int
    lib.qnn_qgemm_workspace_bytes.restype = sz
    lib.qnn_qgemm_workspace_bytes.argtypes = [i64, i64, i64, ci, ci]
    lib.qnn_qconv2d_workspace_bytes.restype = sz
    lib.qnn_qconv2d_workspace_bytes.argtypes = [ci] * 13
    lib.qnn_w4_matmul_plan.restype = C.c_char_p
    lib.qnn_w4_matmul_plan.argtypes = [i64] * 4
    lib.qnn_w4_matmul_workspace_bytes.restype = sz
    lib.qnn_w4_matmul_workspace_bytes.argtypes = [i64] * 4
    lib.qnn_kv_attention_workspace_bytes.restype = sz
    lib.qnn_kv_attention_workspace_bytes.argtypes = [vp, i32, i64, i64, i64, i64, i64]
    lib.qnn_f8_matmul_plan.restype = C.c_char_p
    lib.qnn_f8_matmul_plan.argtypes = [i64, i64, i64, ci]
    lib.qnn_f8_matmul_workspace_bytes.restype = sz
    lib.qnn_f8_matmul_workspace_bytes.argtypes = [i64, i64, i64, ci]
    lib.qnn_f8_moe_workspace_bytes.restype = sz
    lib.qnn_f8_moe_workspace_bytes.argtypes = [i64] * 5
    _lib = lib
    return lib


def _check(name, rc):
    if rc != 0:
        detail = load_library().qnn_last_error().decode() if rc in (2, 3) else ""
        raise QnnError(name, rc, detail)


def _torch():
    import torch

    return torch


_nat = None  # the compiled module, once loaded


def _native():
    """Load the compiled binding (and with it libqnn.so).  There is no fallback: a missing module is an error."""
    global _nat
    if _nat is None:
        load_library()
        _torch()  # its shared libraries are what the module links against
        try:
            from . import _native as mod
        except ImportError as e:
            raise RuntimeError(f"the compiled binding is missing or unusable ({e}): build it first (python -m "
                               "paper_1806_08342_amd._build, or __graft_entry__.build()); there is no Python fallback") from e
        mod.set_check(_check)
        _nat = mod
    return _nat


def _stream():
    return C.c_void_p(_torch().cuda.current_stream().cuda_stream)


def _dev(t, dtype, name):
    torch = _torch()
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError(f"{name}: expected a contiguous device tensor of {dtype}, got "
                        f"{getattr(t, 'dtype', type(t))} on {getattr(t, 'device', '?')}")
    return C.c_void_p(t.data_ptr())


def _dev_rows(t, dtype, name):
    """Pointer and row pitch (in elements) of a 2-D device tensor whose rows are contiguous but may be
    spaced apart (a column slice of a wider matrix)."""
    torch = _torch()
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.dim() == 2 and
            (t.shape[1] == 1 or t.stride(1) == 1) and (t.shape[0] == 1 or t.stride(0) >= t.shape[1])):
        raise TypeError(f"{name}: expected a 2-D device tensor of {dtype} with contiguous rows")
    return C.c_void_p(t.data_ptr()), (t.stride(0) if t.shape[0] > 1 else t.shape[1])


def _workspace(nbytes, device, workspace):
    """(pointer, size) of the scratch memory of a dense call: the caller's uint8 tensor, else a fresh
    one of the size the library asks for (none when that is 0).  The tensor is returned too, so that it
    stays referenced until the call has been enqueued (torch frees memory in stream order)."""
    torch = _torch()
    if workspace is not None:
        if not (isinstance(workspace, torch.Tensor) and workspace.is_cuda and workspace.dtype == torch.uint8 and
                workspace.is_contiguous()):
            raise TypeError("workspace: expected a contiguous uint8 device tensor")
        return C.c_void_p(workspace.data_ptr()), workspace.numel(), workspace
    if nbytes == 0:
        return None, 0, None
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return C.c_void_p(ws.data_ptr()), nbytes, ws


def qgemm_workspace_bytes(M, N, K, weight_bits=8, asym=False):
    return int(load_library().qnn_qgemm_workspace_bytes(int(M), int(N), int(K), int(weight_bits), int(bool(asym))))


def qconv2d_workspace_bytes(N, H, W, Cin, Cout, kh, kw, stride, pad, weight_bits=8, asym=False):
    return int(load_library().qnn_qconv2d_workspace_bytes(int(N), int(H), int(W), int(Cin), int(Cout), int(kh), int(kw),
                                                          int(weight_bits), stride[0], stride[1], pad[0], pad[1],
                                                          int(bool(asym))))


def calibrate_mfma(workgroups, iters, random_operands, sink):
    """Enqueue the register-only MFMA loop; returns the integer operations of the launch."""
    torch = _torch()
    ops = C.c_double()
    _check("qnn_calibrate_mfma", load_library().qnn_calibrate_mfma(int(workgroups), int(iters), int(bool(random_operands)),
                                                                   _dev(sink, torch.int32, "sink"), C.byref(ops), _stream()))
    return float(ops.value)


def calibrate_rescale(workgroups, iters, sink):
    """Enqueue the register-only rescale loop; returns the number of accumulators it rescales."""
    torch = _torch()
    n = C.c_double()
    _check("qnn_calibrate_rescale", load_library().qnn_calibrate_rescale(int(workgroups), int(iters), _dev(sink, torch.int32, "sink"),
                                                                         C.byref(n), _stream()))
    return float(n.value)


def calibrate_copy(src, dst):
    torch = _torch()
    _check("qnn_calibrate_copy", load_library().qnn_calibrate_copy(_dev(src, torch.uint8, "src"), _dev(dst, torch.uint8, "dst"),
                                                                   src.numel(), _stream()))
    return dst


def tuning_set(name, value=None):
    """Set a tuning switch of the library (see qnn_tuning_set); value None restores the default."""
    v = None if value is None else str(value).encode()
    _check("qnn_tuning_set", load_library().qnn_tuning_set(name.encode(), v))


# ------------------------------------------------------------------ host helpers

def choose_qparams(xmin, xmax, bits=8):
    s, z = C.c_float(), C.c_int32()
    _check("qnn_choose_qparams", load_library().qnn_choose_qparams(xmin, xmax, bits, C.byref(s), C.byref(z)))
    return float(s.value), int(z.value)


def quantize_multiplier(real_mult):
    m, s = C.c_int32(), C.c_int32()
    _check("qnn_quantize_multiplier", load_library().qnn_quantize_multiplier(float(real_mult), C.byref(m), C.byref(s)))
    return int(m.value), int(s.value)


def quantize_multipliers(real_mults):
    """Vector form: returns (mult, shift) as int32 numpy arrays."""
    vals = np.asarray(real_mults, dtype=np.float64).ravel()
    out = [quantize_multiplier(v) for v in vals]
    return (np.array([o[0] for o in out], dtype=np.int32), np.array([o[1] for o in out], dtype=np.int32))


def act_range(kind, s_out, z_out):
    lo, hi = C.c_int32(), C.c_int32()
    _check("qnn_act_range", load_library().qnn_act_range(int(kind), float(s_out), int(z_out), C.byref(lo), C.byref(hi)))
    return int(lo.value), int(hi.value)


def qadd_params(s_a, s_b, s_out):
    v = [C.c_int32() for _ in range(7)]
    _check("qnn_qadd_params", load_library().qnn_qadd_params(float(s_a), float(s_b), float(s_out), *[C.byref(t) for t in v]))
    names = ["left_shift", "mult_a", "shift_a", "mult_b", "shift_b", "mult_o", "shift_o"]
    return {k: int(t.value) for k, t in zip(names, v)}


def quantize_weights(w, bits=8, restricted=True):
    """Host fp32 array [channels, ...] -> (int8 array of the same shape, Delta_c[channels])."""
    w = np.ascontiguousarray(w, dtype=np.float32)
    ch = w.shape[0]
    wq = np.empty(w.shape, dtype=np.int8)
    d = np.empty(ch, dtype=np.float32)
    _check("qnn_quantize_weights", load_library().qnn_quantize_weights(
        w.ctypes.data, ch, w.size // ch, int(bits), int(bool(restricted)), wq.ctypes.data, d.ctypes.data))
    return wq, d


def pack_int4(v):
    v = np.ascontiguousarray(v, dtype=np.int8)
    out = np.empty(v.shape[:-1] + (v.shape[-1] // 2,), dtype=np.uint8)
    _check("qnn_pack_int4", load_library().qnn_pack_int4(v.ctypes.data, v.size, out.ctypes.data))
    return out


def qgemm_plan(M, N, K):
    """Tile configuration the dense kernels pick for an M x N x K product."""
    return load_library().qnn_qgemm_plan(int(M), int(N), int(K)).decode()


# ---------------------------------------------------------------- device kernels

def quantize(x, scale, zero_point, qmin=0, qmax=255, out=None):
    return (_nat or _native()).quantize(x, scale, zero_point, qmin, qmax, out)


def dequantize(q, scale, zero_point, out=None):
    return (_nat or _native()).dequantize(q, scale, zero_point, out)


def quantize_u16(x, scale, zero_point, qmin=0, qmax=65535, out=None):
    """Codes of up to 16 bits as a uint16 tensor."""
    return (_nat or _native()).quantize_u16(x, scale, zero_point, qmin, qmax, out)


def dequantize_u16(q, scale, zero_point, out=None):
    return (_nat or _native()).dequantize_u16(q, scale, zero_point, out)


def requantize(acc, mult, shift, per_channel, z_out, act_min, act_max, out=None):
    return (_nat or _native()).requantize(acc, mult, shift, per_channel, z_out, act_min, act_max, out)


def qgemm(A, z_a, B, mult, shift, z_out, act_min, act_max, bias=None, weight_bits=8,
          b_layout=B_COLUMNS_CONTIGUOUS, out=None, workspace=None):
    """A: uint8 [M,K] (rows may be spaced apart: a column slice of a wider matrix; same for `out`).  B: int8 [N,K] (columns contiguous), int8 [K,N] (rows contiguous), or uint8
    [N,K/2] nibble-packed when weight_bits == 4.  Returns uint8 [M,N]."""
    return (_nat or _native()).qgemm(A, z_a, B, mult, shift, z_out, act_min, act_max, bias, weight_bits, b_layout, out, workspace)


def qgemm_noalloc(A, z_a, B, mult, shift, z_out, act_min, act_max, out, bias=None, weight_bits=8):
    """qnn_qgemm_noalloc: `qgemm` with columns-contiguous B into the caller's `out`, with the library's static
    scratch array; neither this wrapper nor the library allocates."""
    return (_nat or _native()).qgemm_noalloc(A, z_a, B, mult, shift, z_out, act_min, act_max, out, bias, weight_bits)


def prepare_qgemm(A, z_a, B, mult, shift, z_out, act_min, act_max, out, bias=None, weight_bits=8,
                  b_layout=B_COLUMNS_CONTIGUOUS, workspace=None):
    """Marshal the arguments of `qgemm` once and return a zero-argument callable that enqueues the
    product on the current stream.  For launch-bound loops: the per-call Python work shrinks to one
    foreign call.  The tensors must stay alive and unchanged in shape while the callable is used."""
    torch = _torch()
    M, K = A.shape
    if weight_bits == 4:
        N, ldb, bp = B.shape[0], B.shape[1] * 2, _dev(B, torch.uint8, "B")
    elif b_layout == B_COLUMNS_CONTIGUOUS:
        (N, ldb), bp = B.shape, _dev(B, torch.int8, "B")
    else:
        ldb = N = B.shape[1]
        bp = _dev(B, torch.int8, "B")
    fn = load_library().qnn_qgemm
    ap, lda = _dev_rows(A, torch.uint8, "A")
    cp, ldc = _dev_rows(out, torch.uint8, "C")
    wp, wbytes, ws = _workspace(qgemm_workspace_bytes(M, N, K, weight_bits), A.device, workspace)
    args = (ap, lda, z_a, bp, ldb, b_layout, weight_bits, M, N, K, _dev(bias, torch.int32, "bias"),
            _dev(mult, torch.int32, "mult"), _dev(shift, torch.int32, "shift"), z_out, act_min, act_max, cp, ldc,
            wp, wbytes)
    keep = (A, B, mult, shift, bias, out, ws)
    current_stream = torch.cuda.current_stream

    def launch(_keep=keep):
        rc = fn(*args, current_stream().cuda_stream)
        if rc != 0:
            _check("qnn_qgemm", rc)

    return launch


def pack_b(B_rows):
    """int8 [K,N] with contiguous rows -> int8 [N,K] (the layout qgemm runs fastest on)."""
    return (_nat or _native()).pack_b(B_rows)


def qconv2d(x, z_x, w, stride, pad, mult, shift, z_out, act_min, act_max, bias=None, weight_bits=8, out=None,
            workspace=None):
    """x: uint8 NHWC.  w: int8 [Cout,kh,kw,Cin], or uint8 [Cout,kh,kw,Cin/2] packed 4-bit."""
    return (_nat or _native()).qconv2d(x, z_x, w, stride, pad, mult, shift, z_out, act_min, act_max, bias, weight_bits, out, workspace)


class _AddParams(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("mult_m", "shift_m", "z_r", "mult_r", "shift_r", "left_shift", "mult_o",
                                         "shift_o", "z_out", "act_min", "act_max")]


def qgemm_add(A, z_a, B, mult, shift, z_mid, mid_min, mid_max, residual, z_r, params, z_out, act_min, act_max,
              bias=None, weight_bits=8, out=None, workspace=None):
    """qgemm (columns-contiguous B) whose uint8 result, quantized with (z_mid, mid_min, mid_max), is added to
    `residual` (uint8 [M,N], rows may be spaced apart) with the rescaling add of `params` (what
    qadd_params(s_mid, s_residual, s_out) returns); returns uint8 [M,N]."""
    return (_nat or _native()).qgemm_add(A, z_a, B, mult, shift, z_mid, mid_min, mid_max, residual, z_r, params, z_out, act_min,
                                         act_max, bias, weight_bits, out, workspace)


def qconv2d_add(x, z_x, w, stride, pad, mult, shift, z_mid, mid_min, mid_max, residual, z_r, params, z_out, act_min,
                act_max, bias=None, weight_bits=8, out=None, workspace=None):
    """qconv2d followed by the rescaling add with `residual` (uint8 NHWC, the shape of the output), fused."""
    return (_nat or _native()).qconv2d_add(x, z_x, w, stride, pad, mult, shift, z_mid, mid_min, mid_max, residual, z_r, params, z_out,
                                           act_min, act_max, bias, weight_bits, out, workspace)


def qgemm_asym(A, z_a, B, z_w, mult, shift, z_out, act_min, act_max, bias=None, weight_bits=8, out=None, workspace=None):
    """qgemm with a zero-point per weight column: z_w int32 [N] on the device.  B: int8 [N,K] (columns
    contiguous) or uint8 [N,K/2] nibble-packed."""
    return (_nat or _native()).qgemm_asym(A, z_a, B, z_w, mult, shift, z_out, act_min, act_max, bias, weight_bits, out, workspace)


def qconv2d_asym(x, z_x, w, z_w, stride, pad, mult, shift, z_out, act_min, act_max, bias=None, weight_bits=8, out=None,
                 workspace=None):
    """qconv2d with a zero-point per output channel: z_w int32 [Cout] on the device."""
    return (_nat or _native()).qconv2d_asym(x, z_x, w, z_w, stride, pad, mult, shift, z_out, act_min, act_max, bias, weight_bits, out,
                                            workspace)


def new_range_state(xmin=0.0, xmax=0.0):
    """Device-resident quantizer state (qnn_dyn_qparams: scale, zero_point, xmin, xmax, 2 work words) as
    an int32 tensor of 6 elements; `read_range_state` decodes it."""
    torch = _torch()
    host = np.zeros(6, dtype=np.int32)
    host[2:4] = np.array([xmin, xmax], dtype=np.float32).view(np.int32)
    return torch.from_numpy(host).to("cuda:0")


def read_range_state(state):
    h = state.cpu().numpy()
    f = h.view(np.float32)
    return dict(scale=float(f[0]), zero_point=int(h[1]), xmin=float(f[2]), xmax=float(f[3]))


def minmax(x, state, momentum=0.0, bits=8):
    """Range of the finite elements of x (or its moving average) and the quantizer parameters, into `state`."""
    return (_nat or _native()).minmax(x, state, momentum, bits)


def quantize_with(x, state, out=None):
    return (_nat or _native()).quantize_with(x, state, out)


def quantize_dynamic(x, state, out=None):
    """uint8 codes of x with the quantizer of its own range; the parameters are left in `state`."""
    return (_nat or _native()).quantize_dynamic(x, state, out)


def simquant(x, scale, zero_point, qmin=0, qmax=255, out=None):
    return (_nat or _native()).simquant(x, scale, zero_point, qmin, qmax, out)


def simquant_backward(x, grad_y, scale, zero_point, qmin=0, qmax=255, out=None):
    return (_nat or _native()).simquant_backward(x, grad_y, scale, zero_point, qmin, qmax, out)


def rescale_u8(x, z_in, mult, shift, z_out, act_min=0, act_max=255, out=None):
    """uint8 [rows, cols] (rows may be spaced apart) re-quantized to another quantizer; `out` may be a
    column slice of a wider tensor (the destination of a concatenation)."""
    return (_nat or _native()).rescale_u8(x, z_in, mult, shift, z_out, act_min, act_max, out)


def qdwconv2d_asym(x, z_x, w, z_w, stride, pad, mult, shift, z_out, act_min, act_max, bias=None, out=None):
    """Depthwise layer with a weight zero-point per channel: z_w int32 [C] on the device."""
    return (_nat or _native()).qdwconv2d_asym(x, z_x, w, z_w, stride, pad, mult, shift, z_out, act_min, act_max, bias, out)


def qdwconv2d(x, z_x, w, stride, pad, mult, shift, z_out, act_min, act_max, bias=None, out=None):
    """x: uint8 NHWC.  w: int8 [kh,kw,C]."""
    return (_nat or _native()).qdwconv2d(x, z_x, w, stride, pad, mult, shift, z_out, act_min, act_max, bias, out)


def qadd(a, z_a, b, z_b, params, z_out, act_min, act_max, out=None):
    return (_nat or _native()).qadd(a, z_a, b, z_b, params, z_out, act_min, act_max, out)


# ------------------------------------------------------------------------------- quantized language models

BF16, F16 = 0, 1


def _half_code(dtype):
    torch = _torch()
    if dtype not in (torch.bfloat16, torch.float16):
        raise ValueError(f"expected torch.bfloat16 or torch.float16, got {dtype}")
    return BF16 if dtype == torch.bfloat16 else F16


def quantize_weights_grouped(w, group=128, dtype=None, asymmetric=False):
    """fp32 [N,K] (numpy, finite, K even) -> what `w4_matmul` takes, on the host: codes uint8 [N,K/2], scales
    [ceil(K/group),N] of `dtype` (torch.bfloat16 unless given), zeros int8 of the same shape or None (symmetric)."""
    torch = _torch()
    dtype = dtype or torch.bfloat16
    w = np.ascontiguousarray(w, dtype=np.float32)
    if w.ndim != 2:
        raise ValueError(f"expected weights [N, K], got shape {w.shape}")
    n, k = w.shape
    groups = -(-k // group) if group > 0 else 0
    codes = np.empty((n, k // 2), np.uint8)
    scales = np.empty((groups, n), np.uint16)
    zeros = np.empty((groups, n), np.int8) if asymmetric else None
    _check("qnn_quantize_weights_grouped", load_library().qnn_quantize_weights_grouped(
        w.ctypes.data, n, k, max(group, 0), _half_code(dtype), codes.ctypes.data, scales.ctypes.data, zeros.ctypes.data if asymmetric else None))
    as_half = torch.from_numpy(scales.view(np.int16)).view(dtype)
    return torch.from_numpy(codes), as_half, torch.from_numpy(zeros) if asymmetric else None


def w4_matmul(x, codes, scales, group, zeros=None, bias=None, out=None, workspace=None):
    """x [M,K] (bfloat16 or float16, rows may be spaced apart) times 4-bit weights [N,K] with one scale per `group` weights of
    a row: y[m,n] = bias[n] + sum_k x[m,k] * (c[n,k] - zeros[k//group,n]) * scales[k//group,n].  codes: uint8 [N,K/2]
    (as `pack_int4` packs rows); scales: [ceil(K/group),N] of x's type; zeros: int8 of that shape or None; group: a multiple of
    32.  Returns [M,N] of x's type.  For inference: tensors that require grad are refused while gradients are recorded."""
    return (_nat or _native()).w4_matmul(x, codes, scales, group, zeros, bias, out, workspace)


def w4_matmul_plan(M, N, K, group=128):
    """Name of the kernel that `w4_matmul` runs for these sizes."""
    return load_library().qnn_w4_matmul_plan(M, N, K, group).decode()


def new_kv_cache(pages, heads, dim, block=64, device="cuda:0"):
    """A cache of keys and values in 8 bits with one scale per page (`block` tokens of a request) and head:
    (k_codes int8 [pages,heads,block,dim], k_scales float32 [pages,heads], v_codes int8 [pages,heads,dim,block], v_scales)."""
    torch = _torch()
    return (torch.zeros(pages, heads, block, dim, dtype=torch.int8, device=device), torch.zeros(pages, heads, device=device),
            torch.zeros(pages, heads, dim, block, dtype=torch.int8, device=device), torch.zeros(pages, heads, device=device))


def kv_append(cache, k, v, cu, start, table):
    """Append rows cu[r]:cu[r+1] of k and v ([T,heads,dim], bfloat16 or float16, views with a contiguous last dimension will do)
    to request r, which holds start[r] tokens.  cu int32 [R+1], start int32 [R], table int32 [R,W]: page of its tokens
    j*block and up.  Where a block's range grows, the codes it holds are rescaled.  Tensors that require grad are refused while
    gradients are recorded."""
    (_nat or _native()).kv_append(cache, k, v, cu, start, table)


def kv_gather(cache, cu, first, table, tokens, dtype):
    """The cached tokens first[r] + i as rows cu[r] + i of (k, v), each [tokens,heads,dim] of `dtype`.  Rows from cu[-1] on are
    uninitialised; a token without a page gives 0."""
    return (_nat or _native()).kv_gather(cache, cu, first, table, tokens, _half_code(dtype))


def kv_attention(cache, q, cu, lengths, table, scale=None, window=0, max_queries=None, with_lse=False, out=None, workspace=None):
    """Attention of q [T,q_heads,dim] over the cache: rows cu[r]:cu[r+1] are the queries of request r's last tokens (of
    lengths[r] in the cache), each sees the tokens up to its own, the last `window` of them if window > 0.  q_heads is a multiple
    of the cache's heads.  scale: 1/sqrt(dim) unless given.  max_queries: the largest number of queries of a request (T unless
    given).  Returns [T,q_heads,dim] of q's type, with_lse: and the logarithm of each row's sum, float32 [T,q_heads].  A query
    that sees nothing gives 0 (and -inf); rows that no request has stay as they are (uninitialised without `out`).  For inference:
    tensors that require grad are refused while gradients are recorded."""
    if scale is None:
        scale = q.shape[-1] ** -0.5
    return (_nat or _native()).kv_attention(cache, q, cu, lengths, table, scale, window, max_queries or 0, with_lse, out, workspace)


# ------------------------------------------------------------------------------- language models in 8-bit floating point

F32 = 2


def _float_code(dtype):
    torch = _torch()
    codes = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}
    if dtype not in codes:
        raise ValueError(f"expected torch.bfloat16, torch.float16 or torch.float32, got {dtype}")
    return codes[dtype]


def quantize_weights_blocks(w):
    """fp32 [N,K] (numpy, finite) -> what `f8_matmul` takes, on the host: codes float8_e4m3fn [N,K] and float32 scales
    [ceil(N/128),ceil(K/128)], one per block of 128 x 128: max|w| / 448.  [E,N,K]: the same for each expert of `f8_moe`."""
    torch = _torch()
    w = np.ascontiguousarray(w, dtype=np.float32)
    if w.ndim == 3 and w.shape[0] > 0:
        each = [quantize_weights_blocks(m) for m in w]
        return torch.stack([c.view(torch.uint8) for c, _ in each]).view(torch.float8_e4m3fn), torch.stack([s for _, s in each])
    if w.ndim != 2:
        raise ValueError(f"expected weights [N, K] or [E, N, K], got shape {w.shape}")
    n, k = w.shape
    codes = np.empty((n, k), np.uint8)
    scales = np.empty((-(-n // 128), -(-k // 128)), np.float32)
    _check("qnn_quantize_weights_blocks", load_library().qnn_quantize_weights_blocks(w.ctypes.data, n, k, codes.ctypes.data, scales.ctypes.data))
    return torch.from_numpy(codes).view(torch.float8_e4m3fn), torch.from_numpy(scales)


def f8_quantize(x, gated=False, out=None):
    """Rows of x [M,K] (bfloat16 or float16, rows may be spaced apart) as (codes float8_e4m3fn [M,K], scales float32
    [ceil(K/128),M]): one scale for 128 consecutive elements, their largest finite one / 448 (2^-80 at least).  gated: x is [M,2K],
    and silu(x[:,:K]) * x[:,K:] is what is quantized.  out: (codes, scales) to write to, rows may be spaced apart; new ones are two
    tensors in one piece of memory, which stays while either lives."""
    return (_nat or _native()).f8_quantize(x, gated, out)


def f8_rmsnorm(x, weight=None, eps=1e-6, residual=None, total=None, with_y=False, out=None):
    """Root-mean-square norm of rows as codes and scales (see `f8_quantize`): h = x, or x + residual rounded to x's type;
    v = h / sqrt(mean(h^2) + eps) * weight.  Returns (codes, scales), with a residual (codes, scales, h), and with_y one more: v
    rounded to x's type (codes may then differ from those without where a quotient lies next to the middle of two, and scales in their
    last bits).  total: where to write h (residual or x themselves will do: in place); out: (codes, scales) to write to."""
    return (_nat or _native()).f8_rmsnorm(x, weight, eps, residual, total, with_y, out)


def f8_matmul(x, x_scales, w, w_scales, bias=None, dtype=None, out=None, workspace=None):
    """x [M,K] times w [N,K] transposed, both float8_e4m3fn: y[m,n] = bias[n] + sum_k x[m,k] * x_scales[k//128,m] * w[n,k] *
    w_scales[n//128,k//128].  x's rows may be spaced apart; where K is a multiple of 16 and x's pitch or address is not, many rows take several
    times as long (a copy of it first is faster).  dtype: bfloat16 (unless given), float16, or float32, whose sums are exact
    to binary32 (at half the matrix rate; with 16-bit results a block's sum has a relative error of about 1e-5); the bias is of that type.
    For inference: tensors that require grad are refused while gradients are recorded."""
    return (_nat or _native()).f8_matmul(x, x_scales, w, w_scales, bias, dtype, out, workspace)


def f8_matmul_plan(M, N, K, dtype=None):
    """Name of the kernel that `f8_matmul` runs for these sizes (x and its pitch at multiples of 16 bytes)."""
    return load_library().qnn_f8_matmul_plan(M, N, K, BF16 if dtype is None else _float_code(dtype)).decode()


def f8_moe(x, x_scales, logits, up, up_scales, down, down_scales, top_k, renormalize=True, dtype=None, with_choice=False, out=None, workspace=None):
    """A layer of experts for a few tokens: x [T,H] codes and scales as `f8_quantize` and `f8_rmsnorm` give them, logits [T,E]
    (float32, bfloat16 or float16), up float8_e4m3fn [E,2*I,H] (gate's rows, then up's) with scales [E,ceil(2I/128),ceil(H/128)], down
    [E,H,I] with [E,ceil(H/128),ceil(I/128)].  A token goes to its top_k largest logits (ties: the lowest index; never to -inf or NaN),
    weighed by softmax over these (renormalize) or over all logits: y[t] = sum_e weight * down[e] @ (silu(gate[e] @ x) * (up[e] @ x)).
    Returns [T,H] of dtype (bfloat16 unless given, or float16), with_choice: (y, experts int32 [T,top_k], weights float32).
    H and I: multiples of 16.  Reads the chosen experts' weights once for every 64 tokens."""
    return (_nat or _native()).f8_moe(x, x_scales, logits, up, up_scales, down, down_scales, top_k, renormalize, dtype, with_choice, out, workspace)
