"""ctypes binding of libfq (argument marshalling only).

Function names and arguments mirror ``include/fq.h``.  The ``*_raw`` functions
take integer device addresses exactly as the C ABI does; the helpers below them
take torch tensors (torch is used for device memory and streams only).
"""
from __future__ import annotations

import array
import ctypes
import importlib.util
import os
import warnings

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfq.so")

FQ_OK = 0
FQ_ERR_INVALID_ARG = 1
FQ_ERR_UNSUPPORTED = 2
FQ_ERR_WORKSPACE = 3
FQ_ERR_HIP = 4
FQ_F16 = 0
FQ_BF16 = 1
FQ_SCALE_F16 = 0
FQ_SCALE_BF16 = 1

_lib = None


class Heads(ctypes.Structure):
    """fq_heads: rows of heads in device memory, strides in elements."""
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class KvPages(ctypes.Structure):
    """fq_kv_pages: a cache of keys and values in pages, strides in elements."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("pages", ctypes.c_int64), ("page_size", ctypes.c_int),
                ("page_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class FqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)}")


def load(build_if_missing: bool = True) -> ctypes.CDLL:
    """Loads libfq.so (building it with hipcc first if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        if not build_if_missing:
            raise FileNotFoundError(LIB_PATH)
        from . import build

        build.build_lib(verbose=False)
    lib = ctypes.CDLL(LIB_PATH)
    i64, i32, vp, sz, f32 = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float
    sigs = {
        "fq_codes_bytes": (sz, [i64, i64, i32]),
        "fq_scales_bytes": (sz, [i64, i64, i32]),
        "fq_gemm_workspace_bytes": (sz, [i64, i64, i64, i32, i32]),
        "fq_gemm_workspace_bytes_for": (sz, [i64, i64, i64, i32, i32, i32, i32]),
        "fq_gemm_grouped_workspace_bytes": (sz, [i64, i32, i64, i64, i32, i32]),
        "fq_choose_group_workspace_bytes": (sz, [i64, i64, i32, i32]),
        "fq_quantize": (i32, [vp, i64, i64, i32, i32, vp, vp, vp]),
        "fq_unpack": (i32, [vp, i64, i64, i32, vp, vp]),
        "fq_choose_group": (i32, [vp, i64, i64, i32, i32, f32, ctypes.POINTER(ctypes.c_int), vp, sz, vp]),
        "fq_quant_error_workspace_bytes": (sz, [i64, i64]),
        "fq_quant_error": (i32, [vp, i64, i64, i32, i32, vp, vp, ctypes.POINTER(ctypes.c_double),
                                 ctypes.POINTER(ctypes.c_double), vp, sz, vp]),
        "fq_gemm": (i32, [vp, i32, i64, i64, i64, vp, vp, i32, i32, vp, vp, sz, vp]),
        "fq_gemm_grouped": (i32, [vp, i32, ctypes.POINTER(ctypes.c_int32), i32, i64, i64, vp, vp, i32, i32,
                                  vp, vp, sz, vp]),
        "fq_quantize_sf": (i32, [vp, i64, i64, i32, i32, i32, vp, vp, vp]),
        "fq_quant_error_sf": (i32, [vp, i64, i64, i32, i32, i32, vp, vp, ctypes.POINTER(ctypes.c_double),
                                    ctypes.POINTER(ctypes.c_double), vp, sz, vp]),
        "fq_gemm_sf": (i32, [vp, i32, i64, i64, i64, vp, vp, i32, i32, i32, vp, vp, sz, vp]),
        "fq_gemm_grouped_sf": (i32, [vp, i32, ctypes.POINTER(ctypes.c_int32), i32, i64, i64, vp, vp, i32, i32, i32,
                                     vp, vp, sz, vp]),
        "fq_gemm_noalloc": (i32, [vp, i32, i64, i64, i64, vp, vp, i32, i32, vp, vp]),
        "fq_gemm_noalloc_scratch_bytes": (sz, []),
        "fq_zscale_bytes": (sz, [i64, i64, i32]),
        "fq_quantize_w4a8": (i32, [vp, i64, i64, i32, vp, vp, vp, vp]),
        "fq_quantize_act_i8": (i32, [vp, i32, i64, i64, vp, vp, vp]),
        "fq_unpack_w4a8": (i32, [vp, i64, i64, vp, vp]),
        "fq_gemm_w4a8_workspace_bytes": (sz, [i64, i64, i64, i32]),
        "fq_gemm_w4a8": (i32, [vp, vp, i64, i64, i64, vp, vp, vp, i32, vp, i32, vp, sz, vp]),
        "fq_gemm_describe": (i32, [i64, i64, i64, i32, i32, ctypes.c_char_p, sz]),
        "fq_gemm_grouped_describe": (i32, [ctypes.POINTER(ctypes.c_int32), i32, i64, i64, i32, i32, ctypes.c_char_p, sz]),
        "fq_stream_read_probe": (i32, [vp, sz, vp, vp]),
        "fq_mfma_rate_probe_operand_bytes": (sz, []),
        "fq_mfma_rate_probe_sink_bytes": (sz, []),
        "fq_mfma_rate_probe_flops": (ctypes.c_double, [i32, i32]),
        "fq_mfma_rate_probe": (i32, [vp, sz, vp, sz, i32, i32, i32, vp]),
        "fq_qk_norm_rope": (i32, [vp, i32, i64, i64, i32, i32, i32, vp, vp, f32, vp, i64, i32, i32, vp, vp, vp,
                                  ctypes.POINTER(KvPages), vp, vp]),
        "fq_attention_prompt_workspace_bytes": (sz, [i32, i32, i32, ctypes.POINTER(ctypes.c_int32),
                                                     ctypes.POINTER(ctypes.c_int32), i32]),
        "fq_attention_prompt": (i32, [ctypes.POINTER(Heads), ctypes.POINTER(Heads), ctypes.POINTER(Heads), i32, i32, i32, i32,
                                      ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32), i32, f32, vp, vp, sz, vp]),
        "fq_attention_tree_workspace_bytes": (sz, [i64, i64, i32, i32, i32, i64, i32]),
        "fq_attention_tree": (i32, [ctypes.POINTER(Heads), i32, i64, i64, i32, i32, i32, ctypes.POINTER(KvPages), vp, i64, vp, vp,
                                    i64, f32, vp, vp, sz, vp]),
        "fq_status_string": (ctypes.c_char_p, [i32]),
        "fq_version": (ctypes.c_char_p, []),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


EXPORTED = [
    "fq_codes_bytes", "fq_scales_bytes", "fq_gemm_workspace_bytes", "fq_gemm_grouped_workspace_bytes",
    "fq_choose_group_workspace_bytes", "fq_quantize", "fq_unpack", "fq_choose_group", "fq_gemm",
    "fq_gemm_grouped", "fq_gemm_describe", "fq_gemm_grouped_describe", "fq_status_string", "fq_version",
    "fq_quant_error_workspace_bytes", "fq_quant_error",
    "fq_quantize_sf", "fq_quant_error_sf", "fq_gemm_sf", "fq_gemm_grouped_sf", "fq_gemm_workspace_bytes_for",
    "fq_stream_read_probe", "fq_gemm_noalloc", "fq_gemm_noalloc_scratch_bytes",
    "fq_mfma_rate_probe_operand_bytes", "fq_mfma_rate_probe_sink_bytes", "fq_mfma_rate_probe_flops", "fq_mfma_rate_probe",
    "fq_zscale_bytes", "fq_unpack_w4a8", "fq_quantize_w4a8", "fq_quantize_act_i8", "fq_gemm_w4a8_workspace_bytes", "fq_gemm_w4a8",
    "fq_qk_norm_rope", "fq_attention_prompt_workspace_bytes", "fq_attention_prompt", "fq_attention_tree_workspace_bytes",
    "fq_attention_tree",
]


def stream_read_probe_raw(buf_ptr, nbytes, sink_ptr, stream=0):
    return int(load().fq_stream_read_probe(buf_ptr, nbytes, sink_ptr, stream))


def mfma_rate_probe_operand_bytes():
    return int(load().fq_mfma_rate_probe_operand_bytes())


def mfma_rate_probe_sink_bytes():
    return int(load().fq_mfma_rate_probe_sink_bytes())


def mfma_rate_probe_flops(iterations, int8=0):
    return float(load().fq_mfma_rate_probe_flops(int(iterations), int(int8)))


def mfma_rate_probe_raw(operands_ptr, operand_bytes, sink_ptr, sink_bytes, iterations, lds_reads, int8=0, stream=0):
    return int(load().fq_mfma_rate_probe(operands_ptr, operand_bytes, sink_ptr, sink_bytes, iterations, lds_reads,
                                         int8, stream))


def status_string(status: int) -> str:
    return load().fq_status_string(int(status)).decode()


def version() -> str:
    return load().fq_version().decode()


# ------------------------------------------------------------------ raw (addresses) layer
def codes_bytes(K, N, bits):
    return int(load().fq_codes_bytes(K, N, bits))


def scales_bytes(K, N, group_size):
    return int(load().fq_scales_bytes(K, N, group_size))


def gemm_workspace_bytes(M, N, K, bits, group_size):
    return int(load().fq_gemm_workspace_bytes(M, N, K, bits, group_size))


def gemm_workspace_bytes_for(M, N, K, bits, group_size, act_dtype, scale_format=FQ_SCALE_F16):
    return int(load().fq_gemm_workspace_bytes_for(M, N, K, bits, group_size, act_dtype, scale_format))


def gemm_describe(M, N, K, bits, group_size):
    buf = ctypes.create_string_buffer(256)
    st = int(load().fq_gemm_describe(M, N, K, bits, group_size, buf, 256))
    if st != FQ_OK:
        raise FqError(st, "fq_gemm_describe")
    return buf.value.decode()


def gemm_grouped_describe(offsets, N, K, bits, group_size):
    buf = ctypes.create_string_buffer(256)
    E = len(offsets) - 1
    arr = _int32_array(offsets)
    st = int(load().fq_gemm_grouped_describe(arr, E, N, K, bits, group_size, buf, 256))
    if st != FQ_OK:
        raise FqError(st, "fq_gemm_grouped_describe")
    return buf.value.decode()


def choose_group_workspace_bytes(K, N, g_start, g_min):
    return int(load().fq_choose_group_workspace_bytes(K, N, g_start, g_min))


def quantize_raw(W_ptr, K, N, bits, group_size, codes_ptr, scales_ptr, stream=0):
    return int(load().fq_quantize(W_ptr, K, N, bits, group_size, codes_ptr, scales_ptr, stream))


def quantize_sf_raw(W_ptr, K, N, bits, group_size, scale_format, codes_ptr, scales_ptr, stream=0):
    return int(load().fq_quantize_sf(W_ptr, K, N, bits, group_size, scale_format, codes_ptr, scales_ptr, stream))


def unpack_raw(codes_ptr, K, N, bits, q_ptr, stream=0):
    return int(load().fq_unpack(codes_ptr, K, N, bits, q_ptr, stream))


def choose_group_raw(W_ptr, K, N, g_start, g_min, alpha, ws_ptr, ws_bytes, stream=0):
    out = ctypes.c_int(-1)
    st = int(load().fq_choose_group(W_ptr, K, N, g_start, g_min, alpha, ctypes.byref(out), ws_ptr, ws_bytes,
                                    stream))
    return st, out.value


def quant_error_workspace_bytes(K, N):
    return int(load().fq_quant_error_workspace_bytes(K, N))


def quant_error_raw(W_ptr, K, N, bits, group_size, codes_ptr, scales_ptr, ws_ptr, ws_bytes, stream=0):
    sse = ctypes.c_double(-1.0)
    mx = ctypes.c_double(-1.0)
    st = int(load().fq_quant_error(W_ptr, K, N, bits, group_size, codes_ptr, scales_ptr, ctypes.byref(sse),
                                   ctypes.byref(mx), ws_ptr, ws_bytes, stream))
    return st, sse.value, mx.value


def quant_error_sf_raw(W_ptr, K, N, bits, group_size, scale_format, codes_ptr, scales_ptr, ws_ptr, ws_bytes,
                       stream=0):
    sse = ctypes.c_double(-1.0)
    mx = ctypes.c_double(-1.0)
    st = int(load().fq_quant_error_sf(W_ptr, K, N, bits, group_size, scale_format, codes_ptr, scales_ptr,
                                      ctypes.byref(sse), ctypes.byref(mx), ws_ptr, ws_bytes, stream))
    return st, sse.value, mx.value


def gemm_raw(A_ptr, act_dtype, M, N, K, codes_ptr, scales_ptr, bits, group_size, C_ptr, ws_ptr, ws_bytes,
             stream=0):
    return int(load().fq_gemm(A_ptr, act_dtype, M, N, K, codes_ptr, scales_ptr, bits, group_size, C_ptr,
                              ws_ptr, ws_bytes, stream))


def gemm_noalloc_raw(A_ptr, act_dtype, M, N, K, codes_ptr, scales_ptr, bits, group_size, C_ptr, stream=0):
    return int(load().fq_gemm_noalloc(A_ptr, act_dtype, M, N, K, codes_ptr, scales_ptr, bits, group_size, C_ptr,
                                      stream))


def gemm_noalloc_scratch_bytes():
    return int(load().fq_gemm_noalloc_scratch_bytes())


def gemm_sf_raw(A_ptr, act_dtype, M, N, K, codes_ptr, scales_ptr, scale_format, bits, group_size, C_ptr, ws_ptr,
                ws_bytes, stream=0):
    return int(load().fq_gemm_sf(A_ptr, act_dtype, M, N, K, codes_ptr, scales_ptr, scale_format, bits, group_size,
                                 C_ptr, ws_ptr, ws_bytes, stream))


def _int32_array(values):
    """The values as a ctypes array."""
    if isinstance(values, (list, tuple)) and values:     # (ints packed at once: a tenth of the time that converting each one takes)
        try:
            packed = array.array("i", values)
            return (ctypes.c_int32 * len(packed)).from_buffer(packed)
        except (TypeError, OverflowError):
            pass
    return (ctypes.c_int32 * len(values))(*[int(v) for v in values])


def gemm_grouped_raw(A_ptr, act_dtype, offsets, N, K, codes_ptr, scales_ptr, bits, group_size, C_ptr,
                     ws_ptr=None, ws_bytes=0, stream=0):
    E = len(offsets) - 1
    arr = _int32_array(offsets)
    return int(load().fq_gemm_grouped(A_ptr, act_dtype, arr, E, N, K, codes_ptr, scales_ptr, bits, group_size,
                                      C_ptr, ws_ptr, ws_bytes, stream))


def gemm_grouped_sf_raw(A_ptr, act_dtype, offsets, N, K, codes_ptr, scales_ptr, scale_format, bits, group_size,
                        C_ptr, ws_ptr=None, ws_bytes=0, stream=0):
    E = len(offsets) - 1
    arr = _int32_array(offsets)
    return int(load().fq_gemm_grouped_sf(A_ptr, act_dtype, arr, E, N, K, codes_ptr, scales_ptr, scale_format, bits,
                                         group_size, C_ptr, ws_ptr, ws_bytes, stream))


def zscale_bytes(K, N, group_size):
    return int(load().fq_zscale_bytes(K, N, group_size))


def quantize_w4a8_raw(W_ptr, K, N, group_size, codes_ptr, z_ptr, t_ptr, stream=0):
    return int(load().fq_quantize_w4a8(W_ptr, K, N, group_size, codes_ptr, z_ptr, t_ptr, stream))


def unpack_w4a8_raw(codes_ptr, K, N, q_ptr, stream=0):
    return int(load().fq_unpack_w4a8(codes_ptr, K, N, q_ptr, stream))


def quantize_act_i8_raw(A_ptr, act_dtype, M, K, Aq_ptr, alpha_ptr, stream=0):
    return int(load().fq_quantize_act_i8(A_ptr, act_dtype, M, K, Aq_ptr, alpha_ptr, stream))


def gemm_w4a8_workspace_bytes(M, N, K, group_size):
    return int(load().fq_gemm_w4a8_workspace_bytes(M, N, K, group_size))


def gemm_w4a8_raw(Aq_ptr, alpha_ptr, M, N, K, codes_ptr, z_ptr, t_ptr, group_size, C_ptr, out_dtype, ws_ptr, ws_bytes,
                  stream=0):
    return int(load().fq_gemm_w4a8(Aq_ptr, alpha_ptr, M, N, K, codes_ptr, z_ptr, t_ptr, group_size, C_ptr, out_dtype,
                                   ws_ptr, ws_bytes, stream))


def qk_norm_rope_raw(qkv_ptr, act_dtype, tokens, row_stride, q_heads, kv_heads, head_dim, q_weight_ptr, k_weight_ptr, eps,
                     table_ptr, table_rows, rot_dim, interleaved, positions_ptr, q_out_ptr, k_out_ptr, cache=None,
                     slots_ptr=None, stream=0):
    return int(load().fq_qk_norm_rope(qkv_ptr, act_dtype, tokens, row_stride, q_heads, kv_heads, head_dim, q_weight_ptr,
                                      k_weight_ptr, eps, table_ptr, table_rows, rot_dim, interleaved, positions_ptr, q_out_ptr,
                                      k_out_ptr, cache, slots_ptr, stream))


def attention_prompt_workspace_bytes(q_heads, kv_heads, head_dim, q_offsets, k_offsets=None):
    return int(load().fq_attention_prompt_workspace_bytes(q_heads, kv_heads, head_dim, _int32_array(q_offsets),
                                                          None if k_offsets is None else _int32_array(k_offsets),
                                                          len(q_offsets) - 1))


def attention_prompt_raw(q, k, v, act_dtype, q_heads, kv_heads, head_dim, q_offsets, k_offsets, scale, out_ptr, ws_ptr=None,
                         ws_bytes=0, stream=0):
    """q, k, v: Heads."""
    return int(load().fq_attention_prompt(q, k, v, act_dtype, q_heads, kv_heads, head_dim, _int32_array(q_offsets),
                                          None if k_offsets is None else _int32_array(k_offsets), len(q_offsets) - 1, scale,
                                          out_ptr, ws_ptr, ws_bytes, stream))


def attention_tree_workspace_bytes(sequences, nodes, q_heads, kv_heads, head_dim, table_width, page_size):
    return int(load().fq_attention_tree_workspace_bytes(sequences, nodes, q_heads, kv_heads, head_dim, table_width, page_size))


def attention_tree_raw(q, act_dtype, sequences, nodes, q_heads, kv_heads, head_dim, cache, page_table_ptr, table_width,
                       context_lens_ptr, mask_ptr, mask_stride, scale, out_ptr, ws_ptr=None, ws_bytes=0, stream=0):
    """q: Heads; cache: KvPages."""
    return int(load().fq_attention_tree(q, act_dtype, sequences, nodes, q_heads, kv_heads, head_dim, cache, page_table_ptr,
                                        table_width, context_lens_ptr, mask_ptr, mask_stride, scale, out_ptr, ws_ptr, ws_bytes,
                                        stream))


# ------------------------------------------------------------------ torch-tensor conveniences
# (What a call spends here counts on small products: asking torch for its current stream as an object took 2.9 us of the
# 9.1 us of a fq.gemm of one launch; the stream's address alone, and functions looked up once, leave 5.8, and the native calls
# below 3.5.)
def _torch():
    """torch, and the function that gives a device's current stream as an address, looked up on the first call."""
    global _torch_mod, _raw_stream, _device, _native
    import torch

    load()
    _native = _load_native()

    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if _raw_stream is None:
        _raw_stream = lambda device: torch.cuda.current_stream(device).cuda_stream  # noqa: E731
    _device = torch.cuda.current_device
    _torch_mod = torch
    return torch


_torch_mod = _raw_stream = _device = None

# The calls that a program makes over and over, in native code (csrc/fq_binding.cpp).  A function of it returns None where a
# call is out of the ordinary; the Python below it then reports the error, or does without.  (Errors of the HIP runtime, which
# may come after launches, it raises itself.)
NATIVE_PATH = os.path.join(_HERE, "_fqcall.so")
_NATIVE_FUNCTIONS = ("fq_gemm_sf", "fq_gemm_workspace_bytes", "fq_gemm_grouped_sf", "fq_gemm_w4a8", "fq_gemm_w4a8_workspace_bytes",
                     "fq_quantize_act_i8", "fq_quantize_sf", "fq_quantize_w4a8", "fq_codes_bytes", "fq_scales_bytes", "fq_zscale_bytes",
                     "fq_qk_norm_rope", "fq_attention_prompt", "fq_attention_prompt_workspace_bytes", "fq_attention_tree",
                     "fq_attention_tree_workspace_bytes")
_native = None


class _NoNative:
    """In place of the native calls where they are not built or do not fit this torch: every call goes the Python way."""

    def __getattr__(self, name):
        return lambda *args: None


def _load_native():
    """The native calls, bound to the library that load() has loaded."""
    try:
        spec = importlib.util.spec_from_file_location("_fqcall", NATIVE_PATH)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        lib = load()
        module.bind(FqError, *(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _NATIVE_FUNCTIONS))
    except (ImportError, OSError, TypeError) as e:      # not there, another torch's or Python's, another build's
        warnings.warn(f"calls are issued from Python, which takes about twice as long: {e}", RuntimeWarning, stacklevel=2)
        return _NoNative()
    return module


def _stream():
    """Address of the current device's current stream."""
    if _torch_mod is None:
        _torch()
    return _raw_stream(_device())


def _check(status, where):
    if status != FQ_OK:
        raise FqError(status, where)


def _act_code(t):
    torch = _torch_mod or _torch()
    if t.dtype == torch.float16:
        return FQ_F16
    if t.dtype == torch.bfloat16:
        return FQ_BF16
    raise TypeError("activations must be float16 or bfloat16")


def _scale_format_of(scales):
    """The fq_scale_format a scale tensor's dtype stands for."""
    torch = _torch_mod or _torch()
    if scales.dtype == torch.float16:
        return FQ_SCALE_F16
    if scales.dtype == torch.bfloat16:
        return FQ_SCALE_BF16
    raise TypeError("scales must be float16 or bfloat16")


def quantize(W, bits, group_size, scale_format=FQ_SCALE_F16):
    """W: cuda float16 [K, N] -> (codes uint8 [K*N*bits/8], scales [K/g, N] float16, or bfloat16 for
    scale_format=FQ_SCALE_BF16)."""
    torch = _torch_mod or _torch()
    done = _native.quantize(W, bits, group_size, scale_format)
    if done is not None:
        return done
    assert W.is_cuda and W.dtype == torch.float16 and W.is_contiguous()
    K, N = W.shape
    g = K if group_size in (0, K) else group_size
    nbytes = codes_bytes(K, N, bits)
    sbytes = scales_bytes(K, N, group_size)
    if nbytes == 0 or sbytes == 0:
        raise FqError(FQ_ERR_INVALID_ARG, "fq_quantize")
    codes = torch.empty(nbytes, dtype=torch.uint8, device=W.device)
    sdtype = torch.bfloat16 if scale_format == FQ_SCALE_BF16 else torch.float16
    scales = torch.empty((K // g, N), dtype=sdtype, device=W.device)
    _check(quantize_sf_raw(W.data_ptr(), K, N, bits, group_size, scale_format, codes.data_ptr(), scales.data_ptr(),
                           _stream()), "fq_quantize_sf")
    return codes, scales


def unpack(codes, K, N, bits):
    torch = _torch_mod or _torch()
    q = torch.empty((K, N), dtype=torch.int8, device=codes.device)
    _check(unpack_raw(codes.data_ptr(), K, N, bits, q.data_ptr(), _stream()), "fq_unpack")
    return q


def choose_group(W, g_start, g_min, alpha):
    torch = _torch_mod or _torch()
    K, N = W.shape
    ws_bytes = choose_group_workspace_bytes(K, N, g_start, g_min)
    ws = torch.empty(max(ws_bytes, 16), dtype=torch.uint8, device=W.device)
    st, g = choose_group_raw(W.data_ptr(), K, N, g_start, g_min, float(alpha), ws.data_ptr(), ws_bytes, _stream())
    _check(st, "fq_choose_group")
    return g


def quant_error(W, codes, scales, bits, group_size):
    """Round-trip error of a quantised matrix: (sum of squared errors, largest absolute error)."""
    torch = _torch_mod or _torch()
    assert W.is_cuda and W.dtype == torch.float16 and W.is_contiguous()
    K, N = W.shape
    ws_bytes = quant_error_workspace_bytes(K, N)
    ws = torch.empty(max(ws_bytes, 16), dtype=torch.uint8, device=W.device)
    st, sse, mx = quant_error_sf_raw(W.data_ptr(), K, N, bits, group_size, _scale_format_of(scales),
                                     codes.data_ptr(), scales.data_ptr(), ws.data_ptr(), ws_bytes, _stream())
    _check(st, "fq_quant_error_sf")
    return sse, mx


def gemm(A, codes, scales, bits, group_size, out=None, workspace=None):
    """A: cuda [M, K] float16/bfloat16 -> C [M, N] of the same dtype."""
    torch = _torch_mod or _torch()
    done = _native.gemm(A, codes, scales, bits, group_size, out, workspace)
    if done is not None:
        return done
    assert A.is_cuda and A.is_contiguous()
    M, K = A.shape
    N = scales.shape[1]
    C = out if out is not None else torch.empty((M, N), dtype=A.dtype, device=A.device)
    size = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if workspace is None:
        size = gemm_workspace_bytes(M, N, K, bits, group_size)
        workspace = torch.empty(size, dtype=torch.uint8, device=A.device) if size else None

    args = (A.data_ptr(), _act_code(A), M, N, K, codes.data_ptr(), scales.data_ptr(), _scale_format_of(scales), bits,
            group_size, C.data_ptr())
    status = gemm_sf_raw(*args, workspace.data_ptr() if workspace is not None else None, size, _stream())
    if status == FQ_ERR_WORKSPACE:      # the caller's is too small (asked only now: the query plans the product once more)
        size = gemm_workspace_bytes(M, N, K, bits, group_size)
        workspace = torch.empty(size, dtype=torch.uint8, device=A.device)
        status = gemm_sf_raw(*args, workspace.data_ptr(), size, _stream())
    _check(status, "fq_gemm_sf")
    return C


def gemm_grouped(A, offsets, codes, scales, bits, group_size, N, out=None):
    """A: cuda [rows, K]; codes / scales: the experts' buffers back to back."""
    torch = _torch_mod or _torch()
    done = _native.gemm_grouped(A, offsets, codes, scales, bits, group_size, N, out)
    if done is not None:
        return done
    rows, K = A.shape
    C = out if out is not None else torch.empty((rows, N), dtype=A.dtype, device=A.device)
    _check(gemm_grouped_sf_raw(A.data_ptr(), _act_code(A), offsets, N, K, codes.data_ptr(), scales.data_ptr(),
                               _scale_format_of(scales), bits, group_size, C.data_ptr(), None, 0, _stream()),
           "fq_gemm_grouped_sf")
    return C


def quantize_w4a8(W, group_size):
    """W: cuda float16 [K, N] -> (codes uint8 [K*N/2], z uint8 [K/g, N], t float16 [N]) of the integer path."""
    torch = _torch_mod or _torch()
    done = _native.quantize_w4a8(W, group_size)
    if done is not None:
        return done
    assert W.is_cuda and W.dtype == torch.float16 and W.is_contiguous()
    K, N = W.shape
    g = K if group_size in (0, K) else group_size
    zb = zscale_bytes(K, N, group_size)
    if zb == 0:
        raise FqError(FQ_ERR_UNSUPPORTED, "fq_quantize_w4a8")
    codes = torch.empty(codes_bytes(K, N, 4), dtype=torch.uint8, device=W.device)
    z = torch.empty((K // g, N), dtype=torch.uint8, device=W.device)
    t = torch.empty((N,), dtype=torch.float16, device=W.device)
    _check(quantize_w4a8_raw(W.data_ptr(), K, N, group_size, codes.data_ptr(), z.data_ptr(), t.data_ptr(), _stream()),
           "fq_quantize_w4a8")
    return codes, z, t


def unpack_w4a8(codes, K, N):
    torch = _torch_mod or _torch()
    q = torch.empty((K, N), dtype=torch.int8, device=codes.device)
    _check(unpack_w4a8_raw(codes.data_ptr(), K, N, q.data_ptr(), _stream()), "fq_unpack_w4a8")
    return q


def quantize_act_i8(A):
    """A: cuda [M, K] float16/bfloat16 -> (Aq int8 [M, K], alpha float32 [M])."""
    torch = _torch_mod or _torch()
    done = _native.quantize_act_i8(A)
    if done is not None:
        return done
    assert A.is_cuda and A.is_contiguous()
    M, K = A.shape
    Aq = torch.empty((M, K), dtype=torch.int8, device=A.device)
    alpha = torch.empty((M,), dtype=torch.float32, device=A.device)
    _check(quantize_act_i8_raw(A.data_ptr(), _act_code(A), M, K, Aq.data_ptr(), alpha.data_ptr(), _stream()),
           "fq_quantize_act_i8")
    return Aq, alpha


def gemm_w4a8(Aq, alpha, codes, z, t, group_size, out_dtype, out=None, workspace=None):
    """C [M, N] (torch dtype out_dtype: float16 or bfloat16) = alpha * t * (Aq . (q * z))."""
    torch = _torch_mod or _torch()
    done = _native.gemm_w4a8(Aq, alpha, codes, z, t, group_size, out_dtype, out, workspace)
    if done is not None:
        return done
    M, K = Aq.shape
    N = t.shape[0]
    C = out if out is not None else torch.empty((M, N), dtype=out_dtype, device=Aq.device)
    size = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if workspace is None:
        size = gemm_w4a8_workspace_bytes(M, N, K, group_size)
        workspace = torch.empty(size, dtype=torch.uint8, device=Aq.device) if size else None
    args = (Aq.data_ptr(), alpha.data_ptr(), M, N, K, codes.data_ptr(), z.data_ptr(), t.data_ptr(), group_size, C.data_ptr(),
            FQ_F16 if out_dtype == torch.float16 else FQ_BF16)
    status = gemm_w4a8_raw(*args, workspace.data_ptr() if workspace is not None else None, size, _stream())
    if status == FQ_ERR_WORKSPACE:      # the caller's is too small
        size = gemm_w4a8_workspace_bytes(M, N, K, group_size)
        workspace = torch.empty(size, dtype=torch.uint8, device=Aq.device)
        status = gemm_w4a8_raw(*args, workspace.data_ptr(), size, _stream())
    _check(status, "fq_gemm_w4a8")
    return C


# ------------------------------------------------------------------ attention
def _require(condition, where):
    if not condition:
        raise FqError(FQ_ERR_INVALID_ARG, where)


def _plain(t, dtype, device, where):
    """Whether t is a contiguous tensor of this type on this device."""
    _require(t.dtype == dtype and t.device == device and t.is_contiguous(), where)


def rope_table(rows, rot_dim, base=10000.0, device="cuda"):
    """The table of qk_norm_rope for positions 0 .. rows - 1: cosines, then sines, of position * base^(-2 i / rot_dim);
    float32 [rows, rot_dim]."""
    torch = _torch_mod or _torch()
    turns = base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64) / rot_dim)
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * turns
    return torch.cat([angle.cos(), angle.sin()], 1).float().to(device)


def tree_mask(parents, device="cuda"):
    """Masks of attention_tree for drafted trees: parents[i] < i is the node that node i hangs from, -1 for the context itself (one
    list, or one of the same length per sequence) -> int64 [nodes, words] or [sequences, nodes, words]: each node's ancestors and itself."""
    torch = _torch_mod or _torch()

    def words(tree):
        seen = []
        for i, p in enumerate(tree):
            if not -1 <= p < i:
                raise ValueError(f"node {i} hangs from {p}: -1 or a node before it")
            seen.append((seen[p] if p >= 0 else 0) | 1 << i)
        rows = [[s >> 64 * w & (1 << 64) - 1 for w in range((len(tree) + 63) // 64)] for s in seen]
        return [[x - (1 << 64) if x >> 63 else x for x in row] for row in rows]

    several = len(parents) > 0 and not isinstance(parents[0], int)
    return torch.tensor([words(t) for t in parents] if several else words(parents), dtype=torch.int64, device=device)


def _heads(t, where):
    """Heads of a tensor [rows, heads, head_dim]."""
    _require(t.is_cuda and t.dim() == 3 and (t.stride(2) == 1 or t.shape[2] <= 1), where)
    return Heads(t.data_ptr(), t.stride(0), t.stride(1))


def _pages(k_cache, v_cache, like, kv_heads, head_dim, where):
    """KvPages of two tensors [pages, page_size, kv_heads, head_dim] with the same strides."""
    for c in (k_cache, v_cache):
        _require(c.dim() == 4 and c.dtype == like.dtype and c.device == like.device and c.stride(3) == 1, where)
        _require(c.shape[2] == kv_heads and c.shape[3] == head_dim, where)
    _require(k_cache.shape == v_cache.shape and k_cache.stride() == v_cache.stride(), where)
    return KvPages(k_cache.data_ptr(), v_cache.data_ptr(), k_cache.shape[0], k_cache.shape[1], *k_cache.stride()[:3])


def _output(out, shape, like, where):
    torch = _torch_mod or _torch()
    if out is None:
        return torch.empty(shape, dtype=like.dtype, device=like.device)
    _require(tuple(out.shape) == tuple(shape), where)
    _plain(out, like.dtype, like.device, where)
    return out


def _offsets(offsets, rows, where):
    """Offsets that end at `rows`, as a list of integers of which none is another in 32 bits."""
    offsets = [int(x) for x in offsets]
    _require(len(offsets) >= 1 and offsets[-1] == rows and min(offsets) >= 0 and max(offsets) <= rows, where)
    return offsets


def _scratch(workspace, need, like, where):
    """A caller's workspace (contiguous, on like's device) where it is large enough, or a new one of `need` bytes; and its size."""
    torch = _torch_mod or _torch()
    size = 0
    if workspace is not None:
        _require(workspace.device == like.device and workspace.is_contiguous(), where)
        size = workspace.numel() * workspace.element_size()
    if size < need:
        workspace, size = torch.empty(need, dtype=torch.uint8, device=like.device), need
    return workspace, size


def _given_scale(scale, where):
    """A scale that was given, as binary32; 0 for the library's own."""
    if scale is None:
        return 0.0
    scale = ctypes.c_float(scale).value
    _require(scale > 0.0, where)
    return scale


def qk_norm_rope(qkv, heads, kv_heads, table, positions, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, q_out=None,
                 k_out=None, k_cache=None, v_cache=None, slots=None):
    """qkv: cuda [tokens, (heads + 2 kv_heads) * head_dim] float16/bfloat16, rows of any stride -> (q [tokens, heads, head_dim],
    k [tokens, kv_heads, head_dim]), normalised (with q_weight, k_weight [head_dim]) and rotated by positions (int32 [tokens]) with
    table (rope_table; None: not rotated).  With k_cache, v_cache [pages, page_size, kv_heads, head_dim] and slots (int64 [tokens])
    keys and values go to the cache, and k is None unless k_out is given."""
    torch = _torch_mod or _torch()
    done = _native.qk_norm_rope(qkv, heads, kv_heads, table, positions, q_weight, k_weight, eps, interleaved, q_out, k_out, k_cache,
                                v_cache, slots)
    if done is not None:
        return done
    where = "fq_qk_norm_rope"
    _require(qkv.is_cuda and qkv.dim() == 2 and heads > 0 and kv_heads > 0 and qkv.shape[1] % (heads + 2 * kv_heads) == 0, where)
    _require(qkv.stride(1) == 1, where)
    tokens, D = qkv.shape[0], qkv.shape[1] // (heads + 2 * kv_heads)
    act = _act_code(qkv)
    for w in (q_weight, k_weight):
        if w is not None:
            _require(w.numel() == D, where)
            _plain(w, qkv.dtype, qkv.device, where)
    rot = 0
    if table is not None:
        _require(table.dim() == 2 and positions is not None and positions.numel() == tokens, where)
        _plain(table, torch.float32, qkv.device, where)
        _plain(positions, torch.int32, qkv.device, where)
        rot = table.shape[1]
    cache = None
    _require((k_cache is None) == (v_cache is None) == (slots is None), where)
    if k_cache is not None:
        cache = _pages(k_cache, v_cache, qkv, kv_heads, D, where)
        _require(slots.numel() == tokens, where)
        _plain(slots, torch.int64, qkv.device, where)
    q = _output(q_out, (tokens, heads, D), qkv, where)
    k = _output(k_out, (tokens, kv_heads, D), qkv, where) if k_out is not None or cache is None else None

    def at(t):
        return None if t is None else t.data_ptr()

    _check(qk_norm_rope_raw(qkv.data_ptr(), act, tokens, qkv.stride(0), heads, kv_heads, D, at(q_weight), at(k_weight), eps,
                            at(table) if rot else None, table.shape[0] if rot else 0, rot, int(interleaved),
                            at(positions) if rot else None, q.data_ptr(), at(k), cache, at(slots), _stream()), where)
    return q, k


def attention_prompt(q, k, v, q_offsets, k_offsets=None, scale=None, out=None, workspace=None):
    """Causal attention over packed sequences: q cuda [rows, heads, head_dim], k and v [keys, kv_heads, head_dim] (float16 or bfloat16,
    any row and head strides), sequence b's rows q_offsets[b] .. q_offsets[b + 1] - 1 (host integers) and keys k_offsets[b] .. (None: the
    same) -> [rows, heads, head_dim].  scale: 1 / sqrt(head_dim) unless given.  workspace: scratch on the same device, contiguous
    (attention_prompt_workspace_bytes; a smaller one is as none, for which some is allocated)."""
    torch = _torch_mod or _torch()
    done = _native.attention_prompt(q, k, v, q_offsets, k_offsets, scale, out, workspace)
    if done is not None:
        return done
    where = "fq_attention_prompt"
    act = _act_code(q)
    hq, hk, hv = _heads(q, where), _heads(k, where), _heads(v, where)
    (rows, heads, D), (keys, kv_heads, _) = q.shape, k.shape
    for t in (k, v):
        _require(tuple(t.shape) == (keys, kv_heads, D) and t.dtype == q.dtype and t.device == q.device, where)
    q_offsets = _offsets(q_offsets, rows, where)
    k_offsets = None if k_offsets is None else _offsets(k_offsets, keys, where)
    _require(len(k_offsets) == len(q_offsets) if k_offsets is not None else keys == rows, where)
    scale = _given_scale(scale, where)
    o = _output(out, (rows, heads, D), q, where)
    workspace, size = _scratch(workspace, attention_prompt_workspace_bytes(heads, kv_heads, D, q_offsets, k_offsets), q, where)
    _check(attention_prompt_raw(hq, hk, hv, act, heads, kv_heads, D, q_offsets, k_offsets, scale, o.data_ptr(),
                                workspace.data_ptr() if size else None, size, _stream()), where)
    return o


def attention_tree(q, k_cache, v_cache, page_table, context_lens, mask=None, scale=None, out=None, workspace=None):
    """Attention of drafted tokens over a paged cache: q cuda [sequences, nodes, heads, head_dim] (float16 or bfloat16; the tokens of all
    sequences evenly apart), caches [pages, page_size, kv_heads, head_dim], page_table int32 [sequences, width], context_lens int32 [sequences]
    (tokens in the cache before the drafted ones, whose keys and values lie in the places behind them), mask int64 [nodes, words] or
    [sequences, nodes, words] (tree_mask; None: a chain) -> [sequences, nodes, heads, head_dim].  scale: 1 / sqrt(head_dim) unless given.
    workspace: as attention_prompt's (attention_tree_workspace_bytes)."""
    torch = _torch_mod or _torch()
    done = _native.attention_tree(q, k_cache, v_cache, page_table, context_lens, mask, scale, out, workspace)
    if done is not None:
        return done
    where = "fq_attention_tree"
    act = _act_code(q)
    _require(q.is_cuda and q.dim() == 4 and (q.stride(3) == 1 or q.shape[3] <= 1), where)
    sequences, nodes, heads, D = q.shape
    row = 0 if sequences * nodes <= 1 else q.stride(0) if nodes == 1 else q.stride(1)      # (of one token, or one sequence, the stride says nothing)
    _require(q.stride(0) == nodes * row or sequences <= 1, where)
    kv_heads = k_cache.shape[2] if k_cache.dim() == 4 else 0
    cache = _pages(k_cache, v_cache, q, kv_heads, D, where)
    _require(page_table.dim() == 2 and page_table.shape[0] == sequences and context_lens.numel() == sequences, where)
    _plain(page_table, torch.int32, q.device, where)
    _plain(context_lens, torch.int32, q.device, where)
    stride = 0
    if mask is not None:
        words = (nodes + 63) // 64
        _plain(mask, torch.int64, q.device, where)
        _require(tuple(mask.shape) in ((nodes, words), (sequences, nodes, words)), where)
        stride = nodes * words if mask.dim() == 3 else 0
    scale = _given_scale(scale, where)
    o = _output(out, (sequences, nodes, heads, D), q, where)
    width, page = page_table.shape[1], k_cache.shape[1]
    workspace, size = _scratch(workspace, attention_tree_workspace_bytes(sequences, nodes, heads, kv_heads, D, width, page), q, where)
    _check(attention_tree_raw(Heads(q.data_ptr(), row, q.stride(2)), act, sequences, nodes, heads, kv_heads, D, cache,
                              page_table.data_ptr(), width, context_lens.data_ptr(), None if mask is None else mask.data_ptr(), stride,
                              scale, o.data_ptr(), workspace.data_ptr() if size else None, size, _stream()), where)
    return o
