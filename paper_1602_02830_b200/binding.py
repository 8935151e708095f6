"""ctypes binding of libbnn_b200.so: same names as the C ABI, argument marshalling only.

Tensors are torch tensors that own device (or, where the C call says so, host) memory; this module
passes their data pointers, leading dimensions and sizes and raises on a non-zero status.  No step of
the method is computed here.  The library is loaded on first use; if it has not been built the call
fails with an error -- there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, Structure, c_double, c_float, c_int, c_int32, c_int64, c_size_t, c_uint64, c_void_p

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbnn_b200.so")

BNN_F32, BNN_F16, BNN_I8, BNN_BF16 = 0, 1, 2, 3
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4, "sigmoid": 5, "htanh": 6}
NORMS = {"rms": 0, "layer": 1}
MX_FORMATS = {"e4m3": 0, "e2m1": 1}
_REAL_TYPES = {torch.float32: BNN_F32, torch.float16: BNN_F16, torch.bfloat16: BNN_BF16}
_PRODUCT_TYPES = (torch.float16, torch.bfloat16)
VARIANT_AUTO, VARIANT_PLAIN, VARIANT_CSA = 0, 1, 2
ENGINE_AUTO, ENGINE_POPC, ENGINE_TENSOR = 0, 1, 2

EXPORTS = (
    "bnn_create", "bnn_destroy", "bnn_status_string", "bnn_last_cuda_error", "bnn_set_workspace",
    "bnn_set_popc_variant", "bnn_pack_signs", "bnn_xnor_gemm", "bnn_binary_dense", "bnn_first_layer_bitplanes",
    "bnn_binary_conv2d", "bnn_mlp_workspace_bytes", "bnn_mlp_forward", "bnn_mlp_forward_host",
    "bnn_fold_batchnorm", "bnn_mlp_noalloc_max_bytes", "bnn_mlp_forward_noalloc", "bnn_set_engine",
    "bnn_gemm_workspace_bytes", "bnn_device_status", "bnn_conv_workspace_bytes", "bnn_set_tile_rows", "bnn_set_pair_mode", "bnn_expanded_ld",
    "bnn_expanded_bytes", "bnn_expand_signs", "bnn_baseline_gemm_f32", "bnn_convnet_workspace_bytes",
    "bnn_convnet_forward", "bnn_set_operand_bits", "bnn_expanded_ld_f4",
    "bnn_expanded_bytes_f4", "bnn_expand_signs_f4", "bnn_binary_dense_expanded", "bnn_set_wait_limit_ns",
    "bnn_debug_drop_loads", "bnn_debug_ring_position", "bnn_set_conv_form", "bnn_measure_pipe_rates", "bnn_last_tensor_kernel", "bnn_last_tensor_kernel_clock", "bnn_set_conv_filter_repetition",
    "bnn_filter_repetition_workspace_bytes", "bnn_filter_repetition_count",
    "bnn_linear_workspace_bytes", "bnn_linear", "bnn_linear_backward", "bnn_gated_workspace_bytes", "bnn_gated",
    "bnn_gated_backward", "bnn_block_norm", "bnn_block_norm_workspace_bytes", "bnn_block_norm_backward", "bnn_dropout",
    "bnn_mx_ld", "bnn_mx_scale_bytes", "bnn_mx_quantize", "bnn_mx_values", "bnn_block_norm_mx", "bnn_mx_linear", "bnn_mx_gated",
    "bnn_clip_workspace_bytes", "bnn_clip_gradients",
)


class LayerDesc(Structure):
    _fields_ = [("Wp", c_void_p), ("ldw_w", c_int64), ("K", c_int64), ("N", c_int64), ("thr", c_void_p),
                ("flip", c_void_p), ("gamma", c_void_p), ("beta", c_void_p), ("mean", c_void_p), ("var", c_void_p),
                ("eps", c_double), ("W8", c_void_p), ("W4", c_void_p)]


class MlpDesc(Structure):
    _fields_ = [("n_layers", c_int32), ("layers", POINTER(LayerDesc))]


class ConvLayerDesc(Structure):
    _fields_ = [("Wp", c_void_p), ("C_in", c_int64), ("C_out", c_int64), ("pool", c_int32), ("thr", c_void_p),
                ("flip", c_void_p), ("W8", c_void_p), ("W4", c_void_p)]


class ConvNetDesc(Structure):
    _fields_ = [("n_layers", c_int32), ("layers", POINTER(ConvLayerDesc))]


class LinearDesc(Structure):
    _fields_ = [("dtype", c_int32), ("act", c_int32), ("K", c_int64), ("N", c_int64), ("W", c_void_p), ("ldw", c_int64),
                ("bias", c_void_p)]


class GatedDesc(Structure):
    _fields_ = [("dtype", c_int32), ("act", c_int32), ("K", c_int64), ("N", c_int64), ("Wg", c_void_p), ("ldg", c_int64),
                ("Wu", c_void_p), ("ldu", c_int64)]


class BlockNormDesc(Structure):
    _fields_ = [("dtype", c_int32), ("kind", c_int32), ("D", c_int64), ("eps", c_float), ("alpha", c_float), ("post", c_int32),
                ("pre", c_int32), ("post_weight", c_void_p), ("post_shift", c_void_p), ("pre_weight", c_void_p),
                ("pre_shift", c_void_p), ("gate", c_void_p), ("ld_gate", c_int64), ("rows_per_gate", c_int64)]


class BlockNormGrads(Structure):
    _fields_ = [("dx", c_void_p), ("lddx", c_int64), ("dblock", c_void_p), ("lddb", c_int64), ("dpost_weight", c_void_p),
                ("dpost_shift", c_void_p), ("dpre_weight", c_void_p), ("dpre_shift", c_void_p), ("dgate", c_void_p),
                ("ld_dgate", c_int64)]


class MxDesc(Structure):
    _fields_ = [("format", c_int32), ("rows", c_int64), ("cols", c_int64), ("values", c_void_p), ("scales", c_void_p)]


class MxLinearDesc(Structure):
    _fields_ = [("dtype", c_int32), ("act", c_int32), ("W", MxDesc), ("bias", c_void_p)]


class MxGatedDesc(Structure):
    _fields_ = [("dtype", c_int32), ("act", c_int32), ("Wg", MxDesc), ("Wu", MxDesc)]


class Gradient(Structure):
    _fields_ = [("g", c_void_p), ("out", c_void_p), ("n", c_int64), ("dtype", c_int32)]


class MxMatrix:
    """A microscaled matrix (made by Context.make_mx): rows x cols elements of `format` ("e4m3" or "e2m1") with a power of two for each 32
    neighbours of a row.  values [rows, pitch] and scales are bytes in the library's layout (bnn_mx_matrix); Context.mx_values reads them back."""

    def __init__(self, format, rows, cols, values, scales, device):
        self.format, self.rows, self.cols, self.values, self.scales, self.device = format, rows, cols, values, scales, device
        self.desc = MxDesc(MX_FORMATS[format], rows, cols, values.data_ptr(), scales.data_ptr())
        self.ref = ctypes.byref(self.desc)

    @property
    def shape(self):
        return self.rows, self.cols


class Gradients:
    """The tensors whose norm is taken together (made by Context.make_gradients), and where their clipped values go."""

    def __init__(self, tensors, out, device):
        self.tensors, self.out, self.device = tensors, out, device
        self.list = (Gradient * max(1, len(tensors)))(*[Gradient(g.data_ptr(), o.data_ptr(), g.numel(), _REAL_TYPES[g.dtype]) for g, o in zip(tensors, out)])


class Layer:
    """A descriptor of the real-valued operators with the tensors it points to (made by Context.make_linear, make_gated and
    make_block_norm).  The tensors' contents may change between calls, their storage may not."""

    def __init__(self, desc, dtype, device, inner, outer, tensors):
        self.desc, self.ref = desc, ctypes.byref(desc)
        self.dtype, self.device, self.inner, self.outer, self.tensors = dtype, device, inner, outer, tensors


class BnnError(RuntimeError):
    def __init__(self, status: int, what: str, cuda_error: int = 0):
        self.status = status
        self.cuda_error = cuda_error
        msg = f"{what} failed: {status} ({_status_string(status)})"
        if cuda_error:
            msg += f", cudaError {cuda_error}"
        super().__init__(msg)


_lib = None
_raw_stream = torch._C._cuda_getCurrentRawStream if torch.cuda._is_compiled() else None
_empty_strided = torch.empty_strided


def lib() -> ctypes.CDLL:
    """The loaded C library.  Raises if it has not been built (python -m paper_1602_02830_b200.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_1602_02830_b200.build` "
                               "(there is no CPU or PyTorch fallback)")
        L = ctypes.CDLL(LIB_PATH)
        i64, vp = c_int64, c_void_p
        L.bnn_create.argtypes = [POINTER(vp), c_int, vp]
        L.bnn_destroy.argtypes = [vp]
        L.bnn_status_string.argtypes = [c_int]
        L.bnn_status_string.restype = ctypes.c_char_p
        L.bnn_last_cuda_error.argtypes = [vp]
        L.bnn_set_workspace.argtypes = [vp, vp, c_size_t]
        L.bnn_set_popc_variant.argtypes = [vp, c_int]
        L.bnn_set_engine.argtypes = [vp, c_int]
        L.bnn_set_tile_rows.argtypes = [vp, c_int]
        L.bnn_set_pair_mode.argtypes = [vp, c_int]
        L.bnn_set_operand_bits.argtypes = [vp, c_int]
        L.bnn_set_wait_limit_ns.argtypes = [vp, ctypes.c_uint64]
        L.bnn_debug_drop_loads.argtypes = [vp, c_int]
        L.bnn_debug_ring_position.argtypes = [ctypes.c_uint32] * 3 + [vp] * 8
        L.bnn_debug_ring_position.restype = c_int
        L.bnn_set_conv_form.argtypes = [vp, c_int]
        L.bnn_measure_pipe_rates.argtypes = [vp, vp, c_size_t, POINTER(c_double), POINTER(c_double), POINTER(c_double)]
        L.bnn_last_tensor_kernel.argtypes = [vp]
        L.bnn_last_tensor_kernel.restype = ctypes.c_char_p
        L.bnn_last_tensor_kernel_clock.argtypes = [vp, POINTER(c_double), POINTER(c_double)]
        L.bnn_set_conv_filter_repetition.argtypes = [vp, c_int]
        L.bnn_filter_repetition_workspace_bytes.argtypes = [i64, i64]
        L.bnn_filter_repetition_workspace_bytes.restype = c_size_t
        L.bnn_filter_repetition_count.argtypes = [vp, vp, i64, i64, POINTER(c_int64)]
        L.bnn_expanded_ld_f4.argtypes = [i64]
        L.bnn_expanded_ld_f4.restype = i64
        L.bnn_expanded_bytes_f4.argtypes = [i64, i64]
        L.bnn_expanded_bytes_f4.restype = c_size_t
        L.bnn_expand_signs_f4.argtypes = [vp, vp, i64, i64, i64, vp]
        L.bnn_binary_dense_expanded.argtypes = [vp, vp, i64, vp, i64, ctypes.c_int, vp, vp, vp, i64, vp, i64, i64, i64, i64]
        L.bnn_expanded_ld.argtypes = [i64]
        L.bnn_expanded_ld.restype = i64
        L.bnn_expanded_bytes.argtypes = [i64, i64]
        L.bnn_expanded_bytes.restype = c_size_t
        L.bnn_expand_signs.argtypes = [vp, vp, i64, i64, i64, vp]
        L.bnn_baseline_gemm_f32.argtypes = [vp, vp, vp, vp, i64, i64, i64]
        L.bnn_convnet_workspace_bytes.argtypes = [POINTER(ConvNetDesc), i64, i64, i64]
        L.bnn_convnet_workspace_bytes.restype = c_size_t
        L.bnn_convnet_forward.argtypes = [vp, POINTER(ConvNetDesc), vp, i64, i64, i64, vp, POINTER(vp)]
        L.bnn_gemm_workspace_bytes.argtypes = [i64, i64, i64]
        L.bnn_gemm_workspace_bytes.restype = c_size_t
        L.bnn_device_status.argtypes = [vp]
        L.bnn_conv_workspace_bytes.argtypes = [i64, i64, i64, i64, i64, c_int]
        L.bnn_conv_workspace_bytes.restype = c_size_t
        L.bnn_pack_signs.argtypes = [vp, vp, c_int, i64, i64, i64, c_int, c_int, vp, i64]
        L.bnn_xnor_gemm.argtypes = [vp, vp, i64, vp, i64, vp, i64, i64, i64, i64]
        L.bnn_binary_dense.argtypes = [vp, vp, i64, vp, i64, vp, vp, vp, i64, i64, i64, i64]
        L.bnn_first_layer_bitplanes.argtypes = [vp, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, i64, i64, i64]
        L.bnn_binary_conv2d.argtypes = [vp, vp, vp, i64, i64, i64, i64, vp, i64, c_int, vp, vp, vp, vp]
        L.bnn_mlp_workspace_bytes.argtypes = [POINTER(MlpDesc), i64, c_int]
        L.bnn_mlp_workspace_bytes.restype = c_size_t
        L.bnn_mlp_forward.argtypes = [vp, POINTER(MlpDesc), vp, i64, i64, vp, i64, POINTER(vp)]
        L.bnn_mlp_forward_host.argtypes = [vp, POINTER(MlpDesc), vp, i64, i64, vp, i64]
        L.bnn_fold_batchnorm.argtypes = [vp, vp, vp, vp, c_double, i64, i64, vp, vp]
        L.bnn_linear_workspace_bytes.argtypes = [POINTER(LinearDesc), i64, c_int, c_int]
        L.bnn_linear_workspace_bytes.restype = c_size_t
        L.bnn_linear.argtypes = [vp, POINTER(LinearDesc), vp, i64, i64, vp, i64, vp, i64, vp, i64]
        L.bnn_linear_backward.argtypes = [vp, POINTER(LinearDesc), vp, i64, vp, i64, i64, vp, i64, vp, i64, vp, i64, vp]
        L.bnn_gated_workspace_bytes.argtypes = [POINTER(GatedDesc), i64, c_int, c_int]
        L.bnn_gated_workspace_bytes.restype = c_size_t
        L.bnn_gated.argtypes = [vp, POINTER(GatedDesc), vp, i64, i64, vp, i64, vp, i64]
        L.bnn_gated_backward.argtypes = [vp, POINTER(GatedDesc), vp, i64, vp, i64, i64, vp, i64, vp, i64, vp, i64, vp, i64]
        L.bnn_block_norm.argtypes = [vp, POINTER(BlockNormDesc), vp, i64, vp, i64, i64, vp, i64, vp, i64, vp]
        L.bnn_block_norm_workspace_bytes.argtypes = [POINTER(BlockNormDesc), i64]
        L.bnn_block_norm_workspace_bytes.restype = c_size_t
        L.bnn_block_norm_backward.argtypes = [vp, POINTER(BlockNormDesc), vp, i64, vp, i64, vp, i64, vp, i64, vp, i64,
                                              POINTER(BlockNormGrads)]
        L.bnn_dropout.argtypes = [vp, c_int, vp, i64, vp, i64, vp, i64, i64, i64, c_double, c_uint64, c_uint64]
        L.bnn_mx_ld.argtypes = [c_int, i64]
        L.bnn_mx_ld.restype = i64
        L.bnn_mx_scale_bytes.argtypes = [i64, i64]
        L.bnn_mx_scale_bytes.restype = c_size_t
        L.bnn_mx_quantize.argtypes = [vp, c_int, vp, i64, POINTER(MxDesc), vp, i64]
        L.bnn_mx_values.argtypes = [vp, POINTER(MxDesc), c_int, vp, i64]
        L.bnn_block_norm_mx.argtypes = [vp, POINTER(BlockNormDesc), vp, i64, vp, i64, i64, vp, i64, POINTER(MxDesc), vp, i64, vp]
        L.bnn_mx_linear.argtypes = [vp, POINTER(MxLinearDesc), POINTER(MxDesc), vp, i64, vp, i64, vp, i64, POINTER(MxDesc)]
        L.bnn_mx_gated.argtypes = [vp, POINTER(MxGatedDesc), POINTER(MxDesc), vp, i64, vp, i64, POINTER(MxDesc)]
        L.bnn_clip_workspace_bytes.argtypes = [i64]
        L.bnn_clip_workspace_bytes.restype = c_size_t
        L.bnn_clip_gradients.argtypes = [vp, POINTER(Gradient), i64, c_double, c_double, vp]
        L.bnn_mlp_noalloc_max_bytes.argtypes = []
        L.bnn_mlp_noalloc_max_bytes.restype = c_size_t
        L.bnn_mlp_forward_noalloc.argtypes = [vp, POINTER(MlpDesc), vp, i64, i64, vp, i64]
        _lib = L
    return _lib


def _status_string(status: int) -> str:
    try:
        return lib().bnn_status_string(status).decode()
    except Exception:  # pragma: no cover
        return "?"


def _ptr(t):
    return None if t is None else c_void_p(t.data_ptr())


def words(k: int) -> int:
    return (k + 31) // 32


def packed_ld(k: int) -> int:
    """Smallest legal leading dimension (in 32-bit words) of a packed matrix with k bits per row."""
    return ((k + 127) // 128) * 4


class Context:
    """bnn_ctx bound to a device and to torch's current stream on it (or to an explicit stream)."""

    def __init__(self, device: int = 0, stream: "torch.cuda.Stream | None" = None):
        if not torch.cuda.is_available():
            raise RuntimeError("a CUDA device is required; the library has no CPU path")
        self.device = device
        self.stream = stream if stream is not None else torch.cuda.current_stream(device)
        h = c_void_p()
        st = lib().bnn_create(ctypes.byref(h), device, c_void_p(self.stream.cuda_stream))
        if st:
            raise BnnError(st, "bnn_create")
        self._h = h
        self._ws = None
        self._device, self._raw = torch.device("cuda", device), self.stream.cuda_stream
        self._destroy = lib().bnn_destroy      # kept here: module globals may be gone when __del__ runs at interpreter exit

    def close(self):
        h, destroy = getattr(self, "_h", None), getattr(self, "_destroy", None)
        if h and destroy is not None:
            destroy(h)
        self._h = None

    __del__ = close

    def _ck(self, st: int, what: str):
        if st:
            raise BnnError(st, what, lib().bnn_last_cuda_error(self._h))

    def empty(self, *shape, dtype=torch.int32):
        return torch.empty(*shape, dtype=dtype, device=self._device)

    # -- plumbing ------------------------------------------------------------------------------
    def set_workspace(self, ws: "torch.Tensor | None"):
        self._ws = ws
        if ws is None:
            self._ck(lib().bnn_set_workspace(self._h, None, 0), "bnn_set_workspace")
        else:
            self._ck(lib().bnn_set_workspace(self._h, _ptr(ws), ws.numel() * ws.element_size()), "bnn_set_workspace")

    def expand_signs(self, packed, rows: int, K: int):
        """bnn_expand_signs: packed rows x K -> int8 tensor [rows, bnn_expanded_ld(K)] of +1 / -1 (0 beyond K)."""
        ld = int(lib().bnn_expanded_ld(K))
        dst = self.empty(rows, ld, dtype=torch.int8)
        self._ck(lib().bnn_expand_signs(self._h, _ptr(packed), packed.stride(0), rows, K, _ptr(dst)), "bnn_expand_signs")
        return dst

    def baseline_gemm_f32(self, A, B, C=None):
        """bnn_baseline_gemm_f32: the paper's unoptimized float32 comparison kernel (context only)."""
        M, K = A.shape
        N = B.shape[1]
        if C is None:
            C = self.empty(M, N, dtype=torch.float32)
        self._ck(lib().bnn_baseline_gemm_f32(self._h, _ptr(A), _ptr(B), _ptr(C), M, N, K), "bnn_baseline_gemm_f32")
        return C

    def expand_signs_f4(self, packed, rows: int, K: int):
        """bnn_expand_signs_f4: packed rows x K -> uint8 tensor [rows, bnn_expanded_ld_f4(K)] of e2m1 nibbles."""
        ld = int(lib().bnn_expanded_ld_f4(K))
        dst = self.empty(rows, ld, dtype=torch.uint8)
        self._ck(lib().bnn_expand_signs_f4(self._h, _ptr(packed), packed.stride(0), rows, K, _ptr(dst)), "bnn_expand_signs_f4")
        return dst

    def binary_dense_expanded(self, A_exp, W_exp, bits: int, thr, flip, M, N, K, want_bits=True, want_exp=False):
        """bnn_binary_dense_expanded: operands as written by expand_signs (bits 8) or expand_signs_f4 (bits 4).
        Returns (packed signs or None, signs in the next layer's operand format or None)."""
        out = self.empty(M, packed_ld(N)) if want_bits else None
        out_exp = None
        if want_exp:
            ld = int(lib().bnn_expanded_ld_f4(N) if bits == 4 else lib().bnn_expanded_ld(N))
            out_exp = self.empty(M, ld, dtype=torch.uint8 if bits == 4 else torch.int8)
        self._ck(lib().bnn_binary_dense_expanded(self._h, _ptr(A_exp), A_exp.stride(0) * A_exp.element_size(), _ptr(W_exp),
                                                 W_exp.stride(0) * W_exp.element_size(), bits, _ptr(thr), _ptr(flip), _ptr(out),
                                                 packed_ld(N), _ptr(out_exp), out_exp.stride(0) if out_exp is not None else 0,
                                                 M, N, K), "bnn_binary_dense_expanded")
        return out, out_exp

    def set_operand_bits(self, bits: int):
        self._ck(lib().bnn_set_operand_bits(self._h, bits), "bnn_set_operand_bits")

    def set_wait_limit_ns(self, ns: int):
        self._ck(lib().bnn_set_wait_limit_ns(self._h, ns), "bnn_set_wait_limit_ns")

    def debug_drop_loads(self, on: "bool | int"):
        self._ck(lib().bnn_debug_drop_loads(self._h, int(on)), "bnn_debug_drop_loads")

    def measure_pipe_rates(self):
        """bnn_measure_pipe_rates -> dict of thread-level results per clock and SM (popc, lop3, xor+popc+add)."""
        sms = torch.cuda.get_device_properties(self.device).multi_processor_count
        scratch = self.empty(sms * 4104, dtype=torch.uint8)
        a, b, c = c_double(), c_double(), c_double()
        self._ck(lib().bnn_measure_pipe_rates(self._h, _ptr(scratch), scratch.numel(), ctypes.byref(a), ctypes.byref(b),
                                              ctypes.byref(c)), "bnn_measure_pipe_rates")
        return {"popc": a.value, "lop3": b.value, "xor_popc_add": c.value}

    def last_tensor_kernel(self) -> str:
        return lib().bnn_last_tensor_kernel(self._h).decode()

    def last_tensor_kernel_clock(self):
        """(SM MHz inside the tensor-core kernel that ran last, microseconds its first CTA lived)."""
        mhz, us = c_double(), c_double()
        self._ck(lib().bnn_last_tensor_kernel_clock(self._h, ctypes.byref(mhz), ctypes.byref(us)), "bnn_last_tensor_kernel_clock")
        return mhz.value, us.value

    def set_conv_filter_repetition(self, on: bool):
        self._ck(lib().bnn_set_conv_filter_repetition(self._h, int(on)), "bnn_set_conv_filter_repetition")

    def filter_repetition_workspace_bytes(self, C_in: int, C_out: int) -> int:
        return int(lib().bnn_filter_repetition_workspace_bytes(C_in, C_out))

    def filter_repetition_count(self, Wp, C_in: int, C_out: int) -> int:
        """bnn_filter_repetition_count: distinct 2-D filters (up to sign) summed over the input channels."""
        out = c_int64()
        self._ck(lib().bnn_filter_repetition_count(self._h, _ptr(Wp), C_in, C_out, ctypes.byref(out)), "bnn_filter_repetition_count")
        return int(out.value)

    def set_conv_form(self, form: int):
        self._ck(lib().bnn_set_conv_form(self._h, form), "bnn_set_conv_form")

    def set_pair_mode(self, mode: int):
        self._ck(lib().bnn_set_pair_mode(self._h, mode), "bnn_set_pair_mode")

    def set_tile_rows(self, rows: int):
        self._ck(lib().bnn_set_tile_rows(self._h, rows), "bnn_set_tile_rows")

    def set_engine(self, engine: int):
        self._ck(lib().bnn_set_engine(self._h, engine), "bnn_set_engine")

    def gemm_workspace_bytes(self, M: int, N: int, K: int) -> int:
        return int(lib().bnn_gemm_workspace_bytes(M, N, K))

    def conv_workspace_bytes(self, B, H, W, C_in, C_out, pool) -> int:
        return int(lib().bnn_conv_workspace_bytes(B, H, W, C_in, C_out, int(pool)))

    def device_status(self):
        """Synchronises the stream; raises if a kernel reported that one of its bounded waits gave up."""
        self._ck(lib().bnn_device_status(self._h), "bnn_device_status")

    def set_popc_variant(self, variant: int):
        self._ck(lib().bnn_set_popc_variant(self._h, variant), "bnn_set_popc_variant")

    # -- calls, one per C entry point ----------------------------------------------------------------
    def pack_signs(self, src: torch.Tensor, pack_along: int = 0, word_bits: int = 32, dst=None, dst_ld_w=None):
        """src: 2-D tensor (float32 / float16 / int8), row-major.  Returns the packed int32 tensor."""
        dtype = {torch.float32: BNN_F32, torch.float16: BNN_F16, torch.int8: BNN_I8}[src.dtype]
        rows, cols = src.shape
        assert src.stride(1) == 1 or cols <= 1
        out_rows, out_k = (rows, cols) if pack_along == 0 else (cols, rows)
        ld = dst_ld_w if dst_ld_w is not None else packed_ld(out_k)
        if dst is None:
            dst = self.empty(out_rows, ld)
        self._ck(lib().bnn_pack_signs(self._h, _ptr(src), dtype, rows, cols, src.stride(0) if rows > 1 else max(cols, 1),
                                      pack_along, word_bits, _ptr(dst), ld), "bnn_pack_signs")
        return dst

    def xnor_gemm(self, Ap, Bp, M, N, K, C=None, lda_w=None, ldb_w=None, ldc=None):
        if C is None:
            C = self.empty(M, N)
        self._ck(lib().bnn_xnor_gemm(self._h, _ptr(Ap), lda_w if lda_w is not None else Ap.stride(0), _ptr(Bp),
                                     ldb_w if ldb_w is not None else Bp.stride(0), _ptr(C),
                                     ldc if ldc is not None else (C.stride(0) if C.dim() == 2 and M > 1 else max(N, 1)),
                                     M, N, K), "bnn_xnor_gemm")
        return C

    def binary_dense(self, Ap, Wp, thr, flip, M, N, K, out=None, ldo_w=None):
        ld = ldo_w if ldo_w is not None else packed_ld(N)
        if out is None:
            out = self.empty(M, ld)
        self._ck(lib().bnn_binary_dense(self._h, _ptr(Ap), Ap.stride(0), _ptr(Wp), Wp.stride(0), _ptr(thr), _ptr(flip),
                                        _ptr(out), ld, M, N, K), "bnn_binary_dense")
        return out

    def first_layer_bitplanes(self, X, Wp, M, N, K, thr=None, flip=None, want_bits=True, want_sums=False):
        ld = packed_ld(N)
        bits = self.empty(M, ld) if want_bits else None
        sums = self.empty(M, N) if want_sums else None
        self._ck(lib().bnn_first_layer_bitplanes(self._h, _ptr(X), X.stride(0) if M > 1 else max(K, 1), _ptr(Wp),
                                                 Wp.stride(0), _ptr(thr), _ptr(flip), _ptr(bits), ld, _ptr(sums), N,
                                                 M, N, K), "bnn_first_layer_bitplanes")
        return bits, sums

    def binary_conv2d(self, act, B, H, W, C_in, Wp, C_out, pool=False, thr=None, flip=None, want_bits=True,
                      want_sums=False):
        """act: packed int32 [B,H,W,C_in/32] or uint8 [B,H,W,C_in] (first layer)."""
        Ho, Wo = (H // 2, W // 2) if pool else (H, W)
        bits = self.empty(B, Ho, Wo, words(C_out)) if want_bits else None
        sums = self.empty(B, Ho, Wo, C_out) if want_sums else None
        is_u8 = act.dtype == torch.uint8
        self._ck(lib().bnn_binary_conv2d(self._h, None if is_u8 else _ptr(act), _ptr(act) if is_u8 else None, B, H, W,
                                         C_in, _ptr(Wp), C_out, int(pool), _ptr(thr), _ptr(flip), _ptr(bits),
                                         _ptr(sums)), "bnn_binary_conv2d")
        return bits, sums

    def make_mlp_desc(self, layers):
        """layers: list of dicts with Wp, K, N and thr/flip (hidden) or gamma/beta/mean/var/eps (last).
        Returns (MlpDesc, keep-alive tuple)."""
        arr = (LayerDesc * len(layers))()
        for d, L in zip(arr, layers):
            d.Wp = L["Wp"].data_ptr()
            d.ldw_w = L["Wp"].stride(0)
            d.K, d.N = L["K"], L["N"]
            for name in ("thr", "flip", "gamma", "beta", "mean", "var", "W8", "W4"):
                t = L.get(name)
                setattr(d, name, t.data_ptr() if t is not None else None)
            d.eps = float(L.get("eps", 0.0))
        desc = MlpDesc(len(layers), arr)
        return desc, (arr, layers)

    def make_convnet_desc(self, layers):
        """layers: list of dicts with Wp, Cin, Cout, pool, thr, flip and optionally W8, W4.  Returns (ConvNetDesc, keep-alive)."""
        arr = (ConvLayerDesc * len(layers))()
        for d, L in zip(arr, layers):
            d.Wp = L["Wp"].data_ptr()
            d.C_in, d.C_out, d.pool = L["Cin"], L["Cout"], int(L["pool"])
            d.thr = L["thr"].data_ptr()
            d.flip = L["flip"].data_ptr() if L.get("flip") is not None else None
            d.W8 = L["W8"].data_ptr() if L.get("W8") is not None else None
            d.W4 = L["W4"].data_ptr() if L.get("W4") is not None else None
        return ConvNetDesc(len(layers), arr), (arr, layers)

    def convnet_workspace_bytes(self, desc, B: int, H: int, W: int) -> int:
        return int(lib().bnn_convnet_workspace_bytes(ctypes.byref(desc), B, H, W))

    def convnet_forward(self, desc, X, B: int, H: int, W: int, out_bits, layer_out=None):
        hp = None
        if layer_out is not None:
            hp = (c_void_p * desc.n_layers)(*[t.data_ptr() if t is not None else None for t in layer_out])
        self._ck(lib().bnn_convnet_forward(self._h, ctypes.byref(desc), _ptr(X), B, H, W, _ptr(out_bits), hp),
                 "bnn_convnet_forward")
        return out_bits

    def mlp_workspace_bytes(self, desc, batch: int, host_io: bool = False) -> int:
        return int(lib().bnn_mlp_workspace_bytes(ctypes.byref(desc), batch, int(host_io)))

    def mlp_forward(self, desc, X, batch, scores=None, hidden_out=None):
        n_out = desc.layers[desc.n_layers - 1].N
        if scores is None:
            scores = self.empty(batch, n_out, dtype=torch.float32)
        hp = None
        if hidden_out is not None:
            hp = (c_void_p * (desc.n_layers - 1))(*[t.data_ptr() if t is not None else None for t in hidden_out])
        self._ck(lib().bnn_mlp_forward(self._h, ctypes.byref(desc), _ptr(X), X.stride(0) if batch > 1 else X.shape[-1],
                                       batch, _ptr(scores), n_out, hp), "bnn_mlp_forward")
        return scores

    def mlp_forward_noalloc(self, desc, X, batch, scores):
        """bnn_mlp_forward_noalloc: the caller passes the output too, so that nothing is allocated here either."""
        n_out = desc.layers[desc.n_layers - 1].N
        self._ck(lib().bnn_mlp_forward_noalloc(self._h, ctypes.byref(desc), _ptr(X),
                                               X.stride(0) if batch > 1 else X.shape[-1], batch, _ptr(scores), n_out),
                 "bnn_mlp_forward_noalloc")
        return scores

    def mlp_forward_host(self, desc, X_host, batch, scores_host):
        n_out = desc.layers[desc.n_layers - 1].N
        self._ck(lib().bnn_mlp_forward_host(self._h, ctypes.byref(desc), _ptr(X_host), X_host.stride(0), batch,
                                            _ptr(scores_host), n_out), "bnn_mlp_forward_host")
        return scores_host

    # -- real-valued feed-forward sublayer ---------------------------------------------------------------
    def _fit(self, t, rows, cols, dtype, what):
        """Checks a row-major matrix; returns (address, leading dimension)."""
        if t is None:
            return None, 0
        if t.dtype is not dtype or t.shape != (rows, cols) or t.get_device() != self.device:
            raise ValueError(f"{what}: expected {dtype} [{rows}, {cols}] on cuda:{self.device}, got {t.dtype} {list(t.shape)} on {t.device}")
        ld, step = t.stride()
        if step != 1 and cols > 1 and rows:
            raise ValueError(f"{what}: rows must be contiguous (row-major), strides are {t.stride()}")
        if rows <= 1:
            return t.data_ptr(), cols
        if ld < cols:
            raise ValueError(f"{what}: rows overlap, strides are {t.stride()}")
        return t.data_ptr(), ld

    def _vector(self, t, n, dtype, what):
        if t is None:
            return None
        if t.dtype is not dtype or t.dim() != 1 or t.shape[0] != n or t.get_device() != self.device or (n > 1 and t.stride(0) != 1):
            raise ValueError(f"{what}: expected contiguous {dtype} [{n}] on cuda:{self.device}, got {t.dtype} {list(t.shape)} on {t.device}")
        return t.data_ptr()

    def _on(self, layer: Layer):
        """Refuses a layer whose tensors are on another device: their addresses mean nothing on this one."""
        if layer.device != self.device:
            raise ValueError(f"layer: its tensors are on cuda:{layer.device}, the context is on cuda:{self.device}")

    def _here(self):
        """Whether torch's current stream is the context's: then memory needs no care across streams."""
        return _raw_stream(self.device) == self._raw

    def _new(self, rows, cols, dtype, here):
        """A row-major matrix for a result, from the pool of the stream that the library writes it on."""
        if here:
            return _empty_strided((rows, cols), (cols, 1), dtype=dtype, device=self._device)
        with torch.cuda.stream(self.stream):
            t = _empty_strided((rows, cols), (cols, 1), dtype=dtype, device=self._device)
        t.record_stream(torch.cuda.current_stream(self.device))
        return t

    def _new_vector(self, n, dtype, here):
        if here:
            return _empty_strided((n,), (1,), dtype=dtype, device=self._device)
        return self._new(1, n, dtype, here).view(n)

    def _used(self, *tensors):
        """Keeps the memory of tensors of another stream until the work queued on the context's stream is done with it."""
        for t in tensors:
            if t is not None:
                t.record_stream(self.stream)

    def make_linear(self, W, bias=None, act: str = "none") -> Layer:
        """Dense layer y = residual + act(x W^T + bias): W [N, K] float16 or bfloat16, bias [N] or None."""
        if W.dtype not in _PRODUCT_TYPES:
            raise ValueError(f"W: expected float16 or bfloat16, got {W.dtype}")
        if act not in ACTIVATIONS:
            raise ValueError(f"act: one of {', '.join(ACTIVATIONS)}, got {act!r}")
        N, K = W.shape
        p, ld = self._fit(W, N, K, W.dtype, "W")
        d = LinearDesc(_REAL_TYPES[W.dtype], ACTIVATIONS[act], K, N, p, ld, self._vector(bias, N, W.dtype, "bias"))
        return Layer(d, W.dtype, self.device, K, N, (W, bias))

    def make_gated(self, Wg, Wu, act: str = "silu") -> Layer:
        """Gated projections h = act(x Wg^T) * (x Wu^T): Wg, Wu [N, K] float16 or bfloat16."""
        if Wg.dtype not in _PRODUCT_TYPES:
            raise ValueError(f"Wg: expected float16 or bfloat16, got {Wg.dtype}")
        if act not in ACTIVATIONS:
            raise ValueError(f"act: one of {', '.join(ACTIVATIONS)}, got {act!r}")
        N, K = Wg.shape
        pg, ldg = self._fit(Wg, N, K, Wg.dtype, "Wg")
        pu, ldu = self._fit(Wu, N, K, Wg.dtype, "Wu")
        return Layer(GatedDesc(_REAL_TYPES[Wg.dtype], ACTIVATIONS[act], K, N, pg, ldg, pu, ldu), Wg.dtype, self.device, K, N, (Wg, Wu))

    def make_block_norm(self, D: int, dtype, kind: str = "rms", eps: float = 1e-6, alpha: float = 1.0, post: bool = False,
                        post_weight=None, post_shift=None, pre: bool = True, pre_weight=None, pre_shift=None, gate=None,
                        rows_per_gate: int | None = None) -> Layer:
        """Norms around a block: stream = alpha x + gate * (post ? Norm(block) : block), normed = Norm(stream) if pre.
        gate: [D] (one for all rows) or [G, D] with rows_per_gate."""
        if kind not in NORMS:
            raise ValueError(f"kind: one of {', '.join(NORMS)}, got {kind!r}")
        if dtype not in _REAL_TYPES:
            raise ValueError(f"dtype: expected float32, float16 or bfloat16, got {dtype}")
        if gate is not None and gate.dim() == 1:
            gate = gate.unsqueeze(0)
        if gate is not None and rows_per_gate is None:
            if gate.shape[0] != 1:
                raise ValueError("rows_per_gate: needed for a gate of several rows")
            rows_per_gate = 0x7fffffff
        gp, gl = self._fit(gate, gate.shape[0], D, dtype, "gate") if gate is not None else (None, 0)
        v = [self._vector(t, D, dtype, n) for t, n in ((post_weight, "post_weight"), (post_shift, "post_shift"), (pre_weight, "pre_weight"),
                                                       (pre_shift, "pre_shift"))]
        d = BlockNormDesc(_REAL_TYPES[dtype], NORMS[kind], D, eps, alpha, int(post), int(pre), *v, gp, gl, rows_per_gate or 1)
        layer = Layer(d, dtype, self.device, D, D, (post_weight, post_shift, pre_weight, pre_shift, gate))
        layer.gates, layer.rows_per_gate, layer.pre = gate.shape[0] if gate is not None else 0, d.rows_per_gate, bool(pre)
        layer.grads = [n for n, t, on in (("dpost_weight", post_weight, post), ("dpost_shift", post_shift, post),
                                          ("dpre_weight", pre_weight, pre), ("dpre_shift", pre_shift, pre)) if on and t is not None]
        return layer

    @staticmethod
    def _rows16(*tensors):
        return all(t is None or (t.data_ptr() % 16 == 0 and (t.shape[0] <= 1 or t.stride(0) * t.element_size() % 16 == 0)) for t in tensors)

    def linear_workspace_bytes(self, layer: Layer, x, backward: bool = False, dy=None) -> int:
        """Workspace of linear / linear_backward for inputs laid out like x and dy (None: contiguous rows).  A layer without
        activation multiplies dy itself, so its rows count like those of x and W."""
        rows16 = self._rows16(x, dy, layer.tensors[0])
        if backward and dy is None and layer.desc.act == ACTIVATIONS["none"] and x.shape[0] > 1:
            rows16 = rows16 and layer.outer * x.element_size() % 16 == 0
        return int(lib().bnn_linear_workspace_bytes(layer.ref, x.shape[0], int(backward), int(rows16)))

    def gated_workspace_bytes(self, layer: Layer, x, backward: bool = False) -> int:
        """Workspace of gated / gated_backward for inputs laid out like x."""
        return int(lib().bnn_gated_workspace_bytes(layer.ref, x.shape[0], int(backward), int(self._rows16(x, *layer.tensors))))

    def block_norm_workspace_bytes(self, layer: Layer, rows: int) -> int:
        return int(lib().bnn_block_norm_workspace_bytes(layer.ref, rows))

    def linear(self, layer: Layer, x, residual=None, out=None, pre=None):
        """bnn_linear.  pre: float32 [M, N] that receives x W^T + bias for linear_backward.  out may be residual."""
        self._on(layer)
        M, N, dtype, here = x.shape[0], layer.outer, layer.dtype, self._here()
        xp, ldx = self._fit(x, M, layer.inner, dtype, "x")
        rp = pp = None
        ldr = ldp = 0
        if residual is not None:
            rp, ldr = self._fit(residual, M, N, dtype, "residual")
        if pre is not None:
            pp, ldp = self._fit(pre, M, N, torch.float32, "pre")
        if out is None:
            out = self._new(M, N, dtype, here)
            op, ldo = out.data_ptr(), N
        else:
            op, ldo = self._fit(out, M, N, dtype, "out")
        st = lib().bnn_linear(self._h, layer.ref, xp, ldx, M, rp, ldr, op, ldo, pp, ldp)
        if st:
            self._ck(st, "bnn_linear")
        if not here:
            self._used(x, residual, out, pre, *layer.tensors)
        return out

    def linear_backward(self, layer: Layer, dy, x, pre=None, want_dx: bool = True, want_dW: bool = True, want_db: bool = True):
        """bnn_linear_backward -> (dx, dW, dbias); dbias is None for a layer without bias, what is not wanted is None."""
        self._on(layer)
        M, N, K, dtype, here = x.shape[0], layer.outer, layer.inner, layer.dtype, self._here()
        gp, ldg = self._fit(dy, M, N, dtype, "dy")
        xp, ldx = self._fit(x, M, K, dtype, "x")
        pp, ldp = self._fit(pre, M, N, torch.float32, "pre") if pre is not None else (None, 0)
        dx = self._new(M, K, dtype, here) if want_dx else None
        dW = self._new(N, K, dtype, here) if want_dW else None
        db = self._new_vector(N, dtype, here) if want_db and layer.tensors[1] is not None else None
        st = lib().bnn_linear_backward(self._h, layer.ref, gp, ldg, xp, ldx, M, pp, ldp, dx.data_ptr() if want_dx else None, K,
                                       dW.data_ptr() if want_dW else None, K, db.data_ptr() if db is not None else None)
        if st:
            self._ck(st, "bnn_linear_backward")
        if not here:
            self._used(dy, x, pre, *layer.tensors)
        return dx, dW, db

    def _planes(self, pre, M, N):
        if pre is None:
            return None, 0
        if pre.shape != (2, M, N) or pre.dtype is not torch.float32 or pre.get_device() != self.device or not pre.is_contiguous():
            raise ValueError(f"pre: expected contiguous torch.float32 [2, {M}, {N}] on cuda:{self.device}, got {pre.dtype} {list(pre.shape)} "
                             f"with strides {pre.stride()} on {pre.device}")
        return pre.data_ptr(), N

    def gated(self, layer: Layer, x, out=None, pre=None):
        """bnn_gated.  pre: contiguous float32 [2, M, N] that receives x Wg^T and x Wu^T for gated_backward."""
        self._on(layer)
        M, N, dtype, here = x.shape[0], layer.outer, layer.dtype, self._here()
        xp, ldx = self._fit(x, M, layer.inner, dtype, "x")
        pp, ldp = self._planes(pre, M, N)
        if out is None:
            out = self._new(M, N, dtype, here)
            op, ldo = out.data_ptr(), N
        else:
            op, ldo = self._fit(out, M, N, dtype, "out")
        st = lib().bnn_gated(self._h, layer.ref, xp, ldx, M, op, ldo, pp, ldp)
        if st:
            self._ck(st, "bnn_gated")
        if not here:
            self._used(x, out, pre, *layer.tensors)
        return out

    def gated_backward(self, layer: Layer, dh, x, pre=None, want_dx: bool = True, want_dW: bool = True):
        """bnn_gated_backward -> (dx, dWg, dWu); what is not wanted is None.  Without pre both products are computed again."""
        self._on(layer)
        M, N, K, dtype, here = x.shape[0], layer.outer, layer.inner, layer.dtype, self._here()
        gp, ldg = self._fit(dh, M, N, dtype, "dh")
        xp, ldx = self._fit(x, M, K, dtype, "x")
        pp, ldp = self._planes(pre, M, N)
        dx = self._new(M, K, dtype, here) if want_dx else None
        dWg = dWu = wgp = wup = None
        if want_dW:
            dWg, dWu = self._new(N, K, dtype, here), self._new(N, K, dtype, here)
            wgp, wup = dWg.data_ptr(), dWu.data_ptr()
        st = lib().bnn_gated_backward(self._h, layer.ref, gp, ldg, xp, ldx, M, pp, ldp, dx.data_ptr() if want_dx else None, K, wgp, K, wup, K)
        if st:
            self._ck(st, "bnn_gated_backward")
        if not here:
            self._used(dh, x, pre, *layer.tensors)
        return dx, dWg, dWu

    def _gate_rows(self, layer: Layer, M: int):
        if layer.gates * layer.rows_per_gate < M:
            raise ValueError(f"gate: {layer.gates} rows of {layer.rows_per_gate} cover fewer than {M}")

    def _stats(self, stats, M):
        if stats is None:
            return None
        tp, ldt = self._fit(stats, M, 4, torch.float32, "stats")
        if M > 1 and ldt != 4:
            raise ValueError("stats: expected a contiguous tensor")
        return tp

    def block_norm(self, layer: Layer, x, block=None, stream=None, normed=None, stats=None):
        """bnn_block_norm -> (stream, normed); normed is None for a layer without pre.  stream may be x.
        stats: contiguous float32 [M, 4] kept for block_norm_backward."""
        self._on(layer)
        M, D, dtype, here = x.shape[0], layer.inner, layer.dtype, self._here()
        if layer.gates:
            self._gate_rows(layer, M)
        xp, ldx = self._fit(x, M, D, dtype, "x")
        bp, ldb = self._fit(block, M, D, dtype, "block") if block is not None else (None, 0)
        tp = self._stats(stats, M)
        if stream is None:
            stream = self._new(M, D, dtype, here)
            sp, lds = stream.data_ptr(), D
        else:
            sp, lds = self._fit(stream, M, D, dtype, "stream")
        if normed is None and layer.pre:
            normed = self._new(M, D, dtype, here)
            np_, ldn = normed.data_ptr(), D
        else:
            np_, ldn = self._fit(normed, M, D, dtype, "normed")
        st = lib().bnn_block_norm(self._h, layer.ref, xp, ldx, bp, ldb, M, sp, lds, np_, ldn, tp)
        if st:
            self._ck(st, "bnn_block_norm")
        if not here:
            self._used(x, block, stream, normed, stats, *layer.tensors)
        return stream, normed

    def block_norm_backward(self, layer: Layer, dstream, dnormed, x, block=None, stats=None):
        """bnn_block_norm_backward -> dict with dx, dblock and, as far as the layer has them, dgate, dpost_weight, dpost_shift,
        dpre_weight, dpre_shift (None otherwise)."""
        self._on(layer)
        M, D, dtype, here = x.shape[0], layer.inner, layer.dtype, self._here()
        if layer.gates:
            self._gate_rows(layer, M)
        sp, lds = self._fit(dstream, M, D, dtype, "dstream")
        np_, ldn = self._fit(dnormed, M, D, dtype, "dnormed")
        xp, ldx = self._fit(x, M, D, dtype, "x")
        bp, ldb = self._fit(block, M, D, dtype, "block")
        tp = self._stats(stats, M)
        out = dict.fromkeys(("dx", "dblock", "dgate", "dpost_weight", "dpost_shift", "dpre_weight", "dpre_shift"))
        dx = out["dx"] = self._new(M, D, dtype, here)
        g = BlockNormGrads(dx.data_ptr(), D)
        if block is not None:
            t = out["dblock"] = self._new(M, D, dtype, here)
            g.dblock, g.lddb = t.data_ptr(), D
            if layer.gates:
                t = out["dgate"] = self._new(layer.gates, D, dtype, here)
                g.dgate, g.ld_dgate = t.data_ptr(), D
                used = -(-M // layer.rows_per_gate)
                if used < layer.gates:                    # gate rows that no row of the stream uses
                    with torch.cuda.stream(self.stream):
                        t[used:].zero_()
        for name in layer.grads:
            t = out[name] = self._new_vector(D, dtype, here)
            setattr(g, name, t.data_ptr())
        st = lib().bnn_block_norm_backward(self._h, layer.ref, sp, lds, np_, ldn, xp, ldx, bp, ldb, tp, M, ctypes.byref(g))
        if st:
            self._ck(st, "bnn_block_norm_backward")
        if not here:
            self._used(dstream, dnormed, x, block, stats, *layer.tensors)
        return out

    # -- microscaled operands ----------------------------------------------------------------------------
    def make_mx(self, rows: int, cols: int, format: str = "e4m3") -> MxMatrix:
        """Room for a microscaled matrix; its contents are whatever the memory held."""
        if format not in MX_FORMATS:
            raise ValueError(f"format: one of {', '.join(MX_FORMATS)}, got {format!r}")
        if rows < 0 or cols < 0:
            raise ValueError(f"rows, cols: expected sizes, got {rows}, {cols}")
        L, here = lib(), self._here()
        values = self._new(rows, int(L.bnn_mx_ld(MX_FORMATS[format], cols)), torch.uint8, here)
        scales = self._new_vector(int(L.bnn_mx_scale_bytes(rows, cols)), torch.uint8, here)
        return MxMatrix(format, rows, cols, values, scales, self.device)

    def _mx(self, q, rows, cols, what):
        if not isinstance(q, MxMatrix):
            raise ValueError(f"{what}: expected a microscaled matrix (make_mx, mx_quantize), got {type(q).__name__}")
        if (q.rows, q.cols) != (rows, cols) or q.device != self.device:
            raise ValueError(f"{what}: expected [{rows}, {cols}] on cuda:{self.device}, got [{q.rows}, {q.cols}] on cuda:{q.device}")
        return q.ref

    def mx_quantize(self, x, format: str | None = None, out: MxMatrix | None = None, values=None) -> MxMatrix:
        """bnn_mx_quantize: x [M, K] float32, float16 or bfloat16 to `format` ("e4m3" if nothing says otherwise) or into out.  values: a matrix like x that receives
        what the elements stand for; may be x."""
        dtype, here = x.dtype, self._here()
        if dtype not in _REAL_TYPES:
            raise ValueError(f"x: expected float32, float16 or bfloat16, got {dtype}")
        if out is not None and format is not None and format != out.format:
            raise ValueError(f"format: out is {out.format}, got {format!r}")
        M, K = x.shape
        xp, ldx = self._fit(x, M, K, dtype, "x")
        vp, ldv = self._fit(values, M, K, dtype, "values")
        if out is None:
            out = self.make_mx(M, K, format or "e4m3")
        st = lib().bnn_mx_quantize(self._h, _REAL_TYPES[dtype], xp, ldx, self._mx(out, M, K, "out"), vp, ldv)
        if st:
            self._ck(st, "bnn_mx_quantize")
        if not here:
            self._used(x, values, out.values, out.scales)
        return out

    def mx_values(self, q: MxMatrix, dtype=torch.float32, out=None):
        """bnn_mx_values: what the elements of q stand for, [rows, cols] of dtype."""
        here = self._here()
        if dtype not in _REAL_TYPES:
            raise ValueError(f"dtype: expected float32, float16 or bfloat16, got {dtype}")
        ref = self._mx(q, q.rows, q.cols, "q") if isinstance(q, MxMatrix) else self._mx(q, 0, 0, "q")
        if out is None:
            out = self._new(q.rows, q.cols, dtype, here)
        op, ldo = self._fit(out, q.rows, q.cols, dtype, "out")
        st = lib().bnn_mx_values(self._h, ref, _REAL_TYPES[dtype], op, ldo)
        if st:
            self._ck(st, "bnn_mx_values")
        if not here:
            self._used(q.values, q.scales, out)
        return out

    def block_norm_mx(self, layer: Layer, x, block=None, format: str | None = None, out: MxMatrix | None = None, stream=None, values=None, stats=None):
        """bnn_block_norm_mx -> (stream, normed microscaled).  layer: make_block_norm with pre; format as in mx_quantize; values: a matrix like x
        that receives what the normed elements stand for; stream may be x; stats as in block_norm."""
        self._on(layer)
        M, D, dtype, here = x.shape[0], layer.inner, layer.dtype, self._here()
        if out is not None and format is not None and format != out.format:
            raise ValueError(f"format: out is {out.format}, got {format!r}")
        if not layer.pre:
            raise ValueError("layer: has no norm of the stream (pre)")
        if layer.gates:
            self._gate_rows(layer, M)
        xp, ldx = self._fit(x, M, D, dtype, "x")
        bp, ldb = self._fit(block, M, D, dtype, "block")
        vp, ldv = self._fit(values, M, D, dtype, "values")
        tp = self._stats(stats, M)
        if stream is None:
            stream = self._new(M, D, dtype, here)
            sp, lds = stream.data_ptr(), D
        else:
            sp, lds = self._fit(stream, M, D, dtype, "stream")
        if out is None:
            out = self.make_mx(M, D, format or "e4m3")
        st = lib().bnn_block_norm_mx(self._h, layer.ref, xp, ldx, bp, ldb, M, sp, lds, self._mx(out, M, D, "out"), vp, ldv, tp)
        if st:
            self._ck(st, "bnn_block_norm_mx")
        if not here:
            self._used(x, block, stream, values, stats, out.values, out.scales, *layer.tensors)
        return stream, out

    def _mx_layer(self, W, act, dtype, *weights):
        for q in weights:
            if not isinstance(q, MxMatrix):
                raise ValueError(f"weights: expected microscaled matrices (make_mx, mx_quantize), got {type(q).__name__}")
            if q.shape != W.shape or q.format != W.format or q.device != self.device:
                raise ValueError(f"weights: expected {W.format} {list(W.shape)} on cuda:{self.device}, got {q.format} {list(q.shape)} on cuda:{q.device}")
        if dtype not in _PRODUCT_TYPES:
            raise ValueError(f"dtype: expected float16 or bfloat16, got {dtype}")
        if act not in ACTIVATIONS:
            raise ValueError(f"act: one of {', '.join(ACTIVATIONS)}, got {act!r}")

    def make_mx_linear(self, W: MxMatrix, bias=None, act: str = "none", dtype=torch.bfloat16) -> Layer:
        """Dense layer of microscaled operands y = residual + act(x W^T + bias): W [N, K], bias [N] of dtype or None; residual and y are of dtype."""
        self._mx_layer(W, act, dtype, W)
        N, K = W.shape
        d = MxLinearDesc(_REAL_TYPES[dtype], ACTIVATIONS[act], W.desc, self._vector(bias, N, dtype, "bias"))
        layer = Layer(d, dtype, self.device, K, N, (W.values, W.scales, bias))
        layer.format = W.format
        return layer

    def make_mx_gated(self, Wg: MxMatrix, Wu: MxMatrix, act: str = "silu", dtype=torch.bfloat16) -> Layer:
        """Gated projections of microscaled operands h = act(x Wg^T) * (x Wu^T): Wg, Wu [N, K] of one format; h is of dtype."""
        self._mx_layer(Wg, act, dtype, Wg, Wu)
        N, K = Wg.shape
        layer = Layer(MxGatedDesc(_REAL_TYPES[dtype], ACTIVATIONS[act], Wg.desc, Wu.desc), dtype, self.device, K, N,
                      (Wg.values, Wg.scales, Wu.values, Wu.scales))
        layer.format = Wg.format
        return layer

    def _mx_inputs(self, layer, x, kind, made):
        if type(layer.desc) is not kind:
            raise ValueError(f"layer: expected one of microscaled weights, made by {made}")
        self._on(layer)
        if type(x) is not MxMatrix:
            raise ValueError(f"x: expected a microscaled matrix (mx_quantize, block_norm_mx), got {type(x).__name__}")
        if x.format == "e2m1" and layer.format != "e2m1":
            raise ValueError("x: e2m1 inputs go with e2m1 weights")
        return self._mx(x, x.rows, layer.inner, "x")

    def mx_linear(self, layer: Layer, x: MxMatrix, residual=None, out=None, pre=None):
        """bnn_mx_linear.  x: e4m3 (weights of either format) or e2m1 (weights too).  out: a matrix of the layer's type (may be residual), or an MxMatrix
        that receives y microscaled (without residual and pre).  pre: float32 [M, N] that receives x W^T + bias for linear_backward."""
        ref = self._mx_inputs(layer, x, MxLinearDesc, "make_mx_linear")
        M, N, dtype, here = x.rows, layer.outer, layer.dtype, self._here()
        rp, ldr = self._fit(residual, M, N, dtype, "residual")
        pp, ldp = self._fit(pre, M, N, torch.float32, "pre")
        qp = None
        if out is None:
            out = self._new(M, N, dtype, here)
            op, ldo = out.data_ptr(), N
        elif type(out) is MxMatrix:
            op, ldo, qp = None, 0, self._mx_out(out, x, M, N, residual is not None or pre is not None)
        else:
            op, ldo = self._fit(out, M, N, dtype, "out")
        st = lib().bnn_mx_linear(self._h, layer.ref, ref, rp, ldr, op, ldo, pp, ldp, qp)
        if st:
            self._ck(st, "bnn_mx_linear")
        if not here:
            self._used(x.values, x.scales, residual, pre, *self._memory(out), *layer.tensors)
        return out

    def mx_gated(self, layer: Layer, x: MxMatrix, out=None, pre=None):
        """bnn_mx_gated.  x and out as in mx_linear.  pre: contiguous float32 [2, M, N] for gated_backward."""
        ref = self._mx_inputs(layer, x, MxGatedDesc, "make_mx_gated")
        M, N, dtype, here = x.rows, layer.outer, layer.dtype, self._here()
        pp, ldp = self._planes(pre, M, N)
        qp = None
        if out is None:
            out = self._new(M, N, dtype, here)
            op, ldo = out.data_ptr(), N
        elif type(out) is MxMatrix:
            op, ldo, qp = None, 0, self._mx_out(out, x, M, N, pre is not None)
        else:
            op, ldo = self._fit(out, M, N, dtype, "out")
        st = lib().bnn_mx_gated(self._h, layer.ref, ref, op, ldo, pp, ldp, qp)
        if st:
            self._ck(st, "bnn_mx_gated")
        if not here:
            self._used(x.values, x.scales, pre, *self._memory(out), *layer.tensors)
        return out

    def _mx_out(self, out, x, M, N, more):
        if more:
            raise ValueError("out: microscaled results come without residual and pre")
        if out.desc.values == x.desc.values and out.desc.values:
            raise ValueError("out: must not be x, which is read until the end")
        return self._mx(out, M, N, "out")

    @staticmethod
    def _memory(out):
        return (out.values, out.scales) if type(out) is MxMatrix else (out,)

    # -- gradients of a model ----------------------------------------------------------------------------
    def make_gradients(self, tensors, out=None) -> Gradients:
        """The gradients whose norm is taken together: contiguous float32, float16 or bfloat16 tensors that share no memory.  out: where the clipped ones go,
        tensors like them (None: in place).  Storage must stay where it is."""
        tensors = list(tensors)
        to = tensors if out is None else list(out)
        if len(to) != len(tensors):
            raise ValueError(f"out: expected {len(tensors)} tensors, got {len(to)}")
        spans = []
        for i, (g, o) in enumerate(zip(tensors, to)):
            if g.dtype not in _REAL_TYPES or g.get_device() != self.device or not g.is_contiguous():
                raise ValueError(f"tensors[{i}]: expected contiguous float32, float16 or bfloat16 on cuda:{self.device}, got {g.dtype} with strides {g.stride()} on {g.device}")
            if o.dtype is not g.dtype or o.shape != g.shape or o.get_device() != self.device or not o.is_contiguous():
                raise ValueError(f"out[{i}]: expected contiguous {g.dtype} {list(g.shape)} on cuda:{self.device}, got {o.dtype} {list(o.shape)} with strides {o.stride()} on {o.device}")
            n = g.numel() * g.element_size()
            if n:
                spans.append((g.data_ptr(), n, i))
                if o.data_ptr() != g.data_ptr():
                    spans.append((o.data_ptr(), n, i))
        spans.sort()
        for (a, n, i), (b, _, j) in zip(spans, spans[1:]):
            if a + n > b:
                raise ValueError(f"tensors[{i}] and tensors[{j}] (or their out) share memory")
        return Gradients(tensors, to, self.device)

    def clip_workspace_bytes(self, gradients: Gradients) -> int:
        return int(lib().bnn_clip_workspace_bytes(len(gradients.tensors)))

    def clip_gradients(self, gradients: Gradients, max_norm: float, eps: float = 1e-6):
        """bnn_clip_gradients: scales all tensors by min(1, max_norm / (n + eps)); returns n, their norm before that, as one float32 on the device."""
        if gradients.device != self.device:
            raise ValueError(f"gradients: on cuda:{gradients.device}, the context is on cuda:{self.device}")
        if not (max_norm >= 0 and eps >= 0):
            raise ValueError(f"max_norm, eps: expected numbers from 0 on, got {max_norm}, {eps}")
        here = self._here()
        norm = _empty_strided((), (), dtype=torch.float32, device=self._device) if here else self._new(1, 1, torch.float32, here)[0, 0]
        st = lib().bnn_clip_gradients(self._h, gradients.list, len(gradients.tensors), max_norm, eps, norm.data_ptr())
        if st:
            self._ck(st, "bnn_clip_gradients")
        if not here:
            self._used(*gradients.tensors, *gradients.out)
        return norm

    def dropout(self, x, p: float, seed: int, offset: int = 0, residual=None, out=None):
        """bnn_dropout: residual + (kept ? x / (1 - p) : 0); the backward pass is the same call on the gradient.  out may be x."""
        dtype, here = x.dtype, self._here()
        if dtype not in _REAL_TYPES:
            raise ValueError(f"x: expected float32, float16 or bfloat16, got {dtype}")
        if not 0.0 <= p <= 1.0:
            raise ValueError(f"p: expected 0 to 1, got {p}")
        if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
            raise ValueError("seed, offset: expected 64-bit unsigned numbers")
        M, D = x.shape
        xp, ldx = self._fit(x, M, D, dtype, "x")
        rp, ldr = self._fit(residual, M, D, dtype, "residual") if residual is not None else (None, 0)
        if out is None:
            out = self._new(M, D, dtype, here)
            op, ldo = out.data_ptr(), D
        else:
            op, ldo = self._fit(out, M, D, dtype, "out")
        st = lib().bnn_dropout(self._h, _REAL_TYPES[dtype], xp, ldx, rp, ldr, op, ldo, M, D, p, seed, offset)
        if st:
            self._ck(st, "bnn_dropout")
        if not here:
            self._used(x, residual, out)
        return out


def debug_ring_position(stage: int, slots: int, step: int = 1) -> dict:
    """bnn_debug_ring_position: host-only view of the operand-ring arithmetic of the tensor-engine kernels."""
    o = [ctypes.c_uint32() for _ in range(3)] + [ctypes.c_int32()] + [ctypes.c_uint32() for _ in range(4)]
    st = lib().bnn_debug_ring_position(stage, slots, step, *[ctypes.byref(x) for x in o])
    if st:
        raise BnnError(st, "bnn_debug_ring_position")
    keys = ("slot", "barrier", "parity", "reuses", "prev_barrier", "prev_parity", "next_barrier", "next_parity")
    return {k: int(v.value) for k, v in zip(keys, o)}


def fold_batchnorm(gamma, beta, mean, var, eps: float, x_max: int):
    """Host helper bnn_fold_batchnorm: float32 CPU tensors in, (thr int32[n], flip packed int32[ceil(n/32)]) out."""
    n = gamma.numel()
    g, b, m, v = (t.detach().to(torch.float32).contiguous().cpu() for t in (gamma, beta, mean, var))
    thr = torch.empty(n, dtype=torch.int32)
    flip = torch.zeros(words(n), dtype=torch.int32)
    st = lib().bnn_fold_batchnorm(_ptr(g), _ptr(b), _ptr(m), _ptr(v), float(eps), n, int(x_max), _ptr(thr), _ptr(flip))
    if st:
        raise BnnError(st, "bnn_fold_batchnorm")
    return thr, flip
