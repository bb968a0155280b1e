"""Thin ctypes binding of libfluxbin (include/fluxbin.h, include/fluxbin_quant.h): argument marshalling only.

Every step of the hot path runs in the library's HIP kernels; PyTorch only provides device memory and the stream.
The functions keep the C names. Tensors must be on the current CUDA (HIP) device unless stated otherwise.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional, Tuple

HERE = os.path.dirname(os.path.abspath(__file__))
# FLUXBIN_LIBRARY selects another build of the same library (the host-sanitizer build of the CPU tests)
LIB_PATH = os.environ.get("FLUXBIN_LIBRARY") or os.path.join(HERE, "libfluxbin.so")

FLUXBIN_OK = 0
FLUXBIN_ERR_INVALID_ARG = 1
FLUXBIN_ERR_UNSUPPORTED = 2
FLUXBIN_ERR_BUFFER_TOO_SMALL = 3
FLUXBIN_ERR_HIP = 4
FORMAT_VERSION = 2
HEADER_BYTES = 256

# Entry points declared in include/fluxbin.h.
EXPORTS = (
    "fluxbin_status_string", "fluxbin_last_error_message", "fluxbin_pack_query", "fluxbin_pack",
    "fluxbin_layer_from_header", "fluxbin_workspace_query", "fluxbin_workspace_init", "fluxbin_lut_gemv",
    "fluxbin_lut_gemm_smallbatch", "fluxbin_debug_indices", "fluxbin_unpack_canonical", "fluxbin_stream_probe",
    "fluxbin_rc_workspace_query", "fluxbin_rc_decompose", "fluxbin_structural_search", "fluxbin_get_tuning",
    "fluxbin_set_tuning", "fluxbin_plan_query", "fluxbin_lut_gemv_noalloc",
)
# Entry points declared in include/fluxbin_quant.h.
QUANT_EXPORTS = (
    "fluxbin_w4_quantize", "fluxbin_w4_pack_query", "fluxbin_w4_pack", "fluxbin_w4_workspace_query", "fluxbin_w4_gemm",
    "fluxbin_kv8_cache_query", "fluxbin_kv8_append", "fluxbin_kv8_read", "fluxbin_kv8_workspace_query",
    "fluxbin_kv8_attention",
)
NOALLOC_SCRATCH_BYTES = 8 << 20

KERNEL_NAMES = {0: "batch1", 1: "generic", 2: "lut_batch", 3: "mfma", 4: "rows", 5: "mfma_rows"}


class FluxbinError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"fluxbin status {status}: {message}")
        self.status = status


class Shape(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64), ("N", ctypes.c_int64), ("Kb", ctypes.c_int32), ("Ks", ctypes.c_int32),
                ("mu", ctypes.c_int32), ("reserved0", ctypes.c_int32), ("g_r", ctypes.c_int64),
                ("S", ctypes.c_int64), ("g_s", ctypes.c_int64)]


class Weights(ctypes.Structure):
    _fields_ = [("signs", ctypes.c_void_p), ("alpha_r", ctypes.c_void_p), ("alpha_c", ctypes.c_void_p),
                ("sal_idx", ctypes.c_void_p), ("sal_signs", ctypes.c_void_p), ("alpha_sr", ctypes.c_void_p),
                ("alpha_sc", ctypes.c_void_p), ("inputs_on_device", ctypes.c_int32)]


class Layer(ctypes.Structure):
    _fields_ = [("shape", Shape), ("d_base", ctypes.c_void_p), ("bytes", ctypes.c_uint64),
                ("format_version", ctypes.c_uint32), ("reserved1", ctypes.c_uint32),
                ("Npad", ctypes.c_int64), ("Sv", ctypes.c_int64), ("NC", ctypes.c_int64), ("NSC", ctypes.c_int64),
                ("Mp", ctypes.c_int64), ("Gr", ctypes.c_int64), ("Gs", ctypes.c_int64), ("NRP", ctypes.c_int64),
                ("off_signs", ctypes.c_uint64), ("off_rscale", ctypes.c_uint64), ("off_colscale", ctypes.c_uint64),
                ("off_xidx", ctypes.c_uint64), ("off_chunk_plane", ctypes.c_uint64), ("off_sal_idx", ctypes.c_uint64)]


class W4Shape(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64), ("N", ctypes.c_int64), ("g", ctypes.c_int64), ("has_zeros", ctypes.c_int32),
                ("reserved0", ctypes.c_int32)]


class W4Layer(ctypes.Structure):
    _fields_ = [("shape", W4Shape), ("d_base", ctypes.c_void_p), ("bytes", ctypes.c_uint64),
                ("format_version", ctypes.c_uint32), ("reserved1", ctypes.c_uint32)]


class Kv8CacheDesc(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_int64), ("page_size", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("format_version", ctypes.c_uint32), ("d_base", ctypes.c_void_p),
                ("bytes", ctypes.c_uint64)]


class Kv8Batch(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("sequences", ctypes.c_int32), ("max_blocks", ctypes.c_int32),
                ("block_table_stride", ctypes.c_int64), ("d_offsets", ctypes.c_void_p), ("d_context", ctypes.c_void_p),
                ("d_block_table", ctypes.c_void_p)]


class Tuning(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("nt", "min_units", "blocks", "blocks_per_cu", "depth", "mfma_depth",
                                             "early", "rpt", "mfma", "generic", "mfma_r2", "bat_r2", "rows",
                                             "batch_tile", "mfma_rows", "align", "big_units")]


class PlanInfo(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_int32), ("threads", ctypes.c_int32), ("rows_per_tile", ctypes.c_int32),
                ("depth", ctypes.c_int32), ("batch_groups", ctypes.c_int32),
                ("second_kernel_reduction", ctypes.c_int32), ("early", ctypes.c_int32), ("batch_tiles", ctypes.c_int32),
                ("batch_tile_rows", ctypes.c_int32), ("workgroups_per_tile", ctypes.c_int32),
                ("tiles", ctypes.c_int64), ("units", ctypes.c_int64), ("workgroups", ctypes.c_int64),
                ("workspace_bytes", ctypes.c_uint64)]


_lib = None


def lib() -> ctypes.CDLL:
    """Load libfluxbin.so (built by ``python -m paper_2608_15602_amd.build``). Raises if it is missing: there is no
    fallback implementation."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FluxbinError(-1, f"{LIB_PATH} is missing; build it with `python -m paper_2608_15602_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        L.fluxbin_status_string.restype = ctypes.c_char_p
        L.fluxbin_status_string.argtypes = [ctypes.c_int]
        L.fluxbin_last_error_message.restype = ctypes.c_char_p
        L.fluxbin_last_error_message.argtypes = []
        L.fluxbin_pack_query.argtypes = [ctypes.POINTER(Shape), ctypes.POINTER(sz)]
        L.fluxbin_pack.argtypes = [ctypes.POINTER(Shape), ctypes.POINTER(Weights), vp, sz, ctypes.POINTER(Layer), vp]
        L.fluxbin_layer_from_header.argtypes = [vp, vp, sz, ctypes.POINTER(Layer)]
        L.fluxbin_workspace_query.argtypes = [ctypes.POINTER(Layer), i32, ctypes.POINTER(sz)]
        L.fluxbin_workspace_init.argtypes = [vp, sz, vp]
        L.fluxbin_lut_gemv.argtypes = [ctypes.POINTER(Layer), vp, vp, i32, vp, sz, vp]
        L.fluxbin_lut_gemm_smallbatch.argtypes = [ctypes.POINTER(Layer), i32, vp, i64, vp, i64, i32, vp, sz, vp]
        L.fluxbin_debug_indices.argtypes = [ctypes.POINTER(Layer), vp, vp]
        L.fluxbin_unpack_canonical.argtypes = [ctypes.POINTER(Layer), vp, vp, vp]
        L.fluxbin_stream_probe.argtypes = [ctypes.POINTER(Layer), vp, sz, vp]
        L.fluxbin_rc_workspace_query.argtypes = [i64, i64, i32, ctypes.POINTER(sz)]
        L.fluxbin_rc_decompose.argtypes = [vp, vp, vp, vp, vp, i32, i64, i64, i64, i32, i32, i64, ctypes.c_double,
                                           vp, vp, vp, vp, sz, vp]
        L.fluxbin_structural_search.argtypes = [vp, vp, i64, i64, i64, i64, vp, vp, vp, vp]
        L.fluxbin_get_tuning.argtypes = [ctypes.POINTER(Tuning)]
        L.fluxbin_set_tuning.argtypes = [ctypes.POINTER(Tuning)]
        L.fluxbin_plan_query.argtypes = [ctypes.POINTER(Layer), i32, ctypes.POINTER(PlanInfo)]
        L.fluxbin_lut_gemv_noalloc.argtypes = [ctypes.POINTER(Layer), vp, vp, i32, vp]
        L.fluxbin_w4_quantize.argtypes = [ctypes.POINTER(W4Shape), vp, i32, i64, vp, vp, vp, vp, i64, vp]
        L.fluxbin_w4_pack_query.argtypes = [ctypes.POINTER(W4Shape), ctypes.POINTER(sz)]
        L.fluxbin_w4_pack.argtypes = [ctypes.POINTER(W4Shape), vp, vp, vp, vp, sz, ctypes.POINTER(W4Layer), vp]
        L.fluxbin_w4_workspace_query.argtypes = [ctypes.POINTER(W4Layer), i32, ctypes.POINTER(sz)]
        L.fluxbin_w4_gemm.argtypes = [ctypes.POINTER(W4Layer), i32, vp, i64, vp, i64, i32, vp, sz, vp]
        L.fluxbin_kv8_cache_query.argtypes = [i64, i32, i32, i32, ctypes.POINTER(sz)]
        cache_p, batch_p = ctypes.POINTER(Kv8CacheDesc), ctypes.POINTER(Kv8Batch)
        L.fluxbin_kv8_append.argtypes = [cache_p, batch_p, vp, i64, i64, vp, i64, i64, vp]
        L.fluxbin_kv8_read.argtypes = [cache_p, batch_p, vp, vp, vp]
        L.fluxbin_kv8_workspace_query.argtypes = [cache_p, i64, i32, i32, ctypes.POINTER(sz)]
        L.fluxbin_kv8_attention.argtypes = [cache_p, batch_p, i32, vp, i64, i64, vp, i64, i64, ctypes.c_float, i32, i32, vp,
                                            sz, vp]
        for name in EXPORTS + QUANT_EXPORTS:
            if name not in ("fluxbin_status_string", "fluxbin_last_error_message"):
                getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def _check(status: int) -> None:
    if status != FLUXBIN_OK:
        msg = lib().fluxbin_last_error_message().decode(errors="replace")
        raise FluxbinError(status, msg or lib().fluxbin_status_string(status).decode())


def make_shape(M, N, Kb, Ks, mu, g_r, S, g_s) -> Shape:
    return Shape(int(M), int(N), int(Kb), int(Ks), int(mu), 0, int(g_r), int(S), int(g_s))


def _stream(stream) -> Optional[int]:
    if stream is None:
        # the current stream's handle from torch's own binding: 0.3 us, against 2.7 us (a third of a small call) for
        # building the torch.cuda.Stream object that holds it
        import torch
        if torch.cuda.is_initialized() and hasattr(torch._C, "_cuda_getCurrentRawStream"):
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        return torch.cuda.current_stream().cuda_stream
    return int(stream) if not hasattr(stream, "cuda_stream") else stream.cuda_stream


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if hasattr(t, "data_ptr"):
        return t.data_ptr()
    return t.ctypes.data  # numpy array (host inputs)


def fluxbin_pack_query(shape: Shape) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().fluxbin_pack_query(ctypes.byref(shape), ctypes.byref(n)))
    return n.value


class PackedLayer:
    """A packed device buffer (torch uint8 tensor) and its C descriptor."""

    def __init__(self, buf, layer: Layer):
        self.buf = buf
        self.layer = layer

    @property
    def shape(self) -> Shape:
        return self.layer.shape


def fluxbin_pack(shape: Shape, weights: Dict[str, object], stream=None, device=None) -> PackedLayer:
    """Pack canonical weights. ``weights`` maps the fluxbin_weights field names to torch tensors on the device (or to
    numpy arrays in host memory, then all of them must be numpy)."""
    import torch
    nbytes = fluxbin_pack_query(shape)
    on_dev = all(hasattr(v, "data_ptr") for v in weights.values() if v is not None)
    buf = torch.empty(nbytes, dtype=torch.uint8, device=device or "cuda")
    keep = {k: (v.contiguous() if hasattr(v, "contiguous") else v) for k, v in weights.items()}
    w = Weights(_ptr(keep.get("signs")), _ptr(keep.get("alpha_r")), _ptr(keep.get("alpha_c")),
                _ptr(keep.get("sal_idx")), _ptr(keep.get("sal_signs")), _ptr(keep.get("alpha_sr")),
                _ptr(keep.get("alpha_sc")), 1 if on_dev else 0)
    out = Layer()
    _check(lib().fluxbin_pack(ctypes.byref(shape), ctypes.byref(w), buf.data_ptr(), nbytes, ctypes.byref(out),
                              _stream(stream)))
    return PackedLayer(buf, out)


def fluxbin_layer_from_header(header: bytes, buf) -> PackedLayer:
    out = Layer()
    hb = ctypes.create_string_buffer(bytes(header[:HEADER_BYTES]), HEADER_BYTES)
    _check(lib().fluxbin_layer_from_header(hb, buf.data_ptr(), buf.numel(), ctypes.byref(out)))
    return PackedLayer(buf, out)


def fluxbin_workspace_query(layer: PackedLayer, B: int = 1) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().fluxbin_workspace_query(ctypes.byref(layer.layer), int(B), ctypes.byref(n)))
    return n.value


def fluxbin_workspace_init(ws, stream=None) -> None:
    _check(lib().fluxbin_workspace_init(ws.data_ptr(), ws.numel() * ws.element_size(), _stream(stream)))


def make_workspace(layer: PackedLayer, B: int = 1, stream=None):
    """Allocate (torch) and zero-fill (library kernel) a workspace for batch B."""
    import torch
    n = fluxbin_workspace_query(layer, B)
    ws = torch.empty(max(256, (n + 255) // 256 * 256), dtype=torch.uint8, device=layer.buf.device)
    fluxbin_workspace_init(ws, stream)
    return ws


def _check_io(layer: PackedLayer, x, y, out_fp32: bool, B: int) -> None:
    """The library takes raw pointers: dtype, device, length and inner stride are checked here, before the call."""
    import torch
    s = layer.shape
    dev = layer.buf.device
    if x.dtype != torch.float16 or x.device != dev or x.stride(-1) != 1:
        raise FluxbinError(FLUXBIN_ERR_INVALID_ARG, f"x must be fp16 on {dev} with unit inner stride")
    if x.shape[-1] < s.N or (x.dim() == 2 and x.shape[0] < B):
        raise FluxbinError(FLUXBIN_ERR_INVALID_ARG, f"x has shape {tuple(x.shape)}, needs [{B}, >= {s.N}]")
    want = torch.float32 if out_fp32 else torch.float16
    if y.dtype != want or y.device != dev or y.stride(-1) != 1:
        raise FluxbinError(FLUXBIN_ERR_INVALID_ARG, f"y must be {want} on {dev} with unit inner stride")
    if y.shape[-1] < s.M or (y.dim() == 2 and y.shape[0] < B):
        raise FluxbinError(FLUXBIN_ERR_INVALID_ARG, f"y has shape {tuple(y.shape)}, needs [{B}, >= {s.M}]")


def fluxbin_lut_gemv(layer: PackedLayer, x, y=None, out_fp32: bool = False, workspace=None, stream=None):
    import torch
    M = layer.shape.M
    if y is None:
        y = torch.empty(M, dtype=torch.float32 if out_fp32 else torch.float16, device=x.device)
    if x.dim() != 1 or y.dim() != 1:
        raise FluxbinError(FLUXBIN_ERR_INVALID_ARG, "fluxbin_lut_gemv takes one activation vector x [N] and y [M]")
    _check_io(layer, x, y, out_fp32, 1)
    if workspace is None:
        workspace = make_workspace(layer, 1, stream)
    _check(lib().fluxbin_lut_gemv(ctypes.byref(layer.layer), x.data_ptr(), y.data_ptr(), 1 if out_fp32 else 0,
                                  workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream(stream)))
    return y


def fluxbin_lut_gemv_noalloc(layer: PackedLayer, x, y, out_fp32: bool = False, stream=None):
    """fluxbin_lut_gemv without a workspace (the library's static device scratch); y must be preallocated."""
    if x.dim() != 1 or y.dim() != 1:
        raise FluxbinError(FLUXBIN_ERR_INVALID_ARG, "fluxbin_lut_gemv_noalloc takes x [N] and y [M]")
    _check_io(layer, x, y, out_fp32, 1)
    _check(lib().fluxbin_lut_gemv_noalloc(ctypes.byref(layer.layer), x.data_ptr(), y.data_ptr(), 1 if out_fp32 else 0,
                                          _stream(stream)))
    return y


def fluxbin_lut_gemm_smallbatch(layer: PackedLayer, x, y=None, out_fp32: bool = False, workspace=None, stream=None):
    """x: fp16 [B, N] (row stride x.stride(0)); returns y [B, M]."""
    import torch
    B = x.shape[0]
    M = layer.shape.M
    if y is None:
        y = torch.empty(B, M, dtype=torch.float32 if out_fp32 else torch.float16, device=x.device)
    if x.dim() != 2 or y.dim() != 2:
        raise FluxbinError(FLUXBIN_ERR_INVALID_ARG, "fluxbin_lut_gemm_smallbatch takes x [B, N] and y [B, M]")
    _check_io(layer, x, y, out_fp32, B)
    if workspace is None:
        workspace = make_workspace(layer, B, stream)
    _check(lib().fluxbin_lut_gemm_smallbatch(ctypes.byref(layer.layer), int(B), x.data_ptr(), int(x.stride(0)),
                                             y.data_ptr(), int(y.stride(0)), 1 if out_fp32 else 0,
                                             workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                             _stream(stream)))
    return y


def fluxbin_debug_indices(layer: PackedLayer, stream=None):
    import torch
    s = layer.shape
    n = (2 * layer.layer.NSC) * s.M * (128 // s.mu)
    out = torch.empty(n, dtype=torch.uint8, device=layer.buf.device)
    _check(lib().fluxbin_debug_indices(ctypes.byref(layer.layer), out.data_ptr(), _stream(stream)))
    return out.view(2 * layer.layer.NSC, s.M, 128 // s.mu)


def fluxbin_unpack_canonical(layer: PackedLayer, stream=None) -> Tuple[object, object]:
    import torch
    s = layer.shape
    W = (s.N + 31) // 32
    signs = torch.empty(s.Kb * s.M * W, dtype=torch.int32, device=layer.buf.device)
    dense = None
    if s.S > 0 and s.Ks > 0:
        dense = torch.empty(s.Ks * s.M * ((s.S + 31) // 32), dtype=torch.int32, device=layer.buf.device)
    _check(lib().fluxbin_unpack_canonical(ctypes.byref(layer.layer), signs.data_ptr(),
                                          dense.data_ptr() if dense is not None else None, _stream(stream)))
    return signs.view(s.Kb, s.M, W), (dense.view(s.Ks, s.M, -1) if dense is not None else None)


def fluxbin_stream_probe(layer: PackedLayer, sink, stream=None) -> None:
    """Launch the measurement-only stream probe (the batch-1 kernel's weight requests without the table work) on
    ``sink``, a device buffer of at least 1024 bytes."""
    _check(lib().fluxbin_stream_probe(ctypes.byref(layer.layer), sink.data_ptr(), sink.numel() * sink.element_size(),
                                      _stream(stream)))


def fluxbin_rc_decompose(X, K: int, T: int, g: int, mask=None, prior=None, eps: float = 1e-12, stream=None):
    """RC_Decomp of X * mask (X: float32 [M, N] device tensor; mask: uint8 [N] device tensor or None) into K bases
    with one row scale per (row, block of g columns). prior: None, or (signs, alpha_r, alpha_c, gp) of earlier bases
    (as returned here) whose approximation is subtracted from X first. Returns (signs int32 [K, M, ceil(N/32)]
    canonical bit planes, alpha_r float64 [K, M, ceil(N/g)], alpha_c float64 [K, N])."""
    import torch
    M, N = X.shape
    ws_n = ctypes.c_size_t(0)
    _check(lib().fluxbin_rc_workspace_query(int(M), int(N), int(K), ctypes.byref(ws_n)))
    ws = torch.empty(ws_n.value, dtype=torch.uint8, device=X.device)
    signs = torch.empty(K, M, (N + 31) // 32, dtype=torch.int32, device=X.device)
    ar = torch.empty(K, M, -(-N // g), dtype=torch.float64, device=X.device)
    ac = torch.empty(K, N, dtype=torch.float64, device=X.device)
    ps, par, pac, gp = prior if prior is not None else (None, None, None, 1)
    kp = int(ps.shape[0]) if ps is not None else 0
    _check(lib().fluxbin_rc_decompose(X.data_ptr(), _ptr(mask), _ptr(ps), _ptr(par), _ptr(pac), kp, int(gp), int(M),
                                      int(N), int(K), int(T), int(g), float(eps), signs.data_ptr(), ar.data_ptr(),
                                      ac.data_ptr(), ws.data_ptr(), ws_n.value, _stream(stream)))
    return signs, ar, ac


def fluxbin_structural_search(W, hinv_diag, g: int, s: int, stream=None):
    """Column saliency with a diagonal inverse Hessian and the s most salient columns of every block of g columns.
    W: float32 [M, N] device tensor, hinv_diag: float64 [N] device tensor. Returns (scores float64 [N], indices int32,
    column mask uint8 [N])."""
    import torch
    M, N = W.shape
    n_sal = sum(min(s, N - b0) for b0 in range(0, N, g))
    scores = torch.empty(N, dtype=torch.float64, device=W.device)
    idx = torch.empty(n_sal, dtype=torch.int32, device=W.device)
    mask = torch.empty(N, dtype=torch.uint8, device=W.device)
    _check(lib().fluxbin_structural_search(W.data_ptr(), hinv_diag.data_ptr(), int(M), int(N), int(g), int(s),
                                           scores.data_ptr(), idx.data_ptr(), mask.data_ptr(), _stream(stream)))
    return scores, idx, mask


# ---- linears in 4 bits with group scales ----

def _invalid(message: str) -> FluxbinError:
    return FluxbinError(FLUXBIN_ERR_INVALID_ARG, message)


def _fits(name: str, value, bits: int = 32) -> int:
    """ctypes cuts numbers to their field's bits without a word: what does not fit is refused here."""
    n = int(value)
    if not -(1 << (bits - 1)) <= n < 1 << (bits - 1):
        raise _invalid(f"{name} = {n} is out of range")
    return n


def _on_device(device, **tensors) -> None:
    """Launches go to the current device: it must be the operands'."""
    import torch
    if device.type != "cuda" or device.index != torch.cuda.current_device():
        raise _invalid(f"operands are on {device}, which is not the current CUDA (HIP) device")
    for name, t in tensors.items():
        if t is not None and t.device != device:
            raise _invalid(f"{name} is on {t.device}, not on {device}")


class _Handles:
    """What the calls of a layer or cache need again and again: looked up once, a small call's time is that of its Python."""

    def __init__(self):
        import torch
        self.half, self.single, self.int32 = torch.float16, torch.float32, torch.int32
        self.empty = torch.empty
        self.current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device
        self.raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self.lib = lib()

    def new(self, stream, *size, dtype, device):
        """A tensor whose memory belongs to the stream that the call runs on (the allocator may give memory that other
        work on the current stream still uses, and give it away again before another stream is done with it)."""
        if stream is None:
            return self.empty(size, dtype=dtype, device=device)
        import torch
        if not hasattr(stream, "cuda_stream"):   # a handle; that of the null stream is 0, which ExternalStream takes for none
            stream = torch.cuda.ExternalStream(int(stream)) if int(stream) else torch.cuda.default_stream(device)
        with torch.cuda.stream(stream):
            return self.empty(size, dtype=dtype, device=device)

    def stream(self, stream, index: int):
        if stream is None and self.raw_stream is not None:
            return self.raw_stream(index)
        return _stream(stream)


def _dense(name: str, t, dtype, shape) -> None:
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise _invalid(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}, got {t.dtype} "
                       f"{tuple(t.shape)}")


def fluxbin_w4_quantize(W, g: int, asymmetric: bool = True, values: bool = False, stream=None):
    """Round-to-nearest 4-bit quantization of W (fp16 or fp32 [M, N], unit inner stride) with one scale per row and group of
    g columns, and a zero point where asymmetric. Returns (codes int32 [M, ceil(N/8)], scales fp16 [M, G], zeros uint8
    [M, G] or None, the values the codes stand for as fp16 [M, N] with values, else None)."""
    import torch
    if W.dim() != 2 or W.dtype not in (torch.float16, torch.float32) or (W.shape[1] > 1 and W.stride(1) != 1):
        raise _invalid("W must be fp16 or fp32 [M, N] with unit inner stride")
    M, N = W.shape
    g = _fits("g", g, 64)
    if g < 1:
        raise _invalid(f"g = {g} must be >= 1")
    _on_device(W.device)
    G = -(-N // g)
    use = _Handles()
    new = lambda dtype, *size: use.new(stream, *size, dtype=dtype, device=W.device)
    codes, scales = new(torch.int32, M, -(-N // 8)), new(torch.float16, M, G)
    zeros = new(torch.uint8, M, G) if asymmetric else None
    out = new(torch.float16, M, N) if values else None
    shape = W4Shape(M, N, g, 1 if asymmetric else 0, 0)
    _check(lib().fluxbin_w4_quantize(ctypes.byref(shape), W.data_ptr(), 1 if W.dtype == torch.float32 else 0,
                                     max(N, W.stride(0)) if M == 1 else W.stride(0), codes.data_ptr(), scales.data_ptr(),
                                     _ptr(zeros), _ptr(out), N, _stream(stream)))
    return codes, scales, zeros, out


class PackedW4:
    """A packed 4-bit layer: its device buffer (torch uint8 tensor) and C descriptor."""

    def __init__(self, buf, layer: W4Layer):
        self.buf = buf
        self.layer = layer
        self.M, self.N, self.device, self.ref = layer.shape.M, layer.shape.N, buf.device, ctypes.byref(layer)
        self.index = buf.device.index
        self.use = _Handles()

    @property
    def shape(self) -> W4Shape:
        return self.layer.shape


def fluxbin_w4_pack_query(shape: W4Shape) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().fluxbin_w4_pack_query(ctypes.byref(shape), ctypes.byref(n)))
    return n.value


def fluxbin_w4_pack(codes, scales, zeros, N: int, g: int, stream=None) -> PackedW4:
    """Pack codes, scales and zero points (None: 8 everywhere) as fluxbin_w4_quantize returns them."""
    import torch
    N, g = _fits("N", N, 64), _fits("g", g, 64)
    if codes.dim() != 2 or g < 1 or N < 1:
        raise _invalid("codes must be int32 [M, ceil(N/8)], N and g at least 1")
    M, G = codes.shape[0], -(-N // g)
    _on_device(codes.device, scales=scales, zeros=zeros)
    _dense("codes", codes, torch.int32, (M, -(-N // 8)))
    _dense("scales", scales, torch.float16, (M, G))
    if zeros is not None:
        _dense("zeros", zeros, torch.uint8, (M, G))
    shape = W4Shape(M, N, g, 0 if zeros is None else 1, 0)
    n = fluxbin_w4_pack_query(shape)
    buf = _Handles().new(stream, n, dtype=torch.uint8, device=codes.device)
    out = W4Layer()
    _check(lib().fluxbin_w4_pack(ctypes.byref(shape), codes.data_ptr(), scales.data_ptr(), _ptr(zeros), buf.data_ptr(), n,
                                 ctypes.byref(out), _stream(stream)))
    return PackedW4(buf, out)


def fluxbin_w4_workspace_query(layer: PackedW4, B: int = 1) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().fluxbin_w4_workspace_query(layer.ref, _fits("B", B), ctypes.byref(n)))
    return n.value


def make_w4_workspace(layer: PackedW4, B: int = 1, stream=None):
    """A workspace (torch uint8 tensor, nothing to clear) for calls of up to B rows."""
    import torch
    return layer.use.new(stream, max(256, fluxbin_w4_workspace_query(layer, B)), dtype=torch.uint8, device=layer.device)


def fluxbin_w4_gemm(layer: PackedW4, x, y=None, out_fp32: bool = False, workspace=None, stream=None):
    """y = What x: x fp16 [N] or [B, N] with unit inner stride, y [M] or [B, M]."""
    M, N, index, use = layer.M, layer.N, layer.index, layer.use
    dtype = use.single if out_fp32 else use.half
    one = x.dim() == 1
    B = x.size(0) if x.dim() == 2 else 1
    if x.dtype is not use.half or x.get_device() != index or x.dim() not in (1, 2) or x.size(-1) != N or \
            (N > 1 and x.stride(-1) != 1) or B > 0x7FFFFFFF:
        raise _invalid(f"x must be fp16 [{N}] or [B, {N}] on {layer.device} with unit inner stride, got {x.dtype} "
                       f"{tuple(x.shape)} on {x.device}")
    if y is None:
        y = use.new(stream, *((M,) if one else (B, M)), dtype=dtype, device=layer.device)
    elif y.dtype is not dtype or y.get_device() != index or y.dim() != x.dim() or y.size(-1) != M or \
            not (one or y.size(0) == B) or (M > 1 and y.stride(-1) != 1):
        raise _invalid(f"y must be {dtype} {[M] if one else [B, M]} on {layer.device} with unit inner stride, got {y.dtype} "
                       f"{tuple(y.shape)} on {y.device}")
    if use.current_device() != index:
        raise _invalid(f"operands are on {layer.device}, which is not the current CUDA (HIP) device")
    if workspace is None:
        workspace = make_w4_workspace(layer, B, stream)
    elif workspace.get_device() != index:
        raise _invalid(f"workspace is on {workspace.device}, not on {layer.device}")
    status = use.lib.fluxbin_w4_gemm(layer.ref, B, x.data_ptr(), 0 if B == 1 else x.stride(0), y.data_ptr(),
                                     0 if B == 1 else y.stride(0), 1 if out_fp32 else 0, workspace.data_ptr(),
                                     workspace.nbytes, use.stream(stream, index))
    if status:
        _check(status)
    return y


# ---- paged key/value cache in 8 bits ----

class Kv8Cache:
    """A paged 8-bit key/value cache: its device buffer (torch uint8 tensor, nothing to clear) and C descriptor."""

    def __init__(self, buf, desc: Kv8CacheDesc):
        self.buf = buf
        self.desc = desc
        self.kv_heads, self.head_dim, self.device, self.ref = desc.kv_heads, desc.head_dim, buf.device, ctypes.byref(desc)
        self.index = buf.device.index
        self.use = _Handles()


def fluxbin_kv8_cache_query(pages: int, page_size: int, kv_heads: int, head_dim: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().fluxbin_kv8_cache_query(_fits("pages", pages, 64), _fits("page_size", page_size), _fits("kv_heads", kv_heads),
                                         _fits("head_dim", head_dim), ctypes.byref(n)))
    return n.value


def make_kv8_cache(pages: int, page_size: int, kv_heads: int, head_dim: int, device=None) -> Kv8Cache:
    import torch
    n = fluxbin_kv8_cache_query(pages, page_size, kv_heads, head_dim)
    buf = torch.empty(n, dtype=torch.uint8, device=device or "cuda")
    return Kv8Cache(buf, Kv8CacheDesc(int(pages), int(page_size), int(kv_heads), int(head_dim), 1, buf.data_ptr(), n))


def _kv8_batch(cache: Kv8Cache, rows: int, offsets, context, block_table) -> Kv8Batch:
    index, int32 = cache.index, cache.use.int32
    if cache.use.current_device() != index:
        raise _invalid(f"the cache is on {cache.device}, which is not the current CUDA (HIP) device")
    if offsets.dtype is not int32 or context.dtype is not int32 or block_table.dtype is not int32 or \
            offsets.get_device() != index or context.get_device() != index or block_table.get_device() != index:
        raise _invalid(f"offsets, context and block_table must be int32 on {cache.device}")
    if context.dim() != 1 or offsets.dim() != 1 or block_table.dim() != 2:
        raise _invalid("offsets must be [B + 1], context [B], block_table [B, blocks]")
    B, blocks = block_table.shape
    if context.size(0) != B or offsets.size(0) != B + 1 or not (context.is_contiguous() and offsets.is_contiguous()) or \
            (blocks > 1 and block_table.stride(1) != 1):
        raise _invalid("offsets must be [B + 1], context [B] (contiguous), block_table [B, blocks] with unit inner stride")
    if B > 0x7FFFFFFF or blocks > 0x7FFFFFFF:
        raise _invalid(f"block_table {[B, blocks]} is too large")
    return Kv8Batch(rows, B, blocks, blocks if B == 1 else block_table.stride(0), offsets.data_ptr(), context.data_ptr(),
                    block_table.data_ptr())


def _kv8_rows(cache: Kv8Cache, name: str, t, heads: int) -> int:
    if t.dim() != 3 or t.dtype is not cache.use.half or t.get_device() != cache.index or t.size(1) != heads or \
            t.size(2) != cache.head_dim or t.stride(2) != 1:
        raise _invalid(f"{name} must be fp16 [rows, {heads}, {cache.head_dim}] on {cache.device} with unit inner stride, got "
                       f"{t.dtype} {tuple(t.shape)} on {t.device}")
    return t.size(0)


def fluxbin_kv8_append(cache: Kv8Cache, k, v, offsets, context, block_table, stream=None) -> None:
    """Store keys and values fp16 [rows, kv_heads, head_dim] (rows and heads at any stride). Sequence b has rows
    offsets[b] .. offsets[b+1] - 1, its newest context[b] - n_b .. context[b] - 1; its position p is in page
    block_table[b, p // page_size]. offsets, context and block_table: int32 on the device."""
    rows = _kv8_rows(cache, "k", k, cache.kv_heads)
    if rows != _kv8_rows(cache, "v", v, cache.kv_heads):
        raise _invalid(f"k has {rows} rows, v {v.shape[0]}")
    b = _kv8_batch(cache, rows, offsets, context, block_table)
    status = cache.use.lib.fluxbin_kv8_append(cache.ref, ctypes.byref(b), k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(),
                                              v.stride(0), v.stride(1), cache.use.stream(stream, cache.index))
    if status:
        _check(status)


def fluxbin_kv8_read(cache: Kv8Cache, offsets, context, block_table, rows: int, stream=None):
    """The cached values (k, v), fp16 [rows, kv_heads, head_dim], of the sequences' newest tokens (as fluxbin_kv8_append
    counts them). Rows of no sequence are not written."""
    use, rows = cache.use, _fits("rows", rows, 64)
    if rows < 0:
        raise _invalid(f"rows = {rows} must not be negative")
    b = _kv8_batch(cache, rows, offsets, context, block_table)
    k = use.new(stream, rows, cache.kv_heads, cache.head_dim, dtype=use.half, device=cache.device)
    v = use.new(stream, rows, cache.kv_heads, cache.head_dim, dtype=use.half, device=cache.device)
    status = use.lib.fluxbin_kv8_read(cache.ref, ctypes.byref(b), k.data_ptr(), v.data_ptr(), use.stream(stream, cache.index))
    if status:
        _check(status)
    return k, v


def fluxbin_kv8_workspace_query(cache: Kv8Cache, rows: int, sequences: int, q_heads: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().fluxbin_kv8_workspace_query(cache.ref, _fits("rows", rows, 64), _fits("sequences", sequences),
                                             _fits("q_heads", q_heads), ctypes.byref(n)))
    return n.value


def make_kv8_workspace(cache: Kv8Cache, rows: int, sequences: int, q_heads: int, stream=None):
    """A workspace (torch uint8 tensor, nothing to clear) for attention calls of up to that many rows and sequences."""
    import torch
    n = fluxbin_kv8_workspace_query(cache, rows, sequences, q_heads)
    return cache.use.new(stream, max(256, n), dtype=torch.uint8, device=cache.device)


def fluxbin_kv8_attention(cache: Kv8Cache, q, offsets, context, block_table, out=None, scale: Optional[float] = None,
                          causal: bool = True, window: int = 0, workspace=None, stream=None):
    """Attention of q fp16 [rows, q_heads, head_dim] (rows and heads at any stride) over the cached tokens of the rows'
    sequences, given as to fluxbin_kv8_append. scale: 1 / sqrt(head_dim) by default. causal: a row attends positions up to
    its own; window > 0: only those after its own - window. Returns out, fp16 like q; rows of no sequence are not written."""
    use, heads = cache.use, q.size(1) if q.dim() == 3 else 0
    rows = _kv8_rows(cache, "q", q, heads)
    if out is None:
        out = use.new(stream, *q.shape, dtype=use.half, device=cache.device)
    elif rows != _kv8_rows(cache, "out", out, heads):
        raise _invalid(f"q has {rows} rows, out {out.shape[0]}")
    b = _kv8_batch(cache, rows, offsets, context, block_table)
    if workspace is None:
        workspace = make_kv8_workspace(cache, rows, b.sequences, heads, stream)
    elif workspace.get_device() != cache.index:
        raise _invalid(f"workspace is on {workspace.device}, not on {cache.device}")
    status = use.lib.fluxbin_kv8_attention(cache.ref, ctypes.byref(b), heads, q.data_ptr(), q.stride(0), q.stride(1),
                                           out.data_ptr(), out.stride(0), out.stride(1),
                                           cache.head_dim ** -0.5 if scale is None else scale, 1 if causal else 0,
                                           max(-1, min(int(window), 0x7FFFFFFF)), workspace.data_ptr(), workspace.nbytes,
                                           use.stream(stream, cache.index))
    if status:
        _check(status)
    return out


def fluxbin_get_tuning() -> Dict[str, int]:
    t = Tuning()
    _check(lib().fluxbin_get_tuning(ctypes.byref(t)))
    return {n: getattr(t, n) for n, _ in Tuning._fields_}


def fluxbin_set_tuning(values: Optional[Dict[str, int]]) -> None:
    """Set the process-wide launch-plan tuning (None: the library defaults)."""
    if values is None:
        _check(lib().fluxbin_set_tuning(None))
        return
    t = Tuning(**{n: int(values[n]) for n, _ in Tuning._fields_})
    _check(lib().fluxbin_set_tuning(ctypes.byref(t)))


class tuning:
    """Context manager: the current tuning with some fields overridden, restored on exit.
    Example: ``with fluxbin.tuning(mfma=0): ...`` runs the LUT batch kernel for every small batch."""

    def __init__(self, **overrides):
        self.overrides = overrides

    def __enter__(self):
        self.saved = fluxbin_get_tuning()
        new = dict(self.saved)
        for k, v in self.overrides.items():
            if k not in new:
                raise KeyError(f"unknown tuning field {k}")
            new[k] = int(v)
        fluxbin_set_tuning(new)
        return self

    def __exit__(self, *exc):
        fluxbin_set_tuning(self.saved)
        return False


def fluxbin_plan_query(layer: PackedLayer, B: int = 1) -> Dict[str, object]:
    """The launch plan a call with batch B would use (kernel name, workgroups, ...)."""
    p = PlanInfo()
    _check(lib().fluxbin_plan_query(ctypes.byref(layer.layer), int(B), ctypes.byref(p)))
    out = {n: getattr(p, n) for n, _ in PlanInfo._fields_}
    out["kernel_name"] = KERNEL_NAMES.get(p.kernel, str(p.kernel))
    return out
