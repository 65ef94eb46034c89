"""ctypes binding of libllmint8.so.  Argument marshalling only."""
import ctypes as C
import os
from dataclasses import dataclass

HERE = os.path.dirname(os.path.abspath(__file__))
# LLMINT8_LIB names another build of the same library (the measurement build libllmint8_stamps.so)
LIB_PATH = os.environ.get("LLMINT8_LIB") or os.path.join(HERE, "libllmint8.so")

SYMBOLS = [
    "llmint8_status_string", "llmint8_last_hip_error", "llmint8_opad", "llmint8_wq_bytes", "llmint8_xq_bytes",
    "llmint8_workspace_bytes", "llmint8_quantize_weight", "llmint8_find_outliers",
    "llmint8_quantize_rows", "llmint8_matmul", "llmint8_linear", "llmint8_linear_events", "llmint8_dequantize_rows",
    "llmint8_init", "llmint8_linear_static", "llmint8_probe_mfma", "llmint8_probe_read",
    "llmint8_quantize_weight_granular", "llmint8_quantize_rows_granular", "llmint8_linear_granular",
    "llmint8_zp_quantize_weight", "llmint8_zp_quantize_rows", "llmint8_zp_matmul", "llmint8_zp_linear",
    "llmint8_export_weight",
    "llmint8_export_rows", "llmint8_debug_prefill_tile", "llmint8_debug_prefill_tile_for",
    "llmint8_debug_decode_shape", "llmint8_debug_kernel_for", "llmint8_debug_mfma_for",
    "llmint8_debug_weight_reads_for",
    "llmint8_kv_codes_bytes", "llmint8_kv_consts_bytes", "llmint8_kv_ring_bytes", "llmint8_kv_append",
    "llmint8_kv_attention_workspace_bytes", "llmint8_kv_attention", "llmint8_kv_read", "llmint8_debug_kv_plan_for",
]

_lib = None
_f16 = None  # torch.float16, once torch is there


class _KvCache(C.Structure):  # llmint8_kv_cache_t
    _fields_ = [("codes", C.c_void_p), ("consts", C.c_void_p), ("ring", C.c_void_p), ("n_pages", C.c_int),
                ("page_tokens", C.c_int), ("n_slots", C.c_int), ("heads", C.c_int), ("d", C.c_int)]


class _KvBatch(C.Structure):  # llmint8_kv_batch_t
    _fields_ = [("row_start", C.c_void_p), ("kv_len", C.c_void_p), ("pages", C.c_void_p), ("slots", C.c_void_p),
                ("status", C.c_void_p), ("n_seqs", C.c_int), ("n_rows", C.c_int), ("page_stride", C.c_int),
                ("max_rows", C.c_int), ("max_len", C.c_int)]


class KvPlan(C.Structure):  # llmint8_kv_plan_t
    _fields_ = [("tile", C.c_int), ("parts", C.c_int), ("halves", C.c_int), ("workgroups", C.c_int64)]


class Llmint8Error(RuntimeError):
    pass


def lib():
    """Load the library (built by paper_2208_07339_amd.build); fail loudly if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise Llmint8Error(f"{LIB_PATH} is missing: run `python -m paper_2208_07339_amd.build` "
                           "(hipcc, gfx950). There is no fallback path.")
    # torch first: it ships its own HIP runtime, and the library must bind to the one the tensors and
    # streams it is handed come from (a second runtime loaded earlier sees no device)
    import torch
    global _f16
    _f16 = torch.float16
    L = C.CDLL(LIB_PATH)
    vp, i32, sz, f32 = C.c_void_p, C.c_int, C.c_size_t, C.c_float
    L.llmint8_status_string.restype = C.c_char_p
    L.llmint8_status_string.argtypes = [i32]
    L.llmint8_last_hip_error.restype = C.c_char_p
    L.llmint8_last_hip_error.argtypes = []
    L.llmint8_opad.restype = i32
    L.llmint8_opad.argtypes = [i32]
    L.llmint8_wq_bytes.restype = sz
    L.llmint8_wq_bytes.argtypes = [i32, i32]
    L.llmint8_xq_bytes.restype = sz
    L.llmint8_xq_bytes.argtypes = [i32, i32]
    L.llmint8_workspace_bytes.restype = sz
    L.llmint8_workspace_bytes.argtypes = [i32, i32, i32, i32]
    L.llmint8_quantize_weight.restype = i32
    L.llmint8_quantize_weight.argtypes = [vp, i32, i32, vp, vp, vp, sz, vp]
    L.llmint8_find_outliers.restype = i32
    L.llmint8_find_outliers.argtypes = [vp, i32, i32, f32, vp, i32, vp, vp, vp, sz, vp]
    L.llmint8_quantize_rows.restype = i32
    L.llmint8_quantize_rows.argtypes = [vp, i32, i32, vp, vp, i32, vp, vp, vp, vp]
    L.llmint8_matmul.restype = i32
    L.llmint8_matmul.argtypes = [vp, vp, vp, vp, vp, i32, vp, vp, vp, i32, i32, i32, vp, vp, vp, sz, vp]
    L.llmint8_linear.restype = i32
    L.llmint8_linear.argtypes = [vp, i32, i32, f32, vp, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.llmint8_init.restype = i32
    L.llmint8_init.argtypes = []
    L.llmint8_linear_static.restype = i32
    L.llmint8_linear_static.argtypes = [vp, i32, i32, f32, vp, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, vp]
    L.llmint8_probe_mfma.restype = i32
    L.llmint8_probe_mfma.argtypes = [vp, sz, vp, sz, i32, vp, C.POINTER(C.c_double), vp]
    L.llmint8_probe_read.restype = i32
    L.llmint8_probe_read.argtypes = [vp, sz, vp, vp]
    L.llmint8_dequantize_rows.restype = i32
    L.llmint8_dequantize_rows.argtypes = [vp, vp, i32, i32, vp, vp, i32, vp, vp]
    L.llmint8_quantize_weight_granular.restype = i32
    L.llmint8_quantize_weight_granular.argtypes = [vp, i32, i32, i32, vp, vp, vp, sz, vp]
    L.llmint8_quantize_rows_granular.restype = i32
    L.llmint8_quantize_rows_granular.argtypes = [vp, i32, i32, vp, vp, i32, i32, vp, vp, vp, vp]
    L.llmint8_linear_granular.restype = i32
    L.llmint8_linear_granular.argtypes = [vp, i32, i32, f32, i32, vp, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp,
                                          vp, sz, vp]
    L.llmint8_linear_events.restype = i32
    L.llmint8_linear_events.argtypes = L.llmint8_linear_granular.argtypes + [vp, vp]
    L.llmint8_zp_quantize_weight.restype = i32
    L.llmint8_zp_quantize_weight.argtypes = [vp, i32, i32, vp, vp, vp, sz, vp]
    L.llmint8_zp_quantize_rows.restype = i32
    L.llmint8_zp_quantize_rows.argtypes = [vp, i32, i32, vp, vp, i32, vp, vp, vp, vp]
    L.llmint8_zp_matmul.restype = i32
    L.llmint8_zp_matmul.argtypes = [vp, vp, vp, vp, vp, i32, vp, vp, vp, i32, i32, i32, vp, vp, vp, sz, vp]
    L.llmint8_zp_linear.restype = i32
    L.llmint8_zp_linear.argtypes = [vp, i32, i32, f32, vp, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.llmint8_export_weight.restype = i32
    L.llmint8_export_weight.argtypes = [vp, i32, i32, vp, vp]
    L.llmint8_export_rows.restype = i32
    L.llmint8_export_rows.argtypes = [vp, i32, i32, vp, vp]
    L.llmint8_debug_prefill_tile.restype = i32
    L.llmint8_debug_prefill_tile.argtypes = [i32]
    L.llmint8_debug_prefill_tile_for.restype = i32
    L.llmint8_debug_prefill_tile_for.argtypes = [i32, i32, i32]
    L.llmint8_debug_kernel_for.restype = i32
    L.llmint8_debug_kernel_for.argtypes = [i32, i32, i32, i32]
    L.llmint8_debug_mfma_for.restype = i32
    L.llmint8_debug_mfma_for.argtypes = [i32, i32, i32, i32]
    L.llmint8_debug_weight_reads_for.restype = i32
    L.llmint8_debug_weight_reads_for.argtypes = [i32, i32, i32]
    L.llmint8_debug_decode_shape.restype = i32
    L.llmint8_debug_decode_shape.argtypes = [i32]
    i64, cache, batch = C.c_int64, C.POINTER(_KvCache), C.POINTER(_KvBatch)
    L.llmint8_kv_codes_bytes.restype = sz
    L.llmint8_kv_codes_bytes.argtypes = [i32, i32, i32, i32]
    L.llmint8_kv_consts_bytes.restype = sz
    L.llmint8_kv_consts_bytes.argtypes = [i32, i32, i32]
    L.llmint8_kv_ring_bytes.restype = sz
    L.llmint8_kv_ring_bytes.argtypes = [i32, i32, i32]
    L.llmint8_kv_append.restype = i32
    L.llmint8_kv_append.argtypes = [cache, batch, vp, i64, vp, i64, vp, i64, vp, i64, i32, vp, vp, i32, i32, i32, vp]
    L.llmint8_kv_attention_workspace_bytes.restype = sz
    L.llmint8_kv_attention_workspace_bytes.argtypes = [batch, i32, i32, i32]
    L.llmint8_kv_attention.restype = i32
    L.llmint8_kv_attention.argtypes = [cache, batch, vp, i64, i32, f32, i32, i32, vp, i64, vp, sz, vp]
    L.llmint8_debug_kv_plan_for.restype = i32
    L.llmint8_debug_kv_plan_for.argtypes = [batch, i32, i32, i32, i32, C.POINTER(KvPlan)]
    L.llmint8_kv_read.restype = i32
    L.llmint8_kv_read.argtypes = [cache, batch, vp, vp, vp]
    _lib = L
    return L


def _check(code):
    if code != 0:
        detail = f" ({lib().llmint8_last_hip_error().decode()})" if code == 4 else ""
        raise Llmint8Error(f"llmint8 status {code}: {lib().llmint8_status_string(code).decode()}{detail}")


def _torch():
    import torch
    return torch


_raw_stream = None  # (current device, its current stream's handle): torch's own functions, looked up by the first call


def _stream():
    """Handle of the current device's current stream.  The public call makes a Stream object each time, 1.3 us; the function
    behind it, which torch's own generated code uses, is taken once the public one has set the device up."""
    global _raw_stream
    if _raw_stream is not None:
        return _raw_stream[1](_raw_stream[0]())
    torch = _torch()
    handle = torch.cuda.current_stream().cuda_stream
    try:
        _raw_stream = (torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)
    except AttributeError:
        pass
    return handle


def _ptr(t):
    """The address as a plain integer, which ctypes converts by the argument types (an object of c_void_p for each of the
    eleven to fourteen pointers of a call took 4 us of the 10 that a call of one small kernel takes)."""
    return t.data_ptr() if t is not None else None


def opad(cap):
    return lib().llmint8_opad(cap)


def wq_bytes(h, o):
    return lib().llmint8_wq_bytes(h, o)


def xq_bytes(s, h):
    return lib().llmint8_xq_bytes(s, h)


def workspace_bytes(s, h, o, cap):
    return lib().llmint8_workspace_bytes(s, h, o, cap)


@dataclass
class Workspace:
    buf: object  # torch.uint8 device tensor

    @staticmethod
    def allocate(s, h, o, cap, device="cuda"):
        torch = _torch()
        return Workspace(torch.empty(workspace_bytes(s, h, o, cap), dtype=torch.uint8, device=device))

    @property
    def nbytes(self):
        return self.buf.numel()


@dataclass
class QuantizedWeight:
    Wq: object     # uint8/int8 device tensor, private tiled layout
    cw: object     # [o] fp16
    W: object      # [h, o] fp16 original (rows O are read by matmul), or None: rows rebuilt from the codes
    h: int
    o: int


@dataclass
class Outliers:
    idx: object    # [cap] int32
    count: object  # [1] int32
    status: object  # [1] int32
    cap: int


@dataclass
class QuantizedRows:
    Xq: object     # int8 device tensor, private tiled layout
    cx: object     # [s] fp16
    Xo: object     # [s, opad] fp16
    s: int
    h: int


GRANULARITY = {"vectorwise": 0, "rowwise": 1, "tensorwise": 2}  # LLMINT8_VECTORWISE / _ROWWISE / _TENSORWISE


def quantize_weight(W, ws=None, granularity="vectorwise"):
    """llmint8_quantize_weight(_granular): W [h, o] fp16 (device, contiguous) -> QuantizedWeight."""
    torch = _torch()
    assert W.is_cuda and W.dtype == torch.float16 and W.is_contiguous() and W.dim() == 2
    h, o = W.shape
    Wq = torch.empty(wq_bytes(h, o), dtype=torch.int8, device=W.device)
    cw = torch.empty(o, dtype=torch.float16, device=W.device)
    if ws is None:
        ws = Workspace.allocate(1, h, o, 1, W.device)
    if granularity == "vectorwise":
        _check(lib().llmint8_quantize_weight(_ptr(W), h, o, _ptr(Wq), _ptr(cw), _ptr(ws.buf), ws.nbytes, _stream()))
    else:
        _check(lib().llmint8_quantize_weight_granular(_ptr(W), h, o, GRANULARITY[granularity], _ptr(Wq), _ptr(cw),
                                                      _ptr(ws.buf), ws.nbytes, _stream()))
    return QuantizedWeight(Wq, cw, W, h, o)


def find_outliers(X, alpha, cap, ws, out=None):
    """llmint8_find_outliers: X [s, h] fp16 -> Outliers (all on device)."""
    torch = _torch()
    assert X.is_cuda and X.dtype == torch.float16 and X.is_contiguous() and X.dim() == 2
    s, h = X.shape
    if out is None:
        out = Outliers(torch.empty(cap, dtype=torch.int32, device=X.device),
                       torch.empty(1, dtype=torch.int32, device=X.device),
                       torch.empty(1, dtype=torch.int32, device=X.device), cap)
    _check(lib().llmint8_find_outliers(_ptr(X), s, h, float(alpha), _ptr(out.idx), cap, _ptr(out.count),
                                       _ptr(out.status), _ptr(ws.buf), ws.nbytes, _stream()))
    return out


def quantize_rows(X, outl, out=None, granularity="vectorwise"):
    """llmint8_quantize_rows(_granular): X [s, h] fp16 + Outliers -> QuantizedRows."""
    torch = _torch()
    assert X.is_cuda and X.dtype == torch.float16 and X.is_contiguous() and X.dim() == 2
    s, h = X.shape
    if out is None:
        out = QuantizedRows(torch.empty(xq_bytes(s, h), dtype=torch.int8, device=X.device),
                            torch.empty(s, dtype=torch.float16, device=X.device),
                            torch.empty((s, opad(outl.cap)), dtype=torch.float16, device=X.device), s, h)
    if granularity == "vectorwise":
        _check(lib().llmint8_quantize_rows(_ptr(X), s, h, _ptr(outl.idx), _ptr(outl.count), outl.cap, _ptr(out.Xq),
                                           _ptr(out.cx), _ptr(out.Xo), _stream()))
    else:
        _check(lib().llmint8_quantize_rows_granular(_ptr(X), s, h, _ptr(outl.idx), _ptr(outl.count), outl.cap,
                                                    GRANULARITY[granularity], _ptr(out.Xq), _ptr(out.cx),
                                                    _ptr(out.Xo), _stream()))
    return out


def matmul(rows, outl, qw, ws, out=None, want_c_i32=False):
    """llmint8_matmul -> Out [s, o] fp16 (and the raw int32 accumulators if asked)."""
    torch = _torch()
    s, h, o = rows.s, rows.h, qw.o
    assert h == qw.h
    if out is None:
        out = torch.empty((s, o), dtype=torch.float16, device=rows.Xq.device)
    Cd = torch.empty((s, o), dtype=torch.int32, device=rows.Xq.device) if want_c_i32 else None
    _check(lib().llmint8_matmul(_ptr(rows.Xq), _ptr(rows.cx), _ptr(rows.Xo), _ptr(outl.idx), _ptr(outl.count),
                                outl.cap, _ptr(qw.Wq), _ptr(qw.cw), _ptr(qw.W), s, h, o, _ptr(out), _ptr(Cd),
                                _ptr(ws.buf), ws.nbytes, _stream()))
    return (out, Cd) if want_c_i32 else out


def linear(X, qw, alpha, outl, rows, ws, out=None, events=None, granularity="vectorwise"):
    """llmint8_linear(_granular): the three per-call steps in one C call, into preallocated buffers.
    granularity must be the one qw was quantized with (it selects the constants of X here).
    events = (before_matmul, after_matmul): two torch.cuda.Event(enable_timing=True) that have been
    recorded once already (so that their handles exist); llmint8_linear_events records them again."""
    torch = _torch()
    s, h = X.shape
    if out is None:
        out = torch.empty((s, qw.o), dtype=torch.float16, device=X.device)
    head = (_ptr(X), s, h, float(alpha))
    tail = (_ptr(qw.Wq), _ptr(qw.cw), _ptr(qw.W), qw.o, _ptr(outl.idx), outl.cap,
            _ptr(outl.count), _ptr(outl.status), _ptr(rows.Xq), _ptr(rows.cx), _ptr(rows.Xo), _ptr(out),
            _ptr(ws.buf), ws.nbytes, _stream())
    g = GRANULARITY[granularity]
    if events is not None:
        _check(lib().llmint8_linear_events(*head, g, *tail, C.c_void_p(events[0].cuda_event),
                                           C.c_void_p(events[1].cuda_event)))
    elif g == 0:
        _check(lib().llmint8_linear(*head, *tail))
    else:
        _check(lib().llmint8_linear_granular(*head, g, *tail))
    return out


STATIC_SCRATCH_BYTES = 16 << 20  # LLMINT8_STATIC_SCRATCH_BYTES


def init():
    """llmint8_init: per-device set-up of the current device (optional; the first call does the same)."""
    _check(lib().llmint8_init())


def linear_static(X, qw, alpha, outl, rows, out):
    """llmint8_linear_static: llmint8_linear on the library's static scratch; every buffer is the caller's,
    nothing is allocated (out is required)."""
    s, h = X.shape
    _check(lib().llmint8_linear_static(_ptr(X), s, h, float(alpha), _ptr(qw.Wq), _ptr(qw.cw), _ptr(qw.W), qw.o,
                                       _ptr(outl.idx), outl.cap, _ptr(outl.count), _ptr(outl.status), _ptr(rows.Xq),
                                       _ptr(rows.cx), _ptr(rows.Xo), _ptr(out), _stream()))
    return out


def probe_mfma(A_tiles, B_tiles, iters, sink):
    """llmint8_probe_mfma on two tiled int8 device buffers; returns the int8 operations of the launch."""
    ops = C.c_double(0.0)
    _check(lib().llmint8_probe_mfma(_ptr(A_tiles), A_tiles.numel(), _ptr(B_tiles), B_tiles.numel(), int(iters),
                                    _ptr(sink), C.byref(ops), _stream()))
    return ops.value


def probe_read(buf, sink):
    """llmint8_probe_read over a device buffer (bytes)."""
    _check(lib().llmint8_probe_read(_ptr(buf), buf.numel() * buf.element_size(), _ptr(sink), _stream()))


def debug_prefill_tile(cfg):
    """llmint8_debug_prefill_tile: force the prefill GEMM's workgroup tile (-1 = automatic)."""
    _check(lib().llmint8_debug_prefill_tile(int(cfg)))


def debug_prefill_tile_for(s, h, o):
    """llmint8_debug_prefill_tile_for: the tile the library chooses for [s x h] by [h x o] (no GPU needed)."""
    return int(lib().llmint8_debug_prefill_tile_for(int(s), int(h), int(o)))


def debug_kernel_for(s, h, o, zeropoint=False):
    """llmint8_debug_kernel_for: the kernel a product takes: 0 tiled, 1 weight-streaming, 2 .. 5 K split over the waves."""
    return int(lib().llmint8_debug_kernel_for(int(s), int(h), int(o), int(zeropoint)))


def debug_mfma_for(s, h, o, zeropoint=False):
    """llmint8_debug_mfma_for: 16 or 32, the MFMA the tiled kernel uses for a product."""
    return int(lib().llmint8_debug_mfma_for(int(s), int(h), int(o), int(zeropoint)))


def debug_weight_reads_for(h, o, zeropoint=False):
    """llmint8_debug_weight_reads_for: 1 or 2, how often the conversion reads a W of [h x o]."""
    return int(lib().llmint8_debug_weight_reads_for(int(h), int(o), int(zeropoint)))


def debug_decode_shape(cfg):
    """llmint8_debug_decode_shape: force the decode kernel's work split (-1 = default)."""
    _check(lib().llmint8_debug_decode_shape(int(cfg)))


def dequantize_rows(qw, outl):
    """llmint8_dequantize_rows: rows O of W rebuilt from the codes -> [opad, o] fp16."""
    torch = _torch()
    out = torch.empty((opad(outl.cap), qw.o), dtype=torch.float16, device=qw.Wq.device)
    _check(lib().llmint8_dequantize_rows(_ptr(qw.Wq), _ptr(qw.cw), qw.h, qw.o, _ptr(outl.idx), _ptr(outl.count),
                                         outl.cap, _ptr(out), _stream()))
    return out


# ---- zeropoint variant (Eq. 1-5) -------------------------------------------------

@dataclass
class ZpWeight:
    Wq: object     # int8 device tensor, private tiled layout
    zc: object     # [o, 4] int32 records: lo | hi << 16 (fp16 bits), zp, column sum of the codes, 0
    W: object      # [h, o] fp16 original (rows O are read by zp_matmul)
    h: int
    o: int


@dataclass
class ZpRows:
    Xq: object     # int8 device tensor, private tiled layout
    zc: object     # [s, 4] int32 records: lo | hi << 16, zp, row sum of the codes, 0
    Xo: object     # [s, opad] fp16
    s: int
    h: int


def zp_quantize_weight(W, ws=None):
    """llmint8_zp_quantize_weight: W [h, o] fp16 (device, contiguous) -> ZpWeight."""
    torch = _torch()
    assert W.is_cuda and W.dtype == torch.float16 and W.is_contiguous() and W.dim() == 2
    h, o = W.shape
    Wq = torch.empty(wq_bytes(h, o), dtype=torch.int8, device=W.device)
    zc = torch.empty((o, 4), dtype=torch.int32, device=W.device)
    if ws is None:
        ws = Workspace.allocate(1, h, o, 1, W.device)
    _check(lib().llmint8_zp_quantize_weight(_ptr(W), h, o, _ptr(Wq), _ptr(zc), _ptr(ws.buf), ws.nbytes, _stream()))
    return ZpWeight(Wq, zc, W, h, o)


def zp_quantize_rows(X, outl, out=None):
    """llmint8_zp_quantize_rows: X [s, h] fp16 + Outliers -> ZpRows."""
    torch = _torch()
    assert X.is_cuda and X.dtype == torch.float16 and X.is_contiguous() and X.dim() == 2
    s, h = X.shape
    if out is None:
        out = ZpRows(torch.empty(xq_bytes(s, h), dtype=torch.int8, device=X.device),
                     torch.empty((s, 4), dtype=torch.int32, device=X.device),
                     torch.empty((s, opad(outl.cap)), dtype=torch.float16, device=X.device), s, h)
    _check(lib().llmint8_zp_quantize_rows(_ptr(X), s, h, _ptr(outl.idx), _ptr(outl.count), outl.cap, _ptr(out.Xq),
                                          _ptr(out.zc), _ptr(out.Xo), _stream()))
    return out


def zp_matmul(rows, outl, qw, ws, out=None, want_c_i32=False):
    """llmint8_zp_matmul -> Out [s, o] fp16 (and the plain int8 product if asked)."""
    torch = _torch()
    s, h, o = rows.s, rows.h, qw.o
    assert h == qw.h
    if out is None:
        out = torch.empty((s, o), dtype=torch.float16, device=rows.Xq.device)
    Cd = torch.empty((s, o), dtype=torch.int32, device=rows.Xq.device) if want_c_i32 else None
    _check(lib().llmint8_zp_matmul(_ptr(rows.Xq), _ptr(rows.zc), _ptr(rows.Xo), _ptr(outl.idx), _ptr(outl.count),
                                   outl.cap, _ptr(qw.Wq), _ptr(qw.zc), _ptr(qw.W), s, h, o, _ptr(out), _ptr(Cd),
                                   _ptr(ws.buf), ws.nbytes, _stream()))
    return (out, Cd) if want_c_i32 else out


def zp_linear(X, qw, alpha, outl, rows, ws, out=None):
    """llmint8_zp_linear: outlier scan, zeropoint quantization of X and the matmul in one C call."""
    torch = _torch()
    s, h = X.shape
    if out is None:
        out = torch.empty((s, qw.o), dtype=torch.float16, device=X.device)
    _check(lib().llmint8_zp_linear(_ptr(X), s, h, float(alpha), _ptr(qw.Wq), _ptr(qw.zc), _ptr(qw.W), qw.o,
                                   _ptr(outl.idx), outl.cap, _ptr(outl.count), _ptr(outl.status), _ptr(rows.Xq),
                                   _ptr(rows.zc), _ptr(rows.Xo), _ptr(out), _ptr(ws.buf), ws.nbytes, _stream()))
    return out


# ---- 8-bit key/value cache and its attention ----------------------------------------

KV_BLOCK, KV_RING, KV_MAX_D = 32, 64, 256  # LLMINT8_KV_BLOCK / _RING / _MAX_D
KV_BAD_BATCH, KV_BAD_PAGE, KV_NOT_FINITE = 1, 2, 4  # bits of a batch's status word


@dataclass(frozen=True)
class KvCache:
    """Keys and values of a layer (llmint8_kv_cache_t; include/llmint8.h has the layout).  Holds the tensors it is made of."""
    codes: object   # int8 device tensor [n_pages, heads, page_tokens / 32, 2, 32 * dpad]
    consts: object  # fp16 [n_pages, heads, page_tokens / 32, 2]
    ring: object    # fp16 [n_slots, heads, 2, 64, d]
    page_tokens: int
    d: int

    def __post_init__(self):
        torch = _torch()
        dpad = (self.d + 31) // 32 * 32
        n_pages, heads, blocks = self.codes.shape[:3]
        assert self.codes.dtype == torch.int8 and self.consts.dtype == self.ring.dtype == torch.float16
        assert self.page_tokens == blocks * KV_BLOCK and 1 <= self.d <= KV_MAX_D
        assert tuple(self.codes.shape) == (n_pages, heads, blocks, 2, KV_BLOCK * dpad)
        assert tuple(self.consts.shape) == (n_pages, heads, blocks, 2)
        assert tuple(self.ring.shape) == (self.ring.shape[0], heads, 2, KV_RING, self.d)
        for t in (self.codes, self.consts, self.ring):
            assert t.is_cuda and t.is_contiguous() and t.device == self.codes.device
        c = _KvCache(_ptr(self.codes), _ptr(self.consts), _ptr(self.ring), n_pages, self.page_tokens, self.ring.shape[0],
                     heads, self.d)
        object.__setattr__(self, "_c", c)
        object.__setattr__(self, "heads", heads)
        lib()  # (fails here if it is missing, and sets torch up)

    @staticmethod
    def allocate(n_pages, page_tokens, n_slots, heads, d, device="cuda"):
        torch = _torch()
        assert page_tokens % KV_BLOCK == 0
        dpad, blocks = (d + 31) // 32 * 32, page_tokens // KV_BLOCK
        return KvCache(torch.empty((n_pages, heads, blocks, 2, KV_BLOCK * dpad), dtype=torch.int8, device=device),
                       torch.empty((n_pages, heads, blocks, 2), dtype=torch.float16, device=device),
                       torch.empty((n_slots, heads, 2, KV_RING, d), dtype=torch.float16, device=device), page_tokens, d)


@dataclass(frozen=True)
class KvBatch:
    """Which rows of a call belong to which sequence, and where these are in the cache (llmint8_kv_batch_t).  The tensors'
    contents may change from call to call, within max_rows and max_len."""
    row_start: object  # int32 [n_seqs + 1]
    kv_len: object     # int32 [n_seqs], the call's own tokens included
    pages: object      # int32 [n_seqs, most pages of a sequence]
    slots: object      # int32 [n_seqs], or None: sequence b has slot b
    n_rows: int
    max_rows: int
    max_len: int
    status: object = None  # int32 [1], or None

    def __post_init__(self):
        torch = _torch()
        n = self.kv_len.numel()
        given = [t for t in (self.row_start, self.kv_len, self.pages, self.slots, self.status) if t is not None]
        assert all(t.is_cuda and t.dtype == torch.int32 and t.is_contiguous() for t in given)
        assert all(t.device == self.kv_len.device for t in given)
        assert self.row_start.numel() == n + 1 and self.pages.dim() == 2 and self.pages.shape[0] == n
        assert self.slots is None or self.slots.numel() == n
        c = _KvBatch(_ptr(self.row_start), _ptr(self.kv_len), _ptr(self.pages), _ptr(self.slots), _ptr(self.status), n,
                     self.n_rows, self.pages.shape[1], self.max_rows, self.max_len)
        object.__setattr__(self, "_c", c)


def _head_rows(t, n_rows, heads, d):
    """Row stride of fp16 rows [n_rows, heads, d] whose heads lie one after the other."""
    assert t.dtype == _f16 and t.shape == (n_rows, heads, d) and t.is_cuda
    row, head, one = t.stride()
    assert (one == 1 or d == 1) and (head == d or heads == 1)
    return row if n_rows > 1 else max(row, heads * d)


def kv_append(cache, batch, k, v, q=None, q_out=None, cos=None, sin=None, pairs=False):
    """llmint8_kv_append: k, v [n_rows, heads, d] fp16 (rows may be slices of wider ones) into the cache; q [n_rows, heads_q, d],
    if given, rotated like the keys into q_out, which is returned (made if not given; may be q).  cos, sin: fp32
    [positions, rotated features / 2], or None: no rotation."""
    n, d, heads = batch.n_rows, cache.d, cache.heads
    rot = n_pos = ld_q = ld_out = heads_q = 0
    if cos is not None:
        n_pos, half = cos.shape
        rot = 2 * half
        assert cos.shape == sin.shape and cos.dtype == sin.dtype == _torch().float32 and cos.is_cuda and sin.is_cuda
        assert cos.is_contiguous() and sin.is_contiguous()
    if q is not None:
        heads_q = q.shape[1]
        if q_out is None:
            q_out = _torch().empty((n, heads_q, d), dtype=_f16, device=q.device)
        ld_q, ld_out = _head_rows(q, n, heads_q, d), _head_rows(q_out, n, heads_q, d)
    _check(lib().llmint8_kv_append(cache._c, batch._c, _ptr(k), _head_rows(k, n, heads, d), _ptr(v), _head_rows(v, n, heads, d),
                                   _ptr(q), ld_q, _ptr(q_out) if q is not None else None, ld_out, heads_q, _ptr(cos), _ptr(sin),
                                   n_pos, rot, int(pairs), _stream()))
    return q_out


def kv_attention_workspace(cache, batch, heads_q):
    """Scratch of kv_attention for this batch's sizes: kept from call to call and layer to layer."""
    n = lib().llmint8_kv_attention_workspace_bytes(C.byref(batch._c), heads_q, cache.heads, cache.d)
    return Workspace(_torch().empty(n, dtype=_torch().uint8, device=cache.codes.device))


def kv_attention(cache, batch, q, scale=None, causal=True, window=0, ws=None, out=None):
    """llmint8_kv_attention: q [n_rows, heads_q, d] fp16 over the cache -> out, the same shape.  scale: 1 / sqrt(d) if None."""
    n, d, heads_q = batch.n_rows, cache.d, q.shape[1]
    if out is None:
        out = _torch().empty((n, heads_q, d), dtype=_f16, device=q.device)
    if ws is None:
        ws = kv_attention_workspace(cache, batch, heads_q)
    _check(lib().llmint8_kv_attention(cache._c, batch._c, _ptr(q), _head_rows(q, n, heads_q, d), heads_q,
                                      d ** -0.5 if scale is None else scale, int(causal), window, _ptr(out),
                                      _head_rows(out, n, heads_q, d), _ptr(ws.buf), ws.nbytes, _stream()))
    return out


def debug_kv_plan_for(cache, batch, heads_q, window=0):
    """llmint8_debug_kv_plan_for: rows of a tile, parts, halves and workgroups of a call of kv_attention (no GPU needed)."""
    p = KvPlan()
    _check(lib().llmint8_debug_kv_plan_for(batch._c, heads_q, cache.heads, cache.d, window, p))
    return p


def kv_read(cache, batch, k=None, v=None):
    """llmint8_kv_read: keys and values at the batch's rows' positions, fp16 [n_rows, heads, d] each."""
    shape = (batch.n_rows, cache.heads, cache.d)
    if k is None and v is None:
        k, v = (_torch().empty(shape, dtype=_f16, device=cache.codes.device) for _ in range(2))
    for t in (k, v):
        assert t is None or (t.dtype == _f16 and t.shape == shape and t.is_contiguous() and t.is_cuda)
    _check(lib().llmint8_kv_read(cache._c, batch._c, _ptr(k), _ptr(v), _stream()))
    return k, v


def export_weight(qw):
    """Private tiled W_i8 -> [h, o] int8 row-major (test support)."""
    torch = _torch()
    out = torch.empty((qw.h, qw.o), dtype=torch.int8, device=qw.Wq.device)
    _check(lib().llmint8_export_weight(_ptr(qw.Wq), qw.h, qw.o, _ptr(out), _stream()))
    return out


def export_rows(rows):
    """Private tiled X_i8 -> [s, h] int8 row-major (test support)."""
    torch = _torch()
    out = torch.empty((rows.s, rows.h), dtype=torch.int8, device=rows.Xq.device)
    _check(lib().llmint8_export_rows(_ptr(rows.Xq), rows.s, rows.h, _ptr(out), _stream()))
    return out
