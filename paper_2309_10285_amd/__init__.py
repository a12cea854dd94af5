"""Python binding of libfls (argument marshalling only; every step of the path runs in the HIP kernels).

Function names and argument order follow include/fls.h.  Tensors are torch tensors on the GPU,
used for device memory and streams only:
  W  dense : float16 [M, K] contiguous            (row-major M x K)
  X        : float16 [N, K] contiguous            (== column-major K x N, ld = K)
  C        : float16 [N, M] contiguous            (== column-major M x N, ld = M)
  blob     : uint8 1-D
  Wq, Ws   : float8_e4m3fn [M, K], float8_e8m0fnu [M, scale_stride(K)], contiguous
There is no CPU fallback: without the built library, or without a GPU, calls raise.
"""
import ctypes
import operator
import os
import struct
import weakref

TILE_M = 128
TILE_K = 32
MAX_N = 8192
ORDER_LOCATION = 0
ORDER_BANK = 1

OK, EINVAL, EALIGN, ECAPACITY, EFORMAT, EWORKSPACE, EHIP, EHANDOVER, ESCRATCH = 0, -1, -2, -3, -4, -5, -6, -7, -8
NOALLOC_MAX_N = 32

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfls.so")
_lib = None
_ws_tensor = None  # keeps the registered workspace alive
_ws_made = []      # and those that the ensure_... functions made: a recorded graph uses the one that was registered when it was recorded

EXPORTS = ("fls_compress_bound", "fls_compress", "fls_compress_bound_v2", "fls_compress_v2", "fls_inspect", "fls_workspace_bytes", "fls_set_workspace",
           "fls_check_workspace", "fls_spmm", "fls_spmm_stats", "fls_spmm_noalloc", "fls_forget", "fls_dense_gemm", "fls_quantize",
           "fls_fp8_workspace_bytes", "fls_fp8_gemm", "fls_attention_workspace_bytes", "fls_attention", "fls_strerror")


class FlsStats(ctypes.Structure):
    _fields_ = [("format_version", ctypes.c_uint32), ("tile_m", ctypes.c_uint32), ("tile_k", ctypes.c_uint32),
                ("order_policy", ctypes.c_uint32), ("M", ctypes.c_uint64), ("K", ctypes.c_uint64),
                ("nnz", ctypes.c_uint64), ("num_tiles", ctypes.c_uint64), ("max_tile_words", ctypes.c_uint64),
                ("bytes_total", ctypes.c_uint64), ("bytes_header", ctypes.c_uint64),
                ("bytes_offsets", ctypes.c_uint64), ("bytes_nonzeros", ctypes.c_uint64)]

    def as_dict(self):
        return dict(zip(_STATS_NAMES, _STATS_LAYOUT.unpack_from(self)))


# A call of a few microseconds feels every attribute that Python looks up, so a struct is filled and read in one go, pointers go to
# ctypes as integers, and the current stream is asked for as a number.
_STATS_NAMES = tuple(k for k, _ in FlsStats._fields_)
_STATS_LAYOUT = struct.Struct("<4I9Q")
_stats_values = operator.itemgetter(*_STATS_NAMES)
assert _STATS_LAYOUT.size == ctypes.sizeof(FlsStats)


def _stats_struct(stats):
    try:
        return FlsStats.from_buffer_copy(_STATS_LAYOUT.pack(*_stats_values(stats)))
    except struct.error:  # a value that its field does not hold: cut to the field as ctypes does, for the library to judge; TypeError for one that is no integer
        return FlsStats(**{k: stats[k] for k in _STATS_NAMES})


class FlsError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} ({code})")


def lib():
    """The loaded C-ABI library; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_2309_10285_amd._build.build()")
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, sz, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int
        L.fls_compress_bound.argtypes = [i64, i64, ctypes.POINTER(sz)]
        L.fls_compress_bound.restype = ci
        L.fls_compress.argtypes = [vp, i64, i64, vp, sz, ci, ctypes.POINTER(FlsStats), vp]
        L.fls_compress.restype = ci
        L.fls_compress_bound_v2.argtypes = [i64, i64, ctypes.POINTER(sz)]
        L.fls_compress_bound_v2.restype = ci
        L.fls_compress_v2.argtypes = [vp, i64, i64, vp, sz, ctypes.POINTER(FlsStats), vp]
        L.fls_compress_v2.restype = ci
        L.fls_inspect.argtypes = [vp, ctypes.POINTER(FlsStats)]
        L.fls_inspect.restype = ci
        L.fls_workspace_bytes.argtypes = [i64, i64, i64]
        L.fls_workspace_bytes.restype = sz
        L.fls_set_workspace.argtypes = [vp, sz, vp]
        L.fls_set_workspace.restype = ci
        L.fls_check_workspace.argtypes = [vp]
        L.fls_check_workspace.restype = ci
        L.fls_spmm.argtypes = [vp, vp, vp, i64, i64, i64, vp]
        L.fls_spmm.restype = ci
        L.fls_spmm_stats.argtypes = [vp, ctypes.POINTER(FlsStats), vp, vp, i64, i64, i64, vp]
        L.fls_spmm_stats.restype = ci
        L.fls_spmm_noalloc.argtypes = [vp, ctypes.POINTER(FlsStats), vp, vp, i64, i64, i64, vp]
        L.fls_spmm_noalloc.restype = ci
        L.fls_forget.argtypes = [vp]
        L.fls_forget.restype = None
        L.fls_dense_gemm.argtypes = [vp, vp, vp, i64, i64, i64, vp]
        L.fls_dense_gemm.restype = ci
        L.fls_quantize.argtypes = [vp, i64, i64, vp, vp, vp]
        L.fls_quantize.restype = ci
        L.fls_fp8_workspace_bytes.argtypes = [i64, i64, i64]
        L.fls_fp8_workspace_bytes.restype = sz
        L.fls_fp8_gemm.argtypes = [vp, vp, vp, vp, i64, i64, i64, vp]
        L.fls_fp8_gemm.restype = ci
        L.fls_attention_workspace_bytes.argtypes = [vp]
        L.fls_attention_workspace_bytes.restype = sz
        L.fls_attention.argtypes = [vp] * 10
        L.fls_attention.restype = ci
        L.fls_internal_fp8_plan.argtypes = [ctypes.c_uint32] * 3 + [ci, ctypes.POINTER(ctypes.c_uint32)]
        L.fls_internal_fp8_plan.restype = None
        L.fls_internal_attention_plan.argtypes = [i64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, i64, i64, ci, ctypes.POINTER(ctypes.c_uint32)]
        L.fls_internal_attention_plan.restype = None
        L.fls_internal_spmm_plan.argtypes = [ctypes.c_uint32] * 5 + [ci, ci, ctypes.POINTER(ctypes.c_uint32)]
        L.fls_internal_spmm_plan.restype = None
        L.fls_strerror.argtypes = [ci]
        L.fls_strerror.restype = ctypes.c_char_p
        _lib = L
    return _lib


def strerror(code):
    return lib().fls_strerror(code).decode()


_raw_stream = None
_several_devices = False


def _stream():
    """The current stream of the current device, as hipStream_t."""
    global _raw_stream, _several_devices
    if _raw_stream is None:
        import torch

        _several_devices = torch.cuda.device_count() > 1

        torch.cuda.current_stream()  # initialises torch's GPU side, or raises
        # what that call is made of, without the Stream object: a microsecond less, but names that torch does not promise
        get, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        if get and device:
            _raw_stream = lambda: get(device())
        else:
            _raw_stream = lambda: torch.cuda.current_stream().cuda_stream
    return _raw_stream()


def _check(rc, where):
    if rc != OK:
        raise FlsError(rc, where)


_forgets = {}  # address of a blob -> the finalizer of its memory


def _forget_when_freed(blob):
    """The library remembers a blob's address until the memory goes back to torch's allocator, which hands it out again for something else: an entry of the
    other format version would be read wrongly.  What is copied over a blob in memory that stays is for fls_forget."""
    storage, at = blob.untyped_storage(), blob.data_ptr()
    known = _forgets.get(at)
    alive = known.peek() if known is not None else None
    if alive is None or alive[0] is not storage:
        _forgets[at] = end = weakref.finalize(storage, _freed, at)
        end.atexit = False


def _freed(at):
    _forgets.pop(at, None)
    lib().fls_forget(at)


def fls_compress_bound(M, K):
    out = ctypes.c_size_t(0)
    _check(lib().fls_compress_bound(M, K, ctypes.byref(out)), "fls_compress_bound")
    return out.value


def fls_inspect(header_bytes):
    """header_bytes: the first 64 bytes of a blob, on the host (bytes / bytearray / numpy uint8)."""
    buf = (ctypes.c_uint8 * 64).from_buffer_copy(bytes(header_bytes)[:64])
    st = FlsStats()
    _check(lib().fls_inspect(ctypes.cast(buf, ctypes.c_void_p), ctypes.byref(st)), "fls_inspect")
    return st.as_dict()


def fls_workspace_bytes(M, K, N):
    return int(lib().fls_workspace_bytes(M, K, N))


def fls_set_workspace(ws):
    """ws: uint8 CUDA tensor (caller-owned device memory); kept referenced until replaced."""
    global _ws_tensor
    _check(lib().fls_set_workspace(ws.data_ptr(), ws.numel() * ws.element_size(), _stream()),
           "fls_set_workspace")
    _ws_tensor = ws


def ensure_workspace(M, K, N):
    """Registers a (torch-allocated) workspace large enough for this shape if the current one is not; not while a graph is recorded, unless it is large enough already."""
    need = lib().fls_workspace_bytes(M, K, N)
    if need == 0 or _ws_tensor is None or _ws_tensor.numel() < need:
        _ensure(need, "fls_workspace_bytes")


def _ensure(need, where):
    import torch

    if need == 0:
        raise FlsError(EINVAL, where)
    if torch.cuda.is_current_stream_capturing():  # memory of the graph's own, cleared in each replay
        raise FlsError(EWORKSPACE, where)
    # a power of two, and one of each: all that were ever made are together less than twice the largest, four times what was needed at most
    size = 1 << (need - 1).bit_length()
    for ws in _ws_made:  # a caller's own was registered since
        if ws.numel() == size and (not _several_devices or _on_this_device(ws)):
            break
    else:
        ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        _ws_made.append(ws)
    fls_set_workspace(ws)


def fls_compress(W, out=None, order_policy=ORDER_LOCATION):
    """W: float16 [M, K] CUDA tensor.  Returns (blob uint8 CUDA tensor trimmed to its size, stats dict)."""
    import torch

    assert W.is_cuda and W.dtype == torch.float16 and W.is_contiguous() and W.dim() == 2
    M, K = W.shape
    if out is None:
        out = torch.empty(fls_compress_bound(M, K), dtype=torch.uint8, device=W.device)
    _forget_when_freed(out)
    st = FlsStats()
    rc = lib().fls_compress(W.data_ptr(), M, K, out.data_ptr(), out.numel(),
                            order_policy, ctypes.byref(st), _stream())
    _check(rc, "fls_compress")
    return out[:st.bytes_total], st.as_dict()


def fls_compress_bound_v2(M, K):
    out = ctypes.c_size_t(0)
    _check(lib().fls_compress_bound_v2(M, K, ctypes.byref(out)), "fls_compress_bound_v2")
    return out.value


def fls_compress_v2(W, out=None):
    """fls_compress for format version 2 (four entries share a word of locations, 3 bytes per nonzero)."""
    import torch

    assert W.is_cuda and W.dtype == torch.float16 and W.is_contiguous() and W.dim() == 2
    M, K = W.shape
    if out is None:
        out = torch.empty(fls_compress_bound_v2(M, K), dtype=torch.uint8, device=W.device)
    _forget_when_freed(out)
    st = FlsStats()
    rc = lib().fls_compress_v2(W.data_ptr(), M, K, out.data_ptr(), out.numel(),
                               ctypes.byref(st), _stream())
    _check(rc, "fls_compress_v2")
    return out[:st.bytes_total], st.as_dict()


def fls_spmm(blob, X, C, M, K, N):
    import torch

    assert blob.is_cuda and blob.dtype == torch.uint8 and blob.is_contiguous()
    assert X.is_cuda and X.dtype == torch.float16 and X.is_contiguous() and X.shape == (N, K)
    assert C.is_cuda and C.dtype == torch.float16 and C.is_contiguous() and C.shape == (N, M)
    at = blob.data_ptr()
    if at not in _forgets:
        _forget_when_freed(blob)
    _check(lib().fls_spmm(at, X.data_ptr(),
                          C.data_ptr(), M, K, N, _stream()), "fls_spmm")
    return C


def fls_spmm_stats(blob, stats, X, C, M, K, N):
    """fls_spmm with the blob's statistics passed in (the dict fls_compress / fls_compress_v2 / fls_inspect returned):
    no header read-back, nothing remembered about the blob."""
    import torch

    assert blob.is_cuda and blob.dtype == torch.uint8 and blob.is_contiguous()
    assert X.is_cuda and X.dtype == torch.float16 and X.is_contiguous() and X.shape == (N, K)
    assert C.is_cuda and C.dtype == torch.float16 and C.is_contiguous() and C.shape == (N, M)
    st = _stats_struct(stats)
    _check(lib().fls_spmm_stats(blob.data_ptr(), ctypes.byref(st), X.data_ptr(),
                                C.data_ptr(), M, K, N, _stream()), "fls_spmm_stats")
    return C


def fls_spmm_noalloc(blob, stats, X, C, M, K, N):
    """fls_spmm on the library's static scratch (no workspace, no header read-back); stats: the dict fls_compress
    or fls_inspect returned for this blob."""
    import torch

    assert blob.is_cuda and blob.dtype == torch.uint8 and blob.is_contiguous()
    assert X.is_cuda and X.dtype == torch.float16 and X.is_contiguous() and X.shape == (N, K)
    assert C.is_cuda and C.dtype == torch.float16 and C.is_contiguous() and C.shape == (N, M)
    st = _stats_struct(stats)
    _check(lib().fls_spmm_noalloc(blob.data_ptr(), ctypes.byref(st), X.data_ptr(),
                                  C.data_ptr(), M, K, N, _stream()), "fls_spmm_noalloc")
    return C


def prepare_spmm(blob, X, C, M, K, N):
    """Checks and marshals the arguments of fls_spmm once; returns a callable that enqueues the call on the stream
    that was current when it was prepared.  For tight loops: a Python-side check per call costs as much time as
    the kernel runs."""
    import torch

    assert blob.is_cuda and blob.dtype == torch.uint8 and blob.is_contiguous()
    assert X.is_cuda and X.dtype == torch.float16 and X.is_contiguous() and X.shape == (N, K)
    assert C.is_cuda and C.dtype == torch.float16 and C.is_contiguous() and C.shape == (N, M)
    f = lib().fls_spmm
    _forget_when_freed(blob)
    args = (blob.data_ptr(), X.data_ptr(), C.data_ptr(),
            M, K, N, _stream())
    keep = (blob, X, C)  # the tensors stay alive as long as the callable does

    def call(_keep=keep):
        rc = f(*args)
        if rc != OK:
            _check(rc, "fls_spmm")

    return call


def prepare_spmm_noalloc(blob, stats, X, C, M, K, N):
    """As prepare_spmm, for fls_spmm_noalloc (stats: the dict fls_compress or fls_inspect returned for this blob)."""
    import torch

    assert blob.is_cuda and blob.dtype == torch.uint8 and blob.is_contiguous()
    assert X.is_cuda and X.dtype == torch.float16 and X.is_contiguous() and X.shape == (N, K)
    assert C.is_cuda and C.dtype == torch.float16 and C.is_contiguous() and C.shape == (N, M)
    f = lib().fls_spmm_noalloc
    st = _stats_struct(stats)
    args = (blob.data_ptr(), ctypes.byref(st), X.data_ptr(),
            C.data_ptr(), M, K, N, _stream())
    keep = (blob, X, C, st)

    def call(_keep=keep):
        rc = f(*args)
        if rc != OK:
            _check(rc, "fls_spmm_noalloc")

    return call


def prepare_dense_gemm(W, X, C, M, K, N):
    """As prepare_spmm, for fls_dense_gemm."""
    import torch

    assert W.is_cuda and W.dtype == torch.float16 and W.is_contiguous() and W.shape == (M, K)
    assert X.is_cuda and X.dtype == torch.float16 and X.is_contiguous() and X.shape == (N, K)
    assert C.is_cuda and C.dtype == torch.float16 and C.is_contiguous() and C.shape == (N, M)
    f = lib().fls_dense_gemm
    args = (W.data_ptr(), X.data_ptr(), C.data_ptr(),
            M, K, N, _stream())
    keep = (W, X, C)

    def call(_keep=keep):
        rc = f(*args)
        if rc != OK:
            _check(rc, "fls_dense_gemm")

    return call


def spmm_plan(stats, N, cus=256, entry="fls_spmm"):
    """What a product with that blob and N columns runs on a GPU of that many CUs, from the library's own rule: a dict of pass
    ("narrow", "wide": the 64-column pass, "block"), share, rounds and slices.  Needs no GPU."""
    out = (ctypes.c_uint32 * 4)()
    lib().fls_internal_spmm_plan(stats["max_tile_words"], stats["format_version"], stats["M"], stats["K"], N, cus,
                                 int(entry != "fls_spmm_noalloc"), out)
    return dict(zip(("pass", "share", "rounds", "slices"), (("narrow", "wide", "block")[out[0]], *out[1:])))


def fls_check_workspace():
    """Waits for the current stream; raises FlsError(EHANDOVER) if a kernel gave up on a split-K hand-over."""
    _check(lib().fls_check_workspace(_stream()), "fls_check_workspace")


def fls_forget(blob=None):
    lib().fls_forget(blob.data_ptr() if blob is not None else None)


def fls_dense_gemm(W, X, C, M, K, N):
    import torch

    assert W.is_cuda and W.dtype == torch.float16 and W.is_contiguous() and W.shape == (M, K)
    assert X.is_cuda and X.dtype == torch.float16 and X.is_contiguous() and X.shape == (N, K)
    assert C.is_cuda and C.dtype == torch.float16 and C.is_contiguous() and C.shape == (N, M)
    _check(lib().fls_dense_gemm(W.data_ptr(), X.data_ptr(),
                                C.data_ptr(), M, K, N, _stream()), "fls_dense_gemm")
    return C


def scale_stride(K):
    """Scales to a row of K quantised values: one for each 128, up to a multiple of four."""
    return (K + 511) // 512 * 4


def fls_quantize(W, out=None):
    """W: float16 [M, K] CUDA tensor, K a multiple of 16.  Returns (Wq float8_e4m3fn [M, K], Ws float8_e8m0fnu [M, scale_stride(K)])."""
    import torch

    assert W.is_cuda and W.dtype == torch.float16 and W.is_contiguous() and W.dim() == 2
    M, K = W.shape
    if out is None:
        Wq = torch.empty_like(W, dtype=torch.float8_e4m3fn)
        Ws = W.new_empty((M, scale_stride(K)), dtype=torch.float8_e8m0fnu)
    else:
        Wq, Ws = out
        assert Wq.is_cuda and Wq.dtype == torch.float8_e4m3fn and Wq.is_contiguous() and Wq.shape == (M, K)
        assert Ws.is_cuda and Ws.dtype == torch.float8_e8m0fnu and Ws.is_contiguous() and Ws.shape == (M, scale_stride(K))
    stream = _stream()
    assert not _several_devices or _on_this_device(W, Wq, Ws)
    rc = lib().fls_quantize(W.data_ptr(), M, K, Wq.data_ptr(), Ws.data_ptr(), stream)
    if rc != OK:
        _check(rc, "fls_quantize")
    return Wq, Ws


def fls_fp8_workspace_bytes(M, K, N):
    return int(lib().fls_fp8_workspace_bytes(M, K, N))


def _on_this_device(*tensors):
    """Called where there are several devices: that of the stream has to be the tensors'."""
    import torch

    device = torch.cuda.current_device()
    return all(t.get_device() == device for t in tensors)


def _check_devices(*tensors):
    """That, and the workspace's: there is one."""
    assert _on_this_device(*tensors)
    if _ws_tensor is not None and not _on_this_device(_ws_tensor):
        raise FlsError(EWORKSPACE, "the workspace is another device's")


def ensure_fp8_workspace(M, K, N):
    """ensure_workspace for fls_fp8_gemm; not while a graph is recorded, unless it is large enough already."""
    need = lib().fls_fp8_workspace_bytes(M, K, N)
    if need == 0 or _ws_tensor is None or _ws_tensor.numel() < need:
        _ensure(need, "fls_fp8_workspace_bytes")


def _fp8_args(Wq, Ws, X, C, M, K, N):
    import torch

    assert Wq.is_cuda and Wq.dtype == torch.float8_e4m3fn and Wq.is_contiguous() and Wq.shape == (M, K)
    assert Ws.is_cuda and Ws.dtype == torch.float8_e8m0fnu and Ws.is_contiguous() and Ws.shape == (M, scale_stride(K))
    assert X.is_cuda and X.dtype == torch.float16 and X.is_contiguous() and X.shape == (N, K)
    assert C.is_cuda and C.dtype == torch.float16 and C.is_contiguous() and C.shape == (N, M)
    stream = _stream()
    if _several_devices:
        _check_devices(Wq, Ws, X, C)
    return Wq.data_ptr(), Ws.data_ptr(), X.data_ptr(), C.data_ptr(), M, K, N, stream


def fls_fp8_gemm(Wq, Ws, X, C, M, K, N):
    """C = W . X with W as fls_quantize returned it; X float16 [N, K], C float16 [N, M] as everywhere."""
    rc = lib().fls_fp8_gemm(*_fp8_args(Wq, Ws, X, C, M, K, N))
    if rc != OK:
        _check(rc, "fls_fp8_gemm")
    return C


def prepare_fp8_gemm(Wq, Ws, X, C, M, K, N):
    """As prepare_spmm, for fls_fp8_gemm."""
    f, args = lib().fls_fp8_gemm, _fp8_args(Wq, Ws, X, C, M, K, N)
    keep = (Wq, Ws, X, C)

    def call(_keep=keep):
        rc = f(*args)
        if rc != OK:
            _check(rc, "fls_fp8_gemm")

    return call


_ATTENTION_LAYOUT = struct.Struct("<10q4i2qf4x")  # fls_attention_shape
_pack_attention = _ATTENTION_LAYOUT.pack


def _attention_workspace_bytes(q_rows, heads, dim, k_rows, kv_heads, sequences, max_q, max_k):
    # strides do not matter here
    return lib().fls_attention_workspace_bytes(_pack_attention(q_rows, k_rows, 0, 0, 0, 0, 0, 0, heads * dim, dim, sequences, heads, kv_heads, dim, max_q, max_k, 1.0))


def fls_attention_workspace_bytes(Q, K, sequences, max_q, max_k):
    return int(_attention_workspace_bytes(*Q.shape, *K.shape[:2], sequences, max_q, max_k))


def ensure_attention_workspace(Q, K, q_start, max_q, max_k):
    """ensure_workspace for fls_attention; not while a graph is recorded, unless it is large enough already."""
    need = _attention_workspace_bytes(*Q.shape, *K.shape[:2], q_start.shape[0] - 1, max_q, max_k)
    if need == 0 or _ws_tensor is None or _ws_tensor.numel() < need:
        _ensure(need, "fls_attention_workspace_bytes")


def _attention_args(Q, K, V, O, q_start, k_start, k_len, max_q, max_k, scale, lse):
    import torch

    f16, i32 = torch.float16, torch.int32
    q_rows, heads, dim = shape = Q.shape
    k_rows, kv_heads, k_dim = k_shape = K.shape
    (q0, q1, q2), (k0, k1, k2), (v0, v1, v2), (o0, o1, o2) = Q.stride(), K.stride(), V.stride(), O.stride()
    sequences = k_len.shape[0]
    assert Q.is_cuda and K.is_cuda and V.is_cuda and O.is_cuda and Q.dtype == f16 and K.dtype == f16 and V.dtype == f16 and O.dtype == f16
    assert k_dim == dim and V.shape == k_shape and O.shape == shape and q2 == k2 == v2 == o2 == 1
    assert q_start.is_cuda and k_start.is_cuda and k_len.is_cuda and q_start.dtype == i32 and k_start.dtype == i32 and k_len.dtype == i32
    assert q_start.shape == (sequences + 1,) and k_start.shape == k_len.shape == (sequences,) and q_start.is_contiguous() and k_start.is_contiguous() and k_len.is_contiguous()
    if lse is not None:
        assert lse.is_cuda and lse.dtype == torch.float32 and lse.shape == (heads, q_rows) and lse.is_contiguous()
    stream = _stream()
    if _several_devices:
        _check_devices(Q, K, V, O, q_start, k_start, k_len, Q if lse is None else lse)
    if q_rows <= 1:  # the stride of one row or one head says nothing
        q0 = o0 = 0
    if k_rows <= 1:
        k0 = v0 = 0
    if heads == 1:
        q1 = o1 = 0
    if kv_heads == 1:
        k1 = v1 = 0
    return (Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), None if lse is None else lse.data_ptr(), q_start.data_ptr(), k_start.data_ptr(), k_len.data_ptr(),
            _pack_attention(q_rows, k_rows, q0, q1, k0, k1, v0, v1, o0, o1, sequences, heads, kv_heads, dim, max_q, max_k, scale), stream)


def fls_attention(Q, K, V, O, q_start, k_start, k_len, max_q, max_k, scale, lse=None):
    """Causal attention of packed sequences: Q, O float16 [rows, heads, head_dim], K, V float16 [rows, kv_heads, head_dim], any strides but a last
    one of 1 - slices of the QKV product's C, a cache.  q_start int32 [sequences + 1], k_start and k_len int32 [sequences], on the GPU: sequence b has
    queries q_start[b] ... q_start[b + 1] - 1 and k_len[b] keys from row k_start[b] on, its last query sees all of them.  max_q, max_k: the most queries and
    keys that a sequence has, or more.  lse: float32 [heads, rows] or None."""
    rc = lib().fls_attention(*_attention_args(Q, K, V, O, q_start, k_start, k_len, max_q, max_k, scale, lse))
    if rc != OK:
        _check(rc, "fls_attention")
    return O


def prepare_attention(Q, K, V, O, q_start, k_start, k_len, max_q, max_k, scale, lse=None):
    """As prepare_spmm, for fls_attention; the lengths are read when the call runs."""
    f, args = lib().fls_attention, _attention_args(Q, K, V, O, q_start, k_start, k_len, max_q, max_k, scale, lse)
    keep = (Q, K, V, O, q_start, k_start, k_len, lse)

    def call(_keep=keep):
        rc = f(*args)
        if rc != OK:
            _check(rc, "fls_attention")

    return call
