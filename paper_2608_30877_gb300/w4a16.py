"""Thin Python binding of libw4a16.so (include/w4a16.h).

Argument marshalling only: torch tensors supply device memory and the
current CUDA stream; every step of the computation runs in the library's
kernels.  There is no fallback -- if the library is not built or the GPU is
missing, the call raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import re
import weakref

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
# W4A16_DEBUG=1 loads the build with the kernels' index checks
LIB_PATH = os.path.join(_PKG, "libw4a16_debug.so" if os.environ.get("W4A16_DEBUG") == "1"
                        else "libw4a16.so")
HEADER = os.path.join(os.path.dirname(_PKG), "include", "w4a16.h")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_ALIGNMENT, ERR_CUDA, ERR_TIMEOUT, ERR_INDEX, \
    ERR_CAPACITY = range(8)
ACT_NONE, ACT_SWIGLU, ACT_GELU = range(3)
NORM_RMS, NORM_LAYER = range(2)
ROTARY_HALF, ROTARY_PAIRS = range(2)
ROTARY_SCALE_NONE, ROTARY_SCALE_LINEAR, ROTARY_SCALE_BY_TURNS, ROTARY_SCALE_BY_INDEX = range(4)

_lib = None
_caches = weakref.WeakSet()  # whose own workspaces an error may have left in use


class W4A16Error(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn} failed: {status_string(status)} (status {status})")


class Layer(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("w_packed", ctypes.c_void_p),
                ("scales", ctypes.c_void_p), ("out", ctypes.c_void_p),
                ("N", ctypes.c_int64), ("K", ctypes.c_int64)]


class KVCacheStruct(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("pages", "exponents", "page_table", "seq_len",
                                               "page_refs", "scratch")] + \
               [(n, ctypes.c_int64) for n in ("layers", "num_pages", "kv_heads", "page_tokens",
                                              "head_dim", "num_slots", "max_pages", "kv_bits")]


def header_functions() -> list[str]:
    """Names of the functions include/w4a16.h declares."""
    text = open(HEADER).read()
    return sorted(set(re.findall(r"^\s*(?:const\s+)?\w[\w\s\*]*?\b(w4a16_\w+)\s*\(", text, re.M)))


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run `python -c 'import __graft_entry__ as g; "
                               "g.build()'` first (needs nvcc)")
        L = ctypes.CDLL(LIB_PATH)
        i64, p = ctypes.c_int64, ctypes.c_void_p
        L.w4a16_linear.argtypes = [p, p, p, p, i64, i64, i64, i64, p]
        L.w4a16_linear_fused.argtypes = [p, p, p, p, p, p, i64, i64, i64, i64, ctypes.c_int, p]
        L.w4a16_linear_stack.argtypes = [ctypes.POINTER(Layer), i64, i64, i64, p]
        L.w4a16_dequant.argtypes = [p, p, p, i64, i64, i64, p]
        L.w4a16_stack_graph_create.argtypes = [ctypes.POINTER(Layer), i64, i64, i64,
                                               ctypes.POINTER(ctypes.c_void_p)]
        L.w4a16_stack_graph_launch.argtypes = [p, p]
        L.w4a16_stack_graph_destroy.argtypes = [p]
        L.w4a16_gather_rows.argtypes = [p, i64, i64, p, i64, p, p]
        L.w4a16_attention_prefill.argtypes = [p, p, i64, i64, i64, i64, i64, p, p]
        L.w4a16_attention_zero_outside.argtypes = [p, i64, i64, i64, i64, p, p]
        L.w4a16_topk_smallest.argtypes = [p, ctypes.c_int, i64, i64, p, p, p]
        L.w4a16_quantize.argtypes = [p, p, p, i64, i64, i64, p]
        kv = ctypes.POINTER(KVCacheStruct)
        L.w4a16_kv_scratch_bytes.argtypes = [i64, i64]
        L.w4a16_kv_scratch_bytes.restype = i64
        L.w4a16_kv_extend.argtypes = [kv, p, p, i64, p]
        L.w4a16_kv_fork.argtypes = [kv, p, p, i64, p]
        L.w4a16_kv_trim.argtypes = [kv, p, p, i64, p]
        L.w4a16_kv_compact.argtypes = [kv, p]
        L.w4a16_kv_write.argtypes = [kv, i64, p, p, p, i64, i64, i64, p]
        L.w4a16_attention_decode.argtypes = [kv, i64, p, p, i64, i64, i64, p, p, p]
        L.w4a16_attention_decode_workspace.argtypes = [i64, i64, ctypes.POINTER(i64)]
        i32, f32, f64 = ctypes.c_int, ctypes.c_float, ctypes.c_double
        L.w4a16_residual_norm.argtypes = [p, i32, p, p, i64, p, p, p, p, i64, i64, i32, f32, f32, f32, p, p, p]
        L.w4a16_rotary_table.argtypes = [i64, f64, i32, f64, i64, f64, f64, p]
        L.w4a16_rotary.argtypes = [p, p, p, i64, i64, i64, i64, i64, p, i64, i32, f32, p]
        L.w4a16_kv_rotary.argtypes = [kv, p, p, p, i64, i64, i64, p, i64, i32, f32, p]
        L.w4a16_log_probs.argtypes = [p, i32, i64, i64, i64, p, i64, p, p, p, p, p]
        L.w4a16_add_adapters.argtypes = [p, p, p, p, i64, p, p, i64, i64, i64, i64, i64, p, p, p, p]
        L.w4a16_add_adapters_workspace.argtypes = [i64, i64]
        L.w4a16_add_adapters_workspace.restype = i64
        L.w4a16_get_device_error.argtypes = [p]
        L.w4a16_selftest_wait_timeout.argtypes = [i64, p]
        L.w4a16_selftest_set_wait_limit.argtypes = [i64]
        L.w4a16_selftest_route.argtypes = [i64, i64, i64, i64, ctypes.c_int, ctypes.c_int,
                                           ctypes.POINTER(ctypes.c_int32)]
        L.w4a16_status_string.argtypes = [ctypes.c_int]
        L.w4a16_status_string.restype = ctypes.c_char_p
        L.w4a16_version.restype = ctypes.c_int
        for f in ("w4a16_linear", "w4a16_linear_fused", "w4a16_linear_stack",
                  "w4a16_gather_rows", "w4a16_topk_smallest", "w4a16_attention_prefill",
                  "w4a16_attention_zero_outside", "w4a16_stack_graph_create", "w4a16_stack_graph_launch",
                  "w4a16_stack_graph_destroy", "w4a16_dequant", "w4a16_quantize",
                  "w4a16_kv_extend", "w4a16_kv_fork", "w4a16_kv_trim", "w4a16_kv_compact",
                  "w4a16_kv_write", "w4a16_attention_decode", "w4a16_attention_decode_workspace",
                  "w4a16_residual_norm", "w4a16_rotary_table", "w4a16_rotary", "w4a16_kv_rotary",
                  "w4a16_log_probs", "w4a16_add_adapters",
                  "w4a16_get_device_error", "w4a16_selftest_wait_timeout",
                  "w4a16_selftest_set_wait_limit", "w4a16_selftest_route"):
            getattr(L, f).restype = ctypes.c_int
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().w4a16_status_string(int(status)).decode()


def version() -> int:
    return int(lib().w4a16_version())


# The current stream's handle alone takes 0.3 us, a Stream object for it 2.9; the
# function is not public, so a torch without it goes by the object.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)


def _check(fn: str, rc: int):
    if rc != OK:
        raise W4A16Error(fn, rc)


def _need_cuda(*ts):
    for t in ts:
        if not (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous()):
            raise ValueError("expected contiguous CUDA tensors")


def linear(x: torch.Tensor, w_packed: torch.Tensor, scales: torch.Tensor, g: int = 128,
           out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """out[M, N] = x[M, K] @ dequant(w_packed[N, K/2], scales[N, K/g])^T, bf16."""
    M, K = x.shape
    N = w_packed.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=x.device)
    _need_cuda(x, w_packed, scales, out)
    assert x.dtype == torch.bfloat16 and w_packed.dtype == torch.uint8
    assert scales.dtype == torch.bfloat16 and out.dtype == torch.bfloat16
    assert w_packed.shape[1] * 2 == K and scales.shape == (N, K // g) and out.shape == (M, N)
    _check("w4a16_linear", lib().w4a16_linear(x.data_ptr(), w_packed.data_ptr(), scales.data_ptr(),
                                              out.data_ptr(), M, N, K, g, _stream(stream)))
    return out


def linear_fused(x: torch.Tensor, w_packed: torch.Tensor, scales: torch.Tensor, g: int = 128,
                 act: int = ACT_NONE, bias: torch.Tensor | None = None,
                 residual: torch.Tensor | None = None, out: torch.Tensor | None = None,
                 stream=None) -> torch.Tensor:
    """out = act(x @ dequant(w)^T + bias) + residual (include/w4a16.h); for
    ACT_SWIGLU rows (2j, 2j+1) of w are (gate, up) and out has N/2 columns."""
    M, K = x.shape
    N = w_packed.shape[0]
    n_out = N // 2 if act == ACT_SWIGLU else N
    if out is None:
        out = torch.empty((M, n_out), dtype=torch.bfloat16, device=x.device)
    _need_cuda(x, w_packed, scales, out, *(t for t in (bias, residual) if t is not None))
    _check("w4a16_linear_fused", lib().w4a16_linear_fused(
        x.data_ptr(), w_packed.data_ptr(), scales.data_ptr(),
        None if bias is None else bias.data_ptr(),
        None if residual is None else residual.data_ptr(),
        out.data_ptr(), M, N, K, g, int(act), _stream(stream)))
    return out


def linear_raw(x_ptr: int, w_ptr: int, s_ptr: int, out_ptr: int, M: int, N: int, K: int, g: int,
               stream: int) -> int:
    """Direct call with raw pointers; returns the status code."""
    return lib().w4a16_linear(x_ptr, w_ptr, s_ptr, out_ptr, M, N, K, g, stream)


def linear_stack(layers, M: int, g: int = 128, stream=None) -> None:
    """layers: sequence of (x, w_packed, scales, out) tensors, run in order."""
    arr = (Layer * len(layers))()
    for i, (x, w, s, o) in enumerate(layers):
        _need_cuda(x, w, s, o)
        arr[i] = Layer(x.data_ptr(), w.data_ptr(), s.data_ptr(), o.data_ptr(), w.shape[0],
                       w.shape[1] * 2)
    _check("w4a16_linear_stack", lib().w4a16_linear_stack(arr, len(layers), M, g, _stream(stream)))


def make_layer_array(layers) -> ctypes.Array:
    """Pre-built Layer array for repeated w4a16_linear_stack calls."""
    arr = (Layer * len(layers))()
    for i, (x, w, s, o) in enumerate(layers):
        arr[i] = Layer(x.data_ptr(), w.data_ptr(), s.data_ptr(), o.data_ptr(), w.shape[0],
                       w.shape[1] * 2)
    return arr


class StackGraph:
    """A layer stack captured as a CUDA graph (include/w4a16.h); replay with
    launch(), release with close() (or as a context manager)."""

    def __init__(self, layers, M: int, g: int = 128):
        self._arr = make_layer_array(layers)
        self._h = ctypes.c_void_p()
        _check("w4a16_stack_graph_create", lib().w4a16_stack_graph_create(
            self._arr, len(self._arr), M, g, ctypes.byref(self._h)))

    def launch(self, stream=None):
        _check("w4a16_stack_graph_launch", lib().w4a16_stack_graph_launch(self._h, _stream(stream)))

    def close(self):
        if self._h:
            _check("w4a16_stack_graph_destroy", lib().w4a16_stack_graph_destroy(self._h))
            self._h = ctypes.c_void_p()

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


def linear_stack_array(arr: ctypes.Array, M: int, g: int = 128, stream=None) -> None:
    _check("w4a16_linear_stack", lib().w4a16_linear_stack(arr, len(arr), M, g, _stream(stream)))


def attention_prefill(qkv: torch.Tensor, seq_start: torch.Tensor, H: int, window: int = 32768,
                      out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Causal sliding-window attention over packed sequences (include/w4a16.h):
    qkv bf16 [M, 3 H 128], seq_start int32 [nseq + 1] -> out bf16 [M, H 128]."""
    M = qkv.shape[0]
    d = qkv.shape[1] // (3 * H)
    fresh = out is None
    if fresh:
        out = torch.empty((M, H * d), dtype=torch.bfloat16, device=qkv.device)
    _need_cuda(qkv, seq_start, out)
    assert qkv.dtype == torch.bfloat16 and seq_start.dtype == torch.int32
    _check("w4a16_attention_prefill", lib().w4a16_attention_prefill(
        qkv.data_ptr(), seq_start.data_ptr(), seq_start.shape[0] - 1, M, H, d, int(window),
        out.data_ptr(), _stream(stream)))
    if fresh:  # tokens outside every sequence are zero
        _check("w4a16_attention_zero_outside", lib().w4a16_attention_zero_outside(
            seq_start.data_ptr(), seq_start.shape[0] - 1, M, H, d, out.data_ptr(), _stream(stream)))
    return out


def gather_rows(src: torch.Tensor, index: torch.Tensor, out=None, stream=None) -> torch.Tensor:
    """dst[p] = src[index[p]] for bf16 rows; index int32 (include/w4a16.h)."""
    rows, D = src.shape
    P = index.shape[0]
    if out is None:
        out = torch.empty((P, D), dtype=torch.bfloat16, device=src.device)
    _need_cuda(src, index, out)
    assert src.dtype == torch.bfloat16 and index.dtype == torch.int32
    _check("w4a16_gather_rows", lib().w4a16_gather_rows(src.data_ptr(), rows, D, index.data_ptr(),
                                                        P, out.data_ptr(), _stream(stream)))
    return out


def topk_smallest(scores: torch.Tensor, k: int, stream=None):
    """(int32 indices [k], fp32 scores [k]) of the k smallest scores (fp32 or
    bf16), ascending by totalOrder, NaN last, ties by index."""
    n = scores.shape[0]
    _need_cuda(scores)
    bits = {torch.float32: 32, torch.bfloat16: 16}[scores.dtype]
    idx = torch.empty(k, dtype=torch.int32, device=scores.device)
    val = torch.empty(k, dtype=torch.float32, device=scores.device)
    _check("w4a16_topk_smallest", lib().w4a16_topk_smallest(
        scores.data_ptr(), bits, n, k, idx.data_ptr(), val.data_ptr(), _stream(stream)))
    return idx, val


def dequant(w_packed: torch.Tensor, scales: torch.Tensor, g: int = 128, out=None,
            stream=None) -> torch.Tensor:
    N, K2 = w_packed.shape
    K = 2 * K2
    if out is None:
        out = torch.empty((N, K), dtype=torch.bfloat16, device=w_packed.device)
    _need_cuda(w_packed, scales, out)
    _check("w4a16_dequant", lib().w4a16_dequant(w_packed.data_ptr(), scales.data_ptr(),
                                                out.data_ptr(), N, K, g, _stream(stream)))
    return out


def quantize(w: torch.Tensor, g: int = 128, stream=None):
    """fp32 [N, K] (CUDA) -> (packed uint8 [N, K/2], scales bf16 [N, K/g])."""
    N, K = w.shape
    _need_cuda(w)
    assert w.dtype == torch.float32
    packed = torch.empty((N, K // 2), dtype=torch.uint8, device=w.device)
    scales = torch.empty((N, K // g), dtype=torch.bfloat16, device=w.device)
    _check("w4a16_quantize", lib().w4a16_quantize(w.data_ptr(), packed.data_ptr(),
                                                  scales.data_ptr(), N, K, g, _stream(stream)))
    return packed, scales


def _allocating_on(stream):
    """Context in which torch allocates (and fills) for use on `stream`."""
    if stream is None:
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(_stream(stream))
    return torch.cuda.stream(stream)


class KVCache:
    """A paged key-value cache (include/w4a16.h): the tensors and the handle that the kv_*
    functions and attention_decode take.  dtype torch.bfloat16, or torch.float8_e4m3fn with
    a power-of-two exponent for each token's key and value of a head.  Calls on one cache
    are ordered by the caller, who keeps it until they, and graphs with them, have run."""

    def __init__(self, layers: int, num_pages: int, kv_heads: int, num_slots: int, max_pages: int,
                 page_tokens: int = 64, dtype=torch.bfloat16, head_dim: int = 128, device="cuda"):
        i32 = {"dtype": torch.int32, "device": device}
        e4m3 = dtype == torch.float8_e4m3fn
        self._bind(torch.empty((layers, 2, num_pages, kv_heads, page_tokens, head_dim), dtype=dtype,
                               device=device),
                   torch.zeros((num_slots, max_pages), **i32), torch.zeros(num_slots, **i32),
                   torch.zeros(num_pages, **i32),
                   torch.empty((layers, num_pages, kv_heads, page_tokens, 2), dtype=torch.uint8,
                               device=device) if e4m3 else None)

    @classmethod
    def from_tensors(cls, pages: torch.Tensor, page_table: torch.Tensor, seq_len: torch.Tensor,
                     page_refs: torch.Tensor, exponents: torch.Tensor | None = None) -> "KVCache":
        """A cache over tensors that the caller keeps (shapes as in include/w4a16.h)."""
        cache = cls.__new__(cls)
        cache._bind(pages, page_table, seq_len, page_refs, exponents)
        return cache

    def _bind(self, pages, page_table, seq_len, page_refs, exponents):
        given = (page_table, seq_len, page_refs) + (() if exponents is None else (exponents,))
        _need_cuda(pages, *given)
        if pages.dtype not in (torch.bfloat16, torch.float8_e4m3fn):
            raise ValueError("a cache's pages are torch.bfloat16 or torch.float8_e4m3fn")
        if pages.dim() != 6 or pages.shape[1] != 2 or page_table.dim() != 2:
            raise ValueError("expected pages [layers, 2, num_pages, kv_heads, page_tokens, head_dim] "
                             "and page_table [num_slots, max_pages]")
        layers, _, num_pages, kv_heads, page_tokens, head_dim = pages.shape
        num_slots, max_pages = page_table.shape
        if (any(t.dtype != torch.int32 for t in (page_table, seq_len, page_refs))
                or seq_len.shape != (num_slots,) or page_refs.shape != (num_pages,)):
            raise ValueError("expected int32 page_table, seq_len [num_slots] and page_refs [num_pages]")
        e4m3 = pages.dtype == torch.float8_e4m3fn
        if e4m3 != (exponents is not None) or (e4m3 and (
                exponents.dtype != torch.uint8
                or exponents.shape != (layers, num_pages, kv_heads, page_tokens, 2))):
            raise ValueError("exponents uint8 [layers, num_pages, kv_heads, page_tokens, 2] come with "
                             "pages in e4m3, and only with them")
        if any(t.device != pages.device for t in given):
            raise ValueError("a cache's tensors are on one device")
        self.pages, self.page_table, self.seq_len = pages, page_table, seq_len
        self.page_refs, self.exponents = page_refs, exponents
        self.layers, self.num_pages, self.kv_heads, self.page_tokens = layers, num_pages, kv_heads, page_tokens
        self.num_slots, self.max_pages = num_slots, max_pages
        size = lib().w4a16_kv_scratch_bytes(num_pages, num_slots)
        if size == 0:
            raise W4A16Error("w4a16_kv_scratch_bytes", ERR_UNSUPPORTED)
        self._workspace_bytes = {}
        self._scratch = torch.zeros(size, dtype=torch.uint8, device=pages.device)
        self._workspace = None  # for calls that name none
        if not torch.cuda.is_current_stream_capturing():
            self._workspace = self._largest_workspace()
            # (the first call may be on another stream)
            torch.cuda.current_stream(pages.device).synchronize()
        self._struct = KVCacheStruct(
            pages.data_ptr(), None if exponents is None else exponents.data_ptr(), page_table.data_ptr(),
            seq_len.data_ptr(), page_refs.data_ptr(), self._scratch.data_ptr(), layers, num_pages, kv_heads,
            page_tokens, head_dim, num_slots, max_pages, 8 if e4m3 else 16)
        self._ref = ctypes.byref(self._struct)
        _caches.add(self)

    def new_workspace(self, H: int, stream=None) -> torch.Tensor:
        """A workspace for attention_decode with H query heads, zeroed on `stream`."""
        with _allocating_on(stream):
            return torch.zeros(self.workspace_bytes(H), dtype=torch.uint8, device=self.pages.device)

    def _largest_workspace(self) -> torch.Tensor:
        """For any number of query heads: the size does not decrease with it."""
        return self.new_workspace(self.kv_heads * (65535 // self.kv_heads))

    def _own_workspace(self, H: int, stream) -> torch.Tensor:
        if self._workspace is None:  # the cache was made under capture
            with _allocating_on(stream):
                if torch.cuda.is_current_stream_capturing():
                    # zeroed by the graph whenever it runs, and no other call's
                    return self.new_workspace(H)
                self._workspace = self._largest_workspace()
                torch.cuda.current_stream(self.pages.device).synchronize()
        return self._workspace

    def workspace_bytes(self, H: int) -> int:
        if H not in self._workspace_bytes:
            size = ctypes.c_int64()
            _check("w4a16_attention_decode_workspace", lib().w4a16_attention_decode_workspace(
                H, self.kv_heads, ctypes.byref(size)))
            self._workspace_bytes[H] = size.value
        return self._workspace_bytes[H]


def _need_list(t: torch.Tensor, n: int | None = None) -> int:
    if not (t.is_cuda and t.dtype == torch.int32 and t.dim() == 1 and t.is_contiguous()
            and (n is None or t.shape[0] == n)):
        raise ValueError("expected contiguous int32 CUDA lists of one length")
    return t.shape[0]


def kv_extend(cache: KVCache, slots: torch.Tensor, add: torch.Tensor, stream=None) -> None:
    """Grows the sequences of `slots` by `add` tokens each (int32 lists): allocates pages, and
    copies a part-full last page that others share (include/w4a16.h)."""
    n = _need_list(slots)
    _need_list(add, n)
    _check("w4a16_kv_extend", lib().w4a16_kv_extend(cache._ref, slots.data_ptr(), add.data_ptr(), n,
                                                    _stream(stream)))


def kv_fork(cache: KVCache, parents: torch.Tensor, children: torch.Tensor, stream=None) -> None:
    """Gives the empty slots `children` the sequences of `parents`, sharing their pages."""
    n = _need_list(parents)
    _need_list(children, n)
    _check("w4a16_kv_fork", lib().w4a16_kv_fork(cache._ref, parents.data_ptr(), children.data_ptr(), n,
                                                _stream(stream)))


def kv_trim(cache: KVCache, slots: torch.Tensor, keep: torch.Tensor | None = None, stream=None) -> None:
    """Shortens the sequences of `slots` to `keep` tokens each; None frees them."""
    n = _need_list(slots)
    if keep is not None:
        _need_list(keep, n)
    _check("w4a16_kv_trim", lib().w4a16_kv_trim(cache._ref, slots.data_ptr(),
                                                None if keep is None else keep.data_ptr(), n,
                                                _stream(stream)))


def kv_compact(cache: KVCache, stream=None) -> None:
    """Moves the pages in use to the front of the pool."""
    _check("w4a16_kv_compact", lib().w4a16_kv_compact(cache._ref, _stream(stream)))


def _need_qkv(cache: KVCache, qkv: torch.Tensor, H: int) -> None:
    if not (qkv.is_cuda and qkv.dtype == torch.bfloat16 and qkv.dim() == 2 and qkv.is_contiguous()
            and qkv.shape[1] == (H + 2 * cache.kv_heads) * cache.pages.shape[5]):
        raise ValueError("expected a contiguous bf16 CUDA qkv [rows, (H + 2 kv_heads) * head_dim]")


def kv_write(cache: KVCache, layer: int, qkv: torch.Tensor, seq_start: torch.Tensor, slots: torch.Tensor,
             H: int, stream=None) -> None:
    """Stores the keys and values of a packed batch in one layer's pages: rows
    [seq_start[i], seq_start[i+1]) are the last tokens of slots[i]'s sequence."""
    _need_qkv(cache, qkv, H)
    n = _need_list(slots)
    _need_list(seq_start, n + 1)
    _check("w4a16_kv_write", lib().w4a16_kv_write(
        cache._ref, layer, qkv.data_ptr(), seq_start.data_ptr(), slots.data_ptr(), n, qkv.shape[0], H,
        _stream(stream)))


def attention_decode(cache: KVCache, layer: int, qkv: torch.Tensor, slots: torch.Tensor, H: int,
                     window: int = 32768, out: torch.Tensor | None = None,
                     workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Attention of one new token per sequence over the cache, its key and value stored
    (include/w4a16.h): qkv bf16 [n, (H + 2 kv_heads) 128], slots int32 [n] -> out bf16
    [n, H 128].  Without `workspace` the cache's own is used: calls on several streams at once
    need one each (KVCache.new_workspace)."""
    _need_qkv(cache, qkv, H)
    n = _need_list(slots, qkv.shape[0])
    if workspace is None:
        workspace = cache._own_workspace(H, stream)
    elif not (workspace.is_cuda and workspace.is_contiguous()
              and workspace.numel() * workspace.element_size() >= cache.workspace_bytes(H)):
        raise ValueError("expected a workspace of KVCache.new_workspace(H)")
    if out is None:
        if stream is None:
            out = torch.empty((n, H * 128), dtype=torch.bfloat16, device=qkv.device)
        else:
            with _allocating_on(stream):
                out = torch.empty((n, H * 128), dtype=torch.bfloat16, device=qkv.device)
    elif not (out.is_cuda and out.dtype == torch.bfloat16 and out.is_contiguous()
              and out.shape == (n, H * 128)):
        raise ValueError("expected a contiguous bf16 CUDA out [n, H * 128]")
    _check("w4a16_attention_decode", lib().w4a16_attention_decode(
        cache._ref, layer, qkv.data_ptr(), slots.data_ptr(), n, H, int(window), out.data_ptr(),
        workspace.data_ptr(), _stream(stream)))
    return out


# (what a call checks takes as long as a small kernel: one look at the current device, and shapes
# as they are)
def _fits(t, dtype, shape, device: int) -> bool:
    """A contiguous tensor of this type and shape on the device."""
    return t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.get_device() == device


def _device_of(t: torch.Tensor) -> int:
    """The tensor's device, which has to be the current one (the library launches there)."""
    device = t.get_device()
    if device < 0 or device != torch.cuda.current_device():
        raise ValueError("expected CUDA tensors on the current device")
    return device


def _stream_on(stream, device: int) -> int:
    if stream is None and _raw_stream is not None:
        return _raw_stream(device)
    return _stream(stream)


def _new(stream, shape, dtype, like) -> torch.Tensor:
    """An output, allocated on the stream that writes it.  (torch.empty 1.6 us, new_empty 2.9)"""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    with _allocating_on(stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


def _ptr(t):
    return None if t is None else t.data_ptr()


def residual_norm(residual: torch.Tensor, weight: torch.Tensor | None = None,
                  block: torch.Tensor | None = None, *, bias: torch.Tensor | None = None,
                  gate: torch.Tensor | None = None, post_weight: torch.Tensor | None = None,
                  post_bias: torch.Tensor | None = None, kind: int = NORM_RMS, eps: float = 1e-5,
                  weight_offset: float = 0.0, residual_scale: float = 1.0,
                  residual_out: torch.Tensor | None = None, out: torch.Tensor | None = None,
                  stream=None):
    """(out, h): h = residual_scale * residual + gate * post(block), out = norm of h
    (include/w4a16.h).  residual [M, D] bf16 or fp32, block bf16 [M, D], gate bf16 [1 or M, D], the
    weights and biases bf16 [D]; post(block) is block without post_weight.  residual_out may be
    residual.  Without block and residual_out h is not stored (None; residual itself where
    residual_scale is 1)."""
    bf16, shape, device = torch.bfloat16, residual.shape, _device_of(residual)
    M, D = shape
    vector = shape[1:]
    if not (_fits(residual, residual.dtype, shape, device) and (residual.dtype is bf16 or residual.dtype is torch.float32)):
        raise ValueError("expected a contiguous residual [M, D] in bf16 or fp32 on the current device")
    for t in (weight, bias, post_weight, post_bias):
        if t is not None and not _fits(t, bf16, vector, device):
            raise ValueError("expected contiguous bf16 weights and biases [D] on the current device")
    if block is not None and not _fits(block, bf16, shape, device):
        raise ValueError("expected a contiguous bf16 block [M, D] on the current device")
    if gate is not None and not (_fits(gate, bf16, (1, D), device) or _fits(gate, bf16, shape, device)):
        raise ValueError("expected a contiguous bf16 gate [1, D] or [M, D] on the current device")
    if residual_out is None:
        if block is not None:
            residual_out = _new(stream, shape, residual.dtype, residual)
    elif not _fits(residual_out, residual.dtype, shape, device):
        raise ValueError("expected residual_out like residual")
    if out is None:
        out = _new(stream, shape, bf16, residual)
    elif not _fits(out, bf16, shape, device):
        raise ValueError("expected a contiguous bf16 out [M, D] on the current device")
    _check("w4a16_residual_norm", lib().w4a16_residual_norm(
        residual.data_ptr(), 16 if residual.dtype is bf16 else 32, _ptr(block), _ptr(gate),
        0 if gate is None else gate.shape[0], _ptr(post_weight), _ptr(post_bias), _ptr(weight), _ptr(bias),
        M, D, kind, residual_scale, eps, weight_offset, _ptr(residual_out), out.data_ptr(),
        _stream_on(stream, device)))
    if residual_out is None and residual_scale == 1.0:
        residual_out = residual
    return out, residual_out


class RotaryTable:
    """Frequencies of rotary positions for the first rot_dim values of a head, on the device
    (include/w4a16.h).  attention_factor multiplies the turned queries and keys (for BY_INDEX
    usually 0.1 ln factor + 1)."""

    def __init__(self, rot_dim: int, base: float = 10000.0, scaling: int = ROTARY_SCALE_NONE,
                 factor: float = 1.0, trained_tokens: int = 0, low_turns: float = 1.0,
                 high_turns: float = 32.0, layout: int = ROTARY_HALF, attention_factor: float = 1.0,
                 device="cuda"):
        if layout not in (ROTARY_HALF, ROTARY_PAIRS):
            raise ValueError("layout is ROTARY_HALF or ROTARY_PAIRS")
        host = torch.zeros(max(rot_dim, 2) // 2, dtype=torch.int64)
        _check("w4a16_rotary_table", lib().w4a16_rotary_table(
            rot_dim, base, scaling, factor, trained_tokens, low_turns, high_turns, host.data_ptr()))
        self.rot_dim, self.layout, self.attention_factor = rot_dim, layout, float(attention_factor)
        self.turns = host.to(device)  # (from pageable memory: the copy has been made)


def _rotary_qkv(qkv: torch.Tensor, table: RotaryTable, columns: int, device: int) -> int:
    M = qkv.shape[0]
    if not _fits(qkv, torch.bfloat16, (M, columns), device):
        raise ValueError("expected a contiguous bf16 qkv [M, (H + 2 kv_heads) * head_dim] on the current device")
    if table.turns.get_device() != device:
        raise ValueError("the table is on another device")
    return M


def _sequences(M: int, seq_start, list_, device: int) -> int:
    """The number of sequences: of the table, or a row each; list_ has an entry for each."""
    if seq_start is None:
        nseq = M
    else:
        nseq = seq_start.shape[0] - 1
        if not _fits(seq_start, torch.int32, (nseq + 1,), device):
            raise ValueError("expected a contiguous int32 seq_start [nseq + 1] on the current device")
    if list_ is not None and not _fits(list_, torch.int32, (nseq,), device):
        raise ValueError("expected contiguous int32 lists with an entry for each sequence on the current device")
    return nseq


def rotary(qkv: torch.Tensor, table: RotaryTable, H: int, kv_heads: int | None = None,
           seq_start: torch.Tensor | None = None, first: torch.Tensor | None = None, head_dim: int = 128,
           stream=None) -> torch.Tensor:
    """Turns the queries and keys of qkv bf16 [M, (H + 2 kv_heads) head_dim] by their positions, in
    place (include/w4a16.h): row m of sequence s has position first[s] + m - seq_start[s] (int32 lists;
    without seq_start each row is a sequence, without first they begin at 0)."""
    if kv_heads is None:
        kv_heads = H
    device = _device_of(qkv)
    M = _rotary_qkv(qkv, table, (H + 2 * kv_heads) * head_dim, device)
    nseq = _sequences(M, seq_start, first, device)
    _check("w4a16_rotary", lib().w4a16_rotary(
        qkv.data_ptr(), _ptr(seq_start), _ptr(first), nseq, M, H, kv_heads, head_dim, table.turns.data_ptr(),
        table.rot_dim, table.layout, table.attention_factor, _stream_on(stream, device)))
    return qkv


def kv_rotary(cache: KVCache, qkv: torch.Tensor, slots: torch.Tensor, H: int, table: RotaryTable,
              seq_start: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The same with the positions that the cache's sequences have grown to: rows [seq_start[i],
    seq_start[i+1]) are the last tokens of slots[i]'s sequence (before kv_write), or without seq_start row i
    is the last one (before attention_decode)."""
    device = _device_of(qkv)
    M = _rotary_qkv(qkv, table, (H + 2 * cache.kv_heads) * 128, device)
    nseq = _sequences(M, seq_start, slots, device)
    if cache.pages.get_device() != device:
        raise ValueError("the cache is on another device")
    _check("w4a16_kv_rotary", lib().w4a16_kv_rotary(
        cache._ref, qkv.data_ptr(), _ptr(seq_start), slots.data_ptr(), nseq, M, H, table.turns.data_ptr(),
        table.rot_dim, table.layout, table.attention_factor, _stream_on(stream, device)))
    return qkv


def log_probs(logits: torch.Tensor, targets: torch.Tensor | None = None, k: int = 0, entropy: bool = True,
              stream=None):
    """(logp [M], entropy [M], index [M, k], score [M, k]) of logits [M, V] in bf16 or fp32, rows
    contiguous (include/w4a16.h): log probabilities of targets (int32 [M], -1: none, 0), the
    entropy, and the k largest logits' columns and log probabilities.  None where not asked for."""
    M, V = logits.shape
    device = _device_of(logits)
    bf16 = logits.dtype is torch.bfloat16
    if not (bf16 or logits.dtype is torch.float32) or (V > 1 and logits.stride(1) != 1):
        raise ValueError("expected logits [M, V] in bf16 or fp32 with contiguous rows on the current device")
    if targets is not None and not _fits(targets, torch.int32, (M,), device):
        raise ValueError("expected contiguous int32 targets [M] on the current device")
    f32 = torch.float32
    logp = None if targets is None else _new(stream, (M,), f32, logits)
    h = _new(stream, (M,), f32, logits) if entropy else None
    index = _new(stream, (M, k), torch.int32, logits) if k else None
    score = _new(stream, (M, k), f32, logits) if k else None
    _check("w4a16_log_probs", lib().w4a16_log_probs(
        logits.data_ptr(), 16 if bf16 else 32, M, V, logits.stride(0) if M > 1 else V, _ptr(targets), k, _ptr(logp),
        _ptr(h), _ptr(index), _ptr(score), _stream_on(stream, device)))
    return logp, h, index, score


def add_adapters(base: torch.Tensor, x: torch.Tensor, A: torch.Tensor, B: torch.Tensor, scale: torch.Tensor,
                 adapters: torch.Tensor, seq_start: torch.Tensor | None = None, out: torch.Tensor | None = None,
                 workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """out[m] = base[m] + scale[a] (x[m] A[a]^T) B[a]^T with a = adapters[s] of row m's sequence s
    (include/w4a16.h): x bf16 [M, K] and base bf16 [M, N], a projection's input and output; A bf16
    [pool, R, K], B bf16 [pool, N, R], scale fp32 [pool]; adapters int32 [nseq], -1 for none, and
    seq_start int32 [nseq + 1] (without it each row is a sequence; rows outside every sequence have no
    adapter).  out may be base.  Without `workspace` (adapters_workspace_bytes) one is allocated."""
    M, K = x.shape
    N = base.shape[1]
    pool, R = A.shape[0], A.shape[1]
    bf16, device = torch.bfloat16, _device_of(x)
    if not (_fits(x, bf16, (M, K), device) and _fits(base, bf16, (M, N), device)
            and _fits(A, bf16, (pool, R, K), device) and _fits(B, bf16, (pool, N, R), device)
            and _fits(scale, torch.float32, (pool,), device)):
        raise ValueError("expected contiguous bf16 x [M, K], base [M, N], A [pool, R, K], B [pool, N, R] and fp32 "
                         "scale [pool] on the current device")
    nseq = _sequences(M, seq_start, adapters, device)
    if workspace is None:
        workspace = _new(stream, (M, R), bf16, x)
    elif not (workspace.get_device() == device and workspace.is_contiguous()
              and workspace.numel() * workspace.element_size() >= adapters_workspace_bytes(M, R)):
        raise ValueError("expected a workspace of adapters_workspace_bytes")
    if out is None:
        out = _new(stream, (M, N), bf16, x)
    elif not _fits(out, bf16, (M, N), device):
        raise ValueError("expected a contiguous bf16 out [M, N] on the current device")
    _check("w4a16_add_adapters", lib().w4a16_add_adapters(
        x.data_ptr(), A.data_ptr(), B.data_ptr(), scale.data_ptr(), pool, _ptr(seq_start), adapters.data_ptr(),
        nseq, M, N, K, R, base.data_ptr(), out.data_ptr(), workspace.data_ptr(), _stream_on(stream, device)))
    return out


def adapters_workspace_bytes(M: int, R: int) -> int:
    """Bytes of a workspace for add_adapters; 0 for sizes that are not supported."""
    return lib().w4a16_add_adapters_workspace(M, R)


def selftest_wait_timeout(limit_ns: int, stream=None) -> None:
    """Launch the bounded-wait self test (see include/w4a16.h)."""
    _check("w4a16_selftest_wait_timeout",
           lib().w4a16_selftest_wait_timeout(int(limit_ns), _stream(stream)))


def set_wait_limit(limit_ns: int) -> None:
    """Wait limit of the kernels launched from now on (0: the default);
    test hook, see include/w4a16.h."""
    _check("w4a16_selftest_set_wait_limit", lib().w4a16_selftest_set_wait_limit(int(limit_ns)))


ROUTES = ("head", "rows", "stream", "gemm")


def route(M: int, N: int, K: int, g: int = 128, act: int = ACT_NONE, residual: bool = False):
    """(kernel of ROUTES, tokens per tile, CTAs per cluster, rows per CTA) that linear_fused
    runs with these arguments; test hook, see include/w4a16.h."""
    r = (ctypes.c_int32 * 4)()
    _check("w4a16_selftest_route", lib().w4a16_selftest_route(
        M, N, K, g, int(act), int(residual), r))
    return ROUTES[r[0]], r[1], r[2], r[3]


def get_device_error(stream=None) -> int:
    """Synchronises the stream, reads and clears the device status word.  After an error the
    caches' own workspaces are zeroed, which a call that gave up leaves in use (a workspace
    that the caller passes is the caller's to zero)."""
    rc = int(lib().w4a16_get_device_error(_stream(stream)))
    if rc != OK:  # (the word keeps the first error: any may hide a timeout)
        used = [c._workspace for c in list(_caches) if c._workspace is not None]
        if used and rc != ERR_CUDA:
            torch.cuda.synchronize()
            with _allocating_on(stream):
                for workspace in used:
                    workspace.zero_()
            torch.cuda.synchronize()
    return rc
