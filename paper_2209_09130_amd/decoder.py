"""ctypes binding of the decoder's entry points in include/samp.h (same names, argument marshalling only).

Every call runs on the current stream of its tensors' device, allocates its output (and workspace, where the C entry takes one) from
torch's allocator, and raises SampError for what the library refuses.  Activations are fp16 or bfloat16 tensors on the GPU.
"""
from __future__ import annotations

import ctypes as C
import functools
from typing import Optional, Tuple

import torch

from .binding import SampError, lib

_TYPES = {torch.float16: 0, torch.bfloat16: 1}
_P, _I, _L, _F, _Z = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
_SIGNATURES = {
    "samp_quantize_tokens": (_P, _L, _I, _I, _I, _P, _P, _P),
    "samp_gemm_i8_tokens_packed": (_P, _P, _P, _P, _P, _I, _P, _I, _I, _I, _I, _P),
    "samp_linear_i8_tokens_workspace_bytes": (_I, _I),
    "samp_linear_i8_tokens": (_P, _L, _I, _P, _P, _P, _I, _P, _I, _I, _I, _P, _Z, _P),
    "samp_cache_write": (_P, _P, _L, _P, _L, _I, _P, _I, _P, _P, _I, _I, _I, _P),
    "samp_cache_read": (_P, _P, _P, _I, _P, _I, _P, _P, _I, _I, _I, _P),
    "samp_attention_cache_workspace_bytes": (_I,) * 7,
    "samp_attention_cache": (_P, _L, _I, _I, _P, _P, _I, _P, _P, _I, _I, _I, _I, _F, _P, _P, _P, _Z, _P),
    "samp_attention_causal": (_P, _L, _P, _L, _P, _L, _I, _I, _I, _I, _P, _I, _I, _I, _F, _P, _P),
}
_entry = {}


def _fn(name: str):
    f = _entry.get(name)
    if f is None:
        f = getattr(lib(), name)
        f.argtypes, f.restype = _SIGNATURES[name], _Z if name.endswith("_bytes") else C.c_int
        _entry[name] = f
    return f


@functools.lru_cache(maxsize=4096)
def _workspace_bytes(name: str, *sizes: int) -> int:
    return _fn(name)(*sizes)


def _refuse(why: str):
    raise SampError(-1, why)


# ctypes passes the low 32 bits of a larger number without a word
_INT_MAX = 2 ** 31 - 1


def _most(n: int) -> int:
    """A maximum that the host counts with, which may be more than there is: one past int32 counts as that, one below zero is for the entry to refuse."""
    return max(-1, min(int(n), _INT_MAX))


def _device(t: torch.Tensor) -> int:
    if not t.is_cuda:
        _refuse(f"tensors must be on the GPU ({t.device})")
    return t.get_device()


def _elsewhere(t: torch.Tensor, device: int):
    _refuse(f"tensors on different devices: {t.device}, cuda:{device}")


def _flat(what: str, t: Optional[torch.Tensor], dtype: torch.dtype, device: int, size: Optional[int] = None) -> int:
    """The address of a contiguous tensor of one type (0 for None)."""
    if t is None:
        return 0
    if t.get_device() != device:
        _elsewhere(t, device)
    if t.dtype is not dtype or not t.is_contiguous() or (size is not None and t.numel() != size):
        _refuse(f"{what}: a contiguous {dtype} tensor{'' if size is None else f' of {size} elements'} is needed, not {t.dtype} {tuple(t.shape)} {t.stride()}")
    return t.data_ptr()


def _heads(what: str, t: torch.Tensor, device: int) -> Tuple[int, int]:
    """Address and row distance of [rows, heads, head_dim] whose heads lie next to each other."""
    if t.get_device() != device:
        _elsewhere(t, device)
    shape = t.shape
    if len(shape) != 3 or t.dtype not in _TYPES:
        _refuse(f"{what}: fp16 or bfloat16 [rows, heads, head_dim] is needed, not {t.dtype} {tuple(shape)}")
    rows, heads, dim = shape
    row, head, one = t.stride()
    if one != 1 or (head != dim and heads > 1):
        _refuse(f"{what}: the heads of a row must lie next to each other (strides {t.stride()})")
    return t.data_ptr(), row if rows > 1 else heads * dim


def _rows2(what: str, x: torch.Tensor) -> Tuple[int, int, int, int]:
    """Address, row distance, rows and width of a matrix with dense rows."""
    if x.dim() != 2 or x.dtype not in _TYPES or (x.stride(1) != 1 and x.shape[1] > 1):
        _refuse(f"{what}: an fp16 or bfloat16 matrix with dense rows is needed, not {x.dtype} {tuple(x.shape)} {x.stride()}")
    M, K = x.shape
    if M > _INT_MAX or K > _INT_MAX:
        _refuse(f"{what}: {M} x {K} is more than int32 counts")
    return x.data_ptr(), x.stride(0) if M > 1 else K, M, K


# torch.cuda.current_stream(device).cuda_stream and torch.cuda.current_device() without their objects; a call on another device than the current one is made again
# with that device current
_raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


def _on(device: int, f, *args, **kwargs):
    with torch.cuda.device(device):
        return f(*args, **kwargs)


def _raise(rc: int):
    raise SampError(rc, lib().samp_last_error().decode())


def quantize_tokens(x: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """samp_quantize_tokens: int8 codes [M, K] and float32 steps [M] of the rows of x (step = the row's absmax / 127)."""
    device = _device(x)
    if device != _current_device():
        return _on(device, quantize_tokens, x)
    at, ld, M, K = _rows2("x", x)
    codes, steps = x.new_empty((M, K), dtype=torch.int8), x.new_empty((M,), dtype=torch.float32)
    if M:
        rc = _fn("samp_quantize_tokens")(at, ld, _TYPES[x.dtype], M, K, codes.data_ptr(), steps.data_ptr(), _raw_stream(device))
        if rc:
            _raise(rc)
    return codes, steps


def gemm_i8_tokens_packed(codes: torch.Tensor, steps: torch.Tensor, Wp: torch.Tensor, s_w: torch.Tensor, bias: Optional[torch.Tensor] = None,
                          gelu: bool = False, dtype: torch.dtype = torch.float16) -> torch.Tensor:
    """samp_gemm_i8_tokens_packed: [M, N] of `dtype` from int8 codes [M, K] with a step for each row and weights that pack_weight_i8 packed, with a
    step for each channel."""
    device = _device(codes)
    if device != _current_device():
        return _on(device, gemm_i8_tokens_packed, codes, steps, Wp, s_w, bias, gelu, dtype)
    if codes.dim() != 2 or dtype not in _TYPES:
        _refuse("codes must be a matrix, and the result's type fp16 or bfloat16")
    M, K = codes.shape
    N = s_w.numel()
    c, st, w = _flat("codes", codes, torch.int8, device), _flat("steps", steps, torch.float32, device, M), _flat("Wp", Wp, torch.int8, device, N * K)
    sw, b = _flat("s_w", s_w, torch.float32, device), _flat("bias", bias, torch.float32, device, N)
    out = codes.new_empty((M, N), dtype=dtype)
    if M:
        rc = _fn("samp_gemm_i8_tokens_packed")(c, st, w, sw, b, int(bool(gelu)), out.data_ptr(), _TYPES[dtype], M, N, K, _raw_stream(device))
        if rc:
            _raise(rc)
    return out


def linear_i8_tokens(x: torch.Tensor, Wp: torch.Tensor, s_w: torch.Tensor, bias: Optional[torch.Tensor] = None, gelu: bool = False) -> torch.Tensor:
    """samp_linear_i8_tokens: quantize_tokens and gemm_i8_tokens_packed in one call, x [M, K] -> [M, N] of x's type."""
    device = _device(x)
    if device != _current_device():
        return _on(device, linear_i8_tokens, x, Wp, s_w, bias, gelu)
    at, ld, M, K = _rows2("x", x)
    N = s_w.numel()
    w, s, b = _flat("Wp", Wp, torch.int8, device, N * K), _flat("s_w", s_w, torch.float32, device), _flat("bias", bias, torch.float32, device, N)
    out = x.new_empty((M, N))
    if M:
        need = _workspace_bytes("samp_linear_i8_tokens_workspace_bytes", M, K)
        ws = x.new_empty((need,), dtype=torch.uint8) if need else None
        rc = _fn("samp_linear_i8_tokens")(at, ld, _TYPES[x.dtype], w, s, b, int(bool(gelu)), out.data_ptr(), M, N, K, ws.data_ptr() if need else 0, need,
                                          _raw_stream(device))
        if rc:
            _raise(rc)
    return out


class _CacheStruct(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k", "v", "k_step", "v_step")] + [(n, C.c_int32) for n in ("pages", "kv_heads", "page_len", "head_dim")]


class KVCache:
    """A paged int8 cache: codes k, v [pages, kv_heads, page_len, head_dim] and float32 steps k_step, v_step [pages, kv_heads, page_len] (contiguous,
    kept alive by this object), and the samp_kv_cache_t that points at them."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_step: torch.Tensor, v_step: torch.Tensor):
        device = _device(k)
        if k.dim() != 4 or v.shape != k.shape or k_step.shape != k.shape[:3] or v_step.shape != k.shape[:3]:
            _refuse(f"a cache is codes [pages, kv_heads, page_len, head_dim] and steps [pages, kv_heads, page_len], not {tuple(k.shape)} {tuple(v.shape)} "
                    f"{tuple(k_step.shape)} {tuple(v_step.shape)}")
        self.k, self.v, self.k_step, self.v_step = k, v, k_step, v_step
        self.device = device
        self.pages, self.kv_heads, self.page_len, self.head_dim = k.shape
        self.struct = _CacheStruct(_flat("k", k, torch.int8, device), _flat("v", v, torch.int8, device), _flat("k_step", k_step, torch.float32, device),
                                   _flat("v_step", v_step, torch.float32, device), *k.shape)
        self.address = C.addressof(self.struct)

    @classmethod
    def empty(cls, pages: int, kv_heads: int, page_len: int, head_dim: int, device="cuda") -> "KVCache":
        """A cache of zeros (what a sequence has not written is never seen)."""
        codes = [torch.zeros((pages, kv_heads, page_len, head_dim), dtype=torch.int8, device=device) for _ in range(2)]
        return cls(*codes, *(torch.zeros((pages, kv_heads, page_len), dtype=torch.float32, device=device) for _ in range(2)))


def _places(device: int, table: torch.Tensor, cu: Optional[torch.Tensor], lens: torch.Tensor):
    shape = table.shape
    if len(shape) != 2:
        _refuse("the page table is [sequences, pages of a sequence]")
    B, width = shape
    if B > _INT_MAX or width > _INT_MAX:
        _refuse(f"the page table: {B} x {width} is more than int32 counts")
    return (_flat("table", table, torch.int32, device), width, _flat("cu", cu, torch.int32, device, B + 1) if cu is not None else 0,
            _flat("lens", lens, torch.int32, device, B), B)


def cache_write(cache: KVCache, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, cu: Optional[torch.Tensor], lens: torch.Tensor, max_new: int) -> None:
    """samp_cache_write: the packed rows k, v [rows, kv_heads, head_dim] become the last cu[b + 1] - cu[b] of the lens[b] positions of each sequence.
    table int32 [B, width]; cu int32 [B + 1] or None (max_new rows each); lens int32 [B], the new positions counted."""
    device = cache.device
    if device != _current_device():
        return _on(device, cache_write, cache, k, v, table, cu, lens, max_new)
    (pk, ldk), (pv, ldv) = _heads("k", k, device), _heads("v", v, device)
    shape = k.shape
    if shape != v.shape or k.dtype is not v.dtype or shape[1] != cache.kv_heads or shape[2] != cache.head_dim:
        _refuse(f"k and v must be [rows, {cache.kv_heads}, {cache.head_dim}] of one type, not {tuple(k.shape)} and {tuple(v.shape)}")
    t, width, pcu, plens, B = _places(device, table, cu, lens)
    rows = shape[0]
    if rows and B:
        rc = _fn("samp_cache_write")(cache.address, pk, ldk, pv, ldv, _TYPES[k.dtype], t, width, pcu, plens, B, _most(max_new), rows, _raw_stream(device))
        if rc:
            _raise(rc)


def cache_read(cache: KVCache, table: torch.Tensor, cu: Optional[torch.Tensor], lens: torch.Tensor, max_rows: int, rows: int,
               dtype: torch.dtype = torch.float16, out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """samp_cache_read: k, v [rows, kv_heads, head_dim] of `dtype`, sequence b's rows the last cu[b + 1] - cu[b] of its lens[b] positions."""
    device = cache.device
    if device != _current_device():
        return _on(device, cache_read, cache, table, cu, lens, max_rows, rows, dtype, out)
    if dtype not in _TYPES:
        _refuse("the result's type must be fp16 or bfloat16")
    t, width, pcu, plens, B = _places(device, table, cu, lens)
    if out is None:
        out = cache.k.new_empty((2, rows, cache.kv_heads, cache.head_dim), dtype=dtype).unbind()
        k, v = out[0].data_ptr(), out[1].data_ptr()
    else:
        size = rows * cache.kv_heads * cache.head_dim
        k, v = _flat("out", out[0], dtype, device, size), _flat("out", out[1], dtype, device, size)
    if rows and B:
        rc = _fn("samp_cache_read")(cache.address, k, v, _TYPES[dtype], t, width, pcu, plens, B, _most(max_rows), rows, _raw_stream(device))
        if rc:
            _raise(rc)
    return out


def attention_cache(q: torch.Tensor, cache: KVCache, table: torch.Tensor, cu: Optional[torch.Tensor], lens: torch.Tensor, max_new: int,
                    max_len: Optional[int] = None, scale: Optional[float] = None, tree: Optional[torch.Tensor] = None,
                    out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """samp_attention_cache: [rows, heads, head_dim] of the new tokens q over the cache that holds their keys and values already.
    max_len: the longest context expected (None: what the page table has room for).  scale: None for 1 / sqrt(head_dim).  tree: int64 words [rows]."""
    device = cache.device
    if device != _current_device():
        return _on(device, attention_cache, q, cache, table, cu, lens, max_new, max_len, scale, tree, out)
    at, ld = _heads("q", q, device)
    rows, heads, dim = q.shape
    if dim != cache.head_dim:
        _refuse(f"q has heads of {dim}, the cache of {cache.head_dim}")
    t, width, pcu, plens, B = _places(device, table, cu, lens)
    words = _flat("tree", tree, torch.int64, device, rows) if tree is not None else 0
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        to = out.data_ptr()
    else:
        to = _flat("out", out, q.dtype, device, rows * heads * dim)
    if rows and B:
        max_new, max_len = _most(max_new), _most(width * cache.page_len if max_len is None else max_len)
        need = _workspace_bytes("samp_attention_cache_workspace_bytes", rows, B, heads, cache.kv_heads, dim, max_new, max_len)
        ws = q.new_empty((need,), dtype=torch.uint8) if need else None
        rc = _fn("samp_attention_cache")(at, ld, _TYPES[q.dtype], heads, cache.address, t, width, pcu, plens, B, max_new, max_len, rows,
                                         dim ** -0.5 if scale is None else float(scale), words, to, ws.data_ptr() if need else 0, need, _raw_stream(device))
        if rc:
            _raise(rc)
    return out


def attention_causal(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu: Optional[torch.Tensor], max_len: int, scale: Optional[float] = None,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """samp_attention_causal: [rows, heads, head_dim] from q [rows, heads, head_dim] and k, v [rows, kv_heads, head_dim] (views into a fused
    projection's rows are read in place).  cu int32 [B + 1], or None for sequences of max_len rows each."""
    device = _device(q)
    if device != _current_device():
        return _on(device, attention_causal, q, k, v, cu, max_len, scale, out)
    (pq, ldq), (pk, ldk), (pv, ldv) = _heads("q", q, device), _heads("k", k, device), _heads("v", v, device)
    (rows, heads, dim), shape, dtype = q.shape, k.shape, q.dtype
    if shape != v.shape or shape[0] != rows or shape[2] != dim or k.dtype is not dtype or v.dtype is not dtype:
        _refuse(f"q {tuple(q.shape)}, k {tuple(k.shape)} and v {tuple(v.shape)} do not belong together")
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        to = out.data_ptr()
    else:
        to = _flat("out", out, dtype, device, rows * heads * dim)
    if rows == 0:
        return out
    max_len = _most(max_len)
    if cu is not None:
        B, pcu = cu.numel() - 1, _flat("cu", cu, torch.int32, device)
    else:
        if max_len < 1 or rows % max_len:
            _refuse("without sequence offsets every sequence has max_len rows")
        B, pcu = rows // max_len, 0
    if B:
        rc = _fn("samp_attention_causal")(pq, ldq, pk, ldk, pv, ldv, _TYPES[dtype], heads, shape[1], dim, pcu, B, max_len, rows,
                                          dim ** -0.5 if scale is None else float(scale), to, _raw_stream(device))
        if rc:
            _raise(rc)
    return out
