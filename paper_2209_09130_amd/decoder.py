"""ctypes binding of the decoder's entry points in include/samp.h (same names, argument marshalling only).

Every call runs on the current stream of its tensors' device, allocates its output (and workspace, where the C entry takes one) from
torch's allocator, and raises SampError for what the library refuses.  Activations are fp16 or bfloat16 tensors on the GPU (logits float32 too).  Results of one
call may be parts of one allocation.
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
    "samp_beam_select_workspace_bytes": (_I,) * 5,
    "samp_beam_select": (_P, _L, _I, _P, _P, _I, _I, _I, _I, _I, _P, _P, _P, _P, _Z, _P),
    "samp_pages_fork_workspace_bytes": (_I,) * 4,
    "samp_pages_fork": (_P, _I, _P, _P, _I, _I, _I, _P, _P, _I, _I, _P, _P, _P, _P, _P, _P, _Z, _P),
    "samp_pages_compact_workspace_bytes": (_I, _I),
    "samp_pages_compact": (_P, _I, _P, _I, _I, _P, _P, _P, _P, _P, _Z, _P),
    "samp_cache_copy": (_P, _P, _P, _I, _P),
    "samp_cache_bounds": (_P, _P, _P, _I, _P, _P, _I, _I, _I, _P),
    "samp_cache_select_workspace_bytes": (_I,) * 3,
    "samp_cache_select": (_P, _L, _I, _I, _P, _P, _P, _I, _P, _P, _I, _I, _I, _I, _I, _I, _P, _P, _P, _Z, _P),
    "samp_attention_sparse_workspace_bytes": (_I,) * 10,
    "samp_attention_sparse": (_P, _L, _I, _I, _P, _P, _P, _I, _P, _P, _I, _I, _I, _I, _I, _I, _I, _F, _P, _P, _P, _Z, _P),
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


# ---- beam search and long contexts ---------------------------------------------------------------------
_LOGITS = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}


def beam_select(logits: torch.Tensor, scores: torch.Tensor, beams: int, keep: Optional[int] = None, finished: Optional[torch.Tensor] = None,
                end: int = 0) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """samp_beam_select: (scores float32, parents int32, tokens int32), each [batch, keep], the best first, of logits [batch * beams, vocabulary] (fp16, bfloat16 or
    float32, dense rows) and scores float32 [batch * beams].  parents are rows of logits, as pages_fork takes them; -1 behind the last candidate.
    keep: None for beams.  finished: bool or uint8 [batch * beams], rows that go on with `end` alone."""
    device = _device(logits)
    if device != _current_device():
        return _on(device, beam_select, logits, scores, beams, keep, finished, end)
    if logits.dim() != 2 or logits.dtype not in _LOGITS or (logits.stride(1) != 1 and logits.shape[1] > 1):
        _refuse(f"logits: a matrix of fp16, bfloat16 or float32 with dense rows is needed, not {logits.dtype} {tuple(logits.shape)} {logits.stride()}")
    rows, vocab = logits.shape
    keep = beams if keep is None else keep
    if not 1 <= beams <= 64 or rows % beams or not 1 <= keep <= 64 or vocab > _INT_MAX:
        _refuse(f"logits have rows of whole sequences, 1 to 64 beams each, and 1 to 64 candidates are kept ({rows} rows, {beams}, {keep})")
    if not -_INT_MAX <= end <= _INT_MAX:
        _refuse(f"end is an int32 ({end})")
    batch = rows // beams
    at = _flat("scores", scores, torch.float32, device, rows)
    done = 0
    if finished is not None:
        done = _flat("finished", finished, torch.bool if finished.dtype is torch.bool else torch.uint8, device, rows)
    best, parents, tokens = scores.new_empty((3, batch, keep)).unbind()
    parents, tokens = parents.view(torch.int32), tokens.view(torch.int32)
    if batch:
        need = _workspace_bytes("samp_beam_select_workspace_bytes", _LOGITS[logits.dtype], batch, beams, vocab, keep)
        ws = logits.new_empty((need,), dtype=torch.uint8) if need else None
        rc = _fn("samp_beam_select")(logits.data_ptr(), logits.stride(0) if rows > 1 else vocab, _LOGITS[logits.dtype], at, done, end, batch, beams, vocab, keep,
                                     best.data_ptr(), parents.data_ptr(), tokens.data_ptr(), ws.data_ptr() if need else 0, need, _raw_stream(device))
        if rc:
            _raise(rc)
    return best, parents, tokens


def _parts(like: torch.Tensor, sizes: Tuple[int, ...]) -> Tuple[torch.Tensor, ...]:
    """Flat results in one allocation (an allocation and a view take about as long as a call's checks)."""
    return torch.unsafe_split_with_sizes(like.new_empty(sum(sizes)), sizes)          # (views that autograd does not follow: 1.3 us for 1.7)


def _table(table: torch.Tensor, device: int) -> Tuple[int, int, int]:
    if table.dim() != 2 or table.numel() > _INT_MAX:
        _refuse(f"a page table is [sequences, pages of a sequence], of at most 2^30 entries, not {tuple(table.shape)}")
    return _flat("table", table, torch.int32, device), table.shape[0], table.shape[1]


def pages_fork(refs: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, page_len: int, parents: Optional[torch.Tensor] = None,
               cu: Optional[torch.Tensor] = None, max_new: int = 0) -> Tuple[torch.Tensor, ...]:
    """samp_pages_fork: (refs, table, lens, copies, lacking) of the sequences that continue rows `parents` (int32; None: each its own) of table int32 [rows, width], with
    room for their next cu[i + 1] - cu[i] positions (cu None: max_new).  refs int32 [pages]: table entries that name a page, 0 for a free one.  copies int32 [3, rows] is
    for cache_copy, on every cache that the table is for; lacking int32 [1]: pages that were not there."""
    device = _device(refs)
    if device != _current_device():
        return _on(device, pages_fork, refs, table, lens, page_len, parents, cu, max_new)
    pages = refs.numel()
    if pages > _INT_MAX:
        _refuse(f"{pages} pages are more than int32 counts")
    pr = _flat("refs", refs, torch.int32, device)
    pt, rows_from, width = _table(table, device)
    pl = _flat("lens", lens, torch.int32, device, rows_from)
    pp, rows = (0, rows_from) if parents is None else (_flat("parents", parents, torch.int32, device), parents.numel())
    pc = _flat("cu", cu, torch.int32, device, rows + 1) if cu is not None else 0
    if not 0 < rows <= 8192:
        _refuse(f"1 to 8192 rows are supported ({rows})")
    if rows * width > _INT_MAX:
        _refuse("a page table has at most 2^30 entries")
    refs_out, table_out, lens_out, copies, lacking = _parts(refs, (pages, rows * width, rows, 3 * rows, 1))
    need = _workspace_bytes("samp_pages_fork_workspace_bytes", pages, rows_from, width, rows)
    ws = refs.new_empty((need,), dtype=torch.uint8) if need else None
    rc = _fn("samp_pages_fork")(pr, pages, pt, pl, rows_from, width, _most(page_len), pp, pc, _most(max_new), rows, refs_out.data_ptr(), table_out.data_ptr(),
                                lens_out.data_ptr(), copies.data_ptr(), lacking.data_ptr(), ws.data_ptr() if need else 0, need, _raw_stream(device))
    if rc:
        _raise(rc)
    return refs_out, table_out.view(rows, width), lens_out, copies.view(3, rows), lacking


def pages_compact(refs: torch.Tensor, table: torch.Tensor, page_len: int) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """samp_pages_compact: (refs, table, copies, used) with the pages in use as the first `used` (int32 [1]).  table: int32 of any shape; copies for cache_copy, as from
    pages_fork."""
    device = _device(refs)
    if device != _current_device():
        return _on(device, pages_compact, refs, table, page_len)
    pages, entries = refs.numel(), table.numel()
    if pages > _INT_MAX or entries > _INT_MAX:
        _refuse(f"{pages} pages or {entries} entries are more than int32 counts")
    pr, pt = _flat("refs", refs, torch.int32, device), _flat("table", table, torch.int32, device)
    n = max(1, pages // 2)
    refs_out, table_out, copies, used = _parts(refs, (pages, entries, 3 * n, 1))
    need = _workspace_bytes("samp_pages_compact_workspace_bytes", pages, entries)
    ws = refs.new_empty((need,), dtype=torch.uint8) if need else None
    rc = _fn("samp_pages_compact")(pr, pages, pt, entries, _most(page_len), refs_out.data_ptr(), table_out.data_ptr(), copies.data_ptr(), used.data_ptr(),
                                   ws.data_ptr() if need else 0, need, _raw_stream(device))
    if rc:
        _raise(rc)
    return refs_out, table_out.view(table.shape), copies.view(3, n), used


class _BoundsStruct(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("steps", C.c_void_p)]


class KeyBounds:
    """Bounds of the keys of a cache's pages: codes int8 [pages, kv_heads, 2, head_dim] (largest, smallest) and float32 steps [pages, kv_heads] (contiguous, kept alive by
    this object), and the samp_key_bounds_t that points at them."""

    def __init__(self, codes: torch.Tensor, steps: torch.Tensor):
        device = _device(codes)
        if codes.dim() != 4 or codes.shape[2] != 2 or steps.shape != codes.shape[:2]:
            _refuse(f"bounds are codes [pages, kv_heads, 2, head_dim] and steps [pages, kv_heads], not {tuple(codes.shape)} {tuple(steps.shape)}")
        self.codes, self.steps = codes, steps
        self.device = device
        self.struct = _BoundsStruct(_flat("codes", codes, torch.int8, device), _flat("steps", steps, torch.float32, device))
        self.address = C.addressof(self.struct)
        self.sizes = (codes.shape[0], codes.shape[1], codes.shape[3])

    @classmethod
    def empty(cls, cache: KVCache) -> "KeyBounds":
        """Bounds for a cache, none of them written."""
        return cls(cache.k.new_zeros((cache.pages, cache.kv_heads, 2, cache.head_dim)), cache.k_step.new_zeros((cache.pages, cache.kv_heads)))

    def of(self, cache: KVCache) -> int:
        if self.device != cache.device or self.sizes != (cache.pages, cache.kv_heads, cache.head_dim):
            _refuse(f"bounds for {self.sizes} (pages, kv_heads, head_dim) are not those of a cache of {(cache.pages, cache.kv_heads, cache.head_dim)}")
        return self.address


def cache_copy(cache: KVCache, copies: torch.Tensor, bounds: Optional[KeyBounds] = None) -> None:
    """samp_cache_copy: for every column (from, to, positions) of copies int32 [3, n] the first positions of page `from` become those of page `to`."""
    device = cache.device
    if device != _current_device():
        return _on(device, cache_copy, cache, copies, bounds)
    if copies.dim() != 2 or copies.shape[0] != 3 or copies.shape[1] > _INT_MAX:
        _refuse(f"copies are int32 [3, n], not {tuple(copies.shape)}")
    n = copies.shape[1]
    at, kb = _flat("copies", copies, torch.int32, device), bounds.of(cache) if bounds is not None else 0
    if n:
        rc = _fn("samp_cache_copy")(cache.address, kb, at, n, _raw_stream(device))
        if rc:
            _raise(rc)


def cache_bounds(cache: KVCache, bounds: KeyBounds, table: torch.Tensor, cu: Optional[torch.Tensor], lens: torch.Tensor, max_new: int,
                 rows: Optional[int] = None) -> None:
    """samp_cache_bounds: the bounds of the pages that the last cu[b + 1] - cu[b] of the lens[b] positions of each sequence have filled, after cache_write wrote them.
    rows: as many as cache_write was given, which an offset may not pass (None: any number)."""
    device = cache.device
    if device != _current_device():
        return _on(device, cache_bounds, cache, bounds, table, cu, lens, max_new, rows)
    kb = bounds.of(cache)
    t, width, pcu, plens, B = _places(device, table, cu, lens)
    max_new = _most(max_new)
    if rows is None:
        rows = B * max_new if cu is None else 1 << 24
    if rows and B:
        rc = _fn("samp_cache_bounds")(cache.address, kb, t, width, pcu, plens, B, max_new, _most(rows), _raw_stream(device))
        if rc:
            _raise(rc)


def cache_select(q: torch.Tensor, cache: KVCache, bounds: KeyBounds, table: torch.Tensor, cu: Optional[torch.Tensor], lens: torch.Tensor, max_new: int, keep: int,
                 sinks: int = 1, recent: Optional[int] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """samp_cache_select: (tables int32 [batch, kv_heads, keep], lens int32 [batch]) of the pages that the new tokens q [rows, heads, head_dim] are to read: the first `sinks`, the
    last `recent` (None: those that max_new tokens may lie in) and of the others those whose bounds promise most."""
    device = cache.device
    if device != _current_device():
        return _on(device, cache_select, q, cache, bounds, table, cu, lens, max_new, keep, sinks, recent)
    at, ld = _heads("q", q, device)
    rows, heads, dim = q.shape
    if dim != cache.head_dim:
        _refuse(f"q has heads of {dim}, the cache of {cache.head_dim}")
    kb = bounds.of(cache)
    t, width, pcu, plens, B = _places(device, table, cu, lens)
    tables, lens_out = table.new_empty((B, cache.kv_heads, _choice(keep))), torch.empty_like(lens)
    max_new = _most(max_new)
    if rows and B:
        need = _workspace_bytes("samp_cache_select_workspace_bytes", B, cache.kv_heads, width)
        ws = q.new_empty((need,), dtype=torch.uint8) if need else None
        rc = _fn("samp_cache_select")(at, ld, _TYPES[q.dtype], heads, cache.address, kb, t, width, pcu, plens, B, max_new, rows, keep, *_ends(cache, max_new, rows, sinks, recent),
                                      tables.data_ptr(), lens_out.data_ptr(), ws.data_ptr() if need else 0, need, _raw_stream(device))
        if rc:
            _raise(rc)
    else:
        tables.fill_(-1)
        lens_out.zero_()
    return tables, lens_out


def _choice(keep: int) -> int:
    if not 1 <= keep <= 32768:
        _refuse(f"keep is 1 to 32768 pages ({keep})")
    return keep


def _ends(cache: KVCache, max_new: int, rows: int, sinks: int, recent: Optional[int]) -> Tuple[int, int]:
    if recent is None:
        recent = (min(max_new, rows) + cache.page_len - 2) // cache.page_len + 1
    return _most(sinks), _most(recent)


def attention_sparse(q: torch.Tensor, cache: KVCache, bounds: KeyBounds, table: torch.Tensor, cu: Optional[torch.Tensor], lens: torch.Tensor, max_new: int, keep: int,
                     sinks: int = 1, recent: Optional[int] = None, max_len: Optional[int] = None, scale: Optional[float] = None, tree: Optional[torch.Tensor] = None,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """samp_attention_sparse: attention_cache over the `keep` pages for each sequence and key head that cache_select chooses."""
    device = cache.device
    if device != _current_device():
        return _on(device, attention_sparse, q, cache, bounds, table, cu, lens, max_new, keep, sinks, recent, max_len, scale, tree, out)
    at, ld = _heads("q", q, device)
    rows, heads, dim = q.shape
    if dim != cache.head_dim:
        _refuse(f"q has heads of {dim}, the cache of {cache.head_dim}")
    kb = bounds.of(cache)
    t, width, pcu, plens, B = _places(device, table, cu, lens)
    words = _flat("tree", tree, torch.int64, device, rows) if tree is not None else 0
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        to = out.data_ptr()
    else:
        to = _flat("out", out, q.dtype, device, rows * heads * dim)
    if rows and B:
        max_new, max_len = _most(max_new), _most(width * cache.page_len if max_len is None else max_len)
        need = _workspace_bytes("samp_attention_sparse_workspace_bytes", rows, B, heads, cache.kv_heads, dim, cache.page_len, width, max_new, max_len, _choice(keep))
        ws = q.new_empty((need,), dtype=torch.uint8) if need else None
        rc = _fn("samp_attention_sparse")(at, ld, _TYPES[q.dtype], heads, cache.address, kb, t, width, pcu, plens, B, max_new, max_len, rows, keep,
                                          *_ends(cache, max_new, rows, sinks, recent), dim ** -0.5 if scale is None else float(scale), words, to,
                                          ws.data_ptr() if need else 0, need, _raw_stream(device))
        if rc:
            _raise(rc)
    return out
