"""Binding of the head norm and rotation and of the paged 8-bit cache (include/decoquant.h): argument
checks and marshalling only."""
from __future__ import annotations

import ctypes as C
import struct
from dataclasses import dataclass
from typing import Dict, Optional, Sequence

import torch

from .binding import DQError, _check, _raw_stream, lib, workspace_init

PAGED_CAUSAL = 1
_I32 = torch.int32
_DTYPES = {torch.float16: 0, torch.bfloat16: 1}
_CODES = {torch.int8: 0, torch.float8_e4m3fn: 1}


# The small structs of a call (dq_heads, dq_head_norm, dq_rotary, dq_paged_batch), packed: a ctypes structure takes three times
# as long to fill, and a call of these operators on the GPU is over in a few microseconds.
_pack_heads = struct.Struct("@Pqqqi4x").pack
_pack_norm = struct.Struct("@PPf4x").pack
_pack_rotary = struct.Struct("@PPPqiii4x").pack
_pack_batch = struct.Struct("@PPPPiiii").pack


class _CPaged(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_codes", C.c_void_p), ("v_scales", C.c_void_p),
                ("k_tail", C.c_void_p), ("v_tail", C.c_void_p), ("pages", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("page_tokens", C.c_int32), ("slots", C.c_int32), ("dtype", C.c_int32), ("codes", C.c_int32)]


def _declare() -> None:
    cache, i32, ptr = C.POINTER(_CPaged), C.c_int32, C.c_void_p
    heads = norm = rot = batch = ptr
    lib.dq_rotate_heads.restype = i32
    lib.dq_rotate_heads.argtypes = [heads, heads, heads, heads, i32, i32, i32, i32, norm, rot, ptr]
    lib.dq_paged_append.restype = i32
    lib.dq_paged_append.argtypes = [cache, batch, heads, heads, heads, heads, norm, rot, ptr]
    lib.dq_paged_read.restype = i32
    lib.dq_paged_read.argtypes = [cache, batch, ptr, ptr, heads, heads, ptr]
    lib.dq_paged_workspace_bytes.restype = C.c_size_t
    lib.dq_paged_workspace_bytes.argtypes = [cache, i32, i32, i32, i32, i32]
    lib.dq_paged_attention.restype = i32
    lib.dq_paged_attention.argtypes = [cache, batch, heads, heads, i32, i32, C.c_float, i32, ptr, C.c_size_t, C.c_uint32, ptr]


_declare()


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _on(index: int, *tensors) -> None:
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise DQError("all tensors of a call must be on one GPU (cuda:%d and %s given)" % (index, t.device))


def _call(what: str, fn, index: int, *args) -> None:
    """fn(*args, stream) on device `index`'s current stream, with that device current."""
    if index != _current_device():
        with torch.cuda.device(index):
            st = fn(*args, torch.cuda.current_stream(index).cuda_stream)
    else:
        st = fn(*args, _raw_stream(index) if _raw_stream else torch.cuda.current_stream(index).cuda_stream)
    if st:
        _check(st, what)


def _heads(name: str, t: torch.Tensor, dtype, dim: int, index: int, written: bool = False):
    """[rows, heads, dim] or [batch, rows, heads, dim] with channels side by side: (packed dq_heads, (batch,) rows, heads)."""
    shape, strides = t.shape, t.stride()
    if len(shape) == 3:
        rows, heads, d = shape
        s1, s2, s3 = strides
        batch, s0 = 1, 0
    elif len(shape) == 4:
        batch, rows, heads, d = shape
        s0, s1, s2, s3 = strides
        if batch == 1:
            s0 = 0
    else:
        raise DQError("%s must be [rows, heads, %d] or [batch, rows, heads, %d]" % (name, dim, dim))
    if rows == 1:                                    # a stride over one entry says nothing
        s1 = 0
    if heads == 1:
        s2 = 0
    ptr = t.data_ptr()
    if t.dtype is not dtype or d != dim or t.get_device() != index:
        raise DQError("%s must be a %s tensor on cuda:%d with %d channels a head" % (name, dtype, index, dim))
    if s3 != 1 or (s0 | s1 | s2) & 7 or ptr & 15:
        raise DQError("%s: channels must be neighbours, the other strides multiples of 8 elements, the data 16-byte aligned" % name)
    if written and ((rows > 1 and s1 == 0) or (heads > 1 and s2 == 0) or (batch > 1 and s0 == 0)):
        raise DQError("%s must not be an expanded tensor" % name)
    return _pack_heads(ptr, s0, s1, s2, heads), (batch, rows) if len(shape) == 4 else rows, heads


def _weight(name: str, w: Optional[torch.Tensor], dtype, dim: int, index: int) -> int:
    if w is None:
        return 0
    ptr = w.data_ptr()
    if w.dtype is not dtype or w.numel() != dim or not w.is_contiguous() or ptr & 15 or w.get_device() != index:
        raise DQError("%s must be %d contiguous %s on cuda:%d, 16-byte aligned" % (name, dim, dtype, index))
    return ptr


def _norm(q_weight, k_weight, eps: float, dtype, dim: int, index: int) -> Optional[bytes]:
    if q_weight is None and k_weight is None:
        return None
    if not eps >= 0.0:
        raise DQError("eps must not be negative")
    return _pack_norm(_weight("q_weight", q_weight, dtype, dim, index), _weight("k_weight", k_weight, dtype, dim, index), eps)


@dataclass(frozen=True)
class Rotary:
    """Position rotation of the first 2 * len(inv_freq) channels of a head (dq_rotary): pair i turns by
    position * inv_freq[i] radians, the position on axis axis_of_pair[i] where there are several.
    interleaved: pairs are channels (2i, 2i + 1) instead of (i, i + half)."""
    inv_freq: torch.Tensor                          # float64 [rot_dim / 2], on the device
    interleaved: bool = False
    axis_of_pair: Optional[torch.Tensor] = None     # uint8 [rot_dim / 2]
    axes: int = 1

    def __post_init__(self):
        f, a = self.inv_freq, self.axis_of_pair
        if f.dtype != torch.float64 or f.dim() != 1 or not f.is_contiguous() or not f.numel() or f.numel() % 8:
            raise DQError("inv_freq must be a contiguous float64 vector, its length a multiple of 8")
        if not 1 <= self.axes <= 8 or (self.axes > 1) != (a is not None):
            raise DQError("axes must be 1..8, with axis_of_pair where there are several")
        if a is not None and (a.dtype != torch.uint8 or a.shape != f.shape or not a.is_contiguous()):
            raise DQError("axis_of_pair must be one uint8 per pair")

    @property
    def rot_dim(self) -> int:
        return 2 * self.inv_freq.numel()

    def _c(self, positions: Optional[torch.Tensor], rows: int, index: int) -> bytes:
        fixed = self.__dict__.get("_fixed")
        if fixed is None:                            # a Rotary never changes
            a = self.axis_of_pair
            if a is not None and a.device != self.inv_freq.device:
                raise DQError("inv_freq and axis_of_pair must be on one device")
            fixed = (self.inv_freq.get_device(), self.inv_freq.data_ptr(), 0 if a is None else a.data_ptr(), self.axes, self.rot_dim,
                     int(self.interleaved))
            object.__setattr__(self, "_fixed", fixed)   # (the dataclass is frozen)
        if fixed[0] != index:
            raise DQError("the rotation's frequencies must be on cuda:%d" % index)
        at = 0
        if positions is not None:
            if positions.dtype is not torch.int32 or positions.numel() != self.axes * rows or not positions.is_contiguous() \
                    or positions.get_device() != index:
                raise DQError("positions must be contiguous int32 on cuda:%d, one per row%s" % (index, " and axis [axes, rows]" if self.axes > 1 else ""))
            at = positions.data_ptr()
        elif self.axes > 1:
            raise DQError("several axes need positions")
        return _pack_rotary(fixed[1], at, fixed[2], rows, fixed[3], fixed[4], fixed[5])


def rotary(rot_dim: int, base: float = 10000.0, sections: Optional[Sequence[int]] = None, interleaved: bool = False,
           device="cuda:0") -> Rotary:
    """The usual frequencies base^(-2i / rot_dim).  sections: pairs per axis, one run of pairs after the
    other (time, height, width, ...), summing to rot_dim / 2."""
    if rot_dim <= 0 or rot_dim % 16:
        raise DQError("rot_dim must be a multiple of 16")
    half = rot_dim // 2
    inv = float(base) ** (-torch.arange(half, dtype=torch.float64) / half)
    axis = None
    if sections is not None and len(sections) > 1:
        if sum(sections) != half or min(sections) < 0:
            raise DQError("sections must sum to rot_dim / 2")
        axis = torch.repeat_interleave(torch.arange(len(sections), dtype=torch.uint8), torch.tensor(list(sections))).to(device)
    return Rotary(inv.to(device), interleaved, axis, 1 if axis is None else len(sections))


def rotate_heads(q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: Optional[torch.Tensor] = None,
                 rotary: Optional[Rotary] = None, q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None,
                 eps: float = 1e-6, q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
    """RMS norm (where a weight is given) and rotation of query and key heads, fp16 or bf16, in one pass
    (dq_rotate_heads); returns (q_out, k_out).  q, k: [rows, heads, d] or [batch, rows, heads, d], any strides with
    channels side by side (views of a fused projection, transposed layouts); either may be None.  positions:
    int32, one per row ([axes, ...] with several axes).  An output may be its own input."""
    first = q if q is not None else k
    if first is None:
        raise DQError("rotate_heads needs q or k")
    dtype, dim, index = first.dtype, first.shape[-1], first.get_device()
    if dtype not in _DTYPES or index < 0:
        raise DQError("heads must be float16 or bfloat16 on a GPU")
    cq = cqo = ck = cko = lead = None
    if q is not None:
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=dtype, device=q.device)
        cq, lead, heads = _heads("q", q, dtype, dim, index)
        cqo, lead_o, heads_o = _heads("q_out", q_out, dtype, dim, index, True)
        if lead_o != lead or heads_o != heads:
            raise DQError("q_out must have q's shape")
    elif q_out is not None:
        raise DQError("q_out without q")
    if k is not None:
        if k_out is None:
            k_out = torch.empty(k.shape, dtype=dtype, device=k.device)
        ck, lead_k, heads = _heads("k", k, dtype, dim, index)
        cko, lead_o, heads_o = _heads("k_out", k_out, dtype, dim, index, True)
        if lead_o != lead_k or heads_o != heads:
            raise DQError("k_out must have k's shape")
        if lead is not None and lead_k != lead:
            raise DQError("q and k must have the same rows")
        lead = lead_k
    elif k_out is not None:
        raise DQError("k_out without k")
    batch, tokens = lead if type(lead) is tuple else (1, lead)
    norm = _norm(q_weight, k_weight, eps, dtype, dim, index)
    rot = None
    if rotary is not None:
        if positions is None:
            raise DQError("rotate_heads needs positions")
        rot = rotary._c(positions, batch * tokens, index)
    elif norm is None:
        raise DQError("rotate_heads needs a rotation or a norm")
    if batch and tokens:
        _call("dq_rotate_heads", lib.dq_rotate_heads, index, cq, cqo, ck, cko, batch, tokens, dim, _DTYPES[dtype], norm, rot)
    return q_out, k_out


class PagedCache:
    """Device tensors of a layer's paged 8-bit cache plus the C struct that points at them (dq_paged_cache):
    k_codes [pages, H, P, d], v_codes [pages, H, P/64, d, 64] (int8 or float8_e4m3fn), k_scales and v_scales
    float32 [pages, H], k_tail [slots, H, P, d], v_tail [slots, H, P/64, d, 64] (float16 or bfloat16)."""

    def __init__(self, tensors: Dict[str, torch.Tensor]):
        names = ("k_codes", "k_scales", "v_codes", "v_scales", "k_tail", "v_tail")
        if any(n not in tensors for n in names) or tensors["k_codes"].dim() != 4 or tensors["k_tail"].dim() != 4:
            raise DQError("a paged cache has the tensors %s" % ", ".join(names))
        self.t = {n: tensors[n] for n in names}
        kc, kt = self.t["k_codes"], self.t["k_tail"]
        self.pages, self.kv_heads, self.page_tokens, self.head_dim = kc.shape
        self.slots, self.dtype, self.codes, self.device = kt.shape[0], kt.dtype, kc.dtype, kc.device
        if self.dtype not in _DTYPES or self.codes not in _CODES:
            raise DQError("rows are float16 or bfloat16, codes int8 or float8_e4m3fn")
        if self.head_dim not in (64, 128) or self.page_tokens not in (64, 128):
            raise DQError("head_dim and page_tokens must be 64 or 128")
        for name, (shape, dtype) in _paged_shapes(self.pages, self.slots, self.kv_heads, self.head_dim, self.page_tokens, self.dtype, self.codes).items():
            t = self.t[name]
            if not (t.is_cuda and t.is_contiguous()) or tuple(t.shape) != shape or t.dtype != dtype or t.data_ptr() % 16:
                raise DQError("%s must be a contiguous, 16-byte aligned %s device tensor of shape %s" % (name, dtype, shape))
        self.index = kc.get_device()
        _on(self.index, *self.t.values())
        self.c = _CPaged(*(self.t[n].data_ptr() for n in names), self.pages, self.kv_heads, self.head_dim, self.page_tokens, self.slots,
                         _DTYPES[self.dtype], _CODES[self.codes])
        self._ref = C.byref(self.c)

    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in self.t.values())


def _paged_shapes(pages, slots, h, d, p, dtype, codes):
    return {"k_codes": ((pages, h, p, d), codes), "k_scales": ((pages, h), torch.float32),
            "v_codes": ((pages, h, p // 64, d, 64), codes), "v_scales": ((pages, h), torch.float32),
            "k_tail": ((slots, h, p, d), dtype), "v_tail": ((slots, h, p // 64, d, 64), dtype)}


def alloc_paged_cache(pages: int, slots: int, kv_heads: int, head_dim: int, page_tokens: int = 64, dtype=torch.float16,
                      codes=torch.int8, device="cuda:0") -> PagedCache:
    """A paged cache for `slots` sequences at a time (one 16-bit tail each)."""
    if min(pages, slots, kv_heads) < 1 or page_tokens not in (64, 128):
        raise DQError("pages, slots and kv_heads must be positive, page_tokens 64 or 128")
    return PagedCache({n: torch.zeros(shape, dtype=torch.uint8 if t == codes else t, device=device).view(t)
                       for n, (shape, t) in _paged_shapes(pages, slots, kv_heads, head_dim, page_tokens, dtype, codes).items()})


def _vector(name: str, t: torch.Tensor, n: int, index: int) -> int:
    """Address of n int32 side by side on device `index`."""
    if t.dtype is not _I32 or t.numel() != n or not t.is_contiguous() or t.get_device() != index:
        raise DQError("%s must hold %d int32, side by side on cuda:%d" % (name, n, index))
    return t.data_ptr()


def _batch(cache: PagedCache, starts, seq_lens, page_table, tail_slots, rows: int, uses_starts: bool = True) -> bytes:
    """Sizes are checked here (the library sees pointers only)."""
    index = cache.index
    n = seq_lens.numel()
    if n < 1:
        raise DQError("a batch has at least one sequence")
    shape = page_table.shape
    if len(shape) != 2 or shape[0] != n or shape[1] < 1 or page_table.dtype is not _I32 or page_table.get_device() != index:
        raise DQError("page_table must be int32 [batch, pages], on the cache's GPU")
    width = shape[1]
    stride, inner = page_table.stride()
    if n == 1:
        stride = width
    if (inner != 1 and width > 1) or stride < width:
        raise DQError("a sequence's pages must lie side by side in page_table")
    if starts is None and uses_starts and rows != n:
        raise DQError("without starts there is one row per sequence")
    if tail_slots is None and n > cache.slots:
        raise DQError("more sequences than the cache has slots")
    return _pack_batch(0 if starts is None else _vector("starts", starts, n + 1, index), _vector("seq_lens", seq_lens, n, index),
                       page_table.data_ptr(), 0 if tail_slots is None else _vector("tail_slots", tail_slots, n, index), n, rows, width, stride)


def _rows(cache: PagedCache, name: str, t: torch.Tensor, heads: Optional[int], rows: Optional[int], written: bool = False):
    """(packed dq_heads, rows, heads) of rows [rows, heads, head_dim] of the cache's type."""
    shape = t.shape
    if len(shape) == 3:                                  # the usual case with as few looks at the tensor as can be
        n, h, d = shape
        s0, s1, s2 = t.stride()
        ptr = t.data_ptr()
        if d == cache.head_dim and s2 == 1 and s0 and s1 and not (s0 | s1) & 7 and not ptr & 15 and t.dtype is cache.dtype \
                and t.get_device() == cache.index and (rows is None or n == rows) and (heads is None or h == heads):
            return _pack_heads(ptr, 0, s0, s1, h), n, h
    c, r, h = _heads(name, t, cache.dtype, cache.head_dim, cache.index, written)
    if type(r) is tuple or (rows is not None and r != rows) or (heads is not None and h != heads):
        raise DQError("%s must be [rows%s, %sheads, head_dim]" % (name, "" if rows is None else " = %d" % rows, "" if heads is None else "%d " % heads))
    return c, r, h


def paged_append(cache: PagedCache, k: torch.Tensor, v: torch.Tensor, starts: Optional[torch.Tensor], seq_lens: torch.Tensor,
                 page_table: torch.Tensor, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                 rotary: Optional[Rotary] = None, positions: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None,
                 k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, tail_slots: Optional[torch.Tensor] = None):
    """Append the rows k, v [rows, kv_heads, d] of a ragged batch (dq_paged_append); keys, and q beside them, are normed
    and rotated on the way.  starts: int32 [batch + 1], rows starts[b] .. starts[b+1] - 1 are sequence b's last tokens
    (None: one row each); seq_lens: int32, the new rows included; page_table: int32 [batch, pages].  positions None: a
    token's place in its sequence.  Returns q_out (None without q)."""
    index = cache.index
    ck, rows, _ = _rows(cache, "k", k, cache.kv_heads, None)
    cv, _, _ = _rows(cache, "v", v, cache.kv_heads, rows)
    cb = _batch(cache, starts, seq_lens, page_table, tail_slots, rows)
    cq = co = None
    if q is not None:
        cq, _, heads = _rows(cache, "q", q, None, rows)
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        co, _, _ = _rows(cache, "q_out", q_out, heads, rows, True)
    elif q_out is not None:
        raise DQError("q_out without q")
    norm = _norm(q_weight, k_weight, eps, cache.dtype, cache.head_dim, index)
    rot = None
    if rotary is not None:
        rot = rotary._c(positions, rows, index)
        if rotary.rot_dim > cache.head_dim:
            raise DQError("rot_dim is larger than head_dim")
    if rows:
        _call("dq_paged_append", lib.dq_paged_append, index, cache._ref, cb, ck, cv, cq, co, norm, rot)
    return q_out


def paged_read(cache: PagedCache, first: Optional[torch.Tensor], seq_lens: torch.Tensor, out_starts: torch.Tensor, page_table: torch.Tensor,
               k_out: torch.Tensor, v_out: torch.Tensor, tail_slots: Optional[torch.Tensor] = None):
    """The rows that tokens first[b] <= t < seq_lens[b] of the cache stand for, into k_out and v_out [rows, kv_heads, d]
    from row out_starts[b] on (dq_paged_read; first None: from 0).  Returns (k_out, v_out)."""
    ck, rows, _ = _rows(cache, "k_out", k_out, cache.kv_heads, None, True)
    cv, _, _ = _rows(cache, "v_out", v_out, cache.kv_heads, rows, True)
    if out_starts is None:
        raise DQError("paged_read needs out_starts")
    cb = _batch(cache, out_starts, seq_lens, page_table, tail_slots, rows, False)
    at = 0
    if first is not None:
        at = _vector("first", first, seq_lens.numel(), cache.index)
    if rows:
        _call("dq_paged_read", lib.dq_paged_read, cache.index, cache._ref, cb, at, out_starts.data_ptr(), ck, cv)
    return k_out, v_out


def paged_workspace(cache: PagedCache, batch: int, rows: int, q_heads: int, max_rows: int, max_seq_len: int) -> torch.Tensor:
    """Workspace of paged_attention for these sizes."""
    n = lib.dq_paged_workspace_bytes(cache._ref, batch, rows, q_heads, max_rows, max_seq_len)
    if n == 0:
        raise DQError("dq_paged_workspace_bytes rejected the arguments")
    ws = torch.empty((n + 15) // 16 * 16, dtype=torch.uint8, device=cache.device)
    with torch.cuda.device(cache.device):
        workspace_init(ws)
    return ws


def paged_attention(cache: PagedCache, q: torch.Tensor, starts: Optional[torch.Tensor], seq_lens: torch.Tensor, page_table: torch.Tensor,
                    max_rows: int, max_seq_len: int, workspace: torch.Tensor, out: Optional[torch.Tensor] = None, softmax_scale: float = 0.0,
                    causal: bool = True, window: int = 0, tail_slots: Optional[torch.Tensor] = None, splits: int = 0) -> torch.Tensor:
    """softmax(q . K * scale) V of the batch's rows q [rows, q_heads, d] over the cached tokens of their sequences
    (dq_paged_attention); rows are the last tokens of their sequence (append them first).  max_rows: host bound on the
    rows of any sequence; max_seq_len: on its tokens (a guess does).  window > 0: the last `window` tokens only.  out may be q.
    splits: launch override for sweeps (DQ_PAGED_SPLITS)."""
    cq, rows, heads = _rows(cache, "q", q, None, None)
    if heads == 0 or heads % cache.kv_heads:
        raise DQError("q_heads must be a multiple of kv_heads")
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    co, _, _ = _rows(cache, "out", out, heads, rows, True)
    cb = _batch(cache, starts, seq_lens, page_table, tail_slots, rows)
    if workspace.dtype is not torch.uint8 or not workspace.is_contiguous() or workspace.get_device() != cache.index:
        raise DQError("workspace must be contiguous uint8 on the cache's GPU")
    if max_rows < 0 or max_seq_len < 0 or window < 0 or (window and not causal):
        raise DQError("max_rows, max_seq_len and window must not be negative, and a window needs causal")
    if rows:
        _call("dq_paged_attention", lib.dq_paged_attention, cache.index, cache._ref, cb, cq, co, max_rows, max_seq_len, softmax_scale, window,
              workspace.data_ptr(), workspace.numel(), (PAGED_CAUSAL if causal else 0) | ((splits & 0x7F) << 8))
    return out


class PagedKVLayer:
    """One layer's keys and values in 8-bit pages, as KVCacheLayer is for the DecoQuant form: `batch` sequences of up to
    max_tokens tokens, each with its own pages and tail, the lengths on the device.  Rows come packed, sequence by
    sequence (`starts`, int32 [batch + 1]; None: one row each); the host tracks only bounds, which size the launches.
    (Loops with a page allocator of their own call paged_append and paged_attention.)"""

    def __init__(self, batch: int, q_heads: int, kv_heads: int, head_dim: int, max_tokens: int, page_tokens: int = 64,
                 dtype=torch.float16, codes=torch.int8, device="cuda:0"):
        if batch < 1 or max_tokens < 1 or q_heads < 1 or q_heads % kv_heads:
            raise DQError("a layer has sequences, room for tokens and q_heads a multiple of kv_heads")
        self.batch, self.q_heads, self.max_tokens = batch, q_heads, max_tokens
        width = -(-max_tokens // page_tokens)
        self.cache = alloc_paged_cache(batch * width, batch, kv_heads, head_dim, page_tokens, dtype, codes, device)
        self.page_table = torch.arange(batch * width, dtype=torch.int32, device=device).view(batch, width)
        self.seq_lens = torch.zeros(batch, dtype=torch.int32, device=device)
        self.tokens_upper = 0               # no sequence holds more tokens than this (host-side bound)
        self._ws, self._outgrown = None, []

    def append(self, k: torch.Tensor, v: torch.Tensor, starts: Optional[torch.Tensor] = None, max_rows: int = 1,
               q: Optional[torch.Tensor] = None, rotary: Optional[Rotary] = None, positions: Optional[torch.Tensor] = None,
               q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6):
        """Append rows k, v [rows, kv_heads, d], no sequence more than max_rows; norm and rotation as paged_append does
        them; returns q normed and rotated (None without q)."""
        if starts is None and max_rows != 1:
            raise DQError("several rows per sequence need starts")
        if self.tokens_upper + max_rows > self.max_tokens:
            # the bound may be ahead of the lengths (ragged rows); only then is it worth a look at them
            self.tokens_upper = int(self.seq_lens.max())
            if self.tokens_upper + max_rows > self.max_tokens:
                raise DQError("the rows exceed the layer's %d tokens per sequence" % self.max_tokens)
        new = 1 if starts is None else starts.diff()
        self.seq_lens += new
        try:
            q = paged_append(self.cache, k, v, starts, self.seq_lens, self.page_table, q=q, rotary=rotary, positions=positions,
                             q_weight=q_weight, k_weight=k_weight, eps=eps)
        except DQError:                     # nothing was launched
            self.seq_lens -= new
            raise
        self.tokens_upper += max_rows
        return q

    def attend(self, q: torch.Tensor, starts: Optional[torch.Tensor] = None, max_rows: int = 1, out: Optional[torch.Tensor] = None,
               softmax_scale: float = 0.0, causal: bool = True, window: int = 0) -> torch.Tensor:
        """Attention of the rows just appended, q [rows, q_heads, d] (paged_attention)."""
        rows, bound = q.shape[0], min(self.tokens_upper, self.max_tokens)
        if self._ws is None or rows > self._ws[0] or max_rows > self._ws[1]:
            sizes = (rows, max_rows)
            if self._ws:
                sizes = (max(rows, self._ws[0]), max(max_rows, self._ws[1]))
                self._outgrown.append(self._ws[2])   # a captured graph may still work in it
            self._ws = (*sizes, paged_workspace(self.cache, self.batch, sizes[0], self.q_heads, sizes[1], self.max_tokens))
        return paged_attention(self.cache, q, starts, self.seq_lens, self.page_table, max_rows, bound, self._ws[2], out=out,
                               softmax_scale=softmax_scale, causal=causal, window=window)

    def read(self, lengths: Sequence[int]):
        """The rows the layer stands for, k and v [batch, kv_heads, max(lengths), d]; sequence b's first lengths[b] (host
        integers, its tokens) are written, the rest is zero.  Goes into KVCacheLayer.prefill (fp16 layers)."""
        c = self.cache
        n = max(lengths)
        k = torch.zeros((self.batch, c.kv_heads, n, c.head_dim), dtype=c.dtype, device=c.device)
        v = torch.zeros_like(k)
        lens = torch.tensor(list(lengths), dtype=torch.int32, device=c.device)
        for b in range(self.batch):
            if lengths[b] > 0:
                one = torch.tensor([0, lengths[b]], dtype=torch.int32, device=c.device)
                paged_read(c, None, lens[b:b + 1], one, self.page_table[b:b + 1], k[b].transpose(0, 1), v[b].transpose(0, 1),
                           tail_slots=torch.tensor([b], dtype=torch.int32, device=c.device))
        return k, v
