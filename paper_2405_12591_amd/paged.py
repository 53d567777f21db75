"""Binding of the head norm and rotation and of the paged 8-bit cache (include/decoquant.h): argument
checks and marshalling only."""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass
from typing import Dict, Optional, Sequence, Tuple

import torch

from .binding import DQError, KVCacheLayer, _check, _raw_stream, lib, workspace_init

PAGED_CAUSAL = 1
_DTYPES = {torch.float16: 0, torch.bfloat16: 1}
_CODES = {torch.int8: 0, torch.float8_e4m3fn: 1}


class _CHeads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64),
                ("heads", C.c_int32)]


class _CNorm(C.Structure):
    _fields_ = [("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("eps", C.c_float)]


class _CRotary(C.Structure):
    _fields_ = [("inv_freq", C.c_void_p), ("positions", C.c_void_p), ("axis_of_pair", C.c_void_p), ("position_stride", C.c_int64),
                ("axes", C.c_int32), ("rot_dim", C.c_int32), ("interleaved", C.c_int32)]


class _CPaged(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_codes", C.c_void_p), ("v_scales", C.c_void_p),
                ("k_tail", C.c_void_p), ("v_tail", C.c_void_p), ("pages", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("page_tokens", C.c_int32), ("slots", C.c_int32), ("dtype", C.c_int32), ("codes", C.c_int32)]


class _CBatch(C.Structure):
    _fields_ = [("starts", C.c_void_p), ("seq_lens", C.c_void_p), ("page_table", C.c_void_p), ("tail_slots", C.c_void_p),
                ("batch", C.c_int32), ("rows", C.c_int32), ("table_width", C.c_int32), ("table_stride", C.c_int32)]


def _declare() -> None:
    heads, norm, rot, cache, batch = (C.POINTER(t) for t in (_CHeads, _CNorm, _CRotary, _CPaged, _CBatch))
    i32, ptr = C.c_int32, C.c_void_p
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


def _on(device, *tensors) -> None:
    for t in tensors:
        if t is not None and t.device != device:
            raise DQError("all tensors of a call must be on one device (%s and %s given)" % (device, t.device))


def _call(what: str, fn, device, *args) -> None:
    """fn(*args, stream) on `device`'s current stream, with that device current."""
    index = device.index
    if index is None or index != torch.cuda.current_device():
        with torch.cuda.device(device):
            st = fn(*args, torch.cuda.current_stream(device).cuda_stream)
    else:
        st = fn(*args, _raw_stream(index) if _raw_stream else torch.cuda.current_stream(device).cuda_stream)
    if st:
        _check(st, what)


def _heads(name: str, t: torch.Tensor, dtype, dim: int) -> Tuple[_CHeads, Tuple[int, ...]]:
    """[rows, heads, dim] or [batch, rows, heads, dim] with channels side by side; (struct, shape without heads and dim)."""
    if t.dtype != dtype or not t.is_cuda or t.dim() not in (3, 4) or t.shape[-1] != dim:
        raise DQError("%s must be a %s device tensor [rows, heads, %d] or [batch, rows, heads, %d]" % (name, dtype, dim, dim))
    s = t.stride()
    if s[-1] != 1 or any(x % 8 or x < 0 for x in s[:-1]) or t.data_ptr() % 16:
        raise DQError("%s: channels must be neighbours, the other strides multiples of 8 elements, the data 16-byte aligned" % name)
    return _CHeads(t.data_ptr(), s[0] if t.dim() == 4 else 0, s[-3], s[-2], t.shape[-2]), tuple(t.shape[:-2])


def _spread(name: str, t: torch.Tensor) -> None:
    """Outputs may not lie on themselves (an expanded tensor)."""
    if any(n > 1 and s == 0 for n, s in zip(t.shape, t.stride())):
        raise DQError("%s must not be an expanded tensor" % name)


def _weight(name: str, w: Optional[torch.Tensor], dtype, dim: int):
    if w is None:
        return None
    if w.dtype != dtype or w.numel() != dim or not w.is_contiguous() or w.data_ptr() % 16:
        raise DQError("%s must be %d contiguous %s, 16-byte aligned" % (name, dim, dtype))
    return w.data_ptr()


def _norm(q_weight, k_weight, eps: float, dtype, dim: int) -> Optional[_CNorm]:
    if q_weight is None and k_weight is None:
        return None
    if not eps >= 0.0:
        raise DQError("eps must not be negative")
    return _CNorm(_weight("q_weight", q_weight, dtype, dim), _weight("k_weight", k_weight, dtype, dim), eps)


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

    def _c(self, positions: Optional[torch.Tensor], rows: int, device) -> _CRotary:
        _on(device, self.inv_freq, self.axis_of_pair, positions)
        stride, at = rows, None
        if positions is not None:
            if positions.dtype != torch.int32 or not positions.is_contiguous() or positions.numel() != self.axes * rows:
                raise DQError("positions must be contiguous int32, one per row%s" % (" and axis [axes, rows]" if self.axes > 1 else ""))
            at = positions.data_ptr()
        elif self.axes > 1:
            raise DQError("several axes need positions")
        return _CRotary(self.inv_freq.data_ptr(), at, None if self.axis_of_pair is None else self.axis_of_pair.data_ptr(), stride,
                        self.axes, self.rot_dim, int(self.interleaved))


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
    dtype, dim, device = first.dtype, first.shape[-1], first.device
    if dtype not in _DTYPES:
        raise DQError("heads must be float16 or bfloat16")
    structs, lead = [], None
    outs = []
    for name, x, out in (("q", q, q_out), ("k", k, k_out)):
        if x is None:
            if out is not None:
                raise DQError("%s_out without %s" % (name, name))
            structs += [None, None]
            outs.append(None)
            continue
        if out is None:
            out = torch.empty(x.shape, dtype=dtype, device=device)
        elif out.shape != x.shape:
            raise DQError("%s_out must have %s's shape" % (name, name))
        _on(device, x, out)
        cx, shape = _heads(name, x, dtype, dim)
        co, _ = _heads(name + "_out", out, dtype, dim)
        _spread(name + "_out", out)
        if lead is not None and shape != lead:
            raise DQError("q and k must have the same rows")
        lead = shape
        structs += [cx, co]
        outs.append(out)
    batch, tokens = lead if len(lead) == 2 else (1, lead[0])
    _on(device, q_weight, k_weight)
    norm = _norm(q_weight, k_weight, eps, dtype, dim)
    if rotary is None and norm is None:
        raise DQError("rotate_heads needs a rotation or a norm")
    if rotary is not None and positions is None:
        raise DQError("rotate_heads needs positions")
    rot = None if rotary is None else rotary._c(positions, batch * tokens, device)
    if batch and tokens:
        _call("dq_rotate_heads", lib.dq_rotate_heads, device, *(None if s is None else C.byref(s) for s in structs), batch, tokens, dim,
              _DTYPES[dtype], None if norm is None else C.byref(norm), None if rot is None else C.byref(rot))
    return outs[0], outs[1]


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
        _on(self.device, *self.t.values())
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


def _batch(cache: PagedCache, starts, seq_lens, page_table, tail_slots, rows: int, uses_starts: bool = True) -> _CBatch:
    """Sizes are checked here (the library sees pointers only)."""
    _on(cache.device, starts, seq_lens, page_table, tail_slots)
    for name, t in (("starts", starts), ("seq_lens", seq_lens), ("tail_slots", tail_slots)):
        if t is not None and (t.dtype != torch.int32 or t.dim() != 1 or not t.is_contiguous()):
            raise DQError("%s must be a contiguous int32 vector" % name)
    n = seq_lens.numel()
    if n < 1:
        raise DQError("a batch has at least one sequence")
    if starts is not None and starts.numel() != n + 1:
        raise DQError("starts must have one entry more than the batch has sequences")
    if uses_starts and starts is None and rows != n:
        raise DQError("without starts there is one row per sequence")
    if tail_slots is not None and tail_slots.numel() != n:
        raise DQError("tail_slots must have one slot per sequence")
    if tail_slots is None and n > cache.slots:
        raise DQError("more sequences than the cache has slots")
    if page_table.dtype != torch.int32 or page_table.dim() != 2 or page_table.shape[0] != n or page_table.shape[1] < 1 or page_table.stride(1) != 1 \
            or (n > 1 and page_table.stride(0) < page_table.shape[1]):
        raise DQError("page_table must be int32 [batch, pages], a sequence's pages side by side")
    width = page_table.shape[1]
    return _CBatch(None if starts is None else starts.data_ptr(), seq_lens.data_ptr(), page_table.data_ptr(),
                   None if tail_slots is None else tail_slots.data_ptr(), n, rows, width, page_table.stride(0) if n > 1 else width)


def _rows(cache: PagedCache, name: str, t: torch.Tensor, heads: Optional[int], rows: Optional[int]) -> _CHeads:
    _on(cache.device, t)
    c, lead = _heads(name, t, cache.dtype, cache.head_dim)
    if len(lead) != 1 or (rows is not None and lead[0] != rows) or (heads is not None and t.shape[1] != heads):
        raise DQError("%s must be [rows%s, %sheads, head_dim]" % (name, "" if rows is None else " = %d" % rows, "" if heads is None else "%d " % heads))
    return c


def paged_append(cache: PagedCache, k: torch.Tensor, v: torch.Tensor, starts: Optional[torch.Tensor], seq_lens: torch.Tensor,
                 page_table: torch.Tensor, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                 rotary: Optional[Rotary] = None, positions: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None,
                 k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, tail_slots: Optional[torch.Tensor] = None):
    """Append the rows k, v [rows, kv_heads, d] of a ragged batch (dq_paged_append); keys, and q beside them, are normed
    and rotated on the way.  starts: int32 [batch + 1], rows starts[b] .. starts[b+1] - 1 are sequence b's last tokens
    (None: one row each); seq_lens: int32, the new rows included; page_table: int32 [batch, pages].  positions None: a
    token's place in its sequence.  Returns q_out (None without q)."""
    ck = _rows(cache, "k", k, cache.kv_heads, None)
    rows = k.shape[0]
    cv = _rows(cache, "v", v, cache.kv_heads, rows)
    cb = _batch(cache, starts, seq_lens, page_table, tail_slots, rows)
    cq = co = None
    if q is not None:
        cq = _rows(cache, "q", q, None, rows)
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        co = _rows(cache, "q_out", q_out, q.shape[1], rows)
        _spread("q_out", q_out)
    elif q_out is not None:
        raise DQError("q_out without q")
    _on(cache.device, q_weight, k_weight)
    norm = _norm(q_weight, k_weight, eps, cache.dtype, cache.head_dim)
    if rotary is not None and rotary.rot_dim > cache.head_dim:
        raise DQError("rot_dim is larger than head_dim")
    rot = None if rotary is None else rotary._c(positions, rows, cache.device)
    if rows:
        _call("dq_paged_append", lib.dq_paged_append, cache.device, cache._ref, C.byref(cb), C.byref(ck), C.byref(cv),
              None if cq is None else C.byref(cq), None if co is None else C.byref(co), None if norm is None else C.byref(norm),
              None if rot is None else C.byref(rot))
    return q_out


def paged_read(cache: PagedCache, first: Optional[torch.Tensor], seq_lens: torch.Tensor, out_starts: torch.Tensor, page_table: torch.Tensor,
               k_out: torch.Tensor, v_out: torch.Tensor, tail_slots: Optional[torch.Tensor] = None):
    """The rows that tokens first[b] <= t < seq_lens[b] of the cache stand for, into k_out and v_out [rows, kv_heads, d]
    from row out_starts[b] on (dq_paged_read; first None: from 0).  Returns (k_out, v_out)."""
    ck = _rows(cache, "k_out", k_out, cache.kv_heads, None)
    cv = _rows(cache, "v_out", v_out, cache.kv_heads, k_out.shape[0])
    _spread("k_out", k_out)
    _spread("v_out", v_out)
    cb = _batch(cache, out_starts, seq_lens, page_table, tail_slots, k_out.shape[0], uses_starts=False)
    _on(cache.device, first)
    if first is not None and (first.dtype != torch.int32 or first.numel() != seq_lens.numel() or not first.is_contiguous()):
        raise DQError("first must hold one int32 per sequence")
    if out_starts is None:
        raise DQError("paged_read needs out_starts")
    if k_out.shape[0]:
        _call("dq_paged_read", lib.dq_paged_read, cache.device, cache._ref, C.byref(cb), None if first is None else first.data_ptr(),
              out_starts.data_ptr(), C.byref(ck), C.byref(cv))
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
                    causal: bool = True, window: int = 0, tail_slots: Optional[torch.Tensor] = None) -> torch.Tensor:
    """softmax(q . K * scale) V of the batch's rows q [rows, q_heads, d] over the cached tokens of their sequences
    (dq_paged_attention); rows are the last tokens of their sequence (append them first).  max_rows, max_seq_len: host
    bounds on the rows and tokens of any sequence.  window > 0: the last `window` tokens only.  out may be q."""
    cq = _rows(cache, "q", q, None, None)
    rows, heads = q.shape[0], q.shape[1]
    if heads == 0 or heads % cache.kv_heads:
        raise DQError("q_heads must be a multiple of kv_heads")
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    co = _rows(cache, "out", out, heads, rows)
    _spread("out", out)
    cb = _batch(cache, starts, seq_lens, page_table, tail_slots, rows)
    _on(cache.device, workspace)
    if workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise DQError("workspace must be contiguous uint8")
    if max_rows < 0 or max_seq_len < 0 or window < 0 or (window and not causal):
        raise DQError("max_rows, max_seq_len and window must not be negative, and a window needs causal")
    if rows:
        _call("dq_paged_attention", lib.dq_paged_attention, cache.device, cache._ref, C.byref(cb), C.byref(cq), C.byref(co), max_rows,
              max_seq_len, softmax_scale, window, workspace.data_ptr(), workspace.numel(), PAGED_CAUSAL if causal else 0)
    return out
