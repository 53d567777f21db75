"""Binding of the head norm and rotation and of the paged 8-bit cache (include/decoquant.h): argument
checks and marshalling only, the checks of tensors in csrc/paged_bind.cpp.  These operators serve: tensors that require gradients are
taken as they are, outputs carry none, and what is written in place (an output that is its own input, a cache) is not recorded."""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Dict, Optional, Sequence

import torch

from . import build as _build
from .binding import DQError, _check, _raw_stream, lib, workspace_init

_DTYPES = {torch.float16: 0, torch.bfloat16: 1}
_CODES = {torch.int8: 0, torch.float8_e4m3fn: 1}


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


def _load_module():
    if not os.path.exists(_build.BIND_PATH):
        _build.build_binding()
    from . import _paged
    if getattr(_paged, "stamp", None) != _build.bind_stamp():   # its structs would not match the library's
        raise DQError("%s was built from other sources: rebuild it" % _build.BIND_PATH)
    _paged.set_up(DQError, _check, *(C.cast(getattr(lib, n), C.c_void_p).value
                                     for n in ("dq_rotate_heads", "dq_paged_append", "dq_paged_read", "dq_paged_attention")))
    return _paged


class _Module:
    """The compiled checks, loaded (and built where they are missing) with their first use: callers of the rest need neither them nor g++."""

    def __getattr__(self, name):
        if name.startswith("_"):
            raise AttributeError(name)
        loaded = _load_module()
        for n in ("rotate_heads", "paged_append", "paged_read", "paged_attention"):
            setattr(self, n, getattr(loaded, n))
        return getattr(loaded, name)


_module = _Module()
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _call(fn, index: int, *args) -> None:
    """fn(*args, stream) with device `index`'s current stream, that device current."""
    if index < 0:
        raise DQError("the tensors must be on a GPU")
    if index != _current_device():
        with torch.cuda.device(index):
            fn(*args, torch.cuda.current_stream(index).cuda_stream)
    else:
        fn(*args, _raw_stream(index) if _raw_stream else torch.cuda.current_stream(index).cuda_stream)


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
        if a is not None and a.device != f.device:
            raise DQError("inv_freq and axis_of_pair must be on one device")

    @property
    def _c(self):
        return self.inv_freq, self.axis_of_pair, self.axes, bool(self.interleaved)   # what the compiled checks take

    @property
    def rot_dim(self) -> int:
        return 2 * self.inv_freq.numel()


def rotary(rot_dim: int, base: float = 10000.0, sections: Optional[Sequence[int]] = None, interleaved: bool = False,
           device="cuda:0") -> Rotary:
    """The usual frequencies base^(-2i / rot_dim).  sections: pairs per axis, one run of pairs after the
    other (time, height, width, ...), summing to rot_dim / 2."""
    if rot_dim <= 0 or rot_dim % 16 or not float(base) > 0:
        raise DQError("rot_dim must be a multiple of 16, base positive")
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
    int32, one per row ([axes, ...] with several axes).  An output may be its own input.  No gradients."""
    first = q if q is not None else k
    if first is None:
        raise DQError("rotate_heads needs q or k")
    if q is None:
        if q_out is not None:
            raise DQError("q_out without q")
    elif q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if k is None:
        if k_out is not None:
            raise DQError("k_out without k")
    elif k_out is None:
        k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
    index = first.get_device()
    _call(_module.rotate_heads, index, q, q_out, k, k_out, positions, None if rotary is None else rotary._c, q_weight, k_weight, eps, index)
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
        for n, t in self.t.items():
            if t.get_device() != self.index:
                raise DQError("all tensors of a cache must be on one GPU (cuda:%d, and %s on %s)" % (self.index, n, t.device))
        self.c = _CPaged(*(self.t[n].data_ptr() for n in names), self.pages, self.kv_heads, self.head_dim, self.page_tokens, self.slots,
                         _DTYPES[self.dtype], _CODES[self.codes])
        self._at = C.addressof(self.c)

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


def paged_append(cache: PagedCache, k: torch.Tensor, v: torch.Tensor, starts: Optional[torch.Tensor], seq_lens: torch.Tensor,
                 page_table: torch.Tensor, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                 rotary: Optional[Rotary] = None, positions: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None,
                 k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, tail_slots: Optional[torch.Tensor] = None):
    """Append the rows k, v [rows, kv_heads, d] of a ragged batch (dq_paged_append); keys, and q beside them, are normed
    and rotated on the way.  starts: int32 [batch + 1], rows starts[b] .. starts[b+1] - 1 are sequence b's last tokens
    (None: one row each); seq_lens: int32, the new rows included; page_table: int32 [batch, pages].  positions None: a
    token's place in its sequence.  Returns q_out (None without q).  No gradients.  seq_lens may go back later within the page being filled or to
    a page's end; into a page that was quantized as PagedKVLayer.shorten does it."""
    if q is None:
        if q_out is not None:
            raise DQError("q_out without q")
    elif q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    index = cache.index
    _call(_module.paged_append, index, cache._at, index, k, v, starts, seq_lens, page_table, tail_slots, q, q_out,
          None if rotary is None else rotary._c, positions, q_weight, k_weight, eps)
    return q_out


def paged_read(cache: PagedCache, first: Optional[torch.Tensor], seq_lens: torch.Tensor, out_starts: torch.Tensor, page_table: torch.Tensor,
               k_out: torch.Tensor, v_out: torch.Tensor, tail_slots: Optional[torch.Tensor] = None):
    """The rows that tokens first[b] <= t < seq_lens[b] of the cache stand for, into k_out and v_out [rows, kv_heads, d]
    from row out_starts[b] to out_starts[b+1] - 1 at most (dq_paged_read; first None: from 0).  seq_lens: the sequences' own lengths, also
    for a read that ends earlier.  Returns (k_out, v_out)."""
    index = cache.index
    _call(_module.paged_read, index, cache._at, index, first, seq_lens, out_starts, page_table, tail_slots, k_out, v_out)
    return k_out, v_out


def _workspace_bytes(cache: PagedCache, batch: int, rows: int, q_heads: int, max_rows: int, max_seq_len: int) -> int:
    n = lib.dq_paged_workspace_bytes(C.byref(cache.c), batch, rows, q_heads, max_rows, max_seq_len)
    if n == 0:
        raise DQError("dq_paged_workspace_bytes rejected the arguments")
    return (n + 15) // 16 * 16


def _new_workspace(cache: PagedCache, n: int) -> torch.Tensor:
    ws = torch.empty(n, dtype=torch.uint8, device=cache.device)
    with torch.cuda.device(cache.device):
        workspace_init(ws)
    return ws


def paged_workspace(cache: PagedCache, batch: int, rows: int, q_heads: int, max_rows: int, max_seq_len: int) -> torch.Tensor:
    """Workspace of paged_attention for these sizes."""
    return _new_workspace(cache, _workspace_bytes(cache, batch, rows, q_heads, max_rows, max_seq_len))


def paged_attention(cache: PagedCache, q: torch.Tensor, starts: Optional[torch.Tensor], seq_lens: torch.Tensor, page_table: torch.Tensor,
                    max_rows: int, max_seq_len: int, workspace: torch.Tensor, out: Optional[torch.Tensor] = None, softmax_scale: float = 0.0,
                    causal: bool = True, window: int = 0, tail_slots: Optional[torch.Tensor] = None, splits: int = 0) -> torch.Tensor:
    """softmax(q . K * scale) V of the batch's rows q [rows, q_heads, d] over the cached tokens of their sequences
    (dq_paged_attention); rows are the last tokens of their sequence (append them first).  max_rows: host bound on the
    rows of any sequence; max_seq_len: on its tokens (a guess does).  window > 0: the last `window` tokens only.  out may be q.  No gradients.
    Rows of no sequence and a sequence's rows past max_rows are not written.  splits: launch override for sweeps (DQ_PAGED_SPLITS)."""
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    index = cache.index
    _call(_module.paged_attention, index, cache._at, index, q, out, starts, seq_lens, page_table, tail_slots, max_rows, max_seq_len,
          softmax_scale, causal, window, splits, workspace)
    return out


class PagedKVLayer:
    """One layer's keys and values in 8-bit pages, as KVCacheLayer is for the DecoQuant form: `batch` sequences of up to
    max_tokens tokens, each with its own pages and tail, the lengths on the device.  Rows come packed, sequence by
    sequence (`starts`, int32 [batch + 1]; None: one row each); the host tracks only bounds, which size the launches.
    Replays of a captured step count on the device only: add their rows to tokens_upper (which refuses what is too much;
    rows of replays past max_tokens' pages are left out).
    (Loops with a page allocator of their own call paged_append and paged_attention.)"""

    def __init__(self, batch: int, q_heads: int, kv_heads: int, head_dim: int, max_tokens: int, page_tokens: int = 64,
                 dtype=torch.float16, codes=torch.int8, device="cuda:0"):
        if min(batch, max_tokens, q_heads, kv_heads) < 1 or q_heads % kv_heads or page_tokens not in (64, 128):
            raise DQError("a layer has sequences, room for tokens, q_heads a multiple of kv_heads and pages of 64 or 128 tokens")
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
        q_out = None if q is None else torch.empty(q.shape, dtype=q.dtype, device=q.device)
        self.seq_lens += new
        try:
            q = paged_append(self.cache, k, v, starts, self.seq_lens, self.page_table, q=q, q_out=q_out, rotary=rotary, positions=positions,
                             q_weight=q_weight, k_weight=k_weight, eps=eps)
        except Exception:                   # whatever it was, nothing was launched
            self.seq_lens -= new
            raise
        self.tokens_upper += max_rows
        return q

    _fits = (0, 0)                          # rows of a call and of a sequence that the workspace is known to be enough for

    def _make_room(self, rows: int, max_rows: int) -> torch.Tensor:
        need = _workspace_bytes(self.cache, self.batch, rows, self.q_heads, max_rows, self.max_tokens)
        if self._ws is None or need > self._ws.numel():
            if torch.cuda.is_current_stream_capturing():
                # zeroed by the graph's replays only: this call's own, none for calls outside the graph
                self._outgrown.append(_new_workspace(self.cache, need))
                return self._outgrown[-1]
            if self._ws is not None:
                self._outgrown.append(self._ws)      # a captured graph may still work in it
                need = max(need, 2 * self._ws.numel())   # (all that were outgrown together are smaller than the next one)
            self._ws = _new_workspace(self.cache, need)
        self._fits = (rows, max_rows)
        return self._ws

    def attend(self, q: torch.Tensor, starts: Optional[torch.Tensor] = None, max_rows: int = 1, out: Optional[torch.Tensor] = None,
               softmax_scale: float = 0.0, causal: bool = True, window: int = 0) -> torch.Tensor:
        """Attention of the rows just appended, q [rows, q_heads, d] (paged_attention)."""
        bound = min(self.tokens_upper, self.max_tokens)
        ws = self._ws
        if q.shape[0] > self._fits[0] or max_rows > self._fits[1]:
            ws = self._make_room(max(q.shape[0], self._fits[0]), max(max_rows, self._fits[1]))
        return paged_attention(self.cache, q, starts, self.seq_lens, self.page_table, max_rows, bound, ws, out=out,
                               softmax_scale=softmax_scale, causal=causal, window=window)

    def shorten(self, lengths: Sequence[int]) -> None:
        """Drop tokens from the ends: sequence b keeps its first lengths[b] (host integers; 0 empties it), after drafted tokens
        were refused or a sequence ended.  In the page being filled nothing moves, and what is appended next gives the bits it
        would have given without them; where a page that was quantized becomes the last one again, its rows go back to the
        tail as what their codes stand for.  Looks at the device's lengths, so not for captures."""
        c, page = self.cache, self.cache.page_tokens
        have = [min(n, self.page_table.shape[1] * page) for n in self.seq_lens.tolist()]
        if len(lengths) != self.batch or any(not 0 <= n <= h for n, h in zip(lengths, have)):
            raise DQError("shorten needs a length for every sequence, at most its tokens")
        back = [n % page if n // page < h // page else 0 for n, h in zip(lengths, have)]
        lens = torch.tensor(list(lengths), dtype=torch.int32, device=c.device)
        if any(back):
            first = torch.tensor([n - b for n, b in zip(lengths, back)], dtype=torch.int32, device=c.device)
            starts = torch.tensor([sum(back[:b]) for b in range(self.batch + 1)], dtype=torch.int32, device=c.device)
            k, v = (torch.empty((sum(back), c.kv_heads, c.head_dim), dtype=c.dtype, device=c.device) for _ in range(2))
            paged_read(c, first, self.seq_lens, starts, self.page_table, k, v)
            paged_append(c, k, v, starts, lens, self.page_table)
        self.seq_lens.copy_(lens)
        self.tokens_upper = max(lengths)

    def read(self, lengths: Sequence[int]):
        """The rows the layer stands for, k and v [batch, kv_heads, max(lengths), d]; of sequence b the first lengths[b] (host
        integers) are written, the rest, and what lies behind its tokens, is zero.  Goes into KVCacheLayer.prefill (fp16 layers)."""
        c = self.cache
        if len(lengths) != self.batch or min(lengths) < 0:
            raise DQError("read needs a length for every sequence, none negative")
        k = torch.zeros((self.batch, c.kv_heads, max(lengths), c.head_dim), dtype=c.dtype, device=c.device)
        v = torch.zeros_like(k)
        rows = torch.tensor([[0, n] for n in lengths], dtype=torch.int32, device=c.device)
        slots = torch.arange(self.batch, dtype=torch.int32, device=c.device)
        for b in range(self.batch):
            if lengths[b]:                  # (the sequence's own length says which page is its tail, rows[b] where to stop)
                paged_read(c, None, self.seq_lens[b:b + 1], rows[b], self.page_table[b:b + 1], k[b].transpose(0, 1), v[b].transpose(0, 1),
                           tail_slots=slots[b:b + 1])
        return k, v
