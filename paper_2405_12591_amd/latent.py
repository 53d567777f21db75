"""Binding of attention over one latent vector a token (include/decoquant.h): the paged cache of latents with its append, read-back and
absorbed attention, and attention over expanded keys and values.  Argument checks and marshalling only, the checks of tensors
in csrc/paged_bind.cpp.  These operators serve: tensors that require gradients are taken as they are, outputs carry none."""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence

import torch

from .binding import DQError, lib
from .paged import _DTYPES, Rotary, _Workspace, _call, _module


class _CLatent(C.Structure):
    _fields_ = [("rows", C.c_void_p), ("pages", C.c_int32), ("page_tokens", C.c_int32), ("latent_dim", C.c_int32), ("rot_dim", C.c_int32),
                ("dtype", C.c_int32)]


def _declare() -> None:
    i32, i64, f32, u32, size, ptr = C.c_int32, C.c_int64, C.c_float, C.c_uint32, C.c_size_t, C.c_void_p
    cache = C.POINTER(_CLatent)
    batch = heads = rot = ptr
    lib.dq_latent_append.restype = i32
    lib.dq_latent_append.argtypes = [cache, batch, ptr, i64, ptr, i64, ptr, f32, heads, heads, rot, ptr]
    lib.dq_latent_read.restype = i32
    lib.dq_latent_read.argtypes = [cache, batch, ptr, ptr, ptr, i64, ptr]
    lib.dq_latent_workspace_bytes.restype = size
    lib.dq_latent_workspace_bytes.argtypes = [cache, i32, i32, i32, i32, i32]
    lib.dq_latent_attention.restype = i32
    lib.dq_latent_attention.argtypes = [cache, batch, heads, heads, ptr, i32, i32, f32, ptr, size, u32, ptr]
    lib.dq_expanded_workspace_bytes.restype = size
    lib.dq_expanded_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32]
    lib.dq_expanded_attention.restype = i32
    lib.dq_expanded_attention.argtypes = [ptr, i32, i32, f32, ptr, size, u32, ptr]


_declare()

LATENT_FORMS = ((512, 64), (256, 32))     # channels of the latent and of the shared, rotated key


class LatentCache:
    """Device tensor of a layer's paged cache of latents, rows [pages, P, latent_dim + rot_dim] (float16 or bfloat16, P 64 or 128),
    plus the C struct that points at it (dq_latent_cache)."""

    def __init__(self, rows: torch.Tensor, latent_dim: int):
        if rows.dim() != 3 or (latent_dim, rows.shape[2] - latent_dim) not in LATENT_FORMS or rows.shape[1] not in (64, 128):
            raise DQError("rows must be [pages, 64 or 128, latent_dim + rot_dim], of 512 + 64 or 256 + 32 channels")
        if rows.dtype not in _DTYPES or not (rows.is_cuda and rows.is_contiguous()) or rows.data_ptr() % 16 or not rows.shape[0]:
            raise DQError("rows must be a contiguous, 16-byte aligned float16 or bfloat16 device tensor of at least one page")
        if rows.shape[0] >= 1 << 31:
            raise DQError("too many pages")
        self.rows, self.latent_dim, self.rot_dim = rows, latent_dim, rows.shape[2] - latent_dim
        self.pages, self.page_tokens, self.dtype, self.device, self.index = rows.shape[0], rows.shape[1], rows.dtype, rows.device, rows.get_device()
        self.c = _CLatent(rows.data_ptr(), self.pages, self.page_tokens, self.latent_dim, self.rot_dim, _DTYPES[self.dtype])
        self._at = C.addressof(self.c)

    def nbytes(self) -> int:
        return self.rows.numel() * self.rows.element_size()


def alloc_latent_cache(pages: int, latent_dim: int = 512, rot_dim: int = 64, page_tokens: int = 64, dtype=torch.bfloat16,
                       device="cuda:0") -> LatentCache:
    """A paged cache of latents."""
    if pages < 1 or (latent_dim, rot_dim) not in LATENT_FORMS or page_tokens not in (64, 128):
        raise DQError("a cache of latents has pages of 64 or 128 tokens and 512 + 64 or 256 + 32 channels")
    return LatentCache(torch.zeros((pages, page_tokens, latent_dim + rot_dim), dtype=dtype, device=device), latent_dim)


def latent_append(cache: LatentCache, latent: torch.Tensor, k_rot: torch.Tensor, starts: Optional[torch.Tensor], seq_lens: torch.Tensor,
                  page_table: torch.Tensor, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                  rotary: Optional[Rotary] = None, positions: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
                  eps: float = 1e-6):
    """Append the rows of a ragged batch (dq_latent_append): latent [rows, latent_dim], normed where a weight is given, and k_rot [rows,
    rot_dim], rotated where a rotation is; q [rows, heads, rot_dim], the queries' channels that meet k_rot, takes the same rotation
    on the way, into q_out, which may be q itself and shares no memory with the others.  Rows are views of a fused projection as
    they lie there.  starts: int32 [batch + 1], rows starts[b] .. starts[b+1] - 1 are sequence b's last tokens (None: one row each);
    seq_lens: int32, the new rows included; page_table: int32 [batch, pages].  positions None: a token's place in its sequence.
    Returns q_out (None without q).  Rows of no sequence stay as they are.  seq_lens may go back at will: rows behind a sequence's
    end are never read."""
    if q is None:
        if q_out is not None:
            raise DQError("q_out without q")
    elif q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    index = cache.index
    _call(_module.latent_append, index, cache._at, index, latent, k_rot, starts, seq_lens, page_table, q, q_out,
          None if rotary is None else rotary._c, positions, weight, eps)
    return q_out


def latent_read(cache: LatentCache, first: Optional[torch.Tensor], seq_lens: torch.Tensor, out_starts: torch.Tensor, page_table: torch.Tensor,
                out: torch.Tensor) -> torch.Tensor:
    """The rows of tokens first[b] <= t < seq_lens[b] into out [rows, latent_dim + rot_dim], from row out_starts[b] to out_starts[b+1] - 1
    at most (dq_latent_read; first None: from 0): what expanded_attention's keys and values are expanded from."""
    index = cache.index
    _call(_module.latent_read, index, cache._at, index, first, seq_lens, out_starts, page_table, out)
    return out


def _workspace_bytes(cache: LatentCache, batch: int, rows: int, q_heads: int, max_rows: int, max_seq_len: int) -> int:
    n = lib.dq_latent_workspace_bytes(C.byref(cache.c), batch, rows, q_heads, max_rows, max_seq_len)
    if n == 0:
        raise DQError("dq_latent_workspace_bytes rejected the arguments")
    return n


def latent_workspace(cache: LatentCache, batch: int, rows: int, q_heads: int, max_rows: int, max_seq_len: int) -> torch.Tensor:
    """Workspace of latent_attention for these sizes and all smaller ones with the same heads: 17 to 135 MB for 512 channels, by the columns max_rows *
    q_heads alone.  Calls that share it must be ordered; a model's layers are."""
    return torch.empty(_workspace_bytes(cache, batch, rows, q_heads, max_rows, max_seq_len), dtype=torch.uint8, device=cache.device)


def latent_attention(cache: LatentCache, q: torch.Tensor, starts: Optional[torch.Tensor], seq_lens: torch.Tensor, page_table: torch.Tensor,
                     max_rows: int, max_seq_len: int, softmax_scale: float, workspace: torch.Tensor, out: Optional[torch.Tensor] = None,
                     causal: bool = True, seen: Optional[torch.Tensor] = None) -> torch.Tensor:
    """softmax(q . [c | k_rot] * softmax_scale) c of the batch's rows q [rows, heads, latent_dim + rot_dim] over the cached tokens of their
    sequences, [rows, heads, latent_dim] (dq_latent_attention); rows are the last tokens of their sequence (append them first).
    max_rows: host bound on the rows of any sequence; max_seq_len: on its tokens (any will do: it is not looked at).  seen: int64, a mask for each row: bit j
    names the j-th row of the sequence (a tree of drafted tokens; at most 64 rows); None: every row up to its own place.
    Rows of no sequence and a sequence's rows past max_rows are not written.  No gradients."""
    if out is None:
        out = torch.empty(q.shape[:2] + (cache.latent_dim,), dtype=q.dtype, device=q.device)
    index = cache.index
    _call(_module.latent_attention, index, cache._at, index, q, out, starts, seq_lens, page_table, seen, max_rows, max_seq_len, softmax_scale,
          causal, workspace)
    return out


def expanded_workspace(batch: int, rows: int, heads: int, head_dim: int, max_rows: int, max_seq_len: int, device="cuda:0") -> torch.Tensor:
    """Workspace of expanded_attention for these sizes and all smaller ones with the same heads."""
    n = lib.dq_expanded_workspace_bytes(batch, rows, heads, head_dim, max_rows, max_seq_len)
    if n == 0:
        raise DQError("dq_expanded_workspace_bytes rejected the arguments")
    return torch.empty(n, dtype=torch.uint8, device=device)


def expanded_attention(q: torch.Tensor, k: torch.Tensor, k_rot: torch.Tensor, v: torch.Tensor, starts: torch.Tensor, kv_starts: torch.Tensor,
                       max_rows: int, max_seq_len: int, workspace: torch.Tensor, out: Optional[torch.Tensor] = None,
                       softmax_scale: float = 0.0, causal: bool = True) -> torch.Tensor:
    """softmax((q . [k | k_rot]) * scale) v of ragged prompts (dq_expanded_attention): q [rows, heads, d + d / 2], k and v [tokens, heads, d],
    k_rot [tokens, d / 2] for all heads, d 128 or 64; views of one projection as they lie.  starts, kv_starts: int32 [batch + 1],
    the rows and the tokens of each sequence; its rows are its last tokens.  max_rows: host bound on the rows of any sequence;
    max_seq_len: on its tokens (a guess does).  softmax_scale <= 0: 1 / sqrt(d + d / 2).  Rows of no sequence and a sequence's rows past
    max_rows are not written.  No gradients."""
    if out is None:
        out = torch.empty(q.shape[:2] + v.shape[2:], dtype=q.dtype, device=q.device)
    index = q.get_device()
    _call(_module.expanded_attention, index, index, q, k, k_rot, v, out, starts, kv_starts, max_rows, max_seq_len, softmax_scale, causal, workspace)
    return out


class LatentKVLayer:
    """One layer's latents, as PagedKVLayer is for keys and values of their own: `batch` sequences of up to max_tokens tokens, each with its own
    pages, the lengths on the device.  Rows come packed, sequence by sequence (`starts`, int32 [batch + 1]; None: one row each);
    the host tracks only a bound, which sizes the launches.  Replays of a captured step count on the device only: add their rows to
    tokens_upper.  workspace_of: another layer, in whose workspace (17 to 135 MB, by the columns) this one works too, where their calls are
    ordered, as a model's layers' are.  (Loops with a page allocator of their own call latent_append and latent_attention.)"""

    def __init__(self, batch: int, heads: int, max_tokens: int, latent_dim: int = 512, rot_dim: int = 64, page_tokens: int = 64,
                 dtype=torch.bfloat16, device="cuda:0", workspace_of: Optional["LatentKVLayer"] = None):
        if min(batch, heads, max_tokens) < 1 or page_tokens not in (64, 128):
            raise DQError("a layer has sequences, heads, room for tokens and pages of 64 or 128 tokens")
        self.batch, self.heads, self.max_tokens = batch, heads, max_tokens
        width = -(-max_tokens // page_tokens)
        self.cache = alloc_latent_cache(batch * width, latent_dim, rot_dim, page_tokens, dtype, device)
        self.page_table = torch.arange(batch * width, dtype=torch.int32, device=device).view(batch, width)
        self.seq_lens = torch.zeros(batch, dtype=torch.int32, device=device)
        self.tokens_upper = 0               # no sequence holds more tokens than this (host-side bound)
        self._ws = _Workspace.made_or_shared(self.cache.device, workspace_of, LatentKVLayer, "_ws")

    def append(self, latent: torch.Tensor, k_rot: torch.Tensor, starts: Optional[torch.Tensor] = None, max_rows: int = 1,
               q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None, rotary: Optional[Rotary] = None,
               positions: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None, eps: float = 1e-6):
        """Append rows, no sequence more than max_rows; norm, rotation and the queries' channels as latent_append takes them.  Returns
        q_out (None without q)."""
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
            q = latent_append(self.cache, latent, k_rot, starts, self.seq_lens, self.page_table, q=q, q_out=q_out, rotary=rotary,
                              positions=positions, weight=weight, eps=eps)
        except Exception:                   # whatever it was, nothing was launched
            self.seq_lens -= new
            raise
        self.tokens_upper += max_rows
        return q

    def attend(self, q: torch.Tensor, softmax_scale: float, starts: Optional[torch.Tensor] = None, max_rows: int = 1,
               out: Optional[torch.Tensor] = None, causal: bool = True, seen: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Absorbed attention of the rows just appended, q [rows, heads, latent_dim + rot_dim] (latent_attention)."""
        bound = min(self.tokens_upper, self.max_tokens)
        ws = self._ws.of(_workspace_bytes(self.cache, self.batch, q.shape[0], self.heads, max_rows, bound))
        return latent_attention(self.cache, q, starts, self.seq_lens, self.page_table, max_rows, bound, softmax_scale, ws, out=out, causal=causal,
                                seen=seen)

    def shorten(self, lengths: Sequence[int]) -> None:
        """Drop tokens from the ends: sequence b keeps its first lengths[b] (host integers).  Rows stay where they are until others
        take their places; a drafted path is kept by appending its rows again behind the shortened lengths.  Looks at the device's
        lengths, so not for captures."""
        have = [min(n, self.page_table.shape[1] * self.cache.page_tokens) for n in self.seq_lens.tolist()]
        if len(lengths) != self.batch or any(not 0 <= n <= h for n, h in zip(lengths, have)):
            raise DQError("shorten needs a length for every sequence, at most its tokens")
        self.seq_lens.copy_(torch.tensor(list(lengths), dtype=torch.int32))
        self.tokens_upper = max(lengths)

    def read(self, lengths: Sequence[int]):
        """The first lengths[b] rows (host integers) of every sequence b, packed, [sum, latent_dim + rot_dim], and their int32 starts: what a
        prompt's keys and values are expanded from (expanded_attention's kv_starts)."""
        if len(lengths) != self.batch or min(lengths) < 0:
            raise DQError("read needs a length for every sequence, none negative")
        c = self.cache
        starts = torch.tensor([sum(lengths[:b]) for b in range(self.batch + 1)], dtype=torch.int32, device=c.device)
        out = torch.zeros((sum(lengths), c.latent_dim + c.rot_dim), dtype=c.dtype, device=c.device)
        return latent_read(c, None, self.seq_lens, starts, self.page_table, out), starts
