"""Plain 64-bit forms of the head norm and rotation, of the paged 8-bit cache and of attention over it,
and inputs for their tests.  Written from the definitions in include/decoquant.h, on the CPU."""
import math

import torch

import paper_2405_12591_amd as dq

DEV = "cuda:0"
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}     # half a step relative to the value
QMAX = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def rows(shape, dtype, gen, outliers=True):
    """Rows on the CPU with a range per token and some wide channels; [..., heads, d]."""
    x = torch.randn(shape, generator=gen) * torch.exp(0.5 * torch.randn(*shape[:-1], 1, generator=gen))
    if outliers:
        x[..., ::37] *= 20
    return x.to(dtype)


def heads64(x, w, eps, inv, axis, positions, rot, interleaved):
    """x [rows, heads, d] -> float64 norm and rotation, and the size of the terms every channel is summed from."""
    y = x.double()
    if w is not None:
        y = y * w.double() / (y.square().mean(-1, keepdim=True) + eps).sqrt()
    mag = y.abs().clone()
    if rot:
        half = rot // 2
        pos = positions.reshape(-1, x.shape[0]).double()
        a = torch.zeros(half, dtype=torch.long) if axis is None else axis.long()
        ang = pos[a].t() * inv                                       # [rows, half]
        c, s = ang.cos()[:, None], ang.sin()[:, None]
        i = torch.arange(half)
        f, g = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        u, v = y[..., f].clone(), y[..., g].clone()
        y[..., f], y[..., g] = u * c - v * s, u * s + v * c
        mag[..., f] = mag[..., g] = u.abs() + v.abs()
    return y, mag


def rotate_tolerance(y, mag, dtype):
    """Half a step of the result; fp32 sums of up to 256 squares, and sines and cosines from an angle that fp32
    holds to 2^-22 radians and an instruction good to about 2^-19: 2^-17 of the terms; fp16's smallest step."""
    return y.abs() * HALF[dtype] + mag * 2.0 ** -17 + 2.0 ** -24


def e4m3(x):
    """To the nearest 8-bit float 1-4-3, ties to even, from float64."""
    unit = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -40))).clamp(min=-6) - 3)
    return (x / unit).round() * unit


def quantize64(x, codes):
    """A block [rows, d] (16-bit values in float64) -> codes as float64, the fp32 scale."""
    top = float(x.abs().max())
    if top < 2.0 ** -100:
        return torch.zeros_like(x), 1.0
    m, e = math.frexp(QMAX[codes] / top)
    r = math.ldexp(math.floor(m * 4096), e - 12)
    y = x * r
    return (y.round() if codes == torch.int8 else e4m3(y)), float(torch.tensor(1.0 / r, dtype=torch.float32))


class Sequences:
    """The tokens of a batch as plain lists of rows, and what the cache stands for."""

    def __init__(self, lens, heads, d, dtype, codes, page, gen, v_range=None):
        self.heads, self.d, self.dtype, self.codes, self.page = heads, d, dtype, codes, page
        self.k = [rows((n, heads, d), dtype, gen) for n in lens]
        self.v = [rows((n, heads, d), dtype, gen) for n in lens]
        if v_range is not None:                                     # very different scales from page to page
            for v in self.v:
                for i in range(0, len(v), page):
                    v[i:i + page] = (v[i:i + page].double() * 2.0 ** v_range[(i // page) % len(v_range)]).to(dtype)

    def stored(self, x, length=None):
        """[tokens, heads, d] float64: full pages quantized, the rest as it is."""
        n = len(x) if length is None else length
        out = x[:n].double().clone()
        for p in range(n // self.page):
            for h in range(self.heads):
                at = slice(p * self.page, (p + 1) * self.page)
                c, s = quantize64(out[at, h], self.codes)
                out[at, h] = c * s
        return out


def attend64(q, k, v, place, causal, window, scale):
    """q [rows, q_heads, d], k and v float64 [tokens, heads, d], place [rows].  Returns the result, what its terms
    add up to and how far scores in fp32 may be off, all [rows, q_heads, ...]."""
    g = q.shape[1] // k.shape[1]
    out = torch.zeros(q.shape, dtype=torch.float64)
    size, ds = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape[:2] + (1,), dtype=torch.float64)
    j = torch.arange(len(k))
    for h in range(q.shape[1]):
        kk, vv, qq = k[:, h // g], v[:, h // g], q[:, h].double()
        s = qq @ kk.t() * scale
        see = torch.ones_like(s, dtype=torch.bool)
        if causal:
            see &= j[None] <= place[:, None]
        if window:
            see &= j[None] > place[:, None] - window
        some = see.any(1)
        if not some.any():
            continue
        p = torch.softmax(s.masked_fill(~see, -math.inf)[some], 1)
        vz = torch.where(torch.isnan(vv), 0.0, vv)
        out[some, h] = p @ vz
        size[some, h] = p @ vz.abs()
        mag = (qq.abs() @ torch.nan_to_num(kk).abs().t() * scale).masked_fill(~see, 0)
        ds[some, h] = mag.amax(1, keepdim=True)[some]
    return out, size, ds


def attend_tolerance(out, size, ds, v_max, tokens, dtype, tail):
    """Half a step of the result; probabilities in f16 (in the rows' own type for the tail's tokens): half a step of
    every term, and their smallest step 2^-25 per token; scores: fp32 sums of 128 products, off by 2^-17 of the sum
    of their sizes at the most, twice (numerator and sum); 2^-18 for exponentials, scales and the sums over tokens."""
    half_p = HALF[dtype] if tail else 2.0 ** -11
    return out.abs() * HALF[dtype] + size * (half_p + 2.0 ** -18 + 2 * 2.0 ** -17 * ds) + tokens * 2.0 ** -25 * v_max + 2.0 ** -24


def device_tables(lens, page, gen, extra=2, width=None):
    """A page table over a shuffled pool; (int32 [B, width] on the device, pages in the pool)."""
    need = [-(-n // page) for n in lens]
    pool = sum(need) + extra
    order = torch.randperm(pool, generator=gen).to(torch.int32)
    table = torch.full((len(lens), max(1, max(need) if width is None else width)), -7, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table.to(DEV), pool


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def fill_tails(cache, value=float("nan")):
    """A tail's rows behind the last token may hold anything."""
    cache.t["k_tail"].fill_(value)
    cache.t["v_tail"].fill_(value)


def filled_cache(seqs, lens, gen, slots=None, poison=True, extra=2):
    """A cache that holds the sequences, appended in one call; (cache, table, tail_slots)."""
    table, pool = device_tables(lens, seqs.page, gen, extra)
    b = len(lens)
    cache = dq.alloc_paged_cache(pool, b + 2, seqs.heads, seqs.d, seqs.page, seqs.dtype, seqs.codes, DEV)
    if poison:
        fill_tails(cache)
        for n in ("k_scales", "v_scales"):
            cache.t[n].fill_(float("nan"))
    slots = (torch.randperm(b + 2, generator=gen)[:b].to(torch.int32)).to(DEV) if slots is None else slots
    starts = [0]
    for n in lens:
        starts.append(starts[-1] + n)
    k, v = torch.cat(seqs.k).to(DEV), torch.cat(seqs.v).to(DEV)
    dq.paged_append(cache, k, v, ints(starts), ints(lens), table, tail_slots=slots)
    return cache, table, slots


def read_back(cache, lens, table, slots, first=None):
    first = [0] * len(lens) if first is None else first
    starts = [0]
    for n, f in zip(lens, first):
        starts.append(starts[-1] + max(n - f, 0))
    k = torch.full((starts[-1], cache.kv_heads, cache.head_dim), 7.0, dtype=cache.dtype, device=DEV)
    v = k.clone()
    dq.paged_read(cache, ints(first), ints(lens), ints(starts), table, k, v, tail_slots=slots)
    return k.cpu(), v.cpu(), starts
