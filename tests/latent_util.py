"""Plain 64-bit forms of the cache of latents and of attention over it, written from the definitions in include/decoquant.h, on the
CPU, and inputs for their tests."""
import math

import torch

import paper_2405_12591_amd as dq
from paged_util import DEV, HALF, ints

FORMS = {512: 64, 256: 32}


def starts_of(counts, gap=0):
    out = [gap]
    for n in counts:
        out.append(out[-1] + n)
    return out


def normal(shape, dtype, gen, spread=0.5):
    x = torch.randn(shape, generator=gen) * torch.exp(spread * torch.randn(*shape[:-1], 1, generator=gen))
    return x.to(dtype)


def attend64(q, k, v, see, scale):
    """q [rows, heads, d], k [tokens, d], v [tokens, e] (or [tokens, heads, ..]), see bool [rows, tokens].  The result, what its terms
    add up to and the size of the sums that scores are, [rows, heads, ...], in float64.  Hidden tokens have no part in it."""
    rows, heads = q.shape[:2]
    e = v.shape[-1]
    out, size, ds = torch.zeros(rows, heads, e, dtype=torch.float64), torch.zeros(rows, heads, e, dtype=torch.float64), torch.zeros(rows, heads, 1, dtype=torch.float64)
    for h in range(heads):
        kk, vv = (k[:, h], v[:, h]) if k.dim() == 3 else (k, v)
        for i in range(rows):
            at = see[i].nonzero()[:, 0]
            if not len(at):
                continue
            s = kk[at].double() @ q[i, h].double() * scale
            p = torch.softmax(s, 0)
            out[i, h], size[i, h] = p @ vv[at].double(), p @ vv[at].double().abs()
            ds[i, h] = (kk[at].double().abs() @ q[i, h].double().abs() * scale).max()
    return out, size, ds


def tolerance(out, size, ds, v_max, tokens, dtype):
    """Half a step of the result; probabilities in the rows' type: half a step of every term, and f16's smallest step 2^-25 for each token;
    scores: up to 36 matrix instructions of 16 products, four roundings each, 2^-16.8 of the sum of their sizes at the most, twice
    (numerator and sum); 2^-18 for exponentials and the sums over tokens."""
    return out.abs() * HALF[dtype] + size * (HALF[dtype] + 2.0 ** -18 + 2 * 2.0 ** -16.8 * ds) + tokens * 2.0 ** -25 * v_max + 2.0 ** -24


class Latents:
    """A batch's rows on the CPU and a cache of them on the device: pages in any order, everything else in the pool NaN."""

    def __init__(self, lens, latent, dtype, page, gen, extra=2):
        self.lens, self.latent, self.rot, self.dtype, self.page = lens, latent, FORMS[latent], dtype, page
        w = latent + self.rot
        self.rows = [normal((n, w), dtype, gen) for n in lens]
        for r in self.rows:
            r[:, 3:latent:37] *= 8
        need = [-(-n // page) for n in lens]
        self.pool = sum(need) + extra
        order = torch.randperm(self.pool, generator=gen).to(torch.int32)
        self.table = torch.full((len(lens), max(1, max(need))), -7, dtype=torch.int32)
        pages = torch.full((self.pool, page, w), float("nan"), dtype=dtype)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
            for j in range(n):
                part = self.rows[b][j * page:(j + 1) * page]
                pages[int(self.table[b, j]), :len(part)] = part
        self.cache = dq.LatentCache(pages.to(DEV), latent)

    def attend(self, q, counts, scale, gap=0, causal=True, seen=None, max_rows=None, max_len=None, out=None, table=None, ws=None):
        """The device's result, rows of no sequence filled with 7."""
        total, heads = q.shape[:2]
        max_rows = max(counts) if max_rows is None else max_rows
        max_len = max(self.lens) if max_len is None else max_len
        if ws is None:
            ws = dq.latent_workspace(self.cache, len(counts), total, heads, max_rows, max_len)
            ws.fill_(255)                                           # nothing in it counts (NaN)
        out = torch.full((total, heads, self.latent), 7.0, dtype=self.dtype, device=DEV) if out is None else out
        starts = None if counts is None else ints(starts_of(counts, gap))
        dq.latent_attention(self.cache, q, starts, ints(self.lens), (self.table if table is None else table).to(DEV), max_rows, max_len, scale, ws,
                            out=out, causal=causal, seen=None if seen is None else seen.to(DEV))
        return out

    def want(self, q, counts, scale, gap=0, causal=True, seen=None):
        """float64 result, tolerance of it, and which rows belong to a sequence."""
        total, heads = q.shape[:2]
        out = torch.full((total, heads, self.latent), 7.0, dtype=torch.float64)
        tol, own = torch.zeros_like(out), torch.zeros(total, dtype=torch.bool)
        at = gap
        for b, c in enumerate(counts):
            rows, n = self.rows[b], self.lens[b]
            j, place = torch.arange(n), n - c + torch.arange(c)
            see = j[None] <= place[:, None] if causal else torch.ones(c, n, dtype=torch.bool)
            if seen is not None:
                for i in range(c):
                    for t in range(max(n - c, 0), n):
                        see[i, t] = bool(int(seen[at + i]) >> (t - (n - c)) & 1)
            o, size, ds = attend64(q[at:at + c], rows, rows[:, :self.latent], see, scale)
            v_max = float(rows[:, :self.latent].double().abs().max()) if n else 0.0
            out[at:at + c], tol[at:at + c], own[at:at + c] = o, tolerance(o, size, ds, v_max, n, self.dtype), True
            at += c
        return out, tol, own


def check(got, want, tol, own, what=""):
    got = got.double().cpu()
    assert torch.equal(got[~own], want[~own]), "%s: rows of no sequence" % what
    err = (got - want).abs()
    bad = ~(err <= tol)
    assert not bool(bad.any()), "%s: %d of %d off, worst %g of its tolerance" % (what, int(bad.sum()), bad.numel(), float((err / tol.clamp(min=1e-30)).nan_to_num(1e9).max()))
