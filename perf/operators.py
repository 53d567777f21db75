"""Serving attention over a paged cache held in 8 bits, from the raw projections to the output.

Three kinds of case, all on the ragged batches a serving loop has (rows of all sequences one behind the
other, `starts` says where each begins; `lens` counts a sequence's tokens with the new ones):

  rotate   RMS norm and position rotation of every query and key head of a fused projection's rows
  append   the new rows go into the cache: keys normed and rotated on the way, queries too; pages that
           fill are quantized.  What the cache then stands for in the touched pages is read back as rows
  attend   softmax(q K^T / sqrt(d)) V over pages and the 16-bit rows of the last, not yet full page

Layout of the cache (P tokens a page, H kv heads, D channels; 64 tokens of values are kept channel by
channel):
  k_codes [pages, H, P, D]    v_codes [pages, H, P / 64, D, 64]    k_scales, v_scales f32 [pages, H]
  k_tail  [slots, H, P, D]    v_tail  [slots, H, P / 64, D, 64]    16-bit rows of the page being filled
A block is a page's rows of one head.  Its inverse step r is Q / max|x| (Q = 127 for int8, 448 for e4m3)
cut off behind 12 significant bits, so that x * r is exact in 32 bits and no code lies on a border by
chance; a code is round(x * r) and stands for code * scale, scale = 1 / r.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
QMAX = {"e4m3": 448.0, "int8": 127.0}
EPS = 1e-6
BASE = 10000.0


# ------------------------------------------------------------------------------------------------
# The cases
# ------------------------------------------------------------------------------------------------
def _rotate(dtype, dim, q_heads, kv_heads, batch, tokens, rot, axes=1, interleaved=False, norm=True):
    return {"kind": "rotate", "dtype": dtype, "dim": dim, "q_heads": q_heads, "kv_heads": kv_heads, "batch": batch,
            "new_lo": tokens, "new_hi": tokens, "rot": rot, "axes": axes, "interleaved": interleaved, "norm": norm}


def _append(dtype, codes, dim, page, q_heads, kv_heads, batch, old, new_lo, new_hi, rot, norm, axes=1, interleaved=False):
    return {"kind": "append", "dtype": dtype, "codes": codes, "dim": dim, "page": page, "q_heads": q_heads,
            "kv_heads": kv_heads, "batch": batch, "old": old, "new_lo": new_lo, "new_hi": new_hi, "rot": rot,
            "axes": axes, "interleaved": interleaved, "norm": norm}


def _attend(dtype, codes, dim, page, q_heads, kv_heads, batch, lo, hi, new_lo=1, new_hi=1, window=0):
    return {"kind": "attend", "dtype": dtype, "codes": codes, "dim": dim, "page": page, "q_heads": q_heads,
            "kv_heads": kv_heads, "batch": batch, "lo": lo, "hi": hi, "new_lo": new_lo, "new_hi": new_hi, "window": window}


def listed():
    named = [
        # one generated token of each of 16 sequences, grouped heads: latency and host work
        ("rotate_step", _rotate("bf16", 128, 32, 8, 16, 1, 128)),
        # a long prompt with images: three position axes on a grouped layer, 16384 tokens
        ("rotate_axes", _rotate("bf16", 128, 32, 8, 4, 4096, 128, axes=3)),
        # heads of 64 channels, half of them rotated in neighbouring pairs, no norm, an odd length
        ("rotate_partial", _rotate("f16", 64, 32, 32, 1, 2999, 32, interleaved=True, norm=False)),
        # one generated token per sequence buffered at odd lengths; some of the pages fill
        ("append_step", _append("bf16", "e4m3", 128, 64, 32, 8, 16, 8001, 1, 1, 128, True)),
        # prompts of mixed lengths on the 7B-shaped layer
        ("append_prompt", _append("f16", "int8", 128, 128, 32, 32, 8, 0, 3000, 4096, 128, False)),
        # a conversation goes on: pieces of odd lengths behind caches that end inside a page
        ("append_chunk", _append("bf16", "e4m3", 128, 64, 32, 8, 16, 1543, 100, 777, 128, True)),
        # the smallest call: one short sequence, four heads of 64 channels
        ("attend_tiny", _attend("f16", "int8", 64, 64, 4, 4, 1, 257, 257)),
        # the 13B-shaped layer: 40 heads, sequences of mixed, odd lengths, int8 codes
        ("attend_ragged", _attend("f16", "int8", 128, 128, 40, 40, 4, 8192, 16384)),
        # long context, four query heads per kv head
        ("attend_gqa4_long", _attend("bf16", "e4m3", 128, 64, 32, 8, 16, 32768, 32768)),
        # drafted tokens checked against a windowed cache: four queries a sequence
        ("attend_draft", _attend("bf16", "e4m3", 64, 64, 32, 8, 8, 2048, 9001, 4, 4, window=4096)),
        # whole prompts, causal: bound by the matrix products
        ("attend_prompt", _attend("bf16", "e4m3", 128, 64, 32, 8, 4, 3500, 4096, 3500, 4096)),
        # a piece of a prompt behind a long cache
        ("attend_chunk", _attend("f16", "int8", 128, 128, 32, 8, 2, 15000, 16384, 400, 512)),
    ]
    return [dict(c, name=n) for n, c in named]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["rotate", "append", "append", "attend", "attend", "attend", "attend"])
    dim = rng.choice([128, 128, 64])
    dtype, codes, page = rng.choice(["bf16", "f16"]), rng.choice(["e4m3", "int8"]), rng.choice([64, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16, 32, 40])
    q_heads = kv_heads * (rng.choice([1, 2, 3, 4, 8]) if kv_heads <= 8 else 1)
    batch = _log_int(rng, 1, 16)
    rot, axes = rng.choice([dim, dim, dim // 2]), rng.choice([1, 1, 1, 3])
    interleaved, norm = rng.random() < 0.3, rng.random() < 0.6
    if kind == "rotate":
        tokens = _log_int(rng, 1, max(2, 16384 * 40 // (batch * (q_heads + kv_heads))))
        return _rotate(dtype, dim, q_heads, kv_heads, batch, tokens, rot, axes, interleaved, norm)
    if kind == "append":
        old = 0 if rng.random() < 0.4 else _log_int(rng, 1, 8000)
        new = 1 if rng.random() < 0.4 else _log_int(rng, 2, max(3, min(4096, 8 * 4096 * 32 // (batch * kv_heads), 8 * 4096 * 64 // (batch * (q_heads + kv_heads)))))
        lo = new if rng.random() < 0.4 else max(1, int(new * rng.uniform(0.1, 1.0)))
        return _append(dtype, codes, dim, page, q_heads, kv_heads, batch, old, lo, new, rot, norm, axes, interleaved)
    hi = _log_int(rng, 1, max(300, min(32768, 16 * 8 * 32768 // (batch * max(kv_heads, q_heads // 4)))))
    lo = hi if rng.random() < 0.4 else max(1, int(hi * rng.uniform(0.3, 1.0)))
    # queries: a generated token, a few drafted ones, or a prompt; visible (query, key) pairs stay under attend_prompt's
    most = 4 * 4096 * 4096 * 32 // (batch * q_heads * hi)
    new = rng.choice([1, 1, 1, rng.randint(2, 8), _log_int(rng, 9, max(10, min(lo, most)))])
    new = max(1, min(new, lo, max(1, most)))
    new_lo = new if rng.random() < 0.6 else max(1, int(new * rng.uniform(0.3, 1.0)))
    window = _log_int(rng, 16, 8192) if rng.random() < 0.15 else 0
    return _attend(dtype, codes, dim, page, q_heads, kv_heads, batch, lo, hi, new_lo, new, window)


def _spread(lo, hi, n):
    """n sizes over [lo, hi], the first one hi, odd ones among them."""
    return [hi - int((hi - lo) * ((i * 0.618034) % 1.0)) for i in range(n)]


def _counts(case):
    """New rows of every sequence."""
    return _spread(case["new_lo"], case["new_hi"], case["batch"])


def _old(case):
    """Tokens of every sequence before the new ones: `old` and some odd number more, none where it is 0."""
    if case["kind"] == "rotate":
        return [37 * i for i in range(case["batch"])]
    if case["kind"] == "append":
        return [case["old"] + (9 * i if case["old"] else 0) for i in range(case["batch"])]
    return [n - c for n, c in zip(_spread(case["lo"], case["hi"], case["batch"]), _counts(case))]


def _lens(case):
    return [a + b for a, b in zip(_old(case), _counts(case))]


# ------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------
def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _sums(values):
    out = [0]
    for v in values:
        out.append(out[-1] + v)
    return out


def _amp(heads, dim, gen):
    """[heads, dim] channel ranges: 1, and 20 on a few channels of every head, as keys have them."""
    amp = torch.ones(heads, dim, device=DEV)
    ch = torch.rand(heads, dim, device=DEV, generator=gen).argsort(1)[:, :dim // 32]
    return amp.scatter_(1, ch, 20.0)


def _random_rows(n, heads, dim, gen, amp):
    """f32 [n, heads, dim]: normal, a range per token, outlier channels."""
    x = torch.randn(n, heads, dim, device=DEV, generator=gen)
    return x * torch.exp(0.5 * torch.randn(n, heads, 1, device=DEV, generator=gen)) * amp


def _store(x, codes):
    """f32 blocks [..., rows, channels] -> codes and their scales [...], by the rule above."""
    top = x.abs().amax((-1, -2))
    r = (QMAX[codes] / torch.where(top > 0, top, torch.ones_like(top))).view(torch.int32).bitwise_and(~0xfff).view(torch.float32)
    r = torch.where(top > 0, r, torch.ones_like(r))
    y = x * r[..., None, None]
    return y.round().to(torch.int8) if codes == "int8" else y.to(torch.float8_e4m3fn), 1 / r


def _by_channel(x):
    """[..., P, D] -> [..., P / 64, D, 64]"""
    return x.unflatten(-2, (-1, 64)).transpose(-1, -2).contiguous()


def _by_token(x):
    """[..., P / 64, D, 64] -> [..., P, D]"""
    return x.transpose(-1, -2).flatten(-3, -2)


def _raw(x):
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _rotation(case, gen):
    """Frequencies (64 bits), the axis of every pair, positions [axes, T] of the new rows."""
    half, axes = case["rot"] // 2, case["axes"]
    inv = BASE ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
    axis = torch.zeros(half, dtype=torch.uint8, device=DEV)
    if axes == 3:      # time, height, width: a quarter of the pairs and three eighths twice
        axis[half // 4:] = 1
        axis[half // 4 + 3 * half // 8:] = 2
    pos = torch.cat([torch.arange(o, o + c, device=DEV) for o, c in zip(_old(case), _counts(case))])
    if case["kind"] == "rotate":
        pos = pos * 7 + torch.randint(4096, (1,), device=DEV, generator=gen)     # far positions too
    pos = pos[None]
    if axes == 3:      # an image's rows and columns beside the time
        pos = torch.cat([pos, pos + torch.arange(pos.shape[1], device=DEV) // 40 % 40, pos + torch.arange(pos.shape[1], device=DEV) % 40])
    return inv, axis, pos.to(torch.int32)


def _inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    kind, d, hq, h, bsz = case["kind"], case["dim"], case["q_heads"], case["kv_heads"], case["batch"]
    dtype = DTYPES[case["dtype"]]
    counts, lens = _counts(case), _lens(case)
    total = sum(counts)
    s = {"case": case, "starts": _ints(_sums(counts)), "lens": _ints(lens), "max_new": max(counts), "max_len": max(lens)}
    if kind != "attend":
        # what a fused projection leaves: a token's query, key and value heads side by side
        qkv = torch.empty(total, hq + 2 * h, d, dtype=dtype, device=DEV)
        qkv[:, :hq] = torch.randn(total, hq, d, device=DEV, generator=gen).to(dtype)
        for lo in (hq, hq + h):
            qkv[:, lo:lo + h] = _random_rows(total, h, d, gen, _amp(h, d, gen)).to(dtype)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + h], qkv[:, hq + h:]
        s["inv"], s["axis"], s["pos"] = _rotation(case, gen)
        s["wq"] = s["wk"] = None
        if case["norm"]:
            s["wq"], s["wk"] = (1 + 0.2 * torch.randn(2, d, device=DEV, generator=gen)).to(dtype)
    if kind == "rotate":
        return s
    p, codes = case["page"], case["codes"]
    need = [-(-n // p) for n in lens]
    pool = sum(need) + 3
    order = torch.randperm(pool, device=DEV, generator=gen).to(torch.int32)
    s["table"] = torch.zeros(bsz, max(need), dtype=torch.int32, device=DEV)
    for b, at in enumerate(_sums(need)[:-1]):
        s["table"][b, :need[b]] = order[at:at + need[b]]
    s["slots"] = torch.randperm(bsz, device=DEV, generator=gen).to(torch.int32)
    for x in "kv":
        amp = _amp(h, d, gen)
        c = torch.empty(pool, h, p, d, dtype=CODES[codes], device=DEV)
        c = c if x == "k" else c.view(pool, h, p // 64, d, 64)
        scales = torch.empty(pool, h, device=DEV)
        if kind == "attend":
            for at in range(0, pool, 1024):
                n = min(1024, pool - at)
                rows = _random_rows(n * p, h, d, gen, amp).view(n, p, h, d).transpose(1, 2)
                cc, scales[at:at + n] = _store(rows, codes)
                c[at:at + n] = cc if x == "k" else _by_channel(_raw(cc)).view(cc.dtype)
        else:           # the pages' old contents: a free page holds anything
            _raw(c).zero_()
            scales.fill_(1.0)
        rows = _random_rows(bsz * p, h, d, gen, amp).view(bsz, p, h, d).transpose(1, 2).to(dtype)
        s[x + "_codes"], s[x + "_scales"] = c, scales
        s[x + "_tail"] = rows.contiguous() if x == "k" else _by_channel(rows)
        s[x + "_tail0"] = s[x + "_tail"].clone()
    if kind == "attend":
        s["q"] = torch.randn(total, hq, d, device=DEV, generator=gen).to(dtype)
    else:
        # a page that fills and rows behind it: a second pass over the same state needs the old tail back
        s["again"] = any(o % p and n // p > o // p and n % p for o, n in zip(_old(case), lens))
        first = [o // p * p for o in _old(case)]
        s["first"], s["out_starts"] = _ints(first), _ints(_sums([n - f for n, f in zip(lens, first)]))
        s["read"] = sum(lens) - sum(first)
        s["max_read"] = max(n - f for n, f in zip(lens, first))
    return s


def prepare(case, seed):
    """What a serving program holds before the call; with `own`, the cache's handle and buffers too."""
    s = _inputs(case, seed)
    if own:
        import paper_2405_12591_amd as dq
        if case["kind"] != "attend":
            s["rotary"] = dq.Rotary(s["inv"], case["interleaved"], s["axis"] if case["axes"] > 1 else None, case["axes"])
            s["q_out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEV)
            s["k_out"] = torch.empty(s["k"].shape, dtype=s["k"].dtype, device=DEV)
        if case["kind"] != "rotate":
            s["cache"] = dq.PagedCache({n: s[n] for n in ("k_codes", "k_scales", "v_codes", "v_scales", "k_tail", "v_tail")})
        if case["kind"] == "append":
            s["rows"] = torch.empty(2, s["read"], case["kv_heads"], case["dim"], dtype=s["k"].dtype, device=DEV)
        if case["kind"] == "attend":
            s["ws"] = dq.paged_workspace(s["cache"], case["batch"], s["q"].shape[0], case["q_heads"], s["max_new"], s["max_len"])
            s["out"] = torch.empty_like(s["q"])
    return s


# ------------------------------------------------------------------------------------------------
# One pass
# ------------------------------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if kind == "append" and s["again"]:
        s["k_tail"].copy_(s["k_tail0"])
        s["v_tail"].copy_(s["v_tail0"])
    if not own:
        return {"rotate": _plain_rotate, "append": _plain_append, "attend": _plain_attend}[kind](s)
    import paper_2405_12591_amd as dq
    if kind == "rotate":
        return dq.rotate_heads(s["q"], s["k"], s["pos"], s["rotary"], q_weight=s["wq"], k_weight=s["wk"], eps=EPS,
                               q_out=s["q_out"], k_out=s["k_out"])
    if kind == "append":
        q = dq.paged_append(s["cache"], s["k"], s["v"], s["starts"], s["lens"], s["table"], q=s["q"], q_out=s["q_out"],
                            rotary=s["rotary"], positions=s["pos"], q_weight=s["wq"], k_weight=s["wk"], eps=EPS, tail_slots=s["slots"])
        k, v = dq.paged_read(s["cache"], s["first"], s["lens"], s["out_starts"], s["table"], s["rows"][0], s["rows"][1], tail_slots=s["slots"])
        return q, k, v
    return dq.paged_attention(s["cache"], s["q"], s["starts"], s["lens"], s["table"], s["max_new"], s["max_len"], s["ws"],
                              out=s["out"], window=s["case"]["window"], tail_slots=s["slots"])


def _plain_heads(s, x, w):
    """Norm and rotation of f32 heads [T, heads, D], rounded once."""
    case, dtype = s["case"], x.dtype
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
    angle = s["pos"].double()[s["axis"].long()].transpose(0, 1) * s["inv"]          # [T, rot / 2], in 64 bits: far positions
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    r = case["rot"]
    if case["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([y, x[..., r:]], -1).to(dtype)


def _plain_rotate(s):
    return _plain_heads(s, s["q"], s["wq"]), _plain_heads(s, s["k"], s["wk"])


def _owner(starts, total):
    """Sequence and place in it of every packed row."""
    t = torch.arange(total, device=DEV)
    b = torch.searchsorted(starts, t, right=True) - 1
    return b, t - starts[b]


def _plain_append(s):
    case, p = s["case"], s["case"]["page"]
    q, k = _plain_heads(s, s["q"], s["wq"]), _plain_heads(s, s["k"], s["wk"])
    lens, slots, h, d = s["lens"].long(), s["slots"].long(), case["kv_heads"], case["dim"]
    old = lens - s["starts"].diff().long()
    page0 = old // p
    b, i = _owner(s["starts"].long(), k.shape[0])
    at = (old - page0 * p)[b] + i                          # place among the touched pages' rows
    n_pages = -(-(s["max_read"]) // p)
    pages = torch.arange(n_pages, device=DEV)[None] + page0[:, None]
    full = pages < (lens // p)[:, None]
    where = (pages == (lens // p)[:, None]) & ((lens % p) > 0)[:, None]
    table = s["table"].long().gather(1, pages.clamp(max=s["table"].shape[1] - 1))
    rb, ri = _owner(s["out_starts"].long(), s["read"])
    outs = [q]
    for x, new in (("k", k), ("v", s["v"])):
        tail = s[x + "_tail"] if x == "k" else _by_token(s[x + "_tail"])
        rows = torch.zeros(len(lens), n_pages * p, h, d, dtype=new.dtype, device=DEV)
        rows[:, :p] = tail[slots].transpose(1, 2)
        rows[b, at] = new
        blocks = rows.unflatten(1, (n_pages, p)).transpose(2, 3)          # [B, pages, H, P, D]
        c, scale = _store(blocks.float(), case["codes"])
        # only full pages are written
        pool, pool_s = s[x + "_codes"], s[x + "_scales"]
        cc = _raw(c if x == "k" else _by_channel(_raw(c)).view(c.dtype))
        _raw(pool)[table[full]] = cc[full]
        pool_s[table[full]] = scale[full]
        keep = torch.zeros_like(tail).index_copy(0, slots, (blocks * where[..., None, None, None]).sum(1).to(tail.dtype))
        fresh = torch.zeros(tail.shape[0], dtype=torch.bool, device=DEV).index_copy(0, slots, where.any(1))
        used = torch.zeros_like(lens).index_copy(0, slots, lens % p)
        new_tail = torch.where(fresh[:, None, None, None] & (torch.arange(p, device=DEV)[None, :] < used[:, None])[:, None, :, None], keep, tail)
        s[x + "_tail"].copy_(new_tail if x == "k" else _by_channel(new_tail))
        value = torch.where(full[..., None, None, None], c.float() * scale[..., None, None], blocks.float()).to(new.dtype)
        outs.append(value.transpose(2, 3).flatten(1, 2)[rb, ri])
    return tuple(outs)


def _plain_rows(s, x):
    """What the cache stands for: f32 [B, H, tokens, D], zero behind a sequence's end."""
    case, p = s["case"], s["case"]["page"]
    lens = s["lens"].long()
    n = -(-s["max_len"] // p)
    table = s["table"].long()[:, :n]
    c = _raw(s[x + "_codes"])[table].view(s[x + "_codes"].dtype).float()
    tail = s[x + "_tail"][s["slots"].long()].float()[:, None]
    rows = torch.where((torch.arange(n, device=DEV)[None] == (lens // p)[:, None]).view(len(lens), n, *[1] * (c.dim() - 2)), tail,
                       c * s[x + "_scales"][table].view(*table.shape, -1, *[1] * (c.dim() - 3)))
    if x == "v":
        rows = _by_token(rows)
    rows = rows.transpose(1, 2).flatten(2, 3)
    return torch.where((torch.arange(n * p, device=DEV)[None] < lens[:, None])[:, None, :, None], rows, torch.zeros_like(rows))


def _plain_attend(s):
    case = s["case"]
    h, d, n = case["kv_heads"], case["dim"], s["max_new"]
    g = case["q_heads"] // h
    starts, lens = s["starts"].long(), s["lens"].long()
    bsz = len(lens)
    counts = starts.diff()
    at = (starts[:-1, None] + torch.arange(n, device=DEV)[None]).clamp(max=s["q"].shape[0] - 1)
    q = s["q"].float()[at].view(bsz, n, h, g, d).permute(0, 2, 1, 3, 4).reshape(bsz, h, n * g, d)
    k, v = _plain_rows(s, "k"), _plain_rows(s, "v")
    j = torch.arange(k.shape[2], device=DEV)
    place = lens[:, None] - counts[:, None] + torch.arange(n, device=DEV)[None]            # a query's own place
    seen = (j <= place[..., None]) & (j < lens[:, None, None])
    if case["window"]:
        seen &= j > place[..., None] - case["window"]
    seen = seen[:, None, :, None].expand(bsz, 1, n, g, len(j)).reshape(bsz, 1, n * g, len(j))
    score = (q @ k.transpose(-1, -2)) * (1 / math.sqrt(d))
    score.masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    e = score.sub_(torch.where(top.isfinite(), top, torch.zeros_like(top))).exp_()
    total = e.sum(-1, keepdim=True)
    o = (e @ v) / torch.where(total > 0, total, torch.ones_like(total))
    o = o.view(bsz, h, n, g, d).permute(0, 2, 1, 3, 4).reshape(bsz, n, h * g, d)
    b, i = _owner(starts, s["q"].shape[0])
    return o[b, i].to(s["q"].dtype)


# ------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ------------------------------------------------------------------------------------------------
def _pairs(case):
    """Visible (query, key) pairs of one head, and tokens that some query sees."""
    pairs = tokens = 0
    for n, c in zip(_lens(case), _counts(case)):
        w = case["window"] or n
        sees = [min(n - c + i + 1, w) for i in range(c)]
        pairs += sum(sees)
        tokens += n - max(0, n - c + 1 - w)
    return pairs, tokens


def work(case):
    kind, d, hq, h, total = case["kind"], case["dim"], case["q_heads"], case["kv_heads"], sum(_counts(case))
    if kind == "rotate":
        return {"bytes": 4 * total * (hq + h) * d + 4 * total * case["axes"], "flops": 7 * total * (hq + h) * d}
    p = case["page"]
    if kind == "append":
        # rows in, rotated queries out; codes (or 16-bit rows) written; the old rows of a page that fills;
        # then the touched pages' values out
        coded = sum(n // p * p - o // p * p for o, n in zip(_old(case), _lens(case)))
        kept = sum(n % p if n // p > o // p else n - o for o, n in zip(_old(case), _lens(case)))
        filled = sum(o % p for o, n in zip(_old(case), _lens(case)) if n // p > o // p)
        read = sum(n - o // p * p for o, n in zip(_old(case), _lens(case)))
        return {"bytes": 4 * total * hq * d + 2 * h * d * (2 * total + coded + 2 * kept + 2 * filled + 2 * read),
                "flops": 7 * total * (hq + h) * d + 6 * h * d * coded}
    pairs, tokens = _pairs(case)
    tails = sum(n % p for n in _lens(case))
    return {"bytes": 4 * total * hq * d + 2 * h * (tokens * d + tails * d) + 8 * h * (tokens // p), "flops": 4 * pairs * hq * d}


# ------------------------------------------------------------------------------------------------
# The same from the definition, in 64 bits
# ------------------------------------------------------------------------------------------------
def _exact_heads(s, x, w):
    """Every pair of channels is a complex number that is multiplied by exp(i * angle)."""
    case = s["case"]
    x = x.double()
    if w is not None:
        x = w.double() * x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt()
    y, half = x.clone(), case["rot"] // 2
    first = [2 * i if case["interleaved"] else i for i in range(half)]
    second = [2 * i + 1 if case["interleaved"] else i + half for i in range(half)]
    for i in range(half):
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), s["pos"][int(s["axis"][i])].double() * s["inv"][i])
        z = torch.complex(x[..., first[i]], x[..., second[i]]) * turn[:, None]
        y[..., first[i]], y[..., second[i]] = z.real, z.imag
    return y


def _exact_values(x, codes):
    """What the block [rows, H, D] stands for after quantization."""
    top = x.abs().amax((0, 2), keepdim=True)
    m, e = torch.frexp(QMAX[codes] / torch.where(top > 0, top, torch.ones_like(top)))
    r = torch.ldexp(torch.floor(m * 4096), e - 12)
    y = x * r
    if codes == "int8":
        return y.round() / r
    # e4m3: three bits behind the leading one, exponents from -6 on
    unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -30))).clamp(min=-6) - 3)
    return (y / unit).round() * unit / r


def _exact_cache(s, x, b):
    """Rows [tokens, H, D] of sequence b of the given cache."""
    p, n, slot = s["case"]["page"], int(s["lens"][b]), int(s["slots"][b])
    pages = s["table"][b, :n // p].long()
    c = _raw(s[x + "_codes"])[pages].view(s[x + "_codes"].dtype).double() if len(pages) else None
    parts = []
    if c is not None:
        c = (c if x == "k" else _by_token(c)) * s[x + "_scales"][pages].double()[..., None, None]
        parts.append(c.transpose(1, 2).flatten(0, 1))
    t = s[x + "_tail"][slot] if x == "k" else _by_token(s[x + "_tail"][slot])
    parts.append(t.transpose(0, 1)[:n % p].double())
    return torch.cat(parts)


def exact(case, seed):
    s = _inputs(case, seed)
    dtype, counts, lens, old = DTYPES[case["dtype"]], _counts(case), _lens(case), _old(case)
    starts = _sums(counts)
    if case["kind"] == "rotate":
        return _exact_heads(s, s["q"], s["wq"]), _exact_heads(s, s["k"], s["wk"])
    if case["kind"] == "append":
        p = case["page"]
        q, k = _exact_heads(s, s["q"], s["wq"]), _exact_heads(s, s["k"], s["wk"])
        outs = {"k": [], "v": []}
        for x, new in (("k", k.to(dtype).double()), ("v", s["v"].double())):       # the cache takes 16-bit rows
            for b in range(case["batch"]):
                t = s[x + "_tail0"][int(s["slots"][b])]
                t = (t if x == "k" else _by_token(t)).transpose(0, 1).double()
                rows = torch.cat([t[:old[b] % p], new[starts[b]:starts[b + 1]]])
                whole = len(rows) // p
                outs[x] += [_exact_values(rows[i * p:(i + 1) * p], case["codes"]) for i in range(whole)] + [rows[whole * p:]]
        return q, torch.cat(outs["k"]), torch.cat(outs["v"])
    g, outs = case["q_heads"] // case["kv_heads"], []
    for b in range(case["batch"]):
        k, v = _exact_cache(s, "k", b), _exact_cache(s, "v", b)
        q = s["q"][starts[b]:starts[b + 1]].double()
        i = torch.arange(old[b], lens[b], device=DEV)[:, None]
        j = torch.arange(lens[b], device=DEV)[None]
        hidden = (j > i) | (j <= i - case["window"] if case["window"] else j < 0)
        o = torch.empty_like(q)
        for head in range(case["q_heads"]):
            score = q[:, head] @ k[:, head // g].t().contiguous() / math.sqrt(case["dim"])
            o[:, head] = torch.softmax(score.masked_fill(hidden, -math.inf), -1) @ v[:, head // g]
        outs.append(o)
    return torch.cat(outs)
