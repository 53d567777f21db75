"""Serving attention over one latent vector a token, and for trees of drafted tokens over an 8-bit cache.

Four kinds of case, all on the ragged batches a serving loop has (rows of all sequences one behind the
other, `starts` says where each begins):

  append    new tokens go into a paged cache of latents: the latent normed, the key channels that all heads
            share rotated, and so the queries' channels that meet them; the touched pages read back as rows
  absorbed  attention of query rows that were taken into the latent's space:
            softmax(q . [c | k_rot] * scale) c, one key and value for all heads
  expanded  attention of prompts over keys and values expanded from the latents:
            softmax((q . [k | k_rot]) * scale) v, k and v of each head, k_rot shared
  tree      drafted rows, not in the cache, attend to the cached tokens of their sequence and to those
            drafted rows that a bit mask names (their ancestors)

Cache of latents: [pages, P, R + r] 16-bit rows, page table [batch, pages].  The 8-bit cache (H kv heads, D
channels; 64 tokens of values are kept channel by channel): k_codes [pages, H, P, D], v_codes [pages, H, P / 64,
D, 64], a scale for each (page, head), and 16-bit rows of the page that is not yet full (k_tail, v_tail).
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
# latent and shared key channels with the channels of a head's expanded key and value
FORMS = {"512+64": (512, 64, 128), "256+32": (256, 32, 64)}


# ------------------------------------------------------------------------------------------------
# The cases
# ------------------------------------------------------------------------------------------------
def _append(dtype, form, page, heads, batch, old, new_lo, new_hi, interleaved=False):
    return {"kind": "append", "dtype": dtype, "form": form, "page": page, "heads": heads, "batch": batch, "old": old,
            "new_lo": new_lo, "new_hi": new_hi, "interleaved": interleaved}


def _absorbed(dtype, form, page, heads, batch, lo, hi, new_lo=1, new_hi=1, tree=False):
    return {"kind": "absorbed", "dtype": dtype, "form": form, "page": page, "heads": heads, "batch": batch, "lo": lo, "hi": hi,
            "new_lo": new_lo, "new_hi": new_hi, "tree": tree}


def _expanded(dtype, form, heads, batch, old, new_lo, new_hi):
    return {"kind": "expanded", "dtype": dtype, "form": form, "heads": heads, "batch": batch, "old": old, "new_lo": new_lo, "new_hi": new_hi}


def _tree(dtype, codes, dim, page, q_heads, kv_heads, batch, lo, hi, new_lo, new_hi, window=0):
    return {"kind": "tree", "dtype": dtype, "codes": codes, "dim": dim, "page": page, "q_heads": q_heads, "kv_heads": kv_heads,
            "batch": batch, "lo": lo, "hi": hi, "new_lo": new_lo, "new_hi": new_hi, "window": window}


def listed():
    named = [
        # one generated token of each of 16 sequences, queries of 128 heads rotated with it: latency and host work
        ("append_step", _append("bf16", "512+64", 64, 128, 16, 4001, 1, 1)),
        # prompts of mixed lengths on a part of the heads
        ("append_prompt", _append("f16", "512+64", 128, 16, 8, 0, 3000, 4096, interleaved=True)),
        # the smallest call: one short sequence, eight heads
        ("latent_tiny", _absorbed("f16", "256+32", 64, 8, 1, 300, 300)),
        # a generated token each for many sequences on a GPU that holds 16 of the heads: the cache's bytes
        ("latent_shard", _absorbed("bf16", "512+64", 64, 16, 64, 2000, 8192)),
        # a generated token each, all 128 heads, long caches: bytes and matrix products in balance
        ("latent_wide", _absorbed("bf16", "512+64", 64, 128, 16, 12000, 16384)),
        # a tree of drafted tokens checked over the latents, odd lengths
        ("latent_tree", _absorbed("bf16", "512+64", 64, 32, 8, 5000, 9001, 24, 24, tree=True)),
        # whole prompts, causal, expanded keys and values: bound by the matrix products
        ("expanded_prompt", _expanded("bf16", "512+64", 32, 4, 0, 3500, 4096)),
        # a piece of a prompt behind a long cache that was read back and expanded
        ("expanded_chunk", _expanded("f16", "256+32", 40, 2, 15000, 400, 512)),
        # the smallest tree: one short sequence, five drafted tokens
        ("tree_tiny", _tree("f16", "int8", 64, 64, 4, 4, 1, 257, 257, 5, 5)),
        # long context, four query heads per kv head, sixteen drafted tokens
        ("tree_gqa4_long", _tree("bf16", "e4m3", 128, 64, 32, 8, 16, 32768, 32768, 16, 16)),
        # the 13B-shaped layer: 40 heads, mixed, odd lengths, large trees of mixed sizes
        ("tree_ragged", _tree("f16", "int8", 128, 128, 40, 40, 4, 8192, 16384, 30, 64)),
        # heads of 64 channels, eight query heads per kv head, a windowed cache
        ("tree_window", _tree("bf16", "e4m3", 64, 64, 64, 8, 8, 2048, 9001, 13, 13, window=4096)),
    ]
    return [dict(c, name=n) for n, c in named]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _some(rng, n, share):
    """n, or a lower bound below it."""
    return n if rng.random() < share else max(1, int(n * rng.uniform(0.3, 1.0)))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["append", "absorbed", "absorbed", "expanded", "tree", "tree"])
    dtype, page, form = rng.choice(["bf16", "f16"]), rng.choice([64, 128]), rng.choice(["512+64", "512+64", "256+32"])
    heads = rng.choice([1, 8, 16, 16, 20, 32, 40, 64, 128])
    if kind == "append":
        batch = _log_int(rng, 1, 32)
        old = 0 if rng.random() < 0.4 else _log_int(rng, 1, 8000)
        new = 1 if rng.random() < 0.4 else _log_int(rng, 2, max(3, min(4096, 8 * 4096 * 32 // (batch * (heads + 16)))))
        return _append(dtype, form, page, heads, batch, old, _some(rng, new, 0.4), new, rng.random() < 0.5)
    if kind == "absorbed":
        # up to latent_wide's visible pairs and latent_shard's bytes
        batch, new = _log_int(rng, 1, 64), rng.choice([1, 1, 1, rng.randint(2, 4), _log_int(rng, 5, 64)])
        hi = _log_int(rng, 1, max(2, min(32768, 64 * 6000 // batch, 16 * 14000 * 128 // (batch * new * heads))))
        new = min(new, hi)
        lo = max(new, _some(rng, hi, 0.4))
        return _absorbed(dtype, form, page, heads, batch, lo, hi, _some(rng, new, 0.6), new, rng.random() < 0.4)
    if kind == "expanded":
        batch = _log_int(rng, 1, 4)
        old = 0 if rng.random() < 0.5 else _log_int(rng, 1, min(15000, 4000000 // (batch * heads)))
        # rows whose visible pairs are no more than expanded_prompt's: n (old + n / 2) batch heads <= 4 heads of 32 of 3800^2 / 2
        most = 4 * 3800 * 3800 // 2 * 32 // (batch * heads)
        new = _log_int(rng, 1, max(2, min(4096, int(math.sqrt(old * old + 2 * most) - old))))
        return _expanded(dtype, form, heads, batch, old, _some(rng, new, 0.4), new)
    dim, codes = rng.choice([128, 128, 64]), rng.choice(["e4m3", "int8"])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16, 32, 40])
    group = rng.choice([1, 2, 3, 4, 8]) if kv_heads <= 8 else 1
    batch, new = _log_int(rng, 1, 16), rng.choice([_log_int(rng, 2, 64), _log_int(rng, 2, 64), 64])
    # up to tree_gqa4_long's bytes and visible pairs
    hi = _log_int(rng, 1, max(2, min(32768, 16 * 8 * 32768 // (batch * kv_heads), 16 * 32768 * 16 * 32 // (batch * new * kv_heads * group))))
    window = _log_int(rng, 64, 8192) if rng.random() < 0.15 else 0
    return _tree(dtype, codes, dim, page, kv_heads * group, kv_heads, batch, _some(rng, hi, 0.4), hi, _some(rng, new, 0.5), new, window)


def _spread(lo, hi, n):
    """n sizes over [lo, hi], the first one hi, odd ones among them."""
    return [hi - int((hi - lo) * ((i * 0.618034) % 1.0)) for i in range(n)]


def _counts(case):
    """New rows of every sequence."""
    return _spread(case["new_lo"], case["new_hi"], case["batch"])


def _lens(case):
    """Tokens of every sequence: with the new ones, but for a tree's, which are not in the cache."""
    if "old" in case:
        return [case["old"] + (9 * i if case["old"] else 0) + c for i, c in enumerate(_counts(case))]
    return _spread(case["lo"], case["hi"], case["batch"])


def _old(case):
    return [n - (0 if case["kind"] == "tree" else c) for n, c in zip(_lens(case), _counts(case))]


def _sums(values):
    out = [0]
    for v in values:
        out.append(out[-1] + v)
    return out


# ------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------
def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _normal(shape, gen, spread=0.5):
    """f32, normal, a range per row."""
    x = torch.randn(shape, device=DEV, generator=gen)
    return x * torch.exp(spread * torch.randn(*shape[:-1], 1, device=DEV, generator=gen))


def _pages(case, lens, gen):
    """A page table over a shuffled pool, and the pool's size."""
    need = [-(-n // case["page"]) for n in lens]
    pool = sum(need) + 3
    order = torch.randperm(pool, device=DEV, generator=gen).to(torch.int32)
    table = torch.zeros(len(lens), max(1, max(need)), dtype=torch.int32, device=DEV)
    for b, at in enumerate(_sums(need)[:-1]):
        table[b, :need[b]] = order[at:at + need[b]]
    return table, pool


def _masks(counts, gen):
    """Bit masks of random trees: a row's parent is one of the rows before it, or it begins a branch of its own."""
    pick = torch.rand(sum(counts), device=DEV, generator=gen).tolist()
    at, out = 0, []
    for n in counts:
        seen = []
        for i in range(n):
            parent = int(pick[at + i] * (i + 1)) - 1 if i < 4 else i - 1 - int(pick[at + i] * min(i, 6))
            seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
        out += seen
        at += n
    return out


def _signed(masks):
    return [m - (1 << 64) if m >> 63 else m for m in masks]


def _inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    counts, lens, old = _counts(case), _lens(case), _old(case)
    total = sum(counts)
    s = {"case": case, "starts": _ints(_sums(counts)), "lens": _ints(lens), "max_new": max(counts), "max_len": max(lens)}
    if kind == "tree" or case.get("tree"):
        s["masks"] = _masks(counts, gen)
        s["seen"] = torch.tensor(_signed(s["masks"]), dtype=torch.int64, device=DEV)
    if kind == "tree":
        return _tree_inputs(case, s, gen)
    R, r, d = FORMS[case["form"]]
    heads = case["heads"]
    if kind == "append":
        # what the fused down-projection leaves: a token's latent and its shared key channels; and the queries' heads
        down = torch.empty(total, R + r + 24, dtype=dtype, device=DEV)
        down[:, :R + r] = _normal((total, R + r), gen)
        down[:, :R:37] *= 8
        s["latent"], s["k_rot"] = down[:, :R], down[:, None, R:R + r]
        s["q"] = torch.randn(total, heads, d + r, device=DEV, generator=gen).to(dtype)[..., d:]
        s["weight"] = (1 + 0.2 * torch.randn(R, device=DEV, generator=gen)).to(dtype)
        s["inv"] = BASE ** (-torch.arange(r // 2, dtype=torch.float64, device=DEV) / (r // 2))
        s["pos"] = torch.cat([torch.arange(o, o + c, device=DEV) for o, c in zip(old, counts)]).to(torch.int32)
        s["table"], pool = _pages(case, lens, gen)
        s["rows"] = torch.zeros(pool, case["page"], R + r, dtype=dtype, device=DEV)
        for at in range(0, pool, 1024):
            n = min(1024, pool - at)
            s["rows"][at:at + n] = torch.randn(n, case["page"], R + r, device=DEV, generator=gen).to(dtype)
        first = [o // case["page"] * case["page"] for o in old]
        s["first"], s["out_starts"] = _ints(first), _ints(_sums([n - f for n, f in zip(lens, first)]))
        s["read"] = sum(lens) - sum(first)
        # rows of the touched pages that were there before, and where each is kept
        s["kept"] = s["rows"].clone() if any(f < o for f, o in zip(first, old)) else None
        return s
    s["scale"] = 1 / math.sqrt(d + r)
    if kind == "absorbed":
        s["table"], pool = _pages(case, lens, gen)
        amp = 1 + 0.2 * torch.randn(R + r, device=DEV, generator=gen)
        amp[:R:37] *= 8
        s["rows"] = torch.empty(pool, case["page"], R + r, dtype=dtype, device=DEV)
        for at in range(0, pool, 1024):
            n = min(1024, pool - at)
            s["rows"][at:at + n] = (torch.randn(n, case["page"], R + r, device=DEV, generator=gen) * amp).to(dtype)
        s["q"] = _normal((total, heads, R + r), gen).to(dtype)
        return s
    s["kv_starts"] = _ints(_sums(lens))
    tokens = sum(lens)
    # keys and values as one up-projection leaves them, the shared key channels as they lie in the rows read back
    kv = torch.empty(tokens, heads, 2 * d, dtype=dtype, device=DEV)
    for at in range(0, tokens, 4096):
        n = min(4096, tokens - at)
        kv[at:at + n] = _normal((n, heads, 2 * d), gen).to(dtype)
    kv[..., 5:d:37] *= 8
    s["k"], s["v"] = kv[..., :d], kv[..., d:]
    s["k_rot"] = torch.randn(tokens, R + r, device=DEV, generator=gen).to(dtype)[:, None, R:]
    s["q"] = torch.randn(total, heads, d + r, device=DEV, generator=gen).to(dtype)
    return s


def _store(x, codes):
    """f32 blocks [..., rows, channels] -> codes and their scales [...]: the inverse step has 12 significant bits."""
    top = x.abs().amax((-1, -2))
    r = (QMAX[codes] / top).view(torch.int32).bitwise_and(~0xfff).view(torch.float32)
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


def _tree_inputs(case, s, gen):
    dtype, codes, p = DTYPES[case["dtype"]], case["codes"], case["page"]
    hq, h, d, bsz = case["q_heads"], case["kv_heads"], case["dim"], case["batch"]
    total = sum(_counts(case))
    s["table"], pool = _pages(case, _lens(case), gen)
    s["slots"] = torch.randperm(bsz, device=DEV, generator=gen).to(torch.int32)
    # the drafted tokens' heads as a fused projection leaves them (turned in place)
    qkv = torch.randn(total, hq + 2 * h, d, device=DEV, generator=gen)
    for i, x in enumerate("kv"):
        amp = torch.ones(h, 1, d, device=DEV)
        amp[..., 3 + i::37] = 20.0
        c = torch.empty(pool, h, p, d, dtype=CODES[codes], device=DEV)
        c = c if x == "k" else c.view(pool, h, p // 64, d, 64)
        scales = torch.empty(pool, h, device=DEV)
        for at in range(0, pool, 1024):
            n = min(1024, pool - at)
            cc, scales[at:at + n] = _store(_normal((n, h, p, d), gen) * amp, codes)
            c[at:at + n] = cc if x == "k" else _by_channel(_raw(cc)).view(cc.dtype)
        rows = (_normal((bsz, h, p, d), gen) * amp).to(dtype)
        s[x + "_codes"], s[x + "_scales"] = c, scales
        s[x + "_tail"] = rows if x == "k" else _by_channel(rows)
        qkv[:, hq + i * h:hq + (i + 1) * h] *= amp[:, 0]
    qkv = qkv.to(dtype)
    s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + h], qkv[:, hq + h:]
    return s


def prepare(case, seed):
    """What a serving program holds before the call; with `own`, the cache's handle and buffers too."""
    s = _inputs(case, seed)
    kind = case["kind"]
    if own:
        import paper_2405_12591_amd as dq
        total = s["q"].shape[0]
        if kind == "tree":
            s["cache"] = dq.PagedCache({n: s[n] for n in ("k_codes", "k_scales", "v_codes", "v_scales", "k_tail", "v_tail")})
            s["ws"] = dq.paged_tree_workspace(s["cache"], case["batch"], total, case["q_heads"], s["max_new"], s["max_len"])
            s["out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEV)
            return s
        R, r, d = FORMS[case["form"]]
        if kind != "expanded":
            s["cache"] = dq.LatentCache(s["rows"], R)
        if kind == "append":
            s["rotary"] = dq.Rotary(s["inv"], case["interleaved"])
            # the queries that the absorbed attention takes: their first R channels come from a product
            s["q_out"] = torch.zeros(total, case["heads"], R + r, dtype=s["q"].dtype, device=DEV)[..., R:]
            s["read_out"] = torch.empty(s["read"], R + r, dtype=s["q"].dtype, device=DEV)
        elif kind == "absorbed":
            s["ws"] = dq.latent_workspace(s["cache"], case["batch"], total, case["heads"], s["max_new"], s["max_len"])
            s["out"] = torch.empty(total, case["heads"], R, dtype=s["q"].dtype, device=DEV)
        else:
            s["ws"] = dq.expanded_workspace(case["batch"], total, case["heads"], d, s["max_new"], s["max_len"], DEV)
            s["out"] = torch.empty(total, case["heads"], d, dtype=s["q"].dtype, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------
# One pass
# ------------------------------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"append": _plain_append, "absorbed": _plain_absorbed, "expanded": _plain_expanded, "tree": _plain_tree}[kind](s)
    import paper_2405_12591_amd as dq
    if kind == "append":
        q = dq.latent_append(s["cache"], s["latent"], s["k_rot"][:, 0], s["starts"], s["lens"], s["table"], q=s["q"], q_out=s["q_out"],
                             rotary=s["rotary"], positions=s["pos"], weight=s["weight"], eps=EPS)
        return q, dq.latent_read(s["cache"], s["first"], s["lens"], s["out_starts"], s["table"], s["read_out"])
    if kind == "absorbed":
        return dq.latent_attention(s["cache"], s["q"], s["starts"], s["lens"], s["table"], s["max_new"], s["max_len"], s["scale"], s["ws"],
                                   out=s["out"], seen=s.get("seen"))
    if kind == "expanded":
        return dq.expanded_attention(s["q"], s["k"], s["k_rot"][:, 0], s["v"], s["starts"], s["kv_starts"], s["max_new"], s["max_len"], s["ws"],
                                     out=s["out"], softmax_scale=s["scale"])
    return dq.paged_tree_attention(s["cache"], s["q"], s["k"], s["v"], s["seen"], s["starts"], s["lens"], s["table"], s["max_new"], s["max_len"],
                                   s["ws"], out=s["out"], window=s["case"]["window"], tail_slots=s["slots"])


def _owner(starts, total):
    """Sequence and place in it of every packed row."""
    t = torch.arange(total, device=DEV)
    b = torch.searchsorted(starts, t, right=True) - 1
    return b, t - starts[b]


def _plain_turn(s, x):
    """Rotation of heads [T, heads, r], rounded once."""
    angle = s["pos"].double()[:, None] * s["inv"]          # in 64 bits: far positions
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    y, half = x.float(), x.shape[-1] // 2
    if s["case"]["interleaved"]:
        a, b = y[..., 0::2], y[..., 1::2]
        return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2).to(x.dtype)
    a, b = y[..., :half], y[..., half:]
    return torch.cat([a * cos - b * sin, a * sin + b * cos], -1).to(x.dtype)


def _plain_append(s):
    page = s["case"]["page"]
    x = s["latent"].float()
    c = (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * s["weight"].float()).to(s["latent"].dtype)
    rows = torch.cat([c, _plain_turn(s, s["k_rot"])[:, 0]], -1)
    starts, lens, table = s["starts"].long(), s["lens"].long(), s["table"].long()
    b, i = _owner(starts, rows.shape[0])
    at = (lens - starts.diff())[b] + i
    s["rows"][table[b, at // page], at % page] = rows
    b, i = _owner(s["out_starts"].long(), s["read"])
    at = s["first"].long()[b] + i
    return _plain_turn(s, s["q"]), s["rows"][table[b, at // page], at % page]


def _softmax(score, hidden):
    """Of f32 scores, in place; rows that see nothing are zero."""
    score.masked_fill_(hidden, -math.inf)
    top = score.amax(-1, keepdim=True)
    e = score.sub_(torch.where(top.isfinite(), top, torch.zeros_like(top))).exp_()
    total = e.sum(-1, keepdim=True)
    return e.div_(torch.where(total > 0, total, torch.ones_like(total)))


def _bits(seen, n):
    """int64 [rows] -> bool [rows, n]"""
    return (seen[:, None] >> torch.arange(n, device=DEV)[None] & 1).bool()


def _plain_absorbed(s):
    case, page = s["case"], s["case"]["page"]
    R, _, _ = FORMS[case["form"]]
    starts, outs = _sums(_counts(case)), []
    for b, (n, new) in enumerate(zip(_lens(case), _counts(case))):
        rows = s["rows"][s["table"][b, :-(-n // page)].long()].flatten(0, 1)[:n].float()
        q = s["q"][starts[b]:starts[b + 1]].float()
        j = torch.arange(n, device=DEV)
        hidden = j[None] > torch.arange(n - new, n, device=DEV)[:, None]
        if case["tree"]:
            hidden[:, n - new:] = ~_bits(s["seen"][starts[b]:starts[b + 1]], new)
        p = _softmax(q @ rows.t() * s["scale"], hidden[:, None])
        outs.append((p @ rows[:, :R]).to(s["q"].dtype))
    return torch.cat(outs)


def _plain_expanded(s):
    case = s["case"]
    starts, at, out = _sums(_counts(case)), _sums(_lens(case)), torch.empty(s["q"].shape[:2] + s["v"].shape[2:], dtype=s["q"].dtype, device=DEV)
    for b, n in enumerate(_lens(case)):
        new = starts[b + 1] - starts[b]
        hidden = torch.arange(n, device=DEV)[None] > torch.arange(n - new, n, device=DEV)[:, None]
        kr = s["k_rot"][at[b]:at[b + 1]].float()
        for h in range(0, case["heads"], 8):
            q = s["q"][starts[b]:starts[b + 1], h:h + 8].float().transpose(0, 1)
            k = torch.cat([s["k"][at[b]:at[b + 1], h:h + 8].float(), kr.expand(-1, q.shape[0], -1)], -1).permute(1, 2, 0).contiguous()
            p = _softmax(q @ k * s["scale"], hidden)
            v = s["v"][at[b]:at[b + 1], h:h + 8].float().transpose(0, 1).contiguous()
            out[starts[b]:starts[b + 1], h:h + 8] = (p @ v).transpose(0, 1).to(out.dtype)
    return out


def _plain_tree(s):
    case, p = s["case"], s["case"]["page"]
    h, d = case["kv_heads"], case["dim"]
    g = case["q_heads"] // h
    starts, outs = _sums(_counts(case)), []
    for b, (n, new) in enumerate(zip(_lens(case), _counts(case))):
        own_rows = slice(starts[b], starts[b + 1])
        both = []
        for x in "kv":
            pages = s["table"][b, :n // p].long()
            c = _raw(s[x + "_codes"])[pages].view(s[x + "_codes"].dtype).float() * s[x + "_scales"][pages].view(-1, h, *[1] * (2 if x == "k" else 3))
            t = s[x + "_tail"][int(s["slots"][b])][None].float()
            if x == "v":
                c, t = _by_token(c), _by_token(t)
            c = torch.cat([c.transpose(0, 1).flatten(1, 2), t[0, :, :n % p], s[x][own_rows].float().transpose(0, 1)], 1)     # [h, tokens, d]
            both.append(c)
        k, v = both
        q = s["q"][own_rows].float().view(new, h, g, d).permute(1, 0, 2, 3).reshape(h, new * g, d)
        bits = _bits(s["seen"][own_rows], new)
        hidden = torch.zeros(new, n + new, dtype=torch.bool, device=DEV)
        hidden[:, n:] = ~bits
        if case["window"]:
            place = n + bits.sum(-1, keepdim=True) - 1
            hidden[:, :n] = torch.arange(n, device=DEV)[None] <= place - case["window"]
        w = _softmax(q @ k.transpose(-1, -2).contiguous() * (1 / math.sqrt(d)), hidden[:, None].expand(new, g, n + new).reshape(new * g, n + new))
        outs.append((w @ v).view(h, new, g, d).permute(1, 0, 2, 3).reshape(new, h * g, d).to(s["q"].dtype))
    return torch.cat(outs)


# ------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ------------------------------------------------------------------------------------------------
def work(case):
    counts, lens, total = _counts(case), _lens(case), sum(_counts(case))
    if case["kind"] == "tree":
        # half of the drafted pairs, about, are ancestors; a window is counted from the cached tokens' end
        hq, h, d, p, w = case["q_heads"], case["kv_heads"], case["dim"], case["page"], case["window"] or 1 << 30
        tokens = sum(min(n, w) for n in lens)
        pairs = sum(c * min(n, w) + c * (c + 1) // 4 for n, c in zip(lens, counts))
        tails = sum(n % p for n in lens)
        return {"bytes": 4 * total * (hq + h) * d + 2 * h * d * (tokens + tails) + 8 * h * (tokens // p), "flops": 4 * pairs * hq * d}
    R, r, d = FORMS[case["form"]]
    heads, pairs = case["heads"], sum(c * (n - c) + c * (c + 1) // 2 for n, c in zip(lens, counts))
    if case["kind"] == "append":
        # rows and queries in and out, then the touched pages' rows in and out
        read = sum(n - o // case["page"] * case["page"] for n, o in zip(lens, _old(case)))
        return {"bytes": 4 * total * (R + r + heads * r) + 4 * read * (R + r), "flops": total * (4 * R + 3 * r * (heads + 1))}
    if case["kind"] == "absorbed":
        return {"bytes": 2 * sum(lens) * (R + r) + 2 * total * heads * (2 * R + r), "flops": 2 * pairs * heads * (2 * R + r)}
    return {"bytes": 2 * sum(lens) * (2 * heads * d + r) + 2 * total * heads * (2 * d + r), "flops": 2 * pairs * heads * (2 * d + r)}


# ------------------------------------------------------------------------------------------------
# The same from the definition, in 64 bits
# ------------------------------------------------------------------------------------------------
def _exact_turn(s, x):
    """Every pair of channels is a complex number that is multiplied by exp(i * angle)."""
    x = x.double()
    y, half = x.clone(), x.shape[-1] // 2
    for i in range(half):
        f, g = (2 * i, 2 * i + 1) if s["case"]["interleaved"] else (i, i + half)
        z = torch.complex(x[..., f], x[..., g]) * torch.polar(torch.ones((), dtype=torch.float64, device=DEV), s["pos"].double() * s["inv"][i])[:, None]
        y[..., f], y[..., g] = z.real, z.imag
    return y


def _exact_append(s):
    case = s["case"]
    x = s["latent"].double()
    new = torch.cat([x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * s["weight"].double(), _exact_turn(s, s["k_rot"])[:, 0]], 1)
    starts, rows = _sums(_counts(case)), []
    for b, (o, n) in enumerate(zip(_old(case), _lens(case))):
        for t in range(o // case["page"] * case["page"], o):
            rows.append(s["kept"][int(s["table"][b, t // case["page"]]), t % case["page"]].double()[None])
        rows.append(new[starts[b]:starts[b + 1]])
    return _exact_turn(s, s["q"]), torch.cat(rows)


def _exact_attend(q, k, v, hidden, scale):
    """q [rows, d], k [tokens, d], v [tokens, e]; a row that sees nothing is zero."""
    out = torch.zeros(q.shape[0], v.shape[1], dtype=torch.float64, device=DEV)
    some = ~hidden.all(1)
    if bool(some.any()):
        score = (q.double() @ k.double().t().contiguous() * scale).masked_fill(hidden, -math.inf)
        out[some] = torch.softmax(score[some], 1) @ v.double()
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "append":
        return _exact_append(s)
    starts, at = _sums(_counts(case)), _sums(_lens(case))
    q = s["q"]
    outs = torch.empty(q.shape[0], q.shape[1], FORMS[case["form"]][0 if case["kind"] == "absorbed" else 2] if "form" in case else case["dim"],
                       dtype=torch.float64, device=DEV)
    for b, n in enumerate(_lens(case)):
        rows = slice(starts[b], starts[b + 1])
        new = starts[b + 1] - starts[b]
        cached = n if case["kind"] == "tree" else n - new
        hidden = torch.arange(cached + new, device=DEV)[None] > cached + torch.arange(new, device=DEV)[:, None]
        if "masks" in s:
            for i, m in enumerate(s["masks"][rows]):
                hidden[i, cached:] = torch.tensor([not m >> j & 1 for j in range(new)], device=DEV)
                if case.get("window"):
                    hidden[i, :max(0, min(n, n + bin(m).count("1") - case["window"]))] = True
        if case["kind"] == "absorbed":
            page = case["page"]
            c = torch.cat([s["rows"][int(s["table"][b, j]), :min(page, n - j * page)] for j in range(-(-n // page))])
            R = FORMS[case["form"]][0]
            wide = hidden.repeat_interleave(case["heads"], 0)
            outs[rows] = _exact_attend(q[rows].flatten(0, 1), c, c[:, :R], wide, s["scale"]).view(new, case["heads"], R)
        elif case["kind"] == "expanded":
            tokens = slice(at[b], at[b + 1])
            for h in range(case["heads"]):
                outs[rows, h] = _exact_attend(q[rows, h], torch.cat([s["k"][tokens, h], s["k_rot"][tokens, 0]], 1), s["v"][tokens, h], hidden, s["scale"])
        else:
            p, slot, g = case["page"], int(s["slots"][b]), case["q_heads"] // case["kv_heads"]
            pages = s["table"][b, :n // p].long()
            for h in range(case["kv_heads"]):
                kv = []
                for x in "kv":
                    c = _raw(s[x + "_codes"])[pages, h].view(s[x + "_codes"].dtype).double()
                    t = s[x + "_tail"][slot, h].double()
                    c, t = (c, t) if x == "k" else (_by_token(c), _by_token(t))
                    c = (c * s[x + "_scales"][pages, h].double()[:, None, None]).flatten(0, 1)
                    kv.append(torch.cat([c, t[:n % p], s[x][rows, h].double()]))
                for j in range(h * g, h * g + g):
                    outs[rows, j] = _exact_attend(q[rows, j], kv[0], kv[1], hidden, 1 / math.sqrt(case["dim"]))
    return outs
