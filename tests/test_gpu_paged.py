"""The paged 8-bit cache: appended rows, what they stand for, and attention over them against 64-bit forms."""
import math

import pytest
import torch

import paper_2405_12591_amd as dq
from paged_util import (DEV, Sequences, attend64, attend_tolerance, filled_cache, fill_tails, device_tables, ints, quantize64, read_back, rows)

pytestmark = pytest.mark.gpu
E4M3, INT8, F16, BF16 = torch.float8_e4m3fn, torch.int8, torch.float16, torch.bfloat16
FORMATS = [(F16, INT8), (BF16, E4M3), (F16, E4M3), (BF16, INT8)]


def _sums(v):
    out = [0]
    for x in v:
        out.append(out[-1] + x)
    return out


# ---------------------------------------------------------------------------------------- append, read
def _codes_of(cache, page, h):
    kc, vc = cache.t["k_codes"][page, h], cache.t["v_codes"][page, h]
    return kc.cpu().double(), vc.cpu().double().transpose(-1, -2).reshape(cache.page_tokens, -1)   # [P/64, d, 64] -> [P, d]


@pytest.mark.parametrize("dtype,codes", FORMATS)
@pytest.mark.parametrize("d,page", [(128, 64), (128, 128), (64, 64), (64, 128)])
def test_appended_rows_and_their_codes(dtype, codes, d, page):
    """Codes, scales and tails exactly as the definition says, whatever pieces the rows come in."""
    gen = torch.Generator().manual_seed(d + page)
    lens, heads = [0, 1, page - 1, page, page + 1, 3 * page + 17], 3
    seqs = Sequences(lens, heads, d, dtype, codes, page, gen)
    seqs.v[3][:, 1] = 0                                   # a block of zeros
    seqs.k[5][page:2 * page, 2] = (seqs.k[5][page:2 * page, 2].double() * 2.0 ** -20).to(dtype)
    print("append", dtype, codes, d, page, flush=True)
    cache, table, slots = filled_cache(seqs, lens, gen)
    before = {n: t.clone() for n, t in cache.t.items()}
    for b, n in enumerate(lens):
        for p in range(n // page):
            for h in range(heads):
                at, pid = slice(p * page, (p + 1) * page), int(table[b, p])
                kc, vc = _codes_of(cache, pid, h)
                for x, c, scale in ((seqs.k[b], kc, cache.t["k_scales"]), (seqs.v[b], vc, cache.t["v_scales"])):
                    want, s = quantize64(x[at, h].double(), codes)
                    assert torch.equal(c, want)
                    assert float(scale[pid, h]) == s
    k, v, starts = read_back(cache, lens, table, slots)
    for b, n in enumerate(lens):
        for got, x in ((k, seqs.k[b]), (v, seqs.v[b])):
            assert torch.equal(got[starts[b]:starts[b + 1]], seqs.stored(x).to(dtype)) or \
                (got[starts[b]:starts[b + 1]].double() - seqs.stored(x)).abs().le(seqs.stored(x).abs() * (2.0 ** -11 if dtype == F16 else 2.0 ** -8) * (1 + 2.0 ** -12) + 2.0 ** -25).all()
    # the same rows in other pieces: the same bits
    other = dq.alloc_paged_cache(cache.pages, cache.slots, heads, d, page, dtype, codes, DEV)
    fill_tails(other)
    for n_ in ("k_scales", "v_scales"):
        other.t[n_].fill_(float("nan"))
    have = [0] * len(lens)
    for step in (5, page - 3, 1, 2 * page, page + 9, 10 ** 6):
        take = [min(step, n - a) for n, a in zip(lens, have)]
        kk = torch.cat([s[a:a + t] for s, a, t in zip(seqs.k, have, take)])
        vv = torch.cat([s[a:a + t] for s, a, t in zip(seqs.v, have, take)])
        have = [a + t for a, t in zip(have, take)]
        dq.paged_append(other, kk.to(DEV), vv.to(DEV), ints(_sums(take)), ints(have), table, tail_slots=slots)
    for n_ in ("k_codes", "v_codes", "k_scales", "v_scales"):
        a, c = before[n_], other.t[n_]
        a, c = (a.view(torch.uint8), c.view(torch.uint8)) if a.element_size() == 1 else (a.view(torch.int32), c.view(torch.int32))
        assert torch.equal(a, c), n_
    k2, v2, _ = read_back(other, lens, table, slots)
    assert torch.equal(k, k2) and torch.equal(v, v2)
    # a part of the tokens, and one whose range is empty
    first = [0, 1, 3, 0, page, page + 5]
    k3, v3, st3 = read_back(cache, lens, table, slots, first)
    for b, n in enumerate(lens):
        assert torch.equal(k3[st3[b]:st3[b + 1]], k[starts[b] + first[b]:starts[b + 1]])
        assert torch.equal(v3[st3[b]:st3[b + 1]], v[starts[b] + first[b]:starts[b + 1]])


@pytest.mark.parametrize("dtype,codes", FORMATS[:2])
@pytest.mark.parametrize("d,page,sections,interleaved", [(128, 64, None, False), (128, 128, (16, 24, 24), False), (64, 64, None, True)])
def test_append_norms_and_rotates_as_rotate_heads_does(dtype, codes, d, page, sections, interleaved):
    """One call with norm and rotation leaves the bits of rotate_heads followed by a plain append, queries too; with
    one axis the positions may be left out."""
    gen = torch.Generator().manual_seed(9)
    old, new, heads, hq = [0, 70, page - 1, 2 * page - 2], [130, 1, 1, 40], 2, 6
    lens = [a + b for a, b in zip(old, new)]
    rot = dq.rotary(d if not interleaved else d // 2, sections=sections, interleaved=interleaved, device=DEV)
    wq, wk = (1 + 0.2 * torch.randn(2, d, generator=gen)).to(dtype).to(DEV)
    before = Sequences(old, heads, d, dtype, codes, page, gen)
    table, pool = device_tables(lens, page, gen)
    total = sum(new)
    fused = rows((total + 4, hq + 2 * heads, d), dtype, gen).to(DEV)      # four rows behind the last sequence's
    q, k, v = fused[:, :hq], fused[:, hq:hq + heads], fused[:, hq + heads:]
    place = torch.cat([torch.arange(o, n) for o, n in zip(old, lens)] + [torch.zeros(4, dtype=torch.long)]).to(torch.int32).to(DEV)
    pos = place if sections is None else torch.stack([place, place // 3, place % 7])
    results = []
    for fused_call in (True, False):
        cache = dq.alloc_paged_cache(pool, 4, heads, d, page, dtype, codes, DEV)
        dq.paged_append(cache, torch.cat(before.k).to(DEV), torch.cat(before.v).to(DEV), ints(_sums(old)), ints(old), table)
        q_out = torch.full((total + 4, hq, d), 5.0, dtype=dtype, device=DEV)
        if fused_call:
            dq.paged_append(cache, k, v, ints(_sums(new)), ints(lens), table, q=q, q_out=q_out, rotary=rot,
                            positions=None if sections is None else pos, q_weight=wq, k_weight=wk)
            assert (q_out[total:] == 5.0).all()                       # rows of no sequence stay
        else:
            qq, kk = dq.rotate_heads(q, k, pos, rot, q_weight=wq, k_weight=wk)
            q_out[:total] = qq[:total]
            dq.paged_append(cache, kk, v, ints(_sums(new)), ints(lens), table)
        results.append((q_out, *read_back(cache, lens, table, None)[:2]))
    for a, b in zip(*results):
        assert torch.equal(a.cpu(), b.cpu())


@pytest.mark.parametrize("dtype,codes", FORMATS[:2])
def test_rows_that_are_not_finite(dtype, codes):
    """A token with such a row yields NaN for the queries that see it (its block's tokens once quantized) and nothing
    for the others, masked or in another head."""
    gen = torch.Generator().manual_seed(10)
    d, page, heads, n = 64, 64, 2, 150
    seqs = Sequences([n], heads, d, dtype, codes, page, gen)
    seqs.k[0][140, 0, 3] = float("inf")                   # in the tail
    seqs.v[0][70, 1, 9] = float("nan")                    # in a page
    cache, table, slots = filled_cache(seqs, [n], gen)
    q = rows((n, 2 * heads, d), dtype, gen, outliers=False).to(DEV)
    ws = dq.paged_workspace(cache, 1, n, 2 * heads, n, n)
    out = dq.paged_attention(cache, q, ints([0, n]), ints([n]), table, n, n, ws, tail_slots=slots).cpu()
    bad = torch.isnan(out).any(-1)
    assert torch.equal(torch.isnan(out).all(-1), bad)
    want = torch.zeros(n, 4, dtype=torch.bool)
    want[140:, :2] = True
    want[64:, 2:] = True
    assert torch.equal(bad, want)
    # one row per call, the same
    ws = dq.paged_workspace(cache, 1, 1, 2 * heads, 1, n)
    for i in (63, 69, 139, 149):
        one = dq.paged_attention(cache, q[i:i + 1], None, ints([i + 1]) if i >= 128 else ints([i + 1]), table, 1, n, ws, tail_slots=slots) \
            if i >= 128 else None
        if one is not None:
            assert torch.equal(torch.isnan(one.cpu()).any(-1)[0], want[i])


# ---------------------------------------------------------------------------------------- attention
def _run(seqs, lens, new, hq, gen, causal=True, window=0, scale=0.0, max_len=None, cache=None, strided=False, tail=None):
    dtype, d = seqs.dtype, seqs.d
    if cache is None:
        cache = filled_cache(seqs, lens, gen)
    cache, table, slots = cache
    total = sum(new)
    q = rows((total + 3, hq, d), dtype, gen, outliers=False)
    qd = q.to(DEV)
    if strided:                                           # heads of a wider row
        wide = torch.zeros((total + 3, hq + 5, d), dtype=dtype, device=DEV)
        wide[:, 2:2 + hq] = qd
        qd = wide[:, 2:2 + hq]
    out = torch.full((total + 3, hq, d), 5.0, dtype=dtype, device=DEV)
    max_len = max(lens) if max_len is None else max_len
    ws = dq.paged_workspace(cache, len(lens), total + 3, hq, max(new), max_len)
    starts = ints(_sums(new))
    got = None
    for _ in range(2):                                    # the workspace is left as it was found
        out.fill_(5.0)
        dq.paged_attention(cache, qd, starts, ints(lens), table, max(new), max_len, ws, out=out, softmax_scale=scale, causal=causal,
                           window=window, tail_slots=slots)
        assert got is None or torch.equal(got, out.cpu())
        got = out.cpu()
    assert (got[total:] == 5.0).all()                     # rows behind the last sequence's
    at = 0
    for b, n in enumerate(new):
        if not n:
            continue
        ln = lens[b]
        k, v = seqs.stored(seqs.k[b], lens[b])[:ln], seqs.stored(seqs.v[b], lens[b])[:ln]
        place = torch.arange(ln - n, ln)
        want, size, ds = attend64(q[at:at + n], k, v, place, causal, window, scale if scale > 0 else 1 / math.sqrt(d))
        tol = attend_tolerance(want, size, ds, float(v.abs().max()) if ln else 0.0, ln, dtype, True)
        err = (got[at:at + n].double() - want).abs()
        assert (err <= tol).all(), (b, n, lens[b], float(err.max()), float((err / tol).max()))
        at += n
    return got


@pytest.mark.parametrize("dtype,codes", FORMATS)
@pytest.mark.parametrize("d,page,heads,group", [(128, 64, 2, 1), (128, 128, 3, 4), (64, 64, 1, 16), (64, 128, 2, 7)])
def test_one_token_per_sequence(dtype, codes, d, page, heads, group):
    gen = torch.Generator().manual_seed(d + page + group)
    lens = [1, 2, 63, 64, 65, 127, 128, 129, 200, 1000]
    print("decode", dtype, codes, d, page, heads, group, flush=True)
    seqs = Sequences(lens, heads, d, dtype, codes, page, gen)
    _run(seqs, lens, [1] * len(lens), heads * group, gen, strided=group == 4)


@pytest.mark.parametrize("dtype,codes", FORMATS[:2])
@pytest.mark.parametrize("batch,heads,group,length", [(1, 1, 1, 9000), (2, 1, 8, 5001), (1, 2, 3, 20000)])
def test_one_token_long_and_split(dtype, codes, batch, heads, group, length):
    gen = torch.Generator().manual_seed(length)
    lens = [length - 333 * i for i in range(batch)]
    seqs = Sequences(lens, heads, 128, dtype, codes, 64, gen)
    _run(seqs, lens, [1] * batch, heads * group, gen)


@pytest.mark.parametrize("dtype,codes", FORMATS[:2])
@pytest.mark.parametrize("window,causal", [(0, True), (50, True), (1, True), (1000, True), (0, False)])
def test_drafted_tokens_windows_and_no_causality(dtype, codes, window, causal):
    gen = torch.Generator().manual_seed(window)
    lens, new = [5, 64, 70, 129, 300, 777, 0, 3], [5, 4, 1, 5, 2, 5, 0, 5]      # the last has more rows than tokens
    seqs = Sequences(lens, 2, 128, dtype, codes, 64, gen)
    _run(seqs, lens, new, 6, gen, causal=causal, window=window)


@pytest.mark.parametrize("dtype,codes", FORMATS)
@pytest.mark.parametrize("d,page,heads,group", [(128, 64, 2, 1), (128, 128, 1, 4), (64, 64, 2, 3), (64, 128, 1, 1)])
def test_prompts(dtype, codes, d, page, heads, group):
    gen = torch.Generator().manual_seed(d + page + group)
    lens = [1, 33, 64, 65, 130, 200, 517, 0, 700]
    new = [1, 33, 64, 65, 130, 150, 517, 0, 3]
    print("prompt", dtype, codes, d, page, heads, group, flush=True)
    seqs = Sequences(lens, heads, d, dtype, codes, page, gen)
    _run(seqs, lens, new, heads * group, gen, strided=group == 3)


@pytest.mark.parametrize("window,causal,scale", [(100, True, 0.0), (1, True, 0.0), (0, False, 0.01), (0, True, 1.0)])
def test_prompts_windows_scales_and_no_causality(window, causal, scale):
    gen = torch.Generator().manual_seed(window + 1)
    lens, new = [300, 90, 40, 17], [300, 60, 3, 25]       # the last has more rows than tokens
    seqs = Sequences(lens, 2, 64, F16, E4M3, 64, gen)
    _run(seqs, lens, new, 4, gen, causal=causal, window=window, scale=scale)


@pytest.mark.parametrize("dtype,codes", FORMATS[:2])
def test_a_piece_of_a_prompt_behind_a_long_cache(dtype, codes):
    gen = torch.Generator().manual_seed(77)
    lens, new = [6001, 3333], [70, 40]
    seqs = Sequences(lens, 1, 128, dtype, codes, 64, gen)
    _run(seqs, lens, new, 4, gen)


@pytest.mark.parametrize("new", [1, 60])
@pytest.mark.parametrize("dtype,codes", FORMATS[:2])
def test_values_of_very_different_ranges(dtype, codes, new):
    """The largest contribution may come from a page whose tokens weigh little."""
    gen = torch.Generator().manual_seed(3)
    span = (0, 5, -9, 3, -12) if dtype == F16 else (0, 30, -30, 12, -60)
    seqs = Sequences([700, 400], 2, 64, dtype, codes, 64, gen, v_range=span)
    _run(seqs, [700, 400], [new, new], 4, gen)


@pytest.mark.parametrize("new", [1, 3, 50])
def test_results_do_not_depend_on_the_bound_on_lengths(new):
    """max_seq_len sizes the launch only: a guess far too small or too large gives results within the tolerance."""
    gen = torch.Generator().manual_seed(4)
    lens = [3000, 100]
    seqs = Sequences(lens, 1, 64, F16, INT8, 64, gen)
    cache = filled_cache(seqs, lens, gen)
    for bound in (0, 64, 1000, 3000, 10 ** 6):
        _run(seqs, lens, [new, new], 2, torch.Generator().manual_seed(5), max_len=bound, cache=cache)


def test_rows_behind_the_bound_on_rows_leave_the_others_right():
    """A sequence with more rows than max_rows: those up to the bound come out as they would, none out of bounds."""
    gen = torch.Generator().manual_seed(6)
    seqs = Sequences([200], 1, 64, F16, INT8, 64, gen)
    cache, table, slots = filled_cache(seqs, [200], gen)
    q = rows((9, 2, 64), F16, gen, outliers=False).to(DEV)
    ws = dq.paged_workspace(cache, 1, 9, 2, 9, 200)
    want = dq.paged_attention(cache, q, ints([0, 9]), ints([200]), table, 9, 200, ws, tail_slots=slots).cpu().double()
    got = dq.paged_attention(cache, q, ints([0, 9]), ints([200]), table, 4, 200, ws, tail_slots=slots).cpu().double()
    # the two kernels round differently: twice the half step of the result and of the probabilities, whose terms are at most max |v|
    assert ((got[:4] - want[:4]).abs() <= 2 * (want[:4].abs() + float(seqs.v[0].abs().max())) * 2.0 ** -11).all()


@pytest.mark.parametrize("new", [1, 40])
def test_pages_and_slots_that_do_not_exist(new):
    """No read or write follows them: their tokens make NaN for those who see them, appended rows are dropped."""
    gen = torch.Generator().manual_seed(11)
    lens = [200, 200, 200]
    seqs = Sequences(lens, 1, 64, F16, INT8, 64, gen)
    cache, table, slots = filled_cache(seqs, lens, gen)
    good = table.clone()
    table[0, 1] = 10 ** 9
    table[1, 0] = -1
    bad_slots = slots.clone()
    bad_slots[2] = 99
    q = rows((3 * new, 2, 64), F16, gen, outliers=False).to(DEV)
    starts = ints(_sums([new] * 3))
    ws = dq.paged_workspace(cache, 3, 3 * new, 2, new, 200)
    fine = dq.paged_attention(cache, q, starts, ints(lens), good, new, 200, ws, tail_slots=slots).cpu()
    assert torch.isfinite(fine).all()
    got = dq.paged_attention(cache, q, starts, ints(lens), table, new, 200, ws, tail_slots=bad_slots).cpu().view(3, new, 2, 64)
    assert torch.isnan(got[0]).all() and torch.isnan(got[1]).all()
    sees = torch.arange(200 - new, 200) >= 192            # rows before the tail do not see it
    assert torch.isnan(got[2, sees]).all() and torch.equal(got[2, ~sees], fine.view(3, new, 2, 64)[2, ~sees])
    # a window that ends before the bad page does not see it
    w = dq.paged_attention(cache, q, starts, ints(lens), table, new, 200, ws, window=64 - new, tail_slots=slots).cpu() if new < 60 else None
    ok = dq.paged_attention(cache, q, starts, ints(lens), good, new, 200, ws, window=64 - new, tail_slots=slots).cpu()
    assert torch.equal(w, ok)
    kept = {n: t.clone() for n, t in cache.t.items()}
    rows_k = rows((70 * 3, 1, 64), F16, gen).to(DEV)
    table[:, :] = 10 ** 9
    dq.paged_append(cache, rows_k, rows_k, ints([0, 70, 140, 210]), ints([256 + 6] * 3), torch.cat([table, table], 1), tail_slots=ints([-1, 99, 2 ** 30]))
    dq.paged_append(cache, rows_k, rows_k, ints([0, 70, 140, 210]), ints([10 ** 6] * 3), table, tail_slots=slots)     # past the table
    torch.cuda.synchronize()
    for n, t in cache.t.items():
        assert torch.equal(t.view(torch.uint8), kept[n].view(torch.uint8)), n


@pytest.mark.parametrize("starts", [[0, 1000, 40], [-5, 20, 40], [0, 30, 10], [2 ** 31 - 1, -1, 2 ** 31 - 1], [40, 0, 40]])
def test_starts_that_make_no_sense_stay_in_bounds(starts):
    gen = torch.Generator().manual_seed(12)
    seqs = Sequences([200, 200], 1, 64, F16, INT8, 64, gen)
    cache, table, slots = filled_cache(seqs, [200, 200], gen)
    q = rows((40, 2, 64), F16, gen, outliers=False).to(DEV)
    ws = dq.paged_workspace(cache, 2, 40, 2, 40, 200)
    dq.paged_attention(cache, q, ints(starts), ints([200, 200]), table, 40, 200, ws, tail_slots=slots)
    k = rows((40, 1, 64), F16, gen).to(DEV)
    dq.paged_append(cache, k, k, ints(starts), ints([200, 200]), table, q=q, rotary=dq.rotary(64, device=DEV), tail_slots=slots)
    dq.paged_read(cache, None, ints([200, 200]), ints(starts), table, torch.empty_like(k), torch.empty_like(k), tail_slots=slots)
    torch.cuda.synchronize()


def test_a_pool_past_32_bit_offsets():
    """Pages and slots whose bytes lie past 2^32."""
    gen = torch.Generator().manual_seed(13)
    heads, d, page = 16, 128, 64
    lens = [150, 64]
    seqs = Sequences(lens, heads, d, F16, INT8, page, gen)
    pages = (1 << 32) // (heads * d * page) + 200
    slots = (1 << 32) // (heads * d * page * 2) + 200
    cache = dq.PagedCache({n: torch.empty(shape, dtype=t, device=DEV) for n, (shape, t) in
                           dq.paged._paged_shapes(pages, slots, heads, d, page, F16, INT8).items()})
    table = ints([[pages - 1, pages - 50, 3], [pages - 7, 0, 0]])
    at = ints([slots - 1, slots - 2])
    dq.paged_append(cache, torch.cat(seqs.k).to(DEV), torch.cat(seqs.v).to(DEV), ints(_sums(lens)), ints(lens), table, tail_slots=at)
    k, v, starts = read_back(cache, lens, table, at)
    for b in range(2):
        want = seqs.stored(seqs.k[b])
        assert (k[starts[b]:starts[b + 1]].double() - want).abs().le(want.abs() * 2.0 ** -11 * 1.01 + 2.0 ** -24).all()
    for new in ([1, 1], [30, 20]):
        _run(seqs, lens, new, heads, gen, cache=(cache, table, at))


def test_a_shared_prefix_a_chain_of_calls_and_a_captured_graph():
    """A serving run: two sequences share their first page, a prompt is appended and attended, then tokens one by one
    through a captured graph whose inputs change, across a page's end; every step against the 64-bit form."""
    gen = torch.Generator().manual_seed(14)
    heads, hq, d, page, n0, steps = 2, 4, 64, 64, 120, 14
    seqs = Sequences([n0 + steps, n0 + steps], heads, d, BF16, E4M3, page, gen)
    seqs.k[1][:page], seqs.v[1][:page] = seqs.k[0][:page], seqs.v[0][:page]
    cache = dq.alloc_paged_cache(8, 2, heads, d, page, BF16, E4M3, DEV)
    fill_tails(cache)
    table = ints([[5, 1, 7], [5, 2, 0]])                  # page 5 is both sequences' first
    lens = ints([n0, n0])
    dq.paged_append(cache, torch.cat([s[:n0] for s in seqs.k]).to(DEV), torch.cat([s[:n0] for s in seqs.v]).to(DEV), ints([0, n0, 2 * n0]), lens, table)
    _run(seqs, [n0, n0], [n0, n0], hq, gen, cache=(cache, table, None))
    k1, v1 = (torch.empty((2, heads, d), dtype=BF16, device=DEV) for _ in range(2))
    q1 = torch.empty((2, hq, d), dtype=BF16, device=DEV)
    out = torch.empty_like(q1)
    ws = dq.paged_workspace(cache, 2, 2, hq, 1, 3 * page)

    def step():
        lens.add_(1)
        dq.paged_append(cache, k1, v1, None, lens, table)
        dq.paged_attention(cache, q1, None, lens, table, 1, 3 * page, ws, out=out)

    st, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    for i in range(steps):
        n = n0 + i
        k1.copy_(torch.stack([s[n] for s in seqs.k]))
        v1.copy_(torch.stack([s[n] for s in seqs.v]))
        q = rows((2, hq, d), BF16, gen, outliers=False)
        q1.copy_(q)
        torch.cuda.synchronize()
        if i == 0:
            with torch.cuda.stream(st):
                step()
                st.synchronize()
                with torch.cuda.graph(graph, stream=st):
                    step()
        else:
            torch.randn(1 << 16, device=DEV).sum()        # eager work between the replays
            graph.replay()
        torch.cuda.synchronize()
        assert lens.tolist() == [n + 1, n + 1]
        for b in range(2):
            kk, vv = seqs.stored(seqs.k[b], n + 1), seqs.stored(seqs.v[b], n + 1)
            want, size, ds = attend64(q[b:b + 1], kk, vv, torch.tensor([n]), True, 0, 1 / math.sqrt(d))
            tol = attend_tolerance(want, size, ds, float(vv.abs().max()), n + 1, BF16, True)
            assert ((out[b:b + 1].cpu().double() - want).abs() <= tol).all(), (i, b)


def test_two_streams_with_a_workspace_each():
    gen = torch.Generator().manual_seed(15)
    seqs = Sequences([3000, 2000], 2, 128, F16, E4M3, 64, gen)
    cache, table, slots = filled_cache(seqs, [3000, 2000], gen)
    q = [rows((2, 4, 128), F16, gen, outliers=False).to(DEV) for _ in range(2)]
    lens = ints([3000, 2000])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    want = []
    for x in q:
        ws = dq.paged_workspace(cache, 2, 2, 4, 1, 3000)
        want.append(dq.paged_attention(cache, x, None, lens, table, 1, 3000, ws, tail_slots=slots).cpu())
    spaces = [dq.paged_workspace(cache, 2, 2, 4, 1, 3000) for _ in range(2)]
    outs = [torch.empty_like(x) for x in q]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, x, ws, o in zip(streams, q, spaces, outs):
            with torch.cuda.stream(st):
                dq.paged_attention(cache, x, None, lens, table, 1, 3000, ws, out=o, tail_slots=slots)
    torch.cuda.synchronize()
    assert all(torch.equal(o.cpu(), w) for o, w in zip(outs, want))


def test_the_output_may_be_the_query():
    gen = torch.Generator().manual_seed(16)
    seqs = Sequences([500], 2, 64, F16, INT8, 64, gen)
    cache, table, slots = filled_cache(seqs, [500], gen)
    for n in (1, 3, 100):
        q = rows((n, 4, 64), F16, gen, outliers=False).to(DEV)
        ws = dq.paged_workspace(cache, 1, n, 4, n, 500)
        want = dq.paged_attention(cache, q, ints([0, n]), ints([500]), table, n, 500, ws, tail_slots=slots)
        dq.paged_attention(cache, q, ints([0, n]), ints([500]), table, n, 500, ws, out=q, tail_slots=slots)
        assert torch.equal(q, want)


def test_from_pages_to_the_decoquant_cache():
    """paged_read's rows go straight into a DecoQuant layer, whose decode then agrees with attention over the pages as
    far as its own quantization lets it."""
    gen = torch.Generator().manual_seed(17)
    n, heads, hq = 300, 2, 4
    seqs = Sequences([n, n], heads, 128, F16, INT8, 64, gen)
    cache, table, slots = filled_cache(seqs, [n, n], gen)
    layer = dq.KVCacheLayer(dq.Format(8, 128, 128, 16, 8, 128), 2, hq, heads, 512, DEV)
    k, v = (torch.empty((2, heads, n, 128), dtype=F16, device=DEV) for _ in range(2))
    for b in range(2):
        dq.paged_read(cache, None, ints([n]), ints([0, n]), table[b:b + 1], k[b].transpose(0, 1), v[b].transpose(0, 1), tail_slots=slots[b:b + 1])
    layer.prefill(k, v)
    q = rows((2, hq, 128), F16, gen, outliers=False).to(DEV)
    a = layer.decode(q).cpu().double()
    ws = dq.paged_workspace(cache, 2, 2, hq, 1, n)
    p = dq.paged_attention(cache, q, None, ints([n, n]), table, 1, n, ws, tail_slots=slots).cpu().double()
    assert torch.equal(k[0].transpose(0, 1).cpu(), read_back(cache, [n, n], table, slots)[0][:n])
    # 8-bit codes of the factored block: keys and values off by under 2 % of their norm, and attention to what the scores make of that
    assert float((a - p).norm() / p.norm()) < 0.2


def test_a_workspace_of_the_largest_sizes_serves_all_smaller_ones_in_turn():
    """Prompts, pieces, drafted and single tokens, long and short, one workspace after the other call's leavings."""
    gen = torch.Generator().manual_seed(18)
    lens = [9000, 300, 64, 4000]
    seqs = Sequences(lens, 2, 64, F16, E4M3, 64, gen)
    cache, table, slots = filled_cache(seqs, lens, gen)
    ws = dq.paged_workspace(cache, 4, 1200, 4, 300, 9000)
    want = {}
    for turn in range(2):
        for new, cut in (([300, 300, 60, 300], 9000), ([1, 1, 1, 1], 9000), ([40, 1, 2, 90], 9000), ([4, 4, 4, 4], 9000), ([1, 1, 1, 1], 320), ([64, 64, 64, 64], 256)):
            now = [min(n, cut // 64 * 64) if n > cut else n for n in lens]
            q = rows((sum(new), 4, 64), F16, torch.Generator().manual_seed(len(want) if turn == 0 else list(want).index((tuple(new), cut))), outliers=False)
            out = dq.paged_attention(cache, q.to(DEV), ints(_sums(new)), ints(now), table, max(new), cut, ws, tail_slots=slots).cpu()
            key = (tuple(new), cut)
            if turn == 0:
                own = dq.paged_workspace(cache, 4, sum(new), 4, max(new), cut)
                want[key] = dq.paged_attention(cache, q.to(DEV), ints(_sums(new)), ints(now), table, max(new), cut, own, tail_slots=slots).cpu()
            assert torch.equal(out, want[key]), key


@pytest.mark.parametrize("dtype,codes", FORMATS[:2])
def test_splits_of_every_kernel_agree(dtype, codes):
    """The launch override changes how the work is dealt, not what is computed."""
    gen = torch.Generator().manual_seed(19)
    lens = [3000, 700, 65]
    seqs = Sequences(lens, 2, 128, dtype, codes, 128, gen)
    cache, table, slots = filled_cache(seqs, lens, gen)
    for new in ([1, 1, 1], [100, 33, 64]):
        q = rows((sum(new), 8, 128), dtype, gen, outliers=False).to(DEV)
        ws = torch.zeros(1 << 28, dtype=torch.uint8, device=DEV)
        outs = [dq.paged_attention(cache, q, ints(_sums(new)), ints(lens), table, max(new), 3000, ws, tail_slots=slots, splits=n).cpu().double()
                for n in (1, 2, 5, 32, 64)]
        at = 0
        for b, n in enumerate(new):
            k, v = seqs.stored(seqs.k[b]), seqs.stored(seqs.v[b])
            want, size, ds = attend64(q[at:at + n].cpu(), k, v, torch.arange(lens[b] - n, lens[b]), True, 0, 128 ** -0.5)
            tol = attend_tolerance(want, size, ds, float(v.abs().max()), lens[b], dtype, True)
            for o in outs:
                assert ((o[at:at + n] - want).abs() <= tol).all()
            at += n


def test_a_layer_from_projections_to_outputs():
    """PagedKVLayer: prompts of mixed lengths, a step, drafted tokens, all from raw projections with norm and rotation,
    against the 64-bit forms of every stage; then its rows move to a DecoQuant layer."""
    from paged_util import heads64
    gen = torch.Generator().manual_seed(20)
    heads, hq, d, dtype = 2, 6, 128, F16
    layer = dq.PagedKVLayer(3, hq, heads, d, 300, 64, dtype, INT8, DEV)
    rot = dq.rotary(d, device=DEV)
    wq, wk = (1 + 0.2 * torch.randn(2, d, generator=gen)).to(dtype)
    seen = Sequences([0, 0, 0], heads, d, dtype, INT8, 64, gen)
    for new in ([130, 63, 1], [1, 1, 1], [3, 0, 2], [64, 64, 64]):
        total = sum(new)
        fused = rows((total, hq + 2 * heads, d), dtype, gen).to(DEV)
        starts = None if new == [1, 1, 1] else ints(_sums(new))
        q = layer.append(fused[:, hq:hq + heads], fused[:, hq + heads:], starts, max(new), q=fused[:, :hq], rotary=rot, q_weight=wq.to(DEV), k_weight=wk.to(DEV))
        out = layer.attend(q, starts, max(new))
        host, at = fused.cpu(), 0
        place = torch.cat([torch.arange(len(k), len(k) + n) for k, n in zip(seen.k, new)])
        q64, _ = heads64(host[:, :hq], wq, 1e-6, rot.inv_freq.cpu(), None, place, d, False)
        assert ((q.cpu().double() - q64).abs() <= q64.abs() * 2.0 ** -11 + 2.0 ** -17 * q64.abs().amax(-1, keepdim=True) + 2.0 ** -24).all()
        # (the rows the cache took are the operator's own: their rounding is checked above and in the tests of the norm)
        kk, _ = dq.rotate_heads(fused[:, hq:hq + heads], None, place.to(torch.int32).to(DEV), rot, q_weight=wk.to(DEV))
        for b, n in enumerate(new):
            seen.k[b] = torch.cat([seen.k[b], kk[at:at + n].cpu()])
            seen.v[b] = torch.cat([seen.v[b], host[at:at + n, hq + heads:]])
            if n:
                k, v, ln = seen.stored(seen.k[b]), seen.stored(seen.v[b]), len(seen.k[b])
                want, size, ds = attend64(q[at:at + n].cpu(), k, v, torch.arange(ln - n, ln), True, 0, d ** -0.5)
                tol = attend_tolerance(want, size, ds, float(v.abs().max()), ln, dtype, True)
                assert ((out[at:at + n].cpu().double() - want).abs() <= tol).all(), (b, new)
            at += n
    lens = [len(k) for k in seen.k]
    assert layer.seq_lens.tolist() == lens
    k, v = layer.read(lens)
    for b, n in enumerate(lens):
        for got, x in ((k, seen.k), (v, seen.v)):
            want = seen.stored(x[b])
            assert ((got[b, :, :n].transpose(0, 1).cpu().double() - want).abs() <= want.abs() * 2.0 ** -11 * (1 + 2.0 ** -12) + 2.0 ** -25).all()
            assert (got[b, :, n:] == 0).all()
    small = dq.KVCacheLayer(dq.Format(8, 128, d, 16, 8, 128), 3, hq, heads, 512, DEV)
    small.prefill(k, v, counts=lens)
    assert torch.isfinite(small.decode(torch.ones((3, hq, d), dtype=dtype, device=DEV))).all()
    with pytest.raises(dq.DQError, match="exceed"):
        layer.append(fused[:3, hq:hq + heads], fused[:3, hq + heads:], ints([0, 3, 3, 3]), 200)


def test_the_decoquant_layer_takes_projections():
    """KVCacheLayer.append_projected is rotate_heads and append (prefill) of its rows, bit for bit."""
    gen = torch.Generator().manual_seed(21)
    bsz, heads, hq, d = 2, 2, 4, 128
    fmt = dq.Format(4, 128, d, 16, 8, 128)
    a, b = (dq.KVCacheLayer(fmt, bsz, hq, heads, 512, DEV) for _ in range(2))
    rot = dq.rotary(d, device=DEV)
    w = (1 + 0.2 * torch.randn(2, d, generator=gen)).to(F16).to(DEV)
    have = 0
    for n in (150, 1, 130):
        fused = rows((bsz, n, hq + 2 * heads, d), F16, gen).to(DEV)
        q, k, v = fused[:, :, :hq], fused[:, :, hq:hq + heads], fused[:, :, hq + heads:]
        pos = torch.arange(have, have + n, dtype=torch.int32, device=DEV).expand(bsz, n).contiguous()
        have += n
        qa = a.append_projected(q, k, v, pos, rot, q_weight=w[0], k_weight=w[1], prompt=n == 150)
        qb, kb = dq.rotate_heads(q, k, pos, rot, q_weight=w[0], k_weight=w[1])
        (b.prefill if n == 150 else b.append)(kb.transpose(1, 2).contiguous(), v.transpose(1, 2).contiguous())
        assert torch.equal(qa, qb)
        oa, ob = a.decode(qa[:, -1].contiguous()), b.decode(qb[:, -1].contiguous())
        assert torch.equal(oa, ob)
    for n in a.cache.t:
        assert torch.equal(a.cache.t[n], b.cache.t[n]), n


@pytest.mark.parametrize("dtype,codes", FORMATS[:2])
def test_batches_of_very_different_lengths(dtype, codes):
    """Slots are dealt by length: one long sequence among short and empty ones, rows without tokens before them, more
    sequences than a wave has lanes, with and without a window."""
    gen = torch.Generator().manual_seed(22)
    lens = [3, 9000, 0, 64, 1, 700, 2500, 65]
    new = [1, 1, 0, 1, 1, 1, 0, 1]
    seqs = Sequences(lens, 1, 128, dtype, codes, 64, gen)
    cache = filled_cache(seqs, lens, gen)
    for window in (0, 300):
        _run(seqs, lens, new, 4, torch.Generator().manual_seed(1), cache=cache, window=window)
    lens = [int(x) for x in torch.randint(0, 400, (70,), generator=gen)]
    lens[5], lens[66] = 4000, 1500
    seqs = Sequences(lens, 1, 64, dtype, codes, 64, gen)
    _run(seqs, lens, [min(n, 1 + i % 3) for i, n in enumerate(lens)], 4, gen)


@pytest.mark.parametrize("new", [1, 3, 300])
def test_rows_that_belong_to_no_sequence_may_come_first(new):
    """starts[0] > 0: the same bits as without the rows before it, which stay as they are, whatever bound on rows is given."""
    gen = torch.Generator().manual_seed(23)
    skip, have, hq = 700, 100, 4
    lens = [have + new] * 2
    seqs = Sequences(lens, 2, 64, F16, INT8, 64, gen)
    cache, table, slots = filled_cache(seqs, lens, gen)
    q = rows((skip + 2 * new, hq, 64), F16, gen, outliers=False).to(DEV)
    ws = dq.paged_workspace(cache, 2, skip + 2 * new, hq, new, have + new)
    out = torch.full_like(q, 5.0)
    dq.paged_attention(cache, q, ints([skip, skip + new, skip + 2 * new]), ints(lens), table, new, have + new, ws, out=out, tail_slots=slots)
    want = dq.paged_attention(cache, q[skip:], ints([0, new, 2 * new]), ints(lens), table, new, have + new, ws, tail_slots=slots)
    assert torch.equal(out[skip:], want) and (out[:skip] == 5.0).all()
    # append: keys, and queries beside them
    rot = dq.rotary(64, device=DEV)
    fused = rows((skip + 2 * new, hq + 4, 64), F16, gen).to(DEV)
    both = []
    for at, starts in ((0, [skip, skip + new, skip + 2 * new]), (skip, [0, new, 2 * new])):
        c = dq.alloc_paged_cache(cache.pages, 2, 2, 64, 64, F16, INT8, DEV)
        f = fused[at:]
        qo = torch.full((len(f), hq, 64), 5.0, dtype=F16, device=DEV)
        dq.paged_append(c, f[:, hq:hq + 2], f[:, hq + 2:], ints(starts), ints(lens), table, q=f[:, :hq], q_out=qo, rotary=rot)
        assert (qo[:starts[0]] == 5.0).all()
        back = torch.full((len(f), 2, 64), 5.0, dtype=F16, device=DEV), torch.full((len(f), 2, 64), 5.0, dtype=F16, device=DEV)
        dq.paged_read(c, ints([have, have]), ints(lens), ints(starts), table, *back)
        assert all((x[:starts[0]] == 5.0).all() for x in back)
        both.append([qo[starts[0]:]] + [x[starts[0]:] for x in back] + list(c.t.values()))
    for a, b in zip(*both):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_a_layer_after_a_refused_append_and_with_a_captured_step():
    """A refused append leaves the lengths alone; a step captured before a larger call replays with it between the replays."""
    gen = torch.Generator().manual_seed(24)
    heads, hq, d = 2, 4, 64
    layer, plain = (dq.PagedKVLayer(2, hq, heads, d, 4000, 64, F16, INT8, DEV) for _ in range(2))
    k, v = (rows((2, heads, d), F16, gen).to(DEV) for _ in range(2))
    q = rows((2, hq, d), F16, gen, outliers=False).to(DEV)
    pk, pv = (rows((1400, heads, d), F16, gen).to(DEV) for _ in range(2))
    pq = rows((1400, hq, d), F16, gen, outliers=False).to(DEV)
    starts = ints([0, 700, 1400])

    def step(x):
        x.append(k, v)
        return x.attend(q)

    for x in (layer, plain):
        x.append(pk, pv, starts, 700)
    with pytest.raises(dq.DQError):
        layer.append(k.bfloat16(), v)
    with pytest.raises(dq.DQError):
        layer.append(k, v, ints([0, 1]))
    assert layer.seq_lens.tolist() == [700, 700] and layer.tokens_upper == 700
    step(layer)                                          # (the workspace of one row each)
    step(plain)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        out = step(layer)
    for i in range(3):
        graph.replay()
        assert torch.equal(out, step(plain))
        if i:
            continue
        for x in (layer, plain):                         # needs a larger workspace
            x.append(pk, pv, starts, 700)
        hold = [layer.attend(pq, starts, 700)] + [torch.full((1 << 20,), 7, dtype=torch.uint8, device=DEV) for _ in range(64)]
        assert torch.equal(hold[0], plain.attend(pq, starts, 700))
    assert torch.equal(layer.seq_lens, plain.seq_lens)
