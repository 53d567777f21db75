"""Append, read-back and absorbed attention of the cache of latents against the definitions in 64 bits."""
import pytest
import torch

import paper_2405_12591_amd as dq
from latent_util import FORMS, Latents, attend64, check, normal, starts_of, tolerance
from paged_util import DEV, HALF, heads64, ints, rotate_tolerance

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16]


def _tree(counts, gen):
    """Random masks: a row sees itself, mostly, and any of the others."""
    out = []
    for c in counts:
        for i in range(c):
            m = int(torch.randint(0, 1 << 62, (1,), generator=gen)) * 4 + int(torch.randint(0, 4, (1,), generator=gen))
            out.append(m if i % 5 == 3 else m | 1 << i)             # bits of rows that are not there count for nothing
    return torch.tensor([m - (1 << 64) if m >> 63 else m for m in (x & (1 << 64) - 1 for x in out)], dtype=torch.int64)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("heads,lens,counts", [
    (16, [1, 31, 32, 33, 64, 65, 200], [1] * 7),                    # lengths around the tiles, a row each
    (3, [77, 5, 130], [5, 5, 2]),                                   # odd heads, a sequence that is all rows
    (8, [9, 0, 300, 40], [4, 3, 0, 7]),                             # rows of a sequence without tokens, tokens without rows
    (1, [700], [1]),
    (128, [129, 64], [1, 3]),
    (20, [513, 100, 2], [3, 1, 2]),
])
def test_attention(dtype, latent, heads, lens, counts):
    gen = torch.Generator().manual_seed(heads)
    x = Latents(lens, latent, dtype, 64 if heads != 20 else 128, gen)
    total = sum(counts) + 3
    q = normal((total, heads, latent + x.rot), dtype, gen)
    for causal in (True, False):
        got = x.attend(q.to(DEV), counts, 0.07, gap=2, causal=causal)
        check(got, *x.want(q, counts, 0.07, gap=2, causal=causal), "causal %s" % causal)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,lens,counts", [(16, [100, 64, 40], [24, 64, 40]), (5, [1000, 33], [13, 2])])
def test_trees(dtype, heads, lens, counts):
    gen = torch.Generator().manual_seed(7)
    x = Latents(lens, 512, dtype, 64, gen)
    q = normal((sum(counts), heads, 576), dtype, gen)
    seen = _tree(counts, gen)
    seen[1] = 0                                                     # a row that sees the tokens before the tree only
    got = x.attend(q.to(DEV), counts, 0.07, seen=seen)
    check(got, *x.want(q, counts, 0.07, seen=seen))
    # a chain of masks is what the places say
    chain = torch.tensor([(1 << (i + 1)) - 1 if i < 63 else -1 for c in counts for i in range(c)], dtype=torch.int64)
    assert torch.equal(x.attend(q.to(DEV), counts, 0.07, seen=chain), x.attend(q.to(DEV), counts, 0.07))


def test_a_row_of_an_empty_mask_without_tokens_before_it_is_zero():
    gen = torch.Generator().manual_seed(8)
    x = Latents([6], 256, torch.float16, 64, gen)
    q = normal((6, 9, 288), torch.float16, gen)
    seen = torch.tensor([1, 3, 0, 9, 0, 1 << 60], dtype=torch.int64)
    got = x.attend(q.to(DEV), [6], 0.1, seen=seen)
    check(got, *x.want(q, [6], 0.1, seen=seen))
    assert not got[[2, 4, 5]].any()


@pytest.mark.parametrize("latent", [512, 256])
def test_long_caches_and_many_sequences(latent):
    """Pieces of units over many workgroups; more sequences than a wave has lanes."""
    gen = torch.Generator().manual_seed(9)
    for lens in ([5000, 17, 2600], [1 + 7 * i % 190 for i in range(150)]):
        x = Latents(lens, latent, torch.bfloat16, 64, gen)
        counts = [1 + i % 2 if n > 1 else 1 for i, n in enumerate(lens)]
        q = normal((sum(counts), 6, latent + x.rot), torch.bfloat16, gen)
        want = x.want(q, counts, 0.05)
        for max_len in (max(lens), 1, 100000):                      # the bound sizes the launch only
            check(x.attend(q.to(DEV), counts, 0.05, max_len=max_len), *want, "bound %d" % max_len)


def test_a_line_of_more_than_24_bits():
    """2^24 tiles and units in one sequence: 8 million tokens over 64 pages that the table names again and again, 8192 columns."""
    gen = torch.Generator().manual_seed(10)
    x = Latents([4096], 256, torch.float16, 64, gen)
    n, rows, heads = 1 << 23, 64, 128
    table = x.table[:, :64].repeat_interleave(2048, 1)
    x.lens = [n]
    q = normal((rows, heads, 288), torch.float16, gen)
    got = x.attend(q.to(DEV), [rows], 0.05, causal=False, table=table).double().cpu()
    some = slice(0, 64, 21)
    see = torch.ones(4, 4096, dtype=torch.bool)
    o, size, ds = attend64(q[some], x.rows[0], x.rows[0][:, :256], see, 0.05)
    # on top of what shorter caches may be off by: a workgroup's 2^16 tiles are 2^17 additions to a result, four roundings each, and 2^19
    # to a lane's sum of probabilities, at half a step each
    v_max = float(x.rows[0][:, :256].double().abs().max())
    tol = tolerance(o, size, ds, v_max, 4096, torch.float16) + size * (2.0 ** -5 + 2.0 ** -5)
    assert bool(((got[some] - o).abs() <= tol).all())


@pytest.mark.parametrize("heads", [16, 24, 128])
def test_pages_whose_offsets_take_more_than_32_bits(heads):
    gen = torch.Generator().manual_seed(11)
    x, off = Latents([300, 65], 512, torch.bfloat16, 64, gen), 60000
    far = torch.empty((off + x.pool, 64, 576), dtype=torch.bfloat16, device=DEV)
    far[off:] = x.cache.rows
    x.cache = dq.LatentCache(far, 512)
    x.table = torch.where(x.table >= 0, x.table + off, x.table)
    q = normal((4, heads, 576), torch.bfloat16, gen)
    check(x.attend(q[:2].to(DEV), [1, 1], 0.05), *x.want(q[:2], [1, 1], 0.05))
    check(x.attend(q.to(DEV), [2, 2], 0.05), *x.want(q, [2, 2], 0.05))
    new = normal((2, 576), torch.bfloat16, gen).to(DEV)
    dq.latent_append(x.cache, new[:, :512], new[:, 512:], None, ints([300, 65]), x.table.to(DEV))     # the last tokens again
    out = torch.zeros((365, 576), dtype=torch.bfloat16, device=DEV)
    dq.latent_read(x.cache, None, ints([300, 65]), ints([0, 300, 365]), x.table.to(DEV), out)
    want = torch.cat([x.rows[0][:299], new[:1].cpu(), x.rows[1][:64], new[1:].cpu()])
    assert torch.equal(out.cpu(), want)


def test_rows_past_the_bound_are_left():
    gen = torch.Generator().manual_seed(10)
    x = Latents([90, 40], 512, torch.float16, 64, gen)
    q = normal((9, 4, 576), torch.float16, gen)
    want, tol, own = x.want(q, [6, 3], 0.07)
    got = x.attend(q.to(DEV), [6, 3], 0.07, max_rows=3).double().cpu()
    assert bool(((got - want).abs() <= tol)[[0, 1, 2, 6, 7, 8]].all()) and bool((got[3:6] == 7).all())


def test_places_past_the_page_table_and_pages_that_do_not_exist():
    gen = torch.Generator().manual_seed(11)
    x = Latents([200, 150], 512, torch.bfloat16, 64, gen)
    q = normal((2, 7, 576), torch.bfloat16, gen)
    table = x.table.clone()
    table[0, 1] = x.pool                                            # a page that does not exist: NaN for who sees it
    got = x.attend(q.to(DEV), [1, 1], 0.07, table=table)
    want, tol, _ = x.want(q, [1, 1], 0.07)
    assert got[0].isnan().all() and bool(((got[1].double().cpu() - want[1]).abs() <= tol[1]).all())
    # lengths past the table: tokens behind it are not there, places stay
    narrow = x.table[:, :2].contiguous()
    got = x.attend(q.to(DEV), [1, 1], 0.07, table=narrow)
    y = Latents([128, 128], 512, torch.bfloat16, 64, gen)
    y.rows = [r[:128] for r in x.rows]
    check(got, *y.want(q, [1, 1], 0.07, causal=False))


def test_not_finite_rows_are_nan_for_those_who_see_them_only():
    gen = torch.Generator().manual_seed(12)
    dtype, lens, counts = torch.float16, [70, 64], [10, 4]
    x = Latents(lens, 512, dtype, 64, gen)
    # appended again, two rows with values that are not finite
    x.rows[0][65, 17], x.rows[1][61, 500] = float("inf"), float("nan")
    new = torch.cat([x.rows[0][60:], x.rows[1][60:]]).to(DEV)
    dq.latent_append(x.cache, new[:, :512], new[:, 512:], ints(starts_of(counts)), ints(lens), x.table.to(DEV))
    q = normal((14, 3, 576), dtype, gen)
    got = x.attend(q.to(DEV), counts, 0.07)
    clean = [r.clone() for r in x.rows]
    x.rows[0][65, 17], x.rows[1][61, 500] = 1.0, 1.0
    want, tol, _ = x.want(q, counts, 0.07)
    x.rows = clean
    see = [i for i in range(14) if (i < 10 and i >= 5) or i >= 11]
    rest = [i for i in range(14) if i not in see]
    assert got[see].isnan().all()
    assert bool(((got.double().cpu() - want).abs() <= tol)[rest].all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("latent,page,interleaved,normed,own_places", [(512, 64, False, True, True), (512, 128, True, False, False), (256, 64, True, True, False),
                                                                       (256, 128, False, True, True)])
def test_append_and_read(dtype, latent, page, interleaved, normed, own_places):
    gen = torch.Generator().manual_seed(13)
    rot_dim, heads = FORMS[latent], 5
    lens, counts, gap = [5, 300, 64, 7, 129, 1], [5, 170, 1, 0, 129, 1], 2
    total = sum(counts) + gap + 4
    x = Latents(lens, latent, dtype, page, gen)
    before = x.cache.rows.cpu().clone()
    fused = normal((total, latent + rot_dim + heads * rot_dim + 8), dtype, gen)
    weight = (1 + 0.2 * torch.randn(latent, generator=gen)).to(dtype) if normed else None
    places = [n - c + i for n, c in zip(lens, counts) for i in range(c)]
    positions = torch.zeros(total, dtype=torch.int32)
    positions[gap:gap + len(places)] = torch.tensor(places) if own_places else torch.randint(-5, 1 << 30, (len(places),), generator=gen).to(torch.int32)
    rotary = dq.rotary(rot_dim, interleaved=interleaved)
    f = fused.to(DEV)
    view = f[:, latent + rot_dim:latent + rot_dim + heads * rot_dim].view(total, heads, rot_dim)
    out = torch.full((total, heads, latent + rot_dim), 7.0, dtype=dtype, device=DEV)
    dq.latent_append(x.cache, f[:, :latent], f[:, latent:latent + rot_dim], ints(starts_of(counts, gap)), ints(lens), x.table.to(DEV), q=view,
                     q_out=out[..., latent:], rotary=rotary, positions=None if own_places else positions.to(DEV),
                     weight=None if weight is None else weight.to(DEV), eps=1e-5)
    # the queries: rows of no sequence, and channels that are not theirs, as they were
    rows = slice(gap, gap + len(places))
    inv = rotary.inv_freq.cpu()
    y, mag = heads64(view.cpu()[rows], None, 0, inv, None, positions[rows], rot_dim, interleaved)
    got = out.cpu()
    assert bool(((got[rows, :, latent:].double() - y).abs() <= rotate_tolerance(y, mag, dtype)).all())
    assert bool((got[:gap] == 7).all()) and bool((got[gap + len(places):] == 7).all()) and bool((got[..., :latent] == 7).all())
    # the cache
    c = fused[rows, :latent].double()
    if normed:
        c = c * weight.double() / (c.square().mean(-1, keepdim=True) + 1e-5).sqrt()
    k, mag = heads64(fused[rows, None, latent:latent + rot_dim], None, 0, inv, None, positions[rows], rot_dim, interleaved)
    tol = torch.cat([c.abs() * (HALF[dtype] + 2.0 ** -17 if normed else 0) + (2.0 ** -24 if normed else 0), rotate_tolerance(k, mag, dtype)[:, 0]], 1)
    c = torch.cat([c, k[:, 0]], 1)
    first = [max(n - k - 3, 0) for n, k in zip(lens, counts)]
    at = starts_of([n - f for n, f in zip(lens, first)], 1)
    read = torch.full((at[-1] + 2, latent + rot_dim), 7.0, dtype=dtype, device=DEV)
    dq.latent_read(x.cache, ints(first), ints(lens), ints(at), x.table.to(DEV), read)
    read, row = read.cpu(), 0
    assert bool((read[0] == 7).all()) and bool((read[-2:] == 7).all())
    for b, (n, k, f) in enumerate(zip(lens, counts, first)):
        part = read[at[b]:at[b + 1]]
        assert torch.equal(part[:n - k - f], x.rows[b][f:n - k])
        assert bool(((part[n - k - f:].double() - c[row:row + k]).abs() <= tol[row:row + k]).all())
        row += k
    # nothing else was written
    after = x.cache.rows.cpu()
    written = torch.zeros(x.pool, page, dtype=torch.bool)
    for b, (n, k) in enumerate(zip(lens, counts)):
        for t in range(n - k, n):
            written[int(x.table[b, t // page]), t % page] = True
    same = (after.view(torch.int16) == before.view(torch.int16)).all(-1)
    assert bool((same | written).all())


def test_appended_rows_do_not_depend_on_the_cut_and_queries_may_be_their_own_output():
    gen = torch.Generator().manual_seed(14)
    lens = [150, 61]
    weight, rotary = (1 + 0.1 * torch.randn(512, generator=gen)).half().to(DEV), dq.rotary(64)
    rows = normal((211, 576), torch.float16, gen).to(DEV)
    q = normal((211, 3, 64), torch.float16, gen).to(DEV)
    x, y = (Latents(lens, 512, torch.float16, 64, torch.Generator().manual_seed(1)) for _ in range(2))
    whole = q.clone()
    dq.latent_append(x.cache, rows[:, :512], rows[:, 512:], ints([0, 150, 211]), ints(lens), x.table.to(DEV), q=whole, q_out=whole, rotary=rotary, weight=weight)
    done = [0, 0]
    parts = torch.empty_like(q)
    for step in ([1, 5], [64, 1], [85, 55]):
        own = [rows[done[0]:done[0] + step[0]], rows[150 + done[1]:150 + done[1] + step[1]]]
        qq = torch.cat([q[done[0]:done[0] + step[0]], q[150 + done[1]:150 + done[1] + step[1]]])
        r = torch.cat(own)
        now = [done[0] + step[0], done[1] + step[1]]
        o = dq.latent_append(y.cache, r[:, :512], r[:, 512:], ints(starts_of(step)), ints(now), y.table.to(DEV), q=qq, rotary=rotary, weight=weight)
        parts[done[0]:now[0]], parts[150 + done[1]:150 + now[1]] = o[:step[0]], o[step[0]:]
        done = now
    assert torch.equal(whole, parts)
    assert torch.equal(x.cache.rows.view(torch.int16), y.cache.rows.view(torch.int16))


def test_append_and_read_without_a_page():
    gen = torch.Generator().manual_seed(15)
    x = Latents([130, 64], 256, torch.bfloat16, 64, gen)
    before = x.cache.rows.clone()
    table = x.table.clone()
    table[0, 1] = -1
    rows = normal((194, 288), torch.bfloat16, gen).to(DEV)
    dq.latent_append(x.cache, rows[:, :256], rows[:, 256:], ints([0, 130, 194]), ints([130, 64]), table.to(DEV))
    assert torch.equal(x.cache.rows[int(x.table[0, 1])].view(torch.int16), before[int(x.table[0, 1])].view(torch.int16))
    out = torch.full((194, 288), 7.0, dtype=torch.bfloat16, device=DEV)
    dq.latent_read(x.cache, None, ints([130, 64]), ints([0, 130, 194]), table.to(DEV), out)
    assert torch.equal(out[:64], rows[:64]) and torch.equal(out[128:], rows[128:])
    assert not out[64:128, :256].any() and out[64:128, 256:].isnan().all()


def test_a_captured_step_and_streams():
    """A step (append, then attend) captured and replayed, with the program's own work between the replays, and on another stream."""
    gen = torch.Generator().manual_seed(16)
    heads, width = 16, 8
    rotary = dq.rotary(64)
    cache = dq.alloc_latent_cache(2 * width, dtype=torch.bfloat16)
    table = torch.arange(2 * width, dtype=torch.int32, device=DEV).view(2, width)
    rows, q = torch.zeros(2, 576, dtype=torch.bfloat16, device=DEV), torch.zeros(2, heads, 576, dtype=torch.bfloat16, device=DEV)
    lens, out = torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(2, heads, 512, dtype=torch.bfloat16, device=DEV)
    ws = dq.latent_workspace(cache, 2, 2, heads, 1, 512)

    def step(c, n, ws, out):
        n += 1
        turned = q.clone()
        dq.latent_append(c, rows[:, :512], rows[:, 512:], None, n, table, q=q[..., 512:], q_out=turned[..., 512:], rotary=rotary)
        dq.latent_attention(c, turned, None, n, table, 1, 512, 0.07, ws, out=out)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step(cache, lens, ws, out)
    torch.cuda.current_stream().wait_stream(stream)
    lens.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cache, lens, ws, out)
    eager, eager_lens, eager_out = dq.alloc_latent_cache(2 * width, dtype=torch.bfloat16), torch.zeros_like(lens), torch.zeros_like(out)
    eager_ws = dq.latent_workspace(eager, 2, 2, heads, 1, 512)
    lens.zero_()
    for i in range(130):
        rows.copy_(normal((2, 576), torch.bfloat16, gen))
        q.copy_(normal((2, heads, 576), torch.bfloat16, gen))
        graph.replay()
        step(eager, eager_lens, eager_ws, eager_out)
        if i % 13 == 0:
            torch.cuda.synchronize()
            assert torch.equal(out, eager_out), i
    assert torch.equal(out, eager_out) and lens.tolist() == [130, 130]
