"""The cache of latents at the edges of its calls: one row, rows that are not finite in any channel."""
import pytest
import torch

import paper_2405_12591_amd as dq
from latent_util import FORMS, Latents, attend64, check, normal, starts_of, tolerance
from paged_util import DEV, ints

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16]


@pytest.mark.parametrize("latent", [512, 256])
def test_one_row_is_read(latent):
    x = Latents([130, 70], latent, torch.float16, 64, torch.Generator().manual_seed(0))
    w = latent + FORMS[latent]
    wide = torch.full((3, w + 8), 7.0, dtype=torch.float16, device=DEV)
    for first, want in (([129, 70], x.rows[0][129]), ([130, 69], x.rows[1][69])):
        for out in (torch.full((1, w), 7.0, dtype=torch.float16, device=DEV), wide[1:2, :w]):
            at = [0, 1, 1] if first[0] == 129 else [0, 0, 1]
            dq.latent_read(x.cache, ints(first), ints([130, 70]), ints(at), x.table.to(DEV), out)
            assert torch.equal(out[0].cpu(), want)
    assert bool((wide[0] == 7).all()) and bool((wide[2] == 7).all()) and bool((wide[1, w:] == 7).all())


def test_a_layer_reads_one_row():
    gen = torch.Generator().manual_seed(1)
    rows = normal((2, 576), torch.bfloat16, gen).to(DEV)
    layer = dq.LatentKVLayer(2, 16, 100)
    layer.append(rows[:, :512], rows[:, 512:])
    for lengths, want in (([1, 0], rows[:1]), ([0, 1], rows[1:]), ([1, 1], rows), ([0, 0], rows[:0])):
        got, starts = layer.read(lengths)
        assert torch.equal(got, want) and starts.tolist() == starts_of(lengths)


@pytest.mark.parametrize("what", ["inf", "-inf", "nan", "turned", "overflow"])
@pytest.mark.parametrize("heads", [1, 3, 6, 13])                    # 16, 32, 64 and 128 columns
@pytest.mark.parametrize("dtype,latent", [(torch.bfloat16, 512), (torch.float16, 512), (torch.float16, 256), (torch.bfloat16, 256)])
def test_key_channels_that_are_not_finite_are_nan_for_those_who_see_them_only(dtype, latent, heads, what):
    """Whether they came so or rotation took them out of the type's range, and whichever sign the scores would have."""
    gen = torch.Generator().manual_seed(2)
    lens, counts, rot = [70, 64], [10, 4], FORMS[latent]
    x = Latents(lens, latent, dtype, 64, gen)
    new = torch.cat([x.rows[0][60:], x.rows[1][60:]])
    rotary = dq.rotary(rot) if what in ("turned", "overflow") else None
    for row in (5, 11):
        if what == "overflow":                                      # both of a pair, turned by one radian: 1.38 times as large
            new[row, latent] = new[row, latent + rot // 2] = torch.finfo(dtype).max * 0.9
        else:
            new[row, latent + 7] = float("inf" if what == "turned" else what)
    new = new.to(DEV)
    dq.latent_append(x.cache, new[:, :latent], new[:, latent:], ints(starts_of(counts)), ints(lens), x.table.to(DEV), rotary=rotary,
                     positions=None if rotary is None else ints([1] * 14))
    read = torch.zeros((14, latent + rot), dtype=dtype, device=DEV)
    dq.latent_read(x.cache, ints([60, 60]), ints(lens), ints(starts_of(counts)), x.table.to(DEV), read)
    others = [i for i in range(14) if i not in (5, 11)]
    assert torch.equal(read[:, :latent], new[:, :latent]) and bool(read[others].isfinite().all())
    assert bool(read[[5, 11], latent:].isnan().all())
    read = read.cpu()
    read[[5, 11]] = 1.0
    x.rows[0][60:], x.rows[1][60:] = read[:10], read[10:]
    q = normal((14, heads, latent + rot), dtype, gen)
    got = x.attend(q.to(DEV), counts, 0.07)
    want, tol, _ = x.want(q, counts, 0.07)
    see = [i for i in range(14) if (i < 10 and i >= 5) or i >= 11]
    rest = [i for i in range(14) if i not in see]
    assert got[see].isnan().all()
    assert bool(((got.double().cpu() - want).abs() <= tol)[rest].all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("latent,page", [(512, 64), (512, 128), (256, 64), (256, 128)])
@pytest.mark.parametrize("heads,counts", [(1, [16, 3, 9]), (2, [8, 8, 1]), (3, [5, 4, 5]), (4, [4, 0, 3]), (16, [1, 1, 1])])
def test_masks_of_up_to_16_columns(dtype, latent, page, heads, counts):
    """The kernel that takes them, whose waves each form a tile's mask from bits that begin anywhere in it."""
    gen = torch.Generator().manual_seed(heads + page)
    x = Latents([165, 33, 64 + 9], latent, dtype, page, gen)
    q = normal((sum(counts) + 2, heads, latent + FORMS[latent]), dtype, gen)
    seen = torch.randint(-1 << 62, 1 << 62, (sum(counts) + 2,), generator=gen, dtype=torch.int64)   # any rows, and bits of rows that are not there
    seen[0], seen[sum(counts) - 1] = 0, -1
    check(x.attend(q.to(DEV), counts, 0.07, seen=seen), *x.want(q, counts, 0.07, seen=seen))


@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("heads", [3, 6, 12, 30])                   # of four rows: 16, 32, 64 and 128 columns
def test_the_bound_on_lengths_is_not_looked_at(latent, heads):
    gen = torch.Generator().manual_seed(heads)
    x = Latents([2100, 40, 700], latent, torch.bfloat16, 64, gen)
    q = normal((9, heads, latent + FORMS[latent]), torch.bfloat16, gen).to(DEV)
    assert len({dq.latent_workspace(x.cache, 3, 9, heads, 4, n).numel() for n in (0, 700, 2100, 1 << 30)}) == 1
    first = x.attend(q, [4, 3, 2], 0.07)
    for n in (0, 1, 64, 700, 1 << 30):
        assert torch.equal(x.attend(q, [4, 3, 2], 0.07, max_len=n), first), n


@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("heads", [16, 32, 64, 128])
def test_sums_over_a_million_tokens(latent, heads):
    """2^20 tokens over 32 pages that the table names again and again: what 2^11 tokens give."""
    gen = torch.Generator().manual_seed(heads)
    x = Latents([2048], latent, torch.float16, 64, gen)
    table = x.table[:, :32].repeat(1, 512)
    x.lens = [1 << 20]
    q = normal((1, heads, latent + FORMS[latent]), torch.float16, gen)
    got = x.attend(q.to(DEV), [1], 0.05, table=table).double().cpu()
    o, size, ds = attend64(q, x.rows[0], x.rows[0][:, :latent], torch.ones(1, 2048, dtype=torch.bool), 0.05)
    # on top of what 2^11 tokens may be off by: a workgroup has 128 tiles of 32 tokens (2^20 / 32 / 256), two matrix instructions each to a result, of
    # four roundings each, 2^10 2^-24 of the terms' sizes, and eight instructions of two roundings each to a sum of probabilities, 2^11 2^-24.  (f16's smallest
    # step counts 512 times as often against a sum that is 512 times as large.)
    v_max = float(x.rows[0][:, :latent].double().abs().max())
    tol = tolerance(o, size, ds, v_max, 2048, torch.float16) + size * 3 * 2.0 ** -14
    assert bool(((got - o).abs() <= tol).all())


def test_layers_that_share_a_workspace():
    """A model's layers one after the other, eagerly and in a captured step, while a larger call of one outgrows what they share: as layers with
    workspaces of their own."""
    gen = torch.Generator().manual_seed(40)
    heads, n = 16, 3
    first = dq.LatentKVLayer(2, heads, 300)
    shared, alone = [first] + [dq.LatentKVLayer(2, heads, 300, workspace_of=first) for _ in range(n - 1)], [dq.LatentKVLayer(2, heads, 300) for _ in range(n)]
    rows, q = normal((n, 2, 576), torch.bfloat16, gen).to(DEV), normal((n, 2, heads, 576), torch.bfloat16, gen).to(DEV)
    out, want = (torch.zeros((n, 2, heads, 512), dtype=torch.bfloat16, device=DEV) for _ in range(2))

    def step(layers, out):
        for i, layer in enumerate(layers):
            layer.append(rows[i, :, :512], rows[i, :, 512:])
            layer.attend(q[i], 0.07, out=out[i])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(shared, out)
    torch.cuda.current_stream().wait_stream(side)
    step(alone, want)
    assert torch.equal(out, want) and len({layer._ws.ws.data_ptr() for layer in shared}) == 1
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(shared, out)
    for layer in shared:
        layer.tokens_upper -= 1                                     # (the capture itself appended nothing)
    big, big_q, starts = normal((80, 576), torch.bfloat16, gen).to(DEV), normal((80, heads, 576), torch.bfloat16, gen).to(DEV), ints([0, 40, 80])
    for layers in (shared, alone):
        layers[1].append(big[:, :512], big[:, 512:], starts, 40)
    assert torch.equal(shared[1].attend(big_q, 0.07, starts, 40), alone[1].attend(big_q, 0.07, starts, 40))
    for i in range(4):
        rows.copy_(normal(rows.shape, torch.bfloat16, gen))
        graph.replay()
        step(alone, want)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        for layer in shared:
            layer.tokens_upper += 1
    step(shared, out)
    step(alone, want)
    assert torch.equal(out, want)
    with pytest.raises(dq.DQError, match="workspace_of"):
        dq.LatentKVLayer(2, heads, 300, workspace_of=dq.PagedKVLayer(1, 4, 4, 64, 100))
