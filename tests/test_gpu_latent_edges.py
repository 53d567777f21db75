"""The cache of latents at the edges of its calls: one row, rows that are not finite in any channel."""
import pytest
import torch

import paper_2405_12591_amd as dq
from latent_util import FORMS, Latents, normal, starts_of
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
    assert torch.equal(read[others, :latent], new[others, :latent]) and bool(read[others].isfinite().all())
    assert not read[[5, 11], :latent].any() and bool(read[[5, 11], latent:].isnan().all())
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
