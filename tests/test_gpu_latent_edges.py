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
