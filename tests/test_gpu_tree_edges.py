"""Drafted trees over the paged 8-bit cache: windows in every build, blocks of zero values, bounds."""
import pytest
import torch

import paper_2405_12591_amd as dq
from latent_util import attend64, check
from paged_util import DEV, HALF, filled_cache, ints
from test_gpu_paged_tree import Trees

pytestmark = pytest.mark.gpu

BF, F16, I8, E4 = torch.bfloat16, torch.float16, torch.int8, torch.float8_e4m3fn


@pytest.mark.parametrize("d,page,dtype,codes", [(128, 64, BF, E4), (64, 128, F16, I8), (128, 128, F16, E4), (64, 64, BF, I8)])
@pytest.mark.parametrize("most", [8, 16, 32])                       # with four query heads a kv head 32, 64 and 128 columns
@pytest.mark.parametrize("window", [64, 130, 1000])
def test_windows_in_every_build(d, page, dtype, codes, most, window):
    """Tiles before the window are left out of a unit's places, which the groups of waves share: lengths around the window, its end in every place of a tile."""
    x = Trees([1700, 63, 0, 64 + window, window + 7, 965], [most, 3, 5, most - 1, 1, most // 2], 8, 2, d, dtype, codes, page, most + window)
    check(x.run(window=window), *x.want(window=window))


@pytest.mark.parametrize("dtype,codes", [(F16, I8), (F16, E4), (BF, E4), (BF, I8)])
@pytest.mark.parametrize("page,most,small", [(64, 4, True), (128, 12, True), (64, 32, False), (128, 30, True)])
def test_blocks_of_zero_values_beside_small_ones(dtype, codes, page, most, small):
    """The scale 1 of a block of zeros takes no bits from blocks of small values, wherever it stands; all values zero yield zeros."""
    lens, counts = [5 * page + 9, 300, 64 * 130 + 5, 4 * page], [most, 2, 3, 5]
    x = Trees(lens, counts, 8, 2, 64, dtype, codes, page, page + most)
    power, gen = (-11 if dtype == F16 else -60) if small else 4, torch.Generator().manual_seed(30)
    for b in range(4):
        x.seqs.v[b] = (x.seqs.v[b].double() * 2.0 ** power).to(dtype)
    x.seqs.v[0][:page] = 0
    x.seqs.k[0][:page] *= 3                                         # its tokens may weigh most
    x.seqs.v[1][page:2 * page, 1] = -0.0
    for p in range(0, lens[2] // page, 3):
        x.seqs.v[2][p * page:(p + 1) * page, p % 2] = 0
    x.seqs.v[3][:] = 0
    x.qkv[:, 10:] = (x.qkv[:, 10:].double() * 2.0 ** power).to(dtype)
    x.qkv[sum(counts[:3]):, 10:] = 0
    x.cache, x.table, x.slots = filled_cache(x.seqs, lens, gen)
    got, (want, tol, own) = x.run(), x.want()
    # values of the size that these have: bf16 has no smallest step here, fp16's results one of 2^-24, half of which the rounding may take
    # (rows of no sequence have to be equal, and have no tolerance to take from)
    check(got, want, tol - own[:, None, None] * (2.0 ** -24 if dtype == BF else 2.0 ** -25), own)
    assert not got[sum(counts[:3]):sum(counts)].any()


@pytest.mark.parametrize("most", [8, 16, 32])
def test_the_bound_on_lengths_is_not_looked_at(most):
    x = Trees([2100, 40, 700], [most, 3, 5], 8, 2, 128, BF, E4, 64, most)
    assert len({dq.paged_tree_workspace(x.cache, 3, len(x.qkv), 8, most, n).numel() for n in (0, 700, 2100, 1 << 30)}) == 1
    first = x.run()
    for n in (0, 1, 64, 700, 1 << 30):
        assert torch.equal(x.run(max_len=n), first), n


def test_layers_that_share_a_workspace():
    gen = torch.Generator().manual_seed(41)
    first = dq.PagedKVLayer(2, 4, 2, 64, 300, dtype=BF)
    layers = [first, dq.PagedKVLayer(2, 4, 2, 64, 300, dtype=BF, workspace_of=first), dq.PagedKVLayer(2, 4, 2, 64, 300, dtype=BF)]
    for most in (3, 30):                                            # the second call outgrows the first one's
        q, k, v = (torch.randn((2 * most, n, 64), generator=gen).to(BF).to(DEV) for n in (4, 2, 2))
        starts, seen = ints([0, most, 2 * most]), torch.tensor([(1 << i + 1) - 1 for i in range(most)] * 2, device=DEV)
        outs = []
        for layer in layers:
            layer.append(k, v, starts, most)
            outs.append(layer.attend_tree(q, k, v, seen, starts, most))
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
        ws = [layer._tree_ws.ws.data_ptr() for layer in layers]
        assert ws[0] == ws[1] != ws[2]
