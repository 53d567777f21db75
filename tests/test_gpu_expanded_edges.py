"""Attention over expanded keys and values at the edges of its calls."""
import pytest
import torch

import paper_2405_12591_amd as dq
from latent_util import attend64, check, tolerance
from paged_util import DEV, ints
from test_gpu_expanded import Prompt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [128, 64])
def test_rows_without_a_token_in_the_batch_are_zeros(d):
    q, kv, kr = (torch.ones(shape, dtype=torch.bfloat16, device=DEV) for shape in ((5, 3, d + d // 2), (0, 3, 2 * d), (0, d // 2)))
    for causal in (True, False):
        out = torch.full((5, 3, d), 7.0, dtype=torch.bfloat16, device=DEV)
        dq.expanded_attention(q, kv[..., :d], kr, kv[..., d:], ints([1, 3, 4]), ints([0, 0, 0]), 2, 0, dq.expanded_workspace(2, 5, 3, d, 2, 0), out=out, causal=causal)
        assert not out[1:4].any() and bool((out[[0, 4]] == 7).all())


@pytest.mark.parametrize("where", ["k", "k_rot"])
@pytest.mark.parametrize("value", [float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype,d", [(torch.float16, 128), (torch.bfloat16, 64)])
def test_an_infinite_key_counts_by_its_scores(dtype, d, value, where):
    """A score of +inf makes a row NaN, one of -inf is a weight of 0, in tiles with a mask (the first rows') and without one."""
    x = Prompt([200], [200], 2, d, dtype, torch.Generator().manual_seed(20))
    channel = 5 if where == "k" else d + 9
    q_sign = x.q[:200, :, channel].double().sign()
    token, n, scale = 20, 200, (1.5 * d) ** -0.5
    heads = [1] if where == "k" else [0, 1]
    clean = (x.kv.clone(), x.kr.clone())
    if where == "k":
        x.kv[token, 1, 5] = value
    else:
        x.kr[token, 4 * d + 9] = value
    got = x.run().double().cpu()[:200]
    x.kv, x.kr = clean
    k = torch.cat([x.kv[:n, :, :d], x.kr[:n, None, 4 * d:].expand(-1, 2, -1)], 2)
    see = torch.arange(n)[None] <= torch.arange(n)[:, None]
    less = see.clone()
    less[:, token] = False
    for h in range(2):
        hit = (torch.arange(n) >= token) & (q_sign[:, h] * value > 0) if h in heads else torch.zeros(n, dtype=torch.bool)
        assert h not in heads or 20 < int(hit.sum()) < 160
        o, size, ds = attend64(x.q[:n, h:h + 1], k[:, h], x.kv[:n, h, d:2 * d], less if h in heads else see, scale)
        v_max = float(x.kv[:n, h, d:2 * d].double().abs().max())
        assert bool(got[hit, h].isnan().all())
        assert bool(((got[:, h:h + 1] - o).abs() <= tolerance(o, size, ds, v_max, n, dtype))[~hit].all())


def test_scores_that_are_all_minus_infinity_are_no_weight():
    q, k, v = (torch.ones(shape, dtype=torch.float16, device=DEV) for shape in ((3, 1, 96), (3, 1, 64), (3, 1, 64)))
    k[0, 0, 3] = -float("inf")
    out = dq.expanded_attention(q, k, torch.ones(3, 32, dtype=torch.float16, device=DEV), v, ints([0, 3]), ints([0, 3]), 3, 3, dq.expanded_workspace(1, 3, 1, 64, 3, 3))
    assert not out[0].any() and bool((out[1:] == 1).all())


@pytest.mark.parametrize("far", ["k", "k_rot", "v"])
def test_whole_tiles_of_strides_that_pass_32_bits(far):
    """64 tokens are a whole tile, whose rows are found by 32-bit offsets where those do: 15 rows of 9 * 2^24 elements are 2^32 bytes and 5 * 2^28 more."""
    d, n, stride, gen = 64, 64, 9 << 24, torch.Generator().manual_seed(21)
    assert 15 * stride * 2 > 1 << 32
    try:
        room = torch.zeros((n - 1) * stride + 64, dtype=torch.float16, device=DEV)
    except torch.cuda.OutOfMemoryError:
        pytest.skip("no room")
    x = Prompt([n], [n], 1, d, torch.float16, gen)
    near = {"k": x.kv[:n, 0, :d], "k_rot": x.kr[:n, 4 * d:], "v": x.kv[:n, 0, d:2 * d]}
    t = {name: (torch.as_strided(room, rows.shape, (stride, 1)).copy_(rows) if name == far else rows.contiguous().to(DEV)) for name, rows in near.items()}
    out = torch.full((x.q.shape[0], 1, d), 7.0, dtype=torch.float16, device=DEV)
    dq.expanded_attention(x.q.to(DEV), t["k"][:, None], t["k_rot"], t["v"][:, None], ints([0, n]), ints([0, n]), n, n, dq.expanded_workspace(1, n, 1, d, n, n), out=out)
    check(out, *x.want())
