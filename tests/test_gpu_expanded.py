"""Attention over expanded keys and values (ragged prompts) against the definition in 64 bits."""
import pytest
import torch

import paper_2405_12591_amd as dq
from latent_util import attend64, check, normal, starts_of, tolerance
from paged_util import DEV, ints

pytestmark = pytest.mark.gpu


class Prompt:
    """Sequences' rows and tokens, `gap` of each that belong to none ahead of them; what lies around is NaN."""

    def __init__(self, counts, lens, heads, d, dtype, gen, gap=0):
        self.counts, self.lens, self.heads, self.d, self.dtype, self.gap = counts, lens, heads, d, dtype, gap
        rows, tokens = sum(counts) + gap + 3, sum(lens) + gap + 3
        self.q = normal((rows, heads, d + d // 2), dtype, gen)
        self.kv = normal((tokens, heads, 2 * d + 8), dtype, gen)
        self.kv[..., 3:d:37] *= 8
        self.kr = normal((tokens, 4 * d + d // 2), dtype, gen)
        if gap:
            self.kv[:gap] = self.kv[-3:] = self.kr[:gap] = self.kr[-3:] = float("nan")
        self.starts, self.kv_starts = starts_of(counts, gap), starts_of(lens, gap)

    def run(self, causal=True, max_rows=None, max_len=None, scale=0.0, ws=None):
        d, max_rows, max_len = self.d, max(self.counts) if max_rows is None else max_rows, max(self.lens) if max_len is None else max_len
        if ws is None:
            ws = dq.expanded_workspace(len(self.lens), self.q.shape[0], self.heads, d, max_rows, max_len)
            ws.fill_(255)
        kv, out = self.kv.to(DEV), torch.full((self.q.shape[0], self.heads, d), 7.0, dtype=self.dtype, device=DEV)
        dq.expanded_attention(self.q.to(DEV), kv[..., :d], self.kr.to(DEV)[:, 4 * d:], kv[..., d:2 * d], ints(self.starts), ints(self.kv_starts), max_rows,
                              max_len, ws, out=out, causal=causal, softmax_scale=scale)
        return out

    def want(self, causal=True, scale=None):
        d = self.d
        scale = (1.5 * d) ** -0.5 if scale is None else scale
        out = torch.full((self.q.shape[0], self.heads, d), 7.0, dtype=torch.float64)
        tol, own = torch.zeros_like(out), torch.zeros(len(out), dtype=torch.bool)
        for b, (c, n) in enumerate(zip(self.counts, self.lens)):
            r, t = slice(self.starts[b], self.starts[b + 1]), slice(self.kv_starts[b], self.kv_starts[b + 1])
            k = torch.cat([self.kv[t, :, :d], self.kr[t, None, 4 * d:].expand(-1, self.heads, -1)], 2)
            place, j = n - c + torch.arange(c), torch.arange(n)
            see = j[None] <= place[:, None] if causal else torch.ones(c, n, dtype=torch.bool)
            o, size, ds = attend64(self.q[r], k, self.kv[t, :, d:2 * d], see, scale)
            v_max = float(self.kv[t, :, d:2 * d].double().abs().nan_to_num(0, 0, 0).max()) if n else 0.0
            out[r], tol[r], own[r] = o, tolerance(o, size, ds, v_max, n, self.dtype), True
        return out, tol, own


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("counts,lens,heads,gap", [
    ([1, 63, 64, 65, 129], [1, 63, 64, 65, 129], 3, 2),             # whole prompts around the tiles
    ([5, 0, 130, 1], [400, 20, 131, 1], 2, 1),                      # behind earlier tokens; no rows
    ([4, 3], [2, 0], 5, 3),                                         # more rows than tokens: the first ones see nothing
    ([300], [900], 1, 0),                                           # splits
])
def test_attention(dtype, d, counts, lens, heads, gap):
    x = Prompt(counts, lens, heads, d, dtype, torch.Generator().manual_seed(d + heads), gap)
    for causal in (True, False):
        check(x.run(causal), *x.want(causal), "causal %s" % causal)


def test_bounds_choose_the_launch_only():
    x = Prompt([40, 200, 7], [700, 200, 350], 4, 64, torch.bfloat16, torch.Generator().manual_seed(1))
    want = x.want(scale=0.2)
    for max_rows, max_len in ((200, 1), (200, 20000), (5000, 700), (200, 700)):
        check(x.run(scale=0.2, max_rows=max_rows, max_len=max_len), *want, "%d %d" % (max_rows, max_len))


def test_one_workspace_serves_smaller_calls_and_needs_no_zeros():
    big = Prompt([300, 260], [1500, 900], 4, 128, torch.float16, torch.Generator().manual_seed(2))
    ws = dq.expanded_workspace(2, big.q.shape[0], 4, 128, 300, 1500)
    ws.fill_(255)
    for x in (big, Prompt([9], [1500], 4, 128, torch.float16, torch.Generator().manual_seed(3)), Prompt([130, 3], [200, 1400], 4, 128, torch.bfloat16, torch.Generator().manual_seed(4))):
        check(x.run(ws=ws), *x.want())


def test_rows_past_the_bound_are_left_and_the_others_are_not():
    x = Prompt([140, 30, 128], [140, 60, 128], 2, 64, torch.float16, torch.Generator().manual_seed(5))
    want, tol, _ = x.want()
    got = x.run(max_rows=128).double().cpu()
    fine = (got - want).abs() <= tol
    assert bool(fine[:128].all()) and bool(fine[140:298].all()) and bool((got[128:140] == 7).all())


@pytest.mark.parametrize("d", [128, 64])
def test_not_finite_tokens_do_nothing_to_rows_that_do_not_see_them(d):
    x = Prompt([200, 70], [200, 140], 2, d, torch.float16, torch.Generator().manual_seed(6))
    clean = x.kv.clone()
    for token, channel, value in ((90, d + 5, float("inf")), (197, 3, float("nan")), (199, 2 * d - 1, float("-inf")), (200 + 130, d, float("nan"))):
        x.kv[token, 1, channel] = value
    got = x.run().double().cpu()
    x.kv = clean
    want, tol, _ = x.want()
    fine = (got - want).abs() <= tol
    hit = torch.zeros(len(got), dtype=torch.bool)
    hit[90:200] = True
    hit[200 + 60:270] = True
    assert bool(fine[:, 0].all()) and bool(fine[~hit].all())
    assert not bool(got[hit, 1].isfinite().all(1).any())


def test_strides_that_pass_32_bits():
    """Tokens so far apart that the largest offset takes 34 bits."""
    d, heads, n, stride = 64, 1, 5, 1 << 31
    gen = torch.Generator().manual_seed(7)
    try:
        far = torch.zeros((n - 1) * stride + 256, dtype=torch.float16, device=DEV)
    except torch.cuda.OutOfMemoryError:
        pytest.skip("no room")
    x = Prompt([n], [n], heads, d, torch.float16, gen)
    k, kr, v = (torch.as_strided(far, (n, w), (stride, 1), at) for w, at in ((d, 0), (d // 2, 64), (d, 128)))
    k.copy_(x.kv[:n, 0, :d])
    kr.copy_(x.kr[:n, 4 * d:])
    v.copy_(x.kv[:n, 0, d:2 * d])
    out = torch.full((x.q.shape[0], 1, d), 7.0, dtype=torch.float16, device=DEV)
    dq.expanded_attention(x.q.to(DEV), k[:, None], kr, v[:, None], ints([0, n]), ints([0, n]), n, n, dq.expanded_workspace(1, n, 1, d, n, n), out=out)
    check(out, *x.want())


def test_a_captured_call():
    x = Prompt([33, 150], [600, 150], 4, 128, torch.bfloat16, torch.Generator().manual_seed(8))
    d = 128
    q, kv, kr = x.q.to(DEV), x.kv.to(DEV), x.kr.to(DEV)
    out, ws = torch.zeros((x.q.shape[0], 4, d), dtype=x.dtype, device=DEV), dq.expanded_workspace(2, x.q.shape[0], 4, d, 150, 600)
    starts, kv_starts = ints(x.starts), ints(x.kv_starts)

    def call(out, ws):
        dq.expanded_attention(q, kv[..., :d], kr[:, 4 * d:], kv[..., d:2 * d], starts, kv_starts, 150, 600, ws, out=out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, ws)
    other, other_ws = torch.zeros_like(out), torch.zeros_like(ws)
    for i in range(5):
        q.copy_(normal(x.q.shape, x.dtype, torch.Generator().manual_seed(i)))
        out.zero_()
        graph.replay()
        call(other, other_ws)
        torch.cuda.synchronize()
        assert torch.equal(out, other)
