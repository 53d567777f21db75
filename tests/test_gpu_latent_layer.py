"""A layer's run over latents and over a paged cache with drafted trees, as a serving loop makes it, against plain forms in 64 bits."""
import pytest
import torch

import paper_2405_12591_amd as dq
from latent_util import attend64, normal, starts_of, tolerance
from paged_util import DEV, HALF, Sequences, ints

pytestmark = pytest.mark.gpu


def _close(got, want, tol):
    assert bool(((got.double().cpu() - want).abs() <= tol).all())


def test_prompt_expanded_then_drafted_tree_then_single_tokens():
    """Prompts in the expanded form, a piece behind them over rows read back, a tree of drafted rows in the absorbed form, its path kept, one token
    more."""
    gen = torch.Generator().manual_seed(0)
    dtype, heads, d, R, r = torch.float16, 4, 64, 256, 32
    layer = dq.LatentKVLayer(2, heads, 400, R, r, dtype=dtype)
    rotary, weight = dq.rotary(r), (1 + 0.1 * torch.randn(R, generator=gen)).to(dtype).to(DEV)
    up = (torch.randn(R, heads * 2 * d, generator=gen) / 16).to(dtype).to(DEV)
    scale, kept = (d + r) ** -0.5, [[], []]

    def rows(counts):
        n = sum(counts)
        return normal((n, R + r), dtype, gen).to(DEV), normal((n, heads, d + r), dtype, gen).to(DEV)

    def append(counts, places=None):
        x, q = rows(counts)
        starts = ints(starts_of(counts))
        layer.append(x[:, :R], x[:, R:], starts, max(counts), q=q[..., d:], q_out=q[..., d:], rotary=rotary, weight=weight,
                     positions=None if places is None else ints(places))
        return x, q, starts

    for counts, lens in (([150, 37], [150, 37]), ([20, 65], [170, 102])):          # prompts; pieces behind them
        x, q, starts = append(counts)
        c, kv_starts = layer.read(lens)
        kv = (c[:, :R] @ up).view(-1, heads, 2 * d)
        ws = dq.expanded_workspace(2, len(q), heads, d, max(counts), max(lens))
        out = dq.expanded_attention(q, kv[..., :d], c[:, R:], kv[..., d:], starts, kv_starts, max(counts), max(lens), ws)
        c, kv = c.cpu(), kv.cpu()
        for b in range(2):
            t, own = slice(sum(lens[:b]), sum(lens[:b + 1])), slice(sum(counts[:b]), sum(counts[:b + 1]))
            k = torch.cat([kv[t, :, :d], c[t, None, R:].expand(-1, heads, -1)], 2)
            see = torch.arange(lens[b])[None] <= (lens[b] - counts[b] + torch.arange(counts[b]))[:, None]
            o, size, ds = attend64(q[own].cpu(), k, kv[t, :, d:], see, scale)
            _close(out[own], o, tolerance(o, size, ds, float(kv[t, :, d:].double().abs().max()), lens[b], dtype))

    # a tree: rows 0; 1, 2 behind 0; 3 behind 2, for both sequences; places by depth
    base, counts, depth, masks, path = [170, 102], [4, 4], [0, 1, 1, 2], [1, 3, 5, 13], [0, 2, 3]
    x, _, starts = append(counts, [n + i for n in base for i in depth])
    q = normal((8, heads, R + r), dtype, gen).to(DEV)
    out = layer.attend(q, scale, starts, 4, seen=torch.tensor(masks * 2, device=DEV))
    c, _ = layer.read([174, 106])
    c = c.cpu()
    for b in range(2):
        t = slice(0, 174) if b == 0 else slice(174, 280)
        see = torch.ones(4, base[b] + 4, dtype=torch.bool)
        for i in range(4):
            see[i, base[b]:] = torch.tensor([bool(masks[i] >> j & 1) for j in range(4)])
        o, size, ds = attend64(q[4 * b:4 * b + 4].cpu(), c[t], c[t, :R], see, scale)
        _close(out[4 * b:4 * b + 4], o, tolerance(o, size, ds, float(c[t, :R].double().abs().max()), base[b] + 4, dtype))
    # the path is kept: the same rows again behind the shortened lengths, at the same places
    layer.shorten(base)
    keep = torch.tensor([4 * b + i for b in range(2) for i in path], device=DEV)
    layer.append(x[keep, :R], x[keep, R:], ints([0, 3, 6]), 3, rotary=rotary, weight=weight)
    again, _ = layer.read([173, 105])
    again = again.cpu()
    assert torch.equal(again[170:173], c[[170 + i for i in path]]) and torch.equal(again[173 + 102:], c[[174 + 102 + i for i in path]])
    x, _ = rows([1, 1])
    layer.append(x[:, :R], x[:, R:], rotary=rotary, weight=weight)
    q = normal((2, heads, R + r), dtype, gen).to(DEV)
    out = layer.attend(q, scale)
    c, _ = layer.read([174, 106])
    c = c.cpu()
    for b, t in enumerate((slice(0, 174), slice(174, 280))):
        o, size, ds = attend64(q[b:b + 1].cpu(), c[t], c[t, :R], torch.ones(1, t.stop - t.start, dtype=torch.bool), scale)
        _close(out[b:b + 1], o, tolerance(o, size, ds, float(c[t, :R].double().abs().max()), 174, dtype))
    with pytest.raises(dq.DQError, match="exceed"):
        layer.append(x[:1, :R].expand(400, R), x[:1, R:].expand(400, r), ints([0, 400, 400]), 400)
    assert layer.seq_lens.tolist() == [174, 106]


def test_a_paged_layer_checks_a_tree_and_keeps_its_path():
    gen = torch.Generator().manual_seed(1)
    dtype, hq, h, d = torch.bfloat16, 4, 2, 64
    layer = dq.PagedKVLayer(2, hq, h, d, 300, dtype=dtype, codes=torch.float8_e4m3fn)
    lens, masks = [130, 64], [1, 3, 5, 13, 1 << 4]
    seqs = Sequences(lens, h, d, dtype, torch.float8_e4m3fn, 64, gen)
    layer.append(torch.cat(seqs.k).to(DEV), torch.cat(seqs.v).to(DEV), ints([0, 130, 194]), 130)
    q, k, v = (normal((10, n, d), dtype, gen) for n in (hq, h, h))
    out = layer.attend_tree(q.to(DEV), k.to(DEV), v.to(DEV), torch.tensor(masks * 2, device=DEV), ints([0, 5, 10]), 5)
    for b, n in enumerate(lens):
        own = slice(5 * b, 5 * b + 5)
        kk = torch.cat([seqs.stored(seqs.k[b]), k[own].double()]).repeat_interleave(2, 1)
        vv = torch.cat([seqs.stored(seqs.v[b]), v[own].double()]).repeat_interleave(2, 1)
        see = torch.ones(5, n + 5, dtype=torch.bool)
        see[:, n:] = torch.tensor([[bool(m >> j & 1) for j in range(5)] for m in masks])
        o, size, ds = attend64(q[own], kk, vv, see, d ** -0.5)
        _close(out[own], o, o.abs() * HALF[dtype] + size * (HALF[dtype] + 2.0 ** -18 + 2.0 ** -17 * ds) + 2.0 ** -20)
    assert layer.seq_lens.tolist() == lens                          # nothing was appended
    path = torch.tensor([0, 2, 3, 5, 7, 8])
    layer.append(k[path].to(DEV), v[path].to(DEV), ints([0, 3, 6]), 3)
    rk, rv = layer.read([133, 67])
    assert torch.equal(rk[0, :, 130:133].transpose(0, 1).cpu(), k[path[:3]]) and torch.equal(rv[1, :, 64:67].transpose(0, 1).cpu(), v[path[3:]])


def test_a_layers_captured_step_keeps_its_workspace():
    """A step captured in a graph goes on working while larger calls outgrow the layer's workspace."""
    gen = torch.Generator().manual_seed(2)
    layer = dq.LatentKVLayer(2, 16, 300)
    rotary = dq.rotary(64)
    x, q = normal((2, 576), torch.bfloat16, gen).to(DEV), normal((2, 16, 576), torch.bfloat16, gen).to(DEV)
    out = torch.zeros((2, 16, 512), dtype=torch.bfloat16, device=DEV)

    def step():
        layer.append(x[:, :512], x[:, 512:], rotary=rotary)
        layer.attend(q, 0.07, out=out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    layer.tokens_upper -= 1                                         # (the capture itself appended nothing)
    big = normal((80, 576), torch.bfloat16, gen).to(DEV)
    layer.append(big[:, :512], big[:, 512:], ints([0, 40, 80]), 40, rotary=rotary)
    layer.attend(normal((80, 16, 576), torch.bfloat16, gen).to(DEV), 0.07, ints([0, 40, 80]), 40)
    for _ in range(4):
        graph.replay()
        layer.tokens_upper += 1
        want = layer.attend(q, 0.07)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    assert layer.seq_lens.tolist() == [45, 45]
