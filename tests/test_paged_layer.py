"""What a program keeps between calls: rotations, layers, the compiled part of the binding.  Most of it on the CPU."""
import copy
import io
import pickle

import pytest
import torch

DEV = "cuda:0"


def _lib():
    import paper_2405_12591_amd as dq
    from paper_2405_12591_amd import paged
    return dq, paged


def _copies(r):
    """Copies by every way a model takes."""
    buf = io.BytesIO()
    torch.save(r, buf)
    buf.seek(0)
    return {"copy": copy.copy(r), "deepcopy": copy.deepcopy(r), "pickle": pickle.loads(pickle.dumps(r)), "torch": torch.load(buf, weights_only=False),
            "of a copy": copy.deepcopy(pickle.loads(pickle.dumps(r)))}


@pytest.mark.parametrize("sections", [None, (8, 12, 12)])
def test_a_copied_rotation_hands_over_its_own_tensors(sections):
    dq, paged = _lib()
    r = dq.rotary(64, sections=sections, interleaved=True, device="cpu")
    for how, c in _copies(r).items():
        assert c is not r and torch.equal(c.inv_freq, r.inv_freq) and c.axes == r.axes and c.interleaved and c.rot_dim == 64, how
        freq, axis, axes, interleaved = c._c
        assert freq is c.inv_freq and axis is c.axis_of_pair and axes == c.axes and interleaved is True, how


@pytest.mark.gpu
@pytest.mark.parametrize("sections", [None, (8, 12, 12)])
def test_a_copied_rotation_turns_by_its_own_frequencies(sections):
    """The copy's tensors, also after they changed in place or the original's memory holds something else."""
    dq, _ = _lib()
    gen = torch.Generator().manual_seed(1)
    x = torch.randn((20, 3, 64), generator=gen).half().to(DEV)
    pos = torch.randint(0, 5000, (1 if sections is None else 3, 20), generator=gen).to(torch.int32).to(DEV)
    r = dq.rotary(64, sections=sections, device=DEV)
    want, _ = dq.rotate_heads(x, None, pos, r)
    copies = {n: c for n, c in _copies(r).items() if n != "copy"}
    r.inv_freq.fill_(0.25)                               # (the original's)
    if sections is not None:
        r.axis_of_pair.zero_()
    for how, c in copies.items():
        got, _ = dq.rotate_heads(x, None, pos, c)
        assert torch.equal(got, want), how
        k = dq.alloc_paged_cache(2, 1, 3, 64, device=DEV)
        got = dq.paged_append(k, x, x, torch.tensor([0, 20], dtype=torch.int32, device=DEV), torch.tensor([20], dtype=torch.int32, device=DEV),
                              torch.zeros((1, 1), dtype=torch.int32, device=DEV), q=x, rotary=c, positions=pos)
        assert torch.equal(got, want), how


@pytest.mark.gpu
def test_a_rotation_whose_tensors_were_exchanged_is_looked_at_again():
    dq, _ = _lib()
    x = torch.zeros((2, 1, 64), dtype=torch.float16, device=DEV)
    pos = torch.zeros(2, dtype=torch.int32, device=DEV)
    for bad in (torch.zeros(32, device=DEV), torch.zeros(32, dtype=torch.float64), torch.zeros(64, dtype=torch.float64, device=DEV),
                torch.zeros(64, dtype=torch.float64, device=DEV)[::2], torch.zeros(4, dtype=torch.float64, device=DEV)):
        r = dq.rotary(64, device=DEV)
        r.inv_freq.data = bad if bad.is_cuda else r.inv_freq.data
        if not bad.is_cuda:
            object.__setattr__(r, "inv_freq", bad)
        with pytest.raises(dq.DQError):
            dq.rotate_heads(x, None, pos, r)
    r = dq.rotary(64, sections=(16, 16), device=DEV)
    object.__setattr__(r, "axis_of_pair", r.axis_of_pair[:8])
    with pytest.raises(dq.DQError):
        dq.rotate_heads(x, None, torch.zeros(4, dtype=torch.int32, device=DEV), r)


class _CacheOnTheHost:
    """A layer whose cache is never reached."""
    kv_heads, head_dim, page_tokens, dtype, device, index = 2, 64, 64, torch.float16, torch.device("cpu"), 0


def _host_layer(paged, max_tokens=100):
    layer = object.__new__(paged.PagedKVLayer)
    layer.batch, layer.q_heads, layer.max_tokens, layer.cache = 2, 4, max_tokens, _CacheOnTheHost()
    layer.page_table = torch.arange(4, dtype=torch.int32).view(2, 2)
    layer.seq_lens, layer.tokens_upper = torch.tensor([7, 3], dtype=torch.int32), 7
    layer._ws, layer._outgrown = None, []
    return layer


@pytest.mark.parametrize("error", [TypeError("eps"), MemoryError(), torch.OutOfMemoryError("no memory"), OverflowError(), RuntimeError("x"), AttributeError("x")])
def test_lengths_stay_where_they_were_after_any_error(monkeypatch, error):
    dq, paged = _lib()
    layer = _host_layer(paged)

    def fails(*a, **k):
        raise error

    monkeypatch.setattr(paged, "paged_append", fails)
    rows = torch.zeros((5, 2, 64), dtype=torch.float16)
    for starts, n in ((None, 1), (torch.tensor([0, 4, 5], dtype=torch.int32), 4)):
        with pytest.raises(type(error)):
            layer.append(rows, rows, starts, n)
        assert layer.seq_lens.tolist() == [7, 3] and layer.tokens_upper == 7
    monkeypatch.setattr(paged.torch, "empty", fails)     # no room for the queries
    with pytest.raises(type(error)):
        layer.append(rows, rows, None, 1, q=rows)
    assert layer.seq_lens.tolist() == [7, 3]


@pytest.mark.gpu
def test_a_layer_after_arguments_that_are_no_numbers_or_tensors():
    dq, _ = _lib()
    layer = dq.PagedKVLayer(2, 4, 2, 64, 100, device=DEV)
    k = torch.ones((2, 2, 64), dtype=torch.float16, device=DEV)
    q = torch.ones((2, 4, 64), dtype=torch.float16, device=DEV)
    layer.append(k, k)
    for bad in (dict(eps="small", k_weight=k[0, 0]), dict(eps=None, k_weight=k[0, 0]), dict(q="queries"), dict(rotary=3), dict(positions=3, rotary=dq.rotary(64, device=DEV)),
                dict(q=q.float()), dict(k_weight=5)):
        with pytest.raises((TypeError, AttributeError, dq.DQError)):
            layer.append(k, k, **bad)
        assert layer.seq_lens.tolist() == [1, 1] and layer.tokens_upper == 1, bad
    layer.append(k, k)
    assert layer.seq_lens.tolist() == [2, 2]
    assert (layer.attend(q) == 1).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,codes,page", [(torch.float16, torch.int8, 64), (torch.bfloat16, torch.float8_e4m3fn, 128)])
def test_a_layer_reads_any_prefix(dtype, codes, page):
    """Prefixes that end inside a quantized page, in the tail, at a page's end, at 0 and behind the tokens: the rows of the whole
    read, zeros behind them."""
    dq, _ = _lib()
    gen = torch.Generator().manual_seed(page)
    heads, d, lens = 2, 64, [3 * page + 8, page, 17]
    layer = dq.PagedKVLayer(3, 4, heads, d, 4 * page, page, dtype, codes, DEV)
    k, v = (torch.randn((sum(lens), heads, d), generator=gen).to(dtype).to(DEV) for _ in range(2))
    layer.append(k, v, torch.tensor([0, lens[0], lens[0] + lens[1], sum(lens)], dtype=torch.int32, device=DEV), max(lens))
    whole = layer.read(lens)
    at = torch.tensor([0, lens[0], lens[0] + lens[1]])
    for got, x in zip(whole, (k, v)):
        for b, n in enumerate(lens):
            # codes of a block are off by half a step of its largest value at most: 1 / 254, or 2^-4 of the value itself
            err = (got[b, :, :n].transpose(0, 1).float() - x[at[b]:at[b] + n].float()).abs()
            assert (err <= x.float().abs().max() / 250 + x[at[b]:at[b] + n].float().abs() * 2.0 ** -4 * 1.1).all()
    for lengths in ([page + 36, page - 1, 3], [2 * page, 1, 17], [3 * page + 1, 0, 0], [1, page, 16], [0, 0, 0], [4 * page, 2 * page, page]):
        for got, full in zip(layer.read(lengths), whole):
            assert got.shape[2] == max(lengths)
            for b, n in enumerate(lengths):
                m = min(n, lens[b])
                assert torch.equal(got[b, :, :m], full[b, :, :m]), (lengths, b)
                assert (got[b, :, m:] == 0).all(), (lengths, b)
    for bad in ([1, 2], [1, 2, -1], [1, 2, 3, 4]):
        with pytest.raises(dq.DQError, match="length"):
            layer.read(bad)


def test_the_workspaces_of_a_layer_stay_within_twice_the_largest(monkeypatch):
    """Prompts that are each a little longer than the last: a new workspace only where its bytes grew, each at least twice the one before."""
    dq, paged = _lib()
    made, given = [], []
    monkeypatch.setattr(paged.torch.cuda, "is_current_stream_capturing", lambda: False)      # (raises where there is no GPU)
    monkeypatch.setattr(paged, "_new_workspace", lambda cache, n: made.append(n) or torch.empty(n, dtype=torch.uint8))
    monkeypatch.setattr(paged, "paged_attention", lambda cache, q, starts, lens, table, most, bound, ws, **k: given.append(ws) or q)
    for kv_heads, d, batch, top in ((8, 128, 8, 4096), (1, 64, 1, 1200), (2, 64, 3, 300)):
        layer = _host_layer(paged, 8192)
        layer.batch, layer.q_heads = batch, 4 * kv_heads
        layer.cache = type("Cache", (), {})()
        layer.cache.c = paged._CPaged(*[0x1000] * 6, 10, kv_heads, d, 64, 8, 0, 0)
        made.clear()
        for rows in [1] + [5 + i * top // 100 for i in range(100)] + [1, 3]:
            layer.attend(torch.empty((batch * rows, 4 * kv_heads, d), dtype=torch.float16, device="meta"), None, rows)
            need = dq.lib.dq_paged_workspace_bytes(layer.cache.c, batch, batch * rows, 4 * kv_heads, rows, 8192)
            assert given[-1].numel() >= need and given[-1] is layer._ws
        assert sum(made) < 2 * made[-1] and len(made) <= 12, made
        assert made == sorted(made) and all(b >= 2 * a for a, b in zip(made, made[1:]))
        assert made[-1] <= 2 * dq.lib.dq_paged_workspace_bytes(layer.cache.c, batch, batch * top, 4 * kv_heads, top, 8192)
        assert len(layer._outgrown) == len(made) - 1


def test_a_workspace_made_in_a_capture_is_for_that_call_alone(monkeypatch):
    dq, paged = _lib()
    given = []
    monkeypatch.setattr(paged, "_new_workspace", lambda cache, n: torch.empty(n, dtype=torch.uint8))
    monkeypatch.setattr(paged, "paged_attention", lambda cache, q, starts, lens, table, most, bound, ws, **k: given.append(ws) or q)
    layer = _host_layer(paged, 8192)
    layer.cache = type("Cache", (), {})()
    layer.cache.c = paged._CPaged(*[0x1000] * 6, 10, 1, 64, 64, 8, 0, 0)
    q = [torch.empty((2 * n, 4, 64), dtype=torch.float16, device="meta") for n in (1, 300)]
    for capturing in (True, False, True, True, False):
        monkeypatch.setattr(paged.torch.cuda, "is_current_stream_capturing", lambda: capturing)
        layer.attend(q[0], None, 1)
    layer.attend(q[1], None, 300)
    assert given[0] is layer._outgrown[0] and given[0] is not given[1]           # the first call was captured
    assert all(x is given[1] for x in given[1:5])                               # there was one from then on
    monkeypatch.setattr(paged.torch.cuda, "is_current_stream_capturing", lambda: True)
    kept = layer._ws
    layer.attend(torch.empty((2000, 4, 64), dtype=torch.float16, device="meta"), None, 1000)
    assert layer._ws is kept and given[-1] is layer._outgrown[-1] or given[-1] is kept


@pytest.mark.gpu
def test_a_layer_whose_first_attention_is_captured():
    """Outside the graph and in its replays, in any order, the results of a layer that was never captured."""
    dq, _ = _lib()
    gen = torch.Generator().manual_seed(5)
    heads, hq, d, n = 1, 4, 64, 3000
    k, v = (torch.randn((2 * n, heads, d), generator=gen).half().to(DEV) for _ in range(2))
    q = torch.randn((2, hq, d), generator=gen).half().to(DEV)
    starts = torch.tensor([0, n, 2 * n], dtype=torch.int32, device=DEV)
    layer, plain = (dq.PagedKVLayer(2, hq, heads, d, 4000, device=DEV) for _ in range(2))
    for x in (layer, plain):
        x.append(k, v, starts, n)
    want = plain.attend(q)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        out = layer.attend(q)
    for _ in range(3):
        assert torch.equal(layer.attend(q), want)        # before the first replay too
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.gpu
def test_tensors_that_require_gradients_are_taken_and_outputs_carry_none():
    dq, paged = _lib()
    x = torch.ones((2, 2, 64), dtype=torch.float16, device=DEV, requires_grad=True)
    w = torch.ones(64, dtype=torch.float16, device=DEV, requires_grad=True)
    q, _ = dq.rotate_heads(x, None, q_weight=w)
    assert not q.requires_grad
    layer = dq.PagedKVLayer(2, 2, 2, 64, 64, device=DEV)
    q = layer.append(x, x, q=x, k_weight=w, q_weight=w)
    out = layer.attend(q)
    assert not q.requires_grad and not out.requires_grad and (out == 1).all()
    for f in (dq.rotate_heads, dq.paged_append, dq.paged_attention):
        assert "No gradients" in f.__doc__


def test_a_layer_and_a_rotation_refuse_sizes_that_make_no_sense():
    """Before anything is allocated, by the package's own error."""
    dq, _ = _lib()
    good = dict(batch=2, q_heads=4, kv_heads=2, head_dim=64, max_tokens=100, device="cpu")
    for bad in (dict(batch=0), dict(q_heads=0), dict(kv_heads=0), dict(kv_heads=-2), dict(kv_heads=3), dict(max_tokens=0), dict(page_tokens=0), dict(page_tokens=96)):
        with pytest.raises(dq.DQError, match="a layer has"):
            dq.PagedKVLayer(**dict(good, **bad))
    for base in (0, -10.0, float("nan")):
        with pytest.raises(dq.DQError, match="base"):
            dq.rotary(64, base=base, device="cpu")
