"""What the entry points of drafted trees, latents and expanded attention refuse before anything is launched: the C ABI with pointers that are
never followed, the binding's checks, and that its calls have the compiled functions' arguments.  No GPU needed."""
import ctypes as C
import struct

import pytest
import torch

PTR = 0x10000     # never dereferenced: the checks come first
FAR = 0x90000000
_pack_heads = struct.Struct("@Pqqqi4x").pack
_pack_rotary = struct.Struct("@PPPqiii4x").pack
_pack_batch = struct.Struct("@PPPPiiii").pack
_pack_expanded = struct.Struct("@PqPPiiiiii").pack       # behind its four dq_heads


def _lib():
    import paper_2405_12591_amd as dq
    from paper_2405_12591_amd import latent, paged
    return dq, latent, paged


def _heads(data=PTR, heads=8, strides=(0, 1024, 128)):
    return _pack_heads(data, *strides, heads)


def _batch(starts=PTR, lens=PTR, table=PTR, slots=0, batch=4, rows=4, width=5, stride=5):
    return _pack_batch(starts, lens, table, slots, batch, rows, width, stride)


def _paged(paged, **change):
    f = dict(k_codes=PTR, k_scales=PTR, v_codes=PTR, v_scales=PTR, k_tail=PTR, v_tail=PTR, pages=10, kv_heads=8, head_dim=128,
             page_tokens=64, slots=4, dtype=0, codes=0)
    f.update(change)
    return C.byref(paged._CPaged(*f.values()))


def _latent(latent, **change):
    f = dict(rows=PTR, pages=10, page_tokens=64, latent_dim=512, rot_dim=64, dtype=1)
    f.update(change)
    return C.byref(latent._CLatent(*f.values()))


BAD_HEADS = [dict(data=0), dict(data=PTR + 2), dict(heads=0), dict(heads=-1), dict(strides=(0, 1020, 128)), dict(strides=(0, 1024, 4)), dict(strides=(0, -8, 128)),
             dict(strides=(0, 1024, -128))]
BAD_BATCHES = [dict(lens=0), dict(table=0), dict(batch=0), dict(batch=-1), dict(rows=-1), dict(width=0), dict(stride=4), dict(width=1 << 26, stride=1 << 26)]
BAD_LATENTS = [dict(rows=0), dict(rows=PTR + 8), dict(pages=0), dict(pages=-1), dict(page_tokens=32), dict(page_tokens=256), dict(latent_dim=576), dict(latent_dim=256),
               dict(rot_dim=32), dict(rot_dim=0), dict(dtype=2), dict(dtype=-1)]


def test_trees_refuse():
    dq, _, paged = _lib()
    need = dq.lib.dq_paged_tree_workspace_bytes
    assert need(_paged(paged), 4, 32, 32, 8, 300) > 0
    for bad in ((0, 32, 32, 8, 300), (4, -1, 32, 8, 300), (4, 32, 12, 8, 300), (4, 32, 0, 8, 300), (4, 32, 32, 65, 300), (4, 32, 32, -1, 300), (4, 32, 32, 8, -1)):
        assert need(_paged(paged), *bad) == 0, bad
    assert need(None, 4, 32, 32, 8, 300) == 0

    def call(cache=None, batch=None, q=_heads(heads=32), k=_heads(), v=_heads(), out=_heads(heads=32), seen=PTR, max_rows=4, max_len=300, scale=0.0, window=0, ws=PTR,
             size=1 << 40, flags=0):
        return dq.lib.dq_paged_tree_attention(cache or _paged(paged), batch or _batch(rows=0), q, k, v, out, seen, max_rows, max_len, scale, window, ws, size,
                                              flags, None)

    assert call() == 0                                                                  # no rows: nothing to launch
    for name in ("q", "k", "v", "out"):
        n = 32 if name in ("q", "out") else 8
        for bad in BAD_HEADS:
            assert call(**{name: _heads(**{"heads": n, **bad})}) == -1, (name, bad)
        assert call(**{name: None}) == -1 and call(**{name: _heads(heads=16)}) == -1
    for bad in BAD_BATCHES + [dict(starts=0, rows=3)]:
        assert call(batch=_batch(**{"rows": 0, **bad})) == -1, bad
    for bad in (dict(seen=0), dict(seen=PTR + 4), dict(max_rows=65), dict(max_rows=-1), dict(max_len=-1), dict(window=63), dict(window=-1), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(ws=0), dict(ws=PTR + 4), dict(flags=1)):
        assert call(batch=_batch(), **bad) == -1, bad
    assert call(batch=_batch(), size=need(_paged(paged), 4, 4, 32, 4, 300) - 1) == -2
    for bad in (dict(k_codes=0), dict(v_scales=0), dict(v_tail=PTR + 8), dict(pages=0), dict(slots=0), dict(head_dim=96), dict(page_tokens=32), dict(dtype=2), dict(codes=2)):
        assert call(cache=_paged(paged, **bad)) == -1, bad


def test_latent_append_and_read_refuse():
    dq, latent, _ = _lib()
    rot, q = _pack_rotary(PTR, 0, 0, 4, 1, 64, 0), _heads(heads=32, strides=(0, 2048, 64))

    def append(cache=None, batch=None, c=PTR, c_stride=576, k=PTR, k_stride=576, weight=0, eps=1e-6, q=None, q_out=None, rot=rot):
        return dq.lib.dq_latent_append(cache or _latent(latent), batch or _batch(rows=0), c, c_stride, k, k_stride, weight, eps, q, q_out, rot, None)

    assert append() == 0 and append(q=q, q_out=q) == 0 and append(rot=None) == 0 and append(weight=PTR) == 0
    for bad in BAD_LATENTS:
        assert append(cache=_latent(latent, **bad)) == -1, bad
    for bad in BAD_BATCHES + [dict(starts=0, rows=3)]:
        assert append(batch=_batch(**{"rows": 0, **bad})) == -1, bad
    for bad in (dict(c=0), dict(c=PTR + 8), dict(c_stride=580), dict(c_stride=-8), dict(k=0), dict(k=PTR + 8), dict(k_stride=4), dict(k_stride=-576),
                dict(weight=PTR + 2), dict(weight=PTR, eps=-1.0), dict(weight=PTR, eps=float("nan")), dict(q=q), dict(q_out=q), dict(q=q, q_out=_heads(heads=16))):
        assert append(**bad) == -1, bad
    for bad in BAD_HEADS:
        assert append(q=_heads(**{"heads": 32, **bad}), q_out=q) == -1 and append(q=q, q_out=_heads(**{"heads": 32, **bad})) == -1, bad
    for bad in ((0, 0, 0, 4, 1, 64, 0), (PTR, 0, 0, 4, 1, 32, 0), (PTR, 0, 0, 4, 1, 128, 0), (PTR, 0, 0, 4, 1, 64, 2), (PTR, 0, 0, 4, 0, 64, 0), (PTR, PTR, 0, 4, 2, 64, 0),
                (PTR, 0, 0, 4, 9, 64, 0)):
        assert append(rot=_pack_rotary(*bad)) == -1, bad

    def read(cache=None, batch=None, first=PTR, starts=PTR, out=PTR, stride=576):
        return dq.lib.dq_latent_read(cache or _latent(latent), batch or _batch(rows=0), first, starts, out, stride, None)

    assert read() == 0 and read(first=None) == 0
    for bad in BAD_LATENTS:
        assert read(cache=_latent(latent, **bad)) == -1, bad
    for bad in BAD_BATCHES:
        assert read(batch=_batch(**{"rows": 0, **bad})) == -1, bad
    for bad in (dict(starts=0), dict(out=0), dict(out=PTR + 8), dict(stride=568), dict(stride=580), dict(stride=-576)):
        assert read(**bad) == -1, bad


def test_latent_attention_refuses():
    dq, latent, _ = _lib()
    need = dq.lib.dq_latent_workspace_bytes
    assert need(_latent(latent), 4, 32, 16, 8, 300) > 0
    for bad in ((0, 32, 16, 8, 300), (4, -1, 16, 8, 300), (4, 32, 0, 8, 300), (4, 32, 16, -1, 300), (4, 32, 16, 8, -1)):
        assert need(_latent(latent), *bad) == 0, bad
    assert need(None, 4, 32, 16, 8, 300) == 0
    q, out = _heads(heads=16, strides=(0, 9216, 576)), _heads(data=FAR, heads=16, strides=(0, 8192, 512))

    def call(cache=None, batch=None, q=q, out=out, seen=None, max_rows=4, max_len=300, scale=0.1, ws=PTR, size=1 << 40, flags=1):
        return dq.lib.dq_latent_attention(cache or _latent(latent), batch or _batch(rows=0), q, out, seen, max_rows, max_len, scale, ws, size, flags, None)

    assert call() == 0 and call(seen=PTR) == 0 and call(flags=0) == 0
    for bad in BAD_LATENTS:
        assert call(cache=_latent(latent, **bad)) == -1, bad
    for bad in BAD_BATCHES + [dict(starts=0, rows=3)]:
        assert call(batch=_batch(**{"rows": 0, **bad})) == -1, bad
    for bad in BAD_HEADS:
        assert call(q=_heads(**{"heads": 16, **bad})) == -1 and call(out=_heads(**{"heads": 16, **bad})) == -1, bad
    for bad in (dict(q=None), dict(out=None), dict(out=_heads(heads=8)), dict(seen=PTR, flags=0), dict(seen=PTR, max_rows=65), dict(seen=PTR + 4), dict(max_rows=-1),
                dict(max_len=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(ws=0), dict(ws=PTR + 4), dict(flags=2),
                dict(flags=1 << 31)):
        assert call(batch=_batch(), **bad) == -1, bad
    assert call(batch=_batch(), size=need(_latent(latent), 4, 4, 16, 4, 300) - 1) == -2


def test_expanded_attention_refuses():
    dq, _, _ = _lib()
    need = dq.lib.dq_expanded_workspace_bytes
    assert need(4, 32, 16, 128, 8, 300) > 0
    for bad in ((0, 32, 16, 128, 8, 300), (4, -1, 16, 128, 8, 300), (4, 32, 0, 128, 8, 300), (4, 32, 16, 96, 8, 300), (4, 32, 16, 128, -1, 300), (4, 32, 16, 128, 8, -1)):
        assert need(*bad) == 0, bad
    good = dict(q=dict(heads=16, strides=(0, 3200, 200)), k=dict(heads=16, strides=(0, 4096, 256)), v=dict(heads=16, strides=(0, 4096, 256)),
                out=dict(data=FAR, heads=16, strides=(0, 2048, 128)))
    tail = dict(k_rot=PTR, k_rot_stride=64, starts=PTR, kv_starts=PTR, batch=4, rows=0, tokens=100, head_dim=128, rot_dim=64, dtype=1)

    def call(args=None, max_rows=4, max_len=300, scale=0.1, ws=PTR, size=1 << 40, flags=1, **change):
        packed = b"".join(_heads(**{**good[n], **change.pop(n, {})}) for n in ("q", "k", "v", "out"))
        return dq.lib.dq_expanded_attention(packed + _pack_expanded(*{**tail, **change}.values()), max_rows, max_len, scale, ws, size, flags, None)

    assert call() == 0 and call(flags=0) == 0 and call(scale=0.0) == 0
    assert dq.lib.dq_expanded_attention(None, 4, 300, 0.1, PTR, 1 << 40, 1, None) == -1
    for name in ("q", "k", "v", "out"):
        for bad in BAD_HEADS + [dict(heads=8)]:
            assert call(**{name: bad}) == -1, (name, bad)
    for bad in (dict(k_rot=0), dict(k_rot=PTR + 8), dict(k_rot_stride=60), dict(k_rot_stride=-64), dict(starts=0), dict(kv_starts=0), dict(batch=0), dict(rows=-1),
                dict(tokens=-1), dict(head_dim=96), dict(head_dim=64), dict(rot_dim=32), dict(dtype=2), dict(max_rows=-1), dict(max_len=-1), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(flags=2), dict(ws=PTR + 4), dict(ws=0)):
        assert call(**{"rows": 4, **bad}) == -1, bad
    assert call(rows=4, size=need(4, 4, 16, 128, 4, 300) - 1) == -2


def test_outputs_that_share_channels_with_inputs_are_refused():
    """What is refused for its places gives -1, what is not goes on to the size of the workspace (-2)."""
    dq, latent, _ = _lib()

    def absorbed(q, out, rows=4):
        return dq.lib.dq_latent_attention(_latent(latent), _batch(rows=rows, batch=rows), q, out, None, 4, 300, 0.1, PTR, 0, 1, None)

    q = _heads(data=FAR, heads=16, strides=(0, 9216, 576))      # (below PTR there would be no address left for the outputs)
    end = FAR + 2 * 4 * 9216
    for data, strides, status in ((FAR, (0, 9216, 576), -1), (FAR + 128, (0, 9216, 576), -1), (end, (0, 8192, 512), -2), (end - 16, (0, 8192, 512), -1),
                                  (FAR - 2 * 4 * 8192, (0, 8192, 512), -2), (FAR - 2 * 4 * 8192 + 16, (0, 8192, 512), -1), (FAR + 64, (0, 8192, 512), -1)):
        assert absorbed(q, _heads(data=data, heads=16, strides=strides)) == status, (data - FAR, strides)
    # slices of one buffer: [rows, heads, 576 + 512], [rows, 16 heads of 576 and then 16 of 512], [heads, rows, ..]
    assert absorbed(_heads(heads=16, strides=(0, 16 * 1088, 1088)), _heads(data=PTR + 2 * 576, heads=16, strides=(0, 16 * 1088, 1088))) == -2
    assert absorbed(_heads(heads=16, strides=(0, 16 * 1088, 1088)), _heads(data=PTR + 2 * 568, heads=16, strides=(0, 16 * 1088, 1088))) == -1
    assert absorbed(_heads(heads=16, strides=(0, 16 * 1088, 576)), _heads(data=PTR + 2 * 9216, heads=16, strides=(0, 16 * 1088, 512))) == -2
    assert absorbed(_heads(heads=16, strides=(0, 16 * 1088, 576)), _heads(data=PTR + 2 * 9208, heads=16, strides=(0, 16 * 1088, 512))) == -1
    assert absorbed(_heads(heads=16, strides=(0, 576, 4 * 576)), _heads(data=PTR + 2 * 16 * 4 * 576, heads=16, strides=(0, 512, 4 * 512))) == -2
    assert absorbed(_heads(heads=16, strides=(0, 1 << 62, 1 << 60)), _heads(data=PTR + 2 * 576, heads=16, strides=(0, 1 << 62, 1 << 60))) == -2

    def expanded(**out):
        heads = [dict(heads=16, strides=(0, 6144, 384)), dict(data=PTR + 2 * 192, heads=16, strides=(0, 6144, 384)), dict(data=PTR + 2 * 256, heads=16, strides=(0, 6144, 384))]
        packed = b"".join(_heads(**h) for h in heads + [dict(heads=16, strides=(0, 2048, 128), **out)])
        tail = dict(k_rot=FAR, k_rot_stride=64, starts=PTR, kv_starts=PTR, batch=4, rows=4, tokens=4, head_dim=128, rot_dim=64, dtype=1)
        return dq.lib.dq_expanded_attention(packed + _pack_expanded(*tail.values()), 4, 300, 0.1, PTR, 0, 1, None)

    for data, status in ((PTR, -1), (PTR + 2 * 192, -1), (PTR + 2 * 256, -1), (PTR + 2 * 4 * 6144, -2), (FAR, -1), (FAR + 16, -1), (FAR + 2 * 4 * 64, -2),
                         (FAR - 2 * 4 * 2048, -2)):
        assert expanded(data=data) == status, data


def test_the_binding_refuses_before_it_looks_for_a_gpu():
    dq, latent, paged = _lib()
    ok = torch.zeros(3, 64, 576, dtype=torch.bfloat16)
    for bad, dim in ((ok, 256), (ok[0], 512), (ok[:, :32], 512), (ok.float(), 512), (ok, 512)):       # (the last: not on a GPU)
        with pytest.raises(dq.DQError):
            dq.LatentCache(bad, dim)
    for bad in (dict(pages=0), dict(latent_dim=128), dict(rot_dim=32), dict(page_tokens=32)):
        with pytest.raises(dq.DQError):
            dq.alloc_latent_cache(**{"pages": 4, "device": "cpu", **bad})
    for bad in (dict(batch=0), dict(heads=0), dict(max_tokens=0), dict(page_tokens=96), dict(latent_dim=511)):
        with pytest.raises(dq.DQError):
            dq.LatentKVLayer(**{"batch": 1, "heads": 4, "max_tokens": 100, "device": "cpu", **bad})
    with pytest.raises(dq.DQError):
        dq.expanded_workspace(4, 32, 16, 96, 8, 300, "cpu")


def test_calls_have_the_compiled_functions_arguments(monkeypatch):
    """Every wrapper's call reaches the compiled function's own checks, old ones among them: it is refused for its tensors (none is on a GPU), not
    for their number."""
    dq, latent, paged = _lib()
    calls = []

    def call(fn, index, *args):
        calls.append(fn)
        fn(*args, 0)

    monkeypatch.setattr(paged, "_call", call)
    monkeypatch.setattr(latent, "_call", call)

    class Cache:
        index, device, kv_heads, head_dim, latent_dim, dtype = 0, "cpu", 8, 128, 512, torch.float16

    h = torch.zeros(1, 8, 128, dtype=torch.float16)
    i, table, ws = torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32), torch.zeros(64, dtype=torch.uint8)
    pc, lc = Cache(), Cache()
    pc.c = paged._CPaged(PTR, PTR, PTR, PTR, PTR, PTR, 10, 8, 128, 64, 4, 0, 0)
    lc.c = latent._CLatent(PTR, 10, 64, 512, 64, 0)
    pc._at, lc._at = C.addressof(pc.c), C.addressof(lc.c)
    wide = torch.zeros(1, 8, 576, dtype=torch.float16)
    for run in (lambda: dq.paged_append(pc, h, h, None, i, table), lambda: dq.paged_read(pc, None, i, i, table, h, h),
                lambda: dq.paged_attention(pc, h, None, i, table, 1, 1, ws), lambda: dq.paged_tree_attention(pc, h, h, h, i, None, i, table, 1, 1, ws),
                lambda: dq.latent_append(lc, h[:, 0], h[:, 0], None, i, table), lambda: dq.latent_read(lc, None, i, i, table, wide[:, 0]),
                lambda: dq.latent_attention(lc, wide, None, i, table, 1, 1, 0.1, ws),
                lambda: dq.expanded_attention(torch.zeros(1, 8, 192, dtype=torch.float16), h, h[:, 0, :64], h, i, i, 1, 1, ws)):
        with pytest.raises(dq.DQError):
            run()
    assert len(set(calls)) == 8
