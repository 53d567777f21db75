"""What the entry points of the head rotation and the paged cache refuse before anything is launched: the C ABI
with pointers that are never followed, and the binding's checks.  No GPU needed."""
import ctypes as C
import struct

import pytest
import torch

PTR = 0x1000      # never dereferenced: the checks come first
# the header's small structs
_pack_heads = struct.Struct("@Pqqqi4x").pack
_pack_norm = struct.Struct("@PPf4x").pack
_pack_rotary = struct.Struct("@PPPqiii4x").pack
_pack_batch = struct.Struct("@PPPPiiii").pack


def _lib():
    import paper_2405_12591_amd as dq
    from paper_2405_12591_amd import paged
    return dq, paged


def _heads(paged, data=PTR, heads=8, strides=(0, 1024, 128)):
    return _pack_heads(data, *strides, heads)


def _cache(paged, **change):
    f = dict(k_codes=PTR, k_scales=PTR, v_codes=PTR, v_scales=PTR, k_tail=PTR, v_tail=PTR, pages=10, kv_heads=8, head_dim=128,
             page_tokens=64, slots=4, dtype=0, codes=0)
    f.update(change)
    return C.byref(paged._CPaged(*f.values()))


def _batch(paged, starts=PTR, lens=PTR, table=PTR, slots=0, batch=4, rows=4, width=5, stride=5):
    return _pack_batch(starts, lens, table, slots, batch, rows, width, stride)


def test_rotate_heads_refuses():
    dq, paged = _lib()
    norm, rot = _pack_norm(PTR, PTR, 1e-6), _pack_rotary(PTR, PTR, 0, 4, 1, 128, 0)

    def call(q=None, q_out=None, k=None, k_out=None, batch=1, tokens=0, d=128, dtype=0, norm=norm, rot=rot):
        return dq.lib.dq_rotate_heads(q, q_out, k, k_out, batch, tokens, d, dtype, norm, rot, None)

    h = _heads(paged)
    assert call(h, h) == 0 and call(None, None, h, h) == 0 and call(h, h, h, h) == 0     # no rows: nothing to launch
    assert call() == -1 and call(h, None) == -1 and call(None, None, h, None) == -1
    assert call(h, h, norm=None, rot=None) == -1
    assert call(h, _heads(paged, heads=4)) == -1
    for bad in (dict(data=0), dict(data=PTR + 2), dict(heads=0), dict(strides=(0, 1020, 128)), dict(strides=(0, 1024, 4)), dict(strides=(4, 0, 0)),
                dict(strides=(0, -8, 128))):
        assert call(_heads(paged, **bad), h) == -1, bad
        assert call(h, _heads(paged, **bad)) == -1, bad
    for bad in (dict(d=24), dict(d=16), dict(d=272), dict(d=0), dict(dtype=2), dict(dtype=-1), dict(batch=0), dict(tokens=-1), dict(batch=1 << 20, tokens=1 << 12)):
        assert call(h, h, **bad) == -1, bad
    for r in ((0, PTR, 0, 4, 1, 128, 0), (PTR, 0, 0, 4, 1, 128, 0), (PTR, PTR, 0, 4, 1, 120, 0), (PTR, PTR, 0, 4, 1, 144, 0), (PTR, PTR, 0, 4, 1, 0, 0),
              (PTR, PTR, 0, 4, 0, 128, 0), (PTR, PTR, PTR, 4, 9, 128, 0), (PTR, PTR, 0, 4, 2, 128, 0), (PTR, PTR, 0, 4, 1, 128, 2)):
        assert call(h, h, rot=_pack_rotary(*r)) == -1, r
    assert call(h, h, tokens=5, rot=_pack_rotary(PTR, PTR, PTR, 4, 2, 128, 0)) == -1        # fewer positions than rows
    for n in ((PTR + 2, 0, 1e-6), (0, PTR + 8, 1e-6), (PTR, 0, -1.0), (PTR, 0, float("nan"))):
        assert call(h, h, norm=_pack_norm(*n)) == -1, n


BAD_CACHES = [dict(k_codes=0), dict(v_scales=0), dict(k_tail=0), dict(v_tail=PTR + 8), dict(k_codes=PTR + 4), dict(k_scales=PTR + 2), dict(pages=0),
              dict(kv_heads=0), dict(slots=0), dict(head_dim=96), dict(page_tokens=32), dict(page_tokens=256), dict(dtype=2), dict(codes=2),
              dict(pages=1 << 30), dict(slots=1 << 29)]
BAD_BATCHES = [dict(lens=0), dict(table=0), dict(batch=0), dict(rows=-1), dict(width=0), dict(stride=4), dict(width=1 << 26, stride=1 << 26)]


def test_paged_append_and_read_refuse():
    dq, paged = _lib()
    h, q = _heads(paged), _heads(paged, heads=32)
    lib = dq.lib

    def append(cache=None, batch=None, k=h, v=h, q=None, q_out=None, norm=None, rot=None):
        return lib.dq_paged_append(cache or _cache(paged), batch or _batch(paged, rows=0), k, v, q, q_out, norm, rot, None)

    assert append() == 0 and append(q=q, q_out=q) == 0                                     # no rows: nothing to launch
    for c in BAD_CACHES:
        assert append(cache=_cache(paged, **c)) == -1, c
    for b in BAD_BATCHES:
        assert append(batch=_batch(paged, **b)) == -1, b
    assert append(batch=_batch(paged, starts=0, rows=3)) == -1                             # one row per sequence
    assert append(batch=_batch(paged, batch=5, rows=5)) == -1                              # more sequences than slots
    assert append(k=None) == -1 and append(v=None) == -1 and append(k=_heads(paged, heads=4)) == -1 and append(v=q) == -1
    assert append(q=q) == -1 and append(q_out=q) == -1 and append(q=q, q_out=h) == -1
    assert append(k=_heads(paged, data=PTR + 2)) == -1 and append(v=_heads(paged, strides=(0, 1, 128))) == -1
    assert append(rot=_pack_rotary(PTR, 0, 0, 4, 1, 144, 0)) == -1 and append(norm=_pack_norm(PTR + 1, 0, 1e-6)) == -1
    assert append(rot=_pack_rotary(PTR, 0, PTR, 4, 3, 128, 0)) == -1                 # several axes need positions
    assert append(rot=_pack_rotary(PTR, 0, 0, 4, 1, 128, 0)) == 0                    # one may do without
    assert lib.dq_paged_append(None, _batch(paged), h, h, None, None, None, None, None) == -1
    assert lib.dq_paged_append(_cache(paged), None, h, h, None, None, None, None, None) == -1

    def read(cache=None, batch=None, first=None, out_starts=PTR, k=h, v=h):
        return lib.dq_paged_read(cache or _cache(paged), batch or _batch(paged, rows=0), first, out_starts, k, v, None)

    assert read() == 0 and read(batch=_batch(paged, starts=0, rows=0)) == 0
    assert read(out_starts=None) == -1 and read(k=None) == -1 and read(v=q) == -1
    for c in BAD_CACHES:
        assert read(cache=_cache(paged, **c)) == -1, c
    for b in BAD_BATCHES:
        assert read(batch=_batch(paged, **b)) == -1, b


def test_paged_attention_refuses():
    dq, paged = _lib()
    lib, q = dq.lib, _heads(paged, heads=32, strides=(0, 4096, 128))
    need = lib.dq_paged_workspace_bytes(_cache(paged), 4, 4, 32, 1, 20000)
    assert need > 0

    def call(cache=None, batch=None, q=q, out=q, max_rows=1, max_len=20000, scale=0.0, window=0, ws=PTR, size=need, flags=1):
        return lib.dq_paged_attention(cache or _cache(paged), batch or _batch(paged, rows=0), q, out, max_rows, max_len, scale, window, ws, size, flags, None)

    assert call() == 0 and call(max_rows=0) == 0 and call(max_rows=0, max_len=0, batch=_batch(paged, starts=0, rows=4)) == 0
    for c in BAD_CACHES:
        assert call(cache=_cache(paged, **c)) == -1, c
    for b in BAD_BATCHES:
        assert call(batch=_batch(paged, **b)) == -1, b
    assert call(q=None) == -1 and call(out=None) == -1 and call(out=_heads(paged)) == -1
    assert call(q=_heads(paged, heads=12), out=_heads(paged, heads=12)) == -1
    assert call(ws=None) == -1 and call(ws=PTR + 8) == -1
    assert call(flags=2) == -1 and call(flags=1 | 65 << 8) == -1 and call(flags=1 << 31) == -1
    assert call(window=-1) == -1 and call(window=5, flags=0) == -1 and call(max_rows=-1) == -1 and call(max_len=-1) == -1 and call(scale=float("nan")) == -1
    assert call(size=255) == -2 and call(size=need, flags=1 | 64 << 8, batch=_batch(paged, starts=0), max_len=1 << 24) == -2
    # the workspace of some sizes is enough for all smaller ones
    for sizes in ((16, 5000, 4096, 40000), (3, 200, 70, 9000), (1, 1, 1, 1 << 20), (64, 64, 1, 100)):
        b, rows, most, length = sizes
        bound = lib.dq_paged_workspace_bytes(_cache(paged, slots=64), b, rows, 32, most, length)
        for bb in {1, b // 2, b} - {0}:
            for rr in {1, bb, rows // 7, rows} - {0}:
                for mm in {1, 3, 5, most // 3, most} - {0}:
                    for ll in {0, 64, 700, length // 3, length}:
                        if bb <= rr <= bb * mm and mm <= most:
                            assert lib.dq_paged_workspace_bytes(_cache(paged, slots=64), bb, rr, 32, mm, ll) <= bound, (sizes, bb, rr, mm, ll)
    for bad in ((0, 4, 32, 1, 100), (4, -1, 32, 1, 100), (4, 4, 12, 1, 100), (4, 4, 0, 1, 100), (4, 4, 32, -1, 100), (4, 4, 32, 1, -1), (1 << 22, 1 << 22, 32, 1, 100)):
        assert lib.dq_paged_workspace_bytes(_cache(paged), *bad) == 0, bad
    for c in BAD_CACHES:
        assert lib.dq_paged_workspace_bytes(_cache(paged, **c), 4, 4, 32, 1, 100) == 0, c


def test_the_binding_refuses_host_tensors_and_wrong_frequencies():
    dq, paged = _lib()
    x = torch.zeros((2, 4, 64), dtype=torch.float16)
    r = dq.rotary(64, device="cpu")
    with pytest.raises(dq.DQError, match="GPU"):
        dq.rotate_heads(x, None, torch.zeros(2, dtype=torch.int32), r)
    with pytest.raises(dq.DQError, match="q or k"):
        dq.rotate_heads(None, None)
    for bad in (torch.zeros(12, dtype=torch.float64), torch.zeros(8), torch.zeros((8, 8), dtype=torch.float64), torch.zeros(0, dtype=torch.float64),
                torch.zeros(16, dtype=torch.float64)[::2]):
        with pytest.raises(dq.DQError, match="inv_freq"):
            dq.Rotary(bad)
    f = torch.zeros(8, dtype=torch.float64)
    for kw in (dict(axes=3), dict(axes=9), dict(axes=0), dict(axis_of_pair=torch.zeros(8, dtype=torch.uint8)),
               dict(axes=2, axis_of_pair=torch.zeros(7, dtype=torch.uint8)), dict(axes=2, axis_of_pair=torch.zeros(8, dtype=torch.int32))):
        with pytest.raises(dq.DQError):
            dq.Rotary(f, **kw)
    for bad in (0, 8, 24, -16):
        with pytest.raises(dq.DQError):
            dq.rotary(bad, device="cpu")
    with pytest.raises(dq.DQError, match="sections"):
        dq.rotary(64, sections=(16, 17), device="cpu")
    with pytest.raises(dq.DQError, match="tensors"):
        dq.PagedCache({})
    good = {n: torch.zeros(shape, dtype=torch.uint8 if t == torch.int8 else t).view(t)
            for n, (shape, t) in paged._paged_shapes(3, 2, 2, 64, 64, torch.float16, torch.int8).items()}
    with pytest.raises(dq.DQError):                              # on the host
        dq.PagedCache(good)
    for kw in (dict(pages=0), dict(slots=0), dict(page_tokens=96)):
        with pytest.raises(dq.DQError):
            dq.alloc_paged_cache(**dict(dict(pages=1, slots=1, kv_heads=1, head_dim=64, device="cpu"), **kw))


@pytest.mark.gpu
def test_the_binding_refuses_tensors_that_do_not_fit():
    """Every call is refused by a check; nothing is launched."""
    dq, paged = _lib()
    dev, i32, f16 = "cuda:0", torch.int32, torch.float16
    c = dq.alloc_paged_cache(6, 3, 2, 64, 64, f16, torch.int8, dev)
    k = torch.zeros((2, 2, 64), dtype=f16, device=dev)
    lens, table = torch.ones(2, dtype=i32, device=dev), torch.zeros((2, 3), dtype=i32, device=dev)
    starts = torch.tensor([0, 1, 2], dtype=i32, device=dev)
    q = torch.zeros((2, 4, 64), dtype=f16, device=dev)
    ws = dq.paged_workspace(c, 2, 2, 4, 1, 192)
    good = dict(cache=c, k=k, v=k, starts=starts, seq_lens=lens, page_table=table)
    wide = torch.zeros((2, 2, 72), dtype=f16, device=dev)
    for bad in (dict(k=k.float()), dict(k=k[0]), dict(v=k[:1]), dict(k=wide[..., 4:68]), dict(k=torch.zeros((2, 3, 64), dtype=f16, device=dev)),
                dict(k=torch.zeros((2, 64, 2), dtype=f16, device=dev).transpose(1, 2)), dict(starts=starts[:2]), dict(starts=starts.long()),
                dict(starts=starts.cpu()), dict(starts=None, k=k[:1], v=k[:1]), dict(seq_lens=lens.float()), dict(seq_lens=lens[:0]), dict(page_table=table[:1]),
                dict(page_table=table.t()), dict(page_table=table[:, :0]), dict(page_table=table.long()), dict(tail_slots=lens[:1]), dict(q_out=q),
                dict(q=q, q_out=q[:1]), dict(q=q.bfloat16()), dict(q=q, q_out=q[:1].expand(2, 4, 64)), dict(k_weight=k[0, 0, :32]), dict(eps=-1.0, k_weight=k[0, 0]),
                dict(rotary=dq.rotary(128, device=dev)), dict(rotary=dq.rotary(64, device="cpu")),
                dict(rotary=dq.rotary(64, device=dev), positions=starts), dict(rotary=dq.rotary(64, sections=(16, 16), device=dev))):
        with pytest.raises(dq.DQError):
            dq.paged_append(**dict(good, **bad))
    with pytest.raises(dq.DQError):                              # more sequences than slots
        five = torch.ones(5, dtype=i32, device=dev)
        dq.paged_append(c, k[:1].expand(5, 2, 64), k[:1].expand(5, 2, 64), None, five, torch.zeros((5, 3), dtype=i32, device=dev))
    good = dict(cache=c, q=q, starts=starts, seq_lens=lens, page_table=table, max_rows=1, max_seq_len=192, workspace=ws)
    for bad in (dict(q=q[:, :3]), dict(q=q.bfloat16()), dict(out=q[:1]), dict(out=q[:, :1].expand(2, 4, 64)), dict(workspace=ws.float()), dict(workspace=ws[:128]),
                dict(window=-1), dict(window=4, causal=False), dict(max_rows=-1), dict(max_seq_len=-1), dict(workspace=ws.cpu()), dict(splits=65)):
        with pytest.raises(dq.DQError):
            dq.paged_attention(**dict(good, **bad))
    out = torch.zeros((5, 2, 64), dtype=f16, device=dev)
    for bad in (dict(first=lens[:1]), dict(out_starts=None), dict(v_out=out[:4]), dict(k_out=out[:1].expand(5, 2, 64))):
        with pytest.raises(dq.DQError):
            dq.paged_read(**dict(dict(cache=c, first=None, seq_lens=lens, out_starts=starts, page_table=table, k_out=out, v_out=out), **bad))
    pos = torch.zeros(2, dtype=i32, device=dev)
    r = dq.rotary(64, device=dev)
    for bad in (dict(positions=None), dict(positions=pos[:1]), dict(positions=pos.long()), dict(q_out=q[:1]), dict(k=k[:1]), dict(k_out=k), dict(q=q.double()),
                dict(rotary=None), dict(rotary=dq.rotary(128, device=dev)), dict(q_weight=k[0, 0].bfloat16())):
        with pytest.raises(dq.DQError):
            dq.rotate_heads(**dict(dict(q=q, k=None, positions=pos, rotary=r), **bad))
    layer = dq.PagedKVLayer(2, 4, 2, 64, 100, device=dev)
    with pytest.raises(dq.DQError, match="starts"):
        layer.append(k, k, max_rows=2)
    with pytest.raises(dq.DQError, match="exceed"):
        layer.append(k, k, starts, max_rows=101)
    torch.cuda.synchronize()


def test_the_compiled_checks_refuse_what_is_no_tensor():
    """Before any address is looked at; no GPU needed."""
    dq, paged = _lib()
    m = paged._module
    with pytest.raises(TypeError):
        m.rotate_heads()
    cache = paged._CPaged(*[PTR] * 6, 10, 8, 128, 64, 4, 0, 0)
    at = C.addressof(cache)
    x = torch.zeros((4, 8, 128), dtype=torch.float16)
    for bad in (None, [1, 2], 3.5, "k"):
        with pytest.raises(dq.DQError, match="tensor"):
            m.paged_append(at, 0, bad, x, None, x, x, None, None, None, None, None, None, None, 0.0, 0)
        with pytest.raises(dq.DQError, match="tensor"):
            m.paged_attention(at, 0, bad, x, None, x, x, None, 1, 100, 0.0, True, 0, 0, x, 0)
        with pytest.raises(dq.DQError, match="tensor"):
            m.paged_read(at, 0, None, x, x, x, None, bad, x, 0)
        with pytest.raises(dq.DQError):
            m.rotate_heads(bad, x, None, None, None, None, None, None, 0.0, 0, 0)
    for wrong in (x, x.bfloat16(), x[0], x[..., :64], x[None, None]):            # on the host, of another type, shape
        with pytest.raises(dq.DQError):
            m.paged_append(at, 0, wrong, x, None, x, x, None, None, None, None, None, None, None, 0.0, 0)
    with pytest.raises(TypeError):
        m.paged_append("cache", 0, x, x, None, x, x, None, None, None, None, None, None, None, 0.0, 0)


@pytest.mark.gpu
def test_the_compiled_checks_refuse_numbers_that_do_not_fit():
    dq, paged = _lib()
    dev, i32, f16 = "cuda:0", torch.int32, torch.float16
    c = dq.alloc_paged_cache(6, 3, 2, 64, 64, f16, torch.int8, dev)
    lens, table = torch.ones(2, dtype=i32, device=dev), torch.zeros((2, 3), dtype=i32, device=dev)
    q = torch.zeros((2, 4, 64), dtype=f16, device=dev)
    ws = dq.paged_workspace(c, 2, 2, 4, 1, 192)
    good = dict(cache=c, q=q, starts=None, seq_lens=lens, page_table=table, max_rows=1, max_seq_len=192, workspace=ws)
    for bad in (dict(max_rows=1 << 31), dict(max_seq_len=1 << 40), dict(window=-(1 << 33)), dict(splits=-1), dict(splits=128), dict(q=q[None]),
                dict(starts=[0, 1, 2]), dict(workspace=None)):
        with pytest.raises(dq.DQError):
            dq.paged_attention(**dict(good, **bad))
    for bad in (dict(max_rows=1.5), dict(max_seq_len="long"), dict(softmax_scale="s")):
        with pytest.raises(TypeError):
            dq.paged_attention(**dict(good, **bad))
    assert torch.equal(dq.paged_attention(**good), torch.zeros_like(q))
    torch.cuda.synchronize()
