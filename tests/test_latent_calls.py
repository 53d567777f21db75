"""Calls of the operators over latents and drafted trees at the edge of what they take, with pointers that are never followed: no GPU needed."""
import ctypes as C
import struct

import pytest
import torch

PTR = 0x10000     # never dereferenced
_pack_batch = struct.Struct("@PPPPiiii").pack


def _batch(rows=4, batch=4):
    return _pack_batch(PTR, PTR, PTR, 0, batch, rows, 5, 5)


def _latent(**change):
    from paper_2405_12591_amd import latent
    f = dict(rows=PTR, pages=10, page_tokens=64, latent_dim=512, rot_dim=64, dtype=1)
    f.update(change)
    return C.byref(latent._CLatent(*f.values()))


@pytest.mark.skipif(torch.cuda.is_available(), reason="its accepted calls would be launched")
def test_a_row_read_alone_needs_no_stride():
    """One row lies nowhere else than at its own start: the stride that the binding gives for it is 0.  (Accepted: a launch that finds no GPU.)"""
    import paper_2405_12591_amd as dq

    def read(rows, stride, **cache):
        return dq.lib.dq_latent_read(_latent(**cache), _batch(rows), None, PTR, PTR, stride, None)

    accepted = read(2, 576)
    assert accepted not in (0, -1, -2)
    for stride in (0, 8, 568, 576):
        assert read(1, stride) == accepted, stride
        assert read(1, stride, latent_dim=256, rot_dim=32) == accepted, stride
        assert read(2, stride) == (accepted if stride == 576 else -1), stride
    for stride in (-8, 4, 580):
        assert read(1, stride) == -1 and read(2, stride) == -1, stride


_pack_heads = struct.Struct("@Pqqqi4x").pack
FAR = 1 << 40


def _meeting(a, b):
    """Whether two sets of runs of channels (first element, length) have an element in common."""
    runs = sorted([(x, x + n, 0) for x, n in a] + [(x, x + n, 1) for x, n in b])
    end = [-1 << 60, -1 << 60]
    for x, y, side in runs:
        if x < end[1 - side]:
            return True
        end[side] = max(end[side], y)
    return False


def _absorbed(q_heads, q_token, q_head, out_at, out_token, out_head, rows):
    import paper_2405_12591_amd as dq
    q = _pack_heads(FAR, 0, q_token, q_head, q_heads)
    out = _pack_heads(FAR + 2 * out_at, 0, out_token, out_head, q_heads)
    status = dq.lib.dq_latent_attention(_latent(), _batch(rows, rows), q, out, None, 1, 300, 0.1, PTR, 0, 1, None)
    assert status in (-1, -2)                                       # refused for its places, or for the workspace, which is looked at next
    cells = [(r, h) for r in range(rows) for h in range(q_heads)]
    return status == -1, _meeting([(r * q_token + h * q_head, 576) for r, h in cells], [(out_at + r * out_token + h * out_head, 512) for r, h in cells])


def test_outputs_beside_inputs_in_one_buffer_are_taken():
    """Slices of [rows, heads * (576 + 512) + 8]: no channel in common, whatever multiple a row is of a head."""
    for rows in (1, 2, 5):
        for heads in (1, 2, 16):
            for pad in (0, 8, 24, 1088):
                row = heads * 1088 + pad
                assert _absorbed(heads, row, 1088, 576, row, 1088, rows) == (False, False), (rows, heads, pad)
                assert _absorbed(heads, row, 1088, 568, row, 1088, rows) == (True, True), (rows, heads, pad)
                assert _absorbed(heads, 1088, 1088 * rows + pad, 576, 1088, 1088 * rows + pad, rows) == (False, False), (rows, heads, pad)


def test_what_meets_is_refused_and_the_same_strides_exactly_that():
    import random
    rng = random.Random(0)
    met = apart = 0
    for i in range(6000):
        rows, heads = rng.randint(1, 4), rng.randint(1, 4)
        strides = [8 * rng.choice([0, 8, 64, 72, 73, 136, 137, 200, 272, 300, 545, 600, rng.randint(0, 700)]) for _ in range(4)]
        if i % 2:
            strides[2:] = strides[:2]
        q_token, q_head, out_token, out_head = strides
        refused, meet = _absorbed(heads, q_token, q_head, 8 * rng.randint(-800, 800), out_token, out_head, rows)
        assert refused or not meet, (rows, heads, strides)
        nested = max(strides[0], strides[1]) >= 1088 + (max(rows, heads) - 1) * min(strides[0], strides[1])
        if i % 2 and nested:
            assert refused == meet, (rows, heads, strides)
            met, apart = met + meet, apart + (not meet)
    assert met > 100 and apart > 100



def _tree(rows, q, k, v, out, q_heads=32, kv_heads=8):
    """Status of a call over heads (first element from FAR, token stride, head stride): -1 refused, -3 a launch that finds no GPU."""
    import paper_2405_12591_amd as dq
    from paper_2405_12591_amd import paged
    cache = C.byref(paged._CPaged(PTR, PTR, PTR, PTR, PTR, PTR, 10, kv_heads, 128, 64, 8, 0, 0))
    heads = [_pack_heads(FAR + 2 * at, 0, token, head, n) for (at, token, head), n in zip((q, k, v, out), (q_heads, kv_heads, kv_heads, q_heads))]
    return dq.lib.dq_paged_tree_attention(cache, _batch(rows, rows), *heads, PTR, 4, 300, 0.0, 0, PTR, 1 << 40, 0, None)


@pytest.mark.skipif(torch.cuda.is_available(), reason="its accepted calls would be launched")
@pytest.mark.parametrize("rows", [1, 2, 5])
def test_a_trees_output_is_the_queries_or_apart(rows):
    w = 48 * 128                                                    # a fused projection's row: 32 query heads, 8 of keys, 8 of values
    q, k, v, far = (0, w, 128), (4096, w, 128), (5120, w, 128), 1 << 30
    assert _tree(rows, q, k, v, (far, 4096, 128)) == -3 and _tree(rows, q, k, v, q) == -3
    # over keys or values, wholly or in part, and over other queries than its own
    for out in (k, v, (4096 - 8, w, 128), (4096 + 1024 + 1016, w, 128), (128, w, 128), (8, w, 128), (-8, w, 128), (0, w + 8, 128) if rows > 1 else k, (0, w, 136)):
        assert _tree(rows, q, k, v, out) == -1, out
    # queries elsewhere, the output in the place of the queries that were projected beside the keys; keys of every second head's place
    assert _tree(rows, (far, 4096, 128), k, v, q) == -3
    assert _tree(rows, (0, 16384, 512), (128, 16384, 512), (256, 16384, 512), (384, 16384, 512), q_heads=8) == -3
    assert _tree(rows, (0, 16384, 512), (128, 16384, 512), (256, 16384, 512), (376, 16384, 512), q_heads=8) == -1
    # one head, one row: their strides say nothing
    assert _tree(1, (0, 8, 0), (far, 16, 0), (2 * far, 8, 0), (0, 0, 64), q_heads=1, kv_heads=1) == -3


def _append(rows, c, k, q, q_out, q_heads=32):
    """Status of a call over rows (first element from FAR, stride) and heads (.., token stride, head stride): -1 refused, -3 a launch that finds no GPU."""
    import paper_2405_12591_amd as dq
    rot = struct.Struct("@PPPqiii4x").pack(PTR, 0, 0, rows, 1, 64, 0)
    heads = [_pack_heads(FAR + 2 * at, 0, token, head, q_heads) for at, token, head in (q, q_out)]
    return dq.lib.dq_latent_append(_latent(), _batch(rows, rows), FAR + 2 * c[0], c[1], FAR + 2 * k[0], k[1], 0, 0.0, *heads, rot, None)


@pytest.mark.skipif(torch.cuda.is_available(), reason="its accepted calls would be launched")
@pytest.mark.parametrize("rows", [1, 2, 300])
def test_turned_queries_are_their_own_output_or_apart(rows):
    w = 576 + 32 * 192                                              # a fused projection's row: [c | k_rot | 32 heads of 128 + 64]
    c, k, q, far = (0, w), (512, w), (576 + 128, w, 192), 1 << 30
    assert _append(rows, c, k, q, q) == -3 and _append(rows, c, k, q, (far, 32 * 64, 64)) == -3
    assert _append(rows, c, k, (far, 32 * 64, 64), q) == -3 and _append(rows, c, k, q, (576, w, 192)) == -3 and _append(rows, c, k, q, (576 + 64, w, 192)) == -3
    for out in ((0, w, 192), (512, w, 192), (448, w, 64), (568, w, 192), (576 + 120, w, 192), (576 + 136, w, 192), (576 + 128 + 192, w, 192)):
        assert _append(rows, c, k, q, out) == -1, out
    # one head, one row: their strides say nothing; rows that are all the same one
    assert _append(1, (0, 0), (512, 0), (far, 0, 0), (far, 8, 16), q_heads=1) == -3
    assert _append(rows, (0, 0), (512, 0), (far, 64, 64), (576, 64, 64), q_heads=1) == -3
    assert _append(rows, (0, 0), (512, 0), (far, 64, 64), (568, 64, 64), q_heads=1) == -1


@pytest.mark.skipif(torch.cuda.is_available(), reason="its accepted calls would be launched")
def test_keys_of_no_tokens_have_no_address():
    import paper_2405_12591_amd as dq

    def call(tokens, k=PTR, v=PTR, k_rot=PTR, out=FAR, rows=4):
        heads = [_pack_heads(data, 0, token, head, 16) for data, token, head in ((PTR, 3200, 200), (k, 4096, 256), (v, 4096, 256), (out, 2048, 128))]
        tail = struct.Struct("@PqPPiiiiii").pack(k_rot, 64, PTR, PTR, 4, rows, tokens, 128, 64, 1)
        return dq.lib.dq_expanded_attention(b"".join(heads) + tail, 4, 300, 0.1, PTR, 1 << 40, 1, None)

    assert call(100) == call(0) == call(0, 0, 0, 0) == -3 and call(0, 0, 0, 0, rows=0) == 0
    for none in (dict(k=0), dict(v=0), dict(k_rot=0)):
        assert call(100, **none) == -1 and call(0, **none) == -3
    assert call(0, out=0) == -1 and call(100, out=0) == -1


def test_a_workspace_is_shared_by_layers_of_a_kind_on_a_device():
    import paper_2405_12591_amd as dq
    from paper_2405_12591_amd.paged import _Workspace

    class Layer:
        _ws = _Workspace(torch.device("cpu"))

    class Other:
        _ws = _Workspace(torch.device("cpu"))

    make = _Workspace.made_or_shared
    assert make(torch.device("cpu"), Layer(), Layer, "_ws") is Layer._ws
    alone = make(torch.device("cpu"), None, Layer, "_ws")
    assert alone is not Layer._ws and alone.ws is None
    for device, layer in (("cpu", Other()), ("cpu", "a layer"), ("meta", Layer())):
        with pytest.raises(dq.DQError, match="workspace"):
            make(torch.device(device), layer, Layer, "_ws")
    small = Layer._ws.of(100)
    assert Layer._ws.of(50) is small and Layer._ws.of(101).numel() >= 200 and Layer._ws.outgrown == [small]
