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
