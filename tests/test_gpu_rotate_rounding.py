"""Norm and rotation to the bound of their arithmetic: every result is the 16-bit number next to the 64-bit form's, up to
what fp32 sines, cosines and sums may move it."""
import pytest
import torch

import paper_2405_12591_amd as dq
from paged_util import DEV, heads64, rows

pytestmark = pytest.mark.gpu


def _neighbours(x):
    """The 16-bit numbers below and above, as float64 (x finite; the sign's two zeros are one)."""
    i = x.view(torch.int16).int()
    order = torch.where(i < 0, -(i & 0x7FFF), i)          # ascending with the values
    back = lambda o: torch.where(o < 0, (-o) | 0x8000, o).to(torch.int16).view(x.dtype).double()   # noqa: E731
    return back(order - 1), back(order + 1)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d,rot,interleaved,normed,far", [(128, 128, False, False, 2 ** 20), (64, 32, True, False, 2 ** 20), (128, 128, False, True, 9000),
                                                           (256, 256, True, True, 300)])
def test_results_are_the_nearest_numbers(dtype, d, rot, interleaved, normed, far):
    """What may move a result before it is rounded, in units u = 2^-24 of the terms a channel is summed from:
    sine and cosine: the reduced angle, |x| <= pi / 4, is rounded once, multiplied by a rounded pi / 2 and rounded (3 u of x, 2.4 u), the
    polynomials are cut off at 0.04 u and their last two steps round (1.5 u): 4 u; two products and a sum: 2 u.  6 u < 2^-21.
    Norm: a sum of d squares, 16 in a row and 4 levels of lanes (20 u, half of it in the root), mean, eps, root and inverse (2.5 u), weight and
    channel (2 u): 14.5 u < 2^-20.  The angle itself, in fp64, is off by 2^-32 of a turn at positions below 2^20."""
    gen = torch.Generator().manual_seed(d + rot)
    x = rows((600, 8, d), dtype, gen, outliers=False)
    pos = torch.randint(0, far, (600,), generator=gen).to(torch.int32)
    r = dq.rotary(rot, interleaved=interleaved, device=DEV)
    w = (1 + 0.3 * torch.randn(d, generator=gen)).to(dtype) if normed else None
    got, _ = dq.rotate_heads(x.to(DEV), None, pos.to(DEV), r, q_weight=None if w is None else w.to(DEV))
    got = got.cpu()
    y, mag = heads64(x, w, 1e-6, r.inv_freq.cpu(), None, pos, rot, interleaved)
    below, above = _neighbours(got)
    slack = mag * (2.0 ** -21 + (2.0 ** -20 if normed else 0.0))
    g = got.double()
    assert ((y >= (below + g) / 2 - slack) & (y <= (above + g) / 2 + slack)).all(), \
        float(torch.maximum((below + g) / 2 - y, y - (above + g) / 2).div(mag).max()) * 2 ** 24
    # typical errors of 2^-23 (2^-22 with the norm) cross a border of fp16's steps of 2^-10.5 in one result of 3000 (1500); channels that
    # nearly cancel more often: five times that
    nearest = y.to(dtype)
    assert (got != nearest).double().mean() < (0.004 if normed else 0.002)
