"""Norm of query and key heads and their position rotation against the 64-bit form."""
import pytest
import torch

import paper_2405_12591_amd as dq
from paged_util import DEV, heads64, rotate_tolerance, rows

pytestmark = pytest.mark.gpu


def _check(got, x, w, rot, pos, eps=1e-6):
    inv = None if rot is None else rot.inv_freq.cpu()
    axis = None if rot is None or rot.axis_of_pair is None else rot.axis_of_pair.cpu()
    y, mag = heads64(x, w, eps, inv, axis, pos, 0 if rot is None else rot.rot_dim, rot is not None and rot.interleaved)
    err = (got.cpu().double() - y).abs()
    assert (err <= rotate_tolerance(y, mag, x.dtype)).all(), float((err - rotate_tolerance(y, mag, x.dtype)).max())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d,rot,interleaved", [(128, 128, False), (128, 64, True), (64, 64, False), (64, 16, False), (32, 32, True),
                                               (96, 96, False), (80, 48, False), (256, 256, False), (256, 128, True)])
@pytest.mark.parametrize("tokens,hq,hk", [(1, 1, 1), (33, 7, 3), (130, 12, 0), (5, 0, 2)])
def test_norm_and_rotation(dtype, d, rot, interleaved, tokens, hq, hk):
    gen = torch.Generator().manual_seed(d + rot + tokens)
    x = rows((tokens, hq + hk, d), dtype, gen)
    pos = torch.randint(-5, 2 ** 20, (tokens,), generator=gen).to(torch.int32)
    r = dq.rotary(rot, interleaved=interleaved, device=DEV)
    w = (1 + 0.3 * torch.randn(2, d, generator=gen)).to(dtype)
    xd = x.to(DEV)
    q, k = xd[:, :hq] if hq else None, xd[:, hq:] if hk else None
    print("rotate", dtype, d, rot, interleaved, tokens, hq, hk, flush=True)
    qo, ko = dq.rotate_heads(q, k, pos.to(DEV), r, q_weight=w[0].to(DEV), k_weight=None)
    if hq:
        _check(qo, x[:, :hq], w[0], r, pos)
    if hk:
        _check(ko, x[:, hq:], None, r, pos)
    # the norm alone, with another eps
    qo, ko = dq.rotate_heads(q, k, q_weight=w[0].to(DEV), k_weight=w[1].to(DEV), eps=0.5)
    if hq:
        _check(qo, x[:, :hq], w[0], None, None, 0.5)
    if hk:
        _check(ko, x[:, hq:], w[1], None, None, 0.5)


def test_several_axes_and_far_positions():
    gen = torch.Generator().manual_seed(5)
    for sections, interleaved in (((16, 24, 24), False), ((1, 62, 1), True), ((10, 0, 54), False), ((8,) * 8, False)):
        r = dq.rotary(128, base=1e6, sections=sections, interleaved=interleaved, device=DEV)
        pos = torch.randint(0, 2 ** 31 - 1, (len(sections), 50), generator=gen).to(torch.int32)
        x = rows((50, 3, 128), torch.float16, gen)
        got, _ = dq.rotate_heads(x.to(DEV), None, pos.to(DEV), r)
        _check(got, x, None, r, pos)


def test_layouts_in_place_and_batches():
    """[B, n, H, d] into the cache's [B, H, n, d]; in place on a view of a fused projection, whose other parts stay."""
    gen = torch.Generator().manual_seed(6)
    x = rows((3, 17, 6, 64), torch.bfloat16, gen)
    pos = torch.randint(0, 9999, (3, 17), generator=gen).to(torch.int32)
    r = dq.rotary(64, device=DEV)
    out = torch.full((3, 6, 17, 64), 9.0, dtype=torch.bfloat16, device=DEV)
    dq.rotate_heads(None, x.to(DEV), pos.to(DEV), r, k_out=out.transpose(1, 2))
    _check(out.transpose(1, 2).reshape(51, 6, 64), x.view(51, 6, 64), None, r, pos.view(-1))
    fused = rows((20, 9, 64), torch.bfloat16, gen)
    fd = fused.to(DEV)
    q, k = fd[:, :4], fd[:, 4:6]
    dq.rotate_heads(q, k, pos.view(-1)[:20].to(DEV), r, q_out=q, k_out=k)
    _check(fd[:, :6], fused[:, :6], None, r, pos.view(-1)[:20])
    assert torch.equal(fd[:, 6:].cpu(), fused[:, 6:])


def test_zero_rows_zero_values_and_values_that_are_not_finite():
    r = dq.rotary(64, device=DEV)
    empty = torch.empty((0, 2, 64), dtype=torch.float16, device=DEV)
    out, _ = dq.rotate_heads(empty, None, torch.empty(0, dtype=torch.int32, device=DEV), r)
    assert out.shape == empty.shape
    x = torch.zeros((4, 2, 64), dtype=torch.float16, device=DEV)
    x[1, 0, 3] = float("nan")
    x[2, 1, 5] = float("inf")
    w = torch.ones(64, dtype=torch.float16, device=DEV)
    got, _ = dq.rotate_heads(x, None, torch.arange(4, dtype=torch.int32, device=DEV), r, q_weight=w)
    got = got.cpu()
    assert (got[0] == 0).all() and (got[3] == 0).all() and (got[1, 1] == 0).all() and (got[2, 0] == 0).all()   # other heads are untouched
    assert torch.isnan(got[1, 0]).all()


def test_another_stream_and_a_captured_graph():
    gen = torch.Generator().manual_seed(8)
    x = [rows((40, 5, 128), torch.float16, gen) for _ in range(3)]
    pos = torch.arange(40, dtype=torch.int32)
    r = dq.rotary(128, device=DEV)
    src, dst = x[0].to(DEV), torch.empty((40, 5, 128), dtype=torch.float16, device=DEV)
    pd = pos.to(DEV)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(st):
        dq.rotate_heads(src, None, pd, r, q_out=dst)
        st.synchronize()
        _check(dst, x[0], None, r, pos)
        with torch.cuda.graph(graph, stream=st):
            dq.rotate_heads(src, None, pd, r, q_out=dst)
    for y in x:
        src.copy_(y)
        dst.zero_()
        graph.replay()
        torch.cuda.synchronize()
        _check(dst, y, None, r, pos)
