"""The calls of a student's block at their edges: layouts of what a call takes without a stride, levels behind entries that do not exist, long sums, infinities and
far arguments, forms of the loss that a bound on the rows chooses. Tolerances as in `test_student_block`."""
import math

import numpy as np
import pytest
import torch

from tests import student_reference as R
from tests.test_student_block import B, HALF, T, TINY, act_code, close, code, sentinel, stride, values  # noqa: F401 (B: the fixture)

gpu = pytest.mark.gpu


def refused(B, fn, *a, **k):
    """The code of a call that the library, or the binding before it, refuses."""
    with pytest.raises(B.FgError) as e:
        fn(*a, **k)
    return e.value.code


def full(*shape):
    return torch.full(shape, -77.0, device="cuda")


# ---- layouts ----

def backward_of(B, x, dy, mean, rstd, blocks, off, act="silu", **k):
    n, d = x.shape
    G = len(off) - 1
    dx, dw, db = full(n, d), full(d), full(d)
    ws = torch.full((B.fg_group_norm_backward_workspace_bytes(n, G, d, blocks),), 255, dtype=torch.uint8, device="cuda")
    B.fg_group_norm_backward(dy, stride(dy), B.FG_F32, x, stride(x), B.FG_F32, mean, rstd, None, None, act_code(B, act), None, off, n, G, n, d, blocks, dx, stride(dx), dw, db, ws, len(ws),
                             **k)
    torch.cuda.synchronize()
    return dx, dw, db


@gpu
@pytest.mark.parametrize("n, n_groups, d, blocks", [(777, 9, 88, 8), (300, 100, 16, 16), (40_000, 3, 256, 8), (500, 4, 600, 2), (30_000, 2, 1024, 1), (9, 1, 64, 4)])
def test_statistics_in_any_layout(B, n, n_groups, d, blocks):
    """mean and rstd as tensor operations leave them: a block's groups behind each other, parts of a wider table, one row for all groups."""
    g = torch.Generator(device="cuda").manual_seed(n)
    kw = dict(device="cuda", generator=g)
    off = torch.linspace(0, n, n_groups + 1).long().cuda()
    x, dy = torch.randn(n, d, **kw), torch.randn(n, d, **kw)
    mean, rstd = 0.3 * torch.randn(n_groups, blocks, **kw), 0.5 + torch.rand(n_groups, blocks, **kw)
    want = backward_of(B, x, dy, mean, rstd, blocks, off)
    assert all(bool(torch.isfinite(t).all()) for t in want)

    def wider(t):
        v = torch.full((n_groups, 2, blocks, 3), math.nan, device="cuda")[:, 1, :, 1]
        return v.copy_(t)

    for layout in (lambda t: t.T.contiguous().T, wider, lambda t: t.flatten()):
        a, b = layout(mean), layout(rstd)
        for got, v in zip(backward_of(B, x, dy, a, b, blocks, off), want):
            assert torch.equal(got, v)
    a, b = wider(mean), wider(rstd)
    for got, v in zip(backward_of(B, x, dy, a.data_ptr(), b.data_ptr(), blocks, off, stat_strides=a.stride()), want):
        assert torch.equal(got, v)
    want = backward_of(B, x, dy, mean[:1].repeat(n_groups, 1), rstd[:1].repeat(n_groups, 1), blocks, off)
    for got, v in zip(backward_of(B, x, dy, mean[:1].expand(n_groups, -1), rstd[:1].expand(n_groups, -1), blocks, off), want):
        assert torch.equal(got, v)


def test_statistics_whose_layout_no_stride_can_say(B):
    P, off = 4096, 4096
    def bw(mean, rstd, **k):
        return refused(B, B.fg_group_norm_backward, P, 256, B.FG_F32, P, 256, B.FG_F32, mean, rstd, None, None, B.FG_ACT_SILU, None, off, 10, 4, 10, 64, 8, P + 4096, 256, P, P, P, 1 << 40, **k)
    t = torch.ones(8, 4).T
    assert bw(t, torch.ones(4, 8)) == B.FG_ERR_SHAPE and bw(torch.ones(4, 8), t) == B.FG_ERR_SHAPE      # of two layouts
    assert bw(t[:3], t[:3]) == B.FG_ERR_SHAPE and bw(torch.ones(64)[::2], torch.ones(64)[::2]) == B.FG_ERR_SHAPE
    for bad in ((-1, 1), (8, -1), (1 << 31, 1), (8, 2 * B.FG_MAX_NORM_GROUPS + 1)):
        assert bw(P, P, stat_strides=bad) == B.FG_ERR_SHAPE, bad
