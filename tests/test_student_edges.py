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


P = 4096
CALLS = {  # every array that a call takes without a stride, and (after "/") every one of rows that lie a stride apart
    "fg_group_rows": "groups ids rows n_rows order offsets ws /",
    "fg_linear_grouped": "x_scale src_ids order offsets W w_scale bias / x h_out",
    "fg_linear_grouped_backward": "src_ids order offsets W dw db ws / x dh h dx",
    "fg_dropout": "rows n_rows / x out",
    "fg_residual_norm": "rows n_rows weight y_scale rstd_out / x residual sum_out y",
    "fg_residual_norm_backward": "rstd weight rows n_rows dw ws / dy sum_ dsum_in dsum_out dx",
    "fg_quantize_rows": "scale / x q",
    "fg_gated_linear_grouped": "src_ids order offsets W bias / x h_out z_out",
    "fg_gated_linear_grouped_backward": "src_ids order offsets W dw db ws / x dh z dx",
    "fg_group_norm": "order offsets weight bias mean_out rstd_out ws / x y",
    "fg_group_norm_backward": "weight bias order offsets dw db ws / dy x dx",
    "fg_distill_loss": "rows n_rows ids top_idx top_val labels weight loss_out / h dh",
}


@pytest.mark.parametrize("name", CALLS)
def test_layouts_that_a_call_has_no_stride_for(B, name):
    """Refused by the binding, an array at a time; the same arrays behind each other go on to the library, which refuses what is asked for here (nothing is launched)."""
    import inspect
    flat, rows = (part.split() for part in CALLS[name].split("/"))
    fn = getattr(B, name)
    call = {p: 0 for p in inspect.signature(fn).parameters if p not in ("stream", "stat_strides")}
    assert set(flat + rows) | ({"mean", "rstd"} if name == "fg_group_norm_backward" else set()) <= set(call)
    call.update({a: P for a in flat + rows}, max_rows=-1, n_rows=-1 if name == "fg_quantize_rows" else P)
    call = {p: v for p, v in call.items() if p in inspect.signature(fn).parameters}
    apart = [torch.ones(6, 8).T, torch.ones(4, 3, 8)[:, 1, ::2]]                                                    # a row's elements are
    strided = [torch.ones(4, 6)[:, :4], torch.ones(3, 2)[:, :1]]                                                     # the rows are
    for array in flat + rows:
        for t in apart + ([*strided, torch.ones(20)[::2], torch.ones(1).expand(9)] if array in flat else []):
            with pytest.raises(B.FgError, match="contiguous|behind each other") as e:
                fn(**{**call, array: t})
            assert e.value.code == B.FG_ERR_INVALID_ARG, array
        for t in [torch.ones(4, 8), torch.ones(5), torch.ones(1, 8)] + (strided if array in rows else []):
            with pytest.raises(B.FgError) as e:
                fn(**{**call, array: t})
            assert "contiguous" not in str(e.value) and "behind each other" not in str(e.value), array


# ---- levels ----

@gpu
@pytest.mark.parametrize("dtype, n, d, blocks", [("f32", 60, 24, 3), ("f32", 60, 600, 2), ("f32", 1000, 16, 16), ("f32", 40_000, 256, 8), ("f32", 40_000, 512, 1), ("f32", 90_000, 24, 24),
                                                 ("bf16", 50_000, 1024, 32), ("f16", 30_000, 2048, 256)])
def test_levels_behind_entries_that_do_not_exist(B, dtype, n, d, blocks):
    """A group's first entries do not exist, and whole runs of entries further on: in groups of one workgroup and in split ones. The level of what is there still takes
    nothing from the variance: of equal values it is 0, of values about 300 or 10^7 as exact as for a level of 0."""
    r = np.random.default_rng(n + d)
    order = r.permutation(n).astype(np.int32)
    offsets = np.array([0, n // 3, n // 3, n], np.int64)
    for at in (0, n // 3):
        order[at:at + 1 + n // 50] = -1
    order[n // 2:n // 2 + n // 4] = n
    order[n - 3:] = 2 ** 31 - 1
    equal = 1e7 + 1 if dtype == "f32" else 300.0
    o, f = torch.from_numpy(order).cuda(), torch.from_numpy(offsets).cuda()
    ws = torch.full((B.fg_group_norm_workspace_bytes(n, 3, d, blocks),), 255, dtype=torch.uint8, device="cuda")
    for level, spread in ((equal, 0.0), (300.0, 1.5), (equal, 5.0)):
        x = values(r, n, d, dtype, 0, spread, level)
        y, mean, rstd = sentinel(n, d, "f32").cuda(), full(3, blocks), full(3, blocks)
        B.fg_group_norm(x.cuda(), d * T[dtype].itemsize, code(B, dtype), o, f, n, 3, n, d, blocks, None, None, 0.25, B.FG_ACT_NONE, y, d * 4, B.FG_F32, mean, rstd, ws, len(ws))
        torch.cuda.synchronize()
        taken = torch.zeros(n, dtype=torch.bool)
        for g, pos, _ in R.members(order, offsets.tolist(), n):
            taken[pos] = True
            m, s = R.norm_statistics(x[pos], blocks, 0.25)
            # fp64 sums of at most 2^26 distances of up to 2^6 (or equal values): 2^-53 * 2^6 * 2^26 of the mean at most
            close(mean.cpu()[g], m, 2.0 ** -24 * m.abs() + 2.0 ** -21, f"mean of group {g} about {level}")
            close(rstd.cpu()[g], s, 2.0 ** -23 * s, f"rstd of group {g} about {level}")
            if len(pos):
                want, tol, _, _ = R.norm_rows(x[pos], m, s, None, None, "none")
                close(y.cpu()[pos], want, tol + 2.0 ** -24 * want.abs(), "y")
        assert bool((y.cpu()[~taken] == -77).all())
        if spread == 0:
            assert not bool(y.cpu()[taken].any()) and bool((rstd == 2).all())


@gpu
@pytest.mark.parametrize("n, d", [(100, 16), (50_000, 64)])
def test_a_group_none_of_whose_entries_exists(B, n, d):
    order = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    off = torch.tensor([0, n // 2, n], device="cuda")
    order[n // 2:] = torch.arange(n // 2, n, device="cuda")
    x, y, mean, rstd = torch.randn(n, d, device="cuda") + 5, full(n, d), full(2, 4), full(2, 4)
    ws = torch.zeros(B.fg_group_norm_workspace_bytes(n, 2, d, 4), dtype=torch.uint8, device="cuda")
    B.fg_group_norm(x, d * 4, B.FG_F32, order, off, n, 2, n, d, 4, None, None, 0.25, B.FG_ACT_NONE, y, d * 4, B.FG_F32, mean, rstd, ws, len(ws))
    torch.cuda.synchronize()
    assert bool((mean[0] == 0).all()) and bool((rstd[0] == 2).all()) and bool((y[:n // 2] == -77).all()) and bool((mean[1] > 4).all()) and not bool((y[n // 2:] == -77).any())


# ---- long sums ----

@gpu
@pytest.mark.parametrize("n, n_groups, d, blocks", [(16_400_000, 1, 256, 256), (16_400_000, 2, 256, 8), (8_200_000, 1, 512, 1), (2_050_000, 1, 4096, 1), (16_000_000, 100_000, 512, 1)])
def test_gradients_of_groups_whose_threads_have_thousands_of_rows(B, n, n_groups, d, blocks):
    """Terms that are all the same within a column: fp32 sums that went on for 2000 of them would be off by up to 2000 / 2^25 of the sum, always to one side."""
    g = torch.Generator().manual_seed(d)
    w, b = (0.5 + torch.rand(d, generator=g) for _ in range(2))
    off = torch.linspace(0, n, n_groups + 1, dtype=torch.float64).long().cuda()
    x = torch.ones(n, d, dtype=torch.bfloat16, device="cuda")
    dy = torch.empty_like(x)
    ws = torch.empty(B.fg_group_norm_backward_workspace_bytes(n, n_groups, d, blocks), dtype=torch.uint8, device="cuda")
    rstd = torch.ones(n_groups, blocks, device="cuda")
    wd, bd = w.cuda(), b.cuda()
    u = 2.0 ** -24
    # up to 128 rows of a thread in fp32, 8 sums over lanes, the joins' rounding, and what 2000 / 128 sums of those lose in fp32 (rows of more than 2048 columns)
    steps = 128 + 8 + 4 + 16
    for level in (0.0, 1.0):      # xh is 1 or 0
        dy.fill_(1)
        dw, db, mean = full(d), full(d), torch.full((n_groups, blocks), level, device="cuda")
        B.fg_group_norm_backward(dy, 2 * d, B.FG_BF16, x, 2 * d, B.FG_BF16, mean, rstd, wd, bd, B.FG_ACT_SILU, None, off, n, n_groups, n, d, blocks, dy, 2 * d, dw, db, ws, len(ws))
        torch.cuda.synchronize()
        xh = 1.0 - level
        arg = w.double() * xh + b.double()
        t = R.slope("silu", arg)
        t_off = R.slope_off("silu", arg) + 0.5 * 4 * u * arg.abs() + u * t
        close(db.cpu(), n * t, n * (t_off + steps * u * t), f"db, xh {xh}")
        close(dw.cpu(), n * t * xh, xh * n * (t_off + steps * u * t), f"dw, xh {xh}")
        tw, tw_off = (t * w.double()).view(blocks, -1), ((t_off + u * t) * w.double()).view(blocks, -1)
        m1 = tw.mean(1, keepdim=True)
        want = (tw - m1 - xh * xh * m1).flatten()
        tolerance = (tw_off + (1 + xh) * (tw_off.mean(1, keepdim=True) + steps * u * m1) + 8 * u * (tw + 2 * m1)).flatten() + HALF["bf16"] * want.abs()
        for rows in (dy[:64], dy[n // 2:n // 2 + 64], dy[-64:]):
            close(rows.cpu(), want.expand(64, -1), tolerance.expand(64, -1), f"dx, xh {xh}")


# ---- the loss ----

@gpu
@pytest.mark.parametrize("lead", [0, 1])
@pytest.mark.parametrize("dtype, d", [("f32", 600), ("f32", 3000), ("f32", 20_000), ("f32", 140_000), ("bf16", 1000), ("bf16", 50_000)])
def test_sums_of_wide_rows_to_the_last_step(B, dtype, d, lead):
    """One class of 1 and groups of classes that come to just under half a step of 1 each: added to it in fp32 one after the other, every one of them is lost. The largest class's share
    is 1 / sum: half a step for the sum in fp32 (2^-24 above 1), half for the quotient (2^-25 below 1), and what the exponentials of the small ones are off."""
    n, rows = 64, d + 5
    want = []
    h = torch.full((n, rows), -math.inf, dtype=T[dtype])
    r = np.random.default_rng(d)
    for i in range(n):
        top = int(r.integers(0, d))
        h[i, lead + top] = 0
        groups = [r.integers(0, d, 2 ** int(r.integers(0, 5))) for _ in range(7)]
        for at in groups:
            h[i, lead + at] = torch.tensor(math.log(0.96 * 2.0 ** -24 / len(at)), dtype=torch.float64).to(T[dtype])
        h[i, lead + top] = 0
        want.append((top, float(torch.exp(h[i, lead:lead + d].double()).sum())))
    hd = h.cuda()
    dh = full(n, d)
    label = torch.tensor([(top + 1) % d for top, _ in want], dtype=torch.int32, device="cuda")
    e = T[dtype].itemsize
    B.fg_distill_loss(hd.data_ptr() + lead * e, rows * e, code(B, dtype), None, None, n, n, d, None, None, None, B.FG_F32, 0, 0, label, 1.0, 0.0, None, 1.0, None, dh, 4 * d, B.FG_F32)
    torch.cuda.synchronize()
    for i, (top, total) in enumerate(want):
        got = float(dh[i, top])
        # (the exponentials: 7 * 2^-24 of them, each to 2^-18 of itself)
        assert abs(got - 1 / total) <= (2.0 ** -24 + 2.0 ** -25 + 2.0 ** -38) / total, (i, got, 1 / total)


@gpu
@pytest.mark.parametrize("dtype, d, bound", [("f32", 40, 0), ("f32", 120, 0), ("bf16", 256, 0), ("f32", 500, 0), ("f16", 1500, 0), ("bf16", 3000, 0), ("f32", 3000, 20_000), ("bf16", 8000, 5000), ("f32", 20_000, 0),
                                             ("bf16", 90_000, 0)])
def test_shares_of_one_class_are_added_in_the_entries_order(B, dtype, d, bound):
    """The entries' shares as a row of different classes shows them, each by itself where no logit can be chosen; then rows whose entries share classes: the fp32 sums of
    those shares, one after the other, to the bit, and the label's behind them."""
    n, k, r = 40, 50, np.random.default_rng(d)
    k = min(k, d - 1)
    h = torch.full((n, d), -math.inf, dtype=T[dtype])
    h[:, d - 1] = 0      # the one class that can be
    val = (3 * torch.randn(1, k, generator=torch.Generator().manual_seed(d))).repeat(n, 1)
    idx = np.empty((n, k), np.int32)
    for i in range(n):      # row 0: all different; the others: more and more alike
        idx[i] = r.permutation(d - 1)[:k] if i == 0 else r.integers(0, d - 1, max(1, k - i))[r.integers(0, max(1, k - i), k)]
    idx[3] = idx[3, 0]
    label = np.full(n, -1, np.int32)
    label[4::3] = idx[4::3, 7]
    rows = torch.full((max(bound, n),), -1, dtype=torch.int32, device="cuda")
    rows[:n] = torch.arange(n)
    count = torch.full((1,), n, device="cuda")
    dev = h.cuda(), torch.from_numpy(idx).cuda(), val.cuda(), torch.from_numpy(label).cuda()

    def call(label):
        dh = full(n, d)
        B.fg_distill_loss(dev[0], stride(h), code(B, dtype), rows, count, len(rows), n, d, None, dev[1], dev[2], B.FG_F32, n, k, label, 1.0, 0.75, None, 1.0, None, dh, 4 * d, B.FG_F32)
        torch.cuda.synchronize()
        return dh.cpu().numpy()

    plain = call(None)
    share = -plain[0, idx[0]]
    assert (share > 0).all() and abs(float(share.astype(np.float64).sum()) - 0.75) < 1e-5
    got = call(dev[3])
    for i in range(1, n):
        want = np.zeros(d, np.float32)
        for j in range(k):
            want[idx[i, j]] += share[j]
        assert np.array_equal(plain[i, :d - 1], -want[:d - 1]), i
        if label[i] >= 0:
            want[label[i]] += np.float32(0.25)
        assert np.array_equal(got[i, :d - 1], -want[:d - 1]), i
    for _ in range(3):
        assert np.array_equal(call(dev[3]), got)


def distill_case(B, dtype, dh_type, n, d, k, bound, pad, seed, temp=2.0, alpha=0.6, over=False):
    """n rows of a list whose bound is `bound`, a count on the device; against the statement."""
    r = np.random.default_rng(seed)
    h = values(r, n, d, dtype, pad, 3.0)
    idx = np.stack([r.permutation(d)[:k] for _ in range(n)]).astype(np.int32)
    idx[r.random(idx.shape) < 0.1] = -1
    idx[::3, 1] = idx[::3, 0]
    idx[1], idx[2, 0] = -1, d - 1
    val = torch.from_numpy(4 * r.standard_normal((n, k))).to(torch.float16)
    label = r.integers(-1, d, n).astype(np.int32)
    label[1], label[2] = -1, d - 1
    h[4, :d] = -math.inf      # no class to choose
    label[4] = 0
    h[5, :d] = -math.inf
    idx[5], label[5] = -1, -1
    h[6, 0] = math.nan
    rows = torch.full((bound,), -1, dtype=torch.int32)
    order = r.permutation(n).astype(np.int32)
    rows[:n] = torch.from_numpy(order)
    hd, loss, dh = h.cuda(), full(n), sentinel(n, d, dh_type, pad).cuda()
    out = hd if over else dh
    B.fg_distill_loss(hd, stride(hd), code(B, dtype), rows.cuda(), torch.full((1,), n, device="cuda"), bound, n, d, None, torch.from_numpy(idx).cuda(), val.cuda(), B.FG_F16, n, k,
                      torch.from_numpy(label).cuda(), temp, alpha, None, 0.5, loss, out, stride(out), code(B, dh_type))
    torch.cuda.synchronize()
    loss, got = loss.cpu(), out.cpu()
    assert bool((dh.cpu()[:, d:] == -77).all()) and (not over or bool(torch.isnan(got[:, d:]).all()))
    for i in (4, 6):
        if i == 4 or label[6] >= 0 or (idx[6] >= 0).any():
            assert bool(torch.isnan(loss[i])) and bool(torch.isnan(got[i, :d]).all()), i
    for i in (1, 5):
        assert float(loss[i]) == 0 and not bool(got[i, :d].any())
    rest = [i for i in range(n) if i not in (4, 6)]
    want, off, grad, grad_off = R.distill(h[rest, :d], torch.from_numpy(idx[rest]), val[rest], label[rest], temp, alpha, None, 0.5)
    close(loss[rest], want, off + 2.0 ** -24 * want.abs(), "loss")
    close(got[rest, :d], grad, grad_off + HALF[dh_type] * grad.abs() + TINY[dh_type], "dh")


@gpu
@pytest.mark.parametrize("over", [False, True])
@pytest.mark.parametrize("dtype, d, bound, pad", [("f32", 2100, 5000, 0), ("f32", 4000, 5000, 3), ("f32", 4080, 17_000, 1), ("f32", 2500, 17_000, 5), ("bf16", 3000, 17_000, 1), ("bf16", 4081, 17_000, 3),
                                                   ("bf16", 5000, 5000, 0), ("bf16", 8000, 5000, 3), ("f16", 8176, 20_000, 5), ("f16", 4100, 4097, 2)])
def test_wide_rows_one_to_a_wavefront(B, dtype, d, bound, pad, over):
    """More rows may be listed than rows of one wavefront need: those of up to 4088 columns, in 16 bits 8184, at strides that are no multiples of a line."""
    distill_case(B, dtype, dtype, 12, d, 30, bound, pad, d, over=over)


@gpu
@pytest.mark.parametrize("temp", [1.0, 2.5, 4.0])
def test_wide_rows_one_to_a_wavefront_at_other_temperatures(B, temp):
    distill_case(B, "bf16", "f32", 10, 6001, 64, 4500, 1, 7, temp, 1.0)
    distill_case(B, "f32", "f32", 10, 3001, 64, 4500, 1, 8, temp, 0.0)


# ---- far arguments, infinities, NaN ----

def far_arguments(name, count):
    """Arguments of an activation: near zero, through its bend, into both tails to where they leave fp32, and the largest numbers."""
    u = torch.cat([torch.linspace(-20, 20, count // 2), torch.linspace(-120, 120, count // 4), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 2.0 ** -126, 1e-40, -1e-40, 1e30, -1e30, 3e38, -3e38]),
                   torch.linspace(-104, -86, 40), torch.linspace(86, 104, 40), torch.linspace(-15, -12, 60)])
    return torch.cat([u, torch.linspace(-1, 1, count - len(u))])


def act_at(name, u):
    """R.act, with the lower tail of the normal distribution function as it is (1 + erf(x) leaves nothing of it below -8)."""
    return u * 0.5 * torch.special.erfc(-u * math.sqrt(0.5)) if name == "gelu" else R.act(name, u)


def far_off(name, u):
    """act_off and slope_off; beyond where a tail has left fp32 an argument's size adds nothing: act(u) is u or 1 there, and its slope 1 or 0."""
    near = u.double().clamp(-104, 104) if name != "gelu" else u.double().clamp(-15, 15)
    steps = (16 + near.abs() + (near * near if name == "gelu" else 0)) * 2.0 ** -24
    f = act_at(name, u.double()).abs()
    return (f * steps if name not in ("none", "relu") else 0 * f) + 2.0 ** -100, R.slope_off(name, near) + 0 * f


def slope_at(name, u):
    if name != "gelu" and name != "silu":
        return R.slope(name, u)
    return torch.where(u.abs() > 200, (u > 0).double(), R.slope(name, u.clamp(-200, 200)))      # (0 * infinity in the statement)


@gpu
@pytest.mark.parametrize("name", R.ACTS)
@pytest.mark.parametrize("rows", [3, 40_000])
def test_far_arguments_of_the_gated_layer(B, name, rows):
    """z is the bias (x is 0), the other projection 1: h is the activation, and with dh = 1 db is its slope. Few rows and many, which are kernels of their own."""
    b, a = 2048, 8
    u = far_arguments(name, b)
    bias = torch.cat([u, torch.ones(b)])[None]
    x, W = torch.zeros(rows, a, device="cuda"), torch.ones(1, a, 2 * b, device="cuda")
    h, z, off = torch.empty(rows, b, device="cuda"), torch.empty(rows, 2 * b, device="cuda"), torch.tensor([0, rows], device="cuda")
    B.fg_gated_linear_grouped(x, rows, 4 * a, B.FG_F32, None, None, off, rows, 1, a, b, W, bias.cuda(), act_code(B, name), h, rows, 4 * b, B.FG_F32, z, 8 * b)
    f_off, s_off = far_off(name, u)
    for r in (0, rows - 1):
        assert torch.equal(z[r].cpu() + 0.0, bias[0] + 0.0)
        close(h[r].cpu(), act_at(name, u.double()), f_off, "h")
    assert torch.equal(h[1:], h[:1].expand(rows - 1, -1))
    need = B.fg_gated_linear_grouped_backward_workspace_bytes(B.FG_F32, 1, 1, a, b)
    ws, db, one = torch.empty(need, dtype=torch.uint8, device="cuda"), full(1, 2 * b), torch.tensor([0, 1], device="cuda")
    B.fg_gated_linear_grouped_backward(x, rows, 4 * a, B.FG_F32, None, torch.ones(rows, b, device="cuda"), 4 * b, B.FG_F32, z, 8 * b, rows, None, one, 1, 1, a, b, W, act_code(B, name), None, 0,
                                       B.FG_F32, None, B.FG_F32, db, ws, need)
    torch.cuda.synchronize()
    s = torch.where(u == 0, torch.zeros(()).double(), slope_at(name, u.double())) if name == "relu" else slope_at(name, u.double())
    close(db[0, :b].cpu(), s, s_off, "slope")
    close(db[0, b:].cpu(), act_at(name, u.double()), f_off, "act")


@gpu
@pytest.mark.parametrize("name", R.ACTS)
@pytest.mark.parametrize("rows, blocks", [(5, 64), (5, 1), (3000, 64)])
def test_far_arguments_of_the_group_norm(B, name, rows, blocks):
    """Rows that are all alike: y is the activation of the bias, db the rows' number times its slope."""
    d = 2048
    u = far_arguments(name, d)
    x, y, off = torch.full((rows, d), 3.0, device="cuda"), torch.empty(rows, d, device="cuda"), torch.tensor([0, rows], device="cuda")
    mean, rstd, bias = full(1, blocks), full(1, blocks), u.cuda()
    ws = torch.empty(B.fg_group_norm_backward_workspace_bytes(rows, 1, d, blocks), dtype=torch.uint8, device="cuda")
    B.fg_group_norm(x, 4 * d, B.FG_F32, None, off, rows, 1, rows, d, blocks, None, bias, 0.25, act_code(B, name), y, 4 * d, B.FG_F32, mean, rstd, ws, len(ws))
    dx, dw, db = full(rows, d), full(d), full(d)
    B.fg_group_norm_backward(torch.ones_like(x), 4 * d, B.FG_F32, x, 4 * d, B.FG_F32, mean, rstd, None, bias, act_code(B, name), None, off, rows, 1, rows, d, blocks, dx, 4 * d, dw, db, ws,
                             len(ws))
    torch.cuda.synchronize()
    assert bool((mean == 3).all()) and bool((rstd == 2).all()) and bool((dw == 0).all()) and bool(torch.isfinite(dx).all())
    f_off, s_off = far_off(name, u)
    close(y[0].cpu(), act_at(name, u.double()), f_off, "y")
    assert torch.equal(y, y[:1].expand(rows, -1))
    s = slope_at(name, u.double())
    close(db.cpu(), rows * s, rows * (s_off + 160 * 2.0 ** -24 * s.abs()) + 2.0 ** -100, "db")


@gpu
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n, a, b", [(9, 64, 40), (40_000, 72, 264)])
def test_the_gated_layer_keeps_what_is_not_finite_in_its_row(B, dtype, n, a, b, bad):
    c, e = code(B, dtype), T[dtype].itemsize
    g = torch.Generator(device="cuda").manual_seed(n)
    kw = dict(device="cuda", generator=g)
    x, W = torch.randn(n, a, **kw).to(T[dtype]), (torch.randn(2, a, 2 * b, **kw) / 8).to(T[dtype])
    dh, off = torch.randn(n, b, **kw).to(T[dtype]), torch.tensor([0, n // 3, n], device="cuda")
    need = B.fg_gated_linear_grouped_backward_workspace_bytes(c, n, 2, a, b)

    def run(x, dh, z=None):
        h, own_z = torch.empty(n, b, dtype=T[dtype], device="cuda"), torch.empty(n, 2 * b, dtype=T[dtype], device="cuda")
        B.fg_gated_linear_grouped(x, n, a * e, c, None, None, off, n, 2, a, b, W, None, B.FG_ACT_SILU, h, n, b * e, c, own_z, 2 * b * e)
        z = own_z if z is None else z
        dx, dw, db = torch.empty(n, a, dtype=T[dtype], device="cuda"), full(2, a, 2 * b), full(2, 2 * b)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        B.fg_gated_linear_grouped_backward(x, n, a * e, c, None, dh, b * e, c, z, 2 * b * e, n, None, off, n, 2, a, b, W, B.FG_ACT_SILU, dx, a * e, c, dw, B.FG_F32, db, ws, need)
        torch.cuda.synchronize()
        return h, dx, dw, db, z

    want = run(x, dh)
    row = n // 3 + 2      # of the second group
    others = torch.arange(n, device="cuda") != row
    xb, dhb = x.clone(), dh.clone()
    xb[row, 5], dhb[row, 7] = bad, bad
    h, dx, dw, db, _ = run(xb, dhb, want[4])      # (the gradients with the projections of the rows as they were)
    assert not bool(torch.isfinite(h[row]).any()) and not bool(torch.isfinite(dx[row]).any())
    assert torch.equal(h[others], want[0][others]) and torch.equal(dx[others], want[1][others])
    assert torch.equal(dw[0], want[2][0]) and torch.equal(db[0], want[3][0])
    bad_columns = torch.zeros(2 * b, dtype=torch.bool, device="cuda")
    bad_columns[[7, b + 7]] = True
    assert not bool(torch.isfinite(db[1][bad_columns]).any()) and torch.equal(db[1][~bad_columns], want[3][1][~bad_columns])
    assert not bool(torch.isfinite(dw[1][:, bad_columns]).any()) and not bool(torch.isfinite(dw[1][5]).any())
    there = torch.arange(a, device="cuda") != 5
    assert torch.equal(dw[1][there][:, ~bad_columns], want[2][1][there][:, ~bad_columns])


@gpu
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype, n, n_groups, d, blocks", [("f32", 300, 3, 88, 8), ("bf16", 50_000, 3, 256, 8), ("f32", 30_000, 2, 512, 1), ("f16", 600, 30, 96, 96), ("bf16", 300, 2, 4096, 1),
                                                         ("f32", 4000, 1000, 40, 2)])
def test_the_group_norm_keeps_what_is_not_finite_in_its_block(B, dtype, n, n_groups, d, blocks, bad):
    c, e = code(B, dtype), T[dtype].itemsize
    g = torch.Generator(device="cuda").manual_seed(n)
    kw = dict(device="cuda", generator=g)
    x, dy, off = torch.randn(n, d, **kw).to(T[dtype]), torch.randn(n, d, **kw).to(T[dtype]), torch.linspace(0, n, n_groups + 1, dtype=torch.float64).long().cuda()
    ws = torch.empty(B.fg_group_norm_backward_workspace_bytes(n, n_groups, d, blocks), dtype=torch.uint8, device="cuda")
    mean, rstd = torch.zeros(n_groups, blocks, device="cuda"), torch.ones(n_groups, blocks, device="cuda")

    def run(x, dy):
        y, m, r, dx, dw, db = torch.empty_like(x), full(n_groups, blocks), full(n_groups, blocks), torch.empty_like(x), full(d), full(d)
        B.fg_group_norm(x, d * e, c, None, off, n, n_groups, n, d, blocks, None, None, 1e-5, B.FG_ACT_SILU, y, d * e, c, m, r, ws, len(ws))
        B.fg_group_norm_backward(dy, d * e, c, x, d * e, c, mean, rstd, None, None, B.FG_ACT_SILU, None, off, n, n_groups, n, d, blocks, dx, d * e, dw, db, ws, len(ws))
        torch.cuda.synchronize()
        return y, m, r, dx, dw, db

    good = run(x, dy)
    group, column = n_groups - 1, d - 3
    block, size = column // (d // blocks), d // blocks
    for row in (int(off[group]), int(off[group]) + int(off[group + 1] - off[group]) // 2):      # the group's first, whose values are the level; another
        for of_x in (True, False):
            xb, dyb = x.clone(), dy.clone()
            (xb if of_x else dyb)[row, column] = bad
            y, m, r, dx, dw, db = run(xb, dyb)
            inside = torch.zeros(n, d, dtype=torch.bool, device="cuda")
            inside[off[group]:off[group + 1], block * size:(block + 1) * size] = True
            one = torch.zeros(d, dtype=torch.bool, device="cuda")
            one[column] = True
            if of_x:
                assert not bool(torch.isfinite(y[inside]).any()) and not bool(torch.isfinite(r[group, block])) and not bool(torch.isfinite(m[group, block]))
                m[group, block], r[group, block] = good[1][group, block], good[2][group, block]
            else:
                assert torch.equal(y, good[0])
            assert torch.equal(y[~inside], good[0][~inside]) and torch.equal(m, good[1]) and torch.equal(r, good[2])
            assert torch.equal(dx[~inside], good[3][~inside]) and torch.equal(dw[~one], good[4][~one]) and torch.equal(db[~one], good[5][~one])
            assert not bool(torch.isfinite(dx[inside]).any()) and not bool(torch.isfinite(dw[column])), (row, of_x)


def test_temperatures_beyond_what_fp32_can_square(B):
    """1e-39 gave NaN (0 times the infinite reciprocal), 1e20 an infinite loss."""
    for t in (1e-39, 2.0 ** -61, 1e20, 2.0 ** 61, 0.0, -1.0, math.inf, math.nan):
        assert refused(B, B.fg_distill_loss, P, 256, B.FG_F32, None, None, 10, 10, 64, None, P, P, B.FG_F16, 10, 4, None, t, 0.5, None, 1.0, P, P + 4096, 256, B.FG_F32) == B.FG_ERR_INVALID_ARG, t


@gpu
@pytest.mark.parametrize("d", [40, 600, 9000])
def test_the_least_and_the_largest_temperature(B, d):
    """At 2^-60 the softmax is the largest logit's alone, at 2^60 all classes are alike."""
    h = torch.zeros(1, d)
    h[0, 3] = 1.0
    idx, val = torch.tensor([[3, 7]], dtype=torch.int32, device="cuda"), torch.tensor([[1.0, 0.0]], device="cuda")
    for t, q, p in ((2.0 ** -60, 1.0, (1.0, 0.0)), (2.0 ** 60, 1.0 / d, (0.5, 0.5))):
        loss, dh = full(1), full(1, d)
        B.fg_distill_loss(h.cuda(), 4 * d, B.FG_F32, None, None, 1, 1, d, None, idx, val, B.FG_F32, 1, 2, None, t, 1.0, None, 1.0, loss, dh, 4 * d, B.FG_F32)
        torch.cuda.synchronize()
        got = dh.cpu().double()[0] / t
        want = torch.full((d,), 0.0 if t < 1 else 1.0 / d, dtype=torch.float64)
        want[3] = q
        want[3] -= p[0]
        want[7] -= p[1]
        assert bool(torch.isfinite(loss).all()) and bool(((got - want).abs() <= 2.0 ** -20).all()), t
