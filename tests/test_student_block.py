"""The calls of a student's block (fg_gated_linear_grouped, fg_group_norm and their gradients, fg_distill_loss) against plain 64-bit statements of them,
at the sizes and masks where they can go wrong.

Tolerances are those of `student_reference`: a sum of K products in fp32 is off by at most K steps of 2^-24 of the products' magnitudes, twice that is
granted (the matrix cores' sums need not round to nearest); what a function makes of a value that is off goes by its largest slope; a
result rounded to a type is off by half a step of it besides (`HALF`)."""
import math

import numpy as np
import pytest
import torch

from tests import student_reference as R

T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -25, "bf16": 2.0 ** -126}      # half the distance of the smallest fp16 numbers; below the smallest normal ones
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2301_07482_amd import binding
    return binding


def code(B, name):
    return {"f32": B.FG_F32, "f16": B.FG_F16, "bf16": B.FG_BF16}[name]


def act_code(B, name):
    return {"none": B.FG_ACT_NONE, "relu": B.FG_ACT_RELU, "silu": B.FG_ACT_SILU, "gelu": B.FG_ACT_GELU, "sigmoid": B.FG_ACT_SIGMOID}[name]


def cuda(t):
    return t.cuda() if t is not None else None


def values(r, n, d, dtype, pad=0, scale=1.0, level=0.0):
    """[n, d] values in rows that are `pad` longer (NaN there, which nothing may read into a result)."""
    full = torch.full((n, d + pad), float("nan"), dtype=T[dtype])
    full[:, :d] = torch.from_numpy(r.standard_normal((n, d)) * scale + level).to(T[dtype])
    return full


def sentinel(n, d, dtype, pad=0):
    return torch.full((n, d + pad), -77.0, dtype=T[dtype])


def close(got, want, tolerance, what):
    off = (got.double() - want).abs()
    bad = ~((off <= tolerance) | (got.double() == want))
    assert not bool(bad.any()), f"{what}: off by {float(off[bad].max()):.3e} where {float(tolerance[bad].min()):.3e} is allowed, {int(bad.sum())} values"


def stride(t):
    return t.stride(0) * t.element_size()


def refused(B, fn, *a, **k):
    with pytest.raises(B.FgError) as e:
        fn(*a, **k)
    assert B.fg_last_error() != ""
    return e.value.code


# ---- refusals: on the host, before anything is launched ----

def test_gated_refusals(B):
    P = 4096
    lin = lambda **k: B.fg_gated_linear_grouped(**{**dict(x=P, x_rows=10, x_stride=256, dtype=B.FG_F32, src_ids=None, order=P, offsets=P, max_rows=10, n_groups=4,
                                                          d_in=64, d_out=32, W=P, bias=None, act=B.FG_ACT_SILU, h_out=P, n_out=10, out_stride=128,
                                                          out_dtype=B.FG_F32, z_out=None, z_stride=0), **k})
    for bad, want in ((dict(x=None), 1), (dict(W=None), 1), (dict(h_out=None), 1), (dict(offsets=None), 1), (dict(offsets=P + 4), 1), (dict(order=P + 2), 1),
                      (dict(n_groups=0), 1), (dict(n_groups=1025), 1), (dict(max_rows=-1), 1), (dict(max_rows=B.FG_MAX_GROUPED_ROWS + 1, n_out=1 << 30), 1),
                      (dict(x_rows=-1), 1), (dict(n_out=1 << 31), 1), (dict(d_in=62), 2), (dict(d_in=0), 2), (dict(d_out=30), 2), (dict(d_out=0), 2),
                      (dict(d_out=B.FG_MAX_GROUPED_DIM // 2 + 4, out_stride=1 << 20), 2), (dict(d_in=B.FG_MAX_GROUPED_DIM + 4, x_stride=1 << 20), 2),
                      (dict(x_stride=128), 2), (dict(out_stride=112), 2), (dict(z_out=P, z_stride=240), 2), (dict(z_out=P + 8, z_stride=256), 1), (dict(x=P + 4), 1),
                      (dict(W=P + 8), 1), (dict(h_out=P + 4), 1), (dict(x_stride=264), 1), (dict(bias=P + 2), 1), (dict(src_ids=P + 1), 1), (dict(dtype=7), 3),
                      (dict(dtype=B.FG_E4M3), 3), (dict(out_dtype=B.FG_BF16), 3), (dict(dtype=B.FG_BF16, out_dtype=B.FG_F16), 3),
                      (dict(dtype=B.FG_BF16, d_out=36), 2), (dict(act=5), 1), (dict(act=-1), 1)):
        assert refused(B, lin, **bad) == want, bad
    bw = lambda **k: B.fg_gated_linear_grouped_backward(**{**dict(x=P, x_rows=10, x_stride=256, dtype=B.FG_F32, src_ids=None, dh=P, dh_stride=128, dh_dtype=B.FG_F32,
                                                                  z=P, z_stride=256, n=10, order=P, offsets=P, max_rows=10, n_groups=4, d_in=64, d_out=32, W=P,
                                                                  act=B.FG_ACT_SILU, dx=P, dx_stride=256, dx_dtype=B.FG_F32, dw=P, dw_dtype=B.FG_F32, db=P,
                                                                  ws=P, ws_bytes=1 << 40), **k})
    for bad, want in ((dict(x=None), 1), (dict(dh=None), 1), (dict(z=None), 1), (dict(W=None), 1), (dict(dx=None, dw=None, db=None), 1), (dict(ws=None), 1), (dict(ws=P + 4), 1),
                      (dict(ws_bytes=0), 2), (dict(dtype=B.FG_E4M3), 3), (dict(dh_dtype=B.FG_BF16), 3), (dict(dx_dtype=B.FG_F16), 3), (dict(dw_dtype=B.FG_F16), 3),
                      (dict(d_in=2), 2), (dict(d_out=2), 2), (dict(dh_stride=112), 2), (dict(z_stride=128), 2), (dict(dx_stride=16), 2), (dict(dw=P + 4), 1),
                      (dict(db=P + 8), 1), (dict(n_groups=2000), 1), (dict(act=9), 1), (dict(offsets=None), 1), (dict(z=P + 4), 1)):
        assert refused(B, bw, **bad) == want, bad
    need = B.fg_gated_linear_grouped_backward_workspace_bytes
    assert need(B.FG_E4M3, 10, 4, 64, 64) == 0 and need(B.FG_F32, -1, 4, 64, 64) == 0 and need(B.FG_F32, 10, 4, 64, B.FG_MAX_GROUPED_DIM) == 0
    assert refused(B, bw, ws_bytes=need(B.FG_F32, 10, 4, 64, 32) - 1) == 2


def test_group_norm_refusals(B):
    P = 4096
    norm = lambda **k: B.fg_group_norm(**{**dict(x=P, x_stride=256, dtype=B.FG_F32, order=None, offsets=P, max_rows=10, n_groups=4, n=10, d=64, channel_groups=8, weight=None,
                                                 bias=None, eps=1e-5, act=B.FG_ACT_SILU, y=P + 4096, y_stride=256, y_dtype=B.FG_F32, mean_out=None, rstd_out=None, ws=P,
                                                 ws_bytes=1 << 40), **k})
    for bad, want in ((dict(x=None), 1), (dict(y=None), 1), (dict(offsets=None), 1), (dict(offsets=P + 4), 1), (dict(order=P + 2), 1), (dict(ws=None), 1), (dict(ws=P + 8), 1),
                      (dict(ws_bytes=8), 2), (dict(max_rows=-1), 1), (dict(max_rows=1 << 31), 1), (dict(n=-1), 1), (dict(n_groups=0), 1), (dict(n_groups=B.FG_MAX_NORM_GROUPS + 1), 1),
                      (dict(d=0), 2), (dict(d=7, channel_groups=1), 2), (dict(d=B.FG_MAX_NORM_DIM + 1, channel_groups=1, x_stride=1 << 20, y_stride=1 << 20), 2), (dict(channel_groups=0), 2),
                      (dict(channel_groups=7), 2), (dict(channel_groups=128), 2), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(act=5), 1), (dict(dtype=3), 3),
                      (dict(y_dtype=B.FG_BF16), 3), (dict(y_dtype=3), 3), (dict(x_stride=252), 2), (dict(y_stride=16), 2), (dict(x=P + 2), 1), (dict(y=P + 1), 1),
                      (dict(weight=P + 2), 1), (dict(bias=P + 1), 1), (dict(mean_out=P + 1), 1), (dict(rstd_out=P + 2), 1), (dict(y=P, y_stride=512), 1),
                      (dict(dtype=B.FG_BF16, y=P, y_dtype=B.FG_F32), 1)):
        assert refused(B, norm, **bad) == want, bad
    bw = lambda **k: B.fg_group_norm_backward(**{**dict(dy=P, dy_stride=256, grad_dtype=B.FG_F32, x=P, x_stride=256, dtype=B.FG_F32, mean=P, rstd=P, weight=None, bias=None,
                                                        act=B.FG_ACT_SILU, order=None, offsets=P, max_rows=10, n_groups=4, n=10, d=64, channel_groups=8, dx=P + 4096,
                                                        dx_stride=256, dw=P, db=P, ws=P, ws_bytes=1 << 40), **k})
    for bad, want in ((dict(dy=None), 1), (dict(x=None), 1), (dict(mean=None), 1), (dict(rstd=None), 1), (dict(dx=None), 1), (dict(offsets=None), 1), (dict(ws=None), 1),
                      (dict(ws_bytes=64), 2), (dict(grad_dtype=3), 3), (dict(grad_dtype=B.FG_BF16), 3), (dict(dtype=4), 3), (dict(channel_groups=5), 2), (dict(dy_stride=4), 2), (dict(dx_stride=128), 2),
                      (dict(dw=P + 1), 1), (dict(mean=P + 2), 1), (dict(dx=P, dx_stride=512), 1), (dict(act=-2), 1), (dict(n_groups=-1), 1)):
        assert refused(B, bw, **bad) == want, bad
    for need in (B.fg_group_norm_workspace_bytes, B.fg_group_norm_backward_workspace_bytes):
        assert need(-1, 4, 64, 8) == 0 and need(10, 0, 64, 8) == 0 and need(10, 4, 64, 7) == 0 and need(10, 4, B.FG_MAX_NORM_DIM * 2, 1) == 0
    assert refused(B, norm, ws_bytes=B.fg_group_norm_workspace_bytes(10, 4, 64, 8) - 1) == 2
    assert refused(B, bw, ws_bytes=B.fg_group_norm_backward_workspace_bytes(10, 4, 64, 8) - 1) == 2


def test_distill_refusals(B):
    P = 4096
    loss = lambda **k: B.fg_distill_loss(**{**dict(h=P, h_stride=256, dtype=B.FG_F32, rows=None, n_rows=None, max_rows=10, n=10, d=64, ids=None, top_idx=P, top_val=P,
                                                   top_dtype=B.FG_F16, table_rows=10, k=4, labels=None, temperature=2.0, alpha=0.5, weight=None, grad_scale=1.0,
                                                   loss_out=P, dh=P + 4096, dh_stride=256, dh_dtype=B.FG_F32), **k})
    for bad, want in ((dict(h=None), 1), (dict(top_idx=None), 1), (dict(top_val=None), 1), (dict(loss_out=None, dh=None), 1), (dict(max_rows=-1), 1), (dict(max_rows=11), 2),
                      (dict(n=1 << 31, rows=P), 1), (dict(d=0), 2), (dict(d=B.FG_MAX_CLASSES + 1, h_stride=1 << 34, dh_stride=1 << 34), 2), (dict(k=-1), 2), (dict(k=B.FG_MAX_TOP + 1), 2), (dict(table_rows=-1), 1), (dict(table_rows=1 << 31), 1),
                      (dict(temperature=0.0), 1), (dict(temperature=-1.0), 1), (dict(temperature=float("nan")), 1), (dict(temperature=float("inf")), 1),
                      (dict(alpha=-0.1), 1), (dict(alpha=1.5), 1), (dict(alpha=float("nan")), 1), (dict(dtype=3), 3), (dict(top_dtype=3), 3), (dict(dh_dtype=B.FG_BF16), 3),
                      (dict(h_stride=252), 2), (dict(dh_stride=128), 2), (dict(h=P + 2), 1), (dict(dh=P + 1), 1), (dict(dh=P, dh_stride=512), 1),
                      (dict(dtype=B.FG_BF16, dh=P, dh_dtype=B.FG_F32), 1), (dict(ids=P + 2), 1), (dict(labels=P + 1), 1), (dict(weight=P + 2), 1), (dict(loss_out=P + 1), 1),
                      (dict(top_idx=P + 2), 1), (dict(top_val=P + 1), 1), (dict(rows=P + 2), 1), (dict(n_rows=P + 4), 1)):
        assert refused(B, loss, **bad) == want, bad


def test_workspaces_of_a_bound_serve_every_smaller_call(B):
    sizes = sorted({*range(0, 400), *range(1000, 1100), *range(4000, 4200), *range(16300, 16500), *range(30000, 300000, 1000), 10 ** 6, 3 * 10 ** 6, 10 ** 7, 2 ** 31 - 1})
    for d, blocks in ((9, 1), (8, 8), (88, 8), (100, 5), (100, 100), (256, 32), (1024, 32), (1024, 1), (1024, 1024), (4096, 2), (16384, 1), (16384, 16384), (1500, 3)):
        for need in (B.fg_group_norm_workspace_bytes, B.fg_group_norm_backward_workspace_bytes):
            got = [need(n, 37, d, blocks) for n in sizes]
            assert got == sorted(got) and min(got) > 0
    sizes = [n for n in sizes if n <= 10 ** 7]
    for t, a, b in ((B.FG_F32, 96, 256), (B.FG_BF16, 264, 520), (B.FG_F16, 1024, 1024)):
        got = [B.fg_gated_linear_grouped_backward_workspace_bytes(t, n, 5, a, b) for n in sizes]
        assert got == sorted(got) and min(got) > 0


# ---- the statements themselves, against differences ----

def test_statements_of_the_gradients_agree_with_differences():
    g = torch.Generator().manual_seed(3)
    step = 1e-6
    rand = lambda *s: torch.randn(*s, dtype=torch.float64, generator=g)
    def along(f, x):
        d = rand(*x.shape)
        return d, (f(x + step * d) - f(x - step * d)) / (2 * step)
    for name in R.ACTS:
        x, W, b, dh = rand(5, 4), rand(4, 6), rand(6), rand(5, 3)
        f = lambda x, W, b: (R.gated(x, W, b, name)[1] * dh).sum()
        dz, _ = R.gated_dz(R.gated(x, W, b, name)[0], dh, name)
        for grad, (d, want) in ((dz @ W.T, along(lambda v: f(v, W, b), x)), (x.T @ dz, along(lambda v: f(x, v, b), W)), (dz.sum(0), along(lambda v: f(x, W, v), b))):
            assert abs(float((grad * d).sum() - want)) < 1e-6 * (1 + abs(float(want))), name
        x, w, b, dy = rand(7, 6), rand(6), rand(6), rand(7, 6)
        def f(x, w, b):
            mean, rstd = R.norm_statistics(x, 2, 1e-5)
            return (R.norm_rows(x, mean, rstd, w, b, name)[0] * dy).sum()
        (dx, _), (dw, _), (db, _), _ = R.norm_backward(x, dy, *R.norm_statistics(x, 2, 1e-5), w, b, name)
        for grad, (d, want) in ((dx, along(lambda v: f(v, w, b), x)), (dw, along(lambda v: f(x, v, b), w)), (db, along(lambda v: f(x, w, v), b))):
            assert abs(float((grad * d).sum() - want)) < 1e-6 * (1 + abs(float(want))), name
    z, idx, val, label = rand(6, 9), torch.randint(-1, 10, (6, 4), generator=g), rand(6, 4), torch.tensor([0, -1, 3, 9, 8, 2])
    weight = torch.rand(6, generator=g)
    for alpha in (0.0, 0.5, 1.0):
        f = lambda v: R.distill(v, idx, val, label, 2.0, alpha, weight, 1.0)[0].sum()
        d, want = along(f, z)
        assert abs(float((R.distill(z, idx, val, label, 2.0, alpha, weight, 1.0)[2] * d).sum() - want)) < 1e-6 * (1 + abs(float(want)))


# ---- gated layer ----

def groups_of(r, n, listed, n_groups, options, table=None):
    """order, offsets and source rows: listed positions dealt to groups at random (some of them empty), or positions that lie sorted."""
    k = max(1, int(n * listed))
    if "order0" in options:
        order = np.arange(k, dtype=np.int32)
    else:
        order = r.permutation(n)[:k].astype(np.int32)
    cuts = np.sort(r.integers(0, k + 1, n_groups - 1))
    if "empty" in options and n_groups > 2:
        cuts[:2] = 0
        cuts = np.sort(cuts)
    offsets = np.concatenate([[0], cuts, [k]]).astype(np.int64)
    src = r.integers(0, table, n).astype(np.int32) if table else None
    return order, offsets, src


GATED = [  # dtype, out, n, groups, d_in, d_out, act, options
    ("f32", "f32", 1, 1, 4, 4, "silu", ""), ("f32", "f32", 5, 1, 64, 256, "gelu", "keep"), ("f32", "f32", 70, 3, 100, 36, "relu", "keep src pad"),
    ("f32", "f32", 300, 7, 88, 256, "sigmoid", "keep empty"), ("f32", "f32", 33, 2, 260, 128, "none", "nobias order0"),
    ("bf16", "bf16", 1, 1, 8, 8, "silu", "keep"), ("bf16", "bf16", 16, 1, 1024, 1024, "silu", ""), ("bf16", "f32", 17, 1, 264, 40, "gelu", "keep"),
    ("bf16", "bf16", 130, 4, 72, 136, "relu", "keep src pad empty"), ("f16", "f16", 64, 2, 128, 32, "silu", "nobias"), ("f16", "f32", 200, 5, 40, 264, "sigmoid", "keep src"),
    ("f16", "f16", 1000, 3, 200, 72, "gelu", "keep order0"), ("bf16", "bf16", 3, 3, 2048, 64, "silu", "keep"), ("f16", "f16", 31, 31, 96, 96, "silu", "keep empty pad"),
    ("f32", "f32", 1000, 1024, 32, 64, "silu", "src"),
    # few rows, the contraction split: none, one and several steps to a share of it, the last of them partly filled
    ("f32", "f32", 40, 1, 2052, 20, "silu", "keep src"), ("f32", "f32", 35, 2, 388, 132, "gelu", "keep pad"), ("bf16", "bf16", 33, 1, 1096, 24, "gelu", "keep pad"),
    ("f16", "f32", 64, 2, 520, 72, "silu", "keep empty"), ("bf16", "f32", 2, 1, 4096, 8, "silu", "src"), ("f16", "f16", 250, 1, 776, 1000, "silu", ""),
    ("f32", "f32", 12_000, 5, 100, 36, "silu", "keep"), ("bf16", "bf16", 9000, 7, 136, 72, "gelu", "keep src"), ("f16", "f32", 5000, 2, 72, 200, "silu", "keep"),
]


def run_gated(B, x, d_in, W, bias, order, offsets, src, name, h, d_out, z, dtype, out, stream=None, max_rows=None):
    n_groups = len(offsets) - 1
    B.fg_gated_linear_grouped(x, len(x), stride(x), code(B, dtype), src, order, offsets, len(order) if max_rows is None else max_rows, n_groups, d_in, d_out, W, bias,
                              act_code(B, name), h, len(h), stride(h), code(B, out), z, stride(z) if z is not None else 0, stream)


@gpu
@pytest.mark.parametrize("dtype, out, n, n_groups, d_in, d_out, name, options", GATED)
def test_gated_linear(B, dtype, out, n, n_groups, d_in, d_out, name, options):
    r = np.random.default_rng(n * 31 + d_in + d_out)
    pad = 8 if "pad" in options else 0
    table = 2 * n + 3 if "src" in options else None
    order, offsets, src = groups_of(r, n, 0.8, n_groups, options, table)
    x = values(r, table or n, d_in, dtype, pad)
    W = torch.from_numpy(r.standard_normal((n_groups, d_in, 2 * d_out)) / math.sqrt(d_in)).to(T[dtype])
    bias = None if "nobias" in options else torch.from_numpy(r.standard_normal((n_groups, 2 * d_out))).float()
    h, z = sentinel(n, d_out, out, pad).cuda(), sentinel(n, 2 * d_out, dtype, pad).cuda() if "keep" in options else None
    run_gated(B, x.cuda(), d_in, W.cuda(), cuda(bias), None if "order0" in options else torch.from_numpy(order).cuda(), torch.from_numpy(offsets).cuda(),
              torch.from_numpy(src).cuda() if src is not None else None, name, h, d_out, z, dtype, out, max_rows=len(order))
    torch.cuda.synchronize()
    h, z = h.cpu(), z.cpu() if z is not None else None
    rest = np.setdiff1d(np.arange(n), order)
    for t, d in ((h, d_out), (z, 2 * d_out)):
        assert t is None or (bool((t[rest] == -77).all()) and bool((t[:, d:] == -77).all())), "rows that are not listed, and the ends of the rows, stay"
    for g, pos, rows in R.members(order, offsets.tolist(), n, src):
        want_z, want_h, z_off, h_off = R.gated(x[rows, :d_in], W[g], bias[g] if bias is not None else None, name)
        close(h[pos, :d_out], want_h, h_off + HALF[out] * want_h.abs() + TINY[out], f"h of group {g}")
        if z is not None:
            close(z[pos, :2 * d_out], want_z, z_off + HALF[dtype] * want_z.abs() + TINY[dtype], f"z of group {g}")


MANY = [  # tiles of 256, 128 and 64 rows, several to a workgroup; whole steps of the contraction and parts of one
    ("bf16", "bf16", 40_000, 3, 64, 264, "silu", "keep src"), ("bf16", "f32", 70_001, 2, 72, 136, "gelu", "keep"), ("f16", "f16", 36_000, 40, 136, 264, "relu", ""),
    ("f16", "f16", 90_000, 1, 264, 40, "silu", "keep src"), ("f16", "f32", 160_000, 600, 40, 72, "sigmoid", ""), ("bf16", "bf16", 33_100, 1, 1024, 520, "silu", "keep"),
    ("f32", "f32", 50_000, 3, 100, 256, "silu", "keep src"), ("f32", "f32", 90_000, 60, 36, 132, "gelu", "keep"), ("f32", "f32", 20_000, 1, 260, 36, "relu", ""),
]


def many(n, n_groups, d_in, d_out, dtype, options):
    g = torch.Generator(device="cuda").manual_seed(n + d_in + d_out)
    kw = dict(device="cuda", generator=g)
    rows = torch.randperm(n, **kw)[:n - n // 7]
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), torch.randint(0, len(rows) + 1, (n_groups - 1,), **kw).sort().values,
                         torch.full((1,), len(rows), dtype=torch.int64, device="cuda")])
    src = torch.randint(0, n, (n,), **kw).int() if "src" in options else None
    return rows.int(), offsets, src, torch.randn(n, d_in, **kw).to(T[dtype]), (torch.randn(n_groups, d_in, 2 * d_out, **kw) / math.sqrt(d_in)).to(T[dtype]), \
        torch.randn(n_groups, 2 * d_out, **kw)


@gpu
@pytest.mark.parametrize("dtype, out, n, n_groups, d_in, d_out, name, options", MANY)
def test_gated_linear_of_many_rows(B, dtype, out, n, n_groups, d_in, d_out, name, options):
    order, offsets, src, x, W, bias = many(n, n_groups, d_in, d_out, dtype, options)
    h, z = sentinel(n, d_out, out).cuda(), sentinel(n, 2 * d_out, dtype).cuda() if "keep" in options else None
    for _ in range(2):      # the second time over the first one's results
        run_gated(B, x, d_in, W, bias, order, offsets, src, name, h, d_out, z, dtype, out)
    torch.cuda.synchronize()
    at, listed = offsets.tolist(), torch.zeros(n, dtype=torch.bool, device="cuda")
    listed[order.long()] = True
    assert bool((h[~listed] == -77).all()) and (z is None or bool((z[~listed] == -77).all()))
    for g in range(n_groups):
        pos = order[at[g]:at[g + 1]].long()
        want_z, want_h, z_off, h_off = R.gated(x[src[pos].long() if src is not None else pos], W[g], bias[g], name)
        close(h[pos], want_h, h_off + HALF[out] * want_h.abs() + TINY[out], f"h of group {g}")
        if z is not None:
            close(z[pos], want_z, z_off + HALF[dtype] * want_z.abs() + TINY[dtype], f"z of group {g}")


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gated_linear_skips_what_is_out_of_range(B, dtype):
    r = np.random.default_rng(4)
    n, a, b, table = 50, 64, 40, 20
    order = r.permutation(n)[:30].astype(np.int32)
    order[[3, 7, 29]] = (-1, n, 2 ** 31 - 1)
    src = r.integers(0, table, n).astype(np.int32)
    src[order[[0, 11]]] = (-5, table)
    offsets = np.array([0, 12, 12, 30], np.int64)
    x, W = values(r, table, a, dtype), torch.from_numpy(r.standard_normal((3, a, 2 * b)) / 8).to(T[dtype])
    h, z, dh = sentinel(n, b, dtype).cuda(), sentinel(n, 2 * b, dtype).cuda(), values(r, n, b, dtype)
    dev = [t.cuda() for t in (x, W, torch.from_numpy(order), torch.from_numpy(offsets), torch.from_numpy(src))]
    run_gated(B, dev[0], a, dev[1], None, dev[2], dev[3], dev[4], "silu", h, b, z, dtype, dtype)
    torch.cuda.synchronize()
    taken = np.zeros(n, bool)
    dW = torch.zeros(3, a, 2 * b, dtype=torch.float64)
    dW_off = torch.zeros_like(dW)
    zc = z.cpu()
    for g, pos, rows in R.members(order, offsets.tolist(), n, src, table):
        taken[pos] = True
        _, want, _, off = R.gated(x[rows], W[g], None, "silu")
        close(h.cpu()[pos], want, off + HALF[dtype] * want.abs() + TINY[dtype], "h")
        dz, dz_off = R.gated_dz(zc[pos], dh[pos], "silu")
        dz_off = dz_off + (HALF[dtype] if dtype != "f32" else 0) * dz.abs()
        dW[g] = x[rows].double().T @ dz
        dW_off[g] = x[rows].double().abs().T @ (dz_off + (len(rows) + 8) * 2.0 ** -23 * dz.abs())
    assert bool((h.cpu()[~taken] == -77).all()) and bool((zc[~taken] == -77).all())
    # gradients: the entries that are skipped have no part in them (their z and dh are NaN here)
    z_bad, dh_bad = z.clone(), dh.cuda()
    z_bad[torch.from_numpy(~taken).cuda()] = float("nan")
    dh_bad[torch.from_numpy(~taken).cuda()] = float("nan")
    dw, db, dx = torch.empty(3, a, 2 * b, device="cuda"), torch.empty(3, 2 * b, device="cuda"), sentinel(n, a, dtype).cuda()
    need = B.fg_gated_linear_grouped_backward_workspace_bytes(code(B, dtype), 30, 3, a, b)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    B.fg_gated_linear_grouped_backward(dev[0], table, stride(x), code(B, dtype), dev[4], dh_bad, stride(dh), code(B, dtype), z_bad, stride(z_bad), n, dev[2], dev[3], 30, 3, a, b,
                                       dev[1], B.FG_ACT_SILU, dx, stride(dx), code(B, dtype), dw, B.FG_F32, db, ws, need)
    torch.cuda.synchronize()
    close(dw.cpu(), dW, dW_off + 2.0 ** -24 * dW.abs(), "dW")
    assert bool((dx.cpu()[~taken] == -77).all()) and bool(torch.isfinite(dx.cpu()[taken].float()).all()) and bool(torch.isfinite(db).all())


GATED_BW = [  # dtype, dh, dx, dw, n, groups, d_in, d_out, act, options
    ("f32", "f32", "f32", "f32", 1, 1, 4, 4, "silu", ""), ("f32", "f32", "f32", "f32", 300, 3, 88, 256, "silu", ""), ("f32", "f32", "f32", "f32", 500, 5, 100, 36, "gelu", "src pad"),
    ("f32", "f32", "f32", "f32", 65, 2, 64, 12, "relu", "empty order0"), ("f32", "f32", "f32", "f32", 2000, 1, 132, 64, "sigmoid", ""),
    ("bf16", "bf16", "bf16", "bf16", 400, 1, 264, 136, "silu", ""), ("bf16", "f32", "f32", "f32", 130, 4, 72, 40, "gelu", "src pad empty"),
    ("f16", "f16", "f16", "f16", 700, 3, 64, 64, "silu", "src"), ("f16", "f32", "f16", "f32", 90, 2, 40, 8, "none", "order0"), ("bf16", "bf16", "f32", "bf16", 5, 1, 1024, 512, "silu", ""),
    ("f16", "f16", "f32", "f16", 1500, 40, 136, 72, "relu", ""), ("bf16", "bf16", "bf16", "bf16", 30_000, 2, 136, 264, "silu", ""), ("f32", "f32", "f32", "f32", 20_000, 3, 64, 132, "silu", ""),
    ("f16", "f16", "f16", "f16", 20_000, 1, 520, 520, "gelu", "src"),
]


@gpu
@pytest.mark.parametrize("dtype, dh_type, dx_type, dw_type, n, n_groups, d_in, d_out, name, options", GATED_BW)
def test_gated_linear_backward(B, dtype, dh_type, dx_type, dw_type, n, n_groups, d_in, d_out, name, options):
    r = np.random.default_rng(n + 7 * d_in + d_out)
    pad = 8 if "pad" in options else 0
    table = n + 11 if "src" in options else None
    order, offsets, src = groups_of(r, n, 0.9, n_groups, options, table)
    x, W = values(r, table or n, d_in, dtype, pad).cuda(), torch.from_numpy(r.standard_normal((n_groups, d_in, 2 * d_out)) / math.sqrt(d_in)).to(T[dtype]).cuda()
    z, dh = values(r, n, 2 * d_out, dtype, pad).cuda(), values(r, n, d_out, dh_type, pad).cuda()
    dx = sentinel(n, d_in, dx_type, pad).cuda()
    dw = torch.full((n_groups, d_in, 2 * d_out), -77.0, dtype=T[dw_type], device="cuda")
    db = torch.full((n_groups, 2 * d_out), -77.0, device="cuda")
    need = B.fg_gated_linear_grouped_backward_workspace_bytes(code(B, dtype), len(order), n_groups, d_in, d_out)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    t_order, t_offsets = None if "order0" in options else torch.from_numpy(order).cuda(), torch.from_numpy(offsets).cuda()
    t_src = torch.from_numpy(src).cuda() if src is not None else None

    def call(dx, dw, db):
        B.fg_gated_linear_grouped_backward(x, len(x), stride(x), code(B, dtype), t_src, dh, stride(dh), code(B, dh_type), z, stride(z), n, t_order, t_offsets, len(order), n_groups,
                                           d_in, d_out, W, act_code(B, name), dx, stride(dx) if dx is not None else 0, code(B, dx_type), dw, code(B, dw_type), db, ws, need)

    call(dx, dw, db)
    torch.cuda.synchronize()
    rest = torch.from_numpy(np.setdiff1d(np.arange(n), order)).cuda()
    assert bool((dx[rest] == -77).all()) and bool((dx[:, d_in:] == -77).all())
    op = HALF[dtype] if dtype != "f32" else 0.0
    for g, pos, rows in R.members(order, offsets.tolist(), n, src):
        dz, off = R.gated_dz(z[pos.cuda(), :2 * d_out], dh[pos.cuda(), :d_out], name)
        dz_off = off + op * (dz.abs() + off) + (TINY[dtype] if op else 0)      # as it is multiplied
        xs, Wt = x[rows.cuda(), :d_in].double(), W[g].double().T.contiguous()
        want = torch.mm(dz, Wt)
        close(dx[pos.cuda(), :d_in], want, torch.mm(dz_off + (2 * d_out + 8) * 2.0 ** -23 * dz.abs(), Wt.abs()) + HALF[dx_type] * want.abs() + TINY[dx_type], f"dx of group {g}")
        xt = xs.T.contiguous()
        want = torch.mm(xt, dz)
        close(dw[g], want, torch.mm(xt.abs(), dz_off + (len(rows) + 8) * 2.0 ** -23 * dz.abs()) + HALF[dw_type] * want.abs() + TINY[dw_type], f"dW of group {g}")
        close(db[g], dz.sum(0), (off + (len(rows) + 8) * 2.0 ** -23 * dz.abs()).sum(0) + 2.0 ** -24 * dz.sum(0).abs(), f"db of group {g}")
    # each by itself, and again: the same bits
    for want in ((dx, None, None), (None, dw, None), (None, None, db), (dx, dw, db)):
        again = [torch.full_like(t, -77) if t is not None else None for t in want]
        call(*again)
        torch.cuda.synchronize()
        assert all(t is None or torch.equal(t[:, :d_in] if t is again[0] else t, w[:, :d_in] if t is again[0] else w) for t, w in zip(again, want))


@gpu
def test_gated_linear_of_no_rows(B):
    W, off = torch.ones(2, 64, 64, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    x, h, z = torch.ones(4, 64, device="cuda"), sentinel(4, 32, "f32").cuda(), torch.ones(4, 64, device="cuda")
    dw, db, dx = torch.ones(2, 64, 64, device="cuda"), torch.ones(2, 64, device="cuda"), sentinel(4, 64, "f32").cuda()
    need = B.fg_gated_linear_grouped_backward_workspace_bytes(B.FG_F32, 4, 2, 64, 32)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    for rows in (0, 4):      # none by the bound, none by the offsets
        B.fg_gated_linear_grouped(x, 4, 256, B.FG_F32, None, None, off, rows, 2, 64, 32, W, None, B.FG_ACT_SILU, h, 4, 128, B.FG_F32, None, 0)
        dw.fill_(1), db.fill_(1)
        B.fg_gated_linear_grouped_backward(x, 4, 256, B.FG_F32, None, h, 128, B.FG_F32, z, 256, 4, None, off, rows, 2, 64, 32, W, B.FG_ACT_SILU, dx, 256, B.FG_F32, dw, B.FG_F32, db,
                                           ws, need)
        torch.cuda.synchronize()
        assert bool((h == -77).all()) and bool((dx == -77).all()) and not bool(dw.any()) and not bool(db.any())


# ---- group norm ----

NORM = [  # dtype, out, n, groups, d, channel groups, act, options
    ("f32", "f32", 1, 1, 9, 1, "none", ""), ("f32", "f32", 1, 1, 8, 2, "silu", ""), ("bf16", "bf16", 50, 3, 8827, 1261, "silu", "gather"), ("f32", "f32", 777, 9, 88, 8, "gelu", ""), ("f32", "f32", 3000, 100, 100, 5, "relu", "empty"),
    ("f32", "f32", 2000, 3, 100, 100, "silu", "gather"), ("f32", "f32", 500, 4, 89, 1, "sigmoid", "gather pad noaffine"), ("f32", "f32", 9000, 2, 256, 32, "silu", "gather level"),
    ("bf16", "bf16", 700, 6, 256, 8, "silu", "gather pad"), ("bf16", "f32", 400, 3, 35, 7, "none", "empty"), ("bf16", "bf16", 5000, 2, 1024, 32, "silu", "gather"),
    ("f16", "f16", 6000, 5000, 64, 4, "gelu", "empty"), ("f16", "f32", 300, 2, 514, 2, "silu", "gather level pad"), ("f16", "f16", 90, 2, 4096, 1, "relu", ""),
    ("bf16", "bf16", 40, 3, 16384, 4, "silu", "empty"), ("f32", "f32", 300, 1, 5000, 1, "silu", "gather"), ("bf16", "bf16", 20_000, 3, 24, 3, "silu", "gather"),
    ("f32", "f32", 20_000, 1, 16, 16, "none", "level"), ("bf16", "bf16", 3000, 1, 2048, 2048, "silu", ""), ("f16", "f16", 2500, 7, 600, 200, "sigmoid", "gather"),
    ("f32", "f32", 70_000, 3, 260, 1, "gelu", "gather"),
]


def norm_inputs(dtype, n, n_groups, d, options):
    r = np.random.default_rng(n + d + n_groups)
    pad = 3 if "pad" in options else 0
    if "gather" in options:
        order, offsets, _ = groups_of(r, n, 0.85, n_groups, options)
    else:
        order, offsets, _ = groups_of(r, n, 1.0, n_groups, options + " order0")
    level = 300.0 if "level" in options else r.standard_normal(d)
    x = values(r, n, d, dtype, pad, 1.5, level)
    w, b = (None, None) if "noaffine" in options else (torch.from_numpy(1 + 0.3 * r.standard_normal(d)).float(), torch.from_numpy(0.3 * r.standard_normal(d)).float())
    return r, pad, order, offsets, x, w, b


@gpu
@pytest.mark.parametrize("dtype, out, n, n_groups, d, blocks, name, options", NORM)
def test_group_norm(B, dtype, out, n, n_groups, d, blocks, name, options):
    r, pad, order, offsets, x, w, b = norm_inputs(dtype, n, n_groups, d, options)
    eps = 1e-5
    y, mean, rstd = sentinel(n, d, out, pad).cuda(), torch.full((n_groups, blocks), -77.0, device="cuda"), torch.full((n_groups, blocks), -77.0, device="cuda")
    need = B.fg_group_norm_workspace_bytes(len(order), n_groups, d, blocks)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    xd, ordered, off = x.cuda(), torch.from_numpy(order).cuda() if "gather" in options else None, torch.from_numpy(offsets).cuda()

    def call(x, y, out, mean, rstd):
        B.fg_group_norm(x, stride(x), code(B, dtype), ordered, off, len(order), n_groups, n, d, blocks, cuda(w), cuda(b), eps, act_code(B, name), y, stride(y), code(B, out),
                        mean, rstd, ws, need)
        torch.cuda.synchronize()

    call(xd, y, out, mean, rstd)
    rest = np.setdiff1d(np.arange(n), order)
    assert bool((y[torch.from_numpy(rest).cuda()] == -77).all()) and bool((y[:, d:] == -77).all())
    got, m, s = y.cpu(), mean.cpu(), rstd.cpu()
    eps64 = float(np.float32(eps))
    for g, pos, _ in R.members(order, offsets.tolist(), n) if n_groups < 200 else R.members(order, offsets.tolist(), n)[::37]:
        want_m, want_s = R.norm_statistics(x[pos, :d], blocks, eps64)
        largest = x[pos, :d].double().abs().max() if len(pos) else torch.zeros((), dtype=torch.float64)
        close(m[g], want_m, 2.0 ** -24 * want_m.abs() + 2.0 ** -40 * largest, f"mean of group {g}")
        close(s[g], want_s, 2.0 ** -23 * want_s, f"rstd of group {g}")
        if len(pos):
            want, tol, _, _ = R.norm_rows(x[pos, :d], want_m, want_s, w, b, name)
            close(got[pos, :d], want, tol + HALF[out] * want.abs() + TINY[out], f"y of group {g}")
    # without statistics, over x itself, again: the same bits
    again = sentinel(n, d, out, pad).cuda()
    call(xd, again, out, None, None)
    assert torch.equal(again, y)
    if out == dtype:
        call(xd, xd, out, None, None)
        listed = torch.from_numpy(order).cuda().long()
        assert torch.equal(xd[listed, :d], y[listed, :d]) and torch.equal(xd.cpu()[rest][:, :d], x[rest][:, :d])


@gpu
@pytest.mark.parametrize("grad", ["f32", "same"])
@pytest.mark.parametrize("dtype, out, n, n_groups, d, blocks, name, options", NORM)
def test_group_norm_backward(B, dtype, out, n, n_groups, d, blocks, name, options, grad):
    if grad == "same":
        grad = dtype
    r, pad, order, offsets, x, w, b = norm_inputs(dtype, n, n_groups, d, options)
    dy = values(r, n, d, grad, pad)
    parts = R.members(order, offsets.tolist(), n)
    mean, rstd = torch.zeros(n_groups, blocks), torch.zeros(n_groups, blocks)
    for g, pos, _ in parts:
        m, s = R.norm_statistics(x[pos, :d], blocks, 1e-5)
        mean[g], rstd[g] = m.float(), s.float()
    if name == "relu":      # nothing near the corner, where the slope is one of two
        for g, pos, _ in parts:
            if len(pos):
                _, _, _, u = R.norm_rows(x[pos, :d], mean[g].double(), rstd[g].double(), w, b, name)
                dy[pos, :d] = torch.where(u.abs() < 1e-3, torch.zeros((), dtype=dy.dtype), dy[pos, :d])
    dx, dw, db = sentinel(n, d, grad, pad).cuda(), torch.full((d + 2,), -77.0, device="cuda"), torch.full((d + 2,), -77.0, device="cuda")
    need = B.fg_group_norm_backward_workspace_bytes(len(order), n_groups, d, blocks)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    xd, gd, ordered, off = x.cuda(), dy.cuda(), torch.from_numpy(order).cuda() if "gather" in options else None, torch.from_numpy(offsets).cuda()
    md, sd = mean.cuda(), rstd.cuda()

    def call(dy, dx, dw, db):
        B.fg_group_norm_backward(dy, stride(dy), code(B, grad), xd, stride(xd), code(B, dtype), md, sd, cuda(w), cuda(b), act_code(B, name), ordered, off, len(order), n_groups,
                                 n, d, blocks, dx, stride(dx), dw, db, ws, need)
        torch.cuda.synchronize()

    call(gd, dx, dw, db)
    rest = np.setdiff1d(np.arange(n), order)
    got = dx.cpu()
    assert bool((got[rest] == -77).all()) and bool((got[:, d:] == -77).all()) and bool((dw[d:] == -77).all()) and bool((db[d:] == -77).all())
    sums = [torch.zeros(d, dtype=torch.float64) for _ in range(4)]
    for i, (g, pos, _) in enumerate(parts):
        if not len(pos):
            continue
        (want, tol), (gw, gw_off), (gb, gb_off), _ = R.norm_backward(x[pos, :d], dy[pos, :d], mean[g], rstd[g], w, b, name)
        for t, v in zip(sums, (gw, gw_off, gb, gb_off)):
            t += v
        close(got[pos, :d], want, tol + HALF[grad] * want.abs() + TINY[grad], f"dx of group {g}")
    close(dw.cpu()[:d], sums[0], sums[1] + 2.0 ** -23 * sums[0].abs() + 2.0 ** -100, "dw")
    close(db.cpu()[:d], sums[2], sums[3] + 2.0 ** -23 * sums[2].abs() + 2.0 ** -100, "db")
    again, one = sentinel(n, d, grad, pad).cuda(), torch.zeros(d, device="cuda")
    call(gd, again, None, None)
    assert torch.equal(again, dx)
    call(gd, again, None, one)
    assert torch.equal(one, db[:d])
    call(gd, gd, one, None)      # over dy
    listed = torch.from_numpy(order).cuda().long()
    assert torch.equal(one, dw[:d]) and torch.equal(gd[listed, :d], dx[listed, :d]) and torch.equal(gd.cpu()[rest][:, :d], dy[rest][:, :d])


@gpu
def test_group_norm_of_no_rows_and_of_one_value(B):
    off = torch.zeros(4, dtype=torch.int64, device="cuda")
    x, y = torch.full((5, 8), 3.0, device="cuda"), sentinel(5, 8, "f32").cuda()
    ws = torch.zeros(B.fg_group_norm_backward_workspace_bytes(5, 3, 8, 2), dtype=torch.uint8, device="cuda")
    for rows in (0, 5):
        mean, rstd = torch.full((3, 2), -77.0, device="cuda"), torch.full((3, 2), -77.0, device="cuda")
        B.fg_group_norm(x, 32, B.FG_F32, None, off, rows, 3, 5, 8, 2, None, None, 0.25, 0, y, 32, B.FG_F32, mean, rstd, ws, len(ws))
        dw, db, dx = torch.ones(8, device="cuda"), torch.ones(8, device="cuda"), sentinel(5, 8, "f32").cuda()
        B.fg_group_norm_backward(x, 32, B.FG_F32, x, 32, B.FG_F32, mean, rstd, None, None, 0, None, off, rows, 3, 5, 8, 2, dx, 32, dw, db, ws, len(ws))
        torch.cuda.synchronize()
        assert bool((y == -77).all()) and bool((mean == 0).all()) and bool((rstd == 2).all()) and bool((dx == -77).all()) and not bool(dw.any()) and not bool(db.any())
    # values that are all the same have variance 0, whatever their level: no value is made of their rounding
    off[1:] = torch.tensor([2, 4, 5])
    x.fill_(1e7 + 1)
    B.fg_group_norm(x, 32, B.FG_F32, None, off, 5, 3, 5, 8, 2, None, None, 0.25, 0, y, 32, B.FG_F32, mean, rstd, ws, len(ws))
    torch.cuda.synchronize()
    assert not bool(y.any()) and bool((mean == 1e7 + 1).all()) and bool((rstd == 2).all())


@gpu
def test_group_norm_leaves_out_what_is_out_of_range(B):
    r = np.random.default_rng(8)
    for n, d, blocks in ((60, 24, 3), (4000, 200, 4), (5000, 64, 1)):
        order = r.permutation(n)[:n - 10].astype(np.int32)
        order[[0, 5, len(order) - 1]] = (-1, n, 2 ** 31 - 1)      # the group's first entry among them
        offsets = np.array([0, len(order) - 20, len(order)], np.int64)
        x, dy = values(r, n, d, "f32"), values(r, n, d, "f32")
        y, mean, rstd = sentinel(n, d, "f32").cuda(), torch.zeros(2, blocks, device="cuda"), torch.zeros(2, blocks, device="cuda")
        ws = torch.full((B.fg_group_norm_backward_workspace_bytes(len(order), 2, d, blocks),), 255, dtype=torch.uint8, device="cuda")
        dx, dw, db = sentinel(n, d, "f32").cuda(), torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
        o, f, xd, gd = torch.from_numpy(order).cuda(), torch.from_numpy(offsets).cuda(), x.cuda(), dy.cuda()
        B.fg_group_norm(xd, d * 4, B.FG_F32, o, f, len(order), 2, n, d, blocks, None, None, 1e-5, B.FG_ACT_SILU, y, d * 4, B.FG_F32, mean, rstd, ws, len(ws))
        B.fg_group_norm_backward(gd, d * 4, B.FG_F32, xd, d * 4, B.FG_F32, mean, rstd, None, None, B.FG_ACT_SILU, o, f, len(order), 2, n, d, blocks, dx, d * 4, dw, db, ws, len(ws))
        torch.cuda.synchronize()
        taken = np.zeros(n, bool)
        for g, pos, _ in R.members(order, offsets.tolist(), n):
            taken[pos] = True
            m, s = R.norm_statistics(x[pos], blocks, float(np.float32(1e-5)))
            close(mean.cpu()[g], m, 2.0 ** -24 * m.abs() + 2.0 ** -36, "mean")
            close(rstd.cpu()[g], s, 2.0 ** -23 * s, "rstd")
            want, tol, _, _ = R.norm_rows(x[pos], m, s, None, None, "silu")
            close(y.cpu()[pos], want, tol + 2.0 ** -24 * want.abs(), "y")
            (want, tol), _, _, _ = R.norm_backward(x[pos], dy[pos], mean.cpu()[g], rstd.cpu()[g], None, None, "silu")
            close(dx.cpu()[pos], want, tol + 2.0 ** -24 * want.abs(), "dx")
        assert bool((y.cpu()[~taken] == -77).all()) and bool((dx.cpu()[~taken] == -77).all())


@gpu
@pytest.mark.parametrize("dtype, n, d, blocks", [("f32", 40_000, 256, 8), ("bf16", 300_000, 64, 8), ("f32", 20_000, 64, 2), ("f16", 30_000, 512, 1), ("bf16", 9000, 1024, 32)])
def test_group_norm_of_split_groups_over_their_own_rows(B, dtype, n, d, blocks):
    """Rows of groups that many workgroups share are overwritten while others still form the statistics: the same bits as beside them, every time."""
    g = torch.Generator(device="cuda").manual_seed(n)
    x = (torch.randn(n, d, device="cuda", generator=g) + 5 * torch.randn(d, device="cuda", generator=g)).to(T[dtype])
    off = torch.tensor([0, n // 3, n], device="cuda")
    ws = torch.zeros(B.fg_group_norm_workspace_bytes(n, 2, d, blocks), dtype=torch.uint8, device="cuda")
    y = torch.empty_like(x)

    def call(x, y):
        B.fg_group_norm(x, stride(x), code(B, dtype), None, off, n, 2, n, d, blocks, None, None, 1e-5, B.FG_ACT_NONE, y, stride(y), code(B, dtype), None, None, ws, len(ws))

    call(x, y)
    for _ in range(20):
        over = x.clone()
        call(over, over)
        assert torch.equal(over, y)


@gpu
@pytest.mark.parametrize("n", [300, 60_000])
def test_group_norm_of_the_most_groups(B, n):
    """2^20 groups, nearly all of them without rows, one of half of the rows among them; forward and back."""
    G, d, blocks = B.FG_MAX_NORM_GROUPS, 16, 2
    r = np.random.default_rng(n)
    group = r.integers(0, G, n)
    group[:n // 2] = G // 3
    group[-1] = G - 1
    group = np.sort(group)
    off = torch.from_numpy(np.searchsorted(group, np.arange(G + 1))).cuda()
    x, dy = values(r, n, d, "f32"), values(r, n, d, "f32")
    y, dx, mean, rstd = (torch.full(s, -77.0, device="cuda") for s in ((n, d), (n, d), (G, blocks), (G, blocks)))
    dw, db = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
    ws = torch.full((B.fg_group_norm_backward_workspace_bytes(n, G, d, blocks),), 255, dtype=torch.uint8, device="cuda")
    xd, gd = x.cuda(), dy.cuda()
    B.fg_group_norm(xd, d * 4, B.FG_F32, None, off, n, G, n, d, blocks, None, None, 0.25, B.FG_ACT_SILU, y, d * 4, B.FG_F32, mean, rstd, ws, len(ws))
    B.fg_group_norm_backward(gd, d * 4, B.FG_F32, xd, d * 4, B.FG_F32, mean, rstd, None, None, B.FG_ACT_SILU, None, off, n, G, n, d, blocks, dx, d * 4, dw, db, ws, len(ws))
    torch.cuda.synchronize()
    y, dx, mean, rstd, dw, db = (t.cpu() for t in (y, dx, mean, rstd, dw, db))
    there = np.unique(group)
    none = np.setdiff1d(np.arange(G), there)
    assert bool((mean[none] == 0).all()) and bool((rstd[none] == 2).all())
    sums = [torch.zeros(d, dtype=torch.float64) for _ in range(4)]
    for g in there if n < 1000 else there[:40].tolist() + [G // 3, G - 1]:
        pos = torch.from_numpy(np.flatnonzero(group == g))
        m, s = R.norm_statistics(x[pos], blocks, 0.25)
        close(mean[g], m, 2.0 ** -24 * m.abs() + 2.0 ** -40 * x[pos].double().abs().max(), "mean")
        close(rstd[g], s, 2.0 ** -23 * s, "rstd")
        want, tol, _, _ = R.norm_rows(x[pos], m, s, None, None, "silu")
        close(y[pos], want, tol + 2.0 ** -24 * want.abs(), "y")
        (want, tol), (gw, gw_off), (gb, gb_off), _ = R.norm_backward(x[pos], dy[pos], mean[g], rstd[g], None, None, "silu")
        close(dx[pos], want, tol + 2.0 ** -24 * want.abs(), "dx")
        for t, v in zip(sums, (gw, gw_off, gb, gb_off)):
            t += v
    if n < 1000:
        close(dw, sums[0], sums[1] + 2.0 ** -23 * sums[0].abs(), "dw")
        close(db, sums[2], sums[3] + 2.0 ** -23 * sums[2].abs(), "db")


# ---- distillation ----

DISTILL = [  # dtype, dh, n, d, k, top, T, alpha, options
    ("f32", "f32", 1, 1, 1, "f32", 1.0, 0.5, ""), ("f32", "f32", 40, 47, 8, "f16", 2.0, 0.5, "ids weight"), ("f32", "f32", 33, 64, 64, "f32", 4.0, 1.0, "pad"),
    ("f32", "f32", 70, 256, 16, "bf16", 4.0, 0.9, "ids list weight"), ("f32", "f32", 9, 1000, 3, "f16", 2.5, 0.5, ""), ("bf16", "bf16", 50, 172, 10, "f16", 1.0, 0.3, "ids list pad"),
    ("bf16", "f32", 20, 513, 50, "f32", 2.0, 0.5, "twice"), ("f16", "f16", 30, 1024, 64, "f16", 2.0, 0.9, "ids scale weight"), ("f16", "f16", 12, 1025, 7, "bf16", 3.0, 0.5, "twice list"),
    ("f32", "f32", 6, 2049, 32, "f16", 2.0, 0.5, "ids"), ("bf16", "bf16", 5, 8193, 16, "f16", 2.0, 0.5, ""), ("f16", "f32", 4, 16_385, 64, "f16", 2.0, 0.7, "ids twice"),
    ("bf16", "bf16", 3, 50_003, 32, "f16", 2.0, 0.5, "list"), ("f32", "f32", 2, 70_001, 8, "f32", 2.0, 0.5, "ids twice"), ("bf16", "bf16", 2, 131_072, 50, "f16", 4.0, 0.5, ""),
    ("f32", "f32", 30, 100, 0, "f32", 2.0, 0.5, "weight"), ("bf16", "bf16", 30, 100, 5, "f16", 2.0, 0.0, "ids"), ("f32", "f32", 20, 300, 5, "f16", 2.0, 1.0, "nolabels"),
    ("f32", "f32", 300, 8, 2, "f16", 2.0, 0.5, "ids list"), ("f16", "f16", 100, 3, 3, "f32", 1.5, 0.5, "twice"),
]


@gpu
@pytest.mark.parametrize("dtype, dh_type, n, d, k, top, temp, alpha, options", DISTILL)
def test_distill_loss(B, dtype, dh_type, n, d, k, top, temp, alpha, options):
    r = np.random.default_rng(n + d + k)
    pad = 3 if "pad" in options else 0
    h = values(r, n, d, dtype, pad, 3.0)
    table = 2 * n + 1 if "ids" in options else n
    ids = r.integers(0, table, n).astype(np.int32) if "ids" in options else None
    if ids is not None and n > 4:
        ids[[0, 2]] = (-1, table)                                   # nodes without a teacher
    idx = np.stack([r.permutation(max(d, k))[:k] for _ in range(table)]).astype(np.int32).reshape(table, k)
    idx[r.random(idx.shape) < 0.05] = -1
    idx[r.random(idx.shape) < 0.03] = d                             # classes that do not exist
    if "twice" in options and k > 2:
        idx[:, 1] = idx[:, 0]
        idx[::2, 2] = idx[::2, 0]
    val = torch.from_numpy(4 * r.standard_normal((table, k))).to(T[top])
    idx[table // 2] = -1
    label = None if "nolabels" in options else r.integers(-1, d, n).astype(np.int32)
    if label is not None and n > 6:
        label[5] = d
        if k:
            label[6] = idx[ids[6] if ids is not None else 6, 0]     # the label among the teacher's classes
    weight = torch.from_numpy(r.random(n)).float() if "weight" in options else None
    scale = 64.0 if "scale" in options else 0.5
    rows = np.sort(r.permutation(n)[:max(1, n - n // 4)]).astype(np.int32) if "list" in options else np.arange(n, dtype=np.int32)
    dev = dict(ids=cuda(torch.from_numpy(ids)) if ids is not None else None, idx=torch.from_numpy(idx).cuda() if k else None, val=val.cuda() if k else None,
               label=torch.from_numpy(label).cuda() if label is not None else None, weight=cuda(weight))
    listed = torch.from_numpy(rows).cuda() if "list" in options else None
    count = torch.full((1,), len(rows), dtype=torch.int64, device="cuda") if "list" in options else None

    def call(h, loss, dh, dh_type, bound=None):
        B.fg_distill_loss(h, stride(h), code(B, dtype), listed, count, bound or len(rows), n, d, dev["ids"], dev["idx"], dev["val"], code(B, top), table, k, dev["label"], temp, alpha,
                          dev["weight"], scale, loss, dh, stride(dh) if dh is not None else 0, code(B, dh_type))
        torch.cuda.synchronize()

    hd, loss, dh = h.cuda(), torch.full((n,), -77.0, device="cuda"), sentinel(n, d, dh_type, pad).cuda()
    call(hd, loss, dh, dh_type)
    node = ids[rows] if ids is not None else rows
    there = (node >= 0) & (node < table)
    t_idx = torch.from_numpy(np.where(there[:, None], idx[np.clip(node, 0, table - 1)], -1)) if k else None
    t_val = val[np.clip(node, 0, table - 1)] if k else None
    want, off, grad, grad_off = R.distill(h[rows, :d], t_idx, t_val, label[rows] if label is not None else None, temp, alpha, weight[rows] if weight is not None else None, scale)
    rest = np.setdiff1d(np.arange(n), rows)
    assert bool((loss.cpu()[rest] == -77).all()) and bool((dh.cpu()[rest] == -77).all()) and bool((dh.cpu()[:, d:] == -77).all())
    close(loss.cpu()[rows], want, off + 2.0 ** -24 * want.abs(), "loss")
    close(dh.cpu()[rows, :d], grad, grad_off + HALF[dh_type] * grad.abs() + TINY[dh_type], "dh")
    # one of the two, again, over h itself: the same bits
    again, dh2 = torch.full((n,), -77.0, device="cuda"), sentinel(n, d, dh_type, pad).cuda()
    call(hd, again, None, dh_type)
    call(hd, None, dh2, dh_type)
    assert torch.equal(again, loss) and torch.equal(dh2, dh)
    if dh_type == dtype:
        call(hd, None, hd, dh_type)
        assert torch.equal(hd[rows, :d], dh[rows, :d]) and torch.equal(hd.cpu()[rest][:, :d], h[rest][:, :d])


@gpu
@pytest.mark.parametrize("d", [5, 70, 3000, 20_000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_distill_loss_of_masked_classes(B, dtype, d):
    """Rows whose masks leave one class, none, or not the teacher's; the type's lowest value; infinities and NaN where nothing may read them."""
    inf, low = math.inf, float(torch.finfo(T[dtype]).min)
    h = torch.randn(8, d, generator=torch.Generator().manual_seed(1)).to(T[dtype])
    idx, val = torch.full((8, 2), -1, dtype=torch.int32), torch.full((8, 2), math.nan)
    label = torch.full((8,), -1, dtype=torch.int32)
    h[0, 1:] = -inf                                       # one class is left, the teacher's and the label
    idx[0, 0], val[0, 0], label[0] = 0, 1.0, 0
    h[1] = math.nan                                       # neither teacher nor label: nothing is read
    h[2, 3] = -inf                                        # the label's class is masked: an infinite loss, finite gradients
    label[2] = 3
    h[3, :2] = low                                        # the type's lowest value in a masked place
    idx[3], val[3] = torch.tensor([2, 3]), torch.tensor([0.5, -0.5])
    idx[4], val[4], label[4] = torch.tensor([1, 2]), torch.tensor([-inf, 2.0]), 2      # a stored value of -infinity has no share
    idx[5], val[5] = torch.tensor([1, 2]), torch.tensor([-inf, -inf])                  # no share at all: no teacher
    h[6, 0] = math.nan                                    # a NaN logit shows
    label[6] = 1
    h[7, 4], idx[7], val[7] = -inf, torch.tensor([4, 1]), torch.tensor([-inf, 1.0])    # a masked class without a share costs nothing
    loss, dh = torch.full((8,), -77.0, device="cuda"), torch.full((8, d), -77.0, dtype=T[dtype], device="cuda")
    B.fg_distill_loss(h.cuda(), stride(h), code(B, dtype), None, None, 8, 8, d, None, idx.cuda(), val.cuda(), B.FG_F32, 8, 2, label.cuda(), 2.0, 0.5, None, 1.0, loss, dh, stride(dh),
                      code(B, dtype))
    torch.cuda.synchronize()
    loss, dh = loss.cpu(), dh.cpu().double()
    assert float(loss[0]) == 0 and not bool(dh[0].any())
    assert float(loss[1]) == 0 and not bool(dh[1].any()) and float(loss[5]) == 0 and not bool(dh[5].any())
    assert float(loss[2]) == inf and bool(torch.isfinite(dh[2]).all()) and float(dh[2, 3]) == -0.5
    assert bool(torch.isnan(loss[6])) and bool(torch.isnan(dh[6]).all())
    for i in (2, 3, 4, 7):
        want, off, grad, grad_off = R.distill(h[i:i + 1], idx[i:i + 1], val[i:i + 1], label[i:i + 1], 2.0, 0.5, None, 1.0)
        if i != 2:
            close(loss[i:i + 1], want, off + 2.0 ** -24 * want.abs(), f"loss of row {i}")
        close(dh[i:i + 1], grad, grad_off + HALF[dtype] * grad.abs() + TINY[dtype], f"dh of row {i}")


@gpu
@pytest.mark.parametrize("d", [1, 40, 500, 3000, 20_000])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_distill_loss_of_rows_without_a_class_to_choose(B, dtype, d):
    """All classes masked: NaN where there is a teacher or a label, nothing where there is neither; the rows beside them as if they were not there."""
    h = torch.randn(5, d, generator=torch.Generator().manual_seed(2)).to(T[dtype])
    h[:3] = -math.inf
    h[3, d // 2] = math.inf
    idx, val = torch.tensor([[0], [-1], [-1], [0], [d - 1]], dtype=torch.int32), torch.zeros(5, 1)
    label = torch.tensor([-1, 0, -1, -1, 0], dtype=torch.int32)
    for temperature in (1.0, 2.0, 3.0):
        loss, dh = torch.full((5,), -77.0, device="cuda"), torch.full((5, d), -77.0, dtype=T[dtype], device="cuda")
        B.fg_distill_loss(h.cuda(), stride(h), code(B, dtype), None, None, 5, 5, d, None, idx.cuda(), val.cuda(), B.FG_F32, 5, 1, label.cuda(), temperature, 0.5, None, 1.0, loss, dh,
                          stride(dh), code(B, dtype))
        torch.cuda.synchronize()
        loss, dh = loss.cpu(), dh.cpu()
        for i in (0, 1, 3):
            assert bool(torch.isnan(loss[i])) and bool(torch.isnan(dh[i]).all()), i
        assert float(loss[2]) == 0 and not bool(dh[2].any())
        want, off, grad, grad_off = R.distill(h[4:], idx[4:], val[4:], label[4:], temperature, 0.5, None, 1.0)
        close(loss[4:], want, off + 2.0 ** -24 * want.abs(), "loss")
        close(dh[4:], grad, grad_off + HALF[dtype] * grad.abs() + TINY[dtype], "dh")


@gpu
def test_distill_loss_of_no_rows(B):
    h, loss = torch.ones(3, 8, device="cuda"), torch.full((3,), -77.0, device="cuda")
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    B.fg_distill_loss(h, 32, B.FG_F32, None, count, 3, 3, 8, None, None, None, B.FG_F32, 0, 0, None, 2.0, 0.5, None, 1.0, loss, h, 32, B.FG_F32)
    B.fg_distill_loss(h, 32, B.FG_F32, None, None, 0, 3, 8, None, None, None, B.FG_F32, 0, 0, None, 2.0, 0.5, None, 1.0, loss, h, 32, B.FG_F32)
    torch.cuda.synchronize()
    assert bool((h == 1).all()) and bool((loss == -77).all())
