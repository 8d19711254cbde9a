"""The calls of a typed layer (fg_group_rows, fg_linear_grouped and its gradients, fg_residual_norm and its gradients, fg_dropout,
fg_quantize_rows) against plain 64-bit statements of them, at the sizes and masks where they can go wrong.

Tolerances. A sum of K products in fp32 is off by at most K steps of 2^-24 of the sum of the products' magnitudes, whatever its order; twice
that is granted (2^-23), the matrix cores' sums need not round to nearest. A result rounded to a type is off by half a step of it besides
(bf16 2^-8 / 2 ...: `HALF`)."""
import math

import numpy as np
import pytest
import torch

from tests import typed_reference as R

T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 0.0, "f16": 2.0 ** -25, "bf16": 0.0}      # half the distance of the smallest fp16 numbers


@pytest.fixture(scope="module")
def B():
    from paper_2301_07482_amd import binding
    return binding


def code(B, name):
    return {"f32": B.FG_F32, "f16": B.FG_F16, "bf16": B.FG_BF16, "e4m3": B.FG_E4M3}[name]


def cuda(t):
    return t.cuda() if t is not None else None


def matrix(r, n, d, dtype, pad=0, scale=1.0):
    """[n, d] host values in a buffer of rows d + pad long (pad elements of NaN, which nothing may read into a result)."""
    full = torch.full((n, d + pad), float("nan"), dtype=T[dtype])
    full[:, :d] = torch.from_numpy(r.standard_normal((n, d)) * scale).to(T[dtype])
    return full


def sentinel(n, d, dtype, pad=0):
    return torch.full((n, d + pad), -77.0, dtype=dtype if isinstance(dtype, torch.dtype) else T[dtype])


def close(got, want, tolerance, what):
    off = (got.double() - want).abs()
    bad = ~(off <= tolerance)
    assert not bool(bad.any()), f"{what}: off by {float(off[bad].max()):.3e} where {float(tolerance[bad].min() if tolerance.ndim else tolerance):.3e} is allowed, {int(bad.sum())} values"


def stride(t):
    return t.stride(0) * t.element_size()


# ---- refusals: on the host, before anything is launched ----

def refused(B, fn, *a, **k):
    with pytest.raises(B.FgError) as e:
        fn(*a, **k)
    assert B.fg_last_error() != ""
    return e.value.code


def test_refusals(B):
    P = 4096
    grp = lambda **k: B.fg_group_rows(**{**dict(groups=P, n_table=10, ids=None, n_positions=10, rows=None, n_rows=None, max_rows=10, n_groups=4, order=P,
                                                offsets=P, ws=P, ws_bytes=1 << 30), **k})
    for bad in (dict(max_rows=-1), dict(n_groups=0), dict(n_groups=1025), dict(groups=None), dict(order=None), dict(offsets=None), dict(ws=None),
                dict(offsets=P + 4), dict(order=P + 2), dict(ws=P + 8), dict(n_table=-1), dict(max_rows=1 << 31)):
        assert refused(B, grp, **bad) == B.FG_ERR_INVALID_ARG, bad
    assert refused(B, grp, ws_bytes=16) == B.FG_ERR_SHAPE
    assert B.fg_group_rows_workspace_bytes(-1, 4) == 0 and B.fg_group_rows_workspace_bytes(10, 1025) == 0

    lin = lambda **k: B.fg_linear_grouped(**{**dict(x=P, x_rows=10, x_stride=256, dtype=B.FG_F32, x_scale=None, src_ids=None, order=P, offsets=P, max_rows=10,
                                                    n_groups=4, d_in=64, d_out=64, W=P, w_scale=None, bias=None, relu=0, h_out=P, n_out=10,
                                                    out_stride=256, out_dtype=B.FG_F32), **k})
    for bad, want in ((dict(x=None), 1), (dict(W=None), 1), (dict(h_out=None), 1), (dict(offsets=None), 1), (dict(n_groups=0), 1), (dict(max_rows=-1), 1),
                      (dict(d_in=62), 2), (dict(d_out=62), 2), (dict(d_in=0), 2), (dict(x_stride=128), 2), (dict(out_stride=128), 2),
                      (dict(x=P + 4), 1), (dict(W=P + 8), 1), (dict(h_out=P + 4), 1), (dict(x_stride=264), 1), (dict(bias=P + 2), 1), (dict(dtype=7), 3),
                      (dict(out_dtype=B.FG_BF16), 3), (dict(out_dtype=B.FG_E4M3), 3), (dict(x_scale=P), 1), (dict(dtype=B.FG_E4M3), 1),
                      (dict(dtype=B.FG_BF16, d_in=60), 2), (dict(dtype=B.FG_BF16, d_out=60), 2),
                      (dict(dtype=B.FG_E4M3, x_scale=P, w_scale=P, d_in=72), 2), (dict(dtype=B.FG_E4M3, x_scale=P), 1)):
        assert refused(B, lin, **bad) == want, bad

    bw = lambda **k: B.fg_linear_grouped_backward(**{**dict(x=P, x_rows=10, x_stride=256, dtype=B.FG_F32, src_ids=None, dh=P, dh_stride=256, dh_dtype=B.FG_F32,
                                                            h=None, h_stride=0, n=10, order=P, offsets=P, max_rows=10, n_groups=4, d_in=64, d_out=64, W=P,
                                                            dx=P, dx_stride=256, dx_dtype=B.FG_F32, dw=P, db=P, ws=P, ws_bytes=1 << 40), **k})
    for bad, want in ((dict(x=None), 1), (dict(dh=None), 1), (dict(W=None), 1), (dict(dx=None, dw=None, db=None), 1), (dict(ws=None), 1), (dict(ws_bytes=0), 2),
                      (dict(dtype=B.FG_E4M3), 3), (dict(dh_dtype=B.FG_BF16), 3), (dict(dx_dtype=B.FG_F16), 3), (dict(d_in=2), 2), (dict(dh_stride=128), 2),
                      (dict(h=P, h_stride=128), 2), (dict(dx_stride=16), 2), (dict(dw=P + 4), 1), (dict(n_groups=2000), 1), (dict(ws=P + 4), 1)):
        assert refused(B, bw, **bad) == want, bad
    assert B.fg_linear_grouped_backward_workspace_bytes(B.FG_E4M3, 10, 4, 64, 64) == 0

    assert refused(B, lin, max_rows=B.FG_MAX_GROUPED_ROWS + 1, n_out=1 << 30) == B.FG_ERR_INVALID_ARG
    assert refused(B, bw, max_rows=B.FG_MAX_GROUPED_ROWS + 1, n=1 << 30) == B.FG_ERR_INVALID_ARG
    assert B.fg_linear_grouped_backward_workspace_bytes(B.FG_F32, B.FG_MAX_GROUPED_ROWS + 1, 4, 64, 64) == 0

    drop = lambda **k: B.fg_dropout(**{**dict(x=P, x_stride=256, dtype=B.FG_F32, rows=None, n_rows=None, max_rows=10, n=10, d=64, p=0.5, key=1, out=P,
                                              out_stride=256), **k})
    for bad, want in ((dict(x=None), 1), (dict(out=None), 1), (dict(p=-0.1), 1), (dict(p=1.1), 1), (dict(p=float("nan")), 1), (dict(dtype=3), 3), (dict(d=0), 2),
                      (dict(x_stride=128), 2), (dict(out_stride=255), 2), (dict(x=P + 2), 1), (dict(max_rows=11), 2), (dict(max_rows=-1), 1)):
        assert refused(B, drop, **bad) == want, bad

    norm = lambda **k: B.fg_residual_norm(**{**dict(x=P, x_stride=256, dtype=B.FG_F32, residual=None, residual_stride=0, sum_dtype=B.FG_F32, rows=None, n_rows=None,
                                                    max_rows=10, n=10, d=64, p=0.0, key=1, weight=None, eps=1e-6, sum_out=None, sum_stride=0, y=P,
                                                    y_stride=256, y_dtype=B.FG_F32, y_scale=None, rstd_out=None), **k})
    for bad, want in ((dict(x=None), 1), (dict(y=None), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(y_scale=P), 1), (dict(y_dtype=B.FG_E4M3), 1),
                      (dict(y_dtype=B.FG_BF16), 3), (dict(sum_dtype=B.FG_F16), 3), (dict(dtype=3), 3), (dict(d=16385), 2), (dict(d=-4), 2), (dict(p=2.0), 1),
                      (dict(residual=P, residual_stride=128), 2), (dict(sum_out=P, sum_stride=4), 2), (dict(weight=P + 1), 1), (dict(rstd_out=P + 2), 1)):
        assert refused(B, norm, **bad) == want, bad

    nbw = lambda **k: B.fg_residual_norm_backward(**{**dict(dy=P, dy_stride=256, grad_dtype=B.FG_F32, sum_=P, sum_stride=256, sum_dtype=B.FG_F32, rstd=P, weight=None,
                                                            dsum_in=None, dsum_in_stride=0, rows=None, n_rows=None, max_rows=10, n=10, d=64, p=0.0, key=1,
                                                            dsum_out=P, dsum_stride=256, dx=None, dx_stride=0, dw=P, ws=P, ws_bytes=1 << 30), **k})
    for bad, want in ((dict(dy=None), 1), (dict(sum_=None), 1), (dict(rstd=None), 1), (dict(dsum_out=None), 1), (dict(ws=None), 1), (dict(ws_bytes=8), 2),
                      (dict(grad_dtype=3), 3), (dict(sum_dtype=9), 3), (dict(dx=P, dx_stride=8), 2), (dict(dsum_in=P, dsum_in_stride=8), 2), (dict(d=20000), 2)):
        assert refused(B, nbw, **bad) == want, bad

    qnt = lambda **k: B.fg_quantize_rows(**{**dict(x=P, x_stride=256, dtype=B.FG_F32, n_rows=10, d=64, q=P, q_stride=64, scale=P), **k})
    for bad, want in ((dict(x=None), 1), (dict(q=None), 1), (dict(scale=None), 1), (dict(dtype=3), 3), (dict(q_stride=63), 2), (dict(d=0), 2), (dict(n_rows=-1), 1)):
        assert refused(B, qnt, **bad) == want, bad


def test_workspaces_of_a_bound_serve_every_smaller_call(B):
    sizes = sorted({*range(0, 400), *range(4000, 4200), *range(8100, 8300), *range(16300, 16500), *range(30000, 70000, 1000), 70000, 10 ** 6, 3 * 10 ** 6, 10 ** 7})
    for need in (lambda n: B.fg_group_rows_workspace_bytes(n, 37), lambda n: B.fg_residual_norm_backward_workspace_bytes(n, 88),
                 *(lambda n, t=t, g=g, a=a, b=b: B.fg_linear_grouped_backward_workspace_bytes(t, n, g, a, b) for t in (0, 1, 2) for g in (1, 5, 300)
                   for a, b in ((96, 256), (264, 520), (1024, 1024), (2048, 4096), (4096, 4096), (8, 65536)))):
        got = [need(n) for n in sizes]
        assert got == sorted(got) and min(got) >= 0


# ---- fg_group_rows ----

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("n, n_groups, mode", [(1, 1, "all"), (1, 1024, "list"), (63, 3, "list"), (64, 2, "all"), (1000, 7, "ids"), (1025, 1, "all"), (8192, 64, "ids"), (6144, 9, "all"), (6145, 9, "all"),
                                               (8193, 5, "list"), (20000, 1024, "ids"), (70001, 33, "list"), (300000, 3, "ids"), (2500000, 17, "all")])
def test_group_rows(B, n, n_groups, mode):
    r = np.random.default_rng(n + n_groups)
    table = n if mode != "ids" else 2 * n + 5
    groups = r.integers(-1, n_groups + 1, table).astype(np.int32)      # some without a group
    ids = r.integers(-2, table + 2, n).astype(np.int32) if mode == "ids" else None
    rows = None if mode == "all" else np.sort(r.choice(n, max(1, (3 * n) // 4), replace=False)).astype(np.int32)
    if rows is not None and n > 10:
        rows[5], rows[-1] = -3, n + 4                                  # bad entries are left out
    bound = len(rows) if rows is not None else n
    for count in {bound, bound // 2, 0}:
        listed = (rows if rows is not None else np.arange(n))[:count]
        v = np.where((listed >= 0) & (listed < n), listed, 0)
        v = np.where((listed >= 0) & (listed < n), ids[v] if ids is not None else v, -1)
        g = np.where((v >= 0) & (v < table), groups[np.clip(v, 0, table - 1)], -1)
        has = (g >= 0) & (g < n_groups)
        want = listed[has][np.argsort(g[has], kind="stable")]
        offsets = np.searchsorted(np.sort(g[has]), np.arange(n_groups + 1))
        ws = torch.zeros(B.fg_group_rows_workspace_bytes(bound, n_groups), dtype=torch.uint8, device="cuda")
        order = torch.full((bound + 3,), -9, dtype=torch.int32, device="cuda")
        off = torch.full((n_groups + 2,), -9, dtype=torch.int64, device="cuda")
        args = (torch.from_numpy(groups).cuda(), table, cuda(torch.from_numpy(ids)) if ids is not None else None, n,
                cuda(torch.from_numpy(rows)) if rows is not None else None, torch.tensor([count], device="cuda"), bound, n_groups, order, off, ws, ws.numel())
        B.fg_group_rows(*args)
        torch.cuda.synchronize()
        assert off.tolist() == offsets.tolist() + [-9]
        assert np.array_equal(order.cpu().numpy(), np.concatenate([want, np.full(bound + 3 - len(want), -9)]))


# ---- fg_linear_grouped ----

def layout(r, n, n_groups, share=0.8, empty=()):
    """Listed positions in group order, with their offsets; groups in `empty` have none."""
    rows = np.sort(r.choice(n, max(1, int(n * share)), replace=False))
    g = r.choice([i for i in range(n_groups) if i not in empty], len(rows), p=None)
    return rows[np.argsort(g, kind="stable")].astype(np.int32), np.searchsorted(np.sort(g), np.arange(n_groups + 1)).astype(np.int64)


LINEAR = [  # dtype, out, n, groups, d_in, d_out, options
    ("f32", "f32", 1, 1, 4, 4, ""), ("f32", "f32", 70, 3, 64, 64, "bias relu"), ("f32", "f32", 333, 5, 100, 256, "bias relu src pad"),
    ("f32", "f32", 1000, 2, 36, 132, "order0"), ("f32", "f32", 129, 40, 260, 20, "bias src"), ("f32", "f32", 2100, 4, 128, 96, "bias relu"),
    ("f16", "f16", 1, 1, 8, 8, ""), ("f16", "f32", 300, 3, 72, 136, "bias src pad"), ("f16", "f16", 777, 9, 768, 64, "bias relu"),
    ("bf16", "bf16", 257, 4, 64, 128, "bias relu pad"), ("bf16", "f32", 65, 64, 200, 24, "bias"), ("bf16", "f16", 500, 1, 1024, 256, "order0"),
    ("bf16", "bf16", 5000, 6, 264, 520, "bias relu src"), ("f16", "f16", 3000, 2, 520, 264, "relu"),
    ("e4m3", "bf16", 1, 1, 16, 8, ""), ("e4m3", "f32", 300, 3, 80, 136, "bias src pad"), ("e4m3", "bf16", 1500, 7, 1024, 264, "bias relu"),
    ("e4m3", "f16", 130, 33, 48, 40, "bias"), ("e4m3", "f32", 2600, 2, 528, 512, "relu"),
]


def linear_inputs(B, dtype, out, n, n_groups, d_in, d_out, options):
    r = np.random.default_rng(n * 7 + d_in + d_out)
    opt = options.split()
    share = 1.0 if "order0" in opt else 0.8
    order, offsets = layout(r, n, n_groups, share, empty=(1,) if n_groups > 2 else ())
    if "order0" in opt:
        order = np.arange(n, dtype=np.int32)
    src = r.integers(0, 2 * n, n).astype(np.int32) if "src" in opt else None
    pad = 16 if "pad" in opt else 0
    rows = 2 * n if src is not None else n
    W = torch.from_numpy(r.standard_normal((n_groups, d_in, d_out)) / math.sqrt(d_in)).float()
    bias = torch.from_numpy(r.standard_normal((n_groups, d_out))).float() if "bias" in opt else None
    if dtype == "e4m3":
        q, xs = R.quantise(torch.from_numpy(r.standard_normal((rows, d_in)) * np.exp(r.standard_normal((rows, 1)))))
        x = torch.zeros(rows, d_in + pad, dtype=torch.float8_e4m3fn)
        x[:, :d_in] = q.to(torch.float8_e4m3fn)
        wq, ws = R.quantise(W.transpose(1, 2).contiguous().reshape(n_groups * d_out, d_in))
        dev = dict(x=x, x_scale=xs, W=wq.to(torch.float8_e4m3fn), w_scale=ws)
        x64 = q.double() * xs.double()[:, None]
        W64 = (wq.double() * ws.double()[:, None]).reshape(n_groups, d_out, d_in).transpose(1, 2)
    else:
        x = matrix(r, rows, d_in, dtype, pad)
        dev = dict(x=x, x_scale=None, W=W.to(T[dtype]), w_scale=None)
        x64, W64 = x[:, :d_in], dev["W"]
    return order, offsets, src, bias, dev, x64, W64, "relu" in opt, pad


@gpu
@pytest.mark.parametrize("dtype, out, n, n_groups, d_in, d_out, options", LINEAR)
def test_linear_grouped(B, dtype, out, n, n_groups, d_in, d_out, options):
    order, offsets, src, bias, dev, x64, W64, relu, pad = linear_inputs(B, dtype, out, n, n_groups, d_in, d_out, options)
    want, size = R.grouped_linear(x64, W64, bias, order.tolist(), offsets.tolist(), src.tolist() if src is not None else None, relu)
    x, W = dev["x"].cuda(), dev["W"].cuda()
    h = sentinel(n, d_out, out, pad).cuda()
    bad = order.copy()
    n_rows = len(order)
    ordered = None if "order0" in options else torch.from_numpy(order).cuda()
    B.fg_linear_grouped(x, len(x), stride(x), code(B, dtype), cuda(dev["x_scale"]), cuda(torch.from_numpy(src)) if src is not None else None, ordered,
                        torch.from_numpy(offsets).cuda(), n_rows, n_groups, d_in, d_out, W, cuda(dev["w_scale"]), cuda(bias), int(relu), h, n,
                        stride(h), code(B, out))
    torch.cuda.synchronize()
    h = h.cpu()
    rest = np.setdiff1d(np.arange(n), order)
    assert bool((h[rest] == -77).all()) and bool((h[:, d_out:] == -77).all()), "rows that are not listed, and the ends of the rows, stay"
    close(h[order.astype(np.int64), :d_out], want, (d_in + 8) * 2.0 ** -23 * size + HALF[out] * want.abs() + TINY[out], f"{dtype} {n} x {d_in} x {d_out}")
    assert np.array_equal(bad, order)


def large(dtype, out, n, n_groups, d_in, d_out, options=""):
    """A call whose tiles are several to a workgroup, on the GPU in fp64 (products of contiguous operands)."""
    g = torch.Generator(device="cuda").manual_seed(n + d_in + d_out)
    kw = dict(device="cuda", generator=g)
    rows = torch.randperm(n, **kw)[:n - n // 7]
    types = torch.randint(0, n_groups, (len(rows),), **kw).sort()
    order = rows[torch.argsort(torch.rand(len(rows), **kw))].int()
    offsets = torch.searchsorted(types.values, torch.arange(n_groups + 1, device="cuda"))
    src = torch.randint(0, n, (n,), **kw).int() if "src" in options else None
    x = torch.randn(n, d_in, **kw)
    W = torch.randn(n_groups, d_in, d_out, **kw) / math.sqrt(d_in)
    return order, offsets, src, x, W, torch.randn(n_groups, d_out, **kw)


LARGE = [  # tiles of 256, 128 and 64 rows, one step of the contraction and several, whole steps and parts of one
    ("bf16", "bf16", 33_500, 3, 64, 264, "src relu"), ("bf16", "f32", 70_001, 2, 72, 256, ""), ("f16", "f16", 40_000, 5, 200, 512, "src"),
    ("f16", "f32", 36_000, 40, 136, 264, "relu"), ("bf16", "bf16", 33_100, 4, 328, 520, ""), ("bf16", "bf16", 70_500, 3, 40, 128, "relu"), ("f16", "f16", 71_000, 9, 264, 72, "src"),
    ("bf16", "f32", 72_000, 2, 64, 64, ""), ("f16", "f16", 90_000, 1024, 136, 40, "src relu"), ("bf16", "bf16", 130_000, 1, 8, 16, ""),
    ("e4m3", "bf16", 70_000, 3, 128, 256, "src relu"), ("e4m3", "f32", 40_000, 4, 272, 512, "relu"), ("e4m3", "bf16", 36_000, 7, 400, 264, ""), ("e4m3", "f16", 90_000, 2, 16, 48, ""),
    ("e4m3", "f32", 170_000, 1024, 64, 264, ""), ("f16", "f16", 160_000, 1024, 40, 136, "src"),
    ("f32", "f32", 50_000, 3, 100, 256, "src relu"), ("f32", "f32", 34_000, 60, 36, 132, ""), ("f32", "f32", 70_000, 2, 260, 64, "relu"),
]


@gpu
@pytest.mark.parametrize("dtype, out, n, n_groups, d_in, d_out, options", LARGE)
def test_linear_grouped_of_many_rows(B, dtype, out, n, n_groups, d_in, d_out, options):
    order, offsets, src, x, W, bias = large(dtype, out, n, n_groups, d_in, d_out, options)
    relu = "relu" in options
    xs = ws = None
    if dtype == "e4m3":
        xq, xs = R.quantise(x)
        wq, ws = R.quantise(W.transpose(1, 2).contiguous().reshape(n_groups * d_out, d_in))
        x64, W64 = xq.double() * xs.double()[:, None], (wq.double() * ws.double()[:, None]).reshape(n_groups, d_out, d_in).transpose(1, 2).contiguous()
        x, W = xq.to(torch.float8_e4m3fn), wq.to(torch.float8_e4m3fn)
    else:
        x, W = x.to(T[dtype]), W.to(T[dtype])
        x64, W64 = x.double(), W.double()
    h = torch.full((n, d_out), -77.0, dtype=T[out], device="cuda")
    # twice, the second time over the first one's results: nothing may depend on what was there
    for _ in range(2):
        B.fg_linear_grouped(x, n, stride(x), code(B, dtype), xs, src, order, offsets, len(order), n_groups, d_in, d_out, W, ws, bias, int(relu), h, n, stride(h),
                            code(B, out))
    torch.cuda.synchronize()
    want, size = torch.full((n, d_out), -77.0, dtype=torch.float64, device="cuda"), torch.zeros(n, d_out, dtype=torch.float64, device="cuda")
    at = offsets.tolist()
    for g in range(n_groups):
        pos = order[at[g]:at[g + 1]].long()
        a = x64[src[pos].long() if src is not None else pos]
        v = torch.mm(a, W64[g]) + bias[g].double()
        want[pos] = v.clamp_min(0) if relu else v
        size[pos] = torch.mm(a.abs(), W64[g].abs()) + bias[g].double().abs()
    close(h, want, (d_in + 8) * 2.0 ** -23 * size + HALF[out] * want.abs() + TINY[out], f"{dtype} {n} x {d_in} x {d_out}")


@gpu
@pytest.mark.parametrize("dtype, out, n, n_groups, d_in, d_out", [("bf16", "bf16", 40_000, 3, 264, 136), ("f16", "f32", 70_000, 2, 256, 64), ("bf16", "f32", 33_500, 40, 520, 264),
                                                                   ("f32", "f32", 45_000, 3, 88, 256), ("bf16", "bf16", 50_000, 1, 64, 64), ("f16", "f16", 9_000, 300, 72, 40),
                                                                   ("f32", "f32", 33_000, 5, 132, 400), ("bf16", "bf16", 66_000, 5, 520, 520),
                                                                   ("f16", "f32", 30_000, 3, 1160, 1032)])
def test_linear_grouped_backward_of_many_rows(B, dtype, out, n, n_groups, d_in, d_out):
    order, offsets, _, x, W, _ = large(dtype, out, n, n_groups, d_in, d_out)
    x, W = x.to(T[dtype]), W.to(T[dtype])
    dh, h = torch.randn(n, d_out, device="cuda").to(T[dtype]), torch.randn(n, d_out, device="cuda").to(T[dtype])
    dx = torch.full((n, d_in), -77.0, dtype=T[out], device="cuda")
    dw, db = torch.full((n_groups, d_in, d_out), -77.0, device="cuda"), torch.full((n_groups, d_out), -77.0, device="cuda")
    ws = torch.full((B.fg_linear_grouped_backward_workspace_bytes(code(B, dtype), len(order), n_groups, d_in, d_out),), 255, dtype=torch.uint8, device="cuda")
    for mask in (h, None):
        for _ in range(2):
            B.fg_linear_grouped_backward(x, n, stride(x), code(B, dtype), None, dh, stride(dh), code(B, dtype), mask, stride(h) if mask is not None else 0, n, order, offsets,
                                         len(order), n_groups, d_in, d_out, W, dx, stride(dx), code(B, out), dw, db, ws, ws.numel())
        torch.cuda.synchronize()
        z = dh.double() if mask is None else torch.where(h > 0, dh.double(), torch.zeros((), dtype=torch.float64, device="cuda"))
        at = offsets.tolist()
        for g in range(n_groups):
            pos = order[at[g]:at[g + 1]].long()
            zg, xg, wt = z[pos], x[pos].double(), W[g].double().T.contiguous()
            want = torch.mm(zg, wt)
            close(dx[pos], want, (d_out + 8) * 2.0 ** -23 * torch.mm(zg.abs(), wt.abs()) + HALF[out] * want.abs() + TINY[out], "dx")
            # rows' sums in fp32: a rounding of 2^-24 of the running sum a row at most, granted twice as everywhere here
            rows = len(pos) + 16
            xt = xg.T.contiguous()
            want = torch.mm(xt, zg)
            close(dw[g], want, rows * 2.0 ** -23 * torch.mm(xt.abs(), zg.abs()) + 2.0 ** -24 * want.abs(), "dW")
            close(db[g], zg.sum(0), rows * 2.0 ** -23 * zg.abs().sum(0), "db")
            if len(pos) > 2000:      # and as near as sums of independent roundings are: the square root of that
                assert float((dw[g].double() - want).norm() / want.norm()) < 2e-6


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "e4m3"])
def test_linear_grouped_skips_what_is_out_of_range(B, dtype):
    """Entries with bad positions or rows, offsets that end before the bound or lie beyond it, non-finite rows beside others."""
    n, G, a, b = 150, 3, 64, 64
    order, offsets, src, bias, dev, x64, W64, _, _ = linear_inputs(B, dtype, "f32", n, G, a, b, "src bias")
    src[order[3]], src[order[10]] = -1, 2 * n
    good = [k for k in range(len(order)) if k not in (3, 10, 7)]
    entries = order.copy()
    entries[7] = n + 5
    x = dev["x"].clone()
    x.view(torch.uint8)[src[order[20]]] = 0x7F if dtype == "e4m3" else 0xFF      # a row of NaN: only its own output shows it
    x64 = x64.clone().double()
    x64[src[order[20]]] = float("nan")
    want, size = R.grouped_linear(x64, W64, bias, order.tolist(), offsets.tolist(), np.clip(src, 0, 2 * n - 1).tolist(), True)
    for bound, offs in ((len(order), offsets), (len(order), offsets + np.array([0] * G + [1000])), (len(order) - 40, offsets)):
        h = sentinel(n, b, "f32").cuda()
        B.fg_linear_grouped(x.cuda(), len(x), stride(x), code(B, dtype), cuda(dev["x_scale"]), torch.from_numpy(src).cuda(), torch.from_numpy(entries).cuda(),
                            torch.from_numpy(offs).cuda(), bound, G, a, b, dev["W"].cuda(), cuda(dev["w_scale"]), bias.cuda(), 1, h, n, stride(h), B.FG_F32)
        torch.cuda.synchronize()
        h = h.cpu()
        taken = [k for k in good if k < bound]
        pos = order[taken].astype(np.int64)
        clean = [i for i, k in enumerate(taken) if src[order[k]] != src[order[20]]]
        dirty = [i for i, k in enumerate(taken) if src[order[k]] == src[order[20]]]
        close(h[pos[clean]], want[taken][clean], (a + 8) * 2.0 ** -23 * size[taken][clean] + 2.0 ** -24, dtype)
        assert dirty and bool(h[pos[dirty]].isnan().all())
        assert bool((h[np.setdiff1d(np.arange(n), pos)] == -77).all())


# ---- fg_linear_grouped_backward ----

BACKWARD = [  # dtype, dh, dx, n, groups, d_in, d_out, options
    ("f32", "f32", "f32", 1, 1, 4, 4, ""), ("f32", "f32", "f32", 200, 3, 88, 64, "relu"), ("f32", "f32", "f32", 700, 5, 100, 256, "relu src pad"),
    ("f32", "f32", "f32", 90, 30, 36, 132, ""), ("f32", "f32", "f32", 9000, 2, 64, 64, "relu"), ("f32", "f32", "f32", 2500, 3, 132, 260, "relu order0"),
    ("bf16", "bf16", "bf16", 300, 4, 64, 128, "relu pad"), ("bf16", "f32", "f32", 500, 3, 200, 72, "relu src"), ("bf16", "bf16", "f32", 1200, 2, 264, 520, ""),
    ("bf16", "bf16", "bf16", 9000, 3, 136, 264, "relu"), ("bf16", "f32", "bf16", 65, 64, 72, 24, "relu"),
    ("f16", "f16", "f16", 1, 1, 8, 8, "relu"), ("f16", "f32", "f16", 333, 2, 96, 40, "relu pad"), ("f16", "f16", "f32", 5000, 3, 512, 256, "src"),
]


@gpu
@pytest.mark.parametrize("dtype, dh_type, dx_type, n, n_groups, d_in, d_out, options", BACKWARD)
def test_linear_grouped_backward(B, dtype, dh_type, dx_type, n, n_groups, d_in, d_out, options):
    r = np.random.default_rng(n + d_in + 3 * d_out)
    pad = 16 if "pad" in options else 0
    order, offsets = layout(r, n, n_groups, 1.0 if "order0" in options else 0.85, empty=(1,) if n_groups > 2 else ())
    if "order0" in options:
        order = np.arange(n, dtype=np.int32)
    src = r.integers(0, 2 * n, n).astype(np.int32) if "src" in options else None
    x, dh = matrix(r, 2 * n if src is not None else n, d_in, dtype, pad), matrix(r, n, d_out, dh_type, pad)
    h = matrix(r, n, d_out, dtype, pad) if "relu" in options else None
    W = torch.from_numpy(r.standard_normal((n_groups, d_in, d_out)) / math.sqrt(d_in)).to(T[dtype])
    rounds = T[dtype] if dtype != "f32" and dh_type == "f32" else None
    (dx, dxs), (dW, dWs), (db, dbs) = R.grouped_linear_backward(x[:, :d_in], W, dh[:, :d_out], h[:, :d_out] if h is not None else None, order.tolist(),
                                                               offsets.tolist(), src.tolist() if src is not None else None, rounds)
    got_dx = sentinel(n, d_in, dx_type, pad).cuda()
    dw, gb = torch.full((n_groups, d_in, d_out), -77.0, device="cuda"), torch.full((n_groups, d_out), -77.0, device="cuda")
    xd, dhd, hd = x.cuda(), dh.cuda(), cuda(h)
    ws = torch.zeros(B.fg_linear_grouped_backward_workspace_bytes(code(B, dtype), len(order), n_groups, d_in, d_out), dtype=torch.uint8, device="cuda")
    ordered = None if "order0" in options else torch.from_numpy(order).cuda()

    def call(**k):
        a = dict(x=xd, x_rows=len(xd), x_stride=stride(xd), dtype=code(B, dtype), src_ids=cuda(torch.from_numpy(src)) if src is not None else None, dh=dhd,
                 dh_stride=stride(dhd), dh_dtype=code(B, dh_type), h=hd, h_stride=stride(hd) if hd is not None else 0, n=n, order=ordered,
                 offsets=torch.from_numpy(offsets).cuda(), max_rows=len(order), n_groups=n_groups, d_in=d_in, d_out=d_out, W=W.cuda(), dx=got_dx,
                 dx_stride=stride(got_dx), dx_dtype=code(B, dx_type), dw=dw, db=gb, ws=ws, ws_bytes=ws.numel())
        B.fg_linear_grouped_backward(**{**a, **k})
        torch.cuda.synchronize()

    call()
    pos = order.astype(np.int64)
    out = got_dx.cpu()
    close(out[pos, :d_in], dx, (d_out + 8) * 2.0 ** -23 * dxs + HALF[dx_type] * dx.abs() + TINY[dx_type], "dx")
    assert bool((out[np.setdiff1d(np.arange(n), pos)] == -77).all()) and bool((out[:, d_in:] == -77).all())
    rows = torch.from_numpy(np.diff(offsets)).double().clamp(max=4096) + 16      # a range of rows, at these sizes fewer than 4096, in fp32, the ranges in fp64
    close(dw.cpu(), dW, rows[:, None, None] * 2.0 ** -23 * dWs + 2.0 ** -24 * dW.abs(), "dW")
    close(gb.cpu(), db, rows[:, None] * 2.0 ** -23 * dbs + 2.0 ** -24 * db.abs(), "db")
    assert n_groups <= 2 or not bool(dw[1].any()), "a group without rows has a zero gradient"
    # the parts by themselves, and the same bits again
    first = got_dx.clone(), dw.clone(), gb.clone()
    for alone in ("dx", "dw", "db"):
        for t in (got_dx, dw, gb):
            t.fill_(-77.0)
        call(**{k: None for k in ("dx", "dw", "db") if k != alone}, **({"x": None} if alone == "dx" and n % 2 else {}))
        for name, t, was in zip(("dx", "dw", "db"), (got_dx, dw, gb), first):
            assert torch.equal(t, was) if name == alone else bool((t == -77).all()), (alone, name)


@gpu
def test_linear_grouped_gradients_against_differences(B):
    """Without an activation the product is linear in each factor: the fp32 call's own differences are its gradients, up to its rounding."""
    n, G, a, b = 120, 3, 32, 48
    r = np.random.default_rng(11)
    order, offsets = layout(r, n, G)
    x, W, c = matrix(r, n, a, "f32"), torch.from_numpy(r.standard_normal((G, a, b))).float(), matrix(r, n, b, "f32")
    vx, vW = matrix(r, n, a, "f32"), torch.from_numpy(r.standard_normal((G, a, b))).float()
    od, fd, pos = torch.from_numpy(order).cuda(), torch.from_numpy(offsets).cuda(), order.astype(np.int64)

    def loss(x, W):
        h = torch.zeros(n, b, device="cuda")
        B.fg_linear_grouped(x.cuda(), n, 4 * a, B.FG_F32, None, None, od, fd, len(order), G, a, b, W.cuda(), None, None, 0, h, n, 4 * b, B.FG_F32)
        return float((h.cpu()[pos].double() * c[pos].double()).sum()), float((h.cpu()[pos].double() * c[pos].double()).abs().sum())

    dx, dw, db = torch.zeros(n, a, device="cuda"), torch.zeros(G, a, b, device="cuda"), torch.zeros(G, b, device="cuda")
    ws = torch.zeros(B.fg_linear_grouped_backward_workspace_bytes(B.FG_F32, len(order), G, a, b), dtype=torch.uint8, device="cuda")
    B.fg_linear_grouped_backward(x.cuda(), n, 4 * a, B.FG_F32, None, c.cuda(), 4 * b, B.FG_F32, None, 0, n, od, fd, len(order), G, a, b, W.cuda(), dx, 4 * a, B.FG_F32,
                                 dw, db, ws, ws.numel())
    for got, plus, minus in ((float((dx.cpu().double() * vx.double())[pos].sum()), loss(x + vx, W), loss(x - vx, W)),
                             (float((dw.cpu().double() * vW.double()).sum()), loss(x, W + vW), loss(x, W - vW))):
        # every value of h is off by (a + 8) 2^-23 of its products' magnitudes, which sqrt(a) of it bounds loosely here; x +- v is rounded once more
        room = (a + 8) * 2.0 ** -22 * 8 * (plus[1] + minus[1])
        assert abs(got - (plus[0] - minus[0]) / 2) <= room, (got, plus, minus, room)


# ---- fg_dropout ----

@gpu
@pytest.mark.parametrize("dtype, n, d, p, mode", [("f32", 1, 1, 0.5, ""), ("f32", 777, 89, 0.5, "list"), ("f32", 40, 256, 0.0, "pad"), ("f16", 300, 100, 0.1, "pad list"),
                                                  ("bf16", 129, 768, 0.2, "inplace"), ("bf16", 65, 7, 0.8, "list pad"), ("f16", 50, 33, 1.0, ""), ("f32", 9, 5000, 0.3, "list")])
def test_dropout(B, dtype, n, d, p, mode):
    r = np.random.default_rng(n + d)
    pad = 3 if "pad" in mode else 0
    x = matrix(r, n, d, dtype, pad)
    x[n // 2, d // 2] = float("inf")
    x[0, 0] = float("nan")
    rows = np.sort(r.choice(n, (3 * n + 3) // 4, replace=False)) if "list" in mode else np.arange(n)
    key = 0xDEADBEEF12345678 if n % 2 else 5
    want = R.dropout(x[:, :d], rows, p, key).float().to(T[dtype])
    xd = x.cuda()
    out = xd if "inplace" in mode else sentinel(n, d, dtype, pad).cuda()
    listed = torch.from_numpy(rows.astype(np.int32)).cuda() if "list" in mode else None
    if listed is not None:
        listed = torch.cat([listed, torch.tensor([n + 1, -1, 0], dtype=torch.int32, device="cuda")])
    count = torch.tensor([len(rows) + (2 if listed is not None else 0)], device="cuda")
    B.fg_dropout(xd, stride(xd), code(B, dtype), listed, count, len(listed) if listed is not None else n, n, d, p, key, out, stride(out))
    torch.cuda.synchronize()
    got = out.cpu()
    assert torch.equal(torch.nan_to_num(got[rows, :d].float(), nan=-1234.0), torch.nan_to_num(want.float(), nan=-1234.0))
    if "inplace" not in mode:
        assert bool((got[np.setdiff1d(np.arange(n), rows)] == -77).all()) and bool((got[:, d:] == -77).all())
    if 0 < p < 1 and n * d > 10000:      # the share that is kept: within five standard deviations of its mean
        kept = float(R.keep(key, rows, d, p).double().mean())
        q = 1 - R.threshold(p) / 65536
        assert abs(kept - q) < 5 * math.sqrt(q * (1 - q) / (len(rows) * d))


# ---- fg_residual_norm ----

NORM = [  # dtype, sum, y, n, d, p, options
    ("f32", "f32", "f32", 1, 1, 0.0, ""), ("f32", "f32", "f32", 301, 88, 0.1, "res list w"), ("f32", "f32", "e4m3", 65, 256, 0.5, "res w"),
    ("f16", "f16", "f16", 130, 100, 0.0, "res pad"), ("f16", "f32", "f16", 64, 513, 0.3, "res list pad w"), ("f16", "f16", "e4m3", 33, 1023, 0.0, "w"),
    ("bf16", "bf16", "bf16", 257, 1024, 0.5, "res w inplace"), ("bf16", "f32", "f32", 40, 2048, 0.0, "res w"), ("bf16", "bf16", "e4m3", 100, 72, 0.2, "res list w"),
    ("f32", "f32", "f32", 7, 2049, 0.0, "res"), ("bf16", "bf16", "bf16", 9, 4097, 0.1, "res w"), ("f32", "f32", "e4m3", 5, 8200, 0.0, "w"),
    ("bf16", "bf16", "e4m3", 3, 16384, 0.0, "res"), ("f32", "f32", "f32", 6, 9001, 0.5, "list"),
]


@gpu
@pytest.mark.parametrize("dtype, sum_type, y_type, n, d, p, options", NORM)
def test_residual_norm(B, dtype, sum_type, y_type, n, d, p, options):
    r = np.random.default_rng(n + d)
    opt = options.split()
    pad, eps, key = 5 if "pad" in opt else 0, 1e-6, 99
    spread = torch.from_numpy(np.exp(r.standard_normal((n, 1))))
    x = (matrix(r, n, d, dtype, pad).double() * spread).to(T[dtype])
    res = (matrix(r, n, d, sum_type, pad).double() * spread).to(T[sum_type]) if "res" in opt else None
    if n > 20:      # a row of zeros, and one so small that eps decides
        x[3, :d], x[4, :d] = 0, x[4, :d] * 2.0 ** -12
        if res is not None:
            res[3, :d], res[4, :d] = 0, res[4, :d] * 2.0 ** -12
    w = torch.from_numpy(1 + 0.2 * r.standard_normal(d)).float() if "w" in opt else None
    rows = np.sort(r.choice(n, (3 * n + 3) // 4, replace=False)) if "list" in opt else np.arange(n)
    s, rstd, y, size = R.residual_norm(x[:, :d], res[:, :d] if res is not None else None, rows, p, key, w, eps)
    xd, rd = x.cuda(), cuda(res)
    sum_out = rd if "inplace" in opt else sentinel(n, d, sum_type, pad).cuda()
    eight = y_type == "e4m3"
    yd = torch.full((n, d + pad), 0x55, dtype=torch.uint8, device="cuda") if eight else sentinel(n, d, y_type, pad).cuda()
    scale = torch.full((n,), -77.0, device="cuda") if eight else None
    got_rstd = torch.full((n,), -77.0, device="cuda")
    listed = torch.from_numpy(rows.astype(np.int32)).cuda() if "list" in opt else None
    B.fg_residual_norm(xd, stride(xd), code(B, dtype), rd, stride(rd) if rd is not None else 0, code(B, sum_type), listed, None, len(rows), n, d, p, key, cuda(w), eps,
                       sum_out, stride(sum_out), yd, stride(yd), code(B, y_type), scale, got_rstd)
    torch.cuda.synchronize()
    u = 2.0 ** -24
    ds = 2 * u * size                                              # the scaled branch and the sum are rounded
    close(sum_out.cpu()[rows, :d], s, ds + HALF[sum_type] * s.abs() + TINY[sum_type], "sum")
    off = (s.abs() * ds).mean(1) * rstd.square()                   # rstd: what the addends' rounding does to the mean square, and its own
    close(got_rstd.cpu()[rows], rstd, rstd * (off + 4 * u), "rstd")
    wa = w.double().abs() if w is not None else 1.0
    ty = rstd[:, None] * wa * ds + y.abs() * (off[:, None] + 8 * u)
    rest = np.setdiff1d(np.arange(n), rows)
    if eight:
        q, sc = yd.view(torch.float8_e4m3fn).float().cpu()[rows, :d].double(), scale.cpu().double()[rows]
        top = y.abs().amax(1).clamp_min(2.0 ** -100)
        close(sc, top / 448, (ty.amax(1) + top * 2 * u) / 448, "scale")
        close(q * sc[:, None], y, 2.0 ** -4 * y.abs() + sc[:, None] * 2.0 ** -10 + 2 * ty, "8-bit values")      # half a step, of the smallest numbers at least
        assert bool((yd.cpu()[rest] == 0x55).all()) and bool((yd.cpu()[:, d:] == 0x55).all()) and bool((scale.cpu()[rest] == -77).all())
    else:
        close(yd.cpu()[rows, :d], y, ty + HALF[y_type] * y.abs() + TINY[y_type], "y")
        assert bool((yd.cpu()[rest] == -77).all()) and bool((yd.cpu()[:, d:] == -77).all())
    assert bool((got_rstd.cpu()[rest] == -77).all())
    if "inplace" not in opt:
        assert bool((sum_out.cpu()[rest] == -77).all()) and bool((sum_out.cpu()[:, d:] == -77).all())


@gpu
def test_residual_norm_of_rows_that_are_not_finite(B):
    """A NaN or an infinity stays in its own row; large values do not overflow on the way."""
    n, d = 8, 96
    x = torch.ones(n, d)
    x[1, 5], x[2, 7], x[3], x[4] = float("nan"), float("inf"), 3e38, -2e-38
    q, scale, rstd, y = torch.zeros(n, d, dtype=torch.uint8, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, d, device="cuda")
    B.fg_residual_norm(x.cuda(), 4 * d, B.FG_F32, None, 0, B.FG_F32, None, None, n, n, d, 0.0, 0, None, 1e-6, None, 0, q, d, B.FG_E4M3, scale, rstd)
    B.fg_residual_norm(x.cuda(), 4 * d, B.FG_F32, None, 0, B.FG_F32, None, None, n, n, d, 0.0, 0, None, 1e-6, None, 0, y, 4 * d, B.FG_F32, None, None)
    y, v = y.cpu(), q.view(torch.float8_e4m3fn).float().cpu() * scale.cpu()[:, None]
    assert bool(y[1].isnan().all()) and bool(y[2, 7].isnan()) and bool(v[1].isnan().all())
    for i, want in ((0, 1 / math.sqrt(1 + 1e-6)), (3, 1.0), (5, 1 / math.sqrt(1 + 1e-6))):
        assert float((y[i] - want).abs().max()) <= 2.0 ** -21 and float((v[i] - want).abs().max()) <= 2.0 ** -21
    assert float((y[4] + 2e-38 * 1000).abs().max()) <= 1e-41      # eps decides: a subnormal row times 1000


@gpu
@pytest.mark.parametrize("grad, sum_type, n, d, p, options", [
    ("f32", "f32", 1, 1, 0.0, "dw"), ("f32", "f32", 777, 88, 0.1, "ds dx dw w list"), ("f32", "bf16", 300, 256, 0.5, "ds dx dw w"), ("bf16", "bf16", 2000, 1024, 0.5, "ds dx dw w"),
    ("f16", "f32", 64, 100, 0.2, "dx dw pad"), ("bf16", "f32", 40, 2047, 0.0, "ds w pad"), ("f16", "f16", 9, 3000, 0.3, "ds dx dw w list"), ("f32", "f32", 5, 8200, 0.0, "dw w"),
    ("bf16", "bf16", 3, 16384, 0.1, "ds dx dw"), ("f32", "f32", 20000, 17, 0.5, "ds dx dw w list"), ("f16", "bf16", 50, 600, 0.0, "ds dw w inplace")])
def test_residual_norm_backward(B, grad, sum_type, n, d, p, options):
    r = np.random.default_rng(n + d)
    opt = options.split()
    pad, key = 5 if "pad" in opt else 0, 1234567
    dy, s = matrix(r, n, d, grad, pad), matrix(r, n, d, sum_type, pad)
    ds_in = matrix(r, n, d, grad, pad) if "ds" in opt else None
    w = torch.from_numpy(1 + 0.2 * r.standard_normal(d)).float() if "w" in opt else None
    rows = np.sort(r.choice(n, (3 * n + 3) // 4, replace=False)) if "list" in opt else np.arange(n)
    rstd = (1 / torch.sqrt(s[:, :d].double().square().mean(1) + 1e-6)).float()
    ds, dx, dw, size, dw_size = R.residual_norm_backward(dy[:, :d], s[:, :d], rstd, w, ds_in[:, :d] if ds_in is not None else None, rows, p, key)
    dyd, sd, di = dy.cuda(), s.cuda(), cuda(ds_in)
    out = di if "inplace" in opt else sentinel(n, d, grad, pad).cuda()
    gx = sentinel(n, d, grad, pad).cuda() if "dx" in opt else None
    gw = torch.full((d + 1,), -77.0, device="cuda") if "dw" in opt else None
    ws = torch.zeros(max(16, B.fg_residual_norm_backward_workspace_bytes(len(rows), d)), dtype=torch.uint8, device="cuda") if gw is not None else None
    B.fg_residual_norm_backward(dyd, stride(dyd), code(B, grad), sd, stride(sd), code(B, sum_type), rstd.cuda(), cuda(w), di, stride(di) if di is not None else 0,
                                torch.from_numpy(rows.astype(np.int32)).cuda() if "list" in opt else None, torch.tensor([len(rows)], device="cuda"), len(rows), n, d, p,
                                key, out, stride(out), gx, stride(gx) if gx is not None else 0, gw, ws, ws.numel() if ws is not None else 0)
    torch.cuda.synchronize()
    tol = 2.0 ** -21 * size      # six roundings of a relative 2^-24
    close(out.cpu()[rows, :d], ds, tol + HALF[grad] * ds.abs() + TINY[grad], "dsum")
    rest = np.setdiff1d(np.arange(n), rows)
    if gx is not None:
        factor = 65536 / (65536 - R.threshold(p))
        close(gx.cpu()[rows, :d], dx, factor * tol + HALF[grad] * dx.abs() * (1 + 2.0 ** -8) + TINY[grad], "dx")
        assert bool((gx.cpu()[rest] == -77).all()) and bool((gx.cpu()[:, d:] == -77).all())
    if gw is not None:
        close(gw.cpu()[:d], dw, (min(len(rows), 4096) + 8) * 2.0 ** -23 * dw_size, "dw")
        assert float(gw[d]) == -77
    if "inplace" not in opt:
        assert bool((out.cpu()[rest] == -77).all()) and bool((out.cpu()[:, d:] == -77).all())


def test_residual_norm_gradients_against_differences():
    """The formulas the backward call is held to, against central differences of the forward formula in 64 bits."""
    r = np.random.default_rng(3)
    n, d, p, key = 6, 20, 0.3, 77
    x, res, c, e = (torch.from_numpy(r.standard_normal((n, d))) for _ in range(4))
    w = torch.from_numpy(1 + 0.2 * r.standard_normal(d))
    rows, step = np.arange(n), 1e-5

    def loss(x, res, w):
        s, _, y, _ = R.residual_norm(x, res, rows, p, key, w, 1e-6)
        return float((c * y).sum() + (e * s).sum())

    s, rstd, _, _ = R.residual_norm(x, res, rows, p, key, w, 1e-6)
    ds, dx, dw, _, _ = R.residual_norm_backward(c, s, rstd, w, e, rows, p, key)
    for grad, at in ((dx, 0), (ds, 1), (dw, 2)):
        v = torch.from_numpy(r.standard_normal(grad.shape))
        args = [x, res, w]
        hi, lo = list(args), list(args)
        hi[at], lo[at] = args[at] + step * v, args[at] - step * v
        want = (loss(*hi) - loss(*lo)) / (2 * step)
        # truncation step^2 times a third derivative of order 100 here, rounding 1e-16 x 100 / step
        assert abs(float((grad * v).sum()) - want) <= 1e-6


@gpu
@pytest.mark.parametrize("d, dtype, skipped", [(8000, "f16", 4_300_000), (2056, "bf16", 8_400_000), (8200, "f32", 8_390_000)])
def test_lists_that_are_longer_than_a_launch_can_have_threads_for(B, d, dtype, skipped):
    """What the last of 2^32 threads and more would do: the list ends in the only positions that exist."""
    n, p, key = 40, 0.3, 77
    g = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn(n, d, device="cuda", generator=g).to(T[dtype])
    tail = torch.randperm(n, device="cuda", generator=g)[:33].int()
    rows = torch.cat([torch.full((skipped,), -1, dtype=torch.int32, device="cuda"), tail])
    got = {}
    for name, list_ in (("short", tail), ("long", rows)):
        out, y = torch.full_like(x, -77.0), torch.full_like(x, -77.0)
        rstd = torch.full((n,), -77.0, device="cuda")
        B.fg_dropout(x, stride(x), code(B, dtype), list_, None, len(list_), n, d, p, key, out, stride(out))
        B.fg_residual_norm(x, stride(x), code(B, dtype), None, 0, code(B, dtype), list_, None, len(list_), n, d, p, key, None, 1e-6, None, 0, y, stride(y),
                           code(B, dtype), None, rstd)
        torch.cuda.synchronize()
        got[name] = out, y, rstd
    for a, b in zip(got["short"], got["long"]):
        assert torch.equal(a, b) and bool((a[tail.long()] != -77).any())


# ---- fg_quantize_rows ----

@gpu
@pytest.mark.parametrize("dtype, n, d, pad", [("f32", 1, 1, 0), ("f32", 50, 100, 3), ("f16", 33, 1024, 0), ("bf16", 200, 80, 0), ("bf16", 7, 5001, 1), ("f32", 3, 16384, 0)])
def test_quantize_rows(B, dtype, n, d, pad):
    r = np.random.default_rng(n + d)
    x = (matrix(r, n, d, dtype, pad).double() * torch.from_numpy(np.exp(2 * r.standard_normal((n, 1))))).to(T[dtype])
    if n > 5:
        x[2, :d] = 0
        x[4, :d] = x[4, :d] * (2.0 ** -110 if dtype != "f16" else 2.0 ** -14)
    q, scale = R.quantise(x[:, :d])
    got, gs = torch.full((n, d + pad), 0x55, dtype=torch.uint8, device="cuda"), torch.zeros(n, device="cuda")
    xd = x.cuda()
    B.fg_quantize_rows(xd, stride(xd), code(B, dtype), n, d, got, d + pad, gs)
    torch.cuda.synchronize()
    assert torch.equal(gs.cpu(), scale) and torch.equal(got.view(torch.float8_e4m3fn).float().cpu()[:, :d], q)
    assert bool((got[:, d:] == 0x55).all())


# ---- together ----

def block(B, st, G, a, b, p, key, t):
    """Typed product with ReLU, then residual norm with dropout on the branch; gradients of both. `t`: device tensors by name."""
    n, k = len(t["x"]), t["n_rows"]
    B.fg_group_rows(t["types"], len(t["types"]), t["ids"], n, t["rows"], k, len(t["rows"]), G, t["order"], t["offsets"], t["ws"], t["ws"].numel(), st)
    B.fg_linear_grouped(t["x"], n, 4 * a, B.FG_F32, None, None, t["order"], t["offsets"], len(t["rows"]), G, a, b, t["W"], None, t["bias"], 1, t["h"], n, 4 * b, B.FG_F32, st)
    B.fg_residual_norm(t["h"], 4 * b, B.FG_F32, t["res"], 4 * b, B.FG_F32, t["rows"], k, len(t["rows"]), n, b, p, key, t["gain"], 1e-6, t["sum"], 4 * b, t["y"], 4 * b, B.FG_F32,
                       None, t["rstd"], st)
    B.fg_residual_norm_backward(t["dy"], 4 * b, B.FG_F32, t["sum"], 4 * b, B.FG_F32, t["rstd"], t["gain"], None, 0, t["rows"], k, len(t["rows"]), n, b, p, key, t["dres"], 4 * b,
                                t["dh"], 4 * b, t["dgain"], t["ws"], t["ws"].numel(), st)
    B.fg_linear_grouped_backward(t["x"], n, 4 * a, B.FG_F32, None, t["dh"], 4 * b, B.FG_F32, t["h"], 4 * b, n, t["order"], t["offsets"], len(t["rows"]), G, a, b, t["W"], t["dx"],
                                 4 * a, B.FG_F32, t["dW"], t["db"], t["ws"], t["ws"].numel(), st)


def block_tensors(B, seed, n, G, a, b):
    r = np.random.default_rng(seed)
    f = lambda *s: torch.from_numpy(r.standard_normal(s)).float().cuda()
    rows = torch.from_numpy(np.sort(r.choice(n, n - n // 5, replace=False)).astype(np.int32)).cuda()
    t = dict(types=torch.from_numpy(r.integers(0, G, 3 * n).astype(np.int32)).cuda(), ids=torch.from_numpy(r.integers(0, 3 * n, n).astype(np.int32)).cuda(), rows=rows,
             n_rows=torch.tensor([len(rows)], device="cuda"), x=f(n, a), W=f(G, a, b) / math.sqrt(a), bias=f(G, b), res=f(n, b), gain=1 + 0.1 * f(b), dy=f(n, b))
    t |= {k: torch.zeros(n, b, device="cuda") for k in ("h", "sum", "y", "dres", "dh")}
    t |= dict(order=torch.zeros(n, dtype=torch.int32, device="cuda"), offsets=torch.zeros(G + 1, dtype=torch.int64, device="cuda"), rstd=torch.zeros(n, device="cuda"),
              dgain=torch.zeros(b, device="cuda"), dx=torch.zeros(n, a, device="cuda"), dW=torch.zeros(G, a, b, device="cuda"), db=torch.zeros(G, b, device="cuda"))
    size = max(B.fg_group_rows_workspace_bytes(n, G), B.fg_residual_norm_backward_workspace_bytes(n, b), B.fg_linear_grouped_backward_workspace_bytes(B.FG_F32, n, G, a, b))
    return t | dict(ws=torch.zeros(size, dtype=torch.uint8, device="cuda"))


OUTPUTS = ("order", "offsets", "h", "sum", "y", "rstd", "dres", "dh", "dgain", "dx", "dW", "db")


@gpu
@pytest.mark.parametrize("bound", [0, 1, 300, 9000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nothing_is_listed(B, dtype, bound):
    """A count of zero on the device under any bound: sums are zeros, nothing else is touched."""
    n, G, d = max(bound, 4), 3, 64
    x, zero = torch.randn(n, d, device="cuda").to(T[dtype]), torch.zeros(1, dtype=torch.int64, device="cuda")
    c = code(B, dtype)
    order = torch.full((max(bound, 1),), -77, dtype=torch.int32, device="cuda")
    offsets = torch.full((G + 1,), -77, dtype=torch.int64, device="cuda")
    ws = torch.full((1 << 26,), 255, dtype=torch.uint8, device="cuda")      # more than any of the calls needs
    B.fg_group_rows(torch.zeros(n, dtype=torch.int32, device="cuda"), n, None, n, None, zero, bound, G, order, offsets, ws, ws.numel())
    torch.cuda.synchronize()
    assert bool((order == -77).all()) and bool((offsets == 0).all())
    W, h, dx = torch.randn(G, d, d, device="cuda").to(T[dtype]), torch.full_like(x, -77.0), torch.full_like(x, -77.0)
    B.fg_linear_grouped(x, n, stride(x), c, None, None, order, offsets, bound, G, d, d, W, None, None, 1, h, n, stride(h), c)
    dw, db = torch.full((G, d, d), -77.0, device="cuda"), torch.full((G, d), -77.0, device="cuda")
    B.fg_linear_grouped_backward(x, n, stride(x), c, None, x, stride(x), c, x, stride(x), n, order, offsets, bound, G, d, d, W, dx, stride(dx), c, dw, db, ws, ws.numel())
    y, rstd, gw = torch.full_like(x, -77.0), torch.full((n,), -77.0, device="cuda"), torch.full((d,), -77.0, device="cuda")
    B.fg_dropout(x, stride(x), c, None, zero, bound, n, d, 0.5, 1, y, stride(y))
    B.fg_residual_norm(x, stride(x), c, None, 0, c, None, zero, bound, n, d, 0.5, 1, None, 1e-6, None, 0, y, stride(y), c, None, rstd)
    B.fg_residual_norm_backward(x, stride(x), c, x, stride(x), c, rstd, None, None, 0, None, zero, bound, n, d, 0.5, 1, y, stride(y), None, 0, gw, ws, ws.numel())
    torch.cuda.synchronize()
    assert all(bool((t == -77).all()) for t in (h, dx, y, rstd))
    assert all(not bool(t.any()) for t in (dw, db, gw))


@gpu
def test_a_typed_layer_and_its_gradients(B):
    """The calls one behind the other, as a training step makes them, against automatic differentiation in 64 bits."""
    n, G, a, b, p, key = 700, 4, 52, 88, 0.3, 4242
    t = block_tensors(B, 1, n, G, a, b)
    block(B, None, G, a, b, p, key, t)
    torch.cuda.synchronize()
    c = {k: v.cpu() for k, v in t.items()}
    order, offsets = R.group(c["types"].tolist(), c["ids"].tolist(), c["rows"].tolist(), G)
    assert c["order"][:len(order)].tolist() == order and c["offsets"].tolist() == offsets
    leaf = {k: c[k].double().requires_grad_() for k in ("x", "W", "bias", "res", "gain")}
    h = torch.cat([leaf["x"][order[offsets[g]:offsets[g + 1]]] @ leaf["W"][g] + leaf["bias"][g] for g in range(G)]).clamp_min(0)
    pos = torch.tensor(order)
    keep = R.keep(key, order, b, p)
    s = torch.where(keep, h * float(np.float32(65536 / (65536 - R.threshold(p)))), torch.zeros((), dtype=torch.float64)) + leaf["res"][pos]
    y = s / torch.sqrt(s.square().mean(1, keepdim=True) + float(np.float32(1e-6))) * leaf["gain"]
    (y * c["dy"].double()[pos]).sum().backward()
    for name, want in (("h", h), ("sum", s), ("y", y)):
        assert float((c[name][pos].double() - want.detach()).norm() / want.detach().norm()) <= 2e-6, name      # 2^-24 sqrt(52) and a few roundings
    near = lambda got, want, name: float((got.double() - want).norm() / want.norm()) <= 4e-6 or pytest.fail(name)
    near(c["dx"][pos], leaf["x"].grad[pos], "dx"), near(c["dW"], leaf["W"].grad, "dW"), near(c["db"], leaf["bias"].grad, "db")
    near(c["dres"][pos], leaf["res"].grad[pos], "dres"), near(c["dgain"], leaf["gain"].grad, "dgain")


@gpu
def test_a_typed_layer_captured_and_on_other_streams(B):
    """The same calls in a graph that is replayed with new inputs between eager ones, and on two streams at once with workspaces of their own."""
    n, G, a, b, p, key = 900, 5, 64, 96, 0.5, 7
    t, other = block_tensors(B, 2, n, G, a, b), block_tensors(B, 3, n, G, a, b)
    names = ("types", "ids", "rows", "x", "W", "bias", "res", "gain", "dy")
    def eager(src):
        e = block_tensors(B, 9, n, G, a, b)
        for k in names:
            e[k].copy_(src[k])
        block(B, torch.cuda.current_stream().cuda_stream, G, a, b, p, key, e)
        torch.cuda.synchronize()
        return {k: e[k].clone() for k in OUTPUTS}
    want = [eager(t), eager(other)]
    inputs = [{k: s[k].clone() for k in names} for s in (t, other)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        block(B, torch.cuda.current_stream().cuda_stream, G, a, b, p, key, t)
    for i in (0, 1, 0, 0, 1):
        for k in names:
            t[k].copy_(inputs[i][k])
        for k in OUTPUTS:
            t[k].zero_()
        g.replay()
        torch.cuda.synchronize()
        for k in OUTPUTS:
            assert torch.equal(t[k], want[i][k]), (i, k)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for k in names:
        t[k].copy_(inputs[0][k]), other[k].copy_(inputs[1][k])
    for k in OUTPUTS:
        t[k].zero_(), other[k].zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for s, e in zip(streams, (t, other)):
            block(B, s.cuda_stream, G, a, b, p, key, e)
    torch.cuda.synchronize()
    for i, e in enumerate((t, other)):
        for k in OUTPUTS:
            assert torch.equal(e[k], want[i][k]), (i, k)


@gpu
def test_a_layer_served_in_8_bits(B):
    """Residual norm with 8-bit rows, then the typed product of those rows: the product is that of the values the rows stand for."""
    n, G, a, b = 500, 6, 256, 128
    r = np.random.default_rng(8)
    x, res = matrix(r, n, a, "bf16"), matrix(r, n, a, "bf16")
    W, bias = torch.from_numpy(r.standard_normal((G, a, b)) / 16).float(), torch.from_numpy(r.standard_normal((G, b))).float()
    types = torch.from_numpy(r.integers(0, G, n).astype(np.int32)).cuda()
    q, qs = torch.zeros(n, a, dtype=torch.uint8, device="cuda"), torch.zeros(n, device="cuda")
    wq, ws = torch.zeros(G * b, a, dtype=torch.uint8, device="cuda"), torch.zeros(G * b, device="cuda")
    B.fg_quantize_rows(W.transpose(1, 2).contiguous().cuda(), 4 * a, B.FG_F32, G * b, a, wq, a, ws)
    order, offsets = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(G + 1, dtype=torch.int64, device="cuda")
    space = torch.zeros(B.fg_group_rows_workspace_bytes(n, G), dtype=torch.uint8, device="cuda")
    B.fg_group_rows(types, n, None, n, None, None, n, G, order, offsets, space, space.numel())
    B.fg_residual_norm(x.cuda(), 2 * a, B.FG_BF16, res.cuda(), 2 * a, B.FG_BF16, None, None, n, n, a, 0.0, 0, None, 1e-6, None, 0, q, a, B.FG_E4M3, qs, None)
    h = torch.zeros(n, b, device="cuda")
    B.fg_linear_grouped(q, n, a, B.FG_E4M3, qs, None, order, offsets, n, G, a, b, wq, ws, bias.cuda(), 1, h, n, 4 * b, B.FG_F32)
    torch.cuda.synchronize()
    xv = q.view(torch.float8_e4m3fn).float().cpu().double() * qs.cpu().double()[:, None]
    wv = (wq.view(torch.float8_e4m3fn).float().cpu().double() * ws.cpu().double()[:, None]).reshape(G, b, a).transpose(1, 2)
    o = order.cpu().tolist()
    want, size = R.grouped_linear(xv, wv, bias, o, offsets.cpu().tolist(), None, True)
    close(h.cpu()[o], want, (a + 8) * 2.0 ** -23 * size, "product of the 8-bit rows")
    # against the layer without 8 bits: a factor of (1 + 2^-4)^2 - 1 of the products' magnitudes at most
    _, _, y, _ = R.residual_norm(x, res, np.arange(n), 0.0, 0, None, 1e-6)
    full, fsize = R.grouped_linear(y, W, bias, o, offsets.cpu().tolist(), None, True)
    close(h.cpu()[o], full, 0.14 * fsize, "against full precision")
