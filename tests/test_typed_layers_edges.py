"""The calls of a typed layer where one kind of input decides: 8-bit rows whose products differ by many orders of magnitude, entries that are
skipped in the gradients, lists longer than a launch, limits. Tolerances as in tests/test_typed_layers.py: a sum of K products in fp32 is granted
K steps of 2^-23 of the sum of the products' magnitudes, a result half a step of its type."""
import glob
import os
import re

import numpy as np
import pytest
import torch

from tests import typed_reference as R
from tests.test_typed_layers import HALF, T, TINY, B, close, code, cuda, gpu, layout, matrix, refused, stride  # noqa: F401 (B: the fixture)


def e4m3(v):
    q = v.to(torch.float8_e4m3fn)
    assert torch.equal(q.to(v.dtype), v), "values that 8 bits hold"
    return q


# ---- limits ----

def test_widths_beyond_the_limit_are_refused(B):
    """As the header names it; the workspace query knows the same limit."""
    P, stride_ = 4096, 1 << 20
    most = B.FG_MAX_GROUPED_DIM
    for dtype in (B.FG_F32, B.FG_F16, B.FG_BF16, B.FG_E4M3):
        scale = P if dtype == B.FG_E4M3 else None
        for a, b in ((most + 16, 64), (64, most + 16)):
            assert refused(B, B.fg_linear_grouped, P, 10, stride_, dtype, scale, None, P, P, 10, 4, a, b, P, scale, None, 0, P, 10, stride_, B.FG_F32) == B.FG_ERR_SHAPE
            if dtype != B.FG_E4M3:
                assert refused(B, B.fg_linear_grouped_backward, P, 10, stride_, dtype, None, P, stride_, dtype, None, 0, 10, P, P, 10, 4, a, b, P, P, stride_, dtype, P, P, P,
                               1 << 62) == B.FG_ERR_SHAPE
                assert B.fg_linear_grouped_backward_workspace_bytes(dtype, 10, 4, a, b) == 0
                assert B.fg_linear_grouped_backward_workspace_bytes(dtype, 10, 4, min(a, most), min(b, most)) > 0


# ---- statements the compiler does not see into ----

def test_statements_that_write_m0_put_it_back():
    """M0 cannot be named as overwritten, so that a statement has to leave it as it was."""
    found = 0
    for path in sorted(glob.glob(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2301_07482_amd", "csrc", "*"))):
        for text in re.findall(r'asm\s*(?:volatile)?\s*\(\s*"((?:[^"\\]|\\.)*)"', open(path).read()):
            lines = [line.strip() for line in re.split(r"\\n|\\t|;", text) if line.strip()]
            if not any(re.match(r"s_mov_b32 m0,", line) for line in lines):
                assert "m0" not in text, (path, text)
                continue
            found += 1
            kept = re.match(r"s_mov_b32 (%\d), m0$", lines[0])
            assert kept and lines[-1] == f"s_mov_b32 m0, {kept.group(1)}", (path, text)
    assert found


# ---- 8-bit rows ----

@gpu
@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("signs", ["alternating", "equal", "random"])
@pytest.mark.parametrize("n, n_groups, d_in, d_out", [(150, 3, 64, 40), (300, 2, 400, 136), (34_000, 3, 80, 264), (68_000, 2, 64, 512)])
def test_8_bit_rows_with_one_large_value_in_eight(B, n, n_groups, d_in, d_out, signs, out):
    """A feature in eight whose products are 2^13 times the others' and more, as outlying features of activations are. Where the large products
    cancel, what is left is made of the small ones."""
    g = torch.Generator(device="cuda").manual_seed(n + d_in)
    kw = dict(device="cuda", generator=g)
    pick = lambda *s: 2.0 ** torch.randint(-1, 3, s, **kw).float() * (1 - 2 * torch.randint(0, 2, s, **kw)).float()
    x, W = pick(n, d_in), pick(n_groups, d_out, d_in)
    eighth = torch.arange(0, d_in, 8, device="cuda") + 3
    sign = {"alternating": 1 - 2 * (torch.arange(len(eighth), device="cuda") % 2), "equal": torch.ones(len(eighth), device="cuda"),
            "random": 1 - 2 * torch.randint(0, 2, (n, len(eighth)), **kw)}[signs].float()
    x[:, eighth], W[:, :, eighth] = 256.0 * sign.expand(n, -1), 256.0
    xs, ws = torch.rand(n, **kw) * 2.0 ** -7, torch.rand(n_groups * d_out, **kw) * 2.0 ** -7
    types = torch.randint(0, n_groups, (n,), **kw).sort()
    offsets = torch.searchsorted(types.values, torch.arange(n_groups + 1, device="cuda"))
    order = torch.randperm(n, **kw).int()
    h = torch.full((n, d_out), -77.0, dtype=T[out], device="cuda")
    B.fg_linear_grouped(e4m3(x), n, d_in, B.FG_E4M3, xs, None, order, offsets, n, n_groups, d_in, d_out, e4m3(W), ws, None, 0, h, n, stride(h), code(B, out))
    torch.cuda.synchronize()
    for k in range(n_groups):
        pos = order[int(offsets[k]):int(offsets[k + 1])].long()
        a, w = x[pos].double() * xs[pos].double()[:, None], (W[k].double() * ws.view(n_groups, -1)[k].double()[:, None]).T.contiguous()
        want, size = torch.mm(a, w), torch.mm(a.abs(), w.abs())
        close(h[pos], want, (d_in + 8) * 2.0 ** -23 * size + HALF[out] * want.abs() + TINY[out], f"{signs} {out}")


@gpu
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("x_scale, w_scale", [(1.37 * 2.0 ** 100, 1.61 * 2.0 ** 40), (1.37 * 2.0 ** 40, 1.61 * 2.0 ** 100), (1.37 * 2.0 ** -100, 1.61 * 2.0 ** -45),
                                              (1.37 * 2.0 ** -45, 1.61 * 2.0 ** -100), (1.37 * 2.0 ** 110, 1.61 * 2.0 ** -30), (1.37 * 2.0 ** -30, 1.61 * 2.0 ** 110)])
def test_8_bit_rows_with_scales_far_from_one(B, x_scale, w_scale, out):
    """The product of the two scales may leave fp32 where the result does not: sums of zeros, and sums that are far from one the other way."""
    n, a, b = 70, 64, 24
    g = torch.Generator().manual_seed(7)
    x = torch.randint(1, 8, (n, a), generator=g).float() * 64
    x[:35] = 0
    w = torch.randint(1, 8, (b, a), generator=g).float() * 64
    if x_scale * w_scale > 2.0 ** 127:
        x[35:] = 0
    bias = torch.randn(1, b, generator=g)
    if x_scale * w_scale < 1:
        bias.zero_()
    xs, ws = torch.full((n,), x_scale), torch.full((b,), w_scale)
    h = torch.full((n, b), -77.0, dtype=T[out], device="cuda")
    B.fg_linear_grouped(e4m3(x).cuda(), n, a, B.FG_E4M3, xs.cuda(), None, None, torch.tensor([0, n], device="cuda"), n, 1, a, b, e4m3(w).cuda(), ws.cuda(), bias.cuda(), 0, h, n,
                        stride(h), code(B, out))
    torch.cuda.synchronize()
    want = (x.double() @ w.double().T) * float(xs[0]) * float(ws[0]) + bias.double()      # (whole numbers below 2^24: the sum is exact)
    # four roundings: the two scales' products, the bias, the type
    close(h.cpu(), want, 2.0 ** -22 * (want.abs() + bias.double().abs()) + HALF[out] * want.abs(), f"{x_scale:g} {w_scale:g} {out}")


# ---- dropout ----

@gpu
def test_dropout_in_place_of_a_list_longer_than_a_launch(B):
    """Every row is dropped once: the row at the place where a launch ends and the next one begins, too."""
    n, d, p, key, dtype = 40, 8000, 0.3, 77, "f16"
    at = ((1 << 24) - 1) * 256 // (d // 8)      # rows of a launch: 2^32 threads less 256, 1000 to a row
    x = torch.randn(n, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(d)).to(T[dtype])
    listed = torch.tensor([5, 11, 7], dtype=torch.int32, device="cuda")
    rows = torch.full((at + 40,), -1, dtype=torch.int32, device="cuda")
    rows[at - 1], rows[at], rows[at + 1] = 5, 11, 7
    got = {}
    for name, list_ in (("short", listed), ("long", rows)):
        got[name] = x.clone()
        B.fg_dropout(got[name], stride(x), code(B, dtype), list_, None, len(list_), n, d, p, key, got[name], stride(x))
    torch.cuda.synchronize()
    assert torch.equal(got["short"], got["long"]) and not torch.equal(got["short"], x)


# ---- gradients ----

def test_a_call_is_refused_before_anything_is_launched(B):
    """Weight gradients that one launch cannot sum; without a GPU a launch would end the call with another error."""
    P = 4096
    for dtype in (B.FG_F32, B.FG_BF16):
        for n in (10, 0):
            assert refused(B, B.fg_linear_grouped_backward, P, n, 1 << 20, dtype, None, P, 1 << 20, dtype, P, 1 << 20, n, P, P, 1000, 1024, 65536, 65536, P, P, 1 << 20, dtype, P, P, P,
                           1 << 62) == B.FG_ERR_SHAPE


def test_refusals_of_the_output_s_type(B):
    P = 4096
    bw = lambda **k: B.fg_linear_grouped_backward(**{**dict(x=P, x_rows=10, x_stride=256, dtype=B.FG_BF16, src_ids=None, dh=P, dh_stride=256, dh_dtype=B.FG_BF16,
                                                            h=P, h_stride=128, n=10, order=P, offsets=P, max_rows=10, n_groups=4, d_in=64, d_out=64, W=P,
                                                            dx=P, dx_stride=256, dx_dtype=B.FG_F32, dw=P, db=P, ws=P, ws_bytes=1 << 40, h_dtype=B.FG_BF16), **k})
    for bad, want in ((dict(h_dtype=B.FG_E4M3), 3), (dict(h_dtype=7), 3), (dict(h_dtype=B.FG_F32), 2), (dict(dtype=B.FG_F32, dh_dtype=B.FG_F32), 3),
                      (dict(h_dtype=B.FG_F16, h_stride=112), 2)):
        assert refused(B, bw, **bad) == want, bad


@gpu
@pytest.mark.parametrize("dtype, out, dh_type", [("bf16", "f32", "bf16"), ("bf16", "f32", "f32"), ("bf16", "f16", "bf16"), ("bf16", "f16", "f32"), ("f16", "f32", "f16"),
                                                 ("f16", "f32", "f32"), ("f16", "bf16", "f16"), ("f16", "bf16", "f32"), ("bf16", "bf16", "f32"), ("f32", "f32", "f32")])
@pytest.mark.parametrize("named", [True, False])
def test_gradients_of_a_relu_layer_by_the_type_of_its_output(B, dtype, out, dh_type, named):
    """The mask is h > 0 of the rows as the forward call wrote them, in each type that it writes; what has no sign to speak of among them too."""
    n, G, a, b = 400, 3, 64, 72
    r = np.random.default_rng(17)
    order, offsets = layout(r, n, G, 0.9)
    x, W, dh = matrix(r, n, a, dtype), torch.from_numpy(r.standard_normal((G, a, b)) / 8).to(T[dtype]), matrix(r, n, b, dh_type)
    bias = torch.from_numpy(r.standard_normal((G, b))).float().cuda()
    od, fd, xd, Wd = torch.from_numpy(order).cuda(), torch.from_numpy(offsets).cuda(), x.cuda(), W.cuda()
    h = torch.full((n, b + 8), -77.0, dtype=T[out], device="cuda")
    B.fg_linear_grouped(xd, n, stride(xd), code(B, dtype), None, None, od, fd, len(order), G, a, b, Wd, None, bias, 1, h, n, stride(h), code(B, out))
    low = torch.finfo(T[out]).smallest_normal
    h[:5, :6] = torch.tensor([0.0, -0.0, float("nan"), low, -low, low / 8], device="cuda").to(T[out])
    h[5:9, :2] = torch.tensor([float("inf"), -float("inf")], device="cuda").to(T[out])
    rounds = T[dtype] if dtype != "f32" and dh_type == "f32" else None
    (dx, dxs), (dW, dWs), (db, dbs) = R.grouped_linear_backward(x, W, dh, h.cpu()[:, :b], order.tolist(), offsets.tolist(), None, rounds)
    gx, gw, gb = torch.full((n, a), -77.0, device="cuda"), torch.full((G, a, b), -77.0, device="cuda"), torch.full((G, b), -77.0, device="cuda")
    ws = torch.zeros(B.fg_linear_grouped_backward_workspace_bytes(code(B, dtype), len(order), G, a, b), dtype=torch.uint8, device="cuda")
    dhd = dh.cuda()
    B.fg_linear_grouped_backward(xd, n, stride(xd), code(B, dtype), None, dhd, stride(dhd), code(B, dh_type), h, stride(h), n, od, fd, len(order), G, a, b, Wd, gx, 4 * a,
                                 B.FG_F32, gw, gb, ws, ws.numel(), **(dict(h_dtype=code(B, out)) if named else {}))
    torch.cuda.synchronize()
    pos = order.astype(np.int64)
    close(gx.cpu()[pos], dx, (b + 8) * 2.0 ** -23 * dxs + HALF["f32"] * dx.abs(), "dx")
    close(gw.cpu(), dW, (len(order) + 16) * 2.0 ** -23 * dWs, "dW")
    close(gb.cpu(), db, (len(order) + 16) * 2.0 ** -23 * dbs, "db")


@gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16", "e4m3"])
@pytest.mark.parametrize("a, b", [(65536, 24), (32, 65536)])
def test_the_widest_rows(B, dtype, a, b):
    n, G = 70, 2
    g = torch.Generator(device="cuda").manual_seed(a)
    kw = dict(device="cuda", generator=g)
    offsets, order = torch.tensor([0, 30, n - 5], device="cuda"), torch.randperm(n, **kw).int()
    x, W = torch.randn(n, a, **kw), torch.randn(G, a, b, **kw) / 8
    out = "f32"
    xs = ws = None
    if dtype == "e4m3":
        (xq, xs), (wq, ws) = R.quantise(x), R.quantise(W.transpose(1, 2).contiguous().reshape(G * b, a))
        x64, W64 = xq.double() * xs.double()[:, None], (wq.double() * ws.double()[:, None]).reshape(G, b, a).transpose(1, 2).contiguous()
        x, W = e4m3(xq), e4m3(wq)
    else:
        x, W = x.to(T[dtype]), W.to(T[dtype])
        x64, W64 = x.double(), W.double()
    h = torch.full((n, b), -77.0, device="cuda")
    B.fg_linear_grouped(x, n, stride(x), code(B, dtype), xs, None, order, offsets, n, G, a, b, W, ws, None, 0, h, n, 4 * b, B.FG_F32)
    if dtype != "e4m3":
        dh = torch.randn(n, b, **kw).to(T[dtype])
        dx, dw, db = torch.full((n, a), -77.0, device="cuda"), torch.full((G, a, b), -77.0, device="cuda"), torch.full((G, b), -77.0, device="cuda")
        space = torch.zeros(B.fg_linear_grouped_backward_workspace_bytes(code(B, dtype), n, G, a, b), dtype=torch.uint8, device="cuda")
        B.fg_linear_grouped_backward(x, n, stride(x), code(B, dtype), None, dh, stride(dh), code(B, dtype), h, 4 * b, n, order, offsets, n, G, a, b, W, dx, 4 * a, B.FG_F32, dw, db,
                                     space, space.numel())
    torch.cuda.synchronize()
    for k in range(G):
        pos = order[int(offsets[k]):int(offsets[k + 1])].long()
        want, size = torch.mm(x64[pos], W64[k]), torch.mm(x64[pos].abs(), W64[k].abs())
        close(h[pos], want, (a + 8) * 2.0 ** -23 * size + HALF[out] * want.abs(), "h")
        if dtype != "e4m3":
            z, wt, xt = torch.where(h[pos] > 0, dh[pos].double(), torch.zeros((), dtype=torch.float64, device="cuda")), W64[k].T.contiguous(), x64[pos].T.contiguous()
            want = torch.mm(z, wt)
            close(dx[pos], want, (b + 8) * 2.0 ** -23 * torch.mm(z.abs(), wt.abs()) + HALF[out] * want.abs(), "dx")
            close(dw[k], torch.mm(xt, z), (len(pos) + 16) * 2.0 ** -23 * torch.mm(xt.abs(), z.abs()), "dW")
            close(db[k], z.sum(0), (len(pos) + 16) * 2.0 ** -23 * z.abs().sum(0), "db")
    rest = order[int(offsets[G]):].long()
    assert bool((h[rest] == -77).all()) and (dtype == "e4m3" or bool((dx[rest] == -77).all()))


def guarded(shape, dtype, fill=-77.0, guard=64):
    """A tensor with sentinels around it (16-byte aligned): (the whole, the part that calls get)."""
    count = int(np.prod(shape))
    whole = torch.full((guard + count + guard,), fill, dtype=dtype, device="cuda")
    return whole, whole[guard:guard + count].view(shape)


def untouched(whole, fill=-77.0, guard=64):
    return bool((whole[:guard] == fill).all()) and bool((whole[-guard:] == fill).all())


@gpu
@pytest.mark.parametrize("dtype, n, a, b", [("f32", 150, 64, 64), ("bf16", 150, 64, 64), ("f16", 150, 72, 40), ("f32", 9_000, 36, 132), ("bf16", 9_000, 264, 136), ("bf16", 40_000, 520, 520)])
@pytest.mark.parametrize("masked", [True, False])
@pytest.mark.parametrize("with_src", [True, False])
def test_gradients_skip_what_the_forward_call_skips(B, dtype, n, a, b, masked, with_src):
    """Bad positions, bad rows, entries beyond the bound: no part in dx, dW or db, though the rows they would take are NaN."""
    r = np.random.default_rng(n + a + masked)
    G = 3
    order, offsets = layout(r, n, G, 0.9)
    x_rows = 2 * n if with_src else n - 4
    src = r.integers(0, x_rows, n).astype(np.int32) if with_src else None
    entries = order.copy()
    skipped = set(r.choice(len(order), 12, replace=False).tolist())
    for i, k in enumerate(sorted(skipped)):
        if with_src and i % 2:
            src[order[k]] = (-1, x_rows, -2 ** 31, 2 ** 31 - 1)[i // 2 % 4]
        else:
            entries[k] = (-1, n, -2 ** 31, 2 ** 31 - 1)[i // 2 % 4]
    if not with_src:
        skipped |= {k for k in range(len(order)) if order[k] >= x_rows}
    bound = len(order) - 30
    taken = [k for k in range(bound) if k not in skipped]
    members = [[int(order[k]) for k in taken if offsets[g] <= k < offsets[g + 1]] for g in range(G)]
    good, at = [p for m in members for p in m], np.cumsum([0] + [len(m) for m in members]).tolist()
    x, dh, h = matrix(r, max(x_rows, n), a, dtype), matrix(r, n, b, dtype), matrix(r, n, b, dtype)
    W = torch.from_numpy(r.standard_normal((G, a, b)) / 8).to(T[dtype])
    (dx, dxs), (dW, dWs), (db, dbs) = R.grouped_linear_backward(x, W, dh, h if masked else None, good, at, src.tolist() if with_src else None)
    used = np.array([src[p] if with_src else p for p in good])
    x[np.setdiff1d(np.arange(len(x)), used)] = float("nan")
    rest = np.setdiff1d(np.arange(n), good)
    dh[rest], h[rest] = float("nan"), float("nan")
    xd, dhd, hd, Wd = x.cuda(), dh.cuda(), h.cuda(), W.cuda()
    (gx_all, gx), (gw_all, gw), (gb_all, gb) = guarded((n, a), torch.float32), guarded((G, a, b), torch.float32), guarded((G, b), torch.float32)
    size = B.fg_linear_grouped_backward_workspace_bytes(code(B, dtype), bound, G, a, b)
    ws_all, ws = guarded((size,), torch.uint8, 0xAB, 4096)
    B.fg_linear_grouped_backward(xd, x_rows, stride(xd), code(B, dtype), cuda(torch.from_numpy(src)) if with_src else None, dhd, stride(dhd), code(B, dtype), hd if masked else None,
                                 stride(hd) if masked else 0, n, torch.from_numpy(entries).cuda(), torch.from_numpy(offsets).cuda(), bound, G, a, b, Wd, gx, 4 * a, B.FG_F32, gw, gb,
                                 ws, size)
    torch.cuda.synchronize()
    close(gx.cpu()[good], dx, (b + 8) * 2.0 ** -23 * dxs + HALF["f32"] * dx.abs(), "dx")
    rows = (np.diff(at).max() + 16) * 2.0 ** -23
    close(gw.cpu(), dW, rows * dWs + 2.0 ** -24 * dW.abs(), "dW")
    close(gb.cpu(), db, rows * dbs + 2.0 ** -24 * db.abs(), "db")
    assert bool((gx.cpu()[rest] == -77).all())
    assert all(untouched(w) for w in (gx_all, gw_all, gb_all)) and untouched(ws_all, 0xAB, 4096)


@gpu
@pytest.mark.parametrize("dtype, n, a, b", [("f32", 300, 64, 64), ("bf16", 300, 64, 64), ("f32", 9_000, 132, 260), ("f16", 20_000, 264, 136)])
@pytest.mark.parametrize("masked", [True, False])
@pytest.mark.parametrize("shape", ["falling", "overlapping", "beyond", "negative"])
def test_offsets_that_do_not_ascend_stay_in_bounds(B, dtype, n, a, b, masked, shape):
    """Not what fg_group_rows leaves: no memory but the call's own is touched. A group whose end lies before its begin has no rows, and as long as no entry has two
    groups, the other groups' weight gradients are those of their entries."""
    r = np.random.default_rng(n + a)
    at = {"falling": [0, n, n // 2, n // 3, 0], "overlapping": [0, n - 7, 30, n, n // 2, n], "beyond": [0, n // 2, n + 1000, 2 ** 40, n + 5], "negative": [-5, -2 ** 40, n // 3, n, n]}[shape]
    G = len(at) - 1
    order = r.permutation(n).astype(np.int32)
    x, dh, h = matrix(r, n, a, dtype), matrix(r, n, b, dtype), matrix(r, n, b, dtype)
    W = torch.from_numpy(r.standard_normal((G, a, b)) / 8).to(T[dtype])
    xd, dhd, hd, Wd, od, fd = x.cuda(), dh.cuda(), h.cuda(), W.cuda(), torch.from_numpy(order).cuda(), torch.tensor(at, dtype=torch.int64, device="cuda")
    (h_all, out), (gx_all, gx), (gw_all, gw), (gb_all, gb) = (guarded(s, torch.float32) for s in ((n, b), (n, a), (G, a, b), (G, b)))
    size = B.fg_linear_grouped_backward_workspace_bytes(code(B, dtype), n, G, a, b)
    ws_all, ws = guarded((size,), torch.uint8, 0xAB, 4096)
    B.fg_linear_grouped(xd, n, stride(xd), code(B, dtype), None, None, od, fd, n, G, a, b, Wd, None, None, 0, out, n, 4 * b, B.FG_F32)
    B.fg_linear_grouped_backward(xd, n, stride(xd), code(B, dtype), None, dhd, stride(dhd), code(B, dtype), hd if masked else None, stride(hd) if masked else 0, n, od, fd, n, G, a,
                                 b, Wd, gx, 4 * a, B.FG_F32, gw, gb, ws, size)
    torch.cuda.synchronize()
    assert all(untouched(w) for w in (h_all, gx_all, gw_all, gb_all)) and untouched(ws_all, 0xAB, 4096)
    if shape == "overlapping":
        return
    inside = [min(max(o, 0), n) for o in at]
    for g in range(G):
        pos = order[inside[g]:max(inside[g], inside[g + 1])].astype(np.int64)
        z = dh[pos].double()
        if masked:
            z = torch.where(h[pos] > 0, z, torch.zeros((), dtype=torch.float64))
        xs = x[pos].double().T
        close(gw[g].cpu(), xs @ z, (len(pos) + 16) * 2.0 ** -23 * (xs.abs() @ z.abs()), f"dW of group {g}")


# ---- memory ----

@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_lie_further_apart_than_32_bits_count(B, dtype):
    """Row strides of 64 MB: the last rows' offsets are beyond 2^32. Results as with packed rows, bit for bit."""
    n, G, a, b, p, key = 70, 2, 64, 64, 0.3, 9
    r = np.random.default_rng(5)
    size, row = T[dtype].itemsize, (1 << 26) + 16
    c = code(B, dtype)
    order, offsets = layout(r, n, G, 0.9)
    od, fd = torch.from_numpy(order).cuda(), torch.from_numpy(offsets).cuda()
    src = torch.from_numpy(r.permutation(n).astype(np.int32)).cuda()
    W, values = torch.from_numpy(r.standard_normal((G, a, b)) / 8).to(T[dtype]).cuda(), {k: matrix(r, n, a, dtype).cuda() for k in ("x", "dh", "h", "res")}
    ws = torch.zeros(max(B.fg_linear_grouped_backward_workspace_bytes(c, n, G, a, b), B.fg_residual_norm_backward_workspace_bytes(n, a)), dtype=torch.uint8, device="cuda")

    def far(v):
        t = torch.empty(n * row // size, dtype=v.dtype, device="cuda").as_strided(v.shape, (row // size, 1))
        return t.copy_(v)

    results = []
    for place in (lambda v: v.clone(), far):
        t = {k: place(v) for k, v in values.items()}
        o = {k: place(torch.full_like(values["x"], -77.0)) for k in ("out", "dx", "drop", "sum", "y", "dsum", "dres")}
        dw, db, rstd, gain = (torch.zeros(s, device="cuda") for s in ((G, a, b), (G, b), (n,), (a,)))
        B.fg_linear_grouped(t["x"], n, stride(t["x"]), c, None, src, od, fd, len(order), G, a, b, W, None, None, 0, o["out"], n, stride(o["out"]), c)
        B.fg_linear_grouped_backward(t["x"], n, stride(t["x"]), c, src, t["dh"], stride(t["dh"]), c, t["h"], stride(t["h"]), n, od, fd, len(order), G, a, b, W, o["dx"],
                                     stride(o["dx"]), c, dw, db, ws, ws.numel())
        B.fg_dropout(t["x"], stride(t["x"]), c, od, None, len(order), n, a, p, key, o["drop"], stride(o["drop"]))
        B.fg_residual_norm(t["x"], stride(t["x"]), c, t["res"], stride(t["res"]), c, od, None, len(order), n, a, p, key, None, 1e-6, o["sum"], stride(o["sum"]), o["y"],
                           stride(o["y"]), c, None, rstd)
        B.fg_residual_norm_backward(t["dh"], stride(t["dh"]), c, o["sum"], stride(o["sum"]), c, rstd, None, t["res"], stride(t["res"]), od, None, len(order), n, a, p, key,
                                    o["dsum"], stride(o["dsum"]), o["dres"], stride(o["dres"]), gain, ws, ws.numel())
        torch.cuda.synchronize()
        results.append([v.clone(memory_format=torch.contiguous_format) for v in (*o.values(), dw, db, rstd, gain)])
        del t, o
    for near, away in zip(*results):
        assert torch.equal(near, away) and bool((near != -77).any())


@gpu
def test_16_and_8_bit_layers_captured(B):
    """A serving step in 8 bits and a training step in bf16 with an fp32 sum, captured with one workspace and replayed with new inputs between eager calls."""
    n, G, a, b, p, key = 900, 4, 128, 136, 0.25, 11
    c = B.FG_BF16
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")
    bf = torch.bfloat16

    def inputs(seed):
        r = np.random.default_rng(seed)
        f = lambda *s: torch.from_numpy(r.standard_normal(s)).to(bf).cuda()
        return dict(types=torch.from_numpy(r.integers(0, G, n).astype(np.int32)).cuda(), x=f(n, a), W=f(G, a, b) / 8, dy=f(n, b), res=torch.from_numpy(r.standard_normal((n, b))).float().cuda(),
                    Wt=f(G, b, a), n_rows=torch.tensor([n - seed], device="cuda"))

    def outputs():
        return dict(order=z(n, dtype=torch.int32), offsets=z(G + 1, dtype=torch.int64), q=z(n, a, dtype=torch.float8_e4m3fn), qs=z(n), wq=z(G, b, a, dtype=torch.float8_e4m3fn), wqs=z(G, b),
                    served=z(n, b, dtype=bf), h=z(n, b), sum=z(n, b), y=z(n, b, dtype=torch.float8_e4m3fn), ys=z(n), rstd=z(n), dres=z(n, b), dh=z(n, b), gain=z(b), dx=z(n, a, dtype=bf),
                    dW=z(G, a, b), db=z(G, b))

    def steps(t, o, ws):
        st = torch.cuda.current_stream().cuda_stream
        B.fg_group_rows(t["types"], n, None, n, None, t["n_rows"], n, G, o["order"], o["offsets"], ws, ws.numel(), st)
        B.fg_quantize_rows(t["x"], 2 * a, c, n, a, o["q"], a, o["qs"], st)
        B.fg_quantize_rows(t["Wt"], 2 * a, c, G * b, a, o["wq"], a, o["wqs"], st)
        B.fg_linear_grouped(o["q"], n, a, B.FG_E4M3, o["qs"], None, o["order"], o["offsets"], n, G, a, b, o["wq"], o["wqs"], None, 1, o["served"], n, 2 * b, c, st)
        B.fg_linear_grouped(t["x"], n, 2 * a, c, None, None, o["order"], o["offsets"], n, G, a, b, t["W"], None, None, 1, o["h"], n, 4 * b, B.FG_F32, st)
        B.fg_residual_norm(o["h"], 4 * b, B.FG_F32, t["res"], 4 * b, B.FG_F32, None, t["n_rows"], n, n, b, p, key, None, 1e-6, o["sum"], 4 * b, o["y"], b, B.FG_E4M3, o["ys"],
                           o["rstd"], st)
        B.fg_residual_norm_backward(t["res"], 4 * b, B.FG_F32, o["sum"], 4 * b, B.FG_F32, o["rstd"], None, None, 0, None, t["n_rows"], n, n, b, p, key, o["dres"], 4 * b, o["dh"],
                                    4 * b, o["gain"], ws, ws.numel(), st)
        B.fg_linear_grouped_backward(t["x"], n, 2 * a, c, None, o["dh"], 4 * b, B.FG_F32, o["h"], 4 * b, n, o["order"], o["offsets"], n, G, a, b, t["W"], o["dx"], 2 * a, c, o["dW"],
                                     o["db"], ws, ws.numel(), st)

    space = lambda: z(max(B.fg_group_rows_workspace_bytes(n, G), B.fg_residual_norm_backward_workspace_bytes(n, b), B.fg_linear_grouped_backward_workspace_bytes(c, n, G, a, b)),
                      dtype=torch.uint8)
    data = [inputs(1), inputs(200)]
    want = []
    for d in data:
        want.append(outputs())
        steps(d, want[-1], space())
    torch.cuda.synchronize()
    assert all(bool((w["served"].float() != 0).any()) and bool((w["dW"] != 0).any()) for w in want)
    t, o, ws = inputs(3), outputs(), space()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        steps(t, o, ws)
    for i in (0, 1, 1, 0, 1):
        for k, v in data[i].items():
            t[k].copy_(v)
        for v in o.values():
            v.view(torch.uint8).zero_()
        g.replay()
        steps(data[1 - i], outputs(), space())      # an eager call between the replays
        torch.cuda.synchronize()
        for k, v in o.items():
            assert torch.equal(v.view(torch.uint8), want[i][k].view(torch.uint8)), (i, k)
