"""The calls of a student's block as they are used together: rows of a table by node, grouped by type; a gated layer, a group norm over each type's rows, a
linear layer to classes, the loss against stored logits, and every gradient back. Each call against the statement of what it was given; the whole against
64-bit gradients by autograd and by differences; captured and replayed; on streams of their own; rows more than 2^32 bytes apart."""
import math

import numpy as np
import pytest
import torch

from tests import student_reference as R
from tests.test_student_block import B, HALF, T, TINY, act_code, close, code, stride  # noqa: F401 (B: the fixture)

gpu = pytest.mark.gpu
SIZES = dict(n=700, table=1500, groups=3, d_in=96, hidden=64, blocks=4, classes=56, k=8)
TEMP, ALPHA, EPS = 2.0, 0.6, 1e-3


def inputs(seed, dtype, s=SIZES):
    r = np.random.default_rng(seed)
    f = lambda *shape, scale=1.0: torch.from_numpy(r.standard_normal(shape) * scale)
    n, table, G, a, b, c, k = (s[x] for x in ("n", "table", "groups", "d_in", "hidden", "classes", "k"))
    listed = np.sort(r.permutation(n)[:n - n // 8]).astype(np.int32)
    t = dict(types=torch.from_numpy(r.integers(0, G, table).astype(np.int32)), ids=torch.from_numpy(r.integers(0, table, n).astype(np.int32)),
             rows=torch.from_numpy(np.concatenate([listed, np.zeros(n - len(listed), np.int32)])), n_rows=torch.tensor([len(listed)]),
             x=f(table, a).to(T[dtype]), W=f(G, a, 2 * b, scale=a ** -0.5).to(T[dtype]), bias=f(G, 2 * b, scale=0.3).float(), gain=(1 + f(b, scale=0.2)).float(),
             shift=f(b, scale=0.2).float(), head=f(G, b, c, scale=b ** -0.5).to(T[dtype]), hbias=f(G, c, scale=0.1).float(),
             top=torch.from_numpy(np.stack([r.permutation(c)[:k] for _ in range(table)]).astype(np.int32)), val=f(table, k, scale=2.0).to(torch.float16),
             label=torch.from_numpy(r.integers(-1, c, n).astype(np.int32)), weight=torch.from_numpy(r.random(n)).float())
    t["types"][r.permutation(table)[:20]] = -1      # nodes of no type
    return {key: v.cuda() for key, v in t.items()}


def outputs(dtype, s=SIZES, fill=0.0):
    n, G, a, b, c = (s[x] for x in ("n", "groups", "d_in", "hidden", "classes"))
    z = lambda *shape, dtype=torch.float32: torch.full(shape, fill, dtype=dtype, device="cuda")
    e = T[dtype]
    return dict(order=z(n, dtype=torch.int32), offsets=z(G + 1, dtype=torch.int64), h=z(n, b, dtype=e), z=z(n, 2 * b, dtype=e), y=z(n, b, dtype=e), mean=z(G, s["blocks"]),
                rstd=z(G, s["blocks"]), logits=z(n, c, dtype=e), loss=z(n), dlogits=z(n, c, dtype=e), dy=z(n, b, dtype=e), dhead=z(G, b, c), dhbias=z(G, c), dh=z(n, b, dtype=e),
                dgain=z(b), dshift=z(b), dx=z(n, a, dtype=e), dW=z(G, a, 2 * b), dbias=z(G, 2 * b))


def space(B, dtype, s=SIZES, fill=255):
    n, G, a, b, c, blocks = (s[x] for x in ("n", "groups", "d_in", "hidden", "classes", "blocks"))
    d = code(B, dtype)
    need = max(B.fg_group_rows_workspace_bytes(n, G), B.fg_gated_linear_grouped_backward_workspace_bytes(d, n, G, a, b), B.fg_group_norm_workspace_bytes(n, G, b, blocks),
               B.fg_group_norm_backward_workspace_bytes(n, G, b, blocks), B.fg_linear_grouped_backward_workspace_bytes(d, n, G, b, c))
    return torch.full((need,), fill, dtype=torch.uint8, device="cuda")


def step(B, t, o, ws, dtype, act="silu", s=SIZES, stream=None):
    n, table, G, a, b, c, k, blocks = (s[x] for x in ("n", "table", "groups", "d_in", "hidden", "classes", "k", "blocks"))
    st = torch.cuda.current_stream().cuda_stream if stream is None else stream
    d, w = code(B, dtype), ws.numel()
    B.fg_group_rows(t["types"], table, t["ids"], n, t["rows"], t["n_rows"], n, G, o["order"], o["offsets"], ws, w, st)
    B.fg_gated_linear_grouped(t["x"], table, stride(t["x"]), d, t["ids"], o["order"], o["offsets"], n, G, a, b, t["W"], t["bias"], act_code(B, act), o["h"], n, stride(o["h"]), d, o["z"],
                              stride(o["z"]), st)
    B.fg_group_norm(o["h"], stride(o["h"]), d, o["order"], o["offsets"], n, G, n, b, blocks, t["gain"], t["shift"], EPS, act_code(B, act), o["y"], stride(o["y"]), d, o["mean"], o["rstd"],
                    ws, w, st)
    B.fg_linear_grouped(o["y"], n, stride(o["y"]), d, None, None, o["order"], o["offsets"], n, G, b, c, t["head"], None, t["hbias"], 0, o["logits"], n, stride(o["logits"]), d, st)
    B.fg_distill_loss(o["logits"], stride(o["logits"]), d, t["rows"], t["n_rows"], n, n, c, t["ids"], t["top"], t["val"], B.FG_F16, table, k, t["label"], TEMP, ALPHA, t["weight"], 1.0,
                      o["loss"], o["dlogits"], stride(o["dlogits"]), d, st)
    B.fg_linear_grouped_backward(o["y"], n, stride(o["y"]), d, None, o["dlogits"], stride(o["dlogits"]), d, None, 0, n, o["order"], o["offsets"], n, G, b, c, t["head"], o["dy"],
                                 stride(o["dy"]), d, o["dhead"], o["dhbias"], ws, w, st)
    B.fg_group_norm_backward(o["dy"], stride(o["dy"]), d, o["h"], stride(o["h"]), d, o["mean"], o["rstd"], t["gain"], t["shift"], act_code(B, act), o["order"], o["offsets"], n, G, n, b,
                             blocks, o["dh"], stride(o["dh"]), o["dgain"], o["dshift"], ws, w, st)
    B.fg_gated_linear_grouped_backward(t["x"], table, stride(t["x"]), d, t["ids"], o["dh"], stride(o["dh"]), d, o["z"], stride(o["z"]), n, o["order"], o["offsets"], n, G, a, b, t["W"],
                                       act_code(B, act), o["dx"], stride(o["dx"]), d, o["dW"], B.FG_F32, o["dbias"], ws, w, st)


def cpu(d):
    return {k: v.cpu() for k, v in d.items()}


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_each_call_of_a_step(B, dtype, act):
    """Every call against the statement of what the calls before it left."""
    s = SIZES
    t, o = inputs(5, dtype), outputs(dtype, fill=-77)
    step(B, t, o, space(B, dtype), dtype, act)
    torch.cuda.synchronize()
    t, o = cpu(t), cpu(o)
    listed = t["rows"][:int(t["n_rows"])].long()
    types = t["types"][t["ids"].long()]
    half, op = HALF[dtype], HALF[dtype] if dtype != "f32" else 0.0
    grouped = listed[types[listed] >= 0]
    rest = np.setdiff1d(np.arange(s["n"]), grouped.numpy())
    assert int(o["offsets"][-1]) == len(grouped)
    for name in ("h", "z", "y", "logits", "dy", "dh", "dx"):
        assert bool((o[name][rest] == -77).all()), name
    gain, gain_off, shift, shift_off = (torch.zeros(s["hidden"], dtype=torch.float64) for _ in range(4))
    at = o["offsets"].tolist()
    for g in range(s["groups"]):
        pos = o["order"][at[g]:at[g + 1]].long()
        assert torch.equal(pos.sort().values, listed[types[listed] == g])
        x = t["x"][t["ids"][pos].long()]
        want_z, want_h, z_off, h_off = R.gated(x, t["W"][g], t["bias"][g], act)
        close(o["z"][pos], want_z, z_off + half * want_z.abs() + TINY[dtype], "z")
        close(o["h"][pos], want_h, h_off + half * want_h.abs() + TINY[dtype], "h")
        m, r = R.norm_statistics(o["h"][pos], s["blocks"], float(np.float32(EPS)))
        want, off, _, _ = R.norm_rows(o["h"][pos], m, r, t["gain"], t["shift"], act)
        close(o["y"][pos], want, off + half * want.abs() + TINY[dtype], "y")
        (want, off), (gw, gw_off), (gb, gb_off), _ = R.norm_backward(o["h"][pos], o["dy"][pos], o["mean"][g], o["rstd"][g], t["gain"], t["shift"], act)
        close(o["dh"][pos], want, off + half * want.abs() + TINY[dtype], "dh")
        for sum_, v in ((gain, gw), (gain_off, gw_off), (shift, gb), (shift_off, gb_off)):
            sum_ += v
        dz, dz_off = R.gated_dz(o["z"][pos], o["dh"][pos], act)
        close(o["dbias"][g], dz.sum(0), (dz_off + (len(pos) + 8) * 2.0 ** -23 * dz.abs()).sum(0) + 2.0 ** -24 * dz.sum(0).abs(), "dbias")
        dz_off = dz_off + op * (dz.abs() + dz_off) + (TINY[dtype] if op else 0)
        Wt = t["W"][g].double().T
        want = dz @ Wt
        close(o["dx"][pos], want, (dz_off + (2 * s["hidden"] + 8) * 2.0 ** -23 * dz.abs()) @ Wt.abs() + half * want.abs() + TINY[dtype], "dx")
        want = x.double().T @ dz
        close(o["dW"][g], want, x.double().abs().T @ (dz_off + (len(pos) + 8) * 2.0 ** -23 * dz.abs()) + 2.0 ** -24 * want.abs(), "dW")
    close(o["dgain"], gain, gain_off + 2.0 ** -23 * gain.abs() + 2.0 ** -100, "dgain")
    close(o["dshift"], shift, shift_off + 2.0 ** -23 * shift.abs() + 2.0 ** -100, "dshift")
    # (a listed row of no type has no logits: its -77 are all alike)
    node = t["ids"][listed].long()
    want, off, grad, grad_off = R.distill(o["logits"][listed], t["top"][node], t["val"][node], t["label"][listed], TEMP, ALPHA, t["weight"][listed], 1.0)
    close(o["loss"][listed], want, off + 2.0 ** -24 * want.abs(), "loss")
    close(o["dlogits"][listed], grad, grad_off + half * grad.abs() + TINY[dtype], "dlogits")


def whole(t, act, s, listed, types, p):
    """The sum of the losses in 64 bits, of parameters and rows `p` (x by position)."""
    f = lambda u: u * torch.sigmoid(u) if act == "silu" else 0.5 * u * (1 + torch.erf(u / math.sqrt(2.0)))
    b, total = s["hidden"], 0.0
    for g in range(s["groups"]):
        pos = listed[types[listed] == g]
        z = p["x"][pos] @ p["W"][g] + p["bias"][g]
        h = (f(z[:, :b]) * z[:, b:]).reshape(len(pos), s["blocks"], -1)
        mean = h.mean((0, 2), keepdim=True)
        xh = ((h - mean) * ((h - mean).square().mean((0, 2), keepdim=True) + float(np.float32(EPS))) ** -0.5).reshape(len(pos), b)
        logits = f(xh * p["gain"] + p["shift"]) @ p["head"][g] + p["hbias"][g]
        node = t["ids"][pos].long()
        share = torch.softmax(t["val"][node].double() / TEMP, 1)
        log_q, label = torch.log_softmax(logits / TEMP, 1), t["label"][pos].long()
        loss = ALPHA32 * TEMP ** 2 * (share * (share.log() - log_q.gather(1, t["top"][node].long()))).sum(1)
        hard = -torch.log_softmax(logits, 1).gather(1, label.clamp(min=0)[:, None])[:, 0]
        total = total + (t["weight"][pos].double() * (loss + (1 - ALPHA32) * torch.where(label >= 0, hard, torch.zeros(()).double()))).sum()
    return total


ALPHA32 = float(np.float32(ALPHA))
NAMES = dict(x="dx", W="dW", bias="dbias", gain="dgain", shift="dshift", head="dhead", hbias="dhbias")


@gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradients_of_a_step_by_autograd_and_by_differences(B, act):
    """fp32. Six calls in a row, each off by at most 2 K 2^-24 of the magnitudes that it sums with K of 256 rows or fewer columns at most; where values cancel
    the magnitudes are some ten times the sums: 6 * 2^-15 * 10 < 2^-9 of a tensor's largest gradient."""
    s = SIZES
    t, o = inputs(6, "f32"), outputs("f32")
    step(B, t, o, space(B, "f32"), "f32", act)
    torch.cuda.synchronize()
    t, o = cpu(t), cpu(o)
    listed = t["rows"][:int(t["n_rows"])].long()
    types = t["types"][t["ids"].long()]
    p = {k: t[k].double() for k in NAMES}
    p["x"] = p["x"][t["ids"].long()]
    leaves = {k: v.clone().requires_grad_(True) for k, v in p.items()}
    whole(t, act, s, listed, types, leaves).backward()
    for k, name in NAMES.items():
        want = leaves[k].grad
        assert float((o[name].double() - want).abs().max()) <= 2.0 ** -9 * float(want.abs().max()), name
    # a leaf at a time, along a random direction; the differences are off by the third derivative times the square of the step, 1e-12, and rounding over it, 1e-9
    g = torch.Generator().manual_seed(8)
    for k, name in NAMES.items():
        d = torch.randn(p[k].shape, dtype=torch.float64, generator=g)
        ends = [float(whole(t, act, s, listed, types, {**p, k: p[k] + e * d})) for e in (1e-6, -1e-6)]
        got, size = float((o[name].double() * d).sum()), float((o[name].double() * d).square().sum().sqrt())
        assert abs(got - (ends[0] - ends[1]) / 2e-6) <= 2.0 ** -9 * size + 1e-5, name


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_step_captured_twice_with_one_workspace(B, dtype):
    """Two graphs whose kernels share a workspace, replayed in turn with new inputs, eager calls of the same tensors between them."""
    sizes = [SIZES, dict(n=3000, table=900, groups=5, d_in=40, hidden=136, blocks=17, classes=1032, k=20)]
    data = [[inputs(10 + i, dtype, s) for i in range(2)] for s in sizes]
    want = []
    for s, two in zip(sizes, data):
        want.append([])
        for d in two:
            want[-1].append(outputs(dtype, s))
            step(B, d, want[-1][-1], space(B, dtype, s), dtype, s=s)
    torch.cuda.synchronize()
    ws = max((space(B, dtype, s) for s in sizes), key=len)
    held, graphs = [], []
    for s in sizes:
        t, o = inputs(3, dtype, s), outputs(dtype, s)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(B, t, o, ws, dtype, s=s)
        held.append((t, o))
        graphs.append(g)
    for which, i in ((0, 0), (1, 1), (0, 1), (1, 0), (1, 1), (0, 0), (1, 0)):
        t, o = held[which]
        for k, v in data[which][i].items():
            t[k].copy_(v)
        for v in o.values():
            v.view(torch.uint8).zero_()
        ws.fill_(255)
        graphs[which].replay()
        step(B, data[which][1 - i], outputs(dtype, sizes[which]), ws, dtype, s=sizes[which])
        torch.cuda.synchronize()
        for k, v in o.items():
            assert torch.equal(v.view(torch.uint8), want[which][i][k].view(torch.uint8)), (which, i, k)


@gpu
def test_steps_on_two_streams_at_once(B):
    s = dict(n=20_000, table=5000, groups=6, d_in=64, hidden=128, blocks=8, classes=504, k=16)
    data, want = [inputs(i, "bf16", s) for i in (1, 2)], []
    for d in data:
        want.append(outputs("bf16", s))
        step(B, d, want[-1], space(B, "bf16", s), "bf16", s=s)
    torch.cuda.synchronize()
    got, streams, spaces = [outputs("bf16", s) for _ in data], [torch.cuda.Stream() for _ in data], [space(B, "bf16", s) for _ in data]
    torch.cuda.synchronize()
    for _ in range(3):
        for d, o, st, ws in zip(data, got, streams, spaces):
            step(B, d, o, ws, "bf16", s=s, stream=st.cuda_stream)
    torch.cuda.synchronize()
    for o, w in zip(got, want):
        for k in o:
            assert torch.equal(o[k].view(torch.uint8), w[k].view(torch.uint8)), k


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_more_than_32_bits_apart(B, dtype):
    """The same values in rows that lie 64 MiB apart: the same bits, in every call that takes a stride; few rows and a group norm and a loss of wider ones."""
    n, a, b, apart = 75, 72, 40, 1 << 26
    e, c = T[dtype].itemsize, code(B, dtype)
    d = 600
    r = torch.Generator().manual_seed(3)
    f = lambda *s: torch.randn(*s, generator=r).to(T[dtype]).cuda()
    far = [torch.empty(n * apart // e, dtype=T[dtype], device="cuda").as_strided((n, d), (apart // e, 1)) for _ in range(3)]
    order = torch.randperm(n, generator=r).int().cuda()
    off = torch.tensor([0, 30, n], device="cuda")
    W, x, z, dh, wide, dy = f(2, a, 2 * b), f(n, a), f(n, 2 * b), f(n, b), f(n, d), f(n, d)
    idx, val = torch.randint(0, d, (n, 6), generator=r).int().cuda(), torch.randn(n, 6, generator=r).cuda()
    mean, rstd = (torch.empty(2, 4, device="cuda") for _ in range(2))
    dw, db, gw, gb, loss = (torch.zeros(s, device="cuda") for s in ((2, a, 2 * b), (2, 2 * b), (d,), (d,), (n,)))
    ws = torch.zeros(max(B.fg_gated_linear_grouped_backward_workspace_bytes(c, n, 2, a, b), B.fg_group_norm_workspace_bytes(n, 2, d, 4),
                         B.fg_group_norm_backward_workspace_bytes(n, 2, d, 4)), dtype=torch.uint8, device="cuda")
    w = ws.numel()

    def put(t, v):
        t[:, :v.shape[1]].copy_(v)
        return t

    def calls(place):
        got = []
        p, q, s = place(0, x), place(1, torch.zeros(n, b, dtype=T[dtype], device="cuda")), place(2, torch.zeros(n, 2 * b, dtype=T[dtype], device="cuda"))
        B.fg_gated_linear_grouped(p, n, stride(p), c, None, order, off, n, 2, a, b, W, None, B.FG_ACT_SILU, q, n, stride(q), c, s, stride(s))
        got += [q[:, :b].clone(), s[:, :2 * b].clone()]
        p, q, s = place(0, x), place(1, dh), place(2, z)
        B.fg_gated_linear_grouped_backward(p, n, stride(p), c, None, q, stride(q), c, s, stride(s), n, order, off, n, 2, a, b, W, B.FG_ACT_SILU, None, 0, c, dw, B.FG_F32, db, ws, w)
        got += [dw.clone(), db.clone()]
        s = place(2, z)
        p = place(0, torch.zeros(n, a, dtype=T[dtype], device="cuda"))
        B.fg_gated_linear_grouped_backward(x, n, stride(x), c, None, q, stride(q), c, s, stride(s), n, order, off, n, 2, a, b, W, B.FG_ACT_SILU, p, stride(p), c, None, B.FG_F32, None, ws, w)
        got += [p[:, :a].clone()]
        p, q = place(0, wide), place(1, torch.zeros_like(wide))
        B.fg_group_norm(p, stride(p), c, order, off, n, 2, n, d, 4, None, None, 1e-5, B.FG_ACT_GELU, q, stride(q), c, mean, rstd, ws, w)
        got += [q.clone(), mean.clone(), rstd.clone()]
        q, s = place(1, dy), place(2, torch.zeros_like(wide))
        B.fg_group_norm_backward(q, stride(q), c, p, stride(p), c, mean, rstd, None, None, B.FG_ACT_GELU, order, off, n, 2, n, d, 4, s, stride(s), gw, gb, ws, w)
        got += [s.clone(), gw.clone(), gb.clone()]
        s = place(2, torch.zeros_like(wide))
        B.fg_distill_loss(p, stride(p), c, order, None, n, n, d, None, idx, val, B.FG_F32, n, 6, None, 2.0, 1.0, None, 1.0, loss, s, stride(s), c)
        got += [s.clone(), loss.clone()]
        torch.cuda.synchronize()
        return got

    want = calls(lambda i, v: v.clone())
    got = calls(lambda i, v: put(far[i], v))
    for i, (g, v) in enumerate(zip(got, want)):
        assert bool((v != 0).any()) and torch.equal(g, v), i


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_groups_far_into_the_weights(B, dtype):
    """Weights of more than 2^31 values: the last groups' products."""
    G, a, b, n = 600, 2048, 1024, 64      # 2.5e9 values
    c, e = code(B, dtype), T[dtype].itemsize
    W = torch.empty(G, a, 2 * b, dtype=T[dtype], device="cuda")
    r = torch.Generator().manual_seed(4)
    for g in (0, 1, G - 1):
        W[g] = (torch.randn(a, 2 * b, generator=r) / math.sqrt(a)).to(T[dtype]).cuda()
    x, dh = torch.randn(n, a, generator=r).to(T[dtype]).cuda(), torch.randn(n, b, generator=r).to(T[dtype]).cuda()
    off = torch.full((G + 1,), 40, dtype=torch.int64)
    off[0], off[-1] = 0, n
    off = off.cuda()
    h, z, dx = torch.empty(n, b, dtype=T[dtype], device="cuda"), torch.empty(n, 2 * b, dtype=T[dtype], device="cuda"), torch.empty(n, a, dtype=T[dtype], device="cuda")
    B.fg_gated_linear_grouped(x, n, a * e, c, None, None, off, n, G, a, b, W, None, B.FG_ACT_SILU, h, n, b * e, c, z, 2 * b * e)
    need = B.fg_gated_linear_grouped_backward_workspace_bytes(c, n, G, a, b)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    B.fg_gated_linear_grouped_backward(x, n, a * e, c, None, dh, b * e, c, z, 2 * b * e, n, None, off, n, G, a, b, W, B.FG_ACT_SILU, dx, a * e, c, None, B.FG_F32, None, ws, need)
    torch.cuda.synchronize()
    op = HALF[dtype] if dtype != "f32" else 0.0
    for g, lo, hi in ((0, 0, 40), (G - 1, 40, n)):
        want_z, want, z_off, off_h = R.gated(x[lo:hi].cpu(), W[g].cpu(), None, "silu")
        close(h[lo:hi].cpu(), want, off_h + HALF[dtype] * want.abs() + TINY[dtype], "h")
        close(z[lo:hi].cpu(), want_z, z_off + HALF[dtype] * want_z.abs() + TINY[dtype], "z")
        dz, dz_off = R.gated_dz(z[lo:hi].cpu(), dh[lo:hi].cpu(), "silu")
        dz_off = dz_off + op * (dz.abs() + dz_off) + (TINY[dtype] if op else 0)
        Wt = W[g].cpu().double().T
        want = dz @ Wt
        close(dx[lo:hi].cpu(), want, (dz_off + (2 * b + 8) * 2.0 ** -23 * dz.abs()) @ Wt.abs() + HALF[dtype] * want.abs() + TINY[dtype], "dx")
