"""Plain 64-bit statements of a student block's calls (gated layer, group norm, distillation loss) and their gradients, and how far a computation in
fp32 may be from them. Everything is on the device that its inputs are on."""
import math

import torch

F64 = torch.float64
ACTS = ("none", "relu", "silu", "gelu", "sigmoid")
# |act'| and |act''| are at most
SLOPE = {"none": 1.0, "relu": 1.0, "silu": 1.1, "gelu": 1.13, "sigmoid": 0.25}
BEND = {"none": 0.0, "relu": 0.0, "silu": 0.5, "gelu": 0.8, "sigmoid": 0.1}


def act(name, u):
    if name == "none":
        return u
    if name == "relu":
        return torch.where(u > 0, u, torch.zeros((), dtype=u.dtype, device=u.device))
    if name == "gelu":
        return u * torch.special.ndtr(u)
    return u * torch.sigmoid(u) if name == "silu" else torch.sigmoid(u)


def slope(name, u):
    if name == "none":
        return torch.ones_like(u)
    if name == "relu":
        return (u > 0).to(u.dtype)
    if name == "gelu":
        return torch.special.ndtr(u) + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(u)
    return s + u * s * (1 - s) if name == "silu" else s * (1 - s)


def act_off(name, u):
    """How far act(u) in fp32 may be for an exact u: a handful of roundings, each to half a step, exp and erfc to 4 steps; e^x and erfc(x) of a rounded
    argument are off by that rounding times |x| and 2 x^2 (x^2 = u^2 / 2). Results below 2^-100 may vanish."""
    f = act(name, u).abs()
    if name in ("none", "relu"):
        return torch.zeros_like(f)
    return f * (16 + u.abs() + u * u) * 2.0 ** -24 + 2.0 ** -100


def slope_off(name, u):
    """The same for act'(u), whose terms are up to 1 and |u| e^(-u^2/2) or |u| s (1 - s), all below 1.2."""
    if name in ("none", "relu"):
        return torch.zeros_like(u)
    return (24 + 3 * u.abs().clamp(max=20)) * 2.0 ** -24 + torch.zeros_like(u)


def members(order, offsets, n, ids=None, rows=None):
    """[(group, positions, rows of x)] of the entries that exist; order None: position k itself."""
    out = []
    for g in range(len(offsets) - 1):
        got = []
        for k in range(offsets[g], offsets[g + 1]):
            r = int(order[k]) if order is not None else k
            if not 0 <= r < n:
                continue
            s = int(ids[r]) if ids is not None else r
            if rows is not None and not 0 <= s < rows:
                continue
            got.append((r, s))
        out.append((g, torch.tensor([p for p, _ in got], dtype=torch.long), torch.tensor([s for _, s in got], dtype=torch.long)))
    return out


def gated(x, W, bias, name):
    """z, h of rows x with one group's weights; and how far they may be."""
    x, W = x.to(F64), W.to(F64)
    z, size = torch.mm(x, W), torch.mm(x.abs(), W.abs())
    if bias is not None:
        z, size = z + bias.to(F64), size + bias.to(F64).abs()
    z_off = (x.shape[1] + 8) * 2.0 ** -23 * size
    b = W.shape[1] // 2
    u, v, du, dv = z[:, :b], z[:, b:], z_off[:, :b], z_off[:, b:]
    f = act(name, u)
    df = SLOPE[name] * du + act_off(name, u)
    h = f * v
    return z, h, z_off, df * (v.abs() + dv) + f.abs() * dv + 2.0 ** -23 * h.abs()


def gated_dz(z, dh, name):
    """dz, and how far it may be before its rounding to a narrower type."""
    z, dh = z.to(F64), dh.to(F64)
    b = dh.shape[1]
    u, v = z[:, :b], z[:, b:]
    du, dv = dh * v * slope(name, u), dh * act(name, u)
    off_u = dh.abs() * v.abs() * slope_off(name, u) + 2.0 ** -22 * du.abs()
    off_v = dh.abs() * act_off(name, u) + 2.0 ** -22 * dv.abs()
    return torch.cat([du, dv], 1), torch.cat([off_u, off_v], 1)


def norm_statistics(x, blocks, eps):
    """mean, rstd [blocks] of one group's rows."""
    if not len(x):
        return torch.zeros(blocks, dtype=F64, device=x.device), torch.full((blocks,), eps, dtype=F64, device=x.device) ** -0.5
    x = x.to(F64).reshape(len(x), blocks, -1)
    mean = x.mean((0, 2))
    return mean, ((x - mean[:, None]).square().mean((0, 2)) + eps) ** -0.5


def norm_rows(x, mean, rstd, weight, bias, name):
    """y for given statistics, and how far it may be where mean and rstd are rounded to fp32."""
    n, blocks = len(x), len(mean)
    x = x.to(F64).reshape(n, blocks, -1)
    w = weight.to(F64) if weight is not None else torch.ones(x.shape[1] * x.shape[2], dtype=F64, device=x.device)
    b = bias.to(F64) if bias is not None else torch.zeros_like(w)
    c, r = x - mean[:, None], rstd[:, None]
    xh, off = (c * r).flatten(1), ((2.0 ** -23 * mean.abs()[:, None] + 2.0 ** -23 * c.abs()) * r).flatten(1) + 2.0 ** -22 * (c * r).abs().flatten(1)
    u, off = xh * w + b, off * w.abs() + 2.0 ** -23 * ((xh * w).abs() + b.abs())
    return act(name, u), SLOPE[name] * off + act_off(name, u), xh, u


def norm_backward(x, dy, mean, rstd, weight, bias, name):
    """dx, dw, db of one group's rows for the given (fp32) statistics, each with how far it may be; and the smallest |u|, where ReLU has its corner."""
    n, blocks = len(x), len(mean)
    mean, rstd, dy = mean.to(F64), rstd.to(F64), dy.to(F64)
    _, _, xh, u = norm_rows(x, mean, rstd, weight, bias, name)
    c = x.to(F64).reshape(n, blocks, -1) - mean[:, None]
    # here mean and rstd are what they are: their difference from x and two products are rounded
    xh_off = 3 * 2.0 ** -24 * xh.abs()
    w = weight.to(F64) if weight is not None else torch.ones(xh.shape[1], dtype=F64, device=x.device)
    b = bias.to(F64) if bias is not None else torch.zeros_like(w)
    u_off = w.abs() * xh_off + 2.0 ** -23 * ((xh * w).abs() + b.abs())
    t = dy * slope(name, u)
    t_off = dy.abs() * (BEND[name] * u_off + slope_off(name, u)) + 2.0 ** -24 * t.abs()
    split = lambda v: v.reshape(n, blocks, -1)
    q, q_off = split(t * w), split(t_off * w.abs() + 2.0 ** -24 * (t * w).abs())
    xg, xg_off = split(xh), split(xh_off)
    m1, m2 = q.mean((0, 2)), (q * xg).mean((0, 2))
    m1_off = q_off.mean((0, 2)) + 2.0 ** -24 * m1.abs()
    m2_off = (q_off * xg.abs() + q.abs() * xg_off).mean((0, 2)) + 2.0 ** -24 * m2.abs()
    r = rstd[:, None]
    dx = r * (q - m1[:, None] - xg * m2[:, None])
    off = r * (q_off + m1_off[:, None] + xg.abs() * m2_off[:, None] + xg_off * m2.abs()[:, None] + 2.0 ** -22 * (q.abs() + m1.abs()[:, None] + (xg * m2[:, None]).abs()))
    dw, db = (t * xh).sum(0), t.sum(0)
    # sums in fp32 of up to 256 rows a thread (2^-24 each of what has been added up), then in fp64
    dw_off = (t_off * xh.abs() + t.abs() * xh_off).sum(0) + 300 * 2.0 ** -24 * (t * xh).abs().sum(0)
    db_off = t_off.sum(0) + 300 * 2.0 ** -24 * t.abs().sum(0)
    return (dx.flatten(1), off.flatten(1)), (dw, dw_off), (db, db_off), float(u.abs().min()) if u.numel() else math.inf


def distill(z, idx, val, label, T, alpha, weight, scale):
    """loss [n], dh [n, d] of rows z with their teacher's entries idx, val [n, k] (None: none), each with how far it may be."""
    z = z.to(F64)
    n, d = z.shape
    T, alpha = float(torch.tensor(T, dtype=torch.float32)), float(torch.tensor(alpha, dtype=torch.float32))
    w = weight.to(F64) if weight is not None else torch.ones(n, dtype=F64, device=z.device)
    loss, dh = torch.zeros(n, dtype=F64, device=z.device), torch.zeros_like(z)
    loss_off, dh_off = torch.zeros_like(loss), torch.zeros_like(z)
    u = 2.0 ** -24
    eps = lambda log_q: (24 + 3 * log_q.abs().clamp(max=200)) * u      # e^x in fp32 of an x that is off by 3 roundings, over a sum of such
    for i in range(n):
        y = int(label[i]) if label is not None else -1
        taught, P = False, torch.zeros(d, dtype=F64, device=z.device)
        if idx is not None and alpha > 0:
            there = (idx[i] >= 0) & (idx[i] < d)
            c, v = idx[i][there].long(), val[i][there].to(F64) / T
            taught = bool((v != -math.inf).any())
        if taught:
            log_p, log_q = torch.log_softmax(v, 0), torch.log_softmax(z[i] / T, 0)
            p = log_p.exp()
            P.index_add_(0, c, p)
            terms = torch.where(p > 0, p * (log_p - log_q[c]), torch.zeros((), dtype=F64, device=z.device))
            size = torch.where(p > 0, p * (log_p.abs() + log_q[c].abs() + z[i][c].abs() / T + v.abs() + 1), torch.zeros((), dtype=F64, device=z.device))
            loss[i] += alpha * T * T * terms.sum()
            loss_off[i] += alpha * T * T * (size * (24 + 3 * log_p.abs().clamp(max=200)) * u).sum()
            q = log_q.exp()
            dh[i] += alpha * T * (q - P)
            dh_off[i] += alpha * T * (q * eps(log_q) + P * (40 + 3 * v[v != -math.inf].abs().max()) * u)
        if 0 <= y < d and alpha < 1:
            log_q = torch.log_softmax(z[i], 0)
            one = torch.zeros(d, dtype=F64, device=z.device)
            one[y] = 1
            loss[i] -= (1 - alpha) * log_q[y]
            loss_off[i] += (1 - alpha) * (log_q[y].abs() + z[i][y].abs() + 1) * 24 * u
            q = log_q.exp()
            dh[i] += (1 - alpha) * (q - one)
            dh_off[i] += (1 - alpha) * (q * eps(log_q) + one * 8 * u)
    loss, loss_off = loss * w, loss_off * w.abs() + 4 * u * (loss * w).abs()
    g = (scale * w)[:, None]
    return loss, loss_off, dh * g, (dh_off + 4 * u * dh.abs()) * g.abs()
