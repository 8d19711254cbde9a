"""Plain 64-bit statements of the typed layer calls (group, grouped product, residual norm, dropout, rows in 8 bits), on the CPU."""
import numpy as np
import torch

F8_MAX = 448.0
MASK = (1 << 64) - 1


def mix(z):
    z = np.asarray(z, np.uint64)
    z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
    z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    return z ^ (z >> np.uint64(31))


def word(key, counter):
    return mix(key + (np.asarray(counter, np.uint64) + np.uint64(1)) * np.uint64(0x9E3779B97F4A7C15))


def threshold(p):
    return int(np.floor(float(np.float32(p)) * 65536 + 0.5))


def keep(key, rows, d, p):
    """[rows, d]: which elements stay."""
    with np.errstate(over="ignore"):
        row = word(mix(np.uint64(key & MASK)), np.asarray(rows, np.uint64))
        bits = word(row[:, None], np.arange((d + 3) // 4))
    draws = np.stack([(bits >> np.uint64(16 * i)) & np.uint64(0xFFFF) for i in range(4)], -1).reshape(len(rows), -1)[:, :d]
    return torch.from_numpy(draws >= threshold(p))


def dropout(x, rows, p, key):
    """Rows `rows` of x (any type), dropped and scaled in fp64; the factor as fp32 holds it."""
    t = threshold(p)
    v = x[rows].double()
    if t == 0:
        return v
    factor = float(np.float32(65536 / (65536 - t))) if t < 65536 else 0.0
    return torch.where(keep(key, rows, x.shape[1], p), v * factor, torch.zeros((), dtype=torch.float64))


def group(groups, ids, rows, n_groups):
    """(order, offsets) as lists."""
    members = [[] for _ in range(n_groups)]
    n_positions = len(ids) if ids is not None else len(groups)
    for r in rows:
        if not 0 <= r < n_positions:
            continue
        v = ids[r] if ids is not None else r
        if 0 <= v < len(groups) and 0 <= groups[v] < n_groups:
            members[groups[v]].append(r)
    return [r for m in members for r in m], np.cumsum([0] + [len(m) for m in members]).tolist()


def quantise(x):
    """(8-bit values as fp32, scales): every step in fp32, as the calls define it."""
    x = x.float()
    amax = x.abs().amax(1).clamp_min(2.0 ** -100)
    q = (x * (F8_MAX * amax.reciprocal())[:, None]).clamp(-F8_MAX, F8_MAX)
    return q.to(torch.float8_e4m3fn).float(), amax / F8_MAX


def grouped_linear(x, W, bias, order, offsets, src, relu):
    """h rows in the order of `order` and, beside them, the sum of the products' magnitudes (what rounding goes by)."""
    x, W = x.double(), W.double()
    h = torch.zeros(len(order), W.shape[2], dtype=torch.float64)
    size = torch.zeros_like(h)
    for g in range(W.shape[0]):
        k = slice(offsets[g], offsets[g + 1])
        a = x[[src[r] if src is not None else r for r in order[k]]]
        h[k] = a @ W[g] + (bias[g].double() if bias is not None else 0)
        size[k] = a.abs() @ W[g].abs() + (bias[g].double().abs() if bias is not None else 0)
    return (h.clamp_min(0) if relu else h), size


def grouped_linear_backward(x, W, dh, h, order, offsets, src, operand=None):
    """dx (rows in the order of `order`), dW, db, each with the sum of magnitudes; dz is rounded to `operand` where it is multiplied."""
    x, W = x.double(), W.double()
    G, a, b = W.shape
    dx, dxs = torch.zeros(len(order), a, dtype=torch.float64), torch.zeros(len(order), a, dtype=torch.float64)
    dW, dWs = torch.zeros(G, a, b, dtype=torch.float64), torch.zeros(G, a, b, dtype=torch.float64)
    db, dbs = torch.zeros(G, b, dtype=torch.float64), torch.zeros(G, b, dtype=torch.float64)
    for g in range(G):
        k = slice(offsets[g], offsets[g + 1])
        pos = order[k]
        z = dh[pos].double()
        if h is not None:
            z = torch.where(h[pos] > 0, z, torch.zeros((), dtype=torch.float64))
        db[g], dbs[g] = z.sum(0), z.abs().sum(0)
        if operand is not None:
            z = z.to(operand).double()
        xs = x[[src[r] if src is not None else r for r in pos]]
        dx[k], dxs[k] = z @ W[g].T, z.abs() @ W[g].abs().T
        dW[g], dWs[g] = xs.T @ z, xs.abs().T @ z.abs()
    return (dx, dxs), (dW, dWs), (db, dbs)


def residual_norm(x, residual, rows, p, key, weight, eps):
    """s, rstd, y of the listed rows, and the size of the addends of s."""
    v = dropout(x, rows, p, key)
    size = v.abs()
    if residual is not None:
        v = v + residual[rows].double()
        size = size + residual[rows].double().abs()
    rstd = 1 / torch.sqrt((v * v).mean(1) + float(np.float32(eps)))
    y = v * rstd[:, None] * (weight.double() if weight is not None else 1.0)
    return v, rstd, y, size


def residual_norm_backward(dy, s, rstd, weight, dsum_in, rows, p, key):
    """ds, dx, dw of the listed rows (rstd as given), and the sizes that rounding goes by."""
    dy, s, r = dy[rows].double(), s[rows].double(), rstd[rows].double()[:, None]
    xh = s * r
    t = dy * (weight.double() if weight is not None else 1.0)
    ds = r * (t - xh * (t * xh).mean(1, keepdim=True))
    size = r * (t.abs() + xh.abs() * (t * xh).abs().mean(1, keepdim=True))
    if dsum_in is not None:
        ds, size = ds + dsum_in[rows].double(), size + dsum_in[rows].double().abs()
    full = torch.zeros(int(max(rows)) + 1 if len(rows) else 0, ds.shape[1], dtype=torch.float64)
    if len(rows):
        full[rows] = ds
    return ds, dropout(full, rows, p, key), (dy * xh).sum(0), size, (dy * xh).abs().sum(0)
