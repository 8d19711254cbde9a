"""The operators of a typed layer block, as they are measured: each case one pass through one of them.

  grouped     rows are sorted by their node type on the device and multiplied with their type's weight matrix
              (`fg_group_rows`, `fg_linear_grouped`; 8 bits: `fg_quantize_rows` in front): forward
  grouped_bw  the gradients of that product: rows, weights, biases (`fg_linear_grouped_backward`)
  norm        residual sum with dropout on the branch, root-mean-square norm, output in the rows' type or in 8 bits
              with a scale per row (`fg_residual_norm`)
  norm_bw     its gradients: both addends and the gain (`fg_residual_norm_backward`)
  dropout     dropout whose mask is computed again wherever it is needed (`fg_dropout`; on a gradient it is its own backward pass)

Widths and row counts are those of the repository's workloads (`fg_inputs.workload`) and of its ragged cases: listed
rows (the computed ones, `listed_share` of the positions) of a layer, in ascending order.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1}
_E4M3_MAX, _AMAX_MIN, _EPS = 448.0, 2.0 ** -100, 1e-6


def listed():
    return [
        # one mini-batch of the smallest workload, four node types: launches and host time decide
        dict(name="grouped_few", op="grouped", dtype="f32", out="f32", n=256, listed_share=1.0, groups=4, d_in=64, d_out=64, table=0),
        # a hidden layer over a products-like graph: 100 features are no multiple of a tile, the types are uneven
        dict(name="grouped_f32", op="grouped", dtype="f32", out="f32", n=67_584, listed_share=0.8, groups=5, d_in=100, d_out=256, table=0),
        # the typed projection of a heterogeneous graph's raw fp16 features, read from the table by node id
        dict(name="grouped_table_f16", op="grouped", dtype="f16", out="f16", n=409_600, listed_share=0.9, groups=3, d_in=768, d_out=1024,
             table=1_000_000),
        # a wide hidden layer served in 8 bits: rows quantised, then multiplied with weights that were quantised once
        dict(name="grouped_e4m3", op="grouped", dtype="e4m3", out="bf16", n=65_536, listed_share=0.9, groups=16, d_in=1024, d_out=1024, table=0),
        # training: fp32 at widths that are no multiple of a tile, and the wide mixed-precision layer
        dict(name="grouped_bw_f32", op="grouped_bw", dtype="f32", out="f32", n=51_003, listed_share=0.85, groups=7, d_in=88, d_out=256, relu=True),
        dict(name="grouped_bw_bf16", op="grouped_bw", dtype="bf16", out="bf16", n=65_536, listed_share=0.9, groups=8, d_in=1024, d_out=1024, relu=True),
        # between two layers of a papers-like model, training: dropout on the branch
        dict(name="norm_f32", op="norm", dtype="f32", out="f32", n=61_440, listed_share=0.8, d=256, p=0.5, residual=True),
        # between two wide layers, serving: no dropout, 8 bits for the product that follows
        dict(name="norm_e4m3", op="norm", dtype="bf16", out="e4m3", n=65_536, listed_share=1.0, d=1024, p=0.0, residual=True),
        # gradients of a user's own small model, and of the wide one
        dict(name="norm_bw_ragged", op="norm_bw", dtype="f32", n=7_771, listed_share=0.9, d=88, p=0.1, residual=True),
        dict(name="norm_bw_bf16", op="norm_bw", dtype="bf16", n=65_536, listed_share=1.0, d=1024, p=0.5, residual=True),
        # the seeds' embeddings of a small model, and the input features of the wide one
        dict(name="dropout_few", op="dropout", dtype="f32", n=777, listed_share=1.0, d=89, p=0.5),
        dict(name="dropout_bf16", op="dropout", dtype="bf16", n=409_600, listed_share=0.9, d=768, p=0.2),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["grouped", "grouped", "grouped", "grouped_bw", "grouped_bw", "norm", "norm_bw", "dropout"])
    n, share = log_int(1, 200_000), round(rng.uniform(0.5, 1.0), 3)
    if op in ("grouped", "grouped_bw"):
        dtype = rng.choice(["f32", "f16", "bf16", "e4m3"] if op == "grouped" else ["f32", "f16", "bf16"])
        step = {"f32": 4, "f16": 8, "bf16": 8, "e4m3": 16}[dtype]
        width = lambda: step * max(1, log_int(32, 1024) // step)
        case = dict(op=op, dtype=dtype, n=n, listed_share=share, groups=log_int(1, 64), d_in=width(), d_out=width())
        if op == "grouped":
            out = rng.choice({"f32": ["f32"], "f16": ["f16", "f32"], "bf16": ["bf16", "f32"], "e4m3": ["bf16", "f32"]}[dtype])
            return dict(case, out=out, table=rng.choice([0, 300_000]) if dtype in ("f32", "f16") else 0)
        return dict(case, n=min(n, 100_000), out=rng.choice(["f32", dtype]), relu=rng.random() < 0.7)
    dtype, d = rng.choice(["f32", "f16", "bf16"]), log_int(16, 4096)
    n = min(n, 200_000_000 // d)
    if op == "dropout":
        return dict(op=op, dtype=dtype, n=n, listed_share=share, d=d, p=rng.choice([0.1, 0.2, 0.5, 0.8]))
    case = dict(op=op, dtype=dtype, n=n, listed_share=share, d=d, p=rng.choice([0.0, 0.1, 0.5]), residual=rng.random() < 0.8)
    return dict(case, out=rng.choice([dtype, "e4m3"])) if op == "norm" else case


class _State:
    pass


def _count(case):
    return max(1, int(case["n"] * case["listed_share"]))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kw = dict(device="cuda", generator=gen)
    s = _State()
    s.case, s.n = case, case["n"]
    op, n, t = case["op"], case["n"], _TYPES[case["dtype"]]
    k = _count(case)
    s.rows = torch.randperm(n, **kw)[:k].sort().values.int() if k < n else None
    s.n_rows = torch.full((1,), k, dtype=torch.int64, device="cuda")
    s.k = k
    if op in ("grouped", "grouped_bw"):
        G, a, b = case["groups"], case["d_in"], case["d_out"]
        share = 1.0 / torch.arange(1, G + 1, device="cuda").float()      # a few frequent types, many rare ones
        table = case.get("table", 0)
        s.types = torch.multinomial(share, table or n, replacement=True, generator=gen).int()
        s.ids = torch.randint(0, table, (n,), **kw).int() if table else None
        rows = table or n
        w = (torch.rand(G, a, b, **kw) * 2 - 1) * math.sqrt(6.0 / (a + b))
        s.bias = torch.randn(G, b, **kw) * 0.1
        if case["dtype"] == "e4m3":
            s.x = torch.randn(rows, a, **kw).bfloat16()
            s.w, s.w_scale = _quantize(w.transpose(1, 2).contiguous().reshape(G * b, a))     # quantised once, a scale per output column
            s.w = s.w.reshape(G, b, a)
            s.q, s.x_scale = torch.zeros(rows, a, dtype=t, device="cuda"), torch.zeros(rows, device="cuda")
        else:
            s.x, s.w = torch.randn(rows, a, **kw).to(t), w.to(t)
        if op == "grouped":
            s.order, s.offsets = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(G + 1, dtype=torch.int64, device="cuda")
            s.h = torch.zeros(n, b, dtype=_TYPES[case["out"]], device="cuda")
        else:
            s.order, s.offsets = _group(s)
            s.h = torch.randn(n, b, **kw).clamp_min(0).to(t) if case["relu"] else None
            s.dh = torch.randn(n, b, **kw).to(t)
            s.dx = torch.zeros(n, a, dtype=_TYPES[case["out"]], device="cuda")
            s.dw, s.db = torch.zeros(G, a, b, device="cuda"), torch.zeros(G, b, device="cuda")
    else:
        d = case["d"]
        s.key, s.p = int(seed) * 0x9E3779B1 + 17, case["p"]
        spread = torch.exp(torch.randn(n, 1, **kw))      # rows of different magnitude
        if op != "norm_bw":
            s.x = (torch.randn(n, d, **kw) * spread).to(t)
        if op == "dropout":
            s.out = torch.zeros(n, d, dtype=t, device="cuda")
        else:
            s.w = 1 + 0.1 * torch.randn(d, **kw)
            s.residual = (torch.randn(n, d, **kw) * spread).to(t) if case["residual"] else None
            if op == "norm":
                s.sum = torch.zeros(n, d, dtype=t, device="cuda")
                s.y = torch.zeros(n, d, dtype=_TYPES[case["out"]], device="cuda")
                s.scale = torch.zeros(n, device="cuda") if case["out"] == "e4m3" else None
                s.rstd = torch.zeros(n, device="cuda")
            else:
                s.sum = (torch.randn(n, d, **kw) * spread).to(t)
                s.rstd = torch.rsqrt(s.sum.float().square().mean(1) + _EPS)
                s.dy = torch.randn(n, d, **kw).to(t)
                s.dsum_in = torch.randn(n, d, **kw).to(t) if case["residual"] else None
                s.dsum = torch.zeros(n, d, dtype=t, device="cuda")
                s.dx = torch.zeros(n, d, dtype=t, device="cuda") if s.p else None      # without dropout it is dsum
                s.dw = torch.zeros(d, device="cuda")
    s.ws = None      # the workspace: laid out by the first call, kept as a program keeps it
    return s


def run(state):
    return (_own if own else _plain)[state.case["op"]](state)


# ---- plain forms ----

def _quantize(x):
    """Rows in 8 bits with a scale each."""
    x = x.float()
    amax = x.abs().amax(1).clamp_min(_AMAX_MIN)
    return (x * (_E4M3_MAX / amax)[:, None]).clamp(-_E4M3_MAX, _E4M3_MAX).to(torch.float8_e4m3fn), amax / _E4M3_MAX


def _listed_rows(s):
    return s.rows if s.rows is not None else torch.arange(s.n, device="cuda", dtype=torch.int32)


def _group(s):
    rows = _listed_rows(s)
    types = s.types[rows if s.ids is None else s.ids[rows]]
    order = torch.zeros(s.n, dtype=torch.int32, device="cuda")
    order[:len(rows)] = rows[torch.sort(types, stable=True).indices]
    edges = torch.arange(s.case["groups"] + 1, device="cuda", dtype=torch.int32)
    return order, (types[:, None] < edges[None, :]).sum(0)


def _plain_grouped(s):
    order, offsets = _group(s)
    x, w, bias = s.x, s.w.float(), s.bias
    if s.case["dtype"] == "e4m3":
        q, scale = _quantize(s.x)
        x, w = q.float() * scale[:, None], (w * s.w_scale.view(w.shape[0], -1, 1)).transpose(1, 2)
    h = torch.zeros_like(s.h)
    at = offsets.tolist()
    for g in range(s.case["groups"]):      # a product for each type, as many rows as it has
        pos = order[at[g]:at[g + 1]]
        rows = pos if s.ids is None else s.ids[pos]
        h[pos] = (x[rows].float() @ w[g] + bias[g]).clamp_min(0).to(h.dtype)
    return dict(h=h, order=order, offsets=offsets)


def _plain_grouped_bw(s):
    dz = s.dh.float()
    if s.h is not None:
        dz = torch.where(s.h > 0, dz, torch.zeros_like(dz))
    w = s.w.float()
    dx, dw, db = torch.zeros_like(s.dx), torch.zeros_like(s.dw), torch.zeros_like(s.db)
    at = s.offsets.tolist()
    for g in range(s.case["groups"]):
        pos = s.order[at[g]:at[g + 1]]
        z = dz[pos]
        dx[pos] = (z @ w[g].T).to(dx.dtype)
        dw[g] = s.x[pos].float().T @ z
        db[g] = z.double().sum(0)
    return dict(dx=dx, dw=dw, db=db)


def _mix(z):
    """The output function of the SplitMix64 generator on 64-bit integers (Steele, Lea, Flood 2014)."""
    shr = lambda v, k: (v >> k) & ((1 << (64 - k)) - 1)
    z = (z ^ shr(z, 30)) * (0xBF58476D1CE4E5B9 - (1 << 64))
    z = (z ^ shr(z, 27)) * (0x94D049BB133111EB - (1 << 64))
    return z ^ shr(z, 31)


def _kept(key, rows, d, p):
    """[rows, d] truth values: which elements dropout leaves, by position and column."""
    golden = 0x9E3779B97F4A7C15 - (1 << 64)
    signed = (int(key) + (1 << 63)) % (1 << 64) - (1 << 63)
    base = _mix(torch.tensor([signed], dtype=torch.int64, device=rows.device))
    row = _mix(base + (rows.long() + 1) * golden)
    blocks = torch.arange((d + 3) // 4, device=rows.device, dtype=torch.int64)
    bits = _mix(row[:, None] + (blocks + 1) * golden)
    draws = torch.stack([(bits >> (16 * i)) & 0xFFFF for i in range(4)], -1).reshape(len(rows), -1)[:, :d]
    return draws >= math.floor(p * 65536 + 0.5)


def _drop(s, rows, x):
    """Dropout of the listed rows' values (fp32 or fp64), kept ones scaled to keep the mean."""
    if s.p == 0:
        return x
    scale = 65536 / (65536 - math.floor(s.p * 65536 + 0.5))
    return torch.where(_kept(s.key, rows, x.shape[1], s.p), x * scale, torch.zeros_like(x))


def _placed(like, rows, v):
    out = torch.zeros_like(like)
    out[rows] = v.to(like.dtype)
    return out


def _plain_norm(s):
    rows = _listed_rows(s)
    v = _drop(s, rows, s.x[rows].float())
    if s.residual is not None:
        v = v + s.residual[rows].float()
    rstd = torch.rsqrt(v.square().mean(1) + _EPS)
    y = v * rstd[:, None] * s.w
    out = dict(sum=_placed(s.sum, rows, v), rstd=_placed(s.rstd, rows, rstd))
    if s.scale is None:
        return dict(out, y=_placed(s.y, rows, y))
    q, scale = _quantize(y)
    full = torch.zeros_like(s.y)
    full.view(torch.uint8)[rows] = q.view(torch.uint8)
    return dict(out, y=full, scale=_placed(s.scale, rows, scale))


def _plain_norm_bw(s):
    rows = _listed_rows(s)
    dy, rstd = s.dy[rows].float(), s.rstd[rows][:, None]
    xh, t = s.sum[rows].float() * rstd, dy * s.w
    ds = rstd * (t - xh * (t * xh).mean(1, keepdim=True))
    if s.dsum_in is not None:
        ds = ds + s.dsum_in[rows].float()
    out = dict(dsum=_placed(s.dsum, rows, ds), dw=(dy.double() * xh).sum(0).float())
    return dict(out, dx=_placed(s.dx, rows, _drop(s, rows, ds))) if s.p else out


def _plain_dropout(s):
    rows = _listed_rows(s)
    return _placed(s.out, rows, _drop(s, rows, s.x[rows].float()))


_plain = dict(grouped=_plain_grouped, grouped_bw=_plain_grouped_bw, norm=_plain_norm, norm_bw=_plain_norm_bw, dropout=_plain_dropout)


# ---- the framework's calls ----

def _lib():
    from paper_2301_07482_amd import binding
    return binding, {"f32": binding.FG_F32, "f16": binding.FG_F16, "bf16": binding.FG_BF16, "e4m3": binding.FG_E4M3}


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _workspace(s, size):
    if s.ws is None:
        s.ws = torch.zeros(max(size, 16), dtype=torch.uint8, device="cuda")
    return s.ws, s.ws.numel()


def _own_grouped(s):
    B, T = _lib()
    c, st = s.case, _stream()
    a, b, G = c["d_in"], c["d_out"], c["groups"]
    ws, ws_bytes = _workspace(s, B.fg_group_rows_workspace_bytes(s.k, G)) if s.ws is None else (s.ws, s.ws.numel())
    B.fg_group_rows(s.types, len(s.types), s.ids, s.n, s.rows, s.n_rows, s.k, G, s.order, s.offsets, ws, ws_bytes, st)
    x, e = s.x, _SIZE[c["dtype"]]
    if c["dtype"] == "e4m3":
        B.fg_quantize_rows(s.x, 2 * a, B.FG_BF16, len(s.x), a, s.q, a, s.x_scale, st)
        x = s.q
    quantised = c["dtype"] == "e4m3"
    B.fg_linear_grouped(x, len(x), a * e, T[c["dtype"]], s.x_scale if quantised else None, s.ids, s.order, s.offsets, s.k, G, a, b, s.w,
                        s.w_scale if quantised else None, s.bias, 1, s.h, s.n, b * _SIZE[c["out"]], T[c["out"]], st)
    return dict(h=s.h, order=s.order, offsets=s.offsets)


def _own_grouped_bw(s):
    B, T = _lib()
    c, st = s.case, _stream()
    a, b, G, e, t = c["d_in"], c["d_out"], c["groups"], _SIZE[c["dtype"]], T[c["dtype"]]
    ws, ws_bytes = _workspace(s, B.fg_linear_grouped_backward_workspace_bytes(t, s.k, G, a, b)) if s.ws is None else (s.ws, s.ws.numel())
    B.fg_linear_grouped_backward(s.x, len(s.x), a * e, t, None, s.dh, b * e, t, s.h, b * e if s.h is not None else 0, s.n, s.order, s.offsets, s.k,
                                 G, a, b, s.w, s.dx, a * _SIZE[c["out"]], T[c["out"]], s.dw, s.db, ws, ws_bytes, st)
    return dict(dx=s.dx, dw=s.dw, db=s.db)


def _own_norm(s):
    B, T = _lib()
    c = s.case
    d, e = c["d"], _SIZE[c["dtype"]]
    t = T[c["dtype"]]
    B.fg_residual_norm(s.x, d * e, t, s.residual, d * e if s.residual is not None else 0, t, s.rows, s.n_rows, s.k, s.n, d, s.p, s.key,
                       s.w, _EPS, s.sum, d * e, s.y, d * _SIZE[c["out"]], T[c["out"]], s.scale, s.rstd, _stream())
    out = dict(sum=s.sum, rstd=s.rstd, y=s.y)
    return dict(out, scale=s.scale) if s.scale is not None else out


def _own_norm_bw(s):
    B, T = _lib()
    c = s.case
    d, e = c["d"], _SIZE[c["dtype"]]
    ws, ws_bytes = _workspace(s, B.fg_residual_norm_backward_workspace_bytes(s.k, d)) if s.ws is None else (s.ws, s.ws.numel())
    t = T[c["dtype"]]
    B.fg_residual_norm_backward(s.dy, d * e, t, s.sum, d * e, t, s.rstd, s.w, s.dsum_in, d * e if s.dsum_in is not None else 0, s.rows, s.n_rows,
                                s.k, s.n, d, s.p, s.key, s.dsum, d * e, s.dx, d * e if s.p else 0, s.dw, ws, ws_bytes, _stream())
    return dict(dsum=s.dsum, dx=s.dx, dw=s.dw) if s.p else dict(dsum=s.dsum, dw=s.dw)


def _own_dropout(s):
    B, T = _lib()
    c = s.case
    stride = c["d"] * _SIZE[c["dtype"]]
    B.fg_dropout(s.x, stride, T[c["dtype"]], s.rows, s.n_rows, s.k, s.n, c["d"], s.p, s.key, s.out, stride, _stream())
    return s.out


_own = dict(grouped=_own_grouped, grouped_bw=_own_grouped_bw, norm=_own_norm, norm_bw=_own_norm_bw, dropout=_own_dropout)


# ---- what a pass cannot do without ----

def work(case):
    k, op, e = _count(case), case["op"], _SIZE[case["dtype"]]
    lists = 4 * k if k < case["n"] else 0
    if op in ("grouped", "grouped_bw"):
        a, b, G = case["d_in"], case["d_out"], case["groups"]
        if op == "grouped":
            read = k * a * (2 if case["dtype"] == "e4m3" else e) + G * a * b * e + 4 * G * b + lists + (8 * k if case["table"] else 4 * k)
            return dict(bytes=read + k * b * _SIZE[case["out"]] + 4 * k + 8 * (G + 1), flops=2 * k * a * b)
        read = k * a * e + k * b * e * (2 if case["relu"] else 1) + G * a * b * e + 4 * k + 8 * (G + 1)
        return dict(bytes=read + k * a * _SIZE[case["out"]] + 4 * G * (a * b + b), flops=4 * k * a * b)
    d = case["d"]
    if op == "dropout":
        return dict(bytes=2 * k * d * e + lists, flops=k * d)
    extra = 1 if case["residual"] else 0
    if op == "norm":
        return dict(bytes=k * d * (e * (2 + extra) + _SIZE[case["out"]]) + 4 * d + lists + 4 * k + (4 * k if case["out"] == "e4m3" else 0), flops=6 * k * d)
    return dict(bytes=k * d * e * (3 + extra + (1 if case["p"] else 0)) + 8 * d + lists + 4 * k, flops=12 * k * d)


# ---- the definitions in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    rows = torch.arange(s.n, device="cuda") if s.rows is None else s.rows.long()
    if op in ("grouped", "grouped_bw"):
        types = s.types.long()[rows if s.ids is None else s.ids.long()[rows]]
        members = [rows[types == g] for g in range(case["groups"])]
        if op == "grouped":
            h = torch.zeros(s.n, case["d_out"], dtype=torch.float64, device="cuda")
            for g, pos in enumerate(members):
                src = pos if s.ids is None else s.ids.long()[pos]
                x, w = s.x[src].double(), s.w[g].double()
                if case["dtype"] == "e4m3":
                    amax = x.abs().amax(1, keepdim=True).clamp_min(_AMAX_MIN).float()
                    x = (x.float() * (_E4M3_MAX / amax)).to(torch.float8_e4m3fn).double() * (amax / _E4M3_MAX).double()
                    w = (w * s.w_scale.view(case["groups"], -1)[g].double()[:, None]).T
                h[pos] = torch.relu(torch.mm(x, w) + s.bias[g].double())
            return dict(h=h, order=None, offsets=None)
        dx = torch.zeros(s.n, case["d_in"], dtype=torch.float64, device="cuda")
        dw, db = torch.zeros_like(s.dw, dtype=torch.float64), torch.zeros_like(s.db, dtype=torch.float64)
        for g, pos in enumerate(members):
            dz = s.dh[pos].double()
            if s.h is not None:
                dz = dz * (s.h[pos] > 0)
            dx[pos] = torch.mm(dz, s.w[g].double().T.contiguous())
            dw[g], db[g] = torch.mm(s.x[pos].double().T.contiguous(), dz), dz.sum(0)
        return dict(dx=dx, dw=dw, db=db)
    keep, factor = None, 1.0
    if s.p:
        threshold = round(s.p * 65536)
        keep, factor = _keep_exact(s, rows, threshold), 65536 / (65536 - threshold)
    dropped = lambda v: v if keep is None else torch.where(keep, v * factor, 0.0)
    place = lambda v: torch.zeros(s.n, *v.shape[1:], dtype=torch.float64, device="cuda").index_copy_(0, rows, v)
    if op == "dropout":
        return place(dropped(s.x[rows].double()))
    w = s.w.double()
    if op == "norm":
        v = dropped(s.x[rows].double())
        if s.residual is not None:
            v = v + s.residual[rows].double()
        rstd = (v.square().mean(1) + _EPS).rsqrt()
        y = v * rstd[:, None] * w
        if s.scale is None:
            return dict(sum=place(v), rstd=place(rstd), y=place(y))
        scale = y.abs().amax(1).clamp_min(_AMAX_MIN) / _E4M3_MAX
        return dict(sum=place(v), rstd=place(rstd), y=place(y / scale[:, None]), scale=place(scale))
    dy, rstd = s.dy[rows].double(), s.rstd[rows].double()[:, None]
    xh = s.sum[rows].double() * rstd
    t = dy * w
    ds = rstd * (t - xh * (t * xh).mean(1, keepdim=True))
    if s.dsum_in is not None:
        ds = ds + s.dsum_in[rows].double()
    out = dict(dsum=place(ds), dw=(dy * xh).sum(0))
    return dict(out, dx=place(dropped(ds))) if s.p else out


def _keep_exact(s, rows, threshold):
    """The draws of the generator's definition, two 32-bit halves at a time (no product leaves 64 bits)."""
    low = 0xFFFFFFFF

    def times(h, l, c):
        p = l * (c & low)      # the bits beyond 64 of this product's sign are masked below
        ph = (p >> 32) & low
        return ((h * (c & low)) + (l * (c >> 32)) + ph) & low, p & low

    def plus(h, l, ch, cl):
        t = l + cl
        return (h + ch + (t >> 32)) & low, t & low

    def mix(h, l):
        for shift, c in ((30, 0xBF58476D1CE4E5B9), (27, 0x94D049BB133111EB)):
            l, h = l ^ ((l >> shift) | ((h << (32 - shift)) & low)), h ^ (h >> shift)
            h, l = times(h, l, c)
        return h ^ (h >> 31), l ^ ((l >> 31) | ((h << 1) & low))

    def step(h, l, count):
        return mix(*plus(h, l, *times(torch.zeros_like(count), count, 0x9E3779B97F4A7C15)))

    key = int(s.key) % (1 << 64)
    one = lambda v: torch.full((1, 1), v, dtype=torch.int64, device="cuda")
    h, l = step(*mix(one(key >> 32), one(key & low)), rows[:, None].long() + 1)
    d = s.case["d"]
    h, l = step(h, l, torch.arange(1, (d + 3) // 4 + 1, device="cuda")[None, :])
    draws = torch.stack([l & 0xFFFF, l >> 16, h & 0xFFFF, h >> 16], -1).reshape(len(rows), -1)[:, :d]
    return draws >= threshold
