"""The operators that training a DSVT layer needs between its matrix products, with their plain forms: what is measured of them.

`listed()` gives the fixed cases, `draw(rng)` one more of the same ranges, `prepare(case, seed)` what a program holds before the
call, `run(state)` one pass (through the library where `own` is true, in elementary torch operations where it is not),
`exact(case, seed)` the same results in 64 bits and `work(case)` the bytes and operations the pass cannot do without.

Operators of a case ("op"), each with "back" for its backward pass:
  attention  dsvt_segment_attention: multi-head attention inside the segments of a partition, whole windows or the sets cut
             from them, with a learned relative position bias by buckets and a tanh cap on the logits.
  norm       dsvt_layer_norm: LayerNorm of a residual sum.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _attention(n, shape, **kw):
    c = dict(op="attention", back=False, n=n, shape=shape, grid=468, depth=1, window=12, set_size=36, heads=8, dim=24,
             type="bf16", bias=True, cap=0.0)
    c.update(kw)
    return c


def _norm(n, C, **kw):
    c = dict(op="norm", back=False, n=n, C=C, type="bf16", residual=True)
    c.update(kw)
    return c


def listed():
    return [
        # the smallest call: a few thousand pillars in sets of 36, 128 channels in fp32; latency counts
        dict(_attention(2000, "uniform", grid=64, dim=16, type="fp32"), name="sets_tiny_fp32"),
        # the ordinary one: a pillar frame of 150 m x 150 m, 192 channels
        dict(_attention(32000, "pillar"), name="sets_frame_bf16"),
        # windows of 30 x 30 in sets of 90, in fp16 with capped logits
        dict(_attention(30011, "pillar", grid=360, window=30, set_size=90, dim=16, type="fp16", cap=20.0), name="sets_wide_fp16_capped"),
        # the voxel variant without the cut into sets: windows of one to more than a thousand voxels
        dict(_attention(120000, "voxel", depth=32, set_size=0), name="windows_voxel_bf16"),
        # the backward passes of the same kinds: a sparse crop, the pillar frame, fp32 training, whole windows
        dict(_attention(2531, "pillar", back=True), name="sets_small_back_bf16"),
        dict(_attention(32000, "pillar", back=True), name="sets_frame_back_bf16"),
        dict(_attention(12345, "pillar", back=True, type="fp32", cap=30.0), name="sets_back_fp32_capped"),
        dict(_attention(60000, "voxel", depth=32, set_size=0, back=True), name="windows_voxel_back_bf16"),
        # LayerNorm behind a layer's residual sum: the smallest frame, and two stages' worth of a batch of frames
        dict(_norm(2000, 128, type="fp32"), name="norm_tiny_fp32"),
        dict(_norm(200000, 192), name="norm_batch_bf16"),
        dict(_norm(12345, 192, back=True, type="fp32"), name="norm_back_fp32"),
        dict(_norm(200000, 192, back=True), name="norm_batch_back_bf16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    back = rng.random() < 0.5
    typ = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    family = rng.choice(["sets", "sets", "wide", "windows", "norm", "norm"])
    if family == "norm":
        C = rng.choice([64, 96, 128, 192, 256, 384, 8 * rng.randint(4, 64), rng.randint(30, 500)])
        return _norm(_log_uniform(rng, 500, 38400000 // C // (2 if typ == "fp32" else 1)), C, back=back, type=typ, residual=rng.random() < 0.7)
    kw = dict(back=back, type=typ, bias=rng.random() < 0.8, cap=rng.choice([0.0, 0.0, 15.0, 30.0]))
    heads, dim = rng.choice([(8, 24), (8, 24), (8, 16), (4, 32), (4, 64), (6, 32), (12, 16), (3, 40)])
    kw.update(heads=heads, dim=dim)
    if family == "wide":
        return _attention(_log_uniform(rng, 2000, 36000), "pillar", grid=360, window=30, set_size=rng.choice([90, 72, 128]), **kw)
    if family == "windows":
        if rng.random() < 0.5:
            return _attention(_log_uniform(rng, 2000, 36000), "pillar", set_size=0, **kw)
        return _attention(_log_uniform(rng, 8000, 30000 if back else 60000), "voxel", depth=32, set_size=0, **kw)
    if rng.random() < 0.3:
        return _attention(_log_uniform(rng, 8000, 60000), "voxel", depth=32, set_size=rng.choice([36, 48]), **kw)
    return _attention(_log_uniform(rng, 1500, 36000), "pillar", set_size=rng.choice([36, 24, 48, rng.randint(8, 60)]), **kw)


# ---- inputs --------------------------------------------------------------------------------------------------------
def _cells(case, rng):
    """int64 [n][3]: distinct cells (x, y, z) of a frame, in arbitrary order."""
    n, grid, depth = case["n"], case["grid"], case["depth"]
    if case["shape"] == "uniform":
        flat = rng.permutation(grid * grid * depth)[:n]
        return np.stack([flat // depth // grid, flat // depth % grid, flat % depth], axis=1)
    half, keys = 0.5 * grid, np.zeros(0, dtype=np.int64)
    while len(keys) < n:  # rings around the sensor and clutter whose density falls with the distance's square
        ring = rng.random(2 * n) < 0.5
        reach = 1.42 * half
        r = np.where(ring, 0.04 * half * 25.0 ** (rng.integers(0, 64, 2 * n) / 63.0) + 0.3 * rng.standard_normal(2 * n),
                     np.exp(rng.uniform(math.log(0.027 * half), math.log(reach), 2 * n)))
        az = rng.uniform(0.0, 2.0 * math.pi, 2 * n)
        x, y = np.floor(half + r * np.cos(az)).astype(np.int64), np.floor(half + r * np.sin(az)).astype(np.int64)
        z = np.where(ring, rng.integers(0, 2, 2 * n), np.minimum(rng.geometric(0.3, 2 * n) - 1, 7)) if depth > 1 else np.zeros(2 * n, dtype=np.int64)
        ok = (x >= 0) & (x < grid) & (y >= 0) & (y < grid)
        keys = np.concatenate([keys, ((x * grid + y) * depth + z)[ok]])
        _, first = np.unique(keys, return_index=True)
        keys = keys[np.sort(first)]
    keys = keys[:n]
    return np.stack([keys // depth // grid, keys // depth % grid, keys % depth], axis=1)


def _segments(case, cells):
    """The voxels in the order of their windows (x, y, z inside), and where each segment starts: windows, or their sets."""
    w, side = case["window"], -(-case["grid"] // case["window"])
    win = cells[:, 0] // w * side + cells[:, 1] // w
    order = np.lexsort((cells[:, 2], cells[:, 1], cells[:, 0], win))
    count = np.bincount(win, minlength=side * side)
    start = np.concatenate([[0], np.cumsum(count)])
    if case["set_size"] == 0:
        return order, start, int(count.max())
    sets = -(-count // case["set_size"])
    which = np.repeat(np.arange(len(count)), sets)
    j = np.arange(len(which)) - np.repeat(np.cumsum(sets) - sets, sets)
    return order, np.concatenate([start[which] + j * count[which] // sets[which], [case["n"]]]), case["set_size"]


def _axis_buckets(extent, near, side):
    """Bucket of a displacement -(extent - 1) ... extent - 1 along one axis: exact below `near`, then by logarithm, `side` buckets
    for each sign (0 shared)."""
    d = np.arange(-(extent - 1), extent)
    a = np.abs(d)
    far = near + np.floor(np.log(np.maximum(a, near) / near) / math.log(max(extent, near + 1) / near) * (side - near) + 1e-9)
    m = np.minimum(np.where(a < near, a, far), side - 1).astype(np.int64)
    return side - 1 + np.sign(d) * m


def _buckets(case):
    """The extent, the additive index of each axis and the number of buckets of the case's bias."""
    w, depth = case["window"], case["depth"]
    sides = (6, 6, 1) if depth == 1 and w <= 12 else (7, 7, 1) if depth == 1 else (5, 5, 4)
    by = [_axis_buckets(e, min(3, s), s) for e, s in zip((w, w, depth), sides)]
    widths = [2 * s - 1 for s in sides]
    return (w, w, depth), [by[0] * widths[1] * widths[2], by[1] * widths[2], by[2]], widths[0] * widths[1] * widths[2]


def _randn(g, *shape, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda") * scale


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    t, n = _TYPES[case["type"]], case["n"]
    st = {"case": case}
    if case["op"] == "norm":
        C = case["C"]
        st["x"] = (_randn(g, n, C) + 0.2 * _randn(g, C)).to(t)  # a post-norm stream: unit variance, some offset per channel
        st["r"] = _randn(g, n, C, scale=0.5).to(t) if case["residual"] else None
        st["g"], st["b"] = 1.0 + 0.1 * _randn(g, C), 0.1 * _randn(g, C)
        st["dy"] = _randn(g, n, C, scale=0.3).to(t) if case["back"] else None
        if own:
            from paper_2301_06051_b200 import api
            st["ctx"] = api.Context(n, 1, C)
        return st
    heads, dim = case["heads"], case["dim"]
    rng = np.random.default_rng(seed)
    cells = _cells(case, rng)
    order, start, longest = _segments(case, cells)
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()
    st["coords"] = put(np.concatenate([np.zeros((n, 1), dtype=np.int64), cells], axis=1))
    st["order"], st["start"], st["longest"] = put(order), put(start), longest
    st["qkv"] = _randn(g, n, 3, heads, dim).to(t)  # one projection's output: queries, keys and values side by side
    st["scale"] = dim ** -0.5
    st["extent"], by, st["buckets"] = _buckets(case)
    st["index"] = np.concatenate(by).astype(np.int32)
    st["bias"] = _randn(g, heads, st["buckets"], scale=0.5) if case["bias"] else None
    st["do"] = _randn(g, n, heads, dim, scale=0.5).to(t) if case["back"] else None
    st["groups"] = _groups(start, heads)
    if own:
        from paper_2301_06051_b200 import api
        ctx = st["ctx"] = api.Context(n, len(start), heads * dim)
        st["seg"] = api.Segments(st["start"], longest, order=st["order"], coords=st["coords"])
        st["rel"] = api.BucketBias(st["bias"], st["extent"], st["index"]) if case["bias"] else None
        st["out"] = torch.empty((n, heads, dim), dtype=t, device=ctx.device)
        st["grad"] = torch.empty((n, 3, heads, dim), dtype=t, device=ctx.device) if case["back"] else None
    return st


def _groups(start, heads):
    """Segments of similar length together: (padded length, their numbers), cut so that a group's scores fit in memory."""
    length = np.diff(start)
    wide = np.where(length <= 64, -(-length // 8) * 8, -(-length // 64) * 64).astype(np.int64)
    out = []
    for L in np.unique(wide[length > 0]):
        ids = np.nonzero((wide == L) & (length > 0))[0]
        step = max(1, (1 << 27) // int(L * L * heads))
        out += [(int(L), torch.from_numpy(ids[i:i + step]).cuda()) for i in range(0, len(ids), step)]
    return out


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(st):
    case = st["case"]
    if own:
        return _library(st)
    if case["op"] == "norm":
        return _plain_norm(st)
    return _plain_attention(st)


def _library(st):
    case, ctx = st["case"], st["ctx"]
    if case["op"] == "norm":
        if case["back"]:
            return ctx.layer_norm_backward(st["x"], st["dy"], st["g"], residual=st["r"])
        return ctx.layer_norm(st["x"], st["g"], st["b"], residual=st["r"])
    q, k, v = st["qkv"].unbind(1)
    if not case["back"]:
        return ctx.segment_attention(q, k, v, st["seg"], bias=st["rel"], cap=case["cap"], out=st["out"])
    dq, dk, dv, dbias = ctx.segment_attention_backward(q, k, v, st["do"], st["seg"], bias=st["rel"], cap=case["cap"],
                                                       out=tuple(st["grad"].unbind(1)))
    return [dq, dk, dv] + ([dbias] if case["bias"] else [])


def _plain_norm(st):
    u = st["x"].float() + (st["r"].float() if st["r"] is not None else 0.0)
    c = u - u.mean(dim=1, keepdim=True)
    rstd = 1.0 / torch.sqrt((c * c).mean(dim=1, keepdim=True) + 1e-5)
    h = c * rstd
    if not st["case"]["back"]:
        return (h * st["g"] + st["b"]).to(st["x"].dtype)
    dy = st["dy"].float()
    w = dy * st["g"]
    dx = rstd * (w - w.mean(dim=1, keepdim=True) - h * (w * h).mean(dim=1, keepdim=True))
    return [dx.to(st["x"].dtype), (dy * h).sum(dim=0), dy.sum(dim=0)]


def _plain_attention(st):
    case, order, start = st["case"], st["order"].long(), st["start"].long()
    n, heads, dim = case["n"], case["heads"], case["dim"]
    L, W, H = st["extent"]
    index = torch.from_numpy(st["index"]).cuda().long()
    ix, iy, iz = index[:2 * L - 1], index[2 * L - 1:2 * (L + W) - 2], index[2 * (L + W) - 2:]
    out = torch.zeros((n, heads, dim), device="cuda")
    grad = torch.zeros((3, n, heads, dim), device="cuda") if case["back"] else None
    dbias = torch.zeros((heads, st["buckets"]), dtype=torch.float64, device="cuda")
    for length, ids in st["groups"]:
        at = start[ids, None] + torch.arange(length, device="cuda")
        ok = at < start[ids + 1, None]
        rows = order[at.clamp(max=n - 1)]
        q, k, v = (st["qkv"][rows, i].float().transpose(1, 2) for i in range(3))  # [segments, heads, length, dim]
        z = torch.matmul(q, k.transpose(2, 3)) * st["scale"]
        t = torch.tanh(z / case["cap"]) if case["cap"] > 0 else None
        s = case["cap"] * t if case["cap"] > 0 else z
        if case["bias"]:
            c = st["coords"][rows].long()
            d = c[:, :, None, 1:] - c[:, None, :, 1:]
            b = ix[d[..., 0].clamp(1 - L, L - 1) + L - 1] + iy[d[..., 1].clamp(1 - W, W - 1) + W - 1] + iz[d[..., 2].clamp(1 - H, H - 1) + H - 1]
            s = s + st["bias"][:, b].transpose(0, 1)
        s = s.masked_fill(~ok[:, None, None, :], -math.inf)
        p = torch.exp(s - s.amax(dim=3, keepdim=True))
        p = p / p.sum(dim=3, keepdim=True)
        if not case["back"]:
            out[rows[ok]] = torch.matmul(p, v).transpose(1, 2)[ok]
            continue
        do = (st["do"][rows].float() * ok[:, :, None, None]).transpose(1, 2)
        dp = torch.matmul(do, v.transpose(2, 3))
        ds = p * (dp - (p * dp).sum(dim=3, keepdim=True))
        if case["bias"]:
            spread = torch.zeros((heads, len(ids) * st["buckets"]), dtype=torch.float64, device="cuda")
            where = b + torch.arange(len(ids), device="cuda")[:, None, None] * st["buckets"]
            spread.index_add_(1, where.reshape(-1), ds.transpose(0, 1).reshape(heads, -1).double())
            dbias += spread.reshape(heads, len(ids), -1).sum(dim=1)
        dz = ds * (1.0 - t * t) if case["cap"] > 0 else ds
        dq, dk = torch.matmul(dz, k) * st["scale"], torch.matmul(dz.transpose(2, 3), q) * st["scale"]
        dv = torch.matmul(p.transpose(2, 3), do)
        at = rows[ok]
        grad[0, at], grad[1, at], grad[2, at] = dq.transpose(1, 2)[ok], dk.transpose(1, 2)[ok], dv.transpose(1, 2)[ok]
    if not case["back"]:
        return out.to(_TYPES[case["type"]])
    return [x.to(_TYPES[case["type"]]) for x in grad] + ([dbias.float()] if case["bias"] else [])


# ---- the same in 64 bits, segment after segment, gradients by differentiation of the definition -----------------------
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "norm":
        x = st["x"].double().requires_grad_()
        g, b = st["g"].double().requires_grad_(), st["b"].double().requires_grad_()
        u = x if st["r"] is None else x + st["r"].double()
        mean = u.sum(1, keepdim=True) / case["C"]
        var = ((u - mean) ** 2).sum(1, keepdim=True) / case["C"]
        y = (u - mean) / (var + 1e-5).sqrt() * g + b
        return y.detach() if not case["back"] else list(torch.autograd.grad(y, (x, g, b), st["dy"].double()))
    qkv = st["qkv"].double().requires_grad_(case["back"])
    bias = st["bias"].double().requires_grad_(case["back"]) if case["bias"] else None
    order, start = st["order"].cpu().numpy(), st["start"].cpu().numpy()
    cells = st["coords"].cpu().numpy()[:, 1:]
    splits = np.split(st["index"], np.cumsum([2 * e - 1 for e in st["extent"]])[:-1])
    out = torch.zeros((case["n"], case["heads"], case["dim"]), dtype=torch.float64, device="cuda")
    grad = [torch.zeros_like(qkv), torch.zeros_like(bias) if case["bias"] else None]
    for s in np.nonzero(np.diff(start))[0]:
        ids = order[start[s]:start[s + 1]]
        rows = torch.from_numpy(ids).cuda().long()
        part = qkv.detach()[rows].requires_grad_(case["back"])
        z = torch.einsum("ihd,jhd->hij", part[:, 0], part[:, 1]) / math.sqrt(case["dim"])
        if case["cap"] > 0:
            z = torch.tanh(z / case["cap"]) * case["cap"]
        if case["bias"]:
            far = [cells[ids, a][:, None] - cells[ids, a][None, :] for a in range(3)]
            which = sum(splits[a][np.clip(far[a], 1 - e, e - 1) + e - 1] for a, e in enumerate(st["extent"]))
            z = z + bias[:, torch.from_numpy(which).cuda().long()]
        o = torch.einsum("hij,jhd->ihd", torch.softmax(z, dim=2), part[:, 2])
        if not case["back"]:
            out[rows] = o
            continue
        got = torch.autograd.grad(o, (part, bias) if case["bias"] else (part,), st["do"][rows].double())
        grad[0][rows] = got[0]
        if case["bias"]:
            grad[1] += got[1]
    if not case["back"]:
        return out
    return list(grad[0].unbind(1)) + ([grad[1]] if case["bias"] else [])


def work(case):
    e = 4 if case["type"] == "fp32" else 2
    if case["op"] == "norm":
        passes = 2 + (1 if case["residual"] else 0) + (1 if case["back"] else 0)
        return {"bytes": case["n"] * case["C"] * e * passes + 8.0 * case["C"] * (2 if case["back"] else 1), "flops": (16.0 if case["back"] else 8.0) * case["n"] * case["C"]}
    _, start, _ = _segments(case, _cells(case, np.random.default_rng(0)))
    pairs = float((np.diff(start).astype(np.float64) ** 2).sum())
    width = case["heads"] * case["dim"]
    rows = case["n"] * (width * e * (7 if case["back"] else 4) + 4.0 + (16.0 if case["bias"] else 0.0)) + 4.0 * len(start)
    table = 4.0 * case["heads"] * _buckets(case)[2] * (2 if case["back"] else 1) if case["bias"] else 0.0
    return {"bytes": rows + table, "flops": pairs * width * (10.0 if case["back"] else 4.0)}
