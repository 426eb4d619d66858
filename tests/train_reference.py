"""Float64 definitions of the training operators and how far a kernel may lie from them.

The bounds follow the arithmetic that include/dsvt.h states.  u = 2^-23 bounds one fp32 operation, truncating additions of the tensor
cores included; tf32 parts leave out at most 3 x 2^-22 of a product, 6 u.  A sum of m products is off by at most (m + 8) u times the
sum of their magnitudes.  eps is torch.finfo(type).eps; a rounding to the type is off by eps / 2 of the value."""
import math

import numpy as np
import torch

U = 2.0 ** -23
LOG2E = 1.0 / math.log(2.0)


def bucket_index(cells_i, cells_j, extent, index):
    """Buckets of all pairs: cells int64 [m, 3] on the host."""
    parts = np.split(np.asarray(index, dtype=np.int64), np.cumsum([2 * e - 1 for e in extent])[:-1])
    total = 0
    for a, e in enumerate(extent):
        d = np.clip(cells_i[:, None, a] - cells_j[None, :, a], 1 - e, e - 1)
        total = total + parts[a][d + e - 1]
    return total


def attention(q, k, v, segments, scale, cap=0.0, bias=None, buckets=None, d_out=None, eps=0.0, device="cpu"):
    """q, k, v, d_out: float64 [n, heads, dim].  segments: list of index arrays; buckets(ids): [len, len] integers.  Returns a dict of
    (value, bound) for out or dq, dk, dv and dbias, and the rows that belong to a segment."""
    n, heads, dim = q.shape
    q, k, v = (t.to(device) for t in (q, k, v))
    bias = None if bias is None else bias.double().to(device)
    back = d_out is not None
    names = ("dq", "dk", "dv") if back else ("out",)
    val = {m: torch.zeros((n, heads, dim), dtype=torch.float64, device=device) for m in names}
    tol = {m: torch.zeros_like(val[m]) for m in names}
    if back and bias is not None:
        val["dbias"], tol["dbias"] = torch.zeros_like(bias), torch.zeros_like(bias)
        most, counts = 0.0, torch.zeros(bias.shape[1], dtype=torch.float64, device=device)
    covered = torch.zeros(n, dtype=torch.bool)
    low = -float(np.finfo(np.float32).max)
    # float16 weights below 2^-14 are multiples of 2^-24, off by half of that whatever their size
    low_weight = 2.0 ** -25 if eps == 2.0 ** -10 else 0.0
    for ids in segments:
        if len(ids) == 0:
            continue
        L = len(ids)
        rows = torch.as_tensor(np.asarray(ids), dtype=torch.long)
        covered[rows] = True
        rows = rows.to(device)
        a, b, c = q[rows].transpose(0, 1), k[rows].transpose(0, 1), v[rows].transpose(0, 1)  # [heads, L, dim]
        z = a @ b.transpose(1, 2) * scale
        mag = a.abs() @ b.abs().transpose(1, 2) * abs(scale)
        err = (dim + 8) * U * mag
        t = torch.tanh(z / cap) if cap > 0 else None
        s = cap * t if cap > 0 else z
        err = err + (8 * U * s.abs() if cap > 0 else 0.0)
        if bias is not None:
            w = torch.as_tensor(buckets(ids), device=device)
            add = bias[:, w]
            s = s + add
            err = err + 4 * U * torch.where(add > -1e30, add.abs(), 0.0)
        real = s > -1e30  # masked scores are the lowest float in fp32 whatever is added
        s = torch.where(real, s, torch.where(s < -1e300, s, torch.full_like(s, low)))
        m = s.amax(dim=2, keepdim=True)
        m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
        e = torch.exp(s - m)
        l = e.sum(dim=2, keepdim=True)
        p = torch.where(l > 0, e / torch.where(l > 0, l, 1.0), 0.0)
        # relative error of a weight: scores (its own, the maximum's and the sum's), the exponential, the sum and the division
        spread = torch.where(real, (s - m).abs(), 0.0)
        r = 2 * (err + 4 * U * spread).amax(dim=2, keepdim=True) + (L + 16) * U
        r = torch.expm1(r.clamp(max=1.0))
        if not back:
            o, oa = p @ c, p @ c.abs()
            val["out"][rows] = o.transpose(0, 1)
            tol["out"][rows] = ((r + eps / 2 + (L + 8) * U) * oa * (1 + eps) + eps / 2 * o.abs() + low_weight * c.abs().sum(1, keepdim=True)).transpose(0, 1)
            continue
        do = d_out.to(device)[rows].transpose(0, 1)
        dp = do @ c.transpose(1, 2)
        dpe = (dim + 8) * U * (do.abs() @ c.abs().transpose(1, 2))
        D = (p * dp).sum(2, keepdim=True)
        De = (p * (dpe + (r + (L + 8) * U) * dp.abs())).sum(2, keepdim=True)
        ds = p * (dp - D)
        dse = p * (dpe + De + (r + 4 * U) * (dp.abs() + D.abs()))
        if bias is not None:
            flat = w.reshape(-1)
            val["dbias"].index_add_(1, flat, ds.reshape(heads, -1))
            tol["dbias"].index_add_(1, flat, (dse + 64 * U * ds.abs()).reshape(heads, -1))
            # the header: multiples of 2^-33 of the call's largest bound, each value off by half of one
            most = max(most, float(((p * dp).abs().amax(2, keepdim=True) + D.abs() * p.amax(2, keepdim=True)).max()))
            counts.index_add_(0, flat, torch.ones_like(flat, dtype=torch.float64))
        slope = 1 - t * t if cap > 0 else torch.ones_like(ds)
        dz = ds * slope * scale
        # (the slope's own error: t's, doubled)
        dze = abs(scale) * (dse * slope + ds.abs() * ((2 * err / cap + 16 * U) if cap > 0 else 2 * U)) + eps / 2 * dz.abs() * (1 + eps)
        for name, w1, w1e, other in (("dq", dz, dze, b), ("dk", dz.transpose(1, 2), dze.transpose(1, 2), a),
                                     ("dv", p.transpose(1, 2), (p * (r + eps / 2) * (1 + eps)).transpose(1, 2), do)):
            g = w1 @ other
            ga = w1e @ other.abs() + (L + 8) * U * (w1.abs() @ other.abs())
            val[name][rows] = g.transpose(0, 1)
            if name == "dv":
                ga = ga + low_weight * other.abs().sum(1, keepdim=True)
            tol[name][rows] = (ga * (1 + eps) + eps / 2 * g.abs()).transpose(0, 1)
    # results below the type's normal range round to multiples of its smallest step
    floor = {0.0: 1e-37}.get(eps, 2.0 ** -24 if eps == 2.0 ** -10 else 1e-37)
    if "dbias" in tol:
        tol["dbias"] = tol["dbias"] + 2 * L_SUM * val["dbias"].abs() + 2.0 ** -34 * most * counts
    return {m: (val[m].cpu(), tol[m].cpu() + (floor if m != "dbias" else 1e-37)) for m in val}, covered


L_SUM = 256 * U  # joining the partial sums of a bias entry


def layer_norm(x, r, g, b, layer_eps, dy=None, eps=0.0):
    """x, r, dy float64 [n, C]; g, b float64 [C].  (value, bound) of y, or of dx, dg and db."""
    n, C = x.shape
    u = x if r is None else x + r
    mean = u.mean(1, keepdim=True)
    c = u - mean
    var = (c * c).mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + layer_eps)
    h = c * rstd
    # a lane's sum of up to 32 entries, a tree over lanes: 48 additions at most, each of magnitude sum |u|
    ce = 2 * U * u.abs() + 50 * U * u.abs().mean(1, keepdim=True)
    rel = (c.abs() * ce).mean(1, keepdim=True) / (var + layer_eps) + 60 * U  # of rstd
    he = ce * rstd + h.abs() * (rel + 2 * U)
    if dy is None:
        y = h * g + b
        return y, he * g.abs() + 2 * U * (h * g).abs() + 2 * U * y.abs() + (eps / 2) * y.abs() * (1 + 8 * U) + 1e-37 + eps * he * g.abs()
    w = dy * g
    mw, mwh = w.mean(1, keepdim=True), (w * h).mean(1, keepdim=True)
    mwe = 50 * U * w.abs().mean(1, keepdim=True)
    mwhe = (w.abs() * he).mean(1, keepdim=True) + 50 * U * (w * h).abs().mean(1, keepdim=True)
    inner = w - mw - h * mwh
    ie = 4 * U * (w.abs() + mw.abs() + (h * mwh).abs()) + mwe + he * mwh.abs() + h.abs() * mwhe
    dx = rstd * inner
    dxe = (rstd * (ie + inner.abs() * (rel + 2 * U))) * (1 + eps) + eps / 2 * dx.abs() + (2.0 ** -25 if eps == 2.0 ** -10 else 1e-37)
    # sums over the rows: a lane's in sequence, groups and blocks after one another
    steps = n / 64 + 64
    dg, db = (dy * h).sum(0), dy.sum(0)
    dge = (dy.abs() * he).sum(0) + steps * U * (dy * h).abs().sum(0)
    return {"dx": (dx, dxe), "dg": (dg, dge + 1e-37), "db": (db, steps * U * dy.abs().sum(0) + 1e-37)}


def check(got, want, what):
    value, bound = want
    got = got.detach().double().cpu()
    assert got.shape == value.shape, (what, got.shape, value.shape)
    assert torch.isfinite(got).all(), "%s: not finite" % what
    over = (got - value).abs() / bound
    worst = float(over.max()) if over.numel() else 0.0
    assert worst <= 1.0, "%s: %.3g times its bound (value %.6g, got %.6g)" % (
        what, worst, float(value.reshape(-1)[over.argmax()]), float(got.reshape(-1)[over.argmax()]))
    return worst
