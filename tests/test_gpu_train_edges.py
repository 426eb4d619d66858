"""The training operators on the GPU where inputs, sizes and streams are at the edge of what the header allows: entries of the bias that
are not finite, starts of segments that do not ascend, calls without voxels, gradients at both ends of float's range, results whose
memory another stream wants, two threads, calls between layers."""
import ctypes
import math
import threading

import numpy as np
import pytest
import torch

import dsvt_inputs as di
import train_reference as ref
from gpu_helpers import dev
from paper_2301_06051_b200 import api
from test_gpu_train_ops import EPS, TYPES, Problem

pytestmark = pytest.mark.gpu

BIG = float(np.finfo(np.float32).max)


@pytest.fixture(scope="module")
def ctx():
    c = api.Context(70000, 4096, 256)
    yield c
    c.close()


# ---- the bias's entries ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("lens", [[17, 36, 5, 36], [150, 20, 200]])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_bias_entry_that_is_not_finite_spoils_its_rows_alone(ctx, typ, lens, bad):
    """softmax of a row with a score of NaN or +inf is NaN; rows without such a pair are what they were."""
    p = Problem(lens, 4, 24, typ, seed=23, packed=False, spread=12, extent=(9, 9, 3))
    head, bucket = 1, int(p.buckets(p.segments[0])[2, 5])
    out, (dq, dk, dv, _) = p.forward(ctx), p.backward(ctx)
    p.rel.table[head, bucket] = bad
    rows, segments = torch.zeros(p.n, dtype=torch.bool), torch.zeros(p.n, dtype=torch.bool)
    met = np.zeros(p.table.shape[1], dtype=bool)
    for ids in p.segments:
        hit = (p.buckets(ids) == bucket).any(1)
        rows[torch.from_numpy(ids[hit])] = True
        if hit.any():
            segments[torch.from_numpy(ids)] = True
            met[p.buckets(ids)[hit].reshape(-1)] = True
    assert rows.any() and not rows.all()
    got, (gq, gk, gv, dbias) = p.forward(ctx), p.backward(ctx)
    others = [h for h in range(4) if h != head]
    for what, a, b, spoilt in (("out", got, out, rows), ("dq", gq, dq, rows), ("dk", gk, dk, segments), ("dv", gv, dv, segments)):
        a, b = a.cpu(), b.cpu()
        assert torch.isnan(a[spoilt][:, head]).all(), what
        assert torch.equal(a[~spoilt][:, head], b[~spoilt][:, head]) and torch.equal(a[:, others], b[:, others]), what
    # the bias's gradient: of the buckets that a spoilt row has a pair of, and of these alone
    assert torch.isnan(dbias[head, torch.from_numpy(met)]).all()
    p.host[3] = p.host[3].clone()
    p.host[3][rows, head] = 0  # (what is left are the other rows' sums)
    value, bound = p.want(back=True)[0]["dbias"]
    rest = torch.from_numpy(~met)
    ref.check(dbias[head, rest.cuda()], (value[head, rest], bound[head, rest]), "dbias")
    ref.check(dbias[others], (value[others], bound[others]), "dbias of the other heads")
    assert ctx.status_sync() == 0


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("lens", [[17, 36, 5], [150, 20, 200]])
def test_a_bias_of_the_largest_float_takes_all_the_weight(ctx, typ, lens):
    p = Problem(lens, 2, 16, typ, seed=24, packed=False)
    bucket = int(p.buckets(p.segments[0])[0, 0])  # of a voxel and itself, and of what shares its cell
    p.rel.table[:, bucket] = BIG
    got = p.forward(ctx).double().cpu()
    dq, dk, dv, dbias = (t.double().cpu() for t in p.backward(ctx))
    assert all(torch.isfinite(t).all() for t in (got, dq, dk, dv, dbias))
    for ids in p.segments:
        mine = torch.from_numpy(p.buckets(ids) == bucket).double()
        w = mine / mine.sum(1, keepdim=True)  # equal weights
        v = p.host[2].double()[torch.from_numpy(ids)]
        want, size = torch.einsum("ij,jhd->ihd", w, v), torch.einsum("ij,jhd->ihd", w, v.abs())
        # the weights' rounding, the result's, and fp32 sums of up to 200 terms
        bound = (EPS[typ] / 2 + (len(ids) + 24) * ref.U) * size * (1 + EPS[typ]) + EPS[typ] / 2 * want.abs() + 1e-6 * EPS[typ]
        assert ((got[torch.from_numpy(ids)] - want).abs() <= bound).all()
    assert ctx.status_sync() == 0


# ---- nothing to do -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("max_len", [36, 0])
def test_no_voxels_with_a_bias(ctx, max_len):
    index, buckets = api.log_buckets((6, 6, 1), (2, 2, 1), (4, 4, 1))
    rel = api.BucketBias(torch.randn((4, buckets), device="cuda"), (6, 6, 1), index)
    e = torch.empty((0, 4, 16), dtype=torch.bfloat16, device="cuda")
    seg = api.Segments(torch.zeros(3, dtype=torch.int32, device="cuda"), max_len, torch.empty(0, dtype=torch.int32, device="cuda"),
                       torch.empty((0, 4), dtype=torch.int32, device="cuda"))
    assert ctx.segment_attention(e, e, e, seg, bias=rel).shape == e.shape
    dbias = torch.full_like(rel.table, 9.0)
    grads = ctx.segment_attention_backward(e, e, e, e, seg, bias=rel, dbias=dbias)
    assert all(t.shape == e.shape for t in grads[:3]) and torch.all(dbias == 0)
    bad = api.BucketBias(rel.table, (6, 6, 1), np.full(23, 10000))
    with pytest.raises(api.DsvtError):  # the tables are looked at all the same
        ctx.segment_attention(e, e, e, seg, bias=bad)
    assert ctx.status_sync() == 0
