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


# ---- starts that do not ascend -----------------------------------------------------------------------------------------
def _starts_problem(kind):
    lens = {"sets": [30, 7, 36, 1] * 60, "windows": [200, 90, 7, 130] * 20, "voxels": [3] * 3000}[kind]
    p = Problem(lens, 2 if kind != "voxels" else 1, 16, torch.float32, seed=len(lens), packed=False, lead=2, tail=3)
    p.whole = {**p.want()[0], **p.want(back=True)[0]}
    return p


def _check_starts(ctx, p, dropped, what):
    """All segments but the dropped ones are right, the others' rows stay as they were, and the call says so."""
    covered = torch.zeros(p.n, dtype=torch.bool)
    for i, ids in enumerate(p.segments):
        covered[torch.from_numpy(ids)] = i not in dropped
    out = torch.full((p.n, p.heads, p.dim), 7.0, device="cuda")
    grads = [torch.full_like(out, 7.0) for _ in range(3)]
    p.forward(ctx, out)
    assert ctx.status_sync() == api.STATUS_BAD_INDEX, what
    *_, dbias = p.backward(ctx, grads)
    assert ctx.status_sync() == api.STATUS_BAD_INDEX, what
    for name, got in zip(("out", "dq", "dk", "dv"), [out] + grads):
        ref.check(got.cpu()[covered], tuple(t[covered] for t in p.whole[name]), what + ": " + name)
        assert torch.all(got.cpu()[~covered] == 7.0), (what, name)
    value, bound = p.whole["dbias"]
    if dropped:
        segments, p.segments = p.segments, [p.segments[i] for i in sorted(dropped)]
        less, more = p.want(back=True)[0]["dbias"]
        value, bound, p.segments = value - less, bound + more, segments
    ref.check(dbias, (value, bound), what + ": dbias")


@pytest.mark.parametrize("kind", ["sets", "windows", "voxels"])
@pytest.mark.parametrize("value", [-1, None], ids=["below", "beyond"])
def test_one_bad_start_costs_its_two_segments_and_no_others(ctx, kind, value):
    p = _starts_problem(kind)
    start, count = p.seg.start.clone(), len(p.segments)
    bad = -1 if value == -1 else p.n + 9
    for at in (1, 2, 3, count // 3, count // 2 + 1, count - 2, count - 1):
        p.seg.start.copy_(start)
        p.seg.start[at] = bad
        _check_starts(ctx, p, {at - 1, at}, "%s, entry %d" % (kind, at))
    if kind == "windows":  # several, each between two that are in place
        p.seg.start.copy_(start)
        p.seg.start[5:70:8] = bad
        _check_starts(ctx, p, {i - d for i in range(5, 70, 8) for d in (0, 1)}, "several")


@pytest.mark.parametrize("kind", ["sets", "windows", "voxels"])
def test_starts_that_were_never_written_behind_the_last_segment(ctx, kind):
    """A table of starts with room for more segments than there are, zeros behind the last one's end and no count on the device."""
    p = _starts_problem(kind)
    p.seg.start = torch.cat([p.seg.start, torch.zeros(400, dtype=torch.int32, device="cuda")])
    _check_starts(ctx, p, set(), kind)  # (the pair at the seam is no segment: said; all others are)


@pytest.mark.parametrize("kind", ["sets", "windows", "voxels"])
def test_any_start_out_of_place_is_said(ctx, kind):
    """Neighbours out of place together: which segments are worked on beside them is open, that the starts are bad is not."""
    p = _starts_problem(kind)
    start = p.seg.start.clone()
    g = torch.Generator().manual_seed(3)
    for i in range(12):
        at, m = int(torch.randint(1, len(p.segments) - 12, (1,), generator=g)), int(torch.randint(2, 11, (1,), generator=g))
        p.seg.start.copy_(start)
        p.seg.start[at:at + m] = start[max(at - 4, 0)] if i % 2 else p.n + 1
        if i % 3 == 0:
            p.seg.start[at:at + m] += torch.arange(m, dtype=torch.int32, device="cuda")
        p.forward(ctx)
        assert ctx.status_sync() & api.STATUS_BAD_INDEX, (i, at, m)
        p.backward(ctx)
        assert ctx.status_sync() & api.STATUS_BAD_INDEX, (i, at, m)


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


# ---- more voxels than statistics ------------------------------------------------------------------------------------------
def test_segments_that_are_held_whole_take_any_number_of_voxels():
    """1,800,000 voxels: the backward pass keeps statistics in the workspace for longer segments alone."""
    n, each = 1800000, 60
    own = api.Context(n, 1, 256)
    p = Problem([each] * (n // each), 1, 8, torch.bfloat16, seed=5, packed=False, max_len=80)
    p.segments = p.segments[:3] + p.segments[n // each // 2:][:3] + p.segments[-3:]
    for p.seg.max_len in (80, 120):
        out, (dq, dk, dv, _) = p.forward(own), p.backward(own)
        want = {**p.want()[0], **p.want(back=True)[0]}
        rows = torch.from_numpy(np.concatenate(p.segments))
        for name, got in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv)):
            ref.check(got.cpu()[rows], tuple(t[rows] for t in want[name]), name)
    p.seg.max_len = 121
    p.forward(own)
    with pytest.raises(api.DsvtError) as e:
        p.backward(own)
    assert e.value.code == -2
    assert own.status_sync() == 0
    own.close()


# ---- the ends of float's range -----------------------------------------------------------------------------------------
def _two_clusters(rest, near, dp, do):
    """Voxels 0 and 1 attend to each other alone (`near`: the bias between them), the `rest` others among themselves; the rows' products
    with v are dp for query 0 where d_out is `do`.  Returns the problem with everything but that zero."""
    p = Problem([2 + rest], 1, 8, torch.float32, seed=31, ordered=False, packed=False, extent=(4, 4, 1), scale=0.0)
    p.cells[:] = [100, 0, 0]
    p.cells[0], p.cells[1] = [0, 0, 0], [1, 0, 0]
    p.seg.coords.copy_(torch.from_numpy(np.concatenate([np.zeros((p.n, 1)), p.cells], 1).astype(np.int32)))
    d = np.arange(7)
    p.index = np.concatenate([7 * d, d, [0]]).astype(np.int32)  # a bucket per displacement
    p.table = torch.zeros((1, 49))
    p.table[0, [7 * 6 + 3, 3]] = -math.inf  # between the clusters, either way
    p.table[0, [7 * 2 + 3, 7 * 4 + 3]] = near
    p.rel = api.BucketBias(p.table.cuda(), p.extent, p.index)
    for t in p.host:
        t.zero_()
    p.host[2][0, 0, 0], p.host[2][1, 0, 0] = dp
    p.host[3][0, 0, 0] = do
    p.q, p.k, p.v, p.do = (t.contiguous().cuda() for t in p.host)
    return p


@pytest.mark.parametrize("rest", [1, 140])
@pytest.mark.parametrize("near,dp", [(0.0, (1.0, -1.0)), (-7.0, (1.0, 0.5)), (-7.0, (1.0, 0.25))])
def test_bias_gradients_near_the_largest_float(ctx, rest, near, dp):
    """dS of up to half the largest float; products and D so large that their bound passes it."""
    p = _two_clusters(rest, near, dp, 3.2e38)
    *_, dbias = p.backward(ctx)
    want, _ = p.want(back=True)
    assert float(want["dbias"][0].abs().max()) > 1e35
    ref.check(dbias, want["dbias"], "dbias")
    assert ctx.status_sync() == 0


@pytest.mark.parametrize("lens", [[36, 20, 3, 36], [150, 36]])
def test_bias_gradients_near_the_smallest_float(ctx, lens):
    p = Problem(lens, 4, 24, torch.bfloat16, seed=32, packed=False)
    p.host[3] = (p.host[3].double() * 2.0 ** -122).to(torch.bfloat16)
    p.do = p.host[3].contiguous().cuda()
    *_, dbias = p.backward(ctx)
    value, bound = p.want(back=True)[0]["dbias"]
    counts = torch.zeros(p.table.shape[1], dtype=torch.float64)
    for ids in p.segments:
        counts += torch.from_numpy(np.bincount(p.buckets(ids).reshape(-1), minlength=p.table.shape[1]))
    # beside the bound of ordinary sizes: results of fp32 operations here are multiples of 2^-149, a dS comes from dim + length and some 16
    # of them, and the header's multiples are of 2^-145
    step = (24 + max(lens) + 16) * 2.0 ** -150 + 2.0 ** -146
    ref.check(dbias, (value, bound + counts * step), "dbias")
    # the products' bound is a loose one: without it, that many half steps to a dS of 2^-125 or so leave 1e-4 of sums of up to 1000
    assert (dbias.double().cpu() - value).norm() <= 1e-4 * value.norm()


def test_a_cap_beyond_the_arithmetic_is_refused(ctx):
    p = Problem([20, 5], 2, 16, torch.float32, seed=2)
    for cap in (1e-44, 1e-40, 3e38):
        p.cap = cap
        with pytest.raises(api.DsvtError):
            p.forward(ctx)
        with pytest.raises(api.DsvtError):
            p.backward(ctx)
    for cap in (1e-30, 1e30):  # almost no score at all, and none that is capped
        p.cap = cap
        got = p.forward(ctx)
        want, covered = p.want()
        ref.check(got, want["out"], "cap %g" % cap)
    assert ctx.status_sync() == 0


# ---- streams and threads -----------------------------------------------------------------------------------------------
def _calls(own):
    """Calls that make their own results, by name: each returns tensors."""
    p = Problem([36, 20, 200, 1, 50], 8, 24, torch.bfloat16, seed=8, packed=False)
    x = torch.randn((p.n, 192), device="cuda")
    cells = torch.randperm(900, generator=torch.Generator().manual_seed(1))[:300]
    coords = torch.stack([torch.zeros_like(cells), cells // 30, cells % 30, torch.zeros_like(cells)], 1).to(torch.int32).cuda()
    feats = torch.randn((300, 64), device="cuda")
    sets = lambda t: [t.set_table, t.set_rowoff, t.num_sets]
    return {
        "segment_attention": lambda: [p.forward(own)],
        "segment_attention_backward": lambda: list(p.backward(own)),
        "layer_norm": lambda: [own.layer_norm(x, None, None)],
        "layer_norm_backward": lambda: list(own.layer_norm_backward(x, x, None)),
        "partition": lambda: sets(own.partition(coords, 1, (30, 30, 1), (12, 12, 1), 16, 0)),
        "partition_rotated": lambda: [t for s in own.partition_rotated(coords, 1, (30, 30, 1), (12, 12, 1), 16) for t in sets(s)],
        "bev_scatter": lambda: [own.bev_scatter(coords, feats, 1, (30, 30, 1))],
    }


CALLS = ["segment_attention", "segment_attention_backward", "layer_norm", "layer_norm_backward", "partition", "partition_rotated",
         "bev_scatter"]


@pytest.mark.parametrize("name", CALLS)
def test_a_result_dropped_while_the_contexts_stream_is_busy(name):
    """Its memory may not go to the current stream's next tensor while the context's stream has still to write it."""
    own = api.Context(2000, 64, 256, stream=torch.cuda.Stream())
    call = _calls(own)[name]
    torch.cuda.synchronize()
    call()  # (kernels loaded)
    torch.cuda.synchronize()
    with torch.cuda.stream(own.stream):
        torch.cuda._sleep(200_000_000)
    sizes = [(t.shape, t.dtype) for t in call()]
    mine = [torch.full(shape, 3, dtype=dtype, device="cuda") for shape, dtype in sizes for _ in range(2)]
    assert not own.stream.query()  # the kernels are still to come
    torch.cuda.synchronize()
    assert all(torch.all(t == 3) for t in mine)
    assert own.status_sync() == 0
    own.close()


@pytest.mark.parametrize("name", CALLS)
def test_a_result_in_memory_that_the_current_stream_still_reads(name):
    own = api.Context(2000, 64, 256, stream=torch.cuda.Stream())
    call = _calls(own)[name]
    sizes = [(t.shape, t.dtype) for t in call()]
    torch.cuda.synchronize()
    old = [torch.full(shape, 3, dtype=dtype, device="cuda") for shape, dtype in sizes for _ in range(2)]
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    read = [t.clone() for t in old]
    del old
    got = call()
    own.stream.synchronize()
    assert not torch.cuda.current_stream().query()  # the reads are still to come
    torch.cuda.synchronize()
    assert all(torch.all(t == 3) for t in read)
    again = call()
    own.stream.synchronize()
    if name != "partition" and name != "partition_rotated":  # (tables have rows that no set fills)
        assert all(torch.equal(a, b) for a, b in zip(got, again) if a is not None)
    own.close()


def test_layer_norms_of_two_threads_at_once():
    """Rows of 8192 and of 6144 channels go through one kernel, whose room in shared memory is the process's."""
    widths, failed, go = (8192, 6144), [], threading.Barrier(2)
    own = [api.Context(64, 1, 256, stream=torch.cuda.Stream()) for _ in widths]
    xs = [torch.randn((37, C), device="cuda") for C in widths]
    outs = [[torch.empty_like(x), torch.empty(x.shape[1], device="cuda"), torch.empty(x.shape[1], device="cuda")] for x in xs]
    torch.cuda.synchronize()

    def work(i):
        at = [t.data_ptr() for t in outs[i]]
        call = (own[i]._h, 0, xs[i].data_ptr(), None, xs[i].data_ptr(), 37, widths[i], None, 1e-5, *at)
        go.wait()
        for _ in range(30000):
            rc = own[i].lib.dsvt_layer_norm_backward(*call)
            if rc:
                failed.append((widths[i], rc, own[i].lib.dsvt_last_cuda_error(own[i]._h)))
                return

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    torch.cuda.synchronize()
    assert not failed, failed
    for i, x in enumerate(xs):
        one = torch.ones(x.shape[1], dtype=torch.float64)
        want = ref.layer_norm(x.double().cpu(), None, one, 0 * one, 1e-5, x.double().cpu())
        for name, got in zip(("dx", "dg", "db"), outs[i]):
            ref.check(got, want[name], name)
        own[i].close()


# ---- between layers ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("C,hidden", [(192, 384), (128, 256)])
def test_calls_between_fp32_layers(C, hidden):
    """fp32 layers keep their weights' parts and intermediate rows where the backward passes keep their sums; kernels overlap their
    neighbours' tails.  Together without a wait: the same bits as alone."""
    n = 3000
    case = di.random_case(C, n, (60, 60, 1), (12, 12, 1), 36, C, 8, hidden, layernorm=True)
    own = api.Context(n, 25, C)
    coords, x = dev(case["coords"]), dev(case["feats"])
    table = own.partition(coords, 1, case["grid"], case["window"], 36, 0)
    w = api.device_weights(case["blocks"][0][0], api.FP32, own.device)
    p = Problem([36, 20, 200, 1, 50] * 5, 8, 24, torch.bfloat16, seed=8)
    dy = torch.randn((n, C), device="cuda")
    layer = lambda to: own.layer(x, table, w, to, coords=coords)
    chain = lambda to: own.layers(x, [table, table], [w, w], to, coords=coords)
    alone = []
    for f in (layer, chain):
        y = torch.empty_like(x)
        f(y)
        torch.cuda.synchronize()
        alone.append(y)
    grads = p.backward(own)
    torch.cuda.synchronize()
    norm = own.layer_norm_backward(x, dy, None)
    torch.cuda.synchronize()
    for order in ("lbn", "bln", "cbncb", "nlbcnl", "bcb", "ncn"):
        got = []
        for _ in range(4):
            for c in order:
                if c in "lc":
                    y = torch.full_like(x, 5.0)
                    (layer if c == "l" else chain)(y)
                    got.append(((y,), (alone["lc".index(c)],)))
                elif c == "b":
                    got.append((p.backward(own), grads))
                else:
                    got.append((own.layer_norm_backward(x, dy, None), norm))
        torch.cuda.synchronize()
        for have, want in got:
            assert all(torch.equal(a, b) for a, b in zip(have, want)), order
    assert own.status_sync() == 0
    own.close()


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("C", [192, 250, 1028])
def test_layer_norm_of_constant_rows_whose_sum_rounds(ctx, typ, C):
    x = (torch.tensor([0.1, -0.7, 1 / 3, 5.1, 1e-3])[:, None] * torch.ones(C)).to(typ)
    one = torch.ones(C, dtype=torch.float64)
    y = ctx.layer_norm(x.cuda(), None, None, eps=1e-3)
    ref.check(y, ref.layer_norm(x.double(), None, one, 0 * one, 1e-3, eps=EPS[typ]), "y")
    dx, dg, db = ctx.layer_norm_backward(x.cuda(), x.cuda(), None, eps=1e-3)
    want = ref.layer_norm(x.double(), None, one, 0 * one, 1e-3, x.double(), eps=EPS[typ])
    for name, got in (("dx", dx), ("dg", dg), ("db", db)):
        ref.check(got, want[name], name)
