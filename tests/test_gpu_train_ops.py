"""The training operators on the GPU against their float64 definitions (tests/train_reference.py), elementwise within the bounds
that follow from the arithmetic."""
import ctypes
import math

import numpy as np
import pytest
import torch

import train_reference as ref
from paper_2301_06051_b200 import api

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
EPS = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -7, torch.float16: 2.0 ** -10}
LOW = float(np.finfo(np.float32).min)


@pytest.fixture(scope="module")
def ctx():
    c = api.Context(70000, 4096, 256)
    yield c
    c.close()


class Problem:
    """Segments of the given lengths over the rows of n voxels: `lead` rows in front, `tail` rows behind them in no segment."""

    def __init__(self, lens, heads, dim, typ, seed=0, lead=0, tail=0, ordered=True, packed=True, bias=True, extent=(6, 6, 3), cap=0.0,
                 spread=7, scale=None, max_len=None):
        g = torch.Generator().manual_seed(seed)
        self.n = n = sum(lens) + lead + tail
        self.heads, self.dim, self.typ, self.cap = heads, dim, typ, cap
        self.scale = dim ** -0.5 if scale is None else scale
        rows = torch.randn((n, 4, heads, dim), generator=g).to(typ)
        self.host = [rows[:, i] for i in range(4)]
        if packed:  # one projection's output
            dev = rows[:, :3].contiguous().cuda()
            self.q, self.k, self.v = dev.unbind(1)
        else:
            self.q, self.k, self.v = (rows[:, i].contiguous().cuda() for i in range(3))
        self.do = rows[:, 3].contiguous().cuda()
        order = torch.randperm(n, generator=g) if ordered else torch.arange(n)
        start = lead + np.concatenate([[0], np.cumsum(lens)])
        self.segments = [order[start[i]:start[i + 1]].numpy() for i in range(len(lens))]
        self.cells = torch.randint(0, spread, (n, 3), generator=g).numpy()
        coords = np.concatenate([np.zeros((n, 1), dtype=np.int64), self.cells], 1).astype(np.int32)
        self.seg = api.Segments(torch.from_numpy(start.astype(np.int32)).cuda(), max_len or max(list(lens) + [1]),
                                order.to(torch.int32).cuda() if ordered else None, torch.from_numpy(coords).cuda())
        self.extent = extent
        self.index, count = api.log_buckets(extent, (2, 2, 1), (4, 4, 2))
        self.table = torch.randn((heads, count), generator=g) if bias else None
        self.rel = api.BucketBias(self.table.cuda(), extent, self.index) if bias else None

    def buckets(self, ids):
        return ref.bucket_index(self.cells[ids], self.cells[ids], self.extent, self.index)

    def want(self, back=False):
        q, k, v, do = (t.double() for t in self.host)
        return ref.attention(q, k, v, self.segments, self.scale, self.cap, self.table, self.buckets if self.table is not None else None,
                             d_out=do if back else None, eps=EPS[self.typ], device="cuda")

    def forward(self, ctx, out=None):
        return ctx.segment_attention(self.q, self.k, self.v, self.seg, bias=self.rel, scale=self.scale, cap=self.cap, out=out)

    def backward(self, ctx, out=None):
        return ctx.segment_attention_backward(self.q, self.k, self.v, self.do, self.seg, bias=self.rel, scale=self.scale, cap=self.cap, out=out)


def _same_outside(t, covered, mark):
    assert torch.equal(t[~covered].float().cpu(), torch.full_like(t[~covered].float().cpu(), mark))


def _check_both(ctx, p):
    out = torch.full((p.n, p.heads, p.dim), 7.0, dtype=p.typ, device="cuda")
    p.forward(ctx, out)
    want, covered = p.want()
    _same_outside(out, covered, 7.0)
    ref.check(out[covered], tuple(t[covered] for t in want["out"]), "out")
    grads = [torch.full((p.n, p.heads, p.dim), 7.0, dtype=p.typ, device="cuda") for _ in range(3)]
    *_, dbias = p.backward(ctx, grads)
    want, covered = p.want(back=True)
    for name, got in zip(("dq", "dk", "dv"), grads):
        _same_outside(got, covered, 7.0)
        ref.check(got[covered], tuple(t[covered] for t in want[name]), name)
    if p.table is not None:
        ref.check(dbias, want["dbias"], "dbias")
    else:
        assert dbias is None
    assert ctx.status_sync() == 0


LENGTHS = [[1], [2, 1, 3], [0, 1, 2, 0, 0, 3, 8, 16, 17, 15, 36, 7, 0], [31, 32, 33], [64, 63, 65], [36] * 9, [90, 72, 1], [127, 128],
           [129], [128, 1, 130, 0, 5], [300, 7, 200, 64, 65], [1000]]


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("lens", LENGTHS, ids=[str(len(l)) + "x" + str(max(l)) for l in LENGTHS])
def test_attention_of_segments_of_every_length(ctx, typ, lens):
    _check_both(ctx, Problem(lens, 8, 24, typ, seed=sum(lens), lead=3, tail=5))


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("heads,dim", [(1, 8), (8, 16), (3, 40), (4, 32), (2, 48), (5, 56), (4, 64), (2, 72), (1, 128), (12, 16), (17, 24)])
def test_attention_of_every_head_layout(ctx, typ, heads, dim):
    _check_both(ctx, Problem([5, 36, 20, 1, 70, 150], heads, dim, typ, seed=heads * dim, tail=1))


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("kw", [dict(bias=False), dict(cap=2.0), dict(cap=2.0, bias=False), dict(ordered=False), dict(packed=False),
                                dict(scale=2.5), dict(scale=0.0), dict(scale=-0.5), dict(extent=(1, 1, 1)), dict(extent=(128, 3, 2), spread=200),
                                dict(max_len=100000)],
                         ids=lambda kw: "-".join(kw))
def test_attention_variants(ctx, typ, kw):
    _check_both(ctx, Problem([19, 36, 1, 5, 140, 33], 4, 24, typ, seed=11, lead=2, **kw))


@pytest.mark.parametrize("lens", [[20, 36, 7], [200, 30]])
@pytest.mark.parametrize("mask", [-math.inf, LOW])
def test_masked_pairs(ctx, lens, mask):
    """Far pairs masked; then every pair but those of one displacement, which leaves rows with a single key or none."""
    p = Problem(lens, 4, 16, torch.float32, seed=3)
    p.table[:, :p.table.shape[1] // 3] = mask
    p.rel.table.copy_(p.table)
    _check_both(ctx, p)
    p.table[:] = mask
    p.table[:, p.buckets(p.segments[0])[0, 1]] = 0.5
    p.rel.table.copy_(p.table)
    _check_both(ctx, p)
    p.table[:] = mask  # no pair is left: zeros, or equal weights
    p.rel.table.copy_(p.table)
    _check_both(ctx, p)


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("lens", [[17, 20, 5, 36], [150, 20, 200]])
def test_what_is_not_finite_stays_in_its_segment(ctx, typ, lens):
    p = Problem(lens, 4, 24, typ, seed=5, packed=False, bias=False)
    clean, grads = p.forward(ctx).clone(), [g.clone() for g in p.backward(ctx)[:3]]
    for t, bad in ((p.q, math.nan), (p.k, math.inf), (p.v, math.nan), (p.do, -math.inf)):
        t[torch.from_numpy(p.segments[1]).cuda()[3]] = bad
    other = torch.from_numpy(np.concatenate([p.segments[0], *p.segments[2:]])).cuda()
    assert torch.equal(p.forward(ctx)[other], clean[other])
    for got, want in zip(p.backward(ctx)[:3], grads):
        assert torch.equal(got[other], want[other])
    assert torch.isnan(p.forward(ctx)[torch.from_numpy(p.segments[1]).cuda()]).any()


@pytest.mark.parametrize("lens", [[17, 20, 5, 36], [150, 20, 200]])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_gradient_that_is_not_finite_reaches_its_buckets_alone(ctx, lens, bad):
    p = Problem(lens, 4, 24, torch.bfloat16, seed=6, packed=False)
    voxel, ids = int(p.segments[0][2]), p.segments[0]
    p.do[voxel] = bad
    *_, dbias = p.backward(ctx)
    hit = np.unique(p.buckets(ids)[2])  # of the pairs of that query
    rest = np.setdiff1d(np.arange(p.table.shape[1]), hit)
    assert torch.isnan(dbias[:, hit]).all() and torch.isfinite(dbias[:, rest]).all() and len(rest)
    p.host[3] = p.host[3].clone()
    p.host[3][voxel] = 0  # the other rows' sums: that row's are zero then
    want, _ = p.want(back=True)
    ref.check(dbias[:, rest], tuple(t[:, rest] for t in want["dbias"]), "dbias")
    assert ctx.status_sync() == 0


@pytest.mark.parametrize("lens", [[30, 36, 3], [200, 70]])
def test_float16_gradients_beyond_its_range_on_the_way(ctx, lens):
    """dS of a million, results of thousands."""
    p = Problem(lens, 4, 24, torch.float16, seed=14, packed=False)
    for i, factor in enumerate((2.0 ** -10, 2.0 ** -10, 64.0, 2000.0)):
        p.host[i] = (p.host[i].float() * factor).half()
    p.q, p.k, p.v, p.do = (t.contiguous().cuda() for t in p.host)
    grads = p.backward(ctx)
    want, _ = p.want(back=True)
    assert float(want["dbias"][0].abs().max()) > 65504
    for name, got in zip(("dq", "dk", "dv", "dbias"), grads):
        ref.check(got, want[name], name)


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("lens", [[36, 20, 3, 36], [256, 100]])
def test_a_bias_for_every_displacement(ctx, typ, lens):
    """One bucket per displacement: the largest tables."""
    p = Problem(lens, 8, 16, typ, seed=17, spread=16)
    p.extent = (16, 16, 1)
    d = np.arange(31)
    p.index = np.concatenate([31 * d, d, [0]]).astype(np.int32)
    p.table = torch.randn((8, 961), generator=torch.Generator().manual_seed(1))
    p.rel = api.BucketBias(p.table.cuda(), p.extent, p.index)
    _check_both(ctx, p)


def test_the_segments_of_a_partition(ctx):
    """Sets and windows as dsvt_partition_rotated leaves them, counts on the device."""
    g = torch.Generator().manual_seed(9)
    n, grid, window, tau = 1500, (60, 60, 1), (12, 12, 1), 16
    cells = torch.randperm(3600, generator=g)[:n]
    cells = cells[cells % 60 < 45]  # some windows are empty
    n = len(cells)
    coords = torch.stack([torch.zeros(n, dtype=torch.int64), cells // 60, cells % 60, torch.zeros(n, dtype=torch.int64)], 1).to(torch.int32)
    t = ctx.partition(coords.cuda(), 1, grid, window, tau, 0, extras=True)
    p = Problem([n], 8, 24, torch.bfloat16, seed=2, extent=window)
    p.cells = coords[:, 1:].numpy().astype(np.int64)
    start, setoff, perm = (x.cpu().numpy() for x in (t.win_start, t.set_rowoff, t.perm))
    sets = int(t.num_sets.item())
    for seg, at, m in ((api.Segments.of_sets(t, coords.cuda()), setoff[:sets + 1], tau),
                       (api.Segments.of_windows(t, 144, coords.cuda()), start, 144)):
        p.seg, p.segments = seg, [perm[at[i]:at[i + 1]] for i in range(len(at) - 1)]
        assert max(len(s) for s in p.segments) <= m
        if m == tau:  # the members of a set are the distinct entries of its table row
            rows = t.set_table[:sets].cpu().numpy()
            assert all(set(rows[i]) == set(p.segments[i]) for i in range(sets))
        _check_both(ctx, p)


@pytest.mark.parametrize("max_len", [36, 200])
def test_bad_segments_are_left_out_and_reported(ctx, max_len):
    p = Problem([20, 30, 25, 10], 4, 16, torch.float32, seed=1, max_len=max_len)
    want, _ = p.want()
    bad = torch.from_numpy(p.segments[1]).cuda()
    keep = torch.from_numpy(np.concatenate([p.segments[0], p.segments[2], p.segments[3]]))
    # an order entry outside of the rows: that place is skipped, the others of its segment attend without it
    order, start = p.seg.order.clone(), p.seg.start.clone()
    p.seg.order[int(start[1]) + 4] = p.n
    out = torch.full((p.n, 4, 16), 7.0, device="cuda")
    p.forward(ctx, out)
    assert ctx.status_sync() == api.STATUS_BAD_INDEX
    ref.check(out.cpu()[keep], tuple(t[keep] for t in want["out"]), "others")
    assert torch.equal(out[bad[4]], torch.full((4, 16), 7.0, device="cuda"))
    p.segments[1] = np.delete(p.segments[1], 4)
    want, covered = p.want()
    ref.check(out.cpu()[covered], tuple(t[covered] for t in want["out"]), "without it")
    p.seg.order[int(start[1]) + 4] = -5
    *grads, dbias = p.backward(ctx)
    assert ctx.status_sync() == api.STATUS_BAD_INDEX
    back, covered = p.want(back=True)
    for name, got in zip(("dq", "dk", "dv"), grads):
        ref.check(got.cpu()[covered], tuple(t[covered] for t in back[name]), name)
    ref.check(dbias, back["dbias"], "dbias")
    p.seg.order.copy_(order)
    # an end beyond the rows: the last segment is dropped
    p.seg.start[4] = p.n + 9
    out.fill_(7.0)
    p.forward(ctx, out)
    assert ctx.status_sync() == api.STATUS_BAD_INDEX
    assert torch.all(out[torch.from_numpy(p.segments[3]).cuda()] == 7.0)
    p.backward(ctx)
    assert ctx.status_sync() == api.STATUS_BAD_INDEX
    p.seg.start.copy_(start)
    # longer than max_len said
    p.seg.max_len = 22
    out.fill_(7.0)
    p.forward(ctx, out)
    assert ctx.status_sync() == api.STATUS_TABLE_OVERFLOW
    assert torch.all(out[bad] == 7.0)
    ref.check(out.cpu()[torch.from_numpy(p.segments[0])], tuple(t[torch.from_numpy(p.segments[0])] for t in want["out"]), "first")
    p.backward(ctx)
    assert ctx.status_sync() == api.STATUS_TABLE_OVERFLOW


def test_nothing_to_do(ctx):
    """No voxels, no segments, a device count of none: outputs stay, the bias's gradient is zero."""
    p = Problem([20, 30], 4, 16, torch.bfloat16, seed=1)
    out = torch.full((p.n, 4, 16), 7.0, dtype=torch.bfloat16, device="cuda")
    for change in (dict(num=torch.zeros(1, dtype=torch.int32, device="cuda")), dict(start=p.seg.start[:1]),
                   dict(num=torch.full((1,), -3, dtype=torch.int32, device="cuda"))):
        seg = api.Segments(**{**dict(start=p.seg.start, max_len=30, order=p.seg.order, coords=p.seg.coords), **change})
        ctx.segment_attention(p.q, p.k, p.v, seg, bias=p.rel, out=out)
        grads = [torch.full_like(out, 7.0) for _ in range(3)]
        dbias = torch.full_like(p.rel.table, 9.0)
        ctx.segment_attention_backward(p.q, p.k, p.v, p.do, seg, bias=p.rel, out=grads, dbias=dbias)
        assert all(torch.all(t == 7.0) for t in [out] + grads) and torch.all(dbias == 0)
    e = torch.empty((0, 4, 16), dtype=torch.bfloat16, device="cuda")
    seg = api.Segments(torch.zeros(3, dtype=torch.int32, device="cuda"), 5)
    assert ctx.segment_attention(e, e, e, seg).shape == e.shape
    assert ctx.segment_attention_backward(e, e, e, e, seg)[0].shape == e.shape
    x = torch.empty((0, 24), device="cuda")
    assert ctx.layer_norm(x, None, None).shape == (0, 24)
    dx, dg, db = ctx.layer_norm_backward(x, x, None)
    assert torch.all(dg == 0) and torch.all(db == 0)
    # a device count below the capacity
    seg = api.Segments(p.seg.start, 30, p.seg.order, p.seg.coords, torch.ones(1, dtype=torch.int32, device="cuda"))
    out.fill_(7.0)
    ctx.segment_attention(p.q, p.k, p.v, seg, bias=p.rel, out=out)
    assert torch.all(out[torch.from_numpy(p.segments[1]).cuda()] == 7.0) and not torch.all(out == 7.0)
    assert ctx.status_sync() == 0


def test_many_heads_whose_statistics_take_several_passes(ctx):
    """More rows x heads of long segments than the workspace holds statistics of; heads whose gradients differ in size by far."""
    p = Problem([130] * 440, 32, 8, torch.bfloat16, seed=21, packed=False)
    p.host[3] = p.host[3] * torch.where(torch.arange(32) < 30, 1.0, 256.0).view(1, 32, 1).to(p.typ)
    p.do = p.host[3].contiguous().cuda()
    before = ctx.launch_count()
    *grads, dbias = p.backward(ctx)
    assert ctx.launch_count() - before > 4
    want, covered = p.want(back=True)
    for name, got in zip(("dq", "dk", "dv"), grads):
        ref.check(got, want[name], name)
    ref.check(dbias, want["dbias"], "dbias")
    # the bound counts the call's largest values for every head: of the heads with small ones too what their own allow
    got, (value, _) = dbias.double().cpu()[:30], want["dbias"]
    assert (got - value[:30]).norm() <= 1e-5 * value[:30].norm()
    assert ctx.status_sync() == 0


def test_same_inputs_same_bits(ctx):
    p = Problem([36, 20, 200, 1, 50, 300], 8, 24, torch.bfloat16, seed=8)
    first = [t.clone() for t in p.backward(ctx)]
    p.forward(ctx)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(p.backward(ctx), first))
    x = torch.randn((5000, 192), device="cuda")
    first = [t.clone() for t in ctx.layer_norm_backward(x, x, None)]
    assert all(torch.equal(a, b) for a, b in zip(ctx.layer_norm_backward(x, x, None), first))


def test_strides_beyond_32_bits(ctx):
    """Rows so far apart that their offsets pass 2^31 elements."""
    n, ld = 260, 9000000
    big = torch.empty((n - 1) * ld + 2 * 16, dtype=torch.bfloat16, device="cuda")
    far = lambda: big.as_strided((n, 2, 16), (ld, 16, 1))
    p = Problem([n - 40, 40], 2, 16, torch.bfloat16, seed=4, packed=False)
    plain = p.forward(ctx).clone()
    grads = [g.clone() for g in p.backward(ctx)]
    assert (n - 1) * ld > 2 ** 31
    for name in ("q", "k", "v"):
        was = getattr(p, name)
        far().copy_(was)
        setattr(p, name, far())
        assert torch.equal(p.forward(ctx), plain)
        assert all(torch.equal(a, b) for a, b in zip(p.backward(ctx), grads))
        setattr(p, name, was)
    p.forward(ctx, far())
    assert torch.equal(far().contiguous(), plain)
    small = [torch.empty_like(plain) for _ in range(3)]
    for i in range(3):
        p.backward(ctx, small[:i] + [far()] + small[i + 1:])
        assert torch.equal(far().contiguous(), grads[i])
    far().copy_(p.do)
    p.do = far()
    assert all(torch.equal(a, b) for a, b in zip(p.backward(ctx), grads))


def test_a_context_on_its_own_stream_and_captured_graphs():
    """Calls on a context whose stream is not the current one, captured and replayed with new inputs."""
    stream = torch.cuda.Stream()
    own = api.Context(2000, 64, 256, stream=stream)
    p = Problem([36, 20, 200, 1, 50], 8, 24, torch.bfloat16, seed=8, packed=False)
    x = torch.randn((307, 192), device="cuda")
    g, b = torch.randn(192, device="cuda"), torch.randn(192, device="cuda")
    out, y = torch.zeros_like(p.do), torch.zeros_like(x)
    grads = [torch.zeros_like(p.do) for _ in range(3)]
    dbias, dx, dg, db = torch.zeros_like(p.rel.table), torch.zeros_like(x), torch.zeros_like(g), torch.zeros_like(b)

    def step():
        own.segment_attention(p.q, p.k, p.v, p.seg, bias=p.rel, out=out)
        own.segment_attention_backward(p.q, p.k, p.v, p.do, p.seg, bias=p.rel, out=grads, dbias=dbias)
        own.layer_norm(x, g, b, out=y)
        own.layer_norm_backward(x, y, g, out=dx, dg=dg, db=db)

    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    results = []
    for seed in (1, 2):
        gen = torch.Generator("cuda").manual_seed(seed)
        for t in (p.q, p.k, p.v, p.do, x):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in (out, *grads, dbias, y, dx, dg, db)]
        for t in (out, *grads, dbias, y, dx, dg, db):
            t.zero_()
        torch.cuda.synchronize()
        step()
        stream.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(replayed, (out, *grads, dbias, y, dx, dg, db)))
        results.append(replayed)
    assert not torch.equal(results[0][0], results[1][0])
    assert own.status_sync() == 0
    del graph
    own.close()


def test_two_contexts_at_once():
    """Calls of two contexts, each with its stream and workspace, in flight together."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    own = [api.Context(3000, 64, 256, stream=s) for s in streams]
    problems = [Problem([36, 20, 200, 1, 50] * 5, 8, 24, torch.bfloat16, seed=i, packed=False) for i in range(2)]
    torch.cuda.synchronize()
    alone = []
    for c, p in zip(own, problems):
        with torch.cuda.stream(c.stream):
            alone.append([t.clone() for t in (p.forward(c), *p.backward(c))])
        torch.cuda.synchronize()
    for _ in range(5):
        together = []
        for c, p in zip(own, problems):
            with torch.cuda.stream(c.stream):
                together.append([p.forward(c), *p.backward(c)])
        torch.cuda.synchronize()
        for a, b in zip(alone, together):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
    for c in own:
        assert c.status_sync() == 0
        c.close()


def test_calls_in_turn_with_partitions_and_layers(ctx):
    """The workspace is the partition's: one leaves nothing behind that the other takes for its own."""
    g = torch.Generator().manual_seed(4)
    cells = torch.randperm(3600, generator=g)[:1200]
    coords = torch.stack([torch.zeros_like(cells), cells // 60, cells % 60, torch.zeros_like(cells)], 1).to(torch.int32).cuda()
    p = Problem([36, 200, 7], 8, 24, torch.bfloat16, seed=3)
    first = ctx.partition(coords, 1, (60, 60, 1), (12, 12, 1), 16, 0, extras=True)
    grads = [t.clone() for t in p.backward(ctx)]
    x = torch.randn((1200, 192), device="cuda")
    dx = [t.clone() for t in ctx.layer_norm_backward(x, x, None)]
    for _ in range(3):
        again = ctx.partition(coords, 1, (60, 60, 1), (12, 12, 1), 16, 0, extras=True)
        assert all(torch.equal(a, b) for a, b in zip(p.backward(ctx), grads))
        assert all(torch.equal(a, b) for a, b in zip(ctx.layer_norm_backward(x, x, None), dx))
        sets = int(first.num_sets.item())
        assert int(again.num_sets.item()) == sets and torch.equal(again.set_table[:sets], first.set_table[:sets])
        assert torch.equal(again.perm, first.perm) and torch.equal(again.win_start, first.win_start)
    assert ctx.status_sync() == 0


def test_refusals(ctx):
    lib, h = ctx.lib, ctx._h
    p = Problem([5, 6], 2, 16, torch.bfloat16, seed=1, packed=False)

    def call(change=None, out=p.do, ld=32, back=False, dbias=None, grads=None):
        prm = ctx._segment_params(p.q, p.k, p.v, p.seg, p.rel, 0.25, 0.0)
        for k, v in (change or {}).items():
            setattr(prm, k, v)
        if back:
            d = [torch.empty_like(p.do) for _ in range(3)] if grads is None else grads
            return lib.dsvt_segment_attention_backward(h, ctypes.byref(prm), out.data_ptr() if out is not None else None, ld, d[0].data_ptr(), 32,
                                                       d[1].data_ptr(), 32, d[2].data_ptr(), 32, dbias)
        return lib.dsvt_segment_attention(h, ctypes.byref(prm), out.data_ptr() if out is not None else None, ld)

    bad, capacity, unsupported = -1, -2, -3
    index = np.array(p.index)
    over = np.array(index)
    over[0] = 10000
    under = np.array(index)
    under[3] = -1
    cases = [(dict(n=-1), bad), (dict(heads=0), bad), (dict(head_dim=0), bad), (dict(type=3), bad), (dict(max_len=0), bad),
             (dict(cap=-1.0), bad), (dict(cap=math.nan), bad), (dict(cap=math.inf), bad), (dict(cap_segments=-1), bad), (dict(q=None), bad), (dict(k=p.k.data_ptr() + 2), bad),
             (dict(ld_q=31), bad), (dict(ld_v=36), bad), (dict(seg_start=None), bad), (dict(order=p.seg.order.data_ptr() + 1), bad),
             (dict(coords=None), bad), (dict(coords=p.seg.coords.data_ptr() + 4), bad), (dict(bucket_of=None), bad), (dict(buckets=0), bad),
             (dict(bucket_of=over.ctypes.data), bad), (dict(bucket_of=under.ctypes.data), bad), (dict(extent=(0, 1, 1)), bad),
             (dict(buckets=int(index[10] + 1)), bad), (dict(head_dim=12), unsupported), (dict(head_dim=136, ld_q=272, ld_k=272, ld_v=272), unsupported),
             (dict(buckets=1025), unsupported), (dict(extent=(129, 1, 1)), unsupported), (dict(n=70001), capacity)]
    for change, code in cases:
        assert call(change) == code, change
        assert call(change, back=True) == code, change
    assert call(out=None) == bad and call(out=p.q) == bad and call(ld=24) == bad and call(ld=33) == bad
    assert call(out=None, back=True) == bad and call(ld=8, back=True) == bad
    d = [torch.empty_like(p.do) for _ in range(2)]
    assert call(back=True, grads=[d[0], d[1], d[0]]) == bad and call(back=True, grads=[d[0], p.v, d[1]]) == bad
    assert call(dict(bias=None), back=True, dbias=p.rel.table.data_ptr()) == bad
    # what the binding refuses
    for kw in (dict(q=p.q.float()), dict(q=p.q[:5]), dict(k=p.k.transpose(1, 2)), dict(q=p.q.double(), k=p.k.double(), v=p.v.double())):
        a = {**dict(q=p.q, k=p.k, v=p.v), **kw}
        with pytest.raises(ValueError):
            ctx.segment_attention(a["q"], a["k"], a["v"], p.seg)
    with pytest.raises(ValueError):
        ctx.segment_attention(p.q, p.k, p.v, api.Segments(p.seg.start.long(), 6, p.seg.order))
    with pytest.raises(ValueError):
        ctx.segment_attention(p.q, p.k, p.v, api.Segments(p.seg.start, 6, p.seg.order[:4]))
    with pytest.raises(ValueError):
        ctx.segment_attention(p.q, p.k, p.v, api.Segments(p.seg.start, 6, p.seg.order), bias=p.rel)
    with pytest.raises(ValueError):
        ctx.segment_attention(p.q[:, :1], p.k[:, :1], p.v[:, :1], p.seg, bias=p.rel)
    x = torch.zeros((4, 8), device="cuda")
    X = x.data_ptr()
    for args, code in (((0, None, None, 4, 8, None, None, 1e-5, X), bad), ((0, X, None, 4, 8, None, None, 1e-5, None), bad),
                       ((5, X, None, 4, 8, None, None, 1e-5, X), bad), ((0, X, None, -1, 8, None, None, 1e-5, X), bad),
                       ((0, X, None, 4, 0, None, None, 1e-5, X), bad), ((0, X, None, 4, 8, None, None, -1.0, X), bad),
                       ((0, X, None, 4, 8, None, None, math.nan, X), bad), ((0, X + 4, None, 2, 8, None, None, 1e-5, X), bad),
                       ((0, X, X + 8, 2, 8, None, None, 1e-5, X), bad), ((0, X, None, 4, 8, X + 2, None, 1e-5, X), bad),
                       ((0, X, None, 4, 8193, None, None, 1e-5, X), unsupported)):
        assert lib.dsvt_layer_norm(h, *args) == code, args
    assert lib.dsvt_layer_norm_backward(h, 0, X, None, None, 4, 8, None, 1e-5, X, None, None) == bad
    assert lib.dsvt_layer_norm_backward(h, 0, X, None, X, 4, 8, None, 1e-5, X, X + 2, None) == bad
    with pytest.raises(ValueError):
        ctx.layer_norm(x, torch.zeros(7, device="cuda"), None)
    with pytest.raises(ValueError):
        ctx.layer_norm(x, None, None, residual=x.half())
    with pytest.raises(ValueError):
        ctx.layer_norm(x.double(), None, None)
    assert ctx.status_sync() == 0


# ---- LayerNorm ----------------------------------------------------------------------------------------------------
def _norm_problem(n, C, typ, residual, seed, offset=0.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((n, C), generator=g) + offset).to(typ)
    r = (0.5 * torch.randn((n, C), generator=g)).to(typ) if residual else None
    dy = torch.randn((n, C), generator=g).to(typ)
    return x, r, dy, 1 + 0.2 * torch.randn(C, generator=g), torch.randn(C, generator=g)


@pytest.mark.parametrize("typ", TYPES)
@pytest.mark.parametrize("n,C", [(1, 1), (3, 2), (5, 4), (1, 192), (1000, 192), (257, 128), (64, 96), (300, 20), (77, 250), (31, 333), (9, 513),
                                 (40, 1024), (21, 1028), (6, 2047), (11, 4096), (5, 8191), (3, 8192), (4000, 64), (20011, 48)])
def test_layer_norm(ctx, typ, n, C):
    residual = (n + C) % 2 == 0
    x, r, dy, g, b = _norm_problem(n, C, typ, residual, n + C)
    dev = lambda t: None if t is None else t.cuda()
    wide = lambda t: None if t is None else t.double()
    y = ctx.layer_norm(dev(x), dev(g), dev(b), residual=dev(r), eps=1e-3)
    ref.check(y, ref.layer_norm(wide(x), wide(r), wide(g), wide(b), 1e-3, eps=EPS[typ]), "y")
    dx, dg, db = ctx.layer_norm_backward(dev(x), dev(dy), dev(g), residual=dev(r), eps=1e-3)
    want = ref.layer_norm(wide(x), wide(r), wide(g), wide(b), 1e-3, wide(dy), eps=EPS[typ])
    for name, got in (("dx", dx), ("dg", dg), ("db", db)):
        ref.check(got, want[name], name)


@pytest.mark.parametrize("typ", TYPES)
def test_layer_norm_without_weights_in_place_and_with_an_offset(ctx, typ):
    x, r, dy, _, _ = _norm_problem(700, 192, typ, True, 5, offset=8.0)
    one, none = torch.ones(192, dtype=torch.float64), torch.zeros(192, dtype=torch.float64)
    want = ref.layer_norm(x.double(), r.double(), one, none, 1e-5, eps=EPS[typ])
    for at in ("x", "r", None):
        xd, rd = x.cuda(), r.cuda()
        got = ctx.layer_norm(xd, None, None, residual=rd, out={"x": xd, "r": rd, None: None}[at])
        ref.check(got, want, "y in %s" % at)
    want = ref.layer_norm(x.double(), r.double(), one, none, 1e-5, dy.double(), eps=EPS[typ])
    for at in ("x", "r", "dy"):
        t = dict(x=x.cuda(), r=r.cuda(), dy=dy.cuda())
        for name, got in zip(("dx", "dg", "db"), ctx.layer_norm_backward(t["x"], t["dy"], None, residual=t["r"], out=t[at])):
            ref.check(got, want[name], "%s in %s" % (name, at))


def test_layer_norm_on_another_stream_than_the_current_one(ctx):
    """A context's calls run on its own stream, whatever the current one is; waiting for that stream is enough."""
    own = api.Context(1000, 1, 256, stream=torch.cuda.Stream())
    x = torch.randn((1000, 192), device="cuda")
    torch.cuda.synchronize()
    y = own.layer_norm(x, None, None)
    own.stream.synchronize()
    assert torch.equal(y, ctx.layer_norm(x, None, None))
    own.close()


def test_layer_norm_rows_that_are_not_finite_or_constant(ctx):
    x = torch.randn((50, 192), device="cuda")
    clean = ctx.layer_norm(x, None, None)
    x[7, 3], x[9, 0], x[11] = math.nan, math.inf, 2.5
    y = ctx.layer_norm(x, None, None, eps=1e-5)
    rest = [i for i in range(50) if i not in (7, 9, 11)]
    assert torch.equal(y[rest], clean[rest])
    assert torch.isnan(y[7]).all() and torch.isnan(y[9]).any()
    assert torch.equal(y[11], torch.zeros(192, device="cuda"))
    # eps of zero: rows beyond the last one of a group add nothing
    dx, dg, db = ctx.layer_norm_backward(x[:3].contiguous(), x[:3].contiguous(), None, eps=0.0)
    assert torch.isfinite(dx).all() and torch.isfinite(dg).all()


# ---- together ---------------------------------------------------------------------------------------------------
def test_a_training_step_of_a_layers_attention_half(ctx):
    """x1 = LN(x + W_o attend(W_qkv x)): the operators between torch's products against float64 differentiation of the whole."""
    p = Problem([36, 20, 1, 30, 150], 4, 24, torch.float32, seed=12, packed=False)
    n, C = p.n, 96
    g = torch.Generator().manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=g)
    x, dy = rnd(n, C), rnd(n, C)
    Wqkv, Wo, gam, bet = rnd(3 * C, C) / C ** 0.5, rnd(C, C) / C ** 0.5, 1 + 0.1 * rnd(C), rnd(C)
    xd, Wq, Wod, gd, bd, dyd = (t.cuda() for t in (x, Wqkv, Wo, gam, bet, dy))
    qkv = (xd @ Wq.t()).view(n, 3, 4, 24)
    q, k, v = qkv.unbind(1)
    att = ctx.segment_attention(q, k, v, p.seg, bias=p.rel, cap=5.0)
    a = att.view(n, C) @ Wod.t()
    y = ctx.layer_norm(a, gd, bd, residual=xd)
    du, dgam, dbet = ctx.layer_norm_backward(a, dyd, gd, residual=xd)
    datt = (du @ Wod).view(n, 4, 24)
    dqkv = torch.empty_like(qkv)
    _, _, _, dbias = ctx.segment_attention_backward(q, k, v, datt, p.seg, bias=p.rel, cap=5.0, out=dqkv.unbind(1))
    dx = du + dqkv.view(n, 3 * C) @ Wq
    got = dict(y=y, x=dx, Wqkv=dqkv.view(n, 3 * C).t() @ xd, Wo=du.t() @ att.view(n, C), gam=dgam, bet=dbet, bias=dbias)

    leaves = {m: t.double().requires_grad_() for m, t in (("x", x), ("Wqkv", Wqkv), ("Wo", Wo), ("gam", gam), ("bet", bet), ("bias", p.table))}
    w = (leaves["x"] @ leaves["Wqkv"].t()).view(n, 3, 4, 24)
    rows, places = [], []
    for ids in p.segments:
        i = torch.from_numpy(ids)
        s = 5.0 * torch.tanh(torch.einsum("ihd,jhd->hij", w[i, 0], w[i, 1]) * 24 ** -0.5 / 5.0)
        s = s + leaves["bias"][:, torch.from_numpy(p.buckets(ids))]
        rows.append(torch.einsum("hij,jhd->ihd", torch.softmax(s, 2), w[i, 2]))
        places.append(i)
    whole = torch.zeros((n, 4, 24), dtype=torch.float64).index_copy(0, torch.cat(places), torch.cat(rows))
    out = torch.nn.functional.layer_norm(leaves["x"] + whole.reshape(n, C) @ leaves["Wo"].t(), (C,), leaves["gam"], leaves["bet"], 1e-5)
    grads = dict(zip(leaves, torch.autograd.grad(out, list(leaves.values()), dy.double())))
    grads["y"] = out
    for name, value in got.items():
        want = grads[name].detach()
        # five chained fp32 products of up to 237 terms and a softmax: each off by at most (terms + 8) u of its terms' magnitudes, which
        # are at most 30 times the result's root mean square here
        bound = 5 * (237 + 8) * ref.U * 30 * want.square().mean().sqrt()
        err = (value.double().cpu() - want).abs().max()
        assert err <= bound, (name, float(err), float(bound))
    # and against differences of the function along a direction
    step = 1e-5

    def loss(table):
        total = 0.0
        for ids in p.segments:
            i = torch.from_numpy(ids)
            s = 5.0 * torch.tanh(torch.einsum("ihd,jhd->hij", w[i, 0], w[i, 1]) * 24 ** -0.5 / 5.0) + table[:, torch.from_numpy(p.buckets(ids))]
            total = total + (torch.einsum("hij,jhd->ihd", torch.softmax(s, 2), w[i, 2]) * datt.double().cpu()[i]).sum()
        return float(total)

    with torch.no_grad():
        way = rnd(*p.table.shape).double()
        slope = (loss(leaves["bias"].detach() + step * way) - loss(leaves["bias"].detach() - step * way)) / (2 * step)
    size = float((dbias.double().cpu().abs() * way.abs()).sum())
    assert abs(slope - float((dbias.double().cpu() * way).sum())) <= 1e-4 * size
    assert ctx.status_sync() == 0
