"""The training operators without a GPU: bucket tables, argument checks that need no device, and the float64 definitions that the
kernels are held to against differences of the function itself."""
import ctypes
import math

import numpy as np
import pytest
import torch

import train_reference as ref
from paper_2301_06051_b200 import api


def test_log_buckets_are_exact_near_and_shared_far():
    index, count = api.log_buckets((12, 12, 1), (3, 3, 1), (6, 6, 1))
    assert count == 11 * 11 and index.shape == (23 + 23 + 1,) and index.dtype == np.int32
    x, y, z = index[:23], index[23:46], index[46:]
    assert list(z) == [0]
    assert list(y) == sorted(y) and y[0] == 0 and y[-1] == 10 and y[11] == 5
    assert list(y[9:14]) == [3, 4, 5, 6, 7]  # -2 ... 2 have buckets of their own
    assert y[8] < 3 and y[14] > 7
    assert np.array_equal(x, 11 * y)
    total = x[:, None, None] + y[None, :, None] + z[None, None, :]
    assert total.min() == 0 and total.max() == count - 1


@pytest.mark.parametrize("extent,near,sides", [((1, 1, 1), (1, 1, 1), (1, 1, 1)), ((30, 30, 1), (3, 3, 1), (7, 7, 1)),
                                               ((12, 12, 32), (3, 3, 2), (5, 5, 4)), ((4, 5, 6), (4, 5, 6), (4, 5, 6))])
def test_log_buckets_stay_in_range_and_mirror(extent, near, sides):
    index, count = api.log_buckets(extent, near, sides)
    at, spans = 0, []
    for e in extent:
        part = index[at:at + 2 * e - 1]
        assert np.all(np.diff(part) >= 0)
        assert np.array_equal(part + part[::-1], np.full(2 * e - 1, 2 * part[e - 1]))  # a displacement and its opposite
        spans.append((part.min(), part.max()))
        at += 2 * e - 1
    assert sum(s[0] for s in spans) >= 0 and sum(s[1] for s in spans) < count


def test_log_buckets_refuses_bad_axes():
    for args in (((0, 1, 1), (1, 1, 1), (1, 1, 1)), ((4, 4, 4), (0, 1, 1), (2, 2, 2)), ((4, 4, 4), (3, 1, 1), (2, 2, 2))):
        with pytest.raises(ValueError):
            api.log_buckets(*args)


def test_bucket_bias_and_segments_refuse_what_does_not_fit():
    table = torch.zeros((2, 9))
    api.BucketBias(table, (2, 2, 1), np.zeros(7))
    with pytest.raises(ValueError):
        api.BucketBias(table, (2, 2, 1), np.zeros(8))
    with pytest.raises(ValueError):
        api.BucketBias(table.double(), (2, 2, 1), np.zeros(7))
    with pytest.raises(ValueError):
        api.BucketBias(table, (2, 2), np.zeros(6))
    t = api.SetTable(torch.zeros((4, 3), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(20, dtype=torch.int32), 4, 3)
    with pytest.raises(ValueError):
        api.Segments.of_sets(t)
    with pytest.raises(ValueError):
        api.Segments.of_windows(t, 9)
    t.perm = torch.zeros(5, dtype=torch.int32)
    seg = api.Segments.of_sets(t)
    assert seg.start.numel() == 5 and seg.max_len == 3 and seg.num is t.num_sets


def test_a_null_context_is_an_error():
    lib = api.load()
    p = api.SegmentAttentionParams()
    assert lib.dsvt_segment_attention(None, ctypes.byref(p), None, 0) == -1
    assert lib.dsvt_segment_attention_backward(None, ctypes.byref(p), None, 0, None, 0, None, 0, None, 0, None) == -1
    assert lib.dsvt_layer_norm(None, 0, None, None, 0, 1, None, None, 1e-5, None) == -1
    assert lib.dsvt_layer_norm_backward(None, 0, None, None, None, 0, 1, None, 1e-5, None, None, None) == -1


def _problem(lens, heads, dim, cap, seed):
    g = torch.Generator().manual_seed(seed)
    n = sum(lens) + 2
    q, k, v, do = (torch.randn((n, heads, dim), generator=g, dtype=torch.float64) for _ in range(4))
    order = torch.randperm(n, generator=g).numpy()
    at = np.concatenate([[1], 1 + np.cumsum(lens)])
    segments = [order[at[i]:at[i + 1]] for i in range(len(lens))]
    cells = torch.randint(0, 5, (n, 3), generator=g).numpy()
    extent = (4, 4, 3)  # (cells lie farther apart than the extent here: displacements are clipped)
    index, count = api.log_buckets(extent, (2, 2, 1), (3, 3, 2))
    bias = torch.randn((heads, count), generator=g, dtype=torch.float64)
    buckets = lambda ids: ref.bucket_index(cells[ids], cells[ids], extent, index)
    return q, k, v, do, segments, bias, buckets


@pytest.mark.parametrize("cap", [0.0, 3.0])
def test_the_gradients_formulas_match_differences(cap):
    q, k, v, do, segments, bias, buckets = _problem([1, 4, 0, 7], 2, 8, cap, 3)
    scale = 8 ** -0.5

    def loss(q, k, v, bias):
        out, covered = ref.attention(q, k, v, segments, scale, cap, bias, buckets)
        return float((out["out"][0] * do)[covered].sum())

    grads, _ = ref.attention(q, k, v, segments, scale, cap, bias, buckets, d_out=do)
    g = torch.Generator().manual_seed(5)
    step = 1e-5
    for name, at in (("dq", 0), ("dk", 1), ("dv", 2), ("dbias", 3)):
        inputs = [q, k, v, bias]
        way = torch.randn(inputs[at].shape, generator=g, dtype=torch.float64)
        ends = []
        for sign in (1, -1):
            moved = list(inputs)
            moved[at] = inputs[at] + sign * step * way
            ends.append(loss(*moved))
        slope = (ends[0] - ends[1]) / (2 * step)
        assert abs(slope - float((grads[name][0] * way).sum())) <= 1e-7 * max(1.0, abs(slope)), name


def test_a_row_without_keys_gives_zeros_and_the_lowest_float_equal_weights():
    q, k, v, do, segments, bias, buckets = _problem([5], 2, 8, 0.0, 4)
    out, covered = ref.attention(q, k, v, segments, 1.0, 0.0, torch.full_like(bias, -math.inf), buckets)
    assert torch.equal(out["out"][0], torch.zeros_like(v))
    low = torch.full_like(bias, float(np.finfo(np.float32).min))
    out, _ = ref.attention(q, k, v, segments, 1.0, 0.0, low, buckets)
    assert torch.allclose(out["out"][0][segments[0]], v[segments[0]].mean(0).expand(5, -1, -1), atol=1e-14)


def test_layer_norms_formulas_match_differences():
    g = torch.Generator().manual_seed(6)
    n, C = 5, 7
    x, r, dy = (torch.randn((n, C), generator=g, dtype=torch.float64) for _ in range(3))
    w, b = torch.randn(C, generator=g, dtype=torch.float64), torch.randn(C, generator=g, dtype=torch.float64)
    got = ref.layer_norm(x, r, w, b, 1e-5, dy)
    step = 1e-6
    for name, at in (("dx", 0), ("dg", 1), ("db", 2)):
        inputs = [x, w, b]
        way = torch.randn(inputs[at].shape, generator=g, dtype=torch.float64)
        ends = []
        for sign in (1, -1):
            moved = list(inputs)
            moved[at] = inputs[at] + sign * step * way
            ends.append(float((ref.layer_norm(moved[0], r, moved[1], moved[2], 1e-5)[0] * dy).sum()))
        slope = (ends[0] - ends[1]) / (2 * step)
        assert abs(slope - float((got[name][0] * way).sum())) <= 1e-7 * max(1.0, abs(slope)), name
