// Segment attention: the call as its kernels see it, and the launchers.
#pragma once
#include <type_traits>

#include "train_types.cuh"

namespace dsvt_train {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxExtent = 128, kMaxBuckets = 1024, kMaxDim = 128, kMaxHeads = 65535;
constexpr int64_t kMaxBiasTable = 1 << 18;  // entries of a bias whose gradient is asked for: what the workspace has room for

// The additive bucket indexes of the displacements along x, y and z: at [0, 2L-1), [at_y, at_y + 2W-1), [at_z, ...).
struct BucketMaps {
  int32_t extent[3], at_y, at_z;
  uint16_t of[3 * (2 * kMaxExtent - 1)];
};

struct SegArgs {
  const void *q, *k, *v, *d_out;
  void *out, *dq, *dk, *dv;  // (out: the forward pass)
  int64_t ld_q, ld_k, ld_v, ld_do, ld_out, ld_dq, ld_dk, ld_dv;
  const int32_t *order, *seg_start, *num_segments;
  const int4* coords;
  const float* bias;  // [heads][buckets] or NULL
  float* dbias;       // or NULL
  int32_t n, heads, dim, cap_segments, max_len, buckets;
  float scale, cap;
  int32_t* status;
  BucketMaps maps;
};

__device__ __forceinline__ int segment_count(const SegArgs& a) {
  int s = a.cap_segments;
  if (a.num_segments) { const int m = *a.num_segments; s = m < s ? (m < 0 ? 0 : m) : s; }
  return s;
}

// Whether rows [lo, hi) are a segment to work on; what is wrong with one that is not goes to the status word.
__device__ __forceinline__ bool segment_sound(const SegArgs& a, int lo, int hi) {
  if (lo < 0 || hi < lo || hi > a.n) { atomicOr(a.status, DSVT_STATUS_BAD_INDEX); return false; }
  if (hi - lo > a.max_len) { atomicOr(a.status, DSVT_STATUS_TABLE_OVERFLOW); return false; }
  return hi > lo;
}

// The voxel at a place of the order, or -1.
__device__ __forceinline__ int voxel_at(const SegArgs& a, int row) {
  if (!a.order) return row;
  const int v = a.order[row];
  if ((unsigned)v < (unsigned)a.n) return v;
  atomicOr(a.status, DSVT_STATUS_BAD_INDEX);
  return -1;
}

template <typename T>
int launch_forward(dsvt_ctx* ctx, const SegArgs& a);
template <typename T>
int launch_backward(dsvt_ctx* ctx, const SegArgs& a);

}  // namespace dsvt_train
