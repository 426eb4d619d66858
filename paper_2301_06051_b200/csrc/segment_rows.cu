// Segment attention, a warp to a row and head: the plain kernels.
#include <float.h>

#include "segment.cuh"

namespace dsvt_train {
namespace {

constexpr int kThreads = 256;
constexpr unsigned kAll = 0xffffffffu;

__device__ __forceinline__ float warp_sum(float v) {
  for (int m = 16; m > 0; m >>= 1) v += __shfl_xor_sync(kAll, v, m);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
  for (int m = 16; m > 0; m >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, m));
  return v;
}

template <typename T>
__device__ __forceinline__ float dot(const T* x, const T* y, int dim) {
  float s = 0.f;
  for (int c = 0; c < dim; ++c) s = fmaf(to_float(x[c]), to_float(y[c]), s);
  return s;
}

// The score of voxels i and j (natural units), its bucket and the derivative of the cap.
template <typename T>
__device__ __forceinline__ float score(const SegArgs& a, int h, int i, int j, int* bucket, float* slope) {
  float z = a.scale * dot((const T*)a.q + i * a.ld_q + h * a.dim, (const T*)a.k + j * a.ld_k + h * a.dim, a.dim);
  *slope = 1.f;
  if (a.cap > 0.f) {
    const float t = tanhf(z / a.cap);
    z = a.cap * t;
    *slope = 1.f - t * t;
  }
  *bucket = 0;
  if (a.bias) {
    const int4 p = a.coords[i], r = a.coords[j];
    *bucket = bucket_of(a.maps, p.y - r.y, p.z - r.z, p.w - r.w);
    z += a.bias[h * a.buckets + *bucket];
  }
  return z;
}

// Rows (or, in the second backward pass, keys) of the segments, one to a warp.
template <typename T, int PASS>  // 0 forward, 1 dq and statistics, 2 dk, dv and dbias
__global__ void __launch_bounds__(kThreads) rows_kernel(const SegArgs a, float* stats) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = kThreads / 32;
  const int h = blockIdx.y;
  const int count = segment_count(a);
  for (int s = blockIdx.x; s < count; s += gridDim.x) {
    const int lo = a.seg_start[s], hi = a.seg_start[s + 1];
    if (!segment_sound(a, lo, hi)) continue;
    for (int row = lo + warp; row < hi; row += warps) {
      const int i = voxel_at(a, row);
      if (i < 0) continue;
      float acc[2][kMaxDim / 32] = {};
      if (PASS < 2) {
        float m = -INFINITY, l = 0.f, D = 0.f, inv = 0.f;
        int b;
        float slope;
        for (int j0 = lo; j0 < hi; j0 += 32) {
          const int j = j0 + lane < hi ? voxel_at(a, j0 + lane) : -1;
          if (j >= 0) m = fmaxf(m, score<T>(a, h, i, j, &b, &slope));
        }
        m = warp_max(m);
        const float base = m == -INFINITY ? 0.f : m;
        for (int pass = 0; pass < (PASS == 0 ? 2 : 3); ++pass) {
          for (int j0 = lo; j0 < hi; j0 += 32) {
            const int j = j0 + lane < hi ? voxel_at(a, j0 + lane) : -1;
            const float sc = j >= 0 ? score<T>(a, h, i, j, &b, &slope) : -INFINITY;
            float p = expf(sc - base), w;
            if (pass == 0) { l += p; continue; }
            p *= inv;
            if (PASS == 0) {
              w = p;
            } else {
              const float dp = j >= 0 ? dot((const T*)a.d_out + i * a.ld_do + h * a.dim, (const T*)a.v + j * a.ld_v + h * a.dim, a.dim) : 0.f;
              if (pass == 1) { if (j >= 0) D = fmaf(p, dp, D); continue; }
              w = a.scale * p * (dp - D) * slope;
            }
            const T* other = PASS == 0 ? (const T*)a.v : (const T*)a.k;
            const int64_t ld = PASS == 0 ? a.ld_v : a.ld_k;
            for (int t = 0; t < 32; ++t) {
              const int jt = __shfl_sync(kAll, j, t);
              const float wt = __shfl_sync(kAll, w, t);
              if (jt >= 0)
                for (int c = lane, e = 0; c < a.dim; c += 32, ++e) acc[0][e] = fmaf(wt, to_float(other[jt * ld + h * a.dim + c]), acc[0][e]);
            }
          }
          if (pass == 0) { l = warp_sum(l); inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l); }
          if (PASS == 1 && pass == 1) D = warp_sum(D);
        }
        T* to = PASS == 0 ? (T*)a.out + i * a.ld_out : (T*)a.dq + i * a.ld_dq;
        for (int c = lane, e = 0; c < a.dim; c += 32, ++e) to[h * a.dim + c] = from_float<T>(acc[0][e]);
        if (PASS == 1 && lane == 0) {
          float* st = stats + ((int64_t)row * a.heads + h) * 3;
          st[0] = base; st[1] = inv; st[2] = D;
        }
      } else {  // i is the key; lanes are queries
        for (int j0 = lo; j0 < hi; j0 += 32) {
          const int j = j0 + lane < hi ? voxel_at(a, j0 + lane) : -1;
          float p = 0.f, ds = 0.f;
          if (j >= 0) {
            int b;
            float slope;
            const float* st = stats + ((int64_t)(j0 + lane) * a.heads + h) * 3;
            p = expf(score<T>(a, h, j, i, &b, &slope) - st[0]) * st[1];
            ds = p * (dot((const T*)a.d_out + j * a.ld_do + h * a.dim, (const T*)a.v + i * a.ld_v + h * a.dim, a.dim) - st[2]);
            if (a.dbias) atomicAdd(a.dbias + h * a.buckets + b, ds);
            ds *= slope * a.scale;
          }
          for (int t = 0; t < 32; ++t) {
            const int jt = __shfl_sync(kAll, j, t);
            const float pt = __shfl_sync(kAll, p, t), dt = __shfl_sync(kAll, ds, t);
            if (jt >= 0)
              for (int c = lane, e = 0; c < a.dim; c += 32, ++e) {
                acc[0][e] = fmaf(dt, to_float(((const T*)a.q)[jt * a.ld_q + h * a.dim + c]), acc[0][e]);
                acc[1][e] = fmaf(pt, to_float(((const T*)a.d_out)[jt * a.ld_do + h * a.dim + c]), acc[1][e]);
              }
          }
        }
        for (int c = lane, e = 0; c < a.dim; c += 32, ++e) {
          ((T*)a.dk)[i * a.ld_dk + h * a.dim + c] = from_float<T>(acc[0][e]);
          ((T*)a.dv)[i * a.ld_dv + h * a.dim + c] = from_float<T>(acc[1][e]);
        }
      }
    }
  }
}

}  // namespace

template <typename T>
int launch_backward(dsvt_ctx* ctx, const SegArgs& a) {
  if ((int64_t)a.n * a.heads * 3 > (int64_t)(4 * ctx->bm_words)) return DSVT_ERR_CAPACITY;
  float* stats = reinterpret_cast<float*>(ctx->bm_zero);
  const int blocks = a.cap_segments < 16 * ctx->sm_count ? a.cap_segments : 16 * ctx->sm_count;
  if (a.dbias) DSVT_CUDA_TRY(ctx, cudaMemsetAsync(a.dbias, 0, (size_t)a.heads * a.buckets * sizeof(float), ctx->stream));
  rows_kernel<T, 1><<<dim3(blocks, a.heads), kThreads, 0, ctx->stream>>>(a, stats);
  DSVT_LAUNCHED(ctx);
  rows_kernel<T, 2><<<dim3(blocks, a.heads), kThreads, 0, ctx->stream>>>(a, stats);
  DSVT_LAUNCHED(ctx);
  return DSVT_OK;
}

template int launch_backward<float>(dsvt_ctx*, const SegArgs&);
template int launch_backward<__nv_bfloat16>(dsvt_ctx*, const SegArgs&);
template int launch_backward<__half>(dsvt_ctx*, const SegArgs&);

}  // namespace dsvt_train
