// Segment attention on the tensor cores: tiles of 16 rows times the rows of a chunk, operands in shared memory.
//
// Two products carry every pass.  scores(): C[16][cols] = A B^T over the channels (q k^T, do v^T and their transposes); weigh():
// acc[16][dim] += W B, where W is a result of scores() in registers (p v, dz k, ...).  A score tile's accumulator layout is the
// next product's operand layout, so W never leaves the registers; and since a pass exists for either side of the score matrix, none
// is ever transposed.
//
// mma.sync and not tcgen05: a segment has a few dozen to a thousand rows and a head 16 to 64 channels, so that a score takes 2 dim
// multiply-adds beside a table look-up, an exponential and some 45 (forward) to 110 (backward, by queries) instructions in all.  m16n8k16 runs at 556 TFLOP/s here (1.1 ns an
// instruction and SM); the tile's look-ups in shared memory take longer than its products (dim 24: 3.9 ns of products beside 5.2 ns of
// look-ups).  Tiles of 128 rows in TMEM would leave most of their rows empty in sets of 36 and add a round trip to each score.
//
// 16-bit types: products exact, sums fp32, W rounded to the type: half of the tensor cores' products, for an error that the result's own
// rounding covers (2-norm against float64: 32,000 pillars bf16 2.0e-3, where rounding the exact result alone leaves 1.7e-3; their
// gradients 2.4e-3 and 1.7e-3; float16 2.5e-4 and 2.1e-4).  For float16's gradients W goes in as tf32 (same 11 bits, but
// float's range: dz of large gradients passes 65504), and the other operand, exact in tf32, with it.
// fp32: both operands as two tf32 parts x = hi + lo (each rounded: |x - hi - lo| <= 2^-22 |x|); hi hi, hi lo and lo hi are formed,
// lo lo (2^-22) is left out (2.1e-7 against 1.9e-7 of plain fp32, gradients of 12,345 capped pillars).  The tensor cores truncate when they add, so the small products have accumulators of their own and a
// chunk's sums meet the running ones in additions that round.
#pragma once
#include "segment.cuh"
#include "tc_ptx.cuh"

namespace dsvt_train {

constexpr unsigned kAll = 0xffffffffu;

using dsvt_tc::ex2_approx;
using dsvt_tc::smem_u32;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool real) {
  const int size = real ? 16 : 0;  // (nothing read: zeros)
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(size) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm2(uint32_t& r0, uint32_t& r1, uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.shared.b16 {%0,%1}, [%2];" : "=r"(r0), "=r"(r1) : "r"(a) : "memory");
}
__device__ __forceinline__ uint32_t ldsm1(uint32_t a) {
  uint32_t r;
  asm volatile("ldmatrix.sync.aligned.m8n8.x1.shared.b16 {%0}, [%1];" : "=r"(r) : "r"(a) : "memory");
  return r;
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm2_t(uint32_t& r0, uint32_t& r1, uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0,%1}, [%2];" : "=r"(r0), "=r"(r1) : "r"(a) : "memory");
}
__device__ __forceinline__ float lds(uint32_t a) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}

// c += a b; FRESH: c = a b.
#define DSVT_MMA(NAME, SHAPE, TYPE, ARGS, A, B, ...)                                                                                  \
  template <bool FRESH>                                                                                                               \
  __device__ __forceinline__ void NAME(float (&c)[4], ARGS) {                                                                         \
    if (FRESH)                                                                                                                        \
      asm("mma.sync.aligned." SHAPE ".row.col.f32." TYPE "." TYPE ".f32 {%0,%1,%2,%3}, {" A "}, {" B "}, {%4,%4,%4,%4};"      \
                   : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "f"(0.f), __VA_ARGS__);                                         \
    else                                                                                                                              \
      asm("{.reg .f32 z; mov.f32 z, %4; mma.sync.aligned." SHAPE ".row.col.f32." TYPE "." TYPE ".f32 {%0,%1,%2,%3}, {" A "}, {" B "}, {%0,%1,%2,%3};}" \
                   : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "f"(0.f), __VA_ARGS__);                                         \
  }
#define DSVT_COMMA ,
#define DSVT_MMA_K16(NAME, SHAPE, TYPE)                                                                                                \
  DSVT_MMA(NAME, SHAPE, TYPE, uint32_t a0 DSVT_COMMA uint32_t a1 DSVT_COMMA uint32_t a2 DSVT_COMMA uint32_t a3 DSVT_COMMA uint32_t b0 DSVT_COMMA uint32_t b1, \
           "%5,%6,%7,%8", "%9,%10", "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1))
#define DSVT_MMA_K8(NAME, SHAPE, TYPE) \
  DSVT_MMA(NAME, SHAPE, TYPE, uint32_t a0 DSVT_COMMA uint32_t a1 DSVT_COMMA uint32_t b0, "%5,%6", "%7", "r"(a0), "r"(a1), "r"(b0))
DSVT_MMA_K16(mma_bf16, "m16n8k16", "bf16")
DSVT_MMA_K8(mma_bf16_k8, "m16n8k8", "bf16")
DSVT_MMA_K16(mma_f16, "m16n8k16", "f16")
DSVT_MMA_K8(mma_f16_k8, "m16n8k8", "f16")
DSVT_MMA_K16(mma_tf32, "m16n8k8", "tf32")
__device__ __forceinline__ uint32_t tf32(float v) {
  uint32_t r;
  asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(r) : "f"(v));
  return r;
}
struct Parts { uint32_t hi, lo; };
__device__ __forceinline__ Parts split(float v) {
  Parts p;
  p.hi = tf32(v);
  p.lo = tf32(v - __uint_as_float(p.hi));
  return p;
}

template <typename T>
struct Mma;
template <>
struct Mma<__nv_bfloat16> {
  template <bool FRESH>
  static __device__ __forceinline__ void k16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) { mma_bf16<FRESH>(c, a0, a1, a2, a3, b0, b1); }
  template <bool FRESH>
  static __device__ __forceinline__ void k8(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t b0) { mma_bf16_k8<FRESH>(c, a0, a1, b0); }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return dsvt_tc::pack_bf16(lo, hi); }
};
template <>
struct Mma<__half> {
  template <bool FRESH>
  static __device__ __forceinline__ void k16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) { mma_f16<FRESH>(c, a0, a1, a2, a3, b0, b1); }
  template <bool FRESH>
  static __device__ __forceinline__ void k8(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t b0) { mma_f16_k8<FRESH>(c, a0, a1, b0); }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};

// DT of 16, 24 and 32 are the channels of a head; 64 and 128 take any multiple of 8 up to them.
template <int DT>
constexpr bool kExact = DT <= 32;

// One step of scores(): channels k * 16 (fp32: k * 8) on.
template <typename T, int NT, bool FRESH>
__device__ __forceinline__ void scores_k16(float (&c)[NT][4], uint32_t ra, uint32_t rb, uint32_t rl, uint32_t pitch) {
  uint32_t f[4];
  ldsm4(f, ra);
#pragma unroll
  for (int p = 0; p < NT / 2; ++p) {
    uint32_t g[4];
    ldsm4(g, rb + p * 16 * pitch);
    Mma<T>::template k16<FRESH>(c[2 * p], f[0], f[1], f[2], f[3], g[0], g[1]);
    Mma<T>::template k16<FRESH>(c[2 * p + 1], f[0], f[1], f[2], f[3], g[2], g[3]);
  }
  if (NT & 1) {
    uint32_t g0, g1;
    ldsm2(g0, g1, rl);
    Mma<T>::template k16<FRESH>(c[NT - 1], f[0], f[1], f[2], f[3], g0, g1);
  }
}
template <typename T, int NT, bool FRESH>
__device__ __forceinline__ void scores_k8(float (&c)[NT][4], uint32_t a, uint32_t b, uint32_t pitch) {
  const int lane = threadIdx.x & 31;
  uint32_t f0, f1;
  ldsm2(f0, f1, a + (lane & 15) * pitch);
#pragma unroll
  for (int p = 0; p < NT / 4; ++p) {
    uint32_t g[4];
    ldsm4(g, b + (p * 32 + lane) * pitch);
#pragma unroll
    for (int i = 0; i < 4; ++i) Mma<T>::template k8<FRESH>(c[4 * p + i], f0, f1, g[i]);
  }
  if (NT & 2) {
    uint32_t g0, g1;
    ldsm2(g0, g1, b + (NT / 4 * 32 + (lane & 15)) * pitch);
    Mma<T>::template k8<FRESH>(c[NT / 4 * 4], f0, f1, g0);
    Mma<T>::template k8<FRESH>(c[NT / 4 * 4 + 1], f0, f1, g1);
  }
  if (NT & 1) Mma<T>::template k8<FRESH>(c[NT - 1], f0, f1, ldsm1(b + ((NT - 1) * 8 + (lane & 7)) * pitch));
}
template <int NT, bool FRESH>
__device__ __forceinline__ void scores_tf32(float (&c)[NT][4], float (&s)[NT][4], uint32_t ra, uint32_t rb, uint32_t pitch) {
  Parts f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = split(lds(ra + (i & 1) * 8 * pitch + (i >> 1) * 16));
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const Parts g0 = split(lds(rb + t * 8 * pitch)), g1 = split(lds(rb + t * 8 * pitch + 16));
    mma_tf32<FRESH>(s[t], f[0].lo, f[1].lo, f[2].lo, f[3].lo, g0.hi, g1.hi);
    mma_tf32<false>(s[t], f[0].hi, f[1].hi, f[2].hi, f[3].hi, g0.lo, g1.lo);
    mma_tf32<FRESH>(c[t], f[0].hi, f[1].hi, f[2].hi, f[3].hi, g0.hi, g1.hi);
  }
}

// C[i][j] for the 16 rows at a and the 8 NT rows at b; both addresses are of a head's first channel, rows `pitch` bytes apart.
template <typename T, int DT, int NT>
__device__ __forceinline__ void scores(float (&c)[NT][4], uint32_t a, uint32_t b, uint32_t pitch, int dim) {
  const int lane = threadIdx.x & 31;
  if constexpr (sizeof(T) == 2) {
    const uint32_t ra = a + (lane & 15) * pitch + (lane >> 4) * 16;
    const uint32_t rb = b + ((lane & 7) + (lane >> 4) * 8) * pitch + ((lane >> 3) & 1) * 16;  // (two tiles; the last of an odd number: its own)
    const uint32_t rl = b + ((NT - 1) * 8 + (lane & 7)) * pitch + ((lane >> 3) & 1) * 16;
    if constexpr (kExact<DT>) {
      scores_k16<T, NT, true>(c, ra, rb, rl, pitch);
      if constexpr (DT >= 32) scores_k16<T, NT, false>(c, ra + 32, rb + 32, rl + 32, pitch);
      if constexpr (DT % 16 == 8) scores_k8<T, NT, false>(c, a + DT / 16 * 32, b + DT / 16 * 32, pitch);
    } else {
      if (dim == 8) {
        scores_k8<T, NT, true>(c, a, b, pitch);
        return;
      }
      scores_k16<T, NT, true>(c, ra, rb, rl, pitch);
#pragma unroll 1
      for (int k = 1; k * 16 + 16 <= dim; ++k) scores_k16<T, NT, false>(c, ra + k * 32, rb + k * 32, rl + k * 32, pitch);
      if (dim & 8) scores_k8<T, NT, false>(c, a + (dim >> 4) * 32, b + (dim >> 4) * 32, pitch);
    }
  } else {
    float s[NT][4];  // hi lo + lo hi
    const uint32_t ra = a + (lane >> 2) * pitch + (lane & 3) * 4, rb = b + (lane >> 2) * pitch + (lane & 3) * 4;
    scores_tf32<NT, true>(c, s, ra, rb, pitch);
    if constexpr (kExact<DT>) {
#pragma unroll
      for (int k = 1; k < DT / 8; ++k) scores_tf32<NT, false>(c, s, ra + k * 32, rb + k * 32, pitch);
    } else {
#pragma unroll 1
      for (int k = 1; k < dim / 8; ++k) scores_tf32<NT, false>(c, s, ra + k * 32, rb + k * 32, pitch);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) c[t][e] += s[t][e];
  }
}

// acc += W B: W[i][j] over the 8 NT rows j at b.  Rows that hold no voxel are zeros there, and columns of W without one are zero: what lies
// in other segments' rows is not touched, finite or not.  WIDE: W in tf32 (float16's gradients).
template <typename T, int DT, int NT, bool WIDE>
__device__ __forceinline__ void weigh(float (&acc)[DT / 8][4], const float (&w)[NT][4], uint32_t b, uint32_t pitch, int dim) {
  const int lane = threadIdx.x & 31, q2 = (lane & 3) * 2;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int p = 0; p < (NT + 1) / 2; ++p) {  // 16 rows at a time, and the last 8 of an odd number of tiles
      const bool half = 2 * p + 1 == NT;
      const int o = half ? 2 * p : 2 * p + 1;
      uint32_t a[4] = {};
      if (!WIDE) {
        a[0] = Mma<T>::pack(w[2 * p][0], w[2 * p][1]);
        a[1] = Mma<T>::pack(w[2 * p][2], w[2 * p][3]);
        if (!half) {
          a[2] = Mma<T>::pack(w[o][0], w[o][1]);
          a[3] = Mma<T>::pack(w[o][2], w[o][3]);
        }
      }
      auto tile = [&](int n, uint32_t b0, uint32_t b1) {
        if (!WIDE) {
          if (half) Mma<T>::template k8<false>(acc[n], a[0], a[1], b0);
          else Mma<T>::template k16<false>(acc[n], a[0], a[1], a[2], a[3], b0, b1);
        } else {  // eight rows each; their order in the product is that of the accumulators: 0, 2, 4, 6, 1, 3, 5, 7
          const float2 u = __half22float2(*reinterpret_cast<const __half2*>(&b0));
          mma_tf32<false>(acc[n], tf32(w[2 * p][0]), tf32(w[2 * p][2]), tf32(w[2 * p][1]), tf32(w[2 * p][3]), __float_as_uint(u.x), __float_as_uint(u.y));
          if (!half) {
            const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&b1));
            mma_tf32<false>(acc[n], tf32(w[o][0]), tf32(w[o][2]), tf32(w[o][1]), tf32(w[o][3]), __float_as_uint(v.x), __float_as_uint(v.y));
          }
        }
      };
      const uint32_t rb = half ? b + (p * 16 + (lane & 7)) * pitch + ((lane >> 3) & 1) * 16 : b + (p * 16 + (lane & 15)) * pitch + (lane >> 4) * 16;
#pragma unroll
      for (int n = 0; n < DT / 8; n += 2) {
        if (!kExact<DT> && n * 8 >= dim) break;
        const bool two = kExact<DT> ? n + 2 <= DT / 8 : n * 8 + 16 <= dim;
        const int n1 = n + 1 < DT / 8 ? n + 1 : n;
        if (half) {
          uint32_t g0, g1;  // (behind the last channel: the next head's, or the end of the row, not used)
          ldsm2_t(g0, g1, rb + n * 16);
          tile(n, g0, 0u);
          if (two) tile(n1, g1, 0u);
        } else if (two) {
          uint32_t g[4];
          ldsm4_t(g, rb + n * 16);
          tile(n, g[0], g[1]);
          tile(n1, g[2], g[3]);
        } else {
          uint32_t g0, g1;
          ldsm2_t(g0, g1, b + (p * 16 + (lane & 15)) * pitch + n * 16);
          tile(n, g0, g1);
        }
      }
    }
  } else {
    const uint32_t rb = b + q2 * pitch + (lane >> 2) * 4;
    Parts a[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      a[t][0] = split(w[t][0]);
      a[t][1] = split(w[t][2]);
      a[t][2] = split(w[t][1]);
      a[t][3] = split(w[t][3]);
    }
#pragma unroll
    for (int n = 0; n < DT / 8; ++n) {
      if (!kExact<DT> && n * 8 >= dim) break;
      float c[4] = {}, s[4] = {};
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const Parts g0 = split(lds(rb + t * 8 * pitch + n * 32)), g1 = split(lds(rb + (t * 8 + 1) * pitch + n * 32));
        mma_tf32<false>(s, a[t][0].lo, a[t][1].lo, a[t][2].lo, a[t][3].lo, g0.hi, g1.hi);
        mma_tf32<false>(s, a[t][0].hi, a[t][1].hi, a[t][2].hi, a[t][3].hi, g0.lo, g1.lo);
        mma_tf32<false>(c, a[t][0].hi, a[t][1].hi, a[t][2].hi, a[t][3].hi, g0.hi, g1.hi);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[n][e] += c[e] + s[e];
    }
  }
}

// Two neighbours of a tile's four values.
__device__ __forceinline__ F2 two(const float (&z)[4], int e) { return pair(z[e], z[e + 1]); }
__device__ __forceinline__ void put(float (&z)[4], int e, F2 v) {
  const float2 f = parts(v);
  z[e] = f.x;
  z[e + 1] = f.y;
}

// From products to scores in units of log 2: capped first, where there is a cap, then fma(x, scale, bias).  (The cap is a pass of its
// own, and where its derivative is needed the products are formed again: what has no cap is straight-line code.)
struct Scoring {
  float scale;   // of a product to units of log 2; 1 behind a cap
  float inner;   // with a cap: of a product to tanh's argument
  float cap;     // in units of log 2, or 0
  bool bias;
};
static inline Scoring scoring_of(const SegArgs& a) {
  Scoring s;
  s.scale = a.cap > 0.f ? 1.f : a.scale * kLog2e;
  s.inner = a.cap > 0.f ? a.scale / a.cap : 0.f;
  s.cap = a.cap * kLog2e;
  s.bias = a.bias != nullptr;
  return s;
}
// tanh without a branch, off by 3e-7 of the value at most: near 0 the first five terms of its series (the next one is 1e-8 of the value at
// 1/4), else (1 - e) / (1 + e) with e = exp(-2 |x|).
__device__ __forceinline__ float tanh_of(float x) {
  const float y = x * x, a = fabsf(x);
  float near = fmaf(y, 62.f / 2835.f, -17.f / 315.f);
  near = fmaf(y, near, 2.f / 15.f);
  near = fmaf(y, near, -1.f / 3.f);
  near = fmaf(y * near, x, x);
  const float e = ex2_approx(a * (-2.f * kLog2e));
  const float far = copysignf(__fdividef(1.f - e, 1.f + e), x);
  return a < 0.25f ? near : far;  // (NaN: far)
}
// A bias entry in units of log 2.  (Clamped where it is finite: the lowest float stays the lowest, whatever is added, differences of two
// are zero, and the largest is no infinity.  NaN stays NaN: minimum and maximum functions would return the other operand.)
__device__ __forceinline__ float bias_log2(float b) {
  const float x = b * kLog2e;
  return isinf(x) && !isinf(b) ? copysignf(3.402823466e38f, b) : x;
}

template <int NT>
__device__ __forceinline__ void cap_products(float (&s)[NT][4], const Scoring& sc) {
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[t][e] = sc.cap * tanh_of(s[t][e] * sc.inner);
}
// x *= the cap's derivative at the products z.
template <int NT>
__device__ __forceinline__ void cap_slope(float (&x)[NT][4], const float (&z)[NT][4], const Scoring& sc) {
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float u = tanh_of(z[t][e] * sc.inner);
      x[t][e] *= fmaf(-u, u, 1.f);
    }
}

}  // namespace dsvt_train
