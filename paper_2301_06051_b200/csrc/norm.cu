// LayerNorm of a residual sum and its backward pass (the Add & Norm of App. B.1.1, as operators of their own).
//
//   u = x + r,  y = (u - mean(u)) rstd(u) g + b,  h = (u - mean(u)) rstd(u),  w = dy g
//   dx = rstd (w - mean(w) - h mean(w h)),  dg = sum over rows of dy h,  db = sum over rows of dy
//
// Bound by memory: x, r (and dy) are read once and y (dx) written once.  200,000 x 192 bfloat16: 39.7 us in a graph of calls (5.8 TB/s, 89 %
// of a copy's rate; 86 % by single calls), backward 59 us (5.2 TB/s).  A row lies in the registers of a group of lanes, so the
// backward pass takes mean and rstd from the row again, which costs no memory, where reading saved ones would.  Statistics,
// sums and gradients of the weights are fp32; the mean is subtracted before the squares are summed.
// The weights' gradients: a lane adds up its columns over all rows of its group, the groups of a block meet in shared memory,
// and a second kernel adds the blocks, each in a fixed order, so that the same inputs give the same bits.
#include <type_traits>

#include "train_types.cuh"

namespace {
using namespace dsvt_train;

constexpr int kWide = 1024;  // most channels of a row that lies in one warp
template <bool BLOCK>
constexpr int kThreads = BLOCK ? 256 : 128;

template <typename T>
struct NormArgs {
  const T *x, *r, *dy;
  const float *g, *b;
  T* out;          // y or dx
  float* partial;  // [blocks][2][C]: sums of dy h and of dy
  int64_t n;
  int32_t C, lanes;  // lanes of a group (BLOCK: kThreads)
  float eps;
};

// V elements of a row as they are stored, and as numbers: pairs of floats, or single ones (V = 1).
template <typename T, int V>
struct Chunk {
  using Num = F2;
  static constexpr int nums = V / 2, words = V * (int)sizeof(T) / 4;
  alignas(V * sizeof(T)) uint32_t w[words];
  __device__ __forceinline__ void read(F2 (&to)[nums]) const {
#pragma unroll
    for (int i = 0; i < nums; ++i) {
      if constexpr (sizeof(T) == 4) to[i] = pair(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
      else if constexpr (std::is_same<T, __half>::value) { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i])); to[i] = pair(f.x, f.y); }
      else to[i] = pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
  }
  __device__ __forceinline__ void write(const F2 (&from)[nums]) {
#pragma unroll
    for (int i = 0; i < nums; ++i) {
      const float2 f = parts(from[i]);
      if constexpr (sizeof(T) == 4) { w[2 * i] = __float_as_uint(f.x); w[2 * i + 1] = __float_as_uint(f.y); }
      else if constexpr (std::is_same<T, __half>::value) { const __half2 h = __floats2half2_rn(f.x, f.y); w[i] = *reinterpret_cast<const uint32_t*>(&h); }
      else { const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y); w[i] = *reinterpret_cast<const uint32_t*>(&h); }
    }
  }
  static __device__ __forceinline__ F2 splat(float v) { return pair(v, v); }
  static __device__ __forceinline__ F2 weight(const float* p, int i, bool in, float none) { return in && p ? pair(p[2 * i], p[2 * i + 1]) : pair(none, none); }
  static __device__ __forceinline__ void put(float* to, int i, F2 v, bool first) {
    const float2 f = parts(v);
    to[2 * i] = (first ? 0.f : to[2 * i]) + f.x;
    to[2 * i + 1] = (first ? 0.f : to[2 * i + 1]) + f.y;
  }
  static __device__ __forceinline__ F2 over_lanes(F2 v, int m) {
    F2 o;
    o.v = __shfl_xor_sync(0xffffffffu, v.v, m);
    return add(v, o);
  }
};
template <typename T>
struct Chunk<T, 1> {
  using Num = float;
  static constexpr int nums = 1;
  T w[1];
  __device__ __forceinline__ void read(float (&to)[1]) const { to[0] = to_float(w[0]); }
  __device__ __forceinline__ void write(const float (&from)[1]) { w[0] = from_float<T>(from[0]); }
  static __device__ __forceinline__ float splat(float v) { return v; }
  static __device__ __forceinline__ float weight(const float* p, int, bool in, float none) { return in && p ? p[0] : none; }
  static __device__ __forceinline__ void put(float* to, int, float v, bool first) { to[0] = (first ? 0.f : to[0]) + v; }
  static __device__ __forceinline__ float over_lanes(float v, int m) { return v + __shfl_xor_sync(0xffffffffu, v, m); }
};

// The sum of v over a group: a power of two of neighbouring lanes, or the block.  TWO: of both parts.
template <bool BLOCK, bool TWO>
__device__ __forceinline__ float2 group_sum(float2 v, int lanes, float2* scratch) {
  const int width = BLOCK ? 32 : lanes;
  for (int m = width >> 1; m > 0; m >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, m);
    if (TWO) v.y += __shfl_xor_sync(0xffffffffu, v.y, m);
  }
  if (BLOCK) {
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    v = scratch[0];
#pragma unroll
    for (int i = 1; i < kThreads<BLOCK> / 32; ++i) { v.x += scratch[i].x; v.y += scratch[i].y; }
  }
  return v;
}

// Rows on their way: a ring of stages in shared memory, of which every lane fills and reads its own chunks, so that nothing but its own
// copies is waited for.  (With the next row in registers instead, 200,000 x 192 bfloat16 takes 93 us backward and 44 forward.)
template <int V, int VPL, int SIZE, bool BLOCK>
struct Ring {
  static constexpr bool used = V > 1 && !BLOCK;  // (cp.async copies 4 bytes at least; whole blocks' rows would not fit)
  static constexpr int stages = VPL * V * SIZE <= 48 ? 3 : 2;
  static constexpr int chunk = V * SIZE;
  static constexpr int bytes(int arrays) { return used ? stages * arrays * VPL * kThreads<BLOCK> * chunk : 0; }
};
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t to, const void* from) {
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(BYTES) : "memory");
}

// VPL chunks of V elements to a lane: chunks lane, lane + lanes, ...  FULL: they are all there.
template <typename T, int V, int VPL, bool FULL, bool BLOCK, bool BACK>
__global__ void __launch_bounds__(kThreads<BLOCK>) norm_kernel(const NormArgs<T> a) {
  using Ch = Chunk<T, V>;
  using Num = typename Ch::Num;
  constexpr int N = Ch::nums;
  __shared__ float2 scratch[kThreads<BLOCK> / 32];
  pdl_enter();
  const int lanes = BLOCK ? kThreads<BLOCK> : a.lanes, groups = kThreads<BLOCK> / lanes;
  const int group = threadIdx.x / lanes, lane = threadIdx.x % lanes;
  const int nc = a.C / V;
  const float C = (float)a.C;  // (divided by, which rounds once; a constant row's mean is off by what its sum is, and eps takes that up)
  int at[VPL];
  bool in[VPL];
  Num g[VPL][N], b[BACK ? 1 : VPL][N], dg[BACK ? VPL : 1][N], db[BACK ? VPL : 1][N];
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    in[i] = FULL || lane + i * lanes < nc;
    at[i] = in[i] ? (lane + i * lanes) * V : 0;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      g[i][e] = Ch::weight(a.g ? a.g + at[i] : nullptr, e, in[i], 1.f);
      if (!BACK) b[i][e] = Ch::weight(a.b ? a.b + at[i] : nullptr, e, in[i], 0.f);
      if (BACK) dg[i][e] = db[i][e] = Ch::splat(0.f);
    }
  }
  using R = Ring<V, VPL, (int)sizeof(T), BLOCK>;
  extern __shared__ __align__(16) unsigned char smem[];
  const uint32_t mine = (uint32_t)__cvta_generic_to_shared(smem) + threadIdx.x * R::chunk;
  constexpr int kArray = VPL * kThreads<BLOCK> * R::chunk, kStage = (BACK ? 3 : 2) * kArray;
  Ch x[VPL], r[VPL], dy[BACK ? VPL : 1];
  const bool summed = a.r != nullptr;
  auto load = [&](int64_t row, int stage) {
    if constexpr (R::used) {
      if (row < a.n) {
#pragma unroll
        for (int i = 0; i < VPL; ++i)
          if (in[i]) {
            const uint32_t to = mine + stage * kStage + i * kThreads<BLOCK> * R::chunk;
            copy_async<R::chunk>(to, a.x + row * a.C + at[i]);
            if (summed) copy_async<R::chunk>(to + kArray, a.r + row * a.C + at[i]);
            if (BACK) copy_async<R::chunk>(to + 2 * kArray, a.dy + row * a.C + at[i]);
          }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    } else {
      const int64_t from = row < a.n ? row * a.C : 0;  // (behind the last row, and behind a row's last chunk: something that is there, not used)
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        x[i] = *reinterpret_cast<const Ch*>(a.x + from + at[i]);
        if (summed) r[i] = *reinterpret_cast<const Ch*>(a.r + from + at[i]);
        if (BACK) dy[i] = *reinterpret_cast<const Ch*>(a.dy + from + at[i]);
      }
    }
  };
  // every group of a warp makes the same number of rounds (the sums' shuffles need all lanes)
  const int64_t step = (int64_t)gridDim.x * groups;
  int stage = 0;
  constexpr int kAhead = R::used ? R::stages - 1 : 1;
#pragma unroll
  for (int k = 0; k < kAhead; ++k) load((int64_t)blockIdx.x * groups + group + k * step, k);
  for (int64_t row0 = (int64_t)blockIdx.x * groups; row0 < a.n; row0 += step) {
    const int64_t row = row0 + group;
    const bool there = row < a.n;
    if constexpr (R::used) {
      load(row + kAhead * step, stage == 0 ? R::stages - 1 : stage - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(R::stages - 1) : "memory");
      const unsigned char* from = smem + threadIdx.x * R::chunk + stage * kStage;
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        x[i] = *reinterpret_cast<const Ch*>(from + i * kThreads<BLOCK> * R::chunk);
        if (summed) r[i] = *reinterpret_cast<const Ch*>(from + kArray + i * kThreads<BLOCK> * R::chunk);
        if (BACK) dy[i] = *reinterpret_cast<const Ch*>(from + 2 * kArray + i * kThreads<BLOCK> * R::chunk);
      }
      stage = stage + 1 == R::stages ? 0 : stage + 1;
    }
    Num u[VPL][N], w[BACK ? VPL : 1][N], su = Ch::splat(0.f), sw = Ch::splat(0.f);
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      x[i].read(u[i]);
      if (summed) {
        Num o[N];
        r[i].read(o);
#pragma unroll
        for (int e = 0; e < N; ++e) u[i][e] = add(u[i][e], o[e]);
      }
      if (BACK) dy[i].read(w[i]);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (!FULL && !in[i]) {
          u[i][e] = Ch::splat(0.f);
          if (BACK) w[i][e] = Ch::splat(0.f);
        }
        su = add(su, u[i][e]);
        if (BACK) sw = fma2(w[i][e], g[i][e], sw);
      }
    }
    if constexpr (!R::used) load(row + step, 0);  // the next row is on its way while this one is worked on
    float2 s = group_sum<BLOCK, BACK>(make_float2(sum_of(su), BACK ? sum_of(sw) : 0.f), lanes, scratch);
    const Num mean = Ch::splat(-(s.x / C)), mw = Ch::splat(-(s.y / C));
    su = sw = Ch::splat(0.f);
#pragma unroll
    for (int i = 0; i < VPL; ++i)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        u[i][e] = add(u[i][e], mean);
        if (!FULL && !in[i]) u[i][e] = Ch::splat(0.f);
        su = fma2(u[i][e], u[i][e], su);
        if (BACK) sw = fma2(mul(w[i][e], g[i][e]), u[i][e], sw);
      }
    s = group_sum<BLOCK, BACK>(make_float2(sum_of(su), BACK ? sum_of(sw) : 0.f), lanes, scratch);
    const float rs = there ? 1.f / sqrtf(s.x / C + a.eps) : 0.f;
    const Num rstd = Ch::splat(rs), mwh = Ch::splat(-(s.y / C * rs));
    T* to = a.out + row * a.C;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      Num o[N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const Num h = mul(u[i][e], rstd);
        if (BACK) {
          o[e] = mul(rstd, fma2(h, mwh, fma2(w[i][e], g[i][e], mw)));
          if (there) {  // (else it is another row's)
            dg[i][e] = fma2(w[i][e], h, dg[i][e]);
            db[i][e] = add(db[i][e], w[i][e]);
          }
        } else {
          o[e] = fma2(h, g[i][e], b[i][e]);
        }
      }
      Ch out;
      out.write(o);
      if (there && in[i]) *reinterpret_cast<Ch*>(to + at[i]) = out;
    }
  }
  if (BACK) {
    float* sums = reinterpret_cast<float*>(smem);  // [2][C]; the ring is done with
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    // groups of one warp by shuffles, then warp after warp
    if (!BLOCK)
      for (int m = 16; m >= lanes; m >>= 1)
#pragma unroll
        for (int i = 0; i < VPL; ++i)
#pragma unroll
          for (int e = 0; e < N; ++e) {
            dg[i][e] = Ch::over_lanes(dg[i][e], m);
            db[i][e] = Ch::over_lanes(db[i][e], m);
          }
    const int warps = BLOCK ? 1 : kThreads<BLOCK> / 32;
    for (int t = 0; t < warps; ++t) {
      if (BLOCK || ((int)threadIdx.x >> 5 == t && ((int)threadIdx.x & 31) < lanes)) {
#pragma unroll
        for (int i = 0; i < VPL; ++i)
          if (in[i])
#pragma unroll
            for (int e = 0; e < N; ++e) {
              Ch::put(sums + at[i], e, dg[i][e], t == 0);
              Ch::put(sums + a.C + at[i], e, db[i][e], t == 0);
            }
      }
      __syncthreads();
    }
    for (int i = threadIdx.x; i < 2 * a.C; i += kThreads<BLOCK>) a.partial[(int64_t)blockIdx.x * 2 * a.C + i] = sums[i];
  }
}

// dg and db: 32 columns to a block, every warp a share of the partial sums.
constexpr int kGradThreads = 1024;
__global__ void __launch_bounds__(kGradThreads) norm_weight_grad_kernel(const float* partial, int blocks, int C, float* dg, float* db) {
  __shared__ float part[kGradThreads / 32][33];
  pdl_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (col < 2 * C)
#pragma unroll 16
    for (int p = warp; p < blocks; p += kGradThreads / 32) s += partial[(int64_t)p * 2 * C + col];
  part[warp][lane] = s;
  __syncthreads();
  s = part[lane][warp];  // a warp adds up one column
  for (int m = 16; m > 0; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
  const int mine = blockIdx.x * 32 + warp;
  if (lane != 0 || mine >= 2 * C) return;
  float* out = mine < C ? dg : db;
  if (out) out[mine < C ? mine : mine - C] = s;
}

constexpr int kMaxC = 8192;

template <typename T, int V, int VPL, bool FULL, bool BLOCK, bool BACK>
int launch(dsvt_ctx* ctx, NormArgs<T> a, float* dg, float* db) {
  constexpr int threads = kThreads<BLOCK>;
  constexpr auto kernel = norm_kernel<T, V, VPL, FULL, BLOCK, BACK>;
  const int groups = threads / (BLOCK ? threads : a.lanes);
  int64_t blocks = dsvt_ceil_div(a.n, groups);
  // as many blocks as can be resident, each about the same number of rows
  constexpr int ring = Ring<V, VPL, (int)sizeof(T), BLOCK>::bytes(BACK ? 3 : 2);
  constexpr int sums = BACK ? 2 * (BLOCK ? kMaxC : kWide) * (int)sizeof(float) : 0, room = ring > sums ? ring : sums;
  const int mine = BACK ? 2 * a.C * (int)sizeof(float) : 0, smem = mine > ring ? mine : ring;
  if constexpr (room > 47 * 1024) {
    const int rc = allow_smem<kernel>(ctx, room);
    if (rc != DSVT_OK) return rc;
  }
  int per_sm = 0;
  DSVT_CUDA_TRY(ctx, cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem));
  int64_t most = (int64_t)ctx->sm_count * (per_sm > 0 ? per_sm : 1);
  if (BACK && most > (int64_t)(4 * ctx->bm_words) / (2 * a.C)) most = (int64_t)(4 * ctx->bm_words) / (2 * a.C);  // (the workspace)
  if (blocks > most) blocks = most;
  launch_pdl(kernel, dim3((unsigned)blocks), dim3(threads), smem, ctx->stream, a);
  DSVT_LAUNCHED(ctx);
  if (BACK && (dg || db)) {
    launch_pdl(norm_weight_grad_kernel, dim3((unsigned)dsvt_ceil_div(2 * a.C, 32)), dim3(kGradThreads), 0, ctx->stream,
               (const float*)a.partial, (int)blocks, a.C, dg, db);
    DSVT_LAUNCHED(ctx);
  }
  return DSVT_OK;
}

// Chunks of 16 bytes where rows are whole ones, else of 4 elements, else single elements.  Of the groups that give a lane at most 24
// (backward, fp32: 16) elements the one that wastes fewest lanes, and of these the smallest: fewer steps to its sums.
template <typename T, int V, bool BACK>
int chunked(dsvt_ctx* ctx, NormArgs<T> a, float* dg, float* db) {
  const int nc = a.C / V, most = V == 8 ? 3 : 4;
  int best = 32, vpl = (nc + 31) / 32;
  for (int lanes = 16; lanes >= 4; lanes >>= 1) {
    const int v = (nc + lanes - 1) / lanes;
    if (v <= most && v * lanes <= vpl * best) { best = lanes; vpl = v; }
  }
  a.lanes = best;
  const bool full = vpl * best == nc;
#define DSVT_NORM(VPL) return full ? launch<T, V, VPL, true, false, BACK>(ctx, a, dg, db) : launch<T, V, VPL, false, false, BACK>(ctx, a, dg, db)
  switch (vpl) {
    case 1: DSVT_NORM(1);
    case 2: DSVT_NORM(2);
    case 3: DSVT_NORM(3);
    case 4: DSVT_NORM(4);
  }
#undef DSVT_NORM
  if constexpr (V == 4) return launch<T, V, 8, false, false, BACK>(ctx, a, dg, db);
  return DSVT_ERR_UNSUPPORTED;  // (not reached: 32 lanes of 4 chunks of 8 hold kWide channels)
}

template <typename T, bool BACK>
int dispatch(dsvt_ctx* ctx, NormArgs<T> a, float* dg, float* db) {
  if (a.C > kWide) {
    if (a.C % 4 == 0) return a.C <= 4096 ? launch<T, 4, 4, false, true, BACK>(ctx, a, dg, db) : launch<T, 4, 8, false, true, BACK>(ctx, a, dg, db);
    return a.C <= 2048 ? launch<T, 1, 8, false, true, BACK>(ctx, a, dg, db) : launch<T, 1, 32, false, true, BACK>(ctx, a, dg, db);
  }
  if constexpr (sizeof(T) == 2)
    if (a.C % 8 == 0) return chunked<T, 8, BACK>(ctx, a, dg, db);
  if (a.C % 4 == 0) return chunked<T, 4, BACK>(ctx, a, dg, db);
  a.lanes = 32;
  if (a.C <= 128) return launch<T, 1, 4, false, false, BACK>(ctx, a, dg, db);
  if (a.C <= 512) return launch<T, 1, 16, false, false, BACK>(ctx, a, dg, db);
  return launch<T, 1, 32, false, false, BACK>(ctx, a, dg, db);
}

template <typename T>
int run(dsvt_ctx* ctx, bool back, const void* x, const void* r, const void* dy, int32_t n, int32_t C, const float* g, const float* b,
        float eps, void* out, float* dg, float* db) {
  NormArgs<T> a = {};
  a.x = (const T*)x; a.r = (const T*)r; a.dy = (const T*)dy; a.g = g; a.b = b; a.out = (T*)out; a.n = n; a.C = C; a.eps = eps;
  a.partial = reinterpret_cast<float*>(ctx->bm_zero);  // (the partition's bitmaps and their ranks, 4 bm_words words)
  return back ? dispatch<T, true>(ctx, a, dg, db) : dispatch<T, false>(ctx, a, dg, db);
}

int norm(dsvt_ctx* ctx, bool back, int type, const void* x, const void* r, const void* dy, int32_t n, int32_t C, const float* g,
         const float* b, float eps, void* out, float* dg, float* db) {
  if (!ctx || !type_known(type) || n < 0 || C < 1 || !(eps >= 0.f)) return DSVT_ERR_INVALID_ARG;
  if (n > 0 && (!x || !out || (back && !dy))) return DSVT_ERR_INVALID_ARG;
  const void* ptrs[] = {x, r, dy, out};
  for (const void* q : ptrs)
    if (((uintptr_t)q & 15) != 0) return DSVT_ERR_INVALID_ARG;
  const void* words[] = {g, b, dg, db};
  for (const void* q : words)
    if (((uintptr_t)q & 3) != 0) return DSVT_ERR_INVALID_ARG;
  if (C > kMaxC) return DSVT_ERR_UNSUPPORTED;
  DeviceGuard on(ctx->device);
  if (n == 0) {
    if (dg) DSVT_CUDA_TRY(ctx, cudaMemsetAsync(dg, 0, (size_t)C * sizeof(float), ctx->stream));
    if (db) DSVT_CUDA_TRY(ctx, cudaMemsetAsync(db, 0, (size_t)C * sizeof(float), ctx->stream));
    return DSVT_OK;
  }
  if (type == DSVT_TYPE_F32) return run<float>(ctx, back, x, r, dy, n, C, g, b, eps, out, dg, db);
  if (type == DSVT_TYPE_BF16) return run<__nv_bfloat16>(ctx, back, x, r, dy, n, C, g, b, eps, out, dg, db);
  return run<__half>(ctx, back, x, r, dy, n, C, g, b, eps, out, dg, db);
}

}  // namespace

extern "C" int dsvt_layer_norm(dsvt_ctx* ctx, int type, const void* x, const void* residual, int32_t n, int32_t C, const float* g,
                               const float* b, float eps, void* y) {
  return norm(ctx, false, type, x, residual, nullptr, n, C, g, b, eps, y, nullptr, nullptr);
}

extern "C" int dsvt_layer_norm_backward(dsvt_ctx* ctx, int type, const void* x, const void* residual, const void* dy, int32_t n,
                                        int32_t C, const float* g, float eps, void* dx, float* dg, float* db) {
  return norm(ctx, true, type, x, residual, dy, n, C, g, nullptr, eps, dx, dg, db);
}
