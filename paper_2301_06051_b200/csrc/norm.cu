// LayerNorm of a residual sum and its backward pass (the Add & Norm of App. B.1.1, as operators of their own).
//
//   u = x + r,  y = (u - mean(u)) rstd(u) g + b,  h = (u - mean(u)) rstd(u),  w = dy g
//   dx = rstd (w - mean(w) - h mean(w h)),  dg = sum over rows of dy h,  db = sum over rows of dy
//
// Bound by memory: x, r (and dy) are read once and y (dx) written once.  A row lies in the registers of a group of lanes, so the
// backward pass takes mean and rstd from the row again, which costs no memory, where reading saved ones would.  Statistics,
// sums and gradients of the weights are fp32; the mean is subtracted before the squares are summed.
// The weights' gradients: a lane adds up its columns over all rows of its group, the groups of a block meet in shared memory,
// and a second kernel adds the blocks, each in a fixed order, so that the same inputs give the same bits.
#include "train_types.cuh"

namespace {
using namespace dsvt_train;

constexpr int kThreads = 256;

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

// V elements from p on as they are stored.
template <typename T, int V>
struct alignas(sizeof(T) * V) Chunk { T v[V]; };

// The sum of v over a group: a power of two of neighbouring lanes, or the block.
template <bool BLOCK>
__device__ __forceinline__ float2 group_sum(float2 v, int lanes, float2* scratch) {
  const int width = BLOCK ? 32 : lanes;
  for (int m = width >> 1; m > 0; m >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, m);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, m);
  }
  if (BLOCK) {
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    v = scratch[0];
#pragma unroll
    for (int i = 1; i < kThreads / 32; ++i) { v.x += scratch[i].x; v.y += scratch[i].y; }
  }
  return v;
}

// VPL chunks of V elements to a lane: chunks lane, lane + lanes, ...
template <typename T, int V, int VPL, bool BLOCK, bool BACK>
__global__ void __launch_bounds__(kThreads) norm_kernel(const NormArgs<T> a) {
  using Ch = Chunk<T, V>;
  __shared__ float2 scratch[kThreads / 32];
  pdl_enter();
  const int lanes = BLOCK ? kThreads : a.lanes, groups = kThreads / lanes;
  const int group = threadIdx.x / lanes, lane = threadIdx.x % lanes;
  const int nc = a.C / V;
  const float C = (float)a.C;  // (divided by: the mean of a constant row is the constant)
  float g[VPL * V], b[BACK ? 1 : VPL * V], dg[BACK ? VPL * V : 1], db[BACK ? VPL * V : 1];
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    const int c = lane + i * lanes;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      g[i * V + e] = c < nc && a.g ? a.g[c * V + e] : 1.f;
      if (!BACK) b[i * V + e] = c < nc && a.b ? a.b[c * V + e] : 0.f;
      if (BACK) dg[i * V + e] = db[i * V + e] = 0.f;
    }
  }
  Ch x[VPL], r[VPL], dy[BACK ? VPL : 1];
  const Ch zero = {};
  auto load = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const int c = lane + i * lanes;
      const int64_t at = row * a.C + (int64_t)c * V;
      const bool in = row < a.n && c < nc;
      x[i] = in ? *reinterpret_cast<const Ch*>(a.x + at) : zero;
      r[i] = in && a.r ? *reinterpret_cast<const Ch*>(a.r + at) : zero;
      if (BACK) dy[i] = in ? *reinterpret_cast<const Ch*>(a.dy + at) : zero;
    }
  };
  // every group of a warp makes the same number of rounds (the sums' shuffles need all lanes); rows beyond the last are zeros
  const int64_t step = (int64_t)gridDim.x * groups;
  load((int64_t)blockIdx.x * groups + group);
  for (int64_t row0 = (int64_t)blockIdx.x * groups; row0 < a.n; row0 += step) {
    const int64_t row = row0 + group;
    float u[VPL * V], w[BACK ? VPL * V : 1];
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < VPL; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int k = i * V + e;
        u[k] = to_float(x[i].v[e]) + to_float(r[i].v[e]);
        s.x += u[k];
        if (BACK) w[k] = to_float(dy[i].v[e]);
      }
    load(row + step);  // the next row is on its way while this one is worked on
    const float mean = group_sum<BLOCK>(s, lanes, scratch).x / C;
    s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const bool in = lane + i * lanes < nc;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int k = i * V + e;
        u[k] = in ? u[k] - mean : 0.f;
        s.x = fmaf(u[k], u[k], s.x);
        if (BACK) s.y = fmaf(w[k], g[k], s.y);
      }
    }
    s = group_sum<BLOCK>(s, lanes, scratch);
    const float rstd = row < a.n ? 1.f / sqrtf(s.x / C + a.eps) : 0.f;
    float mw = 0.f, mwh = 0.f;
    if (BACK) {
      mw = s.y / C;
      float2 t = make_float2(0.f, 0.f);
#pragma unroll
      for (int k = 0; k < VPL * V; ++k) {
        u[k] *= rstd;
        t.x = fmaf(w[k] * g[k], u[k], t.x);
        dg[k] = fmaf(w[k], u[k], dg[k]);
        db[k] += w[k];
      }
      mwh = group_sum<BLOCK>(t, lanes, scratch).x / C;
    }
    if (row < a.n) {
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const int c = lane + i * lanes;
        Ch o;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const int k = i * V + e;
          o.v[e] = from_float<T>(BACK ? rstd * (fmaf(w[k], g[k], -mw) - u[k] * mwh) : fmaf(u[k] * rstd, g[k], b[k]));
        }
        if (c < nc) *reinterpret_cast<Ch*>(a.out + row * a.C + (int64_t)c * V) = o;
      }
    }
  }
  if (BACK) {
    extern __shared__ float sums[];  // [2][C]
    // groups of one warp by shuffles, then warp after warp
    if (!BLOCK)
#pragma unroll
      for (int k = 0; k < VPL * V; ++k)
        for (int m = 16; m >= lanes; m >>= 1) {
          dg[k] += __shfl_xor_sync(0xffffffffu, dg[k], m);
          db[k] += __shfl_xor_sync(0xffffffffu, db[k], m);
        }
    const int warps = BLOCK ? 1 : kThreads / 32;
    for (int t = 0; t < warps; ++t) {
      if (BLOCK || ((int)threadIdx.x >> 5 == t && ((int)threadIdx.x & 31) < lanes)) {
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
          const int c = lane + i * lanes;
          if (c < nc)
#pragma unroll
            for (int e = 0; e < V; ++e) {
              const int k = i * V + e, at = c * V + e;
              sums[at] = (t == 0 ? 0.f : sums[at]) + dg[k];
              sums[a.C + at] = (t == 0 ? 0.f : sums[a.C + at]) + db[k];
            }
        }
      }
      __syncthreads();
    }
    for (int i = threadIdx.x; i < 2 * a.C; i += kThreads) a.partial[(int64_t)blockIdx.x * 2 * a.C + i] = sums[i];
  }
}

// dg and db: 32 columns to a block, every warp a share of the partial sums.
__global__ void __launch_bounds__(kThreads) norm_weight_grad_kernel(const float* partial, int blocks, int C, float* dg, float* db) {
  __shared__ float part[kThreads / 32][32];
  pdl_enter();
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), warp = threadIdx.x >> 5;
  float s = 0.f;
  if (col < 2 * C)
#pragma unroll 4
    for (int p = warp; p < blocks; p += kThreads / 32) s += partial[(int64_t)p * 2 * C + col];
  part[warp][threadIdx.x & 31] = s;
  __syncthreads();
  if (warp != 0 || col >= 2 * C) return;
  for (int i = 1; i < kThreads / 32; ++i) s += part[i][threadIdx.x];
  float* out = col < C ? dg : db;
  if (out) out[col < C ? col : col - C] = s;
}

constexpr int kMaxC = 8192;

template <typename T, int V, int VPL, bool BLOCK, bool BACK>
int launch(dsvt_ctx* ctx, NormArgs<T> a, float* dg, float* db) {
  const int groups = kThreads / (BLOCK ? kThreads : a.lanes);
  int64_t blocks = dsvt_ceil_div(a.n, groups);
  int64_t most = (int64_t)ctx->sm_count * 4;
  if (BACK && most > (int64_t)(4 * ctx->bm_words) / (2 * a.C)) most = (int64_t)(4 * ctx->bm_words) / (2 * a.C);  // (the workspace)
  if (blocks > most) blocks = most;
  const size_t smem = BACK ? 2 * (size_t)a.C * sizeof(float) : 0;
  auto kernel = norm_kernel<T, V, VPL, BLOCK, BACK>;
  if (smem > 48 * 1024) DSVT_CUDA_TRY(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  launch_pdl(kernel, dim3((unsigned)blocks), dim3(kThreads), smem, ctx->stream, a);
  DSVT_LAUNCHED(ctx);
  if (BACK && (dg || db)) {
    launch_pdl(norm_weight_grad_kernel, dim3((unsigned)dsvt_ceil_div(2 * a.C, 32)), dim3(kThreads), 0, ctx->stream,
               (const float*)a.partial, (int)blocks, a.C, dg, db);
    DSVT_LAUNCHED(ctx);
  }
  return DSVT_OK;
}

// The group that wastes fewest lanes: chunks nc over `lanes` lanes, VPL to each.
template <typename T, bool BACK>
int dispatch(dsvt_ctx* ctx, NormArgs<T> a, float* dg, float* db) {
  if (a.C % 4 == 0) {
    const int nc = a.C / 4;
    if (nc > 256) return nc <= 1024 ? launch<T, 4, 4, true, BACK>(ctx, a, dg, db) : launch<T, 4, 8, true, BACK>(ctx, a, dg, db);
    int best = 32, vpl = (nc + 31) / 32;
    for (int lanes = 16; lanes >= 4; lanes >>= 1) {
      const int v = (nc + lanes - 1) / lanes;
      if (v <= 4 && v * lanes < vpl * best) { best = lanes; vpl = v; }
    }
    a.lanes = best;
    switch (vpl) {
      case 1: return launch<T, 4, 1, false, BACK>(ctx, a, dg, db);
      case 2: return launch<T, 4, 2, false, BACK>(ctx, a, dg, db);
      case 3: return launch<T, 4, 3, false, BACK>(ctx, a, dg, db);
      case 4: return launch<T, 4, 4, false, BACK>(ctx, a, dg, db);
      case 5: case 6: return launch<T, 4, 6, false, BACK>(ctx, a, dg, db);
      default: return launch<T, 4, 8, false, BACK>(ctx, a, dg, db);
    }
  }
  a.lanes = 32;
  if (a.C <= 128) return launch<T, 1, 4, false, BACK>(ctx, a, dg, db);
  if (a.C <= 512) return launch<T, 1, 16, false, BACK>(ctx, a, dg, db);
  if (a.C <= 2048) return launch<T, 1, 8, true, BACK>(ctx, a, dg, db);
  return launch<T, 1, 32, true, BACK>(ctx, a, dg, db);
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
