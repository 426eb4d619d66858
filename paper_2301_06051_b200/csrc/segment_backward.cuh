// Segment attention, backward: two passes over the scores, each with them in registers the way it needs them.
//
//   by queries: maximum, sum and D of a row, then dq = scale dz k
//   by keys:    p and dz again from those three, dk = scale dz^T q, dv = p^T do, and the bias's gradient
//
// Short segments do both in one block, long ones in two kernels.  Measured (bf16, dim 24, 8 heads): 32,000 pillars in sets of 36 95 us,
// where the bytes that it cannot do without take 13; 60,000 voxels in whole windows of up to 850, 1196 us (bytes 25).  Bound by
// instructions and their latencies (long segments: 111 a score by queries, 97 by keys): warps issue in 41 to 52 % of the cycles, the tensor
// pipe is busy for 5 to 10 %, DRAM for 1 to 7 %.
// D = sum_j p dp is formed from the scores and not from the output: the output's rounding to 16 bits would reach the bias's gradient,
// which is fp32.
//
// The bias's gradient adds up ds by bucket, a scatter.  It is held as integers, so that their order does not matter and the same
// inputs give the same bits: v = (hi 2^-17 + lo 2^-35) limit with |hi|, |lo| <= 2^17, two words of shared memory to a bucket, which
// take 16,000 values before they are emptied into floats (short: the block's own partial sums) or 64-bit integers in global memory
// (long).  limit is a power of two, 2^-110 ... 2^128, that bounds |ds|, from the first pass: |p dp| + |p D| <= max_j |p dp| + |D| max_j p, and
// at most four times that.  A value is off by 2^-36 of the limit.  Integer additions in shared memory are also the fast ones here: 1.4 ns a warp where
// the addresses differ, fp32's 6 ns, 64-bit 11 ns.  Where they are the same they follow one another (8 lanes to an address: 5 ns), and
// neighbouring keys and queries have the same displacements; so the four lanes that share a key add to tables of their own where there
// is room, or two and two.
#pragma once
#include "segment_forward.cuh"

namespace dsvt_train {

constexpr int kMaxPending = 16000;
constexpr int kShortBack = 120;  // most rows of a segment that is held whole here: its pairs may all be of one bucket
static_assert(kShortBack * kShortBack <= kMaxPending && kShortBack <= kShort, "a batch of one segment is counted without being emptied");
constexpr int kHiBits = 17, kLoBits = 18;
constexpr float kMagic = 12582912.f;  // 1.5 x 2^23: adding it rounds to a whole number in the low bits

// The context's workspace (the partition's bitmaps and ranks) in 32-bit words.
constexpr size_t kPartialWords = (size_t)1 << 21, kTotalWords = 4 * (size_t)kMaxBiasTable;
struct BackWork {
  float* partial;               // [blocks][table]: the short ones' sums
  unsigned long long* total;    // [2][table]: the long ones', hi and lo
  uint32_t* spoilt;             // [table / 32] bits: a value that was not finite
  uint32_t* bounds;             // [launches]: what the long ones' |ds| is at most, as a float's bits
  float* stats;                 // [heads of a launch][n][3]
  int32_t table, blocks, n;
  int32_t head0, head_end, at_once, launches;  // heads of a launch of the long ones, how many to a launch, and how many launches
};

// A value that need not be within the limit (the two passes' roundings of large scores may leave one beyond it), nor finite.
static __device__ __noinline__ void odd_value(int* at, uint32_t* spoilt, int entry, float v, float limit, float to_hi, int buckets) {
  if (!isfinite(v)) {
    atomicOr(spoilt + (entry >> 5), 1u << (entry & 31));
    return;
  }
  v = fminf(fmaxf(v, -limit), limit);
  const float t = fmaf(v, to_hi, kMagic), r = fmaf(v, to_hi, -(t - kMagic)), u = fmaf(r, (float)(1 << kLoBits), kMagic);
  atomicAdd(at, __float_as_int(t) - __float_as_int(kMagic));
  atomicAdd(at + buckets, __float_as_int(u) - __float_as_int(kMagic));
}

struct Tally {
  int* hist;           // [copies][heads][2][buckets]
  uint32_t* spoilt;    // bits [heads][buckets]
  int buckets, copies, copy;  // copy: entries of one
  float limit, to_hi;  // to_hi = 2^kHiBits / limit, where a limit of 2^128 is held as the largest float
  bool on;
  __device__ __forceinline__ void bound(float b) {
    int e = (int)((__float_as_uint(b) >> 23) & 255) - 127 + 2;
    e = min(max(e, -110), 128);
    limit = e < 128 ? __int_as_float((e + 127) << 23) : 3.402823466e38f;
    to_hi = __int_as_float((kHiBits - e + 127) << 23);
  }
  template <int N>
  __device__ __forceinline__ void clear_all(int heads) const {
    for (int i = threadIdx.x; i < copies * copy; i += N) hist[i] = 0;
    for (int i = threadIdx.x; i < (heads * buckets + 31) / 32; i += N) spoilt[i] = 0;
  }
  // Entry i of the table [heads][buckets]: its words, which are cleared, and whether a value of it was not finite.
  __device__ __forceinline__ bool take(int i, long long& hi, long long& lo) const {
    const int h = i / buckets, at = 2 * h * buckets + i - h * buckets;
    hi = lo = 0;
    for (int c = 0; c < copies; ++c) {
      int* p = hist + c * copy + at;
      hi += p[0];
      lo += p[buckets];
      p[0] = p[buckets] = 0;
    }
    return spoilt[i >> 5] >> (i & 31) & 1;
  }
  // A chunk's values of head h; bk: their buckets times 4.  SOME: those whose bit, 4 t + e, is set.
  template <int NT, bool SOME>
  __device__ __forceinline__ void count(int h, const int (&bk)[NT][4], const float (&v)[NT][4], uint32_t which) const {
    char* base = reinterpret_cast<char*>(hist + (threadIdx.x & (copies - 1)) * copy + 2 * h * buckets);
    float most = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (!SOME || (which >> (4 * t + e) & 1)) asm("max.NaN.f32 %0, %0, %1;" : "+f"(most) : "f"(fabsf(v[t][e])));
    if (__any_sync(kAll, !(most <= limit))) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!SOME || (which >> (4 * t + e) & 1))
            odd_value(reinterpret_cast<int*>(base + bk[t][e]), spoilt, h * buckets + (bk[t][e] >> 2), v[t][e], limit, to_hi, buckets);
      return;
    }
    const F2 scale = pair(to_hi, to_hi), magic = pair(kMagic, kMagic), back = pair(-kMagic, -kMagic), minus = pair(-1.f, -1.f);
    const F2 lo = pair((float)(1 << kLoBits), (float)(1 << kLoBits));
    const int zero = __float_as_int(kMagic);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const F2 z = two(v[t], e), x = fma2(z, scale, magic);
        const F2 u = fma2(fma2(z, scale, mul(add(x, back), minus)), lo, magic);
        if (!SOME || (which >> (4 * t + e) & 1)) {
          int* p = reinterpret_cast<int*>(base + bk[t][e]);
          atomicAdd(p, __float_as_int(parts(x).x) - zero);
          atomicAdd(p + buckets, __float_as_int(parts(u).x) - zero);
        }
        if (!SOME || (which >> (4 * t + e + 1) & 1)) {
          int* q = reinterpret_cast<int*>(base + bk[t][e + 1]);
          atomicAdd(q, __float_as_int(parts(x).y) - zero);
          atomicAdd(q + buckets, __float_as_int(parts(u).y) - zero);
        }
      }
  }
};

// What the words stand for.
__device__ __forceinline__ float tally_value(long long hi, long long lo, float to_hi) {
  const double unit = __hiloint2double((1023 + 127 - (__float_as_int(to_hi) >> 23)) << 20, 0);  // 1 / to_hi
  return (float)(((double)hi + (double)lo * (1.0 / (1 << kLoBits))) * unit);
}

// A tile's two rows of the first pass: maximum and sum as in Flow, D and the largest |p dp| before they are divided by the sum.
struct RowSums {
  float m[2], l[2], d[2], most[2];
  __device__ __forceinline__ void start() {
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = d[0] = d[1] = most[0] = most[1] = 0.f;
  }
};
// (s: scores, then weights; dp: products of do and v)
template <int NT>
__device__ __forceinline__ void sum_rows(RowSums& f, float (&s)[NT][4], const float (&dp)[NT][4]) {
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    float m = f.m[r];
#pragma unroll
    for (int t = 0; t < NT; ++t) m = fmaxf(m, fmaxf(s[t][2 * r], s[t][2 * r + 1]));
    m = quad_max(m);
    const float base = m == -INFINITY ? 0.f : m, fade = ex2_approx(f.m[r] - base);
    f.m[r] = m;
    const F2 down = pair(-base, -base);
    F2 l = pair(f.l[r] * fade, 0.f), d = pair(f.d[r] * fade, 0.f);
    float most = f.most[r] * fade;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float2 x = parts(add(two(s[t], 2 * r), down));
      s[t][2 * r] = ex2_approx(x.x);
      s[t][2 * r + 1] = ex2_approx(x.y);
      const F2 p = two(s[t], 2 * r), y = mul(p, two(dp[t], 2 * r));
      l = add(l, p);
      d = add(d, y);
      most = fmaxf(most, fmaxf(fabsf(parts(y).x), fabsf(parts(y).y)));
    }
    f.l[r] = sum_of(l); f.d[r] = sum_of(d); f.most[r] = most;
  }
}
// Row r's maximum, 1 / sum and D, and the bound of its |ds| (0 where D is not finite: such a row's values are counted apart).
__device__ __forceinline__ float3 row_stats(const RowSums& f, int r, float* bound) {
  const float inv = inverse(quad_sum(f.l[r])), D = quad_sum(f.d[r]) * inv;
  const float b = quad_max(f.most[r]) * inv + fabsf(D) * fminf(inv, 1.f);
  *bound = isfinite(D) ? fminf(b, 3.402823466e38f) : 0.f;
  return make_float3(f.m[r] == -INFINITY ? 0.f : f.m[r], inv, D);
}

// dz of the rows' chunk into dp, from weights relative to the maximum (calls without a cap).
template <int NT>
__device__ __forceinline__ void differ_weights(const float (&s)[NT][4], float (&dp)[NT][4], const float3 (&st)[2]) {
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const F2 inv = pair(st[r].y, st[r].y), D = pair(-st[r].z, -st[r].z);
#pragma unroll
    for (int t = 0; t < NT; ++t) put(dp[t], 2 * r, mul(mul(two(s[t], 2 * r), inv), add(two(dp[t], 2 * r), D)));
  }
}

// The same from scores.
template <int NT>
__device__ __forceinline__ void differ_rows(const float (&s)[NT][4], float (&dp)[NT][4], const float3 (&st)[2]) {
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const F2 down = pair(-st[r].x, -st[r].x), inv = pair(st[r].y, st[r].y), D = pair(-st[r].z, -st[r].z);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float2 x = parts(add(two(s[t], 2 * r), down));
      put(dp[t], 2 * r, mul(mul(pair(ex2_approx(x.x), ex2_approx(x.y)), inv), add(two(dp[t], 2 * r), D)));
    }
  }
}

// The second pass's columns' maximum, 1 / sum and D: three arrays, `step` floats apart.
struct ColumnStats {
  const float* at;
  int step;
};

// The second pass's chunk: rows are keys, columns queries.  s: scores -> p; dp: products v do -> ds.
template <int NT>
__device__ __forceinline__ void differ_columns(float (&s)[NT][4], float (&dp)[NT][4], const ColumnStats& stats) {
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const float* st = stats.at + t * 8 + (threadIdx.x & 3) * 2;
    const float2 m = *reinterpret_cast<const float2*>(st), i = *reinterpret_cast<const float2*>(st + stats.step), D = *reinterpret_cast<const float2*>(st + 2 * stats.step);
    const F2 down = pair(-m.x, -m.y), inv = pair(i.x, i.y), less = pair(-D.x, -D.y);
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
      const float2 x = parts(add(two(s[t], e), down));
      const F2 p = mul(pair(ex2_approx(x.x), ex2_approx(x.y)), inv);
      put(s[t], e, p);
      put(dp[t], e, mul(p, add(two(dp[t], e), less)));
    }
  }
}

// Rows of an accumulator to global memory.
template <typename T, int DT>
__device__ __forceinline__ void store_rows(const float (&acc)[DT / 8][4], float scale, void* to, int64_t ld, int64_t col, int dim, int id0, int id1) {
  T* at = (T*)to + col + (threadIdx.x & 3) * 2;
#pragma unroll
  for (int n = 0; n < DT / 8; ++n) {
    if (!kExact<DT> && n * 8 >= dim) break;
    if (id0 >= 0) store2<T>(at + id0 * ld + n * 8, acc[n][0] * scale, acc[n][1] * scale);
    if (id1 >= 0) store2<T>(at + id1 * ld + n * 8, acc[n][2] * scale, acc[n][3] * scale);
  }
}

template <int DT>
__device__ __forceinline__ void clear(float (&acc)[DT / 8][4]) {
#pragma unroll
  for (int n = 0; n < DT / 8; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;
}

template <typename T>
constexpr bool kWide = std::is_same<T, __half>::value;

// Heads of a block that holds its segments whole.
template <typename T, int DT>
constexpr int kBackHeads = DT * sizeof(T) <= 32 ? 8 : DT * sizeof(T) <= 64 ? 4 : DT * sizeof(T) <= 128 ? 2 : 1;

// A tile of 16 rows against a chunk of its segment's rows, in one block's shared memory: addresses of a head's first channel.
struct Operands {
  uint32_t q, k, v, o;          // at the tile's first row
  uint32_t cq, ck, cv, co;      // at the chunk's
  const float* bias;
  const uint16_t* index;        // at the tile's first row and the chunk's first column (by keys: the chunk's first row, the tile's first column)
  int pitch_idx;
  uint32_t pitch;
  int dim;
};

// By queries: products into s and dp.
template <typename T, int DT, int NT>
__device__ __forceinline__ void products(float (&s)[NT][4], float (&dp)[NT][4], const Operands& x, uint64_t keys) {
  scores<T, DT, NT>(s, x.q, x.ck, x.pitch, x.dim);
  scores<T, DT, NT>(dp, x.o, x.cv, x.pitch, x.dim);
  set_columns<NT>(dp, keys, 0.f);  // (whatever lies there)
}
// dp: ds -> dz; s is written over.
template <typename T, int DT, int NT>
__device__ __forceinline__ void through_cap(float (&s)[NT][4], float (&dp)[NT][4], uint32_t a, uint32_t b, const Operands& x, const Scoring& sc, uint64_t real) {
  if (sc.cap == 0.f) return;
  scores<T, DT, NT>(s, a, b, x.pitch, x.dim);
  cap_slope<NT>(dp, s, sc);
  set_columns<NT>(dp, real, 0.f);
}
// A segment whose keys are one chunk: everything of the tile's rows at once.
template <typename T, int DT, int NT>
__device__ __forceinline__ void rows_at_once(float (&acc)[DT / 8][4], float3 (&st)[2], float (&bound)[2], const Operands& x, const Scoring& sc, uint64_t keys) {
  float s[NT][4], dp[NT][4];
  products<T, DT, NT>(s, dp, x, keys);
  transform<NT>(s, sc, x.bias, x.index, x.pitch_idx, keys);
  RowSums f;
  f.start();
  sum_rows<NT>(f, s, dp);
  st[0] = row_stats(f, 0, &bound[0]);
  st[1] = row_stats(f, 1, &bound[1]);
  differ_weights<NT>(s, dp, st);
  through_cap<T, DT, NT>(s, dp, x.q, x.ck, x, sc, keys);
  weigh<T, DT, NT, kWide<T>>(acc, dp, x.ck, x.pitch, x.dim);
}
template <typename T, int DT, int NT>
__device__ __forceinline__ void rows_first(RowSums& f, const Operands& x, const Scoring& sc, uint64_t keys) {
  float s[NT][4], dp[NT][4];
  products<T, DT, NT>(s, dp, x, keys);
  transform<NT>(s, sc, x.bias, x.index, x.pitch_idx, keys);
  sum_rows<NT>(f, s, dp);
}
template <typename T, int DT, int NT>
__device__ __forceinline__ void rows_second(float (&acc)[DT / 8][4], const float3 (&st)[2], const Operands& x, const Scoring& sc, uint64_t keys) {
  float s[NT][4], dp[NT][4];
  products<T, DT, NT>(s, dp, x, keys);
  transform<NT>(s, sc, x.bias, x.index, x.pitch_idx, keys);
  differ_rows<NT>(s, dp, st);
  through_cap<T, DT, NT>(s, dp, x.q, x.ck, x, sc, keys);
  weigh<T, DT, NT, kWide<T>>(acc, dp, x.ck, x.pitch, x.dim);
}
// By keys.  `rows`: bit i says whether row i of the tile holds a voxel.
template <typename T, int DT, int NT, bool ROWS>
__device__ __forceinline__ void columns(float (&dk)[DT / 8][4], float (&dv)[DT / 8][4], const Operands& x, const Scoring& sc, const ColumnStats& stats, uint64_t queries,
                                        const Tally& tally, int h, uint32_t rows) {
  float s[NT][4], dp[NT][4];
  int bk[NT][4];
  scores<T, DT, NT>(s, x.k, x.cq, x.pitch, x.dim);
  scores<T, DT, NT>(dp, x.v, x.co, x.pitch, x.dim);
  score_tiles<NT, ROWS>(s, bk, sc, x.bias, x.index, x.pitch_idx);
  differ_columns<NT>(s, dp, stats);
  set_columns<NT>(s, queries, 0.f);  // (whatever lies there)
  set_columns<NT>(dp, queries, 0.f);
  if (tally.on) {
    const uint64_t full = ((uint64_t)1 << (8 * NT)) - 1;
    if (ROWS && rows == 0xffffu && (queries & full) == full) {  // (of short segments hardly a tile is full: no code of its own)
      tally.count<NT, false>(h, bk, dp, 0u);
    } else {  // what lies in other rows and columns does not count
      const int g = (threadIdx.x & 31) >> 2, q2 = (threadIdx.x & 3) * 2;
      const uint32_t r0 = rows >> g & 1, r1 = rows >> (g + 8) & 1;
      uint32_t which = 0;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const uint32_t c = (uint32_t)(queries >> (8 * t + q2)) & 3u;
        which |= ((r0 ? c : 0u) | (r1 ? c << 2 : 0u)) << (4 * t);
      }
      tally.count<NT, true>(h, bk, dp, which);
    }
  }
  weigh<T, DT, NT, false>(dv, s, x.co, x.pitch, x.dim);
  through_cap<T, DT, NT>(s, dp, x.k, x.cq, x, sc, queries);
  weigh<T, DT, NT, kWide<T>>(dk, dp, x.cq, x.pitch, x.dim);
}

// ---- short segments ------------------------------------------------------------------------------------------------
struct BackLayout {
  ShortLayout s;
  int copies;  // of the tally
  uint32_t stats, hist, spoilt, bytes;
};
// As many tables of a tally, up to four, as fit into `room` bytes.
static int tally_copies(int bytes, int room) { return 4 * bytes <= room ? 4 : 2 * bytes <= room ? 2 : 1; }

template <typename T, int DT>
static BackLayout back_layout(const SegArgs& a, int limit, int batch) {
  BackLayout l = {};
  l.s = short_layout<T>(a, kBackHeads<T, DT>, limit, 4, batch);
  uint32_t at = l.s.bytes;
  l.stats = at; at += l.s.heads * 3 * (l.s.batch + 16) * 4;
  if (a.dbias) {
    l.copies = tally_copies(l.s.heads * 2 * a.buckets * 4, 16 * 1024);
    l.hist = at; at += l.copies * l.s.heads * 2 * a.buckets * 4;
    l.spoilt = at; at += (l.s.heads * a.buckets + 31) / 32 * 4;
  }
  l.bytes = (at + 15) / 16 * 16;
  return l;
}

template <typename T, int DT>
__global__ void __launch_bounds__(kThreads, DT <= 32 ? 2 : 1) short_backward_kernel(const __grid_constant__ SegArgs a, const BackLayout L, const Scoring sc, const BackWork work) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int HG = kBackHeads<T, DT>;
  const int dim = kExact<DT> ? DT : a.dim;
  __shared__ uint32_t block_bound;
  pdl_enter();
  Plan& plan = *reinterpret_cast<Plan*>(smem);
  uint16_t* maps = reinterpret_cast<uint16_t*>(smem + L.s.maps);
  float* bias = reinterpret_cast<float*>(smem + L.s.bias);
  int4* cells = reinterpret_cast<int4*>(smem + L.s.cells);
  uint16_t* index = reinterpret_cast<uint16_t*>(smem + L.s.index);
  float* stats = reinterpret_cast<float*>(smem + L.stats);  // [heads][3][stat_rows]
  const int stat_rows = L.s.batch + 16;
  const int head0 = blockIdx.y * HG, heads = min(HG, a.heads - head0);
  const uint32_t pitch = kExact<DT> ? HG * DT * sizeof(T) + 16 : L.s.pitch;
  const uint32_t q0 = smem_u32(smem + L.s.rows), k0 = q0 + L.s.array, v0 = k0 + L.s.array, o0 = v0 + L.s.array;
  Tally tally;
  tally.hist = reinterpret_cast<int*>(smem + L.hist);
  tally.spoilt = reinterpret_cast<uint32_t*>(smem + L.spoilt);
  tally.buckets = a.buckets;
  tally.copies = L.copies;
  tally.copy = HG * 2 * a.buckets;
  tally.on = a.dbias != nullptr;
  tally.bound(0.f);
  StartCheck<kThreads> starts;
  starts.begin(a);
  stage_tables<kThreads>(a, maps, bias, head0, HG);
  float* mine = work.partial + (int64_t)blockIdx.x * work.table + head0 * a.buckets;
  if (tally.on) {
    tally.clear_all<kThreads>(HG);
    // what the long segments' kernels add to starts at zero
    const int first = (blockIdx.y * gridDim.x + blockIdx.x) * kThreads + threadIdx.x, step = gridDim.x * gridDim.y * kThreads;
    for (int i = first; i < 2 * work.table; i += step) work.total[i] = 0;
    for (int i = first; i < (work.table + 31) / 32; i += step) work.spoilt[i] = 0;
    for (int i = first; i < work.launches; i += step) work.bounds[i] = 0;
  }
  starts.end(a);
  bool emptied = false;
  int pending = 0;
  auto empty = [&]() {  // all threads; a barrier before and after
    for (int i = threadIdx.x; i < heads * a.buckets; i += kThreads) {
      long long hi, lo;
      const bool spoilt = tally.take(i, hi, lo);
      const float v = tally_value(hi, lo, tally.to_hi), sum = emptied ? mine[i] + v : v;
      mine[i] = spoilt ? NAN : sum;
    }
    emptied = true;
    pending = 0;
  };
  const int chunks = HG * dim * (int)sizeof(T) / 16, real = heads * dim * (int)sizeof(T) / 16;
  const int64_t col = (int64_t)head0 * dim;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, h = warp % HG, g = lane >> 2;
  const uint32_t at_head = h * dim * sizeof(T);
  const Rows<4> src = {{first_head<T>(a.q, col), first_head<T>(a.k, col), first_head<T>(a.v, col), first_head<T>(a.d_out, col)},
                       {a.ld_q * (int64_t)sizeof(T), a.ld_k * (int64_t)sizeof(T), a.ld_v * (int64_t)sizeof(T), a.ld_do * (int64_t)sizeof(T)}};
  Operands x = {};
  x.bias = bias + h * a.buckets;
  x.pitch_idx = L.s.pitch_idx; x.pitch = pitch; x.dim = dim;
  for (int r = blockIdx.x; r < L.s.ranges; r += gridDim.x) {
    __syncthreads();
    const Range range = start_range<kThreads>(a, plan, r, L.s.ranges, L.s.per);
    while (next_batch<kThreads>(a, plan, range, L.s.limit, L.s.batch)) {
      if (threadIdx.x == 0) block_bound = 0;
      if (a.bias) {
        load_cells<kThreads>(a, smem_u32(cells), plan.ids, plan.rows);
        cp_commit();
      }
      load_rows<T, kThreads, 4>(q0, L.s.array, pitch, src, plan.ids, plan.rows, chunks, real);
      cp_commit();
      if (a.bias) {
        cp_wait<1>();
        __syncthreads();
        fill_index<kThreads>(a, plan, cells, maps, index, L.s.pitch_idx);
      }
      cp_wait<0>();
      __syncthreads();
      if (h < heads) {
        float most = 0.f;
        for (int it = warp / HG; it < plan.items; it += kWarps / HG) {
          const Item item = plan.item[it];
          const int row = item.at + 16 * item.tile, r0 = 16 * item.tile + g;
          x.q = q0 + row * pitch + at_head; x.o = o0 + row * pitch + at_head;
          auto to_chunk = [&](int j) {
            const uint32_t at = (item.at + j) * pitch + at_head;
            x.ck = k0 + at; x.cv = v0 + at;
            x.index = index + row * L.s.pitch_idx + j;
          };
          float acc[DT / 8][4], bound[2];
          float3 st[2];
          clear<DT>(acc);
          to_chunk(0);
          if (item.len <= 40) {
            const uint64_t keys = real_rows(plan, item.at, item.len);
            switch ((item.len + 7) >> 3) {
              case 1: rows_at_once<T, DT, 1>(acc, st, bound, x, sc, keys); break;
              case 2: rows_at_once<T, DT, 2>(acc, st, bound, x, sc, keys); break;
              case 3: rows_at_once<T, DT, 3>(acc, st, bound, x, sc, keys); break;
              case 4: rows_at_once<T, DT, 4>(acc, st, bound, x, sc, keys); break;
              default: rows_at_once<T, DT, 5>(acc, st, bound, x, sc, keys);
            }
          } else {
            RowSums f;
            f.start();
            const int tiles = (item.len + 7) >> 3;
            for (int pass = 0; pass < 2; ++pass) {  // two tiles at a time
              for (int j = 0; j < item.len; j += 16) {
                const int now = min(2, tiles - (j >> 3));
                const uint64_t keys = real_rows(plan, item.at + j, min(8 * now, item.len - j));
                to_chunk(j);
                if (pass == 0) {
                  if (now == 2) rows_first<T, DT, 2>(f, x, sc, keys);
                  else rows_first<T, DT, 1>(f, x, sc, keys);
                } else {
                  if (now == 2) rows_second<T, DT, 2>(acc, st, x, sc, keys);
                  else rows_second<T, DT, 1>(acc, st, x, sc, keys);
                }
              }
              if (pass == 0) {
                st[0] = row_stats(f, 0, &bound[0]);
                st[1] = row_stats(f, 1, &bound[1]);
              }
            }
          }
          const int id0 = r0 < item.len ? plan.ids[item.at + r0] : -1, id1 = r0 + 8 < item.len ? plan.ids[item.at + r0 + 8] : -1;
          if (id0 >= 0) most = fmaxf(most, bound[0]);
          if (id1 >= 0) most = fmaxf(most, bound[1]);
          if ((lane & 3) == 0) {
            float* to = stats + 3 * h * stat_rows + row + g;
            if (r0 < item.len) { to[0] = st[0].x; to[stat_rows] = st[0].y; to[2 * stat_rows] = st[0].z; }
            if (r0 + 8 < item.len) { to[8] = st[1].x; to[stat_rows + 8] = st[1].y; to[2 * stat_rows + 8] = st[1].z; }
          }
          store_rows<T, DT>(acc, a.scale, a.dq, a.ld_dq, col + h * dim, dim, id0, id1);
        }
        if (tally.on) {
          for (int m = 16; m > 0; m >>= 1) most = fmaxf(most, __shfl_xor_sync(kAll, most, m));
          if (lane == 0) atomicMax(&block_bound, __float_as_uint(most));
        }
      }
      __syncthreads();
      if (tally.on) {
        const int pairs = plan.pairs;
        const float b = __uint_as_float(block_bound);
        if (2.f * b > tally.limit || pending + pairs > kMaxPending) {  // (a value of the second pass may round to more than the bound)
          if (pending > 0) empty();
          if (2.f * b > tally.limit) tally.bound(b);
          __syncthreads();
        }
        pending += pairs;
      }
      if (h < heads) {
        for (int it = warp / HG; it < plan.items; it += kWarps / HG) {
          const Item item = plan.item[it];
          const int row = item.at + 16 * item.tile, r0 = 16 * item.tile + g;
          const int id0 = r0 < item.len ? plan.ids[item.at + r0] : -1, id1 = r0 + 8 < item.len ? plan.ids[item.at + r0 + 8] : -1;
          float dk[DT / 8][4], dv[DT / 8][4];
          clear<DT>(dk);
          clear<DT>(dv);
          x.k = k0 + row * pitch + at_head; x.v = v0 + row * pitch + at_head;
          const uint32_t tile_rows = (uint32_t)real_rows(plan, row, min(16, item.len - 16 * item.tile));
          // (Two tiles at a time and not four: half the code and fewer registers.  Kernels of this size miss in the instruction cache: 32,000
          // pillars bf16 148 us with four, 127 with two; fp32, 12,345 with a cap, 352 and 255.  With two, 16-bit types spill
          // no registers; fp32 stores 64, 300 and 932 bytes of them at 16, 24 and 32 channels a head.)
          for (int j = 0; j < item.len; j += 16) {
            const int cols = min(16, item.len - j);
            const uint64_t queries = real_rows(plan, item.at + j, cols);
            const uint32_t at = (item.at + j) * pitch + at_head;
            const ColumnStats from = {stats + 3 * h * stat_rows + item.at + j, stat_rows};
            x.cq = q0 + at; x.co = o0 + at;
            x.index = index + (item.at + j) * L.s.pitch_idx + 16 * item.tile;
            if (cols > 8) columns<T, DT, 2, false>(dk, dv, x, sc, from, queries, tally, h, tile_rows);
            else columns<T, DT, 1, false>(dk, dv, x, sc, from, queries, tally, h, tile_rows);
          }
          store_rows<T, DT>(dk, a.scale, a.dk, a.ld_dk, col + h * dim, dim, id0, id1);
          store_rows<T, DT>(dv, 1.f, a.dv, a.ld_dv, col + h * dim, dim, id0, id1);
        }
      }
      if (plan.cursor >= range.end) break;
      __syncthreads();
    }
  }
  if (tally.on) {
    __syncthreads();
    empty();
  }
}

// ---- long segments -------------------------------------------------------------------------------------------------
template <typename T, int DT>
struct BackShape {
  static constexpr int HG = DT * sizeof(T) <= 64 ? 4 : DT * sizeof(T) <= 128 ? 2 : 1, WH = HG < 2 ? HG : 2, HPW = HG / WH, rows = 16 * kWarps / WH;
  static constexpr int chunk = sizeof(T) == 2 || DT <= 64 ? 32 : 16, NT = chunk < 32 ? 2 : 4;  // rows that pass at a time; tiles of 8 of them in registers
};

struct BackLongLayout {
  int pitch_idx, copies;
  uint32_t pitch, tile, chunk;
  uint32_t maps, bias, cells, passing_cells, ids, index, stats, hist, spoilt, rows, passing, bytes;
};

template <typename T, int DT>
static BackLongLayout back_long_layout(const SegArgs& a, bool by_keys, int copies = 4) {
  using S = BackShape<T, DT>;
  BackLongLayout l = {};
  l.pitch = (uint32_t)(S::HG * a.dim * sizeof(T) + 16);
  l.tile = S::rows * l.pitch;
  l.chunk = S::chunk * l.pitch;
  uint32_t at = 0;
  auto take = [&](size_t bytes) { const uint32_t was = at; at += (uint32_t)((bytes + 15) / 16 * 16); return was; };
  l.ids = take((size_t)(S::rows + 3 * S::chunk) * 4);
  if (a.bias) {
    l.maps = take(sizeof(a.maps.of));
    l.bias = take((size_t)S::HG * a.buckets * 4);
    l.cells = take((size_t)S::rows * 16);
    l.passing_cells = take((size_t)3 * S::chunk * 16);
    l.pitch_idx = S::chunk + 8;
    l.index = take((size_t)(by_keys ? 1 : 2) * S::rows * l.pitch_idx * 2);
  }
  if (by_keys) {
    l.stats = take((size_t)3 * S::HG * 3 * S::chunk * 4);
    if (a.dbias) {
      l.copies = copies;
      l.hist = take((size_t)l.copies * S::HG * 2 * a.buckets * 4);
      l.spoilt = take((size_t)(S::HG * a.buckets + 31) / 32 * 4);
    }
  }
  l.rows = take((size_t)2 * l.tile + 64);
  l.passing = take((size_t)4 * l.chunk + 64);
  l.bytes = at;
  // (as many tables of the tally as leave room for two blocks on an SM)
  return by_keys && a.dbias && copies > 1 && at > kSmemHalf ? back_long_layout<T, DT>(a, by_keys, copies / 2) : l;
}

// A tile of a long segment's queries (BY_KEYS: keys) against all of the segment's keys (queries).
template <typename T, int DT, bool BY_KEYS>
__global__ void __launch_bounds__(kThreads, DT <= 32 ? 2 : 1) long_backward_kernel(const __grid_constant__ SegArgs a, const BackLongLayout L, const Scoring sc, const BackWork work, int above) {
  extern __shared__ __align__(16) unsigned char smem[];
  using S = BackShape<T, DT>;
  constexpr int NT = S::NT, HPW = S::HPW;
  __shared__ Tile tiles[kMaxTiles];
  __shared__ int tile_count;
  const int dim = kExact<DT> ? DT : a.dim;
  pdl_enter();
  const int found = find_tiles(a, tiles, &tile_count, blockIdx.x * S::rows, S::rows, above);
  if (found == 0) return;
  uint16_t* maps = reinterpret_cast<uint16_t*>(smem + L.maps);
  float* bias = reinterpret_cast<float*>(smem + L.bias);
  int4* cells = reinterpret_cast<int4*>(smem + L.cells);
  uint16_t* index = reinterpret_cast<uint16_t*>(smem + L.index);
  int32_t* ids = reinterpret_cast<int32_t*>(smem + L.ids);
  const int head0 = work.head0 + blockIdx.y * S::HG, heads = min(S::HG, work.head_end - head0);
  const uint32_t pitch = kExact<DT> ? S::HG * DT * sizeof(T) + 16 : L.pitch;
  const uint32_t own0 = smem_u32(smem + L.rows), own1 = own0 + L.tile;
  Tally tally;
  tally.hist = reinterpret_cast<int*>(smem + L.hist);
  tally.spoilt = reinterpret_cast<uint32_t*>(smem + L.spoilt);
  tally.buckets = a.buckets;
  tally.copies = L.copies;
  tally.copy = S::HG * 2 * a.buckets;
  tally.on = BY_KEYS && a.dbias != nullptr;
  if (tally.on) {
    tally.bound(__uint_as_float(work.bounds[work.head0 / work.at_once]));
    tally.clear_all<kThreads>(S::HG);
  }
  auto empty = [&]() {  // all threads; a barrier before and after
    for (int i = threadIdx.x; i < heads * a.buckets; i += kThreads) {
      long long hi, lo;
      const int w = head0 * a.buckets + i;
      if (tally.take(i, hi, lo)) atomicOr(work.spoilt + (w >> 5), 1u << (w & 31));
      if (hi) atomicAdd(work.total + w, (unsigned long long)hi);
      if (lo) atomicAdd(work.total + w + work.table, (unsigned long long)lo);
    }
  };
  stage_tables<kThreads>(a, maps, bias, head0, S::HG);
  const int chunks = S::HG * dim * (int)sizeof(T) / 16, real = heads * dim * (int)sizeof(T) / 16;
  const int64_t col = (int64_t)head0 * dim;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2;
  const int row = 16 * (warp / S::WH);
  const Rows<2> by_q = {{first_head<T>(a.q, col), first_head<T>(a.d_out, col)}, {a.ld_q * (int64_t)sizeof(T), a.ld_do * (int64_t)sizeof(T)}};
  const Rows<2> by_k = {{first_head<T>(a.k, col), first_head<T>(a.v, col)}, {a.ld_k * (int64_t)sizeof(T), a.ld_v * (int64_t)sizeof(T)}};
  const Rows<2>&own = BY_KEYS ? by_k : by_q, &passing = BY_KEYS ? by_q : by_k;
  float most = 0.f;
  for (int ti = 0; ti < found; ++ti) {
    const Tile tile = tiles[ti];
    const int rows = min(S::rows, tile.hi - tile.row);
    const int parts = (tile.hi - tile.lo + S::chunk - 1) / S::chunk;
    auto ids_of = [&](int c) { return ids + S::rows + c % 3 * S::chunk; };
    auto cells_of = [&](int c) { return reinterpret_cast<int4*>(smem + L.passing_cells) + c % 3 * S::chunk; };
    auto stats_of = [&](int c) { return reinterpret_cast<float*>(smem + L.stats) + c % 3 * (S::HG * 3 * S::chunk); };  // [heads][3][chunk]
    auto array = [&](int c, int which) { return smem_u32(smem + L.passing) + ((c & 1) * 2 + which) * L.chunk; };
    // Rows of whole tiles and chunks are dealt out, so that the 8 rows and 4 columns of a score tile that a warp counts at once lie apart:
    // neighbours' displacements would meet in the same bucket, and additions to one address follow one another.
    auto dealt = [&](int place, int count) { return BY_KEYS ? place % 8 * (count / 8) + place / 8 : place; };
    __syncthreads();  // (the tile before is done with the shared memory)
    if (threadIdx.x < S::rows) {
      const int at = rows == S::rows ? dealt(threadIdx.x, S::rows) : threadIdx.x;
      const int id = at < rows ? voxel_at(a, tile.row + at) : -1;
      ids[threadIdx.x] = id;
      if (a.bias) cells[threadIdx.x] = id >= 0 ? a.coords[id] : make_int4(0, 0, 0, 0);
    }
    auto chunk_row = [&](int c, int place) {
      const int from = tile.lo + c * S::chunk;
      return from + (from + S::chunk <= tile.hi ? dealt(place, S::chunk) : place);
    };
    int next = -1;  // this thread's voxel of the next chunk
    auto fetch_id = [&](int c) {
      next = -1;
      if (threadIdx.x < S::chunk) {
        const int at = chunk_row(c, threadIdx.x);
        if (at < tile.hi) next = voxel_at(a, at);
      }
    };
    auto publish = [&](int c) {
      if (threadIdx.x < S::chunk) {
        ids_of(c)[threadIdx.x] = next;
        if (a.bias) cells_of(c)[threadIdx.x] = next >= 0 ? a.coords[next] : make_int4(0, 0, 0, 0);
      }
      if (BY_KEYS)
        for (int i = threadIdx.x; i < heads * S::chunk; i += kThreads) {
          const int h = i / S::chunk, j = i % S::chunk, at = chunk_row(c, j);
          const float* from = work.stats + ((int64_t)(head0 - work.head0 + h) * work.n + at) * 3;
#pragma unroll
          for (int k = 0; k < 3; ++k) stats_of(c)[(3 * h + k) * S::chunk + j] = at < tile.hi ? from[k] : 0.f;
        }
    };
    auto load = [&](int c) {
      load_rows<T, kThreads, 2>(array(c, 0), L.chunk, pitch, passing, ids_of(c), S::chunk, chunks, real);
      cp_commit();
    };
    RowSums f[BY_KEYS ? 1 : HPW];
    float3 st[BY_KEYS ? 1 : HPW][2];
    float acc[HPW][DT / 8][4], dv[BY_KEYS ? HPW : 1][DT / 8][4];
#pragma unroll
    for (int i = 0; i < HPW; ++i) {
      if (!BY_KEYS) f[i].start();
      clear<DT>(acc[i]);
      if (BY_KEYS) clear<DT>(dv[i]);
    }
    // (by queries a chunk's buckets are looked up while the one before is worked on; by keys the tally takes that room)
    auto index_of = [&](int c) { return BY_KEYS ? index : index + (c & 1) * S::rows * L.pitch_idx; };
    auto look_up = [&](int c) {
      if (!a.bias) return;
      uint16_t* to = index_of(c);
      const int4* passing_cells = cells_of(c);
      for (int i = threadIdx.x; i < S::rows * S::chunk; i += kThreads) {
        const int r = i / S::chunk, j = i % S::chunk;
        to[r * L.pitch_idx + j] = (uint16_t)(BY_KEYS ? bucket_at(a.maps, maps, passing_cells[j], cells[r]) : bucket_at(a.maps, maps, cells[r], passing_cells[j]));
      }
    };
    int pending = 0;
    for (int sweep = BY_KEYS ? 1 : 0; sweep < 2; ++sweep) {
      fetch_id(0);
      __syncthreads();
      publish(0);
      fetch_id(1);
      __syncthreads();
      if (BY_KEYS || sweep == 0) {
        load_rows<T, kThreads, 2>(own0, L.tile, pitch, own, ids, S::rows, chunks, real);
      }
      load(0);
      if (!BY_KEYS) look_up(0);
      for (int c = 0; c < parts; ++c) {
        const int all = min(S::chunk, tile.hi - tile.lo - c * S::chunk);
        if (c + 1 < parts) publish(c + 1);
        cp_wait<0>();
        __syncthreads();  // this chunk and its buckets are there, the other one's buffers free
        if (c + 1 < parts) {
          load(c + 1);
          fetch_id(c + 2);
          if (!BY_KEYS) look_up(c + 1);
        }
        if (tally.on && pending + S::rows * S::chunk > kMaxPending) {
          empty();
          pending = 0;
        }
        pending += S::rows * S::chunk;
        if (BY_KEYS && a.bias) {  // (counting without a bias there is none)
          look_up(c);
          __syncthreads();
        }
        const uint64_t there = __ballot_sync(kAll, lane < S::chunk && ids_of(c)[lane] >= 0);
        const uint32_t tile_rows = BY_KEYS ? __ballot_sync(kAll, lane < 16 && ids[row + lane] >= 0) : 0u;
#pragma unroll
        for (int i = 0; i < HPW; ++i) {
          const int h = (warp % S::WH) * HPW + i;
          if (h >= heads || row >= rows) continue;
          const uint32_t at_head = h * dim * sizeof(T);
          Operands x = {};
          x.bias = bias + h * a.buckets;
          x.pitch_idx = L.pitch_idx; x.pitch = pitch; x.dim = dim;
          x.q = x.k = own0 + row * pitch + at_head;
          x.o = x.v = own1 + row * pitch + at_head;
          for (int j = 0; j < all; j += 8 * NT) {
            const uint64_t bits = there >> j & (((uint64_t)1 << (8 * NT)) - 1);
            x.cq = x.ck = array(c, 0) + j * pitch + at_head;
            x.co = x.cv = array(c, 1) + j * pitch + at_head;
            x.index = index_of(c) + row * L.pitch_idx + j;
            if constexpr (BY_KEYS) {
              columns<T, DT, NT, true>(acc[i], dv[i], x, sc, ColumnStats{stats_of(c) + 3 * h * S::chunk + j, S::chunk}, bits, tally, h, tile_rows);
            } else {
              if (sweep == 0) rows_first<T, DT, NT>(f[i], x, sc, bits);
              else rows_second<T, DT, NT>(acc[i], st[i], x, sc, bits);
            }
          }
        }
      }
      if (!BY_KEYS && sweep == 0) {
#pragma unroll
        for (int i = 0; i < HPW; ++i) {
          const int h = (warp % S::WH) * HPW + i;
          float bound[2];
          st[i][0] = row_stats(f[i], 0, &bound[0]);
          st[i][1] = row_stats(f[i], 1, &bound[1]);
          if (h < heads && row < rows)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              if (ids[row + g + 8 * r] < 0) continue;
              most = fmaxf(most, bound[r]);
              if ((lane & 3) == 0) {
                float* to = work.stats + ((int64_t)(head0 - work.head0 + h) * work.n + tile.row + row + g + 8 * r) * 3;
                to[0] = st[i][r].x; to[1] = st[i][r].y; to[2] = st[i][r].z;
              }
            }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < HPW; ++i) {
      const int h = (warp % S::WH) * HPW + i;
      if (h >= heads || row >= rows) continue;
      const int id0 = ids[row + g], id1 = ids[row + g + 8];
      store_rows<T, DT>(acc[i], a.scale, BY_KEYS ? a.dk : a.dq, BY_KEYS ? a.ld_dk : a.ld_dq, col + h * dim, dim, id0, id1);
      if (BY_KEYS) store_rows<T, DT>(dv[i], 1.f, a.dv, a.ld_dv, col + h * dim, dim, id0, id1);
    }
    if (tally.on) {
      __syncthreads();
      empty();
    }
  }
  if (!BY_KEYS && a.dbias) {
    for (int m = 16; m > 0; m >>= 1) most = fmaxf(most, __shfl_xor_sync(kAll, most, m));
    if (lane == 0 && most > 0.f) atomicMax(work.bounds + work.head0 / work.at_once, __float_as_uint(most));
  }
}

// dbias: the blocks' partial sums in a fixed order, and the long segments' integers.  32 entries to a block, a warp a share of the blocks.
constexpr int kGradThreads = 1024;  // (256: 8 us for 148 blocks' sums, most of it the loads' latency)
static __global__ void __launch_bounds__(kGradThreads) bias_grad_kernel(const BackWork work, int buckets, bool longer, float* dbias) {
  __shared__ float part[kGradThreads / 32][33];
  pdl_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, at = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (at < work.table)
#pragma unroll 8
    for (int p = warp; p < work.blocks; p += kGradThreads / 32) s += work.partial[(int64_t)p * work.table + at];
  part[warp][lane] = s;
  __syncthreads();
  s = part[lane][warp];  // a warp adds up one entry
  for (int m = 16; m > 0; m >>= 1) s += __shfl_xor_sync(kAll, s, m);
  const int mine = blockIdx.x * 32 + warp;
  if (lane != 0 || mine >= work.table) return;
  if (longer) {
    Tally t;
    t.bound(__uint_as_float(work.bounds[mine / buckets / work.at_once]));
    s += tally_value((long long)work.total[mine], (long long)work.total[mine + work.table], t.to_hi);
    if (work.spoilt[mine >> 5] >> (mine & 31) & 1) s = NAN;
  }
  dbias[mine] = s;
}

template <typename T, int DT>
int backward_of(dsvt_ctx* ctx, const SegArgs& a) {
  int limit = a.max_len <= kShortBack ? a.max_len : 64;
  // the largest batch that leaves room for two blocks on an SM (32,000 pillars bf16: 64 rows 103 us, 80 rows 97), if one does
  int batch = 96;
  BackLayout l = back_layout<T, DT>(a, limit, batch);
  while (l.bytes > kSmemHalf && batch > 48) l = back_layout<T, DT>(a, limit, batch -= 8);
  if (l.bytes > kSmemMost) l = back_layout<T, DT>(a, limit = 64, batch);  // (some heads of fp32 and large biases, from 81 rows on; 64 always fit)
  const Scoring sc = scoring_of(a);
  const int groups = (int)dsvt_ceil_div(a.heads, kBackHeads<T, DT>);
  BackWork w = {};
  uint32_t* base = reinterpret_cast<uint32_t*>(ctx->bm_zero);
  w.partial = reinterpret_cast<float*>(base);
  w.total = reinterpret_cast<unsigned long long*>(base + kPartialWords);
  w.spoilt = base + kPartialWords + kTotalWords;
  w.bounds = w.spoilt + kMaxBiasTable / 32;
  w.stats = reinterpret_cast<float*>(w.bounds + kMaxHeads);
  const int64_t stat_words = (int64_t)(4 * ctx->bm_words) - (w.stats - reinterpret_cast<float*>(base));
  w.table = a.dbias ? a.heads * a.buckets : 0;
  w.n = a.n;
  // blocks that stay: two to an SM where they fit, and as many as have room for their partial sums
  const int per_sm = DT <= 32 && l.bytes <= kSmemHalf ? 2 : 1;
  int64_t stay = dsvt_ceil_div(per_sm * ctx->sm_count, groups);
  if (w.table > 0 && stay > (int64_t)kPartialWords / w.table) stay = kPartialWords / w.table;
  set_ranges(l.s, a.n, (int)stay, limit < a.max_len ? 128 : 1 << 20);
  if (stay > l.s.ranges) stay = l.s.ranges;
  w.blocks = (int)stay;
  // as many heads to a launch of the long ones as the workspace has room for the statistics of, whole blocks' if it can be
  const bool longer = limit < a.max_len;
  using S = BackShape<T, DT>;
  int64_t at_once = stat_words / ((int64_t)3 * a.n);
  if (longer && at_once < 1) return DSVT_ERR_CAPACITY;
  if (at_once > S::HG) at_once = at_once / S::HG * S::HG;
  w.at_once = (int)(at_once < 1 ? 1 : at_once < a.heads ? at_once : a.heads);
  w.launches = (int)dsvt_ceil_div(a.heads, w.at_once);
  constexpr auto kernel = short_backward_kernel<T, DT>;
  int rc = allow_smem<kernel>(ctx, kSmemMost);
  if (rc != DSVT_OK) return rc;
  launch_pdl(kernel, dim3((unsigned)stay, groups), dim3(kThreads), l.bytes, ctx->stream, a, l, sc, w);
  DSVT_LAUNCHED(ctx);
  if (longer) {
    const BackLongLayout lq = back_long_layout<T, DT>(a, false), lk = back_long_layout<T, DT>(a, true);
    constexpr auto by_queries = long_backward_kernel<T, DT, false>;
    constexpr auto by_keys = long_backward_kernel<T, DT, true>;
    if ((rc = allow_smem<by_queries>(ctx, kSmemMost)) != DSVT_OK || (rc = allow_smem<by_keys>(ctx, kSmemMost)) != DSVT_OK) return rc;
    for (int h = 0; h < a.heads; h += w.at_once) {
      w.head0 = h;
      w.head_end = h + w.at_once < a.heads ? h + w.at_once : a.heads;
      const dim3 grid((unsigned)dsvt_ceil_div(a.n, S::rows), (unsigned)dsvt_ceil_div(w.head_end - h, S::HG));
      launch_pdl(by_queries, grid, dim3(kThreads), lq.bytes, ctx->stream, a, lq, sc, w, limit);
      DSVT_LAUNCHED(ctx);
      launch_pdl(by_keys, grid, dim3(kThreads), lk.bytes, ctx->stream, a, lk, sc, w, limit);
      DSVT_LAUNCHED(ctx);
    }
  }
  if (a.dbias) {
    launch_pdl(bias_grad_kernel, dim3((unsigned)dsvt_ceil_div(w.table, 32)), dim3(kGradThreads), 0, ctx->stream, w, a.buckets, longer, a.dbias);
    DSVT_LAUNCHED(ctx);
  }
  return DSVT_OK;
}

template <typename T>
int launch_backward(dsvt_ctx* ctx, const SegArgs& a) {
  if (a.dim == 16) return backward_of<T, 16>(ctx, a);
  if (a.dim == 24) return backward_of<T, 24>(ctx, a);
  if (a.dim == 32) return backward_of<T, 32>(ctx, a);
  if (a.dim <= 64) return backward_of<T, 64>(ctx, a);
  return backward_of<T, 128>(ctx, a);
}

}  // namespace dsvt_train
