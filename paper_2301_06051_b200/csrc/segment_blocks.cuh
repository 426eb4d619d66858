// Segment attention: what a block works on.  Short segments: all those that start in a block's kRowBlock rows, whole, in shared
// memory.  Long ones: a tile of the rows of one segment, the segment's other rows passing by in chunks.
#pragma once
#include "segment_mma.cuh"

namespace dsvt_train {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kRowBlock = 32;
constexpr int kShort = 128;                         // most rows of a segment that is held whole
constexpr int kBatch = 48;                          // rows in shared memory at a time, or the longest segment's if that is more
constexpr int kMaxItems = kRowBlock * (kShort / 16);

// 16 rows of a segment: its first row's place in the batch, its length, the tile.
struct Item { uint8_t at, len, tile, pad; };

// A block's segments, and the batch of them in shared memory: mostly all of them, else as many as fit.
struct Plan {
  int rows, items, pairs, next;        // of the batch (pairs: of queries and keys); where the next batch starts
  int first;                           // the batch's first row, from the block's
  uint32_t starts;                     // bit i: a segment starts at place i
  uint8_t len_at[kRowBlock];           // by row of the block: length of the segment that starts there
  uint32_t real[kShort / 32 + 3];      // bit i: place i holds a voxel
  int32_t ids[kShort];
  Item item[kMaxItems];
};

// Which entries of seg_start can be of segments that start in rows [from, to): found by 256 probes a round (one for most calls).
// `first`, `last`: nothing lies before or behind the rows.
__device__ __forceinline__ int2 segments_near(const SegArgs& a, int from, int to, bool first, bool last) {
  const int tid = threadIdx.x;
  int lo = 0, hi = a.cap_segments, end = hi;
  if (a.num_segments) { const int m = *a.num_segments; end = m < 0 ? 0 : m < end ? m : end; }
  while (true) {
    const int span = hi - lo, step = (span + kThreads - 1) / kThreads;
    const int64_t i = lo + (int64_t)tid * step;
    const int v = i < hi ? a.seg_start[i] : 0;
    const bool in = i < hi && i < end;
    const int below = __syncthreads_count(in && v < from), upto = __syncthreads_count(in && v < to);
    const int64_t next_hi = lo + (int64_t)upto * step;
    if (!last && next_hi < hi) hi = (int)next_hi;
    if (!first && below > 0) lo += (below - 1) * step;
    if (hi > end) hi = end;
    if (hi - lo <= 8 * kThreads || hi - lo >= span) break;
  }
  return make_int2(lo, hi);
}

// Copies what every block reads: the index tables of the displacements and its heads' bias, in units of log 2.
__device__ __forceinline__ void stage_tables(const SegArgs& a, uint16_t* maps, float* bias, int head0, int heads) {
  if (!a.bias) return;
  for (int i = threadIdx.x; i < a.maps.at_z + 2 * a.maps.extent[2] - 1; i += kThreads) maps[i] = (uint16_t)(4 * a.maps.of[i]);
  const int count = min(heads, a.heads - head0) * a.buckets;
  const float* from = a.bias + (int64_t)head0 * a.buckets;
  for (int i = threadIdx.x; i < count; i += kThreads) bias[i] = bias_log2(from[i]);
}

__device__ __forceinline__ int bucket_at(const BucketMaps& m, const uint16_t* maps, int4 i, int4 j) {
  const int ex = m.extent[0] - 1, ey = m.extent[1] - 1, ez = m.extent[2] - 1;
  const int dx = min(max(i.y - j.y, -ex), ex) + ex, dy = min(max(i.z - j.z, -ey), ey) + ey + m.at_y, dz = min(max(i.w - j.w, -ez), ez) + ez + m.at_z;
  return maps[dx] + maps[dy] + maps[dz];  // (the maps in shared memory hold four times the index: a bias's offset)
}

// Finds the block's segments, of at most `limit` rows.
__device__ __forceinline__ void make_plan(const SegArgs& a, Plan& p, int block, int blocks, int limit) {
  const int tid = threadIdx.x, base = block * kRowBlock;
  if (tid < kRowBlock) p.len_at[tid] = 0;
  if (tid == 0) p.next = 0;
  const int2 near = segments_near(a, base, base + kRowBlock, block == 0, block == blocks - 1);
  for (int s = near.x + tid; s < near.y; s += kThreads) {
    const int lo = a.seg_start[s], hi = a.seg_start[s + 1];
    if (segment_sound(a, lo, hi) && hi - lo <= limit && lo >= base && lo < base + kRowBlock) p.len_at[lo - base] = (uint8_t)(hi - lo);
  }
  __syncthreads();
}

// The next batch of the block's segments, of at most `most` rows together: their rows' voxels and cells and the list of their tiles.
// False if there are no more.  A barrier comes before.
__device__ __forceinline__ bool next_batch(const SegArgs& a, Plan& p, int4* cells, int block, int most) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (warp == 0) {
    const int len = p.len_at[lane];
    const uint32_t left = __ballot_sync(kAll, len > 0 && lane >= p.next);
    const int first = __ffs(left) - 1, at = lane - first;
    const bool in = (left >> lane & 1) && at + len <= most;
    const uint32_t taken = __ballot_sync(kAll, in), rest = left & ~taken;
    const int tiles = in ? (len + 15) >> 4 : 0;
    int rows = in ? at + len : 0, upto = tiles, pairs = in ? len * len : 0;
    for (int m = 1; m < 32; m <<= 1) {
      rows = max(rows, __shfl_xor_sync(kAll, rows, m));
      pairs += __shfl_xor_sync(kAll, pairs, m);
      const int before = __shfl_up_sync(kAll, upto, m);
      if (lane >= m) upto += before;
    }
    for (int t = 0; t < tiles; ++t) p.item[upto - tiles + t] = Item{(uint8_t)at, (uint8_t)len, (uint8_t)t, 0};
    if (lane == 31) p.items = upto;
    if (lane == 0) {
      p.rows = rows;
      p.pairs = pairs;
      p.first = first;
      p.starts = left ? taken >> first : 0u;
      p.next = rest ? __ffs(rest) - 1 : kRowBlock;
    }
  }
  __syncthreads();
  if (p.items == 0) return false;
  if (tid < (int)(sizeof(p.real) / 4) * 32) {
    int id = -1;
    const uint32_t upto = p.starts & (tid >= 31 ? kAll : (2u << tid) - 1u);
    if (tid < p.rows && upto) {
      const int at = 31 - __clz(upto);
      if (tid < at + p.len_at[p.first + at]) id = voxel_at(a, block * kRowBlock + p.first + tid);
    }
    const uint32_t real = __ballot_sync(kAll, id >= 0);
    if (lane == 0) p.real[warp] = real;
    if (tid < kShort) p.ids[tid] = id;
    if (a.bias && id >= 0) cells[tid] = a.coords[id];
  }
  __syncthreads();
  return true;
}

// Bit j: place at + j (j < count <= 64) holds a voxel.
__device__ __forceinline__ uint64_t real_rows(const Plan& p, int at, int count) {
  const int w = at >> 5, s = at & 31;
  const uint64_t lo = (uint64_t)p.real[w] | (uint64_t)p.real[w + 1] << 32;
  uint64_t v = lo >> s;
  if (s) v |= (uint64_t)p.real[w + 2] << (64 - s);
  return count >= 64 ? v : v & (((uint64_t)1 << count) - 1);
}

// Entries to a row of the bucket tile, for segments of at most `cols` rows: rows of an odd multiple of 16 bytes, so that the eight
// rows of a score tile's fragment lie in different banks.
__host__ __device__ constexpr int index_pitch(int cols) { return 8 * (((cols + 7) / 8) | 1); }

// The buckets (times 4) of all pairs of the batch: index[i][j - first of i's segment].  The rest of the tile is never written.
__device__ __forceinline__ void fill_index(const SegArgs& a, const Plan& p, const int4* cells, const uint16_t* maps, uint16_t* index, int pitch) {
  const int part = threadIdx.x & 15;
  for (int i = threadIdx.x >> 4; i < p.rows; i += kThreads / 16) {
    const uint32_t upto = p.starts & (i >= 31 ? kAll : (2u << i) - 1u);
    const int at = upto ? 31 - __clz(upto) : 0, len = p.len_at[p.first + at];
    if (i >= at + len || p.ids[i] < 0) continue;
    const int4 mine = cells[i];
#pragma unroll 3
    for (int j = part; j < len; j += 16) index[i * pitch + j] = (uint16_t)bucket_at(a.maps, maps, mine, cells[at + j]);
  }
}

// Rows' parts of a block's heads to shared memory, N arrays of them: `chunks` pieces of 16 bytes to a row, of which the first `real`
// exist.  Eight threads to a row.
template <int N>
struct Rows {
  const char* from[N];  // at the block's first head
  int64_t ld[N];        // bytes
};
template <typename T, int N>
__device__ __forceinline__ void load_rows(uint32_t to, uint32_t array, uint32_t pitch, const Rows<N>& src, const int32_t* ids, int rows, int chunks, int real) {
  const int part = threadIdx.x & 7;
  for (int r = threadIdx.x >> 3; r < rows; r += kThreads / 8) {
    const int id = ids[r];
    const char* at[N];
#pragma unroll
    for (int i = 0; i < N; ++i) at[i] = src.from[i] + (id < 0 ? 0 : id) * src.ld[i];
    const uint32_t dst = to + r * pitch;
#pragma unroll 4
    for (int c = part; c < chunks; c += 8) {
      const bool in = id >= 0 && c < real;
#pragma unroll
      for (int i = 0; i < N; ++i) cp_async16(dst + i * array + c * 16, at[i] + (in ? c * 16 : 0), in);
    }
  }
}
template <typename T>
__device__ __forceinline__ const char* first_head(const void* p, int64_t col) { return reinterpret_cast<const char*>(p) + col * (int64_t)sizeof(T); }

// Rounds two neighbouring channels into a row in shared or global memory.
template <typename T>
__device__ __forceinline__ void store2(T* to, float x, float y) {
  if constexpr (sizeof(T) == 4) *reinterpret_cast<float2*>(to) = make_float2(x, y);
  else *reinterpret_cast<uint32_t*>(to) = Mma<T>::pack(x, y);
}

constexpr uint32_t kBucketMask = 4 * (kMaxBuckets - 1);
// The buckets of a tile's four pairs, times 4; `index`: at its first row and column.
__device__ __forceinline__ void buckets_of(int (&bk)[4], const uint16_t* index, int pitch) {
  const int lane = threadIdx.x & 31;
  const uint16_t* at = index + (lane >> 2) * pitch + (lane & 3) * 2;
  const uint32_t i0 = *reinterpret_cast<const uint32_t*>(at), i1 = *reinterpret_cast<const uint32_t*>(at + 8 * pitch);
  // (kept in range: where a row or column of the tile lies beyond the segment, nothing may have been written)
  bk[0] = i0 & kBucketMask; bk[1] = i0 >> 16 & kBucketMask; bk[2] = i1 & kBucketMask; bk[3] = i1 >> 16 & kBucketMask;
}
__device__ __forceinline__ float bias_at(const float* bias, int bk) { return *reinterpret_cast<const float*>(reinterpret_cast<const char*>(bias) + bk); }

// A tile of scores of queries (rows) and keys (columns) from products; -inf where a column holds no key.
template <bool SLOPE>
__device__ __forceinline__ void score_tile(float (&s)[4], float (&slope)[4], const Scoring& sc, const float* bias, const uint16_t* index, int pitch, uint32_t bits) {
  float b[4] = {};
  if (sc.bias) {
    int bk[4];
    buckets_of(bk, index, pitch);
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = bias_at(bias, bk[e]);
  }
  score_of<SLOPE>(sc, s, b, slope);
  if ((bits & 0xffu) != 0xffu) {
    const uint32_t mine = bits >> ((threadIdx.x & 3) * 2);
    if (!(mine & 1)) {
      s[0] = s[2] = -INFINITY;
      if (SLOPE) slope[0] = slope[2] = 0.f;
    }
    if (!(mine & 2)) {
      s[1] = s[3] = -INFINITY;
      if (SLOPE) slope[1] = slope[3] = 0.f;
    }
  }
}

// Sets the columns that hold no row.  Without gaps only the last tile has some.
template <int NT>
__device__ __forceinline__ void set_columns(float (&c)[NT][4], uint64_t real, float to) {
  constexpr uint64_t before = ((uint64_t)1 << (8 * (NT - 1))) - 1;
  const int q2 = (threadIdx.x & 3) * 2;
  if ((real & before) != before) {
    const uint64_t mine = real >> q2;
#pragma unroll
    for (int t = 0; t < NT - 1; ++t) {
      if (!(mine >> (8 * t) & 1)) c[t][0] = c[t][2] = to;
      if (!(mine >> (8 * t + 1) & 1)) c[t][1] = c[t][3] = to;
    }
  }
  const uint32_t last = (uint32_t)(real >> (8 * (NT - 1))) >> q2;
  if (!(last & 1)) c[NT - 1][0] = c[NT - 1][2] = to;
  if (!(last & 2)) c[NT - 1][1] = c[NT - 1][3] = to;
}

// `index`: the fragment's first row's buckets at the chunk's first column (rows g and g + 8 of the tile).
template <int NT>
__device__ __forceinline__ void transform(float (&s)[NT][4], const Scoring& sc, const float* bias, const uint16_t* index, int pitch, uint64_t real) {
  float b[NT][4];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    b[t][0] = b[t][1] = b[t][2] = b[t][3] = 0.f;
    if (sc.bias) {
      int bk[4];
      buckets_of(bk, index + t * 8, pitch);
#pragma unroll
      for (int e = 0; e < 4; ++e) b[t][e] = bias_at(bias, bk[e]);
    }
  }
  float none[4];
#pragma unroll
  for (int t = 0; t < NT; ++t) score_of<false>(sc, s[t], b[t], none);
  set_columns<NT>(s, real, -INFINITY);
}

__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, __shfl_xor_sync(kAll, v, 1));
  return fmaxf(v, __shfl_xor_sync(kAll, v, 2));
}
__device__ __forceinline__ float quad_sum(float v) {
  v += __shfl_xor_sync(kAll, v, 1);
  return v + __shfl_xor_sync(kAll, v, 2);
}
// 1 / l; a row without keys (l = 0) gives 0.
__device__ __forceinline__ float inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }

// Running maximum and sum of a fragment's two rows, and the weighted sums.
template <int DT>
struct Flow {
  float m[2], l[2], acc[DT / 8][4];
  __device__ __forceinline__ void start() {
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
#pragma unroll
    for (int n = 0; n < DT / 8; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;
  }
};

// One chunk of keys: s holds the scores, and the weights afterwards.  (l: the lane's share; quad_sum at the end.)  FIRST: of a row.
template <bool FIRST, int DT, int NT>
__device__ __forceinline__ void soften(Flow<DT>& f, float (&s)[NT][4]) {
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    float m = FIRST ? -INFINITY : f.m[r];
#pragma unroll
    for (int t = 0; t < NT; ++t) m = fmaxf(m, fmaxf(s[t][2 * r], s[t][2 * r + 1]));
    m = quad_max(m);
    const float base = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    if (!FIRST) {
      const float fade = ex2_approx(f.m[r] - base);
      l = f.l[r] * fade;
#pragma unroll
      for (int n = 0; n < DT / 8; ++n) {
        f.acc[n][2 * r] *= fade;
        f.acc[n][2 * r + 1] *= fade;
      }
    }
    f.m[r] = m;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      s[t][2 * r] = ex2_approx(s[t][2 * r] - base);
      s[t][2 * r + 1] = ex2_approx(s[t][2 * r + 1] - base);
      l += s[t][2 * r] + s[t][2 * r + 1];
    }
    f.l[r] = l;
  }
}

// ---- long segments ---------------------------------------------------------------------------------------------------
struct Tile { int lo, hi, row; };  // a segment and the first row of a tile of it
constexpr int kMaxTiles = 8;       // tiles that start in one block's rows (at most 128, of segments of more than 24 rows)

// The tiles of `tile` rows of segments longer than `above` that start in rows [base, base + tile).
__device__ __forceinline__ int find_tiles(const SegArgs& a, Tile* tiles, int* count, int base, int tile, int above) {
  if (threadIdx.x == 0) *count = 0;
  const int2 near = segments_near(a, base + 1, base + tile, false, false);
  __syncthreads();
  for (int s = near.x + (int)threadIdx.x; s < near.y; s += kThreads) {
    const int lo = a.seg_start[s], hi = a.seg_start[s + 1];
    if (lo < 0 || hi > a.n || lo > hi || hi - lo > a.max_len || hi - lo <= above) continue;  // (reported by the short ones' blocks)
    const int row = lo >= base ? lo : lo + (base - lo + tile - 1) / tile * tile;
    if (row < hi && row < base + tile) {
      const int at = atomicAdd(count, 1);
      if (at < kMaxTiles) tiles[at] = Tile{lo, hi, row};
    }
  }
  __syncthreads();
  return min(*count, kMaxTiles);
}

}  // namespace dsvt_train
