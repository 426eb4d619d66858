// Segment attention: what a block works on.  Short segments: those that start in a range of rows, whole, as many at a time as fit in
// shared memory.  Long ones: a tile of the rows of one segment, the segment's other rows passing by in chunks.
#pragma once
#include <limits.h>

#include "segment_mma.cuh"

namespace dsvt_train {

constexpr int kThreads = 256, kWarps = kThreads / 32;  // of the long ones' blocks
constexpr int kShort = 128;                         // most rows of a segment that is held whole
constexpr int kBatch = 48;                          // rows in shared memory at a time, or the longest segment's if that is more

// 16 rows of a segment: its first row's place in the batch, its length, the tile.
struct Item { uint8_t at, len, tile, pad; };

// A batch of segments in shared memory.  A segment's place is a multiple of 8 rows, so that tiles of 8 rows are its own; the places
// behind its end are zeros.
struct Plan {
  int rows, items, pairs, longest;     // (pairs: of queries and keys; longest: segment's length)
  int cursor;                          // the first segment that has not been looked at
  int lo[kShort / 8];                  // by segment: first row, length, place
  uint8_t len[kShort / 8], place[kShort / 8];
  uint8_t owner[kShort / 8];           // by 8 places: the segment
  uint32_t real[kShort / 32 + 3];      // bit i: place i holds a voxel
  uint16_t span[kShort];               // by place: its segment's place, and length << 8; 0 where there is no voxel
  int32_t ids[kShort];
  Item item[kShort / 8];
};

// Which entries of seg_start can be of segments that start in rows [from, to): found by a probe per thread and round (one or two for most calls); N: threads of the block.
// Right where starts ascend; find_tiles does without where they may not.
template <int N>
__device__ __forceinline__ int2 segments_near(const SegArgs& a, int from, int to) {
  const int tid = threadIdx.x;
  int lo = 0, hi = a.cap_segments;
  const int end = segment_count(a);
  while (true) {
    const int span = hi - lo, step = (span + N - 1) / N;
    const int64_t i = lo + (int64_t)tid * step;
    const int v = i < hi ? a.seg_start[i] : 0;
    const bool in = i < hi && i < end;
    const int below = __syncthreads_count(in && v < from), upto = __syncthreads_count(in && v < to);
    const int64_t next_hi = lo + (int64_t)upto * step;
    if (next_hi < hi) hi = (int)next_hi;
    if (below > 0) lo += (below - 1) * step;
    if (hi > end) hi = end;
    if (hi - lo <= 8 * N || hi - lo >= span) break;
  }
  return make_int2(lo, hi);
}

// p.cursor: the entry of seg_start to look from for segments that start in rows from `from` on, which is the last of a probe per thread that
// lies below it.  Entries may be out of place: it is 0 where the probes' answers do not change once, from below to not below, or the one
// that counts lies below its neighbour.  So an entry out of place between two that are not keeps no other segment from being found.
// A barrier before and after.
template <int N>
static __device__ __noinline__ void search_on(const SegArgs& a, Plan& p, int from, int lo, int step) {  // (a quarter of a million entries)
  const int end = segment_count(a);
  while (step > 4 * N) {
    const int64_t hi = lo + (int64_t)step + 1;
    step = (int)((hi - lo + N - 1) / N);
    const int64_t i = lo + (int64_t)threadIdx.x * step;
    const bool below = i < hi && i < end && a.seg_start[i] < from;
    const int count = __syncthreads_count(below);
    if (below != (int)threadIdx.x < count || (below && i > 0 && a.seg_start[i - 1] > a.seg_start[i])) atomicMin(&p.cursor, 0);
    if (count > 0) lo += (count - 1) * step;
  }
  if (threadIdx.x == 0) atomicMin(&p.cursor, lo);
}
template <int N>
__device__ __forceinline__ void search(const SegArgs& a, Plan& p, int from) {
  const int step = (a.cap_segments + N - 1) / N;
  const int64_t i = (int64_t)threadIdx.x * step;
  const bool there = i < a.cap_segments;
  const int v = there ? a.seg_start[i] : INT_MAX, before = there && i > 0 ? a.seg_start[i - 1] : INT_MIN;
  if (threadIdx.x == 0) p.cursor = INT_MAX;
  const bool below = v < from && i < segment_count(a);  // (what lies behind the last segment's end may be anything)
  const int count = __syncthreads_count(below);
  if (below != (int)threadIdx.x < count || (below && before > v)) atomicMin(&p.cursor, 0);
  const int lo = count > 0 ? (count - 1) * step : 0;
  if (step > 4 * N) search_on<N>(a, p, from, lo, step);
  else if (threadIdx.x == 0) atomicMin(&p.cursor, lo);
}

// Every pair of seg_start that is no segment is said, whether a block's search comes across it or not: a share for each block of the grid's row 0.
// A thread's pair is loaded before the search and looked at behind it.  (This, the search's second load and the look behind its last
// segment take 0.1 us of 2,000 pillars' 11.8 us and 0.4 of 32,000 pillars' 36.9; waiting for the pair at once, 0.2 and 0.6.)
__device__ __forceinline__ void check_pair(const SegArgs& a, int2 pair) {
  if (pair.x < 0 || pair.y < pair.x || pair.y > a.n) atomicOr(a.status, DSVT_STATUS_BAD_INDEX);
}
template <int N>
static __device__ __noinline__ void check_more(const SegArgs& a) {
  const int count = segment_count(a);
  const int64_t step = (int64_t)gridDim.x * N;
  for (int64_t s = (int64_t)blockIdx.x * N + threadIdx.x + step; s < count; s += step) check_pair(a, make_int2(a.seg_start[s], a.seg_start[s + 1]));
}
template <int N>
struct StartCheck {
  int2 pair;
  __device__ __forceinline__ void begin(const SegArgs& a) {
    const uint32_t at = blockIdx.x * N + threadIdx.x;  // (of 16 rows at least: within 32 bits)
    pair = blockIdx.y == 0 && at < (uint32_t)segment_count(a) ? make_int2(a.seg_start[at], a.seg_start[at + 1]) : make_int2(0, 0);
  }
  __device__ __forceinline__ void end(const SegArgs& a) {
    check_pair(a, pair);
    if (blockIdx.y == 0 && gridDim.x * N < (uint32_t)a.cap_segments) check_more<N>(a);
  }
};

// Copies what every block reads: the index tables of the displacements and its heads' bias, in units of log 2.
template <int N>
__device__ __forceinline__ void stage_tables(const SegArgs& a, uint16_t* maps, float* bias, int head0, int heads) {
  if (!a.bias) return;
  for (int i = threadIdx.x; i < a.maps.at_z + 2 * a.maps.extent[2] - 1; i += N) maps[i] = (uint16_t)(4 * a.maps.of[i]);
  const int count = min(heads, a.heads - head0) * a.buckets;
  const float* from = a.bias + (int64_t)head0 * a.buckets;
  for (int i = threadIdx.x; i < count; i += N) bias[i] = bias_log2(from[i]);
}

__device__ __forceinline__ int bucket_at(const BucketMaps& m, const uint16_t* maps, int4 i, int4 j) {
  const int ex = m.extent[0] - 1, ey = m.extent[1] - 1, ez = m.extent[2] - 1;
  const int dx = min(max(i.y - j.y, -ex), ex) + ex, dy = min(max(i.z - j.z, -ey), ey) + ey + m.at_y, dz = min(max(i.w - j.w, -ez), ez) + ez + m.at_z;
  return maps[dx] + maps[dy] + maps[dz];  // (the maps in shared memory hold four times the index: a bias's offset)
}

// The segments that start in rows [from, to) of a call, the first range and the last open to their side.  They are among the entries from
// the plan's cursor to the first start in place that lies at `to` or behind, or to `end`.
struct Range { int from, to, end; };
template <int N>
__device__ __forceinline__ Range start_range(const SegArgs& a, Plan& p, int range, int ranges, int per) {
  if (range > 0) search<N>(a, p, range * per);
  else if (threadIdx.x == 0) p.cursor = 0;
  __syncthreads();
  return Range{range == 0 ? INT_MIN : range * per, range == ranges - 1 ? INT_MAX : (range + 1) * per, segment_count(a)};
}

// The next batch of a range's segments of up to `limit` rows, at most `most` places together: their rows' voxels and the list of their
// tiles.  False if there are no more.  A barrier comes before.
template <int N>
__device__ __forceinline__ bool next_batch(const SegArgs& a, Plan& p, const Range& range, int limit, int most) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (warp == 0) {
    int at = 0, segments = 0, items = 0, pairs = 0, longest = 0, cursor = p.cursor;
    bool open = true;
    while (open && cursor < range.end) {  // 32 segments at a time
      const int s = cursor + lane;
      int lo = 0, hi = 0;
      if (s < range.end) { lo = a.seg_start[s]; hi = a.seg_start[s + 1]; }
      const bool here = s < range.end && lo >= range.from && lo < range.to;
      const bool mine = here && segment_sound(a, lo, hi) && hi - lo <= limit;
      const int len = mine ? hi - lo : 0, tiles = (len + 15) >> 4, size = (len + 7) & ~7;
      int end = size, upto = tiles;  // sums up to and with this lane's segment
      for (int m = 1; m < 32; m <<= 1) {
        const int e = __shfl_up_sync(kAll, end, m), u = __shfl_up_sync(kAll, upto, m);
        if (lane >= m) {
          end += e;
          upto += u;
        }
      }
      const bool in = mine && at + end <= most;
      const uint32_t taken = __ballot_sync(kAll, in), rest = __ballot_sync(kAll, mine) & ~taken;
      if (in) {
        const int place = at + end - size, slot = segments + __popc(taken & ((1u << lane) - 1u));
        p.lo[slot] = lo;
        p.len[slot] = (uint8_t)len;
        p.place[slot] = (uint8_t)place;
        for (int t = 0; t < tiles; ++t) p.item[items + upto - tiles + t] = Item{(uint8_t)place, (uint8_t)len, (uint8_t)t, 0};
        for (int t = 0; t < size; t += 8) p.owner[(place + t) >> 3] = (uint8_t)slot;
        pairs += len * len;
        longest = max(longest, len);
      }
      if (taken) {
        const int last = 31 - __clz(taken);
        at += __shfl_sync(kAll, end, last);
        items += __shfl_sync(kAll, upto, last);
        segments += __popc(taken);
      }
      const uint32_t behind = __ballot_sync(kAll, s < range.end && lo >= range.to && lo <= hi);  // (a start above the next one is out of place)
      if (rest) {
        cursor += __ffs(rest) - 1;
        open = false;
      } else {
        cursor = behind ? range.end : cursor + 32;
        open = at + 8 <= most;
      }
    }
    pairs = __reduce_add_sync(kAll, pairs);
    longest = __reduce_max_sync(kAll, longest);
    if (lane == 0) {
      p.longest = longest;
      p.rows = at;
      p.items = items;
      p.pairs = pairs;
      p.cursor = cursor;
    }
  }
  __syncthreads();
  if (p.items == 0) return false;
  if (tid < 3) p.real[kShort / 32 + tid] = 0;
  for (int i = tid; i < kShort; i += N) {
    int id = -1, span = 0;
    if (i < p.rows) {
      const int own = p.owner[i >> 3], at = p.place[own], len = p.len[own];
      if (i - at < len) id = voxel_at(a, p.lo[own] + i - at);
      span = at | len << 8;
    }
    const uint32_t real = __ballot_sync(kAll, id >= 0);
    if (lane == 0) p.real[i >> 5] = real;
    p.ids[i] = id;
    p.span[i] = (uint16_t)(id >= 0 ? span : 0);
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

// The buckets (times 4) of all pairs of the batch: index[i][j - first of i's segment].  The rest of the tile is never written.  Four rows
// at a time, so that their look-ups overlap.
template <int N>
__device__ __forceinline__ void fill_index(const SegArgs& a, const Plan& p, const int4* cells, const uint16_t* maps, uint16_t* index, int pitch) {
  const int part = threadIdx.x & 15, rows = p.rows, longest = p.longest;
  constexpr int step = N / 16;
  for (int i = threadIdx.x >> 4; i < rows; i += 4 * step) {
    int at[4], len[4];
    int4 mine[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int r = min(i + u * step, rows - 1), span = i + u * step < rows ? p.span[r] : 0;
      at[u] = span & 255;
      len[u] = span >> 8;
      mine[u] = cells[r];
    }
    for (int j = part; j < longest; j += 16) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int b = bucket_at(a.maps, maps, mine[u], cells[at[u] + min(j, max(len[u] - 1, 0))]);
        if (j < len[u]) index[(i + u * step) * pitch + j] = (uint16_t)b;
      }
    }
  }
}

// Rows' parts of a block's heads to shared memory, N arrays of them: `chunks` pieces of 16 bytes to a row, of which the first `real`
// exist.  Eight threads to a row.
template <int N>
struct Rows {
  const char* from[N];  // at the block's first head
  int64_t ld[N];        // bytes
};
template <typename T, int THREADS, int N>
__device__ __forceinline__ void load_rows(uint32_t to, uint32_t array, uint32_t pitch, const Rows<N>& src, const int32_t* ids, int rows, int chunks, int real) {
  const int part = threadIdx.x & 7;
  for (int r = threadIdx.x >> 3; r < rows; r += THREADS / 8) {
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
// The batch's voxels' cells.
template <int N>
__device__ __forceinline__ void load_cells(const SegArgs& a, uint32_t to, const int32_t* ids, int rows) {
  for (int i = threadIdx.x; i < rows; i += N) cp_async16(to + i * 16, a.coords + max(ids[i], 0), true);
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

// Scores from products, with the buckets' offsets in bk (by ROWS of the index as in buckets_of, else with the index's rows as columns).
// `index`: at the tile's first row and the chunk's first column.
template <int NT, bool ROWS>
__device__ __forceinline__ void score_tiles(float (&s)[NT][4], int (&bk)[NT][4], const Scoring& sc, const float* bias, const uint16_t* index, int pitch) {
  if (sc.cap != 0.f) cap_products<NT>(s, sc);
  const F2 scale = pair(sc.scale, sc.scale);
  if (sc.bias) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (ROWS) {
        buckets_of(bk[t], index + t * 8, pitch);
      } else {
        const uint16_t* at = index + (t * 8 + (threadIdx.x & 3) * 2) * pitch + ((threadIdx.x & 31) >> 2);
        bk[t][0] = at[0] & kBucketMask; bk[t][1] = at[pitch] & kBucketMask; bk[t][2] = at[8] & kBucketMask; bk[t][3] = at[pitch + 8] & kBucketMask;
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; e += 2) put(s[t], e, fma2(two(s[t], e), scale, pair(bias_at(bias, bk[t][e]), bias_at(bias, bk[t][e + 1]))));
  } else {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; e += 2) put(s[t], e, mul(two(s[t], e), scale));
  }
}
// Scores of queries (rows) and keys (columns); -inf where a column holds no key.
template <int NT>
__device__ __forceinline__ void transform(float (&s)[NT][4], const Scoring& sc, const float* bias, const uint16_t* index, int pitch, uint64_t real) {
  int bk[NT][4];
  score_tiles<NT, true>(s, bk, sc, bias, index, pitch);
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
__device__ __forceinline__ float inverse(float l) { return l == 0.f ? 0.f : __fdividef(1.f, l); }

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
    const F2 down = pair(-base, -base);
    F2 sum = pair(l, 0.f);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float2 x = parts(add(two(s[t], 2 * r), down));
      s[t][2 * r] = ex2_approx(x.x);
      s[t][2 * r + 1] = ex2_approx(x.y);
      sum = add(sum, two(s[t], 2 * r));
    }
    f.l[r] = sum_of(sum);
  }
}

// ---- long segments ---------------------------------------------------------------------------------------------------
struct Tile { int lo, hi, row; };  // a segment and the first row of a tile of it
constexpr int kMaxTiles = 8;       // tiles that start in one block's rows: at most three, of segments of more than 64 rows that do not overlap

// The tiles of `tile` rows of segments longer than `above` that start in rows [base, base + tile).  Where an index was bad, in this call's
// starts perhaps (the short ones' kernel has been through them all), every segment is looked at: the blocks of a segment's tiles, and in the
// backward pass both kernels, then know the same segments.
__device__ __forceinline__ int find_tiles(const SegArgs& a, Tile* tiles, int* count, int base, int tile, int above) {
  if (threadIdx.x == 0) *count = 0;
  const bool odd = (__ldcg(a.status) & DSVT_STATUS_BAD_INDEX) != 0;
  int2 near = segments_near<kThreads>(a, base + 1, base + tile);
  if (odd) near = make_int2(0, segment_count(a));
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
