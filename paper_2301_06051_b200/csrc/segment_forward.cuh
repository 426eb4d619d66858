// Segment attention, forward: softmax(q k^T + bias) v inside each segment.
//
// Measured (bf16, dim 24, 8 heads, bias of 121 and 567 buckets): 32,000 pillars in sets of 36 37 us, where q, k, v and the result take 8 at
// a copy's rate; 120,000 voxels in whole windows of up to 1055 475 us (bytes 29, operations 14).  Bound by instructions and their
// latencies, not by the tensor pipe (5 and 12 % busy) or DRAM (12 and 4 %): in the windows' tiles some 45 instructions a score (issue slots
// times 32 lanes, by pairs and heads), of which its 2 x 24 multiply-adds are few; each group of four heads looks a pair's bucket up.  In sets, a third of the warps' time goes to the barriers between planning, loading, looking up and
// attending; warps of their own for the first three, over a ring of batches, came to the same time (30 us where this took 32), and four
// blocks of 128 threads or two of 256 with two heads to a warp to more.
#pragma once
#include "segment_blocks.cuh"

namespace dsvt_train {

// Heads of a block that holds its segments whole: rows of at most 400 bytes, which leaves room for three blocks of 36-voxel sets on an SM
// (32,000 pillars: 24 warps an SM at 80 registers 34 us, 16 at 123 45).
template <typename T, int DT>
constexpr int kHeads = DT * sizeof(T) <= 48 ? 8 : DT * sizeof(T) <= 96 ? 4 : DT * sizeof(T) <= 128 ? 2 : 1;

constexpr int kShortThreads = 256;

struct ShortLayout {
  int heads, batch, per, ranges;               // of a block; rows at a time; rows of a range, and ranges of the call
  int pitch_idx, limit;                        // entries to a row of the bucket tile; longest segment
  uint32_t pitch, array;                       // bytes of a row and of an array of rows
  uint32_t maps, bias, cells, index, rows, bytes;
};

template <typename T>
static ShortLayout short_layout(const SegArgs& a, int heads, int limit, int arrays, int batch) {
  ShortLayout l = {};
  l.heads = heads;
  l.limit = limit;
  l.batch = limit > batch ? (limit + 7) / 8 * 8 : batch;
  l.pitch = (uint32_t)(heads * a.dim * sizeof(T) + 16);
  l.array = l.batch * l.pitch;
  uint32_t at = (sizeof(Plan) + 15) / 16 * 16;
  auto take = [&](size_t bytes) { const uint32_t was = at; at += (uint32_t)((bytes + 15) / 16 * 16); return was; };
  if (a.bias) {
    l.maps = take((size_t)(a.maps.at_z + 2 * a.maps.extent[2] - 1) * 2);
    l.cells = take((size_t)l.batch * 16);
    l.pitch_idx = index_pitch(limit);
    l.index = take(((size_t)(l.batch + 16) * l.pitch_idx + 64) * 2);
    l.bias = take((size_t)heads * a.buckets * 4);  // (a look-up of an unwritten bucket ends within 4 KB of a head's first: the rows follow)
  }
  // (a tile of 16 rows may begin at an array's last 8: what follows is read, and not used)
  l.rows = take((size_t)arrays * l.array + 8 * l.pitch);
  if (at - l.rows < 4096) at = l.rows + 4096;
  l.bytes = at;
  return l;
}

// Rows of a range: an equal share for every block that can be resident, at most `most`, where ranges of more and fewer short segments
// have to even out.  (Sets of 32,000 pillars, backward: ranges of 128 rows 117 us, an equal share 97.)
static void set_ranges(ShortLayout& l, int n, int resident, int most) {
  int per = (n + resident - 1) / resident;
  per = per < 16 ? 16 : per > most ? most : per;
  l.per = per;
  l.ranges = (n + per - 1) / per;
}

// A tile of 16 queries against its segment's keys, NT tiles of them at a time: all of them where ONLY.
template <typename T, int DT, int NT, bool ONLY>
__device__ __forceinline__ void attend_tile(Flow<DT>& f, uint32_t q, uint32_t k, uint32_t v, uint32_t pitch, int dim, const Scoring& sc, const float* bias,
                                            const uint16_t* index, int pitch_idx, uint64_t keys) {
  float s[NT][4];
  scores<T, DT, NT>(s, q, k, pitch, dim);
  transform<NT>(s, sc, bias, index, pitch_idx, keys);
  soften<ONLY>(f, s);
  weigh<T, DT, NT, false>(f.acc, s, v, pitch, dim);
}

template <typename T, int DT>
__global__ void __launch_bounds__(kShortThreads, DT <= 24 && sizeof(T) == 2 ? 3 : DT <= 32 ? 2 : 1) short_forward_kernel(const __grid_constant__ SegArgs a, const ShortLayout L, const Scoring sc) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int HG = kHeads<T, DT>;
  const int dim = kExact<DT> ? DT : a.dim;
  pdl_enter();
  Plan& plan = *reinterpret_cast<Plan*>(smem);
  uint16_t* maps = reinterpret_cast<uint16_t*>(smem + L.maps);
  float* bias = reinterpret_cast<float*>(smem + L.bias);
  int4* cells = reinterpret_cast<int4*>(smem + L.cells);
  uint16_t* index = reinterpret_cast<uint16_t*>(smem + L.index);
  const int head0 = blockIdx.y * HG, heads = min(HG, a.heads - head0);
  const uint32_t pitch = kExact<DT> ? HG * DT * sizeof(T) + 16 : L.pitch;
  const uint32_t q0 = smem_u32(smem + L.rows), k0 = q0 + L.array, v0 = k0 + L.array;
  StartCheck<kShortThreads> starts;
  starts.begin(a);
  const Range range = start_range<kShortThreads>(a, plan, blockIdx.x, L.ranges, L.per);
  starts.end(a);
  const int chunks = HG * dim * (int)sizeof(T) / 16, real = heads * dim * (int)sizeof(T) / 16;
  const int64_t col = (int64_t)head0 * dim;
  const Rows<3> src = {{first_head<T>(a.q, col), first_head<T>(a.k, col), first_head<T>(a.v, col)},
                       {a.ld_q * (int64_t)sizeof(T), a.ld_k * (int64_t)sizeof(T), a.ld_v * (int64_t)sizeof(T)}};
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  bool staged = false;
  while (next_batch<kShortThreads>(a, plan, range, L.limit, L.batch)) {
    if (a.bias) {
      load_cells<kShortThreads>(a, smem_u32(cells), plan.ids, plan.rows);
      cp_commit();
    }
    load_rows<T, kShortThreads, 3>(q0, L.array, pitch, src, plan.ids, plan.rows, chunks, real);
    cp_commit();
    if (a.bias) {
      if (!staged) {  // (while the rows are on their way)
        stage_tables<kShortThreads>(a, maps, bias, head0, HG);
        staged = true;
      }
      cp_wait<1>();
      __syncthreads();
      fill_index<kShortThreads>(a, plan, cells, maps, index, L.pitch_idx);
    }
    cp_wait<0>();
    __syncthreads();
    const int h = warp % HG;
    for (int it = warp / HG; it < plan.items; it += kShortThreads / 32 / HG) {
      if (h >= heads) break;
      const Item item = plan.item[it];
      const uint32_t at_head = h * dim * sizeof(T);
      const float* mine = bias + h * a.buckets;
      const int row = item.at + 16 * item.tile;
      const uint32_t q = q0 + row * pitch + at_head, k = k0 + item.at * pitch + at_head, v = v0 + item.at * pitch + at_head;
      const uint16_t* at = index + row * L.pitch_idx;
      Flow<DT> f;
      f.start();
#define DSVT_ATTEND(NT) attend_tile<T, DT, NT, true>(f, q, k, v, pitch, dim, sc, mine, at, L.pitch_idx, real_rows(plan, item.at, item.len))
#define DSVT_ATTEND_PART(NT)                                                                               \
    attend_tile<T, DT, NT, false>(f, q, k + j * pitch, v + j * pitch, pitch, dim, sc, mine, at + j, L.pitch_idx, \
                                  real_rows(plan, item.at + j, min(8 * NT, item.len - j)))
      // Up to 40 keys at once, in 16-bit types; more, and fp32, in parts of up to 24.  (Fewer widths in fp32, and no wider parts: kernels of
      // this size miss in the instruction cache.  12,345 pillars fp32 38.2 us with five widths, 35.6 with three; sets of 90 in parts of
      // up to 40 65.1, of up to 24 61.4.)
      const int tiles = (item.len + 7) >> 3;
      if (sizeof(T) == 2 && tiles <= 5) {
        switch (tiles) {
          case 1: DSVT_ATTEND(1); break;
          case 2: DSVT_ATTEND(2); break;
          case 3: DSVT_ATTEND(3); break;
          case 4: DSVT_ATTEND(4); break;
          default: DSVT_ATTEND(5);
        }
      } else {
        for (int j = 0; j < item.len; j += 24) {
          if (item.len - j > 16) DSVT_ATTEND_PART(3);
          else if (item.len - j > 8) DSVT_ATTEND_PART(2);
          else DSVT_ATTEND_PART(1);
        }
      }
#undef DSVT_ATTEND
#undef DSVT_ATTEND_PART
      // the result takes the place of the queries (this warp's alone: its head's channels of a tile's rows)
      const int r0 = 16 * item.tile + (lane >> 2);
      const float i0 = inverse(quad_sum(f.l[0])), i1 = inverse(quad_sum(f.l[1]));
      T* to = reinterpret_cast<T*>(smem + L.rows + (item.at + r0) * pitch + at_head) + (lane & 3) * 2;
      __syncwarp();
#pragma unroll
      for (int n = 0; n < DT / 8; ++n) {
        if (!kExact<DT> && n * 8 >= dim) break;
        if (r0 < item.len) store2<T>(to + n * 8, f.acc[n][0] * i0, f.acc[n][1] * i0);
        if (r0 + 8 < item.len) store2<T>(reinterpret_cast<T*>(reinterpret_cast<char*>(to) + 8 * pitch) + n * 8, f.acc[n][2] * i1, f.acc[n][3] * i1);
      }
    }
    __syncthreads();
    const int part = threadIdx.x & 7;
    for (int r = threadIdx.x >> 3; r < plan.rows; r += kShortThreads / 8) {
      const int id = plan.ids[r];
      if (id < 0) continue;
      char* to = (char*)a.out + (id * a.ld_out + col) * (int64_t)sizeof(T);
#pragma unroll 4
      for (int c = part; c < real; c += 8) *reinterpret_cast<uint4*>(to + c * 16) = *reinterpret_cast<const uint4*>(smem + L.rows + r * pitch + c * 16);
    }
    if (plan.cursor >= range.end) break;
    __syncthreads();
  }
}

// Shared memory of a tile of a long segment: `own` arrays of the tile's rows, `passing` arrays of two chunks.
struct LongLayout {
  int pitch_idx;
  uint32_t pitch, tile, chunk;  // bytes of a row, of an array of the tile's rows, of an array of a chunk's rows
  uint32_t maps, bias, cells, passing_cells, ids, index, rows, passing, bytes;
};

template <typename T, int DT>
struct LongShape {
  static constexpr int HG = DT * sizeof(T) <= 64 ? 4 : DT * sizeof(T) <= 128 ? 2 : 1, WH = HG < 2 ? HG : 2, HPW = HG / WH, rows = 16 * kWarps / WH;
  static constexpr bool three = sizeof(T) == 2 && DT <= 24;  // blocks on an SM: three of chunks of 32 rows rather than two of 64 (565 and 591 us)
  static constexpr int NT = three ? 4 : sizeof(T) == 2 ? 8 : 6, chunk = 8 * NT;
};

template <typename T, int DT>
static LongLayout long_layout(const SegArgs& a, int own, int passing) {
  using S = LongShape<T, DT>;
  LongLayout l = {};
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
    l.index = take((size_t)2 * S::rows * l.pitch_idx * 2);
  }
  l.rows = take((size_t)own * l.tile + 64);
  l.passing = take((size_t)2 * passing * l.chunk + 64);
  l.bytes = at;
  return l;
}

// The chunks of a segment's rows on their way through shared memory, one ahead of the one in work.  Rows have two buffers; voxels
// and cells, which are written before the barrier that frees the chunk before, three.
template <typename T, int DT>
struct Passing {
  using S = LongShape<T, DT>;
  const SegArgs& a;
  const LongLayout& L;
  unsigned char* smem;
  int lo, hi, mine;  // the segment, and this thread's voxel of the next chunk
  __device__ __forceinline__ int32_t* ids(int c) const { return reinterpret_cast<int32_t*>(smem + L.ids) + S::rows + c % 3 * S::chunk; }
  __device__ __forceinline__ int4* cells(int c) const { return reinterpret_cast<int4*>(smem + L.passing_cells) + c % 3 * S::chunk; }
  __device__ __forceinline__ uint32_t array(int c, int which, int arrays) const { return smem_u32(smem + L.passing) + ((c & 1) * arrays + which) * L.chunk; }
  __device__ __forceinline__ void fetch_id(int at) {
    mine = -1;
    if (threadIdx.x < S::chunk && at + (int)threadIdx.x < hi) mine = voxel_at(a, at + threadIdx.x);
  }
};

template <typename T, int DT>
__global__ void __launch_bounds__(kThreads, LongShape<T, DT>::three ? 3 : DT <= 32 ? 2 : 1) long_forward_kernel(const __grid_constant__ SegArgs a, const LongLayout L, const Scoring sc, int above) {
  extern __shared__ __align__(16) unsigned char smem[];
  using S = LongShape<T, DT>;
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
  const int head0 = blockIdx.y * S::HG, heads = min(S::HG, a.heads - head0);
  const uint32_t pitch = kExact<DT> ? S::HG * DT * sizeof(T) + 16 : L.pitch;
  const uint32_t q0 = smem_u32(smem + L.rows);
  stage_tables<kThreads>(a, maps, bias, head0, S::HG);
  const int chunks = S::HG * dim * (int)sizeof(T) / 16, real = heads * dim * (int)sizeof(T) / 16;
  const int64_t col = (int64_t)head0 * dim;
  const Rows<1> own = {{first_head<T>(a.q, col)}, {a.ld_q * (int64_t)sizeof(T)}};
  const Rows<2> passing = {{first_head<T>(a.k, col), first_head<T>(a.v, col)}, {a.ld_k * (int64_t)sizeof(T), a.ld_v * (int64_t)sizeof(T)}};
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row = 16 * (warp / S::WH);  // of the warp's tile of 16
  for (int ti = 0; ti < found; ++ti) {
    const Tile tile = tiles[ti];
    const int rows = min(S::rows, tile.hi - tile.row);
    Passing<T, DT> pass{a, L, smem, tile.lo, tile.hi, -1};
    __syncthreads();  // (the tile before is done with the shared memory)
    if (threadIdx.x < S::rows) {
      const int id = (int)threadIdx.x < rows ? voxel_at(a, tile.row + threadIdx.x) : -1;
      ids[threadIdx.x] = id;
      if (a.bias) cells[threadIdx.x] = id >= 0 ? a.coords[id] : make_int4(0, 0, 0, 0);
    }
    auto publish = [&](int c) {
      if (threadIdx.x < S::chunk) {
        pass.ids(c)[threadIdx.x] = pass.mine;
        if (a.bias) pass.cells(c)[threadIdx.x] = pass.mine >= 0 ? a.coords[pass.mine] : make_int4(0, 0, 0, 0);
      }
    };
    auto load = [&](int c) {
      load_rows<T, kThreads, 2>(pass.array(c, 0, 2), L.chunk, pitch, passing, pass.ids(c), S::chunk, chunks, real);
      cp_commit();
    };
    pass.fetch_id(tile.lo);
    publish(0);
    pass.fetch_id(tile.lo + S::chunk);
    __syncthreads();
    load_rows<T, kThreads, 1>(q0, 0, pitch, own, ids, S::rows, chunks, real);
    load(0);
    auto index_of = [&](int c) { return index + (c & 1) * S::rows * L.pitch_idx; };
    auto look_up = [&](int c) {
      if (!a.bias) return;
      uint16_t* to = index_of(c);
      const int4* passing_cells = pass.cells(c);
      for (int i = threadIdx.x; i < S::rows * S::chunk; i += kThreads) {
        const int r = i / S::chunk, j = i % S::chunk;
        to[r * L.pitch_idx + j] = (uint16_t)bucket_at(a.maps, maps, cells[r], passing_cells[j]);
      }
    };
    look_up(0);
    Flow<DT> f[S::HPW];
#pragma unroll
    for (int i = 0; i < S::HPW; ++i) f[i].start();
    const int parts = (tile.hi - tile.lo + S::chunk - 1) / S::chunk;
    for (int c = 0; c < parts; ++c) {
      if (c + 1 < parts) publish(c + 1);
      cp_wait<0>();
      __syncthreads();  // this chunk and its buckets are there, the other one's buffers free
      if (c + 1 < parts) {
        load(c + 1);
        pass.fetch_id(tile.lo + (c + 2) * S::chunk);
        look_up(c + 1);
      }
      uint64_t keys = 0;
      {
        const int32_t* at = pass.ids(c);
        keys = __ballot_sync(kAll, at[lane] >= 0);
        const bool second = 32 + lane < S::chunk && at[32 + lane] >= 0;
        keys |= (uint64_t)__ballot_sync(kAll, second) << 32;
      }
#pragma unroll
      for (int i = 0; i < S::HPW; ++i) {
        const int h = (warp % S::WH) * S::HPW + i;
        if (h < heads && row < rows) {
          const uint32_t at_head = h * dim * sizeof(T);
          attend_tile<T, DT, S::NT, false>(f[i], q0 + row * pitch + at_head, pass.array(c, 0, 2) + at_head, pass.array(c, 1, 2) + at_head, pitch, dim, sc,
                                           bias + h * a.buckets, index_of(c) + row * L.pitch_idx, L.pitch_idx, keys);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < S::HPW; ++i) {
      const int h = (warp % S::WH) * S::HPW + i;
      if (h >= heads || row >= rows) continue;
      const float i0 = inverse(quad_sum(f[i].l[0])), i1 = inverse(quad_sum(f[i].l[1]));
      const int r0 = row + (lane >> 2), id0 = ids[r0], id1 = ids[r0 + 8];
      T* to = (T*)a.out + col + h * dim + (lane & 3) * 2;
#pragma unroll
      for (int n = 0; n < DT / 8; ++n) {
        if (!kExact<DT> && n * 8 >= dim) break;
        if (id0 >= 0) store2<T>(to + id0 * a.ld_out + n * 8, f[i].acc[n][0] * i0, f[i].acc[n][1] * i0);
        if (id1 >= 0) store2<T>(to + id1 * a.ld_out + n * 8, f[i].acc[n][2] * i1, f[i].acc[n][3] * i1);
      }
    }
  }
}

// Up to kShort rows a segment is held whole where that leaves room for two blocks on an SM, or at least for one; in calls with longer
// ones up to 64 rows, and the longer ones go through in tiles.
constexpr uint32_t kSmemHalf = 112 * 1024;  // two blocks
constexpr uint32_t kSmemMost = 226 * 1024;  // (of 227 KB; the rest for what kernels declare themselves)

template <typename T, int DT>
int forward_of(dsvt_ctx* ctx, const SegArgs& a) {
  int limit = a.max_len <= kShort ? a.max_len : 64;
  ShortLayout l = short_layout<T>(a, kHeads<T, DT>, limit, 3, kBatch);
  if (l.bytes > kSmemMost) l = short_layout<T>(a, kHeads<T, DT>, limit = 64, 3, kBatch);
  const Scoring sc = scoring_of(a);
  const int groups = (int)dsvt_ceil_div(a.heads, kHeads<T, DT>);
  set_ranges(l, a.n, (int)dsvt_ceil_div((DT <= 24 && sizeof(T) == 2 ? 3 : 2) * ctx->sm_count, groups), limit < a.max_len ? 128 : 1 << 20);
  constexpr auto kernel = short_forward_kernel<T, DT>;
  int rc = allow_smem<kernel>(ctx, kSmemMost);
  if (rc != DSVT_OK) return rc;
  launch_pdl(kernel, dim3((unsigned)l.ranges, (unsigned)groups), dim3(kShortThreads), l.bytes, ctx->stream, a, l, sc);
  DSVT_LAUNCHED(ctx);
  if (limit >= a.max_len) return DSVT_OK;
  using S = LongShape<T, DT>;
  const LongLayout g = long_layout<T, DT>(a, 1, 2);
  constexpr auto longer = long_forward_kernel<T, DT>;
  rc = allow_smem<longer>(ctx, kSmemMost);
  if (rc != DSVT_OK) return rc;
  launch_pdl(longer, dim3((unsigned)dsvt_ceil_div(a.n, S::rows), (unsigned)dsvt_ceil_div(a.heads, S::HG)), dim3(kThreads), g.bytes, ctx->stream, a, g, sc, limit);
  DSVT_LAUNCHED(ctx);
  return DSVT_OK;
}

template <typename T>
int launch_forward(dsvt_ctx* ctx, const SegArgs& a) {
  if (a.dim == 16) return forward_of<T, 16>(ctx, a);
  if (a.dim == 24) return forward_of<T, 24>(ctx, a);
  if (a.dim == 32) return forward_of<T, 32>(ctx, a);
  if (a.dim <= 64) return forward_of<T, 64>(ctx, a);
  return forward_of<T, 128>(ctx, a);
}

}  // namespace dsvt_train
