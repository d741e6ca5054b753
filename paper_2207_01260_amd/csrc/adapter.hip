// Entry points of the low-rank adapters, and the launches around their products (adapter_kernel.hpp): rows sorted by adapter, transposes of A and B, sums of slices.
#include <algorithm>
#include <limits>

#include "adapter_kernel.hpp"

namespace cprune {
namespace {

constexpr int kMostRank = 128, kMostAdapters = 1024;
constexpr int kFewRows = 64;      // rows that a wavefront's ballot sorts

struct SortArgs {
  const int* which;
  int rows, adapters, places;
  int waves;                 // that walk
  int *order, *tile_of;      // [places], [places / 64]
  int* tile_at;              // [adapters + 1], an adapter's first tile, or null
};

constexpr int kSortWaves = 16;

// last of n + 1 ascending numbers in `from` that is not past x
__device__ __forceinline__ int last_of(const int* from, int n, int x) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (from[mid] <= x) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// One work-group: the rows of each adapter behind each other in their order, in tiles of their own, rows without an adapter last.  Wavefronts count runs of rows and
// place them on a second walk, behind what the others have counted.
__device__ void sort_rows(const SortArgs& p, int* shared, int* waves) {
  const int t = (int)threadIdx.x, lane = t & 63, wave = t >> 6, n = p.adapters, buckets = n + 1, threads = 64 * kSortWaves;
  int* const count = shared;                              // [wavefront][bucket]
  int* const tile_at = count + p.waves * buckets;      // [buckets + 1]
  for (int i = t; i < p.waves * buckets; i += threads) count[i] = 0;
  __syncthreads();
  const int run = ((p.rows - 1) / (64 * p.waves) + 1) * 64, from = (int)min((long)wave * run, (long)p.rows), end = (int)min((long)from + run, (long)p.rows);
  const int bits = 32 - __clz(n);
  int* const mine = count + wave * buckets;
  // The wavefront's rows 1024 at a time: their adapters are asked for at once and kept in LDS, so that the loops over them are short code.
  unsigned short* const kept = reinterpret_cast<unsigned short*>(tile_at + buckets + 1) + wave * 1024;
  auto load = [&](int r0) __attribute__((always_inline)) {
    int b[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) {
      const int r = r0 + 64 * u + lane;
      b[u] = r < end ? p.which[r] : -1;
    }
#pragma unroll
    for (int u = 0; u < 16; ++u) kept[64 * u + lane] = (unsigned short)((unsigned)b[u] < (unsigned)n ? b[u] : n);
  };
  const bool once = run <= 1024;
  for (int r0 = from; r0 < end; r0 += 1024) {
    load(r0);
#pragma unroll 4
    for (int u = 0; u < 16; ++u) {
      const int r = r0 + 64 * u, v = kept[64 * u + lane], one = __builtin_amdgcn_readfirstlane(v), here = min(64, end - r);
      if (__all(v == one || lane >= here)) {      // (as in a long request's rows)
        if (lane == 0 && here > 0) atomicAdd(&mine[one], here);
      } else if (lane < here) {
        atomicAdd(&mine[v], 1);
      }
    }
  }
  __syncthreads();
  // Where each bucket's tiles begin, and in them each wavefront's rows: 16 lanes have a bucket, those of the wavefronts beside each other.
  if (t == 0) tile_at[0] = 0;
  const int w = t & 15;
  for (int b0 = 0; b0 < buckets; b0 += threads / 16) {
    const int b = b0 + t / 16;
    const int c = b < buckets && w < p.waves ? count[w * buckets + b] : 0;
    int upto = c;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      const int v = __shfl_up(upto, o, 16);
      upto += w >= o ? v : 0;
    }
    const int rows = __shfl(upto, 15, 16), tiles = (rows + kTileRows - 1) / kTileRows;
    // (over the wavefront's four buckets, the work-group's wavefronts and the buckets before)
    int before = w == 0 ? tiles : 0;
#pragma unroll
    for (int o = 16; o < 64; o <<= 1) {
      const int v = __shfl_up(before, o, 64);
      before += lane >= o ? v : 0;
    }
    __syncthreads();      // (tile_at and `waves` of the buckets before)
    if (lane == 48) waves[wave] = before;
    __syncthreads();
    int base = tile_at[b0];
    for (int v = 0; v < wave; ++v) base += waves[v];
    const int first_tile = __shfl(base + before - tiles, lane & 48, 64);
    if (b < buckets) {
      const int at = first_tile * kTileRows;
      if (w < p.waves) count[w * buckets + b] = at + upto - c;
      for (int i = at + rows + w; i < at + tiles * kTileRows; i += 16) p.order[i] = -1;
      if (w == 0) tile_at[b + 1] = first_tile + tiles;
    }
  }
  __syncthreads();
  const int tiles = tile_at[buckets];
  for (int i = t; i < p.places / kTileRows; i += threads) {
    const int b = last_of(tile_at, buckets, i);
    p.tile_of[i] = i >= tiles ? -2 : b < n ? b : -1;
  }
  if (p.tile_at)
    for (int i = t; i <= n; i += threads) p.tile_at[i] = tile_at[i];
  // The rows' places.  In 64 rows the equal ones find each other by the bits of their adapter, and their first counts for all; four times 64 rows side by side.
  for (int r0 = from; r0 < end; r0 += 1024) {
    if (!once) load(r0);
#pragma unroll 1
    for (int u0 = 0; u0 < 16 && r0 + 64 * u0 < end; u0 += 4) {
      int v[4], at[4];
      unsigned long long same[4];
      bool runs = true;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        v[u] = kept[64 * (u0 + u) + lane];
        same[u] = __ballot(r0 + 64 * (u0 + u) + lane < end);
        runs &= __all(v[u] == __builtin_amdgcn_readfirstlane(v[u])) != 0;
      }
      if (!runs) {
#pragma unroll 1
        for (int i = 0; i < bits; ++i) {
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const unsigned long long set = __ballot(v[u] >> i & 1);
            same[u] &= v[u] >> i & 1 ? set : ~set;
          }
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        at[u] = 0;
        if (same[u] >> lane & 1 && lane == __ffsll(same[u]) - 1) at[u] = atomicAdd(&mine[v[u]], __popcll(same[u]));      // (the wavefront's own, in its order)
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int to = __shfl(at[u], (__ffsll(same[u]) - 1) & 63, 64) + __popcll(same[u] & ((1ull << lane) - 1));
        if (same[u] >> lane & 1) p.order[to] = r0 + 64 * (u0 + u) + lane;
      }
    }
  }
}

// Matrices [rows][cols] one behind the other -> [cols][pitch], zeros from `rows` to the pitch; 64 x 64 of one through LDS.
struct TurnArgs {
  const void* from;
  void* to;
  int rows, cols, pitch;
  int row_tiles, col_tiles;
};
template <typename T> __device__ __forceinline__ void turn_tile(const TurnArgs& p, int tile, T* shared) {
  constexpr int PITCH = 65;
  const int t = (int)threadIdx.x, lane = t & 63, line = t >> 6;
  const int per = p.row_tiles * p.col_tiles, matrix = tile / per, in = tile - matrix * per, r0 = in / p.col_tiles * 64, c0 = in % p.col_tiles * 64;
  const T* const from = static_cast<const T*>(p.from) + (long)matrix * p.rows * p.cols;
  T* const to = static_cast<T*>(p.to) + (long)matrix * p.cols * p.pitch;
  constexpr int LINES = kSortWaves, EACH = 64 / LINES;
  T v[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int r = r0 + line + LINES * i, c = c0 + lane;
    v[i] = r < p.rows && c < p.cols ? from[(long)r * p.cols + c] : T(0);
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i) shared[(line + LINES * i) * PITCH + lane] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int c = c0 + line + LINES * i, r = r0 + lane;
    if (c < p.cols && r < p.pitch) to[(long)c * p.pitch + r] = shared[lane * PITCH + line + LINES * i];
  }
}

// What the products need first: the rows' order, by the first work-group where it is asked for, beside it the transposes of A, [k][rank filled up to eight],
// and B, [rank][c].
template <typename T>
__global__ __launch_bounds__(64 * kSortWaves) void adapter_prepare_kernel(const SortArgs sort, const TurnArgs a, const TurnArgs b, int tiles_a) {
  extern __shared__ int shared[];
  __shared__ int waves[kSortWaves];
  int i = blockIdx.x;
  if (sort.which) {
    if (i == 0) {
      sort_rows(sort, shared, waves);
      return;
    }
    --i;
  }
  if (i < tiles_a) turn_tile<T>(a, i, reinterpret_cast<T*>(shared));
  else turn_tile<T>(b, i - tiles_a, reinterpret_cast<T*>(shared));
}

// Sums of an adapter's slices in their order: db [adapter][c][rank] and da [adapter][rank][k], from what the outer products leave (OuterSide::sums).  A thread has four results,
// those of a lane; da's are neighbouring columns in neighbouring threads, db's neighbouring ranks.  Where there are few, LANES threads have every LANES-th slice of them each.
struct JoinArgs {
  const float4_t *sums_b, *sums_a;
  const int* tile_at;
  int tile_count, slices, adapters;
  int rank, ranks, v, k, c;          // ranks, v: powers of two
  int groups_b, groups_a;            // of 16 v columns
  int blocks_b, blocks_a;            // work-groups of an adapter
  float *da, *db;
};
template <int LANES>
__global__ __launch_bounds__(256) void adapter_join_kernel(const JoinArgs p) {
  constexpr int RESULTS = 256 / LANES;
  __shared__ float4_t parts[LANES > 1 ? 256 : 1];
  const int t = (int)threadIdx.x, in_group = t % RESULTS, turn = t / RESULTS;
  const int blocks = p.blocks_a + p.blocks_b, adapter = blockIdx.x / (unsigned)blocks, block = blockIdx.x - adapter * blocks;
  const bool of_b = block < p.blocks_b;
  const unsigned m = (unsigned)(of_b ? block : block - p.blocks_b) * RESULTS + in_group, wide = 16u * p.v;
  const unsigned columns = (of_b ? p.groups_b : p.groups_a) * wide, rp = 16u * p.ranks;
  const bool in = m < columns * rp / 4;
  // (column of the products, rank) of the first of the four, and where they lie
  unsigned lane_row, i, group, quarter, n, low;
  if (of_b) {      // rank, then quarter, i, group: four lane rows of a rank
    const unsigned rank = m % rp, rest = m / rp;
    n = rank / 16, low = rank % 16, quarter = rest % 4, i = rest / 4 % p.v, group = rest / 4 / p.v, lane_row = 4 * quarter;
  } else {         // column, then four ranks
    const unsigned column = m % columns, four = m / columns;
    n = four / 4, quarter = four % 4, i = column % p.v, lane_row = low = column / p.v % 16, group = column / wide;
  }
  const long at = ((long)(group * p.v + i) * p.ranks + n) * 64 + quarter * 16 + low, pitch = (long)columns * rp / 4;
  // slices that the adapter's tiles lie in: slice s begins at tile s tiles / slices, and there are no more of them than tiles
  const int t0 = p.tile_at ? p.tile_at[adapter] : 0, t1 = p.tile_at ? p.tile_at[adapter + 1] : adapter == 0 ? p.tile_count : 0, tiles = p.tile_at ? p.tile_at[p.adapters] : p.tile_count;
  const int slices = min(p.slices, tiles);
  const int first = t0 < t1 ? (int)(((long)(t0 + 1) * slices - 1) / tiles) + adapter : 0, last = t0 < t1 ? (int)(((long)t1 * slices - 1) / tiles) + adapter + 1 : 0;
  const float4_t* const sums = (of_b ? p.sums_b : p.sums_a) + at;
  float4_t s = {0.f, 0.f, 0.f, 0.f};
  if (in) {
    int q = first + turn;
    for (; q + 3 * LANES < last; q += 4 * LANES) {
      const float4_t v[4] = {sums[q * pitch], sums[(q + LANES) * pitch], sums[(q + 2 * LANES) * pitch], sums[(q + 3 * LANES) * pitch]};
      s += v[0], s += v[1], s += v[2], s += v[3];
    }
    for (; q < last; q += LANES) s += sums[q * pitch];
  }
  if constexpr (LANES > 1) {
    parts[t] = s;
    __syncthreads();
    if (turn) return;
#pragma unroll
    for (int l = 1; l < LANES; ++l) s += parts[l * RESULTS + in_group];
  }
  if (!in) return;
  const int c = of_b ? p.c : p.k;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int of = (int)(lane_row + (of_b ? e : 0)), column = outer_lane(c, p.v, (int)group, of).column + (int)i;
    const int rank = (int)(16 * n + (of_b ? low : 4 * quarter + e));
    if ((int)(group * wide) + of * p.v >= c || column >= c || rank >= p.rank) continue;
    if (of_b) p.db[((long)adapter * c + column) * p.rank + rank] = s[e];
    else p.da[((long)adapter * p.rank + rank) * c + column] = s[e];
  }
}

// ---- host ------------------------------------------------------------------------

bool act_of_adapter(int act) { return act_ok(act) || act == CPRUNE_ACT_SILU; }

int check(const cprune_adapter_desc* d, bool backward) {
  if (!d || d->rows < 1 || d->k < 1 || d->c_out < 1 || d->rank < 1 || d->adapters < 1 || !dtype_ok(d->dtype) || (d->mixed != 0 && d->mixed != 1) ||
      d->x_stride < d->k || (backward ? d->dy_stride < d->c_out : !act_of_adapter(d->act)))
    return CPRUNE_ERR_INVALID_ARG;
  auto many = [](double a, double b) { return a * b >= 2147483648.0; };
  if (many(d->rows, d->x_stride) || many(d->rows, d->c_out) || many(d->rows, d->rank) || (backward && many(d->rows, d->dy_stride)) ||
      many((double)d->adapters * d->rank, d->k) || many((double)d->adapters * d->rank, d->c_out))
    return CPRUNE_ERR_INVALID_ARG;
  if (d->rank > kMostRank || d->adapters > kMostAdapters) return CPRUNE_ERR_UNSUPPORTED;
  return CPRUNE_OK;
}
bool base_fits(const cprune_adapter_desc* d, int columns) { return d->base_stride >= columns && (double)d->rows * d->base_stride < 2147483648.0; }

size_t round256(size_t b) { return (b + 255) & ~(size_t)255; }

struct AdapterPlan {
  int ranks, rp, step;                 // RP / 16, RP, terms of a step
  bool few, sorted;
  int tiles, places;                   // tiles there may be
  int splits, per;                     // of narrow
  int padded;                          // backward: rank of A's transpose
  int slices;
  int groups_b, groups_a;              // work-groups a slice, for dB and dA
  size_t order, tile_of, tile_at, part, bt, at, g, parts, sums_b, sums_a;      // bytes
  size_t total() const { return order + tile_of + tile_at + part + bt + at + g + 2 * parts + sums_b + sums_a; }
};

// Tiles as they are likely to be: half of the adapters' last ones are there, half are not.
int rounded_tiles(const cprune_adapter_desc& d, const AdapterPlan& q) {
  if (q.few) return std::min(q.tiles, d.adapters + 1 + d.rows / kFewTile);
  return q.sorted ? std::min(q.tiles, d.rows / kTileRows + 1 + d.adapters / 2) : q.tiles;
}

AdapterPlan plan_of(const cprune_adapter_desc& d, bool backward) {
  AdapterPlan q = {};
  const size_t es = dtype_size(d.dtype);
  q.ranks = d.rank <= 16 ? 1 : d.rank <= 32 ? 2 : d.rank <= 64 ? 4 : 8;
  q.rp = 16 * q.ranks;
  q.step = 64 / (int)es;
  q.few = d.mixed && !backward && d.rows <= kFewRows;
  q.sorted = d.mixed && !q.few;
  q.tiles = q.few ? d.rows : (d.rows - 1) / kTileRows + 1;
  if (q.sorted) q.tiles = std::min(d.rows, d.rows / kTileRows + d.adapters + 1);
  q.places = (int)std::min(2147483647L, (long)q.tiles * kTileRows);      // (more is refused)
  // Work-groups that share a sum: as many as leave the busiest compute unit least to do, by the chunks of its work-groups and what each does but once, some three
  // chunks' time.
  const int terms = backward ? d.c_out : d.k, chunks = std::max(1, terms / (4 * q.step));      // (whole ones)
  const long tiles = rounded_tiles(d, q);
  long least = std::numeric_limits<long>::max();
  for (int splits = 1; splits <= std::min(chunks, 32); ++splits) {
    const int per = (chunks - 1) / splits + 1;
    const long cost = ((tiles * ((chunks - 1) / per + 1) - 1) / 256 + 1) * (per + 3);
    if (cost < least) least = cost, q.per = per;
  }
  q.splits = (chunks - 1) / q.per + 1;
  q.part = round256((size_t)q.splits * d.rows * q.rp * sizeof(float));
  if (q.sorted) {
    q.order = round256((size_t)q.places * sizeof(int));
    q.tile_of = round256((size_t)q.tiles * sizeof(int));
  }
  q.padded = (d.rank + 7) / 8 * 8;
  if (!backward) {
    if (d.rank % 8) q.bt = round256((size_t)d.adapters * d.c_out * q.padded * es);
    return q;
  }
  q.bt = round256((size_t)d.adapters * d.rank * d.c_out * es);
  q.at = round256((size_t)d.adapters * d.k * q.padded * es);
  q.g = round256((size_t)d.rows * q.rp * sizeof(float));
  q.parts = round256((size_t)q.rp * q.places * (es == 4 ? 4 : 6));
  const int wide = 16 * (16 / (int)es);      // columns of a work-group
  q.groups_b = (d.c_out - 1) / wide + 1, q.groups_a = (d.k - 1) / wide + 1;
  // slices: a round of work-groups, of two tiles at least
  const int groups = q.groups_a + q.groups_b;
  q.slices = std::max(1, std::min(256 * kOuterWaves / groups, (d.rows - 1) / kTileRows / 2 + 1));
  if (q.sorted) q.tile_at = round256((size_t)(d.adapters + 1) * sizeof(int));
  const size_t sums = q.slices + (q.sorted ? d.adapters : 1) - 1;
  q.sums_b = round256(sums * q.groups_b * wide * q.rp * sizeof(float));
  q.sums_a = round256(sums * q.groups_a * wide * q.rp * sizeof(float));
  return q;
}

// What a launch holds: fewer than 2^32 threads.
bool fits(const cprune_adapter_desc& d, const AdapterPlan& q, bool backward) {
  const double most = 4294967296.0 / 256;
  const int c = backward ? d.k : d.c_out;
  if ((double)q.tiles * q.splits >= most || (double)q.tiles * ((c - 1) / 256 + 1) >= most || (double)q.tiles * kTileRows >= 2147483648.0 || (double)q.tiles * q.ranks >= most) return false;
  if (!backward) return (double)q.tiles * q.splits * 256 + (double)d.adapters * d.c_out * q.padded / 4 < 4294967040.0;
  const double turned = (double)d.adapters * ((d.k + 63.0) / 64 + (d.c_out + 63.0) / 64) * 2;      // (ranks of up to 128 are two tiles)
  return turned < most / 4 - 1 && (double)q.slices * (q.groups_a + q.groups_b) < most && (double)d.adapters * (q.rp / 4.0 * ((double)d.k + d.c_out + 256) / 256 + 2) < most &&
         (double)std::max(q.groups_a, q.groups_b) * 128 * q.rp < 4294967296.0;
}

void launch(int dtype, AdapterPass pass, const void* args, const AdapterLaunch& l, hipStream_t s) {
  if (dtype == CPRUNE_F32) launch_adapter_f32(pass, args, l, s);
  else if (dtype == CPRUNE_F16) launch_adapter_f16(pass, args, l, s);
  else launch_adapter_bf16(pass, args, l, s);
}

struct Scratch {
  char* at;
  template <typename T> T* take(size_t bytes) {
    char* const p = at;
    at += bytes;
    return bytes ? reinterpret_cast<T*>(p) : nullptr;
  }
};

AdapterTiles tiles_of(const cprune_adapter_desc& d, const AdapterPlan& q, const int32_t* which) {
  AdapterTiles t = {};
  t.which = which, t.rows = d.rows, t.adapters = d.adapters, t.count = q.tiles, t.few = q.few;
  return t;
}

// The launch before the products; a, b: what is turned over, or empty
void prepare(const cprune_adapter_desc& d, const AdapterPlan& q, AdapterTiles& t, int* tile_at, const TurnArgs& a, const TurnArgs& b, Scratch& ws,
             hipStream_t s) {
  SortArgs sort = {};
  if (q.sorted) {
    int* const order = ws.take<int>(q.order);
    int* const tile_of = ws.take<int>(q.tile_of);
    sort = {t.which, d.rows, d.adapters, q.places, d.adapters > 384 ? kSortWaves / 2 : kSortWaves, order, tile_of, tile_at};
    t.order = order, t.tile_of = tile_of;
  }
  const int tiles_a = a.row_tiles * a.col_tiles * d.adapters, tiles_b = b.row_tiles * b.col_tiles * d.adapters;
  const unsigned grid = (unsigned)(q.sorted + tiles_a + tiles_b);
  if (!grid) return;
  const size_t es = dtype_size(d.dtype);
  size_t lds = q.sorted ? ((size_t)sort.waves * (d.adapters + 1) + d.adapters + 2) * sizeof(int) + 2048 * sort.waves : 0;
  if (tiles_a + tiles_b) lds = std::max(lds, 64 * 65 * es);
  if (es == 4) adapter_prepare_kernel<unsigned><<<grid, 64 * kSortWaves, lds, s>>>(sort, a, b, tiles_a);
  else adapter_prepare_kernel<unsigned short><<<grid, 64 * kSortWaves, lds, s>>>(sort, a, b, tiles_a);
}

// Columns of a work-group: by what the busiest compute unit has to bring and by the rounds of work-groups, each with its columns' waits and what it does but once, some
// 150 columns' time.
int columns_of(const cprune_adapter_desc& d, const AdapterPlan& q, int c) {
  const long tiles = rounded_tiles(d, q);
  int best = 256;
  if (q.few) {      // (a few rows each, all waiting for memory: side by side; 48 x 8192 x 8192, 32 adapters, 9.4 us in 256 columns, 11.2 in 512)
    while (best < 2048 && tiles * ((c - 1) / best + 1) > 1536) best *= 2;
    return best;
  }
  long least = std::numeric_limits<long>::max();
  for (int columns = 256; columns <= 2048; columns += 256) {
    const long groups = tiles * ((c - 1) / columns + 1), each = std::min(columns, c);
    const long cost = ((groups - 1) / 256 + 1) * each / 2 + ((groups - 1) / (256 * widen_waves(q.ranks, (int)dtype_size(d.dtype), d.dtype == CPRUNE_F16)) + 1) * (each + 150);
    if (cost < least) least = cost, best = columns;
  }
  return best;
}

}  // namespace
}  // namespace cprune

using namespace cprune;

extern "C" size_t cprune_adapter_workspace_bytes(const cprune_adapter_desc* d, int backward) {
  if (check(d, backward != 0) != CPRUNE_OK) return 0;
  const AdapterPlan q = plan_of(*d, backward != 0);
  return fits(*d, q, backward != 0) ? q.total() : 0;
}

extern "C" int cprune_adapter_linear(const cprune_adapter_desc* d, const void* x, const void* a, const void* b, const int32_t* which, const float* scale,
                                     const void* base, void* y, float* hidden, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check(d, false);
  if (rc != CPRUNE_OK) return rc;
  if (!x || !a || !b || !y || (d->mixed && !which) || (base && !base_fits(d, d->c_out)) || (base == y && base && d->base_stride != d->c_out)) return CPRUNE_ERR_INVALID_ARG;
  const AdapterPlan q = plan_of(*d, false);
  if (!fits(*d, q, false)) return CPRUNE_ERR_UNSUPPORTED;
  if (!ws || ws_bytes < q.total()) return CPRUNE_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(ws) & 15) return CPRUNE_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  Scratch scratch = {static_cast<char*>(ws)};
  AdapterTiles tiles = tiles_of(*d, q, which);
  prepare(*d, q, tiles, nullptr, {}, {}, scratch, s);
  float* const part = scratch.take<float>(q.part);
  AdapterLaunch l = {(unsigned)(q.tiles * q.splits), q.ranks, q.few || d->rows <= kFewTile, false};
  NarrowArgs n = {tiles, x, d->x_stride, d->k, d->rank, a, part, q.splits, q.per};
  if (d->rank % 8) {
    n.b = b, n.b_out = scratch.take<char>(q.bt), n.b_rank = d->rank, n.b_padded = q.padded;
    n.b_vectors = (long)d->adapters * d->c_out * q.padded / (16 / (long)dtype_size(d->dtype));
    b = n.b_out;
    l.grid += (unsigned)((n.b_vectors + 255) / 256);
  }
  launch(d->dtype, kAdapterNarrow, &n, l, s);
  WidenArgs w = {};
  w.tiles = tiles, w.part = part, w.splits = q.splits, w.rank = d->rank, w.scale = scale, w.b = b, w.c = d->c_out, w.b_stride = q.padded;
  w.base = base, w.base_stride = d->base_stride, w.y = y, w.hidden = hidden;
  w.act = d->act;
  w.columns = columns_of(*d, q, d->c_out);
  w.past = past_caches((double)d->rows * d->c_out * dtype_size(d->dtype));
  l.grid = (unsigned)(q.tiles * ((d->c_out - 1) / w.columns + 1));
  launch(d->dtype, kAdapterWiden, &w, l, s);
  CPRUNE_LAUNCH_CHECK();
  return CPRUNE_OK;
}

extern "C" int cprune_adapter_linear_backward(const cprune_adapter_desc* d, const void* dy, const void* x, const float* hidden, const void* a, const void* b,
                                              const int32_t* which, const float* scale, const void* dx_base, void* dx, float* da, float* db, void* ws,
                                              size_t ws_bytes, void* stream) {
  const int rc = check(d, true);
  if (rc != CPRUNE_OK) return rc;
  if (!dy || !a || !b || (d->mixed && !which) || (!dx && !da) || (da == nullptr) != (db == nullptr) || (da && (!x || !hidden)) ||
      (dx && dx_base && (!base_fits(d, d->k) || (dx_base == dx && d->base_stride != d->k))))
    return CPRUNE_ERR_INVALID_ARG;
  const AdapterPlan q = plan_of(*d, true);
  if (!fits(*d, q, true)) return CPRUNE_ERR_UNSUPPORTED;
  if (!ws || ws_bytes < q.total()) return CPRUNE_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(ws) & 15) return CPRUNE_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  Scratch scratch = {static_cast<char*>(ws)};
  AdapterTiles tiles = tiles_of(*d, q, which);
  int* const tile_at = scratch.take<int>(q.tile_at);
  char* const bt = scratch.take<char>(q.bt);
  char* const at = scratch.take<char>(q.at);
  auto tiles64 = [](int n) { return (n + 63) / 64; };
  const TurnArgs turn_a = {a, at, d->rank, d->k, q.padded, tiles64(q.padded), tiles64(d->k)}, turn_b = {b, bt, d->c_out, d->rank, d->c_out, tiles64(d->c_out), tiles64(d->rank)};
  prepare(*d, q, tiles, tile_at, dx ? turn_a : TurnArgs(), turn_b, scratch, s);
  float* const part = scratch.take<float>(q.part);
  float* const g = scratch.take<float>(q.g);
  char* const g_parts = scratch.take<char>(q.parts);
  char* const hidden_parts = scratch.take<char>(q.parts);
  float4_t* const sums_b = scratch.take<float4_t>(q.sums_b);
  float4_t* const sums_a = scratch.take<float4_t>(q.sums_a);
  const int v = 16 / (int)dtype_size(d->dtype);
  AdapterLaunch l = {(unsigned)(q.tiles * q.splits), q.ranks, d->rows <= kFewTile, d->k < v || d->c_out < v};
  const NarrowArgs n = {tiles, dy, d->dy_stride, d->c_out, d->rank, bt, part, q.splits, q.per};
  launch(d->dtype, kAdapterNarrow, &n, l, s);
  PartsArgs r = {};
  r.tiles = tiles, r.part = part, r.splits = q.splits, r.hidden = hidden, r.scale = scale, r.rank = d->rank, r.places = q.places;
  r.g = dx ? g : nullptr;
  if (da) r.g_out = g_parts, r.hidden_out = hidden_parts;
  l.grid = (unsigned)(q.tiles * q.ranks);
  launch(d->dtype, kAdapterParts, &r, l, s);
  if (dx) {
    WidenArgs w = {};
    w.tiles = tiles, w.part = g, w.splits = 1, w.rank = d->rank, w.b = at, w.c = d->k, w.b_stride = q.padded;
    w.base = dx_base, w.base_stride = d->base_stride, w.y = dx, w.act = CPRUNE_ACT_NONE;
    w.columns = columns_of(*d, q, d->k);
    w.past = past_caches((double)d->rows * d->k * dtype_size(d->dtype));
    l.grid = (unsigned)(q.tiles * ((d->k - 1) / w.columns + 1));
    launch(d->dtype, kAdapterWiden, &w, l, s);
  }
  if (da) {
    OuterArgs o = {};
    o.tiles = tiles, o.rank = d->rank, o.places = q.places;
    o.tile_at = tile_at, o.tile_count = q.tiles, o.slices = q.slices;
    o.side[0] = {dy, d->dy_stride, d->c_out, hidden_parts, sums_b, q.groups_b};
    o.side[1] = {x, d->x_stride, d->k, g_parts, sums_a, q.groups_a};
    l.grid = (unsigned)(q.slices * (q.groups_a + q.groups_b));
    launch(d->dtype, kAdapterOuter, &o, l, s);
    auto join = [&](auto lanes) {
      constexpr int LANES = decltype(lanes)::value, RESULTS = 256 / LANES;
      auto blocks = [&](int groups) { return (int)(((long)groups * 16 * v * q.rp / 4 - 1) / RESULTS + 1); };
      const JoinArgs j = {sums_b, sums_a, tile_at, q.tiles, q.slices, d->adapters, d->rank, q.ranks, v, d->k, d->c_out, q.groups_b, q.groups_a, blocks(q.groups_b), blocks(q.groups_a), da, db};
      adapter_join_kernel<LANES><<<(unsigned)(d->adapters * (j.blocks_b + j.blocks_a)), 256, 0, s>>>(j);
    };
    // (12544 x 576 x 96, rank 8, 85 slices: 12.2 us with one thread for a result, 4.9 with eight)
    if ((long)d->adapters * q.rp * (q.groups_a + q.groups_b) * 16 * v <= 262144 && q.slices >= 8) join(std::integral_constant<int, 8>());
    else join(std::integral_constant<int, 1>());
  }
  CPRUNE_LAUNCH_CHECK();
  return CPRUNE_OK;
}
