// Entry points of the low-rank adapters, and the launches around their products (adapter_kernel.hpp): rows sorted by adapter, transposes of A and B, sums of spans.
#include <algorithm>
#include <limits>

#include "adapter_kernel.hpp"

namespace cprune {
namespace {

constexpr int kMostRank = 128, kMostAdapters = 1024;
constexpr int kFewRows = 64;      // rows that a wavefront's ballot sorts

struct SortArgs {
  const int* which;
  int rows, adapters, places, span_tiles, spans;
  int *order, *tile_of;      // [places], [places / 64]
  int *span_first;           // [spans + 1]
  int *span_of;              // [adapters + 1], an adapter's first span
};

constexpr int kSortWaves = 8;

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

// One work-group: the rows of each adapter behind each other in their order, in tiles of their own, rows without an adapter last.  Wavefronts count runs of rows,
// a group of equal ones at a time, and place them on a second walk.
__global__ __launch_bounds__(64 * kSortWaves) void adapter_sort_kernel(const SortArgs p) {
  extern __shared__ int shared[];
  __shared__ int2 waves[kSortWaves];
  const int t = (int)threadIdx.x, lane = t & 63, wave = t >> 6, n = p.adapters, buckets = n + 1, threads = 64 * kSortWaves;
  int* const count = shared;                              // [wavefront][bucket]
  int* const tile_at = count + kSortWaves * buckets;      // [buckets + 1]
  int* const span_at = tile_at + buckets + 1;             // [adapters + 1]
  for (int i = t; i < kSortWaves * buckets; i += threads) count[i] = 0;
  __syncthreads();
  const int run = ((p.rows - 1) / threads + 1) * 64, from = (int)min((long)wave * run, (long)p.rows), end = (int)min((long)from + run, (long)p.rows);
  int* const mine = count + wave * buckets;
  auto walk = [&](auto&& place) __attribute__((always_inline)) {
    for (int r0 = from; r0 < end; r0 += 64) {
      const int r = r0 + lane;
      int b = r < end ? p.which[r] : 0;
      if ((unsigned)b >= (unsigned)n) b = n;
      unsigned long long left = __ballot(r < end);
      while (left) {
        const int lead = __ffsll(left) - 1, value = __shfl(b, lead, 64);
        const unsigned long long same = __ballot(r < end && b == value);
        int at = 0;
        if (lane == lead) {
          at = mine[value];
          mine[value] = at + __popcll(same);
        }
        at = __shfl(at, lead, 64);
        if (same >> lane & 1) place(at + __popcll(same & ((1ull << lane) - 1)), r);
        left &= ~same;
        __builtin_amdgcn_wave_barrier();      // (the next of the same adapter may be another lane's)
      }
    }
  };
  walk([](int, int) {});
  __syncthreads();
  // tiles and spans of each bucket, and where they begin
  const int each = (buckets - 1) / threads + 1, b0 = min(t * each, buckets), b1 = min(b0 + each, buckets);
  int2 sum = {0, 0};
  auto tiles_of = [&](int b) {
    int rows = 0;
    for (int w = 0; w < kSortWaves; ++w) rows += count[w * buckets + b];
    return make_int2(rows, (rows + kTileRows - 1) / kTileRows);
  };
  auto spans_of = [&](int b, int tiles) { return b < n ? (tiles + p.span_tiles - 1) / p.span_tiles : 0; };
  for (int b = b0; b < b1; ++b) {
    const int tiles = tiles_of(b).y;
    sum.x += tiles, sum.y += spans_of(b, tiles);
  }
  int2 before = sum;
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(before.x, o, 64), y = __shfl_up(before.y, o, 64);
    if (lane >= o) before.x += x, before.y += y;
  }
  if (lane == 63) waves[wave] = before;
  __syncthreads();
  before.x -= sum.x, before.y -= sum.y;
  for (int w = 0; w < wave; ++w) before.x += waves[w].x, before.y += waves[w].y;
  for (int b = b0; b < b1; ++b) {
    const int2 of = tiles_of(b);
    tile_at[b] = before.x;
    if (b <= n) span_at[b] = before.y;
    int at = before.x * kTileRows;
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = count[w * buckets + b];
      count[w * buckets + b] = at;
      at += c;
    }
    before.x += of.y, before.y += spans_of(b, of.y);
    for (; at < before.x * kTileRows; ++at) p.order[at] = -1;
    if (b == n) tile_at[buckets] = before.x;
  }
  __syncthreads();
  const int tiles = tile_at[buckets];
  for (int i = t; i < p.places / kTileRows; i += threads) {
    const int b = last_of(tile_at, buckets, i);
    p.tile_of[i] = i >= tiles ? -2 : b < n ? b : -1;
  }
  if (p.span_first) {
    for (int i = t; i <= p.spans; i += threads) {
      const int b = last_of(span_at, n, i);
      p.span_first[i] = b < n ? tile_at[b] + (i - span_at[b]) * p.span_tiles : tile_at[n];
    }
    for (int i = t; i <= n; i += threads) p.span_of[i] = span_at[i];
  }
  walk([&](int at, int r) { p.order[at] = r; });
}

// A [adapter][rank][k] -> [adapter][k][padded], zeros past the rank; B [adapter][c][rank] -> [adapter][rank][c].  A thread has a column of one.
template <typename T>
__global__ __launch_bounds__(256) void adapter_turn_kernel(const T* __restrict__ a, const T* __restrict__ b, int adapters, int rank, int padded, int k, int c, T* __restrict__ at,
                                                           T* __restrict__ bt) {
  const unsigned i = blockIdx.x * 256u + threadIdx.x;
  if (i < (unsigned)adapters * k) {
    if (!at) return;
    const unsigned n = i / k, col = i - n * k;
    for (int j = 0; j < padded; ++j) at[(long)i * padded + j] = j < rank ? a[((long)n * rank + j) * k + col] : (T)0.0f;
  } else if (i - (unsigned)adapters * k < (unsigned)adapters * c) {
    const unsigned m = i - (unsigned)adapters * k, n = m / c, col = m - n * c;
    for (int j = 0; j < rank; ++j) bt[((long)n * rank + j) * c + col] = b[(long)m * rank + j];
  }
}

// Sums of an adapter's spans, one behind the other: db [adapter][c][rank] from [span][c][RP], da [adapter][rank][k] from [span][RP][k].
__global__ __launch_bounds__(256) void adapter_join_kernel(const float* __restrict__ sums_b, const float* __restrict__ sums_a, const int* __restrict__ span_of, int spans, int adapters,
                                                           int rank, int rp, int k, int c, float* __restrict__ da, float* __restrict__ db) {
  const long all_b = (long)adapters * c * rank, i = (long)blockIdx.x * 256 + threadIdx.x;
  const bool of_b = i < all_b;
  const long m = of_b ? i : i - all_b;
  if (!of_b && m >= (long)adapters * rank * k) return;
  const long per = of_b ? (long)c * rank : (long)rank * k;
  const int n = (int)(m / per);
  const long in = m - n * per, pitch = of_b ? (long)c * rp : (long)rp * k;
  const long at = of_b ? in / rank * rp + in % rank : in;
  const int first = span_of ? span_of[n] : 0, last = span_of ? span_of[n + 1] : n == 0 ? spans : 0;
  const float* const from = (of_b ? sums_b : sums_a) + at;
  float s = 0.0f;
  for (int q = first; q < last; ++q) s += from[q * pitch];
  (of_b ? db : da)[m] = s;
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
  int span_tiles, spans;
  int groups_b, groups_a;              // work-groups a span, for dB and dA
  size_t order, tile_of, span_first, span_of, part, bt, at, g, parts, sums_b, sums_a;      // bytes
  size_t total() const { return order + tile_of + span_first + span_of + part + bt + at + g + 2 * parts + sums_b + sums_a; }
};

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
  // enough work-groups to bring x, each wavefront four steps at least
  const int terms = backward ? d.c_out : d.k, steps = (terms - 1) / q.step + 1;
  const int splits = std::max(1, std::min({1024 / q.tiles, steps / 16, 16}));
  q.per = (steps - 1) / splits + 1;
  q.splits = (steps - 1) / q.per + 1;
  q.part = round256((size_t)q.splits * d.rows * q.rp * sizeof(float));
  if (q.sorted) {
    q.order = round256((size_t)q.places * sizeof(int));
    q.tile_of = round256((size_t)q.tiles * sizeof(int));
  }
  if (!backward) return q;
  q.padded = (d.rank + 7) / 8 * 8;
  q.bt = round256((size_t)d.adapters * d.rank * d.c_out * es);
  q.at = round256((size_t)d.adapters * d.k * q.padded * es);
  q.g = round256((size_t)d.rows * q.rp * sizeof(float));
  q.parts = round256((size_t)q.rp * q.places * (es == 4 ? 4 : 6));
  const int wide = 4 * 16 * (16 / (int)es);      // columns of a work-group
  q.groups_b = (d.c_out - 1) / wide + 1, q.groups_a = (d.k - 1) / wide + 1;
  // spans: enough work-groups, and long enough that their sums are few beside what is read
  const int groups = q.groups_a + q.groups_b, want = std::max(1, 1024 / groups);
  q.span_tiles = std::max({1, (d.rows / kTileRows) / want, d.rank / 16});
  q.spans = q.sorted ? std::min(q.tiles, q.tiles / q.span_tiles + d.adapters) : (q.tiles - 1) / q.span_tiles + 1;
  if (q.sorted) {
    q.span_first = round256((size_t)(q.spans + 1) * sizeof(int));
    q.span_of = round256((size_t)(d.adapters + 1) * sizeof(int));
  }
  q.sums_b = round256((size_t)q.spans * d.c_out * q.rp * sizeof(float));
  q.sums_a = round256((size_t)q.spans * d.k * q.rp * sizeof(float));
  return q;
}

// What a launch holds: fewer than 2^32 threads.
bool fits(const cprune_adapter_desc& d, const AdapterPlan& q, bool backward) {
  const double most = 4294967296.0 / 256;
  const int c = backward ? d.k : d.c_out;
  if ((double)q.tiles * q.splits >= most || (double)q.tiles * ((c - 1) / 128 + 1) >= most || (double)q.tiles * kTileRows >= 2147483648.0) return false;
  if (!backward) return true;
  return (double)q.spans * (q.groups_a + q.groups_b) < most && (double)d.adapters * d.rank * ((double)d.k + d.c_out) < 4294967040.0;
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
  t.which = which, t.rows = d.rows, t.adapters = d.adapters, t.few = q.few;
  return t;
}

void sort_rows(const cprune_adapter_desc& d, const AdapterPlan& q, AdapterTiles& t, int* span_first, int* span_of, Scratch& ws, hipStream_t s) {
  int* const order = ws.take<int>(q.order);
  int* const tile_of = ws.take<int>(q.tile_of);
  const SortArgs a = {t.which, d.rows, d.adapters, q.places, std::max(1, q.span_tiles), q.spans, order, tile_of, span_first, span_of};
  const size_t lds = ((size_t)kSortWaves * (d.adapters + 1) + 2 * d.adapters + 4) * sizeof(int);
  adapter_sort_kernel<<<1, 64 * kSortWaves, lds, s>>>(a);
  t.order = order, t.tile_of = tile_of;
}

int columns_of(const AdapterPlan& q, int c) {      // of a work-group: fewer where tiles are few
  int columns = 512;
  while (columns > 128 && (long)q.tiles * ((c - 1) / columns + 1) < 1024) columns /= 2;
  return columns;
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
  if (q.sorted) sort_rows(*d, q, tiles, nullptr, nullptr, scratch, s);
  float* const part = scratch.take<float>(q.part);
  AdapterLaunch l = {(unsigned)(q.tiles * q.splits), q.ranks, d->act == CPRUNE_ACT_SILU};
  const NarrowArgs n = {tiles, x, d->x_stride, d->k, d->rank, a, part, q.splits, q.per};
  launch(d->dtype, kAdapterNarrow, &n, l, s);
  const float open = std::numeric_limits<float>::infinity();
  WidenArgs w = {};
  w.tiles = tiles, w.part = part, w.splits = q.splits, w.rank = d->rank, w.scale = scale, w.b = b, w.c = d->c_out, w.b_stride = d->rank;
  w.base = base, w.base_stride = d->base_stride, w.y = y, w.hidden = hidden;
  w.lo = d->act == CPRUNE_ACT_NONE || d->act == CPRUNE_ACT_SILU ? -open : 0.0f, w.hi = d->act == CPRUNE_ACT_RELU6 ? 6.0f : open;
  w.columns = columns_of(q, d->c_out);
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
  int* const span_first = scratch.take<int>(q.span_first);
  int* const span_of = scratch.take<int>(q.span_of);
  if (q.sorted) sort_rows(*d, q, tiles, span_first, span_of, scratch, s);
  float* const part = scratch.take<float>(q.part);
  char* const bt = scratch.take<char>(q.bt);
  char* const at = scratch.take<char>(q.at);
  float* const g = scratch.take<float>(q.g);
  char* const g_parts = scratch.take<char>(q.parts);
  char* const hidden_parts = scratch.take<char>(q.parts);
  float* const sums_b = scratch.take<float>(q.sums_b);
  float* const sums_a = scratch.take<float>(q.sums_a);
  const unsigned turns = (unsigned)(((long)d->adapters * ((long)d->k + d->c_out) + 255) / 256);
  if (d->dtype == CPRUNE_F32)
    adapter_turn_kernel<unsigned><<<turns, 256, 0, s>>>(static_cast<const unsigned*>(a), static_cast<const unsigned*>(b), d->adapters, d->rank, q.padded, d->k, d->c_out,
                                                        dx ? reinterpret_cast<unsigned*>(at) : nullptr, reinterpret_cast<unsigned*>(bt));
  else
    adapter_turn_kernel<unsigned short><<<turns, 256, 0, s>>>(static_cast<const unsigned short*>(a), static_cast<const unsigned short*>(b), d->adapters, d->rank, q.padded, d->k,
                                                              d->c_out, dx ? reinterpret_cast<unsigned short*>(at) : nullptr, reinterpret_cast<unsigned short*>(bt));
  AdapterLaunch l = {(unsigned)(q.tiles * q.splits), q.ranks, false};
  const NarrowArgs n = {tiles, dy, d->dy_stride, d->c_out, d->rank, bt, part, q.splits, q.per};
  launch(d->dtype, kAdapterNarrow, &n, l, s);
  PartsArgs r = {};
  r.tiles = tiles, r.part = part, r.splits = q.splits, r.hidden = hidden, r.scale = scale, r.rank = d->rank, r.places = q.places;
  r.g = dx ? g : nullptr;
  if (da) r.g_out = g_parts, r.hidden_out = hidden_parts;
  l.grid = (unsigned)q.tiles;
  launch(d->dtype, kAdapterParts, &r, l, s);
  if (dx) {
    const float open = std::numeric_limits<float>::infinity();
    WidenArgs w = {};
    w.tiles = tiles, w.part = g, w.splits = 1, w.rank = q.padded, w.b = at, w.c = d->k, w.b_stride = q.padded;
    w.base = dx_base, w.base_stride = d->base_stride, w.y = dx, w.lo = -open, w.hi = open;
    w.columns = columns_of(q, d->k);
    l.grid = (unsigned)(q.tiles * ((d->k - 1) / w.columns + 1));
    launch(d->dtype, kAdapterWiden, &w, l, s);
  }
  if (da) {
    OuterArgs o = {};
    o.tiles = tiles, o.rank = d->rank, o.places = q.places;
    o.span_first = span_first, o.span_tiles = q.span_tiles, o.tile_count = q.tiles;
    o.side[0] = {dy, d->dy_stride, d->c_out, hidden_parts, sums_b, q.groups_b};
    o.side[1] = {x, d->x_stride, d->k, g_parts, sums_a, q.groups_a};
    l.grid = (unsigned)(q.spans * (q.groups_a + q.groups_b));
    launch(d->dtype, kAdapterOuter, &o, l, s);
    const long all = (long)d->adapters * d->rank * ((long)d->k + d->c_out);
    adapter_join_kernel<<<(unsigned)((all + 255) / 256), 256, 0, s>>>(sums_b, sums_a, span_of, q.spans, d->adapters, d->rank, q.rp, d->k, d->c_out, da, db);
  }
  CPRUNE_LAUNCH_CHECK();
  return CPRUNE_OK;
}
