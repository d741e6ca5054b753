// Low-rank adapters: hidden_r = scale_i A_i x_r, y_r = act(base_r + B_i hidden_r), and their gradients, i the row's adapter.
//
// Rows in tiles of 64 with one adapter: all rows in their order where there is one adapter, the rows of each adapter behind each other where a launch before has
// sorted them, or, up to 64 rows, sixteen at most that a work-group finds with a ballot.  A tile's rows are gathered: a row is long, its place is not.
//
// Products on the matrix cores, an operand 16 bytes of a row for each lane: lane l has row l % 16 and the terms from 4 V times the step and V (l / 16) on, V numbers of 16
// bytes.  fp32 takes four instructions a step, one for each of a lane's four terms (the terms' order does not matter, both operands
// have the same).
//  - narrow: 64 rows of x against A (or of dy against B's transpose) through LDS, 4 wavefronts sharing the terms, work-groups sharing long sums; bound by reading x.
//  - widen: hidden against B (or g against A's transpose), 8 neighbouring results in each lane; bound by reading base and writing y.
//  - outer: dy against hidden (x against g), summed over rows.  The terms are rows: a lane reads 16 bytes of V rows and turns the V x V numbers over in registers.
//    Equal slices of the rows leave sums for each adapter that they meet, joined in a fixed order.  Bound by reading dy (x).
// hidden and g are fp32; against 16-bit operands they go as three bf16 parts, of 8 bits each, which are all of it.  An fp16 operand beside them is two bf16 parts itself,
// exactly, so that every product is whole.  (Two parts for y and dx left out up to 2^-15 of a term, which is seen where terms cancel, and took as long up to rank 32, 1% less at
// rank 64 in bf16, 8% in fp16.)
#pragma once
#include <type_traits>

#include "conv_kernel.hpp"
#include "adapter_columns.hpp"
#include "past_caches.hpp"

namespace cprune {

constexpr int kTileRows = 64, kFewTile = 16;

// Work-groups of 256 that a compute unit holds at once, by registers; what is cut into work-groups is cut for whole rounds of them.
// (widen in fp16 at rank 64 has B's parts besides: three spill 32 registers, and 16384 x 4096 x 11008 takes 290 us and not 242)
constexpr int narrow_waves(int ranks) { return ranks <= 2 ? 3 : ranks <= 4 ? 2 : 1; }
constexpr int widen_waves(int ranks, int size, bool fp16) { return ranks * size <= (fp16 ? 4 : 8) ? 3 : ranks * size <= 16 ? 2 : 1; }
constexpr int kOuterWaves = 2;

// Places: tile t has rows order[64 t .. 64 t + 63], -1 where it has fewer.
struct AdapterTiles {
  const int* which;        // few: the rows' adapters; tile t is that of row t and the next ones of its adapter, if as many as fill tiles are before it
  const int* order;        // sorted, or null: row 64 t + i
  const int* tile_of;      // sorted: adapter of a tile, -1 for rows without; past the last tile -2
  int rows, adapters, count;      // (tiles there may be)
  bool few;
};

struct NarrowArgs {
  AdapterTiles tiles;
  const void* x;           // [rows][stride]
  long stride;
  int k, rank;
  const void* a;           // [adapters][rank][k]
  float* part;             // [splits][rows][RP]
  int splits, per;         // work-groups that share a sum, chunks of 256 bytes of each
  // B filled up for widen by the work-groups past these, 16 bytes a thread: [row][b_rank] -> [row][b_padded], zeros past the rank; b_vectors 0: none
  const void* b;
  void* b_out;
  long b_vectors;
  int b_rank, b_padded;
};

struct WidenArgs {
  AdapterTiles tiles;
  const float* part;       // [splits][rows][RP]
  int splits, rank;
  const float* scale;      // or null
  const void* b;           // [adapters][c][b_stride], rank numbers of each row, then zeros: a multiple of 8
  int c, b_stride;
  const void* base;
  long base_stride;
  void* y;                 // [rows][c]
  float* hidden;           // [rows][rank] or null
  int act;
  int columns;             // of a work-group, a multiple of 128
  bool past;               // y is stored past the caches
};

// hidden and g as the outer product's operands, by steps of its terms, places: 16-bit, three bf16 parts [3][places / 32][RP][32], fp32 [places / 16][RP][16]
struct PartsArgs {
  AdapterTiles tiles;
  const float* part;       // g: [splits][rows][RP]
  int splits;
  const float* hidden;     // [rows][rank]
  const float* scale;
  int rank, places;
  void *g_out, *hidden_out;
  float* g;                // [rows][RP], summed and scaled; or null
};

struct OuterSide {
  const void* x;           // [rows][stride]
  long stride;
  int c;                   // columns
  const void* parts;       // the other operand
  float4_t* sums;          // [slices + adapters - 1][groups][V][NR][lane], as the products leave them
  int groups;              // work-groups for a slice, of 16 V columns
};
struct OuterArgs {
  AdapterTiles tiles;
  OuterSide side[2];       // dy and hidden; x and g
  int rank, places;
  const int* tile_at;      // sorted: [adapters + 1], an adapter's first tile
  int tile_count;          // otherwise
  int slices;              // at most, that the tiles are cut into, whatever their adapters: what adapter i has of slice s is sum s + i
};

struct AdapterLaunch {
  unsigned grid;
  int ranks;               // RP / 16, RP the rank filled up to 16, 32, 64 or 128
  bool few;                // tiles of up to 16 rows (narrow, widen)
  bool thin;               // a side has fewer than V columns (outer)
};
enum AdapterPass { kAdapterNarrow, kAdapterWiden, kAdapterParts, kAdapterOuter };
void launch_adapter_f32(AdapterPass pass, const void* args, const AdapterLaunch& l, hipStream_t s);
void launch_adapter_f16(AdapterPass pass, const void* args, const AdapterLaunch& l, hipStream_t s);
void launch_adapter_bf16(AdapterPass pass, const void* args, const AdapterLaunch& l, hipStream_t s);

namespace adapter {

template <typename T> constexpr int kV = 16 / (int)sizeof(T);       // numbers of 16 bytes
template <typename T> constexpr int kStep = 4 * kV<T>;              // terms of a step

// V numbers at p, at any element
template <typename T> __device__ __forceinline__ uint4 load(const T* p) {
  typedef unsigned uint4u __attribute__((ext_vector_type(4), aligned(2)));
  const uint4u v = *reinterpret_cast<const uint4u*>(p);
  return make_uint4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ uint4 keep(const uint4& v, bool all) { return make_uint4(all ? v.x : 0u, all ? v.y : 0u, all ? v.z : 0u, all ? v.w : 0u); }
// V numbers at p, of which `valid` are there, zeros past them.  Long code: for what is left at an end, not for a loop's every load.
template <typename T> __device__ __forceinline__ uint4 load_some(const T* p, int valid) {
  if (valid >= kV<T>) return load(p);
  if (valid <= 0) return make_uint4(0, 0, 0, 0);
  unsigned w[4];
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(p[min(i, valid - 1)]);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = i < valid ? w[i] : 0u;
  } else {
    const unsigned short* const h = reinterpret_cast<const unsigned short*>(p);
    unsigned v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = h[min(i, valid - 1)];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (2 * i < valid ? v[2 * i] : 0u) | (2 * i + 1 < valid ? v[2 * i + 1] << 16 : 0u);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// result v of lane l: row 4 (l / 16) + v of the first operand, l % 16 of the second
template <typename T> __device__ __forceinline__ float4_t mma(const uint4& a, const uint4& b, float4_t acc) {
  if constexpr (sizeof(T) == 4) {
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(b.x), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(b.y), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(b.z), acc, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(b.w), acc, 0, 0, 0);
  } else if constexpr (std::is_same<T, _Float16>::value) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), acc, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
  }
}

// Numbers in fp32 as bf16 parts: the first 8 bits, cut off, then of what is left; three parts are all 24 (an infinity is the first part alone)
__device__ __forceinline__ float part_of(float& left) {
  const float p = __uint_as_float(__float_as_uint(left) & 0xffff0000u);
  left = __builtin_isinf(left) ? 0.0f : left - p;
  return p;
}
__device__ __forceinline__ unsigned pair(float a, float b) { return __float_as_uint(a) >> 16 | (__float_as_uint(b) & 0xffff0000u); }
template <int N> __device__ __forceinline__ void parts_of(float (&v)[8], uint4 (&p)[N]) {
#pragma unroll
  for (int n = 0; n < N; ++n) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = part_of(v[i]);
    p[n] = make_uint4(pair(f[0], f[1]), pair(f[2], f[3]), pair(f[4], f[5]), pair(f[6], f[7]));
  }
}
// eight fp16 numbers as two bf16 parts
__device__ __forceinline__ void halves_of(const uint4& r, uint4 (&p)[2]) {
  const half8_t h = __builtin_bit_cast(half8_t, r);
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)h[i];
  parts_of<2>(v, p);
}

// What an operand of memory and N parts of an fp32 one make; a and p either way round (SWAP: p's are the first operand)
template <typename T, int N, bool SWAP> __device__ __forceinline__ float4_t mma_parts(const uint4& a, const uint4 (&p)[N], float4_t acc) {
  auto go = [&](const uint4& u, const uint4& v) __attribute__((always_inline)) { acc = SWAP ? mma<__bf16>(v, u, acc) : mma<__bf16>(u, v, acc); };
  if constexpr (std::is_same<T, _Float16>::value) {
    uint4 h[2];
    halves_of(a, h);
#pragma unroll
    for (int n = N - 1; n >= 0; --n) go(h[1], p[n]);
#pragma unroll
    for (int n = N - 1; n >= 0; --n) go(h[0], p[n]);
  } else {
#pragma unroll
    for (int n = N - 1; n >= 0; --n) go(a, p[n]);
  }
  return acc;
}

// A tile's adapter (-1: none, -2: no such tile) and rows, -1 where there are fewer; in LDS
struct Tile {
  int row[kTileRows];
};
__device__ __forceinline__ int open_tile(const AdapterTiles& t, int tile, Tile& out, int& count) {
  const int i = (int)threadIdx.x;
  int adapter = 0;
  if (t.few) {
    const int lane = i & 63;
    int mine = lane < t.rows ? t.which[lane] : -2;
    if (lane < t.rows && (unsigned)mine >= (unsigned)t.adapters) mine = -1;
    adapter = __shfl(mine, tile, 64);
    unsigned long long same = __ballot(mine == adapter);
    if (__popcll(same & ((1ull << tile) - 1)) % kFewTile) return -2;
    same &= ~0ull << tile;
    count = min(__popcll(same), kFewTile);
    if (i < kTileRows) out.row[i] = -1;
    __syncthreads();
    const int at = __popcll(same & ((1ull << lane) - 1));
    if (i < kTileRows && (same >> lane & 1) && at < kFewTile) out.row[at] = lane;
  } else if (t.order) {
    adapter = t.tile_of[tile];
    if (adapter == -2) return -2;
    if (i < kTileRows) out.row[i] = t.order[tile * kTileRows + i];
    count = kTileRows;
  } else {
    if (i < kTileRows) {
      const int r = tile * kTileRows + i;
      out.row[i] = r < t.rows ? r : -1;
    }
    count = min(kTileRows, t.rows - tile * kTileRows);
    if (t.adapters < 1) adapter = -1;
  }
  __syncthreads();
  return adapter;
}

// what a wavefront has written to LDS is there for its other lanes
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// four numbers of each of the splits' parts, added up; four loads under way
__device__ __forceinline__ float4_t sum_parts(const float* from, int splits, long pitch) {
  float4_t v = {0.f, 0.f, 0.f, 0.f};
  int s = 0;
  for (; s + 4 <= splits; s += 4) {
    float4_t q[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) q[u] = *reinterpret_cast<const float4_t*>(from + (s + u) * pitch);
#pragma unroll
    for (int u = 0; u < 4; ++u) v += q[u];
  }
  for (; s < splits; ++s) v += *reinterpret_cast<const float4_t*>(from + s * pitch);
  return v;
}

// ---- narrow ----------------------------------------------------------------------

// 256 bytes of every row at a time through LDS, two ahead of what is multiplied: asked for in whole lines, 16 lanes a row.  As operands, 16 rows x 64 bytes, a compute
// unit brings half as much: 8192 x 4096 bf16 rank 64 took 31 us, now 23; 16384 x 4096 rank 32 took 42, now 39 (3.4 TB/s of x; 28 where part of
// x is still in the last-level cache).  F: a tile's rows in sixteens, 4, or 1 where
// there are no more.  Rows that a tile has not are its first one again: they make results of their own, which nobody reads.  Ranks past the last are the last
// again, left out by who reads them.
template <typename T, int NR, int F>
__global__ __launch_bounds__(256, narrow_waves(NR)) void adapter_narrow_kernel(const NarrowArgs p) {
  constexpr int V = kV<T>, RP = 16 * NR, PIECES = 16, CHUNK = PIECES * V, PITCH = PIECES + 1, LINES = 16 * (F + NR);
  __shared__ Tile tile;
  __shared__ uint4 staged[2][LINES][PITCH];
  const int t = (int)threadIdx.x, lane = t & 63, wave = t >> 6, quarter = lane >> 4, lrow = lane & 15;
  const int tile_no = blockIdx.x / (unsigned)p.splits, split = blockIdx.x - tile_no * p.splits;
  if (tile_no >= p.tiles.count) {
    const long i = (long)(blockIdx.x - p.tiles.count * p.splits) * 256 + t;
    if (i >= p.b_vectors) return;
    const int per = p.b_padded / V;
    const long row = i / per;
    const int at = (int)(i - row * per) * V;
    static_cast<uint4*>(p.b_out)[i] = load_some(static_cast<const T*>(p.b) + row * p.b_rank + at, p.b_rank - at);
    return;
  }
  int count;
  const int adapter = open_tile(p.tiles, tile_no, tile, count);
  if (adapter < 0) return;      // (rows without an adapter: what would be read here is known to be 0)
  // this thread's piece of every sixteenth line: rows, then ranks
  const int line = t >> 4, piece = t & 15;
  const T* from[F + NR];
#pragma unroll
  for (int f = 0; f < F; ++f) {
    const int r = tile.row[16 * f + line];
    from[f] = static_cast<const T*>(p.x) + (long)(r >= 0 ? r : tile.row[0]) * p.stride + piece * V;
  }
#pragma unroll
  for (int n = 0; n < NR; ++n) from[F + n] = static_cast<const T*>(p.a) + ((long)adapter * p.rank + min(16 * n + line, p.rank - 1)) * p.k + piece * V;
  struct Chunk {
    uint4 v[F + NR];
  };
  auto fetch = [&](int c, Chunk& q) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < F + NR; ++i) q.v[i] = load(from[i] + (long)c * CHUNK);
  };
  auto stage = [&](int buffer, const Chunk& q) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < F + NR; ++i) staged[buffer][16 * i + line][piece] = q.v[i];
  };
  float4_t acc[F][NR];
#pragma unroll
  for (int f = 0; f < F; ++f)
#pragma unroll
    for (int n = 0; n < NR; ++n) acc[f][n] = (float4_t){0.f, 0.f, 0.f, 0.f};
  // a wavefront has a quarter of the chunk's terms: four pieces of every line
  auto multiply = [&](int buffer) __attribute__((always_inline)) {
    uint4 x[F];
#pragma unroll
    for (int f = 0; f < F; ++f) x[f] = staged[buffer][16 * f + lrow][4 * wave + quarter];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const uint4 a = staged[buffer][16 * (F + n) + lrow][4 * wave + quarter];
#pragma unroll
      for (int f = 0; f < F; ++f) acc[f][n] = mma<T>(a, x[f], acc[f][n]);
    }
  };
  const int whole = p.k / CHUNK, first = split * p.per, last = min(first + p.per, whole);
  Chunk now, next;
  if (first < last) {
    fetch(first, now);
    fetch(min(first + 1, last - 1), next);
    stage(0, now);
  }
#pragma unroll 1
  for (int c = first; c < last; c += 2) {
    __syncthreads();
    fetch(min(c + 2, last - 1), now);
    multiply(0);
    stage(1, next);
    if (c + 1 >= last) break;
    __syncthreads();
    fetch(min(c + 3, last - 1), next);
    multiply(1);
    stage(0, now);
  }
  if (p.k % CHUNK && split == p.splits - 1) {      // what is left of the rows, zeros past it
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < F + NR; ++i) {
      const T* q = from[0];
#pragma unroll
      for (int u = 1; u < F + NR; ++u) q = i == u ? from[u] : q;
      staged[0][16 * i + line][piece] = load_some(q + (long)whole * CHUNK, p.k - whole * CHUNK - piece * V);
    }
    __syncthreads();
    multiply(0);
  }
  __syncthreads();
  float (*const sums)[16][RP + 4] = reinterpret_cast<float (*)[16][RP + 4]>(staged);      // [wavefront]
  static_assert(sizeof(float) * 4 * 16 * (RP + 4) <= sizeof(staged), "the wavefronts' sums take the chunks' place");
  const int frags = min((count + 15) / 16, F);
#pragma unroll
  for (int f = 0; f < F; ++f) {
    if (f >= frags) break;
    if (f) __syncthreads();
#pragma unroll
    for (int n = 0; n < NR; ++n) *reinterpret_cast<float4_t*>(&sums[wave][lrow][16 * n + 4 * quarter]) = acc[f][n];
    __syncthreads();
    for (int i = t; i < 16 * RP / 4; i += 256) {
      const int r = i / (RP / 4), j = 4 * (i - r * (RP / 4)), row = tile.row[16 * f + r];
      if (row < 0) continue;
      float4_t v = *reinterpret_cast<const float4_t*>(&sums[0][r][j]);
#pragma unroll
      for (int w = 1; w < 4; ++w) v += *reinterpret_cast<const float4_t*>(&sums[w][r][j]);
      *reinterpret_cast<float4_t*>(p.part + ((long)split * p.tiles.rows + row) * RP + j) = v;
    }
  }
}

// ---- widen -----------------------------------------------------------------------

// A wavefront has 64 columns at a time of a tile's rows: B's numbers in registers, hidden in LDS as operands, results through LDS so that base and y are met in whole lines,
// the next rows' base asked for as this one's is used.  Bound by base and y: 16384 x 11008, rank 32, bf16 148 us, 4.9 TB/s; 8192 x 4096, rank 64, 44 us.
template <typename T, int NR, int F>
__global__ __launch_bounds__(256, (widen_waves(NR, sizeof(T), std::is_same<T, _Float16>::value))) void adapter_widen_kernel(const WidenArgs p) {
  constexpr int V = kV<T>, STEP = kStep<T>, RP = 16 * NR, NS = (RP + STEP - 1) / STEP, N = sizeof(T) == 4 ? 1 : 3, M = std::is_same<T, _Float16>::value ? 2 : 1;
  __shared__ Tile tile;
  // Two buffers, the next rows multiplied while these are finished; one where hidden's parts and a second one leave room for fewer work-groups (8192 x 4096 x 4096 bf16, rank
  // 64 87.6 us with two and 77.6 with one, rank 128 178 and 126).
  constexpr int BUFS = F == 1 || (sizeof(T) == 2 && NR >= 4) ? 1 : 2;
  __shared__ alignas(16) float results[4][BUFS][16][64 + 4];
  __shared__ uint4 hidden[16 * F][NS * N * 4 + 1];      // as operands: step, part, quarter
  const int t = (int)threadIdx.x, lane = t & 63, wave = t >> 6, quarter = lane >> 4, lrow = lane & 15;
  const int chunks = (p.c - 1) / p.columns + 1;
  const int tile_no = blockIdx.x / (unsigned)chunks, chunk = blockIdx.x - tile_no * chunks;
  int count;
  const int adapter = open_tile(p.tiles, tile_no, tile, count);
  if (adapter == -2) return;
  const int frags = min((count + 15) / 16, F);      // (a sorted tile is 64 places, whatever its rows)
  // The rows' hidden numbers, zeros past the rank: asked for before all else, so that what is asked for next need not be waited for with them.
  constexpr int ITEMS = (16 * F * NS * STEP / 4 + 255) / 256;
  float4_t held[ITEMS];
  const float scale = adapter >= 0 && p.scale ? p.scale[adapter] : 1.0f;
#pragma unroll
  for (int u = 0; u < ITEMS; ++u) {
    const int i = t + 256 * u, r = i / (NS * STEP / 4), j = 4 * (i - r * (NS * STEP / 4)), row = r < 16 * F ? tile.row[r] : -1;
    held[u] = (float4_t){0.f, 0.f, 0.f, 0.f};
    if (row >= 0 && adapter >= 0 && j < p.rank) held[u] = sum_parts(p.part + (long)row * RP + j, p.splits, (long)p.tiles.rows * RP);
  }
  // 64 columns at a time.  Columns past the last are the last again, whose results nobody stores.
  const T* const b = static_cast<const T*>(p.b) + (long)max(adapter, 0) * p.c * p.b_stride;
  const int run = p.columns / 4, begin = chunk * p.columns + wave * run, end = min(p.c, begin + run);
  auto weights = [&](int c0, uint4 (&w)[4][NS]) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const T* const from = b + (long)min(c0 + 16 * g + lrow, p.c - 1) * p.b_stride;
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const int j = s * STEP + quarter * V;
        w[g][s] = keep(load(from + (j < p.b_stride ? j : 0)), j < p.b_stride && adapter >= 0);
      }
    }
  };
  constexpr bool AHEAD = NS <= 2;      // the next columns' weights are asked for before these are multiplied, where registers hold both
  uint4 next[4][NS];
  if (AHEAD && begin < end) weights(begin, next);
  // base, of the next columns as soon as these rows' have been used; LINE lanes of 16 bytes a row, so that it and y are met in whole lines
  constexpr int LINE = 64 / V, EACH = 16 * LINE / 64;
  const int line = lane / LINE, col = lane % LINE * V, tail = p.c % V;
  const T* const base = static_cast<const T*>(p.base);
  T* const y = static_cast<T*>(p.y);
  const bool with_base = base && p.c >= V;
  uint4 z[F][EACH];
  auto ask = [&](int f, int c0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int row = tile.row[16 * f + i * (64 / LINE) + line];
      z[f][i] = load(base + (long)(row >= 0 ? row : tile.row[0]) * p.base_stride + min(c0 + col, p.c - V));
    }
  };
  if (with_base && begin < end) {
#pragma unroll
    for (int f = 0; f < F; ++f)
      if (f < frags) ask(f, begin);
  }
#pragma unroll
  for (int u = 0; u < ITEMS; ++u) {
    const int i = t + 256 * u, r = i / (NS * STEP / 4), j = 4 * (i - r * (NS * STEP / 4));
    if (r >= 16 * F) break;
    const int row = tile.row[r];
    float4_t v = scale * held[u];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = j + e < p.rank && row >= 0 && adapter >= 0 ? v[e] : 0.0f;
      if (p.hidden && chunk == 0 && row >= 0 && j + e < p.rank) p.hidden[(long)row * p.rank + j + e] = v[e];
    }
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<float4_t*>(&hidden[r][j / 4]) = v;
    } else {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        float f[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float left = v[e];
          f[e] = part_of(left);
          v[e] = left;
        }
        uint2* const to = reinterpret_cast<uint2*>(&hidden[r][(j / STEP * N + n) * 4 + j % STEP / V]);
        to[j / 4 & 1] = make_uint2(pair(f[0], f[1]), pair(f[2], f[3]));
      }
    }
  }
  __syncthreads();
  auto finish = [&](float v) __attribute__((always_inline)) {
    if (p.act == CPRUNE_ACT_SILU) return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.44269504f));      // (2^x flushes below 2^-126: 1 + e^-z does not see it)
    if (p.act != CPRUNE_ACT_NONE) v = v < 0.0f ? 0.0f : v;      // (comparisons and not minimum / maximum: a NaN stays one)
    return p.act == CPRUNE_ACT_RELU6 && v > 6.0f ? 6.0f : v;
  };
  typedef T numbers __attribute__((ext_vector_type(V)));
  typedef T outs __attribute__((ext_vector_type(V), aligned(2)));
  // Results go through LDS, 16 rows of a wavefront at a time
#pragma unroll 1
  for (int c0 = begin; c0 < end; c0 += 64) {
    const int c = c0 + col;
    const bool whole = c + V <= p.c;
    uint4 w[4][NS][M];
    if constexpr (!AHEAD) weights(c0, next);
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        if constexpr (M == 2) halves_of(next[g][s], w[g][s]);
        else w[g][s][0] = next[g][s];
      }
    if constexpr (AHEAD) weights(min(c0 + 64, end - 1), next);
    auto multiply = [&](int f) __attribute__((always_inline)) {
      float (*const out)[64 + 4] = results[wave][f % BUFS];
      uint4 h[NS][N];
#pragma unroll
      for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int n = 0; n < N; ++n) h[s][n] = hidden[16 * f + lrow][(s * N + n) * 4 + quarter];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        float4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          if constexpr (sizeof(T) == 4) {
            acc = mma<float>(w[g][s][0], h[s][0], acc);
          } else {
#pragma unroll
            for (int m = M - 1; m >= 0; --m)
#pragma unroll
              for (int n = N - 1; n >= 0; --n) acc = mma<__bf16>(w[g][s][m], h[s][n], acc);
          }
        }
        *reinterpret_cast<float4_t*>(&out[lrow][16 * g + 4 * quarter]) = acc;
      }
    };
    if constexpr (BUFS == 2) {
      multiply(0);
      wave_sync();
    }
#pragma unroll
    for (int f = 0; f < F; ++f) {
      if (f >= frags) break;
      if constexpr (BUFS == 2) {
        if (f + 1 < F && f + 1 < frags) multiply(f + 1);
      } else {
        multiply(f);
        wave_sync();
      }
      const float (*const out)[64 + 4] = results[wave][f % BUFS];
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const int in = i * (64 / LINE) + line, row = tile.row[16 * f + in];
        float v[V];
#pragma unroll
        for (int e = 0; e < V; e += 4) {
          const float4_t q = *reinterpret_cast<const float4_t*>(&out[in][col + e]);
#pragma unroll
          for (int u = 0; u < 4; ++u) v[e + u] = q[u];
        }
        if (with_base) {
          const numbers n = __builtin_bit_cast(numbers, z[f][i]);
#pragma unroll
          for (int e = 0; e < V; ++e) v[e] += Elem<T>::to_f32(n[e]);
        }
        if (p.act != CPRUNE_ACT_NONE) {
#pragma unroll
          for (int e = 0; e < V; ++e) v[e] = finish(v[e]);
        }
        outs o;
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = Elem<T>::from_f32(v[e]);
        if (row >= 0 && whole) {
          outs* const to = reinterpret_cast<outs*>(y + (long)row * p.c + c);
          CPRUNE_STORE(to, o, p.past);
        }
      }
      if (tail && c0 + 64 >= p.c) {      // the last columns, fewer than a vector
#pragma unroll 1
        for (int i = lane; i < 16 * tail; i += 64) {
          const int in = i / tail, at = p.c - tail + i - in * tail, row = tile.row[16 * f + in];
          if (row < 0) continue;
          float v = out[in][at - c0];
          if (base) v += Elem<T>::to_f32(base[(long)row * p.base_stride + at]);
          y[(long)row * p.c + at] = Elem<T>::from_f32(finish(v));
        }
      }
      if (with_base && c0 + 64 < end) ask(f, c0 + 64);
      wave_sync();
    }
  }
}

// ---- operands of the outer products ----------------------------------------------

// A work-group has 64 places of 16 ranks: read four ranks of a place at a time, turned over in LDS, written 8 (4) places of a rank at a time.
template <typename T, int NR>
__global__ __launch_bounds__(256) void adapter_parts_kernel(const PartsArgs p) {
  constexpr int V = kV<T>, RP = 16 * NR, N = sizeof(T) == 4 ? 1 : 3;
  __shared__ Tile tile;
  __shared__ alignas(16) float turned[2][16][kTileRows + 4];
  const int t = (int)threadIdx.x, tile_no = blockIdx.x / NR, j0 = 16 * (blockIdx.x - tile_no * NR);
  int count;
  const int adapter = open_tile(p.tiles, tile_no, tile, count);
  if (adapter == -2) return;
  const float scale = adapter >= 0 && p.scale ? p.scale[adapter] : 1.0f;
  {
    const int place = t >> 2, j = 4 * (t & 3), row = tile.row[place];
    float4_t g = {0.f, 0.f, 0.f, 0.f};
    float h[4] = {0.f, 0.f, 0.f, 0.f};
    if (row >= 0 && adapter >= 0) {
      if (p.g_out) {
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = j0 + j + e < p.rank ? p.hidden[(long)row * p.rank + j0 + j + e] : 0.0f;
      }
      g = scale * sum_parts(p.part + (long)row * RP + j0 + j, p.splits, (long)p.tiles.rows * RP);
#pragma unroll
      for (int e = 0; e < 4; ++e) g[e] = j0 + j + e < p.rank ? g[e] : 0.0f;
    }
    if (p.g && row >= 0) *reinterpret_cast<float4_t*>(p.g + (long)row * RP + j0 + j) = g;
#pragma unroll
    for (int e = 0; e < 4; ++e) turned[0][j + e][place] = g[e], turned[1][j + e][place] = h[e];
  }
  if (!p.g_out) return;
  __syncthreads();
  constexpr int PER = kTileRows / V;      // threads a rank
  for (int i = t; i < 2 * 16 * PER; i += 256) {
    const int which = i / (16 * PER), j = i / PER % 16, at = i % PER * V;
    const float* const from = &turned[which][j][at];
    void* const out = which ? p.hidden_out : p.g_out;
    const long place = (long)tile_no * kTileRows + at, to = (place / kStep<T> * RP + j0 + j) * kStep<T> + place % kStep<T>;
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<float4_t*>(static_cast<float*>(out) + to) = *reinterpret_cast<const float4_t*>(from);
    } else {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = from[e];
      uint4 q[N];
      parts_of<N>(v, q);
#pragma unroll
      for (int n = 0; n < N; ++n) *reinterpret_cast<uint4*>(static_cast<__bf16*>(out) + (long)n * RP * p.places + to) = q[n];
    }
  }
}

// ---- outer -----------------------------------------------------------------------

// V rows of V numbers, turned over: out[i] has number i of every row
template <typename T> __device__ __forceinline__ void turn(const uint4 (&r)[kV<T>], uint4 (&out)[kV<T>]) {
  if constexpr (sizeof(T) == 4) {
    out[0] = make_uint4(r[0].x, r[1].x, r[2].x, r[3].x);
    out[1] = make_uint4(r[0].y, r[1].y, r[2].y, r[3].y);
    out[2] = make_uint4(r[0].z, r[1].z, r[2].z, r[3].z);
    out[3] = make_uint4(r[0].w, r[1].w, r[2].w, r[3].w);
  } else {
    auto word = [](const uint4& v, int i) __attribute__((always_inline)) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; };
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      unsigned w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) w[q] = __builtin_amdgcn_perm(word(r[2 * q + 1], i / 2), word(r[2 * q], i / 2), i & 1 ? 0x07060302u : 0x05040100u);
      out[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

// A work-group has 16 V columns of a run of tiles with one adapter, all ranks; 128 rows of them at a time go through LDS, the next ones asked for meanwhile.  Its wavefronts
// share the ranks, 32 each, so that two fit a SIMD, and the rows where ranks are fewer.  ACROSS: ranks are the products' first operand, so that a lane's four results are ranks of
// one column and not columns of one rank.
// THIN: a side has fewer than V columns, read one by one.  Which columns a lane has: adapter_columns.hpp.
constexpr int kOuterRows = 128;
struct OuterShared {
  uint4 staged[2][kOuterRows][16 + 1];
};
template <typename T, int NR, bool ACROSS, bool THIN>
__device__ __forceinline__ void outer_side(const OuterArgs& p, const OuterSide& side, int group, int slice, OuterShared& shared) {
  constexpr int V = kV<T>, STEP = kStep<T>, RP = 16 * NR, N = sizeof(T) == 4 ? 1 : 3, NW = NR < 2 ? NR : 2, SHARES = NR / NW, STREAMS = 4 / SHARES, EACH = kOuterRows / 16;
  const int t = (int)threadIdx.x, lane = t & 63, wave = t >> 6, quarter = lane >> 4, lrow = lane & 15, share = wave % SHARES, stream = wave / SHARES;
  const OuterLane mine = outer_lane(side.c, V, group, t & 15);
  const T* const x = static_cast<const T*>(side.x) + mine.column;
  const long part = (long)RP * p.places;
  const int line = t >> 4, tiles = p.tile_at ? p.tile_at[p.tiles.adapters] : p.tile_count;
  // (no more slices than tiles, which rows without an adapter have none of: every slice has one, and leaves the sums that the join reads)
  const int slices = min(p.slices, tiles);
  if (slice >= slices) return;
  const int begin = (int)((long)slice * tiles / slices), slice_end = (int)((long)(slice + 1) * tiles / slices);
  // an adapter's places of the slice
  struct Run {
    int adapter, first, end, any_row;      // (a row to read in the place of none, kept out)
  };
  auto run_at = [&](int tile) __attribute__((always_inline)) {
    Run r;
    r.adapter = p.tile_at ? p.tiles.tile_of[tile] : 0;
    r.first = tile * kTileRows;
    r.end = (p.tile_at ? min(slice_end, p.tile_at[r.adapter + 1]) : slice_end) * kTileRows;
    r.any_row = p.tiles.order ? p.tiles.order[r.first] : r.first;
    return r;
  };
  auto find = [&](const Run& r, int at, int (&rows)[EACH]) __attribute__((always_inline)) {      // this thread's rows of those from place `at` on
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int place = at + 16 * e + line;
      rows[e] = place >= r.end ? -1 : p.tiles.order ? p.tiles.order[place] : place < p.tiles.rows ? place : -1;
    }
  };
  auto fetch = [&](const Run& r, const int (&rows)[EACH], uint4 (&v)[EACH]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const T* const from = x + (long)(rows[e] >= 0 ? rows[e] : r.any_row) * side.stride;
      v[e] = THIN ? load_some(from, mine.there) : load(from);
    }
  };
  auto stage = [&](int buffer, const int (&rows)[EACH], const uint4 (&v)[EACH]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < EACH; ++e) shared.staged[buffer][16 * e + line][t & 15] = keep(v[e], rows[e] >= 0);
  };
  // the other operand of the step at a place, a step ahead; (past the last one: the first again)
  auto operand = [&](const Run& r, int place, uint4 (&q)[NW][N]) __attribute__((always_inline)) {
    const long from = ((long)(place < r.end ? place : r.first) / STEP * RP + 16 * share * NW + lrow) * STEP + quarter * V;
#pragma unroll
    for (int n = 0; n < NW; ++n)
#pragma unroll
      for (int m = 0; m < N; ++m) {
        if constexpr (sizeof(T) == 4) q[n][m] = *reinterpret_cast<const uint4*>(static_cast<const float*>(side.parts) + from + 16 * STEP * n);
        else q[n][m] = *reinterpret_cast<const uint4*>(static_cast<const __bf16*>(side.parts) + m * part + from + 16 * STEP * n);
      }
  };
  Run run = run_at(begin);
  int rows[EACH], ahead[EACH];
  uint4 v[EACH], q[NW][N];
  find(run, run.first, rows);
  fetch(run, rows, v);
  operand(run, run.first + stream * STEP, q);
  find(run, run.first + kOuterRows, ahead);
#pragma unroll 1
  for (;;) {
    float4_t acc[V][NW];
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int n = 0; n < NW; ++n) acc[i][n] = (float4_t){0.f, 0.f, 0.f, 0.f};
    stage(0, rows, v);
    int buffer = 0;
#pragma unroll 1
    for (int at = run.first; at < run.end; at += kOuterRows, buffer ^= 1) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < EACH; ++e) rows[e] = ahead[e];
      fetch(run, rows, v);
      find(run, at + 2 * kOuterRows, ahead);
#pragma unroll 1
      for (int in = stream * STEP; in < kOuterRows && at + in < run.end; in += STREAMS * STEP) {
        uint4 next[NW][N], r[V], turned[V];
        operand(run, at + in + STREAMS * STEP, next);
#pragma unroll
        for (int e = 0; e < V; ++e) r[e] = shared.staged[buffer][in + quarter * V + e][lrow];
        turn<T>(r, turned);
        // (column by column, so that what an fp16 one is made into is used up before the next: rank by rank it spilled 74 registers; 8192 x 4096, rank 64: fp16 84 -> 71 us with five products, 76 with all six, bf16 49 -> 47 us.  bf16 still spills 2 registers at rank 64 and 1 at 128)
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
          for (int n = 0; n < NW; ++n) {
            if constexpr (sizeof(T) == 4) acc[i][n] = ACROSS ? mma<float>(q[n][0], turned[i], acc[i][n]) : mma<float>(turned[i], q[n][0], acc[i][n]);
            else acc[i][n] = mma_parts<T, N, ACROSS>(turned[i], q[n], acc[i][n]);
          }
#pragma unroll
        for (int n = 0; n < NW; ++n)
#pragma unroll
          for (int m = 0; m < N; ++m) q[n][m] = next[n][m];
      }
      stage(buffer ^ 1, rows, v);      // (read two steps ago)
    }
    // the next adapter's first rows are asked for before these sums are joined
    const int sum = slice + run.adapter, tile = run.end / kTileRows;
    if (tile < slice_end) {
      run = run_at(tile);
      find(run, run.first, rows);
      fetch(run, rows, v);
      operand(run, run.first + stream * STEP, q);
      find(run, run.first + kOuterRows, ahead);
    }
    // the wavefronts' sums joined through LDS, up to 8 results of each at a time
    float4_t* const joined = reinterpret_cast<float4_t*>(&shared);
    static_assert(sizeof(OuterShared) >= 8 * 4 * 64 * sizeof(float4_t), "the wavefronts' sums take the rows' place");
    float4_t* const sums = side.sums + ((long)sum * side.groups + group) * (V * NR * 64);
    constexpr int G = 8 / NW < V ? 8 / NW : V;
#pragma unroll
    for (int i0 = 0; i0 < V; i0 += G) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int n = 0; n < NW; ++n) joined[((i * NW + n) * 4 + wave) * 64 + lane] = acc[i0 + i][n];
      __syncthreads();
#pragma unroll
      for (int item = 0; item < G * NR; item += 4) {
        const int mine = item + wave, of = mine % SHARES, in = mine / SHARES, i = i0 + in / NW, n = of * NW + in % NW;
        if (mine >= G * NR) break;
        float4_t s = joined[(in * 4 + of) * 64 + lane];
#pragma unroll
        for (int w = 1; w < STREAMS; ++w) s += joined[(in * 4 + w * SHARES + of) * 64 + lane];
        sums[(i * NR + n) * 64 + lane] = s;
      }
    }
    if (tile >= slice_end) break;
    __syncthreads();
  }
}

template <typename T, int NR, bool THIN>
__global__ __launch_bounds__(256, kOuterWaves) void adapter_outer_kernel(const OuterArgs p) {
  __shared__ OuterShared shared;
  const int groups = p.side[0].groups + p.side[1].groups;
  const int slice = blockIdx.x / (unsigned)groups, group = blockIdx.x - slice * groups;
  if (group < p.side[0].groups) outer_side<T, NR, false, THIN>(p, p.side[0], group, slice, shared);
  else outer_side<T, NR, true, THIN>(p, p.side[1], group - p.side[0].groups, slice, shared);
}

template <typename T, int NR> void launch_ranks(AdapterPass pass, const void* args, const AdapterLaunch& l, hipStream_t s) {
  if (pass == kAdapterNarrow && l.few) adapter_narrow_kernel<T, NR, 1><<<l.grid, 256, 0, s>>>(*static_cast<const NarrowArgs*>(args));
  else if (pass == kAdapterNarrow) adapter_narrow_kernel<T, NR, 4><<<l.grid, 256, 0, s>>>(*static_cast<const NarrowArgs*>(args));
  else if (pass == kAdapterWiden && l.few) adapter_widen_kernel<T, NR, 1><<<l.grid, 256, 0, s>>>(*static_cast<const WidenArgs*>(args));
  else if (pass == kAdapterWiden) adapter_widen_kernel<T, NR, 4><<<l.grid, 256, 0, s>>>(*static_cast<const WidenArgs*>(args));
  else if (pass == kAdapterParts) adapter_parts_kernel<T, NR><<<l.grid, 256, 0, s>>>(*static_cast<const PartsArgs*>(args));
  else if (l.thin) adapter_outer_kernel<T, NR, true><<<l.grid, 256, 0, s>>>(*static_cast<const OuterArgs*>(args));
  else adapter_outer_kernel<T, NR, false><<<l.grid, 256, 0, s>>>(*static_cast<const OuterArgs*>(args));
}

}  // namespace adapter

template <typename T> void launch_adapter(AdapterPass pass, const void* args, const AdapterLaunch& l, hipStream_t s) {
  if (l.ranks == 1) adapter::launch_ranks<T, 1>(pass, args, l, s);
  else if (l.ranks == 2) adapter::launch_ranks<T, 2>(pass, args, l, s);
  else if (l.ranks == 4) adapter::launch_ranks<T, 4>(pass, args, l, s);
  else adapter::launch_ranks<T, 8>(pass, args, l, s);
}

}  // namespace cprune
