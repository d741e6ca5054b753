// Microscaled 4-bit numbers: quantisation, the way back, and products on the scaled matrix instruction.
#pragma once
#include <type_traits>

#include "conv_kernel.hpp"

namespace cprune {

struct Mx4Args {
  const unsigned char *a, *as;   // weights' codes and scales, [c_out][blocks * 16], [c_out][blocks]
  const unsigned char *b, *bs;   // the rows', [rows][blocks * 16], [rows][blocks]; or
  const void* x;                 // the rows as numbers, [rows][x_stride]
  long x_stride;
  int k;
  const float* bias;
  void* y;                       // [rows][c_out]
  int rows, c_out, blocks;
  float lo, hi;
  int tiles, row_tiles;          // tiles of c_out, of rows
  // tile kernel: both sides in operand order, zeros past the last row and block, from mx4_arrange_kernel
  const uint4 *ao, *bo;          // [tile][step, a multiple of four][16-row block of the tile][lane]
  const unsigned *aso, *bso;     // [tile][four steps][16-row block of the tile][lane], byte t the scale of step t
};

namespace mx4 {

typedef int int8v __attribute__((ext_vector_type(8)));

// The matrix instruction's operand: lane l holds row l % 16 and the 32 elements of block l / 16, in four registers; byte BYTE of `as` and `bs` is the
// block's scale.
template <int BYTE = 0> __device__ __forceinline__ float4_t mma(uint4 a, int as, uint4 b, int bs, float4_t acc) {
  const int8v av = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, bv = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv, acc, 4, 4, BYTE, as, BYTE, bs);
}

// The same for 32 x 32 results and 64 terms: lane l holds row l % 32 and block l / 32; result v of lane l is row 8 (v / 4) + 4 (l / 32) + v % 4, column l % 32.
typedef float float16v __attribute__((ext_vector_type(16)));
template <int BYTE> __device__ __forceinline__ float16v mma32(uint4 a, int as, uint4 b, int bs, float16v acc) {
  const int8v av = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, bv = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(av, bv, acc, 4, 4, BYTE, as, BYTE, bs);
}

template <bool SILU> __device__ __forceinline__ float finish(float z, float lo, float hi) {
  if constexpr (SILU) return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));      // (2^x flushes below 2^-126: 1 + e^-z does not see it)
  z = z < lo ? lo : z;      // (comparisons and not minimum / maximum: a NaN stays one)
  return z > hi ? hi : z;
}

__device__ __forceinline__ uint4 load16(__amdgpu_buffer_rsrc_t r, unsigned off) {
  typedef unsigned int uint32x4_t __attribute__((ext_vector_type(4)));
  const uint32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, 0);
  return make_uint4(v.x, v.y, v.z, v.w);
}

}  // namespace mx4

// ---- numbers to codes ------------------------------------------------------------------------------
namespace mx4 {

// Eight neighbouring numbers as they are in memory, zeros past the last.
template <typename X> struct Eight {
  typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
  unsigned w[4];
  __device__ __forceinline__ void load(const X* p, int valid) {
    typedef unsigned uint4u __attribute__((ext_vector_type(4), aligned(2)));
    if (valid >= 8) {
      const uint4u v = *reinterpret_cast<const uint4u*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = v[i];
    } else if (valid > 0) {      // (the last one again where there is none: loads that wait for nothing, a branch each would have them one by one)
      const unsigned short* h = reinterpret_cast<const unsigned short*>(p);
      unsigned short v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = h[min(i, valid - 1)];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (2 * i < valid ? (unsigned)v[2 * i] : 0u) | (2 * i + 1 < valid ? (unsigned)v[2 * i + 1] << 16 : 0u);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = 0;
    }
  }
  // largest magnitude, in a form that orders like it (as integers, magnitudes order like numbers, NaN above infinity)
  __device__ __forceinline__ unsigned top() const {
    ushort2v m = __builtin_bit_cast(ushort2v, w[0] & 0x7fff7fffu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(ushort2v, w[i] & 0x7fff7fffu));
    return max((unsigned)m[0], (unsigned)m[1]);
  }
  // the same as the bits of an fp32 number
  static __device__ __forceinline__ unsigned widen(unsigned top) {
    if constexpr (std::is_same<X, __bf16>::value) return top << 16;
    else return __float_as_uint((float)__builtin_bit_cast(_Float16, (unsigned short)top));
  }
  template <int I> __device__ __forceinline__ unsigned pair(unsigned c, float scale) const {
    if constexpr (std::is_same<X, __bf16>::value) {
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[I]), scale, I);
    } else {
      typedef _Float16 half2v __attribute__((ext_vector_type(2)));
      return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(half2v, w[I]), scale, I);
    }
  }
};
template <> struct Eight<float> {
  float v[8];
  __device__ __forceinline__ void load(const float* p, int valid) {
    typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));
    if (valid >= 8) {
      const float4u lo = *reinterpret_cast<const float4u*>(p), hi = *reinterpret_cast<const float4u*>(p + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = lo[i], v[4 + i] = hi[i];
    } else if (valid > 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = p[min(i, valid - 1)];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < valid ? v[i] : 0.0f;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    }
  }
  __device__ __forceinline__ unsigned top() const {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
  }
  static __device__ __forceinline__ unsigned widen(unsigned top) { return top; }
  template <int I> __device__ __forceinline__ unsigned pair(unsigned c, float scale) const {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2 * I], v[2 * I + 1], scale, I);
  }
};

// the scale's byte from the largest magnitude's bits
__device__ __forceinline__ int scale_byte(unsigned top) {
  const int e = (int)(top >> 23);
  return e == 255 ? 255 : max(e - 2, 0);
}
__device__ __forceinline__ float scale_value(int s) {      // 2^(s - 127), NaN for 255
  return __uint_as_float(s == 255 ? 0x7fc00000u : s == 0 ? 0x00400000u : (unsigned)s << 23);
}
// eight codes; the instruction divides by the scale, rounds half to even and stops at 6
template <typename X> __device__ __forceinline__ unsigned codes_of(const Eight<X>& e, int s) {
  const float f = scale_value(s);
  unsigned c = 0;
  c = e.template pair<0>(c, f);
  c = e.template pair<1>(c, f);
  c = e.template pair<2>(c, f);
  c = e.template pair<3>(c, f);
  return s == 255 ? 0u : c;
}

// A block of 32 by one lane: the matrix instruction's operand and its scale.
template <typename X> struct Block {
  Eight<X> e[4];
  __device__ __forceinline__ void load(const X* p, int valid) {
    if (valid >= 32) {
#pragma unroll
      for (int i = 0; i < 4; ++i) e[i].load(p + 8 * i, 8);
    } else if (valid > 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) e[i].load(p + 8 * i, valid - 8 * i);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) e[i] = Eight<X>();
    }
  }
  __device__ __forceinline__ void quantize(uint4& codes, int& scale) const {
    scale = scale_byte(Eight<X>::widen(max(max(e[0].top(), e[1].top()), max(e[2].top(), e[3].top()))));
    codes = make_uint4(codes_of(e[0], scale), codes_of(e[1], scale), codes_of(e[2], scale), codes_of(e[3], scale));
  }
};

// The rows' side of a product: numbers of X, or codes (X = void).  Held: a lane's block on its way.
template <typename X> struct Rows {
  struct Held {
    Block<X> b;
    __device__ __forceinline__ void operand(uint4& codes, int& scale) const { b.quantize(codes, scale); }
  };
  const X* x;
  long stride;
  int rows, k;
  __device__ __forceinline__ explicit Rows(const Mx4Args& p) : x(static_cast<const X*>(p.x)), stride(p.x_stride), rows(p.rows), k(p.k) {}
  __device__ __forceinline__ void load(Held& h, int r, int blk) const { h.b.load(x + min(r, rows - 1) * stride + blk * 32l, r < rows ? k - blk * 32 : 0); }
};
template <> struct Rows<void> {
  struct Held {
    uint4 c;
    int s;
    __device__ __forceinline__ void operand(uint4& codes, int& scale) const { codes = c, scale = s; }
  };
  __amdgpu_buffer_rsrc_t codes_at, scales_at;
  int rows, blocks;
  __device__ __forceinline__ explicit Rows(const Mx4Args& p)
      : codes_at(make_rsrc(p.b, (unsigned)p.rows * p.blocks * 16u)), scales_at(make_rsrc(p.bs, (unsigned)p.rows * p.blocks)), rows(p.rows), blocks(p.blocks) {}
  __device__ __forceinline__ void load(Held& h, int r, int blk) const {
    const bool in = r < rows && blk < blocks;
    const unsigned at = (unsigned)r * blocks + blk;
    h.c = load16(codes_at, in ? at * 16 : kOutOfRange);
    h.s = (int)__builtin_amdgcn_raw_buffer_load_b8(scales_at, in ? (int)at : (int)kOutOfRange, 0, 0);      // (0 out of range: as good a scale as any for zeros)
  }
};

// The weights' operands: rows o of 16, straight from memory.
struct Weights {
  __amdgpu_buffer_rsrc_t codes_at, scales_at;
  int c_out, blocks;
  __device__ __forceinline__ explicit Weights(const Mx4Args& p)
      : codes_at(make_rsrc(p.a, (unsigned)p.c_out * p.blocks * 16u)), scales_at(make_rsrc(p.as, (unsigned)p.c_out * p.blocks)), c_out(p.c_out), blocks(p.blocks) {}
  __device__ __forceinline__ void load(int o, int blk, uint4& c, int& s) const {
    const bool in = o < c_out && blk < blocks;
    const unsigned at = (unsigned)o * blocks + blk;
    c = load16(codes_at, in ? at * 16 : kOutOfRange);
    s = (int)__builtin_amdgcn_raw_buffer_load_b8(scales_at, in ? (int)at : (int)kOutOfRange, 0, 0);
  }
};

// The first of the four outputs, counted from the tile's, that block i of MB and lane group g (of four) work out: the groups' 16-byte pieces of a row lie side by
// side, so that a store covers 64 bytes of it (200704 x 24 x 144 bf16 24.0 -> 22.4 us, 11910 x 23 x 1630 18.6 -> 16.5, against a lane with its outputs in one run).
template <typename T, int MB> __device__ __forceinline__ int output_of(int i, int g) {
  constexpr int P = MB > 1 && sizeof(T) == 2 ? 2 : 1;      // blocks of a piece
  return 16 * P * (i / P) + 4 * P * g + 4 * (i % P);
}
// The outputs of lane group g from the sums of MB blocks; o is the tile's first.
template <typename T, bool SILU, int MB> __device__ __forceinline__ void store_outputs(const Mx4Args& p, const float4_t (&v)[MB], const float4_t (&bias)[MB], int r, int o, int g) {
  if (r >= p.rows) return;
  constexpr int P = MB > 1 && sizeof(T) == 2 ? 2 : 1, W = 4 * P;      // numbers of a piece
  T* y = static_cast<T*>(p.y) + (long)r * p.c_out + o;
  typedef T outs __attribute__((ext_vector_type(W), aligned(sizeof(T))));
#pragma unroll
  for (int h = 0; h < MB; h += P) {
    outs q;
#pragma unroll
    for (int e = 0; e < W; ++e) q[e] = Elem<T>::from_f32(finish<SILU>(v[h + e / 4][e & 3] + bias[h + e / 4][e & 3], p.lo, p.hi));
    const int at = output_of<T, MB>(h, g);
    if (o + at + W <= p.c_out) {
      *reinterpret_cast<outs*>(y + at) = q;
    } else {
#pragma unroll
      for (int e = 0; e < W; ++e)
        if (o + at + e < p.c_out) y[at + e] = q[e];
    }
  }
}

}  // namespace mx4

// ---- few rows: the wavefronts of a work-group share the sum ------------------------------------------
// 16 MB outputs by 16 NB rows a work-group; wavefront w takes steps w, w + WAVES, ... of 128 terms, both operands straight from memory (each weight is read
// once, by one wavefront), the rows' numbers made codes by the lane that multiplies them.  The sums are joined through LDS in a fixed order.  Bound by the chain of
// one or two loads a wavefront, codes, product and joining: 1 x 4096 x 4096 bf16, 9 MB, 6.2 us from memory, 4.7 from the caches.
template <typename X, typename T, bool SILU, int MB, int NB, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void mx4_few_kernel(const Mx4Args p) {
  using namespace mx4;
  constexpr int U = 2;      // steps under way
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lrow = lane & 15, lblk = lane >> 4;
  const int tr = blockIdx.x / (unsigned)p.tiles, o0 = ((int)blockIdx.x - tr * p.tiles) * 16 * MB, r0 = tr * 16 * NB;
  const Weights w(p);
  const Rows<X> x(p);
  float4_t acc[NB][MB];
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int i = 0; i < MB; ++i) acc[j][i] = (float4_t){0.f, 0.f, 0.f, 0.f};
  const int steps = (p.blocks + 3) / 4;
  for (int st = wave; st < steps; st += U * WAVES) {
    uint4 a[U][MB];
    int as[U][MB];
    typename Rows<X>::Held rows[U][NB];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int blk = (st + u * WAVES) * 4 + lblk;      // (past the last one: zeros)
#pragma unroll
      for (int i = 0; i < MB; ++i) w.load(o0 + output_of<T, MB>(i, lrow >> 2) + (lrow & 3), blk, a[u][i], as[u][i]);
#pragma unroll
      for (int j = 0; j < NB; ++j) x.load(rows[u][j], r0 + 16 * j + lrow, blk);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        uint4 b;
        int bs;
        rows[u][j].operand(b, bs);
#pragma unroll
        for (int i = 0; i < MB; ++i) acc[j][i] = mma(a[u][i], as[u][i], b, bs, acc[j][i]);
      }
  }
  __shared__ float4_t sums[WAVES - 1][MB * NB][64];
  if (wave > 0) {
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int i = 0; i < MB; ++i) sums[wave - 1][j * MB + i][lane] = acc[j][i];
  }
  __syncthreads();
  if (wave > 0) return;
  float4_t bias[MB];
#pragma unroll
  for (int i = 0; i < MB; ++i) bias[i] = load_bias4(p.bias, p.c_out, o0 + output_of<T, MB>(i, lblk));
#pragma unroll
  for (int j = 0; j < NB; ++j) {
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int q = 0; q < WAVES - 1; ++q) acc[j][i] += sums[q][j * MB + i][lane];
    store_outputs<T, SILU, MB>(p, acc[j], bias, r0 + 16 * j + lrow, o0, lblk);
  }
}

// ---- many rows of short sums: the rows stay in registers ----------------------------------------------
// A wavefront holds the codes of 16 NB rows, all of their at most 128 STEPS terms, and goes over all outputs; the weights come from the caches, where the
// four wavefronts of a work-group read the same ones at about the same time.  x is read once and y written once: 200704 x 144 x 24-term sums, 67 MB, 22.4 us, bound by
// the stores; 12544 x 576 x 96 from codes 7.8 us, by its chain of dependent loads.
template <typename X, typename T, bool SILU, int MB, int NB, int STEPS>
__global__ __launch_bounds__(256) void mx4_rows_kernel(const Mx4Args p) {
  using namespace mx4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lrow = lane & 15, lblk = lane >> 4;
  const int r0 = ((int)blockIdx.x * 4 + wave) * 16 * NB;
  if (r0 >= p.rows) return;
  const Weights w(p);
  const Rows<X> x(p);
  uint4 b[NB][STEPS];
  int bs[NB][STEPS];
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    typename Rows<X>::Held rows[STEPS];
#pragma unroll
    for (int st = 0; st < STEPS; ++st) x.load(rows[st], r0 + 16 * j + lrow, st * 4 + lblk);
#pragma unroll
    for (int st = 0; st < STEPS; ++st) rows[st].operand(b[j][st], bs[j][st]);
  }
  for (int o0 = (int)blockIdx.y * 16 * MB; o0 < p.c_out; o0 += (int)gridDim.y * 16 * MB) {
      float4_t bias[MB], acc[NB][MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) bias[i] = load_bias4(p.bias, p.c_out, o0 + output_of<T, MB>(i, lblk));
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int i = 0; i < MB; ++i) acc[j][i] = (float4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      uint4 a[MB];
      int as[MB];
#pragma unroll
      for (int i = 0; i < MB; ++i) w.load(o0 + output_of<T, MB>(i, lrow >> 2) + (lrow & 3), st * 4 + lblk, a[i], as[i]);
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int i = 0; i < MB; ++i) acc[j][i] = mma(a[i], as[i], b[j][st], bs[j][st], acc[j][i]);
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) store_outputs<T, SILU, MB>(p, acc[j], bias, r0 + 16 * j + lrow, o0, lblk);
  }
}

// ---- many rows: tiles through LDS -----------------------------------------------------------------
// Four wavefronts (2 x 2) of MI x MI blocks each: 32 MI outputs of c_out by 32 MI rows a work-group, K in steps of 128 terms.  A stage is the tile's codes
// of one step in operand order, [16-row block][lane][16 bytes], as a launch before has laid them out in memory: a step of a tile is one run of memory, so its
// loads spread over all channels of the L2 (rows of 2^n bytes read side by side would meet in one), and they write to LDS themselves.
// While step s is multiplied, the operands of s + 1 go to registers and the codes of s + STAGES into the stage that s has left.
// 16384 x 8192 x 8192 from operands in place: 504 to 525 us, 4.2 to 4.4 PFLOP/s, tiles of 256.  The matrix pipes are busy 58 % of the clocks, and the clock itself is down: the same
// instructions on codes that are all zero take a fifth less.  The rest is a tile's first loads and last stores, some 14 us of 65 a round.
// The matrix instruction takes 32 rows of each side; those of a wavefront's c_out are dealt so that a lane's results are 8 MI neighbours of one row of y.
namespace mx4 {

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

// row of c_out, counted from the 16 MI outputs it belongs to, that is row m of 16-row block i: of the instruction's rows 8 q + 4 g + e, g picks the half
template <int MI> __device__ __forceinline__ int spread_row(int i, int m) {
  const int r = (i & 1) * 16 + m;
  return 8 * MI * ((r >> 2) & 1) + 16 * (i >> 1) + 4 * (r >> 3) + (r & 3);
}

// Waits until all but the last `newer` loads and all LDS accesses of this wavefront are done, then for the others.
template <int NEWER> __device__ __forceinline__ void wait_and_meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);      // (nor do products drift past it: their operands would be held for another step)
  __builtin_amdgcn_s_waitcnt((NEWER & 15) | (7 << 4) | ((NEWER >> 4) << 14));
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}

// The tile of a work-group: neighbouring work-groups run on different XCDs, each with an L2 of its own, so each XCD gets a run of tiles, and a run walks
// eight tiles of rows before the next tile of c_out.
__device__ __forceinline__ void tile_of(const Mx4Args& p, int& tr, int& tc) {
  const unsigned total = gridDim.x, xcd = blockIdx.x & 7, per = total >> 3, rest = total & 7;
  const unsigned t = xcd * per + min(xcd, rest) + (blockIdx.x >> 3);
  const unsigned group = t / (8u * p.tiles), local = t - group * 8u * p.tiles;
  const unsigned wide = min(8u, (unsigned)p.row_tiles - group * 8u);
  tc = (int)(local / wide);
  tr = (int)(group * 8u + (local - (unsigned)tc * wide));
}

}  // namespace mx4

template <typename T, bool SILU, int MI, int STAGES>
__global__ __launch_bounds__(256) void mx4_tile_kernel(const Mx4Args p) {
  using namespace mx4;
  constexpr int NI = MI, AB = 2 * MI;               // 16-row blocks of a side of the tile
  constexpr int LOADS = AB / 2;                     // of which a wavefront loads these a step
  constexpr int CHUNKS = AB / 4;                    // of four blocks each, whose scales of four steps are one load
  // (arrays of their own: an index into one would have every read wait for every load on its way)
  __shared__ uint4 st0[2 * AB * 64], st1[2 * AB * 64], st2[2 * AB * 64], st3[STAGES > 3 ? 2 * AB * 64 : 1];
  __shared__ unsigned sc0[2 * AB * 64];      // [16-row block][lane]: the scales of four steps
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), lrow = lane & 15;
  const int wm = wave & 1, wn = wave >> 1;
  int tr, tc;
  tile_of(p, tr, tc);
  const int o0 = tc * 16 * AB, r0 = tr * 16 * AB;
  const int steps = (p.blocks + 3) / 4, fours = (steps + 3) / 4;

  // Wavefronts 0 and 1 load the weights, 2 and 3 the rows.  Steps past the last one read that one again.
  const int half = wave & 1;
  const uint4* const from = (wave < 2 ? p.ao + (size_t)tc * fours * 4 * AB * 64 : p.bo + (size_t)tr * fours * 4 * AB * 64) + half * LOADS * 64;
  const unsigned* const scales_from = wave < 2 ? p.aso + (size_t)tc * fours * AB * 64 : p.bso + (size_t)tr * fours * AB * 64;
  auto fetch = [&](uint4* stage, int s) __attribute__((always_inline)) {
    const uint4* const at = from + (size_t)min(s, 4 * fours - 1) * (AB * 64);
#pragma unroll
    for (int q = 0; q < LOADS; ++q)
      __builtin_amdgcn_global_load_lds((global_void*)(at + q * 64 + lane), (lds_void*)(stage + (wave * LOADS + q) * 64), 16, 0, 0);
  };
  auto fetch_scales = [&](unsigned* sc, int four) __attribute__((always_inline)) {
    const unsigned* const at = scales_from + (size_t)min(four, fours - 1) * (AB * 64);
    constexpr int EACH = (CHUNKS + 1) / 2;
#pragma unroll
    for (int q = 0; q < EACH; ++q) {
      const int c = half * EACH + q;
      if (c < CHUNKS)
        __builtin_amdgcn_global_load_lds((global_void*)(at + c * 256 + lane * 4), (lds_void*)(sc + ((wave >> 1) * CHUNKS + c) * 256), 16, 0, 0);
    }
  };

  constexpr int M = MI / 2, N = NI / 2;      // 32 x 32 results of a wavefront
  float16v acc[M][N];
#pragma unroll
  for (int i = 0; i < M; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  // operands and scales of a step's two halves
  uint4 fa[2][2][M], fb[2][2][N];
  int sa[2][M], sb[2][N];
  const int at0 = ((lane >> 4) & 1) * 64 + (lane >> 5) * 16 + lrow;      // a lane's place in two 16-row blocks, of the first half
  auto operands = [&](const uint4* stage, uint4 (&a)[2][M], uint4 (&b)[2][N]) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < M; ++i) a[h][i] = stage[(wm * MI + 2 * i) * 64 + h * 32 + at0];
#pragma unroll
      for (int j = 0; j < N; ++j) b[h][j] = stage[(AB + wn * NI + 2 * j) * 64 + h * 32 + at0];
    }
  };
  auto scales = [&](const unsigned* sc) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < M; ++i) sa[h][i] = (int)sc[(wm * MI + 2 * i) * 64 + h * 32 + at0];
#pragma unroll
      for (int j = 0; j < N; ++j) sb[h][j] = (int)sc[(AB + wn * NI + 2 * j) * 64 + h * 32 + at0];
    }
  };

  fetch_scales(sc0, 0);
  fetch(st0, 0);
  fetch(st1, 1);
  fetch(st2, 2);
  if constexpr (STAGES > 3) fetch(st3, 3);
  wait_and_meet<(STAGES - 1) * LOADS>();
  operands(st0, fa[0], fb[0]);
  scales(sc0);
  // Step s: its operands are in fa[B & 1], fb[B & 1], its scales byte B of sa and sb.  sc_own: the scales of this step's four, whose place is free while they
  // are multiplied; sc_next: those of the next.
  auto step = [&](auto byte, int s, uint4* own, uint4* next) __attribute__((always_inline)) {
    constexpr int B = decltype(byte)::value;
    wait_and_meet<(STAGES - 2) * LOADS>();      // the codes of s + 1 are there (later ones may be under way), and nobody reads `own` any more
    if (B == 0) fetch_scales(sc0, s / 4 + 1);      // (ahead of the codes of s + STAGES: there when those are, a step before they are read)
    fetch(own, s + STAGES);
    operands(next, fa[(B + 1) & 1], fb[(B + 1) & 1]);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < N; ++j)
#pragma unroll
        for (int i = 0; i < M; ++i) acc[i][j] = mma32<B>(fa[B & 1][h][i], sa[h][i], fb[B & 1][h][j], sb[h][j], acc[i][j]);
    // an LDS read, a load and some products in turn
#pragma unroll
    for (int q = 0; q < 2 * (M + N); ++q) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      if (q < LOADS) __builtin_amdgcn_sched_group_barrier(0x20, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x8, M * N > M + N ? M * N / (M + N) : 1, 0);
    }
    if (B == 3) scales(sc0);
    asm volatile("" ::: "memory");      // (the reads above belong to this turn of the loop)
  };
  typedef std::integral_constant<int, 0> byte0;
  typedef std::integral_constant<int, 1> byte1;
  typedef std::integral_constant<int, 2> byte2;
  typedef std::integral_constant<int, 3> byte3;
  if constexpr (STAGES == 4) {
    // (One way out of the loop where the sums fill half the registers: with an exit behind each step they are copied at every turn.  The steps that fill up
    // the last four multiply zeros.)
    for (int s = 0;; s += 4) {
      step(byte0(), s, st0, st1);
      step(byte1(), s + 1, st1, st2);
      step(byte2(), s + 2, st2, st3);
      step(byte3(), s + 3, st3, st0);
      if (s + 4 >= steps) break;
    }
  } else {
    for (int s = 0;; s += 12) {
      step(byte0(), s, st0, st1);
      step(byte1(), s + 1, st1, st2);
      step(byte2(), s + 2, st2, st0);
      step(byte3(), s + 3, st0, st1);
      if (s + 4 >= steps) break;
      step(byte0(), s + 4, st1, st2);
      step(byte1(), s + 5, st2, st0);
      step(byte2(), s + 6, st0, st1);
      step(byte3(), s + 7, st1, st2);
      if (s + 8 >= steps) break;
      step(byte0(), s + 8, st2, st0);
      step(byte1(), s + 9, st0, st1);
      step(byte2(), s + 10, st1, st2);
      step(byte3(), s + 11, st2, st0);
      if (s + 12 >= steps) break;
    }
  }

  // A lane has 8 MI neighbouring outputs of a row.  They go through LDS, each wavefront's own stage, so that a store covers whole runs of a row: straight
  // from the registers every lane would write 8 bytes of another row.  16-byte pieces are moved by their row (exclusive or): neither side meets in a bank.
  if constexpr (MI == 8) {
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) asm volatile("" : "+a"(acc[i][j]));      // (the sums leave the loop where they were in it)
  }
  wait_and_meet<0>();
  constexpr int W = 16 / (int)sizeof(T);                    // numbers of a piece
  constexpr int PIECES = 16 * MI / W;                       // of a row of the wavefront's outputs
  constexpr int ROOM = STAGES == 4 ? 2 * AB * 64 : AB * 64;
  constexpr int J = N * 32 * PIECES > ROOM ? N / 2 : N;      // 32-row blocks that fit
  uint4* const mine = STAGES == 4 ? (wave == 0 ? st0 : wave == 1 ? st1 : wave == 2 ? st2 : st3) : (wave < 2 ? st0 : st1) + (wave & 1) * ROOM;
  int l = threadIdx.x & 63;
  asm volatile("" : "+v"(l));      // (what follows from it is worked out here and not held through the loop, where there is no register for it)
  const int o = o0 + wm * 16 * MI, row = l & 31, first = (l >> 5) * (8 * MI / W);
  typedef T outs __attribute__((ext_vector_type(W), aligned(sizeof(T))));
#pragma unroll
  for (int j0 = 0; j0 < N; j0 += J) {
#pragma unroll
    for (int i = 0; i < M; ++i) {
      float4_t bias[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) bias[q] = load_bias4(p.bias, p.c_out, o + 8 * MI * (l >> 5) + 16 * i + 4 * q);
#pragma unroll
      for (int j = j0; j < j0 + J; ++j)
#pragma unroll
        for (int h = 0; h < 16; h += W) {
          outs z;
#pragma unroll
          for (int e = 0; e < W; ++e) z[e] = Elem<T>::from_f32(finish<SILU>(acc[i][j][h + e] + bias[(h + e) / 4][(h + e) & 3], p.lo, p.hi));
          const int piece = first + (16 * i + h) / W;
          mine[((j - j0) * 32 + row) * PIECES + (piece ^ (row & (PIECES - 1)))] = __builtin_bit_cast(uint4, z);
          __builtin_amdgcn_sched_barrier(0);      // (one piece after another: all sums at once are more than the registers)
        }
    }
    __builtin_amdgcn_wave_barrier();
    constexpr int AT_ONCE = 64 / PIECES;                    // rows of a store
#pragma unroll 4
    for (int it = 0; it < J * 32 / AT_ONCE; ++it) {
      const int at = it * AT_ONCE + l / PIECES, piece = l % PIECES;
      const outs z = __builtin_bit_cast(outs, mine[at * PIECES + (piece ^ (at & 31 & (PIECES - 1)))]);
      const int r = r0 + (wn * N + j0) * 32 + at, col = o + piece * W;
      if (r >= p.rows) continue;
      T* y = static_cast<T*>(p.y) + (long)r * p.c_out + col;
      if (col + W <= p.c_out) {
        *reinterpret_cast<outs*>(y) = z;
      } else {
#pragma unroll
        for (int e = 0; e < W; ++e)
          if (col + e < p.c_out) y[e] = z[e];
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

}  // namespace cprune
