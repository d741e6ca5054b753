// Entry points of the microscaled 4-bit numbers; quantisation and the way back (mx4_kernel.hpp has the products).
#include <algorithm>
#include <limits>

#include "mx4_kernel.hpp"

namespace cprune {
namespace {

constexpr int kQuad = 256;      // threads; eight numbers each, four threads a block of 32

// largest of an integer over the four lanes of a quad
__device__ __forceinline__ unsigned quad_max(unsigned v) {
  v = max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));
  return max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));
}

// Codes and scale of eight numbers at p, of which `valid` are there; the four lanes of a quad hold a block.
template <typename T> __device__ __forceinline__ unsigned quantize8(const T* p, int valid, int& s) {
  mx4::Eight<T> e;
  e.load(p, valid);
  s = mx4::scale_byte(mx4::Eight<T>::widen(quad_max(e.top())));
  return mx4::codes_of(e, s);
}

// A thread has eight numbers, so that a row's blocks are read and written in runs, whatever its length: bound by memory, 200704 x 144 bf16, 75 MB, 13.1 us, 5.7 TB/s.
template <typename T>
__global__ __launch_bounds__(kQuad) void mx4_quantize_kernel(const T* __restrict__ x, int rows, int k, long x_stride, int blocks,
                                                             unsigned* __restrict__ codes, unsigned char* __restrict__ scales) {
  const unsigned i = blockIdx.x * (unsigned)kQuad + threadIdx.x, per = 4u * blocks;
  if (i >= (unsigned)rows * per) return;      // (whole quads)
  const unsigned row = i / per, at = (i - row * per) * 8;
  int s;
  codes[i] = quantize8(x + row * x_stride + at, k - (int)at, s);
  if ((threadIdx.x & 3) == 0) scales[i >> 2] = (unsigned char)s;
}

// What the tile kernel reads: a work-group lays out 16 rows x 512 terms of a side, the rows' first, then the weights'.  A wavefront takes every fourth block of
// a row, a quad of lanes one block, four loads each at a time.  Rows of numbers become codes on the way.  16384 x 8192 bf16 beside 8192 x 8192 codes: 411 MB, 91 us,
// 4.5 TB/s.
struct Mx4Arrange {
  const void* x;                     // numbers, or codes
  const unsigned char *xs, *w, *ws;  // scales of codes; the weights' codes and scales
  long x_stride;
  int rows, k, c_out, blocks, mi;    // mi: blocks of a wavefront of the tile kernel on a side
  int row_groups;
  unsigned *x_codes, *x_scales, *w_codes, *w_scales;
};

template <typename T> __global__ __launch_bounds__(256) void mx4_arrange_kernel(const Mx4Arrange p) {
  const int fours = (p.blocks + 15) / 16, ab = 2 * p.mi;
  const bool weights = (int)blockIdx.x >= p.row_groups;
  const unsigned group = blockIdx.x - (weights ? p.row_groups : 0);
  const int b = group / (unsigned)fours, four = (int)group - b * fours;      // 16-row block, four steps
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, lrow = lane >> 2, quarter = lane & 3;
  int row = b * 16 + lrow;
  if (weights) row = b / p.mi * 16 * p.mi + (p.mi == 8 ? mx4::spread_row<8>(b % 8, lrow) : p.mi == 4 ? mx4::spread_row<4>(b % 4, lrow) : mx4::spread_row<2>(b % 2, lrow));
  const bool from_codes = weights || std::is_same<T, void>::value;
  const unsigned* const codes_in = static_cast<const unsigned*>(weights ? static_cast<const void*>(p.w) : p.x);
  const unsigned char* const scales_in = weights ? p.ws : p.xs;
  const int rows = weights ? p.c_out : p.rows;
  const int tile = b / ab, in_tile = b - tile * ab;
  unsigned* const codes = (weights ? p.w_codes : p.x_codes) + ((long)(tile * fours + four) * 4 * ab + in_tile) * 256 + (wave * 16 + lrow) * 4 + quarter;
  unsigned scales = 0;
  auto keep = [&](int t, unsigned c, int s) __attribute__((always_inline)) {
    codes[(long)t * ab * 256] = c;
    scales |= (unsigned)s << (8 * t);
  };
  if (from_codes) {
    unsigned c[4];
    int s[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int blk = (four * 4 + t) * 4 + wave;
      const bool in = row < rows && blk < p.blocks;
      const long at = (long)row * p.blocks + blk;
      c[t] = in ? codes_in[at * 4 + quarter] : 0u;
      s[t] = in ? scales_in[at] : 0;
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) keep(t, c[t], s[t]);
  } else if constexpr (!std::is_same<T, void>::value) {
    mx4::Eight<T> e[4];
    const T* const from = static_cast<const T*>(p.x) + min(row, p.rows - 1) * p.x_stride;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int at = ((four * 4 + t) * 4 + wave) * 32 + quarter * 8;
      e[t].load(from + at, row < p.rows ? p.k - at : 0);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int s = mx4::scale_byte(mx4::Eight<T>::widen(quad_max(e[t].top())));
      keep(t, mx4::codes_of(e[t], s), s);
    }
  }
  if (quarter == 0) (weights ? p.w_scales : p.x_scales)[((long)(tile * fours + four) * ab + in_tile) * 64 + wave * 16 + lrow] = scales;
}

// The same way back: 12.4 us, 6.0 TB/s.
template <typename T>
__global__ __launch_bounds__(kQuad) void mx4_dequantize_kernel(const unsigned* __restrict__ codes, const unsigned char* __restrict__ scales,
                                                               int rows, int k, int blocks, T* __restrict__ y) {
  const unsigned i = blockIdx.x * (unsigned)kQuad + threadIdx.x, per = 4u * blocks;
  if (i >= (unsigned)rows * per) return;
  const unsigned row = i / per, at = (i - row * per) * 8;
  const int valid = k - (int)at;
  if (valid <= 0) return;
  const unsigned c = codes[i];
  const float f = mx4::scale_value(scales[i >> 2]);
  typedef float float2v __attribute__((ext_vector_type(2)));
  // (exact: a code's value times a power of two; the product and not the instruction's own scale, whose NaN and 2^-127 it need not know)
  const float2v q[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3)};
  constexpr int V = 16 / (int)sizeof(T);
  typedef T outs __attribute__((ext_vector_type(V), aligned(sizeof(T))));
  T* p = y + (long)row * k + at;
#pragma unroll
  for (int h = 0; h < 8; h += V) {
    outs v;
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = Elem<T>::from_f32(q[(h + j) / 2][j & 1] * f);
    if (valid - h >= V) {
      *reinterpret_cast<outs*>(p + h) = v;
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (h + j < valid) p[h + j] = v[j];
    }
  }
}

bool act_of_product(int act) { return act_ok(act) || act == CPRUNE_ACT_SILU; }
int blocks_of(int k) { return (k + 31) / 32; }
// (with the zeros that fill up a row's last block counted)
bool too_many(int rows, int k) { return (double)rows * blocks_of(k) * 32.0 >= 2147483648.0; }

int check_numbers(int rows, int k, int x_stride, int dtype) {
  if (rows < 1 || k < 1 || k > 0x7fffffff - 31 || x_stride < k || !dtype_ok(dtype)) return CPRUNE_ERR_INVALID_ARG;
  return too_many(rows, k) || (double)rows * x_stride >= 2147483648.0 ? CPRUNE_ERR_INVALID_ARG : CPRUNE_OK;
}

template <typename F> void with_type(int dtype, F&& f) {
  if (dtype == CPRUNE_F32) f(float());
  else if (dtype == CPRUNE_F16) f(_Float16());
  else f(__bf16());
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

void launch_quantize(const void* x, int rows, int k, int x_stride, int dtype, void* codes, void* scales, hipStream_t s) {
  const int blocks = blocks_of(k);
  const unsigned grid = (unsigned)(((long)rows * blocks * 4 + kQuad - 1) / kQuad);
  with_type(dtype, [&](auto t) {
    using T = decltype(t);
    mx4_quantize_kernel<T><<<grid, kQuad, 0, s>>>(static_cast<const T*>(x), rows, k, x_stride, blocks, static_cast<unsigned*>(codes),
                                                  static_cast<unsigned char*>(scales));
  });
}

constexpr int kShortSteps = 5;      // steps of 128 terms that the rows kernel is built for

// How a product runs, and its scratch.
enum ProductForm { kFew, kShort, kTiles };
struct ProductPlan {
  ProductForm form;
  int mi;                            // kTiles: 16-row blocks a wavefront has on a side
  bool codes_first;                  // the rows' codes are made by a launch of their own, row by row
  size_t codes, x_scales, w_codes, w_scales;  // bytes
  size_t total() const { return codes + x_scales + w_codes + w_scales; }
};

// dtype: of the rows' numbers, -1 for codes
ProductPlan plan_product(int rows, int k, int c_out, int dtype) {
  const long blocks = blocks_of(k), steps = (blocks + 3) / 4, fours = (steps + 3) / 4;
  ProductPlan q = {};
  // Measured on bf16 numbers, us (short / few / tiles): 12544 x 200 x 64 4.0 / 7.9 / 8.2; 784 x 160 x 960 4.0 / 6.9 / 6.2; 3136 x 576 x 96 7.1 / 7.6 / 7.7; 3136 x 128 x
  // 2048 9.2 / 25 / 11.9; but many weights read by every 16 rows 12544 x 512 x 512 38 / 43 / 15, and six to eight steps 500 x 1000 x 100 12.6 / 9.1 / 6.6.  (784 x 512 x
  // 512 8.5 / 7.4 / 5.9: short all the same, its one launch and no scratch are less than the host needs for two.)
  const double work = (double)rows * c_out * k;
  const bool is_short = (steps <= kShortSteps && ((double)c_out * k <= 65536.0 || work <= 268435456.0)) || (steps <= 2 && work <= 1073741824.0);
  // The tiles' launch that lays both sides out reads and writes all weights, us (few / tiles): 40 x 2048 x 8192 10.0 / 13.9, 64 x 4096 x 4096 16.8 / 16.0,
  // 256 x 4096 x 4096 27.4 / 16.2, 64 x 1024 x 256 8.9 / 6.2.
  const bool enough = rows > 64 || (rows > 32 && (double)c_out * k <= 1048576.0);
  if (rows > 32 && is_short) {
    q.form = kShort;
  } else if (enough && (double)(rows + 255) * fours * 512 < 2147483648.0 && (double)(c_out + 255) * fours * 512 < 2147483648.0) {
    q.form = kTiles;
    // Tiles of 128, of which two or three work-groups share a compute unit, one's first loads and last stores beside another's products; of 64 where that leaves
    // less than half of the compute units one (1024 x 8192 x 1024 22.2 by 64, 24.7 by 128; 2048 x 2048 x 2048 17.3 and 16.0); of 256, alone on a compute unit
    // but with half the bytes through the caches, for many tiles of long sums (us by 256 / by 128: 16384 x 8192 x 8192 549 / 609, 8192 x 4096 x 8192 167 / 174,
    // but 16384 x 2048 x 8192 209 / 194, 16384 x 8192 x 2100 212 / 198).
    auto tiles_of = [&](long side) { return ((rows + side - 1) / side) * ((c_out + side - 1) / side); };
    q.mi = steps >= 32 && tiles_of(256) >= 1024 ? 8 : tiles_of(128) >= 128 ? 4 : 2;
    const long side = 32L * q.mi, row_tiles = (rows + side - 1) / side, tiles = (c_out + side - 1) / side, run = 2L * q.mi * fours;
    q.codes = (size_t)(row_tiles * run * 4096), q.x_scales = (size_t)(row_tiles * run * 256);
    q.w_codes = (size_t)(tiles * run * 4096), q.w_scales = (size_t)(tiles * run * 256);
  } else {
    q.form = kFew;
    // Up to 16 rows the work-groups make the codes themselves, each all of them, a lane reading 64 or 128 bytes of a row of its own.  Where that is much and slow,
    // by twice the bytes or as 16-bit rows of odd length begin between two dwords, a launch before is quicker: 16 x 4097 x 1000 bf16 15.6 -> 6.1 us and 10.4 -> 6.3 in
    // fp32; but 8 x 1025 x 1000 no difference, 8 x 4096 x 1000 bf16 6.6 and 7.3.  (4 x 8191 x 1000, just under the limit, 13.5 and 9.1.  The length stands for the rows'
    // distance, which the question for scratch does not say: 16 rows of 4096 bf16 at a distance of 4109 stay without the launch, 12.3 us; at 4096 7.9, at 4108 5.6.)
    q.codes_first = dtype >= 0 && (rows > 16 || ((dtype == CPRUNE_F32 || k % 2) && (long)rows * k >= 32768));
  }
  if (q.codes_first) {
    q.codes = (size_t)((long)rows * blocks * 16);
    q.x_scales = ((size_t)((long)rows * blocks) + 15) & ~(size_t)15;
  }
  return q;
}

template <typename F> void with_flag(bool b, F&& f) { b ? f(std::true_type()) : f(std::false_type()); }
template <typename X, typename T, bool SILU> void launch_few(Mx4Args p, hipStream_t s) {
  const int steps = (p.blocks + 3) / 4;
  auto go = [&](auto mb, auto nb, auto waves) {
    constexpr int MB = decltype(mb)::value, NB = decltype(nb)::value, WAVES = decltype(waves)::value;
    p.tiles = (p.c_out + 16 * MB - 1) / (16 * MB);
    const unsigned grid = (unsigned)((long)p.tiles * ((p.rows + 16 * NB - 1) / (16 * NB)));
    mx4_few_kernel<X, T, SILU, MB, NB, WAVES><<<grid, 64 * WAVES, 0, s>>>(p);
  };
  typedef std::integral_constant<int, 1> one;
  typedef std::integral_constant<int, 2> two;
  typedef std::integral_constant<int, 4> four;
  typedef std::integral_constant<int, 16> sixteen;
  if (p.rows <= 16) {
    if (steps > 8) go(one(), one(), sixteen());
    else go(one(), one(), four());
  } else if constexpr (std::is_same<X, void>::value) {
    if (p.rows <= 32) go(one(), two(), std::integral_constant<int, 8>());
    else go(two(), four(), std::integral_constant<int, 8>());
  }
}
template <typename X, typename T, bool SILU> void launch_short(const Mx4Args& p, hipStream_t s) {
  const int steps = (p.blocks + 3) / 4;
  const unsigned row_groups = (unsigned)((p.rows + 63) / 64), tiles = (unsigned)((p.c_out + (p.c_out > 32 ? 63 : 31)) / (p.c_out > 32 ? 64 : 32));
  // (outputs are shared out where there are few rows: 12544 x 96 x 576 12.1 -> 9.2 us, 784 x 160 x 960 18.5 -> 4.0)
  const dim3 grid(row_groups, std::min(tiles, std::max(1u, 1024u / row_groups)));
  auto go = [&](auto n) {
    if (p.c_out > 32) mx4_rows_kernel<X, T, SILU, 4, 1, decltype(n)::value><<<grid, 256, 0, s>>>(p);
    else mx4_rows_kernel<X, T, SILU, 2, 1, decltype(n)::value><<<grid, 256, 0, s>>>(p);
  };
  if (steps <= 1) go(std::integral_constant<int, 1>());
  else if (steps <= 2) go(std::integral_constant<int, 2>());
  else if (steps <= 3) go(std::integral_constant<int, 3>());
  else go(std::integral_constant<int, kShortSteps>());
}
template <typename T, bool SILU> void launch_tiles(Mx4Args p, int mi, hipStream_t s) {
  p.tiles = (p.c_out + 32 * mi - 1) / (32 * mi);
  p.row_tiles = (p.rows + 32 * mi - 1) / (32 * mi);
  const unsigned grid = (unsigned)((long)p.tiles * p.row_tiles);
  // three stages where a compute unit has work for a third work-group (11008 x 256 x 2880 30.8 -> 27.7 us; 1024 x 8192 x 1024, one each, 28.6 and with four 24.7)
  if (mi == 8) mx4_tile_kernel<T, SILU, 8, 4><<<grid, 256, 0, s>>>(p);
  else if (mi == 4 && grid > 256) mx4_tile_kernel<T, SILU, 4, 3><<<grid, 256, 0, s>>>(p);
  else if (mi == 4) mx4_tile_kernel<T, SILU, 4, 4><<<grid, 256, 0, s>>>(p);
  else mx4_tile_kernel<T, SILU, 2, 4><<<grid, 256, 0, s>>>(p);
}

// x: numbers of `dtype`, or (x_scales given) codes
void launch_product(Mx4Args p, const void* x, const void* x_scales, int k, long x_stride, int act, int dtype, void* ws, const ProductPlan& q, hipStream_t s) {
  const float inf = std::numeric_limits<float>::infinity();
  p.lo = act == CPRUNE_ACT_NONE ? -inf : 0.0f;
  p.hi = act == CPRUNE_ACT_RELU6 ? 6.0f : inf;
  char* const scratch = static_cast<char*>(ws);
  bool codes = x_scales != nullptr;
  if (q.form == kTiles) {
    const int fours = (p.blocks + 15) / 16;
    Mx4Arrange r = {};
    r.x = x, r.xs = static_cast<const unsigned char*>(x_scales), r.w = p.a, r.ws = p.as, r.x_stride = x_stride;
    r.rows = p.rows, r.k = k, r.c_out = p.c_out, r.blocks = p.blocks, r.mi = q.mi;
    r.x_codes = reinterpret_cast<unsigned*>(scratch);
    r.x_scales = reinterpret_cast<unsigned*>(scratch + q.codes);
    r.w_codes = reinterpret_cast<unsigned*>(scratch + q.codes + q.x_scales);
    r.w_scales = reinterpret_cast<unsigned*>(scratch + q.codes + q.x_scales + q.w_codes);
    r.row_groups = (int)(q.codes / 4096);
    const unsigned groups = (unsigned)(r.row_groups + q.w_codes / 4096);
    if (codes) mx4_arrange_kernel<void><<<groups, 256, 0, s>>>(r);
    else with_type(dtype, [&](auto t) { mx4_arrange_kernel<decltype(t)><<<groups, 256, 0, s>>>(r); });
    p.bo = reinterpret_cast<const uint4*>(r.x_codes), p.bso = r.x_scales;
    p.ao = reinterpret_cast<const uint4*>(r.w_codes), p.aso = r.w_scales;
  } else if (q.codes_first) {
    launch_quantize(x, p.rows, k, (int)x_stride, dtype, scratch, scratch + q.codes, s);
    p.b = reinterpret_cast<const unsigned char*>(scratch), p.bs = p.b + q.codes;
    codes = true;
  } else if (codes) {
    p.b = static_cast<const unsigned char*>(x), p.bs = static_cast<const unsigned char*>(x_scales);
  } else {
    p.x = x, p.x_stride = x_stride, p.k = k;
  }
  with_type(dtype, [&](auto t) {
    using T = decltype(t);
    with_flag(act == CPRUNE_ACT_SILU, [&](auto silu) {
      constexpr bool SILU = decltype(silu)::value;
      if (q.form == kTiles) launch_tiles<T, SILU>(p, q.mi, s);
      else if (q.form == kShort && codes) launch_short<void, T, SILU>(p, s);
      else if (q.form == kShort) launch_short<T, T, SILU>(p, s);
      else if (codes) launch_few<void, T, SILU>(p, s);
      else launch_few<T, T, SILU>(p, s);
    });
  });
}

int check_product(int rows, int k, int c_out, int act, int dtype) {
  if (rows < 1 || k < 1 || k > 0x7fffffff - 31 || c_out < 1 || !act_of_product(act) || !dtype_ok(dtype)) return CPRUNE_ERR_INVALID_ARG;
  return too_many(rows, k) || too_many(c_out, k) || (double)rows * c_out >= 2147483648.0 ? CPRUNE_ERR_INVALID_ARG : CPRUNE_OK;
}

}  // namespace
}  // namespace cprune

using namespace cprune;

extern "C" int cprune_mx4_quantize(const void* x, int rows, int k, int x_stride, cprune_dtype dtype, void* codes, void* scales, void* stream) {
  const int rc = check_numbers(rows, k, x_stride, dtype);
  if (rc != CPRUNE_OK) return rc;
  if (!x || !codes || !scales || !aligned16(codes)) return CPRUNE_ERR_INVALID_ARG;
  launch_quantize(x, rows, k, x_stride, dtype, codes, scales, static_cast<hipStream_t>(stream));
  CPRUNE_LAUNCH_CHECK();
  return CPRUNE_OK;
}

extern "C" int cprune_mx4_dequantize(const void* codes, const void* scales, int rows, int k, cprune_dtype dtype, void* y, void* stream) {
  const int rc = check_numbers(rows, k, k, dtype);
  if (rc != CPRUNE_OK) return rc;
  if (!codes || !scales || !y || !aligned16(codes)) return CPRUNE_ERR_INVALID_ARG;
  const int blocks = blocks_of(k);
  const unsigned grid = (unsigned)(((long)rows * blocks * 4 + kQuad - 1) / kQuad);
  with_type(dtype, [&](auto t) {
    using T = decltype(t);
    mx4_dequantize_kernel<T><<<grid, kQuad, 0, static_cast<hipStream_t>(stream)>>>(
        static_cast<const unsigned*>(codes), static_cast<const unsigned char*>(scales), rows, k, blocks, static_cast<T*>(y));
  });
  CPRUNE_LAUNCH_CHECK();
  return CPRUNE_OK;
}

extern "C" size_t cprune_mx4_matmul_workspace_bytes(int rows, int k, int c_out) {
  if (check_product(rows, k, c_out, CPRUNE_ACT_NONE, CPRUNE_F32) != CPRUNE_OK) return 0;
  return plan_product(rows, k, c_out, -1).total();
}

extern "C" int cprune_mx4_matmul(const void* x_codes, const void* x_scales, int rows, int k, const void* w_codes, const void* w_scales,
                                 int c_out, const float* bias, cprune_act act, cprune_dtype dtype, void* y, void* ws, size_t ws_bytes,
                                 void* stream) {
  const int rc = check_product(rows, k, c_out, act, dtype);
  if (rc != CPRUNE_OK) return rc;
  if (!x_codes || !x_scales || !w_codes || !w_scales || !y || !aligned16(x_codes) || !aligned16(w_codes)) return CPRUNE_ERR_INVALID_ARG;
  const ProductPlan q = plan_product(rows, k, c_out, -1);
  if (q.total() && (!ws || ws_bytes < q.total())) return CPRUNE_ERR_WORKSPACE;
  if (!aligned16(ws)) return CPRUNE_ERR_INVALID_ARG;
  Mx4Args p = {};
  p.a = static_cast<const unsigned char*>(w_codes), p.as = static_cast<const unsigned char*>(w_scales);
  p.bias = bias, p.y = y, p.rows = rows, p.c_out = c_out, p.blocks = blocks_of(k);
  launch_product(p, x_codes, x_scales, k, 0, act, dtype, ws, q, static_cast<hipStream_t>(stream));
  CPRUNE_LAUNCH_CHECK();
  return CPRUNE_OK;
}

extern "C" size_t cprune_mx4_linear_workspace_bytes(int rows, int k, int c_out, cprune_dtype dtype) {
  if (check_product(rows, k, c_out, CPRUNE_ACT_NONE, dtype) != CPRUNE_OK) return 0;
  return plan_product(rows, k, c_out, dtype).total();
}

extern "C" int cprune_mx4_linear(const void* x, int rows, int k, int x_stride, const void* w_codes, const void* w_scales, int c_out,
                                 const float* bias, cprune_act act, cprune_dtype dtype, void* y, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_product(rows, k, c_out, act, dtype);
  if (rc == CPRUNE_OK) rc = check_numbers(rows, k, x_stride, dtype);
  if (rc != CPRUNE_OK) return rc;
  if (!x || !w_codes || !w_scales || !y || !aligned16(w_codes)) return CPRUNE_ERR_INVALID_ARG;
  const ProductPlan q = plan_product(rows, k, c_out, dtype);
  if (q.total() && (!ws || ws_bytes < q.total())) return CPRUNE_ERR_WORKSPACE;
  if (!aligned16(ws)) return CPRUNE_ERR_INVALID_ARG;
  Mx4Args p = {};
  p.a = static_cast<const unsigned char*>(w_codes), p.as = static_cast<const unsigned char*>(w_scales);
  p.bias = bias, p.y = y, p.rows = rows, p.c_out = c_out, p.blocks = blocks_of(k);
  launch_product(p, x, nullptr, k, x_stride, act, dtype, ws, q, static_cast<hipStream_t>(stream));
  CPRUNE_LAUNCH_CHECK();
  return CPRUNE_OK;
}
