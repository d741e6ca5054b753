// Entry points of the microscaled 4-bit numbers; quantisation and the way back (mx4_kernel.hpp has the products).
#include <limits>

#include "group_norm_kernel.hpp"
#include "mx4_kernel.hpp"

namespace cprune {
namespace {

constexpr int kQuad = 256;      // threads; eight numbers each, four threads a block of 32

// largest of an integer over the four lanes of a quad
__device__ __forceinline__ unsigned quad_max(unsigned v) {
  v = max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));
  return max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));
}

// The scale's byte from the largest magnitude's bits (as integers, magnitudes order like numbers, NaN above infinity).
__device__ __forceinline__ int scale_byte(unsigned top) {
  const int e = (int)(top >> 23);
  return e == 255 ? 255 : max(e - 2, 0);
}
__device__ __forceinline__ float scale_value(int s) {      // 2^(s - 127), NaN for 255
  return __uint_as_float(s == 255 ? 0x7fc00000u : s == 0 ? 0x00400000u : (unsigned)s << 23);
}

template <typename T>
__global__ __launch_bounds__(kQuad) void mx4_quantize_kernel(const T* __restrict__ x, int rows, int k, long x_stride, int blocks,
                                                             unsigned* __restrict__ codes, unsigned char* __restrict__ scales) {
  constexpr int V = 16 / (int)sizeof(T);
  const unsigned i = blockIdx.x * (unsigned)kQuad + threadIdx.x, per = 4u * blocks;
  if (i >= (unsigned)rows * per) return;      // (whole quads)
  const unsigned row = i / per, at = (i - row * per) * 8;
  const T* p = x + row * x_stride + at;
  const int valid = k - (int)at;
  float v[8];
#pragma unroll
  for (int h = 0; h < 8; h += V) {
    if (valid - h > 0) {
      const auto raw = norm::load<T, V>(p + h, valid - h);
#pragma unroll
      for (int j = 0; j < V; ++j) v[h + j] = norm::widen<T>(raw[j]);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) v[h + j] = 0.0f;
    }
  }
  unsigned top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
  const int s = scale_byte(quad_max(top));
  const float f = scale_value(s);
  unsigned c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], f, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], f, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], f, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], f, 3);
  codes[i] = s == 255 ? 0u : c;
  if ((threadIdx.x & 3) == 0) scales[i >> 2] = (unsigned char)s;
}

template <typename T>
__global__ __launch_bounds__(kQuad) void mx4_dequantize_kernel(const unsigned* __restrict__ codes, const unsigned char* __restrict__ scales,
                                                               int rows, int k, int blocks, T* __restrict__ y) {
  constexpr int V = 16 / (int)sizeof(T);
  const unsigned i = blockIdx.x * (unsigned)kQuad + threadIdx.x, per = 4u * blocks;
  if (i >= (unsigned)rows * per) return;
  const unsigned row = i / per, at = (i - row * per) * 8;
  const int valid = k - (int)at;
  if (valid <= 0) return;
  const unsigned c = codes[i];
  const float f = scale_value(scales[i >> 2]);
  typedef float float2v __attribute__((ext_vector_type(2)));
  float v[8];
  // (exact: a code's value times a power of two; the product and not the instruction's own scale, whose NaN and 2^-127 it need not know)
#define CPRUNE_MX4_PAIR(n)                                                       \
  {                                                                              \
    const float2v q = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, n);      \
    v[2 * n] = q.x * f, v[2 * n + 1] = q.y * f;                                  \
  }
  CPRUNE_MX4_PAIR(0) CPRUNE_MX4_PAIR(1) CPRUNE_MX4_PAIR(2) CPRUNE_MX4_PAIR(3)
#undef CPRUNE_MX4_PAIR
  T* p = y + (long)row * k + at;
#pragma unroll
  for (int h = 0; h < 8; h += V) {
    if (valid - h <= 0) break;
    float part[V];
#pragma unroll
    for (int j = 0; j < V; ++j) part[j] = v[h + j];
    norm::store<T, V>(p + h, part, valid - h);
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

void launch_product(Mx4Args p, int act, int dtype, hipStream_t s) {
  const float inf = std::numeric_limits<float>::infinity();
  p.lo = act == CPRUNE_ACT_NONE ? -inf : 0.0f;
  p.hi = act == CPRUNE_ACT_RELU6 ? 6.0f : inf;
  p.tiles = (p.c_out + 31) / 32;
  const dim3 grid((unsigned)((long)p.tiles * ((p.rows + 31) / 32)));
  with_type(dtype, [&](auto t) {
    using T = decltype(t);
    if (act == CPRUNE_ACT_SILU) mx4_wave_kernel<T, true, 2, 2, 4><<<grid, 256, 0, s>>>(p);
    else mx4_wave_kernel<T, false, 2, 2, 4><<<grid, 256, 0, s>>>(p);
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

extern "C" int cprune_mx4_matmul(const void* x_codes, const void* x_scales, int rows, int k, const void* w_codes, const void* w_scales,
                                 int c_out, const float* bias, cprune_act act, cprune_dtype dtype, void* y, void* stream) {
  const int rc = check_product(rows, k, c_out, act, dtype);
  if (rc != CPRUNE_OK) return rc;
  if (!x_codes || !x_scales || !w_codes || !w_scales || !y || !aligned16(x_codes) || !aligned16(w_codes)) return CPRUNE_ERR_INVALID_ARG;
  Mx4Args p = {};
  p.a = static_cast<const unsigned char*>(w_codes), p.as = static_cast<const unsigned char*>(w_scales);
  p.b = static_cast<const unsigned char*>(x_codes), p.bs = static_cast<const unsigned char*>(x_scales);
  p.bias = bias, p.y = y, p.rows = rows, p.c_out = c_out, p.blocks = blocks_of(k);
  launch_product(p, act, dtype, static_cast<hipStream_t>(stream));
  CPRUNE_LAUNCH_CHECK();
  return CPRUNE_OK;
}

extern "C" size_t cprune_mx4_linear_workspace_bytes(int rows, int k, int c_out, cprune_dtype dtype) {
  if (check_product(rows, k, c_out, CPRUNE_ACT_NONE, dtype) != CPRUNE_OK) return 0;
  const size_t blocks = (size_t)rows * blocks_of(k);
  return blocks * 16 + ((blocks + 15) & ~(size_t)15);
}

extern "C" int cprune_mx4_linear(const void* x, int rows, int k, int x_stride, const void* w_codes, const void* w_scales, int c_out,
                                 const float* bias, cprune_act act, cprune_dtype dtype, void* y, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_product(rows, k, c_out, act, dtype);
  if (rc == CPRUNE_OK) rc = check_numbers(rows, k, x_stride, dtype);
  if (rc != CPRUNE_OK) return rc;
  if (!x || !w_codes || !w_scales || !y || !aligned16(w_codes)) return CPRUNE_ERR_INVALID_ARG;
  if (!ws || ws_bytes < cprune_mx4_linear_workspace_bytes(rows, k, c_out, dtype)) return CPRUNE_ERR_WORKSPACE;
  if (!aligned16(ws)) return CPRUNE_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  unsigned char* codes = static_cast<unsigned char*>(ws);
  unsigned char* scales = codes + (size_t)rows * blocks_of(k) * 16;
  Mx4Args p = {};
  p.a = static_cast<const unsigned char*>(w_codes), p.as = static_cast<const unsigned char*>(w_scales);
  p.b = codes, p.bs = scales;
  p.bias = bias, p.y = y, p.rows = rows, p.c_out = c_out, p.blocks = blocks_of(k);
  launch_quantize(x, rows, k, x_stride, dtype, codes, scales, s);
  launch_product(p, act, dtype, s);
  CPRUNE_LAUNCH_CHECK();
  return CPRUNE_OK;
}
