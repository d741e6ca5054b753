// Microscaled 4-bit numbers: quantisation, the way back, and products on the scaled matrix instruction.
#pragma once
#include <type_traits>

#include "conv_kernel.hpp"

namespace cprune {

struct Mx4Args {
  const unsigned char *a, *as;   // weights' codes and scales, [c_out][blocks * 16], [c_out][blocks]
  const unsigned char *b, *bs;   // the rows', [rows][blocks * 16], [rows][blocks]
  const float* bias;
  void* y;                       // [rows][c_out]
  int rows, c_out, blocks;
  float lo, hi;
  int tiles;                     // tiles of c_out; work-groups are (rows, c_out), c_out first
};

namespace mx4 {

typedef int int8v __attribute__((ext_vector_type(8)));
constexpr unsigned kOne = 127;   // the scale's byte that stands for 1

// The matrix instruction's operand: lane l holds row l % 16 and the 32 elements of block l / 16, in four registers.
__device__ __forceinline__ float4_t mma(uint4 a, int as, uint4 b, int bs, float4_t acc) {
  const int8v av = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, bv = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv, acc, 4, 4, 0, as, 0, bs);
}

__device__ __forceinline__ uint4 load16(__amdgpu_buffer_rsrc_t r, unsigned off) {
  typedef unsigned int uint32x4_t __attribute__((ext_vector_type(4)));
  const uint32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, 0);
  return make_uint4(v.x, v.y, v.z, v.w);
}

}  // namespace mx4

// One wavefront-wide operand straight from memory, MB x NB blocks of 16 x 16 results a work-group, its WAVES wavefronts taking every WAVES-th
// 128 terms; their sums are joined through LDS in a fixed order.  Blocks past the last row or term read zeros with scale 1.
template <typename T, bool SILU, int MB, int NB, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void mx4_wave_kernel(const Mx4Args p) {
  using namespace mx4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lrow = lane & 15, lblk = lane >> 4;
  const int tr = blockIdx.x / (unsigned)p.tiles, o0 = ((int)blockIdx.x - tr * p.tiles) * 16 * MB, r0 = tr * 16 * NB;
  const unsigned a_bytes = (unsigned)p.c_out * p.blocks, b_bytes = (unsigned)p.rows * p.blocks;
  const __amdgpu_buffer_rsrc_t ar = make_rsrc(p.a, a_bytes * 16), asr = make_rsrc(p.as, a_bytes), br = make_rsrc(p.b, b_bytes * 16),
                               bsr = make_rsrc(p.bs, b_bytes);
  float4_t acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = (float4_t){0.f, 0.f, 0.f, 0.f};
  const int steps = (p.blocks + 3) / 4;
  for (int st = wave; st < steps; st += WAVES) {
    const int blk = st * 4 + lblk;
    uint4 av[MB], bv[NB];
    int as[MB], bs[NB];
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      const int o = o0 + 16 * i + lrow;
      const bool in = blk < p.blocks && o < p.c_out;
      const unsigned at = (unsigned)o * p.blocks + blk;
      av[i] = load16(ar, in ? at * 16 : kOutOfRange);
      as[i] = in ? (int)__builtin_amdgcn_raw_buffer_load_b8(asr, (int)at, 0, 0) : (int)kOne;
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int r = r0 + 16 * j + lrow;
      const bool in = blk < p.blocks && r < p.rows;
      const unsigned at = (unsigned)r * p.blocks + blk;
      bv[j] = load16(br, in ? at * 16 : kOutOfRange);
      bs[j] = in ? (int)__builtin_amdgcn_raw_buffer_load_b8(bsr, (int)at, 0, 0) : (int)kOne;
    }
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = mma(av[i], as[i], bv[j], bs[j], acc[i][j]);
  }
  __shared__ float4_t sums[WAVES - 1][MB * NB][64];
  if (wave > 0) {
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) sums[wave - 1][i * NB + j][lane] = acc[i][j];
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    const int o = o0 + 16 * i + 4 * lblk;
    const float4_t bias = load_bias4(p.bias, p.c_out, o);
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      float4_t v = acc[i][j];
      for (int w = 0; w < WAVES - 1; ++w) v += sums[w][i * NB + j][lane];
      const int r = r0 + 16 * j + lrow;
      if (r >= p.rows) continue;
      T* y = static_cast<T*>(p.y) + (long)r * p.c_out + o;
      float z[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        z[e] = v[e] + bias[e];
        if constexpr (SILU) {
          z[e] = z[e] * __builtin_amdgcn_rcpf(1.0f + __expf(-z[e]));
        } else {
          z[e] = z[e] < p.lo ? p.lo : z[e];     // (comparisons: a NaN stays one)
          z[e] = z[e] > p.hi ? p.hi : z[e];
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (o + e < p.c_out) y[e] = Elem<T>::from_f32(z[e]);
    }
  }
}

}  // namespace cprune
