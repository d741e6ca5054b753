// Rows of logits: what the top-logits and the distillation kernels share.
//
// A work-group has a row, or a run of one; a thread reads 16 bytes at a time, V numbers, vector t + i NT of the row its i-th.  Rows may begin at any element
// (an odd number of classes, the first classes of wider rows): loads and stores of 16 bytes need the element's alignment only.  Places past a row's
// end hold -infinity, a class that is not there.
#pragma once
#include <cfloat>
#include <type_traits>

#include "common.hpp"
#include "past_caches.hpp"

namespace cprune {
namespace logits {

constexpr float kLog2e = 1.44269504f;

template <typename T> struct Raw;
template <> struct Raw<float> {
  static constexpr int V = 4;
  static constexpr unsigned kNone = 0xff800000u;
};
template <> struct Raw<_Float16> {
  static constexpr int V = 8;
  static constexpr unsigned kNone = 0xfc00fc00u;
};
template <> struct Raw<__bf16> {
  static constexpr int V = 8;
  static constexpr unsigned kNone = 0xff80ff80u;
};

template <typename T> __device__ __forceinline__ float widen(T v) { return (float)v; }
template <> __device__ __forceinline__ float widen<__bf16>(__bf16 v) { return __uint_as_float((unsigned)__builtin_bit_cast(unsigned short, v) << 16); }

template <typename T> __device__ __forceinline__ void unpack(const uint4& r, float (&x)[Raw<T>::V]) {
  const unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      x[i] = __uint_as_float(w[i]);
    } else if constexpr (std::is_same<T, __bf16>::value) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      x[2 * i] = (float)__builtin_bit_cast(_Float16, (unsigned short)w[i]);
      x[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (unsigned short)(w[i] >> 16));
    }
  }
}

// (What is held is unpacked again each time: without this the compiler keeps the unpacked numbers, twice the registers and more.)
__device__ __forceinline__ void pin(uint4& r) { asm volatile("" : "+v"(r.x), "+v"(r.y), "+v"(r.z), "+v"(r.w)); }

// `classes` numbers at p: whole vectors and, past them, an edge of fewer than V numbers, which is one thread's and apart from the loops (its code in each of
// their steps would be most of a kernel).
template <typename T> struct Row {
  static constexpr int V = Raw<T>::V;
  const T* p;
  int full, tail;      // whole vectors, numbers behind them
  __device__ __forceinline__ Row(const T* p, int classes) : p(p), full(classes / V), tail(classes % V) {}
  static __device__ __forceinline__ uint4 none() { return make_uint4(Raw<T>::kNone, Raw<T>::kNone, Raw<T>::kNone, Raw<T>::kNone); }
  // vector i of those before `end`
  __device__ __forceinline__ uint4 load(int i, int end) const {
    typedef unsigned uint4u __attribute__((ext_vector_type(4), aligned(2)));
    uint4 r = none();
    if (i < end) {
      const uint4u v = *reinterpret_cast<const uint4u*>(p + (long)i * V);
      r = make_uint4(v.x, v.y, v.z, v.w);
    }
    return r;
  }
  // the edge, for the thread that asks for it
  __device__ __forceinline__ void edge(bool mine, float (&x)[V]) const {
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = -__builtin_inff();
    if (mine) {
#pragma unroll
      for (int j = 0; j < V - 1; ++j)
        if (j < tail) x[j] = widen<T>(p[(long)full * V + j]);
    }
  }
};

template <typename T> __device__ __forceinline__ void store(T* p, int i, const float (&x)[Raw<T>::V], bool past) {
  constexpr int V = Raw<T>::V;
  typedef T outs __attribute__((ext_vector_type(V), aligned(2)));
  outs v;
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = (T)x[j];
  outs* const to = reinterpret_cast<outs*>(p + (long)i * V);
  CPRUNE_STORE(to, v, past);
}
template <typename T> __device__ __forceinline__ void store_edge(T* p, const Row<T>& row, const float (&x)[Raw<T>::V]) {
#pragma unroll
  for (int j = 0; j < Raw<T>::V - 1; ++j)
    if (j < row.tail) p[(long)row.full * Raw<T>::V + j] = (T)x[j];
}

// Largest of two, NaN where one is.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

template <int V> __device__ __forceinline__ float largest(const float (&x)[V]) {
  float m = x[0];
#pragma unroll
  for (int i = 1; i < V; ++i) m = larger(m, x[i]);
  return m;
}

template <typename F> void with_type(int dtype, F&& f) {
  if (dtype == CPRUNE_F32) f(float());
  else if (dtype == CPRUNE_F16) f(_Float16());
  else f(__bf16());
}

}  // namespace logits
}  // namespace cprune
