// Group norm with an activation, channels last, and its gradient.
//
// The lanes of a map.  x is [n][pixels][c]; a thread reads V numbers (16 bytes) at a time and keeps the channels it reads for the whole
// kernel, so that what belongs to a channel (weight, bias, statistics, sums) stays in registers.  Where V does not divide c and pixels lie
// without gaps, a "superrow" of R = V / gcd(V, c) pixels is P = R c / V whole vectors; its element q is channel q mod c, and it
// comes back every superrow.  83 channels of fp32: R = 4, P = 83.  Maps with gaps between pixels: R = 1 and the largest V that divides c.
// A work-group is `rpi` superrows of `tp` vectors; it walks over a run ("chunk") of superrows of one image.  The last superrow of an image may hold fewer
// than R pixels: its elements are checked one by one.  No alignment is assumed (loads of 16 bytes may begin at any element).
#pragma once
#include <type_traits>

#include "common.hpp"

namespace cprune {

struct NormGeom {
  int V, R, P;         // as above
  int tp, tiles, rpi;  // vectors of a superrow a work-group takes, work-groups side by side, superrows at a time
  int threads;
  int SR, spc, chunks;  // superrows of an image, of a chunk; chunks of an image
  int tail;             // pixels of the last superrow
};

struct NormArgs {
  const void *x, *dy;
  const float *weight, *bias;
  const float *mean, *rstd;   // [n][g]
  const float2* terms;        // backward: (mean(w dz), mean(w dz xhat)) [n][g]
  void* y;                    // forward: y, backward: dx
  float2* part;               // [n][chunk][R * c]: forward (mean, squares about it), backward (sum dz, sum dz xhat)
  int pixels, c, cg, groups;
  long x_image, x_pitch, dy_image, dy_pitch;   // elements from image to image, from superrow to superrow
  float lo, hi;               // clamp of the activation
  NormGeom g;
};

namespace norm {

template <typename T> struct Bits { typedef unsigned short type; };
template <> struct Bits<float> { typedef float type; };
template <typename B, int V> struct RawOf { typedef B type __attribute__((ext_vector_type(V), aligned(sizeof(B)))); };

template <typename T> __device__ __forceinline__ float widen(typename Bits<T>::type b) {
  if constexpr (std::is_same<T, float>::value) return b;
  else if constexpr (std::is_same<T, __bf16>::value) return __uint_as_float((unsigned)b << 16);
  else return (float)__builtin_bit_cast(_Float16, b);
}
template <typename T> __device__ __forceinline__ typename Bits<T>::type narrow(float v) {
  if constexpr (std::is_same<T, float>::value) return v;
  else return __builtin_bit_cast(unsigned short, (T)v);
}

// V numbers at p, the first `valid` of them
template <typename T, int V> __device__ __forceinline__ typename RawOf<typename Bits<T>::type, V>::type load(const void* p, int valid) {
  typedef typename Bits<T>::type B;
  typedef typename RawOf<B, V>::type Raw;
  if (V == 1 || valid >= V) return *static_cast<const Raw*>(p);
  Raw r;
#pragma unroll
  for (int j = 0; j < V; ++j) r[j] = j < valid ? static_cast<const B*>(p)[j] : B(0);
  return r;
}
template <typename T, int V> __device__ __forceinline__ void store(void* p, const float (&v)[V], int valid) {
  typedef typename Bits<T>::type B;
  typedef typename RawOf<B, V>::type Raw;
  Raw r;
#pragma unroll
  for (int j = 0; j < V; ++j) r[j] = narrow<T>(v[j]);
  if (V == 1 || valid >= V) {
    *static_cast<Raw*>(p) = r;
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (j < valid) static_cast<B*>(p)[j] = r[j];
  }
}

// z / (1 + e^-z): the exponential's overflow at very negative z gives z * 0
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }
template <bool SILU> __device__ __forceinline__ float activate(float z, float lo, float hi) {
  if constexpr (SILU) return z * sigmoid(z);
  z = z < lo ? lo : z;      // (comparisons and not minimum / maximum: a NaN stays one)
  return z > hi ? hi : z;
}
template <bool SILU> __device__ __forceinline__ float slope(float z, float lo, float hi) {
  if constexpr (SILU) {
    const float s = sigmoid(z);
    return s * (1.0f + z * (1.0f - s));
  }
  return z <= lo || z >= hi ? 0.0f : 1.0f;
}
// xhat and the activation's argument with each operation rounded, as the formula has them: whether a clamp passes a gradient does not
// depend on which products and sums the compiler joins
__device__ __forceinline__ float centred(float x, float mean, float rstd) {
#pragma clang fp contract(off)
  return (x - mean) * rstd;
}
__device__ __forceinline__ float argument(float xhat, float w, float b) {
#pragma clang fp contract(off)
  const float p = xhat * w;
  return p + b;
}

// What a thread works on.
struct Place {
  int image, chunk, r, p, sr0, sr1;
  bool active;
};
__device__ __forceinline__ Place place(const NormGeom& g) {
  Place k;
  unsigned b = blockIdx.x;
  const int tile = (int)(b % (unsigned)g.tiles);
  b /= (unsigned)g.tiles;
  k.chunk = (int)(b % (unsigned)g.chunks);
  k.image = (int)(b / (unsigned)g.chunks);
  k.r = (int)threadIdx.x / g.tp;
  k.p = tile * g.tp + ((int)threadIdx.x - k.r * g.tp);
  k.active = k.r < g.rpi && k.p < g.P;
  k.sr0 = k.chunk * g.spc;
  k.sr1 = min(g.SR, k.sr0 + g.spc);
  return k;
}
// elements of the vector at position p that superrow sr has
__device__ __forceinline__ int valid_of(const NormGeom& g, int c, int sr, int p) {
  return sr == g.SR - 1 ? g.tail * c - p * g.V : g.V;
}

constexpr int kThreads = 256;

}  // namespace norm

// Statistics of a chunk: each thread's running mean and squares about it (an update by 1 / count per number: no difference of large sums, whatever
// the numbers' mean), then joined over the work-group's superrows pair by pair.
template <typename T, int V>
__global__ __launch_bounds__(norm::kThreads) void norm_stats_kernel(const NormArgs a) {
  using namespace norm;
  __shared__ float s_mean[V][kThreads], s_sq[V][kThreads], s_n[V][kThreads];
  const Place k = place(a.g);
  float mean[V], sq[V], cnt[V];
#pragma unroll
  for (int j = 0; j < V; ++j) mean[j] = sq[j] = cnt[j] = 0.0f;
  if (k.active) {
    const char* base = static_cast<const char*>(a.x) + (k.image * a.x_image + (long)k.p * V) * (long)sizeof(T);
    int i = 0;
    for (int sr = k.sr0 + k.r; sr < k.sr1; sr += a.g.rpi, ++i) {
      const int valid = valid_of(a.g, a.c, sr, k.p);
      if (valid <= 0) break;
      const auto raw = load<T, V>(base + sr * a.x_pitch * (long)sizeof(T), valid);
      const float rc = __builtin_amdgcn_rcpf((float)(i + 1));
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (j < valid) {
          const float v = widen<T>(raw[j]), d = v - mean[j];
          mean[j] = fmaf(d, rc, mean[j]);
          sq[j] = fmaf(d, v - mean[j], sq[j]);
          cnt[j] += 1.0f;
        }
      }
    }
  }
  const int t = threadIdx.x;
  int half = 1;
  while (2 * half < a.g.rpi) half *= 2;
#pragma unroll
  for (int j = 0; j < V; ++j) s_mean[j][t] = mean[j], s_sq[j][t] = sq[j], s_n[j][t] = cnt[j];
  for (; half > 0; half >>= 1) {
    __syncthreads();
    if (k.active && k.r < half && k.r + half < a.g.rpi) {
      const int o = t + half * a.g.tp;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float nb = s_n[j][o], n = cnt[j] + nb;
        if (nb > 0.0f) {
          const float d = s_mean[j][o] - mean[j], f = nb / n;
          mean[j] = fmaf(d, f, mean[j]);
          sq[j] += s_sq[j][o] + d * d * cnt[j] * f;
          cnt[j] = n;
        }
        s_mean[j][t] = mean[j], s_sq[j][t] = sq[j], s_n[j][t] = cnt[j];
      }
    }
  }
  if (k.active && k.r == 0) {
    float2* out = a.part + ((long)k.image * a.g.chunks + k.chunk) * a.g.P * V + (long)k.p * V;
#pragma unroll
    for (int j = 0; j < V; ++j) out[j] = make_float2(mean[j], sq[j]);
  }
}

template <typename T, int V, bool SILU>
__global__ __launch_bounds__(norm::kThreads) void norm_apply_kernel(const NormArgs a) {
  using namespace norm;
  const Place k = place(a.g);
  if (!k.active) return;
  float mean[V], w[V], b[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int ch = (k.p * V + j) % a.c, s = k.image * a.groups + ch / a.cg;
    mean[j] = a.mean[s];
    w[j] = a.rstd[s] * (a.weight ? a.weight[ch] : 1.0f);
    b[j] = a.bias ? a.bias[ch] : 0.0f;
  }
  const char* base = static_cast<const char*>(a.x) + (k.image * a.x_image + (long)k.p * V) * (long)sizeof(T);
  char* out = static_cast<char*>(a.y) + ((long)k.image * a.pixels * a.c + (long)k.p * V) * (long)sizeof(T);
  for (int sr = k.sr0 + k.r; sr < k.sr1; sr += a.g.rpi) {
    const int valid = valid_of(a.g, a.c, sr, k.p);
    if (valid <= 0) break;
    const auto raw = load<T, V>(base + sr * a.x_pitch * (long)sizeof(T), valid);
    float v[V];
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = activate<SILU>(fmaf(widen<T>(raw[j]) - mean[j], w[j], b[j]), a.lo, a.hi);
    store<T, V>(out + (long)sr * a.g.P * V * (long)sizeof(T), v, valid);
  }
}

// Sums of dz and dz xhat over a chunk.
template <typename T, int V, bool SILU>
__global__ __launch_bounds__(norm::kThreads) void norm_grad_sums_kernel(const NormArgs a) {
  using namespace norm;
  __shared__ float s_b[V][kThreads], s_w[V][kThreads];
  const Place k = place(a.g);
  float sb[V], sw[V];
#pragma unroll
  for (int j = 0; j < V; ++j) sb[j] = sw[j] = 0.0f;
  if (k.active) {
    float mean[V], rstd[V], w[V], b[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int ch = (k.p * V + j) % a.c, s = k.image * a.groups + ch / a.cg;
      mean[j] = a.mean[s];
      rstd[j] = a.rstd[s];
      w[j] = a.weight ? a.weight[ch] : 1.0f;
      b[j] = a.bias ? a.bias[ch] : 0.0f;
    }
    const char* xb = static_cast<const char*>(a.x) + (k.image * a.x_image + (long)k.p * V) * (long)sizeof(T);
    const char* db = static_cast<const char*>(a.dy) + (k.image * a.dy_image + (long)k.p * V) * (long)sizeof(T);
    for (int sr = k.sr0 + k.r; sr < k.sr1; sr += a.g.rpi) {
      const int valid = valid_of(a.g, a.c, sr, k.p);
      if (valid <= 0) break;
      const auto xr = load<T, V>(xb + sr * a.x_pitch * (long)sizeof(T), valid);
      const auto dr = load<T, V>(db + sr * a.dy_pitch * (long)sizeof(T), valid);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (j < valid) {
          const float xhat = centred(widen<T>(xr[j]), mean[j], rstd[j]);
          const float dz = widen<T>(dr[j]) * slope<SILU>(argument(xhat, w[j], b[j]), a.lo, a.hi);
          sb[j] += dz;
          sw[j] = fmaf(dz, xhat, sw[j]);
        }
      }
    }
  }
  const int t = threadIdx.x;
  int half = 1;
  while (2 * half < a.g.rpi) half *= 2;
#pragma unroll
  for (int j = 0; j < V; ++j) s_b[j][t] = sb[j], s_w[j][t] = sw[j];
  for (; half > 0; half >>= 1) {
    __syncthreads();
    if (k.active && k.r < half && k.r + half < a.g.rpi) {
      const int o = t + half * a.g.tp;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        s_b[j][t] = sb[j] += s_b[j][o];
        s_w[j][t] = sw[j] += s_w[j][o];
      }
    }
  }
  if (k.active && k.r == 0) {
    float2* out = a.part + ((long)k.image * a.g.chunks + k.chunk) * a.g.P * V + (long)k.p * V;
#pragma unroll
    for (int j = 0; j < V; ++j) out[j] = make_float2(sb[j], sw[j]);
  }
}

template <typename T, int V, bool SILU>
__global__ __launch_bounds__(norm::kThreads) void norm_grad_apply_kernel(const NormArgs a) {
  using namespace norm;
  const Place k = place(a.g);
  if (!k.active) return;
  float mean[V], rstd[V], w[V], b[V];
  float2 t[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int ch = (k.p * V + j) % a.c, s = k.image * a.groups + ch / a.cg;
    mean[j] = a.mean[s];
    rstd[j] = a.rstd[s];
    w[j] = a.weight ? a.weight[ch] : 1.0f;
    b[j] = a.bias ? a.bias[ch] : 0.0f;
    t[j] = a.terms[s];
  }
  const char* xb = static_cast<const char*>(a.x) + (k.image * a.x_image + (long)k.p * V) * (long)sizeof(T);
  const char* db = static_cast<const char*>(a.dy) + (k.image * a.dy_image + (long)k.p * V) * (long)sizeof(T);
  char* out = static_cast<char*>(a.y) + ((long)k.image * a.pixels * a.c + (long)k.p * V) * (long)sizeof(T);
  for (int sr = k.sr0 + k.r; sr < k.sr1; sr += a.g.rpi) {
    const int valid = valid_of(a.g, a.c, sr, k.p);
    if (valid <= 0) break;
    const auto xr = load<T, V>(xb + sr * a.x_pitch * (long)sizeof(T), valid);
    const auto dr = load<T, V>(db + sr * a.dy_pitch * (long)sizeof(T), valid);
    float v[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float xhat = centred(widen<T>(xr[j]), mean[j], rstd[j]);
      const float dz = widen<T>(dr[j]) * slope<SILU>(argument(xhat, w[j], b[j]), a.lo, a.hi);
      v[j] = rstd[j] * (fmaf(w[j], dz, -t[j].x) - xhat * t[j].y);
    }
    store<T, V>(out + (long)sr * a.g.P * V * (long)sizeof(T), v, valid);
  }
}

}  // namespace cprune
