// Entry points of the channels-last group norm and the kernels that join the chunks' sums (group_norm_kernel.hpp has the others).
#include <algorithm>
#include <cmath>
#include <limits>
#include <numeric>

#include "group_norm_kernel.hpp"

namespace cprune {
namespace {

// pixels of a superrow that chunk `chunk` counts at pixel rr
__device__ __forceinline__ int chunk_count(const NormGeom& g, int chunk, int rr) {
  const int sr0 = chunk * g.spc, sr1 = min(g.SR, sr0 + g.spc);
  return sr1 - sr0 - (sr1 == g.SR && rr >= g.tail ? 1 : 0);
}

__device__ __forceinline__ double2 group_sum(double2 v) {
  __shared__ double2 part[norm::kThreads / 64];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    v.x += __shfl_down(v.x, o, 64);
    v.y += __shfl_down(v.y, o, 64);
  }
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
  for (int i = 1; i < norm::kThreads / 64; ++i) v.x += part[i].x, v.y += part[i].y;
  return v;
}

// The chunks' statistics as those of an (image, group), one work-group each: sums over (count, mean, squares) about the first mean, in 64 bits.
__global__ __launch_bounds__(norm::kThreads) void norm_join_stats_kernel(const NormArgs a, float eps, float* __restrict__ mean_out,
                                                                         float* __restrict__ rstd_out) {
  const int image = blockIdx.x / a.groups, group = blockIdx.x - image * a.groups;
  const float2* part = a.part + (long)image * a.g.chunks * a.g.R * a.c + group * a.cg;
  const double first = part[0].x;
  const int per = a.g.R * a.cg, count = per * a.g.chunks;
  double2 s = {0.0, 0.0};
  for (int i = threadIdx.x; i < count; i += norm::kThreads) {
    const int chunk = i / per, e = i - chunk * per, rr = e / a.cg, ch = e - rr * a.cg;
    const int n = chunk_count(a.g, chunk, rr);
    if (n == 0) continue;
    const float2 p = part[(long)chunk * a.g.R * a.c + rr * a.c + ch];
    const double d = (double)p.x - first;
    s.x += n * d;
    s.y += (double)p.y + n * d * d;
  }
  s = group_sum(s);
  if (threadIdx.x == 0) {
    const double m = (double)a.pixels * a.cg, shift = s.x / m;
    double var = s.y / m - shift * shift;
    var = var < 0.0 ? 0.0 : var;
    mean_out[blockIdx.x] = (float)(first + shift);
    rstd_out[blockIdx.x] = (float)(1.0 / sqrt(var + (double)eps));
  }
}

// Work-groups up to n * groups: the two means of an (image, group).  The others: 32 channels of dweight and dbias each, eight threads a channel.
__global__ __launch_bounds__(norm::kThreads) void norm_join_grads_kernel(const NormArgs a, int n, float2* __restrict__ terms,
                                                                         float* __restrict__ dweight, float* __restrict__ dbias) {
  const long row = (long)a.g.R * a.c;      // partial sums of a chunk
  if ((int)blockIdx.x < n * a.groups) {
    const int image = blockIdx.x / a.groups, group = blockIdx.x - image * a.groups;
    const float2* part = a.part + (long)image * a.g.chunks * row + group * a.cg;
    const int per = a.g.R * a.cg, count = per * a.g.chunks;
    double2 s = {0.0, 0.0};
    for (int i = threadIdx.x; i < count; i += norm::kThreads) {
      const int chunk = i / per, e = i - chunk * per, rr = e / a.cg, ch = e - rr * a.cg;
      const float2 p = part[chunk * row + rr * a.c + ch];
      const double w = a.weight ? a.weight[group * a.cg + ch] : 1.0f;
      s.x += w * p.x;
      s.y += w * p.y;
    }
    s = group_sum(s);
    const double m = (double)a.pixels * a.cg;
    if (threadIdx.x == 0) terms[blockIdx.x] = make_float2((float)(s.x / m), (float)(s.y / m));
    return;
  }
  const int ch = ((int)blockIdx.x - n * a.groups) * 32 + (threadIdx.x & 31), lane = threadIdx.x >> 5;
  __shared__ double2 sums[8][32];
  double2 s = {0.0, 0.0};
  if (ch < a.c) {
    const long count = (long)n * a.g.chunks * a.g.R;
    for (long i = lane; i < count; i += 8) {
      const float2 p = a.part[i * a.c + ch];
      s.x += p.x;
      s.y += p.y;
    }
  }
  sums[lane][threadIdx.x & 31] = s;
  __syncthreads();
  if (lane == 0 && ch < a.c) {
    for (int i = 1; i < 8; ++i) s.x += sums[i][threadIdx.x].x, s.y += sums[i][threadIdx.x].y;
    if (dbias) dbias[ch] = (float)s.x;
    if (dweight) dweight[ch] = (float)s.y;
  }
}

int vector_of(int c, int dtype, bool dense) {
  int v = dtype == CPRUNE_F32 ? 4 : 8;
  if (!dense)
    while (c % v) v /= 2;
  return v;
}

NormGeom geometry(const cprune_norm_desc& d, bool backward) {
  NormGeom g;
  const bool dense = d.x_stride == d.c && (!backward || d.dy_stride == d.c);
  g.V = vector_of(d.c, d.dtype, dense);
  g.R = g.V / std::gcd(g.V, d.c);
  g.P = (int)((long)g.R * d.c / g.V);
  g.tiles = (g.P + norm::kThreads - 1) / norm::kThreads;
  g.tp = (g.P + g.tiles - 1) / g.tiles;
  g.rpi = norm::kThreads / g.tp;
  g.threads = norm::kThreads;
  g.SR = (d.pixels + g.R - 1) / g.R;
  g.tail = d.pixels - (g.SR - 1) * g.R;
  // about eight work-groups a compute unit, and at least four vectors a thread
  const long want = (2048 + (long)d.n * g.tiles - 1) / ((long)d.n * g.tiles);
  const long most = (g.SR + 4L * g.rpi - 1) / (4L * g.rpi);
  const long chunks = std::max(1L, std::min(want, most));
  g.spc = (int)((g.SR + chunks - 1) / chunks);
  g.spc = (g.spc + g.rpi - 1) / g.rpi * g.rpi;
  g.chunks = (g.SR + g.spc - 1) / g.spc;
  return g;
}

bool act_of_norm(int act) { return act_ok(act) || act == CPRUNE_ACT_SILU; }

int check(const cprune_norm_desc* d, bool backward) {
  if (!d || d->n < 1 || d->pixels < 1 || d->c < 1 || d->groups < 1 || d->c % d->groups || !dtype_ok(d->dtype) || !act_of_norm(d->act) ||
      d->x_stride < d->c || (backward && d->dy_stride < d->c))
    return CPRUNE_ERR_INVALID_ARG;
  if (!backward && !(d->eps > 0.0f && std::isfinite(d->eps))) return CPRUNE_ERR_INVALID_ARG;
  const int stride = backward ? std::max(d->x_stride, d->dy_stride) : d->x_stride;
  if ((double)d->n * d->pixels * stride >= 2147483648.0) return CPRUNE_ERR_INVALID_ARG;
  return CPRUNE_OK;
}

// (a launch holds fewer than 2^32 threads)
bool too_many_groups(const cprune_norm_desc& d, const NormGeom& g) {
  return std::max((double)d.n * g.chunks * g.tiles, (double)d.n * d.groups + (d.c + 31) / 32) * norm::kThreads >= 4294967296.0;
}

size_t round16(size_t b) { return (b + 15) & ~(size_t)15; }
size_t part_bytes(const cprune_norm_desc& d, const NormGeom& g) {
  return round16((size_t)d.n * g.chunks * g.R * d.c * sizeof(float2));
}
size_t stats_bytes(const cprune_norm_desc& d) { return round16((size_t)d.n * d.groups * sizeof(float2)); }

NormArgs args_of(const cprune_norm_desc& d, const NormGeom& g) {
  NormArgs a = {};
  a.pixels = d.pixels, a.c = d.c, a.groups = d.groups, a.cg = d.c / d.groups;
  a.x_image = (long)d.pixels * d.x_stride, a.x_pitch = (long)g.R * d.x_stride;
  a.dy_image = (long)d.pixels * d.dy_stride, a.dy_pitch = (long)g.R * d.dy_stride;
  const float inf = std::numeric_limits<float>::infinity();
  a.lo = d.act == CPRUNE_ACT_NONE ? -inf : 0.0f;
  a.hi = d.act == CPRUNE_ACT_RELU6 ? 6.0f : inf;
  a.g = g;
  return a;
}

// calls f(type, vector length, activation) with what the call needs
template <typename F> void with_form(int dtype, int v, bool silu, F&& f) {
  auto act = [&](auto t, auto vec) {
    if (silu) f(t, vec, std::true_type());
    else f(t, vec, std::false_type());
  };
  auto vec = [&](auto t) {
    if (v == 4) act(t, std::integral_constant<int, 4>());
    else if (v == 2) act(t, std::integral_constant<int, 2>());
    else act(t, std::integral_constant<int, 1>());
  };
  if (dtype == CPRUNE_F32) vec(float());
  else if (dtype == CPRUNE_F16) v == 8 ? act(_Float16(), std::integral_constant<int, 8>()) : vec(_Float16());
  else v == 8 ? act(__bf16(), std::integral_constant<int, 8>()) : vec(__bf16());
}

}  // namespace
}  // namespace cprune

using namespace cprune;

extern "C" size_t cprune_group_norm_workspace_bytes(const cprune_norm_desc* d, int backward) {
  if (check(d, backward != 0) != CPRUNE_OK) return 0;
  return part_bytes(*d, geometry(*d, backward != 0)) + stats_bytes(*d);
}

extern "C" int cprune_group_norm_act(const cprune_norm_desc* d, const void* x, const float* weight, const float* bias, void* y,
                                     float* mean_out, float* rstd_out, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check(d, false);
  if (rc != CPRUNE_OK) return rc;
  if (!x || !y) return CPRUNE_ERR_INVALID_ARG;
  const NormGeom g = geometry(*d, false);
  if (too_many_groups(*d, g)) return CPRUNE_ERR_UNSUPPORTED;
  if (!ws || ws_bytes < part_bytes(*d, g) + stats_bytes(*d)) return CPRUNE_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  NormArgs a = args_of(*d, g);
  a.x = x, a.y = y, a.weight = weight, a.bias = bias;
  a.part = static_cast<float2*>(ws);
  float* stats = reinterpret_cast<float*>(static_cast<char*>(ws) + part_bytes(*d, g));
  float* mean = mean_out ? mean_out : stats;
  float* rstd = rstd_out ? rstd_out : stats + (size_t)d->n * d->groups;
  a.mean = mean, a.rstd = rstd;
  const dim3 grid((unsigned)(d->n * g.chunks * g.tiles)), block(g.threads);
  with_form(d->dtype, g.V, d->act == CPRUNE_ACT_SILU, [&](auto t, auto v, auto silu) {
    using T = decltype(t);
    norm_stats_kernel<T, decltype(v)::value><<<grid, block, 0, s>>>(a);
    norm_join_stats_kernel<<<d->n * d->groups, norm::kThreads, 0, s>>>(a, d->eps, mean, rstd);
    norm_apply_kernel<T, decltype(v)::value, decltype(silu)::value><<<grid, block, 0, s>>>(a);
  });
  CPRUNE_LAUNCH_CHECK();
  return CPRUNE_OK;
}

extern "C" int cprune_group_norm_act_backward(const cprune_norm_desc* d, const void* dy, const void* x, const float* mean,
                                              const float* rstd, const float* weight, const float* bias, void* dx, float* dweight,
                                              float* dbias, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check(d, true);
  if (rc != CPRUNE_OK) return rc;
  if (!dy || !x || !mean || !rstd || !dx) return CPRUNE_ERR_INVALID_ARG;
  const NormGeom g = geometry(*d, true);
  if (too_many_groups(*d, g)) return CPRUNE_ERR_UNSUPPORTED;
  if (!ws || ws_bytes < part_bytes(*d, g) + stats_bytes(*d)) return CPRUNE_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  NormArgs a = args_of(*d, g);
  a.x = x, a.dy = dy, a.y = dx, a.weight = weight, a.bias = bias, a.mean = mean, a.rstd = rstd;
  a.part = static_cast<float2*>(ws);
  float2* terms = reinterpret_cast<float2*>(static_cast<char*>(ws) + part_bytes(*d, g));
  a.terms = terms;
  const dim3 grid((unsigned)(d->n * g.chunks * g.tiles)), block(g.threads);
  const int sums = dweight || dbias ? (d->c + 31) / 32 : 0;
  with_form(d->dtype, g.V, d->act == CPRUNE_ACT_SILU, [&](auto t, auto v, auto silu) {
    using T = decltype(t);
    norm_grad_sums_kernel<T, decltype(v)::value, decltype(silu)::value><<<grid, block, 0, s>>>(a);
    norm_join_grads_kernel<<<d->n * d->groups + sums, norm::kThreads, 0, s>>>(a, d->n, terms, dweight, dbias);
    norm_grad_apply_kernel<T, decltype(v)::value, decltype(silu)::value><<<grid, block, 0, s>>>(a);
  });
  CPRUNE_LAUNCH_CHECK();
  return CPRUNE_OK;
}
