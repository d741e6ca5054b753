// Entry points of the channels-last group norm and the kernels that join the chunks' sums (group_norm_kernel.hpp has the others).
// Figures at a rule are of both its sides, measured beside each other when it was chosen.
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

// A work-group's sum of its threads' pairs, in a fixed order, in every thread.
__device__ __forceinline__ double2 block_sum(double2 s) {
  __shared__ double2 sums[1024 / 64];
  const int t = (int)threadIdx.x;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    s.x += __shfl_down(s.x, o, 64);
    s.y += __shfl_down(s.y, o, 64);
  }
  if ((t & 63) == 0) sums[t >> 6] = s;
  __syncthreads();
  s = sums[0];
  for (int i = 1; i < (int)blockDim.x / 64; ++i) s.x += sums[i].x, s.y += sums[i].y;
  return s;
}

// Sum over the entries (chunk, pixel of the superrow, channel of the group) of an (image, group), one work-group, in 64 bits and a fixed order: f(chunk,
// pixel, entry, weight).  Eight entries are under way at a time; a thread counts its place on instead of dividing.
template <typename F> __device__ __forceinline__ double2 entries_sum(const NormArgs& a, const float2* part, const float* weight, F&& f) {
  const int t = (int)threadIdx.x, n = (int)blockDim.x, row = a.g.R * a.c, per = a.g.R * a.cg;
  int chunk = t / per, rr = (t - chunk * per) / a.cg, ch = t - chunk * per - rr * a.cg;
  const int d_chunk = n / per, d_rr = (n - d_chunk * per) / a.cg, d_ch = n - d_chunk * per - d_rr * a.cg;
  double2 s = {0.0, 0.0};
  while (chunk < a.g.chunks) {
    float2 e[8];
    float w[8];
    int at[8][2];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      at[u][0] = chunk, at[u][1] = rr;
      const int from = min(chunk, a.g.chunks - 1);      // (past the last chunk: counted out below)
      e[u] = part[(long)from * row + rr * a.c + ch];
      w[u] = weight ? weight[ch] : 1.0f;
      ch += d_ch, rr += d_rr, chunk += d_chunk;
      if (ch >= a.cg) ch -= a.cg, ++rr;
      if (rr >= a.g.R) rr -= a.g.R, ++chunk;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (at[u][0] < a.g.chunks) {
        const double2 v = f(at[u][0], at[u][1], e[u], w[u]);
        s.x += v.x, s.y += v.y;
      }
  }
  return block_sum(s);
}

// The chunks' statistics as those of an (image, group), where a superrow is wider than a work-group and groups are many.
__global__ __launch_bounds__(1024) void norm_join_stats_kernel(const NormArgs a, float* __restrict__ mean_out, float* __restrict__ rstd_out) {
  const int image = blockIdx.x / (unsigned)a.groups, group = blockIdx.x - image * a.groups;
  const float2* part = a.part + (long)image * a.g.chunks * a.g.R * a.c + group * a.cg;
  const double2 s = entries_sum(a, part, nullptr, [&](int chunk, int rr, float2 e, float) __attribute__((always_inline)) {
    return norm::raw_sums((double)chunk_count(a.g, chunk, rr), e);
  });
  if (threadIdx.x == 0) {
    const float2 m = norm::statistics(s, a);
    mean_out[blockIdx.x] = m.x;
    rstd_out[blockIdx.x] = m.y;
  }
}

// The two means of an (image, group), likewise.
__global__ __launch_bounds__(1024) void norm_join_grads_kernel(const NormArgs a, float2* __restrict__ terms) {
  const int image = blockIdx.x / (unsigned)a.groups, group = blockIdx.x - image * a.groups;
  const float2* part = a.part + (long)image * a.g.chunks * a.g.R * a.c + group * a.cg;
  const double2 s = entries_sum(a, part, a.weight ? a.weight + group * a.cg : nullptr, [&](int, int, float2 e, float w) __attribute__((always_inline)) {
    return make_double2((double)w * e.x, (double)w * e.y);
  });
  if (threadIdx.x == 0) terms[blockIdx.x] = make_float2((float)(s.x * a.inv_count), (float)(s.y * a.inv_count));
}

// The chunks' and tiles' sums of an (image, group) as its statistics, or as the two means (GRAD).
template <bool GRAD> __global__ __launch_bounds__(1024) void norm_join_groups_kernel(const NormArgs a, float* __restrict__ mean_out, float* __restrict__ rstd_out, float2* __restrict__ terms) {
  const int image = blockIdx.x / (unsigned)a.groups, group = blockIdx.x - image * a.groups, count = a.g.chunks * a.g.tiles, n = (int)blockDim.x;
  const double2* const part = a.gpart + (long)image * count * a.groups + group;
  double2 s = {0.0, 0.0};
  for (int i = (int)threadIdx.x; i < count; i += 8 * n) {
    double2 e[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) e[u] = part[(long)min(i + u * n, count - 1) * a.groups];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (i + u * n < count) s.x += e[u].x, s.y += e[u].y;
  }
  s = block_sum(s);
  if (threadIdx.x != 0) return;
  if constexpr (GRAD) {
    terms[blockIdx.x] = make_float2((float)(s.x * a.inv_count), (float)(s.y * a.inv_count));
  } else {
    const float2 m = norm::statistics(s, a);
    mean_out[blockIdx.x] = m.x;
    rstd_out[blockIdx.x] = m.y;
  }
}

// threads of those: four entries each or more, 64 to 1024
int join_threads(const NormGeom& g, int cg) {
  const long entries = g.joined ? (long)g.chunks * g.tiles : (long)g.chunks * g.R * cg;
  int t = 64;
  while (t < 1024 && 4L * t < entries) t *= 2;
  return t;
}

int vector_of(int c, int dtype, bool dense) {
  int v = dtype == CPRUNE_F32 ? 4 : 8;
  if (!dense)
    while (c % v) v /= 2;
  return v;
}

constexpr int kWholeColumns = 4096;      // elements of a slab's superrow (LDS)

// Threads that sum one of `groups` groups of `entries` each so that they fill the work-group: a power of two, past a wavefront where that leaves each four entries.
int lanes_of(int groups, int threads, long entries) {
  int lanes = 1024;
  while (lanes > 1 && ((long)lanes * groups > threads || (lanes > 64 && lanes * 4L > entries))) lanes /= 2;
  return lanes;
}

// Work-groups of the whole form for a slab of `tp` vectors a superrow: as few threads as hold half of what a thread can, or up to all of it.  (Bringing fewer
// threads to a map: 64 x 14 x 14 x 576 bf16 with eight vectors each 12.6 us, four 15.3; its gradient at 32 images with four 15.2, eight 18.1.)  false: too much.
bool fit_whole(NormGeom& g, int tp, int cg, bool backward, int most_threads, int most_vectors) {
  if (tp > most_threads || (long)tp * g.V > kWholeColumns) return false;
  for (int t = 256; t <= most_threads; t *= 2) {
    if (t < tp) continue;
    const int rpi = std::min(t / tp, g.SR), nv = (g.SR + rpi - 1) / rpi;
    if (nv <= most_vectors / 2 || (t == most_threads && nv <= most_vectors)) {
      g.tp = tp, g.rpi = rpi, g.nv = nv, g.slabs = g.P / tp;
      g.threads = (tp * rpi + 63) / 64 * 64;
      g.few = g.SR / rpi, g.more = g.SR % rpi, g.last_r = (g.SR - 1) % rpi;
      g.by_tp = norm_div(tp, 1024);
      g.groups = tp * g.V / (g.R * cg);
      g.lanes = lanes_of(g.groups, g.threads, (backward ? 1L : (long)rpi * g.R) * (cg % g.V || backward ? cg : cg / g.V));
      return true;
    }
  }
  return false;
}

// The whole form where a slab's pixels fit a work-group's registers: of the slabs of whole groups, the widest up to a cache line that still gives every
// compute unit one, otherwise the narrowest.
bool choose_whole(const cprune_norm_desc& d, bool backward, NormGeom& g) {
  const int v = d.dtype == CPRUNE_F32 ? 4 : 8, cg = d.c / d.groups;
  if (g.V != v) return false;
  const bool merge = cg % v == 0;
  const int most_threads = backward || merge || v == 4 ? 1024 : 512;      // (LDS: a pair a thread, or one for each of its elements)
  const int most_vectors = backward ? kNormWholeGradVectors : kNormWholeVectors;
  const int least = g.R > 1 ? g.P : std::lcm(v, cg) / v;                  // vectors
  const int times = g.P / least;
  for (int k = times; k > 1; --k)
    if (times % k == 0 && (long)least * k * 16 <= 128 && (long)d.n * (times / k) >= 256 && fit_whole(g, least * k, cg, backward, most_threads, most_vectors)) return true;
  // A compute unit alone brings some 10 to 20 GB/s from memory: the gradient of few and large slabs is split (27 x 7 x 22 x 111 fp16, 34 KB and 27 of them, 18.8 us
  // whole, 13.1 split; but 6 x 20 x 15 x 608 fp32, 114 of them, 10.3 and 13.5, and one of 11 KB, 7 x 99 x 16, 6.6 and 10.0).
  const double slab = (double)least * g.SR * 16;
  const long slabs = (long)d.n * times;
  if (backward && slab > 20000.0 && slabs < 64) return false;
  // (forward only where a thread's numbers are of several groups, whose sums take longer here: 20 x 67 x 9 x 98 fp16, 20 of 118 KB, 17.7 whole, 11.8 split; 13 x 38 x 30 x 160,
  // 52 of 91 KB, 10.8 and 13.1)
  if (!backward && !merge && slab > 65536.0 && slabs < 32) return false;
  if (!fit_whole(g, least, cg, backward, most_threads, most_vectors)) return false;
  // (the gradient's fullest form spills registers: not for more than one round of it, 31 x 108 x 10 x 800 bf16 62 whole, 50 split)
  return !(backward && g.nv > 4 && slabs > 256);
}

// Split form: the work-groups that read x leave sums of groups, and those that read it again join them.  Not where each of many work-groups beside each other
// would leave sums of many groups: a launch between has a work-group for each (image, group) then.
bool sums_groups(const cprune_norm_desc& d, const NormGeom& g) { return g.tiles == 1 || d.groups <= 64; }

constexpr int kChain = 512;

NormGeom geometry(const cprune_norm_desc& d, bool backward) {
  NormGeom g = {};
  const bool dense = d.x_stride == d.c && (!backward || d.dy_stride == d.c);
  g.V = vector_of(d.c, d.dtype, dense);
  g.R = g.V / std::gcd(g.V, d.c);
  g.P = (int)((long)g.R * d.c / g.V);
  g.SR = (int)(((long)d.pixels + g.R - 1) / g.R);
  g.tail = d.pixels - (g.SR - 1) * g.R;
  g.tiles = g.chunks = 1;
  if (choose_whole(d, backward, g)) return g;
  g.slabs = g.nv = 0;
  g.tiles = (g.P + norm::kThreads - 1) / norm::kThreads;
  g.tp = (g.P + g.tiles - 1) / g.tiles;
  g.rpi = norm::kThreads / g.tp;
  g.threads = norm::kThreads;
  g.groups = d.groups;
  g.by_tp = norm_div(g.tp, 1024);
  // two work-groups a compute unit, which run at once (registers): what a work-group does but once, its sums' way through LDS before all, is much of a
  // launch on maps of some MB (32 x 56 x 56 x 64 bf16 with 512 work-groups 18.7 us, 1024 21.7, 256 18.5; 64 x 112 x 112 x 96 fp16 105, 108, 110).  At least
  // four vectors a thread.
  const long want = std::max(1L, 512 / ((long)d.n * g.tiles));
  const long most = (g.SR + 4L * g.rpi - 1) / (4L * g.rpi);
  // (and few enough that a work-group joins an image's sums with sixteen entries a thread, or where a launch of its own does it with 64: one image of 64 groups has
  // 64 work-groups by that, 1 x 12544 x 1280 fp16 79 us, 0.8 TB/s)
  const long few = std::max(4L, sums_groups(d, g) ? 16L * norm::kThreads / ((long)d.groups * g.tiles) : 65536L / ((long)g.R * (d.c / d.groups)));
  // A thread adds no more than kChain numbers one after another in 32 bits, which lose up to a part in 2^24 each of what is there already: longer runs have more
  // chunks, whose sums are joined in 64 bits.  Where those are more than the work-groups may join themselves, a launch between does it, and nothing limits them
  // (1 x 16500 x 1280 fp16 of 1280 groups in 4 chunks 1430 us, with the launch 46; its gradient 3170 and 67).
  const long least = (g.SR + (long)kChain * g.rpi - 1) / ((long)kChain * g.rpi);
  g.joined = sums_groups(d, g) && least > few;
  const long chunks = std::max({1L, least, std::min({want, most, g.joined ? want : few})});
  g.spc = (int)((g.SR + chunks - 1) / chunks);
  g.spc = (g.spc + g.rpi - 1) / g.rpi * g.rpi;
  g.chunks = (g.SR + g.spc - 1) / g.spc;
  g.lanes = lanes_of(d.groups, norm::kThreads, (backward ? 1L : g.R) * (d.c / d.groups));
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

// A launch holds fewer than 2^32 threads, and places in a superrow are counted in 32 bits.
bool fits(const cprune_norm_desc& d, const NormGeom& g, bool backward) {
  const double vectors = ((long)d.c + 7) / 8;      // work-groups for dweight and dbias
  if (g.nv) return std::max((double)d.n * g.slabs * g.threads, backward && d.n > 1 ? vectors * norm::kThreads : 0.0) < 4294967296.0;
  const double join = sums_groups(d, g) && !g.joined ? 0.0 : (double)d.n * d.groups * join_threads(g, d.c / d.groups);
  return std::max(((double)d.n * g.chunks * g.tiles + vectors) * norm::kThreads, join) < 4294967296.0;
}
// The geometry of a call that has passed check(); false where it is more than the launches hold.
bool plan(const cprune_norm_desc& d, bool backward, NormGeom& g) {
  if (d.c >= 1 << 27 && d.c % (d.dtype == CPRUNE_F32 ? 4 : 8)) return false;      // (split, so its vectors are too many; a superrow might pass 2^31)
  g = geometry(d, backward);
  return fits(d, g, backward);
}

size_t round16(size_t b) { return (b + 15) & ~(size_t)15; }
// Scratch, as far as a form needs each: sums of elements, sums of groups, statistics or means of (image, group).
struct NormScratch {
  size_t part, gpart, stats;
  size_t total() const { return part + gpart + stats; }
};
NormScratch scratch_of(const cprune_norm_desc& d, const NormGeom& g, bool backward) {
  const size_t pair = sizeof(float2);
  NormScratch q = {};
  if (g.nv) {
    if (backward && d.n > 1) q.part = round16((size_t)d.n * d.c * pair);
    return q;
  }
  const bool groups = sums_groups(d, g);
  if (backward || !groups) q.part = round16((size_t)d.n * g.chunks * (g.tiles > 1 ? g.R : 1) * d.c * pair);
  if (groups) q.gpart = (size_t)d.n * g.chunks * g.tiles * d.groups * sizeof(double2);
  if (!groups || g.joined) q.stats = round16((size_t)d.n * d.groups * pair);
  return q;
}

NormArgs args_of(const cprune_norm_desc& d, const NormGeom& g) {
  NormArgs a = {};
  a.pixels = d.pixels, a.c = d.c, a.groups = d.groups, a.cg = d.c / d.groups;
  a.x_image = (long)d.pixels * d.x_stride, a.x_pitch = (long)g.R * d.x_stride;
  a.dy_image = (long)d.pixels * d.dy_stride, a.dy_pitch = (long)g.R * d.dy_stride;
  const float open = std::numeric_limits<float>::quiet_NaN();
  a.lo = d.act == CPRUNE_ACT_NONE ? open : 0.0f;
  a.hi = d.act == CPRUNE_ACT_RELU6 ? 6.0f : open;
  a.n = d.n, a.eps = d.eps;
  a.by_cg = norm_div(a.cg, a.c);
  a.inv_count = 1.0 / ((double)d.pixels * a.cg);
  a.g = g;
  return a;
}

void launch(int dtype, NormPass pass, const NormArgs& a, const NormLaunch& l, hipStream_t s) {
  if (dtype == CPRUNE_F32) launch_norm_f32(pass, a, l, s);
  else if (dtype == CPRUNE_F16) launch_norm_f16(pass, a, l, s);
  else launch_norm_bf16(pass, a, l, s);
}

NormLaunch launch_of(const cprune_norm_desc& d, const NormArgs& a, bool backward) {
  const NormGeom& g = a.g;
  NormLaunch l = {};
  l.silu = d.act == CPRUNE_ACT_SILU;
  // A map that does not stay in the last-level cache (256 MB, shared with what else is in use) is stored past it: kept there, it leaves while the next
  // launch reads (64 x 112 x 112 x 96 fp16 107 -> 93 us, the gradient of 64 x 56 x 56 x 144 59 -> 56; 58 MB forward no difference).
  l.stream = (backward ? 3.0 : 2.0) * d.n * d.pixels * d.c * dtype_size(d.dtype) > 134217728.0;
  if (backward && (a.dweight || a.dbias)) l.vector_groups = (unsigned)(d.c + 7) / 8;
  if (g.nv) {
    l.grid = (unsigned)(d.n * g.slabs);
    const int cols = g.tp * g.V;
    const size_t pairs = backward ? std::max(g.V * g.threads / 2, cols + g.groups) : (a.cg % g.V == 0 ? g.tp : cols) * g.rpi + g.groups;
    l.lds = (unsigned)(pairs * sizeof(float2));
  } else {
    if (sums_groups(d, g)) l.lds = (unsigned)(d.groups * sizeof(float2));
    l.grid = (unsigned)(d.n * g.chunks * g.tiles);
  }
  return l;
}

}  // namespace
}  // namespace cprune

using namespace cprune;

extern "C" size_t cprune_group_norm_workspace_bytes(const cprune_norm_desc* d, int backward) {
  NormGeom g;
  if (check(d, backward != 0) != CPRUNE_OK || !plan(*d, backward != 0, g)) return 0;
  return scratch_of(*d, g, backward != 0).total();
}

extern "C" int cprune_group_norm_act(const cprune_norm_desc* d, const void* x, const float* weight, const float* bias, void* y,
                                     float* mean_out, float* rstd_out, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check(d, false);
  if (rc != CPRUNE_OK) return rc;
  if (!x || !y) return CPRUNE_ERR_INVALID_ARG;
  NormGeom g;
  if (!plan(*d, false, g)) return CPRUNE_ERR_UNSUPPORTED;
  const NormScratch q = scratch_of(*d, g, false);
  if (q.total() && (!ws || ws_bytes < q.total())) return CPRUNE_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(ws) & 15) return CPRUNE_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  NormArgs a = args_of(*d, g);
  a.x = x, a.y = y, a.weight = weight, a.bias = bias;
  a.mean_out = mean_out, a.rstd_out = rstd_out;
  const NormLaunch l = launch_of(*d, a, false);
  char* const scratch = static_cast<char*>(ws);
  if (g.nv) {
    launch(d->dtype, kNormWhole, a, l, s);
  } else {
    if (q.gpart) a.gpart = reinterpret_cast<double2*>(scratch);
    else a.part = reinterpret_cast<float2*>(scratch);
    launch(d->dtype, kNormStats, a, l, s);
    if (q.stats) {
      float* stats = reinterpret_cast<float*>(scratch + q.part + q.gpart);
      float* mean = mean_out ? mean_out : stats;
      float* rstd = rstd_out ? rstd_out : stats + (size_t)d->n * d->groups;
      if (g.joined) norm_join_groups_kernel<false><<<d->n * d->groups, join_threads(g, a.cg), 0, s>>>(a, mean, rstd, nullptr);
      else norm_join_stats_kernel<<<d->n * d->groups, join_threads(g, a.cg), 0, s>>>(a, mean, rstd);
      a.mean = mean, a.rstd = rstd, a.gpart = nullptr;
    }
    launch(d->dtype, kNormApply, a, l, s);
  }
  CPRUNE_LAUNCH_CHECK();
  return CPRUNE_OK;
}

extern "C" int cprune_group_norm_act_backward(const cprune_norm_desc* d, const void* dy, const void* x, const float* mean,
                                              const float* rstd, const float* weight, const float* bias, void* dx, float* dweight,
                                              float* dbias, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check(d, true);
  if (rc != CPRUNE_OK) return rc;
  if (!dy || !x || !mean || !rstd || !dx) return CPRUNE_ERR_INVALID_ARG;
  NormGeom g;
  if (!plan(*d, true, g)) return CPRUNE_ERR_UNSUPPORTED;
  const NormScratch q = scratch_of(*d, g, true);
  if (q.total() && (!ws || ws_bytes < q.total())) return CPRUNE_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(ws) & 15) return CPRUNE_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  NormArgs a = args_of(*d, g);
  a.x = x, a.dy = dy, a.y = dx, a.weight = weight, a.bias = bias, a.mean = mean, a.rstd = rstd;
  a.dweight = dweight, a.dbias = dbias;
  a.part = static_cast<float2*>(ws);
  const NormLaunch l = launch_of(*d, a, true);
  if (g.nv) {
    launch(d->dtype, kNormWholeGrad, a, l, s);
    if (l.vector_groups && d->n > 1) norm_vectors_kernel<<<l.vector_groups, norm::kThreads, 0, s>>>(a);
  } else {
    char* const behind = static_cast<char*>(ws) + q.part;
    float2* const terms = reinterpret_cast<float2*>(behind + q.gpart);
    if (q.gpart) a.gpart = reinterpret_cast<double2*>(behind);
    a.terms = terms;
    launch(d->dtype, kNormGradSums, a, l, s);
    if (g.joined) norm_join_groups_kernel<true><<<d->n * d->groups, join_threads(g, a.cg), 0, s>>>(a, nullptr, nullptr, terms);
    else if (!q.gpart) norm_join_grads_kernel<<<d->n * d->groups, join_threads(g, a.cg), 0, s>>>(a, terms);
    if (g.joined) a.gpart = nullptr;
    launch(d->dtype, kNormGradApply, a, l, s);
  }
  CPRUNE_LAUNCH_CHECK();
  return CPRUNE_OK;
}
