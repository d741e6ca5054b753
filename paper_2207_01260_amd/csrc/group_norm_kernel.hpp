// Group norm with an activation, channels last, and its gradient.
//
// The lanes of a map.  x is [n][pixels][c]; a thread reads V numbers (16 bytes) at a time and keeps the channels it reads for the whole
// kernel, so that what belongs to a channel (weight, bias, statistics, sums) stays in registers.  Where V does not divide c and pixels lie
// without gaps, a "superrow" of R = V / gcd(V, c) pixels is P = R c / V whole vectors; its element q is channel q mod c, and it
// comes back every superrow.  83 channels of fp32: R = 4, P = 83.  Maps with gaps between pixels: R = 1 and the largest V that divides c.
// A work-group is `rpi` superrows of `tp` vectors.  The last superrow of an image may hold fewer than R pixels: its elements are checked one by one.  No
// alignment is assumed (loads of 16 bytes may begin at any element).
//
// Two forms, chosen by what an image's channels take:
//  - whole: a work-group holds all pixels of some whole groups' channels in registers, so x is read once, in one launch (two for the gradient);
//  - split: work-groups walk over runs ("chunks") of superrows of an image, leaving sums for each group; a second launch joins an image's sums where
//    it needs them and reads x again.  Where a superrow is wider than a work-group and groups are many, sums are left for each of its elements and a launch
//    between joins them; one joins the sums of groups where many groups have many chunks.
#pragma once
#include <type_traits>

#include "common.hpp"

namespace cprune {

// Division of numbers below `limit` by d: the high half of a product where that is exact (n d < 2^32), the instruction sequence otherwise.
struct NormDiv {
  unsigned d, magic;
};
inline NormDiv norm_div(long d, long limit) { return {(unsigned)d, d > 1 && limit * d < (1l << 32) ? (unsigned)(((1l << 32) + d - 1) / d) : 0u}; }

struct NormGeom {
  int V, R, P;         // as above
  int tp, tiles, rpi;  // vectors of a superrow a work-group takes, work-groups side by side, superrows at a time
  int threads;
  int SR, spc, chunks;  // superrows of an image, of a chunk; chunks of an image
  int tail;             // pixels of the last superrow
  NormDiv by_tp;        // of a thread's number
  int few, more, last_r;   // whole form: superrows of a thread, one more for r < more; the r that has the last one
  int slabs, nv;        // whole form: work-groups an image (of tp vectors a superrow each), vectors a thread holds
  int groups, lanes;    // groups of a slab; threads that sum one, a power of two
  bool joined;          // split form: a launch between joins the work-groups' sums of groups
};

constexpr int kNormWholeVectors = 16, kNormWholeGradVectors = 8;      // a thread of the whole form holds at most, of x or of x and dy each

struct NormArgs {
  const void *x, *dy;
  const float *weight, *bias;
  const float *mean, *rstd;   // [n][g]; forward: where gpart is null
  const float2* terms;        // backward: (mean(w dz), mean(w dz xhat)) [n][g]
  float *mean_out, *rstd_out; // whole form, or null
  float eps;
  float *dweight, *dbias;     // backward, or null
  int n;
  void* y;                    // forward: y, backward: dx
  float2* part;               // sums of channels or of a superrow's elements: forward (mean, squares about it), backward (sum dz, sum dz xhat)
  double2* gpart;             // split form, sums of groups [n][chunk][tile][group]: forward (numbers, their squares), backward weighted; or null
  int pixels, c, cg, groups;
  NormDiv by_cg;              // of a channel
  double inv_count;           // 1 / (numbers of an (image, group))
  long x_image, x_pitch, dy_image, dy_pitch;   // elements from image to image, from superrow to superrow
  float lo, hi;               // clamp of the activation; NaN where there is none: no number is past it, no infinity at it
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
  Raw r = B(0);
  if (valid <= 0) return r;
  // (the last one again where there is none: loads that wait for nothing, a branch each would have them one by one)
#pragma unroll
  for (int j = 0; j < V; ++j) r[j] = static_cast<const B*>(p)[min(j, valid - 1)];
#pragma unroll
  for (int j = 0; j < V; ++j) r[j] = j < valid ? r[j] : B(0);
  return r;
}
// STREAM: past the caches, for a map that would only push itself out of them
template <typename T, int V, bool STREAM = false> __device__ __forceinline__ void store(void* p, const float (&v)[V], int valid) {
  typedef typename Bits<T>::type B;
  typedef typename RawOf<B, V>::type Raw;
  Raw r;
#pragma unroll
  for (int j = 0; j < V; ++j) r[j] = narrow<T>(v[j]);
  if (V == 1 || valid >= V) {
    if constexpr (STREAM) __builtin_nontemporal_store(r, static_cast<Raw*>(p));
    else *static_cast<Raw*>(p) = r;
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (j < valid) static_cast<B*>(p)[j] = r[j];
  }
}

// 1 / (1 + e^-z) on the bare instruction for 2^x (the exponential of the library mends results below 2^-126, which 1 + e^-z does not see); its
// overflow at very negative z gives z * 0
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f)); }
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
// depend on which products and sums the compiler joins.  (The forward pass has weight * rstd as one factor and one rounding less, so that within a few roundings
// of a kink a clamped output may have a gradient, or one that is not clamped none.)
__device__ __forceinline__ float centred(float x, float mean, float rstd) {
#pragma clang fp contract(off)
  return (x - mean) * rstd;
}
__device__ __forceinline__ float argument(float xhat, float w, float b) {
#pragma clang fp contract(off)
  const float p = xhat * w;
  return p + b;
}

__device__ __forceinline__ int quotient(int n, const NormDiv& d) { return d.magic ? (int)__umulhi((unsigned)n, d.magic) : d.d == 1 ? n : (int)((unsigned)n / d.d); }

// What a thread works on: vector p of the superrows sr0 + r, sr0 + r + rpi, ... below sr1.
struct Place {
  int image, part, r, p, sr0, sr1;      // part: chunk or slab
  bool active;
};
__device__ __forceinline__ Place place(const NormGeom& g, unsigned block) {
  Place k;
  const int tile = (int)(block % (unsigned)g.tiles);
  block /= (unsigned)g.tiles;
  k.part = (int)(block % (unsigned)g.chunks);
  k.image = (int)(block / (unsigned)g.chunks);
  k.r = quotient((int)threadIdx.x, g.by_tp);
  k.p = tile * g.tp + ((int)threadIdx.x - k.r * g.tp);
  k.active = k.r < g.rpi && k.p < g.P;
  k.sr0 = k.part * g.spc;
  k.sr1 = min(g.SR, k.sr0 + g.spc);
  return k;
}
// Whole form.  Work-groups next to each other run on different XCDs; each XCD gets a run of (image, slab), so that slabs of an image, which share
// cache lines where a slab is narrower than one, share an L2.
__device__ __forceinline__ Place place_whole(const NormGeom& g) {
  Place k;
  const unsigned total = gridDim.x, xcd = blockIdx.x & 7, per = total >> 3, rest = total & 7;
  const unsigned t = xcd * per + min(xcd, rest) + (blockIdx.x >> 3);
  k.image = (int)(t / (unsigned)g.slabs);
  k.part = (int)t - k.image * g.slabs;
  k.r = quotient((int)threadIdx.x, g.by_tp);
  const int q = (int)threadIdx.x - k.r * g.tp;
  k.p = k.part * g.tp + q;
  k.active = k.r < g.rpi;
  k.sr0 = 0;
  k.sr1 = g.SR;
  return k;
}
// elements of the vector at position p that superrow sr has
__device__ __forceinline__ int valid_of(const NormGeom& g, int c, int sr, int p) {
  return sr == g.SR - 1 ? g.tail * c - p * g.V : g.V;
}
// superrows below which every element is there
__device__ __forceinline__ int full_rows(const NormGeom& g) { return g.tail == g.R ? g.SR : g.SR - 1; }

constexpr int kThreads = 256;
// The split form's loops: `whole` batches of vectors and one of what is left, the loads of a batch ahead of the work on the one before.
// The caller has fetched the first one into `a`.
template <typename Batch, typename Fetch, typename Work, typename Rest> __device__ __forceinline__ void walk(Batch& a, int whole, Fetch&& fetch, Work&& work, Rest&& rest) {
  Batch b;
  for (int i = 0;; i += 2) {
    if (i == whole) return rest(a);
    fetch(b, i + 1);
    work(a);
    if (i + 1 == whole) return rest(b);
    fetch(a, i + 2);
    work(b);
  }
}
// vectors of a batch, of x alone and of x and dy
constexpr int kBatch = 4, kGradBatch = 2;

// Sum of a pair over the superrows of a work-group, in threads of r = 0; buffer: V * threads / 2 pairs.  The upper half hands over to the lower one,
// halving: a fixed order.
template <int V> __device__ __forceinline__ void add_rows(float (&a)[V], float (&b)[V], int r, int tp, int rpi, bool active, float2* buffer) {
  int half = 1;
  while (2 * half < rpi) half *= 2;
  const int stride = tp * max(rpi - half, half >> 1), t = (int)threadIdx.x;      // (threads that hand over, at most half of them)
  if (rpi == 1) return;
  for (int live = rpi; half > 0; live = half, half >>= 1) {
    const bool gives = active && r >= half && r < live, takes = active && r < half && r + half < live;
    if (gives) {
#pragma unroll
      for (int j = 0; j < V; ++j) buffer[j * stride + t - half * tp] = make_float2(a[j], b[j]);
    }
    __syncthreads();
    if (takes) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float2 o = buffer[j * stride + t];
        a[j] += o.x, b[j] += o.y;
      }
    }
    __syncthreads();
  }
}

// channels and groups of a vector's elements, which begin at element q of a superrow: one division, then counted on
template <int V> struct Where {
  int ch[V], group[V];
};
template <int V> __device__ __forceinline__ Where<V> where(const NormArgs& a, int q) {
  Where<V> k;
  int ch = a.g.R == 1 ? q : q % a.c, group = quotient(ch, a.by_cg), left = a.cg - (ch - group * a.cg);      // (left: channels of the group from here on)
#pragma unroll
  for (int j = 0; j < V; ++j) {
    k.ch[j] = ch, k.group[j] = group;
    ++ch;
    if (--left == 0) {
      left = a.cg, ++group;
      if (ch == a.c) ch = 0, group = 0;
    }
  }
  return k;
}

// weight, bias and statistics of a vector's elements
template <int V> struct Terms {
  float mean[V], rstd[V], w[V], b[V];
};
// A vector's channels follow each other, unless a superrow's next pixel begins in it: their terms are 16-byte loads, one each for what a group shares.  (A load of
// each by itself, 32 of them for eight elements, is a microsecond or two of a work-group.)
template <int V> __device__ __forceinline__ void channel_values(const float* from, float without, const Where<V>& at, float (&v)[V]) {
  if (!from) {
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = without;
  } else if (at.ch[V - 1] - at.ch[0] == V - 1) {
    constexpr int W = V < 4 ? V : 4;
    typedef typename RawOf<float, W>::type Some;
#pragma unroll
    for (int h = 0; h < V; h += W) {
      const Some q = *reinterpret_cast<const Some*>(from + at.ch[0] + h);
#pragma unroll
      for (int j = 0; j < W; ++j) v[h + j] = q[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = from[at.ch[j]];
  }
}
template <int V> __device__ __forceinline__ void channel_terms(const NormArgs& a, const Where<V>& at, Terms<V>& k) {
  channel_values<V>(a.weight, 1.0f, at, k.w);
  channel_values<V>(a.bias, 0.0f, at, k.b);
}
template <int V> __device__ __forceinline__ void all_terms(const NormArgs& a, int image, const Where<V>& at, Terms<V>& k) {
  channel_terms<V>(a, at, k);
  const float *const mean = a.mean + image * a.groups, *const rstd = a.rstd + image * a.groups;
  if (at.group[V - 1] == at.group[0] && at.ch[V - 1] - at.ch[0] == V - 1) {      // (past a pixel's end the last may be of the first one's group again, others between)
    const float m = mean[at.group[0]], r = rstd[at.group[0]];
#pragma unroll
    for (int j = 0; j < V; ++j) k.mean[j] = m, k.rstd[j] = r;
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) k.mean[j] = mean[at.group[j]], k.rstd[j] = rstd[at.group[j]];
  }
}

// mean and rstd from the sums of the numbers and of their squares (in 64 bits: the difference below loses what (mean / spread)^2 takes of 53 bits)
__device__ __forceinline__ float2 statistics(double2 s, const NormArgs& a) {
  const double mean = s.x * a.inv_count, var = s.y * a.inv_count - mean * mean;
  return make_float2((float)mean, 1.0f / sqrtf((var < 0.0 ? 0.0f : (float)var) + a.eps));
}

// a vector of outputs; k.w holds weight * rstd
template <typename T, int V, bool SILU, bool STREAM, typename Raw>
__device__ __forceinline__ void normalise(const NormArgs& a, const Raw& raw, const Terms<V>& k, char* out, int valid) {
  float v[V];
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = activate<SILU>(fmaf(widen<T>(raw[j]) - k.mean[j], k.w[j], k.b[j]), a.lo, a.hi);
  store<T, V, STREAM>(out, v, valid);
}
template <typename T, int V, bool SILU, bool STREAM, typename Raw>
__device__ __forceinline__ void gradient(const NormArgs& a, const Raw& x, const Raw& dy, const Terms<V>& k, const float2 (&t)[V], char* out, int valid) {
  float v[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const float xhat = centred(widen<T>(x[j]), k.mean[j], k.rstd[j]);
    const float dz = widen<T>(dy[j]) * slope<SILU>(argument(xhat, k.w[j], k.b[j]), a.lo, a.hi);
    v[j] = k.rstd[j] * (fmaf(k.w[j], dz, -t[j].x) - xhat * t[j].y);
  }
  store<T, V, STREAM>(out, v, valid);
}
template <typename T, int V, bool SILU, typename Raw>
__device__ __forceinline__ void gradient_sums(const NormArgs& a, const Raw& x, const Raw& dy, const Terms<V>& k, float (&sb)[V], float (&sw)[V], int valid) {
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const float xhat = centred(widen<T>(x[j]), k.mean[j], k.rstd[j]);
    const float dz = widen<T>(dy[j]) * slope<SILU>(argument(xhat, k.w[j], k.b[j]), a.lo, a.hi);
    if (j < valid) {      // (elements past the image: zeros may still have a slope)
      sb[j] += dz;
      sw[j] = fmaf(dz, xhat, sw[j]);
    }
  }
}

// The sum over neighbouring lanes, a power of two of them up to 64, in every one of them.
template <int CTRL> __device__ __forceinline__ double from_lane(double v) {
  const long long b = __double_as_longlong(v);
  const unsigned lo = (unsigned)__builtin_amdgcn_mov_dpp((int)b, CTRL, 0xF, 0xF, true), hi = (unsigned)__builtin_amdgcn_mov_dpp((int)(b >> 32), CTRL, 0xF, 0xF, true);
  return __longlong_as_double((long long)hi << 32 | lo);
}
__device__ __forceinline__ double2 sum_lanes(double2 s, int lanes) {
  if (lanes > 1) s.x += from_lane<0xB1>(s.x), s.y += from_lane<0xB1>(s.y);          // the other of a pair
  if (lanes > 2) s.x += from_lane<0x4E>(s.x), s.y += from_lane<0x4E>(s.y);          // the other pair of a quad
  if (lanes > 4) s.x += from_lane<0x141>(s.x), s.y += from_lane<0x141>(s.y);        // mirrored in eight
  if (lanes > 8) s.x += from_lane<0x140>(s.x), s.y += from_lane<0x140>(s.y);        // mirrored in sixteen
  if (lanes > 16) s.x += __shfl_xor(s.x, 16, 64), s.y += __shfl_xor(s.y, 16, 64);
  if (lanes > 32) s.x += __shfl_xor(s.x, 32, 64), s.y += __shfl_xor(s.y, 32, 64);
  return s;
}

// Sum over a group's `outer` x `inner` entries of pairs add(outer, inner, get(outer, inner)), in 64 bits and a fixed order, by `lanes` neighbouring lanes; all
// of them get it.  U entries are under way at a time; a lane counts its place on instead of dividing.
template <int U, typename Get, typename Add> __device__ __forceinline__ double2 lanes_sum(int lane, int lanes, int outer, int inner, Get&& get, Add&& add) {
  double2 s = {0.0, 0.0};
  const int skip = lanes / inner, step = lanes - skip * inner;
  int o = lane / inner, in = lane - o * inner;
  while (o < outer) {
    decltype(get(0, 0)) e[U];
    int at[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      at[u][0] = o, at[u][1] = in;
      if (o < outer) e[u] = get(o, in);
      o += skip, in += step;
      if (in >= inner) in -= inner, ++o;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (at[u][0] < outer) {
        const double2 v = add(at[u][0], at[u][1], e[u]);
        s.x += v.x, s.y += v.y;
      }
  }
  return sum_lanes(s, lanes);
}

// done(group, sum) for each of a work-group's groups, by one thread; sum(group, lane) is what a lane's wavefront (or less, where lanes are fewer) has of it.  More
// than a wavefront's lanes, where there are few groups: their sums are joined through LDS, in a fixed order.  All threads call it; it ends without a barrier.
template <typename Sum, typename Done> __device__ __forceinline__ void each_group(int lanes, int groups, Sum&& sum, Done&& done) {
  const int t = (int)threadIdx.x, lane = t & (lanes - 1);
  if (lanes <= 64) {
    const int per = (int)blockDim.x / lanes;
    for (int g = t / lanes; g < groups; g += per) {
      const double2 s = sum(g, lane);
      if (lane == 0) done(g, s);
    }
    return;
  }
  __shared__ double2 waves[1024 / 64];
  const int mine = t / lanes, each = lanes / 64;
  if (mine < groups) {
    const double2 s = sum(mine, lane);
    if ((t & 63) == 0) waves[t >> 6] = s;
  }
  __syncthreads();
  if (t < groups) {
    double2 s = waves[t * each];
    for (int i = 1; i < each; ++i) s.x += waves[t * each + i].x, s.y += waves[t * each + i].y;
    done(t, s);
  }
}

// sums of n numbers and of their squares from their (mean, squares about it)
__device__ __forceinline__ double2 raw_sums(double n, float2 e) {
  const double nm = n * e.x;
  return n > 0.0 ? make_double2(nm, (double)e.y + nm * e.x) : make_double2(0.0, 0.0);
}

// The sums of dz and dz xhat of a superrow's elements (LDS) as those of its channels, which go to out(channel, sums), and with weights in their place in LDS:
// a thread a channel, so that a weight is loaded once.  All threads call it; ch0 is the first of the `channels`.
template <typename Out> __device__ __forceinline__ void fold_columns(const NormArgs& a, float2* col, int channels, int ch0, Out&& out) {
  __syncthreads();
  for (int ch = threadIdx.x; ch < channels; ch += (int)blockDim.x) {
    const float w = a.weight ? a.weight[ch0 + ch] : 1.0f;
    float2 s = col[ch];
    for (int rr = 1; rr < a.g.R; ++rr) s.x += col[rr * a.c + ch].x, s.y += col[rr * a.c + ch].y;
    out(ch, s);
    col[ch] = make_float2(w * s.x, w * s.y);
  }
  __syncthreads();
}
// The sum of add(place in the tile, ...) over the elements of group g that a work-group's tile of the superrow has, `count` of them from element q0 on.
template <typename At> __device__ __forceinline__ double2 tile_sum(const NormArgs& a, int lane, int lanes, int g, int q0, int count, At&& at) {
  double2 s = {0.0, 0.0};
  for (int rr = 0; rr < a.g.R; ++rr) {
    const int base = rr * a.c + g * a.cg - q0, end = min(base + a.cg, count);
    for (int e = max(base, 0) + lane; e < end; e += lanes) {
      const double2 v = at(e);
      s.x += v.x, s.y += v.y;
    }
  }
  return sum_lanes(s, lanes);
}
// Their sum over group g.
__device__ __forceinline__ double2 group_terms(const NormArgs& a, const float2* col, int lane, int lanes, int g) {
  return lanes_sum<4>(
      lane, lanes, a.cg, 1, [&](int ch, int) __attribute__((always_inline)) { return col[g * a.cg + ch]; },
      [&](int, int, float2 e) __attribute__((always_inline)) { return make_double2(e.x, e.y); });
}

}  // namespace norm

// ---- split form ----------------------------------------------------------------------------------

// Statistics of a chunk: each thread's running mean and squares about it, four numbers at a time about their own mean (no difference of large sums, whatever
// the numbers' mean), then joined over the work-group's superrows pair by pair, and as sums of groups in 64 bits.  Bound by memory on large maps: 64 x 112 x 112
// x 96 fp16, 154 MB read, 29.7 us, 5.2 TB/s; on small ones by the chain load, sum, LDS, store (1 x 112 x 112 x 96 some 6 us).
template <typename T, int V>
__global__ __launch_bounds__(norm::kThreads, 4) void norm_stats_kernel(const NormArgs a) {
  using namespace norm;
  constexpr int U = kBatch;
  __shared__ float s_mean[V][kThreads], s_sq[V][kThreads], s_n[V][kThreads];
  const Place k = place(a.g, blockIdx.x);
  float mean[V], sq[V], cnt[V];
#pragma unroll
  for (int j = 0; j < V; ++j) mean[j] = sq[j] = 0.0f;
  float n = 0.0f;
  int missing = V;      // elements from this one on lack the last vector
  if (k.active) {
    const char* base = static_cast<const char*>(a.x) + (k.image * a.x_image + (long)k.p * V) * (long)sizeof(T);
    const long pitch = a.x_pitch * (long)sizeof(T);
    const int step = a.g.rpi, full = min(k.sr1, full_rows(a.g));
    auto one = [&](const auto& raw, int valid) __attribute__((always_inline)) {
      n += 1.0f;
      const float rc = __builtin_amdgcn_rcpf(n);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (j < valid) {
          const float v = widen<T>(raw[j]), d = v - mean[j];
          mean[j] = fmaf(d, rc, mean[j]);
          sq[j] = fmaf(d, v - mean[j], sq[j]);
        }
      }
    };
    struct Batch {
      typename RawOf<typename Bits<T>::type, V>::type raw[U];
    };
    const int sr = k.sr0 + k.r, whole = max(full - k.sr0, 0) / (U * step);
    auto fetch = [&](Batch& q, int i) __attribute__((always_inline)) {
      const int at = sr + i * U * step;
      if (i < whole) {
#pragma unroll
        for (int u = 0; u < U; ++u) q.raw[u] = load<T, V>(base + (at + u * step) * pitch, V);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (at + u * step < full) q.raw[u] = load<T, V>(base + (at + u * step) * pitch, V);
      }
    };
    Batch head;
    fetch(head, 0);
    walk(
        head, whole, fetch,
        [&](const Batch& q) __attribute__((always_inline)) {
          const float f = (float)U * __builtin_amdgcn_rcpf(n + (float)U), nf = n * f;
#pragma unroll
          for (int j = 0; j < V; ++j) {
            float m = 0.0f, sum = 0.0f;
#pragma unroll
            for (int u = 0; u < U; ++u) m += widen<T>(q.raw[u][j]);
            m *= 1.0f / U;
#pragma unroll
            for (int u = 0; u < U; ++u) {
              const float d = widen<T>(q.raw[u][j]) - m;
              sum = fmaf(d, d, sum);
            }
            const float d = m - mean[j];
            mean[j] = fmaf(d, f, mean[j]);
            sq[j] += fmaf(d * d, nf, sum);
          }
          n += (float)U;
        },
        [&](const Batch& q) __attribute__((always_inline)) {
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (sr + (whole * U + u) * step < full) one(q.raw[u], V);
        });
    const int end = a.g.SR - 1, valid = valid_of(a.g, a.c, end, k.p);
    if (full < k.sr1 && (unsigned)(end - k.sr0) % (unsigned)step == (unsigned)k.r && valid > 0) {
      one(load<T, V>(base + end * pitch, valid), valid);
      missing = valid;
    }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) cnt[j] = j < missing ? n : n - 1.0f;
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
        const float nb = s_n[j][o], sum = cnt[j] + nb;
        if (nb > 0.0f) {
          const float d = s_mean[j][o] - mean[j], f = nb * __builtin_amdgcn_rcpf(sum);
          mean[j] = fmaf(d, f, mean[j]);
          sq[j] += s_sq[j][o] + d * d * cnt[j] * f;
          cnt[j] = sum;
        }
        s_mean[j][t] = mean[j], s_sq[j][t] = sq[j], s_n[j][t] = cnt[j];
      }
    }
  }
  if (!a.gpart) {
    if (k.active && k.r == 0) {
      float2* out = a.part + ((long)k.image * a.g.chunks + k.part) * a.g.P * V + (long)k.p * V;
#pragma unroll
      for (int j = 0; j < V; ++j) out[j] = make_float2(mean[j], sq[j]);
    }
    return;
  }
  __syncthreads();
  // the tile's elements as groups
  const int lanes = a.g.lanes;
  const int p0 = k.p - (t - k.r * a.g.tp), count = min(a.g.tp, a.g.P - p0) * V;
  double2* const out = a.gpart + (((long)k.image * a.g.chunks + k.part) * a.g.tiles + p0 / a.g.tp) * a.groups;
  each_group(
      lanes, a.groups,
      [&](int g, int lane) __attribute__((always_inline)) {
        return tile_sum(a, lane, lanes, g, p0 * V, count, [&](int e) __attribute__((always_inline)) {
          return raw_sums(s_n[e % V][e / V], make_float2(s_mean[e % V][e / V], s_sq[e % V][e / V]));
        });
      },
      [&](int g, double2 s) __attribute__((always_inline)) { out[g] = s; });
}

// The second pass: an image's statistics from its work-groups' sums (each work-group for itself: a launch between costs more than reading some KB again), then y.
// Its first loads are under way meanwhile.  64 x 112 x 112 x 96 fp16, 308 MB read and written, 56.6 us, 5.4 TB/s.
template <typename T, int V, bool SILU, bool STREAM>
__global__ __launch_bounds__(norm::kThreads, 4) void norm_apply_kernel(const NormArgs a) {
  using namespace norm;
  constexpr int U = kBatch;
  extern __shared__ char lds[];
  float2* const stat = reinterpret_cast<float2*>(lds);      // [group]: (mean, rstd), where sums are a group's
  const Place k = place(a.g, blockIdx.x);
  const char* base = static_cast<const char*>(a.x) + (k.image * a.x_image + (long)k.p * V) * (long)sizeof(T);
  char* out = static_cast<char*>(a.y) + ((long)k.image * a.pixels * a.c + (long)k.p * V) * (long)sizeof(T);
  const long pitch = a.x_pitch * (long)sizeof(T), out_pitch = (long)a.g.P * V * (long)sizeof(T);
  const int step = a.g.rpi, full = min(k.sr1, full_rows(a.g));
  struct Batch {
    typename RawOf<typename Bits<T>::type, V>::type raw[U];
  };
  const int sr = k.sr0 + k.r, whole = max(full - k.sr0, 0) / (U * step);
  auto fetch = [&](Batch& q, int i) __attribute__((always_inline)) {
    const int at = sr + i * U * step;
    if (i < whole) {
#pragma unroll
      for (int u = 0; u < U; ++u) q.raw[u] = load<T, V>(base + (at + u * step) * pitch, V);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int valid = at + u * step < k.sr1 ? valid_of(a.g, a.c, at + u * step, k.p) : 0;
        if (valid > 0) q.raw[u] = load<T, V>(base + (at + u * step) * pitch, valid);
      }
    }
  };
  // (what does not wait for the image's statistics is under way before they are joined)
  Batch head;
  Terms<V> c;
  Where<V> here;
  if (k.active) {
    fetch(head, 0);
    here = where<V>(a, k.p * V);
    channel_terms<V>(a, here, c);
  }
  if (a.gpart) {
    const int lanes = a.g.lanes;
    const double2* const part = a.gpart + (long)k.image * a.g.chunks * a.g.tiles * a.groups;
    each_group(
        lanes, a.groups,
        [&](int g, int lane) __attribute__((always_inline)) {
          return lanes_sum<8>(
              lane, lanes, a.g.chunks * a.g.tiles, 1, [&](int i, int) __attribute__((always_inline)) { return part[i * a.groups + g]; },
              [&](int, int, double2 e) __attribute__((always_inline)) { return e; });
        },
        [&](int g, double2 s) __attribute__((always_inline)) {
          const float2 m = statistics(s, a);
          stat[g] = m;
          if (k.part == 0 && a.mean_out) a.mean_out[k.image * a.groups + g] = m.x;      // (each tile the same)
          if (k.part == 0 && a.rstd_out) a.rstd_out[k.image * a.groups + g] = m.y;
        });
    __syncthreads();
  }
  if (!k.active) return;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int at = k.image * a.groups + here.group[j];
    const float2 m = a.gpart ? stat[here.group[j]] : make_float2(a.mean[at], a.rstd[at]);
    c.mean[j] = m.x;
    c.w[j] *= m.y;
  }
  int at = sr;
  walk(
      head, whole, fetch,
      [&](const Batch& q) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u, at += step) normalise<T, V, SILU, STREAM>(a, q.raw[u], c, out + at * out_pitch, V);
      },
      [&](const Batch& q) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u, at += step) {
          const int valid = at < k.sr1 ? valid_of(a.g, a.c, at, k.p) : 0;
          if (valid > 0) normalise<T, V, SILU, STREAM>(a, q.raw[u], c, out + at * out_pitch, valid);
        }
      });
}

// Sums of dz and dz xhat over a chunk; the activation's argument is worked out again from x, which costs less than a map of it.  64 x 56 x 56 x 144 fp16, 116 MB
// read, 22.1 us, 5.2 TB/s.
template <typename T, int V, bool SILU>
__global__ __launch_bounds__(norm::kThreads, 4) void norm_grad_sums_kernel(const NormArgs a) {
  using namespace norm;
  constexpr int U = kGradBatch;
  __shared__ float2 buffer[V * kThreads];
  const Place k = place(a.g, blockIdx.x);
  float sb[V], sw[V], weight[V];
#pragma unroll
  for (int j = 0; j < V; ++j) sb[j] = sw[j] = 0.0f, weight[j] = 1.0f;
  if (k.active) {
    Terms<V> c;
    const char* xb = static_cast<const char*>(a.x) + (k.image * a.x_image + (long)k.p * V) * (long)sizeof(T);
    const char* db = static_cast<const char*>(a.dy) + (k.image * a.dy_image + (long)k.p * V) * (long)sizeof(T);
    const long pitch = a.x_pitch * (long)sizeof(T), dy_pitch = a.dy_pitch * (long)sizeof(T);
    const int step = a.g.rpi, full = min(k.sr1, full_rows(a.g));
    struct Batch {
      typename RawOf<typename Bits<T>::type, V>::type x[U], dy[U];
    };
    const int sr = k.sr0 + k.r, whole = max(full - k.sr0, 0) / (U * step);
    auto fetch = [&](Batch& q, int i) __attribute__((always_inline)) {
      const int at = sr + i * U * step;
      if (i < whole) {
#pragma unroll
        for (int u = 0; u < U; ++u) q.x[u] = load<T, V>(xb + (at + u * step) * pitch, V), q.dy[u] = load<T, V>(db + (at + u * step) * dy_pitch, V);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int valid = at + u * step < k.sr1 ? valid_of(a.g, a.c, at + u * step, k.p) : 0;
          if (valid > 0) q.x[u] = load<T, V>(xb + (at + u * step) * pitch, valid), q.dy[u] = load<T, V>(db + (at + u * step) * dy_pitch, valid);
        }
      }
    };
    Batch head;
    fetch(head, 0);
    all_terms<V>(a, k.image, where<V>(a, k.p * V), c);
#pragma unroll
    for (int j = 0; j < V; ++j) weight[j] = c.w[j];
    walk(
        head, whole, fetch,
        [&](const Batch& q) __attribute__((always_inline)) {
#pragma unroll
          for (int u = 0; u < U; ++u) gradient_sums<T, V, SILU>(a, q.x[u], q.dy[u], c, sb, sw, V);
        },
        [&](const Batch& q) __attribute__((always_inline)) {
          int at = sr + whole * U * step;
#pragma unroll
          for (int u = 0; u < U; ++u, at += step) {
            const int valid = at < k.sr1 ? valid_of(a.g, a.c, at, k.p) : 0;
            if (valid > 0) gradient_sums<T, V, SILU>(a, q.x[u], q.dy[u], c, sb, sw, valid);
          }
        });
  }
  add_rows<V>(sb, sw, k.r, a.g.tp, a.g.rpi, k.active, buffer);
  // Sums of channels where a work-group has whole superrows, otherwise of their elements.
  const bool whole_rows = a.g.tiles == 1;
  const int p0 = k.p - ((int)threadIdx.x - k.r * a.g.tp), count = min(a.g.tp, a.g.P - p0) * V;
  float2* const part = a.part + ((long)k.image * a.g.chunks + k.part) * (whole_rows ? a.c : a.g.P * V);
  if (k.active && k.r == 0) {
    float2* const out = buffer + (k.p - p0) * V;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (!whole_rows) part[k.p * V + j] = make_float2(sb[j], sw[j]);
      const float w = whole_rows ? 1.0f : weight[j];
      out[j] = make_float2(w * sb[j], w * sw[j]);
    }
  }
  if (!a.gpart) return;
  const int lanes = a.g.lanes;
  double2* const out = a.gpart + (((long)k.image * a.g.chunks + k.part) * a.g.tiles + p0 / a.g.tp) * a.groups;
  if (whole_rows) fold_columns(a, buffer, a.c, 0, [&](int ch, float2 s) __attribute__((always_inline)) { part[ch] = s; });
  else __syncthreads();
  each_group(
      lanes, a.groups,
      [&](int g, int lane) __attribute__((always_inline)) {
        return whole_rows ? group_terms(a, buffer, lane, lanes, g)
                          : tile_sum(a, lane, lanes, g, p0 * V, count, [&](int e) __attribute__((always_inline)) { return make_double2(buffer[e].x, buffer[e].y); });
      },
      [&](int g, double2 s) __attribute__((always_inline)) { out[g] = s; });
}

// dweight and dbias of eight channels from all images' partial sums, `per` rows of c of them an image; 32 threads a channel, 64 bits, a fixed order.
__device__ inline void norm_vector_sums(const NormArgs& a, unsigned block, long count) {
  __shared__ double2 waves[norm::kThreads / 64][8];
  const int t = (int)threadIdx.x, ch = (int)block * 8 + (t & 7), lane = t >> 3;
  double2 s = {0.0, 0.0};
  if (ch < a.c) {
    for (long i = lane; i < count; i += 8 * 32) {
      float2 p[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) p[u] = a.part[min(i + u * 32, count - 1) * a.c + ch];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i + u * 32 < count) s.x += p[u].x, s.y += p[u].y;
    }
  }
#pragma unroll
  for (int o = 8; o < 64; o *= 2) s.x += __shfl_xor(s.x, o, 64), s.y += __shfl_xor(s.y, o, 64);
  if ((t & 63) < 8) waves[t >> 6][t & 7] = s;
  __syncthreads();
  if (t < 8 && ch < a.c) {
    for (int i = 1; i < norm::kThreads / 64; ++i) s.x += waves[i][t].x, s.y += waves[i][t].y;
    if (a.dbias) a.dbias[ch] = (float)s.x;
    if (a.dweight) a.dweight[ch] = (float)s.y;
  }
}

__global__ __launch_bounds__(norm::kThreads) inline void norm_vectors_kernel(const NormArgs a) { norm_vector_sums(a, blockIdx.x, a.n); }

// The first `vector_groups` work-groups sum dweight and dbias (few numbers, long chains: beside the others they cost nothing), the others dx from x and dy again.
// 64 x 56 x 56 x 144 fp16, 173 MB, 29.2 us, 5.9 TB/s.
template <typename T, int V, bool SILU, bool STREAM>
__global__ __launch_bounds__(norm::kThreads, 4) void norm_grad_apply_kernel(const NormArgs a, unsigned vector_groups) {
  using namespace norm;
  constexpr int U = kGradBatch;
  if (blockIdx.x < vector_groups) {
    norm_vector_sums(a, blockIdx.x, (long)a.n * a.g.chunks * (a.g.tiles == 1 ? 1 : a.g.R));
    return;
  }
  extern __shared__ char lds[];
  float2* const term = reinterpret_cast<float2*>(lds);      // [group], where sums are a group's
  const Place k = place(a.g, blockIdx.x - vector_groups);
  const char* xb = static_cast<const char*>(a.x) + (k.image * a.x_image + (long)k.p * V) * (long)sizeof(T);
  const char* db = static_cast<const char*>(a.dy) + (k.image * a.dy_image + (long)k.p * V) * (long)sizeof(T);
  char* out = static_cast<char*>(a.y) + ((long)k.image * a.pixels * a.c + (long)k.p * V) * (long)sizeof(T);
  const long pitch = a.x_pitch * (long)sizeof(T), dy_pitch = a.dy_pitch * (long)sizeof(T), out_pitch = (long)a.g.P * V * (long)sizeof(T);
  const int step = a.g.rpi, full = min(k.sr1, full_rows(a.g));
  struct Batch {
    typename RawOf<typename Bits<T>::type, V>::type x[U], dy[U];
  };
  const int sr = k.sr0 + k.r, whole = max(full - k.sr0, 0) / (U * step);
  auto fetch = [&](Batch& q, int i) __attribute__((always_inline)) {
    const int at = sr + i * U * step;
    if (i < whole) {
#pragma unroll
      for (int u = 0; u < U; ++u) q.x[u] = load<T, V>(xb + (at + u * step) * pitch, V), q.dy[u] = load<T, V>(db + (at + u * step) * dy_pitch, V);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int valid = at + u * step < k.sr1 ? valid_of(a.g, a.c, at + u * step, k.p) : 0;
        if (valid > 0) q.x[u] = load<T, V>(xb + (at + u * step) * pitch, valid), q.dy[u] = load<T, V>(db + (at + u * step) * dy_pitch, valid);
      }
    }
  };
  Batch head;
  Terms<V> c;
  Where<V> here;
  if (k.active) {
    fetch(head, 0);
    here = where<V>(a, k.p * V);
    all_terms<V>(a, k.image, here, c);
  }
  if (a.gpart) {
    const int lanes = a.g.lanes;
    const double2* const part = a.gpart + (long)k.image * a.g.chunks * a.g.tiles * a.groups;
    each_group(
        lanes, a.groups,
        [&](int g, int lane) __attribute__((always_inline)) {
          return lanes_sum<8>(
              lane, lanes, a.g.chunks * a.g.tiles, 1, [&](int i, int) __attribute__((always_inline)) { return part[i * a.groups + g]; },
              [&](int, int, double2 e) __attribute__((always_inline)) { return e; });
        },
        [&](int g, double2 s) __attribute__((always_inline)) {
          term[g] = make_float2((float)(s.x * a.inv_count), (float)(s.y * a.inv_count));
        });
    __syncthreads();
  }
  if (!k.active) return;
  float2 t[V];
#pragma unroll
  for (int j = 0; j < V; ++j) t[j] = a.gpart ? term[here.group[j]] : a.terms[k.image * a.groups + here.group[j]];
  int at = sr;
  walk(
      head, whole, fetch,
      [&](const Batch& q) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u, at += step) gradient<T, V, SILU, STREAM>(a, q.x[u], q.dy[u], c, t, out + at * out_pitch, V);
      },
      [&](const Batch& q) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u, at += step) {
          const int valid = at < k.sr1 ? valid_of(a.g, a.c, at, k.p) : 0;
          if (valid > 0) gradient<T, V, SILU, STREAM>(a, q.x[u], q.dy[u], c, t, out + at * out_pitch, valid);
        }
      });
}

// ---- whole form ----------------------------------------------------------------------------------
// V numbers are 16 bytes; a thread holds NV vectors.  x is read once and y follows from registers; statistics are of the numbers about each thread's own mean, joined
// through LDS.  Bound by that chain, one work-group or two a compute unit: 32 x 56 x 56 x 64 bf16, 26 MB, 15.1 us (in two passes 18.7), 1 x 14 x 14 x 96 fp32 4.9 us.

// What holds of the slab's layout, known when the kernel is built: kMerge, V divides a group's channels, so a thread's numbers are of one group; kTail, the last superrow lacks pixels.
enum NormSlab { kPlain, kMerge, kTail };

template <typename T, int NV, int SLAB, bool SILU>
__global__ __launch_bounds__(1024) void norm_whole_kernel(const NormArgs a) {
  using namespace norm;
  constexpr int V = 16 / (int)sizeof(T);
  constexpr bool MERGE = SLAB == kMerge, STREAM = false;
  extern __shared__ char lds[];
  const Place k = place_whole(a.g);
  const int cols = a.g.tp * V, groups = a.g.groups;                 // of the slab
  float2* const part = reinterpret_cast<float2*>(lds);              // [r][vector or element]: (mean, squares)
  float2* const stat = part + (MERGE ? a.g.tp : cols) * a.g.rpi;    // [group]: (mean, rstd)
  const char* base = static_cast<const char*>(a.x) + (k.image * a.x_image + (long)k.p * V + k.r * a.x_pitch) * (long)sizeof(T);
  const long step = a.g.rpi * a.x_pitch * (long)sizeof(T);
  // superrows of this thread, and the elements of the last one
  const int rows = k.active ? a.g.few + (k.r < a.g.more ? 1 : 0) : 0;
  const int last = SLAB == kTail && k.r == a.g.last_r ? min(a.g.tail * a.c - k.p * V, V) : V;
  typename RawOf<typename Bits<T>::type, V>::type raw[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (i < rows) raw[i] = load<T, V>(base + i * step, i == rows - 1 ? last : V);
  Terms<V> c;
  Where<V> here;
  if (k.active) {
    here = where<V>(a, k.p * V);
    channel_terms<V>(a, here, c);
    if constexpr (MERGE) {
      float m = 0.0f, q = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i < rows)
#pragma unroll
          for (int j = 0; j < V; ++j) m += widen<T>(raw[i][j]);
      m *= __builtin_amdgcn_rcpf((float)(rows * V));
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i < rows)
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float d = widen<T>(raw[i][j]) - m;
            q = fmaf(d, d, q);
          }
      part[threadIdx.x] = make_float2(m, q);
    } else {
      float m[V], q[V];
#pragma unroll
      for (int j = 0; j < V; ++j) m[j] = q[j] = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i < rows)
#pragma unroll
          for (int j = 0; j < V; ++j)
            if (SLAB != kTail || i < rows - 1 || j < last) m[j] += widen<T>(raw[i][j]);
      const float all = __builtin_amdgcn_rcpf((float)rows), less = __builtin_amdgcn_rcpf((float)max(rows - 1, 1));
#pragma unroll
      for (int j = 0; j < V; ++j) m[j] *= j < last ? all : less;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i < rows)
#pragma unroll
          for (int j = 0; j < V; ++j)
            if (SLAB != kTail || i < rows - 1 || j < last) {
              const float d = widen<T>(raw[i][j]) - m[j];
              q[j] = fmaf(d, d, q[j]);
            }
      float4* const out = reinterpret_cast<float4*>(part + threadIdx.x * V);
#pragma unroll
      for (int j = 0; j < V; j += 2) out[j / 2] = make_float4(m[j], q[j], m[j + 1], q[j + 1]);
    }
  }
  __syncthreads();
  const int lanes = a.g.lanes, more = a.g.more, few = a.g.few, last_r = a.g.last_r;
  each_group(
      lanes, groups,
      [&](int g, int lane) __attribute__((always_inline)) {
        if constexpr (MERGE) {
          const int vg = a.cg / V;
          return lanes_sum<4>(
              lane, lanes, a.g.rpi, vg, [&](int r, int v) __attribute__((always_inline)) { return part[r * a.g.tp + g * vg + v]; },
              [&](int r, int, float2 e) __attribute__((always_inline)) { return raw_sums((double)((few + (r < more ? 1 : 0)) * V), e); });
        } else {
          return lanes_sum<4>(
              lane, lanes, a.g.rpi * a.g.R, a.cg,
              [&](int o, int ch) __attribute__((always_inline)) {
                const int r = a.g.R == 1 ? o : o / a.g.R, rr = o - r * a.g.R;
                return part[r * cols + rr * a.c + g * a.cg + ch];
              },
              [&](int o, int, float2 e) __attribute__((always_inline)) {
                const int r = a.g.R == 1 ? o : o / a.g.R, rr = o - r * a.g.R;
                return raw_sums((double)(few + (r < more ? 1 : 0) - (SLAB == kTail && r == last_r && rr >= a.g.tail ? 1 : 0)), e);
              });
        }
      },
      [&](int g, double2 s) __attribute__((always_inline)) {
        const float2 m = statistics(s, a);
        stat[g] = m;
        const int at = k.image * a.groups + k.part * groups + g;
        if (a.mean_out) a.mean_out[at] = m.x;
        if (a.rstd_out) a.rstd_out[at] = m.y;
      });
  __syncthreads();
  if (!k.active) return;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const float2 s = stat[here.group[MERGE ? 0 : j] - k.part * groups];
    c.mean[j] = s.x;
    c.w[j] *= s.y;
  }
  char* out = static_cast<char*>(a.y) + ((long)k.image * a.pixels * a.c + (long)(k.r * a.g.P + k.p) * V) * (long)sizeof(T);
  const long out_step = (long)a.g.rpi * a.g.P * V * (long)sizeof(T);
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (i < rows) normalise<T, V, SILU, STREAM>(a, raw[i], c, out + i * out_step, i == rows - 1 ? last : V);
}

// The gradient; dweight and dbias go to `part` [n][c] as an image's sums (or straight to their place where there is one image).  32 x 14 x 14 x 576 bf16, 22 MB, 12.8 us
// and the launch that sums the images' vectors 3.8.
template <typename T, int NV, int SLAB, bool SILU>
__global__ __launch_bounds__(1024) void norm_whole_grad_kernel(const NormArgs a) {
  using namespace norm;
  constexpr int V = 16 / (int)sizeof(T);
  constexpr bool STREAM = false;
  extern __shared__ char lds[];
  const Place k = place_whole(a.g);
  const int cols = a.g.tp * V, groups = a.g.groups, channels = groups * a.cg;      // of the slab
  float2* const buffer = reinterpret_cast<float2*>(lds);
  float2* const col = buffer;                                // [element of the superrow]: sums (the buffer is free by then)
  float2* const term = buffer + cols;                        // [group]
  const char* xb = static_cast<const char*>(a.x) + (k.image * a.x_image + (long)k.p * V + k.r * a.x_pitch) * (long)sizeof(T);
  const char* db = static_cast<const char*>(a.dy) + (k.image * a.dy_image + (long)k.p * V + k.r * a.dy_pitch) * (long)sizeof(T);
  const long step = a.g.rpi * a.x_pitch * (long)sizeof(T), dy_step = a.g.rpi * a.dy_pitch * (long)sizeof(T);
  const int rows = k.active ? a.g.few + (k.r < a.g.more ? 1 : 0) : 0;
  const int last = SLAB == kTail && k.r == a.g.last_r ? min(a.g.tail * a.c - k.p * V, V) : V;
  typename RawOf<typename Bits<T>::type, V>::type x[NV], dy[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (i < rows) {
      x[i] = load<T, V>(xb + i * step, i == rows - 1 ? last : V);
      dy[i] = load<T, V>(db + i * dy_step, i == rows - 1 ? last : V);
    }
  Terms<V> c;
  Where<V> here;
  float sb[V], sw[V];
#pragma unroll
  for (int j = 0; j < V; ++j) sb[j] = sw[j] = 0.0f;
  if (k.active) {
    here = where<V>(a, k.p * V);
    all_terms<V>(a, k.image, here, c);
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i < rows) gradient_sums<T, V, SILU>(a, x[i], dy[i], c, sb, sw, i == rows - 1 ? last : V);
  }
  add_rows<V>(sb, sw, k.r, a.g.tp, a.g.rpi, k.active, buffer);
  if (k.active && k.r == 0) {
#pragma unroll
    for (int j = 0; j < V; ++j) col[(int)threadIdx.x * V + j] = make_float2(sb[j], sw[j]);
  }
  const int ch0 = k.part * channels;
  fold_columns(a, col, channels, ch0, [&](int ch, float2 s) __attribute__((always_inline)) {
    if (a.n > 1) {
      if (a.dweight || a.dbias) a.part[(long)k.image * a.c + ch0 + ch] = s;
    } else {
      if (a.dbias) a.dbias[ch0 + ch] = s.x;
      if (a.dweight) a.dweight[ch0 + ch] = s.y;
    }
  });
  const int lanes = a.g.lanes;
  each_group(
      lanes, groups, [&](int g, int lane) __attribute__((always_inline)) { return group_terms(a, col, lane, lanes, g); },
      [&](int g, double2 s) __attribute__((always_inline)) { term[g] = make_float2((float)(s.x * a.inv_count), (float)(s.y * a.inv_count)); });
  __syncthreads();
  if (!k.active) return;
  float2 t[V];
#pragma unroll
  for (int j = 0; j < V; ++j) t[j] = term[here.group[j] - k.part * groups];
  char* out = static_cast<char*>(a.y) + ((long)k.image * a.pixels * a.c + (long)(k.r * a.g.P + k.p) * V) * (long)sizeof(T);
  const long out_step = (long)a.g.rpi * a.g.P * V * (long)sizeof(T);
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (i < rows) gradient<T, V, SILU, STREAM>(a, x[i], dy[i], c, t, out + i * out_step, i == rows - 1 ? last : V);
}

// ---- launches of a type ---------------------------------------------------------------------------

enum NormPass { kNormWhole, kNormWholeGrad, kNormStats, kNormApply, kNormGradSums, kNormGradApply };

struct NormLaunch {
  unsigned grid, lds, vector_groups;      // bytes of LDS; work-groups for dweight and dbias
  bool silu, stream;
};

namespace norm {

template <typename F> void with_flag(bool b, F&& f) { b ? f(std::true_type()) : f(std::false_type()); }
template <typename F> void with_vectors(int nv, F&& f) {      // rounded up to a built form
  if (nv <= 1) f(std::integral_constant<int, 1>());
  else if (nv <= 2) f(std::integral_constant<int, 2>());
  else if (nv <= 4) f(std::integral_constant<int, 4>());
  else if (nv <= 8) f(std::integral_constant<int, 8>());
  else f(std::integral_constant<int, 16>());
}
template <typename F> void with_slab(int slab, F&& f) {
  if (slab == kMerge) f(std::integral_constant<int, kMerge>());
  else if (slab == kTail) f(std::integral_constant<int, kTail>());
  else f(std::integral_constant<int, kPlain>());
}
template <typename T, typename F> void with_length(int v, F&& f) {
  if (v == 1) f(std::integral_constant<int, 1>());
  else if (v == 2) f(std::integral_constant<int, 2>());
  else if (v == 4 || sizeof(T) == 4) f(std::integral_constant<int, 4>());
  else f(std::integral_constant<int, sizeof(T) == 4 ? 4 : 8>());
}

}  // namespace norm

template <typename T> void launch_norm(NormPass pass, const NormArgs& a, const NormLaunch& l, hipStream_t s) {
  using namespace norm;
  const NormGeom& g = a.g;
  with_flag(l.silu, [&](auto silu) {
    constexpr bool SILU = decltype(silu)::value;
    if (pass == kNormWhole || pass == kNormWholeGrad) {
      const int slab = g.tail != g.R ? kTail : pass == kNormWhole && a.cg % g.V == 0 ? kMerge : kPlain;
      with_vectors(g.nv, [&](auto nv) {
        with_slab(slab, [&](auto form) {
          constexpr int NV = decltype(nv)::value, SLAB = decltype(form)::value;
          if (pass == kNormWhole) {
            norm_whole_kernel<T, NV, SLAB, SILU><<<l.grid, g.threads, l.lds, s>>>(a);
          } else if constexpr (NV <= kNormWholeGradVectors && SLAB != kMerge) {
            norm_whole_grad_kernel<T, NV, SLAB, SILU><<<l.grid, g.threads, l.lds, s>>>(a);
          }
        });
      });
      return;
    }
    with_length<T>(g.V, [&](auto v) {
      constexpr int V = decltype(v)::value;
      with_flag(l.stream, [&](auto stream) {
        constexpr bool STREAM = decltype(stream)::value;
        if (pass == kNormStats) norm_stats_kernel<T, V><<<l.grid, kThreads, 0, s>>>(a);
        else if (pass == kNormApply) norm_apply_kernel<T, V, SILU, STREAM><<<l.grid, kThreads, l.lds, s>>>(a);
        else if (pass == kNormGradSums) norm_grad_sums_kernel<T, V, SILU><<<l.grid, kThreads, 0, s>>>(a);
        else norm_grad_apply_kernel<T, V, SILU, STREAM><<<l.grid + l.vector_groups, kThreads, l.lds, s>>>(a, l.vector_groups);
      });
    });
  });
}
void launch_norm_f32(NormPass pass, const NormArgs& a, const NormLaunch& l, hipStream_t s);
void launch_norm_f16(NormPass pass, const NormArgs& a, const NormLaunch& l, hipStream_t s);
void launch_norm_bf16(NormPass pass, const NormArgs& a, const NormLaunch& l, hipStream_t s);

}  // namespace cprune
