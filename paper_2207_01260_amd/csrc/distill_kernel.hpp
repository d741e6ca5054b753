// Distillation of a row's logits z from a list of a teacher's logits t and their classes, with a label beside it where there is one:
//
//   loss = (1 - h) T^2 sum_k p_k (log p_k - log q_T[id_k]) - h log q_1[label],   p = softmax(t / T) over the list, q_T = softmax(z / T) over all classes
//   dz   = dloss ((1 - h) T (q_T - p) + h (q_1 - [label]))
//
// One pass over a row keeps its largest number m and the sums of exp((z - m) / T) and exp(z - m): a thread's, rescaled where its m grows, then joined over the
// work-group.  All in 32 bits, a thread's in chains of 256 numbers at most, joined in another; the exponent's argument is (z - m) times log2(e) / T, a difference before the product, so that it is no less exact far from 0.
//
// Forms:
//  - rows: a work-group has a row.  Where the gradient is wanted too the row stays in registers (65536 numbers of 16 bits, 32768 of 32) between its sums and
//    its gradient: z is read once.  What is past them is read again.
//  - parts: few long rows; work-groups leave the sums of a run of a row, and those of a second launch join them and take the gradient of their run.
//  - the backward call has the sums already: the second launch alone.
// Bound by memory: the step of 4096 x 131072 bf16 439 us, 4.9 TB/s of z and dz; the loss of 4096 x 32768 fp16 52 us, 5.2 TB/s (its exponentials take nearly as long).
#pragma once
#include "logits.hpp"

namespace cprune {

constexpr int kMostList = 256;      // of a row

struct DistillArgs {
  const void* z;
  long z_stride;                // elements from row to row
  int rows, classes;
  const int* ids;               // [rows][k], outside [0, classes): no entry
  const void* teacher;          // [rows][k] of teacher_type
  int k, teacher_type;
  const int* labels;            // [rows] or null, outside [0, classes): none
  const float* dloss;           // [rows]; null: no gradient
  float *loss, *stats_out;      // [rows], [3][rows], or null
  const float* stats;           // backward: [3][rows]
  void* dz;                     // [rows][classes] or null
  float scale;                  // log2(e) / T
  float soft, hard;             // 1 - h, h
  float t, inv_t;
  float4* part;                 // [rows][parts]: m, the two sums
  int parts;
  int chunks, per;              // runs of a row, a work-group each; vectors of a run
  bool past;                    // dz is stored past the caches
};

enum DistillPass { kDistillRows, kDistillParts, kDistillFinish };
struct DistillLaunch {
  unsigned grid;
  int threads, held;            // held: vectors a thread (0: read again)
  int two;                      // distill::Second
};
void launch_distill_f32(DistillPass pass, const DistillArgs& a, const DistillLaunch& l, hipStream_t s);
void launch_distill_f16(DistillPass pass, const DistillArgs& a, const DistillLaunch& l, hipStream_t s);
void launch_distill_bf16(DistillPass pass, const DistillArgs& a, const DistillLaunch& l, hipStream_t s);

namespace distill {

using logits::Raw;
using logits::kLog2e;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// Over a wavefront, in every lane: rows of 16 lanes step by step, their results handed on to the next row and the next two.
template <int CTRL, int ROWS> __device__ __forceinline__ float from_lane(float old, float v) {
  return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp((int)__float_as_uint(old), (int)__float_as_uint(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float last_lane(float v) { return __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63)); }
__device__ __forceinline__ float wave_sum(float v) {
  v += from_lane<0x111, 0xf>(0.0f, v);      // one to the right, two, four, eight
  v += from_lane<0x112, 0xf>(0.0f, v);
  v += from_lane<0x114, 0xf>(0.0f, v);
  v += from_lane<0x118, 0xf>(0.0f, v);
  v += from_lane<0x142, 0xa>(0.0f, v);      // lane 15 of a row to the next one
  v += from_lane<0x143, 0xc>(0.0f, v);      // lane 31 to the upper half
  return last_lane(v);
}
__device__ __forceinline__ float wave_max(float v) {
  v = logits::larger(v, from_lane<0x111, 0xf>(v, v));
  v = logits::larger(v, from_lane<0x112, 0xf>(v, v));
  v = logits::larger(v, from_lane<0x114, 0xf>(v, v));
  v = logits::larger(v, from_lane<0x118, 0xf>(v, v));
  v = logits::larger(v, from_lane<0x142, 0xa>(v, v));
  v = logits::larger(v, from_lane<0x143, 0xc>(v, v));
  return last_lane(v);
}

// How the second exponential of a number, at temperature 1, is had beside the one at T: not wanted; by itself; where T is 2 or 4, the usual ones, as the first
// one's square or fourth power (an exponential takes as long as four products: 4096 x 32768 fp16 loss, temperature 2: 56.1 us with one of its own, 52.1 with the square).  The gradients' errors against 64
// bits are the same within a tenth, fp32 at T = 4 4000 x 16000 2.71e-8 and 2.66e-8, 3000 x 1000 3.0e-8 and 2.8e-8: the rounding of the exponent's argument, which is most of it, is smaller by as much.
enum Second { kNone, kOwn, kSquare, kFourth };
template <int TWO> __device__ __forceinline__ float second_of(float first, float d) {
  if constexpr (TWO == kSquare) return first * first;
  if constexpr (TWO == kFourth) return (first * first) * (first * first);
  return exp2_of(d * kLog2e);
}

// Largest number so far (from the lowest finite one, so that no difference is of two infinities unless a number is +infinity: then, as with a NaN, the sums are
// NaN) and the sums against it; TWO: at temperature 1 beside T.
template <int TWO> struct Sums {
  float m = -FLT_MAX, at_t = 0.0f, at_1 = 0.0f;
  float done_t = 0.0f, done_1 = 0.0f;      // of the numbers that are folded away
  __device__ __forceinline__ void rescale(float to, float scale) {
    const float d = m - to, by_t = exp2_of(d * scale);
    at_t *= by_t, done_t *= by_t;
    if constexpr (TWO != kNone) {
      const float by_1 = exp2_of(d * kLog2e);
      at_1 *= by_1, done_1 *= by_1;
    }
    m = to;
  }
  // Behind every 256 numbers at most: a chain of n equal terms is off by up to n / 4 units of 2^-24 (131072 of one thread: 0.2%).
  __device__ __forceinline__ void fold() {
    done_t += at_t, at_t = 0.0f;
    if constexpr (TWO != kNone) done_1 += at_1, at_1 = 0.0f;
  }
  template <int V> __device__ __forceinline__ void add(const float (&x)[V], float scale) {
    const float top = logits::largest(x);
    if (__any(!(top <= m))) rescale(logits::larger(m, top), scale);      // (seldom past a row's first vectors)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float d = x[j] - m;
      const float first = exp2_of(d * scale);
      at_t += first;
      if constexpr (TWO != kNone) at_1 += second_of<TWO>(first, d);
    }
  }
  __device__ __forceinline__ void over_wave(float scale) {
    rescale(wave_max(m), scale);
    fold();
    at_t = wave_sum(done_t), done_t = 0.0f;
    if constexpr (TWO != kNone) at_1 = wave_sum(done_1), done_1 = 0.0f;
  }
};

// A row's list, in the lanes of a wavefront: entry lane + 64 e its e-th.
struct List {
  static constexpr int E = kMostList / 64;
  int id[E];
  float t[E], z[E], p[E], log_p[E];
  int label;
  float z_label;
  bool any;

  template <typename T> static __device__ __forceinline__ float at(const T* z, int i) { return logits::widen<T>(z[i]); }

  __device__ __forceinline__ void load(const DistillArgs& a, int row) {
    const int lane = (int)threadIdx.x & 63;
    const long from = (long)row * a.k;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      id[e] = -1, t[e] = -__builtin_inff();
      const int i = lane + 64 * e;
      if (64 * e < a.k && i < a.k) {
        id[e] = a.ids[from + i];
        t[e] = a.teacher_type == CPRUNE_F32 ? static_cast<const float*>(a.teacher)[from + i]
               : a.teacher_type == CPRUNE_F16 ? (float)static_cast<const _Float16*>(a.teacher)[from + i]
                                              : logits::widen<__bf16>(static_cast<const __bf16*>(a.teacher)[from + i]);
      }
    }
    label = a.labels ? a.labels[row] : -1;
    if ((unsigned)label >= (unsigned)a.classes || a.hard == 0.0f) label = -1;
  }
  // their logits in the row, and the probabilities: p and T log p
  template <typename T> __device__ __forceinline__ void read(const DistillArgs& a, const T* row) {
    float m = -__builtin_inff();
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if ((unsigned)id[e] >= (unsigned)a.classes || t[e] == -__builtin_inff()) id[e] = -1, t[e] = -__builtin_inff();
      z[e] = id[e] >= 0 ? at(row, id[e]) : 0.0f;
      m = logits::larger(m, t[e]);
    }
    z_label = label >= 0 ? at(row, label) : 0.0f;
    m = wave_max(m);
    any = m != -__builtin_inff() && a.soft != 0.0f;
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      log_p[e] = (t[e] - m) * a.inv_t;
      p[e] = id[e] >= 0 ? exp2_of((t[e] - m) * a.scale) : 0.0f;
      s += p[e];
    }
    s = wave_sum(s);
    const float log_s = logf(s), inv = 1.0f / s;
#pragma unroll
    for (int e = 0; e < E; ++e) p[e] *= inv, log_p[e] -= log_s;
  }
  // the row's loss; log_t, log_1: logarithms of the row's sums
  __device__ __forceinline__ float loss(const DistillArgs& a, float m, float log_t, float log_1) const {
    float v = 0.0f;
    if (any) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float term = p[e] * (log_p[e] - (z[e] - m) * a.inv_t + log_t);
        if (p[e] != 0.0f) v += term;      // (a NaN is one: its row's loss is NaN)
      }
      v = wave_sum(v) * (a.soft * a.t * a.t);
    }
    if (label >= 0) v += a.hard * (log_1 - (z_label - m));
    return v;
  }
};

// What a class listed more than once has of p, and whether an entry is the first of its class; in LDS for as long as they are counted, read four at a time.
struct Shares {
  alignas(16) int id[kMostList];
  alignas(16) float p[kMostList];
  __device__ __forceinline__ void put(const List& l, int k) {
    const int lane = (int)threadIdx.x & 63;
#pragma unroll
    for (int e = 0; e < List::E; ++e)
      if (64 * e < k) id[lane + 64 * e] = l.id[e], p[lane + 64 * e] = l.p[e];
  }
  // f(e, share) for the entries of this lane that are first of their class
  template <typename F> __device__ __forceinline__ void each(const List& l, int k, F&& f) const {
    const int lane = (int)threadIdx.x & 63;
#pragma unroll
    for (int e = 0; e < List::E; ++e) {
      if (64 * e >= k) break;
      float share = 0.0f;
      bool first = l.id[e] >= 0;
      for (int j = 0; j < k; j += 4) {
        const int4 i = *reinterpret_cast<const int4*>(id + j);
        const float4 q = *reinterpret_cast<const float4*>(p + j);
        const int me = lane + 64 * e;
        share += (i.x == l.id[e] ? q.x : 0.0f) + (i.y == l.id[e] ? q.y : 0.0f) + (i.z == l.id[e] ? q.z : 0.0f) + (i.w == l.id[e] ? q.w : 0.0f);
        if ((i.x == l.id[e] && j < me) || (i.y == l.id[e] && j + 1 < me) || (i.z == l.id[e] && j + 2 < me) || (i.w == l.id[e] && j + 3 < me)) first = false;
      }
      if (first) f(e, share);
    }
  }
};

// A row's gradient: of a number x, q_T and q_1 times what each term counts.
struct Slope {
  float m, of_t, of_1, by_t, by_1;      // by: over the row's sums
  bool none;                            // no term counts: 0, whatever the row holds
  __device__ __forceinline__ void set(const DistillArgs& a, int row, float m_, float inv_sum_t, float inv_sum_1, bool any, bool label) {
    const float d = a.dloss[row];
    m = m_;
    of_t = any ? d * a.soft * a.t : 0.0f;
    of_1 = label ? d * a.hard : 0.0f;
    by_t = any ? of_t * inv_sum_t : 0.0f;
    by_1 = label ? of_1 * inv_sum_1 : 0.0f;
    none = d == 0.0f || !(any || label);
  }
  template <int TWO> __device__ __forceinline__ float at(float x, float scale) const {
    const float d = x - m;
    const float first = exp2_of(d * scale);
    float v = first * by_t;
    if constexpr (TWO != kNone) v += second_of<TWO>(first, d) * by_1;
    return v;
  }
  template <int TWO, int V> __device__ __forceinline__ void over(float (&x)[V], float scale) const {
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = at<TWO>(x[j], scale);
  }
};

// zeros for vectors of a row, and its edge
template <typename T> __device__ __forceinline__ void clear(T* dz, const logits::Row<T>& row, int first, int step, int end, bool edge) {
  const float zeros[Raw<T>::V] = {};
#pragma unroll 1
  for (int i = first; i < end; i += step) logits::store<T>(dz, i, zeros, false);
  if (edge) logits::store_edge<T>(dz, row, zeros);
}

// LDS of a work-group with a row or a run of one
template <int NT> struct Shared {
  float4 sums[NT / 64];
  int terms;
  Shares shares;
};

// The gradient's patches, by wavefront 0 behind the barrier that follows the stores: classes of the list, and the label where the list has it not.
template <typename T, int TWO> __device__ __forceinline__ void patch(const DistillArgs& a, const List& l, const Shares& shares, const Slope& g, T* dz, int lo, int hi) {
  bool listed = false;
#pragma unroll
  for (int e = 0; e < List::E; ++e) listed |= l.label >= 0 && l.id[e] == l.label && l.any;
  if (l.any)
    shares.each(l, a.k, [&](int e, float share) __attribute__((always_inline)) {
      if (l.id[e] < lo || l.id[e] >= hi) return;
      dz[l.id[e]] = (T)(g.at<TWO>(l.z[e], a.scale) - g.of_t * share - (l.id[e] == l.label ? g.of_1 : 0.0f));
    });
  if (l.label >= lo && l.label < hi && !__any(listed) && (threadIdx.x & 63) == 0) dz[l.label] = (T)(g.at<TWO>(l.z_label, a.scale) - g.of_1);
}

// A work-group has a row: its sums, its loss and, with dz, its gradient.  It holds the row's first NT NV vectors; those past them are read again.
template <typename T, int NT, int NV, int TWO>
__global__ __launch_bounds__(NT, NT == 512 ? 4 : 1) void distill_rows_kernel(const DistillArgs a) {
  constexpr int V = Raw<T>::V, NW = NT / 64;
  __shared__ Shared<NT> sh;
  const int t = (int)threadIdx.x, lane = t & 63, wave = t >> 6, row_no = blockIdx.x;
  const logits::Row<T> row(static_cast<const T*>(a.z) + row_no * a.z_stride, a.classes);
  List l;
  if (wave == 0) l.load(a, row_no);
  uint4 held[NV ? NV : 1];
  if constexpr (NV != 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) held[i] = row.load(t + i * NT, row.full);
  }
  float edge[V];
  row.edge(t == NT - 1, edge);
  if (wave == 0) {
    l.read<T>(a, row.p);
    if (a.dz) sh.shares.put(l, a.k);
    if (lane == 0) sh.terms = (l.any ? 1 : 0) | (l.label >= 0 ? 2 : 0);
  }
  Sums<TWO> s;
  if constexpr (NV != 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float x[V];
      logits::pin(held[i]);
      logits::unpack<T>(held[i], x);
      s.add(x, a.scale);
    }
  }
  constexpr int HELD = NV * NT, U = NV == 16 ? 4 : 8;
  if (NV == 0 || row.full > HELD) {
    int since = 0;
#pragma unroll 1
    for (int i = HELD + t; i - lane < row.full; i += U * NT) {      // (whole wavefronts)
      uint4 r[U];
#pragma unroll
      for (int u = 0; u < U; ++u) r[u] = row.load(i + u * NT, row.full);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float x[V];
        logits::unpack<T>(r[u], x);
        s.add(x, a.scale);
      }
      if ((++since & (NV ? 3 : 256 / (U * V) - 1)) == 0) s.fold();      // (of 512 threads' rows 128 are held before the first)
    }
  }
  if (row.tail) s.add(edge, a.scale);
  s.over_wave(a.scale);
  if (lane == 0) sh.sums[wave] = make_float4(s.m, s.at_t, s.at_1, 0.0f);
  __syncthreads();
  if constexpr (NW > 1) {
    const float4 v = sh.sums[lane & (NW - 1)];
    s.m = v.x, s.at_t = lane < NW ? v.y : 0.0f, s.at_1 = lane < NW ? v.z : 0.0f;
    s.over_wave(a.scale);
  }
  const float sum_1 = TWO != kNone ? s.at_1 : s.at_t;
  const bool empty = s.at_t == 0.0f;      // every class masked
  if (wave == 0 && a.loss) {
    const float log_t = logf(s.at_t), log_1 = TWO != kNone ? logf(s.at_1) : log_t;
    const float v = l.loss(a, s.m, log_t, log_1);
    if (lane == 0) {
      a.loss[row_no] = empty ? 0.0f : v;
      if (a.stats_out) {
        a.stats_out[row_no] = empty ? -__builtin_inff() : s.m;
        a.stats_out[a.rows + row_no] = empty ? 0.0f : log_t;
        a.stats_out[2 * a.rows + row_no] = empty ? 0.0f : log_1;
      }
    }
  }
  if (!a.dz) return;
  Slope g;
  const int terms = sh.terms;
  g.set(a, row_no, s.m, 1.0f / s.at_t, 1.0f / sum_1, (terms & 1) != 0, (terms & 2) != 0);
  g.none |= empty;
  if constexpr (TWO == kNone) g.by_t += g.by_1;
  T* const dz = static_cast<T*>(a.dz) + (long)row_no * a.classes;
  if (g.none) {
    clear<T>(dz, row, t, NT, row.full, t == NT - 1);
    return;
  }
  auto out = [&](int i, const uint4& r) __attribute__((always_inline)) {
    float x[V];
    logits::unpack<T>(r, x);
    g.over<TWO>(x, a.scale);
    if (i < row.full) logits::store<T>(dz, i, x, a.past);
  };
  if constexpr (NV != 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      logits::pin(held[i]);
      out(t + i * NT, held[i]);
    }
  }
  if (NV == 0 || row.full > HELD) {
#pragma unroll 1
    for (int i = HELD + t; i < row.full; i += U * NT) {
      uint4 r[U];
#pragma unroll
      for (int u = 0; u < U; ++u) r[u] = row.load(i + u * NT, row.full);
#pragma unroll
      for (int u = 0; u < U; ++u) out(i + u * NT, r[u]);
    }
  }
  if (t == NT - 1) {
    g.over<TWO>(edge, a.scale);
    logits::store_edge<T>(dz, row, edge);
  }
  __syncthreads();
  if (wave == 0) patch<T, TWO>(a, l, sh.shares, g, dz, 0, a.classes);
}

// Sums of a run of a row.
template <typename T, int TWO>
__global__ __launch_bounds__(256) void distill_parts_kernel(const DistillArgs a) {
  constexpr int V = Raw<T>::V;
  __shared__ float4 sums[4];
  const int t = (int)threadIdx.x, lane = t & 63, wave = t >> 6, row_no = blockIdx.x / (unsigned)a.chunks, chunk = blockIdx.x - row_no * a.chunks;
  const logits::Row<T> row(static_cast<const T*>(a.z) + row_no * a.z_stride, a.classes);
  const int end = min((chunk + 1) * a.per, row.full);
  Sums<TWO> s;
  int since = 0;
#pragma unroll 1
  for (int i = chunk * a.per + t; i - lane < end; i += 1024) {      // (whole wavefronts)
    uint4 r[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) r[u] = row.load(i + u * 256, end);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      float x[V];
      logits::unpack<T>(r[u], x);
      s.add(x, a.scale);
    }
    if ((++since & (64 / V - 1)) == 0) s.fold();
  }
  if (row.tail && chunk == a.chunks - 1) {
    float x[V];
    row.edge(t == 0, x);
    s.add(x, a.scale);
  }
  s.over_wave(a.scale);
  if (lane == 0) sums[wave] = make_float4(s.m, s.at_t, s.at_1, 0.0f);
  __syncthreads();
  if (wave == 0) {
    const float4 v = sums[lane & 3];
    s.m = v.x, s.at_t = lane < 4 ? v.y : 0.0f, s.at_1 = lane < 4 ? v.z : 0.0f;
    s.over_wave(a.scale);
    if (lane == 0) a.part[(long)row_no * a.parts + chunk] = make_float4(s.m, s.at_t, s.at_1, 0.0f);
  }
}

// With the row's sums, from up to 64 parts or given: the gradient of a run, and the loss by the row's first work-group.
template <typename T, int NT, int TWO>
__global__ __launch_bounds__(NT) void distill_finish_kernel(const DistillArgs a) {
  constexpr int V = Raw<T>::V;
  __shared__ Shared<NT> sh;
  const int t = (int)threadIdx.x, lane = t & 63, wave = t >> 6, row_no = blockIdx.x / (unsigned)a.chunks, chunk = blockIdx.x - row_no * a.chunks;
  const logits::Row<T> row(static_cast<const T*>(a.z) + row_no * a.z_stride, a.classes);
  List l;
  if (wave == 0) l.load(a, row_no);
  const int from = chunk * a.per, end = min(from + a.per, row.full);
  const bool last = chunk == a.chunks - 1;
  uint4 r[4];
  float edge[V];
  if (a.dz) {
#pragma unroll
    for (int u = 0; u < 4; ++u) r[u] = row.load(from + t + u * NT, end);
    row.edge(last && t == NT - 1, edge);
  }
  if (wave == 0) {
    l.read<T>(a, row.p);
    if (a.dz) sh.shares.put(l, a.k);
    if (lane == 0) sh.terms = (l.any ? 1 : 0) | (l.label >= 0 ? 2 : 0);
  }
  float m, log_t = 0.0f, log_1 = 0.0f, inv_t, inv_1;
  bool empty;
  if (a.stats) {
    m = a.stats[row_no];
    inv_t = expf(-a.stats[a.rows + row_no]);
    inv_1 = expf(-a.stats[2 * a.rows + row_no]);
    empty = m == -__builtin_inff();
  } else {
    Sums<TWO> s;
    if (lane < a.parts) {
      const float4 v = a.part[(long)row_no * a.parts + lane];
      s.m = v.x, s.at_t = v.y, s.at_1 = v.z;
    }
    s.over_wave(a.scale);
    m = s.m;
    empty = s.at_t == 0.0f;
    inv_t = 1.0f / s.at_t, inv_1 = TWO != kNone ? 1.0f / s.at_1 : inv_t;
    if (wave == 0 && chunk == 0 && a.loss) {
      log_t = logf(s.at_t), log_1 = TWO != kNone ? logf(s.at_1) : log_t;
      const float v = l.loss(a, m, log_t, log_1);
      if (lane == 0) {
        a.loss[row_no] = empty ? 0.0f : v;
        if (a.stats_out) {
          a.stats_out[row_no] = empty ? -__builtin_inff() : m;
          a.stats_out[a.rows + row_no] = empty ? 0.0f : log_t;
          a.stats_out[2 * a.rows + row_no] = empty ? 0.0f : log_1;
        }
      }
    }
  }
  if (!a.dz) return;
  __syncthreads();
  Slope g;
  const int terms = sh.terms;
  g.set(a, row_no, m, inv_t, inv_1, (terms & 1) != 0, (terms & 2) != 0);
  g.none |= empty;
  if constexpr (TWO == kNone) g.by_t += g.by_1;
  T* const dz = static_cast<T*>(a.dz) + (long)row_no * a.classes;
  if (g.none) {
    clear<T>(dz, row, from + t, NT, end, last && t == NT - 1);
    return;
  }
#pragma unroll 1
  for (int i = from + t; i < end; i += 4 * NT) {
    uint4 next[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) next[u] = row.load(i + (4 + u) * NT, end);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      float x[V];
      logits::unpack<T>(r[u], x);
      g.over<TWO>(x, a.scale);
      if (i + u * NT < end) logits::store<T>(dz, i + u * NT, x, a.past);
      r[u] = next[u];
    }
  }
  if (last && t == NT - 1) {
    g.over<TWO>(edge, a.scale);
    logits::store_edge<T>(dz, row, edge);
  }
  __syncthreads();
  if (wave == 0) patch<T, TWO>(a, l, sh.shares, g, dz, from * V, last ? a.classes : end * V);
}

template <typename T, int TWO> void launch_two(DistillPass pass, const DistillArgs& a, const DistillLaunch& l, hipStream_t s) {
  if (pass == kDistillParts) distill_parts_kernel<T, TWO><<<l.grid, 256, 0, s>>>(a);
  else if (pass == kDistillFinish && l.threads == 64) distill_finish_kernel<T, 64, TWO><<<l.grid, 64, 0, s>>>(a);
  else if (pass == kDistillFinish) distill_finish_kernel<T, 256, TWO><<<l.grid, 256, 0, s>>>(a);
  else if (l.threads == 64 && l.held) distill_rows_kernel<T, 64, 4, TWO><<<l.grid, 64, 0, s>>>(a);
  else if (l.threads == 64) distill_rows_kernel<T, 64, 0, TWO><<<l.grid, 64, 0, s>>>(a);
  else if (l.threads == 512) distill_rows_kernel<T, 512, 16, TWO><<<l.grid, 512, 0, s>>>(a);
  else if (l.held) distill_rows_kernel<T, 256, 8, TWO><<<l.grid, 256, 0, s>>>(a);
  else distill_rows_kernel<T, 256, 0, TWO><<<l.grid, 256, 0, s>>>(a);
}

}  // namespace distill

template <typename T> void launch_distill(DistillPass pass, const DistillArgs& a, const DistillLaunch& l, hipStream_t s) {
  using namespace distill;
  if (l.two == kNone) launch_two<T, kNone>(pass, a, l, s);
  else if (l.two == kSquare) launch_two<T, kSquare>(pass, a, l, s);
  else if (l.two == kFourth) launch_two<T, kFourth>(pass, a, l, s);
  else launch_two<T, kOwn>(pass, a, l, s);
}

}  // namespace cprune
