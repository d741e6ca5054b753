// The largest logits of each row with their classes: descending, equal ones by their class, NaN before all; -infinity is a class that is not there and is never
// listed.
//
// A bound first: each thread's largest number is one of the row's, so at least k numbers reach the k-th largest of those.  With more threads than k the numbers
// that reach it are hardly more than k.  They are looked for where a thread's run of vectors reaches it, go to a list in LDS, in any order, and each one's place
// is the count of those before it.  What bounds it is reading z once: 2048 x 50257 bf16, k 32, 53 us, 3.9 TB/s, the
// look at the runs and the places not hidden behind other rows.
#include <algorithm>

#include "logits.hpp"

namespace cprune {
namespace {

using logits::Raw;

constexpr int kMostK = 256;
constexpr int kSlots = 8, kRuns = 512;
constexpr int kList = 1024;      // numbers that reach the bound, in LDS; kMostK more of its equals

// 32 bits that order like numbers, -0 as 0, NaN above all; and the number again
__device__ __forceinline__ unsigned key_of(float x) {
  const unsigned u = __float_as_uint(x + 0.0f);
  return x != x ? 0xffffffffu : u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float number_of(unsigned key) {
  return key == 0xffffffffu ? __uint_as_float(0x7fc00000u) : __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

struct TopArgs {
  const void* z;
  long stride;                 // elements from row to row
  int classes, k;
  int chunks, per;             // runs that a row is cut into, numbers of a run (a multiple of whole vectors)
  const int* map;              // class of a place, [rows][classes], or null: the place itself
  void* values;                // [rows][chunks][k]
  int* ids;
};

// One row, or one run of it, a work-group.
template <typename T, typename OUT, int NT>
__global__ __launch_bounds__(NT) void top_kernel(const TopArgs a) {
  constexpr int V = Raw<T>::V, NW = NT / 64;
  __shared__ unsigned keys[NT], list_key[kList + kMostK];
  __shared__ int list_at[kList + kMostK];
  __shared__ int count, owners, sums[NW];
  __shared__ unsigned short slots[kSlots][NT];
  __shared__ int runs[kRuns];
  __shared__ unsigned bound;
  const int t = (int)threadIdx.x, lane = t & 63, wave = t >> 6;
  const int row_no = blockIdx.x / (unsigned)a.chunks, chunk = blockIdx.x - row_no * a.chunks;
  const long first = (long)chunk * a.per;
  const logits::Row<T> row(static_cast<const T*>(a.z) + row_no * a.stride + first, (int)min((long)a.per, a.classes - first));
  const int rounds = (row.full + NT - 1) / NT;
  // f(number of the vector, its numbers), a vector at a time; the edge is the last thread's
  auto each_slowly = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll 1
    for (int i = t; i < row.full + (row.tail && t == NT - 1 ? NT : 0); i += NT) {
      float x[V];
      int at = i;
      if (i < row.full) {
        logits::unpack<T>(row.load(i, row.full), x);
      } else {
        row.edge(true, x);
        at = row.full;
      }
      f(at, x);
    }
  };
  // A thread's largest number, and of each of up to kSlots runs of four or more of its vectors the upper half of the largest one's key
  const int fours = (rounds + 3) / 4, per = (fours + kSlots - 1) / kSlots;
  for (int i = 0; i < min(fours, kSlots); ++i) slots[i][t] = 0;
  float top = -__builtin_inff();
#pragma unroll 1
  for (int q = 0; q < fours; q += 2) {
    constexpr int U = 8;
    uint4 r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) r[u] = row.load(t + (4 * q + u) * NT, row.full);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float m = -__builtin_inff();
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float x[V];
        logits::unpack<T>(r[4 * h + u], x);
        m = logits::larger(m, logits::largest(x));
      }
      top = logits::larger(top, m);
      unsigned short* const slot = &slots[min((q + h) / per, kSlots - 1)][t];      // (past the last four: nothing)
      *slot = max(*slot, (unsigned short)(key_of(m) >> 16));
    }
  }
  if (row.tail && t == NT - 1) {
    float x[V];
    row.edge(true, x);
    top = logits::larger(top, logits::largest(x));
  }
  keys[t] = key_of(top);
  if (t == 0) count = owners = 0;
  __syncthreads();
  if (wave == 0) {      // bit by bit the largest bound that k threads reach, or one that few more do
    unsigned mine[NW], b = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) mine[i] = keys[lane + 64 * i];
    for (unsigned bit = 0x80000000u; bit; bit >>= 1) {
      int reach = 0;
#pragma unroll
      for (int i = 0; i < NW; ++i) reach += __popcll(__ballot(mine[i] >= (b | bit)));
      if (reach < a.k) continue;
      b |= bit;
      if (reach <= a.k + a.k / 4) break;
    }
    if (lane == 0) bound = b;
  }
  __syncthreads();
  // -infinity reaches no bound
  const unsigned least = 0x00800000u;                       // the key of the lowest finite number
  unsigned low = max(bound, least);
  float from = number_of(low);
  auto append = [&](float x, int at) __attribute__((always_inline)) {
    const int i = atomicAdd(&count, 1);      // (in any order: places are counted below)
    if (i < kList) list_key[i] = key_of(x), list_at[i] = at;
  };
  // the runs that reach it are read again, four lanes each
  auto look = [&](int i, const float (&x)[V]) __attribute__((always_inline)) {
    if (logits::largest(x) < from) return;
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (!(x[j] < from)) append(x[j], i * V + j);
  };
  if (!(top < from)) {
#pragma unroll 1
    for (int i = 0; i < min(fours, kSlots); ++i)
      if (slots[i][t] >= low >> 16) {
        const int at = atomicAdd(&owners, 1);      // (in any order, as the list)
        if (at < kRuns) runs[at] = i * NT + t;
      }
  }
  __syncthreads();
  const int found = min(owners, kRuns);
#pragma unroll 1
  for (int o = t >> 2; o < found; o += NT / 4) {
    const int run = runs[o] / NT, of = runs[o] % NT;
#pragma unroll 1
    for (int f = run * per; f < (run + 1) * per; ++f) {
      const int i = of + (4 * f + (t & 3)) * NT;
      float x[V];
      logits::unpack<T>(row.load(i, row.full), x);
      look(i, x);
    }
  }
  if (row.tail && t == NT - 1) {
    float x[V];
    row.edge(true, x);
    look(row.full, x);
  }
  __syncthreads();
  int n = count;
  // Many equal to the bound, as where most of a row has the type's lowest value: of those only the first k can count.  The row is read again three times, or, where
  // more than kList lie above the bound, some 35 times: 2048 x 50257 bf16, k 32 and 256, ordinary rows 46 and 219 us, one value throughout 142 and 259, mostly the lowest value 80 and
  // 304, sorted rows 168 and 1310, 5000 NaN a row 1186 and 1220.
  if (n > kList || owners > kRuns) {
    auto total = [&](int mine) __attribute__((always_inline)) {
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o, 64);
      __syncthreads();
      if (lane == 0) sums[wave] = mine;
      __syncthreads();
      int s = 0;
#pragma unroll
      for (int i = 0; i < NW; ++i) s += sums[i];
      return s;
    };
    auto reach = [&](unsigned b) __attribute__((always_inline)) {
      int mine = 0;
      each_slowly([&](int, const float (&x)[V]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < V; ++j) mine += key_of(x[j]) >= b;
      });
      return total(mine);
    };
    if (low == 0xffffffffu || reach(low + 1) > kList) {      // or a few threads have most of the largest numbers: the k-th largest itself
      unsigned b = 0;
      for (unsigned bit = 0x80000000u; bit; bit >>= 1)
        if (reach(b | bit) >= a.k) b |= bit;
      low = max(b, least);
    }
    if (t == 0) count = 0;
    __syncthreads();
    each_slowly([&](int i, const float (&x)[V]) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (key_of(x[j]) > low) append(x[j], i * V + j);
    });
    __syncthreads();
    const int above = count;
    // the first of the equal ones, round by round of NT vectors and the edge, in their order
    int have = 0;
    for (int i = 0; i <= rounds && have < a.k; ++i) {
      float x[V];
      const int at = i < rounds ? t + i * NT : row.full;
      if (i < rounds) logits::unpack<T>(row.load(at, row.full), x);
      else row.edge(t == 0, x);
      int mine = 0;
#pragma unroll
      for (int j = 0; j < V; ++j) mine += key_of(x[j]) == low;
      int before = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(before, o, 64);
        before += lane >= o ? v : 0;
      }
      __syncthreads();
      if (lane == 63) sums[wave] = before;
      __syncthreads();
      before += have - mine;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        before += w < wave ? sums[w] : 0;
        have += sums[w];
      }
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (key_of(x[j]) == low) {
          if (before < a.k) list_key[above + before] = low, list_at[above + before] = at * V + j;
          ++before;
        }
    }
    n = above + min(have, a.k);
    __syncthreads();
  }
  // places
  const long out = (long)blockIdx.x * a.k;
  OUT* const values = static_cast<OUT*>(a.values) + out;
  int* const ids = a.ids + out;
  for (int i = t; i < n; i += NT) {
    const unsigned key = list_key[i];
    const int at = list_at[i];
    int place = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) place += list_key[j] > key || (list_key[j] == key && list_at[j] < at);
    if (place < a.k) {
      values[place] = (OUT)number_of(key);
      ids[place] = a.map ? a.map[(long)row_no * a.classes + at] : (int)first + at;
    }
  }
  for (int i = n + t; i < a.k; i += NT) values[i] = (OUT)-__builtin_inff(), ids[i] = -1;
}

// Few very long rows are cut into runs, each with its own list, and the lists are searched by a launch behind it.  That pays where reading a row by one compute unit takes
// longer than another launch, and for short lists: descending lists beside each other make the search's bound a loose one (one row in fp32, whole and cut: 131072
// classes k 32 19 and 23 us, 300000 k 8 28 and 12, k 32 33 and 24, k 64 40 and 116; 64 rows of 300000 k 32 43 and 39, of 131072 25 and 30).
struct TopPlan {
  int chunks, per;
  size_t values, ids;
  size_t total() const { return values + ids; }
};
TopPlan plan_top(int rows, int classes, int k, int dtype) {
  const int v = dtype == CPRUNE_F32 ? 4 : 8;
  TopPlan q = {1, classes, 0, 0};
  if (rows <= 64 && k <= 32 && classes / v >= 65536) {
    q.per = 4096;
    while (q.per / v < 4 * k || (classes - 1) / q.per >= 64) q.per *= 2;
    q.chunks = (classes - 1) / q.per + 1;
    if (q.chunks > 1) {
      q.values = ((size_t)rows * q.chunks * k * sizeof(float) + 15) & ~(size_t)15;
      q.ids = (size_t)rows * q.chunks * k * sizeof(int);
    } else {
      q.per = classes;
    }
  }
  return q;
}

template <typename T, typename OUT> void launch_top(const TopArgs& a, int rows, hipStream_t s) {
  const unsigned grid = (unsigned)rows * a.chunks;
  const int vectors = (a.per + Raw<T>::V - 1) / Raw<T>::V;
  // Four threads or more for each of the k, if the row has them, fewer where rows are many: a loose bound costs some rows' places, 1024 threads a row leave two rows to a
  // compute unit.  16384 x 1000 fp32 k 8: 32 us with 64, 45 with 256.  bf16 with 256 and 1024:
  //   2048 x 50257   k 32 55 and 98, k 64 66 and 104, k 72 65 and 104, k 100 78 and 109, k 128 113 and 118, k 160 167 and 129, k 256 1342 and 233
  //   16384 x 4000   k 72 131 and 479, k 128 296 and 552      512 x 50257   k 72 28 and 32, k 128 65 and 40
  //   512 x 10000    k 100 26 and 29                          256, 64 x 50257   k 100 31 and 26, 29 and 24
  const int most = rows >= 2048 ? 128 : rows >= 512 ? 100 : 64;
  if (vectors <= 512 && (a.k <= 16 || vectors <= 64)) top_kernel<T, OUT, 64><<<grid, 64, 0, s>>>(a);
  else if (a.k <= most || vectors <= 256) top_kernel<T, OUT, 256><<<grid, 256, 0, s>>>(a);
  else top_kernel<T, OUT, 1024><<<grid, 1024, 0, s>>>(a);
}

int check_top(int rows, int classes, long stride, int k, int dtype) {
  if (rows < 1 || classes < 1 || stride < classes || k < 1 || k > classes || !dtype_ok(dtype) || (double)rows * stride >= 2147483648.0) return CPRUNE_ERR_INVALID_ARG;
  return k > kMostK || rows >= 1 << 22 ? CPRUNE_ERR_UNSUPPORTED : CPRUNE_OK;      // (a launch holds fewer than 2^32 threads)
}

}  // namespace
}  // namespace cprune

using namespace cprune;

extern "C" size_t cprune_top_logits_workspace_bytes(int rows, int classes, int k, cprune_dtype dtype) {
  return check_top(rows, classes, classes, k, dtype) == CPRUNE_OK ? plan_top(rows, classes, k, dtype).total() : 0;
}

extern "C" int cprune_top_logits(const void* z, int rows, int classes, int z_stride, int k, cprune_dtype dtype, void* values, int32_t* ids, void* ws,
                                 size_t ws_bytes, void* stream) {
  const int rc = check_top(rows, classes, z_stride, k, dtype);
  if (rc != CPRUNE_OK) return rc;
  if (!z || !values || !ids) return CPRUNE_ERR_INVALID_ARG;
  const TopPlan q = plan_top(rows, classes, k, dtype);
  if (q.total() && (!ws || ws_bytes < q.total())) return CPRUNE_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(ws) & 15) return CPRUNE_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  TopArgs a = {z, z_stride, classes, k, q.chunks, q.per, nullptr, values, ids};
  logits::with_type(dtype, [&](auto t) {
    using T = decltype(t);
    if (q.chunks == 1) {
      launch_top<T, T>(a, rows, s);
      return;
    }
    float* const some = static_cast<float*>(ws);
    int* const at = reinterpret_cast<int*>(static_cast<char*>(ws) + q.values);
    a.values = some, a.ids = at;
    launch_top<T, float>(a, rows, s);
    const int all = q.chunks * k;
    const TopArgs b = {some, all, all, k, 1, all, at, values, ids};
    launch_top<float, T>(b, rows, s);
  });
  CPRUNE_LAUNCH_CHECK();
  return CPRUNE_OK;
}
