// Entry points of the distillation loss (distill_kernel.hpp has the kernels).
#include <algorithm>
#include <cmath>

#include "distill_kernel.hpp"

namespace cprune {
namespace {

int check(const cprune_distill_desc* d) {
  if (!d || d->rows < 1 || d->classes < 1 || d->k < 1 || d->z_stride < d->classes || !dtype_ok(d->dtype) || !dtype_ok(d->teacher_dtype)) return CPRUNE_ERR_INVALID_ARG;
  const float t = d->temperature;
  if (!(t > 0.0f) || !std::isfinite(t * t) || !std::isfinite(2.0f / t) || !(d->hard >= 0.0f && d->hard <= 1.0f)) return CPRUNE_ERR_INVALID_ARG;
  if ((double)d->rows * d->z_stride >= 2147483648.0 || (double)d->rows * d->k >= 2147483648.0) return CPRUNE_ERR_INVALID_ARG;
  return d->k > kMostList || d->rows >= 1 << 22 ? CPRUNE_ERR_UNSUPPORTED : CPRUNE_OK;      // (a launch holds fewer than 2^32 threads)
}

int vectors_of(const cprune_distill_desc& d) {
  const int v = d.dtype == CPRUNE_F32 ? 4 : 8;
  return (d.classes - 1) / v + 1;
}

// Runs of a row for the launches that cut rows: a work-group of 256 has a vector or more for each thread.  Few rows, so that compute units would have none, and long ones,
// so that a second launch costs less than it gains (bf16 steps, rows whole and cut: 8 x 16384 9.8 and 9.9 us, 8 x 32768 12.4 and 10.3, 64 x 131072 27.8 and 18.0, 127 x
// 131072 29.4 and 23.3, 200 x 131072 32.4 and 33.6, 1 x 1000000 137 and 11.9).
constexpr int kMostParts = 64;      // (joined by the lanes of a wavefront)
bool by_parts(const cprune_distill_desc& d) { return d.rows < 128 && vectors_of(d) >= 4096; }
void cut(const cprune_distill_desc& d, int runs, DistillArgs& a) {
  const int vectors = vectors_of(d);
  a.per = std::max(256, ((vectors - 1) / runs + 256) / 256 * 256);
  a.chunks = (vectors - 1) / a.per + 1;
}

DistillArgs args_of(const cprune_distill_desc& d, const void* z, const int32_t* ids, const void* teacher, const int32_t* labels) {
  DistillArgs a = {};
  a.z = z, a.z_stride = d.z_stride, a.rows = d.rows, a.classes = d.classes;
  a.ids = ids, a.teacher = teacher, a.k = d.k, a.teacher_type = d.teacher_dtype, a.labels = labels;
  a.scale = (float)(1.4426950408889634 / d.temperature);
  a.soft = 1.0f - d.hard, a.hard = d.hard, a.t = d.temperature, a.inv_t = 1.0f / d.temperature;
  a.chunks = 1;
  a.past = past_caches((double)d.rows * d.classes * dtype_size(d.dtype));
  return a;
}

int second_of(const cprune_distill_desc& d, bool wanted) {
  if (!wanted || d.temperature == 1.0f) return distill::kNone;
  return d.temperature == 2.0f ? distill::kSquare : d.temperature == 4.0f ? distill::kFourth : distill::kOwn;
}

void launch(int dtype, DistillPass pass, const DistillArgs& a, const DistillLaunch& l, hipStream_t s) {
  if (dtype == CPRUNE_F32) launch_distill_f32(pass, a, l, s);
  else if (dtype == CPRUNE_F16) launch_distill_f16(pass, a, l, s);
  else launch_distill_bf16(pass, a, l, s);
}

// Loss, with statistics or gradient.
int forward(const cprune_distill_desc& d, DistillArgs a, void* ws, size_t ws_bytes, hipStream_t s) {
  const size_t need = cprune_distill_workspace_bytes(&d);
  if (need && (!ws || ws_bytes < need)) return CPRUNE_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(ws) & 15) return CPRUNE_ERR_INVALID_ARG;
  const int vectors = vectors_of(d);
  DistillLaunch l = {};
  l.two = second_of(d, a.stats_out || (a.labels && d.hard > 0.0f));
  if (by_parts(d)) {
    cut(d, std::min(kMostParts, std::max(8, 1024 / d.rows)), a);
    a.part = static_cast<float4*>(ws), a.parts = a.chunks;
    l.grid = (unsigned)d.rows * a.chunks, l.threads = 256;
    launch(d.dtype, kDistillParts, a, l, s);
    if (!a.dz) a.chunks = 1, l.grid = (unsigned)d.rows;
    launch(d.dtype, kDistillFinish, a, l, s);
  } else {
    // the fewest threads that hold the row (16384 x 1000 fp32: 33 us with 64, 74 with 256; 2048 x 16384 bf16: 39 with 256, 60 with 512)
    l.grid = (unsigned)d.rows;
    if (vectors <= 256) l.threads = 64, l.held = a.dz ? 4 : 0;
    else if (!a.dz || vectors <= 2048) l.threads = 256, l.held = a.dz ? 8 : 0;
    else l.threads = 512, l.held = 16;
    launch(d.dtype, kDistillRows, a, l, s);
  }
  CPRUNE_LAUNCH_CHECK();
  return CPRUNE_OK;
}

}  // namespace
}  // namespace cprune

using namespace cprune;

extern "C" size_t cprune_distill_workspace_bytes(const cprune_distill_desc* d) {
  if (check(d) != CPRUNE_OK || !by_parts(*d)) return 0;
  return (size_t)d->rows * kMostParts * sizeof(float4);
}

extern "C" int cprune_distill_loss(const cprune_distill_desc* d, const void* z, const int32_t* ids, const void* teacher, const int32_t* labels, float* loss,
                                   float* stats, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check(d);
  if (rc != CPRUNE_OK) return rc;
  if (!z || !ids || !teacher || !loss) return CPRUNE_ERR_INVALID_ARG;
  DistillArgs a = args_of(*d, z, ids, teacher, labels);
  a.loss = loss, a.stats_out = stats;
  return forward(*d, a, ws, ws_bytes, static_cast<hipStream_t>(stream));
}

extern "C" int cprune_distill_step(const cprune_distill_desc* d, const float* dloss, const void* z, const int32_t* ids, const void* teacher,
                                   const int32_t* labels, float* loss, void* dz, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check(d);
  if (rc != CPRUNE_OK) return rc;
  if (!dloss || !z || !ids || !teacher || !loss || !dz) return CPRUNE_ERR_INVALID_ARG;
  DistillArgs a = args_of(*d, z, ids, teacher, labels);
  a.loss = loss, a.dloss = dloss, a.dz = dz;
  return forward(*d, a, ws, ws_bytes, static_cast<hipStream_t>(stream));
}

extern "C" int cprune_distill_loss_backward(const cprune_distill_desc* d, const float* dloss, const void* z, const int32_t* ids, const void* teacher,
                                            const int32_t* labels, const float* stats, void* dz, void* stream) {
  const int rc = check(d);
  if (rc != CPRUNE_OK) return rc;
  if (!dloss || !z || !ids || !teacher || !stats || !dz) return CPRUNE_ERR_INVALID_ARG;
  DistillArgs a = args_of(*d, z, ids, teacher, labels);
  a.stats = stats, a.dloss = dloss, a.dz = dz;
  DistillLaunch l = {};
  l.two = second_of(*d, labels && d->hard > 0.0f);
  const int vectors = vectors_of(*d);
  if (vectors <= 256) {
    l.threads = 64, a.per = vectors;
  } else {
    l.threads = 256;
    cut(*d, std::max(std::min(vectors / 4096, 64), 2048 / d->rows) + 1, a);
  }
  l.grid = (unsigned)d->rows * a.chunks;
  launch(d->dtype, kDistillFinish, a, l, static_cast<hipStream_t>(stream));
  CPRUNE_LAUNCH_CHECK();
  return CPRUNE_OK;
}
