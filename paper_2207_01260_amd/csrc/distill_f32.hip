// fp32 kernels of the distillation loss.
#include "distill_kernel.hpp"

namespace cprune {

void launch_distill_f32(DistillPass pass, const DistillArgs& a, const DistillLaunch& l, hipStream_t s) { launch_distill<float>(pass, a, l, s); }

}  // namespace cprune
