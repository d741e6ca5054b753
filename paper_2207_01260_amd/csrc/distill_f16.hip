// fp16 kernels of the distillation loss.
#include "distill_kernel.hpp"

namespace cprune {

void launch_distill_f16(DistillPass pass, const DistillArgs& a, const DistillLaunch& l, hipStream_t s) { launch_distill<_Float16>(pass, a, l, s); }

}  // namespace cprune
