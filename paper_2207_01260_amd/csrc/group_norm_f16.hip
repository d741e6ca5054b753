// fp16 kernels of the channels-last group norm.
#include "group_norm_kernel.hpp"

namespace cprune {

void launch_norm_f16(NormPass pass, const NormArgs& a, const NormLaunch& l, hipStream_t s) { launch_norm<_Float16>(pass, a, l, s); }

}  // namespace cprune
