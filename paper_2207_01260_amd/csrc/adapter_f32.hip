// fp32 kernels of the low-rank adapters.
#include "adapter_kernel.hpp"

namespace cprune {

void launch_adapter_f32(AdapterPass pass, const void* args, const AdapterLaunch& l, hipStream_t s) { launch_adapter<float>(pass, args, l, s); }

}  // namespace cprune
