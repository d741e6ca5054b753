// bf16 kernels of the low-rank adapters.
#include "adapter_kernel.hpp"

namespace cprune {

void launch_adapter_bf16(AdapterPass pass, const void* args, const AdapterLaunch& l, hipStream_t s) { launch_adapter<__bf16>(pass, args, l, s); }

}  // namespace cprune
