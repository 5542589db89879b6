// The experts' products on bf16 elements.
#include "experts_kernels.h"

namespace gsn {

template hipError_t launch_experts<gsn::bf16_t>(const Experts&, hipStream_t);
template hipError_t launch_experts_backward<gsn::bf16_t>(const Experts&, hipStream_t);

}  // namespace gsn
