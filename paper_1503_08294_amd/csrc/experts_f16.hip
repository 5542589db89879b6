// The experts' products on f16 elements.
#include "experts_kernels.h"

namespace gsn {

template hipError_t launch_experts<gsn::f16_t>(const Experts&, hipStream_t);
template hipError_t launch_experts_backward<gsn::f16_t>(const Experts&, hipStream_t);

}  // namespace gsn
