// The experts' products on f32 elements.
#include "experts_kernels.h"

namespace gsn {

template hipError_t launch_experts<float>(const Experts&, hipStream_t);
template hipError_t launch_experts_backward<float>(const Experts&, hipStream_t);

}  // namespace gsn
