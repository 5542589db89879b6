// The softmax cross entropy on bf16 elements.
#include "entropy_kernels.h"

namespace gsn {

template hipError_t launch_entropy<gsn::bf16_t>(const Entropy&, hipStream_t);
template hipError_t launch_entropy_backward<gsn::bf16_t>(const Entropy&, hipStream_t);

}  // namespace gsn
