// The softmax cross entropy on f32 elements.
#include "entropy_kernels.h"

namespace gsn {

template hipError_t launch_entropy<float>(const Entropy&, hipStream_t);
template hipError_t launch_entropy_backward<float>(const Entropy&, hipStream_t);

}  // namespace gsn
