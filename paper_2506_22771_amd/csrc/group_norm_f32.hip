// The group norm's kernels for one element type: see group_norm.hpp.
#include "group_norm_backward.hpp"
#include "group_norm_forward.hpp"

namespace ffi {

template hipError_t gn_forward_typed<float>(const GroupNormForwardLaunch& f, hipStream_t s);
template hipError_t gn_backward_typed<float>(const GroupNormBackwardLaunch& g, hipStream_t s);

}  // namespace ffi
