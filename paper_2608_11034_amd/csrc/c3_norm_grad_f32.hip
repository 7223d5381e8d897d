// The gradient of the residual norm, blocks in fp32 (one source a type: they compile side by side).
#include "c3_norm_grad.h"

namespace c3 {

template hipError_t launch_norm_grad<float, float>(const NormArgs&, bool, unsigned, hipStream_t);

}  // namespace c3
