// The gradient of the residual norm, blocks in bf16 (one source a type: they compile side by side).
#include "c3_norm_grad.h"

namespace c3 {

template hipError_t launch_norm_grad<__bf16, __bf16>(const NormArgs&, bool, unsigned, hipStream_t);
template hipError_t launch_norm_grad<float, __bf16>(const NormArgs&, bool, unsigned, hipStream_t);

}  // namespace c3
