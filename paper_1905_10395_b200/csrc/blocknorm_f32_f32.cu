// The block-boundary kernels of blocknorm.h for fp32 residual and activations (a file for each pair of types: they compile side by side).
#define LSGD_BLOCKNORM_KERNELS
#include "blocknorm.h"

namespace lsgd {
namespace blocknorm {
cudaError_t launch_f32_f32(const Args& a, const Launch& l, cudaStream_t s) { return launch_types<float, float>(a, l, s); }
}  // namespace blocknorm
}  // namespace lsgd
