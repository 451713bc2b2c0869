// The block-boundary kernels of blocknorm.h for bf16 residual and activations (a file for each pair of types: they compile side by side).
#define LSGD_BLOCKNORM_KERNELS
#include "blocknorm.h"

namespace lsgd {
namespace blocknorm {
cudaError_t launch_bf16_bf16(const Args& a, const Launch& l, cudaStream_t s) { return launch_types<bf16, bf16>(a, l, s); }
}  // namespace blocknorm
}  // namespace lsgd
