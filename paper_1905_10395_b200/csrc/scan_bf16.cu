// The scan's kernels for bf16 activations.
#include "scan.h"

namespace lsgd {
namespace scan {
cudaError_t launch_forward_bf16(const Args& a, const Launch& l, cudaStream_t s) { return forward_any<__nv_bfloat16>(a, l, s); }
cudaError_t launch_backward_bf16(const Args& a, const Launch& l, cudaStream_t s) { return backward_any<__nv_bfloat16>(a, l, s); }
}  // namespace scan
}  // namespace lsgd
