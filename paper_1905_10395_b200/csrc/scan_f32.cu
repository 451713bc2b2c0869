// The scan's kernels for f32 activations.
#include "scan.h"

namespace lsgd {
namespace scan {
cudaError_t launch_forward_f32(const Args& a, const Launch& l, cudaStream_t s) { return forward_any<float>(a, l, s); }
cudaError_t launch_backward_f32(const Args& a, const Launch& l, cudaStream_t s) { return backward_any<float>(a, l, s); }
cudaError_t launch_join_f32(const Args& a, cudaStream_t s) { return launch_join<float>(a, s); }
}  // namespace scan
}  // namespace lsgd
