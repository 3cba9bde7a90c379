// moe4_bf16.cu -- instances of moe4_kernel.cuh.
#include "moe4_kernel.cuh"

namespace samd {
namespace moe {
cudaError_t launch_bf16(const MoeArgs &a, bool gated, cudaStream_t s) { return launch_type<__nv_bfloat16>(a, gated, s); }
}  // namespace moe
}  // namespace samd
