// moe4_f16.cu -- instances of moe4_kernel.cuh.
#include "moe4_kernel.cuh"

namespace samd {
namespace moe {
cudaError_t launch_f16(const MoeArgs &a, bool gated, cudaStream_t s) { return launch_type<__half>(a, gated, s); }
}  // namespace moe
}  // namespace samd
