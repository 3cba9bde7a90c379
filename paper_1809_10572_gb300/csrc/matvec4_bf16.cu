// matvec4_bf16.cu -- the matrix-vector kernels for bf16 tokens.
#include "matvec4_kernel.cuh"

namespace samd {
namespace mv {
cudaError_t launch_bf16(const MvArgs &a, cudaStream_t s) { return launch_type<__nv_bfloat16>(a, s); }
}  // namespace mv
}  // namespace samd
