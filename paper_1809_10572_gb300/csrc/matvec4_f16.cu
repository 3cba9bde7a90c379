// matvec4_f16.cu -- the matrix-vector kernels for f16 tokens.
#include "matvec4_kernel.cuh"

namespace samd {
namespace mv {
cudaError_t launch_f16(const MvArgs &a, cudaStream_t s) { return launch_type<__half>(a, s); }
}  // namespace mv
}  // namespace samd
