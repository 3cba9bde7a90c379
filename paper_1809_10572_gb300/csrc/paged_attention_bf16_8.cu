// paged_attention_bf16_8.cu -- instances of paged_attention_kernel.cuh.
#include "paged_attention_kernel.cuh"

namespace samd {
namespace kv {
cudaError_t launch_att_bf16_8(const AttArgs &a, int nb, int grid, cudaStream_t s) {
  return launch_dims<__nv_bfloat16, 8>(a, nb, grid, s);
}
}  // namespace kv
}  // namespace samd
