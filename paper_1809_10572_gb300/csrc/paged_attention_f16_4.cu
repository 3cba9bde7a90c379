// paged_attention_f16_4.cu -- instances of paged_attention_kernel.cuh.
#include "paged_attention_kernel.cuh"

namespace samd {
namespace kv {
cudaError_t launch_att_f16_4(const AttArgs &a, int nb, int grid, cudaStream_t s) {
  return launch_dims<__half, 4>(a, nb, grid, s);
}
}  // namespace kv
}  // namespace samd
