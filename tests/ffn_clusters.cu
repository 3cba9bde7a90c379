// Host-only: the gated block's counts of resident clusters are a device's, and
// a query that failed is asked again. The runtime's answers are replaced; no
// kernel is launched. Compiled and run by tests/test_ffn_plan_cpu.py.
#include <cuda_runtime.h>

namespace fake {
int device = 0, asked = 0;
cudaError_t answer = cudaSuccess;
cudaError_t get_device(int *d) {
  *d = device;
  return cudaSuccess;
}
template <typename K>
cudaError_t max_clusters(int *n, K, const cudaLaunchConfig_t *) {
  ++asked;
  *n = 10 + device;
  return answer;
}
}  // namespace fake
#define cudaGetDevice fake::get_device
#define cudaOccupancyMaxActiveClusters fake::max_clusters

#include "../paper_1809_10572_gb300/csrc/ffn.cu"

namespace samd {
int sm_count() { return 152; }
cudaError_t device_status_ptr(int **) { return cudaErrorInvalidValue; }
EncodeTiledFn tensor_map_encoder() { return nullptr; }
namespace conv {
cudaError_t ensure_smem_attr(const void *, size_t) { return cudaErrorInvalidValue; }
}  // namespace conv
}  // namespace samd

#include <cstdio>

int main() {
  using namespace samd;
  constexpr auto kern = ffn_gemm_kernel<DX, __half, 0, 64, true>;
  auto ask = [&](int device, cudaError_t answer) {
    fake::device = device;
    fake::answer = answer;
    return resident_clusters<kern>(4, 1024);
  };
  const int failed = ask(0, cudaErrorInvalidValue), first = ask(0, cudaSuccess), again = ask(0, cudaErrorInvalidValue);
  const int other = ask(1, cudaSuccess), back = ask(0, cudaSuccess);
  printf("failed %d first %d again %d other %d back %d asked %d\n", failed, first, again, other, back, fake::asked);
  return 0;
}
