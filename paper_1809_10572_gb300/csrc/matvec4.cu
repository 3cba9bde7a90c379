// matvec4.cu -- host side of the 4-bit matrix-vector products; the kernel is in
// matvec4_kernel.cuh, its instances in matvec4_bf16.cu and matvec4_f16.cu.
#include "matvec4_kernel.cuh"

namespace samd {

// act < 0 (wu null): one matrix.
cudaError_t launch_matvec4(const samd_matvec_desc &d, int act, samd_fmt fw, const void *x, const samd_weights4 &wg,
                           const samd_weights4 *wu, void *y, cudaStream_t s) {
  mv::MvArgs a = {};
  const samd_weights4 *const w[2] = {&wg, wu ? wu : &wg};
  for (int i = 0; i < 2; ++i) {
    a.lanes[i] = static_cast<const uint8_t *>(w[i]->lanes);
    a.scales[i] = static_cast<const uint8_t *>(w[i]->scales);
    a.zeros[i] = w[i]->zeros;
  }
  a.ldx = d.ldx;
  a.ldy = d.ldy;
  a.row_bytes = words_per_row(fw, d.K) * (fw.word_bits / 8);
  while ((1 << a.group_shift) < d.group && (1 << a.group_shift) < d.K) ++a.group_shift;
  if (a.group_shift < 5) a.group_shift = 5;
  a.groups = (d.K + (1LL << a.group_shift) - 1) >> a.group_shift;
  a.n_scales = a.groups * d.N;
  a.N = d.N;
  a.K = d.K;
  a.tma = a.row_bytes % 16 == 0;
  if (a.tma) {
    const cudaError_t e = device_status_ptr(&a.status);
    if (e != cudaSuccess) return e;
  }
  a.x_vec = d.M == 1 || d.ldx % 8 == 0;
  a.is_signed = fw.is_signed;
  a.act = act;
  // the grid's second axis counts up to 65535 blocks of tokens
  constexpr int kMost = 65535 * 8;
  for (int m = 0; m < d.M; m += kMost) {
    a.M = d.M - m < kMost ? d.M - m : kMost;
    a.x = static_cast<const uint8_t *>(x) + m * d.ldx * 2;
    a.y = static_cast<uint8_t *>(y) + m * d.ldy * 2;
    const cudaError_t e = d.type == SAMD_BF16 ? mv::launch_bf16(a, s) : mv::launch_f16(a, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace samd
