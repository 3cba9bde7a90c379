// Host-only: from which number of rows the matrix-vector kernel gives a CTA two
// row tiles, by the number of SMs. Compiled and run by tests/test_ffn_plan_cpu.py.
#include "../paper_1809_10572_gb300/csrc/matvec4_kernel.cuh"

#include <cstdio>

namespace samd {
int sms;
int sm_count() { return sms; }
}  // namespace samd

int main() {
  for (int s : {100, 148, 152, 160}) {
    samd::sms = s;
    int n = 1;
    while (!samd::mv::two_row_tiles(n)) ++n;
    printf("%d %d\n", s, n);
  }
  return 0;
}
