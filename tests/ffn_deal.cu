// Host-only: the dealing of a joint backward launch's tiles over its CTAs. Every
// tile goes to one CTA, once, whatever the numbers of tiles and of rounds, and
// DX's tiles come before DW's. Compiled and run by tests/test_ffn_plan_cpu.py.
#include "../paper_1809_10572_gb300/csrc/ffn.cu"

namespace samd {
int sms = 152;
int sm_count() { return sms; }
cudaError_t device_status_ptr(int **) { return cudaErrorInvalidValue; }
EncodeTiledFn tensor_map_encoder() { return nullptr; }
namespace conv {
cudaError_t ensure_smem_attr(const void *, size_t) { return cudaErrorInvalidValue; }
}  // namespace conv
}  // namespace samd

#include <cstdio>
#include <vector>

using namespace samd;

// What the kernel's roles do: their first tile, and one after the other.
bool dealt_right(int first, int total, int fill) {
  const int P = total < sm_count() ? total : sm_count();
  std::vector<unsigned char> seen(total, 0);
  long long n = 0;
  for (int c = 0; c < P; ++c) {
    int before = -1;
    for (int tile = c >= first ? dealt_next(c - P, c, P, first, fill) : c; tile < total;
         tile = dealt_next(tile, c, P, first, fill)) {
      if (tile < 0 || tile <= before || seen[tile]) return false;
      seen[tile] = 1;
      before = tile;
      ++n;
    }
  }
  return n == total;
}

int main() {
  long long n = 0, bad = 0;
  auto check = [&](int first, int w, int64_t steps_x, int64_t steps_w) {
    const int fill = deal_fill(first, first + w, fill_of(steps_x, steps_w));
    ++n;
    if (!dealt_right(first, first + w, fill) && ++bad < 10)
      printf("BAD %d SMs, %d and %d tiles, %lld and %lld steps: fill %d\n", sms, first, w, (long long)steps_x,
             (long long)steps_w, fill);
  };
  for (int s : {1, 2, 7, 148, 152}) {
    sms = s;
    for (int first : {1, 2, 3, 6, 7, 8, 100, 147, 148, 149, 151, 152, 153, 300, 304, 305, 1000})
      for (int w : {1, 2, 5, 64, 147, 151, 152, 153, 400, 3000})
        for (int64_t sx : {1, 2, 9, 50, 1000, 100000})
          for (int64_t sw : {1, 2, 13, 128, 5000}) check(first, w, sx, sw);
    // the longest reductions of a dx that the block's sizes allow, by weight gradients of one step
    for (int64_t sx : {int64_t(1) << 22, int64_t(1) << 24, int64_t(1) << 25}) check(1, 1 << 20, sx, 1), check(151, 1 << 20, sx, 1);
  }
  printf("dealt %lld, bad %lld\n", n, bad);
  return bad != 0;
}
