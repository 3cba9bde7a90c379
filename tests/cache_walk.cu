// Host-only: how the attention deals the steps of a batch over its CTAs, and
// where a new token's row lies. Every step of every key head is one CTA's, once,
// in order, and its rows lie in the cache, whatever the lengths, the table's
// entries and the number of CTAs; the first CTA of a head names the last.
// Compiled and run by tests/test_cache_plan_cpu.py.
#include "../paper_1809_10572_gb300/csrc/paged_attention.cu"

#include <cstdio>
#include <cstdlib>
#include <vector>

namespace samd {
int sm_count() { return 152; }
namespace conv {
cudaError_t ensure_smem_attr(const void *, size_t) { return cudaErrorInvalidValue; }
}  // namespace conv
namespace kv {
cudaError_t launch_att_bf16_8(const AttArgs &, int, int, cudaStream_t) { return cudaErrorInvalidValue; }
cudaError_t launch_att_bf16_4(const AttArgs &, int, int, cudaStream_t) { return cudaErrorInvalidValue; }
cudaError_t launch_att_f16_8(const AttArgs &, int, int, cudaStream_t) { return cudaErrorInvalidValue; }
cudaError_t launch_att_f16_4(const AttArgs &, int, int, cudaStream_t) { return cudaErrorInvalidValue; }
}  // namespace kv
}  // namespace samd

using namespace samd;
using namespace samd::kv;

static long long cases = 0, bad = 0;
static void fail(const char *what) {
  if (++bad < 10) printf("BAD case %lld: %s\n", cases, what);
}

static void walk(const std::vector<int32_t> &lengths, int heads, int slots, int max_pages, int shift, int whole) {
  ++cases;
  AttArgs a = {};
  a.s = Seqs{nullptr, lengths.data(), max_pages, static_cast<int>(lengths.size()), max_pages, 1, shift};
  a.heads = heads, a.slots = slots, a.whole = whole, a.parts = 1;
  std::vector<int64_t> first;  // of every unit, among all steps
  int64_t all = 0;
  for (int b = 0; b < a.s.seqs; ++b)
    for (int h = 0; h < heads; ++h) first.push_back(all), all += dealt_of(steps_of(a.s, b));
  const int units = a.s.seqs * heads;
  int64_t some = 0;
  for (int b = 0; b < a.s.seqs; ++b) some += steps_of(a.s, b) > 0;
  const int64_t used = whole ? slots : used_of(all, some * heads, slots);
  std::vector<int> done(units, 0), seen(units, 0), last_slot(units, -1), said(units, -2);
  for (int slot = 0; slot < slots; ++slot) {
    Walk w;
    if (whole) {
      w.start_whole(a, slot);
    } else {
      if (slot >= used) continue;
      const int64_t begin = begin_of(slot, all, used), end = begin_of(slot + 1, all, used);
      if (begin >= end) return fail("a CTA without a share");
      int b = 0;
      while (begin >= first[b * heads] + heads * dealt_of(steps_of(a.s, b))) ++b;
      w.start(a, b, begin - first[b * heads], begin, end - begin);
    }
    while (whole ? w.b * heads + w.h < units : w.on()) {
      const int u = w.b * heads + w.h;
      if (u < 0 || u >= units || w.steps != steps_of(a.s, w.b) || w.first != done[u] || w.last > w.steps)
        return fail("a part out of order");
      if (whole && (w.first != 0 || w.last != w.steps)) return fail("a head that is not whole");
      if (!whole && w.unit != first[u]) return fail("a head's place");
      if (w.first == 0) {
        if (seen[u]++) return fail("a head begun twice");
        if (!whole) said[u] = slot_of(w.unit + dealt_of(w.steps) - 1, all, used);
      }
      done[u] = w.last;
      last_slot[u] = slot;
      w.next(a);
    }
  }
  for (int u = 0; u < units; ++u) {
    if (done[u] != steps_of(a.s, u / heads)) return fail("steps left over");
    if (whole ? seen[u] != 1 : done[u] > 0 && said[u] != last_slot[u]) return fail("a head's last CTA");
  }
}

int main() {
  srand(1);
  const int lists[][6] = {{0}, {1}, {16}, {17}, {0, 0, 5, 0}, {1000000, 0, 0, 1}, {15, 16, 17, 0, 4096, 33}, {-5, 70, 99999999}};
  for (const auto &l : lists)
    for (int heads : {1, 3, 8})
      for (int slots : {1, 2, 57, 456})
        for (int whole = 0; whole < 2; ++whole)
          walk(std::vector<int32_t>(l, l + 6), heads, slots, whole ? 16 : 70000, 4, whole);
  for (int i = 0; i < 3000; ++i) {
    std::vector<int32_t> l(1 + rand() % 300);
    const int most = 1 + rand() % (i % 3 ? 300 : 20000);
    for (auto &n : l) n = rand() % 5 ? rand() % most : 0;
    walk(l, 1 + rand() % 12, 1 + rand() % 500, 1 + most / 16, 4, i % 4 == 3);
  }
  // rows of new tokens: inside the cache or refused, and each once, with any table, lengths and rising starts
  for (int i = 0; i < 2000; ++i) {
    ++cases;
    const int seqs = 1 + rand() % 9, width = rand() % 5, pages = 1 + rand() % 20, heads = 1 + rand() % 4, shift = 4 + rand() % 3;
    const int slots = 1 << shift;
    std::vector<int32_t> table(seqs * width + 1), lengths(seqs), starts(seqs + 1);
    for (auto &p : table) p = rand() % 4 ? rand() % pages : rand() % 3 ? -1 - rand() % 99 : rand();
    for (auto &n : lengths) n = rand() % 7 ? rand() % (width * slots + 9) : -rand() % 50;
    starts[0] = rand() % 3;
    for (int b = 0; b < seqs; ++b) starts[b + 1] = starts[b] + rand() % 40;
    const Seqs s = {table.data(), lengths.data(), width, seqs, width, pages, shift};
    for (int token = 0; token < starts[seqs] + 5; ++token) {
      int b = 0;
      while (b < seqs && token >= starts[b + 1]) ++b;
      const int64_t p = place_of(s, starts.data(), token);
      if (token < starts[0] || b == seqs) {
        if (p != -2) fail("a row of no sequence");
        continue;
      }
      const int64_t pos = static_cast<int64_t>(lengths[b]) - (starts[b + 1] - token);
      const bool in = pos >= 0 && pos < width * slots;
      const int page = in ? table[b * width + pos / slots] : -1;
      if (!in || page < 0 || page >= pages) {
        if (p != -1) fail("a token without a place");
        continue;
      }
      if (p != static_cast<int64_t>(page) * slots + pos % slots) fail("a token's place");
      for (int h = 0; h < heads; ++h)
        if (row_of(s, p, heads, h) != (static_cast<int64_t>(page) * heads + h) * slots + pos % slots) fail("a head's row");
    }
    for (int b = 0; b < seqs; ++b) {
      const int64_t pos = static_cast<int64_t>(lengths[b]) - 1, p = place_of(s, nullptr, b);
      if ((p >= 0) != (pos >= 0 && pos < width * slots && page_of(s, b, pos) >= 0)) fail("a token's place without starts");
    }
  }
  printf("cases %lld, bad %lld\n", cases, bad);
  return bad != 0;
}
