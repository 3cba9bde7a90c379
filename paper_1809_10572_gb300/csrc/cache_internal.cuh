// cache_internal.cuh -- what the translation units of the packed key-value
// cache share: where a token's row lies, the sizes of a row, launchers.
#pragma once

#include "ffn_internal.cuh"

namespace samd {
namespace kv {

constexpr int kStep = 16;  // tokens the attention takes at a time: a page holds whole steps

// Sequences as the kernels see them. page is a power of two of at least kStep.
struct Seqs {
  const int32_t *table, *lengths;
  int64_t ld;
  int seqs, max_pages, pages, page_shift;
};

inline Seqs make_seqs(const samd_cache &c, const samd_cache_seqs &s) {
  Seqs q = {s.table, s.lengths, s.ld, s.seqs, s.max_pages, c.pages, 0};
  while ((1 << q.page_shift) < c.page) ++q.page_shift;
  return q;
}

// Tokens of sequence b: what its pages can hold at most.
__host__ __device__ __forceinline__ int64_t length_of(const Seqs &s, int b) {
  const int64_t n = s.lengths[b], most = static_cast<int64_t>(s.max_pages) << s.page_shift;
  return n < 0 ? 0 : n > most ? most : n;
}

// The page that holds token `pos` of sequence b, -1 where the table names none of the cache's pages.
__host__ __device__ __forceinline__ int page_of(const Seqs &s, int b, int64_t pos) {
  const int p = s.table[b * s.ld + (pos >> s.page_shift)];
  return static_cast<unsigned>(p) < static_cast<unsigned>(s.pages) ? p : -1;
}

// Where the row of new token i lies in a cache of one head: page * slots + slot; -1: it has no place; -2: it is no
// sequence's. starts: see samd_cache_append.
__host__ __device__ __forceinline__ int64_t place_of(const Seqs &s, const int32_t *starts, int token) {
  int b = token, n = 1, i = 0;
  if (starts) {
    if (token < starts[0] || token >= starts[s.seqs]) return -2;
    int hi = s.seqs;  // starts[b] <= token < starts[hi]
    b = 0;
    while (hi - b > 1) {
      const int mid = (b + hi) >> 1;
      if (starts[mid] <= token)
        b = mid;
      else
        hi = mid;
    }
    const int first = starts[b];
    n = starts[b + 1] - first;
    i = token - first;
  }
  const int64_t pos = static_cast<int64_t>(s.lengths[b]) - n + i;
  if (pos < 0 || pos >= static_cast<int64_t>(s.max_pages) << s.page_shift) return -1;
  const int page = page_of(s, b, pos);
  if (page < 0) return -1;
  return (static_cast<int64_t>(page) << s.page_shift) + (pos & ((1 << s.page_shift) - 1));
}

// The same row of head h of `heads`.
__host__ __device__ __forceinline__ int64_t row_of(const Seqs &s, int64_t place, int heads, int h) {
  return place + ((place >> s.page_shift) * (heads - 1) + h) * (int64_t(1) << s.page_shift);
}

}  // namespace kv

cudaError_t launch_cache_append(const samd_cache &c, const samd_cache_seqs &s, const int32_t *starts, int tokens,
                                const void *k, int64_t ldk, const void *v, int64_t ldv, cudaStream_t stream);
cudaError_t launch_cache_read(const samd_cache &c, const samd_cache_seqs &s, const int32_t *starts, int tokens, void *k,
                              int64_t ldk, void *v, int64_t ldv, cudaStream_t stream);
size_t paged_attention_workspace(const samd_cache &c, const samd_cache_seqs &s, int q_heads, bool scores);
cudaError_t launch_paged_attention(const samd_cache &c, const samd_cache_seqs &s, int q_heads, const void *q,
                                   int64_t ldq, float scale, void *out, int64_t ldo, float *scores, int64_t ld_scores,
                                   void *workspace, cudaStream_t stream);
cudaError_t launch_cache_evict(const samd_cache &c, const samd_cache_seqs &s, const samd_cache_seqs &dst,
                               const float *scores, int64_t ld_scores, int keep, int recent, int32_t *kept,
                               int32_t *new_lengths, float *new_scores, cudaStream_t stream);

}  // namespace samd
