// cache_evict.cu -- which tokens of a cached head stay, by the weight that they
// got, and their rows into other pages.
//
// Choosing: a row of scores (one key head of one sequence) is a cluster of one
// to eight CTAs, each with a run of 8192 tokens in its registers. The score
// under which nothing stays is found digit by digit, 11, 11 and 10 bits from the
// top: a histogram of the tokens that agree so far, in each CTA's shared memory,
// added up over the cluster (distributed shared memory) by every CTA for itself.
// What is above it stays, and the first ones at it, as many as are missing; a
// token's place among the kept is a count of those before it. Rows of more
// tokens than a cluster holds are read again for every digit. Bound by latency:
// four passes with a barrier each; the scores are read once (128 rows of up to 8192
// tokens 14 us; 20 when the kept ones were read again).
//
// Copying: one pass over the kept rows, 16 bytes a thread for keys and for
// values, four of each in flight (119 MB in 23 us, 0.77 of the copy bandwidth; one of
// each 25); bound by HBM. New pages and not moves within the old ones, so that
// nothing has to be ordered, and pages that sequences share stay as they are.
#include "cache_internal.cuh"
#include "tc_ptx.cuh"

namespace samd {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kKeys = 16;                    // of a thread
constexpr int kChunk = kThreads * kKeys;     // tokens of a CTA at a time
constexpr int kMaxCluster = 8;
constexpr int kBins = 2048;
constexpr int kRanges = kWarps * kKeys;      // of 32 neighbouring tokens

struct EvictArgs {
  kv::Seqs s;
  const float *scores;
  int64_t ld_scores;
  int heads, keep, recent;
  int32_t *kept, *new_lengths;
  float *new_scores;
};

// Scores as unsigned integers of the same order: -0 as +0, NaN below everything.
__device__ __forceinline__ uint32_t order_of(float f) {
  if (f != f) return 0u;
  const uint32_t u = __float_as_uint(f + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ uint4 ld_cluster_u4(uint32_t addr, uint32_t rank) {
  const float4 v = ptx::ld_cluster_v4(ptx::map_to_rank(addr, rank));
  return make_uint4(__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w));
}

// Sum over the threads before this one; *all: over all of them. (Barriers of the CTA inside; tmp: kWarps words.)
__device__ __forceinline__ uint32_t sum_before(uint32_t v, uint32_t *tmp, uint32_t *all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t up = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += up;
  }
  __syncthreads();
  if (lane == 31) tmp[warp] = incl;
  __syncthreads();
  uint32_t before = 0;
  *all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += tmp[w];
    *all += tmp[w];
  }
  return before + incl - v;
}

template <bool kHeld>
__global__ void __launch_bounds__(kThreads) cache_choose_kernel(const EvictArgs a, int cluster) {
  __shared__ __align__(16) uint32_t hist[3][kBins];
  __shared__ uint32_t range[2][kRanges];  // of every 32 tokens: kept above the score, and at it; then the sums before
  __shared__ uint32_t tmp[kWarps];
  __shared__ __align__(16) uint32_t counts[4];  // of the CTA, for the others
  __shared__ uint32_t found[2];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row = blockIdx.x / cluster, rank = blockIdx.x - row * cluster;
  const int b = row / a.heads;
#pragma unroll
  for (int i = 0; i < 3 * kBins / kThreads; ++i) (&hist[0][0])[i * kThreads + tid] = 0;
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();
  const int n = static_cast<int>(kv::length_of(a.s, b));
  const float *const scores = a.scores + row * a.ld_scores;
  const int64_t out = static_cast<int64_t>(row) * a.keep;
  if (rank == 0 && row % a.heads == 0 && tid == 0) a.new_lengths[b] = n < a.keep ? n : a.keep;
  auto score_at = [&](int64_t i) { return i < a.ld_scores ? scores[i] : 0.0f; };

  if (n <= a.keep) {  // (the whole cluster)
    for (int64_t i = rank * kThreads + tid; i < a.keep; i += cluster * kThreads) {
      a.kept[out + i] = i < n ? static_cast<int>(i) : -1;
      if (a.new_scores) a.new_scores[out + i] = i < n ? score_at(i) : 0.0f;
    }
    return;
  }
  const int old = n - a.recent;  // tokens behind these stay
  auto key_of = [&](int64_t i, float f) { return i >= old ? 0xFFFFFFFFu : order_of(f); };
  auto key_at = [&](int64_t i) { return key_of(i, score_at(i)); };
  // this CTA's tokens: [first, last), a run of the row
  const int64_t per = kHeld ? kChunk : (static_cast<int64_t>((n + cluster - 1) / cluster) + kChunk - 1) / kChunk * kChunk;
  const int64_t first = rank * per, last = first + per < n ? first + per : n;
  float score[kKeys];
  if constexpr (kHeld) {
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      const int64_t at = first + i * kThreads + tid;
      score[i] = at < last ? score_at(at) : 0.0f;
    }
  }
  __syncthreads();  // the histograms are zero

  uint32_t prefix = 0, want = a.keep;  // the digits found; how many of those that agree with them stay
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    auto count = [&](uint32_t k) {
      if (pass == 0 || k >> ((shift + bits) & 31) == prefix >> ((shift + bits) & 31))
        atomicAdd(&hist[pass][(k >> shift) & ((1u << bits) - 1)], 1u);
    };
    if constexpr (kHeld) {
#pragma unroll
      for (int i = 0; i < kKeys; ++i)
        if (first + i * kThreads + tid < last) count(key_of(first + i * kThreads + tid, score[i]));
    } else {
      for (int64_t at = first + tid; at < last; at += kThreads) count(key_at(at));
    }
    __syncthreads();
    if (cluster > 1) ptx::cluster_sync();
    // four bins a thread, from the top down
    const int bin = kBins - 4 - 4 * tid;
    uint4 c = *reinterpret_cast<const uint4 *>(&hist[pass][bin]);
    if (cluster > 1) {
      c = make_uint4(0, 0, 0, 0);
      const uint32_t at = ptx::smem_addr(&hist[pass][bin]);
      for (int r = 0; r < cluster; ++r) {
        const uint4 v = ld_cluster_u4(at, r);
        c.x += v.x, c.y += v.y, c.z += v.z, c.w += v.w;
      }
    }
    uint32_t all;
    uint32_t above = sum_before(c.x + c.y + c.z + c.w, tmp, &all);
    const uint32_t four[4] = {c.w, c.z, c.y, c.x};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (above < want && above + four[i] >= want) {
        found[0] = prefix | static_cast<uint32_t>(bin + 3 - i) << shift;
        found[1] = want - above;
      }
      above += four[i];
    }
    __syncthreads();
    prefix = found[0];
    want = found[1];
    // (found and tmp are written again only behind the next pass's barriers)
  }

  // Kept: keys above `prefix`, and the first `want` that equal it.
  uint32_t n_gt = 0, n_eq = 0;
  if constexpr (kHeld) {
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      const int64_t at = first + i * kThreads + tid;
      const uint32_t k = key_of(at, score[i]);
      const uint32_t gt = __ballot_sync(0xffffffffu, at < last && k > prefix), eq = __ballot_sync(0xffffffffu, at < last && k == prefix);
      if (lane == 0) range[0][i * kWarps + warp] = __popc(gt), range[1][i * kWarps + warp] = __popc(eq);
    }
    __syncthreads();
    const uint32_t g = tid < kRanges ? range[0][tid] : 0, e = tid < kRanges ? range[1][tid] : 0;
    const uint32_t bg = sum_before(g, tmp, &n_gt), be = sum_before(e, tmp, &n_eq);
    if (tid < kRanges) range[0][tid] = bg, range[1][tid] = be;
  } else {
    uint32_t g = 0, e = 0;
    for (int64_t at = first + tid; at < last; at += kThreads) {
      const uint32_t k = key_at(at);
      g += k > prefix, e += k == prefix;
    }
    sum_before(g, tmp, &n_gt);
    sum_before(e, tmp, &n_eq);
  }
  uint32_t gt0 = 0, eq0 = 0;  // in the CTAs before
  if (cluster > 1) {
    if (tid == 0) counts[0] = n_gt, counts[1] = n_eq;
    __syncthreads();
    ptx::cluster_sync();
    for (int r = 0; r < rank; ++r) {
      const uint4 v = ld_cluster_u4(ptx::smem_addr(counts), r);
      gt0 += v.x, eq0 += v.y;
    }
  }
  __syncthreads();
  auto put = [&](int64_t at, float f, bool gt, bool eq, uint32_t gts, uint32_t eqs) {
    if (gt || (eq && eqs < want)) {
      const uint32_t to = gts + (eqs < want ? eqs : want);
      a.kept[out + to] = static_cast<int>(at);
      if (a.new_scores) a.new_scores[out + to] = f;
    }
  };
  const uint32_t below = (1u << lane) - 1;
  if constexpr (kHeld) {
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      const int64_t at = first + i * kThreads + tid;
      const uint32_t k = key_of(at, score[i]);
      const bool gt = at < last && k > prefix, eq = at < last && k == prefix;
      const uint32_t g = __ballot_sync(0xffffffffu, gt), e = __ballot_sync(0xffffffffu, eq);
      put(at, score[i], gt, eq, gt0 + range[0][i * kWarps + warp] + __popc(g & below), eq0 + range[1][i * kWarps + warp] + __popc(e & below));
    }
  } else {
    for (int64_t base = first; base < last; base += kThreads) {
      const int64_t at = base + tid;
      const float f = at < last ? score_at(at) : 0.0f;
      const uint32_t k = key_of(at, f);
      const bool gt = at < last && k > prefix, eq = at < last && k == prefix;
      uint32_t all_gt, all_eq;
      const uint32_t g = sum_before(gt, tmp, &all_gt), e = sum_before(eq, tmp, &all_eq);
      put(at, f, gt, eq, gt0 + g, eq0 + e);
      gt0 += all_gt, eq0 += all_eq;
    }
  }
  __syncwarp();
  if (cluster > 1) ptx::cluster_sync();  // no CTA ends while another reads its counts
}

struct CopyArgs {
  kv::Seqs s, dst;
  const int32_t *kept;
  uint8_t *lanes[2], *scales[2];
  int heads, keep;
  int units, parts;      // 16-byte units of a row of lanes; pieces of a row of scales
  int unit_mul, part_mul;  // 2^16 / them, and one more: a division of less than 32 * 16
  int64_t rows, chunks;  // pairs of a sequence and a head; runs of 32 kept rows of one
  IndexDiv by_chunks, by_heads;
};

// A warp copies 32 kept rows of one head: lane r finds out where row r comes from and goes to, then all lanes copy units
// of all rows, four of keys and four of values in flight. Part: two bytes of scales, or four where a row has an even number.
template <typename Part>
__global__ void __launch_bounds__(256) cache_copy_kernel(const CopyArgs a) {
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();
  const int lane = threadIdx.x & 31;
  const int64_t tasks = a.rows * a.chunks;
  for (int64_t task = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5); task < tasks; task += static_cast<int64_t>(gridDim.x) * 8) {
    const int64_t bh = idiv(task, a.by_chunks);
    const int r = static_cast<int>(task - bh * a.chunks) * 32 + lane;
    const int b = static_cast<int>(idiv(bh, a.by_heads)), h = static_cast<int>(bh - static_cast<int64_t>(b) * a.heads);
    const int from = r < a.keep ? a.kept[bh * a.keep + r] : -1;
    const int sp = from < 0 ? -1 : kv::page_of(a.s, b, from), dp = from < 0 ? -1 : kv::page_of(a.dst, b, r);
    const int mask = (1 << a.s.page_shift) - 1;
    const bool on = sp >= 0 && dp >= 0;
    const int64_t src = on ? ((static_cast<int64_t>(sp) * a.heads + h) << a.s.page_shift) + (from & mask) : -1;
    const int64_t dst = on ? ((static_cast<int64_t>(dp) * a.heads + h) << a.s.page_shift) + (r & mask) : 0;
    for (int i0 = 0; i0 < a.units; i0 += 4) {
      uint4 v[4][2];
      int64_t to[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int idx = (i0 + i) * 32 + lane, row = (idx * a.unit_mul) >> 16, u = idx - row * a.units;
        const int64_t s = __shfl_sync(0xffffffffu, src, row & 31);
        to[i] = __shfl_sync(0xffffffffu, dst, row & 31) * a.units + u;
        if (row > 31 || s < 0) {
          to[i] = -1;
        } else {
#pragma unroll
          for (int m = 0; m < 2; ++m) v[i][m] = *reinterpret_cast<const uint4 *>(a.lanes[m] + (s * a.units + u) * 16);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (to[i] >= 0)
#pragma unroll
          for (int m = 0; m < 2; ++m) *reinterpret_cast<uint4 *>(a.lanes[m] + to[i] * 16) = v[i][m];
    }
    for (int i = 0; i < a.parts; ++i) {
      const int idx = i * 32 + lane, row = (idx * a.part_mul) >> 16, u = idx - row * a.parts;
      const int64_t s = __shfl_sync(0xffffffffu, src, row), d = __shfl_sync(0xffffffffu, dst, row);
      if (s >= 0)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          Part *const p = reinterpret_cast<Part *>(a.scales[m]);
          p[d * a.parts + u] = p[s * a.parts + u];
        }
    }
  }
}

template <typename Part>
cudaError_t launch_copy(CopyArgs a, int blocks, cudaStream_t stream) {
  constexpr auto kern = cache_copy_kernel<Part>;
  a.parts = blocks * 2 / static_cast<int>(sizeof(Part));
  a.part_mul = 65536 / a.parts + 1;
  return launch_dependent(kern, dim3(resident_grid<kern>(a.rows * a.chunks * 32, 256)), 256, 0, stream, 1, a);
}

}  // namespace

cudaError_t launch_cache_evict(const samd_cache &c, const samd_cache_seqs &s, const samd_cache_seqs &dst,
                               const float *scores, int64_t ld_scores, int keep, int recent, int32_t *kept,
                               int32_t *new_lengths, float *new_scores, cudaStream_t stream) {
  EvictArgs e = {kv::make_seqs(c, s), scores, ld_scores, c.heads, keep, recent, kept, new_lengths, new_scores};
  const int64_t rows = static_cast<int64_t>(s.seqs) * c.heads, most = static_cast<int64_t>(s.max_pages) * c.page;
  int cluster = 1;
  while (cluster < kMaxCluster && static_cast<int64_t>(cluster) * kChunk < most) cluster *= 2;
  const bool held = static_cast<int64_t>(cluster) * kChunk >= most;
  const dim3 grid(static_cast<unsigned>(rows * cluster));
  cudaError_t err = held ? launch_dependent(cache_choose_kernel<true>, grid, kThreads, 0, stream, cluster, e, cluster)
                         : launch_dependent(cache_choose_kernel<false>, grid, kThreads, 0, stream, cluster, e, cluster);
  if (err != cudaSuccess) return err;
  CopyArgs a = {};
  a.s = e.s, a.dst = kv::make_seqs(c, dst), a.kept = kept;
  a.lanes[0] = static_cast<uint8_t *>(c.k_lanes), a.lanes[1] = static_cast<uint8_t *>(c.v_lanes);
  a.scales[0] = static_cast<uint8_t *>(c.k_scales), a.scales[1] = static_cast<uint8_t *>(c.v_scales);
  a.heads = c.heads, a.keep = keep;
  a.units = c.dim * c.fmt.bits / 128, a.unit_mul = 65536 / a.units + 1;
  a.rows = rows, a.chunks = (keep + 31) / 32;
  a.by_chunks = make_index_div(rows * a.chunks, a.chunks);
  a.by_heads = make_index_div(rows, c.heads);
  const int blocks = c.dim / 32;
  return blocks % 2 == 0 ? launch_copy<uint32_t>(a, blocks, stream) : launch_copy<uint16_t>(a, blocks, stream);
}

}  // namespace samd
