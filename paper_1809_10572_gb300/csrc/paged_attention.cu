// paged_attention.cu -- host side of the attention over a packed cache, and the
// kernel that joins what several CTAs have of a head and counts the tokens'
// weights; the attention itself is in paged_attention_kernel.cuh.
#include "paged_attention_kernel.cuh"

namespace samd {
namespace kv {
namespace {

constexpr int kJoinThreads = 256;
constexpr int kMaxSlots = 1024;

// Up to this many steps a head is one CTA's work, and nothing is joined: 16 tokens for each of four warps, four times.
constexpr int kWholeSteps = 16;

struct JoinArgs {
  AttArgs a;
  int dim;
  int joins;  // CTAs of the grid's second axis that join a head; those behind them count weights
  float *scores;
  int64_t ld_scores;
};

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Reference and sum of weights of part i (0 .. n - 1) of head `h` of a unit whose parts lie in slots from s0 on.
__device__ __forceinline__ float2 stat_of(const AttArgs &a, int64_t unit_part, int part, int s0, int i, int h) {
  return i == 0 ? a.head_stat[unit_part * kHeads + h] : a.stat[(static_cast<int64_t>(s0 + i) * a.parts + part) * kHeads + h];
}

// The head's reference and sum of weights over all its parts, by one warp.
__device__ __forceinline__ float2 stat_all(const AttArgs &a, int64_t unit_part, int part, int2 span, int h, int lane) {
  const int n = span.y - span.x + 1;
  float top = -3e38f, weight = 0.0f;
  for (int i = lane; i < n; i += 32) {
    const float2 s = stat_of(a, unit_part, part, span.x, i, h);
    const float now = fmaxf(top, s.x);
    weight = fmaf(weight, exp2_of(top - now), s.y * exp2_of(s.x - now));
    top = now;
  }
  const float all = warp_max(top);
  return make_float2(all, warp_sum(weight * exp2_of(top - all)));
}

// What a thread has of a head: four elements' sums and the sum of weights, under a reference.
struct Joined {
  float4 v;
  float top, weight;

  __device__ __forceinline__ void add(const float4 &p, float2 s) {
    const float now = fmaxf(top, s.x), mine = exp2_of(top - now), its = exp2_of(s.x - now);
    v.x = fmaf(v.x, mine, p.x * its), v.y = fmaf(v.y, mine, p.y * its);
    v.z = fmaf(v.z, mine, p.z * its), v.w = fmaf(v.w, mine, p.w * its);
    weight = fmaf(weight, mine, s.y * its);
    top = now;
  }
};

template <typename T>
__global__ void __launch_bounds__(kJoinThreads) paged_attention_join(const JoinArgs j) {
  __shared__ Joined red[kJoinThreads];
  extern __shared__ float2 head[];  // with scores: reference and 1 / sum of weights of the unit's query heads
  const AttArgs &a = j.a;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();
  const int64_t unit_part = blockIdx.x;
  const int unit = blockIdx.x / a.parts, part = blockIdx.x - unit * a.parts;
  const int b = unit / a.heads, kv_head = unit - b * a.heads;
  const int n_heads = min(a.per, a.group - part * a.per);
  const int head0 = kv_head * a.group + part * a.per;
  const int len = static_cast<int>(length_of(a.s, b));

  if (static_cast<int>(blockIdx.y) < j.joins) {
    const int2 span = a.span[unit_part];  // (not yet written where there are no tokens)
    if (len == 0) {
      uint32_t *const out = reinterpret_cast<uint32_t *>(a.out + b * a.ldo + static_cast<int64_t>(head0) * j.dim * 2);
      if (blockIdx.y == 0)
        for (int i = tid; i < n_heads * j.dim / 2; i += kJoinThreads) out[i] = 0;
      return;
    }
    const int n = span.y - span.x + 1;
    if (n > 1) {
      // columns of four elements by groups of threads that take parts in turn
      const int cols = j.dim / 4, groups = kJoinThreads / cols, col = tid % cols, grp = tid / cols;
      for (int h = blockIdx.y; h < n_heads; h += j.joins) {
        Joined mine = {make_float4(0.0f, 0.0f, 0.0f, 0.0f), -3e38f, 0.0f};
        if (grp < groups)
#pragma unroll 4
          for (int i = grp; i < n; i += groups) {
            const int64_t cta = static_cast<int64_t>(span.x + i) * a.parts + part;
            mine.add(*reinterpret_cast<const float4 *>(a.sums + ((cta * 2 + (i == 0)) * kHeads + h) * j.dim + col * 4),
                     stat_of(a, unit_part, part, span.x, i, h));
          }
        red[tid] = mine;
        __syncthreads();
        if (grp == 0) {
          for (int i = 1; i < groups && i < n; ++i) {
            const Joined p = red[i * cols + col];
            mine.add(p.v, make_float2(p.top, p.weight));
          }
          const float inv = mine.weight == 0.0f ? 0.0f : 1.0f / mine.weight;
          *reinterpret_cast<uint2 *>(a.out + b * a.ldo + (static_cast<int64_t>(head0 + h) * j.dim + col * 4) * 2) =
              make_uint2(pack2<T>(mine.v.x * inv, mine.v.y * inv), pack2<T>(mine.v.z * inv, mine.v.w * inv));
        }
        __syncthreads();
      }
    }
    return;
  }

  if (part != 0 || len == 0) return;
  const int slice = blockIdx.y - j.joins, slices = gridDim.y - j.joins;
  for (int i = warp; i < a.group; i += kJoinThreads / 32) {
    const int p = i / a.per;
    const int2 span = a.whole ? make_int2(0, 0) : a.span[unit_part + p];
    const float2 all = stat_all(a, unit_part + p, p, span, i - p * a.per, lane);
    if (lane == 0) head[i] = make_float2(all.x, all.y == 0.0f ? 0.0f : 1.0f / all.y);
  }
  __syncthreads();
  const int64_t tokens = static_cast<int64_t>(a.s.max_pages) << a.s.page_shift;
  const int64_t end = len < j.ld_scores ? len : j.ld_scores;
  float *const row = j.scores + unit * j.ld_scores;
  for (int64_t t = static_cast<int64_t>(slice) * kJoinThreads + tid; t < end; t += static_cast<int64_t>(slices) * kJoinThreads) {
    float w = 0.0f;
    for (int p = 0; p < a.parts; ++p) {
      const float4 *const lp = reinterpret_cast<const float4 *>(a.logits + ((unit_part + p) * tokens + t) * kHeads);
      const int n = min(a.per, a.group - p * a.per);
      const float4 lo = lp[0], hi = n > 4 ? lp[1] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      const float x[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
      for (int i = 0; i < kHeads; ++i)
        if (i < n) {
          const float2 s = head[p * a.per + i];
          w = fmaf(exp2_of(x[i] - s.x), s.y, w);
        }
    }
    row[t] += w;
  }
}

// How a call is dealt out, and where its parts of the workspace lie.
struct Plan {
  int parts, per, slots, whole;
  int64_t units;
  size_t sums, stat, head_stat, span, logits, bytes;
};

Plan plan_of(const samd_cache &c, const samd_cache_seqs &s, int q_heads, bool scores) {
  Plan p = {};
  const int group = q_heads / c.heads;
  p.parts = (group + kHeads - 1) / kHeads;
  p.per = (group + p.parts - 1) / p.parts;
  p.units = static_cast<int64_t>(s.seqs) * c.heads;
  const int64_t tokens = static_cast<int64_t>(s.max_pages) * c.page;
  p.whole = tokens <= kWholeSteps * kStep;
  const int ctas = (c.fmt.bits == 8 ? ctas_of<8>(c.dim / 32) : ctas_of<4>(c.dim / 32)) * sm_count();
  int64_t slots = ctas / p.parts < 1 ? 1 : ctas / p.parts;
  if (slots > kMaxSlots) slots = kMaxSlots;
  const int64_t most = p.whole ? p.units : used_of(p.units * dealt_of(static_cast<int>((tokens + kStep - 1) / kStep)), p.units, kMaxSlots);
  p.slots = static_cast<int>(slots < most ? slots : most < 1 ? 1 : most);
  size_t at = 0;
  auto take = [&at](int64_t bytes) {
    const size_t was = at;
    at += static_cast<size_t>((bytes + 127) / 128 * 128);
    return was;
  };
  const int64_t grid = static_cast<int64_t>(p.slots) * p.parts;
  if (!p.whole) {
    p.sums = take(grid * 2 * kHeads * c.dim * 4);
    p.stat = take(grid * kHeads * 8);
    p.span = take(p.units * p.parts * 8);
  }
  if (!p.whole || scores) p.head_stat = take(p.units * p.parts * kHeads * 8);
  if (scores) p.logits = take(p.units * p.parts * tokens * kHeads * 4);
  p.bytes = at;
  return p;
}

}  // namespace
}  // namespace kv

size_t paged_attention_workspace(const samd_cache &c, const samd_cache_seqs &s, int q_heads, bool scores) {
  return kv::plan_of(c, s, q_heads, scores).bytes;
}

cudaError_t launch_paged_attention(const samd_cache &c, const samd_cache_seqs &s, int q_heads, const void *q,
                                   int64_t ldq, float scale, void *out, int64_t ldo, float *scores, int64_t ld_scores,
                                   void *workspace, cudaStream_t stream) {
  using namespace kv;
  const Plan p = plan_of(c, s, q_heads, scores != nullptr);
  uint8_t *const ws = static_cast<uint8_t *>(workspace);
  AttArgs a = {};
  a.s = make_seqs(c, s);
  a.k = static_cast<const uint8_t *>(c.k_lanes), a.v = static_cast<const uint8_t *>(c.v_lanes);
  a.ks = static_cast<const uint8_t *>(c.k_scales), a.vs = static_cast<const uint8_t *>(c.v_scales);
  a.q = static_cast<const uint8_t *>(q), a.out = static_cast<uint8_t *>(out);
  a.ldq = ldq * 2, a.ldo = ldo * 2;
  a.scale = scale;
  a.heads = c.heads, a.group = q_heads / c.heads;
  a.page_rows = static_cast<uint32_t>(c.heads) * static_cast<uint32_t>(c.page);
  a.parts = p.parts, a.per = p.per, a.slots = p.slots, a.whole = p.whole;
  if (!p.whole) {
    a.sums = reinterpret_cast<float *>(ws + p.sums);
    a.stat = reinterpret_cast<float2 *>(ws + p.stat);
    a.span = reinterpret_cast<int2 *>(ws + p.span);
  }
  if (!p.whole || scores) a.head_stat = reinterpret_cast<float2 *>(ws + p.head_stat);
  if (scores) a.logits = reinterpret_cast<float *>(ws + p.logits);
  const int nb = c.dim / 32, grid = p.slots * p.parts;
  cudaError_t e = c.type == SAMD_BF16
                      ? (c.fmt.bits == 8 ? launch_att_bf16_8(a, nb, grid, stream) : launch_att_bf16_4(a, nb, grid, stream))
                      : (c.fmt.bits == 8 ? launch_att_f16_8(a, nb, grid, stream) : launch_att_f16_4(a, nb, grid, stream));
  if (e != cudaSuccess || (p.whole && !scores)) return e;
  // few heads: more CTAs for each
  const int64_t ups = p.units * p.parts;
  auto share = [](int64_t all, int64_t of, int64_t most) {
    const int64_t n = (all + of - 1) / of;
    return static_cast<int>(n < 1 ? 1 : n < most ? n : most);
  };
  const int joins = p.whole ? 0 : share(4 * sm_count(), ups, p.per);
  const int64_t runs = (static_cast<int64_t>(s.max_pages) * c.page + kJoinThreads - 1) / kJoinThreads;
  const int slices = !scores ? 0 : share(8 * sm_count(), p.units, runs < 60000 ? runs < 1 ? 1 : runs : 60000);
  const JoinArgs j = {a, c.dim, joins, scores, ld_scores};
  const size_t smem = scores ? static_cast<size_t>(a.group) * sizeof(float2) : 0;
  const dim3 jgrid(static_cast<unsigned>(ups), static_cast<unsigned>(joins + slices));
  return c.type == SAMD_BF16 ? launch_dependent(paged_attention_join<__nv_bfloat16>, jgrid, kJoinThreads, smem, stream, 1, j)
                             : launch_dependent(paged_attention_join<__half>, jgrid, kJoinThreads, smem, stream, 1, j);
}

}  // namespace samd
