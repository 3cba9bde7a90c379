// moe4.cu -- which experts a token goes to, and the host side of the layer of
// experts; the layer's kernels are in moe4_kernel.cuh.
//
// Routing: a cluster of one to eight CTAs a token; every warp takes experts in
// turn, or slices of the inputs of few ones (16 bytes a lane of the router's row
// and of the token, products and sums in fp32); the logits meet in the first
// CTA, where one warp takes the largest, topk times. Bound by latency: the
// router's matrix comes from L2 for every token.
#include "moe4_kernel.cuh"

namespace samd {
namespace {

constexpr int kRouteThreads = 256;
constexpr int kRouteWarps = kRouteThreads / 32;
constexpr int kMaxCluster = 8;

struct RouteArgs {
  const uint8_t *x, *router;
  int64_t ldx;  // bytes
  int32_t *ids;
  float *weights;
  int K, E, topk, normalize, cluster;
  int slices, per;  // warps that share an expert, and the inputs of one (a multiple of 256, or all)
};

__device__ __forceinline__ uint32_t order_of(float f) {
  if (f != f) return 0u;  // below -infinity
  const uint32_t u = __float_as_uint(f + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <typename T>
__device__ __forceinline__ float dot8(uint4 a, uint4 b, float s) {
  const uint32_t u[4] = {a.x, a.y, a.z, a.w}, v[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 p = unpack2<T>(u[i]), q = unpack2<T>(v[i]);
    s = fmaf(p.x, q.x, s);
    s = fmaf(p.y, q.y, s);
  }
  return s;
}

template <typename T>
__global__ void __launch_bounds__(kRouteThreads) moe_route_kernel(const RouteArgs a) {
  __shared__ float logits[moe::kMaxExperts];
  __shared__ float parts[kRouteWarps * kMaxCluster];  // [expert][slice], where an expert has several
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t token = blockIdx.x / a.cluster;
  const int rank = blockIdx.x % a.cluster;
  if (a.cluster > 1) ptx::cluster_sync();  // the first CTA, which the others write to, has begun
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();
  const uint8_t *const x = a.x + token * a.ldx;
  float *const out = a.slices > 1 ? parts : logits;
  for (int task = rank * kRouteWarps + warp; task < a.E * a.slices; task += a.cluster * kRouteWarps) {
    const int e = task / a.slices, end = min(a.K, (task - e * a.slices + 1) * a.per);
    const uint8_t *const r = a.router + static_cast<int64_t>(e) * a.K * 2;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    int k = (task - e * a.slices) * a.per + lane * 8;
    for (; k + 3 * 256 < end; k += 4 * 256) {
      uint4 u[4], v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u[i] = *reinterpret_cast<const uint4 *>(r + (k + i * 256) * 2);
        v[i] = *reinterpret_cast<const uint4 *>(x + (k + i * 256) * 2);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = dot8<T>(u[i], v[i], s[i]);
    }
#pragma unroll 2
    for (; k < end; k += 256)
      s[0] = dot8<T>(*reinterpret_cast<const uint4 *>(r + k * 2), *reinterpret_cast<const uint4 *>(x + k * 2), s[0]);
    float v = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0) {
      if (a.cluster == 1)
        out[task] = v;
      else
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(ptx::map_to_rank(ptx::smem_addr(out + task), 0)), "f"(v) : "memory");
    }
  }
  __syncthreads();
  if (a.cluster > 1) ptx::cluster_sync();
  if (rank == 0 && warp == 0 && a.slices > 1) {
    for (int e = lane; e < a.E; e += 32) {
      float v = 0.0f;
      for (int i = 0; i < a.slices; ++i) v += parts[e * a.slices + i];
      logits[e] = v;
    }
    __syncwarp();
  }
  if (rank != 0 || warp != 0) return;

  float all_top = -INFINITY, all_sum = 0.0f;
  if (!a.normalize) {
    for (int e = lane; e < a.E; e += 32) all_top = fmaxf(all_top, logits[e]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all_top = fmaxf(all_top, __shfl_xor_sync(0xffffffffu, all_top, o));
    for (int e = lane; e < a.E; e += 32) all_sum += __expf(logits[e] - all_top);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all_sum += __shfl_xor_sync(0xffffffffu, all_sum, o);
  }
  // lane i keeps the i-th choice
  float mine = -INFINITY;
  int expert = 0;
  uint32_t taken = 0;  // of this lane's experts lane, lane + 32, ..
  for (int i = 0; i < a.topk; ++i) {
    uint32_t best = 0;
    int at = moe::kMaxExperts;
    for (int j = 0, e = lane; e < a.E; ++j, e += 32) {
      const uint32_t o = order_of(logits[e]);
      if (!(taken >> j & 1) && (at == moe::kMaxExperts || o > best)) best = o, at = e;
    }
    // the largest, and of equal ones the first: lanes without an expert left come behind all
    const uint32_t top = __reduce_max_sync(0xffffffffu, at < moe::kMaxExperts ? best : 0u);
    const int who = __reduce_min_sync(0xffffffffu, static_cast<unsigned>(at < moe::kMaxExperts && best == top ? at : moe::kMaxExperts));
    if ((who & 31) == lane) taken |= 1u << (who >> 5);
    if (lane == i) expert = who, mine = logits[who];
  }
  const float first = __shfl_sync(0xffffffffu, mine, 0);
  float w = lane < a.topk ? __expf(mine - (a.normalize ? first : all_top)) : 0.0f, sum = w;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (!a.normalize) sum = all_sum;
  if (lane < a.topk) {
    a.ids[token * a.topk + lane] = expert;
    a.weights[token * a.topk + lane] = __fdiv_rn(w, sum);
  }
}

int chunk_tokens(const samd_moe_desc &d) {
  const int most = moe::kMaxPairs / d.topk;
  return most < moe::kMaxTokens ? most : moe::kMaxTokens;
}

}  // namespace

cudaError_t launch_moe_route(const samd_moe_desc &d, bool normalize, const void *x, const void *router, int32_t *ids,
                             float *weights, cudaStream_t s) {
  // few experts: their inputs in slices of 512 or more, while the cluster has warps for them
  int slices = 1, cluster = 1;
  while (d.E * slices * 2 <= kMaxCluster * kRouteWarps && d.K >= 1024 * slices) slices *= 2;
  const int per = slices == 1 ? d.K : (d.K + slices * 256 - 1) / (slices * 256) * 256;
  while (cluster < kMaxCluster && cluster * kRouteWarps < d.E * slices) cluster *= 2;
  constexpr int kMost = 1 << 27;  // tokens of a launch: its CTAs are counted in 31 bits
  for (int64_t m = 0; m < d.M; m += kMost) {
    const int n = d.M - m < kMost ? static_cast<int>(d.M - m) : kMost;
    const RouteArgs a = {static_cast<const uint8_t *>(x) + m * d.ldx * 2, static_cast<const uint8_t *>(router), d.ldx * 2,
                         ids + m * d.topk, weights + m * d.topk, d.K, d.E, d.topk, normalize, cluster, slices, per};
    const cudaError_t e = d.type == SAMD_BF16
                              ? launch_dependent(moe_route_kernel<__nv_bfloat16>, dim3(n * cluster), kRouteThreads, 0, s, cluster, a)
                              : launch_dependent(moe_route_kernel<__half>, dim3(n * cluster), kRouteThreads, 0, s, cluster, a);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

size_t moe4_workspace(const samd_moe_desc &d) {
  const int64_t tokens = d.M < chunk_tokens(d) ? d.M : chunk_tokens(d);
  return static_cast<size_t>(tokens * d.topk) * static_cast<size_t>(d.F) * 2;
}

cudaError_t launch_moe4(const samd_moe_desc &d, samd_fmt fw, const void *x, const int32_t *ids, const float *weights,
                        const samd_weights4 &gate, const samd_weights4 &up, const samd_weights4 &down, void *y,
                        void *workspace, cudaStream_t s) {
  moe::MoeArgs a = {};
  a.E = d.E, a.topk = d.topk, a.act = d.act, a.is_signed = fw.is_signed;
  // a group of all inputs, or more, is one of the next power of two
  auto sized = [&](int N, int K) {
    a.N = N, a.K = K;
    a.group_shift = 5;
    while ((1 << a.group_shift) < d.group && (1 << a.group_shift) < K) ++a.group_shift;
    a.groups = (K + (int64_t(1) << a.group_shift) - 1) >> a.group_shift;
    a.row_bytes = K / 2;
  };
  auto matrix = [&](int i, const samd_weights4 &w) {
    a.lanes[i] = static_cast<const uint8_t *>(w.lanes);
    a.scales[i] = static_cast<const uint8_t *>(w.scales);
    a.zeros[i] = w.zeros;
  };
  auto run = [&](bool gated) { return d.type == SAMD_BF16 ? moe::launch_bf16(a, gated, s) : moe::launch_f16(a, gated, s); };
  const int most = chunk_tokens(d);
  for (int m = 0; m < d.M; m += most) {
    a.M = d.M - m < most ? d.M - m : most;
    a.ids = ids + static_cast<int64_t>(m) * d.topk;
    a.weights = weights + static_cast<int64_t>(m) * d.topk;
    sized(d.F, d.K);
    matrix(0, gate), matrix(1, up);
    a.x = static_cast<const uint8_t *>(x) + m * d.ldx * 2, a.ldx = d.ldx * 2;
    a.y = static_cast<uint8_t *>(workspace), a.ldy = static_cast<int64_t>(d.F) * 2;
    cudaError_t e = run(true);
    if (e != cudaSuccess) return e;
    sized(d.K, d.F);
    matrix(0, down), matrix(1, down);
    a.x = a.y, a.ldx = a.ldy;
    a.y = static_cast<uint8_t *>(y) + m * d.ldy * 2, a.ldy = d.ldy * 2;
    e = run(false);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace samd
