// block8.cu -- activations into their 8-bit form (blocks of 32 with one power
// of two, ffn_internal.cuh) and back.
//
// Both are one pass over HBM: 2 or 4 bytes an element on the wide side and
// 33/32 on the other. Two neighbouring lanes hold a block, sixteen elements
// each (two 16-byte loads of a 16-bit type, one 16-byte store of codes), and
// find its largest magnitude with a shuffle. Eight elements a thread, a 64-bit
// division a step and converted codes took 54.6 us for 8192 x 4096 bf16 there
// and back; this 35 (203 MB, 0.87 of the copy bandwidth), bound by HBM.
#include "ffn_internal.cuh"
#include "tc_ptx.cuh"

namespace samd {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 16;             // elements a thread handles at a time
constexpr int kRowStep = 32 * kPer;  // elements of a row a warp handles at a time

struct Block8Args {
  int64_t rows, inner, ld, segs;  // segs: warps' steps in a row
  int64_t wpr, bpr;               // words and blocks of a row
  IndexDiv by_segs;
  int x_vec, l_vec;               // rows of x, and of lanes, are 16-byte aligned
};

template <typename T>
__device__ __forceinline__ void load16(const T *p, int n, float *v) {
  if (n == kPer) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 f = __ldcs(reinterpret_cast<const float4 *>(p) + i);
        v[4 * i] = f.x, v[4 * i + 1] = f.y, v[4 * i + 2] = f.z, v[4 * i + 3] = f.w;
      }
    } else {
      const uint4 q[2] = {__ldcs(reinterpret_cast<const uint4 *>(p)), __ldcs(reinterpret_cast<const uint4 *>(p) + 1)};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t w[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 f = unpack2<T>(w[k]);
          v[8 * i + 2 * k] = f.x;
          v[8 * i + 2 * k + 1] = f.y;
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = i < n ? to_f32<T>(p[i]) : 0.0f;
  }
}

template <typename T>
__device__ __forceinline__ void store16(T *p, int n, const float *v) {
  if (n == kPer) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        __stcs(reinterpret_cast<float4 *>(p) + i, make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]));
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        __stcs(reinterpret_cast<uint4 *>(p) + i,
               make_uint4(pack2<T>(v[8 * i], v[8 * i + 1]), pack2<T>(v[8 * i + 2], v[8 * i + 3]),
                          pack2<T>(v[8 * i + 4], v[8 * i + 5]), pack2<T>(v[8 * i + 6], v[8 * i + 7])));
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (i < n) p[i] = from_f32<T>(v[i]);
  }
}

// Rows that are not 16-byte aligned go through shared memory, so that a warp's
// accesses are neighbouring elements: place i of the warp's 512 elements, one
// word further behind every sixteen, which puts the lanes' runs of sixteen into
// different banks.
__device__ __forceinline__ int place(int i) { return i + (i >> 4); }
constexpr int kStageWords = kRowStep + kRowStep / 16;

// The warp's 512 elements from `p`, of which the row holds `left` (at least
// one): sixteen for each lane, zeros past the row's end.
template <typename T>
__device__ __forceinline__ void load_staged(const T *p, int64_t left, float *stage, int lane, float *v) {
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int at = i * 32 + lane;
    stage[place(at)] = at < left ? to_f32<T>(p[at]) : 0.0f;
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kPer; ++i) v[i] = stage[place(lane * kPer) + i];
  __syncwarp();
}
template <typename T>
__device__ __forceinline__ void store_staged(T *p, int64_t left, float *stage, int lane, const float *v) {
#pragma unroll
  for (int i = 0; i < kPer; ++i) stage[place(lane * kPer) + i] = v[i];
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int at = i * 32 + lane;
    if (at < left) p[at] = from_f32<T>(stage[place(at)]);
  }
  __syncwarp();
}

// (No const __restrict__ parameters: they allow loads by the read-only path,
// which is for data that nothing writes while a kernel lives, and these are
// set up while their input may still be written.)
template <typename T, bool kVec>
__global__ void __launch_bounds__(kThreads) block8_quantize_kernel(const T *x, uint32_t *lanes, uint8_t *exps,
                                                                   const Block8Args a) {
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();
  __shared__ float stage[kVec ? 1 : kThreads / 32][kVec ? 1 : kStageWords];
  const int lane = threadIdx.x & 31;
  const int64_t nwarps = static_cast<int64_t>(gridDim.x) * (kThreads / 32);
  const int64_t first = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
  for (int64_t step = first; step < a.rows * a.segs; step += nwarps) {
    const int64_t row = idiv(step, a.by_segs);
    const int64_t col = (step - row * a.segs) * kRowStep + lane * kPer;
    const int64_t left = a.inner - col;
    const int n = left < 0 ? 0 : left < kPer ? static_cast<int>(left) : kPer;
    float v[kPer];
    if constexpr (kVec)
      load16<T>(x + row * a.ld + (n ? col : 0), n, v);
    else
      load_staged<T>(x + row * a.ld + col - lane * kPer, left + lane * kPer, stage[threadIdx.x >> 5], lane, v);
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) top = max_abs(top, v[i]);
    top = max_abs(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const uint32_t e = block8_exp(top);
    if (n) {
      uint32_t w[4];
      block8_words_of<false, kPer>(v, top, e, block8_inv(e), w);
      uint32_t *const out = lanes + row * a.wpr + col / 4;
      if (a.l_vec && n > 12) {
        __stcs(reinterpret_cast<uint4 *>(out), make_uint4(w[0], w[1], w[2], w[3]));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (4 * i < n) out[i] = w[i];
      }
      if ((lane & 1) == 0) exps[row * a.bpr + col / kBlock8] = static_cast<uint8_t>(e);
    }
  }
}

template <typename T, bool kVec>
__global__ void __launch_bounds__(kThreads)
    block8_dequantize_kernel(const uint32_t *lanes, const uint8_t *exps, T *y, const Block8Args a) {
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();
  __shared__ float stage[kVec ? 1 : kThreads / 32][kVec ? 1 : kStageWords];
  const int lane = threadIdx.x & 31;
  const int64_t nwarps = static_cast<int64_t>(gridDim.x) * (kThreads / 32);
  const int64_t first = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
  for (int64_t step = first; step < a.rows * a.segs; step += nwarps) {
    const int64_t row = idiv(step, a.by_segs);
    const int64_t col = (step - row * a.segs) * kRowStep + lane * kPer;
    const int64_t left = a.inner - col;
    const int n = left < 0 ? 0 : left < kPer ? static_cast<int>(left) : kPer;
    float v[kPer];
    if (n) {
      const uint32_t *const in = lanes + row * a.wpr + col / 4;
      uint32_t w[4];
      if (a.l_vec && n > 12) {
        const uint4 q = __ldcs(reinterpret_cast<const uint4 *>(in));
        w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = 4 * i < n ? in[i] : 0u;
      }
      const float scale = block8_scale(exps[row * a.bpr + col / kBlock8]);
#pragma unroll
      for (int i = 0; i < 4; ++i) block8_values(w[i], scale, v + 4 * i);
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) v[i] = 0.0f;
    }
    if constexpr (kVec) {
      if (n) store16<T>(y + row * a.ld + col, n, v);
    } else {
      store_staged<T>(y + row * a.ld + col - lane * kPer, left + lane * kPer, stage[threadIdx.x >> 5], lane, v);
    }
  }
}

Block8Args make_args(size_t esize, const void *x, int64_t ld, int64_t rows, int64_t inner, const samd_block8 &b) {
  Block8Args a;
  a.rows = rows;
  a.inner = inner;
  a.ld = ld;
  a.segs = (inner + kRowStep - 1) / kRowStep;
  a.by_segs = make_index_div(rows * a.segs, a.segs);
  a.wpr = block8_words(inner);
  a.bpr = block8_blocks(inner);
  a.x_vec = aligned16(x) && (rows == 1 || ld * static_cast<int64_t>(esize) % 16 == 0);
  a.l_vec = aligned16(b.lanes) && (rows == 1 || a.wpr % 4 == 0);
  return a;
}

template <typename T, bool kVec>
cudaError_t quantize_as(const Block8Args &a, const void *x, samd_block8 out, cudaStream_t s) {
  constexpr auto kern = block8_quantize_kernel<T, kVec>;
  return launch_dependent(kern, dim3(resident_grid<kern>(a.rows * a.segs * 32, kThreads)), kThreads, 0, s, 1,
                          static_cast<const T *>(x), static_cast<uint32_t *>(out.lanes), out.exps, a);
}
template <typename T>
cudaError_t quantize(const void *x, int64_t ldx, int64_t rows, int64_t inner, samd_block8 out, cudaStream_t s) {
  const Block8Args a = make_args(sizeof(T), x, ldx, rows, inner, out);
  return a.x_vec ? quantize_as<T, true>(a, x, out, s) : quantize_as<T, false>(a, x, out, s);
}

template <typename T, bool kVec>
cudaError_t dequantize_as(const Block8Args &a, samd_block8 in, void *y, cudaStream_t s) {
  constexpr auto kern = block8_dequantize_kernel<T, kVec>;
  return launch_dependent(kern, dim3(resident_grid<kern>(a.rows * a.segs * 32, kThreads)), kThreads, 0, s, 1,
                          static_cast<const uint32_t *>(in.lanes), in.exps, static_cast<T *>(y), a);
}
template <typename T>
cudaError_t dequantize(samd_block8 in, int64_t rows, int64_t inner, void *y, int64_t ldy, cudaStream_t s) {
  const Block8Args a = make_args(sizeof(T), y, ldy, rows, inner, in);
  return a.x_vec ? dequantize_as<T, true>(a, in, y, s) : dequantize_as<T, false>(a, in, y, s);
}

}  // namespace

cudaError_t launch_block8_quantize(samd_dtype t, const void *x, int64_t ldx, int64_t rows, int64_t inner,
                                   samd_block8 out, cudaStream_t s) {
  if (t == SAMD_F32) return quantize<float>(x, ldx, rows, inner, out, s);
  if (t == SAMD_F16) return quantize<__half>(x, ldx, rows, inner, out, s);
  return quantize<__nv_bfloat16>(x, ldx, rows, inner, out, s);
}

cudaError_t launch_block8_dequantize(samd_dtype t, samd_block8 in, int64_t rows, int64_t inner, void *y, int64_t ldy,
                                     cudaStream_t s) {
  if (t == SAMD_F32) return dequantize<float>(in, rows, inner, y, ldy, s);
  if (t == SAMD_F16) return dequantize<__half>(in, rows, inner, y, ldy, s);
  return dequantize<__nv_bfloat16>(in, rows, inner, y, ldy, s);
}

}  // namespace samd
