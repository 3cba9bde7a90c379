// block8.cu -- activations into their 8-bit form (blocks of 32 with one power
// of two, ffn_internal.cuh) and back.
//
// Both are one pass over HBM: 2 or 4 bytes an element on the wide side and
// 33/32 on the other. Four neighbouring lanes hold a block, eight elements
// each (one 16-byte load of a 16-bit type), and find its largest magnitude
// with two shuffles; magnitudes are compared as bit patterns, which puts
// infinities and NaNs above every number.
#include "ffn_internal.cuh"

namespace samd {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;  // elements a thread handles at a time
constexpr int kRowStep = 32 * kPer;  // elements of a row a warp handles at a time

struct Block8Args {
  int64_t rows, inner, ld, segs;  // segs: warps' steps in a row
  int64_t wpr, bpr;               // words and blocks of a row
  int x_vec, l_vec;               // rows of x are 16-byte, rows of lanes 8-byte aligned
};

template <typename T>
__device__ __forceinline__ void load8(const T *p, int n, bool vec, float *v) {
  if (vec && n == kPer) {
    if constexpr (sizeof(T) == 4) {
      const float4 a = __ldcs(reinterpret_cast<const float4 *>(p)), b = __ldcs(reinterpret_cast<const float4 *>(p) + 1);
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
      const uint4 a = __ldcs(reinterpret_cast<const uint4 *>(p));
      const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2<T>(w[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = i < n ? to_f32<T>(p[i]) : 0.0f;
  }
}

template <typename T>
__device__ __forceinline__ void store8(T *p, int n, bool vec, const float *v) {
  if (vec && n == kPer) {
    if constexpr (sizeof(T) == 4) {
      __stcs(reinterpret_cast<float4 *>(p), make_float4(v[0], v[1], v[2], v[3]));
      __stcs(reinterpret_cast<float4 *>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
    } else {
      __stcs(reinterpret_cast<uint4 *>(p), make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]),
                                                      pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7])));
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (i < n) p[i] = from_f32<T>(v[i]);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) block8_quantize_kernel(const T *__restrict__ x, uint32_t *__restrict__ lanes,
                                                                   uint8_t *__restrict__ exps, const Block8Args a) {
  const int lane = threadIdx.x & 31;
  const int64_t nwarps = static_cast<int64_t>(gridDim.x) * (kThreads / 32);
  const int64_t first = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
  for (int64_t step = first; step < a.rows * a.segs; step += nwarps) {
    const int64_t row = step / a.segs;
    const int64_t col = (step - row * a.segs) * kRowStep + lane * kPer;
    const int64_t left = a.inner - col;
    const int n = left < 0 ? 0 : left < kPer ? static_cast<int>(left) : kPer;
    float v[kPer];
    load8<T>(x + row * a.ld + (n ? col : 0), n, a.x_vec, v);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const uint32_t e = block8_exp(top);
    const float inv = block8_inv(e);
    if (n) {
      const uint32_t lo = block8_word(v[0], v[1], v[2], v[3], inv);
      const uint32_t hi = block8_word(v[4], v[5], v[6], v[7], inv);
      uint32_t *out = lanes + row * a.wpr + col / 4;
      if (a.l_vec && n > 4) {
        __stcs(reinterpret_cast<uint2 *>(out), make_uint2(lo, hi));
      } else {
        out[0] = lo;
        if (n > 4) out[1] = hi;
      }
      if ((lane & 3) == 0) exps[row * a.bpr + col / kBlock8] = static_cast<uint8_t>(e);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
    block8_dequantize_kernel(const uint32_t *__restrict__ lanes, const uint8_t *__restrict__ exps, T *__restrict__ y,
                             const Block8Args a) {
  const int lane = threadIdx.x & 31;
  const int64_t nwarps = static_cast<int64_t>(gridDim.x) * (kThreads / 32);
  const int64_t first = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
  for (int64_t step = first; step < a.rows * a.segs; step += nwarps) {
    const int64_t row = step / a.segs;
    const int64_t col = (step - row * a.segs) * kRowStep + lane * kPer;
    const int64_t left = a.inner - col;
    const int n = left < 0 ? 0 : left < kPer ? static_cast<int>(left) : kPer;
    if (n) {
      const uint32_t *in = lanes + row * a.wpr + col / 4;
      uint2 w;
      if (a.l_vec && n > 4)
        w = __ldcs(reinterpret_cast<const uint2 *>(in));
      else
        w = make_uint2(in[0], n > 4 ? in[1] : 0u);
      const float scale = block8_scale(exps[row * a.bpr + col / kBlock8]);
      float v[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) v[i] = block8_value(i < 4 ? w.x : w.y, i & 3, scale);
      store8<T>(y + row * a.ld + col, n, a.x_vec, v);
    }
  }
}

Block8Args make_args(size_t esize, const void *x, int64_t ld, int64_t rows, int64_t inner, const samd_block8 &b) {
  Block8Args a;
  a.rows = rows;
  a.inner = inner;
  a.ld = ld;
  a.segs = (inner + kRowStep - 1) / kRowStep;
  a.wpr = block8_words(inner);
  a.bpr = block8_blocks(inner);
  a.x_vec = aligned16(x) && (rows == 1 || ld * static_cast<int64_t>(esize) % 16 == 0);
  a.l_vec = aligned16(b.lanes) && (rows == 1 || a.wpr % 2 == 0);
  return a;
}

template <typename T>
cudaError_t quantize(const void *x, int64_t ldx, int64_t rows, int64_t inner, samd_block8 out, cudaStream_t s) {
  const Block8Args a = make_args(sizeof(T), x, ldx, rows, inner, out);
  const int grid = resident_grid<block8_quantize_kernel<T>>(a.rows * a.segs * 32, kThreads);
  block8_quantize_kernel<T><<<grid, kThreads, 0, s>>>(static_cast<const T *>(x), static_cast<uint32_t *>(out.lanes),
                                                      out.exps, a);
  return cudaGetLastError();
}

template <typename T>
cudaError_t dequantize(samd_block8 in, int64_t rows, int64_t inner, void *y, int64_t ldy, cudaStream_t s) {
  const Block8Args a = make_args(sizeof(T), y, ldy, rows, inner, in);
  const int grid = resident_grid<block8_dequantize_kernel<T>>(a.rows * a.segs * 32, kThreads);
  block8_dequantize_kernel<T><<<grid, kThreads, 0, s>>>(static_cast<const uint32_t *>(in.lanes), in.exps,
                                                        static_cast<T *>(y), a);
  return cudaGetLastError();
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
