// ffn_internal.cuh -- what the translation units of the gated feed-forward
// block share: element types, activations, 8-bit blocks, launchers.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "samd_internal.cuh"

namespace samd {

// ---- element types -----------------------------------------------------------

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) {
  return v;
}
template <>
__device__ __forceinline__ float to_f32<__half>(__half v) {
  return __half2float(v);
}
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) {
  return __bfloat162float(v);
}

template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) {
  return v;
}
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) {
  return __float2half_rn(v);
}
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) {
  return __float2bfloat16_rn(v);
}

// Two values of a 16-bit type in one word, the first in the low half.
template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const T a = from_f32<T>(lo), b = from_f32<T>(hi);
  return static_cast<uint32_t>(reinterpret_cast<const uint16_t &>(a)) |
         static_cast<uint32_t>(reinterpret_cast<const uint16_t &>(b)) << 16;
}
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  return reinterpret_cast<const uint32_t &>(p);
}
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
  const __half2 p = __floats2half2_rn(lo, hi);
  return reinterpret_cast<const uint32_t &>(p);
}
template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t w);
template <>
__device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <>
__device__ __forceinline__ float2 unpack2<__half>(uint32_t w) {
  return __half22float2(reinterpret_cast<const __half2 &>(w));
}

// ---- activations ---------------------------------------------------------------

// 1 / (1 + exp(-v)); exp overflows to infinity below -88, which gives 0.
__device__ __forceinline__ float sigmoid(float v) { return __fdividef(1.0f, 1.0f + __expf(-v)); }

// Phi(g) by the complementary error function, which keeps its relative
// precision in the lower tail, where 1 + erf cancels.
__device__ __forceinline__ float normal_cdf(float g) { return 0.5f * erfcf(-0.70710678118654752f * g); }

// act(g) and, for the backward pass, its derivative.
template <int ACT>
__device__ __forceinline__ float act_value(float g) {
  if constexpr (ACT == SAMD_SILU) return g * sigmoid(g);
  if constexpr (ACT == SAMD_GELU) return g * normal_cdf(g);
  // (1 + tanh(a)) / 2 = sigmoid(2 a)
  if constexpr (ACT == SAMD_GELU_TANH)
    return g * sigmoid(1.5957691216057308f * (g + 0.044715f * g * g * g));
  return g <= 0.0f ? 0.0f : g;  // a NaN stays one
}

// The same for an activation known at run time.
__device__ __forceinline__ float act_of(int act, float g) {
  return act == SAMD_SILU        ? act_value<SAMD_SILU>(g)
         : act == SAMD_GELU      ? act_value<SAMD_GELU>(g)
         : act == SAMD_GELU_TANH ? act_value<SAMD_GELU_TANH>(g)
                                 : act_value<SAMD_RELU_ACT>(g);
}

template <int ACT>
__device__ __forceinline__ float act_value_grad(float g, float &grad) {
  if constexpr (ACT == SAMD_SILU) {
    const float s = sigmoid(g);
    grad = s * (1.0f + g * (1.0f - s));
    return g * s;
  }
  if constexpr (ACT == SAMD_GELU) {
    const float p = normal_cdf(g);
    grad = p + g * 0.39894228040143268f * __expf(-0.5f * g * g);
    return g * p;
  }
  if constexpr (ACT == SAMD_GELU_TANH) {
    const float s = sigmoid(1.5957691216057308f * (g + 0.044715f * g * g * g));
    const float b = s * (1.0f - s);  // zero far out, where g * g may be infinite
    grad = b == 0.0f ? s : s + g * b * 1.5957691216057308f * (1.0f + 0.134145f * g * g);
    return g * s;
  }
  grad = g > 0.0f ? 1.0f : g <= 0.0f ? 0.0f : g;
  return g <= 0.0f ? 0.0f : g;
}

// ---- 8-bit blocks ----------------------------------------------------------------
//
// A block of 32 elements shares a power of two: e = max(E - 6, 0) with E the
// biased exponent of the largest magnitude, so a code v * 2^(127 - e) lies in
// (-128, 128) and is clamped to -127 .. 127 (only magnitudes over 127.5 / 128
// of the next power of two are). A power of two costs up to one of the eight
// bits against amax / 127, and buys codes that 16-bit types and the tensor
// cores take without another rounding.
constexpr int kBlock8 = 32;

// Exponent byte of a block from the bits of its largest magnitude.
__device__ __forceinline__ uint32_t block8_exp(uint32_t amax_bits) {
  const int E = static_cast<int>(amax_bits >> 23);
  return E == 255 ? 255u : static_cast<uint32_t>(E > 6 ? E - 6 : 0);
}
// 2^(127 - e) for e <= 248 (a finite block has no larger one); a block of NaNs
// gets the factor zero, and its codes are masked.
__device__ __forceinline__ float block8_inv(uint32_t e) { return e == 255u ? 0.0f : __uint_as_float((254u - e) << 23); }
// 2^(e - 127), or a NaN; e = 0 is a subnormal.
__device__ __forceinline__ float block8_scale(uint32_t e) {
  return e == 255u ? __uint_as_float(0x7FC00000u) : e == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(e << 23);
}
__device__ __forceinline__ uint32_t block8_code(float v, float inv) {
  const int c = __float2int_rn(v * inv);
  return static_cast<uint32_t>(c > 127 ? 127 : c < -127 ? -127 : c) & 255u;
}
// Four codes as a word of lanes (in a block of NaNs inf * 0 converts to 0).
__device__ __forceinline__ uint32_t block8_word(float a, float b, float c, float d, float inv) {
  return block8_code(a, inv) | block8_code(b, inv) << 8 | block8_code(c, inv) << 16 | block8_code(d, inv) << 24;
}
__device__ __forceinline__ float block8_value(uint32_t word, int lane, float scale) {
  return static_cast<float>(static_cast<int>(word << (24 - 8 * lane)) >> 24) * scale;
}

inline int64_t block8_words(int64_t inner) { return (inner + 3) / 4; }
inline int64_t block8_blocks(int64_t inner) { return (inner + kBlock8 - 1) / kBlock8; }

// ---- launchers -------------------------------------------------------------------

cudaError_t launch_matvec4(const samd_matvec_desc &d, int act, samd_fmt fw, const void *x, const samd_weights4 &wg,
                           const samd_weights4 *wu, void *y, cudaStream_t s);
cudaError_t launch_block8_quantize(samd_dtype t, const void *x, int64_t ldx, int64_t rows, int64_t inner,
                                   samd_block8 out, cudaStream_t s);
cudaError_t launch_block8_dequantize(samd_dtype t, samd_block8 in, int64_t rows, int64_t inner, void *y, int64_t ldy,
                                     cudaStream_t s);
size_t ffn_backward_workspace(const samd_ffn_desc &d);
cudaError_t launch_ffn_forward(const samd_ffn_desc &d, const void *x, const void *wg, const void *wu, void *h,
                               samd_block8 cg, samd_block8 cu, cudaStream_t s);
cudaError_t launch_ffn_backward(const samd_ffn_desc &d, const void *dh, samd_block8 cx, samd_block8 cg, samd_block8 cu,
                                const void *wg, const void *wu, void *dx, void *dwg, void *dwu, void *h,
                                void *workspace, cudaStream_t s);

// ---- from conv2d.cu ----------------------------------------------------------------

// Device address of the sticky status word that bounded waits record into.
cudaError_t device_status_ptr(int **out);
// cuTensorMapEncodeTiled, or null.
using EncodeTiledFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                   const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                   CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn tensor_map_encoder();
namespace conv {
cudaError_t ensure_smem_attr(const void *kern, size_t smem);
}

}  // namespace samd
