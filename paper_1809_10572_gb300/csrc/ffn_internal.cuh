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

// Exponent byte of a block from its largest magnitude.
__device__ __forceinline__ uint32_t block8_exp(float top) {
  const int E = static_cast<int>(__float_as_uint(top) >> 23);
  return E == 255 ? 255u : static_cast<uint32_t>(E > 6 ? E - 6 : 0);
}
// 2^(127 - e) for e <= 248 (a finite block has no larger one); a block of NaNs
// gets the factor zero, and its codes are masked.
__device__ __forceinline__ float block8_inv(uint32_t e) { return e == 255u ? 0.0f : __uint_as_float((254u - e) << 23); }
// 2^(e - 127), or a NaN; e = 0 is a subnormal.
__device__ __forceinline__ float block8_scale(uint32_t e) {
  return e == 255u ? __uint_as_float(0x7FC00000u) : e == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(e << 23);
}

// The larger magnitude; a NaN is larger than everything.
__device__ __forceinline__ float max_abs(float top, float v) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(top), "f"(fabsf(v)));
  return r;
}

// N values of a block (N a multiple of 4), whose largest magnitude is `top`,
// as words of four lanes, with the block's exponent e and factor inv. Adding
// 1.5 * 2^23 rounds v * inv to an integer (the product is exact, so this is
// its one rounding) and leaves the code in the sum's low byte; a conversion
// would take the quarter-rate pipe. Blocks with something to clamp (one in a
// hundred or so) and blocks of NaNs go the long way round.
// kKeep: the code of a positive value is at least 1.
template <bool kKeep, int N>
__device__ __forceinline__ void block8_words_of(const float *v, float top, uint32_t e, float inv, uint32_t *w) {
  if (top * inv < 127.5f) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      uint32_t c[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        c[j] = __float_as_uint(fmaf(v[4 * i + j], inv, 12582912.0f));
        if constexpr (kKeep)
          if (v[4 * i + j] > 0.0f) c[j] = max(c[j], 0x4B400001u);
      }
      w[i] = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      w[i] = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float f = fminf(fmaxf(v[4 * i + j] * inv, -127.0f), 127.0f);
        if constexpr (kKeep)
          if (v[4 * i + j] > 0.0f) f = fmaxf(f, 1.0f);
        if (e != 255u) w[i] |= (__float_as_uint(f + 12582912.0f) & 255u) << 8 * j;
      }
    }
  }
}

// The four values of a word: lane + 128 under the exponent of 2^23, less
// 2^23 + 128 (exact, and not on the conversions' pipe).
__device__ __forceinline__ void block8_values(uint32_t word, float scale, float *v) {
  const uint32_t u = word ^ 0x80808080u;
  v[0] = (__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7440)) - 8388736.0f) * scale;
  v[1] = (__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7441)) - 8388736.0f) * scale;
  v[2] = (__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7442)) - 8388736.0f) * scale;
  v[3] = (__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7443)) - 8388736.0f) * scale;
}

inline int64_t block8_words(int64_t inner) { return (inner + 3) / 4; }
inline int64_t block8_blocks(int64_t inner) { return (inner + kBlock8 - 1) / kBlock8; }

// Division of an index below `count` by d: in 32 bits where they suffice.
struct IndexDiv {
  FastDiv f;
  int64_t d;
  bool small;
};
inline IndexDiv make_index_div(int64_t count, int64_t d) {
  const bool small = count < (int64_t(1) << 31) && d < (int64_t(1) << 31);
  return IndexDiv{make_fastdiv(small ? static_cast<uint32_t>(d) : 1u), d, small};
}
__device__ __forceinline__ int64_t idiv(int64_t n, const IndexDiv &v) {
  return v.small ? static_cast<int64_t>(fdiv(static_cast<uint32_t>(n), v.f)) : n / v.d;
}

// A launch that may be set up while the kernel before it in the stream drains
// (the kernel calls grid_dependency_wait before it touches global memory), in
// clusters of `cluster` neighbouring CTAs.
template <typename... P, typename... A>
cudaError_t launch_dependent(void (*kern)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, int cluster,
                             A... args) {
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...);
  return e != cudaSuccess ? e : cudaGetLastError();
}

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
