// kv_cache.cu -- rows of keys and values into the packed cache, and back.
//
//   scale = round16(max |v| / L), lane = round(v / scale) clamped to -L .. L,
//   L = 2^(bits - 1) - 1, for every 32 neighbouring elements of a row.
//
// Both are one pass: 2 bytes an element on the wide side, bits / 8 + 1/16 in
// the cache. Two neighbouring lanes hold a block, sixteen elements of a key and
// of a value each, and find its largest magnitude with a shuffle.
//
// The lane is the rounded quotient, without a division: v and the scale have
// at most 11 significant bits each, so a quotient that is not half way between
// two integers is at least 2^-12 away from there, and v * (1 / scale), whose
// error is below 2^-15, rounds to the same integer. A quotient that is half way
// leaves a remainder v - lane * scale (exact) of half a scale: then, and where a
// block has something to clamp, sixteen elements are divided after all. 7040 tokens
// of 8 heads of 128 elements in fp16 into 4 bits take 17 us and back 15 (28 together
// in a graph; their bytes 11): instructions, about 20 an element in and 13 out. With
// a key or a value a thread, a division's steps for every element and converted
// lanes it was 23 and 14.5.
#include "cache_internal.cuh"
#include "tc_ptx.cuh"

namespace samd {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 16;  // elements a thread handles

struct RowArgs {
  kv::Seqs s;
  const int32_t *starts;
  uint8_t *lanes[2], *scales[2];  // of keys and of values
  uint8_t *x[2];
  int64_t ld[2];                  // of x, in bytes
  int64_t items;                  // tokens x heads x dim / kPer
  IndexDiv by_token, by_head;
  int heads, dim;
};

// A thread's sixteen elements of a key and of the same of a value.
struct Item {
  int64_t at[2], row;  // bytes from x; row of the cache, or below 0
  int e;               // first element
};

__device__ __forceinline__ Item item_of(const RowArgs &a, int64_t n) {
  Item it;
  const int64_t token = idiv(n, a.by_token), left = n - token * a.by_token.d;
  const int h = static_cast<int>(idiv(left, a.by_head));
  it.e = static_cast<int>(left - h * a.by_head.d) * kPer;
#pragma unroll
  for (int m = 0; m < 2; ++m) it.at[m] = token * a.ld[m] + (static_cast<int64_t>(h) * a.dim + it.e) * 2;
  const int64_t p = kv::place_of(a.s, a.starts, static_cast<int>(token));
  it.row = p < 0 ? p : kv::row_of(a.s, p, a.heads, h);
  return it;
}

template <typename T>
__device__ __forceinline__ uint16_t bits_of(float v) {
  const T t = from_f32<T>(v);
  return reinterpret_cast<const uint16_t &>(t);
}

constexpr float kMagic = 12582912.0f;  // 1.5 * 2^23: adding it rounds to an integer, which its low bits then hold

// Sixteen elements as words of lanes, for a scale s > 0; top: the largest magnitude of the block.
template <int BITS>
__device__ __forceinline__ void lanes_of(const float (&v)[kPer], float top, float s, uint32_t (&w)[BITS / 2]) {
  constexpr float kMost = BITS == 8 ? 127.0f : 7.0f;
  const float inv = __fdiv_rn(1.0f, s);
  uint32_t q[kPer];
  float far = 0.0f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const float k = fmaf(v[i], inv, kMagic);
    q[i] = __float_as_uint(k);
    far = fmaxf(far, fabsf(fmaf(kMagic - k, s, v[i])));
  }
  // a tie, something to clamp, or a reciprocal past fp32's range (a scale of bfloat16 below 2^-127): the long way
  if (!(far + far < s) || !(top * inv < kMost + 0.49f) || !(inv <= 3.402823466e38f)) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const float k = fminf(fmaxf(rintf(__fdiv_rn(v[i], s)), -kMost), kMost);
      q[i] = __float_as_uint(k + kMagic);
    }
  }
#pragma unroll
  for (int i = 0; i < BITS / 2; ++i) {
    if constexpr (BITS == 8) {
      w[i] = __byte_perm(__byte_perm(q[4 * i], q[4 * i + 1], 0x0040), __byte_perm(q[4 * i + 2], q[4 * i + 3], 0x0040), 0x5410);
    } else {
      w[i] = 0;
#pragma unroll
      for (int j = 7; j >= 0; --j) w[i] = w[i] << 4 | (q[8 * i + j] & 15u);
    }
  }
}

template <typename T, int BITS>
__global__ void __launch_bounds__(kThreads) cache_append_kernel(const RowArgs a) {
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();
  constexpr float kMost = BITS == 8 ? 127.0f : 7.0f;
  for (int64_t n = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;; n += static_cast<int64_t>(gridDim.x) * kThreads) {
    // (a block's two threads, an even lane and the next, are both in or both out)
    const bool on = n < a.items;
    if (!__any_sync(0xffffffffu, on)) break;
    Item it = {};
    it.row = -1;
    uint4 x[2][2] = {};
    if (on) {
      it = item_of(a, n);
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const uint4 *const p = reinterpret_cast<const uint4 *>(a.x[m] + it.at[m]);
        x[m][0] = p[0], x[m][1] = p[1];
      }
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      float v[kPer], top = 0.0f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t w[4] = {x[m][i].x, x[m][i].y, x[m][i].z, x[m][i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 f = unpack2<T>(w[k]);
          v[8 * i + 2 * k] = f.x, v[8 * i + 2 * k + 1] = f.y;
        }
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) top = max_abs(top, v[i]);
      top = max_abs(top, __shfl_xor_sync(0xffffffffu, top, 1));
      if (it.row < 0) continue;
      const bool fine = top <= 3.402823466e38f;  // no infinity, no NaN
      const uint16_t raw = fine ? bits_of<T>(__fdiv_rn(top, kMost)) : static_cast<uint16_t>(0x7FFF);
      const float s = fine ? to_f32<T>(reinterpret_cast<const T &>(raw)) : 0.0f;
      uint32_t w[BITS / 2] = {};
      if (s > 0.0f) lanes_of<BITS>(v, top, s, w);
      uint8_t *const to = a.lanes[m] + (it.row * a.dim + it.e) / 8 * BITS;
      if constexpr (BITS == 8)
        *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
      else
        *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
      if ((it.e & 16) == 0) *reinterpret_cast<uint16_t *>(a.scales[m] + (it.row * a.dim + it.e) / 16) = raw;
    }
  }
}

template <typename T, int BITS>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const RowArgs a) {
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();
  for (int64_t n = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; n < a.items;
       n += static_cast<int64_t>(gridDim.x) * kThreads) {
    const Item it = item_of(a, n);
    if (it.row == -2) continue;
    uint32_t w[2][BITS / 2] = {};
    float s[2] = {0.0f, 0.0f};
    if (it.row >= 0) {
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const uint8_t *const from = a.lanes[m] + (it.row * a.dim + it.e) / 8 * BITS;
        if constexpr (BITS == 8) {
          const uint4 q = *reinterpret_cast<const uint4 *>(from);
          w[m][0] = q.x, w[m][1] = q.y, w[m][2] = q.z, w[m][3] = q.w;
        } else {
          const uint2 q = *reinterpret_cast<const uint2 *>(from);
          w[m][0] = q.x, w[m][1] = q.y;
        }
        s[m] = to_f32<T>(*reinterpret_cast<const T *>(a.scales[m] + (it.row * a.dim + it.e) / 32 * 2));
      }
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      uint32_t out[kPer / 2];
      constexpr uint32_t kFlip = BITS == 8 ? 0x80808080u : 0x88888888u;
      constexpr float kLess = 8388608.0f + (1 << (BITS - 1));  // a lane plus 2^(bits - 1) under the exponent of 2^23
#pragma unroll
      for (int i = 0; i < kPer / 2; ++i) {
        float f[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int at = (2 * i + j) * BITS;
          const uint32_t u = (w[m][at / 32] ^ kFlip) >> (at % 32) & ((1u << BITS) - 1);
          f[j] = (__uint_as_float(u | 0x4B000000u) - kLess) * s[m];
        }
        out[i] = pack2<T>(f[0], f[1]);
      }
      uint4 *const p = reinterpret_cast<uint4 *>(a.x[m] + it.at[m]);
      p[0] = make_uint4(out[0], out[1], out[2], out[3]);
      p[1] = make_uint4(out[4], out[5], out[6], out[7]);
    }
  }
}

RowArgs make_args(const samd_cache &c, const samd_cache_seqs &s, const int32_t *starts, int tokens, const void *k,
                  int64_t ldk, const void *v, int64_t ldv) {
  RowArgs a = {};
  a.s = kv::make_seqs(c, s);
  a.starts = starts;
  a.lanes[0] = static_cast<uint8_t *>(c.k_lanes), a.lanes[1] = static_cast<uint8_t *>(c.v_lanes);
  a.scales[0] = static_cast<uint8_t *>(c.k_scales), a.scales[1] = static_cast<uint8_t *>(c.v_scales);
  a.x[0] = static_cast<uint8_t *>(const_cast<void *>(k)), a.x[1] = static_cast<uint8_t *>(const_cast<void *>(v));
  a.ld[0] = ldk * 2, a.ld[1] = ldv * 2;
  a.heads = c.heads, a.dim = c.dim;
  const int64_t head = c.dim / kPer, token = head * c.heads;
  a.items = token * tokens;
  a.by_token = make_index_div(a.items, token);
  a.by_head = make_index_div(token, head);
  return a;
}

template <typename T, int BITS, bool kAppend>
cudaError_t launch_as(const RowArgs &a, cudaStream_t s) {
  constexpr auto kern = kAppend ? cache_append_kernel<T, BITS> : cache_read_kernel<T, BITS>;
  return launch_dependent(kern, dim3(resident_grid<kern>(a.items, kThreads)), kThreads, 0, s, 1, a);
}
template <bool kAppend>
cudaError_t launch(const samd_cache &c, const RowArgs &a, cudaStream_t s) {
  if (c.type == SAMD_BF16)
    return c.fmt.bits == 8 ? launch_as<__nv_bfloat16, 8, kAppend>(a, s) : launch_as<__nv_bfloat16, 4, kAppend>(a, s);
  return c.fmt.bits == 8 ? launch_as<__half, 8, kAppend>(a, s) : launch_as<__half, 4, kAppend>(a, s);
}

}  // namespace

cudaError_t launch_cache_append(const samd_cache &c, const samd_cache_seqs &s, const int32_t *starts, int tokens,
                                const void *k, int64_t ldk, const void *v, int64_t ldv, cudaStream_t stream) {
  return launch<true>(c, make_args(c, s, starts, tokens, k, ldk, v, ldv), stream);
}

cudaError_t launch_cache_read(const samd_cache &c, const samd_cache_seqs &s, const int32_t *starts, int tokens, void *k,
                              int64_t ldk, void *v, int64_t ldv, cudaStream_t stream) {
  return launch<false>(c, make_args(c, s, starts, tokens, k, ldk, v, ldv), stream);
}

}  // namespace samd
