// matvec4_kernel.cuh -- products of a few tokens with 4-bit weights, and the gated
// pair of them with the activation and the product.
//
//   y[m][n] = sum_G s[n][G] * sum_{k in G} (q[n][k] - z[n][G]) * x[m][k]
//
// Bound by its reads: the weights, half a byte each, come once; a token adds one
// multiply-add to each. At the copy bandwidth an SM receives about 46 weights
// a clock, which is more than its CUDA cores can widen, scale and multiply
// one by one, so the products go through mma.sync (m16n8k16, weights as the
// 16-row operand, tokens as the 8 columns): the tensor memory and the shared
// operands of tcgen05 would cost a pass through shared memory as 16-bit values,
// four times the bytes that come from HBM.
//
// Widening: a nibble over the mantissa of a power of two is that power plus
// the nibble (fp16: 1024 + q, or 64 + q four bits up; bf16: 128 + q), and
// subtracting the power plus the zero point is exact, so the products are
// those of the integers q - z (also with infinities in x). Signed lanes are
// flipped to offset binary by the same logic operation. The group's sum stays
// in the fp32 accumulators of its MMAs and is scaled in fp32.
//
// Layout: a word holds lanes 8w .. 8w + 7, and one mask takes lanes i and i + 4
// out together, so the reduction index runs in the order (0,4), (1,5), (2,6),
// (3,7) of every word; x is put in the same order by byte permutes. A chunk of
// 32 inputs is four words of a row, which ldmatrix deals out as the MMA wants
// them: word t of row r to lane 4 r + t.
//
// Split: the grid is at most one wave of resident CTAs, each taking tiles of
// 16 * RT rows (of both matrices of the pair) in turn. Its eight warps share a
// tile's blocks of KB inputs, each through its own ring of stages (weights by
// one TMA tile, scales and zero points by cp.async) that runs on into the next
// tile; their sums are joined in a fixed order behind the tile's one barrier.
// Tokens come through L1, which holds a CTA's x from tile to tile.
//
// Measured (one GB300, weights not in L2): one bf16 token by 65536 x 4096 with
// scales for 64 inputs 34.5 us, 4.1 TB/s, 0.62 of the copy bandwidth (fp16 0.69,
// scales for 32 inputs 0.64, zero points 0.57). About 42 instructions for 512
// weights, half of them on the 64-lane integer pipe. No unit is full: issue
// slots are 58% busy, that pipe 55%. Sixteen warps an SM do not hide what an
// instruction waits for: of the 6.3 clocks from one of a warp's to its next, 1.1
// go to others' turns, 1.1 to the pipe, 1.0 to fixed latencies, 0.7 to tokens. A
// CTA for each tile took 65 us (rings that start and drain for every tile);
// shifts on the multiplier instead 40; tokens permuted once into shared memory
// 36. From nine tokens on x's way from L2 (every tile reads all of it) and its
// latency bound it: 16 tokens by 8192 x 8192 18 us, 32 tokens 34 (four row tiles
// a CTA: 24 and 32).
#pragma once

#include "ffn_internal.cuh"
#include "tc_ptx.cuh"

#include <type_traits>

namespace samd {
namespace mv {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr uint64_t kWaitLimitNs = 1000000000ull;  // 1 s

struct MvArgs {
  const uint8_t *lanes[2];
  const uint8_t *scales[2];
  const uint8_t *zeros[2];
  const void *x;
  void *y;
  int64_t ldx, ldy;
  int64_t row_bytes;  // of a row of lanes
  int64_t groups;     // scales of a row
  int64_t n_scales;   // of a matrix
  int M, N, K;
  int group_shift;    // log2(group)
  int nblk;           // blocks of KB inputs
  int tiles;          // of 16 * RT rows
  int tma, x_vec;     // rows of lanes are whole 16-byte units; rows of x are 16-byte aligned
  int *status;        // of the device, for waits that give up
  int s_vec;          // a row's scales of a block lie on a multiple of their size
  int is_signed;
  int act;            // of the gated pair; -1: one matrix
};

__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}

// d = a b, or d += a b.
template <typename T, bool kAdd>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  const float c0 = kAdd ? d[0] : 0.0f, c1 = kAdd ? d[1] : 0.0f, c2 = kAdd ? d[2] : 0.0f, c3 = kAdd ? d[3] : 0.0f;
  if constexpr (std::is_same<T, __half>::value)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%10, %11, %12, %13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%10, %11, %12, %13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}

// What is subtracted from the widened lanes of a group with zero point z.
template <typename T>
struct Offset;
template <>
struct Offset<__nv_bfloat16> {
  uint32_t a;
  __device__ __forceinline__ void set(uint32_t zz) { a = 0x43004300u | zz; }  // z in both halves
};
template <>
struct Offset<__half> {
  uint32_t a, b;
  __device__ __forceinline__ void set(uint32_t zz) {
    a = 0x64006400u | zz;
    b = 0x54005400u | zz << 4;
  }
};

template <typename V>
__device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b) {
  const V d = __hsub2(reinterpret_cast<const V &>(a), reinterpret_cast<const V &>(b));
  return reinterpret_cast<const uint32_t &>(d);
}

// The eight lanes of a word as four pairs (i, i + 4); flip is 8 for signed
// lanes (in both halves), else 0.
__device__ __forceinline__ void widen(uint32_t w, uint32_t flip, const Offset<__nv_bfloat16> &o, uint32_t (&p)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    p[i] = sub2<__nv_bfloat162>(((w >> 4 * i) & 0x000F000Fu) ^ (0x43004300u | flip), o.a);
}
__device__ __forceinline__ void widen(uint32_t w, uint32_t flip, const Offset<__half> &o, uint32_t (&p)[4]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t v = w >> 8 * i;
    p[2 * i] = sub2<__half2>((v & 0x000F000Fu) ^ (0x64006400u | flip), o.a);
    p[2 * i + 1] = sub2<__half2>((v & 0x00F000F0u) ^ (0x54005400u | flip << 4), o.b);
  }
}

template <typename T>
__device__ __forceinline__ float f32_of_bits(uint16_t v) {
  return to_f32<T>(reinterpret_cast<const T &>(v));
}

// The lane's eight inputs k .. k + 7 of a token; those past K are zero and not read. Rows that are not 16-byte
// aligned (kXVec false) are read by the 4-byte words that hold the inputs, shifted by half a word where those begin
// in a word's middle (then with a ninth input of the row). Plain loads: the read-only path is for data that nothing
// writes while a kernel lives, and this one is set up while x may still be written.
template <typename T, bool kXVec>
__device__ __forceinline__ uint4 load_x8(const T *row, int64_t k, int K) {
  const int64_t left = K - k;
  if constexpr (kXVec) {
    if (left >= 8) return *reinterpret_cast<const uint4 *>(row + k);
  } else {
    if (left > 8) {
      const uintptr_t at = reinterpret_cast<uintptr_t>(row + k);
      const uint32_t *const p = reinterpret_cast<const uint32_t *>(at & ~uintptr_t(3));
      const bool half = (at & 2) != 0;
      uint32_t v[5];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = p[i];
      v[4] = half ? p[4] : 0u;
      if (half) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __funnelshift_r(v[i], v[i + 1], 16);
      }
      return make_uint4(v[0], v[1], v[2], v[3]);
    }
  }
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < left) w[i / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t *>(row)[k + i]) << 16 * (i & 1);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// CH: chunks of 32 inputs in a block; CPG: chunks of a block that share a scale.
template <typename T, bool kGated, bool kZeros, int RT, int NT, int CH, int CPG>
struct Mv {
  static constexpr int kMats = kGated ? 2 : 1;
  static constexpr int kTiles = RT * kMats;  // 16-row tiles of a CTA's tile: the first matrix's, then the second's
  static constexpr int kRows = 16 * kTiles;
  static constexpr int KB = 32 * CH;
  static constexpr int kPitch = 16 * CH;  // bytes of a row of weights in a stage
  static constexpr int kGroups = CH / CPG;  // scales of a row in a block
  // bytes of a row's scales, and of its zero points, in a stage: the 4-byte
  // words that hold them at any alignment, in a power of two
  static constexpr int kSPitch = kGroups == 1 ? 4 : 4 * kGroups;
  static constexpr int kZPitch = kGroups == 1 ? 4 : kGroups <= 4 ? 8 : 16;
  static constexpr int kWBytes = kRows * kPitch;  // a stage's weights (whole 1024- or 512-byte swizzle patterns)
  static constexpr int kZOff = kRows * kSPitch;
  static constexpr int kSzBytes = kZOff + (kZeros ? kRows * kZPitch : 0);  // its scales and zero points
  // as many stages as leave an SM two CTAs of one token (one by 65536 x 4096 with zero points: 43.3 us with three stages
  // and one CTA). The sums of more tokens are not counted: with scales for 32 inputs 32 tokens leave one CTA an SM, with
  // zero points 24 of them, and 32 with zero points and scales for 64.
  static constexpr int fit(int stages) {
    return kWarps * stages * (kWBytes + kSzBytes + 8) + kWarps * kRows * 4 + 1024 <= 114 * 1024;
  }
  static constexpr int kStages = fit(4) ? 4 : fit(3) ? 3 : 2;
  // shared memory: [warp][stage] weights, [warp][stage] scales and zero points, [warp][stage] barriers, the sums
  static constexpr int kSzAt = kWarps * kStages * kWBytes;
  static constexpr int kBarAt = kSzAt + kWarps * kStages * kSzBytes;
  static constexpr int kRedAt = kBarAt + kWarps * kStages * 8;
  static constexpr int kBufs = NT == 1 && kRows == 16 ? 2 : 1;
  // the warps' sums: rows of an odd number of tokens, so that neighbouring rows lie in other banks
  static __host__ __device__ constexpr int red_pitch(int tokens) { return tokens | 1; }
  static __host__ __device__ constexpr int red_floats(int tokens) { return kWarps * kRows * red_pitch(tokens); }  // of one buffer
  static constexpr size_t smem(int tokens) {
    return static_cast<size_t>(kRedAt) + static_cast<size_t>(kBufs) * red_floats(tokens) * 4;
  }
};

template <typename T, bool kGated, bool kZeros, bool kXVec, int RT, int NT, int CH, int CPG>
__global__ void __launch_bounds__(kThreads, 2) matvec4_kernel(const __grid_constant__ CUtensorMap map0,
                                                                const __grid_constant__ CUtensorMap map1,
                                                                const MvArgs a) {
  using P = Mv<T, kGated, kZeros, RT, NT, CH, CPG>;
  constexpr int kTiles = P::kTiles, kRows = P::kRows, KB = P::KB, kPitch = P::kPitch, kStages = P::kStages;
  constexpr int kSwz = CH >= 8 ? 0 : 1;  // rows that share a 128-byte line: 2^kSwz
  static_assert(CH == 4 || CH == 8, "a row of a stage is 64 or 128 bytes");
  extern __shared__ __align__(1024) uint8_t smem[];
  float *const red = reinterpret_cast<float *>(smem + P::kRedAt);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t bar0 = ptx::smem_addr(smem + P::kBarAt) + warp * kStages * 8;  // this warp's stages' weights
  if (a.tma && lane == 0) {
    for (int i = 0; i < kStages; ++i) ptx::mbar_init(bar0 + 8 * i, 1);
    ptx::fence_barrier_init();
  }
  __syncwarp();

  // weights and tokens may come from the kernel before; the next one may be set up
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();

  const int g = lane >> 2, t = lane & 3;
  const int m0 = blockIdx.y * (8 * NT);
  const int tokens = min(a.M - m0, 8 * NT);
  const uint32_t w_s = ptx::smem_addr(smem) + warp * kStages * P::kWBytes;
  const uint8_t *const sz = smem + P::kSzAt + warp * kStages * P::kSzBytes;
  const uint32_t sz_s = ptx::smem_addr(sz);
  const T *const x = static_cast<const T *>(a.x) + m0 * a.ldx;

  const bool one_scale = P::kGroups > 1 && CPG == 4 && a.group_shift > 7;  // groups that hold whole blocks
  // the scales of a block in row `row` of a tile; past N, row N - 1 again (its sums are not stored)
  auto scale_of = [&](int n0, int row, int blk) -> const uint8_t * {
    const int mat = kGated && row >= 16 * RT;
    const int64_t n = min(n0 + row - mat * 16 * RT, a.N - 1);
    return a.scales[mat] + (n * a.groups + ((static_cast<int64_t>(blk) * KB) >> a.group_shift)) * 2;
  };
  // One block's weights, scales and zero points into a stage: the weights by
  // one TMA tile where rows are whole 16-byte units (rows past N and bytes past
  // a row's end are zero), else by 4-byte copies. Where a row's scales of a
  // block do not lie on their own size (s_vec = 0), the 4-byte words around them
  // are copied, a word past the end of the array is clipped, and the reader
  // finds its place in the first word from the same index. scale: scale_of for
  // the lane's row.
  auto load = [&](int n0, int blk, int stage, const uint8_t *scale) {
    const int last = a.N - 1 - n0;  // of the tile's rows
    const uint32_t sw = w_s + stage * P::kWBytes, ss = sz_s + stage * P::kSzBytes;
    if (a.tma) {
      if (lane == 0) {
        const uint32_t bar = bar0 + 8 * stage;
        ptx::mbar_arrive_expect_tx(bar, P::kWBytes);
        ptx::tma_load_2d(sw, &map0, blk * kPitch, n0, bar);
        if constexpr (kGated) ptx::tma_load_2d(sw + P::kWBytes / 2, &map1, blk * kPitch, n0, bar);
      }
    } else {
      constexpr int kPer = 4 * CH;  // words of a row
      for (int i = 0; i < kRows * kPer / 32; ++i) {
        const int idx = i * 32 + lane, row = idx / kPer, w = idx % kPer, ch = w >> 2;
        const int mat = kGated && row >= 16 * RT;
        const int64_t at = static_cast<int64_t>(blk) * (KB / 2) + w * 4;
        const bool in = at < a.row_bytes;
        ptx::cp_async_4(sw + row * kPitch + ((ch ^ ((row >> kSwz) & (CH - 1))) * 16) + (w & 3) * 4,
                        a.lanes[mat] + (n0 + min(row - mat * 16 * RT, last)) * a.row_bytes + (in ? at : 0),
                        in ? 4u : 0u);
      }
    }
    if (P::kGroups > 1 && a.s_vec) {
      // one copy for a row: lane r brings row r of the tile (and row r + 32)
#pragma unroll
      for (int i = 0; i < (kRows + 31) / 32; ++i)
        if (kRows % 32 == 0 || lane < kRows) {
          const uint32_t dst = ss + (i * 32 + lane) * P::kSPitch;
          const uint8_t *const src = i == 0 ? scale : scale_of(n0, i * 32 + lane, blk);
          if constexpr (P::kGroups == 8) ptx::cp_async_16(dst, src, 16);
          if constexpr (P::kGroups == 4) ptx::cp_async_8(dst, src, 8);
          if constexpr (P::kGroups == 2) ptx::cp_async_4(dst, src, 4);
        }
    } else if (P::kGroups == 1 || one_scale) {
      // the word that holds a row's one scale of the block
#pragma unroll
      for (int i = 0; i < (kRows + 31) / 32; ++i)
        if (kRows % 32 == 0 || lane < kRows) {
          const int row = i * 32 + lane;
          const uint8_t *const base = a.scales[kGated && row >= 16 * RT];
          const int64_t at = (scale_of(n0, row, blk) - base) & ~int64_t(3), left = a.n_scales * 2 - at;
          ptx::cp_async_4(ss + row * P::kSPitch, base + at, left >= 4 ? 4u : static_cast<uint32_t>(left));
        }
    } else {
      const int64_t tile_g = n0 * a.groups + ((static_cast<int64_t>(blk) * KB) >> a.group_shift);
      constexpr int kWords = P::kGroups == 1 ? 1 : P::kGroups / 2 + 1;
#pragma unroll
      for (int i = 0; i < (kRows * kWords + 31) / 32; ++i) {
        const int idx = i * 32 + lane, row = idx / kWords, w = idx % kWords, mat = kGated && row >= 16 * RT;
        if (kRows * kWords % 32 == 0 || row < kRows) {
          const int64_t n = tile_g + min(row - mat * 16 * RT, last) * a.groups;
          const int64_t at = (n * 2 & ~int64_t(3)) + w * 4, left = a.n_scales * 2 - at;
          ptx::cp_async_4(ss + row * P::kSPitch + w * 4, a.scales[mat] + (left > 0 ? at : 0),
                          left >= 4 ? 4u : left > 0 ? static_cast<uint32_t>(left) : 0u);
        }
      }
    }
    if constexpr (kZeros) {
      if (P::kGroups >= 4 && a.s_vec) {
#pragma unroll
        for (int i = 0; i < (kRows + 31) / 32; ++i)
          if (kRows % 32 == 0 || lane < kRows) {
            const int row = i * 32 + lane, mat = kGated && row >= 16 * RT;
            // the zero points' index is the scales'
            const uint8_t *const src =
                a.zeros[mat] + ((i == 0 ? scale : scale_of(n0, row, blk)) - a.scales[mat]) / 2;
            if constexpr (P::kGroups == 8) ptx::cp_async_8(ss + P::kZOff + row * P::kZPitch, src, 8);
            if constexpr (P::kGroups == 4) ptx::cp_async_4(ss + P::kZOff + row * P::kZPitch, src, 4);
          }
      } else {
        const int64_t tile_g = n0 * a.groups + ((static_cast<int64_t>(blk) * KB) >> a.group_shift);
        constexpr int kWords = P::kGroups == 1 ? 1 : P::kGroups <= 4 ? 2 : 3;
#pragma unroll
        for (int i = 0; i < (kRows * kWords + 31) / 32; ++i) {
          const int idx = i * 32 + lane, row = idx / kWords, w = idx % kWords, mat = kGated && row >= 16 * RT;
          if (kRows * kWords % 32 == 0 || row < kRows) {
            const int64_t n = tile_g + min(row - mat * 16 * RT, last) * a.groups;
            const int64_t at = (n & ~int64_t(3)) + w * 4, left = a.n_scales - at;
            ptx::cp_async_4(ss + P::kZOff + row * P::kZPitch + w * 4, a.zeros[mat] + (left > 0 ? at : 0),
                            left >= 4 ? 4u : left > 0 ? static_cast<uint32_t>(left) : 0u);
          }
        }
      }
    }
  };

  // The lane's place in a stage for ldmatrix: row lane % 16, chunk lane / 16,
  // with the row's swizzle. A row of tiles further is 16 rows, whole swizzle
  // patterns, and chunk c is an exclusive or of the address (the weights start
  // on a multiple of the pattern).
  const uint32_t lm = (lane & 15) * kPitch + ((lane >> 4) ^ (((lane & 15) >> kSwz) & (CH - 1))) * 16;

  const uint32_t flip = a.is_signed ? 0x00080008u : 0u;
  Offset<T> plain;  // without zero points: offset binary's 8 for signed lanes, else 0
  plain.set(flip);

  // the ring's next block to load, which runs ahead of the one in hand, over the CTA's tiles
  int l_tile = blockIdx.x, l_blk = warp, fill = 0, slot = 0, loaded = 0, used = 0;
  uint32_t par = 0;  // of the ring's round in hand
  bool ok = true;    // no wait has given up
  if (warp >= a.nblk) l_tile = a.tiles;  // no block is this warp's
  const uint8_t *l_scale = scale_of(l_tile * (16 * RT), lane, warp);  // the lane's row's, of the next block
  auto load_next = [&]() {
    if (l_tile < a.tiles) {
      load(l_tile * (16 * RT), l_blk, fill, l_scale);
      ++loaded;
      l_blk += kWarps;
      l_scale += kWarps * P::kGroups * 2;
      if (l_blk >= a.nblk) {
        l_blk = warp;
        l_tile += gridDim.x;
        l_scale = scale_of(l_tile * (16 * RT), lane, warp);
      }
    }
    ptx::cp_async_commit();
    fill = fill + 1 == kStages ? 0 : fill + 1;
  };
#pragma unroll 1
  for (int s = 0; s < kStages - 1; ++s) load_next();

  // the block's tokens (8 of them), or those of the chunk in hand and of the next (16: 20.4 us for 16 tokens by 8192 x
  // 8192 without the next, 18.0 with; for 32 the registers cost more, 33 us to 40); lanes without a token keep zeros
  constexpr int kHeld = NT == 1 ? CH : NT == 2 ? 4 : 1;
  uint4 xq[kHeld];
#pragma unroll
  for (int c = 0; c < kHeld; ++c) xq[c] = make_uint4(0, 0, 0, 0);
  const T *const x_lane = x + g * a.ldx + t * 8;
  auto load_token = [&](int64_t k0, int c, int j, uint4 &q) {
    if (8 * j + g < tokens) {
      if (kXVec && k0 + KB <= a.K)
        q = *reinterpret_cast<const uint4 *>(x_lane + (8 * j) * a.ldx + k0 + c * 32);
      else
        q = load_x8<T, kXVec>(x + (8 * j + g) * a.ldx, k0 + c * 32 + t * 8, a.K);
    }
  };
  auto load_tokens = [&](int64_t k0, int c) {  // NT = 2
    load_token(k0, c, 0, xq[(c & 1) * 2]);
    load_token(k0, c, 1, xq[(c & 1) * 2 + 1]);
  };
  int buf = 0;
  for (int tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const int n0 = tile * (16 * RT);
    float acc[kTiles][NT][4];
#pragma unroll
    for (int r = 0; r < kTiles; ++r)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[r][j][i] = 0.0f;
    // index of the rows' first scales, low bits (the place in a staged word)
    int first[kTiles][2];
    if (kZeros || P::kGroups == 1 || !a.s_vec)
#pragma unroll
      for (int r = 0; r < kTiles; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          first[r][h] = static_cast<int>(min(n0 + (kGated && r >= RT ? r - RT : r) * 16 + g + 8 * h, a.N - 1) * a.groups & 3);

    for (int blk = warp; blk < a.nblk; blk += kWarps) {
      const int64_t k0 = static_cast<int64_t>(blk) * KB;
      // tokens first: their way through L1 overlaps the wait for the stage
      const bool x_whole = kXVec && k0 + KB <= a.K;
      if constexpr (NT == 1) {
        if (g < tokens) {
          const T *const xr = x_lane + k0;
          if (x_whole) {
#pragma unroll
            for (int c = 0; c < CH; ++c) xq[c] = *reinterpret_cast<const uint4 *>(xr + c * 32);
          } else {
#pragma unroll
            for (int c = 0; c < CH; ++c) xq[c] = load_x8<T, kXVec>(x + g * a.ldx, k0 + c * 32 + t * 8, a.K);
          }
        }
      }
      if constexpr (NT == 2) load_tokens(k0, 0);
      ptx::cp_async_wait<kStages - 2>();
      __syncwarp();  // every lane's copies are in, and the slot filled next has been read by every lane
      load_next();
      const uint8_t *const st = sz + slot * P::kSzBytes;
      const uint32_t sw = w_s + slot * P::kWBytes;
      if (a.tma && ok) {
        ok = __all_sync(0xffffffffu, ptx::mbar_wait(bar0 + 8 * slot, par, a.status, SAMD_ETIMEOUT, kWaitLimitNs));
        used += ok;
        if (!ok) l_tile = a.tiles;  // nothing more is loaded
      }
      if (++slot == kStages) {
        slot = 0;
        par ^= 1;
      }
      const int g0 = static_cast<int>((k0 >> a.group_shift) & 3);
      // the rows' scales of the block, two in a word
      constexpr int kSW = (P::kGroups + 1) / 2;
      uint32_t sraw[kTiles][2][kSW];
#pragma unroll
      for (int r = 0; r < kTiles; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint8_t *const sp = st + (r * 16 + g + 8 * h) * P::kSPitch;
          if (P::kGroups > 1 && a.s_vec) {
            if constexpr (P::kGroups == 8) {
              const uint4 v = *reinterpret_cast<const uint4 *>(sp);
              sraw[r][h][0] = v.x, sraw[r][h][1] = v.y, sraw[r][h][2] = v.z, sraw[r][h][3] = v.w;
            }
            if constexpr (P::kGroups == 4) {
              const uint2 v = *reinterpret_cast<const uint2 *>(sp);
              sraw[r][h][0] = v.x, sraw[r][h][1] = v.y;
            }
            if constexpr (P::kGroups == 2) sraw[r][h][0] = *reinterpret_cast<const uint32_t *>(sp);
          } else {
            const uint16_t *const sh = reinterpret_cast<const uint16_t *>(sp) + ((first[r][h] + g0) & 1);
#pragma unroll
            for (int i = 0; i < kSW; ++i) {
              const int i0 = one_scale ? 0 : 2 * i;
              sraw[r][h][i] = sh[i0];
              if constexpr (P::kGroups > 1) sraw[r][h][i] |= static_cast<uint32_t>(sh[one_scale ? 0 : i0 + 1]) << 16;
            }
          }
        }
      // and their zero points, four in a word
      constexpr int kZW = (P::kGroups + 3) / 4;
      uint32_t zraw[kTiles][2][kZW];
      if constexpr (kZeros) {
#pragma unroll
        for (int r = 0; r < kTiles; ++r)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint8_t *const zp = st + P::kZOff + (r * 16 + g + 8 * h) * P::kZPitch;
            if (P::kGroups >= 4 && a.s_vec) {
#pragma unroll
              for (int i = 0; i < kZW; ++i) zraw[r][h][i] = reinterpret_cast<const uint32_t *>(zp)[i];
            } else {
              const uint8_t *const zb = zp + ((first[r][h] + g0) & 3);
#pragma unroll
              for (int i = 0; i < kZW; ++i) {
                zraw[r][h][i] = 0;
#pragma unroll
                for (int b = 0; b < 4; ++b)
                  if (4 * i + b < P::kGroups)
                    zraw[r][h][i] |= static_cast<uint32_t>(zb[one_scale ? 0 : 4 * i + b]) << 8 * b;
              }
            }
          }
      }
      if (k0 + KB > a.K) {
        // The last block of a row: past the row's end lanes and tokens are zero
        // and add nothing, whatever their scale, unless that is not finite.
        const int ng = static_cast<int>((a.K - k0 + 32 * CPG - 1) / (32 * CPG));  // groups with inputs
#pragma unroll
        for (int gi = 0; gi < P::kGroups; ++gi)
          if (gi >= ng) {
#pragma unroll
            for (int r = 0; r < kTiles; ++r)
#pragma unroll
              for (int h = 0; h < 2; ++h) sraw[r][h][gi / 2] &= gi & 1 ? 0x0000FFFFu : 0xFFFF0000u;
          }
      }
      uint32_t words[kTiles][4];
#pragma unroll
      for (int gi = 0; gi < P::kGroups; ++gi) {
        {
          float s[kTiles][2], d[kTiles][NT][4];
          Offset<T> o[kTiles][2];
#pragma unroll
          for (int r = 0; r < kTiles; ++r) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t w = sraw[r][h][gi / 2];
              s[r][h] = f32_of_bits<T>(static_cast<uint16_t>(gi & 1 ? w >> 16 : w));
              if constexpr (kZeros)
                // byte gi % 4, low four bits, in both halves
                o[r][h].set(__byte_perm(zraw[r][h][gi / 4], 0, 0x4040 | (gi & 3) | (gi & 3) << 8) & 0x000F000Fu);
              else
                o[r][h] = plain;
            }
          }
#pragma unroll
          for (int cc = 0; cc < CPG; ++cc) {
            const int c = gi * CPG + cc;
            {
              if ((c & 1) == 0) {  // two chunks at a time
#pragma unroll
                for (int r = 0; r < kTiles; ++r) {
                  ldmatrix_x4(((sw + lm) ^ (c * 16)) + r * (16 * kPitch), words[r]);
                }
              }
              if constexpr (NT == 2)
                if (c + 1 < CH) load_tokens(k0, c + 1);
              uint32_t b[NT][4];
#pragma unroll
              for (int j = 0; j < NT; ++j) {
                uint4 q = make_uint4(0, 0, 0, 0);
                if constexpr (NT == 1)
                  q = xq[c];
                else if constexpr (NT == 2)
                  q = xq[(c & 1) * 2 + j];
                else
                  load_token(k0, c, j, q);
                b[j][0] = __byte_perm(q.x, q.z, 0x5410);
                b[j][1] = __byte_perm(q.x, q.z, 0x7632);
                b[j][2] = __byte_perm(q.y, q.w, 0x5410);
                b[j][3] = __byte_perm(q.y, q.w, 0x7632);
              }
#pragma unroll
              for (int r = 0; r < kTiles; ++r) {
                uint32_t lo[4], hi[4];
                widen(words[r][2 * (c & 1)], flip, o[r][0], lo);
                widen(words[r][2 * (c & 1) + 1], flip, o[r][1], hi);
                const uint32_t a0[4] = {lo[0], hi[0], lo[1], hi[1]}, a1[4] = {lo[2], hi[2], lo[3], hi[3]};
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                  if (cc == 0)
                    mma16816<T, false>(d[r][j], a0, b[j][0], b[j][1]);
                  else
                    mma16816<T, true>(d[r][j], a0, b[j][0], b[j][1]);
                  mma16816<T, true>(d[r][j], a1, b[j][2], b[j][3]);
                }
              }
            }
          }
#pragma unroll
          for (int r = 0; r < kTiles; ++r)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[r][j][i] = fmaf(s[r][i >> 1], d[r][j][i], acc[r][j][i]);
        }
      }
    }

    // Join the warps' sums: [warp][row][token].
    const int pitch = P::red_pitch(tokens);
    float *const rb = red + buf * P::red_floats(tokens);
    if constexpr (P::kBufs == 2) buf ^= 1;
#pragma unroll
    for (int r = 0; r < kTiles; ++r)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (8 * j + 2 * t + (i & 1) < tokens)
            rb[(warp * kRows + r * 16 + g + (i >> 1) * 8) * pitch + 8 * j + 2 * t + (i & 1)] = acc[r][j][i];
    __syncthreads();
    T *const y = static_cast<T *>(a.y);
    for (int idx = threadIdx.x; idx < 16 * RT * tokens; idx += kThreads) {
      const int m = idx / (16 * RT), row = idx % (16 * RT);
      if (n0 + row < a.N) {
        float v = 0.0f, u = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          v += rb[(w * kRows + row) * pitch + m];
          if constexpr (kGated) u += rb[(w * kRows + 16 * RT + row) * pitch + m];
        }
        if constexpr (kGated) v = act_of(a.act, v) * u;
        y[(m0 + m) * a.ldy + n0 + row] = from_f32<T>(v);
      }
    }
    if constexpr (P::kBufs == 1) __syncthreads();
  }
  ptx::cp_async_wait<0>();
  if (!ok) {  // the CTA does not exit with a copy in flight
    int quiet = 0;
    for (int i = used; i < loaded; ++i)
      ptx::mbar_wait_bounded(bar0 + 8 * (i % kStages), (i / kStages) & 1, &quiet, kWaitLimitNs / 10);
  }
}

template <typename T, bool kGated, bool kZeros, bool kXVec, int RT, int NT, int CH, int CPG>
cudaError_t launch_as(MvArgs a, cudaStream_t s) {
  using P = Mv<T, kGated, kZeros, RT, NT, CH, CPG>;
  static_assert(P::smem(8 * NT) <= 227 * 1024, "a CTA's shared memory");
  a.nblk = (a.K + P::KB - 1) / P::KB;
  a.tiles = (a.N + 16 * RT - 1) / (16 * RT);
  a.s_vec = a.groups % P::kGroups == 0 && (1 << a.group_shift) * P::kGroups == P::KB;
  constexpr auto kern = matvec4_kernel<T, kGated, kZeros, kXVec, RT, NT, CH, CPG>;
  CUtensorMap map[2] = {};
  if (a.tma) {
    // bytes of a row by rows, in boxes of one block of one tile, swizzled as the kernel's ldmatrix reads them
    const EncodeTiledFn enc = tensor_map_encoder();
    if (!enc) return cudaErrorNotSupported;
    for (int i = 0; i < P::kMats; ++i) {
      const cuuint64_t dim[2] = {static_cast<cuuint64_t>(a.row_bytes), static_cast<cuuint64_t>(a.N)};
      const cuuint64_t stride[1] = {static_cast<cuuint64_t>(a.row_bytes)};
      const cuuint32_t box[2] = {P::kPitch, 16 * RT}, es[2] = {1, 1};
      if (enc(&map[i], CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t *>(a.lanes[i]), dim, stride, box, es,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CH == 8 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;
    }
  }
  const int most = a.M < 8 * NT ? a.M : 8 * NT;  // tokens of a CTA
  const size_t smem = P::smem(most);
  const cudaError_t e = conv::ensure_smem_attr(reinterpret_cast<const void *>(kern), smem);
  if (e != cudaSuccess) return e;
  int per_sm = resident_ctas<kern>(kThreads, P::smem(1));
  while (per_sm > 1 && per_sm * (smem + 1024) > (228u << 10)) --per_sm;  // (an SM's shared memory, 1 KB a CTA reserved)
  const int cap = sm_count() * per_sm;
  return launch_dependent(kern, dim3(a.tiles < cap ? a.tiles : cap, (a.M + 8 * NT - 1) / (8 * NT)), kThreads, smem, s, 1,
                          map[0], map[1], a);
}

template <typename T, bool kGated, bool kZeros, bool kXVec, int RT, int NT, int CH>
cudaError_t launch_grouped(const MvArgs &a, cudaStream_t s) {
  if (a.group_shift == 5) return launch_as<T, kGated, kZeros, kXVec, RT, NT, CH, 1>(a, s);
  if (a.group_shift == 6) return launch_as<T, kGated, kZeros, kXVec, RT, NT, CH, 2>(a, s);
  return launch_as<T, kGated, kZeros, kXVec, RT, NT, CH, 4>(a, s);
}

// Whether tiles of 32 rows still give every SM two CTAs.
inline bool two_row_tiles(int N) { return N >= 2 * 32 * sm_count(); }

// Which instance: 8, 16 or 32 tokens a pass. Up to eight: blocks of 256 inputs
// where there are at least eight of them for the warps (K = 1024 leaves half
// the warps idle with them), of 128 otherwise; two row tiles share a CTA's
// tokens and its fixed work where that still gives every SM two CTAs' worth
// (one token by 65536 x 4096 took 45.7 us with one and 37.8 with two, before
// the weights came by TMA), with blocks of 128 for more than two tokens, whose
// stages and sums would leave an SM one CTA.
template <typename T, bool kGated, bool kZeros>
cudaError_t launch_sized(const MvArgs &a, cudaStream_t s) {
  constexpr int kRT = kGated ? 1 : 2;
  if (!a.x_vec) {
    if (a.M > 16) return launch_grouped<T, kGated, kZeros, false, kRT, 4, 4>(a, s);
    if (a.M > 8) return launch_grouped<T, kGated, kZeros, false, kRT, 2, 4>(a, s);
    return launch_grouped<T, kGated, kZeros, false, 1, 1, 4>(a, s);
  }
  if (a.M > 16) return launch_grouped<T, kGated, kZeros, true, kRT, 4, 4>(a, s);
  if (a.M > 8) return launch_grouped<T, kGated, kZeros, true, kRT, 2, 4>(a, s);
  if (a.K < 2048) return launch_grouped<T, kGated, kZeros, true, 1, 1, 4>(a, s);
  if constexpr (!kGated)
    if (two_row_tiles(a.N))
      return a.M <= 2 ? launch_grouped<T, kGated, kZeros, true, 2, 1, 8>(a, s)
                      : launch_grouped<T, kGated, kZeros, true, 2, 1, 4>(a, s);
  return launch_grouped<T, kGated, kZeros, true, 1, 1, 8>(a, s);
}

template <typename T>
cudaError_t launch_type(const MvArgs &a, cudaStream_t s) {
  if (a.zeros[0]) return a.act >= 0 ? launch_sized<T, true, true>(a, s) : launch_sized<T, false, true>(a, s);
  return a.act >= 0 ? launch_sized<T, true, false>(a, s) : launch_sized<T, false, false>(a, s);
}

// One launcher a token type, each compiled in its own unit.
cudaError_t launch_bf16(const MvArgs &a, cudaStream_t s);
cudaError_t launch_f16(const MvArgs &a, cudaStream_t s);

}  // namespace mv
}  // namespace samd
