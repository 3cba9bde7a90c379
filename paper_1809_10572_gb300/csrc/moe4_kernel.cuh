// moe4_kernel.cuh -- a layer of experts on 4-bit weights for a few tokens:
//
//   h_p = w_p act(Wg_e x_m) * (Wu_e x_m),   y_m = sum over m's pairs p of Wd_e h_p
//
// for pairs p of a token m and an expert e = ids[p] with the weight w_p; two
// kernels, one for each line. h is rounded to the tokens' type, the second
// line's operand; everything else is in fp32 and rounded once.
//
// Bound by its reads: the weights of the experts that some token chose, half a
// byte each, come once for every eight pairs. An SM receives about 47 weights a
// clock, so what counts is instructions for a weight. The products go through
// mma.sync (m16n8k16: 16 rows of weights by eight pairs). A nibble over the
// mantissa of a power of two is that power plus the nibble; it is not taken off
// the weight, which would be an instruction for two of them, but off the sum:
// the accumulator starts with minus the power and the zero point times the same
// inputs, an MMA whose first operand is a constant row by row. Both products
// are exact; the sum of 32 .. 128 inputs then carries fp32's rounding of terms
// up to 1040 (fp16) or 143 (bf16) times an input, 2^-14 and 2^-17 of it at
// most: below the result's own rounding. (An infinity among a token's inputs
// gives that token NaNs.)
//
// Layout: as in matvec4_kernel.cuh: a word holds lanes 8w .. 8w + 7, one mask
// takes lanes i and i + 4 out together, so inputs run in the order (0,4),
// (1,5), (2,6), (3,7); ldmatrix deals word t of row r to lane 4 r + t. A tile is
// 16 rows: eight of Wg and the same eight of Wu, or 16 of Wd. Each warp has a
// ring of stages (16 rows of a block of 32 CH inputs, cp.async of 16 bytes a
// lane) that runs on over its tiles. A row's scales of a block are one load of
// lane r, a block ahead, dealt out by shuffles.
//
// Split: first kernel: tiles of all experts' rows in turn over one wave of
// CTAs, whose warps share a tile's inputs; second: a tile's pairs and inputs
// over the warps of a cluster of one to eight CTAs, each warp with its own sums
// of all tokens in shared memory, joined in a fixed order.
#pragma once

#include "matvec4_kernel.cuh"

namespace samd {
namespace moe {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kMaxPairs = 1024;    // of a launch
constexpr int kMaxTokens = 64;     // of a launch
constexpr int kMaxExperts = 1024;
constexpr int kCols = 8;           // pairs of a pass: the MMA's columns

struct MoeArgs {
  const uint8_t *lanes[2], *scales[2], *zeros[2];
  const uint8_t *x;        // tokens, or h (rows of pairs)
  uint8_t *y;              // h, or the layer's output
  const int32_t *ids;
  const float *weights;
  int64_t ldx, ldy;        // bytes
  int64_t row_bytes, groups;
  int M, N, K, E, topk;    // N rows of an expert's matrix, K inputs
  int group_shift;
  int nblk, tiles;
  int s_vec;               // a row's scales of a block lie on a multiple of their size
  int is_signed, act, splits;
};

// Which pairs go to which expert, in passes of up to kCols pairs of one expert.
struct Lists {
  uint16_t order[kMaxPairs];   // pairs, expert by expert, rising within one
  uint16_t expert[kMaxPairs];  // of a pass
  uint16_t first[kMaxPairs + 1];  // of a pass in `order`
  int passes;
};

// By one warp. count: E words. Pairs whose expert is none are in no list.
__device__ __forceinline__ void make_lists(const int32_t *ids, int pairs, int E, Lists *l, int *count, uint16_t *place, int lane) {
  for (int e = lane; e < E; e += 32) count[e] = 0;
  __syncwarp();
  for (int p0 = 0; p0 < pairs; p0 += 32) {
    const int p = p0 + lane;
    int e = p < pairs ? ids[p] : -1;
    if (e >= E || e < 0) e = -1;
    const uint32_t same = __match_any_sync(0xffffffffu, e);
    const int before = __popc(same & ((1u << lane) - 1));
    const int had = e >= 0 ? count[e] : 0;
    __syncwarp();
    if (e >= 0) {
      place[p] = static_cast<uint16_t>(had + before);
      if (before == 0) count[e] = had + __popc(same);
    }
    __syncwarp();
  }
  int pass = 0, at = 0;
  for (int e0 = 0; e0 < E; e0 += 32) {
    const int e = e0 + lane, n = e < E ? count[e] : 0, np = (n + kCols - 1) / kCols;
    int pn = np, nn = n;  // sums up to this lane
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int a = __shfl_up_sync(0xffffffffu, pn, o), b = __shfl_up_sync(0xffffffffu, nn, o);
      if (lane >= o) pn += a, nn += b;
    }
    for (int i = 0; i < np; ++i) {
      l->expert[pass + pn - np + i] = static_cast<uint16_t>(e);
      l->first[pass + pn - np + i] = static_cast<uint16_t>(at + nn - n + i * kCols);
    }
    __syncwarp();
    if (e < E) count[e] = at + nn - n;
    pass += __shfl_sync(0xffffffffu, pn, 31);
    at += __shfl_sync(0xffffffffu, nn, 31);
  }
  if (lane == 0) l->passes = pass, l->first[pass] = static_cast<uint16_t>(at);
  __syncwarp();
  for (int p = lane; p < pairs; p += 32) {
    const int e = ids[p];
    if (e >= 0 && e < E) l->order[count[e] + place[p]] = static_cast<uint16_t>(p);
  }
}

// Minus the power and the zero point z (in both halves), for the nibbles at bit 0 (lo) and bit 4 (hi).
template <typename T>
__device__ __forceinline__ void minus(uint32_t zz, uint32_t &lo, uint32_t &hi) {
  if constexpr (std::is_same<T, __half>::value)
    lo = 0xE400E400u | zz, hi = 0xD400D400u | zz << 4;
  else
    lo = hi = 0xC300C300u | zz;
}

// The eight lanes of a word as four pairs (i, i + 4), each plus its power; flip is 8 for signed lanes (both halves).
template <typename T>
__device__ __forceinline__ void widen(uint32_t w, uint32_t flip, uint32_t (&p)[4]) {
  if constexpr (std::is_same<T, __half>::value) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t v = w >> 8 * i;
      p[2 * i] = (v & 0x000F000Fu) ^ (0x64006400u | flip);
      p[2 * i + 1] = (v & 0x00F000F0u) ^ (0x54005400u | flip << 4);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = ((w >> 4 * i) & 0x000F000Fu) ^ (0x43004300u | flip);
  }
}

// CH: chunks of 32 inputs in a block; CPG: chunks of a block that share a scale.
template <int CH, int CPG>
struct Moe {
  static constexpr int KB = 32 * CH;
  static constexpr int kPitch = 16 * CH;
  static constexpr int kStage = 16 * kPitch;
  static constexpr int kStages = 4;
  static constexpr int kGroups = CH / CPG;  // scales of a row in a block
  static constexpr int kRing = kWarps * kStages * kStage;
  // first kernel: two buffers of [warp][row][pair]; second: [warp][row][token], then the joined [row][token]
  static constexpr int kRedPitch = kCols + 1;
  static constexpr int red_bytes(bool gated, int tokens) {
    return gated ? 2 * kWarps * 16 * kRedPitch * 4 : (kWarps + 1) * 16 * (tokens | 1) * 4;
  }
  static constexpr size_t smem(bool gated, int tokens) { return static_cast<size_t>(kRing) + red_bytes(gated, tokens); }
};

template <typename T, bool kGated, bool kZeros, int CH, int CPG>
__global__ void __launch_bounds__(kThreads, 2) moe4_kernel(const MoeArgs a) {
  using P = Moe<CH, CPG>;
  constexpr int KB = P::KB, kPitch = P::kPitch, kStages = P::kStages, kG = P::kGroups;
  constexpr int kSwz = CH >= 8 ? 0 : 1;  // rows that share a 128-byte line: 2^kSwz
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Lists lists;
  __shared__ int count[kMaxExperts];
  float *const red = reinterpret_cast<float *>(smem + P::kRing);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;

  // everything read may come from the kernel before; the next one may be set up
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();
  if (warp == 0) make_lists(a.ids, a.M * a.topk, a.E, &lists, count, reinterpret_cast<uint16_t *>(smem), lane);
  if constexpr (!kGated)
    for (int i = tid; i < kWarps * 16 * (a.M | 1); i += kThreads) red[i] = 0.0f;
  __syncthreads();

  const int rank = kGated ? 0 : blockIdx.x % a.splits;
  const int tile0 = kGated ? 0 : blockIdx.x / a.splits;  // the CTA's only tile
  const uint32_t ring = ptx::smem_addr(smem) + warp * kStages * P::kStage;
  // A walk over this warp's blocks: gated: items (pass, tile) of the CTA, and the warp's blocks of each; else the
  // warp's share of the blocks of all passes.
  struct At {
    int item, pass, tile, blk;
  };
  const int items = lists.passes * a.tiles;
  auto settle = [&](At &w) {  // pass and tile of an item, the pass behind the last at the end
    if constexpr (kGated) {
      if (w.item >= items) {
        w.pass = lists.passes;
      } else {
        w.pass = w.item / a.tiles;
        w.tile = w.item - w.pass * a.tiles;
      }
    } else {
      while (w.blk >= a.nblk) w.blk -= a.nblk, ++w.pass;
    }
  };
  auto begin = [&]() {
    At w = {static_cast<int>(blockIdx.x), 0, tile0, kGated ? warp : rank * kWarps + warp};
    settle(w);
    if (kGated && warp >= a.nblk) w.pass = lists.passes;  // no block is this warp's
    return w;
  };
  auto next = [&](At &w) {
    if constexpr (kGated) {
      w.blk += kWarps;
      if (w.blk >= a.nblk) {
        w.blk = warp;
        w.item += gridDim.x;
        settle(w);
      }
    } else {
      w.blk += kWarps * a.splits;
      settle(w);
    }
  };

  // ---- loading: row r of a tile is row n of matrix m
  auto row_index = [&](const At &w, int r) -> int64_t {
    const int n = kGated ? w.tile * 8 + (r & 7) : w.tile * 16 + r;
    return static_cast<int64_t>(lists.expert[w.pass]) * a.N + n;
  };
  At ahead = begin();
  int fill = 0;
  auto load_next = [&]() {
    if (ahead.pass < lists.passes) {
      const uint32_t st = ring + fill * P::kStage;
      constexpr int kLanes = CH, kStep = 32 / kLanes;  // lanes of a row, rows of a warp's copy
      const int c = lane % kLanes, r0 = lane / kLanes;
      const int64_t at = static_cast<int64_t>(ahead.blk) * (KB / 2) + c * 16;
      const uint32_t n = at < a.row_bytes ? 16u : 0u;
      const int64_t off = row_index(ahead, r0) * a.row_bytes + (n ? at : 0);
#pragma unroll
      for (int i = 0; i < 16 / kStep; ++i) {
        const int r = i * kStep + r0;
        const uint8_t *const m = a.lanes[kGated && i * kStep >= 8];
        const int up = kGated ? (i * kStep) & 7 : i * kStep;  // rows further than r0
        ptx::cp_async_16(st + r * kPitch + ((c ^ ((r >> kSwz) & (CH - 1))) * 16), m + off + up * a.row_bytes, n);
      }
      next(ahead);
    }
    ptx::cp_async_commit();
    fill = fill + 1 == kStages ? 0 : fill + 1;
  };
  // lane r's row's scales and zero points of a block; those behind the row's end are zero
  constexpr int kSW = (kG + 1) / 2, kZW = (kG + 3) / 4;
  auto load_scales = [&](const At &w, uint32_t (&s)[kSW], uint32_t (&z)[kZW]) {
#pragma unroll
    for (int i = 0; i < kSW; ++i) s[i] = 0;
#pragma unroll
    for (int i = 0; i < kZW; ++i) z[i] = 0;
    if (lane < 16 && w.pass < lists.passes) {
      const int m = kGated && lane >= 8;
      const int64_t grp = (static_cast<int64_t>(w.blk) * KB) >> a.group_shift;
      const int64_t at = row_index(w, lane) * a.groups + grp;
      const uint16_t *const sp = reinterpret_cast<const uint16_t *>(a.scales[m]) + at;
      const uint8_t *const zp = a.zeros[m] + at;
      if (kG > 1 && a.s_vec) {
        if constexpr (kG == 8) {
          const uint4 v = *reinterpret_cast<const uint4 *>(sp);
          s[0] = v.x, s[1] = v.y, s[2] = v.z, s[3] = v.w;
          if constexpr (kZeros) {
            const uint2 q = *reinterpret_cast<const uint2 *>(zp);
            z[0] = q.x, z[1] = q.y;
          }
        } else if constexpr (kG == 4) {
          const uint2 v = *reinterpret_cast<const uint2 *>(sp);
          s[0] = v.x, s[1] = v.y;
          if constexpr (kZeros) z[0] = *reinterpret_cast<const uint32_t *>(zp);
        } else if constexpr (kG == 2) {
          s[0] = *reinterpret_cast<const uint32_t *>(sp);
          if constexpr (kZeros) z[0] = *reinterpret_cast<const uint16_t *>(zp);
        }
      } else {
#pragma unroll
        for (int i = 0; i < kG; ++i) {
          // groups of more than a block: the same one for all of it
          const int j = CPG == 4 && a.group_shift > 7 ? static_cast<int>(((static_cast<int64_t>(w.blk) * KB + i * 128) >> a.group_shift) - grp) : i;
          if (grp + j < a.groups) {
            s[i / 2] |= static_cast<uint32_t>(sp[j]) << 16 * (i & 1);
            if constexpr (kZeros) z[i / 4] |= static_cast<uint32_t>(zp[j]) << 8 * (i & 3);
          }
        }
      }
    }
  };

  At have = begin();
  uint32_t s_next[kSW], z_next[kZW];
  load_scales(have, s_next, z_next);
#pragma unroll 1
  for (int i = 0; i < kStages - 1; ++i) load_next();

  const uint32_t lm = (lane & 15) * kPitch + ((lane >> 4) ^ (((lane & 15) >> kSwz) & (CH - 1))) * 16;
  const uint32_t flip = a.is_signed ? 0x00080008u : 0u;
  uint32_t plain_lo, plain_hi;
  minus<T>(flip, plain_lo, plain_hi);

  float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  int slot = 0;
  // one block: its products into acc
  auto block = [&]() {
    const int first = lists.first[have.pass], n = min(static_cast<int>(lists.first[have.pass + 1]) - first, kCols);
    const int64_t k0 = static_cast<int64_t>(have.blk) * KB;
    uint4 xq[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) xq[c] = make_uint4(0, 0, 0, 0);
    if (g < n) {
      const int pair = lists.order[first + g];
      const uint8_t *const xr = a.x + (kGated ? pair / a.topk : pair) * a.ldx + (k0 + t * 8) * 2;
#pragma unroll
      for (int c = 0; c < CH; ++c)
        if (k0 + c * 32 < a.K) xq[c] = *reinterpret_cast<const uint4 *>(xr + c * 64);
    }
    uint32_t s[kSW], z[kZW];
#pragma unroll
    for (int i = 0; i < kSW; ++i) s[i] = s_next[i];
#pragma unroll
    for (int i = 0; i < kZW; ++i) z[i] = z_next[i];
    At then = have;
    next(then);
    load_scales(then, s_next, z_next);
    ptx::cp_async_wait<kStages - 2>();
    __syncwarp();  // every lane's copies are in, and the stage filled next has been read by every lane
    load_next();
    const uint32_t sw = ring + slot * P::kStage;
    slot = slot + 1 == kStages ? 0 : slot + 1;
    uint32_t words[4], s0 = 0, s1 = 0, z0 = 0, z1 = 0;
#pragma unroll
    for (int gi = 0; gi < kG; ++gi) {
      if ((gi & 1) == 0) {
        s0 = __shfl_sync(0xffffffffu, s[gi / 2], g);
        s1 = __shfl_sync(0xffffffffu, s[gi / 2], g + 8);
      }
      uint32_t lo0 = plain_lo, lo1 = plain_lo, hi0 = plain_hi, hi1 = plain_hi;
      if constexpr (kZeros) {
        if ((gi & 3) == 0) {
          z0 = __shfl_sync(0xffffffffu, z[gi / 4], g);
          z1 = __shfl_sync(0xffffffffu, z[gi / 4], g + 8);
        }
        constexpr uint32_t kLow = 0x000F000Fu;
        minus<T>(__byte_perm(z0, 0, 0x4040 | (gi & 3) | (gi & 3) << 8) & kLow, lo0, hi0);
        minus<T>(__byte_perm(z1, 0, 0x4040 | (gi & 3) | (gi & 3) << 8) & kLow, lo1, hi1);
      }
      const uint32_t less[4] = {lo0, lo1, hi0, hi1};
      float d[4];
#pragma unroll
      for (int cc = 0; cc < CPG; ++cc) {
        const int c = gi * CPG + cc;
        if ((c & 1) == 0) mv::ldmatrix_x4((sw + lm) ^ (c * 16), words);
        const uint4 q = xq[c];
        const uint32_t b0 = __byte_perm(q.x, q.z, 0x5410), b1 = __byte_perm(q.x, q.z, 0x7632);
        const uint32_t b2 = __byte_perm(q.y, q.w, 0x5410), b3 = __byte_perm(q.y, q.w, 0x7632);
        uint32_t lo[4], hi[4];
        widen<T>(words[2 * (c & 1)], flip, lo);
        widen<T>(words[2 * (c & 1) + 1], flip, hi);
        const uint32_t a0[4] = {lo[0], hi[0], lo[1], hi[1]}, a1[4] = {lo[2], hi[2], lo[3], hi[3]};
        if (cc == 0)
          mv::mma16816<T, false>(d, less, b0, b1);
        else
          mv::mma16816<T, true>(d, less, b0, b1);
        mv::mma16816<T, true>(d, less, b2, b3);
        mv::mma16816<T, true>(d, a0, b0, b1);
        mv::mma16816<T, true>(d, a1, b2, b3);
      }
      const float f0 = mv::f32_of_bits<T>(static_cast<uint16_t>(gi & 1 ? s0 >> 16 : s0));
      const float f1 = mv::f32_of_bits<T>(static_cast<uint16_t>(gi & 1 ? s1 >> 16 : s1));
      acc[0] = fmaf(f0, d[0], acc[0]), acc[1] = fmaf(f0, d[1], acc[1]);
      acc[2] = fmaf(f1, d[2], acc[2]), acc[3] = fmaf(f1, d[3], acc[3]);
    }
    have = then;
  };

  if constexpr (kGated) {
    int buf = 0;
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
      while (have.pass < lists.passes && have.item == item) block();
      const int pass = item / a.tiles, n0 = (item - pass * a.tiles) * 8;
      const int first = lists.first[pass], n = min(static_cast<int>(lists.first[pass + 1]) - first, kCols);
      float *const rb = red + buf * (kWarps * 16 * P::kRedPitch);
      buf ^= 1;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        rb[(warp * 16 + g + (i >> 1) * 8) * P::kRedPitch + 2 * t + (i & 1)] = acc[i];
        acc[i] = 0.0f;
      }
      __syncthreads();
      // (the other buffer is written next, and this one only behind another barrier)
      if (tid < 8 * n) {
        const int r = tid & 7, c = tid >> 3, pair = lists.order[first + c];
        float gate = 0.0f, up = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          gate += rb[(w * 16 + r) * P::kRedPitch + c];
          up += rb[(w * 16 + 8 + r) * P::kRedPitch + c];
        }
        reinterpret_cast<T *>(a.y + pair * a.ldy)[n0 + r] = from_f32<T>(a.weights[pair] * (act_of(a.act, gate) * up));
      }
    }
  } else {
    const int pitch = a.M | 1;
    float *const mine = red + warp * 16 * pitch;
    while (have.pass < lists.passes) {
      const int pass = have.pass;
      block();
      if (have.pass != pass) {
        // into the tokens' sums, column by column: a token may have the same expert twice
        const int first = lists.first[pass], n = min(static_cast<int>(lists.first[pass + 1]) - first, kCols);
        for (int c = 0; c < n; ++c) {
          if (t == c >> 1) {
            const int m = lists.order[first + c] / a.topk;
            mine[g * pitch + m] += c & 1 ? acc[1] : acc[0];
            mine[(g + 8) * pitch + m] += c & 1 ? acc[3] : acc[2];
          }
          __syncwarp();
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = 0.0f;
      }
    }
    __syncthreads();
    float *const sum = red + kWarps * 16 * pitch;
    for (int i = tid; i < 16 * a.M; i += kThreads) {
      const int m = i >> 4, r = i & 15;
      float v = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) v += red[(w * 16 + r) * pitch + m];
      if (a.splits == 1)
        reinterpret_cast<T *>(a.y + m * a.ldy)[tile0 * 16 + r] = from_f32<T>(v);
      else
        sum[r * pitch + m] = v;
    }
    if (a.splits > 1) {
      __syncthreads();
      ptx::cluster_sync();
      if (rank == 0)
        for (int i = tid; i < 16 * a.M; i += kThreads) {
          const int m = i >> 4, r = i & 15;
          float v = 0.0f;
          for (int k = 0; k < a.splits; ++k) {
            float p;
            asm volatile("ld.shared::cluster.f32 %0, [%1];"
                         : "=f"(p)
                         : "r"(ptx::map_to_rank(ptx::smem_addr(sum + r * pitch + m), k))
                         : "memory");
            v += p;
          }
          reinterpret_cast<T *>(a.y + m * a.ldy)[tile0 * 16 + r] = from_f32<T>(v);
        }
      __syncthreads();
      ptx::cluster_sync();  // no CTA ends while its sums are read
    }
  }
  ptx::cp_async_wait<0>();
}

template <typename T, bool kGated, bool kZeros, int CH, int CPG>
cudaError_t launch_as(MoeArgs a, cudaStream_t s) {
  using P = Moe<CH, CPG>;
  a.nblk = (a.K + P::KB - 1) / P::KB;
  a.tiles = a.N / (kGated ? 8 : 16);
  a.s_vec = a.groups % P::kGroups == 0 && (1 << a.group_shift) * P::kGroups == P::KB;
  constexpr auto kern = moe4_kernel<T, kGated, kZeros, CH, CPG>;
  const size_t smem = P::smem(kGated, a.M);
  const cudaError_t e = conv::ensure_smem_attr(reinterpret_cast<const void *>(kern), smem);
  if (e != cudaSuccess) return e;
  const int64_t pairs = static_cast<int64_t>(a.M) * a.topk;
  const int slots = 2 * sm_count();
  if (kGated) {
    const int64_t most = pairs * a.tiles;
    a.splits = 1;
    return launch_dependent(kern, dim3(static_cast<unsigned>(most < slots ? most : slots)), kThreads, smem, s, 1, a);
  }
  // a tile's blocks over as many CTAs as fill the GPU, while each warp still has a block
  const int64_t blocks = (pairs < a.E ? pairs : a.E) * a.nblk;
  a.splits = 1;
  while (a.splits < 8 && static_cast<int64_t>(a.tiles) * a.splits * 2 <= slots && blocks >= 2 * kWarps * a.splits) a.splits *= 2;
  return launch_dependent(kern, dim3(a.tiles * a.splits), kThreads, smem, s, a.splits, a);
}

template <typename T, bool kGated, bool kZeros, int CH>
cudaError_t launch_grouped(const MoeArgs &a, cudaStream_t s) {
  if (a.group_shift == 5) return launch_as<T, kGated, kZeros, CH, 1>(a, s);
  if (a.group_shift == 6) return launch_as<T, kGated, kZeros, CH, 2>(a, s);
  return launch_as<T, kGated, kZeros, CH, 4>(a, s);
}

// Blocks of 256 inputs where every warp gets one, else of 128.
template <typename T, bool kGated, bool kZeros>
cudaError_t launch_sized(const MoeArgs &a, cudaStream_t s) {
  return a.K >= 256 * kWarps ? launch_grouped<T, kGated, kZeros, 8>(a, s) : launch_grouped<T, kGated, kZeros, 4>(a, s);
}

template <typename T>
cudaError_t launch_type(const MoeArgs &a, bool gated, cudaStream_t s) {
  if (gated) return a.zeros[0] ? launch_sized<T, true, true>(a, s) : launch_sized<T, true, false>(a, s);
  return a.zeros[0] ? launch_sized<T, false, true>(a, s) : launch_sized<T, false, false>(a, s);
}

// One launcher a token type, each compiled in its own unit.
cudaError_t launch_bf16(const MoeArgs &a, bool gated, cudaStream_t s);
cudaError_t launch_f16(const MoeArgs &a, bool gated, cudaStream_t s);

}  // namespace moe

cudaError_t launch_moe_route(const samd_moe_desc &d, bool normalize, const void *x, const void *router, int32_t *ids,
                             float *weights, cudaStream_t s);
size_t moe4_workspace(const samd_moe_desc &d);
cudaError_t launch_moe4(const samd_moe_desc &d, samd_fmt fw, const void *x, const int32_t *ids, const float *weights,
                        const samd_weights4 &gate, const samd_weights4 &up, const samd_weights4 &down, void *y,
                        void *workspace, cudaStream_t s);

}  // namespace samd
