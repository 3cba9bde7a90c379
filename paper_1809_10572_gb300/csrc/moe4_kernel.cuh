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
// mantissa of a power of two is that power plus the nibble; the power and the zero
// point are taken off it, exactly, so that the products are those of the integers
// and a sum knows nothing of inputs whose weights are zero. Taken off the sums
// instead (an MMA with a constant operand for each of these) a channel 1000 times
// the others left half of fp16's rounding in them, and the time is the same: the
// subtraction has a pipe of its own, and the chains of MMAs are half as long (13
// tokens, 46 of 64 experts of 2048 x 1408, bf16: 79.9 us a layer, off the sums 80.5;
// with zero points in fp16 83.4 and 82.1).
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
// warps, where there are enough, or of CTAs, whose warps share a tile's inputs;
// second: a tile's pairs and inputs in runs over the warps of a cluster of one to
// eight CTAs, each warp with its own sums of all tokens in shared memory, joined
// in a fixed order.
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
  float weight[kMaxPairs];     // of the pairs in `order`
  int passes;
};

// By one warp. count: E words. Pairs whose expert is none are in no list.
__device__ __forceinline__ void make_lists(const int32_t *ids, const float *weights, int pairs, int E, Lists *l, int *count,
                                           uint16_t *place, int lane) {
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
    if (e >= 0 && e < E) {
      l->order[count[e] + place[p]] = static_cast<uint16_t>(p);
      l->weight[count[e] + place[p]] = weights[p];
    }
  }
}

// d = a b, or d += a b; without side effects, so that the compiler may place it.
template <typename T>
__device__ __forceinline__ void mma_pure(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, bool add) {
  const float c0 = add ? d[0] : 0.0f, c1 = add ? d[1] : 0.0f, c2 = add ? d[2] : 0.0f, c3 = add ? d[3] : 0.0f;
  if constexpr (std::is_same<T, __half>::value)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, "
        "%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, "
        "%12, %13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}

// RT: row tiles of 16 rows in a tile; CH: chunks of 32 inputs in a block; CPG: chunks of a block that share a scale.
template <int RT, int CH, int CPG>
struct Moe {
  static constexpr int KB = 32 * CH;
  static constexpr int kRows = 16 * RT;
  static constexpr int kPitch = 16 * CH;
  static constexpr int kStage = kRows * kPitch;
  static constexpr int kStages = 4;
  static constexpr int kGroups = CH / CPG;  // scales of a row in a block
  static constexpr int kRing = kWarps * kStages * kStage;
  // first kernel: two buffers of [warp][row][pair]; second: [warp][row][token], then the joined [row][token]
  static constexpr int kRedPitch = kCols + 1;
  static constexpr int red_bytes(bool gated, int tokens) {
    return gated ? 2 * kWarps * kRows * kRedPitch * 4 : (kWarps + 1) * kRows * (tokens | 1) * 4;
  }
  static constexpr size_t smem(bool gated, int tokens) { return static_cast<size_t>(kRing) + red_bytes(gated, tokens); }
};

// kOwn (first kernel): a tile is one warp's, over all inputs; else the CTA's, and its warps share the inputs.
template <typename T, bool kGated, bool kOwn, bool kZeros, int RT, int CH, int CPG>
__global__ void __launch_bounds__(kThreads, 2) moe4_kernel(const MoeArgs a) {
  using P = Moe<RT, CH, CPG>;
  constexpr int KB = P::KB, kRows = P::kRows, kPitch = P::kPitch, kStages = P::kStages, kG = P::kGroups;
  static_assert(CH == 4, "a row of a stage is 64 bytes");
  constexpr int kSwz = 1;                          // rows that share a 128-byte line: 2^kSwz
  constexpr int kOut = kGated ? kRows / 2 : kRows; // rows of a matrix in a tile
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Lists lists;
  float *const red = reinterpret_cast<float *>(smem + P::kRing);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;

  // everything read may come from the kernel before; the next one may be set up
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();
  if (warp == 0)  // (the ring is not in use yet)
    make_lists(a.ids, a.weights, a.M * a.topk, a.E, &lists, reinterpret_cast<int *>(smem),
               reinterpret_cast<uint16_t *>(smem + kMaxExperts * 4), lane);
  if constexpr (!kGated)
    for (int i = tid; i < kWarps * kRows * (a.M | 1); i += kThreads) red[i] = 0.0f;
  __syncthreads();

  // A warp's blocks, one after the other. First kernel: items (pass and tile) of the warp, with all of their blocks, or of
  // the CTA, with every eighth; second: the CTA's tile, and of the blocks of all passes a run (which ends few passes, where
  // sums change hands).
  const int rank = kGated ? 0 : blockIdx.x % a.splits;
  const int passes = lists.passes, items = passes * a.tiles;
  const int first_blk = kGated && !kOwn ? warp : 0, stride = kGated && !kOwn ? kWarps : 1;
  const int first_item = kOwn ? static_cast<int>(blockIdx.x) * kWarps + warp : static_cast<int>(blockIdx.x);
  const int item_step = kOwn ? static_cast<int>(gridDim.x) * kWarps : static_cast<int>(gridDim.x);
  struct At {
    int item, pass, tile, blk;  // item: second kernel: blocks of the run from this one on
  };
  auto seek_item = [&](At &w) {
    w.pass = passes;
    if (w.item < items) {
      w.pass = w.item / a.tiles;
      w.tile = w.item - w.pass * a.tiles;
    }
  };
  auto advance = [&](At &w) {  // to the next block; true where the pass or the tile is another one
    w.blk += stride;
    if constexpr (kGated) {
      if (w.blk < a.nblk) return false;
      w.blk = first_blk;
      w.item += item_step;
      seek_item(w);
    } else {
      if (--w.item <= 0) {
        w.pass = passes;
        return true;
      }
      if (w.blk < a.nblk) return false;
      w.blk = 0;
      ++w.pass;
    }
    return true;
  };
  At have = {first_item, 0, kGated ? 0 : static_cast<int>(blockIdx.x) / a.splits, first_blk};
  if constexpr (kGated) {
    seek_item(have);
    if (first_blk >= a.nblk) have.pass = passes;  // nothing is this warp's
  } else {
    const int64_t all = static_cast<int64_t>(passes) * a.nblk, me = rank * kWarps + warp, of = kWarps * a.splits;
    const int begin = static_cast<int>(all * me / of);
    have.item = static_cast<int>(all * (me + 1) / of) - begin;
    have.pass = have.item > 0 ? begin / a.nblk : passes;
    have.blk = begin % a.nblk;
  }

  // ---- loading. Row r of a tile: 16-row tiles of eight rows of each matrix, or of sixteen of the one.
  const int64_t expert_bytes = a.N * a.row_bytes, expert_scales = a.N * a.groups;
  const int lc = (lane % CH) * 16, lr = lane / CH;  // a copy: the lane's bytes of a row, and row
  const uint32_t ring = ptx::smem_addr(smem) + warp * kStages * P::kStage;
  const uint32_t copy_at = lr * kPitch + ((lc / 16) ^ ((lr >> kSwz) & (CH - 1))) * 16;
  At ahead = have;
  const uint8_t *w_row[kGated ? 2 : 1];
  auto seek = [&]() {
    if (ahead.pass < passes) {
      const int64_t off = lists.expert[ahead.pass] * expert_bytes + static_cast<int64_t>(ahead.tile * kOut + lr) * a.row_bytes + lc;
      w_row[0] = a.lanes[0] + off;
      if constexpr (kGated) w_row[1] = a.lanes[1] + off;
    }
  };
  seek();
  int fill = 0;
  auto load_next = [&]() {
    if (ahead.pass < passes) {
      const uint32_t st = ring + fill * P::kStage;
      const int at = ahead.blk * (KB / 2);
      if (at + lc < a.row_bytes) {  // (behind a row's end the stage keeps what it holds: any lanes, times inputs of zero)
        constexpr int kStep = 32 / CH;  // rows of a warp's copy
#pragma unroll
        for (int i = 0; i < kRows / kStep; ++i) {
          constexpr int kEight = 8 / kStep;  // copies of eight rows
          const int r = i * kStep;           // and lr: of the stage
          const int m = kGated ? (i / kEight) & 1 : 0;
          const int n = kGated ? (i / (2 * kEight)) * 8 + (i % kEight) * kStep : r;  // of the matrix
          // (lr is below kStep, so row lr + r is swizzled by the exclusive or of both)
          ptx::cp_async_16(st + (copy_at ^ ((r >> kSwz) & (CH - 1)) * 16) + r * kPitch, w_row[m] + n * a.row_bytes + at);
        }
      }
      if (advance(ahead)) seek();
    }
    ptx::cp_async_commit();
    fill = fill + 1 == kStages ? 0 : fill + 1;
  };
  // lane r's row's scales and zero points of a block; those behind the row's end are zero
  constexpr int kSW = (kG + 1) / 2, kZW = (kG + 3) / 4;
  const bool scale_lane = kRows >= 32 || lane < kRows;
  int64_t s_row = 0;  // of the item in hand: the row's first scale
  const uint16_t *s_base = reinterpret_cast<const uint16_t *>(a.scales[0]);
  const uint8_t *z_base = a.zeros[0];
  if (kGated && (lane & 8)) s_base = reinterpret_cast<const uint16_t *>(a.scales[1]), z_base = a.zeros[1];
  auto seek_scales = [&](const At &w) {
    const int n = kGated ? w.tile * kOut + (lane >> 4) * 8 + (lane & 7) : w.tile * kOut + lane;
    if (w.pass < passes && scale_lane) s_row = lists.expert[w.pass] * expert_scales + n * a.groups;
  };
  auto load_scales = [&](const At &w, uint32_t (&s)[kSW], uint32_t (&z)[kZW]) {
    if (!scale_lane || w.pass >= passes) return;
    const int64_t grp = (static_cast<int64_t>(w.blk) * KB) >> a.group_shift;
    const uint16_t *const sp = s_base + s_row + grp;
    const uint8_t *const zp = z_base + s_row + grp;
    if (kG > 1 && a.s_vec) {
      if constexpr (kG == 4) {
        const uint2 v = *reinterpret_cast<const uint2 *>(sp);
        s[0] = v.x, s[1] = v.y;
        if constexpr (kZeros) z[0] = *reinterpret_cast<const uint32_t *>(zp);
      } else if constexpr (kG == 2) {
        s[0] = *reinterpret_cast<const uint32_t *>(sp);
        if constexpr (kZeros) z[0] = *reinterpret_cast<const uint16_t *>(zp);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kSW; ++i) s[i] = 0;
#pragma unroll
      for (int i = 0; i < kZW; ++i) z[i] = 0;
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
  };

  uint32_t s_next[kSW] = {}, z_next[kZW] = {};
  seek_scales(have);
  load_scales(have, s_next, z_next);
  const uint8_t *x_row = nullptr;
  // the lane's column of a pass: its inputs; lanes without a pair read the first one's, and their sums are not used
  auto seek_inputs = [&](int pass) {
    if (pass < passes) {
      const int first = lists.first[pass], n = min(static_cast<int>(lists.first[pass + 1]) - first, kCols);
      const int pair = lists.order[first + (g < n ? g : 0)];
      x_row = a.x + (kGated ? pair / a.topk : pair) * a.ldx + t * 16;
    }
  };
  seek_inputs(have.pass);
#pragma unroll 1
  for (int i = 0; i < kStages - 1; ++i) load_next();

  const uint32_t lm = (lane & 15) * kPitch + ((lane >> 4) ^ (((lane & 15) >> kSwz) & (CH - 1))) * 16;
  const uint32_t flip = a.is_signed ? 0x00080008u : 0u;
  mv::Offset<T> plain;
  plain.set(flip);

  float acc[RT][4] = {};
  int slot = 0;
  // one block: its products into acc; true where the next one is of another pass or tile
  auto block = [&]() {
    uint4 xq[CH];
    const int k0 = have.blk * KB;
    if (k0 + KB <= a.K) {
#pragma unroll
      for (int c = 0; c < CH; ++c) xq[c] = *reinterpret_cast<const uint4 *>(x_row + k0 * 2 + c * 64);
    } else {
#pragma unroll
      for (int c = 0; c < CH; ++c)
        xq[c] = k0 + c * 32 < a.K ? *reinterpret_cast<const uint4 *>(x_row + k0 * 2 + c * 64) : make_uint4(0, 0, 0, 0);
    }
    uint32_t s[kSW], z[kZW];
#pragma unroll
    for (int i = 0; i < kSW; ++i) s[i] = s_next[i];
#pragma unroll
    for (int i = 0; i < kZW; ++i) z[i] = z_next[i];
    const bool other = advance(have);
    if (other) {
      seek_scales(have);
      seek_inputs(have.pass);
    }
    load_scales(have, s_next, z_next);
    ptx::cp_async_wait<kStages - 2>();
    __syncwarp();  // every lane's copies are in, and the stage filled next has been read by every lane
    load_next();
    const uint32_t sw = ring + slot * P::kStage;
    slot = slot + 1 == kStages ? 0 : slot + 1;
    uint32_t words[RT][4], sc[RT][2] = {}, zc[RT][2] = {};
#pragma unroll
    for (int gi = 0; gi < kG; ++gi) {
      mv::Offset<T> less[RT][2];
#pragma unroll
      for (int q = 0; q < RT; ++q) {
        if ((gi & 1) == 0) {
          sc[q][0] = __shfl_sync(0xffffffffu, s[gi / 2], 16 * q + g);
          sc[q][1] = __shfl_sync(0xffffffffu, s[gi / 2], 16 * q + g + 8);
        }
        less[q][0] = less[q][1] = plain;
        if constexpr (kZeros) {
          if ((gi & 3) == 0) {
            zc[q][0] = __shfl_sync(0xffffffffu, z[gi / 4], 16 * q + g) & 0x0F0F0F0Fu;
            zc[q][1] = __shfl_sync(0xffffffffu, z[gi / 4], 16 * q + g + 8) & 0x0F0F0F0Fu;
          }
          const int sel = 0x4040 | (gi & 3) | (gi & 3) << 8;
#pragma unroll
          for (int r = 0; r < 2; ++r) less[q][r].set(__byte_perm(zc[q][r], 0, sel));
        }
      }
      float d[RT][4];
#pragma unroll
      for (int cc = 0; cc < CPG; ++cc) {
        const int c = gi * CPG + cc;
        if ((c & 1) == 0)
#pragma unroll
          for (int q = 0; q < RT; ++q) mv::ldmatrix_x4(((sw + lm) ^ (c * 16)) + q * (16 * kPitch), words[q]);
        const uint4 v = xq[c];
        const uint32_t b0 = __byte_perm(v.x, v.z, 0x5410), b1 = __byte_perm(v.x, v.z, 0x7632);
        const uint32_t b2 = __byte_perm(v.y, v.w, 0x5410), b3 = __byte_perm(v.y, v.w, 0x7632);
#pragma unroll
        for (int q = 0; q < RT; ++q) {
          uint32_t lo[4], hi[4];
          mv::widen(words[q][2 * (c & 1)], flip, less[q][0], lo);
          mv::widen(words[q][2 * (c & 1) + 1], flip, less[q][1], hi);
          const uint32_t a0[4] = {lo[0], hi[0], lo[1], hi[1]}, a1[4] = {lo[2], hi[2], lo[3], hi[3]};
          mma_pure<T>(d[q], a0, b0, b1, cc > 0);
          mma_pure<T>(d[q], a1, b2, b3, true);
        }
      }
#pragma unroll
      for (int q = 0; q < RT; ++q) {
        const float f0 = mv::f32_of_bits<T>(static_cast<uint16_t>(gi & 1 ? sc[q][0] >> 16 : sc[q][0]));
        const float f1 = mv::f32_of_bits<T>(static_cast<uint16_t>(gi & 1 ? sc[q][1] >> 16 : sc[q][1]));
        acc[q][0] = fmaf(f0, d[q][0], acc[q][0]), acc[q][1] = fmaf(f0, d[q][1], acc[q][1]);
        acc[q][2] = fmaf(f1, d[q][2], acc[q][2]), acc[q][3] = fmaf(f1, d[q][3], acc[q][3]);
      }
    }
    return other;
  };

  if constexpr (kOwn) {
    // gate and up of a hidden column are the same thread's
    while (have.pass < passes) {
      const int pass = have.pass, n0 = have.tile * kOut;
      while (!block()) {
      }
      const int first = lists.first[pass], n = min(static_cast<int>(lists.first[pass + 1]) - first, kCols);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (2 * t + i < n) {
          const int c = first + 2 * t + i;
          T *const to = reinterpret_cast<T *>(a.y + lists.order[c] * a.ldy) + n0 + g;
#pragma unroll
          for (int q = 0; q < RT; ++q) to[8 * q] = from_f32<T>(lists.weight[c] * (act_of(a.act, acc[q][i]) * acc[q][2 + i]));
        }
#pragma unroll
      for (int q = 0; q < RT; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[q][i] = 0.0f;
    }
  } else if constexpr (kGated) {
    int buf = 0, turn = 0;
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
      const int pass = item / a.tiles, n0 = (item - pass * a.tiles) * kOut;
      if (have.pass < passes && have.item == item)
        while (!block()) {
        }
      const int first = lists.first[pass], n = min(static_cast<int>(lists.first[pass + 1]) - first, kCols);
      float *const rb = red + buf * (kWarps * kRows * P::kRedPitch);
      buf ^= 1;
#pragma unroll
      for (int q = 0; q < RT; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          rb[(warp * kRows + q * 16 + g + (i >> 1) * 8) * P::kRedPitch + 2 * t + (i & 1)] = acc[q][i];
          acc[q][i] = 0.0f;
        }
      __syncthreads();
      // (the other buffer is written next, and this one only behind another barrier)
      const int mine = (tid + 32 * turn++) % kThreads;  // warps in turn
      if (mine < kOut * n) {
        const int r = mine % kOut, c = mine / kOut, pair = lists.order[first + c], row = (r >> 3) * 16 + (r & 7);
        float gate = 0.0f, up = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          gate += rb[(w * kRows + row) * P::kRedPitch + c];
          up += rb[(w * kRows + row + 8) * P::kRedPitch + c];
        }
        reinterpret_cast<T *>(a.y + pair * a.ldy)[n0 + r] = from_f32<T>(lists.weight[first + c] * (act_of(a.act, gate) * up));
      }
    }
  } else {
    const int pitch = a.M | 1, n0 = have.tile * kOut;
    float *const mine = red + warp * kRows * pitch;
    while (have.pass < passes) {
      const int pass = have.pass;
      if (block()) {
        // into the tokens' sums, column by column: a token may have the same expert twice
        const int first = lists.first[pass], n = min(static_cast<int>(lists.first[pass + 1]) - first, kCols);
        for (int c = 0; c < n; ++c) {
          if (t == c >> 1) {
            const int m = lists.order[first + c] / a.topk;
#pragma unroll
            for (int q = 0; q < RT; ++q) {
              mine[(16 * q + g) * pitch + m] += c & 1 ? acc[q][1] : acc[q][0];
              mine[(16 * q + g + 8) * pitch + m] += c & 1 ? acc[q][3] : acc[q][2];
            }
          }
          __syncwarp();
        }
#pragma unroll
        for (int q = 0; q < RT; ++q)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[q][i] = 0.0f;
      }
    }
    __syncthreads();
    float *const sum = red + kWarps * kRows * pitch;
    for (int i = tid; i < kRows * a.M; i += kThreads) {
      const int m = i / kRows, r = i % kRows;
      float v = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) v += red[(w * kRows + r) * pitch + m];
      if (a.splits == 1)
        reinterpret_cast<T *>(a.y + m * a.ldy)[n0 + r] = from_f32<T>(v);
      else
        sum[r * pitch + m] = v;
    }
    if (a.splits > 1) {
      __syncthreads();
      ptx::cluster_sync();
      if (rank == 0)
        for (int i = tid; i < kRows * a.M; i += kThreads) {
          const int m = i / kRows, r = i % kRows;
          float v = 0.0f;
          for (int k = 0; k < a.splits; ++k) {
            float p;
            asm volatile("ld.shared::cluster.f32 %0, [%1];"
                         : "=f"(p)
                         : "r"(ptx::map_to_rank(ptx::smem_addr(sum + r * pitch + m), k))
                         : "memory");
            v += p;
          }
          reinterpret_cast<T *>(a.y + m * a.ldy)[n0 + r] = from_f32<T>(v);
        }
      __syncthreads();
      ptx::cluster_sync();  // no CTA ends while its sums are read
    }
  }
  ptx::cp_async_wait<0>();
}

template <typename T, bool kGated, bool kOwn, bool kZeros, int RT, int CH, int CPG>
cudaError_t launch_as(MoeArgs a, cudaStream_t s) {
  using P = Moe<RT, CH, CPG>;
  a.nblk = (a.K + P::KB - 1) / P::KB;
  a.tiles = a.N / (kGated ? 8 * RT : 16 * RT);
  a.s_vec = a.groups % P::kGroups == 0 && (1 << a.group_shift) * P::kGroups == P::KB;
  constexpr auto kern = moe4_kernel<T, kGated, kOwn, kZeros, RT, CH, CPG>;
  const size_t smem = kOwn ? P::kRing : P::smem(kGated, a.M);
  const cudaError_t e = conv::ensure_smem_attr(reinterpret_cast<const void *>(kern), smem);
  if (e != cudaSuccess) return e;
  const int64_t pairs = static_cast<int64_t>(a.M) * a.topk;
  const int slots = 2 * sm_count();
  a.splits = 1;
  if (kGated) {
    const int64_t most = kOwn ? (pairs * a.tiles + kWarps - 1) / kWarps : pairs * a.tiles;
    return launch_dependent(kern, dim3(static_cast<unsigned>(most < slots ? most : slots)), kThreads, smem, s, 1, a);
  }
  // a tile's blocks over as many CTAs as fill the GPU, while each warp still has a block
  const int64_t blocks = (pairs < a.E ? pairs : a.E) * a.nblk;
  while (a.splits < 8 && static_cast<int64_t>(a.tiles) * a.splits * 2 <= slots && blocks >= 2 * kWarps * a.splits) a.splits *= 2;
  return launch_dependent(kern, dim3(a.tiles * a.splits), kThreads, smem, s, a.splits, a);
}

template <typename T, bool kGated, bool kOwn, bool kZeros, int RT>
cudaError_t launch_grouped(const MoeArgs &a, cudaStream_t s) {
  if (a.group_shift == 5) return launch_as<T, kGated, kOwn, kZeros, RT, 4, 1>(a, s);
  if (a.group_shift == 6) return launch_as<T, kGated, kOwn, kZeros, RT, 4, 2>(a, s);
  return launch_as<T, kGated, kOwn, kZeros, RT, 4, 4>(a, s);
}

// First kernel: tiles of 32 rows are a warp's where there are one and a half times as many as warps or more, or three
// quarters where a CTA's warps would have one block each of a tile; else the CTA's, of 32 rows (inputs are put in order and
// looked up for twice the weights) where they give every SM four, else of 16. us of a layer with a warp's tiles, the CTA's
// of 32 rows, of 16 (tokens, experts of each, K x F; groups of 64): 13, 6 of 64, 2048 x 1408: 80, 88, 107; 32, 4 of 32, 1024
// x 1024: 47, 54, 60; 24, 4 of 64, 512 x 1024: 37, 43, 53; 3, 8 of 64, 7168 x 2048: 169, 172, 209; 8, 4 of 16, 2048 x 2048:
// 44, 44, 53; 4, 2 of 8, 4096 x 4096: 56, 47, 55; 6, 4 of 32, 4096 x 1408: 70, 60, 68; 1, 2 of 8, 4096 x 8192: 47, 46, 51.
// Where the rule is not the best: 16, 2 of 16, 1024 x 2048: 39, 34, 49 (it takes the warp's); 1, 8 of 64, 2048 x 768: 27,
// 20.5, 22.4 and 2, 2 of 16, 4096 x 2048: 41, 30, 34 (it takes those of 16 rows).
// Second: of 32 rows where the warps of twice as many CTAs as fit get a block. A layer with 32 and 16 rows: 80 and 85, 172
// and 179, 47 and 49 us for the first, the fourth and the sixth of these; but 47 and 36 for the second, 37 and 33
// for the third, 39 and 28 for the 16 tokens: many pairs of few columns, for which the rule is wrong.
template <typename T, bool kGated, bool kZeros>
cudaError_t launch_sized(const MoeArgs &a, cudaStream_t s) {
  const int64_t pairs = static_cast<int64_t>(a.M) * a.topk, experts = pairs < a.E ? pairs : a.E;
  if constexpr (kGated) {
    const int64_t tiles = experts * (a.N / 8), warps = 2 * kWarps * sm_count();
    const int64_t per_warp = (a.K + 127) / 128 <= kWarps ? 3 * warps / 2 : 3 * warps;  // tiles of eight rows of each matrix
    if (tiles >= per_warp) return launch_grouped<T, true, true, kZeros, 2>(a, s);
    if (tiles >= 8 * sm_count()) return launch_grouped<T, true, false, kZeros, 2>(a, s);
    return launch_grouped<T, true, false, kZeros, 1>(a, s);
  } else {
    const int64_t work = experts * (a.N / 32) * ((a.K + 127) / 128) / kWarps;
    return work >= 4 * sm_count() ? launch_grouped<T, false, false, kZeros, 2>(a, s)
                                  : launch_grouped<T, false, false, kZeros, 1>(a, s);
  }
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
