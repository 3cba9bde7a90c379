// ffn.cu -- the gated feed-forward block for training: forward with 8-bit
// checkpoints, and the backward pass from them.
//
//   forward   g = x Wg^T, u = x Wu^T, h = act(g) * u
//   backward  dg = dh * u * act'(g), du = dh * act(g)
//             dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x
//
// Four large products (2 M K F multiply-adds forward, 4 M K F backward) on
// tcgen05 with fp32 accumulators, through one persistent kernel in three forms
// (BWD: DX and DW in one launch, where their tiles fill the GPU together):
//   FWD  tile 128 tokens x 128 hidden columns of both projections: the B
//        operand stacks 128 rows of Wg on 128 rows of Wu, so one MMA of N = 256
//        fills g and u side by side in tensor memory, and the epilogue forms
//        act(g) * u and the two 8-bit blocks of a row without leaving the chip.
//   DX   tile 128 tokens x 256 inputs; the reduction runs over the hidden
//        columns of dg and Wg, then of du and Wu, into the same accumulator.
//        Wg and Wu are read as they lie (rows along the MMA's N).
//   DW   tile 128 hidden columns x 256 inputs of either gradient; the reduction
//        runs over the tokens, and both operands are read as they lie (rows
//        along the MMA's M and N). x comes from its 8-bit form, whose values
//        16-bit types hold without rounding.
// Between FWD and the others an elementwise kernel forms dg and du, rounded to
// the operands' type: with fp32 sums this is the one rounding between the
// gradients' factors and their sums.
//
// Measured (one GB300): 4096 x 4096 x 8192 forward 322 us (1.71 PFLOP/s) in a
// short run, 354 to 366 under the power cap; 8192 x 4096 x 8192 bf16 step 2.01 ms
// (1.64 PFLOP/s), 2.24 to 2.29 under it, where the library product of that size
// holds 1.66 PFLOP/s. Large products are bound by power (1.6 GHz of 2.07), small ones by
// start, end and the reduction steps of one CTA (pick_tile). DX and DW in one
// launch: the step of 2048 x 2048 x 4096 167 -> 153 us, of 777 x 1000 x 2736
// 65 -> 57.
#include <mutex>
#include <type_traits>

#include "ffn_internal.cuh"
#include "tc_ptx.cuh"

namespace samd {
namespace {

enum Form { FWD = 0, DX = 1, DW = 2, BWD = 3 };

constexpr int BM = 128, BK = 64;
constexpr int kEpiWarps = 8, kFirstEpiWarp = 4;
constexpr int kThreads = 32 * (kFirstEpiWarp + kEpiWarps);

// A tile's columns BN, and what follows from them: stages of KS reduction steps,
// each 16 KB of A and BN * 128 bytes of B, as many as 192 KB hold. Narrow tiles
// take two steps a stage: their MMAs are over before the barriers and the issue
// of the next ones are.
template <int BN>
struct Tile {
  static constexpr int KS = BN == 256 ? 1 : 2;
  static constexpr int kABytes = BM * BK * 2, kBBytes = BN * BK * 2, kStepBytes = kABytes + kBBytes;
  static constexpr int kStageBytes = KS * kStepBytes;
  static constexpr int kStages = BN == 128 ? 3 : 4;
  static constexpr size_t kSmemBytes = 1024 + static_cast<size_t>(kStages) * kStageBytes + 256;
  static_assert(kSmemBytes <= 227 * 1024 && 2 * BN <= 512, "shared and tensor memory of an SM");
};
constexpr uint64_t kWaitLimitNs = 1000000000ull;  // 1 s
constexpr int kBand = 12;  // tiles along M that follow one another before the next along N

// One product: its tiles, and where its result goes.
struct Job {
  int M, N;         // of an output: rows and columns
  int steps;        // reduction steps of BK in a segment
  int tiles_m, tiles_n;
  int half_m;       // DW: rows of tiles of the first output; the rest are the second's
  int wide;         // rows of the output start on 32 bytes
  int64_t ld;       // of the output
  void *out[2];     // FWD: h; DX: dx; DW: dwg, dwu
};

struct GemmArgs {
  Job job[2];       // BWD: that of DX and that of DW; else the one
  int first, total; // tiles of job[0]; of both
  int fill;         // BWD: DW tiles that last as long as one of DX
  int split;        // CTAs of a cluster that share a tile's reduction (kSplit)
  // FWD: the checkpoints (null: none), rows of `wpr` words and `bpr` exponents
  uint32_t *lanes[2];
  uint8_t *exps[2];
  int64_t wpr, bpr;
  int wide8;        // rows of the checkpoints' lanes start on 32 bytes
  int *status;
};

// The operands' tensor maps: A of the first and the second segment (DX) or
// output (DW), B of the first and the second segment (DX) or projection (FWD);
// BWD: those of DX, then dg, du and x as DW reads them.
struct Maps {
  CUtensorMap m[7];
};

__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, int *status) {
  return __all_sync(0xffffffffu,
                    ptx::mbar_wait(bar, parity, status, static_cast<int>(SAMD_ETIMEOUT), kWaitLimitNs));
}

// BWD: CTA c's tile after `tile`, of P CTAs. The `first` tiles of DX go in turn
// over the CTAs; those that have none in the last, partial turn take `fill`
// rounds of DW's tiles meanwhile (as many as a DX tile lasts); then DW's go in
// turn over all.
__host__ __device__ inline int dealt_next(int tile, int c, int P, int first, int fill) {
  const int rest = first % P, spare = P - rest;
  const int base = first + (rest ? spare * fill : 0);  // the first tile that is dealt to all
  const bool free = rest != 0 && c >= rest;
  if (tile < first) {
    if (tile + P < first) return tile + P;
    return free && fill ? first + (c - rest) : base + c;
  }
  if (tile < base) return tile + spare < base ? tile + spare : base + c;
  return tile + P;
}

// Columns [c, c + 32) of a row of the output, rounded.
template <typename T>
__device__ __forceinline__ void store_row32(T *row, int c, int N, bool wide, const float *v) {
  if (wide && c + 32 <= N) {
    // neighbouring lanes' rows lie apart, and a store takes a cycle for each: few and wide ones
#pragma unroll
    for (int i = 0; i < 2; ++i)
      ptx::st_global_v8(row + c + 16 * i, pack2<T>(v[16 * i], v[16 * i + 1]), pack2<T>(v[16 * i + 2], v[16 * i + 3]),
                        pack2<T>(v[16 * i + 4], v[16 * i + 5]), pack2<T>(v[16 * i + 6], v[16 * i + 7]),
                        pack2<T>(v[16 * i + 8], v[16 * i + 9]), pack2<T>(v[16 * i + 10], v[16 * i + 11]),
                        pack2<T>(v[16 * i + 12], v[16 * i + 13]), pack2<T>(v[16 * i + 14], v[16 * i + 15]));
  } else if (c + 32 <= N) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<uint4 *>(row + c + 8 * i) =
          make_uint4(pack2<T>(v[8 * i], v[8 * i + 1]), pack2<T>(v[8 * i + 2], v[8 * i + 3]),
                     pack2<T>(v[8 * i + 4], v[8 * i + 5]), pack2<T>(v[8 * i + 6], v[8 * i + 7]));
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (c + i < N) row[c + i] = from_f32<T>(v[i]);
  }
}

// The block [c, c + 32) of a row into its 8-bit form. Columns past N are zero.
// kKeep: the code of a positive value is at least 1 (a ReLU's argument: rounded
// to zero it would lose its derivative, which one in a hundred does on normal
// data, a tenth of the gradient's norm).
template <bool kKeep>
__device__ __forceinline__ void store_block8(uint32_t *lanes, uint8_t *exps, int64_t wpr, int c, bool wide, const float *v) {
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < 32; ++i) top = max_abs(top, v[i]);
  const uint32_t e = block8_exp(top);
  uint32_t w[8];
  block8_words_of<kKeep, 32>(v, top, e, block8_inv(e), w);
  uint32_t *const out = lanes + c / 4;
  if (wide && c / 4 + 8 <= wpr) {
    ptx::st_global_v8(out, w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]);
  } else if (wpr % 4 == 0 && c / 4 + 8 <= wpr) {
    *reinterpret_cast<uint4 *>(out) = make_uint4(w[0], w[1], w[2], w[3]);
    *reinterpret_cast<uint4 *>(out + 4) = make_uint4(w[4], w[5], w[6], w[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c / 4 + i < wpr) out[i] = w[i];
  }
  exps[c / kBlock8] = static_cast<uint8_t>(e);
}

// Columns [c, c + 4) of a row of the output, rounded (rows start on 16 bytes, c is a multiple of 4).
template <typename T>
__device__ __forceinline__ void store_row4(T *row, int c, int N, const float *v) {
  if (c + 4 <= N) {
    *reinterpret_cast<uint2 *>(row + c) = make_uint2(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i < N) row[c + i] = from_f32<T>(v[i]);
  }
}

// Four columns from c on of a block that eight neighbouring lanes hold, into
// its 8-bit form (`in`: the lane's columns are of the output; the same for all
// eight; columns past N are zero). Called by the whole warp.
template <bool kKeep>
__device__ __forceinline__ void split_block8(uint32_t *lanes, uint8_t *exps, int64_t wpr, int c, bool in, const float *v) {
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max_abs(top, v[i]);
#pragma unroll
  for (int s = 1; s < 8; s *= 2) top = max_abs(top, __shfl_xor_sync(0xffffffffu, top, s));
  const uint32_t e = block8_exp(top);
  uint32_t w;
  block8_words_of<kKeep, 4>(v, top, e, block8_inv(e), &w);
  if (in && c / 4 < wpr) {
    lanes[c / 4] = w;
    if (c % kBlock8 == 0) exps[c / kBlock8] = static_cast<uint8_t>(e);
  }
}

// One CTA per SM, looping over tiles; twelve warps: 0 loads operand tiles with
// TMA, 1 issues the MMAs, 2 holds the tensor memory, 4-11 drain one of two
// accumulators while the other fills. Every wait is bounded: a role that gives
// up records it and stops, the others' waits then give up within one poll.
//
// kSplit: few tiles with long reductions. A cluster takes one tile, each of its
// CTAs a part of the reduction; the partial sums meet in distributed shared
// memory, where each CTA adds up (in rank order) and finishes a part of the
// rows.
template <int FORM, typename T, int ACT, int BN, bool kSplit>
__global__ void __launch_bounds__(kThreads, 1)
    ffn_gemm_kernel(const __grid_constant__ Maps maps, const __grid_constant__ GemmArgs a) {
  static_assert(FORM != BWD || !kSplit, "a split takes one product");
  constexpr int kSumPitch = BN * 4 + 16;  // bytes of a row of partial sums (kSplit)
  constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
  constexpr int kStages = Tile<BN>::kStages, kABytes = Tile<BN>::kABytes, kBBytes = Tile<BN>::kBBytes,
                kStepBytes = Tile<BN>::kStepBytes, kStageBytes = Tile<BN>::kStageBytes, KS = Tile<BN>::KS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *const smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t *const bars = reinterpret_cast<uint64_t *>(smem + kStages * kStageBytes);
  const uint32_t full0 = ptx::smem_addr(bars), empty0 = full0 + 8 * kStages, accfull0 = empty0 + 8 * kStages,
                 accempty0 = accfull0 + 16, drain = accempty0 + 16;
  uint32_t *const holder = reinterpret_cast<uint32_t *>(bars + 2 * kStages + 5);
  const uint32_t sbase = ptx::smem_addr(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (warp == 2) {
    ptx::tmem_alloc(ptx::smem_addr(holder), 2 * BN);
    ptx::tmem_relinquish();
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      ptx::mbar_init(full0 + 8 * s, 1);
      ptx::mbar_init(empty0 + 8 * s, 1);
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(accfull0 + 8 * i, 1);
      ptx::mbar_init(accempty0 + 8 * i, kEpiWarps);
    }
    ptx::mbar_init(drain, 1);
    ptx::fence_barrier_init();
  }
  __syncwarp();
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *holder;
  // (every role, before it reads or writes global memory)
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();
  // a CTA's tiles and its steps of their reductions
  const int rank = kSplit ? blockIdx.x % a.split : 0;
  const int tile0 = kSplit ? blockIdx.x / a.split : blockIdx.x, tile_step = kSplit ? a.total : gridDim.x;
  // The CTA's next tile.
  auto next_tile = [&](int tile) {
    if constexpr (FORM != BWD)
      return tile + tile_step;
    else
      return dealt_next(tile, blockIdx.x, gridDim.x, a.first, a.fill);
  };
  const int tile_1 = FORM == BWD && tile0 >= a.first ? next_tile(tile0 - static_cast<int>(gridDim.x)) : tile0;
  // calls f with a tile's form, its job and its number there
  auto on_tile = [&](int tile, auto f) {
    if constexpr (FORM == BWD) {
      if (tile < a.first)
        f(std::integral_constant<int, DX>(), a.job[0], tile);
      else
        f(std::integral_constant<int, DW>(), a.job[1], tile - a.first);
    } else {
      f(std::integral_constant<int, FORM>(), a.job[0], tile);
    }
  };
  // a CTA's reduction steps [k0, k1) of a job
  auto k_begin = [&](int all) { return kSplit ? static_cast<int>(static_cast<int64_t>(all) * rank / a.split) : 0; };
  auto k_end = [&](int all) { return kSplit ? static_cast<int>(static_cast<int64_t>(all) * (rank + 1) / a.split) : all; };

  // tile -> its row and column of tiles: bands of kBand rows, down a band's
  // column before the next, so that the tiles in flight share operands in L2
  auto place = [](const Job &job, int tile, int &tm, int &tn) {
    const int band = tile / (kBand * job.tiles_n);
    const int first = band * kBand;
    const int rows = min(kBand, job.tiles_m - first);
    const int r = tile - band * kBand * job.tiles_n;
    tn = r / rows;
    tm = first + (r - tn * rows);
  };

  if (warp == 0) {
    const uint32_t leader = ptx::elect_one() ? 1u : 0u;
    int s = 0, loaded = 0;
    uint32_t par = 1;
    bool ok = true;
    for (int tile = tile_1; ok && tile < a.total; tile = next_tile(tile))
      on_tile(tile, [&](auto form, const Job &job, int at) {
        constexpr int F = decltype(form)::value, kMap = FORM == BWD && F == DW ? 4 : 0;
        int tm, tn;
        place(job, at, tm, tn);
        const int second = F == DW && tm >= job.half_m;
        const int m0 = (second ? tm - job.half_m : tm) * BM, n0 = tn * (F == FWD ? BN / 2 : BN);
        const int all = job.steps * (F == DX ? 2 : 1), k1 = k_end(all);
        for (int k = k_begin(all); k < k1; k += KS) {
          // A stage is armed again when the MMAs that read it have completed,
          // and they were issued behind a wait for its copies.
          if (loaded == kStages) {
            ok = warp_wait(empty0 + 8 * s, par, a.status);
            if (!ok) break;
          } else {
            ++loaded;
          }
          const int now = KS == 1 ? 1 : min(KS, k1 - k);  // steps of this stage
          const uint32_t full = full0 + 8 * s;
          ptx::mbar_arrive_expect_tx_if(leader, full, now * kStepBytes);
#pragma unroll
          for (int j = 0; j < KS; ++j) {
            if (j < now) {
              const uint32_t sa = sbase + s * kStageBytes + j * kStepBytes, sb = sa + kABytes;
              const bool seg = F == DX && k + j >= job.steps;
              const int kk = (seg ? k + j - job.steps : k + j) * BK;
              const CUtensorMap *const A = &maps.m[kMap + ((F == DX && seg) || second ? 1 : 0)];
              if constexpr (F == DW) {
                ptx::tma_load_2d_if(leader, sa, A, m0, kk, full);
                ptx::tma_load_2d_if(leader, sa + kABytes / 2, A, m0 + 64, kk, full);
              } else {
                ptx::tma_load_2d_if(leader, sa, A, kk, m0, full);
              }
              if constexpr (F == FWD) {
                ptx::tma_load_2d_if(leader, sb, &maps.m[2], kk, n0, full);
                ptx::tma_load_2d_if(leader, sb + kBBytes / 2, &maps.m[3], kk, n0, full);
              } else {
                const CUtensorMap *const B = &maps.m[kMap + 2 + (seg ? 1 : 0)];
#pragma unroll
                for (int q = 0; q < BN / 64; ++q)
                  ptx::tma_load_2d_if(leader, sb + q * (64 * BK * 2), B, n0 + 64 * q, kk, full);
              }
            }
          }
          if (++s == kStages) {
            s = 0;
            par ^= 1;
          }
        }
      });
    // the CTA does not exit with a copy in flight: the ring's last round,
    // oldest first
    int quiet = 0;
    for (int k = 0; k < loaded; ++k) {
      int q = loaded == kStages ? s + k : k;
      if (q >= kStages) q -= kStages;
      ptx::mbar_wait_bounded(full0 + 8 * q, q < s ? par ^ 1u : par, &quiet, kWaitLimitNs / 10);
    }
  } else if (warp == 1) {
    const uint32_t leader = ptx::elect_one() ? 1u : 0u;
    int s = 0, i = 0;
    uint32_t par = 0;
    bool ok = true;
    for (int tile = tile_1; ok && tile < a.total; tile = next_tile(tile), ++i)
      on_tile(tile, [&](auto form, const Job &job, int) {
        constexpr int F = decltype(form)::value;
        constexpr bool kAMn = F == DW, kBMn = F != FWD;
        constexpr uint32_t idesc = ptx::idesc_16_f32(kBf16, kAMn, kBMn, BM, BN);
        // 16 reduction positions further: 32 bytes along a row, or 16 rows down
        constexpr uint64_t kAStep = kAMn ? 2048 >> 4 : 32 >> 4, kBStep = kBMn ? 2048 >> 4 : 32 >> 4;
        const int acc = i & 1;
        if (i >= 2) ok = warp_wait(accempty0 + 8 * acc, ((i >> 1) + 1) & 1u, a.status);
        if (!ok) return;
        ptx::tc_fence_after();
        const uint32_t d = tmem + acc * BN;
        const int all = job.steps * (F == DX ? 2 : 1), k0 = k_begin(all), k1 = k_end(all);
        for (int k = k0; k < k1; k += KS) {
          ok = warp_wait(full0 + 8 * s, par, a.status);
          if (!ok) break;
          ptx::tc_fence_after();
#pragma unroll
          for (int q = 0; q < KS; ++q) {
            if (KS == 1 || k + q < k1) {
              const uint32_t sa = sbase + s * kStageBytes + q * kStepBytes, sb = sa + kABytes;
              const uint64_t da = kAMn ? ptx::sw128_mnmajor_desc(sa, kABytes / 2) : ptx::sw128_kmajor_desc(sa);
              const uint64_t db = kBMn ? ptx::sw128_mnmajor_desc(sb, 64 * BK * 2) : ptx::sw128_kmajor_desc(sb);
#pragma unroll
              for (int j = 0; j < BK / 16; ++j)
                ptx::mma_f16(leader, d, da + j * kAStep, db + j * kBStep, idesc, k > k0 || q > 0 || j > 0);
            }
          }
          ptx::mma_commit(leader, empty0 + 8 * s);
          if (++s == kStages) {
            s = 0;
            par ^= 1;
          }
        }
        if (ok) ptx::mma_commit(leader, accfull0 + 8 * acc);
      });
    // nothing of this CTA's reads shared memory or writes tensor memory after
    // this: every MMA issued has completed
    ptx::mma_commit(leader, drain);
    int quiet = 0;
    ptx::mbar_wait_bounded(drain, 0, &quiet, kWaitLimitNs / 10);
  } else if (warp >= kFirstEpiWarp) {
    const int ew = warp - kFirstEpiWarp;
    const int quad = warp & 3, half = ew >> 2;  // rows 32 * quad .., alternate blocks of 32 columns
    int i = 0;
    for (int tile = tile_1; tile < a.total; tile = next_tile(tile), ++i) {
      const int acc = i & 1;
      if (!warp_wait(accfull0 + 8 * acc, (i >> 1) & 1u, a.status)) break;
      ptx::tc_fence_after();
      // (DX and DW end alike; a DX has one output)
      const bool other = FORM == BWD && tile >= a.first;
      const Job &job = other ? a.job[1] : a.job[0];
      int tm, tn;
      place(job, other ? tile - a.first : tile, tm, tn);
      const int second = tm >= job.half_m;
      const int m = (second ? tm - job.half_m : tm) * BM + quad * 32 + lane;
      const uint32_t t0 = tmem + acc * BN + (static_cast<uint32_t>(quad * 32) << 16);
      if constexpr (kSplit) {
        // this CTA's partial sums, rows a multiple of 16 bytes and four banks apart; the stages are free: every
        // copy has landed and every MMA that read one has completed
#pragma unroll 1
        for (int b = half; b < BN / 32; b += 2) {
          uint32_t r[32];
          __syncwarp();
          ptx::tmem_ld_32x32b_x32(t0 + b * 32, r);
          ptx::tmem_wait_ld(r);
          uint4 *const row = reinterpret_cast<uint4 *>(smem + (quad * 32 + lane) * kSumPitch + b * 128);
#pragma unroll
          for (int q = 0; q < 8; ++q) row[q] = make_uint4(r[4 * q], r[4 * q + 1], r[4 * q + 2], r[4 * q + 3]);
        }
      } else if constexpr (FORM == FWD) {
        const int n0 = tn * (BN / 2);
#pragma unroll 1
        for (int b = half; b < BN / 64; b += 2) {
          uint32_t rg[32], ru[32];
          __syncwarp();
          ptx::tmem_ld_32x32b_x32(t0 + b * 32, rg);
          ptx::tmem_ld_32x32b_x32(t0 + BN / 2 + b * 32, ru);
          ptx::tmem_wait_ld(rg);
          ptx::tmem_wait_ld(ru);
          const float *const gv = reinterpret_cast<const float *>(rg), *const uv = reinterpret_cast<const float *>(ru);
          const int c = n0 + b * 32;
          if (m < job.M && c < job.N) {
            float h[32];
#pragma unroll
            for (int q = 0; q < 32; ++q) h[q] = act_value<ACT>(gv[q]) * uv[q];
            store_row32<T>(static_cast<T *>(job.out[0]) + m * job.ld, c, job.N, job.wide, h);
            if (a.lanes[0]) {
              store_block8<ACT == SAMD_RELU_ACT>(a.lanes[0] + m * a.wpr, a.exps[0] + m * a.bpr, a.wpr, c, a.wide8, gv);
              store_block8<false>(a.lanes[1] + m * a.wpr, a.exps[1] + m * a.bpr, a.wpr, c, a.wide8, uv);
            }
          }
        }
      } else {
        const int n0 = tn * BN;
        T *const out = static_cast<T *>(second ? job.out[1] : job.out[0]) + m * job.ld;
#pragma unroll 1
        for (int b = half; b < BN / 32; b += 2) {
          uint32_t r[32];
          __syncwarp();
          ptx::tmem_ld_32x32b_x32(t0 + b * 32, r);
          ptx::tmem_wait_ld(r);
          const int c = n0 + b * 32;
          if (m < job.M && c < job.N) store_row32<T>(out, c, job.N, job.wide, reinterpret_cast<const float *>(r));
        }
      }
      __syncwarp();
      ptx::tc_fence_before();
      if (lane == 0) ptx::mbar_arrive(accempty0 + 8 * acc);
    }
  }

  if constexpr (kSplit) {
    __syncwarp();
    ptx::cluster_sync();
    const Job &job = a.job[0];
    int tm, tn;
    place(job, tile0, tm, tn);
    const int second = tm >= job.half_m;
    const int m0 = (second ? tm - job.half_m : tm) * BM;
    const int rows = min(BM, job.M - m0), per = (rows + a.split - 1) / a.split;
    const int r0 = rank * per, count = max(0, min(per, rows - r0));
    // a thread takes four columns of a row (FWD: of both projections, eight neighbouring lanes a block of 32)
    constexpr int kPerRow = (FORM == FWD ? BN / 2 : BN) / 4;
    for (int i0 = warp * 32; i0 < count * kPerRow; i0 += kThreads) {
      const int i = i0 + lane, row = r0 + i / kPerRow, c = i % kPerRow * 4;
      const bool in = i < count * kPerRow;
      float g[4] = {0.0f, 0.0f, 0.0f, 0.0f}, u[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      if (in) {
        const uint32_t at = sbase + row * kSumPitch + c * 4;
        for (int r = 0; r < a.split; ++r) {
          const uint32_t from = ptx::map_to_rank(at, r);
          const float4 v = ptx::ld_cluster_v4(from);
          g[0] += v.x, g[1] += v.y, g[2] += v.z, g[3] += v.w;
          if constexpr (FORM == FWD) {
            const float4 w = ptx::ld_cluster_v4(from + BN * 2);
            u[0] += w.x, u[1] += w.y, u[2] += w.z, u[3] += w.w;
          }
        }
      }
      const int col = tn * (kPerRow * 4) + c;
      const int64_t m = m0 + row;
      if constexpr (FORM == FWD) {
        float h[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) h[q] = act_value<ACT>(g[q]) * u[q];
        if (in) store_row4<T>(static_cast<T *>(job.out[0]) + m * job.ld, col, job.N, h);
        if (a.lanes[0]) {
          split_block8<ACT == SAMD_RELU_ACT>(a.lanes[0] + m * a.wpr, a.exps[0] + m * a.bpr, a.wpr, col, in, g);
          split_block8<false>(a.lanes[1] + m * a.wpr, a.exps[1] + m * a.bpr, a.wpr, col, in, u);
        }
      } else if (in) {
        store_row4<T>(static_cast<T *>(second ? job.out[1] : job.out[0]) + m * job.ld, col, job.N, g);
      }
    }
    __syncwarp();
    ptx::cluster_sync();  // no CTA's shared memory goes while another reads it
  }

  __syncwarp();
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 2) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, 2 * BN);
  }
}

// The elementwise part of the backward pass, sixteen columns a thread:
//   dg = dh * u * act'(g) and du = dh * act(g) from the 8-bit forms of g and u,
//   rounded to T; h = act(g) * u again if wanted; and x from its 8-bit form
//   (where the weights' gradients are wanted), which T holds without rounding.
// One pass over HBM: 4 1/16 bytes an element of dh in and 4 or 6 out, 1 1/32 in
// and 2 out for x. dg, du and xb are rows of whole units of eight; past F and K
// their columns are not read. 8192 x 8192 with x of 4096: 642 MB in 111 us, 0.87
// of the copy bandwidth.
struct DgateArgs {
  const void *dh;
  void *dg, *du, *h, *xb;  // h, xb: null if not wanted
  samd_block8 cg, cu, cx;
  int64_t ldh, ldf, ldk, M, items_f, items;  // items: threads' pieces, those of dh first
  int F, K, segs_f, segs_k;                  // pieces of a row
  IndexDiv by_f, by_k;
};

__device__ __forceinline__ void load_words4(const void *lanes, int64_t at, bool vec, int n, uint32_t *w) {
  const uint32_t *const p = static_cast<const uint32_t *>(lanes) + at;
  if (vec && n > 12) {
    const uint4 q = __ldcs(reinterpret_cast<const uint4 *>(p));
    w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = 4 * i < n ? p[i] : 0u;
  }
}

template <typename T>
__device__ __forceinline__ uint4 pack8(const float *v) {
  return make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
}

template <typename T, int ACT>
__global__ void __launch_bounds__(256) ffn_dgate_kernel(const DgateArgs a) {
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();
  const int64_t nthreads = static_cast<int64_t>(gridDim.x) * blockDim.x;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < a.items; i += nthreads) {
    if (i < a.items_f) {
      const int64_t m = idiv(i, a.by_f);
      const int c = static_cast<int>(i - m * a.segs_f) * 16;
      const int n = a.F - c < 16 ? a.F - c : 16;
      const int64_t wpr = (a.F + 3) / 4, bpr = (a.F + kBlock8 - 1) / kBlock8;
      uint32_t gw[4], uw[4];
      load_words4(a.cg.lanes, m * wpr + c / 4, wpr % 4 == 0, n, gw);
      load_words4(a.cu.lanes, m * wpr + c / 4, wpr % 4 == 0, n, uw);
      const float gs = block8_scale(a.cg.exps[m * bpr + c / kBlock8]), us = block8_scale(a.cu.exps[m * bpr + c / kBlock8]);
      const T *const dh = static_cast<const T *>(a.dh) + m * a.ldh + c;
      uint32_t dw[8];
      if (n == 16) {
        const uint4 p = __ldcs(reinterpret_cast<const uint4 *>(dh)), q = __ldcs(reinterpret_cast<const uint4 *>(dh) + 1);
        dw[0] = p.x, dw[1] = p.y, dw[2] = p.z, dw[3] = p.w, dw[4] = q.x, dw[5] = q.y, dw[6] = q.z, dw[7] = q.w;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint16_t *const p = reinterpret_cast<const uint16_t *>(dh) + 2 * j;
          dw[j] = (2 * j < n ? p[0] : 0u) | (2 * j + 1 < n ? static_cast<uint32_t>(p[1]) << 16 : 0u);
        }
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (half * 8 >= n) break;
        float g[8], u[8], vg[8], vu[8];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          block8_values(gw[2 * half + j], gs, g + 4 * j);
          block8_values(uw[2 * half + j], us, u + 4 * j);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 d2 = unpack2<T>(dw[4 * half + j / 2]);
          const float d = j & 1 ? d2.y : d2.x;
          float da;
          const float av = act_value_grad<ACT>(g[j], da);
          vg[j] = d * u[j] * da;
          vu[j] = d * av;
          g[j] = av * u[j];
        }
        const int64_t at = m * a.ldf + c + 8 * half;
        *reinterpret_cast<uint4 *>(static_cast<T *>(a.dg) + at) = pack8<T>(vg);
        *reinterpret_cast<uint4 *>(static_cast<T *>(a.du) + at) = pack8<T>(vu);
        if (a.h) {
          T *const h = static_cast<T *>(a.h) + m * a.ldh + c + 8 * half;
          if (n - 8 * half >= 8) {
            *reinterpret_cast<uint4 *>(h) = pack8<T>(g);
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (8 * half + j < n) h[j] = from_f32<T>(g[j]);
          }
        }
      }
    } else {
      const int64_t k = i - a.items_f, m = idiv(k, a.by_k);
      const int c = static_cast<int>(k - m * a.segs_k) * 16;
      const int n = a.K - c < 16 ? a.K - c : 16;
      const int64_t wpr = (a.K + 3) / 4, bpr = (a.K + kBlock8 - 1) / kBlock8;
      uint32_t w[4];
      load_words4(a.cx.lanes, m * wpr + c / 4, wpr % 4 == 0, n, w);
      const float s = block8_scale(a.cx.exps[m * bpr + c / kBlock8]);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (half * 8 >= n) break;
        float v[8];
        block8_values(w[2 * half], s, v);
        block8_values(w[2 * half + 1], s, v + 4);
        *reinterpret_cast<uint4 *>(static_cast<T *>(a.xb) + m * a.ldk + c + 8 * half) = pack8<T>(v);
      }
    }
  }
}

// ---- host side -------------------------------------------------------------------

int64_t round_up64(int64_t v) { return (v + 63) / 64 * 64; }
size_t round_up256(size_t v) { return (v + 255) / 256 * 256; }

// A tensor of `rows` rows of `cols` 16-bit elements, read in boxes of 64
// columns by box_rows rows with the 128-byte swizzle.
bool make_map(CUtensorMap *map, samd_dtype t, const void *p, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  const EncodeTiledFn enc = tensor_map_encoder();
  if (!enc) return false;
  const cuuint64_t dim[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
  const cuuint64_t stride[1] = {static_cast<cuuint64_t>(ld) * 2};
  const cuuint32_t box[2] = {64, static_cast<cuuint32_t>(box_rows)}, es[2] = {1, 1};
  return enc(map, t == SAMD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
             const_cast<void *>(p), dim, stride, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The tile of a product: its columns, how many CTAs of a cluster share its
// reduction, and the estimated time in ns.
struct Pick {
  int columns, split;
  int64_t cost;
};
// Times measured on one GB300: a reduction step of a tile of 256, 128 or 64
// columns takes 330, 215 or 150 ns (the operands' way into the SM bounds the
// narrow ones); start and end of a launch 1500 and five a column of the last
// tile (FWD: 6000, its epilogue hides less). A tile whose reduction is split
// over a cluster: steps of 64 columns, 3300 for start and meeting (FWD: 6000),
// and 2000 more for every further wave of clusters. For 16 tokens by 1024 by
// 4096, dx: 23.3 us unsplit, 8.6 over four CTAs.
int64_t step_ns(int columns) { return columns == 256 ? 330 : columns == 128 ? 215 : 150; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <typename Clusters>
Pick pick_tile(int form, int64_t rows, int64_t cols, int64_t steps, Clusters clusters) {
  Pick best = {256, 1, INT64_MAX};
  auto offer = [&](int columns, int split, int64_t cost) {
    if (cost < best.cost) best = Pick{columns, split, cost};
  };
  for (const int bn : {256, 128, 64})
    offer(bn, 1, ceil_div(rows * ceil_div(cols, bn), sm_count()) * steps * step_ns(bn) +
                     (form == FWD ? 6000 : 1500 + 5 * bn));
  const int64_t tiles = rows * ceil_div(cols, 64);
  for (const int split : {2, 4, 8}) {
    if (split > steps || 2 * tiles > sm_count()) break;
    const int64_t fit = clusters(split);
    if (fit < 1) break;
    offer(64, split, ceil_div(tiles, fit) * (ceil_div(steps, split) * step_ns(64) + 2000) + (form == FWD ? 4000 : 1300));
  }
  return best;
}

// DW's tiles that a CTA does in the time of one of DX's.
int fill_of(int64_t steps_x, int64_t steps_w) { return static_cast<int>((2 * steps_x + steps_w) / (2 * steps_w)); }

// The rounds of DW's tiles that a joint launch's spare CTAs are dealt: as many
// as they have time for, and no more than there are (a dx of 2^24 reduction
// steps beside weight gradients of one would count tiles past an int).
int deal_fill(int first, int total, int fill) {
  const int P = total < sm_count() ? total : sm_count(), spare = P - first % P;
  const int most = (total - first + spare - 1) / spare;
  return fill < most ? fill : most;
}

// DX and DW in one launch: its columns, and the time.
Pick pick_both(int64_t rows_x, int64_t steps_x, int64_t rows_w, int64_t steps_w, int64_t cols) {
  Pick best = {256, 1, INT64_MAX};
  const int64_t P = sm_count();
  for (const int bn : {256, 128, 64}) {
    const int64_t x = rows_x * ceil_div(cols, bn), w = rows_w * ceil_div(cols, bn), rest = x % P;
    if (x + w < P) continue;  // the GPU is not full: a launch each
    const int64_t early = rest ? (P - rest) * fill_of(steps_x, steps_w) : 0;
    const int64_t steps = ceil_div(x, P) * steps_x + (w > early ? ceil_div(w - early, P) * steps_w : 0);
    const int64_t cost = steps * step_ns(bn) + 1500 + 5 * bn;
    if (cost < best.cost) best = Pick{bn, 1, cost};
  }
  return best;
}

// Clusters of `split` CTAs of the kernel that the current device holds at once
// (0: none, or the query failed); asked once for each device and size.
template <auto Kern>
int resident_clusters(int split, size_t smem) {
  constexpr int kDevices = 64;
  static std::mutex mu;
  static int known[kDevices][9];  // 0: not asked yet, -1: none fit
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) return 0;
  std::lock_guard<std::mutex> lock(mu);
  int &held = known[dev][split];
  if (held == 0) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = split;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(split * sm_count());
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, Kern, &cfg) != cudaSuccess) {
      (void)cudaGetLastError();  // the query's own error; the launch reports any other
      return 0;                  // (asked again by the next call)
    }
    held = n > 0 ? n : -1;
  }
  return held > 0 ? held : 0;
}

// The operands of a product before its tile is picked.
struct Operand {
  const void *p;
  int64_t rows, cols, ld;
};

// Maps at .. at + n - 1 from a product's operands, the first two those of A.
bool make_maps(Maps &maps, int at, int form, int columns, const Operand *op, int n, samd_dtype t) {
  const int a_rows = form == DW ? BK : BM, b_rows = form == FWD ? columns / 2 : BK;  // of a TMA box
  for (int i = 0; i < n; ++i)
    if (!make_map(&maps.m[at + i], t, op[i].p, op[i].rows, op[i].cols, op[i].ld, i < 2 ? a_rows : b_rows)) return false;
  return true;
}

// A job's tiles for a tile width; the number of them.
int set_tiles(Job &job, int form, int columns, bool two) {
  auto on32 = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 31u) == 0; };
  const int cols = form == FWD ? columns / 2 : columns;
  job.half_m = (job.M + BM - 1) / BM;
  job.tiles_m = two ? 2 * job.half_m : job.half_m;
  job.tiles_n = (job.N + cols - 1) / cols;
  job.wide = job.ld % 16 == 0 && on32(job.out[0]) && on32(job.out[1]);
  return job.tiles_m * job.tiles_n;
}

template <int FORM, typename T, int ACT, int BN, bool kSplit = false>
cudaError_t launch_tiled(const Maps &maps, GemmArgs &a, cudaStream_t s) {
  constexpr auto kern = ffn_gemm_kernel<FORM, T, ACT, BN, kSplit>;
  cudaError_t e = device_status_ptr(&a.status);
  if (e == cudaSuccess) e = conv::ensure_smem_attr(reinterpret_cast<const void *>(kern), Tile<BN>::kSmemBytes);
  if (e != cudaSuccess) return e;
  const int grid = kSplit ? a.total * a.split : a.total < sm_count() ? a.total : sm_count();
  return launch_dependent(kern, dim3(grid), kThreads, Tile<BN>::kSmemBytes, s, kSplit ? a.split : 1, maps, a);
}

template <int FORM, typename T, int ACT>
cudaError_t launch_columns(int columns, const Maps &maps, GemmArgs &a, cudaStream_t s) {
  if (columns == 64) return launch_tiled<FORM, T, ACT, 64>(maps, a, s);
  return columns == 128 ? launch_tiled<FORM, T, ACT, 128>(maps, a, s) : launch_tiled<FORM, T, ACT, 256>(maps, a, s);
}

int64_t all_steps(int form, const Job &job) { return static_cast<int64_t>(job.steps) * (form == DX ? 2 : 1); }

template <int FORM, typename T, int ACT>
Pick pick_for(const Job &job, bool two) {
  const int64_t rows = static_cast<int64_t>(job.M + BM - 1) / BM * (two ? 2 : 1);
  const int64_t cols = FORM == FWD ? 2 * static_cast<int64_t>(job.N) : job.N;  // of the MMA
  return pick_tile(FORM, rows, cols, all_steps(FORM, job), [](int split) {
    constexpr auto kern = ffn_gemm_kernel<FORM, T, ACT, 64, true>;
    const size_t smem = Tile<64>::kSmemBytes;
    return conv::ensure_smem_attr(reinterpret_cast<const void *>(kern), smem) == cudaSuccess
               ? resident_clusters<kern>(split, smem)
               : 0;
  });
}

// One product, whose job is a.job[0] (two: a DW with both outputs).
template <int FORM, typename T, int ACT>
cudaError_t launch_gemm(const Pick &p, const Operand (&op)[4], samd_dtype t, bool two, GemmArgs &a, cudaStream_t s) {
  Maps maps = {};
  if (!make_maps(maps, 0, FORM, p.columns, op, 4, t)) return cudaErrorInvalidValue;
  a.first = a.total = set_tiles(a.job[0], FORM, p.columns, two);
  a.split = p.split;
  return p.split > 1 ? launch_tiled<FORM, T, ACT, 64, true>(maps, a, s)
                     : launch_columns<FORM, T, ACT>(p.columns, maps, a, s);
}

template <typename F>
cudaError_t by_act(int act, F f) {
  switch (act) {
    case SAMD_SILU: return f(std::integral_constant<int, SAMD_SILU>());
    case SAMD_GELU: return f(std::integral_constant<int, SAMD_GELU>());
    case SAMD_GELU_TANH: return f(std::integral_constant<int, SAMD_GELU_TANH>());
    default: return f(std::integral_constant<int, SAMD_RELU_ACT>());
  }
}

template <typename T>
cudaError_t forward(const samd_ffn_desc &d, const void *x, const void *wg, const void *wu, void *h, samd_block8 cg,
                    samd_block8 cu, cudaStream_t s) {
  const Operand op[4] = {
      {x, d.M, d.K, d.ldx}, {x, d.M, d.K, d.ldx}, {wg, d.F, d.K, d.ldw}, {wu, d.F, d.K, d.ldw}};
  GemmArgs a = {};
  Job &job = a.job[0];
  job.M = d.M;
  job.N = d.F;
  job.steps = (d.K + BK - 1) / BK;
  job.ld = d.ldh;
  job.out[0] = h;
  a.lanes[0] = static_cast<uint32_t *>(cg.lanes);
  a.lanes[1] = static_cast<uint32_t *>(cu.lanes);
  a.exps[0] = cg.exps;
  a.exps[1] = cu.exps;
  a.wpr = block8_words(d.F);
  a.bpr = block8_blocks(d.F);
  a.wide8 = a.wpr % 8 == 0 && (reinterpret_cast<uintptr_t>(cg.lanes) & 31u) == 0 &&
            (reinterpret_cast<uintptr_t>(cu.lanes) & 31u) == 0;
  return by_act(d.act, [&](auto act) {
    constexpr int kAct = decltype(act)::value;
    return launch_gemm<FWD, T, kAct>(pick_for<FWD, T, kAct>(job, false), op, d.type, false, a, s);
  });
}

// The workspace: dg and du (M rows of F) and x (M rows of K), each row a
// multiple of 64 elements (whole 128-byte lines, what a row of a TMA box is).
struct Workspace {
  size_t dg, du, x, bytes;
  int64_t ldf, ldk;
};
Workspace plan_workspace(const samd_ffn_desc &d) {
  Workspace w;
  w.ldf = round_up64(d.F);
  w.ldk = round_up64(d.K);
  const size_t f = round_up256(static_cast<size_t>(d.M) * w.ldf * 2), k = round_up256(static_cast<size_t>(d.M) * w.ldk * 2);
  w.dg = 0;
  w.du = f;
  w.x = 2 * f;
  w.bytes = 2 * f + k;
  return w;
}

template <typename T>
cudaError_t backward(const samd_ffn_desc &d, const void *dh, samd_block8 cx, samd_block8 cg, samd_block8 cu,
                     const void *wg, const void *wu, void *dx, void *dwg, void *dwu, void *h, void *workspace,
                     cudaStream_t s) {
  const Workspace w = plan_workspace(d);
  uint8_t *const ws = static_cast<uint8_t *>(workspace);
  T *const dg = reinterpret_cast<T *>(ws + w.dg), *const du = reinterpret_cast<T *>(ws + w.du);
  T *const xb = reinterpret_cast<T *>(ws + w.x);
  const bool weights = dwg || dwu;
  DgateArgs g = {};
  g.dh = dh;
  g.dg = dg;
  g.du = du;
  g.h = h;
  g.xb = weights ? xb : nullptr;
  g.cg = cg;
  g.cu = cu;
  g.cx = cx;
  g.ldh = d.ldh;
  g.ldf = w.ldf;
  g.ldk = w.ldk;
  g.M = d.M;
  g.F = d.F;
  g.K = d.K;
  g.segs_f = (d.F + 15) / 16;
  g.segs_k = (d.K + 15) / 16;
  g.items_f = static_cast<int64_t>(d.M) * g.segs_f;
  const int64_t items_k = weights ? static_cast<int64_t>(d.M) * g.segs_k : 0;
  g.items = g.items_f + items_k;
  g.by_f = make_index_div(g.items_f, g.segs_f);
  g.by_k = make_index_div(items_k, g.segs_k);
  cudaError_t e = by_act(d.act, [&](auto act) {
    constexpr auto kern = ffn_dgate_kernel<T, decltype(act)::value>;
    return launch_dependent(kern, dim3(resident_grid<kern>(g.items, 256)), 256, 0, s, 1, g);
  });
  if (e != cudaSuccess) return e;
  const Operand odg = {dg, d.M, d.F, w.ldf}, odu = {du, d.M, d.F, w.ldf}, ox = {xb, d.M, d.K, w.ldk};
  const Operand opx[4] = {odg, odu, {wg, d.F, d.K, d.ldw}, {wu, d.F, d.K, d.ldw}};
  const Operand opw[4] = {dwg ? odg : odu, odu, ox, ox};
  const bool two = dwg && dwu;
  Job jx = {}, jw = {};
  jx.M = d.M;
  jx.N = d.K;
  jx.steps = (d.F + BK - 1) / BK;
  jx.ld = d.ldx;
  jx.out[0] = dx;
  jw.M = d.F;
  jw.N = d.K;
  jw.steps = (d.M + BK - 1) / BK;
  jw.ld = d.ldw;
  jw.out[0] = dwg ? dwg : dwu;
  jw.out[1] = two ? dwu : nullptr;
  GemmArgs a = {};
  const Pick px = dx ? pick_for<DX, T, 0>(jx, false) : Pick{}, pw = weights ? pick_for<DW, T, 0>(jw, two) : Pick{};
  if (dx && weights) {
    // both in one launch where that is the shorter, a launch's start (2 us) counted
    const int64_t sx = all_steps(DX, jx), sw = all_steps(DW, jw);
    const Pick pb = pick_both(ceil_div(jx.M, BM), sx, ceil_div(jw.M, BM) * (two ? 2 : 1), sw, d.K);
    if (pb.cost < px.cost + pw.cost + 2000) {
      Maps maps = {};
      const Operand opd[3] = {opw[0], opw[1], ox};
      if (!make_maps(maps, 0, DX, pb.columns, opx, 4, d.type) || !make_maps(maps, 4, DW, pb.columns, opd, 3, d.type))
        return cudaErrorInvalidValue;
      a.job[0] = jx;
      a.job[1] = jw;
      a.first = set_tiles(a.job[0], DX, pb.columns, false);
      a.total = a.first + set_tiles(a.job[1], DW, pb.columns, two);
      a.fill = deal_fill(a.first, a.total, fill_of(sx, sw));
      a.split = 1;
      return launch_columns<BWD, T, 0>(pb.columns, maps, a, s);
    }
  }
  if (dx) {
    a.job[0] = jx;
    e = launch_gemm<DX, T, 0>(px, opx, d.type, false, a, s);
    if (e != cudaSuccess) return e;
  }
  if (weights) {
    a.job[0] = jw;
    e = launch_gemm<DW, T, 0>(pw, opw, d.type, two, a, s);
  }
  return e;
}

}  // namespace

size_t ffn_backward_workspace(const samd_ffn_desc &d) { return plan_workspace(d).bytes; }

cudaError_t launch_ffn_forward(const samd_ffn_desc &d, const void *x, const void *wg, const void *wu, void *h,
                               samd_block8 cg, samd_block8 cu, cudaStream_t s) {
  return d.type == SAMD_BF16 ? forward<__nv_bfloat16>(d, x, wg, wu, h, cg, cu, s)
                             : forward<__half>(d, x, wg, wu, h, cg, cu, s);
}

cudaError_t launch_ffn_backward(const samd_ffn_desc &d, const void *dh, samd_block8 cx, samd_block8 cg, samd_block8 cu,
                                const void *wg, const void *wu, void *dx, void *dwg, void *dwu, void *h,
                                void *workspace, cudaStream_t s) {
  return d.type == SAMD_BF16
             ? backward<__nv_bfloat16>(d, dh, cx, cg, cu, wg, wu, dx, dwg, dwu, h, workspace, s)
             : backward<__half>(d, dh, cx, cg, cu, wg, wu, dx, dwg, dwu, h, workspace, s);
}

}  // namespace samd
