// paged_attention_kernel.cuh -- attention of one new token of each sequence
// over a paged cache of packed lanes.
//
//   x_t = scale log2(e) sum_d q_d K_td,  out_d = sum_t 2^x_t V_td / sum_t 2^x_t
//
// Bound by its reads: a cached token of a key head comes once, 2 dim bits / 8
// bytes and a scale of 16 bits for 32 lanes. Every lane has to be widened to a
// 16-bit float and multiplied with up to eight query heads, which is more than
// the CUDA cores can do at that rate, so the products go through mma.sync
// (m16n8k16): 16 tokens by the 8 heads for the logits, 16 elements by the 8
// heads for the sums. tcgen05 would want the widened lanes in shared memory, at
// two to four times the bytes that come from HBM.
//
// Numbers: a lane over the mantissa of a power of two is that power plus the
// lane, subtracting both is exact in fp16, so the products are those of the
// integers. q is brought into fp16's range by a power of two of its head (its
// largest magnitude to 2^13 .. 2^14: bfloat16's eight and fp16's eleven bits are
// kept, what lies 2^-27 below the largest is rounded at 2^-38 of it). The sums
// of 32 elements are scaled in fp32. For the second product the weight of a
// token and the scale of its 32 values go together, p = 2^(x - ref + up) s,
// rounded once to fp16 (2^-11, as a result in fp16 is; in 16 bits because the
// lanes are the MMA's other operand). ref is a running reference of each head,
// the largest x rounded up to an integer; up belongs to a head and a block of 32
// elements, and brings the block's largest weight times scale to 2^6 .. 2^7, so
// that an output keeps its bits whatever lies in other elements of the rows and
// in other heads. Both move only when a p passes 2^15 (nine doublings later) or
// a weight 2^16, so that a step's common path has no reduction over tokens; being
// integers, they move the sums by powers of two, exactly. Of a block's weights
// times scales those below 2^-20 of the largest are rounded at 2^-31 of it. Logits,
// weights' sums and outputs are in fp32: weights below 2^-126 of the largest are
// 0. (up ends at 2^120: values' scales below 2^-114 lose bits. Sums of values above
// 2^115 may pass fp32, and keys' scales above 2^100 in a logit.)
//
// Layout: a warp takes 16 tokens (one step, never more than one page) through a
// ring of its own in shared memory, filled by cp.async of 16 bytes a lane; rows
// an odd number of 16-byte units apart, so that ldmatrix reads eight rows
// without conflicts. ldmatrix deals a token's word to the thread that has it
// in the MMA's operand (keys), and transposed two tokens' lanes of one element
// (values). The weights change operand layout by movmatrix.
//
// Split: all steps of all sequences and key heads lie in one line, of which
// every CTA takes an equal part, whatever the lengths (and with what beginning a
// head costs counted in); its warps take steps in turn. A CTA's parts of two heads
// are finished one after the other (the ring runs on); where a head's steps lie in
// several CTAs, each leaves its sums and references in the workspace for
// paged_attention_join (fixed order: the same call gives the same bits). Head
// groups of more than eight query heads are neighbouring CTAs that read the same
// pages at the same time.
//
// Measured on one GB300, with the join (GPU time of a call): one sequence of
// 131072 tokens, 8 key heads of 128 elements: 59 us in 8 bits (285 MB, 0.71 of the
// copy bandwidth; twice the tokens of a call cost 1.04 of what their bytes do, so
// that the rest, about 14 us, is fixed: launches, three dependent loads before the
// first step, the join), 49 us in 4 bits (151 MB, 0.46). A step of 16 tokens by 128
// elements is 468 instructions in 4 bits (160 of the logic pipe, 144 for widening)
// and about 580 in 8 (16 sequences of up to 8192 tokens, what beginning their heads
// takes among them); with sixteen warps an SM issue slots are 64 and 58% busy. Blocks'
// own powers cost 24 multiplications and maxima a step: 3 us of the 49, nothing
// where HBM bounds (one range for all blocks of a head: 45.7 and 59.1 us).
#pragma once

#include "cache_internal.cuh"
#include "tc_ptx.cuh"

namespace samd {
namespace kv {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kHeads = 8;     // query heads of a CTA: the MMA's columns
constexpr int kMinSteps = kWarps;  // a CTA is not used for fewer, unless a head has fewer
// What beginning a head takes of a CTA's time, in steps: a join, the next head's length, pages and query, one after the
// other. Counted when steps are dealt out; us of a call with 1, 8, 12, 16, 20, 24 and 32 for it: 53 sequences of up to 4001
// tokens, 12 heads of 96: 73, 64, 59, 56, 58, 59, 58; 16 of up to 8192, 8 heads of 128: 41, 40, 37, 38, 38, 39, 38; 8 of up
// to 16000 in 4 bits with scores: 29.0, 27.8, 27.4, 26.5, 26.4, 25.8, 25.2; one of 131072 in 4 bits: 49 up to 24, 51 with
// 32; one in 8 bits, of any length: within 3% of each other.
constexpr int kHeadCost = 16;
constexpr int kMostUp = 120;             // largest power of a block's weights (log2)
constexpr float kMostWeight = 65536.0f;  // a weight above it moves the reference, whatever its values are

struct AttArgs {
  Seqs s;
  const uint8_t *k, *v, *ks, *vs;
  const uint8_t *q;
  uint8_t *out;
  int64_t ldq, ldo;  // bytes
  float scale;
  int heads;         // of keys
  uint32_t page_rows;  // rows of a page: heads x slots
  int group;         // query heads of a key head
  int parts;         // CTAs that share a key head's pages: ceil(group / per)
  int per;           // query heads of a CTA
  int slots;         // CTAs of a part
  int whole;         // CTAs take whole heads: nothing is split
  // the workspace
  float *sums;       // [CTA][2][kHeads][dim]
  float2 *stat;      // [CTA][kHeads]: reference and sum of weights, of the part of a head that it goes on with
  float2 *head_stat; // [unit][part][kHeads]: of a head's first part; or null, where nothing is split or counted
  int2 *span;        // [unit][part]: first and last slot
  float *logits;     // [unit][part][tokens of max_pages][kHeads]; or null
};

// ---- where the steps lie ---------------------------------------------------------

__host__ __device__ __forceinline__ int steps_of(const Seqs &s, int b) {
  return static_cast<int>((length_of(s, b) + kStep - 1) / kStep);
}

// The steps of a sequence's head as they are dealt out: with what beginning it costs before the first of them.
__host__ __device__ __forceinline__ int64_t dealt_of(int steps) { return steps > 0 ? steps + kHeadCost : 0; }

// CTAs that are used for so many dealt steps of so many heads that have any, and the first one of a CTA's.
__host__ __device__ __forceinline__ int64_t used_of(int64_t all, int64_t units, int slots) {
  const int64_t steps = (all - units * kHeadCost + kMinSteps - 1) / kMinSteps, most = steps > units ? steps : units;
  return most < slots ? most : slots;
}
__host__ __device__ __forceinline__ int64_t begin_of(int64_t slot, int64_t all, int64_t used) { return slot * all / used; }

// By the whole CTA: its dealt steps [begin, end), the sequence that the first lies in, and the step's place from that
// sequence's first, *rem; *used: the CTAs that have steps. Returns the number of all dealt steps. tmp: 2 kWarps + 2.
__device__ __forceinline__ int64_t locate(const Seqs &s, int heads, int slot, int slots, int64_t *tmp, int *b_out,
                                          int64_t *begin, int64_t *end, int64_t *rem, int64_t *used_out) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int chunk = (s.seqs + kThreads - 1) / kThreads, b0 = tid * chunk;
  int64_t mine = 0;
  int some = 0;  // sequences with steps
  for (int b = b0; b < min(b0 + chunk, s.seqs); ++b) {
    const int n = steps_of(s, b);
    mine += dealt_of(n), some += n > 0;
  }
  some = static_cast<int>(__reduce_add_sync(0xffffffffu, static_cast<unsigned>(some)));
  int64_t incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t up = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) tmp[warp] = incl, tmp[kWarps + 2 + warp] = some;
  __syncthreads();
  int64_t before = 0, all = 0, units = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += tmp[w];
    all += tmp[w];
    units += tmp[kWarps + 2 + w];
  }
  all *= heads;
  const int64_t used = *used_out = used_of(all, units * heads, slots);
  *begin = *end = 0;
  if (slot < used) {
    *begin = begin_of(slot, all, used);
    *end = begin_of(slot + 1, all, used);
    int64_t first = (before + incl - mine) * heads;
    if (*begin >= first && *begin < first + mine * heads) {
      int b = b0;
      for (;; ++b) {
        const int64_t n = dealt_of(steps_of(s, b)) * heads;
        if (*begin < first + n) break;
        first += n;
      }
      tmp[kWarps] = b;
      tmp[kWarps + 1] = *begin - first;
    }
  }
  __syncthreads();
  *b_out = static_cast<int>(tmp[kWarps]);
  *rem = tmp[kWarps + 1];
  __syncthreads();
  return all;
}

// The slot that dealt step x of all `all` lies in, of `used`: the last one whose begin, floor(slot all / used), is at most x.
__host__ __device__ __forceinline__ int slot_of(int64_t x, int64_t all, int64_t used) {
  return static_cast<int>(((x + 1) * used - 1) / all);
}

// A walk over the parts of heads that a CTA has: sequence, key head, steps [first, last) of it.
struct Walk {
  int64_t left;  // dealt steps of the CTA behind this part
  int64_t unit;  // the head's first among all dealt steps
  int b, h, steps, first, last;

  __host__ __device__ __forceinline__ bool on() const { return first < last; }
  __host__ __device__ __forceinline__ static int step_at(int64_t dealt) {  // the step that a dealt step is, or comes before
    return dealt > kHeadCost ? static_cast<int>(dealt - kHeadCost) : 0;
  }
  __host__ __device__ __forceinline__ void take(int64_t from) {
    const int64_t all = dealt_of(steps), to = all - from < left ? all : from + left;
    first = step_at(from), last = step_at(to);
    left -= to - from;
  }
  // From dealt step `rem` of sequence b_, dealt step `begin` of all, n of them.
  __host__ __device__ __forceinline__ void start(const AttArgs &a, int b_, int64_t rem, int64_t begin, int64_t n) {
    b = b_, h = 0, first = last = 0, steps = 0, left = n, unit = begin;
    if (n <= 0) return;
    steps = steps_of(a.s, b);
    const int64_t all = dealt_of(steps);
    h = static_cast<int>(rem / all);
    const int64_t from = rem - h * all;
    unit = begin - from;
    take(from);
  }
  __host__ __device__ __forceinline__ void start_whole(const AttArgs &a, int u) {
    left = 0, unit = 0, first = 0;
    b = u / a.heads, h = u - b * a.heads;
    last = steps = u < a.s.seqs * a.heads ? steps_of(a.s, b) : 0;
  }
  // The next part (or, where nothing is split, the next unit, which may have no steps); steps of none at the end.
  __host__ __device__ __forceinline__ void next(const AttArgs &a) {
    if (a.whole) return start_whole(a, b * a.heads + h + a.slots);
    if (left <= 0) {
      first = last = 0;
      return;
    }
    unit += dealt_of(steps);
    if (++h == a.heads) {
      h = 0;
      do steps = steps_of(a.s, ++b);
      while (steps == 0 && b + 1 < a.s.seqs);
    }
    take(0);
  }
};

// ---- operands --------------------------------------------------------------------

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                              uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, "
      "%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ float exp2_of(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint32_t sub_h2(uint32_t a, uint32_t b) {
  const __half2 d = __hsub2(reinterpret_cast<const __half2 &>(a), reinterpret_cast<const __half2 &>(b));
  return reinterpret_cast<const uint32_t &>(d);
}

// The powers of two with a signed lane's zero, in both halves: 1024 + 128 (8 bits), 1024 + 8 and 64 + 8 (4 bits, at bit 0
// and at bit 4). Held in registers that the compiler does not know the values of: it would spend an instruction more on
// every (w & mask) ^ power of two constants.
template <int BITS>
struct Powers {
  uint32_t v[BITS == 8 ? 1 : 2];
  __device__ __forceinline__ Powers() {
    if constexpr (BITS == 8) {
      asm volatile("mov.u32 %0, 0x64806480;" : "=r"(v[0]));
    } else {
      asm volatile("mov.u32 %0, 0x64086408;" : "=r"(v[0]));
      asm volatile("mov.u32 %0, 0x54805480;" : "=r"(v[1]));
    }
  }
};
__device__ __forceinline__ uint32_t and_xor(uint32_t w, uint32_t mask, uint32_t x) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0x6A;" : "=r"(r) : "r"(w), "r"(mask), "r"(x));
  return r;
}

// Signed lanes of a word, or of two tokens' halves of words, as pairs in fp16: lane i of the low half with lane i of
// the high half.
template <int BITS>
__device__ __forceinline__ void widen(uint32_t w, const Powers<BITS> &c, uint32_t (&p)[16 / BITS]) {
  if constexpr (BITS == 8) {
    p[0] = sub_h2(and_xor(w, 0x00FF00FFu, c.v[0]), c.v[0]);
    p[1] = sub_h2(and_xor(w >> 8, 0x00FF00FFu, c.v[0]), c.v[0]);
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t v = w >> 8 * i;
      p[2 * i] = sub_h2(and_xor(v, 0x000F000Fu, c.v[0]), c.v[0]);
      p[2 * i + 1] = sub_h2(and_xor(v, 0x00F000F0u, c.v[1]), c.v[1]);
    }
  }
}

// ---- sizes -------------------------------------------------------------------------

// NB: blocks of 32 elements in a row.
template <int NB, int BITS>
struct Att {
  static constexpr int kDim = 32 * NB;
  static constexpr int kRow = 4 * NB * BITS;        // bytes of a row of lanes
  static constexpr int kUnits = kRow / 16;
  // Rows in a stage: a power of two of units, swizzled (unit u of row r at u ^ (r >> kShift)), or an odd number of them.
  static constexpr bool kSwizzled = (kUnits & (kUnits - 1)) == 0;
  static constexpr int kShift = kUnits >= 8 ? 0 : kUnits == 4 ? 1 : 2;
  static constexpr int kMask = kUnits >= 8 ? 7 : kUnits - 1;
  static constexpr int kPitch = 16 * (kSwizzled ? kUnits : kUnits | 1);
  static constexpr int kScales = kStep * NB * 2;    // bytes of a step's scales, of keys or values
  // (whole swizzle patterns: a unit's place in a stage is an exclusive or of its address)
  static constexpr int kStage = (2 * kStep * kPitch + 2 * kScales + 255) / 256 * 256;
  // The warps' sums when they are joined, [head][element]: in the stage that each of them fills next, where that holds them
  static constexpr int kSums = kHeads * kDim * 4;
  static constexpr bool kInStage = kStage >= kSums;
  static constexpr int bytes(int stages) { return kWarps * (stages * kStage + (kInStage ? 0 : kSums)); }
  // (with what the system keeps of a CTA's shared memory, and the kernel's own)
  static constexpr bool fits(int stages, int ctas) { return ctas * (bytes(stages) + 1024 + 768) <= 228 * 1024; }
  // CTAs of an SM by their registers (128 a thread with four, 168 with three); then as many stages a warp as fit, up to four
  static constexpr int kCtas = NB <= 4 && fits(2, 4) ? 4 : NB <= 6 && fits(2, 3) ? 3 : 2;
  static constexpr int kStages = fits(4, kCtas) ? 4 : fits(3, kCtas) ? 3 : 2;
  static_assert(fits(kStages, kCtas), "shared memory");
  // where unit u of row r of a stage begins
  static __device__ __forceinline__ int at(int r, int u) {
    return r * kPitch + (kSwizzled ? u ^ ((r >> kShift) & kMask) : u) * 16;
  }
};

// The scales of a row, two in a word, from shared memory.
template <int NB>
__device__ __forceinline__ void load_scales(const uint8_t *p, uint32_t (&w)[(NB + 1) / 2]) {
  if constexpr (NB % 8 == 0) {
    const uint4 v = *reinterpret_cast<const uint4 *>(p);
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
  } else if constexpr (NB % 4 == 0) {
    const uint2 v = *reinterpret_cast<const uint2 *>(p);
    w[0] = v.x, w[1] = v.y;
  } else if constexpr (NB % 2 == 0) {
#pragma unroll
    for (int i = 0; i < NB / 2; ++i) w[i] = reinterpret_cast<const uint32_t *>(p)[i];
  } else {
    const uint16_t *const h = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
    for (int i = 0; i < (NB + 1) / 2; ++i) w[i] = h[2 * i] | (2 * i + 1 < NB ? static_cast<uint32_t>(h[2 * i + 1]) << 16 : 0u);
  }
}
template <typename T>
__device__ __forceinline__ float scale_at(const uint32_t *w, int g) {
  const float2 f = unpack2<T>(w[g / 2]);
  return g & 1 ? f.y : f.x;
}

// 2^n, 0 below fp32's normal range (n up to 127).
__device__ __forceinline__ float power_of_two(int n) { return n < -126 ? 0.0f : __int_as_float((127 + n) << 23); }
// The power of two at or below a magnitude (subnormal ones and 0: 2^-127).
__device__ __forceinline__ int log2_down(float v) { return static_cast<int>((__float_as_uint(v) & 0x7FFFFFFFu) >> 23) - 127; }
// The larger magnitude in both halves, under any sign; NaN where either is one.
__device__ __forceinline__ uint32_t max_abs_h2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

template <typename T, int NB, int BITS>
__global__ void __launch_bounds__(kThreads, Att<NB, BITS>::kCtas) paged_attention_kernel(const AttArgs a) {
  using P = Att<NB, BITS>;
  constexpr int kDim = P::kDim, kUnits = P::kUnits, kPitch = P::kPitch, kStages = P::kStages;
  constexpr int kTiles = kDim / 16;  // of 16 elements
  constexpr float kLow = -3e38f;     // a reference before any token
  extern __shared__ __align__(256) uint8_t smem[];
  __shared__ int64_t tmp[2 * kWarps + 2];
  __shared__ float2 red_stat[kWarps][kHeads];  // references and sums of weights
  __shared__ float *red_at[kWarps];            // the warps' sums
  __shared__ Walk walks[2][kWarps];            // where a warp's loads are, and its sums
  // (the warp's number by a shuffle: what follows from it is the same in all lanes, and the compiler knows)
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, g = lane >> 2, t = lane & 3;
  const Powers<BITS> power;

  // the cache, the lengths and q may come from the kernel before; the next one may be set up
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();

  const int slot = blockIdx.x / a.parts, part = blockIdx.x - slot * a.parts;
  const int64_t span_tokens = static_cast<int64_t>(a.s.max_pages) << a.s.page_shift;
  int64_t all = 0, used = 1;
  Walk have;
  if (a.whole) {
    have.start_whole(a, slot);
  } else {
    int b;
    int64_t begin, end, rem;
    all = locate(a.s, a.heads, slot, a.slots, tmp, &b, &begin, &end, &rem, &used);
    if (begin >= end) return;
    have.start(a, b, rem, begin, end - begin);
  }

  // ---- the ring: this warp's steps, one after the other, over the CTA's parts
  const uint32_t ring = ptx::smem_addr(smem) + warp * kStages * P::kStage;
  constexpr int kCopies = (kStep * kUnits + 31) / 32;
  uint32_t copy_at[kCopies];  // where the lane's units of a step's rows go in a stage
#pragma unroll
  for (int i = 0; i < kCopies; ++i) copy_at[i] = P::at((i * 32 + lane) / kUnits, (i * 32 + lane) % kUnits);
  const uint8_t *const k_lane = a.k + lane * 16, *const v_lane = a.v + lane * 16;
  const uint8_t *const s_lane = lane < 2 * NB ? a.ks + lane * 16 : a.vs + (lane - 2 * NB) * 16;  // (lanes below 4 NB)
  // (what a step has no use for lies in shared memory: the loop has no register left)
  Walk *const ahead = &walks[0][warp], *const kept = &walks[1][warp];
  if (lane == 0) *ahead = have;
  __syncwarp();
  int l_step = have.first + warp, l_last = have.last, fill = 0, slot_used = 0;
  uint32_t missing = 0;  // bit of a stage: its page is none of the cache's
  int l_pages = -1, l_turn = 0;  // pages of the warp's next 32 steps, a step a lane; which of them is next
  uint32_t head_rows = 0;  // of a page, before the key head in hand
  // brings `ahead` and l_step to the next step of this warp, and asks for its page, which the next load waits for
  auto seek = [&]() {
    if (l_step < l_last && l_turn < 32) return;
    Walk w = *ahead;
    bool fresh = false;
    while (l_step >= w.last) {
      const int was = w.b * a.heads + w.h;
      w.next(a);
      if (a.whole ? was + a.slots >= a.s.seqs * a.heads : !w.on()) {
        l_step = -1;
        return;
      }
      l_step = w.first + warp;
      fresh = true;
    }
    __syncwarp();
    if (fresh && lane == 0) *ahead = w;
    __syncwarp();
    l_last = w.last;
    head_rows = static_cast<uint32_t>(w.h) << a.s.page_shift;
    const int step = l_step + kWarps * lane;
    l_pages = step < w.last ? page_of(a.s, w.b, static_cast<int64_t>(step) * kStep) : -1;
    l_turn = 0;
  };
  auto load_next = [&]() {
    if (l_step >= 0) {
      const uint32_t st = ring + fill * P::kStage;
      // (a page that is none of the cache's: the stage keeps what it holds, and the step counts nothing)
      const int l_page = __shfl_sync(0xffffffffu, l_pages, l_turn++);
      missing = l_page >= 0 ? missing & ~(1u << fill) : missing | 1u << fill;
      if (l_page >= 0) {
        const uint32_t pos = static_cast<uint32_t>(l_step * kStep) & ((1u << a.s.page_shift) - 1);  // (tokens are counted in an int)
        const uint64_t row = static_cast<uint64_t>(static_cast<uint32_t>(l_page)) * a.page_rows + (head_rows + pos);
        const uint8_t *const kp = k_lane + row * P::kRow, *const vp = v_lane + row * P::kRow;
#pragma unroll
        for (int i = 0; i < kCopies; ++i)
          if (kStep * kUnits % 32 == 0 || i * 32 + lane < kStep * kUnits) {
            ptx::cp_async_16(st + copy_at[i], kp + i * 512);
            ptx::cp_async_16(st + copy_at[i] + kStep * kPitch, vp + i * 512);
          }
        if (lane < 4 * NB) ptx::cp_async_16(st + 2 * kStep * kPitch + lane * 16, s_lane + row * (2 * NB));
      }
      l_step += kWarps;
      seek();
    }
    ptx::cp_async_commit();
    fill = fill + 1 == kStages ? 0 : fill + 1;
  };
  l_turn = 32;
  seek();
#pragma unroll 1
  for (int i = 0; i < kStages - 1; ++i) load_next();

  // ldmatrix: keys: matrices (rows 0-7, unit c), (rows 8-15, c), (rows 0-7, c + 1), (rows 8-15, c + 1); values the
  // same, transposed: (tokens 0-7), (tokens 8-15) of a unit
  const uint32_t lm = P::at((lane >> 3 & 1) * 8 + (lane & 7), kUnits > 1 ? lane >> 4 : 0);
  // units 2 i and 2 i + 1 of the rows of keys (0) or values (1) of a stage
  auto pair_at = [&](uint32_t st, int v, int i) {
    return P::kSwizzled ? (st + v * kStep * kPitch + lm) ^ (i * 32) : st + v * kStep * kPitch + lm + i * 32;
  };

  // the elements of q that a thread has of a head's row, head g's: those of its word of every unit
  constexpr int kQ = 32 / BITS;
  uint32_t q_raw[kUnits][kQ / 2];
  auto load_q = [&](const Walk &w) {
    const bool on = g < min(a.per, a.group - part * a.per);
    const T *const row = reinterpret_cast<const T *>(a.q + w.b * a.ldq) +
                         static_cast<int64_t>(w.h * a.group + part * a.per + (on ? g : 0)) * kDim;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      if constexpr (BITS == 8) {
        const uint2 v = *reinterpret_cast<const uint2 *>(row + u * 16 + t * 4);
        q_raw[u][0] = on ? v.x : 0u, q_raw[u][1] = on ? v.y : 0u;
      } else {
        const uint4 v = *reinterpret_cast<const uint4 *>(row + u * 32 + t * 8);
        q_raw[u][0] = on ? v.x : 0u, q_raw[u][1] = on ? v.y : 0u, q_raw[u][2] = on ? v.z : 0u, q_raw[u][3] = on ? v.w : 0u;
      }
    }
  };
  const int total_units = a.s.seqs * a.heads;
  auto goes_on = [&](const Walk &w) { return a.whole ? w.b * a.heads + w.h < total_units : w.on(); };
  if (goes_on(have)) load_q(have);
  while (goes_on(have)) {
    const int len = static_cast<int>(length_of(a.s, have.b));
    float *logits = nullptr;  // the thread's two heads of the first token that it has
    if (a.logits)
      logits = a.logits + ((static_cast<int64_t>(have.b * a.heads + have.h) * a.parts + part) * span_tokens + g) * kHeads + 2 * t;

    // q of head g in the MMA's order, in fp16 under a power of two
    uint32_t qb[kUnits][16 / BITS];  // pairs of a unit of 16 bytes: 2 (8 bits) or 4 (4 bits) words
    float mult[2];
    {
      float top = 0.0f;
      float f[kUnits][kQ];
#pragma unroll
      for (int u = 0; u < kUnits; ++u)
#pragma unroll
        for (int i = 0; i < kQ / 2; ++i) {
          const float2 e = unpack2<T>(q_raw[u][i]);
          f[u][2 * i] = e.x, f[u][2 * i + 1] = e.y;
          top = fmaxf(top, fmaxf(fabsf(e.x), fabsf(e.y)));
        }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // to 2^13 .. 2^14; powers of two in two halves, each within fp32's range
      const int e = 13 - (static_cast<int>(__float_as_uint(top) >> 23) - 127);
      const int e0 = e / 2, e1 = e - e0;
      const float up0 = __int_as_float((127 + e0) << 23), up1 = __int_as_float((127 + e1) << 23);
      const float down = __int_as_float((127 - e0) << 23), down1 = __int_as_float((127 - e1) << 23);
#pragma unroll
      for (int u = 0; u < kUnits; ++u)
#pragma unroll
        for (int i = 0; i < kQ / 2; ++i)  // the word's pairs: lanes (i, i + half of them)
          qb[u][i] = pack2<__half>(f[u][i] * up0 * up1, f[u][i + kQ / 2] * up0 * up1);
      // (an infinity: all logits are NaNs, also where the products would be infinities of one sign)
      const float m = top <= 3.402823466e38f ? a.scale * down * down1 * 1.4426950408889634f : NAN;
      mult[0] = __shfl_sync(0xffffffffu, m, 8 * t);
      mult[1] = __shfl_sync(0xffffffffu, m, 8 * t + 4);
    }

    float o[kTiles][4], ref[2] = {kLow, kLow}, sum[2] = {0.0f, 0.0f};
    float up[NB][2];  // 2^up of every block, for each of the two heads
#pragma unroll
    for (int i = 0; i < NB; ++i) up[i][0] = up[i][1] = power_of_two(kMostUp);
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[i][j] = 0.0f;

    const int last = have.last;
    int step = have.first + warp;
    if (lane == 0) *kept = have;
    __syncwarp();
#pragma unroll 1
    for (; step < last; step += kWarps) {
      ptx::cp_async_wait<kStages - 2>();
      __syncwarp();  // every lane's copies are in, and the stage filled next has been read by every lane
      const bool gone = (missing >> slot_used & 1) != 0;
      load_next();
      const uint32_t st = ring + slot_used * P::kStage;
      const uint8_t *const sc = smem + (st - ptx::smem_addr(smem)) + 2 * kStep * kPitch;
      slot_used = slot_used + 1 == kStages ? 0 : slot_used + 1;

      // logits
      uint32_t kw[2][(NB + 1) / 2];
#pragma unroll
      for (int r = 0; r < 2; ++r) load_scales<NB>(sc + (g + 8 * r) * (2 * NB), kw[r]);
      float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      // the products of a unit pair: 8 bits: both halves of block u / 2; 4 bits: blocks u and u + 1
#pragma unroll
      for (int u = 0; u < kUnits; u += 2) {
        uint32_t r[4];
        ldsm4(pair_at(st, 0, u / 2), r);  // (one unit, or past the last of an odd number: the second half is not used)
        if constexpr (BITS == 8) {
          float d[4];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            uint32_t lo[2], hi[2];
            widen<8>(r[2 * i], power, lo);
            widen<8>(r[2 * i + 1], power, hi);
            if (i == 0)
              mma_f16_first(d, lo[0], hi[0], lo[1], hi[1], qb[u][0], qb[u][1]);
            else
              mma_f16(d, lo[0], hi[0], lo[1], hi[1], qb[u + 1][0], qb[u + 1][1]);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = fmaf(scale_at<T>(kw[j >> 1], u / 2), d[j], x[j]);
        } else {
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (u + i < kUnits) {
              float d[4];
              uint32_t lo[4], hi[4];
              widen<4>(r[2 * i], power, lo);
              widen<4>(r[2 * i + 1], power, hi);
              mma_f16_first(d, lo[0], hi[0], lo[1], hi[1], qb[u + i][0], qb[u + i][1]);
              mma_f16(d, lo[2], hi[2], lo[3], hi[3], qb[u + i][2], qb[u + i][3]);
#pragma unroll
              for (int j = 0; j < 4; ++j) x[j] = fmaf(scale_at<T>(kw[j >> 1], u + i), d[j], x[j]);
            }
        }
      }

      // the values' scales
      const int tok = step * kStep + g;
      uint32_t vw[2][(NB + 1) / 2];
#pragma unroll
      for (int r = 0; r < 2; ++r) load_scales<NB>(sc + P::kScales + (g + 8 * r) * (2 * NB), vw[r]);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] *= mult[j & 1];
      if (gone || (step + 1) * kStep > len) {  // a token that is not there has no scale and no weight
#pragma unroll
        for (int r = 0; r < 2; ++r)
          if (gone || tok + 8 * r >= len) {
#pragma unroll
            for (int i = 0; i < (NB + 1) / 2; ++i) vw[r][i] = 0u;
            x[2 * r] = x[2 * r + 1] = -INFINITY;
          }
      }
      if (logits) {
        float *const lp = logits + static_cast<int64_t>(step) * (kStep * kHeads);
        *reinterpret_cast<float2 *>(lp) = make_float2(x[0], x[1]);
        *reinterpret_cast<float2 *>(lp + 8 * kHeads) = make_float2(x[2], x[3]);
      }

      float e[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) e[j] = exp2_of(x[j] - ref[j & 1]);
      uint32_t w[NB][2];  // weights times scales, of the thread's two tokens
      auto weigh = [&]() {
        uint32_t most[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) {
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const float s = scale_at<T>(vw[r], i);
            w[i][r] = pack2<__half>(e[2 * r] * s * up[i][0], e[2 * r + 1] * s * up[i][1]);
          }
          most[i] = max_abs_h2(w[i][0], w[i][1]);
        }
#pragma unroll
        for (int n = 1; n < NB; n *= 2)
#pragma unroll
          for (int i = 0; i + n < NB; i += 2 * n) most[i] = max_abs_h2(most[i], most[i + n]);
        return most[0] & 0x7FFF7FFFu;
      };
      const uint32_t most = weigh();
      // (a half above 2^15 carries into its sign)
      const bool past = ((most + 0x07FF07FFu) & 0x80008000u) != 0 ||
                        fmaxf(fmaxf(e[0], e[1]), fmaxf(e[2], e[3])) > kMostWeight;
      if (__any_sync(0xffffffffu, past)) {
        int by[2];
        bool moves[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          // (of this head's column alone: a head's bits do not depend on its neighbours)
          const bool over = (most >> 16 * c & 0x7FFFu) > 0x7800u || fmaxf(e[c], e[2 + c]) > kMostWeight;
          moves[c] = (__ballot_sync(0xffffffffu, over) & 0x11111111u << t) != 0;
          float top = fmaxf(x[c], x[2 + c]);
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
          top = moves[c] ? fmaxf(ceilf(top), ref[c]) : ref[c];
          const float far = top - ref[c];
          by[c] = far < 512.0f ? static_cast<int>(far) : 512;
          ref[c] = top;
          sum[c] *= power_of_two(-by[c]);
#pragma unroll
          for (int r = 0; r < 2; ++r) e[2 * r + c] = exp2_of(x[2 * r + c] - top);
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          uint32_t sizes = 0;  // exponents of the largest weight times scale, of both heads
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const float m = fmaxf(fabsf(e[c] * scale_at<T>(vw[0], i)), fabsf(e[2 + c] * scale_at<T>(vw[1], i)));
            sizes |= static_cast<uint32_t>(log2_down(m) + 127) << 16 * c;
          }
          sizes = __vmaxu2(sizes, __shfl_xor_sync(0xffffffffu, sizes, 4));
          sizes = __vmaxu2(sizes, __shfl_xor_sync(0xffffffffu, sizes, 8));
          sizes = __vmaxu2(sizes, __shfl_xor_sync(0xffffffffu, sizes, 16));
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            // what the block's power is under the new reference, and with it what its sums are worth
            const int had = log2_down(up[i][c]) + by[c], size = static_cast<int>(sizes >> 16 * c & 0xFFFFu) - 127;
            int now = had < kMostUp ? had : kMostUp;
            if (moves[c] && size + now >= 15) now = 6 - size;
            up[i][c] = power_of_two(now);
            const float f = power_of_two(now - had);
            o[2 * i][c] *= f, o[2 * i][2 + c] *= f, o[2 * i + 1][c] *= f, o[2 * i + 1][2 + c] *= f;
          }
        }
        weigh();
      }
      sum[0] += e[0] + e[2];
      sum[1] += e[1] + e[3];

      // outputs: a block's weights, and the two units (8 bits) or the one (4 bits) that hold its values
      uint32_t r[4];
#pragma unroll
      for (int blk = 0; blk < NB; ++blk) {
        const uint32_t b0 = transpose8x8(w[blk][0]), b1 = transpose8x8(w[blk][1]);
        if (BITS == 8 || (blk & 1) == 0) ldsm4_trans(pair_at(st, 1, BITS == 8 ? blk : blk / 2), r);
        uint32_t lo[16 / BITS], hi[16 / BITS];
        if constexpr (BITS == 8) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            widen<8>(r[2 * i], power, lo);
            widen<8>(r[2 * i + 1], power, hi);
            mma_f16(o[2 * blk + i], lo[0], lo[1], hi[0], hi[1], b0, b1);
          }
        } else {
          widen<4>(r[2 * (blk & 1)], power, lo);
          widen<4>(r[2 * (blk & 1) + 1], power, hi);
          mma_f16(o[2 * blk], lo[0], lo[1], hi[0], hi[1], b0, b1);
          mma_f16(o[2 * blk + 1], lo[2], lo[3], hi[2], hi[3], b0, b1);
        }
      }
    }

    have = *kept;
    const int unit = have.b * a.heads + have.h;
    const int head0 = have.h * a.group + part * a.per;  // the CTA's first query head
    const int n_heads = min(a.per, a.group - part * a.per);
    Walk then = have;
    then.next(a);
    if (goes_on(then)) load_q(then);  // on its way while the warps join

    // ---- join the warps: sums [warp][head][element], references and weights [warp][head]
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      sum[c] += __shfl_xor_sync(0xffffffffu, sum[c], 4);
      sum[c] += __shfl_xor_sync(0xffffffffu, sum[c], 8);
      sum[c] += __shfl_xor_sync(0xffffffffu, sum[c], 16);
      // the sum of weights to 1 .. 2, and the blocks' powers off: what is left is the size of values, in any scales (past
      // 2^24 a reference may not hold the sum's power, which then stays where it is)
      int size = sum[c] > 0.0f ? log2_down(sum[c]) : 0;
      if (ref[c] + static_cast<float>(size) - ref[c] != static_cast<float>(size)) size = 0;
      ref[c] += static_cast<float>(size);
      sum[c] *= power_of_two(-size);
#pragma unroll
      for (int i = 0; i < NB; ++i) up[i][c] = power_of_two(-size - log2_down(up[i][c]));
    }
    if (g == 0) {
#pragma unroll
      for (int c = 0; c < 2; ++c) red_stat[warp][2 * t + c] = make_float2(ref[c], sum[c]);
    }
    // (the stage filled next holds nothing that is still wanted)
    float *const red = reinterpret_cast<float *>(P::kInStage ? smem + (warp * kStages + fill) * P::kStage
                                                             : smem + kWarps * kStages * P::kStage + warp * P::kSums);
    if (lane == 0) red_at[warp] = red;
    __syncwarp();  // every lane has read the last stage
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // row g (and g + 8) of tile i is this element
        const int d = BITS == 8 ? 16 * i + 2 * g + (j >> 1) : 32 * (i / 2) + 4 * g + 2 * (i & 1) + (j >> 1);
        red[(2 * t + (j & 1)) * kDim + d] = o[i][j] * up[i / 2][j & 1];
      }
    __syncthreads();
    const bool first_part = have.first == 0, last_part = have.last == have.steps;
    for (int idx = tid; idx < n_heads * (kDim / 2); idx += kThreads) {
      const int h = idx / (kDim / 2), d = (idx - h * (kDim / 2)) * 2;
      float top = kLow;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, red_stat[w][h].x);
      float2 v = make_float2(0.0f, 0.0f);
      float weight = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = exp2_of(red_stat[w][h].x - top);
        const float2 p = *reinterpret_cast<const float2 *>(red_at[w] + h * kDim + d);
        v.x = fmaf(f, p.x, v.x);
        v.y = fmaf(f, p.y, v.y);
        weight = fmaf(f, red_stat[w][h].y, weight);
      }
      if (d == 0 && a.head_stat) {
        float2 *const to = first_part ? a.head_stat + (static_cast<int64_t>(unit) * a.parts + part) * kHeads
                                      : a.stat + static_cast<int64_t>(blockIdx.x) * kHeads;
        to[h] = make_float2(top, weight);
      }
      if (first_part && last_part) {
        const float inv = weight == 0.0f ? 0.0f : 1.0f / weight;  // no tokens: zeros
        *reinterpret_cast<uint32_t *>(a.out + have.b * a.ldo + (static_cast<int64_t>(head0 + h) * kDim + d) * 2) =
            pack2<T>(v.x * inv, v.y * inv);
      } else {
        float *const to = a.sums + ((static_cast<int64_t>(blockIdx.x) * 2 + first_part) * kHeads + h) * kDim + d;
        *reinterpret_cast<float2 *>(to) = v;
      }
    }
    if (!a.whole && first_part && tid == 0)
      a.span[static_cast<int64_t>(unit) * a.parts + part] =
          make_int2(slot, slot_of(have.unit + dealt_of(have.steps) - 1, all, used));
    __syncthreads();
    have = then;
  }
  ptx::cp_async_wait<0>();
}

// ---- host ----------------------------------------------------------------------------

template <typename T, int NB, int BITS>
cudaError_t launch_att(const AttArgs &a, int grid, cudaStream_t s) {
  using P = Att<NB, BITS>;
  constexpr auto kern = paged_attention_kernel<T, NB, BITS>;
  const cudaError_t e = conv::ensure_smem_attr(reinterpret_cast<const void *>(kern), P::bytes(P::kStages));
  if (e != cudaSuccess) return e;
  return launch_dependent(kern, dim3(grid), kThreads, P::bytes(P::kStages), s, 1, a);
}

// CTAs on an SM of the instance for rows of nb blocks.
template <int BITS>
constexpr int ctas_of(int nb) {
  return nb == 1   ? Att<1, BITS>::kCtas
         : nb == 2 ? Att<2, BITS>::kCtas
         : nb == 3 ? Att<3, BITS>::kCtas
         : nb == 4 ? Att<4, BITS>::kCtas
         : nb == 5 ? Att<5, BITS>::kCtas
         : nb == 6 ? Att<6, BITS>::kCtas
         : nb == 7 ? Att<7, BITS>::kCtas
                   : Att<8, BITS>::kCtas;
}

// One launcher a type and lane width, each compiled in its own unit.
template <typename T, int BITS>
cudaError_t launch_dims(const AttArgs &a, int nb, int grid, cudaStream_t s) {
  switch (nb) {
    case 1: return launch_att<T, 1, BITS>(a, grid, s);
    case 2: return launch_att<T, 2, BITS>(a, grid, s);
    case 3: return launch_att<T, 3, BITS>(a, grid, s);
    case 4: return launch_att<T, 4, BITS>(a, grid, s);
    case 5: return launch_att<T, 5, BITS>(a, grid, s);
    case 6: return launch_att<T, 6, BITS>(a, grid, s);
    case 7: return launch_att<T, 7, BITS>(a, grid, s);
    default: return launch_att<T, 8, BITS>(a, grid, s);
  }
}
cudaError_t launch_att_bf16_8(const AttArgs &a, int nb, int grid, cudaStream_t s);
cudaError_t launch_att_bf16_4(const AttArgs &a, int nb, int grid, cudaStream_t s);
cudaError_t launch_att_f16_8(const AttArgs &a, int nb, int grid, cudaStream_t s);
cudaError_t launch_att_f16_4(const AttArgs &a, int nb, int grid, cudaStream_t s);

}  // namespace kv
}  // namespace samd
