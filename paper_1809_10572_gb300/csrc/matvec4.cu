// matvec4.cu -- products of a few tokens with 4-bit weights, and the gated
// pair of them with the activation and the product.
//
//   y[m][n] = sum_G s[n][G] * sum_{k in G} (q[n][k] - z[n][G]) * x[m][k]
//
// Bound: the weights, half a byte each, are read once; a token adds one
// multiply-add to each. At the copy bandwidth a SM receives about 46 weights
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
// Split: a CTA takes 16 * RT rows (of both matrices of the pair) and its eight
// warps take blocks of KB inputs in turn, each through its own ring of cp.async
// stages (weights, tokens, scales, zero points), without a barrier until their
// sums are joined, in a fixed order, at the end.
#include "ffn_internal.cuh"
#include "tc_ptx.cuh"

namespace samd {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;

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
  int nb;             // groups that a block of KB inputs touches
  int nblk;           // blocks of KB inputs
  int s_words, z_words;  // 4-byte words staged for a row's scales and zero points of a block
  int x_rows;         // tokens staged
  int w_vec, x_vec;   // rows are 16-byte aligned
  int is_signed;
  int act;            // of the gated pair; -1: one matrix
  int x_off, s_off, z_off, stage_bytes;  // of a warp's stage
};

__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}

template <typename T>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0,
                                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<__half>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// What is subtracted from the widened lanes of a group with zero point z.
template <typename T>
struct Offset;
template <>
struct Offset<__nv_bfloat16> {
  uint32_t a;
  __device__ __forceinline__ void set(uint32_t z) { a = 0x43004300u | z | z << 16; }
};
template <>
struct Offset<__half> {
  uint32_t a, b;
  __device__ __forceinline__ void set(uint32_t z) {
    const uint32_t zz = z | z << 16;
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

// CH: chunks of 32 inputs in a block.
template <typename T, bool kGated, int RT, int NT, int CH, int STAGES>
__global__ void __launch_bounds__(kThreads) matvec4_kernel(const MvArgs a) {
  constexpr int kMats = kGated ? 2 : 1;
  constexpr int kTiles = RT * kMats;  // 16-row tiles of a CTA: those of the first matrix, then the second's
  constexpr int kRows = 16 * kTiles;
  constexpr int KB = 32 * CH;
  constexpr int kPitch = 16 * CH;      // bytes of a row of weights in a stage
  constexpr int kXPitch = 2 * KB + 64;  // of a token: eight lanes read two tokens' neighbouring 64 bytes without conflict
  constexpr int kSwz = CH >= 8 ? 0 : CH == 4 ? 1 : 2;  // rows that share a 128-byte line
  static_assert(CH == 2 || CH == 4 || CH == 8, "a row of a stage is 32, 64 or 128 bytes");
  extern __shared__ __align__(128) uint8_t smem[];

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;
  const int n0 = blockIdx.x * (16 * RT);
  const int m0 = blockIdx.y * (8 * NT);
  const int tokens = min(a.M - m0, 8 * NT);
  uint8_t *const mine = smem + static_cast<size_t>(warp) * STAGES * a.stage_bytes;
  const T *const x = static_cast<const T *>(a.x) + m0 * a.ldx;

  // One block's weights, tokens, scales and zero points into a stage. Rows past
  // N repeat row N - 1 (their sums are not stored); bytes past a row's end, and
  // inputs past K, are zero.
  auto load = [&](int blk, uint8_t *st) {
    const int64_t k0 = static_cast<int64_t>(blk) * KB;
    const uint32_t sw = ptx::smem_addr(st);
    const int64_t off = k0 / 2;
    if (a.w_vec) {
#pragma unroll
      for (int i = 0; i < kRows * CH / 32; ++i) {
        const int idx = i * 32 + lane, row = idx / CH, ch = idx % CH;
        const int mat = kGated ? row / (16 * RT) : 0;
        const int64_t n = min(n0 + row - mat * 16 * RT, a.N - 1);
        const int64_t at = off + ch * 16;
        const bool in = at < a.row_bytes;  // whole 16-byte units: row_bytes is a multiple of 16
        ptx::cp_async_16(sw + row * kPitch + ((ch ^ ((row >> kSwz) & (CH - 1))) * 16),
                         a.lanes[mat] + n * a.row_bytes + (in ? at : 0), in ? 16u : 0u);
      }
    } else {
      for (int i = 0; i < kRows * CH * 4 / 32; ++i) {
        const int idx = i * 32 + lane, row = idx / (4 * CH), w = idx % (4 * CH), ch = w >> 2;
        const int mat = kGated ? row / (16 * RT) : 0;
        const int64_t n = min(n0 + row - mat * 16 * RT, a.N - 1);
        const int64_t at = off + w * 4;
        const bool in = at < a.row_bytes;
        ptx::cp_async_4(sw + row * kPitch + ((ch ^ ((row >> kSwz) & (CH - 1))) * 16) + (w & 3) * 4,
                        a.lanes[mat] + n * a.row_bytes + (in ? at : 0), in ? 4u : 0u);
      }
    }
    const uint32_t sx = sw + a.x_off;
    if (a.x_vec) {
      for (int idx = lane; idx < tokens * 4 * CH; idx += 32) {
        const int m = idx / (4 * CH), p = idx % (4 * CH);
        const int64_t k = k0 + p * 8, left = a.K - k;
        const uint32_t bytes = left >= 8 ? 16u : left > 0 ? static_cast<uint32_t>(left) * 2u : 0u;
        ptx::cp_async_16(sx + m * kXPitch + p * 16, x + m * a.ldx + (bytes ? k : 0), bytes);
      }
    } else {
      for (int idx = lane; idx < tokens * KB; idx += 32) {
        const int m = idx / KB, p = idx % KB;
        uint16_t v = 0;
        if (k0 + p < a.K) v = reinterpret_cast<const uint16_t *>(x)[m * a.ldx + k0 + p];
        *reinterpret_cast<uint16_t *>(st + a.x_off + m * kXPitch + p * 2) = v;
      }
    }
    // The 4-byte words that hold the row's scales of this block; the reader
    // finds its place in the first word from the same index. A word past the
    // end of the array is clipped.
    const int64_t g0 = k0 >> a.group_shift;
    for (int idx = lane; idx < kRows * a.s_words; idx += 32) {
      const int row = idx / a.s_words, w = idx - row * a.s_words;
      const int mat = kGated ? row / (16 * RT) : 0;
      const int64_t n = min(n0 + row - mat * 16 * RT, a.N - 1);
      const int64_t at = ((n * a.groups + g0) * 2 & ~int64_t(3)) + w * 4, left = a.n_scales * 2 - at;
      ptx::cp_async_4(sw + a.s_off + idx * 4, a.scales[mat] + (left > 0 ? at : 0),
                      left >= 4 ? 4u : left > 0 ? static_cast<uint32_t>(left) : 0u);
    }
    if (a.zeros[0]) {
      for (int idx = lane; idx < kRows * a.z_words; idx += 32) {
        const int row = idx / a.z_words, w = idx - row * a.z_words;
        const int mat = kGated ? row / (16 * RT) : 0;
        const int64_t n = min(n0 + row - mat * 16 * RT, a.N - 1);
        const int64_t at = ((n * a.groups + g0) & ~int64_t(3)) + w * 4, left = a.n_scales - at;
        ptx::cp_async_4(sw + a.z_off + idx * 4, a.zeros[mat] + (left > 0 ? at : 0),
                        left >= 4 ? 4u : left > 0 ? static_cast<uint32_t>(left) : 0u);
      }
    }
  };

  float acc[kTiles][NT][4];
#pragma unroll
  for (int r = 0; r < kTiles; ++r)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[r][j][i] = 0.0f;

  const uint32_t flip = a.is_signed ? 0x00080008u : 0u;
  const bool has_zeros = a.zeros[0] != nullptr;

  int next = warp;
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) {
    if (next < a.nblk) load(next, mine + s * a.stage_bytes);
    ptx::cp_async_commit();
    next += kWarps;
  }
  int slot = 0, fill = STAGES - 1;
  for (int blk = warp; blk < a.nblk; blk += kWarps) {
    ptx::cp_async_wait<STAGES - 2>();
    __syncwarp();  // every lane's copies are in, and the slot filled next has been read by every lane
    if (next < a.nblk) load(next, mine + fill * a.stage_bytes);
    ptx::cp_async_commit();
    next += kWarps;
    fill = fill + 1 == STAGES ? 0 : fill + 1;

    uint8_t *const st = mine + slot * a.stage_bytes;
    slot = slot + 1 == STAGES ? 0 : slot + 1;
    const uint32_t sw = ptx::smem_addr(st);
    const int64_t k0 = static_cast<int64_t>(blk) * KB;
    const int64_t g0 = k0 >> a.group_shift;
    const int64_t left = a.K - k0;
    const int nch = left >= KB ? CH : static_cast<int>((left + 31) / 32);
#pragma unroll
    for (int c2 = 0; c2 < CH; c2 += 2) {
      if (c2 < nch) {
        uint32_t words[kTiles][4];
#pragma unroll
        for (int r = 0; r < kTiles; ++r) {
          const int row = r * 16 + (lane & 15), ch = c2 + (lane >> 4);
          ldmatrix_x4(sw + row * kPitch + ((ch ^ ((row >> kSwz) & (CH - 1))) * 16), words[r]);
        }
#pragma unroll
        for (int cc = 0; cc < 2; ++cc) {
          const int c = c2 + cc;
          if (c < nch) {
            uint32_t b[NT][4];
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              uint4 q = make_uint4(0, 0, 0, 0);
              if (8 * j + g < tokens)
                q = *reinterpret_cast<const uint4 *>(st + a.x_off + (8 * j + g) * kXPitch + c * 64 + t * 16);
              b[j][0] = __byte_perm(q.x, q.z, 0x5410);
              b[j][1] = __byte_perm(q.x, q.z, 0x7632);
              b[j][2] = __byte_perm(q.y, q.w, 0x5410);
              b[j][3] = __byte_perm(q.y, q.w, 0x7632);
            }
            const int gi = static_cast<int>(((k0 + c * 32) >> a.group_shift) - g0);
#pragma unroll
            for (int r = 0; r < kTiles; ++r) {
              const int mat_row = kGated && r >= RT ? r - RT : r;
              uint32_t lo[4], hi[4];
              float s[2];
              Offset<T> o[2];
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const int row = r * 16 + g + 8 * h;
                const int64_t n = min(n0 + mat_row * 16 + g + 8 * h, a.N - 1);
                const int64_t first = n * a.groups + g0;
                s[h] = f32_of_bits<T>(*reinterpret_cast<const uint16_t *>(st + a.s_off + row * a.s_words * 4 +
                                                                          (first & 1) * 2 + gi * 2));
                o[h].set(has_zeros ? st[a.z_off + row * a.z_words * 4 + (first & 3) + gi] & 15u
                                   : (flip & 15u));
              }
              widen(words[r][2 * cc], flip, o[0], lo);
              widen(words[r][2 * cc + 1], flip, o[1], hi);
#pragma unroll
              for (int j = 0; j < NT; ++j) {
                float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                const uint32_t a0[4] = {lo[0], hi[0], lo[1], hi[1]}, a1[4] = {lo[2], hi[2], lo[3], hi[3]};
                mma16816<T>(d, a0, b[j][0], b[j][1]);
                mma16816<T>(d, a1, b[j][2], b[j][3]);
                acc[r][j][0] = fmaf(s[0], d[0], acc[r][j][0]);
                acc[r][j][1] = fmaf(s[0], d[1], acc[r][j][1]);
                acc[r][j][2] = fmaf(s[1], d[2], acc[r][j][2]);
                acc[r][j][3] = fmaf(s[1], d[3], acc[r][j][3]);
              }
            }
          }
        }
      }
    }
  }

  // Join the warps' sums: [warp][row][token], rows one float apart from their
  // neighbours' banks.
  ptx::cp_async_wait<0>();
  __syncthreads();
  constexpr int kTok = 8 * NT, kRed = kTok + 1;
  float *const red = reinterpret_cast<float *>(smem);
#pragma unroll
  for (int r = 0; r < kTiles; ++r)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        red[(warp * kRows + r * 16 + g + (i >> 1) * 8) * kRed + 8 * j + 2 * t + (i & 1)] = acc[r][j][i];
  __syncthreads();
  T *const y = static_cast<T *>(a.y);
  for (int idx = threadIdx.x; idx < 16 * RT * tokens; idx += kThreads) {
    const int m = idx / (16 * RT), row = idx % (16 * RT);
    if (n0 + row >= a.N) continue;
    float v = 0.0f, u = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      v += red[(w * kRows + row) * kRed + m];
      if constexpr (kGated) u += red[(w * kRows + 16 * RT + row) * kRed + m];
    }
    if constexpr (kGated) v = act_of(a.act, v) * u;
    y[(m0 + m) * a.ldy + n0 + row] = from_f32<T>(v);
  }
}

template <typename T, bool kGated, int RT, int NT, int CH, int STAGES>
cudaError_t launch_as(MvArgs a, cudaStream_t s) {
  constexpr int kRows = 16 * RT * (kGated ? 2 : 1), KB = 32 * CH;
  const int group = 1 << a.group_shift;
  a.nb = group >= KB ? 1 : KB / group;
  a.nblk = (a.K + KB - 1) / KB;
  a.s_words = a.nb == 1 ? 1 : a.nb / 2 + 1;
  a.z_words = a.nb == 1 ? 1 : a.nb <= 4 ? 2 : 3;
  a.x_rows = a.M < 8 * NT ? a.M : 8 * NT;
  a.x_off = kRows * 16 * CH;
  a.s_off = a.x_off + a.x_rows * (2 * KB + 64);
  a.z_off = a.s_off + kRows * a.s_words * 4;
  a.stage_bytes = (a.z_off + (a.zeros[0] ? kRows * a.z_words * 4 : 0) + 127) / 128 * 128;
  size_t smem = static_cast<size_t>(kWarps) * STAGES * a.stage_bytes;
  const size_t red = static_cast<size_t>(kWarps) * kRows * (8 * NT + 1) * 4;
  if (red > smem) smem = red;
  const auto kern = matvec4_kernel<T, kGated, RT, NT, CH, STAGES>;
  const cudaError_t e = conv::ensure_smem_attr(reinterpret_cast<const void *>(kern), smem);
  if (e != cudaSuccess) return e;
  const dim3 grid((a.N + 16 * RT - 1) / (16 * RT), (a.M + 8 * NT - 1) / (8 * NT));
  kern<<<grid, kThreads, smem, s>>>(a);
  return cudaGetLastError();
}

template <typename T, bool kGated>
cudaError_t launch_sized(const MvArgs &a, cudaStream_t s) {
  constexpr int kRT = kGated ? 1 : 2;
  if (a.M <= 2) return launch_as<T, kGated, 1, 1, 8, 3>(a, s);
  if (a.M <= 8) return launch_as<T, kGated, 1, 1, 4, 3>(a, s);
  if (a.M <= 16) return launch_as<T, kGated, kRT, 2, 4, 3>(a, s);
  return launch_as<T, kGated, kRT, 4, 2, 3>(a, s);
}

template <typename T>
cudaError_t launch_type(const MvArgs &a, cudaStream_t s) {
  return a.act >= 0 ? launch_sized<T, true>(a, s) : launch_sized<T, false>(a, s);
}

}  // namespace

// act < 0 (wu null): one matrix.
cudaError_t launch_matvec4(const samd_matvec_desc &d, int act, samd_fmt fw, const void *x, const samd_weights4 &wg,
                           const samd_weights4 *wu, void *y, cudaStream_t s) {
  MvArgs a = {};
  const samd_weights4 *const w[2] = {&wg, wu ? wu : &wg};
  for (int i = 0; i < 2; ++i) {
    a.lanes[i] = static_cast<const uint8_t *>(w[i]->lanes);
    a.scales[i] = static_cast<const uint8_t *>(w[i]->scales);
    a.zeros[i] = w[i]->zeros;
  }
  a.ldx = d.ldx;
  a.ldy = d.ldy;
  a.row_bytes = words_per_row(fw, d.K) * (fw.word_bits / 8);
  while ((1 << a.group_shift) < d.group && (1 << a.group_shift) < d.K) ++a.group_shift;
  if (a.group_shift < 5) a.group_shift = 5;
  a.groups = (d.K + (1LL << a.group_shift) - 1) >> a.group_shift;
  a.n_scales = a.groups * d.N;
  a.N = d.N;
  a.K = d.K;
  a.w_vec = a.row_bytes % 16 == 0;
  a.x_vec = d.M == 1 || d.ldx % 8 == 0;
  a.is_signed = fw.is_signed;
  a.act = act;
  // the grid's second axis counts up to 65535 blocks of tokens
  constexpr int kMost = 65535 * 8;
  for (int m = 0; m < d.M; m += kMost) {
    a.M = d.M - m < kMost ? d.M - m : kMost;
    a.x = static_cast<const uint8_t *>(x) + m * d.ldx * 2;
    a.y = static_cast<uint8_t *>(y) + m * d.ldy * 2;
    const cudaError_t e = d.type == SAMD_BF16 ? launch_type<__nv_bfloat16>(a, s) : launch_type<__half>(a, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace samd
