// samd_api.cu -- the extern "C" entry points of libsamd: argument checks on
// the host, then one launch (or two, for the convolution) on the caller's
// stream. See include/samd.h for the contract of each call.
#include <mutex>

#include "cache_internal.cuh"
#include "ffn_internal.cuh"
#include "moe4_kernel.cuh"
#include "samd_internal.cuh"

namespace samd {

int sm_count() {
  static std::mutex mu;
  static int cache[64] = {0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  std::lock_guard<std::mutex> lock(mu);
  if (cache[dev] == 0) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) n = 148;
    cache[dev] = n;
  }
  return cache[dev];
}

namespace {

samd_status from_cuda(cudaError_t e) { return e == cudaSuccess ? SAMD_OK : SAMD_ECUDA; }

bool shape_ok(int64_t rows, int64_t inner) { return rows >= 0 && inner >= 0 && (rows == 0 || inner <= INT64_MAX / rows); }

}  // namespace
}  // namespace samd

using namespace samd;

extern "C" {

size_t samd_lanes_per_word(samd_fmt f) { return static_cast<size_t>(lanes_per_word(f)); }

int64_t samd_packed_words(samd_fmt f, int64_t rows, int64_t inner) {
  if (!fmt_valid(f) || !shape_ok(rows, inner)) return -1;
  return rows * words_per_row(f, inner);
}

samd_status samd_pack(samd_fmt f, const int8_t *src, void *dst, int64_t rows, int64_t inner, samd_stream_t stream) {
  if (!fmt_valid(f)) return SAMD_EINVAL;
  if (!shape_ok(rows, inner)) return SAMD_ESHAPE;
  if (rows == 0 || inner == 0) return SAMD_OK;
  if (!src || !dst) return SAMD_EINVAL;
  if (!aligned16(src) || !aligned16(dst)) return SAMD_EALIGN;
  return from_cuda(launch_pack(f, src, dst, rows, inner, reinterpret_cast<cudaStream_t>(stream)));
}

samd_status samd_unpack(samd_fmt f, const void *src, int8_t *dst, int64_t rows, int64_t inner,
                        samd_stream_t stream) {
  if (!fmt_valid(f)) return SAMD_EINVAL;
  if (!shape_ok(rows, inner)) return SAMD_ESHAPE;
  if (rows == 0 || inner == 0) return SAMD_OK;
  if (!src || !dst) return SAMD_EINVAL;
  if (!aligned16(src) || !aligned16(dst)) return SAMD_EALIGN;
  return from_cuda(launch_unpack(f, src, dst, rows, inner, reinterpret_cast<cudaStream_t>(stream)));
}

samd_status samd_elementwise(samd_op op, samd_fmt fa, const void *a, const void *b, samd_fmt fo, void *out,
                             int64_t n, int shift, int saturate, samd_stream_t stream) {
  if (op < SAMD_ADD || op > SAMD_REQUANT) return SAMD_EINVAL;
  if (!fmt_valid(fa) || !fmt_valid(fo)) return SAMD_EINVAL;
  if (saturate != 0 && saturate != 1) return SAMD_EINVAL;
  if (op == SAMD_REQUANT) {
    if (shift < 0 || shift > 31) return SAMD_EINVAL;
  } else if (!same_fmt(fa, fo)) {
    return SAMD_EINVAL;
  }
  if (n < 0) return SAMD_ESHAPE;
  if (n == 0) return SAMD_OK;
  const bool binary = op == SAMD_ADD || op == SAMD_SUB || op == SAMD_MUL;
  if (!a || !out || (binary && !b)) return SAMD_EINVAL;
  if (!aligned16(a) || !aligned16(out) || (binary && !aligned16(b))) return SAMD_EALIGN;
  return from_cuda(launch_elementwise(op, fa, a, binary ? b : nullptr, fo, out, n, op == SAMD_REQUANT ? shift : 0,
                                      binary ? saturate : 0, reinterpret_cast<cudaStream_t>(stream)));
}

size_t samd_conv2d_workspace_size(const samd_conv_desc *d, samd_fmt fa, samd_fmt fw) {
  if (!d || !fmt_valid(fa) || !fmt_valid(fw)) return 0;
  if (d->N < 0 || d->C < 1 || d->H < 1 || d->W < 1 || d->K < 1 || d->R < 1 || d->S < 1 || d->stride < 1 ||
      d->pad < 0)
    return 0;
  if (d->layout == SAMD_NCHW) {
    size_t ws = 0;
    if (fa.spacer != 0 || fw.spacer != 0 || d->R > 16 || d->S > 16) return 0;
    return conv2d_nchw_check(d, fa, fw, samd_fmt{0, 0, 0, 0}, &ws) == SAMD_OK ? ws : 0;
  }
  if (d->layout != SAMD_NHWC) return 0;
  return conv2d_workspace_size(d, fa, fw);
}

samd_status samd_conv2d_set_min_tiles_per_cta(int tiles) {
  if (tiles < 1 || tiles > 1024) return SAMD_EINVAL;
  conv2d_set_min_tiles_per_cta(tiles);
  return SAMD_OK;
}

int samd_conv2d_operand_bits(const samd_conv_desc *d, samd_fmt fa, samd_fmt fw) {
  if (!d || !fmt_valid(fa) || !fmt_valid(fw) || fa.spacer != 0 || fw.spacer != 0) return 0;
  if (d->N < 0 || d->C < 1 || d->H < 1 || d->W < 1 || d->K < 1 || d->R < 1 || d->S < 1 || d->stride < 1 ||
      d->pad < 0 || d->R > 16 || d->S > 16)
    return 0;
  if (d->layout == SAMD_NCHW) return conv2d_nchw_check(d, fa, fw, samd_fmt{0, 0, 0, 0}, nullptr) == SAMD_OK ? 64 : 0;
  if (d->layout != SAMD_NHWC) return 0;
  return conv2d_operand_bits(d, fa, fw);
}

namespace {
// Checks shared by the three convolution entry points. fo.bits == 0 means no
// packed output format.
samd_status conv_common_checks(const samd_conv_desc *d, samd_fmt fa, samd_fmt fw, samd_fmt fo, int shift) {
  if (!d) return SAMD_EINVAL;
  if (!fmt_valid(fa) || !fmt_valid(fw)) return SAMD_EINVAL;
  if (fo.bits != 0 && !fmt_valid(fo)) return SAMD_EINVAL;
  if (shift < 0 || shift > 31) return SAMD_EINVAL;
  if (d->layout != SAMD_NHWC && d->layout != SAMD_NCHW) return SAMD_EINVAL;
  if (d->N < 0 || d->C < 1 || d->H < 1 || d->W < 1 || d->K < 1 || d->R < 1 || d->S < 1 || d->stride < 1 ||
      d->pad < 0)
    return SAMD_ESHAPE;
  if (d->H + 2 * d->pad < d->R || d->W + 2 * d->pad < d->S) return SAMD_ESHAPE;
  if (fa.spacer != 0 || fw.spacer != 0) return SAMD_EUNSUP;
  if (d->R > 16 || d->S > 16) return SAMD_EUNSUP;
  if (d->layout == SAMD_NCHW) return conv2d_nchw_check(d, fa, fw, fo, nullptr);  // wide-multiply engine limits
  return conv2d_check(d, fa, fw);  // exactness bound of the accumulation
}
}  // namespace

samd_status samd_conv2d(const samd_conv_desc *d, samd_fmt fa, const void *act, samd_fmt fw, const void *wt,
                        int32_t *acc_out, samd_fmt fo, void *packed_out, int shift, void *workspace,
                        size_t workspace_bytes, samd_stream_t stream) {
  if (!acc_out && !packed_out) return SAMD_EINVAL;
  const samd_fmt fplan = packed_out ? fo : samd_fmt{0, 0, 0, 0};
  samd_status st = conv_common_checks(d, fa, fw, fplan, packed_out ? shift : 0);
  if (st != SAMD_OK) return st;
  if (d->N == 0) return SAMD_OK;
  if (!act || !wt || !workspace) return SAMD_EINVAL;
  if (!aligned16(act) || !aligned16(wt) || !aligned16(workspace) || (acc_out && !aligned16(acc_out)) ||
      (packed_out && !aligned16(packed_out)))
    return SAMD_EALIGN;
  if (d->layout == SAMD_NCHW)
    return conv2d_nchw(d, fa, act, fw, wt, acc_out, fo, packed_out, shift, workspace, workspace_bytes,
                       reinterpret_cast<cudaStream_t>(stream));
  return conv2d_nhwc(d, fa, act, fw, wt, acc_out, fo, packed_out, shift, workspace, workspace_bytes,
                     reinterpret_cast<cudaStream_t>(stream));
}

samd_status samd_conv2d_noalloc(const samd_conv_desc *d, samd_fmt fa, const void *act, samd_fmt fw, const void *wt,
                                int32_t *acc_out, samd_fmt fo, void *packed_out, int shift, samd_stream_t stream) {
  if (!acc_out && !packed_out) return SAMD_EINVAL;
  const samd_fmt fplan = packed_out ? fo : samd_fmt{0, 0, 0, 0};
  samd_status st = conv_common_checks(d, fa, fw, fplan, packed_out ? shift : 0);
  if (st != SAMD_OK) return st;
  if (d->N == 0) return SAMD_OK;
  if (!act || !wt) return SAMD_EINVAL;
  if (!aligned16(act) || !aligned16(wt) || (acc_out && !aligned16(acc_out)) ||
      (packed_out && !aligned16(packed_out)))
    return SAMD_EALIGN;
  return conv2d_noalloc(d, fa, act, fw, wt, acc_out, fo, packed_out, shift,
                             reinterpret_cast<cudaStream_t>(stream));
}

samd_status samd_conv2d_prepare(const samd_conv_desc *d, samd_fmt fa, samd_fmt fw, const void *wt, samd_fmt fo,
                                void *prepared, size_t prepared_bytes, samd_stream_t stream) {
  samd_status st = conv_common_checks(d, fa, fw, fo, 0);
  if (st != SAMD_OK) return st;
  if (d->layout != SAMD_NHWC) return SAMD_EUNSUP;  // the NCHW engine widens its operands on every call
  if (!wt || !prepared) return SAMD_EINVAL;
  if (!aligned16(wt) || !aligned16(prepared)) return SAMD_EALIGN;
  return conv2d_prepare(d, fa, fw, wt, fo, prepared, prepared_bytes, reinterpret_cast<cudaStream_t>(stream));
}

samd_status samd_conv2d_prepared(const samd_conv_desc *d, samd_fmt fa, const void *act, samd_fmt fw,
                                 const void *prepared, size_t prepared_bytes, int32_t *acc_out, samd_fmt fo,
                                 void *packed_out, int shift, samd_stream_t stream) {
  if (!acc_out && !packed_out) return SAMD_EINVAL;
  if (packed_out && fo.bits == 0) return SAMD_EINVAL;
  samd_status st = conv_common_checks(d, fa, fw, fo, packed_out ? shift : 0);
  if (st != SAMD_OK) return st;
  if (d->layout != SAMD_NHWC) return SAMD_EUNSUP;
  if (d->N == 0) return SAMD_OK;
  if (!act || !prepared) return SAMD_EINVAL;
  if (!aligned16(act) || !aligned16(prepared) || (acc_out && !aligned16(acc_out)) ||
      (packed_out && !aligned16(packed_out)))
    return SAMD_EALIGN;
  return conv2d_run(d, fa, fw, act, prepared, prepared_bytes, acc_out, fo, packed_out, shift,
                    reinterpret_cast<cudaStream_t>(stream));
}

samd_status samd_conv2d_prepared_pool2x2(const samd_conv_desc *d, samd_fmt fa, const void *act, samd_fmt fw,
                                         const void *prepared, size_t prepared_bytes, samd_fmt fo, void *pooled_out,
                                         int shift, samd_stream_t stream) {
  if (!pooled_out || fo.bits == 0) return SAMD_EINVAL;
  samd_status st = conv_common_checks(d, fa, fw, fo, shift);
  if (st != SAMD_OK) return st;
  if (d->layout != SAMD_NHWC) return SAMD_EUNSUP;
  if (d->N == 0) return SAMD_OK;
  if (!conv2d_pool_supported(d, fa, fw, fo)) return SAMD_EUNSUP;
  if (!act || !prepared) return SAMD_EINVAL;
  if (!aligned16(act) || !aligned16(prepared) || !aligned16(pooled_out)) return SAMD_EALIGN;
  return conv2d_run(d, fa, fw, act, prepared, prepared_bytes, nullptr, fo, nullptr, shift,
                    reinterpret_cast<cudaStream_t>(stream), pooled_out);
}

int samd_conv2d_pool2x2_supported(const samd_conv_desc *d, samd_fmt fa, samd_fmt fw, samd_fmt fo) {
  if (!d || fo.bits == 0 || conv_common_checks(d, fa, fw, fo, 0) != SAMD_OK || d->layout != SAMD_NHWC) return 0;
  return conv2d_pool_supported(d, fa, fw, fo);
}

samd_status samd_maxpool2x2(samd_fmt f, const void *in, void *out, int N, int C, int H, int W, samd_layout layout,
                            samd_stream_t stream) {
  if (!fmt_valid(f)) return SAMD_EINVAL;
  if (layout != SAMD_NHWC && layout != SAMD_NCHW) return SAMD_EINVAL;
  if (N < 0 || C < 1 || H < 2 || W < 2 || (H & 1) || (W & 1)) return SAMD_ESHAPE;
  if (layout != SAMD_NHWC) return SAMD_EUNSUP;
  if (N == 0) return SAMD_OK;
  if (!in || !out) return SAMD_EINVAL;
  if (!aligned16(in) || !aligned16(out)) return SAMD_EALIGN;
  return from_cuda(launch_maxpool2x2_nhwc(f, in, out, N, C, H, W, reinterpret_cast<cudaStream_t>(stream)));
}

namespace {
constexpr int kMaxDim = 1 << 30;  // of a matrix product: the kernels' tile coordinates stay within an int

bool type16(samd_dtype t) { return t == SAMD_F16 || t == SAMD_BF16; }
bool act_ok(samd_act a) { return a >= SAMD_SILU && a <= SAMD_RELU_ACT; }

// Checks shared by the two matrix-vector calls; *empty: there is nothing to do.
samd_status matvec4_checks(const samd_matvec_desc *d, samd_fmt fw, const void *x, const samd_weights4 *w, int n_w,
                           const void *y, bool *empty) {
  *empty = false;
  if (!d || !type16(d->type) || !fmt_valid(fw)) return SAMD_EINVAL;
  if (d->group < 32 || (d->group & (d->group - 1)) != 0) return SAMD_EINVAL;
  if (fw.bits != 4 || fw.spacer != 0) return SAMD_EUNSUP;
  if (d->M < 0 || d->N < 0 || d->K < 1 || d->ldx < d->K || d->ldy < d->N) return SAMD_ESHAPE;
  if (d->M > kMaxDim || d->N > kMaxDim || d->K > kMaxDim) return SAMD_EUNSUP;
  *empty = d->M == 0 || d->N == 0;
  if (*empty) return SAMD_OK;
  if (!x || !y) return SAMD_EINVAL;
  for (int i = 0; i < n_w; ++i) {
    if (!w[i].lanes || !w[i].scales) return SAMD_EINVAL;
    if (w[i].zeros && fw.is_signed) return SAMD_EINVAL;
    if (!w[i].zeros != !w[0].zeros) return SAMD_EINVAL;
  }
  if (!aligned16(x) || !aligned16(y)) return SAMD_EALIGN;
  for (int i = 0; i < n_w; ++i)
    if (!aligned16(w[i].lanes) || !aligned16(w[i].scales) || !aligned16(w[i].zeros)) return SAMD_EALIGN;
  return SAMD_OK;
}

// Sizes and strides of the gated block.
samd_status ffn_shape_checks(const samd_ffn_desc *d) {
  if (!d || !type16(d->type) || !act_ok(d->act)) return SAMD_EINVAL;
  if (d->M < 0 || d->K < 1 || d->F < 1 || d->ldx < d->K || d->ldw < d->K || d->ldh < d->F) return SAMD_ESHAPE;
  if (d->ldx % 8 != 0 || d->ldw % 8 != 0 || d->ldh % 8 != 0) return SAMD_EALIGN;
  if (d->M > kMaxDim || d->K > kMaxDim || d->F > kMaxDim) return SAMD_EUNSUP;
  // tiles of an output are counted in an int, strides in bytes by the tensor maps in 40 bits
  const int64_t m = d->M / 128 + 1, k = d->K / 128 + 1, f = d->F / 128 + 1;
  if (m * f >= kMaxDim || m * k >= kMaxDim || 2 * f * k >= kMaxDim) return SAMD_EUNSUP;
  const int64_t ld = (int64_t(1) << 38);
  if (d->ldx >= ld || d->ldw >= ld || d->ldh >= ld) return SAMD_EUNSUP;
  return SAMD_OK;
}
}  // namespace

samd_status samd_matvec4(const samd_matvec_desc *d, samd_fmt fw, const void *x, samd_weights4 w, void *y,
                         samd_stream_t stream) {
  bool empty;
  const samd_status st = matvec4_checks(d, fw, x, &w, 1, y, &empty);
  if (st != SAMD_OK || empty) return st;
  return from_cuda(launch_matvec4(*d, -1, fw, x, w, nullptr, y, reinterpret_cast<cudaStream_t>(stream)));
}

samd_status samd_gated_matvec4(const samd_matvec_desc *d, samd_act act, samd_fmt fw, const void *x, samd_weights4 wg,
                               samd_weights4 wu, void *y, samd_stream_t stream) {
  if (!act_ok(act)) return SAMD_EINVAL;
  const samd_weights4 w[2] = {wg, wu};
  bool empty;
  const samd_status st = matvec4_checks(d, fw, x, w, 2, y, &empty);
  if (st != SAMD_OK || empty) return st;
  return from_cuda(launch_matvec4(*d, act, fw, x, wg, &wu, y, reinterpret_cast<cudaStream_t>(stream)));
}

samd_status samd_block8_quantize(samd_dtype type, const void *x, int64_t ldx, int64_t rows, int64_t inner,
                                 samd_block8 out, samd_stream_t stream) {
  if (!type16(type) && type != SAMD_F32) return SAMD_EINVAL;
  if (!shape_ok(rows, inner) || ldx < inner || (rows > 0 && ldx > INT64_MAX / 8 / rows)) return SAMD_ESHAPE;
  if (rows == 0 || inner == 0) return SAMD_OK;
  if (!x || !out.lanes || !out.exps) return SAMD_EINVAL;
  if (!aligned16(x) || !aligned16(out.lanes) || !aligned16(out.exps)) return SAMD_EALIGN;
  return from_cuda(launch_block8_quantize(type, x, ldx, rows, inner, out, reinterpret_cast<cudaStream_t>(stream)));
}

samd_status samd_block8_dequantize(samd_dtype type, samd_block8 in, int64_t rows, int64_t inner, void *y, int64_t ldy,
                                   samd_stream_t stream) {
  if (!type16(type) && type != SAMD_F32) return SAMD_EINVAL;
  if (!shape_ok(rows, inner) || ldy < inner || (rows > 0 && ldy > INT64_MAX / 8 / rows)) return SAMD_ESHAPE;
  if (rows == 0 || inner == 0) return SAMD_OK;
  if (!y || !in.lanes || !in.exps) return SAMD_EINVAL;
  if (!aligned16(y) || !aligned16(in.lanes) || !aligned16(in.exps)) return SAMD_EALIGN;
  return from_cuda(launch_block8_dequantize(type, in, rows, inner, y, ldy, reinterpret_cast<cudaStream_t>(stream)));
}

samd_status samd_gated_ffn_forward(const samd_ffn_desc *d, const void *x, const void *wg, const void *wu, void *h,
                                   samd_block8 cg, samd_block8 cu, samd_stream_t stream) {
  const samd_status st = ffn_shape_checks(d);
  if (st != SAMD_OK) return st;
  if (d->M == 0) return SAMD_OK;
  if (!x || !wg || !wu || !h) return SAMD_EINVAL;
  const bool keep = cg.lanes != nullptr;  // all four pointers, or none
  if ((cg.exps != nullptr) != keep || (cu.lanes != nullptr) != keep || (cu.exps != nullptr) != keep)
    return SAMD_EINVAL;
  if (!aligned16(x) || !aligned16(wg) || !aligned16(wu) || !aligned16(h) || !aligned16(cg.lanes) ||
      !aligned16(cg.exps) || !aligned16(cu.lanes) || !aligned16(cu.exps))
    return SAMD_EALIGN;
  return from_cuda(launch_ffn_forward(*d, x, wg, wu, h, cg, cu, reinterpret_cast<cudaStream_t>(stream)));
}

size_t samd_gated_ffn_backward_workspace_size(const samd_ffn_desc *d) {
  return ffn_shape_checks(d) == SAMD_OK ? ffn_backward_workspace(*d) : 0;
}

samd_status samd_gated_ffn_backward(const samd_ffn_desc *d, const void *dh, samd_block8 cx, samd_block8 cg,
                                    samd_block8 cu, const void *wg, const void *wu, void *dx, void *dwg, void *dwu,
                                    void *h, void *workspace, size_t workspace_bytes, samd_stream_t stream) {
  const samd_status st = ffn_shape_checks(d);
  if (st != SAMD_OK) return st;
  const bool weights = dwg || dwu;
  if (!aligned16(dx) || !aligned16(dwg) || !aligned16(dwu) || !aligned16(h)) return SAMD_EALIGN;
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (d->M == 0) {  // a sum over no tokens; dx and h have no rows, and may have no address
    for (void *w : {dwg, dwu})
      if (w && cudaMemset2DAsync(w, static_cast<size_t>(d->ldw) * 2, 0, static_cast<size_t>(d->K) * 2, d->F, s) !=
                   cudaSuccess)
        return SAMD_ECUDA;
    return SAMD_OK;
  }
  if (!dx && !weights && !h) return SAMD_EINVAL;
  if (!dh || !cg.lanes || !cg.exps || !cu.lanes || !cu.exps || !workspace) return SAMD_EINVAL;
  if ((dx && (!wg || !wu)) || (weights && (!cx.lanes || !cx.exps))) return SAMD_EINVAL;
  if (!aligned16(dh) || !aligned16(cx.lanes) || !aligned16(cx.exps) || !aligned16(cg.lanes) || !aligned16(cg.exps) ||
      !aligned16(cu.lanes) || !aligned16(cu.exps) || !aligned16(wg) || !aligned16(wu) || !aligned16(workspace))
    return SAMD_EALIGN;
  if (workspace_bytes < ffn_backward_workspace(*d)) return SAMD_ESHAPE;
  return from_cuda(launch_ffn_backward(*d, dh, cx, cg, cu, wg, wu, dx, dwg, dwu, h, workspace, s));
}

namespace {
// Tables, lengths, scores: arrays of 4-byte elements that callers cut out of larger ones.
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// A cache and the sequences in it, without the addresses.
samd_status cache_shape_checks(const samd_cache *c, const samd_cache_seqs *s) {
  if (!c || !s || !type16(c->type) || !fmt_valid(c->fmt)) return SAMD_EINVAL;
  if ((c->fmt.bits != 4 && c->fmt.bits != 8) || !c->fmt.is_signed || c->fmt.spacer != 0 || c->fmt.word_bits != 32)
    return SAMD_EUNSUP;
  if (c->pages < 0 || c->page < 1 || c->heads < 1 || c->dim < 1 || s->seqs < 0 || s->max_pages < 0 ||
      s->ld < s->max_pages)
    return SAMD_ESHAPE;
  if (c->page < 16 || c->page > 65536 || (c->page & (c->page - 1)) != 0 || c->dim % 32 != 0 || c->dim > 256 ||
      c->heads > 65536 || static_cast<int64_t>(c->heads) * c->page > kMaxDim)
    return SAMD_EUNSUP;
  // rows are counted in an int64, tokens of a sequence and pairs of a sequence and a head in an int
  const int64_t tokens = static_cast<int64_t>(s->max_pages) * c->page, rows = static_cast<int64_t>(s->seqs) * c->heads;
  if (tokens > kMaxDim || rows > kMaxDim || (tokens > 0 && rows > (int64_t(1) << 50) / tokens)) return SAMD_EUNSUP;
  return SAMD_OK;
}

samd_status cache_address_checks(const samd_cache *c, const samd_cache_seqs *s) {
  if (c->pages > 0 && (!c->k_lanes || !c->k_scales || !c->v_lanes || !c->v_scales)) return SAMD_EINVAL;
  if (!s->lengths || (!s->table && s->max_pages > 0)) return SAMD_EINVAL;
  if (!aligned16(c->k_lanes) || !aligned16(c->k_scales) || !aligned16(c->v_lanes) || !aligned16(c->v_scales) ||
      !aligned4(s->table) || !aligned4(s->lengths))
    return SAMD_EALIGN;
  return SAMD_OK;
}

// samd_cache_append and samd_cache_read; *empty: there is nothing to do.
samd_status cache_rows_checks(const samd_cache *c, const samd_cache_seqs *s, const int32_t *starts, int tokens,
                              const void *k, int64_t ldk, const void *v, int64_t ldv, bool *empty) {
  *empty = false;
  samd_status st = cache_shape_checks(c, s);
  if (st != SAMD_OK) return st;
  const int64_t row = static_cast<int64_t>(c->heads) * c->dim;
  if (tokens < 0 || ldk < row || ldv < row || (!starts && tokens != s->seqs)) return SAMD_ESHAPE;
  if (ldk % 8 != 0 || ldv % 8 != 0) return SAMD_EALIGN;
  if (tokens > 0 && (ldk > INT64_MAX / 8 / tokens || ldv > INT64_MAX / 8 / tokens)) return SAMD_ESHAPE;
  *empty = tokens == 0 || s->seqs == 0;
  if (*empty) return SAMD_OK;
  if (!k || !v) return SAMD_EINVAL;
  if (!aligned16(k) || !aligned16(v) || !aligned4(starts)) return SAMD_EALIGN;
  return cache_address_checks(c, s);
}

samd_status attention_shape_checks(const samd_cache *c, const samd_cache_seqs *s, int q_heads, bool scores) {
  const samd_status st = cache_shape_checks(c, s);
  if (st != SAMD_OK) return st;
  if (q_heads < 1 || q_heads % c->heads != 0) return SAMD_ESHAPE;
  if (q_heads / c->heads > 256 || static_cast<int64_t>(s->seqs) * q_heads > kMaxDim) return SAMD_EUNSUP;
  // the logits' bytes: up to 15 query heads' room for one
  const int64_t tokens = static_cast<int64_t>(s->max_pages) * c->page;
  if (scores && tokens > 0 && static_cast<int64_t>(s->seqs) * q_heads > (int64_t(1) << 50) / tokens) return SAMD_EUNSUP;
  return SAMD_OK;
}
}  // namespace

samd_status samd_cache_append(const samd_cache *c, const samd_cache_seqs *s, const int32_t *starts, int tokens,
                              const void *k, int64_t ldk, const void *v, int64_t ldv, samd_stream_t stream) {
  bool empty;
  const samd_status st = cache_rows_checks(c, s, starts, tokens, k, ldk, v, ldv, &empty);
  if (st != SAMD_OK || empty) return st;
  return from_cuda(launch_cache_append(*c, *s, starts, tokens, k, ldk, v, ldv, reinterpret_cast<cudaStream_t>(stream)));
}

samd_status samd_cache_read(const samd_cache *c, const samd_cache_seqs *s, const int32_t *starts, int tokens, void *k,
                            int64_t ldk, void *v, int64_t ldv, samd_stream_t stream) {
  bool empty;
  const samd_status st = cache_rows_checks(c, s, starts, tokens, k, ldk, v, ldv, &empty);
  if (st != SAMD_OK || empty) return st;
  return from_cuda(launch_cache_read(*c, *s, starts, tokens, k, ldk, v, ldv, reinterpret_cast<cudaStream_t>(stream)));
}

size_t samd_paged_attention_workspace_size(const samd_cache *c, const samd_cache_seqs *s, int q_heads, int scores) {
  if (attention_shape_checks(c, s, q_heads, scores != 0) != SAMD_OK || s->seqs == 0) return 0;
  return paged_attention_workspace(*c, *s, q_heads, scores != 0);
}

samd_status samd_paged_attention(const samd_cache *c, const samd_cache_seqs *s, int q_heads, const void *q,
                                 int64_t ldq, float scale, void *out, int64_t ldo, float *scores, int64_t ld_scores,
                                 void *workspace, size_t workspace_bytes, samd_stream_t stream) {
  samd_status st = attention_shape_checks(c, s, q_heads, scores != nullptr);
  if (st != SAMD_OK) return st;
  if (!(scale - scale == 0.0f)) return SAMD_EINVAL;
  const int64_t row = static_cast<int64_t>(q_heads) * c->dim;
  if (ldq < row || ldo < row || (scores && ld_scores < 0)) return SAMD_ESHAPE;
  if (ldq % 8 != 0 || ldo % 8 != 0) return SAMD_EALIGN;
  if (s->seqs > 0 && (ldq > INT64_MAX / 8 / s->seqs || ldo > INT64_MAX / 8 / s->seqs)) return SAMD_ESHAPE;
  if (scores && s->seqs > 0 && ld_scores > INT64_MAX / 8 / s->seqs / c->heads) return SAMD_ESHAPE;
  if (s->seqs == 0) return SAMD_OK;
  if (!q || !out) return SAMD_EINVAL;
  if (!aligned16(q) || !aligned16(out) || !aligned4(scores) || !aligned16(workspace)) return SAMD_EALIGN;
  st = cache_address_checks(c, s);
  if (st != SAMD_OK) return st;
  const size_t need = paged_attention_workspace(*c, *s, q_heads, scores != nullptr);
  if (need > 0 && !workspace) return SAMD_EINVAL;
  if (workspace_bytes < need) return SAMD_ESHAPE;
  return from_cuda(launch_paged_attention(*c, *s, q_heads, q, ldq, scale, out, ldo, scores, ld_scores, workspace,
                                          reinterpret_cast<cudaStream_t>(stream)));
}

samd_status samd_cache_evict(const samd_cache *c, const samd_cache_seqs *s, const float *scores, int64_t ld_scores,
                             int keep, int recent, const int32_t *dst_table, int64_t ld_dst, int32_t *kept,
                             int32_t *new_lengths, float *new_scores, samd_stream_t stream) {
  samd_status st = cache_shape_checks(c, s);
  if (st != SAMD_OK) return st;
  if (recent < 0 || recent > keep) return SAMD_EINVAL;
  if (keep < 1 || ld_scores < 0) return SAMD_ESHAPE;
  if (keep > kMaxDim) return SAMD_EUNSUP;
  const int dst_pages = (keep + c->page - 1) / c->page;
  if (ld_dst < dst_pages || (s->seqs > 0 && ld_scores > INT64_MAX / 8 / s->seqs / c->heads)) return SAMD_ESHAPE;
  // a launch's CTAs (a cluster a row) and the index of a row's unit
  if (static_cast<int64_t>(s->seqs) * c->heads > kMaxDim / 8) return SAMD_EUNSUP;
  if (s->seqs == 0) return SAMD_OK;
  if ((!scores && ld_scores > 0) || !dst_table || !kept || !new_lengths || dst_table == s->table) return SAMD_EINVAL;
  if (!aligned4(scores) || !aligned4(dst_table) || !aligned4(kept) || !aligned4(new_lengths) || !aligned4(new_scores))
    return SAMD_EALIGN;
  st = cache_address_checks(c, s);
  if (st != SAMD_OK) return st;
  const samd_cache_seqs dst = {s->seqs, dst_pages, ld_dst, dst_table, new_lengths};
  return from_cuda(launch_cache_evict(*c, *s, dst, scores, ld_scores, keep, recent, kept, new_lengths, new_scores,
                                      reinterpret_cast<cudaStream_t>(stream)));
}

namespace {
// Sizes of a layer of experts; route: those that samd_moe_route reads.
samd_status moe_shape_checks(const samd_moe_desc *d, bool route) {
  if (!d || !type16(d->type)) return SAMD_EINVAL;
  if (!route && (!act_ok(d->act) || d->group < 32 || (d->group & (d->group - 1)) != 0)) return SAMD_EINVAL;
  if (d->M < 0 || d->K < 1 || d->E < 1 || d->topk < 1 || d->ldx < d->K) return SAMD_ESHAPE;
  if (route && d->topk > d->E) return SAMD_ESHAPE;
  if (!route && (d->F < 1 || d->ldy < d->K)) return SAMD_ESHAPE;
  if (d->ldx % 8 != 0 || (!route && d->ldy % 8 != 0)) return SAMD_EALIGN;
  constexpr int kMost = 1 << 20;
  if (d->K % 32 != 0 || d->K > kMost || d->E > 1024 || d->topk > 32 || d->M > kMaxDim) return SAMD_EUNSUP;
  if (!route && (d->F % 32 != 0 || d->F > kMost)) return SAMD_EUNSUP;
  if (d->M > 0 && (d->ldx > INT64_MAX / 8 / d->M || (!route && d->ldy > INT64_MAX / 8 / d->M))) return SAMD_ESHAPE;
  return SAMD_OK;
}
}  // namespace

samd_status samd_moe_route(const samd_moe_desc *d, int normalize, const void *x, const void *router, int32_t *ids,
                           float *weights, samd_stream_t stream) {
  const samd_status st = moe_shape_checks(d, true);
  if (st != SAMD_OK) return st;
  if (normalize != 0 && normalize != 1) return SAMD_EINVAL;
  if (d->M == 0) return SAMD_OK;
  if (!x || !router || !ids || !weights) return SAMD_EINVAL;
  if (!aligned16(x) || !aligned16(router) || !aligned4(ids) || !aligned4(weights)) return SAMD_EALIGN;
  return from_cuda(launch_moe_route(*d, normalize != 0, x, router, ids, weights, reinterpret_cast<cudaStream_t>(stream)));
}

size_t samd_moe4_workspace_size(const samd_moe_desc *d) {
  return moe_shape_checks(d, false) == SAMD_OK ? moe4_workspace(*d) : 0;
}

samd_status samd_moe4(const samd_moe_desc *d, samd_fmt fw, const void *x, const int32_t *ids, const float *weights,
                      samd_weights4 gate, samd_weights4 up, samd_weights4 down, void *y, void *workspace,
                      size_t workspace_bytes, samd_stream_t stream) {
  if (!fmt_valid(fw)) return SAMD_EINVAL;
  const samd_status st = moe_shape_checks(d, false);
  if (st != SAMD_OK) return st;
  if (fw.bits != 4 || fw.spacer != 0) return SAMD_EUNSUP;
  if (d->M == 0) return SAMD_OK;
  if (!x || !ids || !weights || !y || !workspace) return SAMD_EINVAL;
  const samd_weights4 *const w[3] = {&gate, &up, &down};
  for (const samd_weights4 *m : w) {
    if (!m->lanes || !m->scales || (m->zeros && fw.is_signed) || !m->zeros != !gate.zeros) return SAMD_EINVAL;
  }
  for (const samd_weights4 *m : w)
    if (!aligned16(m->lanes) || !aligned16(m->scales) || !aligned16(m->zeros)) return SAMD_EALIGN;
  if (!aligned16(x) || !aligned16(y) || !aligned16(workspace) || !aligned4(ids) || !aligned4(weights)) return SAMD_EALIGN;
  if (workspace_bytes < moe4_workspace(*d)) return SAMD_ESHAPE;
  return from_cuda(launch_moe4(*d, fw, x, ids, weights, gate, up, down, y, workspace,
                               reinterpret_cast<cudaStream_t>(stream)));
}

samd_status samd_device_status(int *status, int reset, samd_stream_t stream) {
  if (!status) return SAMD_EINVAL;
  return from_cuda(read_device_status(status, reset, reinterpret_cast<cudaStream_t>(stream)));
}

samd_status samd_selftest_wait_timeout(uint64_t limit_ns, samd_stream_t stream) {
  if (limit_ns < 1000ull || limit_ns > 2000000000ull) return SAMD_EINVAL;
  return from_cuda(selftest_wait_timeout(limit_ns, reinterpret_cast<cudaStream_t>(stream)));
}

const char *samd_status_str(samd_status s) {
  switch (s) {
    case SAMD_OK: return "SAMD_OK";
    case SAMD_EINVAL: return "SAMD_EINVAL: invalid argument";
    case SAMD_EALIGN: return "SAMD_EALIGN: pointer not 16-byte aligned";
    case SAMD_ESHAPE: return "SAMD_ESHAPE: invalid or inconsistent sizes";
    case SAMD_EUNSUP: return "SAMD_EUNSUP: not supported by the kernels";
    case SAMD_ECUDA: return "SAMD_ECUDA: CUDA error";
    case SAMD_ETIMEOUT: return "SAMD_ETIMEOUT: a kernel gave up on a bounded wait";
  }
  return "unknown samd_status";
}

const char *samd_version(void) { return "samd-gb300 0.2 (sm_103a)"; }

}  // extern "C"
