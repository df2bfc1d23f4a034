// extern "C" entry points: argument validation on the host, then the kernel launchers.
#include "common.cuh"
#include "fp4.cuh"
#include "kv4.cuh"

namespace adadim {
int rtn_launch(const void* W, int wdtype, int64_t out, int64_t in, int64_t ldw, int bits, int group, int dim,
               const adadim_qtensor& qoc, const adadim_qtensor& qic, cudaStream_t st);
int unpack_launch(const uint32_t* codes, int64_t out, int64_t in, int bits, uint8_t* dst, cudaStream_t st);
int hessian_bf16_launch(const void* X, int64_t n_tokens, int64_t in, int64_t ldx, float* H, int* status_dev,
                        cudaStream_t st);
int hessian_f32_launch(const float* X, int64_t n_tokens, int64_t in, int64_t ldx, float* H, cudaStream_t st);
size_t hessian_f32_tc_workspace_bytes(int64_t n_tokens, int64_t in);
int hessian_f32_tc_launch(const float* X, int64_t n_tokens, int64_t in, int64_t ldx, float* H, int* status_dev,
                          void* workspace, cudaStream_t st);
size_t score_workspace_bytes(int64_t out, int64_t in);
int score_launch(const void* W, int wdtype, int64_t out, int64_t in, int64_t ldw, const float* H, int bits, int group,
                 const adadim_qtensor* q_oc, const adadim_qtensor* q_ic, double* err, int* chosen, int* status_dev,
                 void* workspace, cudaStream_t st);
size_t factor_workspace_bytes(int64_t n);
int factor_launch(const float* H, int64_t n, double percdamp, double* U, int* status_dev, void* workspace,
                  cudaStream_t st, const int* perm);
size_t gptq_workspace_bytes(int64_t rows, int64_t in);
struct GptqLayer {
  const void* W;
  int64_t out, ldw;
  const adadim_qtensor* q_oc;
  const adadim_qtensor* q_ic;
  int dim;
  const int* chosen;
  double* loss;
};
int gptq_launch(const GptqLayer* layers, int n_layers, int wdtype, int64_t in, const float* H, const double* U,
                int bits, int group, double percdamp, int* status_dev, void* workspace, cudaStream_t st, bool reorder,
                int* perm_out);

size_t gemv_workspace_bytes(int64_t out, int64_t in, int group);
int gemv_launch(const adadim_qtensor& q, int64_t out, int64_t in, int bits, int group, const void* x, void* y,
                void* workspace, cudaStream_t st);

namespace {

int check_weight(const void* W, int wdtype, int64_t out, int64_t in, int64_t ldw) {
  if (W == nullptr) return ADADIM_ERR_NULL;
  if (wdtype != ADADIM_F16 && wdtype != ADADIM_F32) return ADADIM_ERR_DTYPE;
  if (out < 0 || in < 0 || ldw < in) return ADADIM_ERR_SHAPE;
  const int64_t esz = wdtype == ADADIM_F16 ? 2 : 4;
  if (!aligned16(W) || (ldw * esz) % 16 != 0) return ADADIM_ERR_ALIGN;
  return ADADIM_OK;
}

// every entry point takes groups 32, 64, 128 and 256; at 256 GPTQ needs whole pairs of its 128-row
// slabs and 128-column blocks (out and in multiples of 256)
int check_quant_params(int bits, int group, bool allow_256) {
  if (bits != 2 && bits != 3 && bits != 4 && bits != 8) return ADADIM_ERR_PARAM;
  if (group != 32 && group != 64 && group != 128 && !(allow_256 && group == 256)) return ADADIM_ERR_PARAM;
  return ADADIM_OK;
}

constexpr int64_t kInt32Max = 0x7fffffff;

bool kv4_page_ok(int page) { return page >= kv4::kMinPage && page <= kv4::kMaxPage && (page & (page - 1)) == 0; }
constexpr int64_t kKv4Most = kInt32Max - 4095;   // tokens of a request, rows of a head
int check_kv4_sizes(const adadim_kv4cache& c) {
  if (!kv4_page_ok(c.page) || c.kv_heads < 1 || c.kv_heads > (1 << 16)) return ADADIM_ERR_PARAM;
  if (c.head_dim < 16 || c.head_dim > 256 || c.head_dim % 16 != 0) return ADADIM_ERR_PARAM;
  return c.n_pages < 0 || c.n_pages > kInt32Max / c.page ? ADADIM_ERR_SHAPE : ADADIM_OK;
}
int check_kv4(const adadim_kv4cache* c) {
  if (c == nullptr) return ADADIM_ERR_NULL;
  const int rc = check_kv4_sizes(*c);
  if (rc != ADADIM_OK) return rc;
  if (c->n_pages > 0 && (c->codes == nullptr || c->scales == nullptr)) return ADADIM_ERR_NULL;
  return aligned256(c->codes) && aligned256(c->scales) ? ADADIM_OK : ADADIM_ERR_ALIGN;
}
Kv4Heads heads_of(const adadim_heads& h) { return {h.p, h.ld, h.lh}; }

// Where heads of tokens lie, in bytes.
struct Place {
  const char* p;
  int64_t n, heads, ld, lh, width;
};
Place place_of(const adadim_heads& h, int64_t n, int64_t heads, int64_t dim, int64_t esz) {
  return {static_cast<const char*>(h.p), n, heads, n > 1 ? h.ld * esz : 0, heads > 1 ? h.lh * esz : 0, dim * esz};
}
bool same_place(const Place& a, const Place& b) { return a.p == b.p && a.ld == b.ld && a.lh == b.lh && a.width == b.width; }
// A token's heads, or two tokens, on top of one another: not all such orders are found, and none is that has room for every head.
bool folded(const Place& a) {
  const int64_t ld = a.ld < 0 ? -a.ld : a.ld, lh = a.lh < 0 ? -a.lh : a.lh;
  return (a.n > 1 && ld < a.width) || (a.heads > 1 && lh < a.width) || (a.n > 1 && a.heads > 1 && ld == lh);
}
int64_t gcd(int64_t a, int64_t b) {
  while (b != 0) { const int64_t r = a % b; a = b; b = r; }
  return a < 0 ? -a : a;
}
// Whether no byte belongs to both: their ranges are apart, or apart within the period of the tokens (columns of one matrix), of the
// heads (tokens inside heads), or of both (parts of every head).  False as well for orders that none of these tells apart.
bool apart(const Place& a, const Place& b) {
  typedef __int128 wide;
  struct Range { wide from, bytes; };
  const auto range = [](const Place& x, bool tokens, bool heads) {
    const wide t = tokens ? static_cast<wide>(x.n - 1) * x.ld : 0, h = heads ? static_cast<wide>(x.heads - 1) * x.lh : 0;
    return Range{static_cast<wide>(reinterpret_cast<uintptr_t>(x.p)) + (t < 0 ? t : 0) + (h < 0 ? h : 0), (t < 0 ? -t : t) + (h < 0 ? -h : h) + x.width};
  };
  const Range x = range(a, true, true), y = range(b, true, true);
  if (x.from + x.bytes <= y.from || y.from + y.bytes <= x.from) return true;
  const auto within = [](int64_t period, const Range& x, const Range& y) {
    if (period == 0) return false;
    wide s = (y.from - x.from) % period;
    if (s < 0) s += period;
    return s >= x.bytes && s + y.bytes <= period;
  };
  const int64_t tokens = gcd(a.ld, b.ld), heads = gcd(a.lh, b.lh);
  return within(tokens, range(a, false, true), range(b, false, true)) || within(heads, range(a, true, false), range(b, true, false)) ||
         within(gcd(tokens, heads), range(a, false, false), range(b, false, false));
}

int check_qtensor(const adadim_qtensor* q) {
  if (q == nullptr || q->codes == nullptr || q->scales == nullptr || q->zeros == nullptr) return ADADIM_ERR_NULL;
  if (!aligned16(q->codes) || !aligned16(q->scales) || !aligned16(q->zeros)) return ADADIM_ERR_ALIGN;
  return ADADIM_OK;
}

bool known_dtype(int dtype) { return dtype == ADADIM_F32 || dtype == ADADIM_F16 || dtype == ADADIM_BF16; }
int64_t dtype_size(int dtype) { return dtype == ADADIM_F32 ? 4 : 2; }

constexpr int64_t kFp4MaxIn = 1 << 20, kFp4MaxRows = 1 << 22;
constexpr int64_t kFp4MaxIndex = 0x7fffffff - (1 << 20);          // 32-bit coordinates, and a tile or a stage beyond the end

// A matrix of 16- or 32-bit elements: any row pitch, element-aligned.
int check_matrix(const void* X, int dtype, int64_t cols, int64_t ld) {
  if (!known_dtype(dtype)) return ADADIM_ERR_DTYPE;
  if (ld < cols || ld > (int64_t{1} << 40)) return ADADIM_ERR_SHAPE;
  if (X == nullptr) return ADADIM_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(X) % dtype_size(dtype) != 0) return ADADIM_ERR_ALIGN;
  return ADADIM_OK;
}
int check_fp4(const adadim_fp4tensor* q, int64_t cols) {
  if (q == nullptr || q->codes == nullptr || q->scales == nullptr) return ADADIM_ERR_NULL;
  if (q->ld < (cols + 1) / 2 || q->ld > (int64_t{1} << 30)) return ADADIM_ERR_SHAPE;
  if (!aligned16(q->codes) || q->ld % 16 != 0 || (reinterpret_cast<uintptr_t>(q->scales) & 127u) != 0) return ADADIM_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(q->amax) & 3u) != 0) return ADADIM_ERR_ALIGN;
  return ADADIM_OK;
}
int check_fp4_shape(int format, int64_t rows, int64_t cols) {
  if (format != ADADIM_MXFP4 && format != ADADIM_NVFP4) return ADADIM_ERR_PARAM;
  if (rows < 0 || cols < 0 || rows > kFp4MaxRows || cols > kFp4MaxIn) return ADADIM_ERR_SHAPE;
  return ADADIM_OK;
}
int check_groups(const int32_t* offsets, int n_groups) {
  if (n_groups < 0 || n_groups > fp4::kMaxGroups) return ADADIM_ERR_PARAM;
  if (n_groups == 0) return offsets == nullptr ? ADADIM_OK : ADADIM_ERR_PARAM;
  if (offsets == nullptr) return ADADIM_ERR_NULL;
  return (reinterpret_cast<uintptr_t>(offsets) & 3u) != 0 ? ADADIM_ERR_ALIGN : ADADIM_OK;
}
// The rules of a product's weight and result, shared by the four product entry points.  Returns
// ADADIM_OK with *empty set where there is nothing to compute.
int check_fp4_product(int64_t rows, int64_t out, int64_t in, int format, const int32_t* offsets, int n_experts,
                      const adadim_fp4tensor* B, const void* Y, int ydtype, int64_t ldy, bool* empty) {
  int rc = check_fp4_shape(format, rows, in);
  if (rc != ADADIM_OK) return rc;
  if (out < 0 || out > kFp4MaxRows) return ADADIM_ERR_SHAPE;
  if ((rc = check_groups(offsets, n_experts)) != ADADIM_OK) return rc;
  if (n_experts > 0 && out * n_experts > kFp4MaxIndex) return ADADIM_ERR_SHAPE;
  *empty = rows == 0 || out == 0;
  if (*empty) return ADADIM_OK;
  if (in == 0) return ADADIM_ERR_SHAPE;
  // tile numbers and scale rows are 32-bit in the kernel
  const int64_t tiles = ((rows + 15) / 16 + n_experts) * ((out + 127) / 128);
  const int64_t weights = n_experts > 0 ? n_experts : 1;
  const int64_t sf_rows = weights * static_cast<int64_t>(fp4::scale_bytes(format, out, in, 0)) / 128;
  const int64_t a_sf_rows = fp4_most_tile_rows(rows, n_experts) * fp4::sf_tiles(format, in) * 4;
  if (tiles > kFp4MaxIndex || sf_rows > kFp4MaxIndex || a_sf_rows > kFp4MaxIndex) return ADADIM_ERR_SHAPE;
  if ((rc = check_fp4(B, in)) != ADADIM_OK) return rc;
  return check_matrix(Y, ydtype, out, ldy);
}

// Workspace of the linear entry points: codes, then scale tiles, of the quantized activations.
size_t fp4_code_bytes(int64_t rows, int64_t in) { return round_up(static_cast<size_t>(rows) * fp4::code_pitch(in), 256); }
size_t fp4_workspace_bytes(int64_t rows, int64_t in, int n_groups) {
  // the scales of the finer format; the coarser one needs less
  return fp4_code_bytes(rows, in) +
         round_up(static_cast<size_t>(fp4_most_tile_rows(rows, n_groups)) * fp4::sf_tiles(ADADIM_NVFP4, in) * fp4::kSfTileBytes, 256);
}
bool fp4_fusable(bool aligned, int64_t in) { return aligned && in % fp4::kPer == 0; }
int fp4_linear(const void* X, int xdtype, int64_t x_rows, int64_t in, int64_t ldx, const float* x_amax,
               const int32_t* row_index, const int32_t* offsets, int n_experts, int64_t rows, const adadim_fp4tensor* B,
               int64_t out, int format, void* Y, int ydtype, int64_t ldy, int* status_dev, void* workspace,
               size_t workspace_bytes, cudaStream_t st) {
  bool empty = false;
  int rc = check_fp4_product(rows, out, in, format, offsets, n_experts, B, Y, ydtype, ldy, &empty);
  if (rc != ADADIM_OK || empty) return rc;
  if (x_rows < 0 || (row_index == nullptr && x_rows < rows)) return ADADIM_ERR_SHAPE;
  if (row_index == nullptr || x_rows > 0) {
    if ((rc = check_matrix(X, xdtype, in, ldx)) != ADADIM_OK) return rc;
  }
  if ((reinterpret_cast<uintptr_t>(row_index) & 3u) != 0 || (reinterpret_cast<uintptr_t>(x_amax) & 3u) != 0) return ADADIM_ERR_ALIGN;
  if (workspace == nullptr) return ADADIM_ERR_NULL;
  if (!aligned256(workspace)) return ADADIM_ERR_ALIGN;
  if (workspace_bytes < fp4_workspace_bytes(rows, in, n_experts)) return ADADIM_ERR_WORKSPACE;
  adadim_fp4tensor A;
  A.codes = static_cast<uint8_t*>(workspace);
  A.scales = A.codes + fp4_code_bytes(rows, in);
  A.amax = x_amax;
  A.ld = fp4::code_pitch(in);
  const fp4::Source x = fp4::source_of(X, xdtype, ldx, x_rows, in, row_index);
  const Fp4Plan plan = fp4_plan(rows, out, in, n_experts, format, false, fp4_fusable(xdtype == ydtype && x.wide != 0, in));
  if (!plan.fused) {
    rc = quantize_fp4_launch(x, xdtype, rows, in, format, offsets, n_experts, A, nullptr, plan.n_tile, nullptr, ADADIM_BF16, 0, st);
    if (rc != ADADIM_OK) return rc;
  }
  return fp4_matmul_launch(plan, A, plan.n_tile, x, rows, offsets, n_experts, *B, out, in, format, Y, ydtype, ldy, status_dev,
                           !plan.fused, st);
}

}  // namespace

int check_score_args(const void* W, int wdtype, int64_t out, int64_t in, int64_t ldw, const float* H, int bits,
                     int group, const adadim_qtensor* q_oc, const adadim_qtensor* q_ic, const double* err,
                     const int* chosen) {
  int rc = check_quant_params(bits, group, true);
  if (rc != ADADIM_OK) return rc;
  if (out <= 0 || in <= 0) return ADADIM_ERR_SHAPE;
  rc = check_weight(W, wdtype, out, in, ldw);
  if (rc != ADADIM_OK) return rc;
  if (in % 64 != 0 || out % 128 != 0) return ADADIM_ERR_SHAPE;
  if (q_oc == nullptr && q_ic == nullptr) return ADADIM_ERR_NULL;
  if (q_oc != nullptr && in % group != 0) return ADADIM_ERR_SHAPE;
  if (q_ic != nullptr && out % group != 0) return ADADIM_ERR_SHAPE;
  if (q_oc != nullptr && (rc = check_qtensor(q_oc)) != ADADIM_OK) return rc;
  if (q_ic != nullptr && (rc = check_qtensor(q_ic)) != ADADIM_OK) return rc;
  if (H == nullptr || err == nullptr || chosen == nullptr) return ADADIM_ERR_NULL;
  if (!aligned16(H)) return ADADIM_ERR_ALIGN;
  return ADADIM_OK;
}

}  // namespace adadim

using namespace adadim;

extern "C" {

int adadim_version(void) { return 100; }

const char* adadim_strerror(int status) {
  switch (status) {
    case ADADIM_OK: return "ok";
    case ADADIM_ERR_NULL: return "a required pointer is NULL";
    case ADADIM_ERR_SHAPE: return "a size is negative or violates a divisibility rule";
    case ADADIM_ERR_DTYPE: return "unsupported element type";
    case ADADIM_ERR_PARAM: return "bits, group, dim, percdamp or blocksize out of range";
    case ADADIM_ERR_ALIGN: return "pointer or leading dimension not suitably aligned";
    case ADADIM_ERR_WORKSPACE: return "workspace too small";
    case ADADIM_ERR_NOT_PD: return "damped Hessian is not positive definite";
    case ADADIM_ERR_NUMERIC: return "a reconstruction error is NaN";
    case ADADIM_ERR_TIMEOUT: return "an internal device-side wait exceeded its limit";
    case ADADIM_ERR_CUDA: return "a CUDA call failed";
    case ADADIM_ERR_PAGES: return "no free page left, or a page or block table out of range";
    default: return "unknown status";
  }
}

size_t adadim_workspace_bytes(int kind, int64_t out, int64_t in, int bits, int group) {
  (void)bits;
  if (out < 0 || in < 0) return 0;
  switch (kind) {
    case ADADIM_WS_HESSIAN: return out > 0 ? hessian_f32_tc_workspace_bytes(out, in) : 0;   // out = tokens of an fp32 chunk
    case ADADIM_WS_GPTQ: return gptq_workspace_bytes(2 * out, in);
    case ADADIM_WS_GPTQ_ROWS: return gptq_workspace_bytes(out, in);
    case ADADIM_WS_GEMV: return group > 0 ? gemv_workspace_bytes(out, in, group) : 0;
    case ADADIM_WS_SCORE: return score_workspace_bytes(out, in);
    case ADADIM_WS_FACTOR: return factor_workspace_bytes(in);
    case ADADIM_WS_FP4: return group >= 0 ? fp4_workspace_bytes(out, in, group) : 0;        // out = rows, group = experts
    default: return 0;
  }
}

int adadim_hessian_accumulate(const void* X, int xdtype, int64_t n_tokens, int64_t in, int64_t ldx, float* H,
                              int64_t* n_seen, int* status_dev, void* workspace, size_t workspace_bytes,
                              void* cuda_stream) {
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (xdtype != ADADIM_BF16 && xdtype != ADADIM_F32) return ADADIM_ERR_DTYPE;
  if (n_tokens < 0 || in < 0 || ldx < in || in % 8 != 0) return ADADIM_ERR_SHAPE;
  if (n_tokens > 0x7fffffff || in > (1 << 20)) return ADADIM_ERR_SHAPE;
  if (in == 0) return ADADIM_OK;
  if (H == nullptr) return ADADIM_ERR_NULL;
  if (!aligned16(H)) return ADADIM_ERR_ALIGN;
  if (n_tokens == 0) return ADADIM_OK;
  int rc = ADADIM_OK;
  if (X == nullptr) return ADADIM_ERR_NULL;
  const int64_t esz = xdtype == ADADIM_BF16 ? 2 : 4;
  if (!aligned16(X) || (ldx * esz) % 16 != 0) return ADADIM_ERR_ALIGN;
  if (xdtype == ADADIM_BF16) {
    rc = hessian_bf16_launch(X, n_tokens, in, ldx, H, status_dev, st);
  } else if (workspace != nullptr && aligned256(workspace) &&
             workspace_bytes >= hessian_f32_tc_workspace_bytes(n_tokens, in)) {
    rc = hessian_f32_tc_launch(static_cast<const float*>(X), n_tokens, in, ldx, H, status_dev, workspace, st);
  } else {
    rc = hessian_f32_launch(static_cast<const float*>(X), n_tokens, in, ldx, H, st);
  }
  if (rc == ADADIM_OK && n_seen != nullptr) *n_seen += n_tokens;
  return rc;
}

int adadim_quantize_rtn(const void* W, int wdtype, int64_t out, int64_t in, int64_t ldw, int bits, int group, int dim,
                        const adadim_qtensor* q_oc, const adadim_qtensor* q_ic, void* cuda_stream) {
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  int rc = check_quant_params(bits, group, true);
  if (rc != ADADIM_OK) return rc;
  if (dim != ADADIM_DIM_OC && dim != ADADIM_DIM_IC && dim != ADADIM_DIM_BOTH) return ADADIM_ERR_PARAM;
  if (out < 0 || in < 0) return ADADIM_ERR_SHAPE;
  if (out == 0 || in == 0) return ADADIM_OK;
  rc = check_weight(W, wdtype, out, in, ldw);
  if (rc != ADADIM_OK) return rc;
  if (in % 32 != 0) return ADADIM_ERR_SHAPE;
  const bool oc = dim != ADADIM_DIM_IC, ic = dim != ADADIM_DIM_OC;
  if (oc && in % group != 0) return ADADIM_ERR_SHAPE;
  if (ic && out % group != 0) return ADADIM_ERR_SHAPE;
  if (oc && (rc = check_qtensor(q_oc)) != ADADIM_OK) return rc;
  if (ic && (rc = check_qtensor(q_ic)) != ADADIM_OK) return rc;
  adadim_qtensor none = {nullptr, nullptr, nullptr};
  return rtn_launch(W, wdtype, out, in, ldw, bits, group, dim, oc ? *q_oc : none, ic ? *q_ic : none, st);
}

int adadim_cholesky_inverse_factor(const float* H, int64_t in, double percdamp, double* U, int* status_dev,
                                   void* workspace, size_t workspace_bytes, void* cuda_stream) {
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (in < 0 || in % 64 != 0) return ADADIM_ERR_SHAPE;
  if (!(percdamp >= 0.0) || !(percdamp < 1e6)) return ADADIM_ERR_PARAM;
  if (in == 0) return ADADIM_OK;
  if (H == nullptr || U == nullptr || workspace == nullptr) return ADADIM_ERR_NULL;
  if (!aligned16(H) || !aligned16(U) || !aligned256(workspace)) return ADADIM_ERR_ALIGN;
  if (workspace_bytes < factor_workspace_bytes(in)) return ADADIM_ERR_WORKSPACE;
  return factor_launch(H, in, percdamp, U, status_dev, workspace, st, nullptr);
}

int adadim_quantize_gptq(const void* W, int wdtype, int64_t out, int64_t in, int64_t ldw, const float* H,
                         const double* U, int bits, int group, int dim, double percdamp, int blocksize,
                         const adadim_qtensor* q_oc, const adadim_qtensor* q_ic, double* gptq_loss, int* status_dev,
                         void* workspace, size_t workspace_bytes, void* cuda_stream) {
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  int rc = check_quant_params(bits, group, true);
  if (rc != ADADIM_OK) return rc;
  if (dim != ADADIM_DIM_OC && dim != ADADIM_DIM_IC && dim != ADADIM_DIM_BOTH) return ADADIM_ERR_PARAM;
  if (blocksize != 128) return ADADIM_ERR_PARAM;
  if (!(percdamp >= 0.0) || !(percdamp < 1e6)) return ADADIM_ERR_PARAM;
  if (out < 0 || in < 0) return ADADIM_ERR_SHAPE;
  if (out == 0 || in == 0) return ADADIM_OK;
  rc = check_weight(W, wdtype, out, in, ldw);
  if (rc != ADADIM_OK) return rc;
  if (in % 128 != 0 || out % 128 != 0) return ADADIM_ERR_SHAPE;
  if (group == 256 && (in % 256 != 0 || out % 256 != 0)) return ADADIM_ERR_SHAPE;
  if (H == nullptr || workspace == nullptr) return ADADIM_ERR_NULL;
  if (!aligned16(H) || (U != nullptr && !aligned16(U)) || !aligned256(workspace)) return ADADIM_ERR_ALIGN;
  const bool oc = dim != ADADIM_DIM_IC, ic = dim != ADADIM_DIM_OC;
  if (oc && (rc = check_qtensor(q_oc)) != ADADIM_OK) return rc;
  if (ic && (rc = check_qtensor(q_ic)) != ADADIM_OK) return rc;
  if (workspace_bytes < gptq_workspace_bytes(2 * out, in)) return ADADIM_ERR_WORKSPACE;
  const GptqLayer layer = {W, out, ldw, q_oc, q_ic, dim, nullptr, gptq_loss};
  return gptq_launch(&layer, 1, wdtype, in, H, U, bits, group, percdamp, status_dev, workspace, st, false, nullptr);
}

int adadim_quantize_gptq_batched(const adadim_gptq_layer* layers, int n_layers, int wdtype, int64_t in, const float* H,
                                 const double* U, int bits, int group, double percdamp, int blocksize, int* status_dev,
                                 void* workspace, size_t workspace_bytes, void* cuda_stream) {
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  int rc = check_quant_params(bits, group, true);
  if (rc != ADADIM_OK) return rc;
  if (blocksize != 128) return ADADIM_ERR_PARAM;
  if (!(percdamp >= 0.0) || !(percdamp < 1e6)) return ADADIM_ERR_PARAM;
  if (n_layers < 0 || n_layers > ADADIM_MAX_BATCHED_LAYERS || in < 0) return ADADIM_ERR_SHAPE;
  if (n_layers == 0 || in == 0) return ADADIM_OK;
  if (layers == nullptr || H == nullptr || workspace == nullptr) return ADADIM_ERR_NULL;
  if (in % 128 != 0 || (group == 256 && in % 256 != 0)) return ADADIM_ERR_SHAPE;
  if (!aligned16(H) || (U != nullptr && !aligned16(U)) || !aligned256(workspace)) return ADADIM_ERR_ALIGN;
  GptqLayer ls[ADADIM_MAX_BATCHED_LAYERS];
  int64_t rows = 0;
  int copies = 0;
  for (int l = 0; l < n_layers; ++l) {
    const adadim_gptq_layer& y = layers[l];
    if (y.out <= 0 || y.out % 128 != 0 || (group == 256 && y.out % 256 != 0)) return ADADIM_ERR_SHAPE;
    rc = check_weight(y.W, wdtype, y.out, in, y.ldw);
    if (rc != ADADIM_OK) return rc;
    if (y.dim != ADADIM_DIM_OC && y.dim != ADADIM_DIM_IC && y.dim != ADADIM_DIM_BOTH && y.dim != ADADIM_DIM_CHOSEN)
      return ADADIM_ERR_PARAM;
    if (y.dim == ADADIM_DIM_CHOSEN && y.chosen == nullptr) return ADADIM_ERR_NULL;
    const bool oc = y.dim != ADADIM_DIM_IC, ic = y.dim != ADADIM_DIM_OC;
    if (oc && (rc = check_qtensor(y.q_oc)) != ADADIM_OK) return rc;
    if (ic && (rc = check_qtensor(y.q_ic)) != ADADIM_OK) return rc;
    const int nd = y.dim == ADADIM_DIM_BOTH ? 2 : 1;
    copies += nd;
    rows += nd * y.out;
    ls[l] = {y.W, y.out, y.ldw, y.q_oc, y.q_ic, y.dim, y.chosen, y.gptq_loss};
  }
  if (copies > ADADIM_MAX_BATCHED_LAYERS) return ADADIM_ERR_SHAPE;
  if (workspace_bytes < gptq_workspace_bytes(rows, in)) return ADADIM_ERR_WORKSPACE;
  return gptq_launch(ls, n_layers, wdtype, in, H, U, bits, group, percdamp, status_dev, workspace, st, false, nullptr);
}

int adadim_quantize_gptq_reordered(const void* W, int wdtype, int64_t out, int64_t in, int64_t ldw, const float* H,
                                   int bits, int group, int dim, double percdamp, int blocksize,
                                   const adadim_qtensor* q_oc, const adadim_qtensor* q_ic, double* gptq_loss,
                                   int32_t* perm_out, int* status_dev, void* workspace, size_t workspace_bytes,
                                   void* cuda_stream) {
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  int rc = check_quant_params(bits, group, true);
  if (rc != ADADIM_OK) return rc;
  if (dim != ADADIM_DIM_OC && dim != ADADIM_DIM_IC && dim != ADADIM_DIM_BOTH) return ADADIM_ERR_PARAM;
  if (blocksize != 128) return ADADIM_ERR_PARAM;
  if (!(percdamp >= 0.0) || !(percdamp < 1e6)) return ADADIM_ERR_PARAM;
  if (out < 0 || in < 0) return ADADIM_ERR_SHAPE;
  if (out == 0 || in == 0) return ADADIM_OK;
  rc = check_weight(W, wdtype, out, in, ldw);
  if (rc != ADADIM_OK) return rc;
  if (in % 128 != 0 || out % 128 != 0) return ADADIM_ERR_SHAPE;
  if (group == 256 && (in % 256 != 0 || out % 256 != 0)) return ADADIM_ERR_SHAPE;
  if (H == nullptr || workspace == nullptr) return ADADIM_ERR_NULL;
  if (!aligned16(H) || !aligned256(workspace)) return ADADIM_ERR_ALIGN;
  const bool oc = dim != ADADIM_DIM_IC, ic = dim != ADADIM_DIM_OC;
  if (oc && (rc = check_qtensor(q_oc)) != ADADIM_OK) return rc;
  if (ic && (rc = check_qtensor(q_ic)) != ADADIM_OK) return rc;
  if (workspace_bytes < gptq_workspace_bytes(2 * out, in)) return ADADIM_ERR_WORKSPACE;
  const GptqLayer layer = {W, out, ldw, q_oc, q_ic, dim, nullptr, gptq_loss};
  return gptq_launch(&layer, 1, wdtype, in, H, nullptr, bits, group, percdamp, status_dev, workspace, st, true,
                     perm_out);
}

int adadim_score_select(const void* W, int wdtype, int64_t out, int64_t in, int64_t ldw, const float* H, int bits,
                        int group, const adadim_qtensor* q_oc, const adadim_qtensor* q_ic, double* err, int* chosen,
                        int* status_dev, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const int rc = check_score_args(W, wdtype, out, in, ldw, H, bits, group, q_oc, q_ic, err, chosen);
  if (rc != ADADIM_OK) return rc;
  if (workspace == nullptr) return ADADIM_ERR_NULL;
  if (!aligned256(workspace)) return ADADIM_ERR_ALIGN;
  if (workspace_bytes < score_workspace_bytes(out, in)) return ADADIM_ERR_WORKSPACE;
  return score_launch(W, wdtype, out, in, ldw, H, bits, group, q_oc, q_ic, err, chosen, status_dev, workspace, st);
}

int adadim_dequant_gemv(const adadim_qtensor* q, int dim, int64_t out, int64_t in, int bits, int group, const void* x,
                        void* y, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (bits != 3 && bits != 4) return ADADIM_ERR_PARAM;
  if (dim != ADADIM_DIM_IC) return ADADIM_ERR_PARAM;
  if (group < 16 || group % 16 != 0) return ADADIM_ERR_PARAM;
  if (out < 0 || in < 0) return ADADIM_ERR_SHAPE;
  if (out == 0 || in == 0) return ADADIM_OK;
  if (out % group != 0 || in % 128 != 0) return ADADIM_ERR_SHAPE;
  int rc = check_qtensor(q);
  if (rc != ADADIM_OK) return rc;
  if (x == nullptr || y == nullptr || workspace == nullptr) return ADADIM_ERR_NULL;
  if (!aligned16(x) || !aligned256(workspace) || (reinterpret_cast<uintptr_t>(y) & 1u) != 0) return ADADIM_ERR_ALIGN;
  if (workspace_bytes < gemv_workspace_bytes(out, in, group)) return ADADIM_ERR_WORKSPACE;
  return gemv_launch(*q, out, in, bits, group, x, y, workspace, static_cast<cudaStream_t>(cuda_stream));
}

size_t adadim_fp4_scale_bytes(int format, int64_t rows, int64_t cols, int n_groups) {
  if (check_fp4_shape(format, rows, cols) != ADADIM_OK || n_groups < 0 || n_groups > fp4::kMaxGroups) return 0;
  return fp4::scale_bytes(format, rows, cols, n_groups);
}

int adadim_absmax(const void* X, int xdtype, int64_t rows, int64_t cols, int64_t ldx, float* amax, void* cuda_stream) {
  if (!known_dtype(xdtype)) return ADADIM_ERR_DTYPE;
  if (rows < 0 || cols < 0) return ADADIM_ERR_SHAPE;
  if (rows == 0 || cols == 0) return ADADIM_OK;
  if (cols > (int64_t{1} << 60) / rows) return ADADIM_ERR_SHAPE;
  const int rc = check_matrix(X, xdtype, cols, ldx);
  if (rc != ADADIM_OK) return rc;
  if (amax == nullptr) return ADADIM_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(amax) & 3u) != 0) return ADADIM_ERR_ALIGN;
  return absmax_launch(X, xdtype, rows, cols, ldx, amax, static_cast<cudaStream_t>(cuda_stream));
}

int adadim_quantize_fp4(const void* X, int xdtype, int64_t rows, int64_t cols, int64_t ldx, int64_t x_rows, int format,
                        const int32_t* row_index, const int32_t* offsets, int n_groups, const adadim_fp4tensor* q,
                        void* values, int vdtype, int64_t ldv, void* cuda_stream) {
  return adadim_quantize_fp4_amax(X, xdtype, rows, cols, ldx, x_rows, format, row_index, offsets, n_groups, q, values, vdtype,
                                  ldv, nullptr, cuda_stream);
}

int adadim_quantize_fp4_amax(const void* X, int xdtype, int64_t rows, int64_t cols, int64_t ldx, int64_t x_rows, int format,
                             const int32_t* row_index, const int32_t* offsets, int n_groups, const adadim_fp4tensor* q,
                             void* values, int vdtype, int64_t ldv, const float* amax, void* cuda_stream) {
  int rc = check_fp4_shape(format, rows, cols);
  if (rc != ADADIM_OK) return rc;
  if (!known_dtype(xdtype) || (values != nullptr && vdtype != ADADIM_BF16 && vdtype != ADADIM_F32)) return ADADIM_ERR_DTYPE;
  if ((rc = check_groups(offsets, n_groups)) != ADADIM_OK) return rc;
  if (rows == 0 || cols == 0) return ADADIM_OK;
  if (x_rows < 0 || (row_index == nullptr && x_rows < rows)) return ADADIM_ERR_SHAPE;
  if (x_rows > 0 && (rc = check_matrix(X, xdtype, cols, ldx)) != ADADIM_OK) return rc;
  if ((reinterpret_cast<uintptr_t>(row_index) & 3u) != 0) return ADADIM_ERR_ALIGN;
  if ((rc = check_fp4(q, cols)) != ADADIM_OK) return rc;
  if ((reinterpret_cast<uintptr_t>(amax) & 3u) != 0) return ADADIM_ERR_ALIGN;
  if (format == ADADIM_NVFP4 && amax != nullptr && q->amax == nullptr) return ADADIM_ERR_NULL;
  if (values != nullptr && (rc = check_matrix(values, vdtype, cols, ldv)) != ADADIM_OK) return rc;
  return quantize_fp4_launch(fp4::source_of(X, xdtype, ldx, x_rows, cols, row_index), xdtype, rows, cols, format, offsets,
                             n_groups, *q, amax, fp4::kSfRows, values, vdtype, ldv, static_cast<cudaStream_t>(cuda_stream));
}

int adadim_fp4_matmul(const adadim_fp4tensor* A, int64_t n_tokens, const adadim_fp4tensor* B, int64_t out, int64_t in,
                      int format, void* Y, int ydtype, int64_t ldy, int* status_dev, void* cuda_stream) {
  bool empty = false;
  int rc = check_fp4_product(n_tokens, out, in, format, nullptr, 0, B, Y, ydtype, ldy, &empty);
  if (rc != ADADIM_OK || empty) return rc;
  if ((rc = check_fp4(A, in)) != ADADIM_OK) return rc;
  return fp4_matmul_launch(fp4_plan(n_tokens, out, in, 0, format, true, false), *A, fp4::kSfRows, {}, n_tokens, nullptr, 0, *B, out,
                           in, format, Y, ydtype, ldy, status_dev, false, static_cast<cudaStream_t>(cuda_stream));
}

int adadim_fp4_matmul_grouped(const adadim_fp4tensor* A, int64_t n_rows, const int32_t* offsets, int n_experts,
                              const adadim_fp4tensor* B, int64_t out, int64_t in, int format, void* Y, int ydtype,
                              int64_t ldy, int* status_dev, void* cuda_stream) {
  if (n_experts == 0) return ADADIM_ERR_PARAM;
  bool empty = false;
  int rc = check_fp4_product(n_rows, out, in, format, offsets, n_experts, B, Y, ydtype, ldy, &empty);
  if (rc != ADADIM_OK || empty) return rc;
  if ((rc = check_fp4(A, in)) != ADADIM_OK) return rc;
  return fp4_matmul_launch(fp4_plan(n_rows, out, in, n_experts, format, true, false), *A, fp4::kSfRows, {}, n_rows, offsets, n_experts,
                           *B, out, in, format, Y, ydtype, ldy, status_dev, false, static_cast<cudaStream_t>(cuda_stream));
}

int adadim_fp4_linear(const void* X, int xdtype, int64_t n_tokens, int64_t in, int64_t ldx, const float* x_amax,
                      const adadim_fp4tensor* B, int64_t out, int format, void* Y, int ydtype, int64_t ldy,
                      int* status_dev, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  return fp4_linear(X, xdtype, n_tokens, in, ldx, x_amax, nullptr, nullptr, 0, n_tokens, B, out, format, Y, ydtype, ldy,
                    status_dev, workspace, workspace_bytes, static_cast<cudaStream_t>(cuda_stream));
}

int adadim_fp4_linear_grouped(const void* X, int xdtype, int64_t x_rows, int64_t in, int64_t ldx, const float* x_amax,
                              const int32_t* row_index, const int32_t* offsets, int n_experts, int64_t n_rows,
                              const adadim_fp4tensor* B, int64_t out, int format, void* Y, int ydtype, int64_t ldy,
                              int* status_dev, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (n_experts == 0) return ADADIM_ERR_PARAM;
  return fp4_linear(X, xdtype, x_rows, in, ldx, x_amax, row_index, offsets, n_experts, n_rows, B, out, format, Y, ydtype,
                    ldy, status_dev, workspace, workspace_bytes, static_cast<cudaStream_t>(cuda_stream));
}

int adadim_fp4_plan(int64_t rows, int64_t out, int64_t in, int n_experts, int format, int quantized, int aligned, int* plan) {
  const int rc = check_fp4_shape(format, rows, in);
  if (rc != ADADIM_OK) return rc;
  if (rows == 0 || out <= 0 || out > kFp4MaxRows || in == 0) return ADADIM_ERR_SHAPE;
  if (n_experts < 0 || n_experts > fp4::kMaxGroups) return ADADIM_ERR_PARAM;
  if (plan == nullptr) return ADADIM_ERR_NULL;
  const Fp4Plan p = fp4_plan(rows, out, in, n_experts, format, quantized != 0, fp4_fusable(quantized == 0 && aligned != 0, in));
  const int v[5] = {p.pair, p.n_tile, p.splits, p.per_sm, p.fused};
  for (int k = 0; k < 5; ++k) plan[k] = v[k];
  return ADADIM_OK;
}

size_t adadim_kv4_bytes(int64_t n_pages, int page, int kv_heads, int head_dim, int what) {
  const adadim_kv4cache c = {nullptr, nullptr, nullptr, n_pages, page, kv_heads, head_dim};
  if (check_kv4_sizes(c) != ADADIM_OK || (what != 0 && what != 1)) return 0;
  return static_cast<size_t>(n_pages) * 2 * kv_heads * page * (kv4::held_dim(head_dim) / (what == 0 ? 2 : 16));
}

int adadim_page_tables(const int32_t* past, const int32_t* fresh, int64_t n_requests, int page, int32_t* table, int64_t ldt,
                       int64_t width, const int32_t* free_pages, int64_t n_free, const int32_t* cursor, int64_t rows,
                       int32_t* lengths, int32_t* offsets, int32_t* requests, int32_t* positions, int32_t* slots, int32_t* next,
                       int* status_dev, void* cuda_stream) {
  if (!kv4_page_ok(page)) return ADADIM_ERR_PARAM;
  if (n_requests < 0 || n_requests > kv4::kMaxRequests || width < 0 || ldt < width || n_free < 0 || rows < 0) return ADADIM_ERR_SHAPE;
  if (n_free > kInt32Max || rows > kInt32Max || width > kInt32Max || ldt > (int64_t{1} << 40)) return ADADIM_ERR_SHAPE;
  if (offsets == nullptr || next == nullptr || next == cursor) return ADADIM_ERR_NULL;
  if (n_requests > 0 && (past == nullptr || fresh == nullptr || lengths == nullptr || (width > 0 && table == nullptr))) return ADADIM_ERR_NULL;
  if (n_free > 0 && free_pages == nullptr) return ADADIM_ERR_NULL;
  if (rows > 0 && (requests == nullptr || positions == nullptr || slots == nullptr)) return ADADIM_ERR_NULL;
  {
    // Some CTAs still read what others have written by then.
    struct Ints { const int32_t* p; int64_t n; };
    const Ints read[] = {{past, n_requests}, {fresh, n_requests}, {free_pages, n_free}, {cursor, cursor != nullptr}};
    const Ints written[] = {{lengths, n_requests}, {offsets, n_requests + 1}, {requests, rows}, {positions, rows}, {slots, rows}, {next, 1}};
    const Place whole = {reinterpret_cast<const char*>(table), n_requests, 1, n_requests > 1 ? ldt * 4 : 0, 0, width * 4};
    const auto clear = [](const Ints& a, const Ints& b) {
      const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
      return a.n == 0 || b.n == 0 || x + 4 * a.n <= y || y + 4 * b.n <= x;
    };
    const Ints all_rows = {table, n_requests == 0 || width == 0 ? 0 : (n_requests - 1) * ldt + width};
    const auto beside_table = [&](const Ints& a) {                   // in front, behind, or between the used entries of two rows
      return clear(all_rows, a) || apart(whole, Place{reinterpret_cast<const char*>(a.p), 1, 1, 0, 0, 4 * a.n});
    };
    for (const Ints& a : read)
      if (!beside_table(a)) return ADADIM_ERR_PARAM;
    for (const Ints& a : written) {
      if (!beside_table(a)) return ADADIM_ERR_PARAM;
      for (const Ints& b : read) if (!clear(a, b)) return ADADIM_ERR_PARAM;
      for (const Ints& b : written) if (&a != &b && !clear(a, b)) return ADADIM_ERR_PARAM;
    }
  }
  return page_tables_launch(past, fresh, static_cast<int>(n_requests), page, table, ldt, width, free_pages, static_cast<int>(n_free),
                            cursor, static_cast<int>(rows), lengths, offsets, requests, positions, slots, next, status_dev,
                            static_cast<cudaStream_t>(cuda_stream));
}

int adadim_kv4_append(const adadim_heads* heads, int q_heads, int dtype, int64_t n_tokens, const int32_t* slots,
                      const adadim_rotary* rotary, const adadim_kv4cache* cache, int vdtype, void* cuda_stream) {
  int rc = check_kv4(cache);
  if (rc != ADADIM_OK) return rc;
  if (heads == nullptr) return ADADIM_ERR_NULL;
  const adadim_heads &K = heads[0], &V = heads[1], &Q = heads[2], &Qr = heads[3];
  if (dtype != ADADIM_F32 && dtype != ADADIM_F16 && dtype != ADADIM_BF16) return ADADIM_ERR_DTYPE;
  if ((heads[4].p != nullptr || heads[5].p != nullptr) && vdtype != ADADIM_F32 && vdtype != ADADIM_BF16) return ADADIM_ERR_DTYPE;
  if (n_tokens < 0 || n_tokens > kInt32Max || q_heads < 0 || q_heads > (1 << 16)) return ADADIM_ERR_SHAPE;
  if (rotary != nullptr) {
    if (rotary->axes < 1 || rotary->dim < 8 || rotary->dim > cache->head_dim || rotary->dim % 8 != 0) return ADADIM_ERR_PARAM;
    if (n_tokens > 0 && (rotary->positions == nullptr || rotary->freq == nullptr)) return ADADIM_ERR_NULL;
    if (rotary->axes > 1 && rotary->axis == nullptr) return ADADIM_ERR_NULL;
  }
  if (n_tokens == 0) return ADADIM_OK;
  if ((Q.p == nullptr) != (Qr.p == nullptr)) return ADADIM_ERR_NULL;
  if (Q.p != nullptr && rotary == nullptr) return ADADIM_ERR_PARAM;
  if (K.p == nullptr || V.p == nullptr) return ADADIM_ERR_NULL;
  {
    // What is written lies in memory of its own, or where each thread's numbers come from: a turned key with halves as pairs has its
    // partner's place read by another thread.
    const int64_t esz = dtype == ADADIM_F32 ? 4 : 2, vsz = vdtype == ADADIM_F32 ? 4 : 2, d = cache->head_dim, h = cache->kv_heads;
    const Place k = place_of(K, n_tokens, h, d, esz), v = place_of(V, n_tokens, h, d, esz), q = place_of(Q, n_tokens, q_heads, d, esz);
    const Place to_q = place_of(Qr, n_tokens, q_heads, d, esz), to_k = place_of(heads[4], n_tokens, h, d, vsz), to_v = place_of(heads[5], n_tokens, h, d, vsz);
    const auto clear = [](const Place& to, const Place& from) { return to.p == nullptr || from.p == nullptr || apart(to, from); };
    const bool whole_keys = rotary == nullptr || rotary->adjacent != 0;
    for (const Place& to : {to_q, to_k, to_v})
      if (to.p != nullptr && folded(to)) return ADADIM_ERR_PARAM;
    if (!(clear(to_q, q) || same_place(to_q, q)) || !clear(to_q, k) || !clear(to_q, v)) return ADADIM_ERR_PARAM;
    if (!(clear(to_k, k) || (whole_keys && same_place(to_k, k))) || !clear(to_k, v) || !clear(to_k, q)) return ADADIM_ERR_PARAM;
    if (!(clear(to_v, v) || same_place(to_v, v)) || !clear(to_v, k) || !clear(to_v, q)) return ADADIM_ERR_PARAM;
    if (!clear(to_q, to_k) || !clear(to_q, to_v) || !clear(to_k, to_v)) return ADADIM_ERR_PARAM;
  }
  if (slots == nullptr) return ADADIM_ERR_NULL;
  const Kv4Rotary still = {nullptr, nullptr, nullptr, 0, 1, 0, 0};
  return kv4_append_launch(heads_of(Q), heads_of(Qr), Q.p == nullptr ? 0 : q_heads, heads_of(K), heads_of(V), dtype, n_tokens, slots,
                           rotary == nullptr ? still : Kv4Rotary{rotary->positions, rotary->freq, rotary->axis, rotary->ld, rotary->axes,
                                                                rotary->dim, rotary->adjacent},
                           kv4::cache_of(*cache), heads_of(heads[4]), heads_of(heads[5]), vdtype, static_cast<cudaStream_t>(cuda_stream));
}

size_t adadim_kv4_workspace_bytes(int64_t n_requests, int64_t n_rows, int q_heads, int kv_heads, int head_dim) {
  if (n_requests < 0 || n_rows < 0 || kv_heads < 1 || q_heads < kv_heads || head_dim < 16 || head_dim > 256) return 0;
  return kv4_workspace(n_requests, n_rows, q_heads, kv_heads, head_dim);
}

int adadim_kv4_attention(const adadim_heads* qo, int dtype, int64_t n_rows, int q_heads, const int32_t* offsets, const int32_t* lengths,
                         int64_t n_requests, const int32_t* table, int64_t ldt, int64_t width, const adadim_kv4cache* cache, float scale,
                         int causal, int64_t window, int64_t max_new, int* status_dev, void* workspace,
                         size_t workspace_bytes, void* cuda_stream) {
  int rc = check_kv4(cache);
  if (rc != ADADIM_OK) return rc;
  if (dtype != ADADIM_F16 && dtype != ADADIM_BF16) return ADADIM_ERR_DTYPE;
  if (q_heads < 1 || q_heads > (1 << 16) || q_heads % cache->kv_heads != 0) return ADADIM_ERR_PARAM;
  if (window < 0 || max_new < 0) return ADADIM_ERR_PARAM;
  // the kernels count tokens and rows in 32 bits, up to a chunk or a tile beyond the last one
  if (n_rows < 0 || n_rows > kKv4Most / q_heads || n_requests < 0 || n_requests > kv4::kMaxRequests || width < 0 || ldt < width ||
      width > kKv4Most / cache->page)
    return ADADIM_ERR_SHAPE;
  if (window >= width * cache->page) window = 0;                     // as long as any request may be
  // rows may stand in front of token 0, and see tokens where they are not causal: the window's begin, up to rows + window in front of it
  if (causal == 0 && window > 0 && n_rows > kKv4Most - window) return ADADIM_ERR_SHAPE;
  if (n_rows == 0 || n_requests == 0) return ADADIM_OK;
  if (qo == nullptr || qo[0].p == nullptr || qo[1].p == nullptr || offsets == nullptr || lengths == nullptr || (width > 0 && table == nullptr))
    return ADADIM_ERR_NULL;
  {
    // a row's results are written when its queries have been read, other rows' have not
    const Place q = place_of(qo[0], n_rows, q_heads, cache->head_dim, 2), o = place_of(qo[1], n_rows, q_heads, cache->head_dim, 2);
    if (folded(o) || !(same_place(q, o) || apart(q, o))) return ADADIM_ERR_PARAM;
  }
  if (workspace == nullptr) return ADADIM_ERR_NULL;
  if (!aligned256(workspace)) return ADADIM_ERR_ALIGN;
  if (workspace_bytes < adadim_kv4_workspace_bytes(n_requests, n_rows, q_heads, cache->kv_heads, cache->head_dim)) return ADADIM_ERR_WORKSPACE;
  Kv4Attention a = {};
  a.q = heads_of(qo[0]);
  a.o = heads_of(qo[1]);
  a.n_rows = static_cast<int>(n_rows);
  a.q_heads = q_heads;
  a.group = q_heads / cache->kv_heads;
  a.offsets = offsets;
  a.lengths = lengths;
  a.table = table;
  a.n_requests = static_cast<int>(n_requests);
  a.ldt = ldt;
  a.width = width;
  a.cache = kv4::cache_of(*cache);
  a.scale = scale;
  a.causal = causal != 0;
  a.window = static_cast<int>(window);
  a.status_dev = status_dev;
  a.workspace = static_cast<char*>(workspace);
  return kv4_attention_launch(a, dtype, max_new == 0 || max_new > n_rows ? n_rows : max_new, static_cast<cudaStream_t>(cuda_stream));
}

int adadim_unpack_codes(const uint32_t* codes, int64_t out, int64_t in, int bits, uint8_t* dst, void* cuda_stream) {
  if (bits != 2 && bits != 3 && bits != 4 && bits != 8) return ADADIM_ERR_PARAM;
  if (out < 0 || in < 0 || in % 32 != 0) return ADADIM_ERR_SHAPE;
  if (out == 0 || in == 0) return ADADIM_OK;
  if (codes == nullptr || dst == nullptr) return ADADIM_ERR_NULL;
  if (!aligned16(dst)) return ADADIM_ERR_ALIGN;
  return unpack_launch(codes, out, in, bits, dst, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
