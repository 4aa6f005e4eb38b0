// C ABI of the 8-bit linear layer's operators (declared in include/prm.h):
// argument checks, workspace layout and launches.  No state of their own.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/prm.h"
#include "ops_internal.h"

using namespace prm;

namespace {

constexpr int64_t kMaxCols = 1ll << 24, kMaxRows = (1ll << 31) - 1, kMaxColRows = 1ll << 22;

int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  return set_error(code, buf);
}

int check_type(int32_t t) {
  return t == PRM_F32 || t == PRM_BF16 || t == PRM_F16 ? PRM_OK : fail(PRM_EDTYPE, "unsupported dtype %d", t);
}
int64_t size_of(int32_t t) { return t == PRM_F32 ? 4 : 2; }

struct Buf {
  const void* p;
  const char* name;
  int64_t align;
};

// Every buffer is memory of the current device, on its element's boundary.
template <int N>
int check_buffers(const char* call, const Buf (&b)[N]) {
  for (int i = 0; i < N; ++i) {
    if (!b[i].name) continue;  // an optional one that is not there
    if (!b[i].p) return fail(PRM_EINVAL, "%s: %s is NULL", call, b[i].name);
    if ((uintptr_t)b[i].p % b[i].align)
      return fail(PRM_EALIGN, "%s: %s is not %lld-byte aligned", call, b[i].name, (long long)b[i].align);
  }
  int dev = 0;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return fail(PRM_EHIP, "hipGetDevice failed: %s", hipGetErrorString(e));
  for (int i = 0; i < N; ++i)
    if (b[i].name)
      if (const int rc = device_pointer(dev, b[i].p, call, 0, i)) return rc;
  return PRM_OK;
}
Buf optional(const void* p, const char* name, int64_t align) { return Buf{p, p ? name : nullptr, align}; }

int check_rows(const char* call, int64_t rows, int64_t cols, int64_t least_rows = 0, int64_t most_rows = kMaxRows) {
  if (rows < least_rows || rows > most_rows || cols < 1 || cols > kMaxCols)
    return fail(PRM_EINVAL, "%s: invalid shape %lld x %lld", call, (long long)rows, (long long)cols);
  return PRM_OK;
}
int check_ld(const char* call, const char* name, int64_t ld, int64_t least) {
  return ld >= least ? PRM_OK
                     : fail(PRM_EINVAL, "%s: leading dimension %s = %lld, needs %lld or more", call, name, (long long)ld, (long long)least);
}
int launched(const char* call, hipError_t e) {
  return e == hipSuccess ? PRM_OK : fail(PRM_EHIP, "%s: launch failed: %s", call, hipGetErrorString(e));
}
int check_workspace(const char* call, const void* p, uint64_t have, uint64_t need) {
  if (need && (have < need || !p))
    return fail(PRM_EINVAL, "%s: the workspace has %llu bytes, needs %llu", call, (unsigned long long)(p ? have : 0),
                (unsigned long long)need);
  return PRM_OK;
}

#define TRY(expr)                    \
  do {                               \
    const int rc_ = (expr);          \
    if (rc_ != PRM_OK) return rc_;   \
  } while (0)

}  // namespace

extern "C" {

int prm_quantize_rows(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t ldx, int8_t* q, int64_t ldq,
                      float* scale, void* hip_stream) {
  static const char* const call = "prm_quantize_rows";
  TRY(check_type(dtype));
  TRY(check_rows(call, rows, cols));
  TRY(check_ld(call, "ldx", ldx, cols));
  TRY(check_ld(call, "ldq", ldq, cols));
  if (rows == 0) return PRM_OK;
  TRY(check_buffers(call, {{x, "x", size_of(dtype)}, {q, "q", 1}, {scale, "scale", 4}}));
  QuantArgs a = {};
  a.x = x;
  a.q = q;
  a.scale = scale;
  a.rows = rows;
  a.cols = cols;
  a.ldx = ldx;
  a.ldq = ldq;
  return launched(call, launch_quantize_rows((OpType)dtype, a, (hipStream_t)hip_stream));
}

uint64_t prm_quantize_cols_workspace(int64_t rows, int64_t cols) {
  if (rows < 1 || rows > kMaxColRows || cols < 1 || cols > kMaxCols) return 0;
  int32_t nrb, per;
  quantize_cols_blocks(rows, cols, false, &nrb, &per);
  return (uint64_t)nrb * (uint64_t)cols * 8;
}

int prm_quantize_cols(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t ldx, int8_t* q, int64_t ldq,
                      float* scale, void* sum, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  static const char* const call = "prm_quantize_cols";
  TRY(check_type(dtype));
  TRY(check_rows(call, rows, cols, 1, kMaxColRows));
  QuantArgs a = {};
  a.rows = rows;
  a.cols = cols;
  QuantJobs jobs = {};
  jobs.columns[0] = true;
  jobs.n = 1;
  jobs.a[0] = a;
  if (quantize_tiles(jobs) >= kMaxTiles) return fail(PRM_EINVAL, "%s: %lld x %lld is too large", call, (long long)rows, (long long)cols);
  TRY(check_ld(call, "ldx", ldx, cols));
  TRY(check_ld(call, "ldq", ldq, rows));
  TRY(check_workspace(call, workspace, workspace_bytes, prm_quantize_cols_workspace(rows, cols)));
  TRY(check_buffers(call, {{x, "x", size_of(dtype)}, {q, "q", 1}, {scale, "scale", 4}, optional(sum, "sum", size_of(dtype)),
                           {workspace, "workspace", 16}}));
  a.x = x;
  a.q = q;
  a.scale = scale;
  a.sum = sum;
  a.ldx = ldx;
  a.ldq = ldq;
  // sums are added in one order, alone or in the layer's gradients
  quantize_cols_blocks(rows, cols, !sum, &a.nrb, &a.rows_per_block);
  a.part_max = (uint32_t*)workspace;
  a.part_sum = (float*)workspace + (int64_t)a.nrb * cols;
  jobs.a[0] = a;
  return launched(call, launch_quantize((OpType)dtype, jobs, (hipStream_t)hip_stream));
}

// prm_int8_matmul; `kind`, `splits`, `pack`: a ProductPlan, or 0 for the rule's (tests hold
// every kernel to the sizes that it takes).
int prm_internal_int8_matmul(const int8_t* a, int64_t lda, const float* a_scale, const int8_t* b, int64_t ldb,
                             const float* b_scale, const void* bias, int32_t dtype, void* out, int64_t ldo, int64_t m,
                             int64_t n, int64_t k, void* workspace, uint64_t workspace_bytes, void* hip_stream,
                             int32_t kind, int32_t splits, int32_t pack) {
  static const char* const call = "prm_int8_matmul";
  TRY(check_type(dtype));
  if (m < 0 || n < 0 || m > kMaxCols || n > kMaxCols || k < 1 || k > kMaxProductK)
    return fail(PRM_EINVAL, "%s: invalid sizes m %lld, n %lld, k %lld (1 <= k <= %lld)", call, (long long)m, (long long)n,
                (long long)k, (long long)kMaxProductK);
  TRY(check_ld(call, "lda", lda, k));
  TRY(check_ld(call, "ldb", ldb, k));
  TRY(check_ld(call, "ldo", ldo, n));
  if (m == 0 || n == 0) return PRM_OK;
  ProductArgs p = {a, b, a_scale, b_scale, bias, out, m, n, k, lda, ldb, ldo, (int32_t*)workspace};
  ProductPlan plan = {(ProductKind)kind, splits, pack};
  if (kind == 0) {
    // without the room that the fastest plan needs, the same sums by another
    plan = product_plan(p, true);
    if (!workspace || workspace_bytes < product_workspace(p, plan)) plan = product_plan(p, false);
    if (!product_takes(p, plan))
      return product_takes(p, product_plan(p, true))
                 ? fail(PRM_EINVAL, "%s: sums over more than %lld need their workspace", call, (long long)kMaxPieceK)
                 : fail(PRM_EINVAL, "%s: m %lld, n %lld is too large", call, (long long)m, (long long)n);
  } else if (kind < 0 || kind >= PRODUCT_KINDS || !product_takes(p, plan)) {
    return fail(PRM_EINVAL, "%s: kernel %d does not take this product in %d, %d", call, kind, splits, pack);
  }
  const uint64_t need = product_workspace(p, plan);
  if (need) TRY(check_workspace(call, workspace, workspace_bytes, need));
  TRY(check_buffers(call, {{a, "a", 1}, {a_scale, "a_scale", 4}, {b, "b", 1}, {b_scale, "b_scale", 4},
                           optional(bias, "bias", size_of(dtype)), {out, "out", size_of(dtype)},
                           optional(need ? workspace : nullptr, "workspace", 16)}));
  return launched(call, launch_int8_matmul((OpType)dtype, p, plan, (hipStream_t)hip_stream));
}

uint64_t prm_int8_matmul_workspace(const int8_t* a, int64_t lda, const int8_t* b, int64_t ldb, int64_t m, int64_t n, int64_t k) {
  if (m < 1 || n < 1 || m > kMaxCols || n > kMaxCols || k < 1 || k > kMaxProductK || lda < k || ldb < k) return 0;
  ProductArgs p = {};
  p.a = a;
  p.b = b;
  p.lda = lda;
  p.ldb = ldb;
  p.m = m;
  p.n = n;
  p.k = k;
  const ProductPlan plan = product_plan(p, true);
  return product_takes(p, plan) ? product_workspace(p, plan) : 0;
}

int prm_int8_matmul(const int8_t* a, int64_t lda, const float* a_scale, const int8_t* b, int64_t ldb, const float* b_scale,
                    const void* bias, int32_t dtype, void* out, int64_t ldo, int64_t m, int64_t n, int64_t k,
                    void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  return prm_internal_int8_matmul(a, lda, a_scale, b, ldb, b_scale, bias, dtype, out, ldo, m, n, k, workspace,
                                  workspace_bytes, hip_stream, 0, 0, 0);
}

// The layer's operands in 8 bits, their scales and the statistics' partial sums, one after
// the other in the caller's workspace (base NULL: their size alone).
struct Layout {
  char* base;
  uint64_t used = 0;
  void* take(uint64_t bytes) {
    void* p = base ? base + used : nullptr;
    used += (bytes + 255) & ~uint64_t(255);
    return p;
  }
};
// x (rows x cols) by rows or columns; `sum` as in prm_quantize_cols
static QuantArgs quantiser(Layout& l, const void* x, int64_t rows, int64_t cols, int64_t ldx, bool columns, void* sum) {
  QuantArgs a = {};
  a.x = x;
  a.rows = rows;
  a.cols = cols;
  a.ldx = ldx;
  a.sum = sum;
  const int64_t out_rows = columns ? cols : rows, out_cols = columns ? rows : cols;
  a.ldq = (out_cols + 15) / 16 * 16;
  a.q = (int8_t*)l.take((uint64_t)out_rows * (uint64_t)a.ldq);
  a.scale = (float*)l.take((uint64_t)out_rows * 4);
  if (columns) {
    quantize_cols_blocks(rows, cols, false, &a.nrb, &a.rows_per_block);
    a.part_max = (uint32_t*)l.take((uint64_t)a.nrb * (uint64_t)cols * 4);
    a.part_sum = (float*)l.take((uint64_t)a.nrb * (uint64_t)cols * 4);
  }
  return a;
}
// The workspace of the product of two such operands: their rows start on 16-byte boundaries.
static uint64_t part_bytes(int64_t m, int64_t n, int64_t k) {
  const int64_t ld = (k + 15) / 16 * 16;
  return prm_int8_matmul_workspace(nullptr, ld, nullptr, ld, m, n, k);
}
// p^T q of two quantised operands (k: the length of their rows), split where the rule does
static ProductArgs product_of(const QuantArgs& p, const QuantArgs& q, int64_t m, int64_t n, int64_t k, const void* bias, void* out,
                              int64_t ldo, void* part) {
  return ProductArgs{p.q, q.q, p.scale, q.scale, bias, out, m, n, k, p.ldq, q.ldq, ldo, (int32_t*)part};
}

struct LinearForward {
  QuantArgs x, w;
  void* part;
  uint64_t bytes;
  LinearForward(char* base, const void* xp, int64_t ldx, const void* wp, int64_t ldw, int64_t m, int64_t n, int64_t k) {
    Layout l{base};
    x = quantiser(l, xp, m, k, ldx, false, nullptr);
    w = quantiser(l, wp, n, k, ldw, false, nullptr);
    part = l.take(part_bytes(m, n, k));
    bytes = l.used;
  }
};
// of the gradients asked for
struct LinearBackward {
  QuantArgs g = {}, wt = {}, gt = {}, xt = {};
  void* part;
  uint64_t bytes;
  LinearBackward(char* base, const void* gp, int64_t ldg, const void* xp, int64_t ldx, const void* wp, int64_t ldw, int64_t m,
                 int64_t n, int64_t k, bool dx, bool dw, bool with_sum, void* db) {
    Layout l{base};
    if (dx) {
      g = quantiser(l, gp, m, n, ldg, false, nullptr);
      wt = quantiser(l, wp, n, k, ldw, true, nullptr);
    }
    if (dw || with_sum) gt = quantiser(l, gp, m, n, ldg, true, db);
    if (dw) xt = quantiser(l, xp, m, k, ldx, true, nullptr);
    const uint64_t a = dx ? part_bytes(m, k, n) : 0, b = dw ? part_bytes(n, k, m) : 0;
    part = l.take(a > b ? a : b);  // the products run one after the other
    bytes = l.used;
  }
};
static bool layer_sizes(int64_t m, int64_t n, int64_t k) {
  return m >= 1 && n >= 1 && k >= 1 && m <= kMaxProductK && n <= kMaxProductK && k <= kMaxProductK;
}
static int check_layer(const char* call, int64_t m, int64_t n, int64_t k) {
  if (m != 0 && !layer_sizes(m, n, k))
    return fail(PRM_EINVAL, "%s: invalid sizes m %lld, n %lld, k %lld (at most %lld)", call, (long long)m, (long long)n,
                (long long)k, (long long)kMaxProductK);
  return PRM_OK;
}

static int too_large(const char* call, int64_t m, int64_t n, int64_t k) {
  return fail(PRM_EINVAL, "%s: m %lld, n %lld, k %lld is too large", call, (long long)m, (long long)n, (long long)k);
}
static int check_plan(const char* call, const ProductArgs& p, const ProductPlan& plan) {
  return product_takes(p, plan) ? PRM_OK : too_large(call, p.m, p.n, p.k);
}

uint64_t prm_int8_linear_workspace(int64_t m, int64_t n, int64_t k) {
  return layer_sizes(m, n, k) ? LinearForward(nullptr, nullptr, 0, nullptr, 0, m, n, k).bytes : 0;
}

int prm_int8_linear(const void* x, int64_t ldx, const void* w, int64_t ldw, const void* bias, int32_t dtype, void* y,
                    int64_t ldy, int64_t m, int64_t n, int64_t k, void* workspace, uint64_t workspace_bytes,
                    void* hip_stream) {
  static const char* const call = "prm_int8_linear";
  TRY(check_type(dtype));
  TRY(check_layer(call, m, n, k));
  TRY(check_ld(call, "ldx", ldx, k));
  TRY(check_ld(call, "ldw", ldw, k));
  TRY(check_ld(call, "ldy", ldy, n));
  if (m == 0) return PRM_OK;
  const LinearForward f((char*)workspace, x, ldx, w, ldw, m, n, k);
  TRY(check_workspace(call, workspace, workspace_bytes, f.bytes));
  const int64_t es = size_of(dtype);
  const ProductArgs p = product_of(f.x, f.w, m, n, k, bias, y, ldy, f.part);
  const ProductPlan plan = product_plan(p, true);
  TRY(check_plan(call, p, plan));
  TRY(check_buffers(call, {{x, "x", es}, {w, "w", es}, optional(bias, "bias", es), {y, "y", es}, {workspace, "workspace", 16}}));
  QuantJobs jobs = {};
  jobs.a[0] = f.x;
  jobs.a[1] = f.w;
  jobs.n = 2;
  TRY(launched(call, launch_quantize((OpType)dtype, jobs, (hipStream_t)hip_stream)));
  return launched(call, launch_int8_matmul((OpType)dtype, p, plan, (hipStream_t)hip_stream));
}

// What the gradients asked for need of prm_int8_linear_backward_workspace.
uint64_t prm_internal_int8_linear_backward_workspace(int64_t m, int64_t n, int64_t k, int32_t dx, int32_t dw, int32_t db) {
  return layer_sizes(m, n, k) ? LinearBackward(nullptr, nullptr, 0, nullptr, 0, nullptr, 0, m, n, k, dx, dw, db, nullptr).bytes : 0;
}
uint64_t prm_int8_linear_backward_workspace(int64_t m, int64_t n, int64_t k) {
  return prm_internal_int8_linear_backward_workspace(m, n, k, 1, 1, 1);
}

int prm_int8_linear_backward(const void* gy, int64_t ldgy, const void* x, int64_t ldx, const void* w, int64_t ldw,
                             int32_t dtype, void* dx, int64_t lddx, void* dw, int64_t lddw, void* db, int64_t m, int64_t n,
                             int64_t k, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  static const char* const call = "prm_int8_linear_backward";
  TRY(check_type(dtype));
  TRY(check_layer(call, m, n, k));
  if (m == 0) return fail(PRM_EINVAL, "%s: m is 0", call);
  TRY(check_ld(call, "ldgy", ldgy, n));
  if (dw) {
    TRY(check_ld(call, "ldx", ldx, k));
    TRY(check_ld(call, "lddw", lddw, k));
  }
  if (dx) {
    TRY(check_ld(call, "ldw", ldw, k));
    TRY(check_ld(call, "lddx", lddx, k));
  }
  if (!dx && !dw && !db) return PRM_OK;
  const LinearBackward f((char*)workspace, gy, ldgy, x, ldx, w, ldw, m, n, k, dx, dw, db, db);
  TRY(check_workspace(call, workspace, workspace_bytes, f.bytes));
  QuantJobs jobs = {};
  const auto add = [&](const QuantArgs& a, bool columns) {
    jobs.columns[jobs.n] = columns;
    jobs.a[jobs.n++] = a;
  };
  if (dx) {
    add(f.g, false);
    add(f.wt, true);
  }
  if (dw || db) add(f.gt, true);
  if (dw) add(f.xt, true);
  const ProductArgs px = product_of(f.g, f.wt, m, k, n, nullptr, dx, lddx, f.part);
  const ProductArgs pw = product_of(f.gt, f.xt, n, k, m, nullptr, dw, lddw, f.part);
  const ProductPlan plan_x = product_plan(px, true), plan_w = product_plan(pw, true);
  // all that can be refused is, before the first launch
  if (dx) TRY(check_plan(call, px, plan_x));
  if (dw) TRY(check_plan(call, pw, plan_w));
  if (quantize_tiles(jobs) >= kMaxTiles) return too_large(call, m, n, k);
  const int64_t es = size_of(dtype);
  TRY(check_buffers(call, {{gy, "gy", es}, Buf{x, dw ? "x" : nullptr, es}, Buf{w, dx ? "w" : nullptr, es}, optional(dx, "dx", es),
                           optional(dw, "dw", es), optional(db, "db", es), {workspace, "workspace", 16}}));
  hipStream_t s = (hipStream_t)hip_stream;
  TRY(launched(call, launch_quantize((OpType)dtype, jobs, s)));
  if (dx) TRY(launched(call, launch_int8_matmul((OpType)dtype, px, plan_x, s)));
  if (dw) TRY(launched(call, launch_int8_matmul((OpType)dtype, pw, plan_w, s)));
  return PRM_OK;
}

int prm_rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ldres, const void* w, int32_t dtype,
                 int64_t rows, int64_t cols, float eps, void* h, int64_t ldh, void* y, int64_t ldy, int8_t* q, int64_t ldq,
                 float* scale, void* hip_stream) {
  static const char* const call = "prm_rms_norm";
  TRY(check_type(dtype));
  TRY(check_rows(call, rows, cols));
  if (!(eps > 0.f) || !std::isfinite(eps)) return fail(PRM_EINVAL, "%s: eps must be finite and > 0", call);
  if (!residual != !h) return fail(PRM_EINVAL, "%s: residual and h come together", call);
  if (y ? (q || scale) : rows > 0 && !(q && scale)) return fail(PRM_EINVAL, "%s: either y, or q and scale", call);
  TRY(check_ld(call, "ldx", ldx, cols));
  if (residual) {
    TRY(check_ld(call, "ldres", ldres, cols));
    TRY(check_ld(call, "ldh", ldh, cols));
  }
  TRY(y ? check_ld(call, "ldy", ldy, cols) : check_ld(call, "ldq", ldq, cols));
  if (rows == 0) return PRM_OK;
  const int64_t es = size_of(dtype);
  TRY(check_buffers(call, {{x, "x", es}, optional(residual, "residual", es), optional(w, "w", es), optional(h, "h", es),
                           optional(y, "y", es), optional(q, "q", 1), optional(scale, "scale", 4)}));
  NormArgs a = {x, residual, w, h, y, q, scale, rows, cols, ldx, ldres, ldh, ldy, ldq, eps};
  return launched(call, launch_rms_norm((OpType)dtype, a, (hipStream_t)hip_stream));
}

uint64_t prm_rms_norm_backward_workspace(int64_t rows, int64_t cols) {
  if (rows < 1 || rows > kMaxRows || cols < 1 || cols > kMaxCols) return 0;
  return (uint64_t)rms_norm_grad_parts(OP_BF16, rows, cols) * (uint64_t)cols * 4;
}

int prm_rms_norm_backward(const void* gy, int64_t ldgy, const void* gh, int64_t ldgh, const void* h, int64_t ldh,
                          const void* w, int32_t dtype, int64_t rows, int64_t cols, float eps, void* dx, int64_t lddx,
                          void* dw, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  static const char* const call = "prm_rms_norm_backward";
  TRY(check_type(dtype));
  TRY(check_rows(call, rows, cols));
  if (!(eps > 0.f) || !std::isfinite(eps)) return fail(PRM_EINVAL, "%s: eps must be finite and > 0", call);
  TRY(check_ld(call, "ldgy", ldgy, cols));
  TRY(check_ld(call, "ldh", ldh, cols));
  TRY(check_ld(call, "lddx", lddx, cols));
  if (gh) TRY(check_ld(call, "ldgh", ldgh, cols));
  if (rows == 0 && !dw) return PRM_OK;
  const int64_t es = size_of(dtype);
  if (rows == 0) {
    TRY(check_buffers(call, {{dw, "dw", es}}));
  } else {
    if (dw) TRY(check_workspace(call, workspace, workspace_bytes, prm_rms_norm_backward_workspace(rows, cols)));
    TRY(check_buffers(call, {{gy, "gy", es}, optional(gh, "gh", es), {h, "h", es}, optional(w, "w", es), {dx, "dx", es},
                             optional(dw, "dw", es), optional(dw ? workspace : nullptr, "workspace", 16)}));
  }
  NormGradArgs a = {gy, gh, h, w, dx, dw, (float*)workspace, rows, cols, ldgy, ldgh, ldh, lddx, eps,
                    rms_norm_grad_parts((OpType)dtype, rows, cols)};
  return launched(call, launch_rms_norm_grad((OpType)dtype, a, (hipStream_t)hip_stream));
}

}  // extern "C"
