// Internal definitions of the operators beside the optimizer step (ops_*.hip): the
// 8-bit linear layer's quantiser, norm and product.  Their C ABI is in prm.h.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace prm {

// prm_dtype of an operator's activations and outputs
enum OpType : int32_t { OP_F32 = 0, OP_BF16 = 1, OP_F16 = 2 };

// ---- error state shared with the optimizer step (prm_api.hip) ----------------
int set_error(int code, const char* msg);  // stores msg for prm_last_error, returns code
int device_pointer(int dev, const void* p, const char* what, int i, int k);  // PRM_OK or PRM_EINVAL

// ---- rows (ops_rows.hip) ------------------------------------------------------
// A row of `cols` elements; leading dimensions in elements, any alignment of an element.
struct NormArgs {
  const void* x;
  const void* res;  // or nullptr
  const void* w;    // or nullptr: ones
  void* h;          // x + res in the storage type; with res only
  void* y;          // or nullptr: q and scale instead
  int8_t* q;
  float* scale;
  int64_t rows, cols, ldx, ldres, ldh, ldy, ldq;
  float eps;
};
hipError_t launch_rms_norm(OpType t, const NormArgs& a, hipStream_t s);

struct QuantArgs {
  const void* x;
  int8_t* q;
  float* scale;
  int64_t rows, cols, ldx, ldq;
  // of the columns' form: partial maxima (and sums) of row blocks, nrb x cols each
  uint32_t* part_max;
  float* part_sum;
  void* sum;  // column sums in the type of x, or nullptr
  int32_t nrb, rows_per_block;  // nrb 0: none, the tiles take their columns' statistics
};
hipError_t launch_quantize_rows(OpType t, const QuantArgs& a, hipStream_t s);
// Up to four quantisers of one type, by rows or (`columns`) by columns, in one launch for
// rows and the columns' statistics and one for the columns.
struct QuantJobs {
  QuantArgs a[4];
  bool columns[4];
  int32_t blocks[4];  // of a launch, laid out by it
  int32_t n;
};
hipError_t launch_quantize(OpType t, const QuantJobs& jobs, hipStream_t s);
int64_t quantize_tiles(const QuantJobs& jobs);  // of the columns' launch, less than kMaxTiles
// row blocks of the columns' statistics; alone: of a launch without other quantisers
void quantize_cols_blocks(int64_t rows, int64_t cols, bool alone, int32_t* nrb, int32_t* rows_per_block);

struct NormGradArgs {
  const void* gy;
  const void* gh;  // gradient of the kept sum, or nullptr
  const void* h;
  const void* w;   // or nullptr
  void* dx;
  void* dw;        // or nullptr
  float* part;     // nparts x cols
  int64_t rows, cols, ldgy, ldgh, ldh, lddx;
  float eps;
  int32_t nparts;
};
hipError_t launch_rms_norm_grad(OpType t, const NormGradArgs& a, hipStream_t s);
int32_t rms_norm_grad_parts(OpType t, int64_t rows, int64_t cols);  // most for 16-bit types

// ---- products (ops_matmul.hip) -------------------------------------------------
struct ProductArgs {
  const int8_t* a;  // m x k
  const int8_t* b;  // n x k
  const float* a_scale;
  const float* b_scale;
  const void* bias;  // n of the output's type, or nullptr
  void* out;         // m x n
  int64_t m, n, k, lda, ldb, ldo;
  int32_t* part;     // the splits' sums, or nullptr
};
// The kernels, by tile; ANY: rows that start on any byte; PAIRED: two blocks a CU.  64 and 128 can
// split k over blocks, whose sums meet in `part` (product_workspace bytes), and, as PAIRED and 256, take
// operands that were laid out anew.
enum ProductKind : int32_t {
  PRODUCT_FEW = 1, PRODUCT_ANY64, PRODUCT_ANY128, PRODUCT_64, PRODUCT_128, PRODUCT_128_PAIRED, PRODUCT_256,
  PRODUCT_KINDS
};
struct ProductPlan {
  ProductKind kind;
  int32_t splits;
  int32_t pack;  // 1: a, 2: b laid out anew, in `part` before the splits' sums
};
bool product_takes(const ProductArgs& p, const ProductPlan& plan);
ProductPlan product_plan(const ProductArgs& p, bool workspace);  // the rule, with or without a workspace
uint64_t product_workspace(const ProductArgs& p, const ProductPlan& plan);
// pack_kernel: rows of k bytes, ld apart, to rows of kp
struct PackArgs {
  const int8_t* src[2];
  int8_t* dst[2];
  int64_t rows[2], ld[2];
  int64_t k, kp;
};
hipError_t launch_int8_matmul(OpType t, const ProductArgs& p, const ProductPlan& plan, hipStream_t s);
// 128 * 128 k stays below 2^31 in one piece; longer sums are split and joined in 64 bits
constexpr int64_t kMaxPieceK = 131071, kMaxProductK = 1 << 20;
constexpr int64_t kMaxTiles = 1 << 24;  // a grid holds less than 2^32 threads

}  // namespace prm
