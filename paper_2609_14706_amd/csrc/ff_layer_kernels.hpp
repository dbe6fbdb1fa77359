// Host-side launchers of the layer operators (norm, linear, orthogonalisation).
// As in ff_kernels.hpp: each enqueues on the given stream, checks the
// preconditions its kernels rely on and allocates nothing.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace ff {

typedef uint16_t bf16_t;

// --------------------------------------------------------------------- norm
// eps as it is added to mean s^2, and for s scaled up or down by the kernels' factors
struct Eps {
  float plain, up, down;
};
Eps eps_of(double eps);
// Rows of `cols` elements (bf16 or fp32), leading dimensions in elements.
struct NormArgs {
  int64_t rows, cols;
  const void* x;
  int64_t ldx;
  const void* residual;  // or null
  int64_t ldr;
  const void* weight;      // cols, the rows' type; null: ones
  const float* col_scale;  // q: cols; null: ones
  void* sum;               // x + residual, or null
  int64_t ldsum;
  void* y;  // the norm, or null (then q)
  int64_t ldy;
  int8_t* q;  // codes, or null (then y)
  int64_t ldq;
  float* q_scale;  // rows
  Eps eps;
  int normalise;  // 0: codes of x (+ residual) itself
};
hipError_t launch_norm(const NormArgs& a, bool bf16, hipStream_t s);

struct NormGradArgs {
  int64_t rows, cols;
  const void* s;
  int64_t lds;
  const void* dy;
  int64_t lddy;
  const void* dsum;  // or null
  int64_t lddsum;
  const void* weight;  // or null
  void* dx;
  int64_t lddx;
  float* part;  // norm_grad_parts(rows) x cols partial sums of dw, or null
  Eps eps;
};
int64_t norm_grad_parts(int64_t rows);
hipError_t launch_norm_grad(const NormGradArgs& a, bool bf16, hipStream_t s);
// out[j] (bf16 or fp32) = sum over the rows of part (rows x cols).
hipError_t launch_col_sums(const float* part, int64_t rows, int64_t cols, void* out, bool bf16, hipStream_t s);

// -------------------------------------------------- 8-bit activation checkpoints
// Rows of codes, a scale for every 2^shift columns: value = q scale.
constexpr int kMinGroupShift = 4, kMaxGroupShift = 9;
struct Q8Rows {
  const int8_t* q;  // null: none
  int64_t ldq;
  const float* scale;  // rows x ceil(cols / 2^shift)
  int64_t lds;
  int shift;
};
struct CheckpointArgs {
  int64_t rows, cols;
  void* x;  // read (launch_checkpoint) or written (launch_restore)
  int64_t ldx;
  int8_t* q;
  int64_t ldq;
  float* scale;
  int64_t lds;
  int shift;
};
hipError_t launch_checkpoint(const CheckpointArgs& a, bool bf16, hipStream_t s);
hipError_t launch_restore(const CheckpointArgs& a, bool bf16, hipStream_t s);

// ------------------------------------------------------------------- linear
enum Act : int { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };

// y = act(scale . (x w^T) + bias) + residual, x: tokens x n, w: m x n, of bf16
// or of 8-bit integers (x_scale: tokens, row_scale: m; null with bf16).
struct LinearArgs {
  int64_t tokens, n, m;
  const void* x;
  int64_t ldx;
  const void* w;
  int64_t ldw;
  const float* x_scale;
  const float* row_scale;
  const bf16_t* bias;      // m, or null
  const bf16_t* residual;  // tokens x m, or null
  int64_t ldr;
  bf16_t* y;
  int64_t ldy;
  bf16_t* preact;  // scale . (x w^T) + bias, or null
  int64_t ldz;
  int act;
};
// How a product is run: `skinny` for few tokens, else tiles of
// 32 ti x 32 tj, `slots` pairs of k in LDS, with k in `splits` parts (joined by
// a second kernel).
struct LinearPlan {
  bool skinny;
  int ti, tj, slots;
  int splits;
};
LinearPlan linear_plan(int64_t tokens, int64_t n, int64_t m, int elem_bytes);
// The few-token kernel's 16-token and 16-output tiles and waves of a workgroup.
struct SkinnyPlan {
  int nt, rw, waves;
};
SkinnyPlan skinny_plan(int64_t tokens, int64_t n, int64_t m, int elem_bytes);
// Bytes of the partial sums of a plan (0 with one split).
size_t linear_partial_bytes(const LinearPlan& p, int64_t tokens, int64_t m);
// Whether the tiles take rows from p on, ld elements apart, of n elements:
// 16-byte aligned rows of whole 16-byte pieces of k.
bool tile_rows_ok(const void* p, int64_t ld, int64_t n, int elem_bytes);
// Leading dimension (elements) of launch_pack_rows's rows.
int64_t packed_ld(int64_t n, int elem_bytes);
// dst (rows x packed_ld(n), zeros beyond n) from src (rows x n).
hipError_t launch_pack_rows(const void* src, int64_t ld, int64_t rows, int64_t n, int elem_bytes, void* dst,
                            hipStream_t s);
hipError_t launch_linear(const LinearArgs& a, const LinearPlan& p, int elem_bytes, void* partial, hipStream_t s);

// dst (rows x cols elements, ld apart) = 0.
hipError_t launch_zero(void* dst, int64_t ld, int64_t rows, int64_t cols, int elem_bytes, hipStream_t s);

// g = dy act'(z) (rows x cols; null: not stored), its transpose gt (cols x
// ldgt, zeros beyond rows; null: not stored) and, with part, column sums of
// every 64 rows (act_grad_parts(rows) x cols).  z null: g = dy, so that with
// gt alone a job is a transposition.  One to three jobs in one launch.
struct ActGradArgs {
  int64_t rows, cols;
  const bf16_t* dy;
  int64_t lddy;
  const bf16_t* z;
  int64_t ldz;
  bf16_t* g;
  int64_t ldg;
  bf16_t* gt;
  int64_t ldgt;
  float* part;
  int act;
};
int64_t act_grad_parts(int64_t rows);
hipError_t launch_act_grad(const ActGradArgs* jobs, int count, hipStream_t s);

// ---------------------------------------------------------- orthogonalisation
// X <- a X + (b A + c A^2) X, A = X X^T, `steps` times from G / (||G||_F + eps)
// for each of `batch` matrices m x n (bf16 or fp32), times `scale`.
struct OrthoArgs {
  int64_t batch, m, n;
  const void* g;
  int64_t ldg, sg;  // row and matrix strides in elements
  void* out;
  int64_t ldo, so;
  int steps;
  float a, b, c, scale;
  double eps;
  bool bf16;
};
// Whether the coefficients keep every singular value that starts in [0, 1]
// below 16 through the steps.
bool ortho_bounded(int steps, double a, double b, double c);
// How updates are run: `small` parts in one workgroup each, or (0) step by step,
// the three products of a step by their forms (ff_ortho.hip), A = X X^T with k in
// `gram_splits` parts.
struct OrthoPlan {
  int small;
  int gram, gram_splits, square, apply;
};
OrthoPlan ortho_plan(int64_t batch, int64_t m, int64_t n, bool bf16);
size_t ortho_workspace(int64_t batch, int64_t m, int64_t n, bool bf16);
hipError_t launch_ortho(const OrthoArgs& a, void* workspace, hipStream_t s);

}  // namespace ff
