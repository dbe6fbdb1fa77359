// Host-side launchers of the operators around a layer of experts: routing, the
// experts' products and their gradients.  As in ff_layer_kernels.hpp.
//
// T tokens choose `top` of E experts each: slot s = t top + j is token t's j-th
// choice.  Slots sorted by expert (and by slot within one) are the rows that the
// experts' products work on: row p holds slot order[p], expert e rows offsets[e] ..
// offsets[e + 1] - 1, and slot s lies at row place[s] (-1: not routed, in no row).
#pragma once

#include "ff_layer_kernels.hpp"

namespace ff {

constexpr int kMaxExperts = 1024, kMaxTop = 64, kMaxGroups = 64;

struct RouteArgs {
  int64_t tokens;
  int experts, top;
  const void* logits;  // tokens x experts
  int64_t ldl;
  bool bf16;
  const float* bias;    // experts, or null
  const uint8_t* mask;  // tokens: 0 not routed; or null
  bool sigmoid;         // scores: else softmax
  int groups, top_groups;
  bool renormalise;
  double scale;
  float* weights;   // tokens x top
  int32_t* chosen;  // tokens x top
  int32_t* order;   // tokens x top; null: slots are not sorted
  int32_t* offsets;
  int32_t* place;
};
// Bytes of workspace of the sort (0 where one workgroup does it all).
size_t route_workspace(int64_t tokens, int experts, int top);
hipError_t launch_route(const RouteArgs& a, void* workspace, hipStream_t s);
// order, offsets and place of the experts in a.chosen.
hipError_t launch_order(const RouteArgs& a, void* workspace, hipStream_t s);

struct RouteGradArgs {
  int64_t tokens;
  int experts, top;
  const void* logits;
  int64_t ldl;
  bool bf16;
  const float* dweights;  // tokens x top
  const int32_t* chosen;
  bool sigmoid, renormalise;
  double scale;
  void* dlogits;  // tokens x experts, as logits
  int64_t ldd;
};
hipError_t launch_route_grad(const RouteGradArgs& a, hipStream_t s);

// The rows of a routed batch: `rows` = tokens top of them, those from offsets[experts] on
// in no expert.  What the arrays hold is checked against rows before it is used.  Without
// offsets all rows are the one expert's (experts 1, top 1): a plain layer.
struct SlotRows {
  int64_t tokens, rows;
  int experts, top;
  const int32_t* order;
  const int32_t* offsets;
  const int32_t* place;
  const float* weights;
};

// y_p = act(x W_e^T + b_e) of the rows of each expert e; rows in no expert get zeros.
// x: a token's row for each of its slots (gather), or a row for each slot.
struct ExpertArgs {
  SlotRows at;
  LinearArgs lin;  // w: experts x m rows of n, bias: experts x m; y and preact by row
  bool gather;
};
// How the products are run: `nt` 16-token tiles of the few-token form with `waves` waves a
// workgroup, or (nt 0) tiles of 32 ti x 32 tj, `slots` pairs of k in LDS, k in `splits` parts.
struct ExpertPlan {
  int nt, waves;
  int ti, tj, slots, splits;
};
// w_lies: whether tiles can read the weights as they lie.
ExpertPlan expert_plan(int64_t rows, int experts, int64_t n, int64_t m, bool w_lies);
hipError_t launch_expert_linear(const ExpertArgs& a, const ExpertPlan& p, hipStream_t s);

// out_t = residual_t + sum over the token's slots of weight y (rows of bf16), or the
// plain sum of fp32 rows, `parts` of them part_stride elements apart (weights null).  Without place
// (top 1) token t's row is row t.
struct CombineArgs {
  SlotRows at;
  int64_t cols;
  const void* y;
  int64_t ldy;
  bool f32;
  int parts;
  int64_t part_stride;
  const bf16_t* residual;  // or null
  int64_t ldr;
  bf16_t* out;
  int64_t ldo;
};
hipError_t launch_combine(const CombineArgs& a, hipStream_t s);

// dy_p = weight dout_t (fp32), dweight_s = <dout_t, y_p>; zeros where there is no slot or row.
struct CombineGradArgs {
  SlotRows at;
  int64_t cols;
  const bf16_t* dout;
  int64_t ldd;
  const bf16_t* y;
  int64_t ldy;
  float* dy;  // or null
  int64_t lddy;
  float* dweights;  // or null
};
hipError_t launch_combine_grad(const CombineGradArgs& a, hipStream_t s);

// Rows for the products to read: dst_p = src of row p or (gather) of its token, times
// act'(z_p) where z is given, zeros for rows in no expert.  Stored as `out` (bf16), `laid`
// (bf16, rows of laid_ld(cols) elements with zeros beyond cols) and `scaled` (the same in fp16,
// times the power of two that takes the peaks' largest to 2^14 .. 2^15).
struct RowsArgs {
  SlotRows at;
  bool gather;
  int64_t cols;
  const void* src;  // bf16, or fp32 (src_f32), or null (then src_q8)
  int64_t lds;
  bool src_f32;
  Q8Rows src_q8;
  const bf16_t* z;  // or z_q8, or neither
  int64_t ldz;
  Q8Rows z_q8;
  int act;
  bf16_t* out;  // or null
  int64_t ldo;
  uint16_t* laid;    // or null
  uint16_t* scaled;  // or null
  const uint32_t* peaks;
  float peak_factor;  // scaled: the largest value is at most that times the peak
  float* inverse;     // scaled: receives the power of two that takes its values back
  float* parts;       // column sums of every part_rows(...) rows of an expert (part_count rows of
                      // laid_ld(cols)); or null
};
// Rows of an expert that are summed together, and how many such sums there can be; expert e's
// are those from offsets[e] / part_rows + e on.  With 16 and 64 (g and db alone): 2042 rows of 333 17.3 and 23.5 us,
// 1021 of 777 17.1 and 18.5, 1024 of 4096 the same, 4096 of 11008 45.7 and 38.3.
inline int part_rows(int64_t rows, int64_t cols) { return rows * cols >= (int64_t(1) << 22) ? 64 : 16; }
inline int64_t part_count(int64_t rows, int experts, int64_t cols) { return rows / part_rows(rows, cols) + experts + 1; }
inline int64_t laid_ld(int64_t cols) { return (cols + 7) / 8 * 8; }
// One to three jobs in one launch.
hipError_t launch_rows(const RowsArgs* jobs, int count, hipStream_t s);
// peaks: kPeaks bit patterns of largest finite magnitudes among the `cols` elements that launch_rows makes of
// the rows that are in an expert (gather: of their tokens' rows), zeros where there are none; of a
// checkpoint given as its scales (src fp32) among those.  Two jobs in one launch, the second without z.
constexpr int kPeaks = 1024;
hipError_t launch_peaks(const RowsArgs& g, uint32_t* g_peaks, const RowsArgs& scales, uint32_t* x_peaks, hipStream_t s);

// Gradients of the products; g rows of bf16, or (f16) of fp16 scaled by its peaks, 16-byte
// aligned with zeros up to a multiple of 8.
struct ExpertGradArgs {
  SlotRows at;
  int64_t n, m;
  const uint16_t* g;
  int64_t ldg;
  const bf16_t* w;  // launch_expert_dx: experts x m rows of n, 16-byte aligned
  int64_t ldw;
  const uint16_t* x;  // launch_expert_dw: by row, as g
  int64_t ldx;
  void* out;  // bf16, or fp32 (out_f32, and with splits: parts part_stride elements apart)
  int64_t ldo;
  bool out_f32;
  int64_t part_stride;
  const float* parts;  // column sums of g by launch_rows, of part_rows rows each; or null
  int part_rows;
  bf16_t* db;  // launch_expert_dw, launch_expert_db: their sums
  bool f16;
  const float* inverse;  // f16: what takes g and x back
};
// dx_p = g_p W_e, zeros for rows in no expert.
ExpertPlan expert_dx_plan(int64_t rows, int experts, int64_t n, int64_t m);
hipError_t launch_expert_dx(const ExpertGradArgs& a, const ExpertPlan& p, hipStream_t s);
// dW_e = sum over the rows of expert e of g_p^T x_p (m x n; zeros for an expert without rows).
ExpertPlan expert_dw_plan(int64_t rows, int experts, int64_t n, int64_t m);
hipError_t launch_expert_dw(const ExpertGradArgs& a, const ExpertPlan& p, hipStream_t s);
// Both in one launch, for plans that leave units empty.
bool expert_both(const ExpertPlan& dx, const ExpertPlan& dw);
hipError_t launch_expert_both(const ExpertGradArgs& x, const ExpertPlan& px, const ExpertGradArgs& w, const ExpertPlan& pw,
                              hipStream_t s);
// db_e = sum over the rows of expert e of g_p, from the parts alone.
hipError_t launch_expert_db(const ExpertGradArgs& a, hipStream_t s);

}  // namespace ff
