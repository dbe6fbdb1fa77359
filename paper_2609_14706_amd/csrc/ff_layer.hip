// C ABI of the operators around one layer (ff.h): argument checks, workspace
// layout and the order of the kernels' launches.  No state is kept.
#include <math.h>
#include <stdio.h>

#include <algorithm>
#include <initializer_list>

#include "ff.h"
#include "ff_error.hpp"
#include "ff_kernels.hpp"
#include "ff_layer_checks.hpp"
#include "ff_layer_kernels.hpp"

using namespace ff;

namespace {

// ---------------------------------------------------------------------- norm
ff_status norm_sizes(int64_t rows, int64_t cols, ff_dtype dtype, double eps) {
  if (rows < 0 || rows > kMaxRows || cols < 1 || cols > kMaxCols) return bad("rows must be >= 0, cols 1 .. 2^24");
  if (dtype != FF_F32 && dtype != FF_BF16) return bad("unknown dtype");
  if (!(eps >= 0.0) || !std::isfinite(eps)) return bad("eps must be finite and >= 0");
  return FF_OK;
}

// --------------------------------------------------------------------- linear
struct LinearWs {
  LinearPlan plan;
  bool pack_x, pack_w;
  size_t off_w, off_p, bytes;
};

// w_ready: the rows of w start aligned and hold zeros from n to the next whole
// 16-byte piece.
LinearWs linear_ws(int64_t tokens, int64_t n, int64_t m, const void* x, int64_t ldx, const void* w, int64_t ldw,
                   int eb, bool w_ready = false) {
  LinearWs l{};
  l.plan = linear_plan(tokens, n, m, eb);
  // the tiles copy whole 16-byte pieces; other rows are laid out for them first
  l.pack_x = !l.plan.skinny && !tile_rows_ok(x, ldx, n, eb);
  l.pack_w = !l.plan.skinny && !w_ready && !tile_rows_ok(w, ldw, n, eb);
  size_t off = 0;
  if (l.pack_x) off += up256((size_t)tokens * (size_t)packed_ld(n, eb) * eb);
  l.off_w = off;
  if (l.pack_w) off += up256((size_t)m * (size_t)packed_ld(n, eb) * eb);
  l.off_p = off;
  l.bytes = off + up256(linear_partial_bytes(l.plan, tokens, m));
  return l;
}

// The product with operands packed where they have to be; ws: linear_ws bytes.
ff_status run_linear(LinearArgs a, int eb, char* ws, hipStream_t s, bool w_ready = false) {
  const LinearWs l = linear_ws(a.tokens, a.n, a.m, a.x, a.ldx, a.w, a.ldw, eb, w_ready);
  ff_status rc;
  const int64_t n = a.n;
  if (l.pack_x) {
    if ((rc = hip(launch_pack_rows(a.x, a.ldx, a.tokens, n, eb, ws, s), "packing x")) != FF_OK) return rc;
    a.x = ws;
    a.ldx = packed_ld(n, eb);
  }
  if (l.pack_w) {
    if ((rc = hip(launch_pack_rows(a.w, a.ldw, a.m, n, eb, ws + l.off_w, s), "packing W")) != FF_OK) return rc;
    a.w = ws + l.off_w;
    a.ldw = packed_ld(n, eb);
  }
  if (l.pack_x || l.pack_w) {
    // k up to the next whole 16-byte piece: zeros in both operands (an n that is
    // no multiple of it has both packed, or w ready)
    const int64_t g = 16 / eb;
    a.n = (n + g - 1) / g * g;
  }
  return hip(launch_linear(a, l.plan, eb, ws + l.off_p, s), "linear product");
}

ff_status linear_sizes(int64_t tokens, int64_t n, int64_t m) {
  if (tokens < 0 || tokens > kMaxRows || n < 1 || m < 1 || n > kMaxDim || m > kMaxDim)
    return bad("tokens must be >= 0, n and m 1 .. 2^20");
  return FF_OK;
}

ff_status linear_checks(const ff_linear_args* a, bool q8) {
  if (a == nullptr) return bad("args is NULL");
  ff_status rc = linear_sizes(a->tokens, a->n, a->m);
  if (rc != FF_OK) return rc;
  // 128^2 n reaches 2^31 at most, which the kernels still tell apart
  if (q8 && a->n > 131072) return bad("n must be <= 131072 for 8-bit products");
  if (a->tokens > (int64_t(1) << 31)) return bad("tokens must be <= 2^31");
  return FF_OK;
}

ff_status linear_call(const ff_linear_args* a, bool q8) {
  ff_status rc = linear_checks(a, q8);
  if (rc != FF_OK) return rc;
  if (a->tokens == 0) return FF_OK;
  const int eb = q8 ? 1 : 2;
  if (!rows_ok(a->x, a->ldx, a->n, eb) || !rows_ok(a->w, a->ldw, a->n, eb))
    return bad("x and w must be aligned device pointers to rows of n elements, ld >= n");
  if (!rows_ok(a->y, a->ldy, a->m, 2) || (a->residual != nullptr && !rows_ok(a->residual, a->ldr, a->m, 2)) ||
      (a->preact != nullptr && !rows_ok(a->preact, a->ldz, a->m, 2)))
    return bad("y, residual and preact must be aligned device pointers to rows of m elements, ld >= m");
  if ((uintptr_t)a->bias % 2 != 0) return bad("bias is misaligned");
  if (a->activation < FF_ACT_NONE || a->activation > FF_ACT_SILU) return bad("unknown activation");
  if (q8 && (a->x_scale == nullptr || a->row_scale == nullptr || (uintptr_t)a->x_scale % 4 != 0 ||
             (uintptr_t)a->row_scale % 4 != 0))
    return bad("x_scale and row_scale must be aligned device pointers");
  if (!q8 && (a->x_scale != nullptr || a->row_scale != nullptr)) return bad("scales belong to ff_linear_q8");
  const int64_t T = a->tokens, lm = a->m * 2, ln = a->n * eb;
  const void* outs[2] = {a->y, a->preact};
  const int64_t lo[2] = {a->ldy * 2, a->ldz * 2};
  for (int k = 0; k < 2; ++k)
    if (meet(outs[k], T, lo[k], lm, a->x, T, a->ldx * eb, ln) || meet(outs[k], T, lo[k], lm, a->w, a->m, a->ldw * eb, ln))
      return bad("y and preact must not overlap x or w");
  if (meet(a->y, T, lo[0], lm, a->preact, T, lo[1], lm) ||
      meet(a->preact, T, lo[1], lm, a->residual, T, a->ldr * 2, lm) ||
      (meet(a->y, T, lo[0], lm, a->residual, T, a->ldr * 2, lm) && !(a->y == a->residual && a->ldy == a->ldr)))
    return bad("y, preact and residual must not overlap (y may be the residual itself)");
  const LinearWs l = linear_ws(T, a->n, a->m, a->x, a->ldx, a->w, a->ldw, eb);
  if ((rc = workspace_ok(a->workspace, a->workspace_bytes, l.bytes)) != FF_OK) return rc;
  LinearArgs k{};
  k.tokens = T;
  k.n = a->n;
  k.m = a->m;
  k.x = a->x;
  k.ldx = a->ldx;
  k.w = a->w;
  k.ldw = a->ldw;
  k.x_scale = a->x_scale;
  k.row_scale = a->row_scale;
  k.bias = (const bf16_t*)a->bias;
  k.residual = (const bf16_t*)a->residual;
  k.ldr = a->ldr;
  k.y = (bf16_t*)a->y;
  k.ldy = a->ldy;
  k.preact = (bf16_t*)a->preact;
  k.ldz = a->ldz;
  k.act = a->activation;
  return run_linear(k, eb, (char*)a->workspace, (hipStream_t)a->stream);
}

// ----------------------------------------------------------- linear gradient
// Workspace of the gradient: g (where the caller does not take it and one of
// its products reads it by rows), g^T, x^T, W^T, partial sums of db, then the larger of the two
// products' own.
struct GradWs {
  bool own_g;
  int64_t ldt, ldm;  // leading dimensions of g^T and x^T (tokens), of W^T (m)
  size_t off_g, off_gt, off_xt, off_wt, off_part, off_lin, bytes;
};

bool has_act(const ff_linear_grad_args* a) { return a->activation != FF_ACT_NONE; }

GradWs grad_ws(const ff_linear_grad_args* a) {
  GradWs w{};
  const size_t T = (size_t)a->tokens;
  w.ldt = (a->tokens + 7) / 8 * 8;
  w.ldm = (a->m + 7) / 8 * 8;
  // (whether the caller's g has rows that the tiles take does not matter: they are packed then)
  w.own_g = has_act(a) && a->g == nullptr && a->dx != nullptr;
  size_t off = 0;
  auto take = [&](bool need, size_t bytes) {
    const size_t at = off;
    if (need) off += up256(bytes);
    return at;
  };
  w.off_g = take(w.own_g, T * (size_t)w.ldm * 2);
  w.off_gt = take(a->dw != nullptr, (size_t)a->m * (size_t)w.ldt * 2);
  w.off_xt = take(a->dw != nullptr, (size_t)a->n * (size_t)w.ldt * 2);
  w.off_wt = take(a->dx != nullptr, (size_t)a->n * (size_t)w.ldm * 2);
  w.off_part = take(a->db != nullptr, (size_t)act_grad_parts(a->tokens) * (size_t)a->m * 4);
  w.off_lin = off;
  size_t lin = 0;
  if (a->dx != nullptr) {
    // the caller's g or dy may have to be packed: room for it whatever its alignment
    LinearPlan p = linear_plan(a->tokens, a->m, a->n, 2);
    lin = std::max(lin, up256(p.skinny ? 0 : T * (size_t)packed_ld(a->m, 2) * 2) +
                            up256(linear_partial_bytes(p, a->tokens, a->n)));
  }
  if (a->dw != nullptr) lin = std::max(lin, up256(linear_partial_bytes(linear_plan(a->m, w.ldt, a->n, 2), a->m, a->n)));
  w.bytes = off + lin;
  return w;
}

ff_status grad_checks(const ff_linear_grad_args* a) {
  if (a == nullptr) return bad("args is NULL");
  ff_status rc = linear_sizes(a->tokens, a->n, a->m);
  if (rc != FF_OK) return rc;
  if (a->tokens > (int64_t(1) << 21)) return bad("tokens must be <= 2^21");
  if (a->activation < FF_ACT_NONE || a->activation > FF_ACT_SILU) return bad("unknown activation");
  return FF_OK;
}

ff_status checkpoint_call(const ff_checkpoint_args* a, bool restore) {
  if (a == nullptr) return bad("args is NULL");
  if (a->rows < 0 || a->rows > (int64_t(1) << 32) || a->cols < 1 || a->cols > kMaxCols)
    return bad("rows must be 0 .. 2^32, cols 1 .. 2^24");
  if (a->dtype != FF_F32 && a->dtype != FF_BF16) return bad("unknown dtype");
  if (a->rows == 0) return FF_OK;
  const size_t eb = a->dtype == FF_BF16 ? 2 : 4;
  const ff_q8_rows& c = a->kept;
  if (!q8_ok(c, a->cols)) return bad(kBadQ8);
  if (!rows_ok(a->x, a->ldx, a->cols, eb)) return bad("x must be an aligned device pointer to rows of cols elements, ld >= cols");
  const int64_t groups = (a->cols + c.group - 1) / c.group, len = a->cols * (int64_t)eb;
  if (meet(a->x, a->rows, a->ldx * (int64_t)eb, len, c.q, a->rows, c.ldq, a->cols) ||
      meet(a->x, a->rows, a->ldx * (int64_t)eb, len, c.scale, a->rows, c.ld_scale * 4, groups * 4) ||
      meet(c.q, a->rows, c.ldq, a->cols, c.scale, a->rows, c.ld_scale * 4, groups * 4))
    return bad("x, the codes and their scales must not overlap");
  CheckpointArgs k{};
  k.rows = a->rows;
  k.cols = a->cols;
  k.x = a->x;
  k.ldx = a->ldx;
  k.q = c.q;
  k.ldq = c.ldq;
  k.scale = c.scale;
  k.lds = c.ld_scale;
  k.shift = __builtin_ctzll((unsigned long long)c.group);
  const hipStream_t s = (hipStream_t)a->stream;
  return restore ? hip(launch_restore(k, a->dtype == FF_BF16, s), "restoring a checkpoint")
                 : hip(launch_checkpoint(k, a->dtype == FF_BF16, s), "checkpoint");
}

}  // namespace

extern "C" {

ff_status ff_rms_norm(const ff_norm_args* a) {
  if (a == nullptr) return bad("args is NULL");
  ff_status rc = norm_sizes(a->rows, a->cols, a->dtype, a->eps);
  if (rc != FF_OK) return rc;
  if ((a->y == nullptr) == (a->q == nullptr)) return bad("give either y or q");
  if (a->normalise != 0 && a->normalise != 1) return bad("normalise must be 0 or 1");
  if (a->rows == 0) return FF_OK;
  const size_t eb = a->dtype == FF_BF16 ? 2 : 4;
  if (!rows_ok(a->x, a->ldx, a->cols, eb) || (a->residual != nullptr && !rows_ok(a->residual, a->ldr, a->cols, eb)) ||
      (a->sum != nullptr && !rows_ok(a->sum, a->ldsum, a->cols, eb)) ||
      (a->y != nullptr && !rows_ok(a->y, a->ldy, a->cols, eb)) || (a->q != nullptr && !rows_ok(a->q, a->ldq, a->cols, 1)))
    return bad("x, residual, sum, y and q must be aligned device pointers to rows of cols elements, ld >= cols");
  if ((uintptr_t)a->weight % eb != 0 || (uintptr_t)a->col_scale % 4 != 0) return bad("weight or col_scale is misaligned");
  if (a->q != nullptr && (a->q_scale == nullptr || (uintptr_t)a->q_scale % 4 != 0))
    return bad("q_scale must be an aligned device pointer");
  if (a->q == nullptr && a->col_scale != nullptr) return bad("col_scale belongs to q");
  const int64_t R = a->rows, len = a->cols * (int64_t)eb;
  auto clash = [&](const void* o, int64_t ldo, const void* in, int64_t ldi) {
    return meet(o, R, ldo * (int64_t)eb, len, in, R, ldi * (int64_t)eb, len) && !(o == in && ldo == ldi);
  };
  if (clash(a->sum, a->ldsum, a->x, a->ldx) || clash(a->sum, a->ldsum, a->residual, a->ldr) ||
      clash(a->y, a->ldy, a->x, a->ldx) || clash(a->y, a->ldy, a->residual, a->ldr) ||
      meet(a->y, R, a->ldy * (int64_t)eb, len, a->sum, R, a->ldsum * (int64_t)eb, len))
    return bad("sum and y must not overlap each other, nor x or residual other than as the same rows");
  const void* ins[3] = {a->x, a->residual, a->sum};
  const int64_t lds[3] = {a->ldx, a->ldr, a->ldsum};
  for (int k = 0; k < 3; ++k)
    if (meet(a->q, R, a->ldq, a->cols, ins[k], R, lds[k] * (int64_t)eb, len)) return bad("q must not overlap x, residual or sum");
  NormArgs k{};
  k.rows = a->rows;
  k.cols = a->cols;
  k.x = a->x;
  k.ldx = a->ldx;
  k.residual = a->residual;
  k.ldr = a->ldr;
  k.weight = a->weight;
  k.col_scale = a->col_scale;
  k.sum = a->sum;
  k.ldsum = a->ldsum;
  k.y = a->y;
  k.ldy = a->ldy;
  k.q = a->q;
  k.ldq = a->ldq;
  k.q_scale = a->q_scale;
  k.eps = eps_of(a->eps);
  k.normalise = a->normalise;
  return hip(launch_norm(k, a->dtype == FF_BF16, (hipStream_t)a->stream), "norm");
}

ff_status ff_rms_norm_backward_workspace_size(const ff_norm_grad_args* a, size_t* bytes) {
  if (a == nullptr || bytes == nullptr) return bad("args or bytes is NULL");
  ff_status rc = norm_sizes(a->rows, a->cols, a->dtype, a->eps);
  if (rc != FF_OK) return rc;
  *bytes = a->dweight != nullptr ? (size_t)norm_grad_parts(a->rows) * (size_t)a->cols * 4 : 0;
  return FF_OK;
}

ff_status ff_rms_norm_backward(const ff_norm_grad_args* a) {
  size_t need = 0;
  ff_status rc = ff_rms_norm_backward_workspace_size(a, &need);
  if (rc != FF_OK) return rc;
  const bool bf16 = a->dtype == FF_BF16;
  const size_t eb = bf16 ? 2 : 4;
  const hipStream_t s = (hipStream_t)a->stream;
  if ((uintptr_t)a->weight % eb != 0 || (uintptr_t)a->dweight % eb != 0) return bad("weight or dweight is misaligned");
  if (a->rows == 0) {
    if (a->dweight == nullptr) return FF_OK;
    return hip(launch_zero(a->dweight, a->cols, 1, a->cols, (int)eb, s), "zero gradient");
  }
  if (!rows_ok(a->s, a->lds, a->cols, eb) || !rows_ok(a->dy, a->lddy, a->cols, eb) ||
      !rows_ok(a->ds, a->ldds, a->cols, eb) || (a->dsum != nullptr && !rows_ok(a->dsum, a->lddsum, a->cols, eb)))
    return bad("s, dy, dsum and ds must be aligned device pointers to rows of cols elements, ld >= cols");
  const int64_t R = a->rows, len = a->cols * (int64_t)eb;
  auto clash = [&](const void* in, int64_t ldi) {
    return meet(a->ds, R, a->ldds * (int64_t)eb, len, in, R, ldi * (int64_t)eb, len) && !(a->ds == in && a->ldds == ldi);
  };
  if (clash(a->s, a->lds) || clash(a->dy, a->lddy) || clash(a->dsum, a->lddsum))
    return bad("ds must not overlap s, dy or dsum other than as the same rows");
  if ((rc = workspace_ok(a->workspace, a->workspace_bytes, need)) != FF_OK) return rc;
  NormGradArgs k{};
  k.rows = a->rows;
  k.cols = a->cols;
  k.s = a->s;
  k.lds = a->lds;
  k.dy = a->dy;
  k.lddy = a->lddy;
  k.dsum = a->dsum;
  k.lddsum = a->lddsum;
  k.weight = a->weight;
  k.dx = a->ds;
  k.lddx = a->ldds;
  k.part = a->dweight != nullptr ? (float*)a->workspace : nullptr;
  k.eps = eps_of(a->eps);
  if ((rc = hip(launch_norm_grad(k, bf16, s), "norm gradient")) != FF_OK || a->dweight == nullptr) return rc;
  return hip(launch_col_sums(k.part, norm_grad_parts(a->rows), a->cols, a->dweight, bf16, s), "norm gradient's sums");
}

ff_status ff_linear_workspace_size(const ff_linear_args* a, int q8, size_t* bytes) {
  if (bytes == nullptr) return bad("bytes is NULL");
  ff_status rc = linear_checks(a, q8 != 0);
  if (rc != FF_OK) return rc;
  *bytes = a->tokens == 0 ? 0 : linear_ws(a->tokens, a->n, a->m, a->x, a->ldx, a->w, a->ldw, q8 ? 1 : 2).bytes;
  return FF_OK;
}

ff_status ff_linear(const ff_linear_args* a) { return linear_call(a, false); }

ff_status ff_linear_q8(const ff_linear_args* a) { return linear_call(a, true); }

ff_status ff_linear_backward_workspace_size(const ff_linear_grad_args* a, size_t* bytes) {
  if (bytes == nullptr) return bad("bytes is NULL");
  ff_status rc = grad_checks(a);
  if (rc != FF_OK) return rc;
  *bytes = a->tokens == 0 ? 0 : grad_ws(a).bytes;
  return FF_OK;
}

ff_status ff_linear_backward(const ff_linear_grad_args* a) {
  ff_status rc = grad_checks(a);
  if (rc != FF_OK) return rc;
  const hipStream_t s = (hipStream_t)a->stream;
  if ((uintptr_t)a->db % 2 != 0) return bad("db is misaligned");
  if (a->dw != nullptr && !rows_ok(a->dw, a->lddw, a->n, 2)) return bad("dw must be an aligned device pointer to rows of n elements, ld >= n");
  if (a->tokens == 0) {
    if (a->dw != nullptr && (rc = hip(launch_zero(a->dw, a->lddw, a->m, a->n, 2, s), "zero gradient")) != FF_OK) return rc;
    if (a->db != nullptr) return hip(launch_zero(a->db, a->m, 1, a->m, 2, s), "zero gradient");
    return FF_OK;
  }
  if (!rows_ok(a->dy, a->lddy, a->m, 2) || (has_act(a) && !rows_ok(a->preact, a->ldz, a->m, 2)) ||
      (a->g != nullptr && !rows_ok(a->g, a->ldg, a->m, 2)))
    return bad("dy, g and (with an activation) preact must be aligned device pointers to rows of m elements, ld >= m");
  if ((a->dw != nullptr && !rows_ok(a->x, a->ldx, a->n, 2)) || (a->dx != nullptr && !rows_ok(a->w, a->ldw, a->n, 2)) ||
      (a->dx != nullptr && !rows_ok(a->dx, a->lddx, a->n, 2)))
    return bad("x (for dw), w and dx must be aligned device pointers to rows of n elements, ld >= n");
  const int64_t T = a->tokens, n2 = a->n * 2, m2 = a->m * 2;
  struct Block {
    const void* p;
    int64_t rows, stride, len;
  };
  const Block ins[4] = {{a->dy, T, a->lddy * 2, m2}, {a->x, T, a->ldx * 2, n2}, {a->w, a->m, a->ldw * 2, n2},
                        {has_act(a) ? a->preact : nullptr, T, a->ldz * 2, m2}};
  const Block outs[4] = {{a->g, T, a->ldg * 2, m2}, {a->dx, T, a->lddx * 2, n2}, {a->dw, a->m, a->lddw * 2, n2},
                         {a->db, a->db != nullptr ? 1 : 0, m2, m2}};
  for (int i = 0; i < 4; ++i) {
    for (const Block& in : ins)
      if (meet(outs[i].p, outs[i].rows, outs[i].stride, outs[i].len, in.p, in.rows, in.stride, in.len))
        return bad("gradients must not overlap the inputs");
    for (int j = 0; j < i; ++j)
      if (meet(outs[i].p, outs[i].rows, outs[i].stride, outs[i].len, outs[j].p, outs[j].rows, outs[j].stride, outs[j].len))
        return bad("gradients must not overlap each other");
  }
  const GradWs w = grad_ws(a);
  if ((rc = workspace_ok(a->workspace, a->workspace_bytes, w.bytes)) != FF_OK) return rc;
  char* ws = (char*)a->workspace;
  ActGradArgs k{};
  k.rows = T;
  k.cols = a->m;
  k.dy = (const bf16_t*)a->dy;
  k.lddy = a->lddy;
  k.z = has_act(a) ? (const bf16_t*)a->preact : nullptr;
  k.ldz = a->ldz;
  k.act = a->activation;
  const bf16_t* g = k.dy;  // by rows
  int64_t ldg = a->lddy;
  if (a->g != nullptr) {
    k.g = (bf16_t*)a->g;
    k.ldg = a->ldg;
  } else if (w.own_g) {
    k.g = (bf16_t*)(ws + w.off_g);
    k.ldg = w.ldm;
  }
  if (k.g != nullptr) {
    g = k.g;
    ldg = k.ldg;
  }
  k.gt = a->dw != nullptr ? (bf16_t*)(ws + w.off_gt) : nullptr;
  k.ldgt = w.ldt;
  k.part = a->db != nullptr ? (float*)(ws + w.off_part) : nullptr;
  // one launch for what the products read: g by rows and columns, W^T and x^T
  ActGradArgs jobs[3];
  int count = 0;
  if (k.g != nullptr || k.gt != nullptr || k.part != nullptr) jobs[count++] = k;
  auto turn = [&](const void* src, int64_t ld, int64_t rows, int64_t cols, size_t off, int64_t ldt) {
    ActGradArgs j{};
    j.rows = rows;
    j.cols = cols;
    j.dy = (const bf16_t*)src;
    j.lddy = ld;
    j.gt = (bf16_t*)(ws + off);
    j.ldgt = ldt;
    jobs[count++] = j;
    return j.gt;
  };
  const bf16_t* wt = a->dx != nullptr ? turn(a->w, a->ldw, a->m, a->n, w.off_wt, w.ldm) : nullptr;
  const bf16_t* xt = a->dw != nullptr ? turn(a->x, a->ldx, T, a->n, w.off_xt, w.ldt) : nullptr;
  if (count > 0 && (rc = hip(launch_act_grad(jobs, count, s), "operands of the gradient")) != FF_OK) return rc;
  if (a->db != nullptr &&
      (rc = hip(launch_col_sums(k.part, act_grad_parts(T), a->m, a->db, true, s), "bias gradient")) != FF_OK)
    return rc;
  if (a->dx != nullptr) {
    LinearArgs p{};
    p.tokens = T;
    p.n = a->m;
    p.m = a->n;
    p.x = g;
    p.ldx = ldg;
    p.w = wt;
    p.ldw = w.ldm;
    p.y = (bf16_t*)a->dx;
    p.ldy = a->lddx;
    if ((rc = run_linear(p, 2, ws + w.off_lin, s, true)) != FF_OK) return rc;
  }
  if (a->dw != nullptr) {
    LinearArgs p{};
    p.tokens = a->m;
    p.n = w.ldt;  // (zeros beyond the tokens)
    p.m = a->n;
    p.x = k.gt;
    p.ldx = w.ldt;
    p.w = xt;
    p.ldw = w.ldt;
    p.y = (bf16_t*)a->dw;
    p.ldy = a->lddw;
    if ((rc = run_linear(p, 2, ws + w.off_lin, s)) != FF_OK) return rc;
  }
  return FF_OK;
}

ff_status ff_checkpoint(const ff_checkpoint_args* a) { return checkpoint_call(a, false); }

ff_status ff_checkpoint_restore(const ff_checkpoint_args* a) { return checkpoint_call(a, true); }

ff_status ff_orthogonalize_workspace_size(const ff_ortho_args* a, size_t* bytes) {
  if (a == nullptr || bytes == nullptr) return bad("args or bytes is NULL");
  if (a->batch < 0 || a->batch > 65535 || a->m < 1 || a->n < 1 || a->m > kMaxDim || a->n > kMaxDim)
    return bad("batch must be 0 .. 65535, m and n 1 .. 2^20");
  if (a->dtype != FF_F32 && a->dtype != FF_BF16) return bad("unknown dtype");
  *bytes = a->batch == 0 ? 0 : ortho_workspace(a->batch, a->m, a->n, a->dtype == FF_BF16);
  return FF_OK;
}

ff_status ff_orthogonalize(const ff_ortho_args* a) {
  size_t need = 0;
  ff_status rc = ff_orthogonalize_workspace_size(a, &need);
  if (rc != FF_OK) return rc;
  if (a->steps < 1 || a->steps > 64) return bad("steps must be 1 .. 64");
  for (double v : {a->a, a->b, a->c, a->eps, a->scale})
    if (!std::isfinite(v)) return bad("a, b, c, eps and scale must be finite");
  if (a->eps < 0.0) return bad("eps must be >= 0");
  if (!std::isfinite((float)a->scale)) return bad("scale must be in fp32's range");
  if (!ortho_bounded(a->steps, a->a, a->b, a->c))
    return bad("the coefficients take singular values in [0, 1] to 16 or more");
  if (a->batch == 0) return FF_OK;
  const size_t eb = a->dtype == FF_BF16 ? 2 : 4;
  if (!rows_ok(a->G, a->ldg, a->n, eb) || !rows_ok(a->out, a->ldo, a->n, eb))
    return bad("G and out must be aligned device pointers to rows of n elements, ld >= n");
  const int64_t span_g = (a->m - 1) * a->ldg + a->n, span_o = (a->m - 1) * a->ldo + a->n;
  if (a->batch > 1 && (a->stride_g < 0 || a->stride_g > kMaxRows || a->stride_o < span_o || a->stride_o > kMaxRows))
    return bad("stride_g must be >= 0 and stride_o at least a matrix");
  const int64_t sg = a->batch > 1 ? a->stride_g : span_g, so = a->batch > 1 ? a->stride_o : span_o;
  if (meet(a->G, a->batch, sg * (int64_t)eb, span_g * (int64_t)eb, a->out, a->batch, so * (int64_t)eb,
           span_o * (int64_t)eb))
    return bad("out must not overlap G");
  if ((rc = workspace_ok(a->workspace, a->workspace_bytes, need)) != FF_OK) return rc;
  OrthoArgs k{};
  k.batch = a->batch;
  k.m = a->m;
  k.n = a->n;
  k.g = a->G;
  k.ldg = a->ldg;
  k.sg = sg;
  k.out = a->out;
  k.ldo = a->ldo;
  k.so = so;
  k.steps = a->steps;
  k.a = (float)a->a;
  k.b = (float)a->b;
  k.c = (float)a->c;
  k.eps = a->eps;
  k.scale = (float)a->scale;
  k.bf16 = a->dtype == FF_BF16;
  return hip(launch_ortho(k, a->workspace, (hipStream_t)a->stream), "orthogonalisation");
}

}  // extern "C"
