// C ABI of the operators around a layer of experts (ff.h): argument checks, workspace
// layout and the order of the kernels' launches.  No state is kept.
#include <math.h>

#include <algorithm>
#include <initializer_list>
#include <utility>

#include "ff.h"
#include "ff_expert_kernels.hpp"
#include "ff_layer_checks.hpp"

using namespace ff;

namespace {

constexpr int64_t kMaxSlots = int64_t(1) << 24;

// A block of memory: rows of `len` bytes, `stride` apart.
struct Block {
  const void* p;
  int64_t rows, stride, len;
};
Block flat(const void* p, int64_t bytes) { return {p, p != nullptr && bytes > 0 ? 1 : 0, bytes, bytes}; }
bool meets(const Block& a, const Block& b) { return meet(a.p, a.rows, a.stride, a.len, b.p, b.rows, b.stride, b.len); }
// Whether an output meets an input or another output.
bool clash(std::initializer_list<Block> outs, std::initializer_list<Block> ins) {
  for (auto o = outs.begin(); o != outs.end(); ++o) {
    for (const Block& i : ins)
      if (meets(*o, i)) return true;
    for (auto p = outs.begin(); p != o; ++p)
      if (meets(*o, *p)) return true;
  }
  return false;
}
constexpr const char* kClash = "outputs must not overlap the inputs or each other";

// ------------------------------------------------------------------- routing
ff_status slots_ok(int64_t tokens, int64_t experts, int64_t top) {
  if (experts < 1 || experts > kMaxExperts) return bad("experts must be 1 .. 1024");
  if (top < 1 || top > kMaxTop) return bad("top must be 1 .. 64");
  if (tokens < 0 || tokens > kMaxSlots || tokens * top > kMaxSlots) return bad("tokens top must be 0 .. 2^24");
  return FF_OK;
}

ff_status route_call(const ff_route_args* a, bool choose) {
  if (a == nullptr) return bad("args is NULL");
  ff_status rc = slots_ok(a->tokens, a->experts, a->top);
  if (rc != FF_OK) return rc;
  const int64_t groups = a->groups == 0 ? 1 : a->groups, top_groups = groups == 1 ? 1 : a->top_groups;
  const bool sort = !choose || a->order != nullptr;
  if (choose) {
    if (a->dtype != FF_F32 && a->dtype != FF_BF16) return bad("unknown dtype");
    if (a->score != FF_SCORE_SOFTMAX && a->score != FF_SCORE_SIGMOID) return bad("unknown score");
    if (groups < 1 || groups > kMaxGroups || a->experts % groups != 0) return bad("groups must be 1 .. 64 and divide experts");
    if (top_groups < 1 || top_groups > groups) return bad("top_groups must be 1 .. groups");
    if (a->top > top_groups * (a->experts / groups)) return bad("top must not exceed the experts of top_groups groups");
    if (a->renormalise != 0 && a->renormalise != 1) return bad("renormalise must be 0 or 1");
    if (!std::isfinite((float)a->scale)) return bad("scale must be finite in fp32");
  }
  const hipStream_t s = (hipStream_t)a->stream;
  if (a->tokens == 0) {
    if (a->offsets == nullptr) return FF_OK;
    if ((uintptr_t)a->offsets % 4 != 0) return bad("offsets is misaligned");
    return hip(launch_zero(a->offsets, a->experts + 1, 1, a->experts + 1, 4, s), "offsets");
  }
  if (sort && (a->order == nullptr || a->offsets == nullptr || a->place == nullptr))
    return bad("give order, offsets and place, or (ff_route) none of them");
  if (!sort && (a->offsets != nullptr || a->place != nullptr)) return bad("give order, offsets and place, or none of them");
  if ((uintptr_t)a->order % 4 != 0 || (uintptr_t)a->offsets % 4 != 0 || (uintptr_t)a->place % 4 != 0)
    return bad("order, offsets or place is misaligned");
  const int64_t T = a->tokens, S = T * a->top;
  if (a->chosen == nullptr || (uintptr_t)a->chosen % 4 != 0) return bad("chosen must be an aligned device pointer");
  const size_t eb = a->dtype == FF_BF16 ? 2 : 4;
  if (choose) {
    if (!rows_ok(a->logits, a->ldl, a->experts, eb)) return bad("logits must be an aligned device pointer to rows of experts elements, ld >= experts");
    if (a->weights == nullptr || (uintptr_t)a->weights % 4 != 0 || (uintptr_t)a->bias % 4 != 0)
      return bad("weights and bias must be aligned device pointers");
  }
  const Block order = flat(a->order, S * 4), offsets = flat(a->offsets, (a->experts + 1) * 4), place = flat(a->place, S * 4);
  const Block chosen = flat(a->chosen, S * 4);
  if (choose ? clash({flat(a->weights, S * 4), chosen, order, offsets, place},
                     {{a->logits, T, a->ldl * (int64_t)eb, a->experts * (int64_t)eb}, flat(a->bias, a->experts * 4), flat(a->mask, T)})
             : clash({order, offsets, place}, {chosen}))
    return bad(kClash);
  if (sort) {
    rc = workspace_ok(a->workspace, a->workspace_bytes, route_workspace(T, (int)a->experts, (int)a->top));
    if (rc != FF_OK) return rc;
  }
  RouteArgs k{};
  k.tokens = T;
  k.experts = (int)a->experts;
  k.top = (int)a->top;
  k.logits = a->logits;
  k.ldl = a->ldl;
  k.bf16 = a->dtype == FF_BF16;
  k.bias = a->bias;
  k.mask = a->mask;
  k.sigmoid = a->score == FF_SCORE_SIGMOID;
  k.groups = (int)groups;
  k.top_groups = (int)top_groups;
  k.renormalise = a->renormalise != 0;
  k.scale = a->scale;
  k.weights = a->weights;
  k.chosen = a->chosen;
  k.order = a->order;
  k.offsets = a->offsets;
  k.place = a->place;
  return choose ? hip(launch_route(k, a->workspace, s), "routing") : hip(launch_order(k, a->workspace, s), "order of slots");
}

// ---------------------------------------------------------------- the products
// Which arrays of a routing a call reads.
enum Reads : int { kOrder = 1, kOffsets = 2, kPlace = 4, kWeights = 8 };

ff_status routing_ok(const ff_routing& r, int reads) {
  ff_status rc = slots_ok(r.tokens, r.experts, r.top);
  if (rc != FF_OK || r.tokens == 0) return rc;
  for (auto& p : {std::make_pair(kOrder, (const void*)r.order), std::make_pair(kOffsets, (const void*)r.offsets),
                  std::make_pair(kPlace, (const void*)r.place), std::make_pair(kWeights, (const void*)r.weights)})
    if ((reads & p.first) && (p.second == nullptr || (uintptr_t)p.second % 4 != 0))
      return bad("the routing's arrays must be aligned device pointers");
  return FF_OK;
}
SlotRows slot_rows(const ff_routing& r) {
  SlotRows at{};
  at.tokens = r.tokens;
  at.rows = r.tokens * r.top;
  at.experts = (int)r.experts;
  at.top = (int)r.top;
  at.order = r.order;
  at.offsets = r.offsets;
  at.place = r.place;
  at.weights = r.weights;
  return at;
}
Block block_of(const ff_routing& r, int which) {
  const int64_t S = r.tokens * r.top * 4;
  return which == kOrder ? flat(r.order, S) : which == kOffsets ? flat(r.offsets, (r.experts + 1) * 4)
         : which == kPlace ? flat(r.place, S) : flat(r.weights, S);
}

ff_status sizes_ok(int64_t n, int64_t m) {
  return n < 1 || m < 1 || n > kMaxDim || m > kMaxDim ? bad("n and m must be 1 .. 2^20") : FF_OK;
}

// Rows of x for the tiles: as they lie, packed, or a row for each slot where the
// tokens' rows lie too far apart for the tiles' 32-bit offsets.
struct ForwardWs {
  ExpertPlan plan;
  bool pack_x, pack_w, gather_x;
  size_t off_w, bytes;
};
ForwardWs forward_ws(const ff_expert_linear_args* a) {
  ForwardWs w{};
  const int64_t T = a->routing.tokens, S = T * a->routing.top;
  const bool w_lies = tile_rows_ok(a->w, a->ldw, a->n, 2);
  w.plan = expert_plan(S, (int)a->routing.experts, a->n, a->m, w_lies);
  if (w.plan.nt > 0) return w;
  w.pack_w = !w_lies;
  w.pack_x = !tile_rows_ok(a->x, a->ldx, a->n, 2);
  w.gather_x = a->by_slot == 0 && (T * (w.pack_x ? packed_ld(a->n, 2) : a->ldx) + a->n) * 2 > int64_t(0x7fffffff);
  if (w.gather_x) w.pack_x = false;
  if (w.pack_x || w.gather_x)
    w.off_w = up256((size_t)(w.gather_x || a->by_slot ? S : T) * (size_t)packed_ld(a->n, 2) * 2);
  w.bytes = w.off_w + (w.pack_w ? up256((size_t)a->routing.experts * (size_t)a->m * (size_t)packed_ld(a->n, 2) * 2) : 0);
  return w;
}

ff_status forward_sizes(const ff_expert_linear_args* a) {
  if (a == nullptr) return bad("args is NULL");
  ff_status rc = slots_ok(a->routing.tokens, a->routing.experts, a->routing.top);
  if (rc != FF_OK || (rc = sizes_ok(a->n, a->m)) != FF_OK) return rc;
  if (a->by_slot != 0 && a->by_slot != 1) return bad("by_slot must be 0 or 1");
  return FF_OK;
}

// ------------------------------------------------------------------ gradients
// The gradient of a layer of experts, or (at.offsets null) of one plain layer.
struct Gradient {
  SlotRows at;
  int64_t n, m;
  bool dy_f32;
  const void* dy;
  int64_t lddy;
  bool gather;  // x and dx: the tokens' rows
  const void* x;
  int64_t ldx;
  ff_q8_rows x_q8;
  const void* w;
  int64_t ldw;
  int act;
  const void* z;
  int64_t ldz;
  ff_q8_rows z_q8;
  void *g, *dx, *dw, *db;
  int64_t ldg, lddx, lddw;
};

// Workspace: g and x as the products read them, in bf16 or (x from a checkpoint) in
// fp16 with their peaks, W with its rows laid out, and fp32 results before they are summed.
struct GradWs {
  ExpertPlan dx, dw;
  bool dy_is_g, lay_g, scale, lay_x, lay_w, sum_dx;
  size_t off_g, off_g16, off_x, off_peaks, off_w, off_parts, off_sum_x, off_sum_w, bytes;
};

GradWs grad_ws(const Gradient& a) {
  GradWs w{};
  const int64_t S = a.at.rows, E = a.at.experts;
  const bool dx = a.dx != nullptr, dw = a.dw != nullptr;
  w.scale = dw && a.x_q8.q != nullptr;
  // g in rows that the tiles take: dy itself, the caller's, or a copy
  w.dy_is_g = a.act == FF_ACT_NONE && !a.dy_f32 && a.g == nullptr && a.at.offsets == nullptr && tile_rows_ok(a.dy, a.lddy, a.m, 2);
  w.lay_g = (dx || (dw && !w.scale)) && !w.dy_is_g && (a.g == nullptr || !tile_rows_ok(a.g, a.ldg, a.m, 2));
  w.lay_x = dw && !w.scale && (a.gather || !tile_rows_ok(a.x, a.ldx, a.n, 2));
  w.lay_w = dx && !tile_rows_ok(a.w, a.ldw, a.n, 2);
  size_t off = 0;
  auto take = [&](bool need, size_t bytes) {
    const size_t at = off;
    if (need) off += up256(bytes);
    return at;
  };
  w.off_g = take(w.lay_g, (size_t)S * (size_t)laid_ld(a.m) * 2);
  w.off_g16 = take(w.scale, (size_t)S * (size_t)laid_ld(a.m) * 2);
  w.off_x = take(w.lay_x || w.scale, (size_t)S * (size_t)laid_ld(a.n) * 2);
  w.off_peaks = take(w.scale, 2 * kPeaks * 4 + 8);  // and what takes g and x back
  w.off_parts = take(a.db != nullptr, (size_t)part_count(S, (int)E, a.m) * (size_t)laid_ld(a.m) * 4);
  w.off_w = take(w.lay_w, (size_t)E * (size_t)a.m * (size_t)laid_ld(a.n) * 2);
  if (dx) {
    w.dx = expert_dx_plan(S, (int)E, a.n, a.m);
    w.sum_dx = a.gather || w.dx.splits > 1;
    w.off_sum_x = take(w.sum_dx, (size_t)w.dx.splits * (size_t)S * (size_t)laid_ld(a.n) * 4);
  }
  if (dw) {
    w.dw = expert_dw_plan(S, (int)E, a.n, a.m);
    w.off_sum_w = take(w.dw.splits > 1, (size_t)w.dw.splits * (size_t)E * (size_t)a.m * (size_t)laid_ld(a.n) * 4);
  }
  w.bytes = off;
  return w;
}

// bf16 rows of dst from `parts` sums of fp32 rows.
ff_status sum_parts(const float* parts, int count, int64_t rows, int64_t cols, void* dst, int64_t ld, hipStream_t s) {
  CombineArgs c{};
  c.at.tokens = c.at.rows = rows;
  c.at.experts = c.at.top = 1;
  c.cols = cols;
  c.y = parts;
  c.ldy = laid_ld(cols);
  c.f32 = true;
  c.parts = count;
  c.part_stride = rows * c.ldy;
  c.out = (bf16_t*)dst;
  c.ldo = ld;
  return hip(launch_combine(c, s), "sums of parts");
}

ff_status run_gradient(const Gradient& a, const GradWs& w, char* ws, hipStream_t s) {
  ff_status rc;
  const int64_t S = a.at.rows, E = a.at.experts;
  const bool act = a.act != FF_ACT_NONE;
  uint32_t* peaks = (uint32_t*)(ws + w.off_peaks);
  float* inverse = (float*)(peaks + 2 * kPeaks);
  RowsArgs jobs[3];
  int count = 0;
  RowsArgs r{};
  r.at = a.at;
  r.cols = a.m;
  r.src = a.dy;
  r.lds = a.lddy;
  r.src_f32 = a.dy_f32;
  r.act = a.act;
  if (act) {
    r.z = (const bf16_t*)a.z;
    r.ldz = a.ldz;
    r.z_q8 = q8_of(a.z_q8);
  }
  if (w.scale) {
    RowsArgs x{};
    x.at = a.at;
    x.gather = a.gather;
    x.cols = (a.n + a.x_q8.group - 1) / a.x_q8.group;
    x.src = a.x_q8.scale;
    x.lds = a.x_q8.ld_scale;
    x.src_f32 = true;
    if ((rc = hip(launch_peaks(r, peaks, x, peaks + kPeaks, s), "peaks of g and x")) != FF_OK) return rc;
  }
  r.out = (bf16_t*)a.g;
  r.ldo = a.ldg;
  if (w.lay_g) r.laid = (uint16_t*)(ws + w.off_g);
  if (w.scale) {
    r.scaled = (uint16_t*)(ws + w.off_g16);
    r.peaks = peaks;
    r.peak_factor = 1.0f;
    r.inverse = inverse;
  }
  if (a.db != nullptr) r.parts = (float*)(ws + w.off_parts);
  if (r.out != nullptr || r.laid != nullptr || r.scaled != nullptr || r.parts != nullptr) jobs[count++] = r;
  ExpertGradArgs k{};
  k.at = a.at;
  k.n = a.n;
  k.m = a.m;
  k.g = w.lay_g ? r.laid : (const uint16_t*)(w.dy_is_g ? a.dy : a.g);
  k.ldg = w.lay_g ? laid_ld(a.m) : w.dy_is_g ? a.lddy : a.ldg;
  k.w = (const bf16_t*)a.w;
  k.ldw = a.ldw;
  k.x = (const uint16_t*)a.x;
  k.ldx = a.ldx;
  if (w.lay_x || w.scale) {
    RowsArgs x{};
    x.at = a.at;
    x.gather = a.gather;
    x.cols = a.n;
    x.src = a.x;
    x.lds = a.ldx;
    if (w.scale) {
      x.src_q8 = q8_of(a.x_q8);
      x.scaled = (uint16_t*)(ws + w.off_x);
      x.peaks = peaks + kPeaks;
      x.peak_factor = 127.0f;  // (codes end there)
      x.inverse = inverse + 1;
    } else {
      x.laid = (uint16_t*)(ws + w.off_x);
    }
    jobs[count++] = x;
    k.x = (const uint16_t*)(ws + w.off_x);
    k.ldx = laid_ld(a.n);
  }
  if (w.lay_w) {
    RowsArgs p{};
    p.at.tokens = p.at.rows = E * a.m;
    p.at.experts = p.at.top = 1;
    p.cols = a.n;
    p.src = a.w;
    p.lds = a.ldw;
    p.laid = (uint16_t*)(ws + w.off_w);
    jobs[count++] = p;
    k.w = (const bf16_t*)(ws + w.off_w);
    k.ldw = laid_ld(a.n);
  }
  if (count > 0 && (rc = hip(launch_rows(jobs, count, s), "operands of the gradient")) != FF_OK) return rc;
  k.db = (bf16_t*)a.db;
  k.parts = r.parts;
  k.part_rows = part_rows(S, a.m);
  if (a.db != nullptr && a.dw == nullptr && (rc = hip(launch_expert_db(k, s), "bias gradient")) != FF_OK) return rc;
  ExpertGradArgs x = k;
  float *sum_x = (float*)(ws + w.off_sum_x), *sum_w = (float*)(ws + w.off_sum_w);
  x.out_f32 = w.sum_dx;
  x.out = w.sum_dx ? (void*)sum_x : a.dx;
  x.ldo = w.sum_dx ? laid_ld(a.n) : a.lddx;
  x.part_stride = S * x.ldo;
  if (w.scale) {
    k.f16 = true;
    k.g = (const uint16_t*)(ws + w.off_g16);
    k.ldg = laid_ld(a.m);
    k.inverse = inverse;
  }
  k.out_f32 = w.dw.splits > 1;
  k.out = k.out_f32 ? (void*)sum_w : a.dw;
  k.ldo = k.out_f32 ? laid_ld(a.n) : a.lddw;
  k.part_stride = E * a.m * k.ldo;
  const bool both = a.dx != nullptr && a.dw != nullptr && expert_both(w.dx, w.dw);
  if (both && (rc = hip(launch_expert_both(x, w.dx, k, w.dw, s), "gradients")) != FF_OK) return rc;
  if (a.dx != nullptr) {
    if (!both && (rc = hip(launch_expert_dx(x, w.dx, s), "input gradient")) != FF_OK) return rc;
    if (a.gather) {
      // a token's rows in fp32 until they are summed: a rounding of each would add to g's and dx's own
      CombineArgs c{};
      c.at = k.at;
      c.at.weights = nullptr;
      c.cols = a.n;
      c.y = sum_x;
      c.ldy = x.ldo;
      c.f32 = true;
      c.parts = w.dx.splits;
      c.part_stride = x.part_stride;
      c.out = (bf16_t*)a.dx;
      c.ldo = a.lddx;
      if ((rc = hip(launch_combine(c, s), "input gradient's sums")) != FF_OK) return rc;
    } else if (w.sum_dx && (rc = sum_parts(sum_x, w.dx.splits, S, a.n, a.dx, a.lddx, s)) != FF_OK) {
      return rc;
    }
  }
  if (a.dw == nullptr) return FF_OK;
  if (!both && (rc = hip(launch_expert_dw(k, w.dw, s), "weight gradient")) != FF_OK) return rc;
  return k.out_f32 ? sum_parts(sum_w, w.dw.splits, E * a.m, a.n, a.dw, a.lddw, s) : FF_OK;
}

// What the layers' gradients check alike (rows of dy: S, of x and dx: X).
ff_status gradient_ok(const Gradient& a, int64_t S, int64_t X, std::initializer_list<Block> more) {
  const int64_t E = a.at.experts;
  const bool act = a.act != FF_ACT_NONE, x8 = a.x_q8.q != nullptr, z8 = a.z_q8.q != nullptr && act;
  if ((x8 && a.x != nullptr) || (a.z_q8.q != nullptr && a.z != nullptr))
    return bad("give x and preact either in bf16 or as a checkpoint");
  if ((x8 && !q8_ok(a.x_q8, a.n)) || (z8 && !q8_ok(a.z_q8, a.m))) return bad(kBadQ8);
  const int64_t e = a.dy_f32 ? 4 : 2;
  if (!rows_ok(a.dy, a.lddy, a.m, e) || (act && !z8 && !rows_ok(a.z, a.ldz, a.m, 2)) ||
      (a.g != nullptr && !rows_ok(a.g, a.ldg, a.m, 2)))
    return bad("dy, g and (with an activation) preact must be aligned device pointers to rows of m elements, ld >= m");
  if ((a.dw != nullptr && !x8 && !rows_ok(a.x, a.ldx, a.n, 2)) || (a.dx != nullptr && !rows_ok(a.w, a.ldw, a.n, 2)) ||
      (a.dx != nullptr && !rows_ok(a.dx, a.lddx, a.n, 2)))
    return bad("x (for dw), w and dx must be aligned device pointers to rows of n elements, ld >= n");
  auto scales = [&](bool there, const ff_q8_rows& c, int64_t rows, int64_t cols) {
    return there ? Block{c.scale, rows, c.ld_scale * 4, (cols + c.group - 1) / c.group * 4} : Block{nullptr, 0, 0, 0};
  };
  const std::initializer_list<Block> outs = {{a.g, a.g != nullptr ? S : 0, a.ldg * 2, a.m * 2},
                                             {a.dx, a.dx != nullptr ? X : 0, a.lddx * 2, a.n * 2},
                                             {a.dw, a.dw != nullptr ? E * a.m : 0, a.lddw * 2, a.n * 2},
                                             flat(a.db, E * a.m * 2)};
  if (clash(outs, {{a.dy, S, a.lddy * e, a.m * e},
                   {a.x, a.x != nullptr ? X : 0, a.ldx * 2, a.n * 2},
                   {a.w, a.w != nullptr ? E * a.m : 0, a.ldw * 2, a.n * 2},
                   {a.z, act && !z8 ? S : 0, a.ldz * 2, a.m * 2},
                   {a.x_q8.q, x8 ? X : 0, a.x_q8.ldq, a.n},
                   {a.z_q8.q, z8 ? S : 0, a.z_q8.ldq, a.m},
                   scales(x8, a.x_q8, X, a.n),
                   scales(z8, a.z_q8, S, a.m)}) ||
      clash(outs, more))
    return bad("gradients must not overlap the inputs or each other");
  return FF_OK;
}

// With no tokens.
ff_status zero_gradient(const Gradient& a, hipStream_t s) {
  const int64_t E = a.at.experts;
  ff_status rc = FF_OK;
  if (a.dw != nullptr) rc = hip(launch_zero(a.dw, a.lddw, E * a.m, a.n, 2, s), "zero gradient");
  if (rc == FF_OK && a.db != nullptr) rc = hip(launch_zero(a.db, E * a.m, 1, E * a.m, 2, s), "zero gradient");
  return rc;
}

Gradient gradient_of(const ff_expert_grad_args* a) {
  Gradient k{};
  k.at = slot_rows(a->routing);
  k.n = a->n;
  k.m = a->m;
  k.dy_f32 = a->dy_dtype == FF_F32;
  k.dy = a->dy;
  k.lddy = a->lddy;
  k.gather = a->by_slot == 0;
  k.x = a->x;
  k.ldx = a->ldx;
  k.x_q8 = a->x_q8;
  k.w = a->w;
  k.ldw = a->ldw;
  k.act = a->activation;
  k.z = a->preact;
  k.ldz = a->ldz;
  k.z_q8 = a->preact_q8;
  k.g = a->g;
  k.ldg = a->ldg;
  k.dx = a->dx;
  k.lddx = a->lddx;
  k.dw = a->dw;
  k.lddw = a->lddw;
  k.db = a->db;
  return k;
}
// A plain layer: all rows are one expert's.
Gradient gradient_of(const ff_linear_grad_q8_args* a) {
  const ff_linear_grad_args& b = a->grad;
  Gradient k{};
  k.at.tokens = k.at.rows = b.tokens;
  k.at.experts = k.at.top = 1;
  k.n = b.n;
  k.m = b.m;
  k.dy = b.dy;
  k.lddy = b.lddy;
  k.x = b.x;
  k.ldx = b.ldx;
  k.x_q8 = a->x_q8;
  k.w = b.w;
  k.ldw = b.ldw;
  k.act = b.activation;
  k.z = b.preact;
  k.ldz = b.ldz;
  k.z_q8 = a->preact_q8;
  k.g = b.g;
  k.ldg = b.ldg;
  k.dx = b.dx;
  k.lddx = b.lddx;
  k.dw = b.dw;
  k.lddw = b.lddw;
  k.db = b.db;
  return k;
}

ff_status plain_sizes(const ff_linear_grad_q8_args* a) {
  if (a == nullptr) return bad("args is NULL");
  if (a->grad.tokens < 0 || a->grad.tokens > (int64_t(1) << 21)) return bad("tokens must be 0 .. 2^21");
  ff_status rc = sizes_ok(a->grad.n, a->grad.m);
  if (rc != FF_OK) return rc;
  if (a->grad.activation < FF_ACT_NONE || a->grad.activation > FF_ACT_SILU) return bad("unknown activation");
  return FF_OK;
}

ff_status grad_sizes(const ff_expert_grad_args* a) {
  if (a == nullptr) return bad("args is NULL");
  ff_status rc = slots_ok(a->routing.tokens, a->routing.experts, a->routing.top);
  if (rc != FF_OK || (rc = sizes_ok(a->n, a->m)) != FF_OK) return rc;
  if (a->by_slot != 0 && a->by_slot != 1) return bad("by_slot must be 0 or 1");
  if (a->activation < FF_ACT_NONE || a->activation > FF_ACT_SILU) return bad("unknown activation");
  if (a->dy_dtype != FF_F32 && a->dy_dtype != FF_BF16) return bad("unknown dtype of dy");
  return FF_OK;
}

}  // namespace

extern "C" {

ff_status ff_route_workspace_size(const ff_route_args* a, size_t* bytes) {
  if (a == nullptr || bytes == nullptr) return bad("args or bytes is NULL");
  ff_status rc = slots_ok(a->tokens, a->experts, a->top);
  if (rc != FF_OK) return rc;
  *bytes = a->tokens == 0 ? 0 : route_workspace(a->tokens, (int)a->experts, (int)a->top);
  return FF_OK;
}
ff_status ff_route(const ff_route_args* a) { return route_call(a, true); }
ff_status ff_expert_order(const ff_route_args* a) { return route_call(a, false); }

ff_status ff_route_backward(const ff_route_grad_args* a) {
  if (a == nullptr) return bad("args is NULL");
  ff_status rc = slots_ok(a->tokens, a->experts, a->top);
  if (rc != FF_OK) return rc;
  if (a->dtype != FF_F32 && a->dtype != FF_BF16) return bad("unknown dtype");
  if (a->score != FF_SCORE_SOFTMAX && a->score != FF_SCORE_SIGMOID) return bad("unknown score");
  if (a->renormalise != 0 && a->renormalise != 1) return bad("renormalise must be 0 or 1");
  if (!std::isfinite((float)a->scale)) return bad("scale must be finite in fp32");
  if (a->tokens == 0) return FF_OK;
  const int64_t T = a->tokens, eb = a->dtype == FF_BF16 ? 2 : 4, len = a->experts * eb;
  if (!rows_ok(a->logits, a->ldl, a->experts, eb) || !rows_ok(a->dlogits, a->ldd, a->experts, eb))
    return bad("logits and dlogits must be aligned device pointers to rows of experts elements, ld >= experts");
  if (a->dweights == nullptr || a->chosen == nullptr || (uintptr_t)a->dweights % 4 != 0 || (uintptr_t)a->chosen % 4 != 0)
    return bad("dweights and chosen must be aligned device pointers");
  const Block in{a->logits, T, a->ldl * eb, len}, out{a->dlogits, T, a->ldd * eb, len};
  if ((meets(out, in) && !(a->logits == a->dlogits && a->ldl == a->ldd)) ||
      clash({out}, {flat(a->dweights, T * a->top * 4), flat(a->chosen, T * a->top * 4)}))
    return bad("dlogits must not overlap the inputs (other than logits as the same rows)");
  RouteGradArgs k{};
  k.tokens = T;
  k.experts = (int)a->experts;
  k.top = (int)a->top;
  k.logits = a->logits;
  k.ldl = a->ldl;
  k.bf16 = a->dtype == FF_BF16;
  k.dweights = a->dweights;
  k.chosen = a->chosen;
  k.sigmoid = a->score == FF_SCORE_SIGMOID;
  k.renormalise = a->renormalise != 0;
  k.scale = a->scale;
  k.dlogits = a->dlogits;
  k.ldd = a->ldd;
  return hip(launch_route_grad(k, (hipStream_t)a->stream), "routing gradient");
}

ff_status ff_expert_linear_workspace_size(const ff_expert_linear_args* a, size_t* bytes) {
  if (bytes == nullptr) return bad("bytes is NULL");
  ff_status rc = forward_sizes(a);
  if (rc != FF_OK) return rc;
  *bytes = a->routing.tokens == 0 ? 0 : forward_ws(a).bytes;
  return FF_OK;
}

ff_status ff_expert_linear(const ff_expert_linear_args* a) {
  ff_status rc = forward_sizes(a);
  if (rc != FF_OK) return rc;
  if (a->activation < FF_ACT_NONE || a->activation > FF_ACT_SILU) return bad("unknown activation");
  if (a->routing.tokens == 0) return FF_OK;
  if ((rc = routing_ok(a->routing, kOrder | kOffsets)) != FF_OK) return rc;
  const int64_t T = a->routing.tokens, S = T * a->routing.top, E = a->routing.experts, X = a->by_slot ? S : T;
  if (!rows_ok(a->x, a->ldx, a->n, 2) || !rows_ok(a->w, a->ldw, a->n, 2))
    return bad("x and w must be aligned device pointers to rows of n elements, ld >= n");
  if (!rows_ok(a->y, a->ldy, a->m, 2) || (a->preact != nullptr && !rows_ok(a->preact, a->ldz, a->m, 2)))
    return bad("y and preact must be aligned device pointers to rows of m elements, ld >= m");
  if ((uintptr_t)a->bias % 2 != 0) return bad("bias is misaligned");
  if (clash({{a->y, S, a->ldy * 2, a->m * 2}, {a->preact, a->preact != nullptr ? S : 0, a->ldz * 2, a->m * 2}},
            {{a->x, X, a->ldx * 2, a->n * 2}, {a->w, E * a->m, a->ldw * 2, a->n * 2}, flat(a->bias, E * a->m * 2),
             block_of(a->routing, kOrder), block_of(a->routing, kOffsets)}))
    return bad(kClash);
  const ForwardWs w = forward_ws(a);
  if ((rc = workspace_ok(a->workspace, a->workspace_bytes, w.bytes)) != FF_OK) return rc;
  char* ws = (char*)a->workspace;
  const hipStream_t s = (hipStream_t)a->stream;
  ExpertArgs k{};
  k.at = slot_rows(a->routing);
  k.gather = !a->by_slot && !w.gather_x;
  k.lin.n = a->n;
  k.lin.m = a->m;
  k.lin.x = a->x;
  k.lin.ldx = a->ldx;
  k.lin.w = a->w;
  k.lin.ldw = a->ldw;
  k.lin.bias = (const bf16_t*)a->bias;
  k.lin.act = a->activation;
  k.lin.y = (bf16_t*)a->y;
  k.lin.ldy = a->ldy;
  k.lin.preact = (bf16_t*)a->preact;
  k.lin.ldz = a->ldz;
  if (w.pack_x) {
    if ((rc = hip(launch_pack_rows(a->x, a->ldx, X, a->n, 2, ws, s), "packing x")) != FF_OK) return rc;
    k.lin.x = ws;
    k.lin.ldx = packed_ld(a->n, 2);
  }
  if (w.gather_x) {
    RowsArgs r{};
    r.at = k.at;
    r.gather = true;
    r.cols = a->n;
    r.src = a->x;
    r.lds = a->ldx;
    r.laid = (uint16_t*)ws;
    if ((rc = hip(launch_rows(&r, 1, s), "rows of x")) != FF_OK) return rc;
    k.lin.x = ws;
    k.lin.ldx = laid_ld(a->n);
  }
  if (w.pack_w) {
    if ((rc = hip(launch_pack_rows(a->w, a->ldw, E * a->m, a->n, 2, ws + w.off_w, s), "packing W")) != FF_OK) return rc;
    k.lin.w = ws + w.off_w;
    k.lin.ldw = packed_ld(a->n, 2);
  }
  if (w.plan.nt == 0) k.lin.n = laid_ld(a->n);  // (zeros up to there in both operands)
  return hip(launch_expert_linear(k, w.plan, s), "experts' product");
}

ff_status ff_expert_combine(const ff_expert_combine_args* a) {
  if (a == nullptr) return bad("args is NULL");
  ff_status rc = slots_ok(a->routing.tokens, a->routing.experts, a->routing.top);
  if (rc != FF_OK) return rc;
  if (a->cols < 1 || a->cols > kMaxDim) return bad("cols must be 1 .. 2^20");
  if (a->routing.tokens == 0) return FF_OK;
  if ((rc = routing_ok(a->routing, kOffsets | kPlace)) != FF_OK) return rc;
  if ((uintptr_t)a->routing.weights % 4 != 0) return bad("weights is misaligned");
  const int64_t T = a->routing.tokens, S = T * a->routing.top, len = a->cols * 2;
  if (!rows_ok(a->y, a->ldy, a->cols, 2) || !rows_ok(a->out, a->ldo, a->cols, 2) ||
      (a->residual != nullptr && !rows_ok(a->residual, a->ldr, a->cols, 2)))
    return bad("y, residual and out must be aligned device pointers to rows of cols elements, ld >= cols");
  const Block out{a->out, T, a->ldo * 2, len}, res{a->residual, a->residual != nullptr ? T : 0, a->ldr * 2, len};
  if (clash({out}, {{a->y, S, a->ldy * 2, len}, block_of(a->routing, kPlace), block_of(a->routing, kOffsets), block_of(a->routing, kWeights)}) ||
      (meets(out, res) && !(a->out == a->residual && a->ldo == a->ldr)))
    return bad("out must not overlap the inputs (it may be the residual itself)");
  CombineArgs k{};
  k.at = slot_rows(a->routing);
  k.cols = a->cols;
  k.y = a->y;
  k.ldy = a->ldy;
  k.residual = (const bf16_t*)a->residual;
  k.ldr = a->ldr;
  k.out = (bf16_t*)a->out;
  k.ldo = a->ldo;
  return hip(launch_combine(k, (hipStream_t)a->stream), "combining rows");
}

ff_status ff_expert_combine_backward(const ff_expert_combine_grad_args* a) {
  if (a == nullptr) return bad("args is NULL");
  ff_status rc = slots_ok(a->routing.tokens, a->routing.experts, a->routing.top);
  if (rc != FF_OK) return rc;
  if (a->cols < 1 || a->cols > kMaxDim) return bad("cols must be 1 .. 2^20");
  if (a->routing.tokens == 0 || (a->dy == nullptr && a->dweights == nullptr)) return FF_OK;
  if ((rc = routing_ok(a->routing, kOrder | kOffsets | kPlace | kWeights)) != FF_OK) return rc;
  const int64_t T = a->routing.tokens, S = T * a->routing.top, len = a->cols * 2;
  if (!rows_ok(a->dout, a->ldd, a->cols, 2) || (a->dweights != nullptr && !rows_ok(a->y, a->ldy, a->cols, 2)) ||
      (a->dy != nullptr && !rows_ok(a->dy, a->lddy, a->cols, 4)) || (uintptr_t)a->dweights % 4 != 0)
    return bad("dout, y (for dweights), dy and dweights must be aligned device pointers, rows of cols elements, ld >= cols");
  if (clash({{a->dy, a->dy != nullptr ? S : 0, a->lddy * 4, a->cols * 4}, flat(a->dweights, S * 4)},
            {{a->dout, T, a->ldd * 2, len}, {a->y, a->dweights != nullptr ? S : 0, a->ldy * 2, len}, block_of(a->routing, kOrder),
             block_of(a->routing, kOffsets), block_of(a->routing, kPlace), block_of(a->routing, kWeights)}))
    return bad(kClash);
  CombineGradArgs k{};
  k.at = slot_rows(a->routing);
  k.cols = a->cols;
  k.dout = (const bf16_t*)a->dout;
  k.ldd = a->ldd;
  k.y = (const bf16_t*)a->y;
  k.ldy = a->ldy;
  k.dy = a->dy;
  k.lddy = a->lddy;
  k.dweights = a->dweights;
  return hip(launch_combine_grad(k, (hipStream_t)a->stream), "combining gradient");
}

ff_status ff_expert_linear_backward_workspace_size(const ff_expert_grad_args* a, size_t* bytes) {
  if (bytes == nullptr) return bad("bytes is NULL");
  ff_status rc = grad_sizes(a);
  if (rc != FF_OK) return rc;
  *bytes = a->routing.tokens == 0 ? 0 : grad_ws(gradient_of(a)).bytes;
  return FF_OK;
}

ff_status ff_expert_linear_backward(const ff_expert_grad_args* a) {
  ff_status rc = grad_sizes(a);
  if (rc != FF_OK) return rc;
  const hipStream_t s = (hipStream_t)a->stream;
  const Gradient k = gradient_of(a);
  if ((uintptr_t)k.db % 2 != 0) return bad("db is misaligned");
  if (k.dw != nullptr && !rows_ok(k.dw, k.lddw, k.n, 2)) return bad("dw must be an aligned device pointer to rows of n elements, ld >= n");
  if (k.at.tokens == 0) return zero_gradient(k, s);
  if ((rc = routing_ok(a->routing, kOrder | kOffsets | (k.gather ? kPlace : 0))) != FF_OK) return rc;
  rc = gradient_ok(k, k.at.rows, k.gather ? k.at.tokens : k.at.rows,
                   {block_of(a->routing, kOrder), block_of(a->routing, kOffsets), block_of(a->routing, kPlace)});
  if (rc != FF_OK) return rc;
  const GradWs w = grad_ws(k);
  if ((rc = workspace_ok(a->workspace, a->workspace_bytes, w.bytes)) != FF_OK) return rc;
  return run_gradient(k, w, (char*)a->workspace, s);
}

ff_status ff_linear_backward_q8_workspace_size(const ff_linear_grad_q8_args* a, size_t* bytes) {
  if (bytes == nullptr) return bad("bytes is NULL");
  ff_status rc = plain_sizes(a);
  if (rc != FF_OK) return rc;
  *bytes = a->grad.tokens == 0 ? 0 : grad_ws(gradient_of(a)).bytes;
  return FF_OK;
}

ff_status ff_linear_backward_q8(const ff_linear_grad_q8_args* a) {
  ff_status rc = plain_sizes(a);
  if (rc != FF_OK) return rc;
  const hipStream_t s = (hipStream_t)a->grad.stream;
  Gradient k = gradient_of(a);
  if ((uintptr_t)k.db % 2 != 0) return bad("db is misaligned");
  if (k.dw != nullptr && !rows_ok(k.dw, k.lddw, k.n, 2)) return bad("dw must be an aligned device pointer to rows of n elements, ld >= n");
  if (k.at.tokens == 0) return zero_gradient(k, s);
  if ((rc = gradient_ok(k, k.at.rows, k.at.rows, {})) != FF_OK) return rc;
  const GradWs w = grad_ws(k);
  if ((rc = workspace_ok(a->grad.workspace, a->grad.workspace_bytes, w.bytes)) != FF_OK) return rc;
  return run_gradient(k, w, (char*)a->grad.workspace, s);
}

}  // extern "C"
