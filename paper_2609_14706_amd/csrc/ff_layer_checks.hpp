// What the C entry points of the layer operators check alike.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>

#include "ff.h"
#include "ff_error.hpp"
#include "ff_layer_kernels.hpp"

namespace ff {
namespace {

constexpr int64_t kMaxCols = int64_t(1) << 24, kMaxDim = int64_t(1) << 20, kMaxRows = int64_t(1) << 40;

[[maybe_unused]] size_t up256(size_t v) { return (v + 255) / 256 * 256; }

[[maybe_unused]] ff_status bad(const char* msg) { return report(FF_ERR_INVALID_ARG, msg); }

[[maybe_unused]] ff_status hip(hipError_t e, const char* where) {
  if (e == hipSuccess) return FF_OK;
  char msg[160];
  snprintf(msg, sizeof msg, "%s: %s", where, hipGetErrorString(e));
  return report(FF_ERR_HIP, msg);
}

[[maybe_unused]] ff_status workspace_ok(const void* p, size_t have, size_t need) {
  if (need == 0) return FF_OK;
  if (p != nullptr && (uintptr_t)p % 256 == 0 && have >= need) return FF_OK;
  char msg[160];
  snprintf(msg, sizeof msg, "workspace must be a 256-byte aligned device pointer to >= %zu bytes (got %zu)", need, have);
  return report(FF_ERR_WORKSPACE, msg);
}

// Rows of `len` elements of `bytes` each: `ld` apart, from a pointer aligned to one.
[[maybe_unused]] bool rows_ok(const void* p, int64_t ld, int64_t len, size_t bytes) {
  return p != nullptr && (uintptr_t)p % bytes == 0 && ld >= len && ld <= kMaxRows;
}

// Whether the bytes of two sets of rows (of `la`, `lb` bytes, `sa`, `sb` bytes
// apart) can meet: their whole ranges do, and they are not column blocks of
// one set of wider rows.
[[maybe_unused]] bool meet(const void* a, int64_t rows_a, int64_t sa, int64_t la, const void* b, int64_t rows_b, int64_t sb, int64_t lb) {
  if (a == nullptr || b == nullptr || rows_a <= 0 || rows_b <= 0) return false;
  const char *pa = (const char*)a, *pb = (const char*)b;
  if (pa >= pb + (rows_b - 1) * sb + lb || pb >= pa + (rows_a - 1) * sa + la) return false;
  if (sa != sb || sa <= 0) return true;
  const int64_t d = ((pb - pa) % sa + sa) % sa;  // where b's rows start in a's
  return d < la || d + lb > sa;
}

// A checkpoint of rows x cols: codes and scales in place, groups of a size that is taken.
[[maybe_unused]] bool q8_ok(const ff_q8_rows& c, int64_t cols) {
  if (c.group < (1 << kMinGroupShift) || c.group > (1 << kMaxGroupShift) || (c.group & (c.group - 1)) != 0) return false;
  return rows_ok(c.q, c.ldq, cols, 1) && rows_ok(c.scale, c.ld_scale, (cols + c.group - 1) / c.group, 4);
}
[[maybe_unused]] Q8Rows q8_of(const ff_q8_rows& c) {
  return c.q != nullptr ? Q8Rows{c.q, c.ldq, c.scale, c.ld_scale, __builtin_ctzll((unsigned long long)c.group)} : Q8Rows{};
}
constexpr const char* kBadQ8 =
    "a checkpoint needs codes and scales with ld >= their rows' lengths and a group of 16, 32, 64, 128, 256 or 512 columns";

}  // namespace
}  // namespace ff
