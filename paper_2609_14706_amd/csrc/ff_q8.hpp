// Reading 8-bit activation checkpoints: codes with a scale for each group of
// 16 to 512 columns.
#pragma once

#include "ff_layer_kernels.hpp"
#include "ff_vec.hpp"

namespace ff {

// Eight codes from column `col` on (a multiple of eight: one group's), `count` of
// them in the row, zeros after them.
__device__ __forceinline__ void load_codes(const int8_t* p, int count, uint32_t (&w)[2]) {
  if (count >= 8) {
    __builtin_memcpy(w, p, 8);
  } else {
    w[0] = w[1] = 0;
#pragma unroll
    for (int k = 0; k < 7; ++k)
      if (k < count) w[k / 4] |= (uint32_t)(uint8_t)p[k] << (8 * (k % 4));
  }
}
// Their values, not rounded: a code is exact in fp32, its product rounded once.  One scale that
// k_checkpoint gives has no room for 127 of it in fp32, that of a group whose largest number is fp32's largest:
// the number below it is taken instead.
constexpr float kTopScale = 0x1.fffffep127f / 127.0f;
static_assert(kTopScale == 0x1.020408p121f, "one step up from the largest that 127 times stays finite");
__device__ __forceinline__ void values_of(const uint32_t (&w)[2], float scale, float (&f)[8]) {
  if (scale == kTopScale) scale = 0x1.020406p121f;
#pragma unroll
  for (int k = 0; k < 8; ++k) f[k] = (float)(int8_t)(w[k / 4] >> (8 * (k % 4))) * scale;
}

}  // namespace ff
