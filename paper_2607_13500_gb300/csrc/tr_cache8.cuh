// The paged cache held in 8 bits as its kernels see it: e4m3 codes, and for
// each 16 keys of a head (a block) one exponent e of their scale 2^(e - 127).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tr_cache.cuh"

namespace tr {
namespace cache8 {

constexpr int kBlock = 16;                 // keys that share a scale
constexpr int kMinExp = -117, kMaxExp = 119;  // that append gives a scale: a block's values are then normal numbers of 32 bits

struct Scales {
  uint8_t *k, *v;  // [pages, heads, page / kBlock]
};

// The exponent of a scale as it is held, -127 to 127 (255, no scale, as 254).
__device__ __forceinline__ int exp_of(uint8_t e) { return min((int)e, 254) - 127; }
__device__ __forceinline__ float pow2(int e) { return __int_as_float(e > -127 ? (e + 127) << 23 : 1 << 22); }  // -127 <= e <= 127

// Index of the scale that page `page`, head h, slot s in the page go by.
__device__ __forceinline__ long long scale_at(const CacheView &c, int page, int h, int s) {
  return ((long long)page * c.heads + h) * (c.page / kBlock) + s / kBlock;
}

// Four codes (the low byte first) as two pairs of halves, exactly; NaN stays NaN.
__device__ __forceinline__ void halves4(uint32_t codes, uint32_t &lo, uint32_t &hi) {
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}"
      : "=r"(lo), "=r"(hi)
      : "r"(codes));
}
// Two values to their nearest codes, the low byte first.
__device__ __forceinline__ uint16_t codes_of(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint16_t codes_of_halves(uint32_t h) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(h));
  return r;
}

inline tr_status check_cache8(const tr_cache8 *c) {
  if (!c) return TR_ERR_ARG;
  const tr_status rc = check_cache(&c->c);
  if (rc != TR_OK) return rc;
  return c->k_scale && c->v_scale ? TR_OK : TR_ERR_ARG;
}

}  // namespace cache8
}  // namespace tr
