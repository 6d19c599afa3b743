// The 8-bit KV cache's number format: e4m3 codes (1 sign, 4 exponent, 3 mantissa bits, largest value 448,
// no infinities) and one power-of-two scale per block of 16 tokens of K, or of V, of one kv head.
//
// A power of two costs nothing over a scale of any size - e4m3 is a floating-point format, so its relative
// rounding error is the same wherever in its range the values lie - and keeps everything after the rounding
// exact: code x scale is a number of the pool's 16-bit type (what the matrix instructions take), and a code
// moves to a larger scale by its exponent alone, unless it falls below e4m3's smallest normal number.
//
// The exponents end where code x scale would leave the 16-bit type: below, at 2^-15 x 2^-9 (e4m3's smallest
// step) = fp16's smallest number; bf16 stays far inside its normal numbers.  Above, values that round past
// the type's largest one (240 x 2^8 = 61440 of fp16, 240 x 2^120 of bf16) stay at that.
#pragma once
#include "mc_common.h"

namespace mc {

constexpr int kBlockBytes = kPage * kHeadDim;   // codes of one (page, K|V, head) block: 2 KiB

struct ScaleLimits {
  int lo, hi;
};
__host__ __device__ constexpr ScaleLimits scale_limits(int dtype) {
  return dtype == MC_F16 ? ScaleLimits{-15, 8} : ScaleLimits{-100, 120};
}

// Exponent k of a block's scale from the bits of its largest finite magnitude (as fp32): the least one
// with magnitude <= 448 x 2^k.  448 = 1.75 x 2^8.
__device__ __forceinline__ int scale_exponent(uint32_t bits, ScaleLimits lim) {
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, lim.lo), lim.hi);
}
__device__ __forceinline__ float power_of_two(int k) {
  return __builtin_bit_cast(float, (uint32_t)(k + 127) << 23);
}
// The exponent of a scale in memory; whatever stands there, one that power_of_two takes.
__device__ __forceinline__ int exponent_of(float scale, ScaleLimits lim) {
  return min(max((int)(__builtin_bit_cast(uint32_t, scale) >> 23 & 0xff) - 127, lim.lo), lim.hi);
}
// |x| as bits, 0 for what is not finite
__device__ __forceinline__ uint32_t magnitude(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}
// What is rounded to a code: x / 2^k within the largest code; NaN for what is not finite.
__device__ __forceinline__ float before_code(float x, float inv_scale, float most) {
  const float y = __builtin_amdgcn_fmed3f(x * inv_scale, -most, most);
  return magnitude(x) == 0u && x != 0.f ? __builtin_nanf("") : y;
}
// two codes (round to nearest even) in the low or high half of a word
template <bool kHigh>
__device__ __forceinline__ uint32_t two_codes(float a, float b, uint32_t word) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)word, kHigh);
}
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d) {
  return two_codes<true>(c, d, two_codes<false>(a, b, 0u));
}
// the codes of a word at a scale 1 / by times as large
__device__ __forceinline__ uint32_t move_codes(uint32_t w, float by) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return four_codes(lo[0] * by, lo[1] * by, hi[0] * by, hi[1] * by);
}

inline mc_status check_pool8(const mc_pool8_desc* pool) {
  if (!pool || !pool->codes || !pool->scales) return MC_ERR_INVALID;
  if (!aligned16(pool->codes) || (reinterpret_cast<uintptr_t>(pool->scales) & 7u)) return MC_ERR_INVALID;
  if (reinterpret_cast<uintptr_t>(pool->skipped) & 3u) return MC_ERR_INVALID;
  if (pool->num_layers <= 0 || pool->num_pages <= 0 || pool->num_kv_heads <= 0) return MC_ERR_INVALID;
  if (pool->page_size != kPage || pool->head_dim != kHeadDim) return MC_ERR_UNSUPPORTED;
  if (pool->dtype != MC_F16 && pool->dtype != MC_BF16) return MC_ERR_UNSUPPORTED;
  return MC_OK;
}

// bytes of codes between pages of a layer, and between layers; scales between the same
inline int64_t page8_stride(const mc_pool8_desc* p) { return 2ll * p->num_kv_heads * kBlockBytes; }
inline int64_t layer8_stride(const mc_pool8_desc* p) { return page8_stride(p) * p->num_pages; }
inline int64_t layer8_scales(const mc_pool8_desc* p) { return 2ll * p->num_kv_heads * p->num_pages; }

}  // namespace mc
