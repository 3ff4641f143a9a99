// Pages of 4-bit numbers (the MX format): 32 numbers with a scale of eight bits.  Codes to bf16 (exactly) and fp32 to codes (to nearest, ties to
// even) are instructions of gfx950; both were compared with the definition over all codes and scales and around every border.
#pragma once
#include "ppd_layers_common.h"

namespace ppd {

constexpr int FP4_BLOCK = 32;                      // numbers of a scale
constexpr int FP4_LEAST = -125, FP4_MOST = 125;    // exponents of the scales that are written
constexpr uint32_t FP4_NAN = 253;                  // from this scale on the numbers are NaN

__device__ __forceinline__ float fp4_scale(uint32_t byte) { return __uint_as_float(byte >= FP4_NAN ? 0x7f800000u : byte << 23); }      // (an infinite scale makes every code NaN)
// eight codes as bf16 numbers
__device__ __forceinline__ u32x4 fp4_wide(uint32_t codes, float scale) {
  return (u32x4){__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
}
// eight numbers as codes of a scale
__device__ __forceinline__ uint32_t fp4_narrow(const float (&x)[8], float scale) {
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], scale, 3);
}
// The scale of numbers whose largest magnitude has these bits: the least 2^e with 7 * 2^e at or above it (a significand up to 1.75 is 7 / 4).
__device__ __forceinline__ uint32_t fp4_scale_of(uint32_t most) {
  if (most >= 0x7f800000u) return 255;
  const int e = (int)((most + 0x1fffffu) >> 23) - 127 - 2;
  return 127 + min(max(e, FP4_LEAST), FP4_MOST);
}

// rows of bytes that begin at multiples of `unit`
inline bool good_bytes(int64_t stride, int count, int unit) { return count <= 1 || (stride >= 0 && stride % unit == 0); }
inline int check_paged_fp4(const ppd_paged_cache_fp4* c, const ppd_paged_batch* b) {
  if (!c || !b) return PPD_EINVAL;
  if (c->dtype < PPD_FP32 || c->dtype > PPD_FP16 || (c->head_dim != 64 && c->head_dim != 128)) return PPD_EINVAL;
  const int unit = c->head_dim / FP4_BLOCK;
  if (c->n_pages < 1 || c->page_size < 1 || c->n_kv_heads < 1 || !c->k || !c->v || !c->k_scales || !c->v_scales) return PPD_EINVAL;
  if (((uintptr_t)c->k | (uintptr_t)c->v) & 15 || ((uintptr_t)c->k_scales | (uintptr_t)c->v_scales) & (unit - 1)) return PPD_EINVAL;
  if (!good_bytes(c->k_page, c->n_pages, 16) || !good_bytes(c->v_page, c->n_pages, 16) || !good_bytes(c->k_pos, c->page_size, 16) ||
      !good_bytes(c->v_pos, c->page_size, 16) || !good_bytes(c->k_head, c->n_kv_heads, 16) || !good_bytes(c->v_head, c->n_kv_heads, 16))
    return PPD_EINVAL;
  if (!good_bytes(c->ks_page, c->n_pages, unit) || !good_bytes(c->vs_page, c->n_pages, unit) || !good_bytes(c->ks_pos, c->page_size, unit) ||
      !good_bytes(c->vs_pos, c->page_size, unit) || !good_bytes(c->ks_head, c->n_kv_heads, unit) || !good_bytes(c->vs_head, c->n_kv_heads, unit))
    return PPD_EINVAL;
  return check_batch(b, c->n_kv_heads, c->page_size);
}

}  // namespace ppd
