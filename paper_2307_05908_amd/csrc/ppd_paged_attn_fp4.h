// What the kernels of ppd_paged_attention_fp4 share, beside what they have from ppd_paged_attention's.
//
// Codes become bf16 numbers in registers, without rounding, and from there on both products are those of bf16 keys and values.  What is not bf16
// goes in as a sum of bf16 terms: queries of fp16 in two (11 bits of significand in 8 + 8) and of fp32 in three (24 in 8 + 8 + 8), exactly;
// softmax weights in two for 16-bit results (2^-17 of each is lost, and the result's own rounding is 2^-9 or 2^-12), in three for fp32.
#pragma once
#include "ppd_paged_attn.h"
#include "ppd_paged_fp4.h"

namespace ppd {

// kc, vc and their strides: codes, in bytes
struct Fp4AttnArgs : PagedAttnArgs {
  const void *ks, *vs;
  int64_t ks_page, ks_pos, ks_head, vs_page, vs_pos, vs_head;
  int side, wide_side; // workgroups of a part that follow each other on one XCD, and of four heads each
};

template <typename T> struct Terms;
template <> struct Terms<bf16_t> { static constexpr int Q = 1, W = 2; };
template <> struct Terms<f16_t> { static constexpr int Q = 2, W = 2; };
template <> struct Terms<float> { static constexpr int Q = 3, W = 3; };

// eight numbers of a query as bf16 terms, each cut off, not rounded (so that the largest numbers stay finite): eight bits of the significand a term
__device__ __forceinline__ void query_terms(const bf16_t* p, float, u32x4 (&t)[1]) { t[0] = *(const u32x4*)p; }
template <typename T, int N>
__device__ __forceinline__ void query_terms(const T* p, float factor, u32x4 (&t)[N]) {
  const typename Quad<T>::raw* const r = (const typename Quad<T>::raw*)p;
  f32x4 x[2] = {Quad<T>::wide(r[0]), Quad<T>::wide(r[1])};
  if (sizeof(T) == 4) { x[0] *= factor; x[1] *= factor; }
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const uint32_t a = __float_as_uint(x[h][e]), b = __float_as_uint(x[h][e + 1]);
        t[n][2 * h + e / 2] = __builtin_amdgcn_perm(b, a, 0x07060302u);
        x[h][e] -= __uint_as_float(a & 0xffff0000u);
        x[h][e + 1] -= __uint_as_float(b & 0xffff0000u);
      }
}

inline bool near_pages_fp4(const Fp4AttnArgs& a) { return near_pages(a) && a.ks_pos < 1 << 25 && a.vs_pos < 1 << 25; }
hipError_t launch_paged_tiles_fp4(const Fp4AttnArgs& a, int dtype, int head_dim, hipStream_t stream);

}  // namespace ppd
