// What the kernels of ppd_paged_attention_fp4 share, beside what they have from ppd_paged_attention's.
//
// Codes become bf16 numbers in registers, without rounding, and from there on both products are those of bf16 keys and values.  What is not bf16
// goes in as a sum of bf16 terms: queries of fp16 in two (11 bits of significand in 8 + 8) and of fp32 in three (24 in 8 + 8 + 8), exactly (fp32 ones
// times scale * log2(e), rounded to fp32);
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

// As find_whole, but the tiles are counted, J sequences a lane at a time: an item for each of them and none without one.  (Between workgroups of find_whole's there are
// some without work, and where these come at every second place (16 rows a sequence, or 128) half of the compute units are left idle: bf16, 32 / 8 heads, 64
// sequences of 32 tokens over 1500 positions 86 us, not 148, 256 of them 348, not 521; 1000 of 4 tokens over 700 252, not 373.)
template <int TILE, int J>
__device__ __forceinline__ bool find_tile(const PagedAttnArgs& a, int idx, int lane, Item& it) {
  int before = 0;
  for (int s = 0; s < a.b.n_seqs; s += WAVE * J) {
    int tiles[J], mine = 0;
    SeqRows r1;                                             // (J 1: the lane's sequence)
#pragma unroll
    for (int j = 0; j < J; ++j) {
      SeqPlan p;
      seq_plan<TILE>(a, s + lane * J + j, p);
      tiles[j] = p.tiles; mine += p.tiles;
      if (J == 1) r1 = p.r;
    }
    const int upto = before + scan_up(mine);
    const unsigned long long past = __ballot(upto > idx);
    if (past) {
      const int w = __builtin_ctzll(past);
      int r = idx - (upto - mine), j0 = 0, many = 0;        // (of lane w's sequences, the one that has the item)
      bool there = false;
#pragma unroll
      for (int j = 0; j < J; ++j) {
        if (there) continue;
        if (r < tiles[j]) { there = true; j0 = j; many = tiles[j]; } else r -= tiles[j];
      }
      r = __builtin_amdgcn_readlane(r, w);
      it.s = s + w * J + __builtin_amdgcn_readlane(j0, w);
      SeqRows q;
      if (J == 1) q = {__builtin_amdgcn_readlane(r1.row0, w), __builtin_amdgcn_readlane(r1.rows, w), __builtin_amdgcn_readlane(r1.pos0, w)};
      else q = seq_rows(a.b, it.s);
      it.rows0 = q.row0; it.n = q.rows; it.pos0 = q.pos0;
      it.tile = TILE == TILE_ROWS ? __builtin_amdgcn_readlane(many, w) - 1 - r : r;
      it.part = 0; it.parts = 1; it.slot = idx; it.wide = false;
      const Span span = span_of(it.pos0, it.n, it.tile, TILE, a.group, 0, 1, a.b.room, a.window);
      it.lo = span.lo; it.hi = span.hi;
      return true;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}
template <int TILE>
__device__ __forceinline__ bool find_item_fp4(const PagedAttnArgs& a, int idx, int wide_idx, bool tell, int lane, Item& it) {
  // (over 256 sequences of half a tile or less, gaps are few, and counting takes longer: 1000 of one token over 700 positions 207 us, not 226)
  if (a.least > 0 || (a.b.n_seqs > 4 * WAVE && 2 * (int64_t)a.b.n_tokens * a.group <= (int64_t)TILE * a.b.n_seqs)) return find_item<TILE, TILE != TILE_ROWS>(a, idx, wide_idx, tell, lane, it);
  return a.b.n_seqs <= WAVE ? find_tile<TILE, 1>(a, idx, lane, it) : find_tile<TILE, 4>(a, idx, lane, it);
}

inline bool near_pages_fp4(const Fp4AttnArgs& a) { return near_pages(a) && a.ks_pos < 1 << 25 && a.vs_pos < 1 << 25; }
hipError_t launch_paged_tiles_fp4(const Fp4AttnArgs& a, int dtype, int head_dim, hipStream_t stream);

}  // namespace ppd
