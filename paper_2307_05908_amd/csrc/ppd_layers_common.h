// What the operators on paged caches share: element types, the rows of a ragged batch, argument checks.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ppd_layers.h"
#include "ppd_kernels.h"
#include "ppd_launch.h"

namespace ppd {

struct f16_t { uint16_t v; };
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// four elements in a row <-> fp32, one rounding (to nearest even)
template <typename T> struct Quad;
template <> struct Quad<float> {
  typedef u32x4 raw;
  __device__ static __forceinline__ f32x4 wide(raw r) { return __builtin_bit_cast(f32x4, r); }
  __device__ static __forceinline__ raw narrow(f32x4 v) { return __builtin_bit_cast(raw, v); }
};
template <> struct Quad<bf16_t> {
  typedef u32x2 raw;
  __device__ static __forceinline__ f32x4 wide(raw r) {
    return (f32x4){__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u), __uint_as_float(r.y << 16), __uint_as_float(r.y & 0xffff0000u)};
  }
  __device__ static __forceinline__ raw narrow(f32x4 v) {
    return (raw){(uint32_t)f32_to_bf16(v.x) | (uint32_t)f32_to_bf16(v.y) << 16, (uint32_t)f32_to_bf16(v.z) | (uint32_t)f32_to_bf16(v.w) << 16};
  }
};
template <> struct Quad<f16_t> {
  typedef u32x2 raw;
  typedef _Float16 h4 __attribute__((ext_vector_type(4)));
  __device__ static __forceinline__ f32x4 wide(raw r) {
    const h4 h = __builtin_bit_cast(h4, r);
    return (f32x4){(float)h.x, (float)h.y, (float)h.z, (float)h.w};
  }
  __device__ static __forceinline__ raw narrow(f32x4 v) {
    const h4 h = {(_Float16)v.x, (_Float16)v.y, (_Float16)v.z, (_Float16)v.w};
    return __builtin_bit_cast(raw, h);
  }
};

// A batch as the kernels take it.
struct Batch {
  const int32_t* q_start; const int32_t* kv_len; const int32_t* pages;
  int64_t pages_stride;
  int max_pages, n_seqs, n_tokens, n_pages, page_size;
  int room;              // positions that a row of the table has places for (at most 2^30, so that no loop over them passes 31 bits)
};
// One sequence of it: rows [row0, row0 + rows) of the tensors, the first of them at position pos0 (negative where kv_len is below rows).
struct SeqRows { int row0, rows, pos0; };

__device__ __forceinline__ SeqRows seq_rows(const Batch& b, int s) {
  const int lo = min(max(b.q_start[s], 0), b.n_tokens), hi = min(max(b.q_start[s + 1], lo), b.n_tokens);
  return {lo, hi - lo, max(b.kv_len[s], 0) - (hi - lo)};
}
// The sequence of a row, or -1, by a whole wave: the last one that begins at or before it.  One round of loads for 64 sequences, two for
// more (a binary search is a chain of as many as it has steps).
__device__ __forceinline__ int seq_of_row(const Batch& b, int row, int lane) {
  static_assert(PPD_MAX_SEQS <= WAVE * WAVE, "two rounds of loads");
  const int end = b.q_start[b.n_seqs];
  int from = 0;
  if (b.n_seqs > WAVE) {
    const int s = lane * WAVE;
    from = max(__popcll(__ballot(s < b.n_seqs && b.q_start[min(s, b.n_seqs)] <= row)) - 1, 0) * WAVE;
  }
  const int s = from + lane, n = __popcll(__ballot(s < b.n_seqs && b.q_start[min(s, b.n_seqs)] <= row));
  return n >= 1 && row < end ? from + n - 1 : -1;
}
// The page that holds a position of sequence s, or -1.
__device__ __forceinline__ int page_of(const Batch& b, int s, int pos) {
  if (pos < 0) return -1;
  const int i = (int)((unsigned)pos / (unsigned)b.page_size);
  if (i >= b.max_pages) return -1;
  const int page = b.pages[(int64_t)s * b.pages_stride + i];
  return (unsigned)page < (unsigned)b.n_pages ? page : -1;
}

inline Batch batch_of(const ppd_paged_cache& c, const ppd_paged_batch& b) {
  const int64_t room = (int64_t)b.max_pages * c.page_size;
  return {b.q_start, b.kv_len, b.pages, b.pages_stride, b.max_pages, b.n_seqs, b.n_tokens, c.n_pages, c.page_size, (int)room};
}
inline int elem_size(int dtype) { return dtype == PPD_FP32 ? 4 : 2; }

// strides (in elements) of `count` rows that begin at multiples of 16 bytes each
inline bool good_stride(int64_t stride, int count, int dtype) { return count <= 1 || (stride >= 0 && stride % (16 / elem_size(dtype)) == 0); }

// PPD_OK, or what is wrong with a cache and a batch
inline int check_paged(const ppd_paged_cache* c, const ppd_paged_batch* b) {
  if (!c || !b) return PPD_EINVAL;
  if (c->dtype < PPD_FP32 || c->dtype > PPD_FP16 || (c->head_dim != 64 && c->head_dim != 128)) return PPD_EINVAL;
  if (c->n_pages < 1 || c->page_size < 1 || c->n_kv_heads < 1 || !c->k || !c->v || (((uintptr_t)c->k | (uintptr_t)c->v) & 15)) return PPD_EINVAL;
  if (!good_stride(c->k_page, c->n_pages, c->dtype) || !good_stride(c->v_page, c->n_pages, c->dtype) || !good_stride(c->k_pos, c->page_size, c->dtype) ||
      !good_stride(c->v_pos, c->page_size, c->dtype) || !good_stride(c->k_head, c->n_kv_heads, c->dtype) || !good_stride(c->v_head, c->n_kv_heads, c->dtype))
    return PPD_EINVAL;
  if (b->n_seqs < 1 || b->n_tokens < 0 || b->max_pages < 1 || !b->q_start || !b->kv_len || !b->pages) return PPD_EINVAL;
  if (((uintptr_t)b->q_start | (uintptr_t)b->kv_len | (uintptr_t)b->pages) & 3) return PPD_EINVAL;
  if (b->n_seqs > 1 && b->pages_stride < b->max_pages) return PPD_EINVAL;
  if (b->n_seqs > PPD_MAX_SEQS || b->n_tokens > PPD_MAX_TOKENS || c->n_kv_heads > PPD_MAX_HEADS) return PPD_ELIMIT;
  if ((int64_t)b->max_pages * c->page_size > 1 << 30) return PPD_ELIMIT;
  return PPD_OK;
}
// rows of a batch; written ones must not lie on each other
inline bool good_rows(const ppd_rows* r, int tokens, int heads, int dtype, bool written) {
  if (!r || !r->p || ((uintptr_t)r->p & 15) || !good_stride(r->token, tokens, dtype) || !good_stride(r->head, heads, dtype)) return false;
  return !written || ((tokens <= 1 || r->token > 0) && (heads <= 1 || r->head > 0));
}
inline int launched(hipError_t e) {
  if (e == hipSuccess) return PPD_OK;
  set_global_hip_error((int)e);
  (void)hipGetLastError();
  return PPD_EHIP;
}

}  // namespace ppd
