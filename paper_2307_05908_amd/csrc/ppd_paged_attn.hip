// ppd_paged_attention: attention of ragged runs of new tokens over paged keys and values.
#include "ppd_layers_common.h"

#include <math.h>

using namespace ppd;

namespace {

struct PagedAttnArgs {
  Batch b;
  const void* q; void* out; float* lse; const void *kc, *vc;
  int64_t q_tok, q_head, o_tok, o_head;
  int64_t kc_page, kc_pos, kc_head, vc_page, vc_pos, vc_head;
  int heads, kv_heads, window;
  float scale;
};

template <typename T> __device__ __forceinline__ float elem(const void* p, int64_t i);
template <> __device__ __forceinline__ float elem<float>(const void* p, int64_t i) { return ((const float*)p)[i]; }
template <> __device__ __forceinline__ float elem<bf16_t>(const void* p, int64_t i) { return bf16_to_f32(((const uint16_t*)p)[i]); }
template <> __device__ __forceinline__ float elem<f16_t>(const void* p, int64_t i) { return (float)((const _Float16*)p)[i]; }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16_t* p, float v) { p->v = f32_to_bf16(v); }
__device__ __forceinline__ void put(f16_t* p, float v) { *(_Float16*)p = (_Float16)v; }

// One workgroup for a row and a query head; a wave takes every fourth position, a running maximum and sum, then the four are joined.
template <typename T, int HD>
__global__ __launch_bounds__(256) void paged_attn_kernel(PagedAttnArgs a) {
  constexpr int E = HD / WAVE;
  __shared__ float sm[4], sl[4], so[4][HD];
  const int row = blockIdx.x, h = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int s = seq_of_row(a.b, row, lane);
  if (s < 0) return;
  const SeqRows sr = seq_rows(a.b, s);
  const int pos = sr.pos0 + (row - sr.row0), first = a.window > 0 ? max(pos - a.window + 1, 0) : 0, kvh = h / (a.heads / a.kv_heads);
  float q[E], o[E], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) { q[e] = elem<T>(a.q, row * a.q_tok + h * a.q_head + lane * E + e); o[e] = 0.f; }
  const int end = min(pos, a.b.room - 1);      // (the table ends there, whatever the length says)
  for (int p = first + wave; p <= end; p += 4) {
    const int page = page_of(a.b, s, p);
    if (page < 0) continue;
    const int slot = (int)((unsigned)p % (unsigned)a.b.page_size);
    float t = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) t = fmaf(q[e], elem<T>(a.kc, page * a.kc_page + slot * a.kc_pos + kvh * a.kc_head + lane * E + e), t);
    t = wave_sum(t) * a.scale;
    const float mn = fmaxf(m, t), safe = mn == -INFINITY ? 0.f : mn, keep = expf(m - safe), w = expf(t - safe);
    l = l * keep + w; m = mn;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(w, elem<T>(a.vc, page * a.vc_page + slot * a.vc_pos + kvh * a.vc_head + lane * E + e), o[e] * keep);
  }
  if (lane == 0) { sm[wave] = m; sl[wave] = l; }
#pragma unroll
  for (int e = 0; e < E; ++e) so[wave][lane * E + e] = o[e];
  __syncthreads();
  if (threadIdx.x >= HD) return;
  m = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  const float safe = m == -INFINITY ? 0.f : m;
  float y = 0.f;
  l = 0.f;
  for (int w = 0; w < 4; ++w) { const float f = expf(sm[w] - safe); l = fmaf(f, sl[w], l); y = fmaf(f, so[w][threadIdx.x], y); }
  put((T*)a.out + row * a.o_tok + h * a.o_head + threadIdx.x, l == 0.f ? 0.f : y / l);
  if (a.lse && threadIdx.x == 0) a.lse[(int64_t)row * a.heads + h] = l == 0.f ? -INFINITY : m + logf(l);
}

template <typename T>
hipError_t attn_go(const PagedAttnArgs& a, int head_dim, hipStream_t stream) {
  const dim3 grid(a.b.n_tokens, a.heads);
  if (head_dim == 64) hipLaunchKernelGGL((paged_attn_kernel<T, 64>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((paged_attn_kernel<T, 128>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

int check_attention(const ppd_paged_cache* cache, const ppd_paged_batch* batch, int n_heads) {
  const int rc = check_paged(cache, batch);
  if (rc) return rc;
  if (n_heads < 1 || n_heads % cache->n_kv_heads) return PPD_EINVAL;
  return n_heads > PPD_MAX_HEADS ? PPD_ELIMIT : PPD_OK;
}

}  // namespace

extern "C" int ppd_paged_attention_workspace(const ppd_paged_cache* cache, const ppd_paged_batch* batch, int n_heads, uint64_t* bytes) {
  const int rc = check_attention(cache, batch, n_heads);
  if (rc) return rc;
  if (!bytes) return PPD_EINVAL;
  *bytes = 0;
  return PPD_OK;
}

extern "C" int ppd_paged_attention(const ppd_paged_cache* cache, const ppd_paged_batch* batch, int n_heads, const ppd_rows* q,
                                   const ppd_rows* out, float* lse, float scale, int window, void* workspace,
                                   uint64_t workspace_bytes, void* hip_stream) {
  uint64_t need = 0;
  const int rc = ppd_paged_attention_workspace(cache, batch, n_heads, &need);
  if (rc) return rc;
  const int dt = cache->dtype, n = batch->n_tokens;
  if (!(scale > 0.f && isfinite(scale)) || window < 0) return PPD_EINVAL;
  if (n == 0) return PPD_OK;
  if (!good_rows(q, n, n_heads, dt, false) || !good_rows(out, n, n_heads, dt, true) || ((uintptr_t)lse & 3)) return PPD_EINVAL;
  if (need && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < need)) return PPD_EINVAL;
  PagedAttnArgs a;
  a.b = batch_of(*cache, *batch);
  a.q = q->p; a.out = out->p; a.lse = lse; a.kc = cache->k; a.vc = cache->v;
  a.q_tok = q->token; a.q_head = q->head; a.o_tok = out->token; a.o_head = out->head;
  a.kc_page = cache->k_page; a.kc_pos = cache->k_pos; a.kc_head = cache->k_head; a.vc_page = cache->v_page; a.vc_pos = cache->v_pos; a.vc_head = cache->v_head;
  a.heads = n_heads; a.kv_heads = cache->n_kv_heads; a.window = window; a.scale = scale;
  hipStream_t st = (hipStream_t)hip_stream;
  return launched(dt == PPD_FP32 ? attn_go<float>(a, cache->head_dim, st)
                  : dt == PPD_BF16 ? attn_go<bf16_t>(a, cache->head_dim, st) : attn_go<f16_t>(a, cache->head_dim, st));
}
