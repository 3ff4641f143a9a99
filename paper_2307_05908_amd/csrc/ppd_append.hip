// ppd_paged_append: queries and keys normalised per head and rotated to their positions, keys and values into their pages.  Bound by reading
// and writing each row once (4915 bf16 tokens of 120 rows: 59 us, 5.1 TB/s); few tokens: by the chain of lookups (4 to 6 us).
#include "ppd_layers_common.h"

#include <math.h>

using namespace ppd;

namespace {

struct AppendArgs {
  Batch b;
  const void *q, *k, *v; void* q_out; void *kc, *vc;
  int64_t q_tok, q_head, o_tok, o_head, k_tok, k_head, v_tok, v_head;
  int64_t kc_page, kc_pos, kc_head, vc_page, vc_pos, vc_head;
  const void *q_gain, *k_gain;
  int heads, kv_heads, rotary;
  float eps;
  double turns[64];      // angle of pair i per position, in whole turns
};

// Four sets of heads' rows a workgroup from this many sets on: the lookups and the angles are then found once for them all, and a wave's loads
// cover more of their wait; below, more workgroups are quicker.  us at one / four: 107 bf16 tokens of 48 rows 5.2 / 5.9, 777 fp32 ones of 36
// half-rows 6.2 / 6.1, 4915 bf16 ones of 120 rows 104 / 59 (302 MB: 5.1 TB/s, and a large copy reaches 4.6).
constexpr int MANY = 2048;

// sin and cos of 2 pi t, t a whole number of turns and a rest: in 64 bits to the nearest quarter turn, the rest (at most an eighth, so
// at most pi / 4) by the Taylor series, whose next terms are below 2^-29.
__device__ __forceinline__ void sincos_turns(double t, float& sn, float& cs) {
  t -= rint(t);
  const double quarter = rint(4.0 * t);
  const float x = (float)((t - 0.25 * quarter) * 6.283185307179586476925286766559), y = x * x;
  float s = fmaf(y, fmaf(y, fmaf(y, fmaf(y, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -0.16666667f), 0.0f);
  s = fmaf(s, x, x);
  const float c = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.0f);
  const int n = (int)quarter & 3;
  const float a = n & 1 ? c : s, d = n & 1 ? s : c;
  sn = n & 2 ? -a : a;
  cs = (n + 1) & 2 ? -d : d;
}

// A row of head_dim elements is HD / 8 lanes' work: lane l has two runs of four elements that are turned together (or, behind the rotated
// part, copied), so that nothing crosses lanes but the norm's sum.  A workgroup has one token and ITERS times 16 (32) of its heads' rows, all
// under way while the token's sequence, page and angles are found.
template <typename T, int HD, int ITERS>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
  typedef typename Quad<T>::raw raw;
  constexpr int LPR = HD / 8, RPW = WAVE / LPR;
  const int tok = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l = lane % LPR, half = a.rotary / 2, turning = a.rotary / 8;
  const int lo = l < turning ? 4 * l : a.rotary + 8 * (l - turning), hi = l < turning ? half + 4 * l : lo + 4;
  const int rows = a.heads + 2 * a.kv_heads, first = blockIdx.y * ITERS * 4 * RPW + wave * RPW + lane / LPR;
  raw ra[ITERS], rb[ITERS], gains[4] = {};
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    const int r = first + it * 4 * RPW;
    const T* const src = r < a.heads ? (const T*)a.q + tok * a.q_tok + r * a.q_head
                       : r < a.heads + a.kv_heads ? (const T*)a.k + tok * a.k_tok + (r - a.heads) * a.k_head
                       : (const T*)a.v + tok * a.v_tok + (r - a.heads - a.kv_heads) * a.v_head;
    if (r < rows) { ra[it] = *(const raw*)(src + lo); rb[it] = *(const raw*)(src + hi); } else { ra[it] = {}; rb[it] = {}; }
  }
  if (a.q_gain) { gains[0] = *(const raw*)((const T*)a.q_gain + lo); gains[1] = *(const raw*)((const T*)a.q_gain + hi); }
  if (a.k_gain) { gains[2] = *(const raw*)((const T*)a.k_gain + lo); gains[3] = *(const raw*)((const T*)a.k_gain + hi); }
  const int s = seq_of_row(a.b, tok, lane);
  if (s < 0) return;
  const SeqRows sr = seq_rows(a.b, s);
  const int pos = sr.pos0 + (tok - sr.row0), page = page_of(a.b, s, pos);
  const int slot = page < 0 ? 0 : (int)((unsigned)pos % (unsigned)a.b.page_size);
  f32x4 sn = {0.f, 0.f, 0.f, 0.f}, cs = {1.f, 1.f, 1.f, 1.f};
  if (l < turning) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float u, w;
      sincos_turns((double)pos * a.turns[4 * l + e], u, w);
      sn[e] = u; cs[e] = w;
    }
  }
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    const int r = first + it * 4 * RPW;
    const bool is_q = r < a.heads, is_k = !is_q && r < a.heads + a.kv_heads;
    T* dst;
    if (is_q) dst = (T*)a.q_out + tok * a.o_tok + r * a.o_head;
    else if (is_k) dst = (T*)a.kc + page * a.kc_page + slot * a.kc_pos + (r - a.heads) * a.kc_head;
    else dst = (T*)a.vc + page * a.vc_page + slot * a.vc_pos + (r - a.heads - a.kv_heads) * a.vc_head;
    if (is_q || is_k) {
      f32x4 x = Quad<T>::wide(ra[it]), y = Quad<T>::wide(rb[it]);
      const bool gain = is_q ? a.q_gain != nullptr : a.k_gain != nullptr;
      if (gain) {
        float t = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) t = fmaf(x[e], x[e], fmaf(y[e], y[e], t));
        t += dpp_f32<0xB1>(t);                   // over the row's lanes
        t += dpp_f32<0x4E>(t);
        t += dpp_f32<0x141>(t);
        if (LPR == 16) t += dpp_f32<0x140>(t);
        const float rs = 1.0f / sqrtf(t * (1.0f / HD) + a.eps);
        const f32x4 ga = Quad<T>::wide(is_q ? gains[0] : gains[2]), gb = Quad<T>::wide(is_q ? gains[1] : gains[3]);
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[e] = x[e] * rs * ga[e]; y[e] = y[e] * rs * gb[e]; }
      }
      f32x4 u, w;
#pragma unroll
      for (int e = 0; e < 4; ++e) { u[e] = fmaf(x[e], cs[e], -(y[e] * sn[e])); w[e] = fmaf(y[e], cs[e], x[e] * sn[e]); }
      if (l < turning || gain) { ra[it] = Quad<T>::narrow(l < turning ? u : x); rb[it] = Quad<T>::narrow(l < turning ? w : y); }
    }
    if (r < rows && (is_q || page >= 0)) { *(raw*)(dst + lo) = ra[it]; *(raw*)(dst + hi) = rb[it]; }
  }
}

template <typename T, int HD>
hipError_t append_go(const AppendArgs& a, hipStream_t stream) {
  const int rows = a.heads + 2 * a.kv_heads, per = 4 * (WAVE / (HD / 8)), sets = (rows + per - 1) / per;
  if ((int64_t)a.b.n_tokens * sets <= MANY) hipLaunchKernelGGL((append_kernel<T, HD, 1>), dim3(a.b.n_tokens, sets), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((append_kernel<T, HD, 4>), dim3(a.b.n_tokens, (sets + 3) / 4), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

extern "C" int ppd_paged_append(const ppd_paged_cache* cache, const ppd_paged_batch* batch, int n_heads, const ppd_rows* q,
                                const ppd_rows* q_out, const ppd_rows* k, const ppd_rows* v, const void* q_gain,
                                const void* k_gain, float norm_eps, int rotary_dim, float rope_theta, void* hip_stream) {
  const int rc = check_paged(cache, batch);
  if (rc) return rc;
  const int dt = cache->dtype, n = batch->n_tokens;
  if (n_heads < 0) return PPD_EINVAL;
  const auto apart = [](int64_t stride, int count) { return count <= 1 || stride > 0; };      // (rows that are written must not lie on each other)
  if (!apart(cache->k_page, cache->n_pages) || !apart(cache->v_page, cache->n_pages) || !apart(cache->k_pos, cache->page_size) || !apart(cache->v_pos, cache->page_size) ||
      !apart(cache->k_head, cache->n_kv_heads) || !apart(cache->v_head, cache->n_kv_heads))
    return PPD_EINVAL;
  if (rotary_dim < 0 || rotary_dim > cache->head_dim || rotary_dim % 8) return PPD_EINVAL;
  if (rotary_dim > 0 && !(rope_theta > 0.f && isfinite(rope_theta))) return PPD_EINVAL;
  if ((q_gain || k_gain) && !(norm_eps >= 0.f && isfinite(norm_eps))) return PPD_EINVAL;
  if (((uintptr_t)q_gain | (uintptr_t)k_gain) & (dt == PPD_FP32 ? 15 : 7)) return PPD_EINVAL;
  if (n_heads > PPD_MAX_HEADS) return PPD_ELIMIT;
  if (n == 0) return PPD_OK;
  if (n_heads > 0 && (!good_rows(q, n, n_heads, dt, false) || !good_rows(q_out, n, n_heads, dt, true))) return PPD_EINVAL;
  if (n_heads > 0 && q->p == q_out->p && ((n > 1 && q->token != q_out->token) || (n_heads > 1 && q->head != q_out->head))) return PPD_EINVAL;
  if (!good_rows(k, n, cache->n_kv_heads, dt, false) || !good_rows(v, n, cache->n_kv_heads, dt, false)) return PPD_EINVAL;
  AppendArgs a;
  a.b = batch_of(*cache, *batch);
  a.q = n_heads ? q->p : nullptr; a.q_out = n_heads ? q_out->p : nullptr; a.k = k->p; a.v = v->p; a.kc = cache->k; a.vc = cache->v;
  a.q_tok = n_heads ? q->token : 0; a.q_head = n_heads ? q->head : 0; a.o_tok = n_heads ? q_out->token : 0; a.o_head = n_heads ? q_out->head : 0;
  a.k_tok = k->token; a.k_head = k->head; a.v_tok = v->token; a.v_head = v->head;
  a.kc_page = cache->k_page; a.kc_pos = cache->k_pos; a.kc_head = cache->k_head; a.vc_page = cache->v_page; a.vc_pos = cache->v_pos; a.vc_head = cache->v_head;
  a.q_gain = q_gain; a.k_gain = k_gain; a.heads = n_heads; a.kv_heads = cache->n_kv_heads; a.rotary = rotary_dim; a.eps = norm_eps;
  // theta^(-2i/r) by repeated products: 64 roundings of 2^-53 at most, 1e-8 of a radian at position 10^6
  const double step = rotary_dim ? pow((double)rope_theta, -2.0 / rotary_dim) : 0.0;
  double turn = 1.0 / 6.283185307179586476925286766559;
  for (int i = 0; i < 64; ++i) { a.turns[i] = turn; turn *= step; }
  hipStream_t st = (hipStream_t)hip_stream;
  if (cache->head_dim == 64) return launched(dt == PPD_FP32 ? append_go<float, 64>(a, st) : dt == PPD_BF16 ? append_go<bf16_t, 64>(a, st) : append_go<f16_t, 64>(a, st));
  return launched(dt == PPD_FP32 ? append_go<float, 128>(a, st) : dt == PPD_BF16 ? append_go<bf16_t, 128>(a, st) : append_go<f16_t, 128>(a, st));
}
