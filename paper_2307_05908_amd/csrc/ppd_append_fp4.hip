// ppd_paged_append_fp4: queries and keys normalised per head and rotated to their positions, keys and values into pages of 4-bit numbers.
// Bound by reading the rows and writing queries (and, where asked for, the values that the pages have now), and, close behind, by the keys' arithmetic in 64 bits:
// 4915 bf16 tokens of 40 + 2 * 40 heads, 329 MB, take 84 us among others, 3.9 TB/s (a copy 67; a launch under a trace, or replayed, 94); with the keys' scales and codes from 32 bits
// a trace had 79, but a key next to a border would have a code that depends on the order of operations.  Bounds in 32 bits first, and 64 bits only where these leave it open, were no faster (94 of then 93), and
// no exchange between lanes or other order of the angles in LDS was either.
#include "ppd_divide.h"
#include "ppd_paged_fp4.h"

#include <math.h>

using namespace ppd;

namespace {

struct AppendArgs {
  Batch b;
  const void *q, *k, *v; void *q_out, *k_out, *v_out;
  int64_t q_tok, q_head, qo_tok, qo_head, k_tok, k_head, v_tok, v_head, ko_tok, ko_head, vo_tok, vo_head;
  uint8_t *kc, *vc, *ks, *vs;
  int64_t kc_page, kc_pos, kc_head, vc_page, vc_pos, vc_head, ks_page, ks_pos, ks_head, vs_page, vs_pos, vs_head;
  const void *q_gain, *k_gain;
  int heads, kv_heads, rotary;
  float eps;
  int toks;              // tokens of a workgroup
  Divider by_heads, by_kv_heads;
  double turns[64];      // angle of pair i per position, in whole turns
};

// Four sets of heads' rows a workgroup from this many sets on, see ppd_append.hip (4915 tokens of 8 sets, keys' codes then a little slower: 93 us, one set a workgroup 112, two 96, eight 92).
constexpr int MANY = 2048;
// Of these, several tokens a workgroup, two sets together, where a token's rows fill no more than one (bf16, head_dim 128, us of one token / several: 35291 tokens of 2 + 2 * 1
// heads 107 / 38, 2400 of 8 + 2 * 1 13.5 / 9.7, 16913 of 2 + 2 * 2 56 / 30, 7331 of 8 + 2 * 2 29 / 24; with rows for more than one set, 16 + 2 * 4, in four sets, 39 / 41).
constexpr int TOKENS = 8;      // of a workgroup at most (16 were no faster)

// sin and cos of 2 pi t in 64 bits: the nearest quarter turn taken off, the rest (at most pi / 4) by the Taylor series, whose next terms are
// below 2^-53.
__device__ __forceinline__ double2 sincos_turns(double t) {
  t -= rint(t);
  const double quarter = rint(4.0 * t), x = (t - 0.25 * quarter) * 6.283185307179586476925286766559, y = x * x;
  double s = fma(y, 1.0 / 1307674368000.0, -1.0 / 6227020800.0), c = fma(y, 1.0 / 20922789888000.0, -1.0 / 87178291200.0);
  s = fma(y, s, 1.0 / 39916800.0); s = fma(y, s, -1.0 / 362880.0); s = fma(y, s, 1.0 / 5040.0); s = fma(y, s, -1.0 / 120.0); s = fma(y, s, 1.0 / 6.0);
  s = fma(-y * x, s, x);
  c = fma(y, c, 1.0 / 479001600.0); c = fma(y, c, -1.0 / 3628800.0); c = fma(y, c, 1.0 / 40320.0); c = fma(y, c, -1.0 / 720.0); c = fma(y, c, 1.0 / 24.0); c = fma(y, c, -0.5);
  c = fma(y, c, 1.0);
  const int n = (int)quarter & 3;
  const double a = n & 1 ? c : s, d = n & 1 ? s : c;
  return make_double2(n & 2 ? -a : a, (n + 1) & 2 ? -d : d);
}

template <typename T> __device__ __forceinline__ typename Quad<T>::raw narrow_bf16(uint32_t a, uint32_t b);      // four bf16 numbers in the type
template <> __device__ __forceinline__ u32x4 narrow_bf16<float>(uint32_t a, uint32_t b) { return (u32x4){a << 16, a & 0xffff0000u, b << 16, b & 0xffff0000u}; }
template <> __device__ __forceinline__ u32x2 narrow_bf16<bf16_t>(uint32_t a, uint32_t b) { return (u32x2){a, b}; }
template <> __device__ __forceinline__ u32x2 narrow_bf16<f16_t>(uint32_t a, uint32_t b) { return Quad<f16_t>::narrow(Quad<bf16_t>::wide((u32x2){a, b})); }

__device__ __forceinline__ uint32_t most_of_block(uint32_t m) {      // over the four lanes that have a block
  m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xf, 0xf, false));
  return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xf, 0xf, false));
}
// A 64-bit number below 2^128 as fp32, cut off and with its last bit set where something was: on the same side of every border between codes.  (One below
// 2^-126 as one below 2^-126.)
__device__ __forceinline__ float odd_f32(double d) {
  const uint32_t hi = (uint32_t)__double2hiint(d), lo = (uint32_t)__double2loint(d);
  const uint32_t f = __builtin_amdgcn_alignbit(max(hi & 0x7fffffffu, 896u << 20) - (896u << 20), lo, 29) | min(lo << 3, 1u);
  return __uint_as_float(f | (hi & 0x80000000u));
}

// A row of head_dim elements is HD / 8 lanes' work: lane l has elements 8 l .. 8 l + 7, an eighth of the row's code words and a quarter of a
// block of 32, and brings the elements that its own are turned with, too, so that nothing crosses lanes but the norm's sum and a block's largest
// magnitude.  A workgroup has one token and ITERS times 16 (32) of its heads' rows, or (SEVERAL) that many rows of a few tokens, all under way
// while the tokens' sequences, pages and angles are found.
template <typename T, int HD, int ITERS, bool SEVERAL>
__global__ __launch_bounds__(256) void append_fp4_kernel(AppendArgs a) {
  typedef typename Quad<T>::raw raw;
  constexpr int LPR = HD / 8, RPW = WAVE / LPR, TOKS = SEVERAL ? TOKENS : 1;
  __shared__ double2 angles[TOKS][HD / 2];
  __shared__ int s_pos[TOKS], s_page[TOKS], s_slot[TOKS];      // (s_slot -1: a row of no sequence)
  const int tok0 = SEVERAL ? blockIdx.x * a.toks : blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l = lane % LPR, half = a.rotary / 2;
  int own[2], other[2], angle[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int e = 8 * l + 4 * h;
    own[h] = e;
    angle[h] = e < half ? e : e - half;
    other[h] = e < half ? e + half : e < a.rotary ? e - half : e;
  }
  const int rows = a.heads + 2 * a.kv_heads, first = (SEVERAL ? 0 : blockIdx.y * ITERS * 4 * RPW) + wave * RPW + lane / LPR;
  const int toks = SEVERAL ? min(a.toks, a.b.n_tokens - tok0) : 1, all = toks * rows;
  // number i of the workgroup's rows: its token, and its number r of the token's.  Of several tokens the queries come first, then the keys, and the values: a wave has
  // rows of one kind, mostly (token by token, as one token's are, 54 us, not 44, for the first of TOKENS' sizes in four sets).
  auto row_of = [&](int i, int& t, int& r) {
    t = 0; r = i;
    if constexpr (SEVERAL) {
      const int k = i - toks * a.heads, v = k - toks * a.kv_heads;
      t = (int)(k < 0 ? a.by_heads((uint32_t)i) : a.by_kv_heads((uint32_t)(v < 0 ? k : v)));
      r = k < 0 ? i - t * a.heads : v < 0 ? a.heads + k - t * a.kv_heads : a.heads + a.kv_heads + v - t * a.kv_heads;
    }
  };
  raw ra[ITERS][2], rb[ITERS][2], gains[2][4] = {};
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    int t, r;
    const int i = first + it * 4 * RPW;
    row_of(i, t, r);
    const int tok = tok0 + t;
    const bool turned = r < a.heads + a.kv_heads && half > 0;
    const T* const src = r < a.heads ? (const T*)a.q + tok * a.q_tok + r * a.q_head
                       : r < a.heads + a.kv_heads ? (const T*)a.k + tok * a.k_tok + (r - a.heads) * a.k_head
                       : (const T*)a.v + tok * a.v_tok + (r - a.heads - a.kv_heads) * a.v_head;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      ra[it][h] = {}; rb[it][h] = {};
      if (i < all) ra[it][h] = *(const raw*)(src + own[h]);
      if (i < all && turned) rb[it][h] = *(const raw*)(src + other[h]);
    }
  }
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const T* const gain = (const T*)(g ? a.k_gain : a.q_gain);
    if (gain)
#pragma unroll
      for (int h = 0; h < 2; ++h) { gains[g][h] = *(const raw*)(gain + own[h]); gains[g][2 + h] = *(const raw*)(gain + other[h]); }
  }
  auto find = [&](int tok, int& pos, int& page, int& slot) {
    const int s = seq_of_row(a.b, tok, lane);
    if (s < 0) return false;
    const SeqRows sr = seq_rows(a.b, s);
    pos = sr.pos0 + (tok - sr.row0);
    page = page_of(a.b, s, pos);
    slot = page < 0 ? 0 : (int)((unsigned)pos % (unsigned)a.b.page_size);
    return true;
  };
  int pos, page = -1, slot = 0;
  if constexpr (SEVERAL) {
    for (int t = wave; t < toks; t += 4) {
      const bool there = find(tok0 + t, pos, page, slot);
      if (lane == 0) { s_pos[t] = pos; s_page[t] = page; s_slot[t] = there ? slot : -1; }
    }
    __syncthreads();
    if (half > 0) {
      for (int x = threadIdx.x; x < toks * (HD / 2); x += 256) {
        const int t = x / (HD / 2), i = x % (HD / 2);
        if (i < half && s_slot[t] >= 0) angles[t][i] = sincos_turns((double)s_pos[t] * a.turns[i]);
      }
      __syncthreads();
    }
  } else {
    if (!find(tok0, pos, page, slot)) return;              // (all of the workgroup)
    if (half > 0) {
      if ((int)threadIdx.x < half) angles[0][threadIdx.x] = sincos_turns((double)pos * a.turns[threadIdx.x]);
      __syncthreads();
    }
  }
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    int t, r;
    const int i = first + it * 4 * RPW;
    row_of(i, t, r);
    const int tok = tok0 + t;
    if (i >= all) continue;
    if constexpr (SEVERAL) {
      page = s_page[t]; slot = s_slot[t];
      if (slot < 0) continue;
    }
    if (r < a.heads) {
      f32x4 x[2], y[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) { x[h] = Quad<T>::wide(ra[it][h]); y[h] = Quad<T>::wide(rb[it][h]); }
      if (a.q_gain) {
        float t = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) t = fmaf(x[0][e], x[0][e], fmaf(x[1][e], x[1][e], t));
        t += dpp_f32<0xB1>(t);                   // over the row's lanes
        t += dpp_f32<0x4E>(t);
        t += dpp_f32<0x141>(t);
        if (LPR == 16) t += dpp_f32<0x140>(t);
        const float rs = 1.0f / sqrtf(t * (1.0f / HD) + a.eps);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f32x4 ga = Quad<T>::wide(gains[0][h]), gb = Quad<T>::wide(gains[0][2 + h]);
#pragma unroll
          for (int e = 0; e < 4; ++e) { x[h][e] = x[h][e] * rs * ga[e]; y[h][e] = y[h][e] * rs * gb[e]; }
        }
      }
      T* const dst = (T*)a.q_out + tok * a.qo_tok + r * a.qo_head;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (own[h] < a.rotary) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const double2 sc = angles[t][angle[h] + e];
            const float sn = (float)sc.x, cs = (float)sc.y;
            x[h][e] = own[h] < half ? fmaf(x[h][e], cs, -(y[h][e] * sn)) : fmaf(x[h][e], cs, y[h][e] * sn);
          }
        }
        const bool as_is = own[h] >= a.rotary && !a.q_gain;
        *(raw*)(dst + own[h]) = as_is ? ra[it][h] : Quad<T>::narrow(x[h]);
      }
      continue;
    }
    const bool is_k = r < a.heads + a.kv_heads;
    const int kvh = is_k ? r - a.heads : r - a.heads - a.kv_heads;
    float x[8];
    uint32_t byte, most = 0;
    float scale;
    if (is_k) {
      double d[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4 u = Quad<T>::wide(ra[it][h]);
#pragma unroll
        for (int e = 0; e < 4; ++e) d[4 * h + e] = u[e];
      }
      double rs = 1.0;
      if (a.k_gain) {
        double t = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) t = fma(d[e], d[e], t);
        t += dpp_f64<0xB1>(t);
        t += dpp_f64<0x4E>(t);
        t += dpp_f64<0x141>(t);
        if (LPR == 16) t += dpp_f64<0x140>(t);
        rs = 1.0 / sqrt(t * (1.0 / HD) + (double)a.eps);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f32x4 g = Quad<T>::wide(gains[1][h]);
#pragma unroll
          for (int e = 0; e < 4; ++e) d[4 * h + e] *= rs * g[e];
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (own[h] < a.rotary) {
          const f32x4 u = Quad<T>::wide(rb[it][h]), g = Quad<T>::wide(gains[1][2 + h]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const double2 sc = angles[t][angle[h] + e];
            const double y = a.k_gain ? u[e] * (rs * g[e]) : (double)u[e];
            d[4 * h + e] = fma(d[4 * h + e], sc.y, own[h] < half ? -(y * sc.x) : y * sc.x);
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) most = max(most, ((uint32_t)__double2hiint(d[e]) & 0x7fffffffu) | (__double2loint(d[e]) != 0));
      most = most_of_block(most);
      // the least scale, from the upper words (20 bits of significand, the last of them set where there is more)
      const bool endless = most >= 0x7ff00000u;
      const int exponent = min(max((int)((most + 0x3ffffu) >> 20) - 1023 - 2, FP4_LEAST), FP4_MOST);
      byte = endless ? 255 : 127 + exponent;
      if (__ballot(!endless && (exponent < -110 || exponent > 110))) {      // (where fp32 ends: divided by the scale, and cut to what its numbers are)
        scale = 1.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = odd_f32(fmin(fmax(ldexp(d[e], -exponent), -8.0), 8.0));
      } else {
        scale = __uint_as_float((uint32_t)(127 + exponent) << 23);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = odd_f32(d[e]);
      }
    } else {
      const f32x4 u = Quad<T>::wide(ra[it][0]), w = Quad<T>::wide(ra[it][1]);
#pragma unroll
      for (int e = 0; e < 4; ++e) { x[e] = u[e]; x[4 + e] = w[e]; }
#pragma unroll
      for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(x[e]) & 0x7fffffffu);
      byte = fp4_scale_of(most_of_block(most));
      scale = byte == 255 ? 1.0f : fp4_scale(byte);
    }
    const uint32_t codes = byte == 255 ? 0u : fp4_narrow(x, scale);
    if (page >= 0) {
      uint8_t* const c = is_k ? a.kc + page * a.kc_page + slot * a.kc_pos + kvh * a.kc_head : a.vc + page * a.vc_page + slot * a.vc_pos + kvh * a.vc_head;
      uint8_t* const b = is_k ? a.ks + page * a.ks_page + slot * a.ks_pos + kvh * a.ks_head : a.vs + page * a.vs_page + slot * a.vs_pos + kvh * a.vs_head;
      *(uint32_t*)(c + 4 * l) = codes;
      if (l % 4 == 0) b[l / 4] = (uint8_t)byte;
    }
    T* const values = is_k ? (T*)a.k_out : (T*)a.v_out;
    if (values) {
      T* const to = values + (is_k ? tok * a.ko_tok + kvh * a.ko_head : tok * a.vo_tok + kvh * a.vo_head);
      const u32x4 w = fp4_wide(codes, fp4_scale(byte));
      *(raw*)(to + own[0]) = narrow_bf16<T>(w.x, w.y);
      *(raw*)(to + own[1]) = narrow_bf16<T>(w.z, w.w);
    }
  }
}

template <typename T, int HD>
hipError_t append_go(AppendArgs& a, hipStream_t stream) {
  constexpr int PER = 4 * (WAVE / (HD / 8));               // rows of a set
  const int rows = a.heads + 2 * a.kv_heads, sets = (rows + PER - 1) / PER;
  a.toks = 2 * PER / rows < TOKENS ? 2 * PER / rows : TOKENS;
  a.by_heads = Divider((uint32_t)(a.heads > 0 ? a.heads : 1)); a.by_kv_heads = Divider((uint32_t)a.kv_heads);
  if ((int64_t)a.b.n_tokens * sets <= MANY) hipLaunchKernelGGL((append_fp4_kernel<T, HD, 1, false>), dim3(a.b.n_tokens, sets), dim3(256), 0, stream, a);
  else if (a.toks > 1) hipLaunchKernelGGL((append_fp4_kernel<T, HD, 2, true>), dim3((a.b.n_tokens + a.toks - 1) / a.toks), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((append_fp4_kernel<T, HD, 4, false>), dim3(a.b.n_tokens, (sets + 3) / 4), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

extern "C" int ppd_paged_append_fp4(const ppd_paged_cache_fp4* cache, const ppd_paged_batch* batch, int n_heads, const ppd_rows* q,
                                    const ppd_rows* q_out, const ppd_rows* k, const ppd_rows* v, const ppd_rows* k_out,
                                    const ppd_rows* v_out, const void* q_gain, const void* k_gain, float norm_eps, int rotary_dim,
                                    float rope_theta, void* hip_stream) {
  const int rc = check_paged_fp4(cache, batch);
  if (rc) return rc;
  const int dt = cache->dtype, n = batch->n_tokens, kvh = cache->n_kv_heads;
  if (n_heads < 0) return PPD_EINVAL;
  const auto apart = [](int64_t stride, int count) { return count <= 1 || stride > 0; };      // (rows that are written must not lie on each other)
  if (!apart(cache->k_page, cache->n_pages) || !apart(cache->v_page, cache->n_pages) || !apart(cache->ks_page, cache->n_pages) || !apart(cache->vs_page, cache->n_pages) ||
      !apart(cache->k_pos, cache->page_size) || !apart(cache->v_pos, cache->page_size) || !apart(cache->ks_pos, cache->page_size) || !apart(cache->vs_pos, cache->page_size) ||
      !apart(cache->k_head, kvh) || !apart(cache->v_head, kvh) || !apart(cache->ks_head, kvh) || !apart(cache->vs_head, kvh))
    return PPD_EINVAL;
  if (rotary_dim < 0 || rotary_dim > cache->head_dim || rotary_dim % 8) return PPD_EINVAL;
  if (rotary_dim > 0 && !(rope_theta > 0.f && isfinite(rope_theta))) return PPD_EINVAL;
  if ((q_gain || k_gain) && !(norm_eps >= 0.f && isfinite(norm_eps))) return PPD_EINVAL;
  if (((uintptr_t)q_gain | (uintptr_t)k_gain) & (dt == PPD_FP32 ? 15 : 7)) return PPD_EINVAL;
  if (n_heads > PPD_MAX_HEADS) return PPD_ELIMIT;
  if (n == 0) return PPD_OK;
  const auto in_place = [&](const ppd_rows* from, const ppd_rows* to, int heads) {            // (a row's lanes read it before they write it)
    return from->p != to->p || ((n <= 1 || from->token == to->token) && (heads <= 1 || from->head == to->head));
  };
  if (n_heads > 0 && (!good_rows(q, n, n_heads, dt, false) || !good_rows(q_out, n, n_heads, dt, true) || !in_place(q, q_out, n_heads))) return PPD_EINVAL;
  if (!good_rows(k, n, kvh, dt, false) || !good_rows(v, n, kvh, dt, false)) return PPD_EINVAL;
  if (k_out && (!good_rows(k_out, n, kvh, dt, true) || !in_place(k, k_out, kvh))) return PPD_EINVAL;
  if (v_out && (!good_rows(v_out, n, kvh, dt, true) || !in_place(v, v_out, kvh))) return PPD_EINVAL;
  AppendArgs a = {};
  a.b = batch_of(*cache, *batch);
  a.k = k->p; a.v = v->p; a.k_tok = k->token; a.k_head = k->head; a.v_tok = v->token; a.v_head = v->head;
  if (n_heads) { a.q = q->p; a.q_out = q_out->p; a.q_tok = q->token; a.q_head = q->head; a.qo_tok = q_out->token; a.qo_head = q_out->head; }
  if (k_out) { a.k_out = k_out->p; a.ko_tok = k_out->token; a.ko_head = k_out->head; }
  if (v_out) { a.v_out = v_out->p; a.vo_tok = v_out->token; a.vo_head = v_out->head; }
  a.kc = (uint8_t*)cache->k; a.vc = (uint8_t*)cache->v; a.ks = (uint8_t*)cache->k_scales; a.vs = (uint8_t*)cache->v_scales;
  a.kc_page = cache->k_page; a.kc_pos = cache->k_pos; a.kc_head = cache->k_head; a.vc_page = cache->v_page; a.vc_pos = cache->v_pos; a.vc_head = cache->v_head;
  a.ks_page = cache->ks_page; a.ks_pos = cache->ks_pos; a.ks_head = cache->ks_head; a.vs_page = cache->vs_page; a.vs_pos = cache->vs_pos; a.vs_head = cache->vs_head;
  a.q_gain = q_gain; a.k_gain = k_gain; a.heads = n_heads; a.kv_heads = kvh; a.rotary = rotary_dim; a.eps = norm_eps;
  // theta^(-2i/r) by repeated products of 64-bit significands: off by 64 halves of 2^-63 at most before each is rounded to 53
  const long double step = rotary_dim ? powl((long double)rope_theta, -2.0L / rotary_dim) : 0.0L;
  long double turn = 1.0L / 6.283185307179586476925286766559005768L;
  for (int i = 0; i < 64; ++i) { a.turns[i] = (double)turn; turn *= step; }
  hipStream_t st = (hipStream_t)hip_stream;
  if (cache->head_dim == 64) return launched(dt == PPD_FP32 ? append_go<float, 64>(a, st) : dt == PPD_BF16 ? append_go<bf16_t, 64>(a, st) : append_go<f16_t, 64>(a, st));
  return launched(dt == PPD_FP32 ? append_go<float, 128>(a, st) : dt == PPD_BF16 ? append_go<bf16_t, 128>(a, st) : append_go<f16_t, 128>(a, st));
}
