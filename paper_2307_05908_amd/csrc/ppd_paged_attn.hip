// ppd_paged_attention: attention of ragged runs of new tokens over paged keys and values.  Few rows over many positions, the join of parts,
// and the host's side; many rows: ppd_paged_tiles.hip.
#include "ppd_paged_attn.h"

#include <math.h>

using namespace ppd;

namespace {

constexpr int SPLIT_WAVES = 4;

// ---- few rows, many positions: bound by the stream of keys and values
// A wave has every fourth step of BP positions of its part to itself: keys straight into registers as the left operand, values through
// registers into LDS rows of its own, from where the transposing reads (fp32: plain ones) make them the left operand of the second product.
// The next step's are requested before this one's arithmetic; nothing waits at a barrier until the four waves' results are joined.
template <typename T, int HD>
struct Split {
  static constexpr int SZ = sizeof(T) == 4 ? 4 : 2, BP = SZ == 4 ? 16 : 32, NT = BP / 16;
  static constexpr int NK = HD * SZ / 64;                 // 16-byte pieces of a key per lane
  static constexpr int LPR = HD * SZ / 16, RPI = WAVE / LPR, NV = BP / RPI;
  static constexpr int STRIDE = HD * SZ + (SZ == 4 ? 16 : 32);   // of a row of values in LDS: no two rows of an operand on the same banks
  static constexpr int WAVE_LDS = BP * STRIDE;
  static constexpr int OUT_LDS = SPLIT_ROWS * (HD + 4) * 4 + SPLIT_ROWS * 8; // a wave's results: sums (rows 16 bytes longer than they are), maxima and totals
  static constexpr int LDS = SPLIT_WAVES * (WAVE_LDS > OUT_LDS ? WAVE_LDS : OUT_LDS);
};

template <typename T, int HD>
__global__ __launch_bounds__(256, 2) void paged_split_kernel(PagedAttnArgs a) {
  using C = Split<T, HD>;
  __shared__ __align__(16) char lds[C::LDS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = blockIdx.y, row = lane & 15, quad = lane >> 4;
  Item it;
  if (!find_item(a, blockIdx.x, blockIdx.x == 0 && kvh == 0 && wave == 0 && a.least > 0, lane, it)) return;
  const int all_rows = it.n * a.group;
  const int r = it.tile * SPLIT_ROWS + row, rc = min(r, all_rows - 1), tok = rc / a.group, head = kvh * a.group + rc % a.group;
  const int pos = r < all_rows ? it.pos0 + tok : -1;                          // what the lane's row sees ends there
  const int from = a.window > 0 ? pos - a.window + 1 : 0;
  const int tok_first = it.tile * SPLIT_ROWS / a.group, tok_last = min((it.tile * SPLIT_ROWS + SPLIT_ROWS - 1) / a.group, it.n - 1);
  const int all_see_to = it.pos0 + tok_first, all_see_from = a.window > 0 ? it.pos0 + tok_last - a.window + 1 : 0;
  u32x4 q[C::NK];
  {
    const char* p = (const char*)a.q + ((int64_t)(it.rows0 + tok) * a.q_tok + (int64_t)head * a.q_head) * C::SZ + quad * 16;
#pragma unroll
    for (int i = 0; i < C::NK; ++i) {
      q[i] = *(const u32x4*)(p + i * 64);
      if (C::SZ == 4)                                     // fp32 queries take the scale along: the largest score's weight is 1 to the bit then
#pragma unroll
        for (int e = 0; e < 4; ++e) q[i][e] = __float_as_uint(__uint_as_float(q[i][e]) * a.to_log2);
    }
  }
  const float to_log2 = C::SZ == 4 ? 1.0f : a.to_log2;
  char* const mine = lds + wave * C::WAVE_LDS;
  const char* const kbase = (const char*)a.kc + (int64_t)kvh * a.kc_head * C::SZ + quad * 16;
  const char* const vbase = (const char*)a.vc + (int64_t)kvh * a.vc_head * C::SZ + (lane % C::LPR) * 16;
  const int steps = (it.hi - it.lo + C::BP - 1) / C::BP;
  // the page (or -1) and slot of position lo + step * BP + (lane % BP)
  auto place = [&](int step, int& page, int& slot) {
    const int p = it.lo + step * C::BP + (lane & (C::BP - 1));
    page = step < steps && p < it.hi ? page_of(a.b, it.s, p) : -1;
    slot = (int)((unsigned)p % (unsigned)a.b.page_size);
  };
  u32x4 k[C::NT][C::NK], v[C::NV];
  uint32_t there = 0;                                     // a bit for each of the step's positions that has a page
  auto request = [&](int page, int slot) {
    there = (uint32_t)__ballot(page >= 0) & (uint32_t)((1ull << C::BP) - 1);
    const int pg = max(page, 0), sl = page >= 0 ? slot : 0;      // what has no page is read from where there is something, and not used
    const int64_t ko = ((int64_t)pg * a.kc_page + (int64_t)sl * a.kc_pos) * C::SZ, vo = ((int64_t)pg * a.vc_page + (int64_t)sl * a.vc_pos) * C::SZ;
#pragma unroll
    for (int t = 0; t < C::NT; ++t) {
      const char* p = kbase + __shfl(ko, 16 * t + row, WAVE);
#pragma unroll
      for (int i = 0; i < C::NK; ++i) k[t][i] = *(const u32x4*)(p + i * 64);
    }
#pragma unroll
    for (int i = 0; i < C::NV; ++i) v[i] = *(const u32x4*)(vbase + __shfl(vo, i * C::RPI + lane / C::LPR, WAVE));
  };
  f32x4 o[HD / 16];
#pragma unroll
  for (int i = 0; i < HD / 16; ++i) o[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;                           // the row's maximum (of scores times to_log2; the same in its four lanes) and the lane's part of the sum
  int page, slot;
  int step = wave;
  place(step, page, slot);
  if (step < steps) request(page, slot);
  place(step + SPLIT_WAVES, page, slot);
  for (; step < steps; step += SPLIT_WAVES) {
    const int base = it.lo + step * C::BP;
    const uint32_t have = there;
    const bool whole = have == (uint32_t)((1ull << C::BP) - 1) && base + C::BP - 1 <= all_see_to && base >= all_see_from;
    f32x4 s[C::NT];
#pragma unroll
    for (int t = 0; t < C::NT; ++t) {
      s[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < C::NK; ++i) {
        if constexpr (C::SZ == 2) s[t] = mma16(k[t][i], q[i], s[t], T());
        else
#pragma unroll
          for (int e = 0; e < 4; ++e) s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[t][i][e]), __uint_as_float(q[i][e]), s[t], 0, 0, 0);
      }
    }
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < C::NV; ++i) {
      const int at = i * C::RPI + lane / C::LPR;
      u32x4 w = v[i];
      if (!whole && !((have >> at) & 1)) w = (u32x4){0u, 0u, 0u, 0u};
      most = largest(most, w, T());
      *(u32x4*)(mine + at * C::STRIDE + (lane % C::LPR) * 16) = w;
    }
    if (step + SPLIT_WAVES < steps) request(page, slot);
    place(step + 2 * SPLIT_WAVES, page, slot);
    const bool odd = __ballot(endless(most, T())) != 0;
    if (!whole) {
#pragma unroll
      for (int t = 0; t < C::NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int at = 16 * t + 4 * quad + e, p = base + at;
          if (!((have >> at) & 1) || p > pos || p < from) s[t][e] = -INFINITY;
        }
    }
    // running maximum: joined and sums rescaled only where it grows for some row
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < C::NT; ++t) top = fmaxf(top, fmaxf(fmaxf(s[t].x, s[t].y), fmaxf(s[t].z, s[t].w)));
    top *= to_log2;
    if (__ballot(top > m)) {
      top = fmaxf(top, __shfl_xor(top, 16, WAVE));
      top = fmaxf(top, __shfl_xor(top, 32, WAVE));
      const float mn = fmaxf(m, top), keep = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= keep;
#pragma unroll
      for (int i = 0; i < HD / 16; ++i) o[i] *= keep;
    }
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int t = 0; t < C::NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) { s[t][e] = __builtin_amdgcn_exp2f(fmaf(s[t][e], to_log2, -ref)); l += s[t][e]; }
    if constexpr (C::SZ == 2) {
      // Weights in two terms of the type: the rounding of one alone is as large as the output's own.  Beside infinite values one: what is left
      // of a weight may be zero or negative, and so that no weight above zero becomes one, half floats go no lower than their smallest number.
      if (sizeof(T) == 2 && std::is_same<T, f16_t>::value && odd)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[t][e] = s[t][e] > 0.f ? fmaxf(s[t][e], 0x1p-24f) : s[t][e];
      u32x4 hi, lo;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        hi[2 * t] = pair(s[t].x, s[t].y, T()); hi[2 * t + 1] = pair(s[t].z, s[t].w, T());
        float x = s[t].x, y = s[t].y, z = s[t].z, w = s[t].w;
        rest(hi[2 * t], x, y, T()); rest(hi[2 * t + 1], z, w, T());
        lo[2 * t] = pair(x, y, T()); lo[2 * t + 1] = pair(z, w, T());
      }
      const char* src = mine + (4 * quad + (row >> 2)) * C::STRIDE + (row & 3) * 8;
#pragma unroll
      for (int i = 0; i < HD / 16; ++i) {
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(src + i * 32));
        const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(src + 16 * C::STRIDE + i * 32));
        const u32x2 xu = __builtin_bit_cast(u32x2, x), yu = __builtin_bit_cast(u32x2, y);
        const u32x4 vt = {xu.x, xu.y, yu.x, yu.y};
        if (odd && whole) o[i] = mma16(vt, hi, o[i], T());
        else if (odd) {
          // a value that is no number, or infinite, among positions that not every row sees: position by position, kept where it is seen
#pragma unroll 1
          for (int p = 0; p < 32; ++p) {
            u32x4 only = {0u, 0u, 0u, 0u};
            const int e = (p >> 4) * 4 + (p & 3);
            if (((p >> 2) & 3) == quad) {
#pragma unroll
              for (int z = 0; z < 4; ++z) if (z == e / 2) only[z] = vt[z] & (e & 1 ? 0xffff0000u : 0xffffu);
            }
            const f32x4 n = mma16(only, hi, o[i], T());
            if (((have >> p) & 1) && base + p <= pos && base + p >= from) o[i] = n;
          }
        } else {
          o[i] = mma16(vt, hi, o[i], T());
          o[i] = mma16(vt, lo, o[i], T());
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < HD / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = *(const float*)(mine + (4 * quad + e) * C::STRIDE + (16 * i + row) * 4);
          if (!whole && odd) {
            for (int c = 0; c < 4; ++c) {
              const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x4f32(c == quad ? x : 0.f, s[0][e], o[i], 0, 0, 0);
              const int p = 4 * c + e;
              if (((have >> p) & 1) && base + p <= pos && base + p >= from) o[i] = n;
            }
          } else o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, s[0][e], o[i], 0, 0, 0);
        }
    }
  }
  l += __shfl_xor(l, 16, WAVE);
  l += __shfl_xor(l, 32, WAVE);
  // ---- the four waves' results
  __syncthreads();
  float* const so = (float*)(lds + wave * C::OUT_LDS);
#pragma unroll
  for (int i = 0; i < HD / 16; ++i) *(f32x4*)(so + row * (HD + 4) + 16 * i + 4 * quad) = o[i];
  if (quad == 0) ((float2*)(so + SPLIT_ROWS * (HD + 4)))[row] = make_float2(m, l);
  __syncthreads();
  for (int x = threadIdx.x; x < SPLIT_ROWS * HD / 4; x += 256) {
    const int rr = x / (HD / 4), d = (x % (HD / 4)) * 4, ri = it.tile * SPLIT_ROWS + rr;
    if (ri >= all_rows) break;
    float2 ml[SPLIT_WAVES];
    float mx = -INFINITY, sum = 0.f;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < SPLIT_WAVES; ++w) { ml[w] = ((const float2*)((const float*)(lds + w * C::OUT_LDS) + SPLIT_ROWS * (HD + 4)))[rr]; mx = fmaxf(mx, ml[w].x); }
    const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
    for (int w = 0; w < SPLIT_WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(ml[w].x - ref);
      sum = fmaf(f, ml[w].y, sum);
      const f32x4 z = *(const f32x4*)((const float*)(lds + w * C::OUT_LDS) + rr * (HD + 4) + d);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = fmaf(f, z[e], y[e]);
    }
    if (it.parts > 1) {
      const int64_t at = ((int64_t)it.slot * a.kv_heads + kvh) * SPLIT_ROWS + rr;
      *(f32x4*)(a.part_o + at * HD + d) = y;
      if (d == 0) a.part_ml[at] = make_float2(mx, sum);
    } else {
      const int t = ri / a.group, h = kvh * a.group + ri % a.group;
      const bool none = mx == -INFINITY && sum == 0.f;    // nothing seen (a score that is no number leaves its mark on the sum)
      const float inv = 1.0f / sum;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = none ? 0.f : y[e] * inv;
      T* to = (T*)a.out + (int64_t)(it.rows0 + t) * a.o_tok + (int64_t)h * a.o_head + d;
      *(typename Quad<T>::raw*)to = quad_out<T>(y);
      if (a.lse && d == 0) a.lse[(int64_t)(it.rows0 + t) * a.heads + h] = none ? -INFINITY : (mx + __builtin_amdgcn_logf(sum)) * 0.69314718f;
    }
  }
}

// The parts of a row joined, in their order: HD / 4 lanes for a row.
template <typename T, int HD>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttnArgs a) {
  constexpr int LPR = HD / 4, RPW = 256 / LPR;
  const int row = blockIdx.x, lane = threadIdx.x & 63;
  const int s = seq_of_row(a.b, row, lane);
  if (s < 0) return;
  const int2 plan = a.plan[s];
  const int parts = plan.y, h = blockIdx.y * RPW + threadIdx.x / LPR, d = (threadIdx.x % LPR) * 4;
  if (parts <= 1 || h >= a.heads) return;
  const SeqRows sr = seq_rows(a.b, s);
  const int kvh = h / a.group, r = (row - sr.row0) * a.group + h % a.group;
  const int64_t first = (int64_t)plan.x + (int64_t)(r / a.tile_rows) * parts;
  float mx = -INFINITY, sum = 0.f;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  for (int p = 0; p < parts; ++p) mx = fmaxf(mx, a.part_ml[((first + p) * a.kv_heads + kvh) * a.tile_rows + r % a.tile_rows].x);
  const float ref = mx == -INFINITY ? 0.f : mx;
  for (int p = 0; p < parts; ++p) {
    const int64_t at = ((first + p) * a.kv_heads + kvh) * a.tile_rows + r % a.tile_rows;
    const float2 ml = a.part_ml[at];
    const float f = __builtin_amdgcn_exp2f(ml.x - ref);
    sum = fmaf(f, ml.y, sum);
    const f32x4 z = *(const f32x4*)(a.part_o + at * HD + d);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = fmaf(f, z[e], y[e]);
  }
  const bool none = mx == -INFINITY && sum == 0.f;
  const float inv = 1.0f / sum;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = none ? 0.f : y[e] * inv;
  *(typename Quad<T>::raw*)((T*)a.out + (int64_t)row * a.o_tok + (int64_t)h * a.o_head + d) = quad_out<T>(y);
  if (a.lse && d == 0) a.lse[(int64_t)row * a.heads + h] = none ? -INFINITY : (mx + __builtin_amdgcn_logf(sum)) * 0.69314718f;
}

// ---- host
struct AttnPlan {
  bool tiles;               // paged_tile_kernel, not paged_split_kernel
  int want, least;          // see PagedAttnArgs
  int64_t items;            // workgroups per key/value head: parts aimed at, and a part's end for every tile
  uint64_t o_bytes, ml_bytes, plan_bytes;
};

int check_attention(const ppd_paged_cache* cache, const ppd_paged_batch* batch, int n_heads, AttnPlan* p) {
  const int rc = check_paged(cache, batch);
  if (rc) return rc;
  if (n_heads < 1 || n_heads % cache->n_kv_heads) return PPD_EINVAL;
  if (n_heads > PPD_MAX_HEADS || (int64_t)batch->n_tokens * (n_heads / cache->n_kv_heads) > 1 << 26) return PPD_ELIMIT;
  const int group = n_heads / cache->n_kv_heads;
  const int64_t rows = (int64_t)batch->n_tokens * group, some = batch->n_tokens < batch->n_seqs ? batch->n_tokens : batch->n_seqs;
  p->tiles = cache->dtype != PPD_FP32 && rows > 32 * (int64_t)batch->n_seqs;
  const int tile_rows = p->tiles ? TILE_ROWS : SPLIT_ROWS, slots = p->tiles ? 512 : 1024;
  const int64_t tiles = rows / tile_rows + some;
  p->want = (slots + cache->n_kv_heads - 1) / cache->n_kv_heads;
  p->least = p->tiles ? 8 : 2;
  // tiles enough for the whole chip, or no position to cut at: one part each
  if (tiles >= 2 * p->want || (int64_t)batch->max_pages * cache->page_size <= p->least * PLAN_BLOCK) p->least = 0;
  p->items = tiles + (p->least ? p->want + 1 : 0);
  const uint64_t kept = p->least ? (uint64_t)p->items * cache->n_kv_heads * tile_rows : 0;
  p->o_bytes = kept * cache->head_dim * 4;
  p->ml_bytes = kept * 8;
  p->plan_bytes = p->least ? ((uint64_t)batch->n_seqs * 8 + 15) & ~15ull : 0;
  return PPD_OK;
}

template <typename T, int HD>
hipError_t attn_go(const PagedAttnArgs& a, int dtype, int items, hipStream_t stream) {
  hipError_t e;
  if (a.tile_rows == TILE_ROWS) e = launch_paged_tiles(a, dtype, HD, items, stream);
  else {
    hipLaunchKernelGGL((paged_split_kernel<T, HD>), dim3(items, a.kv_heads), dim3(256), 0, stream, a);
    e = hipGetLastError();
  }
  if (e != hipSuccess || a.least == 0) return e;
  constexpr int rpw = 256 / (HD / 4);
  hipLaunchKernelGGL((paged_merge_kernel<T, HD>), dim3(a.b.n_tokens, (a.heads + rpw - 1) / rpw), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

extern "C" int ppd_paged_attention_workspace(const ppd_paged_cache* cache, const ppd_paged_batch* batch, int n_heads, uint64_t* bytes) {
  AttnPlan p;
  const int rc = check_attention(cache, batch, n_heads, &p);
  if (rc) return rc;
  if (!bytes) return PPD_EINVAL;
  *bytes = p.o_bytes + p.ml_bytes + p.plan_bytes;
  return PPD_OK;
}

extern "C" int ppd_paged_attention(const ppd_paged_cache* cache, const ppd_paged_batch* batch, int n_heads, const ppd_rows* q,
                                   const ppd_rows* out, float* lse, float scale, int window, void* workspace,
                                   uint64_t workspace_bytes, void* hip_stream) {
  AttnPlan p;
  const int rc = check_attention(cache, batch, n_heads, &p);
  if (rc) return rc;
  const int dt = cache->dtype, n = batch->n_tokens;
  if (!(scale > 0.f && isfinite(scale)) || window < 0) return PPD_EINVAL;
  if (n == 0) return PPD_OK;
  if (!good_rows(q, n, n_heads, dt, false) || !good_rows(out, n, n_heads, dt, true) || ((uintptr_t)lse & 3)) return PPD_EINVAL;
  const uint64_t need = p.o_bytes + p.ml_bytes + p.plan_bytes;
  if (need && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < need)) return PPD_EINVAL;
  PagedAttnArgs a;
  a.b = batch_of(*cache, *batch);
  a.q = q->p; a.out = out->p; a.lse = lse; a.kc = cache->k; a.vc = cache->v;
  a.q_tok = q->token; a.q_head = q->head; a.o_tok = out->token; a.o_head = out->head;
  a.kc_page = cache->k_page; a.kc_pos = cache->k_pos; a.kc_head = cache->k_head; a.vc_page = cache->v_page; a.vc_pos = cache->v_pos; a.vc_head = cache->v_head;
  a.heads = n_heads; a.kv_heads = cache->n_kv_heads; a.group = n_heads / cache->n_kv_heads; a.window = window; a.to_log2 = scale * 1.44269504f;
  a.tile_rows = p.tiles ? TILE_ROWS : SPLIT_ROWS; a.last_first = p.tiles; a.want = p.want; a.least = p.least;
  a.part_o = (float*)workspace; a.part_ml = (float2*)((char*)workspace + p.o_bytes); a.plan = (int2*)((char*)workspace + p.o_bytes + p.ml_bytes);
  hipStream_t st = (hipStream_t)hip_stream;
  const int items = (int)p.items;
  if (cache->head_dim == 64)
    return launched(dt == PPD_FP32 ? attn_go<float, 64>(a, dt, items, st) : dt == PPD_BF16 ? attn_go<bf16_t, 64>(a, dt, items, st) : attn_go<f16_t, 64>(a, dt, items, st));
  return launched(dt == PPD_FP32 ? attn_go<float, 128>(a, dt, items, st) : dt == PPD_BF16 ? attn_go<bf16_t, 128>(a, dt, items, st) : attn_go<f16_t, 128>(a, dt, items, st));
}
