// ppd_paged_attention_fp4: attention of ragged runs of new tokens over pages of 4-bit keys and values.  Few rows over many positions, and the
// host's side; many rows: ppd_paged_tiles_fp4.hip.
#include "ppd_paged_attn_fp4.h"

#include <math.h>

using namespace ppd;

namespace {

// ---- few rows, many positions.  As paged_split_kernel: a wave has every fourth step of 32 positions of its part to itself.  A lane's share of a
// key is a quarter of it, 32 numbers of one scale (head_dim 64: 16), which it widens to the left operands of as many products; the queries lie in
// that order, too.  Values are widened in rows, too, and go through LDS rows of the wave's own, from where the transposing reads take them.
// The next step's codes and scales are under way while one is worked on.
template <int HD>
struct Split4 {
  static constexpr int BP = 32, NT = 2;
  static constexpr int ROW = HD / 2, LANE = ROW / 4, NW = LANE / 4;     // bytes of a row and of a lane's quarter; words of that, each of eight codes
  static constexpr int STRIDE = HD * 2 + 32;                            // of a row of values in LDS: no two rows of an operand on the same banks
  static constexpr int WAVE_LDS = BP * STRIDE;
  static constexpr int OUT_LDS = SPLIT_ROWS * (HD + 4) * 4 + SPLIT_ROWS * 8;
  static constexpr int LDS = SPLIT_WAVES * (WAVE_LDS > OUT_LDS ? WAVE_LDS : OUT_LDS);
};
template <int N> struct Words;                // a lane's code words as they are loaded
template <> struct Words<2> { typedef u32x2 type; };
template <> struct Words<4> { typedef u32x4 type; };

template <typename T, int HD, bool NEAR>
__global__ __launch_bounds__(SPLIT_THREADS, sizeof(T) == 4 ? 2 : 3) void paged_split_fp4_kernel(Fp4AttnArgs a) {
  using C = Split4<HD>;
  constexpr int NQ = Terms<T>::Q, NW = Terms<T>::W;
  typedef typename Words<C::NW>::type words;
  __shared__ __align__(16) char lds[C::LDS];
  __shared__ int s_flag;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), kvh = blockIdx.x % a.kv_heads, row = lane & 15, quad = lane >> 4;
  Item it;
  if (!find_item<SPLIT_ROWS>(a, blockIdx.x / a.kv_heads, false, lane, it)) return;
  const int all_rows = it.n * a.group;
  const int r = it.tile * SPLIT_ROWS + row, rc = min(r, all_rows - 1), tok = rc / a.group, head = kvh * a.group + rc % a.group;
  const int pos = r < all_rows ? it.pos0 + tok : -1;                          // what the lane's row sees ends there
  const int from = first_seen(pos, a.window);
  const int tok_first = it.tile * SPLIT_ROWS / a.group, tok_last = min((it.tile * SPLIT_ROWS + SPLIT_ROWS - 1) / a.group, it.n - 1);
  const int all_see_to = it.pos0 + tok_first, all_see_from = first_seen(it.pos0 + tok_last, a.window);
  u32x4 q[C::NW][NQ];
  {
    const T* const p = (const T*)a.q + (int64_t)(it.rows0 + tok) * a.q_tok + (int64_t)head * a.q_head + quad * (HD / 4);
#pragma unroll
    for (int i = 0; i < C::NW; ++i) query_terms(p + 8 * i, a.to_log2, q[i]);
  }
  const float to_log2 = sizeof(T) == 4 ? 1.0f : a.to_log2;                    // (fp32 queries have it already: the largest score's weight is 1 to the bit then)
  char* const mine = lds + wave * C::WAVE_LDS;
  const char* const kbase = (const char*)a.kc + (int64_t)kvh * a.kc_head;
  const char* const vbase = (const char*)a.vc + (int64_t)kvh * a.vc_head;
  const uint8_t* const ksbase = (const uint8_t*)a.ks + (int64_t)kvh * a.ks_head;
  const uint8_t* const vsbase = (const uint8_t*)a.vs + (int64_t)kvh * a.vs_head;
  const int steps = (it.hi - it.lo + C::BP - 1) / C::BP;
  // see paged_split_kernel
  const int32_t* const table = a.b.pages + (int64_t)it.s * a.b.pages_stride;
  int entry, slot;
  auto place = [&](int step) {
    const int p = it.lo + step * C::BP + (lane & (C::BP - 1)), i = (int)((unsigned)p / (unsigned)a.b.page_size);
    slot = p - i * a.b.page_size;
    entry = table[min(i, a.b.max_pages - 1)];
  };
  // keys: lane (row, quad) has quarter `quad` of positions 16 t + row; values: lane has quarter lane % 4 of positions 16 t + lane / 4
  const int vrow = lane >> 2, vquad = lane & 3;
  words k[2][C::NT], v[2][C::NT];
  uint32_t ks[2][C::NT], vs[2][C::NT];
  uint32_t there[2];                                      // a bit for each of a step's positions that has a page
  auto request = [&](int step, auto set) {
    constexpr int S = decltype(set)::value;
    const int page = it.lo + step * C::BP + (lane & (C::BP - 1)) < it.hi && (unsigned)entry < (unsigned)a.b.n_pages ? entry : -1;      // (hi is within the table)
    there[S] = (uint32_t)__ballot(page >= 0);
    // what has no page is read from where there is something, and not used
    if constexpr (NEAR) {
#pragma unroll
      for (int t = 0; t < C::NT; ++t) {
        const int pg = __builtin_amdgcn_readlane(page, 16 * t), sl = pg >= 0 ? __builtin_amdgcn_readlane(slot, 16 * t) : 0;
        const int64_t at = max(pg, 0);
        const char* const kp = kbase + at * a.kc_page + (int64_t)sl * a.kc_pos;
        const char* const vp = vbase + at * a.vc_page + (int64_t)sl * a.vc_pos;
        const uint8_t* const ksp = ksbase + at * a.ks_page + (int64_t)sl * a.ks_pos;
        const uint8_t* const vsp = vsbase + at * a.vs_page + (int64_t)sl * a.vs_pos;
        k[S][t] = *(const words*)(kp + (unsigned)(row * (int)a.kc_pos + quad * C::LANE));
        ks[S][t] = ksp[(unsigned)(row * (int)a.ks_pos + quad * (HD / 4) / FP4_BLOCK)];
        v[S][t] = *(const words*)(vp + (unsigned)(vrow * (int)a.vc_pos + vquad * C::LANE));
        vs[S][t] = vsp[(unsigned)(vrow * (int)a.vs_pos + vquad * (HD / 4) / FP4_BLOCK)];
      }
    } else {
      const int pg = max(page, 0), sl = page >= 0 ? slot : 0;
#pragma unroll
      for (int t = 0; t < C::NT; ++t) {
        const int64_t kpg = __shfl(pg, 16 * t + row, WAVE), ksl = __shfl(sl, 16 * t + row, WAVE);
        const int64_t vpg = __shfl(pg, 16 * t + vrow, WAVE), vsl = __shfl(sl, 16 * t + vrow, WAVE);
        k[S][t] = *(const words*)(kbase + kpg * a.kc_page + ksl * a.kc_pos + quad * C::LANE);
        ks[S][t] = ksbase[kpg * a.ks_page + ksl * a.ks_pos + quad * (HD / 4) / FP4_BLOCK];
        v[S][t] = *(const words*)(vbase + vpg * a.vc_page + vsl * a.vc_pos + vquad * C::LANE);
        vs[S][t] = vsbase[vpg * a.vs_page + vsl * a.vs_pos + vquad * (HD / 4) / FP4_BLOCK];
      }
    }
  };
  f32x4 o[HD / 16];
  float m, l;                                             // the row's reference (its maximum of scores times to_log2; the same in its four lanes) and the lane's part of the sum
  uint32_t nans = 0;                                      // blocks of 32 components with a value that is NaN and seen
  auto work = [&](int step, auto set) {
    constexpr int S = decltype(set)::value;
    const int base = it.lo + step * C::BP;
    const uint32_t have = there[S];
    const bool whole = have == ~0u && base + C::BP - 1 <= all_see_to && base >= all_see_from;
    f32x4 s[C::NT];
#pragma unroll
    for (int t = 0; t < C::NT; ++t) {
      s[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
      const float scale = fp4_scale(ks[S][t]);
#pragma unroll
      for (int i = 0; i < C::NW; ++i) {
        const u32x4 w = fp4_wide(k[S][t][i], scale);
#pragma unroll
        for (int n = 0; n < NQ; ++n) s[t] = mma16(w, q[i][n], s[t], bf16_t());
      }
    }
    if (!whole) {
      asm volatile("");                                   // (a branch, not selections that every step goes through)
      const int to = pos - base - 4 * quad, since = from - base - 4 * quad;
      const uint32_t mapped = have >> (4 * quad);
#pragma unroll
      for (int t = 0; t < C::NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool seen = ((mapped >> (16 * t + e) & 1) != 0) & (16 * t + e <= to) & (16 * t + e >= since);
          s[t][e] = seen ? s[t][e] : -INFINITY;
        }
    }
    // Values that are NaN go in as zeros, as a weight of zero does not silence them, and are put in behind the loop where they are seen.  (All others are
    // finite, whatever lies where nothing is seen.)
    uint64_t nan[C::NT];
#pragma unroll
    for (int t = 0; t < C::NT; ++t) {
      nan[t] = __ballot(vs[S][t] >= FP4_NAN);
      const float scale = vs[S][t] >= FP4_NAN ? 0.0f : __uint_as_float(vs[S][t] << 23);
#pragma unroll
      for (int i = 0; i < C::NW; ++i) *(u32x4*)(mine + (16 * t + vrow) * C::STRIDE + vquad * (HD / 2) + 16 * i) = fp4_wide(v[S][t][i], scale);
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
    float total = 0.f;                                    // (a step's weights among themselves first: one by one, those below half a step of the row's sum would leave no trace in it)
#pragma unroll
    for (int t = 0; t < C::NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) { s[t][e] = __builtin_amdgcn_exp2f(fmaf(s[t][e], to_log2, -ref)); total += s[t][e]; }
    l += total;
    u32x4 w[NW];
#pragma unroll
    for (int n = 0; n < NW; ++n)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const uint32_t p = pair(s[t][e], s[t][e + 1], bf16_t());
          w[n][2 * t + e / 2] = p;
          if (n + 1 < NW) { float x = s[t][e], y = s[t][e + 1]; rest(p, x, y, bf16_t()); s[t][e] = x; s[t][e + 1] = y; }
        }
    const char* src = mine + (4 * quad + (row >> 2)) * C::STRIDE + (row & 3) * 8;
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) {
      const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(src + i * 32));
      const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(src + 16 * C::STRIDE + i * 32));
      const u32x2 xu = __builtin_bit_cast(u32x2, x), yu = __builtin_bit_cast(u32x2, y);
      const u32x4 vt = {xu.x, xu.y, yu.x, yu.y};
#pragma unroll
      for (int n = 0; n < NW; ++n) o[i] = mma16(vt, w[n], o[i], bf16_t());
    }
    if (nan[0] | nan[1])
#pragma unroll
      for (int t = 0; t < C::NT; ++t)
        for (uint64_t bits = nan[t]; bits; bits &= bits - 1) {      // (by position and quarter of the row)
          const int at = __builtin_ctzll(bits), p = 16 * t + at / 4;
          if (((have >> p) & 1) && base + p <= pos && base + p >= from) nans |= 1u << at % 4 * (HD / 4) / FP4_BLOCK;
        }
  };
#pragma unroll
  for (int i = 0; i < HD / 16; ++i) o[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
  m = -INFINITY; l = 0.f;
  const std::integral_constant<int, 0> even;
  const std::integral_constant<int, 1> uneven;
  place(wave);
  if (wave < steps) request(wave, even);
  place(wave + SPLIT_WAVES);
  for (int step = wave; step < steps; step += 2 * SPLIT_WAVES) {
    const int next = step + SPLIT_WAVES, after = next + SPLIT_WAVES;
    if (next < steps) request(next, uneven);
    place(after);
    work(step, even);
    if (next >= steps) break;
    if (after < steps) request(after, even);
    place(after + SPLIT_WAVES);
    work(next, uneven);
  }
#pragma unroll
  for (int i = 0; i < HD / 16; ++i) if (nans >> i / 2 & 1) o[i] = (f32x4){__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
  l += __shfl_xor(l, 16, WAVE);
  l += __shfl_xor(l, 32, WAVE);
  // ---- the waves' results
  __syncthreads();
  float* const so = (float*)(lds + wave * C::OUT_LDS);
#pragma unroll
  for (int i = 0; i < HD / 16; ++i) *(f32x4*)(so + row * (HD + 4) + 16 * i + 4 * quad) = o[i];
  if (quad == 0) ((float2*)(so + SPLIT_ROWS * (HD + 4)))[row] = make_float2(m, l);
  __syncthreads();
  join_waves<T, HD>(a, it, kvh, tid, lds, C::OUT_LDS);
  if (it.parts > 1) join_parts<T, HD>(a, it, kvh, tid, &s_flag);
}

// ---- host
struct AttnPlan {
  bool tiles;               // paged_tile_fp4_kernel, not paged_split_fp4_kernel
  int want, fine, least, whole;      // see PagedAttnArgs
  int64_t items;            // workgroups per key/value head: parts aimed at, and a part's end for every tile
  uint64_t o_bytes, ml_bytes, more_bytes;      // more: stamps, or the plan
};

int check_attention(const ppd_paged_cache_fp4* cache, const ppd_paged_batch* batch, int n_heads, AttnPlan* p) {
  const int rc = check_paged_fp4(cache, batch);
  if (rc) return rc;
  if (n_heads < 1 || n_heads % cache->n_kv_heads) return PPD_EINVAL;
  if (n_heads > PPD_MAX_HEADS || (int64_t)batch->n_tokens * (n_heads / cache->n_kv_heads) > 1 << 26) return PPD_ELIMIT;
  const int group = n_heads / cache->n_kv_heads;
  const int64_t rows = (int64_t)batch->n_tokens * group, some = batch->n_tokens < batch->n_seqs ? batch->n_tokens : batch->n_seqs;
  const int64_t capacity = (int64_t)batch->max_pages * cache->page_size;
  p->tiles = cache->dtype != PPD_FP32 && rows > 32 * (int64_t)batch->n_seqs && (rows * cache->n_kv_heads > 1024 || capacity > 8192);
  const int tile_rows = p->tiles ? TILE_ROWS : SPLIT_ROWS;
  const int64_t tiles = rows / tile_rows + some;
  const int slots = p->tiles ? 512 : 256;
  p->want = slots / cache->n_kv_heads + (slots < cache->n_kv_heads);
  p->fine = p->tiles || tiles * cache->n_kv_heads < 160 ? p->want : p->want * 7 / 4;
  p->whole = p->tiles ? 8 : 4;
  p->least = p->tiles ? 8 : 2;
  // Tiles enough for the whole chip, or no position to cut at: one part each.
  if (tiles >= (p->tiles ? 2 : 8) * p->want || capacity <= p->whole * PLAN_BLOCK) p->least = 0;
  p->items = tiles + (p->least ? p->fine + 1 : 0);
  if (p->items * cache->n_kv_heads >= (int64_t)1 << 24) return PPD_ELIMIT;      // (a launch has fewer than 2^32 threads, 256 to a workgroup)
  const uint64_t places = p->least ? (uint64_t)p->items * cache->n_kv_heads : 0;
  p->o_bytes = places * tile_rows * cache->head_dim * 4;
  p->ml_bytes = places * tile_rows * 8;
  p->more_bytes = !p->least ? 0 : p->tiles ? (uint64_t)batch->n_seqs * 8 : places * 8;
  return PPD_OK;
}

template <typename T, int HD>
hipError_t attn_go(const Fp4AttnArgs& a, int dtype, hipStream_t stream) {
  if (a.tile_rows == TILE_ROWS) return launch_paged_tiles_fp4(a, dtype, HD, stream);
  if (near_pages_fp4(a)) hipLaunchKernelGGL((paged_split_fp4_kernel<T, HD, true>), dim3(a.items * a.kv_heads), dim3(SPLIT_THREADS), 0, stream, a);
  else hipLaunchKernelGGL((paged_split_fp4_kernel<T, HD, false>), dim3(a.items * a.kv_heads), dim3(SPLIT_THREADS), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

extern "C" int ppd_paged_attention_fp4_workspace(const ppd_paged_cache_fp4* cache, const ppd_paged_batch* batch, int n_heads, uint64_t* bytes) {
  AttnPlan p;
  const int rc = check_attention(cache, batch, n_heads, &p);
  if (rc) return rc;
  if (!bytes) return PPD_EINVAL;
  *bytes = p.o_bytes + p.ml_bytes + p.more_bytes;
  return PPD_OK;
}

extern "C" int ppd_paged_attention_fp4(const ppd_paged_cache_fp4* cache, const ppd_paged_batch* batch, int n_heads, const ppd_rows* q,
                                       const ppd_rows* out, float* lse, float scale, int window, void* workspace,
                                       uint64_t workspace_bytes, void* hip_stream) {
  AttnPlan p;
  const int rc = check_attention(cache, batch, n_heads, &p);
  if (rc) return rc;
  const int dt = cache->dtype, n = batch->n_tokens;
  if (!(scale > 0.f && isfinite(scale * 1.44269504f)) || window < 0) return PPD_EINVAL;
  if (n == 0) return PPD_OK;
  if (!good_rows(q, n, n_heads, dt, false) || !good_rows(out, n, n_heads, dt, true) || ((uintptr_t)lse & 3)) return PPD_EINVAL;
  const uint64_t need = p.o_bytes + p.ml_bytes + p.more_bytes;
  if (need && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < need)) return PPD_EINVAL;
  Fp4AttnArgs a;
  a.b = batch_of(*cache, *batch);
  a.q = q->p; a.out = out->p; a.lse = lse; a.kc = cache->k; a.vc = cache->v; a.ks = cache->k_scales; a.vs = cache->v_scales;
  a.q_tok = q->token; a.q_head = q->head; a.o_tok = out->token; a.o_head = out->head;
  a.kc_page = cache->k_page; a.kc_pos = cache->k_pos; a.kc_head = cache->k_head; a.vc_page = cache->v_page; a.vc_pos = cache->v_pos; a.vc_head = cache->v_head;
  a.ks_page = cache->ks_page; a.ks_pos = cache->ks_pos; a.ks_head = cache->ks_head; a.vs_page = cache->vs_page; a.vs_pos = cache->vs_pos; a.vs_head = cache->vs_head;
  a.heads = n_heads; a.kv_heads = cache->n_kv_heads; a.group = n_heads / cache->n_kv_heads; a.window = window; a.to_log2 = scale * 1.44269504f;
  a.tile_rows = p.tiles ? TILE_ROWS : SPLIT_ROWS; a.items = (int)p.items; a.want = p.want; a.fine = p.fine; a.least = p.least; a.whole = p.whole;
  a.part_o = (float*)workspace; a.part_ml = (float2*)((char*)workspace + p.o_bytes); a.stamps = (uint64_t*)((char*)workspace + p.o_bytes + p.ml_bytes);
  a.plan = (int2*)a.stamps;
  a.stamp = next_stamp();
  hipStream_t st = (hipStream_t)hip_stream;
  if (cache->head_dim == 64)
    return launched(dt == PPD_FP32 ? attn_go<float, 64>(a, dt, st) : dt == PPD_BF16 ? attn_go<bf16_t, 64>(a, dt, st) : attn_go<f16_t, 64>(a, dt, st));
  return launched(dt == PPD_FP32 ? attn_go<float, 128>(a, dt, st) : dt == PPD_BF16 ? attn_go<bf16_t, 128>(a, dt, st) : attn_go<f16_t, 128>(a, dt, st));
}
