// ppd_paged_attention_fp4: attention of ragged runs of new tokens over pages of 4-bit keys and values.  Few rows over many positions, and the
// host's side; many rows: ppd_paged_tiles_fp4.hip.
#include "ppd_paged_attn_fp4.h"

#include <math.h>

using namespace ppd;

namespace {

// ---- few rows, many positions.  As paged_split_kernel: a wave has every fourth step of 32 positions of its part to itself.  A lane's share of a
// key is a quarter of it, 32 numbers of one scale (head_dim 64: 16), which it widens to the left operands of as many products; the queries lie in
// that order, too.  Values are widened in rows, too, and go through LDS rows of the wave's own, from where the transposing reads take them.
// The next step's codes and scales are under way while one is worked on.  (Two steps were no faster, at two workgroups a unit or three, nor was a copy of the step's
// codes through LDS.)  Bound by the reads, of half a line each where heads are neighbours: 64 bf16 tokens of 32 / 8 heads over 400 to 32000 positions,
// 488 MB, take 123 us, 4.0 TB/s (bf16 pages of the same positions are 1.8 GB), 64 over 4000 63, 4.4 TB/s; the same with the loads taken out half of that.  With 4.25
// bits a number widening counts, too: 38 % of the cycles are vector instructions.
template <int HD, int G>
struct Split4 {
  static constexpr int BP = 32, NT = 2, ROWS = G * SPLIT_ROWS;
  static constexpr int ROW = HD / 2, LANE = ROW / 4, NW = LANE / 4;     // bytes of a row and of a lane's quarter; words of that, each of eight codes
  static constexpr int STRIDE = HD * 2 + 32;                            // of a row of values in LDS: no two rows of an operand on the same banks
  static constexpr int WAVE_LDS = BP * STRIDE;
  static constexpr int OUT_LDS = ROWS * (HD + 4) * 4 + ROWS * 8;
  static constexpr int LDS = SPLIT_WAVES * (WAVE_LDS > OUT_LDS ? WAVE_LDS : OUT_LDS);
};
template <int N> struct Words;                // a lane's code words as they are loaded
template <> struct Words<2> { typedef u32x2 type; };
template <> struct Words<4> { typedef u32x4 type; };

// G: groups of 16 rows that a tile has, which share what is read and widened.
template <typename T, int HD, bool NEAR, int G>
__global__ __launch_bounds__(SPLIT_THREADS, sizeof(T) == 4 || G > 1 ? 2 : 3) void paged_split_fp4_kernel(Fp4AttnArgs a) {
  using C = Split4<HD, G>;
  constexpr int NQ = Terms<T>::Q, NW = Terms<T>::W;
  typedef typename Words<C::NW>::type words;
  __shared__ __align__(16) char lds[C::LDS];
  __shared__ int s_flag[SPLIT_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = lane & 15, quad = lane >> 4;
  // Rows of neighbouring heads lie in the same lines of the caches, and of these there are as many as XCDs: workgroups go round the XCDs in turn, and `side`
  // workgroups with neighbouring heads of a part follow each other on one.
  auto unit_of = [](int side) { return (int)(blockIdx.x / (8 * side) * 8 + blockIdx.x % 8); };
  const int kvhs = a.kv_heads, narrow = unit_of(a.side), wide = unit_of(a.wide_side), units = kvhs / a.side, wide_units = kvhs / (SPLIT_WAVES * a.wide_side);
  Item it;
  if (!find_item_fp4<C::ROWS>(a, narrow / units, a.wide_want ? wide / wide_units : 0, false, lane, it)) return;
  // which head, and of the part's steps the wave's
  const int kvh0 = it.wide ? (wide % wide_units * a.wide_side + blockIdx.x / 8 % a.wide_side) * SPLIT_WAVES : narrow % units * a.side + blockIdx.x / 8 % a.side;
  const int kvh = it.wide ? kvh0 + wave : kvh0, sub = it.wide ? 0 : wave, each = it.wide ? 1 : SPLIT_WAVES;
  const int all_rows = it.n * a.group;
  int pos[G], from[G];                                                        // what the lane's rows see ends there, and begins
  u32x4 q[G][C::NW][NQ];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int r = it.tile * C::ROWS + 16 * g + row, rc = min(r, all_rows - 1), tok = rc / a.group, head = kvh * a.group + rc % a.group;
    pos[g] = r < all_rows ? it.pos0 + tok : -1;
    from[g] = first_seen(pos[g], a.window);
    const T* const p = (const T*)a.q + (int64_t)(it.rows0 + tok) * a.q_tok + (int64_t)head * a.q_head + quad * (HD / 4);
#pragma unroll
    for (int i = 0; i < C::NW; ++i) query_terms(p + 8 * i, a.to_log2, q[g][i]);
  }
  const int tok_first = it.tile * C::ROWS / a.group, tok_last = min((it.tile * C::ROWS + C::ROWS - 1) / a.group, it.n - 1);
  const int all_see_to = it.pos0 + tok_first, all_see_from = first_seen(it.pos0 + tok_last, a.window);
  const float to_log2 = sizeof(T) == 4 ? 1.0f : a.to_log2;                    // (fp32 queries have it already: the largest score's weight is 1 to the bit then)
  char* const mine = lds + wave * C::WAVE_LDS;
  const char* const kbase = (const char*)a.kc + (int64_t)kvh * a.kc_head;
  const char* const vbase = (const char*)a.vc + (int64_t)kvh * a.vc_head;
  const uint8_t* const ksbase = (const uint8_t*)a.ks + (int64_t)kvh * a.ks_head;
  const uint8_t* const vsbase = (const uint8_t*)a.vs + (int64_t)kvh * a.vs_head;
  const int all_steps = (it.hi - it.lo + C::BP - 1) / C::BP, steps = max(all_steps - sub + each - 1, 0) / each;      // of all waves, of this one
  const int32_t* const table = a.b.pages + (int64_t)it.s * a.b.pages_stride;
  // Where the wave's steps lie, number i of them step sub + each * i.  NEAR: a lane has 16 positions of one of 32 steps, their offsets in the four
  // tensors, and whether they have a page; all 32 are looked up together, so that nothing in the loop waits for an entry of the table
  // behind codes that are under way.  Otherwise, as in paged_split_kernel: the entry for, and the slot of, the step's position lane % 32, asked for a
  // step before it is looked at.
  int entry, slot;
  int64_t offset[4];
  uint64_t mapped16;
  auto place = [&](int i) {
    if constexpr (NEAR) {
      if (i % 32 || i >= steps) return;
      const int p = it.lo + (sub + each * (i + lane / 2)) * C::BP + 16 * (lane & 1), at = (int)((unsigned)p / (unsigned)a.b.page_size), sl = p - at * a.b.page_size;
      const int page = p < it.hi ? table[at] : -1;         // (hi is within the table)
      const bool some = (unsigned)page < (unsigned)a.b.n_pages;
      mapped16 = __ballot(some);
      // what has no page is read from where there is something, and not used
      const int64_t pg = some ? page : 0, s = some ? sl : 0;
      offset[0] = pg * a.kc_page + s * a.kc_pos; offset[1] = pg * a.vc_page + s * a.vc_pos;
      offset[2] = pg * a.ks_page + s * a.ks_pos; offset[3] = pg * a.vs_page + s * a.vs_pos;
    } else {
      const int p = it.lo + (sub + each * i) * C::BP + (lane & (C::BP - 1)), at = (int)((unsigned)p / (unsigned)a.b.page_size);
      slot = p - at * a.b.page_size;
      entry = table[min(at, a.b.max_pages - 1)];
    }
  };
  auto lane64 = [](int64_t v, int l) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, l));
  };
  // keys: lane (row, quad) has quarter `quad` of positions 16 t + row; values: lane has quarter lane % 4 of positions 16 t + lane / 4
  const int vrow = lane >> 2, vquad = lane & 3;
  words k[2][C::NT], v[2][C::NT];
  uint32_t ks[2][C::NT], vs[2][C::NT];
  uint32_t there[2];                                      // a bit for each of a step's positions that has a page
  auto request = [&](int i, auto set) {
    constexpr int S = decltype(set)::value;
    const int base = it.lo + (sub + each * i) * C::BP;
    if constexpr (NEAR) {
      there[S] = base + C::BP <= it.hi ? ~0u : (1u << (it.hi - base)) - 1;
#pragma unroll
      for (int t = 0; t < C::NT; ++t) {
        const int l = 2 * (i % 32) + t;
        if (!(mapped16 >> l & 1)) there[S] &= ~(0xffffu << 16 * t);
        k[S][t] = *(const words*)(kbase + lane64(offset[0], l) + (unsigned)(row * (int)a.kc_pos + quad * C::LANE));
        v[S][t] = *(const words*)(vbase + lane64(offset[1], l) + (unsigned)(vrow * (int)a.vc_pos + vquad * C::LANE));
        ks[S][t] = (ksbase + lane64(offset[2], l))[(unsigned)(row * (int)a.ks_pos + quad * (HD / 4) / FP4_BLOCK)];
        vs[S][t] = (vsbase + lane64(offset[3], l))[(unsigned)(vrow * (int)a.vs_pos + vquad * (HD / 4) / FP4_BLOCK)];
      }
    } else {
      const int page = base + (lane & (C::BP - 1)) < it.hi && (unsigned)entry < (unsigned)a.b.n_pages ? entry : -1;      // (hi is within the table)
      there[S] = (uint32_t)__ballot(page >= 0);
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
  f32x4 o[G][HD / 16];
  float m[G], l[G];                                       // a row's reference (its maximum of scores times to_log2; the same in its four lanes) and the lane's part of the sum
  uint32_t nans[G];                                       // blocks of 32 components with a value that is NaN and seen
  auto work = [&](int i, auto set) {
    constexpr int S = decltype(set)::value;
    const int base = it.lo + (sub + each * i) * C::BP;
    const uint32_t have = there[S];
    const bool whole = have == ~0u && base + C::BP - 1 <= all_see_to && base >= all_see_from;
    f32x4 s[G][C::NT];
#pragma unroll
    for (int t = 0; t < C::NT; ++t) {
#pragma unroll
      for (int g = 0; g < G; ++g) s[g][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
      const float scale = fp4_scale(ks[S][t]);
#pragma unroll
      for (int i = 0; i < C::NW; ++i) {
        const u32x4 w = fp4_wide(k[S][t][i], scale);
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int n = 0; n < NQ; ++n) s[g][t] = mma16(w, q[g][i][n], s[g][t], bf16_t());
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
    u32x4 w[G][NW];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (!whole) {
        asm volatile("");                                 // (a branch, not selections that every step goes through)
        const int to = pos[g] - base - 4 * quad, since = from[g] - base - 4 * quad;
        const uint32_t mapped = have >> (4 * quad);
#pragma unroll
        for (int t = 0; t < C::NT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool seen = ((mapped >> (16 * t + e) & 1) != 0) & (16 * t + e <= to) & (16 * t + e >= since);
            s[g][t][e] = seen ? s[g][t][e] : -INFINITY;
          }
      }
      // running maximum: joined and sums rescaled only where it grows for some row
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < C::NT; ++t) top = fmaxf(top, fmaxf(fmaxf(s[g][t].x, s[g][t].y), fmaxf(s[g][t].z, s[g][t].w)));
      top *= to_log2;
      if (__ballot(top > m[g])) {
        top = fmaxf(top, __shfl_xor(top, 16, WAVE));
        top = fmaxf(top, __shfl_xor(top, 32, WAVE));
        const float mn = fmaxf(m[g], top), keep = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[g] - mn);
        m[g] = mn;
        l[g] *= keep;
#pragma unroll
        for (int i = 0; i < HD / 16; ++i) o[g][i] *= keep;
      }
      const float ref = m[g] == -INFINITY ? 0.f : m[g];
      float total = 0.f;                                  // (a step's weights among themselves first: one by one, those below half a step of the row's sum would leave no trace in it)
#pragma unroll
      for (int t = 0; t < C::NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) { s[g][t][e] = __builtin_amdgcn_exp2f(fmaf(s[g][t][e], to_log2, -ref)); total += s[g][t][e]; }
      l[g] += total;
#pragma unroll
      for (int n = 0; n < NW; ++n)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            uint32_t p = pair(s[g][t][e], s[g][t][e + 1], bf16_t());
            asm("" : "+v"(p));                            // (or each pair is rounded twice, once for what is taken off)
            w[g][n][2 * t + e / 2] = p;
            if (n + 1 < NW) { float x = s[g][t][e], y = s[g][t][e + 1]; rest(p, x, y, bf16_t()); s[g][t][e] = x; s[g][t][e + 1] = y; }
          }
    }
    const char* src = mine + (4 * quad + (row >> 2)) * C::STRIDE + (row & 3) * 8;
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) {
      const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(src + i * 32));
      const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(src + 16 * C::STRIDE + i * 32));
      const u32x2 xu = __builtin_bit_cast(u32x2, x), yu = __builtin_bit_cast(u32x2, y);
      const u32x4 vt = {xu.x, xu.y, yu.x, yu.y};
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int n = 0; n < NW; ++n) o[g][i] = mma16(vt, w[g][n], o[g][i], bf16_t());
    }
    if (nan[0] | nan[1])
#pragma unroll
      for (int t = 0; t < C::NT; ++t)
        for (uint64_t bits = nan[t]; bits; bits &= bits - 1) {      // (by position and quarter of the row)
          const int at = __builtin_ctzll(bits), p = 16 * t + at / 4;
#pragma unroll
          for (int g = 0; g < G; ++g)
            if (((have >> p) & 1) && base + p <= pos[g] && base + p >= from[g]) nans[g] |= 1u << at % 4 * (HD / 4) / FP4_BLOCK;
        }
  };
#pragma unroll
  for (int g = 0; g < G; ++g) {
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) o[g][i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    m[g] = -INFINITY; l[g] = 0.f; nans[g] = 0;
  }
  const std::integral_constant<int, 0> even;
  const std::integral_constant<int, 1> uneven;
  // The next step is asked for whether there is one or not (the last one again then): behind a request that may or may not have been made, the
  // compiler waits for all that is under way.
  if (steps > 0) {
    place(0);
    request(0, even);
    place(1);
    for (int i = 0; i < steps; i += 2) {
      if (it.wide) __builtin_amdgcn_s_barrier();
      request(min(i + 1, steps - 1), uneven);
      place(i + 2);
      work(i, even);
      if (i + 1 >= steps) break;
      if (it.wide) __builtin_amdgcn_s_barrier();
      request(min(i + 2, steps - 1), even);
      place(i + 3);
      work(i + 1, uneven);
    }
  }
#pragma unroll
  for (int g = 0; g < G; ++g) {
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) if (nans[g] >> i / 2 & 1) o[g][i] = (f32x4){__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
    l[g] += __shfl_xor(l[g], 16, WAVE);
    l[g] += __shfl_xor(l[g], 32, WAVE);
  }
  // ---- the waves' results
  __syncthreads();
  float* const so = (float*)(lds + wave * C::OUT_LDS);
#pragma unroll
  for (int g = 0; g < G; ++g) {
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) *(f32x4*)(so + (16 * g + row) * (HD + 4) + 16 * i + 4 * quad) = o[g][i];
    if (quad == 0) ((float2*)(so + C::ROWS * (HD + 4)))[16 * g + row] = make_float2(m[g], l[g]);
  }
  __syncthreads();
  if (it.wide) {
    join_waves<T, HD, true, C::ROWS>(a, it, kvh0, tid, lds, C::OUT_LDS);
    if (it.parts > 1) join_parts<T, HD, true, C::ROWS>(a, it, kvh0, tid, s_flag);
  } else {
    join_waves<T, HD, false, C::ROWS>(a, it, kvh, tid, lds, C::OUT_LDS);
    if (it.parts > 1) join_parts<T, HD, false, C::ROWS>(a, it, kvh, tid, s_flag);
  }
}

// ---- host
struct AttnPlan {
  bool tiles;               // paged_tile_fp4_kernel, not paged_split_fp4_kernel
  int tile_rows;
  int want, fine, least, whole, wide_want;      // see PagedAttnArgs
  float wide_from;
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
  // Which kernel: paged_tile_fp4_kernel for 16-bit types and more than 64 rows a sequence, where there is work for many workgroups: the split kernel reads
  // and widens keys and values anew for every tile, but cuts what there is into more parts.  bf16, 32 / 8 heads, us of the split kernel (the better one) / the
  // tile kernel: 64 sequences of 64 rows over 4000 positions 168 / 174, of 80 253 / 193, of 96 265 / 192; 24 over 2000 of 64 43 / 56, of 80 58 / 60, of 96 65 / 61;
  // one of 128 over 8000 27.2 / 32.5, of 256 over 500 12.7 / 19.1, over 2000 19.3 / 25.5, over 8000 42.7 / 34.8.
  p->tiles = cache->dtype != PPD_FP32 && rows > 64 * (int64_t)batch->n_seqs && (double)rows * cache->n_kv_heads * (double)capacity >= 12e6;
  // The split kernel's tiles of 32 rows where there are many and most of them are full, as far as the host can know, or where there is more to read than the memory-side cache
  // holds.  16-bit types, 32 / 8 heads, us of 16 / 32 rows a tile: 64 sequences of 20 rows over 4000 positions 120 / 77, over 8000 243 / 194; of 32 rows over
  // 1000 37 / 30, 24 of them over 2000 33 / 32, 4 over 500 11.4 / 14.4, one over 8000 20 / 32; of 48 rows over 1000 47 / 52, over 400 to 32000 465 / 309; of 64 rows over 1000
  // 60 / 53, over 4000 212 / 182.  Where sequences have from 4 to 32 rows, 17 of them on average, over 100 to 4000 81 / 86, over 400 to 32000 178 / 203.
  const int64_t wide_tiles = (rows / (2 * SPLIT_ROWS) + some) * cache->n_kv_heads, sixteens = some ? (rows + SPLIT_ROWS * some - 1) / (SPLIT_ROWS * some) : 0;
  const bool full = sixteens % 2 == 0 && 2 * (rows - (sixteens - 1) * SPLIT_ROWS * some) > SPLIT_ROWS * some;
  const bool much = (double)some * (double)capacity * cache->n_kv_heads * (cache->head_dim + cache->head_dim / 16) >= 320e6;
  p->tile_rows = p->tiles ? TILE_ROWS : cache->dtype != PPD_FP32 && rows >= 20 * some && sixteens <= 4 && wide_tiles >= 256 && (full || much) ? 2 * SPLIT_ROWS : SPLIT_ROWS;
  const int tile_rows = p->tile_rows;
  const int64_t tiles = rows / tile_rows + some;
  const int slots = p->tiles ? 512 : 256;                   // (see ppd_paged_attn.hip; 512 for few rows: one sequence of 60000 positions 30.6 us, not 28.3, 8 of 4 rows over 2000 18 / 15)
  p->want = slots / cache->n_kv_heads + (slots < cache->n_kv_heads);
  p->fine = p->tiles || tiles * cache->n_kv_heads < 160 ? p->want : p->want * 7 / 4;
  p->whole = p->tiles ? 8 : 4;
  p->least = p->tiles ? 8 : 2;
  // Tiles enough for the whole chip, or no position to cut at: one part each.  Long runs: from one and a half for every place on, counted as if sequences were
  // alike (us whole / in parts: 96 sequences of 32 tokens over 1500 positions 127 / 138, four prompts of 1000 76 / 81; fewer, where lengths differ, should be cut: 40 of 1
  // to 100 tokens over 100 to 6000 175 / 96).
  const int64_t likely = some ? (rows + some * TILE_ROWS - 1) / (some * TILE_ROWS) * some : 0;
  if ((p->tiles ? 2 * likely >= 3 * p->want : tiles >= 8 * p->want) || capacity <= p->whole * PLAN_BLOCK) p->least = 0;
  // Wide workgroups, four heads side by side, where there is more to read than the memory-side cache holds (320 MB): there the number of requests counts, and
  // waves with neighbouring heads' halves of the same lines at the same time ask for them once.  us of one head a workgroup / wide: 64 sequences of
  // 8000 positions, 8 heads 143 / 128, of 16000 273 / 246, 16 of 8000, 32 heads 187 / 131; of less, 64 of 4000 63 / 66, 64 of 60 to 8000 33 / 44.
  p->wide_from = 320 * 1e6f / (2.f * PLAN_BLOCK * cache->n_kv_heads * (cache->head_dim / 2 + cache->head_dim / FP4_BLOCK));
  p->wide_want = !p->tiles && p->least && cache->n_kv_heads % SPLIT_WAVES == 0 && (float)tiles * (float)((capacity + PLAN_BLOCK - 1) / PLAN_BLOCK) >= p->wide_from
                     ? (2048 + cache->n_kv_heads - 1) / cache->n_kv_heads : 0;
  p->items = tiles + (p->least ? (p->fine > p->wide_want ? p->fine : p->wide_want) + 1 : 0);
  // (a launch has fewer than 2^32 threads, 256 to a workgroup; workgroups are rounded up to eight rounds of up to eight heads, see attn_go)
  if (p->items * cache->n_kv_heads >= ((int64_t)1 << 24) - 64) return PPD_ELIMIT;
  const uint64_t places = p->least ? (uint64_t)p->items * cache->n_kv_heads : 0;
  p->o_bytes = places * tile_rows * cache->head_dim * 4;
  p->ml_bytes = places * tile_rows * 8;
  p->more_bytes = !p->least ? 0 : p->tiles ? (uint64_t)batch->n_seqs * 8 : places * 8;
  return PPD_OK;
}

template <typename T, int HD, int G>
void split_go(const Fp4AttnArgs& a, dim3 grid, hipStream_t stream) {
  if (near_pages_fp4(a)) hipLaunchKernelGGL((paged_split_fp4_kernel<T, HD, true, G>), grid, dim3(SPLIT_THREADS), 0, stream, a);
  else hipLaunchKernelGGL((paged_split_fp4_kernel<T, HD, false, G>), grid, dim3(SPLIT_THREADS), 0, stream, a);
}
template <typename T, int HD>
hipError_t attn_go(const Fp4AttnArgs& a, int dtype, hipStream_t stream) {
  if (a.tile_rows == TILE_ROWS) return launch_paged_tiles_fp4(a, dtype, HD, stream);
  const int units = (a.items * (a.kv_heads / a.side) + 7) / 8 * 8 * a.side, wide = a.wide_want ? (a.items * (a.kv_heads / (SPLIT_WAVES * a.wide_side)) + 7) / 8 * 8 * a.wide_side : 0;
  const dim3 grid(units > wide ? units : wide);
  if (sizeof(T) == 2 && a.tile_rows > SPLIT_ROWS) split_go<T, HD, sizeof(T) == 2 ? 2 : 1>(a, grid, stream);
  else split_go<T, HD, 1>(a, grid, stream);
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
  a.tile_rows = p.tile_rows; a.items = (int)p.items; a.want = p.want; a.fine = p.fine; a.least = p.least; a.whole = p.whole;
  a.part_o = (float*)workspace; a.part_ml = (float2*)((char*)workspace + p.o_bytes); a.stamps = (uint64_t*)((char*)workspace + p.o_bytes + p.ml_bytes);
  a.plan = (int2*)a.stamps;
  a.wide_want = p.wide_want; a.wide_from = p.wide_from;
  a.side = a.wide_side = 1;
  while (a.side < 8 && a.kv_heads % (2 * a.side) == 0) a.side *= 2;
  while (a.wide_side < 2 && a.kv_heads % (2 * SPLIT_WAVES * a.wide_side) == 0) a.wide_side *= 2;
  a.stamp = next_stamp();
  hipStream_t st = (hipStream_t)hip_stream;
  if (cache->head_dim == 64)
    return launched(dt == PPD_FP32 ? attn_go<float, 64>(a, dt, st) : dt == PPD_BF16 ? attn_go<bf16_t, 64>(a, dt, st) : attn_go<f16_t, 64>(a, dt, st));
  return launched(dt == PPD_FP32 ? attn_go<float, 128>(a, dt, st) : dt == PPD_BF16 ? attn_go<bf16_t, 128>(a, dt, st) : attn_go<f16_t, 128>(a, dt, st));
}
