// ppd_paged_attention: attention of ragged runs of new tokens over paged keys and values.  Few rows over many positions,
// and the host's side; many rows: ppd_paged_tiles.hip.
#include "ppd_paged_attn.h"

#include <math.h>

#include <atomic>

using namespace ppd;

namespace {

constexpr int SPLIT_WAVES = 4, SPLIT_THREADS = SPLIT_WAVES * WAVE;

// A part's results: sums of a row's components, and its reference and total, past the L2, for whoever joins them.
__device__ __forceinline__ void leave(float* to, f32x4 v) {
  typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
  const u64x2 u = __builtin_bit_cast(u64x2, v);
  __hip_atomic_store((uint64_t*)to, u.x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __hip_atomic_store((uint64_t*)to + 1, u.y, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void leave(float2* to, float m, float l) {
  const f32x2 v = {m, l};
  __hip_atomic_store((uint64_t*)to, __builtin_bit_cast(uint64_t, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 left(const void* from) {
  return __builtin_bit_cast(f32x2, __hip_atomic_load((const uint64_t*)from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
// The end of a workgroup that had one of several parts (all of its threads, its results left): it puts the call's number beside them and
// looks at the other parts' places; who finds the number everywhere joins them, in their order, and clears the places.  Nobody waits.
// The number goes out, past the L2, before the others are looked at, so the last one to leave it finds all; two may, and write the
// same bits.  Scratch memory needs nothing in it beforehand (numbers are 64 bits wide and never come twice, but for a replayed
// launch's, and that one's own places are clear again by then).
template <typename T, int HD>
__device__ __forceinline__ void join_parts(const PagedAttnArgs& a, const Item& it, int kvh, int tid, int* s_flag) {
  const int lane = tid & 63;
  const int first = it.slot - it.part;                    // (the parts' places lie side by side)
  uint64_t* const stamps = a.stamps + (int64_t)first * a.kv_heads + kvh;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid < WAVE) {
    if (lane == 0) __hip_atomic_store(stamps + (int64_t)it.part * a.kv_heads, a.stamp, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    bool missing = false;
    for (int p = lane; p < it.parts; p += WAVE) missing |= __hip_atomic_load(stamps + (int64_t)p * a.kv_heads, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != a.stamp;
    missing = __ballot(missing) != 0;
    if (lane == 0) *s_flag = !missing;
  }
  __syncthreads();
  if (!*s_flag) return;
  const int rows = min(SPLIT_ROWS, it.n * a.group - it.tile * SPLIT_ROWS);
  for (int x = tid; x < rows * (HD / 4); x += SPLIT_THREADS) {
    const int rr = x / (HD / 4), d = x % (HD / 4) * 4, ri = it.tile * SPLIT_ROWS + rr;
    auto at = [&](int p) { return ((int64_t)(first + p) * a.kv_heads + kvh) * SPLIT_ROWS + rr; };
    float mx = -INFINITY, sum = 0.f;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < it.parts; p0 += 4) {            // four parts at a time, their sums and totals in one go
      f32x2 ml[4], u[4], w[4];
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const int64_t from = at(min(p0 + p, it.parts - 1));
        ml[p] = left(a.part_ml + from); u[p] = left(a.part_o + from * HD + d); w[p] = left(a.part_o + from * HD + d + 2);
      }
      const float before = mx;
#pragma unroll
      for (int p = 0; p < 4; ++p) mx = fmaxf(mx, ml[p].x);
      const float ref = mx == -INFINITY ? 0.f : mx, keep = __builtin_amdgcn_exp2f(before - ref);
      if (p0 > 0) {
        sum *= keep;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] *= keep;
      }
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        if (p0 + p >= it.parts) break;
        const float f = __builtin_amdgcn_exp2f(ml[p].x - ref);
        sum = fmaf(f, ml[p].y, sum);
        y.x = fmaf(f, u[p].x, y.x); y.y = fmaf(f, u[p].y, y.y); y.z = fmaf(f, w[p].x, y.z); y.w = fmaf(f, w[p].y, y.w);
      }
    }
    const bool none = mx == -INFINITY && sum == 0.f;      // nothing seen (a score that is no number leaves its mark on the sum)
    const float inv = 1.0f / sum;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = none ? 0.f : y[e] * inv;
    const int t = ri / a.group, h = kvh * a.group + ri % a.group;
    *(typename Quad<T>::raw*)((T*)a.out + (int64_t)(it.rows0 + t) * a.o_tok + (int64_t)h * a.o_head + d) = quad_out<T>(y);
    if (a.lse && d == 0) a.lse[(int64_t)(it.rows0 + t) * a.heads + h] = none ? -INFINITY : (mx + __builtin_amdgcn_logf(sum)) * 0.69314718f;
  }
  for (int p = tid; p < it.parts; p += SPLIT_THREADS) __hip_atomic_store(stamps + (int64_t)p * a.kv_heads, (uint64_t)0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// ---- few rows, many positions: bound by the stream of keys and values, and, where these are few, by the chain of latencies (lengths, page
// numbers, keys and values, the join).  64 bf16 tokens over 60 to 8000 positions each (411 MB) take 90 us: 4.6 TB/s, and with the products
// taken out no less; 64 of 4000 (1 GB) 197, 5.3 TB/s; a large copy reaches 4.6, a plain stream of reads 7.1.  Long runs of fp32 come here, too: four
// prompts of 3000, 8 heads, 926 us, 80 of the 154 TFLOP/s that a large fp32 product reaches (32 rows a wave, for half the reads: 997, one wave on a
// SIMD instead of two).  One token over 700 positions: 11 us, of
// which 1.5 for the plan, 1 for the waves' results and 3 for the join.
// A wave has every fourth step of BP positions of its part to itself: keys straight into registers as the left operand, values through
// registers into LDS rows of its own, from where the transposing reads (fp32: plain ones) make them the left operand of the second product.
// The next step's are under way, in registers of their own, while one is worked on; nothing waits at a barrier until the waves' results are
// joined.
template <typename T, int HD>
struct Split {
  static constexpr int SZ = sizeof(T) == 4 ? 4 : 2, BP = SZ == 4 ? 16 : 32, NT = BP / 16;
  static constexpr int NK = HD * SZ / 64;                 // 16-byte pieces of a key per lane
  static constexpr int LPR = HD * SZ / 16, RPI = WAVE / LPR, NV = BP / RPI;
  static constexpr int STRIDE = HD * SZ + (SZ == 4 ? 16 : 32);   // of a row of values in LDS: no two rows of an operand on the same banks
  static constexpr int WAVE_LDS = BP * STRIDE;
  static constexpr int OUT_LDS = SPLIT_ROWS * (HD + 4) * 4 + SPLIT_ROWS * 8; // a wave's results: sums (rows 16 bytes longer than they are), references and totals
  static constexpr int LDS = SPLIT_WAVES * (WAVE_LDS > OUT_LDS ? WAVE_LDS : OUT_LDS);
};

// NEAR: 16 positions in a row that begin at a multiple of 16 lie in one page, within 2^31 bytes: addresses are the page's, one for the wave,
// and 32-bit offsets (one bf16 token over 700 positions 11.9 us, not 12.3; fp32 drafts 12.9, not 13.5).
template <typename T, int HD, bool NEAR>
__global__ __launch_bounds__(SPLIT_THREADS, 2) void paged_split_kernel(PagedAttnArgs a) {
  using C = Split<T, HD>;
  __shared__ __align__(16) char lds[C::LDS];
  __shared__ int s_flag;
  // the heads of one part side by side: a position's keys are one run of memory, and its pieces then come at the same time
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), kvh = blockIdx.x % a.kv_heads, row = lane & 15, quad = lane >> 4;
  Item it;
  if (!find_item<SPLIT_ROWS>(a, blockIdx.x / a.kv_heads, false, lane, it)) return;
  const int all_rows = it.n * a.group;
  const int r = it.tile * SPLIT_ROWS + row, rc = min(r, all_rows - 1), tok = rc / a.group, head = kvh * a.group + rc % a.group;
  const int pos = r < all_rows ? it.pos0 + tok : -1;                          // what the lane's row sees ends there
  const int from = first_seen(pos, a.window);
  const int tok_first = it.tile * SPLIT_ROWS / a.group, tok_last = min((it.tile * SPLIT_ROWS + SPLIT_ROWS - 1) / a.group, it.n - 1);
  const int all_see_to = it.pos0 + tok_first, all_see_from = first_seen(it.pos0 + tok_last, a.window);
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
  const char* const kbase = (const char*)a.kc + (int64_t)kvh * a.kc_head * C::SZ;
  const char* const vbase = (const char*)a.vc + (int64_t)kvh * a.vc_head * C::SZ;
  const int steps = (it.hi - it.lo + C::BP - 1) / C::BP;
  // The table's entry for, and the slot of, position lo + step * BP + (lane % BP): asked for here, looked at when the step is requested, a
  // whole step later (looked at here it would wait for the keys and values that are under way).
  const int32_t* const table = a.b.pages + (int64_t)it.s * a.b.pages_stride;
  int entry, slot;
  auto place = [&](int step) {
    const int p = it.lo + step * C::BP + (lane & (C::BP - 1)), i = (int)((unsigned)p / (unsigned)a.b.page_size);
    slot = p - i * a.b.page_size;
    entry = table[min(i, a.b.max_pages - 1)];
  };
  u32x4 k[2][C::NT][C::NK], v[2][C::NV];
  uint32_t there[2];                                      // a bit for each of a step's positions that has a page
  const int vrow = lane / C::LPR, vpiece = lane % C::LPR * 16;
  auto request = [&](int step, auto set) {
    constexpr int S = decltype(set)::value;
    const int page = it.lo + step * C::BP + (lane & (C::BP - 1)) < it.hi && (unsigned)entry < (unsigned)a.b.n_pages ? entry : -1;      // (hi is within the table)
    there[S] = (uint32_t)__ballot(page >= 0) & (uint32_t)((1ull << C::BP) - 1);
    // what has no page is read from where there is something, and not used
    if constexpr (NEAR) {
#pragma unroll
      for (int t = 0; t < C::NT; ++t) {
        const int pg = __builtin_amdgcn_readlane(page, 16 * t), sl = pg >= 0 ? __builtin_amdgcn_readlane(slot, 16 * t) : 0;
        const char* const kp = kbase + ((int64_t)max(pg, 0) * a.kc_page + (int64_t)sl * a.kc_pos) * C::SZ;
        const char* const vp = vbase + ((int64_t)max(pg, 0) * a.vc_page + (int64_t)sl * a.vc_pos) * C::SZ;
        const unsigned ko = (unsigned)(row * (int)a.kc_pos * C::SZ + quad * 16);
#pragma unroll
        for (int i = 0; i < C::NK; ++i) k[S][t][i] = *(const u32x4*)(kp + ko + i * 64);
        const unsigned vo = (unsigned)(vrow * (int)a.vc_pos * C::SZ + vpiece);
#pragma unroll
        for (int i = 0; i < C::NV / C::NT; ++i) v[S][t * (C::NV / C::NT) + i] = *(const u32x4*)(vp + (int64_t)i * C::RPI * a.vc_pos * C::SZ + vo);
      }
    } else {
      const int pg = max(page, 0), sl = page >= 0 ? slot : 0;
      const int64_t ko = ((int64_t)pg * a.kc_page + (int64_t)sl * a.kc_pos) * C::SZ, vo = ((int64_t)pg * a.vc_page + (int64_t)sl * a.vc_pos) * C::SZ;
#pragma unroll
      for (int t = 0; t < C::NT; ++t) {
        const char* const p = kbase + quad * 16 + __shfl(ko, 16 * t + row, WAVE);
#pragma unroll
        for (int i = 0; i < C::NK; ++i) k[S][t][i] = *(const u32x4*)(p + i * 64);
      }
#pragma unroll
      for (int i = 0; i < C::NV; ++i) v[S][i] = *(const u32x4*)(vbase + vpiece + __shfl(vo, i * C::RPI + vrow, WAVE));
    }
  };
  f32x4 o[HD / 16];
  float m, l;                                             // the row's reference (from its maximum of scores times to_log2; the same in its four lanes) and the lane's part of the sum
  // One step.  CAREFUL: with values that are infinite, or no numbers, among it (the first way through gives such a row no number where it
  // should have one: 0 times infinity where the row does not see it, or for the second term of a weight).
  auto work = [&](int step, auto set, auto careful) {
    constexpr int S = decltype(set)::value;
    constexpr bool CAREFUL = decltype(careful)::value;
    const int base = it.lo + step * C::BP;
    const uint32_t have = there[S];
    const bool whole = have == (uint32_t)((1ull << C::BP) - 1) && base + C::BP - 1 <= all_see_to && base >= all_see_from;
    f32x4 s[C::NT];
#pragma unroll
    for (int t = 0; t < C::NT; ++t) {
      s[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < C::NK; ++i) {
        if constexpr (C::SZ == 2) s[t] = mma16(k[S][t][i], q[i], s[t], T());
        else
#pragma unroll
          for (int e = 0; e < 4; ++e) s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[S][t][i][e]), __uint_as_float(q[i][e]), s[t], 0, 0, 0);
      }
    }
    if (!whole) {
      asm volatile("");                                   // (a branch, not selections that every step goes through)
#pragma unroll
      for (int i = 0; i < C::NV; ++i) if (!((have >> (i * C::RPI + vrow)) & 1)) v[S][i] = (u32x4){0u, 0u, 0u, 0u};
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
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < C::NV; ++i) {
      if (CAREFUL) most = largest(most, v[S][i], T());
      *(u32x4*)(mine + (i * C::RPI + vrow) * C::STRIDE + vpiece) = v[S][i];
    }
    const bool odd = CAREFUL && __ballot(endless(most, T())) != 0;
    // running maximum: joined and sums rescaled only where it grows for some row
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < C::NT; ++t) top = fmaxf(top, fmaxf(fmaxf(s[t].x, s[t].y), fmaxf(s[t].z, s[t].w)));
    top = reference<T>(top * to_log2, 0);
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
    if constexpr (C::SZ == 2) {
      // Weights in two terms of the type: the rounding of one alone is as large as the output's own.  Beside infinite values one: what is left
      // of a weight may be zero or negative, and so that no weight above zero becomes one, half floats go no lower than their smallest number.
      if (CAREFUL && std::is_same<T, f16_t>::value && odd)
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
        if (CAREFUL && odd) {
          // position by position, kept where it is seen
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
          if (CAREFUL && odd) {
            for (int c = 0; c < 4; ++c) {
              const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x4f32(c == quad ? x : 0.f, s[0][e], o[i], 0, 0, 0);
              const int p = 4 * c + e;
              if (((have >> p) & 1) && base + p <= pos && base + p >= from) o[i] = n;
            }
          } else o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, s[0][e], o[i], 0, 0, 0);
        }
    }
  };
  auto begin = [&]() {
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) o[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    m = -INFINITY; l = 0.f;
  };
  const std::integral_constant<int, 0> even;
  const std::integral_constant<int, 1> uneven;
  begin();
  place(wave);
  if (wave < steps) request(wave, even);
  place(wave + SPLIT_WAVES);
  for (int step = wave; step < steps; step += 2 * SPLIT_WAVES) {
    const int next = step + SPLIT_WAVES, after = next + SPLIT_WAVES;
    if (next < steps) request(next, uneven);
    place(after);
    work(step, even, std::false_type());
    if (next >= steps) break;
    if (after < steps) request(after, even);
    place(after + SPLIT_WAVES);
    work(next, uneven, std::false_type());
  }
  {
    float sum = l;                                        // (no number, if one is)
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) sum += (o[i].x - o[i].x) + (o[i].y - o[i].y) + (o[i].z - o[i].z) + (o[i].w - o[i].w);
    if (__ballot(!(fabsf(sum) < INFINITY))) {
      begin();
#pragma unroll 1
      for (int step = wave; step < steps; step += SPLIT_WAVES) { place(step); request(step, even); work(step, even, std::true_type()); }
    }
  }
  l += __shfl_xor(l, 16, WAVE);
  l += __shfl_xor(l, 32, WAVE);
  // ---- the waves' results
  __syncthreads();
  float* const so = (float*)(lds + wave * C::OUT_LDS);
#pragma unroll
  for (int i = 0; i < HD / 16; ++i) *(f32x4*)(so + row * (HD + 4) + 16 * i + 4 * quad) = o[i];
  if (quad == 0) ((float2*)(so + SPLIT_ROWS * (HD + 4)))[row] = make_float2(m, l);
  __syncthreads();
  for (int x = tid; x < SPLIT_ROWS * HD / 4; x += SPLIT_THREADS) {
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
      leave(a.part_o + at * HD + d, y);
      if (d == 0) leave(a.part_ml + at, mx, sum);
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
  if (it.parts > 1) join_parts<T, HD>(a, it, kvh, tid, &s_flag);
}

// ---- host
struct AttnPlan {
  bool tiles;               // paged_tile_kernel, not paged_split_kernel
  int want, fine, least, whole;      // see PagedAttnArgs
  int64_t items;            // workgroups per key/value head: parts aimed at, and a part's end for every tile
  uint64_t o_bytes, ml_bytes, more_bytes;      // more: stamps, or the plan
};

int check_attention(const ppd_paged_cache* cache, const ppd_paged_batch* batch, int n_heads, AttnPlan* p) {
  const int rc = check_paged(cache, batch);
  if (rc) return rc;
  if (n_heads < 1 || n_heads % cache->n_kv_heads) return PPD_EINVAL;
  if (n_heads > PPD_MAX_HEADS || (int64_t)batch->n_tokens * (n_heads / cache->n_kv_heads) > 1 << 26) return PPD_ELIMIT;
  const int group = n_heads / cache->n_kv_heads;
  const int64_t rows = (int64_t)batch->n_tokens * group, some = batch->n_tokens < batch->n_seqs ? batch->n_tokens : batch->n_seqs;
  const int64_t capacity = (int64_t)batch->max_pages * cache->page_size;
  // Which kernel: paged_tile_kernel for 16-bit types and more than 32 rows a sequence, where the split kernel reads keys and values a third time.
  // bf16, 8 key/value heads, us of the split / the tile kernel: 8 sequences over 2000 positions of 16 rows each 20.8 / 23.6, of 40 30.7 / 24.6; 32
  // sequences 45.3 / 49.8 and 81.5 / 56.7.  At 17 to 32 rows either may be the quicker one (32 rows: 8 sequences 24.3 / 23.7, 32 of them 53.8 / 51.7,
  // over 8000 positions 60.5 / 51.4 and 239 / 194, but over 500 13.1 / 17.6 and 20.6 / 20.2, with heads of 64 16.8 / 20.9 and 28.3 / 34.3).  The split
  // kernel, too, where rows are few in all, over no great lengths: it then has more workgroups to fill the chip with (one sequence of 128 rows over
  // 200 positions 9.2 / 13.7, over 2000 16.9 / 25.0, over 8000 34.5 / 29.0, over 20000 65 / 46).
  p->tiles = cache->dtype != PPD_FP32 && rows > 32 * (int64_t)batch->n_seqs && (rows * cache->n_kv_heads > 1024 || capacity > 8192);
  const int tile_rows = p->tiles ? TILE_ROWS : SPLIT_ROWS;
  const int64_t tiles = rows / tile_rows + some;
  const int slots = p->tiles ? 512 : 256;
  p->want = slots / cache->n_kv_heads + (slots < cache->n_kv_heads);
  p->fine = p->tiles || tiles * cache->n_kv_heads < 160 ? p->want : p->want * 7 / 4;
  p->whole = p->tiles ? 8 : 4;
  p->least = p->tiles ? 8 : 2;
  // (slots, one sequence of 60000 positions, 8 key/value heads, bf16, at 256 / 512 / 1024 / 2048: 48 / 55 / 67 / 97 us; fine: find_part.
  // Long runs, at 384 / 512 / 640 / 1024: three chunks of 140 over 15000 203 / 171 / 203 / 179, a chunk of 500 over 4000 103 / 86 / 98 / 98.
  // least, at 2 / 4 / 6: one token over 700 positions 10.8 / 11.4 / 12.6, four of 500 9.3 / 10.8 / 10.8, two fp32 ones of 1000 14.2 / 17.1 / 21.0.  whole: one
  // token over 200 positions in one part / two 7.5 / 8.6, over 300 9.7 / 9.3.)
  // Tiles enough for the whole chip, or no position to cut at: one part each.  (At whole / in parts: 300 sequences of 500 positions 128 / 156, of 60 to
  // 8000 462 / 476, but 128 of these 250 / 198; long runs, two prompts of 3800 and 4000 tokens 350 / 366, six chunks of 700 over 500 105 / 114.)
  if (tiles >= (p->tiles ? 2 : 8) * p->want || capacity <= p->whole * PLAN_BLOCK) p->least = 0;
  p->items = tiles + (p->least ? p->fine + 1 : 0);
  if (p->items * cache->n_kv_heads >= (int64_t)1 << 24) return PPD_ELIMIT;      // (a launch has fewer than 2^32 threads, 256 to a workgroup)
  const uint64_t places = p->least ? (uint64_t)p->items * cache->n_kv_heads : 0;
  p->o_bytes = places * tile_rows * cache->head_dim * 4;
  p->ml_bytes = places * tile_rows * 8;
  p->more_bytes = !p->least ? 0 : p->tiles ? (uint64_t)batch->n_seqs * 8 : places * 8;
  return PPD_OK;
}

// Numbers of calls: a product with an odd constant never comes twice in 2^64 calls, and looks like nothing that memory holds by chance.
uint64_t next_stamp() {
  static std::atomic<uint64_t> calls{0};
  return (calls.fetch_add(1, std::memory_order_relaxed) + 1) * 0x9e3779b97f4a7c15ull;
}

template <typename T, int HD>
hipError_t attn_go(const PagedAttnArgs& a, int dtype, hipStream_t stream) {
  if (a.tile_rows == TILE_ROWS) return launch_paged_tiles(a, dtype, HD, stream);
  if (near_pages(a)) hipLaunchKernelGGL((paged_split_kernel<T, HD, true>), dim3(a.items * a.kv_heads), dim3(SPLIT_THREADS), 0, stream, a);
  else hipLaunchKernelGGL((paged_split_kernel<T, HD, false>), dim3(a.items * a.kv_heads), dim3(SPLIT_THREADS), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

extern "C" int ppd_paged_attention_workspace(const ppd_paged_cache* cache, const ppd_paged_batch* batch, int n_heads, uint64_t* bytes) {
  AttnPlan p;
  const int rc = check_attention(cache, batch, n_heads, &p);
  if (rc) return rc;
  if (!bytes) return PPD_EINVAL;
  *bytes = p.o_bytes + p.ml_bytes + p.more_bytes;
  return PPD_OK;
}

extern "C" int ppd_paged_attention(const ppd_paged_cache* cache, const ppd_paged_batch* batch, int n_heads, const ppd_rows* q,
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
  PagedAttnArgs a;
  a.b = batch_of(*cache, *batch);
  a.q = q->p; a.out = out->p; a.lse = lse; a.kc = cache->k; a.vc = cache->v;
  a.q_tok = q->token; a.q_head = q->head; a.o_tok = out->token; a.o_head = out->head;
  a.kc_page = cache->k_page; a.kc_pos = cache->k_pos; a.kc_head = cache->k_head; a.vc_page = cache->v_page; a.vc_pos = cache->v_pos; a.vc_head = cache->v_head;
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
