// ppd_paged_attention_fp4, many rows: paged_tile_kernel's products on blocks of 64 positions that the workgroup widens to bf16 numbers in LDS.
#include "ppd_paged_attn_fp4.h"

namespace ppd {
namespace {

// Four waves of 32 rows each, see paged_tile_kernel: the same operands, orders and exchanged places in LDS.  Codes and scales of the block after the
// next are under way in registers (a thread has a quarter of a row of keys and one of values), and the next block's are widened into the other
// LDS buffer beside this one's products: one barrier a block.  Bound as paged_tile_kernel is, by the products and the vector instructions beside them, which are
// issued in turns (46 and 51 % of the cycles): two bf16 prompts of 3937 and 4013 tokens, 32 / 8 heads, take 366 us, 1050 TFLOP/s with the second
// terms of the weights, 700 without; a chunk of 500 fp16 rows over 4000 positions, 40 heads, 96 with the join of its parts.  Half of what is written to LDS meets
// another lane's on the same banks; without that (lanes' words in another order) it was no faster.
template <typename T, int HD, bool NEAR>
__global__ __launch_bounds__(256, 2) void paged_tile_fp4_kernel(Fp4AttnArgs a) {
  constexpr int KV = PLAN_BLOCK, ROWB = HD * 2, SIDE = KV * ROWB, NQ = Terms<T>::Q;
  constexpr int LANE = HD / 8, NC = LANE / 4;              // bytes of codes of a thread, and words of eight
  typedef typename std::conditional<HD == 128, u32x4, u32x2>::type words;
  __shared__ __align__(1024) char lds[4 * SIDE];           // [2 buffers][keys, values][64 positions][head_dim]
  __shared__ __align__(16) uint64_t s_nan[2][4];                         // values that are NaN: by wave, a bit for each of its positions and quarters of the row
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
  const int kvheads = a.kv_heads, idx = blockIdx.x / kvheads, kvh = blockIdx.x % kvheads;
  Item it;
  if (!find_item_fp4<TILE_ROWS>(a, idx, 0, idx == 0 && kvh == 0 && wave == 0 && a.least > 0, lane, it)) return;
  const int all_rows = it.n * a.group;
  const int r0 = it.tile * TILE_ROWS + 32 * wave, r = r0 + col, rc = min(r, all_rows - 1), tok = rc / a.group, head = kvh * a.group + rc % a.group;
  const int pos = r < all_rows ? it.pos0 + tok : -1, from = first_seen(pos, a.window);
  const bool busy = r0 < all_rows;
  const int wave_first = it.pos0 + min(r0, all_rows - 1) / a.group, wave_last = it.pos0 + min(r0 + 31, all_rows - 1) / a.group;    // positions of the wave's rows
  const int wave_from = first_seen(wave_first, a.window), wave_all = first_seen(wave_last, a.window);                              // from where some row of the wave sees, all of its
  u32x4 q[HD / 16][NQ];
  {
    const T* const p = (const T*)a.q + (int64_t)(it.rows0 + tok) * a.q_tok + (int64_t)head * a.q_head + half * 8;
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) query_terms(p + 16 * i, 1.0f, q[i]);
  }
  const int blocks = (it.hi - it.lo + KV - 1) / KV;
  // see paged_tile_kernel
  const int32_t* const table = a.b.pages + (int64_t)it.s * a.b.pages_stride;
  int index = (int)((unsigned)(it.lo + lane) / (unsigned)a.b.page_size), slot = it.lo + lane - index * a.b.page_size;
  const int more_index = KV / a.b.page_size, more_slot = KV - more_index * a.b.page_size;
  int entry = table[min(index, a.b.max_pages - 1)];
  auto place = [&]() {
    slot += more_slot;
    index += more_index;
    if (slot >= a.b.page_size) { slot -= a.b.page_size; ++index; }
    entry = table[min(index, a.b.max_pages - 1)];
  };
  const char* const kbase = (const char*)a.kc + (int64_t)kvh * a.kc_head;
  const char* const vbase = (const char*)a.vc + (int64_t)kvh * a.vc_head;
  const uint8_t* const ksbase = (const uint8_t*)a.ks + (int64_t)kvh * a.ks_head;
  const uint8_t* const vsbase = (const uint8_t*)a.vs + (int64_t)kvh * a.vs_head;
  const int trow = lane >> 2, quarter = lane & 3, scale_at = quarter * (HD / 4) / FP4_BLOCK;      // the thread's position is 16 wave + trow of a block
  words k, v;
  uint32_t ks, vs;
  uint64_t have_raw = 0;
  auto request = [&](int n) {
    const int page = it.lo + n * KV + lane < it.hi && (unsigned)entry < (unsigned)a.b.n_pages ? entry : -1;      // (hi is within the table)
    have_raw = __ballot(page >= 0);
    // what has no page is read from where there is something, and not seen; so are positions behind the part in a page of its own
    if constexpr (NEAR) {
      const int pg = __builtin_amdgcn_readlane(page, 16 * wave), sl = pg >= 0 ? __builtin_amdgcn_readlane(slot, 16 * wave) : 0;
      const int64_t at = max(pg, 0);
      k = *(const words*)(kbase + at * a.kc_page + (int64_t)sl * a.kc_pos + (unsigned)(trow * (int)a.kc_pos + quarter * LANE));
      v = *(const words*)(vbase + at * a.vc_page + (int64_t)sl * a.vc_pos + (unsigned)(trow * (int)a.vc_pos + quarter * LANE));
      ks = (ksbase + at * a.ks_page + (int64_t)sl * a.ks_pos)[(unsigned)(trow * (int)a.ks_pos + scale_at)];
      vs = (vsbase + at * a.vs_page + (int64_t)sl * a.vs_pos)[(unsigned)(trow * (int)a.vs_pos + scale_at)];
    } else {
      const int pg = max(page, 0), sl = page >= 0 ? slot : 0;
      const int64_t rp = __shfl(pg, 16 * wave + trow, WAVE), rs = __shfl(sl, 16 * wave + trow, WAVE);
      k = *(const words*)(kbase + rp * a.kc_page + rs * a.kc_pos + quarter * LANE);
      v = *(const words*)(vbase + rp * a.vc_page + rs * a.vc_pos + quarter * LANE);
      ks = ksbase[rp * a.ks_page + rs * a.ks_pos + scale_at];
      vs = vsbase[rp * a.vs_page + rs * a.vs_pos + scale_at];
    }
  };
  // Places of 16-byte pieces within a row are exchanged as in paged_tile_kernel: piece p of keys lies at p ^ row (head_dim 64: ^ row / 2), of
  // values at p ^ 2 row (^ 2 (row / 2)), rows counted modulo 16 and 8.
  const int krow = 16 * wave + trow;
  const int kswap = HD == 128 ? krow & 15 : (krow >> 1) & 7, vswap = HD == 128 ? 2 * (krow & 7) : 2 * ((krow >> 1) & 3);
  auto widen = [&](int n) {
    char* const to = lds + (n & 1) * 2 * SIDE + krow * ROWB;
    const float kscale = fp4_scale(ks), vscale = vs >= FP4_NAN ? 0.0f : __uint_as_float(vs << 23);      // (values that are NaN go in as zeros, see below)
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int piece = quarter * NC + i;
      *(u32x4*)(to + (piece ^ kswap) * 16) = fp4_wide(k[i], kscale);
      *(u32x4*)(to + SIDE + (piece ^ vswap) * 16) = fp4_wide(v[i], vscale);
    }
    const uint64_t nan = __ballot(vs >= FP4_NAN);
    if (lane == 0) s_nan[n & 1][wave] = nan;
  };
  f32x16 o[HD / 32];
#pragma unroll
  for (int i = 0; i < HD / 32; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  float m = -INFINITY, l = 0.f;
  uint32_t nans = 0;                                       // blocks of 32 components with a value that is NaN and seen
  // where a lane's operands begin, see paged_tile_kernel
  int kat = col * ROWB + (half ^ (HD == 128 ? col & 15 : (col >> 1) & 7)) * 16;
  const int vrow = 4 * half + ((lane & 15) >> 2);
  int vat = SIDE + vrow * ROWB + ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ (HD == 128 ? 2 * (vrow & 7) : 2 * ((vrow >> 1) & 3))) * 16 + 8 * (lane & 1);
  auto step = [&](int n, int base, uint64_t have, bool whole) {      // whole: every row of the wave sees every position
    const char* const buf = lds + (n & 1) * 2 * SIDE;
    asm volatile("" : "+v"(kat), "+v"(vat));
    f32x16 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
#pragma unroll
      for (int i = 0; i < HD / 16; ++i) {
        const u32x4 x = *(const u32x4*)(buf + (kat ^ 32 * i) + t * 32 * ROWB);
#pragma unroll
        for (int c = 0; c < NQ; ++c) s[t] = mma32(x, q[i][c], s[t], bf16_t());
      }
    }
    if (!whole) {
      asm volatile("");                                    // (a branch, not selections that every block goes through)
      const int to = pos - base - 4 * half, since = from - base - 4 * half;
      const uint32_t have_lo = (uint32_t)(have >> (4 * half)), have_hi = (uint32_t)(have >> (32 + 4 * half));
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int at = 8 * (e / 4) + e % 4;
          const bool seen = (((t ? have_hi : have_lo) >> at & 1) != 0) & (32 * t + at <= to) & (32 * t + at >= since);
          s[t][e] = seen ? s[t][e] : -INFINITY;
        }
    }
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 16; e += 2) top = fmaxf(fmaxf(top, s[t][e]), s[t][e + 1]);
    // the reference that weights are taken from follows the maximum only where that has left it by a factor of 2^8
    constexpr int SLACK = 8;
    top *= a.to_log2;
    if (__ballot(top > m + SLACK)) {
      top = fmaxf(top, __shfl_xor(top, 32, WAVE));
      const float mn = fmaxf(m, top), keep = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= keep;
#pragma unroll
      for (int i = 0; i < HD / 32; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] *= keep;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    // (a block's weights among themselves first: one by one, those below half a step of the row's sum would leave no trace in it)
    float total[2] = {0.f, 0.f};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[t][e] = __builtin_amdgcn_exp2f(fmaf(s[t][e], a.to_log2, -ref));
        total[t] += s[t][e];
      }
    l += total[0] + total[1];
    auto values = [&](int t, int d) {
      const char* p = buf + (vat ^ 64 * d) + t * 16 * ROWB;
      const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)p));
      const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p + 8 * ROWB)));
      return (u32x4){x.x, x.y, y.x, y.y};
    };
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      u32x4 hi, lo;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x = s[t / 2][8 * (t % 2) + 2 * e], y = s[t / 2][8 * (t % 2) + 2 * e + 1];
        hi[e] = pair(x, y, bf16_t());
        asm("" : "+v"(hi[e]));                             // (or each pair is rounded twice, once for what is taken off)
        rest(hi[e], x, y, bf16_t());
        lo[e] = pair(x, y, bf16_t());
      }
#pragma unroll
      for (int d = 0; d < HD / 32; ++d) {
        const u32x4 w = values(t, d);
        o[d] = mma32(w, hi, o[d], bf16_t());
        o[d] = mma32(w, lo, o[d], bf16_t());
      }
    }
    // a weight of zero would not have silenced a value that is NaN: it is put in, behind the loop, where it is seen
    const u32x4 n0 = *(const u32x4*)&s_nan[n & 1][0], n1 = *(const u32x4*)&s_nan[n & 1][2];
    if (__ballot((n0.x | n0.y | n0.z | n0.w | n1.x | n1.y | n1.z | n1.w) != 0))
#pragma unroll 1
      for (int w = 0; w < 4; ++w) {
        const uint64_t some = s_nan[n & 1][w];
        uint64_t bits = (uint64_t)__builtin_amdgcn_readfirstlane((int)(some >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)some);
        for (; bits; bits &= bits - 1) {
          const int at = __builtin_ctzll(bits), p = 16 * w + at / 4;
          if (((have >> p) & 1) && base + p <= pos && base + p >= from) nans |= 1u << at % 4 * (HD / 4) / FP4_BLOCK;
        }
      }
  };
  uint64_t have = 0, have_next = 0;
  if (blocks > 0) {
    request(0);
    place();
    widen(0);
    have_next = have_raw;
    if (blocks > 1) request(1);
    place();
  }
  for (int n = 0; n < blocks; ++n) {
    __syncthreads();                                       // block n is there, and nobody works on the one before
    have = have_next;
    if (n + 1 < blocks) {
      widen(n + 1);
      have_next = have_raw;
      if (n + 2 < blocks) request(n + 2);
      place();
    }
    const int base = it.lo + n * KV;
    if (!busy || base > wave_last || base + KV - 1 < wave_from) continue;      // no row of the wave sees any of it
    const bool whole = have == ~0ull && base + KV - 1 <= wave_first && base >= wave_all;
    step(n, base, have, whole);
  }
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
    if (nans >> d & 1)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] = __builtin_nanf("");
  l += __shfl_xor(l, 32, WAVE);
  if (r >= all_rows) return;
  if (it.parts > 1) {
    const int64_t at = ((int64_t)it.slot * kvheads + kvh) * TILE_ROWS + 32 * wave + col;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4) *(f32x4*)(a.part_o + at * HD + 32 * d + 2 * e + 4 * half) = (f32x4){o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]};
    if (half == 0) a.part_ml[at] = make_float2(m, l);
    return;
  }
  const bool none = m == -INFINITY && l == 0.f;
  const float inv = 1.0f / l;
  T* const to = (T*)a.out + (int64_t)(it.rows0 + tok) * a.o_tok + (int64_t)head * a.o_head + 4 * half;
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      f32x4 y = {o[d][e] * inv, o[d][e + 1] * inv, o[d][e + 2] * inv, o[d][e + 3] * inv};
      if (none) y = (f32x4){0.f, 0.f, 0.f, 0.f};
      *(u32x2*)(to + 32 * d + 2 * e) = quad_out<T>(y);
    }
  if (a.lse && half == 0) a.lse[(int64_t)(it.rows0 + tok) * a.heads + head] = none ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718f;
}

template <typename T, bool NEAR>
hipError_t tiles_go(const Fp4AttnArgs& a, int head_dim, dim3 grid, hipStream_t stream) {
  if (head_dim == 64) hipLaunchKernelGGL((paged_tile_fp4_kernel<T, 64, NEAR>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((paged_tile_fp4_kernel<T, 128, NEAR>), grid, dim3(256), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.least == 0) return e;
  const int rpw = 256 / (head_dim / 4);
  const dim3 rows(a.b.n_tokens, (a.heads + rpw - 1) / rpw);
  const PagedAttnArgs& parts = a;
  if (head_dim == 64) hipLaunchKernelGGL((paged_merge_kernel<T, 64>), rows, dim3(256), 0, stream, parts);
  else hipLaunchKernelGGL((paged_merge_kernel<T, 128>), rows, dim3(256), 0, stream, parts);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_tiles_fp4(const Fp4AttnArgs& a, int dtype, int head_dim, hipStream_t stream) {
  const dim3 grid((unsigned)a.items * a.kv_heads);
  const bool near = near_pages_fp4(a);
  if (dtype == PPD_BF16) return near ? tiles_go<bf16_t, true>(a, head_dim, grid, stream) : tiles_go<bf16_t, false>(a, head_dim, grid, stream);
  if (dtype == PPD_FP16) return near ? tiles_go<f16_t, true>(a, head_dim, grid, stream) : tiles_go<f16_t, false>(a, head_dim, grid, stream);
  return hipErrorInvalidValue;
}

}  // namespace ppd
