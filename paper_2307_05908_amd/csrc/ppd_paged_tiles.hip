// ppd_paged_attention, many rows: bound by the matrix units and the issue of instructions beside them: a 32 x 32 x 16 product keeps its SIMD's
// vector units from the other wave for two thirds of its 32 cycles, and a block of 64 positions is 48 products of a wave (16 of them for the
// weights' second term), 32 exponentials and some 290 other vector instructions (products 53 % of the cycles, vector instructions 55 %, LDS
// 27 %).  Two bf16 prompts of 3800 and 4000 tokens (32 heads, 8 of keys and values, 249 GFLOP, 374 with the second term): 344 to 352 us from
// card to card, 1060 to 1090 TFLOP/s of products; a large matrix product of the library's reaches 1200.  With weights of one term, rounded to
// the type: 267 us, and an error of 2.1e-3 of bf16 outputs where their own rounding is 1.6e-3.
// (Tried and not kept: the first terms' products before the second terms', and weights' rests by a dot instruction, one a weight less: the same
// time.  With one term, beside 283 us at the time: the next block's scores between this one's exponentials, 286 to 292; a higher priority for
// the waves in products or in exponentials, 284 to 292; offsets kept in registers from block to block, 281 to 287.  Blocks of 32 positions and three
// workgroups a unit: 278 beside 279, 500 tokens over 4000 positions 81 beside 77, head_dim 64 113 beside 100.)
#include "ppd_paged_attn.h"

namespace ppd {
namespace {

// Two weights as two terms of the type, side by side.  The first is cut off, not rounded, and the second is not zero where the weight is not (the
// type's smallest normal number, or half floats' smallest one, 2^-31 of the row's largest weight): a value that is infinite has its sign in both
// products.  (The rests of rounded first terms need a second pass without such values, 9 ms, not 0.6, for the two prompts where no value is a number;
// else the same time.)
__device__ __forceinline__ u32x2 two_terms(float x, float y, bf16_t) {
  const uint32_t u = __float_as_uint(x), v = __float_as_uint(y);
  const float a = x - __uint_as_float(u & 0xffff0000u), b = y - __uint_as_float(v & 0xffff0000u);
  return (u32x2){__builtin_amdgcn_perm(v, u, 0x07060302u), pair(__builtin_amdgcn_fmed3f(a, x, 0x1p-126f), __builtin_amdgcn_fmed3f(b, y, 0x1p-126f), bf16_t())};
}
__device__ __forceinline__ u32x2 two_terms(float x, float y, f16_t) {
  const auto h = __builtin_amdgcn_cvt_pkrtz(x, y);
  const float a = x - (float)h[0], b = y - (float)h[1];
  return (u32x2){__builtin_bit_cast(uint32_t, h), pair(__builtin_amdgcn_fmed3f(a, x, 0x1p-24f), __builtin_amdgcn_fmed3f(b, y, 0x1p-24f), f16_t())};
}
// dma16 with the lanes' sources as 32-bit offsets from one address
__device__ __forceinline__ void dma16_near(const void* base, int offset, void* lds_dst) {
  const unsigned la = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds_dst;
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(la) : "memory", "m0");
}

// Four waves of 32 rows each; blocks of 64 positions in two LDS buffers, filled straight from the pages (a lane of a transfer names its own
// source, so the rows of a block may lie anywhere, and 16-byte pieces change places within a row so that no operand's reads meet on a bank):
// keys as they are, the left operand of S^T = K Q^T; values through the transposing reads, the left operand of O^T = V^T P^T.  The next
// block is under way while one is worked on, with one barrier a block; two workgroups on a compute unit fill each other's gaps.
// Heads of 64 leave registers for four workgroups a unit, if the compiler is asked (three: two prompts of 3000 151 us, not 143).
// NEAR: 16 positions in a row that begin at a multiple of 16 lie in one page, within 2^31 bytes, so that a wave's share of a block has one
// page and the lanes 32-bit offsets in it (the two prompts 350 us, not 377; 500 tokens over 4000 positions 86, not 91).
template <typename T, int HD, bool NEAR>
__global__ __launch_bounds__(256, HD == 64 ? 4 : 2) void paged_tile_kernel(PagedAttnArgs a) {
  constexpr int KV = PLAN_BLOCK, ROWB = HD * 2, UNITS = HD / 8, RPI = WAVE / UNITS, NI = 16 / RPI, SIDE = KV * ROWB;
  __shared__ __align__(1024) char lds[4 * SIDE];           // [2 buffers][keys, values][64 positions][head_dim]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
  // Workgroups go round the eight XCDs in turn, so with the heads of a part side by side those of a key/value head meet on one XCD where there are
  // a multiple of eight heads, and its L2 has the head's keys and values; and the longest parts of all heads come first.  (All of a head's
  // tiles before the next head's: 3000 fp16 rows of 40 heads 215 us, not 161.)
  const int kvheads = a.kv_heads, idx = blockIdx.x / kvheads, kvh = blockIdx.x % kvheads;
  __shared__ int s_odd[2];                                 // first and last block with a value that is infinite, or no number, where not every row sees it
  if (threadIdx.x == 0) { s_odd[0] = 0x7fffffff; s_odd[1] = -1; }
  Item it;
  if (!find_item<TILE_ROWS>(a, idx, 0, idx == 0 && kvh == 0 && wave == 0 && a.least > 0, lane, it)) return;
  const int all_rows = it.n * a.group;
  const int r0 = it.tile * TILE_ROWS + 32 * wave, r = r0 + col, rc = min(r, all_rows - 1), tok = rc / a.group, head = kvh * a.group + rc % a.group;
  const int pos = r < all_rows ? it.pos0 + tok : -1, from = first_seen(pos, a.window);
  const bool busy = r0 < all_rows;
  const int wave_first = it.pos0 + min(r0, all_rows - 1) / a.group, wave_last = it.pos0 + min(r0 + 31, all_rows - 1) / a.group;    // positions of the wave's rows
  const int tile_first = it.pos0 + it.tile * TILE_ROWS / a.group, tile_last = it.pos0 + min((it.tile * TILE_ROWS + TILE_ROWS - 1) / a.group, it.n - 1);
  const int wave_from = first_seen(wave_first, a.window), wave_all = first_seen(wave_last, a.window), tile_all = first_seen(tile_last, a.window);   // from where some row of the wave sees, all of its, all of the tile's
  u32x4 q[HD / 16];
  {
    const char* p = (const char*)a.q + ((int64_t)(it.rows0 + tok) * a.q_tok + (int64_t)head * a.q_head) * 2 + half * 16;
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) q[i] = *(const u32x4*)(p + i * 32);
  }
  const int blocks = (it.hi - it.lo + KV - 1) / KV;
  // The table's entry for, and the slot of, a block's position `lane`: asked for a block before it is looked at, when the block is requested.
  // (Looked at at once it would wait for the transfers that are under way.)  From block to block both move on by the same step.
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
  uint64_t have_next = 0;
  const char* const kbase = (const char*)a.kc + (int64_t)kvh * a.kc_head * 2;
  const char* const vbase = (const char*)a.vc + (int64_t)kvh * a.vc_head * 2;
  // (lane / UNITS is the row of a transfer, and the piece that it brings is the one whose place the lane has: see kat, vat)
  const int unit = lane % UNITS;
  int piece_k = (unit ^ (lane >> 4)) * 16, piece_v = (unit ^ 2 * (lane >> 4)) * 16, trow = lane / UNITS;
  auto request = [&](int n) {
    asm volatile("" : "+v"(piece_k), "+v"(piece_v), "+v"(trow));      // (worked out anew for every block: kept, the offsets would cost registers that there are not)
    const int page = it.lo + n * KV + lane < it.hi && (unsigned)entry < (unsigned)a.b.n_pages ? entry : -1;      // (hi is within the table)
    have_next = __ballot(page >= 0);
    char* const to = lds + (n & 1) * 2 * SIDE + 16 * wave * ROWB;
    if constexpr (NEAR) {
      const int pg = __builtin_amdgcn_readlane(page, 16 * wave), sl = pg >= 0 ? __builtin_amdgcn_readlane(slot, 16 * wave) : 0;
      // what has no page is read from where there is something, and not seen; so are positions behind the part in a page of its own
      const char* const kp = kbase + ((int64_t)max(pg, 0) * a.kc_page + (int64_t)sl * a.kc_pos) * 2;
      const char* const vp = vbase + ((int64_t)max(pg, 0) * a.vc_page + (int64_t)sl * a.vc_pos) * 2;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int row = RPI * i + trow;
        dma16_near(kp, row * (int)a.kc_pos * 2 + (piece_k ^ 64 * i), to + i * RPI * ROWB);
        dma16_near(vp, row * (int)a.vc_pos * 2 + (HD == 128 ? piece_v ^ 128 * (i & 1) : piece_v), to + SIDE + i * RPI * ROWB);
      }
    } else {
      const int pg = max(page, 0), sl = page >= 0 ? slot : 0;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int row = 16 * wave + RPI * i + trow;
        const int64_t rp = __shfl(pg, row, WAVE), rs = __shfl(sl, row, WAVE);
        dma16(kbase + (rp * a.kc_page + rs * a.kc_pos) * 2 + (piece_k ^ 64 * i), to + i * RPI * ROWB);
        dma16(vbase + (rp * a.vc_page + rs * a.vc_pos) * 2 + (HD == 128 ? piece_v ^ 128 * (i & 1) : piece_v), to + SIDE + i * RPI * ROWB);
      }
    }
  };
  f32x16 o[HD / 32];
#pragma unroll
  for (int i = 0; i < HD / 32; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  float m = -INFINITY, l = 0.f;
  // Where a lane's operands begin.  A row's 16-byte pieces have changed places by an exclusive or: keys with the row (head_dim 64: half of it),
  // so that eight rows in turn have a piece on eight places; values two pieces at a time, so that the four rows of a transposing read and
  // the four of the other half lie on different banks.  Keys: row col of half a block, piece 2 i + half at kat ^ 32 i.  Values: position
  // 4 half + i / 4 of 16, components 32 d + 16 (g % 2) + 4 (i % 4) at vat ^ 64 d, g = lane / 16, i = lane % 16.
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
      for (int i = 0; i < HD / 16; ++i) s[t] = mma32(*(const u32x4*)(buf + (kat ^ 32 * i) + t * 32 * ROWB), q[i], s[t], T());
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
    top = reference<T>(top * a.to_log2, SLACK);
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
    // Weights go into the second product in two terms of the type: the rounding of one alone is as large as the result's own.
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      u32x4 hi, lo;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const u32x2 w = two_terms(s[t / 2][8 * (t % 2) + 2 * e], s[t / 2][8 * (t % 2) + 2 * e + 1], T());
        hi[e] = w.x; lo[e] = w.y;
      }
#pragma unroll
      for (int d = 0; d < HD / 32; ++d) {
        const u32x4 v = values(t, d);
        o[d] = mma32(v, hi, o[d], T());
        o[d] = mma32(v, lo, o[d], T());
      }
    }
  };
  // Where not every row of the tile sees all of a block: a weight of zero does not silence a value that is infinite or no number, so these
  // are cleared in LDS (each wave its own 16 positions), and put in behind the loop where they are seen.
  auto clean = [&](int n, int base, uint64_t have) {
    char* const p = lds + (n & 1) * 2 * SIDE + SIDE + 16 * wave * ROWB + lane * 16;
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < NI; ++i) most = largest(most, *(const u32x4*)(p + i * RPI * ROWB), T());
    if (__ballot(endless(most, T()))) {
      bool seen = false;
#pragma unroll 1
      for (int i = 0; i < NI; ++i) {
        const int row = 16 * wave + RPI * i + lane / UNITS;
        u32x4 v = *(const u32x4*)(p + i * RPI * ROWB);
        seen |= endless(largest(0, v, T()), T()) && ((have >> row) & 1);
#pragma unroll
        for (int e = 0; e < 4; ++e) { if (endless(v[e] & 0x7fffu, T())) v[e] &= 0xffff0000u; if (endless(v[e] & 0x7fff0000u, T())) v[e] &= 0xffffu; }
        *(u32x4*)(p + i * RPI * ROWB) = v;
      }
      if (__ballot(seen) && lane == 0) { atomicMin(&s_odd[0], n); atomicMax(&s_odd[1], n); }
    }
  };
  if (blocks > 0) request(0);
  place();
  // the queries are waited for here: a wait in the loop would be one for the transfers, of which the compiler knows nothing
#pragma unroll
  for (int i = 0; i < HD / 16; ++i) asm volatile("" : "+v"(q[i]));
  for (int n = 0; n < blocks; ++n) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const uint64_t have = have_next;
    if (n + 1 < blocks) request(n + 1);
    place();
    const int base = it.lo + n * KV;
    if (!(have == ~0ull && base + KV - 1 <= tile_first && base >= tile_all)) {
      clean(n, base, have);
      __syncthreads();
    }
    if (!busy || base > wave_last || base + KV - 1 < wave_from) continue;      // no row of the wave sees any of it
    const bool whole = have == ~0ull && base + KV - 1 <= wave_first && base >= wave_all;
    step(n, base, have, whole);
  }
  __syncthreads();
  const int odd_first = s_odd[0], odd_last = s_odd[1];
#pragma unroll 1
  for (int n = odd_first; n <= odd_last; ++n) {
    // such a block once more, position by position, from the pages: a row that sees an infinite value, or no number, takes it up
    const int base = it.lo + n * KV, x = base + lane;
    const bool there = __ballot(x < it.hi && page_of(a.b, it.s, x) >= 0) == ~0ull;
    if (there && base + KV - 1 <= tile_first && base >= tile_all) continue;
#pragma unroll 1
    for (int p = base; p < min(base + KV, it.hi); ++p) {
      const int pg = page_of(a.b, it.s, p);
      if (pg < 0 || p > pos || p < from) continue;
      const T* const row = (const T*)vbase + (int64_t)pg * a.vc_page + (int64_t)((unsigned)p % (unsigned)a.b.page_size) * a.vc_pos + 4 * half;
#pragma unroll
      for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const f32x4 v = Quad<T>::wide(*(const u32x2*)(row + 32 * d + 2 * e));
#pragma unroll
          for (int z = 0; z < 4; ++z) o[d][e + z] += fabsf(v[z]) < INFINITY ? 0.f : v[z];
        }
    }
  }
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
hipError_t tiles_go(const PagedAttnArgs& a, int head_dim, dim3 grid, hipStream_t stream) {
  if (head_dim == 64) hipLaunchKernelGGL((paged_tile_kernel<T, 64, NEAR>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((paged_tile_kernel<T, 128, NEAR>), grid, dim3(256), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.least == 0) return e;
  const int rpw = 256 / (head_dim / 4);
  const dim3 rows(a.b.n_tokens, (a.heads + rpw - 1) / rpw);
  if (head_dim == 64) hipLaunchKernelGGL((paged_merge_kernel<T, 64>), rows, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((paged_merge_kernel<T, 128>), rows, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_tiles(const PagedAttnArgs& a, int dtype, int head_dim, hipStream_t stream) {
  const dim3 grid((unsigned)a.items * a.kv_heads);
  const bool near = near_pages(a);
  if (dtype == PPD_BF16) return near ? tiles_go<bf16_t, true>(a, head_dim, grid, stream) : tiles_go<bf16_t, false>(a, head_dim, grid, stream);
  if (dtype == PPD_FP16) return near ? tiles_go<f16_t, true>(a, head_dim, grid, stream) : tiles_go<f16_t, false>(a, head_dim, grid, stream);
  return hipErrorInvalidValue;
}

}  // namespace ppd
