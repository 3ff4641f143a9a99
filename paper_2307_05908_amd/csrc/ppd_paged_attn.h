// What the kernels of ppd_paged_attention share: arguments, the plan of parts, element types as operands of the matrix units.
//
// For a key/value head its group of query heads is as many rows for each new token: row r of a sequence is token r / group, head
// r % group of the group, and a tile is a number of rows that read the same keys and values.  Scores are computed transposed, S^T = K Q^T:
// in a matrix product's result a lane then has one row (a column of S^T) and four positions in turn, so a row's maximum and sum stay in a
// lane but for an exchange of two or four lanes, and the weights are, as they lie in the registers, the right operand of O^T = V^T P^T.
#pragma once
#include "ppd_layers_common.h"

#include <type_traits>

namespace ppd {

constexpr int SPLIT_ROWS = 16, TILE_ROWS = 128;   // rows of a tile of paged_split_kernel and of paged_tile_kernel
constexpr int SPLIT_WAVES = 4, SPLIT_THREADS = SPLIT_WAVES * WAVE;
constexpr int PLAN_BLOCK = 64;                    // positions that lengths are cut by

struct PagedAttnArgs {
  Batch b;
  const void* q; void* out; float* lse; const void *kc, *vc;
  int64_t q_tok, q_head, o_tok, o_head;
  int64_t kc_page, kc_pos, kc_head, vc_page, vc_pos, vc_head;
  int heads, kv_heads, group, window;
  int tile_rows, items;               // items: parts of a key/value head that there are workgroups and places for
  float to_log2;                      // scale * log2(e): a score's exponent of two
  int want, fine, least, whole;       // parts per key/value head to aim at, and among sequences of unlike lengths; blocks of a part at least (0:
                                      // one part each), and up to which a tile is not cut
  float* part_o; float2* part_ml;     // [item][kv_heads][rows of a tile][head_dim], [item][kv_heads][rows of a tile]
  uint64_t* stamps; uint64_t stamp;   // paged_split_kernel, [item][kv_heads]: this call's number, once the part is there (see join_parts)
  int2* plan;                         // paged_tile_kernel, [n_seqs]: first item of a sequence, parts of its tiles
  int wide_want; float wide_from;     // 0, or parts to aim at where all tiles together have this many blocks: wide workgroups then (paged_split_fp4_kernel)
};

// ---- element types as matrix operands
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

__device__ __forceinline__ f32x4 mma16(u32x4 a, u32x4 b, f32x4 c, bf16_t) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma16(u32x4 a, u32x4 b, f32x4 c, f16_t) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c, bf16_t) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c, f16_t) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// two numbers rounded to the type, side by side, and what the rounding left of them
__device__ __forceinline__ uint32_t pair(float a, float b, bf16_t) { const bf16x2 v = {(__bf16)a, (__bf16)b}; return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ void rest(uint32_t p, float& a, float& b, bf16_t) { a -= __uint_as_float(p << 16); b -= __uint_as_float(p & 0xffff0000u); }
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pair(float a, float b, f16_t) { const f16x2 v = {(_Float16)a, (_Float16)b}; return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ void rest(uint32_t p, float& a, float& b, f16_t) { const f16x2 v = __builtin_bit_cast(f16x2, p); a -= (float)v.x; b -= (float)v.y; }
// What weights are taken from, as an exponent of two.  For half floats so far below the row's maximum that the largest weight is 2^15, near their
// largest number (2^(15 - slack) where the maximum may leave the reference by slack before that follows): they end at 2^-24, and of many
// weights far below one of 1 the sum has what the products with the values lose (65536 positions at 2^-25.1 beside one: 1.8e-3 of
// the result).  bf16 and fp32 go down to 2^-126 and lower.
template <typename T> __device__ __forceinline__ float reference(float top, int slack) { return std::is_same<T, f16_t>::value ? top - (float)(15 - slack) : top; }
// the largest of the numbers' magnitudes, as bits, and whether it is infinite or no number
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <typename T> __device__ __forceinline__ uint32_t largest(uint32_t m, u32x4 v, T) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if constexpr (sizeof(T) == 4) m = max(m, v[e] & 0x7fffffffu);
    else m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m), __builtin_bit_cast(u16x2, v[e] & 0x7fff7fffu)));
  return m;
}
__device__ __forceinline__ bool endless(uint32_t m, bf16_t) { return m >= 0x7f800000u || (m & 0xffffu) >= 0x7f80u; }
__device__ __forceinline__ bool endless(uint32_t m, f16_t) { return m >= 0x7c000000u || (m & 0xffffu) >= 0x7c00u; }
__device__ __forceinline__ bool endless(uint32_t m, float) { return m >= 0x7f800000u; }
template <typename T> __device__ __forceinline__ typename Quad<T>::raw quad_out(f32x4 v) {
  if constexpr (sizeof(T) == 4) return Quad<T>::narrow(v);
  else return (u32x2){pair(v.x, v.y, T()), pair(v.z, v.w, T())};
}

// ---- what a workgroup does: a part of the positions of one tile of one sequence
struct Item {
  int s, rows0, n, pos0;   // the sequence, its first row of the tensors, its tokens, the first one's position
  int tile, part, parts;
  int slot;                // where its partial results go
  int lo, hi;              // positions of the part, see span_of
  bool wide;               // a workgroup has four heads, a wave each
};

// The first position that a row at `pos` sees.  Positions are negative where kv_len is below the rows, and windows go up to 2^31 - 1.
__host__ __device__ __forceinline__ int first_seen(int pos, int window) { return window > 0 && pos >= window ? pos - window + 1 : 0; }

// Positions of a part of a tile, lo a multiple of PLAN_BLOCK; both 0 where there are none, so that what is looked up ahead of a loop over them is
// no further off than a few steps behind the table's room (2^30 at most), whatever kv_len is.
struct Span { int lo, hi; };
__host__ __device__ __forceinline__ Span span_of(int pos0, int n, int tile, int tile_rows, int group, int part, int parts, int room, int window) {
  const int first = tile * tile_rows / group, end = (tile * tile_rows + tile_rows - 1) / group, last = end < n - 1 ? end : n - 1;
  const int to = pos0 + last + 1, hi = to < room ? to : room, lo = first_seen(pos0 + first, window) & -PLAN_BLOCK;
  if (lo >= hi) return {0, 0};
  const int blocks = (hi - lo + PLAN_BLOCK - 1) / PLAN_BLOCK, per = (blocks + parts - 1) / parts, b0 = part * per, b1 = b0 + per;
  if (b0 >= blocks) return {0, 0};
  return {lo + b0 * PLAN_BLOCK, b1 < blocks ? lo + b1 * PLAN_BLOCK : hi};
}

struct SeqPlan { int tiles, blocks; SeqRows r; };
template <int TILE>
__device__ __forceinline__ void seq_plan(const PagedAttnArgs& a, int s, SeqPlan& p) {
  p.tiles = p.blocks = 0;
  p.r = {0, 0, 0};
  if (s >= a.b.n_seqs) return;
  p.r = seq_rows(a.b, s);
  if (p.r.rows == 0) return;
  p.tiles = (p.r.rows * a.group + TILE - 1) / TILE;                            // (2^26 rows at most)
  const int hi = min(p.r.pos0 + p.r.rows, a.b.room), lo = first_seen(p.r.pos0, a.window) & -PLAN_BLOCK;
  p.blocks = max(1, (hi - lo + PLAN_BLOCK - 1) / PLAN_BLOCK);
}
// One part for each tile: sequence s has items from q_start[s] * group / TILE + min(s, q_start[s]) on.  That leaves room for its tiles (and sometimes
// for one more), is known without the lengths before it, and never decreases: the last sequence that begins at or before the item has it.
template <int TILE>
__device__ __forceinline__ bool find_whole(const PagedAttnArgs& a, int idx, int lane, Item& it) {
  static_assert(PPD_MAX_SEQS <= WAVE * WAVE, "two rounds of loads");
  auto first_of = [&](int s, int row) { return row * a.group / TILE + min(s, row); };
  int from = 0;
  if (a.b.n_seqs > WAVE) {                                  // which 64 sequences
    const int s = lane * WAVE;
    const bool begun = s < a.b.n_seqs && first_of(s, min(max(a.b.q_start[min(s, a.b.n_seqs)], 0), a.b.n_tokens)) <= idx;
    from = max(__popcll(__ballot(begun)) - 1, 0) * WAVE;
  }
  SeqPlan p;
  seq_plan<TILE>(a, from + lane, p);
  const bool begun = from + lane < a.b.n_seqs && first_of(from + lane, p.r.row0) <= idx;
  const int w = __popcll(__ballot(begun)) - 1;
  if (w < 0) return false;
  it.s = from + w;
  it.rows0 = __builtin_amdgcn_readlane(p.r.row0, w);
  it.n = __builtin_amdgcn_readlane(p.r.rows, w);
  it.pos0 = __builtin_amdgcn_readlane(p.r.pos0, w);
  const int tiles = __builtin_amdgcn_readlane(p.tiles, w), r = idx - first_of(it.s, it.rows0);
  it.tile = TILE == TILE_ROWS ? tiles - 1 - r : r;
  it.part = 0; it.parts = 1; it.slot = idx;
  return r >= 0 && r < tiles;
}

// Every wave makes the plan for itself, from the lengths on the device: all tiles' blocks of positions together are cut into about
// `want` parts of equal length, a tile at its own ends.  (The sum is in fp32, one order: every wave has the same; its error is far below
// the one item that the grid has to spare.)  A lane looks at J sequences in turn, all lanes at once: up to 64 J sequences need one look.
// False: there is no such item.  WIDE: workgroups of four heads where there is so much to read (as a part of every kernel this cost one token's attention over 16-bit pages
// 0.2 us of 10.8).
template <int TILE, int J, bool WIDE>
__device__ __forceinline__ bool find_part(const PagedAttnArgs& a, int idx, int wide_idx, bool tell, int lane, Item& it) {
  int tiles[J], blocks[J];
  SeqRows r1;                                               // (J 1: the lane's sequence)
  const bool few = a.b.n_seqs <= WAVE * J;
  auto look = [&](int s) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      SeqPlan p;
      seq_plan<TILE>(a, s + lane * J + j, p);
      tiles[j] = p.tiles; blocks[j] = p.blocks;
      if (J == 1) r1 = p.r;
    }
  };
  float all = 0.f, count = 0.f, longest = 0.f;
  for (int s = 0; s < a.b.n_seqs; s += WAVE * J) {
    look(s);
    float x = 0.f, y = 0.f, z = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) { x += (float)tiles[j] * (float)blocks[j]; y += (float)tiles[j]; z = fmaxf(z, (float)blocks[j]); }
    all += wave_sum(x);
    count += wave_sum(y);
    longest = fmaxf(longest, wave_max(z));
  }
  // Two workgroups run on a unit, and where lengths differ and two long parts meet on one it is the last to end: then shorter parts, if they
  // are not too short for that.  bf16, us at `want` / `fine`: 64 sequences of 60 to 8000 positions 97 / 88, 32 of them 39.2 / 37.2, 64 of 60 to
  // 2000 32.1 / 34.2; of like lengths, 48 of 1000 38.6 / 45.1, 16 of 2000 29.3 / 32.9.
  it.wide = WIDE && a.wide_want > 0 && all >= a.wide_from;
  if (it.wide) idx = wide_idx;
  const float want = it.wide ? (float)a.wide_want : longest * count > 2.f * all && all >= 12.f * (float)a.fine ? (float)a.fine : (float)a.want;
  int len = max(a.least, (int)ceilf(all / want));
  // few tiles: where their ends make it more parts than `want`, longer ones (a second round of workgroups for a few of them would cost more)
  for (int again = 0; again < 3 && few && J == 1; ++again) {
    float x = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) x += (float)(tiles[j] * (blocks[j] <= a.whole ? 1 : (blocks[j] + len - 1) / len));
    const float items = wave_sum(x);
    if (items <= want || 2.f * count > want) break;
    len = (int)ceilf((float)len * items / want);
  }
  // Tiles of several parts come first, then those of more than half a part's length, more than a quarter, and the rest: what is begun late is
  // short.  (Two turns for sequences that take more than one look.)
  int parts[J], turns[J];
  auto cut = [&]() {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      parts[j] = blocks[j] <= a.whole ? 1 : (int)((unsigned)(blocks[j] + len - 1) / (unsigned)len);
      turns[j] = parts[j] > 1 ? 0 : !few || 4 * blocks[j] <= len ? 3 : 2 * blocks[j] <= len ? 2 : 1;
    }
  };
  cut();
  int before = 0;
  bool found = false;
  for (int turn = 0; turn < 4 && (tell || !found); turn += few ? 1 : 3)
    for (int s = 0; s < a.b.n_seqs; s += WAVE * J) {
      if (!few) { look(s); cut(); }
      int items[J], mine = 0;
#pragma unroll
      for (int j = 0; j < J; ++j) { items[j] = turns[j] == turn ? tiles[j] * parts[j] : 0; mine += items[j]; }
      if (!__ballot(mine > 0)) continue;
      const int upto = before + scan_up(mine);
      if (tell) {
        int at = upto - mine;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          if (items[j] > 0) a.plan[s + lane * J + j] = make_int2(at, parts[j]);     // (no items behind the last sequence)
          at += items[j];
        }
      }
      const unsigned long long past = __ballot(upto > idx);
      if (!found && past) {
        const int w = __builtin_ctzll(past);
        int r = idx - (upto - mine), j0 = 0, many = 0, its = 0;                       // (of lane w's sequences, the one that has the item)
        bool there = false;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          if (there) continue;
          if (r < items[j]) { there = true; j0 = j; many = parts[j]; its = tiles[j]; } else r -= items[j];
        }
        r = __builtin_amdgcn_readlane(r, w);
        it.s = s + w * J + __builtin_amdgcn_readlane(j0, w);
        it.parts = __builtin_amdgcn_readlane(many, w);
        SeqRows q;
        if (J == 1) q = {__builtin_amdgcn_readlane(r1.row0, w), __builtin_amdgcn_readlane(r1.rows, w), __builtin_amdgcn_readlane(r1.pos0, w)};
        else q = seq_rows(a.b, it.s);
        it.rows0 = q.row0; it.n = q.rows; it.pos0 = q.pos0;
        it.tile = r / it.parts;
        it.part = r % it.parts;
        if (TILE == TILE_ROWS) it.tile = __builtin_amdgcn_readlane(its, w) - 1 - it.tile;   // (the longest ones first)
        it.slot = idx - r + it.tile * it.parts + it.part;
        found = true;
        if (!tell) break;
      }
      before = __builtin_amdgcn_readlane(upto, 63);
    }
  return found;
}
// Whether parts from place `first` on have places: always, but where q_start decreases and sequences share rows, so that there are more parts than
// the host has counted.
__host__ __device__ __forceinline__ bool have_places(int first, int parts, int items) { return first >= 0 && parts <= items - first; }

template <int TILE, bool WIDE = false>
__device__ __forceinline__ bool find_item(const PagedAttnArgs& a, int idx, int wide_idx, bool tell, int lane, Item& it) {
  it.wide = false;
  if (!(a.least == 0 ? find_whole<TILE>(a, idx, lane, it) : a.b.n_seqs <= WAVE ? find_part<TILE, 1, WIDE>(a, idx, wide_idx, tell, lane, it)
                                                                               : find_part<TILE, 8, WIDE>(a, idx, wide_idx, tell, lane, it))) return false;
  if (!have_places(it.slot - it.part, it.parts, a.items)) return false;
  const Span span = span_of(it.pos0, it.n, it.tile, TILE, a.group, it.part, it.parts, a.b.room, a.window);
  it.lo = span.lo; it.hi = span.hi;
  return true;
}

// ---- parts joined
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
// The waves of a workgroup joined: their results lie out_lds bytes apart, sums in rows of HD + 4 and behind them references and totals.  What comes of it
// is the result, or a part's.  WIDE: every wave has a key/value head of its own, kvh0 and on.
template <typename T, int HD, bool WIDE = false, int ROWS = SPLIT_ROWS>
__device__ __forceinline__ void join_waves(const PagedAttnArgs& a, const Item& it, int kvh0, int tid, const char* lds, int out_lds) {
  constexpr int HEADS = WIDE ? SPLIT_WAVES : 1, WAVES = SPLIT_WAVES / HEADS;
  for (int x = tid; x < HEADS * ROWS * HD / 4; x += SPLIT_THREADS) {
    const int own = x / (ROWS * HD / 4), kvh = kvh0 + own, rr = x / (HD / 4) % ROWS, d = (x % (HD / 4)) * 4, ri = it.tile * ROWS + rr;
    if (ri >= it.n * a.group) continue;
    float2 ml[WAVES];
    float mx = -INFINITY, sum = 0.f;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) { ml[w] = ((const float2*)((const float*)(lds + (own + w) * out_lds) + ROWS * (HD + 4)))[rr]; mx = fmaxf(mx, ml[w].x); }
    const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(ml[w].x - ref);
      sum = fmaf(f, ml[w].y, sum);
      const f32x4 z = *(const f32x4*)((const float*)(lds + (own + w) * out_lds) + rr * (HD + 4) + d);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = fmaf(f, z[e], y[e]);
    }
    if (it.parts > 1) {
      const int64_t at = ((int64_t)it.slot * a.kv_heads + kvh) * ROWS + rr;
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
}
// The end of a workgroup that had one of several parts (all of its threads, its results left): it puts the call's number beside them and
// looks at the other parts' places; who finds the number everywhere joins them, in their order, and clears the places.  Nobody waits.
// The number goes out, past the L2, before the others are looked at, so the last one to leave it finds all; two may, and write the
// same bits.  Scratch memory needs nothing in it beforehand (numbers are 64 bits wide and never come twice, but for a replayed
// launch's, and that one's own places are clear again by then).
template <typename T, int HD, bool WIDE = false, int ROWS = SPLIT_ROWS>
__device__ __forceinline__ void join_parts(const PagedAttnArgs& a, const Item& it, int kvh0, int tid, int* s_flag) {      // s_flag: [heads]
  constexpr int HEADS = WIDE ? SPLIT_WAVES : 1;
  const int lane = tid & 63, own = WIDE ? tid >> 6 : 0;
  const int first = it.slot - it.part;                    // (the parts' places lie side by side)
  uint64_t* const stamps = a.stamps + (int64_t)first * a.kv_heads + kvh0;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid < HEADS * WAVE) {
    if (lane == 0) __hip_atomic_store(stamps + (int64_t)it.part * a.kv_heads + own, a.stamp, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    bool missing = false;
    for (int p = lane; p < it.parts; p += WAVE) missing |= __hip_atomic_load(stamps + (int64_t)p * a.kv_heads + own, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != a.stamp;
    missing = __ballot(missing) != 0;
    if (lane == 0) s_flag[own] = !missing;
  }
  __syncthreads();
#pragma unroll 1
  for (int head = 0; head < HEADS; ++head) {
    if (!s_flag[head]) continue;
    const int kvh = kvh0 + head;
    const int rows = min(ROWS, it.n * a.group - it.tile * ROWS);
    for (int x = tid; x < rows * (HD / 4); x += SPLIT_THREADS) {
      const int rr = x / (HD / 4), d = x % (HD / 4) * 4, ri = it.tile * ROWS + rr;
      auto at = [&](int p) { return ((int64_t)(first + p) * a.kv_heads + kvh) * ROWS + rr; };
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
    for (int p = tid; p < it.parts; p += SPLIT_THREADS) __hip_atomic_store(stamps + (int64_t)p * a.kv_heads + head, (uint64_t)0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

namespace {      // (a kernel that two sources have)

// The parts of a row joined, in their order: HD / 4 lanes for a row.  Bound by reading them (500 rows of 40 heads in 3 parts, 31 MB: 9 us).  A launch
// of its own: joined by the workgroups that had the parts, as paged_split_kernel does, 500 tokens over 4000 positions took 143 us beside 86 then.
template <typename T, int HD>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttnArgs a) {
  constexpr int LPR = HD / 4, RPW = 256 / LPR;
  const int row = blockIdx.x, lane = threadIdx.x & 63;
  const int s = seq_of_row(a.b, row, lane);
  if (s < 0) return;
  const SeqRows sr = seq_rows(a.b, s);
  if ((unsigned)(row - sr.row0) >= (unsigned)sr.rows) return;      // (q_start decreases: the sequence has other rows, or none and no plan)
  const int2 plan = a.plan[s];
  const int parts = plan.y, h = blockIdx.y * RPW + threadIdx.x / LPR, d = (threadIdx.x % LPR) * 4;
  if (parts <= 1 || h >= a.heads) return;
  const int kvh = h / a.group, r = (row - sr.row0) * a.group + h % a.group, first = plan.x + r / TILE_ROWS * parts;
  if (!have_places(first, parts, a.items)) return;
  float mx = -INFINITY, sum = 0.f;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < parts; p0 += 4) {                  // four parts at a time, their sums and totals in one go
    float2 ml[4];
    f32x4 z[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int64_t at = ((int64_t)(first + min(p0 + p, parts - 1)) * a.kv_heads + kvh) * TILE_ROWS + r % TILE_ROWS;
      ml[p] = a.part_ml[at];
      z[p] = *(const f32x4*)(a.part_o + at * HD + d);
    }
    const float before = mx;
#pragma unroll
    for (int p = 0; p < 4; ++p) mx = fmaxf(mx, ml[p].x);
    const float ref = mx == -INFINITY ? 0.f : mx, keep = __builtin_amdgcn_exp2f(before - ref);
    if (p0 > 0) { sum *= keep; y *= keep; }
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      if (p0 + p >= parts) break;
      const float f = __builtin_amdgcn_exp2f(ml[p].x - ref);
      sum = fmaf(f, ml[p].y, sum);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = fmaf(f, z[p][e], y[e]);
    }
  }
  const bool none = mx == -INFINITY && sum == 0.f;
  const float inv = 1.0f / sum;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = none ? 0.f : y[e] * inv;
  *(typename Quad<T>::raw*)((T*)a.out + (int64_t)row * a.o_tok + (int64_t)h * a.o_head + d) = quad_out<T>(y);
  if (a.lse && d == 0) a.lse[(int64_t)row * a.heads + h] = none ? -INFINITY : (mx + __builtin_amdgcn_logf(sum)) * 0.69314718f;
}

}  // namespace

// Whether 16 positions in a row that begin at a multiple of 16 lie in one page, within 2^31 bytes
inline bool near_pages(const PagedAttnArgs& a) { return a.b.page_size % 16 == 0 && a.kc_pos < 1 << 25 && a.vc_pos < 1 << 25; }
hipError_t launch_paged_tiles(const PagedAttnArgs& a, int dtype, int head_dim, hipStream_t stream);
uint64_t next_stamp();      // of a call, see join_parts

}  // namespace ppd
