// ppd_paged_plan: a step's row starts, lengths, pages and slots, from what each sequence keeps and wants.  Bound by latencies: one workgroup
// reads the lengths, sums them up (sequences in their order, so that results do not depend on when a wave runs) and moves the pages' numbers;
// the places of many rows are found by a launch of their own.
#include "ppd_layers_common.h"

using namespace ppd;

namespace {

struct PlanArgs {
  const int64_t* counters; int64_t* counters_out;
  const int32_t *held, *kept, *wanted;
  int32_t *q_start, *kv_len, *granted, *row_seq, *positions; int64_t* slots;
  int32_t *pages, *free_pages;
  int64_t pages_stride;
  int max_pages, n_pages, page_size, n_seqs, n_rows;
  bool rows_here;           // rows' places by plan_kernel
};

template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t dpp_plus(uint32_t v) { return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ uint32_t wave_upto(uint32_t v) {      // sums up to the lane's
  v = dpp_plus<0x111, 0xf>(v);
  v = dpp_plus<0x112, 0xf>(v);
  v = dpp_plus<0x114, 0xf>(v);
  v = dpp_plus<0x118, 0xf>(v);
  v = dpp_plus<0x142, 0xa>(v);
  return dpp_plus<0x143, 0xc>(v);
}
// The sum of the threads before this one, and of all, at most 2^30 of either but for a wave's own share.  `to`: a word for each wave, of no other
// call's.
template <int THREADS>
__device__ __forceinline__ uint32_t block_before(uint32_t v, uint32_t* to, uint32_t& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t upto = wave_upto(v);
  if (lane == 63) to[wave] = upto;
  __syncthreads();
  uint32_t before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < THREADS / WAVE; ++w) {
    if (w == wave) before = all;
    all = min(all + to[w], 1u << 30);
  }
  return before + (upto - v);
}
// the last of n ascending numbers that is not above x (the first one is not)
__device__ __forceinline__ int last_upto(const int32_t* from, int n, int x) {
  int lo = 0, more = n;                                     // the answer is in [lo, lo + more)
  while (more > 1) {
    const int step = more >> 1;
    if (from[lo + step] <= x) { lo += step; more -= step; } else more = step;
  }
  return lo;
}
__device__ __forceinline__ void place_row(const PlanArgs& a, int row, int s, int pos) {
  if (a.row_seq) a.row_seq[row] = s;
  if (a.positions) a.positions[row] = s < 0 ? -1 : pos;
  if (!a.slots) return;
  int64_t slot = -1;
  if (s >= 0) {
    const int i = (int)((unsigned)pos / (unsigned)a.page_size), page = a.pages[(int64_t)s * a.pages_stride + i];
    if ((unsigned)page < (unsigned)a.n_pages) slot = (int64_t)page * a.page_size + (pos - i * a.page_size);
  }
  a.slots[row] = slot;
}

// A thread has J sequences in a row.  Pages are 2^30 at most in all, the places of the table; sums of tokens end there, where no sequence fits any
// more.
template <int THREADS, int J>
__global__ __launch_bounds__(THREADS) void plan_kernel(PlanArgs a) {
  constexpr int MOST = THREADS * J;
  __shared__ uint32_t sums[5][THREADS / WAVE];
  __shared__ int32_t s_start[MOST + 1], s_moved[2][MOST], s_place[MOST], s_len[MOST];     // rows; pages taken, given back, before a sequence's; its first place of them; its length
  const int tid = threadIdx.x, s0 = tid * J, n = a.n_seqs;
  const uint32_t size = (uint32_t)a.page_size;
  const int room = a.max_pages * a.page_size;               // (at most 2^30)
  const int64_t head = a.counters[0], tail = a.counters[1], between = (int64_t)((uint64_t)tail - (uint64_t)head);
  const int free = between < 0 ? 0 : between > a.n_pages ? a.n_pages : (int)between;
  int kept[J], wanted[J], have[J];
  uint32_t ask = 0;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int s = s0 + j;
    const bool there = s < n;
    const int held = there ? min(max(a.held[s], 0), room) : 0;
    kept[j] = there && a.kept ? min(max(a.kept[s], 0), held) : held;
    wanted[j] = there ? max(a.wanted[s], 0) : 0;
    if (wanted[j] > room - kept[j]) wanted[j] = 0;
    have[j] = (int)(((uint32_t)held + size - 1) / size);
    ask += (uint32_t)min(wanted[j], a.n_rows + 1);
  }
  uint32_t all, before = block_before<THREADS>(ask, sums[0], all), need = 0;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    before += (uint32_t)min(wanted[j], a.n_rows + 1);
    if (before > (uint32_t)a.n_rows) wanted[j] = 0;
    need += (uint32_t)max((int)(((uint32_t)(kept[j] + wanted[j]) + size - 1) / size) - have[j], 0);
  }
  before = block_before<THREADS>(need, sums[1], all);
  uint32_t rows = 0, take = 0, give = 0;
  int want[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int more = max((int)(((uint32_t)(kept[j] + wanted[j]) + size - 1) / size) - have[j], 0);
    before += (uint32_t)more;
    if (more > 0 && before > (uint32_t)free) wanted[j] = 0;
    want[j] = (int)(((uint32_t)(kept[j] + wanted[j]) + size - 1) / size);
    rows += (uint32_t)wanted[j];
    take += (uint32_t)max(want[j] - have[j], 0);
    give += (uint32_t)max(have[j] - want[j], 0);
  }
  uint32_t all_rows, all_take, all_give;
  uint32_t at = block_before<THREADS>(rows, sums[2], all_rows), taken = block_before<THREADS>(take, sums[3], all_take), given = block_before<THREADS>(give, sums[4], all_give);
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int s = s0 + j;
    s_start[s] = (int)at; s_moved[0][s] = (int)taken; s_moved[1][s] = (int)given; s_place[s] = min(have[j], want[j]); s_len[s] = kept[j] + wanted[j];
    if (s < n) {
      a.q_start[s] = (int)at; a.kv_len[s] = kept[j] + wanted[j]; a.granted[s] = wanted[j];
    }
    at += (uint32_t)wanted[j]; taken += (uint32_t)max(want[j] - have[j], 0); given += (uint32_t)max(have[j] - want[j], 0);
  }
  if (tid == 0) { a.q_start[n] = (int)all_rows; s_start[MOST] = (int)all_rows; }
  __syncthreads();
  // pages taken: number i of them comes from place head + i of the ring
  const uint32_t from = (uint32_t)((uint64_t)head % (uint32_t)a.n_pages), to = (uint32_t)((uint64_t)tail % (uint32_t)a.n_pages);
  auto ring = [&](uint32_t first, uint32_t i) { const uint32_t x = first + i; return x >= (uint32_t)a.n_pages ? x - (uint32_t)a.n_pages : x; };      // i below n_pages
  for (uint32_t i = tid; i < all_take; i += THREADS) {
    const int s = last_upto(s_moved[0], n, (int)i);
    a.pages[(int64_t)s * a.pages_stride + s_place[s] + ((int)i - s_moved[0][s])] = a.free_pages[ring(from, i)];
  }
  // pages given back, those that are some, in their order, behind what is free
  const uint32_t put_most = (uint32_t)(a.n_pages - free);
  uint32_t put = 0;
  for (uint32_t i0 = 0; i0 < all_give; i0 += THREADS) {
    const uint32_t i = i0 + tid;
    int page = -1;
    if (i < all_give) {
      const int s = last_upto(s_moved[1], n, (int)i);
      page = a.pages[(int64_t)s * a.pages_stride + s_place[s] + ((int)i - s_moved[1][s])];
    }
    const bool some = (unsigned)page < (unsigned)a.n_pages;
    __syncthreads();                                        // (the words that the turn before has read)
    uint32_t now, mine = block_before<THREADS>(some, sums[0], now);
    if (some && put + mine < put_most) a.free_pages[ring(to, put + mine)] = page;
    put = min(put + now, put_most);
  }
  if (tid == 0) { a.counters_out[0] = (int64_t)((uint64_t)head + all_take); a.counters_out[1] = (int64_t)((uint64_t)tail + put); }
  if (!a.rows_here) return;
  __syncthreads();                                          // the table is written
  for (int row = tid; row < a.n_rows; row += THREADS) {
    const int s = row < (int)all_rows ? last_upto(s_start, n, row) : -1;
    place_row(a, row, s, s < 0 ? 0 : s_len[s] - (s_start[s + 1] - row));
  }
}

// Many rows: 1024 of them a workgroup.
constexpr int ROWS_A_GROUP = 1024;
__global__ __launch_bounds__(256) void plan_rows_kernel(PlanArgs a) {
  __shared__ int32_t start[PPD_MAX_SEQS + 1];
  for (int i = threadIdx.x; i <= a.n_seqs; i += 256) start[i] = a.q_start[i];
  __syncthreads();
  for (int row = blockIdx.x * ROWS_A_GROUP + threadIdx.x; row < min(a.n_rows, (int)(blockIdx.x + 1) * ROWS_A_GROUP); row += 256) {
    const int s = row < start[a.n_seqs] ? last_upto(start, a.n_seqs, row) : -1;
    place_row(a, row, s, s < 0 ? 0 : a.kv_len[s] - (start[s + 1] - row));
  }
}

}  // namespace

extern "C" int ppd_paged_plan(const ppd_page_table* table, const int64_t* counters, int64_t* counters_out, const int32_t* held,
                              const int32_t* kept, const int32_t* wanted, int n_rows, int32_t* q_start, int32_t* kv_len,
                              int32_t* granted, int32_t* row_seq, int32_t* positions, int64_t* slots, void* hip_stream) {
  if (!table || !table->pages || !table->free_pages || !counters || !counters_out || !held || !wanted || !q_start || !kv_len || !granted) return PPD_EINVAL;
  if (((uintptr_t)table->pages | (uintptr_t)table->free_pages | (uintptr_t)held | (uintptr_t)kept | (uintptr_t)wanted | (uintptr_t)q_start | (uintptr_t)kv_len |
       (uintptr_t)granted | (uintptr_t)row_seq | (uintptr_t)positions) & 3 || ((uintptr_t)counters | (uintptr_t)counters_out | (uintptr_t)slots) & 7)
    return PPD_EINVAL;
  if (table->n_seqs < 1 || table->max_pages < 1 || table->n_pages < 1 || table->page_size < 1 || n_rows < 0) return PPD_EINVAL;
  if (table->n_seqs > 1 && table->pages_stride < table->max_pages) return PPD_EINVAL;
  if (table->n_seqs > PPD_MAX_SEQS || n_rows > PPD_MAX_TOKENS || (int64_t)table->max_pages * table->page_size > 1 << 30) return PPD_ELIMIT;
  if ((int64_t)table->n_seqs * table->max_pages > 1 << 30) return PPD_ELIMIT;
  PlanArgs a = {counters, counters_out, held, kept, wanted, q_start, kv_len, granted, row_seq, positions, slots, table->pages, table->free_pages,
                table->pages_stride, table->max_pages, table->n_pages, table->page_size, table->n_seqs, n_rows, false};
  const bool rows = n_rows > 0 && (row_seq || positions || slots);
  a.rows_here = rows && n_rows <= 4096;
  hipStream_t st = (hipStream_t)hip_stream;
  if (a.n_seqs <= 256) hipLaunchKernelGGL((plan_kernel<256, 1>), dim3(1), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((plan_kernel<1024, 4>), dim3(1), dim3(1024), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !rows || a.rows_here) return launched(e);
  hipLaunchKernelGGL(plan_rows_kernel, dim3((n_rows + ROWS_A_GROUP - 1) / ROWS_A_GROUP), dim3(256), 0, st, a);
  return launched(hipGetLastError());
}
