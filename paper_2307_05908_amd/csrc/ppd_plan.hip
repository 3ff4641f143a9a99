// ppd_paged_plan: a step's row starts, lengths, pages and slots, from what each sequence keeps and wants.  Bound by latencies: one workgroup
// reads the lengths, sums them up (sequences in their order, so that results do not depend on when a wave runs) and moves the pages' numbers;
// the places of many rows are found by a launch of their own.  24 sequences 6.3 us, an empty kernel takes 2 to 3; 2048 sequences that move 16000 pages' numbers and
// have 131000 rows 18.6 + 6.0 (which sequence a page or a row belongs to by searches instead of marks, see owners: 38 together).
#include "ppd_divide.h"
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
  Divider by_size;          // (by page_size)
};
__device__ __forceinline__ int pages_of(const PlanArgs& a, int positions) { return (int)a.by_size((uint32_t)positions + (uint32_t)a.page_size - 1u); }

// K sums of the threads before this one, and of all, at most 2^30 of either but for a wave's own share.  `to`: words of no other call's.
template <int THREADS, int K>
__device__ __forceinline__ void block_before(uint32_t (&v)[K], uint32_t (*to)[THREADS / WAVE], uint32_t (&all)[K]) {
  constexpr int WAVES = THREADS / WAVE;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t upto[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    upto[k] = (uint32_t)scan_up((int)v[k]);
    if (lane == 63) to[k][wave] = upto[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) {
    // (waves' sums are 2^30 + 2^8 at most, and the sum of the waves up to one saturates by halves: a sum of two is cut to 2^30 before the next)
    uint32_t w = min(lane < WAVES ? to[k][lane] : 0u, 1u << 30);
#pragma unroll
    for (int o = 1; o < WAVES; o <<= 1) {
      const uint32_t x = (uint32_t)__shfl_up((int)w, o, WAVE);
      w = min(w + (lane >= o ? x : 0u), 1u << 30);
    }
    all[k] = (uint32_t)__builtin_amdgcn_readlane((int)w, WAVES - 1);
    const uint32_t before = wave > 0 ? (uint32_t)__builtin_amdgcn_readlane((int)w, max(wave - 1, 0)) : 0u;
    v[k] = before + (upto[k] - v[k]);
  }
}
// the last of n ascending numbers that is not above x (the first one is not)
__device__ __forceinline__ int last_upto(const int32_t* from, int n, int x) {
  int at = 0;
  for (int step = n > 1 ? 1 << (31 - __builtin_clz((uint32_t)(n - 1))) : 0; step > 0; step >>= 1) {
    const int next = at + step;
    at = next < n && from[min(next, n - 1)] <= x ? next : at;
  }
  return at;
}
__device__ __forceinline__ void place_row(const PlanArgs& a, int row, int s, int pos) {
  if (a.row_seq) a.row_seq[row] = s;
  if (a.positions) a.positions[row] = s < 0 ? -1 : pos;
  if (!a.slots) return;
  int64_t slot = -1;
  if (s >= 0) {
    const int i = (int)a.by_size((uint32_t)pos), page = a.pages[(int64_t)s * a.pages_stride + i];
    if ((unsigned)page < (unsigned)a.n_pages) slot = (int64_t)page * a.page_size + (pos - i * a.page_size);
  }
  a.slots[row] = slot;
}

template <int CTRL, int ROWS> __device__ __forceinline__ int dpp_most(int v) { return max(v, __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false)); }
// The sequences that numbers i0 + EACH * tid + u of a line belong to in which sequence s has `count` of them from `start` on, and -1 behind the last one's:
// each sequence marks the place where it begins, and the last mark up to a place is its own.  A thread knows J sequences from s0 on.
constexpr int EACH = 4;
template <int THREADS, int J>
__device__ __forceinline__ void owners(const int (&start)[J], const int (&count)[J], int s0, int i0, int (*mark)[EACH], int* last, int (&s)[EACH]) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  __syncthreads();                                          // (what the turn before has read)
#pragma unroll
  for (int u = 0; u < EACH; ++u) mark[tid][u] = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int at = max(start[j] - i0, 0);
    if (count[j] > 0 && start[j] + count[j] > i0 && at < EACH * THREADS) (&mark[0][0])[at] = s0 + j + 1;
  }
  __syncthreads();
  int most = 0;
#pragma unroll
  for (int u = 0; u < EACH; ++u) { most = max(most, mark[tid][u]); s[u] = most; }
  most = dpp_most<0x111, 0xf>(most);
  most = dpp_most<0x112, 0xf>(most);
  most = dpp_most<0x114, 0xf>(most);
  most = dpp_most<0x118, 0xf>(most);
  most = dpp_most<0x142, 0xa>(most);
  most = dpp_most<0x143, 0xc>(most);
  if (lane == 63) last[wave] = most;
  __syncthreads();
  int before = __builtin_amdgcn_update_dpp(0, most, 0x138, 0xf, 0xf, false);      // the lane before's
#pragma unroll
  for (int w = 0; w < THREADS / WAVE; ++w) if (w < wave) before = max(before, last[w]);
#pragma unroll
  for (int u = 0; u < EACH; ++u) s[u] = max(s[u], before) - 1;
}

// A thread has J sequences in a row.  Pages are 2^30 at most in all, the places of the table; sums of tokens end there, where no sequence fits any
// more.
template <int THREADS, int J>
__global__ __launch_bounds__(THREADS) void plan_kernel(PlanArgs a) {
  constexpr int MOST = THREADS * J;
  __shared__ uint32_t sums[5][THREADS / WAVE], s_ring[2];
  __shared__ __align__(16) int s_mark[THREADS][EACH];
  __shared__ int s_last[THREADS / WAVE];
  __shared__ int32_t s_take[MOST], s_give[MOST], s_row[MOST];
  const int tid = threadIdx.x, s0 = tid * J, n = a.n_seqs;
  const int room = a.max_pages * a.page_size;               // (at most 2^30)
  const int64_t head = a.counters[0], tail = a.counters[1], between = (int64_t)((uint64_t)tail - (uint64_t)head);
  const int free = between < 0 ? 0 : between > a.n_pages ? a.n_pages : (int)between;
  if (tid < 2) s_ring[tid] = (uint32_t)((uint64_t)(tid ? tail : head) % (uint32_t)a.n_pages);      // (one wave's long division, for all)
  int kept[J], wanted[J], have[J], reach[J];                // pages: what is held, and with what is wanted
  uint32_t ask[1] = {0}, need[1] = {0}, all[1];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int s = s0 + j;
    const bool there = s < n;
    const int held = there ? min(max(a.held[s], 0), room) : 0;
    kept[j] = there && a.kept ? min(max(a.kept[s], 0), held) : held;
    wanted[j] = there ? max(a.wanted[s], 0) : 0;
    if (wanted[j] > room - kept[j]) wanted[j] = 0;
    have[j] = pages_of(a, held);
    reach[j] = pages_of(a, kept[j] + wanted[j]);
    ask[0] += (uint32_t)min(wanted[j], a.n_rows + 1);
  }
  block_before<THREADS, 1>(ask, sums, all);
#pragma unroll
  for (int j = 0; j < J; ++j) {
    ask[0] += (uint32_t)min(wanted[j], a.n_rows + 1);
    if (ask[0] > (uint32_t)a.n_rows) wanted[j] = 0;
    need[0] += wanted[j] ? (uint32_t)max(reach[j] - have[j], 0) : 0u;
  }
  block_before<THREADS, 1>(need, sums + 1, all);
  uint32_t moved[3] = {0, 0, 0}, totals[3];                 // rows, pages taken, pages given back
  int want[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int more = wanted[j] ? max(reach[j] - have[j], 0) : 0;
    need[0] += (uint32_t)more;
    if (more > 0 && need[0] > (uint32_t)free) wanted[j] = 0;
    want[j] = wanted[j] ? reach[j] : pages_of(a, kept[j]);
    moved[0] += (uint32_t)wanted[j];
    moved[1] += (uint32_t)max(want[j] - have[j], 0);
    moved[2] += (uint32_t)max(have[j] - want[j], 0);
  }
  block_before<THREADS, 3>(moved, sums + 2, totals);
  const uint32_t all_rows = totals[0], all_take = totals[1], all_give = totals[2];
  int row0[J], rows[J], take0[J], take[J], give0[J], give[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int s = s0 + j;
    row0[j] = (int)moved[0]; rows[j] = wanted[j]; take0[j] = (int)moved[1]; take[j] = max(want[j] - have[j], 0); give0[j] = (int)moved[2]; give[j] = max(have[j] - want[j], 0);
    moved[0] += (uint32_t)rows[j]; moved[1] += (uint32_t)take[j]; moved[2] += (uint32_t)give[j];
    // where a sequence's numbers lie: page number i that is taken (or given back) is its place i - s_take (s_give), row r its position r + s_row
    s_take[s] = have[j] - take0[j]; s_give[s] = want[j] - give0[j]; s_row[s] = kept[j] - row0[j];
    if (s < n) { a.q_start[s] = row0[j]; a.kv_len[s] = kept[j] + wanted[j]; a.granted[s] = wanted[j]; }
  }
  if (tid == 0) a.q_start[n] = (int)all_rows;
  const uint32_t from = s_ring[0], to = s_ring[1];
  auto ring = [&](uint32_t first, uint32_t i) { const uint32_t x = first + i; return x >= (uint32_t)a.n_pages ? x - (uint32_t)a.n_pages : x; };      // i below n_pages
  // pages taken: number i of them comes from place head + i of the ring
  for (int i0 = 0; i0 < (int)all_take; i0 += EACH * THREADS) {
    int s[EACH], page[EACH];
    owners<THREADS, J>(take0, take, s0, i0, s_mark, s_last, s);
#pragma unroll
    for (int u = 0; u < EACH; ++u) page[u] = a.free_pages[ring(from, min((uint32_t)(i0 + EACH * tid + u), all_take - 1))];
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
      const int i = i0 + EACH * tid + u;
      if (i < (int)all_take) a.pages[(int64_t)s[u] * a.pages_stride + (i + s_take[s[u]])] = page[u];
    }
  }
  // pages given back, those that are some, in their order, behind what is free
  const uint32_t put_most = (uint32_t)(a.n_pages - free);
  uint32_t put = 0;
  for (int i0 = 0; i0 < (int)all_give; i0 += EACH * THREADS) {
    int s[EACH], page[EACH];
    owners<THREADS, J>(give0, give, s0, i0, s_mark, s_last, s);
    uint32_t some[1] = {0}, now[1];
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
      const int i = i0 + EACH * tid + u;
      page[u] = i < (int)all_give ? a.pages[(int64_t)s[u] * a.pages_stride + (i + s_give[s[u]])] : -1;
    }
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
      if ((unsigned)page[u] >= (unsigned)a.n_pages) page[u] = -1;
      some[0] += page[u] >= 0;
    }
    block_before<THREADS, 1>(some, sums, now);
    uint32_t at = put + some[0];
#pragma unroll
    for (int u = 0; u < EACH; ++u)
      if (page[u] >= 0) {
        if (at < put_most) a.free_pages[ring(to, at)] = page[u];
        ++at;
      }
    put = min(put + now[0], put_most);
  }
  if (tid == 0) { a.counters_out[0] = (int64_t)((uint64_t)head + all_take); a.counters_out[1] = (int64_t)((uint64_t)tail + put); }
  if (!a.rows_here) return;
  for (int i0 = 0; i0 < a.n_rows; i0 += EACH * THREADS) {
    int s[EACH];
    owners<THREADS, J>(row0, rows, s0, i0, s_mark, s_last, s);      // (the table is written behind its first barrier)
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
      const int row = i0 + EACH * tid + u;
      if (row < a.n_rows) place_row(a, row, row < (int)all_rows ? s[u] : -1, row < (int)all_rows ? row + s_row[s[u]] : 0);
    }
  }
}

// Many rows: 256 of them a workgroup.
constexpr int ROWS_A_GROUP = 256;
__global__ __launch_bounds__(256) void plan_rows_kernel(PlanArgs a) {
  __shared__ int32_t start[PPD_MAX_SEQS + 1];
  for (int i = threadIdx.x; i <= a.n_seqs; i += 256) start[i] = a.q_start[i];
  __syncthreads();
  const int row = blockIdx.x * ROWS_A_GROUP + threadIdx.x;
  if (row >= a.n_rows) return;
  const int s = row < start[a.n_seqs] ? last_upto(start, a.n_seqs, row) : -1;
  place_row(a, row, s, s < 0 ? 0 : a.kv_len[s] - (start[s + 1] - row));
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
                table->pages_stride, table->max_pages, table->n_pages, table->page_size, table->n_seqs, n_rows, false, Divider((uint32_t)table->page_size)};
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
