// ppd_adjust_logits: penalties for tokens that a text has, biases and masks on the logits of its rows.  Bound by reading and writing the
// logits once, see adjust_kernel; 115 fp32 rows of 50272 logits, 46 MB, take 15.8 us, 2.9 TB/s.
#include "ppd_layers_common.h"

using namespace ppd;

namespace {

constexpr int ADJUST_MAX_VOCAB = 1 << 24;
constexpr int AT = 256;                       // threads of a workgroup

struct AdjustArgs {
  const int32_t *row_start, *ids; const void* logits; void* out; int64_t stride, out_stride;
  ppd_logit_rules r;
  int n_seqs, n_rows, vocab, run;      // run: rows of a workgroup, as a power of two
  bool in_place;
};

template <typename T> struct Logits;          // VEC of them are 16 bytes
template <> struct Logits<float> {
  static constexpr int VEC = 4;
  typedef u32x4 loose __attribute__((aligned(4)));
  __device__ static __forceinline__ void wide(u32x4 r, float* f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(r[e]);
  }
  __device__ static __forceinline__ u32x4 narrow(const float* f) { return (u32x4){__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])}; }
};
template <typename T> struct Logits16 {
  static constexpr int VEC = 8;
  typedef u32x4 loose __attribute__((aligned(2)));
  __device__ static __forceinline__ void wide(u32x4 r, float* f) {
    const f32x4 a = Quad<T>::wide((u32x2){r.x, r.y}), b = Quad<T>::wide((u32x2){r.z, r.w});
#pragma unroll
    for (int e = 0; e < 4; ++e) { f[e] = a[e]; f[4 + e] = b[e]; }
  }
  __device__ static __forceinline__ u32x4 narrow(const float* f) {
    const u32x2 a = Quad<T>::narrow((f32x4){f[0], f[1], f[2], f[3]}), b = Quad<T>::narrow((f32x4){f[4], f[5], f[6], f[7]});
    return (u32x4){a.x, a.y, b.x, b.y};
  }
};
template <> struct Logits<bf16_t> : Logits16<bf16_t> {};
template <> struct Logits<f16_t> : Logits16<f16_t> {};

// A run's sequence, that one's rows, and which of its runs it is, LOOK sequences of a lane at a time; false: there are not so many.
template <int LOOK>
__device__ __forceinline__ bool find_run(const AdjustArgs& a, int idx, int lane, int& s, int& row0, int& rows, int& r) {
  auto start_of = [&](int t) { return min(max(a.row_start[min(t, a.n_seqs)], 0), a.n_rows); };
  int before = 0;
  for (int from = 0; from < a.n_seqs; from += LOOK * WAVE) {
    int lo[LOOK + 1], runs[LOOK], mine = 0;
#pragma unroll
    for (int j = 0; j <= LOOK; ++j) lo[j] = start_of(from + LOOK * lane + j);
#pragma unroll
    for (int j = 0; j < LOOK; ++j) { lo[j + 1] = max(lo[j + 1], lo[j]); runs[j] = (lo[j + 1] - lo[j] + (1 << a.run) - 1) >> a.run; mine += runs[j]; }
    const int upto = before + scan_up(mine);
    const unsigned long long past = __ballot(upto > idx);
    if (past) {
      const int w = __builtin_ctzll(past);
      int at = idx - (upto - mine), j0 = 0, l = lo[0], h = lo[1];
      bool there = false;
#pragma unroll
      for (int j = 0; j < LOOK; ++j) {
        if (there) continue;
        if (at < runs[j]) { there = true; j0 = j; l = lo[j]; h = lo[j + 1]; } else at -= runs[j];
      }
      s = from + LOOK * w + __builtin_amdgcn_readlane(j0, w);
      row0 = __builtin_amdgcn_readlane(l, w); rows = __builtin_amdgcn_readlane(h, w) - row0; r = __builtin_amdgcn_readlane(at, w);
      return true;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

// A workgroup has 16 bytes' worth of tokens of the vocabulary a thread, and a run of one sequence's rows.  It counts the text before them in LDS
// (additions of whole numbers, in any order), each thread takes the counts of its own tokens into registers, and from then on nothing crosses
// threads: a row's own token is counted by the thread that has it.  Rows follow each other; what hides their waits is the other workgroups on the unit
// (the next row's logits under way while one is worked on: 30.7 us, not 31.7, for 901 bf16 rows of 32000 logits, 115 MB; pieces of the vocabulary four
// times as large 34.9; five, three, two rows a run 33.7, 37.8, 40.0, as each reads the text anew.  A copy takes 25).
// Every wave counts the runs for itself: a workgroup has sixteen rows at most, however rows are spread over sequences (800 rows of
// one and one of each of 63 others 33 us, by equal shares for all 882), and none without a run lies between others.
// grid: (pieces of the vocabulary, runs of rows, and what is left of them)
template <typename T>
__global__ __launch_bounds__(AT) void adjust_kernel(AdjustArgs a) {
  constexpr int VEC = Logits<T>::VEC, SIZE = 16 / VEC, PIECE = AT * VEC;
  constexpr uint32_t IN_PROMPT = 1u << 31;
  typedef typename Logits<T>::loose loose;
  __shared__ __align__(16) uint32_t count[PIECE];
  __shared__ __align__(16) int entry[PIECE];              // the bias list's entry for a token, and one more; 0: none
  const int tid = threadIdx.x, lane = tid & 63, idx = blockIdx.z * gridDim.y + blockIdx.y, first_id = blockIdx.x * PIECE, first = first_id + tid * VEC;      // (of the workgroup's tokens, of the thread's)
  int s, row0, rows, r;
  if (!(a.n_seqs <= WAVE ? find_run<1>(a, idx, lane, s, row0, rows, r) : find_run<4>(a, idx, lane, s, row0, rows, r))) return;
  const int begin = r << a.run, end = min(begin + (1 << a.run), rows);
  const bool counts = a.r.repetition || a.r.presence || a.r.frequency;
  const int before = counts && a.r.history ? min(max(a.r.history_len[s], 0), (int)a.r.history_stride) : 0;
  const int prompt = a.r.prompt_len ? a.r.prompt_len[s] : 0;
  uint32_t n[VEC];
  float bias[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) { n[e] = 0; bias[e] = -0.0f; }      // (what added to a number leaves it as it is)
  if (counts || a.r.bias) {
#pragma unroll
    for (int e = 0; e < VEC; e += 4) {
      *(u32x4*)(count + tid * VEC + e) = (u32x4){0u, 0u, 0u, 0u};
      *(u32x4*)(entry + tid * VEC + e) = (u32x4){0u, 0u, 0u, 0u};
    }
    __syncthreads();
    auto add = [&](int token, int at) {
      const uint32_t t = (uint32_t)token - (uint32_t)first_id;
      if (t < (uint32_t)PIECE && token < a.vocab) { if (at < prompt) atomicOr(count + t, IN_PROMPT); else atomicAdd(count + t, 1u); }
    };
    auto scan = [&](const int32_t* text, int length, int at) {
      for (int i0 = tid; i0 < length; i0 += 8 * AT) {      // eight loads under way
        int token[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) token[u] = i0 + u * AT < length ? text[i0 + u * AT] : -1;
#pragma unroll
        for (int u = 0; u < 8; ++u) if (token[u] >= 0) add(token[u], at + i0 + u * AT);
      }
    };
    if (before > 0) scan(a.r.history + (int64_t)s * a.r.history_stride, before, 0);
    if (counts && a.ids) scan(a.ids + row0, begin, before);
    if (a.r.bias) {
      const int from = min(max(a.r.bias_start[s], 0), a.r.n_bias), to = min(a.r.bias_start[s + 1], a.r.n_bias);
      for (int e = from + tid; e < to; e += AT) {
        const int token = a.r.bias_ids[e];
        const uint32_t t = (uint32_t)token - (uint32_t)first_id;
        if (t < (uint32_t)PIECE && token >= 0 && token < a.vocab) atomicMax(entry + t, e + 1);
      }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      n[e] = count[tid * VEC + e];
      const int i = entry[tid * VEC + e];
      if (i > 0) bias[e] = a.r.bias[i - 1];
    }
  }
  const float again = a.r.repetition ? a.r.repetition[s] : 1.0f, factor = again > 0.f ? again : 1.0f, inverse = 1.0f / factor;
  const float once = a.r.presence ? a.r.presence[s] : 0.0f, each = a.r.frequency ? a.r.frequency[s] : 0.0f;
  bool touched = false;                                    // where nothing is done, and no mask, logits in place are neither read nor written
#pragma unroll
  for (int e = 0; e < VEC; ++e) touched |= n[e] != 0 || __float_as_uint(bias[e]) != 0x80000000u;
  for (int i = begin; i < end; ++i) {
    const int row = row0 + i;
    if (counts && a.ids) {
      const int token = a.ids[row];
      const uint32_t mine = (uint32_t)token - (uint32_t)first;
      if (token < a.vocab && mine < (uint32_t)VEC) {
        touched = true;
#pragma unroll
        for (int e = 0; e < VEC; ++e) if ((uint32_t)e == mine) n[e] = before + i < prompt ? n[e] | IN_PROMPT : n[e] + 1;
      }
    }
    const int which = a.r.mask ? a.r.mask_row[row] : -1;
    const uint32_t* const mask = (unsigned)which < (unsigned)a.r.n_masks ? a.r.mask + (int64_t)which * a.r.mask_stride : nullptr;
    if (first >= a.vocab || (a.in_place && !mask && !touched)) continue;
    const char* const src = (const char*)a.logits + ((int64_t)row * a.stride + first) * SIZE;
    char* const dst = (char*)a.out + ((int64_t)row * a.out_stride + first) * SIZE;
    const uint32_t allowed = mask ? mask[first / 32] >> first % 32 : ~0u;
    u32x4 raw = {0u, 0u, 0u, 0u};
    if (first + VEC <= a.vocab) raw = *(const loose*)src;
    else {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (first + e < a.vocab) {
          if constexpr (SIZE == 4) raw[e] = ((const uint32_t*)src)[e];
          else raw[e / 2] |= (uint32_t)((const uint16_t*)src)[e] << 16 * (e % 2);
        }
    }
    float x[VEC];
    Logits<T>::wide(raw, x);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const uint32_t said = n[e] & ~IN_PROMPT;
      const float y = x[e] * (x[e] > 0.f ? inverse : factor);
      x[e] = n[e] ? y : x[e];
      const float less = x[e] - (each * (float)said + once);
      x[e] = said ? less : x[e];
      x[e] += bias[e];
      x[e] = allowed >> e & 1 ? x[e] : -INFINITY;
    }
    const u32x4 now = Logits<T>::narrow(x);
    if (first + VEC <= a.vocab) *(loose*)dst = now;
    else {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (first + e < a.vocab) {
          if constexpr (SIZE == 4) ((uint32_t*)dst)[e] = now[e];
          else ((uint16_t*)dst)[e] = (uint16_t)(now[e / 2] >> 16 * (e % 2));
        }
    }
  }
}

template <typename T>
hipError_t adjust_go(AdjustArgs& a, hipStream_t stream) {
  const int64_t pieces = (a.vocab + AT * Logits<T>::VEC - 1) / (AT * Logits<T>::VEC), some = a.n_rows < a.n_seqs ? a.n_rows : a.n_seqs;
  a.run = 4;                                               // sixteen rows a run, or fewer where workgroups are few
  while (a.run > 0 && pieces * ((a.n_rows >> a.run) + some) < 512) --a.run;
  const int64_t runs = (a.n_rows >> a.run) + some;
  const int64_t side = runs < 32768 ? runs : 32768;        // (a grid's second size ends at 65535)
  hipLaunchKernelGGL((adjust_kernel<T>), dim3(pieces, side, (runs + side - 1) / side), dim3(AT), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

extern "C" int ppd_adjust_logits(int n_seqs, int n_rows, int vocab, int dtype, const int32_t* row_start, const int32_t* ids,
                                 const void* logits, int64_t logits_stride, void* out, int64_t out_stride,
                                 const ppd_logit_rules* rules, void* hip_stream) {
  if (n_seqs < 1 || n_rows < 0 || vocab < 1 || dtype < PPD_FP32 || dtype > PPD_FP16 || !rules) return PPD_EINVAL;
  if (n_seqs > PPD_MAX_SEQS || n_rows > PPD_MAX_TOKENS || vocab > ADJUST_MAX_VOCAB) return PPD_ELIMIT;
  const ppd_logit_rules& r = *rules;
  if (!r.history != !r.history_len || !r.bias != !r.bias_start || !r.bias != !r.bias_ids) return PPD_EINVAL;
  if (n_rows > 0 && (!logits || !out || !r.mask != !r.mask_row)) return PPD_EINVAL;      // (what has no rows has no address, either)
  if (((uintptr_t)row_start | (uintptr_t)ids | (uintptr_t)r.history | (uintptr_t)r.history_len | (uintptr_t)r.prompt_len | (uintptr_t)r.repetition |
       (uintptr_t)r.presence | (uintptr_t)r.frequency | (uintptr_t)r.bias_start | (uintptr_t)r.bias_ids | (uintptr_t)r.bias | (uintptr_t)r.mask |
       (uintptr_t)r.mask_row) & 3)
    return PPD_EINVAL;
  if (r.history && r.history_stride < 0) return PPD_EINVAL;
  if (r.history && r.history_stride > 1 << 30) return PPD_ELIMIT;
  if (r.bias && (r.n_bias < 0 || r.n_bias == INT32_MAX)) return PPD_EINVAL;
  if (r.mask && (r.n_masks < 0 || (r.n_masks > 1 && r.mask_stride < (vocab + 31) / 32))) return PPD_EINVAL;
  if (!row_start || ((uintptr_t)logits | (uintptr_t)out) & (elem_size(dtype) - 1)) return PPD_EINVAL;
  if (n_rows > 1 && (logits_stride < vocab || out_stride < vocab || (logits == out && logits_stride != out_stride))) return PPD_EINVAL;
  if (n_rows == 0) return PPD_OK;
  AdjustArgs a = {row_start, ids, logits, out, logits_stride, out_stride, r, n_seqs, n_rows, vocab, 0, logits == out};
  hipStream_t st = (hipStream_t)hip_stream;
  return launched(dtype == PPD_FP32 ? adjust_go<float>(a, st) : dtype == PPD_BF16 ? adjust_go<bf16_t>(a, st) : adjust_go<f16_t>(a, st));
}
