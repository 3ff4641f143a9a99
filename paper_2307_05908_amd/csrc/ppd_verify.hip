// ppd_verify_drafts: drafted tokens against the target model's logits, from given random numbers.
//
// Which token a random number falls on is decided by sums over the whole vocabulary, so that weights exp((z - max) / t) and their sums are
// fp64: in fp32 a border of the cumulative sum lies off by 1e-8 and more, and one draw in some thousands would differ from the rule.
// Two launches: maxima and sums of all rows by chunks (every logit read once), then, per sequence, which drafts are taken, and the draw at
// the row that ends it: one more look at that row where a residual max(p - q, 0) has to be summed.
#include "ppd_layers_common.h"

#include <math.h>

using namespace ppd;

namespace {

constexpr int VERIFY_MAX_VOCAB = 1 << 24;
constexpr int VT = 256;                       // threads of a workgroup
constexpr int PER = 16;                       // logits of a thread
constexpr int CHUNK = VT * PER;               // of a workgroup

struct RowPart { double sum; float top; int arg; };      // of a chunk: the weights' sum relative to top, the largest logit, its lowest id

struct VerifyArgs {
  const int32_t *row_start, *ids; const void *target, *draft; int64_t target_stride, draft_stride;
  const float *temperature, *uniform; int32_t *tokens, *accepted;
  int n_seqs, n_rows, vocab, chunks;
  RowPart* parts;          // [2 (target, draft)][n_rows][chunks]
  double* left;            // [n_seqs][chunks]: sums of the residual
  unsigned* done;          // [n_seqs]: workgroups of a sequence that have left theirs (set to zero by the first launch)
};

template <typename T> struct Logits;
template <> struct Logits<float> {
  static constexpr int VEC = 4;
  typedef u32x4 loose __attribute__((aligned(4)));
  __device__ static __forceinline__ float one(const void* p, int64_t i) { return ((const float*)p)[i]; }
  __device__ static __forceinline__ void wide(u32x4 r, float* f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(r[e]);
  }
};
template <> struct Logits<bf16_t> {
  static constexpr int VEC = 8;
  typedef u32x4 loose __attribute__((aligned(2)));
  __device__ static __forceinline__ float one(const void* p, int64_t i) { return bf16_to_f32(((const uint16_t*)p)[i]); }
  __device__ static __forceinline__ void wide(u32x4 r, float* f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) { f[2 * e] = __uint_as_float(r[e] << 16); f[2 * e + 1] = __uint_as_float(r[e] & 0xffff0000u); }
  }
};
template <> struct Logits<f16_t> {
  static constexpr int VEC = 8;
  typedef u32x4 loose __attribute__((aligned(2)));
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
  __device__ static __forceinline__ float one(const void* p, int64_t i) { return (float)((const _Float16*)p)[i]; }
  __device__ static __forceinline__ void wide(u32x4 r, float* f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) { const uint32_t x = r[e]; const h2 h = __builtin_bit_cast(h2, x); f[2 * e] = (float)h.x; f[2 * e + 1] = (float)h.y; }
  }
};
// NaN counts as -inf, and +inf as the largest number: where there is one, nothing else has a weight
__device__ __forceinline__ float usable(float z) { return fminf(fmaxf(z, -INFINITY), 3.40282347e38f); }
template <typename T> __device__ __forceinline__ float logit(const void* p, int64_t i) { return usable(Logits<T>::one(p, i)); }

// A thread's logits of a chunk: PER / VEC runs of VEC, run v of thread t at (v * VT + t) * VEC.  What lies behind the row: -inf.
// Rows begin at any multiple of the type's size.
template <typename T>
__device__ __forceinline__ void load_chunk(const void* p, int64_t row, int chunk, int vocab, float (&z)[PER]) {
  constexpr int VEC = Logits<T>::VEC;
  typedef typename Logits<T>::loose loose;
  const char* base = (const char*)p + row * (16 / VEC);
#pragma unroll
  for (int v = 0; v < PER / VEC; ++v) {
    const int j = chunk * CHUNK + (v * VT + (int)threadIdx.x) * VEC;
    if (j + VEC <= vocab) Logits<T>::wide(*(const loose*)(base + (int64_t)j * (16 / VEC)), z + v * VEC);
    else
#pragma unroll
      for (int e = 0; e < VEC; ++e) z[v * VEC + e] = j + e < vocab ? Logits<T>::one(base, j + e) : -INFINITY;
  }
#pragma unroll
  for (int e = 0; e < PER; ++e) z[e] = usable(z[e]);
}
__device__ __forceinline__ int id_of(int chunk, int e, int vec) { return chunk * CHUNK + (e / vec * VT + (int)threadIdx.x) * vec + e % vec; }

// exp((z - top) / t), relative error below 2^-43: 2^(y / 64) with y = (z - top) * 64 log2(e) / t, its nearest whole number k from a table
// of 2^(i / 64) and the exponent, the rest (at most a half) by the exponential's series to the fourth power.  -inf, and what is 64000
// and more below (2^-1000): exactly 0.  (Where all of a row is -inf the difference is no number, and that is less than anything, too.)
struct Weigh {
  double scale, top;
  const double* table;
  __device__ __forceinline__ Weigh(float top_, double t, const double* table_) : scale(92.332482616893657 / t), top(top_), table(table_) {}
  __device__ __forceinline__ double operator()(float z) const {
    constexpr double L = 0.010830424696249145, magic = 6755399441055744.0;      // ln 2 / 64; 1.5 * 2^52
    const double y = fmax(((double)z - top) * scale, -128000.0), shifted = y + magic, r = y - (shifted - magic);
    const int k = __double2loint(shifted);
    const double p = fma(r, fma(r, fma(r, fma(r, L * L * L * L / 24, L * L * L / 6), L * L / 2), L), 1.0) * table[k & 63];
    return ldexp(p, k >> 6);
  }
};
__device__ __forceinline__ void fill_table(double* table) { if (threadIdx.x < 64) table[threadIdx.x] = exp2(threadIdx.x * 0.015625); }

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, WAVE);
  return v;
}
__device__ __forceinline__ double temperature_of(const VerifyArgs& a, int s) { return a.temperature ? (double)a.temperature[s] : 1.0; }

// ---- all rows: the largest logit and the weights' sum, chunk by chunk.  grid: (n_rows * chunks, 1 or 2: target, draft)
template <typename T>
__global__ __launch_bounds__(VT) void verify_rows_kernel(VerifyArgs a) {
  constexpr int VEC = Logits<T>::VEC;
  __shared__ double table[64], ds[4];
  __shared__ float fs[4]; __shared__ int is[4];
  const int chunk = blockIdx.x % a.chunks, row = blockIdx.x / a.chunks, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool draft = blockIdx.y == 1;
  if (chunk == 0 && row == 0 && !draft) for (int i = tid; i < a.n_seqs; i += VT) a.done[i] = 0;
  float z[PER];
  if (!draft) load_chunk<T>(a.target, row * a.target_stride, chunk, a.vocab, z);         // (under way while the row's sequence is looked for)
  Batch b = {};
  b.q_start = a.row_start; b.n_seqs = a.n_seqs;
  const int s = seq_of_row(b, row, lane);
  if (s < 0) return;
  const double t = temperature_of(a, s);
  const bool by_max = !(t > 0.0);
  if (draft) {
    if (by_max || row + 1 >= min(a.row_start[s + 1], a.n_rows)) return;                  // rows that nothing asks for
    load_chunk<T>(a.draft, row * a.draft_stride, chunk, a.vocab, z);
  }
  fill_table(table);
  float top = -INFINITY; int arg = 0x7fffffff;
  if (by_max) {
#pragma unroll
    for (int e = 0; e < PER; ++e) if (z[e] > top) { top = z[e]; arg = id_of(chunk, e, VEC); }
    wave_best(top, arg);
  } else {
#pragma unroll
    for (int e = 0; e < PER; ++e) top = fmaxf(top, z[e]);
    top = wave_max(top);
    arg = top > -INFINITY ? chunk * CHUNK : 0x7fffffff;                                  // (only whether there is one is asked)
  }
  if (lane == 0) { fs[wave] = top; is[wave] = arg; }
  __syncthreads();
  top = fs[0]; arg = is[0];
#pragma unroll
  for (int w = 1; w < 4; ++w) if (better(fs[w], is[w], top, arg)) { top = fs[w]; arg = is[w]; }
  double sum = 0.0;
  if (!by_max) {
    const Weigh weigh(top, t, table);
#pragma unroll
    for (int e = 0; e < PER; ++e) sum += weigh(z[e]);
    sum = wave_sum_f64(sum);
    if (lane == 0) ds[wave] = sum;
    __syncthreads();
    sum = ((ds[0] + ds[1]) + ds[2]) + ds[3];
  }
  if (tid == 0) a.parts[((int64_t)(draft ? a.n_rows : 0) + row) * a.chunks + chunk] = {sum, top, arg};
}

// ---- which drafts are taken, and the draw.  grid: (chunks, n_seqs)
struct Row { float top; int arg; double sum; };
// a row's parts joined by 16 lanes, in all of them
__device__ __forceinline__ Row join_row(const RowPart* p, int chunks, double t, bool by_max, const double* table) {
  const int l = threadIdx.x & 15;
  Row r = {-INFINITY, 0x7fffffff, 0.0};
  for (int c = l; c < chunks; c += 16) { const float v = p[c].top; const int i = p[c].arg; if (better(v, i, r.top, r.arg)) { r.top = v; r.arg = i; } }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) {
    const float v = __shfl_xor(r.top, o, WAVE); const int i = __shfl_xor(r.arg, o, WAVE);
    if (better(v, i, r.top, r.arg)) { r.top = v; r.arg = i; }
  }
  if (!by_max) {
    const Weigh weigh(r.top, t, table);
    for (int c = l; c < chunks; c += 16) r.sum += p[c].sum * weigh(p[c].top);
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) r.sum += __shfl_xor(r.sum, o, WAVE);
  }
  return r;
}

template <typename T>
__global__ __launch_bounds__(VT) void verify_draw_kernel(VerifyArgs a) {
  constexpr int VEC = Logits<T>::VEC, RUNS = PER / VEC;
  __shared__ double table[64], seg[RUNS * 4], ds[4], chunk_sum[VT];
  __shared__ int s_end, s_last, s_token;
  __shared__ Row s_p, s_q;
  const int chunk = blockIdx.x, s = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int lo = min(max(a.row_start[s], 0), a.n_rows), hi = min(max(a.row_start[s + 1], lo), a.n_rows);
  if (lo == hi) {
    if (chunk == 0 && tid == 0) a.accepted[s] = 0;
    return;
  }
  const double t = temperature_of(a, s);
  const bool by_max = !(t > 0.0);
  fill_table(table);
  if (tid == 0) s_end = hi;
  __syncthreads();
  // 16 rows at a time until one ends the sequence
  for (int r0 = lo; r0 < hi; r0 += 16) {
    const int r = r0 + (tid >> 4);
    const bool in = r < hi, last = r + 1 >= hi;
    const int rc = in ? r : hi - 1;
    const Row p = join_row(a.parts + (int64_t)rc * a.chunks, a.chunks, t, by_max, table);
    const int d = last ? -1 : a.ids[rc + 1];
    const bool real = (unsigned)d < (unsigned)a.vocab;
    Row q = {0.f, 0, 0.0};
    bool take = false;
    if (by_max) take = real && d == p.arg && p.top > -INFINITY;
    else {
      if (!last && a.draft) q = join_row(a.parts + ((int64_t)a.n_rows + rc) * a.chunks, a.chunks, t, false, table);
      if (real) {
        const double pd = p.sum > 0.0 ? Weigh(p.top, t, table)(logit<T>(a.target, rc * a.target_stride + d)) / p.sum : 0.0;
        const double qd = !a.draft ? 1.0 : q.sum > 0.0 ? Weigh(q.top, t, table)(logit<T>(a.draft, rc * a.draft_stride + d)) / q.sum : 0.0;
        take = (double)a.uniform[2 * (int64_t)rc] * qd < pd;
      }
    }
    if (in && !take && (tid & 15) == 0) atomicMin(&s_end, r);
    __syncthreads();
    const bool ended = s_end < hi;
    if (in && r == s_end && (tid & 15) == 0) { s_p = p; s_q = q; }
    __syncthreads();
    if (ended) break;
  }
  const int end = s_end;                       // (the last row never takes a draft: every sequence ends)
  const Row p = s_p, q = s_q;
  const bool last = end + 1 >= hi;
  const int d = last ? -1 : a.ids[end + 1];
  auto finish = [&](int token) {
    for (int i = lo + tid; i < hi; i += VT) a.tokens[i] = i < end ? a.ids[i + 1] : i == end ? token : -1;
    if (tid == 0) a.accepted[s] = end - lo;
  };
  if (by_max || !(p.sum > 0.0)) {
    if (chunk == 0) finish(p.arg != 0x7fffffff ? p.arg : 0);
    return;
  }
  const bool residual = !last && (a.draft ? q.sum > 0.0 : (unsigned)d < (unsigned)a.vocab);
  const Weigh wp(p.top, t, table), wq(q.top, t, table);
  const double ip = 1.0 / p.sum, iq = q.sum > 0.0 ? 1.0 / q.sum : 0.0;
  // the weights that the draw goes by, of a thread's logits of chunk c
  auto weights = [&](int c, bool rest, double (&w)[PER]) {
    float z[PER], y[PER];
    load_chunk<T>(a.target, end * a.target_stride, c, a.vocab, z);
    if (rest && a.draft) load_chunk<T>(a.draft, end * a.draft_stride, c, a.vocab, y);
#pragma unroll
    for (int e = 0; e < PER; ++e) w[e] = wp(z[e]) * ip;
    if (!rest) return;
    if (a.draft) {
#pragma unroll
      for (int e = 0; e < PER; ++e) w[e] = fmax(w[e] - wq(y[e]) * iq, 0.0);
    } else {
#pragma unroll
      for (int e = 0; e < PER; ++e) if (id_of(c, e, VEC) == d) w[e] = fmax(w[e] - 1.0, 0.0);
    }
  };
  double w[PER];
  if (residual) {
    weights(chunk, true, w);
    double sum = 0.0;
#pragma unroll
    for (int e = 0; e < PER; ++e) sum += w[e];
    sum = wave_sum_f64(sum);
    if (lane == 0) ds[wave] = sum;
    __syncthreads();
    if (tid == 0) {
      __hip_atomic_store(a.left + (int64_t)s * a.chunks + chunk, ((ds[0] + ds[1]) + ds[2]) + ds[3], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      s_last = __hip_atomic_fetch_add(a.done + s, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
    }
    __syncthreads();
    if (!s_last) return;
  } else if (chunk != 0) return;
  // one workgroup is left of the sequence's: the chunk that the number falls into, then the run of a wave's logits in it, the lane, the logit
  const double u = a.uniform[2 * (int64_t)end + 1];
  double total = 0.0;
  bool rest = residual;
  auto part = [&](int c) {
    return rest ? __hip_atomic_load(a.left + (int64_t)s * a.chunks + c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)
                : a.parts[(int64_t)end * a.chunks + c].sum * wp(a.parts[(int64_t)end * a.chunks + c].top) * ip;
  };
  // (all chunks' parts by all threads, 256 at a time, and then in their order; chunks of more than 2^20 tokens come in several turns)
  auto walk = [&](auto&& each) {
    for (int c0 = 0; c0 < a.chunks; c0 += VT) {
      __syncthreads();
      if (c0 + tid < a.chunks) chunk_sum[tid] = part(c0 + tid);
      __syncthreads();
      const int n = min(VT, a.chunks - c0);
      for (int i = 0; i < n; ++i) if (each(c0 + i, chunk_sum[i])) return;
    }
  };
  auto add = [&](int, double x) { total += x; return false; };
  walk(add);
  if (rest && !(total > 0.0)) {                 // p and q are the same: from p
    rest = false;
    total = 0.0;
    walk(add);
  }
  const double aim = u * total;
  double before = 0.0, upto = 0.0;
  int pick = 0;
  walk([&](int c, double x) {
    if (x > 0.0) { pick = c; before = upto; }
    upto += x;
    return x > 0.0 && upto > aim;               // (else the last one that holds anything: sums in another order may fall short of the aim)
  });
  weights(pick, rest, w);
  double mine[RUNS];
#pragma unroll
  for (int v = 0; v < RUNS; ++v) {
    mine[v] = 0.0;
#pragma unroll
    for (int e = 0; e < VEC; ++e) mine[v] += w[v * VEC + e];
    const double x = wave_sum_f64(mine[v]);
    if (lane == 0) seg[v * 4 + wave] = x;
  }
  if (tid == 0) s_token = 0;
  __syncthreads();
  upto = before;
  int at = -1;
#pragma unroll
  for (int i = 0; i < RUNS * 4; ++i) {
    const double x = seg[i];
    if (x > 0.0 && (at < 0 || !(upto > aim))) { at = i; before = upto; }
    if (at < 0 || !(upto > aim)) upto += x;
  }
  if (at >= 0 && (at & 3) == wave) {
    double x = 0.0;
#pragma unroll
    for (int v = 0; v < RUNS; ++v) if (v == at >> 2) x = mine[v];
    double up = x;
#pragma unroll
    for (int o = 1; o < WAVE; o <<= 1) { const double y = __shfl_up(up, o, WAVE); if (lane >= o) up += y; }
    const unsigned long long some = __ballot(x > 0.0), past = __ballot(x > 0.0 && before + up > aim);
    const int who = past ? __builtin_ctzll(past) : some ? 63 - __builtin_clzll(some) : -1;
    if (lane == who) {
      double run = before + (up - x);
      int token = 0;
      bool found = false;
#pragma unroll
      for (int v = 0; v < RUNS; ++v)
        if (v == at >> 2)
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const double y = w[v * VEC + e];
            if (!found && y > 0.0) { token = id_of(pick, v * VEC + e, VEC); run += y; found = run > aim; }
          }
      s_token = token;
    }
  }
  __syncthreads();
  finish(s_token);
}

struct VerifyPlan { int chunks; uint64_t part_bytes, left_bytes, done_bytes; };

int check_verify(int n_seqs, int n_rows, int vocab, int dtype, VerifyPlan* p) {
  if (n_seqs < 1 || n_rows < 0 || vocab < 1 || dtype < PPD_FP32 || dtype > PPD_FP16) return PPD_EINVAL;
  if (n_seqs > PPD_MAX_SEQS || n_rows > PPD_MAX_TOKENS || vocab > VERIFY_MAX_VOCAB) return PPD_ELIMIT;
  p->chunks = (vocab + CHUNK - 1) / CHUNK;
  if ((int64_t)n_rows * p->chunks > 1 << 23) return PPD_ELIMIT;
  p->part_bytes = (uint64_t)2 * n_rows * p->chunks * sizeof(RowPart);
  p->left_bytes = (uint64_t)n_seqs * p->chunks * sizeof(double);
  p->done_bytes = (uint64_t)n_seqs * sizeof(unsigned);
  return PPD_OK;
}

template <typename T>
hipError_t verify_go(const VerifyArgs& a, hipStream_t st) {
  if (a.n_rows > 0) {
    hipLaunchKernelGGL(verify_rows_kernel<T>, dim3(a.n_rows * a.chunks, a.draft ? 2 : 1), dim3(VT), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(verify_draw_kernel<T>, dim3(a.chunks, a.n_seqs), dim3(VT), 0, st, a);
  return hipGetLastError();
}

}  // namespace

extern "C" int ppd_verify_drafts_workspace(int n_seqs, int n_rows, int vocab, int dtype, uint64_t* bytes) {
  VerifyPlan p;
  const int rc = check_verify(n_seqs, n_rows, vocab, dtype, &p);
  if (rc) return rc;
  if (!bytes) return PPD_EINVAL;
  *bytes = p.part_bytes + p.left_bytes + p.done_bytes;
  return PPD_OK;
}

extern "C" int ppd_verify_drafts(int n_seqs, int n_rows, int vocab, int dtype, const int32_t* row_start, const int32_t* ids,
                                 const void* target_logits, int64_t target_stride, const void* draft_logits, int64_t draft_stride,
                                 const float* temperature, const float* uniform, int32_t* tokens, int32_t* accepted,
                                 void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  VerifyPlan p;
  const int rc = check_verify(n_seqs, n_rows, vocab, dtype, &p);
  if (rc) return rc;
  if (!row_start || !accepted || (n_rows > 0 && (!ids || !target_logits || !uniform || !tokens))) return PPD_EINVAL;
  if (n_rows > 1 && (target_stride < vocab || (draft_logits && draft_stride < vocab))) return PPD_EINVAL;
  const uintptr_t words = (uintptr_t)row_start | (uintptr_t)ids | (uintptr_t)temperature | (uintptr_t)uniform | (uintptr_t)tokens | (uintptr_t)accepted;
  if ((words & 3) || (((uintptr_t)target_logits | (uintptr_t)draft_logits) & (elem_size(dtype) - 1))) return PPD_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < p.part_bytes + p.left_bytes + p.done_bytes) return PPD_EINVAL;
  VerifyArgs a = {row_start, ids, target_logits, draft_logits, target_stride, draft_stride, temperature, uniform, tokens, accepted, n_seqs, n_rows, vocab, p.chunks,
                  (RowPart*)workspace, (double*)((char*)workspace + p.part_bytes), (unsigned*)((char*)workspace + p.part_bytes + p.left_bytes)};
  hipStream_t st = (hipStream_t)hip_stream;
  return launched(dtype == PPD_FP32 ? verify_go<float>(a, st) : dtype == PPD_BF16 ? verify_go<bf16_t>(a, st) : verify_go<f16_t>(a, st));
}
