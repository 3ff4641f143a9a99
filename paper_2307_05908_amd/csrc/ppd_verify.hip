// ppd_verify_drafts: drafted tokens against the target model's logits, from given random numbers.
//
// Which token a random number falls on is decided by sums over the whole vocabulary, so that weights exp((z - max) / t) and their sums are
// fp64: in fp32 a border of the cumulative sum lies off by 1e-8 and more, and one draw in some thousands would differ from the rule.
// Two launches: maxima and sums of all rows by pieces (every logit read once), then, per sequence, which drafts are taken, and the draw at
// the row that ends it: one more look at that row where a residual max(p - q, 0) has to be summed.
#include "ppd_layers_common.h"

#include <math.h>

using namespace ppd;

namespace {

constexpr int VERIFY_MAX_VOCAB = 1 << 24;
constexpr int VT = 256;                       // threads of a workgroup
constexpr int PER = 16;                       // logits of a thread
constexpr int PIECE = WAVE * PER;             // of a wave
constexpr int CHUNK = VT * PER;               // of a workgroup

struct RowPart { double sum; float top; int arg; };      // of a piece: the weights' sum relative to top, the largest logit, its lowest id

struct VerifyArgs {
  const int32_t *row_start, *ids; const void *target, *draft; int64_t target_stride, draft_stride;
  const float *temperature, *uniform; int32_t *tokens, *accepted;
  int n_seqs, n_rows, vocab, chunks, pieces;
  int run;                 // pieces that a wave of the first launch takes in turn
  RowPart* parts;          // [2 (target, draft)][n_rows][pieces]
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

// A lane's logits of a piece: PER / VEC runs of VEC, run v of lane l at (v * 64 + l) * VEC.  What lies behind the row: -inf.  Rows begin at
// any multiple of the type's size.
template <typename T>
__device__ __forceinline__ void load_piece(const void* p, int64_t row, int piece, int vocab, int lane, float (&z)[PER]) {
  constexpr int VEC = Logits<T>::VEC;
  typedef typename Logits<T>::loose loose;
  const char* base = (const char*)p + row * (16 / VEC);
  if ((piece + 1) * PIECE <= vocab) {
#pragma unroll
    for (int v = 0; v < PER / VEC; ++v) Logits<T>::wide(*(const loose*)(base + (int64_t)(piece * PIECE + (v * WAVE + lane) * VEC) * (16 / VEC)), z + v * VEC);
  } else {
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int j = piece * PIECE + (e / VEC * WAVE + lane) * VEC + e % VEC;
      z[e] = j < vocab ? Logits<T>::one(base, j) : -INFINITY;
    }
  }
}
__device__ __forceinline__ int id_of(int piece, int e, int vec, int lane) { return piece * PIECE + (e / vec * WAVE + lane) * vec + e % vec; }

// exp((z - top) / t), relative error below 2^-42: 2^(y / 256) with y = (z - top) * 256 log2(e) / t, its nearest whole number k from a table
// of 2^(i / 256) and the exponent, the rest (at most a half) by the exponential's series to the third power.  -inf, and all that is further
// down, comes as 2^-1000, which counts as nothing wherever a weight is looked at by itself (some), and is nothing in a sum beside the
// largest logit's 1.  The table's entries have i << 12 taken off their upper words, so that k << 12 puts the exponent there and leaves the
// rest.  Twelve instructions: these weights, not the reading of the logits, are what the launch takes its time for.
constexpr double SOME = 0x1p-900;
constexpr int STEPS = 256;
struct Weigh {
  double scale, top, least;
  const double* table;
  __device__ __forceinline__ Weigh(float top_, double t, const double* table_) : scale(369.32993046757463 / t), top(top_), least(-693.0 * t), table(table_) {}
  __device__ __forceinline__ double series(float z, double& power) const {
    constexpr double L = 0.0027076061740622863, magic = 6755399441055744.0;      // ln 2 / 256; 1.5 * 2^52
    const double d = fmax((double)z - top, least), shifted = fma(d, scale, magic), r = fma(d, scale, magic - shifted);
    const int k = __double2loint(shifted);
    const double entry = table[k & (STEPS - 1)];
    power = __hiloint2double(__double2hiint(entry) + (k << 12), __double2loint(entry));
    return fma(r, fma(r, fma(r, L * L * L / 6, L * L / 2), L), 1.0);
  }
  __device__ __forceinline__ double operator()(float z) const { double power; const double p = series(z, power); return p * power; }
  __device__ __forceinline__ void add(float z, double& sum) const { double power; const double p = series(z, power); sum = fma(p, power, sum); }
  __device__ __forceinline__ double some(float z) const { const double p = (*this)(z); return p > SOME ? p : 0.0; }
};
// 2^(i / 256) by the bits of i
__device__ __forceinline__ void fill_table(double* table) {
  static_assert(STEPS == VT, "an entry a thread");
  const int i = threadIdx.x;
  const double f[8] = {1.0027112750502025, 1.0054299011128027, 1.0108892860517005, 1.0218971486541166, 1.0442737824274138, 1.0905077326652577, 1.189207115002721, 1.4142135623730951};
  double p = 1.0;
#pragma unroll
  for (int b = 0; b < 8; ++b) p *= i >> b & 1 ? f[b] : 1.0;
  table[i] = __hiloint2double(__double2hiint(p) - (i << 12), __double2loint(p));
}

template <int CTRL> __device__ __forceinline__ double dpp_f64(double v) {
  return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xf, 0xf, false), __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ double lane_f64(double v, int l) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), l), __builtin_amdgcn_readlane(__double2loint(v), l));
}
__device__ __forceinline__ double row_sum_f64(double v) {      // over 16 lanes, the same in all of them
  v += dpp_f64<0xB1>(v);
  v += dpp_f64<0x4E>(v);
  v += dpp_f64<0x141>(v);
  return v + dpp_f64<0x140>(v);
}
__device__ __forceinline__ double wave_sum_f64(double v) {
  v = row_sum_f64(v);
  return ((lane_f64(v, 0) + lane_f64(v, 16)) + lane_f64(v, 32)) + lane_f64(v, 48);
}
__device__ __forceinline__ double scan_f64(double v, int lane) {
#pragma unroll
  for (int o = 1; o < WAVE; o <<= 1) { const double y = __shfl_up(v, o, WAVE); if (lane >= o) v += y; }
  return v;
}
__device__ __forceinline__ double temperature_of(const VerifyArgs& a, int s) {
  const float t = a.temperature ? a.temperature[s] : 1.0f;
  return t > 3.40282347e38f ? 3.40282347e38 : (double)t;             // (infinite: as the largest number)
}

// ---- all rows: the largest logit and the weights' sum, piece by piece.  A wave has `run` pieces of a row, and the next one's logits under way
// while it works on one; nothing waits for another wave but for the table.  Bound by the vector units: 20 instructions a logit, 12 of them for
// its weight (901 bf16 rows of 32000 logits and 773 of drafts', 107 MB: 41 us, 65 % of the cycles with such an instruction under way; reading
// alone would take 15).  Neither fewer instructions (one maximum for eight pieces: 17 a logit), nor more waves, nor four weights side by side in
// each changed that time by more than 5 %.  grid: (runs of all rows / 4, 1 or 2: target, draft)
template <typename T>
__global__ __launch_bounds__(VT, 6) void verify_rows_kernel(VerifyArgs a) {
  constexpr int VEC = Logits<T>::VEC;
  __shared__ double table[STEPS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool draft = blockIdx.y == 1;
  if (blockIdx.x == 0 && !draft) for (int i = tid; i < a.n_seqs; i += VT) a.done[i] = 0;
  fill_table(table);
  __syncthreads();
  const int runs = (a.pieces + a.run - 1) / a.run, at = blockIdx.x * 4 + wave, row = at / runs, first = at % runs * a.run, end = min(first + a.run, a.pieces);
  if (row >= a.n_rows) return;
  const void* const src = draft ? a.draft : a.target;
  const int64_t from = row * (draft ? a.draft_stride : a.target_stride);
  float z[PER], next[PER];
  if (!draft) load_piece<T>(src, from, first, a.vocab, lane, z);         // (under way while the row's sequence is looked for)
  Batch b = {};
  b.q_start = a.row_start; b.n_seqs = a.n_seqs;
  const int s = seq_of_row(b, row, lane);
  if (s < 0) return;
  const double t = temperature_of(a, s);
  const bool by_max = !(t > 0.0);
  if (draft) {
    if (by_max || row + 1 >= min(a.row_start[s + 1], a.n_rows)) return;                  // rows that nothing asks for
    load_piece<T>(src, from, first, a.vocab, lane, z);
  }
  RowPart* const out = a.parts + ((int64_t)(draft ? a.n_rows : 0) + row) * a.pieces;
  for (int piece = first; piece < end; ++piece) {
    if (piece + 1 < end) load_piece<T>(src, from, piece + 1, a.vocab, lane, next);
    float top = -INFINITY; int arg = 0x7fffffff;
    double sum = 0.0;
    if (by_max) {
#pragma unroll
      for (int e = 0; e < PER; ++e) { const float x = usable(z[e]); if (x > top) { top = x; arg = id_of(piece, e, VEC, lane); } }
      wave_best(top, arg);
    } else {
#pragma unroll
      for (int e = 0; e < PER; ++e) top = fmaxf(top, z[e]);              // (no NaN comes out)
      top = wave_max(top);
      if (top == INFINITY) {
        top = usable(top);
#pragma unroll
        for (int e = 0; e < PER; ++e) z[e] = usable(z[e]);
      }
      arg = top > -INFINITY ? piece * PIECE : 0x7fffffff;                // (only whether there is one is asked)
      const Weigh weigh(top, t, table);
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        weigh.add(z[e], sum);
        if (e % 4 == 3) { asm volatile("" : "+v"(sum)); __builtin_amdgcn_sched_barrier(0); }      // (four at a time: sixteen take 144 registers)
      }
      sum = top > -INFINITY ? wave_sum_f64(sum) : 0.0;
    }
    if (lane == 0) out[piece] = {sum, top, arg};
#pragma unroll
    for (int e = 0; e < PER; ++e) z[e] = next[e];
  }
}

// ---- which drafts are taken, and the draw.  Bound by a chain of lookups: the rows' pieces, the logits of the row that ends the sequence, the
// residual's sums, the piece that the number falls into (24 sequences of 50272 logits: 12 us; 128 of 32000: 19).  Every workgroup of a
// sequence finds that row for itself; the one that leaves its sum last draws.  grid: (chunks, n_seqs)
struct Row { float top; int arg; double sum; };
// A row's pieces joined by 16 lanes, in all of them.  The first 64 pieces come in one go (before anything waits for them), the others in turn.
struct First { RowPart x[4]; };
__device__ __forceinline__ First first_parts(const RowPart* p, int pieces) {
  First f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = (threadIdx.x & 15) + 16 * i;
    f.x[i] = {0.0, -INFINITY, 0x7fffffff};
    if (c < pieces) f.x[i] = p[c];
  }
  return f;
}
__device__ __forceinline__ Row join_row(const First& f, const RowPart* p, int pieces, double t, bool by_max, const double* table) {
  const int l = threadIdx.x & 15;
  Row r = {-INFINITY, 0x7fffffff, 0.0};
  auto larger = [&](float v, int i) { if (better(v, i, r.top, r.arg)) { r.top = v; r.arg = i; } };
#pragma unroll
  for (int i = 0; i < 4; ++i) larger(f.x[i].top, f.x[i].arg);
  for (int c = l + 64; c < pieces; c += 16) larger(p[c].top, p[c].arg);
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) larger(__shfl_xor(r.top, o, WAVE), __shfl_xor(r.arg, o, WAVE));
  if (!by_max) {
    const Weigh weigh(r.top, t, table);
#pragma unroll
    for (int i = 0; i < 4; ++i) r.sum += f.x[i].sum * weigh(f.x[i].top);
    for (int c = l + 64; c < pieces; c += 16) r.sum += p[c].sum * weigh(p[c].top);
    r.sum = row_sum_f64(r.sum);
  }
  return r;
}

template <typename T>
__global__ __launch_bounds__(VT) void verify_draw_kernel(VerifyArgs a) {
  constexpr int VEC = Logits<T>::VEC, RUNS = PER / VEC;
  __shared__ double table[STEPS], ds[4];
  __shared__ int s_end, s_last;
  __shared__ Row s_p, s_q;
  const int chunk = blockIdx.x, s = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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
    const int d = last ? -1 : a.ids[rc + 1];
    const bool real = (unsigned)d < (unsigned)a.vocab;
    float zd = -INFINITY, yd = -INFINITY, u = 0.f;
    if (real && !by_max) {
      zd = logit<T>(a.target, rc * a.target_stride + d);
      if (a.draft) yd = logit<T>(a.draft, rc * a.draft_stride + d);
      u = a.uniform[2 * (int64_t)rc];
    }
    const RowPart *const pp = a.parts + (int64_t)rc * a.pieces, *const qp = pp + (int64_t)a.n_rows * a.pieces;
    const bool drawn = !by_max && a.draft && !last;
    const First fp = first_parts(pp, a.pieces), fq = first_parts(qp, drawn ? a.pieces : 0);
    const Row p = join_row(fp, pp, a.pieces, t, by_max, table);
    Row q = {0.f, 0, 0.0};
    if (drawn) q = join_row(fq, qp, a.pieces, t, false, table);
    bool take = false;
    if (by_max) take = real && d == p.arg && p.top > -INFINITY;
    else if (real) {
      const double pd = p.sum > 0.0 ? Weigh(p.top, t, table).some(zd) / p.sum : 0.0;
      const double qd = !a.draft ? 1.0 : q.sum > 0.0 ? Weigh(q.top, t, table).some(yd) / q.sum : 0.0;
      take = (double)u * qd < pd;
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
  auto finish = [&](int token) {               // by one thread: its sequence has few rows as a rule
    a.accepted[s] = end - lo;
    a.tokens[end] = token;
  };
  if (chunk == 0) for (int i = lo + tid; i < hi; i += VT) if (i != end) a.tokens[i] = i < end ? a.ids[i + 1] : -1;
  if (by_max || !(p.sum > 0.0)) {
    if (chunk == 0 && tid == 0) finish(p.arg != 0x7fffffff ? p.arg : 0);
    return;
  }
  const bool residual = !last && (a.draft ? q.sum > 0.0 : (unsigned)d < (unsigned)a.vocab);
  const Weigh wp(p.top, t, table), wq(q.top, t, table);
  const double ip = 1.0 / p.sum, iq = q.sum > 0.0 ? 1.0 / q.sum : 0.0;
  // the weights that the draw goes by, of a lane's logits of a piece
  auto weights = [&](int piece, bool rest, double (&w)[PER]) {
    float z[PER], y[PER];
    load_piece<T>(a.target, end * a.target_stride, piece, a.vocab, lane, z);
    if (rest && a.draft) load_piece<T>(a.draft, end * a.draft_stride, piece, a.vocab, lane, y);
#pragma unroll
    for (int e = 0; e < PER; ++e) w[e] = wp(usable(z[e])) * ip;
    if (!rest) return;
    if (a.draft) {
#pragma unroll
      for (int e = 0; e < PER; ++e) w[e] = fmax(w[e] - wq(usable(y[e])) * iq, 0.0);
    } else {
#pragma unroll
      for (int e = 0; e < PER; ++e) if (id_of(piece, e, VEC, lane) == d) w[e] = fmax(w[e] - 1.0, 0.0);
    }
  };
  double w[PER];
  if (residual) {
    weights(chunk * 4 + wave, true, w);
    double sum = 0.0;
#pragma unroll
    for (int e = 0; e < PER; ++e) sum += w[e];
    sum = wave_sum_f64(sum);
    double* const mine = a.left + (int64_t)s * 4 * a.chunks + chunk * 4 + wave;
    if (lane == 0) __hip_atomic_store(mine, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // the sums are where every XCD finds them
    __syncthreads();
    if (tid == 0) s_last = __hip_atomic_fetch_add(a.done + s, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
    __syncthreads();
    if (!s_last) return;
  } else if (chunk != 0) return;
  if (wave != 0) return;
  // One wave is left of the sequence's: the piece that the number falls into, then the run of 64 lanes' logits in it, the lane, the logit.
  // (Sums in another order may fall short of the aim: then the last one that holds anything.)
  const double u = a.uniform[2 * (int64_t)end + 1];
  bool rest = residual;
  auto part = [&](int c) {
    if (c >= a.pieces) return 0.0;
    if (rest) return __hip_atomic_load(a.left + (int64_t)s * 4 * a.chunks + c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const RowPart x = a.parts[(int64_t)end * a.pieces + c];
    return x.sum * wp(x.top) * ip;
  };
  double near;                                 // this lane's of the first 64 pieces
  auto all = [&]() {
    double x = near = part(lane);
    for (int c = lane + WAVE; c < a.pieces; c += WAVE) x += part(c);
    return wave_sum_f64(x);
  };
  double total = all();
  if (rest && !(total > SOME)) { rest = false; total = all(); }      // p and q are the same: from p
  const double aim = u * total;
  double before = 0.0, upto = 0.0;
  int pick = 0;
  for (int c0 = 0; c0 < a.pieces; c0 += WAVE) {
    const double x = c0 ? part(c0 + lane) : near, up = scan_f64(x, lane);
    const unsigned long long some = __ballot(x > SOME), past = __ballot(x > SOME && upto + up > aim);
    if (past || some) {
      const int l = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
      pick = c0 + l;
      before = upto + lane_f64(up - x, l);
    }
    if (past) break;
    upto += lane_f64(up, 63);
  }
  weights(pick, rest, w);
  int token = 0;
  bool found = false;
#pragma unroll
  for (int v = 0; v < RUNS; ++v) {
    double x = 0.0;
#pragma unroll
    for (int e = 0; e < VEC; ++e) x += w[v * VEC + e];
    const double up = scan_f64(x, lane);
    const unsigned long long some = __ballot(x > SOME), past = __ballot(x > SOME && before + up > aim);
    if (!found && (past || some)) {
      const int l = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
      double run = before + (up - x);
      int mine = 0;
      bool over = false;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const double y = w[v * VEC + e];
        if (!over && y > SOME) { mine = id_of(pick, v * VEC + e, VEC, lane); run += y; over = run > aim; }
      }
      token = __builtin_amdgcn_readlane(mine, l);
      found = past != 0;
    }
    before += lane_f64(up, 63);
  }
  if (lane == 0) finish(token);
}

struct VerifyPlan { int chunks, pieces; uint64_t part_bytes, left_bytes, done_bytes; };

int check_verify(int n_seqs, int n_rows, int vocab, int dtype, VerifyPlan* p) {
  if (n_seqs < 1 || n_rows < 0 || vocab < 1 || dtype < PPD_FP32 || dtype > PPD_FP16) return PPD_EINVAL;
  if (n_seqs > PPD_MAX_SEQS || n_rows > PPD_MAX_TOKENS || vocab > VERIFY_MAX_VOCAB) return PPD_ELIMIT;
  p->chunks = (vocab + CHUNK - 1) / CHUNK;
  if ((int64_t)n_rows * p->chunks > 1 << 23) return PPD_ELIMIT;
  p->pieces = (vocab + PIECE - 1) / PIECE;
  p->part_bytes = (uint64_t)2 * n_rows * p->pieces * sizeof(RowPart);
  p->left_bytes = (uint64_t)n_seqs * p->chunks * 4 * sizeof(double);
  p->done_bytes = (uint64_t)n_seqs * sizeof(unsigned);
  return PPD_OK;
}

// Pieces that a wave takes in turn: as many as leave every unit two dozen waves (its places at the kernel's registers), eight at most.  bf16, a
// target and drafts' logits, us of the launch: 901 rows of 32000 at 4 / 8 pieces 42.2 / 41.4, 163 of 50272 at 1 / 3 pieces 12.7 / 13.4.
int run_of(int pieces, int n_rows, bool draft) {
  const int64_t run = (int64_t)n_rows * (draft ? 2 : 1) * pieces / (256 * 24);
  return run < 1 ? 1 : run > 8 ? 8 : (int)run;
}

template <typename T>
hipError_t verify_go(const VerifyArgs& a, hipStream_t st) {
  if (a.n_rows > 0) {
    const int64_t waves = (int64_t)a.n_rows * ((a.pieces + a.run - 1) / a.run);
    hipLaunchKernelGGL(verify_rows_kernel<T>, dim3((unsigned)((waves + 3) / 4), a.draft ? 2 : 1), dim3(VT), 0, st, a);
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
  VerifyArgs a = {row_start, ids, target_logits, draft_logits, target_stride, draft_stride, temperature, uniform, tokens, accepted,
                  n_seqs, n_rows, vocab, p.chunks, p.pieces, run_of(p.pieces, n_rows, draft_logits != nullptr),
                  (RowPart*)workspace, (double*)((char*)workspace + p.part_bytes), (unsigned*)((char*)workspace + p.part_bytes + p.left_bytes)};
  hipStream_t st = (hipStream_t)hip_stream;
  return launched(dtype == PPD_FP32 ? verify_go<float>(a, st) : dtype == PPD_BF16 ? verify_go<bf16_t>(a, st) : verify_go<f16_t>(a, st));
}
