// ppd_verify_drafts: drafted tokens against the target model's logits, from given random numbers.
#include "ppd_layers_common.h"

#include <math.h>

using namespace ppd;

namespace {

constexpr int VERIFY_MAX_VOCAB = 1 << 24;

struct VerifyArgs {
  const int32_t *row_start, *ids; const void *target, *draft; int64_t target_stride, draft_stride;
  const float *temperature, *uniform; int32_t *tokens, *accepted;
  int n_seqs, n_rows, vocab;
};

template <typename T> __device__ __forceinline__ float logit(const void* p, int64_t i);
template <> __device__ __forceinline__ float logit<float>(const void* p, int64_t i) { const float v = ((const float*)p)[i]; return v == v ? v : -INFINITY; }
template <> __device__ __forceinline__ float logit<bf16_t>(const void* p, int64_t i) { const float v = bf16_to_f32(((const uint16_t*)p)[i]); return v == v ? v : -INFINITY; }
template <> __device__ __forceinline__ float logit<f16_t>(const void* p, int64_t i) { const float v = (float)((const _Float16*)p)[i]; return v == v ? v : -INFINITY; }

// weight of a logit below the row's largest (itself: 1, also where that is infinite; a row of nothing: 0)
__device__ __forceinline__ double weight(float z, float top, double inv_t) {
  return z == -INFINITY ? 0.0 : z == top ? 1.0 : exp(((double)z - (double)top) * inv_t);
}

// One workgroup of 256 threads for a sequence, row by row.
template <typename T>
__global__ __launch_bounds__(256) void verify_kernel(VerifyArgs a) {
  __shared__ float fv[256]; __shared__ int iv[256]; __shared__ double dv[256];
  const int s = blockIdx.x, tid = threadIdx.x;
  const int lo = min(max(a.row_start[s], 0), a.n_rows), hi = min(max(a.row_start[s + 1], lo), a.n_rows);
  const double t = a.temperature ? (double)a.temperature[s] : 1.0;
  const bool by_max = !(t > 0.0);
  const double inv_t = by_max ? 0.0 : 1.0 / t;
  auto best = [&](const void* p, int64_t at, float& v, int& i) {
    v = -INFINITY; i = 0x7fffffff;
    for (int j = tid; j < a.vocab; j += 256) { const float z = logit<T>(p, at + j); if (better(z, j, v, i)) { v = z; i = j; } }
    __syncthreads();
    fv[tid] = v; iv[tid] = i;
    __syncthreads();
    for (int w = 128; w > 0; w >>= 1) {
      if (tid < w && better(fv[tid + w], iv[tid + w], fv[tid], iv[tid])) { fv[tid] = fv[tid + w]; iv[tid] = iv[tid + w]; }
      __syncthreads();
    }
    v = fv[0]; i = iv[0] == 0x7fffffff ? 0 : iv[0];
  };
  auto sum = [&](double x) {
    __syncthreads();
    dv[tid] = x;
    __syncthreads();
    for (int w = 128; w > 0; w >>= 1) { if (tid < w) dv[tid] += dv[tid + w]; __syncthreads(); }
    return dv[0];
  };
  int taken = 0;
  for (int r = lo; r < hi; ++r) {
    const int64_t tp = r * a.target_stride, dp = r * a.draft_stride;
    const bool last = r + 1 == hi;
    const int d = last ? -1 : a.ids[r + 1];
    const bool real = (unsigned)d < (unsigned)a.vocab;
    float top; int arg;
    best(a.target, tp, top, arg);
    int token = arg;
    bool take = real && d == arg && top > -INFINITY;
    if (!by_max) {
      double sp = 0, sq = 0; float dtop = 0; int unused;
      for (int j = tid; j < a.vocab; j += 256) sp += weight(logit<T>(a.target, tp + j), top, inv_t);
      sp = sum(sp);
      if (!last && a.draft) {
        best(a.draft, dp, dtop, unused);
        for (int j = tid; j < a.vocab; j += 256) sq += weight(logit<T>(a.draft, dp + j), dtop, inv_t);
        sq = sum(sq);
      }
      auto p = [&](int j) { return sp > 0 ? weight(logit<T>(a.target, tp + j), top, inv_t) / sp : 0.0; };
      auto q = [&](int j) { return last ? 0.0 : !a.draft ? (j == d ? 1.0 : 0.0) : sq > 0 ? weight(logit<T>(a.draft, dp + j), dtop, inv_t) / sq : 0.0; };
      take = real && (double)a.uniform[2 * (int64_t)r] * q(d) < p(d);
      if (!take) {
        const double u = a.uniform[2 * (int64_t)r + 1];
        const int per = (a.vocab + 255) / 256, j0 = min(tid * per, a.vocab), j1 = min(j0 + per, a.vocab);
        double mine = 0, total;
        for (int j = j0; j < j1; ++j) mine += fmax(p(j) - q(j), 0.0);
        total = sum(mine);
        const bool rest = total > 0;
        if (!rest) { mine = 0; for (int j = j0; j < j1; ++j) mine += p(j); total = sum(mine); }
        __syncthreads();
        dv[tid] = mine;
        if (tid == 0) iv[0] = 0x7fffffff, iv[1] = -1;
        __syncthreads();
        double before = 0;
        for (int w = 0; w < tid; ++w) before += dv[w];
        int first = 0x7fffffff, some = -1;
        for (int j = j0; j < j1; ++j) {
          const double x = rest ? fmax(p(j) - q(j), 0.0) : p(j);
          before += x;
          if (x > 0) { some = j; if (first == 0x7fffffff && before > u * total) first = j; }
        }
        atomicMin(&iv[0], first);
        atomicMax(&iv[1], some);
        __syncthreads();
        token = iv[0] != 0x7fffffff ? iv[0] : max(iv[1], 0);
      }
    }
    if (!take) {
      if (tid == 0) a.tokens[r] = token;
      for (int i = r + 1 + tid; i < hi; i += 256) a.tokens[i] = -1;
      break;
    }
    if (tid == 0) a.tokens[r] = d;
    ++taken;
  }
  if (tid == 0) a.accepted[s] = taken;
}

int check_verify(int n_seqs, int n_rows, int vocab, int dtype) {
  if (n_seqs < 1 || n_rows < 0 || vocab < 1 || dtype < PPD_FP32 || dtype > PPD_FP16) return PPD_EINVAL;
  return n_seqs > PPD_MAX_SEQS || n_rows > PPD_MAX_TOKENS || vocab > VERIFY_MAX_VOCAB ? PPD_ELIMIT : PPD_OK;
}

}  // namespace

extern "C" int ppd_verify_drafts_workspace(int n_seqs, int n_rows, int vocab, int dtype, uint64_t* bytes) {
  const int rc = check_verify(n_seqs, n_rows, vocab, dtype);
  if (rc) return rc;
  if (!bytes) return PPD_EINVAL;
  *bytes = 0;
  return PPD_OK;
}

extern "C" int ppd_verify_drafts(int n_seqs, int n_rows, int vocab, int dtype, const int32_t* row_start, const int32_t* ids,
                                 const void* target_logits, int64_t target_stride, const void* draft_logits, int64_t draft_stride,
                                 const float* temperature, const float* uniform, int32_t* tokens, int32_t* accepted,
                                 void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  uint64_t need = 0;
  const int rc = ppd_verify_drafts_workspace(n_seqs, n_rows, vocab, dtype, &need);
  if (rc) return rc;
  if (!row_start || !accepted || (n_rows > 0 && (!ids || !target_logits || !uniform || !tokens))) return PPD_EINVAL;
  if (n_rows > 1 && (target_stride < vocab || (draft_logits && draft_stride < vocab))) return PPD_EINVAL;
  const uintptr_t words = (uintptr_t)row_start | (uintptr_t)ids | (uintptr_t)temperature | (uintptr_t)uniform | (uintptr_t)tokens | (uintptr_t)accepted;
  if ((words & 3) || (((uintptr_t)target_logits | (uintptr_t)draft_logits) & (elem_size(dtype) - 1))) return PPD_EINVAL;
  if (need && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < need)) return PPD_EINVAL;
  VerifyArgs a = {row_start, ids, target_logits, draft_logits, target_stride, draft_stride, temperature, uniform, tokens, accepted, n_seqs, n_rows, vocab};
  hipStream_t st = (hipStream_t)hip_stream;
  if (dtype == PPD_FP32) hipLaunchKernelGGL(verify_kernel<float>, dim3(n_seqs), dim3(256), 0, st, a);
  else if (dtype == PPD_BF16) hipLaunchKernelGGL(verify_kernel<bf16_t>, dim3(n_seqs), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(verify_kernel<f16_t>, dim3(n_seqs), dim3(256), 0, st, a);
  return launched(hipGetLastError());
}
