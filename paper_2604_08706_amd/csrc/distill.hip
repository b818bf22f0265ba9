// Distillation from a teacher's top logits (policy_distill_fwd_bwd).
//
// Per token t with logits z (temperature folded in: y = z / tau), teacher
// entries (id_k, l_k) and p the teacher's probabilities of them:
//   lse = log sum_v exp(y_v),  KL = sum_k p_k (log p_k - y_{id_k} + lse),
//   dz_v = w / tau (P exp(y_v - lse) - sum_{k: id_k = v} p_k),  P = sum_k p_k,
//   w = scale / (n_seq len_i),  loss += sum_t w_t KL_t.
// Bound by HBM: each logit is read and its gradient written once.

#include "logits_epilogue.h"
#include "rbp_internal.h"

namespace {

using rbp::lp::bf16_to_f32;
using rbp::lp::kLog2e;

constexpr int kThreads = 256;
constexpr int kMaxK = 256;

__device__ __forceinline__ float value(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float value(const uint16_t* p, int64_t i) { return bf16_to_f32(p[i]); }
__device__ __forceinline__ void put(float* p, int64_t i, float v) { p[i] = v; }
__device__ __forceinline__ void put(uint16_t* p, int64_t i, float v) {
  p[i] = __builtin_bit_cast(uint16_t, (__bf16)v);
}

struct Args {
  int64_t ld;
  const int32_t* ids;
  const float *lt, *mass;
  const int32_t *seq, *len;
  int32_t V, K;
  float inv_tau, weight;  // weight = scale / n_seq
  float *kl, *terms;      // terms: [T][2] loss term, 1 if the token counts
};

__device__ __forceinline__ float block_max(float v, float* s) {
  v = rbp::lp::wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
  for (int w = 1; w < kThreads / 64; ++w) v = fmaxf(v, s[w]);
  return v;
}
__device__ __forceinline__ float block_sum(float v, float* s) {
  v = rbp::lp::wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0f;
  for (int w = 0; w < kThreads / 64; ++w) v += s[w];
  return v;
}

// A block per token: the teacher's entries one per thread, then two passes over
// the logits.
template <class X>
__global__ void __launch_bounds__(kThreads) distill_row_kernel(const X* z, X* dz, Args a) {
  __shared__ float s[kThreads / 64], ps[kMaxK];
  __shared__ int32_t is[kMaxK];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x;
  const X* row = z + t * a.ld;
  X* grad = dz == nullptr ? nullptr : dz + t * a.ld;
  const int32_t sq = a.seq[t];
  int32_t id = -1;
  float l = -INFINITY;
  if (sq >= 0 && tid < a.K) {
    id = a.ids[t * a.K + tid];
    if (id >= 0) l = a.lt[t * a.K + tid] * a.inv_tau;
  }
  const bool nan = block_max(l != l ? 1.0f : 0.0f, s) > 0.0f;
  const float lm = block_max(l, s);
  if (sq < 0 || (lm == -INFINITY && !nan)) {
    if (grad != nullptr)
      for (int32_t v = tid; v < a.V; v += kThreads) put(grad, v, 0.0f);
    if (tid == 0) {
      a.kl[t] = 0.0f;
      a.terms[2 * t] = 0.0f;
      a.terms[2 * t + 1] = 0.0f;
    }
    return;
  }
  const float mass =
      a.mass != nullptr ? a.mass[t] : lm + logf(block_sum(id >= 0 ? expf(l - lm) : 0.0f, s));
  const float logp = l - mass, p = id >= 0 ? expf(logp) : 0.0f;
  const float P = block_sum(p, s);
  float m = -INFINITY;
  for (int32_t v = tid; v < a.V; v += kThreads) m = fmaxf(m, value(row, v));
  m = block_max(m, s);
  float sum = 0.0f;
  for (int32_t v = tid; v < a.V; v += kThreads) sum += expf((value(row, v) - m) * a.inv_tau);
  sum = block_sum(sum, s);
  const float lse = m * a.inv_tau + logf(sum);
  float term = 0.0f;
  if (p != 0.0f) term = id < a.V ? p * (logp - value(row, id) * a.inv_tau + lse) : NAN;
  const float kl = block_sum(term, s);
  const float w = a.weight / (float)a.len[sq];
  if (tid == 0) {
    a.kl[t] = kl;
    a.terms[2 * t] = w * kl;
    a.terms[2 * t + 1] = 1.0f;
  }
  if (grad == nullptr) return;
  if (tid < a.K) {
    ps[tid] = p;
    is[tid] = id;
  }
  __syncthreads();
  const float c = w * a.inv_tau, f = c * P / sum;
  for (int32_t v = tid; v < a.V; v += kThreads) {
    float g = f * expf((value(row, v) - m) * a.inv_tau);
    for (int k = 0; k < a.K; ++k)
      if (is[k] == v) g -= c * ps[k];
    put(grad, v, g);
  }
}

// The sums over tokens, in one block and a fixed order.
__global__ void __launch_bounds__(1024) distill_sum_kernel(const float* __restrict__ terms,
                                                           const float* __restrict__ kl, int64_t T,
                                                           float* __restrict__ loss_accum,
                                                           float* __restrict__ stats) {
  __shared__ double s[3][16];
  double v[3] = {0.0, 0.0, 0.0};
  for (int64_t t = threadIdx.x; t < T; t += 1024) {
    v[0] += terms[2 * t];
    v[1] += terms[2 * t + 1];
    v[2] += kl[t];
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    for (int off = 32; off >= 1; off >>= 1) v[k] += __shfl_xor(v[k], off, 64);
    if ((threadIdx.x & 63) == 0) s[k][threadIdx.x >> 6] = v[k];
  }
  __syncthreads();
  if (threadIdx.x >= 3) return;
  double sum = 0.0;
  for (int w = 0; w < 16; ++w) sum += s[threadIdx.x][w];
  float* to = threadIdx.x == 0 ? loss_accum : stats + (threadIdx.x - 1);
  *to = (float)((double)*to + sum);
}

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace

size_t rbp::distill_ws(int64_t T, int32_t K, int32_t V) {
  (void)K, (void)V;
  return align_up((size_t)(T < 1 ? 1 : T) * 2 * sizeof(float), 256);
}

extern "C" int policy_distill_fwd_bwd(const void* logits, int logits_type, int64_t ld,
                                      const int32_t* teacher_ids, const float* teacher_logits,
                                      const float* teacher_lse, const int32_t* seq_of_token,
                                      const int32_t* seq_len, int64_t T, int32_t V, int32_t K,
                                      int32_t B, int64_t n_seq_total, float temperature,
                                      float scale, float* kl, float* loss_accum, float* stats,
                                      void* dlogits, void* ws, size_t ws_bytes, void* stream) {
  rbp::clear_error();
  RBP_REQUIRE(T >= 0 && V >= 1 && K >= 1 && ld >= V, RBP_EINVAL,
              "policy_distill_fwd_bwd: need T >= 0, V >= 1, K >= 1, ld >= V");
  RBP_REQUIRE(B >= 1 && n_seq_total >= 1, RBP_EINVAL,
              "policy_distill_fwd_bwd: need B >= 1 and n_seq_total >= 1");
  RBP_REQUIRE(logits_type == RBP_BF16 || logits_type == RBP_F32, RBP_EINVAL,
              "policy_distill_fwd_bwd: unknown logits_type %d", logits_type);
  RBP_REQUIRE(std::isfinite(temperature) && temperature > 0.0f && std::isfinite(scale), RBP_EINVAL,
              "policy_distill_fwd_bwd: need a positive temperature and a finite scale");
  RBP_REQUIRE(K <= kMaxK, RBP_EUNSUPPORTED, "policy_distill_fwd_bwd: K above %d", kMaxK);
  RBP_REQUIRE(T <= INT32_MAX, RBP_EUNSUPPORTED, "policy_distill_fwd_bwd: T above 2^31 - 1");
  RBP_REQUIRE(loss_accum && stats && seq_len, RBP_EINVAL, "policy_distill_fwd_bwd: null pointer");
  if (T == 0) return RBP_OK;
  RBP_REQUIRE(logits && teacher_ids && teacher_logits && seq_of_token && kl, RBP_EINVAL,
              "policy_distill_fwd_bwd: null per-token pointer");
  const size_t es = logits_type == RBP_F32 ? 4 : 2;
  RBP_REQUIRE(aligned(logits, es) && aligned(dlogits, es), RBP_EINVAL,
              "policy_distill_fwd_bwd: logits or dlogits not aligned to their type");
  const size_t need = rbp::distill_ws(T, K, V);
  RBP_REQUIRE(ws && ws_bytes >= need, RBP_EWORKSPACE,
              "policy_distill_fwd_bwd: workspace needs %zu bytes, got %zu", need, ws_bytes);
  hipStream_t s = rbp::as_stream(stream);
  float* terms = static_cast<float*>(ws);
  const Args a{ld, teacher_ids, teacher_logits, teacher_lse, seq_of_token, seq_len, V, K,
               1.0f / temperature, (float)((double)scale / (double)n_seq_total), kl, terms};
  if (logits_type == RBP_F32)
    hipLaunchKernelGGL(distill_row_kernel<float>, dim3((unsigned)T), dim3(kThreads), 0, s,
                       static_cast<const float*>(logits), static_cast<float*>(dlogits), a);
  else
    hipLaunchKernelGGL(distill_row_kernel<uint16_t>, dim3((unsigned)T), dim3(kThreads), 0, s,
                       static_cast<const uint16_t*>(logits), static_cast<uint16_t*>(dlogits), a);
  hipLaunchKernelGGL(distill_sum_kernel, dim3(1), dim3(1024), 0, s, terms, kl, T, loss_accum,
                     stats);
  RBP_CHECK_LAUNCH("policy_distill_fwd_bwd");
  return RBP_OK;
}
