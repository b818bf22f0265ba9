// Verification of drafted tokens (policy_verify_drafts).
//
// With p_k, q_k the policy's and the draft's distributions at position k of a
// sequence, draft x_k is accepted iff u_k q_k(x_k) < p_k(x_k); at the first
// rejection a the token is drawn from max(p_a - q_a, 0), normalised, and after
// the last accepted draft from p: then every emitted token is distributed as p
// (P(x) = q min(1, p / q) + (1 - sum q min(1, p / q)) max(p - q, 0) / sum max(p - q, 0)
// = min(q, p) + max(p - q, 0) = p).  The drawn token is the least v whose running
// sum of weights exceeds u_K times their total.
//
// A running sum over 152064 tokens has steps of 1e-5 and less, and its rounding
// decides which token a u beside a step draws: 32-bit sums would differ from the
// exact ones in about one draw in a hundred.  So exponentials and sums are in 64
// bits.

#include <cmath>

#include "logits_epilogue.h"
#include "rbp_internal.h"

namespace {

using rbp::lp::bf16_to_f32;

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;

__device__ __forceinline__ double value(const float* p, int64_t i) { return (double)p[i]; }
__device__ __forceinline__ double value(const uint16_t* p, int64_t i) {
  return (double)bf16_to_f32(p[i]);
}

__device__ __forceinline__ double block_max(double v, double* s) {
  for (int off = 32; off >= 1; off >>= 1) v = fmax(v, __shfl_xor(v, off, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
  for (int w = 1; w < kWaves; ++w) v = fmax(v, s[w]);
  return v;
}
__device__ __forceinline__ double block_sum(double v, double* s) {
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
  for (int w = 0; w < kWaves; ++w) v += s[w];
  return v;
}

// A row's distribution: exp((z - max) inv_tau) / sum; sum is NaN if the row has none.
template <class X>
struct Dist {
  const X* z;
  double inv_tau, max, sum;
  __device__ void of(const X* row, int32_t V, double it, double* s) {
    z = row;
    inv_tau = it;
    double m = -INFINITY;
    for (int32_t v = threadIdx.x; v < V; v += kThreads) m = fmax(m, value(z, v));
    max = block_max(m, s);
    double e = 0.0;
    for (int32_t v = threadIdx.x; v < V; v += kThreads) e += exp((value(z, v) - max) * inv_tau);
    sum = block_sum(e, s);
  }
  __device__ double p(int64_t v) const { return exp((value(z, v) - max) * inv_tau) / sum; }
};

// One block per sequence.
template <class X>
__global__ void __launch_bounds__(kThreads) verify_kernel(
    const X* __restrict__ logits, const X* __restrict__ draft_logits, int64_t ld, int64_t ld_draft,
    const int32_t* __restrict__ draft_tokens, const int32_t* __restrict__ n_draft,
    const float* __restrict__ u, int32_t K, int32_t V, double inv_tau,
    int32_t* __restrict__ out_tokens, float* __restrict__ out_logp, int32_t* __restrict__ n_out) {
  __shared__ double s[kWaves];
  __shared__ int32_t found, last;
  const int64_t b = blockIdx.x;
  const int tid = threadIdx.x;
  int32_t n = n_draft == nullptr ? K : min(n_draft[b], K);
  int32_t* tok = out_tokens + b * (K + 1);
  float* lp = out_logp + b * (K + 1);
  for (int k = tid; k <= K; k += kThreads) {
    tok[k] = -1;
    lp[k] = 0.0f;
  }
  if (n < 0) {
    if (tid == 0) n_out[b] = 0;
    return;
  }
  __syncthreads();
  Dist<X> p, q;
  int32_t a = 0, x = -1;
  bool rejected = false;
  for (;; ++a) {
    p.of(logits + (b * (K + 1) + a) * ld, V, inv_tau, s);
    if (a == n) break;
    x = draft_tokens[b * K + a];
    const bool in = x >= 0 && x < V;
    if (draft_logits != nullptr) q.of(draft_logits + (b * K + a) * ld_draft, V, inv_tau, s);
    const double px = in ? p.p(x) : 0.0;
    const double qx = draft_logits == nullptr ? 1.0 : in ? q.p(x) : 0.0;
    if (!((double)u[b * (K + 1) + a] * qx < px)) {
      rejected = true;
      break;
    }
    if (tid == 0) {
      tok[a] = x;
      lp[a] = (float)log(px);
    }
  }
  if (tid == 0) n_out[b] = a + 1;
  if (!(p.sum > 0.0 && p.sum < INFINITY)) {
    if (tid == 0) lp[a] = NAN;
    return;
  }
  int kind = !rejected ? 0 : draft_logits == nullptr ? 1 : q.sum > 0.0 ? 2 : 0;
  auto weight = [&](int32_t v) {
    const double pv = p.p(v);
    return kind == 0 ? pv : kind == 1 ? (v == x ? 0.0 : pv) : fmax(pv - q.p(v), 0.0);
  };
  double total = 0.0;
  for (;;) {
    double e = 0.0;
    for (int32_t v = tid; v < V; v += kThreads) e += weight(v);
    total = block_sum(e, s);
    if (total > 0.0 || kind == 0) break;
    kind = 0;
  }
  const double goal = (double)u[b * (K + 1) + K] * total;
  if (tid == 0) {
    found = V;
    last = -1;
  }
  __syncthreads();
  double before = 0.0;
  for (int32_t v0 = 0; v0 < V; v0 += kThreads) {
    const int32_t v = v0 + tid;
    const double wv = v < V ? weight(v) : 0.0;
    double run = wv;  // inclusive over the tile
    for (int off = 1; off < 64; off <<= 1) {
      const double o = __shfl_up(run, off, 64);
      if ((tid & 63) >= off) run += o;
    }
    __syncthreads();
    if ((tid & 63) == 63) s[tid >> 6] = run;
    __syncthreads();
    double tile = 0.0;
    for (int w = 0; w < kWaves; ++w) {
      if (w < (tid >> 6)) run += s[w];
      tile += s[w];
    }
    if (wv > 0.0) {
      atomicMax(&last, v);
      if (before + run > goal) atomicMin(&found, v);
    }
    before += tile;
    __syncthreads();
    if (found < V) break;
  }
  if (tid == 0) {
    const int32_t v = found < V ? found : last;
    tok[a] = v;
    lp[a] = v < 0 ? NAN : (float)log(p.p(v));
  }
}

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace

size_t rbp::verify_ws(int64_t B, int32_t K, int32_t V) {
  (void)B, (void)K, (void)V;
  return 256;
}

extern "C" int policy_verify_drafts(const void* logits, const void* draft_logits, int logits_type,
                                    int64_t ld, int64_t ld_draft, const int32_t* draft_tokens,
                                    const int32_t* n_draft, const float* u, int32_t B, int32_t K,
                                    int32_t V, float temperature, int32_t* out_tokens,
                                    float* out_logp, int32_t* n_out, void* ws, size_t ws_bytes,
                                    void* stream) {
  rbp::clear_error();
  RBP_REQUIRE(B >= 0 && K >= 0 && V >= 1 && ld >= V && (draft_logits == nullptr || ld_draft >= V),
              RBP_EINVAL, "policy_verify_drafts: need B >= 0, K >= 0, V >= 1, ld and ld_draft >= V");
  RBP_REQUIRE(logits_type == RBP_BF16 || logits_type == RBP_F32, RBP_EINVAL,
              "policy_verify_drafts: unknown logits_type %d", logits_type);
  RBP_REQUIRE(std::isfinite(temperature) && temperature > 0.0f, RBP_EINVAL,
              "policy_verify_drafts: temperature must be positive and finite");
  RBP_REQUIRE(K <= 255 && (int64_t)B * (K + 1) <= (1 << 24), RBP_EUNSUPPORTED,
              "policy_verify_drafts: K above 255 or B (K + 1) above 2^24");
  if (B == 0) return RBP_OK;
  RBP_REQUIRE(logits && u && out_tokens && out_logp && n_out && (K == 0 || draft_tokens),
              RBP_EINVAL, "policy_verify_drafts: null pointer");
  const size_t es = logits_type == RBP_F32 ? 4 : 2;
  RBP_REQUIRE(aligned(logits, es) && aligned(draft_logits, es), RBP_EINVAL,
              "policy_verify_drafts: logits not aligned to their type");
  const size_t need = rbp::verify_ws(B, K, V);
  RBP_REQUIRE(ws && ws_bytes >= need, RBP_EWORKSPACE,
              "policy_verify_drafts: workspace needs %zu bytes, got %zu", need, ws_bytes);
  hipStream_t s = rbp::as_stream(stream);
  const double inv_tau = 1.0 / (double)temperature;
  if (logits_type == RBP_F32)
    hipLaunchKernelGGL(verify_kernel<float>, dim3(B), dim3(kThreads), 0, s,
                       static_cast<const float*>(logits), static_cast<const float*>(draft_logits),
                       ld, ld_draft, draft_tokens, n_draft, u, K, V, inv_tau, out_tokens, out_logp,
                       n_out);
  else
    hipLaunchKernelGGL(verify_kernel<uint16_t>, dim3(B), dim3(kThreads), 0, s,
                       static_cast<const uint16_t*>(logits),
                       static_cast<const uint16_t*>(draft_logits), ld, ld_draft, draft_tokens,
                       n_draft, u, K, V, inv_tau, out_tokens, out_logp, n_out);
  RBP_CHECK_LAUNCH("policy_verify_drafts");
  return RBP_OK;
}
