// Distillation from a teacher's top logits (policy_distill_fwd_bwd).
//
// Per token t with logits z (temperature folded in: y = z / tau), teacher
// entries (id_k, l_k) and p the teacher's probabilities of them:
//   lse = log sum_v exp(y_v),  KL = sum_k p_k (log p_k - y_{id_k} + lse),
//   dz_v = w / tau (P exp(y_v - lse) - sum_{k: id_k = v} p_k),  P = sum_k p_k,
//   w = scale / (n_seq len_i),  loss += sum_t w_t KL_t.
// Bound by HBM: each logit is read and its gradient written once.  A row of
// 152064 bf16 logits (297 KB) fits the 512 KB of registers of a compute unit, so
// one block reads it into registers, reduces it with a running reference and sum
// as it arrives, and writes the gradient from there.

#include "logits_epilogue.h"
#include "rbp_internal.h"

namespace {

using rbp::lp::bf16_to_f32;
using rbp::lp::exp2_hw;
using rbp::lp::kLog2e;
using rbp::lp::pack_bf16x2;

constexpr int kMaxK = 256;

struct Args {
  int64_t ld;
  const int32_t* ids;
  const float *lt, *mass;
  const int32_t *seq, *len;
  int32_t V, K;
  float inv_tau, weight;  // weight = scale / n_seq
  float *kl, *terms;      // terms: [T][2] loss term, 1 if the token counts
};

// A row of logits as 16-byte pieces: the pieces that lie whole and aligned in
// it, and up to 2 (E - 1) elements before and behind them.
template <class X>
struct Row {
  static constexpr int E = 16 / sizeof(X);  // elements per piece
  int32_t head, pieces, V;
  __device__ __forceinline__ Row(const X* row, int32_t V_) : V(V_) {
    const int off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(X));
    head = (E - off) % E;
    if (head > V) head = V;
    pieces = (V - head) / E;
  }
  __device__ __forceinline__ int32_t at(int32_t piece) const { return head + piece * E; }
  // the loose element that thread tid takes, -1 for none
  __device__ __forceinline__ int32_t loose(int tid) const {
    const int32_t v = tid < head ? tid : pieces * E + tid;
    return tid < 2 * E && v < V ? v : -1;
  }
};

__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(uint16_t v) { return bf16_to_f32(v); }
__device__ __forceinline__ void to(float& o, float v) { o = v; }
__device__ __forceinline__ void to(uint16_t& o, float v) {
  o = __builtin_bit_cast(uint16_t, (__bf16)v);
}

// A piece's elements, and back.
__device__ __forceinline__ void unpack(const uint4& p, float (&x)[4]) {
  x[0] = __uint_as_float(p.x), x[1] = __uint_as_float(p.y);
  x[2] = __uint_as_float(p.z), x[3] = __uint_as_float(p.w);
}
__device__ __forceinline__ void unpack(const uint4& p, float (&x)[8]) {
  const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    x[2 * k] = __uint_as_float(w[k] << 16);
    x[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint4 pack(const float (&x)[4]) {
  return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                    __float_as_uint(x[3]));
}
__device__ __forceinline__ uint4 pack(const float (&x)[8]) {
  return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                    pack_bf16x2(x[6], x[7]));
}

// Running reference and sum of a thread: s = sum exp((z - m) inv_tau).  m follows
// the largest logit only once that is kSlack (in powers of two) above it: sums
// stay far from overflow, and rescaling is rare.
constexpr float kSlack = 20.0f;
struct Online {
  float m = -INFINITY, s = 0.0f;
  template <int N>
  __device__ __forceinline__ void add(const float (&x)[N], float k2, float slack) {
    float top = x[0];
#pragma unroll
    for (int k = 1; k < N; ++k) top = fmaxf(top, x[k]);
    if (top > m + slack) {
      s *= exp2_hw((m - top) * k2);
      m = top;
    }
    const float ref = m == -INFINITY ? 0.0f : m;  // nothing but -inf so far
    float e[N];
#pragma unroll
    for (int k = 0; k < N; ++k) e[k] = exp2_hw((x[k] - ref) * k2);
#pragma unroll
    for (int w = N / 2; w >= 1; w /= 2)
#pragma unroll
      for (int k = 0; k < w; ++k) e[k] += e[k + w];
    s += e[0];
  }
};

// A block per token.  Each thread keeps kHold pieces of the row in registers, so
// that a row of up to kThreads * kHold pieces is read from memory once; the
// pieces beyond them are read again for the gradient.  The first wave prepares
// the teacher's entries while the row arrives.  An element that the teacher
// names gets its gradient a second time, behind a barrier, so that the loop over
// the row looks for nothing.
template <class X, int kThreads, int kHold, bool kGrad, bool kBypass>
__global__ void __launch_bounds__(kThreads) distill_row_kernel(const X* z, X* dz, Args a) {
  constexpr int E = Row<X>::E, kWaves = kThreads / 64;
  __shared__ float m_s[kWaves], s_s[kWaves];
  __shared__ float mass_s;                       // P
  __shared__ int32_t any_s;
  __shared__ __attribute__((aligned(16))) int32_t id_s[kMaxK];
  __shared__ __attribute__((aligned(16))) float p_s[kMaxK];
  __shared__ float z_s[kMaxK], e_s[kMaxK];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const X* row = z + t * a.ld;
  X* grad = kGrad ? dz + t * a.ld : nullptr;
  const Row<X> r(row, a.V);
  const bool vec = kGrad && ((reinterpret_cast<uintptr_t>(row) ^
                              reinterpret_cast<uintptr_t>(grad)) & 15) == 0;
  const int32_t loose = r.loose(tid);
  const int32_t sq = a.seq[t];
  auto put = [&](int32_t piece, const uint4& v) {
    X* to_ = grad + r.at(piece);
    if (vec && kBypass) {
      typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<u32x4*>(to_));
    } else if (vec) {
      *reinterpret_cast<uint4*>(to_) = v;
    } else {
      X e[E];
      __builtin_memcpy(e, &v, 16);
#pragma unroll
      for (int k = 0; k < E; ++k) to_[k] = e[k];
    }
  };
  auto zeros = [&] {  // no teacher, or masked
    if (tid == 0) {
      a.kl[t] = 0.0f;
      a.terms[2 * t] = 0.0f;
      a.terms[2 * t + 1] = 0.0f;
    }
    if constexpr (kGrad) {
      for (int32_t c = tid; c < r.pieces; c += kThreads) put(c, make_uint4(0u, 0u, 0u, 0u));
      if (loose >= 0) grad[loose] = X(0);
    }
  };
  if (sq < 0) return zeros();

  uint4 hold[kHold > 0 ? kHold : 1];
#pragma unroll
  for (int i = 0; i < kHold; ++i) {
    const int32_t c = i * kThreads + tid;
    if (c < r.pieces) hold[i] = *reinterpret_cast<const uint4*>(row + r.at(c));
  }
  const float edge = loose >= 0 ? value(row[loose]) : -INFINITY;

  if (wave == 0) {
    constexpr int kPer = kMaxK / 64;
    int32_t id[kPer];
    float l[kPer], p[kPer];
    float top = -INFINITY, nan = 0.0f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int k = j * 64 + lane;
      id[j] = -1;
      l[j] = -INFINITY;
      if (k < a.K) {
        id[j] = a.ids[t * a.K + k];
        if (id[j] >= 0) l[j] = a.lt[t * a.K + k] * a.inv_tau;
      }
      top = fmaxf(top, l[j]);
      if (l[j] != l[j]) nan = 1.0f;
    }
    top = rbp::lp::wave_max(top);
    nan = rbp::lp::wave_max(nan);
    float mass = 0.0f, P = 0.0f;
    if (a.mass != nullptr) {
      mass = a.mass[t];
    } else {
      float sum = 0.0f;
#pragma unroll
      for (int j = 0; j < kPer; ++j) sum += id[j] >= 0 ? expf(l[j] - top) : 0.0f;
      mass = top + logf(rbp::lp::wave_sum(sum));
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int k = j * 64 + lane;
      const float logp = l[j] - mass;
      p[j] = id[j] >= 0 ? expf(logp) : 0.0f;
      P += p[j];
      if (k >= a.K) {  // up to a whole quarter of entries
        if (k < ((a.K + 3) & ~3)) id_s[k] = -1, p_s[k] = 0.0f;
      } else {
        const float zk = id[j] >= 0 && id[j] < a.V ? value(row[id[j]]) : NAN;
        id_s[k] = id[j];
        p_s[k] = p[j];
        z_s[k] = zk;
        e_s[k] = logp - zk * a.inv_tau;
      }
    }
    P = rbp::lp::wave_sum(P);
    if (lane == 0) {
      mass_s = P;
      any_s = top > -INFINITY || nan > 0.0f;
    }
  }

  const float k2 = a.inv_tau * kLog2e, slack = fminf(kSlack / k2, 1e30f);
  Online o;
#pragma unroll
  for (int i = 0; i < kHold; ++i) {
    if (i * kThreads + tid < r.pieces) {
      float x[E];
      unpack(hold[i], x);
      o.add(x, k2, slack);
    }
  }
  constexpr int kBatch = 4;  // loads in flight
  int32_t c = kHold * kThreads + tid;
  for (; c + (kBatch - 1) * kThreads < r.pieces; c += kBatch * kThreads) {
    uint4 v[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      v[i] = *reinterpret_cast<const uint4*>(row + r.at(c + i * kThreads));
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      float x[E];
      unpack(v[i], x);
      o.add(x, k2, slack);
    }
  }
  for (; c < r.pieces; c += kThreads) {
    float x[E];
    unpack(*reinterpret_cast<const uint4*>(row + r.at(c)), x);
    o.add(x, k2, slack);
  }
  const float last[1] = {edge};
  o.add(last, k2, slack);

  // the row's reference (not below its threads') and sum
  auto rebase = [&](float s, float from, float onto) {
    return from == -INFINITY ? s : s * exp2_hw((from - onto) * k2);
  };
  float M = rbp::lp::wave_max(o.m);
  float S = rbp::lp::wave_sum(rebase(o.s, o.m, M));
  if (lane == 0) {
    m_s[wave] = M;
    s_s[wave] = S;
  }
  __syncthreads();
  if constexpr (kWaves > 1) {
    M = m_s[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, m_s[w]);
    S = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) S += rebase(s_s[w], m_s[w], M);
  }
  if (!any_s) return zeros();
  const float w = a.weight / (float)a.len[sq];
  if (wave == 0) {
    const float lse = M * a.inv_tau + logf(S);
    float kl = 0.0f;
    for (int k = lane; k < a.K; k += 64)
      if (p_s[k] != 0.0f) kl += p_s[k] * (e_s[k] + lse);
    kl = rbp::lp::wave_sum(kl);
    if (lane == 0) {
      a.kl[t] = kl;
      a.terms[2 * t] = w * kl;
      a.terms[2 * t + 1] = 1.0f;
    }
  }
  if constexpr (kGrad) {
    const float cw = w * a.inv_tau, f = cw * mass_s / S;
    auto gradient = [&](const uint4& v) {
      float x[E];
      unpack(v, x);
#pragma unroll
      for (int k = 0; k < E; ++k) x[k] = f * exp2_hw((x[k] - M) * k2);
      return pack(x);
    };
    // the pieces that are read again, latest first
    if (kHold * kThreads + tid < r.pieces) {
      int32_t p = kHold * kThreads + tid;
      p += (r.pieces - 1 - p) / kThreads * kThreads;
      for (; p - (kBatch - 1) * kThreads >= kHold * kThreads; p -= kBatch * kThreads) {
        uint4 v[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          v[i] = *reinterpret_cast<const uint4*>(row + r.at(p - i * kThreads));
#pragma unroll
        for (int i = 0; i < kBatch; ++i) put(p - i * kThreads, gradient(v[i]));
      }
      for (; p >= kHold * kThreads; p -= kThreads)
        put(p, gradient(*reinterpret_cast<const uint4*>(row + r.at(p))));
    }
#pragma unroll
    for (int i = 0; i < kHold; ++i) {
      const int32_t p = i * kThreads + tid;
      if (p < r.pieces) put(p, gradient(hold[i]));
    }
    if (loose >= 0) to(grad[loose], f * exp2_hw((edge - M) * k2));
    // the named elements again, once the row's stores are ordered before; an id
    // that occurs twice has all of its mass, and the same value is stored twice
    __syncthreads();
    for (int k = tid; k < a.K; k += kThreads) {
      const int32_t id = id_s[k];
      if (id < 0 || id >= a.V) continue;
      float all = 0.0f;
#pragma unroll 2
      for (int i = 0; i < a.K; i += 4) {
        const int4 o = *reinterpret_cast<const int4*>(id_s + i);
        const float4 q = *reinterpret_cast<const float4*>(p_s + i);
        all += (o.x == id ? q.x : 0.0f) + (o.y == id ? q.y : 0.0f) + (o.z == id ? q.z : 0.0f) +
               (o.w == id ? q.w : 0.0f);
      }
      to(grad[id], f * exp2_hw((z_s[k] - M) * k2) - cw * all);
    }
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

// Threads and pieces held per thread by the row's length: small rows on few
// threads, the largest on 1024 with as many pieces as their registers hold.
template <class X>
void launch_rows(const X* z, X* dz, int64_t T, const Args& a, hipStream_t s) {
  const int64_t pieces = a.V / Row<X>::E;
  // Stores past the caches where part of the row is read twice (the gradient must
  // not push it out: 1301 x 151936 fp32 429 -> 329 us) and for passes of less than
  // 3/4 GiB (512 x 151936 bf16 84 -> 73 us, 8192 x 12000 91 -> 89); beyond, cached
  // stores are faster (16384 x 152064 1962 against 2024 us, 5000 612 / 635).
  const bool bypass = pieces > 1024 * 20 || T * a.ld * (int64_t)sizeof(X) < (3ll << 28);
  auto go = [&](auto threads, auto hold) {
    constexpr int kThreads = decltype(threads)::value, kHold = decltype(hold)::value;
    auto kernel = dz == nullptr ? distill_row_kernel<X, kThreads, 0, false, false>
                  : bypass      ? distill_row_kernel<X, kThreads, kHold, true, true>
                                : distill_row_kernel<X, kThreads, kHold, true, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)T), dim3(kThreads), 0, s, z, dz, a);
  };
  using std::integral_constant;
  if (pieces <= 64 * 4)
    go(integral_constant<int, 64>{}, integral_constant<int, 4>{});
  else if (pieces <= 256 * 4)
    go(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  else if (pieces <= 256 * 8)
    go(integral_constant<int, 256>{}, integral_constant<int, 8>{});
  else if (pieces <= 512 * 8)
    go(integral_constant<int, 512>{}, integral_constant<int, 8>{});
  else if (pieces <= 1024 * 8)
    go(integral_constant<int, 1024>{}, integral_constant<int, 8>{});
  else
    go(integral_constant<int, 1024>{}, integral_constant<int, 20>{});
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
    launch_rows(static_cast<const float*>(logits), static_cast<float*>(dlogits), T, a, s);
  else
    launch_rows(static_cast<const uint16_t*>(logits), static_cast<uint16_t*>(dlogits), T, a, s);
  hipLaunchKernelGGL(distill_sum_kernel, dim3(1), dim3(1024), 0, s, terms, kl, T, loss_accum,
                     stats);
  RBP_CHECK_LAUNCH("policy_distill_fwd_bwd");
  return RBP_OK;
}
