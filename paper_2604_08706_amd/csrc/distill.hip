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

#include <algorithm>

#include "rbp_internal.h"
#include "vocab_rows.h"

namespace {

using rbp::lp::exp2_hw;
using rbp::lp::kLog2e;
using rbp::rows::aligned;
using rbp::rows::pack;
using rbp::rows::Row;
using rbp::rows::to;
using rbp::rows::unpack;
using rbp::rows::value;

constexpr int kMaxK = 256;

struct Args {
  int64_t ld;
  const int32_t* ids;
  const float *lt, *mass;
  const int32_t *seq, *len;
  int32_t V, K;
  float inv_tau, weight;  // weight = scale / n_seq
  double rtau;            // 1 / tau
  float *kl, *terms;      // terms: [T][2] loss term, 1 if the token counts
};

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

// Adding a constant to all logits changes no KL, but its parts log p, z / tau and lse each
// have the constant's size: 32 bits would leave 3e-5 of a constant of 100.  So the teacher's
// logits are taken relative to their largest before anything is rounded, and what the policy's
// have in common cancels in 64 bits (an operation or two per entry).
// (The logarithm of S is its exponent's and, in 32 bits, that of a number between 1/2 and 1:
// to 2^-25 for a fraction of a 64-bit one's operations.)
__device__ __forceinline__ double lse_of(float M, float S, double rtau) {
  int e;
  const float m = frexpf(S, &e);
  return fma((double)M, rtau, fma((double)e, 0.69314718055994530942, (double)logf(m)));
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// The teacher's entries of a token, by one wave: entry k goes to id[k], p[k] (its
// probability), lp[k] = log p_k and z[k] (the policy's logit there); up to a whole
// quarter of entries is filled with absent ones.
struct Teacher {
  float P;        // sum of p
  double A, mass;  // sum of p (log p - z / tau), sum of p: KL = A + mass lse
  bool any;       // an entry of some mass (or a NaN)
};
template <class X>
__device__ __forceinline__ Teacher teacher_entries(const Args& a, int64_t t, const X* row,
                                                   int lane, int32_t* id_s, float* p_s,
                                                   float* z_s, float* lp_s) {
  constexpr int kPer = kMaxK / 64;
  int32_t id[kPer];
  float l[kPer];
  float top = -INFINITY, nan = 0.0f;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int k = j * 64 + lane;
    id[j] = -1;
    l[j] = -INFINITY;
    if (k < a.K) {
      id[j] = a.ids[t * a.K + k];
      if (id[j] >= 0) l[j] = a.lt[t * a.K + k];
    }
    top = fmaxf(top, l[j]);
    if (l[j] != l[j]) nan = 1.0f;
  }
  top = rbp::lp::wave_max(top);
  nan = rbp::lp::wave_max(nan);
  float P = 0.0f;
  if (a.mass != nullptr) {
    const double mass = (double)a.mass[t];
#pragma unroll
    for (int j = 0; j < kPer; ++j) l[j] = (float)((double)l[j] * a.rtau - mass);
  } else {
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      l[j] = (l[j] - top) * a.inv_tau;
      sum += id[j] >= 0 ? expf(l[j]) : 0.0f;
    }
    const float mass = logf(rbp::lp::wave_sum(sum));
#pragma unroll
    for (int j = 0; j < kPer; ++j) l[j] -= mass;
  }
  double A = 0.0, mass = 0.0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int k = j * 64 + lane;
    const float p = id[j] >= 0 ? expf(l[j]) : 0.0f;
    P += p;
    if (k >= a.K) {
      if (k < ((a.K + 3) & ~3)) id_s[k] = -1, p_s[k] = 0.0f;
    } else {
      const float zk = id[j] >= 0 && id[j] < a.V ? value(row[id[j]]) : NAN;
      id_s[k] = id[j];
      p_s[k] = p;
      z_s[k] = zk;
      lp_s[k] = l[j];
      if (p != 0.0f) {
        A += (double)p * ((double)l[j] - (double)zk * a.rtau);
        mass += (double)p;
      }
    }
  }
  return {rbp::lp::wave_sum(P), wave_sum(A), wave_sum(mass), top > -INFINITY || nan > 0.0f};
}

// The mass of an id over all entries that name it.
__device__ __forceinline__ float mass_of(int32_t id, const int32_t* id_s, const float* p_s,
                                         int32_t K) {
  float all = 0.0f;
#pragma unroll 2
  for (int i = 0; i < K; i += 4) {
    const int4 o = *reinterpret_cast<const int4*>(id_s + i);
    const float4 q = *reinterpret_cast<const float4*>(p_s + i);
    all += (o.x == id ? q.x : 0.0f) + (o.y == id ? q.y : 0.0f) + (o.z == id ? q.z : 0.0f) +
           (o.w == id ? q.w : 0.0f);
  }
  return all;
}

// A block per token.  Each thread keeps kHold pieces of the row in registers, so
// that a row of up to kThreads * kHold pieces is read from memory once; the
// pieces beyond them are read again for the gradient.  The first wave prepares
// the teacher's entries while the row arrives.  An element that the teacher
// names gets its gradient a second time, behind a barrier, so that the loop over
// the row looks for nothing.  16384 x 152064 bf16 1.92 ms (5.2 TB/s), 1301 x 151936
// fp32 317 us (5.0 TB/s, the pieces read twice not counted), 3003 x 151936 bf16
// without a gradient 150 us (6.1 TB/s).
template <class X, int kThreads, int kHold, bool kGrad, bool kBypass>
__global__ void __launch_bounds__(kThreads) distill_row_kernel(const X* z, X* dz, Args a) {
  constexpr int E = Row<X>::E, kWaves = kThreads / 64;
  __shared__ float m_s[kWaves], s_s[kWaves];
  __shared__ float mass_s;                       // P
  __shared__ int32_t any_s;
  __shared__ __attribute__((aligned(16))) int32_t id_s[kMaxK];
  __shared__ __attribute__((aligned(16))) float p_s[kMaxK];
  __shared__ float z_s[kMaxK], lp_s[kMaxK];
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
    const Teacher te = teacher_entries(a, t, row, lane, id_s, p_s, z_s, lp_s);
    if (lane == 0) {
      mass_s = te.P;
      any_s = te.any;
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
    const double lse = lse_of(M, S, a.rtau);
    double sum = 0.0;
    for (int k = lane; k < a.K; k += 64)
      if (p_s[k] != 0.0f)
        sum += (double)p_s[k] * ((double)lp_s[k] + (lse - (double)z_s[k] * a.rtau));
    const float kl = (float)wave_sum(sum);
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
      to(grad[id], f * exp2_hw((z_s[k] - M) * k2) - cw * mass_of(id, id_s, p_s, a.K));
    }
  }
}

// ---- few rows -------------------------------------------------------------------

// With few rows (row_parts), `parts` blocks (a power of two, up to 64)
// share a row: the first launch leaves each part's reference and sum, and what
// the teacher says of the row; the second joins them in every block, writes the
// gradient of the block's part, and in one more block the KLs and their sums.
constexpr int kPartThreads = 256;
struct PartsWs {
  float2* stats;  // [T][parts] reference, sum
  double2* A;     // [T] sum of p (log p - z / tau), sum of p
  float2* row;    // [T] P, 1 if the row counts
  float* p;       // [T][K]
  int parts;
};

// (M, S) of a row from its parts, lane j of `parts` lanes holding part j.
__device__ __forceinline__ float2 join(float2 part, int parts, float k2) {
  float M = part.x;
  for (int off = parts >> 1; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor(M, off, 64));
  float S = part.x == -INFINITY ? part.y : part.y * exp2_hw((part.x - M) * k2);
  for (int off = parts >> 1; off >= 1; off >>= 1) S += __shfl_xor(S, off, 64);
  return make_float2(M, S);
}

template <class X>
__global__ void __launch_bounds__(kPartThreads) distill_part_kernel(const X* __restrict__ z,
                                                                    Args a, PartsWs w) {
  constexpr int E = Row<X>::E, kWaves = kPartThreads / 64, kBatch = 4;
  __shared__ float2 s[kWaves];
  __shared__ int32_t id_s[kMaxK];
  __shared__ float p_s[kMaxK], z_s[kMaxK], lp_s[kMaxK];
  const int64_t t = blockIdx.x / w.parts;
  const int part = blockIdx.x % w.parts;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (a.seq[t] < 0) return;
  const X* row = z + t * a.ld;
  const Row<X> r(row, a.V);
  const int32_t end = (int32_t)((int64_t)r.pieces * (part + 1) / w.parts);
  int32_t c = (int32_t)((int64_t)r.pieces * part / w.parts) + tid;
  const float k2 = a.inv_tau * kLog2e, slack = fminf(kSlack / k2, 1e30f);
  Online o;
  const int32_t loose = part == 0 ? r.loose(tid) : -1;
  const float edge[1] = {loose >= 0 ? value(row[loose]) : -INFINITY};
  for (; c < end; c += kBatch * kPartThreads) {
    uint4 v[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (c + i * kPartThreads < end)
        v[i] = *reinterpret_cast<const uint4*>(row + r.at(c + i * kPartThreads));
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (c + i * kPartThreads < end) {
        float x[E];
        unpack(v[i], x);
        o.add(x, k2, slack);
      }
  }
  o.add(edge, k2, slack);
  const float2 mine = join(make_float2(o.m, o.s), 64, k2);
  if (lane == 0) s[wave] = mine;
  if (part == 0 && wave == kWaves - 1) {
    const Teacher te = teacher_entries(a, t, row, lane, id_s, p_s, z_s, lp_s);
    for (int k = lane; k < a.K; k += 64) w.p[t * a.K + k] = p_s[k];
    if (lane == 0) {
      w.A[t] = make_double2(te.A, te.mass);
      w.row[t] = make_float2(te.P, te.any ? 1.0f : 0.0f);
    }
  }
  __syncthreads();
  if (wave == 0) {
    const float2 all = join(lane < kWaves ? s[lane] : make_float2(-INFINITY, 0.0f), kWaves, k2);
    if (lane == 0) w.stats[t * w.parts + part] = all;
  }
}

template <class X>
__global__ void __launch_bounds__(kPartThreads) distill_join_kernel(const X* z, X* dz, Args a,
                                                                    PartsWs w, int64_t T,
                                                                    float* loss_accum,
                                                                    float* stats) {
  constexpr int E = Row<X>::E, kBatch = 4;
  __shared__ __attribute__((aligned(16))) int32_t id_s[kMaxK];
  __shared__ __attribute__((aligned(16))) float p_s[kMaxK];
  __shared__ float z_s[kMaxK];
  __shared__ double sum_s[3][kPartThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float k2 = a.inv_tau * kLog2e;
  if (blockIdx.x == 0) {  // KL of the rows and the sums over them
    double v[3] = {0.0, 0.0, 0.0};
    const int64_t n = T * w.parts;
    for (int64_t i0 = 0; i0 < n; i0 += kPartThreads) {
      const int64_t i = i0 + tid, t = i / w.parts;
      const bool in = i < n, counts = in && a.seq[t] >= 0 && w.row[t].y > 0.0f;
      const float2 all = join(counts ? w.stats[i] : make_float2(-INFINITY, 0.0f), w.parts, k2);
      if (!in || i % w.parts != 0) continue;
      float kl = 0.0f;
      if (counts) {
        kl = (float)(w.A[t].x + w.A[t].y * lse_of(all.x, all.y, a.rtau));
        v[0] += a.weight / (float)a.len[a.seq[t]] * kl;
        v[1] += 1.0;
        v[2] += kl;
      }
      a.kl[t] = kl;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      for (int off = 32; off >= 1; off >>= 1) v[k] += __shfl_xor(v[k], off, 64);
      if (lane == 0) sum_s[k][wave] = v[k];
    }
    __syncthreads();
    if (tid >= 3) return;
    double sum = 0.0;
    for (int q = 0; q < kPartThreads / 64; ++q) sum += sum_s[tid][q];
    float* to_ = tid == 0 ? loss_accum : stats + (tid - 1);
    *to_ = (float)((double)*to_ + sum);
    return;
  }
  const int64_t t = (blockIdx.x - 1) / w.parts;
  const int part = (blockIdx.x - 1) % w.parts;
  const X* row = z + t * a.ld;
  X* grad = dz + t * a.ld;
  const Row<X> r(row, a.V);
  const bool vec =
      ((reinterpret_cast<uintptr_t>(row) ^ reinterpret_cast<uintptr_t>(grad)) & 15) == 0;
  const int32_t begin = (int32_t)((int64_t)r.pieces * part / w.parts),
                end = (int32_t)((int64_t)r.pieces * (part + 1) / w.parts);
  const int32_t loose = part == 0 ? r.loose(tid) : -1;
  const int32_t sq = a.seq[t];
  const bool counts = sq >= 0 && w.row[t].y > 0.0f;
  auto put = [&](int32_t piece, const uint4& v) {
    X* to_ = grad + r.at(piece);
    if (vec) {
      *reinterpret_cast<uint4*>(to_) = v;
    } else {
      X e[E];
      __builtin_memcpy(e, &v, 16);
#pragma unroll
      for (int k = 0; k < E; ++k) to_[k] = e[k];
    }
  };
  if (!counts) {
    for (int32_t c = begin + tid; c < end; c += kPartThreads) put(c, make_uint4(0u, 0u, 0u, 0u));
    if (loose >= 0) grad[loose] = X(0);
    return;
  }
  for (int k = tid; k < ((a.K + 3) & ~3); k += kPartThreads) {
    const int32_t id = k < a.K ? a.ids[t * a.K + k] : -1;
    id_s[k] = id;
    p_s[k] = k < a.K ? w.p[t * a.K + k] : 0.0f;
  }
  const float2 all =
      join(lane < w.parts ? w.stats[t * w.parts + lane] : make_float2(-INFINITY, 0.0f), w.parts, k2);
  const float M = __shfl(all.x, 0, 64), S = __shfl(all.y, 0, 64);
  const float cw = a.weight / (float)a.len[sq] * a.inv_tau, f = cw * w.row[t].x / S;
  auto scaled = [&](float x) { return f * exp2_hw((x - M) * k2); };
  const float edge = loose >= 0 ? value(row[loose]) : 0.0f;
  __syncthreads();
  // the policy's logits that this part's entries name, before the gradient may
  // take their place
  auto in_part = [&](int32_t id) {
    const int32_t p = (id - r.head) / E;
    return id >= 0 && id < a.V &&
           (id < r.head || p >= r.pieces ? part == 0 : p >= begin && p < end);
  };
  for (int k = tid; k < a.K; k += kPartThreads)
    if (in_part(id_s[k])) z_s[k] = value(row[id_s[k]]);
  __syncthreads();
  for (int32_t c = begin + tid; c < end; c += kBatch * kPartThreads) {
    uint4 v[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (c + i * kPartThreads < end)
        v[i] = *reinterpret_cast<const uint4*>(row + r.at(c + i * kPartThreads));
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (c + i * kPartThreads < end) {
        float x[E];
        unpack(v[i], x);
#pragma unroll
        for (int k = 0; k < E; ++k) x[k] = scaled(x[k]);
        put(c + i * kPartThreads, pack(x));
      }
  }
  if (loose >= 0) to(grad[loose], scaled(edge));
  __syncthreads();
  for (int k = tid; k < a.K; k += kPartThreads)
    if (in_part(id_s[k])) to(grad[id_s[k]], scaled(z_s[k]) - cw * mass_of(id_s[k], id_s, p_s, a.K));
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

// Blocks that share a row, 1 for a block per row.  Sharing pays for up to 64 rows
// of long vocabularies (bf16, one block against shared: 1 x 151936 23.4 / 10.0 us,
// 32 24.6 / 15.3, 64 25.1 / 20.6, 128 28.4 / 32.0; 1 x 16000 11.0 / 9.5, 64 x 16000
// fp32 10.6 / 11.6).  The type does not enter: a workspace is sized without it.
constexpr int64_t kFewRows = 64, kPartBlocks = 512, kRowElements = 512;
constexpr int32_t kLongRow = 8192;
constexpr int kMostParts = 64;
int row_parts(int64_t T, int32_t V) {
  int parts = 1;
  if (T <= kFewRows && V >= kLongRow && V >= kRowElements * T)
    while (parts < kMostParts && T * parts < kPartBlocks && V / (2 * parts) >= 2048) parts *= 2;
  return parts;
}

struct DistillWs {
  float* terms;
  PartsWs w;
  size_t bytes;
};

// Room for every batch of up to T rows, shared ones and others: one sized for the largest
// batch serves all.
DistillWs carve_distill(void* base, int64_t T, int32_t K, int32_t V) {
  rbp::WsCarver c(base);
  DistillWs d{};
  d.w.parts = row_parts(T, V);
  d.terms = c.take<float>((size_t)T * 2);
  const int64_t shared =
      V < kLongRow ? 0 : std::min(std::min(T, kFewRows), (int64_t)V / kRowElements);
  if (shared > 0) {
    d.w.A = c.take<double2>((size_t)shared);
    d.w.stats = c.take<float2>((size_t)std::min(shared * kMostParts, 2 * kPartBlocks));
    d.w.row = c.take<float2>((size_t)shared);
    d.w.p = c.take<float>((size_t)shared * K);
  }
  d.bytes = rbp::align_up(c.used, 256);
  return d;
}

template <class X>
void launch_parts(const X* z, X* dz, int64_t T, const Args& a, const PartsWs& w, float* loss_accum,
                  float* stats, hipStream_t s) {
  const int64_t blocks = T * w.parts;
  hipLaunchKernelGGL(distill_part_kernel<X>, dim3((unsigned)blocks), dim3(kPartThreads), 0, s, z, a,
                     w);
  hipLaunchKernelGGL(distill_join_kernel<X>, dim3((unsigned)(dz == nullptr ? 1 : 1 + blocks)),
                     dim3(kPartThreads), 0, s, z, dz, a, w, T, loss_accum, stats);
}

}  // namespace

size_t rbp::distill_ws(int64_t T, int32_t K, int32_t V) {
  return carve_distill(nullptr, T < 1 ? 1 : T, K < 1 ? 1 : K, V < 1 ? 1 : V).bytes;
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
  RBP_REQUIRE(temperature >= 0x1p-100f && temperature <= 0x1p100f && std::isfinite(scale),
              RBP_EINVAL, "policy_distill_fwd_bwd: need a temperature in [2^-100, 2^100] and a "
              "finite scale");
  RBP_REQUIRE(K <= kMaxK, RBP_EUNSUPPORTED, "policy_distill_fwd_bwd: K above %d", kMaxK);
  // (a block of up to 1024 threads a token: less than 2^32 in all)
  RBP_REQUIRE(T < (1 << 22), RBP_EUNSUPPORTED, "policy_distill_fwd_bwd: T of 2^22 or more");
  RBP_REQUIRE(V <= rbp::rows::kMaxVocab, RBP_EUNSUPPORTED,
              "policy_distill_fwd_bwd: V above 2^31 - 2^14 - 1");
  RBP_REQUIRE(loss_accum && stats && seq_len, RBP_EINVAL, "policy_distill_fwd_bwd: null pointer");
  if (T == 0) return RBP_OK;
  RBP_REQUIRE(logits && teacher_ids && teacher_logits && seq_of_token && kl, RBP_EINVAL,
              "policy_distill_fwd_bwd: null per-token pointer");
  const size_t es = logits_type == RBP_F32 ? 4 : 2;
  RBP_REQUIRE(aligned(logits, es) && aligned(dlogits, es) && aligned(ws, 16), RBP_EINVAL,
              "policy_distill_fwd_bwd: logits or dlogits not aligned to their type, or ws to 16 "
              "bytes");
  const size_t need = rbp::distill_ws(T, K, V);
  RBP_REQUIRE(ws && ws_bytes >= need, RBP_EWORKSPACE,
              "policy_distill_fwd_bwd: workspace needs %zu bytes, got %zu", need, ws_bytes);
  hipStream_t s = rbp::as_stream(stream);
  const DistillWs d = carve_distill(ws, T, K, V);
  const Args a{ld, teacher_ids, teacher_logits, teacher_lse, seq_of_token, seq_len, V, K,
               1.0f / temperature, (float)((double)scale / (double)n_seq_total),
               1.0 / (double)temperature, kl, d.terms};
  auto go = [&](auto type) {
    using X = decltype(type);
    const X* z = static_cast<const X*>(logits);
    X* dz = static_cast<X*>(dlogits);
    if (d.w.parts > 1) {
      launch_parts(z, dz, T, a, d.w, loss_accum, stats, s);
    } else {
      launch_rows(z, dz, T, a, s);
      hipLaunchKernelGGL(distill_sum_kernel, dim3(1), dim3(1024), 0, s, d.terms, kl, T, loss_accum,
                         stats);
    }
  };
  if (logits_type == RBP_F32)
    go(float{});
  else
    go(uint16_t{});
  RBP_CHECK_LAUNCH("policy_distill_fwd_bwd");
  return RBP_OK;
}
