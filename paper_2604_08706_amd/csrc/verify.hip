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
// exact ones in about one draw in a hundred.  So the sums of the row that is drawn
// from are in 64 bits, whose operations this chip runs at the rate of 32-bit ones (52
// lanes a clock and compute unit measured), but an exponential takes 13 of them.
//
// Every row is cut into segments of consecutive tokens, a wave each: the running sum
// of a whole row exists only by segments.  Without draft logits, two launches: the
// segments' 64-bit sums (stats); then a block per sequence (finish) decides, finds the
// segment that u_K falls into, and the token inside it.  With draft logits, where there
// are twice the rows and two of them are drawn from, three: 32-bit sums of all rows
// (rough), which the load of the logits bounds -- 576 rows of 152064 bf16 in 60 us in 64
// bits --; 64-bit sums of the rows to draw from (exact), whose blocks decide first, an
// acceptance too near for the rough sums by a 64-bit pass over its two rows; finish.

#include <algorithm>
#include <cmath>

#include "rbp_internal.h"
#include "vocab_rows.h"

namespace {

using rbp::rows::aligned;
using rbp::rows::Row;
using rbp::rows::unpack;
using rbp::rows::value;

constexpr double kLog2eD = 1.4426950408889634074;
constexpr double kLn2 = 0.69314718055994530942;

// 2^y for y <= 1000, to 1.5e-14: the nearest integer apart, a polynomial for the
// rest, whose coefficients are a least-squares fit of the relative error on
// [-1/2, 1/2] that was reweighted until it was level, with 2^0 = 1 exactly.  -inf
// and everything below -1100 give 0; so does a NaN (rows with one are found by
// their largest logit).
__device__ __forceinline__ double exp2_d(double y) {
  y = fmax(y, -1100.0);
  const double t = y + 0x1.8p52;
  const double f = y - (t - 0x1.8p52);
  double p = 0x1.b3dde4196d3a9p-24;
  p = fma(p, f, 0x1.63e69a73f6558p-20);
  p = fma(p, f, 0x1.ffce301d64a90p-17);
  p = fma(p, f, 0x1.430897ef02c7ep-13);
  p = fma(p, f, 0x1.5d87fd9362c75p-10);
  p = fma(p, f, 0x1.3b2ab72414d27p-7);
  p = fma(p, f, 0x1.c6b08d70c8985p-5);
  p = fma(p, f, 0x1.ebfbdff81bde4p-3);
  p = fma(p, f, 0x1.62e42fefa37d1p-1);
  return __builtin_amdgcn_ldexp(fma(p, f, 1.0), __double2loint(t));
}

// The same where whole rows are summed, to 8e-14: 2^(x k2) as a power of two, a root
// from a table of 32 in LDS (banks of their own: no conflicts; 128 roots and one
// multiplication less took as long), and a polynomial of degree 4 instead of 9, fitted
// likewise.  With n = rint(32 x k2), the sum of 32 x k2 and 1.5 2^52 - c (c an integer
// near the reference's 32 ref k2) holds n - c in its low bits: three operations for n
// and the fraction, exact before the last rounding.
constexpr int kRoots = 32;
__constant__ double g_roots[kRoots] = {
    0x1.0000000000000p+0, 0x1.059b0d3158574p+0, 0x1.0b5586cf9890fp+0, 0x1.11301d0125b51p+0,
    0x1.172b83c7d517bp+0, 0x1.1d4873168b9aap+0, 0x1.2387a6e756238p+0, 0x1.29e9df51fdee1p+0,
    0x1.306fe0a31b715p+0, 0x1.371a7373aa9cbp+0, 0x1.3dea64c123422p+0, 0x1.44e086061892dp+0,
    0x1.4bfdad5362a27p+0, 0x1.5342b569d4f82p+0, 0x1.5ab07dd485429p+0, 0x1.6247eb03a5585p+0,
    0x1.6a09e667f3bcdp+0, 0x1.71f75e8ec5f74p+0, 0x1.7a11473eb0187p+0, 0x1.82589994cce13p+0,
    0x1.8ace5422aa0dbp+0, 0x1.93737b0cdc5e5p+0, 0x1.9c49182a3f090p+0, 0x1.a5503b23e255dp+0,
    0x1.ae89f995ad3adp+0, 0x1.b7f76f2fb5e47p+0, 0x1.c199bdd85529cp+0, 0x1.cb720dcef9069p+0,
    0x1.d5818dcfba487p+0, 0x1.dfc97337b9b5fp+0, 0x1.ea4afa2a490dap+0, 0x1.f50765b6e4540p+0};
__device__ __forceinline__ void load_roots(double* roots) {
  const int i = threadIdx.x;
  if (i < kRoots)
    roots[i] = __hiloint2double(__double2hiint(g_roots[i]) - (i << 15), __double2loint(g_roots[i]));
}
struct Scaled {
  double p, root;  // their product is 2^(x k2 - c / 32)
};
struct Grid {
  double k, c;   // 32 k2; 1.5 2^52 minus the integer
  double shift;  // (the integer) / 32
  float floor;   // logits below are taken for this one: 2^-1000 beside the reference
  // Whether the reference and the temperature allow it; where not (logits beyond
  // 2^24 temperatures, temperatures beyond 1e27) exp2_d serves.
  bool near;
  __device__ __forceinline__ void refer(double ref, double k2, double span) {
    k = kRoots * k2;
    const double n = rint(ref * k);
    c = 0x1.8p52 - n;
    shift = n * (1.0 / kRoots);
    const double low = ref - span;
    near = fabs(ref) * k2 < 0x1p24 && low > -1e30;
    floor = (float)low;
  }
  // (fmaxf would quiet each operand first; a NaN may pass)
  __device__ __forceinline__ void clamp(float& z) const {
    asm("v_max_f32 %0, %1, %2" : "=v"(z) : "v"(z), "v"(floor));
  }
  // Exponentials of N clamped logits: the roots' loads of all, then the polynomials.
  template <int N>
  __device__ __forceinline__ void operator()(const float (&z)[N], const double* roots,
                                             Scaled (&y)[N]) const {
    double f[N], r[N];
    int n[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const double x = (double)z[i], t = fma(x, k, c);
      f[i] = fma(x, k, c - t);
      n[i] = __double2loint(t);
      r[i] = roots[n[i] & (kRoots - 1)];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      double p = 0x1.3b2aa27434ff1p-27;
      p = fma(p, f[i], 0x1.c6b167e2738bcp-20);
      p = fma(p, f[i], 0x1.ebfbdff87858dp-13);
      p = fma(p, f[i], 0x1.62e42fef6d042p-6);
      y[i].p = fma(p, f[i], 1.0);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      // n / 32 goes into the exponent, which stays in range; what n % 32 adds below it
      // is off the table's
      y[i].root = __hiloint2double((n[i] << 15) + __double2hiint(r[i]), __double2loint(r[i]));
    }
  }
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

__device__ __forceinline__ float uniform(float v) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v)));
}
// The value of one lane, the same in all.
__device__ __forceinline__ double lane_of(double v, int lane) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane),
                          __builtin_amdgcn_readlane(__double2loint(v), lane));
}

// s = sum of 2^((z - m) k2) over some logits; m = -inf and s = 0 for none but
// -inf, and s a NaN where one is.
struct Part {
  double s;
  float m, pad;
};

// Sums over some tokens of a row to draw from: 2^((z - m) k2) of the policy (p) and of
// the draft (q), and both over the tokens where the policy's probability is larger (a,
// b): there max(p - q, 0) = p - q, so its sum is a / sum p - b / sum q.  Which tokens
// these are is told by the rough sums; `near` is the sum of p over those that they may
// mistake.
struct Drawn {
  double p, q, a, b, near;
};

struct Args {
  int64_t ld, ld_draft;
  const int32_t *draft_tokens, *n_draft;
  const float* u;
  int32_t B, K, V, segments, log_segments;
  double k2;    // log2 e / temperature
  double span;  // 1000 / k2
  float slack;  // kSlack / k2
  int32_t* out_tokens;
  float* out_logp;
  int32_t* n_out;
  Part* parts;  // [B][K + 1 + K][segments]: the policy's rows, then the draft's
  Drawn* drawn;  // [B][segments][kShares]
  __device__ __forceinline__ int32_t drafts(int64_t b) const {
    return n_draft == nullptr ? K : min(n_draft[b], K);
  }
};

// Tokens of a segment: whole pieces, with the loose elements at a row's ends.
template <class X>
struct Segment {
  int32_t p0, p1, v0, v1;  // pieces, tokens
  __device__ __forceinline__ Segment(const Row<X>& r, int seg, int log_n) {
    p0 = (int32_t)(((int64_t)r.pieces * seg) >> log_n);
    p1 = (int32_t)(((int64_t)r.pieces * (seg + 1)) >> log_n);
    v0 = seg == 0 ? 0 : r.at(p0);
    v1 = (seg + 1) >> log_n ? r.V : r.at(p1);
  }
};

// The row and segment of a wave of the first launch, none where its position has no
// draft.
template <class X>
struct Place {
  const X* row;
  uint32_t row_id;
  int seg;
  bool kept;  // a row of the policy's whose draft may be accepted
};
template <bool kDrafts, class X>
__device__ __forceinline__ Place<X> place_of(const X* logits, const X* draft_logits, const Args& a,
                                             int64_t n_items) {
  Place<X> p{nullptr, 0, 0, false};
  // (rows times segments may pass 31 bits, rows may not)
  const int64_t item = (int64_t)blockIdx.x * (blockDim.x >> 6) +
                       __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (item >= n_items) return p;
  p.seg = (int)(item & (a.segments - 1));
  p.row_id = (uint32_t)(item >> a.log_segments);
  const uint32_t rows = kDrafts ? 2 * a.K + 1 : a.K + 1;
  const int64_t b = p.row_id / rows;
  const int k = (int)(p.row_id % rows);
  const int32_t n = a.drafts(b);  // (negative: no row)
  if (k <= a.K) {
    if (k <= n) p.row = logits + (b * (a.K + 1) + k) * a.ld;
    p.kept = k < n;
  } else if constexpr (kDrafts) {
    const int at = k - a.K - 1;
    if (at < n) p.row = draft_logits + (b * a.K + at) * a.ld_draft;
  }
  return p;
}

constexpr int kStatsThreads = 256;
// the reference follows the largest logit once it is that many powers of two above
constexpr double kSlack = 200.0;
constexpr float kRoughSlack = 8.0f;

// A wave per segment of a row, in 32 bits: s by pieces of exponentials whose argument y
// is off by 3 2^-24 |y|, and they by one unit in the last place.  Weighted by the
// probabilities, |y| is at most log2 V + 2 kRoughSlack (the entropy bounds the distance
// from the largest logit; the reference lags behind it, and moves), so the sum of a row
// of 2^18 tokens is off by 5e-6 of itself at most, one of 2^31 by 7e-6, and p / q by
// less than kUnsure.  Bound by HBM: 576 rows of 152064 bf16 32 us (5.4 TB/s), 34 with 256 of
// them summed as the struct after this one does.
constexpr double kUnsure = 0x1p-16;
struct Rough {
  float m = -INFINITY;
  double s = 0.0;
  float k2, slack;
  __device__ __forceinline__ explicit Rough(const Args& a)
      : k2((float)a.k2), slack(fminf(kRoughSlack / k2, 1e30f)) {}
  __device__ __forceinline__ double sum() const { return s; }
  template <int N>
  __device__ __forceinline__ void add(const float (&x)[N]) {
    float top = x[0];
#pragma unroll
    for (int k = 1; k < N; ++k) top = fmaxf(top, x[k]);
    if (top > m + slack) {
      s *= (double)rbp::lp::exp2_hw((m - top) * k2);
      m = top;
    }
    const float ref = m == -INFINITY ? 0.0f : m;
    float e[N];
#pragma unroll
    for (int k = 0; k < N; ++k) e[k] = rbp::lp::exp2_hw((x[k] - ref) * k2);
#pragma unroll
    for (int w = N / 2; w >= 1; w /= 2)
#pragma unroll
      for (int k = 0; k < w; ++k) e[k] += e[k + w];
    s += (double)e[0];
  }
};

// The same for the policy's rows whose drafts may be accepted, since their sums are in those
// tokens' log-probs, without the roundings of the argument d k2.
// - The difference d loses nothing: the reference is 0 while the largest logit is within 64
//   powers of two of it, else a logit at most 32 below the largest: those that matter differ
//   from it by less than half of it.
// - What the product of d and k2's 32 bits loses (l: 2^l is 1 + l ln 2) is summed beside it, in c.
// - What k2's 32 bits lose, `lo`, up to 2^-24 of it, counts lo d for the largest of a piece and
//   its other elements alike: weighted, those are 3 powers of two less at most.
// So a sum is off by its exponentials' errors (1.43 2^-24 at most, over all arguments), three
// additions of eight (3 2^-24) and 3 ln 2 2^-24 for the third point: 6.6 2^-24 of itself at most.
struct Fine {
  static constexpr float kNear = 64.0f, kGone = -160.0f;  // in powers of two
  float m = -INFINITY, top = -INFINITY, c = 0.0f;
  float limit = -INFINITY;  // a logit above it moves the reference
  double s = 0.0, k2;
  float hi, lo, near, gone;
  __device__ __forceinline__ explicit Fine(const Args& a)
      : k2(a.k2), hi((float)k2), lo((float)(k2 - (double)hi)), near(kNear / hi), gone(kGone / hi) {}
  // (a row with a NaN has no sum; the clamp below lets none through)
  __device__ __forceinline__ double sum() const {
    return top != top ? (double)NAN : fma((double)c, kLn2, s);
  }
  template <int N>
  __device__ __forceinline__ void add(const float (&x)[N]) {
    float largest = x[0];
#pragma unroll
    for (int k = 1; k < N; ++k) largest = __builtin_elementwise_maximum(largest, x[k]);
    top = __builtin_elementwise_maximum(top, largest);
    if (largest > limit) {
      const float to = fabsf(largest) <= near ? 0.0f : largest;
      if (m != -INFINITY) {
        const double f = exp2_d(((double)m - (double)to) * k2);
        s *= f;
        c *= (float)f;
      }
      m = to;
      limit = to == 0.0f ? near : to + 0.5f * near;
    }
    const float ref = m == -INFINITY ? 0.0f : m;
    float e[N], l[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float d = fmaxf(x[k] - ref, gone), y = d * hi;
      l[k] = fmaf(d, hi, -y);
      e[k] = rbp::lp::exp2_hw(y);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) c = fmaf(e[k], l[k], c);
#pragma unroll
    for (int w = N / 2; w >= 1; w /= 2)
#pragma unroll
      for (int k = 0; k < w; ++k) e[k] += e[k + w];
    c = fmaf(e[0], fmaxf(largest - ref, gone) * lo, c);
    s += (double)e[0];
  }
};
template <class X>
__global__ void __launch_bounds__(kStatsThreads) rough_kernel(const X* __restrict__ logits,
                                                              const X* __restrict__ draft_logits,
                                                              Args a, int64_t n_items) {
  constexpr int E = Row<X>::E, kBatch = 4;
  const Place<X> place = place_of<true, X>(logits, draft_logits, a, n_items);
  if (place.row == nullptr) return;
  const int lane = threadIdx.x & 63;
  const Row<X> r(place.row, a.V);
  const Segment<X> g(r, place.seg, a.log_segments);
  auto run = [&](auto o) {
    for (int32_t c = g.p0 + lane; c < g.p1; c += kBatch * 64) {
      uint4 v[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        if (c + i * 64 < g.p1) v[i] = *reinterpret_cast<const uint4*>(place.row + r.at(c + i * 64));
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        if (c + i * 64 < g.p1) {
          float x[E];
          unpack(v[i], x);
          o.add(x);
        }
    }
    const int32_t loose = r.loose(lane);
    if (loose >= 0 && (loose < r.head ? place.seg == 0 : place.seg == a.segments - 1)) {
      const float x[1] = {value(place.row[loose])};
      o.add(x);
    }
    float M = o.m;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor(M, off, 64));
    double s = o.sum();
    if (o.m != M) s *= exp2_d(((double)o.m - (double)M) * a.k2);
    s = wave_sum(s);
    if (lane == 0) a.parts[(int64_t)place.row_id * a.segments + place.seg] = Part{s, M, 0.0f};
  };
  if (place.kept)
    run(Fine(a));
  else
    run(Rough(a));
}

// A wave per segment of a row, in 64 bits: bound by its 13 64-bit operations a logit
// and, with few rows, latency.  192 rows of 151936 fp32 21 us (5.5 TB/s), 5 of bf16 5 us.
template <class X>
__global__ void __launch_bounds__(kStatsThreads) stats_kernel(const X* __restrict__ logits,
                                                              Args a, int64_t n_items) {
  constexpr int E = Row<X>::E, kBatch = 4;
  __shared__ double roots[kRoots];
  load_roots(roots);
  __syncthreads();
  const Place<X> place = place_of<false, X>(logits, nullptr, a, n_items);
  if (place.row == nullptr) return;
  const X* row = place.row;
  const int seg = place.seg, lane = threadIdx.x & 63;
  const Row<X> r(row, a.V);
  const Segment<X> g(r, seg, a.log_segments);
  float m = -INFINITY, top = -INFINITY;
  double s = 0.0;  // relative to 2^(grid.shift), or to the reference where that is far
  Grid grid;
  grid.refer(0.0, a.k2, a.span);
  auto refer = [&](float largest) {
    top = __builtin_elementwise_maximum(top, largest);
    if (largest > m + a.slack) {
      const Grid old = grid;
      grid.refer((double)largest, a.k2, a.span);
      if (m == -INFINITY)
        s = 0.0;
      else if (old.near && grid.near)
        s *= exp2_d(old.shift - grid.shift);
      else
        s *= exp2_d((old.near ? old.shift : (double)m * a.k2) - (double)largest * a.k2);
      m = largest;
    }
  };
  auto add = [&](const uint4& piece) {
    float x[E];
    unpack(piece, x);
    float largest = x[0];
#pragma unroll
    for (int i = 1; i < E; ++i) largest = __builtin_elementwise_maximum(largest, x[i]);
    refer(largest);
    if (!grid.near) {
#pragma unroll 1
      for (int i = 0; i < E; ++i) {
        s += exp2_d(((double)x[0] - (double)m) * a.k2);
#pragma unroll
        for (int j = 1; j < E; ++j) x[j - 1] = x[j];
      }
      return;
    }
    double e[4] = {s, 0.0, 0.0, 0.0};  // sums of their own: no chain of 8 additions
    Scaled y[E];
#pragma unroll
    for (int i = 0; i < E; ++i) grid.clamp(x[i]);
    grid(x, roots, y);
#pragma unroll
    for (int i = 0; i < E; ++i) e[i & 3] = fma(y[i].p, y[i].root, e[i & 3]);
    s = (e[0] + e[1]) + (e[2] + e[3]);
  };
  for (int32_t c = g.p0 + lane; c < g.p1; c += kBatch * 64) {
    uint4 v[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (c + i * 64 < g.p1) v[i] = *reinterpret_cast<const uint4*>(row + r.at(c + i * 64));
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (c + i * 64 < g.p1) add(v[i]);
  }
  const int32_t loose = r.loose(lane);
  if (loose >= 0 && (loose < r.head ? seg == 0 : seg == a.segments - 1)) {
    const float x = value(row[loose]);
    refer(x);
    s += exp2_d(grid.near ? fma((double)x, a.k2, -grid.shift) : ((double)x - (double)m) * a.k2);
  }
  float M = m;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    M = fmaxf(M, __shfl_xor(M, off, 64));
    top = __builtin_elementwise_maximum(top, __shfl_xor(top, off, 64));
  }
  // relative to the largest reference
  s = m == -INFINITY ? 0.0
      : s * exp2_d(grid.near ? fma((double)-M, a.k2, grid.shift)
                             : ((double)m - (double)M) * a.k2);
  s = wave_sum(s);
  if (lane == 0)
    a.parts[(int64_t)place.row_id * a.segments + seg] =
        Part{top != top ? (double)NAN : s, M, 0.0f};
}

// A row's reference and sum from its segments, by one wave; sum is NaN or 0 where
// the row has no distribution.
struct Dist {
  double m, sum, ls;  // p = 2^((z - m) k2 - ls), ls = log2 sum
  __device__ __forceinline__ double log2_of(float z, double k2) const {
    return fma((double)z - m, k2, -ls);
  }
  __device__ __forceinline__ bool valid() const { return sum > 0.0 && sum < INFINITY; }
};
__device__ __forceinline__ Dist dist_of(const Part* parts, int n, double k2, int lane) {
  const Part p = lane < n ? parts[lane] : Part{0.0, -INFINITY, 0.0f};
  float M = p.m;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor(M, off, 64));
  Dist d;
  d.m = (double)M;
  d.sum = wave_sum(p.m == M || p.s != p.s ? p.s : p.s * exp2_d(((double)p.m - (double)M) * k2));
  if (!(M < INFINITY)) d.sum = NAN;
  d.ls = log2(d.sum);
  return d;
}

constexpr int kMaxK = 255;
constexpr int kShares = 2;  // waves of a segment in exact_kernel
// A total of max(p - q, 0) that counts as 0.  It is a difference of sums whose exponentials are
// off by 8e-14, so by 4e-13 at most; above this, by 3 in a hundred of itself at most.
constexpr double kNothing = 0x1p-36;
constexpr int kFinishThreads = 1024;
// Tokens of a thread: a segment of up to 5120 in one tile, as of 152064 in 32 (64 sequences of 4
// drafts 67.5 us; with 3, 4 and 8 69.6, 69.9 and 69.2; 100 rows of 50000 17.1 / 16.6, 16.7, 17.7).
constexpr int kRun = 5;
constexpr int kMaxSegments = 64;

// What is decided of a sequence: drafts accepted, and the weights of the drawn
// token: 0 p, 1 p without the draft, 2 max(p - q, 0); -1: no distribution.
struct Decision {
  int32_t accepted, kind, x;
  Dist p, q;
};

// Whether draft k is accepted: 0 yes, 1 no, 2 too near for sums that are off by up to
// `unsure`.
template <class X>
__device__ __forceinline__ int test_draft(const X* __restrict__ logits,
                                          const X* __restrict__ draft_logits, const Args& a,
                                          int64_t b, int k, const Dist& p, const Dist* q,
                                          double unsure) {
  const int32_t x = a.draft_tokens[b * a.K + k];
  if (x < 0 || x >= a.V || !p.valid()) return 1;
  const double px = exp2_d(p.log2_of(value(logits[(b * (a.K + 1) + k) * a.ld + x]), a.k2));
  double qx = 1.0;
  if (q != nullptr) {
    if (!q->valid()) return 1;
    qx = exp2_d(q->log2_of(value(draft_logits[(b * a.K + k) * a.ld_draft + x]), a.k2));
  }
  const double uq = (double)a.u[b * (a.K + 1) + k] * qx;
  if (px > 0.0 && fabs(uq - px) < unsure * px) return 2;
  return uq < px ? 0 : 1;
}

// A row's sum in 64 bits, by a block.
template <class X>
__device__ double exact_sum(const X* __restrict__ row, int32_t V, double m, double k2,
                            double* wave_s) {
  double s = 0.0;
#pragma unroll 4
  for (int32_t v = threadIdx.x; v < V; v += blockDim.x)
    s += exp2_d(((double)value(row[v]) - m) * k2);
  s = wave_sum(s);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) wave_s[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) s += wave_s[w];
  return s;
}

// By a block, which takes the rows' distributions into LDS: the policy's of the
// positions 0 .. n, then the draft's.  kRough: the sums are rough.
struct DecideLds {
  int32_t first, code;
  double wave_s[16];
};
template <class X, bool kRough>
__device__ void decide(const X* __restrict__ logits, const X* __restrict__ draft_logits,
                       const Args& a, int64_t b, int32_t n, Dist* rows_s, DecideLds* lds,
                       Decision* out) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int rows = kRough ? 2 * a.K + 1 : a.K + 1;
  const Part* parts = a.parts + b * rows * a.segments;
  // row k of the policy, or k - n - 1 of the draft
  for (int k = wave; k <= (kRough ? 2 * n : n); k += waves) {
    const int row = k <= n ? k : a.K + 1 + (k - n - 1);
    const Dist d = dist_of(parts + row * a.segments, a.segments, a.k2, lane);
    if (lane == 0) rows_s[k] = d;
  }
  // the first draft from `from` on that is not accepted, 64 at a time
  auto search = [&](int32_t from) {
    __syncthreads();
    if (wave == 0) {
      int32_t first = n;
      int code = 0;
      for (int k0 = from; k0 < n && first == n; k0 += 64) {
        const int k = k0 + lane;
        const int c = k < n ? test_draft(logits, draft_logits, a, b, k, rows_s[k],
                                         kRough ? rows_s + n + 1 + k : nullptr,
                                         kRough ? kUnsure : 0.0)
                            : 0;
        const uint64_t no = __ballot(c != 0);
        if (no != 0) {
          const int j = __builtin_ctzll(no);
          first = k0 + j;
          code = __shfl(c, j, 64);
        }
      }
      if (lane == 0) {
        lds->first = first;
        lds->code = code;
      }
    }
    __syncthreads();
  };
  search(0);
  if constexpr (kRough) {
    while (lds->code == 2) {  // too near: both rows again in 64 bits
      const int32_t k = lds->first;
      Dist p = rows_s[k], q = rows_s[n + 1 + k];
      p.sum = exact_sum(logits + (b * (a.K + 1) + k) * a.ld, a.V, p.m, a.k2, lds->wave_s);
      q.sum = exact_sum(draft_logits + (b * a.K + k) * a.ld_draft, a.V, q.m, a.k2, lds->wave_s);
      p.ls = log2(p.sum);
      q.ls = log2(q.sum);
      if (test_draft(logits, draft_logits, a, b, k, p, &q, 0.0) != 0) break;
      search(k + 1);
    }
  }
  if (threadIdx.x == 0) {
    const int32_t first = lds->first;
    const bool drawn_from_p = first == n;
    out->accepted = first;
    out->x = drawn_from_p ? -1 : a.draft_tokens[b * a.K + first];
    out->p = rows_s[first];
    out->q = rows_s[drawn_from_p || !kRough ? first : n + 1 + first];
    out->kind = !out->p.valid() ? -1
                : drawn_from_p ? 0
                : !kRough ? (out->x >= 0 && out->x < a.V ? 1 : 0)
                : out->q.valid() ? 2 : 0;
  }
  __syncthreads();
}

// The accepted drafts and their log-probs, -1 and 0 (NaN where there is nothing to
// draw from) behind them, and the number of tokens.
template <class X>
__device__ __forceinline__ float logp_of(const X* row, int32_t x, const Dist& d, double k2) {
  return (float)(kLn2 * d.log2_of(value(row[x]), k2));
}
template <class X>
__device__ void emit_accepted(const X* __restrict__ logits, const Args& a, int64_t b,
                              const Decision& d, const Dist* rows_s) {
  for (int k = threadIdx.x; k <= a.K; k += blockDim.x) {
    const int64_t i = b * (a.K + 1) + k;
    const int32_t x = k < d.accepted ? a.draft_tokens[b * a.K + k] : -1;
    a.out_tokens[i] = x;
    a.out_logp[i] = x >= 0 ? logp_of(logits + i * a.ld, x, rows_s[k], a.k2)
                    : k == d.accepted && d.kind < 0 ? NAN : 0.0f;
  }
  if (threadIdx.x == 0) a.n_out[b] = d.accepted + 1;
}

// Weight of token v under a decision.
template <class X>
struct Weight {
  const X *p, *q;
  double mp, mq, lp, lq;
  int32_t kind, x;
};
template <class X>
__device__ __forceinline__ Weight<X> weight_of(const Decision& d, const X* logits,
                                               const X* draft_logits, const Args& a, int64_t b) {
  Weight<X> w;
  w.p = logits + (b * (a.K + 1) + d.accepted) * a.ld;
  w.q = d.kind == 2 ? draft_logits + (b * a.K + d.accepted) * a.ld_draft : nullptr;
  // (p itself is drawn from unnormalised, as its segments' sums are)
  w.mp = d.p.m;
  w.lp = d.kind == 2 ? d.p.ls : 0.0;
  w.mq = d.kind == 2 ? d.q.m : 0.0;
  w.lq = d.kind == 2 ? d.q.ls : 0.0;
  w.kind = d.kind;
  w.x = d.x;
  return w;
}

// Whether p > q by a decision's sums: z_p - z_q beyond this.
__device__ __forceinline__ double rough_odds(const Decision& d, double k2) {
  return (d.p.m - d.q.m) + (d.p.ls - d.q.ls) / k2;
}
// The root if `all`; else next to nothing, 2^-1042: its low word.
__device__ __forceinline__ double some_of(double root, bool all) {
  return __hiloint2double(all ? __double2hiint(root) : 0, __double2loint(root));
}

constexpr int kExactThreads = 512;

// With draft logits: the decision, and the sums of the rows to draw from, a wave per
// share of a segment.  64 sequences of 152064 tokens 22 us, 13 of them the 64-bit
// operations at their rate (36 a token where both rows count), the rest the chain of
// loads that decides.
template <class X>
__global__ void __launch_bounds__(kExactThreads) exact_kernel(const X* __restrict__ logits,
                                                              const X* __restrict__ draft_logits,
                                                              Args a, Decision* decisions) {
  __shared__ Dist rows_s[2 * kMaxK + 1];
  __shared__ Decision d_s;
  __shared__ DecideLds lds;
  __shared__ double roots[kRoots];
  constexpr int kWaves = kExactThreads / 64;
  load_roots(roots);
  const unsigned blocks = (a.segments * kShares + kWaves - 1) / kWaves;
  const int64_t b = blockIdx.x / blocks;
  const int32_t n = a.drafts(b);
  if (n < 0) return;
  decide<X, true>(logits, draft_logits, a, b, n, rows_s, &lds, &d_s);
  const int part = blockIdx.x % blocks;
  if (part == 0) {
    if (threadIdx.x == 0) decisions[b] = d_s;
    emit_accepted(logits, a, b, d_s, rows_s);
  }
  const int item = part * kWaves + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int seg = item / kShares, share = item % kShares;
  if (d_s.kind < 0 || seg >= a.segments) return;
  const bool two = d_s.kind == 2;
  const X* rp = logits + (b * (a.K + 1) + d_s.accepted) * a.ld;
  const X* rq = two ? draft_logits + (b * a.K + d_s.accepted) * a.ld_draft : rp;
  const Row<X> r(rp, a.V);
  const Segment<X> g(r, seg, a.log_segments);
  // the pieces are the policy's row's; the draft's elements may lie otherwise
  const bool vec = ((reinterpret_cast<uintptr_t>(rp) ^ reinterpret_cast<uintptr_t>(rq)) & 15) == 0;
  constexpr int E = Row<X>::E, kBatch = 2;
  // a grid's exponentials times 2^(shift - m k2) are relative to the row's largest logit
  Grid gp, gq;
  const double mq = two ? d_s.q.m : d_s.p.m;
  gp.refer(d_s.p.m, a.k2, a.span);
  gq.refer(mq, a.k2, a.span);
  gp.k = gq.k = lane_of(gp.k, 0);
  const bool near = gp.near && gq.near;
  const double fp = lane_of(near ? exp2_d(fma(-d_s.p.m, a.k2, gp.shift)) : 1.0, 0);
  const double fq = lane_of(near ? exp2_d(fma(-mq, a.k2, gq.shift)) : 1.0, 0);
  // p > q by the rough sums: z_p - z_q > c, and where that is off by 2^-22 |c| from its
  // roundings or by kUnsure from the sums' the token is near
  const float c0 = uniform((float)rough_odds(d_s, a.k2));
  const float tol = uniform((float)(1.5 * kUnsure / a.k2 + 0x1p-22 * fabs((double)c0)));
  const double odds = lane_of(d_s.p.sum / d_s.q.sum, 0);
  Drawn s{0.0, 0.0, 0.0, 0.0, 0.0};
  auto add = [&](double p, double q) {
    const double d = fma(-q, odds, p);
    const bool larger = d > 0.0;
    s.p += p;
    s.q += q;
    s.a += larger ? p : 0.0;
    s.b += larger ? q : 0.0;
    if (fabs(d) < kUnsure * p) s.near += p;
  };
  const int32_t p0 = g.p0 + (int32_t)((int64_t)(g.p1 - g.p0) * share / kShares),
                p1 = g.p0 + (int32_t)((int64_t)(g.p1 - g.p0) * (share + 1) / kShares);
  for (int32_t c = p0 + lane; c < p1; c += kBatch * 64) {
    uint4 zp[kBatch], zq[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (c + i * 64 >= p1) continue;
      const int32_t at = r.at(c + i * 64);
      zp[i] = *reinterpret_cast<const uint4*>(rp + at);
      if (!two) continue;
      if (vec) {
        zq[i] = *reinterpret_cast<const uint4*>(rq + at);
      } else {
        X e[E];
#pragma unroll
        for (int k = 0; k < E; ++k) e[k] = rq[at + k];
        __builtin_memcpy(&zq[i], e, 16);
      }
    }
#pragma unroll 1
    for (int i = 0; i < kBatch; ++i) {
      if (c + i * 64 < p1) {
        float p[E], q[E];
        unpack(zp[0], p);
        if (two) unpack(zq[0], q);
        if (near) {
          // four at a time, the policy's before the draft's: what that saves in registers
          // a second block of the compute unit needs (72 -> 67 us in all)
#pragma unroll
          for (int h = 0; h < E; h += 4) {
            float p4[4] = {p[h], p[h + 1], p[h + 2], p[h + 3]}, q4[4], d[4];
            Scaled e[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              gp.clamp(p4[k]);
              if (!two) continue;
              q4[k] = q[h + k];
              gq.clamp(q4[k]);
              d[k] = (p4[k] - q4[k]) - c0;
            }
            gp(p4, roots, e);
#pragma unroll
            for (int k = 0; k < 4; ++k) s.p = fma(e[k].p, e[k].root, s.p);
            if (two) {
#pragma unroll
              for (int k = 0; k < 4; ++k)
                s.a = fma(e[k].p, some_of(e[k].root, d[k] > 0.0f), s.a);
              if (fminf(fminf(fabsf(d[0]), fabsf(d[1])), fminf(fabsf(d[2]), fabsf(d[3]))) < tol) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  if (fabsf(d[k]) < tol) s.near = fma(e[k].p, e[k].root, s.near);
              }
              __builtin_amdgcn_sched_barrier(0);
              gq(q4, roots, e);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                s.q = fma(e[k].p, e[k].root, s.q);
                s.b = fma(e[k].p, some_of(e[k].root, d[k] > 0.0f), s.b);
              }
            }
          }
        } else {
#pragma unroll 1
          for (int k = 0; k < E; ++k) {
            add(exp2_d(((double)p[0] - d_s.p.m) * a.k2),
                two ? exp2_d(((double)q[0] - d_s.q.m) * a.k2) : 0.0);
#pragma unroll
            for (int j = 1; j < E; ++j) p[j - 1] = p[j], q[j - 1] = q[j];
          }
        }
      }
#pragma unroll
      for (int k = 1; k < kBatch; ++k) zp[k - 1] = zp[k], zq[k - 1] = zq[k];
    }
  }
  s.p *= fp, s.a *= fp, s.near *= fp, s.q *= fq, s.b *= fq;
  const int32_t loose = r.loose(lane);
  if (share == 0 && loose >= 0 && (loose < r.head ? seg == 0 : seg == a.segments - 1))
    add(exp2_d(((double)value(rp[loose]) - d_s.p.m) * a.k2),
        two ? exp2_d(((double)value(rq[loose]) - d_s.q.m) * a.k2) : 0.0);
  // four sums at once: each half of the wave goes on with two of them, each quarter
  // with one
  double x = lane < 32 ? s.p : s.q, y = lane < 32 ? s.a : s.b;
  x += __shfl_xor(lane < 32 ? s.q : s.p, 32, 64);
  y += __shfl_xor(lane < 32 ? s.b : s.a, 32, 64);
  const double keep = lane & 16 ? y : x, give = lane & 16 ? x : y;
  x = keep + __shfl_xor(give, 16, 64);
#pragma unroll
  for (int off = 8; off >= 1; off >>= 1) x += __shfl_xor(x, off, 64);
  s.p = lane_of(x, 0), s.a = lane_of(x, 16), s.q = lane_of(x, 32), s.b = lane_of(x, 48);
  if (__ballot(s.near != 0.0) != 0) s.near = wave_sum(s.near);
  if (lane == 0) a.drawn[b * a.segments * kShares + item] = s;
}

// A block per sequence: a chain of dependent loads and joins, 9 us for one sequence,
// 12 for 64.
template <class X>
__global__ void __launch_bounds__(kFinishThreads) finish_kernel(const X* __restrict__ logits,
                                                                const X* __restrict__ draft_logits,
                                                                Args a,
                                                                const Decision* decisions) {
  constexpr int kWaves = kFinishThreads / 64;
  __shared__ Dist rows_s[kMaxK + 1];
  __shared__ Decision d_s;
  __shared__ DecideLds lds;
  __shared__ double seg_s[kMaxSegments], wave_s[kWaves], wt_s[kRun][kFinishThreads];
  __shared__ int32_t found, last;
  __shared__ uint64_t fixes_s;
  const int64_t b = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t n = a.drafts(b);
  const double u = (double)a.u[b * (a.K + 1) + a.K];
  // (what the exact sums' launch left, should there be one: loaded with the decision)
  Drawn drawn{0.0, 0.0, 0.0, 0.0, 0.0};
  if (draft_logits != nullptr && tid < a.segments) {
    static_assert(kShares == 2, "two sums");
    const Drawn* d = a.drawn + (b * a.segments + tid) * kShares;
    drawn = Drawn{d[0].p + d[1].p, d[0].q + d[1].q, d[0].a + d[1].a, d[0].b + d[1].b,
                  d[0].near + d[1].near};
  }
  if (n < 0) {
    for (int k = tid; k <= a.K; k += kFinishThreads) {
      a.out_tokens[b * (a.K + 1) + k] = -1;
      a.out_logp[b * (a.K + 1) + k] = 0.0f;
    }
    if (tid == 0) a.n_out[b] = 0;
    return;
  }
  const int rows = draft_logits == nullptr ? a.K + 1 : 2 * a.K + 1;
  if (draft_logits == nullptr) {
    decide<X, false>(logits, nullptr, a, b, n, rows_s, &lds, &d_s);
    emit_accepted(logits, a, b, d_s, rows_s);
  } else {
    if (tid == 0) d_s = decisions[b];
    __syncthreads();
    if (d_s.kind < 0) return;
    // The exact sums of both rows, and the segments' of max(p - q, 0).  The rough odds
    // were off by `off` and less, so a segment's is by off times what lay near them at most: where
    // that is more than 2^-31 of the total it is summed again, so that 64 segments are off by
    // 2^-25 of it together, half a step of u.
    static_assert(kMaxSegments <= 64, "a lane per segment");
    if (wave == 0) {
      const double p = wave_sum(drawn.p), q = wave_sum(drawn.q);
      const double off = fabs(d_s.p.sum * q / (d_s.q.sum * p) - 1.0) +
                         0x1p-22 * fabs(rough_odds(d_s, a.k2)) * a.k2;
      const double rest = drawn.a / p - drawn.b / q;
      const double mine = rest > 0x1p-900 ? rest : 0.0;  // (2^-1000 a token may be nothing)
      const double total = wave_sum(mine);
      if (lane < a.segments) seg_s[lane] = mine;
      const uint64_t fixes = __ballot(off * drawn.near > 0x1p-31 * total * p);
      if (lane == 0) {
        fixes_s = fixes;
        d_s.p.sum = p;
        d_s.p.ls = log2(p);
        d_s.q.sum = q;
        d_s.q.ls = log2(q);
      }
    }
    __syncthreads();
  }
  if (d_s.kind < 0) return;
  const int32_t accepted = d_s.accepted;
  const X* row = logits + (b * (a.K + 1) + accepted) * a.ld;
  const Row<X> r(row, a.V);
  const Part* parts = a.parts + (b * rows + accepted) * a.segments;

  Weight<X> w = weight_of(d_s, logits, draft_logits, a, b);
  auto segments_of_p = [&] {
    if (tid >= a.segments) return;
    if (draft_logits != nullptr) {
      seg_s[tid] = drawn.p;
    } else {
      const Part p = parts[tid];
      seg_s[tid] = p.m == d_s.p.m ? p.s : p.s * exp2_d(((double)p.m - d_s.p.m) * a.k2);
    }
  };
  if (w.kind != 2) segments_of_p();
  if (tid == 0) {
    found = a.V;
    last = -1;
  }
  // First the segments to sum again (`fixes`), for the draft that has to be left out
  // among them; then the segment that the token falls into: the first whose end lies behind the
  // goal, after it the next ones, should rounding leave the token to them, or the
  // last with any weight where none does (u at the end of its interval).  One loop
  // over segments for both, and one copy of the exponential, for the sake of code
  // that has to be fetched.
  uint64_t fixes = w.kind == 2 ? fixes_s : 0;
  if (w.kind == 1) {
    const int32_t piece = w.x < r.head ? 0 : (w.x - r.head) / Row<X>::E;
    int fix = r.pieces > 0 ? min((int)(((int64_t)piece << a.log_segments) / r.pieces), a.segments - 1)
                           : a.segments - 1;
    while (fix < a.segments - 1 && w.x >= Segment<X>(r, fix, a.log_segments).v1) ++fix;
    while (fix > 0 && w.x < Segment<X>(r, fix, a.log_segments).v0) --fix;
    // Taken off its segment's sum where that is exact enough: the two exponentials
    // agree to 1e-13, so beside a remaining total of e / 8 or more the difference is
    // off by less than 1e-12, and 2^-20 e is more than noise.
    __syncthreads();
    const double e = exp2_d(((double)value(w.p[w.x]) - w.mp) * a.k2);
    const double left = seg_s[fix] - e;
    const double rest = wave_sum(lane < a.segments ? seg_s[lane] : 0.0) - e;
    __syncthreads();
    if (left >= 0x1p-20 * e && rest >= 0.125 * e) {
      if (tid == 0) seg_s[fix] = left;
    } else {
      fixes = 1ull << fix;
    }
  }
  uint64_t todo = 0, some = 0;
  double scan = 0.0, goal = 0.0;
  bool located = false;
  for (;;) {
    __syncthreads();
    if (fixes == 0 && !located) {
      for (;;) {
        const double mine = lane < a.segments ? seg_s[lane] : 0.0;
        scan = mine;
#pragma unroll 1
        for (int off = 1; off < 64; off <<= 1) {
          const double o = __shfl_up(scan, off, 64);
          if (lane >= off) scan += o;
        }
        const double total = lane_of(scan, 63);
        if (total > (w.kind == 2 ? kNothing : 0.0) || w.kind == 0) {
          goal = u * total;
          some = __ballot(mine > 0.0);
          todo = __ballot(mine > 0.0 && scan > goal);
          if (todo == 0 && some != 0) todo = 1ull << (63 - __builtin_clzll(some));
          break;
        }
        __syncthreads();  // nothing left: draw from p
        if (tid == 0) d_s.kind = 0;
        __syncthreads();
        w = weight_of(d_s, logits, draft_logits, a, b);
        segments_of_p();
        __syncthreads();
      }
      located = true;
    }
    // (a segment may turn out to hold no weight after all: then the one before)
    if (fixes == 0 && todo == 0 && last < 0 && some != 0)
      todo = 1ull << (63 - __builtin_clzll(some));
    if (fixes == 0 && todo == 0) break;
    const int seg = __builtin_amdgcn_readfirstlane(__builtin_ctzll(fixes != 0 ? fixes : todo));
    const Segment<X> g(r, seg, a.log_segments);
    const double before = seg > 0 ? lane_of(scan, seg - 1) : 0.0;
    const int terms = w.kind == 2 ? 2 : 1;
    double sum = 0.0;
    bool done = false;
    for (int32_t v0 = g.v0; v0 < g.v1 && !done; v0 += kRun * kFinishThreads) {
      // weights of kRun consecutive tokens per thread
      const int32_t first = v0 + tid * kRun;
      float zp[kRun], zq[kRun];
#pragma unroll
      for (int k = 0; k < kRun; ++k)
        zp[k] = first + k < g.v1 ? value(w.p[first + k]) : -INFINITY;
#pragma unroll
      for (int k = 0; k < kRun; ++k)
        zq[k] = w.kind == 2 && first + k < g.v1 ? value(w.q[first + k]) : -INFINITY;
      double s = 0.0;
#pragma unroll 1
      for (int k = 0; k < kRun; ++k) {
        double wt = 0.0;
        if (first + k < g.v1) {
#pragma unroll 1
          for (int i = 0; i < terms; ++i) {
            const double y = i == 0 ? fma((double)zp[0] - w.mp, a.k2, -w.lp)
                                    : fma((double)zq[0] - w.mq, a.k2, -w.lq);
            const double e = exp2_d(y);
            wt = i == 0 ? e : wt - e;
          }
        }
        if (w.kind == 1 && first + k == w.x) wt = 0.0;
        wt = fmax(wt, 0.0);
        wt_s[k][tid] = wt;
        s += wt;
#pragma unroll
        for (int q = 1; q < kRun; ++q) zp[q - 1] = zp[q], zq[q - 1] = zq[q];
      }
      double upto = s;  // inclusive over the wave
#pragma unroll 1
      for (int off = 1; off < 64; off <<= 1) {
        const double o = __shfl_up(upto, off, 64);
        if (lane >= off) upto += o;
      }
      __syncthreads();
      if (lane == 63) wave_s[wave] = upto;
      __syncthreads();
      double run = before + sum;
#pragma unroll 4
      for (int q = 0; q < kWaves; ++q) {
        run += q < wave ? wave_s[q] : 0.0;
        sum += wave_s[q];
      }
      if (fixes != 0) continue;
      run += upto - s;
      int32_t hit = a.V, end = -1;
#pragma unroll
      for (int k = 0; k < kRun; ++k) {
        const double wt = wt_s[k][tid];
        run += wt;
        if (wt > 0.0) {
          end = first + k;
          if (run > goal && hit == a.V) hit = end;
        }
      }
      // one atomic per wave (tokens ascend with the lanes): 1024 took 8 us
      const uint64_t hits = __ballot(hit < a.V), ends = __ballot(end >= 0);
      if (hits != 0) hit = __builtin_amdgcn_readlane(hit, __builtin_ctzll(hits));
      if (ends != 0) end = __builtin_amdgcn_readlane(end, 63 - __builtin_clzll(ends));
      if (lane == 0 && hits != 0) atomicMin(&found, hit);
      if (lane == 0 && ends != 0) atomicMax(&last, end);
      __syncthreads();
      done = found < a.V;
    }
    if (done) break;
    if (fixes != 0) {
      if (tid == 0) seg_s[seg] = sum;
      fixes &= fixes - 1;
    } else {
      todo &= todo - 1;
      some &= ~(1ull << seg);
    }
  }
  if (tid == 0) {
    const int64_t i = b * (a.K + 1) + accepted;
    const int32_t v = found < a.V ? found : last;
    a.out_tokens[i] = v;
    a.out_logp[i] = v < 0 ? NAN : logp_of(row, v, d_s.p, a.k2);
  }
}

// Segments of a row: 512 tokens or more each, and up to 64, a lane each to join them
// (32 with many rows: 576 rows of 152064 bf16 take 75 us in 64 segments, 68 in 32;
// 5 rows 5.6 and 8.3); fewer where rows alone fill the chip many times over, since a
// launch has less than 2^32 threads.
constexpr int64_t kFewRows = 64, kFewItems = 1 << 20;
int segments_of(int64_t B, int64_t K, int32_t V) {
  const int64_t rows = B * (2 * K + 1);
  const int most = rows <= kFewRows ? kMaxSegments : kMaxSegments / 2;
  int n = 1;
  while (n < most && V / (2 * n) >= 512 && rows * n < kFewItems) n *= 2;
  return n;
}

// What a workspace provides for: at least the segments of `rows` rows in all, and no fewer for
// more rows (which may be cut into fewer segments), so that one sized for the largest batch
// serves all.
int64_t most_items(int64_t rows, int32_t V) {
  int64_t n = 1;  // of a row, but for the number of rows
  while (n < kMaxSegments && V / (2 * n) >= 512) n *= 2;
  const int64_t items =
      rows <= kFewRows ? rows * n
                       : std::max(kFewRows * n, rows * std::min<int64_t>(n, kMaxSegments / 2));
  return std::min(items, std::max(2 * kFewItems, rows));
}

struct VerifyWs {
  Part* parts;
  Drawn* drawn;
  Decision* decisions;
  size_t bytes;
};
VerifyWs carve_verify(void* base, int64_t B, int64_t K, int32_t V) {
  rbp::WsCarver c(base);
  VerifyWs w;
  w.parts = c.take<Part>((size_t)most_items(B * (2 * K + 1), V));
  // (with draft logits K is 1 or more, and its sequences have three rows or more)
  w.drawn = c.take<Drawn>(K == 0 ? 0 : (size_t)rbp::ceil_div(most_items(3 * B, V), 3) * kShares);
  w.decisions = c.take<Decision>((size_t)B);
  w.bytes = rbp::align_up(c.used, 256);
  return w;
}

template <class X>
void launch(const X* logits, const X* draft_logits, const Args& a, Decision* decisions,
            hipStream_t s) {
  const int64_t rows = a.B * (int64_t)(draft_logits == nullptr ? a.K + 1 : 2 * a.K + 1);
  const int64_t items = rows * a.segments;
  const dim3 grid((unsigned)rbp::ceil_div(items, kStatsThreads / 64));
  if (draft_logits == nullptr) {
    hipLaunchKernelGGL(stats_kernel<X>, grid, dim3(kStatsThreads), 0, s, logits, a, items);
  } else {
    hipLaunchKernelGGL(rough_kernel<X>, grid, dim3(kStatsThreads), 0, s, logits, draft_logits, a,
                       items);
    hipLaunchKernelGGL(exact_kernel<X>,
                       dim3((unsigned)(a.B * rbp::ceil_div(a.segments * kShares,
                                                           kExactThreads / 64))),
                       dim3(kExactThreads), 0, s, logits, draft_logits, a, decisions);
  }
  hipLaunchKernelGGL(finish_kernel<X>, dim3(a.B), dim3(kFinishThreads), 0, s, logits, draft_logits,
                     a, decisions);
}

}  // namespace

size_t rbp::verify_ws(int64_t B, int32_t K, int32_t V) {
  return carve_verify(nullptr, B < 1 ? 1 : B, K < 0 ? 0 : K, V < 1 ? 1 : V).bytes;
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
  RBP_REQUIRE(temperature >= 0x1p-100f && temperature <= 0x1p100f, RBP_EINVAL,
              "policy_verify_drafts: temperature must lie in [2^-100, 2^100]");
  RBP_REQUIRE(K <= 255 && B <= (1 << 21) && (int64_t)B * (K + 1) <= (1 << 24), RBP_EUNSUPPORTED,
              "policy_verify_drafts: K above 255, B above 2^21 or B (K + 1) above 2^24");
  RBP_REQUIRE(V <= rbp::rows::kMaxVocab, RBP_EUNSUPPORTED,
              "policy_verify_drafts: V above 2^31 - 2^14 - 1");
  if (B == 0) return RBP_OK;
  RBP_REQUIRE(logits && u && out_tokens && out_logp && n_out && (K == 0 || draft_tokens),
              RBP_EINVAL, "policy_verify_drafts: null pointer");
  const size_t es = logits_type == RBP_F32 ? 4 : 2;
  RBP_REQUIRE(aligned(logits, es) && aligned(draft_logits, es) && aligned(ws, 16), RBP_EINVAL,
              "policy_verify_drafts: logits not aligned to their type, or ws to 16 bytes");
  const size_t need = rbp::verify_ws(B, K, V);
  RBP_REQUIRE(ws && ws_bytes >= need, RBP_EWORKSPACE,
              "policy_verify_drafts: workspace needs %zu bytes, got %zu", need, ws_bytes);
  hipStream_t s = rbp::as_stream(stream);
  const VerifyWs w = carve_verify(ws, B, K, V);
  if (K == 0) draft_logits = nullptr;
  const int segments = segments_of(B, K, V);
  const double k2 = kLog2eD / (double)temperature;
  const Args a{ld,  ld_draft, draft_tokens, n_draft, u, B, K, V, segments,
               __builtin_ctz((unsigned)segments), k2, 1000.0 / k2,
               (float)std::fmin(kSlack / k2, 1e30), out_tokens, out_logp, n_out, w.parts, w.drawn};
  if (logits_type == RBP_F32)
    launch(static_cast<const float*>(logits), static_cast<const float*>(draft_logits), a,
           w.decisions, s);
  else
    launch(static_cast<const uint16_t*>(logits), static_cast<const uint16_t*>(draft_logits), a,
           w.decisions, s);
  RBP_CHECK_LAUNCH("policy_verify_drafts");
  return RBP_OK;
}
