// Embedding lookup (policy_embed_fwd) and its table's gradient (policy_embed_bwd).
//
//   out_t = bf16(scale table[y_t]),   dW_v (+)= scale sum_{t: y_t = v} dx_t.
//
// Both are bound by HBM: the lookup reads the rows it needs and writes T d bf16
// values; the gradient reads T d values of dx and writes (or reads and writes)
// the rows of dW that have a token, or all V rows when it overwrites.
//
// The gradient without atomics on floats: the tokens are sorted by id (stable
// least-significant-digit radix sort of (id, position) pairs, up to 9 bits a
// pass), so that a row's gradients are a run of sorted positions in batch order.
// The sorted positions are cut into slices of equal length, whatever the tokens'
// frequencies: a group of lanes walks a slice, sums runs in registers and writes
// the runs that lie inside it; the ends of runs that cross a slice's border go to
// the workspace and are summed there, in order, by the group where the run begins.

#include "logits_epilogue.h"
#include "rbp_internal.h"

namespace {

using rbp::lp::bf16_to_f32;
using rbp::lp::pack_bf16x2;

// ---- forward ------------------------------------------------------------------

// One 16-byte piece of a row per thread.
__global__ void __launch_bounds__(256) embed_kernel(const uint16_t* __restrict__ table,
                                                    const int32_t* __restrict__ tokens,
                                                    const int32_t* __restrict__ seq, int64_t n,
                                                    int32_t d8, int32_t V, float scale,
                                                    uint4* __restrict__ out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const int64_t t = i / d8;
  const int32_t c = (int32_t)(i - t * d8);
  uint4 o = make_uint4(0u, 0u, 0u, 0u);
  if (seq == nullptr || seq[t] >= 0) {
    const int32_t y = tokens[t];
    if (y >= 0 && y < V) {
      const uint4 w = reinterpret_cast<const uint4*>(table)[(int64_t)y * d8 + c];
      const uint32_t a[4] = {w.x, w.y, w.z, w.w};
      uint32_t r[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        r[k] = pack_bf16x2(scale * bf16_to_f32((uint16_t)(a[k] & 0xffff)),
                           scale * bf16_to_f32((uint16_t)(a[k] >> 16)));
      o = make_uint4(r[0], r[1], r[2], r[3]);
    } else {
      o = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
    }
  }
  out[i] = o;
}

// ---- sorting the tokens ---------------------------------------------------------

constexpr int kSortThreads = 512;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kItems = 8;  // keys per thread
constexpr int kTile = kSortThreads * kItems;
constexpr int kMaxDigit = 9;
constexpr int kBins = 1 << kMaxDigit;
static_assert(kBins == kSortThreads, "one bin per thread");

// A token's sort key: its id, or V (behind every id) if it adds nothing.
__device__ __forceinline__ uint32_t key_of(const int32_t* __restrict__ tokens,
                                           const int32_t* __restrict__ seq, int64_t t, int32_t V) {
  const int32_t y = tokens[t];
  return (seq == nullptr || seq[t] >= 0) && y >= 0 && y < V ? (uint32_t)y : (uint32_t)V;
}

// Keys of a pass: the tokens' in the first, the previous pass's output later.
struct Keys {
  const int32_t *tokens, *seq;
  const uint32_t *key, *at;
  int32_t V;
  __device__ __forceinline__ uint32_t load(int64_t i) const {
    return key == nullptr ? key_of(tokens, seq, i, V) : key[i];
  }
  __device__ __forceinline__ uint32_t position(int64_t i) const {
    return key == nullptr ? (uint32_t)i : at[i];
  }
};

// hist[block][digit]: the keys of the block's tile by digit.
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(Keys in, int64_t T, int shift,
                                                                  uint32_t* __restrict__ hist) {
  __shared__ uint32_t bins[kBins];
  bins[threadIdx.x] = 0;
  __syncthreads();
  const int64_t t0 = (int64_t)blockIdx.x * kTile;
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    const int64_t i = t0 + k * kSortThreads + threadIdx.x;
    if (i < T) atomicAdd(&bins[(in.load(i) >> shift) & (kBins - 1)], 1u);
  }
  __syncthreads();
  hist[(int64_t)blockIdx.x * kBins + threadIdx.x] = bins[threadIdx.x];
}

// One pass: every key of the tile to its place, keys of equal digits in order.
// A wave takes 512 consecutive keys, 64 at a time; lanes with the same digit find
// each other by ballots over its bits, and the wave's counts so far give their
// ranks.
__global__ void __launch_bounds__(kSortThreads) sort_scatter_kernel(
    Keys in, int64_t T, int shift, const uint32_t* __restrict__ hist, int n_tiles,
    uint32_t* __restrict__ key_out, uint32_t* __restrict__ at_out) {
  __shared__ uint32_t cnt[kSortWaves][kBins];
  __shared__ uint32_t base[kBins], wave_sum[kSortWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) cnt[w][tid] = 0;
  // this thread's bin: keys of it in all tiles, and in those before this one
  uint32_t total = 0, before = 0;
  for (int b = 0; b < n_tiles; ++b) {
    const uint32_t h = hist[(int64_t)b * kBins + tid];
    total += h;
    if (b < (int)blockIdx.x) before += h;
  }
  uint32_t scan = total;  // inclusive over the bins
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t o = __shfl_up(scan, off, 64);
    if (lane >= off) scan += o;
  }
  if (lane == 63) wave_sum[wave] = scan;
  __syncthreads();
  uint32_t lower = scan - total;
  for (int w = 0; w < wave; ++w) lower += wave_sum[w];
  base[tid] = lower + before;

  const int64_t t0 = (int64_t)blockIdx.x * kTile + wave * (64 * kItems);
  uint32_t key[kItems], place[kItems];
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    const int64_t i = t0 + k * 64 + lane;
    const bool live = i < T;
    key[k] = live ? in.load(i) : 0u;
    const uint32_t digit = (key[k] >> shift) & (kBins - 1);
    uint64_t same = __ballot(live);
#pragma unroll
    for (int bit = 0; bit < kMaxDigit; ++bit) {
      const uint64_t set = __ballot((digit >> bit) & 1);
      same &= (digit >> bit) & 1 ? set : ~set;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    place[k] = cnt[wave][digit] + rank;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (live && rank == 0) cnt[wave][digit] += (uint32_t)__popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  uint32_t run = 0;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    const uint32_t c = cnt[w][tid];
    cnt[w][tid] = run;
    run += c;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    const int64_t i = t0 + k * 64 + lane;
    if (i >= T) continue;
    const uint32_t digit = (key[k] >> shift) & (kBins - 1);
    const uint32_t to = base[digit] + cnt[wave][digit] + place[k];
    key_out[to] = key[k];
    at_out[to] = in.position(i);
  }
}

// ---- sums over runs -------------------------------------------------------------

constexpr uint32_t kNoKey = 0xffffffffu;
constexpr int kSlice = 32;  // sorted positions per slice

struct Sorted {
  const uint32_t *key, *at;
  int64_t T;
  __device__ __forceinline__ uint32_t key_at(int64_t i) const {
    return i >= 0 && i < T ? key[i] : kNoKey;
  }
};

struct Row8 {
  float v[8];
};

__device__ __forceinline__ Row8 load8(const float* __restrict__ p) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
__device__ __forceinline__ Row8 load8(const uint16_t* __restrict__ p) {
  const uint4 a = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
  Row8 r;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    r.v[2 * k] = bf16_to_f32((uint16_t)(w[k] & 0xffff));
    r.v[2 * k + 1] = bf16_to_f32((uint16_t)(w[k] >> 16));
  }
  return r;
}
__device__ __forceinline__ void store8(float* __restrict__ p, const Row8& r) {
  reinterpret_cast<float4*>(p)[0] = make_float4(r.v[0], r.v[1], r.v[2], r.v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(r.v[4], r.v[5], r.v[6], r.v[7]);
}

// dW's 8 columns at p: scale sum, added to what is there or in its place.
__device__ __forceinline__ void put8(float* __restrict__ p, const Row8& sum, float scale,
                                     bool accumulate) {
  Row8 o{};
  if (accumulate) o = load8(static_cast<const float*>(p));
#pragma unroll
  for (int k = 0; k < 8; ++k) o.v[k] = fmaf(scale, sum.v[k], o.v[k]);
  store8(p, o);
}

// A group of kLanes lanes (8 columns each) per slice and kLanes * 8 columns.
// part[slice][0]: the sum of the run that came in from the slice before,
// part[slice][1]: of the run that begins here and goes on behind it.
template <class X, int kLanes>
__global__ void __launch_bounds__(256) run_sum_kernel(const X* __restrict__ dx, Sorted in,
                                                      int64_t n_slices, int n_chunks, int32_t d,
                                                      int32_t V, float scale, int accumulate,
                                                      float* __restrict__ dW,
                                                      float* __restrict__ part) {
  const int64_t g = ((int64_t)blockIdx.x * 256 + threadIdx.x) / kLanes;
  const int64_t slice = g / n_chunks;
  const int32_t col = ((int32_t)(g % n_chunks) * kLanes + (int)(threadIdx.x % kLanes)) * 8;
  if (slice >= n_slices || col >= d) return;
  const int64_t i0 = slice * kSlice, i1 = i0 + kSlice < in.T ? i0 + kSlice : in.T;
  uint32_t cur = in.key_at(i0);
  bool begins = cur != in.key_at(i0 - 1);
  Row8 acc{};
  auto flush = [&](bool ends) {
    if (cur >= (uint32_t)V) return;
    if (begins && ends)
      put8(dW + (int64_t)cur * d + col, acc, scale, accumulate != 0);
    else
      store8(part + (slice * 2 + (begins ? 1 : 0)) * d + col, acc);
  };
  for (int64_t i = i0; i < i1; ++i) {
    const uint32_t k = in.key[i];
    if (k != cur) {
      flush(true);
      cur = k;
      begins = true;
      acc = Row8{};
    }
    if (k >= (uint32_t)V) break;
    const Row8 r = load8(dx + (int64_t)in.at[i] * d + col);
#pragma unroll
    for (int q = 0; q < 8; ++q) acc.v[q] += r.v[q];
  }
  flush(cur != in.key_at(i1));
}

// The runs that cross slices, by the slice they begin in.
template <int kLanes>
__global__ void __launch_bounds__(256) run_join_kernel(Sorted in, int64_t n_slices, int n_chunks,
                                                       int32_t d, int32_t V, float scale,
                                                       int accumulate, float* __restrict__ dW,
                                                       const float* __restrict__ part) {
  const int64_t g = ((int64_t)blockIdx.x * 256 + threadIdx.x) / kLanes;
  const int64_t slice = g / n_chunks;
  const int32_t col = ((int32_t)(g % n_chunks) * kLanes + (int)(threadIdx.x % kLanes)) * 8;
  if (slice >= n_slices || col >= d) return;
  const int64_t i0 = slice * kSlice, i1 = i0 + kSlice;
  if (i1 >= in.T) return;
  const uint32_t cur = in.key[i1 - 1];
  if (cur >= (uint32_t)V || in.key[i1] != cur) return;
  if (in.key[i0] == cur && in.key_at(i0 - 1) == cur) return;  // began before
  Row8 acc = load8(part + (slice * 2 + 1) * d + col);
  for (int64_t j = slice + 1;; ++j) {
    const Row8 r = load8(part + j * 2 * d + col);
#pragma unroll
    for (int q = 0; q < 8; ++q) acc.v[q] += r.v[q];
    const int64_t end = (j + 1) * kSlice;  // behind slice j
    if (end >= in.T || in.key[end] != cur) break;
  }
  put8(dW + (int64_t)cur * d + col, acc, scale, accumulate != 0);
}

__global__ void __launch_bounds__(256) zero_kernel(float4* __restrict__ p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256)
    p[i] = make_float4(0.f, 0.f, 0.f, 0.f);
}

struct EmbedWs {
  uint32_t *key[2], *at[2], *hist;
  float* part;
  size_t bytes;
};

EmbedWs carve_embed(void* base, int64_t T, int32_t d) {
  rbp::WsCarver c(base);
  const size_t n = (size_t)T;
  EmbedWs w;
  for (int k = 0; k < 2; ++k) {
    w.key[k] = c.take<uint32_t>(n);
    w.at[k] = c.take<uint32_t>(n);
  }
  w.hist = c.take<uint32_t>((size_t)rbp::ceil_div(T, kTile) * kBins);
  w.part = c.take<float>((size_t)rbp::ceil_div(T, kSlice) * 2 * (size_t)d);
  w.bytes = rbp::align_up(c.used, 256);
  return w;
}

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

template <class Launch>
void with_lanes(int32_t d8, Launch&& launch) {
  if (d8 <= 8)
    launch(std::integral_constant<int, 8>{});
  else if (d8 <= 16)
    launch(std::integral_constant<int, 16>{});
  else if (d8 <= 32)
    launch(std::integral_constant<int, 32>{});
  else
    launch(std::integral_constant<int, 64>{});
}

}  // namespace

size_t rbp::embed_bwd_ws(int64_t T, int32_t d, int32_t V) {
  (void)V;
  return carve_embed(nullptr, T < 1 ? 1 : T, d < 1 ? 1 : d).bytes;
}

extern "C" int policy_embed_fwd(const uint16_t* table, const int32_t* tokens,
                                const int32_t* seq_of_token, int64_t T, int32_t d, int32_t V,
                                float scale, uint16_t* out, void* stream) {
  rbp::clear_error();
  RBP_REQUIRE(T >= 0 && d >= 1 && V >= 1, RBP_EINVAL,
              "policy_embed_fwd: need T >= 0, d >= 1, V >= 1");
  RBP_REQUIRE(std::isfinite(scale), RBP_EINVAL, "policy_embed_fwd: scale is not finite");
  RBP_REQUIRE(d % 8 == 0, RBP_EUNSUPPORTED, "policy_embed_fwd: d %% 8 != 0 (d = %d)", d);
  RBP_REQUIRE(T <= INT32_MAX, RBP_EUNSUPPORTED, "policy_embed_fwd: T above 2^31 - 1");
  if (T == 0) return RBP_OK;
  RBP_REQUIRE(table && tokens && out, RBP_EINVAL, "policy_embed_fwd: null pointer");
  RBP_REQUIRE(aligned(table, 16) && aligned(out, 16), RBP_EUNSUPPORTED,
              "policy_embed_fwd: table and out must be aligned to 16 bytes");
  const int64_t n = T * (d / 8);
  RBP_REQUIRE(rbp::ceil_div(n, 256) <= INT32_MAX, RBP_EUNSUPPORTED,
              "policy_embed_fwd: T * d too large");
  hipLaunchKernelGGL(embed_kernel, dim3((unsigned)rbp::ceil_div(n, 256)), dim3(256), 0,
                     rbp::as_stream(stream), table, tokens, seq_of_token, n, d / 8, V, scale,
                     reinterpret_cast<uint4*>(out));
  RBP_CHECK_LAUNCH("policy_embed_fwd");
  return RBP_OK;
}

extern "C" int policy_embed_bwd(const void* dx, int dx_type, const int32_t* tokens,
                                const int32_t* seq_of_token, int64_t T, int32_t d, int32_t V,
                                float scale, float* dW, int accumulate_dW, void* ws,
                                size_t ws_bytes, void* stream) {
  rbp::clear_error();
  RBP_REQUIRE(T >= 0 && d >= 1 && V >= 1, RBP_EINVAL,
              "policy_embed_bwd: need T >= 0, d >= 1, V >= 1");
  RBP_REQUIRE(dx_type == RBP_BF16 || dx_type == RBP_F32, RBP_EINVAL,
              "policy_embed_bwd: unknown dx_type %d", dx_type);
  RBP_REQUIRE(std::isfinite(scale), RBP_EINVAL, "policy_embed_bwd: scale is not finite");
  RBP_REQUIRE(d % 8 == 0, RBP_EUNSUPPORTED, "policy_embed_bwd: d %% 8 != 0 (d = %d)", d);
  RBP_REQUIRE(T <= (int64_t(1) << 30), RBP_EUNSUPPORTED, "policy_embed_bwd: T above 2^30");
  RBP_REQUIRE(dW && (T == 0 || (dx && tokens)), RBP_EINVAL, "policy_embed_bwd: null pointer");
  RBP_REQUIRE(aligned(dW, 16) && aligned(dx, 16), RBP_EUNSUPPORTED,
              "policy_embed_bwd: dx and dW must be aligned to 16 bytes");
  const size_t need = T == 0 ? 0 : rbp::embed_bwd_ws(T, d, V);
  RBP_REQUIRE(T == 0 || (ws && ws_bytes >= need), RBP_EWORKSPACE,
              "policy_embed_bwd: workspace needs %zu bytes, got %zu", need, ws_bytes);
  hipStream_t s = rbp::as_stream(stream);
  if (!accumulate_dW) {
    const int64_t n = (int64_t)V * (d / 4), blocks = rbp::ceil_div(n, 256 * 4);
    hipLaunchKernelGGL(zero_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0,
                       s, reinterpret_cast<float4*>(dW), n);
    RBP_CHECK_LAUNCH("policy_embed_bwd");
  }
  if (T == 0) return RBP_OK;
  const EmbedWs w = carve_embed(ws, T, d);
  const int n_tiles = (int)rbp::ceil_div(T, kTile);
  int bits = 1;
  while (bits < 31 && (V >> bits) != 0) ++bits;  // keys go up to V
  const int passes = (bits + kMaxDigit - 1) / kMaxDigit;
  Keys in{tokens, seq_of_token, nullptr, nullptr, V};
  for (int p = 0; p < passes; ++p) {
    const int shift = p * kMaxDigit;
    hipLaunchKernelGGL(sort_count_kernel, dim3(n_tiles), dim3(kSortThreads), 0, s, in, T, shift,
                       w.hist);
    hipLaunchKernelGGL(sort_scatter_kernel, dim3(n_tiles), dim3(kSortThreads), 0, s, in, T, shift,
                       w.hist, n_tiles, w.key[p & 1], w.at[p & 1]);
    in.key = w.key[p & 1];
    in.at = w.at[p & 1];
  }
  RBP_CHECK_LAUNCH("policy_embed_bwd");
  const Sorted sorted{in.key, in.at, T};
  const int64_t n_slices = rbp::ceil_div(T, kSlice);
  with_lanes(d / 8, [&](auto lanes) {
    constexpr int kLanes = decltype(lanes)::value;
    const int n_chunks = (int)rbp::ceil_div(d / 8, kLanes);
    const dim3 grid((unsigned)rbp::ceil_div(n_slices * n_chunks * kLanes, 256));
    if (dx_type == RBP_F32)
      hipLaunchKernelGGL((run_sum_kernel<float, kLanes>), grid, dim3(256), 0, s,
                         static_cast<const float*>(dx), sorted, n_slices, n_chunks, d, V, scale,
                         accumulate_dW, dW, w.part);
    else
      hipLaunchKernelGGL((run_sum_kernel<uint16_t, kLanes>), grid, dim3(256), 0, s,
                         static_cast<const uint16_t*>(dx), sorted, n_slices, n_chunks, d, V, scale,
                         accumulate_dW, dW, w.part);
    hipLaunchKernelGGL(run_join_kernel<kLanes>, grid, dim3(256), 0, s, sorted, n_slices, n_chunks,
                       d, V, scale, accumulate_dW, dW, w.part);
  });
  RBP_CHECK_LAUNCH("policy_embed_bwd");
  return RBP_OK;
}
