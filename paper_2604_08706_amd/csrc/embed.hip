// Embedding lookup (policy_embed_fwd) and its table's gradient (policy_embed_bwd).
//
//   out_t = bf16(scale table[y_t]),   dW_v (+)= scale sum_{t: y_t = v} dx_t.
//
// Both are bound by HBM: the lookup reads the rows it needs and writes T d bf16
// values; the gradient reads T d values of dx and writes (or reads and writes)
// the rows of dW that have a token, or all V rows when it overwrites.
//
// The gradient without atomics on floats: a few tokens' blocks look for tokens of
// their id themselves (few_kernel); more tokens are sorted by id, stably (thousands by
// counting, beyond that by a least-significant-digit radix sort of (id, position)
// pairs, up to 9 bits a pass), so that a row's gradients are a run of sorted positions
// in batch order.
// The sorted positions are cut into slices of equal length, whatever the tokens'
// frequencies: a group of lanes walks a slice, sums runs in registers and writes
// the runs that lie inside it; the ends of runs that cross a slice's border go to
// the workspace and are summed there, in order, by the group where the run begins.

#include <algorithm>

#include "logits_epilogue.h"
#include "rbp_internal.h"

namespace {

using rbp::lp::bf16_to_f32;
using rbp::lp::pack_bf16x2;

// ---- forward ------------------------------------------------------------------

constexpr int kRowPieces = 4;  // 16-byte pieces of a thread, their loads in flight together

// Pieces of rows by a block: kRowPieces times 256 consecutive ones.  Large outputs
// are stored past the caches (kBypass), which then keep the rows that tokens share:
// 16384 x 3584 43.7 -> 35.5 us (4.7 TB/s), 16384 x 896 11.5 -> 9.0.
template <bool kBypass>
__global__ void __launch_bounds__(256) embed_kernel(const uint16_t* __restrict__ table,
                                                    const int32_t* __restrict__ tokens,
                                                    const int32_t* __restrict__ seq, int64_t n,
                                                    uint32_t d8, int32_t V, float scale,
                                                    uint4* __restrict__ out) {
  const int64_t first = (int64_t)blockIdx.x * (256 * kRowPieces);
  // row and piece of the block's first piece; the others are less than 2^31 behind it
  const int64_t t0 = first / d8;
  const uint32_t c0 = (uint32_t)(first - t0 * d8);
  uint4 w[kRowPieces];
  bool zero[kRowPieces], bad[kRowPieces];
#pragma unroll
  for (int k = 0; k < kRowPieces; ++k) {
    const uint32_t i = k * 256 + threadIdx.x, at = c0 + i;
    zero[k] = bad[k] = false;
    w[k] = make_uint4(0u, 0u, 0u, 0u);
    if (first + i >= n) continue;
    const int64_t t = t0 + at / d8;
    const int32_t y = tokens[t];
    zero[k] = seq != nullptr && seq[t] < 0;
    bad[k] = !(y >= 0 && y < V);
    if (!zero[k] && !bad[k])
      w[k] = reinterpret_cast<const uint4*>(table)[(int64_t)y * d8 + at % d8];
  }
#pragma unroll
  for (int k = 0; k < kRowPieces; ++k) {
    const int64_t i = first + k * 256 + threadIdx.x;
    if (i >= n) continue;
    const uint32_t a[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
    uint32_t r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      r[j] = pack_bf16x2(scale * bf16_to_f32((uint16_t)(a[j] & 0xffff)),
                         scale * bf16_to_f32((uint16_t)(a[j] >> 16)));
    const bool nan = bad[k] && !zero[k];
    const uint4 o = nan       ? make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u)
                    : zero[k] ? make_uint4(0u, 0u, 0u, 0u)
                              : make_uint4(r[0], r[1], r[2], r[3]);
    if constexpr (kBypass) {
      typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4, o), reinterpret_cast<u32x4*>(out + i));
    } else {
      out[i] = o;
    }
  }
}

// ---- sorting the tokens ---------------------------------------------------------

constexpr int kSortThreads = 512;
constexpr int kMaxDigit = 9;
constexpr int kBins = 1 << kMaxDigit;
static_assert(kBins == kSortThreads, "one bin per thread");

// A token's sort key: its id, or V (behind every id) if it adds nothing.
__device__ __forceinline__ uint32_t key_of(const int32_t* __restrict__ tokens,
                                           const int32_t* __restrict__ seq, int64_t t, int32_t V) {
  const int32_t y = tokens[t];
  return (seq == nullptr || seq[t] >= 0) && y >= 0 && y < V ? (uint32_t)y : (uint32_t)V;
}
constexpr uint32_t kNoKey = 0xffffffffu;  // behind all of them
__device__ __forceinline__ uint32_t digit_of(uint32_t key, int shift) {
  return (key >> shift) & (kBins - 1);
}

// dW's rows are cleared by blocks behind those of the sort's launches, so that the
// sort, which keeps few units busy, costs next to nothing beside it.
struct Fill {
  float4* p;
  int64_t n;
  int blocks;  // of this launch, behind the sort's
};
template <int kThreads>
__device__ __forceinline__ void fill(const Fill& f, int block) {
  const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int64_t i = (int64_t)block * kThreads + threadIdx.x; i < f.n;
       i += (int64_t)f.blocks * kThreads)
    f.p[i] = zero;
}

// Ranks of a tile's keys by digit, in order: a wave takes kItems * 64 consecutive
// keys, 64 at a time; lanes with the same digit find each other by ballots over its
// bits, and the wave's counts so far give their ranks.  place[k] is the key's rank
// among the wave's keys of its digit; cnt[wave][digit] ends up as the number of them
// in the waves before, cnt[kWaves][digit] as that of the tile.
template <int kItems, int kWaves>
__device__ __forceinline__ void rank_tile(const uint32_t (&key)[kItems], int live_items,
                                          int shift, uint32_t (*cnt)[kBins],
                                          uint32_t (&place)[kItems]) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < kWaves * kBins; i += kWaves * 64) cnt[0][i] = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    const bool live = k * 64 + lane < live_items;
    const uint32_t digit = digit_of(key[k], shift);
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
  if (tid < kBins) {
    uint32_t run = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const uint32_t c = cnt[w][tid];
      cnt[w][tid] = run;
      run += c;
    }
    cnt[kWaves][tid] = run;
  }
  __syncthreads();
}

// Exclusive sum over the bins, one per thread (threads behind them bring 0).
__device__ __forceinline__ uint32_t scan_bins(uint32_t total, uint32_t* wave_sum) {
  constexpr int kBinWaves = kBins / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t scan = total;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t o = __shfl_up(scan, off, 64);
    if (lane >= off) scan += o;
  }
  if (lane == 63 && wave < kBinWaves) wave_sum[wave] = scan;
  __syncthreads();
  uint32_t lower = scan - total;
#pragma unroll
  for (int w = 0; w < kBinWaves - 1; ++w)
    if (w < wave) lower += wave_sum[w];
  return lower;
}

// The sort of some thousand tokens, in one launch: a block finds the places of kOwn of
// them among all, by counting the keys that belong before each.  A lane has kPer tokens,
// for which it reads every kParts-th four of the keys from LDS (two: 8192 x 896 25.3 us
// in all, 27.4 with one, 25.4 with four, which lose 0.5 us with fewer tokens).
constexpr int kRankThreads = 1024, kRankKeys = 12288;
template <int kOwn>
__global__ void __launch_bounds__(kRankThreads) rank_kernel(
    const int32_t* __restrict__ tokens, const int32_t* __restrict__ seq, int32_t V, int32_t T,
    uint32_t* __restrict__ key_out, uint32_t* __restrict__ at_out, Fill f) {
  constexpr int kPer = 2, kLanes = kOwn / kPer, kParts = kRankThreads / kLanes,
                kWaves = kRankThreads / 64;
  __shared__ uint4 key_s[kRankKeys / 4];
  __shared__ uint32_t cnt_s[kWaves][kOwn];
  const int n_blocks = (T + kOwn - 1) / kOwn;
  if ((int)blockIdx.x >= n_blocks) return fill<kRankThreads>(f, blockIdx.x - n_blocks);
  uint32_t* keys = reinterpret_cast<uint32_t*>(key_s);
  const int tid = threadIdx.x, part = tid / kLanes;
  for (int i = tid; i < n_blocks * kOwn; i += kRankThreads)
    keys[i] = i < T ? key_of(tokens, seq, i, V) : kNoKey;
  __syncthreads();
  const int i0 = blockIdx.x * kOwn, own = tid % kLanes * kPer;
  uint32_t mine[kPer], cnt[kPer] = {};
#pragma unroll
  for (int p = 0; p < kPer; ++p) mine[p] = keys[i0 + own + p];
  // up to the block's own tokens equal keys come before, from there on smaller ones, and
  // of its own the equal ones at lower positions
  const int n4 = n_blocks * (kOwn / 4);
  int j = part;
#pragma unroll 2
  for (; j < i0 / 4; j += kParts) {
    const uint4 k = key_s[j];
#pragma unroll
    for (int p = 0; p < kPer; ++p)
      cnt[p] += (k.x <= mine[p]) + (k.y <= mine[p]) + (k.z <= mine[p]) + (k.w <= mine[p]);
  }
#pragma unroll 2
  for (; j < n4; j += kParts) {
    const uint4 k = key_s[j];
#pragma unroll
    for (int p = 0; p < kPer; ++p)
      cnt[p] += (k.x < mine[p]) + (k.y < mine[p]) + (k.z < mine[p]) + (k.w < mine[p]);
  }
#pragma unroll
  for (int p = 0; p < kPer; ++p) {
    for (int t = part; t < own + p; t += kParts) cnt[p] += keys[i0 + t] == mine[p];
#pragma unroll
    for (int off = kLanes; off < 64; off <<= 1) cnt[p] += __shfl_xor(cnt[p], off, 64);
    if ((tid & 63) < kLanes) cnt_s[tid >> 6][own + p] = cnt[p];
  }
  __syncthreads();
  if (tid >= kOwn || i0 + tid >= T) return;
  uint32_t to = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) to += cnt_s[w][tid];
  key_out[to] = keys[i0 + tid];
  at_out[to] = i0 + tid;
}

// Keys of a pass: the tokens' in the first, the previous pass's output later.
struct Keys {
  const int32_t *tokens, *seq;
  const uint32_t *key, *at;
  int32_t V;
  __device__ __forceinline__ uint32_t load(int64_t i) const {
    return key == nullptr ? key_of(tokens, seq, i, V) : key[i];
  }
};

// hist[block][digit] of a pass: a block takes a tile, or `steps` consecutive ones (kMany; known
// to be one, 0.2 us less a launch).  (Counted by
// atomics where the pass before puts its keys instead, a frequent token's take turns: 8 us
// more there, 4.6 for this launch.)
template <int kItems, bool kMany>
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(Keys in, int64_t T, int shift,
                                                                  int n_blocks, int steps,
                                                                  uint32_t* __restrict__ hist,
                                                                  Fill f) {
  __shared__ uint32_t bins[kBins];
  if ((int)blockIdx.x >= n_blocks) return fill<kSortThreads>(f, blockIdx.x - n_blocks);
  bins[threadIdx.x] = 0;
  __syncthreads();
  if constexpr (!kMany) steps = 1;
  int64_t t0 = (int64_t)blockIdx.x * steps * (kSortThreads * kItems);
  for (int step = 0; step < steps; ++step, t0 += kSortThreads * kItems) {
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int64_t i = t0 + k * kSortThreads + threadIdx.x;
      if (i < T) atomicAdd(&bins[digit_of(in.load(i), shift)], 1u);
    }
  }
  __syncthreads();
  hist[(int64_t)blockIdx.x * kBins + threadIdx.x] = bins[threadIdx.x];
}

// One pass: every key of the block's tiles to its place, tile after tile.  16384 tokens: 5 us,
// as the count before it takes.
template <int kItems, bool kMany>
__global__ void __launch_bounds__(kSortThreads) sort_scatter_kernel(
    Keys in, int64_t T, int shift, const uint32_t* __restrict__ hist, int n_blocks, int steps,
    uint32_t* __restrict__ key_out, uint32_t* __restrict__ at_out, Fill f) {
  constexpr int kTile = kSortThreads * kItems, kWaves = kSortThreads / 64;
  __shared__ uint32_t cnt[kWaves + 1][kBins];
  __shared__ uint32_t base[kBins], wave_sum[kBins / 64];
  if ((int)blockIdx.x >= n_blocks) return fill<kSortThreads>(f, blockIdx.x - n_blocks);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if constexpr (!kMany) steps = 1;
  int64_t t0 = (int64_t)blockIdx.x * steps * kTile + wave * (64 * kItems);
  uint32_t key[kItems], at[kItems], place[kItems];
  auto load = [&] {
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int64_t i = t0 + k * 64 + lane;
      key[k] = i >= T ? 0u : in.load(i);
      at[k] = i >= T || in.key == nullptr ? (uint32_t)i : in.at[i];
    }
  };
  load();
  // this thread's bin: keys of it in all blocks, and in those before this one
  uint32_t total = 0, before = 0;
#pragma unroll 8
  for (int b = 0; b < n_blocks; ++b) {
    const uint32_t h = hist[(int64_t)b * kBins + tid];
    total += h;
    before += b < (int)blockIdx.x ? h : 0u;
  }
  base[tid] = scan_bins(total, wave_sum) + before;
  for (int step = 0;;) {
    const int live = T - t0 < kTile ? (int)(T - t0) : kTile;
    rank_tile<kItems, kWaves>(key, live, shift, cnt, place);
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      if (k * 64 + lane >= live) continue;
      const uint32_t digit = digit_of(key[k], shift);
      const uint32_t to = base[digit] + cnt[wave][digit] + place[k];
      key_out[to] = key[k];
      at_out[to] = at[k];
    }
    if (++step == steps) break;
    t0 += kTile;
    load();
    __syncthreads();  // base and cnt have been read
    base[tid] += cnt[kWaves][tid];
  }
}

// ---- sums over runs -------------------------------------------------------------

struct Sorted {
  const uint32_t *key, *at;
  int64_t T;
  int32_t slice;     // positions per slice, a power of two
  int64_t n_slices;
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
__device__ __forceinline__ void add8(Row8& a, const Row8& b) {
#pragma unroll
  for (int k = 0; k < 8; ++k) a.v[k] += b.v[k];
}
// old + scale sum
__device__ __forceinline__ Row8 scaled(const Row8& old, const Row8& sum, float scale) {
  Row8 o;
#pragma unroll
  for (int k = 0; k < 8; ++k) o.v[k] = fmaf(scale, sum.v[k], old.v[k]);
  return o;
}

constexpr int kBatch = 4;  // rows of dx, and of dW, in flight

// A group of kLanes lanes (8 columns each) per slice and kLanes * 8 columns.
// part[slice][0]: the sum of the run that came in from the slice before,
// part[slice][1]: of the run that begins here and goes on behind it.  16384 x 3584
// fp32 added to 152064 rows: 91 us, 4.8 TB/s of dx and of the rows read and written.
template <class X, int kLanes, bool kAdd>
__global__ void __launch_bounds__(256) run_sum_kernel(const X* __restrict__ dx, Sorted in,
                                                      int n_chunks, int32_t d, int32_t V,
                                                      float scale, float* __restrict__ dW,
                                                      float* __restrict__ part) {
  const int64_t g = ((int64_t)blockIdx.x * 256 + threadIdx.x) / kLanes;
  const int64_t slice = g / n_chunks;
  const int q = threadIdx.x % kLanes;
  const int32_t col = ((int32_t)(g % n_chunks) * kLanes + q) * 8;
  if (slice >= in.n_slices) return;  // whole groups
  const bool live = col < d;
  const int64_t i0 = slice * in.slice, i1 = i0 + in.slice < in.T ? i0 + in.slice : in.T;
  bool begins = in.key_at(i0 - 1) != in.key[i0], open = false;
  Row8 acc{};
  for (int64_t base = i0; base < i1; base += kLanes) {
    // a lane per position: its key, its row, and whether its run ends there
    const int64_t mine = base + q;
    const uint32_t key = mine < i1 ? in.key[mine] : kNoKey;
    const uint32_t at = mine < i1 ? in.at[mine] : 0u;
    const bool end = key != in.key_at(mine + 1);
    const int here = i1 - base < kLanes ? (int)(i1 - base) : kLanes;
    for (int j0 = 0; j0 < here; j0 += kBatch) {
      Row8 row[kBatch], old[kBatch];
      uint32_t k[kBatch];
      bool ends[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        // (kLanes is a multiple of kBatch: the lane exists)
        k[j] = __shfl(key, j0 + j, kLanes);
        ends[j] = __shfl((int)end, j0 + j, kLanes) != 0;
        const uint32_t t = __shfl(at, j0 + j, kLanes);
        row[j] = Row8{};
        old[j] = Row8{};
        if (!live || k[j] >= (uint32_t)V) continue;
        row[j] = load8(dx + (int64_t)t * d + col);
        if (kAdd && ends[j]) old[j] = load8(static_cast<const float*>(dW) + (int64_t)k[j] * d + col);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (!live || k[j] >= (uint32_t)V) continue;
        add8(acc, row[j]);
        open = !ends[j];
        if (!ends[j]) continue;
        if (begins)
          store8(dW + (int64_t)k[j] * d + col, scaled(old[j], acc, scale));
        else
          store8(part + slice * 2 * d + col, acc);
        acc = Row8{};
        begins = true;
      }
    }
  }
  if (open) store8(part + (slice * 2 + (begins ? 1 : 0)) * d + col, acc);
}

// The runs that cross slices, by a block for each slice that one begins in and chunk
// of columns: its groups of lanes take equal stretches of the run's slices, and
// the first adds their sums: 6 us behind the above.
template <int kLanes, bool kAdd>
__global__ void __launch_bounds__(256) run_join_kernel(Sorted in, int n_chunks, int32_t d,
                                                       int32_t V, float scale,
                                                       float* __restrict__ dW,
                                                       const float* __restrict__ part) {
  constexpr int kGroups = 256 / kLanes, kJoin = 4;
  __shared__ Row8 sum_s[kGroups][kLanes];
  const int64_t slice = blockIdx.x / n_chunks;
  const int q = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  const int32_t col = ((int32_t)(blockIdx.x % n_chunks) * kLanes + q) * 8;
  const int64_t i0 = slice * in.slice, i1 = i0 + in.slice;
  if (i1 >= in.T) return;
  const uint32_t cur = in.key[i1 - 1], next = in.key[i1], first = in.key[i0],
                 prev = in.key_at(i0 - 1);
  if (cur >= (uint32_t)V || next != cur) return;
  if (first == cur && prev == cur) return;  // began before
  // slices behind this one that the run reaches into, tried 64 at a time by each wave
  int64_t more = 1;
  for (;;) {
    const int lane = threadIdx.x & 63;
    const uint64_t on = __ballot(in.key_at(i1 + (more + lane) * in.slice) == cur);
    if (on != ~0ull) {
      more += __builtin_ctzll(~on);
      break;
    }
    more += 64;
  }
  const bool live = col < d;
  Row8 acc{};
  if (live) {
    const float* p = part + (slice + 1) * 2 * d + col;
    const int64_t from = more * group / kGroups, to = more * (group + 1) / kGroups;
    if (group == 0) acc = load8(part + (slice * 2 + 1) * d + col);
    for (int64_t j = from; j < to; j += kJoin) {
      Row8 r[kJoin];
#pragma unroll
      for (int i = 0; i < kJoin; ++i)
        if (j + i < to) r[i] = load8(p + (j + i) * 2 * d);
#pragma unroll
      for (int i = 0; i < kJoin; ++i)
        if (j + i < to) add8(acc, r[i]);
    }
  }
  sum_s[group][q] = acc;
  __syncthreads();
  if (group != 0 || !live) return;
  for (int g = 1; g < kGroups; ++g) add8(acc, sum_s[g][q]);
  float* o = dW + (int64_t)cur * d + col;
  store8(o, scaled(kAdd ? load8(static_cast<const float*>(o)) : Row8{}, acc, scale));
}

// ---- few tokens -----------------------------------------------------------------

// Up to kFewMost tokens in one launch, without a sort: a block per token and chunk of
// columns marks the tokens of its id, goes on only if its own is the first of them,
// and sums their rows, a group of lanes an equal stretch of them.  The blocks behind
// clear the rows of dW that no token names, kFewFill float4 each.  Bound by latency:
// 256 x 64 into 1024 rows 4.5 us against 12.4 of the three launches with a sort, 512 x
// 3584 added 6.7 against 13.6.  A run is summed by one block for each of its chunks,
// so 512 equal tokens take 23 against 14 (1024 would 43 against 19), and clearing
// more than kFewClear is done sooner beside the sort (2.2 GB 379 against 391, but
// 545 MB 102 against 99).
// (A launch has less than 2^32 threads, 4 of them for 8 elements of dx: kFewPieces.)
constexpr int kFewMost = 512, kFewFill = 2048;
constexpr int64_t kFewPieces = 1 << 29;
constexpr int64_t kFewClear = 1 << 26;  // float4 of dW
template <class X, int kLanes, bool kAdd>
__global__ void __launch_bounds__(256) few_kernel(const X* __restrict__ dx,
                                                  const int32_t* __restrict__ tokens,
                                                  const int32_t* __restrict__ seq, int32_t T,
                                                  int n_chunks, int32_t d, int32_t V, float scale,
                                                  float* __restrict__ dW) {
  constexpr int kGroups = 256 / kLanes, kTokens = kFewMost / 256, kWords = kFewMost / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t key[kTokens];
#pragma unroll
  for (int c = 0; c < kTokens; ++c)
    key[c] = c * 256 + tid < T ? key_of(tokens, seq, c * 256 + tid, V) : kNoKey;
  if (!kAdd && (int)blockIdx.x >= T * n_chunks) {
    __shared__ uint8_t named[kFewFill];
    const int32_t d4 = d / 4, rows = d4 < kFewFill ? kFewFill / d4 : 1;
    const int64_t r0 = (int64_t)(blockIdx.x - T * n_chunks) * rows;
    const int32_t n = (int32_t)(r0 + rows < V ? rows : V - r0);
    for (int i = tid; i < n; i += 256) named[i] = 0;
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kTokens; ++c)
      if (key[c] >= r0 && key[c] - r0 < n) named[key[c] - r0] = 1;
    __syncthreads();
    float4* o = reinterpret_cast<float4*>(dW) + r0 * d4;
    for (uint32_t i = tid; i < (uint32_t)n * d4; i += 256)
      if (!named[i / d4]) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    return;
  }
  __shared__ uint64_t word[kWords];
  __shared__ uint16_t at_s[kFewMost];
  __shared__ Row8 sum_s[kGroups][kLanes];
  const int32_t t = blockIdx.x / n_chunks;
  const uint32_t id = key_of(tokens, seq, t, V);
  if (id >= (uint32_t)V) return;
  bool on[kTokens];
#pragma unroll
  for (int c = 0; c < kTokens; ++c) {
    on[c] = key[c] == id;
    const uint64_t m = __ballot(on[c]);
    if (lane == 0) word[c * 4 + wave] = m;
  }
  __syncthreads();
  const uint64_t mine = lane < kWords ? word[lane] : 0;
  const uint64_t below = lane < (t >> 6) ? ~0ull : lane == (t >> 6) ? (1ull << (t & 63)) - 1 : 0;
  if (__ballot((mine & below) != 0) != 0) return;  // not the first (the same in every wave)
  int upto = __popcll(mine);
#pragma unroll
  for (int off = 1; off < kWords; off <<= 1) {
    const int o = __shfl_up(upto, off, 64);
    if (lane >= off) upto += o;
  }
  const int m = __builtin_amdgcn_readlane(upto, kWords - 1);
#pragma unroll
  for (int c = 0; c < kTokens; ++c) {
    const int w = c * 4 + wave;
    const int before = w > 0 ? __builtin_amdgcn_readlane(upto, w - 1) : 0;
    if (on[c])
      at_s[before + __popcll(word[w] & ((1ull << lane) - 1))] = (uint16_t)(c * 256 + tid);
  }
  __syncthreads();
  const int q = tid % kLanes, group = tid / kLanes;
  const int32_t col = ((int32_t)(blockIdx.x % n_chunks) * kLanes + q) * 8;
  const bool live = col < d;
  const int each = (m + kGroups - 1) / kGroups, used = (m + each - 1) / each;
  const int from = group * each, to = from + each < m ? from + each : m;
  float* o = dW + (int64_t)id * d + col;
  Row8 acc{}, old{};
  if (kAdd && live && group == 0) old = load8(static_cast<const float*>(o));
  if (live) {
    for (int j = from; j < to; j += kBatch) {
      Row8 r[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        if (j + i < to) r[i] = load8(dx + (int64_t)at_s[j + i] * d + col);
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        if (j + i < to) add8(acc, r[i]);
    }
  }
  if (used > 1) {
    sum_s[group][q] = acc;
    __syncthreads();
  }
  if (group != 0 || !live) return;
  for (int g = 1; g < used; ++g) add8(acc, sum_s[g][q]);
  store8(o, scaled(old, acc, scale));
}

__global__ void __launch_bounds__(kSortThreads) zero_kernel(Fill f) { fill<kSortThreads>(f, blockIdx.x); }

// Keys per thread of a sort's tile: small tiles while their counts, which every block
// reads, stay few.
constexpr int64_t kShortSort = 65536;
inline int sort_items(int64_t T) { return T <= kShortSort ? 2 : 8; }
// Tiles of a block, so that those counts stay few however many tokens there are: every block
// reads the 2 KB of every block (2^22 tokens of 64 bf16 in all 414 us, with a tile a block 555;
// 2^23 596 / 1129; with 256 blocks 412 and 611).
constexpr int kSortBlocks = 512;
inline int sort_steps(int64_t T) {
  return (int)rbp::ceil_div(rbp::ceil_div(T, kSortThreads * sort_items(T)), kSortBlocks);
}
// Tokens sorted in one launch, by counting, which takes their square: up to kRankMost
// (4096 tokens of 896 bf16 17.2 us in all against 27.0 by tiles, 8192 25.3 / 30.4, 10007
// 34.5 / 34.0), or all kRankKeys that fit beside the clearing of much of dW, which
// hides it (8500 to 12288 tokens beside 272 MB 65 to 68 us against 71 to 76, 545 MB 110 to 112 /
// 116 to 119, 934 MB 183 to 189 / 187 to 191).
constexpr int kRankMost = 8192;
constexpr int64_t kBesideFill = 1 << 24;  // float4 of dW

// Positions per slice: enough slices to fill the chip (a group of lanes each, and
// chunk of columns), few enough that a run over many slices is joined soon.
constexpr int32_t kSliceLeast = 8, kSliceMost = 256, kSliceGroups = 4096;
inline int32_t slice_of(int64_t T, int n_chunks) {
  int32_t s = kSliceLeast;
  while (s < kSliceMost && T * n_chunks > (int64_t)s * kSliceGroups) s *= 2;
  return s;
}

// What a workspace provides for: at least the slices and sorting blocks of T tokens, and no fewer for
// more tokens (a longer batch may be cut into fewer of them), so that one sized for the largest
// batch serves all.
inline int64_t most_slices(int64_t T, int n_chunks) {
  return std::min(rbp::ceil_div(T, kSliceLeast),
                  std::max(rbp::ceil_div(T, kSliceMost), (int64_t)(kSliceGroups / n_chunks + 1)));
}
inline int64_t most_blocks(int64_t T) {
  return T <= kShortSort ? rbp::ceil_div(T, kSortThreads * 2)
                         : std::clamp<int64_t>(rbp::ceil_div(T, kSortThreads * 8),
                                               rbp::ceil_div(kShortSort, kSortThreads * 2),
                                               kSortBlocks);
}

struct EmbedWs {
  uint32_t *key[2], *at[2], *hist;
  float* part;
  size_t bytes;
};

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

int chunks_of(int32_t d) {
  int n = 1;
  with_lanes(d / 8, [&](auto lanes) {
    n = (int)rbp::ceil_div(d / 8, decltype(lanes)::value);
  });
  return n;
}

EmbedWs carve_embed(void* base, int64_t T, int32_t d) {
  rbp::WsCarver c(base);
  const size_t n = (size_t)T;
  EmbedWs w;
  for (int k = 0; k < 2; ++k) {
    w.key[k] = c.take<uint32_t>(n);
    w.at[k] = c.take<uint32_t>(n);
  }
  w.hist = c.take<uint32_t>((size_t)most_blocks(T) * kBins);
  const int32_t dd = d < 8 ? 8 : d;
  w.part = c.take<float>((size_t)most_slices(T, chunks_of(dd)) * 2 * (size_t)dd);
  w.bytes = rbp::align_up(c.used, 256);
  return w;
}

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

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
  const int64_t n = T * (d / 8), blocks = rbp::ceil_div(n, 256 * kRowPieces);
  // (a launch has less than 2^32 threads)
  RBP_REQUIRE(blocks < (1 << 24), RBP_EUNSUPPORTED, "policy_embed_fwd: T * d above 2^37 - 2^13");
  hipLaunchKernelGGL(n >= (1 << 19) ? embed_kernel<true> : embed_kernel<false>,
                     dim3((unsigned)blocks), dim3(256), 0, rbp::as_stream(stream), table, tokens,
                     seq_of_token, n, (uint32_t)(d / 8), V, scale, reinterpret_cast<uint4*>(out));
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
  // (columns are counted in 32 bits up to the end of a chunk of 512)
  RBP_REQUIRE(d <= INT32_MAX - 511, RBP_EUNSUPPORTED, "policy_embed_bwd: d above 2^31 - 512");
  RBP_REQUIRE(T * (d / 8) <= (int64_t(1) << 34), RBP_EUNSUPPORTED,
              "policy_embed_bwd: T * d above 2^37");
  RBP_REQUIRE(dW && (T == 0 || (dx && tokens)), RBP_EINVAL, "policy_embed_bwd: null pointer");
  RBP_REQUIRE(aligned(dW, 16) && aligned(dx, 16), RBP_EUNSUPPORTED,
              "policy_embed_bwd: dx and dW must be aligned to 16 bytes");
  RBP_REQUIRE(aligned(ws, 16), RBP_EINVAL, "policy_embed_bwd: ws must be aligned to 16 bytes");
  const size_t need = T == 0 ? 0 : rbp::embed_bwd_ws(T, d, V);
  RBP_REQUIRE(T == 0 || (ws && ws_bytes >= need), RBP_EWORKSPACE,
              "policy_embed_bwd: workspace needs %zu bytes, got %zu", need, ws_bytes);
  hipStream_t s = rbp::as_stream(stream);
  int bits = 1;
  while (bits < 31 && (V >> bits) != 0) ++bits;  // keys go up to V
  const int passes = (bits + kMaxDigit - 1) / kMaxDigit;
  // dW's rows to be cleared, in equal shares behind each launch of the sort
  const int64_t n_fill = accumulate_dW ? 0 : (int64_t)V * (d / 4);
  const bool one = T <= kRankMost || (T <= kRankKeys && n_fill >= kBesideFill);
  const int n_launches = T == 0 || one ? 1 : 2 * passes;
  int launch = 0;
  auto share = [&] {
    const int64_t from = n_fill * launch / n_launches, to = n_fill * (launch + 1) / n_launches;
    ++launch;
    // (a few stores a thread: 545 MB 93 us with 4096 blocks, 86 so; more where the
    // launch would have 2^32 threads)
    const int64_t blocks = rbp::ceil_div(to - from, kSortThreads * 4);
    return Fill{reinterpret_cast<float4*>(dW) + from, to - from,
                (int)(blocks < (1 << 21) ? blocks : (1 << 21))};
  };
  if (T == 0) {
    const Fill f = share();
    if (f.blocks == 0) return RBP_OK;
    hipLaunchKernelGGL(zero_kernel, dim3(f.blocks), dim3(kSortThreads), 0, s, f);
    RBP_CHECK_LAUNCH("policy_embed_bwd");
    return RBP_OK;
  }
  if (T <= kFewMost && n_fill <= kFewClear && T * (d / 8) < kFewPieces) {
    with_lanes(d / 8, [&](auto lanes) {
      constexpr int kLanes = decltype(lanes)::value;
      const int n_chunks = (int)rbp::ceil_div(d / 8, kLanes);
      const int32_t rows = d / 4 < kFewFill ? kFewFill / (d / 4) : 1;
      const int64_t blocks = T * n_chunks + (accumulate_dW ? 0 : rbp::ceil_div(V, rows));
      auto go = [&](auto kernel, auto* x) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, s, x, tokens, seq_of_token,
                           (int32_t)T, n_chunks, d, V, scale, dW);
      };
      const auto* x32 = static_cast<const float*>(dx);
      const auto* x16 = static_cast<const uint16_t*>(dx);
      if (dx_type == RBP_F32 && accumulate_dW)
        go(few_kernel<float, kLanes, true>, x32);
      else if (dx_type == RBP_F32)
        go(few_kernel<float, kLanes, false>, x32);
      else if (accumulate_dW)
        go(few_kernel<uint16_t, kLanes, true>, x16);
      else
        go(few_kernel<uint16_t, kLanes, false>, x16);
    });
    RBP_CHECK_LAUNCH("policy_embed_bwd");
    return RBP_OK;
  }
  const EmbedWs w = carve_embed(ws, T, d);
  const uint32_t *key = w.key[0], *at = w.at[0];
  if (one) {
    const Fill f = share();
    auto go = [&](auto own) {
      constexpr int kOwn = decltype(own)::value;
      hipLaunchKernelGGL(rank_kernel<kOwn>, dim3((unsigned)(rbp::ceil_div(T, kOwn) + f.blocks)),
                         dim3(kRankThreads), 0, s, tokens, seq_of_token, V, (int32_t)T, w.key[0],
                         w.at[0], f);
    };
    // Few tokens a block where many would leave units idle (4096 tokens 21.2 us in all
    // with 64, 19.1 with 32, 17.8 with 16; 8192 30.8 / 27.9 with 64 and 32), many beside
    // the clearing, which has use for the units (10007 tokens 111 us, 117 with 32).
    if (n_fill >= kBesideFill)
      go(std::integral_constant<int, 64>{});
    else if (T <= 16 * 256)
      go(std::integral_constant<int, 16>{});
    else
      go(std::integral_constant<int, 32>{});
  } else {
    auto go = [&](auto items, auto many) {
      constexpr int kItems = decltype(items)::value;
      constexpr bool kMany = decltype(many)::value;
      const int steps = sort_steps(T);
      const int n_blocks = (int)rbp::ceil_div(T, (int64_t)kSortThreads * kItems * steps);
      Keys in{tokens, seq_of_token, nullptr, nullptr, V};
      for (int p = 0; p < passes; ++p) {
        const int shift = p * kMaxDigit;
        Fill f = share();
        hipLaunchKernelGGL((sort_count_kernel<kItems, kMany>), dim3(n_blocks + f.blocks), dim3(kSortThreads),
                           0, s, in, T, shift, n_blocks, steps, w.hist, f);
        f = share();
        hipLaunchKernelGGL((sort_scatter_kernel<kItems, kMany>), dim3(n_blocks + f.blocks),
                           dim3(kSortThreads), 0, s, in, T, shift, w.hist, n_blocks, steps,
                           w.key[p & 1], w.at[p & 1], f);
        in.key = key = w.key[p & 1];
        in.at = at = w.at[p & 1];
      }
    };
    if (sort_items(T) == 2)
      go(std::integral_constant<int, 2>{}, std::false_type{});
    else if (sort_steps(T) == 1)
      go(std::integral_constant<int, 8>{}, std::false_type{});
    else
      go(std::integral_constant<int, 8>{}, std::true_type{});
  }
  RBP_CHECK_LAUNCH("policy_embed_bwd");
  with_lanes(d / 8, [&](auto lanes) {
    constexpr int kLanes = decltype(lanes)::value;
    const int n_chunks = (int)rbp::ceil_div(d / 8, kLanes);
    const int32_t slice = slice_of(T, n_chunks);
    const Sorted sorted{key, at, T, slice, rbp::ceil_div(T, slice)};
    const dim3 grid((unsigned)rbp::ceil_div(sorted.n_slices * n_chunks * kLanes, 256));
    auto go = [&](auto sum, auto join, auto* x) {
      hipLaunchKernelGGL(sum, grid, dim3(256), 0, s, x, sorted, n_chunks, d, V, scale, dW, w.part);
      hipLaunchKernelGGL(join, dim3((unsigned)(sorted.n_slices * n_chunks)), dim3(256), 0, s,
                         sorted, n_chunks, d, V, scale, dW, (const float*)w.part);
    };
    const auto* x32 = static_cast<const float*>(dx);
    const auto* x16 = static_cast<const uint16_t*>(dx);
    if (dx_type == RBP_F32 && accumulate_dW)
      go(run_sum_kernel<float, kLanes, true>, run_join_kernel<kLanes, true>, x32);
    else if (dx_type == RBP_F32)
      go(run_sum_kernel<float, kLanes, false>, run_join_kernel<kLanes, false>, x32);
    else if (accumulate_dW)
      go(run_sum_kernel<uint16_t, kLanes, true>, run_join_kernel<kLanes, true>, x16);
    else
      go(run_sum_kernel<uint16_t, kLanes, false>, run_join_kernel<kLanes, false>, x16);
  });
  RBP_CHECK_LAUNCH("policy_embed_bwd");
  return RBP_OK;
}
