// Rows of logits, bf16 or fp32, with any alignment and distance between them
// (distill.hip, verify.hip).
#pragma once

#include "logits_epilogue.h"

namespace rbp {
namespace rows {

// The longest row that is taken.  Indices into a row are 32 bits wide and are compared with
// its end after they have stepped over it: by a tile of verify.hip's search (5120 tokens) or a
// block's threads, times the loads that are unrolled, at most 2^14 in all.
constexpr int32_t kMaxVocab = INT32_MAX - (1 << 14);

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
__device__ __forceinline__ float value(uint16_t v) { return rbp::lp::bf16_to_f32(v); }
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
  return make_uint4(rbp::lp::pack_bf16x2(x[0], x[1]), rbp::lp::pack_bf16x2(x[2], x[3]), rbp::lp::pack_bf16x2(x[4], x[5]),
                    rbp::lp::pack_bf16x2(x[6], x[7]));
}

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace rows
}  // namespace rbp
