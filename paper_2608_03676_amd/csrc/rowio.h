// Rows of 16- and 32-bit floating values: eight at a time as 32-bit floats, and
// reductions over neighbouring lanes of a wave.
#pragma once

#include <type_traits>

#include "common.h"

namespace taot {

typedef float f32x8 __attribute__((ext_vector_type(8)));

// Eight values of type T at any address that T allows: a row of odd length
// starts off every wider boundary, and the memory system takes 16-byte
// accesses there as well.
template <typename T>
struct Row8 {
  typedef T vec __attribute__((ext_vector_type(8)));
  typedef __attribute__((aligned(sizeof(T)))) vec at;
};

// n values from p, as they are (n of 8 and more: eight; 0 and less: none), zeros behind them.
template <typename T>
__device__ __forceinline__ typename Row8<T>::vec load_raw(const T* p, int n) {
  if (n >= 8) return *reinterpret_cast<const typename Row8<T>::at*>(p);
  typename Row8<T>::vec v;
#pragma unroll
  for (int u = 0; u < 8; ++u) v[u] = u < n ? p[u] : (T)0.f;
  return v;
}
template <typename V>
__device__ __forceinline__ f32x8 widen(V v) {
  return __builtin_convertvector(v, f32x8);
}
template <typename T>
__device__ __forceinline__ f32x8 load_row(const T* p, int n) {
  return widen(load_raw(p, n));
}

// Rounds to nearest even.  FAR: past the caches.
template <bool FAR = false, typename T>
__device__ __forceinline__ void store_row(T* p, f32x8 v, int n) {
  if (n >= 8) {
    const typename Row8<T>::vec r = __builtin_convertvector(v, typename Row8<T>::vec);
    auto* to = reinterpret_cast<typename Row8<T>::at*>(p);
    if constexpr (FAR) __builtin_nontemporal_store(r, to);
    else *to = r;
    return;
  }
#pragma unroll
  for (int u = 0; u < 8; ++u)
    if (u < n) p[u] = (T)v[u];
}

// A call's outputs of as much as the memory-side cache holds (256 MiB) are written
// past the caches: little of them would be left for who reads them next, and what
// is being read keeps its place.  Smaller ones are not, though the call itself may
// be faster so, for the next reader finds them there.  Call and the reader of its
// output (combine_rows of 8), us past the caches and through them, by the outputs'
// size; bfloat16, 4096 columns, inputs of several calls in turn:
//                               32       64       128       256       384 MiB
//   norm, y alone             21, 21   38, 36   76,  68  150, 144  219, 223
//   norm's gradient with dh   44, 41   74, 69  137, 134  262, 270
//   8 copies of a row         15, 14   27, 25   55,  47  118, 106  178, 208
//   the way back's gradient   22, 22   42, 40   90,  74  177, 180  264, 269
// Norm with h, y and groups of 128, and y's reader, 160, 240 and 320 MiB: 64, 63;
// 92, 99; 133, 138.
constexpr int64_t kFarBytes = 256 << 20;

// Blocks of a launch: their threads, up to 1024 each, are counted in 32 bits.
// Larger work is done by several launches.
constexpr int64_t kMaxBlocks = 1 << 21;

// f by whether `bytes` of output go past the caches.
template <typename F>
auto with_far(int64_t bytes, F f) {
  return bytes >= kFarBytes ? f(std::true_type()) : f(std::false_type());
}

// The same from a vector of T or of floats, chosen at run time by a value that
// all lanes share.
template <typename T>
__device__ __forceinline__ f32x8 load_row_either(const void* base, bool f32, int64_t col, int n) {
  return f32 ? load_row(static_cast<const float*>(base) + col, n) : load_row(static_cast<const T*>(base) + col, n);
}

// ---- lanes -------------------------------------------------------------------
// The value of the lane that step S pairs this one with: S = 0, 1: the lane
// whose number differs in bit S; 2: the mirror image in a half row of 8 lanes;
// 3: in a row of 16.  After steps 0..S of a reduction every lane of a block of
// 2^(S+1) lanes holds the block's result.  All lanes have to be active.
template <int S>
__device__ __forceinline__ int lane_step(int v) {
  static_assert(S >= 0 && S < 4, "steps within a row of 16 lanes");
  constexpr int ctrl = S == 0 ? 0xB1 : S == 1 ? 0x4E : S == 2 ? 0x141 : 0x140;
  return __builtin_amdgcn_mov_dpp(v, ctrl, 0xF, 0xF, true);
}
template <int S>
__device__ __forceinline__ float lane_step(float v) {
  return __int_as_float(lane_step<S>(__float_as_int(v)));
}

// The value of one lane, the same for all.
__device__ __forceinline__ int lane_value(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ float lane_value(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

// Result of `op` over blocks of L neighbouring lanes (L a power of two), in
// every lane of the block; op has to commute.  The order is fixed.  A whole
// wave's four rows of 16 lanes meet in scalar registers.
template <int L, typename V, typename Op>
__device__ __forceinline__ V block_reduce(V v, Op op) {
  if constexpr (L >= 2) v = op(v, lane_step<0>(v));
  if constexpr (L >= 4) v = op(v, lane_step<1>(v));
  if constexpr (L >= 8) v = op(v, lane_step<2>(v));
  if constexpr (L >= 16) v = op(v, lane_step<3>(v));
  if constexpr (L == 32) v = op(v, __shfl_xor(v, 16, kWave));
  if constexpr (L == 64) v = op(op(lane_value(v, 0), lane_value(v, 16)), op(lane_value(v, 32), lane_value(v, 48)));
  return v;
}

struct MaxOp {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
  __device__ __forceinline__ int operator()(int a, int b) const { return max(a, b); }
};
struct MinOp {
  __device__ __forceinline__ int operator()(int a, int b) const { return min(a, b); }
};
struct SumOp {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};

// The maximum over blocks of `lanes` neighbouring lanes, `lanes` a power of two
// that the whole wave shares.
__device__ __forceinline__ float block_max(float v, int lanes) {
  if (lanes >= 2) v = fmaxf(v, lane_step<0>(v));
  if (lanes >= 4) v = fmaxf(v, lane_step<1>(v));
  if (lanes >= 8) v = fmaxf(v, lane_step<2>(v));
  if (lanes >= 16) v = fmaxf(v, lane_step<3>(v));
  if (lanes >= 32) v = fmaxf(v, __shfl_xor(v, 16, kWave));
  if (lanes >= 64) v = fmaxf(v, __shfl_xor(v, 32, kWave));
  return v;
}

}  // namespace taot
