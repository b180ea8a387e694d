// Rows as 8-bit integers with a scale each: what the products of 8-bit integers read.
//
//   v = x, or silu(g) u of a row [g | u];  a = max(max |v|, floor);
//   q = v (127 / a) to the nearest integer, to even where two are as near;  scale = a / 127
//
// Bound by memory: a row is read once, held in registers and written once (16384 gated
// rows of 2048 in bfloat16: 28 us for 168 MB, 5.9 TB/s; 37 with a division and the
// library's exponential a value).  The
// maximum is taken of the magnitudes' bits, in which NaN lies above infinity above
// all numbers: a row that holds either has no scale (NaN), and zeros.
#include "rowio.h"

namespace taot {
namespace {

constexpr float kMost = 127.f;
constexpr float kFloor = 1e-30f;  // a row of smaller values (all zero) has floor / 127 as its scale

typedef int8_t i8x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((aligned(1))) i8x8 i8x8_at;

__device__ __forceinline__ int row_max(int v, int (*part)[16], int waves) {
  v = block_reduce<kWave>(v, MaxOp());
  if (waves > 1) {
    if ((threadIdx.x & (kWave - 1)) == 0) part[0][threadIdx.x / kWave] = v;
    __syncthreads();
    v = part[0][0];
    for (int w = 1; w < waves; ++w) v = max(v, part[0][w]);
  }
  return v;
}

// Lanes hold columns as in the norm.
template <typename T, int CPL, bool GATED, bool FAR>
__global__ void __launch_bounds__(1024)
quantize_rows_kernel(const T* __restrict__ x, int64_t rows, int32_t H, int8_t* __restrict__ q,
                     float* __restrict__ scale, int waves) {
  __shared__ int part[1][16];
  const int lanes = waves * kWave;
  const int lane = waves == 1 ? threadIdx.x & (kWave - 1) : threadIdx.x;
  const int64_t row = waves == 1 ? (int64_t)blockIdx.x * kRowsOfBlock + threadIdx.x / kWave : blockIdx.x;
  if (row >= rows) return;  // whole waves, and only where no wave waits for another
  const T* src = x + row * H * (GATED ? 2 : 1);
  f32x8 v[CPL];
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int col = 8 * (i * lanes + lane);
    v[i] = load_row(src + col, H - col);
  }
  if constexpr (GATED) {
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int col = 8 * (i * lanes + lane);
      const f32x8 up = load_row(src + H + col, H - col);
#pragma unroll
      for (int u = 0; u < 8; ++u) v[i][u] = v[i][u] * __builtin_amdgcn_rcpf(1.f + exponential(within(-v[i][u], -150.f, 88.f))) * up[u];
    }
  }
  int top = __float_as_int(kFloor);
#pragma unroll
  for (int i = 0; i < CPL; ++i)
#pragma unroll
    for (int u = 0; u < 8; ++u) top = max(top, __float_as_int(v[i][u]) & 0x7fffffff);
  top = row_max(top, part, waves);
  const bool bad = top >= 0x7f800000;
  const float a = __int_as_float(top), inv = bad ? 0.f : kMost / a;
  if (lane == 0) scale[row] = bad ? __int_as_float(0x7fc00000) : a / kMost;
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int col = 8 * (i * lanes + lane), n = H - col;
    i8x8 r;
#pragma unroll
    for (int u = 0; u < 8; ++u) r[u] = bad ? (int8_t)0 : (int8_t)(int)rintf(v[i][u] * inv);
    int8_t* to = q + row * H + col;
    if (n >= 8) {
      if constexpr (FAR) __builtin_nontemporal_store(r, reinterpret_cast<i8x8_at*>(to));
      else *reinterpret_cast<i8x8_at*>(to) = r;
    } else {
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (u < n) to[u] = r[u];
    }
  }
}

template <typename T>
taot_status quantize(const void* x, int64_t rows, int32_t H, bool gated, int8_t* q, float* scale, hipStream_t stream) {
  const int chunks = (H + 7) / 8;
  // Rows of 16 bits take two chunks a lane, for loads under way (128 MiB of bfloat16, us with one and two: rows of 4096
  // 40.5 and 31.8, of 1024, 64 MiB, 21.7 and 17.8); gated rows have two loads as it is (16384 of 2048: 28.3 and 29.0).
  int cpl = sizeof(T) == 2 && !gated && chunks > kWave ? 2 : 1;
  while (cpl * 16 * kWave < chunks) cpl *= 2;
  const int waves = (chunks + cpl * kWave - 1) / (cpl * kWave), per = waves == 1 ? kRowsOfBlock : 1;
  const bool ok = with_chunks(cpl, [&](auto C) {
    auto* kernel = with_far(rows * H, [&](auto far) {
      return gated ? quantize_rows_kernel<T, decltype(C)::value, true, far.value>
                   : quantize_rows_kernel<T, decltype(C)::value, false, far.value>;
    });
    for (int64_t r = 0; r < rows; r += kMaxBlocks * per) {
      const int64_t n = rows - r < kMaxBlocks * per ? rows - r : kMaxBlocks * per;
      kernel<<<(unsigned)((n + per - 1) / per), kWave * waves * per, 0, stream>>>(
          static_cast<const T*>(x) + r * H * (gated ? 2 : 1), n, H, q + r * H, scale + r, waves);
    }
    return true;
  });
  return ok && hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

}  // namespace

taot_status launch_quantize_rows(const void* x, int64_t rows, int32_t H, bool gated, int32_t dtype, int8_t* q,
                                 float* scale, hipStream_t stream) {
  auto* call = dtype == TAOT_BF16 ? quantize<__bf16> : dtype == TAOT_F16 ? quantize<_Float16> : quantize<float>;
  return call(x, rows, H, gated, q, scale, stream);
}

}  // namespace taot
