// Root-mean-square norm with the residual's addition and an 8-bit output, and
// its gradient.
//
//   h = x + residual,  s = 1 / sqrt(mean(h^2) + eps),  y = h s w
//   8 bits: per group of columns (or per row) a = max(max |y|, floor),
//   scale = a / 448, q = e4m3(y 448 / a).
//   With g = dy w:  dx = dh + s (g - h s^2 mean(g h)),  dw = sum_t dy h s.
//
// Both directions are bound by memory: a row is read once, held in registers
// as 32-bit floats and written once.  h is rounded only where it is stored; y,
// its scales and q come from the unrounded sum, so each output is rounded once.
#include "rowio.h"

namespace taot {
namespace {

constexpr float kF8Max = 448.f;       // largest finite e4m3 value
constexpr float kF8Floor = 1e-30f;    // a group of smaller values (all zero) has floor / 448 as its scale
constexpr int kRowsOfBlock = 4;       // where a wave holds a row

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((aligned(1))) u32x2 u32x2_at;

// Eight values times inv in e4m3, to nearest even.  |v| inv exceeds 448 by a
// few units in the last place at most, which round to 448; NaN stays NaN.
__device__ __forceinline__ u32x2 to_f8(f32x8 v, float inv) {
  u32x2 r;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    int p = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * w] * inv, v[4 * w + 1] * inv, 0, false);
    r[w] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * w + 2] * inv, v[4 * w + 3] * inv, p, true);
  }
  return r;
}

template <bool FAR>
__device__ __forceinline__ void store_f8(uint8_t* p, u32x2 v, int n) {
  if (n >= 8) {
    auto* to = reinterpret_cast<u32x2_at*>(p);
    if constexpr (FAR) __builtin_nontemporal_store(v, to);
    else *to = v;
    return;
  }
#pragma unroll
  for (int u = 0; u < 8; ++u)
    if (u < n) p[u] = (uint8_t)(v[u / 4] >> (8 * (u % 4)));
}

// Sum (or maximum) over the `waves` waves of a row.  `slot` alternates between
// two sets of words from call to call, so one barrier a call is enough.
template <typename Op>
__device__ __forceinline__ float row_reduce(float v, Op op, float (*part)[16], int slot, int waves) {
  v = block_reduce<kWave>(v, op);
  if (waves > 1) {
    if ((threadIdx.x & (kWave - 1)) == 0) part[slot][threadIdx.x / kWave] = v;
    __syncthreads();
    v = part[slot][0];
    for (int w = 1; w < waves; ++w) v = op(v, part[slot][w]);
  }
  return v;
}

// `waves` waves hold a row (one: four rows a block); of their lanes, lane l has
// columns 8 (i lanes + l) .. + 7 for i < CPL, so a wave's accesses are contiguous
// and a group of 8 m columns is m neighbouring lanes at one i.
// h and y may lie in x's or the residual's memory: a lane has read all of its columns before it writes them.
// Bound by memory: 16384 x 4096 bfloat16, residual, groups of 128: 99 us for
// 604 MB, 6.1 TB/s.  1237 x 5003 float16, one scale a row: 10 us for 31 MB; all of
// its waves are resident at once, so nothing loads while others reduce and store.
template <typename T, int CPL, bool FAR>
__global__ void __launch_bounds__(1024)
add_rms_norm_kernel(const T* x, const T* residual, const void* __restrict__ weight, bool w_f32, int64_t rows,
                    int32_t H, float eps, int32_t group, T* h, T* y, uint8_t* __restrict__ q,
                    float* __restrict__ scale, float* __restrict__ rstd, int waves) {
  __shared__ float part[2][16];
  const int lanes = waves * kWave;
  const int lane = waves == 1 ? threadIdx.x & (kWave - 1) : threadIdx.x;
  const int64_t row = waves == 1 ? (int64_t)blockIdx.x * kRowsOfBlock + threadIdx.x / kWave : blockIdx.x;
  if (row >= rows) return;  // whole waves, and only where no wave waits for another
  const int64_t at = row * H;
  f32x8 v[CPL];
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int col = 8 * (i * lanes + lane), n = H - col;
    v[i] = load_row(x + at + col, n);
    if (residual) v[i] += load_row(residual + at + col, n);
  }
#pragma unroll
  for (int i = 0; i < CPL; ++i)
#pragma unroll
    for (int u = 0; u < 8; ++u) ss = fmaf(v[i][u], v[i][u], ss);
  if (h) {
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int col = 8 * (i * lanes + lane);
      store_row<FAR>(h + at + col, v[i], H - col);
    }
  }
  const float s = 1.f / sqrtf(row_reduce(ss, SumOp(), part, 0, waves) / (float)H + eps);
  if (lane == 0 && rstd) rstd[row] = s;
  float amax = 0.f;
  const int32_t groups = group > 0 ? (H + group - 1) / group : 1;
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int col = 8 * (i * lanes + lane), n = H - col;
    v[i] = v[i] * s * load_row_either<T>(weight, w_f32, col, n);
    if (y) store_row<FAR>(y + at + col, v[i], n);
    if (q) {
      float a = 0.f;
#pragma unroll
      for (int u = 0; u < 8; ++u) a = fmaxf(a, fabsf(v[i][u]));
      if (group > 0) {
        a = fmaxf(block_max(a, group / 8), kF8Floor);
        store_f8<FAR>(q + at + col, to_f8(v[i], kF8Max / a), n);
        if (n > 0 && col % group == 0) scale[row * groups + col / group] = a / kF8Max;
      } else {
        amax = fmaxf(amax, a);
      }
    }
  }
  if (q && group == 0) {
    amax = fmaxf(row_reduce(amax, MaxOp(), part, 1, waves), kF8Floor);
    const float inv = kF8Max / amax;
    if (lane == 0) scale[row] = amax / kF8Max;
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int col = 8 * (i * lanes + lane);
      store_f8<FAR>(q + at + col, to_f8(v[i], inv), H - col);
    }
  }
}

// A worker (`waves` waves) takes rows worker, worker + workers, ... and keeps its
// share of dw in registers until it writes it as one row of `partial`.  The
// next row is on its way while the present one is worked on, as long as the
// registers of 16 waves hold both (CPL <= 2).  dx may lie in dy's, dh's or h's
// memory: a row is read by its worker alone, each place by the lane that writes
// it, before it does.  8192 x 5120 bfloat16 with a
// residual's gradient: 68 us for 335 MB, 4.9 TB/s.
template <typename T, int CPL, bool FAR>
__global__ void __launch_bounds__(1024)
add_rms_norm_backward_kernel(const T* dy, const T* dh, const T* h, const float* __restrict__ rstd,
                             const void* __restrict__ weight, bool w_f32, int64_t rows, int32_t H, T* dx,
                             float* __restrict__ partial, int32_t workers, int waves) {
  using Raw = typename Row8<T>::vec;
  constexpr bool kAhead = CPL <= 2;
  __shared__ float part[2][16];
  const int lanes = waves * kWave;
  const int lane = waves == 1 ? threadIdx.x & (kWave - 1) : threadIdx.x;
  const int32_t worker = waves == 1 ? blockIdx.x * kRowsOfBlock + threadIdx.x / kWave : blockIdx.x;
  if (worker >= workers) return;
  f32x8 dw[CPL];
  Raw a[CPL], g[CPL], d[CPL], next_a[CPL], next_g[CPL], next_d[CPL];
  float s = rstd[worker], next_s = 0.f;
  auto fetch = [&](int64_t row, Raw* to_a, Raw* to_g, Raw* to_d) {
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int col = 8 * (i * lanes + lane), n = H - col;
      to_a[i] = load_raw(h + row * H + col, n);
      to_g[i] = load_raw(dy + row * H + col, n);
      if (dh && kAhead) to_d[i] = load_raw(dh + row * H + col, n);
    }
  };
#pragma unroll
  for (int i = 0; i < CPL; ++i) dw[i] = 0.f;
  fetch(worker, a, g, d);
  int slot = 0;
  for (int64_t row = worker; row < rows; row += workers) {
    const int64_t then = row + workers < rows ? row + workers : row;
    if constexpr (kAhead) {
      next_s = rstd[then];
      fetch(then, next_a, next_g, next_d);
    }
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int col = 8 * (i * lanes + lane), n = H - col;
      const f32x8 w = load_row_either<T>(weight, w_f32, col, n), A = widen(a[i]), G = widen(g[i]);
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        dw[i][u] = fmaf(G[u], A[u] * s, dw[i][u]);
        dot = fmaf(G[u] * w[u], A[u], dot);
      }
    }
    const float c = s * s * (row_reduce(dot, SumOp(), part, slot, waves) / (float)H);
    slot ^= 1;
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int col = 8 * (i * lanes + lane), n = H - col;
      f32x8 r = s * (widen(g[i]) * load_row_either<T>(weight, w_f32, col, n) - widen(a[i]) * c);
      if (dh) r += kAhead ? widen(d[i]) : load_row(dh + row * H + col, n);
      store_row<FAR>(dx + row * H + col, r, n);
    }
    if constexpr (kAhead) {
      s = next_s;
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        a[i] = next_a[i];
        g[i] = next_g[i];
        d[i] = next_d[i];
      }
    } else {
      s = rstd[then];
      fetch(then, a, g, d);
    }
  }
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int col = 8 * (i * lanes + lane);
    store_row(partial + (int64_t)worker * H + col, dw[i], H - col);
  }
}

// dw[c] = sum over the workers' rows, always in the same order: 32 columns a
// block, 32 threads a column.
__global__ void __launch_bounds__(1024)
dweight_kernel(const float* __restrict__ partial, int32_t workers, int32_t H, float* __restrict__ dweight) {
  __shared__ float sum[32][33];
  const int c = threadIdx.x % 32, r = threadIdx.x / 32;
  const int32_t col = blockIdx.x * 32 + c;
  float s = 0.f;
  if (col < H)
#pragma unroll 8
    for (int32_t w = r; w < workers; w += 32) s += partial[(int64_t)w * H + col];
  sum[r][c] = s;
  __syncthreads();
  if (r == 0 && col < H) {
#pragma unroll
    for (int k = 1; k < 32; ++k) s += sum[k][c];
    dweight[col] = s;
  }
}

struct Shape {
  int waves, cpl;
};
// Waves, and chunks of eight columns per lane, that hold a row of H: as few
// chunks as 16 waves allow (16384 rows of 2048 in 32 bits: 109 us, 116 with two;
// the gradient of 16384 x 4096, 98 and 124).
// Forward, rows of 16 bits take two where one would take 8 to 16 waves, with a
// residual 9 to 15.  128 MiB of bfloat16, new outputs, us with two and one chunk;
// y alone without a residual, then h, y and groups of 128 with one:
//   3592 columns, 8 waves    51, 58     112, 107
//   4096,         8          47, 53     104, 99
//   5120,        10          51, 65     102, 112
//   7168,        14          50, 59     102, 105
//   8184,        16          52, 60     113, 108
//   8192,        16          48, 59     104, 103
Shape shape_of(int32_t H, bool forward16, bool residual) {
  const int chunks = (H + 7) / 8, waves = (chunks + kWave - 1) / kWave;
  int cpl = forward16 && waves >= (residual ? 9 : 8) && waves <= (residual ? 15 : 16) ? 2 : 1;
  while (cpl * 16 * kWave < chunks) cpl *= 2;
  return {(chunks + cpl * kWave - 1) / (cpl * kWave), cpl};
}

// Workers of the gradient: as many on each of the 256 compute units, for a unit
// with one more than others is waited for by all.  16 waves a unit and up to what
// fills the last block, where the registers hold those (24 waves with one chunk a
// lane, 16 with more), else one block less.  In 16 bits, us with 4096 waves shared
// out as they come and so: 8192 rows of 5120 79 and 71, 8192 of 6144 97 and 79,
// 10000 of 3584 68 and 60; 4096 of 7168 84, 60 with the last block and 57 without.
// Of many more the partial sums cost more than they bring (60000 rows of 512: 57
// us, 62 with 24 waves a unit).
int32_t backward_workers(int64_t rows, int32_t H) {
  const Shape s = shape_of(H, false, true);
  int blocks = (16 + s.waves - 1) / s.waves;
  if (blocks * s.waves > (s.cpl == 1 ? 24 : 16)) --blocks;
  const int64_t most = 256 * blocks;
  return (int32_t)(rows < most ? rows : most);
}

template <typename F>
bool with_chunks(int cpl, F f) {
  if (cpl == 1) return f(std::integral_constant<int, 1>());
  if (cpl == 2) return f(std::integral_constant<int, 2>());
  if (cpl == 4) return f(std::integral_constant<int, 4>());
  return false;
}

template <typename T>
taot_status forward(const void* x, const void* residual, const void* weight, bool w_f32, int64_t rows, int32_t H,
                    float eps, int32_t group, void* h, void* y, uint8_t* q, float* scale, float* rstd,
                    hipStream_t stream) {
  const Shape s = shape_of(H, sizeof(T) == 2, residual != nullptr);
  const int per = s.waves == 1 ? kRowsOfBlock : 1;
  const int64_t groups = group > 0 ? (H + group - 1) / group : 1;
  const int64_t bytes = rows * H * (((h != nullptr) + (y != nullptr)) * (int64_t)sizeof(T) + (q != nullptr));
  const bool ok = with_chunks(s.cpl, [&](auto C) {
    auto* kernel = with_far(bytes, [](auto far) {
      return add_rms_norm_kernel<T, decltype(C)::value, far.value>;
    });
    for (int64_t r = 0; r < rows; r += kMaxBlocks * per) {
      const int64_t n = rows - r < kMaxBlocks * per ? rows - r : kMaxBlocks * per, at = r * H;
      kernel<<<(unsigned)((n + per - 1) / per), kWave * s.waves * per, 0, stream>>>(
          static_cast<const T*>(x) + at, residual ? static_cast<const T*>(residual) + at : nullptr, weight, w_f32, n, H,
          eps, group, h ? static_cast<T*>(h) + at : nullptr, y ? static_cast<T*>(y) + at : nullptr, q ? q + at : nullptr,
          scale ? scale + r * groups : nullptr, rstd ? rstd + r : nullptr, s.waves);
    }
    return true;
  });
  return ok && hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

template <typename T>
taot_status backward(const void* dy, const void* dh, const void* h, const float* rstd, const void* weight, bool w_f32,
                     int64_t rows, int32_t H, void* dx, float* dweight, float* partial, hipStream_t stream) {
  const int32_t workers = backward_workers(rows, H);
  bool ok = true;
  if (rows > 0) {
    const Shape s = shape_of(H, false, true);
    const int per = s.waves == 1 ? kRowsOfBlock : 1;
    ok = with_chunks(s.cpl, [&](auto C) {
      auto* kernel = with_far(rows * H * (int64_t)sizeof(T), [](auto far) {
        return add_rms_norm_backward_kernel<T, decltype(C)::value, far.value>;
      });
      kernel<<<(unsigned)((workers + per - 1) / per), kWave * s.waves * per, 0, stream>>>(
          static_cast<const T*>(dy), static_cast<const T*>(dh), static_cast<const T*>(h), rstd, weight, w_f32, rows, H,
          static_cast<T*>(dx), partial, workers, s.waves);
      return true;
    });
  }
  dweight_kernel<<<(unsigned)((H + 31) / 32), 1024, 0, stream>>>(partial, workers, H, dweight);
  return ok && hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

}  // namespace

size_t add_rms_norm_backward_ws(int64_t rows, int32_t H) {
  Carver c{nullptr};
  c.take<float>((size_t)backward_workers(rows, H) * (size_t)H);
  return c.off;
}

taot_status launch_add_rms_norm(const void* x, const void* residual, const void* weight, int64_t rows, int32_t H,
                                int32_t dtype, int32_t weight_dtype, float eps, int32_t group, void* h, void* y,
                                uint8_t* q, float* scale, float* rstd, hipStream_t stream) {
  const bool f32 = weight_dtype == TAOT_F32;
  if (dtype == TAOT_BF16)
    return forward<__bf16>(x, residual, weight, f32, rows, H, eps, group, h, y, q, scale, rstd, stream);
  if (dtype == TAOT_F16)
    return forward<_Float16>(x, residual, weight, f32, rows, H, eps, group, h, y, q, scale, rstd, stream);
  return forward<float>(x, residual, weight, f32, rows, H, eps, group, h, y, q, scale, rstd, stream);
}

taot_status launch_add_rms_norm_backward(const void* dy, const void* dh, const void* h, const float* rstd,
                                         const void* weight, int64_t rows, int32_t H, int32_t dtype,
                                         int32_t weight_dtype, void* dx, float* dweight, void* ws,
                                         hipStream_t stream) {
  const bool f32 = weight_dtype == TAOT_F32;
  Carver c{static_cast<char*>(ws)};
  float* partial = c.take<float>((size_t)backward_workers(rows, H) * (size_t)H);
  if (dtype == TAOT_BF16)
    return backward<__bf16>(dy, dh, h, rstd, weight, f32, rows, H, dx, dweight, partial, stream);
  if (dtype == TAOT_F16)
    return backward<_Float16>(dy, dh, h, rstd, weight, f32, rows, H, dx, dweight, partial, stream);
  return backward<float>(dy, dh, h, rstd, weight, f32, rows, H, dx, dweight, partial, stream);
}

}  // namespace taot
