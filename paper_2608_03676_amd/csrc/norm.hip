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
constexpr int kManyRows = 4096;

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

__device__ __forceinline__ void store_f8(uint8_t* p, u32x2 v, int n) {
  if (n >= 8) {
    *reinterpret_cast<u32x2_at*>(p) = v;
    return;
  }
#pragma unroll
  for (int u = 0; u < 8; ++u)
    if (u < n) p[u] = (uint8_t)(v[u / 4] >> (8 * (u % 4)));
}

// Sum (or maximum) over the WAVES waves of a row.  `slot` alternates between
// two sets of words from call to call, so one barrier a call is enough.
template <int WAVES, typename Op>
__device__ __forceinline__ float row_reduce(float v, Op op, float (*part)[16], int slot) {
  v = block_reduce<kWave>(v, op);
  if constexpr (WAVES > 1) {
    const int wid = threadIdx.x / kWave;
    if ((threadIdx.x & (kWave - 1)) == 0) part[slot][wid] = v;
    __syncthreads();
    v = part[slot][0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v = op(v, part[slot][w]);
  }
  return v;
}

constexpr int rows_of_block(int waves) { return waves == 1 ? 4 : 1; }

// WAVES waves hold a row; lane l has columns 8 (i LANES + l) .. + 7 for i < CPL,
// so a wave's accesses are contiguous and a group of 8 m columns is m
// neighbouring lanes at one i.
template <typename T, int WAVES, int CPL>
__global__ void __launch_bounds__(kWave* WAVES* rows_of_block(WAVES))
add_rms_norm_kernel(const T* __restrict__ x, const T* __restrict__ residual, const void* __restrict__ weight,
                    bool w_f32, int64_t rows, int32_t H, float eps, int32_t group, T* __restrict__ h,
                    T* __restrict__ y, uint8_t* __restrict__ q, float* __restrict__ scale,
                    float* __restrict__ rstd) {
  constexpr int kLanes = WAVES * kWave;
  __shared__ float part[2][16];
  const int lane = threadIdx.x % kLanes;
  const int64_t row = (int64_t)blockIdx.x * rows_of_block(WAVES) + threadIdx.x / kLanes;
  if (row >= rows) return;  // whole waves, and only where no wave waits for another
  const int64_t at = row * H;
  f32x8 v[CPL];
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int col = 8 * (i * kLanes + lane), n = H - col;
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
      const int col = 8 * (i * kLanes + lane);
      store_row(h + at + col, v[i], H - col);
    }
  }
  const float s = 1.f / sqrtf(row_reduce<WAVES>(ss, SumOp(), part, 0) / (float)H + eps);
  if (lane == 0 && rstd) rstd[row] = s;
  float amax = 0.f;
  const int32_t groups = group > 0 ? (H + group - 1) / group : 1;
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int col = 8 * (i * kLanes + lane), n = H - col;
    v[i] = v[i] * s * load_row_either<T>(weight, w_f32, col, n);
    if (y) store_row(y + at + col, v[i], n);
    if (q) {
      float a = 0.f;
#pragma unroll
      for (int u = 0; u < 8; ++u) a = fmaxf(a, fabsf(v[i][u]));
      if (group > 0) {
        a = fmaxf(block_max(a, group / 8), kF8Floor);
        store_f8(q + at + col, to_f8(v[i], kF8Max / a), n);
        if (n > 0 && col % group == 0) scale[row * groups + col / group] = a / kF8Max;
      } else {
        amax = fmaxf(amax, a);
      }
    }
  }
  if (q && group == 0) {
    amax = fmaxf(row_reduce<WAVES>(amax, MaxOp(), part, 1), kF8Floor);
    const float inv = kF8Max / amax;
    if (lane == 0) scale[row] = amax / kF8Max;
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int col = 8 * (i * kLanes + lane);
      store_f8(q + at + col, to_f8(v[i], inv), H - col);
    }
  }
}

// A worker (WAVES waves) takes rows worker, worker + workers, ... and keeps its
// share of dw in registers until it writes it as one row of `partial`.
template <typename T, int WAVES, int CPL>
__global__ void __launch_bounds__(kWave* WAVES* rows_of_block(WAVES))
add_rms_norm_backward_kernel(const T* __restrict__ dy, const T* __restrict__ dh, const T* __restrict__ h,
                             const float* __restrict__ rstd, const void* __restrict__ weight, bool w_f32,
                             int64_t rows, int32_t H, T* __restrict__ dx, float* __restrict__ partial,
                             int32_t workers) {
  constexpr int kLanes = WAVES * kWave;
  __shared__ float part[2][16];
  const int lane = threadIdx.x % kLanes;
  const int32_t worker = blockIdx.x * rows_of_block(WAVES) + threadIdx.x / kLanes;
  if (worker >= workers) return;
  f32x8 dw[CPL];
#pragma unroll
  for (int i = 0; i < CPL; ++i) dw[i] = 0.f;
  int slot = 0;
  for (int64_t row = worker; row < rows; row += workers) {
    const int64_t at = row * H;
    const float s = rstd[row];
    f32x8 a[CPL], g[CPL];
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int col = 8 * (i * kLanes + lane), n = H - col;
      a[i] = load_row(h + at + col, n);
      g[i] = load_row(dy + at + col, n);
    }
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int col = 8 * (i * kLanes + lane), n = H - col;
      const f32x8 w = load_row_either<T>(weight, w_f32, col, n);
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        dw[i][u] = fmaf(g[i][u], a[i][u] * s, dw[i][u]);
        g[i][u] *= w[u];
        dot = fmaf(g[i][u], a[i][u], dot);
      }
    }
    const float c = s * s * (row_reduce<WAVES>(dot, SumOp(), part, slot) / (float)H);
    slot ^= 1;
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
      const int col = 8 * (i * kLanes + lane), n = H - col;
      f32x8 r = s * (g[i] - a[i] * c);
      if (dh) r += load_row(dh + at + col, n);
      store_row(dx + at + col, r, n);
    }
  }
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const int col = 8 * (i * kLanes + lane);
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

int32_t backward_workers(int64_t rows) { return (int32_t)(rows < 512 ? rows : 512); }

struct Shape {
  int waves, cpl;
};
// Waves and chunks of eight columns per lane that hold a row of H.
Shape shape_of(int64_t rows, int32_t H) {
  const int chunks = (H + 7) / 8;
  int waves = 1;
  if (rows >= kManyRows) {
    if (chunks > 64 * 8) waves = chunks > 256 * 8 ? 16 : 4;
  } else {
    if (chunks > 64) waves = chunks > 256 ? 16 : 4;
  }
  int cpl = 1;
  while (cpl * waves * kWave < chunks) cpl *= 2;
  return {waves, cpl};
}

template <typename F>
bool with_shape(Shape s, F f) {
#define TAOT_SHAPE(W, C) \
  if (s.waves == W && s.cpl == C) return f(std::integral_constant<int, W>(), std::integral_constant<int, C>())
  TAOT_SHAPE(1, 1); TAOT_SHAPE(1, 2); TAOT_SHAPE(1, 4); TAOT_SHAPE(1, 8);
  TAOT_SHAPE(4, 1); TAOT_SHAPE(4, 2); TAOT_SHAPE(4, 4); TAOT_SHAPE(4, 8);
  TAOT_SHAPE(16, 1); TAOT_SHAPE(16, 2); TAOT_SHAPE(16, 4);
#undef TAOT_SHAPE
  return false;
}

template <typename T>
taot_status forward(const void* x, const void* residual, const void* weight, bool w_f32, int64_t rows, int32_t H,
                    float eps, int32_t group, void* h, void* y, uint8_t* q, float* scale, float* rstd,
                    hipStream_t stream) {
  const bool ok = with_shape(shape_of(rows, H), [&](auto W, auto C) {
    constexpr int w = W.value, c = C.value, per = rows_of_block(w);
    add_rms_norm_kernel<T, w, c><<<(unsigned)((rows + per - 1) / per), kWave * w * per, 0, stream>>>(
        static_cast<const T*>(x), static_cast<const T*>(residual), weight, w_f32, rows, H, eps, group,
        static_cast<T*>(h), static_cast<T*>(y), q, scale, rstd);
    return true;
  });
  return ok && hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

template <typename T>
taot_status backward(const void* dy, const void* dh, const void* h, const float* rstd, const void* weight, bool w_f32,
                     int64_t rows, int32_t H, void* dx, float* dweight, float* partial, hipStream_t stream) {
  const int32_t workers = backward_workers(rows);
  bool ok = true;
  if (rows > 0) {
    ok = with_shape(shape_of(rows, H), [&](auto W, auto C) {
      constexpr int w = W.value, c = C.value, per = rows_of_block(w);
      add_rms_norm_backward_kernel<T, w, c><<<(unsigned)((workers + per - 1) / per), kWave * w * per, 0, stream>>>(
          static_cast<const T*>(dy), static_cast<const T*>(dh), static_cast<const T*>(h), rstd, weight, w_f32, rows,
          H, static_cast<T*>(dx), partial, workers);
      return true;
    });
  }
  dweight_kernel<<<(unsigned)((H + 31) / 32), 1024, 0, stream>>>(partial, workers, H, dweight);
  return ok && hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

}  // namespace

size_t add_rms_norm_backward_ws(int64_t rows, int32_t H) {
  Carver c{nullptr};
  c.take<float>((size_t)backward_workers(rows) * (size_t)H);
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
  float* partial = c.take<float>((size_t)backward_workers(rows) * (size_t)H);
  if (dtype == TAOT_BF16)
    return backward<__bf16>(dy, dh, h, rstd, weight, f32, rows, H, dx, dweight, partial, stream);
  if (dtype == TAOT_F16)
    return backward<_Float16>(dy, dh, h, rstd, weight, f32, rows, H, dx, dweight, partial, stream);
  return backward<float>(dy, dh, h, rstd, weight, f32, rows, H, dx, dweight, partial, stream);
}

}  // namespace taot
