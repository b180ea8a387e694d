// Norms before and after a block, fused with its gate and the scaled residual,
// and their gradient.
//
//   a = 1 / sqrt(mean(x^2) + eps),  n = x a post     (n = x without post)
//   h = alpha residual + g n                         (g = 1 without a gate)
//   b = 1 / sqrt(mean(h^2) + eps),  y = h b w
//   With u = dy w:  D = dh + b (u - h b^2 mean(u h)),  dresidual = alpha D,
//   t = g D post,  dx = a (t - x a^2 mean(t x)),  dw = sum dy h b;
//   S_g = sum of D x a over the rows of gate g:  dgate_g = post S_g,
//   dpost = sum_g g S_g.
//
// Both directions are bound by memory: a row is read once, held in registers and
// written once.  h is rounded only where it is stored; y comes from the unrounded sum.
#include "rowio.h"

namespace taot {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// A norm's weights or a gate: null, of the rows' type, or floats.
struct Vector {
  const void* p;
  bool f32;
};
template <typename T>
__device__ __forceinline__ f32x8 factor(const Vector& v, int64_t col, int n) {
  return v.p ? load_row_either<T>(v.p, v.f32, col, n) : f32x8(1.f);
}

// A row's odd end.  Its lane takes the row's last eight columns, some of which the lane
// before it has too: both work the same out and write it, and one of them adds it to the
// row's sums.  (With single loads there, for which the others of the row wait: 16384 x
// 4095 141 us, 127 so, gradient of 8192 x 5119 195 and 133.)
enum Edge { kWholeRows, kOddRows, kAnyRows };  // H % 8 == 0; other H from 8 on; any H, with single loads
template <Edge EDGE>
struct Place {
  // first column, how many (8 or 0, kAnyRows: up to the row's end), how many of them the lane before has too
  int col, n, back;
  __device__ __forceinline__ Place(int chunk, int32_t H)
      : col(8 * chunk), n(EDGE == kAnyRows ? H - col : col < H ? 8 : 0), back(0) {
    if (EDGE == kOddRows && n && H - col < 8) {
      back = 8 - (H - col);
      col -= back;
    }
  }
  __device__ __forceinline__ bool adds(int u) const { return EDGE != kOddRows || u >= back; }
  template <typename T>
  __device__ __forceinline__ void load(const T* from, typename Row8<T>::vec& to) const {  // `to` is 0 if there are no columns
    if (EDGE == kAnyRows) to = load_raw(from + col, n);
    else if (n) to = *reinterpret_cast<const typename Row8<T>::at*>(from + col);
  }
  template <bool FAR, typename T>
  __device__ __forceinline__ void store(T* to, f32x8 v) const {
    if (EDGE == kAnyRows || n) store_row<FAR>(to + col, v, n);
  }
};

// Lanes hold columns as in the norm without a gate; h may lie in x's or the
// residual's memory: all of a lane's columns are read before they are written.
// 16384 x 4096 bfloat16, post and gate: 95 us for 537 MB, 5.7 TB/s.
template <typename T, int CPL, bool FAR, Edge EDGE>
__global__ void __launch_bounds__(1024)
block_norm_kernel(const T* x, const T* residual, Vector post, Vector gate, int64_t per_gate, int64_t first,
                  Vector weight, int64_t rows, int32_t H, float eps, float alpha, T* h, T* y,
                  float* __restrict__ rstd_x, float* __restrict__ rstd_h, int waves) {
  using At = Place<EDGE>;
  __shared__ float part[2][16];
  const int lanes = waves * kWave;
  const int lane = waves == 1 ? threadIdx.x & (kWave - 1) : threadIdx.x;
  const int64_t row = waves == 1 ? (int64_t)blockIdx.x * kRowsOfBlock + threadIdx.x / kWave : blockIdx.x;
  if (row >= rows) return;  // whole waves, and only where no wave waits for another
  const int64_t at = row * H, gate_at = gate.p ? (first + row) / per_gate * H : 0;
  f32x8 v[CPL];
  typename Row8<T>::vec raw[CPL], r[CPL];
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    raw[i] = r[i] = (T)0.f;
    At(i * lanes + lane, H).load(x + at, raw[i]);
    v[i] = widen(raw[i]);
    At(i * lanes + lane, H).load(residual + at, r[i]);
  }
  float a = 1.f;
  if (post.p) {
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < CPL; ++i)
#pragma unroll
      for (int u = 0; u < 8; ++u) ss = At(i * lanes + lane, H).adds(u) ? fmaf(v[i][u], v[i][u], ss) : ss;
    a = 1.f / sqrtf(row_reduce(ss, SumOp(), part, 0, waves) / (float)H + eps);
    if (lane == 0 && rstd_x) rstd_x[row] = a;
  } else if (EDGE == kOddRows && waves > 1) {
    __syncthreads();  // the lane before may be another wave's, and write where this one reads
  }
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const At p(i * lanes + lane, H);
    if (post.p) v[i] = v[i] * a * factor<T>(post, p.col, p.n);
    if (gate.p) v[i] = v[i] * factor<T>(gate, gate_at + p.col, p.n);
    v[i] = alpha * widen(r[i]) + v[i];
#pragma unroll
    for (int u = 0; u < 8; ++u) ss = p.adds(u) ? fmaf(v[i][u], v[i][u], ss) : ss;
    if (h) p.template store<FAR>(h + at, v[i]);
  }
  if (!weight.p) return;
  const float b = 1.f / sqrtf(row_reduce(ss, SumOp(), part, 1, waves) / (float)H + eps);
  if (lane == 0 && rstd_h) rstd_h[row] = b;
#pragma unroll
  for (int i = 0; i < CPL; ++i) {
    const At p(i * lanes + lane, H);
    if (y) p.template store<FAR>(y + at, v[i] * b * factor<T>(weight, p.col, p.n));
  }
}

// The rows of a worker: of one gate, where gates are few and several workers share
// one (rows first, first + step, ...), or all rows of gates worker, worker + workers, ...
struct Share {
  int64_t gates, per_gate, each;  // `each` workers a gate; 0: a worker has whole gates
};

template <bool MANY>
struct Rows {
  int64_t row, step, left, seg, in_seg = 0, per_gate;
  int32_t workers;
  __device__ __forceinline__ Rows(const Share& s, int32_t worker, int32_t all) : per_gate(s.per_gate), workers(all) {
    if (MANY) {
      seg = worker;
      row = worker * s.per_gate;
      step = 1;
      left = (s.gates - worker + all - 1) / all * s.per_gate;
    } else {
      seg = worker / s.each;
      const int64_t j = worker % s.each;
      row = seg * s.per_gate + j;
      step = s.each;
      left = (s.per_gate - j + s.each - 1) / s.each;
    }
  }
  // The row is the last of a gate that the worker has whole.
  __device__ __forceinline__ bool ends() const { return in_seg + 1 == per_gate; }
  // The row behind this one; the last row itself.
  __device__ __forceinline__ int64_t then() const {
    return left == 1 ? row : MANY && ends() ? (seg + workers) * per_gate : row + step;
  }
  __device__ __forceinline__ void next() {
    row = then();
    if (MANY) {
      const bool e = ends();
      seg += e ? workers : 0;
      in_seg = e ? 0 : in_seg + 1;
    }
    --left;
  }
};

// Sums of three values over a row's waves, with one barrier: `slot` takes turns.
struct Three {
  float a, b, c;
};
__device__ __forceinline__ Three row_sums(Three v, f32x4 (*part)[16], int slot, int waves) {
  v = {block_reduce<kWave>(v.a, SumOp()), block_reduce<kWave>(v.b, SumOp()), block_reduce<kWave>(v.c, SumOp())};
  if (waves > 1) {
    const int lane = threadIdx.x & (kWave - 1), wid = threadIdx.x / kWave;
    if (lane == 0) part[slot][wid] = f32x4{v.a, v.b, v.c, 0.f};
    __syncthreads();
    const f32x4 w = lane % 16 < waves ? part[slot][lane % 16] : f32x4(0.f);
    v = {block_reduce<16>(w[0], SumOp()), block_reduce<16>(w[1], SumOp()), block_reduce<16>(w[2], SumOp())};
  }
  return v;
}

// A worker (`waves` waves) keeps its share of dw and of S (MANY: of dpost) in
// registers until it writes them as one row of the partial sums; a gate that a
// worker has alone gets its gradient at once.  The next row is on its way while
// the present one is worked on.  dresidual and dx may lie in an input's memory: a row
// is read by its worker alone, and all of it before any of it is written.
//
// With H = b h, X = a x, q = gate post, e = b dy w + dh and c = b mean(dy w H) it is
// D = e - c H, so sum(D q X) = sum(e q X) - c sum(H q X): all sums of a row are taken at
// once, of normed rows, for powers of b and a leave 32 bits where D and dx do not (8192 x 5120
// bfloat16, dh, post, 4 gates: 136 us with a sum after the other, 108 so and with as many
// workers as are resident).  101 us for 503 MB, 5.0 TB/s, and 6 for the workers' sums: of
// the 16 waves whose registers a compute unit holds, a row of 5120 fills ten.
template <typename T, bool FAR, bool MANY, Edge EDGE>
__global__ void __launch_bounds__(1024)
block_norm_backward_kernel(const T* dy, const T* dh, const T* x, const T* h, const float* __restrict__ rstd_x,
                           const float* __restrict__ rstd_h, Vector post, Vector gate, Share share, Vector weight,
                           int32_t H, float alpha, T* dx, T* dresidual, float* __restrict__ dgate,
                           float* __restrict__ part_w, float* __restrict__ part_s, int32_t workers, int waves) {
  using Raw = typename Row8<T>::vec;
  __shared__ f32x4 part[2][16];
  const int lane = waves == 1 ? threadIdx.x & (kWave - 1) : threadIdx.x;
  const int32_t worker = waves == 1 ? blockIdx.x * kRowsOfBlock + threadIdx.x / kWave : blockIdx.x;
  if (worker >= workers) return;
  const Place<EDGE> place(lane, H);
  const int col = place.col, n = place.n;
  constexpr bool kAhead = sizeof(T) == 2;  // the registers of 16 waves hold two rows of 16 bits
  const bool sums = post.p || gate.p;
  Rows<MANY> rows(share, worker, workers);
  auto load = [&](const T* from, int64_t row, Raw& to) { place.load(from + row * H, to); };
  const f32x8 w = factor<T>(weight, col, n);
  f32x8 q = factor<T>(gate, rows.seg * H + col, n) * factor<T>(post, col, n);
  f32x8 dw = 0.f, S = 0.f, dp = 0.f;
  Raw rx = {}, rh = {}, ry = {}, rd = {}, nx = {}, nh = {}, ny = {}, nd = {};
  auto fetch = [&](int64_t row, Raw& fx, Raw& fh, Raw& fy, Raw& fd) {
    if (sums) load(x, row, fx);
    if (weight.p) {
      load(h, row, fh);
      load(dy, row, fy);
    }
    if (dh) load(dh, row, fd);
  };
  if (kAhead) fetch(rows.row, rx, rh, ry, rd);
  float a = post.p ? rstd_x[rows.row] : 1.f, b = weight.p ? rstd_h[rows.row] : 0.f;
  int slot = 0;
  for (; rows.left > 0; rows.next()) {
    const int64_t at = rows.row * H, gate_at = rows.seg * H + col, then = rows.then();
    if (kAhead) fetch(then, nx, nh, ny, nd);
    if constexpr (!kAhead) {
      // Zeros for what is not read, so that the row before keeps no registers: rows scaled by b and a are new ones
      // (8192 x 4096 float32, a gate a row: 281 us with the old rows kept, 256 unscaled, 212 so).
      rx = rh = ry = rd = Raw{};
      fetch(rows.row, rx, rh, ry, rd);
    }
    const float next_a = post.p ? rstd_x[then] : 1.f, next_b = weight.p ? rstd_h[then] : 0.f;
    const f32x8 Y = widen(ry), Hh = widen(rh) * b, X = widen(rx) * a;
    f32x8 e = widen(rd);
    Three s = {0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float v = Y[u] * w[u], qx = q[u] * X[u];
      e[u] = fmaf(b, v, e[u]);
      dw[u] = fmaf(Y[u], Hh[u], dw[u]);
      const bool mine = place.adds(u);
      s.a = mine ? fmaf(v, Hh[u], s.a) : s.a;
      s.b = mine ? fmaf(e[u], qx, s.b) : s.b;
      s.c = mine ? fmaf(Hh[u], qx, s.c) : s.c;
    }
    s = row_sums(s, part, slot, waves);
    slot ^= 1;
    const float c = b * (s.a / (float)H), m = fmaf(-c, s.c, s.b) / (float)H;
    f32x8 D, t;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      D[u] = fmaf(-c, Hh[u], e[u]);
      S[u] = fmaf(D[u], X[u], S[u]);
      t[u] = D[u] * q[u];
      if (post.p) t[u] = a * fmaf(-m, X[u], t[u]);
    }
    place.template store<FAR>(dresidual + at, alpha * D);
    place.template store<FAR>(dx + at, t);
    if (MANY && rows.ends()) {
      const f32x8 p = factor<T>(post, col, n);
      if (dgate) store_row(dgate + gate_at, S * p, n);
      dp += S * factor<T>(gate, gate_at, n);
      S = 0.f;
      if (rows.left > 1) q = factor<T>(gate, gate_at + (int64_t)workers * H, n) * p;
    }
    a = next_a;
    b = next_b;
    if constexpr (kAhead) {
      rx = nx;
      rh = nh;
      ry = ny;
      rd = nd;
    }
  }
  if (part_w) store_row(part_w + (int64_t)worker * H + col, dw, n);
  if (part_s) store_row(part_s + (int64_t)worker * H + col, MANY ? dp : S, n);
}

// The same for rows wider than the registers hold beside the sums (more than 8192
// columns), and for those of less than eight: the 16 waves read a row's inputs three
// times, the later ones out of the L2 cache, and keep their sums in memory, each lane its
// own columns.  A gate that a worker has alone is summed where its gradient goes.  4096 x
// 8200 bfloat16, dh, post, a gate: 277 us for 403 MB (8192 columns 87), 2048 x 16384 234; the
// sums in memory are another 16 bytes a column, read and written, and issue is 72.
template <typename T, bool FAR, bool MANY>
__global__ void __launch_bounds__(1024)
block_norm_backward_wide_kernel(const T* dy, const T* dh, const T* x, const T* h, const float* __restrict__ rstd_x,
                                const float* __restrict__ rstd_h, Vector post, Vector gate, Share share, Vector weight,
                                int32_t H, float alpha, T* dx, T* dresidual, float* dgate, float* part_w,
                                float* part_s, int32_t workers) {
  constexpr int kWaves = 16;
  __shared__ float part[2][16];
  const int32_t worker = blockIdx.x;
  const bool sums = post.p || gate.p;
  Rows<MANY> rows(share, worker, workers);
  bool first = true;
  int slot = 0;
  auto add = [](float* to, f32x8 v, int n, bool begins) {
    if (!begins) v += load_row(to, n);
    store_row(to, v, n);
  };
  for (; rows.left > 0; rows.next()) {
    const int64_t at = rows.row * H, gate_at = rows.seg * H;
    const float a = post.p ? rstd_x[rows.row] : 1.f, b = weight.p ? rstd_h[rows.row] : 0.f;
    float dot = 0.f;
    if (weight.p) {
      for (int col = 8 * (int)threadIdx.x; col < H; col += 8 * kWaves * kWave) {
        const int n = H - col;
        const f32x8 w = factor<T>(weight, col, n), Y = load_row(dy + at + col, n), Hh = load_row(h + at + col, n) * b;
#pragma unroll
        for (int u = 0; u < 8; ++u) dot = fmaf(Y[u] * w[u], Hh[u], dot);
      }
      dot = row_reduce(dot, SumOp(), part, slot, kWaves) / (float)H;
      slot ^= 1;
    }
    const float c = b * dot;
    auto D_of = [&](int col, int n) {
      f32x8 D = 0.f;
      if (weight.p) D = b * (load_row(dy + at + col, n) * factor<T>(weight, col, n) - load_row(h + at + col, n) * c);
      if (dh) D += load_row(dh + at + col, n);
      return D;
    };
    float m = 0.f;
    if (post.p) {
      dot = 0.f;
      for (int col = 8 * (int)threadIdx.x; col < H; col += 8 * kWaves * kWave) {
        const int n = H - col;
        const f32x8 t = D_of(col, n) * factor<T>(gate, gate_at + col, n) * factor<T>(post, col, n);
        const f32x8 X = load_row(x + at + col, n) * a;
#pragma unroll
        for (int u = 0; u < 8; ++u) dot = fmaf(t[u], X[u], dot);
      }
      m = row_reduce(dot, SumOp(), part, slot, kWaves) / (float)H;
      slot ^= 1;
    }
    for (int col = 8 * (int)threadIdx.x; col < H; col += 8 * kWaves * kWave) {
      const int n = H - col;
      const f32x8 D = D_of(col, n), g = factor<T>(gate, gate_at + col, n), p = factor<T>(post, col, n);
      f32x8 X = 0.f;
      if (sums) X = load_row(x + at + col, n) * a;
      if (part_w) add(part_w + (int64_t)worker * H + col, load_row(dy + at + col, n) * load_row(h + at + col, n) * b, n, first);
      if (MANY) {
        if (dgate) add(dgate + gate_at + col, D * X * p, n, rows.in_seg == 0);
        if (part_s) add(part_s + (int64_t)worker * H + col, D * X * g, n, first);
      } else if (part_s) {
        add(part_s + (int64_t)worker * H + col, D * X, n, first);
      }
      f32x8 t = D * g;
      if (post.p) t = a * (t * p - X * m);
      store_row<FAR>(dresidual + at + col, alpha * D, n);
      store_row<FAR>(dx + at + col, t, n);
    }
    first = false;
  }
}

// Column sums of `n` rows of partial sums in a fixed order: 32 columns a block, 32 threads a column.
__device__ __forceinline__ float column_sum(const float* __restrict__ partial, int64_t n, int32_t H, int32_t col, int r,
                                            int c, float (*sum)[33]) {
  float s = 0.f;
  if (col < H)
#pragma unroll 8
    for (int64_t w = r; w < n; w += 32) s += partial[w * H + col];
  sum[r][c] = s;
  __syncthreads();
  if (r == 0)
#pragma unroll
    for (int k = 1; k < 32; ++k) s += sum[k][c];
  return s;
}

// blockIdx.y < sets: S of that gate from its workers' rows (MANY: dpost itself), or of
// all gates where they are few, and with them dpost; the row of blocks behind: dw.
constexpr int kFewGates = 32;
template <typename T>
__global__ void __launch_bounds__(1024)
block_norm_sums_kernel(const float* __restrict__ part_w, const float* __restrict__ part_s, int64_t workers, bool many,
                       int64_t sets, int64_t gates, int64_t each, Vector post, Vector gate, int32_t H,
                       float* __restrict__ dweight, float* __restrict__ dpost, float* __restrict__ dgate,
                       float* __restrict__ S) {
  __shared__ float sum[32][33];
  const int c = threadIdx.x % 32, r = threadIdx.x / 32;
  const int32_t col = blockIdx.x * 32 + c;
  const int64_t set = blockIdx.y;
  if (set == sets) {
    if (!dweight) return;
    const float s = column_sum(part_w, workers, H, col, r, c, sum);
    if (r == 0 && col < H) dweight[col] = s;
    return;
  }
  if (many) {
    const float s = column_sum(part_s, workers, H, col, r, c, sum);
    if (r == 0 && col < H) dpost[col] = s;
    return;
  }
  const float p = col < H ? factor<T>(post, col, 1)[0] : 0.f;
  if (gates > kFewGates) {
    const float s = column_sum(part_s + set * each * H, each, H, col, r, c, sum);
    if (r != 0 || col >= H) return;
    if (dgate) dgate[set * H + col] = s * p;
    if (dpost) S[set * H + col] = s;
    return;
  }
  // thread r: gate r % gates, every `per`-th of its workers
  const int n = (int)gates, mine = r % n, per = 32 / n;
  float s = 0.f;
  if (col < H && r < per * n)
#pragma unroll 8
    for (int64_t w = r / n; w < each; w += per) s += part_s[(mine * each + w) * H + col];
  sum[r][c] = s;
  __syncthreads();
  if (r != 0 || col >= H) return;
  float all = 0.f;
  for (int g = 0; g < n; ++g) {
    s = 0.f;
    for (int k = 0; k < per; ++k) s += sum[k * n + g][c];
    if (dgate) dgate[(int64_t)g * H + col] = s * p;
    all = fmaf(s, gate.p ? factor<T>(gate, (int64_t)g * H + col, 1)[0] : 1.f, all);
  }
  if (dpost) dpost[col] = all;
}

// dpost = sum over the gates of g S_g.
template <typename T>
__global__ void __launch_bounds__(1024)
block_norm_post_kernel(const float* __restrict__ S, Vector gate, int64_t gates, int32_t H, float* __restrict__ dpost) {
  __shared__ float sum[32][33];
  const int c = threadIdx.x % 32, r = threadIdx.x / 32;
  const int32_t col = blockIdx.x * 32 + c;
  float s = 0.f;
  if (col < H)
    for (int64_t g = r; g < gates; g += 32) s = fmaf(S[g * H + col], factor<T>(gate, g * H + col, 1)[0], s);
  sum[r][c] = s;
  __syncthreads();
  if (r == 0 && col < H) {
#pragma unroll
    for (int k = 1; k < 32; ++k) s += sum[k][c];
    dpost[col] = s;
  }
}

struct Shape {
  int waves, cpl;
};
// Waves, and chunks of eight columns a lane, that hold a row.  Forward, rows of 16 bits
// take two chunks where one is more than a wave (us with one and two, bfloat16 with post
// and gate: 16384 rows of 4096 108 and 96, of 2048 54 and 49, 8192 of 5120 79 and 66, of
// 8192 112 and 96; 8192 of 4096 in 32 bits 102 and 111).
Shape shape_of(int32_t H, bool forward16 = false) {
  const int chunks = (H + 7) / 8;
  int cpl = forward16 && chunks > kWave ? 2 : 1;
  while (cpl * 16 * kWave < chunks) cpl *= 2;
  return {(chunks + cpl * kWave - 1) / (cpl * kWave), cpl};
}

struct Split {
  Share share;
  int32_t workers;
  bool many;
};
// Workers of the gradient: as many on each compute unit as its registers hold, 16
// waves.  Gates that are as many, or have one row each, are taken whole (1753 x 511 in
// 32 bits, a gate a row: 98 us where each gate's sums are a launch's blocks, 28 so).
Split split_of(int64_t rows, int32_t H, int64_t gates) {
  const int waves = shape_of(H).waves;
  const int64_t most = 256 * (16 / waves), per = rows / gates;
  if (gates >= most || (gates > 1 && per == 1)) return {{gates, per, 0}, (int32_t)(gates < most ? gates : most), true};
  int64_t each = (most + gates - 1) / gates;
  if (each > per) each = per;
  return {{gates, per, each}, (int32_t)(each * gates), false};
}

struct Partial {
  float *w, *s, *S;
  size_t bytes;
};
Partial carve(void* ws, int64_t rows, int32_t H, int64_t gates) {
  Carver c{static_cast<char*>(ws)};
  const Split s = split_of(rows, H, gates);
  Partial p;
  p.w = c.take<float>((size_t)s.workers * H);
  p.s = c.take<float>((size_t)s.workers * H);
  p.S = c.take<float>(s.many || gates <= kFewGates ? 0 : (size_t)gates * H);
  p.bytes = c.off;
  return p;
}

__global__ void __launch_bounds__(256) zero_kernel(float* __restrict__ p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = 0.f;
}

template <typename T>
taot_status forward(const BlockNormArgs& a, hipStream_t stream) {
  const Shape s = shape_of(a.H, sizeof(T) == 2);
  const int per = s.waves == 1 ? kRowsOfBlock : 1;
  const Vector post{a.post, a.weight_f32}, gate{a.gate, a.gate_f32}, weight{a.weight, a.weight_f32};
  const int64_t per_gate = a.gate ? a.rows / a.gates : 1;
  const bool ok = with_chunks(s.cpl, [&](auto C) {
    auto* kernel = with_far(a.rows * a.H * ((a.h != nullptr) + (a.y != nullptr)) * (int64_t)sizeof(T), [&](auto far) {
      return a.H % 8 && a.H >= 8 ? block_norm_kernel<T, decltype(C)::value, far.value, kOddRows>
                                 : block_norm_kernel<T, decltype(C)::value, far.value, kAnyRows>;
    });
    for (int64_t r = 0; r < a.rows; r += kMaxBlocks * per) {
      const int64_t n = a.rows - r < kMaxBlocks * per ? a.rows - r : kMaxBlocks * per, at = r * a.H;
      kernel<<<(unsigned)((n + per - 1) / per), kWave * s.waves * per, 0, stream>>>(
          static_cast<const T*>(a.x) + at, static_cast<const T*>(a.residual) + at, post, gate, per_gate, r, weight, n,
          a.H, a.eps, a.alpha, a.h ? static_cast<T*>(a.h) + at : nullptr, a.y ? static_cast<T*>(a.y) + at : nullptr,
          a.rstd_x ? a.rstd_x + r : nullptr, a.rstd_h ? a.rstd_h + r : nullptr, s.waves);
    }
    return true;
  });
  return ok && hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

template <typename T>
taot_status backward(const BlockNormGradArgs& a, void* ws, hipStream_t stream) {
  if (a.rows == 0) {
    if (a.dweight) zero_kernel<<<64, 256, 0, stream>>>(a.dweight, a.H);
    if (a.dpost) zero_kernel<<<64, 256, 0, stream>>>(a.dpost, a.H);
    if (a.dgate) zero_kernel<<<256, 256, 0, stream>>>(a.dgate, a.gates * a.H);
    return hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
  }
  const Shape s = shape_of(a.H);
  const int per = s.waves == 1 ? kRowsOfBlock : 1;
  const Vector post{a.post, a.weight_f32}, gate{a.gate, a.gate_f32}, weight{a.weight, a.weight_f32};
  const int64_t gates = a.gate ? a.gates : 1;
  const Split sp = split_of(a.rows, a.H, gates);
  const Partial p = carve(ws, a.rows, a.H, gates);
  const bool sums = a.dpost || (a.dgate && !sp.many);
  with_far(2 * a.rows * a.H * (int64_t)sizeof(T), [&](auto far) {
    const T *dy = static_cast<const T*>(a.dy), *dh = static_cast<const T*>(a.dh), *x = static_cast<const T*>(a.x),
            *h = static_cast<const T*>(a.h);
    T *dx = static_cast<T*>(a.dx), *dr = static_cast<T*>(a.dresidual);
    float *part_w = a.dweight ? p.w : nullptr, *part_s = sums ? p.s : nullptr;
    if (s.cpl == 1 && a.H >= 8) {
      const bool whole = a.H % 8 == 0;
      auto* kernel = sp.many ? whole ? block_norm_backward_kernel<T, far.value, true, kWholeRows>
                                     : block_norm_backward_kernel<T, far.value, true, kOddRows>
                     : whole ? block_norm_backward_kernel<T, far.value, false, kWholeRows>
                             : block_norm_backward_kernel<T, far.value, false, kOddRows>;
      kernel<<<(unsigned)((sp.workers + per - 1) / per), kWave * s.waves * per, 0, stream>>>(
          dy, dh, x, h, a.rstd_x, a.rstd_h, post, gate, sp.share, weight, a.H, a.alpha, dx, dr, a.dgate, part_w, part_s,
          sp.workers, s.waves);
    } else {
      auto* kernel = sp.many ? block_norm_backward_wide_kernel<T, far.value, true>
                             : block_norm_backward_wide_kernel<T, far.value, false>;
      kernel<<<(unsigned)sp.workers, 1024, 0, stream>>>(dy, dh, x, h, a.rstd_x, a.rstd_h, post, gate, sp.share, weight, a.H,
                                                        a.alpha, dx, dr, a.dgate, part_w, part_s, sp.workers);
    }
  });
  const unsigned cols = (unsigned)((a.H + 31) / 32);
  const int64_t sets = !sums ? 0 : sp.many || gates <= kFewGates ? 1 : gates;
  if (sets || a.dweight)
    block_norm_sums_kernel<T><<<dim3(cols, (unsigned)sets + 1), 1024, 0, stream>>>(
        p.w, p.s, sp.workers, sp.many, sets, gates, sp.share.each, post, gate, a.H, a.dweight, a.dpost,
        sp.many ? nullptr : a.dgate, p.S);
  if (a.dpost && !sp.many && gates > kFewGates)
    block_norm_post_kernel<T><<<cols, 1024, 0, stream>>>(p.S, gate, gates, a.H, a.dpost);
  return hipGetLastError() == hipSuccess ? TAOT_OK : TAOT_ERR_LAUNCH;
}

}  // namespace

size_t block_norm_backward_ws(int64_t rows, int32_t H, int64_t gates) {
  return rows > 0 ? carve(nullptr, rows, H, gates).bytes : 0;
}

taot_status launch_block_norm(const BlockNormArgs& a, int32_t dtype, hipStream_t stream) {
  return dtype == TAOT_BF16 ? forward<__bf16>(a, stream) : dtype == TAOT_F16 ? forward<_Float16>(a, stream)
                                                                            : forward<float>(a, stream);
}

taot_status launch_block_norm_backward(const BlockNormGradArgs& a, int32_t dtype, void* ws, hipStream_t stream) {
  return dtype == TAOT_BF16 ? backward<__bf16>(a, ws, stream) : dtype == TAOT_F16 ? backward<_Float16>(a, ws, stream)
                                                                                 : backward<float>(a, ws, stream);
}

}  // namespace taot
