// Layer and RMS norm of the residual stream with the sum before it, and the gradients.
//
//   h = x + residual        (rounded to the stream's type; the norm reads what is rounded)
//   mu = mean h             (RMS: 0)
//   r = 1 / sqrt(mean (h - mu)^2 + eps)
//   y = (h - mu) r w + b
//
//   g = dy w,  xh = (h - mu) r
//   dh = r (g - xh mean(g xh) - mean g) + dsum      (RMS: without mean g)
//   dw = sum over rows of dy xh,  db = sum over rows of dy
//
// Bound: memory; every row is read once and kept in registers between its sums.  A row
// is one wave's up to 64 x 2 pieces of 16 bytes, four waves' or sixteen's above.  mu is
// corrected by the mean of h - mu, which is what its rounding left.  4096 x 8192 bf16 with a
// residual 48 us (5.6 TB/s); the gradients of 2048 x 4096 fp16 18 us and 4 for the parts of dw: a
// row's sums wait for its loads, and their stores for them.
#include "ends.h"

#include "common.h"
#include "elements.h"
#include "launch.h"
#include "lds_sync.h"

namespace aqlm {

namespace {

// WAVES of a row; of a workgroup: at least four.
template <int WAVES>
constexpr int kNormThreads = WAVES == 1 ? 4 * kWave : WAVES * kWave;

// Sums of K values over the row's threads, in every thread.  `red`: [2][waves][K] in LDS;
// `turn` alternates, so that one barrier is enough.
template <int WAVES, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float (*red)[16][2], int& turn) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = wave_sum(v[k]);
  if constexpr (WAVES > 1) {
    const int wave = threadIdx.x / kWave;
    if (threadIdx.x % kWave == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) red[turn][wave][k] = v[k];
    }
    lds_barrier();
    const int first = wave / WAVES * WAVES;  // (of this row)
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) s += red[turn][first + w][k];
      v[k] = s;
    }
    turn ^= 1;
  }
}

// mu and r of a row held as pieces h (elements past its end are 0).
template <int TY, int WAVES, int PER, bool WHOLE>
__device__ __forceinline__ void row_stats(const typename Elem<TY>::V (&h)[PER], int t, int dim, bool rms, float eps,
                                          float (*red)[16][2], int& turn, float& mu, float& r) {
  constexpr int N = kPiece<TY>;
  float s[1] = {0.f}, q[2] = {0.f, 0.f};
  mu = 0.f;
  if (!rms) {
#pragma unroll
    for (int j = 0; j < PER; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) s[0] += (float)h[j][e];
    row_sums<WAVES>(s, red, turn);
    mu = s[0] / (float)dim;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int left = dim - (t + j * WAVES * kWave) * N;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float d = (WHOLE ? 0 : e) < left ? (float)h[j][e] - mu : 0.f;
        q[0] += d;
        q[1] += d * d;
      }
    }
    row_sums<WAVES>(q, red, turn);
    const float off = q[0] / (float)dim;
    mu += off;
    r = rsqrtf(fmaxf(q[1] / (float)dim - off * off, 0.f) + eps);
  } else {
#pragma unroll
    for (int j = 0; j < PER; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) s[0] += (float)h[j][e] * (float)h[j][e];
    row_sums<WAVES>(s, red, turn);
    r = rsqrtf(s[0] / (float)dim + eps);
  }
}

// WHOLE: rows are whole pieces.
template <int TY, int WAVES, int PER, bool WHOLE>
__global__ void __launch_bounds__(kNormThreads<WAVES>) k_norm(NormArgs a) {
  typedef typename Elem<TY>::T T;
  typedef typename Elem<TY>::V V;
  constexpr int N = kPiece<TY>, kRows = WAVES == 1 ? 4 : 1;
  __shared__ float red[2][16][2];
  const int t = WAVES == 1 ? threadIdx.x % kWave : threadIdx.x;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * kRows + (WAVES == 1 ? threadIdx.x / kWave : 0); row < a.rows;
       row += (int64_t)gridDim.x * kRows) {
    V h[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) h[j] = load_piece<TY, WHOLE>((const T*)a.x + row * a.x_row, (t + j * WAVES * kWave) * N, a.dim);
    if (a.residual != nullptr) {
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const int c = (t + j * WAVES * kWave) * N;
        const V o = load_piece<TY, WHOLE>((const T*)a.residual + row * a.residual_row, c, a.dim);
#pragma unroll
        for (int e = 0; e < N; ++e) h[j][e] = (T)((float)h[j][e] + (float)o[e]);
        if (a.sum != nullptr) store_piece<TY, false, WHOLE>((T*)a.sum + row * a.sum_row, c, a.dim, h[j]);
      }
    }
    float mu, r;
    row_stats<TY, WAVES, PER, WHOLE>(h, t, a.dim, a.rms, a.eps, red, turn, mu, r);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int c = (t + j * WAVES * kWave) * N;
      float y[N];
#pragma unroll
      for (int e = 0; e < N; ++e) y[e] = ((float)h[j][e] - mu) * r;
      if (a.weight != nullptr) {
        const V w = load_piece<TY, WHOLE>(a.weight, c, a.dim);
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] *= (float)w[e];
      }
      if (a.bias != nullptr) {
        const V b = load_piece<TY, WHOLE>(a.bias, c, a.dim);
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] += (float)b[e];
      }
      V o;
#pragma unroll
      for (int e = 0; e < N; ++e) o[e] = (T)y[e];
      store_piece<TY, false, WHOLE>((T*)a.out + row * a.out_row, c, a.dim, o);
    }
  }
}

// Gradients: a workgroup (of a row, or of four rows of a wave each) takes every gridDim-th set of
// rows and adds up the weight's and the bias's gradients of its columns, which go to `parts`.  The
// next set is loaded while one is worked on, where the registers hold two.  (Four sets at a time, or
// sixteen waves a workgroup, two rows: no faster, 2048 x 4096 fp16.)
template <int WAVES>
constexpr int kGradRows = WAVES == 1 ? 4 : 1;

template <int TY, int WAVES, int PER, bool WHOLE>
__global__ void __launch_bounds__((WAVES * kGradRows<WAVES> * kWave)) k_norm_grad(NormGradArgs a) {
  typedef typename Elem<TY>::T T;
  typedef typename Elem<TY>::V V;
  constexpr int N = kPiece<TY>, kRows = kGradRows<WAVES>, kThreads = WAVES * kRows * kWave;
  constexpr int kRing = PER * N <= 16 ? 2 : 1;  // sets that are loaded or worked on at a time
  __shared__ float red[2][16][2];
  const int t = threadIdx.x % (WAVES * kWave), own = kRows > 1 ? threadIdx.x / kWave : 0;
  static_assert(WAVES == 1 || kRows == 1, "waves of several rows and of a row each");
  const int64_t step = (int64_t)gridDim.x * kRows, slot = (int64_t)blockIdx.x * kRows;
  int turn = 0;
  float dw[PER][N], db[PER][N];
#pragma unroll
  for (int j = 0; j < PER; ++j)
#pragma unroll
    for (int e = 0; e < N; ++e) dw[j][e] = db[j][e] = 0.f;
  struct Row {
    V h[PER], dy[PER], ds[PER];
  };
  auto load = [&](Row& r, int64_t row) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int c = (t + j * WAVES * kWave) * N;
      r.h[j] = load_piece<TY, WHOLE>((const T*)a.x + row * a.x_row, c, a.dim);
      r.dy[j] = load_piece<TY, WHOLE>((const T*)a.dy + row * a.dy_row, c, a.dim);
      if (a.dsum != nullptr) r.ds[j] = load_piece<TY, WHOLE>((const T*)a.dsum + row * a.dsum_row, c, a.dim);
    }
  };
  V w[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j)
    if (a.weight != nullptr) w[j] = load_piece<TY, WHOLE>(a.weight, (t + j * WAVES * kWave) * N, a.dim);
  // (A wave without a row is done: its row's sums need no other wave.  Zeros in the place of a row would add
  // NaN to dw where eps is 0.)
  Row ring[kRing];
#pragma unroll
  for (int d = 0; d < kRing; ++d)
    if (kRing > 1 && slot + own + d * step < a.rows) load(ring[d], slot + own + d * step);
  for (int64_t first = slot + own; first < a.rows; first += kRing * step) {
#pragma unroll
    for (int d = 0; d < kRing; ++d) {
      const int64_t row = first + d * step;
      if (row >= a.rows) break;
      Row& r = ring[d];
      if (kRing == 1) load(r, row);
      float mu, rs;
      row_stats<TY, WAVES, PER, WHOLE>(r.h, t, a.dim, a.rms, a.eps, red, turn, mu, rs);
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < PER; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          // (past the row's end dy is 0)
          const float d = (float)r.dy[j][e], xh = ((float)r.h[j][e] - mu) * rs, g = a.weight != nullptr ? d * (float)w[j][e] : d;
          dw[j][e] += d * xh;
          db[j][e] += d;
          s[0] += g * xh;
          s[1] += g;
        }
      row_sums<WAVES>(s, red, turn);
      const float by = s[0] / (float)a.dim, mean = a.rms ? 0.f : s[1] / (float)a.dim;
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        V o;
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float d = (float)r.dy[j][e], xh = ((float)r.h[j][e] - mu) * rs, g = a.weight != nullptr ? d * (float)w[j][e] : d;
          float y = rs * (g - xh * by - mean);
          if (a.dsum != nullptr) y += (float)r.ds[j][e];
          o[e] = (T)y;
        }
        store_piece<TY, false, WHOLE>((T*)a.out + row * a.out_row, (t + j * WAVES * kWave) * N, a.dim, o);
      }
      if (kRing > 1 && row + kRing * step < a.rows) load(r, row + kRing * step);
    }
  }
  if (a.dweight == nullptr && a.dbias == nullptr) return;
  const int64_t second = (int64_t)gridDim.x * a.dim;  // (the bias's parts)
  if constexpr (kRows > 1) {  // the workgroup's rows together
    constexpr int kWidth = PER * WAVES * kWave * N;
    __shared__ float sums[kRows][kWidth];
#pragma unroll
    for (int which = 0; which < 2; ++which) {
#pragma unroll
      for (int j = 0; j < PER; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) sums[own][(t + j * WAVES * kWave) * N + e] = which == 0 ? dw[j][e] : db[j][e];
      __syncthreads();
      if (which == 0 ? a.dweight != nullptr : a.dbias != nullptr)
        for (int c = threadIdx.x; c < a.dim; c += kThreads) {
          float s = 0.f;
#pragma unroll
          for (int r = 0; r < kRows; ++r) s += sums[r][c];
          a.parts[which * second + (int64_t)blockIdx.x * a.dim + c] = s;
        }
      __syncthreads();
    }
  } else {
    float* const part = a.parts + (int64_t)blockIdx.x * a.dim;
#pragma unroll
    for (int j = 0; j < PER; ++j)
#pragma unroll
      for (int e = 0; e < N; e += 4) {
        const int c = (t + j * WAVES * kWave) * N + e;
        const Elem<kF32>::V w4 = {dw[j][e], dw[j][e + 1], dw[j][e + 2], dw[j][e + 3]};
        const Elem<kF32>::V b4 = {db[j][e], db[j][e + 1], db[j][e + 2], db[j][e + 3]};
        if (c >= a.dim) continue;
        if (a.dweight != nullptr) store_piece<kF32, false, WHOLE>(part, c, a.dim, w4);
        if (a.dbias != nullptr) store_piece<kF32, false, WHOLE>(part + second, c, a.dim, b4);
      }
  }
}

// The workgroups' parts of a column in a fixed order: a workgroup takes 32 columns, every 32 threads a
// 32nd of the parts.
__global__ void __launch_bounds__(1024) k_norm_grad_sum(NormGradArgs a, int parts) {
  __shared__ float red[32][33];
  const int x = threadIdx.x % 32, y = threadIdx.x / 32, c = blockIdx.x * 32 + x;
  float* const out = blockIdx.y == 0 ? a.dweight : a.dbias;
  if (out == nullptr) return;
  const float* const in = a.parts + (int64_t)blockIdx.y * parts * a.dim + min(c, a.dim - 1);
  float s = 0.f;
#pragma unroll 8
  for (int i = y; i < parts; i += 32) s += in[(int64_t)i * a.dim];
  red[y][x] = s;
  __syncthreads();
  // (32 lanes a column)
  s = red[x][y];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) s += __shfl_xor(s, o);
  if (x == 0 && blockIdx.x * 32 + y < a.dim) out[blockIdx.x * 32 + y] = s;
}

// Calls f with the waves of a row and the pieces of a thread.
template <int TY, typename F>
hipError_t by_width(int dim, F f) {
  const int pieces = (dim + kPiece<TY> - 1) / kPiece<TY>;
  if (pieces <= 64) return f(IntC<1>(), IntC<1>());
  if (pieces <= 128) return f(IntC<1>(), IntC<2>());
  if (pieces <= 256) return f(IntC<4>(), IntC<1>());
  if (pieces <= 512) return f(IntC<4>(), IntC<2>());
  if (pieces <= 1024) return f(IntC<4>(), IntC<4>());
  if constexpr (TY == kF32) {
    if (pieces > 2048) return f(IntC<16>(), IntC<4>());
  }
  return f(IntC<16>(), IntC<2>());
}

// The same for the gradients, which keep two sums of each column.
template <int TY, typename F>
hipError_t by_width_grad(int dim, F f) {
  const int pieces = (dim + kPiece<TY> - 1) / kPiece<TY>;
  if (pieces <= 64) return f(IntC<1>(), IntC<1>());
  if (pieces <= 128) return f(IntC<1>(), IntC<2>());
  if (pieces <= 256) return f(IntC<4>(), IntC<1>());
  if (pieces <= 512) return f(IntC<8>(), IntC<1>());
  if (pieces <= 1024) return f(IntC<8>(), IntC<2>());
  if (pieces <= 1536) return f(IntC<8>(), IntC<3>());
  if constexpr (TY == kF32) {
    if (pieces > 2048) return f(IntC<8>(), IntC<8>());
  }
  return f(IntC<8>(), IntC<4>());
}

template <int TY>
hipError_t launch_norm_typed(const NormArgs& a, hipStream_t s) {
  return by_width<TY>(a.dim, [&](auto waves, auto per) {
    constexpr int W = decltype(waves)::value, P = decltype(per)::value;
    const int64_t blocks = W == 1 ? (a.rows + 3) / 4 : a.rows;
    const unsigned grid = (unsigned)min(blocks, (int64_t)1 << 20);
    if (a.dim % kPiece<TY> == 0) k_norm<TY, W, P, true><<<grid, kNormThreads<W>, 0, s>>>(a);
    else k_norm<TY, W, P, false><<<grid, kNormThreads<W>, 0, s>>>(a);
    return hipGetLastError();
  });
}

template <int TY>
hipError_t launch_grad_typed(const NormGradArgs& a, hipStream_t s) {
  // Workgroups, each with a part of the weight's gradient: one a CU, whose parts cost less (2048 x
  // 4096 fp16 23 us, with two 25; 2048 x 8192 35 and 44), two for many rows (8192 x 4096 60 and 56) or
  // rows that are not whole pieces (4000 x 3001 62 and 46).
  const int most = a.rows < 16 * num_cus() && a.dim % kPiece<TY> == 0 ? num_cus() : norm_grad_parts();
  int parts = 0;
  const hipError_t e = by_width_grad<TY>(a.dim, [&](auto waves, auto per) {
    constexpr int W = decltype(waves)::value, P = decltype(per)::value, kRows = kGradRows<W>;
    constexpr int kThreads = W * kRows * kWave;
    parts = (int)min((a.rows + kRows - 1) / kRows, (int64_t)most);
    if (parts == 0) return hipSuccess;  // (no rows: the sums are zeros)
    if (a.dim % kPiece<TY> == 0) k_norm_grad<TY, W, P, true><<<(unsigned)parts, kThreads, 0, s>>>(a);
    else k_norm_grad<TY, W, P, false><<<(unsigned)parts, kThreads, 0, s>>>(a);
    return hipGetLastError();
  });
  if (e != hipSuccess || (a.dweight == nullptr && a.dbias == nullptr)) return e;
  k_norm_grad_sum<<<dim3((unsigned)((a.dim + 31) / 32), 2), 1024, 0, s>>>(a, parts);
  return hipGetLastError();
}

}  // namespace

int norm_grad_parts() { return 2 * num_cus(); }

hipError_t launch_norm(const NormArgs& a, int dtype, hipStream_t s) {
  if (dtype == kF16) return launch_norm_typed<kF16>(a, s);
  if (dtype == kBf16) return launch_norm_typed<kBf16>(a, s);
  return launch_norm_typed<kF32>(a, s);
}

hipError_t launch_norm_grad(const NormGradArgs& a, int dtype, hipStream_t s) {
  if (dtype == kF16) return launch_grad_typed<kF16>(a, s);
  if (dtype == kBf16) return launch_grad_typed<kBf16>(a, s);
  return launch_grad_typed<kF32>(a, s);
}

}  // namespace aqlm
