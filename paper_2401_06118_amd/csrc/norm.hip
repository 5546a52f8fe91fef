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
// corrected by the mean of h - mu, which is what its rounding left.
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
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) s += red[turn][w][k];
      v[k] = s;
    }
    turn ^= 1;
  }
}

// mu and r of a row held as pieces h (elements past its end are 0).
template <int TY, int WAVES, int PER>
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
        const float d = e < left ? (float)h[j][e] - mu : 0.f;
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

template <int TY, int WAVES, int PER>
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
    for (int j = 0; j < PER; ++j) h[j] = load_piece<TY>((const T*)a.x + row * a.x_row, (t + j * WAVES * kWave) * N, a.dim);
    if (a.residual != nullptr) {
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const int c = (t + j * WAVES * kWave) * N;
        const V o = load_piece<TY>((const T*)a.residual + row * a.residual_row, c, a.dim);
#pragma unroll
        for (int e = 0; e < N; ++e) h[j][e] = (T)((float)h[j][e] + (float)o[e]);
        if (a.sum != nullptr) store_piece<TY>((T*)a.sum + row * a.sum_row, c, a.dim, h[j]);
      }
    }
    float mu, r;
    row_stats<TY, WAVES, PER>(h, t, a.dim, a.rms, a.eps, red, turn, mu, r);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int c = (t + j * WAVES * kWave) * N;
      float y[N];
#pragma unroll
      for (int e = 0; e < N; ++e) y[e] = ((float)h[j][e] - mu) * r;
      if (a.weight != nullptr) {
        const V w = load_piece<TY>(a.weight, c, a.dim);
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] *= (float)w[e];
      }
      if (a.bias != nullptr) {
        const V b = load_piece<TY>(a.bias, c, a.dim);
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] += (float)b[e];
      }
      V o;
#pragma unroll
      for (int e = 0; e < N; ++e) o[e] = (T)y[e];
      store_piece<TY>((T*)a.out + row * a.out_row, c, a.dim, o);
    }
  }
}

// Gradients: a slot (the waves of one row) takes every gridDim-th row and adds up the
// weight's and the bias's gradients of its columns, which go to `parts`.
template <int TY, int WAVES, int PER>
__global__ void __launch_bounds__(kNormThreads<WAVES>) k_norm_grad(NormGradArgs a) {
  typedef typename Elem<TY>::T T;
  typedef typename Elem<TY>::V V;
  constexpr int N = kPiece<TY>, kRows = WAVES == 1 ? 4 : 1;
  __shared__ float red[2][16][2];
  const int t = WAVES == 1 ? threadIdx.x % kWave : threadIdx.x;
  const int slot = blockIdx.x * kRows + (WAVES == 1 ? threadIdx.x / kWave : 0), slots = gridDim.x * kRows;
  int turn = 0;
  float dw[PER][N], db[PER][N];
#pragma unroll
  for (int j = 0; j < PER; ++j)
#pragma unroll
    for (int e = 0; e < N; ++e) dw[j][e] = db[j][e] = 0.f;
  for (int64_t row = slot; row < a.rows; row += slots) {
    V h[PER], dy[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int c = (t + j * WAVES * kWave) * N;
      h[j] = load_piece<TY>((const T*)a.x + row * a.x_row, c, a.dim);
      dy[j] = load_piece<TY>((const T*)a.dy + row * a.dy_row, c, a.dim);
    }
    float mu, r;
    row_stats<TY, WAVES, PER>(h, t, a.dim, a.rms, a.eps, red, turn, mu, r);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int c = (t + j * WAVES * kWave) * N;
      V w;
      if (a.weight != nullptr) w = load_piece<TY>(a.weight, c, a.dim);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        // (past the row's end dy is 0)
        const float d = (float)dy[j][e], xh = ((float)h[j][e] - mu) * r, g = a.weight != nullptr ? d * (float)w[e] : d;
        dw[j][e] += d * xh;
        db[j][e] += d;
        s[0] += g * xh;
        s[1] += g;
      }
    }
    row_sums<WAVES>(s, red, turn);
    const float by = s[0] / (float)a.dim, mean = a.rms ? 0.f : s[1] / (float)a.dim;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int c = (t + j * WAVES * kWave) * N;
      V w, o;
      float d[N];
      if (a.weight != nullptr) w = load_piece<TY>(a.weight, c, a.dim);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float xh = ((float)h[j][e] - mu) * r, g = a.weight != nullptr ? (float)dy[j][e] * (float)w[e] : (float)dy[j][e];
        d[e] = r * (g - xh * by - mean);
      }
      if (a.dsum != nullptr) {
        const V v = load_piece<TY>((const T*)a.dsum + row * a.dsum_row, c, a.dim);
#pragma unroll
        for (int e = 0; e < N; ++e) d[e] += (float)v[e];
      }
#pragma unroll
      for (int e = 0; e < N; ++e) o[e] = (T)d[e];
      store_piece<TY>((T*)a.out + row * a.out_row, c, a.dim, o);
    }
  }
  if (a.dweight == nullptr && a.dbias == nullptr) return;
#pragma unroll
  for (int j = 0; j < PER; ++j)
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int c = (t + j * WAVES * kWave) * N + e;
      if (c >= a.dim) continue;
      if (a.dweight != nullptr) a.parts[(int64_t)slot * a.dim + c] = dw[j][e];
      if (a.dbias != nullptr) a.parts[((int64_t)slots + slot) * a.dim + c] = db[j][e];
    }
}

// The slots' parts of a column in a fixed order: a workgroup takes 64 columns, each wave
// every 16th slot.
__global__ void __launch_bounds__(1024) k_norm_grad_sum(NormGradArgs a, int slots) {
  __shared__ float red[16][kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, c = blockIdx.x * kWave + lane;
  float* const out = blockIdx.y == 0 ? a.dweight : a.dbias;
  if (out == nullptr) return;
  const float* const parts = a.parts + (int64_t)blockIdx.y * slots * a.dim;
  float s = 0.f;
  if (c < a.dim) {
#pragma unroll 8
    for (int i = wave; i < slots; i += 16) s += parts[(int64_t)i * a.dim + c];
  }
  red[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || c >= a.dim) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) s += red[w][lane];
  out[c] = s;
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

template <int TY>
hipError_t launch_norm_typed(const NormArgs& a, hipStream_t s) {
  return by_width<TY>(a.dim, [&](auto waves, auto per) {
    constexpr int W = decltype(waves)::value, P = decltype(per)::value;
    const int64_t blocks = W == 1 ? (a.rows + 3) / 4 : a.rows;
    k_norm<TY, W, P><<<(unsigned)min(blocks, (int64_t)1 << 20), kNormThreads<W>, 0, s>>>(a);
    return hipGetLastError();
  });
}

template <int TY>
hipError_t launch_grad_typed(const NormGradArgs& a, hipStream_t s) {
  int slots = 0;
  const hipError_t e = by_width<TY>(a.dim, [&](auto waves, auto per) {
    constexpr int W = decltype(waves)::value, P = decltype(per)::value, kRows = W == 1 ? 4 : 1;
    const int64_t most = norm_grad_slots(a.dim) / kRows, blocks = (a.rows + kRows - 1) / kRows;
    const unsigned grid = (unsigned)min(blocks, most);
    slots = (int)grid * kRows;
    if (grid == 0) return hipSuccess;  // (no rows: the sums are zeros)
    k_norm_grad<TY, W, P><<<grid, kNormThreads<W>, 0, s>>>(a);
    return hipGetLastError();
  });
  if (e != hipSuccess || (a.dweight == nullptr && a.dbias == nullptr)) return e;
  k_norm_grad_sum<<<dim3((unsigned)((a.dim + kWave - 1) / kWave), 2), 1024, 0, s>>>(a, slots);
  return hipGetLastError();
}

}  // namespace

int norm_grad_slots(int32_t dim) { return dim <= 1024 ? 4 * num_cus() : 2 * num_cus(); }

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
