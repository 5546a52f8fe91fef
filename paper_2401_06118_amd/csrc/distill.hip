// The loss of a student's logits against the largest logits of a teacher, and its gradient.
// With q = softmax(z / tau) over the vocabulary and p over a token's listed ids:
//
//   p_k = softmax over the list of t_k / tau                      (without teacher_lse)
//   p_k = exp(t_k / tau - lse), p_r = max(0, 1 - sum p)           (with it; p_r = 0 where
//                                                                  every id is listed)
//   loss = sum_k p_k log(p_k / q_k) + p_r log(p_r / q_r),   q_r = sum of q outside the list
//   dloss/dz_j = (q_j P - p_j) / tau                              in the list, P = sum p + p_r
//              = (q_j / q_r) (q_r P - p_r) / tau                  outside it
//
// The sum outside the list is taken without the listed ids (a bit per id in LDS), so that q_r
// is no difference; the list's terms are computed in 64 bits, as the loss is a
// difference of larger ones.  Bound: memory; logits are read once and the gradient is
// written once.
#include "ends.h"

#include "common.h"
#include "elements.h"
#include "launch.h"
#include "lds_sync.h"

namespace aqlm {

namespace {

constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ double teacher_at(const DistillArgs& a, int64_t row, int k) {
  const int64_t i = row * a.teacher_row + k;
  if (a.teacher_dtype == kF16) return (double)(float)((const _Float16*)a.teacher)[i];
  if (a.teacher_dtype == kBf16) return (double)(float)((const __bf16*)a.teacher)[i];
  return (double)((const float*)a.teacher)[i];
}

// NV: pieces of the row that a thread keeps in registers (0: the row is read twice).  A
// row's last piece ends at its end and may begin inside the one before: what both hold
// counts for the first and is written alike by both.
template <int TY, int kThreads, int NV>
__global__ void __launch_bounds__(kThreads, 4) k_distill(DistillArgs a) {
  constexpr int kWaves = kThreads / kWave;
  typedef typename Elem<TY>::T T;
  typedef typename Elem<TY>::V V;
  constexpr int N = kPiece<TY>, kAll = (1 << N) - 1;
  constexpr float kLowest = -3.402823466e38f;
  extern __shared__ __align__(16) uint8_t lds[];
  double* const p_of = (double*)lds;                   // [listed]
  int32_t* const id_of = (int32_t*)(p_of + a.listed);  // [listed], -1: no entry
  float* const z_of = (float*)(id_of + a.listed);      // [listed]
  uint32_t* const bits = (uint32_t*)(z_of + a.listed);  // a bit per id: listed, or past the vocabulary
  __shared__ double red[2][kWaves][5];
  __shared__ int twice;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int64_t row = blockIdx.x;
  const T* const in = (const T*)a.logits + row * a.logits_row;
  T* const out = a.grad != nullptr ? (T*)a.grad + row * a.grad_row : nullptr;
  const int pieces = (a.vocab + N - 1) / N;
  auto place = [&](int i) { return NV > 0 ? min(i * N, a.vocab - N) : i * N; };
  const float weight = a.weights != nullptr ? a.weights[row] : 1.f;
  if (weight == 0.f) {  // a token that does not count: its logits are not looked at
    if (tid == 0) a.loss[row] = 0.f;
    V zero;
#pragma unroll
    for (int e = 0; e < N; ++e) zero[e] = (T)0.f;
    if (out != nullptr)
      for (int i = tid; i < pieces; i += kThreads) store_piece<TY>(out, place(i), a.vocab, zero);
    return;
  }
  V x[NV > 0 ? NV : 1];
  if constexpr (NV > 0) {
#pragma unroll
    for (int j = 0; j < NV; ++j) x[j] = *(const V*)(in + place(tid + j * kThreads));
  }
  const int words = (a.vocab + 31) / 32;
  for (int i = tid; i < words; i += kThreads) bits[i] = i == words - 1 && (a.vocab & 31) != 0 ? ~0u << (a.vocab & 31) : 0u;
  if (tid == 0) twice = 0;
  lds_barrier();
  const float c = kLog2e / a.tau;
  const double inv = 1.0 / (double)a.tau;
  double top = -INFINITY, zmax = -INFINITY;
  for (int k = tid; k < a.listed; k += kThreads) {
    const int id = a.ids[row * a.ids_row + k];
    const bool held = (uint32_t)id < (uint32_t)a.vocab;
    id_of[k] = held ? id : -1;
    if (!held) continue;
    const float z = (float)in[id];
    const double t = teacher_at(a, row, k) * inv;
    z_of[k] = z;
    p_of[k] = t;
    top = fmax(top, t);
    zmax = fmax(zmax, (double)z);
    if (atomicOr(&bits[id / 32], 1u << (id % 32)) >> (id % 32) & 1) twice = 1;
  }
  lds_barrier();

  // Outside the list: this thread's maximum and the sum relative to it.
  int skip_last = 0;  // elements of the last piece that do not count
  {
    const int at = place(pieces - 1);
    for (int e = 0; e < N; ++e)
      skip_last |= (int)(at + e < (pieces - 1) * N || at + e >= a.vocab || (bits[(at + e) / 32] >> ((at + e) % 32) & 1)) << e;
  }
  float m = kLowest, s = 0.f;
  auto add = [&](const V& v, int i) {
    int b = (int)(((const uint8_t*)bits)[min(i, pieces - 1) * N / 8] >> (i * N % 8)) & kAll;
    b = i < pieces - 1 ? b : i == pieces - 1 ? skip_last : kAll;
    float f[N], m1 = m;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      f[e] = b >> e & 1 ? -INFINITY : (float)v[e];
      m1 = fmaxf(m1, f[e]);
    }
    s *= __builtin_amdgcn_exp2f((m - m1) * c);
    m = m1;
#pragma unroll
    for (int e = 0; e < N; ++e) s += __builtin_amdgcn_exp2f((f[e] - m) * c);
  };
  if constexpr (NV > 0) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (NV > 4) asm volatile("" : "+v"(x[j]), "+v"(s), "+v"(m));  // (all at once would take too many registers)
      add(x[j], tid + j * kThreads);
    }
  } else {
    for (int i = tid; i < pieces; i += kThreads) add(load_piece<TY>(in, i * N, a.vocab), i);
  }
  // The row's maxima: outside the list, in it, of the teacher.
  double most[3] = {(double)m, zmax, top};
#pragma unroll
  for (int k = 0; k < 3; ++k) {
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) most[k] = fmax(most[k], __shfl_xor(most[k], o));
    if (lane == 0) red[0][wave][k] = most[k];
  }
  lds_barrier();
#pragma unroll 1
  for (int w = 0; w < kWaves; ++w)
#pragma unroll
    for (int k = 0; k < 3; ++k) most[k] = fmax(most[k], red[0][w][k]);
  const double m_rest = most[0], m_all = fmax(most[0], most[1]);
  // The list: teacher's mass, sum of p (log p' - z / tau), student's mass; the rest's sum; how
  // many ids are listed.
  // With lse log p' is log p, without it p and log p' are relative to the largest.
  const double lse = a.teacher_lse != nullptr ? (double)a.teacher_lse[row] : most[2] == -INFINITY ? 0.0 : most[2];
  const bool dup = twice != 0;
  double sum[5] = {0.0, 0.0, 0.0, (double)s * exp(((double)m - m_rest) * inv), 0.0};
  for (int k = tid; k < a.listed; k += kThreads) {
    const int id = id_of[k];
    if (id < 0) continue;
    const double lp = p_of[k] - lse, p = exp(lp), z = ((double)z_of[k] - m_all) * inv;
    p_of[k] = p;
    sum[0] += p;
    if (p != 0.0) sum[1] += p * (lp - z);
    bool firstly = true;
    if (dup)
      for (int i = 0; i < k; ++i) firstly = firstly && id_of[i] != id;
    if (firstly) {
      sum[2] += exp(z);
      sum[4] += 1.0;
    }
  }
#pragma unroll
  for (int k = 0; k < 5; ++k) {
    sum[k] = wave_sum64(sum[k]);
    if (lane == 0) red[1][wave][k] = sum[k];
    sum[k] = 0.0;
  }
  lds_barrier();  // (p_of too)
#pragma unroll 1
  for (int w = 0; w < kWaves; ++w)
#pragma unroll
    for (int k = 0; k < 5; ++k) sum[k] += red[1][w][k];
  const double s_rest = sum[3], shift = exp((m_rest - m_all) * inv);
  const double s_all = sum[2] + (s_rest != 0.0 ? s_rest * shift : 0.0), log_all = log(s_all);
  double p_scale = 1.0, mass = sum[0], c_rest = 1.0, loss;
  if (a.teacher_lse != nullptr) {
    const double p_rest = sum[4] == (double)a.vocab ? 0.0 : sum[0] == sum[0] ? fmax(1.0 - sum[0], 0.0) : sum[0];
    const double q_rest = s_rest != 0.0 ? s_rest * shift / s_all : 0.0;
    mass = sum[0] + p_rest;
    loss = sum[1] + sum[0] * log_all;
    if (p_rest != 0.0) loss += p_rest * log(p_rest / q_rest);
    c_rest = q_rest * mass - p_rest;
  } else if (sum[0] != 0.0) {
    p_scale = 1.0 / sum[0];
    mass = 1.0;
    loss = sum[1] * p_scale - log(sum[0]) + log_all;
    c_rest = s_rest * shift / s_all;
  } else {  // nothing is listed
    loss = c_rest = 0.0;
  }
  if (tid == 0) a.loss[row] = (float)loss;
  if (out == nullptr) return;
  const double scale = (double)weight * inv;
  const float by = s_rest != 0.0 ? (float)(c_rest / s_rest * scale) : 0.f, m0 = (float)m_rest;
  auto write = [&](const V& v, int i) {
    V g;
#pragma unroll
    for (int e = 0; e < N; ++e) g[e] = (T)(__builtin_amdgcn_exp2f(((float)v[e] - m0) * c) * by);
    if constexpr (NV > 0) *(V*)(out + place(i)) = g;
    else store_piece<TY>(out, i * N, a.vocab, g);
  };
  if constexpr (NV > 0) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      asm volatile("" : "+v"(x[j]));  // (otherwise the converted elements are kept, which spills)
      if (tid + j * kThreads < pieces) write(x[j], tid + j * kThreads);
    }
  } else {
    for (int i = tid; i < pieces; i += kThreads) write(load_piece<TY>(in, i * N, a.vocab), i);
  }
  __syncthreads();  // the listed ids' gradients go over what was written there
  for (int k = tid; k < a.listed; k += kThreads) {
    const int id = id_of[k];
    if (id < 0) continue;
    double p = p_of[k];
    if (dup) {  // one that is listed several times: their sum
      p = 0.0;
      for (int i = 0; i < a.listed; ++i) p += id_of[i] == id ? p_of[i] : 0.0;
    }
    out[id] = (T)(float)((exp(((double)z_of[k] - m_all) * inv) / s_all * mass - p * p_scale) * scale);
  }
}

template <int TY, int kThreads, int NV>
hipError_t launch(const DistillArgs& a, hipStream_t s) {
  const int lds = a.listed * 16 + (a.vocab + 31) / 32 * 4;
  const hipError_t e = allow_dynamic_lds((const void*)k_distill<TY, kThreads, NV>, lds);
  if (e != hipSuccess) return e;
  k_distill<TY, kThreads, NV><<<(unsigned)a.rows, kThreads, lds, s>>>(a);
  return hipGetLastError();
}

template <int TY>
hipError_t launch_typed(const DistillArgs& a, hipStream_t s) {
  if (a.vocab < kPiece<TY>) return launch<TY, 256, 0>(a, s);
  const int pieces = (a.vocab + kPiece<TY> - 1) / kPiece<TY>;
  if (pieces <= 256) return launch<TY, 256, 1>(a, s);
  if (pieces <= 4 * 256) return launch<TY, 256, 4>(a, s);
  if (pieces <= 16 * 256) return launch<TY, 256, 16>(a, s);
  if (pieces <= 16 * 512) return launch<TY, 512, 16>(a, s);
  if (pieces <= 16 * 1024) return launch<TY, 1024, 16>(a, s);
  return launch<TY, 1024, 0>(a, s);
}

}  // namespace

hipError_t launch_distill(const DistillArgs& a, int dtype, hipStream_t s) {
  if (dtype == kF16) return launch_typed<kF16>(a, s);
  if (dtype == kBf16) return launch_typed<kBf16>(a, s);
  return launch_typed<kF32>(a, s);
}

}  // namespace aqlm
