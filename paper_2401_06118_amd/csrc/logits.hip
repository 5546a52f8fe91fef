// Penalties for repeated tokens, biases and grammar masks on logits, in one pass:
//
//   l = l > 0 ? l / r : l r        for tokens of the prompt or the output
//   l = l - f count - p            for tokens of the output, count times in it
//   l = l + the token's biases
//   l = -inf                       where the mask's bit is not set
//
// in fp32, rounded once.  Bound: memory; the logits are read and written once.  A
// workgroup owns a slice of a row's vocabulary and keeps a 32-bit word per token
// of it in LDS: bit 31 for a token of the prompt, bits 20..30 the first of the
// row's biases that is the token's (plus one), bits 0..19 its count in the output.  The
// words are integers, so the order of the atomics does not matter.  The slice's
// logits are loaded into registers before the row's history is walked, which hides
// the one under the other.  Every workgroup of a row walks the whole history
// (4 bytes a token, from the L2 after the first).  A slice is every 2^n-th block of
// 64 tokens, not a range: frequent tokens have neighbouring numbers, and their
// atomics would all be one workgroup's.
#include "logits.h"

#include "common.h"
#include "launch.h"
#include "lds_sync.h"
#include "rope.h"

namespace aqlm {

namespace {

constexpr uint32_t kPrompt = 0x80000000u, kCount = 0xFFFFFu;
constexpr int kBiasShift = 20;
constexpr int kThreads = 512;

template <int TY>
struct Logit;
template <>
struct Logit<kF16> {
  typedef _Float16 T;
};
template <>
struct Logit<kBf16> {
  typedef __bf16 T;
};
template <>
struct Logit<kF32> {
  typedef float T;
};

// PER logits a thread, in vectors of 4 (ALIGNED: the rows allow it).
template <int TY, int PER, bool ALIGNED>
__global__ void __launch_bounds__(kThreads) k_logits(LogitsArgs a) {
  typedef typename Logit<TY>::T T;
  typedef T V4 __attribute__((ext_vector_type(4)));
  constexpr int kSlice = kThreads * PER;
  extern __shared__ __align__(16) uint32_t lds[];
  uint32_t* const word = lds;                    // [kSlice]
  float* const bias = (float*)(lds + kSlice);    // [biases]
  int32_t* const ids = (int32_t*)(bias + a.biases);
  int32_t* const twice = ids + a.biases;         // a token has several biases
  const int tid = threadIdx.x, row = blockIdx.y;
  const int turn = blockIdx.x, lg = a.slices_log2;
  // place l of the slice holds token token_at(l)
  auto token_at = [&](int l) { return ((((l >> 6) << lg) + turn) << 6) + (l & 63); };
  // place of a token, or kSlice and more (ids outside the vocabulary too)
  auto place_of = [&](int id) -> uint32_t {
    const uint32_t block = (uint32_t)id >> 6;
    if ((uint32_t)id >= (uint32_t)a.vocab || (int)(block & ((1u << lg) - 1)) != turn) return ~0u;
    return ((block >> lg) << 6) + (id & 63);
  };
  const T* const in = (const T*)a.in + row * a.in_row;
  T* const out = (T*)a.out + row * a.out_row;

  V4 x[PER / 4];
#pragma unroll
  for (int j = 0; j < PER / 4; ++j) {
    const int v = token_at((j * kThreads + tid) * 4);
    if (ALIGNED && v + 4 <= a.vocab) {
      x[j] = *(const V4*)(in + v);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[j][e] = v + e < a.vocab ? in[v + e] : (T)0.f;
    }
  }
#pragma unroll
  for (int j = 0; j < PER / 4; ++j) *(u32x4_t*)(word + (j * kThreads + tid) * 4) = u32x4_t{0, 0, 0, 0};
  if (tid == 0) *twice = 0;
  lds_barrier();

  if (a.biases > 0) {
    for (int i = tid; i < a.biases; i += kThreads) {
      const uint32_t at = place_of(a.bias_ids[row * a.bias_row + i]);
      const bool here = at < (uint32_t)kSlice;
      ids[i] = here ? (int)at : -1;
      bias[i] = here ? a.bias_values[row * a.bias_row + i] : 0.f;
      if (here) {  // the first bias of a token has the largest number here
        const uint32_t old = atomicMax(&word[at], (uint32_t)(a.biases - i) << kBiasShift);
        if (old != 0) *twice = 1;
      }
    }
    lds_barrier();
    if (*twice) {  // the first one takes the sum, in the order of the list
      for (int i = tid; i < a.biases; i += kThreads) {
        const int at = ids[i];
        if (at < 0 || (word[at] & ~kPrompt) >> kBiasShift != (uint32_t)(a.biases - i)) continue;
        float t = bias[i];
        for (int j = i + 1; j < a.biases; ++j)
          if (ids[j] == at) t += bias[j];
        bias[i] = t;  // (read by this thread only: later ones are not first)
      }
    }
  }
  if (a.tokens != nullptr) {
    const int n = min(max(a.token_lens[row], 0), a.history);
    const int p = a.prompt_lens != nullptr ? min(max(a.prompt_lens[row], 0), n) : 0;
    const int32_t* t = a.tokens + row * a.token_row;
    constexpr int kBatch = 8;  // loads in flight
    for (int i0 = tid; i0 < n; i0 += kBatch * kThreads) {
      int id[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) id[j] = i0 + j * kThreads < n ? t[i0 + j * kThreads] : -1;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const uint32_t at = place_of(id[j]);
        if (at < (uint32_t)kSlice) {
          if (i0 + j * kThreads < p) atomicOr(&word[at], kPrompt);
          else atomicAdd(&word[at], 1u);
        }
      }
    }
  }
  lds_barrier();

  const float rep = a.repetition != nullptr ? a.repetition[row] : 1.f;
  const float freq = a.frequency != nullptr ? a.frequency[row] : 0.f;
  const float pres = a.presence != nullptr ? a.presence[row] : 0.f;
#pragma unroll
  for (int j = 0; j < PER / 4; ++j) {
    const int l = (j * kThreads + tid) * 4, v = token_at(l);
    if (v >= a.vocab) continue;
    const u32x4_t w = *(const u32x4_t*)(word + l);
    uint32_t allowed = 0xFu;
    if (a.mask != nullptr) allowed = a.mask[row * a.mask_row + v / 32] >> (v % 32);
    V4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float f = (float)x[j][e];
      if (w[e] != 0) {
        const uint32_t count = w[e] & kCount, first = (w[e] & ~kPrompt) >> kBiasShift;
        if (a.repetition != nullptr && ((w[e] & kPrompt) | count) != 0) f = f > 0.f ? f / rep : f * rep;
        if (count != 0) f = f - freq * (float)count - pres;
        if (first != 0) f += bias[a.biases - (int)first];
      }
      y[e] = (T)((allowed >> e) & 1 ? f : -INFINITY);
    }
    if (ALIGNED && v + 4 <= a.vocab) {
      *(V4*)(out + v) = y;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (v + e < a.vocab) out[v + e] = y[e];
    }
  }
}

template <int TY, int PER>
hipError_t launch(LogitsArgs a, bool aligned, hipStream_t s) {
  const size_t lds = (size_t)kThreads * PER * 4 + (size_t)a.biases * 8 + 16;
  a.slices_log2 = 0;
  while ((int64_t)kThreads * PER << a.slices_log2 < a.vocab) ++a.slices_log2;
  const dim3 grid(1u << a.slices_log2, (unsigned)a.rows);
  if (aligned) k_logits<TY, PER, true><<<grid, kThreads, lds, s>>>(a);
  else k_logits<TY, PER, false><<<grid, kThreads, lds, s>>>(a);
  return hipGetLastError();
}

template <int TY>
hipError_t launch_typed(const LogitsArgs& a, hipStream_t s) {
  const uintptr_t v4 = 4 * (uintptr_t)dtype_bytes(TY) - 1;
  const bool aligned = (((uintptr_t)a.in | (uintptr_t)a.out) & v4) == 0 && ((a.in_row | a.out_row) & 3) == 0;
  // slices of 8192 tokens, or of 2048 where those would leave CUs without one
  const int64_t wgs = (int64_t)a.rows * ((a.vocab + 16 * kThreads - 1) / (16 * kThreads));
  return wgs >= num_cus() ? launch<TY, 16>(a, aligned, s) : launch<TY, 4>(a, aligned, s);
}

}  // namespace

hipError_t launch_logits(const LogitsArgs& a, int dtype, hipStream_t s) {
  if (dtype == kF16) return launch_typed<kF16>(a, s);
  if (dtype == kBf16) return launch_typed<kBf16>(a, s);
  return launch_typed<kF32>(a, s);
}

}  // namespace aqlm
