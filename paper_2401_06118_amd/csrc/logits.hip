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
// (4 bytes a token, from the L2 after the first).  128 rows of 128256 in fp32 with
// everything (135 MB): 28 us, 4.8 TB/s; without rules 20 (a copy: 26).  A slice is every 2^n-th block of
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

// PER logits a thread, in vectors of 4 (ALIGNED: rows and vocabulary allow it).
// STREAM: outputs that do not fit the L2s go past them.
template <int TY, int PER, bool ALIGNED>
__global__ void __launch_bounds__(kThreads) k_logits(LogitsArgs a) {
  typedef typename Logit<TY>::T T;
  typedef T V4 __attribute__((ext_vector_type(4)));
  constexpr int kSlice = kThreads * PER;
  constexpr bool STREAM = PER > 4;
  extern __shared__ __align__(16) uint32_t lds[];
  uint32_t* const word = lds;                    // [kSlice]
  float* const bias = (float*)(lds + kSlice);    // [biases]
  int32_t* const ids = (int32_t*)(bias + a.biases);
  int32_t* const twice = ids + a.biases;         // a token has several biases
  uint32_t* const marks = (uint32_t*)twice + 1;  // a bit per bias: the first of several
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

  // All loads go out first, those that are needed first before the logits: waiting
  // for one after another took half of the kernel's time.
  constexpr int kBatch = 8;  // of the history, per thread
  const int32_t* const t = a.tokens + row * a.token_row;
  // (No load is under a condition of its own lane, but cut to the arrays' ends: the
  // compiler's waits for the first ones then leave the later ones in flight.)
  int id[kBatch], bias_id = -1;
  float bias_value = 0.f;
  if (a.tokens != nullptr) {
#pragma unroll
    for (int j = 0; j < kBatch; ++j) id[j] = t[min(tid + j * kThreads, a.history - 1)];
  }
  if (a.biases > 0) {
    bias_id = a.bias_ids[row * a.bias_row + min(tid, a.biases - 1)];
    bias_value = a.bias_values[row * a.bias_row + min(tid, a.biases - 1)];
  }
  const int n = a.tokens != nullptr ? min(max(a.token_lens[row], 0), a.history) : 0;
  const int p = a.prompt_lens != nullptr ? min(max(a.prompt_lens[row], 0), n) : 0;
  const float rep = a.repetition != nullptr ? a.repetition[row] : 1.f;
  const float freq = a.frequency != nullptr ? a.frequency[row] : 0.f;
  const float pres = a.presence != nullptr ? a.presence[row] : 0.f;
  uint32_t allowed[PER / 4];
#pragma unroll
  for (int j = 0; j < PER / 4; ++j) allowed[j] = 0xFFFFFFFFu;
  if (a.mask != nullptr) {
#pragma unroll
    for (int j = 0; j < PER / 4; ++j)
      allowed[j] = a.mask[row * a.mask_row + min(token_at((j * kThreads + tid) * 4), a.vocab - 1) / 32];
  }
  V4 x[PER / 4];
#pragma unroll
  for (int j = 0; j < PER / 4; ++j) {
    const int v = token_at((j * kThreads + tid) * 4);
    if constexpr (ALIGNED) {
      x[j] = *(const V4*)(in + min(v, a.vocab - 4));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[j][e] = in[min(v + e, a.vocab - 1)];
    }
  }
#pragma unroll
  for (int j = 0; j < PER / 4; ++j) *(u32x4_t*)(word + (j * kThreads + tid) * 4) = u32x4_t{0, 0, 0, 0};
  if (tid == 0) *twice = 0;
  if (tid < (a.biases + 31) / 32) marks[tid] = 0;
  lds_barrier();

  if (a.biases > 0) {
    auto note = [&](int i, int token, float value) {
      const uint32_t at = place_of(token);
      const bool here = at < (uint32_t)kSlice;
      ids[i] = here ? (int)at : -1;
      bias[i] = value;
      if (here) {  // the first bias of a token has the largest number here
        const uint32_t old = atomicMax(&word[at], (uint32_t)(a.biases - i) << kBiasShift);
        if (old != 0) *twice = 1;
      }
    };
    if (tid < a.biases) note(tid, bias_id, bias_value);
    for (int i = tid + kThreads; i < a.biases; i += kThreads)
      note(i, a.bias_ids[row * a.bias_row + i], a.bias_values[row * a.bias_row + i]);
    lds_barrier();
    if (*twice) {
      // The first bias of such a token takes the sum, in the order of the list: marked
      // by the others, then a wave for each, 64 entries of the list at a time.
      for (int i = tid; i < a.biases; i += kThreads) {
        if (ids[i] < 0) continue;
        const int first = a.biases - (int)((word[ids[i]] & ~kPrompt) >> kBiasShift);
        if (first != i) atomicOr(&marks[first / 32], 1u << (first % 32));
      }
      lds_barrier();
      const int lane = tid % kWave;
      for (int m = tid / kWave; m < (a.biases + 31) / 32; m += kThreads / kWave) {
        for (uint32_t left = marks[m]; left != 0; left &= left - 1) {
          const int i = m * 32 + __builtin_ctz(left), at = ids[i];
          float sum = bias[i];
          for (int j = i + 1; j < a.biases; j += kWave)
            for (uint64_t same = __ballot(j + lane < a.biases && ids[min(j + lane, a.biases - 1)] == at); same != 0;
                 same &= same - 1)
              sum += bias[j + __builtin_ctzll(same)];
          if (lane == 0) bias[i] = sum;  // (only the first ones' are read from here on)
        }
      }
    }
  }
  auto count = [&](int i, int token) {
    const uint32_t at = place_of(token);
    if (i < n && at < (uint32_t)kSlice) {
      if (i < p) atomicOr(&word[at], kPrompt);
      else atomicAdd(&word[at], 1u);
    }
  };
#pragma unroll
  for (int j = 0; j < kBatch; ++j)
    if (a.tokens != nullptr) count(tid + j * kThreads, id[j]);
  // (the rest in a loop of its own: there a load's wait is one for the logits too)
  for (int i0 = tid + kBatch * kThreads; i0 < n; i0 += kBatch * kThreads) {
#pragma unroll
    for (int j = 0; j < kBatch; ++j) id[j] = i0 + j * kThreads < n ? t[i0 + j * kThreads] : -1;
#pragma unroll
    for (int j = 0; j < kBatch; ++j) count(i0 + j * kThreads, id[j]);
  }
  lds_barrier();

#pragma unroll
  for (int j = 0; j < PER / 4; ++j) {
    const int l = (j * kThreads + tid) * 4, v = token_at(l);
    if (v >= a.vocab) continue;
    const u32x4_t w = *(const u32x4_t*)(word + l);
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
      y[e] = (T)((allowed[j] >> (v % 32 + e)) & 1 ? f : -INFINITY);
    }
    if constexpr (ALIGNED) {
      if constexpr (STREAM) __builtin_nontemporal_store(y, (V4*)(out + v));
      else *(V4*)(out + v) = y;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (v + e < a.vocab) out[v + e] = y[e];
    }
  }
}

template <int TY, int PER>
hipError_t launch(LogitsArgs a, bool aligned, hipStream_t s) {
  const size_t lds = (size_t)kThreads * PER * 4 + (size_t)a.biases * 8 + (size_t)((a.biases + 31) / 32) * 4 + 16;
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
  const bool aligned = (((uintptr_t)a.in | (uintptr_t)a.out) & v4) == 0 && ((a.in_row | a.out_row | a.vocab) & 3) == 0;
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
