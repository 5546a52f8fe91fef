// Rows of fp16, bf16 or fp32 elements in pieces of 16 bytes at any element's address
// (the hardware takes global loads and stores at any address), in 32 bits between.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "rope.h"

namespace aqlm {

template <int TY>
struct Elem;
template <>
struct Elem<kF16> {
  typedef _Float16 T;
  typedef T V __attribute__((ext_vector_type(8), aligned(2)));
};
template <>
struct Elem<kBf16> {
  typedef __bf16 T;
  typedef T V __attribute__((ext_vector_type(8), aligned(2)));
};
template <>
struct Elem<kF32> {
  typedef float T;
  typedef T V __attribute__((ext_vector_type(4), aligned(4)));
};
// Elements of a piece.
template <int TY>
constexpr int kPiece = TY == kF32 ? 4 : 8;

// Elements [at, at + piece) of a row of n; those past its end are 0.  WHOLE: n is whole pieces.
template <int TY, bool WHOLE = false>
__device__ __forceinline__ typename Elem<TY>::V load_piece(const void* row, int at, int n) {
  typedef typename Elem<TY>::T T;
  const T* const p = (const T*)row + at;
  if (at + kPiece<TY> <= n) return *(const typename Elem<TY>::V*)p;
  typename Elem<TY>::V v;
#pragma unroll
  for (int e = 0; e < kPiece<TY>; ++e) v[e] = !WHOLE && at + e < n ? p[e] : (T)0.f;
  return v;
}

// NT: past the L2s (results that nothing reads soon, more than they hold).
template <int TY, bool NT = false, bool WHOLE = false>
__device__ __forceinline__ void store_piece(void* row, int at, int n, const typename Elem<TY>::V& v) {
  typedef typename Elem<TY>::T T;
  T* const p = (T*)row + at;
  if (at + kPiece<TY> <= n) {
    if constexpr (NT) __builtin_nontemporal_store(v, (typename Elem<TY>::V*)p);
    else *(typename Elem<TY>::V*)p = v;
    return;
  }
  if constexpr (!WHOLE) {
#pragma unroll
    for (int e = 0; e < kPiece<TY>; ++e)
      if (at + e < n) p[e] = v[e];
  }
}

// Sum of v over the 64 lanes in a fixed order, in every lane, for 64-bit types.
__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) v += __shfl_xor(v, s);
  return v;
}
__device__ __forceinline__ uint64_t wave_sum64(uint64_t v) {
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) v += __shfl_xor((unsigned long long)v, s);
  return v;
}
// The largest over the lanes, in every lane (rows of 16 by DPP, as wave_sum).
__device__ __forceinline__ float wave_max(float v) {
  auto move = [&](auto c) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), decltype(c)::value, 0xF, 0xF, true));
  };
  v = fmaxf(v, move(IntC<0xB1>()));
  v = fmaxf(v, move(IntC<0x4E>()));
  v = fmaxf(v, move(IntC<0x141>()));
  v = fmaxf(v, move(IntC<0x140>()));
  auto lane = [&](int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l)); };
  return fmaxf(fmaxf(lane(0), lane(16)), fmaxf(lane(32), lane(48)));
}

}  // namespace aqlm
