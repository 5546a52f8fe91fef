// A token of each row of logits by temperature, top-k, top-p and min-p from a given uniform
// number u.  With the row's tokens in the order of falling logits, equal ones by
// number, and weights w = exp((l - max) / T):
//
//   top-k   the first k of them
//   top-p   of these, the ones with less than p times their mass before them
//   min-p   the ones with l - max >= T log(min_p)
//   token   the first, in the order of numbers, at which the kept mass exceeds u times it
//
// Every kept set is a beginning of that order, so it is found as its last member, without
// sorting.  Weights are whole multiples of 2^-44, computed in 64 bits: sums of them are
// exact in any order, so the token does not depend on how the work is divided, and differs
// from that of real numbers only where u is within about 2^-40 of a border.
#include "ends.h"

#include "common.h"
#include "elements.h"
#include "launch.h"
#include "lds_sync.h"

namespace aqlm {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;
constexpr int kBins = 2048;
constexpr int kSegments = 2048;  // of a row: 64 pieces of 16 bytes each
static_assert(kSampleMaxVocab <= kSegments * kWave * 4, "segments");

// The rules of a row and its largest logit.
struct Rules {
  double max, inv, lim;  // weight 2^((l - max) inv); least l - max
  float max_f;
};

// Larger logits have smaller keys; +0 and -0 the same.
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t u = __builtin_bit_cast(uint32_t, l + 0.f);
  return (int32_t)u < 0 ? u : ~u & 0x7FFFFFFFu;
}

// 2^44 exp((l - max) / T), rounded.  2^f for |f| <= 1/2 is the exponential series up to the
// 11th power of f log 2 (the next is below 2^-47).
__device__ __forceinline__ uint64_t weight_of(const Rules& r, float l) {
  if (l == r.max_f) return 1ull << 44;  // (infinite ones too)
  const double y = ((double)l - r.max) * r.inv;
  if (!(y > -46.0)) return 0;
  const double n = __builtin_rint(y), f = (y - n) * 0.69314718055994530942;
  double e = 1.0 / 39916800.0;
  e = e * f + 1.0 / 3628800.0;
  e = e * f + 1.0 / 362880.0;
  e = e * f + 1.0 / 40320.0;
  e = e * f + 1.0 / 5040.0;
  e = e * f + 1.0 / 720.0;
  e = e * f + 1.0 / 120.0;
  e = e * f + 1.0 / 24.0;
  e = e * f + 1.0 / 6.0;
  e = e * f + 0.5;
  e = e * f + 1.0;
  e = e * f + 1.0;
  // (up to 2^44: the last bits of 2^52 + it are its whole part)
  const double whole = __builtin_amdgcn_ldexp(e, (int)n + 44) + 4503599627370496.0;
  return __builtin_bit_cast(uint64_t, whole) & 0xFFFFFFFFFFFFFull;
}

struct Shared {
  uint64_t mass[kBins];  // of bins; then of segments
  uint32_t count[kBins];
  uint64_t wave_mass[kWaves];
  uint32_t wave_count[kWaves];
  uint64_t found_mass;
  uint32_t found_count;
  int32_t found;
  float top[kWaves];
  int32_t bad;
};

// Sums of what the threads before this one have, over the workgroup.
__device__ __forceinline__ void sums_before(Shared& sh, uint64_t& m, uint32_t& c) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  uint64_t im = m;
  uint32_t ic = c;
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) {
    const uint64_t om = __shfl_up((unsigned long long)im, s);
    const uint32_t oc = __shfl_up(ic, s);
    if (lane >= s) {
      im += om;
      ic += oc;
    }
  }
  if (lane == kWave - 1) {
    sh.wave_mass[wave] = im;
    sh.wave_count[wave] = ic;
  }
  __syncthreads();
  m = im - m;
  c = ic - c;
  for (int w = 0; w < wave; ++w) {
    m += sh.wave_mass[w];
    c += sh.wave_count[w];
  }
  __syncthreads();
}

// Calls f(number, logit) for every token of the row that is not masked.
template <int TY, typename F>
__device__ __forceinline__ void each(const void* row, int vocab, F f) {
  constexpr int N = kPiece<TY>;
  for (int i = threadIdx.x * N; i < vocab; i += kThreads * N) {
    const typename Elem<TY>::V v = load_piece<TY>(row, i, vocab);
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (i + e < vocab && (float)v[e] != -INFINITY) f(i + e, (float)v[e]);
  }
}

// The last of the order's tokens up to `most` of them or until they have `mass`, as
// (key, number); with its own and all before it: their mass.  Bits of that pair, 11 at a time.
template <int TY>
__device__ __forceinline__ uint64_t last_kept(Shared& sh, const Rules& r, const void* row, int vocab, bool by_count,
                                              uint32_t most, double mass, uint64_t& kept_mass) {
  const int tid = threadIdx.x;
  uint64_t prefix = 0, above_mass = 0;
  uint32_t above = 0;
  constexpr int kShift[5] = {53, 42, 32, 10, 0}, kDigits[5] = {11, 11, 10, 10, 10};
  for (int d = 0; d < 5; ++d) {
    const int shift = kShift[d], top = shift + kDigits[d] == 20 ? 32 : shift + kDigits[d];
    for (int i = tid; i < kBins; i += kThreads) {
      sh.mass[i] = 0;
      sh.count[i] = 0;
    }
    __syncthreads();
    each<TY>(row, vocab, [&](int i, float l) {
      const uint64_t at = (uint64_t)key_of(l) << 32 | (uint32_t)i;
      if (d != 0 && at >> top != prefix >> top) return;
      const int bin = (int)(at >> shift) & ((1 << kDigits[d]) - 1);
      atomicAdd(&sh.count[bin], 1u);
      atomicAdd((unsigned long long*)&sh.mass[bin], (unsigned long long)weight_of(r, l));
    });
    __syncthreads();
    const uint64_t m0 = sh.mass[2 * tid], m1 = sh.mass[2 * tid + 1];
    const uint32_t c0 = sh.count[2 * tid], c1 = sh.count[2 * tid + 1];
    uint64_t m = m0 + m1;
    uint32_t c = c0 + c1;
    sums_before(sh, m, c);
    m += above_mass;
    c += above;
    // the first bin in which the limit is reached; if it never is, the last one with a token
    if (tid == 0) sh.found = -1;
    __syncthreads();
    auto reached = [&](uint64_t mm, uint32_t cc) { return by_count ? cc >= most : (double)mm >= mass; };
    int mine = -1;
    if (c0 != 0 && !reached(m, c)) mine = 2 * tid;
    if (c1 != 0 && !reached(m + m0, c + c0)) mine = 2 * tid + 1;
    if (mine >= 0) atomicMax(&sh.found, mine);
    __syncthreads();
    if (sh.found >> 1 == tid) {
      const bool second = sh.found & 1;
      sh.found_mass = second ? m + m0 : m;
      sh.found_count = second ? c + c0 : c;
    }
    __syncthreads();
    above_mass = sh.found_mass;
    above = sh.found_count;
    prefix |= (uint64_t)sh.found << shift;
    kept_mass = above_mass + sh.mass[sh.found];
    __syncthreads();
  }
  return prefix;
}

template <int TY>
__global__ void __launch_bounds__(kThreads) k_sample(SampleArgs a) {
  constexpr int N = kPiece<TY>;
  typedef typename Elem<TY>::T T;
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int b = blockIdx.x;
  const T* const row = (const T*)a.logits + b * a.row;
  // largest logit
  float top = -INFINITY;
  bool bad = false;
  each<TY>(row, a.vocab, [&](int, float l) {
    top = fmaxf(top, l);
    bad |= l != l;
  });
  top = wave_max(top);
  if (tid == 0) sh.bad = 0;
  if (lane == 0) sh.top[wave] = top;
  __syncthreads();
  if (bad) sh.bad = 1;
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sh.top[w]);
  if (tid == 0) sh.found = INT32_MAX;
  __syncthreads();
  if (sh.bad || top == -INFINITY) {  // no token can be drawn
    if (tid == 0) {
      a.tokens[b] = -1;
      if (a.logprob != nullptr) a.logprob[b] = NAN;
    }
    return;
  }
  const float t = a.temperature != nullptr ? a.temperature[b] : 1.f;
  if (!(t > 0.f)) {  // the largest, of equal ones the first
    each<TY>(row, a.vocab, [&](int i, float l) {
      if (l == top) atomicMin(&sh.found, i);
    });
    __syncthreads();
    if (tid == 0) {
      a.tokens[b] = sh.found;
      if (a.logprob != nullptr) a.logprob[b] = 0.f;
    }
    return;
  }
  const int k = a.top_k != nullptr ? a.top_k[b] : 0;
  const float p = a.top_p != nullptr ? a.top_p[b] : 1.f, least = a.min_p != nullptr ? a.min_p[b] : 0.f;
  Rules r;
  r.max_f = top;
  r.max = (double)top;
  r.inv = 1.44269504088896340736 / (double)t;
  r.lim = least >= 1.f ? 0.0 : least > 0.f ? (double)t * log((double)least) : -INFINITY;
  uint64_t last = ~0ull, kept = 0;
  if (k > 0 && k < a.vocab) last = last_kept<TY>(sh, r, row, a.vocab, true, (uint32_t)k, 0.0, kept);
  if (p < 1.f) {
    if (last == ~0ull) {
      uint64_t m = 0;
      each<TY>(row, a.vocab, [&](int, float l) { m += weight_of(r, l); });
      m = wave_sum64(m);
      if (lane == 0) sh.wave_mass[wave] = m;
      __syncthreads();
      for (int w = 0; w < kWaves; ++w) kept += sh.wave_mass[w];
      __syncthreads();
    }
    const double mass = fmax((double)p, 0.0) * (double)kept;
    const uint64_t q = last_kept<TY>(sh, r, row, a.vocab, false, 0, fmax(mass, 1.0), kept);
    last = q < last ? q : last;
  }
  auto keeps = [&](int i, float l) {
    return ((uint64_t)key_of(l) << 32 | (uint32_t)i) <= last && (l == top || (double)l - r.max >= r.lim);
  };
  // kept mass of each segment of 64 pieces
  const int segments = (a.vocab + kWave * N - 1) / (kWave * N);
  for (int g = wave; g < segments; g += kWaves) {
    const int i = (g * kWave + lane) * N;
    uint64_t m = 0;
    if (i < a.vocab) {
      const typename Elem<TY>::V v = load_piece<TY>(row, i, a.vocab);
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (i + e < a.vocab && (float)v[e] != -INFINITY && keeps(i + e, (float)v[e])) m += weight_of(r, (float)v[e]);
    }
    m = wave_sum64(m);
    if (lane == 0) sh.mass[g] = m;
  }
  for (int g = segments + tid; g < kSegments; g += kThreads) sh.mass[g] = 0;
  __syncthreads();
  const uint64_t m0 = sh.mass[2 * tid], m1 = sh.mass[2 * tid + 1];
  uint64_t m = m0 + m1;
  uint32_t none = 0;
  sums_before(sh, m, none);
  if (tid == kThreads - 1) sh.found_mass = m + m0 + m1;
  __syncthreads();
  const uint64_t total = sh.found_mass;
  const float u = a.uniform[b];
  // (a whole sum exceeds u total exactly if it exceeds its whole part)
  const double want = (u > 0.f ? (double)u : 0.0) * (double)total;
  const uint64_t target = want < (double)total ? min((uint64_t)want, total - 1) : total - 1;
  __syncthreads();
  if (m <= target && target < m + m0) {
    sh.found = 2 * tid;
    sh.found_mass = m;
  } else if (m + m0 <= target && target < m + m0 + m1) {
    sh.found = 2 * tid + 1;
    sh.found_mass = m + m0;
  }
  __syncthreads();
  if (wave != 0) return;
  // within the segment: a piece a lane
  const int i = (sh.found * kWave + lane) * N;
  uint64_t w[N], own = 0;
  float l[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    w[e] = 0;
    l[e] = 0.f;
  }
  if (i < a.vocab) {
    const typename Elem<TY>::V v = load_piece<TY>(row, i, a.vocab);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      l[e] = (float)v[e];
      if (i + e < a.vocab && l[e] != -INFINITY && keeps(i + e, l[e])) w[e] = weight_of(r, l[e]);
      own += w[e];
    }
  }
  uint64_t upto = own;
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) {
    const uint64_t o = __shfl_up((unsigned long long)upto, s);
    if (lane >= s) upto += o;
  }
  uint64_t before = sh.found_mass + upto - own;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    if (before <= target && target < before + w[e]) {
      a.tokens[b] = i + e;
      if (a.logprob != nullptr)
        a.logprob[b] = (float)((l[e] == top ? 0.0 : ((double)l[e] - r.max) / (double)t) - log((double)total * 0x1p-44));
    }
    before += w[e];
  }
}

template <int TY>
hipError_t launch_typed(const SampleArgs& a, hipStream_t s) {
  k_sample<TY><<<(unsigned)a.rows, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t s) {
  if (dtype == kF16) return launch_typed<kF16>(a, s);
  if (dtype == kBf16) return launch_typed<kBf16>(a, s);
  return launch_typed<kF32>(a, s);
}

}  // namespace aqlm
