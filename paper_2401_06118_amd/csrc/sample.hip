// A token of each row of logits by temperature, top-k, top-p and min-p from a given uniform
// number u.  With the row's tokens in the order of falling logits, equal ones by
// number, and weights w = exp((l - max) / T):
//
//   top-k   the first k of them
//   top-p   of these, the ones with less than p times their mass before them
//   min-p   the ones with l - max >= T log(min_p)
//   token   the first, in the order of numbers, at which the kept mass exceeds u times it
//
// Every kept set is a beginning of that order, so only its last member has to be found.
// Weights are whole multiples of 2^-44 of the largest, computed in 64 bits, and added as integers: the
// token does not depend on the order of the atomics.  Each is off by at most 2^-44 of the largest, the mass of
// n tokens by n 2^-44 of it (by about 2^-37 for 128256 whose roundings cancel as chance has it, by up to 2^-27
// for as many alike): the token and the kept set are those of real numbers but where u or p lies so near a border.
// Rows that are cut round the slices' sums once more, and their tokens to finer multiples.
//
// Counts and masses of the tokens by bins of T / 16 (512 of them: what is lower has no mass
// left) show in which bin the last member lies.  The tokens down to it (or, if those are more
// than a list holds, that bin's) are collected and sorted; the kept ones are the first of
// them.  (A top-p of the first k has two last members: the k-th for the mass, then the limit's.)  What the list does not
// hold either is found by eleven bits of logit and number at a time (draw_slowly): thousands of equal logits; logits of
// more than 2^25 temperatures; and, for top-k up to 256, cut rows a slice of which has more tokens than its list (512),
// but fewer than k threads that hold any (the last 1105 of 50257 logits in 16 bits, with top-k 140 and more: a row 86 us,
// with top-k 100 19).
//
// Rows that are not cut are a workgroup's each, which holds them in registers (up to 32768 logits with top-k, 8192
// without: sample_cut).  Longer ones are cut into slices of 8192: one launch makes the slices' maxima, bins (relative to
// their own maximum) and lists of their first tokens, another joins a row's.  Bound: latency of
// one row's phases (a row of 32000 11 us with top-k and top-p), with many rows the 64-bit
// exponentials and the slowest row's join (128 x 128256 fp32 30 us and 30; the logits alone are 13).
#include "ends.h"

#include "common.h"
#include "elements.h"
#include "launch.h"
#include "lds_sync.h"
#include "sample_bins.h"

namespace aqlm {

namespace {

constexpr int kBins = kSampleBins;
constexpr int kList = 2048;      // tokens that are sorted
constexpr int kFew = 256;        // tokens that are compared with one another, without sorting
constexpr int kMostK = 256;      // up to this top-k bins need no masses: the lists hold all that count
constexpr int kDigit = 2048;     // bins of the search by bits
constexpr int kSegments = 2048;  // of a row: 64 pieces of 16 bytes each
constexpr int kSliceThreads = 512, kJoinThreads = 1024, kRowThreads = 512;
constexpr int kPool = 8192;  // tokens of a bin, of which the list gets a part
static_assert(kSampleMaxVocab <= kSegments * kWave * 4, "segments");
static_assert(kSampleMaxVocab <= kSampleSlice * kWave, "a wave has a row's slices");
static_assert(kMostK <= kSampleListed, "a slice lists the first k");

// The rules of a row and its largest logit.
struct Rules {
  double max, inv, lim;  // weight 2^((l - max) inv); least l - max
  double t, p;
  float max_f, c;        // bin floor(l c)
  int k;                 // 0: all
  bool greedy;
  bool top_p, min_p;
};

__device__ __forceinline__ Rules rules_of(const SampleArgs& a, int b) {
  Rules r;
  const float t = a.temperature != nullptr ? a.temperature[b] : 1.f;
  const int k = a.top_k != nullptr ? a.top_k[b] : 0;
  const float p = a.top_p != nullptr ? a.top_p[b] : 1.f, least = a.min_p != nullptr ? a.min_p[b] : 0.f;
  r.greedy = !(t > 0.f);
  r.t = (double)t;
  r.inv = 1.44269504088896340736 / (double)t;
  r.c = 16.f / t;
  r.k = k > 0 && k < a.vocab ? k : 0;
  r.top_p = p < 1.f;
  r.p = (double)fmaxf(p, 0.f);
  r.min_p = least > 0.f;
  r.lim = least >= 1.f ? 0.0 : r.min_p ? r.t * log((double)least) : -INFINITY;
  return r;
}

// Larger logits have smaller keys; +0 and -0 the same.
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t u = __builtin_bit_cast(uint32_t, l + 0.f);
  return (int32_t)u < 0 ? u : ~u & 0x7FFFFFFFu;
}
__device__ __forceinline__ float logit_of(uint32_t key) {
  return __builtin_bit_cast(float, (int32_t)key < 0 ? key : ~key & 0x7FFFFFFFu);
}
__device__ __forceinline__ uint64_t place_of(float l, int i) { return (uint64_t)key_of(l) << 32 | (uint32_t)i; }

// (The largest of a row is below 2^29 in size, or bins are not used: has_bins.)
__device__ __forceinline__ int bin_of(float l, float c) { return (int)floorf(fminf(fmaxf(l * c, -0x1p30f), 0x1p30f)); }
__device__ __forceinline__ int low_bin_of(float l, float c) { return (int)floorf(fmaxf(l * c, -0x1p30f)); }

// 2^44 exp((l - max) / T), rounded; 0 for masked ones.  2^f for |f| <= 1/2 is the exponential
// series up to the 11th power of f log 2 (the next is below 2^-47).  Without branches, so
// that several are computed at a time: one after another is one chain of 64-bit operations.
__device__ __forceinline__ uint64_t weight_of(const Rules& r, float l) {
  const double d = l == r.max_f ? 0.0 : (double)l - r.max;  // (infinite ones too)
  const double y = fmax(d * r.inv, -60.0), n = __builtin_rint(y), f = (y - n) * 0.69314718055994530942;
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

// 2^y for y <= 0.
__device__ __forceinline__ double factor(double y) { return y > -1000.0 ? exp2(y) : 0.0; }

// About as many tokens as can have this mass in a bin whose lower end is `lower`, or more: each has the
// weight there or more (but for its rounding, where that is a few units: whoever lists them counts again).
__device__ __forceinline__ uint32_t most_of(const Rules& r, uint64_t mass, float lower) {
  const float each = (r.max_f * r.c - lower) * (1.44269504f / 16.f) - 44.f;  // -log2 of the least weight
  return mass == 0 ? 0 : (uint32_t)fminf((float)mass * __builtin_amdgcn_exp2f(each) * 1.01f, 1e9f) + 1;
}

struct Shared {
  union {
    struct {
      uint64_t mass[kDigit];  // of bins; then of segments
      uint32_t count[kDigit];
    } search;
    struct {
      uint64_t list[kList];
      uint64_t mass[kBins];  // by bin, the largest logits' first
      uint32_t count[kBins];
    };
  };
  uint64_t wave_mass[16];
  uint32_t wave_count[16];
  uint64_t parts[2 * kWave];
  uint64_t weight[kFew];
  uint64_t few[2][kFew / kWave];
  double factor[kWave];   // of a slice's masses
  uint64_t slice[kWave];  // kept mass of a slice
  uint64_t found_mass;
  uint32_t found_count, found_in;
  int32_t found, listing;
  float top[16];
};

__device__ __forceinline__ float larger(float a, float b) { return b > a || b != b ? b : a; }  // (NaN stays)
__device__ __forceinline__ float wave_largest(float v) {
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) v = larger(v, __shfl_xor(v, s));
  return v;
}

// Sums of what the threads before this one have, over the workgroup.
template <int THREADS>
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
  lds_barrier();
  m = im - m;
  c = ic - c;
#pragma unroll
  for (int w = 0; w < THREADS / kWave - 1; ++w) {  // (all loads at once)
    const uint64_t om = sh.wave_mass[w];
    const uint32_t oc = sh.wave_count[w];
    m += w < wave ? om : 0;
    c += w < wave ? oc : 0;
  }
  lds_barrier();
}

// The sum over the workgroup, in every thread.
template <int THREADS>
__device__ __forceinline__ uint64_t sum_all(Shared& sh, uint64_t m) {
  m = wave_sum64(m);
  if (threadIdx.x % kWave == 0) sh.wave_mass[threadIdx.x / kWave] = m;
  lds_barrier();
  m = 0;
#pragma unroll
  for (int w = 0; w < THREADS / kWave; ++w) m += sh.wave_mass[w];
  lds_barrier();
  return m;
}

__device__ __forceinline__ uint64_t wave_before(uint64_t v) {
  uint64_t incl = v;
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) {
    const uint64_t o = __shfl_up((unsigned long long)incl, s);
    if ((int)(threadIdx.x % kWave) >= s) incl += o;
  }
  return incl - v;
}

// The token is the first at which the kept mass exceeds this.  (A whole sum exceeds u total
// exactly if it exceeds its whole part; u is cut to [0, 1).)
__device__ __forceinline__ uint64_t target_of(float u, uint64_t total) {
  const double want = (u > 0.f ? (double)u : 0.0) * (double)total;
  return want < (double)total ? min((uint64_t)want, total - 1) : total - 1;
}

// One thread: the result.
__device__ __forceinline__ void finish(const SampleArgs& a, int b, const Rules& r, int token, float l, uint64_t total) {
  a.tokens[b] = token;
  if (a.logprob != nullptr)
    a.logprob[b] = (float)((l == r.max_f ? 0.0 : ((double)l - r.max) / r.t) - log((double)total * 0x1p-44));
}

// The sum over the threads of the first n, n <= kFew, in every one of the workgroup.  `turn`: which of two places.
__device__ __forceinline__ uint64_t sum_few(Shared& sh, int turn, uint64_t m, int n) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  if (wave < kFew / kWave) {
    if (wave * kWave < n) m = wave_sum64(m);
    if (lane == 0) sh.few[turn][wave] = wave * kWave < n ? m : 0;
  }
  lds_barrier();
  m = 0;
#pragma unroll
  for (int w = 0; w < kFew / kWave; ++w) m += sh.few[turn][w];
  return m;
}

// Appends to dest, n of them so far in LDS and `cap` at most, the places of those of a wave's K elements a lane that
// hit; all lanes call it.  One atomic a wave.
template <int K, typename H, typename P>
__device__ __forceinline__ void append(int32_t& n, uint64_t* dest, int cap, H hit, P place) {
  uint64_t masks[K];
  int total = 0;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    masks[k] = __ballot(hit(k));
    total += __popcll(masks[k]);
  }
  if (total == 0) return;
  const int lane = threadIdx.x % kWave;
  int at = 0;
  if (lane == 0) at = atomicAdd(&n, total);
  at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if (masks[k] == 0) continue;
    const int to = at + __popcll(masks[k] & ((1ull << lane) - 1));
    if ((masks[k] >> lane & 1) && to < cap) dest[to] = place(k);
    at += __popcll(masks[k]);
  }
}

// The row's tokens with low <= l c < high appended, by all threads.  The numbers first, a lane's own of 32 at a time
// (few hit: as many steps as the most of a lane), then their logits: 9 us instead of the 20
// that a ballot an element takes for 128256 logits with thousands of hits.
template <int TY, int THREADS>
__device__ __forceinline__ void append_row(int32_t& n, uint64_t* dest, int cap, const void* row, int vocab, float c,
                                           float low, float high) {
  constexpr int N = kPiece<TY>, kBatch = 32 / N;
  typedef typename Elem<TY>::T T;
  const int lane = threadIdx.x % kWave;
  // (whole waves: lanes past the end have nothing)
  for (int i0 = 0; i0 < vocab; i0 += kBatch * THREADS * N) {
    typename Elem<TY>::V v[kBatch];
    const int i1 = i0 + threadIdx.x * N;
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int i = i1 + j * THREADS * N;
      if (i + N <= vocab) {
        v[j] = *(const typename Elem<TY>::V*)((const T*)row + i);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[j][e] = i + e < vocab ? ((const T*)row)[i + e] : (T)-INFINITY;
      }
    }
    uint32_t hits = 0;
#pragma unroll
    for (int k = 0; k < 32; ++k) {
      const float f = (float)v[k / N][k % N] * c;
      hits |= f >= low && f < high ? 1u << k : 0;
    }
    if (__ballot(hits != 0) == 0) continue;
    const int own = __popc(hits);
    int incl = own;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
      const int o = __shfl_up(incl, s);
      if (lane >= s) incl += o;
    }
    int at = 0;
    if (lane == kWave - 1) at = atomicAdd(&n, incl);
    at = __builtin_amdgcn_readlane(at, kWave - 1) + incl - own;
    for (; hits != 0; hits &= hits - 1, ++at) {
      const int k = __builtin_ctz(hits);
      if (at < cap) dest[at] = (uint32_t)(i1 + k / N * (THREADS * N) + k % N);
    }
  }
  lds_barrier();
  const int held = min(n, cap);
  for (int t = threadIdx.x; t < held; t += THREADS) {
    const int i = (int)dest[t];
    dest[t] = place_of((float)((const T*)row)[i], i);
  }
}

// Calls f(number, logit) for every token of the row that is not masked.
template <int TY, int THREADS, typename F>
__device__ __forceinline__ void each(const void* row, int vocab, F f) {
  constexpr int N = kPiece<TY>, kBatch = 8;  // loads in flight
  for (int i0 = threadIdx.x * N; i0 < vocab; i0 += kBatch * THREADS * N) {
    typename Elem<TY>::V v[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int i = i0 + j * THREADS * N;
      if (i < vocab) v[j] = load_piece<TY>(row, i, vocab);
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int i = i0 + j * THREADS * N;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        float l = (float)v[j][e];
        asm volatile("" : "+v"(l));  // (one after another: all at once would take too many registers)
        if (i + e < vocab && l != -INFINITY) f(i + e, l);
      }
    }
  }
}

// The place of the last of the order's tokens up to `most` of them (by_count) or until they
// have `mass`; kept_mass: its own and all before it.
template <int TY, int THREADS>
__device__ __forceinline__ uint64_t last_kept(Shared& sh, const Rules& r, const void* row, int vocab, bool by_count, uint32_t most,
                              double mass, uint64_t& kept_mass) {
  constexpr int kEach = kDigit / THREADS;
  const int tid = threadIdx.x;
  uint64_t prefix = 0, above_mass = 0;
  uint32_t above = 0;
  // bits 53..63, 42..52, 32..41 (the logit), 10..19, 0..9 (the number)
#pragma unroll 1
  for (int d = 0; d < 5; ++d) {
    const int shift = d == 0 ? 53 : d == 1 ? 42 : d == 2 ? 32 : d == 3 ? 10 : 0;
    const int top = d == 0 ? 64 : d == 1 ? 53 : d == 2 ? 42 : d == 3 ? 32 : 10;
    const int mask = d < 2 ? 2047 : 1023;
    for (int i = tid; i < kDigit; i += THREADS) {
      sh.search.mass[i] = 0;
      sh.search.count[i] = 0;
    }
    if (tid == 0) sh.found = -1;
    lds_barrier();
    each<TY, THREADS>(row, vocab, [&](int i, float l) {
      const uint64_t at = place_of(l, i);
      if (d != 0 && at >> top != prefix >> top) return;
      const int bin = (int)(at >> shift) & mask;
      atomicAdd(&sh.search.count[bin], 1u);
      atomicAdd((unsigned long long*)&sh.search.mass[bin], (unsigned long long)weight_of(r, l));
    });
    lds_barrier();
    uint64_t m = 0;
    uint32_t c = 0;
    for (int j = 0; j < kEach; ++j) {
      m += sh.search.mass[kEach * tid + j];
      c += sh.search.count[kEach * tid + j];
    }
    sums_before<THREADS>(sh, m, c);
    m += above_mass;
    c += above;
    // the last bin with a token before which the limit is not reached
    int mine = -1;
    uint64_t mm = 0;
    uint32_t cc = 0;
    for (int j = 0; j < kEach; ++j) {
      const uint32_t n = sh.search.count[kEach * tid + j];
      if (n != 0 && !(by_count ? c >= most : (double)m >= mass)) {
        mine = kEach * tid + j;
        mm = m;
        cc = c;
      }
      m += sh.search.mass[kEach * tid + j];
      c += n;
    }
    if (mine >= 0) atomicMax(&sh.found, mine);
    lds_barrier();
    if (mine >= 0 && sh.found == mine) {
      sh.found_mass = mm;
      sh.found_count = cc;
    }
    lds_barrier();
    above_mass = sh.found_mass;
    above = sh.found_count;
    prefix |= (uint64_t)sh.found << shift;
    kept_mass = above_mass + sh.search.mass[sh.found];
    lds_barrier();
  }
  return prefix;
}

// Everything from the row itself, whatever it holds.
template <int TY, int THREADS>
__device__ __forceinline__ void draw_slowly(Shared& sh, const SampleArgs& a, int b, const Rules& r) {
  constexpr int N = kPiece<TY>, kEach = kSegments / THREADS;
  typedef typename Elem<TY>::T T;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const T* const row = (const T*)a.logits + b * a.row;
  uint64_t last = ~0ull, kept = 0;
  lds_barrier();
  if (r.k > 0) last = last_kept<TY, THREADS>(sh, r, row, a.vocab, true, (uint32_t)r.k, 0.0, kept);
  if (r.top_p) {
    if (last == ~0ull) {
      uint64_t m = 0;
      each<TY, THREADS>(row, a.vocab, [&](int, float l) { m += weight_of(r, l); });
      kept = sum_all<THREADS>(sh, m);
    }
    const uint64_t q = last_kept<TY, THREADS>(sh, r, row, a.vocab, false, 0, fmax(r.p * (double)kept, 1.0), kept);
    last = q < last ? q : last;
  }
  auto weight = [&](int i, float l) -> uint64_t {
    return i < a.vocab && l != -INFINITY && place_of(l, i) <= last && (l == r.max_f || (double)l - r.max >= r.lim)
               ? weight_of(r, l) : 0;
  };
  // kept mass of each segment of 64 pieces
  const int segments = (a.vocab + kWave * N - 1) / (kWave * N);
  for (int g = wave; g < segments; g += THREADS / kWave) {
    const int i = (g * kWave + lane) * N;
    uint64_t m = 0;
    if (i < a.vocab) {
      const typename Elem<TY>::V v = load_piece<TY>(row, i, a.vocab);
#pragma unroll
      for (int e = 0; e < N; ++e) m += weight(i + e, (float)v[e]);
    }
    m = wave_sum64(m);
    if (lane == 0) sh.search.mass[g] = m;
  }
  for (int g = segments + tid; g < kSegments; g += THREADS) sh.search.mass[g] = 0;
  lds_barrier();
  uint64_t m = 0;
  uint32_t none = 0;
  for (int j = 0; j < kEach; ++j) m += sh.search.mass[kEach * tid + j];
  const uint64_t mine = m;
  sums_before<THREADS>(sh, m, none);
  if (tid == THREADS - 1) sh.found_mass = m + mine;
  lds_barrier();
  const uint64_t total = sh.found_mass, target = target_of(a.uniform[b], total);
  lds_barrier();
  for (int j = 0; j < kEach; ++j) {
    const uint64_t w = sh.search.mass[kEach * tid + j];
    if (m <= target && target < m + w) {
      sh.found = kEach * tid + j;
      sh.found_mass = m;
    }
    m += w;
  }
  lds_barrier();
  if (wave != 0) return;
  // within the segment: a piece a lane
  const int i = (sh.found * kWave + lane) * N;
  uint64_t w[N], own = 0;
  typename Elem<TY>::V v;
#pragma unroll
  for (int e = 0; e < N; ++e) w[e] = 0;
  if (i < a.vocab) {
    v = load_piece<TY>(row, i, a.vocab);
#pragma unroll
    for (int e = 0; e < N; ++e) own += w[e] = weight(i + e, (float)v[e]);
  }
  uint64_t before = sh.found_mass + wave_before(own);
  int found = -1;
  float found_l = 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    if (before <= target && target < before + w[e]) {
      found = i + e;
      found_l = (float)v[e];
    }
    before += w[e];
  }
  if (found >= 0) finish(a, b, r, found, found_l, total);
}

// What is kept of a row: logits above l, and l itself up to number i.
struct Edge {
  float l;
  int i;
  int bin;
  float high;  // the upper end of l c in the list
  int pooled;
};
enum Outcome { kDrawn, kKnown, kUnknown };

// k: the first k are kept, 0 for all; counted: sh.count is known.
// The edge's bin by one wave, eight bins a lane, from sh.mass and sh.count, and what lies before them:
// sh.found, that bin, sh.found_in, what it has, and the sums before it; sh.listing: the list's fill.
__device__ __forceinline__ void find_edge(Shared& sh, const Rules& r, int k, bool by_count, bool counted, bool whole,
                                          double most, const Bins& bins, uint64_t mass_before,
                                          uint32_t count_before) {
  constexpr int kEach = kBins / kWave;
  const int lane = threadIdx.x;
  uint64_t mass[kEach], m = 0;
  uint32_t count[kEach], c = 0;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int bin = lane * kEach + j;
    mass[j] = by_count ? 0 : sh.mass[bin];
    count[j] = by_count || counted ? sh.count[bin] : most_of(r, mass[j], bins.lower(bin));
    m += mass[j];
    c += count[j];
  }
  mass_before += wave_before(m);
  uint32_t incl = c;
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) {
    const uint32_t o = __shfl_up(incl, s);
    if (lane >= s) incl += o;
  }
  count_before += incl - c;
  int mine = bins.last();  // at most: the first bin in which a rule's limit lies
  if (r.min_p && !whole) {
    // the largest logit in 32 bits that is not above the limit: what lies in higher bins is kept
    const double least = r.max + r.lim;
    float f = (float)least;
    if ((double)f > least) f = logit_of(key_of(f) + 1);
    f = fminf(fmaxf(f * r.c, bins.lower(bins.last())), bins.upper(0));
    mine = min(max(bins.at(f), 0), mine);
  }
  uint64_t bm = mass_before;
  uint32_t bc = count_before;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    bool limit = k > 0 && bc < (uint32_t)k && (uint32_t)k <= bc + count[j];
    if (!by_count && !whole) limit |= r.top_p && mass[j] != 0 && (double)(bm + mass[j]) >= most;
    if (limit) mine = min(mine, lane * kEach + j);
    bm += mass[j];
    bc += count[j];
  }
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) mine = min(mine, __shfl_xor(mine, s));
  if (lane == mine / kEach) {
    uint32_t in = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      if (j < mine % kEach) {
        mass_before += mass[j];
        count_before += count[j];
      }
      if (j == mine % kEach) in = count[j];
    }
    sh.found = mine;
    sh.found_mass = mass_before;
    sh.found_count = count_before;
    sh.found_in = in;
    sh.listing = 0;
  }
}

// The first n of sh.list in order.
template <int THREADS>
__device__ __forceinline__ void sort(Shared& sh, int n) {
  const int tid = threadIdx.x, wave = tid / kWave;
  if (n <= kFew) {  // each to its rank
    const uint64_t own = tid < n ? sh.list[tid] : 0;
    int rank = 0;
    if (wave * kWave < n) {
#pragma unroll 8
      for (int j = 0; j < n; ++j) rank += sh.list[j] < own;
    }
    lds_barrier();
    if (tid < n) sh.list[rank] = own;
    lds_barrier();
    return;
  }
  int size = 2;
  while (size < n) size <<= 1;
  for (int i = n + tid; i < size; i += THREADS) sh.list[i] = ~0ull;
  lds_barrier();
  for (int k = 2; k <= size; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      for (int i = tid; i < size / 2; i += THREADS) {
        const int lo = 2 * i - (i & (j - 1)), hi = lo + j;
        const uint64_t p = sh.list[lo], q = sh.list[hi];
        if ((p > q) == ((lo & k) == 0)) {
          sh.list[lo] = q;
          sh.list[hi] = p;
        }
      }
      lds_barrier();
    }
}

// The mass of the first k, or kNone if more than the list holds are in the k-th's bin; collect as in choose.  (Sorting
// those of one bin: sorting all k to find top-p's limit takes 12 us for 1000, twice.)
constexpr uint64_t kNone = ~0ull;
template <int THREADS, typename F>
__device__ __forceinline__ uint64_t mass_of_first(Shared& sh, const Rules& r, int top_bin, F collect) {
  constexpr int kEach = kList / THREADS;
  const int tid = threadIdx.x;
  const Bins bins{top_bin, false, 0.f};
  if (tid / kWave == 0) find_edge(sh, r, r.k, false, true, true, 0.0, bins, 0, 0);
  lds_barrier();
  const int bin = sh.found;
  const uint32_t rest = (uint32_t)r.k - min(sh.found_count, (uint32_t)r.k);
  const uint64_t before = sh.found_mass;
  if (sh.found_in > kList) return kNone;
  collect(bins.lower(bin), bins.upper(bin), bin, sh.list, kList);
  lds_barrier();
  const int n = min(sh.listing, kList);
  sort<THREADS>(sh, n);
  uint64_t m = 0;
#pragma unroll 1
  for (int j = 0; j < kEach; ++j) {
    const int i = j * THREADS + tid;
    if (i < n && (uint32_t)i < rest) m += weight_of(r, logit_of((uint32_t)(sh.list[i] >> 32)));
  }
  return before + sum_all<THREADS>(sh, m);
}

// k: of the rules, or 0 if `all`, the mass that top-p is of, is that of the first k: as p <= 1 - 2^-24, its last member
// is one of them.  (Else `all` is the row's.)  collect(low, high, edge bin, dest, cap) appends the places of all tokens with
// low <= l c < high to dest, sh.listing of them.  kDrawn: the token is written; kKnown: the edge is, and sh.list begins
// with the sh.found_in tokens beside it that are kept; kUnknown: draw_slowly.
// by_count: sh.count need not count all, but show a bin down to which there are k.
// pool [kPool]: place for tokens, or null; edge.pooled: how many of the edge's bin it has.
template <int THREADS, typename F>
__device__ __forceinline__ Outcome choose(Shared& sh, uint64_t* pool, const SampleArgs& a, int b, const Rules& r,
                                          int k, bool by_count, uint64_t all, int top_bin, Edge& edge, F collect) {
  constexpr int kEach = kList / THREADS;
  const int tid = threadIdx.x, wave = tid / kWave;
  const bool whole = by_count && r.top_p;  // (top-p's limit needs the first k's mass: the list has them)
  Bins bins{top_bin, false, 0.f};
  if (wave == 0) find_edge(sh, r, k, by_count, r.k > 0, whole, r.p * (double)all, bins, 0, 0);
  lds_barrier();
  edge.bin = sh.found;
  uint32_t before = sh.found_count;
  uint64_t before_mass = sh.found_mass;
  uint32_t in_edge = sh.found_in;
  // Whether all that can be kept is in the list.  (Sorting 2048 takes 12 us, twice; a part of a bin that
  // few share does not need it.)
  const bool listed = by_count || before + in_edge <= (uint32_t)(pool == nullptr ? kList : kFew);
  float low = bins.lower(edge.bin), high = listed ? INFINITY : bins.upper(edge.bin);
  if (listed || in_edge <= (uint32_t)(pool == nullptr ? kList : kFew)) {
    collect(low, high, edge.bin, sh.list, kList);
  } else {
    // more than the list holds: by the 512 parts of the bin
    if (pool == nullptr || in_edge > kPool || !(fabsf(low) < 0x1p14f)) return kUnknown;
    collect(low, high, edge.bin, pool, kPool);
    lds_barrier();
    for (int i = tid; i < kBins; i += THREADS) {
      sh.mass[i] = 0;
      sh.count[i] = 0;
    }
    lds_barrier();
    // (most_of shows too few where weights are a few units of 2^-44, rounded down)
    if (sh.listing > kPool) return kUnknown;
    bins.fine = true;
    bins.low = low;
    edge.pooled = sh.listing;
    for (int i = tid; i < edge.pooled; i += THREADS) {
      const float l = logit_of((uint32_t)(pool[i] >> 32));
      const int bin = bins.at(l * r.c);
      atomicAdd(&sh.count[bin], 1u);
      atomicAdd((unsigned long long*)&sh.mass[bin], (unsigned long long)weight_of(r, l));
    }
    lds_barrier();
    if (wave == 0) find_edge(sh, r, k, false, true, false, r.p * (double)all, bins, before_mass, before);
    lds_barrier();
    before = sh.found_count;
    before_mass = sh.found_mass;
    low = bins.lower(sh.found);
    high = bins.upper(sh.found);
    if (sh.found_in > kList) return kUnknown;
    for (int i = tid; i < edge.pooled; i += THREADS) {
      const float f = logit_of((uint32_t)(pool[i] >> 32)) * r.c;
      if (f >= low && f < high) sh.list[atomicAdd(&sh.listing, 1)] = pool[i];
    }
  }
  if (listed) {
    before = 0;
    before_mass = 0;
  }
  lds_barrier();
  const int n = sh.listing;
  if (n > kList) return kUnknown;  // (where bins do not count all)
  edge.high = high;
  auto keeps = [&](uint32_t rank, uint64_t mass_before, float l, double most) {
    return (k == 0 || rank < (uint32_t)k) && (!r.top_p || (double)mass_before < most) &&
           (l == r.max_f || (double)l - r.max >= r.lim);
  };

  if (listed && n <= kFew) {  // each against all
    uint64_t place = ~0ull, w = 0;
    float l = 0.f;
    if (tid < n) {
      place = sh.list[tid];
      l = logit_of((uint32_t)(place >> 32));
      w = weight_of(r, l);
      sh.weight[tid] = w;
    }
    lds_barrier();
    uint32_t rank = 0;
    uint64_t upto = 0;
    const bool active = wave * kWave < n;
    if (active) {
#pragma unroll 8
      for (int j = 0; j < n; ++j) {
        const uint64_t o = sh.list[j], ow = sh.weight[j];
        rank += o < place;
        upto += o < place ? ow : 0;
      }
    }
    uint64_t limit_mass = all;
    if (whole) limit_mass = sum_few(sh, 0, active && tid < n && rank < (uint32_t)r.k ? w : 0, n);
    if (!(tid < n && (rank == 0 || keeps(rank, upto, l, r.p * (double)limit_mass)))) w = 0;
    const uint64_t total = sum_few(sh, 1, w, n), target = target_of(a.uniform[b], total);
    if (tid < n) sh.weight[tid] = w;
    lds_barrier();
    if (!active) return kDrawn;
    uint64_t from = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) {
      const uint32_t o = (uint32_t)sh.list[j];
      const uint64_t ow = sh.weight[j];
      from += o < (uint32_t)place ? ow : 0;
    }
    if (tid < n && from <= target && target < from + w) finish(a, b, r, (int)(uint32_t)place, l, total);
    return kDrawn;
  }

  sort<THREADS>(sh, n);
  // kEach tokens a thread, in order: the kept ones are the first of them
  uint64_t w[kEach], sum = 0;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int i = tid * kEach + j;
    w[j] = i < n ? weight_of(r, logit_of((uint32_t)(sh.list[i] >> 32))) : 0;
    sum += w[j];
  }
  uint64_t upto = sum;
  uint32_t none = 0;
  sums_before<THREADS>(sh, upto, none);
  upto += before_mass;
  uint64_t limit_mass = all;
  if (whole) {
    uint64_t t = upto;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      t += w[j];
      if (tid * kEach + j == min(r.k, n) - 1) sh.found_mass = t;
    }
    lds_barrier();
    limit_mass = sh.found_mass;
  }
  if (tid == 0) sh.found = 0;
  lds_barrier();
  const double most = r.p * (double)limit_mass;
  int kept = 0;
  uint64_t kept_sum = 0;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int i = tid * kEach + j;
    if (i < n) {
      const bool keep = keeps(before + i, upto, logit_of((uint32_t)(sh.list[i] >> 32)), most);
      if (keep || before + i == 0) {
        kept = i + 1;
        kept_sum += w[j];
      }
    }
    upto += w[j];
  }
  if (kept > 0) atomicMax(&sh.found, kept);
  lds_barrier();
  kept = sh.found;
  if (!listed) {
    if (tid == 0) sh.found_in = (uint32_t)kept;
    if (kept > 0) {
      edge.l = logit_of((uint32_t)(sh.list[kept - 1] >> 32));
      edge.i = (int)(uint32_t)sh.list[kept - 1];
    } else {  // none of that bin: the least logit above it (l c is within a rounding or two of high)
      float l = high / r.c;
      for (int t = 0; t < 4 && !(l * r.c >= high); ++t) l = logit_of(key_of(l) - 1);
      for (int t = 0; t < 8 && logit_of(key_of(l) + 1) * r.c >= high; ++t) l = logit_of(key_of(l) + 1);
      edge.l = l;
      edge.i = INT32_MAX;
    }
    return kKnown;
  }
  // by number; the token
  const uint64_t total = sum_all<THREADS>(sh, kept_sum);
  uint64_t mine[kEach];
#pragma unroll
  for (int j = 0; j < kEach; ++j) mine[j] = sh.list[tid * kEach + j];
  lds_barrier();
#pragma unroll
  for (int j = 0; j < kEach; ++j)
    if (tid * kEach + j < kept) sh.list[tid * kEach + j] = mine[j] << 32 | mine[j] >> 32;
  lds_barrier();
  sort<THREADS>(sh, kept);
  const uint64_t target = target_of(a.uniform[b], total);
  uint64_t from = 0;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int i = tid * kEach + j;
    w[j] = i < kept ? weight_of(r, logit_of((uint32_t)sh.list[i])) : 0;
    from += w[j];
  }
  sums_before<THREADS>(sh, from, none);
  int found = -1;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    if (from <= target && target < from + w[j]) found = tid * kEach + j;
    from += w[j];
  }
  if (found >= 0) {
    const uint64_t e = sh.list[found];
    finish(a, b, r, (int)(e >> 32), logit_of((uint32_t)e), total);
  }
  return kDrawn;
}

// The first token at which the kept mass of ROUNDS pieces a thread, numbers from `first` on,
// exceeds `rest`.  piece(j): a round's.  whole_row: the row's token, rest and total follow from the
// sum; else total is the row's kept mass.  False if none of them has mass.
template <int TY, int THREADS, int ROUNDS, typename P>
__device__ __forceinline__ bool draw(Shared& sh, const SampleArgs& a, int b, const Rules& r, const Edge& edge, int first,
                                     uint64_t rest, bool whole_row, uint64_t total, P piece) {
  constexpr int N = kPiece<TY>, kWaves = THREADS / kWave, kParts = ROUNDS * kWaves;
  typedef typename Elem<TY>::V V;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  // (masked tokens are not above any l)
  auto keeps = [&](float l, int i) { return l > edge.l || (l == edge.l && i <= edge.i); };
  auto weights = [&](const V& v, int i, uint64_t* w) {
#pragma unroll
    for (int e = 0; e < N; e += 4) {  // (all at once would take too many registers)
      float l[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        l[k] = (float)v[e + k];
        asm volatile("" : "+v"(l[k]));
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint64_t x = weight_of(r, l[k]);
        w[e + k] = keeps(l[k], i + e + k) ? x : 0;
      }
    }
  };
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j) {
    const V v = piece(j);
    const int i = first + (j * THREADS + tid) * N;
    bool any = false;
#pragma unroll
    for (int e = 0; e < N; ++e) any |= keeps((float)v[e], i + e);
    uint64_t s = 0;
    if (__ballot(any) != 0) {
      uint64_t w[N];
      weights(v, i, w);
#pragma unroll
      for (int e = 0; e < N; ++e) s += w[e];
      s = wave_sum64(s);
    }
    if (lane == 0) sh.parts[j * kWaves + wave] = s;
  }
  lds_barrier();
  // the round and wave that it is in: the parts by lanes, two each
  static_assert(kParts <= 2 * kWave, "parts");
  const uint64_t p0 = 2 * lane < kParts ? sh.parts[2 * lane] : 0, p1 = 2 * lane + 1 < kParts ? sh.parts[2 * lane + 1] : 0;
  uint64_t before = wave_before(p0 + p1);
  const uint64_t sum = __shfl((unsigned long long)(before + p0 + p1), kWave - 1);
  if (sum == 0) return false;
  if (whole_row) {
    total = sum;
    rest = target_of(a.uniform[b], total);
  }
  rest = min(rest, sum - 1);
  const int at = __builtin_ctzll(__ballot(rest < before + p0 + p1));
  const bool second = rest >= before + p0;
  const int g = 2 * at + __shfl((int)second, at);
  before = __shfl((unsigned long long)(second ? before + p0 : before), at);
  if (g % kWaves != wave) return true;
  const int i = first + (g / kWaves * THREADS + tid) * N;
  const V f = load_piece<TY>((const typename Elem<TY>::T*)a.logits + b * a.row, min(i, a.vocab), a.vocab);
  uint64_t w[N], own = 0;
  weights(f, i, w);
#pragma unroll
  for (int e = 0; e < N; ++e) own += w[e] = i + e < a.vocab ? w[e] : 0;
  uint64_t from = before + wave_before(own);
  int found = -1;
  float found_l = 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    if (from <= rest && rest < from + w[e]) {
      found = i + e;
      found_l = (float)f[e];
    }
    from += w[e];
  }
  if (found >= 0) finish(a, b, r, found, found_l, total);
  return true;
}

__device__ __forceinline__ void no_token(const SampleArgs& a, int b) {
  if (threadIdx.x != 0) return;
  a.tokens[b] = -1;
  if (a.logprob != nullptr) a.logprob[b] = NAN;
}

// Pieces of elements [first, ...) of a row, THREADS apart; masked past its end.
template <int TY, int THREADS, int ROUNDS>
__device__ __forceinline__ void load_rounds(const void* row, int first, int vocab, typename Elem<TY>::V (&v)[ROUNDS]) {
  constexpr int N = kPiece<TY>;
  typedef typename Elem<TY>::T T;
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j) {
    const int i = first + (j * THREADS + threadIdx.x) * N;
    if (i + N <= vocab) {
      v[j] = *(const typename Elem<TY>::V*)((const T*)row + i);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) v[j][e] = i + e < vocab ? ((const T*)row)[i + e] : (T)-INFINITY;
    }
  }
}

// The largest of what the workgroup holds; NaN if one is.  mine: the thread's.
template <int TY, int THREADS, int ROUNDS>
__device__ __forceinline__ float largest(Shared& sh, const typename Elem<TY>::V (&v)[ROUNDS], float& mine) {
  float top = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j)
#pragma unroll
    for (int e = 0; e < kPiece<TY>; ++e) {
      const float l = (float)v[j][e];
      top = fmaxf(top, l);
      bad |= l != l;
    }
  mine = top;
  top = wave_largest(bad ? NAN : top);
  if (threadIdx.x % kWave == 0) sh.top[threadIdx.x / kWave] = top;
  lds_barrier();
#pragma unroll
  for (int w = 0; w < THREADS / kWave; ++w) top = larger(top, sh.top[w]);
  return top;
}

// The number of the first element that is `top`; sh.found is INT32_MAX before, and a barrier lies between.
template <int TY, int THREADS, int ROUNDS>
__device__ __forceinline__ int first_of(Shared& sh, const typename Elem<TY>::V (&v)[ROUNDS], int first, float top) {
  constexpr int N = kPiece<TY>;
  int at = INT32_MAX;
#pragma unroll
  for (int j = ROUNDS - 1; j >= 0; --j)
#pragma unroll
    for (int e = N - 1; e >= 0; --e)
      if ((float)v[j][e] == top) at = first + (j * THREADS + threadIdx.x) * N + e;
  if (at != INT32_MAX) atomicMin(&sh.found, at);
  lds_barrier();
  return sh.found;
}

// Bins and mass (of the thread) of what the workgroup holds, relative to its largest (r).
// slot(bin): where a bin is kept.
template <int TY, int ROUNDS, typename S>
__device__ __forceinline__ uint64_t count_bins(Shared& sh, const Rules& r, typename Elem<TY>::V (&v)[ROUNDS], bool filtered,
                                               S slot) {
  constexpr int G = 4;  // weights at a time (all at once would take too many registers)
  const int upper = bin_of(r.max_f, r.c);
  uint64_t total = 0;
#pragma unroll
  for (int j = 0; j < ROUNDS; ++j)
#pragma unroll
    for (int e0 = 0; e0 < kPiece<TY>; e0 += G) {
      float l[G];
      uint64_t w[G];
#pragma unroll
      for (int e = 0; e < G; ++e) {
        l[e] = (float)v[j][e0 + e];
        asm volatile("" : "+v"(l[e]));
      }
#pragma unroll
      for (int e = 0; e < G; ++e) total += w[e] = weight_of(r, l[e]);
      if (filtered) {
#pragma unroll
        for (int e = 0; e < G; ++e) {
          const int bin = upper - low_bin_of(l[e], r.c);  // (masked ones: far below)
          if (bin >= kBins - 1) continue;
          if (r.k > 0) atomicAdd(&sh.count[slot(bin)], 1u);  // (else: most_of)
          atomicAdd((unsigned long long*)&sh.mass[slot(bin)], (unsigned long long)w[e]);
        }
      }
    }
  return total;
}

__device__ __forceinline__ bool by_counts(const Rules& r) { return r.k > 0 && r.k <= kMostK; }
__device__ __forceinline__ bool is_filtered(const Rules& r) { return r.k > 0 || r.top_p || r.min_p; }
// Bins are whole numbers of 32 bits only for logits that are not huge next to T.
__device__ __forceinline__ bool has_bins(const Rules& r) { return fabsf(r.max_f * r.c) < 0x1p29f; }

// A row that a workgroup holds, ROUNDS pieces a thread.
template <int TY, int ROUNDS>
__global__ void __launch_bounds__(kRowThreads) k_sample_row(SampleArgs a) {
  constexpr int N = kPiece<TY>, THREADS = kRowThreads;
  typedef typename Elem<TY>::T T;
  typedef typename Elem<TY>::V V;
  __shared__ Shared sh;
  constexpr int kHits = ROUNDS > 8 ? 128 : 256;  // threads whose tokens are dealt out, at most
  __shared__ V dealt[ROUNDS > 1 ? kHits : 1][ROUNDS];
  __shared__ int whose[kHits], hits;
  const int tid = threadIdx.x, b = blockIdx.x;
  const void* const row = (const T*)a.logits + b * a.row;
  V v[ROUNDS];
  load_rounds<TY, THREADS, ROUNDS>(row, 0, a.vocab, v);
  Rules r = rules_of(a, b);
  for (int i = tid; i < kBins; i += THREADS) {
    sh.mass[i] = 0;
    sh.count[i] = 0;
  }
  if (tid == 0) {
    sh.found = INT32_MAX;
    hits = 0;
  }
  float mine;
  r.max_f = largest<TY, THREADS, ROUNDS>(sh, v, mine);
  if (!(r.max_f > -INFINITY)) return no_token(a, b);
  if (r.greedy) {
    const int first = first_of<TY, THREADS, ROUNDS>(sh, v, 0, r.max_f);
    if (tid == 0) {
      a.tokens[b] = first;
      if (a.logprob != nullptr) a.logprob[b] = 0.f;
    }
    return;
  }
  r.max = (double)r.max_f;
  Edge edge{-INFINITY, -1, 0, 0.f, 0};
  if (is_filtered(r)) {
    Outcome o = kUnknown;
    if (has_bins(r)) {
      const bool by_count = by_counts(r);
      const int top_bin = bin_of(r.max_f, r.c);
      uint64_t all = 0;
      if (by_count) {
        // the threads' largest alone: where k of them lie, at least k tokens do
        const int bin = top_bin - low_bin_of(mine, r.c);
        if (bin < kBins - 1) atomicAdd(&sh.count[bin], 1u);
        lds_barrier();
      } else {
        all = sum_all<THREADS>(sh, count_bins<TY, ROUNDS>(sh, r, v, true, [](int bin) { return bin; }));
      }
      auto collect = [&](float low, float high, int, uint64_t* dest, int cap) {
        if (ROUNDS > 1 && by_count) {
          // few threads hold any: theirs are dealt to all
          const bool hit = mine * r.c >= low;
          const int at = hit ? atomicAdd(&hits, 1) : kHits;
          if (at < kHits) {
            whose[at] = tid;
#pragma unroll
            for (int j = 0; j < ROUNDS; ++j) dealt[at][j] = v[j];
          }
          lds_barrier();
          const int n = hits;
          if (n <= kHits) {
            for (int i0 = 0; i0 < n * ROUNDS * N; i0 += THREADS) {
              const int i = min(i0 + tid, n * ROUNDS * N - 1), w = i / (ROUNDS * N), j = i / N % ROUNDS, e = i % N;
              const float l = (float)((const T*)&dealt[w][j])[e];
              append<1>(sh.listing, dest, cap, [&](int) { return i == i0 + tid && l * r.c >= low; },
                        [&](int) { return place_of(l, (j * THREADS + whose[w]) * N + e); });
            }
            return;
          }
        }
#pragma unroll
        for (int j = 0; j < ROUNDS; ++j) {
          asm volatile("" : "+v"(v[j]));
          append<N>(sh.listing, dest, cap, [&](int e) {
            const float f = (float)v[j][e] * r.c;
            return f >= low && f < high;
          }, [&](int e) { return place_of((float)v[j][e], (j * THREADS + tid) * N + e); });
        }
      };
      const bool first = r.k > 0 && r.top_p && !by_count;
      if (first) all = mass_of_first<THREADS>(sh, r, top_bin, collect);
      if (all != kNone)
        o = choose<THREADS>(sh, nullptr, a, b, r, first ? 0 : r.k, by_count, all, top_bin, edge, collect);
    }
    if (o == kDrawn) return;
    if (o == kUnknown) return draw_slowly<TY, THREADS>(sh, a, b, r);
  }
  draw<TY, THREADS, ROUNDS>(sh, a, b, r, edge, 0, 0, true, 0, [&](int j) {
    asm volatile("" : "+v"(v[j]));  // (otherwise the elements converted above are kept, which spills)
    return v[j];
  });
}

// A slice of a longer row.
template <int TY>
__global__ void __launch_bounds__(kSliceThreads) k_sample_slices(SampleArgs a) {
  constexpr int N = kPiece<TY>, THREADS = kSliceThreads, ROUNDS = kSampleSlice / (THREADS * N);
  typedef typename Elem<TY>::V V;
  __shared__ Shared sh;
  const int tid = threadIdx.x, b = blockIdx.y, slice = blockIdx.x;
  const int64_t at = (int64_t)b * gridDim.x + slice;
  const void* const row = (const typename Elem<TY>::T*)a.logits + b * a.row;
  V v[ROUNDS];
  load_rounds<TY, THREADS, ROUNDS>(row, slice * kSampleSlice, a.vocab, v);
  Rules r = rules_of(a, b);
  const bool by_count = by_counts(r), filtered = is_filtered(r);
  sh.mass[tid] = 0;
  sh.count[tid] = 0;
  if (tid == 0) sh.found = INT32_MAX;
  float mine;
  r.max_f = largest<TY, THREADS, ROUNDS>(sh, v, mine);
  SampleRecord rec{};
  rec.top = r.max_f;
  rec.cut = -1;
  if (r.max_f > -INFINITY) {
    if (r.greedy) {
      rec.mass = (uint64_t)first_of<TY, THREADS, ROUNDS>(sh, v, slice * kSampleSlice, r.max_f);
    } else {
      r.max = (double)r.max_f;
      const int upper = bin_of(r.max_f, r.c);
      // (a bin's place does not depend on the slice's maximum, so that those of a row lie beside one another)
      auto slot = [&](int bin) { return (upper - bin) & (kBins - 1); };
      if (by_count) {
        // the threads' largest alone: where k of them lie, at least k tokens do
        const int bin = upper - low_bin_of(mine, r.c);
        if (bin < kBins - 1) atomicAdd(&sh.count[slot(bin)], 1u);
        lds_barrier();
      } else {
        rec.mass = sum_all<THREADS>(sh, count_bins<TY, ROUNDS>(sh, r, v, filtered, slot));
      }
      if (filtered) {
        if (!by_count) a.masses[at * kBins + tid] = sh.mass[tid];
        if (!by_count && r.k > 0) a.counts[at * kBins + tid] = sh.count[tid];
        // the first tokens: down to the bin with the k-th, or to the last one up to which a list holds all
        uint64_t none = 0;
        const uint32_t own = by_count || r.k > 0 ? sh.count[slot(tid)] : most_of(r, sh.mass[slot(tid)], (float)(upper - tid));
        uint32_t c = own;
        sums_before<THREADS>(sh, none, c);
        if (tid == 0) {
          sh.found = by_count ? kBins - 1 : 0;
          sh.listing = 0;
        }
        lds_barrier();
        if (by_count && c < (uint32_t)r.k && (uint32_t)r.k <= c + own) sh.found = tid + 1;
        if (!by_count && tid < kBins - 1 && c + own <= kSampleListed) atomicMax(&sh.found, tid + 1);
        lds_barrier();
        rec.cut = sh.found - 1;
        const float low = least_not_below(upper - rec.cut);
#pragma unroll
        for (int j = 0; j < ROUNDS; j += 8 / N)
          append<8>(sh.listing, a.lists + at * kSampleListed, kSampleListed,
                    [&](int k) { return (float)v[j + k / N][k % N] * r.c >= low; }, [&](int k) {
                      return place_of((float)v[j + k / N][k % N],
                                      slice * kSampleSlice + ((j + k / N) * THREADS + tid) * N + k % N);
                    });
        lds_barrier();
        rec.listed = sh.listing;
        if (rec.listed > kSampleListed) {  // (more than the counts show)
          rec.cut = -1;
          rec.listed = 0;
        }
      }
    }
  }
  if (tid == 0) a.records[at] = rec;
}

// A row from its slices.
template <int TY>
__global__ void __launch_bounds__(kJoinThreads) k_sample_join(SampleArgs a, int slices) {
  constexpr int N = kPiece<TY>, THREADS = kJoinThreads, ROUNDS = kSampleSlice / (THREADS * N);
  typedef typename Elem<TY>::V V;
  __shared__ Shared sh;
  extern __shared__ __align__(16) uint64_t pool[];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, b = blockIdx.x;
  const int64_t at = (int64_t)b * slices;
  const void* const row = (const typename Elem<TY>::T*)a.logits + b * a.row;
  Rules r = rules_of(a, b);
  SampleRecord rec{};
  rec.top = -INFINITY;
  if (lane < slices) rec = a.records[at + lane];
  r.max_f = wave_largest(rec.top);
  if (!(r.max_f > -INFINITY)) return no_token(a, b);
  if (r.greedy) {
    if (tid == __builtin_ctzll(__ballot(rec.top == r.max_f))) {
      a.tokens[b] = (int32_t)rec.mass;
      if (a.logprob != nullptr) a.logprob[b] = 0.f;
    }
    return;
  }
  r.max = (double)r.max_f;
  const bool by_count = by_counts(r), filtered = is_filtered(r);
  // slices' masses in multiples of 2^-44 of the row's largest weight
  const bool some = rec.top > -INFINITY;
  const double by = !some ? 0.0 : rec.top == r.max_f ? 1.0 : factor(((double)rec.top - r.max) * r.inv);
  uint64_t mass = (uint64_t)((double)rec.mass * by + 0.5);
  Edge edge{-INFINITY, -1, 0, 0.f, 0};
  if (filtered) {
    Outcome o = kUnknown;
    const int top_bin = bin_of(r.max_f, r.c), lower = some ? top_bin - bin_of(rec.top, r.c) : 2 * kBins;
    if (has_bins(r)) {
      uint64_t all = wave_sum64(mass);
      // Calls f(held, place) for all that the slices' lists hold, by whole waves.
      auto lists = [&](auto f) {
        for (int s = wave; s < slices; s += THREADS / kWave) {
          const int n = __builtin_amdgcn_readlane(rec.listed, s);
          const uint64_t* const list = a.lists + (at + s) * kSampleListed;
          uint64_t e[kSampleListed / kWave];
#pragma unroll
          for (int j = 0; j < kSampleListed / kWave; ++j)
            if (j * kWave < n) e[j] = list[min(j * kWave + lane, n - 1)];
#pragma unroll
          for (int j = 0; j < kSampleListed / kWave; ++j)
            if (j * kWave < n) f(j * kWave + lane < n, e[j]);
        }
      };
      if (by_count) {
        if (tid < kBins) sh.count[tid] = 0;
        lds_barrier();
        lists([&](bool held, uint64_t place) {
          const int bin = top_bin - low_bin_of(logit_of((uint32_t)(place >> 32)), r.c);
          if (held && bin < kBins - 1) atomicAdd(&sh.count[bin], 1u);
        });
      } else if (tid < kBins) {
        // the row's bins, a thread each; the lowest one has what has no mass
        const int bin = (top_bin - tid) & (kBins - 1);
        double m = 0.0;
        uint32_t c = 0;
        constexpr int kBatch = 16;
        for (int s0 = 0; s0 < slices; s0 += kBatch) {
          uint64_t masses[kBatch];
          uint32_t counts[kBatch];
#pragma unroll
          for (int j = 0; j < kBatch; ++j) {
            const int64_t i = (at + min(s0 + j, slices - 1)) * kBins + tid;
            counts[j] = r.k > 0 ? a.counts[i] : 0;
            masses[j] = a.masses[i];
          }
#pragma unroll
          for (int j = 0; j < kBatch; ++j) {
            const int s = min(s0 + j, kWave - 1);
            // (a slice's place holds another bin where the row's is above its maximum)
            const bool has = s0 + j < slices && bin >= __builtin_amdgcn_readlane(lower, s) && bin < kBins - 1;
            const double f = __shfl(by, s);  // (by all lanes)
            c += has ? counts[j] : 0;
            m += has ? (double)masses[j] * f : 0.0;
          }
        }
        sh.mass[bin] = (uint64_t)(m + 0.5);
        sh.count[bin] = c;
      }
      lds_barrier();
      // (of counted rows every slice lists the first k, or it does not count here)
      if (!by_count || __ballot(some && rec.cut < 0) == 0) {
        auto collect = [&](float low, float high, int edge_bin, uint64_t* dest, int cap) {
          if (by_count || __ballot(some && edge_bin - lower > rec.cut) == 0)
            lists([&](bool held, uint64_t place) {
              const float f = logit_of((uint32_t)(place >> 32)) * r.c;
              append<1>(sh.listing, dest, cap, [&](int) { return held && f >= low && f < high; }, [&](int) { return place; });
            });
          else
            append_row<TY, THREADS>(sh.listing, dest, cap, row, a.vocab, r.c, low, high);
        };
        const bool first = r.k > 0 && r.top_p && !by_count;
        if (first) all = mass_of_first<THREADS>(sh, r, top_bin, collect);
        if (all != kNone) o = choose<THREADS>(sh, pool, a, b, r, first ? 0 : r.k, by_count, all, top_bin, edge, collect);
      }
    }
    if (o == kDrawn) return;
    if (o == kUnknown) return draw_slowly<TY, THREADS>(sh, a, b, r);
    // kept mass of the slices: their bins above the edge, and what the list keeps
    if (wave == 0) sh.factor[lane] = by;
    lds_barrier();
    for (int s = wave; s < slices; s += THREADS / kWave) {
      uint64_t m = 0;
      const int from = __builtin_amdgcn_readlane(lower, s);
      for (int i = lane; i < edge.bin - from; i += kWave)
        m += a.masses[(at + s) * kBins + ((top_bin - from - i) & (kBins - 1))];
      m = wave_sum64(m);
      if (lane == 0) sh.slice[s] = (uint64_t)((double)m * sh.factor[s] + 0.5);
    }
    lds_barrier();
    for (int i = tid; i < edge.pooled; i += THREADS) {  // of its bin, what lies above the list
      const float l = logit_of((uint32_t)(pool[i] >> 32));
      if (l * r.c >= edge.high)
        atomicAdd((unsigned long long*)&sh.slice[(uint32_t)pool[i] / kSampleSlice], (unsigned long long)weight_of(r, l));
    }
    for (int i = tid; i < (int)sh.found_in; i += THREADS)
      atomicAdd((unsigned long long*)&sh.slice[(uint32_t)sh.list[i] / kSampleSlice],
                (unsigned long long)weight_of(r, logit_of((uint32_t)(sh.list[i] >> 32))));
    lds_barrier();
    mass = lane < slices ? sh.slice[lane] : 0;
  }
  // the slice, then the token in it
  const uint64_t before = wave_before(mass), total = wave_sum64(mass), target = target_of(a.uniform[b], total);
  int s = __builtin_ctzll(__ballot(before <= target && target < before + mass));
  uint64_t rest = target - __shfl((unsigned long long)before, s);
#pragma unroll 1
  for (int turn = 0; turn < 2; ++turn) {
    V v[ROUNDS];
    load_rounds<TY, THREADS, ROUNDS>(row, s * kSampleSlice, a.vocab, v);
    if (draw<TY, THREADS, ROUNDS>(sh, a, b, r, edge, s * kSampleSlice, rest, false, total, [&](int j) { return v[j]; })) return;
    // (the slice's mass is less than the multiples show: the largest one's has some)
    s = __builtin_ctzll(__ballot(rec.top == r.max_f));
    rest = 0;
    lds_barrier();
  }
}

template <int TY>
hipError_t launch_typed(SampleArgs a, hipStream_t s) {
  constexpr int kRound = kRowThreads * kPiece<TY>;
  if (!sample_cut(a.vocab, a.top_k != nullptr)) {
    if (a.vocab <= kRound) k_sample_row<TY, 1><<<(unsigned)a.rows, kRowThreads, 0, s>>>(a);
    else if (a.vocab <= kSampleSlice) k_sample_row<TY, kSampleSlice / kRound><<<(unsigned)a.rows, kRowThreads, 0, s>>>(a);
    else k_sample_row<TY, kSampleRow / kRound><<<(unsigned)a.rows, kRowThreads, 0, s>>>(a);
    return hipGetLastError();
  }
  const int slices = (a.vocab + kSampleSlice - 1) / kSampleSlice, most = kSampleSlices / slices;
  hipError_t e = allow_dynamic_lds((const void*)k_sample_join<TY>, kPool * 8);
  if (e != hipSuccess) return e;
  for (int rows = a.rows; rows > 0; rows -= most) {
    const unsigned n = (unsigned)(rows < most ? rows : most);
    k_sample_slices<TY><<<dim3((unsigned)slices, n), kSliceThreads, 0, s>>>(a);
    k_sample_join<TY><<<n, kJoinThreads, kPool * 8, s>>>(a, slices);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.logits = (const uint8_t*)a.logits + most * a.row * dtype_bytes(TY);
    a.uniform += most;
    a.tokens += most;
    if (a.logprob != nullptr) a.logprob += most;
    if (a.temperature != nullptr) a.temperature += most;
    if (a.top_k != nullptr) a.top_k += most;
    if (a.top_p != nullptr) a.top_p += most;
    if (a.min_p != nullptr) a.min_p += most;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t s) {
  if (dtype == kF16) return launch_typed<kF16>(a, s);
  if (dtype == kBf16) return launch_typed<kBf16>(a, s);
  return launch_typed<kF32>(a, s);
}

}  // namespace aqlm
