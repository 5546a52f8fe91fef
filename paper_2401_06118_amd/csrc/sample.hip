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
// Weights are whole multiples of 2^-44, computed in 64 bits, and added as integers: the
// token does not depend on an order of sums, and differs from that of real numbers
// only where u is within about 2^-40 of a border.
//
// A workgroup takes a slice of 8192 logits and holds it in registers: its maximum, and
// relative to that counts and masses by bins of 1/16 of T (512 of them: what is lower has
// no mass left).  The last workgroup of a row joins the slices', finds the bin in which the
// last member lies, collects the tokens down to it from the row (or, if those are more
// than the list holds, that bin's), sorts them, and draws.  What the list does
// not hold (thousands of equal logits) is found by eleven bits of logit and number at a time.
#include "ends.h"

#include "common.h"
#include "elements.h"
#include "join.h"
#include "launch.h"
#include "lds_sync.h"

namespace aqlm {

namespace {

constexpr int kThreads = 512, kWaves = kThreads / kWave;
constexpr int kBins = 512;    // of a slice, one a thread
constexpr int kList = 2048;   // tokens that are sorted
constexpr int kMostK = 1024;  // up to this top-k bins need no masses: the list holds all that count
constexpr int kDigit = 2048;  // bins of the search by bits
constexpr int kSegments = 2048;  // of a row: 64 pieces of 16 bytes each
static_assert(kBins == kThreads, "a thread has a bin");
static_assert(kSampleMaxVocab <= kSegments * kWave * 4, "segments");
static_assert(kSampleMaxVocab <= kSampleSlice * kWave, "a wave has a row's slices");

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

__device__ __forceinline__ int bin_of(float l, float c) {
  return (int)floorf(fminf(fmaxf(l * c, -0x1p30f), 0x1p30f));
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


// 2^y for y <= 0.
__device__ __forceinline__ double factor(double y) { return y > -1000.0 ? exp2(y) : 0.0; }

struct Search {
  uint64_t mass[kDigit];  // of bins; then of segments
  uint32_t count[kDigit];
};
struct Joined {
  double factor[kWave];  // of a slice's masses
  uint64_t mass[kWave];  // of a slice
  int32_t offset[kWave];  // of its bins
  uint64_t list[kList];
};
struct Shared {
  union {
    Search search;
    Joined joined;
    struct {
      uint64_t mass[kBins];
      uint32_t count[kBins];
    } slice;
  };
  uint64_t wave_mass[kWaves];
  uint32_t wave_count[kWaves];
  uint64_t waves[4][kWaves];
  uint64_t found_mass;
  uint32_t found_count;
  int32_t found;
  int32_t flag;
  float top[kWaves];
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
  lds_barrier();
  m = im - m;
  c = ic - c;
  for (int w = 0; w < wave; ++w) {
    m += sh.wave_mass[w];
    c += sh.wave_count[w];
  }
  lds_barrier();
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

// Calls f(number, logit) for every token of the row that is not masked.
template <int TY, typename F>
__device__ __forceinline__ void each(const void* row, int vocab, F f) {
  constexpr int N = kPiece<TY>;
  for (int i = threadIdx.x * N; i < vocab; i += kThreads * N) {
    const typename Elem<TY>::V v = load_piece<TY>(row, i, vocab);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float l = (float)v[e];
      asm volatile("" : "+v"(l));  // (one after another: all at once would take too many registers)
      if (i + e < vocab && l != -INFINITY) f(i + e, l);
    }
  }
}

// The place of the last of the order's tokens up to `most` of them (by_count) or until they
// have `mass`; kept_mass: its own and all before it.
template <int TY>
__device__ __forceinline__ uint64_t last_kept(Shared& sh, const Rules& r, const void* row, int vocab, bool by_count, uint32_t most,
                              double mass, uint64_t& kept_mass) {
  constexpr int kEach = kDigit / kThreads;
  const int tid = threadIdx.x;
  uint64_t prefix = 0, above_mass = 0;
  uint32_t above = 0;
  // bits 53..63, 42..52, 32..41 (the logit), 10..19, 0..9 (the number)
#pragma unroll 1
  for (int d = 0; d < 5; ++d) {
    const int shift = d == 0 ? 53 : d == 1 ? 42 : d == 2 ? 32 : d == 3 ? 10 : 0;
    const int top = d == 0 ? 64 : d == 1 ? 53 : d == 2 ? 42 : d == 3 ? 32 : 10;
    const int mask = d < 2 ? 2047 : 1023;
    for (int i = tid; i < kDigit; i += kThreads) {
      sh.search.mass[i] = 0;
      sh.search.count[i] = 0;
    }
    if (tid == 0) sh.found = -1;
    lds_barrier();
    each<TY>(row, vocab, [&](int i, float l) {
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
    sums_before(sh, m, c);
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
template <int TY>
__device__ __forceinline__ void draw_slowly(Shared& sh, const SampleArgs& a, int b, const Rules& r) {
  constexpr int N = kPiece<TY>, kEach = kSegments / kThreads;
  typedef typename Elem<TY>::T T;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const T* const row = (const T*)a.logits + b * a.row;
  uint64_t last = ~0ull, kept = 0;
  lds_barrier();
  if (r.k > 0) last = last_kept<TY>(sh, r, row, a.vocab, true, (uint32_t)r.k, 0.0, kept);
  if (r.top_p) {
    if (last == ~0ull) {
      uint64_t m = 0;
      each<TY>(row, a.vocab, [&](int, float l) { m += weight_of(r, l); });
      m = wave_sum64(m);
      if (lane == 0) sh.wave_mass[wave] = m;
      lds_barrier();
      for (int w = 0; w < kWaves; ++w) kept += sh.wave_mass[w];
      lds_barrier();
    }
    const uint64_t q = last_kept<TY>(sh, r, row, a.vocab, false, 0, fmax(r.p * (double)kept, 1.0), kept);
    last = q < last ? q : last;
  }
  auto weight = [&](int i, float l) -> uint64_t {
    return i < a.vocab && l != -INFINITY && place_of(l, i) <= last && (l == r.max_f || (double)l - r.max >= r.lim)
               ? weight_of(r, l) : 0;
  };
  // kept mass of each segment of 64 pieces
  const int segments = (a.vocab + kWave * N - 1) / (kWave * N);
  for (int g = wave; g < segments; g += kWaves) {
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
  for (int g = segments + tid; g < kSegments; g += kThreads) sh.search.mass[g] = 0;
  lds_barrier();
  uint64_t m = 0;
  uint32_t none = 0;
  for (int j = 0; j < kEach; ++j) m += sh.search.mass[kEach * tid + j];
  const uint64_t mine = m;
  sums_before(sh, m, none);
  if (tid == kThreads - 1) sh.found_mass = m + mine;
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

// One workgroup a slice; the last of a row goes on with it.
template <int TY>
__global__ void __launch_bounds__(kThreads) k_sample(SampleArgs a) {
  constexpr int N = kPiece<TY>, PER = kSampleSlice / (kThreads * N);
  typedef typename Elem<TY>::T T;
  typedef typename Elem<TY>::V V;
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int b = blockIdx.y, slices = gridDim.x, slice = blockIdx.x;
  const T* const row = (const T*)a.logits + b * a.row;
  // (rows of a launch have a workspace each)
  uint64_t* const records = a.records + (int64_t)b * slices * 2;
  uint64_t* const masses = a.masses + (int64_t)b * slices * kBins;
  uint32_t* const counts = a.counts + (int64_t)b * slices * kBins;
  float x[PER][N];
  {
    V v[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int i = slice * kSampleSlice + (j * kThreads + tid) * N;
      if (i + N <= a.vocab) v[j] = *(const V*)(row + i);
      else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[j][e] = i + e < a.vocab ? row[i + e] : (T)-INFINITY;
      }
    }
#pragma unroll
    for (int j = 0; j < PER; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) x[j][e] = (float)v[j][e];
  }
  Rules r = rules_of(a, b);
  const bool by_count = r.k > 0 && r.k <= kMostK, filtered = r.k > 0 || r.top_p || r.min_p;
  sh.slice.mass[tid] = 0;
  sh.slice.count[tid] = 0;
  float top = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int j = 0; j < PER; ++j)
#pragma unroll
    for (int e = 0; e < N; ++e) {
      top = fmaxf(top, x[j][e]);
      bad |= x[j][e] != x[j][e];
    }
  top = bad ? NAN : top;
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) {
    const float o = __shfl_xor(top, s);
    top = o > top || o != o ? o : top;  // (NaN stays)
  }
  if (lane == 0) sh.top[wave] = top;
  if (tid == 0) sh.found = INT32_MAX;
  lds_barrier();
  for (int w = 0; w < kWaves; ++w) {
    const float o = sh.top[w];
    top = o > top || o != o ? o : top;
  }
  uint64_t total = 0;  // greedy rows: the first of the largest
  if (top > -INFINITY) {
    if (r.greedy) {
      int first = INT32_MAX;
#pragma unroll
      for (int j = PER - 1; j >= 0; --j)
#pragma unroll
        for (int e = N - 1; e >= 0; --e)
          if (x[j][e] == top) first = slice * kSampleSlice + (j * kThreads + tid) * N + e;
      if (first != INT32_MAX) atomicMin(&sh.found, first);
      lds_barrier();
      total = (uint64_t)(uint32_t)sh.found;
    } else {
      r.max_f = top;
      r.max = (double)top;
      const int upper = bin_of(top, r.c);
#pragma unroll
      for (int j = 0; j < PER; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          float l = x[j][e];
          asm volatile("" : "+v"(l));  // (one after another: all at once would take too many registers)
          const int bin = filtered ? upper - bin_of(l, r.c) : 0;
          if (l == -INFINITY || bin >= kBins - 1) continue;
          if (filtered) atomicAdd(&sh.slice.count[bin], 1u);
          if (!by_count) {
            const uint64_t w = weight_of(r, l);
            total += w;
            if (filtered) atomicAdd((unsigned long long*)&sh.slice.mass[bin], (unsigned long long)w);
          }
        }
      total = wave_sum64(total);
      if (lane == 0) sh.wave_mass[wave] = total;
      lds_barrier();
      total = 0;
      for (int w = 0; w < kWaves; ++w) total += sh.wave_mass[w];
      if (filtered) {
        put_through(counts + slice * kBins + tid, sh.slice.count[tid]);
        if (!by_count) put_through(masses + slice * kBins + tid, sh.slice.mass[tid]);
      }
    }
  }
  if (tid == 0) {
    put_through(records + slice * 2, (uint64_t)__builtin_bit_cast(uint32_t, top));
    put_through(records + slice * 2 + 1, total);
  }
  if (!last_of(a.counters + b, (uint32_t)slices, &sh.flag)) return;

  // The row: a lane has a slice.
  uint64_t rec_mass = 0;
  float rec_top = -INFINITY;
  if (lane < slices) {
    rec_top = __builtin_bit_cast(float, (uint32_t)get_through(records + lane * 2));
    rec_mass = get_through(records + lane * 2 + 1);
  }
  top = rec_top;
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) {
    const float o = __shfl_xor(top, s);
    top = o > top || o != o ? o : top;
  }
  if (!(top > -INFINITY)) {  // NaN, or nothing that could be drawn
    if (tid == 0) {
      a.tokens[b] = -1;
      if (a.logprob != nullptr) a.logprob[b] = NAN;
    }
    return;
  }
  if (r.greedy) {
    const uint64_t which = __ballot(rec_top == top);
    if (tid == __builtin_ctzll(which)) {
      a.tokens[b] = (int32_t)rec_mass;
      if (a.logprob != nullptr) a.logprob[b] = 0.f;
    }
    return;
  }
  r.max_f = top;
  r.max = (double)top;
  const float top_c = top * r.c;
  bool slowly = filtered && !(fabsf(top_c) < 0x1p29f);
  // slices' masses in multiples of 2^-44 of the row's largest weight
  const int top_bin = bin_of(top, r.c);
  const bool some = rec_top > -INFINITY;
  const double by = some ? rec_top == top ? 1.0 : factor(((double)rec_top - r.max) * r.inv) : 0.0;
  const int offset = some ? min(top_bin - bin_of(rec_top, r.c), kBins) : kBins;
  uint64_t mass = (uint64_t)((double)rec_mass * by + 0.5);
  const uint64_t all = wave_sum64(mass);
  const float u = a.uniform[b];
  // kept: bins above the edge, and in it up to the last one
  float edge_low = -INFINITY, edge_high = -INFINITY;
  uint64_t last = 0;
  do {
    if (!filtered || slowly) break;
    if (wave == 0) {
      sh.joined.factor[lane] = by;
      sh.joined.offset[lane] = offset;
    }
    lds_barrier();
    // the row's bins, a thread each; the lowest one has what has no mass
    double bin_mass = 0.0;
    uint32_t bin_count = 0;
    for (int s = 0; s < slices; ++s) {
      const int from = tid - sh.joined.offset[s];
      if (from < 0 || tid >= kBins - 1) continue;
      bin_count += get_through(counts + s * kBins + from);
      if (!by_count) bin_mass += (double)get_through(masses + s * kBins + from) * sh.joined.factor[s];
    }
    const uint64_t own = (uint64_t)(bin_mass + 0.5);
    uint64_t m = own;
    uint32_t c = bin_count;
    sums_before(sh, m, c);
    // the bin of the last kept one: the first of those in which a rule's limit lies
    if (tid == 0) sh.found = kBins - 2;
    lds_barrier();
    const bool whole = r.k > 0 && r.top_p;  // (top-p's limit needs the first k's mass)
    slowly = whole && !by_count;
    if (slowly) break;
    bool limit = r.k > 0 && c < (uint32_t)r.k && (uint32_t)r.k <= c + bin_count;
    if (!by_count) limit |= r.top_p && bin_count != 0 && (double)(m + own) >= r.p * (double)all;
    if (limit) atomicMin(&sh.found, tid);
    if (r.min_p && !whole && tid == 0) {
      // the largest logit in 32 bits that is not above the limit: what lies in higher bins is kept
      const double least = r.max + r.lim;
      float f = (float)least;
      if ((double)f > least) f = key_of(f) == ~0u ? f : logit_of(key_of(f) + 1);
      atomicMin(&sh.found, max(0, min(top_bin - bin_of(f, r.c), kBins - 2)));
    }
    lds_barrier();
    const int edge = sh.found;
    lds_barrier();
    if (tid == edge) {
      sh.found_mass = m;
      sh.found_count = c;
      sh.flag = (int)bin_count;
    }
    if (tid == 0) sh.found = 0;
    lds_barrier();
    uint32_t before = sh.found_count;
    uint64_t before_mass = sh.found_mass;
    const uint32_t in_edge = (uint32_t)sh.flag;
    const bool listed = before + in_edge <= kList;  // all that can be kept is in the list
    slowly = !listed && (by_count || in_edge > kList);
    if (slowly) break;
    if (listed) {
      before = 0;
      before_mass = 0;
    }
    // collect
    const float low = (float)(top_bin - edge), high = listed ? INFINITY : low + 1.f;
    each<TY>(row, a.vocab, [&](int i, float l) {
      const float f = l * r.c;
      if (f >= low && f < high) {
        const int at = atomicAdd(&sh.found, 1);
        if (at < kList) sh.joined.list[at] = place_of(l, i);
      }
    });
    lds_barrier();
    const int n = min(sh.found, kList);
    auto sort = [&](int n) {
      int size = 2;
      while (size < n) size <<= 1;
      for (int i = n + tid; i < size; i += kThreads) sh.joined.list[i] = ~0ull;
      lds_barrier();
      for (int k = 2; k <= size; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
          for (int i = tid; i < size / 2; i += kThreads) {
            const int lo = 2 * i - (i & (j - 1)), hi = lo + j;
            const uint64_t p = sh.joined.list[lo], q = sh.joined.list[hi];
            if ((p > q) == ((lo & k) == 0)) {
              sh.joined.list[lo] = q;
              sh.joined.list[hi] = p;
            }
          }
          lds_barrier();
        }
    };
    sort(n);
    // four tokens a thread, in order: the kept ones are the first of them
    constexpr int kEach = kList / kThreads;
    uint64_t w[kEach], sum = 0;
    for (int j = 0; j < kEach; ++j) {
      const int i = tid * kEach + j;
      w[j] = i < n ? weight_of(r, logit_of((uint32_t)(sh.joined.list[i] >> 32))) : 0;
      sum += w[j];
    }
    uint64_t upto = sum;
    uint32_t none = 0;
    sums_before(sh, upto, none);
    upto += before_mass;
    uint64_t limit_mass = all;
    if (whole) {
      uint64_t t = upto;
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
    for (int j = 0; j < kEach; ++j) {
      const int i = tid * kEach + j;
      if (i < n) {
        const float l = logit_of((uint32_t)(sh.joined.list[i] >> 32));
        const bool keep = (r.k == 0 || before + i < (uint32_t)r.k) && (!r.top_p || (double)upto < most) &&
                          (l == top || (double)l - r.max >= r.lim);
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
    if (listed) {
      // by number; the token
      kept_sum = wave_sum64(kept_sum);
      if (lane == 0) sh.wave_mass[wave] = kept_sum;
      uint64_t mine[kEach];
      for (int j = 0; j < kEach; ++j) mine[j] = sh.joined.list[tid * kEach + j];
      lds_barrier();
      uint64_t sum_all = 0;
      for (int v = 0; v < kWaves; ++v) sum_all += sh.wave_mass[v];
      for (int j = 0; j < kEach; ++j)
        if (tid * kEach + j < kept) sh.joined.list[tid * kEach + j] = mine[j] << 32 | mine[j] >> 32;
      lds_barrier();
      sort(kept);
      const uint64_t target = target_of(u, sum_all);
      uint64_t m2 = 0;
      for (int j = 0; j < kEach; ++j) {
        const int i = tid * kEach + j;
        w[j] = i < kept ? weight_of(r, logit_of((uint32_t)sh.joined.list[i])) : 0;
        m2 += w[j];
      }
      sums_before(sh, m2, none);
      int found = -1;
      for (int j = 0; j < kEach; ++j) {
        if (m2 <= target && target < m2 + w[j]) found = tid * kEach + j;
        m2 += w[j];
      }
      if (found >= 0) {
        const uint64_t e = sh.joined.list[found];
        finish(a, b, r, (int)(e >> 32), logit_of((uint32_t)e), sum_all);
      }
      return;
    }
    // kept mass of the slices: their bins above the edge, and what the list keeps
    last = kept > 0 ? sh.joined.list[kept - 1] : 0;
    edge_low = low;
    edge_high = high;
    if (tid < kWave) sh.joined.mass[tid] = 0;
    lds_barrier();
    for (int s = wave; s < slices; s += kWaves) {
      uint64_t v = 0;
      for (int i = lane; i < edge - sh.joined.offset[s]; i += kWave) v += get_through(masses + s * kBins + i);
      v = wave_sum64(v);
      if (lane == 0) sh.joined.mass[s] = (uint64_t)((double)v * sh.joined.factor[s] + 0.5);
    }
    lds_barrier();
    for (int j = 0; j < kEach; ++j) {
      const int i = tid * kEach + j;
      if (i < kept)
        atomicAdd((unsigned long long*)&sh.joined.mass[(uint32_t)sh.joined.list[i] / kSampleSlice],
                  (unsigned long long)w[j]);
    }
    lds_barrier();
    mass = sh.joined.mass[lane];
  } while (false);
  if (slowly) return draw_slowly<TY>(sh, a, b, r);

  // The slice, then the token in it.
  const uint64_t mass_before = wave_before(mass), mass_all = wave_sum64(mass), target = target_of(u, mass_all);
  const uint64_t which = __ballot(mass_before <= target && target < mass_before + mass);
  int at = __builtin_ctzll(which);
  uint64_t rest = target - __shfl((unsigned long long)mass_before, at);
  auto weight = [&](int i, float l) -> uint64_t {
    const float f = l * r.c;
    return i < a.vocab && l != -INFINITY && (!filtered || f >= edge_high || (f >= edge_low && place_of(l, i) <= last))
               ? weight_of(r, l) : 0;
  };
#pragma unroll 1
  for (int turn = 0; turn < 2; ++turn) {
    const int i0 = at * kSampleSlice + tid * N;
    V v[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (i0 + j * kThreads * N < a.vocab) v[j] = load_piece<TY>(row, i0 + j * kThreads * N, a.vocab);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      uint64_t s = 0;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        float l = (float)v[j][e];
        asm volatile("" : "+v"(l), "+v"(s));
        s += weight(i0 + j * kThreads * N + e, l);
      }
      s = wave_sum64(s);
      if (lane == 0) sh.waves[j][wave] = s;
    }
    lds_barrier();
    uint64_t sum = 0;
#pragma unroll 1
    for (int g = 0; g < PER * kWaves; ++g) sum += sh.waves[g / kWaves][g % kWaves];
    if (sum == 0) {  // (its mass is less than the multiples show: the largest one's slice has some)
      at = __builtin_ctzll(__ballot(rec_top == top));
      rest = 0;
      lds_barrier();
      continue;
    }
    rest = min(rest, sum - 1);
    // the round and wave that it is in
    uint64_t before = 0;
    int g = 0;
#pragma unroll 1
    for (; g < PER * kWaves - 1; ++g) {
      const uint64_t m = sh.waves[g / kWaves][g % kWaves];
      if (rest < before + m) break;
      before += m;
    }
    if (g % kWaves != wave) return;
    const int i = i0 + g / kWaves * kThreads * N;
    const V f = load_piece<TY>(row, min(i, a.vocab), a.vocab);
    uint64_t w[N], own = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) own += w[e] = weight(i + e, (float)f[e]);
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
    if (found >= 0) finish(a, b, r, found, found_l, mass_all);
    return;
  }
}

template <int TY>
hipError_t launch_typed(SampleArgs a, hipStream_t s) {
  const int slices = (a.vocab + kSampleSlice - 1) / kSampleSlice, most = kSampleSlices / slices;
  const int64_t size = dtype_bytes(TY);
  for (int rows = a.rows; rows > 0; rows -= most) {
    k_sample<TY><<<dim3((unsigned)slices, (unsigned)(rows < most ? rows : most)), kThreads, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.logits = (const uint8_t*)a.logits + most * a.row * size;
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
