// Attention over a paged key/value cache: arguments, the division of the work
// over workgroups, and the joining of split rows, shared by the kernel for a few
// rows per sequence (attention_step.hip) and the one for many
// (attention_chunk.hip).
//
//   out[t][e] = sum_j p_j V[j] / sum_j p_j,   p_j = exp(scale <q[t][e], K[j]>)
//
// over the keys j that token t may see, with the running maximum taken out of
// the exponents.  The query heads e of one kv head h share its keys, so a
// sequence's new tokens and those heads are packed into rows (row r: token
// r / group, head h * group + r % group) and the rows are cut into units of R.
// A unit reads the key tiles between the first key that its first token sees
// and the last one that its last token sees.
//
// Division of the work.  Lengths live on the device (a captured launch serves
// any lengths), so every workgroup adds up the tiles of all units by itself,
// and takes an equal, contiguous share of the sequence (kv head, sequence,
// unit, tile), where a unit counts as EXTRA tiles more than it has: what its
// beginning and end cost.  A share may hold many short units, or a piece of a long one.  A
// workgroup that holds a whole unit writes its rows.  The pieces of a split one
// (unnormalised sums, maximum, denominator, all fp32) go to the workspace, where
// a workgroup has two places: one for the unit that it continues, one for the
// unit that it begins.  The workgroup that finishes a unit's last piece (a
// counter per beginning workgroup) adds the pieces up in the order of the
// keys, so results do not depend on the order in which workgroups run, and sets
// the counter back to zero for the next launch.
#pragma once

#include <limits.h>

#include "attention_rows.h"
#include "common.h"

namespace aqlm {

typedef float f16_t __attribute__((ext_vector_type(16)));
typedef __bf16 b8_t __attribute__((ext_vector_type(8)));
typedef __bf16 b2_t __attribute__((ext_vector_type(2)));
typedef float f2_t __attribute__((ext_vector_type(2)));
typedef short s4_t __attribute__((ext_vector_type(4)));

constexpr int kAttnMaxSeqs = 2032;  // (their entries and two stages of 256-element heads fill the LDS)

struct AttnArgs {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* out;
  float* lse;  // [tokens][kv_heads * group] or null
  const int32_t* block_table;
  const int32_t* kv_lens;
  const int32_t* cu_new;
  uint32_t* counters;  // [grid]
  float* parts;        // [2 * grid] places
  int64_t q_token, q_head, out_token, out_head;  // strides, in elements
  int64_t k_page, k_slot, k_head, v_page, v_slot, v_head;
  int64_t table_stride;
  int32_t tokens, seqs, kv_heads, group, head_dim;
  uint32_t group_mul, group_shift;  // row / group = hi32(row * group_mul) >> group_shift (group_mul 0: row)
  int32_t pages, page_shift, table_width;
  int32_t causal, window;
  int32_t whole_rows;  // 16 aligned keys share a page, their offsets in it fit 31 bits
  // |scale| * log2(e), above 0 (so that a masked score stays -inf under it); the
  // queries are read as (q & q_keep) ^ q_flip, which brings in the sign, and a
  // scale of 0 as queries of 0.
  float scale_log2;
  uint32_t q_keep, q_flip;
};

__device__ __forceinline__ u32x4_t attn_query(const AttnArgs& a, const u32x4_t& q) {
  u32x4_t r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (q[i] & a.q_keep) ^ a.q_flip;
  return r;
}

// Sequence b by itself; `falls` is set where its offsets do.
__device__ __forceinline__ AttnSeq attn_seq(const AttnArgs& a, int b, bool& falls) {
  const int cu0 = a.cu_new[b], cu1 = a.cu_new[b + 1];
  falls |= cu1 < cu0;
  return attn_cut(cu0, cu1, a.kv_lens[b], a.tokens, (int64_t)a.table_width << a.page_shift);
}

// The token of a sequence's row (rows are below 2^31).
__device__ __forceinline__ int attn_token(const AttnArgs& a, int row) {
  return a.group_mul == 0 ? row : (int)(__umulhi((uint32_t)row, a.group_mul) >> a.group_shift);
}

// Keys [lo, hi) that token i of a sequence sees (hi <= lo: none).
__device__ __forceinline__ void attn_visible(const AttnArgs& a, const AttnSeq& s, int i, int& lo, int& hi) {
  const int pos = s.keys - s.count + i;
  hi = a.causal ? min(pos + 1, s.keys) : s.keys;
  lo = a.window > 0 ? (int)max((int64_t)0, (int64_t)pos - a.window + 1) : 0;
}

// Key tiles of KT of unit t: the first one and their number (at least one, so
// that some workgroup writes the rows of a unit without keys).
template <int R, int KT>
__device__ __forceinline__ int attn_tiles(const AttnArgs& a, const AttnSeq& s, int t, int& tile0, int& k0, int& k1) {
  int lo, hi, x;
  attn_visible(a, s, attn_token(a, t * R), lo, x);
  attn_visible(a, s, min(s.count - 1, attn_token(a, t * R + R - 1)), x, hi);
  k0 = lo;
  k1 = max(hi, lo);
  tile0 = lo / KT;
  return hi > lo ? (hi + KT - 1) / KT - tile0 : 1;
}

__device__ __forceinline__ int attn_units(const AttnArgs& a, const AttnSeq& s, int R) {
  return (int)(((int64_t)s.count * a.group + R - 1) / R);
}

// Inclusive prefix sums over the wave, and maxima of values of 0 and more, by moves
// between lanes (shuffles go through the LDS).
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_or_0(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ int wave_scan(int v) {
  v += dpp_or_0<0x111, 0xF>(v);  // row_shr 1, 2, 4, 8
  v += dpp_or_0<0x112, 0xF>(v);
  v += dpp_or_0<0x114, 0xF>(v);
  v += dpp_or_0<0x118, 0xF>(v);
  v += dpp_or_0<0x142, 0xA>(v);  // row_bcast 15, 31
  v += dpp_or_0<0x143, 0xC>(v);
  return v;
}
__device__ __forceinline__ int wave_scan_most(int v) {
  v = max(v, dpp_or_0<0x111, 0xF>(v));
  v = max(v, dpp_or_0<0x112, 0xF>(v));
  v = max(v, dpp_or_0<0x114, 0xF>(v));
  v = max(v, dpp_or_0<0x118, 0xF>(v));
  v = max(v, dpp_or_0<0x142, 0xA>(v));
  v = max(v, dpp_or_0<0x143, 0xC>(v));
  return v;
}
__device__ __forceinline__ int wave_most(int v) { return __builtin_amdgcn_readlane(wave_scan_most(v), kWave - 1); }

// A sequence in LDS: the cost of one kv head before it, and what it holds.
struct __align__(16) AttnEntry {
  int before, first, count, keys;
};

// Entries whose offsets fall somewhere: each keeps what those before it leave
// (attn_after).  One wave runs it.
__device__ __forceinline__ void attn_apart(const AttnArgs& a, AttnEntry* list) {
  const int lane = threadIdx.x & (kWave - 1);
  int end = 0;
  for (int b = 0; b < a.seqs; b += kWave) {
    const int i = b + lane;
    AttnSeq s = {0, 0, 0};
    if (i < a.seqs) s = {list[i].first, list[i].count, list[i].keys};
    const int ends = wave_scan_most(s.first + s.count);
    const int others = __shfl_up(ends, 1);
    s = attn_after(s, lane > 0 ? max(end, others) : end);
    if (i < a.seqs) {
      list[i].first = s.first;
      list[i].count = s.count;
    }
    end = max(end, __builtin_amdgcn_readlane(ends, kWave - 1));
  }
}

struct AttnShare {
  int per_head;    // cost of one kv head over all sequences
  int64_t total;   // cost of all heads
  int64_t quota;   // cost of a workgroup's share
  int64_t slack;   // how far an end of a share moves to an end of a unit
  int64_t begin, end;
};

struct AttnUnit;
template <int R, int KT, int EXTRA>
__device__ __forceinline__ AttnUnit attn_find(const AttnArgs& a, const AttnShare& h, const AttnEntry* list, int64_t at);

// One unit of a share: where it is, and the part of its tiles that the share holds.
struct AttnUnit {
  AttnSeq s;
  int b, head, t;
  int tile0, tiles, k0, k1;
  int from, to;         // tiles [from, to) of the unit are in the share
  int64_t start, stop;  // where the unit's cost is in the sequence of all
};

// Unit i of a sequence in the order first, last, second, last but one, ...
__device__ __forceinline__ int attn_folded(int i, int units) { return (i & 1) == 0 ? i / 2 : units - 1 - i / 2; }

// Fills `list` (LDS, seqs + 1 entries; `scratch`: two ints per wave) and returns this
// workgroup's share.  `pieces`: the most whole shares that a unit is split
// into; `least`: the least cost of a share, if a unit has that much.
template <int R, int KT, int EXTRA, int WAVES>
__device__ __forceinline__ AttnShare attn_share(const AttnArgs& a, AttnEntry* list, int* scratch, int wg, int grid,
                                                int pieces, int least) {
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  int most = 1, tile0, k0, k1;
  // a thread per sequence; those of several units are left to a wave each
  bool many = false, falls = false;
  auto enter = [&](int b, const AttnSeq& s) {
    const int units = attn_units(a, s, R);
    int cost = 0;
    if (units == 1) cost = attn_tiles<R, KT>(a, s, 0, tile0, k0, k1) + EXTRA;
    most = max(most, cost);
    many |= units > 1;
    list[b] = AttnEntry{units > 1 ? -1 : cost, s.first, s.count, s.keys};
  };
  // what any thread found: 1 sequences of several units, 2 offsets that fall
  auto found = [&]() {
    const int mine = (__ballot(many) != 0 ? 1 : 0) | (__ballot(falls) != 0 ? 2 : 0);
    if (lane == 0) scratch[WAVES + wave] = mine;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) all |= scratch[WAVES + w];
    return all;
  };
  for (int b = tid; b < a.seqs; b += WAVES * kWave) enter(b, attn_seq(a, b, falls));
  int marked = found();
  if (__builtin_expect((marked & 2) != 0, 0)) {
    if (wave == 0) attn_apart(a, list);
    __syncthreads();
    most = 1;
    many = falls = false;
    for (int b = tid; b < a.seqs; b += WAVES * kWave)
      enter(b, AttnSeq{list[b].first, list[b].count, list[b].keys});
    marked = found();
  }
  if (marked != 0) {
    for (int i = 0; i < a.seqs; i += kWave) {
      uint64_t left = __ballot(i + lane < a.seqs && list[i + lane].before == -1);
      __syncthreads();  // (every wave has read the marks before one is replaced)
      for (int n = 0; left != 0; ++n, left &= left - 1) {
        if (n % WAVES != wave) continue;
        const int b = i + __builtin_ctzll(left);
        const AttnSeq s = {list[b].first, list[b].count, list[b].keys};
        const int units = attn_units(a, s, R);
        int sum = 0;
        for (int t = lane; t < units; t += kWave) {
          const int cost = attn_tiles<R, KT>(a, s, t, tile0, k0, k1) + EXTRA;
          sum += cost;
          most = max(most, cost);
        }
        sum = wave_scan(sum);
        if (lane == kWave - 1) list[b].before = sum;
      }
    }
  }
  most = wave_most(most);
  if (lane == 0) scratch[wave] = most;
  if (marked != 0) __syncthreads();
  if (wave == 0) {  // costs to the costs before
    int before = 0;
    for (int b = 0; b < a.seqs; b += kWave) {
      const int i = b + lane;
      const int cost = i < a.seqs ? list[i].before : 0;
      const int incl = wave_scan(cost) + before;
      if (i < a.seqs) list[i].before = incl - cost;
      before = __builtin_amdgcn_readlane(incl, kWave - 1);
    }
    if (lane == 0) list[a.seqs].before = before;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) most = max(most, scratch[w]);
  AttnShare h;
  h.per_head = list[a.seqs].before;
  h.total = (int64_t)h.per_head * a.kv_heads;
  h.quota = max((h.total + grid - 1) / grid, (int64_t)((most + pieces - 1) / pieces));
  h.quota = max(h.quota, (int64_t)min(least, most));
  h.slack = max(h.quota / 8, (int64_t)EXTRA);  // (a piece has a tile at least)
  h.begin = min(h.total, h.quota * wg);
  h.end = min(h.total, h.begin + h.quota);
  if (h.slack > 0) {
    const int64_t last = h.end;
    auto moved = [&](int64_t x) {
      if (x == 0 || x >= h.total) return x;
      const AttnUnit u = attn_find<R, KT, EXTRA>(a, h, list, x);
      if (x - u.start <= h.slack) return u.start;
      return u.stop - x <= h.slack ? u.stop : x;
    };
    h.end = moved(last);
    h.begin = h.begin < last ? moved(h.begin) : h.end;
  }
  return h;
}

// The workgroups that hold the first and the last piece of a unit.
__device__ __forceinline__ void attn_holders(const AttnShare& h, const AttnUnit& u, int& w0, int& w1) {
  w0 = (int)((u.start + h.slack) / h.quota);
  w1 = max(w0, (int)((u.stop - h.slack - 1) / h.quota));
}

// The place of piece p of a unit: of the unit that its workgroup begins (the
// first piece) or continues.
__device__ __forceinline__ float* attn_place(const AttnArgs& a, int w0, int p, int64_t floats) {
  return a.parts + (2 * (int64_t)(w0 + p) + (p == 0 ? 1 : 0)) * floats;
}

// Written through to memory, and read from there.
__device__ __forceinline__ void put2(float* p, float x, float y) {
  const u32x2_t w = {__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, y)};
  __hip_atomic_store((uint64_t*)p, __builtin_bit_cast(uint64_t, w), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f2_t get2(const float* p) {
  return __builtin_bit_cast(f2_t, __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
__device__ __forceinline__ void put4(float* p, const f4_t& v) {
#if defined(__HIP_DEVICE_COMPILE__)
  // one 16-byte store; the pause keeps its data registers as they are until it
  // has read them (attn_last waits for it to reach memory)
  asm volatile("global_store_dwordx4 %0, %1, off sc1\n\ts_nop 1" ::"v"(p), "v"(v) : "memory");
#endif
}
__device__ __forceinline__ f4_t get4(const float* p) {
  const f2_t x = get2(p), y = get2(p + 2);
  return f4_t{x[0], x[1], y[0], y[1]};
}

// After a workgroup's stores of a piece: true in the workgroup that wrote the last
// of a unit's pieces (`count` of them).  Its stores have reached memory before the
// counter moves.  `flag`: an LDS word.
__device__ __forceinline__ bool attn_last(uint32_t* counter, int count, int* flag) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const bool last =
        __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(count - 1);
    if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *flag = last;
  }
  __syncthreads();
  return *flag != 0;
}

// The unit that holds `at` of the sequence of all costs.  Uniform over the
// workgroup; every wave finds it by itself.
template <int R, int KT, int EXTRA>
__device__ __forceinline__ AttnUnit attn_find(const AttnArgs& a, const AttnShare& h, const AttnEntry* list,
                                              int64_t at) {
  const int lane = threadIdx.x & (kWave - 1);
  AttnUnit u;
  u.head = a.kv_heads == 1 ? 0 : (int)(at / h.per_head);
  const int rem = (int)(at - (int64_t)u.head * h.per_head);
  // the last sequence that begins at or before (empty ones have no cost)
  int b = 0;
  for (int i = 0; i < a.seqs; i += kWave) {
    const uint64_t le = __ballot(i + lane < a.seqs && list[i + lane].before <= rem);
    if (le == 0) break;
    b = i + 63 - __builtin_clzll(le);
  }
  u.b = __builtin_amdgcn_readfirstlane(b);
  const AttnEntry e = list[u.b];
  u.s.first = __builtin_amdgcn_readfirstlane(e.first);
  u.s.count = __builtin_amdgcn_readfirstlane(e.count);
  u.s.keys = __builtin_amdgcn_readfirstlane(e.keys);
  int left = rem - e.before;
  const int units = attn_units(a, u.s, R);
  int tile0, k0, k1, t = 0;
  if (units > 1) {
    int before = 0;
    for (int i = 0; i < units; i += kWave) {
      const int n = i + lane < units ? attn_tiles<R, KT>(a, u.s, attn_folded(i + lane, units), tile0, k0, k1) + EXTRA : 0;
      const int incl = wave_scan(n) + before;
      const uint64_t gt = __ballot(incl > left);
      if (gt != 0) {
        const int l = __builtin_ctzll(gt);
        t = attn_folded(i + l, units);
        before = l > 0 ? __builtin_amdgcn_readlane(incl, l - 1) : before;
        break;
      }
      before = __builtin_amdgcn_readlane(incl, kWave - 1);
    }
    left -= before;
  }
  u.t = __builtin_amdgcn_readfirstlane(t);
  u.tiles = attn_tiles<R, KT>(a, u.s, u.t, u.tile0, u.k0, u.k1);
  left = __builtin_amdgcn_readfirstlane(left);
  u.start = at - left;
  u.stop = u.start + u.tiles + EXTRA;
  u.from = max(0, left - EXTRA);
  u.to = (int)min((int64_t)u.tiles, h.end - u.start - EXTRA);
  return u;
}

// Rows of tokens that no sequence holds (the sequences' tokens are one run): zeros, as
// rows without keys.
template <int THREADS>
__device__ __forceinline__ void attn_unheld(const AttnArgs& a, const AttnEntry* list, int wg, int grid) {
  const int begin = list[0].first, end = list[a.seqs - 1].first + list[a.seqs - 1].count;
  if (end - begin == a.tokens) return;
  const int heads = a.kv_heads * a.group, pieces = a.head_dim / 8;
  const int64_t rows = (int64_t)(a.tokens - (end - begin)) * heads;
  for (int64_t i = (int64_t)wg * THREADS + threadIdx.x; i < rows * pieces; i += (int64_t)grid * THREADS) {
    const int64_t row = i / pieces;
    const int t = (int)(row / heads), head = (int)(row - (int64_t)t * heads), piece = (int)(i - row * pieces);
    const int token = t < begin ? t : t + (end - begin);
    *(u32x4_t*)(a.out + token * a.out_token + head * a.out_head + piece * 8) = u32x4_t{0, 0, 0, 0};
    if (piece == 0 && a.lse) a.lse[(int64_t)token * heads + head] = -INFINITY;
  }
}

// The page of key j of sequence b, kept inside the cache.
__device__ __forceinline__ int attn_page(const AttnArgs& a, int b, int j) {
  const int p = a.block_table[b * a.table_stride + (j >> a.page_shift)];
  return min(max(p, 0), a.pages - 1);
}

// fp32 to the cache's type, two at a time, and the types' products.
template <bool BF>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  if constexpr (BF) {
    const b2_t r = {(__bf16)x, (__bf16)y};
    return __builtin_bit_cast(uint32_t, r);
  } else {
    const h2_t r = {(_Float16)x, (_Float16)y};
    return __builtin_bit_cast(uint32_t, r);
  }
}
template <bool BF>
__device__ __forceinline__ float low_of(uint32_t w) {
  if constexpr (BF) return __builtin_bit_cast(float, w << 16);
  return (float)as_h2(w)[0];
}
template <bool BF>
__device__ __forceinline__ float high_of(uint32_t w) {
  if constexpr (BF) return __builtin_bit_cast(float, w & 0xFFFF0000u);
  return (float)as_h2(w)[1];
}
template <bool BF>
__device__ __forceinline__ f4_t mfma16(const u32x4_t& x, const u32x4_t& y, const f4_t& c) {
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8_t, x), __builtin_bit_cast(b8_t, y), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8_t, x), __builtin_bit_cast(h8_t, y), c, 0, 0, 0);
#else
  return c;
#endif
}
template <bool BF>
__device__ __forceinline__ f16_t mfma32(const u32x4_t& x, const u32x4_t& y, const f16_t& c) {
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8_t, x), __builtin_bit_cast(b8_t, y), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8_t, x), __builtin_bit_cast(h8_t, y), c, 0, 0, 0);
#else
  return c;
#endif
}

// Factor of sums whose maximum rises by -x (log2).  Never 0, so that an infinite
// sum stays what it is; finite ones vanish either way.
__device__ __forceinline__ float rescale(float x) { return fmaxf(__builtin_amdgcn_exp2f(x), 1e-30f); }

// Values that are not finite.  A masked key has weight 0, and 0 times an
// infinite or NaN value would be NaN in rows that do not see the key.  Where some
// row does not see some key of a tile, a tile with such values takes the values
// as 0 in the product, and rows that do see one get it by another: the number
// of +inf (or NaN) and of -inf (or NaN) values that a row sees, from 0/1 weights
// and 0/1 values, exactly.
template <bool BF>
struct Bits16 {
  static constexpr uint32_t kExp = BF ? 0x7F80u : 0x7C00u;
  static constexpr uint32_t kOne = BF ? 0x3F80u : 0x3C00u;
};
// Bit 15 and bit 31: halves with all exponent bits set.
template <bool BF>
__device__ __forceinline__ uint32_t non_finite(uint32_t w) {
  constexpr uint32_t e = Bits16<BF>::kExp, low = e & (~e + 1);
  return ((w & (e * 0x10001u)) + low * 0x10001u) & 0x80008000u;
}
template <bool BF>
__device__ __forceinline__ uint32_t non_finite_any(const u32x4_t& f) {
  return non_finite<BF>(f[0]) | non_finite<BF>(f[1]) | non_finite<BF>(f[2]) | non_finite<BF>(f[3]);
}
template <bool BF>
__device__ __forceinline__ u32x4_t finite_or_zero(const u32x4_t& f) {
  u32x4_t r;
#pragma unroll
  for (int w = 0; w < 4; ++w) r[w] = f[w] & ~((non_finite<BF>(f[w]) >> 15) * 0xFFFFu);
  return r;
}
// 1 for halves that are +inf or NaN (`sign` 0x10001: -inf or NaN), else 0.
template <bool BF>
__device__ __forceinline__ u32x4_t infinite_ones(const u32x4_t& f, uint32_t sign) {
  constexpr uint32_t e = Bits16<BF>::kExp, mant = ~e & 0x7FFFu;
  u32x4_t r;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint32_t odd = non_finite<BF>(f[w]) >> 15;
    const uint32_t nan = (((f[w] & (mant * 0x10001u)) + mant * 0x10001u) / (mant + 1)) & 0x10001u;
    r[w] = (odd & (nan | ~((f[w] >> 15) ^ sign))) * Bits16<BF>::kOne;
  }
  return r;
}
// Adds +inf where a row sees such values (counts nu), -inf likewise (nd).
template <typename V>
__device__ __forceinline__ void add_infinities(V& acc, const V& nu, const V& nd) {
#pragma unroll
  for (int i = 0; i < (int)(sizeof(V) / 4); ++i) {
    acc[i] += nu[i] > 0.f ? INFINITY : 0.f;
    acc[i] -= nd[i] > 0.f ? INFINITY : 0.f;
  }
}

hipError_t launch_attention_step(const AttnArgs& a, bool bf, int grid, hipStream_t s);
hipError_t launch_attention_chunk(const AttnArgs& a, bool bf, int grid, hipStream_t s);
// The padded head size a kernel runs (64, 128 or 256), workgroups per launch and
// floats of a workspace place.
inline int attention_dim(int head_dim) { return head_dim <= 64 ? 64 : (head_dim <= 128 ? 128 : 256); }
int attention_step_grid();
int attention_chunk_grid(int head_dim);
int64_t attention_step_place(int head_dim);
int64_t attention_chunk_place(int head_dim);

}  // namespace aqlm
