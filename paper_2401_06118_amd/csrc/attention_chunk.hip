// Attention over a paged cache for many rows per sequence: chunks of a prompt.
//
// Bound: 4 operations per row, key and element of the head against 4 bytes per key
// and element, so a unit of 128 rows is bound by the matrix cores and by the
// exponentials between their two products.  A workgroup of 4 waves holds a unit
// of 128 rows, 32 a wave, and runs key tiles of 64 through two LDS stages:
// keys and values go from the pages straight into LDS
// (global_load_lds_dwordx4, a lane fetches 16 bytes of its row's page), a tile
// ahead of the one being computed.  Pages of 16 slots and more give each wave's 16
// rows of a tile one page: its address is scalar, and the loads take no vector
// instruction (594 -> 549 us in a kernel trace of the case below); smaller pages, and
// the first and last tile of a unit, look each row's page up (pages of 8 slots: 640 us).
//
// Products, 32 x 32 x 16, rows as columns of the results, so that a lane holds
// one row's weights and a row's maximum, denominator and factors need no
// exchange of lanes but one between the wave's halves:
//   S^T [key][row] = K Q^T      a lane holds 16 of 32 keys of its row
//   O^T [d][row]  += V^T P^T    the lane's keys as they are: the order of the
//                               keys inside a product is free, and V^T's
//                               fragments (ds_read_b64_tr_b16, 4 keys of a
//                               column) follow P's order
// Stage rows hold their 16-byte chunks permuted by the key, so that the fragment
// reads of 16 (keys) and 8 (values, two 32-byte blocks) rows cover all banks; the
// loads apply the permutation on the memory side.
//
// Measured: 2048 new tokens over 8192 keys, 64 heads over 8, bf16, calls back to back: 462
// to 472 us, 1020 to 1040 TFLOP/s (a library product of 8192^3 random values: 1450 here); 2048
// tokens without earlier keys 93 us.  Figures from a kernel trace are of single launches
// with a synchronize between them, which cost this case some clock: 505 to 554 us.  Heads of
// 80 and 96 elements run the form for 128: 1024 tokens over 4097 keys, 32 heads over 8: 83, 84
// and, of 128 elements, 82 us.  The matrix cores are busy 48 % of the cycles and the vector units
// most of the others; the clock gives way under the load (1.7 to 2 GHz), and
// neither priorities that set the two workgroups of a CU against each other nor more
// fragments in flight changed the time.  Running a tile's scores beside the
// exponentials of the tile before needs 32 more registers than there are
// (trace: 770 us, spilled).
//
// The sums are rescaled only where a row's maximum rises by more than 2^8: until
// then the old one stays in the exponents.  Weights are rounded once to the
// cache's type (fp16: up to 2^15, so that small ones stay normal), as the second
// product takes them; the denominator adds them up unrounded.  The error against 64
// bits grows from one rounding's 0.0017 to 0.0023 (bf16; fp16 0.00021 to 0.00027).  Weights
// in two parts, as attention_step.hip has them, would take half as many products again
// and registers that are not there.
#include "attention.h"
#include "launch.h"
#include "lds_sync.h"

namespace aqlm {

namespace {

constexpr int kWaves = 4;
constexpr int kWaveRows = 32;
constexpr int kRows = kWaves * kWaveRows;
constexpr int kTile = 64;
// Division of the work.  A unit's beginning and end cost about three tiles; a share
// has at least two tiles and that, if a unit has: smaller shares write and join
// more pieces, larger ones leave CUs idle.  A trade that no value wins everywhere (kernel
// trace; 14 sequences of 1 to 300 new tokens, 32 heads over 8, window 1024: 33.8 us with 5,
// 38.4 with 6 and 2 extra, 44 with 10 and 2; one of 20 over 1000: 25.5, 22.9, 28.7).  Pieces of a unit are joined one after
// another by the workgroup that finishes last, 64 KB each, so there are few (4
// sequences of up to 100 over 8000: 63 us with 16, 92 with 32).
constexpr int kExtra = 3;
constexpr int kLeast = 5;
constexpr int kPieces = 16;  // whole shares of a split unit (one piece more where it begins inside one)
constexpr float kLazy = 8.f;

typedef __attribute__((address_space(3))) s4_t lds_s4_t;

template <int D>
constexpr int chunk_place() { return kRows * D + 2 * kRows; }

template <int D>
struct ChunkLds {
  static constexpr int kOperand = kTile * D;           // elements
  static constexpr int kStage = 2 * kOperand;          // keys, values
  static constexpr int kFixed = 2 * kStage * 2 + 64;   // bytes, with the scratch words
};

typedef __attribute__((address_space(3))) const u32x4_t lds_v4;
typedef __attribute__((address_space(3))) u32x4_t lds_w4;
typedef const __attribute__((address_space(4))) int32_t const_i32;

// (m0, named as clobbered, is one that the compiler never keeps a value in)
#pragma clang diagnostic ignored "-Winline-asm"

// 16 bytes per lane from base + offset (bytes) into LDS at `lds` + 16 * lane, without
// a vector instruction for the address.  The compiler does not know of these
// loads in flight: a stage is read after stage_ready only, and a wait of its
// own for a vector load waits for these too, which is never too short.
__device__ __forceinline__ void load_to_lds(uint32_t lds, uint32_t offset, const uint8_t* base) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base)
               : "memory", "m0");
#endif
}
// The same from a lane's own address.
__device__ __forceinline__ void load_to_lds(uint32_t lds, const uint16_t* from) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from)
               : "memory", "m0");
#endif
}
__device__ __forceinline__ u32x4_t chunk_read(uint32_t lds) { return *(lds_v4*)(uintptr_t)lds; }
__device__ __forceinline__ u32x2_t chunk_read_tr(uint32_t lds) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_t*)(uintptr_t)lds));
#else
  return u32x2_t{};
#endif
}

// This wave's loads into LDS have landed; then every wave's have.
__device__ __forceinline__ void stage_ready() {
  __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (15 << 8));
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Chunk position of 16-byte chunk c of stage row r.
template <int D>
__device__ __forceinline__ int k_swizzle(int r) { return D == 64 ? (r >> 1) & 7 : r & 15; }
template <int D>
__device__ __forceinline__ int v_swizzle(int r) { return (D == 64 ? (r >> 1) & 3 : r & 7) * 2; }

// Exchanges x's upper half of the wave with y's lower half.
__device__ __forceinline__ void swap_halves(uint32_t& x, uint32_t& y) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
  x = r[0];
  y = r[1];
#endif
}
__device__ __forceinline__ float other_half_max(float v) {
  uint32_t x = __builtin_bit_cast(uint32_t, v), y = x;
  swap_halves(x, y);
  return fmaxf(__builtin_bit_cast(float, x), __builtin_bit_cast(float, y));
}
__device__ __forceinline__ float both_halves_sum(float v) {
  uint32_t x = __builtin_bit_cast(uint32_t, v), y = x;
  swap_halves(x, y);
  return __builtin_bit_cast(float, x) + __builtin_bit_cast(float, y);
}

// What a wave keeps of its rows.
template <int D>
struct ChunkRows {
  u32x4_t q[D / 16];
  f16_t acc[D / 32];
  float m, l;
  int lo, hi;                  // keys that this lane's row sees
  int lo_min, lo_max, hi_min, hi_max;  // over the wave's rows
};

// Loads of a tile: this lane's chunks of the wave's rows of a stage.
template <int D, bool EXACT>
struct ChunkLoad {
  static constexpr int CH = D / 8, PER = CH / kWaves, ROWS = kTile / kWaves, RPI = kWave / CH;
  const uint16_t *k, *v;  // at the head
  int row0;               // the wave's first stage row
  uint32_t at_k[PER], at_v[PER];  // bytes of the lane's chunks past the wave's first row

  // Offsets within a page, for tiles whose rows of a wave share one.
  __device__ __forceinline__ void set(const AttnArgs& a, int wave, int lane) {
    row0 = wave * ROWS;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int rl = i * RPI + lane / CH, slot = lane % CH;
      at_k[i] = (uint32_t)(rl * (int)a.k_slot + (slot ^ k_swizzle<D>(row0 + rl)) * 8) * 2;
      at_v[i] = (uint32_t)(rl * (int)a.v_slot + (slot ^ v_swizzle<D>(row0 + rl)) * 8) * 2;
    }
  }
  // The page of the wave's rows of a tile (a scalar load; used a tile later).
  __device__ __forceinline__ int page_id(const AttnArgs& a, const AttnUnit& u, int base) const {
    const int key = min(max(base + row0, u.k0), u.k1 - 1);
    return ((const_i32*)(uintptr_t)(a.block_table + u.b * a.table_stride))[key >> a.page_shift];
  }
  __device__ __forceinline__ void issue(const AttnArgs& a, const AttnUnit& u, uint32_t stage, int base, int page,
                                        int lane) const {
    const int pmask = (1 << a.page_shift) - 1;
    const uint32_t to = stage + row0 * D * 2;
    if (a.whole_rows && base >= u.k0 && base + kTile <= u.k1) {  // the wave's rows are in one page
      const int64_t id = min(max(page, 0), a.pages - 1), at = (base + row0) & pmask;
      const uint8_t* const pk = (const uint8_t*)(k + id * a.k_page + at * a.k_slot);
      const uint8_t* const pv = (const uint8_t*)(v + id * a.v_page + at * a.v_slot);
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int row = row0 + i * RPI + lane / CH, slot = lane % CH;
        const uint32_t l = to + i * (kWave * 16);
        if (EXACT || (slot ^ k_swizzle<D>(row)) * 8 < a.head_dim) load_to_lds(l, at_k[i], pk);
        if (EXACT || (slot ^ v_swizzle<D>(row)) * 8 < a.head_dim) load_to_lds(l + ChunkLds<D>::kOperand * 2, at_v[i], pv);
      }
      return;
    }
    const int ids = attn_page(a, u.b, min(max(base + row0 + (lane & (ROWS - 1)), u.k0), u.k1 - 1));
#pragma unroll 1
    for (int i = 0; i < PER; ++i) {
      const int rl = i * RPI + lane / CH, row = row0 + rl, slot = lane % CH;
      const int key = min(max(base + row, u.k0), u.k1 - 1);
      const int id = __shfl(ids, rl), at = key & pmask;
      const int ck = slot ^ k_swizzle<D>(row), cv = slot ^ v_swizzle<D>(row);
      const uint16_t* pk = k + id * a.k_page + at * a.k_slot + ck * 8;
      const uint16_t* pv = v + id * a.v_page + at * a.v_slot + cv * 8;
      const uint32_t l = to + i * (kWave * 16);
      if (EXACT || ck * 8 < a.head_dim) load_to_lds(l, pk);
      if (EXACT || cv * 8 < a.head_dim) load_to_lds(l + ChunkLds<D>::kOperand * 2, pv);
    }
  }
};

// V^T of 32 columns (block db) and 16 keys (step s), in P's key order; `at`: the
// values' LDS address plus vt_offset.
template <int D>
__device__ __forceinline__ uint32_t vt_offset(int lane) {
  const int kr = 4 * (lane >> 5) + ((lane & 15) >> 2);
  const int c = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
  return (kr * D + (c ^ v_swizzle<D>(kr)) * 8 + (lane & 1) * 4) * 2;
}
template <int D>
__device__ __forceinline__ u32x4_t read_vt(uint32_t at, int db, int s) {
  const uint32_t p = (at ^ (db * 64)) + 32 * s * D;
  const u32x2_t x = chunk_read_tr(p), y = chunk_read_tr(p + 16 * D);
  return u32x4_t{x[0], x[1], y[0], y[1]};
}

// One tile: the next tile's loads go out (into stage `wr`), then this one (stage
// `rd`, LDS addresses) is computed.
template <bool BF, int D, bool EXACT>
__device__ __forceinline__ void chunk_tile(const AttnArgs& a, const AttnUnit& u, uint32_t rd, uint32_t wr,
                                           const ChunkLoad<D, EXACT>& ld, int base, bool more, int& page, bool active,
                                           int unit_lo, int unit_hi, int* mark, int turn, ChunkRows<D>& r) {
  constexpr float kShift = BF ? 0.f : 7.f;
  const int lane = threadIdx.x & 63, half = lane >> 5, r32 = lane & 31;
  if (more) {
    ld.issue(a, u, wr, base + kTile, page, lane);
    page = ld.page_id(a, u, base + 2 * kTile);
  }
  const uint32_t vst = rd + ChunkLds<D>::kOperand * 2;

  // Values that are not finite, in tiles that some row of the unit does not see
  // all of: each wave notes which of its rows' sums become infinite (bit i of
  // `flags`: +inf, bit 16 + i: -inf), then the tile's are set to 0.  (Loops that
  // are not unrolled: this path must not cost the others registers.)
  uint32_t flags[D / 32] = {};
  bool special = false;
  if (base < unit_lo || base + kTile > unit_hi) {
    const uint32_t mine = vst + (threadIdx.x / kWave) * (kTile / kWaves) * D * 2 + lane * 16;
    constexpr int PER = kTile * D / 8 / (kWaves * kWave);
    uint32_t odd = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) odd |= non_finite_any<BF>(chunk_read(mine + i * kWave * 16));
    if (__ballot(odd != 0) != 0 && lane == 0) *mark = turn;
    lds_barrier();
    special = *mark == turn;
    if (__builtin_expect(special, 0)) {
#pragma unroll 1
      for (int d = 0; d < D / 32; ++d) {
        f16_t nu, nd;
#pragma unroll
        for (int i = 0; i < 16; ++i) nu[i] = nd[i] = 0.f;
#pragma unroll 1
        for (int st = 0; st < 4; ++st) {
          u32x4_t seen;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const int key = base + st * 16 + 8 * (w / 2) + 4 * half + 2 * (w % 2);
            seen[w] = (key >= r.lo && key < r.hi ? Bits16<BF>::kOne : 0u) |
                      (key + 1 >= r.lo && key + 1 < r.hi ? Bits16<BF>::kOne << 16 : 0u);
          }
          const u32x4_t vf = read_vt<D>(vst + vt_offset<D>(lane), d, st);
          nu = mfma32<BF>(infinite_ones<BF>(vf, 0), seen, nu);
          nd = mfma32<BF>(infinite_ones<BF>(vf, 0x10001u), seen, nd);
        }
        uint32_t f = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) f |= (nu[i] > 0.f ? 1u << i : 0u) | (nd[i] > 0.f ? 0x10000u << i : 0u);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) flags[i] = i == d ? f : flags[i];
      }
      lds_barrier();
#pragma unroll 1
      for (int i = 0; i < PER; ++i) {
        const uint32_t p = mine + i * kWave * 16;
        *(lds_w4*)(uintptr_t)p = finite_or_zero<BF>(chunk_read(p));
      }
      lds_barrier();
    }
  }
  if (!active || base >= r.hi_max || base + kTile <= r.lo_min) return;

  // Fragments are read kAhead products ahead: an LDS read takes about as long as
  // four products.
  constexpr int kAhead = 4, kSteps = D / 16;
  f16_t s[2];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
  // (the addresses of the other steps and column blocks differ from the first's by an
  // XOR, and from those of other rows by a constant of the instruction)
  uint32_t k_at = rd + (r32 * D + (half ^ k_swizzle<D>(r32)) * 8) * 2, v_at = vst + vt_offset<D>(lane);
  auto key_frag = [&](int n) {  // keys n % 2, step n / 2
    return chunk_read((k_at ^ ((n / 2) * 32)) + (n % 2) * 32 * D * 2);
  };
  u32x4_t kf[kAhead];
#pragma unroll
  for (int n = 0; n < kAhead; ++n) kf[n] = key_frag(n);
#pragma unroll
  for (int n = 0; n < 2 * kSteps; ++n) {
    s[n % 2] = mfma32<BF>(kf[n % kAhead], r.q[n / 2], s[n % 2]);
    if (n + kAhead < 2 * kSteps) kf[n % kAhead] = key_frag(n + kAhead);
  }

  const bool full = base >= r.lo_max && base + kTile <= r.hi_min;
  if (!full) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = base + b * 32 + 8 * (i / 4) + 4 * half + i % 4;
        const bool ok = key >= r.lo && key < r.hi;
        s[b][i] = ok ? s[b][i] : -INFINITY;
      }
  }
  float top = s[0][0];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
  top = other_half_max(top) * a.scale_log2;
  if (__ballot(top > r.m + kLazy) != 0) {
    const float mn = fmaxf(r.m, top);
    const float alpha = rescale(r.m - (mn == -INFINITY ? 0.f : mn));
    r.m = mn;
    r.l *= alpha;
#pragma unroll
    for (int d = 0; d < D / 32; ++d) r.acc[d] *= alpha;
  }
  u32x4_t vf[kAhead];
#pragma unroll
  for (int n = 0; n < kAhead; ++n) vf[n] = read_vt<D>(v_at, n % (D / 32), n / (D / 32));
  const float off = kShift - (r.m == -INFINITY ? 0.f : r.m);
  u32x4_t pf[4];
  float sum[2] = {0.f, 0.f};
#pragma unroll
  for (int st = 0; st < 4; ++st)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int i = (st % 2) * 8 + 2 * w;
      const float p0 = __builtin_amdgcn_exp2f(fmaf(s[st / 2][i], a.scale_log2, off));
      const float p1 = __builtin_amdgcn_exp2f(fmaf(s[st / 2][i + 1], a.scale_log2, off));
      sum[0] += p0;
      sum[1] += p1;
      pf[st][w] = pack2<BF>(p0, p1);
    }
  r.l += sum[0] + sum[1];

  constexpr int kBlocks = D / 32;
#pragma unroll
  for (int n = 0; n < 4 * kBlocks; ++n) {
    r.acc[n % kBlocks] = mfma32<BF>(vf[n % kAhead], pf[n / kBlocks], r.acc[n % kBlocks]);
    if (n + kAhead < 4 * kBlocks)
      vf[n % kAhead] = read_vt<D>(v_at, (n + kAhead) % kBlocks, (n + kAhead) / kBlocks);
  }
  if (__builtin_expect(special, 0)) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        r.acc[d][i] += (flags[d] >> i) & 1 ? INFINITY : 0.f;
        r.acc[d][i] -= (flags[d] >> (16 + i)) & 1 ? INFINITY : 0.f;
      }
  }
}

template <bool BF, int D, bool EXACT>
__global__ void __launch_bounds__(kWaves* kWave, D == 256 ? 1 : 2) k_attention_chunk(AttnArgs a) {
  constexpr float kShift = BF ? 0.f : 7.f;
  constexpr uint32_t kStageBytes = ChunkLds<D>::kStage * 2;
  extern __shared__ __align__(16) uint8_t lds[];
  uint16_t* const stages = (uint16_t*)lds;
  const uint32_t stage0 = (uint32_t)(uintptr_t)(lds_s4_t*)lds;
  int* const scratch = (int*)(lds + ChunkLds<D>::kFixed - 64);
  AttnEntry* const list = (AttnEntry*)(scratch + 16);
  const int lane = threadIdx.x & 63, half = lane >> 5, r32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int grid = gridDim.x;
  const int wg = (grid & 7) == 0 ? (blockIdx.x & 7) * (grid >> 3) + (blockIdx.x >> 3) : blockIdx.x;

  if (!EXACT) {  // the padding of heads shorter than D is never loaded
    for (int i = threadIdx.x; i < 2 * ChunkLds<D>::kStage / 8; i += kWaves * kWave)
      *(u32x4_t*)(stages + i * 8) = u32x4_t{0, 0, 0, 0};
  }
  const AttnShare h = attn_share<kRows, kTile, kExtra, kWaves>(a, list, scratch, wg, grid, kPieces, kLeast);

  if (threadIdx.x == 0) scratch[9] = 0;  // (ordered by the barriers below)
  int parity = 0, turn = 0;
  ChunkLoad<D, EXACT> ld;
  ld.set(a, wave, lane);
  // A weight that is 0 in 16 bits, times an infinite value, is a NaN that the
  // definition has not.  Tiles that all rows see are not searched for such values,
  // whose sums tell of them: a unit (or piece) with a NaN among them is run again,
  // with care.
  bool care = false;
  for (int64_t at = h.begin; at < h.end;) {
    const AttnUnit u = attn_find<kRows, kTile, kExtra>(a, h, list, at);
    const int rows = min(kRows, u.s.count * a.group - u.t * kRows);
    const int left = rows - wave * kWaveRows;  // rows of this wave
    const bool active = left > 0;
    const uint32_t first = (uint32_t)(u.t * kRows + (active ? wave * kWaveRows : 0));
    const int mine = active ? min(left, kWaveRows) : 1;
    const uint32_t rr = first + (uint32_t)min(r32, mine - 1);
    const int token = attn_token(a, (int)rr);
    const int head = u.head * a.group + (int)(rr - (uint32_t)token * (uint32_t)a.group);

    ChunkRows<D> r;
    attn_visible(a, u.s, token, r.lo, r.hi);
    attn_visible(a, u.s, attn_token(a, (int)first), r.lo_min, r.hi_min);
    attn_visible(a, u.s, attn_token(a, (int)first + mine - 1), r.lo_max, r.hi_max);
    int unit_lo, unit_hi, x;  // keys that all of the unit's rows see
    attn_visible(a, u.s, attn_token(a, u.t * kRows), x, unit_hi);
    attn_visible(a, u.s, attn_token(a, u.t * kRows + rows - 1), unit_lo, x);
    if (care) unit_lo = INT_MAX;  // search every tile
    r.m = -INFINITY;
    r.l = 0.f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) r.acc[d][i] = 0.f;

    if (u.k1 > u.k0) {
      ld.k = a.k + u.head * a.k_head;
      ld.v = a.v + u.head * a.v_head;
      int base = (u.tile0 + u.from) * kTile;
      const int end = (u.tile0 + u.to) * kTile;
      int page = ld.page_id(a, u, base);
      ld.issue(a, u, stage0 + parity * kStageBytes, base, page, lane);
      page = ld.page_id(a, u, base + kTile);
      const uint16_t* qp = a.q + (u.s.first + token) * a.q_token + head * a.q_head;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        const int c = 2 * i + half;
        const bool in = EXACT || c * 8 < a.head_dim;
        r.q[i] = attn_query(a, *(const u32x4_t*)(qp + (in ? c : 0) * 8));
        if (!in) r.q[i] = u32x4_t{0, 0, 0, 0};
      }
      for (; base < end; base += kTile) {
        stage_ready();
        chunk_tile<BF, D, EXACT>(a, u, stage0 + parity * kStageBytes, stage0 + (parity ^ 1) * kStageBytes, ld, base,
                                 base + kTile < end, page, active, unit_lo, unit_hi, scratch + 9, ++turn, r);
        parity ^= 1;
      }
      float z0 = 0.f, z1 = 0.f;  // NaN if a sum is (or if one is infinite: run again in vain)
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          z0 = fmaf(r.acc[d][i], r.acc[d][i + 1], z0);
          z1 = fmaf(r.acc[d][i + 2], r.acc[d][i + 3], z1);
        }
      const float z = z0 + z1;
      const bool bad = __ballot(z != z) != 0;
      if (lane == 0) scratch[12 + wave] = bad;
      lds_barrier();
      int again = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) again |= scratch[12 + w];
      if (__builtin_expect(!care && again != 0, 0)) {
        care = true;
        continue;
      }
    }
    r.l = both_halves_sum(r.l);

    const bool whole = u.from == 0 && u.to == u.tiles;
    bool write = whole;
    if (!whole) {
      int w0, w1;
      attn_holders(h, u, w0, w1);
      const int n = w1 - w0 + 1;
      float* const place = attn_place(a, w0, wg - w0, chunk_place<D>());
      if (active) {
        float* const o = place + wave * kWaveRows * D;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            put4(o + ((d * 4 + i) * kWave + lane) * 4,
                 f4_t{r.acc[d][4 * i], r.acc[d][4 * i + 1], r.acc[d][4 * i + 2], r.acc[d][4 * i + 3]});
        if (half == 0) put2(place + kRows * D + 2 * (wave * kWaveRows + r32), r.m, r.l);
      }
      write = attn_last(&a.counters[w0], n, scratch + 8);
      if (write) {
        if (active) {
          // in the order of the keys, this workgroup's own piece from its registers
          const int row = wave * kWaveRows + r32;
          f16_t own[D / 32];
          const float own_m = r.m, own_l = r.l;
#pragma unroll
          for (int d = 0; d < D / 32; ++d) own[d] = r.acc[d];
          r.m = -INFINITY;
          r.l = 0.f;
#pragma unroll
          for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) r.acc[d][i] = 0.f;
#pragma unroll 1
          for (int p = 0; p < n; ++p) {
            f4_t x[D / 8];
            float pm, pl;
            if (w0 + p == wg) {
#pragma unroll
              for (int i = 0; i < D / 8; ++i)
                x[i] = f4_t{own[i / 4][4 * (i % 4)], own[i / 4][4 * (i % 4) + 1], own[i / 4][4 * (i % 4) + 2],
                            own[i / 4][4 * (i % 4) + 3]};
              pm = own_m;
              pl = own_l;
            } else {
              const float* const pp = attn_place(a, w0, p, chunk_place<D>());
              const float* const o = pp + wave * kWaveRows * D + lane * 4;
#pragma unroll
              for (int i = 0; i < D / 8; ++i) x[i] = get4(o + i * kWave * 4);
              const f2_t ml = get2(pp + kRows * D + 2 * row);
              pm = ml[0];
              pl = ml[1];
            }
            const float mn = fmaxf(r.m, pm);
            const float base = mn == -INFINITY ? 0.f : mn;
            const float wa = rescale(r.m - base), wb = rescale(pm - base);
            // (a piece without keys of this row: nothing, whatever it holds; NaN scores leave
            // the maximum where it was, but not the denominator)
            const bool some = pm != -INFINITY || pl != 0.f;
            r.m = mn;
            r.l = r.l * wa + (some ? wb * pl : 0.f);
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const float y = r.acc[i / 4][4 * (i % 4) + j];
                r.acc[i / 4][4 * (i % 4) + j] = y * wa + (some ? wb * x[i][j] : 0.f);
              }
          }
        }
      }
    }
    if (write && active) {
      const float inv = r.l == 0.f ? 0.f : 1.f / r.l;
      uint16_t* const o = a.out + (u.s.first + token) * a.out_token + head * a.out_head;
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 4; i += 2) {  // blocks i and i + 1 of 8 columns, half of each in a lane
          u32x4_t w;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            uint32_t x = pack2<BF>(r.acc[d][4 * i + 2 * j] * inv, r.acc[d][4 * i + 2 * j + 1] * inv);
            uint32_t y = pack2<BF>(r.acc[d][4 * i + 4 + 2 * j] * inv, r.acc[d][4 * i + 4 + 2 * j + 1] * inv);
            if (r.l == 0.f) x = y = 0;
            swap_halves(x, y);
            w[j] = x;
            w[2 + j] = y;
          }
          const int c = d * 32 + 8 * (i + half);
          if (r32 < mine && (EXACT || c < a.head_dim)) *(u32x4_t*)(o + c) = w;
        }
      if (a.lse && half == 0 && r32 < mine)
        a.lse[(int64_t)(u.s.first + token) * (a.kv_heads * a.group) + head] =
            r.l == 0.f ? -INFINITY : (r.m - kShift + log2f(r.l)) * 0.69314718055994531f;
    }
    care = false;
    at = min(u.stop, h.end);
  }
  attn_unheld<kWaves * kWave>(a, list, wg, grid);
}

template <bool BF, int D, bool EXACT>
hipError_t launch(const AttnArgs& a, int grid, hipStream_t s) {
  constexpr auto kern = k_attention_chunk<BF, D, EXACT>;
  const hipError_t e = allow_dynamic_lds((const void*)kern, ChunkLds<D>::kFixed + (kAttnMaxSeqs + 1) * 16);
  if (e != hipSuccess) return e;
  kern<<<grid, kWaves * kWave, ChunkLds<D>::kFixed + (a.seqs + 1) * 16, s>>>(a);
  return hipGetLastError();
}

template <bool BF, int D>
hipError_t launch(const AttnArgs& a, int grid, hipStream_t s) {
  return a.head_dim == D ? launch<BF, D, true>(a, grid, s) : launch<BF, D, false>(a, grid, s);
}

}  // namespace

int attention_chunk_grid(int head_dim) { return (attention_dim(head_dim) == 256 ? 1 : 2) * num_cus(); }
int64_t attention_chunk_place(int head_dim) { return (int64_t)kRows * (attention_dim(head_dim) + 2); }

hipError_t launch_attention_chunk(const AttnArgs& a, bool bf, int grid, hipStream_t s) {
  switch (attention_dim(a.head_dim)) {
    case 64: return bf ? launch<true, 64>(a, grid, s) : launch<false, 64>(a, grid, s);
    case 128: return bf ? launch<true, 128>(a, grid, s) : launch<false, 128>(a, grid, s);
    default: return bf ? launch<true, 256>(a, grid, s) : launch<false, 256>(a, grid, s);
  }
}

}  // namespace aqlm
