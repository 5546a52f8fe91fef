// Attention over a paged cache for a few rows per sequence: a decode step, or
// short drafts (new tokens times heads per kv head up to 16 rows a unit).
//
// Bound: the keys and values are read once, 4 bytes of them per 8 operations and
// row; memory bandwidth is the limit up to 16 rows.  A workgroup of 4 waves runs
// key tiles of 128, 32 keys a wave, without a barrier inside a unit: every wave
// keeps its own maximum, denominator and sums, joined through LDS when the unit
// (or the workgroup's piece of it) ends.
//
// Products on the matrix cores, 16 x 16 x 32, rows as columns of the results:
//   S^T [key][row] = K Q^T     lane: key = lane % 16, 8 elements of the head;
//                              loaded from memory straight into the fragment
//   O^T [d][row]  += V^T P^T   the lanes that hold S^T for keys 4g..4g+3 of two
//                              16-key blocks use them as the 8 reduction
//                              elements of P^T: the order of the keys inside a
//                              product is free, so P needs no exchange of lanes
// V^T needs 4 keys of one column in a lane: the wave's 32 keys go through LDS and
// come back with the transposing load (ds_read_b64_tr_b16).  Its 32-byte column
// blocks are permuted by the key, so that the 16 rows of a load hit all banks.
//
// A weight p is rounded to two 16-bit parts (the value and what its rounding
// left), two products each: the matrix cores idle here, and the result carries
// one 16-bit rounding instead of two.
//
// Measured, calls back to back: 64 sequences of up to 16000 keys, 64 heads over 8, bf16
// (767 MB): 155 us, 4.9 TB/s; all of 5000 keys 231 us, 5.7 TB/s; traffic as counted is the
// keys and values once.  One sequence of 1024 keys, 32 heads (17 MB): 13.9 us, of which
// about 3 are the launch, 3 the division of the work, 3 the joining of pieces and
// the rest the chain of page number, keys, values.  Heads of 80 and 96 elements run the
// form for 128, whose lanes past the head load its first 16 bytes again: 32 sequences of 4000
// keys, 32 heads over 8 (328 and 393 MB) 84 and 87 us; of 128 elements (525 MB) 103.
//
// The next tile's keys are loaded into the registers of this one's as soon as
// S^T is done, its values as soon as these are in LDS, and the page numbers one
// tile ahead: 16 KB a wave in flight at 128 elements a head.
#include "attention.h"
#include "launch.h"

namespace aqlm {

namespace {

constexpr int kRows = 16;
constexpr int kWaves = 4;
constexpr int kWaveKeys = 32;
constexpr int kTile = kWaves * kWaveKeys;
// Division of the work: a share may be one tile (one sequence of 1024 keys, 32 heads:
// 14.0 us; two tiles at least: 16.5), and a unit many pieces, which the last of its
// workgroups reads (one of 60001 keys, 8 heads over one: 43.8 us with 64, 55 with 16,
// 57 with 256; single launches, kernel trace).
constexpr int kExtra = 0;
constexpr int kLeast = 1;
constexpr int kPieces = 64;  // whole shares of a split unit (one piece more where it begins inside one)

typedef __attribute__((address_space(3))) s4_t lds_s4_t;

template <int D>
struct StepLds {
  static constexpr int kPitch = D + 4;  // floats per row of the joined sums
  static constexpr int kStage = kWaves * kWaveKeys * D * 2;
  static constexpr int kJoin = kWaves * kRows * (kPitch + 2) * 4;
  static constexpr int kUnion = kStage > kJoin ? kStage : kJoin;
  static constexpr int kFixed = kUnion + 64;  // + scratch: waves' maxima, the "last" flag, waves' sums that are not finite
};

template <int D>
constexpr int step_place() { return kRows * (D + 2); }

// 4 keys of one column (16 lanes: 4 keys x 16 columns).
__device__ __forceinline__ s4_t read_tr(const uint16_t* l) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_t*)l);
#else
  return s4_t{};
#endif
}

// LDS element offset of 16-byte chunk c of key row r: 32-byte blocks permuted so
// that rows 4g..4g+3 (g = 0..3) of one column block cover all banks.
template <int D>
__device__ __forceinline__ int v_pos(int r, int c) {
  const int sw = D == 64 ? (r >> 1) & 3 : r & 7;
  return r * D + (((c >> 1) ^ sw) * 2 + (c & 1)) * 8;
}

// V^T of column block d (16 columns): keys 4g..4g+3 of both 16-key blocks.  Lane i
// of each 16 addresses key 4g + i / 4, 8 bytes i % 4.
template <int D>
__device__ __forceinline__ u32x4_t read_vt(const uint16_t* stage, int d, int g, int r16) {
  u32x4_t f;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int kr = b * 16 + 4 * g + (r16 >> 2);
    const u32x2_t w =
        __builtin_bit_cast(u32x2_t, read_tr(stage + v_pos<D>(kr, 2 * d + ((r16 & 3) >> 1)) + (r16 & 1) * 4));
    f[2 * b] = w[0];
    f[2 * b + 1] = w[1];
  }
  return f;
}

// Order of a wave's own LDS stores and loads (the LDS keeps a wave's accesses in
// order; the compiler has to as well).
__device__ __forceinline__ void wave_lds_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

template <bool BF, int D, bool EXACT>
__global__ void __launch_bounds__(kWaves* kWave, D == 256 ? 1 : 2) k_attention_step(AttnArgs a) {
  constexpr int NS = D / 32, NV = D / 16, CH = D / 8, ND = D / 16;
  constexpr float kShift = BF ? 0.f : 14.f;  // fp16: weights up to 2^14, so that small ones stay normal
  extern __shared__ __align__(16) uint8_t lds[];
  int* const scratch = (int*)(lds + StepLds<D>::kUnion);
  AttnEntry* const list = (AttnEntry*)(scratch + 16);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;
  const int grid = gridDim.x;
  const int wg = (grid & 7) == 0 ? (blockIdx.x & 7) * (grid >> 3) + (blockIdx.x >> 3) : blockIdx.x;
  uint16_t* const stage = (uint16_t*)lds + wave * kWaveKeys * D;
  float* const join = (float*)lds;
  float* const join_m = join + kWaves * kRows * StepLds<D>::kPitch;  // [wave][row] maxima, then denominators
  const int pmask = (1 << a.page_shift) - 1;

  const AttnShare h = attn_share<kRows, kTile, kExtra, kWaves>(a, list, scratch, wg, grid, kPieces, kLeast);

  // A weight's second part is 0 or below for some keys, and a weight may be 0 in 16
  // bits: times an infinite value either gives a NaN that the definition has not.
  // Tiles that all rows see are not searched for such values, whose sums tell of
  // them: a unit (or piece) with one that is not finite is run again, with care.
  bool care = false;
  for (int64_t at = h.begin; at < h.end;) {
    const AttnUnit u = attn_find<kRows, kTile, kExtra>(a, h, list, at);
    const int rows = min(kRows, u.s.count * a.group - u.t * kRows);
    const uint32_t rr = (uint32_t)(u.t * kRows + min(r16, rows - 1));
    const int token = attn_token(a, (int)rr);
    const int head = u.head * a.group + (int)(rr - (uint32_t)token * (uint32_t)a.group);
    int lo, hi, lo_max, hi_min, x;
    attn_visible(a, u.s, token, lo, hi);
    attn_visible(a, u.s, attn_token(a, u.t * kRows), x, hi_min);
    attn_visible(a, u.s, attn_token(a, u.t * kRows + rows - 1), lo_max, x);

    // elements past the head (its padding to D): zeros in q and k; v's only
    // reach sums that are not written
    auto inside = [&](int c) { return EXACT || c * 8 < a.head_dim; };
    auto chunk = [&](int c) { return inside(c) ? c : 0; };
    u32x4_t qf[NS];
    const uint16_t* qp = a.q + (u.s.first + token) * a.q_token + head * a.q_head;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const int c = 4 * s + g;
      qf[s] = attn_query(a, *(const u32x4_t*)(qp + chunk(c) * 8));
      if (!inside(c)) qf[s] = u32x4_t{0, 0, 0, 0};
    }

    f4_t acc[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i) acc[i] = f4_t{0, 0, 0, 0};
    float m = -INFINITY, l = 0.f;

    // the wave's first key and the end of its keys, in steps of a tile
    const int end = min(u.k1, (u.tile0 + u.to) * kTile);
    int kb = (u.tile0 + u.from) * kTile + wave * kWaveKeys;
    if (kb + kWaveKeys <= u.k0) kb += kTile;
    const uint16_t* const kbase = a.k + u.head * a.k_head;
    const uint16_t* const vbase = a.v + u.head * a.v_head;

    auto key_at = [&](int j) { return min(max(j, u.k0), u.k1 - 1); };
    auto page_ids = [&](int base) { return attn_page(a, u.b, key_at(base + (lane & 31))); };
    auto load_k = [&](u32x4_t (&t)[2][NS], int base, int ids) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int key = key_at(base + b * 16 + r16);
        const uint16_t* p = kbase + __shfl(ids, b * 16 + r16) * a.k_page + (key & pmask) * a.k_slot;
#pragma unroll
        for (int s = 0; s < NS; ++s) t[b][s] = *(const u32x4_t*)(p + chunk(4 * s + g) * 8);
      }
    };
    auto load_v = [&](u32x4_t (&t)[NV], int base, int ids) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int kl = i * (kWave / CH) + lane / CH, c = lane % CH;
        const int key = key_at(base + kl);
        const uint16_t* p = vbase + __shfl(ids, kl) * a.v_page + (key & pmask) * a.v_slot;
        t[i] = *(const u32x4_t*)(p + chunk(c) * 8);
      }
    };

    if (kb < end) {
      u32x4_t kt[2][NS], vt[NV];
      int ids = page_ids(kb);
      load_k(kt, kb, ids);
      load_v(vt, kb, ids);
      ids = page_ids(kb + kTile);
      for (; kb < end; kb += kTile) {
        const bool more = kb + kTile < end;
        f4_t s[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          s[b] = f4_t{0, 0, 0, 0};
#pragma unroll
          for (int i = 0; i < NS; ++i) {
            if (!inside(4 * i + g)) kt[b][i] = u32x4_t{0, 0, 0, 0};
            s[b] = mfma16<BF>(kt[b][i], qf[i], s[b]);
          }
        }
        if (more) load_k(kt, kb + kTile, ids);

        const bool full = kb >= lo_max && kb + kWaveKeys <= hi_min;
        uint32_t vis = 0xFF;
        if (!full) {
          vis = 0;
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = kb + b * 16 + 4 * g + i;
              const bool ok = key >= lo && key < hi;
              vis |= (uint32_t)ok << (b * 4 + i);
              s[b][i] = ok ? s[b][i] : -INFINITY;
            }
        }
        float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                          fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float mn = fmaxf(m, top * a.scale_log2);
        const float base = mn == -INFINITY ? 0.f : mn;
        const float alpha = rescale(m - base);
        m = mn;
        const float off = kShift - base;
        u32x4_t ph, pl;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(s[w / 2][(w % 2) * 2], a.scale_log2, off));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(s[w / 2][(w % 2) * 2 + 1], a.scale_log2, off));
          sum += p0 + p1;
          ph[w] = pack2<BF>(p0, p1);
          pl[w] = pack2<BF>(p0 - low_of<BF>(ph[w]), p1 - high_of<BF>(ph[w]));
        }
        l = l * alpha + sum;
#pragma unroll
        for (int d = 0; d < ND; ++d) acc[d] *= alpha;

        bool special = false;
        if (!full || care) {
          // values of keys outside the unit's range count as zeros
          uint32_t odd = 0;
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            const int key = kb + i * (kWave / CH) + lane / CH;
            if (key < u.k0 || key >= u.k1) vt[i] = u32x4_t{0, 0, 0, 0};
            odd |= non_finite_any<BF>(vt[i]);
          }
          if (!care && lo_max <= u.k0 && hi_min >= u.k1) odd = 0;  // all rows see the same keys
          special = __ballot(odd != 0) != 0;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
          *(u32x4_t*)(stage + v_pos<D>(i * (kWave / CH) + lane / CH, lane % CH)) = vt[i];
        if (more) load_v(vt, kb + kTile, ids);
        ids = page_ids(kb + 2 * kTile);
        wave_lds_order();
        if (__builtin_expect(special, 0)) {
          u32x4_t seen;
#pragma unroll
          for (int w = 0; w < 4; ++w)
            seen[w] = ((vis >> (2 * w)) & 1) * Bits16<BF>::kOne + (((vis >> (2 * w + 1)) & 1) * Bits16<BF>::kOne << 16);
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            u32x4_t vf = read_vt<D>(stage, d, g, r16);
            const u32x4_t up = infinite_ones<BF>(vf, 0), down = infinite_ones<BF>(vf, 0x10001u);
            const f4_t nu = mfma16<BF>(up, seen, f4_t{0, 0, 0, 0}), nd = mfma16<BF>(down, seen, f4_t{0, 0, 0, 0});
            vf = finite_or_zero<BF>(vf);
            acc[d] = mfma16<BF>(vf, pl, acc[d]);
            acc[d] = mfma16<BF>(vf, ph, acc[d]);
            add_infinities(acc[d], nu, nd);
            __builtin_amdgcn_sched_barrier(0);  // (one fragment at a time: this path must not cost registers)
          }
        } else {
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            const u32x4_t vf = read_vt<D>(stage, d, g, r16);
            acc[d] = mfma16<BF>(vf, pl, acc[d]);
            acc[d] = mfma16<BF>(vf, ph, acc[d]);
          }
        }
        wave_lds_order();
      }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);

    // join the waves
    float z = 0.f;  // NaN if a sum is not finite
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) z = fmaf(acc[d][i], 0.f, z);
    const bool bad = __ballot(z != z) != 0;
    __syncthreads();
#pragma unroll
    for (int d = 0; d < ND; ++d)
      *(f4_t*)(join + (wave * kRows + r16) * StepLds<D>::kPitch + d * 16 + 4 * g) = acc[d];
    if (g == 0) {
      join_m[wave * kRows + r16] = m;
      join_m[(kWaves + wave) * kRows + r16] = l;
    }
    if (lane == 0) scratch[12 + wave] = bad;
    __syncthreads();
    int again = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) again |= scratch[12 + w];
    if (__builtin_expect(!care && again != 0, 0)) {
      care = true;
      continue;
    }
    auto write = [&](int row, int d, f4_t o, float mm, float ll) {
      const float inv = ll > 0.f || ll != ll ? 1.f / ll : 0.f;
      const uint32_t ur = (uint32_t)(u.t * kRows + row);
      const int in_seq = attn_token(a, (int)ur), tok = u.s.first + in_seq;
      const int hd = u.head * a.group + (int)ur - in_seq * a.group;
      if (d < a.head_dim) {
        if (ll == 0.f) o = f4_t{0, 0, 0, 0};
        u32x2_t w = {pack2<BF>(o[0] * inv, o[1] * inv), pack2<BF>(o[2] * inv, o[3] * inv)};
        *(u32x2_t*)(a.out + tok * a.out_token + hd * a.out_head + d) = w;
      }
      if (d == 0 && a.lse)
        a.lse[(int64_t)tok * (a.kv_heads * a.group) + hd] =
            ll == 0.f ? -INFINITY : (mm - kShift + log2f(ll)) * 0.69314718055994531f;
    };

    // 4 elements of a row per thread and turn
    constexpr int kTurns = kRows * D / 4 / (kWaves * kWave);
    f4_t o[kTurns];
    float mm[kTurns], ll[kTurns];
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
      const int i = t * (kWaves * kWave) + threadIdx.x, row = i / (D / 4), d = (i % (D / 4)) * 4;
      mm[t] = -INFINITY;
      ll[t] = 0.f;
      o[t] = f4_t{0, 0, 0, 0};
      if (row >= rows) continue;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) mm[t] = fmaxf(mm[t], join_m[w * kRows + row]);
      const float bm = mm[t] == -INFINITY ? 0.f : mm[t];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        // (a wave without keys of this row; NaN scores leave the maximum where it was,
        // but not the denominator)
        const float mw = join_m[w * kRows + row], lw = join_m[(kWaves + w) * kRows + row];
        if (mw == -INFINITY && lw == 0.f) continue;
        const float e = rescale(mw - bm);
        ll[t] += e * lw;
        o[t] += e * *(const f4_t*)(join + (w * kRows + row) * StepLds<D>::kPitch + d);
      }
    }
    bool done = true;
    if (u.from != 0 || u.to != u.tiles) {
      int w0, w1;
      attn_holders(h, u, w0, w1);
      const int n = w1 - w0 + 1;
      float* const place = attn_place(a, w0, wg - w0, step_place<D>());
#pragma unroll
      for (int t = 0; t < kTurns; ++t) {
        const int i = t * (kWaves * kWave) + threadIdx.x, row = i / (D / 4), d = (i % (D / 4)) * 4;
        if (row >= rows) continue;
        put4(place + row * D + d, o[t]);
        if (d == 0) put2(place + kRows * D + 2 * row, mm[t], ll[t]);
      }
      done = attn_last(&a.counters[w0], n, scratch + 8);
      if (done) {
        // in the order of the keys, four pieces' loads at a time, this
        // workgroup's own from its registers
        const int mine = wg - w0;
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
          const int i = t * (kWaves * kWave) + threadIdx.x, row = i / (D / 4), d = (i % (D / 4)) * 4;
          if (row >= rows) continue;
          const f4_t own = o[t];
          const float own_m = mm[t], own_l = ll[t];
          mm[t] = -INFINITY;
          ll[t] = 0.f;
          o[t] = f4_t{0, 0, 0, 0};
          for (int p0 = 0; p0 < n; p0 += 4) {
            f4_t x[4];
            f2_t ml[4];
#pragma unroll
            for (int p = 0; p < 4; ++p) {
              const float* const pp = attn_place(a, w0, min(p0 + p, n - 1), step_place<D>());
              x[p] = get4(pp + row * D + d);
              ml[p] = get2(pp + kRows * D + 2 * row);
            }
#pragma unroll
            for (int p = 0; p < 4; ++p) {
              if (p0 + p == mine) {
                x[p] = own;
                ml[p] = f2_t{own_m, own_l};
              }
              if (p0 + p >= n || (ml[p][0] == -INFINITY && ml[p][1] == 0.f)) continue;  // (no keys of this row)
              const float mn = fmaxf(mm[t], ml[p][0]);
              const float wa = rescale(mm[t] - mn), wb = rescale(ml[p][0] - mn);
              mm[t] = mn;
              ll[t] = ll[t] * wa + wb * ml[p][1];
              o[t] = o[t] * wa + wb * x[p];
            }
          }
        }
      }
    }
    if (done) {
#pragma unroll
      for (int t = 0; t < kTurns; ++t) {
        const int i = t * (kWaves * kWave) + threadIdx.x, row = i / (D / 4), d = (i % (D / 4)) * 4;
        if (row < rows) write(row, d, o[t], mm[t], ll[t]);
      }
    }
    __syncthreads();
    care = false;
    at = min(u.stop, h.end);
  }
  attn_unheld<kWaves * kWave>(a, list, wg, grid);
}

template <bool BF, int D, bool EXACT>
hipError_t launch(const AttnArgs& a, int grid, hipStream_t s) {
  constexpr auto kern = k_attention_step<BF, D, EXACT>;
  const hipError_t e = allow_dynamic_lds((const void*)kern, StepLds<D>::kFixed + (kAttnMaxSeqs + 1) * 16);
  if (e != hipSuccess) return e;
  kern<<<grid, kWaves * kWave, StepLds<D>::kFixed + (a.seqs + 1) * 16, s>>>(a);
  return hipGetLastError();
}

template <bool BF, int D>
hipError_t launch(const AttnArgs& a, int grid, hipStream_t s) {
  return a.head_dim == D ? launch<BF, D, true>(a, grid, s) : launch<BF, D, false>(a, grid, s);
}

}  // namespace

int attention_step_grid() { return 2 * num_cus(); }
int64_t attention_step_place(int head_dim) { return (int64_t)kRows * (attention_dim(head_dim) + 2); }

hipError_t launch_attention_step(const AttnArgs& a, bool bf, int grid, hipStream_t s) {
  switch (attention_dim(a.head_dim)) {
    case 64: return bf ? launch<true, 64>(a, grid, s) : launch<false, 64>(a, grid, s);
    case 128: return bf ? launch<true, 128>(a, grid, s) : launch<false, 128>(a, grid, s);
    default: return bf ? launch<true, 256>(a, grid, s) : launch<false, 256>(a, grid, s);
  }
}

}  // namespace aqlm
