// Rotary positions of queries and keys, with the RMS norm of each head before
// the rotation, its gradients, and the same on the way into a paged cache.
//
//   y = x rsqrt(mean(x^2) + eps) w            (with a norm)
//   (y_a, y_b) -> (y_a cos - y_b sin, y_b cos + y_a sin)
//
// over the pairs (a, b) = (i, i + rot / 2) or (2i, 2i + 1), i < rot / 2; elements
// from rot on are left.  cos and sin come from a table in fp32, made once in 64
// bits (angles of long contexts lose all their bits in 32).  Backward, with g the
// gradient rotated back, r the norm's factor and n = x r:
//
//   dx = r (g w - n mean(g w n)),   dw = sum over tokens and heads of g n.
//
// Bound: memory; everything is read and written once.  A head is held by 1 to 32
// neighbouring lanes, 16 elements each: two 16-byte pieces (32 bytes in fp32)
// whose elements pair with each other (half layout) or within (interleaved), so a
// pair never crosses lanes, and a lane's 8 cos and sin serve all heads that it
// runs of its token.  All loads of the heads go out before the first is used.
// Measured, calls back to back: norms and rotation of 4096 tokens of 64 + 8 heads of 128,
// bf16 (153 MB): 29.8 us, 5.2 TB/s (a copy of as much: 31); the gradients with norms of 2048
// tokens of 32 + 32 heads (102 MB) 27.8 us, of which 23.5 are the first kernel's and 4.9 the
// sum over workgroups (kernel trace; two heads' loads at a time there: 25.1).
// Any other alignment, head size or rotated part takes the general kernels, one
// wave a head and 2 or 4 bytes a lane, bound by their instructions: 4096 tokens of 32 + 8
// heads of 96 elements, 24 of them rotated, bf16 (63 MB) 62 us, with norms 73, their gradients
// 109 (all 96 rotated, by the vectorised kernels: 19, 20 and 31); appended 98 and 111 (22
// and 27).
#include "rope.h"

#include <algorithm>

#include "common.h"
#include "launch.h"

namespace aqlm {

namespace {

typedef float f8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf8_t __attribute__((ext_vector_type(8)));
typedef uint32_t u32x8_t __attribute__((ext_vector_type(8)));

template <int TY>
struct Elem;
template <>
struct Elem<kF16> {
  typedef _Float16 T;
  typedef h8_t V;
};
template <>
struct Elem<kBf16> {
  typedef __bf16 T;
  typedef bf8_t V;
};
template <>
struct Elem<kF32> {
  typedef float T;
  typedef f8_t V;
};

// Workgroups of 256 threads, one after another along x and then y: a launch may
// not have 2^32 threads along one axis, which one wave a head reaches at 2^26 heads.
constexpr int64_t kMostAlongX = 1 << 22;
dim3 grid_of(int64_t wgs) {
  return wgs <= kMostAlongX ? dim3((unsigned)wgs)
                            : dim3((unsigned)kMostAlongX, (unsigned)((wgs + kMostAlongX - 1) / kMostAlongX));
}
__device__ __forceinline__ int64_t workgroup() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// Sum over groups of n neighbouring lanes (a power of two).
__device__ __forceinline__ float group_sum(float v, int n) {
  for (int d = 1; d < n; d *= 2) v += __shfl_xor(v, d);
  return v;
}

// Where a new token goes: its sequence and position, -1 without a place.
__device__ __forceinline__ int paged_position(const RopeArgs& a, int token, int& seq) {
  int b;
  if (token < a.seqs && a.cu_new[token] <= token && a.cu_new[token + 1] > token) {
    b = token;  // one new token a sequence
  } else {
    int lo = 0, hi = a.seqs;  // the last sequence that begins at or before the token
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.cu_new[mid] <= token) lo = mid;
      else hi = mid;
    }
    b = lo;
  }
  seq = b;
  const int begin = a.cu_new[b], end = a.cu_new[b + 1];
  if (token < begin || token >= end) return -1;
  return (int)max((int64_t)a.kv_lens[b] - end + token, (int64_t)-1);
}

// The page of a position of a sequence, -1 if the table or the cache has none.
__device__ __forceinline__ int paged_page(const RopeArgs& a, int seq, int pos) {
  const int i = pos >> a.page_shift;
  if (pos < 0 || i >= a.table_width) return -1;
  const int p = a.block_table[seq * a.table_stride + i];
  return p >= 0 && p < a.pages ? p : -1;
}

// A lane's two pieces of a head (in units of 8 elements), whether the head has
// them, and the first of the 4 pairs of each half of the lane's 8.
struct Pieces {
  int c[2];
  bool on[2];
  int pair[2];
};
template <bool INTER>
__device__ __forceinline__ Pieces pieces_of(const RopeArgs& a, int i, int lanes) {
  Pieces p;
  const int ch = a.head_dim / 8;
  if (INTER) {  // pairs lie within a piece: neighbouring lanes take neighbouring ones
    p.c[0] = i;
    p.c[1] = i + lanes;
  } else if (i < a.rot / 16) {
    p.c[0] = i;
    p.c[1] = i + a.rot / 16;
  } else {
    p.c[0] = a.rot / 8 + 2 * (i - a.rot / 16);
    p.c[1] = p.c[0] + 1;
  }
  p.on[0] = p.c[0] < ch;
  p.on[1] = p.c[1] < ch;
  p.pair[0] = INTER ? 4 * p.c[0] : 8 * i;
  p.pair[1] = INTER ? 4 * p.c[1] : 8 * i + 4;
  return p;
}

// cos and sin of a lane's 8 pairs; pairs past the rotated part are left as they
// are.  False for a position that the table does not have.
__device__ __forceinline__ bool load_turn(const RopeArgs& a, int pos, const Pieces& p, float (&c)[8], float (&s)[8]) {
  const int half = a.rot / 2;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    c[i] = 1.f;
    s[i] = 0.f;
  }
  if (half == 0) return true;
  if (pos < 0 || pos >= a.rows) return false;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const float* t = a.table + ((int64_t)pos * half + p.pair[e]) * 2;
    if (p.pair[e] + 4 <= half) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float4 v = *(const float4*)(t + 4 * i);
        c[4 * e + 2 * i] = v.x;
        s[4 * e + 2 * i] = v.y;
        c[4 * e + 2 * i + 1] = v.z;
        s[4 * e + 2 * i + 1] = v.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (p.pair[e] + i < half) {
          const float2 v = *(const float2*)(t + 2 * i);
          c[4 * e + i] = v.x;
          s[4 * e + i] = v.y;
        }
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) s[i] *= a.sign;
  return true;
}

// Pairs past the rotated part stay as they are (a turn by cos 1, sin 0 would carry an
// infinite or NaN element to its neighbour).
template <bool INTER>
__device__ __forceinline__ void turn(const RopeArgs& a, int lane, const Pieces& p, float (&y)[16], const float (&c)[8],
                                     const float (&s)[8]) {
  if (!INTER && lane >= a.rot / 16) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int ia = INTER ? 2 * i : i, ib = INTER ? 2 * i + 1 : i + 8;
    const bool rotates = !INTER || p.pair[i / 4] + i % 4 < a.rot / 2;
    const float ya = y[ia], yb = y[ib];
    y[ia] = rotates ? ya * c[i] - yb * s[i] : ya;
    y[ib] = rotates ? yb * c[i] + ya * s[i] : yb;
  }
}

template <int TY>
__device__ __forceinline__ typename Elem<TY>::V load8(const void* base, int64_t off, bool on) {
  typedef typename Elem<TY>::V V;
  V v;
  if (on) return *(const V*)((const typename Elem<TY>::T*)base + off);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (typename Elem<TY>::T)0.f;
  return v;
}
// STREAM: past the L2s, for outputs that do not fit them (4096 tokens of 72
// heads of 128 in bf16, with norms, kernel trace: 41 us with plain stores, 32 with these).
template <int TY, bool STREAM>
__device__ __forceinline__ void store8(void* base, int64_t off, const float* y) {
  typedef typename Elem<TY>::V V;
  V v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (typename Elem<TY>::T)y[i];
  V* const to = (V*)((typename Elem<TY>::T*)base + off);
  if constexpr (STREAM) __builtin_nontemporal_store(v, to);
  else *to = v;
}

// HPT heads of a token for a group of `lanes` lanes; heads counted over q, k (and v).
template <int TY, bool NORM, bool INTER, bool PAGED, int HPT>
__global__ void __launch_bounds__(256) k_rope(RopeArgs a, int lanes, int per_token) {
  typedef typename Elem<TY>::V V;
  const int group = threadIdx.x / lanes, i = threadIdx.x % lanes;
  const int64_t item = workgroup() * (256 / lanes) + group;
  const bool live = item < (int64_t)a.tokens * per_token;
  const int token = live ? (int)(item / per_token) : 0;
  const int h0 = live ? (int)(item - (int64_t)token * per_token) * HPT : 0;
  const int nq = a.side[0].heads, nk = a.side[1].heads, all = nq + nk + (PAGED ? a.side[2].heads : 0);
  const Pieces p = pieces_of<INTER>(a, i, lanes);

  V x[HPT][2];
#pragma unroll
  for (int j = 0; j < HPT; ++j) {
    const int h = h0 + j;
    const int w = h < nq ? 0 : (h < nq + nk ? 1 : 2);
    const RopeSide& sd = a.side[w];
    const int64_t off = token * sd.in_token + (h - (w == 0 ? 0 : (w == 1 ? nq : nq + nk))) * sd.in_head;
#pragma unroll
    for (int e = 0; e < 2; ++e) x[j][e] = load8<TY>(sd.in, off + p.c[e] * 8, live && h < all && p.on[e]);
  }
  int seq = 0, page = -1;
  const int pos = PAGED ? paged_position(a, token, seq) : a.positions[token];
  if (PAGED) page = paged_page(a, seq, pos);
  float c[8], s[8];
  const bool inside = load_turn(a, pos, p, c, s);

#pragma unroll
  for (int j = 0; j < HPT; ++j) {
    const int h = h0 + j;
    const int w = h < nq ? 0 : (h < nq + nk ? 1 : 2);
    const RopeSide& sd = a.side[w];
    const int hs = h - (w == 0 ? 0 : (w == 1 ? nq : nq + nk));
    float y[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) y[e] = (float)x[j][e / 8][e % 8];
    if (NORM && sd.weight != nullptr) {  // (lanes of a group run the same head)
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) ss += y[e] * y[e];
      const float r = rsqrtf(group_sum(ss, lanes) / (float)a.head_dim + a.eps);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const V wt = load8<TY>(sd.weight, p.c[e] * 8, p.on[e]);
#pragma unroll
        for (int n = 0; n < 8; ++n) y[e * 8 + n] = y[e * 8 + n] * r * (float)wt[n];
      }
    }
    if (w != 2) {
      turn<INTER>(a, i, p, y, c, s);
      if (!inside)
#pragma unroll
        for (int e = 0; e < 16; ++e) y[e] = __builtin_nanf("");
    }
    if (!live || h >= all) continue;
    void* out = sd.out;
    int64_t off;
    if (PAGED && w > 0) {
      if (page < 0) continue;
      off = page * a.page_stride[w - 1] + (pos & ((1 << a.page_shift) - 1)) * a.slot_stride[w - 1] + hs * a.cache_head[w - 1];
    } else {
      off = token * sd.out_token + hs * sd.out_head;
      if (PAGED && pos < 0)
#pragma unroll
        for (int e = 0; e < 16; ++e) y[e] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (p.on[e]) store8<TY, (HPT > 1)>(out, off + p.c[e] * 8, y + e * 8);
  }
}

// Gradients with norms.  A workgroup runs heads of q (the first a.blocks[0]
// workgroups) or of k, and writes its sum of the weight's gradient.
template <int TY, bool INTER>
__global__ void __launch_bounds__(256) k_rope_grad(RopeArgs a, int lanes) {
  typedef typename Elem<TY>::V V;
  extern __shared__ float sums[];  // [groups][head_dim]
  const int group = threadIdx.x / lanes, i = threadIdx.x % lanes, groups = 256 / lanes;
  const int w = (int)blockIdx.x < a.blocks[0] ? 0 : 1;
  const int block = (int)blockIdx.x - (w ? a.blocks[0] : 0), blocks = a.blocks[w];
  const RopeSide& sd = a.side[w];
  const Pieces p = pieces_of<INTER>(a, i, lanes);
  float wt[16], dw[16];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const V v = load8<TY>(sd.weight, p.c[e] * 8, p.on[e]);
#pragma unroll
    for (int n = 0; n < 8; ++n) wt[e * 8 + n] = (float)v[n];
  }
#pragma unroll
  for (int e = 0; e < 16; ++e) dw[e] = 0.f;
  const int64_t items = (int64_t)a.tokens * sd.heads;
  const int64_t step = (int64_t)blocks * groups;
  const float inv_d = 1.f / (float)a.head_dim;
  // (every group runs the same number of turns: the sums below are over lanes)
  for (int64_t first = (int64_t)block * groups; first < items; first += step) {
    const int64_t item = first + group;
    const bool live = item < items;
    const int token = live ? (int)(item / sd.heads) : 0;
    const int h = live ? (int)(item - (int64_t)token * sd.heads) : 0;
    const int64_t go = token * sd.in_token + h * sd.in_head, xo = token * sd.x_token + h * sd.x_head;
    V gv[2], xv[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      gv[e] = load8<TY>(sd.in, go + p.c[e] * 8, live && p.on[e]);
      xv[e] = load8<TY>(sd.x, xo + p.c[e] * 8, live && p.on[e]);
    }
    float c[8], s[8];
    const bool inside = load_turn(a, a.positions[token], p, c, s);
    float g[16], x[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      g[e] = inside ? (float)gv[e / 8][e % 8] : __builtin_nanf("");
      x[e] = (float)xv[e / 8][e % 8];
    }
    turn<INTER>(a, i, p, g, c, s);
    float ss = 0.f, dot = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      ss += x[e] * x[e];
      dot += g[e] * wt[e] * x[e];
    }
    for (int d = 1; d < lanes; d *= 2) {
      ss += __shfl_xor(ss, d);
      dot += __shfl_xor(dot, d);
    }
    const float r = rsqrtf(ss * inv_d + a.eps);
    const float k = dot * r * inv_d;  // mean(g w n)
    if (!live) continue;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float n = x[e] * r;
      dw[e] += g[e] * n;
      g[e] = r * (g[e] * wt[e] - n * k);
    }
    const int64_t oo = token * sd.out_token + h * sd.out_head;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (p.on[e]) store8<TY, true>(sd.out, oo + p.c[e] * 8, g + e * 8);
  }
#pragma unroll
  for (int e = 0; e < 16; ++e)
    if (p.on[e / 8]) sums[group * a.head_dim + p.c[e / 8] * 8 + e % 8] = dw[e];
  __syncthreads();
  for (int d = threadIdx.x; d < a.head_dim; d += 256) {
    float t = 0.f;
    for (int n = 0; n < groups; ++n) t += sums[n * a.head_dim + d];
    a.parts[(int64_t)blockIdx.x * a.head_dim + d] = t;
  }
}

// dweight[w][d] = sum over the workgroups of q (w = 0) or k, in their order.
constexpr int kSumCols = 16;
__global__ void __launch_bounds__(256) k_rope_grad_sum(RopeArgs a) {
  __shared__ float sums[256 / kSumCols][kSumCols];
  const int w = blockIdx.y, col = threadIdx.x % kSumCols, row = threadIdx.x / kSumCols;
  const int d = blockIdx.x * kSumCols + col;
  const float* p = a.parts + (int64_t)(w ? a.blocks[0] : 0) * a.head_dim;
  float t = 0.f;
  if (d < a.head_dim)
#pragma unroll 8
    for (int b = row; b < a.blocks[w]; b += 256 / kSumCols) t += p[(int64_t)b * a.head_dim + d];
  sums[row][col] = t;
  __syncthreads();
  if (row == 0 && d < a.head_dim && a.dweight[w] != nullptr) {
    for (int n = 1; n < 256 / kSumCols; ++n) t += sums[n][col];
    a.dweight[w][d] = t;
  }
}

// The general kernels: one wave a head, element by element.  A lane's items are
// pairs (the first rot / 2) and single elements.
template <int TY>
__device__ __forceinline__ float load1(const void* base, int64_t off) {
  return (float)((const typename Elem<TY>::T*)base)[off];
}
template <int TY>
__device__ __forceinline__ void store1(void* base, int64_t off, float y) {
  ((typename Elem<TY>::T*)base)[off] = (typename Elem<TY>::T)y;
}
__device__ __forceinline__ void item_at(const RopeArgs& a, int i, int& ia, int& ib) {
  const int half = a.rot / 2;
  ia = i < half ? (a.interleaved ? 2 * i : i) : i + half;
  ib = i < half ? (a.interleaved ? 2 * i + 1 : i + half) : -1;
}

template <int TY, bool PAGED, int ITEMS>
__global__ void __launch_bounds__(256) k_rope_general(RopeArgs a, int64_t total, int all) {
  const int lane = threadIdx.x & 63;
  const int64_t item = workgroup() * 4 + (threadIdx.x >> 6);
  if (item >= total) return;
  const int token = (int)(item / all), h = (int)(item - (int64_t)token * all);
  const int nq = a.side[0].heads, nk = a.side[1].heads;
  const int w = h < nq ? 0 : (h < nq + nk ? 1 : 2);
  const int hs = h - (w == 0 ? 0 : (w == 1 ? nq : nq + nk));
  const RopeSide& sd = a.side[w];
  const int count = a.head_dim - a.rot / 2;
  const int64_t in = token * sd.in_token + hs * sd.in_head;
  float ya[ITEMS], yb[ITEMS], ss = 0.f;
#pragma unroll
  for (int j = 0; j < ITEMS; ++j) {
    const int i = j * kWave + lane;
    ya[j] = yb[j] = 0.f;
    if (i < count) {
      int ia, ib;
      item_at(a, i, ia, ib);
      ya[j] = load1<TY>(sd.in, in + ia);
      if (ib >= 0) yb[j] = load1<TY>(sd.in, in + ib);
    }
    ss += ya[j] * ya[j] + yb[j] * yb[j];
  }
  int seq = 0, page = -1;
  const int pos = PAGED ? paged_position(a, token, seq) : a.positions[token];
  if (PAGED) page = paged_page(a, seq, pos);
  const bool inside = pos >= 0 && pos < a.rows;
  const float r = sd.weight != nullptr ? rsqrtf(wave_sum(ss) / (float)a.head_dim + a.eps) : 1.f;
  void* const out = sd.out;
  int64_t off = token * sd.out_token + hs * sd.out_head;
  if (PAGED && w > 0) {
    if (page < 0) return;
    off = page * a.page_stride[w - 1] + (pos & ((1 << a.page_shift) - 1)) * a.slot_stride[w - 1] + hs * a.cache_head[w - 1];
  }
#pragma unroll
  for (int j = 0; j < ITEMS; ++j) {
    const int i = j * kWave + lane;
    if (i >= count) continue;
    int ia, ib;
    item_at(a, i, ia, ib);
    if (sd.weight != nullptr) {
      ya[j] = ya[j] * r * load1<TY>(sd.weight, ia);
      if (ib >= 0) yb[j] = yb[j] * r * load1<TY>(sd.weight, ib);
    }
    if (w != 2 && a.rot > 0 && !inside) ya[j] = yb[j] = __builtin_nanf("");
    if (w != 2 && ib >= 0 && inside) {
      const float2 t = *(const float2*)(a.table + ((int64_t)pos * (a.rot / 2) + i) * 2);
      const float c = t.x, s = t.y * a.sign, u = ya[j], v = yb[j];
      ya[j] = u * c - v * s;
      yb[j] = v * c + u * s;
    }
    if (PAGED && w == 0 && pos < 0) ya[j] = yb[j] = 0.f;
    store1<TY>(out, off + ia, ya[j]);
    if (ib >= 0) store1<TY>(out, off + ib, yb[j]);
  }
}

template <int TY, int ITEMS>
__global__ void __launch_bounds__(256) k_rope_grad_general(RopeArgs a) {
  extern __shared__ float sums[];  // [4][head_dim]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int w = (int)blockIdx.x < a.blocks[0] ? 0 : 1;
  const int block = (int)blockIdx.x - (w ? a.blocks[0] : 0), blocks = a.blocks[w];
  const RopeSide& sd = a.side[w];
  const int count = a.head_dim - a.rot / 2;
  float da[ITEMS], db[ITEMS];
#pragma unroll
  for (int j = 0; j < ITEMS; ++j) da[j] = db[j] = 0.f;
  const int64_t items = (int64_t)a.tokens * sd.heads;
  for (int64_t item = (int64_t)block * 4 + wave; item < items; item += (int64_t)blocks * 4) {
    const int token = (int)(item / sd.heads), h = (int)(item - (int64_t)token * sd.heads);
    const int64_t go = token * sd.in_token + h * sd.in_head, xo = token * sd.x_token + h * sd.x_head;
    const int pos = a.positions[token];
    const bool inside = pos >= 0 && pos < a.rows;
    float ga[ITEMS], gb[ITEMS], xa[ITEMS], xb[ITEMS], ss = 0.f, dot = 0.f;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const int i = j * kWave + lane;
      ga[j] = gb[j] = xa[j] = xb[j] = 0.f;
      if (i >= count) continue;
      int ia, ib;
      item_at(a, i, ia, ib);
      ga[j] = load1<TY>(sd.in, go + ia);
      xa[j] = load1<TY>(sd.x, xo + ia);
      if (ib >= 0) {
        gb[j] = load1<TY>(sd.in, go + ib);
        xb[j] = load1<TY>(sd.x, xo + ib);
        if (inside) {
          const float2 t = *(const float2*)(a.table + ((int64_t)pos * (a.rot / 2) + i) * 2);
          const float c = t.x, s = t.y * a.sign, u = ga[j], v = gb[j];
          ga[j] = u * c - v * s;
          gb[j] = v * c + u * s;
        }
      }
      if (a.rot > 0 && !inside) ga[j] = gb[j] = __builtin_nanf("");
      ss += xa[j] * xa[j] + xb[j] * xb[j];
      dot += ga[j] * load1<TY>(sd.weight, ia) * xa[j] + (ib >= 0 ? gb[j] * load1<TY>(sd.weight, ib) * xb[j] : 0.f);
    }
    const float r = rsqrtf(wave_sum(ss) / (float)a.head_dim + a.eps);
    const float k = wave_sum(dot) * r / (float)a.head_dim;
    const int64_t oo = token * sd.out_token + h * sd.out_head;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const int i = j * kWave + lane;
      if (i >= count) continue;
      int ia, ib;
      item_at(a, i, ia, ib);
      const float na = xa[j] * r, nb = xb[j] * r;
      da[j] += ga[j] * na;
      store1<TY>(sd.out, oo + ia, r * (ga[j] * load1<TY>(sd.weight, ia) - na * k));
      if (ib >= 0) {
        db[j] += gb[j] * nb;
        store1<TY>(sd.out, oo + ib, r * (gb[j] * load1<TY>(sd.weight, ib) - nb * k));
      }
    }
  }
#pragma unroll
  for (int j = 0; j < ITEMS; ++j) {
    const int i = j * kWave + lane;
    if (i >= count) continue;
    int ia, ib;
    item_at(a, i, ia, ib);
    sums[wave * a.head_dim + ia] = da[j];
    if (ib >= 0) sums[wave * a.head_dim + ib] = db[j];
  }
  __syncthreads();
  for (int d = threadIdx.x; d < a.head_dim; d += 256)
    a.parts[(int64_t)blockIdx.x * a.head_dim + d] =
        (sums[d] + sums[a.head_dim + d]) + (sums[2 * a.head_dim + d] + sums[3 * a.head_dim + d]);
}

__global__ void __launch_bounds__(256) k_rotary_table(const double* inv_freq, int64_t rows, int half, double scale,
                                                      float* table) {
  const int64_t i = workgroup() * 256 + threadIdx.x;
  if (i >= rows * half) return;
  const int64_t pos = i / half;
  double s, c;
  sincos((double)pos * inv_freq[i - pos * half], &s, &c);
  table[2 * i] = (float)(c * scale);
  table[2 * i + 1] = (float)(s * scale);
}

int lanes_of(int head_dim) {
  int n = 1;
  while (n * 16 < head_dim) n *= 2;
  return n;
}

template <int TY, bool NORM, bool INTER, bool PAGED>
hipError_t launch_vector(const RopeArgs& a, hipStream_t s) {
  const int lanes = lanes_of(a.head_dim);
  const int all = a.side[0].heads + a.side[1].heads + (PAGED ? a.side[2].heads : 0);
  const int groups = 256 / lanes;
  // several heads a group once that still leaves every CU work: the table's row
  // and the position are read once for them.  Two, or four with norms (4096 tokens
  // of 72 heads of 128, bf16, kernel trace: two 28.4 us without norms and 31.9 with them,
  // four 29.3 and 30.7; appending 2700 tokens of 32 + 32 + 32 heads 25.6 against 27.7; eight are slower
  // everywhere).
  const int64_t one = ((int64_t)a.tokens * all + groups - 1) / groups;
  if (one >= 8 * (int64_t)num_cus()) {
    constexpr int kHeads = NORM ? 4 : 2;
    const int per = (all + kHeads - 1) / kHeads;
    const int64_t wgs = ((int64_t)a.tokens * per + groups - 1) / groups;
    k_rope<TY, NORM, INTER, PAGED, kHeads><<<grid_of(wgs), 256, 0, s>>>(a, lanes, per);
  } else {
    k_rope<TY, NORM, INTER, PAGED, 1><<<grid_of(one), 256, 0, s>>>(a, lanes, all);
  }
  return hipGetLastError();
}

template <int TY, bool PAGED>
hipError_t launch_typed(const RopeArgs& a, bool vec, hipStream_t s) {
  const bool norm = a.side[0].weight != nullptr || a.side[1].weight != nullptr;
  if (vec) {
    if (a.interleaved)
      return norm ? launch_vector<TY, true, true, PAGED>(a, s) : launch_vector<TY, false, true, PAGED>(a, s);
    return norm ? launch_vector<TY, true, false, PAGED>(a, s) : launch_vector<TY, false, false, PAGED>(a, s);
  }
  const int all = a.side[0].heads + a.side[1].heads + (PAGED ? a.side[2].heads : 0);
  const int64_t total = (int64_t)a.tokens * all;
  const dim3 wgs = grid_of((total + 3) / 4);
  if (a.head_dim - a.rot / 2 <= 4 * kWave)
    k_rope_general<TY, PAGED, 4><<<wgs, 256, 0, s>>>(a, total, all);
  else
    k_rope_general<TY, PAGED, 16><<<wgs, 256, 0, s>>>(a, total, all);
  return hipGetLastError();
}

template <int TY>
hipError_t launch_grad(const RopeArgs& a, bool vec, hipStream_t s) {
  const unsigned wgs = (unsigned)(a.blocks[0] + a.blocks[1]);
  if (vec) {
    const int lanes = lanes_of(a.head_dim);
    const size_t lds = (size_t)(256 / lanes) * a.head_dim * 4;
    if (a.interleaved) k_rope_grad<TY, true><<<wgs, 256, lds, s>>>(a, lanes);
    else k_rope_grad<TY, false><<<wgs, 256, lds, s>>>(a, lanes);
  } else if (a.head_dim - a.rot / 2 <= 4 * kWave) {
    k_rope_grad_general<TY, 4><<<wgs, 256, 16 * (size_t)a.head_dim, s>>>(a);
  } else {
    k_rope_grad_general<TY, 16><<<wgs, 256, 16 * (size_t)a.head_dim, s>>>(a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  k_rope_grad_sum<<<dim3((unsigned)((a.head_dim + kSumCols - 1) / kSumCols), 2), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

// Whether the kernels of 16-byte pieces take these: heads of up to 512 elements in
// whole pieces, pairs that lie in two pieces of a lane, all addresses multiples of
// 16 bytes.
bool rope_vector(const RopeArgs& a, int dtype, bool paged, bool grad) {
  const int64_t unit = 16 / dtype_bytes(dtype);
  if (a.head_dim % 8 != 0 || a.head_dim > 512 || (!a.interleaved && a.rot % 16 != 0)) return false;
  if (((uintptr_t)a.table & 15) != 0 || (a.rot % 4 != 0 && a.rot >= 8)) return false;
  uintptr_t p = 0;
  int64_t st = 0;
  for (int i = 0; i < (paged ? 3 : 2); ++i) {
    const RopeSide& s = a.side[i];
    if (s.heads == 0) continue;
    p |= (uintptr_t)s.in | (uintptr_t)s.out | (uintptr_t)s.weight;
    st |= s.in_token | s.in_head;
    if (!paged || i == 0) st |= s.out_token | s.out_head;
    if (paged && i > 0) st |= a.page_stride[i - 1] | a.slot_stride[i - 1] | a.cache_head[i - 1];
    if (grad) {
      p |= (uintptr_t)s.x;
      st |= s.x_token | s.x_head;
    }
  }
  return (p & 15) == 0 && (st & (unit - 1)) == 0;
}

hipError_t launch_rope(const RopeArgs& a, int dtype, bool paged, hipStream_t s) {
  const bool vec = rope_vector(a, dtype, paged, false);
  if (paged) {
    if (dtype == kF16) return launch_typed<kF16, true>(a, vec, s);
    if (dtype == kBf16) return launch_typed<kBf16, true>(a, vec, s);
    return launch_typed<kF32, true>(a, vec, s);
  }
  if (dtype == kF16) return launch_typed<kF16, false>(a, vec, s);
  if (dtype == kBf16) return launch_typed<kBf16, false>(a, vec, s);
  return launch_typed<kF32, false>(a, vec, s);
}

int rope_grad_blocks() { return 4 * num_cus(); }

hipError_t launch_rope_grad_norm(RopeArgs a, int dtype, hipStream_t s) {
  const bool vec = rope_vector(a, dtype, false, true);
  const int groups = vec ? 256 / lanes_of(a.head_dim) : 4;
  // workgroups in proportion to the heads, none without a first item
  const int all = a.side[0].heads + a.side[1].heads;
  for (int i = 0; i < 2; ++i) {
    const int64_t items = ((int64_t)a.tokens * a.side[i].heads + groups - 1) / groups;
    const int64_t share = std::max<int64_t>(1, (int64_t)(rope_grad_blocks() - 1) * a.side[i].heads / all);
    a.blocks[i] = (int32_t)std::min(items, share);
  }
  if (dtype == kF16) return launch_grad<kF16>(a, vec, s);
  if (dtype == kBf16) return launch_grad<kBf16>(a, vec, s);
  return launch_grad<kF32>(a, vec, s);
}

hipError_t launch_rotary_table(const double* inv_freq, int64_t rows, int half, double scale, float* table,
                               hipStream_t s) {
  k_rotary_table<<<grid_of((rows * half + 255) / 256), 256, 0, s>>>(inv_freq, rows, half, scale, table);
  return hipGetLastError();
}

}  // namespace aqlm
