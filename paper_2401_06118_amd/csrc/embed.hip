// Rows of the embedding table by token, scaled, and the table's gradient.
//
//   y[t] = scale E[id_t]                        (ids outside the table: zeros)
//   dE[v] = scale sum over t with id_t = v of dy[t]
//
// Both are bound by memory: the first reads each row that occurs and writes one per token,
// the second reads a row per token and writes one per token of the vocabulary, zeros for
// those that do not occur.
#include "ends.h"

#include "common.h"
#include "elements.h"
#include "join.h"
#include "launch.h"

namespace aqlm {

namespace {

constexpr int kThreads = 256;

// Results of more than the L2s hold go past them (8192 rows of 8192 in bf16: 43 -> 36 us, with one
// piece a thread as with four; those of a step stay, for what reads them next).
constexpr int64_t kStreamBytes = 32 << 20;

// A piece of 16 bytes a thread, blocks_per_row workgroups a row.
template <int TY, bool NT>
__global__ void __launch_bounds__(kThreads) k_embed(EmbedArgs a, int blocks_per_row) {
  typedef typename Elem<TY>::T T;
  typedef typename Elem<TY>::V V;
  constexpr int N = kPiece<TY>;
  for (int64_t b = blockIdx.x; b < a.count * blocks_per_row; b += gridDim.x) {
    const int64_t t = b / blocks_per_row;
    const int c = ((int)(b - t * blocks_per_row) * kThreads + threadIdx.x) * N;
    const int id = a.tokens[t];
    if (c >= a.dim) continue;
    const bool held = (uint32_t)id < (uint32_t)a.vocab;
    const V v = load_piece<TY>((const T*)a.table + (held ? id : 0) * a.table_row, c, a.dim);
    V y;
    // (a row that is not held is zeros whatever the first one has)
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = held ? (T)((float)v[e] * a.scale) : (T)0.f;
    store_piece<TY, NT>((T*)a.out + t * a.out_row, c, a.dim, y);
  }
}

template <int TY>
hipError_t launch_embed_typed(const EmbedArgs& a, hipStream_t s) {
  const int pieces = (a.dim + kPiece<TY> - 1) / kPiece<TY>, per_row = (pieces + kThreads - 1) / kThreads;
  const int64_t blocks = a.count * per_row;
  const unsigned grid = (unsigned)(blocks < (1 << 22) ? blocks : (1 << 22));
  if (a.count * a.dim * dtype_bytes(TY) > kStreamBytes) k_embed<TY, true><<<grid, kThreads, 0, s>>>(a, per_row);
  else k_embed<TY, false><<<grid, kThreads, 0, s>>>(a, per_row);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Gradient.  One launch sorts the places 0 .. tokens - 1 by token (stable); the next sums each
// token's rows in the order of its places and, by other workgroups, writes the zero rows: those
// are most of the bytes, and hide the sums' latency (4096 tokens over 32000 x 4096 fp16: 7 us and 52, 5.6 TB/s).
//
// Sorting: workgroup b of 2^lg holds the tokens whose low lg bits are b, so that tokens
// with small numbers, the frequent ones, are spread.  It walks all ids twice: counts (how many
// belong to earlier workgroups, and for each wave's share of the places how many are
// each of its own tokens), then writes places.  2^lg x tokens x 4 bytes from the L2s.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave;
constexpr int kSortOwn = 512;  // tokens of a workgroup

__global__ void __launch_bounds__(kSortThreads) k_embed_sort(EmbedGradArgs a, int lg, int64_t counters) {
  __shared__ int at[kSortWaves][kSortOwn];  // counts, then the next place of a wave's token
  __shared__ int from[kSortOwn], total[kSortOwn];  // where a token's places begin, how many
  __shared__ int below[kSortWaves], sums[kSortWaves];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int b = blockIdx.x, own = (a.vocab - b + (1 << lg) - 1) >> lg;  // tokens b, b + 2^lg, ...
  for (int64_t i = (int64_t)b * kSortThreads + tid; i < counters; i += (int64_t)gridDim.x * kSortThreads) a.counters[i] = 0;
  for (int i = tid; i < kSortWaves * kSortOwn; i += kSortThreads) (&at[0][0])[i] = 0;
  __syncthreads();
  // (shares of whole waves' loads; in 64 bits, as tokens go up to 2^31)
  const int64_t share = ((int64_t)(a.tokens_count + kSortWaves - 1) / kSortWaves + kWave - 1) / kWave * kWave;
  const int begin = (int)min((int64_t)a.tokens_count, wave * share);
  const int end = (int)min((int64_t)a.tokens_count, (wave + 1) * share);
  // The share's ids, kBatch loads of the wave in flight.
  constexpr int kBatch = 8;
  auto walk = [&](auto take) {
    for (int64_t i0 = begin; i0 < end; i0 += kBatch * kWave) {
      int id[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int64_t i = i0 + j * kWave + lane;
        id[j] = i < end ? a.tokens[i] : -1;
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const bool held = (uint32_t)id[j] < (uint32_t)a.vocab;
        take((int)(i0 + j * kWave + lane), id[j], held, held && (id[j] & ((1 << lg) - 1)) == b);
      }
    }
  };
  int before = 0;
  walk([&](int, int id, bool held, bool mine) {
    before += held && (id & ((1 << lg) - 1)) < b;
    if (mine) atomicAdd(&at[wave][id >> lg], 1);
  });
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) before += __shfl_xor(before, s);
  if (lane == 0) below[wave] = before;
  __syncthreads();
  // exclusive sums over the tokens, then over the waves of each
  int n = 0, count[kSortWaves];
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    count[w] = tid < own ? at[w][tid] : 0;
    n += count[w];
  }
  int incl = n;
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) {
    const int o = __shfl_up(incl, s);
    if (lane >= s) incl += o;
  }
  if (lane == kWave - 1) sums[wave] = incl;
  __syncthreads();
  int base = incl - n, all = 0;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    const int o = sums[w];
    base += below[w] + (w < wave ? o : 0);
    all += below[w] + o;
  }
  if (b == (int)gridDim.x - 1 && tid == 0) *a.held = all;
  if (tid < own) {
    int next = base;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      at[w][tid] = next;
      next += count[w];
    }
    from[tid] = base;
    total[tid] = n;
    a.occurs[(int64_t)b * kSortOwn + tid] = n != 0;
  }
  __syncthreads();
  walk([&](int i, int id, bool, bool mine) {
    for (uint64_t left = __ballot(mine); left != 0;) {
      const int lead = __builtin_ctzll(left);
      const int r = __shfl(id, lead) >> lg;
      const uint64_t same = __ballot(mine && id >> lg == r);
      const int p = at[wave][r];
      if (mine && id >> lg == r) {
        const int place = p + __popcll(same & ((1ull << lane) - 1));
        a.order[place] = i;
        a.first[place] = from[r];
        a.last[place] = from[r] + total[r];
      }
      if (lane == lead) at[wave][r] = p + __popcll(same);
      left &= ~same;
    }
  });
}

// Rows of tokens that do not occur: a wave a row.
template <int OTY>
__device__ __forceinline__ void write_zero_rows(const EmbedGradArgs& a, int lg, int64_t wave, int64_t waves) {
  constexpr int N = kPiece<OTY>;
  typename Elem<OTY>::V zero;
#pragma unroll
  for (int e = 0; e < N; ++e) zero[e] = (typename Elem<OTY>::T)0.f;
  constexpr int kBatch = 8;  // rows whose marks are loaded at once
  for (int64_t v0 = wave; v0 < a.vocab; v0 += kBatch * waves) {
    bool occurs[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int64_t v = min(v0 + j * waves, (int64_t)a.vocab - 1);
      occurs[j] = a.occurs[(v & ((1 << lg) - 1)) * kSortOwn + (v >> lg)] != 0;
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int64_t v = v0 + j * waves;
      if (v >= a.vocab || occurs[j]) continue;
      typename Elem<OTY>::T* const out = (typename Elem<OTY>::T*)a.out + v * a.out_row;
      for (int c = threadIdx.x % kWave * N; c < a.dim; c += kWave * N) store_piece<OTY>(out, c, a.dim, zero);
    }
  }
}

// The first units x columns workgroups: the rows of kEmbedUnit sorted places, in a block of columns (a
// piece of 16 bytes a thread).  Sums of tokens that lie in one unit are written; pieces of those
// that do not go to memory, and the last workgroup to bring one adds them in the order of
// the units.  The others write zeros.
template <int TY, int OTY>
__global__ void __launch_bounds__(kThreads) k_embed_sum(EmbedGradArgs a, int lg, int units, int columns) {
  typedef typename Elem<TY>::T T;
  typedef typename Elem<TY>::V V;
  typedef typename Elem<OTY>::T O;
  constexpr int N = kPiece<TY>;
  __shared__ int flag;
  const int summing = units * columns;
  if ((int)blockIdx.x >= summing)
    return write_zero_rows<OTY>(a, lg, (int64_t)(blockIdx.x - summing) * (kThreads / kWave) + threadIdx.x / kWave,
                                (int64_t)(gridDim.x - summing) * (kThreads / kWave));
  const int held = *a.held, column = blockIdx.x % columns;
  const int c = (column * kThreads + threadIdx.x) * N;
  const bool active = c < a.dim;
  for (int64_t begin = (int64_t)(blockIdx.x / columns) * kEmbedUnit; begin < held; begin += (int64_t)units * kEmbedUnit) {
    const int p0 = (int)begin, unit = p0 / kEmbedUnit, p1 = (int)min(begin + kEmbedUnit, (int64_t)held);
    float sum[N];
    auto write = [&](int place, const float* s) {
      if (!active) return;
      O* const out = (O*)a.out + a.tokens[place] * a.out_row;
      if constexpr (kPiece<OTY> == N) {
        typename Elem<OTY>::V o;
#pragma unroll
        for (int e = 0; e < N; ++e) o[e] = (O)(s[e] * a.scale);
        store_piece<OTY>(out, c, a.dim, o);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (c + e < a.dim) out[c + e] = (O)(s[e] * a.scale);
      }
    };
    // (pieces of a unit: of a token that began before it, and of one that goes on behind it; two floats a store)
    auto part = [&](int u, int which) { return (uint64_t*)(a.parts + ((int64_t)u * 2 + which) * a.parts_row + c); };
    auto put = [&](int which) {
      if (!active) return;
#pragma unroll
      for (int e = 0; e < N / 2; ++e)
        put_through(part(unit, which) + e, (uint64_t)__builtin_bit_cast(uint32_t, sum[2 * e]) |
                                               (uint64_t)__builtin_bit_cast(uint32_t, sum[2 * e + 1]) << 32);
    };
    int order[kEmbedUnit], first[kEmbedUnit], last[kEmbedUnit];
#pragma unroll
    for (int i = 0; i < kEmbedUnit; ++i) {
      order[i] = a.order[min(p0 + i, p1 - 1)];
      first[i] = a.first[min(p0 + i, p1 - 1)];
      last[i] = a.last[min(p0 + i, p1 - 1)];
    }
    V v[kEmbedUnit];
#pragma unroll
    for (int i = 0; i < kEmbedUnit; ++i) {
      v[i] = V(0);
      if (active) v[i] = load_piece<TY>((const T*)a.dout + order[i] * a.dout_row, c, a.dim);
    }
    // what is open at this unit's ends
    const int head_first = first[0], head_last = last[0], tail_last = last[kEmbedUnit - 1], tail_first = first[kEmbedUnit - 1];
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = 0.f;
#pragma unroll
    for (int i = 0; i < kEmbedUnit; ++i) {
      if (p0 + i >= p1) break;
#pragma unroll
      for (int e = 0; e < N; ++e) sum[e] += (float)v[i][e];
      if (last[i] == p0 + i + 1) {  // the token's last place
        if (first[i] >= p0) write(order[i], sum);
        else put(0);
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] = 0.f;
      }
    }
    if (tail_last > p1) put(tail_first < p0 ? 0 : 1);
    // join: the token that began before this unit, and the one that goes on behind it
    auto join = [&](int f, int l) {
      const int u0 = f / kEmbedUnit, u1 = (l - 1) / kEmbedUnit;
      if (!last_of(a.counters + (int64_t)u0 * columns + column, u1 - u0 + 1, &flag)) return;
      if (!active) return;
      float s[N];
#pragma unroll
      for (int e = 0; e < N; ++e) s[e] = 0.f;
      constexpr int kBatch = 8;  // units whose pieces are loaded at once
      for (int b0 = u0; b0 <= u1; b0 += kBatch) {
        uint64_t w[kBatch][N / 2];
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
#pragma unroll
          for (int e = 0; e < N / 2; ++e) {
            const int u = min(b0 + j, u1);
            w[j][e] = get_through(part(u, u == u0 ? 1 : 0) + e);
          }
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
#pragma unroll
          for (int e = 0; e < N / 2; ++e)
            if (b0 + j <= u1) {
              s[2 * e] += __builtin_bit_cast(float, (uint32_t)w[j][e]);
              s[2 * e + 1] += __builtin_bit_cast(float, (uint32_t)(w[j][e] >> 32));
            }
      }
      write(a.order[f], s);
    };
    if (head_first < p0) join(head_first, head_last);
    if (tail_last > p1 && tail_first >= p0) join(tail_first, tail_last);
  }
}

template <int TY, int OTY>
hipError_t launch_grad_typed(const EmbedGradArgs& a, hipStream_t s) {
  const int lg = embed_grad_lg(a.vocab);
  const int units = (int)((a.tokens_count + (int64_t)kEmbedUnit - 1) / kEmbedUnit);
  const int columns = embed_grad_column_blocks(a.dim, TY);
  k_embed_sort<<<1u << lg, kSortThreads, 0, s>>>(a, lg, (int64_t)units * columns);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // (a launch has fewer than 2^32 threads)
  const int summing = min(units, max(1, (1 << 23) / columns));
  k_embed_sum<TY, OTY><<<(unsigned)(summing * columns + 16 * num_cus()), kThreads, 0, s>>>(a, lg, summing, columns);
  return hipGetLastError();
}

}  // namespace

int embed_grad_lg(int64_t vocab) {
  int lg = 8;
  while ((int64_t)kSortOwn << lg < vocab) ++lg;
  return lg;
}
int64_t embed_grad_marks(int64_t vocab) { return (int64_t)kSortOwn << embed_grad_lg(vocab); }
int embed_grad_column_blocks(int32_t dim, int dtype) {
  const int columns = kThreads * (dtype == kF32 ? 4 : 8);
  return (dim + columns - 1) / columns;
}

hipError_t launch_embed(const EmbedArgs& a, int dtype, hipStream_t s) {
  if (dtype == kF16) return launch_embed_typed<kF16>(a, s);
  if (dtype == kBf16) return launch_embed_typed<kBf16>(a, s);
  return launch_embed_typed<kF32>(a, s);
}

hipError_t launch_embed_grad(const EmbedGradArgs& a, int dtype, int out_dtype, hipStream_t s) {
  if (dtype == kF32) return launch_grad_typed<kF32, kF32>(a, s);
  if (dtype == kF16) return out_dtype == kF16 ? launch_grad_typed<kF16, kF16>(a, s) : launch_grad_typed<kF16, kF32>(a, s);
  return out_dtype == kBf16 ? launch_grad_typed<kBf16, kBf16>(a, s) : launch_grad_typed<kBf16, kF32>(a, s);
}

}  // namespace aqlm
