// The loss of a student's logits against the largest logits of a teacher, and its gradient.
// With q = softmax(z / tau) over the vocabulary and p over a token's listed ids:
//
//   p_k = softmax over the list of t_k / tau                      (without teacher_lse)
//   p_k = exp(t_k / tau - lse), p_r = max(0, 1 - sum p)           (with it; p_r = 0 where
//                                                                  every id is listed)
//   loss = sum_k p_k log(p_k / q_k) + p_r log(p_r / q_r),   q_r = sum of q outside the list
//   dloss/dz_j = (q_j P - p_j) / tau                              in the list, P = sum p + p_r
//              = (q_j / q_r) (q_r P - p_r) / tau                  outside it
//
// The sum outside the list is taken without the listed ids (a bit per id in LDS), so that q_r
// is no difference; the list's terms are computed in 64 bits, as the loss is a
// difference of larger ones.  Exponentials outside the list are in 32 bits (0 below 2^-126 of the largest there).
// Bound: memory; logits are read once and the gradient is
// written once (2048 x 32000 fp16 54.5 us, 4.8 TB/s of both; where a tenth of the rows does not count 59, at 4.2), by rows
// that are cut logits twice (333 x 128256 bf16 with 200 listed 44 us; 2048 x 128256 fp16 with 64 300, the loss alone 138).
#include "ends.h"

#include "common.h"
#include "elements.h"
#include "launch.h"
#include "lds_sync.h"

namespace aqlm {

namespace {

constexpr float kLog2e = 1.44269504088896341f, kLowest = -3.402823466e38f;

__device__ __forceinline__ float teacher_at(const DistillArgs& a, int64_t row, int k) {
  const int64_t i = row * a.teacher_row + k;
  if (a.teacher_dtype == kF16) return (float)((const _Float16*)a.teacher)[i];
  if (a.teacher_dtype == kBf16) return (float)((const __bf16*)a.teacher)[i];
  return ((const float*)a.teacher)[i];
}

// The listed ids of a row, in LDS; an entry belongs to the thread of its number.
struct List {
  double* p;     // teacher's mass
  int32_t* id;   // -1: no entry
  float* z;      // student's logit
  float* t;      // teacher's
};
// What a workgroup's waves bring together.
template <int WAVES>
struct Parts {
  float top[WAVES][2];   // largest teacher's and student's logit of the list
  double list[WAVES][4];  // teacher's mass, sum of p (log p' - z / tau), student's mass, how many ids differ
  float rest[WAVES][2];   // outside the list: maximum and sum relative to it
  int twice;              // an id is listed several times
};
// Of a row: student's log-sum-exp is log_all + m_all / tau.
struct Sums {
  double m_all, s_all, p_scale, mass, c_rest, loss;
  float m_rest;
};

// Outside the list: maximum and sum relative to it of one piece more, without the elements of `skip`.
template <int N, typename V>
__device__ __forceinline__ void add_piece(const V& v, int skip, float c, float& m, float& s) {
  float f[N], m1 = m;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    f[e] = skip >> e & 1 ? -INFINITY : (float)v[e];
    m1 = fmaxf(m1, f[e]);
  }
  s *= __builtin_amdgcn_exp2f((m - m1) * c);
  m = m1;
#pragma unroll
  for (int e = 0; e < N; ++e) s += __builtin_amdgcn_exp2f((f[e] - m) * c);
}

// A thread's first entry, loaded before anything else is known of the row.
struct Entry {
  int id;
  float t;
};
__device__ __forceinline__ Entry first_entry(const DistillArgs& a, int64_t row) {
  const int k = min((int)threadIdx.x, a.listed - 1);
  return {a.ids[row * a.ids_row + k], teacher_at(a, row, k)};
}

// The entries into LDS, the waves' maxima into parts.  logit(k, id): the student's; mark(id).
template <int THREADS, typename L, typename M>
__device__ __forceinline__ void read_list(const DistillArgs& a, int64_t row, const Entry& own, const List& list,
                                          Parts<THREADS / kWave>& parts, L logit, M mark) {
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  float top = -INFINITY, zmax = -INFINITY;
  for (int k = tid; k < a.listed; k += THREADS) {
    const int id = k == tid ? own.id : a.ids[row * a.ids_row + k];
    const float t = k == tid ? own.t : teacher_at(a, row, k);
    const bool held = (uint32_t)id < (uint32_t)a.vocab;
    list.id[k] = held ? id : -1;
    if (!held) continue;
    const float z = logit(k, id);
    list.z[k] = z;
    list.t[k] = t;
    top = fmaxf(top, t);
    zmax = fmaxf(zmax, z);
    mark(id);
  }
  if (wave * kWave < a.listed) {
    top = wave_max(top);
    zmax = wave_max(zmax);
    if (lane == 0) {
      parts.top[wave][0] = top;
      parts.top[wave][1] = zmax;
    }
  }
}

// The list's sums, in 64 bits.  With teacher_lse log p' is log p, without it p and log p' are
// relative to the largest.
// firstly(k, id): whether entry k is the first of its id.
template <int THREADS, typename F>
__device__ __forceinline__ void sum_list(const DistillArgs& a, int64_t row, const List& list,
                                         Parts<THREADS / kWave>& parts, double& zmax, F firstly) {
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const double inv = 1.0 / (double)a.tau;
  float top = -INFINITY, z0 = -INFINITY;
#pragma unroll
  for (int w = 0; w < THREADS / kWave; ++w) {
    if (w * kWave >= a.listed) break;
    top = fmaxf(top, parts.top[w][0]);
    z0 = fmaxf(z0, parts.top[w][1]);
  }
  zmax = (double)fmaxf(z0, kLowest);  // (masked ones: -inf relative to it)
  if (wave * kWave >= a.listed) return;
  const double shift = a.teacher_lse != nullptr ? (double)a.teacher_lse[row] : top == -INFINITY ? 0.0 : (double)top * inv;
  double sum[4] = {0.0, 0.0, 0.0, 0.0};
  for (int k = tid; k < a.listed; k += THREADS) {
    const int id = list.id[k];
    if (id < 0) continue;
    const double lp = (double)list.t[k] * inv - shift, p = exp(lp), z = ((double)list.z[k] - zmax) * inv;
    list.p[k] = p;
    sum[0] += p;
    if (p != 0.0) sum[1] += p * (lp - z);
    if (firstly(k, id)) {
      sum[2] += exp(z);
      sum[3] += 1.0;
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    sum[k] = wave_sum64(sum[k]);
    if (lane == 0) parts.list[wave][k] = sum[k];
  }
}

template <int WAVES>
__device__ __forceinline__ void add_waves(const DistillArgs& a, const Parts<WAVES>& parts, double (&sum)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) sum[k] = 0.0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w * kWave >= a.listed) break;
#pragma unroll
    for (int k = 0; k < 4; ++k) sum[k] += parts.list[w][k];
  }
}

// Loss and the gradient's factors from the list's sums and the rest's (m, s).
__device__ __forceinline__ Sums join(const DistillArgs& a, const double (&sum)[4], double zmax, float m, double s) {
  const double inv = 1.0 / (double)a.tau;
  Sums r;
  r.m_rest = m;
  // relative to the larger of the two maxima
  const double by = exp(-fabs((double)m - zmax) * inv), listed = zmax >= (double)m ? sum[2] : sum[2] != 0.0 ? sum[2] * by : 0.0;
  const double rest = zmax >= (double)m ? (s != 0.0 ? s * by : 0.0) : s;
  r.m_all = fmax((double)m, zmax);
  r.s_all = listed + rest;
  // (the list's logits are relative to zmax in the sum of p (log p - z / tau))
  const double log_all = log(r.s_all) + (r.m_all - zmax) * inv;
  r.p_scale = 1.0;
  r.mass = sum[0];
  if (a.teacher_lse != nullptr) {
    const double p_rest = sum[3] == (double)a.vocab ? 0.0 : sum[0] == sum[0] ? fmax(1.0 - sum[0], 0.0) : sum[0];
    const double q_rest = rest / r.s_all;  // (0 where it is below all numbers; not so its logarithm in the loss)
    r.mass = sum[0] + p_rest;
    r.loss = sum[0] != 0.0 ? sum[1] + sum[0] * log_all : 0.0;
    if (p_rest != 0.0) r.loss += p_rest * (log(p_rest * r.s_all / s) - ((double)m - r.m_all) * inv);
    r.c_rest = q_rest * r.mass - p_rest;
  } else if (sum[0] != 0.0) {
    r.p_scale = 1.0 / sum[0];
    r.mass = 1.0;
    r.loss = sum[1] * r.p_scale - log(sum[0]) + log_all;
    r.c_rest = rest / r.s_all;
  } else {  // nothing is listed
    r.loss = r.c_rest = 0.0;
  }
  // (nothing outside the list: 0; a row without a softmax, all of it masked: NaN)
  r.c_rest = s != 0.0 || r.c_rest != r.c_rest ? r.c_rest / s : 0.0;
  return r;
}

// A listed id's gradient.
template <typename T>
__device__ __forceinline__ T listed_gradient(const Sums& r, float z, double p, double inv, double scale) {
  return (T)(float)((exp(((double)z - r.m_all) * inv) / r.s_all * r.mass - p * r.p_scale) * scale);
}

template <int TY>
__device__ __forceinline__ typename Elem<TY>::V gradient(const typename Elem<TY>::V& v, float m, float c, float by) {
  typename Elem<TY>::V g;
#pragma unroll
  for (int e = 0; e < kPiece<TY>; ++e)
    g[e] = (typename Elem<TY>::T)(__builtin_amdgcn_exp2f(((float)v[e] - m) * c) * by);
  return g;
}

// Zero loss and gradient of a token that does not count, pieces [i0, i1) of the row.
template <int TY, int THREADS>
__device__ __forceinline__ void write_zeros(void* out, int i0, int i1, int vocab) {
  typename Elem<TY>::V zero;
#pragma unroll
  for (int e = 0; e < kPiece<TY>; ++e) zero[e] = (typename Elem<TY>::T)0.f;
  if (out != nullptr)
    for (int i = i0 + threadIdx.x; i < i1; i += THREADS) store_piece<TY>(out, i * kPiece<TY>, vocab, zero);
}

__device__ __forceinline__ List list_at(const DistillArgs& a, uint8_t* lds) {
  List list;
  list.p = (double*)lds;
  list.id = (int32_t*)(list.p + a.listed);
  list.z = (float*)(list.id + a.listed);
  list.t = list.z + a.listed;
  return list;
}
constexpr int kListBytes = 20;  // of LDS an entry

// One workgroup a row, NV pieces of 16 bytes a thread in registers.  A row's last piece ends at
// its end and may begin inside the one before: what both hold counts for the first and is written
// alike by both.
template <int TY, int THREADS, int NV>
__global__ void __launch_bounds__(THREADS, 4) k_distill(DistillArgs a) {
  typedef typename Elem<TY>::T T;
  typedef typename Elem<TY>::V V;
  constexpr int N = kPiece<TY>, kAll = (1 << N) - 1, kWaves = THREADS / kWave;
  extern __shared__ __align__(16) uint8_t lds[];
  __shared__ Parts<kWaves> parts;
  const List list = list_at(a, lds);
  uint32_t* const bits = (uint32_t*)(list.t + a.listed);  // a bit per id: listed, or past the vocabulary
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int64_t row = blockIdx.x;
  const T* const in = (const T*)a.logits + row * a.logits_row;
  T* const out = a.grad != nullptr ? (T*)a.grad + row * a.grad_row : nullptr;
  const int pieces = (a.vocab + N - 1) / N;
  const Entry own = first_entry(a, row);
  const float weight = a.weights != nullptr ? a.weights[row] : 1.f;
  if (weight == 0.f) {  // its logits are not looked at
    if (tid == 0) a.loss[row] = 0.f;
    return write_zeros<TY, THREADS>(out, 0, pieces, a.vocab);
  }
  auto place = [&](int i) { return min(i * N, a.vocab - N); };
  V x[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) x[j] = *(const V*)(in + place(tid + j * THREADS));
  const int words = (a.vocab + 31) / 32;
  for (int i = tid; i < words; i += THREADS) bits[i] = i == words - 1 && (a.vocab & 31) != 0 ? ~0u << (a.vocab & 31) : 0u;
  if (tid == 0) parts.twice = 0;
  lds_barrier();
  read_list<THREADS>(a, row, own, list, parts, [&](int, int id) { return (float)in[id]; }, [&](int id) {
    if (atomicOr(&bits[id / 32], 1u << (id % 32)) >> (id % 32) & 1) parts.twice = 1;
  });
  lds_barrier();
  const bool dup = parts.twice != 0;
  double zmax;
  sum_list<THREADS>(a, row, list, parts, zmax, [&](int k, int id) {
    bool first = true;
    if (dup)
      for (int i = 0; i < k; ++i) first = first && list.id[i] != id;
    return first;
  });

  int skip_last = 0;  // elements of the last piece that do not count
  {
    const int at = place(pieces - 1);
#pragma unroll
    for (int e = 0; e < N; ++e)
      skip_last |= (int)(at + e < (pieces - 1) * N || (bits[(at + e) / 32] >> ((at + e) % 32) & 1)) << e;
  }
  const float c = kLog2e / a.tau;
  float m = kLowest, s = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if (NV > 4) asm volatile("" : "+v"(x[j]), "+v"(s), "+v"(m));  // (all at once would take too many registers)
    const int i = tid + j * THREADS;
    int skip = (int)(((const uint8_t*)bits)[min(i, pieces - 1) * N / 8] >> (i * N % 8)) & kAll;
    skip = i < pieces - 1 ? skip : i == pieces - 1 ? skip_last : kAll;
    add_piece<N>(x[j], skip, c, m, s);
  }
  const float m_wave = wave_max(m);
  s = wave_sum(s * __builtin_amdgcn_exp2f((m - m_wave) * c));
  if (lane == 0) {
    parts.rest[wave][0] = m_wave;
    parts.rest[wave][1] = s;
  }
  lds_barrier();
  m = kLowest;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) m = fmaxf(m, parts.rest[w][0]);
  double s_rest = 0.0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w)
    s_rest += (double)(parts.rest[w][1] * __builtin_amdgcn_exp2f((parts.rest[w][0] - m) * c));
  double sum[4];
  add_waves<kWaves>(a, parts, sum);
  const Sums r = join(a, sum, zmax, m, s_rest);
  if (tid == 0) a.loss[row] = (float)r.loss;
  if (out == nullptr) return;
  const double scale = (double)weight / (double)a.tau;
  const float by = (float)(r.c_rest * scale);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    asm volatile("" : "+v"(x[j]));  // (otherwise the converted elements are kept, which spills)
    const int i = tid + j * THREADS;
    if (i < pieces) *(V*)(out + place(i)) = gradient<TY>(x[j], m, c, by);
  }
  __syncthreads();  // the listed ids' gradients go over what was written there
  const double inv = 1.0 / (double)a.tau;
  for (int k = tid; k < a.listed; k += THREADS) {
    const int id = list.id[k];
    if (id < 0) continue;
    double p = list.p[k];
    if (dup) {  // one that is listed several times: their sum
      p = 0.0;
      for (int i = 0; i < a.listed; ++i) p += list.id[i] == id ? list.p[i] : 0.0;
    }
    out[id] = listed_gradient<T>(r, list.z[k], p, inv, scale);
  }
}

// Rows that are cut: NV pieces a thread of a slice.  One launch makes the slices' maxima and sums
// outside the list and, by a workgroup of its own, the list's; another writes the gradient.
constexpr int kSliceThreads = 256;

// Slots of a table of the listed ids.
inline __host__ __device__ int table_slots(int listed) {
  int n = 64;
  while (n < 2 * listed) n <<= 1;
  return n;
}

template <int TY>
__device__ __forceinline__ void sum_row_list(const DistillArgs& a, int64_t row, uint8_t* lds) {
  typedef typename Elem<TY>::T T;
  constexpr int THREADS = kSliceThreads;
  __shared__ Parts<THREADS / kWave> parts;
  const List list = list_at(a, lds);
  // the first entry of an id: by a table of ids, linear probing
  const int slots = table_slots(a.listed), tid = threadIdx.x;
  int32_t* const key = (int32_t*)(list.t + a.listed);  // [slots]: id, -1 free
  int32_t* const first = key + slots;                  // [slots]: its first entry
  const T* const in = (const T*)a.logits + row * a.logits_row;
  for (int i = tid; i < slots; i += THREADS) {
    key[i] = -1;
    first[i] = INT32_MAX;
  }
  if (tid == 0) parts.twice = 0;
  lds_barrier();
  auto slot_of = [&](int id) {  // (at most half of the slots are taken)
    int at = (int)((uint32_t)id * 2654435761u) & (slots - 1);
    for (;;) {
      const int was = atomicCAS(&key[at], -1, id);
      if (was == -1 || was == id) return at;
      at = (at + 1) & (slots - 1);
    }
  };
  read_list<THREADS>(a, row, first_entry(a, row), list, parts, [&](int, int id) { return (float)in[id]; }, [&](int) {});
  lds_barrier();
  for (int k = tid; k < a.listed; k += THREADS)
    if (list.id[k] >= 0 && atomicMin(&first[slot_of(list.id[k])], k) != INT32_MAX) parts.twice = 1;
  lds_barrier();
  double zmax;
  sum_list<THREADS>(a, row, list, parts, zmax, [&](int k, int id) { return first[slot_of(id)] == k; });
  for (int k = tid; k < a.listed; k += THREADS) {
    if (list.id[k] < 0) continue;
    a.listed_mass[row * a.listed + k] = list.p[k];
    a.listed_logits[row * a.listed + k] = list.z[k];
  }
  lds_barrier();
  if (tid != 0) return;
  DistillRow r;
  add_waves<THREADS / kWave>(a, parts, r.sum);
  r.zmax = zmax;
  r.twice = parts.twice;
  a.row_lists[row] = r;
}

template <int TY, int NV>
__global__ void __launch_bounds__(kSliceThreads) k_distill_slices(DistillArgs a) {
  typedef typename Elem<TY>::T T;
  typedef typename Elem<TY>::V V;
  constexpr int N = kPiece<TY>, kAll = (1 << N) - 1, THREADS = kSliceThreads, kWaves = THREADS / kWave;
  constexpr int kCount = NV * THREADS * N, kWords = kCount / 32;
  extern __shared__ __align__(16) uint8_t lds[];
  __shared__ uint32_t bits[kWords];
  __shared__ float rest[kWaves][2];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, slices = gridDim.x - 1;
  const int64_t row = a.row0 + blockIdx.y;
  if (a.weights != nullptr && a.weights[row] == 0.f) return;
  if (blockIdx.x == 0) return sum_row_list<TY>(a, row, lds);  // (the longest: first)
  const int slice = blockIdx.x - 1, from = slice * kCount;
  const T* const in = (const T*)a.logits + row * a.logits_row;
  V x[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int at = from + (tid + j * THREADS) * N;
    x[j] = load_piece<TY>(in, min(at, a.vocab), a.vocab);
  }
  // (elements past the end count as listed)
  for (int i = tid; i < kWords; i += THREADS) {
    const int left = a.vocab - from - i * 32;
    bits[i] = left >= 32 ? 0u : left <= 0 ? ~0u : ~0u << left;
  }
  lds_barrier();
  for (int k = tid; k < a.listed; k += THREADS) {
    const int id = a.ids[row * a.ids_row + k];
    const uint32_t at = (uint32_t)(id - from);
    if ((uint32_t)id < (uint32_t)a.vocab && at < (uint32_t)kCount) atomicOr(&bits[at / 32], 1u << (at % 32));
  }
  lds_barrier();
  const float c = kLog2e / a.tau;
  float m = kLowest, s = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if (NV > 4) asm volatile("" : "+v"(x[j]), "+v"(s), "+v"(m));  // (all at once would take too many registers)
    const int i = tid + j * THREADS;
    add_piece<N>(x[j], (int)(((const uint8_t*)bits)[i * N / 8] >> (i * N % 8)) & kAll, c, m, s);
  }
  const float m_wave = wave_max(m);
  s = wave_sum(s * __builtin_amdgcn_exp2f((m - m_wave) * c));
  if (lane == 0) {
    rest[wave][0] = m_wave;
    rest[wave][1] = s;
  }
  lds_barrier();
  if (tid != 0) return;
  m = kLowest;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) m = fmaxf(m, rest[w][0]);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s += rest[w][1] * __builtin_amdgcn_exp2f((rest[w][0] - m) * c);
  a.slices[row * slices + slice] = DistillSlice{m, s};
}

// NT: the gradient goes past the L2s.  Where it is more than they hold, that leaves the logits in the caches between
// the launches (400 x 128256 fp32 125 -> 105 us, 333 x 128256 bf16 50 -> 44; whole rows, read once: 54.5 -> 56.5).
constexpr int64_t kStreamBytes = 32 << 20;
template <int TY, int NV, bool NT>
__global__ void __launch_bounds__(kSliceThreads) k_distill_grad(DistillArgs a) {
  typedef typename Elem<TY>::T T;
  typedef typename Elem<TY>::V V;
  constexpr int N = kPiece<TY>, THREADS = kSliceThreads;
  const int tid = threadIdx.x, lane = tid % kWave, slices = gridDim.x;
  const int64_t row = a.row0 + blockIdx.y;
  const T* const in = (const T*)a.logits + row * a.logits_row;
  T* const out = a.grad != nullptr ? (T*)a.grad + row * a.grad_row : nullptr;
  const int first = blockIdx.x * NV * THREADS, from = first * N;
  const float weight = a.weights != nullptr ? a.weights[row] : 1.f;
  if (weight == 0.f) {
    if (tid == 0 && blockIdx.x == 0) a.loss[row] = 0.f;
    return write_zeros<TY, THREADS>(out, first, min((a.vocab + N - 1) / N, first + NV * THREADS), a.vocab);
  }
  V x[NV];
  if (out != nullptr) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = from + (tid + j * THREADS) * N;
      x[j] = load_piece<TY>(in, min(at, a.vocab), a.vocab);
    }
  }
  DistillSlice own{kLowest, 0.f};  // (a lane has a slice)
  if (lane < slices) own = a.slices[row * slices + lane];
  const DistillRow l = a.row_lists[row];
  const float c = kLog2e / a.tau, m = wave_max(own.m);
  const double s_rest = wave_sum64((double)(own.s * __builtin_amdgcn_exp2f((own.m - m) * c)));
  const Sums r = join(a, l.sum, l.zmax, m, s_rest);
  if (tid == 0 && blockIdx.x == 0) a.loss[row] = (float)r.loss;
  if (out == nullptr) return;
  const double scale = (double)weight / (double)a.tau, inv = 1.0 / (double)a.tau;
  const float by = (float)(r.c_rest * scale);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int at = from + (tid + j * THREADS) * N;
    if (at < a.vocab) store_piece<TY, NT>(out, at, a.vocab, gradient<TY>(x[j], m, c, by));
  }
  __syncthreads();  // the listed ids' gradients go over what was written there
  const int32_t* const ids = a.ids + row * a.ids_row;
  const double* const mass = a.listed_mass + row * a.listed;
  for (int k = tid; k < a.listed; k += THREADS) {
    const int id = ids[k];
    if ((uint32_t)id >= (uint32_t)a.vocab || (uint32_t)(id - from) >= (uint32_t)(NV * THREADS * N)) continue;
    double p = mass[k];
    if (l.twice) {  // one that is listed several times: their sum
      p = 0.0;
      for (int i = 0; i < a.listed; ++i) p += ids[i] == id ? mass[i] : 0.0;
    }
    out[id] = listed_gradient<T>(r, a.listed_logits[row * a.listed + k], p, inv, scale);
  }
}

template <int TY, int THREADS, int NV>
hipError_t launch_rows(const DistillArgs& a, hipStream_t s) {
  const int lds = a.listed * kListBytes + (a.vocab + 31) / 32 * 4;
  const hipError_t e = allow_dynamic_lds((const void*)k_distill<TY, THREADS, NV>, lds);
  if (e != hipSuccess) return e;
  k_distill<TY, THREADS, NV><<<(unsigned)a.rows, THREADS, lds, s>>>(a);
  return hipGetLastError();
}

template <int TY, int NV>
hipError_t launch_slices(DistillArgs a, int slices, hipStream_t s) {
  const int lds = a.listed * kListBytes + table_slots(a.listed) * 8;
  hipError_t e = allow_dynamic_lds((const void*)k_distill_slices<TY, NV>, lds);
  for (a.row0 = 0; a.row0 < a.rows && e == hipSuccess; a.row0 += 65535) {
    const unsigned n = (unsigned)(a.rows - a.row0 < 65535 ? a.rows - a.row0 : 65535);
    k_distill_slices<TY, NV><<<dim3((unsigned)slices + 1, n), kSliceThreads, lds, s>>>(a);
    if (a.rows * a.vocab * dtype_bytes(TY) > kStreamBytes)
      k_distill_grad<TY, NV, true><<<dim3((unsigned)slices, n), kSliceThreads, 0, s>>>(a);
    else
      k_distill_grad<TY, NV, false><<<dim3((unsigned)slices, n), kSliceThreads, 0, s>>>(a);
    e = hipGetLastError();
  }
  return e;
}

template <int TY>
hipError_t launch_typed(const DistillArgs& a, hipStream_t s) {
  const DistillCut cut = distill_cut(a.rows, a.vocab, TY);
  if (cut.slices > 0) return cut.pieces == 8 ? launch_slices<TY, 8>(a, cut.slices, s) : launch_slices<TY, 2>(a, cut.slices, s);
  const int pieces = (a.vocab + kPiece<TY> - 1) / kPiece<TY>;
  if (pieces <= 2 * 64) return launch_rows<TY, 64, 2>(a, s);
  if (pieces <= 8 * 64) return launch_rows<TY, 64, 8>(a, s);
  if (pieces <= 8 * 256) return launch_rows<TY, 256, 8>(a, s);
  if (pieces <= 16 * 256) return launch_rows<TY, 256, 16>(a, s);
  return launch_rows<TY, 512, 16>(a, s);
}

}  // namespace

// Rows stay whole where the registers of 512 threads hold one and there are two a CU: fewer leave CUs without work
// (333 x 128256 bf16 whole 74 us, cut 44; one row 28 and 12).  Slices are narrow where wide ones are fewer than four a
// CU.
DistillCut distill_cut(int64_t rows, int64_t vocab, int dtype) {
  const int n = dtype == kF32 ? 4 : 8;
  const int64_t pieces = (vocab + n - 1) / n;
  if (vocab >= n && pieces <= 16 * 512 && rows >= 2 * num_cus()) return {0, 0};
  const int64_t wide = (pieces + 8 * kSliceThreads - 1) / (8 * kSliceThreads);
  const int64_t narrow = (pieces + 2 * kSliceThreads - 1) / (2 * kSliceThreads);
  if (narrow <= kWave && rows * wide < 4 * num_cus()) return {(int)narrow, 2};
  return {(int)wide, 8};
}

hipError_t launch_distill(const DistillArgs& a, int dtype, hipStream_t s) {
  if (dtype == kF16) return launch_typed<kF16>(a, s);
  if (dtype == kBf16) return launch_typed<kBf16>(a, s);
  return launch_typed<kF32>(a, s);
}

}  // namespace aqlm
