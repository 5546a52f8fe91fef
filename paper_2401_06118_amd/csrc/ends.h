// The ends of a model and the norms of its residual stream: arguments of the kernels in
// embed.hip, norm.hip, distill.hip and sample.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sample_bins.h"

namespace aqlm {

// Row strides in elements.
struct EmbedArgs {
  const void* table;
  void* out;
  const int32_t* tokens;
  int64_t table_row, out_row, count;
  int32_t vocab, dim;
  float scale;
};

struct EmbedGradArgs {
  const void* dout;
  void* out;
  const int32_t* tokens;
  int64_t dout_row, out_row;
  int32_t tokens_count, vocab, dim;
  float scale;
  // workspace
  uint32_t* counters;  // [units][column blocks]
  int32_t* held;       // [1] tokens of the vocabulary
  int32_t* order;      // [tokens] places, those of one token together, ascending
  int32_t* first;      // [tokens] where the token's places begin in order,
  int32_t* last;       // [tokens] and end
  uint8_t* occurs;     // [embed_grad_marks]
  float* parts;        // [units][2][parts_row]
  int64_t parts_row;   // dim, to whole pieces
};

constexpr int kEmbedUnit = 16;  // places of `order` that a workgroup sums
int embed_grad_column_blocks(int32_t dim, int dtype);
int embed_grad_lg(int64_t vocab);
int64_t embed_grad_marks(int64_t vocab);

struct NormArgs {
  const void *x, *residual, *weight, *bias;
  void *out, *sum;
  int64_t x_row, residual_row, out_row, sum_row, rows;
  int32_t dim;
  bool rms;
  float eps;
};

constexpr int kNormMaxDim = 16384;

struct NormGradArgs {
  const void *dy, *x, *weight, *dsum;
  void* out;
  float *dweight, *dbias;
  float* parts;  // [norm_grad_parts()][dim] for each of dweight and dbias
  int64_t dy_row, x_row, dsum_row, out_row, rows;
  int32_t dim;
  bool rms;
  float eps;
};

int norm_grad_parts();  // at most

struct DistillArgs {
  const void *logits, *teacher;
  const int32_t* ids;
  const float *teacher_lse, *weights;
  float* loss;
  void* grad;  // or null
  int64_t logits_row, teacher_row, ids_row, grad_row, rows;
  int32_t vocab, listed, teacher_dtype;
  float tau;
  // workspace, where rows are cut
  struct DistillRow* row_lists;  // [rows]
  double* listed_mass;           // [rows][listed]
  float* listed_logits;          // [rows][listed]
  struct DistillSlice* slices;   // [rows][slices]
  int64_t row0;                  // a launch's first
};

// What a slice of a row has outside the list: largest logit, sum relative to it.
struct DistillSlice {
  float m, s;
};
// What a row's list adds up to; whether an id is listed several times.
struct DistillRow {
  double sum[4], zmax;
  int64_t twice;
};
// Slices of a row (0: rows are not cut), pieces of 16 bytes a thread of a slice has.
struct DistillCut {
  int slices, pieces;
};
DistillCut distill_cut(int64_t rows, int64_t vocab, int dtype);

constexpr int kDistillMaxListed = 2048;
constexpr int kDistillMaxVocab = 1 << 19;
constexpr int64_t kDistillMaxRows = (1 << 22) - 1;  // (a launch has fewer than 2^32 threads)

struct SampleArgs {
  const void* logits;
  const float *uniform, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* tokens;
  float* logprob;  // or null
  int64_t row;
  int32_t rows, vocab;
  // workspace, where a row is cut: [slices of a launch]
  struct SampleRecord* records;
  uint64_t* masses;  // [][kSampleBins]
  uint32_t* counts;  // [][kSampleBins]
  uint64_t* lists;   // [][kSampleListed]
};

// What a slice of a row holds.
struct SampleRecord {
  uint64_t mass;  // relative to its largest weight; where the largest is drawn: its first place
  float top;      // largest logit, or NaN
  int32_t cut;    // the list has all tokens of the bins up to this one
  int32_t listed;
  int32_t pad;
};

constexpr int kSampleRow = 32768;    // logits of a row that a workgroup holds at most
constexpr int kSampleSlice = 8192;   // logits of a slice
// Whether rows are cut into slices.  (A row of 32000 by one workgroup: 11 us with top-k, 40 with top-p, whose masses
// need every token's exponential; by slices 29.)
inline bool sample_cut(int64_t vocab, bool top_k) { return vocab > (top_k ? kSampleRow : kSampleSlice); }
constexpr int kSampleSlices = 4096;  // slices of a launch
constexpr int kSampleListed = 512;
constexpr size_t kSampleSliceBytes = sizeof(SampleRecord) + kSampleBins * 12 + kSampleListed * 8;
constexpr int kSampleMaxVocab = 1 << 19;
constexpr int64_t kSampleMaxRows = 1 << 20;

hipError_t launch_embed(const EmbedArgs& a, int dtype, hipStream_t s);
hipError_t launch_embed_grad(const EmbedGradArgs& a, int dtype, int out_dtype, hipStream_t s);
hipError_t launch_norm(const NormArgs& a, int dtype, hipStream_t s);
hipError_t launch_norm_grad(const NormGradArgs& a, int dtype, hipStream_t s);
hipError_t launch_distill(const DistillArgs& a, int dtype, hipStream_t s);
hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t s);

}  // namespace aqlm
