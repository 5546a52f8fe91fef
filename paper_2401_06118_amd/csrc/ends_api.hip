// C ABI of the operators at the ends of a model and on its residual stream (declared in
// include/aqlm.h): argument validation and dispatch.  Every check runs on the host before
// any launch; on an error nothing is launched.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/aqlm.h"
#include "ends.h"
#include "launch.h"
#include "rope.h"

namespace {

constexpr int64_t k2G = int64_t(1) << 31;
constexpr int64_t kMaxTokens = k2G - 65536;  // (places are held in 32 bits on the device)
constexpr int64_t kMaxTable = int64_t(1) << 30;
constexpr int64_t kMaxDim = int64_t(1) << 24;

bool multiple(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool known_dtype(int32_t t) { return t == AQLM_F16 || t == AQLM_BF16 || t == AQLM_F32; }
int status_of(hipError_t e) { return e == hipSuccess ? AQLM_OK : AQLM_ERR_HIP; }
bool element_aligned(const void* p, int32_t dtype) { return multiple(p, (uintptr_t)aqlm::dtype_bytes(dtype)); }

// Strides of rows of n elements; rows of an output must not share addresses.
bool rows_in(int64_t stride) { return stride >= 0; }
bool rows_out(int64_t stride, int64_t rows, int64_t n) { return stride >= (rows > 1 ? n : 0); }

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

struct EmbedWorkspace {
  size_t counters, held, order, first, last, occurs, parts, parts_row, bytes;
};
EmbedWorkspace embed_workspace(int64_t count, int64_t vocab, int64_t dim, int32_t dtype) {
  EmbedWorkspace w{};
  const size_t units = (size_t)((count + aqlm::kEmbedUnit - 1) / aqlm::kEmbedUnit);
  const size_t places = up16((size_t)count * 4);
  w.counters = 0;
  w.held = up16(units * (size_t)aqlm::embed_grad_column_blocks((int32_t)dim, dtype) * 4);
  w.order = w.held + 16;
  w.first = w.order + places;
  w.last = w.first + places;
  w.occurs = w.last + places;
  w.parts = w.occurs + up16((size_t)aqlm::embed_grad_marks(vocab));
  w.parts_row = ((size_t)dim + 7) / 8 * 8;
  w.bytes = w.parts + units * 2 * w.parts_row * 4;
  return w;
}

// Slices of a launch over rows that are cut.
int64_t sample_slices(int64_t rows, int64_t vocab) {
  const int64_t slices = (vocab + aqlm::kSampleSlice - 1) / aqlm::kSampleSlice;
  return std::min(rows, aqlm::kSampleSlices / slices) * slices;
}

bool embed_sizes(int64_t count, int64_t vocab, int64_t dim) {
  return count >= 0 && count <= kMaxTokens && vocab > 0 && vocab <= kMaxTable && dim > 0 && dim <= kMaxDim;
}

int check_norm(const aqlm_norm* n, int64_t rows, int64_t dim, int32_t dtype) {
  if (!known_dtype(dtype)) return AQLM_ERR_UNSUPPORTED;
  if (rows < 0 || dim <= 0 || dim > aqlm::kNormMaxDim || !(n->eps >= 0.f)) return AQLM_ERR_SHAPE;
  if (!element_aligned(n->weight, dtype) || !element_aligned(n->bias, dtype)) return AQLM_ERR_ALIGN;
  return AQLM_OK;
}

}  // namespace

extern "C" {

int aqlm_embed(const void* table, int64_t table_stride, const int32_t* tokens, void* out, int64_t out_stride,
               int32_t dtype, int64_t count, int64_t vocab, int64_t dim, float scale, void* stream) {
  if (!known_dtype(dtype)) return AQLM_ERR_UNSUPPORTED;
  if (!embed_sizes(count, vocab, dim) || !rows_in(table_stride) || !rows_out(out_stride, count, dim)) return AQLM_ERR_SHAPE;
  if (count == 0) return AQLM_OK;
  if (!table || !tokens || !out) return AQLM_ERR_NULL;
  if (!element_aligned(table, dtype) || !element_aligned(out, dtype) || !multiple(tokens, 4)) return AQLM_ERR_ALIGN;
  aqlm::EmbedArgs a{};
  a.table = table;
  a.out = out;
  a.tokens = tokens;
  a.table_row = table_stride;
  a.out_row = out_stride;
  a.count = count;
  a.vocab = (int32_t)vocab;
  a.dim = (int32_t)dim;
  a.scale = scale;
  return status_of(aqlm::launch_embed(a, dtype, (hipStream_t)stream));
}

size_t aqlm_embed_backward_workspace_bytes(int64_t count, int64_t vocab, int64_t dim, int32_t dtype) {
  if (!embed_sizes(count, vocab, dim) || !known_dtype(dtype)) return 0;
  return embed_workspace(count, vocab, dim, dtype).bytes;
}

int aqlm_embed_backward(const void* dout, int64_t dout_stride, const int32_t* tokens, void* grad, int64_t grad_stride,
                        int32_t dtype, int32_t grad_dtype, int64_t count, int64_t vocab, int64_t dim, float scale,
                        void* workspace, size_t workspace_bytes, void* stream) {
  if (!known_dtype(dtype) || (grad_dtype != dtype && grad_dtype != AQLM_F32)) return AQLM_ERR_UNSUPPORTED;
  if (!embed_sizes(count, vocab, dim) || !rows_in(dout_stride) || !rows_out(grad_stride, vocab, dim)) return AQLM_ERR_SHAPE;
  if (!grad || !workspace || (count > 0 && (!dout || !tokens))) return AQLM_ERR_NULL;
  if (!element_aligned(dout, dtype) || !element_aligned(grad, grad_dtype) || !multiple(tokens, 4) ||
      !multiple(workspace, 16))
    return AQLM_ERR_ALIGN;
  const EmbedWorkspace w = embed_workspace(count, vocab, dim, dtype);
  if (workspace_bytes < w.bytes) return AQLM_ERR_WORKSPACE;
  uint8_t* const ws = static_cast<uint8_t*>(workspace);
  aqlm::EmbedGradArgs a{};
  a.dout = dout;
  a.out = grad;
  a.tokens = tokens;
  a.dout_row = dout_stride;
  a.out_row = grad_stride;
  a.tokens_count = (int32_t)count;
  a.vocab = (int32_t)vocab;
  a.dim = (int32_t)dim;
  a.scale = scale;
  a.counters = reinterpret_cast<uint32_t*>(ws + w.counters);
  a.held = reinterpret_cast<int32_t*>(ws + w.held);
  a.order = reinterpret_cast<int32_t*>(ws + w.order);
  a.first = reinterpret_cast<int32_t*>(ws + w.first);
  a.last = reinterpret_cast<int32_t*>(ws + w.last);
  a.occurs = ws + w.occurs;
  a.parts = reinterpret_cast<float*>(ws + w.parts);
  a.parts_row = (int64_t)w.parts_row;
  return status_of(aqlm::launch_embed_grad(a, dtype, grad_dtype, (hipStream_t)stream));
}

int aqlm_layer_norm(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, void* out,
                    int64_t out_stride, void* sum, int64_t sum_stride, int32_t dtype, int64_t rows, int64_t dim,
                    const aqlm_norm* n, void* stream) {
  if (!n || (sum && !residual)) return AQLM_ERR_NULL;
  if (const int e = check_norm(n, rows, dim, dtype)) return e;
  if (!rows_in(x_stride) || (residual && !rows_in(residual_stride)) || !rows_out(out_stride, rows, dim) ||
      (sum && !rows_out(sum_stride, rows, dim)))
    return AQLM_ERR_SHAPE;
  if (rows == 0) return AQLM_OK;
  if (!x || !out) return AQLM_ERR_NULL;
  if (sum == out) return AQLM_ERR_SHAPE;
  for (const void* p : {x, residual, (const void*)out, (const void*)sum})
    if (!element_aligned(p, dtype)) return AQLM_ERR_ALIGN;
  aqlm::NormArgs a{};
  a.x = x;
  a.residual = residual;
  a.weight = n->weight;
  a.bias = n->bias;
  a.out = out;
  a.sum = sum;
  a.x_row = x_stride;
  a.residual_row = residual_stride;
  a.out_row = out_stride;
  a.sum_row = sum_stride;
  a.rows = rows;
  a.dim = (int32_t)dim;
  a.rms = n->rms != 0;
  a.eps = n->eps;
  return status_of(aqlm::launch_norm(a, dtype, (hipStream_t)stream));
}

size_t aqlm_layer_norm_backward_workspace_bytes(int64_t dim) {
  if (dim <= 0 || dim > aqlm::kNormMaxDim) return 0;
  return (size_t)aqlm::norm_grad_parts() * 2 * (size_t)dim * 4;
}

int aqlm_layer_norm_backward(const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, const void* dsum,
                             int64_t dsum_stride, void* dx, int64_t dx_stride, float* dweight, float* dbias,
                             int32_t dtype, int64_t rows, int64_t dim, const aqlm_norm* n, void* workspace,
                             size_t workspace_bytes, void* stream) {
  if (!n) return AQLM_ERR_NULL;
  if (const int e = check_norm(n, rows, dim, dtype)) return e;
  if (!rows_in(dy_stride) || !rows_in(x_stride) || (dsum && !rows_in(dsum_stride)) || !rows_out(dx_stride, rows, dim))
    return AQLM_ERR_SHAPE;
  if (rows > 0 && (!dy || !x || !dx)) return AQLM_ERR_NULL;
  const bool sums = dweight || dbias;
  if (sums && !workspace) return AQLM_ERR_NULL;
  for (const void* p : {dy, x, dsum, (const void*)dx})
    if (!element_aligned(p, dtype)) return AQLM_ERR_ALIGN;
  if (!multiple(dweight, 4) || !multiple(dbias, 4) || (sums && !multiple(workspace, 16))) return AQLM_ERR_ALIGN;
  if (sums && workspace_bytes < aqlm_layer_norm_backward_workspace_bytes(dim)) return AQLM_ERR_WORKSPACE;
  aqlm::NormGradArgs a{};
  a.dy = dy;
  a.x = x;
  a.weight = n->weight;
  a.dsum = dsum;
  a.out = dx;
  a.dweight = dweight;
  a.dbias = dbias;
  a.parts = static_cast<float*>(workspace);
  a.dy_row = dy_stride;
  a.x_row = x_stride;
  a.dsum_row = dsum_stride;
  a.out_row = dx_stride;
  a.rows = rows;
  a.dim = (int32_t)dim;
  a.rms = n->rms != 0;
  a.eps = n->eps;
  return status_of(aqlm::launch_norm_grad(a, dtype, (hipStream_t)stream));
}

size_t aqlm_distill_loss_workspace_bytes(int64_t rows, int64_t vocab, int64_t listed, int32_t dtype) {
  if (rows <= 0 || rows > aqlm::kDistillMaxRows || vocab <= 0 || vocab > aqlm::kDistillMaxVocab || listed <= 0 ||
      listed > aqlm::kDistillMaxListed || !known_dtype(dtype))
    return 0;
  const aqlm::DistillCut cut = aqlm::distill_cut(rows, vocab, dtype);
  return cut.slices == 0 ? 0 : (size_t)rows * (sizeof(aqlm::DistillRow) + (size_t)cut.slices * sizeof(aqlm::DistillSlice) + (size_t)listed * 12);
}

int aqlm_distill_loss(const void* logits, int64_t logits_stride, int32_t dtype, const void* teacher,
                      int64_t teacher_stride, int32_t teacher_dtype, const int32_t* ids, int64_t ids_stride,
                      const float* teacher_lse, const float* weights, float temperature, float* loss, void* grad,
                      int64_t grad_stride, int64_t rows, int64_t vocab, int64_t listed, void* workspace,
                      size_t workspace_bytes, void* stream) {
  if (!known_dtype(dtype) || !known_dtype(teacher_dtype)) return AQLM_ERR_UNSUPPORTED;
  if (rows < 0 || rows > aqlm::kDistillMaxRows || vocab <= 0 || vocab > aqlm::kDistillMaxVocab || listed <= 0 ||
      listed > aqlm::kDistillMaxListed || !rows_in(logits_stride) || !rows_in(teacher_stride) || !rows_in(ids_stride) ||
      (grad && !rows_out(grad_stride, rows, vocab)))
    return AQLM_ERR_SHAPE;
  if (!(temperature > 0.f) || !std::isfinite(1.44269504f / temperature) || !std::isfinite(temperature)) return AQLM_ERR_SHAPE;
  if (rows == 0) return AQLM_OK;
  if (!logits || !teacher || !ids || !loss) return AQLM_ERR_NULL;
  if (!element_aligned(logits, dtype) || !element_aligned(grad, dtype) || !element_aligned(teacher, teacher_dtype))
    return AQLM_ERR_ALIGN;
  for (const void* p : {(const void*)ids, (const void*)teacher_lse, (const void*)weights, (const void*)loss})
    if (!multiple(p, 4)) return AQLM_ERR_ALIGN;
  const size_t need = aqlm_distill_loss_workspace_bytes(rows, vocab, listed, dtype);
  if (need > 0 && !workspace) return AQLM_ERR_NULL;
  if (need > 0 && !multiple(workspace, 16)) return AQLM_ERR_ALIGN;
  if (workspace_bytes < need) return AQLM_ERR_WORKSPACE;
  aqlm::DistillArgs a{};
  a.logits = logits;
  a.teacher = teacher;
  a.ids = ids;
  a.teacher_lse = teacher_lse;
  a.weights = weights;
  a.loss = loss;
  a.grad = grad;
  a.logits_row = logits_stride;
  a.teacher_row = teacher_stride;
  a.ids_row = ids_stride;
  a.grad_row = grad_stride;
  a.rows = rows;
  a.vocab = (int32_t)vocab;
  a.listed = (int32_t)listed;
  a.teacher_dtype = teacher_dtype;
  a.tau = temperature;
  if (need > 0) {
    a.row_lists = static_cast<aqlm::DistillRow*>(workspace);
    a.listed_mass = reinterpret_cast<double*>(a.row_lists + rows);
    a.slices = reinterpret_cast<aqlm::DistillSlice*>(a.listed_mass + rows * listed);
    a.listed_logits = reinterpret_cast<float*>(a.slices + rows * aqlm::distill_cut(rows, vocab, dtype).slices);
  }
  return status_of(aqlm::launch_distill(a, dtype, (hipStream_t)stream));
}

size_t aqlm_sample_workspace_bytes(int64_t rows, int64_t vocab, const aqlm_sampling* r) {
  if (rows <= 0 || vocab <= 0 || vocab > aqlm::kSampleMaxVocab || !r || !aqlm::sample_cut(vocab, r->top_k != nullptr))
    return 0;
  return (size_t)sample_slices(rows, vocab) * aqlm::kSampleSliceBytes;
}

int aqlm_sample(const void* logits, int64_t logits_stride, int32_t dtype, int64_t rows, int64_t vocab,
                const float* uniform, const aqlm_sampling* r, int32_t* tokens, float* logprob, void* workspace,
                size_t workspace_bytes, void* stream) {
  if (!r) return AQLM_ERR_NULL;
  if (!known_dtype(dtype)) return AQLM_ERR_UNSUPPORTED;
  if (rows < 0 || rows > aqlm::kSampleMaxRows || vocab <= 0 || vocab > aqlm::kSampleMaxVocab || !rows_in(logits_stride))
    return AQLM_ERR_SHAPE;
  if (rows == 0) return AQLM_OK;
  const size_t need = aqlm_sample_workspace_bytes(rows, vocab, r);
  if (!logits || !uniform || !tokens || (need > 0 && !workspace)) return AQLM_ERR_NULL;
  if (!element_aligned(logits, dtype) || (need > 0 && !multiple(workspace, 16))) return AQLM_ERR_ALIGN;
  if (workspace_bytes < need) return AQLM_ERR_WORKSPACE;
  for (const void* p : {(const void*)uniform, (const void*)r->temperature, (const void*)r->top_k, (const void*)r->top_p,
                        (const void*)r->min_p, (const void*)tokens, (const void*)logprob})
    if (!multiple(p, 4)) return AQLM_ERR_ALIGN;
  aqlm::SampleArgs a{};
  a.logits = logits;
  a.uniform = uniform;
  a.temperature = r->temperature;
  a.top_k = r->top_k;
  a.top_p = r->top_p;
  a.min_p = r->min_p;
  a.tokens = tokens;
  a.logprob = logprob;
  a.row = logits_stride;
  a.rows = (int32_t)rows;
  a.vocab = (int32_t)vocab;
  if (need > 0) {
    const size_t n = (size_t)sample_slices(rows, vocab);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    a.records = reinterpret_cast<aqlm::SampleRecord*>(ws);
    a.masses = reinterpret_cast<uint64_t*>(ws += n * sizeof(aqlm::SampleRecord));
    a.lists = reinterpret_cast<uint64_t*>(ws += n * aqlm::kSampleBins * 8);
    a.counts = reinterpret_cast<uint32_t*>(ws + n * aqlm::kSampleListed * 8);
  }
  return status_of(aqlm::launch_sample(a, dtype, (hipStream_t)stream));
}

}  // extern "C"
