// C ABI of the operators around the products of a transformer block and of a
// decode step (declared in include/aqlm.h): argument validation and dispatch.
// Every check runs on the host before any launch; on an error nothing is launched.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/aqlm.h"
#include "attention.h"
#include "launch.h"
#include "logits.h"
#include "rope.h"

namespace {

static_assert(aqlm::kF16 == AQLM_F16 && aqlm::kBf16 == AQLM_BF16 && aqlm::kF32 == AQLM_F32, "types");
static_assert(aqlm::kAttnMaxSeqs == AQLM_MAX_SEQS, "sequences");

constexpr int64_t k2G = int64_t(1) << 31;

bool multiple(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool known_dtype(int32_t t) { return t == AQLM_F16 || t == AQLM_BF16 || t == AQLM_F32; }
int status_of(hipError_t e) { return e == hipSuccess ? AQLM_OK : AQLM_ERR_HIP; }

// An activation's pointer, heads and strides.  Outputs: tokens and heads that
// share addresses are refused.
int check_heads(const aqlm_heads* h, int64_t tokens, int32_t head_dim, int32_t dtype, bool output) {
  if (!h->data) return AQLM_ERR_NULL;
  if (h->heads <= 0 || h->token_stride < 0 || h->head_stride < 0 || tokens * h->heads >= k2G) return AQLM_ERR_SHAPE;
  if (output && ((tokens > 1 && h->token_stride < head_dim) || (h->heads > 1 && h->head_stride < head_dim)))
    return AQLM_ERR_SHAPE;
  if (!multiple(h->data, (uintptr_t)aqlm::dtype_bytes(dtype))) return AQLM_ERR_ALIGN;
  return AQLM_OK;
}

int check_rotation(const aqlm_rotation* r, int32_t head_dim, int32_t dtype) {
  if (r->rot < 0 || r->rot > head_dim || r->rot % 2 != 0) return AQLM_ERR_SHAPE;
  if (r->rot > 0) {
    if (!r->table) return AQLM_ERR_NULL;
    if (r->rows <= 0 || r->rows >= k2G) return AQLM_ERR_SHAPE;
    if (!multiple(r->table, 8)) return AQLM_ERR_ALIGN;
  }
  const uintptr_t unit = (uintptr_t)aqlm::dtype_bytes(dtype);
  if (!multiple(r->q_weight, unit) || !multiple(r->k_weight, unit)) return AQLM_ERR_ALIGN;
  return AQLM_OK;
}

void set_rotation(aqlm::RopeArgs& a, const aqlm_rotation* r, float sign) {
  a.table = r->table;
  a.rows = r->rot > 0 ? r->rows : 0;
  a.rot = r->rot;
  a.interleaved = r->interleaved != 0;
  a.eps = r->eps;
  a.sign = sign;
}

void set_side(aqlm::RopeSide& s, const aqlm_heads* in, const aqlm_heads* out, const void* weight) {
  s.in = in->data;
  s.in_token = in->token_stride;
  s.in_head = in->head_stride;
  s.heads = in->heads;
  s.weight = weight;
  if (out) {
    s.out = out->data;
    s.out_token = out->token_stride;
    s.out_head = out->head_stride;
  }
}

int check_cache(const aqlm_paged_cache* c) {
  if (!c->k || !c->v || !c->block_table || !c->kv_lens || !c->cu_new) return AQLM_ERR_NULL;
  if (c->pages <= 0 || c->pages >= k2G || c->table_width <= 0 || c->table_stride < 0 || c->seqs <= 0 ||
      c->seqs > AQLM_MAX_SEQS || c->kv_heads <= 0 || c->head_dim <= 0)
    return AQLM_ERR_SHAPE;
  if (c->page_size <= 0 || (c->page_size & (c->page_size - 1)) != 0) return AQLM_ERR_SHAPE;
  // (positions are held in 32 bits on the device)
  if ((int64_t)c->table_width * c->page_size >= k2G - 65536) return AQLM_ERR_SHAPE;
  for (const int64_t s : {c->k_page_stride, c->k_slot_stride, c->k_head_stride, c->v_page_stride, c->v_slot_stride,
                          c->v_head_stride})
    if (s < 0) return AQLM_ERR_SHAPE;
  if (!known_dtype(c->dtype)) return AQLM_ERR_UNSUPPORTED;
  if (!multiple(c->block_table, 4) || !multiple(c->kv_lens, 4) || !multiple(c->cu_new, 4)) return AQLM_ERR_ALIGN;
  const uintptr_t unit = (uintptr_t)aqlm::dtype_bytes(c->dtype);
  if (!multiple(c->k, unit) || !multiple(c->v, unit)) return AQLM_ERR_ALIGN;
  return AQLM_OK;
}

int page_shift(int32_t page_size) { return __builtin_ctz((unsigned)page_size); }

}  // namespace

extern "C" {

int aqlm_rotary_table(const double* inv_freq, int64_t rows, int32_t half, double scale, float* table, void* stream) {
  if (!inv_freq || !table) return AQLM_ERR_NULL;
  if (rows <= 0 || half <= 0 || rows >= k2G || rows * half >= k2G * 64) return AQLM_ERR_SHAPE;
  if (!multiple(inv_freq, 8) || !multiple(table, 8)) return AQLM_ERR_ALIGN;
  return status_of(aqlm::launch_rotary_table(inv_freq, rows, half, scale, table, (hipStream_t)stream));
}

int aqlm_rope(const aqlm_heads* q, const aqlm_heads* k, const aqlm_heads* q_out, const aqlm_heads* k_out,
              int32_t dtype, int64_t tokens, int32_t head_dim, const int32_t* positions, const aqlm_rotation* r,
              void* stream) {
  if (!q || !k || !q_out || !k_out || !r) return AQLM_ERR_NULL;
  if (!known_dtype(dtype)) return AQLM_ERR_UNSUPPORTED;
  if (tokens < 0 || tokens >= k2G || head_dim <= 0 || head_dim > 1024) return AQLM_ERR_SHAPE;
  if (tokens == 0) return AQLM_OK;
  if (!positions) return AQLM_ERR_NULL;
  if (q_out->heads != q->heads || k_out->heads != k->heads) return AQLM_ERR_SHAPE;
  const aqlm_heads* in[2] = {q, k};
  const aqlm_heads* out[2] = {q_out, k_out};
  for (int i = 0; i < 2; ++i) {
    if (const int e = check_heads(in[i], tokens, head_dim, dtype, false)) return e;
    if (const int e = check_heads(out[i], tokens, head_dim, dtype, true)) return e;
  }
  if (tokens * ((int64_t)q->heads + k->heads) >= k2G) return AQLM_ERR_SHAPE;
  if (const int e = check_rotation(r, head_dim, dtype)) return e;
  if (!multiple(positions, 4)) return AQLM_ERR_ALIGN;
  aqlm::RopeArgs a{};
  set_rotation(a, r, 1.f);
  set_side(a.side[0], q, q_out, r->q_weight);
  set_side(a.side[1], k, k_out, r->k_weight);
  a.positions = positions;
  a.tokens = (int32_t)tokens;
  a.head_dim = head_dim;
  return status_of(aqlm::launch_rope(a, dtype, false, (hipStream_t)stream));
}

size_t aqlm_rope_backward_workspace_bytes(int32_t head_dim) {
  if (head_dim <= 0 || head_dim > 1024) return 0;
  return (size_t)aqlm::rope_grad_blocks() * (size_t)head_dim * 4;
}

int aqlm_rope_backward(const aqlm_heads* dq, const aqlm_heads* dk, const aqlm_heads* q, const aqlm_heads* k,
                       const aqlm_heads* gq, const aqlm_heads* gk, float* gq_weight, float* gk_weight, int32_t dtype,
                       int64_t tokens, int32_t head_dim, const int32_t* positions, const aqlm_rotation* r,
                       void* workspace, size_t workspace_bytes, void* stream) {
  if (!dq || !dk || !gq || !gk || !r) return AQLM_ERR_NULL;
  if (!known_dtype(dtype)) return AQLM_ERR_UNSUPPORTED;
  if (tokens <= 0 || tokens >= k2G || head_dim <= 0 || head_dim > 1024) return AQLM_ERR_SHAPE;
  if (!positions) return AQLM_ERR_NULL;
  const aqlm_heads* grad[2] = {dq, dk};
  const aqlm_heads* x[2] = {q, k};
  const aqlm_heads* out[2] = {gq, gk};
  const void* weight[2] = {r->q_weight, r->k_weight};
  float* const dweight[2] = {gq_weight, gk_weight};
  if (const int e = check_rotation(r, head_dim, dtype)) return e;
  bool norm = false;
  for (int i = 0; i < 2; ++i) {
    if (const int e = check_heads(grad[i], tokens, head_dim, dtype, false)) return e;
    if (const int e = check_heads(out[i], tokens, head_dim, dtype, true)) return e;
    if (out[i]->heads != grad[i]->heads) return AQLM_ERR_SHAPE;
    if (!weight[i]) continue;
    norm = true;
    if (!x[i] || !dweight[i]) return AQLM_ERR_NULL;
    if (const int e = check_heads(x[i], tokens, head_dim, dtype, false)) return e;
    if (x[i]->heads != grad[i]->heads) return AQLM_ERR_SHAPE;
    if (!multiple(dweight[i], 4)) return AQLM_ERR_ALIGN;
  }
  if (tokens * ((int64_t)dq->heads + dk->heads) >= k2G) return AQLM_ERR_SHAPE;
  if (!multiple(positions, 4)) return AQLM_ERR_ALIGN;
  if (norm) {
    if (!workspace) return AQLM_ERR_NULL;
    if (workspace_bytes < aqlm_rope_backward_workspace_bytes(head_dim)) return AQLM_ERR_WORKSPACE;
    if (!multiple(workspace, 16)) return AQLM_ERR_ALIGN;
  }
  aqlm::RopeArgs a{};
  set_rotation(a, r, -1.f);
  a.positions = positions;
  a.tokens = (int32_t)tokens;
  a.head_dim = head_dim;
  a.parts = static_cast<float*>(workspace);
  // the sides with a norm in one launch, those without in another
  aqlm::RopeArgs plain = a;
  bool any_plain = false;
  for (int i = 0; i < 2; ++i) {
    if (weight[i]) {
      set_side(a.side[i], grad[i], out[i], weight[i]);
      a.side[i].x = x[i]->data;
      a.side[i].x_token = x[i]->token_stride;
      a.side[i].x_head = x[i]->head_stride;
      a.dweight[i] = dweight[i];
    } else {
      set_side(plain.side[i], grad[i], out[i], nullptr);
      any_plain = true;
    }
  }
  if (any_plain) {
    const hipError_t e = aqlm::launch_rope(plain, dtype, false, (hipStream_t)stream);
    if (e != hipSuccess) return AQLM_ERR_HIP;
  }
  if (!norm) return AQLM_OK;
  return status_of(aqlm::launch_rope_grad_norm(a, dtype, (hipStream_t)stream));
}

int aqlm_paged_append(const aqlm_heads* q, const aqlm_heads* k, const aqlm_heads* v, const aqlm_heads* q_out,
                      const aqlm_paged_cache* c, int64_t tokens, const aqlm_rotation* r, void* stream) {
  if (!k || !v || !c || !r || (q == nullptr) != (q_out == nullptr)) return AQLM_ERR_NULL;
  if (const int e = check_cache(c)) return e;
  if (c->head_dim > 1024 || tokens < 0 || tokens >= k2G) return AQLM_ERR_SHAPE;
  if (tokens == 0) return AQLM_OK;
  if (k->heads != c->kv_heads || v->heads != c->kv_heads) return AQLM_ERR_SHAPE;
  if (const int e = check_heads(k, tokens, c->head_dim, c->dtype, false)) return e;
  if (const int e = check_heads(v, tokens, c->head_dim, c->dtype, false)) return e;
  if (q) {
    if (const int e = check_heads(q, tokens, c->head_dim, c->dtype, false)) return e;
    if (const int e = check_heads(q_out, tokens, c->head_dim, c->dtype, true)) return e;
    if (q_out->heads != q->heads) return AQLM_ERR_SHAPE;
  }
  if (tokens * ((int64_t)(q ? q->heads : 0) + 2 * (int64_t)c->kv_heads) >= k2G) return AQLM_ERR_SHAPE;
  if (const int e = check_rotation(r, c->head_dim, c->dtype)) return e;
  aqlm::RopeArgs a{};
  set_rotation(a, r, 1.f);
  if (q) set_side(a.side[0], q, q_out, r->q_weight);
  set_side(a.side[1], k, nullptr, r->k_weight);
  set_side(a.side[2], v, nullptr, nullptr);
  a.side[1].out = c->k;
  a.side[2].out = c->v;
  a.page_stride[0] = c->k_page_stride;
  a.page_stride[1] = c->v_page_stride;
  a.slot_stride[0] = c->k_slot_stride;
  a.slot_stride[1] = c->v_slot_stride;
  a.cache_head[0] = c->k_head_stride;
  a.cache_head[1] = c->v_head_stride;
  a.tokens = (int32_t)tokens;
  a.head_dim = c->head_dim;
  a.block_table = c->block_table;
  a.kv_lens = c->kv_lens;
  a.cu_new = c->cu_new;
  a.table_stride = c->table_stride;
  a.seqs = c->seqs;
  a.pages = (int32_t)c->pages;
  a.page_shift = page_shift(c->page_size);
  a.table_width = c->table_width;
  return status_of(aqlm::launch_rope(a, c->dtype, true, (hipStream_t)stream));
}

size_t aqlm_paged_attention_workspace_bytes(int32_t head_dim) {
  if (head_dim <= 0 || head_dim > 256 || head_dim % 8 != 0) return 0;
  const int64_t step = 2 * (int64_t)aqlm::attention_step_grid() * aqlm::attention_step_place(head_dim);
  const int64_t chunk = 2 * (int64_t)aqlm::attention_chunk_grid(head_dim) * aqlm::attention_chunk_place(head_dim);
  return AQLM_ATTENTION_COUNTER_BYTES + (size_t)std::max(step, chunk) * 4;
}

int aqlm_paged_attention(const aqlm_heads* q, const aqlm_heads* out, float* lse, const aqlm_paged_cache* c,
                         int64_t tokens, int64_t max_new, float scale, int32_t causal, int32_t window,
                         void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !out || !c || !workspace) return AQLM_ERR_NULL;
  if (const int e = check_cache(c)) return e;
  if (c->dtype == AQLM_F32) return AQLM_ERR_UNSUPPORTED;
  if (c->head_dim > 256 || c->head_dim % 8 != 0) return AQLM_ERR_UNSUPPORTED;
  if (tokens < 0 || tokens >= k2G || max_new < 0 || window < 0 || !std::isfinite(scale * 1.44269504088896341f)) return AQLM_ERR_SHAPE;
  if (tokens == 0) return AQLM_OK;
  if (q->heads <= 0 || q->heads % c->kv_heads != 0 || out->heads != q->heads) return AQLM_ERR_SHAPE;
  if (const int e = check_heads(q, tokens, c->head_dim, c->dtype, false)) return e;
  if (const int e = check_heads(out, tokens, c->head_dim, c->dtype, true)) return e;
  const int64_t strides = q->token_stride | q->head_stride | out->token_stride | out->head_stride | c->k_page_stride |
                          c->k_slot_stride | c->k_head_stride | c->v_page_stride | c->v_slot_stride | c->v_head_stride;
  if ((strides & 7) != 0 || !multiple(q->data, 16) || !multiple(out->data, 16) || !multiple(c->k, 16) ||
      !multiple(c->v, 16) || !multiple(workspace, 16) || !multiple(lse, 4))
    return AQLM_ERR_ALIGN;
  if (workspace_bytes < aqlm_paged_attention_workspace_bytes(c->head_dim)) return AQLM_ERR_WORKSPACE;
  const int64_t group = q->heads / c->kv_heads;
  // (rows, and the key tiles of all units of one kv head, are counted in 32 bits)
  const int64_t units = (tokens * group + 15) / 16 + c->seqs;
  const int64_t tiles = ((int64_t)c->table_width * c->page_size + 63) / 64 + 1;
  if (tokens * group >= k2G / 2 || units > (k2G - 1) / tiles) return AQLM_ERR_SHAPE;

  aqlm::AttnArgs a{};
  a.q = static_cast<const uint16_t*>(q->data);
  a.k = static_cast<const uint16_t*>(c->k);
  a.v = static_cast<const uint16_t*>(c->v);
  a.out = static_cast<uint16_t*>(out->data);
  a.lse = lse;
  a.block_table = c->block_table;
  a.kv_lens = c->kv_lens;
  a.cu_new = c->cu_new;
  a.counters = static_cast<uint32_t*>(workspace);
  a.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + AQLM_ATTENTION_COUNTER_BYTES);
  a.q_token = q->token_stride;
  a.q_head = q->head_stride;
  a.out_token = out->token_stride;
  a.out_head = out->head_stride;
  a.k_page = c->k_page_stride;
  a.k_slot = c->k_slot_stride;
  a.k_head = c->k_head_stride;
  a.v_page = c->v_page_stride;
  a.v_slot = c->v_slot_stride;
  a.v_head = c->v_head_stride;
  a.table_stride = c->table_stride;
  a.tokens = (int32_t)tokens;
  a.seqs = c->seqs;
  a.kv_heads = c->kv_heads;
  a.group = (int32_t)group;
  if (group > 1) {  // s = ceil(log2(group)): 2^(31 + s) / group, rounded up, divides rows below 2^31 exactly
    const int s = 64 - __builtin_clzll((uint64_t)group - 1);
    a.group_mul = (uint32_t)((uint64_t(1) << (31 + s)) / (uint64_t)group + 1);
    a.group_shift = (uint32_t)(s - 1);
  }
  a.head_dim = c->head_dim;
  a.pages = (int32_t)c->pages;
  a.page_shift = page_shift(c->page_size);
  a.table_width = c->table_width;
  a.causal = causal != 0;
  a.window = window;
  a.whole_rows = c->page_size >= 16 && std::max(c->k_slot_stride, c->v_slot_stride) < (1 << 25);
  const float scale_log2 = std::fabs(scale) * 1.44269504088896341f;
  a.scale_log2 = scale_log2 > 0.f ? scale_log2 : 1.f;
  a.q_keep = scale_log2 > 0.f ? 0xFFFFFFFFu : 0u;
  a.q_flip = scale < 0.f && scale_log2 > 0.f ? 0x80008000u : 0u;

  // A unit of the one kernel is 16 rows and reads all the sequence's keys, of the other 128.
  // Up to 16 rows of a sequence the first is never behind by more than 3 % and up to twice as
  // fast; past 16 it reads keys twice, which costs what the keys' bytes cost.  bf16, 128
  // elements a head, us (of few rows / of many): 8 sequences of 1000 keys, 32 heads over 8: 14 / 26
  // at 4 rows, 17 / 26 at 16, 18 / 26 at 32, 23 / 29 at 64, 42 / 37 at 128; 64 of 4000, 64 over 8: 192 /
  // 187 at 16, 380 / 188 at 24, 748 / 192 at 64; one of 30000, 64 over 8: 62 / 78 at 24, 83 / 89 at 64,
  // 139 / 122 at 128.
  const bool bf = c->dtype == AQLM_BF16;
  const int64_t most = max_new > 0 ? std::min(max_new, tokens) : tokens;
  if (most * group <= 16)
    return status_of(aqlm::launch_attention_step(a, bf, aqlm::attention_step_grid(), (hipStream_t)stream));
  return status_of(aqlm::launch_attention_chunk(a, bf, aqlm::attention_chunk_grid(c->head_dim), (hipStream_t)stream));
}

int aqlm_process_logits(const void* logits, int64_t logits_stride, void* out, int64_t out_stride, int32_t dtype,
                        int64_t rows, int64_t vocab, const aqlm_logit_rules* r, void* stream) {
  if (!r) return AQLM_ERR_NULL;
  if (!known_dtype(dtype)) return AQLM_ERR_UNSUPPORTED;
  if (rows < 0 || rows > 65535 || vocab <= 0 || vocab >= k2G - 65536 || logits_stride < 0 || out_stride < 0)
    return AQLM_ERR_SHAPE;
  if (rows == 0) return AQLM_OK;
  if (!logits || !out) return AQLM_ERR_NULL;
  if (rows > 1 && out_stride < vocab) return AQLM_ERR_SHAPE;
  if (r->tokens && !r->token_lens) return AQLM_ERR_NULL;
  if (!r->tokens && (r->repetition || r->frequency || r->presence)) return AQLM_ERR_NULL;
  if (r->tokens && (r->history < 0 || r->history > aqlm::kMaxHistory || r->token_stride < 0)) return AQLM_ERR_SHAPE;
  if ((r->bias_ids == nullptr) != (r->bias_values == nullptr)) return AQLM_ERR_NULL;
  if (r->bias_ids && (r->biases < 0 || r->biases > aqlm::kMaxBiases || r->bias_stride < 0)) return AQLM_ERR_SHAPE;
  if (r->mask && r->mask_stride < 0) return AQLM_ERR_SHAPE;
  const uintptr_t unit = (uintptr_t)aqlm::dtype_bytes(dtype);
  if (!multiple(logits, unit) || !multiple(out, unit)) return AQLM_ERR_ALIGN;
  for (const void* p : {(const void*)r->tokens, (const void*)r->token_lens, (const void*)r->prompt_lens,
                        (const void*)r->repetition, (const void*)r->frequency, (const void*)r->presence,
                        (const void*)r->bias_ids, (const void*)r->bias_values, (const void*)r->mask})
    if (!multiple(p, 4)) return AQLM_ERR_ALIGN;
  aqlm::LogitsArgs a{};
  a.in = logits;
  a.out = out;
  a.in_row = logits_stride;
  a.out_row = out_stride;
  a.rows = (int32_t)rows;
  a.vocab = (int32_t)vocab;
  if (r->tokens && r->history > 0) {  // (without history there is nothing to penalise)
    a.tokens = r->tokens;
    a.token_lens = r->token_lens;
    a.prompt_lens = r->prompt_lens;
    a.token_row = r->token_stride;
    a.history = r->history;
    a.repetition = r->repetition;
    a.frequency = r->frequency;
    a.presence = r->presence;
  }
  if (r->bias_ids && r->biases > 0) {
    a.bias_ids = r->bias_ids;
    a.bias_values = r->bias_values;
    a.bias_row = r->bias_stride;
    a.biases = r->biases;
  }
  a.mask = r->mask;
  a.mask_row = r->mask_stride;
  return status_of(aqlm::launch_logits(a, dtype, (hipStream_t)stream));
}

}  // extern "C"
