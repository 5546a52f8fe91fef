// Rotary positions and head norms: arguments of the kernels in rope.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace aqlm {

// The values of aqlm_dtype.
constexpr int kF16 = 0, kBf16 = 1, kF32 = 2;
constexpr int64_t dtype_bytes(int t) { return t == kF32 ? 4 : 2; }

// An activation [tokens][heads][head_dim]; strides in elements.
struct RopeSide {
  const void* in;
  const void* x;  // backward with a norm: what the forward read
  void* out;
  const void* weight;  // [head_dim] or null
  int64_t in_token, in_head, x_token, x_head, out_token, out_head;
  int32_t heads;
};

struct RopeArgs {
  RopeSide side[3];  // q, k, and v (copied) when paged
  const float* table;        // [rows][rot / 2][2]
  const int32_t* positions;  // [tokens]; not when paged
  int64_t rows;
  int32_t tokens, head_dim, rot;
  int32_t interleaved;
  float eps, sign;
  // paged: k and v go to the cache
  const int32_t *block_table, *kv_lens, *cu_new;
  int64_t table_stride, page_stride[2], slot_stride[2], cache_head[2];
  int32_t seqs, pages, page_shift, table_width;
  // backward with a norm
  float* parts;      // [blocks][head_dim]
  float* dweight[2];
  int32_t blocks[2];  // workgroups of q and of k
};

bool rope_vector(const RopeArgs& a, int dtype, bool paged, bool grad);
hipError_t launch_rope(const RopeArgs& a, int dtype, bool paged, hipStream_t s);
// Workgroups that the gradients of the weights are summed over (a multiple of two).
int rope_grad_blocks();
hipError_t launch_rope_grad_norm(RopeArgs a, int dtype, hipStream_t s);
hipError_t launch_rotary_table(const double* inv_freq, int64_t rows, int half, double scale, float* table, hipStream_t s);

}  // namespace aqlm
