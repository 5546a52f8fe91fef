// What a sequence of a paged attention call holds, from device integers that may say
// anything: plain arithmetic, for the kernels and for host code.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>
#define AQLM_BOTH __host__ __device__ __forceinline__
#else
#define AQLM_BOTH inline
#endif

namespace aqlm {

// A sequence's new tokens and its keys.
struct AttnSeq {
  int first, count, keys;
};

// Its tokens [cu0, cu1) cut to those of the call, its keys to the `room` of its
// pages: no read goes past the arrays.
AQLM_BOTH AttnSeq attn_cut(int cu0, int cu1, int kv_len, int tokens, int64_t room) {
  AttnSeq s;
  s.first = cu0 < 0 ? 0 : (cu0 > tokens ? tokens : cu0);
  const int end = cu1 < s.first ? s.first : (cu1 > tokens ? tokens : cu1);
  s.count = end - s.first;
  s.keys = kv_len < 0 ? 0 : ((int64_t)kv_len > room ? (int)room : kv_len);
  return s;
}

// What is left of it behind the sequences before, which end at token `before`.
// Where the offsets ascend nothing changes; where they fall, a token is the first
// sequence's that claims it, so all sequences together hold no token twice (their
// costs are added up in 32 bits).  A sequence's last tokens are left: their
// positions, counted from its last key, stay.
AQLM_BOTH AttnSeq attn_after(AttnSeq s, int before) {
  if (before > s.first) {
    const int end = s.first + s.count;
    s.first = before;
    s.count = end > before ? end - before : 0;
  }
  return s;
}

}  // namespace aqlm
