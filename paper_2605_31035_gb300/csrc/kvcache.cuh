// The paged key-value cache's argument checks, shared by the entry points that
// take one (include/mixfp4.h) and the Python binding.
#pragma once
#include <cstdint>

#include "mixfp4.h"

namespace mixfp4 {

int check_kv_cache(const mixfp4_kv_cache* c);

// Whether a thread of mixfp4_kv_append has both elements of every pair that it rotates: not where the halves of a
// rotation lie in 16-element blocks that it does not take two of.
inline bool owns_pairs(int64_t rot_dim, bool interleaved) { return interleaved || rot_dim % 32 == 0; }

// Whether the `bytes` from `out` on overlap a row (heads of head_dim elements) of a [tokens] input.
inline bool overlaps(const void* out, int64_t bytes, const void* in, int64_t tokens, int64_t token_stride, int64_t heads,
                     int64_t head_stride, int64_t head_dim, int64_t esize) {
  if (bytes <= 0 || tokens <= 0 || heads <= 0) return false;
  const int64_t from = (int64_t) reinterpret_cast<uintptr_t>(out), base = (int64_t) reinterpret_cast<uintptr_t>(in);
  const int64_t step = token_stride * esize, span = ((heads - 1) * head_stride + head_dim) * esize;
  const int64_t ahead = from - base - span;  // the first row that ends behind `from`
  const int64_t t = ahead < 0 ? 0 : (step > 0 ? ahead / step + 1 : tokens);
  return t < tokens && base + t * step < from + bytes;
}

// Whether mixfp4_kv_append's q_out lies where the call reads: on k or v, or on q, except as q itself (bf16, dense) where
// every thread reads what it writes before it does.
inline bool append_overlaps(const void* q, int64_t q_token_stride, int64_t q_head_stride, int64_t q_heads, const void* k,
                            int64_t k_token_stride, int64_t k_head_stride, const void* v, int64_t v_token_stride,
                            int64_t v_head_stride, int dtype, int64_t T, int64_t rot_dim, bool interleaved,
                            int64_t heads, int64_t head_dim, const void* q_out) {
  const int64_t bytes = T * q_heads * head_dim * 2, esize = dtype == MIXFP4_DTYPE_F32 ? 4 : 2;
  const bool in_place = q == q_out && dtype == MIXFP4_DTYPE_BF16 && owns_pairs(rot_dim, interleaved) &&
                        (T == 1 || q_token_stride == q_heads * head_dim) && (q_heads == 1 || q_head_stride == head_dim);
  return (!in_place && overlaps(q_out, bytes, q, T, q_token_stride, q_heads, q_head_stride, head_dim, esize)) ||
         overlaps(q_out, bytes, k, T, k_token_stride, heads, k_head_stride, head_dim, esize) ||
         overlaps(q_out, bytes, v, T, v_token_stride, heads, v_head_stride, head_dim, esize);
}

}  // namespace mixfp4
