// Attention of drafted tokens over the paged cache (mixfp4_tree_attention).
//
// The plain kernel: a CTA to a draft and query head, its warps in turn over the
// tokens, each lane two dimensions of every 64; the softmax's maximum and sum run
// along, and the warps' results are joined in shared memory.
#include <cuda_runtime.h>
#include <cstdint>

#include "host_util.cuh"
#include "kvcache.cuh"
#include "ptx.cuh"

namespace mixfp4 {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kMostDrafts = 64;
constexpr float kNoScore = -3e38f;  // m where nothing has been seen: no difference to a score or to itself is NaN
constexpr float kMostScore = 3.402823466e38f;

struct TreeArgs {
  const uint16_t* q;
  int64_t q_stride, q_token_stride, q_head_stride;
  int B, t, q_heads, group;
  mixfp4_kv_cache c;
  const int32_t* table;
  int64_t table_stride, max_tokens;
  const int32_t* lengths;
  const int64_t* mask;
  int64_t mask_stride;
  const int32_t* counts;
  float scale, softcap;
  int64_t window;
  const float* slopes;
  uint16_t* out;
  float* lse;
};

__device__ __forceinline__ float2 pair_of(const void* base, const uint8_t* scales, int64_t at, int64_t sat, int d,
                                          bool fp4, float ts) {
  if (!fp4) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(base) + at + d);
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  }
  const uint32_t byte = static_cast<const uint8_t*>(base)[at + d / 2], sc = scales[sat + d / 16];
  float lo, hi;
  f16x2_to_f32(cvt_f16x2_from_e4m3x2((uint16_t)(sc & 0x7Fu)), lo, hi);
  auto value = [&](uint32_t nib) {
    const uint32_t p = nib & 7u;
    const float m = sc >> 7 ? (float)p : (p < 4 ? 0.5f * p : (p == 4 ? 2.0f : (p == 5 ? 3.0f : (p == 6 ? 4.0f : 6.0f))));
    return (nib & 8u ? -m : m) * lo * ts;
  };
  return make_float2(value(byte & 15u), value(byte >> 4));
}

__global__ void __launch_bounds__(kThreads) tree_attention_kernel(const TreeArgs p) {
  __shared__ float so[kWarps][256];
  __shared__ float sm[kWarps], sl[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = p.c.head_dim;
  const int64_t row = blockIdx.x;  // [B][t][q_heads]
  const int h = (int)(row % p.q_heads), i = (int)(row / p.q_heads % p.t);
  const int64_t b = row / p.q_heads / p.t;
  const bool fp4 = p.c.dtype == MIXFP4_CACHE_MIXFP4;
  const float kts = fp4 ? *p.c.k_ts : 1.0f, vts = fp4 ? *p.c.v_ts : 1.0f;
  const int n = max(p.lengths[b], 0), c = min(min(p.counts ? max(p.counts[b], 0) : p.t, p.t), n), first = n - c;
  const int end = (int)min((int64_t)n, p.max_tokens);
  const uint64_t there = c == 64 ? ~0ull : (1ull << c) - 1;
  auto bits = [&](int k) {
    return (p.mask ? (uint64_t)p.mask[b * p.mask_stride + k] : (2ull << k) - 1) & there;
  };
  auto depth = [&](int k) { return __popcll(bits(k) & ~(1ull << k)); };
  const uint64_t mine = i < c ? bits(i) : 0;
  const int place = first + depth(i);
  float2 q[4], o[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int d = 2 * lane + 64 * j;
    q[j] = o[j] = make_float2(0.0f, 0.0f);
    if (d < D) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(p.q + b * p.q_stride + i * p.q_token_stride +
                                                            h * p.q_head_stride + d);
      q[j] = make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    }
  }
  float m = kNoScore, l = 0.0f;
  for (int j = warp; j < end && i < c; j += kWarps) {
    const int k = j - first;
    const int at = k < 0 ? j : first + depth(k);
    if (k >= 0 && !(mine >> k & 1)) continue;
    if (p.window > 0 && place - at >= p.window) continue;
    const int page = p.table[b * p.table_stride + j / p.c.page_size], off = j % p.c.page_size;
    if (page < 0 || page >= p.c.pages) continue;
    const int64_t kat = page * p.c.page_stride + off * p.c.token_stride + h / p.group * p.c.head_stride;
    const int64_t sat = page * p.c.scale_page_stride + off * p.c.scale_token_stride + h / p.group * p.c.scale_head_stride;
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int d = 2 * lane + 64 * e;
      if (d >= D) break;
      const float2 v = pair_of(p.c.k, p.c.k_scales, kat, sat, d, fp4, kts);
      s += q[e].x * v.x + q[e].y * v.y;
    }
#pragma unroll
    for (int e = 16; e > 0; e >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, e);
    s *= p.scale;
    if (p.softcap > 0.0f) s = p.softcap * tanhf(s / p.softcap);
    if (p.slopes) s -= p.slopes[h] * (float)(place - at);
    const float top = fminf(fmaxf(m, s), kMostScore), old = expf(m - top), w = expf(s - top);
    m = top;
    l = l * old + w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int d = 2 * lane + 64 * e;
      if (d >= D) break;
      const float2 v = pair_of(p.c.v, p.c.v_scales, kat, sat, d, fp4, vts);
      o[e].x = o[e].x * old + w * v.x, o[e].y = o[e].y * old + w * v.y;
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) so[warp][2 * lane + 64 * e] = o[e].x, so[warp][2 * lane + 64 * e + 1] = o[e].y;
  if (lane == 0) sm[warp] = m, sl[warp] = l;
  __syncthreads();
  float M = kNoScore, L = 0.0f;
  for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sm[w]);
  for (int w = 0; w < kWarps; ++w) L += sl[w] == 0.0f ? 0.0f : sl[w] * expf(sm[w] - M);
  const int d = threadIdx.x;
  float x = 0.0f;
  for (int w = 0; w < kWarps; ++w)
    if (sl[w] != 0.0f) x += so[w][d] * expf(sm[w] - M);
  if (L != 0.0f) x /= L;
  if (d < D) {
    uint16_t r;
    asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(r) : "f"(x));
    p.out[row * D + d] = r;
  }
  if (d == 0 && p.lse) p.lse[row] = L == 0.0f ? -INFINITY : M + logf(L);
}

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline int launch_status() { return cudaGetLastError() == cudaSuccess ? MIXFP4_OK : MIXFP4_ERR_CUDA; }

}  // namespace
}  // namespace mixfp4

extern "C" {

int mixfp4_tree_attention_workspace(const mixfp4_kv_cache* cache, int64_t B, int64_t t, int64_t q_heads,
                                    int64_t* bytes) {
  using namespace mixfp4;
  if (int st = check_kv_cache(cache)) return st;
  if (!bytes) return MIXFP4_ERR_NULL;
  if (B < 0 || t < 0 || t > kMostDrafts || q_heads < 0 || q_heads % cache->heads != 0) return MIXFP4_ERR_SHAPE;
  *bytes = 0;
  if (B == 0 || t == 0 || q_heads == 0) return MIXFP4_OK;
  *bytes = 256;
  return MIXFP4_OK;
}

int mixfp4_tree_attention(const void* q, int64_t q_stride, int64_t q_token_stride, int64_t q_head_stride, int64_t B,
                          int64_t t, int64_t q_heads, const mixfp4_kv_cache* cache, const int32_t* block_table,
                          int64_t table_stride, int64_t table_pages, const int32_t* lengths, const int64_t* mask,
                          int64_t mask_stride, const int32_t* counts, float scale, int64_t window, float softcap,
                          const float* slopes, void* out, float* lse, void* workspace, int64_t workspace_bytes,
                          void* stream) {
  using namespace mixfp4;
  int64_t need = 0;
  if (int st = mixfp4_tree_attention_workspace(cache, B, t, q_heads, &need)) return st;
  if (!(softcap == 0.0f || (softcap >= 1e-6f && softcap <= 1e6f))) return MIXFP4_ERR_ARG;
  if (B > INT32_MAX || q_heads > INT32_MAX || q_stride < 0 || q_token_stride < 0 || q_head_stride < 0 ||
      table_stride < 0 || table_pages < 0 || table_stride < table_pages ||
      table_pages > (INT32_MAX - 4096) / cache->page_size || window < 0 || mask_stride < 0 ||
      (mask_stride != 0 && mask_stride < t) || workspace_bytes < need)
    return MIXFP4_ERR_SHAPE;
  if (need == 0) return MIXFP4_OK;
  if (!q || !out || !lengths || !workspace || (table_pages > 0 && !block_table)) return MIXFP4_ERR_NULL;
  if (!aligned(q, 16) || q_stride % 8 || q_token_stride % 8 || q_head_stride % 8 || !aligned(block_table, 4) ||
      !aligned(lengths, 4) || !aligned(mask, 8) || !aligned(counts, 4) || !aligned(slopes, 4) || !aligned(out, 16) ||
      !aligned(lse, 4) || !aligned(workspace, 256))
    return MIXFP4_ERR_ALIGN;
  TreeArgs p = {};
  p.q = static_cast<const uint16_t*>(q);
  p.q_stride = q_stride, p.q_token_stride = q_token_stride, p.q_head_stride = q_head_stride;
  p.B = (int)B, p.t = (int)t, p.q_heads = (int)q_heads, p.group = (int)(q_heads / cache->heads);
  p.c = *cache;
  p.table = block_table, p.table_stride = table_stride, p.max_tokens = table_pages * cache->page_size;
  p.lengths = lengths, p.mask = mask, p.mask_stride = mask_stride, p.counts = counts;
  p.scale = scale, p.softcap = softcap, p.window = window, p.slopes = slopes;
  p.out = static_cast<uint16_t*>(out), p.lse = lse;
  const int64_t rows = B * t * q_heads;
  if (rows > INT32_MAX) return MIXFP4_ERR_SHAPE;
  tree_attention_kernel<<<(unsigned)rows, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(p);
  return launch_status();
}

}  // extern "C"
