// The paged key-value cache: new tokens appended with the position rotation
// on the way (mixfp4_kv_append), and rows read back (mixfp4_kv_gather).
//
// Both are single passes bound by memory: every input element is read once and
// every output written once, 32 bytes per lane and access.  A thread owns a
// "unit" of a head row (one 16-element block, or the two blocks that a
// rotation of pairs (i, i + rot / 2) couples) and walks over several heads of
// its token, so that the token's angles, slot and address are found once.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "decode.cuh"
#include "kvcache.cuh"
#include "quant_core.cuh"

namespace mixfp4 {
namespace {

constexpr int kThreads = 128;

struct AppendArgs {
  const void* src[3];  // q, k, v
  int64_t token_stride[3], head_stride[3];
  int q_heads;
  int64_t tokens;
  const int64_t* positions;
  const float* cos_sin;
  int64_t max_positions;
  int rot, interleaved, paired;
  int units, groups;  // units of a head row; threads of a token per unit
  mixfp4_kv_cache c;
  const int64_t* slots;
  uint16_t* q_out;
};

// 16 consecutive elements as fp32.
template <bool kF32>
__device__ __forceinline__ void load16(const void* base, int64_t at, float x[16]) {
  uint32_t w[8];
  if (kF32) {
    const float* p = static_cast<const float*>(base) + at;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      ldg256_stream(p + 8 * h, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[8 * h + j] = __uint_as_float(w[j]);
    }
  } else {
    ldg256_stream(static_cast<const uint16_t*>(base) + at, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[2 * j] = __uint_as_float(w[j] << 16);
      x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
  }
}

template <bool kF32>
__device__ __forceinline__ float load1(const void* base, int64_t at) {
  return kF32 ? static_cast<const float*>(base)[at]
              : __uint_as_float((uint32_t) static_cast<const uint16_t*>(base)[at] << 16);
}

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

__device__ __forceinline__ void store16_bf16(uint16_t* p, const float y[16]) {
  uint32_t w[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = bf16x2(y[2 * j], y[2 * j + 1]);
  stg256(p, w);
}

// Algorithm 1 on one block of fp32 values, stored as 8 code bytes and a scale byte.
template <int kMode>
__device__ __forceinline__ void store16_mixfp4(uint8_t* codes, uint8_t* scale, const float y[16],
                                               const TensorConsts& tc, const float4* tab) {
  u64 y2[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) y2[j] = pack2(y[2 * j], y[2 * j + 1]);
  uint32_t lo, hi, sb;
  if (tc.scaled)
    rht_block<kMode, true>(y2, tc, tab, lo, hi, sb);
  else
    rht_block<kMode, false>(y2, tc, tab, lo, hi, sb);
  stg64(codes, lo, hi);
  *scale = (uint8_t)sb;
}

// kMode: a MixFP4 cache's MIXFP4_MODE_*, or -1 for a bf16 cache.
template <bool kF32, int kMode>
__global__ void __launch_bounds__(kThreads) kv_append_kernel(const AppendArgs p) {
  __shared__ float4 tab[kMode >= 0 ? 128 : 1];
  TensorConsts tk, tv;
  if (kMode >= 0) {
    fill_scale_table(tab);
    tk = tensor_consts(const_cast<float*>(p.c.k_ts), nullptr, 1);
    tv = tensor_consts(const_cast<float*>(p.c.v_ts), nullptr, 1);
    __syncthreads();
  }
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t row = id / p.units;
  const int u = (int)(id - row * p.units);
  const int64_t t = row / p.groups;
  const int g = (int)(row - t * p.groups);
  if (t >= p.tokens) return;

  const int D = p.c.head_dim, rot = p.rot, half = rot / 2;
  // The unit's blocks: with `paired`, u and u + half / 16 while they rotate, then one block each.
  const int nrot = p.paired ? rot / 32 : 0;
  const bool pair = u < nrot;
  const int b0 = pair ? u : rot / 16 * (p.paired ? 1 : 0) + u - nrot;
  const bool turns = b0 * 16 < rot;

  const int64_t slot = p.slots[t];
  bool keep = slot >= 0 && slot < p.c.pages * p.c.page_size;
  bool placed = true;  // its position has a row of angles
  float c[16], s[16];
  if (rot > 0) {
    const int64_t pos = p.positions[t];
    placed = pos >= 0 && pos < p.max_positions;
    keep = keep && placed;
    if (turns && placed) {
      const float* cs = p.cos_sin + pos * rot;
      if (pair) {
        load16<true>(cs, b0 * 16, c);
        load16<true>(cs, half + b0 * 16, s);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int d = b0 * 16 + e;
          const int i = p.interleaved ? d / 2 : (d < half ? d : d - half);
          const bool first = p.interleaved ? (e & 1) == 0 : d < half;
          c[e] = d < rot ? cs[i] : 0.0f;
          s[e] = d < rot ? (first ? -cs[half + i] : cs[half + i]) : 0.0f;
        }
      }
    }
  }
  int64_t page = 0, off = 0;
  if (keep) {
    page = slot / p.c.page_size;
    off = slot - page * p.c.page_size;
  }
  const int64_t at = page * p.c.page_stride + off * p.c.token_stride;
  const int64_t sat = page * p.c.scale_page_stride + off * p.c.scale_token_stride;

  const int heads = p.q_heads + 2 * p.c.heads;
  for (int hh = g; hh < heads; hh += p.groups) {
    const int role = hh < p.q_heads ? 0 : (hh < p.q_heads + p.c.heads ? 1 : 2);
    const int h = role == 0 ? hh : (role == 1 ? hh - p.q_heads : hh - p.q_heads - p.c.heads);
    if (role != 0 && !keep) continue;
    const void* src = role == 0 ? p.src[0] : (role == 1 ? p.src[1] : p.src[2]);
    const int64_t from = role == 0   ? t * p.token_stride[0] + h * p.head_stride[0]
                         : role == 1 ? t * p.token_stride[1] + h * p.head_stride[1]
                                     : t * p.token_stride[2] + h * p.head_stride[2];
    float x[2][16];
    load16<kF32>(src, from + b0 * 16, x[0]);
    if (pair) load16<kF32>(src, from + half + b0 * 16, x[1]);
    if (role != 2 && turns) {
      if (pair) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float a = x[0][e], b = x[1][e];
          x[0][e] = __fsub_rn(__fmul_rn(a, c[e]), __fmul_rn(b, s[e]));
          x[1][e] = __fadd_rn(__fmul_rn(b, c[e]), __fmul_rn(a, s[e]));
        }
      } else if (p.interleaved) {
#pragma unroll
        for (int e = 0; e < 16; e += 2) {  // rot is even: a pair turns or stays as a whole
          const float a = x[0][e], b = x[0][e + 1];
          if (b0 * 16 + e < rot) {
            x[0][e] = __fadd_rn(__fmul_rn(a, c[e]), __fmul_rn(b, s[e]));
            x[0][e + 1] = __fadd_rn(__fmul_rn(b, c[e + 1]), __fmul_rn(a, s[e + 1]));
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int d = b0 * 16 + e;
          if (d < rot) {
            const float b = load1<kF32>(src, from + (d < half ? d + half : d - half));
            x[0][e] = __fadd_rn(__fmul_rn(x[0][e], c[e]), __fmul_rn(b, s[e]));
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (i == 1 && !pair) break;
      const int b = i == 0 ? b0 : b0 + nrot;
      if (role == 0) {
        if (!placed) {
#pragma unroll
          for (int e = 0; e < 16; ++e) x[i][e] = __uint_as_float(0x7FC00000u);
        }
        store16_bf16(p.q_out + (t * p.q_heads + h) * D + b * 16, x[i]);
      } else if (kMode < 0) {
        uint16_t* dst = static_cast<uint16_t*>(role == 1 ? p.c.k : p.c.v);
        store16_bf16(dst + at + h * p.c.head_stride + b * 16, x[i]);
      } else {
        uint8_t* codes = static_cast<uint8_t*>(role == 1 ? p.c.k : p.c.v) + at + h * p.c.head_stride + b * 8;
        uint8_t* scale = (role == 1 ? p.c.k_scales : p.c.v_scales) + sat + h * p.c.scale_head_stride + b;
        store16_mixfp4<kMode < 0 ? 0 : kMode>(codes, scale, x[i], role == 1 ? tk : tv, tab);
      }
    }
  }
}

// One 16-element block per thread: slot's row t, tensor (k or v), head, block.
template <bool kFp4, bool kF32>
__global__ void __launch_bounds__(kThreads) kv_gather_kernel(const mixfp4_kv_cache c, const int64_t* slots, int64_t T,
                                                             void* k_out, void* v_out) {
  const int blocks = c.head_dim / 16;
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t per_token = (int64_t)c.heads * blocks;
  const int64_t row = id / per_token;
  if (row >= 2 * T) return;
  const bool is_v = row >= T;
  const int64_t t = is_v ? row - T : row;
  const int r = (int)(id - row * per_token);
  const int h = r / blocks, b = r - h * blocks;
  const int64_t slot = slots[t];
  float y[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) y[e] = 0.0f;
  if (slot >= 0 && slot < c.pages * c.page_size) {
    const int64_t page = slot / c.page_size, off = slot - page * c.page_size;
    const int64_t at = page * c.page_stride + off * c.token_stride + h * c.head_stride;
    const void* src = is_v ? c.v : c.k;
    if (kFp4) {
      const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(src) + at + b * 8);
      const uint32_t sb = (is_v ? c.v_scales : c.k_scales)[page * c.scale_page_stride + off * c.scale_token_stride +
                                                           h * c.scale_head_stride + b];
      const float ts = *(is_v ? c.v_ts : c.k_ts);
      const bool e1m2 = sb >> 7;
      const uint32_t s2 = prmt(cvt_f16x2_from_e4m3x2((uint16_t)(sb & 0x7Fu)), 0u, 0x1010u);
      uint32_t o[8];
      decode8(w.x, e1m2 ? kLutE1M2Lo : kLutE2M1Lo, e1m2 ? kLutE1M2Hi : kLutE2M1Hi, s2, o);
      decode8(w.y, e1m2 ? kLutE1M2Lo : kLutE2M1Lo, e1m2 ? kLutE1M2Hi : kLutE2M1Hi, s2, o + 4);
#pragma unroll
      for (int j = 0; j < 8; ++j) {  // f16 holds twice the value times s8, exactly; one rounding at ts
        float lo, hi;
        f16x2_to_f32(o[j], lo, hi);
        y[2 * j] = __fmul_rn(0.5f * lo, ts);
        y[2 * j + 1] = __fmul_rn(0.5f * hi, ts);
      }
    } else {
      load16<false>(src, at + b * 16, y);
    }
  }
  const int64_t to = (t * c.heads + h) * c.head_dim + b * 16;
  if (kF32) {
    float* dst = static_cast<float*>(is_v ? v_out : k_out) + to;
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(y[8 * i + j]);
      stg256(dst + 8 * i, w);
    }
  } else {
    store16_bf16(static_cast<uint16_t*>(is_v ? v_out : k_out) + to, y);
  }
}

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline int launch_status() { return cudaGetLastError() == cudaSuccess ? MIXFP4_OK : MIXFP4_ERR_CUDA; }

template <bool kF32>
void launch_append(const AppendArgs& p, int mode, int64_t blocks, cudaStream_t s) {
  const unsigned grid = (unsigned)blocks;
  if (p.c.dtype == MIXFP4_CACHE_BF16) return kv_append_kernel<kF32, -1><<<grid, kThreads, 0, s>>>(p);
  switch (mode) {
    case MIXFP4_MODE_MIX: return kv_append_kernel<kF32, MIXFP4_MODE_MIX><<<grid, kThreads, 0, s>>>(p);
    case MIXFP4_MODE_E2M1_ONLY: return kv_append_kernel<kF32, MIXFP4_MODE_E2M1_ONLY><<<grid, kThreads, 0, s>>>(p);
    case MIXFP4_MODE_E1M2_ONLY: return kv_append_kernel<kF32, MIXFP4_MODE_E1M2_ONLY><<<grid, kThreads, 0, s>>>(p);
    default: return kv_append_kernel<kF32, MIXFP4_MODE_FOUR_SIX><<<grid, kThreads, 0, s>>>(p);
  }
}

}  // namespace

int check_kv_cache(const mixfp4_kv_cache* c) {
  if (!c) return MIXFP4_ERR_NULL;
  if (c->dtype != MIXFP4_CACHE_BF16 && c->dtype != MIXFP4_CACHE_MIXFP4) return MIXFP4_ERR_DTYPE;
  if (c->page_size < 1 || c->heads < 1 || c->head_dim < 16 || c->head_dim > 256 || c->head_dim % 16 != 0 ||
      c->pages < 0 || c->pages > INT32_MAX || c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0)
    return MIXFP4_ERR_SHAPE;
  const bool fp4 = c->dtype == MIXFP4_CACHE_MIXFP4;
  if (fp4 && (c->scale_page_stride < 0 || c->scale_token_stride < 0 || c->scale_head_stride < 0))
    return MIXFP4_ERR_SHAPE;
  if (fp4 && (!c->k_ts || !c->v_ts)) return MIXFP4_ERR_NULL;
  if (c->pages > 0 && (!c->k || !c->v || (fp4 && (!c->k_scales || !c->v_scales)))) return MIXFP4_ERR_NULL;
  const int64_t step = fp4 ? 8 : 16;
  const uintptr_t base = fp4 ? 8 : 32;
  if (!aligned(c->k, base) || !aligned(c->v, base) || c->page_stride % step || c->token_stride % step ||
      c->head_stride % step)
    return MIXFP4_ERR_ALIGN;
  if (fp4) {
    const int64_t sb = c->head_dim % 64 == 0 ? c->head_dim / 16 : 1;
    const uintptr_t a = (uintptr_t)(sb == 12 ? 4 : sb);  // head_dim 192: twelve bytes, read in fours
    if (!aligned(c->k_scales, a) || !aligned(c->v_scales, a) || c->scale_page_stride % (int64_t)a ||
        c->scale_token_stride % (int64_t)a || c->scale_head_stride % (int64_t)a)
      return MIXFP4_ERR_ALIGN;
    if (!aligned(c->k_ts, 4) || !aligned(c->v_ts, 4)) return MIXFP4_ERR_ALIGN;
  }
  return MIXFP4_OK;
}

}  // namespace mixfp4

extern "C" {

int mixfp4_kv_append(const void* q, int64_t q_token_stride, int64_t q_head_stride, int64_t q_heads, const void* k,
                     int64_t k_token_stride, int64_t k_head_stride, const void* v, int64_t v_token_stride,
                     int64_t v_head_stride, int dtype, int64_t T, const int64_t* positions, const float* cos_sin,
                     int64_t max_positions, int64_t rot_dim, int interleaved, const mixfp4_kv_cache* cache,
                     const int64_t* slots, void* q_out, int mode, void* stream) {
  using namespace mixfp4;
  if (dtype != MIXFP4_DTYPE_BF16 && dtype != MIXFP4_DTYPE_F32) return MIXFP4_ERR_DTYPE;
  if (mode < MIXFP4_MODE_MIX || mode > MIXFP4_MODE_FOUR_SIX) return MIXFP4_ERR_ARG;
  if (int st = check_kv_cache(cache)) return st;
  if (T < 0 || q_heads < 0 || q_heads > (1 << 20) || rot_dim < 0 || rot_dim > cache->head_dim || rot_dim % 2 != 0 ||
      max_positions < 0 || q_token_stride < 0 || q_head_stride < 0 || k_token_stride < 0 || k_head_stride < 0 ||
      v_token_stride < 0 || v_head_stride < 0)
    return MIXFP4_ERR_SHAPE;
  if (T == 0) return MIXFP4_OK;
  if (!k || !v || !slots || (q_heads > 0 && (!q || !q_out)) || (rot_dim > 0 && (!positions || !cos_sin)))
    return MIXFP4_ERR_NULL;
  if (!aligned(k, 32) || !aligned(v, 32) || !aligned(slots, 8) || k_token_stride % 16 || k_head_stride % 16 ||
      v_token_stride % 16 || v_head_stride % 16)
    return MIXFP4_ERR_ALIGN;
  if (q_heads > 0 && (!aligned(q, 32) || !aligned(q_out, 32) || q_token_stride % 16 || q_head_stride % 16))
    return MIXFP4_ERR_ALIGN;
  if (rot_dim > 0 && (!aligned(positions, 8) || !aligned(cos_sin, 32))) return MIXFP4_ERR_ALIGN;

  AppendArgs p = {};
  p.src[0] = q, p.src[1] = k, p.src[2] = v;
  p.token_stride[0] = q_token_stride, p.token_stride[1] = k_token_stride, p.token_stride[2] = v_token_stride;
  p.head_stride[0] = q_head_stride, p.head_stride[1] = k_head_stride, p.head_stride[2] = v_head_stride;
  p.q_heads = (int)q_heads;
  p.tokens = T;
  p.positions = positions, p.cos_sin = cos_sin, p.max_positions = max_positions;
  p.rot = (int)rot_dim, p.interleaved = interleaved != 0;
  p.paired = !p.interleaved && rot_dim > 0 && rot_dim % 32 == 0;
  p.c = *cache;
  p.slots = slots;
  p.q_out = static_cast<uint16_t*>(q_out);
  p.units = p.paired ? p.rot / 32 + (cache->head_dim - p.rot) / 16 : cache->head_dim / 16;
  const int64_t heads = q_heads + 2 * (int64_t)cache->heads;
  p.groups = (int)heads;
  const int64_t blocks = (T * p.groups * p.units + kThreads - 1) / kThreads;
  if (blocks > INT32_MAX) return MIXFP4_ERR_SHAPE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dtype == MIXFP4_DTYPE_F32)
    launch_append<true>(p, mode, blocks, s);
  else
    launch_append<false>(p, mode, blocks, s);
  return launch_status();
}

int mixfp4_kv_gather(const mixfp4_kv_cache* cache, const int64_t* slots, int64_t T, void* k_out, void* v_out,
                     int out_dtype, void* stream) {
  using namespace mixfp4;
  if (out_dtype != MIXFP4_DTYPE_BF16 && out_dtype != MIXFP4_DTYPE_F32) return MIXFP4_ERR_DTYPE;
  if (int st = check_kv_cache(cache)) return st;
  if (T < 0) return MIXFP4_ERR_SHAPE;
  if (T == 0) return MIXFP4_OK;
  if (!slots || !k_out || !v_out) return MIXFP4_ERR_NULL;
  if (!aligned(slots, 8) || !aligned(k_out, 32) || !aligned(v_out, 32)) return MIXFP4_ERR_ALIGN;
  const int64_t blocks = (2 * T * cache->heads * (cache->head_dim / 16) + kThreads - 1) / kThreads;
  if (blocks > INT32_MAX) return MIXFP4_ERR_SHAPE;
  const unsigned grid = (unsigned)blocks;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool fp4 = cache->dtype == MIXFP4_CACHE_MIXFP4, f32 = out_dtype == MIXFP4_DTYPE_F32;
  if (fp4 && f32)
    kv_gather_kernel<true, true><<<grid, kThreads, 0, s>>>(*cache, slots, T, k_out, v_out);
  else if (fp4)
    kv_gather_kernel<true, false><<<grid, kThreads, 0, s>>>(*cache, slots, T, k_out, v_out);
  else if (f32)
    kv_gather_kernel<false, true><<<grid, kThreads, 0, s>>>(*cache, slots, T, k_out, v_out);
  else
    kv_gather_kernel<false, false><<<grid, kThreads, 0, s>>>(*cache, slots, T, k_out, v_out);
  return launch_status();
}

}  // extern "C"
