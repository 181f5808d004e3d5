// The paged key-value cache: new tokens appended with the position rotation
// on the way (mixfp4_kv_append), and rows read back (mixfp4_kv_gather).
//
// Both are single passes: every input element is read once (but see below) and
// every output written once, 32 bytes per lane and access.  Appending 8111 tokens of 32 + 16
// heads of 128 in fp32 to a bf16 cache (303 MB in all) takes 48 us, 93 % of the
// measured HBM rate.  To a MixFP4 cache it takes 52 us for 279 MB (79 %), the
// rest being the quantizer's steps.  The gather is a row's few bytes to 16 bf16
// values a thread: 12 us for those 8111 tokens (8.8 from a bf16 cache), with an
// instruction issued in 76 % of the cycles, most of them the index arithmetic
// that finds page and address anew for every 16 elements.
//
// A thread owns a "unit" of a head row (one 16-element block, or the two blocks
// that a rotation of pairs (i, i + rot / 2) couples) and walks over several
// heads of its token, so that the token's angles, slot and address are found
// once.  Where a half-split rotation's width is no multiple of 32 a thread has
// one block, and reads the 16 partners of its elements one by one: 8111 tokens of
// 16 + 32 heads of 80 in fp32 to a bf16 cache 71 us with all 80 rotated, 33 with
// 64 (to a MixFP4 cache 77 and 40).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "decode.cuh"
#include "host_util.cuh"
#include "kvcache.cuh"
#include "quant_core.cuh"

namespace mixfp4 {
namespace {

constexpr int kThreads = 128;
// CTAs of an SM by registers.  A MixFP4 cache's quantizer is a long chain of dependent steps and lives on other warps, so
// its angles lie in shared memory and rows are asked for when they are due: 5 / 6 / 7 CTAs 47 / 42 / 40 us at 4000
// interleaved tokens of 32 + 16 heads of 128 in fp32, 22 / 22 / 24 us at 5372 of 8 + 2 heads of 256, 33 / 29 / 31 us at
// 3170 of 40 + 16 heads of 128 in bf16 (with angles in registers and a row ahead, 3 CTAs: 54, 32 and 39 us).  A bf16
// cache keeps both in registers: rows a head ahead are what HBM needs.
template <int kMode>
constexpr int kCtas = kMode < 0 ? 4 : 6;
// What a thread's beginning (slot, angles) costs in head rows; 1 to 8 choose alike.
constexpr int kBegin = 2;

struct AppendArgs {
  const void* src[3];  // q, k, v
  int64_t token_stride[3], head_stride[3];
  int q_heads;
  int64_t tokens;
  const int64_t* positions;
  const float* cos_sin;
  int64_t max_positions;
  int rot, interleaved, paired;
  int units, groups, at_once;  // units of a head row; a CTA's threads of a token per unit; its tokens
  int stride;                  // a token's threads per unit, over all CTAs of its tokens (blockIdx.y)
  mixfp4_kv_cache c;
  const int64_t* slots;
  uint16_t* q_out;
};

// 16 consecutive elements as they lie: 16 words of fp32, 8 of bf16.
template <bool kF32>
__device__ __forceinline__ void load16(const void* base, int64_t at, uint32_t* w) {
  if (kF32) {
    const float* p = static_cast<const float*>(base) + at;
    ldg256_stream(p, w);
    ldg256_stream(p + 8, w + 8);
  } else {
    ldg256_stream(static_cast<const uint16_t*>(base) + at, w);
  }
}
template <bool kF32>
__device__ __forceinline__ void to_float(const uint32_t* w, float x[16]) {
#pragma unroll
  for (int j = 0; j < (kF32 ? 16 : 8); ++j) {
    if (kF32) {
      x[j] = __uint_as_float(w[j]);
    } else {
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
__global__ void __launch_bounds__(kThreads, kCtas<kMode>) kv_append_kernel(const AppendArgs p) {
  __shared__ float4 tab[kMode >= 0 ? 128 : 1];
  __shared__ float angles[kMode >= 0 ? 32 * kThreads : 1];  // [16 cosines, 16 sines][thread]
  const int row = (int)threadIdx.x / p.units, u = (int)threadIdx.x - row * p.units;
  const int tl = row / p.groups, g = (int)blockIdx.y * p.groups + row - tl * p.groups;
  const int64_t t = (int64_t)blockIdx.x * p.at_once + tl;
  const bool mine = tl < p.at_once && t < p.tokens;

  const int D = p.c.head_dim, rot = p.rot, half = rot / 2;
  // The unit's blocks: with `paired`, u and u + half / 16 while they rotate, then one block each.
  const int nrot = p.paired ? rot / 32 : 0;
  const bool pair = u < nrot;
  const int b0 = pair ? u : (p.paired ? rot / 16 : 0) + u - nrot;
  const bool turns = b0 * 16 < rot;
  const int heads = p.q_heads + 2 * p.c.heads;

  // One head row's blocks, for a bf16 cache asked for a head ahead of their use.
  constexpr int kWords = kF32 ? 16 : 8;
  uint32_t next[2][kWords];
  auto role_of = [&](int hh) { return hh < p.q_heads ? 0 : (hh < p.q_heads + p.c.heads ? 1 : 2); };
  auto place = [&](int hh, const void*& base, int64_t& from) {
    const int role = role_of(hh);
    base = role == 0 ? p.src[0] : (role == 1 ? p.src[1] : p.src[2]);
    from = role == 0   ? t * p.token_stride[0] + hh * p.head_stride[0]
           : role == 1 ? t * p.token_stride[1] + (hh - p.q_heads) * p.head_stride[1]
                       : t * p.token_stride[2] + (hh - p.q_heads - p.c.heads) * p.head_stride[2];
  };
  auto fetch = [&](int hh) {
    const void* base;
    int64_t from;
    place(hh, base, from);
    load16<kF32>(base, from + b0 * 16, next[0]);
    if (pair) load16<kF32>(base, from + half + b0 * 16, next[1]);
  };

  int64_t slot = -1, pos = 0;
  if (mine) {
    slot = p.slots[t];
    if (rot > 0) pos = p.positions[t];
    if (kMode < 0 && g < heads) fetch(g);
  }
  TensorConsts tk, tv;
  if (kMode >= 0) {
    fill_scale_table(tab);
    tk = tensor_consts(const_cast<float*>(p.c.k_ts), nullptr, 1);
    tv = tensor_consts(const_cast<float*>(p.c.v_ts), nullptr, 1);
    __syncthreads();
  }
  if (!mine) return;

  bool keep = slot >= 0 && slot < p.c.pages * p.c.page_size;
  const bool placed = pos >= 0 && (rot == 0 || pos < p.max_positions);  // the position has a row of angles
  keep = keep && placed;
  float c[16], s[16];
  if (rot > 0 && turns && placed) {
    const float* cs = p.cos_sin + pos * rot;
    if (pair) {
      load16<true>(cs, b0 * 16, reinterpret_cast<uint32_t*>(c));
      load16<true>(cs, half + b0 * 16, reinterpret_cast<uint32_t*>(s));
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
  if (kMode >= 0) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      angles[e * kThreads + threadIdx.x] = c[e], angles[(16 + e) * kThreads + threadIdx.x] = s[e];
  }
  auto cosine = [&](int e) { return kMode >= 0 ? angles[e * kThreads + threadIdx.x] : c[e]; };
  auto sine = [&](int e) { return kMode >= 0 ? angles[(16 + e) * kThreads + threadIdx.x] : s[e]; };
  int64_t at = 0, sat = 0;
  if (keep) {
    const int64_t page = slot / p.c.page_size, off = slot - page * p.c.page_size;
    at = page * p.c.page_stride + off * p.c.token_stride;
    sat = page * p.c.scale_page_stride + off * p.c.scale_token_stride;
  }

#pragma unroll 1
  for (int hh = g; hh < heads; hh += p.stride) {
    if (kMode >= 0) fetch(hh);
    float x[2][16];
    to_float<kF32>(next[0], x[0]);
    if (pair) to_float<kF32>(next[1], x[1]);
    if (kMode < 0 && hh + p.stride < heads) fetch(hh + p.stride);
    const int role = role_of(hh);
    if (role != 0 && !keep) continue;
    const int h = role == 0 ? hh : (role == 1 ? hh - p.q_heads : hh - p.q_heads - p.c.heads);
    if (role != 2 && turns && placed) {
      if (pair) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float a = x[0][e], b = x[1][e];
          x[0][e] = __fsub_rn(__fmul_rn(a, cosine(e)), __fmul_rn(b, sine(e)));
          x[1][e] = __fadd_rn(__fmul_rn(b, cosine(e)), __fmul_rn(a, sine(e)));
        }
      } else if (p.interleaved) {
#pragma unroll
        for (int e = 0; e < 16; e += 2) {  // rot is even: a pair turns or stays as a whole
          const float a = x[0][e], b = x[0][e + 1];
          if (b0 * 16 + e < rot) {
            x[0][e] = __fadd_rn(__fmul_rn(a, cosine(e)), __fmul_rn(b, sine(e)));
            x[0][e + 1] = __fadd_rn(__fmul_rn(b, cosine(e + 1)), __fmul_rn(a, sine(e + 1)));
          }
        }
      } else {
        const void* base;
        int64_t from;
        place(hh, base, from);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int d = b0 * 16 + e;
          if (d < rot) {
            const float b = load1<kF32>(base, from + (d < half ? d + half : d - half));
            x[0][e] = __fadd_rn(__fmul_rn(x[0][e], cosine(e)), __fmul_rn(b, sine(e)));
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

// One 16-element block per thread: slot t's row, tensor (k or v), head, block.
template <bool kFp4, bool kF32>
__global__ void __launch_bounds__(kThreads) kv_gather_kernel(const mixfp4_kv_cache c, const int64_t* slots, int64_t T,
                                                             void* k_out, void* v_out) {
  const int blocks = c.head_dim / 16;
  const int units = c.heads * blocks, per_cta = kThreads / units > 0 ? kThreads / units : 1;  // rows of a CTA
  const int tl = (int)threadIdx.x / units;
  const int64_t t = (int64_t)blockIdx.x * per_cta + tl;
  const bool is_v = blockIdx.y & 1;
  const int r = (int)(blockIdx.y >> 1) * kThreads + (int)threadIdx.x - tl * units;  // head and block
  if (tl >= per_cta || t >= T || r >= units) return;
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
      uint32_t w[8];
      load16<false>(src, at + b * 16, w);
      to_float<false>(w, y);
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
  const dim3 grid((unsigned)blocks, (unsigned)(p.stride / p.groups));
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
  if (c->page_size < 1 || c->heads < 1 || c->heads > (1 << 20) || c->head_dim < 16 || c->head_dim > 256 ||
      c->head_dim % 16 != 0 || c->pages < 0 || c->pages > INT32_MAX || c->page_stride < 0 ||
      c->token_stride < 0 || c->head_stride < 0)
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
  if (q_heads > 0 && append_overlaps(q, q_token_stride, q_head_stride, q_heads, k, k_token_stride, k_head_stride, v,
                                     v_token_stride, v_head_stride, dtype, T, rot_dim, interleaved != 0, cache->heads,
                                     cache->head_dim, q_out))
    return MIXFP4_ERR_ARG;

  AppendArgs p = {};
  p.src[0] = q, p.src[1] = k, p.src[2] = v;
  p.token_stride[0] = q_token_stride, p.token_stride[1] = k_token_stride, p.token_stride[2] = v_token_stride;
  p.head_stride[0] = q_head_stride, p.head_stride[1] = k_head_stride, p.head_stride[2] = v_head_stride;
  p.q_heads = (int)q_heads;
  p.tokens = T;
  p.positions = positions, p.cos_sin = cos_sin, p.max_positions = max_positions;
  p.rot = (int)rot_dim, p.interleaved = interleaved != 0;
  p.paired = !p.interleaved && rot_dim > 0 && owns_pairs(rot_dim, false);
  p.c = *cache;
  p.slots = slots;
  p.q_out = static_cast<uint16_t*>(q_out);
  p.units = p.paired ? p.rot / 32 + (cache->head_dim - p.rot) / 16 : cache->head_dim / 16;
  // Threads of a token: for few tokens one for each head and unit, spread over CTAs; else as many as make rounds of CTAs
  // times heads of a thread the least, so that the last round is full (3305 tokens of 40 + 16 heads of 128: 42 us with
  // 2.2 rounds, 31 so).
  const int heads = (int)q_heads + 2 * cache->heads, most = kThreads / p.units;
  const int64_t places = (int64_t)num_sms() * (cache->dtype == MIXFP4_CACHE_BF16 ? kCtas<-1> : kCtas<0>);
  int64_t least = INT64_MAX;
  for (int groups = T * p.units * heads <= places * kThreads ? heads : 1; groups <= heads; ++groups) {
    const int slices = (groups + most - 1) / most, each = (groups + slices - 1) / slices, at_once = most / each;
    const int64_t rounds = ((T + at_once - 1) / at_once * slices + places - 1) / places;
    const int64_t cost = rounds * ((heads + each * slices - 1) / (each * slices) + kBegin);
    if (cost < least) least = cost, p.groups = each, p.stride = each * slices, p.at_once = at_once;
  }
  const int64_t blocks = (T + p.at_once - 1) / p.at_once;
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
  // CTAs of whole rows, or, where a row has more blocks than a CTA threads, of a part of one; keys and values.
  const int64_t units = (int64_t)cache->heads * (cache->head_dim / 16), rows = kThreads / units > 0 ? kThreads / units : 1;
  const int64_t blocks = (T + rows - 1) / rows, slices = (units + kThreads - 1) / kThreads;
  if (blocks > INT32_MAX || slices > 32767) return MIXFP4_ERR_SHAPE;
  const dim3 grid((unsigned)blocks, (unsigned)(2 * slices));
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
