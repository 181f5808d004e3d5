// Low-rank adapters of many requests beside a shared projection
// (mixfp4_lora, mixfp4_lora_backward).  Tokens lie request by request; a
// request's tokens use its adapter (A [R][K], B [N][R], scaling s):
//
//   u = x A^T             shrink   y  = base + s u B^T     expand
//   v = s dy B            shrink   dx = base + v A         expand
//   dA = sum_t v^T x      grad     dB = s sum_t dy^T u     grad
//
// R is small, so every product is bound by reading its tall operand (x, dy) or
// by reading and writing its wide result (y, dx) once: 2 R flops per element of
// 2 to 8 bytes.  All three kernels feed m16n8k16 products from registers, which
// global loads fill directly: which 16 contraction indices a step covers, and
// which column a result register holds, is free, so each thread takes 8 or 16
// bytes that lie together.  A matrix that lies the other way round is put
// together from row pairs by byte permutes.
//
// Measured: 2999 tokens of 12 requests, rank 32, 4096 -> 14336 features, 79 us:
// the expansion 65 (344 MB, 78 % of the measured HBM rate), the shrink 15 and
// mostly behind its own latency.  A training step of 4096 tokens, rank 64, 4096
// features either way, 160 us: shrinks 20 and 19, expansions 39 and 36, gradients
// 60, their three products per step at 40 % of the tensor pipe.  32 requests of
// one token, rank 16, 4096 features either way, 8 us of two dependent launches.
//
// u and v are fp32.  Where they enter a product they are cut into three bf16
// parts (24 bits), one product each, so nothing but the inputs' own bf16 is
// rounded below fp32; sums are fp32, each warp's tensor-core chain a share of
// the whole.  The order of every sum depends on the arguments alone (the only
// atomics count tokens).
#include <cuda_runtime.h>
#include <atomic>
#include <cstdint>

#include "host_util.cuh"
#include "kernels.cuh"
#include "ptx.cuh"

namespace mixfp4 {
namespace {

constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;

__device__ __forceinline__ void mma_bf16(float d[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// x, an infinity or NaN as the largest number of its sign.
__device__ __forceinline__ float finite(float x) {
  float y;
  asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(3.402823466e38f));
  return y;
}
// A pair of fp32 as three pairs of bf16 whose sum it is (to 24 bits).  Each part is what the upper 16 bits hold of the
// rest, so all three have the number's sign, and the two lower ones, which 2^-32 of it is added to, are 0 only where it is 0
// (or below 2^-101): of an infinity they are finite, and times an infinity they give that same one.
__device__ __forceinline__ void split3(float lo, float hi, uint32_t w[3]) {
  w[0] = prmt(__float_as_uint(lo), __float_as_uint(hi), 0x7632u);
  lo = finite(lo), hi = finite(hi);
  float l = lo, h = hi;
#pragma unroll
  for (int i = 1; i < 3; ++i) {
    l = __fmaf_rn(lo, 0x1p-32f, __fsub_rn(l, __uint_as_float(__float_as_uint(l) & 0xFFFF0000u)));
    h = __fmaf_rn(hi, 0x1p-32f, __fsub_rn(h, __uint_as_float(__float_as_uint(h) & 0xFFFF0000u)));
    w[i] = prmt(__float_as_uint(l), __float_as_uint(h), 0x7632u);
  }
}

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// A float of the same shared variable in CTA `rank` of the cluster (after a cluster barrier).
__device__ __forceinline__ float peer_load(uint32_t addr, uint32_t rank) {
  float v;
  asm volatile("{ .reg .b32 r; mapa.shared::cluster.u32 r, %1, %2; ld.shared::cluster.f32 %0, [r]; }"
               : "=f"(v) : "r"(addr), "r"(rank) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.aligned;\n barrier.cluster.wait.aligned;" ::: "memory");
}

// 32 bytes of global memory, or zeros.
__device__ __forceinline__ void load32(uint32_t w[8], const void* p, bool ok) {
  if (ok)
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p) : "memory");
  else
    w[0] = w[1] = w[2] = w[3] = w[4] = w[5] = w[6] = w[7] = 0u;
}

struct Segments {
  const int32_t* starts;  // [count + 1]
  const int32_t* ids;     // [count]
  int count, adapters;
  int64_t tokens;
  int grouped;  // tiles of few tokens are taken from all segments of an adapter
};

__device__ __forceinline__ int2 bounds(const Segments& s, int i) {
  const int T = (int)s.tokens;
  const int a = min(max(s.starts[i], 0), T), b = min(max(s.starts[i + 1], 0), T);
  return make_int2(a, max(a, b));
}
__device__ __forceinline__ int adapter_of(const Segments& s, int i) {
  const int a = s.ids[i];
  return a >= 0 && a < s.adapters ? a : -1;
}

struct Tile {
  int t0, t1, adapter;
};

// The `index`-th tile of at most kTile tokens, counted through the segments in
// order (t0 = t1: there is none).  All threads of the CTA call this.
template <int kTile>
__device__ __forceinline__ Tile find_tile(const Segments& s, int index) {
  __shared__ int scan[kWarps];
  __shared__ int found[3];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int strip = (s.count + kThreads - 1) / kThreads;
  const int lo = min(s.count, tid * strip), hi = min(s.count, lo + strip);
  int mine = 0;
  for (int i = lo; i < hi; ++i) {
    const int2 r = bounds(s, i);
    mine += (r.y - r.x + kTile - 1) / kTile;
  }
  int before = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int v = __shfl_up_sync(kAll, before, d);
    if (lane >= d) before += v;
  }
  if (lane == 31) scan[warp] = before;
  if (tid == 0) found[0] = found[1] = 0, found[2] = -1;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w)
    if (w < warp) before += scan[w];
  before -= mine;
  if (index >= before && index < before + mine) {
    int at = before;
    for (int i = lo; i < hi; ++i) {
      const int2 r = bounds(s, i);
      const int n = (r.y - r.x + kTile - 1) / kTile;
      if (index < at + n) {
        found[0] = r.x + (index - at) * kTile;
        found[1] = min(r.y, found[0] + kTile);
        found[2] = adapter_of(s, i);
        break;
      }
      at += n;
    }
  }
  __syncthreads();
  return Tile{found[0], found[1], found[2]};
}

// The same where segments are short: t0 = 0, t1 the number of tokens, and which
// they are in `rows`.  Grouped, an adapter's tokens are one list through its
// segments in order, and tokens without one are another's, so that requests that
// share an adapter share the reading of it and the rows of a product (256
// requests of one token on 32 adapters of rank 16, 8192 features either way: 17
// us against 47; 128 on 4 of rank 64: 15 against 53; 64 on 64: 20 against 19).
// An adapter's count is kept in shared memory, which bounds their number; the
// scan of the segments is every CTA's, which bounds theirs.
constexpr int kBins = 1024, kMostGrouped = 4096;

template <int kTile>
__device__ __forceinline__ Tile find_rows(const Segments& s, int index, int rows[kTile]) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (!s.grouped) {
    const Tile tile = find_tile<kTile>(s, index);
    if (tid < kTile) rows[tid] = tile.t0 + tid;
    __syncthreads();
    return Tile{0, tile.t1 - tile.t0, tile.adapter};
  }
  __shared__ int bins[kBins + 1];  // tokens of every adapter, and of none
  __shared__ int scan[kWarps];
  __shared__ int found[3];         // the adapter, the tile's first token in its list, the tokens from there on
  const int lists = s.adapters + 1;
  for (int i = tid; i < lists; i += kThreads) bins[i] = 0;
  if (tid < kTile) rows[tid] = 0;
  if (tid == 0) found[0] = -1, found[1] = found[2] = 0;
  __syncthreads();
  auto list_of = [&](int i) {
    const int a = adapter_of(s, i);
    return a < 0 ? s.adapters : a;
  };
  for (int i = tid; i < s.count; i += kThreads) {
    const int2 r = bounds(s, i);
    if (r.y > r.x) atomicAdd(&bins[list_of(i)], r.y - r.x);
  }
  __syncthreads();
  const int strip = (lists + kThreads - 1) / kThreads;
  const int lo = min(lists, tid * strip), hi = min(lists, lo + strip);
  int mine = 0;
  for (int i = lo; i < hi; ++i) mine += (bins[i] + kTile - 1) / kTile;
  auto sum_to = [&](int v) {  // over the threads up to this one
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(kAll, v, d);
      if (lane >= d) v += o;
    }
    if (lane == 31) scan[warp] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w)
      if (w < warp) v += scan[w];
    return v;
  };
  int at = sum_to(mine) - mine;
  if (index >= at && index < at + mine)
    for (int i = lo; i < hi; ++i) {
      const int n = (bins[i] + kTile - 1) / kTile;
      if (index < at + n) {
        found[0] = i, found[1] = (index - at) * kTile, found[2] = bins[i] - found[1];
        break;
      }
      at += n;
    }
  __syncthreads();
  const int list = found[0], first = found[1], count = min(kTile, found[2]);
  for (int i0 = 0, done = 0; i0 < s.count && done < first + count; i0 += kThreads) {
    const int i = i0 + tid;
    const int2 r = i < s.count && list_of(i) == list ? bounds(s, i) : make_int2(0, 0);
    const int before = done + sum_to(r.y - r.x) - (r.y - r.x);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) done += scan[w];
    for (int j = 0; j < count; ++j) {
      const int x = first + j - before;
      if (x >= 0 && x < r.y - r.x) rows[j] = r.x + x;
    }
    __syncthreads();  // `scan` has been read
  }
  return Tile{0, count, list < s.adapters ? list : -1};
}

// ---- shrink: out[t][r] = factor_a sum_k in[t][k] W_a[r][k], k < kdim -------------------------------
// Ranks are the rows of the products (RT tiles of 16), tokens their columns
// (TT / 8 tiles of 8).  A step covers 64 k, a whole 128-byte line of a row:
// thread (g, t) holds k 16t .. 16t + 15 of its rows.  A step's sum is its own
// and is added by the fp32 units: in one chain the tensor cores' rounding
// towards zero left dB of 13504 features 1.8e-6 off, so it is 1.6e-7.  Warps
// take steps in turn, the CTAs of a cluster shares of k; both are summed in
// order through shared memory.  (Staging 64 tokens and W's chunks in shared
// memory by cp.async, for half the reads from L2, gained nothing: 160 us
// against 160 us for the training step of 4096 tokens at rank 64.)
struct ShrinkArgs {
  const uint16_t* in;  // [tokens][ld]
  int64_t ld;
  const uint16_t* w;   // [adapters][R][kdim], or kTrans: [adapters][kdim][R]
  const float* factor; // [adapters] or NULL
  float* out;          // [tokens][R]
  int64_t kdim;
  int R, splits;
  Segments seg;
};

template <int RT, int TT, bool kTrans>
__global__ void __launch_bounds__(kThreads, 2) lora_shrink_kernel(const ShrinkArgs p) {
  extern __shared__ float part[];  // [warps][16 RT][TT], then the CTA's sum in the first
  constexpr int kOut = 16 * RT * TT;
  griddep_launch_dependents();  // launched plainly: what comes before it on the stream is done
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int split = (int)(blockIdx.x % p.splits);
  constexpr bool kRows = TT == 8;
  __shared__ int rows[TT];
  const Tile tile = kRows ? find_rows<TT>(p.seg, (int)(blockIdx.x / p.splits), rows)
                          : find_tile<TT>(p.seg, (int)(blockIdx.x / p.splits));
  auto token = [&](int i) { return (int64_t)(kRows ? rows[i] : i); };  // i: from tile.t0 on
  if (tile.t0 >= tile.t1) return;  // the whole cluster alike
  const int r0 = blockIdx.y * 16 * RT;
  if (tile.adapter < 0) {
    if (split == 0)
      for (int i = threadIdx.x; i < kOut; i += kThreads) {
        const int tok = tile.t0 + i / (16 * RT), r = r0 + i % (16 * RT);
        if (tok < tile.t1 && r < p.R) p.out[token(tok) * p.R + r] = 0.0f;
      }
    return;
  }
  const uint16_t* w = p.w + (int64_t)tile.adapter * p.R * p.kdim;
  const int64_t steps = (p.kdim + 63) / 64;
  const int64_t s0 = steps * split / p.splits, s1 = steps * (split + 1) / p.splits;

  float acc[RT][TT / 8][4];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int n = 0; n < TT / 8; ++n) acc[i][n][0] = acc[i][n][1] = acc[i][n][2] = acc[i][n][3] = 0.0f;

  for (int64_t s = s0 + warp; s < s1; s += kWarps) {
    const int64_t k = s * 64 + 16 * t;
    const bool in_k = k < p.kdim;
    uint32_t x[TT / 8][8];
#pragma unroll
    for (int n = 0; n < TT / 8; ++n) {
      const int tok = tile.t0 + 8 * n + g;
      load32(x[n], p.in + token(tok) * p.ld + k, in_k && tok < tile.t1);
    }
    if (!kTrans) {
      uint32_t a[RT][2][8];
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = r0 + 16 * i + 8 * h + g;
          load32(a[i][h], w + (int64_t)r * p.kdim + k, in_k && r < p.R);
        }
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int n = 0; n < TT / 8; ++n) {
          float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int q = 0; q < 4; ++q)
            mma_bf16(d, a[i][0][2 * q], a[i][1][2 * q], a[i][0][2 * q + 1], a[i][1][2 * q + 1], x[n][2 * q],
                     x[n][2 * q + 1]);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][n][e] += d[e];
        }
    } else {
      // Rows k .. k + 15 at the thread's ranks 2 RT g ..: words of rank pairs, permuted to k pairs.
      uint32_t a[16][RT];
      const int r = r0 + 2 * RT * g;
      const bool ok = in_k && r < p.R;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const uint16_t* src = w + (k + j) * p.R + r;
        if constexpr (RT == 2) {
          const uint2 v = ok ? *reinterpret_cast<const uint2*>(src) : make_uint2(0, 0);
          a[j][0] = v.x, a[j][1] = v.y;
        } else {
          a[j][0] = ok ? *reinterpret_cast<const uint32_t*>(src) : 0u;
        }
      }
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        uint32_t f[4][4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            f[q][2 * h] = prmt(a[4 * q + 2 * h][i], a[4 * q + 2 * h + 1][i], 0x5410u);
            f[q][2 * h + 1] = prmt(a[4 * q + 2 * h][i], a[4 * q + 2 * h + 1][i], 0x7632u);
          }
#pragma unroll
        for (int n = 0; n < TT / 8; ++n) {
          float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int q = 0; q < 4; ++q)
            mma_bf16(d, f[q][0], f[q][1], f[q][2], f[q][3], x[n][2 * q], x[n][2 * q + 1]);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][n][e] += d[e];
        }
      }
    }
  }

  // Rank (row) and token (column) of every result register.
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int n = 0; n < TT / 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = kTrans ? 2 * RT * g + 2 * i + (e >> 1) : 16 * i + g + 8 * (e >> 1);
        part[(warp * TT + 8 * n + 2 * t + (e & 1)) * (16 * RT) + r] = acc[i][n][e];
      }
  __syncthreads();
  for (int i = threadIdx.x; i < kOut; i += kThreads) {
    float v = part[i];
#pragma unroll
    for (int q = 1; q < kWarps; ++q) v += part[q * kOut + i];
    part[i] = v;
  }
  if (p.splits > 1) cluster_barrier();
  else __syncthreads();
  const float f = p.factor ? p.factor[tile.adapter] : 1.0f;
  for (int i = split * kThreads + threadIdx.x; i < kOut; i += p.splits * kThreads) {
    const int tok = tile.t0 + i / (16 * RT), r = r0 + i % (16 * RT);
    float v = 0.0f;
    for (int q = 0; q < p.splits; ++q) v += p.splits > 1 ? peer_load(smem_addr(part + i), q) : part[i];
    if (tok < tile.t1 && r < p.R) p.out[token(tok) * p.R + r] = f * v;
  }
  if (p.splits > 1) cluster_barrier();  // no CTA leaves while others read its sum
}

// ---- expand: out[t][n] = base[t][n] + factor_a sum_r u[t][r] W_a[n][r] -----------------------------
// Tokens are the rows of the products (16), features their columns: product j
// of a warp's 8 NP features has column c at feature NP c + j, so that thread
// (g, t) ends with features 2 NP t .. of tokens g and g + 8, which it reads and
// writes 32 bytes at a time.  A step covers 16 ranks, thread t holding
// 4 t .. 4 t + 3.  The CTA's warps share the tokens: u is cut into its three
// parts once, in shared memory as the fragments they read.
struct ExpandArgs {
  const float* u;      // [tokens][R]
  const uint16_t* w;   // [adapters][N][R], or kTrans: [adapters][R][N]
  const float* factor; // [adapters] or NULL
  const float* base;   // [tokens][ld_base] or NULL
  int64_t ld_base;
  float* out;          // [tokens][ld_out]
  int64_t ld_out;
  int64_t N;
  int R, vec;
  Segments seg;
};

// The B fragments of 16 ranks for the warp's features; n: the thread's first (NP g on).
template <bool kTrans, int NP>
__device__ __forceinline__ void expand_w(uint32_t b[NP][2], const uint16_t* w, int r, int R, int64_t n, int64_t N) {
  const bool in_r = r < R;
  if (!kTrans) {
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const uint2 q = in_r && n + j < N ? *reinterpret_cast<const uint2*>(w + (n + j) * R + r) : make_uint2(0, 0);
      b[j][0] = q.x, b[j][1] = q.y;
    }
  } else {
    uint2 q[NP / 4][4];
#pragma unroll
    for (int k = 0; k < NP / 4; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        q[k][i] = in_r && n < N ? *reinterpret_cast<const uint2*>(w + (int64_t)(r + i) * N + n + 4 * k)
                                : make_uint2(0, 0);
#pragma unroll
    for (int k = 0; k < NP / 4; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        b[4 * k][h] = prmt(q[k][2 * h].x, q[k][2 * h + 1].x, 0x5410u);
        b[4 * k + 1][h] = prmt(q[k][2 * h].x, q[k][2 * h + 1].x, 0x7632u);
        b[4 * k + 2][h] = prmt(q[k][2 * h].y, q[k][2 * h + 1].y, 0x5410u);
        b[4 * k + 3][h] = prmt(q[k][2 * h].y, q[k][2 * h + 1].y, 0x7632u);
      }
  }
}

// kHeld: steps (of 16 ranks) whose part of W a warp keeps in registers for all its tokens; further ranks are read
// again for every 16 tokens.
template <int TT, bool kTrans, int kHeld, int NP>
__global__ void __launch_bounds__(kThreads, 2) lora_expand_kernel(const ExpandArgs p) {
  extern __shared__ uint4 frag[];  // [m][step][part][lane]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  constexpr bool kRows = TT == 16;
  __shared__ int rows[TT];
  const Tile tile = kRows ? find_rows<TT>(p.seg, (int)blockIdx.x, rows) : find_tile<TT>(p.seg, (int)blockIdx.x);
  auto token = [&](int i) { return (int64_t)(kRows ? rows[i] : i); };  // i: from tile.t0 on
  const int steps = (p.R + 15) / 16;
  const int64_t n0 = ((int64_t)blockIdx.y * kWarps + warp) * (8 * NP);
  const uint16_t* w = p.w + (int64_t)max(tile.adapter, 0) * p.R * p.N;
  const bool some = tile.t0 < tile.t1 && tile.adapter >= 0;
  uint32_t held[kHeld][NP][2];
#pragma unroll
  for (int st = 0; st < kHeld; ++st)
    expand_w<kTrans, NP>(held[st], w, some ? st * 16 + 4 * t : p.R, p.R, n0 + NP * g, p.N);
  griddep_wait();
  griddep_launch_dependents();  // not before: what may start then counts on the kernel before this one
  if (tile.t0 >= tile.t1) return;
  if (tile.adapter >= 0)
    for (int i = threadIdx.x; i < (tile.t1 - tile.t0 + 15) / 16 * steps * 32; i += kThreads) {
      const int ms = i / 32, m = ms / steps, l = i % 32;
      const int r = (ms - m * steps) * 16 + 4 * (l & 3), ta = tile.t0 + 16 * m + (l >> 2);
      const float4 z = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      const float4 ua = r < p.R && ta < tile.t1 ? *reinterpret_cast<const float4*>(p.u + token(ta) * p.R + r) : z;
      const float4 ub =
          r < p.R && ta + 8 < tile.t1 ? *reinterpret_cast<const float4*>(p.u + token(ta + 8) * p.R + r) : z;
      uint32_t a0[3], a1[3], a2[3], a3[3];
      split3(ua.x, ua.y, a0);
      split3(ub.x, ub.y, a1);
      split3(ua.z, ua.w, a2);
      split3(ub.z, ub.w, a3);
#pragma unroll
      for (int q = 0; q < 3; ++q) frag[(ms * 3 + q) * 32 + l] = make_uint4(a0[q], a1[q], a2[q], a3[q]);
    }
  __syncthreads();
  if (n0 >= p.N) return;
  const float f = tile.adapter < 0 ? 0.0f : (p.factor ? p.factor[tile.adapter] : 1.0f);
  const int64_t nt = n0 + 2 * NP * t;  // this thread's results
  const bool vec = p.vec && nt + 2 * NP <= p.N;
  for (int m = 0; tile.t0 + 16 * m < tile.t1; ++m) {
    const int ta = tile.t0 + 16 * m + g;
    float v[2][2 * NP];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float* b = p.base + token(ta + 8 * h) * p.ld_base + nt;
      const bool there = p.base && ta + 8 * h < tile.t1;
      if (vec) {
#pragma unroll
        for (int q = 0; q < 2 * NP; q += 8) load32(reinterpret_cast<uint32_t*>(v[h] + q), b + q, there);
      } else {
#pragma unroll
        for (int q = 0; q < 2 * NP; ++q) v[h][q] = there && nt + q < p.N ? b[q] : 0.0f;
      }
    }
    float acc[NP][4];
#pragma unroll
    for (int j = 0; j < NP; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
    if (tile.adapter >= 0) {
      auto multiply = [&](int st, const uint32_t(&b)[NP][2]) {
#pragma unroll
        for (int i = 2; i >= 0; --i) {  // the small parts first
          const uint4 a = frag[((m * steps + st) * 3 + i) * 32 + lane];
#pragma unroll
          for (int j = 0; j < NP; ++j) mma_bf16(acc[j], a.x, a.y, a.z, a.w, b[j][0], b[j][1]);
        }
      };
#pragma unroll
      for (int st = 0; st < kHeld; ++st)
        if (st < steps) multiply(st, held[st]);
      if (kHeld == 4)
        for (int st = kHeld; st < steps; ++st) {
          uint32_t b[NP][2];
          expand_w<kTrans, NP>(b, w, st * 16 + 4 * t, p.R, n0 + NP * g, p.N);
          multiply(st, b);
        }
    }
    // acc[j]: (token g, features 2 NP t + j and 2 NP t + NP + j), then token g + 8
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (ta + 8 * h >= tile.t1) continue;
#pragma unroll
      for (int q = 0; q < 2 * NP; ++q) v[h][q] = fmaf(f, acc[q % NP][2 * h + q / NP], v[h][q]);
      float* o = p.out + token(ta + 8 * h) * p.ld_out + nt;
      if (vec) {
#pragma unroll
        for (int q = 0; q < 2 * NP; q += 8) stg256(o + q, reinterpret_cast<const uint32_t*>(v[h] + q));
      } else {
#pragma unroll
        for (int q = 0; q < 2 * NP; ++q)
          if (nt + q < p.N) o[q] = v[h][q];
      }
    }
  }
}

// ---- grad: dW_a[r][n] = factor_a sum_t c[t][r] z[t][n] over adapter a's tokens ----------------------
// Ranks are the rows of the products (RT tiles of 16, thread g holding ranks
// 2 RT g ..), features their columns as in expand (64 to a CTA), tokens the
// contraction (16 a step).  The tokens of an adapter are one list through its
// segments; the CTA's warps take its steps in turn, each on its own (rows of c
// and z asked for a step ahead, c cut into its three parts in registers), and
// their sums are added in order at the end.
struct GradArgs {
  const float* c[2];       // v, u: [tokens][R]
  const uint16_t* z[2];    // x, dy: [tokens][ld]
  int64_t ld[2];
  const float* factor[2];  // NULL, scaling
  float* out[2];           // dA [adapters][R][K], dB [adapters][N][R]
  int64_t dim[2];          // K, N
  int blocks[2];           // 64-feature blocks of each
  int R;
  int beside;              // the kernel before this one on the stream writes nothing that is read here
  Segments seg;
};

constexpr int kTogether = 2;

template <int RT, int NW>
__global__ void __launch_bounds__(32 * NW, NW == 8 ? 1 : (RT == 4 ? 2 : 3)) lora_grad_kernel(const GradArgs p) {
  extern __shared__ float4 sums[];  // [half the warps][tile][product][lane]
  constexpr int threads = 32 * NW, warps = NW;
  __shared__ int ends[threads], first[threads], count[warps], found[warps];
  // Beside the expansion of v, which lets this kernel start when v is there, it waits at its end instead: the stream's
  // next kernel counts on both.
  if (!p.beside) griddep_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int which = (int)blockIdx.x >= p.blocks[0];
  const int64_t n0 = (int64_t)((int)blockIdx.x - (which ? p.blocks[0] : 0)) * 64;
  const int adapter = blockIdx.y, r0 = blockIdx.z * 16 * RT, rg = r0 + 2 * RT * g;
  const int64_t ld = p.ld[which], N = p.dim[which];
  const bool in_n = n0 + 8 * g < N, in_r = rg < p.R;
  const uint16_t* z = p.z[which] + n0 + 8 * g;
  const float* c = p.c[which] + rg;

  float acc[RT][8][4];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j][0] = acc[i][j][1] = acc[i][j][2] = acc[i][j][3] = 0.0f;

  for (int s0 = 0; s0 < p.seg.count; s0 += threads) {
    // This batch's segments of the adapter, in order: first tokens and running ends of their lengths.
    const int i = s0 + tid;
    int2 r = make_int2(0, 0);
    if (i < p.seg.count && adapter_of(p.seg, i) == adapter) r = bounds(p.seg, i);
    const int len = r.y - r.x;
    const uint32_t some = __ballot_sync(kAll, len > 0);
    // Sums end at INT_MAX: segments that overlap may hold more tokens than an int counts.
    auto plus = [](int a, int b) { return (int)min((uint32_t)a + (uint32_t)b, (uint32_t)INT32_MAX); };
    int sum = len;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int v = __shfl_up_sync(kAll, sum, d);
      if (lane >= d) sum = plus(sum, v);
    }
    __syncthreads();  // the batch before has been used
    if (lane == 31) count[warp] = sum, found[warp] = __popc(some);
    __syncthreads();
    int at = __popc(some & ((1u << lane) - 1u)), off = sum, lists = 0, total = 0;
    for (int q = 0; q < warps; ++q) {
      if (q < warp) at += found[q], off = plus(off, count[q]);
      lists += found[q], total = plus(total, count[q]);
    }
    if (total > (int)p.seg.tokens) total = 0;  // more than there are: none is taken
    if (len > 0) first[at] = r.x - (off - len), ends[at] = off;  // token = index + first
    __syncthreads();
    int top = 1;
    while (top < lists) top <<= 1;
    const int steps = (total + 15) / 16;

    // Tokens 2t, 2t + 1, 2t + 8, 2t + 9 of a step (-1 behind the last).  Lane l finds token l % 16: it lies in the
    // first list whose end lies beyond it.
    int tk[4];
    auto find = [&](int step) {
      const int want = step * 16 + (lane & 15);
      int lo = 0;
      for (int h = top >> 1; h; h >>= 1)
        if (lo + h <= lists - 1 && ends[lo + h - 1] <= want) lo += h;
      const int tok = want < total ? want + first[lo] : -1;
#pragma unroll
      for (int q = 0; q < 4; ++q) tk[q] = __shfl_sync(kAll, tok, 2 * t + (q & 1) + 8 * (q >> 1));
    };
    uint4 zw[4];
    float2 cv[RT][4];
    auto load_z = [&]() {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        zw[q] = tk[q] >= 0 && in_n ? *reinterpret_cast<const uint4*>(z + tk[q] * ld) : make_uint4(0, 0, 0, 0);
    };
    auto load_c = [&](int h) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        cv[h][q] = tk[q] >= 0 && in_r ? *reinterpret_cast<const float2*>(c + (int64_t)tk[q] * p.R + 2 * h)
                                      : make_float2(0.0f, 0.0f);
    };
    if (warp < steps) {
      find(warp);
      load_z();
#pragma unroll
      for (int h = 0; h < RT; ++h) load_c(h);
    }
    for (int step = warp; step < steps; step += warps) {
      const bool more = step + warps < steps;
      const uint32_t zz[4][4] = {{zw[0].x, zw[0].y, zw[0].z, zw[0].w},
                                 {zw[1].x, zw[1].y, zw[1].z, zw[1].w},
                                 {zw[2].x, zw[2].y, zw[2].z, zw[2].w},
                                 {zw[3].x, zw[3].y, zw[3].z, zw[3].w}};
      uint32_t b[8][2];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t sel = j & 1 ? 0x7632u : 0x5410u;
        b[j][0] = prmt(zz[0][j / 2], zz[1][j / 2], sel), b[j][1] = prmt(zz[2][j / 2], zz[3][j / 2], sel);
      }
      if (more) {
        find(step + warps);
        load_z();
      }
      // A step's sum is its own and is added by the fp32 units: the tensor cores round a long chain of sums
      // towards zero (4096 tokens of four adapters: the gradients' error 1.9e-6 in one chain, 5.2e-7 so).
#pragma unroll
      for (int h = 0; h < RT; ++h) {
        uint32_t a[4][3];
        split3(cv[h][0].x, cv[h][1].x, a[0]);
        split3(cv[h][0].y, cv[h][1].y, a[1]);
        split3(cv[h][2].x, cv[h][3].x, a[2]);
        split3(cv[h][2].y, cv[h][3].y, a[3]);
        if (more) load_c(h);
#pragma unroll
        for (int j0 = 0; j0 < 8; j0 += kTogether) {
          float d[kTogether][4];
#pragma unroll
          for (int j = 0; j < kTogether; ++j) d[j][0] = d[j][1] = d[j][2] = d[j][3] = 0.0f;
#pragma unroll
          for (int q = 2; q >= 0; --q)
#pragma unroll
            for (int j = 0; j < kTogether; ++j)
              mma_bf16(d[j], a[0][q], a[1][q], a[2][q], a[3][q], b[j0 + j][0], b[j0 + j][1]);
#pragma unroll
          for (int j = 0; j < kTogether; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[h][j0 + j][e] += d[j][e];
        }
      }
    }
  }

  // The upper half of the warps' sums are added to the lower's, and so on.
  for (int half = warps / 2; half >= 1; half /= 2) {
    __syncthreads();
    if (warp >= half && warp < 2 * half) {
#pragma unroll
      for (int h = 0; h < RT; ++h)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          sums[((warp - half) * RT * 8 + h * 8 + j) * 32 + lane] =
              make_float4(acc[h][j][0], acc[h][j][1], acc[h][j][2], acc[h][j][3]);
    }
    __syncthreads();
    if (warp < half) {
#pragma unroll
      for (int h = 0; h < RT; ++h)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float4 v = sums[(warp * RT * 8 + h * 8 + j) * 32 + lane];
          acc[h][j][0] += v.x, acc[h][j][1] += v.y, acc[h][j][2] += v.z, acc[h][j][3] += v.w;
        }
    }
  }
  // acc[h][j]: ranks 2 RT g + 2 h (+ 1 for registers 2, 3), features 16 t + j (+ 8 for registers 1, 3)
  if (p.beside) griddep_wait();
  if (warp > 0 || n0 + 16 * t >= N || !in_r) return;
  const float f = p.factor[which] ? p.factor[which][adapter] : 1.0f;
  if (!which) {  // rows of features
#pragma unroll
    for (int h = 0; h < RT; ++h)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float* to = p.out[0] + ((int64_t)adapter * p.R + rg + 2 * h + e) * N + n0 + 16 * t;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t v[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = __float_as_uint(f * acc[h][j][2 * e + q]);
          stg256(to + 8 * q, v);
        }
      }
  } else {  // rows of ranks
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float* to = p.out[1] + ((int64_t)adapter * N + n0 + 16 * t + 8 * q + j) * p.R + rg;
#pragma unroll
        for (int h = 0; h < RT; ++h)
          *reinterpret_cast<float2*>(to + 2 * h) = make_float2(f * acc[h][j][q], f * acc[h][j][2 + q]);
      }
  }
}

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Tiles of at most `size` tokens, no fewer than there are.
int64_t tiles_of(const Segments& s, int size, bool rows) {
  return s.tokens / size + (rows && s.grouped && s.adapters < s.count ? s.adapters + 1 : s.count);
}

template <int RT, int TT, bool kTrans>
int launch_shrink(const ShrinkArgs& p, cudaStream_t s) {
  const int smem = kWarps * 16 * RT * TT * 4;
  auto* kernel = lora_shrink_kernel<RT, TT, kTrans>;
  static std::atomic<uint64_t> done{0};
  if (smem > 48 * 1024 && !set_dynamic_smem_once(reinterpret_cast<const void*>(kernel), smem, done))
    return MIXFP4_ERR_CUDA;
  const int64_t tiles = tiles_of(p.seg, TT, TT == 8);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.splits, attr[0].val.clusterDim.y = 1, attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * p.splits), (unsigned)((p.R + 16 * RT - 1) / (16 * RT)));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p) == cudaSuccess ? MIXFP4_OK : MIXFP4_ERR_CUDA;
}

// Tiles of 8 tokens where segments are short, of 32 else: 256 requests of one token 46 us against 52 with 32 (before
// grouping), 4096 tokens of one segment 160 against 206 with 8.
template <bool kTrans>
int shrink(ShrinkArgs p, cudaStream_t s) {
  const bool few = p.seg.tokens <= 8 * (int64_t)p.seg.count;
  const int64_t tiles = few ? tiles_of(p.seg, 8, true) : tiles_of(p.seg, 32, false);
  // Ranks of a CTA: 16, or 32 (x is read again for every 32 ranks, from L2; 64 in one CTA left registers for
  // half the loads in flight).  CTAs: k is cut until there are more of them than SMs, which hold two (32 requests, 4096
  // features either way: 10.5 us, 13 with k in one piece).
  const int rt = p.R <= 16 ? 1 : 2;
  const int64_t ctas = tiles * ((p.R + 16 * rt - 1) / (16 * rt));
  p.splits = 1;
  while (p.splits < 8 && ctas * p.splits <= num_sms() && p.kdim >= 128 * kWarps * p.splits) p.splits *= 2;
  if (few) return rt == 1 ? launch_shrink<1, 8, kTrans>(p, s) : launch_shrink<2, 8, kTrans>(p, s);
  return rt == 1 ? launch_shrink<1, 32, kTrans>(p, s) : launch_shrink<2, 32, kTrans>(p, s);
}

template <int TT, bool kTrans, int kHeld, int NP>
int launch_expand(const ExpandArgs& p, cudaStream_t s) {
  constexpr int kStep = TT / 16 * 3 * 512, kMost = 8 * kStep;  // fragments of 16 ranks, of 128
  auto* kernel = lora_expand_kernel<TT, kTrans, kHeld, NP>;
  static std::atomic<uint64_t> done{0};
  if (!set_dynamic_smem_once(reinterpret_cast<const void*>(kernel), kMost, done)) return MIXFP4_ERR_CUDA;
  const dim3 grid((unsigned)tiles_of(p.seg, TT, TT == 16), (unsigned)((p.N + 8 * NP * kWarps - 1) / (8 * NP * kWarps)));
  return launch_pdl(kernel, grid, dim3(kThreads), (size_t)((p.R + 15) / 16 * kStep), s, p) == cudaSuccess
             ? MIXFP4_OK
             : MIXFP4_ERR_CUDA;
}

// Up to 32 ranks a warp takes 64 features (2999 tokens, rank 32, 14336 features: 63 us against 73 us with 32), beyond
// that 32, whose part of W leaves registers for twice the warps (4096 tokens, rank 64, 4096 features: 41 against 47 us).
template <int TT, bool kTrans>
int expand_held(const ExpandArgs& p, cudaStream_t s) {
  if (p.R <= 16) return launch_expand<TT, kTrans, 1, 8>(p, s);
  return p.R <= 32 ? launch_expand<TT, kTrans, 2, 8>(p, s) : launch_expand<TT, kTrans, 4, 4>(p, s);
}

// Tokens of a CTA (W is read, and u cut, once a CTA): no more than most segments have, and no more than leave the
// device a round of CTAs.  64 against 16: 2999 tokens, rank 32, 14336 features 80 against 104 us; 333 tokens of 7
// requests 29 against 25 (a training step), 500 of 3 17 against 12.
template <bool kTrans>
int expand(const ExpandArgs& p, cudaStream_t s) {
  const int64_t features = (p.R <= 32 ? 64 : 32) * kWarps, blocks = (p.N + features - 1) / features;
  const int64_t T = p.seg.tokens, S = p.seg.count;
  auto fits = [&](int tokens) { return T >= tokens / 2 * S && (T / tokens + S / 2) * blocks >= 2 * num_sms(); };
  return fits(64) ? expand_held<64, kTrans>(p, s) : expand_held<16, kTrans>(p, s);
}

template <int RT, int NW>
int launch_grad(const GradArgs& p, dim3 grid, cudaStream_t s) {
  auto* kernel = lora_grad_kernel<RT, NW>;
  static std::atomic<uint64_t> done{0};
  constexpr int kSums = NW / 2 * RT * 8 * 512;
  if (kSums > 32 * 1024 && !set_dynamic_smem_once(reinterpret_cast<const void*>(kernel), kSums, done))
    return MIXFP4_ERR_CUDA;
  return launch_pdl(kernel, grid, dim3(32 * NW), (size_t)kSums, s, p) == cudaSuccess ? MIXFP4_OK : MIXFP4_ERR_CUDA;
}

template <int RT>
int grad(GradArgs p, cudaStream_t s) {
  for (int i = 0; i < 2; ++i) p.blocks[i] = (int)((p.dim[i] + 63) / 64);
  const dim3 grid((unsigned)(p.blocks[0] + p.blocks[1]), (unsigned)p.seg.adapters,
                  (unsigned)((p.R + 16 * RT - 1) / (16 * RT)));
  // Four warps to a CTA, some CTAs side by side on an SM; eight where there would not be two CTAs to an SM.  4 against 8:
  // 4096 tokens of 4 adapters of rank 16 107 against 114 us, of one of rank 64 207 against 168, with 1024 features 90
  // against 65.
  return (int64_t)grid.x * grid.y * grid.z >= 2 * num_sms() ? launch_grad<RT, 4>(p, grid, s)
                                                            : launch_grad<RT, 8>(p, grid, s);
}

// Whether tiles of few tokens are taken from all segments of an adapter.
bool grouped(int64_t T, int64_t adapters, int64_t segments) {
  return T <= 8 * segments && segments > 8 && segments <= kMostGrouped && adapters <= kBins;
}

// The arguments both entry points share.
int check_lora(int64_t T, int64_t K, int64_t N, int64_t R, int64_t adapters, const void* a, const void* b,
               const float* scaling, const int32_t* starts, const int32_t* ids, int64_t segments) {
  if (T < 0 || T > INT32_MAX - 4096 || K < 0 || K % 16 != 0 || N < 0 || R < 8 || R > 128 || R % 8 != 0 ||
      adapters < 0 || adapters > 65535 || segments < 0 || segments > (1 << 20) || N > ((int64_t)1 << 22) ||
      K > ((int64_t)1 << 22))
    return MIXFP4_ERR_SHAPE;
  if (!starts || (segments > 0 && !ids) || (adapters > 0 && ((K > 0 && !a) || (N > 0 && !b) || !scaling)))
    return MIXFP4_ERR_NULL;
  if (!aligned(a, 32) || !aligned(b, 32) || !aligned(scaling, 4) || !aligned(starts, 4) || !aligned(ids, 4))
    return MIXFP4_ERR_ALIGN;
  return MIXFP4_OK;
}

inline bool vec_ok(const float* p, int64_t ld) { return aligned(p, 32) && ld % 8 == 0; }

}  // namespace
}  // namespace mixfp4

extern "C" {

int mixfp4_lora(const void* x, int dtype, int64_t T, int64_t K, int64_t ldx, const void* a, const void* b,
                const float* scaling, int64_t adapters, int64_t R, int64_t N, const int32_t* starts,
                const int32_t* ids, int64_t segments, const float* base, int64_t ld_base, float* out, int64_t ld_out,
                float* u, void* stream) {
  using namespace mixfp4;
  if (dtype != MIXFP4_DTYPE_BF16) return MIXFP4_ERR_DTYPE;
  if (int st = check_lora(T, K, N, R, adapters, a, b, scaling, starts, ids, segments)) return st;
  if (ldx < K || ld_out < N || (base && ld_base < N)) return MIXFP4_ERR_SHAPE;
  if (T == 0 || segments == 0) return MIXFP4_OK;
  if ((K > 0 && !x) || (N > 0 && !out) || !u) return MIXFP4_ERR_NULL;
  if (!aligned(x, 32) || ldx % 16 || !aligned(u, 16) || !aligned(out, 4) || !aligned(base, 4)) return MIXFP4_ERR_ALIGN;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const Segments seg{starts, ids, (int)segments, (int)adapters, T, grouped(T, adapters, segments)};
  const ShrinkArgs sp{static_cast<const uint16_t*>(x), ldx, static_cast<const uint16_t*>(a), nullptr, u, K,
                      (int)R, 1, seg};
  if (int st = shrink<false>(sp, s)) return st;
  if (N == 0) return MIXFP4_OK;
  const ExpandArgs ep{u, static_cast<const uint16_t*>(b), scaling, base, ld_base, out, ld_out, N, (int)R,
                      vec_ok(out, ld_out) && (!base || vec_ok(base, ld_base)), seg};
  return expand<false>(ep, s);
}

int mixfp4_lora_backward(const void* dy, int64_t ldy, const void* x, int64_t ldx, int dtype, int64_t T, int64_t K,
                         const float* u, const void* a, const void* b, const float* scaling, int64_t adapters,
                         int64_t R, int64_t N, const int32_t* starts, const int32_t* ids, int64_t segments,
                         const float* base, int64_t ld_base, float* dx, int64_t ld_dx, float* da, float* db, float* v,
                         void* stream) {
  using namespace mixfp4;
  if (dtype != MIXFP4_DTYPE_BF16) return MIXFP4_ERR_DTYPE;
  if (int st = check_lora(T, K, N, R, adapters, a, b, scaling, starts, ids, segments)) return st;
  if (N % 16 != 0 || ldx < K || ldy < N || ld_dx < K || (base && ld_base < K)) return MIXFP4_ERR_SHAPE;
  const bool tokens = T > 0 && segments > 0;
  if (tokens && ((K > 0 && (!x || !dx)) || (N > 0 && !dy) || !u || !v)) return MIXFP4_ERR_NULL;
  if (adapters > 0 && ((K > 0 && !da) || (N > 0 && !db))) return MIXFP4_ERR_NULL;
  if (!aligned(x, 32) || ldx % 16 || !aligned(dy, 32) || ldy % 16 || !aligned(u, 16) || !aligned(v, 16) ||
      !aligned(dx, 4) || !aligned(base, 4) || !aligned(da, 32) || !aligned(db, 32))
    return MIXFP4_ERR_ALIGN;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const Segments seg{starts, ids, (int)segments, (int)adapters, T, grouped(T, adapters, segments)};
  if (tokens) {
    const ShrinkArgs sp{static_cast<const uint16_t*>(dy), ldy, static_cast<const uint16_t*>(b), scaling, v, N,
                        (int)R, 1, seg};
    if (int st = shrink<true>(sp, s)) return st;
    if (K > 0) {
      const ExpandArgs ep{v, static_cast<const uint16_t*>(a), nullptr, base, ld_base, dx, ld_dx, K, (int)R,
                          vec_ok(dx, ld_dx) && (!base || vec_ok(base, ld_base)), seg};
      if (int st = expand<true>(ep, s)) return st;
    }
  }
  GradArgs gp = {};
  gp.c[0] = v, gp.c[1] = u;
  gp.z[0] = static_cast<const uint16_t*>(x), gp.z[1] = static_cast<const uint16_t*>(dy);
  gp.ld[0] = ldx, gp.ld[1] = ldy;
  gp.factor[1] = scaling;
  gp.out[0] = da, gp.out[1] = db;
  gp.dim[0] = K, gp.dim[1] = N;
  gp.R = (int)R;
  gp.seg = seg;
  if (!tokens) gp.seg.count = 0;
  gp.beside = tokens && K > 0;
  if (adapters == 0 || K + N == 0) return MIXFP4_OK;
  return R <= 16 ? grad<1>(gp, s) : (R <= 32 ? grad<2>(gp, s) : grad<4>(gp, s));
}

}  // extern "C"
