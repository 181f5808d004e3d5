// Attention of one new token per sequence over the paged cache
// (mixfp4_paged_attention).
//
// The cache's rows are read once and met by few queries (q_heads / heads of
// them per key head), so the kernel is bound by HBM: 4 G flops per element
// read, with G = 4 a twentieth of what the tensor cores do meanwhile.  What
// matters is that enough bytes are in flight and that nothing else stands in
// their way.  64 sequences of up to 8192 tokens (half of that on average), 32
// query heads to 8 of 128: 200 us from a bf16 cache, 94 % of the measured HBM
// rate; 2 sequences of 131072 tokens 168 us, likewise.  A MixFP4 cache holds
// 28 % of the bytes, and what is left to do is its decoding: 124 us (44 us of
// HBM time; of the first kernel's 120 us an instruction issues in 62 %, most of
// them of the integer pipe, and the rest is waiting at 12 warps to an SM).
//
//   * Each warp streams 16 tokens at a time into a ring of its own by cp.async,
//     whole rows by neighbouring lanes (an access of half a 128-byte line costs
//     as much as one of the whole: 259 us became 204 us at 64 sequences of up to
//     8192 tokens, 8 heads of 128), and nothing wider than a warp waits for it.
//     Where tiles of 16 positions lie in one page, its number is asked for a
//     tile ahead and one 64-bit address serves the tile.
//   * Tokens are the rows of m16n8k16 products and query heads their 8 columns,
//     so no query row is padded to 16.  S = K Q^T takes K's rows as they lie
//     (four dimensions per thread and step, Q permuted alike); O^T = V^T P^T
//     takes V's as token pairs, put together by byte permutes, and P^T out of
//     S's registers by an 8 x 8 transpose.  m16n8k16 moves these operands from
//     registers; a tcgen05.mma would want them in shared memory in a layout that
//     a paged row does not have.
//   * The weights P keep 16 bits of mantissa in two bf16 parts of one sign (one
//     product each) on a bf16 cache.  On a MixFP4 cache a row's values times its block
//     scales are exact in f16, Q is scaled per head by a power of two into f16
//     (exact but for elements below 2^-31 of the largest, which are off by up to
//     2^-39 of it: half of f16's least step), and P takes 11 bits: the
//     4-bit rows themselves hold 3.
//   * Sequences differ in length, so the axis (sequence, key head, token) is cut
//     into equal shares of 64-token units, one per CTA; where a CTA's share ends
//     inside a row's tokens, both sides leave a partial result (m, l, O) in the
//     workspace, and a second small kernel, launched early, joins them in order
//     (6.6 us of the 200).  Few rows that cannot be long take a cluster of CTAs
//     each instead, joined in shared memory, and many short ones a CTA each (how
//     long they can be is the table's width and the window, all that the host
//     knows: short sequences under a wide table take shares): one sequence of 700
//     tokens 7 us, 40 of up to 120 9 us, 256 of up to 200 30 us.
#include <cuda_runtime.h>
#include <atomic>
#include <cstdint>

#include "decode.cuh"
#include "host_util.cuh"
#include "kernels.cuh"
#include "kvcache.cuh"
#include "ptx.cuh"

namespace mixfp4 {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kJoinThreads = 256;
constexpr int kCluster = 8;
// Tokens to a CTA up to which a cluster to each row (8 CTAs, or 4 or 2 where the rows are more) is the quicker way,
// four times that where clusters fill half the device.  8 key heads of 128, clusters against shares of the whole device
// and a joining kernel: one sequence of 4000 tokens 13 against 25 us, of 8000 19 against 17, of 32000 54 against 33; six
// of 8000 39 against 45, of 16000 67 against 73; 16 of up to 500 10 against 14, of up to 2000 20 against 22.
constexpr int kCtaTokens = 512;
// And up to which one CTA to a row is, whatever their number: 40 sequences of up to 250 12 against 16 us, of up to 500
// 17 against 17; 100 of up to 250 21 against 22, of up to 500 34 against 31; 300 of up to 120 28 against 32.
constexpr int kRowTokens = 256;
// What beginning a row costs (its queries, the way to its first pages, the join of the warps), in units.  Swept in equal
// shares, 0 / 2 / 4 / 6 / 8: 256 sequences of up to 200 tokens under a wide table, 8 heads of 128, 58 / 50 / 46 / 44 / 44
// us; 64 of up to 8192 204 / 198 / 196 / 197 / 197, on a MixFP4 cache 140 / 138 / 136 / 135 / 136.
constexpr int kRowCost = 6;
// Tiles of 16 tokens after which a warp sets its O and l aside.  The tensor cores round a chain of sums towards zero,
// some 2^-25 of the sum a link: a warp that walked 6000 tiles left O 2^-12 too small.  128 tiles (256 links) leave 2^-17,
// for 1 % more bytes, in L2.  In memory the sums take no registers (O joined from registers: 64 sequences of up to 8192
// tokens on a MixFP4 cache 136 to 140 us against 134).
constexpr int kChain = 128;
constexpr int kUnit = 64;  // head rows of a unit of work: 64 / together tokens of `together` key heads
constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// How far a score may lie above the m of its weight 2^(s - m).  On a MixFP4 cache the weights are 2^7 times that:
// below 2^15 in f16, whose least value is then 2^-31 of the weight at m.
constexpr float kSlack = 8.0f, kFp4Exp = 7.0f;
constexpr float kNoScore = -3e38f;  // m where no token has been seen: no difference to a score or to itself is NaN
constexpr float kMostScore = 3.402823466e38f;  // m of a score of +inf, whose weight is then +inf instead of NaN

struct AttnArgs {
  const uint16_t* q;
  int64_t q_stride, q_head_stride;
  int B, q_heads, group, chunks;  // group = q_heads / heads; chunks of 8 NT query heads per key head
  int together;                   // key heads of a CTA: 4, 2 or 1, each a warp's (or two's, or four's)
  int cluster;                    // CTAs to a row: 1, or a cluster of 2, 4 or 8 joined in shared memory; 0: equal shares
  int cluster_shift;              // its log2
  mixfp4_kv_cache c;
  int page_shift;  // log2 page_size, or -1
  const int32_t* table;
  int64_t table_stride;
  int64_t max_tokens;
  const int32_t* lengths;
  float scale;
  int64_t window;
  uint16_t* out;
  float* lse;
  float* part;    // [2 grid][together][8 NT][DT], the partial results
  float2* stat;   // [2 grid][together][8 NT] (m, l)
  float4* aside;  // [grid][warps][NT][kAside][lane]: a warp's O and l so far, in rows of more than kChain tiles
  int4* split;    // rows that go on in later CTAs: (sequence, row, first CTA, last CTA); x < 0: none.  One place for
                  // each row of each sequence, or, where they are fewer, for each CTA, which begins one such row at most.
  int by_row;
  int places;     // of split
  int share;      // warps of the joining kernel to a query head
};

template <int DT, int NT, bool kFp4>
struct Cfg {
  static constexpr int kHeads = 8 * NT;
  static constexpr int kVBytes = kFp4 ? (DT == 64 ? 4 : 8) : 16;       // a thread's piece of a V row
  static constexpr int kVDims = kFp4 ? 2 * kVBytes : 8;
  static constexpr int kVPieces = DT / (8 * kVDims);
  static constexpr int kKDims = kFp4 ? 16 : 8;                         // and of a K row, in elements
  static constexpr int kKPieces = DT / (4 * kKDims);
  // Rows are copied in pieces of kCopy bytes, whole rows by neighbouring lanes, to places that leave the pieces
  // which the lanes read together in different banks: XOR of a piece's number with f(row), for V after rows
  // 2t + e + 8h have been put in the order t + 4e + 8h.
  static constexpr int kCopy = kFp4 ? 8 : 16, kRow = kFp4 ? DT / 2 : DT * 2;
  static constexpr int kPieces = kRow / kCopy, kRowsAtOnce = 32 / kPieces;
  static __device__ __forceinline__ int k_place(int row, int piece) {
    const int f = kFp4 ? (row * kPieces / 16 & (kPieces / 4 - 1)) * 4 : (row & 1) * 4;
    return row * kRow + (piece ^ f) * kCopy;
  }
  static __device__ __forceinline__ int v_place(int row, int piece) {
    const int at = (row & 7) >> 1 | (row & 1) << 2 | (row & 8);
    const int f = kFp4 ? (at * kPieces / 16 & (kPieces / 4 - 1)) * 4 : (at & 3) * 2;
    return at * kRow + (piece ^ f) * kCopy;
  }
  static constexpr int kAside = 2 * (DT / 16) + 1;                     // places of 32 float4 for 8 query heads
  static constexpr int kKTile = 16 * kRow, kVTile = 16 * kRow;
  static constexpr int kScaleTile = kFp4 ? 32 * 16 : 0;                // 16 scale bytes a row at most
  static constexpr int kThere = kKTile + kVTile + kScaleTile;          // which of the tile's tokens there are, a bit each
  static constexpr int kStage = kThere + 128;
  // CTAs of an SM: as many as registers and the rings' 220 KB allow.  A MixFP4 cache of 128 dimensions would hold
  // four with 128 registers each, but three with 168 keep V's codes in registers beside K's: 129 against 145 us.
  // Three stages, or the two that fit (a bf16 cache of 128 dimensions and up to 16 query heads): six with three CTAs 129
  // against 126 us on a MixFP4 cache.
  static constexpr int kCtas = DT == 256 ? (kFp4 ? 2 : 1) : (NT == 3 ? 2 : (NT == 1 && !kFp4 && DT == 64 ? 4 : 3));
  static constexpr int kDepth = 3;
  static constexpr int kFit = 220 * 1024 / kCtas / (kWarps * kStage);
  static constexpr int kStages = kFit < kDepth ? kFit : kDepth;
  static constexpr int kRing = kWarps * kStages * kStage;
  static constexpr int kMerge = (kWarps + 1) * kHeads * (DT + 4) * 4;  // the warps' results, and in a cluster the CTA's
  static constexpr int kSmem = kRing > kMerge ? kRing : kMerge;
};

template <int kBytes>
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src, bool take) {
  const int n = take ? kBytes : 0;
  if constexpr (kBytes == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(kBytes), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int n>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(n) : "memory"); }

__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds8(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void sts32(uint32_t a, uint32_t v) {
  asm volatile("st.shared.b32 [%0], %1;" ::"r"(a), "r"(v) : "memory");
}
__device__ __forceinline__ void sts8(uint32_t a, uint32_t v) {
  asm volatile("st.shared.u8 [%0], %1;" ::"r"(a), "r"(v) : "memory");
}

template <bool kF16>
__device__ __forceinline__ void mma16816(float d[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  if constexpr (kF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The transpose of an 8 x 8 matrix of 16-bit elements, thread (g, t) = (lane / 4, lane % 4) holding row g, columns 2t, 2t + 1.
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
  return d;
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
__device__ __forceinline__ uint32_t f16x2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
// 2^x, results below 2^-126 as zero.
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The factor (f16x2) and the payload tables of a block's scale byte.
struct BlockScale {
  uint32_t s2, lo, hi;
};
__device__ __forceinline__ BlockScale block_scale(uint32_t sc) {
  const uint32_t e1m2 = sc >> 7;  // tables by multiplication: the integer pipe is the one that decoding fills
  return BlockScale{cvt_f16x2_from_e4m3x2((uint16_t)((sc & 0x7Fu) * 0x0101u)),
                    kLutE2M1Lo + e1m2 * (kLutE1M2Lo - kLutE2M1Lo), kLutE2M1Hi + e1m2 * (kLutE1M2Hi - kLutE2M1Hi)};
}
__device__ __forceinline__ float bf_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.aligned;\n barrier.cluster.wait.aligned;" ::: "memory");
}
// Two floats of CTA `rank`'s shared memory, at the address they have in this one's (after a cluster barrier).
__device__ __forceinline__ float2 peer_load(const float* p, uint32_t rank) {
  float2 v;
  asm volatile("{ .reg .b32 r; mapa.shared::cluster.u32 r, %2, %3; ld.shared::cluster.v2.f32 {%0, %1}, [r]; }"
               : "=f"(v.x), "=f"(v.y)
               : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank)
               : "memory");
  return v;
}

// Tokens [first, end) of sequence b that are seen.
__device__ __forceinline__ int2 seen(const AttnArgs& p, int b) {
  int64_t n = p.lengths[b];
  n = n < p.max_tokens ? n : p.max_tokens;
  n = n > 0 ? n : 0;
  const int64_t lo = p.window > 0 && n > p.window ? n - p.window : 0;
  return make_int2((int)lo, (int)n);
}
// Units of work of a row of the sequence: kRowCost for its beginning, then one to 64 head rows.
__device__ __forceinline__ int units(const AttnArgs& p, int2 r) {
  const int n = kUnit / p.together;
  return r.y > r.x ? kRowCost + (r.y - (r.x & ~15) + n - 1) / n : 0;
}

// A finished row's factor of O, and its log-sum-exp, of m and l.  l is 0 only where no token was seen (or all scores
// are -inf); NaN goes through, and so does the +inf of a score of +inf.
template <bool kFp4>
__device__ __forceinline__ float out_factor(float l, float vts) {
  return l == 0.0f ? 0.0f : (kFp4 ? 0.5f * vts : 1.0f) / l;
}
template <bool kFp4>
__device__ __forceinline__ float lse_of(float m, float l) {
  return l == 0.0f ? -INFINITY : (m + log2f(l) - (kFp4 ? kFp4Exp : 0.0f)) * kLn2;
}

// One output element pair of a finished row.
__device__ __forceinline__ void store_out(const AttnArgs& p, int b, int h, int d, float x, float y) {
  *reinterpret_cast<uint32_t*>(p.out + ((int64_t)b * p.q_heads + h) * p.c.head_dim + d) = bf16x2(x, y);
}

// Sequence b's results where it sees no token.
__device__ __forceinline__ void nothing_seen(const AttnArgs& p, int b, int tid) {
  const int64_t words = (int64_t)p.q_heads * p.c.head_dim / 2;
  for (int64_t i = tid; i < words; i += kThreads) reinterpret_cast<uint32_t*>(p.out)[b * words + i] = 0u;
  if (p.lse)
    for (int h = tid; h < p.q_heads; h += kThreads) p.lse[(int64_t)b * p.q_heads + h] = -INFINITY;
}

template <int DT, int NT, bool kFp4>
__global__ void __launch_bounds__(kThreads, Cfg<DT, NT, kFp4>::kCtas) paged_attention_kernel(const AttnArgs p) {
  using C = Cfg<DT, NT, kFp4>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int sh_b;
  __shared__ int64_t sh_before, sh_edge[2], sh_scan[kWarps];
  griddep_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int D = p.c.head_dim;
  const int rows = p.c.heads / p.together * p.chunks;  // rows of work of a sequence
  const int mate = warp % p.together, phase = warp / p.together, phases = kWarps / p.together;

  // This CTA's share [pos, end) of all units, and the sequence it starts in.
  int b = 0;
  int64_t pos = 0, end = 1, base = 0, all = 0, grid = 0;
  if (p.cluster) {
    b = (int)(blockIdx.x >> p.cluster_shift) / rows;
    const int2 r = seen(p, b);
    if (r.y <= r.x) {  // the row sees nothing
      if (blockIdx.x % (p.cluster * rows) == 0) nothing_seen(p, b, tid);
      return;
    }
  } else {
    const int strip = (p.B + kThreads - 1) / kThreads;
    int64_t mine = 0;
    for (int i = tid * strip; i < min(p.B, (tid + 1) * strip); ++i) mine += units(p, seen(p, i));
    int64_t before = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t v = __shfl_up_sync(kAll, before, d);
      if (lane >= d) before += v;
    }
    if (lane == 31) sh_scan[warp] = before;
    if (tid == 0) sh_b = p.B;
    __syncthreads();
    int64_t total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) before += sh_scan[w];
      total += sh_scan[w];
    }
    before -= mine;
    all = total * rows;
    grid = all < (int64_t)gridDim.x ? all : (int64_t)gridDim.x;  // CTAs with a share
    for (int i = blockIdx.x; i < p.B; i += gridDim.x) {  // sequences that see nothing
      const int2 r = seen(p, i);
      if (r.y > r.x) continue;
      if (p.by_row)
        for (int k = tid; k < rows; k += kThreads) p.split[(int64_t)i * rows + k] = make_int4(-1, 0, 0, 0);
      nothing_seen(p, i, tid);
    }
    if (tid == 0 && !p.by_row) p.split[blockIdx.x] = make_int4(-1, 0, 0, 0);
    if ((int64_t)blockIdx.x >= grid) return;
    // An edge between shares that falls into a row's beginning lies before the row.
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int64_t edge = all * (blockIdx.x + k) / grid;
      if (edge >= before * rows && edge < (before + mine) * rows) {
        int i = tid * strip;
        int64_t at = before;
        int u = units(p, seen(p, i));
        for (const int to = min(p.B, i + strip) - 1; i < to && edge >= (at + u) * rows;) {
          at += u;
          u = units(p, seen(p, ++i));
        }
        const int64_t into = u > 0 ? (edge - at * rows) % u : 0;
        sh_edge[k] = into <= kRowCost ? edge - into : edge;
        if (k == 0) sh_b = i, sh_before = at;
      } else if (edge == all && tid == 0) {
        sh_edge[k] = all;
      }
    }
    __syncthreads();
    pos = sh_edge[0];
    end = sh_edge[1];
    b = sh_b;
    base = sh_before * rows;  // first unit of sequence b
  }

  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * C::kStages * C::kStage;
  // Reached in equal shares only: no cluster's or single CTA's part of a row has as many tiles.
  static_assert(kChain * 16 * kWarps > 4 * kCtaTokens + 2 * kUnit && kChain * 16 > kRowTokens + 16);
  auto aside = [&](int n) {  // of query heads 8n ..: the sum of O, m and l, the latest chain's O
    const int64_t w = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    return p.aside + (w * NT + n) * (C::kAside * 32) + (threadIdx.x & 31);
  };
  const float kts = kFp4 ? *p.c.k_ts : 1.0f, vts = kFp4 ? *p.c.v_ts : 1.0f;

  while (pos < end && b < p.B) {
    const int2 range = seen(p, b);
    const int u = units(p, range);
    if (!p.cluster && (u == 0 || pos >= base + (int64_t)u * rows)) {  // the next sequence (this one may have no unit)
      base += (int64_t)u * rows;
      ++b;
      continue;
    }
    int row, k0, cnt;  // row of the sequence, first unit and units of it
    if (p.cluster) {
      const int rank = (int)(blockIdx.x & (p.cluster - 1)), tu = u - kRowCost;
      row = (int)(blockIdx.x >> p.cluster_shift) % rows;
      k0 = rank > 0 ? kRowCost + (int)((int64_t)tu * rank >> p.cluster_shift) : 0;
      cnt = kRowCost + (int)((int64_t)tu * (rank + 1) >> p.cluster_shift) - k0;
    } else {
      row = (int)((pos - base) / u);
      k0 = (int)((pos - base) - (int64_t)row * u);
      cnt = (int)min((int64_t)(u - k0), end - pos);
    }
    const int chunk = row % p.chunks, head = row / p.chunks * p.together + mate;
    const int h0 = head * p.group + chunk * C::kHeads;
    const int nh = min(C::kHeads, p.group - chunk * C::kHeads);  // query heads of this row
    const int n = kUnit / p.together, from = max(k0 - kRowCost, 0), to = max(k0 + cnt - kRowCost, 0);
    const int tok0 = (range.x & ~15) + from * n, tok1 = min(range.y, (range.x & ~15) + to * n);

    // ---- the queries: B fragments, thread (g, t) holding head g's dimensions of its K pieces
    uint32_t qf[NT][DT / 16][2];
    float fs[NT][2];  // factor of the scores of heads 2t, 2t + 1 (of the 8 NT)
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int h = 8 * n + g;
      const uint16_t* q = p.q + (int64_t)b * p.q_stride + (int64_t)(h0 + h) * p.q_head_stride;
      float top = 0.0f;
#pragma unroll
      for (int i = 0; i < C::kKPieces; ++i) {
        const int d = (t + 4 * i) * C::kKDims;
#pragma unroll
        for (int s = 0; s < C::kKDims / 8; ++s) {
          uint4 w = make_uint4(0, 0, 0, 0);
          if (h < nh && d < D) w = *reinterpret_cast<const uint4*>(q + d + 8 * s);
          const int st = (i * C::kKDims / 8 + s) * 2;
          qf[n][st][0] = w.x, qf[n][st][1] = w.y, qf[n][st + 1][0] = w.z, qf[n][st + 1][1] = w.w;
          if (kFp4) {
            const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) top = max3f(top, fabsf(bf_lo(v[j])), fabsf(bf_hi(v[j])));
          }
        }
      }
      float back = 1.0f;
      if (kFp4) {  // q times 2^(14 - exponent of the head's largest) as f16
        top = fmaxf(top, __shfl_xor_sync(kAll, top, 1));
        top = fmaxf(top, __shfl_xor_sync(kAll, top, 2));
        int e = (int)(__float_as_uint(top) >> 23);
        e = min(max(e, 15), 253);
        const float up = __uint_as_float((uint32_t)(268 - e) << 23);
        back = __uint_as_float((uint32_t)(e - 14) << 23);
#pragma unroll
        for (int s = 0; s < DT / 16; ++s)
#pragma unroll
          for (int j = 0; j < 2; ++j) qf[n][s][j] = f16x2(bf_lo(qf[n][s][j]) * up, bf_hi(qf[n][s][j]) * up);
      }
      const float f = p.scale * kLog2e * (kFp4 ? 0.5f * kts : 1.0f);  // the decoded rows are twice the values
#pragma unroll
      for (int j = 0; j < 2; ++j) fs[n][j] = f * (kFp4 ? __shfl_sync(kAll, back, (2 * t + j) * 4) : 1.0f);
    }

    // ---- the ring: this warp's tiles are 16 tokens at tok0 + 16 (phase + phases i)
    const int tiles_all = (tok1 - tok0 + 15) / 16;
    const int tiles = tiles_all > phase ? (tiles_all - phase + phases - 1) / phases : 0;
    const int32_t* table = p.table + (int64_t)b * p.table_stride;
    const uint8_t* kb = static_cast<const uint8_t*>(p.c.k) + (int64_t)head * p.c.head_stride * (kFp4 ? 1 : 2);
    const uint8_t* vb = static_cast<const uint8_t*>(p.c.v) + (int64_t)head * p.c.head_stride * (kFp4 ? 1 : 2);
    const uint8_t* sb = nullptr;
    if (kFp4) sb = (lane < 16 ? p.c.k_scales : p.c.v_scales) + (int64_t)head * p.c.scale_head_stride;

    // Where tiles lie in one page each (page_size % 16 == 0), its number is asked for a tile ahead and a
    // row is token_stride behind the one before; else every row's page is looked up.
    const bool whole = (p.c.page_size & 15) == 0;
    const int64_t esize = kFp4 ? 1 : 2, step = p.c.token_stride * esize;
    auto page_of = [&](int tok) { return p.page_shift >= 0 ? tok >> p.page_shift : tok / p.c.page_size; };
    auto ask = [&](int i) -> int {
      const int tok = tok0 + 16 * (phase + phases * i);
      return whole && i < tiles ? table[page_of(tok)] : -1;
    };
    int asked = ask(0);
    // Asks for tile i.
    auto issue = [&](int i, uint32_t dst) {
      const int tok = tok0 + 16 * (phase + phases * i);
      uint32_t there = (tok1 - tok >= 16 ? 0xFFFFu : (1u << (tok1 - tok)) - 1u);
      if (tok < range.x) there &= 0xFFFFu << (range.x - tok);
      int64_t at = 0, sat = 0;  // of the tile, or of lane l's token l % 16
      if (whole) {
        const int page = asked, off = tok - page_of(tok) * p.c.page_size;
        asked = ask(i + 1);
        if (page < 0 || page >= p.c.pages) there = 0;
        if (there) {
          at = ((int64_t)page * p.c.page_stride + (int64_t)off * p.c.token_stride) * esize;
          sat = (int64_t)page * p.c.scale_page_stride + (int64_t)(off + (lane & 15)) * p.c.scale_token_stride;
        }
      } else {
        const int tk = tok + (lane & 15);
        int page = -1;
        if ((there >> (lane & 15)) & 1u) page = table[page_of(tk)];
        const bool ok = page >= 0 && page < p.c.pages;
        there = __ballot_sync(kAll, ok) & 0xFFFFu;
        if (ok) {
          const int off = tk - page_of(tk) * p.c.page_size;
          at = ((int64_t)page * p.c.page_stride + (int64_t)off * p.c.token_stride) * esize;
          sat = (int64_t)page * p.c.scale_page_stride + (int64_t)off * p.c.scale_token_stride;
        }
      }
      const int r0 = lane / C::kPieces, piece = lane % C::kPieces;
      const bool in_row = piece * (kFp4 ? 16 : 8) < D;
      const int64_t lane_at = r0 * step + piece * C::kCopy;
      if (whole && there == 0xFFFFu) {  // as most tiles are
        const uint8_t *ks = kb + (at + lane_at), *vs = vb + (at + lane_at);
#pragma unroll
        for (int j = 0; j < 16 / C::kRowsAtOnce; ++j) {
          const int r = r0 + j * C::kRowsAtOnce;
          cp_async<C::kCopy>(dst + C::k_place(r, piece), ks, in_row);
          cp_async<C::kCopy>(dst + C::kKTile + C::v_place(r, piece), vs, in_row);
          ks += C::kRowsAtOnce * step;
          vs += C::kRowsAtOnce * step;
        }
      } else {
#pragma unroll 1
        for (int j = 0; j < 16 / C::kRowsAtOnce; ++j) {
        const int r = r0 + j * C::kRowsAtOnce;
        const bool take = ((there >> r) & 1u) && in_row;
        const int64_t from = whole ? at + lane_at + j * C::kRowsAtOnce * step
                                   : __shfl_sync(kAll, at, r) + piece * C::kCopy;
        cp_async<C::kCopy>(dst + C::k_place(r, piece), kb + from, take);
        cp_async<C::kCopy>(dst + C::kKTile + C::v_place(r, piece), vb + from, take);
        }
      }
      if (kFp4) {
        const bool ok = (there >> (lane & 15)) & 1u;
        const uint8_t* src = sb + sat;
        const uint32_t sd = dst + C::kKTile + C::kVTile + lane * 16;
        if (D == 128) {
          cp_async<8>(sd, src, ok);
        } else if (D == 256) {
          cp_async<16>(sd, src, ok);
        } else if (D % 64 == 0) {
          for (int k = 0; k < D / 16; k += 4) cp_async<4>(sd + k, src + k, ok);
        } else {  // rows of an odd number of scale bytes
          for (int k = 0; k < D / 16; ++k) sts8(sd + k, ok ? src[k] : 0u);
        }
      }
      if (lane == 0) sts32(dst + C::kThere, there);
    };

    if constexpr (kFp4) {
      if (D < DT)  // scale bytes behind D are read too, and stay as they are from here on
        for (int i = lane; i < C::kStages * C::kScaleTile / 4; i += 32)
          sts32(ring + i / (C::kScaleTile / 4) * C::kStage + C::kKTile + C::kVTile + i % (C::kScaleTile / 4) * 4, 0u);
    }
    __syncwarp();
#pragma unroll 1
    for (int i = 0; i < C::kStages - 1; ++i) {
      if (i < tiles) issue(i, ring + i * C::kStage);
      cp_commit();
    }
    uint32_t put = ring + (C::kStages - 1) * C::kStage, src = ring;  // the stages to fill and to use next
    const uint32_t behind = ring + C::kStages * C::kStage;

    float o[NT][DT / 16][4];
    float m[NT][2], l[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      m[n][0] = m[n][1] = kNoScore;
      l[n][0] = l[n][1] = 0.0f;
#pragma unroll
      for (int i = 0; i < DT / 16; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.0f;
    }

    // A chain's end: O and l are put into memory and begin at 0; there, in fp32 and by few registers, they join the sums
    // of the chains before.
    auto set_aside = [&](bool more) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < DT / 16; ++k) {
          float* a = o[n][k];
          aside(n)[((more ? DT / 16 + 1 : 0) + k) * 32] = make_float4(a[0], a[1], a[2], a[3]);
          a[0] = a[1] = a[2] = a[3] = 0.0f;
        }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float4* sum = aside(n);
        const float4* last = sum + (DT / 16 + 1) * 32;
        float l0 = l[n][0], l1 = l[n][1];
        l[n][0] = l[n][1] = 0.0f;
        if (more) {
          const float4 then = sum[DT / 16 * 32];
          const float f0 = ex2(then.x - m[n][0]), f1 = ex2(then.y - m[n][1]);
          l0 = fmaf(f0, then.z, l0), l1 = fmaf(f1, then.w, l1);
#pragma unroll 1
          for (int k = 0; k < DT / 16; ++k) {
            const float4 v = sum[k * 32], w = last[k * 32];
            sum[k * 32] = make_float4(fmaf(f0, v.x, w.x), fmaf(f1, v.y, w.y), fmaf(f0, v.z, w.z), fmaf(f1, v.w, w.w));
          }
        }
        sum[DT / 16 * 32] = make_float4(m[n][0], m[n][1], l0, l1);
      }
    };
    int stop = min(tiles, kChain);  // of this chain's tiles
    for (int i = 0; i < tiles;) {
#pragma unroll 1
      for (; i < stop; ++i) {
        __syncwarp();  // the stage about to be filled again has been read by every lane
        if (i + C::kStages - 1 < tiles) issue(i + C::kStages - 1, put);
        cp_commit();
        cp_wait<C::kStages - 1>();
        __syncwarp();
        const uint32_t vs = src + C::kKTile;
        const uint32_t ss = src + C::kKTile + C::kVTile;

        const uint32_t there = lds32(src + C::kThere);
        const bool ok0 = (there >> g) & 1u, ok1 = (there >> (g + 8)) & 1u;
        // A MixFP4 tile's V codes and scale bytes, asked for before the scores so that neither waits for the other.
        uint2 vc[kFp4 ? C::kVPieces : 1][4];
        uint32_t vsc[kFp4 ? C::kVPieces : 1][4];
        if constexpr (kFp4) {
#pragma unroll
          for (int k = 0; k < C::kVPieces; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int tr = 2 * t + (r & 1) + 8 * (r >> 1);
              vsc[k][r] = lds8(ss + (16 + tr) * 16 + (g + 8 * k) * C::kVDims / 16);
              if constexpr (C::kVBytes == 8)
                vc[k][r] = lds64(vs + C::v_place(tr, g + 8 * k));
              else
                vc[k][r].x = lds32(vs + C::v_place(tr, (g + 8 * k) / 2) + (g & 1) * C::kVBytes);
            }
        }

        // ---- scores of 16 tokens x 8 NT heads, in two chains of products
        float s[NT][4], s1[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[n][e] = s1[n][e] = 0.0f;
#pragma unroll
        for (int k = 0; k < C::kKPieces; ++k) {
          uint32_t w[2][C::kKDims / 2];  // rows g and g + 8
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const uint32_t a = src + C::k_place(g, t + 4 * k) + 8 * r * C::kRow;
            if constexpr (kFp4) {
              const uint2 v = lds64(a);
              const BlockScale f = block_scale(lds8(ss + (g + 8 * r) * 16 + t + 4 * k));
              decode8(v.x, f.lo, f.hi, f.s2, w[r]);
              decode8(v.y, f.lo, f.hi, f.s2, w[r] + 4);
            } else {
              const uint4 v = lds128(a);
              w[r][0] = v.x, w[r][1] = v.y, w[r][2] = v.z, w[r][3] = v.w;
            }
          }
#pragma unroll
          for (int st = 0; st < C::kKDims / 4; ++st)
#pragma unroll
            for (int n = 0; n < NT; ++n)
              mma16816<kFp4>(st & 1 ? s1[n] : s[n], w[0][2 * st], w[1][2 * st], w[0][2 * st + 1], w[1][2 * st + 1],
                             qf[n][k * C::kKDims / 4 + st][0], qf[n][k * C::kKDims / 4 + st][1]);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[n][e] += s1[n][e];

        // ---- softmax: thread (g, t) has tokens g, g + 8 and heads 2t, 2t + 1.  The weights are 2^(s - m) for
        // an m that follows the maximum from afar: it moves (and what was summed is scaled) when a score is
        // kSlack above it, which takes a vote a tile instead of a maximum over the lanes.
        uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          bool far = false;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            s[n][j] = ok0 ? s[n][j] * fs[n][j] : -INFINITY;
            s[n][2 + j] = ok1 ? s[n][2 + j] * fs[n][j] : -INFINITY;
            far = far || fmaxf(s[n][j], s[n][2 + j]) > m[n][j] + kSlack;
          }
          if (__any_sync(kAll, far)) {
            float cor[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float v = fmaxf(s[n][j], s[n][2 + j]);
              v = fmaxf(v, __shfl_xor_sync(kAll, v, 4));
              v = fmaxf(v, __shfl_xor_sync(kAll, v, 8));
              v = fmaxf(v, __shfl_xor_sync(kAll, v, 16));
              v = fminf(fmaxf(m[n][j], v), kMostScore);
              cor[j] = ex2(m[n][j] - v);  // 0 at the first score
              m[n][j] = v;
              l[n][j] *= cor[j];
            }
#pragma unroll
            for (int k = 0; k < DT / 16; ++k) {
              o[n][k][0] *= cor[0], o[n][k][1] *= cor[1], o[n][k][2] *= cor[0], o[n][k][3] *= cor[1];
            }
          }
          float w[4];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float top = m[n][j] - (kFp4 ? kFp4Exp : 0.0f);
            w[j] = ex2(s[n][j] - top);
            w[2 + j] = ex2(s[n][2 + j] - top);
            l[n][j] += w[j] + w[2 + j];
          }
          if (kFp4) {
            ph[n][0] = transpose8(f16x2(w[0], w[1]));
            ph[n][1] = transpose8(f16x2(w[2], w[3]));
          } else {
            // The upper part by truncation, so that the lower is not negative, and not 0 either where the weight is not
            // (2^-126 then): times an infinite element of V both give its infinity.
            float low[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) low[e] = fmaxf(w[e] - bf_hi(__float_as_uint(w[e])), fminf(w[e], 0x1p-126f));
            ph[n][0] = transpose8(prmt(__float_as_uint(w[0]), __float_as_uint(w[1]), 0x7632u));
            ph[n][1] = transpose8(prmt(__float_as_uint(w[2]), __float_as_uint(w[3]), 0x7632u));
            pl[n][0] = transpose8(bf16x2(low[0], low[1]));
            pl[n][1] = transpose8(bf16x2(low[2], low[3]));
          }
        }

        // ---- O^T += V^T P^T: rows g and g + 8 of product (k, j) are dimensions 2j, 2j + 1 of the thread's piece k
#pragma unroll
        for (int k = 0; k < C::kVPieces; ++k) {
          uint32_t w[4][C::kVDims / 2];  // tokens 2t, 2t + 1, 2t + 8, 2t + 9
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            if constexpr (kFp4) {
              const BlockScale f = block_scale(vsc[k][r]);
              decode8(vc[k][r].x, f.lo, f.hi, f.s2, w[r]);
              if constexpr (C::kVBytes == 8) decode8(vc[k][r].y, f.lo, f.hi, f.s2, w[r] + 4);
            } else {
              const uint4 v = lds128(vs + C::v_place(2 * t + (r & 1) + 8 * (r >> 1), g + 8 * k));
              w[r][0] = v.x, w[r][1] = v.y, w[r][2] = v.z, w[r][3] = v.w;
            }
          }
#pragma unroll
          for (int j = 0; j < C::kVDims / 2; ++j) {
            const uint32_t a0 = prmt(w[0][j], w[1][j], 0x5410u), a1 = prmt(w[0][j], w[1][j], 0x7632u);
            const uint32_t a2 = prmt(w[2][j], w[3][j], 0x5410u), a3 = prmt(w[2][j], w[3][j], 0x7632u);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              float* acc = o[n][k * C::kVDims / 2 + j];
              mma16816<kFp4>(acc, a0, a1, a2, a3, ph[n][0], ph[n][1]);
              if (!kFp4) mma16816<kFp4>(acc, a0, a1, a2, a3, pl[n][0], pl[n][1]);
            }
          }
        }
        put = src;
        src = src + C::kStage == behind ? ring : src + C::kStage;
      }
      if (stop < tiles) set_aside(stop > kChain);
      stop = min(tiles, stop + kChain);
    }
    cp_wait<0>();
    if (tiles > kChain) {
      set_aside(true);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int k = 0; k < DT / 16; ++k) {
          const float4 v = aside(n)[k * 32];
          o[n][k][0] = v.x, o[n][k][1] = v.y, o[n][k][2] = v.z, o[n][k][3] = v.w;
        }
        const float4 v = aside(n)[DT / 16 * 32];
        l[n][0] = v.z, l[n][1] = v.w;
      }
    }

    // ---- the warps' results joined in shared memory (the ring is drained)
    __syncthreads();
    float* mo = reinterpret_cast<float*>(smem);                              // [warp][head][DT]
    float* ms = mo + kWarps * C::kHeads * DT;                                // [warp][head] m, then l
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float v = l[n][j];
        v += __shfl_xor_sync(kAll, v, 4);
        v += __shfl_xor_sync(kAll, v, 8);
        v += __shfl_xor_sync(kAll, v, 16);
        const int h = 8 * n + 2 * t + j;
        if (g == 0) {
          ms[(warp * C::kHeads + h) * 2] = m[n][j];
          ms[(warp * C::kHeads + h) * 2 + 1] = v;
        }
        float* to = mo + (warp * C::kHeads + h) * DT;
#pragma unroll
        for (int k = 0; k < C::kVPieces; ++k)
#pragma unroll
          for (int i = 0; i < C::kVDims / 2; ++i) {
            const int d = (g + 8 * k) * C::kVDims + 2 * i;
            const float* acc = o[n][k * C::kVDims / 2 + i];
            *reinterpret_cast<float2*>(to + d) = make_float2(acc[j], acc[2 + j]);
          }
      }
    }
    __syncthreads();
    float* js = ms + kWarps * C::kHeads * 2;                                 // [head] m, l of a cluster's CTA
    float* jo = js + C::kHeads * 2;                                          // [head][DT]
    const bool first = k0 == 0, last = k0 + cnt == u;
    const int64_t slot = (2 * (int64_t)blockIdx.x + (first ? 1 : 0)) * p.together;
    for (int i = tid; i < p.together * nh * (DT / 2); i += kThreads) {
      const int hh = i / (DT / 2), d = (i - hh * (DT / 2)) * 2;
      const int w0 = hh / nh, h = hh - w0 * nh;  // key head of the CTA, query head of it
      const int ho = (row / p.chunks * p.together + w0) * p.group + chunk * C::kHeads + h;
      float M = kNoScore, L = 0.0f;
      for (int w = w0; w < kWarps; w += p.together) M = fmaxf(M, ms[(w * C::kHeads + h) * 2]);
      float x = 0.0f, y = 0.0f;
      for (int w = w0; w < kWarps; w += p.together) {
        const float f = exp2f(ms[(w * C::kHeads + h) * 2] - M);
        const float2 v = *reinterpret_cast<const float2*>(mo + (w * C::kHeads + h) * DT + d);
        L += f * ms[(w * C::kHeads + h) * 2 + 1];
        x += f * v.x;
        y += f * v.y;
      }
      if (p.cluster > 1) {
        *reinterpret_cast<float2*>(jo + h * DT + d) = make_float2(x, y);
        if (d == 0) *reinterpret_cast<float2*>(js + 2 * h) = make_float2(M, L);
      } else if (first && last) {
        const float f = out_factor<kFp4>(L, vts);
        if (d < D) store_out(p, b, ho, d, x * f, y * f);
        if (d == 0 && p.lse) p.lse[(int64_t)b * p.q_heads + ho] = lse_of<kFp4>(M, L);
      } else {
        *reinterpret_cast<float2*>(p.part + ((slot + w0) * C::kHeads + h) * DT + d) = make_float2(x, y);
        if (d == 0) p.stat[(slot + w0) * C::kHeads + h] = make_float2(M, L);
      }
    }
    if (p.cluster == 1) return;
    if (p.cluster > 1) {  // each CTA joins its share of the row's outputs
      cluster_barrier();
      for (int i = (int)cluster_rank() * kThreads + tid; i < nh * (DT / 2); i += p.cluster * kThreads) {
        const int h = i / (DT / 2), d = (i - h * (DT / 2)) * 2;
        float2 st[kCluster], v[kCluster];
        float M = kNoScore, L = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll
        for (int q = 0; q < kCluster; ++q) {  // of fewer CTAs some twice, the second time for nothing
          const int rank = q & (p.cluster - 1);
          st[q] = peer_load(js + 2 * h, rank), v[q] = peer_load(jo + h * DT + d, rank);
          if (q >= p.cluster) st[q] = make_float2(kNoScore, 0.0f), v[q] = make_float2(0.0f, 0.0f);
        }
#pragma unroll
        for (int q = 0; q < kCluster; ++q) M = fmaxf(M, st[q].x);
#pragma unroll
        for (int q = 0; q < kCluster; ++q) {
          const float f = exp2f(st[q].x - M);
          L += f * st[q].y;
          x += f * v[q].x;
          y += f * v[q].y;
        }
        const float f = out_factor<kFp4>(L, vts);
        if (d < D) store_out(p, b, h0 + h, d, x * f, y * f);
        if (d == 0 && p.lse) p.lse[(int64_t)b * p.q_heads + h0 + h] = lse_of<kFp4>(M, L);
      }
      cluster_barrier();  // no CTA leaves while others read its results
      return;
    }
    if (tid == 0 && first && (p.by_row || !last)) {
      const int64_t x = base + (int64_t)(row + 1) * u;  // behind the row's last unit
      p.split[p.by_row ? (int64_t)b * rows + row : (int64_t)blockIdx.x] =
          last ? make_int4(-1, 0, 0, 0) : make_int4(b, row, (int)blockIdx.x, (int)((x * grid - 1) / all));
    }
    __syncthreads();
    pos += cnt;
  }
}

// Joins the parts of the row in place blockIdx.x of `split`, key head
// blockIdx.y of it, the query heads of blockIdx.z; `share` warps take one query
// head, in turn over its parts.
template <int DT, int NT, bool kFp4>
__global__ void __launch_bounds__(kJoinThreads) paged_attention_join_kernel(const AttnArgs p) {
  constexpr int kHeads = 8 * NT, kV = DT / 64, kW = kJoinThreads / 32;
  __shared__ float2 red[kW][DT / 2 + 1];
  griddep_wait();
  const int4 s = p.split[blockIdx.x];
  if (s.x < 0) return;
  const int chunk = s.y % p.chunks, mate = blockIdx.y;
  const int nh = min(kHeads, p.group - chunk * kHeads);
  const int h0 = (s.y / p.chunks * p.together + mate) * p.group + chunk * kHeads;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int share = p.share, parts = s.w - s.z + 1;
  const int h = blockIdx.z * (kW / share) + warp / share, ph = warp % share;
  auto slot = [&](int i) { return ((2 * ((int64_t)s.z + i) + (i == 0 ? 1 : 0)) * p.together + mate) * kHeads + h; };
  float2 acc[kV];  // dimensions 2 lane + 64 j and the next
  float M = kNoScore, L = 0.0f;
#pragma unroll
  for (int j = 0; j < kV; ++j) acc[j] = make_float2(0.0f, 0.0f);
  if (h < nh) {
    constexpr int kAtOnce = 4;  // parts asked for at once, with their (m, l)
    for (int i0 = ph; i0 < parts; i0 += kAtOnce * share) {
      float2 st[kAtOnce], v[kAtOnce][kV];
#pragma unroll
      for (int a = 0; a < kAtOnce; ++a) {
        const int i = i0 + a * share;
        st[a] = make_float2(kNoScore, 0.0f);
#pragma unroll
        for (int j = 0; j < kV; ++j) v[a][j] = make_float2(0.0f, 0.0f);
        if (i < parts) {
          st[a] = p.stat[slot(i)];
          const float2* o = reinterpret_cast<const float2*>(p.part + slot(i) * DT) + lane;
#pragma unroll
          for (int j = 0; j < kV; ++j) v[a][j] = o[32 * j];
        }
      }
      float top = M;
#pragma unroll
      for (int a = 0; a < kAtOnce; ++a) top = fmaxf(top, st[a].x);
      const float old = exp2f(M - top);
      M = top;
      L *= old;
#pragma unroll
      for (int j = 0; j < kV; ++j) acc[j].x *= old, acc[j].y *= old;
#pragma unroll
      for (int a = 0; a < kAtOnce; ++a) {
        const float f = exp2f(st[a].x - M);
        L += f * st[a].y;
#pragma unroll
        for (int j = 0; j < kV; ++j) acc[j].x += f * v[a][j].x, acc[j].y += f * v[a][j].y;
      }
    }
  }
  if (share > 1) {  // the first of a head's warps adds the others' sums
#pragma unroll
    for (int j = 0; j < kV; ++j) red[warp][lane + 32 * j] = acc[j];
    if (lane == 0) red[warp][DT / 2] = make_float2(M, L);
    __syncthreads();
    if (ph != 0) return;
    float top = M;
    for (int w = 1; w < share; ++w) top = fmaxf(top, red[warp + w][DT / 2].x);
    const float old = exp2f(M - top);
    L *= old;
#pragma unroll
    for (int j = 0; j < kV; ++j) acc[j].x *= old, acc[j].y *= old;
    for (int w = 1; w < share; ++w) {
      const float2 st = red[warp + w][DT / 2];
      const float f = exp2f(st.x - top);
      L += f * st.y;
#pragma unroll
      for (int j = 0; j < kV; ++j) {
        const float2 v = red[warp + w][lane + 32 * j];
        acc[j].x += f * v.x, acc[j].y += f * v.y;
      }
    }
    M = top;
  }
  if (h >= nh) return;
  const float f = out_factor<kFp4>(L, kFp4 ? *p.c.v_ts : 1.0f);
#pragma unroll
  for (int j = 0; j < kV; ++j) {
    const int d = 2 * lane + 64 * j;
    if (d < p.c.head_dim) store_out(p, s.x, h0 + h, d, acc[j].x * f, acc[j].y * f);
  }
  if (lane == 0 && p.lse) p.lse[(int64_t)s.x * p.q_heads + h0 + h] = lse_of<kFp4>(M, L);
}

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline int launch_status() { return cudaGetLastError() == cudaSuccess ? MIXFP4_OK : MIXFP4_ERR_CUDA; }

inline int padded_dim(int D) { return D <= 64 ? 64 : (D <= 128 ? 128 : 256); }
// Query heads of a row: 24 hold registers for rows of up to 128 dimensions only, and pay where 16 would read the
// cache twice (24 heads to a key head).
inline int padded_heads(const mixfp4_kv_cache* c, int64_t q_heads) {
  const int64_t group = q_heads / c->heads;
  return group <= 8 ? 8 : (group <= 16 || c->head_dim > 128 || (group + 15) / 16 == (group + 23) / 24 ? 16 : 24);
}
// What a CTA of the first kernel may set aside.
inline int64_t aside_bytes(const mixfp4_kv_cache* c, int64_t q_heads) {
  return (int64_t)kWarps * (padded_heads(c, q_heads) / 8) * (padded_dim(c->head_dim) / 16 * 2 + 1) * 32 * 16;
}
// Key heads of a CTA.  Where the heads of a token lie together, neighbouring heads' rows are asked for at the same
// time (64 sequences of up to 8192 tokens, 8 heads of 128: MixFP4 162 us against 185 us with one head to a CTA, whose
// 8 scale bytes of a row cost a whole access; 32 bf16 heads of 128: 91 against 111 us).  Where a head's tokens lie
// together that gains nothing, and with few rows one head to a CTA leaves fewer parts of each to join (2 sequences of
// 131072: 175 us against 188).
inline int together_of(const mixfp4_kv_cache* c, int64_t B, int64_t chunks, int grid) {
  if (c->head_stride >= c->token_stride) return 1;
  for (int n = 4; n > 1; n /= 2)
    if (c->heads % n == 0 && B * (c->heads / n) * chunks >= grid / 4) return n;
  return 1;
}
// CTAs of the first kernel.
template <int DT, bool kFp4>
int ctas_of(int heads) {
  if constexpr (DT <= 128)
    if (heads == 24) return Cfg<DT, 3, kFp4>::kCtas;
  return heads == 8 ? Cfg<DT, 1, kFp4>::kCtas : Cfg<DT, 2, kFp4>::kCtas;
}
template <bool kFp4>
int ctas_of(int dim, int heads) {
  return dim == 64 ? ctas_of<64, kFp4>(heads) : (dim == 128 ? ctas_of<128, kFp4>(heads) : ctas_of<256, kFp4>(heads));
}
inline int grid_of(const mixfp4_kv_cache* c, int64_t q_heads) {
  const int dim = padded_dim(c->head_dim), heads = padded_heads(c, q_heads);
  return num_sms() * (c->dtype == MIXFP4_CACHE_MIXFP4 ? ctas_of<true>(dim, heads) : ctas_of<false>(dim, heads));
}

template <int DT, int NT, bool kFp4>
int launch(const AttnArgs& p, int grid, cudaStream_t s) {
  using C = Cfg<DT, NT, kFp4>;
  static std::atomic<uint64_t> done{0};
  auto* kernel = paged_attention_kernel<DT, NT, kFp4>;
  if (!set_dynamic_smem_once(reinterpret_cast<const void*>(kernel), C::kSmem, done)) return MIXFP4_ERR_CUDA;
  if (p.cluster == 1) {
    kernel<<<(unsigned)(p.B * (p.c.heads / p.together) * p.chunks), kThreads, C::kSmem, s>>>(p);
    return launch_status();
  }
  if (p.cluster) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.cluster, attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.B * p.c.heads * p.chunks * p.cluster));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = C::kSmem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, p) == cudaSuccess ? MIXFP4_OK : MIXFP4_ERR_CUDA;
  }
  kernel<<<grid, kThreads, C::kSmem, s>>>(p);
  if (int st = launch_status()) return st;
  const int nh = p.group < C::kHeads ? p.group : C::kHeads, heads = kJoinThreads / 32 / p.share;
  const dim3 jg((unsigned)p.places, (unsigned)p.together, (unsigned)((nh + heads - 1) / heads));
  return launch_pdl(paged_attention_join_kernel<DT, NT, kFp4>, jg, dim3(kJoinThreads), 0, s, p) == cudaSuccess
             ? MIXFP4_OK
             : MIXFP4_ERR_CUDA;
}

template <int DT, bool kFp4>
int launch_heads(const AttnArgs& p, int grid, int heads, cudaStream_t s) {
  if constexpr (DT <= 128)
    if (heads == 24) return launch<DT, 3, kFp4>(p, grid, s);
  return heads == 8 ? launch<DT, 1, kFp4>(p, grid, s) : launch<DT, 2, kFp4>(p, grid, s);
}

template <bool kFp4>
int launch_dim(const AttnArgs& p, int grid, int heads, cudaStream_t s) {
  switch (padded_dim(p.c.head_dim)) {
    case 64: return launch_heads<64, kFp4>(p, grid, heads, s);
    case 128: return launch_heads<128, kFp4>(p, grid, heads, s);
    default: return launch_heads<256, kFp4>(p, grid, heads, s);
  }
}

}  // namespace
}  // namespace mixfp4

extern "C" {

int mixfp4_paged_attention_workspace(const mixfp4_kv_cache* cache, int64_t B, int64_t q_heads, int64_t* bytes) {
  using namespace mixfp4;
  if (int st = check_kv_cache(cache)) return st;
  if (!bytes) return MIXFP4_ERR_NULL;
  if (B < 0 || q_heads < 0 || q_heads % cache->heads != 0) return MIXFP4_ERR_SHAPE;
  *bytes = 0;
  if (B == 0 || q_heads == 0) return MIXFP4_OK;
  const int64_t grid = grid_of(cache, q_heads), heads = padded_heads(cache, q_heads) * 4;  // at most 4 together
  *bytes = (grid * 16 + 255) / 256 * 256 + grid * aside_bytes(cache, q_heads) + 2 * grid * heads * 8 +
           2 * grid * heads * padded_dim(cache->head_dim) * 4;
  return MIXFP4_OK;
}

int mixfp4_paged_attention(const void* q, int64_t q_stride, int64_t q_head_stride, int64_t B, int64_t q_heads,
                           const mixfp4_kv_cache* cache, const int32_t* block_table, int64_t table_stride,
                           int64_t table_pages, const int32_t* lengths, float scale, int64_t window, void* out,
                           float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  using namespace mixfp4;
  int64_t need = 0;
  if (int st = mixfp4_paged_attention_workspace(cache, B, q_heads, &need)) return st;
  if (B > INT32_MAX || q_heads > INT32_MAX || q_stride < 0 || q_head_stride < 0 || table_stride < 0 ||
      table_pages < 0 || table_stride < table_pages || table_pages > (INT32_MAX - 4096) / cache->page_size || window < 0 ||
      workspace_bytes < need)
    return MIXFP4_ERR_SHAPE;
  if (B == 0 || q_heads == 0) return MIXFP4_OK;
  if (!q || !out || !lengths || !workspace || (table_pages > 0 && !block_table)) return MIXFP4_ERR_NULL;
  if (!aligned(q, 16) || q_stride % 8 || q_head_stride % 8 || !aligned(block_table, 4) || !aligned(lengths, 4) ||
      !aligned(out, 16) || !aligned(lse, 4) || !aligned(workspace, 256))
    return MIXFP4_ERR_ALIGN;
  const int grid = grid_of(cache, q_heads);
  const int heads = padded_heads(cache, q_heads);
  AttnArgs p = {};
  p.q = static_cast<const uint16_t*>(q);
  p.q_stride = q_stride, p.q_head_stride = q_head_stride;
  p.B = (int)B, p.q_heads = (int)q_heads, p.group = (int)(q_heads / cache->heads);
  p.chunks = (int)((p.group + heads - 1) / heads);
  p.c = *cache;
  p.together = together_of(cache, B, p.chunks, grid);
  // Few rows that cannot be long: a cluster to each, all resident at once, which joins its CTAs' parts in shared
  // memory and so saves the second launch and its wait; many short ones: a CTA to each, and nothing to join.
  const int64_t bound = window > 0 && window < table_pages * cache->page_size ? window : table_pages * cache->page_size;
  const int64_t single = B * cache->heads * p.chunks;
  for (int n = kCluster; n > 1 && !p.cluster; n /= 2)
    if (single * n <= grid && bound <= n * kCtaTokens * (single * n >= grid / 2 ? 4 : 1)) p.cluster = n;
  if (!p.cluster && bound <= kRowTokens && single <= INT32_MAX) p.cluster = 1;
  if (p.cluster > 1) p.together = 1;
  while (1 << p.cluster_shift < p.cluster) ++p.cluster_shift;
  p.page_shift = -1;
  for (int i = 0; i < 31; ++i)
    if (cache->page_size == 1 << i) p.page_shift = i;
  p.table = block_table, p.table_stride = table_stride;
  p.max_tokens = table_pages * cache->page_size;
  p.lengths = lengths;
  p.scale = scale, p.window = window;
  p.out = static_cast<uint16_t*>(out), p.lse = lse;
  // The joining kernel gets a CTA for each place, key head and few query heads: where they would be few,
  // more warps to a query head.
  const int64_t all_rows = B * (cache->heads / p.together) * p.chunks;
  p.by_row = all_rows <= grid;
  p.places = (int)(p.by_row ? all_rows : grid);
  p.share = 1;
  while (p.share < 8 && (p.share * 2 * p.group <= 8 || (int64_t)p.places * p.together * p.group * p.share < 4096))
    p.share *= 2;
  uint8_t* w = static_cast<uint8_t*>(workspace);
  p.split = reinterpret_cast<int4*>(w);
  w += ((int64_t)grid * 16 + 255) / 256 * 256;
  p.aside = reinterpret_cast<float4*>(w);
  w += grid * aside_bytes(cache, q_heads);
  p.stat = reinterpret_cast<float2*>(w);
  p.part = reinterpret_cast<float*>(w + 2 * (int64_t)grid * p.together * heads * 8);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return cache->dtype == MIXFP4_CACHE_MIXFP4 ? launch_dim<true>(p, grid, heads, s) : launch_dim<false>(p, grid, heads, s);
}

}  // extern "C"
