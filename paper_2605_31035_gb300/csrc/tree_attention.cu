// Attention of drafted tokens over the paged cache (mixfp4_tree_attention).
//
// A key head's queries, t drafts times the query heads that share it, are the rows of a tcgen05 tile of 128, or of two
// tiles over the same tokens.  To a tile of 64 tokens (128 on a MixFP4 cache with one tile of rows) S = Q K^T goes to
// tensor memory; four warps a tile of rows take it from there, a row to a thread, and put the softmax's weights P back in
// its place; O += P V follows with P from tensor memory.  m and l are held in fp32 beside O, and O is only scaled again
// where the maximum has grown by more than 2^16 (2^8): weights are relative to a maximum that may be an old one.
//
//   * Roles: rows of K and V come by TMA into a ring, boxes of one page, where the strides allow it, by cp.async
//     otherwise; a MixFP4 cache's codes and scale bytes come the same ways and eight warps write them into the ring as
//     exact f16.  One thread issues the products, one warp reads the next part of the work ahead.  Every wait ends
//     after a second at the latest, with an error in the status word; what is in flight then still lands before
//     the CTA ends.
//   * Few rows: 32 (or 64) rows are held four times (twice) in the 128 lanes and each copy takes its quarter (half) of a
//     tile's tokens, by products that write its lanes of O alone; the copies are joined at the end.  A thread then has a
//     quarter of the scores: 179 instead of 192 us at 8 drafts below, 185 instead of 239 on a MixFP4 cache.
//   * More than 128 rows (and up to 128 dimensions): two tiles of rows to a CTA, so that K and V are fetched, and decoded,
//     once for both.  375 instead of 420 us at 64 drafts, 428 instead of 532 on a MixFP4 cache; at 40 drafts 363 and 380,
//     401 and 443.
//   * On a bf16 cache the weights keep 16 bits in two bf16 parts of one sign; on a MixFP4 one f16's 11, and the queries
//     are scaled per row by a power of two into f16: exact but for elements below 2^-31 of the row's largest, which are
//     off by up to 2^-39 of it, half of f16's least step.
//   * Where rows of a tile see different tokens (drafts, a window's edge; one draft alone whose own bit is off sees less
//     than there is), a weight of 0 would still make NaN of an infinite or NaN element of V.  Such tiles are looked over
//     for those, and where there is one the threads take the products themselves, of what each row sees alone.
//   * Tokens are cut into equal shares over the device.  CTAs of neighbouring heads walk the same tokens at the same time,
//     whose rows lie together: 179 instead of 181 us at 8 drafts, 375 instead of 383 at 64, on a MixFP4 cache
//     185 instead of 206 and 428 instead of 467.
//
// Measured on 64 sequences of up to 8192 tokens, 32 query heads on 8, 128 dimensions (bf16 cache 1.1 GB, MixFP4 0.3 GB):
// bf16 179 us at 8 drafts (6.1 TB/s: bound by HBM), 193 at 16, 375 at 64 (658 TFLOP/s: bound by the tensor cores, which
// take P in two parts, and by what the softmax of 256 rows issues); MixFP4 185 us at 8 and 428 at 64 drafts, bound by the
// instructions of decoding and of the softmax (half of the issue slots used).  Short rows are bound by their beginning
// and end, some 7 us each: 142 sequences of 2 tokens with 32 key heads, 30 rows to an SM, 106 us, MixFP4 215.
// The rules here and below give both sides, the other one measured with all else as it is.
#include <cuda_runtime.h>
#include <atomic>
#include <cstdint>

#include "decode.cuh"
#include "host_util.cuh"
#include "kernels.cuh"
#include "kvcache.cuh"
#include "pipeline.cuh"
#include "ptx.cuh"
#include "sm100.cuh"

namespace mixfp4 {
namespace {

using namespace sm100;

constexpr int kMostDrafts = 64;
constexpr int kJoinThreads = 256;
constexpr uint64_t kWaitLimitNs = 1000000000ull;
// Tokens after which O is set aside and begins at 0: the tensor cores round a chain of sums towards zero, some 2^-25 of
// the sum a link, and 8192 tokens are 512 links (1024 with two parts of the weights).
constexpr int kChainTokens = 8192;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// How far a score may lie above the m of its weight 2^(s - m), which follows the maximum from afar (179 us at 8 drafts,
// 375 at 64, MixFP4 185 and 428; 182 and 407, 191 and 478 where it follows at once): bf16 parts and fp32 sums have the
// room.  On a MixFP4 cache the weights are 2^7 times that: at most 2^15 in f16, whose least value is then 2^-31 of the
// weight at m.
constexpr float kSlack = 16.0f, kFp4Slack = 8.0f, kFp4Exp = 7.0f;
// A MixFP4 operand's elements are their values under the block scale over this (fp4_to_f16).
constexpr float kFp4Unit = 512.0f;
constexpr float kNoScore = -3e38f;  // m where no token has been seen: no difference to a score or to itself is NaN
constexpr float kMostScore = 3.402823466e38f;  // m of a score of +inf, whose weight is then +inf instead of NaN
constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr int kMostSlots = 12;
constexpr int kThere = 16;   // tiles whose tokens are known at a time

struct TreeArgs {
  const uint16_t* q;
  int64_t q_stride, q_token_stride, q_head_stride;
  int B, t, q_heads, group;
  int chunks;    // of 128 (or 256) rows to a key head
  int together;  // key heads whose CTAs walk together
  int shares;    // of the tokens; a CTA has one share and one of `together` heads
  int joined;    // whether rows may be cut, and a second kernel joins them
  mixfp4_kv_cache c;
  int page_shift;  // log2 page_size, or -1
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
  int4* split;   // [grid]: the row that a CTA begins and others end: (sequence, row, first share, last); x < 0: none
  float2* stat;  // [2 grid][row tiles][128] (m, l) of parts
  float4* part;  // [2 grid][row tiles][dimensions / 4][128]: O of parts, and what a row in work has set aside
  uint32_t* status;
  uint64_t wait_ns;  // of the self-test: the limit of every wait
  int box;  // rows of a page that one TMA copy brings; 0: cp.async does
  // A MixFP4 cache's scale bytes by TMA: bytes from one row's to the next in shared memory, and whether a copy brings
  // those of neighbouring heads of a token (16 bytes) or of neighbouring tokens of a head.
  int scale_pitch, scale_by_head;
};

// What of a sequence is looked at.
struct Span {
  int n, c, first;  // tokens, drafts, certain tokens
  int from, end;    // tokens [from, end) may be seen; from is a tile's first
  int low;          // tokens below are not
};
// A part of a row: tiles [tile, tile + tiles) of chunk `chunk` of key head `head` of sequence b, walked from the last on.
struct Part {
  Span s;
  int b, row, head, chunk, tile, tiles;
  bool first, last;
  int64_t behind;  // the unit behind the row's last
};

template <int kSlots, int kAddresses, int kWords, int MT, bool kFp4>
struct Shared {
  uint64_t full[kSlots], empty[kSlots], placed[kAddresses], used[kAddresses];
  uint64_t raw_full[3], raw_empty[3];
  // Of a buffer of scores: they are there, their weights are, O has taken those up.  No buffer has two uses under way, so
  // the parity of a wait tells one use from the next.
  uint64_t s_full[2 * MT], p_full[2 * MT], o_done[2 * MT];
  uint64_t told, heard, q_full, end;
  uint32_t tmem;
  int abort;
  int skip[2 * MT];
  int64_t all, shares, before, edge[2];
  int edge_b;
  uint32_t there[kThere][kWords];  // of a tile, which of its tokens there are
  // The part that softmax is at, read ahead by a warp of its own: which drafts each draft sees, and how many.
  uint8_t depth[kMostDrafts];
  uint8_t exponent[kFp4 ? MT * 128 : 8];  // of a row's largest query element
  Part part;
  union {
    uint64_t bits[kMostDrafts];
    int64_t scan[32];  // of the shares, before the first part
  };
};

// Tensor maps of keys and values, and of their scale bytes.
struct Maps {
  CUtensorMap rows[2], scales[2];
};

template <int DT, int MT, bool kFp4>
struct Cfg {
  // With one tile of rows two CTAs share an SM: what one does once a row (its queries, its end) the other's tiles cover
  // (179 instead of 204 us at 8 drafts).  A MixFP4 cache's decoding takes the registers and the shared memory of one.
  static constexpr int kCtas = !kFp4 && MT == 1 && DT <= 128 ? 2 : 1;
  // Of a tile.  A larger one has fewer steps between the roles, which on a MixFP4 cache are most of the time (185 instead
  // of 263 us at 8 drafts); a bf16 one of two CTAs has no room for it, nor have two tiles of rows in tensor memory.
  static constexpr int kTokens = kFp4 && MT == 1 && DT <= 128 ? 128 : 64;
  // What beginning a row costs (its queries, the way to its first pages, its end), in tiles.  64 sequences of up to 8192
  // tokens, us at a cost of 0, 2, 4, 8 and 12: 8 drafts 190, 181, 179, 180, 180, MixFP4 193, 188, 185, 189, 195; 64 drafts
  // 419, 399, 390, 375, 377.
  static constexpr int kRowCost = MT == 2 ? 8 : 4;
  static constexpr int kChain = kChainTokens / kTokens;    // tiles to a chain of sums
  static constexpr int kCw = kTokens / 4;                  // and of its quarter, a thread's step
  static constexpr int kBlock = kTokens * 128;             // 64 dimensions of a tile
  // Columns of scores that a thread has in registers; with one tile of rows its copy's share of a tile, or a part of it;
  // with two 32 (at 40 and 64 drafts 363 and 375 us; with 16 370 and 378, MixFP4 401 and 428, 424 and 438).
  static constexpr int kStep = kTokens == 128 || MT == 2 ? 32 : 16;
  static_assert(kStep == kCw || MT == 2);
  static constexpr int kSlot = kBlock * (DT / 64);
  static constexpr int kSoftmax = 4 * MT;                  // warps, four to a tile of rows
  static constexpr int kQ = MT * 128 * DT * 2;
  // Warps that decode (185 us at 8 drafts; 16 of them, with 80 registers to a thread, 268), or bring a bf16 cache's rows
  // where TMA cannot.
  static constexpr int kProducers = kFp4 ? 8 : 2;
  static constexpr int kThreads = (kSoftmax + 4 + (kFp4 ? kProducers : 0)) * 32;  // the four: products, TMA or helpers
  // Registers of a thread at launch, then of softmax and of the other threads (together no more than at launch).  MixFP4
  // at 64 drafts 428 us; with no split, or with 72 for the others, 436, with 88 432.
  static constexpr int kRegs = 65536 / (kThreads * kCtas) / 8 * 8;
  static constexpr int kOtherRegs = kFp4 && MT == 2 ? 80 : kRegs;
  static constexpr int kLeft = (kRegs * kThreads - kOtherRegs * (kThreads - kSoftmax * 32)) / (kSoftmax * 32) / 8 * 8;
  static constexpr int kSoftRegs = kLeft < 232 ? kLeft : 232;
  static constexpr int kRows = kTokens / kProducers;       // of a tile, to a producer warp
  static constexpr int kCodes = kTokens * (DT / 2);        // bytes of a MixFP4 tile's keys as they lie
  static constexpr int kRawTile = 2 * kCodes + 2 * kTokens * 16;  // keys, values, their scale bytes (16 bytes to a row)
  static constexpr int kRawDepth = kFp4 ? 3 : 0;           // tiles
  static constexpr int kRaw = kRawDepth * kRawTile;
  static constexpr int kAddresses = kFp4 ? 2 : 0;          // tiles whose rows' places are known
  static constexpr int kPlaces = kAddresses * kTokens * 16;
  static constexpr int kWords = kTokens / 32;
  static constexpr int kRoom = (kCtas == 2 ? 113 : 227) * 1024 - kQ - kRaw - kPlaces;
  static constexpr int slots(int n) {  // as many as there is room for
    return n == 1 || n * (kSlot + 16) + (int)sizeof(Shared<1, kFp4 ? 2 : 1, kWords, MT, kFp4>) <= kRoom ? n : slots(n - 1);
  }
  static constexpr int kSlots = slots(kMostSlots);
  using Sh = Shared<kSlots, kFp4 ? 2 : 1, kWords, MT, kFp4>;
  static constexpr int kSmem = kQ + kSlots * kSlot + kRaw + kPlaces + (int)sizeof(Sh);
  static_assert(kSlots >= 3 && sizeof(Sh) % 8 == 0 && kSmem <= (kCtas == 2 ? 113 : 227) * 1024);
  static constexpr uint32_t kScoreCols = 2 * MT * kTokens; // of tensor memory, O behind them
  static constexpr uint32_t kCols = kCtas == 2 ? 256 : 512;
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
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(n) : "memory");
}
__device__ __forceinline__ void cp_wait_at_most(int n) {
  switch (n) {
    case 0: return cp_wait<0>();
    case 1: return cp_wait<1>();
    case 2: return cp_wait<2>();
    case 3: return cp_wait<3>();
    case 4: return cp_wait<4>();
    case 5: return cp_wait<5>();
    default: return cp_wait<6>();
  }
}
__device__ __forceinline__ uint32_t lds8(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void sts8(uint32_t a, uint32_t v) {
  asm volatile("st.shared.u8 [%0], %1;" ::"r"(a), "r"(v) : "memory");
}
__device__ __forceinline__ void bar_sync(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
__device__ __forceinline__ bool bar_or(int id, int threads, bool v) {
  int r;
  asm volatile("{ .reg .pred p, q; setp.ne.s32 p, %3, 0; bar.red.or.pred q, %1, %2, p; selp.s32 %0, 1, 0, q; }"
               : "=r"(r)
               : "r"(id), "r"(threads), "r"((int)v)
               : "memory");
  return r != 0;
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
__device__ __forceinline__ float bf_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }
// 2^x, results below 2^-126 as zero.
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// tanh of two numbers, within 2^-21 of itself: x P(x^2) / Q(x^2) for |x| <= 9, beyond which it is 1 in fp32.  The
// coefficients are a weighted least-squares fit of tanh(x) / x that evens out the relative error (2e-8 before rounding).
// Written out for pairs, on which fp32 products and sums work at once: 11 instructions to a number instead of 17.
__device__ __forceinline__ void tanh2(float& x0, float& x1) {
  auto held = [](float x) {  // NaN stays
    float y;
    asm("{ .reg .f32 t; max.NaN.f32 t, %1, 0fC1100000; min.NaN.f32 %0, t, 0f41100000; }" : "=f"(y) : "f"(x));
    return y;
  };
  auto both = [](float c) { return pack2(c, c); };
  const u64 z = pack2(held(x0), held(x1)), y = mul2(z, z);
  u64 a = fma2(y, both(1.335449179e-08f), both(2.060896267e-05f));
  u64 b = fma2(y, both(7.776489695e-07f), both(3.285623034e-04f));
  a = fma2(y, a, both(3.495580968e-03f)), b = fma2(y, b, both(2.587695507e-02f));
  a = fma2(y, a, both(1.338101964e-01f)), b = fma2(y, b, both(4.671433524e-01f));
  a = fma2(y, a, both(1.0f)), b = fma2(y, b, both(1.0f));
  float b0, b1;
  unpack2(b, b0, b1);
  unpack2(mul2(mul2(z, a), pack2(rcp(b0), rcp(b1))), x0, x1);
}
// As mma_f16_tmem_a, lanes of D whose bit is set in the four words left as they are.
__device__ __forceinline__ void mma_f16_tmem_a_lanes(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                                     uint32_t accumulate, uint4 off) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%5, %6, %7, %8}, p;\n}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(off.x), "r"(off.y), "r"(off.z), "r"(off.w)
      : "memory");
}
// A box of a [page][head][token][element] tensor.
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* m, int x, int token, int head, int page,
                                            uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(token), "r"(head), "r"(page), "r"(bar)
      : "memory");
}
// D[tmem] (+)= A[smem] . B[smem]^T, one CTA, kind::f16.
__device__ __forceinline__ void mma_f16(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                        uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Descriptor of an operand whose rows are its K: 64 elements of M or N to a row of 128 bytes, swizzled as
// smem_desc_sw128's; 8 rows to 1024 bytes, `lbo` bytes to the next 64 elements.
__device__ __forceinline__ uint64_t smem_desc_sw128_mn(uint32_t saddr, uint32_t lbo) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr >> 4) & 0x3FFFu);
  d |= (uint64_t)((lbo >> 4) & 0x3FFFu) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
__device__ __forceinline__ void tmem_ld1(uint32_t taddr, uint32_t& v) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(v) : "r"(taddr) : "memory");
  tmem_ld_wait();
  asm volatile("" : "+r"(v));
}
// kCols (32 or 16) columns of this thread's lane.
template <int kCols>
__device__ __forceinline__ void tmem_load(uint32_t taddr, uint32_t* v) {
  if constexpr (kCols == 32)
    tmem_ld_32x32b_x32(taddr, v);
  else
    tmem_ld_32x32b_x16(taddr, v);
}
// Waits for loaded columns, and keeps their use behind the wait.
template <int kCols>
__device__ __forceinline__ void tmem_loaded(uint32_t* v) {
  if constexpr (kCols == 32)
    tmem_ld_wait_x32(v);
  else
    tmem_ld_wait_x16(v);
}
template <int kCols>
__device__ __forceinline__ void tmem_store(uint32_t taddr, const uint32_t* v) {
  if constexpr (kCols == 32) {
    tmem_st_32x32b_x32(taddr, v);
  } else if constexpr (kCols == 16) {
    tmem_st_32x32b_x16(taddr, v);
  } else {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(v[0]),
                 "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
  }
}

template <class C>
__device__ __forceinline__ Span span_of(const TreeArgs& p, int b) {
  Span s;
  s.n = max(p.lengths[b], 0);
  s.c = p.counts ? min(max(p.counts[b], 0), p.t) : p.t;
  s.c = min(s.c, s.n);
  s.first = s.n - s.c;
  s.end = (int)min((int64_t)s.n, p.max_tokens);
  s.low = p.window > 0 ? (int)max((int64_t)0, s.first + 1 - p.window) : 0;  // of the drafts, those that see none
  s.from = s.low & ~(C::kTokens - 1);
  return s;
}
// Units of work of a row of the sequence: kRowCost for its beginning, then one to a tile.
template <class C>
__device__ __forceinline__ int units_of(const Span& s) {
  return s.c > 0 && s.end > s.low ? C::kRowCost + (s.end - s.from + C::kTokens - 1) / C::kTokens : 0;
}

// Every role walks a CTA's share in the same steps.
template <class C>
struct Walk {
  int64_t pos, end, base;
  int b;
  __device__ __forceinline__ bool next(const TreeArgs& p, int mate, Part& w) {
    const int rows = p.c.heads / p.together * p.chunks;
    while (pos < end && b < p.B) {
      w.s = span_of<C>(p, b);
      const int u = units_of<C>(w.s);
      if (u == 0 || pos >= base + (int64_t)u * rows) {
        base += (int64_t)u * rows;
        ++b;
        continue;
      }
      w.b = b;
      w.row = (int)((pos - base) / u);
      const int k0 = (int)((pos - base) - (int64_t)w.row * u), cnt = (int)min((int64_t)(u - k0), end - pos);
      w.head = w.row / p.chunks * p.together + mate;
      w.chunk = w.row % p.chunks;
      w.tile = max(k0 - C::kRowCost, 0);
      w.tiles = k0 + cnt - C::kRowCost - w.tile;
      w.first = k0 == 0;
      w.last = k0 + cnt == u;
      w.behind = base + (int64_t)(w.row + 1) * u;
      pos += cnt;
      if (w.tiles > 0) return true;
    }
    return false;
  }
};

// A finished row's factor of O, and its log-sum-exp, of m and l.  l is 0 only where no token was seen (or all scores
// are -inf); NaN goes through, and so does the +inf of a score of +inf.
template <bool kFp4>
__device__ __forceinline__ float out_factor(float l, float vts) {
  return l == 0.0f ? 0.0f : (kFp4 ? kFp4Unit * vts : 1.0f) / l;
}
template <bool kFp4>
__device__ __forceinline__ float lse_of(float m, float l) {
  return l == 0.0f ? -INFINITY : (m + log2f(l) - (kFp4 ? kFp4Exp : 0.0f)) * kLn2;
}

// The lowest k bits.
__device__ __forceinline__ uint32_t below(int k) { return k <= 0 ? 0u : (k >= 32 ? kAll : (1u << k) - 1u); }
// Which of the 32 tokens from a on, at column `col` of a tile, there are, a bit each; bit i of `good`: box i has a page.
__device__ __forceinline__ uint32_t there_of(const TreeArgs& p, const Span& s, int a, int col, uint32_t good) {
  uint32_t v = below(s.end - a) & ~below(s.low - a);
  if (!((good >> (col / p.box)) & 1u)) v &= 0xFFFF0000u;
  if (!((good >> ((col + 16) / p.box)) & 1u)) v &= 0xFFFFu;
  return v;
}

// Which drafts draft k of sequence b sees, of its c.
__device__ __forceinline__ uint64_t bits_of(const TreeArgs& p, int b, int k, int c) {
  const uint64_t all = c >= 64 ? ~0ull : (1ull << c) - 1;
  return (p.mask ? (uint64_t)p.mask[b * p.mask_stride + k] : (2ull << k) - 1) & all;
}
__device__ __forceinline__ int depth_of(uint64_t bits, int k) { return __popcll(bits & ~(1ull << k)); }

// Which 16 elements of which row a lane takes of a MixFP4 tile: eight neighbouring lanes four pieces of two rows, whose
// places in the operand are then in different banks.
template <int DT>
struct Lanes {
  static constexpr int kPieces = DT / 16, kRowsAtOnce = 32 / kPieces;
  static constexpr int kShift = DT == 64 ? 3 : (DT == 128 ? 4 : 5);
  static __device__ __forceinline__ int piece(int lane) { return (lane & 3) | ((lane >> 3 & (kPieces / 4 - 1)) << 2); }
  static __device__ __forceinline__ int row(int lane) { return (lane >> 2 & 1) | (lane >> kShift << 1); }
};

// A MixFP4 tile's elements in f16, at 2^-9 of their values under the block scale alone: a payload's three bits are those
// of an f16 below its sign, and hold E2M1's value times 2^-14 at bits 11 to 9, E1M2's times 2^-16 at 10 to 8, subnormals
// included; a factor of the scale times 2^5 (2^7) makes both exact multiples of 2^-19 below 8.
// The order that eight elements then have, and the operands with them: nibbles of even places first, i and i + 4 to a
// word.  It is its own inverse.
__device__ __forceinline__ constexpr int fp4_order(int i) { return (i & 1) << 2 | (i & 2) | (i >> 2 & 1); }
__device__ __forceinline__ void fp4_to_f16(uint32_t w, uint32_t e1m2, uint32_t s2, uint32_t* out) {
  const uint32_t even = ((w << 4) & 0x80808080u) | (w & 0x07070707u) * (2u - e1m2);
  const uint32_t odd = (w & 0x80808080u) | ((w & 0x70707070u) >> (3u + e1m2));
  out[0] = hmul2(prmt(even, 0u, 0x2404u), s2);
  out[1] = hmul2(even & 0xFF00FF00u, s2);
  out[2] = hmul2(prmt(odd, 0u, 0x2404u), s2);
  out[3] = hmul2(odd & 0xFF00FF00u, s2);
}

// A lane's pieces of a MixFP4 tile, 16 elements of each of kSteps rows: all asked for at once, then decoded to the
// operand's swizzled places.
template <int kSteps>
struct Codes {
  uint2 c[kSteps];
  uint32_t scale[kSteps];
  __device__ __forceinline__ void load(uint32_t codes, int step, uint32_t scales, const int* at) {
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      c[j] = lds64(codes + j * step);
      scale[j] = lds8(scales + at[j]);
    }
  }
  // `at`: the first 16 bytes of row j's 32 in the slot `to`; the others are in its other half.
  __device__ __forceinline__ void decode(uint32_t to, const int* at) const {
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const uint32_t e1m2 = scale[j] >> 7;
      const uint32_t s2 = hmul2(cvt_f16x2_from_e4m3x2((uint16_t)((scale[j] & 0x7Fu) * 0x0101u)),
                                0x50005000u + e1m2 * 0x08000800u);
      uint32_t v[2][4];
      fp4_to_f16(c[j].x, e1m2, s2, v[0]);
      fp4_to_f16(c[j].y, e1m2, s2, v[1]);
      sts128(to + at[j], v[0][0], v[0][1], v[0][2], v[0][3]);
      sts128(to + (at[j] ^ 16), v[1][0], v[1][1], v[1][2], v[1][3]);
    }
  }
};

// kWithheld: the self-test of the failure path, in which rows of a CTA's first tile are never sent (an argument instead of
// a variant cost 2 to 4 % on a MixFP4 cache).
template <int DT, int MT, bool kFp4, bool kWithheld>
__global__ void __launch_bounds__(Cfg<DT, MT, kFp4>::kThreads, Cfg<DT, MT, kFp4>::kCtas)
    tree_attention_kernel(const TreeArgs p, const __grid_constant__ Maps tm) {
  using C = Cfg<DT, MT, kFp4>;
  constexpr int TN = C::kTokens, CW = C::kCw, PW = C::kStep;
  extern __shared__ __align__(1024) uint8_t smem[];
  auto& sh = *reinterpret_cast<typename C::Sh*>(smem + C::kQ + C::kSlots * C::kSlot + C::kRaw + C::kPlaces);
  const uint32_t q_smem = smem_u32(smem), ring = q_smem + C::kQ;
  [[maybe_unused]] const uint32_t raw_tiles = ring + C::kSlots * C::kSlot;  // [kRawDepth]
  [[maybe_unused]] const uint32_t places = raw_tiles + C::kRaw;  // [kAddresses][tokens] (row, scales)
  volatile int* abort_flag = &sh.abort;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int share = (int)blockIdx.x / p.together, mate = (int)blockIdx.x % p.together;
  const int D = p.c.head_dim;
  griddep_launch_dependents();

  if (warp == C::kSoftmax) {
    tmem_alloc(smem_u32(&sh.tmem), C::kCols);
    tmem_relinquish();
  } else if (tid == 0) {
    for (int i = 0; i < C::kSlots; ++i) {
      mbar_init(smem_u32(&sh.full[i]), kFp4 ? C::kProducers : (p.box ? 1 : C::kProducers * 32));
      mbar_init(smem_u32(&sh.empty[i]), 1);
    }
    for (int i = 0; i < C::kRawDepth; ++i) {
      mbar_init(smem_u32(&sh.raw_full[i]), 1);
      mbar_init(smem_u32(&sh.raw_empty[i]), C::kProducers);
    }
    for (int i = 0; i < C::kAddresses; ++i) {
      mbar_init(smem_u32(&sh.placed[i]), 1);
      mbar_init(smem_u32(&sh.used[i]), C::kProducers);
    }
    for (int i = 0; i < 2 * MT; ++i) {
      mbar_init(smem_u32(&sh.s_full[i]), 1);
      mbar_init(smem_u32(&sh.p_full[i]), 4);
      mbar_init(smem_u32(&sh.o_done[i]), 1);
    }
    mbar_init(smem_u32(&sh.told), 1);
    mbar_init(smem_u32(&sh.heard), C::kSoftmax);
    mbar_init(smem_u32(&sh.q_full), C::kSoftmax);
    mbar_init(smem_u32(&sh.end), 1);
    sh.abort = 0;
    sh.edge_b = p.B;
    p.split[blockIdx.x] = make_int4(-1, 0, 0, 0);
    fence_mbar_init();
  }

  // This CTA's share [pos, end) of all units, and the sequence it starts in.
  Walk<C> walk;
  const int rows = p.c.heads / p.together * p.chunks;
  {
    const int strip = (p.B + C::kThreads - 1) / C::kThreads, lo = min(p.B, tid * strip), hi = min(p.B, lo + strip);
    int64_t mine = 0;
    for (int i = lo; i < hi; ++i) mine += units_of<C>(span_of<C>(p, i));
    int64_t before = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t v = __shfl_up_sync(kAll, before, d);
      if (lane >= d) before += v;
    }
    if (lane == 31) sh.scan[warp] = before;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    int64_t total = 0;
    for (int w = 0; w < C::kThreads / 32; ++w) {
      if (w < warp) before += sh.scan[w];
      total += sh.scan[w];
    }
    before -= mine;
    const int64_t all = total * rows, shares = min(all, (int64_t)p.shares);
    for (int64_t i = blockIdx.x; i < p.B; i += gridDim.x) {  // sequences that see nothing
      if (units_of<C>(span_of<C>(p, (int)i)) > 0) continue;
      const int64_t heads = (int64_t)p.t * p.q_heads, words = heads * D / 2;
      for (int64_t k = tid; k < words; k += C::kThreads) reinterpret_cast<uint32_t*>(p.out)[i * words + k] = 0u;
      if (p.lse)
        for (int64_t k = tid; k < heads; k += C::kThreads) p.lse[i * heads + k] = -INFINITY;
    }
    walk.pos = 0, walk.end = 0, walk.base = 0, walk.b = 0;
    if (share < shares) {
      // An edge between shares that falls into a row's beginning lies before the row.
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int64_t edge = all * (share + k) / shares;
        if (edge >= before * rows && edge < (before + mine) * rows) {
          int i = lo;
          int64_t at = before;
          int u = units_of<C>(span_of<C>(p, i));
          while (i < hi - 1 && edge >= (at + u) * rows) {
            at += u;
            u = units_of<C>(span_of<C>(p, ++i));
          }
          const int64_t into = u > 0 ? (edge - at * rows) % u : 0;
          sh.edge[k] = into <= C::kRowCost ? edge - into : edge;
          if (k == 0) sh.edge_b = i, sh.before = at;
        } else if (edge == all && tid == 0) {
          sh.edge[k] = all;
        }
      }
    }
    __syncthreads();
    if (share < shares) walk.pos = sh.edge[0], walk.end = sh.edge[1], walk.b = sh.edge_b, walk.base = sh.before * rows;
    // Last share of the row that ends before unit x (see `split`).
    if (tid == 0) sh.all = all, sh.shares = shares;
  }
  const uint32_t tmem = sh.tmem;
  // A wait has run out: no more waits and no more results, but every step, so that all warps meet.  Slots are then freed too
  // early and places not written: whoever asks for copies looks at the flag as well before each, and whoever reads places
  // stops.
  bool dead = false;
  const uint64_t limit = kWithheld ? p.wait_ns : kWaitLimitNs;
  auto wait = [&](uint64_t& bar, uint32_t parity, uint32_t bit) {
    if (!dead && !mbar_wait(smem_u32(&bar), parity, abort_flag, limit)) {
      dead = true;
      if (p.status && !*abort_flag) atomicOr(p.status, bit);
      *abort_flag = 1;
    }
  };
  // The same for a whole warp, whose lanes agree on it.
  auto waits = [&](uint64_t& bar, uint32_t parity, uint32_t bit) {
    wait(bar, parity, bit);
    dead = __any_sync(kAll, dead);
  };
  const float kts = kFp4 ? *p.c.k_ts : 1.0f, vts = kFp4 ? *p.c.v_ts : 1.0f;
  Part w;

  if (warp < C::kSoftmax) {
    if constexpr (C::kSoftRegs > C::kRegs) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kSoftRegs));
    // ================================================= softmax: a row to a thread
    const int m = warp >> 2, qd = warp & 3, tl = tid & 127;
    const uint32_t lanes = tmem + ((uint32_t)qd * 32u << 16);
    const uint32_t o_col = lanes + C::kScoreCols + m * DT;
    uint32_t g = 0, turn = 0;  // tiles and parts before this one
    for (;;) {
      // All warps of softmax have the same parts and so meet at the same barriers, also where a wait has run out.
      if (bar_or(1, C::kSoftmax * 32, !mbar_wait(smem_u32(&sh.told), turn & 1, nullptr, limit))) break;
      w = sh.part;
      if (w.tiles == 0) break;
      const int R = min(128 * MT, p.t * p.group - w.chunk * 128 * MT);
      const int copies = MT == 2 || R > 64 ? 1 : (R > 32 ? 2 : 4), own = 128 / copies, steps = 4 / copies;
      const int r = m * 128 + tl % own, copy = tl / own, step0 = copy * steps;
      const int idx = w.chunk * 128 * MT + r, i = idx / p.group, h = w.head * p.group + idx - i * p.group;
      const bool held = r < R, valid = held && i < w.s.c;  // rows behind the drafts have a result too, of zeros
      const bool idle = m * 128 + (copies == 1 ? qd * 32 : 0) >= R;
      const uint8_t* depth = sh.depth;
      uint64_t sees = valid ? sh.bits[i] : 0;
      const int place = w.s.first + (valid ? depth[i] : 0);
      const float slope = p.slopes && valid ? p.slopes[h] * -kLog2e : 0.0f;

      // ---- the row's queries, into the swizzled tile
      // A warp brings its rows' (those of which it has copies with the warps that have the others), a row by DT / 8
      // neighbouring lanes, to each copy's place.
      float fs = p.scale * (kFp4 ? kFp4Unit * kts : 1.0f);
      {
        constexpr int kLanes = DT / 8, kRowsAtOnce = 32 / kLanes;
        constexpr int kBatch = 4;  // steps asked for at once (2: 396 us at 64 drafts, 4: 375, 8: 373; MixFP4 442, 428, 438)
        const int steps_q = kLanes / copies, u = lane % kLanes, base = copy * (32 / copies) + lane / kLanes;
        const int64_t from = valid ? (int64_t)w.b * p.q_stride + (int64_t)i * p.q_token_stride + (int64_t)h * p.q_head_stride
                                   : -1;
        const uint32_t tile = q_smem + m * (128 * DT * 2) + (tl % own & 96) * 128 + (u >> 3) * 16384;
#pragma unroll 1
        for (int k0 = 0; k0 < steps_q; k0 += kBatch) {
          uint4 v[kBatch];
#pragma unroll
          for (int k = 0; k < kBatch; ++k) {
            v[k] = make_uint4(0, 0, 0, 0);
            const int64_t x = __shfl_sync(kAll, from, base + (k0 + k) * kRowsAtOnce);
            if (x >= 0 && u * 8 < D && k0 + k < steps_q) v[k] = *reinterpret_cast<const uint4*>(p.q + x + u * 8);
          }
#pragma unroll
          for (int k = 0; k < kBatch; ++k) {
            if (k0 + k >= steps_q) break;
            const int row = base + (k0 + k) * kRowsAtOnce;
            if (kFp4) {  // q times 2^(14 - exponent of the row's largest) as f16, in the keys' order
              float top = max3f(fabsf(bf_lo(v[k].x)), fabsf(bf_hi(v[k].x)), fabsf(bf_lo(v[k].y)));
              top = max3f(top, fabsf(bf_hi(v[k].y)), fabsf(bf_lo(v[k].z)));
              top = max3f(top, fabsf(bf_hi(v[k].z)), fabsf(bf_lo(v[k].w)));
              top = fmaxf(top, fabsf(bf_hi(v[k].w)));
#pragma unroll
              for (int d = 1; d < kLanes; d *= 2) top = fmaxf(top, __shfl_xor_sync(kAll, top, d));
              const int e = min(max((int)(__float_as_uint(top) >> 23), 15), 253);
              const float up = __uint_as_float((uint32_t)(268 - e) << 23);
              if (u == 0)
                for (int c = 0; c < copies; ++c) sh.exponent[m * 128 + c * own + (tl % own & 96) + row] = (uint8_t)e;
              const uint4 x = v[k];
              v[k].x = f16x2(bf_lo(x.x) * up, bf_lo(x.z) * up), v[k].y = f16x2(bf_lo(x.y) * up, bf_lo(x.w) * up);
              v[k].z = f16x2(bf_hi(x.x) * up, bf_hi(x.z) * up), v[k].w = f16x2(bf_hi(x.y) * up, bf_hi(x.w) * up);
            }
            for (int c = 0; c < copies; ++c)
              sts128(tile + (c * own + row) * 128 + (((u & 7) ^ (row & 7)) << 4), v[k].x, v[k].y, v[k].z, v[k].w);
          }
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sh.q_full));
      if (kFp4) {
        bar_sync(4 + m, 128);
        fs *= __uint_as_float((uint32_t)(sh.exponent[m * 128 + tl] - 14) << 23);
      }
      const float cap2 = p.softcap * kLog2e;
      fs *= p.softcap > 0.0f ? 1.0f / p.softcap : kLog2e;
      if (p.window > 0)
        for (int k = 0; k < w.s.c; ++k)
          if (place - w.s.first - depth[k] >= p.window) sees &= ~(1ull << k);
      const int low = p.window > 0 ? (int)max((int64_t)0, place + 1 - p.window) : 0;
      const bool plain = p.softcap == 0.0f && !p.slopes && p.scale > 0.0f && kts > 0.0f;

      float mx = kNoScore, l = 0.0f, m_aside = kNoScore;  // mx: the m of the weights
      bool chained = false;
      const int64_t slot = (2 * (int64_t)blockIdx.x + (w.first ? 1 : 0)) * MT + m;
      float4* aside = p.part + slot * (DT / 4 * 128) + tl;
      auto o_ready = [&](uint32_t bit) {  // O of the tile before this one
        waits(sh.o_done[2 * m + ((g - 1) & 1)], ((g - 1) >> 1) & 1, bit);
        tc_fence_after();
      };
      auto set_aside = [&] {  // O joins what was set aside before, and begins at 0
        o_ready(1u);
        const float f = ex2(m_aside - mx);
#pragma unroll 1
        for (int d = 0; d < D; d += 16) {
          uint32_t v[16];
          tmem_load<16>(o_col + d, v);
          tmem_loaded<16>(v);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float4* a = aside + (d / 4 + e) * 128;
            float4 x = make_float4(__uint_as_float(v[4 * e]), __uint_as_float(v[4 * e + 1]),
                                   __uint_as_float(v[4 * e + 2]), __uint_as_float(v[4 * e + 3]));
            if (chained) {
              const float4 y = *a;
              x = make_float4(fmaf(f, y.x, x.x), fmaf(f, y.y, x.y), fmaf(f, y.z, x.z), fmaf(f, y.w, x.w));
            }
            *a = x;
          }
        }
        chained = true;
        m_aside = mx;
      };

      for (int it = 0; it < w.tiles; ++it, ++g) {
        const int buf = 2 * m + (int)(g & 1);
        const uint32_t scores = lanes + buf * TN;
        const bool begins = it % C::kChain == 0;
        if (it > 0 && begins) set_aside();
        waits(sh.s_full[buf], (g >> 1) & 1, 2u);
        tc_fence_after();
        const int j0 = w.s.from + (w.tile + w.tiles - 1 - it) * TN;
        const uint32_t* there = sh.there[g % kThere];
        bool whole = true;
#pragma unroll
        for (int k = 0; k < C::kWords; ++k) whole = whole && there[k] == kAll;
        const bool edge = p.window > 0 && j0 < w.s.first + w.s.c - p.window;  // some rows' windows begin behind j0
        // Rows may see different tokens, or, by a mask, none the only draft.
        const bool uneven = (edge || j0 + TN > w.s.first) && (w.s.c > 1 || (p.mask && !(sh.bits[0] & 1)));
        const bool masked = !whole || edge || j0 + TN > w.s.first;
        const bool general = masked || !plain;

        bool slow = false;
        const bool clear = p.box && !whole && m == 0;
        if (uneven || clear) {
          const uint32_t q = 2 * g + 1, place_v = q % C::kSlots, at = ring + place_v * C::kSlot + tl * 128;
          waits(sh.full[place_v], (q / C::kSlots) & 1, 4u);
          const bool mine = tl < TN, here = mine && (there[(tl & (TN - 1)) >> 5] >> (tl & 31)) & 1u;
          if (clear && mine && !here) {  // TMA brings whole boxes, with whatever lies between a page's tokens
#pragma unroll 4
            for (int u = 0; u < D / 8; ++u) sts128(at + (u >> 3) * C::kBlock + (((u & 7) ^ (tl & 7)) << 4), 0, 0, 0, 0);
            fence_proxy_async_smem();
          }
          if (uneven) {  // a NaN or an infinity in V, in a row that not all see?
            bool bad = false;
            constexpr uint32_t kExp = kFp4 ? 0x7C00u : 0x7F80u;
            // From the first row that not all see to the last that there is (of short rows few: 142 sequences of 2 tokens
            // with 32 key heads 122 us with the tile's other rows, 106 without; MixFP4 283 and 215).
            const int row0 = edge ? 0 : max(w.s.first - j0, 0), rows_v = min(TN, w.s.end - j0) - row0, units = D / 8;
#pragma unroll 2
            for (int x = tl; x < rows_v * units; x += 128) {
              const int y = x / units, u = x - y * units, row = row0 + y;
              const uint4 v =
                  lds128(ring + place_v * C::kSlot + row * 128 + (u >> 3) * C::kBlock + (((u & 7) ^ (row & 7)) << 4));
              const uint32_t z[4] = {v.x, v.y, v.z, v.w};
              bool odd = false;
#pragma unroll
              for (int e = 0; e < 4; ++e) odd = odd || (z[e] & kExp) == kExp || (z[e] & (kExp << 16)) == kExp << 16;
              bad = bad || (odd && ((there[row >> 5] >> (row & 31)) & 1u));
            }
            slow = bar_or(2 + m, 128, bad);
          }
        }
        if (!idle) {
          // Which of the 32 tokens from column `col` on the row sees, a bit each (of the tile's: the rest is 0).
          auto seen_of = [&](int col) -> uint32_t {
            const int a = j0 + col, x = w.s.first - a;
            const uint32_t have = there[col >> 5] >> (col & 31);
            uint32_t v = valid ? below(x) & ~below(low - a) : 0u;
            if (x <= 0)
              v |= x > -64 ? (uint32_t)(sees >> -x) : 0u;
            else if (x < 32)
              v |= (uint32_t)sees << x;
            return v & have;
          };
          // ---- the scores' maximum; scores that need more than a factor are put back as they are to be.  Where the row
          // has one step, it stays in registers.
          float top = -INFINITY;
          uint32_t v[PW];
          const int c_end = (step0 + steps) * CW;
          auto load = [&](int c) {
            tmem_load<PW>(scores + c, v);
            tmem_loaded<PW>(v);
          };
#pragma unroll 1
          for (int c = step0 * CW; c < c_end; c += PW) {
            load(c);
            if (!general) {
              float top2 = -INFINITY;  // two chains
#pragma unroll
              for (int e = 0; e < PW; e += 4) {
                top = max3f(top, __uint_as_float(v[e]), __uint_as_float(v[e + 1]));
                top2 = max3f(top2, __uint_as_float(v[e + 2]), __uint_as_float(v[e + 3]));
              }
              top = fmaxf(top, top2);
            } else {
              const int a = j0 + c;
              const u64 ff = pack2(fs, fs);
#pragma unroll
              for (int e = 0; e < PW; e += 2) {
                float x0, x1;
                unpack2(mul2(bits2(v[e], v[e + 1]), ff), x0, x1);
                v[e] = __float_as_uint(x0), v[e + 1] = __float_as_uint(x1);
              }
              if (p.softcap > 0.0f) {
#pragma unroll
                for (int e = 0; e < PW; e += 2) {
                  float x0 = __uint_as_float(v[e]), x1 = __uint_as_float(v[e + 1]);
                  tanh2(x0, x1);
                  v[e] = __float_as_uint(cap2 * x0), v[e + 1] = __float_as_uint(cap2 * x1);
                }
              }
              if (p.slopes) {
                if (a + PW <= w.s.first) {
                  const float far0 = (float)(place - a);
#pragma unroll
                  for (int e = 0; e < PW; ++e) {
                    v[e] = __float_as_uint(fmaf(slope, far0 - (float)e, __uint_as_float(v[e])));
                  }
                } else {
#pragma unroll
                  for (int e = 0; e < PW; ++e) {
                    const int j = a + e;
                    int far = place - j;
                    if (j >= w.s.first) far = place - w.s.first - depth[min(j - w.s.first, kMostDrafts - 1)];
                    v[e] = __float_as_uint(fmaf(slope, (float)far, __uint_as_float(v[e])));
                  }
                }
              }
              if (masked) {
                const uint32_t seen = seen_of(c);
#pragma unroll
                for (int e = 0; e < PW; ++e) {
                  v[e] = (seen >> e) & 1u ? v[e] : __float_as_uint(-INFINITY);
                }
              }
              float top2 = -INFINITY;
#pragma unroll
              for (int e = 0; e < PW; e += 4) {
                top = max3f(top, __uint_as_float(v[e]), __uint_as_float(v[e + 1]));
                top2 = max3f(top2, __uint_as_float(v[e + 2]), __uint_as_float(v[e + 3]));
              }
              top = fmaxf(top, top2);
              if (c_end - step0 * CW > PW || slow) tmem_store<PW>(scores + c, v);
            }
          }
          if (general)
            tmem_st_wait();
          else
            top *= fs;
          const float f = general ? 1.0f : fs;
          if (__any_sync(kAll, top > mx + (kFp4 ? kFp4Slack : kSlack))) {
            const float v = fminf(fmaxf(mx, top), kMostScore), cor = ex2(mx - v);  // 0 at the first score
            mx = v;
            l *= cor;
            if (!begins) {
              o_ready(8u);
#pragma unroll 1
              for (int d = 0; d < D; d += 32) {  // columns behind D are nobody's
                uint32_t o[32];
                tmem_load<32>(o_col + d, o);
                tmem_loaded<32>(o);
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * cor);
                tmem_store<32>(o_col + d, o);
              }
              tmem_st_wait();
            }
          }

          // ---- the weights
          const float less = (kFp4 ? kFp4Exp : 0.0f) - mx;
          if (!slow) {
            const u64 ff = pack2(f, f), ll = pack2(less, less), tiny = pack2(0x1p-30f, 0x1p-30f);
            u64 sum[2] = {0ull, 0ull};
#pragma unroll 1
            for (int c = step0 * CW; c < c_end; c += PW) {
              if (c_end - step0 * CW > PW) load(c);
              uint32_t out[kFp4 ? PW / 2 : PW];
#pragma unroll
              for (int e = 0; e < PW; e += 2) {
                float x0, x1;
                unpack2(fma2(bits2(v[e], v[e + 1]), ff, ll), x0, x1);
                const float w0 = ex2(x0), w1 = ex2(x1);
                const u64 ww = pack2(w0, w1);
                sum[e / 2 & 1] = add2(sum[e / 2 & 1], ww);
                if (kFp4) {
                  out[e / 2] = f16x2(w0, w1);
                } else {
                  // The upper part by truncation, so that the lower is not negative; 2^-30 of the weight on top, so that
                  // it is not 0 either: times an infinite element of V both give its infinity.
                  const u64 up = bits2(__float_as_uint(w0) & 0xFFFF0000u, __float_as_uint(w1) & 0xFFFF0000u);
                  float l0, l1;
                  unpack2(fma2(ww, tiny, sub2(ww, up)), l0, l1);
                  const int at = e / CW * CW + e % CW / 2;  // the upper parts of a quarter, then its lower ones
                  out[at] = prmt(__float_as_uint(w0), __float_as_uint(w1), 0x7632u);
                  out[at + CW / 2] = bf16x2(l0, l1);
                }
              }
              if constexpr (kFp4) {
                tmem_store<CW / 2>(scores + c, out);
                if constexpr (PW > CW) tmem_store<CW / 2>(scores + c + CW, out + CW / 2);
              } else {
                tmem_store<PW>(scores + c, out);
              }
            }
            float s0, s1;
            unpack2(add2(sum[0], sum[1]), s0, s1);
            l += s0 + s1;
          } else {
            // Products of what the row sees alone.
            const uint32_t v_smem = ring + (2 * g + 1) % C::kSlots * C::kSlot;
            if (!begins) o_ready(16u);
            float sum = 0.0f;
#pragma unroll 1
            for (int d = 0; d < D; d += 16) {
              uint32_t o[16];
              if (!begins) {
                tmem_load<16>(o_col + d, o);
                tmem_loaded<16>(o);
              } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = 0u;
              }
#pragma unroll 1
              for (int k = 0; k < steps * CW; ++k) {
                const int col = step0 * CW + k;
                uint32_t xs;
                tmem_ld1(scores + col, xs);
                const float x = fmaf(__uint_as_float(xs), f, less), wt = ex2(x);
                if (d == 0) sum += wt;
                const bool mine = seen_of(col) & 1u;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                  const uint4 v = lds128(v_smem + (d >> 6) * C::kBlock + col * 128 +
                                         ((((d >> 3) & 7) + u) ^ (col & 7)) * 16);
                  const uint32_t y[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                  for (int e = 0; e < 4; ++e) {
                    float a0, a1;
                    if (kFp4)
                      f16x2_to_f32(y[e], a0, a1);
                    else
                      a0 = bf_lo(y[e]), a1 = bf_hi(y[e]);
                    const float b0 = __uint_as_float(o[8 * u + 2 * e]), b1 = __uint_as_float(o[8 * u + 2 * e + 1]);
                    o[8 * u + 2 * e] = __float_as_uint(mine ? fmaf(wt, a0, b0) : b0);
                    o[8 * u + 2 * e + 1] = __float_as_uint(mine ? fmaf(wt, a1, b1) : b1);
                  }
                }
              }
              tmem_store<16>(o_col + d, o);
            }
            l += sum;
          }
          tmem_st_wait();
        }
        if (tl == 0) sh.skip[buf] = slow;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh.p_full[buf]));
      }

      // ---- the part's end: O, m and l of every row, finished where the part is the whole row.  Copies of a row are added
      // up in shared memory.
      o_ready(32u);
      const bool all = w.first && w.last;
      float4* part = p.part + slot * (DT / 4 * 128);
      const int64_t at = ((int64_t)w.b * p.t + i) * p.q_heads + h;  // of the results
      const float old = chained ? ex2(m_aside - mx) : 0.0f;
      if (!valid) mx = kNoScore, l = 0.0f;
      float M = mx, L = l, part_of[4];  // what a copy's O counts
      if (copies > 1) {  // of one tile of rows
        float2* ml = reinterpret_cast<float2*>(smem);  // where the queries were: no product reads them any more
        ml[tl] = make_float2(mx, l);
        bar_sync(1, 128);
        float2 x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[k] = k < copies ? ml[tl % own + k * own] : make_float2(kNoScore, 0.0f);
          M = fmaxf(M, x[k].x);
        }
        L = 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          part_of[k] = ex2(x[k].x - M);
          L += part_of[k] * x[k].y;
        }
      }
      const float last = all ? out_factor<kFp4>(L, vts) : 1.0f;
      // Columns [d, d + 8) of the row's sum, in their own order from here on, to their place.
      auto put = [&](int d, const float* y) {
        if (!held || dead || d >= D) return;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[kFp4 ? fp4_order(e) : e] = valid ? y[e] * last : 0.0f;
        if (all) {
          *reinterpret_cast<uint4*>(p.out + at * D + d) =
              make_uint4(bf16x2(x[0], x[1]), bf16x2(x[2], x[3]), bf16x2(x[4], x[5]), bf16x2(x[6], x[7]));
        } else {
          float4* to = part + (d / 4) * 128 + tl % own;
          to[0] = make_float4(x[0], x[1], x[2], x[3]), to[128] = make_float4(x[4], x[5], x[6], x[7]);
        }
      };
      auto take = [&](int d, uint32_t* v) {  // 32 columns of O, with what was set aside
        tmem_load<32>(o_col + d, v);
        tmem_loaded<32>(v);
        if (chained) {
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            if (d + e >= D) break;
            const float4 y = aside[(d + e) * 32];
            auto more = [&](int k, float z) { v[e + k] = __float_as_uint(fmaf(old, z, __uint_as_float(v[e + k]))); };
            more(0, y.x), more(1, y.y), more(2, y.z), more(3, y.w);
          }
        }
      };
      if (copies == 1) {
        if (!idle)
#pragma unroll 1
          for (int d = 0; d < D; d += 32) {
            uint32_t v[32];
            take(d, v);
#pragma unroll
            for (int e = 0; e < 32; e += 8) put(d + e, reinterpret_cast<const float*>(v) + e);
          }
      } else {
        // 32 columns of all rows at a time, [row][8 pieces of 16 bytes] swizzled as the operands are, in two places in
        // turn (m and l were in the second's) where the queries' room allows.
        constexpr bool kTwo = C::kQ >= 32768;
        const int each = 32 / copies;
        if (!kTwo) bar_sync(1, 128);
#pragma unroll 1
        for (int d0 = 0; d0 < D; d0 += 32) {
          const uint32_t stage = q_smem + (kTwo && !(d0 & 32) ? 16384 : 0);
          {
            uint32_t v[32];
            take(d0, v);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              sts128(stage + tl * 128 + ((e ^ (tl & 7)) << 4), v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
          }
          bar_sync(1, 128);
#pragma unroll 1
          for (int d = copy * each; d < (copy + 1) * each; d += 8) {
            float x[8] = {};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              if (k >= copies) break;
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const uint4 v = lds128(stage + (tl % own + k * own) * 128 + (((d / 4 + u) ^ (tl & 7)) << 4));
                x[4 * u] = fmaf(part_of[k], __uint_as_float(v.x), x[4 * u]);
                x[4 * u + 1] = fmaf(part_of[k], __uint_as_float(v.y), x[4 * u + 1]);
                x[4 * u + 2] = fmaf(part_of[k], __uint_as_float(v.z), x[4 * u + 2]);
                x[4 * u + 3] = fmaf(part_of[k], __uint_as_float(v.w), x[4 * u + 3]);
              }
            }
            put(d0 + d, x);
          }
          if (!kTwo) bar_sync(1, 128);
        }
      }
      if (held && copy == 0 && !dead) {
        if (!all)
          p.stat[slot * 128 + tl] = make_float2(M, L);
        else if (p.lse)
          p.lse[at] = lse_of<kFp4>(M, L);
      }
      if (tid == 0 && w.first && !w.last)
        p.split[blockIdx.x] = make_int4(w.b, w.row, share, (int)((w.behind * sh.shares - 1) / sh.all));
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sh.heard));
      ++turn;
    }
  } else {
    if constexpr (C::kSoftRegs > C::kRegs) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kOtherRegs));
  if (warp == C::kSoftmax) {
    // ================================================= one thread issues the products
    if (elect_one()) {
      constexpr uint32_t kType = kFp4 ? 0u : (1u << 7) | (1u << 10);
      const uint32_t i_scores = (1u << 4) | kType | ((uint32_t)(TN >> 3) << 17) | (8u << 24);
      const uint32_t i_out = (1u << 4) | kType | (1u << 16) | ((uint32_t)(D >> 3) << 17) | (8u << 24);
      uint32_t g = 0, turn = 0;
      // S_m of tile number `tile`, into its buffer.
      auto scores = [&](uint32_t tile, int m) {
        const uint32_t q = 2 * tile, slot = q % C::kSlots;
        if (m == 0) {
          wait(sh.full[slot], (q / C::kSlots) & 1, 64u);
          if (!kFp4 && !p.box) fence_proxy_async_smem();  // of what cp.async has written
          tc_fence_after();
        }
        const int buf = 2 * m + (int)(tile & 1);
        const uint64_t a = smem_desc_sw128(q_smem + m * (128 * DT * 2)), b = smem_desc_sw128(ring + slot * C::kSlot);
#pragma unroll
        for (int k = 0; k < DT / 16; ++k) {
          if (16 * k >= D) break;
          mma_f16(tmem + buf * TN, a + ((k >> 2) * 16384 + (k & 3) * 32) / 16, b + ((k >> 2) * C::kBlock + (k & 3) * 32) / 16,
                  i_scores, k > 0);
        }
        mma_commit(smem_u32(&sh.s_full[buf]));
        if (m == MT - 1) mma_commit(smem_u32(&sh.empty[slot]));
      };
      while (walk.next(p, mate, w)) {
        wait(sh.q_full, turn & 1, 128u);
        ++turn;
        const int R = min(128 * MT, p.t * p.group - w.chunk * 128 * MT);
        const int copies = MT == 2 || R > 64 ? 1 : (R > 32 ? 2 : 4);
        tc_fence_after();
        // O_m += P_m V of tile g.
        auto weigh = [&](int it, int m) {
          const uint32_t q = 2 * g + 1, slot = q % C::kSlots;
          const int buf = 2 * m + (int)(g & 1);
          const bool begins = it % C::kChain == 0;  // O is at 0
          if (m == 0) {
            wait(sh.full[slot], (q / C::kSlots) & 1, 256u);
            if (!kFp4 && !p.box) fence_proxy_async_smem();
          }
          wait(sh.p_full[buf], (g >> 1) & 1, 512u);
          tc_fence_after();
          if (!*reinterpret_cast<volatile int*>(&sh.skip[buf])) {
            const uint64_t v = smem_desc_sw128_mn(ring + slot * C::kSlot, C::kBlock);
            const uint32_t o = tmem + C::kScoreCols + m * DT;
            // Not written out, as the softmax's queries are not, for the instruction caches' sake: MixFP4 at 8 drafts 187 us
            // with all of it unrolled, 185 so (and 192 one by one); at 64 drafts 454, 441 and 428.
            constexpr int kAtOnce = kFp4 && MT == 2 ? 1 : 2;
#pragma unroll kAtOnce
            for (int k = 0; k < TN / 16; ++k) {
              const uint32_t a = tmem + buf * TN + (k * 16 / CW) * CW + (k * 16 % CW) / 2;
              // A copy's tokens go to its lanes of O alone; the first of them begin it.
              const int copy = k * copies * 16 / TN;
              const bool first = begins && k * 16 % (TN / copies) == 0;
              auto off = [&](int quarter) { return quarter / (4 / copies) == copy ? 0u : kAll; };
              const uint4 lanes = make_uint4(off(0), off(1), off(2), off(3));
              mma_f16_tmem_a_lanes(o, a, v + k * 128, i_out, !first, lanes);
              if (!kFp4) mma_f16_tmem_a_lanes(o, a + CW / 2, v + k * 128, i_out, 1u, lanes);
            }
          }
          mma_commit(smem_u32(&sh.o_done[buf]));
          if (m == MT - 1) mma_commit(smem_u32(&sh.empty[slot]));
        };
        // Products of different shapes have no order among themselves: scores wait until the weights whose place they
        // take have been used up, which with two tiles of rows in turn is while the other's products run.
        auto used_up = [&](uint32_t tile, int m) { wait(sh.o_done[2 * m + (tile & 1)], (tile >> 1) & 1, 1u << 17); };
        const int tiles = w.tiles;
        scores(g, 0);
        if (MT == 2) {
          scores(g, 1);
        }
        for (int it = 0; it < tiles; ++it, ++g) {
          if (MT == 1) {
            if (it + 1 < tiles) {
              if (it > 0) used_up(g - 1, 0);
              scores(g + 1, 0);
            }
            weigh(it, 0);
          } else {
            if (it + 1 < tiles) {
              if (it > 0) used_up(g - 1, 0);
              scores(g + 1, 0);
              if (it > 0) used_up(g - 1, 1);
              scores(g + 1, 1);
            }
            weigh(it, 0);
            weigh(it, 1);
          }
        }
      }
      mma_commit(smem_u32(&sh.end));
      mbar_wait(smem_u32(&sh.end), 0, nullptr, limit);
    }
  } else if (warp == C::kSoftmax + 3) {
    // ================================================= reads a part ahead for softmax, and asks for its queries
    uint32_t turn = 0;
    for (bool more = true; more; ++turn) {
      more = walk.next(p, mate, w);
      uint64_t bits[2] = {0, 0};
      if (more) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
          if (lane + 32 * k < w.s.c) bits[k] = bits_of(p, w.b, lane + 32 * k, w.s.c);
        const int R = min(128 * MT, p.t * p.group - w.chunk * 128 * MT), lines = (D * 2 + 127) / 128;
        for (int x = lane; x < R * lines; x += 32) {
          const int r = x / lines, idx = w.chunk * 128 * MT + r, i = idx / p.group;
          if (i < w.s.c)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(p.q + (int64_t)w.b * p.q_stride + (int64_t)i * p.q_token_stride +
                                                          (int64_t)(w.head * p.group + idx - i * p.group) * p.q_head_stride +
                                                          (x - r * lines) * 64));
        }
      }
      waits(sh.heard, (turn & 1) ^ 1, 1u << 14);
      if (dead) break;  // what softmax may still read stays
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        sh.bits[lane + 32 * k] = bits[k];
        sh.depth[lane + 32 * k] = (uint8_t)depth_of(bits[k], lane + 32 * k);
      }
      if (lane == 0) {
        if (!more) w.tiles = 0;
        sh.part = w;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sh.told));
    }
  } else if (!kFp4 && p.box && warp < C::kSoftmax + 3) {
    // ================================================= rows of a bf16 cache by TMA, boxes of one page, 64 dimensions
    // each: keys by one warp, values by another
    {
      const int kv = warp - C::kSoftmax - 1;
      const int boxes = TN / p.box, blocks = (D + 63) / 64;  // of a tile; at most 16 copies to its keys or values
      const int box = lane % boxes, block = lane / boxes;
      const bool mine = block < blocks;
      uint32_t g = 0;
      while (!dead && walk.next(p, mate, w)) {
        const int32_t* table = p.table + (int64_t)w.b * p.table_stride;
        auto page_of = [&](int tok) { return p.page_shift >= 0 ? tok >> p.page_shift : tok / p.c.page_size; };
        // Page of this lane's box of the tile.
        auto ask = [&](int it) -> int {
          const int tok = w.s.from + (w.tile + w.tiles - 1 - it) * TN + box * p.box;
          return mine && it < w.tiles && tok < w.s.end && tok + p.box > w.s.low ? table[page_of(tok)] : -1;
        };
        int page = ask(0);
#pragma unroll 1
        for (int it = 0; it < w.tiles && !dead; ++it, ++g) {
          const int j0 = w.s.from + (w.tile + w.tiles - 1 - it) * TN, tok = j0 + box * p.box;
          const bool ok = page >= 0 && page < p.c.pages;
          const int from = page, row = tok - page_of(tok) * p.c.page_size;
          page = ask(it + 1);
          const uint32_t good = __ballot_sync(kAll, ok);  // bit i: box i % boxes
          if (kv == 0 && lane < TN / 32) {
            sh.there[g % kThere][lane] = there_of(p, w.s, j0 + lane * 32, lane * 32, good);
          }
          const uint32_t bytes = __popc(good) * p.box * 128;
          __syncwarp();
          const uint32_t q = 2 * g + kv, slot = q % C::kSlots, bar = smem_u32(&sh.full[slot]);
          wait(sh.empty[slot], ((q / C::kSlots) & 1) ^ 1, 1024u);
          dead = __any_sync(kAll, dead || *abort_flag);
          if (dead) break;
          if (kWithheld && q == 0) continue;
          if (lane == 0) mbar_arrive_expect_tx(bar, bytes);
          __syncwarp();
          if (ok)
            tma_load_4d(ring + slot * C::kSlot + block * C::kBlock + box * p.box * 128, &tm.rows[kv], block * 64, row,
                        w.head, from, bar);
          __syncwarp();
        }
      }
      // The copies in flight land before the CTA ends, also where those who would have waited for them have given up: the
      // last use of each slot.
      for (uint32_t q = 2 * g > C::kSlots ? 2 * g - C::kSlots : 0; q < 2 * g; ++q)
        if ((int)(q & 1) == kv)
          mbar_wait(smem_u32(&sh.full[q % C::kSlots]), (q / C::kSlots) & 1, nullptr, limit);
    }
  } else if (!kFp4) {
    // ================================================= or by cp.async, row by row, by two warps
    if constexpr (!kFp4) {
      const int pw = warp - C::kSoftmax - 1;
      constexpr int kRows = C::kRows, kPieces = DT / 8, kRowsAtOnce = 32 / kPieces;
      const int piece = lane % kPieces, r0 = lane / kPieces;
      uint32_t g = 0, q = 0;
      while (!dead && walk.next(p, mate, w)) {
        const int32_t* table = p.table + (int64_t)w.b * p.table_stride;
#pragma unroll 1
        for (int it = 0; it < w.tiles && !dead; ++it, ++g) {
          const int tok0 = w.s.from + (w.tile + w.tiles - 1 - it) * TN + pw * kRows;
          int64_t at[kRows / 32];  // of tokens lane, lane + 32; < 0: not there
#pragma unroll
          for (int j = 0; j < kRows / 32; ++j) {
            const int tok = tok0 + 32 * j + lane, in_page = tok / p.c.page_size;
            int page = -1;
            if (tok >= w.s.low && tok < w.s.end) page = table[in_page];
            const bool ok = page >= 0 && page < p.c.pages;
            at[j] = -1;
            if (ok)
              at[j] = 2 * ((int64_t)page * p.c.page_stride + (int64_t)(tok - in_page * p.c.page_size) * p.c.token_stride +
                           (int64_t)w.head * p.c.head_stride);
            const uint32_t there = __ballot_sync(kAll, ok);
            if (lane == 0) sh.there[g % kThere][pw * (kRows / 32) + j] = there;
          }
#pragma unroll 1
          for (int kv = 0; kv < 2; ++kv, ++q) {
            const uint8_t* base = static_cast<const uint8_t*>(kv ? p.c.v : p.c.k);
            const uint32_t slot = q % C::kSlots;
            waits(sh.empty[slot], ((q / C::kSlots) & 1) ^ 1, 1024u);
            if (dead) break;
            if (kWithheld && q == 0) continue;
            const uint32_t dst = ring + slot * C::kSlot + (piece >> 3) * C::kBlock + pw * kRows * 128;
#pragma unroll
            for (int j = 0; j < kRows / 32; ++j)
#pragma unroll 4
              for (int k = 0; k < 32 / kRowsAtOnce; ++k) {
                const int r = r0 + k * kRowsAtOnce, row = 32 * j + r;
                const int64_t from = __shfl_sync(kAll, at[j], r);
                const bool take = from >= 0 && piece * 8 < D;
                cp_async<16>(dst + row * 128 + (((piece & 7) ^ (row & 7)) << 4), base + (take ? from + piece * 16 : 0), take);
              }
            cp_async_arrive(smem_u32(&sh.full[slot]));  // when this lane's have landed
          }
        }
      }
      cp_async_wait_all();
    }
  } else if (warp < C::kSoftmax + 4) {
    // ================================================= helpers of a MixFP4 cache's producers, every other tile each
    if constexpr (kFp4) {
      const int me = warp - C::kSoftmax - 1;
      uint32_t g = 0, asked = 0;  // tiles, and behind the last that this warp has asked for by TMA
      // Boxes of this lane: keys' and values' codes, then their scale bytes.
      const int boxes = p.box ? TN / p.box : 1, box = lane % boxes, what = lane / boxes;
      const int box_pitch = (p.box * p.scale_pitch + 127) / 128 * 128;
      while (!dead && walk.next(p, mate, w)) {
        const int32_t* table = p.table + (int64_t)w.b * p.table_stride;
        auto page_of = [&](int tok) { return p.page_shift >= 0 ? tok >> p.page_shift : tok / p.c.page_size; };
#pragma unroll 1
        for (int it = 0; it < w.tiles; ++it, ++g) {
          if ((int)(g & 1) != me) continue;
          const int j0 = w.s.from + (w.tile + w.tiles - 1 - it) * TN;
          if (p.box) {
            const int tok = j0 + box * p.box, in_table = page_of(tok);
            const int page = tok < w.s.end && tok + p.box > w.s.low ? table[in_table] : -1;
            const bool here = page >= 0 && page < p.c.pages, ok = here && what < 4;
            const uint32_t good = __ballot_sync(kAll, here), n = g % C::kRawDepth, bar = smem_u32(&sh.raw_full[n]);
            if (lane < TN / 32) sh.there[g % kThere][lane] = there_of(p, w.s, j0 + lane * 32, lane * 32, good);
            __syncwarp();
            wait(sh.raw_empty[n], ((g / C::kRawDepth) & 1) ^ 1, 1u << 18);
            dead = __any_sync(kAll, dead || *abort_flag);
            if (dead) break;
            asked = g + 1;
            if (kWithheld && g == 0) continue;
            const int bytes = what < 2 ? p.box * (D / 2) : (p.scale_by_head ? p.box * 16 : p.box * (D / 16));
            const int all = __reduce_add_sync(kAll, ok ? bytes : 0);
            if (lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)all);
            __syncwarp();
            if (ok) {
              const int row = tok - in_table * p.c.page_size, kv = what & 1;
              const uint32_t to = raw_tiles + n * C::kRawTile, byte_to = to + 2 * C::kCodes + kv * TN * 16 + box * box_pitch;
              if (what < 2)
                tma_load_4d(to + kv * C::kCodes + box * p.box * (D / 2), &tm.rows[kv], 0, row, w.head, page, bar);
              else if (p.scale_by_head)
                tma_load_4d(byte_to, &tm.scales[kv], w.head * (D / 16) & ~15, row, 0, page, bar);
              else
                tma_load_4d(byte_to, &tm.scales[kv], D == 256 ? 2 * row : row, 0, w.head, page, bar);
            }
            __syncwarp();
          } else {  // where each row lies
            const uint32_t at = places + (g % C::kAddresses) * (TN * 16);
            int page[TN / 32];
#pragma unroll
            for (int j = 0; j < TN / 32; ++j) {
              const int tok = j0 + 32 * j + lane;
              page[j] = tok >= w.s.low && tok < w.s.end ? table[page_of(tok)] : -1;
            }
            waits(sh.used[g % C::kAddresses], ((g / C::kAddresses) & 1) ^ 1, 2048u);
            if (dead) break;
            if (kWithheld && g == 0) continue;
#pragma unroll
            for (int j = 0; j < TN / 32; ++j) {
              const int tok = j0 + 32 * j + lane, off = tok - page_of(tok) * p.c.page_size;
              const bool ok = page[j] >= 0 && page[j] < p.c.pages;
              int64_t x = -1, y = 0;
              if (ok) {
                x = (int64_t)page[j] * p.c.page_stride + (int64_t)off * p.c.token_stride + (int64_t)w.head * p.c.head_stride;
                y = (int64_t)page[j] * p.c.scale_page_stride + (int64_t)off * p.c.scale_token_stride +
                    (int64_t)w.head * p.c.scale_head_stride;
              }
              sts128(at + (32 * j + lane) * 16, (uint32_t)x, (uint32_t)(x >> 32), (uint32_t)y, (uint32_t)(y >> 32));
              const uint32_t there = __ballot_sync(kAll, ok);
              if (lane == 0) sh.there[g % kThere][j] = there;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.placed[g % C::kAddresses]));
          }
        }
      }
      // The copies in flight land before the CTA ends, as above.
      const uint32_t end = !p.box ? 0 : (dead ? asked : g);
      for (uint32_t n = end > C::kRawDepth ? end - C::kRawDepth : 0; n < end; ++n)
        if ((int)(n & 1) == me)
          mbar_wait(smem_u32(&sh.raw_full[n % C::kRawDepth]), (n / C::kRawDepth) & 1, nullptr, limit);
    }
  } else if constexpr (kFp4) {
    // ================================================= producers of a MixFP4 cache: codes in, f16 out
    const int pw = warp - C::kSoftmax - 4;
    using L = Lanes<DT>;
    const int piece = L::piece(lane), r0 = L::row(lane);
    constexpr int kRows = C::kRows, kSteps = kRows / L::kRowsAtOnce;
    const int row0 = pw * kRows, pitch = p.box ? D / 2 : DT / 2;  // rows of codes lie as TMA puts them, or apart
    uint32_t g = 0, sent = 0;  // tiles asked for, tiles decoded
    // The oldest tile not decoded yet, with `later` behind it: once it has landed, for the tensor cores.
    const int box_shift = p.box ? __ffs(p.box) - 1 : 31, box_pitch = (p.box * p.scale_pitch + 127) / 128 * 128;
    int scales[kSteps], at_slot[kSteps];  // where a row's scale byte lies, and its elements
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const int r = row0 + r0 + j * L::kRowsAtOnce;
      scales[j] = p.box ? (r >> box_shift) * box_pitch + (r & (p.box - 1)) * p.scale_pitch : r * 16;
      at_slot[j] = (piece >> 2) * C::kBlock + r * 128 + ((((piece & 3) * 2) ^ (r & 7)) << 4);
    }
    auto hand_over = [&](int later) {
      const uint32_t n = sent % C::kRawDepth, raw = raw_tiles + n * C::kRawTile;
      if (p.box)
        wait(sh.raw_full[n], (sent / C::kRawDepth) & 1, 1u << 19);
      else
        cp_wait_at_most(later), __syncwarp();
      dead = __any_sync(kAll, dead);
      const uint32_t bytes = raw + 2 * C::kCodes + piece + (p.box && p.scale_by_head ? w.head * (D / 16) & 15 : 0);
#pragma unroll 1  // one copy of the code: the instruction caches are shared by all roles (215 us written out, 185 so)
      for (int kv = 0; kv < 2; ++kv) {
        const uint32_t q = 2 * sent + kv, slot = q % C::kSlots;
        Codes<kSteps> c;
        if (piece * 16 < D)
          c.load(raw + kv * C::kCodes + (row0 + r0) * pitch + piece * 8, L::kRowsAtOnce * pitch, bytes + kv * TN * 16,
                 scales);
        waits(sh.empty[slot], ((q / C::kSlots) & 1) ^ 1, 1024u);
        if (piece * 16 < D) c.decode(ring + slot * C::kSlot, at_slot);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh.full[slot]));
      }
      if (p.box && lane == 0) mbar_arrive(smem_u32(&sh.raw_empty[n]));
      ++sent;
    };
    // Rows of an odd number of scale bytes (or of pairs): a lane to a byte, asked for with a tile's codes and put in place
    // before the next tile's are, so that no warp waits for them (80 dimensions 744 us, and 740 where they do: the other
    // warps cover that; 128 dimensions, whose loop this is too, 185 and 188).
    constexpr int kMost = (2 * kRows * 15 + 31) / 32;
    uint32_t odd[kMost] = {}, odd_at = 0;  // of a tile, and where its rows' bytes go; 0: none
    auto each_byte = [&](auto&& f) {  // f(k, row, keys or values, byte)
      const int bytes = D / 16, rows_on = 32 / bytes, bytes_on = 32 - rows_on * bytes;
      int y = lane / bytes, e = lane - y * bytes;
#pragma unroll
      for (int k = 0; k < kMost; ++k) {
        if (32 * k >= 2 * kRows * bytes) break;
        if (y < 2 * kRows) f(k, y & (kRows - 1), y / kRows, e);
        y += rows_on, e += bytes_on;
        if (e >= bytes) e -= bytes, ++y;
      }
    };
    auto put_bytes = [&] {
      if (odd_at) each_byte([&](int k, int r, int kv, int e) { sts8(odd_at + (kv * TN + r) * 16 + e, odd[k]); });
      odd_at = 0;
    };
    while (walk.next(p, mate, w)) {
#pragma unroll 1
      for (int it = 0; it < w.tiles; ++it, ++g) {
        if (p.box) {
          hand_over(0);
          continue;
        }
        waits(sh.placed[g % C::kAddresses], (g / C::kAddresses) & 1, 4096u);
        if (dead) break;
        const uint32_t at = places + (g % C::kAddresses) * (TN * 16) + row0 * 16;
        const uint32_t raw = raw_tiles + (g % C::kRawDepth) * C::kRawTile, bytes_at = raw + 2 * C::kCodes + row0 * 16;
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
          const int r = r0 + j * L::kRowsAtOnce;
          const uint2 x = lds64(at + r * 16);
          const bool take = (int32_t)x.y >= 0 && piece * 16 < D;
          const int64_t from = take ? (int64_t)((u64)x.x | (u64)x.y << 32) + piece * 8 : 0;
          const uint32_t to = raw + (row0 + r) * pitch + piece * 8;
          cp_async<8>(to, static_cast<const uint8_t*>(p.c.k) + from, take);
          cp_async<8>(to + C::kCodes, static_cast<const uint8_t*>(p.c.v) + from, take);
        }
        if (D % 64 == 0) {  // scale bytes: some lanes the keys' rows, as many the values'
          const int r = lane & (kRows - 1), kv = lane / kRows;
          if (kv < 2) {
            const uint4 x = lds128(at + r * 16);
            const bool ok = (int32_t)x.y >= 0;
            const uint8_t* src = (kv ? p.c.v_scales : p.c.k_scales) + (ok ? (int64_t)((u64)x.z | (u64)x.w << 32) : 0);
            const uint32_t sd = bytes_at + (kv * TN + r) * 16;
            if (D == 128) {
              cp_async<8>(sd, src, ok);
            } else if (D == 256) {
              cp_async<16>(sd, src, ok);
            } else {
              for (int k = 0; k < D / 16; k += 4) cp_async<4>(sd + k, src + k, ok);
            }
          }
        } else {
          put_bytes();
          each_byte([&](int k, int r, int kv, int e) {
            const uint4 z = lds128(at + r * 16);
            odd[k] = 0u;
            if ((int32_t)z.y >= 0) odd[k] = (kv ? p.c.v_scales : p.c.k_scales)[(int64_t)((u64)z.z | (u64)z.w << 32) + e];
          });
          odd_at = bytes_at;
        }
        cp_commit();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh.used[g % C::kAddresses]));
        if (g - sent >= C::kRawDepth - 1) hand_over(C::kRawDepth - 1);
      }
    }
    put_bytes();
    while (sent < g) hand_over((int)(g - sent - 1));
    cp_async_wait_all();
  }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == C::kSoftmax) {
    tc_fence_after();
    tmem_dealloc(tmem, C::kCols);
  }
}

// Joins the parts of the row that CTA blockIdx.x began: a thread to four dimensions of a query row.
template <int DT, int MT, bool kFp4>
__global__ void __launch_bounds__(kJoinThreads) tree_attention_join_kernel(const TreeArgs p) {
  griddep_wait();
  const int4 s = p.split[blockIdx.x];
  if (s.x < 0) return;
  const int mate = (int)blockIdx.x % p.together, chunk = s.y % p.chunks, head = s.y / p.chunks * p.together + mate;
  const int R = min(128 * MT, p.t * p.group - chunk * 128 * MT), D = p.c.head_dim;
  const int x = (int)blockIdx.y * kJoinThreads + (int)threadIdx.x, r = x % R, d4 = x / R;
  if (d4 >= D / 4) return;
  auto slot = [&](int k) {
    return (2 * ((int64_t)k * p.together + mate) + (k == s.z ? 1 : 0)) * MT + (r >> 7);
  };
  float M = kNoScore, L = 0.0f;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  constexpr int kAtOnce = 4;  // parts asked for at once, with their (m, l)
  for (int k0 = s.z; k0 <= s.w; k0 += kAtOnce) {
    float2 st[kAtOnce];
    float4 v[kAtOnce];
#pragma unroll
    for (int a = 0; a < kAtOnce; ++a) {
      st[a] = make_float2(kNoScore, 0.0f), v[a] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (k0 + a <= s.w) {
        st[a] = p.stat[slot(k0 + a) * 128 + (r & 127)];
        v[a] = p.part[slot(k0 + a) * (DT / 4 * 128) + d4 * 128 + (r & 127)];
      }
    }
    float top = M;
#pragma unroll
    for (int a = 0; a < kAtOnce; ++a) top = fmaxf(top, st[a].x);
    const float old = ex2(M - top);
    M = top;
    L *= old;
    o.x *= old, o.y *= old, o.z *= old, o.w *= old;
#pragma unroll
    for (int a = 0; a < kAtOnce; ++a) {
      const float f = ex2(st[a].x - M);
      L += f * st[a].y;
      o.x = fmaf(f, v[a].x, o.x), o.y = fmaf(f, v[a].y, o.y);
      o.z = fmaf(f, v[a].z, o.z), o.w = fmaf(f, v[a].w, o.w);
    }
  }
  const int idx = chunk * 128 * MT + r, i = idx / p.group, h = head * p.group + idx - i * p.group;
  const int64_t at = ((int64_t)s.x * p.t + i) * p.q_heads + h;
  const float f = out_factor<kFp4>(L, kFp4 ? *p.c.v_ts : 1.0f);
  *reinterpret_cast<uint2*>(p.out + at * D + d4 * 4) = make_uint2(bf16x2(o.x * f, o.y * f), bf16x2(o.z * f, o.w * f));
  if (d4 == 0 && p.lse) p.lse[at] = lse_of<kFp4>(M, L);
}

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline int launch_status() { return cudaGetLastError() == cudaSuccess ? MIXFP4_OK : MIXFP4_ERR_CUDA; }

inline int padded_dim(int D) { return D <= 64 ? 64 : (D <= 128 ? 128 : 256); }
// Tiles of 128 rows that share the tokens.
inline int row_tiles(const mixfp4_kv_cache* c, int64_t t, int64_t q_heads) {
  return c->head_dim <= 128 && t * (q_heads / c->heads) > 128 ? 2 : 1;
}
inline int tile_tokens(const mixfp4_kv_cache* c, int tiles) {
  return c->head_dim <= 128 && tiles == 1 && c->dtype == MIXFP4_CACHE_MIXFP4 ? 128 : 64;
}
// Key heads whose CTAs walk over the same tokens at the same time.
inline int together_of(const mixfp4_kv_cache* c) {
  for (int n = 8; n > 1; n /= 2)
    if (c->heads % n == 0) return n;
  return 1;
}
inline int grid_of(const mixfp4_kv_cache* c, int tiles) {
  const int ctas = num_sms() * (tiles == 1 && c->head_dim <= 128 && c->dtype == MIXFP4_CACHE_BF16 ? 2 : 1);
  return ctas / together_of(c) * together_of(c);
}

// Whether scale bytes of neighbouring heads, or of a head's neighbouring tokens, lie together and at multiples of 16
// bytes: TMA brings no less than 16, from such an address on.
inline bool scales_by_head(const mixfp4_kv_cache& c) {
  const int64_t n = c.head_dim / 16;
  return 16 % n == 0 && c.heads * n % 16 == 0 && (c.scale_head_stride == n || c.heads == 1) &&
         (c.scale_token_stride | c.scale_page_stride) % 16 == 0 && aligned(c.k_scales, 16) && aligned(c.v_scales, 16);
}
inline bool scales_by_token(const mixfp4_kv_cache& c) {
  const int64_t n = c.head_dim / 16;
  return 16 % n == 0 && c.scale_token_stride == n && (c.scale_head_stride | c.scale_page_stride) % 16 == 0 &&
         aligned(c.k_scales, 16) && aligned(c.v_scales, 16);
}
// Rows that one TMA copy brings (bf16 at 8 drafts 179 us, by cp.async 216; MixFP4 185 and 268): of one page, and a part
// of a tile; 0 where TMA's rules do not allow it (pages of no multiple of 16 tokens, rows of codes that are no multiple of
// 16 bytes or lie on none) or bf16 rows of less than 64 elements would not fill the operand's.
inline int box_of(const mixfp4_kv_cache& c, int tokens) {
  const bool fp4 = c.dtype == MIXFP4_CACHE_MIXFP4;
  if (c.page_size % 16 != 0 || c.pages == 0 || (fp4 ? c.head_dim % 32 != 0 : c.head_dim < 64)) return 0;
  if (fp4 && (!aligned(c.k, 16) || !aligned(c.v, 16) || (c.token_stride | c.head_stride | c.page_stride) % 16 ||
              (!scales_by_head(c) && !scales_by_token(c))))
    return 0;
  int n = 16;
  while (n < tokens && c.page_size % (2 * n) == 0) n *= 2;
  return n;
}
// Boxes of 64 elements of bf16 rows, swizzled as the operands are, or whole rows of codes as they lie.
inline bool make_map_rows(CUtensorMap* m, const void* base, const mixfp4_kv_cache& c, int box) {
  auto fn = encode_fn();
  if (!fn) return false;
  const bool fp4 = c.dtype == MIXFP4_CACHE_MIXFP4;
  const int row = fp4 ? c.head_dim / 2 : c.head_dim, esize = fp4 ? 1 : 2;
  // An axis of one element has any stride; 32 bytes will do.
  auto bytes = [&](int64_t stride, int64_t n) { return (cuuint64_t)(n > 1 ? stride * esize : 32); };
  cuuint64_t dims[4] = {(cuuint64_t)row, (cuuint64_t)c.page_size, (cuuint64_t)c.heads, (cuuint64_t)c.pages};
  cuuint64_t strides[3] = {bytes(c.token_stride, c.page_size), bytes(c.head_stride, c.heads), bytes(c.page_stride, c.pages)};
  cuuint32_t boxes[4] = {(cuuint32_t)(fp4 ? row : 64), (cuuint32_t)box, 1, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(m, fp4 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims,
            strides, boxes, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            fp4 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Boxes of 16 bytes of a token's scale bytes, or of `box` tokens' of a head.
inline bool make_map_scales(CUtensorMap* m, const void* base, const mixfp4_kv_cache& c, int box) {
  auto fn = encode_fn();
  if (!fn) return false;
  const int n = c.head_dim / 16;
  const bool by_head = scales_by_head(c);
  // Of a head's tokens, elements of 2 to 8 bytes: a box has at most 256 of them along an axis.
  const int per_token = by_head ? n : (n == 16 ? 2 : 1);
  const auto type = by_head  ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                    : n == 2 ? CU_TENSOR_MAP_DATA_TYPE_UINT16
                    : n == 4 ? CU_TENSOR_MAP_DATA_TYPE_INT32
                             : CU_TENSOR_MAP_DATA_TYPE_INT64;
  auto bytes = [](int64_t stride, int64_t count) { return (cuuint64_t)(count > 1 ? stride : 32); };
  cuuint64_t dims[4] = {(cuuint64_t)(by_head ? c.heads : c.page_size) * per_token, (cuuint64_t)(by_head ? c.page_size : 1),
                        (cuuint64_t)(by_head ? 1 : c.heads), (cuuint64_t)c.pages};
  cuuint64_t strides[3] = {bytes(c.scale_token_stride, (int64_t)dims[1]), bytes(c.scale_head_stride, (int64_t)dims[2]),
                           bytes(c.scale_page_stride, c.pages)};
  cuuint32_t boxes[4] = {(cuuint32_t)(by_head ? 16 : box * per_token), (cuuint32_t)(by_head ? box : 1), 1, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(m, type, 4, const_cast<void*>(base), dims, strides, boxes, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DT, int MT, bool kFp4, bool kWithheld = false>
int launch(TreeArgs p, int grid, cudaStream_t s) {
  using C = Cfg<DT, MT, kFp4>;
  Maps maps = {};
  p.box = box_of(p.c, C::kTokens);
  if (p.box && kFp4) p.scale_by_head = scales_by_head(p.c), p.scale_pitch = p.scale_by_head ? 16 : p.c.head_dim / 16;
  if (p.box && !(make_map_rows(&maps.rows[0], p.c.k, p.c, p.box) && make_map_rows(&maps.rows[1], p.c.v, p.c, p.box) &&
                 (!kFp4 || (make_map_scales(&maps.scales[0], p.c.k_scales, p.c, p.box) &&
                            make_map_scales(&maps.scales[1], p.c.v_scales, p.c, p.box)))))
    p.box = 0;
  static std::atomic<uint64_t> done{0};
  auto* kernel = tree_attention_kernel<DT, MT, kFp4, kWithheld>;
  if (!set_dynamic_smem_once(reinterpret_cast<const void*>(kernel), C::kSmem, done)) return MIXFP4_ERR_CUDA;
  kernel<<<grid, C::kThreads, C::kSmem, s>>>(p, maps);
  if (int st = launch_status()) return st;
  if (!p.joined) return MIXFP4_OK;
  const int rows = p.t * p.group < 128 * MT ? p.t * p.group : 128 * MT;
  const dim3 jg((unsigned)grid, (unsigned)((rows * (p.c.head_dim / 4) + kJoinThreads - 1) / kJoinThreads));
  return launch_pdl(tree_attention_join_kernel<DT, MT, kFp4>, jg, dim3(kJoinThreads), 0, s, p) == cudaSuccess
             ? MIXFP4_OK
             : MIXFP4_ERR_CUDA;
}

template <bool kFp4>
int launch_dim(const TreeArgs& p, int grid, int tiles, cudaStream_t s) {
  if (p.wait_ns) return tiles == 2 ? launch<128, 2, kFp4, true>(p, grid, s) : launch<128, 1, kFp4, true>(p, grid, s);
  switch (padded_dim(p.c.head_dim)) {
    case 64: return tiles == 2 ? launch<64, 2, kFp4>(p, grid, s) : launch<64, 1, kFp4>(p, grid, s);
    case 128: return tiles == 2 ? launch<128, 2, kFp4>(p, grid, s) : launch<128, 1, kFp4>(p, grid, s);
    default: return launch<256, 1, kFp4>(p, grid, s);
  }
}

int tree_attention(const void* q, int64_t q_stride, int64_t q_token_stride, int64_t q_head_stride, int64_t B, int64_t t,
                   int64_t q_heads, const mixfp4_kv_cache* cache, const int32_t* block_table, int64_t table_stride,
                   int64_t table_pages, const int32_t* lengths, const int64_t* mask, int64_t mask_stride,
                   const int32_t* counts, float scale, int64_t window, float softcap, const float* slopes, void* out,
                   float* lse, void* workspace, int64_t workspace_bytes, uint32_t* status_word, uint64_t wait_ns,
                   void* stream) {
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
      !aligned(lse, 4) || !aligned(workspace, 256) || !aligned(status_word, 4))
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
  p.status = status_word;
  p.wait_ns = wait_ns;
  const int tiles = row_tiles(cache, t, q_heads), grid = grid_of(cache, tiles);
  const int64_t rows = t * p.group;
  if (rows > INT32_MAX - 256) return MIXFP4_ERR_SHAPE;
  p.chunks = (int)((rows + 128 * tiles - 1) / (128 * tiles));
  p.together = together_of(cache);
  p.shares = grid / p.together;
  p.joined = p.max_tokens > tile_tokens(cache, tiles);  // rows of one tile are never cut
  p.page_shift = -1;
  for (int i = 0; i < 31; ++i)
    if (cache->page_size == 1 << i) p.page_shift = i;
  uint8_t* w = static_cast<uint8_t*>(workspace);
  p.split = reinterpret_cast<int4*>(w);
  w += ((int64_t)grid * 16 + 255) / 256 * 256;
  p.stat = reinterpret_cast<float2*>(w);
  p.part = reinterpret_cast<float4*>(w + 2 * (int64_t)grid * 128 * tiles * 8);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (status_word && cudaMemsetAsync(status_word, 0, 4, s) != cudaSuccess) return MIXFP4_ERR_CUDA;
  return cache->dtype == MIXFP4_CACHE_MIXFP4 ? launch_dim<true>(p, grid, tiles, s) : launch_dim<false>(p, grid, tiles, s);
}

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
  const int tiles = row_tiles(cache, t, q_heads);
  const int64_t grid = grid_of(cache, tiles), rows = 128 * tiles;
  *bytes = (grid * 16 + 255) / 256 * 256 + 2 * grid * rows * (8 + padded_dim(cache->head_dim) * 4);
  return MIXFP4_OK;
}

int mixfp4_tree_attention(const void* q, int64_t q_stride, int64_t q_token_stride, int64_t q_head_stride, int64_t B,
                          int64_t t, int64_t q_heads, const mixfp4_kv_cache* cache, const int32_t* block_table,
                          int64_t table_stride, int64_t table_pages, const int32_t* lengths, const int64_t* mask,
                          int64_t mask_stride, const int32_t* counts, float scale, int64_t window, float softcap,
                          const float* slopes, void* out, float* lse, void* workspace, int64_t workspace_bytes,
                          uint32_t* status_word, void* stream) {
  return mixfp4::tree_attention(q, q_stride, q_token_stride, q_head_stride, B, t, q_heads, cache, block_table,
                                table_stride, table_pages, lengths, mask, mask_stride, counts, scale, window, softcap,
                                slopes, out, lse, workspace, workspace_bytes, status_word, 0, stream);
}

int mixfp4_selftest_tree_attention_missed_rows(const void* q, int64_t B, int64_t t, int64_t q_heads,
                                               const mixfp4_kv_cache* cache, const int32_t* block_table,
                                               int64_t table_pages, const int32_t* lengths, void* out, void* workspace,
                                               int64_t workspace_bytes, uint32_t* status_word, uint64_t limit_ns,
                                               void* stream) {
  if (B < 1 || t < 1 || q_heads < 1) return MIXFP4_ERR_SHAPE;
  if (limit_ns == 0 || limit_ns > 2000000000ull) return MIXFP4_ERR_ARG;
  if (!cache || !status_word) return MIXFP4_ERR_NULL;
  if (cache->head_dim <= 64 || cache->head_dim > 128) return MIXFP4_ERR_SHAPE;
  const int64_t row = q_heads * (int64_t)cache->head_dim;
  return mixfp4::tree_attention(q, t * row, row, cache->head_dim, B, t, q_heads, cache, block_table, table_pages,
                                table_pages, lengths, nullptr, 0, nullptr, 0.125f, 0, 0.0f, nullptr, out, nullptr,
                                workspace, workspace_bytes, status_word, limit_ns, stream);
}

}  // extern "C"
