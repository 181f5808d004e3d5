// Rows and pages of the paged key-value cache moved on the device: accepted
// drafts (mixfp4_kv_accept), branching sequences (mixfp4_kv_fork) and whole
// pages (mixfp4_kv_copy_pages).
//
// Bytes are read once and written once: 4099 pages of 64 KB move in 82 us, 0.96 of the
// rate of a plain copy; of 18 KB (MixFP4) in 54, 0.41: a CTA's share of one is a single
// piece a thread, and its scale bytes take a CTA of their own.  What is small is a wait for
// lengths and table, then one for the rows: 512 children of 256 sequences 10 us (MixFP4), 200
// sequences' accepted drafts 4.7 us, 256 sequences' 6.9 (512 CTAs of 150 registers, of which
// 456 run at once: a second round), 5 pages or 8 sequences 3 to 4 us.  A page is a set of runs of bytes that
// lie together: the whole page where it is dense in either order of tokens and
// heads, a token's heads or a head's tokens where only those are, else single head
// rows.  A CTA takes a share of one page's keys or values (or their scales), four
// pieces of up to 32 bytes a thread in flight.
#include <cuda_runtime.h>
#include <cstdint>

#include "host_util.cuh"
#include "kvcache.cuh"
#include "ptx.cuh"

namespace mixfp4 {
namespace {

constexpr int kThreads = 256;
constexpr int kInFlight = 4;
constexpr int kMoveThreads = 128;  // of mixfp4_kv_accept
constexpr int kMostDepth = 64;

// One of a cache's arrays (keys, values, their scales), in bytes.
struct Plane {
  uint8_t* base;
  int64_t page_stride, outer_stride, inner_stride;
  int outer, inner;   // runs of a page: outer x inner (tokens x heads, heads x 1 or 1 x 1)
  int run;            // bytes of a run; of one token's share of it where the runs hold tokens
  int by_token;       // 0: `outer` counts tokens; 1: a run holds them
  int piece;          // bytes of an access
};

struct Planes {
  Plane p[4];
  int count;
};

struct Bytes32 {
  uint32_t v[8];
};

template <int kBytes>
struct Piece;
template <>
struct Piece<32> {
  typedef Bytes32 type;
  static __device__ __forceinline__ type load(const uint8_t* p) {
    type t;
    ldg256_stream(p, t.v);
    return t;
  }
  static __device__ __forceinline__ void store(uint8_t* p, const type& t) { stg256(p, t.v); }
};
template <typename T>
struct Plain {
  typedef T type;
  static __device__ __forceinline__ T load(const uint8_t* p) { return *reinterpret_cast<const T*>(p); }
  static __device__ __forceinline__ void store(uint8_t* p, const T& t) { *reinterpret_cast<T*>(p) = t; }
};
template <>
struct Piece<16> : Plain<uint4> {};
template <>
struct Piece<8> : Plain<uint2> {};
template <>
struct Piece<4> : Plain<uint32_t> {};
template <>
struct Piece<1> : Plain<uint8_t> {};

// The first `tokens` places of page src to page dst: the share of slice `at` of `slices` of one plane.
template <int kBytes>
__device__ __forceinline__ void copy_share(const Plane& p, int src, int dst, int tokens, int at, int slices) {
  const int run = p.run * (p.by_token ? tokens : 1) / kBytes;  // pieces
  const int outer = p.by_token ? p.outer : tokens, total = run * outer * p.inner;
  const uint8_t* from = p.base + (int64_t)src * p.page_stride;
  uint8_t* to = p.base + (int64_t)dst * p.page_stride;
  for (int i0 = at * kThreads + (int)threadIdx.x; i0 < total; i0 += kInFlight * slices * kThreads) {
    typename Piece<kBytes>::type v[kInFlight];
    int64_t off[kInFlight];
#pragma unroll
    for (int j = 0; j < kInFlight; ++j) {
      const int i = i0 + j * slices * kThreads;
      if (i >= total) break;
      const int y = i / run, x = i - y * run, o = y / p.inner;
      off[j] = o * p.outer_stride + (y - o * p.inner) * p.inner_stride + (int64_t)x * kBytes;
      v[j] = Piece<kBytes>::load(from + off[j]);
    }
#pragma unroll
    for (int j = 0; j < kInFlight; ++j)
      if (i0 + j * slices * kThreads < total) Piece<kBytes>::store(to + off[j], v[j]);
  }
}
__device__ __forceinline__ void copy_page(const Planes& ps, int src, int dst, int tokens, int part, int slices) {
  const Plane& p = ps.p[part / slices];
  const int at = part % slices;
  switch (p.piece) {
    case 32: return copy_share<32>(p, src, dst, tokens, at, slices);
    case 16: return copy_share<16>(p, src, dst, tokens, at, slices);
    case 8: return copy_share<8>(p, src, dst, tokens, at, slices);
    case 4: return copy_share<4>(p, src, dst, tokens, at, slices);
    default: return copy_share<1>(p, src, dst, tokens, at, slices);
  }
}

__global__ void __launch_bounds__(kThreads) kv_copy_pages_kernel(const Planes ps, int slices, int64_t pages, int tokens,
                                                                 const int32_t* src, const int32_t* dst) {
  const int s = src[blockIdx.x], d = dst[blockIdx.x];
  if (s < 0 || s >= pages || d < 0 || d >= pages || s == d) return;
  copy_page(ps, s, d, tokens, (int)blockIdx.y, slices);
}

struct ForkArgs {
  Planes ps;
  int slices, page_size;
  int64_t pages;
  const int32_t* table;
  int64_t table_stride;
  int table_pages;
  const int32_t* lengths;
  int64_t B;
  const int32_t *parents, *fresh;
  int32_t *table_out, *lengths_out;
};

// Child blockIdx.x: its table and length by the CTAs of row 0, its own page by the others.
__global__ void __launch_bounds__(kThreads) kv_fork_kernel(const ForkArgs a) {
  const int64_t i = blockIdx.x;
  const int parent = a.parents[i];
  const bool known = parent >= 0 && parent < a.B;
  const int n = known ? max(a.lengths[parent], 0) : 0;
  const int32_t* table = a.table + (known ? parent : 0) * a.table_stride;
  const int last = n / a.page_size, part = n - last * a.page_size;
  const int fresh = a.fresh[i];
  const bool own = part > 0 && last < a.table_pages && fresh >= 0 && fresh < a.pages;
  if (blockIdx.y == 0) {
    if (threadIdx.x == 0) a.lengths_out[i] = n;
    int32_t* out = a.table_out + i * a.table_pages;
    for (int j = threadIdx.x; j < a.table_pages; j += kThreads)
      out[j] = !known ? -1 : (own && j == last ? fresh : table[j]);
    return;
  }
  if (!own) return;
  const int src = table[last];
  if (src < 0 || src >= a.pages || src == fresh) return;
  copy_page(a.ps, src, fresh, part, (int)blockIdx.y - 1, a.slices);
}

struct AcceptArgs {
  mixfp4_kv_cache c;
  int esize;         // bytes to a stride's unit
  int piece, pieces; // of a head row's codes (or bf16 elements): bytes of an access, accesses
  int spiece, spieces;
  const int32_t* table;
  int64_t table_stride, max_tokens;
  const int32_t *lengths, *counts, *path;
  int64_t path_stride;
  int depth;
  int32_t* lengths_out;
};

// A thread's column, the same bytes of every row.  Where the path rises, as one from a root to a leaf does whose drafts
// come after their ancestors, no row is written before it has been read if rows go in order: draft path[k] >= k.  Eight at
// a time then wait for memory together.  Any other path is read as a whole first, into the thread's own memory.
template <int kBytes>
__device__ __forceinline__ void move_column(uint8_t* col, const int64_t* from, const int64_t* to, int n, bool rises) {
  typedef typename Piece<kBytes>::type T;
  if (rises) {
    constexpr int kBatch = 8;
#pragma unroll 1
    for (int k0 = 0; k0 < n; k0 += kBatch) {
      T v[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
        if (k0 + k < n && from[k0 + k] >= 0) v[k] = Piece<kBytes>::load(col + from[k0 + k]);
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
        if (k0 + k < n && from[k0 + k] >= 0) Piece<kBytes>::store(col + to[k0 + k], v[k]);
    }
  } else {
    T v[kMostDepth];
#pragma unroll 1
    for (int k = 0; k < n; ++k)
      if (from[k] >= 0) v[k] = Piece<kBytes>::load(col + from[k]);
#pragma unroll 1
    for (int k = 0; k < n; ++k)
      if (from[k] >= 0) Piece<kBytes>::store(col + to[k], v[k]);
  }
}
__device__ __forceinline__ void move_column(int bytes, uint8_t* col, const int64_t* from, const int64_t* to, int n,
                                            bool rises) {
  switch (bytes) {
    case 16: return move_column<16>(col, from, to, n, rises);
    case 8: return move_column<8>(col, from, to, n, rises);
    case 4: return move_column<4>(col, from, to, n, rises);
    default: return move_column<1>(col, from, to, n, rises);
  }
}

// A cluster of CTAs to a sequence; each thread moves whole columns, so no thread writes what another reads.
__global__ void __launch_bounds__(kMoveThreads) kv_accept_kernel(const AcceptArgs a) {
  // Offsets of the moved rows in the arrays and in the scales; from < 0: the row stays.
  __shared__ int64_t from[2][kMostDepth], to[2][kMostDepth];
  __shared__ int sh_path[kMostDepth];
  __shared__ int accepted, falls;  // the path's length; whether some entry is no more than the one before it
  uint32_t rank, ranks;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
  const int64_t b = blockIdx.x / ranks;
  const int tid = threadIdx.x;
  const int n = max(a.lengths[b], 0), c = min(max(a.counts[b], 0), n), first = n - c;
  if (tid == 0) accepted = a.depth, falls = 0;
  __syncthreads();
  if (tid < a.depth) {
    const int v = a.path[b * a.path_stride + tid];
    sh_path[tid] = v;
    if (v < 0 || v >= c) atomicMin(&accepted, tid);
  }
  __syncthreads();
  const int moved = accepted;
  if (tid < moved) {
    int64_t off[2][2];
    bool ok = sh_path[tid] != tid;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int64_t pos = (int64_t)first + (e == 0 ? sh_path[tid] : tid);
      off[e][0] = off[e][1] = -1;
      if (pos < a.max_tokens) {
        const int64_t page = a.table[b * a.table_stride + pos / a.c.page_size], at = pos % a.c.page_size;
        if (page >= 0 && page < a.c.pages) {
          off[e][0] = (page * a.c.page_stride + at * a.c.token_stride) * a.esize;
          off[e][1] = page * a.c.scale_page_stride + at * a.c.scale_token_stride;
        }
      }
      ok = ok && off[e][0] >= 0;
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) from[s][tid] = ok ? off[0][s] : -1, to[s][tid] = off[1][s];
    if (tid > 0 && sh_path[tid] <= sh_path[tid - 1]) falls = 1;
  }
  __syncthreads();
  const int row = a.pieces + a.spieces, columns = 2 * a.c.heads * row;
  for (int x = (int)rank * kMoveThreads + tid; x < columns; x += (int)ranks * kMoveThreads) {
    const int hv = x / row, piece = x - hv * row, h = hv >> 1;
    if (piece < a.pieces) {
      uint8_t* col = static_cast<uint8_t*>(hv & 1 ? a.c.v : a.c.k) + h * a.c.head_stride * a.esize + piece * a.piece;
      move_column(a.piece, col, from[0], to[0], moved, !falls);
    } else {
      uint8_t* col = (hv & 1 ? a.c.v_scales : a.c.k_scales) + h * a.c.scale_head_stride + (piece - a.pieces) * a.spiece;
      move_column(a.spiece, col, from[1], to[1], moved, !falls);
    }
  }
  // lengths_out may be lengths: written when every CTA of the cluster has read it.
  asm volatile("barrier.cluster.arrive.aligned;\n barrier.cluster.wait.aligned;" ::: "memory");
  if (rank == 0 && tid == 0) a.lengths_out[b] = first + moved;
}

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline int launch_status() { return cudaGetLastError() == cudaSuccess ? MIXFP4_OK : MIXFP4_ERR_CUDA; }

Plane plane_of(void* base, int64_t page_stride, int64_t token_stride, int64_t head_stride, int heads, int page_size,
               int row) {
  Plane p = {};
  p.base = static_cast<uint8_t*>(base);
  p.page_stride = page_stride;
  p.inner = 1;
  if (head_stride == row || heads == 1) {
    p.run = heads * row;
    p.by_token = token_stride == p.run || page_size == 1;
    p.outer = 1;  // of runs that hold tokens; else a page's tokens
    p.outer_stride = token_stride;
  } else if (token_stride == row || page_size == 1) {
    p.run = row, p.by_token = 1;
    p.outer = heads, p.outer_stride = head_stride;
  } else {
    p.run = row;
    p.outer_stride = token_stride;
    p.inner = heads, p.inner_stride = head_stride;
  }
  // The widest access that every run begins and ends on.
  const int64_t all = (int64_t)reinterpret_cast<uintptr_t>(base) | page_stride | p.outer_stride | p.inner_stride | p.run;
  p.piece = 1;
  for (int w : {4, 8, 16, 32})
    if (all % w == 0) p.piece = w;
  return p;
}

Planes planes_of(const mixfp4_kv_cache& c) {
  Planes ps = {};
  const bool fp4 = c.dtype == MIXFP4_CACHE_MIXFP4;
  const int64_t e = fp4 ? 1 : 2;
  const int row = fp4 ? c.head_dim / 2 : c.head_dim * 2;
  for (void* base : {c.k, c.v})
    ps.p[ps.count++] = plane_of(base, c.page_stride * e, c.token_stride * e, c.head_stride * e, c.heads, c.page_size, row);
  if (fp4)
    for (uint8_t* base : {c.k_scales, c.v_scales})
      ps.p[ps.count++] = plane_of(base, c.scale_page_stride, c.scale_token_stride, c.scale_head_stride, c.heads,
                                  c.page_size, c.head_dim / 16);
  return ps;
}

// CTAs to a page's share of one array.
int slices_of(const mixfp4_kv_cache& c) {
  const int64_t bytes = (int64_t)c.page_size * c.heads * c.head_dim * (c.dtype == MIXFP4_CACHE_MIXFP4 ? 1 : 4) / 2;
  const int64_t n = (bytes + kThreads * kInFlight * 32 - 1) / (kThreads * kInFlight * 32);
  return (int)(n < 1 ? 1 : (n > 4096 ? 4096 : n));
}

// Pages whose arrays' offsets within a page fit the kernels' 32-bit piece counts.
bool page_fits(const mixfp4_kv_cache& c) {
  return (int64_t)c.page_size * c.heads * c.head_dim * 2 <= INT32_MAX - (1 << 28);
}

bool table_fits(const mixfp4_kv_cache& c, int64_t table_stride, int64_t table_pages) {
  return table_pages >= 0 && table_stride >= table_pages && table_pages <= (INT32_MAX - 4096) / c.page_size;
}

bool meets(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a_bytes > 0 && b_bytes > 0 && x < y + (uintptr_t)b_bytes && y < x + (uintptr_t)a_bytes;
}

}  // namespace
}  // namespace mixfp4

extern "C" {

int mixfp4_kv_copy_pages(const mixfp4_kv_cache* cache, const int32_t* src, const int32_t* dst, int64_t n,
                         void* stream) {
  using namespace mixfp4;
  if (int st = check_kv_cache(cache)) return st;
  if (n < 0 || n > INT32_MAX || !page_fits(*cache)) return MIXFP4_ERR_SHAPE;
  if (n == 0) return MIXFP4_OK;
  if (!src || !dst) return MIXFP4_ERR_NULL;
  if (!aligned(src, 4) || !aligned(dst, 4)) return MIXFP4_ERR_ALIGN;
  const Planes ps = planes_of(*cache);
  const int slices = slices_of(*cache);
  kv_copy_pages_kernel<<<dim3((unsigned)n, (unsigned)(ps.count * slices)), kThreads, 0,
                         static_cast<cudaStream_t>(stream)>>>(ps, slices, cache->pages, cache->page_size, src, dst);
  return launch_status();
}

int mixfp4_kv_fork(const mixfp4_kv_cache* cache, const int32_t* block_table, int64_t table_stride,
                   int64_t table_pages, const int32_t* lengths, int64_t B, const int32_t* parents,
                   const int32_t* fresh, int64_t children, int32_t* table_out, int32_t* lengths_out, void* stream) {
  using namespace mixfp4;
  if (int st = check_kv_cache(cache)) return st;
  if (B < 0 || B > INT32_MAX || children < 0 || children > INT32_MAX || !page_fits(*cache) ||
      !table_fits(*cache, table_stride, table_pages))
    return MIXFP4_ERR_SHAPE;
  if (children == 0) return MIXFP4_OK;
  if (!parents || !fresh || !lengths_out || (B > 0 && !lengths) ||
      (table_pages > 0 && (!table_out || (B > 0 && !block_table))))
    return MIXFP4_ERR_NULL;
  if (!aligned(block_table, 4) || !aligned(lengths, 4) || !aligned(parents, 4) || !aligned(fresh, 4) ||
      !aligned(table_out, 4) || !aligned(lengths_out, 4))
    return MIXFP4_ERR_ALIGN;
  const int64_t in_bytes = B > 0 ? ((B - 1) * table_stride + table_pages) * 4 : 0;
  const struct {
    const void* p;
    int64_t bytes;
  } out[2] = {{table_out, children * table_pages * 4}, {lengths_out, children * 4}},
    in[4] = {{block_table, in_bytes}, {lengths, B * 4}, {parents, children * 4}, {fresh, children * 4}};
  for (const auto& o : out)
    for (const auto& i : in)
      if (meets(o.p, o.bytes, i.p, i.bytes)) return MIXFP4_ERR_ARG;
  if (meets(out[0].p, out[0].bytes, out[1].p, out[1].bytes)) return MIXFP4_ERR_ARG;
  ForkArgs a = {};
  a.ps = planes_of(*cache);
  a.slices = slices_of(*cache);
  a.page_size = cache->page_size, a.pages = cache->pages;
  a.table = block_table, a.table_stride = table_stride, a.table_pages = (int)table_pages;
  a.lengths = lengths, a.B = B, a.parents = parents, a.fresh = fresh;
  a.table_out = table_out, a.lengths_out = lengths_out;
  kv_fork_kernel<<<dim3((unsigned)children, (unsigned)(1 + a.ps.count * a.slices)), kThreads, 0,
                   static_cast<cudaStream_t>(stream)>>>(a);
  return launch_status();
}

int mixfp4_kv_accept(const mixfp4_kv_cache* cache, const int32_t* block_table, int64_t table_stride,
                     int64_t table_pages, const int32_t* lengths, const int32_t* counts, int64_t B,
                     const int32_t* path, int64_t path_stride, int64_t depth, int32_t* lengths_out, void* stream) {
  using namespace mixfp4;
  if (int st = check_kv_cache(cache)) return st;
  if (B < 0 || depth < 0 || depth > kMostDepth || path_stride < 0 || (B > 1 && path_stride < depth) ||
      !table_fits(*cache, table_stride, table_pages))
    return MIXFP4_ERR_SHAPE;
  if (B == 0) return MIXFP4_OK;
  if (!lengths || !counts || !lengths_out || (depth > 0 && !path) || (table_pages > 0 && !block_table))
    return MIXFP4_ERR_NULL;
  if (!aligned(block_table, 4) || !aligned(lengths, 4) || !aligned(counts, 4) || !aligned(path, 4) ||
      !aligned(lengths_out, 4))
    return MIXFP4_ERR_ALIGN;
  const int64_t table_bytes = ((B - 1) * table_stride + table_pages) * 4;
  if ((lengths_out != lengths && meets(lengths_out, B * 4, lengths, B * 4)) ||
      meets(lengths_out, B * 4, counts, B * 4) || meets(lengths_out, B * 4, block_table, table_bytes) ||
      meets(lengths_out, B * 4, path, ((B - 1) * path_stride + depth) * 4))
    return MIXFP4_ERR_ARG;
  AcceptArgs a = {};
  a.c = *cache;
  const bool fp4 = cache->dtype == MIXFP4_CACHE_MIXFP4;
  a.esize = fp4 ? 1 : 2;
  a.piece = fp4 ? 8 : 16, a.pieces = cache->head_dim * (fp4 ? 1 : 4) / 2 / a.piece;
  if (fp4) a.spiece = cache->head_dim % 64 == 0 ? 4 : 1, a.spieces = cache->head_dim / 16 / a.spiece;
  a.table = block_table, a.table_stride = table_stride, a.max_tokens = table_pages * cache->page_size;
  a.lengths = lengths, a.counts = counts, a.path = path, a.path_stride = path_stride, a.depth = (int)depth;
  a.lengths_out = lengths_out;
  const int64_t columns = 2ll * cache->heads * (a.pieces + a.spieces);
  int cluster = 1;
  while (cluster < 8 && cluster * kMoveThreads < columns) cluster *= 2;
  if (B * cluster > INT32_MAX) return MIXFP4_ERR_SHAPE;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cluster, attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(B * cluster));
  cfg.blockDim = dim3(kMoveThreads);
  cfg.stream = static_cast<cudaStream_t>(stream);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kv_accept_kernel, a) == cudaSuccess ? MIXFP4_OK : MIXFP4_ERR_CUDA;
}

}  // extern "C"
