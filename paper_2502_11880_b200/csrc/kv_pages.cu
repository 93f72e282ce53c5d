// The paged key-value cache's books and moves: writing new tokens' rows, giving out pages, forking, releasing and
// compacting sequences, copying pages.
//
// The books are a page table per sequence and one use count per page; a page with count 0 is free.  Pages are always
// given out lowest first, in the order of the list that asks, so every result is determined by the arguments: counts
// move by integer atomics (any order gives the same) and the free pages come from an ordered scan of the counts by one
// CTA.  That scan reads 4 bytes per page (100,000 pages: 0.4 MB) and ends as soon as enough pages are found.
// Moves of data (whole pages for compaction and copies, rows in use for forks) are a grid-stride copy of 16-byte
// pieces over the list of pages that the planning CTA left in the workspace; compaction is bound by HBM (1.74 GB, read and written: 277 to
// 285 us with its planning = 6.1 to 6.25 TB/s).  Forks read a parent's rows once for every child, the later times from L2: 128 forks of 16
// parents, 40 MB of distinct rows read and 317 MB written, take 83 to 91 us, of which HBM needs 54.  Appends read fp32 rows once and write
// 16-bit rows: 8192 tokens of 8 heads of 128, 100 MB, in 23 us with the books' copy and the reserve before it.
#include <cstring>

#include "kv_cache.cuh"

namespace bitnet {

// ------------------------------------------------------------------------------------------------ tensor maps
namespace {
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) != cudaSuccess ||
        qres != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  return fn;
}
}  // namespace

int encode_kv_maps(uint64_t (*maps)[16], int64_t* layer_pages, const KvView& v, int dtype) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return note_cuda_error(cudaErrorNotSupported);
  const CUtensorMapDataType t = dtype == BITNET_KV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  void* const pool[2] = {v.k, v.v};
  // the stride of a dimension of extent 1 is never used, but has to be one that the encoder takes
  auto bytes = [](int64_t extent, int64_t stride) { return extent > 1 ? (cuuint64_t)stride * 2 : (cuuint64_t)16; };
  const cuuint32_t rows = (cuuint32_t)kv_box_rows(v.page_size), estr[5] = {1, 1, 1, 1, 1};
  auto encode = [&](int i, const cuuint64_t* dim, const cuuint64_t* stride, const cuuint32_t* box) {
    CUtensorMap m;
    if (enc(&m, t, 5, pool[i & 1], dim, stride, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return false;
    memcpy(maps[i], &m, sizeof m);
    return true;
  };
  const cuuint64_t dim[5] = {(cuuint64_t)v.head_dim, (cuuint64_t)v.page_size, (cuuint64_t)v.kv_heads, (cuuint64_t)v.num_pages,
                             (cuuint64_t)v.layers};
  const cuuint64_t stride[4] = {(cuuint64_t)v.stride_row * 2, bytes(v.kv_heads, v.stride_head), bytes(v.num_pages, v.stride_page),
                                bytes(v.layers, v.stride_layer)};
  const cuuint32_t box[5] = {64, rows, 1, 1, 1};
  for (int i = 0; i < 2; ++i)
    if (!encode(i, dim, stride, box)) return note_cuda_error(cudaErrorInvalidValue);
  *layer_pages = 0;
  const int64_t apart = v.layers == 1 ? v.num_pages : v.stride_page > 0 && v.stride_layer % v.stride_page == 0 ? v.stride_layer / v.stride_page : 0;
  if (v.head_dim == 128 && apart >= v.num_pages && apart * v.layers < 0x7fffffff) {
    const cuuint64_t dim2[5] = {64, (cuuint64_t)v.page_size, 2, (cuuint64_t)v.kv_heads, (cuuint64_t)(apart * (v.layers - 1) + v.num_pages)};
    const cuuint64_t stride2[4] = {(cuuint64_t)v.stride_row * 2, 128, bytes(v.kv_heads, v.stride_head), bytes((int64_t)dim2[4], v.stride_page)};
    const cuuint32_t box2[5] = {64, rows, 2, 1, 1};
    if (encode(2, dim2, stride2, box2) && encode(3, dim2, stride2, box2)) *layer_pages = apart;
  }
  return BITNET_OK;
}

namespace {

// Division of 0 <= n < 2^31 by d >= 1 as a product: with s = ceil(log2 d), m = ceil(2^(31+s) / d) < 2^32 exceeds 2^(31+s) / d by less
// than 1, so n m / 2^(31+s) exceeds n / d by less than n / 2^(31+s) <= 1 / d, too little to reach the next whole number.
// (With whole divisions pages of 32 heads of 100 moved at 5.5 instead of 6.1 TB/s.)
struct Div {
  uint32_t m;
  int s;
};
__host__ __device__ inline Div div_by(uint32_t d) {
  Div r;
  r.s = 0;
  while ((1u << r.s) < d) ++r.s;
  r.m = (uint32_t)((((uint64_t)1 << (31 + r.s)) + d - 1) / d);
  return r;
}
__device__ __forceinline__ int quotient(int n, const Div& d) { return (int)(((uint64_t)(uint32_t)n * d.m) >> (31 + d.s)); }

// ------------------------------------------------------------------------------------------------ append
struct AppendArgs {
  KvView kv;
  const uint8_t* src[2];
  int64_t stride_token, stride_head;
  const int32_t* table;
  const int32_t* kv_len;
  const int32_t* q_start;
  int64_t width;
  int tokens, seqs, layer;
  Div pieces;                // of a row
  int* dev_status;
};

__device__ __forceinline__ uint32_t to16(uint32_t lo, uint32_t hi, const __nv_bfloat16*) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(__uint_as_float(lo), __uint_as_float(hi));
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t to16(uint32_t lo, uint32_t hi, const __half*) {
  const __half2 v = __floats2half2_rn(__uint_as_float(lo), __uint_as_float(hi));
  return *reinterpret_cast<const uint32_t*>(&v);
}

enum AppendIn { IN_F32, IN_16, IN_16_ALIGNED };

// A warp takes up to 128 pieces of 8 elements of one new token's K or V: 4 per lane, all loaded before the look-ups of the token's
// sequence, position and page, which do not depend on them, have come back one after the other.  fp32 rows are rounded
// once to the cache's type; otherwise the bits move.  A row's last piece, where head_dim is no multiple of 8, ends with zeros in the
// row's padding, so that whole sectors are written.  (32 tokens of 32 heads of 100: 10.6 us with a warp per row that looked up
// first and loaded in turns.)
template <typename KT, int IN>
__global__ void __launch_bounds__(256) kv_append_kernel(const AppendArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x & 31;
  const int pieces = (a.kv.head_dim + 7) >> 3, units = a.kv.kv_heads * pieces, chunks = (units + 127) / 128;
  const int64_t id = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int64_t token_pool = id / chunks;
  if (token_pool >= 2 * (int64_t)a.tokens) return;
  const int n = (int)(token_pool >> 1), pool = (int)(token_pool & 1);
  const int u0 = (int)(id - token_pool * chunks) * 128 + lane;

  const uint8_t* src = a.src[pool] + n * a.stride_token * (IN == IN_F32 ? 4 : 2);
  uint4 lo[4], hi[4];                                      // 8 fp32 values, or 8 of 16 bits in lo
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int u = u0 + 32 * j;
    lo[j] = hi[j] = make_uint4(0u, 0u, 0u, 0u);
    if (u < units) {
      const int h = quotient(u, a.pieces), d = (u - h * pieces) * 8;
      const bool full = d + 8 <= a.kv.head_dim;
      const uint8_t* at = src + (h * a.stride_head + d) * (IN == IN_F32 ? 4 : 2);
      if (IN == IN_F32) {
        lo[j] = __ldg(reinterpret_cast<const uint4*>(at));
        if (full) hi[j] = __ldg(reinterpret_cast<const uint4*>(at) + 1);
      } else if (IN == IN_16_ALIGNED) {
        lo[j] = __ldg(reinterpret_cast<const uint4*>(at));
      } else {
        const uint2 x = __ldg(reinterpret_cast<const uint2*>(at)), y = full ? __ldg(reinterpret_cast<const uint2*>(at) + 1) : make_uint2(0u, 0u);
        lo[j] = make_uint4(x.x, x.y, y.x, y.y);
      }
    }
  }

  int seq = n;
  int64_t pos;
  if (a.q_start) {
    // the number of sequences that begin after the first and not beyond token n, 32 at a time
    seq = 0;
    for (int s0 = 1; s0 < a.seqs; s0 += 32) {
      const int s = s0 + lane;
      const int in = __popc(__ballot_sync(0xffffffffu, s < a.seqs && __ldg(a.q_start + s) <= n));
      seq += in;
      if (in < 32) break;
    }
    pos = (int64_t)__ldg(a.kv_len + seq) - __ldg(a.q_start + seq + 1) + n;
  } else {
    pos = (int64_t)__ldg(a.kv_len + seq) - 1;
  }
  const int64_t entry = pos / a.kv.page_size;
  if (pos < 0) return;
  const int page = entry < a.width ? __ldg(a.table + (int64_t)seq * a.width + entry) : -1;
  if (page < 0 || page >= a.kv.num_pages) {
    if (lane == 0 && a.dev_status) atomicExch(a.dev_status, BITNET_ERR_BAD_PAGE);
    return;
  }
  uint8_t* dst = (pool ? a.kv.v : a.kv.k) +
                 2 * (a.layer * a.kv.stride_layer + page * a.kv.stride_page + (pos & (a.kv.page_size - 1)) * a.kv.stride_row);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int u = u0 + 32 * j;
    if (u < units) {
      const int h = quotient(u, a.pieces), d = (u - h * pieces) * 8;
      uint4 w = lo[j];
      if (IN == IN_F32) {
        const KT* t = nullptr;
        w = make_uint4(to16(lo[j].x, lo[j].y, t), to16(lo[j].z, lo[j].w, t), to16(hi[j].x, hi[j].y, t), to16(hi[j].z, hi[j].w, t));
      }
      *reinterpret_cast<uint4*>(dst + 2 * (h * a.kv.stride_head + d)) = w;
    }
  }
}

// ------------------------------------------------------------------------------------------------ planning
constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_SEQS = 4096;      // entries of the list that one pass plans at most

// Exclusive prefix of `x` over the CTA; `total` is the sum.  All threads take part.
__device__ __forceinline__ int block_scan(int x, int& total, int* warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, inc, d);
    if (lane >= d) inc += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  int v = warp_sums[lane];
  int s = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, s, d);
    if (lane >= d) s += y;
  }
  total = __shfl_sync(0xffffffffu, s, 31);
  const int before = __shfl_sync(0xffffffffu, s - v, warp);
  return before + inc - x;
}

// The counts of a step's 4 pages per thread (a page beyond the pool counts as used).
struct Counts {
  int c[4];
};
__device__ __forceinline__ Counts load_counts(const int32_t* refs, int num_pages, int p0) {
  Counts x;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int p = p0 + (int)threadIdx.x * 4 + j;
    x.c[j] = p < num_pages ? __ldcg(refs + p) : 1;
  }
  return x;
}
// Calls give(rank, page) for the free pages of rank 0..need-1, lowest page first; returns how many free pages there
// were (counted up to where the scan ended: at least `need` if enough).  `x` holds the first step's counts; each step's are loaded
// while the one before is looked at.
template <typename F>
__device__ __forceinline__ int scan_free(const int32_t* refs, int num_pages, int need, Counts x, int* warp_sums, F give) {
  int found = 0;
  for (int p0 = 0; p0 < num_pages && found < need; p0 += PLAN_THREADS * 4) {
    const Counts next = load_counts(refs, num_pages, p0 + PLAN_THREADS * 4);
    const int p = p0 + threadIdx.x * 4;
    int total, mine = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) mine += x.c[j] == 0;
    int rank = found + block_scan(mine, total, warp_sums);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (x.c[j] == 0) {
        if (rank < need) give(rank, p + j);
        ++rank;
      }
    found += total;
    x = next;
  }
  return found;
}

// Pages for the entries [ceil(from / page), ceil(to / page)) of every row, lowest free pages first in the order of the rows; per_pass
// rows (at most PLAN_SEQS) at a time.
__global__ void __launch_bounds__(PLAN_THREADS)
kv_reserve_kernel(int32_t* refs, int num_pages, int32_t* table, int64_t seqs, int64_t width, const int32_t* from_len, const int32_t* to_len,
                  int page_shift, int per_pass, int* dev_status) {
  __shared__ int warp_sums[32];
  __shared__ int start[PLAN_SEQS + 1];     // entries asked for before each row of the pass
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int64_t mask = (1 << page_shift) - 1;
  auto first_entry = [&](int64_t row) { return (max((int64_t)0, (int64_t)from_len[row]) + mask) >> page_shift; };
  bool lacking = false;
  Counts counts = load_counts(refs, num_pages, 0);
  for (int64_t r0 = 0; r0 < seqs; r0 += per_pass) {
    const int rows = (int)min((int64_t)per_pass, seqs - r0);
    // 4 rows per thread: counts, then their prefix
    int cnt[PLAN_SEQS / PLAN_THREADS], sum = 0;
#pragma unroll
    for (int j = 0; j < PLAN_SEQS / PLAN_THREADS; ++j) {
      const int i = threadIdx.x * (PLAN_SEQS / PLAN_THREADS) + j;
      cnt[j] = 0;
      if (i < rows) {
        const int64_t b = first_entry(r0 + i), e = (max((int64_t)0, (int64_t)to_len[r0 + i]) + mask) >> page_shift;
        if (e > width) lacking = true;
        cnt[j] = (int)max((int64_t)0, min(e, width) - b);
      }
      sum += cnt[j];
    }
    int need;
    int at = block_scan(sum, need, warp_sums);
#pragma unroll
    for (int j = 0; j < PLAN_SEQS / PLAN_THREADS; ++j) {
      const int i = threadIdx.x * (PLAN_SEQS / PLAN_THREADS) + j;
      if (i <= rows) start[i] = at;
      at += cnt[j];
    }
    if (threadIdx.x == 0) start[rows] = need;
    __syncthreads();
    if (need == 0) continue;
    auto place = [&](int rank) -> int32_t* {
      int lo = 0, hi = rows;               // start[lo] <= rank < start[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= rank) lo = mid;
        else hi = mid;
      }
      return table + (r0 + lo) * width + first_entry(r0 + lo) + (rank - start[lo]);
    };
    const int found = scan_free(refs, num_pages, need, counts, warp_sums, [&](int rank, int page) {
      *place(rank) = page;
      refs[page] = 1;
    });
    if (found < need) {                    // the pool has no more: the entries left over hold no page
      lacking = true;
      for (int64_t k = found + threadIdx.x; k < need; k += PLAN_THREADS) *place((int)k) = -1;
    }
    __threadfence();
    __syncthreads();
    if (r0 + per_pass < seqs) counts = load_counts(refs, num_pages, 0);
  }
  if (lacking && dev_status) atomicExch(dev_status, BITNET_ERR_NO_PAGE);
}

// A page move: `rows` rows of every head, layer and pool, from page src to page dst; the multiplier of a division by rows.
struct Move {
  int32_t src, dst, rows;
  uint32_t m;
};
// Workspace: the number of moves (and, for compaction, of pages in use), the moves, and the pages' new places.
struct PlanHead {
  int32_t moves, live, pad[2];
};

// Where a fork's parent ends: used tokens, as a number that its row of the table can hold.
__device__ __forceinline__ int64_t fork_used(const int32_t* len, int parent, int64_t width, int page_shift) {
  return min((int64_t)max(0, len[parent]), width << page_shift);
}
__device__ __forceinline__ bool fork_valid(int parent, int child, int64_t seqs) {
  return parent >= 0 && parent < seqs && child >= 0 && child < seqs && parent != child;
}

// Plans a fork's copies: the i-th child whose parent fills a page in part gets the i-th free page.  (Full pages are shared, which
// makes none free or used; kv_move_kernel does that, on all SMs.)
__global__ void __launch_bounds__(PLAN_THREADS)
kv_fork_kernel(int32_t* refs, int num_pages, int32_t* table, int64_t seqs, int64_t width, const int32_t* len, const int32_t* parents,
               const int32_t* children, int n, int page_shift, PlanHead* head, Move* moves, int* dev_status) {
  __shared__ int warp_sums[32];
  __shared__ Move want[PLAN_THREADS];      // of a step's children, by rank; dst: the child
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  Counts counts = load_counts(refs, num_pages, 0);
  int made = 0;
  bool bad = false, lacking = false;
  for (int i0 = 0; i0 < n; i0 += PLAN_THREADS) {
    const int i = i0 + threadIdx.x;
    int src = -1, rows = 0, c = 0;
    int64_t e = 0;
    if (i < n) {
      const int p = parents[i];
      c = children[i];
      if (fork_valid(p, c, seqs)) {
        const int64_t used = fork_used(len, p, width, page_shift);
        rows = (int)(used & ((1 << page_shift) - 1));
        e = used >> page_shift;
        if (rows) src = table[p * width + e];
        if (src >= num_pages) src = -1;
        // no page where rows are in use, or tokens beyond the table
        if ((rows && src < 0) || ((int64_t)len[p] + (1 << page_shift) - 1) >> page_shift > width) bad = true;
        if (rows) table[c * width + e] = -1;
      } else {
        bad = true;
      }
    }
    int total;
    const int rank = block_scan(src >= 0, total, warp_sums);
    if (src >= 0) want[rank] = Move{src, c, rows, (uint32_t)e};
    __threadfence();
    __syncthreads();
    const int found = scan_free(refs, num_pages, total, counts, warp_sums, [&](int k, int id) {
      const Move w = want[k];
      moves[made + k] = Move{w.src, id, w.rows, div_by((uint32_t)w.rows).m};
      table[w.dst * width + w.m] = id;
      refs[id] = 1;
    });
    if (found < total) lacking = true;     // children without a page keep -1 there
    made += min(found, total);
    __threadfence();
    __syncthreads();
    if (i0 + PLAN_THREADS < n) counts = load_counts(refs, num_pages, 0);
  }
  if (threadIdx.x == 0) head->moves = made;
  if (dev_status) {
    if (bad) atomicExch(dev_status, BITNET_ERR_BAD_PAGE);
    if (lacking) atomicExch(dev_status, BITNET_ERR_NO_PAGE);
  }
}

// The number of pages in use (live), and where each in-use page beyond the first `live` places goes.
__global__ void __launch_bounds__(PLAN_THREADS)
kv_compact_plan_kernel(int32_t* refs, int num_pages, int page_size, PlanHead* head, Move* moves, int32_t* place, int32_t* live_out) {
  __shared__ int warp_sums[32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  int live = 0;
#pragma unroll 4
  for (int p0 = 0; p0 < num_pages; p0 += PLAN_THREADS * 4) {
    const Counts x = load_counts(refs, num_pages, p0);
#pragma unroll
    for (int j = 0; j < 4; ++j) live += x.c[j] > 0 && p0 + (int)threadIdx.x * 4 + j < num_pages;
  }
  Counts x = load_counts(refs, num_pages, 0);
  int sum;
  block_scan(live, sum, warp_sums);
  live = sum;
  int holes = 0, tail = 0;                 // free places below `live`, pages in use beyond
  for (int p0 = 0; p0 < num_pages; p0 += PLAN_THREADS * 4) {
    const Counts next = load_counts(refs, num_pages, p0 + PLAN_THREADS * 4);
    const int p = p0 + (int)threadIdx.x * 4;
    int mine = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (p + j < num_pages) mine += p + j < live ? (x.c[j] <= 0 ? 1 : 0) : (x.c[j] > 0 ? 1 << 16 : 0);
    int total;
    const int both = block_scan(mine, total, warp_sums);    // at most 4096 of each per step
    int hole = holes + (both & 0xffff), out = tail + (both >> 16);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (p + j < num_pages) {
        place[p + j] = p + j;
        if (p + j < live && x.c[j] <= 0) moves[hole++].dst = p + j;
        if (p + j >= live && x.c[j] > 0) moves[out++].src = p + j;
      }
    holes += total & 0xffff;
    tail += total >> 16;
    x = next;
  }
  __threadfence();
  __syncthreads();
  for (int i0 = threadIdx.x; i0 < tail; i0 += PLAN_THREADS * 4) {   // four at a time: their latencies overlap
    Move m[4];
    int count[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i0 + PLAN_THREADS * j < tail) m[j] = moves[i0 + PLAN_THREADS * j];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i0 + PLAN_THREADS * j < tail) count[j] = refs[m[j].src];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i0 + PLAN_THREADS * j < tail) {
        moves[i0 + PLAN_THREADS * j].rows = page_size;
        moves[i0 + PLAN_THREADS * j].m = 1u << 31;             // (a power of two)
        place[m[j].src] = m[j].dst;
        refs[m[j].dst] = count[j];
        refs[m[j].src] = 0;
      }
  }
  if (threadIdx.x == 0) {
    head->moves = tail;
    head->live = live;
    if (live_out) *live_out = live;
  }
}

// ------------------------------------------------------------------------------------------------ moving data
struct MoveArgs {
  KvView kv;
  const PlanHead* head;     // null: `count` pages of the lists src, dst
  const Move* moves;
  const int32_t* src;
  const int32_t* dst;
  int64_t count;
  const int32_t* place;     // compaction: the pages' new places, for the table
  int32_t* table;
  int64_t seqs, width;
  const int32_t* parents;   // fork: the children's rows and the counts of what they share
  const int32_t* children;
  int64_t n;
  int32_t* refs;
  int32_t* len;
  int page_shift;
  Div pieces, page_units;   // of a row, of a page
  int* dev_status;
};

// A block takes `jobs` -- a move in one layer of one pool each -- one at a time where a page has many 16-byte pieces, otherwise as
// many at a time as give every thread four: 4 per thread in flight carry the copy.  A row is copied with its padding up to a whole
// piece (8-byte pieces of rows of 100 without it: 3.3 instead of 5.9 TB/s).
template <bool LARGE>
__global__ void __launch_bounds__(256) kv_move_kernel(const MoveArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t moves = a.head ? a.head->moves : a.count;
  const int pieces = (a.kv.head_dim + 7) >> 3;
  const int64_t jobs = moves * a.kv.layers * 2;
  if (a.parents) {
    const int lane = threadIdx.x & 31;
    for (int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); i < a.n; i += (int64_t)gridDim.x * 8) {
      const int p = a.parents[i], c = a.children[i];
      if (!fork_valid(p, c, a.seqs)) continue;
      const int64_t used = fork_used(a.len, p, a.width, a.page_shift), full = used >> a.page_shift;
      const bool part = (used & ((1 << a.page_shift) - 1)) != 0;       // that entry has been seen to
      for (int64_t e = lane; e < a.width; e += 32) {
        int id = -1;
        if (e < full) {
          id = a.table[p * a.width + e];
          if (id >= 0 && id < a.kv.num_pages) atomicAdd(a.refs + id, 1);
          else {
            if (id >= 0 && a.dev_status) atomicExch(a.dev_status, BITNET_ERR_BAD_PAGE);   // (-1: released)
            id = -1;
          }
        }
        if (e != full || !part) a.table[c * a.width + e] = id;
      }
      if (lane == 0) a.len[c] = (int)used;
    }
  }
  struct Job {
    const uint8_t* from;
    uint8_t* to;
    int rows;
    Div by_rows;
  };
  auto job_of = [&](int64_t job) -> Job {
    const int64_t ml = job >> 1, move = ml / a.kv.layers;
    const int layer = (int)(ml - move * a.kv.layers);
    int src, dst, rows = a.kv.page_size;
    Div by_rows = {1u << 31, a.page_shift};
    if (a.head) {
      const Move m = a.moves[move];
      src = m.src;
      dst = m.dst;
      rows = m.rows;
      by_rows = Div{m.m, 32 - __clz(m.rows - 1)};
    } else {
      src = a.src[move];
      dst = a.dst[move];
    }
    if (src < 0 || src >= a.kv.num_pages || dst < 0 || dst >= a.kv.num_pages) {
      if (a.dev_status) atomicExch(a.dev_status, BITNET_ERR_BAD_PAGE);
      return Job{nullptr, nullptr, 0, by_rows};
    }
    uint8_t* base = (job & 1 ? a.kv.v : a.kv.k) + layer * a.kv.stride_layer * 2;
    return Job{base + src * a.kv.stride_page * 2, base + dst * a.kv.stride_page * 2, rows, by_rows};   // (products of 64 bits)
  };
  const int page_units = a.kv.kv_heads * a.kv.page_size * pieces;
  if (LARGE) {
    for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
      const Job x = job_of(job);
      const int units = a.kv.kv_heads * x.rows * pieces;
      for (int u0 = threadIdx.x; u0 < units; u0 += 256 * 4) {
        uint4 w[4];
        int64_t at[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int u = u0 + 256 * j;
          if (u < units) {
            const int hr = quotient(u, a.pieces), h = quotient(hr, x.by_rows);
            at[j] = 2 * (h * a.kv.stride_head + (hr - h * x.rows) * a.kv.stride_row + (u - hr * pieces) * 8);
            w[j] = *reinterpret_cast<const uint4*>(x.from + at[j]);
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (u0 + 256 * j < units) *reinterpret_cast<uint4*>(x.to + at[j]) = w[j];
      }
    }
  } else {
    const int64_t units = jobs * page_units;
    for (int64_t base = (int64_t)blockIdx.x * 1024; base < units; base += (int64_t)gridDim.x * 1024) {
      const int64_t job0 = base / page_units;
      const int skip = (int)(base - job0 * page_units), end = (int)min((int64_t)1024, units - base) + skip;
      uint4 w[4];
      uint8_t* to[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int u = skip + (int)threadIdx.x + 256 * j;
        to[j] = nullptr;
        if (u < end) {
          const int job = quotient(u, a.page_units);
          const Job x = job_of(job0 + job);
          const int v = u - job * page_units, hr = quotient(v, a.pieces), h = hr >> a.page_shift, row = hr & (a.kv.page_size - 1);
          if (row < x.rows) {
            const int64_t at = 2 * (h * a.kv.stride_head + row * a.kv.stride_row + (v - hr * pieces) * 8);
            w[j] = *reinterpret_cast<const uint4*>(x.from + at);
            to[j] = x.to + at;
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (to[j]) *reinterpret_cast<uint4*>(to[j]) = w[j];
    }
  }
  if (a.place)
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.seqs * a.width; i += (int64_t)gridDim.x * 256) {
      const int id = a.table[i];
      if (id >= 0 && id < a.kv.num_pages) a.table[i] = a.place[id];
    }
}

// ------------------------------------------------------------------------------------------------ releasing
// list: the rows to give up (null: rows 0..n-1).  trim: only pages wholly between the first `sinks` tokens and the last
// `window`; otherwise the whole row, whose length becomes 0.  One warp per 32 entries (a warp per row took 22 us for rows of 512); an
// entry is taken out by an exchange, so a row that is listed twice is released once.
__global__ void __launch_bounds__(256)
kv_release_kernel(int32_t* refs, int num_pages, int32_t* table, int64_t seqs, int64_t width, int32_t* len, const int32_t* list, int64_t n,
                  int page_shift, int window, int sinks, int trim, int* dev_status) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x & 31;
  const int64_t id = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), chunks = (width + 31) / 32, i = id / chunks;
  if (i >= n) return;
  const int64_t row = list ? list[i] : i, e = (id - i * chunks) * 32 + lane;
  if (row < 0 || row >= seqs) {
    if (lane == 0 && dev_status) atomicExch(dev_status, BITNET_ERR_BAD_PAGE);
    return;
  }
  int64_t first = 0, last = width;
  if (trim) {
    first = ((int64_t)sinks + (1 << page_shift) - 1) >> page_shift;
    last = min(width, max((int64_t)0, (int64_t)len[row] - window) >> page_shift);
  }
  if (e >= first && e < last && table[row * width + e] >= 0) {
    const int id = atomicExch(table + row * width + e, -1);
    if (id >= 0 && id < num_pages) atomicSub(refs + id, 1);
    else if (id >= 0 && dev_status) atomicExch(dev_status, BITNET_ERR_BAD_PAGE);
  }
  if (!trim && e == 0) len[row] = 0;
}

template <typename K, typename... A>
int launch(K kernel, unsigned grid, unsigned block, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(block);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = early_start_enabled(st) ? 1 : 0;
  cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
  return e == cudaSuccess ? check_launch() : note_cuda_error(e);
}

PlanHead* plan_head(void* ws) { return static_cast<PlanHead*>(ws); }
Move* plan_moves(void* ws) { return reinterpret_cast<Move*>(static_cast<uint8_t*>(ws) + sizeof(PlanHead)); }
int32_t* plan_place(void* ws, int64_t moves) { return reinterpret_cast<int32_t*>(plan_moves(ws) + moves); }

// Up to 32 blocks per SM, which the hardware deals out as others end (8 / 32 / 128 of them: compaction of 1.7 GB 312 / 280 / 275 us,
// 128 forks of 0.6 GB 98 / 90 / 90 us); 16 where a page has fewer than 1024 pieces.
int launch_move(MoveArgs& a, int64_t jobs, cudaStream_t st) {
  const int page_units = a.kv.kv_heads * a.kv.page_size * ((a.kv.head_dim + 7) / 8);
  const bool large = page_units >= 1024;
  a.pieces = div_by((uint32_t)ceil_div(a.kv.head_dim, 8));
  a.page_units = div_by((uint32_t)page_units);
  a.page_shift = __builtin_ctz((unsigned)a.kv.page_size);
  const int64_t most = (int64_t)dev_info().sm_count * (large ? 32 : 16);
  const unsigned grid = (unsigned)(jobs < 1 ? 1 : jobs < most ? jobs : most);
  log_launch("kv_move_kernel jobs=%lld grid=%u", (long long)jobs, grid);
  return large ? launch(kv_move_kernel<true>, grid, 256, st, a) : launch(kv_move_kernel<false>, grid, 256, st, a);
}

}  // namespace

int launch_kv_append(const KvView& kv, int layer, const void* k, const void* v, int in_dtype, int64_t stride_token, int64_t stride_head,
                     int64_t tokens, int64_t seqs, const int32_t* table, int64_t width, const int32_t* kv_len, const int32_t* q_start,
                     int dtype, int* dev_status, cudaStream_t st) {
  AppendArgs a;
  a.kv = kv;
  a.src[0] = static_cast<const uint8_t*>(k);
  a.src[1] = static_cast<const uint8_t*>(v);
  a.stride_token = stride_token;
  a.stride_head = stride_head;
  a.table = table;
  a.kv_len = kv_len;
  a.q_start = q_start;
  a.width = width;
  a.tokens = (int)tokens;
  a.seqs = (int)seqs;
  a.layer = layer;
  a.pieces = div_by((uint32_t)ceil_div(kv.head_dim, 8));
  a.dev_status = dev_status;
  const int64_t chunks = ceil_div((int64_t)kv.kv_heads * ceil_div(kv.head_dim, 8), 128), blocks = ceil_div(2 * tokens * chunks, 8);
  if (blocks > 0x7fffffff) return BITNET_ERR_UNSUPPORTED_SHAPE;
  const unsigned grid = (unsigned)blocks;
  log_launch("kv_append_kernel tokens=%lld grid=%u", (long long)tokens, grid);
  if (in_dtype != BITNET_KV_F32) {
    // same type: bits move, in 16-byte pieces where every row begins at a multiple of 16 bytes and is a whole number of them
    const bool whole = kv.head_dim % 8 == 0 && stride_token % 8 == 0 && stride_head % 8 == 0 && aligned16(k) && aligned16(v);
    return whole ? launch(kv_append_kernel<__half, IN_16_ALIGNED>, grid, 256, st, a) : launch(kv_append_kernel<__half, IN_16>, grid, 256, st, a);
  }
  return dtype == BITNET_KV_BF16 ? launch(kv_append_kernel<__nv_bfloat16, IN_F32>, grid, 256, st, a)
                                 : launch(kv_append_kernel<__half, IN_F32>, grid, 256, st, a);
}

int launch_kv_reserve(int32_t* refs, int64_t num_pages, int32_t* table, int64_t seqs, int64_t width, const int32_t* from_len,
                      const int32_t* to_len, int page_size, int* dev_status, cudaStream_t st) {
  // as many rows to a pass as have fewer than 2^31 entries together, which are counted in int
  const int64_t most = 0x7fffffff / width, per_pass = most < 1 ? 1 : most < PLAN_SEQS ? most : PLAN_SEQS;
  log_launch("kv_reserve_kernel seqs=%lld", (long long)seqs);
  return launch(kv_reserve_kernel, 1, PLAN_THREADS, st, refs, (int)num_pages, table, seqs, width, from_len, to_len,
                __builtin_ctz((unsigned)page_size), (int)per_pass, dev_status);
}

int launch_kv_fork(const KvView& kv, int32_t* refs, int32_t* table, int64_t seqs, int64_t width, int32_t* len, const int32_t* parents,
                   const int32_t* children, int64_t n, void* ws, int* dev_status, cudaStream_t st) {
  log_launch("kv_fork_kernel n=%lld", (long long)n);
  int rc = launch(kv_fork_kernel, 1, PLAN_THREADS, st, refs, kv.num_pages, table, seqs, width, len, parents, children, (int)n,
                  __builtin_ctz((unsigned)kv.page_size), plan_head(ws), plan_moves(ws), dev_status);
  if (rc) return rc;
  MoveArgs m = {};
  m.kv = kv;
  m.head = plan_head(ws);
  m.moves = plan_moves(ws);
  m.table = table;
  m.seqs = seqs;
  m.width = width;
  m.parents = parents;
  m.children = children;
  m.n = n;
  m.refs = refs;
  m.len = len;
  m.dev_status = dev_status;
  return launch_move(m, n * kv.layers * 2, st);
}

int launch_kv_release(int32_t* refs, int64_t num_pages, int32_t* table, int64_t seqs, int64_t width, int32_t* len, const int32_t* list,
                      int64_t n, int page_size, int window, int sinks, bool trim, int* dev_status, cudaStream_t st) {
  const int64_t blocks = ceil_div(n * ceil_div(width, 32), 8);
  if (blocks > 0x7fffffff) return BITNET_ERR_UNSUPPORTED_SHAPE;
  log_launch("kv_release_kernel rows=%lld trim=%d", (long long)n, (int)trim);
  return launch(kv_release_kernel, (unsigned)blocks, 256, st, refs, (int)num_pages, table, seqs, width, len, list, n,
                __builtin_ctz((unsigned)page_size), window, sinks, (int)trim, dev_status);
}

int launch_kv_compact(const KvView& kv, int32_t* refs, int32_t* table, int64_t seqs, int64_t width, int32_t* live_out, void* ws,
                      cudaStream_t st) {
  int32_t* place = plan_place(ws, kv.num_pages);
  log_launch("kv_compact_plan_kernel pages=%d", kv.num_pages);
  int rc = launch(kv_compact_plan_kernel, 1, PLAN_THREADS, st, refs, kv.num_pages, kv.page_size, plan_head(ws), plan_moves(ws), place,
                  live_out);
  if (rc) return rc;
  MoveArgs m = {};
  m.kv = kv;
  m.head = plan_head(ws);
  m.moves = plan_moves(ws);
  m.place = place;
  m.table = table;
  m.seqs = seqs;
  m.width = width;
  return launch_move(m, (int64_t)kv.num_pages * kv.layers, st);   // at most half of the pages move
}

int launch_kv_copy_pages(const KvView& kv, const int32_t* src, const int32_t* dst, int64_t n, int* dev_status, cudaStream_t st) {
  MoveArgs m = {};
  m.kv = kv;
  m.src = src;
  m.dst = dst;
  m.count = n;
  m.dev_status = dev_status;
  return launch_move(m, n * kv.layers * 2, st);
}

// Compaction plans at most num_pages moves and keeps every page's place; a fork plans n.
size_t kv_workspace_bytes(int64_t num_pages, int64_t n) {
  const size_t compact = (size_t)num_pages * (sizeof(Move) + 4), fork = (size_t)n * sizeof(Move);
  return sizeof(PlanHead) + (compact > fork ? compact : fork);
}

}  // namespace bitnet
