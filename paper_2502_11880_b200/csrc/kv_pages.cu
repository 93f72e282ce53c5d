// The paged key-value cache's books and moves: writing new tokens' rows, giving out pages, forking, releasing and
// compacting sequences, copying pages.
//
// The books are a page table per sequence and one use count per page; a page with count 0 is free.  Pages are always
// given out lowest first, in the order of the list that asks, so every result is determined by the arguments: counts
// move by integer atomics (any order gives the same) and the free pages come from an ordered scan of the counts by one
// CTA.  That scan reads 4 bytes per page (100,000 pages: 0.4 MB) and ends as soon as enough pages are found.
// Moves of data (whole pages for compaction and copies, rows in use for forks) are a grid-stride copy of 16-byte
// pieces over the list of pages that the planning CTA left in the workspace; they are bound by HBM.
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
  int* dev_status;
};

__device__ __forceinline__ uint2 to16(const float4& v, const __nv_bfloat16*) {
  __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
  return make_uint2(*reinterpret_cast<uint32_t*>(&a), *reinterpret_cast<uint32_t*>(&b));
}
__device__ __forceinline__ uint2 to16(const float4& v, const __half*) {
  __half2 a = __floats2half2_rn(v.x, v.y), b = __floats2half2_rn(v.z, v.w);
  return make_uint2(*reinterpret_cast<uint32_t*>(&a), *reinterpret_cast<uint32_t*>(&b));
}

// A warp takes up to 256 pieces of 4 elements of one new token's K or V: 8 per lane, all loaded before the look-ups of the token's
// sequence, position and page, which do not depend on them, have come back one after the other.  IN32: fp32 rows, rounded once to the
// cache's type; otherwise the bits move.  (32 tokens of 32 heads of 100: 10.6 us with a warp per row that looked up first and
// loaded in turns.)
template <typename KT, bool IN32>
__global__ void __launch_bounds__(256) kv_append_kernel(const AppendArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x & 31;
  const int quads = a.kv.head_dim >> 2, units = a.kv.kv_heads * quads, chunks = (units + 255) / 256;
  const int64_t id = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int64_t token_pool = id / chunks;
  if (token_pool >= 2 * (int64_t)a.tokens) return;
  const int n = (int)(token_pool >> 1), pool = (int)(token_pool & 1);
  const int u0 = (int)(id - token_pool * chunks) * 256 + lane;

  const uint8_t* src = a.src[pool] + n * a.stride_token * (IN32 ? 4 : 2);
  uint4 raw[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int u = u0 + 32 * j;
    if (u < units) {
      const int h = u / quads, d = (u - h * quads) * 4;
      if (IN32) {
        raw[j] = __ldg(reinterpret_cast<const uint4*>(src + (h * a.stride_head + d) * 4));
      } else {
        const uint2 w = __ldg(reinterpret_cast<const uint2*>(src + (h * a.stride_head + d) * 2));
        raw[j].x = w.x;
        raw[j].y = w.y;
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
  for (int j = 0; j < 8; ++j) {
    const int u = u0 + 32 * j;
    if (u < units) {
      const int h = u / quads, d = (u - h * quads) * 4;
      uint2 w = make_uint2(raw[j].x, raw[j].y);
      if (IN32)
        w = to16(make_float4(__uint_as_float(raw[j].x), __uint_as_float(raw[j].y), __uint_as_float(raw[j].z), __uint_as_float(raw[j].w)),
                 (const KT*)nullptr);
      *reinterpret_cast<uint2*>(dst + 2 * (h * a.kv.stride_head + d)) = w;
    }
  }
}

// ------------------------------------------------------------------------------------------------ planning
constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_SEQS = 4096;      // entries of the list that one pass plans

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

// Pages for the entries [ceil(from / page), ceil(to / page)) of every row, lowest free pages first in the order of the rows.
__global__ void __launch_bounds__(PLAN_THREADS)
kv_reserve_kernel(int32_t* refs, int num_pages, int32_t* table, int64_t seqs, int64_t width, const int32_t* from_len, const int32_t* to_len,
                  int page_shift, int* dev_status) {
  __shared__ int warp_sums[32];
  __shared__ int start[PLAN_SEQS + 1];     // entries asked for before each row of the pass
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int64_t mask = (1 << page_shift) - 1;
  auto first_entry = [&](int64_t row) { return (max((int64_t)0, (int64_t)from_len[row]) + mask) >> page_shift; };
  bool lacking = false;
  Counts counts = load_counts(refs, num_pages, 0);
  for (int64_t r0 = 0; r0 < seqs; r0 += PLAN_SEQS) {
    const int rows = (int)min((int64_t)PLAN_SEQS, seqs - r0);
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
      for (int k = found + threadIdx.x; k < need; k += PLAN_THREADS) *place(k) = -1;
    }
    __threadfence();
    __syncthreads();
    if (r0 + PLAN_SEQS < seqs) counts = load_counts(refs, num_pages, 0);
  }
  if (lacking && dev_status) atomicExch(dev_status, BITNET_ERR_NO_PAGE);
}

// A page move: `rows` rows of every head, layer and pool, from page src to page dst.
struct Move {
  int32_t src, dst, rows, pad;
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
        if (rows) table[c * width + e] = -1;
      } else {
        bad = true;
      }
    }
    int total;
    const int rank = block_scan(src >= 0, total, warp_sums);
    if (src >= 0) want[rank] = Move{src, c, rows, (int)e};
    __threadfence();
    __syncthreads();
    const int found = scan_free(refs, num_pages, total, counts, warp_sums, [&](int k, int id) {
      const Move w = want[k];
      moves[made + k] = Move{w.src, id, w.rows, 0};
      table[w.dst * width + w.pad] = id;
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
  for (int i = threadIdx.x; i < tail; i += PLAN_THREADS) {
    const int src = moves[i].src, dst = moves[i].dst;
    moves[i].rows = page_size;
    place[src] = dst;
    refs[dst] = refs[src];
    refs[src] = 0;
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
  int* dev_status;
};

// One block per (move, layer, pool) at a time; a thread moves pieces of VEC bytes of the rows.
template <typename VEC>
__global__ void __launch_bounds__(256) kv_move_kernel(const MoveArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  constexpr int PER = sizeof(VEC) / 2;     // elements of a piece
  const int64_t moves = a.head ? a.head->moves : a.count;
  const int pieces = a.kv.head_dim / PER;
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
          else id = -1;
        }
        if (e != full || !part) a.table[c * a.width + e] = id;
      }
      if (lane == 0) a.len[c] = (int)used;
    }
  }
  for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
    const int pool = (int)(job & 1);
    const int64_t ml = job >> 1, move = ml / a.kv.layers;
    const int layer = (int)(ml - move * a.kv.layers);
    int src, dst, rows = a.kv.page_size;
    if (a.head) {
      src = a.moves[move].src;
      dst = a.moves[move].dst;
      rows = a.moves[move].rows;
    } else {
      src = a.src[move];
      dst = a.dst[move];
    }
    if (src < 0 || src >= a.kv.num_pages || dst < 0 || dst >= a.kv.num_pages) {
      if (threadIdx.x == 0 && a.dev_status) atomicExch(a.dev_status, BITNET_ERR_BAD_PAGE);
      continue;
    }
    uint8_t* base = (pool ? a.kv.v : a.kv.k) + 2 * layer * a.kv.stride_layer;
    const uint8_t* from = base + 2 * src * a.kv.stride_page;
    uint8_t* to = base + 2 * dst * a.kv.stride_page;
    const int units = a.kv.kv_heads * rows * pieces;
    for (int u0 = threadIdx.x; u0 < units; u0 += 256 * 4) {
      VEC w[4];
      int64_t at[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int u = u0 + 256 * j;
        if (u < units) {
          const int hr = u / pieces, h = hr / rows;
          at[j] = 2 * (h * a.kv.stride_head + (hr - h * rows) * a.kv.stride_row + (u - hr * pieces) * PER);
          w[j] = *reinterpret_cast<const VEC*>(from + at[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (u0 + 256 * j < units) *reinterpret_cast<VEC*>(to + at[j]) = w[j];
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
// `window`; otherwise the whole row, whose length becomes 0.  One warp per row; an entry is taken out by an exchange, so
// a row that is listed twice is released once.
__global__ void __launch_bounds__(256)
kv_release_kernel(int32_t* refs, int num_pages, int32_t* table, int64_t seqs, int64_t width, int32_t* len, const int32_t* list, int64_t n,
                  int page_shift, int window, int sinks, int trim, int* dev_status) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x & 31;
  const int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (i >= n) return;
  const int64_t row = list ? list[i] : i;
  if (row < 0 || row >= seqs) {
    if (lane == 0 && dev_status) atomicExch(dev_status, BITNET_ERR_BAD_PAGE);
    return;
  }
  int64_t first = 0, last = width;
  if (trim) {
    first = ((int64_t)sinks + (1 << page_shift) - 1) >> page_shift;
    last = min(width, max((int64_t)0, (int64_t)len[row] - window) >> page_shift);
  }
  for (int64_t e = first + lane; e < last; e += 32) {
    if (table[row * width + e] < 0) continue;
    const int id = atomicExch(table + row * width + e, -1);
    if (id >= 0 && id < num_pages) atomicSub(refs + id, 1);
  }
  __syncwarp();
  if (!trim && lane == 0) len[row] = 0;
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

// 16-byte pieces where a head's row is a whole number of them, 8-byte pieces otherwise (every row is a multiple of 8 bytes).
int launch_move(const MoveArgs& a, int64_t jobs, cudaStream_t st) {
  const int64_t most = (int64_t)dev_info().sm_count * 8;
  const unsigned grid = (unsigned)(jobs < 1 ? 1 : jobs < most ? jobs : most);
  log_launch("kv_move_kernel jobs=%lld grid=%u", (long long)jobs, grid);
  return a.kv.head_dim % 8 == 0 ? launch(kv_move_kernel<uint4>, grid, 256, st, a) : launch(kv_move_kernel<uint2>, grid, 256, st, a);
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
  a.dev_status = dev_status;
  const int64_t chunks = ceil_div((int64_t)kv.kv_heads * (kv.head_dim / 4), 256), blocks = ceil_div(2 * tokens * chunks, 8);
  if (blocks > 0x7fffffff) return BITNET_ERR_UNSUPPORTED_SHAPE;
  const unsigned grid = (unsigned)blocks;
  log_launch("kv_append_kernel tokens=%lld grid=%u", (long long)tokens, grid);
  if (in_dtype != BITNET_KV_F32) return launch(kv_append_kernel<__half, false>, grid, 256, st, a);   // same type: bits move
  return dtype == BITNET_KV_BF16 ? launch(kv_append_kernel<__nv_bfloat16, true>, grid, 256, st, a)
                                 : launch(kv_append_kernel<__half, true>, grid, 256, st, a);
}

int launch_kv_reserve(int32_t* refs, int64_t num_pages, int32_t* table, int64_t seqs, int64_t width, const int32_t* from_len,
                      const int32_t* to_len, int page_size, int* dev_status, cudaStream_t st) {
  log_launch("kv_reserve_kernel seqs=%lld", (long long)seqs);
  return launch(kv_reserve_kernel, 1, PLAN_THREADS, st, refs, (int)num_pages, table, seqs, width, from_len, to_len,
                __builtin_ctz((unsigned)page_size), dev_status);
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
  m.page_shift = __builtin_ctz((unsigned)kv.page_size);
  m.dev_status = dev_status;
  return launch_move(m, n * kv.layers * 2, st);
}

int launch_kv_release(int32_t* refs, int64_t num_pages, int32_t* table, int64_t seqs, int64_t width, int32_t* len, const int32_t* list,
                      int64_t n, int page_size, int window, int sinks, bool trim, int* dev_status, cudaStream_t st) {
  log_launch("kv_release_kernel rows=%lld trim=%d", (long long)n, (int)trim);
  return launch(kv_release_kernel, (unsigned)ceil_div(n, 8), 256, st, refs, (int)num_pages, table, seqs, width, len, list, n,
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
