// Attention of single tokens over a paged key-value cache, split over the cache's length and joined.
//
//   s_c = scale * <q_h, K[c, g]>,  m = max_c s_c,  l = sum_c exp(s_c - m),  o_h = sum_c exp(s_c - m) V[c, g] / l
//
// over the tokens c that the query's position p sees: c <= p, and with a window either c > p - window or c < sinks.
// Heads h of one kv head g share K and V.  Every K and V element is used for 4 * heads-per-kv-head flops, so the kernel is
// bound by HBM; the design keeps the pool streaming (64 ragged sequences of up to 8192 tokens, 64/8 heads of 128, pages of 16,
// 1.38 GB: 218 to 227 us = 6.1 to 6.35 TB/s; one of 131072: 91 to 94 us; one of 517, 32/8 heads: 11 us, all latency):
//   * the visible tokens of a row (a token and a kv head) are cut into tiles of 64; all rows' tiles together form one
//     list that is dealt to the CTAs (one per SM) in equal contiguous parts, whatever the lengths are.  The list exists only on the
//     device: every CTA derives its part from the lengths.
//   * warp 8 brings tiles in by tensor copies (one per page and pool, and per 64-column half where head_dim is not 128: with
//     pages of 16 tokens twice as many copies took 261 instead of 221 us for the 64 sequences above) into a ring of stages,
//     192 KB in flight; pages outside the visible range are not read.
//   * warps 0-3 and 4-7 take the tiles in turns, 16 tokens a warp: S = Q K^T and O += P V on mma.sync m16n8k16 with the
//     heads as the 16 rows.  At most 8 heads fill rows 0..7; rows 8..15 hold what rounding took from rows 0..7 (below).
//   * every warp keeps its own running maximum and sum; the 8 warps' states meet in shared memory when a row ends, the parts of a
//     row that lies on several CTAs in the workspace, joined by whichever part arrives last in the order of the parts (the
//     result does not depend on who that is).
// Rounding: scores, exponentials, sums and O are fp32.  The probabilities enter the second product as a 16-bit value plus a
// 16-bit remainder (rows 8..15), 16 bits for bf16 and 22 for fp16, so that a 16-bit output is rounded once for all practical
// purposes.  An fp32 query is split the same way; for a bf16 cache a third piece goes through a second product (24 bits).
// fp16 probabilities are scaled by 2^12 and fp32 queries of an fp16 cache by a power of two per row, to keep the
// remainders clear of fp16's smallest steps.
#include <cstring>
#include <type_traits>

#include "kv_cache.cuh"

namespace bitnet {
namespace {

constexpr int TILE = 64;                     // tokens per tile
constexpr int CONSUMER_WARPS = 8;
constexpr int THREADS = (CONSUMER_WARPS + 1) * 32;
constexpr int HALF_BYTES = TILE * 128;       // 64 tokens x 64 columns
constexpr int HEADS = 8;                     // query heads of one row

static __device__ int g_attn_error = 0;

struct DecodeArgs {
  const void* q;
  void* out;
  int64_t q_stride_token, q_stride_head;
  const int32_t* table;
  const int32_t* kv_len;
  const int32_t* q_start;
  int64_t table_width;
  int tokens, seqs;
  int q_heads, kv_heads, group, head_blocks;  // group = query heads per kv head, in blocks of up to 8
  int head_dim, page_shift, num_pages, layer;
  int window, sinks, max_len;                 // max_len = table_width * page_size
  int layer_pages;                            // > 0: the maps take both 64-column halves of a row in one box
  const uint8_t *k, *v;                       // DENSE: the layer's pools, and their strides in bytes
  int64_t page_bytes, head_bytes;
  int row_bytes;
  float c;                                    // scale * log2(e)
  int* counters;                              // [grid], of the row in parts that begins in a CTA; zero between calls
  float2* part_ml;                            // [2 * grid][8] running maximum and sum of a part
  float* part_o;                              // [2 * grid][8][D]
  int* dev_status;
  uint32_t give_up;                           // (test hook) the tile before which a CTA gives up
  const int* route;                           // not 0 there: the kernels of shared prefixes take the call; null: they do not
};

// The visible tokens of one row: [0, s_end) and [lo, len), as tiles; whether a window is that of a position beyond the table (whose
// tokens there are not there; without a window such a position means all of the table).
struct Range {
  int len, s_end, lo, n0, t1, tiles, seq;
  bool beyond;
};
__device__ __forceinline__ Range range_of(const DecodeArgs& a, int n) {
  Range r;
  r.seq = n;
  int64_t len;
  if (a.q_start) {
    r.seq = kv_seq_of(a.q_start, a.seqs, n);
    len = (int64_t)__ldg(a.kv_len + r.seq) - __ldg(a.q_start + r.seq + 1) + n + 1;
  } else {
    len = __ldg(a.kv_len + n);
  }
  r.len = (int)max((int64_t)0, min(len, (int64_t)a.max_len));
  r.beyond = a.window > 0 && len > a.max_len;
  r.lo = a.window > 0 ? (int)min(max((int64_t)0, len - a.window), (int64_t)r.len) : 0;
  r.s_end = min(a.sinks, r.lo);
  if (r.lo <= a.sinks) r.lo = r.s_end = 0;
  if (r.beyond && r.lo == r.len) r.lo = r.len = 0;             // the window lies beyond the table: the sinks alone
  r.n0 = (r.s_end + TILE - 1) / TILE;
  r.t1 = r.lo / TILE;
  r.tiles = max(1, r.n0 + (r.len + TILE - 1) / TILE - r.t1);   // an empty row has one tile with nothing visible
  return r;
}
// First token of tile t, and the visible part [lo, hi) of the range it belongs to.
__device__ __forceinline__ void tile_of(const Range& r, int t, int& first, int& lo, int& hi) {
  if (t < r.n0) {
    first = t * TILE;
    lo = 0;
    hi = r.s_end;
  } else {
    first = (r.t1 + t - r.n0) * TILE;
    lo = r.lo;
    hi = r.len;
  }
}

template <typename T>
struct Pair;
template <>
struct Pair<__nv_bfloat16> {
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
  }
  static __device__ __forceinline__ float2 unpack(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
  static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
};
template <>
struct Pair<__half> {
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
  }
  static __device__ __forceinline__ float2 unpack(uint32_t w) {
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
  }
  static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
};

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}

template <int DT>
struct Layout {
  static constexpr int D = DT * 16;                       // head_dim, padded
  static constexpr int HALVES = DT > 4 ? 2 : 1;
  static constexpr int TILE_BYTES = HALVES * HALF_BYTES;  // of K, and of V
  // An even number: a stage then always belongs to the same group of warps, and a warp that waits for a stage's next
  // fill has seen its previous one.  (A wait tells only the parity of a fill: with an odd number a group could take a
  // fill two rounds old for the one it wants whenever the other group's copy in between was late.)
  static constexpr int STAGES = HALVES == 2 ? 6 : 12;
  static_assert(STAGES % 2 == 0, "a stage belongs to one group");
  static constexpr int O_STRIDE = D + 8;                  // 8 heads x 4 lanes of float2 on distinct banks
  struct Tail {
    float o[4][HEADS][O_STRIDE];
    float m[4][HEADS], l[4][HEADS];
    uint2 q3[DT][32];                                     // third pieces of an fp32 query, as a lane's operand words
    uint64_t full_k[STAGES], full_v[STAGES], empty[STAGES];
    int64_t scan[CONSUMER_WARPS + 2];
    int64_t first_base;                                   // tiles before the token that the CTA's part begins in
    int64_t begin, end;
    int most[CONSUMER_WARPS + 2];
    int first_token;
    int last_part[2];
    int abort_flag;
  };
  static constexpr size_t SMEM = (size_t)STAGES * 2 * TILE_BYTES + sizeof(Tail) + 1024;
};

// KT: element type of the pools; F32: q and out are fp32; DT: head_dim in steps of 16.
// DENSE: a page's rows lie one after the other and each is an odd number of 16-byte pieces (head_dim 100: 13).  A page of a head is then one
// plain bulk copy, and ldmatrix meets distinct banks without a swizzle; tensor copies, whose 128-byte box rows begin at odd
// multiples of 16 bytes there, took 114 instead of 85 us for 9 windows of 4096 tokens, 32 heads of 100.  (Rows of one 64-column half take
// tensor copies whatever their length: not measured there.)
template <typename KT, bool F32, int DT, bool DENSE>
__global__ void __launch_bounds__(THREADS, 1)
attn_decode_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const DecodeArgs a) {
  using L = Layout<DT>;
  constexpr bool HALF_T = sizeof(KT) == 2 && !std::is_same<KT, __nv_bfloat16>::value;
  constexpr bool THREE = F32 && !HALF_T;                  // third piece
  constexpr float P_SHIFT = HALF_T ? 12.0f : 0.0f;
  using P2 = Pair<KT>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  typename L::Tail& s = *reinterpret_cast<typename L::Tail*>(smem + L::STAGES * 2 * L::TILE_BYTES);
  volatile int* abort_flag = &s.abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    for (int i = 0; i < L::STAGES; ++i) {
      kv_mbar_init(&s.full_k[i], 1);
      kv_mbar_init(&s.full_v[i], 1);
      kv_mbar_init(&s.empty[i], 4);
    }
    s.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&kmap) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&vmap) : "memory");
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (a.route && __ldcg(a.route)) return;

  // ---- the list of tiles: total, this CTA's part [item, end), and the token it begins in
  const int rows_per_token = a.kv_heads * a.head_blocks;
  int64_t total = 0;
  int longest = 0;                                         // tiles of the longest row
  int64_t my_excl = 0;                                     // of the last chunk of tokens looked at
  int my_tiles = 0, my_row = 0;
  auto scan_chunk = [&](int n0, int64_t base) {            // tiles before token n0 + tid; returns the chunk's total
    const int n = n0 + tid;
    my_row = n < a.tokens ? range_of(a, n).tiles : 0;
    my_tiles = my_row * rows_per_token;
    int64_t x = my_tiles;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, x, d);
      if (lane >= d) x += y;
    }
    const int most = __reduce_max_sync(0xffffffffu, my_row);
    __syncthreads();
    if (lane == 31) {
      s.scan[warp] = x;
      s.most[warp] = most;
    }
    __syncthreads();
    int64_t before = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < CONSUMER_WARPS + 1; ++w) {
      const int64_t v = s.scan[w];
      if (w < warp) before += v;
      sum += v;
      longest = max(longest, s.most[w]);
    }
    my_excl = base + before + x - my_tiles;
    return sum;
  };
  for (int n0 = 0; n0 < a.tokens; n0 += THREADS) total += scan_chunk(n0, total);
  // How the list is cut:
  //   short rows: at the rows' first tiles, so that no row has parts to be joined.  A join costs about 4 us, a tile 0.6 us
  //     (one sequence, 8 kv heads, 5 tiles a row: 9.8 us whole, 10.4 in parts; 9 tiles: 12.4 and 11.0; 64 ragged sequences of up to
  //     8 tiles, where every CTA has several rows: 39.4 and 45.3);
  //   few rows, all alike: as many parts of a row as fit the CTAs, so that none holds parts of two rows (4096 tokens, 8 kv
  //     heads: 18.5 -> 14.9 us);
  //   otherwise into equal parts.
  const int64_t rows = (int64_t)a.tokens * rows_per_token;
  const bool whole = longest <= 6 || (longest <= 10 && 2 * longest * (int64_t)gridDim.x <= total);
  int64_t parts = min((int64_t)gridDim.x, total);
  if (whole) parts = min((int64_t)gridDim.x, rows);
  else if (rows <= gridDim.x && total == rows * longest) parts = rows * min((int64_t)gridDim.x / rows, (int64_t)longest);
  if (blockIdx.x >= parts) return;
  const int64_t cut0 = total * blockIdx.x / parts, cut1 = total * (blockIdx.x + 1) / parts;
  auto find_cuts = [&](int n0) {
    const int64_t mine = my_excl + my_tiles;
    if (cut0 >= my_excl && cut0 < mine) {
      s.first_token = n0 + tid;
      s.first_base = my_excl;
      s.begin = whole ? my_excl + (cut0 - my_excl) / my_row * my_row : cut0;
    }
    if (cut1 == total && tid == 0) s.end = total;
    if (cut1 >= my_excl && cut1 < mine) s.end = whole ? my_excl + (cut1 - my_excl) / my_row * my_row : cut1;
  };
  if (a.tokens <= THREADS) {
    find_cuts(0);
  } else {
    int64_t base = 0;
    for (int n0 = 0; n0 < a.tokens && base <= cut1; n0 += THREADS) {
      base += scan_chunk(n0, base);
      find_cuts(n0);
    }
  }
  __syncthreads();
  const int64_t begin = s.begin, end = s.end;

  int n = s.first_token;
  int64_t base = s.first_base;                             // tiles before token n
  Range r = range_of(a, n);
  int64_t item = begin;
  uint32_t it = 0;                                         // tiles of this CTA so far

  if (warp == CONSUMER_WARPS) {
    // ------------------------------------------------------------ producer: lane = box of the tile
    const int box_rows = min(1 << a.page_shift, TILE);
    const int boxes = TILE / box_rows;
    const bool both = DENSE || (L::HALVES == 2 && a.layer_pages > 0);   // a box has both halves
    const int per_pool = both ? boxes : boxes * L::HALVES;
    const int pool = lane / per_pool;                      // 0 = K, 1 = V
    const int half = both ? 0 : lane / boxes % L::HALVES;
    const int box = lane % boxes;
    const bool mine = pool < 2;
    const uint32_t box_bytes = (uint32_t)box_rows * (DENSE ? a.row_bytes : both ? 256 : 128);
    bool stop = false;
    while (item < end && !stop) {
      const int64_t off = item - base;
      const int row = (int)(off / r.tiles);
      const int t0 = (int)(off - (int64_t)row * r.tiles);
      const int t_end = (int)min((int64_t)r.tiles, end - base - (int64_t)row * r.tiles);
      const int head = row / a.head_blocks;
      if (r.beyond && lane == 0 && a.dev_status) atomicExch(a.dev_status, BITNET_ERR_BAD_PAGE);
      // the page of a tile's box; -2: nothing visible, not read
      auto look_up = [&](int t) -> int {
        int first, lo, hi;
        tile_of(r, t, first, lo, hi);
        const int tok = first + box * box_rows;
        if (t >= t_end || !mine || tok >= hi || tok + box_rows <= lo) return -2;
        return max(__ldg(a.table + (int64_t)r.seq * a.table_width + (tok >> a.page_shift)), -1);
      };
      // (four tiles' pages are looked up while the four before are copied: one at a time the look-up's latency, 0.7 us, was
      // every tile's time)
      int page[4], next[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) page[k] = look_up(t0 + k);
      const int t_stop = (int)min((int64_t)t_end, (int64_t)t0 + (a.give_up - it));
      for (int tb = t0; tb < t_stop && !stop; tb += 4) {
#pragma unroll
        for (int k = 0; k < 4; ++k) next[k] = look_up(tb + 4 + k);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int t = tb + k, cur = page[k];
          if (t >= t_stop) break;
          const int st = it % L::STAGES;
          stop = !kv_mbar_wait_warp(&s.empty[st], ((it / L::STAGES) & 1u) ^ 1u, abort_flag, &g_attn_error);
          if (stop) break;
          ++it;
          const bool issue = cur != -2;
          const bool bad = issue && (cur < 0 || cur >= a.num_pages);
          if (bad && a.dev_status) atomicExch(a.dev_status, BITNET_ERR_BAD_PAGE);
          const unsigned mask = __ballot_sync(0xffffffffu, issue && !(DENSE && bad));
          if (DENSE && bad) {                                  // (a tensor copy from outside the pool writes zeros by itself)
            uint8_t* dst = smem + (st * 2 + pool) * L::TILE_BYTES + box * box_bytes;
            for (uint32_t i = 0; i < box_bytes; i += 16) *reinterpret_cast<uint4*>(dst + i) = make_uint4(0u, 0u, 0u, 0u);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          }
          __syncwarp();
          if (lane == 0) {
            const unsigned k_mask = (1u << per_pool) - 1u;     // (at most 16 boxes of a pool)
            kv_mbar_expect(&s.full_k[st], __popc(mask & k_mask) * box_bytes);
            kv_mbar_expect(&s.full_v[st], __popc(mask & ~k_mask) * box_bytes);
          }
          __syncwarp();
          if (issue) {
            int first, lo, hi;
            tile_of(r, t, first, lo, hi);
            const int y = (first + box * box_rows) & ((1 << a.page_shift) - 1);
            // a tile lies in shared memory as [box][half][row][64 columns]
            uint8_t* dst = smem + (st * 2 + pool) * L::TILE_BYTES + box * box_rows * (128 * L::HALVES) + half * box_rows * 128;
            uint64_t* full = pool ? &s.full_v[st] : &s.full_k[st];
            if (DENSE) {
              if (!bad)
                kv_bulk_copy(smem_u32(smem + (st * 2 + pool) * L::TILE_BYTES + box * box_bytes),
                             (pool ? a.v : a.k) + cur * a.page_bytes + head * a.head_bytes + (int64_t)y * a.row_bytes, box_bytes, full);
            } else if (both) kv_box_copy2(smem_u32(dst), pool ? &vmap : &kmap, y, head, bad ? -1 : cur + a.layer * a.layer_pages, full);
            else kv_box_copy(smem_u32(dst), pool ? &vmap : &kmap, half * 64, y, head, bad ? -1 : cur, a.layer, full);
          }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) page[k] = next[k];
      }
      if (t_stop < t_end) {
        kv_give_up(abort_flag, &g_attn_error);
        stop = true;
      }
      item += t_end - t0;
      if (row + 1 == rows_per_token && t_end == r.tiles && item < end) {
        base += (int64_t)r.tiles * rows_per_token;
        r = range_of(a, ++n);
      }
    }
    // leaves only when its copies have landed, which matters where the warps that wait for them have given up
    for (uint32_t i = it > L::STAGES ? it - L::STAGES : 0; i < it; ++i)
      for (uint32_t k = 0; k < KV_WAIT_LIMIT && !(kv_mbar_try(&s.full_k[i % L::STAGES], (i / L::STAGES) & 1u) &&
                                                 kv_mbar_try(&s.full_v[i % L::STAGES], (i / L::STAGES) & 1u)); ++k) {
      }
    return;
  }

  // -------------------------------------------------------------- consumers
  const int grp = warp >> 2;                               // takes the tiles with it % 2 == grp
  const int g = lane >> 2, t4 = lane & 3;                  // accumulator row (head) and column pair
  const int tok_w = (warp & 3) * 16;                       // this warp's tokens within a tile
  // lane's row and 16-byte piece in the ldmatrix of K (token = lane % 8 + 8 * (lane / 16), piece 2i + lane / 8 % 2) and of V
  const int k_row = tok_w + (lane & 7) + ((lane >> 4) << 3), k_piece = (lane >> 3) & 1;
  const int v_row = tok_w + (lane & 15), v_piece = lane >> 4;
  const int box_shift = min(a.page_shift, 6), half_bytes = 128 << box_shift;
  // DENSE: a row's pieces lie one after the other
  auto piece_at = [&](int row, int i0, int k, int p) -> uint32_t {       // piece 2 (i0 + k) + p of a row, i0 a multiple of 4
    if (DENSE) return (uint32_t)((2 * (i0 + k) + p) << 4);
    return (uint32_t)((i0 >> 2) * half_bytes + (((2 * k + p) ^ (row & 7)) << 4));
  };
  const uint32_t k_off = DENSE ? (uint32_t)(k_row * a.row_bytes) : (uint32_t)((k_row >> box_shift) * half_bytes * L::HALVES + (k_row & ((1 << box_shift) - 1)) * 128);
  const uint32_t v_off = DENSE ? (uint32_t)(v_row * a.row_bytes) : (uint32_t)((v_row >> box_shift) * half_bytes * L::HALVES + (v_row & ((1 << box_shift) - 1)) * 128);
  bool first_segment = true;
  struct Pending {                                         // a row of which this CTA has a part: its first, its last
    int n, head0, heads, c0, c1, first_slot;
  } pending[2];
  pending[0].n = pending[1].n = -1;
  auto write_row = [&](int tok, int h0, int heads, int hh, int d0, const float4& acc, float sum) {
    if (hh >= heads || d0 >= a.head_dim) return;
    const float inv = sum > 0.0f ? 1.0f / sum : (sum == 0.0f ? 0.0f : sum);   // nothing visible: 0; NaN stays NaN
    const int64_t at = ((int64_t)tok * a.q_heads + h0 + hh) * a.head_dim + d0;
    if (F32) {
      *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    } else {
      *reinterpret_cast<uint2*>(static_cast<KT*>(a.out) + at) =
          make_uint2(P2::pack(acc.x * inv, acc.y * inv), P2::pack(acc.z * inv, acc.w * inv));
    }
  };

  while (item < end) {
    const int64_t off = item - base;
    const int row = (int)(off / r.tiles);
    const int t0 = (int)(off - (int64_t)row * r.tiles);
    const int t_end = (int)min((int64_t)r.tiles, end - base - (int64_t)row * r.tiles);
    const int head_kv = row / a.head_blocks, block = row % a.head_blocks;
    const int heads = min(HEADS, a.group - block * HEADS);  // heads of this row
    const int head0 = head_kv * a.group + block * HEADS;

    // ---- the row's queries as operand A: rows 0..7 the values, rows 8..15 the remainders (and a third piece)
    uint32_t qa[DT][4];
    float c = a.c;
    {
      const bool have = g < heads;
      const int64_t q_at = (int64_t)n * a.q_stride_token + (int64_t)(head0 + (have ? g : 0)) * a.q_stride_head;
      if (F32) {
        float2 x[DT][2];
        const float* qp = static_cast<const float*>(a.q) + q_at;
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int d = 16 * i + 8 * j + 2 * t4;
            x[i][j] = have && d < a.head_dim ? *reinterpret_cast<const float2*>(qp + d) : make_float2(0.0f, 0.0f);
            top = fmaxf(top, fmaxf(fabsf(x[i][j].x), fabsf(x[i][j].y)));
          }
        if (HALF_T) {
          // |q| scaled into [2^13, 2^14): fp16 then holds the value and its remainder to 2^-24
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
          const int e = min(max((int)((__float_as_uint(top) >> 23) & 255) - 127 - 13, -100), 100);
          const float down = __uint_as_float((uint32_t)(127 - e) << 23);
          c *= __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
          for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) x[i][j] = make_float2(x[i][j].x * down, x[i][j].y * down);
        }
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const uint32_t h = P2::pack(x[i][j].x, x[i][j].y);
            const float2 hf = P2::unpack(h);
            const float rx = x[i][j].x - hf.x, ry = x[i][j].y - hf.y;
            const uint32_t m = P2::pack(rx, ry);
            qa[i][2 * j] = h;
            qa[i][2 * j + 1] = m;
            if (THREE && i % CONSUMER_WARPS == warp) {        // (every warp holds the same)
              const float2 mf = P2::unpack(m);
              reinterpret_cast<uint32_t*>(&s.q3[i][lane])[j] = P2::pack(rx - mf.x, ry - mf.y);
            }
          }
        if (THREE) group_barrier(1, CONSUMER_WARPS * 32);
      } else {
        const uint8_t* qp = static_cast<const uint8_t*>(a.q) + q_at * 2;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int d = 16 * i + 8 * j + 2 * t4;
            qa[i][2 * j] = have && d < a.head_dim ? *reinterpret_cast<const uint32_t*>(qp + d * 2) : 0u;
            qa[i][2 * j + 1] = 0u;
          }
      }
    }

    float o[2 * DT][4];
#pragma unroll
    for (int j = 0; j < 2 * DT; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.0f;
    float m = -INFINITY, l = 0.0f;                          // of head g over this warp's tokens (l: this lane's share)

    for (int t = t0; t < t_end; ++t, ++it) {
      if ((int)(it & 1u) != grp) continue;
      const int st = it % L::STAGES;
      const uint32_t par = (it / L::STAGES) & 1u;
      int first, lo, hi;
      tile_of(r, t, first, lo, hi);
      const uint32_t kbase = smem_u32(smem + st * 2 * L::TILE_BYTES), vbase = kbase + L::TILE_BYTES;
      kv_mbar_wait(&s.full_k[st], par, abort_flag, &g_attn_error);

      // (operands four steps at a time, so that their latencies overlap; two chains of sums for each 8 tokens)
      float sc[2][2][4] = {};
#pragma unroll
      for (int i0 = 0; i0 < DT; i0 += 4) {
        uint32_t b[4][4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (i0 + k < DT) ldsm4(kbase + k_off + piece_at(k_row, i0, k, k_piece), b[k]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int i = i0 + k;
          if (i < DT) {
            if (DENSE && 16 * i + 16 > a.head_dim) {            // beyond the row lies something else: it counts as 0
              const uint32_t m0 = 16 * i + 2 * t4 < a.head_dim ? 0xffffffffu : 0u, m1 = 16 * i + 8 + 2 * t4 < a.head_dim ? 0xffffffffu : 0u;
              b[k][0] &= m0;
              b[k][1] &= m1;
              b[k][2] &= m0;
              b[k][3] &= m1;
            }
            P2::mma(sc[k & 1][0], qa[i][0], qa[i][1], qa[i][2], qa[i][3], b[k][0], b[k][1]);
            P2::mma(sc[k & 1][1], qa[i][0], qa[i][1], qa[i][2], qa[i][3], b[k][2], b[k][3]);
            if (THREE) {
              const uint2 q3 = s.q3[i][lane];
              P2::mma(sc[k & 1 ^ 1][0], q3.x, 0u, q3.y, 0u, b[k][0], b[k][1]);
              P2::mma(sc[k & 1 ^ 1][1], q3.x, 0u, q3.y, 0u, b[k][2], b[k][3]);
            }
          }
        }
      }
      float x[4];                                           // scores of head g at tokens 2t, 2t+1, 2t+8, 2t+9 of the 16
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float hi = sc[0][j][e] + sc[1][j][e];
          x[2 * j + e] = (F32 ? hi + (sc[0][j][2 + e] + sc[1][j][2 + e]) : hi) * c;
        }
      const bool edge = first + tok_w < lo || first + tok_w + 16 > hi;   // some of the 16 tokens are not visible
      uint32_t vmask0 = 0xffffffffu, vmask1 = 0xffffffffu;
      if (edge) {
        bool in[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int tok = first + tok_w + 2 * t4 + (j & 1) + (j >> 1) * 8;
          in[j] = tok >= lo && tok < hi;
          if (!in[j]) x[j] = -INFINITY;
        }
        // V of tokens that are not visible may be anything (a page's stale end, NaN): it counts as 0
        vmask0 = (in[0] ? 0xffffu : 0u) | (in[1] ? 0xffff0000u : 0u);
        vmask1 = (in[2] ? 0xffffu : 0u) | (in[3] ? 0xffff0000u : 0u);
      }
      float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float m_new = fmaxf(m, top);
      if (__any_sync(0xffffffffu, m_new > m)) {             // the maximum rose for some head: rescale what was summed
        const float f = m_new == m ? 1.0f : exp2_approx(m - m_new);
        l *= f;
#pragma unroll
        for (int j = 0; j < 2 * DT; ++j) {
          o[j][0] *= f;
          o[j][1] *= f;
          o[j][2] *= f;
          o[j][3] *= f;
        }
        m = m_new;
      }
      const float ref = (m == -INFINITY ? 0.0f : m) - P_SHIFT;
      float p[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) p[j] = exp2_approx(x[j] - ref);
      l += (p[0] + p[1]) + (p[2] + p[3]);
      uint32_t ph[2], pm[2], pl[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        ph[j] = P2::pack(p[2 * j], p[2 * j + 1]);
        const float2 hf = P2::unpack(ph[j]);
        const float rx = p[2 * j] - hf.x, ry = p[2 * j + 1] - hf.y;
        pm[j] = P2::pack(rx, ry);
        if (THREE) {
          const float2 mf = P2::unpack(pm[j]);
          pl[j] = P2::pack(rx - mf.x, ry - mf.y);
        }
      }
      kv_mbar_wait(&s.full_v[st], par, abort_flag, &g_attn_error);
#pragma unroll
      for (int i0 = 0; i0 < DT; i0 += 4) {
        uint32_t b[4][4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (i0 + k < DT) ldsm4_t(vbase + v_off + piece_at(v_row, i0, k, v_piece), b[k]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int i = i0 + k;
          if (i < DT) {
            if (edge) {
              b[k][0] &= vmask0;
              b[k][1] &= vmask1;
              b[k][2] &= vmask0;
              b[k][3] &= vmask1;
            }
            P2::mma(o[2 * i], ph[0], pm[0], ph[1], pm[1], b[k][0], b[k][1]);
            P2::mma(o[2 * i + 1], ph[0], pm[0], ph[1], pm[1], b[k][2], b[k][3]);
            if (THREE) {
              P2::mma(o[2 * i], pl[0], 0u, pl[1], 0u, b[k][0], b[k][1]);
              P2::mma(o[2 * i + 1], pl[0], 0u, pl[1], 0u, b[k][2], b[k][3]);
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) kv_mbar_arrive(&s.empty[st]);
    }

    // ---- the warps' states meet: those of the second group join the first group's, then four are summed
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    if (!first_segment) group_barrier(1, CONSUMER_WARPS * 32);   // the previous row's states have been read
    const int ws = warp & 3;
    if (grp == 1) {
      if (t4 == 0) {
        s.m[ws][g] = m;
        s.l[ws][g] = l;
      }
#pragma unroll
      for (int j = 0; j < 2 * DT; ++j)
        *reinterpret_cast<float2*>(&s.o[ws][g][8 * j + 2 * t4]) = make_float2(o[j][0] + o[j][2], o[j][1] + o[j][3]);
    }
    group_barrier(1, CONSUMER_WARPS * 32);
    if (grp == 0) {
      const float m1 = s.m[ws][g], l1 = s.l[ws][g];
      const float top = fmaxf(m, m1);
      const float f0 = m == -INFINITY ? 0.0f : exp2_approx(m - top), f1 = m1 == -INFINITY ? 0.0f : exp2_approx(m1 - top);
      __syncwarp();
      if (t4 == 0) {
        s.m[ws][g] = top;
        s.l[ws][g] = l * f0 + l1 * f1;
      }
#pragma unroll
      for (int j = 0; j < 2 * DT; ++j) {
        float2* const at = reinterpret_cast<float2*>(&s.o[ws][g][8 * j + 2 * t4]);
        const float2 x = *at;
        *at = make_float2((o[j][0] + o[j][2]) * f0 + x.x * f1, (o[j][1] + o[j][3]) * f0 + x.y * f1);
      }
    }
    group_barrier(1, CONSUMER_WARPS * 32);

    const int hh = warp, d0 = lane * 4;                      // this thread joins 4 columns of head hh
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    float big = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) big = fmaxf(big, s.m[w][hh]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float mw = s.m[w][hh];
      const float f = mw == -INFINITY ? 0.0f : exp2_approx(mw - big);
      sum += f * s.l[w][hh];
      if (d0 < L::D) {
        const float4 v = *reinterpret_cast<const float4*>(&s.o[w][hh][d0]);
        acc.x += f * v.x;
        acc.y += f * v.y;
        acc.z += f * v.z;
        acc.w += f * v.w;
      }
    }

    if (t_end - t0 == r.tiles) {
      write_row(n, head0, heads, hh, d0, acc, sum);
    } else {
      // ---- the row lies on several CTAs: this part goes to the workspace; the last to arrive joins them, at its end
      const int slot = 2 * blockIdx.x + (first_segment ? 0 : 1);
      if (d0 < L::D) *reinterpret_cast<float4*>(a.part_o + ((int64_t)slot * HEADS + hh) * L::D + d0) = acc;
      if (lane == 0) a.part_ml[slot * HEADS + hh] = make_float2(big, sum);
      Pending& p = pending[first_segment ? 0 : 1];
      const int64_t row_begin = base + (int64_t)row * r.tiles, row_last = row_begin + r.tiles - 1;
      p.n = n;
      p.head0 = head0;
      p.heads = heads;
      p.c0 = (int)(((row_begin + 1) * parts - 1) / total);
      p.c1 = (int)(((row_last + 1) * parts - 1) / total);
      // parts of CTAs after c0 are those CTAs' first; c0's is its first too if it begins with this row
      p.first_slot = 2 * p.c0 + (total * p.c0 / parts < row_begin ? 1 : 0);
      group_barrier(1, CONSUMER_WARPS * 32);
      if (tid == 0) {
        int* counter = a.counters + p.c0;                   // (at most one row in parts begins in a CTA)
        __threadfence();                                    // (of all that the barrier ordered before)
        const int done = atomicAdd(counter, 1);
        s.last_part[first_segment ? 0 : 1] = done == p.c1 - p.c0;
        if (done == p.c1 - p.c0) *counter = 0;              // the workspace is left as it was
        __threadfence();
      }
    }
    first_segment = false;
    item += t_end - t0;
    if (row + 1 == rows_per_token && t_end == r.tiles && item < end) {
      base += (int64_t)r.tiles * rows_per_token;
      r = range_of(a, ++n);
    }
  }

  // ---- joins, in the order of the parts whoever does it
  group_barrier(1, CONSUMER_WARPS * 32);
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {
    const Pending p = pending[k];
    if (p.n < 0 || !s.last_part[k]) continue;
    const int hh = warp, d0 = lane * 4;
    float big = -INFINITY, sum = 0.0f;
    for (int cta = p.c0 + lane; cta <= p.c1; cta += 32)
      big = fmaxf(big, __ldcg(&a.part_ml[(cta == p.c0 ? p.first_slot : 2 * cta) * HEADS + hh]).x);
#pragma unroll
    for (int d = 16; d; d >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, d));
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int cta = p.c0; cta <= p.c1; ++cta) {
      const int sl = cta == p.c0 ? p.first_slot : 2 * cta;
      const float2 ml = __ldcg(&a.part_ml[sl * HEADS + hh]);
      const float f = ml.x == -INFINITY ? 0.0f : exp2_approx(ml.x - big);
      sum += f * ml.y;
      if (d0 < L::D) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(a.part_o + ((int64_t)sl * HEADS + hh) * L::D + d0));
        acc.x += f * v.x;
        acc.y += f * v.y;
        acc.z += f * v.z;
        acc.w += f * v.w;
      }
    }
    write_row(p.n, p.head0, p.heads, hh, d0, acc, sum);
  }
}

int padded_steps(int head_dim) {
  const int dt = (head_dim + 15) / 16;
  return dt <= 4 ? 4 : dt <= 6 ? 6 : dt;
}

template <typename KT, bool F32, int DT, bool DENSE = false>
int launch_one(const CUtensorMap& km, const CUtensorMap& vm, const DecodeArgs& d, int grid, cudaStream_t st) {
  auto kernel = attn_decode_kernel<KT, F32, DT, DENSE>;
  constexpr size_t smem = Layout<DT>::SMEM;
  static_assert(smem <= 232448, "shared memory of one CTA");
  static std::atomic<uint64_t> have{0};                  // devices on which the kernel may take that much shared memory
  int rc = allow_smem(kernel, (int)smem, &have);
  if (rc) return rc;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = early_start_enabled(st) ? 1 : 0;
  cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, km, vm, d);
  return e == cudaSuccess ? check_launch() : note_cuda_error(e);
}
template <typename KT, bool F32>
int launch_dt(const CUtensorMap& km, const CUtensorMap& vm, const DecodeArgs& d, int grid, cudaStream_t st) {
  if (d.row_bytes) {
    switch (padded_steps(d.head_dim)) {
      case 6: return launch_one<KT, F32, 6, true>(km, vm, d, grid, st);
      case 7: return launch_one<KT, F32, 7, true>(km, vm, d, grid, st);
      default: return launch_one<KT, F32, 8, true>(km, vm, d, grid, st);
    }
  }
  switch (padded_steps(d.head_dim)) {
    case 4: return launch_one<KT, F32, 4>(km, vm, d, grid, st);
    case 6: return launch_one<KT, F32, 6>(km, vm, d, grid, st);
    case 7: return launch_one<KT, F32, 7>(km, vm, d, grid, st);
    default: return launch_one<KT, F32, 8>(km, vm, d, grid, st);
  }
}

}  // namespace

// The parts of one call: two per CTA, whatever the call.
size_t attn_decode_parts_bytes() { return 2 * (size_t)dev_info().sm_count * HEADS * (8 + 128 * 4); }

int launch_attn_decode(const bitnet_kv_cache_t* c, const AttnArgs& x, void* ws, cudaStream_t st) {
  CUtensorMap km, vm;
  const int first = c->layer_pages > 0 ? 2 : 0;
  memcpy(&km, c->maps[first], sizeof km);
  memcpy(&vm, c->maps[first + 1], sizeof vm);
  DecodeArgs d;
  d.layer_pages = (int)c->layer_pages;
  d.k = static_cast<const uint8_t*>(c->k) + x.layer * c->stride_layer * 2;
  d.v = static_cast<const uint8_t*>(c->v) + x.layer * c->stride_layer * 2;
  d.page_bytes = 2 * c->stride_page;
  d.head_bytes = 2 * c->stride_head;
  const bool dense = c->head_dim > 64 && c->stride_row / 8 == ceil_div(c->head_dim, 8) && c->stride_row / 8 % 2 == 1;
  d.row_bytes = dense ? (int)c->stride_row * 2 : 0;
  d.q = x.q;
  d.out = x.out;
  d.q_stride_token = x.q_stride_token;
  d.q_stride_head = x.q_stride_head;
  d.table = x.table;
  d.kv_len = x.kv_len;
  d.q_start = x.q_start;
  d.table_width = x.table_width;
  d.tokens = (int)x.tokens;
  d.seqs = (int)x.seqs;
  d.q_heads = x.q_heads;
  d.kv_heads = c->kv_heads;
  d.group = x.q_heads / c->kv_heads;
  d.head_blocks = (int)ceil_div(d.group, HEADS);
  d.head_dim = c->head_dim;
  d.page_shift = __builtin_ctz((unsigned)c->page_size);
  d.num_pages = (int)c->num_pages;
  d.layer = x.layer;
  d.window = x.window;
  d.sinks = x.sinks;
  const int64_t most = x.table_width * c->page_size;
  d.max_len = most > 0x7fffff00 ? 0x7fffff00 : (int)most;
  d.c = x.scale * 1.4426950408889634f;
  const int grid = dev_info().sm_count;
  const size_t slots = 2 * (size_t)grid * HEADS;
  d.counters = attn_counters(ws);
  uint8_t* const w = attn_decode_parts(ws);
  d.part_ml = reinterpret_cast<float2*>(w);
  d.part_o = reinterpret_cast<float*>(w + slots * 8);
  d.dev_status = x.dev_status;
  d.give_up = x.give_up;
  d.route = x.route;
  log_launch("attn_decode_kernel tokens=%d q_heads=%d kv_heads=%d head_dim=%d window=%d grid=%d", d.tokens, d.q_heads, d.kv_heads, d.head_dim,
             d.window, grid);
  if (x.dtype == BITNET_KV_BF16)
    return x.io_f32 ? launch_dt<__nv_bfloat16, true>(km, vm, d, grid, st) : launch_dt<__nv_bfloat16, false>(km, vm, d, grid, st);
  return x.io_f32 ? launch_dt<__half, true>(km, vm, d, grid, st) : launch_dt<__half, false>(km, vm, d, grid, st);
}

int attn_status(int* out) {
  cudaError_t e = cudaMemcpyFromSymbol(out, g_attn_error, sizeof(int));
  return e == cudaSuccess ? BITNET_OK : note_cuda_error(e);
}
int attn_status_clear() {
  const int zero = 0;
  cudaError_t e = cudaMemcpyToSymbol(g_attn_error, &zero, sizeof(int));
  return e == cudaSuccess ? BITNET_OK : note_cuda_error(e);
}

}  // namespace bitnet
