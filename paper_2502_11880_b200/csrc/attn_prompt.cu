// Attention of prompts and chunks of prompts over a paged key-value cache, causal, with an optional sliding window and sinks, on
// the 5th-generation tensor cores.
//
//   S = Q K^T;  P = exp(scale * S - m) where visible, 0 elsewhere;  O += P V;  out = O / sum(P)
//
// in one pass over K and V with a running maximum m per row.  The rows of a tile are (token, query head) pairs of ONE kv head:
// with g query heads per kv head a tile of 128 rows holds 128 / g tokens, so K and V are read once for all heads that share them, and
// a window's edges waste fewer columns than a tile of 128 tokens would.  A work item is two such tiles that work on the same
// blocks of 128 cached tokens; one persistent CTA per SM walks items, the last (longest) first:
//   * warp 8 draws the items and brings K and V blocks in by tensor copies (one box per page and 64-column half, 128-byte
//     swizzle) into two rings;
//   * warp 9: one lane issues tcgen05.mma -- S = Q K^T from shared memory, O += P V with P in tensor memory -- for the two
//     tiles in turn, so that the tensor cores work on one tile while the other tile's exponentials are taken;
//   * warps 0-3 and 4-7, one thread per row: S from tensor memory, maximum, exponentials, P back into the tensor-memory
//     columns that S had, rows of O at the end.  O is rescaled only when a row's maximum has risen by more
//     than 2^8 (P and the sums stay below 2^8 times their range, which fp32 and both 16-bit types hold), so rarely;
//   * warps 10, 11 bring Q in for the next item, and clear the V rows of a block that no query of the item sees (the end of a page, a
//     place between the sinks and the window), since 0 * NaN would reach O.
// Bound by a tile's chain per block -- softmax, 1024 cycles of products, 650 until signals are seen -- of which two run in turn: 3100 to
// 3200 cycles a pair of blocks against 2048 of the tensor pipe (8192 tokens, 64/8 heads of 128, window 4096: 805 to 835 us = 1.0
// PFLOP/s at the 1.3 to 1.4 GHz that the power cap leaves; 4 chunks of up to 512 tokens over 5003, 32/8 heads: 76 to 83 us).  Blocks of 64 tokens
// with two buffers of S, P through shared memory, two threads per row, P in halves, S in two products of 64 columns (the first one before
// P) or a lane per tile that issues were each slower.
// Blocks that no row sees are not visited: those of the sinks, then those from the first row's window to the last row.
// Exponentials: the unit that takes them does 16 per SM and cycle, which for head_dim 128 is as long as both products take;
// a share of the columns goes through a polynomial on the fp32 units instead (2^x = 2^n * p(x - n), degree 4, relative error
// 2.6e-6, far below the rounding of P).
// Rounding: S, m, the sums and O are fp32; P is rounded to the cache's 16-bit type, which is what the tensor cores take
// as an operand beside a V of that type (a second 16-bit piece would take half as many products again); out is rounded once.
#include <cmath>
#include <cstring>
#include <type_traits>

#include "kv_cache.cuh"

namespace bitnet {
namespace {

constexpr int ROWS = 128;                     // rows of a tile (MMA M, tensor-memory lanes)
constexpr int KB = 128;                       // cached tokens of a block
constexpr int SOFT_WARPS = 8;                 // one thread per row of the two tiles
constexpr int THREADS = (SOFT_WARPS + 4) * 32;
constexpr int HALF = KB * 128;                // 128 rows x 64 columns of 16 bits
constexpr int STAGES = 2;                     // of K, and of V
constexpr int PART_BLOCKS = 4;                // fewest blocks of a part of an item
constexpr float LAZY = 8.0f;                  // log2 of how far a maximum may rise before O is rescaled

constexpr int POLY_EVERY = 8;                 // every so-manieth pair of columns takes the polynomial (none / 16th / 8th / 4th: 842 / 849 /
                                              // 831 / 854 us for the 8192 tokens above)

static __device__ int g_prompt_error = 0;

struct PromptArgs {
  const uint8_t* q;
  uint8_t* out;
  int64_t q_stride_token, q_stride_head;
  const int32_t* table;
  const int32_t* kv_len;
  const int32_t* q_start;
  int64_t table_width;
  int tokens, seqs;
  int q_heads, kv_heads, group, blocks, per_block;   // query heads per kv head, in `blocks` blocks of per_block <= 128
  int tile_tokens;                                    // tokens of a tile = 128 / per_block
  int head_dim, page_shift, num_pages, layer;
  int window, sinks, max_len;
  float c;                                            // |scale| * log2(e), above 0 so that -inf stays -inf
  int q_wide;                                         // rows of q are whole 16-byte pieces
  uint32_t q_neg;                                     // scale < 0: the products take -Q
  int room;                                           // parts of items that the workspace has room for
  int* counters;                                      // [items][8 warps]: parts that have arrived; zero between calls
  unsigned long long* drawn;                          // [0] units drawn so far, [1] CTAs that have finished; zero between calls
  float2* part_ml;                                    // [units][2 tiles][128 rows]: maximum and sum
  float4* part_o;                                     // [units][8 warps][32 pieces of 4 columns][32 rows]
  int* dev_status;
  uint32_t give_up;                                   // (test hook) the block before which a CTA gives up
};

__device__ __forceinline__ uint64_t desc_k_major(uint32_t saddr) {      // rows of 128 bytes, 128-byte swizzle
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// V as operand B: 64 columns of head_dim are contiguous per token (N-major); the next 64 lie HALF bytes further, the next 8
// tokens 1024 bytes.
__device__ __forceinline__ uint64_t desc_n_major(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(HALF >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
         (uint64_t)2 << 61;
}
// One lane of the warp, in a form that tells the compiler so: the operands of the instructions below are warp-uniform registers
// (against a test of the lane's number: 4 % of a long prompt's time).
__device__ __forceinline__ bool elect_one() {
  uint32_t e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e != 0;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(add)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(add)
      : "memory");
}
__device__ __forceinline__ void commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Waits for this thread's tensor-memory loads; the N registers count as written here, so that nothing reads them earlier.
template <int N>
__device__ __forceinline__ void wait_ld(uint32_t* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+r"(v[i]));
}
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void tm_ld32(uint32_t addr, uint32_t* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
        "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]),
        "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]),
        "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tm_st32(uint32_t addr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(addr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
      "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]),
      "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]),
      "r"(v[31])
      : "memory");
}

__device__ __forceinline__ void tm_ld16(uint32_t addr, uint32_t* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
        "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tm_st16(uint32_t addr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
      "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}

template <typename KT>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  uint32_t r;
  if (std::is_same<KT, __nv_bfloat16>::value) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Pairs of fp32 values (one instruction for two).
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 unpair(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// 2^x for x <= 2^7 by a polynomial, 0 where x rounds to -127 or less (as a hidden score, -inf, does): n = round(x) through the sum
// with 1.5 * 2^23, whose low bits are then the exponent of a factor (bits of 0 for n = -127); p is the degree-4 minimax fit (relative
// error, own exchange iteration) of 2^f on [-1/2, 1/2].  (A product by 2^n, where a sum of the exponents' bits would do for numbers,
// keeps a NaN: the sum makes FLT_MAX of it.)
__device__ __forceinline__ float2 exp2_poly(uint64_t x2) {
  float2 x = unpair(x2);
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.x) : "f"(-127.0f));
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.y) : "f"(-127.0f));
  x2 = pair(x.x, x.y);
  const uint64_t t = add2(x2, pair(12582912.0f, 12582912.0f));
  const uint64_t n = add2(t, pair(-12582912.0f, -12582912.0f));
  const uint64_t f = fma2(n, pair(-1.0f, -1.0f), x2);
  uint64_t p = fma2(f, pair(0.009570102207362652f, 0.009570102207362652f), pair(0.05591785907745361f, 0.05591785907745361f));
  p = fma2(p, f, pair(0.240247443318367f, 0.240247443318367f));
  p = fma2(p, f, pair(0.6931217908859253f, 0.6931217908859253f));
  p = fma2(p, f, pair(0.9999992847442627f, 0.9999992847442627f));
  const float2 e = unpair(t);
  return unpair(mul2(p, pair(__uint_as_float((__float_as_uint(e.x) << 23) + 0x3f800000u), __uint_as_float((__float_as_uint(e.y) << 23) + 0x3f800000u))));
}

// What a row's sum is divided by, as a factor: a row that saw nothing is 0 (as one that saw only scores of -inf), and a NaN sum stays NaN,
// also where all scores were NaN, which leaves the maximum at -inf.
__device__ __forceinline__ float inverse(float sum) { return sum == 0.0f ? 0.0f : 1.0f / sum; }

// Bits of the columns below n, of 32.
__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }
// -inf in those of 32 columns from c that a row at position p does not see.  (Selects by bits: compared column by column, with
// branches, an edge block took as long as ten others.)
__device__ __forceinline__ void hide_columns(uint32_t* x, int c, int p, int wlo, int sinks) {
  const uint32_t see = bits_below(p - c + 1) & (~bits_below(wlo - c) | bits_below(sinks - c));
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i] = see & (1u << i) ? x[i] : 0xff800000u;
}

// What a CTA works on at a time.
struct Item {
  int seq, head_kv, head0, heads;   // heads: query heads of the rows, from head0
  int q0, n_new;                    // first token and number of new tokens of the sequence
  int tok0;                         // first new token of the item
  int pos0;                         // position of new token 0
  int p_last;                       // position of the item's last token
  int lo;                           // first token that the item's first row sees through its window
  int n0, t1;                       // blocks: 0 .. n0-1 (sinks), then t1 ..
  int b0, nb;                       // the part's first block, and its blocks; nb = -1: no more items
  int two;                          // the second tile has rows
  int parts;                        // of the item, which join if there are several
  int part;
  int64_t unit0, id;                // the first part's place in the workspace, the item's number among those cut
};

template <int HALVES>
struct Layout {
  static constexpr int TILE_BYTES = HALVES * HALF;          // of Q, K, V
  static constexpr int Q_OFF = 0, K_OFF = 2 * TILE_BYTES, V_OFF = K_OFF + STAGES * TILE_BYTES, TAIL = V_OFF + STAGES * TILE_BYTES;
};
struct Tail {
  uint4 stage[SOFT_WARPS][128];                 // 32 rows x 32 columns of O on their way out, per warp
  Item item[2];
  uint64_t q_full, q_empty, k_full[STAGES], k_empty[STAGES], v_full[STAGES], v_empty[STAGES], v_clean[STAGES];
  uint64_t s_full[2], p_full[2], o_full[2], o_empty[2], item_full[2], item_empty[2], drained;
  uint32_t tmem;
  int abort_flag;
};

__device__ __forceinline__ int block_start(const Item& x, int j) {
  j += x.b0;
  return (j < x.n0 ? j : x.t1 + j - x.n0) * KB;
}
// Whether the block holds tokens that no row of the item sees, and which of its rows those are.
__device__ __forceinline__ bool unseen(const PromptArgs& a, const Item& x, int c) { return c > x.p_last || (c >= a.sinks && c < x.lo); }
__device__ __forceinline__ bool has_unseen(const PromptArgs& a, const Item& x, int c0) {
  return c0 + KB - 1 > x.p_last || (c0 < x.lo && c0 + KB > a.sinks);
}

// KT: element type of q, the pools and out; HALVES: 64-column halves of a padded row.
template <typename KT, int HALVES>
__global__ void __launch_bounds__(THREADS, 1)
attn_prompt_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const PromptArgs a) {
  using L = Layout<HALVES>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  Tail& s = *reinterpret_cast<Tail*>(smem + L::TAIL);
  volatile int* abort_flag = &s.abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    kv_mbar_init(&s.q_full, 2);
    kv_mbar_init(&s.q_empty, 1);
    for (int i = 0; i < STAGES; ++i) {
      kv_mbar_init(&s.k_full[i], 1);
      kv_mbar_init(&s.k_empty[i], 1);
      kv_mbar_init(&s.v_full[i], 1);
      kv_mbar_init(&s.v_empty[i], 3);            // the products that read it, and the two warps that look it over
      kv_mbar_init(&s.v_clean[i], 2);
    }
    for (int u = 0; u < 2; ++u) {
      kv_mbar_init(&s.s_full[u], 1);
      kv_mbar_init(&s.p_full[u], 4);
      kv_mbar_init(&s.o_full[u], 1);
      kv_mbar_init(&s.o_empty[u], 4);
      kv_mbar_init(&s.item_full[u], 1);
      kv_mbar_init(&s.item_empty[u], SOFT_WARPS + 3);
    }
    kv_mbar_init(&s.drained, 1);
    s.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&kmap) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&vmap) : "memory");
  }
  if (warp == SOFT_WARPS + 1) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t tmem = s.tmem;
  const int steps = (a.head_dim + 15) / 16;                 // of 16 columns of head_dim

  // The `it`-th item of this CTA (every role but the one that finds them); none once somebody has given up.  In the second form all
  // lanes of a warp ask, and get one answer.
  auto next_item = [&](int it) -> Item {
    kv_mbar_wait(&s.item_full[it & 1], (it >> 1) & 1u, abort_flag, &g_prompt_error);
    Item x = s.item[it & 1];
    if (*abort_flag) x.nb = -1;
    return x;
  };
  auto next_item_warp = [&](int it) -> Item {
    const bool there = kv_mbar_wait_warp(&s.item_full[it & 1], (it >> 1) & 1u, abort_flag, &g_prompt_error);
    Item x = s.item[it & 1];
    if (!there) x.nb = -1;
    return x;
  };

  if (warp >= SOFT_WARPS) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    if (warp == SOFT_WARPS) {
      // ---------------------------------------------------------- items, K and V; lane = box of a block
      const int box_rows = min(1 << a.page_shift, 64);
      const int boxes = KB / box_rows;                       // <= 16
      const int half = lane / boxes, box = lane % boxes;
      const bool mine = half < HALVES;
      const uint32_t box_bytes = (uint32_t)box_rows * 128;
      uint32_t kb = 0, kb_v = 0;                             // fills of K, of V so far
      // The items that are left when every SM has had as many as all can have (all items, if there are fewer than SMs) are cut
      // into parts of their blocks: as many as make one part per SM at most.  (8 tokens over 32768, 32/8 heads of 128: 474 us uncut, 72 in one part per
      // SM; with more parts than SMs the joins cost more than the SMs give.)
      // A lane's sequence among the 32 that end before s1: first token, tokens, context.  (Those of the last 32 are kept: with
      // look-ups for every item the first one was there 2.6 us after the start.)
      struct Seq {
        int i, q0, n, len;
      };
      auto seq_at = [&](int s1) -> Seq {
        Seq q = {s1 - 1 - lane, 0, 0, 0};
        if (q.i >= 0) {
          q.q0 = __ldg(a.q_start + q.i);
          q.n = max(0, __ldg(a.q_start + q.i + 1) - q.q0);
          q.len = __ldg(a.kv_len + q.i);
        }
        return q;
      };
      const Seq tail = seq_at(a.seqs);
      const int span = 2 * a.tile_tokens;
      int64_t pairs = (tail.n + span - 1) / span;
      for (int s1 = a.seqs - 32; s1 > 0; s1 -= 32) pairs += (seq_at(s1).n + span - 1) / span;
#pragma unroll
      for (int d = 16; d; d >>= 1) pairs += __shfl_xor_sync(0xffffffffu, pairs, d);
      const int64_t items = pairs * a.kv_heads * a.blocks;
      const int64_t uncut = a.room ? items / a.room * a.room : items, rest = items - uncut;
      const int parts = rest > 0 ? max(1, (int)(a.room / rest)) : 1;
      // A CTA draws its next unit when the last copies of one are on their way.  Without a workspace they are dealt out in rounds, every
      // other round backwards: units get shorter as they go on, and a CTA that had the longest of one round gets the shortest of the next.
      // (Rounds all forwards / there and back / drawn: 4 x 512 tokens 78.5 / 78.6 / 76.4 us, 4096 tokens, 32/4 heads 168 to 184 / 137 to
      // 165 / 141 to 149, 2048 tokens, 32/8 heads 59 / 45 to 48 / 45 to 46; a unit drawn one earlier was in between.)
      const int64_t units = uncut + rest * parts;
      int it = 0;
      for (int64_t round = 0, unit = blockIdx.x;; ++round) {
        if (round > 0) {
          if (a.room) {
            if (lane == 0) unit = gridDim.x + (int64_t)atomicAdd(a.drawn, 1ull);
            unit = __shfl_sync(0xffffffffu, unit, 0);
          } else {
            unit = round * gridDim.x + ((round & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
          }
        }
        // (a place that somebody may still read is left alone)
        if (!kv_mbar_wait_warp(&s.item_empty[it & 1], ((it >> 1) & 1u) ^ 1u, abort_flag, &g_prompt_error)) break;
        // the last sequence's last tokens first (a causal row's work grows with its position), its heads side by side
        const int heads = a.kv_heads * a.blocks;
        const bool whole = unit < uncut;
        const int64_t id = whole ? unit : uncut + (unit - uncut) / parts, want = id / heads;
        const int hb = (int)(id % heads), part = whole ? 0 : (int)((unit - uncut) % parts);
        if (lane == 0) s.item[it & 1].nb = -1;
        __syncwarp();
        bool found = false;
        int64_t before = 0;
        for (int s1 = unit < units ? a.seqs : 0; s1 > 0 && before <= want; s1 -= 32) {
          const Seq q = s1 == a.seqs ? tail : seq_at(s1);
          const int i = q.i, q0 = q.q0, n = q.n;
          const int64_t tiles = (n + span - 1) / span;
          int64_t sum = tiles;
#pragma unroll
          for (int d = 1; d < 32; d <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, sum, d);
            if (lane >= d) sum += y;
          }
          const int64_t excl = before + sum - tiles;
          const bool here = want >= excl && want < excl + tiles;
          if (here) {
            Item t;
            t.seq = i;
            t.head_kv = hb / a.blocks;
            const int b0 = hb % a.blocks * a.per_block;
            t.head0 = t.head_kv * a.group + b0;
            t.heads = min(a.per_block, a.group - b0);
            t.q0 = q0;
            t.n_new = n;
            t.tok0 = (int)(tiles - 1 - (want - excl)) * span;
            t.two = t.tok0 + a.tile_tokens < n;
            // (positions beyond the table: what their windows have of its tokens; without a window, all of them)
            const int64_t pos0 = (int64_t)q.len - n, most = a.max_len - 1;
            t.pos0 = (int)pos0;                              // |pos0| < 2^31
            t.p_last = (int)min(pos0 + min((int64_t)n, (int64_t)t.tok0 + span) - 1, most);
            t.lo = a.window > 0 ? (int)max((int64_t)0, min(pos0 + t.tok0 - a.window + 1, (int64_t)a.max_len)) : 0;
            t.n0 = t.t1 = t.b0 = t.nb = 0;
            t.unit0 = (id - uncut) * parts;                   // (used by cut items only)
            t.part = part;
            t.id = id - uncut;
            int all = 0;
            if (t.p_last >= 0) {
              t.t1 = t.lo / KB;
              t.n0 = min((min(a.sinks, t.lo) + KB - 1) / KB, t.t1);
              all = t.n0 + t.p_last / KB + 1 - t.t1;
            }
            t.parts = whole ? 1 : max(1, min(parts, all / PART_BLOCKS));
            if (part < t.parts) {
              t.b0 = (int)((int64_t)all * part / t.parts);
              t.nb = (int)((int64_t)all * (part + 1) / t.parts) - t.b0;
            } else {
              t.nb = -2;                                     // the item has fewer parts than that
            }
            s.item[it & 1] = t;
          }
          found = found || __any_sync(0xffffffffu, here);
          before += __shfl_sync(0xffffffffu, sum, 31);
        }
        __syncwarp();
        const Item x = s.item[it & 1];
        __syncwarp();
        if (found && x.nb == -2) continue;                   // (the place is free still)
        if (lane == 0) kv_mbar_arrive(&s.item_full[it & 1]);
        ++it;
        if (!found) break;
        if (a.window > 0 && lane == 0 && a.dev_status && (int64_t)x.pos0 + min(x.n_new, x.tok0 + span) > a.max_len)
          atomicExch(a.dev_status, BITNET_ERR_BAD_PAGE);
        auto look_up = [&](int j, int& y) -> int {
          const int tok = block_start(x, j) + box * box_rows;
          y = tok & ((1 << a.page_shift) - 1);
          if (!mine || tok > x.p_last || (tok >= a.sinks && tok + box_rows <= x.lo)) return -2;   // seen by no row
          return __ldg(a.table + (int64_t)x.seq * a.table_width + (tok >> a.page_shift));
        };
        int y = 0, page = x.nb > 0 ? look_up(0, y) : 0;
        const int n_stop = (int)min((int64_t)x.nb, (int64_t)(a.give_up - kb));
        bool stop = false;
        for (int j = 0; j < n_stop; ++j) {
          const int cur = page, cur_y = y;
          if (j + 1 < x.nb) page = look_up(j + 1, y);
          const bool issue = cur != -2;
          const bool bad = issue && (cur < 0 || cur >= a.num_pages);
          if (bad && a.dev_status) atomicExch(a.dev_status, BITNET_ERR_BAD_PAGE);
          const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, issue)) * box_bytes;
          const int st = kb_v % STAGES;
          const uint32_t par = ((kb_v / STAGES) & 1u) ^ 1u;
#pragma unroll
          for (int pool = 0; pool < 2; ++pool) {
            uint64_t* full = pool ? &s.v_full[st] : &s.k_full[st];
            stop = !kv_mbar_wait_warp(pool ? &s.v_empty[st] : &s.k_empty[st], par, abort_flag, &g_prompt_error);
            if (stop) break;
            if (lane == 0) kv_mbar_expect(full, bytes);
            __syncwarp();
            if (issue)
              kv_box_copy(smem_u32(smem + (pool ? L::V_OFF : L::K_OFF) + st * L::TILE_BYTES + half * HALF + box * box_bytes),
                          pool ? &vmap : &kmap, half * 64, cur_y, x.head_kv, bad ? -1 : cur, a.layer, full);
            ++(pool ? kb_v : kb);
          }
          if (stop) break;
        }
        if (n_stop < x.nb) {
          kv_give_up(abort_flag, &g_prompt_error);
          stop = true;
        }
        if (stop) break;
      }
      if (a.room && lane == 0) {                              // the workspace is left as it was
        __threadfence();
        if (atomicAdd(a.drawn + 1, 1ull) == gridDim.x - 1) a.drawn[0] = a.drawn[1] = 0;
      }
      __syncwarp();
      // leave only when the copies have landed, which matters where those that wait for them have given up
      for (uint32_t i = kb > STAGES ? kb - STAGES : 0; i < kb; ++i)
        for (uint32_t k = 0; k < KV_WAIT_LIMIT && !(kv_mbar_try(&s.k_full[i % STAGES], (i / STAGES) & 1u) &&
                                                   (i >= kb_v || kv_mbar_try(&s.v_full[i % STAGES], (i / STAGES) & 1u))); ++k) {
        }
    } else if (warp == SOFT_WARPS + 1) {
      // ---------------------------------------------------------- products
      if (elect_one()) {
        constexpr uint32_t FMT = std::is_same<KT, __nv_bfloat16>::value ? 1u : 0u;
        const uint32_t base = (1u << 4) | (FMT << 7) | (FMT << 10) | ((uint32_t)(ROWS >> 4) << 24);
        const uint32_t id_s = base | ((uint32_t)(KB >> 3) << 17) | (a.q_neg << 13);  // bit 13: operand A negated
        const uint32_t id_o = base | (1u << 16) | ((uint32_t)(steps * 2) << 17);     // N = 16 * steps, B N-major
        const uint64_t dq = desc_k_major(smem_u32(smem + L::Q_OFF));
        const uint64_t dk = desc_k_major(smem_u32(smem + L::K_OFF)), dv = desc_n_major(smem_u32(smem + L::V_OFF));
        // (rolled: the loop's own instructions hide behind the 64 cycles of each product)
        auto qk = [&](int u, uint32_t st) {
          uint64_t da = dq + (uint64_t)(u * (L::TILE_BYTES >> 4)), db = dk + (uint64_t)(st * (L::TILE_BYTES >> 4));
#pragma unroll 1
          for (int i = 0; i < steps; ++i) {
            mma_ss(tmem + u * KB, da, db, id_s, i > 0);
            const uint64_t next = (i & 3) == 3 ? (HALF - 96) >> 4 : 32 >> 4;
            da += next;
            db += next;
          }
          commit(&s.s_full[u]);
        };
        auto pv = [&](int u, uint32_t st, uint32_t add) {
          uint64_t db = dv + (uint64_t)(st * (L::TILE_BYTES >> 4));
#pragma unroll 1
          for (int i = 0; i < KB / 16; ++i) {
            mma_ts(tmem + 256 + u * 128, tmem + u * KB + 8 * i, db, id_o, add);
            add = 1;
            db += (16 * 128) >> 4;
          }
        };
        uint32_t kb = 0, cleaned = 0, items = 0;               // blocks, parities of the stages' next cleaning, items with blocks
        uint32_t p_par = 0, o_par = 3;                         // parities to wait for, one bit per tile
        for (int it = 0;; ++it) {
          const Item x = next_item(it);
          kv_mbar_arrive(&s.item_empty[it & 1]);
          if (x.nb < 0) break;
          if (x.nb == 0) continue;
          kv_mbar_wait(&s.q_full, items & 1u, abort_flag, &g_prompt_error);
          for (int j = 0; j <= x.nb; ++j) {
            const uint32_t cur = kb + j, prev = cur - 1;
            if (j < x.nb) kv_mbar_wait(&s.k_full[cur % STAGES], (cur / STAGES) & 1u, abort_flag, &g_prompt_error);
            // (before P, so that little lies between it and its product)
            if (j > 0) {
              kv_mbar_wait(&s.v_full[prev % STAGES], (prev / STAGES) & 1u, abort_flag, &g_prompt_error);
              if (has_unseen(a, x, block_start(x, j - 1))) {
                kv_mbar_wait(&s.v_clean[prev % STAGES], (cleaned >> (prev % STAGES)) & 1u, abort_flag, &g_prompt_error);
                cleaned ^= 1u << (prev % STAGES);
              }
            }
#pragma unroll 1
            for (int u = 0; u < 2; ++u) {
              if (u == 0 || x.two) {
                if (j > 0) {
                  kv_mbar_wait(&s.p_full[u], (p_par >> u) & 1u, abort_flag, &g_prompt_error);
                  p_par ^= 1u << u;
                  if (j == 1) {                                // the previous item's O has been read
                    kv_mbar_wait(&s.o_empty[u], (o_par >> u) & 1u, abort_flag, &g_prompt_error);
                    o_par ^= 1u << u;
                  }
                  fence_after();
                  pv(u, prev % STAGES, j > 1);
                  if (j == x.nb) commit(&s.o_full[u]);
                }
                if (j < x.nb) {
                  if (j == 0) fence_after();
                  qk(u, cur % STAGES);
                }
              }
            }
            if (j == x.nb - 1) commit(&s.q_empty);
            if (j > 0) commit(&s.v_empty[prev % STAGES]);
            if (j < x.nb) commit(&s.k_empty[cur % STAGES]);
          }
          kb += x.nb;
          ++items;
        }
        // all products, and their signals, before the tensor memory goes back and the CTA ends
        commit(&s.drained);
        for (uint32_t k = 0; k < KV_WAIT_LIMIT && !kv_mbar_try(&s.drained, 0); ++k) {
        }
      }
    } else {
      // ---------------------------------------------------------- Q of the next item; V rows that no query sees count as 0
      const int t = tid - (SOFT_WARPS + 2) * 32;              // 0..63
      const int u = t >> 5;
      // 16 bytes per lane where every row of q begins at a multiple of 16 and is a whole number of them, otherwise 8
      const int bytes = a.q_wide ? 16 : 8, lanes = HALVES * 128 / bytes, per = 32 / lanes;   // lanes per row, rows at a time
      const int my_row = lane / lanes, d = lane % lanes * (bytes / 2);
      uint32_t kb = 0, items = 0;
      for (int it = 0;; ++it) {
        const Item x = next_item_warp(it);
        __syncwarp();
        if (lane == 0) kv_mbar_arrive(&s.item_empty[it & 1]);
        if (x.nb < 0) break;
        if (x.nb == 0) continue;
        int64_t at[4];                                        // where rows lane, lane + 32, .. of this warp's tile begin
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int r = lane + 32 * k;
          const int rt = x.tok0 + u * a.tile_tokens + r / a.per_block, rh = r % a.per_block;
          const bool ok = r < a.tile_tokens * a.per_block && rh < x.heads && rt < x.n_new && x.q0 >= 0 && (int64_t)x.q0 + rt < a.tokens;
          at[k] = ok ? (int64_t)(x.q0 + rt) * a.q_stride_token + (int64_t)(x.head0 + rh) * a.q_stride_head : -1;
        }
        kv_mbar_wait(&s.q_empty, (items & 1u) ^ 1u, abort_flag, &g_prompt_error);
        __syncwarp();
        if (u == 0 || x.two) {
          const uint32_t dst = smem_u32(smem + L::Q_OFF + u * L::TILE_BYTES) + (d >> 6) * HALF + (d & 4) * 2;
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll 8
            for (int i = 0; i < 32; i += per) {
              const int r = i + my_row;
              const int64_t from = __shfl_sync(0xffffffffu, at[k], r);
              const bool ok = from >= 0 && d < a.head_dim;
              const uint32_t to = dst + (32 * k + r) * 128 + ((((d & 63) >> 3) ^ (r & 7)) << 4);
              const uint8_t* src = a.q + 2 * (ok ? from + d : 0);
              if (a.q_wide) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(src), "r"(ok ? 16 : 0) : "memory");
              else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(to), "l"(src), "r"(ok ? 8 : 0) : "memory");
            }
          asm volatile("cp.async.wait_all;" ::: "memory");
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        __syncwarp();
        if (lane == 0) kv_mbar_arrive(&s.q_full);
        ++items;
        for (int j = 0; j < x.nb; ++j, ++kb) {
          const int c0 = block_start(x, j), st = kb % STAGES;
          kv_mbar_wait(&s.v_full[st], (kb / STAGES) & 1u, abort_flag, &g_prompt_error);
          if (has_unseen(a, x, c0)) {
            uint8_t* v = smem + L::V_OFF + st * L::TILE_BYTES;
            for (int i = t; i < KB * 8; i += 64)
              if (unseen(a, x, c0 + (i >> 3)))
#pragma unroll
                for (int h = 0; h < HALVES; ++h) *reinterpret_cast<uint4*>(v + h * HALF + i * 16) = make_uint4(0u, 0u, 0u, 0u);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) kv_mbar_arrive(&s.v_clean[st]);
          }
          // every block is seen, not only those to be cleaned: a wait tells only a fill's parity
          __syncwarp();
          if (lane == 0) kv_mbar_arrive(&s.v_empty[st]);
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    // ------------------------------------------------------------ one thread per row
    const int u = warp >> 2, quarter = warp & 3, row = tid & 127;
    const int row_tok = row / a.per_block, hd = row % a.per_block;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const uint32_t s_addr = tmem + lanes + u * KB, o_addr = tmem + lanes + 256 + u * 128;
    const uint64_t c2 = pair(a.c, a.c);
    const bool wide = a.head_dim % 8 == 0;                    // rows of out begin at multiples of 16 bytes
    uint32_t s_cnt = 0, items = 0;
    for (int it = 0;; ++it) {
      const Item x = next_item_warp(it);
      __syncwarp();
      if (lane == 0) kv_mbar_arrive(&s.item_empty[it & 1]);
      if (x.nb < 0) break;
      const int tok = x.tok0 + u * a.tile_tokens + row_tok;
      const bool valid = row < a.tile_tokens * a.per_block && hd < x.heads && tok < x.n_new && x.q0 >= 0 && (int64_t)x.q0 + tok < a.tokens;
      if (u == 1 && !x.two) continue;
      const int64_t pos = valid ? (int64_t)x.pos0 + tok : -1;
      const int p = (int)min(pos, (int64_t)a.max_len - 1);    // last token that the row may see; < 0: sees nothing
      // first token of its window
      const int wlo = a.window > 0 ? (int)max((int64_t)0, min(pos - a.window + 1, (int64_t)a.max_len)) : 0;
      float m = -INFINITY;
      uint64_t l2 = 0;                                        // a pair of sums
      uint32_t v[64], w[64];
      for (int j = 0; j < x.nb; ++j, ++s_cnt) {
        const int c0 = block_start(x, j);
        const bool edge = __any_sync(0xffffffffu, c0 + KB - 1 > p || (c0 < wlo && c0 + KB > a.sinks));
        kv_mbar_wait(&s.s_full[u], s_cnt & 1u, abort_flag, &g_prompt_error);
        fence_after();
        // ---- the row, -inf where it does not see, and its maximum
        float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        tm_ld32(s_addr, w);
        tm_ld32(s_addr + 32, w + 32);
        wait_ld<64>(w);
        tm_ld32(s_addr + 64, v);
        tm_ld32(s_addr + 96, v + 32);
        auto mask = [&](uint32_t* x, int c) {
          hide_columns(x, c, p, wlo, a.sinks);
          hide_columns(x + 32, c + 32, p, wlo, a.sinks);
        };
        auto maxima = [&](const uint32_t* x) {
#pragma unroll
          for (int i = 0; i < 64; i += 8)
#pragma unroll
            for (int k = 0; k < 4; ++k) top[k] = fmaxf(fmaxf(top[k], __uint_as_float(x[i + 2 * k])), __uint_as_float(x[i + 2 * k + 1]));
        };
        if (edge) mask(w, c0);
        maxima(w);
        wait_ld<64>(v);
        if (edge) mask(v, c0 + 64);
        maxima(v);
        const float big = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
        const float m_new = fmaxf(m, big * a.c);
        if (__any_sync(0xffffffffu, m_new > m + LAZY)) {
          const float f = m == -INFINITY ? 0.0f : exp2_approx(m - m_new);   // (-inf before the first visible token: O is 0)
          m = m_new;
          l2 = fma2(l2, pair(f, f), 0);
          if (j > 0) {
#pragma unroll 1
            for (int i = 0; i < steps * 16; i += 16) {
              uint32_t o[16];
              tm_ld16(o_addr + i, o);
              wait_ld<16>(o);
#pragma unroll
              for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
              tm_st16(o_addr + i, o);
            }
          }
        }
        const float ref = m == -INFINITY ? 0.0f : m;
        const uint64_t r2 = pair(-ref, -ref);
        // ---- exponentials of 64 columns, which become 32 of P
        auto exps = [&](uint32_t* x) {
#pragma unroll
          for (int i = 0; i < 64; i += 2) {
            const uint64_t e = fma2(pair(__uint_as_float(x[i]), __uint_as_float(x[i + 1])), c2, r2);
            float2 y;
            if ((i >> 1) % POLY_EVERY == POLY_EVERY - 1) {
              y = exp2_poly(e);
            } else {
              y = unpair(e);
              y.x = exp2_approx(y.x);
              y.y = exp2_approx(y.y);
            }
            l2 = add2(l2, pair(y.x, y.y));
            x[i >> 1] = pack16<KT>(y.x, y.y);
          }
        };
        exps(v);
        tm_st32(s_addr + 32, v);
        exps(w);
        tm_st32(s_addr, w);
        wait_st();
        fence_before();
        __syncwarp();
        if (lane == 0) kv_mbar_arrive(&s.p_full[u]);
      }

      float inv = 0.0f;
      float top_all = m;                                      // maximum of all parts
      bool mine_to_write = true;
      if (x.nb > 0) {
        const float2 l = unpair(l2);
        const float sum = l.x + l.y;
        inv = inverse(sum);
        kv_mbar_wait(&s.o_full[u], items & 1u, abort_flag, &g_prompt_error);
        fence_after();
        ++items;
        if (x.parts > 1) {
          // ---- a part: each warp's last part to arrive joins its 32 rows, in the order of the parts; its own stay in tensor memory, and
          //      go to the workspace only if the others are not known to be there yet
          int* const counter = a.counters + x.id * 8 + warp;
          int last = 0;
          if (lane == 0) {
            last = *reinterpret_cast<volatile int*>(counter) == x.parts - 1;
            __threadfence();
          }
          last = __shfl_sync(0xffffffffu, last, 0);
          if (!last) {
            float4* const mine = a.part_o + ((x.unit0 + x.part) * 8 + warp) * 1024 + lane;
            a.part_ml[((x.unit0 + x.part) * 2 + u) * ROWS + row] = make_float2(m, sum);
#pragma unroll 1
            for (int i = 0; i < steps * 16; i += 32) {
              tm_ld32(o_addr + i, v);
              wait_ld<32>(v);
#pragma unroll
              for (int k = 0; k < 8; ++k)
                mine[(i / 4 + k) * 32] = make_float4(__uint_as_float(v[4 * k]), __uint_as_float(v[4 * k + 1]), __uint_as_float(v[4 * k + 2]),
                                                     __uint_as_float(v[4 * k + 3]));
            }
            __syncwarp();
            if (lane == 0) {
              __threadfence();                                // (of all that the warp's barrier ordered before)
              last = atomicAdd(counter, 1) == x.parts - 1;
              __threadfence();
            }
            last = __shfl_sync(0xffffffffu, last, 0);
          }
          __syncwarp();
          mine_to_write = last;
          if (last) {
            if (lane == 0) *counter = 0;                      // the workspace is left as it was
            const float2* const ml = a.part_ml + (x.unit0 * 2 + u) * ROWS + row;
            float all = 0.0f;
#pragma unroll 4
            for (int k = 0; k < x.parts; ++k) top_all = fmaxf(top_all, k == x.part ? m : __ldcg(ml + k * 2 * ROWS).x);
#pragma unroll 4
            for (int k = 0; k < x.parts; ++k) {
              const float2 y = k == x.part ? make_float2(m, sum) : __ldcg(ml + k * 2 * ROWS);
              all += (y.x == -INFINITY ? 0.0f : exp2_approx(y.x - top_all)) * y.y;    // (y.y may be NaN)
            }
            inv = inverse(all);
          }
        }
      }
      // ---- O, 32 columns at a time, through this warp's staging rows and out as whole sectors
      const int64_t at = valid ? ((int64_t)(x.q0 + tok) * a.q_heads + x.head0 + hd) * a.head_dim : -1;
      const int piece = lane & 3;                             // 8 columns; rows 8 k + lane / 4
      int64_t to[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        to[k] = __shfl_sync(0xffffffffu, at, 8 * k + (lane >> 2));
        to[k] = to[k] < 0 ? -1 : to[k] + piece * 8;
      }
      uint4* const stage = s.stage[warp];
#pragma unroll 1
      for (int i = 0; i < steps * 16 && mine_to_write; i += 32) {
        uint32_t* const o = v;
        if (x.parts == 1) {
          if (x.nb > 0) tm_ld32(o_addr + i, o);
          wait_ld<32>(o);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0u;
#pragma unroll 1
          for (int k = 0; k < x.parts; ++k) {
            const float mk = k == x.part ? m : __ldcg(a.part_ml + ((x.unit0 + k) * 2 + u) * ROWS + row).x;
            if (k == x.part) {
              tm_ld32(o_addr + i, w);
              wait_ld<32>(w);
            } else {
              const float4* const from = a.part_o + ((x.unit0 + k) * 8 + warp) * 1024 + lane + (i / 4) * 32;
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float4 y = __ldcg(from + e * 32);
                w[4 * e] = __float_as_uint(y.x);
                w[4 * e + 1] = __float_as_uint(y.y);
                w[4 * e + 2] = __float_as_uint(y.z);
                w[4 * e + 3] = __float_as_uint(y.w);
              }
            }
            const float f = mk == -INFINITY ? 0.0f : exp2_approx(mk - top_all);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(fmaf(f, __uint_as_float(w[e]), __uint_as_float(o[e])));
          }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e)
          o[e] = inv == 0.0f ? 0u : pack16<KT>(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv);
#pragma unroll
        for (int k = 0; k < 4; ++k) stage[lane * 4 + (k ^ ((lane >> 1) & 3))] = make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
        __syncwarp();
        uint4 y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = stage[(8 * k + (lane >> 2)) * 4 + (piece ^ ((lane >> 3) & 3))];
        __syncwarp();
        const int left = a.head_dim - i - piece * 8;      // columns from this piece on
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint8_t* const dst = a.out + 2 * (to[k] + i);
          if (to[k] < 0 || left <= 0) continue;
          if (wide) {
            *reinterpret_cast<uint4*>(dst) = y[k];
          } else {
            *reinterpret_cast<uint2*>(dst) = make_uint2(y[k].x, y[k].y);
            if (left > 4) *reinterpret_cast<uint2*>(dst + 8) = make_uint2(y[k].z, y[k].w);
          }
        }
      }
      if (x.nb > 0) {
        fence_before();
        __syncwarp();
        if (lane == 0) kv_mbar_arrive(&s.o_empty[u]);         // O has been read
      }
    }
  }

  // ---- every role has left its loop (all waits are bounded); free the tensor memory
  fence_before();
  __syncthreads();
  fence_after();
  if (warp == SOFT_WARPS + 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

template <typename KT, int HALVES>
int launch_one(const CUtensorMap& km, const CUtensorMap& vm, const PromptArgs& a, int64_t grid, cudaStream_t st) {
  auto kernel = attn_prompt_kernel<KT, HALVES>;
  constexpr size_t smem = Layout<HALVES>::TAIL + sizeof(Tail) + 1024;
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
  cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, km, vm, a);
  return e == cudaSuccess ? check_launch() : note_cuda_error(e);
}

}  // namespace

static constexpr size_t PART_BYTES = 2 * ROWS * 8 + 8 * 1024 * 16;

// Room for the parts of a call: one part per SM.  None where a pair of tiles is more than half as many items (kv heads, blocks of query
// heads) as there are SMs: a call of one pair is not cut then.  (The rest of a call of several pairs could be -- two pairs of 80 items
// leave 12 beyond 148 -- and is not.)
size_t attn_prompt_parts_bytes(int64_t tokens, int q_heads, int kv_heads) {
  const int64_t least = (int64_t)kv_heads * ceil_div(q_heads / kv_heads, ROWS), sms = dev_info().sm_count;
  return tokens > 0 && 2 * least <= sms ? (size_t)sms * PART_BYTES : 0;
}

int launch_attn_prompt(const bitnet_kv_cache_t* c, const AttnArgs& x, void* ws, size_t ws_bytes, cudaStream_t st) {
  CUtensorMap km, vm;
  memcpy(&km, c->maps[0], sizeof km);
  memcpy(&vm, c->maps[1], sizeof vm);
  PromptArgs a;
  a.q = static_cast<const uint8_t*>(x.q);
  a.out = static_cast<uint8_t*>(x.out);
  a.q_stride_token = x.q_stride_token;
  a.q_stride_head = x.q_stride_head;
  a.table = x.table;
  a.kv_len = x.kv_len;
  a.q_start = x.q_start;
  a.table_width = x.table_width;
  a.tokens = (int)x.tokens;
  a.seqs = (int)x.seqs;
  a.q_heads = x.q_heads;
  a.kv_heads = c->kv_heads;
  a.group = x.q_heads / c->kv_heads;
  a.blocks = (int)ceil_div(a.group, ROWS);
  a.per_block = (int)ceil_div(a.group, a.blocks);
  a.tile_tokens = ROWS / a.per_block;
  a.head_dim = c->head_dim;
  a.page_shift = __builtin_ctz((unsigned)c->page_size);
  a.num_pages = (int)c->num_pages;
  a.layer = x.layer;
  a.window = x.window;
  a.sinks = x.sinks;
  const int64_t most = x.table_width * c->page_size;
  a.max_len = most > 0x3fffff00 ? 0x3fffff00 : (int)most;
  a.q_wide = c->head_dim % 8 == 0 && x.q_stride_token % 8 == 0 && x.q_stride_head % 8 == 0;
  a.q_neg = x.scale < 0.0f ? 1u : 0u;
  a.c = fmaxf(fabsf(x.scale) * 1.4426950408889634f, 1e-30f);
  a.dev_status = x.dev_status;
  a.give_up = x.give_up;
  // a sequence has at most one pair of tiles that is not full; which CTA has which, in how many parts, is found on the device
  const int64_t pairs = x.tokens / (2 * a.tile_tokens) + (x.seqs < x.tokens ? x.seqs : x.tokens);
  const int64_t sms = dev_info().sm_count, items = pairs * a.kv_heads * a.blocks;
  a.room = ws_bytes >= attn_decode_workspace_bytes() + (size_t)sms * PART_BYTES ? (int)sms : 0;
  a.counters = attn_counters(ws);
  a.drawn = reinterpret_cast<unsigned long long*>(static_cast<uint8_t*>(ws) + attn_counters_bytes()) - 2;
  a.part_o = reinterpret_cast<float4*>(attn_prompt_parts(ws));
  a.part_ml = reinterpret_cast<float2*>(attn_prompt_parts(ws) + (size_t)sms * (8 * 1024 * 16));
  const int64_t grid = a.room || items > sms ? sms : items;
  log_launch("attn_prompt_kernel tokens=%d q_heads=%d kv_heads=%d head_dim=%d window=%d grid=%lld", a.tokens, a.q_heads, a.kv_heads,
             a.head_dim, a.window, (long long)grid);
  const bool two = a.head_dim > 64;
  if (x.dtype == BITNET_KV_BF16) return two ? launch_one<__nv_bfloat16, 2>(km, vm, a, grid, st) : launch_one<__nv_bfloat16, 1>(km, vm, a, grid, st);
  return two ? launch_one<__half, 2>(km, vm, a, grid, st) : launch_one<__half, 1>(km, vm, a, grid, st);
}

int attn_prompt_status(int* out) {
  cudaError_t e = cudaMemcpyFromSymbol(out, g_prompt_error, sizeof(int));
  return e == cudaSuccess ? BITNET_OK : note_cuda_error(e);
}
int attn_prompt_status_clear() {
  const int zero = 0;
  cudaError_t e = cudaMemcpyToSymbol(g_prompt_error, &zero, sizeof(int));
  return e == cudaSuccess ? BITNET_OK : note_cuda_error(e);
}

}  // namespace bitnet
