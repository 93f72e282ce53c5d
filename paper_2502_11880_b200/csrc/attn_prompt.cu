// Attention of prompts and chunks of prompts over a paged key-value cache, causal, with an optional sliding window and sinks, on
// the 5th-generation tensor cores.
//
//   S = Q K^T;  P = exp(scale * S - m) where visible, 0 elsewhere;  O += P V;  out = O / sum(P)
//
// in one pass over K and V with a running maximum m per row.  The rows of a tile are (token, query head) pairs of ONE kv head:
// with g query heads per kv head a tile of 128 rows holds 128 / g tokens, so K and V are read once for all heads that share them, and
// a window's edges waste fewer columns than a tile of 128 tokens would.  A CTA has two such tiles that work on the same
// blocks of 128 cached tokens:
//   * warp 8: tensor copies of K and V blocks (one box per page and 64-column half, 128-byte swizzle) into two rings;
//   * warp 9: one thread issues tcgen05.mma -- S = Q K^T from shared memory, O += P V with P in tensor memory -- for the two
//     tiles in turn, so that the tensor cores work on one tile while the other tile's exponentials are taken;
//   * warps 0-3 and 4-7, one row per thread: the row of S from tensor memory, mask, maximum, exponentials, P back into the
//     tensor-memory columns that S had, rows of O at the end.  O is rescaled only when a row's maximum has risen by more
//     than 2^8 (P and the sums stay below 2^8 times their range, which fp32 and both 16-bit types hold), so rarely;
//   * warps 10, 11 clear the V rows of a block that no query of the CTA sees (the end of a page, a place between the sinks
//     and the window), since 0 * NaN would reach O.
// Blocks that no row sees are not visited: those of the sinks, then those from the first row's window to the last row.
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
constexpr int THREADS = 384;
constexpr int HALF = KB * 128;                // 128 rows x 64 columns of 16 bits
constexpr int STAGES = 2;                     // of K, and of V
constexpr float LAZY = 8.0f;                  // log2 of how far a maximum may rise before O is rescaled

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
  uint32_t q_sign;                                    // flips q where scale < 0
  int* dev_status;
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
// One lane of the warp, in a form that tells the compiler so: the operands of the instructions below are warp-uniform registers,
// and behind a test of the lane's number each of them would be brought there by a loop over the lanes (measured: 130
// instead of 64 cycles per product issued).
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
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
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

template <typename KT>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  uint32_t r;
  if (std::is_same<KT, __nv_bfloat16>::value) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// What a CTA works on.
struct Item {
  int seq, head_kv, head0, heads;   // heads: query heads of the rows, from head0
  int q0, n_new;                    // first token and number of new tokens of the sequence
  int tok0;                         // first new token of the CTA
  int pos0;                         // position of new token 0
  int p_last;                       // position of the CTA's last token
  int lo;                           // first token that the CTA's first row sees through its window
  int n0, t1, nb;                   // blocks: 0 .. n0-1 (sinks), then t1 ..; nb in all
};

template <int HALVES>
struct Layout {
  static constexpr int TILE_BYTES = HALVES * HALF;          // of Q, K, V
  static constexpr int Q_OFF = 0, K_OFF = 2 * TILE_BYTES, V_OFF = K_OFF + STAGES * TILE_BYTES, TAIL = V_OFF + STAGES * TILE_BYTES;
};
struct Tail {
  uint64_t q_full, k_full[STAGES], k_empty[STAGES], v_full[STAGES], v_empty[STAGES], v_clean[STAGES], s_full[2], p_full[2], o_full[2];
  Item item;
  uint32_t tmem;
  int abort_flag, found;
};

__device__ __forceinline__ int block_start(const Item& x, int j) { return (j < x.n0 ? j : x.t1 + j - x.n0) * KB; }
// Whether the block holds tokens that no row of the CTA sees, and which of its rows those are.
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
    kv_mbar_init(&s.q_full, 8);
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
    }
    s.abort_flag = 0;
    s.found = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&kmap) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&vmap) : "memory");
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // ---- which tile pair this CTA has: the last sequence's last first (a causal row's work grows with its position)
  if (warp == 8) {
    const int heads = a.kv_heads * a.blocks;
    const int64_t want = blockIdx.x / heads;
    const int hb = blockIdx.x % heads;
    const int span = 2 * a.tile_tokens;
    int64_t before = 0;
    for (int s1 = a.seqs; s1 > 0 && before <= want; s1 -= 32) {
      const int i = s1 - 1 - lane;
      const int q0 = i >= 0 ? __ldg(a.q_start + i) : 0;
      const int n = i >= 0 ? max(0, __ldg(a.q_start + i + 1) - q0) : 0;
      const int64_t tiles = (n + span - 1) / span;
      int64_t x = tiles;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
      }
      const int64_t excl = before + x - tiles;
      if (want >= excl && want < excl + tiles) {
        Item t;
        t.seq = i;
        t.head_kv = hb / a.blocks;
        const int b0 = hb % a.blocks * a.per_block;
        t.head0 = t.head_kv * a.group + b0;
        t.heads = min(a.per_block, a.group - b0);
        t.q0 = q0;
        t.n_new = n;
        t.tok0 = (int)(tiles - 1 - (want - excl)) * span;
        const int64_t pos0 = (int64_t)__ldg(a.kv_len + i) - n;
        t.pos0 = (int)pos0;                                // |pos0| < 2^31: both terms are at least 0 or the sequence is empty
        const int64_t most = a.max_len - 1;
        t.p_last = (int)min(pos0 + min((int64_t)n, (int64_t)t.tok0 + span) - 1, most);
        t.lo = a.window > 0 ? (int)max((int64_t)0, min(pos0 + t.tok0, most) - a.window + 1) : 0;
        t.n0 = t.t1 = t.nb = 0;
        if (t.p_last >= 0) {
          t.t1 = t.lo / KB;
          t.n0 = min((min(a.sinks, t.lo) + KB - 1) / KB, t.t1);
          t.nb = t.n0 + t.p_last / KB + 1 - t.t1;
        }
        s.item = t;
        s.found = 1;
      }
      before += __shfl_sync(0xffffffffu, x, 31);
    }
  }
  if (warp == 9) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = s.tmem;
  const Item x = s.item;
  const int nb = s.found ? x.nb : 0;
  const int steps = (a.head_dim + 15) / 16;                 // of 16 columns of head_dim

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    if (warp == 8) {
      // ---------------------------------------------------------- producer: lane = box of a block
      const int box_rows = min(1 << a.page_shift, 64);
      const int boxes = KB / box_rows;                       // <= 16
      const int half = lane / boxes, box = lane % boxes;
      const bool mine = half < HALVES;
      const uint32_t box_bytes = (uint32_t)box_rows * 128;
      auto look_up = [&](int j, int& y) -> int {
        const int tok = block_start(x, j) + box * box_rows;
        y = tok & ((1 << a.page_shift) - 1);
        if (!mine || tok > x.p_last || (tok >= a.sinks && tok + box_rows <= x.lo)) return -2;   // seen by no row
        return __ldg(a.table + (int64_t)x.seq * a.table_width + (tok >> a.page_shift));
      };
      int y = 0, page = nb > 0 ? look_up(0, y) : 0;
      for (int j = 0; j < nb; ++j) {
        const int cur = page, cur_y = y;
        if (j + 1 < nb) page = look_up(j + 1, y);
        const bool issue = cur != -2;
        const bool bad = issue && (cur < 0 || cur >= a.num_pages);
        if (bad && a.dev_status) atomicExch(a.dev_status, BITNET_ERR_BAD_PAGE);
        const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, issue)) * box_bytes;
        const int st = j % STAGES;
        const uint32_t par = ((j / STAGES) & 1u) ^ 1u;
#pragma unroll
        for (int pool = 0; pool < 2; ++pool) {
          uint64_t* full = pool ? &s.v_full[st] : &s.k_full[st];
          kv_mbar_wait(pool ? &s.v_empty[st] : &s.k_empty[st], par, abort_flag, &g_prompt_error);
          __syncwarp();
          if (*abort_flag) continue;
          if (lane == 0) kv_mbar_expect(full, bytes);
          __syncwarp();
          if (issue)
            kv_box_copy(smem_u32(smem + (pool ? L::V_OFF : L::K_OFF) + st * L::TILE_BYTES + half * HALF + box * box_bytes),
                        pool ? &vmap : &kmap, half * 64, cur_y, x.head_kv, bad ? -1 : cur, a.layer, full);
        }
      }
      if (*abort_flag)                                        // leave only when the copies have landed
        for (int j = max(0, nb - STAGES); j < nb; ++j)
          for (uint32_t k = 0; k < KV_WAIT_LIMIT && !(kv_mbar_try(&s.k_full[j % STAGES], (j / STAGES) & 1u) &&
                                                     kv_mbar_try(&s.v_full[j % STAGES], (j / STAGES) & 1u)); ++k) {
          }
    } else if (warp == 9) {
      // ---------------------------------------------------------- MMA issuer
      if (nb > 0 && elect_one()) {
        constexpr uint32_t FMT = std::is_same<KT, __nv_bfloat16>::value ? 1u : 0u;
        const uint32_t base = (1u << 4) | (FMT << 7) | (FMT << 10) | ((uint32_t)(ROWS >> 4) << 24);
        const uint32_t id_s = base | ((uint32_t)(KB >> 3) << 17);
        const uint32_t id_o = base | (1u << 16) | ((uint32_t)(steps * 2) << 17);     // N = 16 * steps, B N-major
        const uint32_t q_addr = smem_u32(smem + L::Q_OFF);
        uint32_t cleaned = 0;                                  // parity of each stage's next cleaning
        const uint64_t dq = desc_k_major(q_addr);
        const uint64_t dk = desc_k_major(smem_u32(smem + L::K_OFF)), dv = desc_n_major(smem_u32(smem + L::V_OFF));
        auto qk = [&](int u, int st) {
          const uint64_t da = dq + (uint64_t)(u * (L::TILE_BYTES >> 4)), db = dk + (uint64_t)(st * (L::TILE_BYTES >> 4));
#pragma unroll
          for (int i = 0; i < 4 * HALVES; ++i)
            if (i < steps) mma_ss(tmem + u * KB, da + (((i >> 2) * HALF + (i & 3) * 32) >> 4), db + (((i >> 2) * HALF + (i & 3) * 32) >> 4), id_s, i > 0);
          commit(&s.s_full[u]);
        };
        auto pv = [&](int u, int st, uint32_t add) {
          const uint64_t db = dv + (uint64_t)(st * (L::TILE_BYTES >> 4));
#pragma unroll
          for (int i = 0; i < KB / 16; ++i)
            mma_ts(tmem + 256 + u * 128, tmem + u * KB + 8 * i, db + ((i * 16 * 128) >> 4), id_o, i > 0 ? 1u : add);
        };
        auto wait_v = [&](int j) {
          kv_mbar_wait(&s.v_full[j % STAGES], (j / STAGES) & 1u, abort_flag, &g_prompt_error);
          if (has_unseen(a, x, block_start(x, j))) {
            kv_mbar_wait(&s.v_clean[j % STAGES], (cleaned >> (j % STAGES)) & 1u, abort_flag, &g_prompt_error);
            cleaned ^= 1u << (j % STAGES);
          }
        };
        kv_mbar_wait(&s.q_full, 0, abort_flag, &g_prompt_error);
        for (int j = 0; j <= nb; ++j) {
          if (j < nb) kv_mbar_wait(&s.k_full[j % STAGES], (j / STAGES) & 1u, abort_flag, &g_prompt_error);
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            if (j > 0) {
              kv_mbar_wait(&s.p_full[u], (j - 1) & 1u, abort_flag, &g_prompt_error);
              if (u == 0) wait_v(j - 1);
              fence_after();
              pv(u, (j - 1) % STAGES, j > 1);
              if (j == nb) commit(&s.o_full[u]);
            }
            if (j < nb) {
              if (j == 0) fence_after();
              qk(u, j % STAGES);
            }
          }
          if (j > 0) commit(&s.v_empty[(j - 1) % STAGES]);
          if (j < nb) commit(&s.k_empty[j % STAGES]);
        }
      }
    } else {
      // ---------------------------------------------------------- V rows that no query sees count as 0
      const int t = tid - 320;                                // 0..63
      for (int j = 0; j < nb; ++j) {
        const int c0 = block_start(x, j);
        kv_mbar_wait(&s.v_full[j % STAGES], (j / STAGES) & 1u, abort_flag, &g_prompt_error);
        if (has_unseen(a, x, c0)) {
          uint8_t* v = smem + L::V_OFF + (j % STAGES) * L::TILE_BYTES;
          for (int i = t; i < KB * 8; i += 64)
            if (unseen(a, x, c0 + (i >> 3)))
#pragma unroll
              for (int h = 0; h < HALVES; ++h) *reinterpret_cast<uint4*>(v + h * HALF + i * 16) = make_uint4(0u, 0u, 0u, 0u);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) kv_mbar_arrive(&s.v_clean[j % STAGES]);
        }
        // every block is seen, not only those to be cleaned: a wait tells only a fill's parity
        __syncwarp();
        if (lane == 0) kv_mbar_arrive(&s.v_empty[j % STAGES]);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    // ------------------------------------------------------------ one row per thread
    const int u = warp >> 2, row = tid & 127;
    const int tok = x.tok0 + u * a.tile_tokens + row / a.per_block, hd = row % a.per_block;
    const bool valid = s.found && row < a.tile_tokens * a.per_block && hd < x.heads && tok < x.n_new && x.q0 >= 0 &&
                       (int64_t)x.q0 + tok < a.tokens;
    const int p = valid ? (int)min((int64_t)x.pos0 + tok, (int64_t)a.max_len - 1) : -1;   // position; < 0 sees nothing
    const int wlo = a.window > 0 ? max(0, p - a.window + 1) : 0;         // first token of its window

    // ---- Q: the warp's 32 rows, one row of 8 bytes per lane at a time, into the swizzled layout of operand A
    uint8_t* const stage = smem + L::Q_OFF + u * L::TILE_BYTES + (warp & 3) * 32 * 128;   // this warp's rows of the tile
    auto staged = [&](int r, int d) { return stage + (d >> 6) * HALF + r * 128 + ((((d & 63) >> 3) ^ (r & 7)) << 4) + (d & 4) * 2; };
    if (nb > 0) {
      const int64_t at = valid ? (int64_t)(x.q0 + tok) * a.q_stride_token + (int64_t)(x.head0 + hd) * a.q_stride_head : -1;
      const int d = lane * 4;
#pragma unroll
      for (int i0 = 0; i0 < 32; i0 += 16) {
        uint2 w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int64_t from = __shfl_sync(0xffffffffu, at, i0 + i);
          w[i] = from >= 0 && d < a.head_dim ? __ldg(reinterpret_cast<const uint2*>(a.q + 2 * (from + d))) : make_uint2(0u, 0u);
        }
        if (d < HALVES * 64)
#pragma unroll
          for (int i = 0; i < 16; ++i) *reinterpret_cast<uint2*>(staged(i0 + i, d)) = make_uint2(w[i].x ^ a.q_sign, w[i].y ^ a.q_sign);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) kv_mbar_arrive(&s.q_full);
    }

    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem + lanes + u * KB, o_addr = tmem + lanes + 256 + u * 128;
    float m = -INFINITY, l = 0.0f;
    for (int j = 0; j < nb; ++j) {
      kv_mbar_wait(&s.s_full[u], j & 1u, abort_flag, &g_prompt_error);
      fence_after();
      uint32_t v[KB];
#pragma unroll
      for (int i = 0; i < KB; i += 32) tm_ld32(s_addr + i, v + i);
      wait_ld();
      const int c0 = block_start(x, j);
      const bool edge = c0 + KB - 1 > p || (c0 < wlo && c0 + KB > a.sinks);
      if (__any_sync(0xffffffffu, edge)) {
        const int hi = p - c0, lo = wlo - c0, sk = a.sinks - c0;
#pragma unroll
        for (int i = 0; i < KB; ++i)
          if (!(i <= hi && (i >= lo || i < sk))) v[i] = 0xff800000u;
      }
      float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int i = 0; i < KB; ++i) top[i & 3] = fmaxf(top[i & 3], __uint_as_float(v[i]));
      const float big = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
      const float m_new = fmaxf(m, big * a.c);
      if (__any_sync(0xffffffffu, m_new > m + LAZY)) {
        const float f = m == -INFINITY ? 0.0f : exp2_approx(m - m_new);   // (-inf before the first visible token: O is 0)
        m = m_new;
        l *= f;
        if (j > 0) {
#pragma unroll 1
          for (int i = 0; i < steps * 16; i += 32) {
            uint32_t o[32];
            tm_ld32(o_addr + i, o);
            wait_ld();
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
            tm_st32(o_addr + i, o);
          }
        }
      }
      const float ref = m == -INFINITY ? 0.0f : m;
      float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < KB; i += 2) {
        const float e0 = exp2_approx(fmaf(__uint_as_float(v[i]), a.c, -ref));
        const float e1 = exp2_approx(fmaf(__uint_as_float(v[i + 1]), a.c, -ref));
        sum[(i >> 1) & 3] += e0 + e1;
        v[i >> 1] = pack16<KT>(e0, e1);
      }
      l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      tm_st32(s_addr, v);
      tm_st32(s_addr + 32, v + 32);
      wait_st();
      fence_before();
      __syncwarp();
      if (lane == 0) kv_mbar_arrive(&s.p_full[u]);
    }

    // ---- rows of O
    if (nb > 0) {
      kv_mbar_wait(&s.o_full[u], 0, abort_flag, &g_prompt_error);
      fence_after();
    }
    // through this warp's rows of Q's place (every product has read it) and out as whole rows
    const float inv = l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l);
    if (nb > 0) {
#pragma unroll
      for (int i = 0; i < 64 * HALVES; i += 32) {
        uint32_t o[32];
        if (i >= steps * 16) break;
        tm_ld32(o_addr + i, o);
        wait_ld();
#pragma unroll
        for (int k = 0; k < 32; k += 8)
          *reinterpret_cast<uint4*>(staged(lane, i + k)) =
              make_uint4(pack16<KT>(__uint_as_float(o[k]) * inv, __uint_as_float(o[k + 1]) * inv),
                         pack16<KT>(__uint_as_float(o[k + 2]) * inv, __uint_as_float(o[k + 3]) * inv),
                         pack16<KT>(__uint_as_float(o[k + 4]) * inv, __uint_as_float(o[k + 5]) * inv),
                         pack16<KT>(__uint_as_float(o[k + 6]) * inv, __uint_as_float(o[k + 7]) * inv));
      }
      __syncwarp();
    }
    {
      const int64_t at = valid ? ((int64_t)(x.q0 + tok) * a.q_heads + x.head0 + hd) * a.head_dim : -1;
      const int d = lane * 4;
#pragma unroll 8
      for (int i = 0; i < 32; ++i) {
        const int64_t to = __shfl_sync(0xffffffffu, at, i);
        if (to >= 0 && d < a.head_dim)
          *reinterpret_cast<uint2*>(a.out + 2 * (to + d)) = nb > 0 ? *reinterpret_cast<const uint2*>(staged(i, d)) : make_uint2(0u, 0u);
      }
    }
  }

  // ---- every role has left its loop (all waits are bounded); free the tensor memory
  fence_before();
  __syncthreads();
  fence_after();
  if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

template <typename KT, int HALVES>
int launch_one(const CUtensorMap& km, const CUtensorMap& vm, const PromptArgs& a, int64_t grid, cudaStream_t st) {
  auto kernel = attn_prompt_kernel<KT, HALVES>;
  constexpr size_t smem = Layout<HALVES>::TAIL + sizeof(Tail) + 1024;
  static_assert(smem <= 232448, "shared memory of one CTA");
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return note_cuda_error(e);
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
  e = cudaLaunchKernelEx(&cfg, kernel, km, vm, a);
  return e == cudaSuccess ? check_launch() : note_cuda_error(e);
}

}  // namespace

int launch_attn_prompt(const bitnet_kv_cache_t* c, const AttnArgs& x, cudaStream_t st) {
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
  a.q_sign = x.scale < 0.0f ? 0x80008000u : 0u;
  a.c = fmaxf(fabsf(x.scale) * 1.4426950408889634f, 1e-30f);
  a.dev_status = x.dev_status;
  // a sequence has at most one tile pair that is not full; which CTA has which is found on the device
  const int64_t pairs = x.tokens / (2 * a.tile_tokens) + (x.seqs < x.tokens ? x.seqs : x.tokens);
  const int64_t grid = pairs * a.kv_heads * a.blocks;
  if (grid > 0x7fffffff) return BITNET_ERR_UNSUPPORTED_SHAPE;
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
