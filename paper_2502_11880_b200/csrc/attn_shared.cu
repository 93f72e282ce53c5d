// Attention of single tokens of sequences that share beginnings, in three kernels:
//   1. the groups' prefixes: rows (sequence, query head) of a group against its prefix, read once, on the 5th-generation tensor cores
//      (attn_prompt.cu), in parts over the CTAs;
//   2. the sequences' own tokens (attn_own_kernel), in parts over the warps;
//   3. the join (attn_join_kernel).
// Where the host cannot tell whether the groups share enough, attn_route_kernel finds out, and these three or the decode kernel end at once.
// A part of a row is its maximum m, its sum l = sum 2^(s - m) and O = sum 2^(s - m) V, s in units of log2.
//
// Measured (us, a B200), bf16: 64 sequences over 16384 tokens with up to 400 of their own, 64/8 heads of 128: 77, by themselves 45, 22 and 8 (35 GFLOP
// of products need 21; the decode kernel, which reads the prefix for every sequence: 382); 40 in three groups over 4000, 704 and 0, 16/16 heads of 96,
// fp16, window 2048: 38 (93).
#include <cstring>
#include <type_traits>

#include "kv_cache.cuh"

namespace bitnet {
namespace {

constexpr int ROWS = 128;                     // of a tile of kernel 1

template <typename KT>
struct Two;
template <>
struct Two<__nv_bfloat16> {
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
struct Two<__half> {
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
  }
  static __device__ __forceinline__ float2 unpack(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
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

// 16 bytes to shared memory, the first `n` from `src`, the rest zeros.
__device__ __forceinline__ void copy16(uint32_t dst, const uint8_t* src, int n, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(dst), "l"(src), "r"(n), "l"(policy) : "memory");
}

// ------------------------------------------------------------------------------------------------ own tokens
// Rows here are (sequence, kv head, block of up to 8 query heads), their tokens cut into tiles of 16.  All rows' tiles form one list that is dealt to the
// warps in equal contiguous parts; a warp works by itself, with a ring of tiles of its own that plain asynchronous copies fill, so that
// some 1200 short rows are under way at a time and none waits for another.  (The decode kernel, whose eight warps meet at every
// row's end, took 55 us for 64 sequences of up to 400 own tokens, 64/8 heads of 128, and 36 for 40 of up to 300, 16/16 heads of 96; HBM needs 8 and 7, this kernel takes 22 and 16.)  A row's
// first part goes to its place in the workspace, a later one (a warp has one at most, at its beginning) to the warp's.
// S = Q K^T and O += P V on mma.sync m16n8k16, the heads as rows 0..7; rows 8..15 of P hold what rounding took from rows 0..7, so that probabilities
// have 16 (bf16) or 22 bits.
constexpr int OWN_WARPS = 8, OWN_THREADS = OWN_WARPS * 32;
constexpr int TILE = 16;                      // tokens
constexpr int HEADS = 8;

struct OwnArgs {
  const uint8_t *q, *k, *v;                   // the layer's pools
  int64_t q_stride_token, q_stride_head;      // elements
  int64_t page_bytes, head_bytes, row_bytes;
  const int32_t* table;
  const int32_t* kv_len;
  const int32_t* group_start;
  const int32_t* prefix_len;
  int64_t table_width;
  int seqs, groups;
  int q_heads, kv_heads, group, head_blocks;  // group = query heads per kv head, in blocks of up to 8
  int head_dim, page_shift, num_pages;
  int window, sinks, max_len;
  float c;                                    // scale * log2(e)
  float4* own_ml;                             // [seqs][q_heads]: maximum, sum, first and last warp of the row
  float* own_o;                               // [seqs][q_heads][padded]
  float2* late_ml;                            // [warps][8]
  float* late_o;                              // [warps][8][padded]
  int padded;
  int* dev_status;
  const int* route;                           // 0 there: the decode kernel takes the call; null: it does not
};

// A sequence's own tokens that its last token sees: [s_lo, s_hi) of the sinks and [lo, hi), as tiles.
struct Own {
  int s_lo, s_hi, lo, hi, n0, tiles;
  bool beyond;                                // a window of a position beyond the table
};
__device__ __forceinline__ Own own_of(const OwnArgs& a, int n) {
  const int64_t len = __ldg(a.kv_len + n);
  const int prefix = kv_group_of(a.group_start, a.prefix_len, a.groups, n, a.max_len).prefix;
  Own r;
  r.hi = (int)max((int64_t)0, min(len, (int64_t)a.max_len));
  r.beyond = a.window > 0 && len > a.max_len;
  const int from = a.window > 0 ? (int)min(max((int64_t)0, len - a.window), (int64_t)a.max_len) : 0;   // the window's first token
  r.s_lo = prefix;
  r.s_hi = min(min(a.sinks, from), r.hi);
  r.lo = max(from, prefix);
  r.n0 = r.s_hi > r.s_lo ? (r.s_hi - 1) / TILE - r.s_lo / TILE + 1 : 0;
  r.tiles = max(1, r.n0 + (r.hi > r.lo ? (r.hi - 1) / TILE - r.lo / TILE + 1 : 0));   // (a row without tokens has a tile with nothing visible)
  return r;
}

template <int DT>
struct OwnLayout {
  static constexpr int ROW = DT > 4 ? 256 : 128;           // bytes of a token's K, or V
  static constexpr int STAGE = 2 * TILE * ROW;
  static constexpr int STAGES = DT > 4 ? 3 : 6;
  struct Tail {
    int64_t scan[OWN_WARPS];
    int most[OWN_WARPS];
    int64_t cut[OWN_WARPS][2];                // of the list: where a warp's part begins, and the next one's
    int64_t begin[OWN_WARPS], end[OWN_WARPS], base[OWN_WARPS];
    int first[OWN_WARPS];
  };
  static constexpr int SMEM = OWN_WARPS * STAGES * STAGE + (int)sizeof(Tail);
};

template <typename KT, int DT>
__global__ void __launch_bounds__(OWN_THREADS, 1) attn_own_kernel(const __grid_constant__ OwnArgs a) {
  using L = OwnLayout<DT>;
  using P2 = Two<KT>;
  constexpr bool HALF_T = std::is_same<KT, __half>::value;
  constexpr float P_SHIFT = HALF_T ? 12.0f : 0.0f;         // keeps fp16 remainders clear of its smallest steps
  extern __shared__ __align__(128) uint8_t smem[];
  typename L::Tail& s = *reinterpret_cast<typename L::Tail*>(smem + OWN_WARPS * L::STAGES * L::STAGE);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // This grid starts where SMs are done with kernel 1, which let it go when all before it was complete, and of whose results nothing is read here.  It
  // ends after kernel 1, so that the join follows both.  (The three in turn: 80.7 and 42.6 us against 76.2 and 38.1.)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  auto others_done = [] { asm volatile("griddepcontrol.wait;" ::: "memory"); };
  if (a.route && !__ldcg(a.route)) {
    others_done();
    return;
  }

  // ---- the list of tiles: total, and where the warps' parts begin
  const int rows_per_seq = a.kv_heads * a.head_blocks;
  int64_t total = 0, my_excl = 0;
  int64_t my_tiles = 0;
  int longest = 0, my_row = 1;
  auto scan_chunk = [&](int n0, int64_t base) {            // tiles before sequence n0 + tid; returns the chunk's total
    const int n = n0 + tid;
    my_row = n < a.seqs ? own_of(a, n).tiles : 0;
    my_tiles = (int64_t)my_row * rows_per_seq;
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
    for (int w = 0; w < OWN_WARPS; ++w) {
      const int64_t v = s.scan[w];
      if (w < warp) before += v;
      sum += v;
      longest = max(longest, s.most[w]);
    }
    my_excl = base + before + x - my_tiles;
    return sum;
  };
  for (int n0 = 0; n0 < a.seqs; n0 += OWN_THREADS) total += scan_chunk(n0, total);
  // Rows that are short, or many and none much longer than a warp's share, stay whole: a part more costs about as much as four tiles.
  // (300 sequences of 1 to 200 own tokens, 32/8 heads of 128: 67 us whole; with one of 2000 among them 146 whole, 72 cut, with one of 32768 1680 and 98.)
  const int64_t warps = (int64_t)gridDim.x * OWN_WARPS, rows = (int64_t)a.seqs * rows_per_seq;
  const bool whole = longest <= 6 || (rows >= 2 * warps && longest * warps <= 2 * total);
  const int64_t parts = min(warps, whole ? rows : total);
  // (warps of different CTAs take neighbouring parts: the SMs have equally many)
  const int64_t id = blockIdx.x + (int64_t)warp * gridDim.x;
  if (lane < 2) {
    s.cut[warp][lane] = id < parts ? kv_quotient(total * (id + lane), parts) : -1;
    if (lane == 0) s.begin[warp] = s.end[warp] = id < parts ? total : 0;
  }
  __syncthreads();
  auto find_cuts = [&](int n0) {
    const int64_t mine = my_excl + my_tiles;
#pragma unroll 1
    for (int k = 0; k < 2 * OWN_WARPS; ++k) {
      const int64_t c = s.cut[k >> 1][k & 1];
      if (c < my_excl || c >= mine) continue;
      const int64_t at = whole ? my_excl + kv_quotient(c - my_excl, my_row) * my_row : c;
      if (k & 1) {
        s.end[k >> 1] = at;
      } else {
        s.begin[k >> 1] = at;
        s.first[k >> 1] = n0 + tid;
        s.base[k >> 1] = my_excl;
      }
    }
  };
  if (a.seqs <= OWN_THREADS) {
    find_cuts(0);
  } else {
    int64_t base = 0;
    for (int n0 = 0; n0 < a.seqs; n0 += OWN_THREADS) {
      base += scan_chunk(n0, base);
      find_cuts(n0);
    }
  }
  __syncthreads();
  if (id >= parts || s.begin[warp] >= s.end[warp]) {
    others_done();
    return;
  }

  // A place in the list, and a second one STAGES - 1 tiles ahead, where the ring is filled.
  struct Place {
    int64_t left;                             // tiles of the part from here on
    int n, t, kv, block;                      // sequence, tile of the row, the row's kv head and block of query heads
    Own r;
  } p, f;
  auto next_row = [&](Place& p) {
    p.t = 0;
    if (++p.block < a.head_blocks) return;
    p.block = 0;
    if (++p.kv < a.kv_heads) return;
    p.kv = 0;
    if (p.left > 0) p.r = own_of(a, ++p.n);
  };
  {
    const int64_t item = s.begin[warp], in_seq = item - s.base[warp];
    p.left = s.end[warp] - item;
    p.n = s.first[warp];
    p.r = own_of(a, p.n);
    const int row = (int)kv_quotient(in_seq, p.r.tiles);
    p.t = (int)(in_seq - (int64_t)row * p.r.tiles);
    p.kv = row / a.head_blocks;
    p.block = row - p.kv * a.head_blocks;
    f = p;
  }
  auto tile_of = [&](const Own& r, int t, int& first, int& lo, int& hi) {
    const bool sink = t < r.n0;
    lo = sink ? r.s_lo : r.lo;
    hi = sink ? r.s_hi : r.hi;
    first = (lo / TILE + (sink ? t : t - r.n0)) * TILE;
  };
  const uint32_t ring = smem_u32(smem) + warp * L::STAGES * L::STAGE;
  constexpr int PIECES = L::ROW / 16, AT_ONCE = 32 / PIECES;          // 16-byte pieces of a row, rows per step
  const int piece = lane % PIECES, sub = lane / PIECES;
  const int bytes = max(0, min(16, 2 * a.head_dim - 16 * piece));    // (the rest is filled with zeros: padding may be anything)
  const uint64_t policy = policy_evict_first();            // (tokens are read once: what else is in L2, the kernels' instructions too, stays)
  // the page of the lane's token in f's tile; -2: not read
  auto look_up = [&]() -> int {
    int first, lo, hi;
    tile_of(f.r, f.t, first, lo, hi);
    const int tok = first + (lane & (TILE - 1));
    return f.left > 0 && tok >= lo && tok < hi ? max(__ldg(a.table + (int64_t)f.n * a.table_width + (tok >> a.page_shift)), -1) : -2;
  };
  int page = look_up();                       // (a tile ahead of the copies)
  uint32_t filled = 0;
  auto fill = [&] {
    if (f.left > 0) {
      int first, lo, hi;
      tile_of(f.r, f.t, first, lo, hi);
      const bool there = page >= 0 && page < a.num_pages;
      if (((page != -2 && !there) || (f.r.beyond && lane == 0)) && a.dev_status) atomicExch(a.dev_status, BITNET_ERR_BAD_PAGE);
      const int tok = first + (lane & (TILE - 1));
      const int64_t of_lane = there ? page * a.page_bytes + (int64_t)(tok & ((1 << a.page_shift) - 1)) * a.row_bytes + f.kv * a.head_bytes : -1;
      --f.left;
      if (++f.t == f.r.tiles) next_row(f);
      page = look_up();
      const uint32_t to = ring + (filled % L::STAGES) * L::STAGE + sub * L::ROW;
#pragma unroll
      for (int i = 0; i < TILE; i += AT_ONCE) {
        const int64_t of_row = __shfl_sync(0xffffffffu, of_lane, i + sub);
        const int64_t at = max(of_row, (int64_t)0) + piece * 16;
        const uint32_t dst = to + i * L::ROW + ((piece & ~7) | ((piece ^ (i + sub)) & 7)) * 16;
        const int n = of_row < 0 ? 0 : bytes;
        copy16(dst, a.k + (n ? at : 0), n, policy);
        copy16(dst + TILE * L::ROW, a.v + (n ? at : 0), n, policy);
      }
      ++filled;
    }
    cp_commit();
  };
#pragma unroll 1
  for (int i = 0; i < L::STAGES - 1; ++i) fill();

  const int g = lane >> 2, t4 = lane & 3;                  // accumulator row (head) and column pair
  const int k_row = (lane & 7) + ((lane >> 4) << 3), k_piece = (lane >> 3) & 1;
  const int v_row = lane & 15, v_piece = lane >> 4;
  uint32_t used = 0;
  while (p.left > 0) {
    const Own r = p.r;
    const int n = p.n, t0 = p.t, t_end = (int)min((int64_t)r.tiles, t0 + p.left);
    const int heads = min(HEADS, a.group - p.block * HEADS), head0 = p.kv * a.group + p.block * HEADS;
    uint32_t qa[DT][2];
    {
      const bool have = g < heads;
      const uint8_t* qp = a.q + 2 * ((int64_t)n * a.q_stride_token + (int64_t)(head0 + (have ? g : 0)) * a.q_stride_head);
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int d = 16 * i + 8 * j + 2 * t4;
          qa[i][j] = have && d < a.head_dim ? *reinterpret_cast<const uint32_t*>(qp + d * 2) : 0u;
        }
    }
    float o[2 * DT][4];
#pragma unroll
    for (int j = 0; j < 2 * DT; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.0f;
    float m = -INFINITY, l = 0.0f;                          // of head g (l: this lane's share)

    for (int t = t0; t < t_end; ++t, ++used) {
      int first, lo, hi;
      tile_of(r, t, first, lo, hi);
      fill();                                               // (the stage that the previous tile left)
      cp_wait<L::STAGES - 1>();
      __syncwarp();
      const uint32_t kbase = ring + (used % L::STAGES) * L::STAGE, vbase = kbase + TILE * L::ROW;
      float sc[2][2][4] = {};
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        const int at = 2 * i + k_piece;
        uint32_t b[4];
        ldsm4(kbase + k_row * L::ROW + ((at & ~7) | ((at ^ k_row) & 7)) * 16, b);
        P2::mma(sc[i & 1][0], qa[i][0], 0u, qa[i][1], 0u, b[0], b[1]);
        P2::mma(sc[i & 1][1], qa[i][0], 0u, qa[i][1], 0u, b[2], b[3]);
      }
      float x[4];                                           // scores of head g at tokens 2 t4, 2 t4 + 1, + 8, + 9
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int tok = first + 8 * j + 2 * t4 + e;
          x[2 * j + e] = tok >= lo && tok < hi ? (sc[0][j][e] + sc[1][j][e]) * a.c : -INFINITY;
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
      float e[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) e[j] = exp2_approx(x[j] - ref);
      l += (e[0] + e[1]) + (e[2] + e[3]);
      uint32_t ph[2], pm[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        ph[j] = P2::pack(e[2 * j], e[2 * j + 1]);
        const float2 hf = P2::unpack(ph[j]);
        pm[j] = P2::pack(e[2 * j] - hf.x, e[2 * j + 1] - hf.y);
      }
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        const int at = 2 * i + v_piece;
        uint32_t b[4];
        ldsm4_t(vbase + v_row * L::ROW + ((at & ~7) | ((at ^ v_row) & 7)) * 16, b);
        P2::mma(o[2 * i], ph[0], pm[0], ph[1], pm[1], b[0], b[1]);
        P2::mma(o[2 * i + 1], ph[0], pm[0], ph[1], pm[1], b[2], b[3]);
      }
      __syncwarp();
    }

    // ---- the part, without fp16's scale: lane has columns 8 j + 2 t4, + 1 of head g
    const float down = HALF_T ? 1.0f / 4096.0f : 1.0f;
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    if (g < heads) {
      const int64_t at = (int64_t)n * a.q_heads + head0 + g, late = id * HEADS + g;
      float* const dst = (t0 == 0 ? a.own_o + at * a.padded : a.late_o + late * a.padded) + 2 * t4;
      if (t4 == 0) {
        if (t0 == 0) {
          // the last warp that has a part of this row
          const int w1 = whole || t_end == r.tiles ? (int)id : (int)kv_quotient((s.end[warp] - p.left + r.tiles) * parts - 1, total);
          a.own_ml[at] = make_float4(m, l * down, __int_as_float((int)id), __int_as_float(w1));
        } else {
          a.late_ml[late] = make_float2(m, l * down);
        }
      }
#pragma unroll
      for (int j = 0; j < 2 * DT; ++j)
        if (8 * j < a.padded)
          *reinterpret_cast<float2*>(dst + 8 * j) = make_float2((o[j][0] + o[j][2]) * down, (o[j][1] + o[j][3]) * down);
    }
    p.left -= t_end - t0;
    if (t_end == r.tiles) next_row(p);
  }
  others_done();
}

// ------------------------------------------------------------------------------------------------ join
// With a row's parts, m = max m_k, out = sum_k 2^(m_k - m) O_k / sum_k 2^(m_k - m) l_k in the order of the parts, in fp32, rounded once.  A warp per row
// (sequence and query head); maxima and sums are read by its lanes side by side, the parts of O eight at a time.  Bound by latency: 26 MB of parts, all in
// L2, in 8 us for 64 sequences with 64 query heads of 128.
constexpr int JOIN_WARPS = 4;

struct JoinArgs {
  SharedParts p;
  const float4* own_ml;
  const float* own_o;
  const float2* late_ml;
  const float* late_o;
  uint8_t* out;
  const int32_t* group_start;
  const int32_t* prefix_len;
  int64_t rows;
  int q_heads, group, per_block, tile_tokens, groups, head_dim, ctas;
  const int* route;
};

template <typename KT>
__global__ void __launch_bounds__(JOIN_WARPS * 32) attn_join_kernel(const __grid_constant__ JoinArgs a) {
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * JOIN_WARPS + (threadIdx.x >> 5);
  const int tok = (int)kv_quotient(row, a.q_heads), head = (int)(row - (int64_t)tok * a.q_heads);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (row >= a.rows || (a.route && !__ldcg(a.route))) return;
  const int d = 4 * lane;
  const bool mine = d < a.p.padded;
  const float4 zero = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const float4 own = __ldcg(a.own_ml + row), base = __ldcg(a.p.base_ml + row);
  const float4 own_o = mine ? __ldcg(reinterpret_cast<const float4*>(a.own_o + row * a.p.padded + d)) : zero;
  const float4 base_o = mine ? __ldcg(reinterpret_cast<const float4*>(a.p.base_o + row * a.p.padded + d)) : zero;
  const KvGroup g = kv_group_of(a.group_start, a.prefix_len, a.groups, tok, 0);
  const bool in_group = g.first >= 0;                      // otherwise there is nothing at the row's place of kernel 1

  float m = in_group ? fmaxf(own.x, base.x) : own.x;
  auto factor = [](float of, float to) { return of == -INFINITY ? 0.0f : exp2_approx(of - to); };
  float4 acc = zero;
  auto add = [&](float f, const float4& o) {
    if (f == 0.0f) return;                                 // (what a part without visible tokens has left may be anything)
    acc.x += f * o.x;
    acc.y += f * o.y;
    acc.z += f * o.z;
    acc.w += f * o.w;
  };
  float sum = factor(own.x, m) * own.y;
  add(factor(own.x, m), own_o);
  if (in_group) {
    sum += factor(base.x, m) * base.y;
    add(factor(base.x, m), base_o);
  }
  // later parts: n of them, `step` places apart
  auto join = [&](int64_t n, const float2* ml_at, const float* o_at, int64_t step) {
    for (int64_t k32 = 0; k32 < n; k32 += 32) {
      const int left = (int)min((int64_t)32, n - k32);
      const float2 ml = lane < left ? __ldcg(ml_at + (k32 + lane) * step) : make_float2(-INFINITY, 0.0f);
      float top = ml.x;
#pragma unroll
      for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      top = fmaxf(top, m);
      const float f = factor(m, top);
      m = top;
      sum *= f;
      acc = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
      const float w = factor(ml.x, m), wl = w * ml.y;
      for (int k0 = 0; k0 < left; k0 += 8) {
        float4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
          v[k] = mine && k0 + k < left ? __ldcg(reinterpret_cast<const float4*>(o_at + (k32 + k0 + k) * step * a.p.padded + d)) : zero;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (k0 + k >= left) break;
          sum += __shfl_sync(0xffffffffu, wl, k0 + k);
          add(__shfl_sync(0xffffffffu, w, k0 + k), v[k]);
        }
      }
    }
  };
  if (in_group) {
    // CTAs c0 + 1 .. c1 (any, where kernel 1 has given up), at this row's place in them
    const int c0 = max(__float_as_int(base.z), 0), c1 = min(__float_as_int(base.w), a.ctas - 1);
    const int at = (tok - g.first) % (2 * a.tile_tokens);
    const int64_t place = (int64_t)(c0 + 1) * 2 * ROWS + at / a.tile_tokens * ROWS + at % a.tile_tokens * a.per_block + head % a.group % a.per_block;
    join(c1 - c0, a.p.spill_ml + place, a.p.spill_o + place * a.p.padded, 2 * ROWS);
  }
  {
    const int w0 = __float_as_int(own.z), w1 = __float_as_int(own.w);
    const int64_t place = (int64_t)(w0 + 1) * HEADS + head % a.group % HEADS;
    join(w1 - w0, a.late_ml + place, a.late_o + place * a.p.padded, HEADS);
  }
  if (d >= a.head_dim) return;
  const float inv = sum > 0.0f ? 1.0f / sum : (sum == 0.0f ? 0.0f : sum);          // nothing visible: 0; NaN stays NaN
  *reinterpret_cast<uint2*>(a.out + 2 * (row * a.head_dim + d)) =
      make_uint2(Two<KT>::pack(acc.x * inv, acc.y * inv), Two<KT>::pack(acc.z * inv, acc.w * inv));
}

// ------------------------------------------------------------------------------------------------ which kernels
// Whether the groups share enough for the three kernels, in tiles of 64 tokens of a kv head: 3 R - T > limit, where T tiles are seen by all sequences and R of
// them, of a group's prefix, by another sequence too.  One CTA: a warp per group, a thread per sequence.
constexpr int ROUTE_THREADS = 1024;

struct RouteArgs {
  const int32_t *kv_len, *group_start, *prefix_len;
  int seqs, groups, window, sinks, max_len;
  int64_t limit;
  int* route;
};

__global__ void __launch_bounds__(ROUTE_THREADS) attn_route_kernel(const __grid_constant__ RouteArgs a) {
  __shared__ unsigned long long seen, again;
  const int tid = threadIdx.x, lane = tid & 31;
  if (tid == 0) seen = again = 0;
  __syncthreads();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // tiles of the first `most` tokens that a sequence's last token sees
  auto tiles = [&](int len, int most) {
    const int end = min(len, most);
    if (end <= 0) return 0;
    const int lo = a.window > 0 ? max(0, len - a.window) : 0;
    const int tokens = lo >= end ? min(a.sinks, end) : min(a.sinks, lo) + end - lo;
    return (int)(((int64_t)tokens + 63) / 64);
  };
  auto add = [&](unsigned long long& to, int64_t v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0 && v) atomicAdd(&to, (unsigned long long)v);
  };
  int64_t mine = 0;
  for (int64_t i = tid; i < a.seqs; i += ROUTE_THREADS) mine += tiles(__ldg(a.kv_len + i), a.max_len);
  add(seen, mine);
  mine = 0;
  for (int64_t g = tid >> 5; g < a.groups; g += ROUTE_THREADS / 32) {
    const int q0 = __ldg(a.group_start + g), q1 = min(__ldg(a.group_start + g + 1), a.seqs);
    if (q0 < 0 || q1 - (int64_t)q0 < 2) continue;
    const int prefix = min(__ldg(a.prefix_len + g), a.max_len);
    int top = 0;
    for (int64_t i = q0 + lane; i < q1; i += 32) {
      const int t = tiles(__ldg(a.kv_len + i), prefix);
      mine += t;
      top = max(top, t);
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) mine -= top;                            // (read once in any case)
  }
  add(again, mine);
  __syncthreads();
  if (tid == 0) *a.route = 3 * (int64_t)again - (int64_t)seen > a.limit;
}

// ------------------------------------------------------------------------------------------------ launches
template <typename K, typename A>
int launch(K kernel, unsigned grid, int threads, int smem, cudaStream_t st, const A& a) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = early_start_enabled(st) ? 1 : 0;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a);
  return e == cudaSuccess ? check_launch() : note_cuda_error(e);
}
template <typename KT, int DT>
int launch_own(const OwnArgs& a, cudaStream_t st) {
  constexpr int smem = OwnLayout<DT>::SMEM;
  static_assert(smem <= 232448, "shared memory of one CTA");
  static std::atomic<uint64_t> have{0};
  const int rc = allow_smem(attn_own_kernel<KT, DT>, smem, &have);
  return rc ? rc : launch(attn_own_kernel<KT, DT>, (unsigned)dev_info().sm_count, OWN_THREADS, smem, st, a);
}
template <typename KT>
int launch_own(const OwnArgs& a, cudaStream_t st) {
  const int steps = (a.head_dim + 15) / 16;
  if (steps <= 4) return launch_own<KT, 4>(a, st);
  return steps <= 6 ? launch_own<KT, 6>(a, st) : launch_own<KT, 8>(a, st);
}

struct Places {
  SharedParts p;
  float4* own_ml;
  float *own_o, *late_o;
  float2* late_ml;
  int* route;
  size_t bytes;
};
// The workspace: that of decode calls, then the rows' places, the CTAs' and the warps'.
Places places(uint8_t* at, int64_t rows, int head_dim) {
  const int64_t sms = dev_info().sm_count, padded = ceil_div(head_dim, 16) * 16;
  uint8_t* const begin = at;
  auto take = [&](int64_t n, int64_t each) {
    uint8_t* const p = at;
    at += n * each;                                        // (multiples of 16 bytes first)
    return p;
  };
  Places x;
  x.p.padded = (int)padded;
  x.p.base_o = reinterpret_cast<float*>(take(rows, padded * 4));
  x.own_o = reinterpret_cast<float*>(take(rows, padded * 4));
  x.p.spill_o = reinterpret_cast<float*>(take(sms * 2 * ROWS, padded * 4));
  x.late_o = reinterpret_cast<float*>(take(sms * OWN_WARPS * HEADS, padded * 4));
  x.p.base_ml = reinterpret_cast<float4*>(take(rows, 16));
  x.own_ml = reinterpret_cast<float4*>(take(rows, 16));
  x.p.spill_ml = reinterpret_cast<float2*>(take(sms * 2 * ROWS, 8));
  x.late_ml = reinterpret_cast<float2*>(take(sms * OWN_WARPS * HEADS, 8));
  x.route = reinterpret_cast<int*>(take(1, 16));
  x.bytes = (size_t)(at - begin);
  return x;
}

}  // namespace

size_t attn_shared_workspace_bytes(int64_t seqs, int64_t q_heads, int head_dim) {
  return attn_decode_workspace_bytes() + places(nullptr, seqs * q_heads, head_dim).bytes;
}

int launch_attn_shared(const bitnet_kv_cache_t* c, const AttnArgs& args, int64_t ask, void* ws, cudaStream_t st) {
  AttnArgs x = args;
  const int64_t rows = x.tokens * x.q_heads;
  const Places w = places(attn_prompt_parts(ws), rows, c->head_dim);
  const int64_t most = x.table_width * c->page_size;
  const int max_len = most > 0x3fffff00 ? 0x3fffff00 : (int)most;     // (as for the prefixes)
  int rc;
  if (ask >= 0) {
    RouteArgs r = {};
    r.kv_len = x.kv_len;
    r.group_start = x.group_start;
    r.prefix_len = x.prefix_len;
    r.seqs = (int)x.tokens;
    r.groups = (int)x.groups;
    r.window = x.window;
    r.sinks = x.sinks;
    r.max_len = max_len;
    r.limit = ask;
    r.route = w.route;
    log_launch("attn_route_kernel sequences=%d groups=%d", r.seqs, r.groups);
    rc = launch(attn_route_kernel, 1, ROUTE_THREADS, 0, st, r);
    if (rc != BITNET_OK) return rc;
    x.route = w.route;
  }
  rc = launch_attn_shared_prefix(c, x, w.p, st);
  if (rc != BITNET_OK) return rc;

  OwnArgs a = {};
  a.q = static_cast<const uint8_t*>(x.q);
  a.k = static_cast<const uint8_t*>(c->k) + x.layer * c->stride_layer * 2;
  a.v = static_cast<const uint8_t*>(c->v) + x.layer * c->stride_layer * 2;
  a.q_stride_token = x.q_stride_token;
  a.q_stride_head = x.q_stride_head;
  a.page_bytes = 2 * c->stride_page;
  a.head_bytes = 2 * c->stride_head;
  a.row_bytes = 2 * c->stride_row;
  a.table = x.table;
  a.kv_len = x.kv_len;
  a.group_start = x.group_start;
  a.prefix_len = x.prefix_len;
  a.table_width = x.table_width;
  a.seqs = (int)x.tokens;
  a.groups = (int)x.groups;
  a.q_heads = x.q_heads;
  a.kv_heads = c->kv_heads;
  a.group = x.q_heads / c->kv_heads;
  a.head_blocks = (int)ceil_div(a.group, HEADS);
  a.head_dim = c->head_dim;
  a.page_shift = __builtin_ctz((unsigned)c->page_size);
  a.num_pages = (int)c->num_pages;
  a.window = x.window;
  a.sinks = x.sinks;
  a.max_len = max_len;
  a.c = x.scale * 1.4426950408889634f;
  a.own_ml = w.own_ml;
  a.own_o = w.own_o;
  a.late_ml = w.late_ml;
  a.late_o = w.late_o;
  a.padded = w.p.padded;
  a.dev_status = x.dev_status;
  a.route = x.route;
  log_launch("attn_own_kernel sequences=%d groups=%d q_heads=%d kv_heads=%d head_dim=%d window=%d", a.seqs, a.groups, a.q_heads, a.kv_heads,
             a.head_dim, a.window);
  rc = x.dtype == BITNET_KV_BF16 ? launch_own<__nv_bfloat16>(a, st) : launch_own<__half>(a, st);
  if (rc != BITNET_OK) return rc;

  JoinArgs j = {};
  j.p = w.p;
  j.own_ml = w.own_ml;
  j.own_o = w.own_o;
  j.late_ml = w.late_ml;
  j.late_o = w.late_o;
  j.out = static_cast<uint8_t*>(x.out);
  j.rows = rows;
  j.group_start = x.group_start;
  j.prefix_len = x.prefix_len;
  j.groups = (int)x.groups;
  j.q_heads = x.q_heads;
  j.group = a.group;
  j.per_block = (int)ceil_div(j.group, ceil_div(j.group, ROWS));
  j.tile_tokens = ROWS / j.per_block;
  j.head_dim = c->head_dim;
  j.ctas = dev_info().sm_count;
  j.route = x.route;
  const unsigned grid = (unsigned)ceil_div(rows, JOIN_WARPS);
  rc = x.dtype == BITNET_KV_BF16 ? launch(attn_join_kernel<__nv_bfloat16>, grid, JOIN_WARPS * 32, 0, st, j)
                                 : launch(attn_join_kernel<__half>, grid, JOIN_WARPS * 32, 0, st, j);
  if (rc != BITNET_OK || ask < 0) return rc;
  return launch_attn_decode(c, x, ws, st);
}

}  // namespace bitnet
