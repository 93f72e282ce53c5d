// New tokens' queries and keys rotated by their positions, keys and values written into the pages of the cache, in one pass over the
// output of the Q/K/V linear.
//
//   (a, b) -> (a cos t - b sin t, b cos t + a sin t),  t = position * frequency of the pair
//
// where pair i of a row is (x[i], x[i + rot/2]) or (x[2i], x[2i + 1]); elements from rot on move as they are.
//
// Angles: a frequency is held as the fraction of a turn per position in 64-bit fixed point, so that position * frequency modulo a turn is
// one integer product that wraps around by itself, right to 2^-32 of a turn at any position (the steps are right to one unit of 2^-64); its top 32
// bits go to sincospi as half turns in binary32, right to 2^-26 of a turn.
// (binary32 products would be off by 0.008 radians at position 131072, and a table of all positions is 67 MB that has to be read.)
// The products and sums are binary32, rounded once to the type written.
//
// Bound by HBM for prompts (rows of odd sizes: by instructions, a vector is what the sizes allow) and by latency for single tokens.  A CTA has a token, or some
// of its heads where tokens are few; its threads compute a sine and a cosine each and share them.  A row's pairs are cut into slots of two vectors of
// VEC elements; a thread keeps its slot, and so its VEC pairs' sines and cosines, over all heads that it visits.
//
// Measured (us, a B200): 32 tokens, 64/8 heads of 128: 3.0; 4 x 2048 tokens, 32/8 heads of 128, fp32 in, bf16 out: 39 (6.1 TB/s); bf16 in and out,
// 3222 tokens: 24 (3.3 TB/s, half of a copy's rate: 8 bytes a vector, two rows of a thread on their way), 4096 tokens: 30.  With every thread computing its
// own sines the first, second and third: 3.8, 43, 34.
#include <cstring>
#include <type_traits>

#include "kv_cache.cuh"

namespace bitnet {
namespace {

constexpr int THREADS = 128;

struct RopeDev {
  KvView kv;
  const uint8_t *q, *k, *v;
  uint8_t* q_out;
  int64_t q_stride_token, q_stride_head, stride_token, stride_head;
  const int32_t* table;
  const int32_t* kv_len;
  const int32_t* q_start;
  int64_t width;
  int tokens, seqs, layer, q_heads, rot, interleaved;
  int page_shift;
  int rotated, slots;        // slots of a row of q or k that hold pairs, and all of them
  int at_once, split;        // rows that a CTA takes at a time, CTAs per token
  int* dev_status;
  float magnitude;
  uint64_t step[64];         // turns per position, in 2^-64
};

// N elements of 4 or 2 bytes as they lie in memory, aligned to N elements (16 bytes at most).  (q may be overwritten by this call: no read-only path.)
template <typename T, int N>
struct alignas(sizeof(T) * N > 16 ? 16 : sizeof(T) * N) Vec {
  T t[N];
};
template <typename T, int N>
__device__ __forceinline__ Vec<T, N> load_vec(const uint8_t* p) {
  constexpr int BYTES = sizeof(T) * N;
  union {
    Vec<T, N> v;
    uint4 a[(BYTES + 15) / 16];
    uint2 b;
    unsigned int c;
    unsigned short d;
  } x;
  if constexpr (BYTES >= 16) {
#pragma unroll
    for (int i = 0; i < BYTES / 16; ++i) x.a[i] = __ldca(reinterpret_cast<const uint4*>(p) + i);
  } else if constexpr (BYTES == 8) {
    x.b = __ldca(reinterpret_cast<const uint2*>(p));
  } else if constexpr (BYTES == 4) {
    x.c = __ldca(reinterpret_cast<const unsigned int*>(p));
  } else {
    x.d = __ldca(reinterpret_cast<const unsigned short*>(p));
  }
  return x.v;
}
template <typename T>
__device__ __forceinline__ T to(float v) {
  if constexpr (std::is_same<T, float>::value) return v;
  else if constexpr (std::is_same<T, __half>::value) return __float2half_rn(v);
  else return __float2bfloat16_rn(v);
}
template <typename T, int N>
__device__ __forceinline__ void store_vec(uint8_t* p, const float (&x)[N]) {
  Vec<T, N> v;
#pragma unroll
  for (int i = 0; i < N; ++i) v.t[i] = to<T>(x[i]);
  *reinterpret_cast<Vec<T, N>*>(p) = v;
}

// KT: the cache's type; IN, OUT: of q, k, v and of q_out; VEC: elements of a vector.
template <typename KT, typename IN, typename OUT, int VEC>
__global__ void __launch_bounds__(THREADS) kv_rope_kernel(const __grid_constant__ RopeDev a) {
  __shared__ float2 turn[64];                // cosine and sine of each pair
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // A thread's rows on their way at a time.  4 x 2048 tokens, 32/8 heads of 128, fp32 in, bf16 out: 43, 39, 38, 48 us with 1, 2, 3, 4; 3 x 517, 32/32 of
  // 100, interleaved, fp16: 19.5, 16.3, 17.0, 24.8 (two with the next ones on their way: 38.9 and 15.7, but 3.3 instead of 3.0 for 32 tokens, and
  // single elements 15 % slower).  By single elements a row in four pieces (74, 81 with two).
  constexpr int AT_A_TIME = VEC == 1 ? 4 : 2;
  constexpr int IN_BYTES = sizeof(IN), OUT_BYTES = sizeof(OUT);
  const int lane = threadIdx.x & 31;
  const int mine = threadIdx.x / a.slots, slot = threadIdx.x - mine * a.slots;
  const int hq = a.q_heads, hkv = a.kv.kv_heads, dim = a.kv.head_dim, rows = hq + 2 * hkv, step = a.split * a.at_once;

  // ---- a row's slot: two vectors, neighbouring threads' vectors side by side.  Pairs of the half layout: a vector of first elements and that of
  // the second ones; elsewhere vectors slot and slot + half of those that there are.
  const bool pairs = slot < a.rotated;
  auto place = [&](int start, int s, int& d0, int& d1) {   // of the vectors from element `start` on
    const int n = (dim - start) / VEC, half = (n + 1) / 2;
    d0 = s < half ? start + s * VEC : dim;
    d1 = s + half < n && s < half ? start + (s + half) * VEC : dim;
  };
  int qd0, qd1, vd0, vd1;
  place(0, slot, vd0, vd1);
  if (a.interleaved) {
    qd0 = vd0;
    qd1 = vd1;
    if (VEC == 1) {                                        // (a pair is two vectors)
      qd0 = 2 * slot;
      qd1 = qd0 + 1;
    }
  } else if (pairs) {
    qd0 = slot * VEC;
    qd1 = qd0 + a.rot / 2;
  } else {
    place(a.rot, slot - a.rotated, qd0, qd1);
  }
  // the first pair of the slot's first vector, and of its second one (of the half layout both have the same)
  const int pair0 = VEC > 1 && a.interleaved ? qd0 / 2 : slot * VEC, pair1 = VEC > 1 && a.interleaved ? qd1 / 2 - VEC / 2 : pair0;

  const int n = a.split == 1 ? blockIdx.x : blockIdx.x / a.split, row0 = (blockIdx.x - n * a.split) * a.at_once + mine;
  const uint8_t* const q_in = a.q + (int64_t)n * a.q_stride_token * IN_BYTES;
  const uint8_t* const k_in = a.k + (int64_t)n * a.stride_token * IN_BYTES;
  const uint8_t* const v_in = a.v + (int64_t)n * a.stride_token * IN_BYTES;
  // (several rows' loads on their way together, the first ones before the look-ups, which they do not depend on)
  Vec<IN, VEC> in0[AT_A_TIME], in1[AT_A_TIME];
  auto load = [&](int first) {
#pragma unroll
    for (int k = 0; k < AT_A_TIME; ++k) {
      const int row = first + k * step;
      const bool is_q = row < hq, is_v = row >= hq + hkv;
      const int d0 = is_v ? vd0 : qd0, d1 = is_v ? vd1 : qd1;
      const uint8_t* const src = (is_q ? q_in : is_v ? v_in : k_in) +
                                 (int64_t)(row - (is_q ? 0 : is_v ? hq + hkv : hq)) * (is_q ? a.q_stride_head : a.stride_head) * IN_BYTES;
      if (row < rows && d0 < dim) in0[k] = load_vec<IN, VEC>(src + d0 * IN_BYTES);
      if (row < rows && d1 < dim) in1[k] = load_vec<IN, VEC>(src + d1 * IN_BYTES);
    }
  };
  const bool active = mine < a.at_once && row0 < rows;
  if (active) load(row0);

  // ---- the token's sequence, position and page
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
    const int end = __ldg(a.q_start + seq + 1);
    // (a token behind the last sequence, or ahead of the first, is nobody's)
    pos = n < end && n >= __ldg(a.q_start + seq) ? (int64_t)__ldg(a.kv_len + seq) - end + n : -1;
  } else {
    pos = (int64_t)__ldg(a.kv_len + seq) - 1;
  }
  if (pos < 0) return;                                   // (so for all threads)
  // sines and cosines, a pair per thread
  if (2 * (int)threadIdx.x < a.rot) {
    const uint64_t turns = (uint64_t)pos * a.step[threadIdx.x];
    float sn, cs;
    sincospif((float)(int)(turns >> 32) * 4.656612873077393e-10f, &sn, &cs);             // 2^-31: half turns
    turn[threadIdx.x] = make_float2(cs * a.magnitude, sn * a.magnitude);
  }
  const int64_t entry = pos >> a.page_shift;
  const int page = entry < a.width ? __ldg(a.table + (int64_t)seq * a.width + entry) : -1;
  const bool bad = page < 0 || page >= a.kv.num_pages;
  if (bad && threadIdx.x == 0 && a.dev_status) atomicExch(a.dev_status, BITNET_ERR_BAD_PAGE);
  __syncthreads();
  if (!active) return;
  float2 cs[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    const int pair = (i < VEC / 2 ? pair0 : pair1) + i;
    cs[i] = pairs && 2 * pair < a.rot ? turn[pair] : make_float2(1.0f, 0.0f);
  }
  const int64_t in_pool = 2 * (a.layer * a.kv.stride_layer + (bad ? 0 : page) * a.kv.stride_page + (pos & (a.kv.page_size - 1)) * a.kv.stride_row);
  uint8_t* const q_out = a.q_out + (int64_t)n * hq * dim * OUT_BYTES;
  for (int first = row0;;) {
#pragma unroll
    for (int k = 0; k < AT_A_TIME; ++k) {
      const int row = first + k * step;
      if (row >= rows) break;
      const bool is_q = row < hq, is_v = row >= hq + hkv;
      float x0[VEC], x1[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        x0[i] = static_cast<float>(in0[k].t[i]);
        x1[i] = static_cast<float>(in1[k].t[i]);
      }
      if (pairs && !is_v) {
        if (a.interleaved) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            // (elements beyond rot move as they are, infinities too)
            if constexpr (VEC == 1) {
              if (2 * slot >= a.rot) continue;
              const float p = x0[0], q = x1[0];
              x0[0] = p * cs[0].x - q * cs[0].y;
              x1[0] = q * cs[0].x + p * cs[0].y;
            } else {
              if ((i < VEC / 2 ? qd0 + 2 * i : qd1 + 2 * i - VEC) >= a.rot) continue;
              float* const e = i < VEC / 2 ? &x0[2 * i] : &x1[2 * i - VEC];
              const float p = e[0], q = e[1];
              e[0] = p * cs[i].x - q * cs[i].y;
              e[1] = q * cs[i].x + p * cs[i].y;
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            const float p = x0[i], q = x1[i];
            x0[i] = p * cs[i].x - q * cs[i].y;
            x1[i] = q * cs[i].x + p * cs[i].y;
          }
        }
      }
      const int d0 = is_v ? vd0 : qd0, d1 = is_v ? vd1 : qd1;
      if (is_q) {
        uint8_t* const dst = q_out + row * dim * OUT_BYTES;
        if (d0 < dim) store_vec<OUT, VEC>(dst + d0 * OUT_BYTES, x0);
        if (d1 < dim) store_vec<OUT, VEC>(dst + d1 * OUT_BYTES, x1);
      } else if (!bad) {
        uint8_t* const dst = (is_v ? a.kv.v : a.kv.k) + in_pool + 2 * ((row - (is_v ? hq + hkv : hq)) * a.kv.stride_head);
        if (d0 < dim) store_vec<KT, VEC>(dst + 2 * d0, x0);
        if (d1 < dim) store_vec<KT, VEC>(dst + 2 * d1, x1);
        // the row's padding (head_dim is a multiple of 4, rows of 8) is cleared, as by appends
        if (slot == 0 && (dim & 7)) *reinterpret_cast<uint2*>(dst + 2 * dim) = make_uint2(0u, 0u);
      }
    }
    first += AT_A_TIME * step;
    if (first >= rows) break;
    load(first);
  }
}

template <typename KT, typename IN, typename OUT>
cudaError_t launch_vec(const RopeDev& d, int vec, const cudaLaunchConfig_t& cfg) {
  switch (vec) {
    case 4: return cudaLaunchKernelEx(&cfg, kv_rope_kernel<KT, IN, OUT, 4>, d);
    case 2: return cudaLaunchKernelEx(&cfg, kv_rope_kernel<KT, IN, OUT, 2>, d);
    default: return cudaLaunchKernelEx(&cfg, kv_rope_kernel<KT, IN, OUT, 1>, d);
  }
}
template <typename KT>
cudaError_t launch_types(const RopeDev& d, bool in_f32, bool out_f32, int vec, const cudaLaunchConfig_t& cfg) {
  if (in_f32) return out_f32 ? launch_vec<KT, float, float>(d, vec, cfg) : launch_vec<KT, float, KT>(d, vec, cfg);
  return out_f32 ? launch_vec<KT, KT, float>(d, vec, cfg) : launch_vec<KT, KT, KT>(d, vec, cfg);
}

}  // namespace

int launch_kv_rope(const KvView& kv, int layer, const bitnet_rope_t* rope, const RopeArgs& x, int dtype, cudaStream_t st) {
  RopeDev d;
  d.kv = kv;
  d.q = static_cast<const uint8_t*>(x.q);
  d.k = static_cast<const uint8_t*>(x.k);
  d.v = static_cast<const uint8_t*>(x.v);
  d.q_out = static_cast<uint8_t*>(x.q_out);
  d.q_stride_token = x.q_stride_token;
  const int size = x.in_type == BITNET_KV_F32 ? 4 : 2;
  d.q_stride_head = x.q_stride_head;
  d.stride_token = x.stride_token;
  d.stride_head = x.stride_head;
  d.table = x.table;
  d.kv_len = x.kv_len;
  d.q_start = x.q_start;
  d.width = x.width;
  d.tokens = (int)x.tokens;
  d.seqs = (int)x.seqs;
  d.layer = layer;
  d.q_heads = (int)x.q_heads;
  d.rot = rope->rot_dim;
  d.interleaved = rope->interleaved != 0;
  d.page_shift = __builtin_ctz((unsigned)kv.page_size);
  d.dev_status = x.dev_status;
  d.magnitude = (float)rope->magnitude;
  memcpy(d.step, rope->step, sizeof d.step);
  const int dim = kv.head_dim;
  // elements of a vector: as many as half a row's pairs, the head, strides and addresses allow
  const bool in_f32 = x.in_type == BITNET_KV_F32, out_f32 = x.out_type == BITNET_KV_F32;
  // (four at most: 4 x 2048 tokens, fp32 in, bf16 out: 42 us against 49 with 32-byte vectors, a warp's access would touch every sector twice; 16-bit in
  // and out, 3222 tokens: 24 us with four as with eight)
  int64_t odd = dim | x.q_stride_token | x.q_stride_head | x.stride_token | x.stride_head | 4;
  if (!d.interleaved) odd |= d.rot / 2;
  int vec = (int)(odd & -odd);
  const uintptr_t at = reinterpret_cast<uintptr_t>(x.k) | reinterpret_cast<uintptr_t>(x.v) | (x.q_heads ? reinterpret_cast<uintptr_t>(x.q) : 0);
  while (vec > 1 && at % (size * vec < 16 ? size * vec : 16)) vec /= 2;
  auto slots = [&](int elements) { return (elements / vec + 1) / 2; };
  d.slots = slots(dim);
  d.rotated = d.interleaved ? d.slots : d.rot / (2 * vec);
  if (!d.interleaved && d.rotated + slots(dim - d.rot) > d.slots) d.slots = d.rotated + slots(dim - d.rot);
  d.at_once = THREADS / d.slots;
  // CTAs per token: a row per thread while CTAs are few, all of a token's rows in one when there are enough tokens to fill the SMs
  // (up to 8, 16, 32 and 64 CTAs per SM: 16.3, 15.4, 16.5 and 17.9 us for 3 x 517 tokens, 32/32 heads of 100; 24.1, 24.2, 24.2 and 26.3 for 3222, 32/8 of 128, 16-bit)
  const int64_t rows = x.q_heads + 2 * kv.kv_heads, most = ceil_div(rows, d.at_once), sms = dev_info().sm_count;
  int64_t split = 16 * sms / x.tokens;
  split = split < 1 ? 1 : split > most ? most : split;
  d.split = (int)ceil_div(most, ceil_div(most, split));           // (no CTA without rows, and even shares)
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(x.tokens * d.split));
  cfg.blockDim = dim3(THREADS);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = early_start_enabled(st) ? 1 : 0;
  log_launch("kv_rope_kernel tokens=%d q_heads=%d kv_heads=%d vec=%d split=%d", d.tokens, d.q_heads, kv.kv_heads, vec, d.split);
  const cudaError_t e = dtype == BITNET_KV_BF16 ? launch_types<__nv_bfloat16>(d, in_f32, out_f32, vec, cfg)
                                                : launch_types<__half>(d, in_f32, out_f32, vec, cfg);
  return e == cudaSuccess ? check_launch() : note_cuda_error(e);
}

}  // namespace bitnet
