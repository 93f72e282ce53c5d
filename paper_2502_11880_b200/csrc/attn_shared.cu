// Attention of single tokens of sequences that share beginnings, in three kernels:
//   1. the groups' prefixes: rows (sequence, query head) of a group against its prefix, read once, on the tensor cores (attn_prompt.cu), in
//      parts over the CTAs;
//   2. the sequences' own tokens (attn_decode.cu);
//   3. here: the join.  With a row's parts (m_k, l_k, O_k), each relative to its own maximum,
//        m = max m_k,  out = sum_k 2^(m_k - m) O_k / sum_k 2^(m_k - m) l_k
//      in the order of the parts, in fp32, rounded once.  A warp per row; its parts' maxima and sums are read by its lanes side by side, and all parts of O
//      are on their way together.
#include "kv_cache.cuh"

namespace bitnet {
namespace {

constexpr int ROWS = 128;                     // of a tile of kernel 1
constexpr int WARPS = 4;

struct JoinArgs {
  SharedParts p;
  uint8_t* out;
  const int32_t* group_start;
  const int32_t* prefix_len;
  int64_t rows;
  int q_heads, group, per_block, tile_tokens, groups, head_dim, ctas;
};

template <typename KT>
__device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

template <typename KT>
__global__ void __launch_bounds__(WARPS * 32) attn_shared_join_kernel(const __grid_constant__ JoinArgs a) {
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * WARPS + (threadIdx.x >> 5);
  // (groups are not written by the kernels before)
  const int tok = (int)(row / a.q_heads), head = (int)(row - (int64_t)tok * a.q_heads);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (row >= a.rows) return;
  const int d = 4 * lane;
  const bool mine = d < a.p.padded;
  const float4 zero = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const float2 own = __ldcg(a.p.own_ml + row);
  const float4 base = __ldcg(a.p.base_ml + row);
  const float4 own_o = mine ? __ldcg(reinterpret_cast<const float4*>(a.p.own_o + row * a.p.padded + d)) : zero;
  const float4 base_o = mine ? __ldcg(reinterpret_cast<const float4*>(a.p.base_o + row * a.p.padded + d)) : zero;
  const KvGroup g = kv_group_of(a.group_start, a.prefix_len, a.groups, tok, 0);

  const bool in_group = g.first >= 0;                      // otherwise there is nothing at the row's place
  // later parts: CTAs c0 + 1 .. c1 (any, where kernel 1 has given up), at this row's place in them
  const int c0 = max(__float_as_int(base.z), 0), c1 = in_group ? min(__float_as_int(base.w), a.ctas - 1) : 0;
  const int of_kv = head % a.group % a.per_block, at = (tok - (in_group ? g.first : tok)) % (2 * a.tile_tokens);
  const int place = at / a.tile_tokens * ROWS + at % a.tile_tokens * a.per_block + of_kv;

  // weights relative to a maximum that later parts may raise: 32 parts at a time
  float m = in_group ? fmaxf(own.x, base.x) : own.x;
  auto factor = [](float of, float to) { return of == -INFINITY ? 0.0f : exp2_approx(of - to); };
  float sum = factor(own.x, m) * own.y;
  float4 acc = zero;
  auto add = [&](float f, const float4& o) {
    if (f == 0.0f) return;                                 // (what a part without visible tokens has left may be anything)
    acc.x += f * o.x;
    acc.y += f * o.y;
    acc.z += f * o.z;
    acc.w += f * o.w;
  };
  add(factor(own.x, m), own_o);
  if (in_group) {
    sum += factor(base.x, m) * base.y;
    add(factor(base.x, m), base_o);
  }
  for (int c = c0 + 1; c <= c1; c += 32) {
    const int n = min(32, c1 - c + 1);
    const float2 ml = lane < n ? __ldcg(a.p.spill_ml + (int64_t)(c + lane) * 2 * ROWS + place) : make_float2(-INFINITY, 0.0f);
    float top = ml.x;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    top = fmaxf(top, m);
    const float f = factor(m, top);
    m = top;
    sum *= f;
    acc = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
    const float w = factor(ml.x, m), wl = w * ml.y;
    const float* o = a.p.spill_o + ((int64_t)c * 2 * ROWS + place) * a.p.padded + d;
    for (int k0 = 0; k0 < n; k0 += 8) {
      float4 v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k)
        v[k] = mine && k0 + k < n ? __ldcg(reinterpret_cast<const float4*>(o + (int64_t)(k0 + k) * 2 * ROWS * a.p.padded)) : zero;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (k0 + k >= n) break;
        sum += __shfl_sync(0xffffffffu, wl, k0 + k);
        add(__shfl_sync(0xffffffffu, w, k0 + k), v[k]);
      }
    }
  }
  if (d >= a.head_dim) return;
  const float inv = sum > 0.0f ? 1.0f / sum : (sum == 0.0f ? 0.0f : sum);          // nothing visible: 0; NaN stays NaN
  *reinterpret_cast<uint2*>(a.out + 2 * (row * a.head_dim + d)) = make_uint2(pack2<KT>(acc.x * inv, acc.y * inv), pack2<KT>(acc.z * inv, acc.w * inv));
}

}  // namespace

// The workspace of attn_shared: that of decode calls, then the rows' places, then the CTAs'.
size_t attn_shared_workspace_bytes(int64_t seqs, int64_t q_heads, int head_dim) {
  const size_t row = (size_t)ceil_div(head_dim, 16) * 64;
  return attn_decode_workspace_bytes() + (size_t)(seqs * q_heads) * (24 + 2 * row) + (size_t)dev_info().sm_count * 2 * ROWS * (8 + row);
}

int launch_attn_shared(const bitnet_kv_cache_t* c, const AttnArgs& x, void* ws, cudaStream_t st) {
  JoinArgs j;
  j.rows = x.tokens * x.q_heads;
  const int64_t padded = ceil_div(c->head_dim, 16) * 16, spill = (int64_t)dev_info().sm_count * 2 * ROWS;
  j.p.base_ml = reinterpret_cast<float4*>(attn_prompt_parts(ws));
  j.p.base_o = reinterpret_cast<float*>(j.p.base_ml + j.rows);
  j.p.own_o = j.p.base_o + j.rows * padded;
  j.p.spill_o = j.p.own_o + j.rows * padded;
  j.p.own_ml = reinterpret_cast<float2*>(j.p.spill_o + spill * padded);
  j.p.spill_ml = j.p.own_ml + j.rows;
  j.p.padded = (int)padded;
  int rc = launch_attn_shared_prefix(c, x, j.p, st);
  if (rc == BITNET_OK) rc = launch_attn_shared_own(c, x, j.p, ws, st);
  if (rc != BITNET_OK) return rc;
  j.out = static_cast<uint8_t*>(x.out);
  j.group_start = x.group_start;
  j.prefix_len = x.prefix_len;
  j.groups = (int)x.groups;
  j.q_heads = x.q_heads;
  j.group = x.q_heads / c->kv_heads;
  j.per_block = (int)ceil_div(j.group, ceil_div(j.group, ROWS));
  j.tile_tokens = ROWS / j.per_block;
  j.head_dim = c->head_dim;
  j.ctas = dev_info().sm_count;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ceil_div(j.rows, WARPS));
  cfg.blockDim = dim3(WARPS * 32);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = early_start_enabled(st) ? 1 : 0;
  const cudaError_t e = x.dtype == BITNET_KV_BF16 ? cudaLaunchKernelEx(&cfg, attn_shared_join_kernel<__nv_bfloat16>, j)
                                                  : cudaLaunchKernelEx(&cfg, attn_shared_join_kernel<__half>, j);
  return e == cudaSuccess ? check_launch() : note_cuda_error(e);
}

}  // namespace bitnet
