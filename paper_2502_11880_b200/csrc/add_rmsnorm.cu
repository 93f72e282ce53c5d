// Residual addition, root-mean-square norm and the int8 quantiser of the next linear (Alg. 1 Phase 1) in one pass over a row:
//
//   h = residual + x;  r = 1 / sqrt(mean(h^2) + eps);  y = (h r) w;  amax = max(max|y|, 1e-5);  q = rint(y * (127 / amax))
//
// One CTA per row, the row in registers between the two reductions, so that it crosses HBM once: x and the residual in, the new
// residual and one byte per element out.
// Rounding: the squares are summed in 64 bits and r is rounded once to binary32, so that it does not depend on the order of the sum
// (a few wrong bits of r would move codes that lie next to a border); from there every step is one binary32 operation, and the codes are
// those that bitnet_quant_act gives for y.
//
// Bound by HBM for many rows, by the latency of loads and two reductions for few.  Measured (us, a B200): 1 x 4096: 2.3; 16 x 28672: 4.2; 4099 x 8192, fp32 x
// and a bf16 residual: 56 (5.4 TB/s, 0.82 of a copy's rate; what is left is the latency of the reductions between loads and codes).  There the next row's loads ahead of the
// reductions took it from 98 to 74, types as template parameters to 69, weights through the first-level cache to 64, one rounding of the new residual for
// the store and the sum to 62, maxima by one instruction a warp to 60, the next row through shared memory to 56.  16-bit rows have the same instructions for half the
// bytes: bf16, without / with a residual: 4096 x 8192: 41 / 53 (HBM needs 15 / 36), 4096 x 14336: 68 / 106 (27 / 63).  The general kernel, three walks over a row by
// single elements: 4096 x 8191, fp32 both: 339 (67), bf16 both: 470 (36); 16 x 8191: 10; 1 x 4095: 7.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "device_utils.cuh"
#include "kv_cache.cuh"

namespace bitnet {
namespace {

constexpr int MOST_STAGED = 64 * 1024;    // bytes of a row in shared memory: 8192 elements of x and residual, or 16384 of x
constexpr int64_t MOST_K = 8 * 16384;     // a cluster of 8 CTAs of 1024 threads with four pieces each

struct NormDev {
  NormArgs a;
  double inv_k;
};

// Four weights, which every row takes again: through the first-level cache.
__device__ __forceinline__ float4 load_weights(const void* p, int i, int type) {
  if (type == BITNET_KV_F32) return __ldg(static_cast<const float4*>(p) + i);
  const uint2 w = __ldg(static_cast<const uint2*>(p) + i);
  if (type == BITNET_KV_BF16)
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
  const float2 lo = __half22float2(*reinterpret_cast<const __half2*>(&w.x)), hi = __half22float2(*reinterpret_cast<const __half2*>(&w.y));
  return make_float4(lo.x, lo.y, hi.x, hi.y);
}
__device__ __forceinline__ float load1(const void* p, int64_t i, int type) {
  if (type == BITNET_KV_F32) return static_cast<const float*>(p)[i];
  if (type == BITNET_KV_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  return __half2float(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ float rounded(float v, int type) {
  if (type == BITNET_KV_F32) return v;
  return type == BITNET_KV_BF16 ? __bfloat162float(__float2bfloat16_rn(v)) : __half2float(__float2half_rn(v));
}
__device__ __forceinline__ void store1(void* p, int64_t i, int type, float v) {
  if (type == BITNET_KV_F32) static_cast<float*>(p)[i] = v;
  else if (type == BITNET_KV_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
  else static_cast<__half*>(p)[i] = __float2half_rn(v);
}
__device__ __forceinline__ void store4(void* p, int64_t i, int type, const float4& v) {
  if (type == BITNET_KV_F32) {
    *reinterpret_cast<float4*>(static_cast<float*>(p) + i) = v;
  } else if (type == BITNET_KV_BF16) {
    const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + i) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
  } else {
    const __half2 lo = __floats2half2_rn(v.x, v.y), hi = __floats2half2_rn(v.z, v.w);
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + i) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
  }
}

// Of all threads of the CTA, the same value in each (every warp sums the warps' parts in the same order).
struct Red {
  double sum[32];
  float top[32];
  int codes[32];
  // of a cluster's CTAs
  double cta_sum[8];
  float cta_top[8];
  int cta_codes[8];
};
__device__ __forceinline__ double block_sum(double v, double* red) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (lane == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  const int slot = blockDim.x > 512 ? lane : lane & 15;
  v = slot < (int)(blockDim.x >> 5) ? red[slot] : 0.0;
  if (blockDim.x > 512) v += __shfl_xor_sync(0xffffffffu, v, 16);
#pragma unroll
  for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float block_max(float v, float* red) {
  // (numbers from 0 on: their bits are in the same order)
  const int lane = threadIdx.x & 31;
  v = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v)));
  if (lane == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = lane < (int)(blockDim.x >> 5) ? red[lane] : 0.0f;
  return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v)));
}
// In thread 0.
__device__ __forceinline__ int sum_of_codes(int v, int* red) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  int total = 0;
  if (threadIdx.x == 0)
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) total += red[w];
  return total;
}
// Into the shared memory of CTA `rank` of the cluster, at the place that p has here.
__device__ __forceinline__ uint32_t peer(const void* p, int rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ void tell(const double* p, int rank, double v) {
  asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(peer(p, rank)), "d"(v) : "memory");
}
__device__ __forceinline__ void tell(const float* p, int rank, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(peer(p, rank)), "f"(v) : "memory");
}
__device__ __forceinline__ void tell(const int* p, int rank, int v) {
  asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(peer(p, rank)), "r"(v) : "memory");
}
__device__ __forceinline__ void arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void await() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// 1 / sqrt(v), rounded once to binary32: two Newton steps in 64 bits from the 32-bit estimate, where that has a range to stand on.
__device__ __forceinline__ float inverse_root(double v) {
  if (!(v > 1e-30 && v < 1e30)) return (float)(1.0 / sqrt(v));
  double y = (double)rsqrtf((float)v);
  const double half = 0.5 * v;
#pragma unroll
  for (int i = 0; i < 2; ++i) y = y * (1.5 - half * y * y);
  return (float)y;
}
__device__ __forceinline__ float scaled(float h, float r, float w) { return __fmul_rn(__fmul_rn(h, r), w); }

// Four elements as they lie in memory: 16 bytes of binary32, or 8.
constexpr int NONE = -1;
template <int TYPE>
struct Raw {
  uint2 v;
};
template <>
struct Raw<BITNET_KV_F32> {
  uint4 v;
};
template <int TYPE>
__device__ __forceinline__ Raw<TYPE> load_raw(const void* p, int64_t i) {
  Raw<TYPE> r;
  if constexpr (TYPE == BITNET_KV_F32) r.v = __ldcg(reinterpret_cast<const uint4*>(static_cast<const float*>(p) + i));
  else r.v = __ldcg(reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + i));
  return r;
}
__device__ __forceinline__ float4 widen(const Raw<BITNET_KV_F32>& r) {
  return make_float4(__uint_as_float(r.v.x), __uint_as_float(r.v.y), __uint_as_float(r.v.z), __uint_as_float(r.v.w));
}
template <int TYPE>
__device__ __forceinline__ float4 widen(const Raw<TYPE>& r) {
  const uint2 w = r.v;
  if (TYPE == BITNET_KV_BF16)
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
  const float2 lo = __half22float2(*reinterpret_cast<const __half2*>(&w.x)), hi = __half22float2(*reinterpret_cast<const __half2*>(&w.y));
  return make_float4(lo.x, lo.y, hi.x, hi.y);
}

template <int TYPE>
__device__ __forceinline__ Raw<TYPE> narrow(const float4& v) {
  Raw<TYPE> r;
  if constexpr (TYPE == BITNET_KV_F32) {
    r.v = make_uint4(__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w));
  } else if constexpr (TYPE == BITNET_KV_BF16) {
    const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
    r.v = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
  } else {
    const __half2 lo = __floats2half2_rn(v.x, v.y), hi = __floats2half2_rn(v.z, v.w);
    r.v = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
  }
  return r;
}
// A thread's piece on its way into shared memory, or from there.
template <int TYPE>
__device__ __forceinline__ void copy_raw(uint32_t dst, const void* p, int64_t i) {
  if constexpr (TYPE == BITNET_KV_F32)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(static_cast<const float*>(p) + i) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(static_cast<const uint16_t*>(p) + i) : "memory");
}
template <int TYPE>
__device__ __forceinline__ void store_raw(void* p, int64_t i, const Raw<TYPE>& r) {
  if constexpr (TYPE == BITNET_KV_F32) *reinterpret_cast<uint4*>(static_cast<float*>(p) + i) = r.v;
  else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + i) = r.v;
}

// VPT: pieces of 4 elements per thread; XT, RT: types of x and of the residual (or NONE).  A CTA takes every gridDim.x-th row, and
// has the next one's loads on their way while it reduces and writes the present one.  WIDE: the CTAs of a cluster share a row; their sums and
// maxima meet in every CTA's shared memory (a barrier of the cluster lies between any two uses of a place there).
// STAGED: the next row comes through shared memory, every thread's pieces by and for itself (which leaves two CTAs of 512 threads per SM the registers
// to have much of a row's work under way: 4099 x 8192: 56 us against 60 by registers, with two rows on their way 63, with three CTAs per SM 62).
template <int VPT, int XT, int RT, bool WIDE, bool STAGED>
__global__ void __launch_bounds__(STAGED ? 512 : 1024, STAGED ? 2 : 1) add_rmsnorm_kernel(const __grid_constant__ NormDev d) {
  const NormArgs& a = d.a;
  __shared__ Red red;
  int ctas = 1, rank = 0;
  if constexpr (WIDE) {
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    arrive();                                    // (the others may write here: awaited before the first such write)
  }
  // this CTA's pieces of a row: [from, n4)
  const int tid = threadIdx.x, nt = blockDim.x, all4 = (int)(a.K / 4), share = (all4 + ctas - 1) / ctas;
  const int from = min(all4, rank * share), n4 = min(all4, from + share);
  const int64_t rows_at_once = gridDim.x / ctas;
  if (tid == 0) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  Raw<XT> x[VPT];
  Raw<RT> e[VPT];
  extern __shared__ __align__(16) uint8_t staged[];        // the pieces of x, then those of the residual
  constexpr int XB = (int)sizeof(Raw<XT>), EB = RT == NONE ? 0 : (int)sizeof(Raw<RT>);
  uint8_t* const x_at = staged + tid * XB;
  uint8_t* const e_at = staged + VPT * nt * XB + tid * EB;
  auto copy = [&](int64_t t) {
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int i = from + tid + k * nt;
      if (i < n4) copy_raw<XT>(smem_u32(x_at) + k * nt * XB, a.x, t * a.stride_x + 4 * (int64_t)i);
    }
    if constexpr (RT != NONE) {
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        const int i = from + tid + k * nt;
        if (i < n4) copy_raw<RT>(smem_u32(e_at) + k * nt * EB, a.residual, t * a.stride_residual + 4 * (int64_t)i);
      }
    }
    cp_commit();
  };
  auto fetch = [&](int64_t t) {
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int i = from + tid + k * nt;
      if (i < n4) x[k] = load_raw<XT>(a.x, t * a.stride_x + 4 * (int64_t)i);
    }
    if constexpr (RT != NONE) {
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        const int i = from + tid + k * nt;
        if (i < n4) e[k] = load_raw<RT>(a.residual, t * a.stride_residual + 4 * (int64_t)i);
      }
    }
  };
  int64_t t = blockIdx.x / ctas;
  bool met = !WIDE;
  if constexpr (STAGED) copy(t);
  else fetch(t);
  for (;;) {
    if constexpr (STAGED) {
      cp_wait<0>();
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        x[k] = *reinterpret_cast<const Raw<XT>*>(x_at + k * nt * XB);
        if constexpr (RT != NONE) e[k] = *reinterpret_cast<const Raw<RT>*>(e_at + k * nt * EB);
      }
    }
    float4 h[VPT];
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int i = from + tid + k * nt;
      h[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i >= n4) continue;
      h[k] = widen(x[k]);
      if constexpr (RT != NONE) {
        const float4 r = widen(e[k]);
        const Raw<RT> stored = narrow<RT>(make_float4(h[k].x + r.x, h[k].y + r.y, h[k].z + r.z, h[k].w + r.w));
        store_raw<RT>(a.residual_out, t * a.stride_residual_out + 4 * (int64_t)i, stored);
        h[k] = widen(stored);
      }
      sum = fma((double)h[k].x, (double)h[k].x, sum);
      sum = fma((double)h[k].y, (double)h[k].y, sum);
      sum = fma((double)h[k].z, (double)h[k].z, sum);
      sum = fma((double)h[k].w, (double)h[k].w, sum);
    }
    const int64_t next = t + rows_at_once;
    if (next < a.T) {
      if constexpr (STAGED) copy(next);          // (in the place of values that have been used above)
      else fetch(next);
    }
    float4 w[VPT <= 2 ? VPT : 1];                // (few pieces: the weights come with the row, ahead of the reductions)
    if constexpr (VPT <= 2) {
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        const int i = from + tid + k * nt;
        w[k] = a.weight && i < n4 ? load_weights(a.weight, i, a.weight_type) : make_float4(1.f, 1.f, 1.f, 1.f);
      }
    }
    sum = block_sum(sum, red.sum);
    if constexpr (WIDE) {
      if (!met) await();
      met = true;
      if (tid < ctas) tell(&red.cta_sum[rank], tid, sum);
      arrive();
      await();
      sum = 0.0;
      for (int p = 0; p < ctas; ++p) sum += red.cta_sum[p];
    }
    const float r = inverse_root(sum * d.inv_k + a.eps);
    float top = 0.0f;
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int i = from + tid + k * nt;
      float4 v = make_float4(1.f, 1.f, 1.f, 1.f);
      if constexpr (VPT <= 2) v = w[k];
      else if (a.weight && i < n4) v = load_weights(a.weight, i, a.weight_type);
      h[k] = make_float4(scaled(h[k].x, r, v.x), scaled(h[k].y, r, v.y), scaled(h[k].z, r, v.z), scaled(h[k].w, r, v.w));
      if (i < n4) top = fmaxf(top, absmax4(h[k]));
    }
    top = block_max(top, red.top);
    if constexpr (WIDE) {
      if (tid < ctas) tell(&red.cta_top[rank], tid, top);
      arrive();
      await();
      for (int p = 0; p < ctas; ++p) top = fmaxf(top, red.cta_top[p]);
    }
    const float amax = fmaxf(top, 1e-5f), s = __fdiv_rn(127.0f, amax);
    int codes = 0;
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int i = from + tid + k * nt;
      if (i >= n4) continue;
      const int c = quant4_packed(h[k], s);
      codes = __dp4a(c, 0x01010101, codes);
      reinterpret_cast<int*>(a.q + t * a.K)[i] = c;
      if (a.y) store4(a.y, t * a.K + 4 * (int64_t)i, a.y_type, h[k]);
    }
    if (tid == 0 && rank == 0) a.act_scale[t] = __fdiv_rn(amax, 127.0f);
    if (a.act_sum) {
      codes = sum_of_codes(codes, red.codes);
      if constexpr (WIDE) {
        if (tid == 0) tell(&red.cta_codes[rank], 0, codes);
        arrive();
        await();
        codes = 0;
        for (int p = 0; p < ctas; ++p) codes += red.cta_codes[p];
      }
      if (tid == 0 && rank == 0) a.act_sum[t] = codes;
    }
    if (next >= a.T) break;
    t = next;
  }
}

// Rows of any length, stride and alignment: three walks over the row (h is read back where it was written, by the same thread).
__global__ void __launch_bounds__(1024) add_rmsnorm_any_kernel(const __grid_constant__ NormDev d) {
  const NormArgs& a = d.a;
  __shared__ Red red;
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, nt = blockDim.x;
  if (tid == 0) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  double sum = 0.0;
  for (int64_t i = tid; i < a.K; i += nt) {
    float h = load1(a.x, t * a.stride_x + i, a.x_type);
    if (a.residual) {
      h = rounded(h + load1(a.residual, t * a.stride_residual + i, a.residual_type), a.residual_type);
      store1(a.residual_out, t * a.stride_residual_out + i, a.residual_type, h);
    }
    sum = fma((double)h, (double)h, sum);
  }
  const float r = inverse_root(block_sum(sum, red.sum) * d.inv_k + a.eps);
  auto value = [&](int64_t i) {
    const float h = a.residual ? load1(a.residual_out, t * a.stride_residual_out + i, a.residual_type) : load1(a.x, t * a.stride_x + i, a.x_type);
    return scaled(h, r, a.weight ? load1(a.weight, i, a.weight_type) : 1.0f);
  };
  float top = 0.0f;
  for (int64_t i = tid; i < a.K; i += nt) top = fmaxf(top, fabsf(value(i)));
  const float amax = fmaxf(block_max(top, red.top), 1e-5f), s = __fdiv_rn(127.0f, amax);
  int codes = 0;
  for (int64_t i = tid; i < a.K; i += nt) {
    const float y = value(i);
    const int c = quant1(y, s);
    codes += c;
    a.q[t * a.K + i] = (int8_t)c;
    if (a.y) store1(a.y, t * a.K + i, a.y_type, y);
  }
  if (tid == 0) a.act_scale[t] = __fdiv_rn(amax, 127.0f);
  if (a.act_sum) {
    codes = sum_of_codes(codes, red.codes);
    if (tid == 0) a.act_sum[t] = codes;
  }
}

bool pieces_of_4(const void* p, int64_t stride, int type) {
  return !p || (reinterpret_cast<uintptr_t>(p) % (type == BITNET_KV_F32 ? 16 : 8) == 0 && stride % 4 == 0);
}
int threads_for(int64_t pieces) {               // whole warps
  const int64_t n = ceil_div(pieces, 32) * 32;
  return (int)(n < 64 ? 64 : n > 1024 ? 1024 : n);
}

template <int VPT, int XT, int RT, bool WIDE, bool STAGED>
cudaError_t launch_one(const NormDev& d, const cudaLaunchConfig_t& cfg) {
  auto kernel = add_rmsnorm_kernel<VPT, XT, RT, WIDE, STAGED>;
  if (STAGED) {
    static std::atomic<uint64_t> have{0};
    if (allow_smem(kernel, MOST_STAGED, &have) != BITNET_OK) return cudaErrorInvalidValue;
  }
  return cudaLaunchKernelEx(&cfg, kernel, d);
}
template <int VPT, int XT, bool WIDE, bool STAGED>
cudaError_t launch_residual(const NormDev& d, const cudaLaunchConfig_t& cfg) {
  if (VPT == 8 || !d.a.residual) return launch_one<VPT, XT, NONE, WIDE, STAGED>(d, cfg);
  if constexpr (VPT < 8) switch (d.a.residual_type) {
    case BITNET_KV_F32: return launch_one<VPT, XT, BITNET_KV_F32, WIDE, STAGED>(d, cfg);
    case BITNET_KV_BF16: return launch_one<VPT, XT, BITNET_KV_BF16, WIDE, STAGED>(d, cfg);
    default: return launch_one<VPT, XT, BITNET_KV_F16, WIDE, STAGED>(d, cfg);
  }
}
template <int VPT, bool WIDE, bool STAGED>
cudaError_t launch_x(const NormDev& d, const cudaLaunchConfig_t& cfg) {
  switch (d.a.x_type) {
    case BITNET_KV_F32: return launch_residual<VPT, BITNET_KV_F32, WIDE, STAGED>(d, cfg);
    case BITNET_KV_BF16: return launch_residual<VPT, BITNET_KV_BF16, WIDE, STAGED>(d, cfg);
    default: return launch_residual<VPT, BITNET_KV_F16, WIDE, STAGED>(d, cfg);
  }
}

}  // namespace

int launch_add_rmsnorm(const NormArgs& a, cudaStream_t st) {
  NormDev d;
  d.a = a;
  d.inv_k = 1.0 / (double)a.K;
  const bool vec = a.K % 4 == 0 && a.K <= MOST_K && pieces_of_4(a.x, a.stride_x, a.x_type) && pieces_of_4(a.residual, a.stride_residual, a.residual_type) &&
                   pieces_of_4(a.residual_out, a.stride_residual_out, a.residual_type) && pieces_of_4(a.weight, 0, a.weight_type) &&
                   pieces_of_4(a.y, 0, a.y_type) && pieces_of_4(a.q, 0, BITNET_KV_BF16);
  const int64_t sms = dev_info().sm_count;
  // A cluster of CTAs for a row that four pieces of 1024 threads do not hold, and for long rows that are few (16 x 28672: 7.0 us by one CTA with eight pieces a
  // thread, 4.5 by four).
  int ctas = 1;
  while (vec && ctas < 8 && (a.K > 16384 * (int64_t)ctas || (a.K >= 16384 && a.T * ctas * 4 <= sms && ctas < 4))) ctas *= 2;
  const int64_t n4 = ceil_div(ceil_div(a.K, 4), ctas);
  // pieces per thread: as many threads as there are pieces where rows are few (latency), four pieces where they fill the SMs
  int vpt = a.T * ctas > 2 * sms ? 4 : 1;
  while (vpt < 4 && ceil_div(n4, vpt) > 1024) vpt *= 2;
  if (ctas > 1 && vpt < 2) vpt = 2;
  // Many rows come through shared memory, two CTAs or more to an SM, except longer ones with a residual, as eight pieces a thread would take more registers
  // than there are (4096 x 14336, bf16: 114 us against 104; without a residual 65 against 73) or 64 KB a row (4096 x 8192, both fp32: 79 against 75).
  const int64_t bytes4 = 4 * ((a.x_type == BITNET_KV_F32 ? 4 : 2) + (!a.residual ? 0 : a.residual_type == BITNET_KV_F32 ? 4 : 2));
  const bool staged = vec && ctas == 1 && a.T > 2 * sms && (!a.residual || (n4 <= 2048 && n4 * bytes4 <= 48 * 1024));
  if (staged && n4 > 2048) vpt = 8;
  const int threads = threads_for(vec ? ceil_div(n4, vpt) : n4);
  const int64_t resident = sms * (1024 / threads) / ctas;          // rows that CTAs of 64 registers a thread hold at a time
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((vec && a.T > resident ? resident : a.T) * ctas));
  cfg.blockDim = dim3((unsigned)threads);
  if (staged) cfg.dynamicSmemBytes = (size_t)(threads * vpt * bytes4);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int attrs = 0;
  if (ctas > 1) {
    attr[attrs].id = cudaLaunchAttributeClusterDimension;
    attr[attrs].val.clusterDim.x = ctas;
    attr[attrs].val.clusterDim.y = 1;
    attr[attrs++].val.clusterDim.z = 1;
  }
  if (early_start_enabled(st)) {
    attr[attrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[attrs++].val.programmaticStreamSerializationAllowed = 1;
  }
  cfg.attrs = attr;
  cfg.numAttrs = attrs;
  if (log_enabled()) log_launch("add_rmsnorm T=%lld K=%lld vec=%d vpt=%d ctas=%d", (long long)a.T, (long long)a.K, (int)vec, vpt, ctas);
  cudaError_t e;
  if (!vec) e = cudaLaunchKernelEx(&cfg, add_rmsnorm_any_kernel, d);
  else if (ctas > 1) e = vpt == 2 ? launch_x<2, true, false>(d, cfg) : launch_x<4, true, false>(d, cfg);
  else if (staged) e = vpt == 4 ? launch_x<4, false, true>(d, cfg) : launch_x<8, false, true>(d, cfg);
  else if (vpt == 1) e = launch_x<1, false, false>(d, cfg);
  else if (vpt == 2) e = launch_x<2, false, false>(d, cfg);
  else e = launch_x<4, false, false>(d, cfg);
  return e == cudaSuccess ? check_launch() : note_cuda_error(e);
}

}  // namespace bitnet
