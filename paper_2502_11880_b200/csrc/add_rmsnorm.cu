// Residual addition, root-mean-square norm and the int8 quantiser of the next linear (Alg. 1 Phase 1) in one pass over a row:
//
//   h = residual + x;  r = 1 / sqrt(mean(h^2) + eps);  y = (h r) w;  amax = max(max|y|, 1e-5);  q = rint(y * (127 / amax))
//
// One CTA per row, the row in registers between the two reductions, so that it crosses HBM once: x and the residual in, the new
// residual and one byte per element out.
// Rounding: the squares are summed in 64 bits and r is rounded once to binary32, so that it does not depend on the order of the sum
// (a few wrong bits of r would move codes that lie next to a border); from there every step is one binary32 operation, and the codes are
// those that bitnet_quant_act gives for y.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "device_utils.cuh"

namespace bitnet {
namespace {

struct NormDev {
  NormArgs a;
  double inv_k;
};

__device__ __forceinline__ float4 load4(const void* p, int64_t i, int type) {     // i: a multiple of 4 elements
  if (type == BITNET_KV_F32) return __ldcg(reinterpret_cast<const float4*>(static_cast<const float*>(p) + i));
  const uint2 w = __ldcg(reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + i));
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
};
__device__ __forceinline__ double block_sum(double v, double* red) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (lane == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = lane < (int)(blockDim.x >> 5) ? red[lane] : 0.0;
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float block_max(float v, float* red) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  if (lane == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = lane < (int)(blockDim.x >> 5) ? red[lane] : 0.0f;
#pragma unroll
  for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ void store_sum(int v, int* red, int32_t* to) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    int total = 0;
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) total += red[w];
    *to = total;
  }
}
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

// VPT: pieces of 4 elements per thread; XT, RT: types of x and of the residual (or NONE).  A CTA takes every gridDim.x-th row, and
// has the next one's loads on their way while it reduces and writes the present one.
template <int VPT, int XT, int RT>
__global__ void __launch_bounds__(1024) add_rmsnorm_kernel(const __grid_constant__ NormDev d) {
  const NormArgs& a = d.a;
  __shared__ Red red;
  const int tid = threadIdx.x, nt = blockDim.x, n4 = (int)(a.K / 4);
  if (tid == 0) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  Raw<XT> x[VPT];
  Raw<RT> e[VPT];
  auto fetch = [&](int64_t t) {
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int i = tid + k * nt;
      if (i < n4) x[k] = load_raw<XT>(a.x, t * a.stride_x + 4 * (int64_t)i);
    }
    if constexpr (RT != NONE) {
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        const int i = tid + k * nt;
        if (i < n4) e[k] = load_raw<RT>(a.residual, t * a.stride_residual + 4 * (int64_t)i);
      }
    }
  };
  constexpr bool AHEAD = VPT <= 4;               // (eight pieces and the next eight would not fit the registers)
  int64_t t = blockIdx.x;
  if (AHEAD) fetch(t);
  for (;;) {
    float4 h[VPT];
    double sum = 0.0;
    if (!AHEAD) {
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        const int i = tid + k * nt;
        if (i < n4) h[k] = widen(load_raw<XT>(a.x, t * a.stride_x + 4 * (int64_t)i));
      }
    }
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int i = tid + k * nt;
      if (AHEAD || i >= n4) h[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i >= n4) continue;
      if (AHEAD) h[k] = widen(x[k]);
      if constexpr (RT != NONE) {
        const float4 r = widen(AHEAD ? e[k] : load_raw<RT>(a.residual, t * a.stride_residual + 4 * (int64_t)i));
        h[k].x = rounded(h[k].x + r.x, RT);
        h[k].y = rounded(h[k].y + r.y, RT);
        h[k].z = rounded(h[k].z + r.z, RT);
        h[k].w = rounded(h[k].w + r.w, RT);
        store4(a.residual_out, t * a.stride_residual_out + 4 * (int64_t)i, RT, h[k]);
      }
      sum = fma((double)h[k].x, (double)h[k].x, sum);
      sum = fma((double)h[k].y, (double)h[k].y, sum);
      sum = fma((double)h[k].z, (double)h[k].z, sum);
      sum = fma((double)h[k].w, (double)h[k].w, sum);
    }
    const int64_t next = t + gridDim.x;
    if (AHEAD && next < a.T) fetch(next);
    float4 w[VPT <= 2 ? VPT : 1];                // (few pieces: the weights come with the row, ahead of the reductions)
    if constexpr (VPT <= 2) {
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        const int i = tid + k * nt;
        w[k] = a.weight && i < n4 ? load4(a.weight, 4 * (int64_t)i, a.weight_type) : make_float4(1.f, 1.f, 1.f, 1.f);
      }
    }
    const float r = inverse_root(block_sum(sum, red.sum) * d.inv_k + a.eps);
    float top = 0.0f;
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int i = tid + k * nt;
      float4 v = make_float4(1.f, 1.f, 1.f, 1.f);
      if constexpr (VPT <= 2) v = w[k];
      else if (a.weight && i < n4) v = load4(a.weight, 4 * (int64_t)i, a.weight_type);
      h[k] = make_float4(scaled(h[k].x, r, v.x), scaled(h[k].y, r, v.y), scaled(h[k].z, r, v.z), scaled(h[k].w, r, v.w));
      if (i < n4) top = fmaxf(top, absmax4(h[k]));
    }
    const float amax = fmaxf(block_max(top, red.top), 1e-5f), s = __fdiv_rn(127.0f, amax);
    int codes = 0;
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int i = tid + k * nt;
      if (i >= n4) continue;
      const int c = quant4_packed(h[k], s);
      codes = __dp4a(c, 0x01010101, codes);
      reinterpret_cast<int*>(a.q + t * a.K)[i] = c;
      if (a.y) store4(a.y, t * a.K + 4 * (int64_t)i, a.y_type, h[k]);
    }
    if (tid == 0) a.act_scale[t] = __fdiv_rn(amax, 127.0f);
    if (a.act_sum) store_sum(codes, red.codes, a.act_sum + t);
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
  if (a.act_sum) store_sum(codes, red.codes, a.act_sum + t);
}

bool pieces_of_4(const void* p, int64_t stride, int type) {
  return !p || (reinterpret_cast<uintptr_t>(p) % (type == BITNET_KV_F32 ? 16 : 8) == 0 && stride % 4 == 0);
}
int threads_for(int64_t pieces) {               // whole warps
  const int64_t n = ceil_div(pieces, 32) * 32;
  return (int)(n < 64 ? 64 : n > 1024 ? 1024 : n);
}

template <int VPT, int XT>
cudaError_t launch_residual(const NormDev& d, const cudaLaunchConfig_t& cfg) {
  if (!d.a.residual) return cudaLaunchKernelEx(&cfg, add_rmsnorm_kernel<VPT, XT, NONE>, d);
  switch (d.a.residual_type) {
    case BITNET_KV_F32: return cudaLaunchKernelEx(&cfg, add_rmsnorm_kernel<VPT, XT, BITNET_KV_F32>, d);
    case BITNET_KV_BF16: return cudaLaunchKernelEx(&cfg, add_rmsnorm_kernel<VPT, XT, BITNET_KV_BF16>, d);
    default: return cudaLaunchKernelEx(&cfg, add_rmsnorm_kernel<VPT, XT, BITNET_KV_F16>, d);
  }
}
template <int VPT>
cudaError_t launch_x(const NormDev& d, const cudaLaunchConfig_t& cfg) {
  switch (d.a.x_type) {
    case BITNET_KV_F32: return launch_residual<VPT, BITNET_KV_F32>(d, cfg);
    case BITNET_KV_BF16: return launch_residual<VPT, BITNET_KV_BF16>(d, cfg);
    default: return launch_residual<VPT, BITNET_KV_F16>(d, cfg);
  }
}

}  // namespace

int launch_add_rmsnorm(const NormArgs& a, cudaStream_t st) {
  NormDev d;
  d.a = a;
  d.inv_k = 1.0 / (double)a.K;
  const bool vec = a.K % 4 == 0 && a.K <= 32768 && pieces_of_4(a.x, a.stride_x, a.x_type) && pieces_of_4(a.residual, a.stride_residual, a.residual_type) &&
                   pieces_of_4(a.residual_out, a.stride_residual_out, a.residual_type) && pieces_of_4(a.weight, 0, a.weight_type) &&
                   pieces_of_4(a.y, 0, a.y_type) && pieces_of_4(a.q, 0, BITNET_KV_BF16);
  const int64_t n4 = ceil_div(a.K, 4);
  // pieces per thread: as many threads as a row has pieces where rows are few (latency), four pieces where they fill the SMs
  int vpt = a.T > 2 * (int64_t)dev_info().sm_count ? 4 : 1;
  while (vpt < 8 && ceil_div(n4, vpt) > 1024) vpt *= 2;
  cudaLaunchConfig_t cfg = {};
  const int threads = threads_for(vec ? ceil_div(n4, vpt) : ceil_div(a.K, 4));
  const int64_t resident = (int64_t)dev_info().sm_count * (1024 / threads);          // CTAs of 64 registers a thread
  cfg.gridDim = dim3((unsigned)(vec && a.T > resident ? resident : a.T));
  cfg.blockDim = dim3((unsigned)threads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = early_start_enabled(st) ? 1 : 0;
  if (log_enabled()) log_launch("add_rmsnorm T=%lld K=%lld vec=%d vpt=%d", (long long)a.T, (long long)a.K, (int)vec, vpt);
  cudaError_t e;
  if (!vec) e = cudaLaunchKernelEx(&cfg, add_rmsnorm_any_kernel, d);
  else if (vpt == 1) e = launch_x<1>(d, cfg);
  else if (vpt == 2) e = launch_x<2>(d, cfg);
  else if (vpt == 4) e = launch_x<4>(d, cfg);
  else e = launch_x<8>(d, cfg);
  return e == cudaSuccess ? check_launch() : note_cuda_error(e);
}

}  // namespace bitnet
