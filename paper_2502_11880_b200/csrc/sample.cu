// Drawing one token per row of logits by temperature, top-k, top-p and min-p from a given random number.
//
//   w[i] = exp((x[i] - max x) / T);  order: by x descending, equal ones by index
//   keep the first top_k of the order; of those the shortest beginning with sum >= top_p * their sum (at least one); of those w >= min_p;
//   token = the first index at which the sum of kept w in the order of the vocabulary exceeds u * (sum of kept w)
//
// No sort: what is kept by the first two rules is the order's beginning up to one item, which is found by descending through histograms
// of counts and sums.  One cluster of CTAs per row reads the row once from HBM into its shared memories; every pass after that runs
// over shared memory, and what the CTAs tell each other goes through distributed shared memory:
//   * the maximum;
//   * a histogram over (max - x) / T, linear, so that broad and peaked rows both spread over it;
//   * while the bin that holds the last kept item has more than LIST items: another histogram over that bin's range of the order
//     (64 bits: the value's bits, then the index, so that any number of equal values is taken apart too);
//   * the bin's items, ranked by counting: the last item kept, as a place in the order;
//   * the sum of what is kept per warp's stretch of the vocabulary; the warp whose stretch holds the token walks it.
// Sums: weights as 32-bit fixed point of the largest (weights below 2^-33 of it count as 0, are never drawn), added as integers of
// 64 bits: no sum depends on an order, a split or the size of the cluster.  The exponent is computed with the rounding errors of
// max - x and of the product carried along, so that a weight is off by the exponential's own 2^-22 only.
#include <cstring>
#include <type_traits>

#include "kv_cache.cuh"

namespace bitnet {
namespace {

constexpr int THREADS = 512, WARPS = THREADS / 32;
constexpr int BINS = THREADS;                // one per thread
constexpr int LIST = 256;                    // items that are ranked by counting
constexpr int MOST_CTAS = 8;                 // of a cluster
constexpr float ONE = 4294967296.0f;         // weight 1

struct Hist {
  uint32_t count[BINS], lo[BINS], hi[BINS];
};
struct Item {
  uint64_t at;                               // place in the order
  uint32_t w;
};
struct Say {                                 // what a CTA tells the others at a step
  float top;
  uint32_t index;
  uint64_t mass;
  uint32_t n;
};
struct Share {
  Hist hist;
  Item list[2][LIST];                        // of every second step, so that a CTA may go on while another one still reads
  Say say[2];
  // this CTA's own
  uint32_t bin_count[BINS];                  // the first histogram, of the whole row
  uint64_t bin_mass[BINS];
  uint64_t warp_mass[WARPS];
  uint32_t warp_count[WARPS];
  float warp_top[WARPS];
  Item all[LIST];
  uint32_t listed;
  // found by one thread
  int bin;
  uint32_t before_n, bin_n;
  uint64_t before_mass, found_at, found_mass;
};

__device__ __forceinline__ uint32_t peer(const void* p, int rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ uint32_t peer_u32(const void* p, int rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(peer(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ uint64_t peer_u64(const void* p, int rank) {
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(peer(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float value(__half v) { return __half2float(v); }
template <typename T>
struct alignas(sizeof(T) * 4) Four {
  T t[4];
};
// A number that is none is never drawn.
__device__ __forceinline__ float drawable(float v) { return v == v ? v : -INFINITY; }

// Ascending with the order: larger values first, then lower indices.
__device__ __forceinline__ uint64_t place(float x, uint32_t index) {
  const uint32_t b = __float_as_uint(x == 0.0f ? 0.0f : x);       // (-0 equals 0)
  const uint32_t up = b & 0x80000000u ? ~b : b | 0x80000000u;     // ascending with the value
  return (uint64_t)~up << 32 | index;
}

// Back to the value.
__device__ __forceinline__ float value_at(uint64_t at) {
  const uint32_t up = ~(uint32_t)(at >> 32);
  return __uint_as_float(up & 0x80000000u ? up & 0x7fffffffu : ~up);
}

constexpr float REACH = 33.0f;               // weights below 2^-33 of the largest count as 0
constexpr float PER_T = (BINS - 1) / REACH;  // bins of the first histogram per log2

struct Weigh {
  float top, c, c_lo;                        // the largest, finite; log2(e) / T in two pieces
  // (max - x) log2(e) / T, which rises as x falls.
  __device__ __forceinline__ float distance(float x, float& d) const {
    d = top - x;
    return d * c;
  }
  // The weight in units of 2^-32.  `exact`: max - x has no rounding error that matters (16-bit logits).
  template <bool EXACT>
  __device__ __forceinline__ float weight(float x, float d, float t) const {
    float low = fmaf(d, c, -t);
    low = fmaf(d, c_lo, low);
    if (!EXACT) {
      const float b = d - top;
      low = fmaf((top - (d - b)) - (x + b), c, low);
    }
    const float m = t + 12582912.0f, n = m - 12582912.0f;                           // 1.5 * 2^23: n = round(t), also in m's low bits
    float f;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(f) : "f"((n - t) - low));
    return f * __uint_as_float(((32u + 127u) << 23) - (__float_as_uint(m) << 23));
  }
};
// The bin of a distance below REACH.
__device__ __forceinline__ int bin_of(float t) { return (int)(__float_as_uint(fmaf(t, PER_T, 8388608.0f)) & (BINS - 1)); }
__device__ __forceinline__ uint32_t fixed(float w) { return __float2uint_rn(w); }   // (1 becomes 2^32 - 1)

template <typename T, bool STAGED>
struct Slice {
  const T* row;        // the row, in global memory
  T* kept;             // STAGED: the slice in shared memory
  int first;           // index of local element 0 (which may lie before the slice, so that pieces of 16 bytes agree)
  int begin, end;      // local elements that belong to the slice
  bool infinite;       // the row's largest is infinite: those count as 0, all others as -infinity
  __device__ __forceinline__ float only_infinite(float v) const { return v == INFINITY ? 0.0f : -INFINITY; }
  // (not STAGED)
  __device__ __forceinline__ float at(int i) const {
    const float v = i >= begin && i < end ? drawable(value(row[(int64_t)first + i])) : -INFINITY;
    return infinite ? only_infinite(v) : v;
  }
  // All elements of this CTA's slice, four at a time, each warp's one after the other; f(value, local index).
  template <typename F>
  __device__ __forceinline__ void each(int w0, int w1, F f) const {
    for (int i = w0 + 4 * (threadIdx.x & 31); i < w1; i += 128) {
      float x[4];
      if (STAGED) {
        const Four<T> v = *reinterpret_cast<const Four<T>*>(kept + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = value(v.t[k]);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = at(i + k);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) f(x[k], i + k);
    }
  }
};

__device__ __forceinline__ uint64_t warp_sum_u64(uint64_t v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <typename T, bool STAGED>
__global__ void __launch_bounds__(THREADS) sample_kernel(const __grid_constant__ SampleArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  Share& s = *reinterpret_cast<Share*>(smem_raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  int rank, ctas;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
  const int64_t r = blockIdx.x / ctas;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // ---- settings
  const float temperature = a.temperature ? __ldg(a.temperature + r) : 1.0f;
  const bool greedy = !(temperature > 0.0f);
  const int top_k = a.top_k ? __ldg(a.top_k + r) : 0;
  const float top_p = a.top_p ? __ldg(a.top_p + r) : 1.0f, min_p = a.min_p ? __ldg(a.min_p + r) : 0.0f;
  float u = __ldg(a.u + r);
  u = !(u > 0.0f) ? 0.0f : fminf(u, 0.99999994f);

  // ---- this CTA's slice of the row
  Slice<T, STAGED> x;
  x.row = static_cast<const T*>(a.logits) + r * a.stride;
  x.kept = reinterpret_cast<T*>(smem_raw + (sizeof(Share) + 15) / 16 * 16);
  const int i0 = min(a.vocab, rank * a.slice), i1 = min(a.vocab, i0 + a.slice);
  constexpr int PIECE = 16 / sizeof(T);
  const int off = (int)((reinterpret_cast<uintptr_t>(x.row + i0) & 15) / sizeof(T));
  x.first = i0 - off;
  x.begin = off;
  x.end = off + i1 - i0;
  x.infinite = false;
  const int length = (x.end + 127) / 128 * 128;              // of the slice with what pads it
  float top = -INFINITY;
  if (STAGED) {
    const T none = T(-INFINITY);
    const T* from = x.row + x.first;                          // (at a multiple of 16 bytes; only [begin, end) is read)
#pragma unroll 4
    for (int i = PIECE * tid; i < length; i += PIECE * THREADS) {
      struct alignas(16) Piece {
        T t[PIECE];
      } p;
      if (i >= x.begin && i + PIECE <= x.end) {
        *reinterpret_cast<uint4*>(&p) = __ldcg(reinterpret_cast<const uint4*>(from + i));
      } else {
#pragma unroll
        for (int k = 0; k < PIECE; ++k) p.t[k] = i + k >= x.begin && i + k < x.end ? from[i + k] : none;
      }
#pragma unroll
      for (int k = 0; k < PIECE; ++k) {
        const float v = value(p.t[k]);
        if (!(v == v)) p.t[k] = none;
        top = fmaxf(top, v);                                  // (a NaN is passed over)
      }
      *reinterpret_cast<uint4*>(x.kept + i) = *reinterpret_cast<const uint4*>(&p);
    }
  } else {
    for (int i = x.begin + tid; i < x.end; i += THREADS) top = fmaxf(top, drawable(value(x.row[(int64_t)x.first + i])));
  }
  s.hist.count[tid] = s.hist.lo[tid] = s.hist.hi[tid] = 0;
#pragma unroll
  for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) s.warp_top[warp] = top;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < WARPS; ++w) top = fmaxf(top, s.warp_top[w]);
    s.say[0].top = top;
  }
  uint32_t step = 0;                                          // the buffers of this step: [step & 1]
  cluster_barrier();
  for (int p = 0; p < ctas; ++p) top = p ? fmaxf(top, __uint_as_float(peer_u32(&s.say[0].top, p))) : __uint_as_float(peer_u32(&s.say[0].top, 0));
  ++step;

  // a warp's stretch of the slice
  const int stretch = (length / 128 + WARPS - 1) / WARPS * 128;
  const int w0 = min(length, warp * stretch), w1 = min(length, w0 + stretch);
  if (top == -INFINITY) {                                     // nothing can be drawn
    if (rank == 0 && tid == 0) {
      a.tokens[r] = -1;
      if (a.prob) a.prob[r] = 0.0f;
    }
    cluster_barrier();                                        // (nobody leaves while the others read)
    return;
  }

  if (top == INFINITY) {
    x.infinite = true;
    top = 0.0f;
    if (STAGED) {
      for (int i = tid; i < length; i += THREADS) x.kept[i] = T(x.only_infinite(value(x.kept[i])));
      __syncthreads();
    }
  }

  constexpr bool EXACT = sizeof(T) == 2;
  Weigh weigh;
  weigh.top = top;
  const double c = greedy ? 1.0 : fmin(1.4426950408889634 / (double)temperature, 3e38);
  weigh.c = (float)c;
  weigh.c_lo = (float)(c - (double)weigh.c);
  const float least = min_p > 0.0f && !greedy ? fminf(min_p, 1.0f) * ONE : 0.0f;

  // ---- the last item that is kept: its value, and its index among equal ones
  float last = greedy ? top : -INFINITY;
  uint32_t last_index = greedy ? 0xffffffffu : 0u;
  const bool by_k = !greedy && top_k > 0 && top_k < a.vocab, by_p = !greedy && top_p < 1.0f;
  if (by_k || by_p) {
    // all items by their distance from the largest
    {
      Hist& h = s.hist;
      x.each(w0, w1, [&](float v, int) {
        float d;
        const float t = weigh.distance(v, d);
        if (!(t < REACH)) return;
        const uint32_t w = fixed(weigh.weight<EXACT>(v, d, t));
        const int b = bin_of(t);
        atomicAdd(&h.count[b], 1u);
        if (atomicAdd(&h.lo[b], w) + w < w) atomicAdd(&h.hi[b], 1u);
      });
    }
    cluster_barrier();
    uint32_t count = 0;
    uint64_t mass = 0;
    // this thread's bin over all CTAs
    auto gather = [&] {
      Hist& h = s.hist;
      count = 0;
      mass = 0;
      for (int p = 0; p < ctas; ++p) {
        count += peer_u32(&h.count[tid], p);
        mass += (uint64_t)peer_u32(&h.hi[tid], p) << 32 | peer_u32(&h.lo[tid], p);
      }
      ++step;
    };
    // the bin where the inclusive count or sum, on top of what comes before the bins, reaches `limit`
    auto find = [&](bool counts, uint64_t limit, uint32_t count, uint64_t mass, uint32_t before_n, uint64_t before_mass) {
      uint32_t n = count;
      uint64_t m = mass;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t yn = __shfl_up_sync(0xffffffffu, n, d);
        const uint64_t ym = __shfl_up_sync(0xffffffffu, m, d);
        if (lane >= d) {
          n += yn;
          m += ym;
        }
      }
      __syncthreads();
      if (lane == 31) {
        s.warp_count[warp] = n;
        s.warp_mass[warp] = m;
      }
      if (tid == 0) s.bin = -1;
      __syncthreads();
      for (int w = 0; w < warp; ++w) {
        n += s.warp_count[w];
        m += s.warp_mass[w];
      }
      n += before_n;
      m += before_mass;
      const uint64_t incl = counts ? n : m, excl = counts ? n - count : m - mass;
      if (count && excl < limit && incl >= limit) {
        s.bin = tid;
        s.bin_n = count;
        s.before_n = n - count;
        s.before_mass = m - mass;
      }
      __syncthreads();
    };
    // the last item kept: the first in the order with which the count or sum reaches `limit`; false: all together do not
    auto resolve = [&](bool counts, uint64_t limit) -> bool {
      find(counts, limit, s.bin_count[tid], s.bin_mass[tid], 0, 0);
      const int b0 = s.bin;
      if (b0 < 0) return false;
      // the range of the order that holds it: at first that of the bin, with something to spare
      uint64_t lo, hi;
      {
        const float margin = 1e-5f * (fabsf(top) + REACH / weigh.c);
        lo = place(top - (b0 - 0.51f) / PER_T / weigh.c + margin, 0u);
        hi = place(top - (b0 + 0.51f) / PER_T / weigh.c - margin, 0xffffffffu);
        if (!(margin < 1e30f)) lo = 0, hi = ~(uint64_t)0;
      }
      auto in_play = [&](float v, int i, uint64_t& at, float& d, float& t) {
        t = weigh.distance(v, d);
        if (!(t < REACH) || bin_of(t) != b0) return false;
        at = place(v, (uint32_t)(x.first + i));
        return at >= lo && at <= hi;
      };
      // (every level takes 9 of 64 bits)
      for (int level = 0; level < 8 && s.bin >= 0 && s.bin_n > LIST; ++level) {
        cluster_barrier();                                    // (the others have read the last histogram)
        Hist& h = s.hist;
        h.count[tid] = h.lo[tid] = h.hi[tid] = 0;
        __syncthreads();
        const int shift = max(0, 64 - __clzll((long long)(hi - lo)) - 9);        // (hi - lo) >> shift < BINS
        x.each(w0, w1, [&](float v, int i) {
          uint64_t at;
          float d, t;
          if (!in_play(v, i, at, d, t)) return;
          const uint32_t w = fixed(weigh.weight<EXACT>(v, d, t));
          const int b = (int)((at - lo) >> shift);
          atomicAdd(&h.count[b], 1u);
          if (atomicAdd(&h.lo[b], w) + w < w) atomicAdd(&h.hi[b], 1u);
        });
        const uint32_t before_n = s.before_n;
        const uint64_t before_mass = s.before_mass;
        cluster_barrier();
        gather();
        find(counts, limit, count, mass, before_n, before_mass);
        lo += (uint64_t)s.bin << shift;
        hi = min(hi, lo + (((uint64_t)1 << shift) - 1));
      }
      // the bin's items, of all CTAs, ranked
      if (tid == 0) s.listed = 0;
      __syncthreads();
      x.each(w0, w1, [&](float v, int i) {
        uint64_t at;
        float d, t;
        if (in_play(v, i, at, d, t)) {
          const uint32_t k = atomicAdd(&s.listed, 1u);
          if (k < LIST) s.list[step & 1][k] = Item{at, fixed(weigh.weight<EXACT>(v, d, t))};
        }
      });
      __syncthreads();
      if (tid == 0) s.say[step & 1].n = s.listed;
      cluster_barrier();
      uint32_t n = 0;
      for (int p = 0; p < ctas; ++p) {
        const uint32_t m = peer_u32(&s.say[step & 1].n, p);
        if (tid < m && n + tid < LIST) {
          s.all[n + tid].at = peer_u64(&s.list[step & 1][tid].at, p);
          s.all[n + tid].w = peer_u32(&s.list[step & 1][tid].w, p);
        }
        n += m;
      }
      n = min(n, (uint32_t)LIST);
      ++step;
      __syncthreads();
      if (tid < n) {
        const Item me = s.all[tid];
        uint32_t k = s.before_n;
        uint64_t m = s.before_mass;
        for (uint32_t j = 0; j < n; ++j) {
          const Item o = s.all[j];
          if (o.at <= me.at) {
            ++k;
            m += o.w;
          }
        }
        const uint64_t incl = counts ? k : m, excl = counts ? k - 1 : m - me.w;
        if (excl < limit && incl >= limit) {
          s.found_at = me.at;
          s.found_mass = m;
        }
      }
      __syncthreads();
      return true;
    };

    gather();
    s.bin_count[tid] = count;
    s.bin_mass[tid] = mass;
    uint64_t all = 0;
    {
      const uint64_t m = warp_sum_u64(mass);
      __syncthreads();
      if (lane == 0) s.warp_mass[warp] = m;
      __syncthreads();
      for (int w = 0; w < WARPS; ++w) all += s.warp_mass[w];
    }
    auto cut = [&] {
      last = value_at(s.found_at);
      last_index = (uint32_t)s.found_at;
    };
    if (by_k && resolve(true, (uint64_t)top_k)) {
      cut();
      all = s.found_mass;
    }
    if (by_p) {
      const double want = top_p > 0.0f ? ceil((double)top_p * (double)all) : 0.0;
      if (resolve(false, want < 1.0 ? (uint64_t)1 : want < (double)all ? (uint64_t)want : all)) cut();
    }
  }

  // ---- the sum of what is kept, by stretches
  auto kept = [&](float v, int i, float& w) -> uint32_t {
    w = 0.0f;
    if (v < last || (v == last && (uint32_t)(x.first + i) > last_index)) return 0u;
    float d;
    const float t = weigh.distance(v, d);
    if (!(t < REACH)) return 0u;
    w = weigh.weight<EXACT>(v, d, t);
    return w < least ? 0u : fixed(w);
  };
  __syncthreads();
  uint64_t mine = 0;
  x.each(w0, w1, [&](float v, int i) {
    float w;
    mine += kept(v, i, w);
  });
  mine = warp_sum_u64(mine);
  if (lane == 0) s.warp_mass[warp] = mine;
  __syncthreads();
  uint64_t before = 0, of_cta = 0;
  for (int w = 0; w < WARPS; ++w) {
    if (w < warp) before += s.warp_mass[w];
    of_cta += s.warp_mass[w];
  }
  if (tid == 0) s.say[step & 1].mass = of_cta;
  cluster_barrier();
  uint64_t total = 0;
  for (int p = 0; p < ctas; ++p) {
    const uint64_t m = peer_u64(&s.say[step & 1].mass, p);
    if (p < rank) before += m;
    total += m;
  }
  cluster_barrier();                                          // (nobody leaves while the others read)

  // ---- the item at which the sum exceeds u * total (greedy rows: the first of the largest)
  uint64_t target = greedy ? 0 : __umul64hi(total, __float2ull_rz(u * 18446744073709551616.0f));
  if (before > target || before + mine <= target) return;
  target -= before;
  uint64_t sum = 0;
  for (int i = w0 + 4 * lane;; i += 128) {                    // (the warp's stretch holds it: the loop ends)
    float v[4], w[4];
    uint32_t q[4];
    uint64_t four = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (STAGED) v[k] = value(x.kept[i + k]);
      else v[k] = x.at(i + k);
      q[k] = kept(v[k], i + k, w[k]);
      four += q[k];
    }
    uint64_t incl = four;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint64_t y = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += y;
    }
    uint64_t at = sum + incl - four;
    const bool here = at <= target && at + four > target;
    if (here) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (at <= target && at + q[k] > target) {
          a.tokens[r] = x.first + i + k;
          if (a.prob) a.prob[r] = greedy ? 1.0f : (float)((double)w[k] / (double)total);
        }
        at += q[k];
      }
    }
    if (__any_sync(0xffffffffu, here)) return;
    sum += __shfl_sync(0xffffffffu, incl, 31);
    if (i - 4 * lane + 128 >= w1) return;
  }
}

template <typename T, bool STAGED>
int launch_one(const SampleArgs& a, int ctas, size_t smem, cudaStream_t st) {
  auto kernel = sample_kernel<T, STAGED>;
  static std::atomic<uint64_t> have{0};
  int rc = allow_smem(kernel, 232448, &have);
  if (rc) return rc;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.rows * ctas));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ctas;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = early_start_enabled(st) ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a);
  return e == cudaSuccess ? check_launch() : note_cuda_error(e);
}

}  // namespace

int launch_sample(SampleArgs a, cudaStream_t st) {
  const int size = a.type == BITNET_KV_F32 ? 4 : 2;
  const int64_t sms = dev_info().sm_count;
  constexpr size_t SHARE = (sizeof(Share) + 15) / 16 * 16;
  auto bytes = [&](int ctas) { return SHARE + (size_t)(ceil_div(ceil_div(a.vocab, ctas), 8) * 8 + 7 + 127) / 128 * 128 * size; };
  // CTAs of a row: as many as its slices need to lie in shared memory, two to an SM; more while SMs are idle
  int ctas = 1;
  while (ctas < MOST_CTAS && (bytes(ctas) > 113 * 1024 || a.rows * ctas * 2 <= sms)) ctas *= 2;
  a.slice = (int)(ceil_div(ceil_div(a.vocab, ctas), 8) * 8);
  const bool staged = bytes(ctas) <= 232448;
  const size_t smem = staged ? bytes(ctas) : SHARE;
  log_launch("sample_kernel rows=%lld vocab=%d ctas=%d staged=%d", (long long)a.rows, a.vocab, ctas, (int)staged);
  switch (a.type) {
    case BITNET_KV_F32: return staged ? launch_one<float, true>(a, ctas, smem, st) : launch_one<float, false>(a, ctas, smem, st);
    case BITNET_KV_BF16: return staged ? launch_one<__nv_bfloat16, true>(a, ctas, smem, st) : launch_one<__nv_bfloat16, false>(a, ctas, smem, st);
    default: return staged ? launch_one<__half, true>(a, ctas, smem, st) : launch_one<__half, false>(a, ctas, smem, st);
  }
}

}  // namespace bitnet
