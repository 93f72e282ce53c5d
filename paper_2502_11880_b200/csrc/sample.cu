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
//   * where the bins up to the one that holds the last kept item have FEW items at most: these, in the first CTA, which ranks them by counting, applies the
//     rules and draws; otherwise
//   * while the bin that holds the last kept item has more than LIST items: another histogram over that bin's range of the order
//     (64 bits: the value's bits, then the index, so that any number of equal values is taken apart too);
//   * the bin's items, ranked by counting: the last item kept, as a place in the order;
//   * the sum of what is kept per warp's stretch of the vocabulary; the warp whose stretch holds the token walks it.
// Sums: weights as 32-bit fixed point of the largest (weights below 2^-33 of it count as 0, are never drawn), added as integers of
// 64 bits: no sum depends on an order, a split or the size of the cluster.  The exponent is computed with the rounding errors of
// the product and, for fp32 logits, of max - x carried along, so that a weight is off by the exponential's own 2^-22 only; of 16-bit logits by what max - x
// loses as well, 2^-24 (max - x) / T, 2^-19.5 for the least weight that counts.  (To carry that too takes 256 x 50021 from 79 to 85 us.)
//
// Bound by barriers for few rows; for many by waits (results of shared atomics, barriers of the cluster) and instructions together: 83 an item at 45 % of the issue
// slots for 64 x 128256, 118 at 61 % for 256 x 50021.  Measured (us, a B200): 1 x 32000, fp32, top-k 50, top-p 0.9: 8.4 (14 without the short list);
// 64 x 128256, fp32, settings per row: 59 (HBM needs 5); 256 x 50021, bf16, top-p 0.92: 79 (HBM needs 4; 75 before there was the short list's code).  Rows that do
// not fit shared memory, read at every pass, temperature alone / with top-p: 1 x 700001, fp32: 50 / 91; 64 x 400000, fp32: 94 / 193; 64 x 700001, bf16: 173 / 423.
#include <cstring>
#include <type_traits>

#include "kv_cache.cuh"

namespace bitnet {
namespace {

constexpr int THREADS = 512, WARPS = THREADS / 32;
constexpr int BINS = THREADS;                // one per thread
constexpr int LIST = 128;                    // items that are ranked by counting
constexpr int FEW = 256;                     // items of a row that are left to one CTA
constexpr int POOL = 1024;                   // items of a bin that are set aside, so that what follows need not look at the whole row
constexpr int MOST_CTAS = 8;                 // of a cluster
constexpr float ONE = 4294967296.0f;         // weight 1

struct Hist {
  uint32_t count[BINS], lo[BINS], hi[BINS];
};
struct Logit {
  float x;
  uint32_t index;
};
struct Sums {
  uint64_t mass[BINS];
  uint32_t count[BINS];
};
// What a division of a bin needs, and what the end of a row with few items needs.
struct Division {
  Sums level;                                // sums over the cluster of a later histogram
  uint64_t item_at[MOST_CTAS][LIST];         // items to be ranked: their places in the order, and weights
  uint32_t item_w[MOST_CTAS][LIST];
  Logit pool[POOL];                          // (this CTA's own)
};
struct End {
  uint64_t at[MOST_CTAS][FEW];
  uint32_t w[MOST_CTAS][FEW];
};
struct Share {
  // written by the others, read after a barrier of the cluster
  float top[MOST_CTAS][WARPS];
  uint64_t part_mass[BINS];                  // of a cluster of C CTAs, BINS / C bins are this CTA's to add up: C parts of each
  uint32_t part_count[BINS];
  Sums row;                                  // sums over the cluster, of the first histogram
  union {
    Division div;
    End few;
  };
  uint32_t items[MOST_CTAS];
  uint64_t cta_mass[MOST_CTAS];
  // this CTA's own
  union {
    Hist hist;
    struct {
      uint64_t few_at[FEW];
      uint32_t few_w[FEW];
    };
  };
  uint64_t warp_mass[WARPS];
  uint32_t warp_count[WARPS];
  uint64_t all_at[LIST];
  uint32_t all_w[LIST];
  uint32_t listed, pooled;
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
__device__ __forceinline__ void tell(const void* p, int rank, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(peer(p, rank)), "r"(v) : "memory");
}
__device__ __forceinline__ void tell(const void* p, int rank, uint64_t v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(peer(p, rank)), "l"(v) : "memory");
}
// A barrier of the cluster in two halves: what was written before `arrive`, the others' memory too, is there after `await`.
__device__ __forceinline__ void arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void await() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
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

// The value of that rank among all, ascending (those that are no numbers lie at both ends).
__device__ __forceinline__ float value_of_rank(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u); }
__device__ __forceinline__ uint32_t rank_of_value(float x) {
  const uint32_t b = __float_as_uint(x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
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
  // The weight in units of 2^-32.  SHORT: max - x as it is rounded (16-bit logits).
  template <bool SHORT>
  __device__ __forceinline__ float weight(float x, float d, float t) const {
    float low = fmaf(d, c, -t);
    low = fmaf(d, c_lo, low);
    if (!SHORT) {
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
__global__ void __launch_bounds__(THREADS, 2) sample_kernel(const __grid_constant__ SampleArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  Share& s = *reinterpret_cast<Share*>(smem_raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  int rank, ctas;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
  const int64_t r = blockIdx.x / ctas;
  arrive();                                                   // (the others may write here: this CTA runs; awaited before the first such write)
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
  bool pending = true;                                        // an arrival that has not been awaited (the same in all CTAs)
  auto settle = [&] {
    if (pending) await();
    pending = false;
  };
  auto meet = [&] {
    settle();
    arrive();
    await();
  };
  settle();
  if (lane < ctas) tell(&s.top[rank][warp], lane, __float_as_uint(top));
  meet();
  top = -INFINITY;
  for (int i = lane; i < ctas * WARPS; i += 32) top = fmaxf(top, (&s.top[0][0])[i]);
#pragma unroll
  for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));

  // a warp's stretch of the slice
  const int stretch = (length / 128 + WARPS - 1) / WARPS * 128;
  const int w0 = min(length, warp * stretch), w1 = min(length, w0 + stretch);
  if (top == -INFINITY) {                                     // nothing can be drawn
    if (rank == 0 && tid == 0) {
      a.tokens[r] = -1;
      if (a.prob) a.prob[r] = 0.0f;
    }
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

  constexpr bool SHORT = sizeof(T) == 2;
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
    // all items by their distance from the largest: counts, and sums of weights where those are asked for
    auto histogram = [&](bool sums) {
      Hist& h = s.hist;
      if (sums) {
        x.each(w0, w1, [&](float v, int) {
          float d;
          const float t = weigh.distance(v, d);
          if (!(t < REACH)) return;
          const uint32_t w = fixed(weigh.weight<SHORT>(v, d, t));
          const int b = bin_of(t);
          atomicAdd(&h.count[b], 1u);
          if (atomicAdd(&h.lo[b], w) + w < w) atomicAdd(&h.hi[b], 1u);
        });
      } else {
        x.each(w0, w1, [&](float v, int) {
          float d;
          const float t = weigh.distance(v, d);
          if (t < REACH) atomicAdd(&h.count[bin_of(t)], 1u);
        });
      }
    };
    // The histogram's bins summed over the cluster, to every CTA's `to`: each CTA adds up its share of the bins, and tells the others.
    auto gather = [&](Sums& to) {
      const int share = BINS / ctas, p = tid / share, of = tid - p * share;
      __syncthreads();
      tell(&s.part_mass[rank * share + of], p, (uint64_t)s.hist.hi[tid] << 32 | s.hist.lo[tid]);
      tell(&s.part_count[rank * share + of], p, s.hist.count[tid]);
      meet();
      // (every bin of the share by as many threads as there are CTAs, each of which tells one)
      const int bin = rank * share + of;
      uint64_t mass = 0;
      uint32_t count = 0;
#pragma unroll
      for (int k = 0; k < MOST_CTAS; ++k)
        if (k < ctas) {
          mass += s.part_mass[k * share + of];
          count += s.part_count[k * share + of];
        }
      tell(&to.mass[bin], p, mass);
      tell(&to.count[bin], p, count);
      meet();
    };
    // the bin where the inclusive count or sum, on top of what comes before the bins, reaches `limit`
    auto find = [&](bool counts, uint64_t limit, const Sums& sums, uint32_t before_n, uint64_t before_mass) {
      const uint32_t count = sums.count[tid];
      const uint64_t mass = sums.mass[tid];
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
    // the last item kept, of the bin that was found: the first in the order with which the count or sum reaches `limit`
    auto resolve = [&](bool counts, uint64_t limit) {
      const int b0 = s.bin;
      // the range of the order that holds it: the bin's, and where that is to be divided its values, [from, to).  The bin falls as the value rises: of all
      // values, by rank, those whose bin lies beyond b are counted digit by digit, 32 at a time.
      uint64_t lo = 0, hi = ~(uint64_t)0;
      if (s.bin_n > LIST) {
        uint32_t beyond[2] = {0, 0};
        const uint32_t of_top = rank_of_value(top);
#pragma unroll 1
        for (int shift = 30; shift >= 0; shift -= 5) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t u = beyond[k] + ((uint32_t)lane << shift) + ((1u << shift) - 1u);     // the last of the lane's block
            float d;
            const float t = weigh.distance(value_of_rank(u), d);
            const bool no = u < of_top && !(t < REACH && bin_of(t) <= b0 - k) && (shift < 30 || lane < 4);
            beyond[k] += (uint32_t)__popc(__ballot_sync(0xffffffffu, no)) << shift;
          }
        }
        lo = place(b0 > 0 ? value_of_rank(beyond[1] - 1) : top, 0u);
        hi = place(value_of_rank(beyond[0]), 0xffffffffu);
      }
      auto in_bin = [&](float v) {
        float d;
        const float t = weigh.distance(v, d);
        return t < REACH && bin_of(t) == b0;
      };
      // the bin's items set aside, where there are not too many
      const bool pool = s.bin_n <= POOL;
      if (pool) {
        if (tid == 0) s.pooled = 0;
        __syncthreads();
        x.each(w0, w1, [&](float v, int i) {
          if (in_bin(v)) {
            const uint32_t k = atomicAdd(&s.pooled, 1u);
            if (k < POOL) s.div.pool[k] = Logit{v, (uint32_t)(x.first + i)};
          }
        });
        __syncthreads();
      }
      // all of the bin's items that lie in the range
      auto in_play = [&](auto f) {
        auto look = [&](float v, uint32_t index) {
          const uint64_t at = place(v, index);
          if (at < lo || at > hi) return;
          float d;
          const float t = weigh.distance(v, d);
          f(at, fixed(weigh.weight<SHORT>(v, d, t)));
        };
        if (pool) {
          for (uint32_t i = tid; i < min(s.pooled, (uint32_t)POOL); i += THREADS) look(s.div.pool[i].x, s.div.pool[i].index);
        } else {
          x.each(w0, w1, [&](float v, int i) {
            if (in_bin(v)) look(v, (uint32_t)(x.first + i));
          });
        }
      };
      // (every level takes 9 of 64 bits)
      for (int level = 0; level < 8 && s.bin >= 0 && s.bin_n > LIST; ++level) {
        Hist& h = s.hist;
        h.count[tid] = h.lo[tid] = h.hi[tid] = 0;
        __syncthreads();
        const int shift = max(0, 64 - __clzll((long long)(hi - lo)) - 9);        // (hi - lo) >> shift < BINS
        in_play([&](uint64_t at, uint32_t w) {
          const int b = (int)((at - lo) >> shift);
          atomicAdd(&h.count[b], 1u);
          if (atomicAdd(&h.lo[b], w) + w < w) atomicAdd(&h.hi[b], 1u);
        });
        const uint32_t before_n = s.before_n;
        const uint64_t before_mass = s.before_mass;
        gather(s.div.level);
        find(counts, limit, s.div.level, before_n, before_mass);
        lo += (uint64_t)s.bin << shift;
        hi = min(hi, lo + (((uint64_t)1 << shift) - 1));
      }
      // the bin's items, of all CTAs, ranked
      if (tid == 0) s.listed = 0;
      __syncthreads();
      settle();                                               // (the others are done with the items before these)
      in_play([&](uint64_t at, uint32_t w) {
        const uint32_t k = atomicAdd(&s.listed, 1u);
        if (k >= LIST) return;
        for (int p = 0; p < ctas; ++p) {
          tell(&s.div.item_at[rank][k], p, at);
          tell(&s.div.item_w[rank][k], p, w);
        }
      });
      __syncthreads();
      if (tid < ctas) tell(&s.items[rank], tid, min(s.listed, (uint32_t)LIST));
      meet();
      uint32_t n = 0;
      for (int p = 0; p < ctas; ++p) {
        const uint32_t m = s.items[p];
        if (tid < m && n + tid < LIST) {
          s.all_at[n + tid] = s.div.item_at[p][tid];
          s.all_w[n + tid] = s.div.item_w[p][tid];
        }
        n += m;
      }
      n = min(n, (uint32_t)LIST);
      __syncthreads();
      arrive();                                               // (awaited ahead of the next items, or the next barrier)
      pending = true;
      // (four threads to an item)
      static_assert(4 * LIST <= THREADS, "");
      {
        const uint32_t i = tid >> 2;
        const uint64_t me = i < n ? s.all_at[i] : 0;
        uint32_t k = 0;
        uint64_t m = 0;
        for (uint32_t j = tid & 3; j < n; j += 4)
          if (s.all_at[j] <= me) {
            ++k;
            m += s.all_w[j];
          }
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
          k += __shfl_xor_sync(0xffffffffu, k, o);
          m += __shfl_xor_sync(0xffffffffu, m, o);
        }
        k += s.before_n;
        m += s.before_mass;
        if (i < n && (tid & 3) == 0) {
          const uint64_t incl = counts ? k : m, excl = counts ? k - 1 : m - s.all_w[i];
          if (excl < limit && incl >= limit) {
            s.found_at = me;
            s.found_mass = m;
          }
        }
      }
      __syncthreads();
    };
    // what top_p of `all` asks for
    auto share_of = [&](uint64_t all) -> uint64_t {
      const double want = top_p > 0.0f ? ceil((double)top_p * (double)all) : 0.0;
      return want < 1.0 ? (uint64_t)1 : want < (double)all ? (uint64_t)want : all;
    };
    // The bin that was found and those before it have FEW items at most: all that may be kept.  They are brought to the cluster's first CTA, which ranks
    // them, applies the rules (the first one if `count_here`) and draws.
    auto few = [&] { return s.bin >= 0 && s.before_n + s.bin_n <= FEW; };
    auto draw_of_few = [&](bool count_here, uint64_t all) {
      const int b0 = s.bin;
      if (tid == 0) s.listed = 0;
      __syncthreads();
      settle();
      x.each(w0, w1, [&](float v, int i) {
        float d;
        const float t = weigh.distance(v, d);
        if (!(t < REACH) || bin_of(t) > b0) return;
        const uint32_t k = atomicAdd(&s.listed, 1u);
        if (k >= FEW) return;
        tell(&s.few.at[rank][k], 0, place(v, (uint32_t)(x.first + i)));
        tell(&s.few.w[rank][k], 0, fixed(weigh.weight<SHORT>(v, d, t)));
      });
      __syncthreads();
      if (tid == 0) tell(&s.items[rank], 0, min(s.listed, (uint32_t)FEW));
      meet();                                                 // (the last one)
      if (rank != 0) return;
      uint32_t n = 0;
      for (int p = 0; p < ctas; ++p) {
        const uint32_t m = s.items[p];
        if (tid < m && n + tid < FEW) {
          s.few_at[n + tid] = s.few.at[p][tid];
          s.few_w[n + tid] = s.few.w[p][tid];
        }
        n += m;
      }
      n = min(n, (uint32_t)FEW);
      __syncthreads();
      // an item's rank, from 1, and the sum up to it; as many threads to an item as there are, up to 32
      static_assert(THREADS == 512 && FEW <= THREADS, "");
      const int log2_per = min(5, __clz((int)max(n, 1u) - 1) - 23), per = 1 << log2_per;
      const uint32_t i = tid >> log2_per, part = tid & (per - 1);
      const uint64_t me = i < n ? s.few_at[i] : 0;
      const uint32_t w = i < n ? s.few_w[i] : 0u;
      uint32_t k = 0;
      uint64_t m = 0;
      for (uint32_t j = part; j < n; j += per)
        if (s.few_at[j] <= me) {
          ++k;
          m += s.few_w[j];
        }
      for (int o = 1; o < per; o <<= 1) {
        k += __shfl_xor_sync(0xffffffffu, k, o);
        m += __shfl_xor_sync(0xffffffffu, m, o);
      }
      if (count_here) {
        if (i < n && (int)k == top_k) s.found_mass = m;
        __syncthreads();
        all = s.found_mass;
      }
      float d;
      const float v = value_at(me), t = weigh.distance(v, d), exact_w = i < n ? weigh.weight<SHORT>(v, d, t) : 0.0f;
      const bool keep = i < n && (!count_here || (int)k <= top_k) && (!by_p || m - w < share_of(all)) && !(exact_w < least);
      __syncthreads();
      if (i < n && part == 0) s.few_w[i] = keep ? w : 0u;
      __syncthreads();
      // those ahead of it in the vocabulary
      uint64_t total = 0, before = 0;
      for (uint32_t j = part; j < n; j += per) {
        const uint32_t of_j = s.few_w[j];
        total += of_j;
        if ((uint32_t)s.few_at[j] < (uint32_t)me) before += of_j;
      }
      for (int o = 1; o < per; o <<= 1) {
        total += __shfl_xor_sync(0xffffffffu, total, o);
        before += __shfl_xor_sync(0xffffffffu, before, o);
      }
      const uint64_t target = __umul64hi(total, __float2ull_rz(u * 18446744073709551616.0f));
      if (keep && part == 0 && before <= target && before + w > target) {
        a.tokens[r] = (int)(uint32_t)me;
        if (a.prob) a.prob[r] = (float)((double)exact_w / (double)total);
      }
    };

    // (no sums where top_k says that few are kept; seldom wrong: many equal values)
    bool short_k = false;
#pragma unroll 1
    for (bool sums = !(by_k && top_k <= FEW - FEW / 8);; sums = true) {
      histogram(sums);
      gather(s.row);
      if (by_k) find(true, (uint64_t)top_k, s.row, 0, 0);
      short_k = by_k && few();
      if (sums || short_k) break;
      s.hist.count[tid] = 0;
      __syncthreads();
    }
    uint64_t all = 0;
    if (!short_k) {
      const uint64_t m = warp_sum_u64(s.row.mass[tid]);
      __syncthreads();
      if (lane == 0) s.warp_mass[warp] = m;
      __syncthreads();
      for (int w = 0; w < WARPS; ++w) all += s.warp_mass[w];
    }
    auto cut = [&] {
      last = value_at(s.found_at);
      last_index = (uint32_t)s.found_at;
    };
    if (by_k && !short_k && s.bin >= 0) {
      resolve(true, (uint64_t)top_k);
      cut();
      all = s.found_mass;
    }
    bool short_p = false;
    if (by_p && !short_k) {
      const uint64_t limit = share_of(all);
      find(false, limit, s.row, 0, 0);
      short_p = few();
      if (!short_p && s.bin >= 0) {
        resolve(false, limit);
        cut();
      }
    }
    if (short_k || short_p) {
      draw_of_few(short_k, all);
      return;
    }
  }

  // ---- the sum of what is kept, by stretches
  auto kept = [&](float v, int i, float& w) -> uint32_t {
    w = 0.0f;
    if (v < last || (v == last && (uint32_t)(x.first + i) > last_index)) return 0u;
    float d;
    const float t = weigh.distance(v, d);
    if (!(t < REACH)) return 0u;
    w = weigh.weight<SHORT>(v, d, t);
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
  settle();
  if (tid < ctas) tell(&s.cta_mass[rank], tid, of_cta);
  meet();                                                     // (the last one: nothing of another CTA is written or read after it)
  uint64_t total = 0;
  for (int p = 0; p < ctas; ++p) {
    const uint64_t m = s.cta_mass[p];
    if (p < rank) before += m;
    total += m;
  }

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
