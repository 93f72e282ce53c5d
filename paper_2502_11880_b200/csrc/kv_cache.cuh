// What the kernels over the paged key-value cache share (internal): the pool's geometry, bounded barrier waits, tensor
// copies of page boxes, exp2.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "common.cuh"
#include "device_utils.cuh"

namespace bitnet {

// Element strides of the K and V pools [layers][pages][kv_heads][page_size][head_dim]; rows of head_dim are contiguous.
struct KvView {
  uint8_t* k;
  uint8_t* v;
  int64_t stride_layer, stride_page, stride_head, stride_row;
  int layers, num_pages, kv_heads, page_size, head_dim;
};

// Rows of one box of a tensor copy: a page, or 64 rows of a larger one.
inline int kv_box_rows(int page_size) { return page_size < 64 ? page_size : 64; }
// Tensor maps of both pools.  maps[0], maps[1]: boxes of 64 columns x kv_box_rows rows, 128-byte swizzle; coordinates
// (column, row, head, page, layer).  maps[2], maps[3], where head_dim is 128 and a layer is a whole number of pages away: boxes of
// both 64-column halves, [half][row][64]; coordinates (column in the half, row, half, head, page + layer * *layer_pages).
int encode_kv_maps(uint64_t (*maps)[16], int64_t* layer_pages, const KvView& v, int dtype);

inline KvView kv_view(const bitnet_kv_cache_t* c) {
  KvView v;
  v.k = static_cast<uint8_t*>(c->k);
  v.v = static_cast<uint8_t*>(c->v);
  v.stride_layer = c->stride_layer;
  v.stride_page = c->stride_page;
  v.stride_head = c->stride_head;
  v.stride_row = c->stride_row;
  v.layers = (int)c->layers;
  v.num_pages = (int)c->num_pages;
  v.kv_heads = c->kv_heads;
  v.page_size = c->page_size;
  v.head_dim = c->head_dim;
  return v;
}

// ---- launchers (one per .cu file)
struct AttnArgs {
  const void* q;            // [tokens][q_heads][head_dim]
  void* out;                // [tokens][q_heads][head_dim], contiguous
  int64_t q_stride_token, q_stride_head;   // elements
  const int32_t* table;     // [seqs][table_width] page ids
  const int32_t* kv_len;    // [seqs]
  const int32_t* q_start;   // [seqs + 1] first token of each sequence; null: token i belongs to sequence i
  int64_t tokens, seqs, table_width;
  int q_heads, layer, window, sinks;
  float scale;
  int io_f32;               // q and out are fp32; otherwise they have the cache's type
  uint32_t give_up;         // the tile before which a CTA gives up (test hook; usually one that never comes)
  int dtype;
  int* dev_status;
};
// The workspace: counters that are zero between calls (of fixed number, so that no call's parts ever lie where another call's
// counters are; the last 16 bytes deal out prompt items), the parts of decode rows, the parts of prompt items (where the caller
// gave the room for them).
size_t attn_decode_parts_bytes();
inline size_t attn_counters_bytes() { return 65536; }
inline int* attn_counters(void* ws) { return static_cast<int*>(ws); }
inline uint8_t* attn_decode_parts(void* ws) { return static_cast<uint8_t*>(ws) + attn_counters_bytes(); }
inline uint8_t* attn_prompt_parts(void* ws) { return attn_decode_parts(ws) + attn_decode_parts_bytes(); }
inline size_t attn_decode_workspace_bytes() { return attn_counters_bytes() + attn_decode_parts_bytes(); }
size_t attn_prompt_parts_bytes(int64_t tokens, int q_heads, int kv_heads);
int launch_attn_decode(const bitnet_kv_cache_t* c, const AttnArgs& a, void* ws, cudaStream_t st);
int launch_attn_prompt(const bitnet_kv_cache_t* c, const AttnArgs& a, void* ws, size_t ws_bytes, cudaStream_t st);

int launch_kv_append(const KvView& kv, int layer, const void* k, const void* v, int in_dtype, int64_t stride_token, int64_t stride_head,
                     int64_t tokens, int64_t seqs, const int32_t* table, int64_t width, const int32_t* kv_len, const int32_t* q_start,
                     int dtype, int* dev_status, cudaStream_t st);
int launch_kv_reserve(int32_t* refs, int64_t num_pages, int32_t* table, int64_t seqs, int64_t width, const int32_t* from_len,
                      const int32_t* to_len, int page_size, int* dev_status, cudaStream_t st);
int launch_kv_fork(const KvView& kv, int32_t* refs, int32_t* table, int64_t seqs, int64_t width, int32_t* len, const int32_t* parents,
                   const int32_t* children, int64_t n, void* ws, int* dev_status, cudaStream_t st);
int launch_kv_release(int32_t* refs, int64_t num_pages, int32_t* table, int64_t seqs, int64_t width, int32_t* len, const int32_t* list,
                      int64_t n, int page_size, int window, int sinks, bool trim, int* dev_status, cudaStream_t st);
int launch_kv_compact(const KvView& kv, int32_t* refs, int32_t* table, int64_t seqs, int64_t width, int32_t* live_out, void* ws,
                      cudaStream_t st);
int launch_kv_copy_pages(const KvView& kv, const int32_t* src, const int32_t* dst, int64_t n, int* dev_status, cudaStream_t st);
size_t kv_workspace_bytes(int64_t num_pages, int64_t n);

// Raises a kernel's limit of dynamic shared memory, once per device (`have`: one bit for each; a device beyond 63 every time).
template <typename K>
int allow_smem(K kernel, int bytes, std::atomic<uint64_t>* have) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return note_cuda_error(cudaGetLastError());
  const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
  if (have->load(std::memory_order_acquire) & bit) return BITNET_OK;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != cudaSuccess) return note_cuda_error(e);
  have->fetch_or(bit, std::memory_order_release);
  return BITNET_OK;
}

#ifdef __CUDACC__
// ---- device side
constexpr uint32_t KV_WAIT_LIMIT = 1u << 22;

__device__ __forceinline__ void kv_mbar_init(uint64_t* bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void kv_mbar_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void kv_mbar_expect(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool kv_mbar_try(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ void kv_give_up(volatile int* abort_flag, int* error) {
  *abort_flag = 1;
  atomicExch(error, BITNET_ERR_TIMEOUT);
}
// Bounded wait.  One that gives up (2^22 tries of 4 us) raises the CTA's abort flag and the device status; the caller goes on (every loop
// of these kernels is counted, so all roles reach their ends), and later waits give up at once.
__device__ __forceinline__ void kv_mbar_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int* error) {
  if (kv_mbar_try(bar, parity)) return;
  for (uint32_t it = 0; it < KV_WAIT_LIMIT; ++it) {
    if (kv_mbar_try(bar, parity)) return;
    if ((it & 255u) == 0u && *abort_flag) return;
  }
  kv_give_up(abort_flag, error);
}
// The same by all lanes of a warp, with one answer: whether the barrier's phase is over.  (Lanes may give up at different times, and
// where full-warp steps follow, or a buffer is filled, all have to go the same way.)
__device__ __forceinline__ bool kv_mbar_wait_warp(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int* error) {
  if (__all_sync(0xffffffffu, kv_mbar_try(bar, parity))) return true;
  kv_mbar_wait(bar, parity, abort_flag, error);
  return __all_sync(0xffffffffu, *abort_flag == 0);
}

// One box of the pool: columns [x, x + 64), rows from `row` of (head, page, layer).  Anything outside the pool reads as 0.
__device__ __forceinline__ void kv_box_copy(uint32_t dst, const CUtensorMap* map, int x, int row, int head, int page, int layer,
                                            uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
      "l"(map), "r"(x), "r"(row), "r"(head), "r"(page), "r"(layer), "r"(smem_u32(bar))
      : "memory");
}

// One box of both halves of rows of 128 columns.
__device__ __forceinline__ void kv_box_copy2(uint32_t dst, const CUtensorMap* map, int row, int head, int page, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
      "l"(map), "r"(0), "r"(row), "r"(0), "r"(head), "r"(page), "r"(smem_u32(bar))
      : "memory");
}

// `bytes` contiguous bytes (a multiple of 16, both addresses too).
__device__ __forceinline__ void kv_bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes),
               "r"(smem_u32(bar))
               : "memory");
}

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Sequence of token n: the number of i in 1..seqs with q_start[i] <= n (sequences without tokens are passed over).
__device__ __forceinline__ int kv_seq_of(const int32_t* q_start, int seqs, int n) {
  int lo = 0, hi = seqs;            // q_start[lo] <= n < q_start[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (__ldg(q_start + mid) <= n) lo = mid;
    else hi = mid;
  }
  return lo;
}
#endif

}  // namespace bitnet
