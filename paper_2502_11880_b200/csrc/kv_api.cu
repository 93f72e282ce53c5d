// C ABI of the paged key-value cache and the attention over it: argument checks and dispatch.
#include <cmath>

#include "kv_cache.cuh"

using namespace bitnet;

namespace {

constexpr uint64_t READY = 0x6b76636163686531ull;   // set by bitnet_kv_cache_init
constexpr int64_t MOST = 0x7fffffff;
constexpr int64_t COUNT = MOST - 8192;              // most pages, rows, tokens, entries of a list: kernels step up to 8191 beyond the last in int

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool ints(const void* p) { return p && aligned(p, 4); }
bool ints_or_null(const void* p) { return aligned(p, 4); }
bool page_size_ok(int64_t n) { return n >= 8 && n <= (1 << 20) && (n & (n - 1)) == 0; }
int64_t clamp_int(int64_t x) { return x < MOST ? x : MOST; }
std::atomic<uint32_t> g_give_up{0xffffffffu};       // bitnet_debug_attn_give_up

// The books: table[seqs][width] and refs[num_pages].
int check_books(const int32_t* refs, int64_t num_pages, const int32_t* table, int64_t seqs, int64_t width) {
  if (!ints(refs) || num_pages < 1 || num_pages > COUNT || seqs < 0 || seqs > COUNT || width < 1 || width > MOST) return BITNET_ERR_INVALID_ARG;
  return seqs == 0 || ints(table) ? BITNET_OK : BITNET_ERR_INVALID_ARG;
}
int check_cache(const bitnet_kv_cache_t* c) {
  if (!c || c->ready != READY) return BITNET_ERR_INVALID_ARG;
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return note_cuda_error(e);
  return dev == c->device ? BITNET_OK : BITNET_ERR_INVALID_ARG;
}
int check_tokens(const int32_t* table, int64_t width, const int32_t* kv_len, const int32_t* q_start, int64_t tokens, int64_t seqs,
                 const int* dev_status) {
  if (seqs < 0 || seqs > COUNT || tokens < 0 || tokens > COUNT || !ints_or_null(q_start) || !ints_or_null(dev_status))
    return BITNET_ERR_INVALID_ARG;
  if (!q_start && tokens != seqs) return BITNET_ERR_INVALID_ARG;
  if (tokens == 0) return BITNET_OK;      // nothing to do, whatever else there is
  if (!ints(table) || !ints(kv_len) || width < 1 || width > MOST || seqs < 1) return BITNET_ERR_INVALID_ARG;
  return BITNET_OK;
}

int attn_args(const bitnet_kv_cache_t* c, int64_t layer, const void* q, int io_dtype, int64_t q_heads, int64_t stride_token,
              int64_t stride_head, int64_t tokens, const int32_t* table, int64_t width, const int32_t* kv_len, const int32_t* q_start,
              int64_t seqs, float scale, int64_t window, int64_t sinks, void* out, void* ws, int* dev_status, AttnArgs* a) {
  int rc = check_cache(c);
  if (rc) return rc;
  rc = check_tokens(table, width, kv_len, q_start, tokens, seqs, dev_status);
  if (rc) return rc;
  if (layer < 0 || layer >= c->layers || window < 0 || sinks < 0 || !std::isfinite(scale)) return BITNET_ERR_INVALID_ARG;
  if (q_heads < 1 || q_heads > 65536) return BITNET_ERR_INVALID_ARG;
  if (q_heads % c->kv_heads) return BITNET_ERR_UNSUPPORTED_SHAPE;
  if (tokens && (!q || !out || !aligned16(q) || !aligned16(out) || (ws && !aligned16(ws)))) return BITNET_ERR_INVALID_ARG;
  if (stride_token % 4 || stride_head % 4) return BITNET_ERR_INVALID_ARG;
  a->q = q;
  a->out = out;
  a->q_stride_token = stride_token;
  a->q_stride_head = stride_head;
  a->table = table;
  a->kv_len = kv_len;
  a->q_start = q_start;
  a->tokens = tokens;
  a->seqs = seqs;
  a->table_width = width;
  a->q_heads = (int)q_heads;
  a->layer = (int)layer;
  a->window = (int)clamp_int(window);
  a->sinks = (int)clamp_int(sinks);
  a->scale = scale;
  a->io_f32 = io_dtype == BITNET_KV_F32;
  a->dtype = c->dtype;
  a->dev_status = dev_status;
  a->give_up = g_give_up.load(std::memory_order_relaxed);
  return BITNET_OK;
}

}  // namespace

extern "C" {

int bitnet_kv_cache_init(bitnet_kv_cache_t* c) {
  if (!c) return BITNET_ERR_INVALID_ARG;
  c->ready = 0;
  if (c->dtype != BITNET_KV_BF16 && c->dtype != BITNET_KV_F16) return BITNET_ERR_INVALID_ARG;
  if (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return BITNET_ERR_INVALID_ARG;
  if (c->kv_heads < 1 || c->layers < 1 || c->num_pages < 1 || c->layers > MOST || c->num_pages > COUNT) return BITNET_ERR_INVALID_ARG;
  if (!page_size_ok(c->page_size) || c->head_dim < 4 || c->head_dim > 128 || c->head_dim % 4) return BITNET_ERR_UNSUPPORTED_SHAPE;
  // 16-byte pieces of a page (at most 16 in a row) are counted in int, by blocks that look 1024 of them ahead
  if ((int64_t)c->kv_heads * c->page_size * 16 > MOST - 1023) return BITNET_ERR_UNSUPPORTED_SHAPE;
  const int64_t strides[4] = {c->stride_layer, c->stride_page, c->stride_head, c->stride_row};
  for (int64_t s : strides)
    if (s < 0 || s % 8 || s >= (int64_t)1 << 38) return BITNET_ERR_INVALID_ARG;
  if (c->stride_row < c->head_dim) return BITNET_ERR_INVALID_ARG;
  cudaPointerAttributes k_at, v_at;
  cudaError_t e = cudaPointerGetAttributes(&k_at, c->k);
  if (e == cudaSuccess) e = cudaPointerGetAttributes(&v_at, c->v);
  if (e != cudaSuccess) return note_cuda_error(cudaGetLastError());
  if ((k_at.type != cudaMemoryTypeDevice && k_at.type != cudaMemoryTypeManaged) || k_at.type != v_at.type || k_at.device != v_at.device)
    return BITNET_ERR_INVALID_ARG;
  c->device = k_at.device;
  const int rc = encode_kv_maps(c->maps, &c->layer_pages, kv_view(c), c->dtype);
  if (rc == BITNET_OK) c->ready = READY;
  return rc;
}

int bitnet_kv_append(const bitnet_kv_cache_t* c, int64_t layer, const void* k, const void* v, int in_dtype, int64_t stride_token,
                     int64_t stride_head, int64_t tokens, const int32_t* table, int64_t table_width, const int32_t* kv_len,
                     const int32_t* q_start, int64_t seqs, int* dev_status, void* stream) {
  int rc = check_cache(c);
  if (rc) return rc;
  rc = check_tokens(table, table_width, kv_len, q_start, tokens, seqs, dev_status);
  if (rc) return rc;
  if (layer < 0 || layer >= c->layers || (in_dtype != BITNET_KV_F32 && in_dtype != c->dtype)) return BITNET_ERR_INVALID_ARG;
  if (stride_token % 4 || stride_head % 4) return BITNET_ERR_INVALID_ARG;
  if (tokens == 0) return BITNET_OK;
  const uintptr_t al = in_dtype == BITNET_KV_F32 ? 16 : 8;
  if (!k || !v || !aligned(k, al) || !aligned(v, al)) return BITNET_ERR_INVALID_ARG;
  return launch_kv_append(kv_view(c), (int)layer, k, v, in_dtype, stride_token, stride_head, tokens, seqs, table, table_width, kv_len,
                          q_start, c->dtype, dev_status, (cudaStream_t)stream);
}

int bitnet_kv_reserve(int32_t* refs, int64_t num_pages, int32_t* table, int64_t seqs, int64_t table_width, const int32_t* from_len,
                      const int32_t* to_len, int64_t page_size, int* dev_status, void* stream) {
  const int rc = check_books(refs, num_pages, table, seqs, table_width);
  if (rc) return rc;
  if (!page_size_ok(page_size)) return BITNET_ERR_UNSUPPORTED_SHAPE;
  if (seqs == 0) return BITNET_OK;
  if (!ints(from_len) || !ints(to_len) || !ints_or_null(dev_status)) return BITNET_ERR_INVALID_ARG;
  return launch_kv_reserve(refs, num_pages, table, seqs, table_width, from_len, to_len, (int)page_size, dev_status, (cudaStream_t)stream);
}

size_t bitnet_kv_workspace_bytes(int64_t num_pages, int64_t n) {
  if (num_pages < 1 || num_pages > COUNT || n < 0 || n > COUNT) return 0;
  return kv_workspace_bytes(num_pages, n);
}

int bitnet_kv_fork(const bitnet_kv_cache_t* c, int32_t* refs, int32_t* table, int64_t seqs, int64_t table_width, int32_t* kv_len,
                   const int32_t* parents, const int32_t* children, int64_t n, void* workspace, size_t workspace_bytes, int* dev_status,
                   void* stream) {
  int rc = check_cache(c);
  if (rc) return rc;
  rc = check_books(refs, c->num_pages, table, seqs, table_width);
  if (rc) return rc;
  if (n < 0 || n > COUNT) return BITNET_ERR_INVALID_ARG;
  if (n == 0) return BITNET_OK;
  if (seqs < 1 || !ints(kv_len) || !ints(parents) || !ints(children) || !ints_or_null(dev_status)) return BITNET_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < kv_workspace_bytes(1, n)) return BITNET_ERR_WORKSPACE;
  if (!aligned16(workspace)) return BITNET_ERR_INVALID_ARG;
  return launch_kv_fork(kv_view(c), refs, table, seqs, table_width, kv_len, parents, children, n, workspace, dev_status,
                        (cudaStream_t)stream);
}

int bitnet_kv_free(int32_t* refs, int64_t num_pages, int32_t* table, int64_t seqs, int64_t table_width, int32_t* kv_len,
                   const int32_t* list, int64_t n, int* dev_status, void* stream) {
  const int rc = check_books(refs, num_pages, table, seqs, table_width);
  if (rc) return rc;
  if (n < 0 || n > COUNT) return BITNET_ERR_INVALID_ARG;
  if (n == 0) return BITNET_OK;
  if (seqs < 1 || !ints(kv_len) || !ints(list) || !ints_or_null(dev_status)) return BITNET_ERR_INVALID_ARG;
  return launch_kv_release(refs, num_pages, table, seqs, table_width, kv_len, list, n, 8, 0, 0, false, dev_status, (cudaStream_t)stream);
}

int bitnet_kv_trim(int32_t* refs, int64_t num_pages, int32_t* table, int64_t seqs, int64_t table_width, const int32_t* kv_len,
                   int64_t page_size, int64_t window, int64_t sinks, void* stream) {
  const int rc = check_books(refs, num_pages, table, seqs, table_width);
  if (rc) return rc;
  if (window < 1 || sinks < 0) return BITNET_ERR_INVALID_ARG;
  if (!page_size_ok(page_size)) return BITNET_ERR_UNSUPPORTED_SHAPE;
  if (seqs == 0) return BITNET_OK;
  if (!ints(kv_len)) return BITNET_ERR_INVALID_ARG;
  return launch_kv_release(refs, num_pages, table, seqs, table_width, const_cast<int32_t*>(kv_len), nullptr, seqs, (int)page_size,
                           (int)clamp_int(window), (int)clamp_int(sinks), true, nullptr, (cudaStream_t)stream);
}

int bitnet_kv_compact(const bitnet_kv_cache_t* c, int32_t* refs, int32_t* table, int64_t seqs, int64_t table_width, int32_t* live_out,
                      void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_cache(c);
  if (rc) return rc;
  rc = check_books(refs, c->num_pages, table, seqs, table_width);
  if (rc) return rc;
  if (!ints_or_null(live_out)) return BITNET_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < kv_workspace_bytes(c->num_pages, 0)) return BITNET_ERR_WORKSPACE;
  if (!aligned16(workspace)) return BITNET_ERR_INVALID_ARG;
  return launch_kv_compact(kv_view(c), refs, table, seqs, table_width, live_out, workspace, (cudaStream_t)stream);
}

int bitnet_kv_copy_pages(const bitnet_kv_cache_t* c, const int32_t* src, const int32_t* dst, int64_t n, int* dev_status, void* stream) {
  const int rc = check_cache(c);
  if (rc) return rc;
  if (n < 0 || n > COUNT || !ints_or_null(dev_status)) return BITNET_ERR_INVALID_ARG;
  if (n == 0) return BITNET_OK;
  if (!ints(src) || !ints(dst)) return BITNET_ERR_INVALID_ARG;
  return launch_kv_copy_pages(kv_view(c), src, dst, n, dev_status, (cudaStream_t)stream);
}

size_t bitnet_attn_workspace_bytes(int64_t tokens, int64_t q_heads, int64_t kv_heads, int64_t head_dim) {
  if (tokens < 0 || tokens > COUNT || kv_heads < 1 || q_heads < kv_heads || q_heads > 65536 || q_heads % kv_heads || head_dim < 4 ||
      head_dim > 128)
    return 0;
  return attn_decode_workspace_bytes() + attn_prompt_parts_bytes(tokens, (int)q_heads, (int)kv_heads);
}

void bitnet_debug_attn_give_up(int64_t tile) { g_give_up = tile < 0 || tile >= 0xffffffffll ? 0xffffffffu : (uint32_t)tile; }

int bitnet_attn_decode(const bitnet_kv_cache_t* c, int64_t layer, const void* q, int io_dtype, int64_t q_heads, int64_t stride_token,
                       int64_t stride_head, const int32_t* table, int64_t table_width, const int32_t* kv_len, int64_t seqs, float scale,
                       int64_t window, int64_t sinks, void* out, void* workspace, size_t workspace_bytes, int* dev_status, void* stream) {
  AttnArgs a;
  const int rc = attn_args(c, layer, q, io_dtype, q_heads, stride_token, stride_head, seqs, table, table_width, kv_len, nullptr, seqs,
                           scale, window, sinks, out, workspace, dev_status, &a);
  if (rc) return rc;
  if (io_dtype != BITNET_KV_F32 && io_dtype != c->dtype) return BITNET_ERR_INVALID_ARG;
  if (seqs == 0) return BITNET_OK;
  if (!workspace || workspace_bytes < attn_decode_workspace_bytes()) return BITNET_ERR_WORKSPACE;
  return launch_attn_decode(c, a, workspace, (cudaStream_t)stream);
}

int bitnet_attn_prompt(const bitnet_kv_cache_t* c, int64_t layer, const void* q, int io_dtype, int64_t q_heads, int64_t stride_token,
                       int64_t stride_head, int64_t tokens, const int32_t* table, int64_t table_width, const int32_t* kv_len,
                       const int32_t* q_start, int64_t seqs, int64_t max_new, float scale, int64_t window, int64_t sinks, void* out,
                       void* workspace, size_t workspace_bytes, int* dev_status, void* stream) {
  AttnArgs a;
  const int rc = attn_args(c, layer, q, io_dtype, q_heads, stride_token, stride_head, tokens, table, table_width, kv_len, q_start, seqs,
                           scale, window, sinks, out, workspace, dev_status, &a);
  if (rc) return rc;
  if (!q_start || io_dtype != c->dtype || max_new < 0 || max_new > tokens) return BITNET_ERR_INVALID_ARG;
  if (tokens == 0) return BITNET_OK;
  if (max_new < 1) return BITNET_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < attn_decode_workspace_bytes()) return BITNET_ERR_WORKSPACE;
  // One or two tokens of each sequence: the decode kernel, which takes every token by itself and splits what it reads over all SMs.
  // Measured, decode / prompt kernel (us), 1, 2, 4 tokens over 32768, 32/8 heads of 128: 33/68, 38/64, 69/64; 32 sequences over 4096:
  // 70/149, 73/149, 143/150; 16/16 heads of 96, one sequence over 4096, 1 and 4 tokens: 16/29, 36/28.
  if (max_new <= 2) return launch_attn_decode(c, a, workspace, (cudaStream_t)stream);
  return launch_attn_prompt(c, a, workspace, workspace_bytes, (cudaStream_t)stream);
}

}  // extern "C"
