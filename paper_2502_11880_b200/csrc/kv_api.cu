// C ABI of the paged key-value cache and the attention over it: argument checks and dispatch.
#include <algorithm>
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
std::atomic<int> g_shared_always{0};                // bitnet_debug_attn_shared

// Which kernels take a shared call.  The decode kernel reads a prefix once for every sequence, from L2 all but the first time, but in one launch and, tile by
// tile (64 tokens of a kv head), in some two thirds of the time.  With T tiles read by all sequences, R of them again for another sequence of a group, the
// shared kernels are faster where 3 R - T > 2 X: X = 32 tiles per SM, 16 where every query head has a kv head of its own, for which the decode kernel takes
// longer.  The host knows the numbers of sequences and groups, and bounds the tokens by the table's width or the window.  It can tell where the groups, if
// they are alike, share enough, and where even all sequences in one group would save less than asking costs.  In between (most sequences alone, groups that are
// empty) the device is asked, which knows lengths and prefixes: two more launches, and the kernels that do not take the call end at once, 4 to 7 us.
// Measured, decode / shared (us): 32/8 heads of 128: 8 over 2048: 19/32, 8 over 4096: 29/33, 16 over 4096: 45/33, 64 over 2048: 82/35; 8 groups of 3 over 2048: 40/47,
// 32 of them 125/95; groups of 2 over 16384: 4: 89/104, 8: 167/165, 32: 656/485; 64 over 16384 and 64 alone with up to 600: 774/108, asked 112; 64 alone over 2048:
// 97/155, asked 104; 16/16 heads of 96: 4 over 2048: 22/26, 4 over 4096: 36/30, 8 over 2048: 33/29; 2 groups of 2 over 16384: 120/95, 64 of 2 over 2048: 406/264.
enum class Route { DECODE, SHARED, ASK };
Route route_of(const AttnArgs& a, const bitnet_kv_cache_t* c, int64_t* limit) {
  const int64_t rows = c->kv_heads * ceil_div(a.q_heads / c->kv_heads, 8);
  *limit = 2 * (a.q_heads == c->kv_heads ? 16 : 32) * (int64_t)dev_info().sm_count / rows;
  if (g_shared_always.load(std::memory_order_relaxed)) return Route::SHARED;
  int64_t tokens = a.table_width * c->page_size;
  if (a.window > 0) tokens = std::min(tokens, (int64_t)a.window + a.sinks + 64);
  const double tiles = (double)ceil_div(tokens, 64);
  if (tiles * (double)(2 * a.tokens - 3 * a.groups) > (double)*limit) return Route::SHARED;
  return tiles * (double)(2 * a.tokens - 3) <= 2.0 * (double)*limit ? Route::DECODE : Route::ASK;
}

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
  a->group_start = a->prefix_len = nullptr;
  a->groups = 0;
  a->route = nullptr;
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

int bitnet_kv_append_rope(const bitnet_kv_cache_t* c, int64_t layer, const bitnet_rope_t* rope, const void* q, int64_t q_heads,
                          int64_t q_stride_token, int64_t q_stride_head, const void* k, const void* v, int in_type, int64_t stride_token,
                          int64_t stride_head, int64_t tokens, const int32_t* table, int64_t table_width, const int32_t* kv_len,
                          const int32_t* q_start, int64_t seqs, void* q_out, int out_type, int* dev_status, void* stream) {
  int rc = check_cache(c);
  if (rc) return rc;
  rc = check_tokens(table, table_width, kv_len, q_start, tokens, seqs, dev_status);
  if (rc) return rc;
  if (!rope_ready(rope) || layer < 0 || layer >= c->layers || (in_type != BITNET_KV_F32 && in_type != c->dtype)) return BITNET_ERR_INVALID_ARG;
  if (rope->rot_dim > c->head_dim) return BITNET_ERR_UNSUPPORTED_SHAPE;
  if (q_heads < 0 || q_heads > 65536 || (q_heads && out_type != BITNET_KV_F32 && out_type != c->dtype)) return BITNET_ERR_INVALID_ARG;
  if (tokens == 0) return BITNET_OK;
  const uintptr_t size = in_type == BITNET_KV_F32 ? 4 : 2;
  if (!k || !v || !aligned(k, size) || !aligned(v, size)) return BITNET_ERR_INVALID_ARG;
  if (q_heads && (!q || !aligned(q, size) || !q_out || !aligned16(q_out))) return BITNET_ERR_INVALID_ARG;
  RopeArgs a;
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_out = q_out;
  a.in_type = in_type;
  a.out_type = q_heads ? out_type : c->dtype;
  a.q_heads = q_heads;
  a.q_stride_token = q_heads ? q_stride_token : 0;
  a.q_stride_head = q_heads ? q_stride_head : 0;
  a.stride_token = stride_token;
  a.stride_head = stride_head;
  a.tokens = tokens;
  a.seqs = seqs;
  a.width = table_width;
  a.table = table;
  a.kv_len = kv_len;
  a.q_start = q_start;
  a.dev_status = dev_status;
  return launch_kv_rope(kv_view(c), (int)layer, rope, a, c->dtype, (cudaStream_t)stream);
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

void bitnet_debug_attn_shared(int always) { g_shared_always = always; }

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

size_t bitnet_attn_shared_workspace_bytes(int64_t seqs, int64_t q_heads, int64_t kv_heads, int64_t head_dim) {
  if (seqs < 0 || seqs > COUNT || kv_heads < 1 || q_heads < kv_heads || q_heads > 65536 || q_heads % kv_heads || head_dim < 4 || head_dim > 128)
    return 0;
  return attn_shared_workspace_bytes(seqs, q_heads, (int)head_dim);
}

int bitnet_attn_shared(const bitnet_kv_cache_t* c, int64_t layer, const void* q, int io_dtype, int64_t q_heads, int64_t stride_token,
                       int64_t stride_head, const int32_t* table, int64_t table_width, const int32_t* kv_len, int64_t seqs,
                       const int32_t* group_start, const int32_t* prefix_len, int64_t groups, float scale, int64_t window, int64_t sinks,
                       void* out, void* workspace, size_t workspace_bytes, int* dev_status, void* stream) {
  AttnArgs a;
  const int rc = attn_args(c, layer, q, io_dtype, q_heads, stride_token, stride_head, seqs, table, table_width, kv_len, nullptr, seqs,
                           scale, window, sinks, out, workspace, dev_status, &a);
  if (rc) return rc;
  if (io_dtype != c->dtype || groups < 0 || groups > COUNT) return BITNET_ERR_INVALID_ARG;
  if (seqs == 0) return BITNET_OK;
  if (groups < 1 || !ints(group_start) || !ints(prefix_len)) return BITNET_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < attn_shared_workspace_bytes(seqs, q_heads, c->head_dim)) return BITNET_ERR_WORKSPACE;
  a.group_start = group_start;
  a.prefix_len = prefix_len;
  a.groups = groups;
  int64_t limit;
  const Route route = route_of(a, c, &limit);
  if (route == Route::DECODE) return launch_attn_decode(c, a, workspace, (cudaStream_t)stream);
  return launch_attn_shared(c, a, route == Route::ASK ? limit : -1, workspace, (cudaStream_t)stream);
}

}  // extern "C"
