// C ABI of the norm, the rotation's description and the drawing of tokens: argument checks and dispatch.
#include <cmath>
#include <limits>

#include "common.cuh"

using namespace bitnet;

namespace {

constexpr uint64_t READY = 0x726f706564657331ull;      // set by bitnet_rope_init
constexpr int64_t MOST = 0x7fffffff;

bool type_ok(int t) { return t == BITNET_KV_BF16 || t == BITNET_KV_F16 || t == BITNET_KV_F32; }
bool of_type(const void* p, int t) { return reinterpret_cast<uintptr_t>(p) % (t == BITNET_KV_F32 ? 4 : 2) == 0; }
bool words(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

}  // namespace

namespace bitnet {
bool rope_ready(const bitnet_rope_t* r) { return r && r->ready == READY; }
}  // namespace bitnet

extern "C" {

int bitnet_add_rmsnorm_quant(const void* x, int x_type, int64_t stride_x, const void* residual, int residual_type, int64_t stride_residual,
                             void* residual_out, int64_t stride_residual_out, const void* weight, int weight_type, float eps, int64_t T,
                             int64_t K, void* y, int y_type, int8_t* q, float* act_scale, int32_t* act_sum, void* stream) {
  if (T < 0 || T > MOST || K < 1 || K > MOST || !(eps >= 0.0f) || std::isinf(eps)) return BITNET_ERR_INVALID_ARG;
  if (!type_ok(x_type) || (residual && !type_ok(residual_type)) || (weight && !type_ok(weight_type)) || (y && !type_ok(y_type)))
    return BITNET_ERR_INVALID_ARG;
  if ((residual != nullptr) != (residual_out != nullptr)) return BITNET_ERR_INVALID_ARG;
  if (T == 0) return BITNET_OK;
  if (!x || !q || !act_scale || !of_type(x, x_type) || !words(act_scale) || !words(act_sum)) return BITNET_ERR_INVALID_ARG;
  if (!aligned16(q) || (y && !aligned16(y))) return BITNET_ERR_INVALID_ARG;
  if (residual && (!of_type(residual, residual_type) || !of_type(residual_out, residual_type))) return BITNET_ERR_INVALID_ARG;
  if (weight && !of_type(weight, weight_type)) return BITNET_ERR_INVALID_ARG;
  // rows that lie on one another would be written by several CTAs, and x in another type be read after it was overwritten
  if (residual && T > 1 && (stride_residual_out < 0 ? -stride_residual_out : stride_residual_out) < K) return BITNET_ERR_INVALID_ARG;
  if (residual && residual_out == x && residual_type != x_type) return BITNET_ERR_INVALID_ARG;
  // (in place, each row in its own place)
  if (residual && T > 1 && ((residual_out == x && stride_residual_out != stride_x) || (residual_out == residual && stride_residual_out != stride_residual)))
    return BITNET_ERR_INVALID_ARG;
  NormArgs a;
  a.x = x;
  a.residual = residual;
  a.weight = weight;
  a.residual_out = residual_out;
  a.y = y;
  a.q = q;
  a.act_scale = act_scale;
  a.act_sum = act_sum;
  a.stride_x = stride_x;
  a.stride_residual = stride_residual;
  a.stride_residual_out = stride_residual_out;
  a.T = T;
  a.K = K;
  a.eps = eps;
  a.x_type = x_type;
  a.residual_type = residual_type;
  a.weight_type = weight_type;
  a.y_type = y_type;
  return launch_add_rmsnorm(a, (cudaStream_t)stream);
}

int bitnet_rope_init(bitnet_rope_t* r) {
  if (!r) return BITNET_ERR_INVALID_ARG;
  r->ready = 0;
  if (r->rot_dim < 2 || r->rot_dim > 128 || r->rot_dim % 2) return BITNET_ERR_UNSUPPORTED_SHAPE;
  if (r->scaling != BITNET_ROPE_NONE && r->scaling != BITNET_ROPE_LINEAR && r->scaling != BITNET_ROPE_BANDS) return BITNET_ERR_INVALID_ARG;
  if (!std::isfinite(r->magnitude)) return BITNET_ERR_INVALID_ARG;
  if (!r->freqs) {
    if (!(r->base > 0.0) || !std::isfinite(r->base)) return BITNET_ERR_INVALID_ARG;
    if (r->scaling != BITNET_ROPE_NONE && (!(r->factor > 0.0) || !std::isfinite(r->factor))) return BITNET_ERR_INVALID_ARG;
    if (r->scaling == BITNET_ROPE_BANDS && !(r->high > r->low && r->context > 0.0 && std::isfinite(r->high) && std::isfinite(r->low) && std::isfinite(r->context)))
      return BITNET_ERR_INVALID_ARG;
  }
  // In 64 bits of mantissa: a step is right to one unit of 2^-64 of a turn.  (53 bits were off by 2^-24 of a turn at positions near 2^31.)
  using Wide = long double;
  static_assert(std::numeric_limits<Wide>::digits >= 64, "");
  constexpr Wide TAU = 6.283185307179586476925286766559005768L;
  for (int i = 0; i < 64; ++i) {
    r->step[i] = 0;
    if (i >= r->rot_dim / 2) continue;
    Wide f;
    if (r->freqs) {
      f = r->freqs[i];
    } else {
      f = std::pow((Wide)r->base, (Wide)(-2 * i) / r->rot_dim);
      if (r->scaling == BITNET_ROPE_LINEAR) f /= r->factor;
      if (r->scaling == BITNET_ROPE_BANDS) {
        Wide s = (f * r->context / TAU - r->low) / ((Wide)r->high - r->low);
        s = s < 0 ? 0 : s > 1 ? 1 : s;
        f = (1 - s) * f / r->factor + s * f;
      }
    }
    if (!std::isfinite((double)f)) return BITNET_ERR_INVALID_ARG;
    Wide turns = f / TAU;
    turns -= std::floor(turns);                            // [0, 1]; backwards is forwards by the rest of a turn
    turns = std::round(std::ldexp(turns, 64));
    r->step[i] = turns >= std::ldexp((Wide)1, 64) ? 0 : (uint64_t)turns;
  }
  if (r->magnitude == 0.0) r->magnitude = 1.0;
  r->ready = READY;
  return BITNET_OK;
}

int bitnet_sample(const void* logits, int type, int64_t stride, int64_t rows, int64_t vocab, const float* u, const float* temperature,
                  const int32_t* top_k, const float* top_p, const float* min_p, int32_t* tokens, float* prob, void* stream) {
  if (!type_ok(type) || rows < 0 || rows > MOST / 8 || vocab < 1 || vocab > (1 << 30)) return BITNET_ERR_INVALID_ARG;
  if (rows == 0) return BITNET_OK;
  if (!logits || !of_type(logits, type) || !u || !tokens) return BITNET_ERR_INVALID_ARG;
  for (const void* p : {(const void*)u, (const void*)temperature, (const void*)top_k, (const void*)top_p, (const void*)min_p,
                        (const void*)tokens, (const void*)prob})
    if (!words(p)) return BITNET_ERR_INVALID_ARG;
  SampleArgs a;
  a.logits = logits;
  a.type = type;
  a.stride = stride;
  a.rows = rows;
  a.vocab = (int)vocab;
  a.u = u;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.tokens = tokens;
  a.prob = prob;
  return launch_sample(a, (cudaStream_t)stream);
}

}  // extern "C"
