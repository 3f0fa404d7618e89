// rotary_api.hip -- the C ABI of rotary positions: argument checks, the frequencies of an angle, the launch.
#include <math.h>

#include "tilemix.h"
#include "tilemix_internal.h"

namespace {

using tilemix::api::fail;
using tilemix::api::ok;

bool aligned(const void* ptr, size_t a) { return ((uintptr_t)ptr % a) == 0; }

constexpr long long kStrideMax = 1LL << 40;
constexpr int32_t kRowsMax = 1 << 28;
constexpr double kPi = 3.14159265358979323846;

}  // namespace

extern "C" {

tilemix_status tilemix_rotary_frequencies(const tilemix_rotary_scaling* s, double* inv_freq, float* magnitude) {
  if (!s || !inv_freq || !magnitude) return fail(TILEMIX_ERR_NULL, "scaling, inv_freq and magnitude must be non-NULL");
  const int r = s->rotary_dim;
  if (r < 2 || r > 128 || r % 2) return fail(TILEMIX_ERR_SHAPE, "rotary_dim (%d) must be even, 2 .. 128", r);
  if (!(isfinite(s->base) && s->base > 0)) return fail(TILEMIX_ERR_SHAPE, "base must be finite and > 0");
  if (s->kind < TILEMIX_SCALING_NONE || s->kind > TILEMIX_SCALING_YARN)
    return fail(TILEMIX_ERR_UNSUPPORTED, "scaling kind %d not supported", s->kind);
  if (s->kind != TILEMIX_SCALING_NONE && !(isfinite(s->factor) && s->factor >= 1))
    return fail(TILEMIX_ERR_SHAPE, "factor must be finite and >= 1");
  double base = s->base;
  if (s->kind == TILEMIX_SCALING_NTK) {
    if (r < 4) return fail(TILEMIX_ERR_SHAPE, "NTK scaling needs rotary_dim >= 4");
    base *= pow(s->factor, (double)r / (r - 2));
  }
  if (s->kind == TILEMIX_SCALING_YARN &&
      !(s->original_len >= 1 && isfinite(s->beta_fast) && s->beta_slow > 0 && s->beta_fast > s->beta_slow))
    return fail(TILEMIX_ERR_SHAPE, "YaRN scaling needs original_len >= 1 and beta_fast > beta_slow > 0");
  *magnitude = s->kind == TILEMIX_SCALING_YARN ? (float)(0.1 * log(s->factor) + 1.0) : 1.0f;
  for (int i = 0; i < r / 2; ++i) {
    const double f = pow(base, -2.0 * i / r);
    if (s->kind == TILEMIX_SCALING_LINEAR) {
      inv_freq[i] = f / s->factor;
    } else if (s->kind == TILEMIX_SCALING_YARN) {
      const double rotations = s->original_len * f / (2 * kPi);
      const double keep = fmin(fmax((rotations - s->beta_slow) / (s->beta_fast - s->beta_slow), 0.0), 1.0);
      inv_freq[i] = keep * f + (1.0 - keep) * f / s->factor;
    } else {
      inv_freq[i] = f;
    }
  }
  return ok();
}

tilemix_status tilemix_rotary(const tilemix_rotary_params* p, const int32_t* positions, const int32_t* seqlens_k,
                              const int32_t* cu_seqlens, int32_t batch, int32_t total, const void* Q, int64_t q_stride,
                              void* Q_out, int64_t q_out_stride, const void* K, int64_t k_stride, void* K_out,
                              int64_t k_out_stride, void* stream) {
  if (!p) return fail(TILEMIX_ERR_NULL, "params is NULL");
  if (p->type != TILEMIX_FP16 && p->type != TILEMIX_BF16)
    return fail(TILEMIX_ERR_UNSUPPORTED, "type %d not supported (FP16 or BF16)", p->type);
  if (p->layout != TILEMIX_ROTARY_HALF && p->layout != TILEMIX_ROTARY_INTERLEAVED)
    return fail(TILEMIX_ERR_UNSUPPORTED, "layout %d not supported", p->layout);
  if (p->head_dim != 64 && p->head_dim != 128)
    return fail(TILEMIX_ERR_UNSUPPORTED, "head_dim %d not supported (64 or 128)", p->head_dim);
  if (p->rotary_dim < 2 || p->rotary_dim > p->head_dim || p->rotary_dim % 2)
    return fail(TILEMIX_ERR_SHAPE, "rotary_dim (%d) must be even, 2 .. head_dim", p->rotary_dim);
  if (p->heads_q < 0 || p->heads_k < 0 || p->heads_q > 65535 || p->heads_k > 65535 || p->heads_q + p->heads_k == 0)
    return fail(TILEMIX_ERR_SHAPE, "heads_q and heads_k must be 0 .. 65535, not both 0");
  if (!isfinite(p->magnitude)) return fail(TILEMIX_ERR_SHAPE, "magnitude must be finite");
  if (total < 0 || total > kRowsMax) return fail(TILEMIX_ERR_SHAPE, "total must be 0 .. %d", kRowsMax);
  if (!positions) {
    if (batch < 1 || batch > 65535) return fail(TILEMIX_ERR_SHAPE, "batch must be 1 .. 65535");
    if (!cu_seqlens && total % batch) return fail(TILEMIX_ERR_SHAPE, "total must be a multiple of batch without cu_seqlens");
  }
  const struct { const void* x; void* y; long long in, out; int heads; const char* name; } ops[2] = {
      {Q, Q_out, q_stride, q_out_stride, p->heads_q, "Q"}, {K, K_out, k_stride, k_out_stride, p->heads_k, "K"}};
  for (const auto& o : ops)
    if (o.heads)
      for (long long s : {o.in, o.out})
        if (s < 0 || s > kStrideMax || s % 8) return fail(TILEMIX_ERR_SHAPE, "row strides must be >= 0 and multiples of 8");
  if (total == 0) return ok();
  if (!p->inv_freq) return fail(TILEMIX_ERR_NULL, "inv_freq is NULL");
  if (!aligned(p->inv_freq, 8)) return fail(TILEMIX_ERR_ALIGN, "inv_freq must be 8-byte aligned");
  if (positions ? !aligned(positions, 4) : !aligned(seqlens_k, 4) || !aligned(cu_seqlens, 4))
    return fail(TILEMIX_ERR_ALIGN, "positions, seqlens_k and cu_seqlens must be 4-byte aligned");
  if (!positions && !seqlens_k) return fail(TILEMIX_ERR_NULL, "positions or seqlens_k is needed");
  int in_place = 0, tensors = 0;
  for (const auto& o : ops) {
    if (!o.heads) continue;
    const long long row = (long long)o.heads * p->head_dim;
    if (!o.x || !o.y) return fail(TILEMIX_ERR_NULL, "%s and %s_out must be non-NULL", o.name, o.name);
    if (!aligned(o.x, 16) || !aligned(o.y, 16)) return fail(TILEMIX_ERR_ALIGN, "%s and %s_out must be 16-byte aligned", o.name, o.name);
    if (total > 1 && o.out < row) return fail(TILEMIX_ERR_SHAPE, "the rows of %s_out overlap", o.name);
    if (o.x == o.y && total > 1 && o.in != o.out) return fail(TILEMIX_ERR_SHAPE, "%s_out is %s with another stride", o.name, o.name);
    in_place += o.x == o.y;
    ++tensors;
  }
  tilemix::RotaryArgs a{};
  a.positions = positions;
  a.seqlens = seqlens_k;
  a.cu = cu_seqlens;
  a.batch = batch;
  a.total = total;
  if (!positions && !cu_seqlens) a.div_len = tilemix::FastDiv((uint32_t)(total / batch));
  a.inv_freq = p->inv_freq;
  a.magnitude = p->magnitude;
  a.inverse = p->inverse ? 1 : 0;
  a.d = p->head_dim;
  a.r = p->rotary_dim;
  a.Hq = p->heads_q;
  a.Hk = p->heads_k;
  a.in_place = in_place == tensors;
  a.Q = Q; a.Q_out = Q_out; a.q_stride = q_stride; a.q_out_stride = q_out_stride;
  a.K = K; a.K_out = K_out; a.k_stride = k_stride; a.k_out_stride = k_out_stride;
  const hipError_t e = tilemix::launch_rotary(a, p->type, p->layout == TILEMIX_ROTARY_HALF, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : fail(TILEMIX_ERR_HIP, "rotary: %s", hipGetErrorString(e));
}

}  // extern "C"
