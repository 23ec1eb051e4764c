// C ABI of the norm in front of the head (include/npd.h): argument checks and launches.  Every check runs before the first HIP call.
#include <math.h>

#include "../../include/npd.h"
#include "npd_check.hpp"
#include "npd_norm.hpp"

namespace {

using namespace npd;

constexpr uint32_t kParameterFlags = NPD_NORM_GRAD_WEIGHT | NPD_NORM_GRAD_BIAS;

// `backward`: which of the two calls
npd_status check_norm(const npd_norm_desc* d, bool backward) {
  if (!d) return NPD_ERR_NULL;
  if (d->n_tokens <= 0 || d->width <= 0) return NPD_ERR_SHAPE;
  if (d->n_tokens > NPD_HEAD_MAX_TOKENS || d->width > kNormMaxWidth) return NPD_ERR_UNSUPPORTED;
  const uint32_t known = backward ? (uint32_t)NPD_NORM_RMS | NPD_NORM_GRAD_X | kParameterFlags | NPD_NORM_ACCUMULATE : (uint32_t)NPD_NORM_RMS;
  if (d->flags & ~known) return NPD_ERR_VALUE;
  if (backward && !(d->flags & (NPD_NORM_GRAD_X | kParameterFlags))) return NPD_ERR_VALUE;
  if ((d->flags & NPD_NORM_ACCUMULATE) && !(d->flags & kParameterFlags)) return NPD_ERR_VALUE;
  const bool has_grad_x = backward && (d->flags & NPD_NORM_GRAD_X);
  if (d->x_stride < d->width || d->y_stride < d->width || (has_grad_x && d->grad_x_stride < d->width)) return NPD_ERR_SHAPE;
  if (!stride_fits(d->n_tokens, d->x_stride) || !stride_fits(d->n_tokens, d->y_stride) ||
      (has_grad_x && !stride_fits(d->n_tokens, d->grad_x_stride)))
    return NPD_ERR_SHAPE;
  if (!backward && (!(d->eps >= 0.0f) || !isfinite(d->eps))) return NPD_ERR_VALUE;
  return NPD_OK;
}

size_t pieces_bytes(const npd_norm_desc& d) {
  const size_t one = ((size_t)norm_pieces(d.n_tokens, d.width) * d.width * 4 + 255) / 256 * 256;
  return ((d.flags & NPD_NORM_GRAD_WEIGHT ? 1 : 0) + (d.flags & NPD_NORM_GRAD_BIAS ? 1 : 0)) * one;
}

}  // namespace

extern "C" {

size_t npd_layer_norm_workspace_bytes(const npd_norm_desc* desc) {
  return check_norm(desc, true) == NPD_OK ? pieces_bytes(*desc) : 0;
}

npd_status npd_layer_norm(const npd_norm_desc* desc, const void* x, const void* weight, const void* bias, void* y, float* mean,
                          float* rstd, void* stream) {
  const npd_status st = check_norm(desc, false);
  if (st != NPD_OK) return st;
  const npd_norm_desc& d = *desc;
  if (!x || !y) return NPD_ERR_NULL;
  if ((d.flags & NPD_NORM_RMS) && mean) return NPD_ERR_VALUE;
  if (misaligned(x, 2) || misaligned(weight, 2) || misaligned(bias, 2) || misaligned(y, 2) || misaligned(mean, 4) || misaligned(rstd, 4))
    return NPD_ERR_VALUE;
  const int64_t T = d.n_tokens;
  const size_t D = (size_t)d.width;
  const Range in[3] = {range_of(x, rows_bytes(T, d.x_stride, d.width, 2)), opt_range(weight, D * 2), opt_range(bias, D * 2)};
  const Range out[3] = {range_of(y, rows_bytes(T, d.y_stride, d.width, 2)), opt_range(mean, (size_t)T * 4), opt_range(rstd, (size_t)T * 4)};
  if (any_alias(in, 3, out, 3)) return NPD_ERR_ALIAS;
  NormArgs a{};
  a.T = T;
  a.D = d.width;
  a.rms = (d.flags & NPD_NORM_RMS) != 0;
  a.x = static_cast<const uint16_t*>(x);
  a.x_stride = d.x_stride;
  a.w = static_cast<const uint16_t*>(weight);
  a.b = static_cast<const uint16_t*>(bias);
  a.y = static_cast<uint16_t*>(y);
  a.y_stride = d.y_stride;
  a.mean = mean;
  a.rstd = rstd;
  a.eps = d.eps;
  return launch_norm(a, static_cast<hipStream_t>(stream)) == hipSuccess ? NPD_OK : NPD_ERR_HIP;
}

npd_status npd_layer_norm_bwd(const npd_norm_desc* desc, const void* grad_y, const void* x, const void* weight, const float* mean,
                              const float* rstd, void* grad_x, void* grad_weight, void* grad_bias, void* workspace,
                              size_t workspace_bytes, void* stream) {
  const npd_status st = check_norm(desc, true);
  if (st != NPD_OK) return st;
  const npd_norm_desc& d = *desc;
  const bool rms = d.flags & NPD_NORM_RMS;
  if (!grad_y || !x || !rstd || (!rms && !mean)) return NPD_ERR_NULL;
  if (rms && mean) return NPD_ERR_VALUE;
  const void* grads[3] = {grad_x, grad_weight, grad_bias};
  const uint32_t flags[3] = {NPD_NORM_GRAD_X, NPD_NORM_GRAD_WEIGHT, NPD_NORM_GRAD_BIAS};
  for (int i = 0; i < 3; ++i) {
    if ((d.flags & flags[i]) && !grads[i]) return NPD_ERR_NULL;
    if (!(d.flags & flags[i]) && grads[i]) return NPD_ERR_VALUE;
  }
  if (misaligned(grad_y, 2) || misaligned(x, 2) || misaligned(weight, 2) || misaligned(mean, 4) || misaligned(rstd, 4) ||
      misaligned(grad_x, 2) || misaligned(grad_weight, 2) || misaligned(grad_bias, 2))
    return NPD_ERR_VALUE;
  const size_t bytes = pieces_bytes(d);
  if (bytes > 0 && (workspace_bytes < bytes || !workspace || misaligned(workspace, 256))) return NPD_ERR_WORKSPACE;
  const int64_t T = d.n_tokens;
  const size_t D = (size_t)d.width;
  const Range in[5] = {range_of(grad_y, rows_bytes(T, d.y_stride, d.width, 2)), range_of(x, rows_bytes(T, d.x_stride, d.width, 2)),
                       opt_range(weight, D * 2), opt_range(mean, (size_t)T * 4), range_of(rstd, (size_t)T * 4)};
  const Range out[4] = {grad_x ? range_of(grad_x, rows_bytes(T, d.grad_x_stride, d.width, 2)) : Range{0, 0}, opt_range(grad_weight, D * 2),
                        opt_range(grad_bias, D * 2), opt_range(workspace, bytes)};
  if (any_alias(in, 5, out, 4)) return NPD_ERR_ALIAS;
  NormGradArgs a{};
  a.T = T;
  a.D = d.width;
  a.rms = rms;
  a.g = static_cast<const uint16_t*>(grad_y);
  a.g_stride = d.y_stride;
  a.x = static_cast<const uint16_t*>(x);
  a.x_stride = d.x_stride;
  a.w = static_cast<const uint16_t*>(weight);
  a.mean = mean;
  a.rstd = rstd;
  a.dx = static_cast<uint16_t*>(grad_x);
  a.dx_stride = d.grad_x_stride;
  a.dw = static_cast<uint16_t*>(grad_weight);
  a.db = static_cast<uint16_t*>(grad_bias);
  char* ws = static_cast<char*>(workspace);
  a.dw_pieces = reinterpret_cast<float*>(ws);
  a.db_pieces = reinterpret_cast<float*>(grad_weight && grad_bias ? ws + bytes / 2 : ws);
  a.pieces = norm_pieces(T, d.width);
  a.accumulate = (d.flags & NPD_NORM_ACCUMULATE) != 0;
  return launch_norm_grad(a, static_cast<hipStream_t>(stream)) == hipSuccess ? NPD_OK : NPD_ERR_HIP;
}

}  // extern "C"
