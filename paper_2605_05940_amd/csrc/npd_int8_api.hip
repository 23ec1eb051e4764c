// C ABI of the head in 8-bit integers (include/npd.h): argument checks, the workspace's layout, and the launches of a call.
// Every check runs before the first HIP call.
#include <float.h>
#include <math.h>

#include "../../include/npd.h"
#include "npd_check.hpp"
#include "npd_int8.hpp"

namespace npd {

namespace {

npd_status check_int8(const npd_head_desc* d) {
  if (!d) return NPD_ERR_NULL;
  if (d->n_tokens <= 0 || d->vocab <= 0 || d->width <= 0) return NPD_ERR_SHAPE;
  // (the sums: 2^16 products of up to 2^14 in 32 bits)
  if (d->n_tokens > NPD_HEAD_MAX_TOKENS || d->vocab > NPD_HEAD_MAX_VOCAB || d->width > NPD_HEAD_MAX_WIDTH) return NPD_ERR_UNSUPPORTED;
  if (d->flags & ~(uint32_t)NPD_HEAD_UNALIGNED) return NPD_ERR_VALUE;
  const int64_t strides[3][2] = {{d->hidden_stride, d->width}, {d->weight_stride, d->width}, {d->logits_stride, d->vocab}};
  for (const auto& s : strides)
    if (s[0] < s[1]) return NPD_ERR_SHAPE;
  for (const auto& s : strides)
    if (s[0] > NPD_HEAD_MAX_VOCAB) return NPD_ERR_UNSUPPORTED;
  if (!(d->softcap >= 0.0f) || !isfinite(d->softcap) || (d->softcap > 0.0f && d->softcap < FLT_MIN)) return NPD_ERR_VALUE;
  return NPD_OK;
}

// What cannot be read where it lies is copied: rows that do not begin on 16 bytes, or whose last 16 are not all theirs.
struct Plan {
  int32_t padded = 0;
  bool few = false, pack_h = false, pack_w = false;
  size_t h = 0, w = 0, bytes = 0;
};

Plan make_plan(const npd_head_desc& d) {
  Plan p;
  p.padded = (d.width + 15) / 16 * 16;
  const bool odd = d.width % 16 != 0 || (d.flags & NPD_HEAD_UNALIGNED);
  // (64 rows of 50,048 x 1,024 take 20.9 us in the kernels that read weights at any alignment, 15.9 in tiles; 17 rows 14.7 and 14.0, of
  // 151,936 x 2,048 61.5 and 65.7)
  p.few = d.n_tokens <= (odd || d.hidden_stride % 16 != 0 || d.weight_stride % 16 != 0 ? kHeadFewRows : kHeadFewRows / 2);
  p.pack_h = !p.few && (odd || d.hidden_stride % 16 != 0);
  p.pack_w = !p.few && (odd || d.weight_stride % 16 != 0);
  auto take = [&p](size_t bytes) {
    const size_t at = p.bytes;
    p.bytes += (bytes + 255) / 256 * 256;
    return at;
  };
  if (p.pack_h) p.h = take((size_t)d.n_tokens * p.padded);
  if (p.pack_w) p.w = take((size_t)d.vocab * p.padded);
  return p;
}

}  // namespace

size_t int8_workspace_bytes(const npd_head_desc* d) { return check_int8(d) == NPD_OK ? make_plan(*d).bytes : 0; }

}  // namespace npd

extern "C" {

npd_status npd_quantize_rows(int64_t n_rows, int32_t width, int64_t x_stride, int64_t q_stride, const void* x, int8_t* q, float* scale,
                             void* stream) {
  using namespace npd;
  if (n_rows <= 0 || width <= 0) return NPD_ERR_SHAPE;
  if (n_rows > NPD_HEAD_MAX_TOKENS || width > NPD_HEAD_MAX_WIDTH) return NPD_ERR_UNSUPPORTED;
  if (x_stride < width || q_stride < width || !stride_fits(n_rows, x_stride) || !stride_fits(n_rows, q_stride)) return NPD_ERR_SHAPE;
  if (!x || !q || !scale) return NPD_ERR_NULL;
  if (misaligned(x, 2) || misaligned(scale, 4)) return NPD_ERR_VALUE;
  const Range in[1] = {range_of(x, rows_bytes(n_rows, x_stride, width, 2))};
  const Range out[2] = {range_of(q, rows_bytes(n_rows, q_stride, width, 1)), range_of(scale, (size_t)n_rows * 4)};
  if (any_alias(in, 1, out, 2)) return NPD_ERR_ALIAS;
  const QuantizeArgs a = {n_rows, width, static_cast<const uint16_t*>(x), x_stride, q, q_stride, scale};
  return launch_quantize(a, static_cast<hipStream_t>(stream)) == hipSuccess ? NPD_OK : NPD_ERR_HIP;
}

npd_status npd_head_logits_int8(const npd_head_desc* desc, const int8_t* hidden, const float* hidden_scale, const int8_t* weight,
                                const float* weight_scale, const void* bias, void* logits, void* workspace, size_t workspace_bytes,
                                void* stream) {
  using namespace npd;
  const npd_status st = check_int8(desc);
  if (st != NPD_OK) return st;
  const npd_head_desc& d = *desc;
  if (!hidden || !hidden_scale || !weight || !weight_scale || !logits) return NPD_ERR_NULL;
  const bool aligned = aligned16(hidden) && aligned16(weight);
  if (misaligned(hidden_scale, 4) || misaligned(weight_scale, 4) || misaligned(bias, 2) || misaligned(logits, 2) ||
      (!aligned && !(d.flags & NPD_HEAD_UNALIGNED)))
    return NPD_ERR_VALUE;
  const Plan p = make_plan(d);
  if (p.bytes > 0 && (workspace_bytes < p.bytes || !workspace || misaligned(workspace, 256))) return NPD_ERR_WORKSPACE;
  const int64_t T = d.n_tokens;
  const size_t V = (size_t)d.vocab;
  const Range in[5] = {range_of(hidden, rows_bytes(T, d.hidden_stride, d.width, 1)), range_of(hidden_scale, (size_t)T * 4),
                       range_of(weight, rows_bytes(d.vocab, d.weight_stride, d.width, 1)), range_of(weight_scale, V * 4), opt_range(bias, V * 2)};
  const Range out[2] = {range_of(logits, rows_bytes(T, d.logits_stride, d.vocab, 2)), opt_range(workspace, p.bytes)};
  if (any_alias(in, 5, out, 2)) return NPD_ERR_ALIAS;
  const hipStream_t on = static_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  Int8Args a{};
  a.T = T;
  a.D = d.width;
  a.V = d.vocab;
  a.h = hidden;
  a.h_stride = d.hidden_stride;
  a.h_scale = hidden_scale;
  a.w = weight;
  a.w_stride = d.weight_stride;
  a.w_scale = weight_scale;
  a.bias = static_cast<const uint16_t*>(bias);
  a.cap = d.softcap;
  a.out = static_cast<uint16_t*>(logits);
  a.out_stride = d.logits_stride;
  if (p.few) return launch_int8_few(a, on) == hipSuccess ? NPD_OK : NPD_ERR_HIP;
  if (p.pack_h || p.pack_w) {
    const Int8Packed h = {a.h, a.h_stride, reinterpret_cast<int8_t*>(ws + p.h), p.pack_h ? T : 0};
    const Int8Packed w = {a.w, a.w_stride, reinterpret_cast<int8_t*>(ws + p.w), p.pack_w ? d.vocab : 0};
    if (launch_int8_pack(h, w, p.padded, d.width, on) != hipSuccess) return NPD_ERR_HIP;
    if (p.pack_h) {
      a.h = h.to;
      a.h_stride = p.padded;
    }
    if (p.pack_w) {
      a.w = w.to;
      a.w_stride = p.padded;
    }
  }
  return launch_int8_many(a, on) == hipSuccess ? NPD_OK : NPD_ERR_HIP;
}

}  // extern "C"
