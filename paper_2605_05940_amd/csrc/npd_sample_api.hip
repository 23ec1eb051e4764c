// C ABI of the tokens drawn from logits (include/npd.h): argument checks and the launch.  Every check runs before the first HIP call.
#include <math.h>

#include "../../include/npd.h"
#include "npd_check.hpp"
#include "npd_sample.hpp"

namespace {

npd_status check_sample(const npd_sample_desc* desc) {
  using namespace npd;
  if (!desc) return NPD_ERR_NULL;
  const npd_sample_desc& d = *desc;
  if (d.n_tokens <= 0 || d.vocab <= 0) return NPD_ERR_SHAPE;
  if (d.n_tokens > NPD_MAX_TOKENS || d.vocab > NPD_MAX_VOCAB) return NPD_ERR_UNSUPPORTED;
  if (d.logits_stride < d.vocab || !stride_fits(d.n_tokens, d.logits_stride)) return NPD_ERR_SHAPE;
  return d.flags != 0 ? NPD_ERR_VALUE : NPD_OK;
}

size_t sample_bytes(const npd_sample_desc& d) {
  const int parts = npd::sample_parts(d.n_tokens, d.vocab);
  return parts < 2 ? 0 : (size_t)d.n_tokens * parts * npd::kSamplePartBytes;
}

}  // namespace

extern "C" size_t npd_sample_workspace_bytes(const npd_sample_desc* desc) {
  return check_sample(desc) == NPD_OK ? sample_bytes(*desc) : 0;
}

extern "C" npd_status npd_sample_tokens(const npd_sample_desc* desc, const void* logits, const float* uniform, const uint8_t* loss_mask,
                                        const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                                        int32_t* token, float* logprob, float* nll, int32_t* kept, int32_t* dev_status, void* workspace,
                                        size_t workspace_bytes, void* stream) {
  using namespace npd;
  const npd_status st = check_sample(desc);
  if (st != NPD_OK) return st;
  const npd_sample_desc& d = *desc;
  if (!logits || !uniform || !token) return NPD_ERR_NULL;
  // (settings that rows have of their own are looked at on the device)
  if (!temperature && !(d.temperature >= 0.0f && isfinite(d.temperature))) return NPD_ERR_VALUE;
  if (!top_k && d.top_k < 0) return NPD_ERR_VALUE;
  if (!top_p && !(d.top_p >= 0.0f && d.top_p <= 1.0f)) return NPD_ERR_VALUE;
  if (!min_p && !(d.min_p >= 0.0f && d.min_p <= 1.0f)) return NPD_ERR_VALUE;
  if (misaligned(logits, 2) || misaligned(uniform, 4) || misaligned(temperature, 4) || misaligned(top_k, 4) || misaligned(top_p, 4) ||
      misaligned(min_p, 4) || misaligned(token, 4) || misaligned(logprob, 4) || misaligned(nll, 4) || misaligned(kept, 4) ||
      misaligned(dev_status, 4))
    return NPD_ERR_VALUE;
  const int64_t T = d.n_tokens;
  const size_t n = (size_t)T * 4;
  const Range in[7] = {range_of(logits, rows_bytes(T, d.logits_stride, d.vocab, 2)), range_of(uniform, n), opt_range(loss_mask, (size_t)T),
                       opt_range(temperature, n), opt_range(top_k, n), opt_range(top_p, n), opt_range(min_p, n)};
  // (rows are counted in parts with a workspace that is large enough; results do not depend on it)
  const size_t bytes = sample_bytes(d);
  const bool split = workspace && bytes > 0 && workspace_bytes >= bytes;
  if (split && misaligned(workspace, 256)) return NPD_ERR_WORKSPACE;
  const Range out[6] = {opt_range(split ? workspace : nullptr, bytes),
                        range_of(token, n), opt_range(logprob, n), opt_range(nll, n), opt_range(kept, n), opt_range(dev_status, 4)};
  if (any_alias(in, 7, out, 6)) return NPD_ERR_ALIAS;
  SampleArgs a{};
  a.T = T;
  a.V = d.vocab;
  a.x = static_cast<const uint16_t*>(logits);
  a.stride = d.logits_stride;
  a.u = uniform;
  a.mask = loss_mask;
  a.tau = d.temperature;
  a.top_p = d.top_p;
  a.min_p = d.min_p;
  a.top_k = d.top_k;
  a.taus = temperature;
  a.top_ks = top_k;
  a.top_ps = top_p;
  a.min_ps = min_p;
  a.token = token;
  a.logprob = logprob;
  a.nll = nll;
  a.kept = kept;
  a.status = dev_status;
  a.parts = split ? sample_parts(T, d.vocab) : 1;
  a.workspace = workspace;
  return launch_sample(a, static_cast<hipStream_t>(stream)) == hipSuccess ? NPD_OK : NPD_ERR_HIP;
}
