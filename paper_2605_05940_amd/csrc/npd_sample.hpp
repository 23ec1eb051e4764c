// Launch interface of the tokens drawn from logits (npd_sample.hip, npd_sample_api.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "npd_internal.hpp"

namespace npd {

struct SampleArgs {
  int64_t T;
  int32_t V;
  const uint16_t* x;   // logits
  int64_t stride;
  const float* u;      // [T] in [0, 1)
  const uint8_t* mask; // [T] or null
  // a setting of all rows, or one for each
  float tau, top_p, min_p;
  int32_t top_k;
  const float *taus, *top_ps, *min_ps;
  const int32_t* top_ks;
  int32_t* token;
  float *logprob, *nll;  // or null
  int32_t* kept;
  int32_t* status;
  int32_t parts;    // of a row that workgroups count each, sample_parts(), 1: none
  void* workspace;  // kSamplePartBytes for each part of each row
};
// Parts of a call's rows that workgroups of their own count, 1 where there are rows enough
constexpr int kSampleParts = 8;
constexpr size_t kSamplePartBytes = 4 * (7936 + 4 + 256);
int sample_parts(int64_t T, int32_t V);
hipError_t launch_sample(const SampleArgs& a, hipStream_t stream);

}  // namespace npd
