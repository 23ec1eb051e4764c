// Launch interface of the norm in front of the head (npd_norm.hip, npd_norm_api.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "npd_internal.hpp"

namespace npd {

constexpr int kNormMaxWidth = 1 << 16;
// Rows' sums of the parameters' gradients: at most so many of them, joined by a second kernel.
constexpr int kNormPieces = 512;
// Widest rows whose gradient kernel also holds its sums of the parameters' gradients in registers; wider rows have theirs
// summed by a kernel of its own, column by column.
constexpr int kNormHeldWidth = 16384;

// y = (x - mean) rstd w + b;  rms: mean = 0
struct NormArgs {
  int64_t T;
  int32_t D;
  int32_t rms;
  const uint16_t* x;
  int64_t x_stride;
  const uint16_t *w, *b;  // or null: 1, 0
  uint16_t* y;
  int64_t y_stride;
  float* mean;            // out, or null
  float* rstd;
  float eps;
};
hipError_t launch_norm(const NormArgs& a, hipStream_t stream);

// With n = (x - mean) rstd and a = g w:  dx = rstd (a - mean(a) - n mean(a n)),  dw = sum over rows of g n,  db of g;  rms: without mean(a)
struct NormGradArgs {
  int64_t T;
  int32_t D;
  int32_t rms;
  const uint16_t* g;
  int64_t g_stride;
  const uint16_t* x;
  int64_t x_stride;
  const uint16_t* w;      // or null: 1
  const float* mean;      // null with rms
  const float* rstd;
  uint16_t* dx;           // or null
  int64_t dx_stride;
  uint16_t *dw, *db;      // or null
  float *dw_pieces, *db_pieces;  // [pieces][D]
  int32_t pieces;         // norm_pieces()
  int32_t accumulate;
};
// pieces of the parameters' gradients, of a call on so many rows
int norm_pieces(int64_t T, int32_t D);
hipError_t launch_norm_grad(const NormGradArgs& a, hipStream_t stream);

}  // namespace npd
