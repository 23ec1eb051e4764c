// Launch interface of the head in 8-bit integers (npd_int8*.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/npd.h"
#include "npd_head.hpp"

namespace npd {

// q = x / scale to the nearest whole number (of two the even one), scale = max |x| / 127, row by row
struct QuantizeArgs {
  int64_t R;
  int32_t D;
  const uint16_t* x;
  int64_t x_stride;
  int8_t* q;
  int64_t q_stride;
  float* scale;
};
hipError_t launch_quantize(const QuantizeArgs& a, hipStream_t stream);

// out[p][v] = (sum_k h[p][k] w[v][k]) h_scale[p] w_scale[v] + bias[v], soft-capped
struct Int8Args {
  int64_t T;
  int32_t D, V;
  const int8_t* h;
  int64_t h_stride;      // bytes, as everywhere here
  const float* h_scale;
  const int8_t* w;
  int64_t w_stride;
  const float* w_scale;
  const uint16_t* bias;  // or null
  float cap;             // 0: none
  uint16_t* out;
  int64_t out_stride;
};

// Up to kHeadFewRows rows, at any alignment.
hipError_t launch_int8_few(const Int8Args& a, hipStream_t stream);
// Any number of rows; rows of h and w begin on 16 bytes and their padding to a multiple of 16 may be read, of which h's is 0.
hipError_t launch_int8_many(const Int8Args& a, hipStream_t stream);
// rows of `to` are those of `from` and zeros up to to_width bytes, a multiple of 16; two matrices of one width, either of no rows
struct Int8Packed {
  const int8_t* from;
  int64_t stride;
  int8_t* to;
  int64_t rows;
};
hipError_t launch_int8_pack(const Int8Packed& first, const Int8Packed& second, int32_t to_width, int32_t cols, hipStream_t stream);

// what npd_head_logits_int8 needs (npd_int8_api.hip)
size_t int8_workspace_bytes(const npd_head_desc* desc);

}  // namespace npd
