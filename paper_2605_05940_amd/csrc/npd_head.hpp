// Launch interface of the head operators: arguments of their kernels, shared by npd_head_api.hip and the kernel files.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "npd_head_gemm.hpp"
#include "npd_internal.hpp"

namespace npd {

// Columns of one partial sum of a row: what a wave of the forward product holds of it, 128, or 64 with the small tiles; with few rows
// what a workgroup holds of it, 128, 64 or 32.
constexpr int kHeadPart = 128, kHeadSmallPart = 64, kHeadTokensPart = 32;

// Tiles of 128 x 128 in place of 256 x 256: where there are so few that each has a compute unit to itself either way, a tile's own
// time decides.  Measured (MI355X, loss of 512 positions of width 1,024 with the hidden states' / the weights' gradient, us, 256 / 128):
// 16 large tiles (2,048 entries) 80, 69 / 52, 42; 32 91, 76 / 62, 50; 64 106, 84 / 79, 75; 128 (16,384 entries) 128, 100 / 140, 112.
inline bool head_small(int64_t rows, int64_t columns) {
  return (rows + 255) / 256 * ((columns + 255) / 256) <= 64;
}

// Workgroups of a kernel whose workgroups take one tile after the other: one per compute unit, whose LDS the stages fill (a
// multiple of eight, see head_tile).
inline unsigned head_grid(int64_t tiles) {
  const int64_t units = compute_units() / 8 * 8;
  return (unsigned)(tiles < units || units == 0 ? tiles : units);
}

enum HeadForward { kHeadLogits = 0, kHeadSums = 1, kHeadSumsKept = 2 };

// x = (q w^T + bias), soft-capped, of a chunk of rows; then by HeadForward
//   kHeadLogits     out = x, rounded to bf16
//   kHeadSums       part[row][v / part_columns] = (r, z): sum over those columns of 2^(x c - r) is z
//   kHeadSumsKept   and e[row][v] = 2^(x c - r) (with a soft cap times dx / d(q w^T)), rounded to bf16; 0 for v >= V
struct HeadForwardArgs {
  HeadChunk chunk;
  HeadMatrix q, w;      // q.rows is the chunk's (set on the device)
  const uint16_t* bias; // or null
  int32_t D, K, V;      // K: D rounded up to eight
  float cap;            // 0: none
  float c;              // log2(e) / tau
  const float* r0;      // [rows] a logit of the row times c, whole, or -1e30: the reference of columns not far above it
  float2* part;
  int32_t parts;
  int32_t part_columns; // up to kHeadFewRows rows head_few_part(): 128, 64 or 32; else 64 with head_small() and 128
  int32_t tokens;       // head_tokens()
  uint16_t* e;
  int64_t e_stride;
  uint16_t* out;
  int64_t out_stride;
};
hipError_t launch_head_forward(const HeadForwardArgs& a, HeadForward what, int64_t rows, hipStream_t stream);

// Rows that are so few that reading the weights is all the time: the weights go straight into registers, at any alignment.
constexpr int64_t kHeadFewRows = 64;
// Up to eight of them are head_tokens_kernel's, unless rows of the weights begin on odd values: the loads that cost least there are
// head_few_kernel's (49,152 x 4,095, 1 / 8 rows, MI355X: 132 / 178 us here, 109 there).  Nine rows of 151,936 x 2,048 take 177 us here, 117
// there.
inline bool head_tokens(int64_t rows, int64_t weight_stride) { return rows <= 8 && weight_stride % 2 == 0; }
// Columns of a workgroup of either.  Narrower ones where 128 columns leave compute units without a workgroup, and always for rows
// that begin on odd values.  Measured (MI355X, us, of 128 and narrower, weights out of the caches):
//   head_tokens_kernel, 1 / 8 rows: 8,000 x 1,024 12.1, 9.5 / 17.1, 10.1; 16,000 x 2,048 20.2, 16.5 / 29.0, 18.8; 32,000 x 4,096 41.9, 52.1 /
//   54.8, 47.6; 50,048 x 1,024 21.8, 23.6 / 26.7, 30.3; 32,000 x 512 (a wave has one block of k) 10.2, 12.8 / 13.0, 18.0
//   head_few_kernel, 16 / 48 rows: 16,000 x 2,048 30.3, 22.5 / 37.6, 28.5; 32,000 x 4,096 62.2, 49.4 / 77.4, 65.8; 50,048 x 1,024 21.7, 26.4 /
//   29.1, 28.0; 98,000 x 1,024 39.2, 43.6 / 42.3, 50.6; odd: 49,152 x 4,095 169, 110 / 177, 136; 100,003 x 1,023 71.1, 66.6 / 90.5, 84.5
inline int head_few_part(int64_t rows, int64_t columns, int64_t width, int64_t weight_stride) {
  if (head_tokens(rows, weight_stride)) return width >= 1024 && columns < 256 * (rows <= 4 ? 96 : 128) ? kHeadTokensPart : kHeadPart;
  return weight_stride % 2 != 0 || columns < 256 * 128 ? kHeadSmallPart : kHeadPart;
}
// Whether workgroups of up to four rows and 128 columns request a block's loads together, by their number: with few of them to a
// compute unit there is little in flight else; with four and more the compiler's order, which multiplies in between, is as fast or
// faster.  Measured (MI355X, us, together / compiler's order, weights out of the caches), one row, logits and scores: 16,000 x 2,048 (parts of
// 32, always together) 16.5 / 23.6, 27.8 / 34.9; 32,000 x 4,096 42.6 / 50.3, 56.3 / 62.8; 98,000 x 1,024 32.7 / 35.2, 44.0 / 46.2; 106,000 x 2,048
// 73.5 / 76.8, 89.6 / 88.8; 120,000 x 2,048 74.7 / 78.0, 91.6 / 90.1; 128,256 x 4,096 153.7 / 157.8, 174.3 / 171.8 and on another card 164.5 /
// 158.0, 189 / 172; 151,936 x 2,048 93.7 / 94.5, 112.5 / 107.1; 262,144 x 1,152 91.0 / 91.2, 108.2 / 104.5.  Four rows alike; of eight the
// compiler's order is faster throughout (32,000 x 4,096 71 / 55).
inline bool head_together(int parts) { return parts <= 256 * 15 / 4; }
hipError_t launch_head_few(const HeadForwardArgs& a, HeadForward what, int64_t rows, hipStream_t stream);

// out[position of row m][n] = scale[m] sum_k g[m][k] w[k][n], k < K: the gradient of the hidden states.  k may be split into
// up to `most_splits` pieces, joined by a second kernel through `partial` [splits][rows][up(N, 4)].
struct HeadHiddenArgs {
  HeadChunk chunk;
  HeadMatrix g, w;
  const float* scale;    // or null: 1
  const int32_t* rows;   // positions of the rows, or null: m itself
  int32_t K, N, most_splits;
  float* partial;
  uint16_t* out;
  int64_t out_stride;
};
hipError_t launch_head_hidden(const HeadHiddenArgs& a, int64_t rows, hipStream_t stream);
// the most pieces that a chunk of up to so many rows is split into, and the floats that they take
int head_hidden_splits(int64_t rows, int32_t K, int32_t N);
size_t head_hidden_floats(int64_t rows, int32_t N, int splits);

// out[m][n] = sum_k g[k][m] h[k][n] over the rows k of the chunk, on top of the chunks before it (`partial`, fp32 [M][up(N, 4)]):
// the gradient of the weights.  `out` is written with the last chunk, on top of what it holds if `accumulate`.
struct HeadWeightArgs {
  HeadChunk chunk;
  HeadMatrix g, h;
  int32_t M, N;
  float* partial;
  uint16_t* out;
  int64_t out_stride;
  int32_t accumulate;
};
hipError_t launch_head_weight(const HeadWeightArgs& a, int64_t chunks, hipStream_t stream);

// both in one launch, where each is a few small tiles (MI355X, 512 x 1,024 x 256: 8.2 and 7.1 us one after the other)
bool head_both_small(const HeadHiddenArgs& h, const HeadWeightArgs& w, int64_t rows, int64_t chunks);
hipError_t launch_head_both(const HeadHiddenArgs& h, const HeadWeightArgs& w, int64_t rows, hipStream_t stream);

// out[m] = sum_k scale[k] g[k][m] likewise: the gradient of the bias
constexpr int kHeadBiasSplits = 32;
struct HeadBiasArgs {
  HeadChunk chunk;
  HeadMatrix g;
  const float* scale;
  int32_t M;
  float* pieces;   // [kHeadBiasSplits][M]
  float* partial;  // [M]
  uint16_t* out;
  int32_t accumulate;
};
hipError_t launch_head_bias(const HeadBiasArgs& a, hipStream_t stream);

// The positions that are scored, in order, their number, and zeros for the outputs of the others.
struct HeadRowsArgs {
  int64_t T;
  const uint8_t* mask;
  int32_t* rows;
  int32_t* count;
  float *kd, *nll, *lse;
  uint16_t* grad_hidden;
  int64_t grad_stride;
  int32_t D;
};
hipError_t launch_head_rows(const HeadRowsArgs& a, hipStream_t stream);

// dst[i][0 .. width) = src[first + i][0 .. cols), 0 behind; with y times 1 - (y / cap)^2, rounded to bf16 once more: an operand of the
// matrix products (error of both gradients against 64 bits, as a share of their norm: .00225, without a soft cap .00166)
struct HeadPackArgs {
  HeadChunk chunk;
  const uint16_t* src;
  int64_t src_stride;
  const uint16_t* y;
  int64_t y_stride;
  float cap;
  int32_t cols, width;
  uint16_t* dst;
  int64_t dst_stride;
};
hipError_t launch_head_pack(const HeadPackArgs& a, int64_t rows, hipStream_t stream);

// What a row of the loss needs besides the sums over the vocabulary: its logits at the label and at the teacher's ids.
struct HeadLossArgs {
  HeadChunk chunk;
  const int32_t* rows;
  const uint16_t* src;   // hidden states and weights as the caller has them
  int64_t src_stride;
  const uint16_t* weight;
  int64_t weight_stride;
  HeadMatrix h;          // packed rows of the chunk
  const uint16_t* bias;
  int32_t D, K, V, k;    // K: D rounded up to eight
  float cap, c;
  const int32_t* labels;  // null: not used
  const int32_t* tidx;
  const float* tval;
  float* x;       // [cap][1 + k] logits at the label (or column 0) and the ids
  float* r0;      // [cap]
  const float2* part;
  int32_t parts, part_columns;
  float *kd, *nll, *lse;
  int32_t* status;
  // gradients
  float kd_weight, ce_weight;  // grad_scale / tau, ce_grad_scale
  uint16_t* e;                 // null: forward only
  int64_t e_stride;
  float* scale;
  uint16_t* hs;                // scaled rows for the weights' gradient, or null
};
hipError_t launch_head_prepare(const HeadRowsArgs& r, const HeadLossArgs& a, hipStream_t stream);
hipError_t launch_head_gather(const HeadLossArgs& a, int64_t rows, hipStream_t stream);
hipError_t launch_head_finish(const HeadLossArgs& a, int64_t rows, hipStream_t stream);

}  // namespace npd
