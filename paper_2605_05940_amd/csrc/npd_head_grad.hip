// Gradients of a head from the gradient G of its logits (or from what the loss keeps in its place: G = scale (row) times e):
// dH = G W, contracted over the vocabulary; dW = G^T H, over the rows; db = column sums of G.
#include "npd_head.hpp"

namespace npd {
namespace {

__device__ __forceinline__ void store4(uint16_t* out, int n, int N, const float v[4]) {
  if (n + 4 <= N && (reinterpret_cast<uintptr_t>(out + n) & 7) == 0) {
    *reinterpret_cast<uint2*>(out + n) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (n + t < N) out[n + t] = one_bf16(v[t]);
  }
}

template <int MF, int NF>
__global__ __launch_bounds__(kHeadThreads, 1) void head_hidden_kernel(HeadHiddenArgs a) {
  using Product = HeadProduct<MF, NF, false, true, false>;
  __shared__ __attribute__((aligned(1024))) char lds[Product::kLds];
  const HeadSpan span = head_span(a.chunk);
  if (!span.there || span.rows == 0) return;
  const int mt = (span.rows + Product::kTileM - 1) / Product::kTileM, nt = (a.N + Product::kTileN - 1) / Product::kTileN;
  // a piece of k after the other (tiles of one piece share its rows of w)
  const unsigned per = (unsigned)(mt * nt + 7) / 8 * 8;
  const int split = (int)(blockIdx.x / per);
  if (split >= a.splits) return;
  const HeadTile tile = head_tile(blockIdx.x % per, mt, nt);
  if (!tile.there) return;
  const int64_t m0 = (int64_t)tile.m * Product::kTileM;
  const int n0 = tile.n * Product::kTileN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // pieces of whole rounds of the stages
  constexpr int kRound = kHeadStep * kHeadStages;
  const int rounds = (a.K + kRound - 1) / kRound;
  const int64_t k0 = (int64_t)rounds * split / a.splits * kRound, k1 = (int64_t)rounds * (split + 1) / a.splits * kRound;
  Product x;
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int j = 0; j < NF; ++j) x.acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  HeadMatrix g = a.g;
  g.rows = span.rows;
  x.run(g, a.w, m0, n0, k0, k1 < a.K ? k1 : a.K, lds);
#pragma unroll
  for (int i = 0; i < MF; ++i) {
    const int64_t m = m0 + (wave >> 1) * 16 * MF + 16 * i + (lane & 15);
    if (m >= span.rows) continue;
    const int nw = n0 + (wave & 1) * 16 * NF + 4 * (lane >> 4);
    if (a.splits > 1) {
      float* out = a.partial + (split * a.partial_rows + m) * a.N;
#pragma unroll
      for (int j = 0; j < NF; ++j)
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (nw + 16 * j + t < a.N) out[nw + 16 * j + t] = x.acc[i][j][t];
    } else {
      const float s = a.scale ? a.scale[m] : 1.0f;
      uint16_t* out = a.out + (a.rows ? (int64_t)a.rows[span.first + m] : span.first + m) * a.out_stride;
#pragma unroll
      for (int j = 0; j < NF; ++j) {
        const float v[4] = {x.acc[i][j][0] * s, x.acc[i][j][1] * s, x.acc[i][j][2] * s, x.acc[i][j][3] * s};
        store4(out, nw + 16 * j, a.N, v);
      }
    }
  }
}

// joins the pieces of head_hidden_kernel in their order
__global__ __launch_bounds__(256) void head_join_kernel(HeadHiddenArgs a) {
  const HeadSpan span = head_span(a.chunk);
  if (!span.there) return;
  for (int64_t m = blockIdx.x; m < span.rows; m += gridDim.x) {
    const float s = a.scale ? a.scale[m] : 1.0f;
    uint16_t* out = a.out + (a.rows ? (int64_t)a.rows[span.first + m] : span.first + m) * a.out_stride;
    for (int n = threadIdx.x; n < a.N; n += 256) {
      float v = 0.0f;
      for (int p = 0; p < a.splits; ++p) v += a.partial[(p * a.partial_rows + m) * a.N + n];
      out[n] = one_bf16(v * s);
    }
  }
}

template <int MF, int NF>
__global__ __launch_bounds__(kHeadThreads, 1) void head_weight_kernel(HeadWeightArgs a) {
  using Product = HeadProduct<MF, NF, true, true, false>;
  __shared__ __attribute__((aligned(1024))) char lds[Product::kLds];
  const HeadSpan span = head_span(a.chunk);
  if (!span.there) return;
  const HeadTile tile = head_tile(blockIdx.x, (a.M + Product::kTileM - 1) / Product::kTileM, (a.N + Product::kTileN - 1) / Product::kTileN);
  if (!tile.there) return;
  const int64_t m0 = (int64_t)tile.m * Product::kTileM;
  const int n0 = tile.n * Product::kTileN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Product x;
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int j = 0; j < NF; ++j) x.acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  // rows of the chunk: behind the last one nothing is read
  x.run(a.g, a.h, m0, n0, 0, span.rows, lds);
#pragma unroll
  for (int i = 0; i < MF; ++i) {
    const int64_t m = m0 + (wave >> 1) * 16 * MF + 16 * i + (lane & 15);
    if (m >= a.M) continue;
#pragma unroll
    for (int j = 0; j < NF; ++j) {
      const int n = n0 + (wave & 1) * 16 * NF + 16 * j + 4 * (lane >> 4);
      float v[4] = {x.acc[i][j][0], x.acc[i][j][1], x.acc[i][j][2], x.acc[i][j][3]};
      float* partial = a.partial + m * a.N;
      if (a.chunk.index > 0) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (n + t < a.N) v[t] += partial[n + t];
      }
      if (span.last) {
        uint16_t* out = a.out + m * a.out_stride;
        if (a.accumulate) {
#pragma unroll
          for (int t = 0; t < 4; ++t)
            if (n + t < a.N) v[t] += bf16_one(out[n + t]);
        }
        store4(out, n, a.N, v);
      } else {
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (n + t < a.N) partial[n + t] = v[t];
      }
    }
  }
}

__global__ __launch_bounds__(256) void head_bias_kernel(HeadBiasArgs a) {
  const HeadSpan span = head_span(a.chunk);
  if (!span.there) return;
  const int m = (blockIdx.x * 256 + threadIdx.x) * 8;  // rows of g begin on 16 bytes and are padded to eight
  if (m >= a.M) return;
  const int s = blockIdx.y;
  const int64_t b = (int64_t)span.rows * s / kHeadBiasSplits, e = (int64_t)span.rows * (s + 1) / kHeadBiasSplits;
  float sum[8] = {};
  for (int64_t r = b; r < e; ++r) {
    float x[8];
    unpack8(*reinterpret_cast<const uint4*>(a.g.p + r * a.g.stride + m), x);
    const float w = a.scale ? a.scale[r] : 1.0f;
    if (w != w) continue;  // a position with a bad label or id: no part of the shared gradients
#pragma unroll
    for (int t = 0; t < 8; ++t) sum[t] = __builtin_fmaf(x[t], w, sum[t]);
  }
#pragma unroll
  for (int t = 0; t < 8; ++t)
    if (m + t < a.M) a.pieces[(int64_t)s * a.M + m + t] = sum[t];
}

__global__ __launch_bounds__(256) void head_bias_join_kernel(HeadBiasArgs a) {
  const HeadSpan span = head_span(a.chunk);
  if (!span.there) return;
  const int m = blockIdx.x * 256 + threadIdx.x;
  if (m >= a.M) return;
  float v = a.chunk.index > 0 ? a.partial[m] : 0.0f;
  for (int s = 0; s < kHeadBiasSplits; ++s) v += a.pieces[(int64_t)s * a.M + m];
  if (!span.last) {
    a.partial[m] = v;
  } else {
    if (a.accumulate) v += bf16_one(a.out[m]);
    a.out[m] = one_bf16(v);
  }
}

template <int MF>
hipError_t launch_hidden(const HeadHiddenArgs& a, int64_t rows, hipStream_t stream) {
  using Product = HeadProduct<MF, 8, false, true, false>;
  const int64_t mt = (rows + Product::kTileM - 1) / Product::kTileM, nt = (a.N + Product::kTileN - 1) / Product::kTileN;
  const int64_t blocks = (mt * nt + 7) / 8 * 8 * a.splits;
  if (blocks >= (int64_t)1 << 24) return hipErrorInvalidConfiguration;
  return launch_kernel(head_hidden_kernel<MF, 8>, dim3((unsigned)blocks), dim3(kHeadThreads), 0, stream, a);
}

int hidden_tile_rows(int64_t rows) { return rows <= 64 ? 64 : rows <= 128 ? 128 : 256; }

}  // namespace

int head_hidden_splits(int64_t rows, int32_t K, int32_t N) {
  const int64_t tiles = (rows + hidden_tile_rows(rows) - 1) / hidden_tile_rows(rows) * ((N + 255) / 256);
  const int64_t most = K / 512 > 1 ? K / 512 : 1;  // a piece pays from 16 steps on
  const int64_t fit = 256 / tiles;
  return (int)(fit < 2 ? 1 : fit < most ? fit : most);
}

hipError_t launch_head_hidden(const HeadHiddenArgs& a, int64_t rows, hipStream_t stream) {
  const int tile = hidden_tile_rows(rows);
  const hipError_t e = tile == 64 ? launch_hidden<2>(a, rows, stream) : tile == 128 ? launch_hidden<4>(a, rows, stream) : launch_hidden<8>(a, rows, stream);
  if (e != hipSuccess || a.splits == 1) return e;
  return launch_kernel(head_join_kernel, dim3((unsigned)(rows < 4096 ? rows : 4096)), dim3(256), 0, stream, a);
}

hipError_t launch_head_weight(const HeadWeightArgs& a, hipStream_t stream) {
  const int64_t tiles = (int64_t)((a.M + 255) / 256) * ((a.N + 255) / 256), blocks = (tiles + 7) / 8 * 8;
  if (blocks >= (int64_t)1 << 24) return hipErrorInvalidConfiguration;
  return launch_kernel(head_weight_kernel<8, 8>, dim3((unsigned)blocks), dim3(kHeadThreads), 0, stream, a);
}

hipError_t launch_head_bias(const HeadBiasArgs& a, hipStream_t stream) {
  const hipError_t e = launch_kernel(head_bias_kernel, dim3((unsigned)((a.M + 2047) / 2048), kHeadBiasSplits), dim3(256), 0, stream, a);
  if (e != hipSuccess) return e;
  return launch_kernel(head_bias_join_kernel, dim3((unsigned)((a.M + 255) / 256)), dim3(256), 0, stream, a);
}

}  // namespace npd
