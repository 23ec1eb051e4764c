// Gradients of a head from the gradient G of its logits (or from what the loss keeps in its place: G = scale (row) times e):
// dH = G W, contracted over the vocabulary; dW = G^T H, over the rows; db = column sums of G.
#include "npd_head.hpp"

namespace npd {
namespace {

// four neighbouring columns of a row of N
__device__ __forceinline__ void store_columns(uint16_t* out, int n, int N, const f32x4& v) {
  if (n + 4 <= N) {
    store4(out + n, make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])));
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (n + t < N) out[n + t] = one_bf16(v[t]);
  }
}
// the same of fragments j and j + 1 (columns n and n + 16 of this lane, neighbours' between them): lanes 16 apart exchange halves,
// so that each stores eight neighbouring columns and the four lanes of a row 64 bytes
// (`whole`, the same for the wave: all 32 columns are there)
__device__ __forceinline__ void store_two(uint16_t* out, int n, int N, bool whole, const f32x4& a, const f32x4& b) {
  const uint32_t a0 = pack_bf16(a[0], a[1]), a1 = pack_bf16(a[2], a[3]), b0 = pack_bf16(b[0], b[1]), b1 = pack_bf16(b[2], b[3]);
  const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(a0, b0, false, false));
  const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(a1, b1, false, false));
  const int at = n + (threadIdx.x & 16 ? 12 : 0);
  const uint32_t v[4] = {x[0], y[0], x[1], y[1]};
  if (whole) {
    store8(out + at, make_uint4(v[0], v[1], v[2], v[3]));
  } else {
#pragma unroll
    for (int t = 0; t < 8; ++t)
      if (at + t < N) out[at + t] = (uint16_t)(v[t >> 1] >> (16 * (t & 1)));
  }
}
__device__ __forceinline__ f32x4 load_columns(const uint16_t* in, int n, int N) {
  f32x4 v;
#pragma unroll
  for (int t = 0; t < 4; ++t) v[t] = n + t < N ? bf16_one(in[n + t]) : 0.0f;
  return v;
}

// How many pieces the contraction over K is split into.  A compute unit has one tile at a time, so `tiles` in s pieces take
// ceil(tiles s / 256) rounds of K / s and what a tile costs besides (about 14 steps of 32, of which a step takes 0.8 us); the pieces are written and
// read once more, at about 3.2 bytes per ns.  Measured (MI355X): 130 tiles of 6,554 x 1,152 over 262,144 5.0 ms in one piece, 3.5 in 16.
constexpr int kUnits = 256;
__host__ __device__ inline int hidden_pieces(int tiles, int rows, int K, int N, int most) {
  const int steps = (K + kHeadStep - 1) / kHeadStep;
  const float join = (float)rows * (float)N * (8.0f / 3.2e6f);  // of one piece, in steps
  int best = 1;
  float least = (float)((tiles + kUnits - 1) / kUnits) * (float)(steps + 14);
  for (int s = 2; s <= most && s * 4 <= steps; s += s < 8 ? 1 : s < 16 ? 2 : s < 64 ? 8 : 32) {
    const float t = (float)((tiles * s + kUnits - 1) / kUnits) * ((float)steps / (float)s + 14.0f) + join * (float)s + 9.0f;
    if (t < least) {
      least = t;
      best = s;
    }
  }
  return best;
}
__host__ __device__ inline int pitch4(int n) { return (n + 3) / 4 * 4; }

template <int MF, int NF>
__device__ __forceinline__ int pieces_of(const HeadHiddenArgs& a, int rows) {
  using Product = HeadProduct<MF, NF, false, true, false>;
  const int mt = (rows + Product::kTileM - 1) / Product::kTileM, nt = (a.N + Product::kTileN - 1) / Product::kTileN;
  return hidden_pieces(mt * nt, rows, a.K, a.N, a.most_splits);
}

template <int MF, int NF>
__device__ __forceinline__ void hidden_tile_of(const HeadHiddenArgs& a, unsigned block, char* lds) {
  using Product = HeadProduct<MF, NF, false, true, false>;
  const HeadSpan span = head_span(a.chunk);
  if (!span.there || span.rows == 0) return;
  const int mt = (span.rows + Product::kTileM - 1) / Product::kTileM, nt = (a.N + Product::kTileN - 1) / Product::kTileN;
  const int pieces = hidden_pieces(mt * nt, span.rows, a.K, a.N, a.most_splits);
  const HeadTile tile = head_tile(block, mt, nt, pieces);
  if (!tile.there) return;
  const int split = tile.piece;
  const int64_t m0 = (int64_t)tile.m * Product::kTileM;
  const int n0 = tile.n * Product::kTileN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // pieces of whole rounds of the stages
  constexpr int kRound = kHeadStep * kHeadStages;
  const int rounds = (a.K + kRound - 1) / kRound;
  const int64_t k0 = (int64_t)rounds * split / pieces * kRound, k1 = (int64_t)rounds * (split + 1) / pieces * kRound;
  Product x;
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int j = 0; j < NF; ++j) x.acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  HeadMatrix g = a.g;
  g.rows = span.rows;
  x.start(g, a.w, m0, n0, k0, k1 < a.K ? k1 : a.K, lds);
  x.run(g, a.w, false, 0, 0, 0, 0, lds);
#pragma unroll
  for (int i = 0; i < MF; ++i) {
    const int64_t m = m0 + (wave >> 1) * 16 * MF + 16 * i + (lane & 15);
    if (m >= span.rows) continue;
    const int columns = n0 + (x.wave & 1) * 16 * NF, nw = columns + 4 * (lane >> 4);
    if (pieces > 1) {
      float* out = a.partial + ((int64_t)split * span.rows + m) * pitch4(a.N);
#pragma unroll
      for (int j = 0; j < NF; ++j)
        if (columns + 16 * j + 16 <= a.N || nw + 16 * j < a.N) *reinterpret_cast<f32x4*>(out + nw + 16 * j) = x.acc[i][j];
    } else {
      const float s = a.scale ? a.scale[m] : 1.0f;
      uint16_t* out = a.out + (a.rows ? (int64_t)a.rows[span.first + m] : span.first + m) * a.out_stride;
#pragma unroll
      for (int j = 0; j < NF; j += 2) store_two(out, nw + 16 * j, a.N, columns + 16 * j + 32 <= a.N, x.acc[i][j] * s, x.acc[i][j + 1] * s);
    }
  }
}

template <int MF, int NF>
__global__ __launch_bounds__(kHeadThreads, 1) void head_hidden_kernel(HeadHiddenArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[HeadProduct<MF, NF, false, true, false>::kLds];
  hidden_tile_of<MF, NF>(a, blockIdx.x, lds);
}

// joins the pieces of head_hidden_kernel in their order
template <int MF, int NF>
__global__ __launch_bounds__(256) void head_join_kernel(HeadHiddenArgs a) {
  const HeadSpan span = head_span(a.chunk);
  if (!span.there || span.rows == 0) return;
  const int pieces = pieces_of<MF, NF>(a, span.rows);
  if (pieces == 1) return;
  const int pitch = pitch4(a.N), quads = pitch / 4;
  const int64_t all = (int64_t)span.rows * quads;
  for (int64_t q = blockIdx.x * 256ll + threadIdx.x; q < all; q += gridDim.x * 256ll) {
    const int64_t m = q / quads;
    const int n = (int)(q - m * quads) * 4;
    const float* at = a.partial + m * pitch + n;
    f32x4 v = *reinterpret_cast<const f32x4*>(at);
#pragma unroll 4
    for (int p = 1; p < pieces; ++p) v += *reinterpret_cast<const f32x4*>(at + (int64_t)p * span.rows * pitch);
    const float s = a.scale ? a.scale[m] : 1.0f;
    store_columns(a.out + (a.rows ? (int64_t)a.rows[span.first + m] : span.first + m) * a.out_stride, n, a.N, v * s);
  }
}

// ADD: on top of the chunks before this one.  Whether a chunk is the last one is known on the device: both forms are launched, and
// the one that does not apply ends at once (a kernel of both would hold more still: the sums and the next tile's fragments are 384
// registers).  Of 256 x 256 the first of several chunks spills nothing; one chunk alone 40 registers (41 where it accumulates), a
// middle one 34, the last of several 140 (149): at a tile's beginning and end, the steps are free of it.
// ACCUMULATE reads the old gradient two bytes at a time in a tile's end.  Measured (MI355X, ms, loss with the weights' gradient alone,
// without / with it): 8,192 positions of 151,936 x 2,048 7.97 / 8.53; 20,000 of 151,936 x 1,024 12.18 / 12.61; 512 of 50,048 x 1,024 .160 /
// .293, of 2,048 x 1,024 .035 / .043.
// `block` of `blocks` workgroups that take one tile after the other.
template <int MF, int NF, bool ADD, bool LAST, bool ACCUMULATE>
__device__ __forceinline__ void weight_tiles_of(const HeadWeightArgs& a, unsigned block0, unsigned blocks, char* lds) {
  using Product = HeadProduct<MF, NF, true, true, false>;
  const HeadSpan span = head_span(a.chunk);
  if (!span.there || span.last != LAST) return;
  const int mt = (a.M + Product::kTileM - 1) / Product::kTileM, nt = (a.N + Product::kTileN - 1) / Product::kTileN;
  HeadTile tile = head_tile(block0, mt, nt);
  if (!tile.there) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Product x;
  // rows of the chunk: behind the last one nothing is read
  x.start(a.g, a.h, (int64_t)tile.m * Product::kTileM, (int64_t)tile.n * Product::kTileN, 0, span.rows, lds);
  for (unsigned block = block0 + blocks; tile.there; block += blocks) {
    const HeadTile next = head_tile(block, mt, nt);
    const int64_t m0 = (int64_t)tile.m * Product::kTileM;
    const int n0 = tile.n * Product::kTileN;
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
      for (int j = 0; j < NF; ++j) x.acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    x.run(a.g, a.h, next.there, (int64_t)next.m * Product::kTileM, (int64_t)next.n * Product::kTileN, 0, span.rows, lds);
    tile = next;
    const int64_t mw = m0 + (wave >> 1) * 16 * MF + (lane & 15);
    const int columns = n0 + (x.wave & 1) * 16 * NF, nw = columns + 4 * (lane >> 4);
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      __builtin_amdgcn_sched_barrier(0);  // (a row's sums at a time)
      const int64_t m = mw + 16 * i;
      if (m >= a.M) continue;
      f32x4* partial = reinterpret_cast<f32x4*>(a.partial + m * pitch4(a.N));
      uint16_t* out = a.out + m * a.out_stride;
#pragma unroll
      for (int j = 0; j < NF; j += 2) {
        f32x4 v[2] = {x.acc[i][j], x.acc[i][j + 1]};
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int n = nw + 16 * (j + t);
          if constexpr (ADD) {
            if (columns + 16 * (j + t) + 16 <= a.N || n < a.N) v[t] += partial[n / 4];
          }
          if constexpr (ACCUMULATE) v[t] += load_columns(out, n, a.N);
          if constexpr (!LAST) {
            if (columns + 16 * (j + t) + 16 <= a.N || n < a.N) partial[n / 4] = v[t];
          }
        }
        if constexpr (LAST) store_two(out, nw + 16 * j, a.N, columns + 16 * j + 32 <= a.N, v[0], v[1]);
      }
    }
  }
}

template <int MF, int NF, bool ADD, bool LAST, bool ACCUMULATE>
__global__ __launch_bounds__(kHeadThreads, 1) void head_weight_kernel(HeadWeightArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[HeadProduct<MF, NF, true, true, false>::kLds];
  weight_tiles_of<MF, NF, ADD, LAST, ACCUMULATE>(a, blockIdx.x, gridDim.x, lds);
}

// Both gradients of a small call in one launch: the first `hidden` workgroups (a multiple of eight) have the hidden states'.
template <bool ACCUMULATE>
__global__ __launch_bounds__(kHeadThreads, 1) void head_small_kernel(HeadHiddenArgs h, HeadWeightArgs w, unsigned hidden) {
  constexpr int kLds = HeadProduct<4, 4, false, true, false>::kLds;
  static_assert(kLds == HeadProduct<4, 4, true, true, false>::kLds, "one array for both");
  __shared__ __attribute__((aligned(1024))) char lds[kLds];
  if (blockIdx.x < hidden)
    hidden_tile_of<4, 4>(h, blockIdx.x, lds);
  else
    weight_tiles_of<4, 4, false, true, ACCUMULATE>(w, blockIdx.x - hidden, gridDim.x - hidden, lds);
}

__global__ __launch_bounds__(256) void head_bias_kernel(HeadBiasArgs a) {
  const HeadSpan span = head_span(a.chunk);
  if (!span.there) return;
  const int m = (blockIdx.x * 256 + threadIdx.x) * 8;  // rows of g begin on 16 bytes and are padded to eight
  if (m >= a.M) return;
  const int piece = blockIdx.y;
  const int64_t b = (int64_t)span.rows * piece / kHeadBiasSplits, e = (int64_t)span.rows * (piece + 1) / kHeadBiasSplits;
  float sum[8] = {};
  for (int64_t r = b; r < e; ++r) {
    float x[8];
    unpack8(*reinterpret_cast<const uint4*>(a.g.p + r * a.g.stride + m), x);
    // (a position with a bad label or id has no part in the shared gradients; one that holds a NaN itself makes them NaN)
    const float s = a.scale ? a.scale[r] : 1.0f, w = s != s ? 0.0f : s;
#pragma unroll
    for (int t = 0; t < 8; ++t) sum[t] = __builtin_fmaf(x[t], w, sum[t]);
  }
#pragma unroll
  for (int t = 0; t < 8; ++t)
    if (m + t < a.M) a.pieces[(int64_t)piece * a.M + m + t] = sum[t];
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

template <int MF, int NF>
int64_t hidden_blocks(const HeadHiddenArgs& a, int64_t rows) {
  using Product = HeadProduct<MF, NF, false, true, false>;
  const int64_t mt = (rows + Product::kTileM - 1) / Product::kTileM, nt = (a.N + Product::kTileN - 1) / Product::kTileN;
  // (fewer rows than the most may be split further: tiles and pieces together never need more workgroups than this)
  return (mt * nt + 7) / 8 * 8 * a.most_splits;
}

template <int MF, int NF>
hipError_t launch_join(const HeadHiddenArgs& a, int64_t rows, hipStream_t stream) {
  if (a.most_splits == 1) return hipSuccess;
  const int64_t quads = rows * ((a.N + 3) / 4), join = (quads + 255) / 256;
  return launch_kernel(head_join_kernel<MF, NF>, dim3((unsigned)(join < 8192 ? join : 8192)), dim3(256), 0, stream, a);
}

template <int MF, int NF>
hipError_t launch_hidden(const HeadHiddenArgs& a, int64_t rows, hipStream_t stream) {
  const int64_t blocks = hidden_blocks<MF, NF>(a, rows);
  if (blocks >= (int64_t)1 << 24) return hipErrorInvalidConfiguration;
  const hipError_t e = launch_kernel(head_hidden_kernel<MF, NF>, dim3((unsigned)blocks), dim3(kHeadThreads), 0, stream, a);
  return e == hipSuccess ? launch_join<MF, NF>(a, rows, stream) : e;
}

// rows and columns of a tile for a chunk of up to so many rows
struct HiddenTile {
  int rows, columns;
};
HiddenTile hidden_tile(int64_t rows, int32_t K, int32_t N) {
  // (K: small products are those whose vocabulary is small as well, so that splitting it cannot fill the chip with large tiles)
  if (head_small(rows, N) && K <= 8192) return HiddenTile{128, 128};
  return HiddenTile{rows <= 64 ? 64 : rows <= 128 ? 128 : 256, 256};
}

}  // namespace

int head_hidden_splits(int64_t rows, int32_t K, int32_t N) {
  // the pieces that this many rows are split into, and half as many again for a chunk that turns out to have fewer
  const HiddenTile t = hidden_tile(rows, K, N);
  const int64_t tiles = (rows + t.rows - 1) / t.rows * ((N + t.columns - 1) / t.columns);
  if (tiles > 4 * kUnits) return 1;
  const int s = hidden_pieces((int)tiles, (int)rows, K, N, kUnits);
  return s + s / 2 < 4 ? 4 : s + s / 2;
}

size_t head_hidden_floats(int64_t rows, int32_t N, int splits) { return splits > 1 ? (size_t)splits * rows * pitch4(N) : 0; }

hipError_t launch_head_hidden(const HeadHiddenArgs& a, int64_t rows, hipStream_t stream) {
  const HiddenTile t = hidden_tile(rows, a.K, a.N);
  if (t.columns == 128) return launch_hidden<4, 4>(a, rows, stream);
  return t.rows == 64 ? launch_hidden<2, 8>(a, rows, stream) : t.rows == 128 ? launch_hidden<4, 8>(a, rows, stream) : launch_hidden<8, 8>(a, rows, stream);
}

namespace {

template <int MF, int NF, bool ADD, bool LAST, bool ACCUMULATE>
hipError_t launch_weight(const HeadWeightArgs& a, hipStream_t stream) {
  using Product = HeadProduct<MF, NF, true, true, false>;
  const int64_t mt = (a.M + Product::kTileM - 1) / Product::kTileM, nt = (a.N + Product::kTileN - 1) / Product::kTileN;
  return launch_kernel(head_weight_kernel<MF, NF, ADD, LAST, ACCUMULATE>, dim3(head_grid((mt * nt + 7) / 8 * 8)), dim3(kHeadThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_head_weight(const HeadWeightArgs& a, int64_t chunks, hipStream_t stream) {
  const bool add = a.chunk.index > 0;
  if (chunks > 1) {
    const hipError_t e = add ? launch_weight<8, 8, true, false, false>(a, stream) : launch_weight<8, 8, false, false, false>(a, stream);
    if (e != hipSuccess) return e;
  }
  if (chunks == 1 && head_small(a.M, a.N))
    return a.accumulate ? launch_weight<4, 4, false, true, true>(a, stream) : launch_weight<4, 4, false, true, false>(a, stream);
  if (a.accumulate) return add ? launch_weight<8, 8, true, true, true>(a, stream) : launch_weight<8, 8, false, true, true>(a, stream);
  return add ? launch_weight<8, 8, true, true, false>(a, stream) : launch_weight<8, 8, false, true, false>(a, stream);
}

bool head_both_small(const HeadHiddenArgs& h, const HeadWeightArgs& w, int64_t rows, int64_t chunks) {
  return chunks == 1 && hidden_tile(rows, h.K, h.N).columns == 128 && head_small(w.M, w.N);
}

hipError_t launch_head_both(const HeadHiddenArgs& h, const HeadWeightArgs& w, int64_t rows, hipStream_t stream) {
  using Product = HeadProduct<4, 4, true, true, false>;
  const unsigned hidden = (unsigned)hidden_blocks<4, 4>(h, rows);
  const int64_t mt = (w.M + Product::kTileM - 1) / Product::kTileM, nt = (w.N + Product::kTileN - 1) / Product::kTileN;
  const dim3 grid(hidden + head_grid((mt * nt + 7) / 8 * 8));
  const hipError_t e = w.accumulate ? launch_kernel(head_small_kernel<true>, grid, dim3(kHeadThreads), 0, stream, h, w, hidden)
                                    : launch_kernel(head_small_kernel<false>, grid, dim3(kHeadThreads), 0, stream, h, w, hidden);
  return e == hipSuccess ? launch_join<4, 4>(h, rows, stream) : e;
}

hipError_t launch_head_bias(const HeadBiasArgs& a, hipStream_t stream) {
  const hipError_t e = launch_kernel(head_bias_kernel, dim3((unsigned)((a.M + 2047) / 2048), kHeadBiasSplits), dim3(256), 0, stream, a);
  if (e != hipSuccess) return e;
  return launch_kernel(head_bias_join_kernel, dim3((unsigned)((a.M + 255) / 256)), dim3(256), 0, stream, a);
}

}  // namespace npd
