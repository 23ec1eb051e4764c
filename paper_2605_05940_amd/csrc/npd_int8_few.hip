// Rows to 8-bit integers, and logits of a head in them for up to 64 rows, where reading the weights is all the time: they go straight
// into registers, at any alignment.
#include "npd_int8.hpp"
#include "npd_softcap.hpp"

namespace npd {
namespace {

// ------------------------------------------------------------------------------------------------------- whole numbers

constexpr int kQuantizeThreads = 256;
template <int TH>
constexpr int quantize_block() { return TH < kQuantizeThreads ? kQuantizeThreads : TH; }

// Eight values over the row's largest, times 127, to the nearest whole number.  With the row's exponent taken out (`down`) everything
// below is exact but the quotient; a quotient of 15 and 8 bits that is not half way between two whole numbers is 2^-17 of itself and
// more away from there, so a product with the reciprocal decides wherever it is further from half way than its own error (two
// roundings of up to 127: 2^-16), and the division, rounded correctly, does where it is not: it is exact half way.
__device__ __forceinline__ uint2 quantize8(const uint4& x, int down, float top, float inv) {
  float v[8], n[8];
  unpack8(x, v);
  bool close = false;
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    v[t] = __builtin_ldexpf(v[t], down) * 127.0f;
    const float y = v[t] * inv;
    n[t] = __builtin_rintf(y);
    close |= __builtin_fabsf(y - n[t]) > 0.4999f;
  }
  if (close) {
#pragma unroll
    for (int t = 0; t < 8; ++t) n[t] = __builtin_rintf(v[t] / top);
  }
  uint32_t w[2] = {};
#pragma unroll
  for (int t = 0; t < 8; ++t) w[t >> 2] |= (uint32_t)((int)n[t] & 255) << (8 * (t & 3));
  return make_uint2(w[0], w[1]);
}

// A row lies in the registers of TH threads from its one read.  Bytes bound it: 151,936 x 2,048 172 us (5.4 TB/s, two thirds of them
// reads).
template <int TH, int G>
__global__ __launch_bounds__(quantize_block<TH>()) void quantize_kernel(QuantizeArgs a) {
  __shared__ uint32_t tops[quantize_block<TH>() / kWave];
  constexpr int kRows = quantize_block<TH>() / TH;
  const int at = (threadIdx.x % TH) * 8;
  for (int64_t p = (int64_t)blockIdx.x * kRows + threadIdx.x / TH; p < a.R; p += (int64_t)gridDim.x * kRows) {
    const uint16_t* row = a.x + p * a.x_stride;
    uint4 x[G];
#pragma unroll
    for (int u = 0; u < G; ++u) x[u] = load8_of(row, at + 8 * TH * u, a.D);
    // largest magnitude, as bits: a NaN is above infinity
    uint32_t top = 0;
#pragma unroll
    for (int u = 0; u < G; ++u) {
      const uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const uint32_t lo = w[t] & 0x7fff, hi = w[t] >> 16 & 0x7fff;
        top = top > lo ? top : lo;
        top = top > hi ? top : hi;
      }
    }
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) {
      const uint32_t o = __shfl_xor(top, off, kWave);
      top = top > o ? top : o;
    }
    if constexpr (TH > kWave) {
      __syncthreads();
      if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < TH / kWave; ++w) top = top > tops[w] ? top : tops[w];
    }
    const bool finite = top < 0x7f80;
    const float most = bf16_one((uint16_t)top);
    if (threadIdx.x % TH == 0) a.scale[p] = finite ? most / 127.0f : __builtin_nanf("");
    const int down = top ? -__builtin_amdgcn_frexp_expf(most) : 0;
    const float m = top ? __builtin_ldexpf(most, down) : 1.0f, inv = 1.0f / m;  // (m in [1/2, 1])
    int8_t* q = a.q + p * a.q_stride;
#pragma unroll
    for (int u = 0; u < G; ++u) {
      const int d = at + 8 * TH * u;
      if (d >= a.D) break;
      const uint2 w = finite ? quantize8(x[u], down, m, inv) : make_uint2(0, 0);
      if (d + 8 <= a.D) {
        __builtin_memcpy(q + d, &w, 8);
      } else {
#pragma unroll
        for (int t = 0; t < 8; ++t)
          if (d + t < a.D) q[d + t] = (int8_t)((t < 4 ? w.x : w.y) >> (8 * (t & 3)));
      }
    }
  }
}

template <int TH, int G>
hipError_t launch_rows(const QuantizeArgs& a, hipStream_t stream) {
  constexpr int kRows = quantize_block<TH>() / TH;
  const int64_t blocks = (a.R + kRows - 1) / kRows;
  return launch_kernel(quantize_kernel<TH, G>, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(quantize_block<TH>()), 0, stream, a);
}

// ------------------------------------------------------------------------------------------------------------- products

// sixteen bytes at any address
__device__ __forceinline__ i32x4 load16(const int8_t* p) {
  i32x4 v;
  __builtin_memcpy(&v, p, 16);
  return v;
}
// bytes [d, d + 16) of a row of `cols`, 0 behind its end
__device__ __forceinline__ i32x4 load16_of(const int8_t* row, int d, int cols) {
  if (d + 16 <= cols) return load16(row + d);
  uint32_t w[4] = {};
#pragma unroll
  for (int t = 0; t < 16; ++t)
    if (d + t < cols) w[t >> 2] |= (uint32_t)(uint8_t)row[d + t] << (8 * (t & 3));
  return i32x4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
}

constexpr int kTokenColumns = 32;

// The end of a workgroup's PART columns, whose sums lie in LDS as [row][PART]: a wave per row, PART / 64 columns per lane.
template <int PART>
__device__ __forceinline__ void finish_columns(const Int8Args& a, const int* x) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const SoftCap soft(a.cap != 0.0f ? a.cap : 1.0f);
  constexpr int N = PART < kWave ? 1 : PART / kWave;
  if (PART < kWave && lane >= PART) return;
  const int n = blockIdx.x * PART + N * lane;
  if (n >= a.V) return;
  float scale[N], bias[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const int v = n + e < a.V ? n + e : n;
    scale[e] = a.w_scale[v];
    bias[e] = a.bias ? bf16_one(a.bias[v]) : 0.0f;
  }
  for (int m = wave; m < (int)a.T; m += kHeadThreads / kWave) {
    const float hs = a.h_scale[m];
    float y[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      y[e] = __builtin_fmaf((float)x[m * PART + N * lane + e] * hs, scale[e], bias[e]);
      if (a.cap != 0.0f) y[e] = soft.cap * soft.tanh_of(y[e]);  // uniform
    }
    uint16_t* out = a.out + m * a.out_stride + n;
    if (N == 2 && n + 2 <= a.V) {
      const uint32_t v = pack_bf16(y[0], y[N - 1]);
      __builtin_memcpy(out, &v, 4);
    } else {
      *out = one_bf16(y[0]);
    }
  }
}

// Up to four rows: v_mfma_i32_4x4x4_16b_i8 as 16 pieces of k of the same four columns and four rows, added up at the end, so that one
// load of a wave is 256 consecutive bytes of each of four rows of the weights, read past the caches; the four waves of a workgroup
// have the same 32 columns and every fourth block of k.  The weights' bytes bound it: 151,936 x 2,048 49.3 us (6.3 TB/s).  Workgroups
// begin at different places of their rows and wrap around (rows of a power of two of bytes would else be read out of few memory
// channels).
__global__ __launch_bounds__(kHeadThreads, 4) void int8_tokens_kernel(Int8Args a) {
  constexpr int kWaves = kHeadThreads / kWave, G = 8;
  constexpr int kBlock = 256;  // bytes of k per load
  __shared__ __attribute__((aligned(16))) int x[kWaves][4][kTokenColumns];
  static_assert(kTokenColumns == 4 * G && 4 * kTokenColumns <= kHeadThreads, "a thread per sum");
  typedef int words __attribute__((ext_vector_type(4), aligned(1)));
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 3, b = lane >> 2;
  const int blocks = a.D / kBlock, tail = blocks * kBlock + 16 * b;
  const int mine = (blocks - wave + kWaves - 1) / kWaves;  // blocks wave, wave + 4 ..
  const int8_t* h = a.h + (i < a.T ? i : a.T - 1) * a.h_stride;
  const int8_t* w[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int v = blockIdx.x * kTokenColumns + 4 * g + i;
    w[g] = a.w + (int64_t)(v < a.V ? v : a.V - 1) * a.w_stride;
  }
  i32x4 acc[G];
#pragma unroll
  for (int g = 0; g < G; ++g) acc[g] = i32x4{0, 0, 0, 0};
  auto multiply = [&](const i32x4 (&wv)[G], const i32x4& hv) {
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[g] = __builtin_amdgcn_mfma_i32_4x4x4i8(wv[g][e], hv[e], acc[g], 0, 0, 0);
  };
  int at = mine > 0 ? (int)((blockIdx.x * 4 + wave) % (unsigned)mine) : 0;
  for (int n = 0; n < mine; ++n) {
    const int d = (wave + at * kWaves) * kBlock + 16 * b;
    at = at + 1 == mine ? 0 : at + 1;
    i32x4 wv[G];
#pragma unroll
    for (int g = 0; g < G; ++g) wv[g] = __builtin_nontemporal_load(reinterpret_cast<const words*>(w[g] + d));
    const i32x4 hv = load16(h + d);
    __builtin_amdgcn_sched_barrier(0);  // (all requested before the first is waited for: 151,936 x 2,048 52.4 us, in the compiler's order 56.3)
    multiply(wv, hv);
  }
  if (tail - 16 * b < a.D && wave == kWaves - 1) {  // uniform (the last wave has the fewest blocks)
    i32x4 wv[G];
#pragma unroll
    for (int g = 0; g < G; ++g) wv[g] = load16_of(w[g], tail, a.D);
    multiply(wv, load16_of(h, tail, a.D));
  }
  // acc[g][e] of lane (b, i): column 4 g + e, row i, piece b of k
#pragma unroll
  for (int g = 0; g < G; ++g) {
#pragma unroll
    for (int off = 4; off < kWave; off <<= 1)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[g][e] += __shfl_xor(acc[g][e], off, kWave);
    if (b == g) *reinterpret_cast<i32x4*>(&x[wave][i][4 * g]) = acc[g];
  }
  __syncthreads();
  const int t = threadIdx.x;
  if (t < 4 * kTokenColumns) {
    int* sum = &x[0][0][0] + t;
#pragma unroll
    for (int u = 1; u < kWaves; ++u) *sum += sum[u * 4 * kTokenColumns];
  }
  __syncthreads();
  finish_columns<kTokenColumns>(a, &x[0][0][0]);
}

// Up to 16 RT rows: a wave reads the weights of 16 FC columns straight into the fragments of 16 x 16 x 64 products, 64 bytes of 16
// rows per load, 256 of each at a time; the hidden states go through LDS, 256 bytes of all rows at a time.  9 rows of 151,936 x 2,048
// take 60 us (5.2 TB/s), of 50,048 x 1,024 12.0.
template <int RT, int FC>
__global__ __launch_bounds__(kHeadThreads, 3) void int8_few_kernel(Int8Args a) {
  constexpr int kPart = 64 * FC;  // columns of the workgroup
  constexpr int kBlock = 256, kStep = 64, kSteps = kBlock / kStep;
  constexpr int kPitch = kBlock + 16;  // (rows 17 groups of 16 bytes apart: 16 rows' reads lie in 16 different ones of 256 bytes)
  __shared__ __attribute__((aligned(16))) union {
    int8_t h[2][16 * RT][kPitch];
    int x[16 * RT][kPart];
  } lds;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
  const int v0 = blockIdx.x * kPart + wave * 16 * FC;
  const int8_t* w[FC];
#pragma unroll
  for (int f = 0; f < FC; ++f) {
    const int v = v0 + 16 * f + i;
    w[f] = a.w + (int64_t)(v < a.V ? v : a.V - 1) * a.w_stride;
  }
  // this thread's share of a block of the hidden states: group threadIdx.x % 16 of rows threadIdx.x / 16 + 16 t
  const int hg = threadIdx.x & 15;
  const int8_t* h[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int m = 16 * t + (threadIdx.x >> 4);
    h[t] = a.h + (m < a.T ? m : a.T - 1) * a.h_stride;
  }
  i32x4 acc[FC][RT];
#pragma unroll
  for (int f = 0; f < FC; ++f)
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[f][t] = i32x4{0, 0, 0, 0};
  const int whole = a.D / kBlock, blocks = (a.D + kBlock - 1) / kBlock;
  int at = whole ? (int)((blockIdx.x * 5) % (unsigned)whole) : 0;  // (where the workgroup begins, see above)
  i32x4 hv[RT];
  auto request = [&](int block) {
#pragma unroll
    for (int t = 0; t < RT; ++t)
      hv[t] = block >= whole ? load16_of(h[t], block * kBlock + 16 * hg, a.D) : load16(h[t] + block * kBlock + 16 * hg);
  };
  request(whole ? at : 0);
  for (int n = 0; n < blocks; ++n) {
    const int block = n < whole ? at : whole;
    if (n < whole) at = at + 1 == whole ? 0 : at + 1;
    i32x4 wv[kSteps][FC];
    const int d = block * kBlock + 16 * g;
    if (block < whole) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int f = 0; f < FC; ++f) wv[s][f] = load16(w[f] + d + s * kStep);
    } else {
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int f = 0; f < FC; ++f) wv[s][f] = load16_of(w[f], d + s * kStep, a.D);
    }
    // (two buffers: what is written here was last read before the barrier of the block before)
#pragma unroll
    for (int t = 0; t < RT; ++t) *reinterpret_cast<i32x4*>(&lds.h[n & 1][16 * t + (threadIdx.x >> 4)][16 * hg]) = hv[t];
    __syncthreads();
    if (n + 1 < blocks) request(n + 1 < whole ? at : whole);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const i32x4 y = *reinterpret_cast<const i32x4*>(&lds.h[n & 1][16 * t + i][16 * g + s * kStep]);
#pragma unroll
        for (int f = 0; f < FC; ++f) acc[f][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[s][f], y, acc[f][t], 0, 0, 0);
      }
    }
  }
  __syncthreads();
  // acc[f][t][e]: row 16 t + i, column v0 + 16 f + 4 g + e
#pragma unroll
  for (int f = 0; f < FC; ++f)
#pragma unroll
    for (int t = 0; t < RT; ++t) *reinterpret_cast<i32x4*>(&lds.x[16 * t + i][wave * 16 * FC + 16 * f + 4 * g]) = acc[f][t];
  __syncthreads();
  finish_columns<kPart>(a, &lds.x[0][0]);
}

// A wave has four rows, of either matrix, whose loads are requested together.  The last bytes of a row come with those before them, and
// are moved to their place (byte by byte behind a branch they take as long as all others).  50,336 rows of 1,000 bytes 18.7 us (5.4
// TB/s; a row at a time and two launches 24).
constexpr int kPackThreads = 256, kPackRows = 4;
__global__ __launch_bounds__(kPackThreads) void int8_pack_kernel(Int8Packed first, Int8Packed second, int32_t to_width, int32_t cols) {
  const int64_t rows = first.rows + second.rows, step = (int64_t)gridDim.x * (kPackThreads / kWave) * kPackRows;
  for (int64_t r = ((int64_t)blockIdx.x * (kPackThreads / kWave) + (threadIdx.x >> 6)) * kPackRows; r < rows; r += step)
    for (int d = (threadIdx.x & 63) * 16; d < to_width; d += kWave * 16) {
      const int at = d + 16 <= cols ? d : cols - 16, behind = d - at;  // (behind: bytes that another lane has, 15 at most)
      i32x4 v[kPackRows];
      int8_t* to[kPackRows];
#pragma unroll
      for (int u = 0; u < kPackRows; ++u) {
        const int64_t p = r + u < rows ? r + u : rows - 1;
        const bool of_first = p < first.rows;
        const int8_t* from = of_first ? first.from + p * first.stride : second.from + (p - first.rows) * second.stride;
        to[u] = (of_first ? first.to + p * to_width : second.to + (p - first.rows) * to_width) + d;
        v[u] = cols >= 16 ? load16(from + at) : load16_of(from, d, cols);  // uniform
      }
#pragma unroll
      for (int u = 0; u < kPackRows; ++u) {
        if (cols >= 16 && behind > 0) v[u] = __builtin_bit_cast(i32x4, __builtin_bit_cast(unsigned __int128, v[u]) >> (8 * behind));
        if (r + u < rows) *reinterpret_cast<i32x4*>(to[u]) = v[u];
      }
    }
}

template <int RT>
hipError_t launch_fragments(const Int8Args& a, hipStream_t stream) {
  // (64 columns to a workgroup where 128 leave compute units without one: 9 rows of 32,000 x 4,096 24 us, 33 with 128; of 50,048 x 1,024
  // 13.8 / 12.0)
  const bool narrow = a.V < 256 * 128;
  const int columns = narrow ? 64 : 128;
  return launch_kernel(narrow ? int8_few_kernel<RT, 1> : int8_few_kernel<RT, 2>, dim3((unsigned)((a.V + (int64_t)columns - 1) / columns)),
                       dim3(kHeadThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_quantize(const QuantizeArgs& a, hipStream_t stream) {
  if (a.D <= 512) return launch_rows<64, 1>(a, stream);
  if (a.D <= 1024) return launch_rows<64, 2>(a, stream);
  if (a.D <= 2048) return launch_rows<64, 4>(a, stream);
  if (a.D <= 4096) return launch_rows<256, 2>(a, stream);
  if (a.D <= 8192) return launch_rows<256, 4>(a, stream);
  if (a.D <= 16384) return launch_rows<1024, 2>(a, stream);
  if (a.D <= 32768) return launch_rows<1024, 4>(a, stream);
  return launch_rows<1024, 8>(a, stream);
}

hipError_t launch_int8_few(const Int8Args& a, hipStream_t stream) {
  // Up to four rows of 1,536 and more bytes are int8_tokens_kernel's, whose waves share a row.  Measured (MI355X, us, one row there / in
  // int8_few_kernel, weights out of the caches): 8,000 x 1,024 6.1 / 4.9 (1,000 entries), 8,000 x 1,536 7.0 / 7.8, 8,000 x 8,192 15.3 / 39.7,
  // 32,000 x 2,048 15.4 / 13.7, 50,048 x 2,048 22.1 / 20.0, 100,000 x 2,048 38.2 / 43.9, 151,936 x 1,024 35.4 / 30.4, x 1,536 40.6 / 44.2, x
  // 2,048 53 / 60, 262,144 x 1,152 82.5 / 56.8.  (The width alone decides: 32,000 to 50,000 entries of 2,048 are 10 to 12 % slower so.)
  // Eight rows in two of its products at once are slower (100,000 x 2,048 70 / 46).
  if (a.T <= 4 && a.D >= 1536)
    return launch_kernel(int8_tokens_kernel, dim3((unsigned)((a.V + (int64_t)kTokenColumns - 1) / kTokenColumns)), dim3(kHeadThreads), 0, stream, a);
  if (a.T <= 16) return launch_fragments<1>(a, stream);
  if (a.T <= 32) return launch_fragments<2>(a, stream);
  if (a.T <= 48) return launch_fragments<3>(a, stream);
  return launch_fragments<4>(a, stream);
}

hipError_t launch_int8_pack(const Int8Packed& first, const Int8Packed& second, int32_t to_width, int32_t cols, hipStream_t stream) {
  constexpr int kRows = kPackThreads / kWave * kPackRows;
  const int64_t blocks = (first.rows + second.rows + kRows - 1) / kRows;
  return launch_kernel(int8_pack_kernel, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(kPackThreads), 0, stream, first, second,
                       to_width, cols);
}

}  // namespace npd
