// Logits of a head and the sums of their softmax: x = h W^T (+ bias, soft cap) in the matrix cores, and what becomes of a tile before it
// leaves the registers.  Workgroups take one tile of 256 x 256 after the other (128 x 256 for up to 128 rows, 128 x 128 in small calls);
// up to 64 rows have kernels of their own, which read the weights straight into registers.
//
// The sums of a row are taken against a reference r: sum 2^(x c - r).  r is the row's own r0 (a true logit of the row, its label's as a rule,
// rounded to a whole number), so that one pass suffices and what is kept of different tiles fits together; only 128 columns whose largest
// logit lies 2^40 and more above it take that one, rounded, instead.  References are whole numbers: bringing two together is exact.
// What is kept is rounded to bf16, as an operand of the gradients' matrix products: half a step of the probability whatever the logit's
// size, in half the bytes of fp32 (2.5 GB for 8,192 rows of 151,936).
#include "npd_head.hpp"
#include "npd_softcap.hpp"

namespace npd {
namespace {

constexpr float kHeadHeadroom = 40.0f;  // log2

template <int MF, int NF, HeadForward WHAT, bool CAP>
__global__ __launch_bounds__(kHeadThreads, 1) void head_forward_kernel(HeadForwardArgs a) {
  using Product = HeadProduct<MF, NF, false, false, true>;
  constexpr int kPart = 16 * NF;  // a wave's columns are one partial sum
  __shared__ __attribute__((aligned(1024))) char lds[Product::kLds];
  const HeadSpan span = head_span(a.chunk);
  if (!span.there || span.rows == 0) return;
  const int mt = (span.rows + Product::kTileM - 1) / Product::kTileM, nt = (a.V + Product::kTileN - 1) / Product::kTileN;
  HeadTile tile = head_tile(blockIdx.x, mt, nt);
  if (!tile.there) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  HeadMatrix q = a.q;
  q.rows = span.rows;
  Product x;
  x.start(q, a.w, (int64_t)tile.m * Product::kTileM, (int64_t)tile.n * Product::kTileN, 0, a.K, lds);
  for (unsigned block = blockIdx.x + gridDim.x; tile.there; block += gridDim.x) {
    const HeadTile next = head_tile(block, mt, nt);
    const int64_t m0 = (int64_t)tile.m * Product::kTileM;
    const int n0 = tile.n * Product::kTileN;
    const int64_t mw = m0 + (wave >> 1) * 16 * MF + (lane & 15);  // + 16 i
    const int columns = n0 + (x.wave & 1) * 16 * NF;              // of the wave
    const int nw = columns + 8 * (lane >> 4);                     // + 32 j + 0 .. 7, fragments 2 j and 2 j + 1
#pragma unroll
    for (int j = 0; j < NF; ++j) {
      f32x4 b = {0.0f, 0.0f, 0.0f, 0.0f};
      if (a.bias) {
        const int n = nw + 32 * (j >> 1) + 4 * (j & 1);
#pragma unroll
        for (int t = 0; t < 4; ++t) b[t] = n + t < a.V ? bf16_one(a.bias[n + t]) : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < MF; ++i) x.acc[i][j] = b;
    }
    float r0[MF];  // (requested here: there is no time to wait for them once the products are done)
    if constexpr (WHAT != kHeadLogits) {
#pragma unroll
      for (int i = 0; i < MF; ++i) r0[i] = a.r0[mw + 16 * i < span.rows ? mw + 16 * i : 0];
    }
    x.run(q, a.w, next.there, (int64_t)next.m * Product::kTileM, (int64_t)next.n * Product::kTileN, 0, a.K, lds);
    tile = next;

    const SoftCap soft(CAP ? a.cap : 1.0f);
    const float c = CAP ? a.cap * a.c : a.c;
    const bool edge = n0 + Product::kTileN > a.V;  // uniform
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      __builtin_amdgcn_sched_barrier(0);  // (a row's sums at a time: the fragments of the next tile are in registers already)
      const int64_t m = mw + 16 * i;
      const bool row = m < span.rows;
      if constexpr (WHAT == kHeadLogits) {
        uint16_t* out = a.out + (row ? m : 0) * a.out_stride;
#pragma unroll
        for (int j = 0; j < NF; j += 2) {
          const int n = nw + 16 * j;
          uint32_t v[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            float lo = x.acc[i][j + (t >> 1)][2 * (t & 1)], hi = x.acc[i][j + (t >> 1)][2 * (t & 1) + 1];
            if constexpr (CAP) {
              lo = soft.cap * soft.tanh_of(lo);
              hi = soft.cap * soft.tanh_of(hi);
            }
            v[t] = pack_bf16(lo, hi);
          }
          if (!row) continue;
          if (columns + 16 * j + 32 <= a.V) {
            stream8(out + n, make_uint4(v[0], v[1], v[2], v[3]));
          } else {
#pragma unroll
            for (int t = 0; t < 8; ++t)
              if (n + t < a.V) out[n + t] = (uint16_t)(v[t >> 1] >> (16 * (t & 1)));
          }
        }
      } else {
        // logits, or with a soft cap their tanh: that times cap is the logit, and one less its square the slope
        float v[4 * NF];
        float top = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
          for (int t = 0; t < 4; ++t) v[4 * j + t] = CAP ? soft.tanh_of(x.acc[i][j][t]) : x.acc[i][j][t];
        if (edge) {  // columns that are not there: e is 0 however small c is, and so is the slope
#pragma unroll
          for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int t = 0; t < 4; ++t)
              if (nw + 32 * (j >> 1) + 4 * (j & 1) + t >= a.V) v[4 * j + t] = -__builtin_inff();
        }
#pragma unroll
        for (int p = 0; p < 4 * NF; p += 2) top = max3(top, v[p], v[p + 1]);
        top = fmaxf(top, __shfl_xor(top, 16, kWave));
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        const float u = top * c;
        const float r = u > r0[i] + kHeadHeadroom ? __builtin_rintf(u) : r0[i];
        float z = 0.0f;
        uint16_t* e = WHAT == kHeadSumsKept ? a.e + (row ? m : 0) * a.e_stride : nullptr;
#pragma unroll
        for (int j = 0; j < NF; j += 2) {
          uint32_t w[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const int p = 4 * j + 2 * t;
            float lo = exp2_fast(__builtin_fmaf(v[p], c, -r)), hi = exp2_fast(__builtin_fmaf(v[p + 1], c, -r));
            z += lo;
            z += hi;
            if constexpr (CAP && WHAT == kHeadSumsKept) {
              lo *= __builtin_amdgcn_fmed3f(__builtin_fmaf(-v[p], v[p], 1.0f), 0.0f, 1.0f);
              hi *= __builtin_amdgcn_fmed3f(__builtin_fmaf(-v[p + 1], v[p + 1], 1.0f), 0.0f, 1.0f);
            }
            if constexpr (WHAT == kHeadSumsKept) w[t] = pack_bf16(lo, hi);
          }
          if constexpr (WHAT == kHeadSumsKept) {
            const int n = nw + 16 * j;
            // (rows of e begin on 16 bytes, n is a multiple of 8)
            if (row && (columns + 16 * j + 32 <= a.V || n < a.e_stride)) stream8(e + n, make_uint4(w[0], w[1], w[2], w[3]));
          }
        }
        z += __shfl_xor(z, 16, kWave);
        z += __shfl_xor(z, 32, kWave);
        const int part = columns / kPart;
        if (lane < 16 && row && part < a.parts) a.part[m * a.parts + part] = make_float2(r, z);
      }
    }
  }
}

// The end of a workgroup's PART columns of up to 64 rows, which lie in LDS as [row][PART]: a wave per row, PART / 64 columns per
// lane (of 32, half the lanes have one).
template <HeadForward WHAT, bool CAP, int PART>
__device__ __forceinline__ void finish_columns(const HeadForwardArgs& a, const float* x, int rows) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const SoftCap soft(CAP ? a.cap : 1.0f);
  constexpr int N = PART < kWave ? 1 : PART / kWave;
  const bool there = PART >= kWave || lane < PART;
  const int n = there ? blockIdx.x * PART + N * lane : a.V, at = there ? N * lane : 0;
  float bias[N] = {};
  if (a.bias) {
#pragma unroll
    for (int e = 0; e < N; ++e) bias[e] = n + e < a.V ? bf16_one(a.bias[n + e]) : 0.0f;
  }
  for (int m = wave; m < rows; m += kHeadThreads / kWave) {
    float y[N], slope[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      y[e] = x[m * PART + at + e] + bias[e];
      slope[e] = 1.0f;
      if constexpr (CAP) {
        const float th = soft.tanh_of(y[e]);
        y[e] = soft.cap * th;
        slope[e] = __builtin_fmaf(-th, th, 1.0f);
      }
    }
    if constexpr (WHAT == kHeadLogits) {
      uint16_t* out = a.out + m * a.out_stride + n;
      if (N == 2 && n + 2 <= a.V) {
        const uint32_t v = pack_bf16(y[0], y[N - 1]);
        __builtin_memcpy(out, &v, 4);
      } else if (n < a.V) {
        *out = one_bf16(y[0]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (n + e >= a.V) y[e] = -__builtin_inff();
      float top = fmaxf(y[0], y[N - 1]);
#pragma unroll
      for (int off = kWave / 2; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, kWave));
      const float r0 = a.r0[m], u = top * a.c;
      const float r = u > r0 + kHeadHeadroom ? __builtin_rintf(u) : r0;
      float g[N], z = 0.0f;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        g[e] = exp2_fast(__builtin_fmaf(y[e], a.c, -r));
        z += g[e];
        g[e] *= slope[e];
      }
      z = wave_sum(z);
      if constexpr (WHAT == kHeadSumsKept) {
        // (a part's columns end within the row: its pitch is a multiple of 64 that covers V)
        uint16_t* e = a.e + m * a.e_stride + n;
        if (there && n < a.e_stride) {
          if constexpr (N == 2)
            *reinterpret_cast<uint32_t*>(e) = pack_bf16(g[0], g[1]);
          else
            *e = one_bf16(g[0]);
        }
      }
      if (lane == 0) a.part[(int64_t)m * a.parts + blockIdx.x] = make_float2(r, z);
    }
  }
}

// Up to 4 NT rows, where reading the weights is all the time.  v_mfma_f32_4x4x4_16b_bf16 is 16 products of 4 x 4 at once; here they
// are 16 pieces of k of the same four columns and four rows, added up at the end, so that one load of a wave is 256 consecutive
// bytes of each of four rows of the weights.  That is what decides: reading 151,936 x 2,048 alone (MI355X) takes 126 us in pieces of 64 bytes
// of 16 rows, 105 in pieces of 256 of four, 91 if the caches are told that nothing is read twice, as here; waves begin at
// different places of their rows and wrap around, since rows of a power of two of bytes would else be read out of few memory
// channels (126 us: 145).
//
// PART 128: a wave has 32 columns of its own.  32: the four waves have the same ones and every fourth block of k, added up at the end.
// TOGETHER: a block's loads are all requested before the first is waited for, and not in the compiler's order; see head_together().
template <int NT, int PART, bool TOGETHER, HeadForward WHAT, bool CAP>
__global__ __launch_bounds__(kHeadThreads, NT == 1 ? 5 : 4) void head_tokens_kernel(HeadForwardArgs a) {
  constexpr int kWaves = kHeadThreads / kWave, G = 8, kShare = PART == 4 * G ? kWaves : 1;
  static_assert(PART == 4 * G * kWaves / kShare, "");
  __shared__ __attribute__((aligned(16))) float x[kShare][4 * NT][PART];
  const HeadSpan span = head_span(a.chunk);
  if (span.rows == 0) return;
  typedef uint32_t words __attribute__((ext_vector_type(4), aligned(2)));
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 3, b = lane >> 2;
  constexpr int kBlock = 128;  // values of k per load
  const int blocks = a.D / kBlock, tail = blocks * kBlock + 8 * b;
  const int first = kShare > 1 ? wave : 0, mine = (blocks - first + kShare - 1) / kShare;  // blocks first, first + kShare ..
  const int c0 = kShare > 1 ? 0 : wave * 4 * G;  // of the workgroup's columns
  const uint16_t *h[NT], *w[G];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int m = 4 * t + i;
    h[t] = a.q.p + (int64_t)(m < span.rows ? m : span.rows - 1) * a.q.stride;
  }
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int v = blockIdx.x * PART + c0 + 4 * g + i;
    w[g] = a.w.p + (int64_t)(v < a.V ? v : a.V - 1) * a.w.stride;
  }
  f32x4 acc[G][NT];
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[g][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  auto multiply = [&](const uint4 (&wv)[G], const uint4 (&hv)[NT]) {
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        acc[g][t] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(__builtin_bit_cast(s16x4, make_uint2(wv[g].x, wv[g].y)),
                                                           __builtin_bit_cast(s16x4, make_uint2(hv[t].x, hv[t].y)), acc[g][t], 0, 0, 0);
        acc[g][t] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(__builtin_bit_cast(s16x4, make_uint2(wv[g].z, wv[g].w)),
                                                           __builtin_bit_cast(s16x4, make_uint2(hv[t].z, hv[t].w)), acc[g][t], 0, 0, 0);
      }
  };
  int at = mine > 0 ? (int)((blockIdx.x * 4 + wave) % (unsigned)mine) : 0;
  for (int n = 0; n < mine; ++n) {
    const int d = (first + at * kShare) * kBlock + 8 * b;
    at = at + 1 == mine ? 0 : at + 1;
    uint4 wv[G], hv[NT];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const words v = __builtin_nontemporal_load(reinterpret_cast<const words*>(w[g] + d));
      wv[g] = make_uint4(v[0], v[1], v[2], v[3]);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) hv[t] = load8(h[t] + d);
    if constexpr (TOGETHER) __builtin_amdgcn_sched_barrier(0);
    multiply(wv, hv);
  }
  if (tail - 8 * b < a.D && (kShare == 1 || wave == kWaves - 1)) {  // uniform (the last wave has the fewest blocks)
    uint4 wv[G], hv[NT];
#pragma unroll
    for (int g = 0; g < G; ++g) wv[g] = load8_of(w[g], tail, a.D);
#pragma unroll
    for (int t = 0; t < NT; ++t) hv[t] = load8_of(h[t], tail, a.D);
    multiply(wv, hv);
  }
  // acc[g][t][e] of lane (b, i): column 4 g + e, row 4 t + i, piece b of k
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int off = 4; off < kWave; off <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[g][t][e] += __shfl_xor(acc[g][t][e], off, kWave);
      if (b == g) *reinterpret_cast<f32x4*>(&x[kShare > 1 ? wave : 0][4 * t + i][c0 + 4 * g]) = acc[g][t];
    }
  __syncthreads();
  if constexpr (kShare > 1) {
    static_assert(4 * NT * PART <= kHeadThreads, "a thread per sum");
    const int t = threadIdx.x;
    if (t < 4 * NT * PART) {
      float* sum = &x[0][0][0] + t;
#pragma unroll
      for (int u = 1; u < kShare; ++u) *sum += sum[u * 4 * NT * PART];
    }
    __syncthreads();
  }
  finish_columns<WHAT, CAP, PART>(a, &x[0][0][0], span.rows);
}

// The same for up to 16 RT rows: a wave reads the weights of 16 FC columns straight into the fragments of 16 x 16 x 32 products (64
// bytes of 16 rows per load, the next 64 with the one after it: 5 TB/s), 4 FC KB at a time; the hidden states go through LDS, 128
// values of k of all rows at a time, so that a compute unit reads them once and not once per wave.
template <int RT, int FC, bool ODD, HeadForward WHAT, bool CAP>
__global__ __launch_bounds__(kHeadThreads, 3) void head_few_kernel(HeadForwardArgs a) {
  constexpr int kPart = 64 * FC;  // columns of the workgroup
  constexpr int kBlock = 128, kSteps = kBlock / kHeadStep;
  constexpr int kPitch = kBlock + 8;  // (rows 17 groups of 16 bytes apart: 16 rows' reads lie in 16 different ones of 256 bytes)
  __shared__ __attribute__((aligned(16))) union {
    uint16_t h[2][16 * RT][kPitch];
    float x[16 * RT][kPart];
  } lds;
  const HeadSpan span = head_span(a.chunk);
  if (span.rows == 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
  const int v0 = blockIdx.x * kPart + wave * 16 * FC;
  const uint16_t* w[FC];
#pragma unroll
  for (int f = 0; f < FC; ++f) {
    const int v = v0 + 16 * f + i;
    w[f] = a.w.p + (int64_t)(v < a.V ? v : a.V - 1) * a.w.stride;
  }
  // this thread's share of a block of the hidden states: group threadIdx.x % 16 of rows threadIdx.x / 16 + 16 t
  const int hg = threadIdx.x & 15;
  const uint16_t* h[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int m = 16 * t + (threadIdx.x >> 4);
    h[t] = a.q.p + (int64_t)(m < span.rows ? m : span.rows - 1) * a.q.stride;
  }
  f32x4 acc[FC][RT];
#pragma unroll
  for (int f = 0; f < FC; ++f)
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[f][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int whole = a.D / kBlock, blocks = (a.D + kBlock - 1) / kBlock;
  int at = whole ? (int)((blockIdx.x * 5) % (unsigned)whole) : 0;  // (where the workgroup begins, see above)
  uint4 hv[RT];
  auto request = [&](int block) {
#pragma unroll
    for (int t = 0; t < RT; ++t)
      hv[t] = block >= whole ? load8_of<ODD>(h[t], block * kBlock + 8 * hg, a.D)
              : ODD          ? load8_odd(h[t] + block * kBlock + 8 * hg)
                             : load8(h[t] + block * kBlock + 8 * hg);
  };
  request(whole ? at : 0);
  for (int n = 0; n < blocks; ++n) {
    const int block = n < whole ? at : whole;
    if (n < whole) at = at + 1 == whole ? 0 : at + 1;
    bf16x8 wv[kSteps][FC];
    const int d = block * kBlock + 8 * g;
    if (block < whole) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int f = 0; f < FC; ++f) {
          const uint16_t* p = w[f] + d + s * kHeadStep;
          wv[s][f] = __builtin_bit_cast(bf16x8, ODD ? load8_odd(p) : load8(p));
        }
    } else {
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int f = 0; f < FC; ++f) wv[s][f] = __builtin_bit_cast(bf16x8, load8_of<ODD>(w[f], d + s * kHeadStep, a.D));
    }
    // (two buffers: what is written here was last read before the barrier of the block before)
#pragma unroll
    for (int t = 0; t < RT; ++t) *reinterpret_cast<uint4*>(&lds.h[n & 1][16 * t + (threadIdx.x >> 4)][8 * hg]) = hv[t];
    __syncthreads();
    if (n + 1 < blocks) request(n + 1 < whole ? at : whole);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const bf16x8 y = *reinterpret_cast<const bf16x8*>(&lds.h[n & 1][16 * t + i][8 * g + s * kHeadStep]);
#pragma unroll
        for (int f = 0; f < FC; ++f) acc[f][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[s][f], y, acc[f][t], 0, 0, 0);
      }
    }
  }
  __syncthreads();
  // acc[f][t][e]: row 16 t + i, column v0 + 16 f + 4 g + e
#pragma unroll
  for (int f = 0; f < FC; ++f)
#pragma unroll
    for (int t = 0; t < RT; ++t) *reinterpret_cast<f32x4*>(&lds.x[16 * t + i][wave * 16 * FC + 16 * f + 4 * g]) = acc[f][t];
  __syncthreads();
  finish_columns<WHAT, CAP, kPart>(a, &lds.x[0][0], span.rows);
}

template <int RT, HeadForward WHAT, bool CAP>
hipError_t launch_fragments(const HeadForwardArgs& a, unsigned grid, bool odd, hipStream_t stream) {
  const dim3 g(grid), block(kHeadThreads);
  if (odd) return launch_kernel(head_few_kernel<RT, 1, true, WHAT, CAP>, g, block, 0, stream, a);
  return launch_kernel(a.part_columns == kHeadSmallPart ? head_few_kernel<RT, 1, false, WHAT, CAP> : head_few_kernel<RT, 2, false, WHAT, CAP>, g, block,
                       0, stream, a);
}

template <HeadForward WHAT, bool CAP>
hipError_t launch_few(const HeadForwardArgs& a, int64_t rows, hipStream_t stream) {
  const unsigned grid = (unsigned)a.parts;
  if (a.tokens) {
    const bool share = a.part_columns == kHeadTokensPart;
    const dim3 g(grid), block(kHeadThreads);
    if (rows > 4)
      return launch_kernel(share ? head_tokens_kernel<2, kHeadTokensPart, false, WHAT, CAP> : head_tokens_kernel<2, kHeadPart, false, WHAT, CAP>, g,
                           block, 0, stream, a);
    if (share) return launch_kernel(head_tokens_kernel<1, kHeadTokensPart, true, WHAT, CAP>, g, block, 0, stream, a);
    return launch_kernel(head_together(a.parts) ? head_tokens_kernel<1, kHeadPart, true, WHAT, CAP> : head_tokens_kernel<1, kHeadPart, false, WHAT, CAP>,
                         g, block, 0, stream, a);
  }
  // load8_odd() where rows of the weights begin on odd values and both matrices on four bytes (parts of 64 columns, see head_few_part())
  const bool odd = a.w.stride % 2 != 0 && a.part_columns == kHeadSmallPart && ((uintptr_t)a.w.p | (uintptr_t)a.q.p) % 4 == 0;
  if (rows <= 16) return launch_fragments<1, WHAT, CAP>(a, grid, odd, stream);
  if (rows <= 32) return launch_fragments<2, WHAT, CAP>(a, grid, odd, stream);
  if (rows <= 48) return launch_fragments<3, WHAT, CAP>(a, grid, odd, stream);
  return launch_fragments<4, WHAT, CAP>(a, grid, odd, stream);
}

template <int MF, int NF, HeadForward WHAT, bool CAP>
hipError_t launch(const HeadForwardArgs& a, int64_t rows, hipStream_t stream) {
  using Product = HeadProduct<MF, NF, false, false, true>;
  const int64_t mt = (rows + Product::kTileM - 1) / Product::kTileM, nt = (a.V + Product::kTileN - 1) / Product::kTileN;
  const int64_t blocks = (mt * nt + 7) / 8 * 8;
  if (blocks >= (int64_t)1 << 30) return hipErrorInvalidConfiguration;
  return launch_kernel(head_forward_kernel<MF, NF, WHAT, CAP>, dim3(head_grid(blocks)), dim3(kHeadThreads), 0, stream, a);
}

template <int MF, int NF>
hipError_t launch_tiles(const HeadForwardArgs& a, HeadForward what, int64_t rows, hipStream_t stream) {
  const bool cap = a.cap != 0.0f;
  switch (what) {
    case kHeadLogits: return cap ? launch<MF, NF, kHeadLogits, true>(a, rows, stream) : launch<MF, NF, kHeadLogits, false>(a, rows, stream);
    case kHeadSums: return cap ? launch<MF, NF, kHeadSums, true>(a, rows, stream) : launch<MF, NF, kHeadSums, false>(a, rows, stream);
    default: return cap ? launch<MF, NF, kHeadSumsKept, true>(a, rows, stream) : launch<MF, NF, kHeadSumsKept, false>(a, rows, stream);
  }
}

}  // namespace

hipError_t launch_head_few(const HeadForwardArgs& a, HeadForward what, int64_t rows, hipStream_t stream) {
  const bool cap = a.cap != 0.0f;
  switch (what) {
    case kHeadLogits: return cap ? launch_few<kHeadLogits, true>(a, rows, stream) : launch_few<kHeadLogits, false>(a, rows, stream);
    case kHeadSums: return cap ? launch_few<kHeadSums, true>(a, rows, stream) : launch_few<kHeadSums, false>(a, rows, stream);
    default: return cap ? launch_few<kHeadSumsKept, true>(a, rows, stream) : launch_few<kHeadSumsKept, false>(a, rows, stream);
  }
}

hipError_t launch_head_forward(const HeadForwardArgs& a, HeadForward what, int64_t rows, hipStream_t stream) {
  if (a.part_columns == kHeadSmallPart) return launch_tiles<4, 4>(a, what, rows, stream);
  if (rows <= 128) return launch_tiles<4, 8>(a, what, rows, stream);
  return launch_tiles<8, 8>(a, what, rows, stream);
}

}  // namespace npd
