// Logits of a head and the sums of their softmax: x = h W^T (+ bias, soft cap) in the matrix cores, one 256 x 256 tile per workgroup
// (64 or 128 rows where there are no more), and what becomes of a tile before it leaves the registers.
//
// The sums of a row are taken against a reference r: sum 2^(x c - r).  r is the row's own r0 (a true logit of the row, its label's as a rule,
// rounded to a whole number), so that one pass suffices and what is kept of different tiles fits together; only 128 columns whose largest
// logit lies 2^40 and more above it take that one, rounded, instead.  References are whole numbers: bringing two together is exact.
#include "npd_head.hpp"

namespace npd {
namespace {

constexpr float kHeadHeadroom = 40.0f;  // log2

// cap tanh(x / cap), by tanh u = 1 - 2 / (1 + e^2u)
struct SoftCap {
  float cap, k2;
  __device__ __forceinline__ explicit SoftCap(float c) : cap(c), k2(2.0f * kLog2e / c) {}
  __device__ __forceinline__ float tanh_of(float x) const {
    return 1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + exp2_fast(x * k2));
  }
};

template <int MF, int NF, HeadForward WHAT, bool CAP>
__global__ __launch_bounds__(kHeadThreads, 1) void head_forward_kernel(HeadForwardArgs a) {
  using Product = HeadProduct<MF, NF, false, false, true>;
  static_assert(16 * NF == kHeadPart, "a wave's columns are one partial sum");
  __shared__ __attribute__((aligned(1024))) char lds[Product::kLds];
  const HeadSpan span = head_span(a.chunk);
  if (!span.there || span.rows == 0) return;
  const HeadTile tile = head_tile(blockIdx.x, (span.rows + Product::kTileM - 1) / Product::kTileM,
                                  (a.V + Product::kTileN - 1) / Product::kTileN);
  if (!tile.there) return;
  const int64_t m0 = (int64_t)tile.m * Product::kTileM;
  const int n0 = tile.n * Product::kTileN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t mw = m0 + (wave >> 1) * 16 * MF + (lane & 15);  // + 16 i
  const int nw = n0 + (wave & 1) * 16 * NF + 8 * (lane >> 4);   // + 32 j + 0 .. 7, fragments 2 j and 2 j + 1
  Product x;
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
  HeadMatrix q = a.q;
  q.rows = span.rows;
  x.run(q, a.w, m0, n0, 0, a.K, lds);

  const SoftCap soft(CAP ? a.cap : 1.0f);
  const bool edge = n0 + Product::kTileN > a.V;  // uniform
#pragma unroll
  for (int i = 0; i < MF; ++i) {
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
        if (n + 8 <= a.V && (reinterpret_cast<uintptr_t>(out + n) & 15) == 0) {
          *reinterpret_cast<uint4*>(out + n) = make_uint4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
          for (int t = 0; t < 8; ++t)
            if (n + t < a.V) out[n + t] = (uint16_t)(v[t >> 1] >> (16 * (t & 1)));
        }
      }
    } else {
      float v[4 * NF], d[CAP ? 4 * NF : 1];
      float top = -__builtin_inff();
#pragma unroll
      for (int j = 0; j < NF; ++j) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          float y = x.acc[i][j][t];
          if constexpr (CAP) {
            const float th = soft.tanh_of(y);
            y = soft.cap * th;
            d[4 * j + t] = __builtin_fmaf(-th, th, 1.0f);
          }
          if (edge && nw + 32 * (j >> 1) + 4 * (j & 1) + t >= a.V) y = -__builtin_inff();
          v[4 * j + t] = y;
          top = fmaxf(top, y);
        }
      }
      top = fmaxf(top, __shfl_xor(top, 16, kWave));
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      const float r0 = a.r0[row ? m : 0];
      const float u = top * a.c;
      const float r = u > r0 + kHeadHeadroom ? __builtin_rintf(u) : r0;
      float z = 0.0f;
      uint16_t* e = WHAT == kHeadSumsKept ? a.e + (row ? m : 0) * a.e_stride : nullptr;
#pragma unroll
      for (int j = 0; j < NF; j += 2) {
        uint32_t w[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int p = 4 * j + 2 * t;
          float lo = exp2_fast(__builtin_fmaf(v[p], a.c, -r)), hi = exp2_fast(__builtin_fmaf(v[p + 1], a.c, -r));
          z += lo;
          z += hi;
          if constexpr (CAP && WHAT == kHeadSumsKept) {
            lo *= d[p];
            hi *= d[p + 1];
          }
          if constexpr (WHAT == kHeadSumsKept) w[t] = pack_bf16(lo, hi);
        }
        if constexpr (WHAT == kHeadSumsKept) {
          const int n = nw + 16 * j;
          // (rows of e begin on 16 bytes, n is a multiple of 8)
          if (row && n < a.e_stride) *reinterpret_cast<uint4*>(e + n) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
      z += __shfl_xor(z, 16, kWave);
      z += __shfl_xor(z, 32, kWave);
      const int part = (n0 + (wave & 1) * 16 * NF) / kHeadPart;
      if (lane < 16 && row && part < a.parts) a.part[m * a.parts + part] = make_float2(r, z);
    }
  }
}

template <int MF, HeadForward WHAT, bool CAP>
hipError_t launch(const HeadForwardArgs& a, int64_t rows, hipStream_t stream) {
  using Product = HeadProduct<MF, 8, false, false, true>;
  const int64_t mt = (rows + Product::kTileM - 1) / Product::kTileM, nt = (a.V + Product::kTileN - 1) / Product::kTileN;
  const int64_t blocks = (mt * nt + 7) / 8 * 8;
  if (blocks >= (int64_t)1 << 24) return hipErrorInvalidConfiguration;
  return launch_kernel(head_forward_kernel<MF, 8, WHAT, CAP>, dim3((unsigned)blocks), dim3(kHeadThreads), 0, stream, a);
}

template <int MF>
hipError_t launch_rows(const HeadForwardArgs& a, HeadForward what, int64_t rows, hipStream_t stream) {
  const bool cap = a.cap != 0.0f;
  switch (what) {
    case kHeadLogits: return cap ? launch<MF, kHeadLogits, true>(a, rows, stream) : launch<MF, kHeadLogits, false>(a, rows, stream);
    case kHeadSums: return cap ? launch<MF, kHeadSums, true>(a, rows, stream) : launch<MF, kHeadSums, false>(a, rows, stream);
    default: return cap ? launch<MF, kHeadSumsKept, true>(a, rows, stream) : launch<MF, kHeadSumsKept, false>(a, rows, stream);
  }
}

}  // namespace

hipError_t launch_head_forward(const HeadForwardArgs& a, HeadForward what, int64_t rows, hipStream_t stream) {
  if (rows <= 64) return launch_rows<2>(a, what, rows, stream);
  if (rows <= 128) return launch_rows<4>(a, what, rows, stream);
  return launch_rows<8>(a, what, rows, stream);
}

}  // namespace npd
