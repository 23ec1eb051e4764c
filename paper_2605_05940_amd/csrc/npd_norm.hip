// Layer norm, forward and backward, and its form without a mean (npd_norm.hpp).  A row lies in the registers of TH threads, G groups
// of eight values each, from its one read to its one write; its sums are taken over what is there (the mean first, then the squares of
// what is left: the difference of two large sums is never formed).
//
// Bytes bound it.  Measured (MI355X, 32,768 x 2,048): forward 48.5 us (5.5 TB/s), backward with both parameters' gradients 83.4 (4.9 TB/s;
// torch's copy of 4 GiB reaches 4.7), of which joining the 512 pieces of those is 4.  With what is unpacked kept in registers, and so one
// or two waves per SIMD, 56.8 and 110.  One row of 2,048 3.7 us.  Rows wider than 16,384 have their gradients read twice (2,048 x 32,768
// 218 us, 10 bytes a value for 6).
#include <float.h>

#include "../../include/npd.h"
#include "npd_head_gemm.hpp"
#include "npd_norm.hpp"

namespace npd {
namespace {

constexpr int kNormThreads = 256;  // of a workgroup with rows of a wave each
constexpr int kNormMostRows = 64;  // one after the other of norm_kernel's threads

template <int TH>
constexpr int norm_block() { return TH < kNormThreads ? kNormThreads : TH; }

// sums of N values over the TH threads of a row, in the same order in every thread
template <int TH, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* smem) {
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = wave_sum(v[n]);
  if constexpr (TH > kWave) {
    constexpr int kWaves = TH / kWave;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __syncthreads();  // (the sums before these have been read)
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (lane == 0) smem[n * kWaves + wave] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float t = smem[n * kWaves];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) t += smem[n * kWaves + w];
      v[n] = t;
    }
  }
}

// the largest of the numbers, of up to 24 bits, of a row's TH threads
template <int TH>
__device__ __forceinline__ uint32_t row_most(uint32_t v, float* smem) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) {
    const uint32_t o = __shfl_xor(v, off, kWave);
    v = v > o ? v : o;
  }
  if constexpr (TH > kWave) {
    __syncthreads();  // (likewise)
    if ((threadIdx.x & 63) == 0) smem[threadIdx.x >> 6] = (float)v;
    __syncthreads();
    for (int w = 0; w < TH / kWave; ++w) {
      const uint32_t o = (uint32_t)smem[w];
      v = v > o ? v : o;
    }
  }
  return v;
}

// Values [d, d + 8) of a row, 0 behind its end.  WHOLE: rows are whole groups of eight (what ends of groups take otherwise, in code and
// registers, costs such rows 20 %).
template <bool WHOLE>
__device__ __forceinline__ uint4 read8(const uint16_t* row, int d, int cols) {
  if constexpr (!WHOLE) return load8_of(row, d, cols);
  const uint4 v = load8(row + (d < cols ? d : 0));
  return d < cols ? v : make_uint4(0, 0, 0, 0);
}
// values [d, d + 8) of a row, those behind its end are left as they are
template <bool WHOLE>
__device__ __forceinline__ void store8_of(uint16_t* row, int d, int cols, const float (&v)[8]) {
  const uint4 w = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  if (WHOLE ? d < cols : d + 8 <= cols) {
    store8(row + d, w);
  } else if constexpr (!WHOLE) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int t = 0; t < 8; ++t)
      if (d + t < cols) row[d + t] = (uint16_t)(u[t >> 1] >> (16 * (t & 1)));
  }
}

constexpr uint32_t kOnes = 0x3f803f80u;  // two bf16 ones

// What stays in registers, for a row or for all rows of a workgroup, stays packed: the compiler would keep what is unpacked once, in
// twice the registers (norm_grad_kernel<64, 4> 256 of them, a wave per SIMD).
template <int G>
__device__ __forceinline__ void stay_packed(uint4 (&w)[G]) {
#pragma unroll
  for (int u = 0; u < G; ++u) asm volatile("" : "+v"(w[u].x), "+v"(w[u].y), "+v"(w[u].z), "+v"(w[u].w));
}

// A row whose sums or squares fp32 does not hold, done again: read for each of its sums and for y, a value at a time (no model has such
// rows; 32,768 of them of 2,048 take 305 us, others 44).  With its largest value's power of two taken out nothing that shows leaves fp32
// (what is less than 2^-126 of that value is rounded to 2^-149 of it; the rest is exact), and the variance is put together in 64 bits.  A
// row that is not finite stays as it came out.  (Threads have the values that they have in norm_kernel: what was written there is
// written again by the same thread.)
template <int TH, int G>
__device__ __forceinline__ void norm_wide_row(const NormArgs& a, int64_t p, float* smem) {
  int thread = threadIdx.x;
  asm volatile("" : "+v"(thread));  // (nothing that this needs is kept in registers over the other rows)
  const uint16_t* row = a.x + p * a.x_stride;
  const auto each = [&](auto&& f) {
#pragma unroll 1
    for (int i = 0; i < 8 * G; ++i) {
      const int d = (thread % TH) * 8 + 8 * TH * (i >> 3) + (i & 7);
      if (d < a.D) f(d, bf16_one(row[d]));
    }
  };
  uint32_t most = 0;
  each([&](int, float v) {
    const uint32_t size = __builtin_bit_cast(uint32_t, v) << 1 >> 17;
    most = most > size ? most : size;
  });
  most = row_most<TH>(most, smem);
  if (most >= 0x7f80) return;  // uniform over the row
  const int e = __builtin_amdgcn_frexp_expf(bf16_one((uint16_t)most)), exponent = e < -100 ? -100 : e > 126 ? 126 : e;
  const float by = __builtin_ldexpf(1.0f, -exponent);
  float mean = 0.0f, s[1] = {0.0f};  // of the row times `by`
  if (!a.rms) {
    each([&](int, float v) { s[0] += v * by; });
    row_sums<TH, 1>(s, smem);
    mean = s[0] / (float)a.D;
  }
  s[0] = 0.0f;
  each([&](int, float v) {
    const float d = __builtin_fmaf(v, by, -mean);
    s[0] = __builtin_fmaf(d, d, s[0]);
  });
  row_sums<TH, 1>(s, smem);
  const double r = 1.0 / __builtin_sqrt(__builtin_ldexp((double)s[0] / a.D, 2 * exponent) + (double)a.eps);
  const float rstd = (float)(s[0] > 0.0f ? __builtin_ldexp(r, exponent) : r);  // (of equal values: any finite number would do)
  if (threadIdx.x % TH == 0) {
    if (a.mean) a.mean[p] = __builtin_ldexpf(mean, exponent);
    if (a.rstd) a.rstd[p] = (float)r;
  }
  uint16_t* out = a.y + p * a.y_stride;
  each([&](int d, float v) {
    const float w = a.w ? bf16_one(a.w[d]) : 1.0f, b = a.b ? bf16_one(a.b[d]) : 0.0f;
    out[d] = one_bf16(__builtin_fmaf(__builtin_fmaf(v, by, -mean) * rstd, w, b));
  });
}

template <int TH, int G, bool WHOLE>
__global__ __launch_bounds__(norm_block<TH>()) void norm_kernel(NormArgs a) {
  __shared__ float smem[norm_block<TH>() / kWave];
  constexpr int kRows = norm_block<TH>() / TH;  // a workgroup's at a time
  const int at = (threadIdx.x % TH) * 8;        // + 8 TH u
  // (of the widest rows the bias is read where it is added: there are no registers for it, 1,024 x 65,536 69 us, with it kept 90)
  constexpr bool kHoldBias = G < 8;
  uint4 w[G], b[kHoldBias ? G : 1];
  const auto bias = [&](int u) { return a.b ? read8<WHOLE>(a.b, at + 8 * TH * u, a.D) : make_uint4(0, 0, 0, 0); };
#pragma unroll
  for (int u = 0; u < G; ++u) {
    w[u] = a.w ? read8<WHOLE>(a.w, at + 8 * TH * u, a.D) : make_uint4(kOnes, kOnes, kOnes, kOnes);
    if constexpr (kHoldBias) b[u] = bias(u);
  }
  const float per = 1.0f / (float)a.D;
  uint64_t wide = 0;  // which of the rows so far are to be done again (kNormMostRows at most)
  int n = 0;
  for (int64_t p = (int64_t)blockIdx.x * kRows + threadIdx.x / TH; p < a.T; p += (int64_t)gridDim.x * kRows) {
    const uint16_t* row = a.x + p * a.x_stride;
    stay_packed(w);
    if constexpr (kHoldBias) stay_packed(b);
    uint4 x[G];
#pragma unroll
    for (int u = 0; u < G; ++u) x[u] = read8<WHOLE>(row, at + 8 * TH * u, a.D);
    float mean = 0.0f;
    if (!a.rms) {
      float s[1] = {0.0f};
#pragma unroll
      for (int u = 0; u < G; ++u) {
        float v[8];
        unpack8(x[u], v);
        s[0] += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
      }
      row_sums<TH, 1>(s, smem);
      mean = s[0] / (float)a.D;  // (rounded once: a row of equal values, whose sums are exact, has its mean exactly)
    }
    stay_packed(x);
    float s[1] = {0.0f};
#pragma unroll
    for (int u = 0; u < G; ++u) {
      float v[8];
      unpack8(x[u], v);
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const float d = (WHOLE ? at + 8 * TH * u : at + 8 * TH * u + t) < a.D ? v[t] - mean : 0.0f;
        s[0] = __builtin_fmaf(d, d, s[0]);
      }
    }
    row_sums<TH, 1>(s, smem);
    stay_packed(x);
    const float rstd = 1.0f / __builtin_sqrtf(__builtin_fmaf(s[0], per, a.eps));
    // (Sums and squares beyond fp32 are not finite.  Squares below it are off by 2^-150 each, nothing beside a variance of 2^-100.)
    if (__ballot(!(rstd >= 0x1p-64f && rstd <= 0x1p50f))) wide |= (uint64_t)1 << n;  // (a row's threads have the same)
    ++n;
    if (threadIdx.x % TH == 0) {
      if (a.mean) a.mean[p] = mean;
      if (a.rstd) a.rstd[p] = rstd;
    }
    uint16_t* out = a.y + p * a.y_stride;
#pragma unroll
    for (int u = 0; u < G; ++u) {
      float v[8], wv[8], bv[8];
      unpack8(x[u], v);
      unpack8(w[u], wv);
      unpack8(kHoldBias ? b[kHoldBias ? u : 0] : bias(u), bv);
#pragma unroll
      for (int t = 0; t < 8; ++t) v[t] = __builtin_fmaf((v[t] - mean) * rstd, wv[t], bv[t]);
      store8_of<WHOLE>(out, at + 8 * TH * u, a.D, v);
    }
  }
  // (Behind the loop, where they need none of its registers, and with the kernel's one argument read again: in the loop 32,768 x 2,047
  // takes 61.7 us, so 56.7.)
  const NormArgs* again = (const NormArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(again));
  for (; wide; wide &= wide - 1)
    norm_wide_row<TH, G>(*again, ((int64_t)blockIdx.x + (int64_t)__builtin_ctzll(wide) * gridDim.x) * kRows + threadIdx.x / TH, smem);
}

// (x - mean) rstd of a row, whose difference is halved first where it could be beyond fp32
struct RowMean {
  float by, mean_by, rstd_by;  // rstd = by rstd_by
  __device__ __forceinline__ float normed(float x) const { return __builtin_fmaf(x, by, -mean_by) * rstd_by; }
};
__device__ __forceinline__ RowMean row_mean(const NormGradArgs& a, int64_t p) {
  const float mean = a.rms ? 0.0f : a.mean[p], rstd = a.rstd[p];
  const bool large = __builtin_fabsf(mean) >= 0x1p119f;  // (bf16 ends 2^120 below 2^128, fp32 2^104)
  return large ? RowMean{0.5f, 0.5f * mean, 2.0f * rstd} : RowMean{1.0f, mean, rstd};
}

// HELD: the workgroup's sums over its rows for the parameters' gradients stay in registers, and go to its piece at the end.
template <int TH, int G, bool HELD, bool WHOLE>
__global__ __launch_bounds__(norm_block<TH>()) void norm_grad_kernel(NormGradArgs a) {
  __shared__ float smem[2 * norm_block<TH>() / kWave];
  __shared__ float joined[HELD && TH == kWave ? 2 * TH * 8 * G : 1];
  constexpr int kRows = norm_block<TH>() / TH;
  const int at = (threadIdx.x % TH) * 8;
  uint4 w[G];
#pragma unroll
  for (int u = 0; u < G; ++u) w[u] = a.w ? read8<WHOLE>(a.w, at + 8 * TH * u, a.D) : make_uint4(kOnes, kOnes, kOnes, kOnes);
  float dw[HELD ? G : 1][8] = {}, db[HELD ? G : 1][8] = {};
  const float per = 1.0f / (float)a.D;
  for (int64_t p = (int64_t)blockIdx.x * kRows + threadIdx.x / TH; p < a.T; p += (int64_t)gridDim.x * kRows) {
    const uint16_t *grow = a.g + p * a.g_stride, *xrow = a.x + p * a.x_stride;
    stay_packed(w);
    uint4 g[G], x[G];
#pragma unroll
    for (int u = 0; u < G; ++u) {
      g[u] = read8<WHOLE>(grow, at + 8 * TH * u, a.D);
      x[u] = read8<WHOLE>(xrow, at + 8 * TH * u, a.D);
    }
    const RowMean row = row_mean(a, p);
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < G; ++u) {
      float gv[8], xv[8], wv[8];
      unpack8(g[u], gv);
      unpack8(x[u], xv);
      unpack8(w[u], wv);
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        // (behind the end g is 0, but the mean times rstd may be beyond fp32)
        const bool inside = (WHOLE ? at + 8 * TH * u : at + 8 * TH * u + t) < a.D;
        const float n = inside ? row.normed(xv[t]) : 0.0f, q = gv[t] * wv[t];
        s[0] = __builtin_fmaf(q, n, s[0]);
        s[1] += q;
        if constexpr (HELD) {
          dw[u][t] = __builtin_fmaf(gv[t], n, dw[u][t]);
          db[u][t] += gv[t];
        }
      }
    }
    if (!a.dx) continue;
    row_sums<TH, 2>(s, smem);
    stay_packed(g);
    stay_packed(x);
    stay_packed(w);
    const float along = s[0] * per, flat = a.rms ? 0.0f : s[1] * per, rstd = row.by * row.rstd_by;
    uint16_t* out = a.dx + p * a.dx_stride;
#pragma unroll
    for (int u = 0; u < G; ++u) {
      float gv[8], xv[8], wv[8];
      unpack8(g[u], gv);
      unpack8(x[u], xv);
      unpack8(w[u], wv);
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        gv[t] = __builtin_fmaf(-row.normed(xv[t]), along, gv[t] * wv[t] - flat) * rstd;
      }
      store8_of<WHOLE>(out, at + 8 * TH * u, a.D, gv);
    }
  }
  if constexpr (HELD) {
    if constexpr (kRows > 1) {
      // the workgroup's rows one after the other
      static_assert(TH == kWave, "rows that share a workgroup are a wave each");
      for (int r = 0; r < kRows; ++r) {
        if (threadIdx.x / TH == r) {
#pragma unroll
          for (int u = 0; u < G; ++u) {
#pragma unroll
            for (int t = 0; t < 8; ++t) {
              const int i = (u * 8 + t) * TH + (threadIdx.x & 63);
              const float w0 = r ? joined[i] : 0.0f, b0 = r ? joined[G * 8 * TH + i] : 0.0f;
              dw[u][t] += w0;
              db[u][t] += b0;
              joined[i] = dw[u][t];
              joined[G * 8 * TH + i] = db[u][t];
            }
            asm volatile("" ::: "memory");  // (a group's sums at a time)
          }
        }
        __syncthreads();
      }
      if (threadIdx.x / TH != kRows - 1) return;
    }
    float* pw = a.dw_pieces + (int64_t)blockIdx.x * a.D;
    float* pb = a.db_pieces + (int64_t)blockIdx.x * a.D;
#pragma unroll
    for (int u = 0; u < G; ++u)
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const int d = at + 8 * TH * u + t;
        if ((WHOLE ? d - t : d) >= a.D) break;
        if (a.dw) pw[d] = dw[u][t];
        if (a.db) pb[d] = db[u][t];
      }
  }
}

// The sums alone, of wide rows: a wave has 512 columns of every fourth row of the workgroup's.
__global__ __launch_bounds__(kNormThreads) void norm_columns_kernel(NormGradArgs a) {
  constexpr int kWaves = kNormThreads / kWave;
  __shared__ float joined[kWaves][2][8][kWave];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = blockIdx.x * (kWave * 8) + lane * 8;
  float dw[8] = {}, db[8] = {};
  for (int64_t p = (int64_t)blockIdx.y * kWaves + wave; p < a.T; p += (int64_t)gridDim.y * kWaves) {
    float g[8], x[8];
    unpack8(load8_of(a.g + p * a.g_stride, d, a.D), g);
    unpack8(load8_of(a.x + p * a.x_stride, d, a.D), x);
    const RowMean row = row_mean(a, p);
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      dw[t] = __builtin_fmaf(g[t], row.normed(x[t]), dw[t]);
      db[t] += g[t];
    }
  }
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    joined[wave][0][t][lane] = dw[t];
    joined[wave][1][t][lane] = db[t];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * kWave * 8; i += kNormThreads) {
    const int what = i / (kWave * 8), t = i % (kWave * 8) / kWave, l = i % kWave;
    float s = joined[0][what][t][l];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) s += joined[w][what][t][l];
    const int e = blockIdx.x * (kWave * 8) + l * 8 + t;
    float* pieces = what ? a.db_pieces : a.dw_pieces;
    if (e < a.D && (what ? a.db : a.dw)) pieces[(int64_t)blockIdx.y * a.D + e] = s;
  }
}

// Joins the pieces: 32 columns to a workgroup, a half wave has every 32nd piece of them.
constexpr int kJoinThreads = 1024, kJoinColumns = 32;
__global__ __launch_bounds__(kJoinThreads) void norm_join_kernel(NormGradArgs a) {
  constexpr int kSlots = kJoinThreads / kJoinColumns;
  __shared__ float joined[kSlots][kJoinColumns];
  const int c = threadIdx.x % kJoinColumns, slot = threadIdx.x / kJoinColumns, d = blockIdx.x * kJoinColumns + c;
  const bool bias = blockIdx.y == 1 || !a.dw;
  const float* pieces = (bias ? a.db_pieces : a.dw_pieces) + (d < a.D ? d : a.D - 1);
  constexpr int kMost = kNormPieces / kSlots;
  float v[kMost], s = 0.0f;
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int piece = slot + i * kSlots;
    v[i] = pieces[(int64_t)(piece < a.pieces ? piece : 0) * a.D];  // (all requested together)
  }
#pragma unroll
  for (int i = 0; i < kMost; ++i) s += slot + i * kSlots < a.pieces ? v[i] : 0.0f;
  joined[slot][c] = s;
  __syncthreads();
  if (threadIdx.x < kJoinColumns && d < a.D) {
#pragma unroll
    for (int i = 1; i < kSlots; ++i) s += joined[i][c];
    uint16_t* out = bias ? a.db : a.dw;
    out[d] = one_bf16(a.accumulate ? s + bf16_one(out[d]) : s);
  }
}

template <int TH, int G>
hipError_t launch_rows(const NormArgs& a, hipStream_t stream) {
  constexpr int kRows = norm_block<TH>() / TH;
  const int64_t blocks = (a.T + kRows - 1) / kRows, least = (blocks + kNormMostRows - 1) / kNormMostRows, most = least > 65536 ? least : 65536;
  return launch_kernel(a.D % 8 == 0 ? norm_kernel<TH, G, true> : norm_kernel<TH, G, false>, dim3((unsigned)(blocks < most ? blocks : most)),
                       dim3(norm_block<TH>()), 0, stream, a);
}

template <int TH, int G>
hipError_t launch_grad(const NormGradArgs& a, hipStream_t stream) {
  constexpr int kRows = norm_block<TH>() / TH;
  const int64_t blocks = (a.T + kRows - 1) / kRows;
  const dim3 block(norm_block<TH>());
  const bool whole = a.D % 8 == 0;
  if constexpr (TH * 8 * G <= kNormHeldWidth) {
    if (a.dw || a.db)
      return launch_kernel(whole ? norm_grad_kernel<TH, G, true, true> : norm_grad_kernel<TH, G, true, false>, dim3((unsigned)a.pieces), block, 0,
                           stream, a);
  }
  if (!a.dx) return hipSuccess;
  return launch_kernel(whole ? norm_grad_kernel<TH, G, false, true> : norm_grad_kernel<TH, G, false, false>,
                       dim3((unsigned)(blocks < 65536 ? blocks : 65536)), block, 0, stream, a);
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t stream) {
  if (a.D <= 512) return launch_rows<64, 1>(a, stream);
  if (a.D <= 1024) return launch_rows<64, 2>(a, stream);
  if (a.D <= 2048) return launch_rows<64, 4>(a, stream);
  if (a.D <= 4096) return launch_rows<256, 2>(a, stream);
  if (a.D <= 8192) return launch_rows<256, 4>(a, stream);
  if (a.D <= 16384) return launch_rows<1024, 2>(a, stream);
  if (a.D <= 32768) return launch_rows<1024, 4>(a, stream);
  return launch_rows<1024, 8>(a, stream);
}

int norm_pieces(int64_t T, int32_t D) {
  const int rows = D <= 2048 ? 4 : D <= kNormHeldWidth ? 1 : 4;  // of a workgroup at a time
  const int64_t blocks = (T + rows - 1) / rows;
  return (int)(blocks < kNormPieces ? blocks : kNormPieces);
}

hipError_t launch_norm_grad(const NormGradArgs& a, hipStream_t stream) {
  const hipError_t e = a.D <= 512     ? launch_grad<64, 1>(a, stream)
                       : a.D <= 1024  ? launch_grad<64, 2>(a, stream)
                       : a.D <= 2048  ? launch_grad<64, 4>(a, stream)
                       : a.D <= 4096  ? launch_grad<256, 2>(a, stream)
                       : a.D <= 8192  ? launch_grad<256, 4>(a, stream)
                       : a.D <= 16384 ? launch_grad<1024, 2>(a, stream)
                       : a.D <= 32768 ? launch_grad<1024, 4>(a, stream)
                                      : launch_grad<1024, 8>(a, stream);
  if (e != hipSuccess || !(a.dw || a.db)) return e;
  if (a.D > kNormHeldWidth) {
    const dim3 grid((unsigned)(a.D + 511) / 512, (unsigned)a.pieces);
    const hipError_t c = launch_kernel(norm_columns_kernel, grid, dim3(kNormThreads), 0, stream, a);
    if (c != hipSuccess) return c;
  }
  return launch_kernel(norm_join_kernel, dim3((unsigned)(a.D + kJoinColumns - 1) / kJoinColumns, a.dw && a.db ? 2 : 1), dim3(kJoinThreads), 0, stream, a);
}

}  // namespace npd
