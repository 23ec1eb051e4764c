// Logits of a head in 8-bit integers, many rows: tiles of the matrix cores' whole-number products (exact), scaled, biased and capped
// in fp32 and rounded to bf16 once before they leave the registers.
//
// A step of 64 bytes of k takes the matrix cores as long as one of 32 bf16 values, so a tile has half the steps and its end weighs
// twice: with the scales loaded there 4,096 x 151,936 x 2,048 took 1,450 us, with them waiting in LDS 1,264.
#include "npd_int8.hpp"
#include "npd_softcap.hpp"

namespace npd {
namespace {

template <int MF, int NF, bool CAP>
__global__ __launch_bounds__(kHeadThreads, 1) void int8_tiles_kernel(Int8Args a) {
  using Product = HeadProduct<MF, NF, false, false, true, true>;
  __shared__ __attribute__((aligned(1024))) char lds[Product::kLds];
  // a wave's factors and biases: requested with a tile's first step, in LDS when its sums are there (no barrier: they are the wave's own)
  constexpr int kColumns = 16 * NF, kRows = 16 * MF, kC = (kColumns + kWave - 1) / kWave, kR = (kRows + kWave - 1) / kWave;
  __shared__ __attribute__((aligned(16))) float factors[kHeadThreads / kWave][2][kColumns], of_rows[kHeadThreads / kWave][kR * kWave];
  const int rows = (int)a.T;
  const int mt = (rows + Product::kTileM - 1) / Product::kTileM, nt = (a.V + Product::kTileN - 1) / Product::kTileN;
  HeadTile tile = head_tile(blockIdx.x, mt, nt);
  if (!tile.there) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int K = (a.D + 15) / 16 * 8;  // pairs of bytes
  const HeadMatrix q = {reinterpret_cast<const uint16_t*>(a.h), a.h_stride / 2, rows, K};
  const HeadMatrix w = {reinterpret_cast<const uint16_t*>(a.w), a.w_stride / 2, a.V, K};
  Product x;
  x.start(q, w, (int64_t)tile.m * Product::kTileM, (int64_t)tile.n * Product::kTileN, 0, K, lds);
  for (unsigned block = blockIdx.x + gridDim.x; tile.there; block += gridDim.x) {
    const HeadTile next = head_tile(block, mt, nt);
    const int64_t mw = (int64_t)tile.m * Product::kTileM + (wave >> 1) * 16 * MF + (lane & 15);  // + 16 i
    const int columns = tile.n * Product::kTileN + (x.wave & 1) * 16 * NF;                       // of the wave
    const int nw = columns + 8 * (lane >> 4);                                                    // + 32 j + 0 .. 7
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
      for (int j = 0; j < NF; ++j) x.acc[i][j] = i32x4{0, 0, 0, 0};
    float ws[kC], bias[kC], hs[kR];
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      const int n = columns + c * kWave + lane, v = n < a.V ? n : a.V - 1;
      ws[c] = a.w_scale[v];
      bias[c] = a.bias ? bf16_one(a.bias[v]) : 0.0f;
    }
#pragma unroll
    for (int c = 0; c < kR; ++c) {
      const int64_t m = mw - (lane & 15) + c * kWave + lane;
      hs[c] = a.h_scale[m < rows ? m : rows - 1];
    }
    x.run(q, w, next.there, (int64_t)next.m * Product::kTileM, (int64_t)next.n * Product::kTileN, 0, K, lds);
    tile = next;
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      factors[wave][0][c * kWave + lane] = ws[c];
      factors[wave][1][c * kWave + lane] = bias[c];
    }
#pragma unroll
    for (int c = 0; c < kR; ++c) of_rows[wave][c * kWave + lane] = hs[c];
    // (Lanes read what others of their wave wrote.  A wave's LDS instructions are done in their order; that this is their order in the code
    // is said here, and takes no instruction.)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();

    const SoftCap soft(CAP ? a.cap : 1.0f);
#pragma unroll
    for (int j = 0; j < NF; j += 2) {
      __builtin_amdgcn_sched_barrier(0);  // (eight columns' scales at a time: the fragments of the next tile are in registers already)
      const int n = nw + 16 * j, at = n - columns;
      f32x4 f[2], g[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        f[t] = *reinterpret_cast<const f32x4*>(&factors[wave][0][at + 4 * t]);
        g[t] = *reinterpret_cast<const f32x4*>(&factors[wave][1][at + 4 * t]);
      }
#pragma unroll
      for (int i = 0; i < MF; ++i) {
        const int64_t m = mw + 16 * i;
        const float by = of_rows[wave][16 * i + (lane & 15)];
        float y[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          y[t] = __builtin_fmaf((float)x.acc[i][j + (t >> 2)][t & 3] * by, f[t >> 2][t & 3], g[t >> 2][t & 3]);
          if constexpr (CAP) y[t] = soft.cap * soft.tanh_of(y[t]);
        }
        if (m >= rows) continue;
        uint16_t* out = a.out + m * a.out_stride + n;
        const uint4 v = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
        if (columns + 16 * j + 32 <= a.V) {
          // (not past the caches: rows that begin on odd values leave lines half written, 2,048 x 151,935 x 2,048 869 us, 1,086 past them)
          store8(out, v);
        } else {
          const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int t = 0; t < 8; ++t)
            if (n + t < a.V) out[t] = (uint16_t)(u[t >> 1] >> (16 * (t & 1)));
        }
      }
    }
  }
}

// `together`: workgroups that a compute unit runs at once (their LDS), so that one's end of a tile lies beside the other's steps
template <int MF, int NF>
hipError_t launch(const Int8Args& a, int together, hipStream_t stream) {
  using Product = HeadProduct<MF, NF, false, false, true, true>;
  const int64_t mt = (a.T + Product::kTileM - 1) / Product::kTileM, nt = (a.V + Product::kTileN - 1) / Product::kTileN;
  const int64_t blocks = (mt * nt + 7) / 8 * 8, units = (int64_t)compute_units() / 8 * 8 * together;
  if (blocks >= (int64_t)1 << 30) return hipErrorInvalidConfiguration;
  return launch_kernel(a.cap != 0.0f ? int8_tiles_kernel<MF, NF, true> : int8_tiles_kernel<MF, NF, false>,
                       dim3((unsigned)(blocks < units || units == 0 ? blocks : units)), dim3(kHeadThreads), 0, stream, a);
}

}  // namespace

// Tiles of 256 x 256 have the highest rate (4,096 x 151,936 x 2,048 1,264 us, 2,020 TOPS; 256 x 128 1,706, 128 x 128 1,850), where there are
// enough of them for the compute units, and where their rows are there.  Measured (MI355X, us; 64 x 128 / 128 x 128 / 256 x 128 / 256 x 256, of
// the first two as many workgroups together as fit):
//   rows  of 32,000 x 4,096             of 50,048 x 1,024              of 151,936 x 2,048
//   64    32.9 / 33.9 / - / -           15.9 / 16.9 / - / -            74.5 / 75.6 / - / -
//   128   49 / 35.4 / 39.4 / 53.5       25.0 / 19.2 / 24.3 / 26.6      111 / 87.3 / 101.5 / 106.6
//   160   - / 49.9 / 42.2 / 58.4        - / 26.0 / 25.7 / 27.0         - / 115 / 104 / 108
//   256   - / 56.1 / 46.0 / 59.3        - / 32.4 / 28.2 / 28.4         - / 136 / 115 / 114
//   333   - / 73.5 / 68.8 / 61.4        - / 35.9 / 43.2 / 43.9         - / 176 / 178 / 157
//   512   - / 101 / 85 / 65             - / 51.8 / 51.4 / 46.1         - / 240 / 219 / 172
hipError_t launch_int8_many(const Int8Args& a, hipStream_t stream) {
  if (a.T <= 64) return launch<2, 4>(a, 3, stream);
  if (a.T <= 128 || head_small(a.T, a.V)) return launch<4, 4>(a, 2, stream);
  const int64_t tiles = (a.T + 255) / 256 * (((int64_t)a.V + 255) / 256);
  // (Up to 384 rows fill three tiles of 128, two of 256 by three quarters; with a short k that decides.  Measured (us, tiles of 128 / the
  // larger ones below, 257 and 384 rows): 50,048 x 256 14.4 / 26.7 and 16.1 / 27.2, x 1,024 32.6 / 42.5 and 38.4 / 44.5; 151,936 x 1,024 87.9 /
  // 100.9 and 108.9 / 105.0, x 1,536 124 / 126 and 150 / 133, x 2,048 154 / 157 and 181 / 162; 262,144 x 1,024 147 / 154 and 182 / 164.  Up to
  // 50,048 entries tiles of 128 are faster at 1,536 and 2,048 too, 44.5 / 52.1 and 63.4 / 66.3 us: the width alone decides.)
  if (a.T > 256 && a.T <= 384 && a.D <= 1024) return launch<4, 4>(a, 2, stream);
  if (tiles <= 128) return launch<8, 4>(a, 1, stream);
  return launch<8, 8>(a, 1, stream);
}

}  // namespace npd
