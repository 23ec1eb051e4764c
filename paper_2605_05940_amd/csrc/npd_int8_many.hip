// Logits of a head in 8-bit integers, many rows: tiles of the matrix cores' whole-number products (exact), scaled, biased and capped
// in fp32 and rounded to bf16 once before they leave the registers.
#include "npd_int8.hpp"
#include "npd_softcap.hpp"

namespace npd {
namespace {

template <int MF, int NF, bool CAP>
__global__ __launch_bounds__(kHeadThreads, 1) void int8_tiles_kernel(Int8Args a) {
  using Product = HeadProduct<MF, NF, false, false, true, true>;
  __shared__ __attribute__((aligned(1024))) char lds[Product::kLds];
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
    x.run(q, w, next.there, (int64_t)next.m * Product::kTileM, (int64_t)next.n * Product::kTileN, 0, K, lds);
    tile = next;

    const SoftCap soft(CAP ? a.cap : 1.0f);
    float hs[MF];
#pragma unroll
    for (int i = 0; i < MF; ++i) hs[i] = a.h_scale[mw + 16 * i < rows ? mw + 16 * i : 0];
#pragma unroll
    for (int j = 0; j < NF; j += 2) {
      __builtin_amdgcn_sched_barrier(0);  // (eight columns' scales at a time: the fragments of the next tile are in registers already)
      const int n = nw + 16 * j;
      float ws[8], bias[8];
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const int v = n + t < a.V ? n + t : a.V - 1;
        ws[t] = a.w_scale[v];
        bias[t] = a.bias ? bf16_one(a.bias[v]) : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < MF; ++i) {
        const int64_t m = mw + 16 * i;
        float y[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          y[t] = __builtin_fmaf((float)x.acc[i][j + (t >> 2)][t & 3] * hs[i], ws[t], bias[t]);
          if constexpr (CAP) y[t] = soft.cap * soft.tanh_of(y[t]);
        }
        if (m >= rows) continue;
        uint16_t* out = a.out + m * a.out_stride + n;
        const uint4 v = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
        if (columns + 16 * j + 32 <= a.V) {
          stream8(out, v);
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

template <int MF, int NF>
hipError_t launch(const Int8Args& a, hipStream_t stream) {
  using Product = HeadProduct<MF, NF, false, false, true, true>;
  const int64_t mt = (a.T + Product::kTileM - 1) / Product::kTileM, nt = (a.V + Product::kTileN - 1) / Product::kTileN;
  const int64_t blocks = (mt * nt + 7) / 8 * 8;
  if (blocks >= (int64_t)1 << 30) return hipErrorInvalidConfiguration;
  return launch_kernel(a.cap != 0.0f ? int8_tiles_kernel<MF, NF, true> : int8_tiles_kernel<MF, NF, false>, dim3(head_grid(blocks)),
                       dim3(kHeadThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_int8_many(const Int8Args& a, hipStream_t stream) {
  if (head_small(a.T, a.V)) return launch<4, 4>(a, stream);
  if (a.T <= 128) return launch<4, 8>(a, stream);
  return launch<8, 8>(a, stream);
}

}  // namespace npd
