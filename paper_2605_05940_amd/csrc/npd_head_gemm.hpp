// The matrix product behind the head operators (npd_head_*.hip): C[m, n] = sum_k Q(m, k) P(n, k) of two bf16 matrices with
// fp32 sums, tile by tile of C in workgroups of four waves, and whatever the caller's epilogue makes of a tile.
//
// Each operand is read along k (KC: a row of memory holds consecutive k) or across it (KS: a row of memory holds one k), so the
// three products of a head -- logits = H W^T, dH = G W, dW = G^T H -- need no transposed copy of anything: a KS operand's
// fragments come out of LDS through ds_read_b64_tr_b16, which hands lane i of 16 the i-th column of a 4 x 16 block.
//
// One step is 32 values of k.  Tiles of four steps are in flight or in use in LDS (buffer_load ... lds, 16 bytes per lane, no
// registers in between); the fragments of step i + 1 are read into registers while the matrix cores work on step i, so a wave
// waits only for the barrier that ends a step.  With 256 x 256 tiles a wave holds 128 x 128 sums (256 registers) and a step is
// 64 v_mfma_f32_16x16x32_bf16, 1,024 cycles of its SIMD.
//
// Measured (MI355X, TFLOP/s): 8,192^3 along k 1,376, across it 1,414 (32,768 x 2,048 x 8,192), 8,192 x 2,048 x 65,536 1,344.  A step
// takes 1.45 times its matrix instructions: without the loads into LDS 1,836 (a compute unit takes 64 bytes of them per cycle, 512
// cycles a step, and they share the L2), without the reads of LDS 1,460, without either 2,072, without the barrier 1,409, without the
// waits for loads 1,375.  Slower: 128 x 256 tiles, two workgroups per compute unit (912 against 1,066 with 151,936 columns);
// 32 x 32 x 16 products (1,268); waves that request at different places of a step (1,187).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "npd_device.hpp"

namespace npd {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kHeadStep = 32;      // values of k per step
constexpr int kHeadStages = 4;     // steps in LDS
constexpr int kHeadThreads = 256;  // four waves, two by two over the tile

// A bf16 matrix.  KC: `rows` along m (or n), `cols` along k.  KS: `rows` along k, `cols` along m (or n).  Rows begin on 16
// bytes.  `rows` / `cols` along m or n are limits that addresses are clamped to (what is computed there is not stored); along k
// the limit is the product's, and what lies behind it counts as 0 without being read.  cols is a multiple of 8.
struct HeadMatrix {
  const uint16_t* p;
  int64_t stride;
  int32_t rows, cols;
};

// The rows of a batch are worked on in chunks of at most `cap` (a multiple of 256).  How many rows there are may be known on the
// device alone (`count`): launches are made for the most there can be, and those of chunks that are not there end at once.
// The chunks that are there share the rows evenly.
struct HeadChunk {
  const int32_t* count;  // null: `total`
  int64_t total;
  int32_t cap, index;
};
struct HeadSpan {
  int64_t first;
  int32_t rows;
  bool there, last;
};
__device__ __forceinline__ HeadSpan head_span(const HeadChunk& c) {
  // (at most 2^30 rows: 32 bits, whose division is short, and none where one chunk is all; every workgroup begins with this)
  const uint32_t n = c.count ? (uint32_t)*c.count : (uint32_t)c.total, cap = (uint32_t)c.cap;
  HeadSpan s;
  if (n <= cap) {
    s.first = 0;
    s.rows = c.index == 0 ? (int32_t)n : 0;
    s.there = s.last = c.index == 0;
    return s;
  }
  const uint32_t chunks = (n + cap - 1) / cap, each = ((n + chunks - 1) / chunks + 255) / 256 * 256, index = (uint32_t)c.index;
  s.there = index < chunks;
  const uint32_t first = s.there ? index * each : n;
  s.first = first;
  s.rows = (int32_t)(first >= n ? 0 : n - first < each ? n - first : each);
  s.last = index == chunks - 1;
  return s;
}

// Which tile a workgroup has.  Workgroups go to the eight XCDs in turn, each with an L2 of its own: an XCD gets consecutive
// tiles, in bands of four tiles of m, so that the 32 that it runs together share 4 + 8 panels of the operands instead of
// reading 64; with fewer than eight tiles of n in bands of 32 over those.  Measured (MI355X, TFLOP/s), 8,192^3 along k / 8,192 x
// 2,048 x 65,536 / 32,768 x 2,048 x 8,192 across it: bands of 2 1,250 / 1,326 / 1,431, of 4 1,378 / 1,344 / 1,431, of 8 1,350 / 1,284
// / 1,380, of 16 1,232 / 1,110 / 1,317; 50,003 x 1,000 (four tiles of n) over 333 rows: of 4 93 us, of 8 76.
__device__ __forceinline__ unsigned head_band(int nt) { return nt >= 8 ? 4u : 32u / (unsigned)nt; }
struct HeadTile {
  int m, n, piece;
  bool there;
};
// (pieces of k: all tiles of a piece, then those of the next one)
__device__ __forceinline__ HeadTile head_tile(unsigned block, int mt, int nt, int pieces = 1) {
  const unsigned tiles = (unsigned)mt * (unsigned)nt, total = tiles * (unsigned)pieces, per = (total + 7) / 8;
  const unsigned local = block / 8, all = block % 8 * per + local;
  HeadTile t;
  t.there = local < per && all < total;
  const unsigned piece = pieces > 1 ? all / tiles : 0, id = all - piece * tiles;
  t.piece = (int)piece;
  const unsigned most = head_band(nt), band = most * (unsigned)nt, b = id / band, in = id % band;
  const unsigned left = (unsigned)mt - b * most, height = left < most ? left : most;
  t.m = (int)(b * most + in % (height ? height : 1));
  t.n = (int)(in / (height ? height : 1));
  return t;
}

#define NPD_LDS __attribute__((address_space(3)))

// Eight or four bf16 values at any even address: one access of 16 or 8 bytes, which global memory takes at any alignment.
__device__ __forceinline__ uint4 load8(const uint16_t* p) {
  uint4 v;
  __builtin_memcpy(&v, p, 16);
  return v;
}
__device__ __forceinline__ void store8(uint16_t* p, const uint4& v) { __builtin_memcpy(p, &v, 16); }
// the same for what is not read again soon: it does not push the operands of the products out of the L2
__device__ __forceinline__ void stream8(uint16_t* p, const uint4& v) {
  typedef uint32_t words __attribute__((ext_vector_type(4), aligned(2)));
  __builtin_nontemporal_store(words{v.x, v.y, v.z, v.w}, reinterpret_cast<words*>(p));
}
__device__ __forceinline__ void store4(uint16_t* p, const uint2& v) { __builtin_memcpy(p, &v, 8); }
// The same of a row that may begin on an odd value, in a matrix that begins on four bytes: the memory pipeline takes 16 bytes from a
// multiple of four at twice the rate of those that are not (49,152 rows of 4,094 values 105 us, of 4,095 214; MI355X), so the four words
// begin a value earlier there, in the row before, and the last value comes by itself.
__device__ __forceinline__ uint4 load8_odd(const uint16_t* p) {
  typedef uint32_t words __attribute__((ext_vector_type(4), aligned(4)));
  const uint32_t odd = (uint32_t)(uintptr_t)p >> 1 & 1;
  const words v = *reinterpret_cast<const words*>(p - odd);
  const uint32_t last = p[7], shift = 16 * odd;
  return make_uint4(__builtin_amdgcn_alignbit(v[1], v[0], shift), __builtin_amdgcn_alignbit(v[2], v[1], shift),
                    __builtin_amdgcn_alignbit(v[3], v[2], shift), __builtin_amdgcn_alignbit(last, v[3], shift));
}
// Values [d, d + 8) of a row of `cols`, 0 behind its end: where that is among them, the last eight of the row, shifted (one load; one
// for each value left of a row of 4,095 took as long as the rest of it where there are few rows).
template <bool ODD = false>
__device__ __forceinline__ uint4 load8_of(const uint16_t* row, int d, int cols) {
  const int over = d + 8 - cols;
  if (cols < 8) {  // uniform
    uint32_t w[4] = {};
#pragma unroll
    for (int t = 0; t < 8; ++t)
      if (d + t < cols) w[t >> 1] |= (uint32_t)row[d + t] << (16 * (t & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  const uint16_t* p = row + (over > 0 ? cols - 8 : d);
  uint4 v = ODD ? load8_odd(p) : load8(p);
  if (over > 0) {
    if (over & 4) v = make_uint4(v.z, v.w, 0, 0);
    if (over & 2) v = make_uint4(v.y, v.z, v.w, 0);
    if (over & 1)
      v = make_uint4(__builtin_amdgcn_alignbit(v.y, v.x, 16), __builtin_amdgcn_alignbit(v.z, v.y, 16), __builtin_amdgcn_alignbit(v.w, v.z, 16),
                     v.w >> 16);
    if (over >= 8) v = make_uint4(0, 0, 0, 0);
  }
  return v;
}

// 16-byte groups of a KC tile's rows (64 bytes: four groups) are stored at group ^ kc_swizzle(row): the lanes of a fragment
// read that are served together (four runs of four lanes of two groups) then hit 16 different groups of the 64 banks, in both
// row orders below
__device__ __forceinline__ int kc_swizzle(int row) {
  const int a = row >> 2;
  return ((a ^ a >> 2) & 1) << 1 ^ (a >> 1 & 1) * 3;
}
// 32-byte granules of a KS tile's rows are stored at granule ^ ks_swizzle(k), so that the eight rows that 32 lanes read
// together lie in different banks
__device__ __forceinline__ int ks_swizzle(int k) { return (k & 3) | ((k >> 3) & 1) << 2; }

constexpr uint32_t kHeadRecords = 0x80000000u;  // bytes behind a tile's base that loads may reach; at offsets from here on they give 0

// Where one operand's values of a tile come from: F fragments of 16 rows (or columns) for each of two waves, 32 F in all.
template <int F, bool KS>
struct HeadSource {
  static_assert(F % 2 == 0, "loads are whole waves");
  static constexpr int kLoads = F / 2;                   // 16-byte loads per lane and step
  static constexpr int kBytes = F * 32 * kHeadStep * 2;  // of a step
  static constexpr int kGran = 2 * F;                    // granules of a KS row
  const uint16_t* base;  // uniform
  int64_t step;          // elements between steps
  uint32_t off[kLoads];
  int kpos[2];           // KC: k of the lane's loads within a step (of even and odd ones)
  uint32_t pitch;        // KS: bytes between rows
  int kend;

  __device__ __forceinline__ void init(const HeadMatrix& x, int64_t tile0, int64_t k0, int64_t k1, int wave) {
    const int lane = threadIdx.x & 63;
    kend = (int)(k1 - k0);
    if constexpr (!KS) {
      base = x.p + tile0 * x.stride + k0;
      step = kHeadStep;
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int row = (wave * kLoads + j) * 16 + (lane >> 2);
        const int group = (lane & 3) ^ kc_swizzle(row);
        const int64_t most = x.rows - 1 - tile0;
        off[j] = (uint32_t)((row < most ? row : most) * x.stride * 2 + group * 16);
        if (j < 2) kpos[j] = group * 8;  // (rows of loads j and j + 2 are 32 apart: the same swizzle)
      }
    } else {
      base = x.p + k0 * x.stride + tile0;
      step = (int64_t)kHeadStep * x.stride;
      pitch = (uint32_t)(x.stride * 2);
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int byte = (wave * kLoads + j) * 1024 + lane * 16;
        const int k = byte / (64 * F), group = byte % (64 * F) / 16;
        const int gran = (group >> 1) ^ (ks_swizzle(k) & (kGran - 1));
        const int64_t col = gran * 16 + (group & 1) * 8, most = x.cols - 8 - tile0;
        off[j] = (uint32_t)(k * x.stride * 2 + (col < most ? col : most) * 2);
      }
    }
  }

  // requests load j of step `s` into `to` (this operand's bytes of the stage); zeros behind the last step
  __device__ __forceinline__ void load(int j, int s, char* to, int wave) const {
    const int left = kend - s * kHeadStep;  // uniform
    uint32_t o = off[j], records = kHeadRecords;
    if constexpr (KS) {
      const int rows = left < kHeadStep ? left : kHeadStep;
      records = __builtin_amdgcn_readfirstlane(rows < 0 ? 0 : rows) * pitch;
    } else {
      if (left <= kpos[j & 1]) o = kHeadRecords;
    }
    // Written out: a wait that the compiler puts in front of every read of LDS behind such a load (it does in front of the
    // transposing ones) would undo what the stages are for.  The instruction writes no register.  Nor does the compiler keep distances to
    // what is written out: a scalar register that a vector instruction wrote (a spilled one comes back through v_readlane) may be read
    // by the load five wait states later, of which s_mov and s_nop are two.  s_nop 3 in here would do, for 3 % of the large calls (loss of
    // 32,768 x 151,936 x 2,048 36.7 ms for 35.5), so the built code is checked instead, with the products' distances (tests/test_head_code.py).
    const uint64_t at = reinterpret_cast<uint64_t>(base + (left > 0 ? s * step : 0));
    const i32x4 r = {(int)(uint32_t)at, (int)(uint32_t)(at >> 32), (int)records, 0x00020000};
    const uint32_t lds = (uint32_t)(uintptr_t)(NPD_LDS char*)(to + (wave * kLoads + j) * 1024);
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (m0 is never allocated; named so that no value of it is kept across this)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(o), "s"(r) : "memory", "m0");
#pragma clang diagnostic pop
  }
};

// Where a wave's fragments lie in a step's bytes.  PAIRED: fragments 2j and 2j + 1 take turns over groups of four rows, so that a
// lane's sums of the two are eight neighbours.
template <int F, bool KS, bool PAIRED>
struct HeadReader {
  uint32_t rd[KS ? F : 2];

  __device__ __forceinline__ void init(int half) {
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    if constexpr (!KS) {
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const int row = PAIRED ? 8 * (i >> 2) + 4 * f + (i & 3) : 16 * f + i;
        rd[f] = (uint32_t)((half * F * 16 + row) * 64 + (g ^ kc_swizzle(row)) * 16);
      }
    } else {
      const int k = 8 * g + (i >> 2);
#pragma unroll
      for (int f = 0; f < F; ++f)
        rd[f] = (uint32_t)(k * 64 * F + ((half * F + f) ^ (ks_swizzle(k) & (2 * F - 1))) * 32 + (i & 3) * 8);
    }
  }

  __device__ __forceinline__ bf16x8 fragment(int f, const char* from) const {
    if constexpr (!KS) {
      return *reinterpret_cast<const bf16x8*>(from + rd[f & 1] + (f >> 1) * 2048);
    } else {
      typedef short tr4 __attribute__((ext_vector_type(4)));
      const tr4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((NPD_LDS tr4*)(from + rd[f]));
      const tr4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((NPD_LDS tr4*)(from + rd[f] + 4 * 64 * F));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

// The sums of tiles of 32 MF rows by 32 NF columns, one after the other: start() with the first, then for every tile run(), which
// requests the next one's first steps while it works on its own last ones, so that they are there when the tile's sums
// have been dealt with.  acc[i][j][e]: row m = 16 i + (lane & 15) of the wave's 16 MF, column 16 j + 4 (lane >> 4) + e of its
// 16 NF (PAIRED: 32 (j / 2) + 8 (lane >> 4) + 4 (j & 1) + e).
//
// BYTES: the operands are 8-bit integers, two to each "value" above (rows of an even number of bytes, k counted in pairs), and the
// sums 32-bit ones.  v_mfma_i32_16x16x64_i8 takes its operands from the same 16 bytes of a lane in the same time.
template <int MF, int NF, bool QKS, bool PKS, bool PAIRED, bool BYTES = false>
struct HeadProduct {
  static_assert(!BYTES || !(QKS || PKS), "bytes are read along k");
  using Sum = std::conditional_t<BYTES, i32x4, f32x4>;
  using Q = HeadSource<MF, QKS>;
  using P = HeadSource<NF, PKS>;
  static constexpr int kLds = kHeadStages * (Q::kBytes + P::kBytes);
  static constexpr int kTileM = 32 * MF, kTileN = 32 * NF;
  static constexpr int kLoads = Q::kLoads + P::kLoads;
  Sum acc[MF][NF];
  Q q;
  P p;
  HeadReader<MF, QKS, false> qr;
  HeadReader<NF, PKS, PAIRED> pr;
  bf16x8 fq[2][MF], fp[2][NF];
  int steps, wave;

  template <int LEFT>
  static __device__ __forceinline__ void meet() {
    // LDS reads done, all but LEFT of the wave's loads landed; then every wave's
    constexpr int imm = 0x70 | (LEFT & 15) | (LEFT >> 4) << 14;
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(imm);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  }
  static __device__ __forceinline__ char* q_stage(char* lds, int s) { return lds + s * Q::kBytes; }
  static __device__ __forceinline__ char* p_stage(char* lds, int s) { return lds + kHeadStages * Q::kBytes + s * P::kBytes; }

  // acc += p q, written out so that the sums stay where they are (256 registers of sums leave the compiler none to move them
  // through: from the builtin it makes copies in every step, 24 of 64 products then wait for one).  An operand that a vector instruction
  // wrote may be read two wait states later, the sums by anything else eleven (see HeadSource::load; with s_nop 1 in here as well: 7 %).
  static __device__ __forceinline__ void multiply(Sum& c, const bf16x8& a, const bf16x8& b) {
    if constexpr (BYTES)
      asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
    else
      asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
  }

  // One step, in stage S; requests step `ahead` of (nq, np) into the same stage.
  template <int S>
  __device__ __forceinline__ void phase(const Q& nq, const P& np, int ahead, char* lds) {
    constexpr int cur = S & 1, nxt = cur ^ 1, sn = (S + 1) % kHeadStages;
    meet<(kHeadStages - 2) * kLoads>();
    constexpr int kReads = MF + NF, kSteps = MF * NF;
    int load = 0, read = 0;
#pragma unroll
    for (int a = 0; a < MF; ++a) {
#pragma unroll
      for (int b = 0; b < NF; ++b) {
        const int done = a * NF + b;
        // loads are spread over the step's matrix instructions (they wait for one another otherwise: a compute unit takes 64 bytes per
        // cycle), reads over the first half of them
        while (load < kLoads && load * kSteps <= done * kLoads) {
          if (load < Q::kLoads)
            nq.load(load, ahead, q_stage(lds, S), wave);
          else
            np.load(load - Q::kLoads, ahead, p_stage(lds, S), wave);
          ++load;
        }
        while (read < kReads && read * (kSteps / 2) <= done * kReads) {
          if (read < NF)
            fp[nxt][read] = pr.fragment(read, p_stage(lds, sn));
          else
            fq[nxt][read - NF] = qr.fragment(read - NF, q_stage(lds, sn));
          ++read;
        }
        multiply(acc[a][b], fp[cur][b], fq[cur][a]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // the first tile: rows m0, columns n0, k in [k0, k1)
  __device__ __forceinline__ void start(const HeadMatrix& qm, const HeadMatrix& pm, int64_t m0, int64_t n0, int64_t k0, int64_t k1,
                                        char* lds) {
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    steps = (int)((k1 - k0 + kHeadStep - 1) / kHeadStep);
    q.init(qm, m0, k0, k1, wave);
    p.init(pm, n0, k0, k1, wave);
    qr.init(wave >> 1);
    pr.init(wave & 1);
#pragma unroll
    for (int s = 0; s < kHeadStages; ++s) {
#pragma unroll
      for (int j = 0; j < Q::kLoads; ++j) q.load(j, s, q_stage(lds, s), wave);
#pragma unroll
      for (int j = 0; j < P::kLoads; ++j) p.load(j, s, p_stage(lds, s), wave);
    }
    meet<(kHeadStages - 1) * kLoads>();
#pragma unroll
    for (int b = 0; b < NF; ++b) fp[0][b] = pr.fragment(b, p_stage(lds, 0));
#pragma unroll
    for (int a = 0; a < MF; ++a) fq[0][a] = qr.fragment(a, q_stage(lds, 0));
  }

  // adds the current tile's products to acc; the tile at (m0, n0) of the same k is the next one if `more`
  __device__ __forceinline__ void run(const HeadMatrix& qm, const HeadMatrix& pm, bool more, int64_t m0, int64_t n0, int64_t k0,
                                      int64_t k1, char* lds) {
    // (the sums' first values are in place well before the first product reads them)
#pragma unroll
    for (int a = 0; a < MF; ++a)
#pragma unroll
      for (int b = 0; b < NF; ++b) asm volatile("" : "+a"(acc[a][b]));
    // (up to three steps of zeros behind the last: leaving between the phases costs the loop its registers)
    int i = 0;
#pragma unroll 1
    for (; i + kHeadStages < steps; i += kHeadStages) {
      phase<0>(q, p, i + kHeadStages, lds);
      phase<1>(q, p, i + kHeadStages + 1, lds);
      phase<2>(q, p, i + kHeadStages + 2, lds);
      phase<3>(q, p, i + kHeadStages + 3, lds);
    }
    if (more) {
      q.init(qm, m0, k0, k1, wave);
      p.init(pm, n0, k0, k1, wave);
    } else {
      q.kend = p.kend = 0;  // (zeros, so that the waits count alike)
    }
    phase<0>(q, p, 0, lds);
    phase<1>(q, p, 1, lds);
    phase<2>(q, p, 2, lds);
    phase<3>(q, p, 3, lds);
    // nothing may still be on its way into LDS when it is given back; the last product takes 8 passes until its sums can be read
    if (!more) meet<0>();
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
    for (int a = 0; a < MF; ++a)
#pragma unroll
      for (int b = 0; b < NF; ++b) asm volatile("" : "+a"(acc[a][b]));
  }
};

}  // namespace npd
