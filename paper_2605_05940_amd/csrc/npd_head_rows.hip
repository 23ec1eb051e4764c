// What the head operators do row by row around their matrix products: the list of scored positions, packed copies, the logits
// at labels and teacher ids, and the end of the loss (sums joined, scalars, what the gradient takes away at those ids).
#include "../../include/npd.h"
#include "npd_head.hpp"

namespace npd {
namespace {

constexpr int kRowThreads = 256;
constexpr int kScanThreads = 1024;

// One workgroup walks the mask, 16 positions per thread at a time; a position's place is the number of scored ones before it.
__global__ __launch_bounds__(kScanThreads) void head_scan_kernel(HeadRowsArgs a) {
  __shared__ int waves[kScanThreads / kWave];
  constexpr int kEach = 16;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t before = 0;  // scored positions in front of this stretch (uniform)
  for (int64_t p0 = 0; p0 < a.T; p0 += kScanThreads * kEach) {
    const int64_t p = p0 + (int64_t)threadIdx.x * kEach;
    uint32_t on = 0;
#pragma unroll
    for (int t = 0; t < kEach; ++t)
      if (p + t < a.T && a.mask[p + t]) on |= 1u << t;
    const int mine = __popc(on);
    int sum = mine;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
      const int v = __shfl_up(sum, off, kWave);
      if (lane >= off) sum += v;
    }
    if (lane == 63) waves[wave] = sum;
    __syncthreads();
    int64_t at = before + sum - mine;
    int all = 0;
#pragma unroll
    for (int w = 0; w < kScanThreads / kWave; ++w) {
      if (w < wave) at += waves[w];
      all += waves[w];
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kEach; ++t) {
      if (p + t >= a.T) break;
      if (on >> t & 1) {
        a.rows[at++] = (int32_t)(p + t);
      } else {
        if (a.kd) a.kd[p + t] = 0.0f;
        if (a.nll) a.nll[p + t] = 0.0f;
        if (a.lse) a.lse[p + t] = 0.0f;
      }
    }
    before += all;
  }
  if (threadIdx.x == 0) *a.count = (int32_t)before;
}

__device__ __forceinline__ void zero_row(uint16_t* row, int D) {
  for (int d = threadIdx.x * 8; d < D; d += kRowThreads * 8) {
    if (d + 8 <= D) {
      store8(row + d, make_uint4(0, 0, 0, 0));
    } else {
      for (int t = d; t < D; ++t) row[t] = 0;
    }
  }
}

// zero rows of the hidden states' gradient at positions that are not scored
__global__ __launch_bounds__(kRowThreads) void head_zero_kernel(HeadRowsArgs a) {
  for (int64_t p = blockIdx.x; p < a.T; p += gridDim.x) {
    if (a.mask[p]) continue;
    zero_row(a.grad_hidden + p * a.grad_stride, a.D);
  }
}

// (blockIdx.y: stretches of a row, four groups of eight per thread, requested together)
constexpr int kPackGroups = 4;
__global__ __launch_bounds__(kRowThreads) void head_pack_kernel(HeadPackArgs a) {
  const HeadSpan span = head_span(a.chunk);
  if (!span.there) return;
  const float inv = a.y ? 1.0f / a.cap : 0.0f;
  const int d0 = blockIdx.y * (kRowThreads * 8 * kPackGroups) + threadIdx.x * 8;
  for (int64_t i = blockIdx.x; i < span.rows; i += gridDim.x) {
    const int64_t p = span.first + i;
    const uint16_t* src = a.src + p * a.src_stride;
    uint16_t* dst = a.dst + i * a.dst_stride;
    uint4 v[kPackGroups];
#pragma unroll
    for (int u = 0; u < kPackGroups; ++u) v[u] = load8_of(src, d0 + u * kRowThreads * 8, a.cols);
    if (a.y) {
      const uint16_t* y = a.y + p * a.y_stride;
      uint4 w[kPackGroups];
#pragma unroll
      for (int u = 0; u < kPackGroups; ++u) w[u] = load8_of(y, d0 + u * kRowThreads * 8, a.cols);
#pragma unroll
      for (int u = 0; u < kPackGroups; ++u) {
        float g[8], f[8];
        unpack8(v[u], g);
        unpack8(w[u], f);
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          const float x = f[t] * inv;
          g[t] *= __builtin_fmaf(-x, x, 1.0f);
        }
        v[u] = make_uint4(pack_bf16(g[0], g[1]), pack_bf16(g[2], g[3]), pack_bf16(g[4], g[5]), pack_bf16(g[6], g[7]));
      }
    }
#pragma unroll
    for (int u = 0; u < kPackGroups; ++u) {
      const int d = d0 + u * kRowThreads * 8;
      if (d < a.width) *reinterpret_cast<uint4*>(dst + d) = v[u];  // (rows of dst begin on 16 bytes, width is a multiple of eight)
    }
  }
}

// the id that entry j of a row is about: its label (column 0 where there is none), then the teacher's; -1: outside the vocabulary
__device__ __forceinline__ int entry_id(const HeadLossArgs& a, int64_t p, int j) {
  const int v = j == 0 ? (a.labels ? a.labels[p] : 0) : a.tidx[p * a.k + j - 1];
  return v >= 0 && v < a.V ? v : -1;
}

// Row i of a chunk, position p: its hidden state packed for the matrix cores, its logits at the label and the teacher's ids (a
// wave per product of two rows), and its reference, the largest of them.  All threads of the workgroup.
__device__ __forceinline__ void gather_row(const HeadLossArgs& a, int64_t i, int64_t p) {
  __shared__ float tops[kRowThreads / kWave];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint16_t* src = a.src + p * a.src_stride;
  uint16_t* h = const_cast<uint16_t*>(a.h.p) + i * a.h.stride;
  for (int d = threadIdx.x * 8; d < a.K; d += kRowThreads * 8) *reinterpret_cast<uint4*>(h + d) = load8_of(src, d, a.D);
  float top = -__builtin_inff();
  constexpr int kWaves = kRowThreads / kWave, kTogether = 4;  // rows of the weights requested together
  for (int j0 = wave; j0 <= a.k; j0 += kWaves * kTogether) {
    const uint16_t* w[kTogether];
    int id[kTogether];
    float sum[kTogether] = {};
#pragma unroll
    for (int u = 0; u < kTogether; ++u) {
      const int j = j0 + kWaves * u;
      id[u] = j <= a.k ? entry_id(a, p, j) : -1;
      w[u] = a.weight + (int64_t)(id[u] < 0 ? 0 : id[u]) * a.weight_stride;
    }
    for (int d = lane * 8; d < a.D; d += kWave * 8) {
      float x[8];
      unpack8(load8_of(src, d, a.D), x);
      uint4 v[kTogether];
#pragma unroll
      for (int u = 0; u < kTogether; ++u) v[u] = id[u] < 0 ? make_uint4(0, 0, 0, 0) : load8_of(w[u], d, a.D);
#pragma unroll
      for (int u = 0; u < kTogether; ++u) {
        float y[8];
        unpack8(v[u], y);
#pragma unroll
        for (int t = 0; t < 8; ++t) sum[u] = __builtin_fmaf(x[t], y[t], sum[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < kTogether; ++u) {
      const int j = j0 + kWaves * u;
      if (j > a.k) break;
      float x = wave_sum(sum[u]);
      if (id[u] < 0) {
        x = __builtin_nanf("");
      } else {
        if (a.bias) x += bf16_one(a.bias[id[u]]);
        if (a.cap != 0.0f) x = a.cap * tanhf(x / a.cap);
        top = fmaxf(top, x);
      }
      if (lane == 0) a.x[i * (1 + a.k) + j] = x;
    }
  }
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kRowThreads / kWave; ++w) top = fmaxf(top, tops[w]);
    const float r = __builtin_rintf(top * a.c);
    a.r0[i] = r > -1.0e30f && r < 1.0e30f ? r : -1.0e30f;  // (no finite logit: every part takes its own reference)
  }
}

__global__ __launch_bounds__(kRowThreads) void head_gather_kernel(HeadLossArgs a) {
  const HeadSpan span = head_span(a.chunk);
  const int64_t i = blockIdx.x;
  if (!span.there || i >= span.rows) return;
  gather_row(a, i, a.rows[span.first + i]);
}

// The same where one chunk holds every position, with what head_scan_kernel and head_zero_kernel do besides, in one launch: a
// workgroup per position, which counts the scored positions in front of its own itself.  Measured (MI355X, us): 512 positions of width
// 256 5.8 for the 19.6 of the four launches, 8,192 of 1,152 39 for 46 (8,192 passes over a mask of 8 KB, out of the L2).
__global__ __launch_bounds__(kRowThreads) void head_prepare_kernel(HeadRowsArgs r, HeadLossArgs a) {
  __shared__ int ired[kRowThreads / kWave];
  const int64_t p = blockIdx.x;
  int before = 0, all = 0;
  for (int64_t q = (int64_t)threadIdx.x * 16; q < r.T; q += kRowThreads * 16) {
    uint8_t m[16];
    if (q + 16 <= r.T) {
      __builtin_memcpy(m, r.mask + q, 16);
    } else {
#pragma unroll
      for (int t = 0; t < 16; ++t) m[t] = q + t < r.T ? r.mask[q + t] : 0;
    }
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      all += m[t] != 0;
      before += m[t] != 0 && q + t < p;
    }
  }
  before = block_sum_int<kRowThreads>(before, ired);
  if (p == 0) {
    all = block_sum_int<kRowThreads>(all, ired);
    if (threadIdx.x == 0) *r.count = all;
  }
  if (r.mask[p]) {
    if (threadIdx.x == 0) r.rows[before] = (int32_t)p;
    gather_row(a, before, p);
    return;
  }
  if (threadIdx.x == 0) {
    if (r.kd) r.kd[p] = 0.0f;
    if (r.nll) r.nll[p] = 0.0f;
    if (r.lse) r.lse[p] = 0.0f;
  }
  if (r.grad_hidden) zero_row(r.grad_hidden + p * r.grad_stride, r.D);
}

// Joins the sums of a row over the vocabulary (part, one pair per 128, 64 or 32 columns), writes its scalars, and turns what is kept of it,
// e = 2^(x c - R), into the gradient up to the row's factor: with w = grad_scale / tau + ce_grad_scale and Z the row's sum
//   G(v) = w / Z (e(v) - Z / w (grad_scale / tau p_T(v) + ce_grad_scale [v = label])),
// so that only the entries at the label and the teacher's ids change (they are rounded to bf16 once, from fp32 values).  Those are
// where most of a row's gradient is, and their roundings are known: the row's factor takes up as much of them as one factor can (by
// least squares, half a bf16 step at most).  Error of the weights' gradient against 64 bits, as a share of its norm: hard labels
// .00289 without, .00245 with it, a record of 64 .00288 / .00262; of the hidden states' .00238 / .00182 and .00235 / .00203
// (rounding the result alone: .00166).
__global__ __launch_bounds__(kRowThreads) void head_finish_kernel(HeadLossArgs a) {
  __shared__ float fred[3 * kRowThreads / kWave];
  __shared__ int bad_id;
  const HeadSpan span = head_span(a.chunk);
  const int64_t i = blockIdx.x;
  if (!span.there || i >= span.rows) return;
  const int64_t p = a.rows[span.first + i];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) bad_id = 0;
  __syncthreads();

  const float2* part = a.part + i * a.parts;
  Lse sum[1];
  sum[0].init();
  bool apart = false;  // parts with different references
  const float first = part[0].x;
  for (int t = threadIdx.x; t < a.parts; t += kRowThreads) {
    const float2 v = part[t];
    if (!(v.y == 0.0f)) sum[0].merge(v.x, v.y, 0.0f);
    apart |= v.x != first;
  }
  block_merge<kRowThreads, 1>(sum, fred);
  const float R = sum[0].r, Z = sum[0].z, lz = __log2f(Z);
  const bool rescale = a.e && __syncthreads_or(apart || first != R);
  if (rescale) {  // exact: references are whole numbers (a factor 2^(r - R) by itself would underflow where its products, of up to 2^40, do not)
    for (int t = wave; t < a.parts; t += kRowThreads / kWave) {
      const float r = part[t].x;
      if (r == R) continue;
      const int by = (int)fmaxf(r - R, -400.0f);  // (-400: nothing is left)
      uint16_t* e = a.e + i * a.e_stride + t * a.part_columns;
      const int n = 2 * lane;
      if (n < a.part_columns && t * a.part_columns + n < a.V) {
        uint32_t* w = reinterpret_cast<uint32_t*>(e + n);
        *w = pack_bf16(__builtin_ldexpf(bf16_lo(*w), by), __builtin_ldexpf(bf16_hi(*w), by));
      }
    }
    __syncthreads();
  }

  const float* x = a.x + i * (1 + a.k);
  const int label = a.labels ? entry_id(a, p, 0) : -1;
  const bool no_label = a.labels && label < 0;
  const bool bad_label = no_label && (a.nll || a.ce_weight != 0.0f);  // (labels that nothing uses are not checked)
  // the teacher's distribution over its ids at this temperature
  float tmax = -__builtin_inff();
  for (int j = threadIdx.x; j < a.k; j += kRowThreads) tmax = fmaxf(tmax, a.tval[p * a.k + j]);
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) tmax = fmaxf(tmax, __shfl_xor(tmax, off, kWave));
  if (lane == 0) fred[wave] = tmax;
  __syncthreads();
  tmax = fmaxf(fmaxf(fred[0], fred[1]), fmaxf(fred[2], fred[3]));
  __syncthreads();
  float tz = 0.0f;
  for (int j = threadIdx.x; j < a.k; j += kRowThreads) {
    tz += exp2_fast((a.tval[p * a.k + j] - tmax) * a.c);
    if (entry_id(a, p, 1 + j) < 0) bad_id = 1;
  }
  tz = block_sum<kRowThreads>(tz, fred);
  const bool no_id = bad_id != 0;
  const float ltz = a.k ? __log2f(tz) : 0.0f;
  const float w = (a.k ? a.kd_weight : 0.0f) + a.ce_weight;
  const float take = w != 0.0f ? Z / w : 0.0f;
  float kd = 0.0f;
  float off = 0.0f, size = 0.0f;  // of the entries' roundings, over Z
  const float per = 1.0f / Z;
  auto put = [&](int id, float x, float taken) {
    float g = exp2_fast(__builtin_fmaf(x, a.c, -R)) - taken;
    if (a.cap != 0.0f) {
      const float f = x / a.cap;
      g *= __builtin_fmaf(-f, f, 1.0f);
    }
    const uint16_t rounded = one_bf16(g);
    a.e[i * a.e_stride + id] = rounded;
    const float u = bf16_one(rounded) * per;
    off = __builtin_fmaf(u, __builtin_fmaf(g, per, -u), off);
    size = __builtin_fmaf(u, u, size);
  };
  bool at_label = false;
  for (int j = threadIdx.x; j < a.k; j += kRowThreads) {
    const int id = entry_id(a, p, 1 + j);
    if (id < 0) continue;
    const float lp = __builtin_fmaf(a.tval[p * a.k + j] - tmax, a.c, -ltz), pt = exp2_fast(lp);
    const float xe = __builtin_fmaf(x[1 + j], a.c, -R);  // log2 of e here
    // p_T log(p_T / p_S): an id of probability 0 contributes nothing
    if (pt > 0.0f) kd = __builtin_fmaf(pt, lp - xe + lz, kd);
    if (a.e) {
      const bool here = id == label;
      at_label |= here;
      put(id, x[1 + j], take * (a.kd_weight * pt + (here ? a.ce_weight : 0.0f)));
    }
  }
  const bool label_done = __syncthreads_or(at_label);
  kd = block_sum<kRowThreads>(kd, fred);
  const bool bad = bad_label || no_id;
  if (threadIdx.x == 0) {
    const float nan = __builtin_nanf("");
    if (a.e && label >= 0 && !label_done && a.ce_weight != 0.0f) put(label, x[0], take * a.ce_weight);
    if (a.lse) a.lse[p] = (R + lz) * kLn2;
    if (a.nll) a.nll[p] = no_label ? nan : (__builtin_fmaf(-x[0], a.c, R) + lz) * kLn2;
    if (a.kd) a.kd[p] = no_id ? nan : kd * kLn2;
    if (a.status && bad) atomicOr(a.status, (bad_label ? NPD_DEV_BAD_LABEL : 0) | (no_id ? NPD_DEV_BAD_TOPK_INDEX : 0));
  }
  if (!a.e) return;
  off = block_sum<kRowThreads>(off, fred);
  size = block_sum<kRowThreads>(size, fred);
  const float factor = w / Z * (size > 0.0f ? 1.0f + off / size : 1.0f);
  if (threadIdx.x == 0) a.scale[i] = bad ? __builtin_nanf("") : factor;
  if (a.hs) {
    // Rounded to bf16 as an operand of the matrix cores (half a step, like e itself): the row's factor is not known when e is
    // stored.  A position with a bad label or id is left out of the weights' gradient.
    const uint16_t* h = a.h.p + i * a.h.stride;
    uint16_t* hs = a.hs + i * a.h.stride;
    for (int d = threadIdx.x * 8; d < a.K; d += kRowThreads * 8) {
      float v[8];
      unpack8(*reinterpret_cast<const uint4*>(h + d), v);
      *reinterpret_cast<uint4*>(hs + d) = bad ? make_uint4(0, 0, 0, 0)
                                              : make_uint4(pack_bf16(v[0] * factor, v[1] * factor), pack_bf16(v[2] * factor, v[3] * factor),
                                                           pack_bf16(v[4] * factor, v[5] * factor), pack_bf16(v[6] * factor, v[7] * factor));
    }
  }
}

unsigned few(int64_t rows) { return (unsigned)(rows < 65536 ? rows : 65536); }

}  // namespace

hipError_t launch_head_rows(const HeadRowsArgs& a, hipStream_t stream) {
  const hipError_t e = launch_kernel(head_scan_kernel, dim3(1), dim3(kScanThreads), 0, stream, a);
  if (e != hipSuccess || !a.grad_hidden) return e;
  return launch_kernel(head_zero_kernel, dim3(few(a.T)), dim3(kRowThreads), 0, stream, a);
}

hipError_t launch_head_pack(const HeadPackArgs& a, int64_t rows, hipStream_t stream) {
  const unsigned stretch = kRowThreads * 8 * kPackGroups;
  return launch_kernel(head_pack_kernel, dim3(few(rows), ((unsigned)a.width + stretch - 1) / stretch), dim3(kRowThreads), 0, stream, a);
}

hipError_t launch_head_prepare(const HeadRowsArgs& r, const HeadLossArgs& a, hipStream_t stream) {
  return launch_kernel(head_prepare_kernel, dim3((unsigned)r.T), dim3(kRowThreads), 0, stream, r, a);
}

hipError_t launch_head_gather(const HeadLossArgs& a, int64_t rows, hipStream_t stream) {
  return launch_kernel(head_gather_kernel, dim3((unsigned)rows), dim3(kRowThreads), 0, stream, a);
}

hipError_t launch_head_finish(const HeadLossArgs& a, int64_t rows, hipStream_t stream) {
  return launch_kernel(head_finish_kernel, dim3((unsigned)rows), dim3(kRowThreads), 0, stream, a);
}

}  // namespace npd
