// A token from a row of logits: temperature, top-k, top-p, min-p, and the entry that a given random number falls on.
//
// Entries are ordered by logit, equal ones by id.  What is kept is the first n of that order, and the token is the first whose
// cumulative weight 2^((x - top) log2(e) / tau) exceeds u times the sum of the first n.  Which entry that is changes with the last
// bits of the sums where many entries are alike, so they are 64-bit.  That is cheap because bf16 has few values: a row's entries are
// counted by value (whole numbers in LDS, exact in any order), and every value that occurs is weighed once, times its count.
//
// The 7,937 values of magnitude 2^-23 .. 2^8 and zero have a counter each; a row with an entry outside of them that may matter is
// done by bisection over the values instead, with a pass over the row for each step.
#include "../../include/npd.h"
#include "npd_device.hpp"
#include "npd_sample.hpp"

namespace npd {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;

// bf16 bits in the order of their values: 0 and -0 alike, -inf below every number, NaN at either end
constexpr uint32_t kLowest = 0x80, kInfinity = 0xff80;  // keys of the lowest number and of +inf
__device__ __forceinline__ uint32_t key_of(uint32_t b) {
  return b & 0x8000 ? (b == 0x8000 ? 0x8000u : ~b & 0xffffu) : b | 0x8000;
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return bf16_one((uint16_t)(key & 0x8000 ? key & 0x7fff : ~key & 0xffffu));
}

// counters: 3,968 positive values by magnitude, as many negative ones, zero
constexpr uint32_t kFirst = (127 - 23) << 7, kValues = 31 << 7;
constexpr int kEach = 8, kOwners = kValues / kEach;  // a thread has eight values; thread kOwners zero
static_assert(2 * kOwners + 1 <= kThreads, "");

struct Place {       // where a search over the order ended
  uint32_t key, before, here;  // the value; entries above it, entries of it
  double mass;       // of those above it
};

struct Shared {
  uint32_t counts[2 * kValues + 1];
  double masses[2][kWaves];
  uint32_t sums[kWaves];
  uint32_t big, odd, first;
  int32_t found;
  Place place;
};

struct Row {
  const uint16_t* p;
  int V;
  RowSplit split;
};

// f(id, bits) of the row's entries: groups of eight, kAhead of them requested together, then what is left
template <class F>
__device__ __forceinline__ void each_entry(const Row& r, F&& f) {
  constexpr int kAhead = 4;
  const uint4* groups = reinterpret_cast<const uint4*>(r.p + r.split.head);
  auto eight = [&](int g, const uint4& v) {
    const int id = r.split.head + 8 * g;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      f(id + 2 * t, w[t] & 0xffff);
      f(id + 2 * t + 1, w[t] >> 16);
    }
  };
  int g = threadIdx.x;
  for (; g + (kAhead - 1) * kThreads < r.split.nvec; g += kAhead * kThreads) {
    uint4 v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = groups[g + u * kThreads];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) eight(g + u * kThreads, v[u]);
  }
  for (; g < r.split.nvec; g += kThreads) eight(g, groups[g]);
  for (int j = threadIdx.x; j < r.V - 8 * r.split.nvec; j += kThreads) {
    const int id = r.split.edge_elem(j);
    f(id, (uint32_t)r.p[id]);
  }
}

// in wave order, so that every thread has the same sum
__device__ __forceinline__ double block_sum64(double v, double* smem) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) smem[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = smem[0];
  for (int w = 1; w < kWaves; ++w) s += smem[w];
  return s;
}
__device__ __forceinline__ uint32_t block_count(uint32_t v, uint32_t* smem) {
  v = (uint32_t)wave_sum_int((int)v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) smem[threadIdx.x >> 6] = v;
  __syncthreads();
  uint32_t s = 0;
  for (int w = 0; w < kWaves; ++w) s += smem[w];
  return s;
}

__device__ __forceinline__ double weight_of(uint32_t key, double top, double tau) {
  return exp(((double)value_of(key) - top) / tau);
}

enum Find { kCount, kMassReaches, kMassExceeds };

// A row by passes over it: counts and masses of its entries from a value on, and the value at which they reach something.
struct Passes {
  const Row& row;
  Shared& s;
  uint32_t top_key, all;
  double top, tau, sum;
  __device__ __forceinline__ void from(uint32_t key, double at_tau, uint32_t* count, double* mass) const {
    uint32_t n = 0;
    double m = 0.0;
    each_entry(row, [&](int, uint32_t b) {
      const uint32_t k = key_of(b);
      if (k < key || k < kLowest) return;
      ++n;
      m += weight_of(k, top, at_tau);
    });
    *count = block_count(n, s.sums);
    *mass = block_sum64(m, s.masses[0]);
  }
  __device__ __forceinline__ void begin(double at_tau) {
    tau = at_tau;
    from(kLowest, tau, &all, &sum);
  }
  __device__ __forceinline__ double sum_at(double at_tau) const {
    uint32_t n;
    double m;
    from(kLowest, at_tau, &n, &m);
    return m;
  }
  // how many weigh `least` and more
  __device__ __forceinline__ uint32_t at_least(double least) const {
    uint32_t n = 0;
    each_entry(row, [&](int, uint32_t b) {
      const uint32_t k = key_of(b);
      n += k >= kLowest && weight_of(k, top, tau) >= least;
    });
    return block_count(n, s.sums);
  }
  __device__ __forceinline__ Place find(Find what, uint32_t count, double mass) const {
    // the largest value from which on there is enough; the lowest one has all there is
    uint32_t lo = kLowest, hi = top_key + 1, n_lo = all, n_hi = 0;
    double m_hi = 0.0;
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      uint32_t n;
      double m;
      from(mid, tau, &n, &m);
      const bool enough = what == kCount ? n >= count : what == kMassReaches ? m >= mass : m > mass;
      if (enough) {
        lo = mid;
        n_lo = n;
      } else {
        hi = mid;
        n_hi = n;
        m_hi = m;
      }
    }
    return Place{lo, n_hi, n_lo - n_hi, m_hi};
  }
};

// A row whose entries are counted: the values' counts and masses are in registers, eight values to a thread, in their order.
struct Counted {
  Shared& s;
  uint32_t top_key, all;
  double top, tau, sum;
  uint32_t n[kEach], before, after;  // of the thread's first and behind its last value
  double m[kEach], mass_before, mass_after;

  static __device__ __forceinline__ uint32_t key(int e) {
    const int t = threadIdx.x;
    if (t < kOwners) return 0x8000u + kFirst + kValues - 1 - (uint32_t)(t * kEach + e);
    if (t == kOwners) return 0x8000u;
    return ~(0x8000u + kFirst + (uint32_t)((t - kOwners - 1) * kEach + e)) & 0xffffu;
  }
  __device__ __forceinline__ void read() {
    const int t = threadIdx.x;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      n[e] = 0;
      if (t < kOwners) n[e] = s.counts[kValues - 1 - (t * kEach + e)];
      if (t == kOwners && e == 0) n[e] = s.counts[2 * kValues];
      if (t > kOwners && t <= 2 * kOwners) n[e] = s.counts[kValues + (t - kOwners - 1) * kEach + e];
    }
    // the first thread that has any has the largest
    uint32_t mine = 0;
#pragma unroll
    for (int e = kEach - 1; e >= 0; --e)
      if (n[e]) mine = key(e);
    const uint64_t any = __ballot(mine != 0);
    __syncthreads();
    if ((t & 63) == 0) s.sums[t >> 6] = 0;
    if (any && (t & 63) == __builtin_ctzll(any)) s.sums[t >> 6] = mine;
    __syncthreads();
    top_key = 0;
    for (int w = kWaves - 1; w >= 0; --w)
      if (s.sums[w]) top_key = s.sums[w];
    top = top_key ? value_of(top_key) : 0.0;
    __syncthreads();
  }
  __device__ __forceinline__ double sum_at(double at_tau) const {
    double mine = 0.0;
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (n[e]) mine += n[e] * weight_of(key(e), top, at_tau);
    return block_sum64(mine, s.masses[0]);
  }
  // cumulative counts and masses; a thread's end is the next one's beginning, bit by bit
  __device__ __forceinline__ void begin(double at_tau) {
    tau = at_tau;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t c = 0;
    double w = 0.0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      m[e] = n[e] ? n[e] * weight_of(key(e), top, tau) : 0.0;
      c += n[e];
      w += m[e];
    }
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
      const uint32_t c2 = __shfl_up(c, off, kWave);
      const double w2 = __shfl_up(w, off, kWave);
      if (lane >= off) {
        c += c2;
        w = w2 + w;
      }
    }
    __syncthreads();
    if (lane == 63) {
      s.sums[wave] = c;
      s.masses[0][wave] = w;
    }
    __syncthreads();
    uint32_t c0 = 0;
    double w0 = 0.0;
    before = 0;
    mass_before = 0.0;
    for (int i = 0; i < kWaves; ++i) {
      if (i == wave) {
        before = c0;
        mass_before = w0;
      }
      c0 += s.sums[i];
      w0 += s.masses[0][i];
    }
    all = c0;
    sum = w0;
    const uint32_t c1 = __shfl_up(c, 1, kWave);
    const double w1 = __shfl_up(w, 1, kWave);
    after = before + c;
    mass_after = mass_before + w;
    if (lane > 0) {
      before += c1;
      mass_before += w1;
    }
    __syncthreads();
  }
  __device__ __forceinline__ uint32_t at_least(double least) const {
    uint32_t mine = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (n[e] && weight_of(key(e), top, tau) >= least) mine += n[e];
    return block_count(mine, s.sums);
  }
  // (there is enough: what is asked for is at most what there is; the last value there is takes what rounding leaves over)
  __device__ __forceinline__ Place find(Find what, uint32_t count, double mass) const {
    if (threadIdx.x == 0) s.first = kThreads;
    __syncthreads();
    const bool enough = what == kCount ? after >= count : what == kMassReaches ? mass_after >= mass : mass_after > mass;
    const bool last = after == all;  // the thread of the lowest value, and those behind it
    if (after != before && (enough || last)) atomicMin(&s.first, threadIdx.x);
    __syncthreads();
    if (threadIdx.x == s.first) {
      uint32_t c = before;
      double w = mass_before;
      Place p{};
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const bool done = p.here && (what == kCount ? c >= count : what == kMassReaches ? w >= mass : w > mass);
        // (what rounding leaves over is not an entry's of weight 0)
        if (!done && n[e] && (what == kCount || !p.here || m[e] > 0.0)) p = Place{key(e), c, n[e], w};
        c += n[e];
        w += m[e];
      }
      s.place = p;
    }
    __syncthreads();
    return s.place;
  }
};

// The settings of a row.
struct Settings {
  double tau, top_p, min_p, u;
  uint32_t top_k;
};

struct Choice {
  uint32_t key, kept, which;  // the token's value, and its place among the entries of that value
  double logprob;
};

template <class Entries>
__device__ __forceinline__ Choice choose(const Entries& x, const Settings& q, bool greedy) {
  uint32_t n = q.top_k > 0 && q.top_k < x.all ? q.top_k : x.all;
  if (greedy) n = 1;
  Place end{};  // where the first n end
  double sum = x.sum;
  auto cut = [&]() {
    if (n == x.all) {
      sum = x.sum;
      return;
    }
    end = x.find(kCount, n, 0.0);
    sum = end.mass + (double)(n - end.before) * weight_of(end.key, x.top, x.tau);
  };
  cut();
  const uint32_t by_k = n;
  if (q.top_p < 1.0 && n > 1) {
    const double enough = q.top_p * sum;
    const Place p = x.find(kMassReaches, 0, enough);
    const double more = ceil((enough - p.mass) / weight_of(p.key, x.top, x.tau));
    const uint32_t here = more < 1.0 ? 1 : more < (double)p.here ? (uint32_t)more : p.here;
    if (p.before + here < n) n = p.before + here;
  }
  if (q.min_p > 0.0 && n > 1) {
    const uint32_t least = x.at_least(q.min_p);
    if (least < n) n = least;
  }
  if (n < 1) n = 1;
  if (n != by_k) cut();
  const double at = q.u * sum;
  Place p = n == 1 ? Place{x.top_key, 0, 1, 0.0} : x.find(kMassExceeds, 0, at);
  uint32_t here = p.here;
  if (n != x.all && n > 1) {
    if (p.before >= end.before) p = end;  // (no further than the last one that is kept)
    if (p.key == end.key) here = n - end.before;
  }
  const double steps = floor((at - p.mass) / weight_of(p.key, x.top, x.tau));
  const uint32_t which = !(steps > 0.0) ? 0 : steps < (double)here ? (uint32_t)steps : here - 1;
  return Choice{p.key, n, which, ((double)value_of(p.key) - x.top) / x.tau - log(sum)};
}

// id of the entry `which` (in order of ids) of those of a value
__device__ __forceinline__ int find_entry(const Row& row, uint32_t key, uint32_t which, Shared& s) {
  if (threadIdx.x == 0) s.found = 0x7fffffff;
  __syncthreads();
  if (which == 0) {
    each_entry(row, [&](int id, uint32_t b) {
      if (key_of(b) == key) atomicMin(&s.found, id);
    });
    __syncthreads();
    return s.found;
  }
  // every wave counts in a stretch of its own, and the one that has it looks again
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int each = ((row.V + kWaves - 1) / kWaves + kWave - 1) / kWave * kWave;
  const int begin = wave * each < row.V ? wave * each : row.V, end = row.V - begin < each ? row.V : begin + each;
  uint32_t n = 0;
  for (int i = begin + lane; i < end; i += kWave) n += key_of(row.p[i]) == key;
  n = (uint32_t)wave_sum_int((int)n);
  if (lane == 0) s.sums[wave] = n;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < wave; ++w) before += s.sums[w];
  if (which >= before && which - before < n) {
    uint32_t left = which - before;
    for (int i = begin; i < end; i += kWave) {
      const bool is = i + lane < end && key_of(row.p[i + lane]) == key;
      const uint64_t all = __ballot(is);
      const uint32_t here = (uint32_t)__popcll(all);
      if (left < here) {
        if (is && (uint32_t)__popcll(all & ((1ull << lane) - 1)) == left) s.found = i + lane;
        break;
      }
      left -= here;
    }
  }
  __syncthreads();
  return s.found;
}

// A row by passes over it (not inlined: the registers of the rows that are counted are the ones that matter); false: not a row to
// draw from.
__device__ __attribute__((noinline)) bool by_passes(const Row row, const Settings q, bool greedy, bool nll, Shared& s, Choice* c, double* sum1,
                                                    double* top) {
  uint32_t most = 0, bad = 0;
  each_entry(row, [&](int, uint32_t b) {
    const uint32_t k = key_of(b);
    most = most > k ? most : k;
    bad |= k >= kInfinity || k < 0x7f;  // (0x7f: -inf)
  });
  __syncthreads();
  if (threadIdx.x == 0) s.first = s.odd = 0;
  __syncthreads();
  atomicMax(&s.first, most);
  if (bad) s.odd = 1;
  __syncthreads();
  most = s.first;
  bad = s.odd;
  __syncthreads();
  if (bad || most < kLowest) return false;
  Passes passes{row, s, most, 0, value_of(most), 0.0, 0.0};
  passes.begin(q.tau);
  *c = choose(passes, q, greedy);
  *sum1 = !nll ? 1.0 : q.tau == 1.0 ? passes.sum : passes.sum_at(1.0);
  *top = passes.top;
  return true;
}

__global__ __launch_bounds__(kThreads, 8) void sample_kernel(SampleArgs a) {
  __shared__ Shared s;
  for (int64_t r = blockIdx.x; r < a.T; r += gridDim.x) {
    auto put = [&](int token, double logprob, double nll, uint32_t kept, int status) {
      if (threadIdx.x != 0) return;
      a.token[r] = token;
      if (a.logprob) a.logprob[r] = (float)logprob;
      if (a.nll) a.nll[r] = (float)nll;
      if (a.kept) a.kept[r] = (int32_t)kept;
      if (status && a.status) atomicOr(a.status, status);
    };
    const double nan = __builtin_nan("");
    if (a.mask && !a.mask[r]) {
      put(-1, 0.0, 0.0, 0, 0);
      continue;
    }
    const float tau = a.taus ? a.taus[r] : a.tau, top_p = a.top_ps ? a.top_ps[r] : a.top_p, min_p = a.min_ps ? a.min_ps[r] : a.min_p;
    const int top_k = a.top_ks ? a.top_ks[r] : a.top_k;
    const float u = a.u[r];
    if (!(tau >= 0.0f && tau <= 3.4028234663852886e38f) || !(top_p >= 0.0f && top_p <= 1.0f) || !(min_p >= 0.0f && min_p <= 1.0f) || top_k < 0 ||
        !(u >= 0.0f && u < 1.0f)) {
      put(-1, nan, nan, 0, NPD_DEV_BAD_SAMPLING);
      continue;
    }
    const bool greedy = tau == 0.0f;
    const Settings q = {greedy ? 1.0 : (double)tau, top_p, min_p, u, (uint32_t)top_k};
    const Row row = {a.x + r * a.stride, a.V, row_split(a.x + r * a.stride, a.V, true)};

    for (int i = threadIdx.x; i < (int)(2 * kValues + 1); i += kThreads) s.counts[i] = 0;
    if (threadIdx.x == 0) s.big = s.odd = 0;
    __syncthreads();
    uint32_t big = 0, odd = 0;  // large negative numbers; entries that have no counter otherwise
    each_entry(row, [&](int, uint32_t b) {
      const uint32_t size = b & 0x7fff, i = size - kFirst;
      if (i < kValues) {
        atomicAdd(&s.counts[i + (b >> 15) * kValues], 1u);
      } else if (size == 0) {
        atomicAdd(&s.counts[2 * kValues], 1u);
      } else if (b != 0xff80) {
        if (b >= 0x8000 + kFirst + kValues && b < 0xff80)
          ++big;
        else
          odd = 1;
      }
    });
    if (big) atomicAdd(&s.big, big);
    if (odd) s.odd = 1;
    __syncthreads();
    big = s.big;
    odd = s.odd;
    Choice c;
    double sum1 = 1.0, top;  // of the weights at temperature 1
    Counted counted{s};
    counted.read();
    // Numbers below -256 have no weight that 64 bits would show beside the largest's (2^-90 times at most 2^26 of them) where that is
    // 64 temperatures above -256, and are none that a min-p would keep.
    const double room = counted.top + 256.0;
    const bool apart = room >= 64.0 && room >= 64.0 * q.tau && (q.min_p == 0.0 || room > q.tau * (1.0 - log(q.min_p)));
    if (!odd && counted.top_key && (!big || apart)) {
      counted.begin(q.tau);
      c = choose(counted, q, greedy);
      // those that are kept if nothing is cut off
      if (c.kept == counted.all && big) c.kept = !greedy && q.min_p == 0.0 && q.top_p == 1.0 ? (q.top_k > 0 && q.top_k < counted.all + big ? q.top_k : counted.all + big) : c.kept;
      if (a.nll) sum1 = q.tau == 1.0 ? counted.sum : counted.sum_at(1.0);
      top = counted.top;
    } else {
      if (!by_passes(row, q, greedy, a.nll != nullptr, s, &c, &sum1, &top)) {
        put(-1, nan, nan, 0, NPD_DEV_BAD_LOGITS);
        continue;
      }
    }
    const int token = find_entry(row, c.key, c.which, s);
    put(token, c.logprob, log(sum1) + (top - (double)value_of(c.key)), c.kept, 0);
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, hipStream_t stream) {
  return launch_kernel(sample_kernel, dim3((unsigned)(a.T < 65536 ? a.T : 65536)), dim3(kThreads), 0, stream, a);
}

}  // namespace npd
