// A token from a row of logits: temperature, top-k, top-p, min-p, and the entry that a given random number falls on.
//
// Entries are ordered by logit, equal ones by id.  What is kept is the first n of that order, and the token is the first whose
// cumulative weight exp((x - top) / tau) exceeds u times the sum of the first n.  Which entry that is changes with the last bits of the
// sums where many entries are alike, so they are 64-bit.  That is cheap because bf16 has few values: a row's entries are counted by
// value (whole numbers in LDS, exact in any order), and every value that occurs is weighed once, times its count.
//
// The 7,936 values of magnitude 2^-23 .. 2^8 have a counter each, zero and up to 255 entries closer to zero are listed; a row with
// more of those, or an entry beyond 2^8 that may matter, is done by bisection over the values, with a pass over the row for each step.
//
// Counting bounds it: eleven vector instructions and two LDS additions for a pair of entries (262,144 take a compute unit 16 us, where
// its share of the memory's rate would be 20), then some 6 us of dependent steps, most of them one wave's or between barriers.
// Measured (MI355X, us): 256 rows of 151,936, temperature 0.7, top-k 50, top-p 0.9: 26.9 (by the clock in an instrumented build: read and
// counted 11.3, largest value 1, weights 2.8, search 2.2, the token's id .5 to 5); one row of 262,144, untruncated, in eight parts 17.0,
// whole 34; 2,048 rows of 151,936 greedy 148 (4.2 TB/s), untruncated 193: where the token's value occurs more than once its row is read
// again.  4,096 rows of 1,000 take 60 greedy, 67 untruncated and 80 with that top-k and top-p: rows that short are not what this is made
// for.  (With longer steps, 112 then, workgroups of 512 threads, three to a compute unit, were 8 to 13 % faster for those, and 16 %
// slower for 48 rows of 50,003.)  By bisection, with logits of a spread of 1,000, 48 rows of 50,003 take 321 untruncated and 1,060 with
// top-k and top-p (14 and 15 counted), 256 of 151,936 803 and 2,705 (34 and 28): 16 passes for each of one to four searches.
#include <stddef.h>

#include "../../include/npd.h"
#include "npd_head_gemm.hpp"
#include "npd_sample.hpp"

namespace npd {
namespace {

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 1024, kWaves = kThreads / kWave;

// threadIdx.x, of which the compiler keeps nothing from one phase of a row to the next (places and keys of eight values, spilled to
// memory over the whole row, took longer than the phases)
__device__ __forceinline__ int thread_of_phase() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// bf16 bits in the order of their values: 0 and -0 alike, -inf below every number, NaN at either end
constexpr uint32_t kLowest = 0x80, kInfinity = 0xff80;  // keys of the lowest number and of +inf
__device__ __forceinline__ uint32_t key_of(uint32_t b) {
  return b & 0x8000 ? (b == 0x8000 ? 0x8000u : ~b & 0xffffu) : b | 0x8000;
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return bf16_one((uint16_t)(key & 0x8000 ? key & 0x7fff : ~key & 0xffffu));
}

// counters: 2 i + sign of the 3,968 magnitudes i, 64 that take what has none
constexpr uint32_t kFirst = (127 - 23) << 7, kValues = 31 << 7, kOthers = 2 * kValues;
constexpr int kTable = 64;  // of the exponential
// a thread has eight values: the positive ones, what is close to zero, the negative ones
constexpr int kEach = 8, kOwners = kValues / kEach, kNear = 256;
static_assert(2 * kOwners + kNear / kEach == kThreads, "");
constexpr uint32_t kBelowNear = 0x8000 - kFirst;  // key below those of what is close to zero

struct Place {       // where a search over the order ended
  uint32_t key, before, here;  // the value; entries above it, entries of it
  double mass;       // of those above it
  double weight;     // of one of them
};

struct Choice {
  uint32_t key, kept, which;  // the token's value, and its place among the entries of that value
  double logit, sum;          // less the largest one, over tau; of the weights of what is kept
};

struct Shared {
  __attribute__((aligned(16))) uint32_t counts[kOthers + kWave];
  double mass_ends[kThreads + 1];  // of the stretches before
  double table[kTable];
  uint32_t count_ends[kThreads + 1];
  double masses[2][kWaves];
  uint32_t near_list[kNear], near_keys[kNear], near_counts[kNear];  // as they came; in order, and how many have that value
  uint32_t sums[kWaves];
  uint32_t big, odd, near, first, listed;
  int32_t found;
  double logs[2];  // of the sums: of what is kept, at temperature 1
  Choice choice;
};

struct Row {
  const uint16_t* p;
  int V;
  RowSplit split;
};

// eight(g, bits of eight entries) of the row's aligned groups, the next kAhead of them always requested, and one(id, bits) of the
// entries around them.  (No load is behind a branch: the compiler would wait for all of them where paths meet.  Those behind the
// row's end read its last group again.)  begin() is done while the first are on their way.
constexpr int kAhead = 6;
template <class E, class F, class B>
__device__ __forceinline__ void each_group(const Row& r, B&& begin, E&& eight, F&& one) {
  const int n = r.split.nvec, t = thread_of_phase();
  if (n == 0) begin();
  if (n > 0) {
    const uint4* groups = reinterpret_cast<const uint4*>(r.p + r.split.head);
    auto load = [&](int g) { return groups[g < n ? g : n - 1]; };
    uint4 v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = load(t + u * kThreads);
    begin();
    int g = 0;
#pragma unroll 1
    for (; g + kAhead * kThreads <= n; g += kAhead * kThreads) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const uint4 now = v[u];
        v[u] = load(g + t + (u + kAhead) * kThreads);
        eight(g + t + u * kThreads, now);
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (g + t + u * kThreads < n) eight(g + t + u * kThreads, v[u]);
  }
#pragma unroll 1
  for (int j = t; j < r.V - 8 * n; j += kThreads) {
    const int id = r.split.edge_elem(j);
    one(id, (uint32_t)r.p[id]);
  }
}

// A counter also says where its value occurs if it does once: the lower bits count, the others add up the numbers of the places (2^shift
// groups) of those that are counted.  Rows of 2^19 entries and more have no bits left for that.
struct Places {
  uint32_t mask;  // of the count
  int shift;
  bool there;
};
constexpr int kCountBits = 19;
constexpr uint32_t kAround = (1u << (32 - kCountBits)) - 1;  // the place of the entries around the groups
// `longest`: entries of the row, of one in parts those of its first part, so that all have the same bits
__device__ __forceinline__ Places places_of(const Row& r, int longest) {
  const int n = r.split.nvec;
  Places p;
  p.there = longest < 1 << kCountBits;
  p.mask = p.there ? (1u << kCountBits) - 1 : 0xffffffffu;
  const int over = 32 - (32 - kCountBits) - __builtin_clz((unsigned)n | 1);  // bits of n beyond those of a place
  p.shift = over > 0 ? over : 0;
  if ((uint32_t)(n >> p.shift) >= kAround) ++p.shift;
  return p;
}

// bits of the row's entries, for rows by passes: in little code (a function whose branches reach further than 128 KB takes the registers
// of its return address for them, and whether the compiler has saved those is chance)
template <class F>
__device__ __forceinline__ void each_entry(const Row& r, F&& f) {
  const uint4* groups = reinterpret_cast<const uint4*>(r.p + r.split.head);
#pragma unroll 1
  for (int g = threadIdx.x; g < r.split.nvec; g += kThreads) {
    const uint4 v = groups[g];
#pragma unroll 1
    for (int t = 0; t < 8; ++t) {
      const uint32_t two = t < 4 ? (t < 2 ? v.x : v.y) : (t < 6 ? v.z : v.w);
      f(t & 1 ? two >> 16 : two & 0xffff);
    }
  }
#pragma unroll 1
  for (int j = threadIdx.x; j < r.V - 8 * r.split.nvec; j += kThreads) f((uint32_t)r.p[r.split.edge_elem(j)]);
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

// exp(y), y <= 0, to about a unit in the last place: y = (64 i + j) ln 2 / 64 + r with |r| <= ln 2 / 128, 2^(j / 64) from a table in LDS
// (begin()), exp(r) by its series (r^6 / 720 is 2^-54.6 at most).  Half the operations of the library's, and few constants.
__device__ __forceinline__ void begin_exponentials(Shared& s) {
  if (threadIdx.x < kTable) s.table[threadIdx.x] = exp2((double)threadIdx.x / kTable);
}
__device__ __forceinline__ double exponential(double y, const Shared& s) {
  y = __builtin_fmin(__builtin_fmax(y, -800.0), 0.0);  // (0 below; searches ask above the largest entry too)
  const double k = __builtin_rint(y * 0x1.71547652b82fep+6);
  double r = __builtin_fma(k, -0x1.62e42fefa39efp-7, y);
  r = __builtin_fma(k, -0x1.abc9e3b39803fp-62, r);
  double p = __builtin_fma(r, 1.0 / 120.0, 1.0 / 24.0);
  p = __builtin_fma(r, p, 1.0 / 6.0);
  p = __builtin_fma(r, p, 0.5);
  p = __builtin_fma(r * r, p, r);
  const int i = (int)k;
  const double t = s.table[i & (kTable - 1)];
  return __builtin_amdgcn_ldexp(__builtin_fma(t, p, t), i >> 6);
}
// `per`: 1 / tau
__device__ __forceinline__ double weight_of(uint32_t key, double top, double per, const Shared& s) {
  return exponential(((double)value_of(key) - top) * per, s);
}

// lane i's
__device__ __forceinline__ double lane_value(double v, int i) {
  const uint2 u = __builtin_bit_cast(uint2, v);
  return __builtin_bit_cast(double, make_uint2(__builtin_amdgcn_readlane(u.x, i), __builtin_amdgcn_readlane(u.y, i)));
}

// sums up to each lane, over rows of N lanes (8: the first eight alone are right); no LDS is waited for
template <int CONTROL, int ROWS>
__device__ __forceinline__ uint32_t shifted(uint32_t v) {  // (lanes that nothing is shifted into: 0)
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CONTROL, ROWS, 0xf, false);
}
template <int CONTROL, int ROWS>
__device__ __forceinline__ double shifted(double v) {
  const uint2 u = __builtin_bit_cast(uint2, v);
  return __builtin_bit_cast(double, make_uint2(shifted<CONTROL, ROWS>(u.x), shifted<CONTROL, ROWS>(u.y)));
}
template <int N, class T>
__device__ __forceinline__ T sums_to(T v) {
  v += shifted<0x111, 0xf>(v);  // row_shr:1, 2, 4, 8
  v += shifted<0x112, 0xf>(v);
  v += shifted<0x114, 0xf>(v);
  if constexpr (N > 8) v += shifted<0x118, 0xf>(v);
  if constexpr (N > 16) {
    v += shifted<0x142, 0xa>(v);  // row_bcast:15, into the odd rows, then :31
    v += shifted<0x143, 0xc>(v);
  }
  return v;
}

enum Find { kCount, kMassReaches, kMassExceeds };

// A row by passes over it: counts and masses of its entries from a value on, and the value at which they reach something.
struct Passes {
  const Row& row;
  Shared& s;
  uint32_t top_key, all;
  double top, per, sum;
  __device__ __attribute__((noinline)) void from(uint32_t key, double at, uint32_t* count, double* mass) const {
    uint32_t n = 0;
    double m = 0.0;
    each_entry(row, [&](uint32_t b) {
      const uint32_t k = key_of(b);
      if (k < key || k < kLowest) return;
      ++n;
      m += weight_of(k, top, at, s);
    });
    *count = block_count(n, s.sums);
    *mass = block_sum64(m, s.masses[0]);
  }
  __device__ __forceinline__ void begin(double at) {
    per = at;
    from(kLowest, per, &all, &sum);
  }
  __device__ __forceinline__ double sum_at(double at) const {
    uint32_t n;
    double m;
    from(kLowest, at, &n, &m);
    return m;
  }
  // how many weigh `least` and more
  __device__ __forceinline__ uint32_t at_least(double least) const {
    uint32_t n = 0;
    each_entry(row, [&](uint32_t b) {
      const uint32_t k = key_of(b);
      n += k >= kLowest && weight_of(k, top, per, s) >= least;
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
      from(mid, per, &n, &m);
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
    return Place{lo, n_hi, n_lo - n_hi, m_hi, weight_of(lo, top, per, s)};
  }
};

// A row whose entries are counted.  Stretches of eight values, in their order, were weighed by a thread each (weigh()), and what there
// is before each stretch is in LDS; one wave searches there, whose lanes have what there is up to the end of every sixteenth.  (One
// wave's instructions are the time: places and keys are chosen, not branched to.)
struct Counted {
  Shared& s;
  uint32_t mask;  // Places::mask
  uint32_t top_key, all;
  double top, per, sum;
  uint32_t ends;
  double mass_ends;

  static __device__ __forceinline__ uint32_t key(const Shared& s, int t, int e) {
    const int i = (t - kOwners) * kEach + e;
    const uint32_t near = s.near_keys[i < 0 ? 0 : i < kNear ? i : kNear - 1];
    const uint32_t positive = 0x8000u + kFirst + kValues - 1 - (uint32_t)(t * kEach + e), negative = 0x7fffu - kFirst - (uint32_t)(i - kNear);
    return t < kOwners ? positive : i < kNear ? near : negative;
  }
  static __device__ __forceinline__ uint32_t count_of(const Shared& s, uint32_t mask, int t, int e) {
    constexpr int kNearCounts = (int)(offsetof(Shared, near_counts) / 4);
    static_assert(offsetof(Shared, counts) == 0, "");
    const int i = (t - kOwners) * kEach + e;
    const int positive = 2 * ((int)kValues - 1 - (t * kEach + e)), negative = 2 * (i - kNear) + 1;
    const int at = t < kOwners ? positive : i < kNear ? kNearCounts + i : negative;
    return reinterpret_cast<const uint32_t*>(&s)[at] & mask;  // (the mask has all bits of any count that may be there)
  }
  static constexpr int kPer = kThreads / kWave;
  // the first of the stretches for which it holds (it does for those behind it too), from lanes' answers for the ends of sixteen each,
  // then for those sixteen
  static __device__ __forceinline__ int first_lane(bool is, int none) {
    const uint64_t lanes = __ballot(is);
    return lanes ? __builtin_ctzll(lanes) : none;
  }
  // how many weigh `least` and more (weights fall along the order whether a value occurs or not)
  __device__ __forceinline__ uint32_t at_least(double least) const {
    const int lane = thread_of_phase() & 63;
    const auto below = [&](uint32_t k) { return weight_of(k, top, per, s) < least; };
    const int group = first_lane(below(key(s, lane * kPer + kPer - 1, kEach - 1)) || lane == kWave - 1, kWave - 1);
    const int in = lane < kPer ? lane : kPer - 1;
    const int t = group * kPer + first_lane(below(key(s, group * kPer + in, kEach - 1)) || in == kPer - 1, kPer - 1);
    const int e = lane & (kEach - 1);
    const uint32_t here = count_of(s, mask, t, e);
    const uint32_t mine = sums_to<kEach>(below(key(s, t, e)) ? 0 : here);
    return s.count_ends[t] + __builtin_amdgcn_readlane(mine, kEach - 1);
  }
  // (there is enough: what is asked for is at most what there is; the last value there is takes what rounding leaves over)
  __device__ __forceinline__ Place find(Find what, uint32_t target, double mass) const {
    const auto reached = [&](double w) { return what == kMassReaches ? w >= mass : w > mass; };
    const auto is = [&](uint32_t c, double w) { return what == kCount ? c >= target : c == all || (c > 0 && reached(w)); };
    const int lane = thread_of_phase() & 63, in = lane < kPer ? lane : kPer - 1, e = lane & (kEach - 1);
    const int group = first_lane(is(ends, mass_ends), kWave - 1), at = group * kPer + in + 1;
    const int t = group * kPer + first_lane(is(s.count_ends[at], what == kCount ? 0.0 : s.mass_ends[at]), kPer - 1);
    const uint32_t n = count_of(s, mask, t, e), k = key(s, t, e);
    const uint32_t c0 = s.count_ends[t];
    const double w0 = s.mass_ends[t], one = weight_of(k, top, per, s);
    // up to the end of each of the eight (the first eight lanes')
    const uint32_t c = c0 + sums_to<kEach>(n);
    const double w = w0 + sums_to<kEach>(n * one);
    // (what rounding leaves over is the last one's that has any weight)
    const uint32_t those = (uint32_t)__ballot(n && (what == kCount ? c >= target : reached(w))) & 0xff;
    const uint32_t some = (uint32_t)__ballot(n && one > 0.0) & 0xff, any = (uint32_t)__ballot(n != 0) & 0xff;
    const int last = 31 - __builtin_clz((some ? some : any) | 1), i = those ? __builtin_ctz(those) : last;
    const uint32_t here = __builtin_amdgcn_readlane(n, i);
    const double before = lane_value(w, i ? i - 1 : 0);
    return Place{(uint32_t)__builtin_amdgcn_readlane(k, i), (uint32_t)__builtin_amdgcn_readlane(c, i) - here, here, i ? before : w0, lane_value(one, i)};
  }
};

// The list of what is close to zero in its order, equal ones in the first of their places, zero (counted in the first place until
// now) in there once.  All threads.
__device__ __attribute__((noinline)) void order_near(Shared& s) {
  const int t = threadIdx.x, n = (int)s.near;
  const uint32_t zeros = s.near_counts[0];
  __syncthreads();
  if (t < kNear) {
    const uint32_t mine = t < n ? s.near_list[t] : t == n ? 0x8000 : kBelowNear;
    int above = t > n ? t : 0, same_before = 0, same = 1;
    if (t <= n) {
      for (int i = 0; i < n; ++i) {
        const uint32_t k = s.near_list[i];
        above += k > mine;
        same += k == mine && i != t;
        same_before += k == mine && i < t;
      }
      above += t != n && mine < 0x8000;  // (zero)
    }
    s.near_keys[above + same_before] = mine;
    s.near_counts[above + same_before] = t > n || same_before ? 0 : t == n ? zeros : same;
  }
  __syncthreads();
}

// (of two elements of an array the compiler would choose the place, and then the element by comparing that to each)
__device__ __forceinline__ uint32_t either(bool first, uint32_t a, uint32_t b) { return first ? a : b; }

// The counts of the thread's eight values, in their order.
__device__ __forceinline__ void read_counts(const Shared& s, uint32_t mask, int t, uint32_t (&n)[kEach]) {
  if (t >= kOwners && t < kOwners + kNear / kEach) {
#pragma unroll
    for (int e = 0; e < kEach; ++e) n[e] = s.near_counts[(t - kOwners) * kEach + e];
    return;
  }
  // (sixteen counters, of both signs: reads of every other word would meet in few banks.  Those of four lanes at the same sixteenth of
  // 256 bytes would too, so each four of the lanes begin at another quarter of their sixteen.)
  const bool negative = t >= kOwners;
  const int at = negative ? 2 * (t - kOwners - kNear / kEach) * kEach : 2 * (kValues - kEach * (t + 1)), turn = t >> 2 & 3;
  uint32_t w[kEach];  // of the sign
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 v = *reinterpret_cast<const uint4*>(&s.counts[at + 4 * ((i + turn) & 3)]);
    w[2 * i] = negative ? v.y : v.x;
    w[2 * i + 1] = negative ? v.w : v.z;
  }
#pragma unroll
  for (int by = 1; by < 4; by <<= 1) {  // quarter i is (i + turn) & 3: turned back
    uint32_t o[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) o[i] = either(turn & by, w[(i - 2 * by) & (kEach - 1)], w[i]);
#pragma unroll
    for (int i = 0; i < kEach; ++i) w[i] = o[i];
  }
#pragma unroll
  for (int e = 0; e < kEach; ++e) n[e] = either(negative, w[e], w[kEach - 1 - e]) & mask;
}

// the largest value that is counted (0: none), all threads
__device__ __forceinline__ uint32_t largest_counted(Shared& s, const uint32_t (&n)[kEach]) {
  const int t = thread_of_phase();
  uint32_t there = 0;
#pragma unroll
  for (int e = 0; e < kEach; ++e) there |= n[e] ? 1u << e : 0;
  const uint64_t any = __ballot(there != 0);
  const int first = any ? __builtin_ctzll(any) : 0;
  if ((t & 63) == first) s.sums[t >> 6] = there ? Counted::key(s, t, __builtin_ctz(there)) : 0;
  __syncthreads();
  const uint32_t mine = s.sums[t & (kWaves - 1)];
  const uint64_t waves = __ballot(mine != 0);
  return waves ? __builtin_amdgcn_readlane(mine, __builtin_ctzll(waves)) : 0;
}

// Weighs the stretches, all threads: what there is up to the end of each (the sum over its wave so far, added to the waves' before), and
// the sum at temperature 1.  Eight values of a stretch lie evenly apart, so that their weights are
// powers of one ratio: two exponentials for eight, and 2^-50 of a weight at most in roundings.
__device__ __forceinline__ void weigh(Shared& s, const uint32_t (&n)[kEach], double top, double per, bool nll, double* sum1) {
  const int t = thread_of_phase(), lane = t & 63, wave = t >> 6;
  uint32_t c = 0;
  double w = 0.0, w1 = 0.0;
  const bool both = nll && per != 1.0, near = t >= kOwners && t < kOwners + kNear / kEach;
  uint32_t there = 0;
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    c += n[e];
    there |= n[e] ? 1u << e : 0;
  }
  if (c && !near) {
    // (from the first that occurs: those before it may lie above the top)
    const int f = __builtin_ctz(there);
    const bool negative = t >= kOwners;
    const uint32_t size = kFirst + (negative ? (t - kOwners) * kEach - kNear + f : kValues - 1 - t * kEach - f);
    const double first = bf16_one((uint16_t)(size | (negative ? 0x8000 : 0)));
    const double step = __builtin_bit_cast(float, ((size >> 7) - 7) << 23);  // (of the eight: 2^-7 of their power of two)
    double one = exponential((first - top) * per, s);
    const double ratio = exponential(-step * per, s);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      w = __builtin_fma((double)n[e], one, w);
      if (e >= f) one *= ratio;
    }
    if (both) {
      one = exponential(first - top, s);
      const double ratio1 = exponential(-step, s);
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        w1 = __builtin_fma((double)n[e], one, w1);
        if (e >= f) one *= ratio1;
      }
    }
  }
  if (c && near) {
#pragma unroll 1
    for (int e = 0; e < kEach; ++e) {
      const double k = s.near_counts[(t - kOwners) * kEach + e];
      const uint32_t key = Counted::key(s, t, e);
      w += k * weight_of(key, top, per, s);
      if (both) w1 += k * weight_of(key, top, 1.0, s);
    }
  }
  c = sums_to<kWave>(c);
  w = sums_to<kWave>(w);
  if (both) w1 = sums_to<kWave>(w1);
  __syncthreads();  // (largest_counted()'s sums have been read)
  if (lane == 63) {
    s.sums[wave] = c;
    s.masses[0][wave] = w;
    s.masses[1][wave] = w1;
  }
  __syncthreads();
  // (lane i has the sums up to wave i)
  const int i = lane & (kWaves - 1);
  const uint32_t cs = sums_to<kWaves>(s.sums[i]);
  const double ws = sums_to<kWaves>(s.masses[0][i]), ws1 = both ? sums_to<kWaves>(s.masses[1][i]) : ws;
  const int before = __builtin_amdgcn_readfirstlane(wave) - 1;
  if (t == 0) {
    s.count_ends[0] = 0;
    s.mass_ends[0] = 0.0;
  }
  s.count_ends[t + 1] = before < 0 ? c : __builtin_amdgcn_readlane(cs, before < 0 ? 0 : before) + c;
  s.mass_ends[t + 1] = before < 0 ? w : lane_value(ws, before < 0 ? 0 : before) + w;
  *sum1 = lane_value(ws1, kWaves - 1);
  __syncthreads();
}

// The settings of a row.
struct Settings {
  double tau, per, top_p, min_p, u;  // per: 1 / tau
  uint32_t top_k;
};

template <class Entries>
__device__ __forceinline__ Choice choose(const Entries& x, const Settings& q) {
  uint32_t n = q.top_k > 0 && q.top_k < x.all ? q.top_k : x.all;
  Place end{};  // where the first n end
  double sum = x.sum;
  auto cut = [&]() {
    if (n == x.all) {
      sum = x.sum;
      return;
    }
    end = x.find(kCount, n, 0.0);
    sum = end.mass + (double)(n - end.before) * end.weight;
  };
  cut();
  const uint32_t by_k = n;
  if (q.top_p < 1.0 && n > 1) {
    const double enough = q.top_p * sum;
    const Place p = x.find(kMassReaches, 0, enough);
    const double more = ceil((enough - p.mass) / p.weight);
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
  Place p = n == 1 ? Place{x.top_key, 0, 1, 0.0, 1.0} : x.find(kMassExceeds, 0, at);
  uint32_t here = p.here;
  if (n != x.all && n > 1) {
    if (p.before >= end.before) p = end;  // (no further than the last one that is kept)
    if (p.key == end.key) here = n - end.before;
  }
  const double steps = floor((at - p.mass) / p.weight);
  const uint32_t which = !(steps > 0.0) ? 0 : steps < (double)here ? (uint32_t)steps : here - 1;
  return Choice{p.key, n, which, ((double)value_of(p.key) - x.top) * x.per, sum};
}

// id of the entry `which` (in order of ids) of those of a value: their ids go into a list where the counters were
__device__ __forceinline__ int find_entry(const Row& row, uint32_t key, uint32_t which, Shared& s) {
  constexpr uint32_t kList = sizeof(s.counts) / sizeof(s.counts[0]);
  __syncthreads();
  if (threadIdx.x == 0) {
    s.found = 0x7fffffff;
    s.listed = 0;
  }
  __syncthreads();
  const uint32_t bits = key == 0x8000 ? 0 : key & 0x8000 ? key & 0x7fff : ~key & 0xffff, mask = bits ? 0xffff : 0x7fff;  // (-0 is 0)
  auto hit = [&](int id) {
    if (which == 0) {
      atomicMin(&s.found, id);
    } else {
      const uint32_t n = atomicAdd(&s.listed, 1u);
      if (n < kList) s.counts[n] = (uint32_t)id;
    }
  };
  const uint32_t bits2 = bits * 0x10001u, mask2 = mask * 0x10001u;
  each_group(
      row, [] {},
      [&](int g, const uint4& v) {
        const int id = row.split.head + 8 * g;
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        u16x2 d[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) d[t] = __builtin_bit_cast(u16x2, (w[t] & mask2) ^ bits2);
        const u16x2 least = __builtin_elementwise_min(__builtin_elementwise_min(d[0], d[1]), __builtin_elementwise_min(d[2], d[3]));
        if (least[0] != 0 && least[1] != 0) return;
        uint32_t hits = 0;
#pragma unroll
        for (int t = 0; t < 8; ++t) hits |= (d[t >> 1][t & 1] == 0 ? 1u : 0u) << t;
#pragma unroll 1
        for (; hits; hits &= hits - 1) hit(id + __builtin_ctz(hits));
      },
      [&](int id, uint32_t b) {
        if ((b & mask) == bits) hit(id);
      });
  __syncthreads();
  if (which == 0) return s.found;
  const uint32_t listed = s.listed;
  if (listed <= kThreads) {
    if (threadIdx.x < 4) s.counts[listed + threadIdx.x] = 0xffffffffu;  // (the list in fours)
    __syncthreads();
    if (threadIdx.x < listed) {
      const uint32_t mine = s.counts[threadIdx.x];
      uint32_t below = 0;
#pragma unroll 4
      for (uint32_t i = 0; i < listed; i += 4) {
        const uint4 v = *reinterpret_cast<const uint4*>(&s.counts[i]);
        below += (v.x < mine) + (v.y < mine) + (v.z < mine) + (v.w < mine);
      }
      if (below == which) s.found = (int32_t)mine;
    }
    __syncthreads();
    return s.found;
  }
  // very many of them: every wave counts in a stretch of its own, and the one that has it looks again
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int groups = (row.V + 7) / 8, each = (groups + kWaves - 1) / kWaves;
  const int begin = wave * each < groups ? wave * each : groups, end = groups - begin < each ? groups : begin + each;
  auto hits_of = [&](int g) {  // which of eight entries
    const uint4 v = load8_of(row.p, 8 * g, row.V);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t hits = 0;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const uint32_t x = t & 1 ? w[t >> 1] >> 16 : w[t >> 1] & 0xffff;
      hits |= ((x & mask) == bits && 8 * g + t < row.V ? 1u : 0u) << t;
    }
    return hits;
  };
  uint32_t n = 0;
#pragma unroll 1
  for (int g = begin + lane; g < end; g += kWave) n += __popc(hits_of(g));
  n = (uint32_t)wave_sum_int((int)n);
  if (lane == 0) s.sums[wave] = n;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < wave; ++w) before += s.sums[w];
  if (which >= before && which - before < n) {
    uint32_t left = which - before;
#pragma unroll 1
    for (int g = begin; g < end; g += kWave) {
      uint32_t hits = g + lane < end ? hits_of(g + lane) : 0;
      uint32_t upto = __popc(hits);
      const uint32_t mine = upto;
#pragma unroll 1
      for (int off = 1; off < kWave; off <<= 1) {
        const uint32_t o = __shfl_up(upto, off, kWave);
        if (lane >= off) upto += o;
      }
      const uint32_t here = __shfl(upto, kWave - 1, kWave);
      if (left < here) {
        if (left >= upto - mine && left < upto) {
          for (uint32_t skip = left - (upto - mine); skip; --skip) hits &= hits - 1;
          s.found = 8 * (g + lane) + __builtin_ctz(hits);
        }
        break;
      }
      left -= here;
    }
  }
  __syncthreads();
  return s.found;
}

// id of the entry of a value that occurs once, at a place
__device__ __forceinline__ int find_place(const Row& row, uint32_t key, uint32_t place, int shift, Shared& s) {
  const int t = thread_of_phase();
  if (place == kAround) {
    if (t < row.V - 8 * row.split.nvec) {
      const int id = row.split.edge_elem(t);
      if (key_of(row.p[id]) == key) s.found = id;
    }
  } else {
    const int g = (int)(place << shift) + t;
    if (t < 1 << shift && g < row.split.nvec) {
      const uint4 v = reinterpret_cast<const uint4*>(row.p + row.split.head)[g];
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (key_of(e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffff) == key) s.found = row.split.head + 8 * g + e;
    }
  }
  __syncthreads();
  return s.found;
}

// A row's outputs.
__device__ __forceinline__ void put(const SampleArgs& a, int64_t r, int token, double logprob, double nll, uint32_t kept, int status) {
  if (threadIdx.x != 0) return;
  a.token[r] = token;
  if (a.logprob) a.logprob[r] = (float)logprob;
  if (a.nll) a.nll[r] = (float)nll;
  if (a.kept) a.kept[r] = (int32_t)kept;
  if (status && a.status) atomicOr(a.status, status);
}

// A row by passes over it.  (Not inlined: the registers of the rows that are counted are the ones that matter.)
__device__ __attribute__((noinline)) void draw_by_passes(const SampleArgs a, int64_t r, const Row row, const Settings q, bool greedy, Shared& s) {
  uint32_t most = 0, bad = 0;
  each_entry(row, [&](uint32_t b) {
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
  if (bad || most < kLowest) {
    put(a, r, -1, __builtin_nan(""), __builtin_nan(""), 0, NPD_DEV_BAD_LOGITS);
    return;
  }
  Passes passes{row, s, most, 0, value_of(most), 0.0, 0.0};
  passes.begin(q.per);
  const Choice c = greedy ? Choice{most, 1, 0, 0.0, 1.0} : choose(passes, q);
  const double sum1 = !a.nll ? 1.0 : q.tau == 1.0 ? passes.sum : passes.sum_at(1.0);
  const int token = find_entry(row, c.key, c.which, s);
  put(a, r, token, c.logit - log(c.sum), log(sum1) + (passes.top - (double)value_of(c.key)), c.kept, 0);
}

// (a workgroup has one row: in a loop over rows what only threadIdx decides would be kept in registers from one to the next)
constexpr int64_t kGrid = 65536;  // workgroups along x

__device__ __forceinline__ void begin_counts(Shared& s) {
  for (int i = threadIdx.x; i < (int)(sizeof(s.counts) / 16); i += kThreads) reinterpret_cast<uint4*>(s.counts)[i] = make_uint4(0, 0, 0, 0);
  if (threadIdx.x < kNear) {
    s.near_keys[threadIdx.x] = threadIdx.x ? kBelowNear : 0x8000;
    s.near_counts[threadIdx.x] = 0;
  }
  if (threadIdx.x == 0) s.big = s.odd = s.near = 0;
}

// an entry with its sign in the lowest place: the first that has a counter, and -inf less that
constexpr unsigned short kTurnedFirst = 2 * kFirst, kTurnedForbidden = 0xff01 - kTurnedFirst;

// Counts a row's entries; zero in the first of near_counts, what else is closer to zero than the counters' in near_list.
template <class B>
__device__ __forceinline__ void count_entries(const Row& row, int longest, Shared& s, B&& begin) {
  uint32_t big = 0, odd = 0;  // large negative numbers; entries that have no counter otherwise
  auto other = [&](uint32_t b) {
    const uint32_t size = b & 0x7fff;
    if (size == 0)
      atomicAdd(&s.near_counts[0], 1u);
    else if (size < kFirst) {
      const uint32_t n = atomicAdd(&s.near, 1u);
      if (n < kNear - 1) s.near_list[n] = key_of(b);
    } else if (size >= kFirst + kValues && b != 0xff80) {
      if (b > 0x8000 && b < 0xff80)
        ++big;
      else
        odd = 1;
    }
  };
  // A counter's number is the entry with its sign in the lowest place, less the first one's.  What is no counter's goes to
  // the lane's own among `kOthers` (a branch around every addition takes twice the time) and is looked at afterwards.
  const uint32_t own = kOthers + (threadIdx.x & 63);
  const Places places = places_of(row, longest);
  each_group(
      row,
      [&] {
        begin();
        begin_counts(s);
        __syncthreads();
      },
      [&](int g, const uint4& v) {
        const uint32_t unit = 1u + (places.there ? (uint32_t)(g >> places.shift) << kCountBits : 0u);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        u16x2 at[4];
        uint32_t most = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const uint32_t turned = (w[t] << 1 & 0xfffefffe) | (w[t] >> 15 & 0x00010001);
          at[t] = __builtin_bit_cast(u16x2, turned) - u16x2{kTurnedFirst, kTurnedFirst};
          const uint32_t lo = at[t][0], hi = at[t][1];
          most = most > lo ? most : lo;
          most = most > hi ? most : hi;
          atomicAdd(&s.counts[lo < own ? lo : own], unit);
          atomicAdd(&s.counts[hi < own ? hi : own], unit);
        }
        if (most < kOthers) return;
        // (-inf is nothing: rows in which some entries are forbidden come here with every group)
        u16x2 some = {0, 0};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const u16x2 forbidden = {kTurnedForbidden, kTurnedForbidden}, one = {1, 1};
          some = __builtin_elementwise_max(some, at[t] * __builtin_elementwise_min(at[t] ^ forbidden, one));
        }
        if (some[0] < kOthers && some[1] < kOthers) return;
#pragma unroll 1
        for (int t = 0; t < 8; ++t) {
          const uint32_t two = t < 4 ? (t < 2 ? w[0] : w[1]) : (t < 6 ? w[2] : w[3]);
          other(t & 1 ? two >> 16 : two & 0xffff);
        }
      },
      [&](int, uint32_t b) {
        const uint32_t i = (b & 0x7fff) - kFirst;
        if (i < kValues)
          atomicAdd(&s.counts[2 * i + (b >> 15)], 1u + (places.there ? kAround << kCountBits : 0u));
        else
          other(b);
      });
  if (big) atomicAdd(&s.big, big);
  if (odd) s.odd = 1;
  __syncthreads();
}

// Rows of calls that have few of them are counted in parts, by a workgroup each.  What a part leaves in the workspace:
struct Part {
  uint32_t counts[kOthers];
  uint32_t zeros, near, big, odd;  // (sixteen bytes, aligned)
  uint32_t near_list[kNear];
};
static_assert(sizeof(Part) == kSamplePartBytes, "");

// entries [first, end) of a row are its part i
struct Span {
  int first, end;
};
__device__ __forceinline__ Span part_of(int V, int parts, int i) {
  const int each = ((V + parts - 1) / parts + 7) / 8 * 8;
  const int first = i * each < V ? i * each : V;
  return Span{first, V - first < each ? V : first + each};
}
__device__ __forceinline__ Row row_part(const uint16_t* p, const Span& at) {
  const int n = at.end - at.first;
  return Row{p + at.first, n, row_split(p + at.first, n, true)};
}

__global__ __launch_bounds__(kThreads, 8) void sample_count_kernel(SampleArgs a) {
  __shared__ Shared s;
  const int64_t r = blockIdx.y;
  if (a.mask && !a.mask[r]) return;
  count_entries(row_part(a.x + r * a.stride, part_of(a.V, a.parts, blockIdx.x)), part_of(a.V, a.parts, 0).end, s, [] {});
  Part& part = reinterpret_cast<Part*>(a.workspace)[r * a.parts + blockIdx.x];
  for (int i = threadIdx.x; i < (int)kOthers / 4; i += kThreads) reinterpret_cast<uint4*>(part.counts)[i] = reinterpret_cast<uint4*>(s.counts)[i];
  if (threadIdx.x < kNear) part.near_list[threadIdx.x] = s.near_list[threadIdx.x];
  if (threadIdx.x == 0) {
    part.zeros = s.near_counts[0];
    part.near = s.near;
    part.big = s.big;
    part.odd = s.odd;
  }
}

// The counts of a row out of those of its parts, all threads.
__device__ __forceinline__ void join_parts(const Part* parts, int n, uint32_t mask, Shared& s) {
  // (all requested together, of parts that are not there the last one's again: a round trip each would take longer than the counts)
  const int t = threadIdx.x;
  constexpr int kQuads = kOthers / 4, kMine = (kQuads + kThreads - 1) / kThreads;
  uint4 rest[kSampleParts], v[kMine][kSampleParts];
#pragma unroll
  for (int p = 0; p < kSampleParts; ++p) {
    const Part& part = parts[p < n ? p : n - 1];
    rest[p] = *reinterpret_cast<const uint4*>(&part.zeros);
#pragma unroll
    for (int m = 0; m < kMine; ++m) v[m][p] = reinterpret_cast<const uint4*>(part.counts)[t + m * kThreads < kQuads ? t + m * kThreads : t];
  }
#pragma unroll
  for (int m = 0; m < kMine; ++m) {
    uint4 sum = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int p = 0; p < kSampleParts; ++p) {
      const uint32_t here = p < n ? mask : 0;
      sum = make_uint4(sum.x + (v[m][p].x & here), sum.y + (v[m][p].y & here), sum.z + (v[m][p].z & here), sum.w + (v[m][p].w & here));
    }
    if (t + m * kThreads < kQuads) reinterpret_cast<uint4*>(s.counts)[t + m * kThreads] = sum;
  }
  uint32_t zeros = 0, near = 0, big = 0, odd = 0;
#pragma unroll
  for (int p = 0; p < kSampleParts; ++p) {
    if (p >= n) break;
    const uint32_t here = rest[p].y;
    zeros += rest[p].x;
    if (near + here < kNear && threadIdx.x < here) s.near_list[near + threadIdx.x] = parts[p].near_list[threadIdx.x];
    near = near + here < kNear ? near + here : kNear;  // (no more than fit are looked at)
    big += rest[p].z;
    odd |= rest[p].w;
  }
  if (threadIdx.x < kNear) {
    s.near_keys[threadIdx.x] = threadIdx.x ? kBelowNear : 0x8000;
    s.near_counts[threadIdx.x] = threadIdx.x ? 0 : zeros;
  }
  if (threadIdx.x == 0) {
    s.near = near;
    s.big = big;
    s.odd = odd;
  }
  __syncthreads();
}

// SPLIT: the row has been counted, in parts
template <bool SPLIT>
__global__ __launch_bounds__(kThreads, SPLIT ? 4 : 8) void sample_kernel(SampleArgs a) {
  __shared__ Shared s;
  const int64_t r = (int64_t)blockIdx.y * kGrid + blockIdx.x;
  if (r >= a.T) return;
  const double nan = __builtin_nan("");
  if (a.mask && !a.mask[r]) {
    put(a, r, -1, 0.0, 0.0, 0, 0);
    return;
  }
  const float tau = a.taus ? a.taus[r] : a.tau, top_p = a.top_ps ? a.top_ps[r] : a.top_p, min_p = a.min_ps ? a.min_ps[r] : a.min_p;
  const int top_k = a.top_ks ? a.top_ks[r] : a.top_k;
  const float u = a.u[r];
  const Row row = {a.x + r * a.stride, a.V, row_split(a.x + r * a.stride, a.V, true)};
  const Part* parts = SPLIT ? reinterpret_cast<const Part*>(a.workspace) + r * a.parts : nullptr;

  const int longest = SPLIT ? part_of(a.V, a.parts, 0).end : a.V;
  if constexpr (SPLIT) {
    begin_exponentials(s);
    join_parts(parts, a.parts, places_of(row, longest).mask, s);
  } else {
    count_entries(row, a.V, s, [&] { begin_exponentials(s); });
  }
  // (they were requested before the row)
  if (!(tau >= 0.0f && tau <= 3.4028234663852886e38f) || !(top_p >= 0.0f && top_p <= 1.0f) || !(min_p >= 0.0f && min_p <= 1.0f) || top_k < 0 ||
      !(u >= 0.0f && u < 1.0f)) {
    put(a, r, -1, nan, nan, 0, NPD_DEV_BAD_SAMPLING);
    return;
  }
  const bool greedy = tau == 0.0f;
  const double t = greedy ? 1.0 : (double)tau;
  const Settings q = {t, 1.0 / t, top_p, min_p, u, (uint32_t)top_k};
  const uint32_t big = s.big;
  const bool odd = s.odd || s.near >= kNear;
  if (s.near && !odd) order_near(s);
  const uint32_t mask = SPLIT ? 0xffffffffu : places_of(row, longest).mask;  // (joined, they are counts alone)
  uint32_t n[kEach];
  read_counts(s, mask, thread_of_phase(), n);
  const uint32_t top_key = largest_counted(s, n);
  const double counted_top = top_key ? value_of(top_key) : 0.0;
  // Numbers below -256 have no weight that 64 bits would show beside the largest's (2^-90 times at most 2^26 of them) where that is
  // 64 temperatures above -256, and are none that a min-p would keep.
  const double room = counted_top + 256.0;
  const bool apart = !big || (room >= 64.0 && room >= 64.0 * q.tau && (q.min_p == 0.0 || room > q.tau * (1.0 - log(q.min_p))));
  if (odd || !top_key || !apart) {
    draw_by_passes(a, r, row, q, greedy, s);
    return;
  }
  double sum1 = 1.0;  // of the weights at temperature 1
  if (!greedy || a.nll) weigh(s, n, counted_top, q.per, a.nll != nullptr, &sum1);
  if (greedy) {
    if (threadIdx.x == 0) s.choice = Choice{top_key, 1, 0, 0.0, 1.0};
  } else if (threadIdx.x < kWave) {
    const int end = (threadIdx.x + 1) * Counted::kPer;
    const Counted counted{s, mask, top_key, s.count_ends[kThreads], counted_top, q.per, s.mass_ends[kThreads], s.count_ends[end], s.mass_ends[end]};
    Choice mine = choose(counted, q);
    if (mine.kept == counted.all && big && q.min_p == 0.0 && q.top_p == 1.0) {  // nothing is cut off, or by top-k alone
      const uint32_t all = counted.all + big;
      mine.kept = q.top_k > 0 && q.top_k < all ? q.top_k : all;
    }
    if (threadIdx.x == 0) s.choice = mine;
  }
  if (threadIdx.x == kWave) s.logs[1] = log(sum1);  // (beside the search)
  __syncthreads();
  const Choice c = s.choice;
  if (threadIdx.x == kWave) s.logs[0] = log(c.sum);  // (likewise: for the entry)
  // what there is about the value where it has a counter; of a row in parts the part that has the entry
  Row where = row;
  int first = 0;
  uint32_t which = c.which, here = 0;
  const uint32_t bits = c.key & 0x8000 ? c.key & 0x7fff : ~c.key & 0x7fff, i = 2 * (bits - kFirst) + (c.key & 0x8000 ? 0 : 1);
  if (bits >= kFirst) {
    if constexpr (SPLIT) {
      const uint32_t part_mask = places_of(row, longest).mask;
      uint32_t of[kSampleParts];  // (all requested together)
#pragma unroll
      for (int p = 0; p < kSampleParts; ++p) of[p] = parts[p < a.parts ? p : a.parts - 1].counts[i];
      int at = -1;
#pragma unroll
      for (int p = 0; p < kSampleParts; ++p) {
        if (at >= 0 || p >= a.parts) continue;
        if (which < (of[p] & part_mask)) {
          at = p;
          here = of[p];
        } else {
          which -= of[p] & part_mask;
        }
      }
      const Span span = part_of(a.V, a.parts, at < 0 ? 0 : at);
      first = span.first;
      where = row_part(row.p, span);
    } else {
      here = s.counts[i];
    }
  }
  const Places places = places_of(where, longest);
  const bool once = places.there && (here & places.mask) == 1;
  const int token = first + (once ? find_place(where, c.key, here >> kCountBits, places.shift, s) : find_entry(where, c.key, which, s));
  put(a, r, token, c.logit - s.logs[0], s.logs[1] + (counted_top - (double)value_of(c.key)), c.kept, 0);
}

}  // namespace

// As many parts as give every compute unit one and leave each 32,768 entries, and at least three: a second launch and the joining of the
// counts have to be earned.  Measured (MI355X, us, whole / in parts, untruncated): 1 row of 100,000 16.1 / 16.4 (3 parts), of 128,256 18.2 / 17.7
// (3), of 151,936 17.8 / 16.3 (4), of 262,144 34 / 18.5 (8), of 600,000 51 / 18.6 (8); 32 rows of 100,000 19.0 / 19.4 (3), of 151,936 24.9 / 21.1
// (4), of 262,144 37 / 22.1 (8); 64 rows of 128,256 23.1 / 23.0 (3), of 151,936 26.1 / 23.2 (4).  With top-k 50 and top-p 0.9, where few rows are
// read again, 64 rows of 100,000 18.9 / 21.9, of 151,936 22.5 / 23.6, of 262,144 30.6 / 25.2.  So at the beginning of the range parts gain
// nothing, and 64 rows of up to 151,936 lose by them if they are truncated, which the host does not know of rows with settings of their own.
int sample_parts(int64_t T, int32_t V) {
  const int64_t most = 256 / T < kSampleParts ? 256 / T : kSampleParts, some = V / 32768, parts = most < some ? most : some;
  return parts < 3 ? 1 : (int)parts;
}

hipError_t launch_sample(const SampleArgs& a, hipStream_t stream) {
  const int64_t rows = a.T < kGrid ? a.T : kGrid;
  const dim3 grid((unsigned)rows, (unsigned)((a.T + kGrid - 1) / kGrid));
  if (a.parts < 2) return launch_kernel(sample_kernel<false>, grid, dim3(kThreads), 0, stream, a);
  const hipError_t e = launch_kernel(sample_count_kernel, dim3((unsigned)a.parts, (unsigned)a.T), dim3(kThreads), 0, stream, a);
  return e != hipSuccess ? e : launch_kernel(sample_kernel<true>, grid, dim3(kThreads), 0, stream, a);
}

}  // namespace npd
