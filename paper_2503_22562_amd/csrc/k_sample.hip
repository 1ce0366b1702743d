// Sampling from rows of logits: temperature, top-k, top-p, min-p, given random numbers.
//
// The tokens of a row stand in descending order of their logits, lower indices first
// among equals; every limit keeps a prefix of that order, and the token drawn is the
// first at which the running weight passes u times the kept weight. All of it is the
// same search -- for the k-th token, for the one that reaches p of the weight, for the
// one drawn -- in one cumulative distribution, so no row is sorted: a histogram over
// the logits' distances to their maximum tells the bins that may hold an element searched
// for, and only their elements (kList at most, or the search is narrowed) are sorted.
//
// Weights w = exp((x - max) / t) are formed in fp64 and summed as integers, w 2^shift
// rounded to the nearest, with a shift that keeps the sum of a row below 2^63: sums then
// do not depend on their order, and two programs that use 64 bits agree on every token
// unless u falls within some 2^-29 of a border (V roundings of 2^-46). In fp32 they would
// disagree more often: 128256 even weights, each off by 2^-25, move some border past u in
// one row of 10^4 to 10^5.
//
// Three launches: the rows' extents (the bins and weights need the maximum); the
// histograms, with the likely tokens listed on the way, which tell the token of most rows;
// and a second look at the rows where they do not. Rows are cut into slices so that few
// rows fill the card, and the last workgroup of a row to finish draws its token: no launch
// of its own for that. Few rows are bound by the launches and by chains of barriers (one
// row of 128256: 15.2 us a call; kernels 3.6, 11.5 and 0.9, or 3.8 where the row is read
// again; by the clock of the second one's last workgroup 1.7 until it has settings and extent,
// 1.5 its weights, 2.4 its additions to the row's bins, 1.9 to read those back and scan
// them, 0.8 to search, 1.7 to draw; of 64 rows with every limit, 27 us, 2.1, 6.0, 5.4, 2.9, 1.2
// and 1.7), many by the vector instructions of the weights (256 rows, 131 MB: 27 us extents,
// 49 weights, of which some 35 instructions an element make 29, 30 the second look at the
// rows whose limits lie among unlikely tokens; 105 us a call, and 19 to read the logits
// once).
#include <algorithm>
#include <cfloat>
#include <cstddef>
#include <type_traits>

#include "hb_device.h"
#include "hb_kernels.h"

namespace hb {
namespace {

typedef unsigned long long u64;

constexpr int kBins = kSampleBins, kList = kSampleList, kNearList = kSampleNear;
constexpr float kNear = 8.f;  // tokens whose weight is above e^-8 are listed while the histogram is made
constexpr int kSteps = 64;    // steps of an octave in the table of powers of two
constexpr int kThreads = 256, kWaves = kThreads / 64;

// 2^(j / kSteps), rounded to fp64
__device__ const double kPow2[kSteps] = {
    0x1.0000000000000p+0, 0x1.02c9a3e778061p+0, 0x1.059b0d3158574p+0, 0x1.0874518759bc8p+0,
    0x1.0b5586cf9890fp+0, 0x1.0e3ec32d3d1a2p+0, 0x1.11301d0125b51p+0, 0x1.1429aaea92de0p+0,
    0x1.172b83c7d517bp+0, 0x1.1a35beb6fcb75p+0, 0x1.1d4873168b9aap+0, 0x1.2063b88628cd6p+0,
    0x1.2387a6e756238p+0, 0x1.26b4565e27cddp+0, 0x1.29e9df51fdee1p+0, 0x1.2d285a6e4030bp+0,
    0x1.306fe0a31b715p+0, 0x1.33c08b26416ffp+0, 0x1.371a7373aa9cbp+0, 0x1.3a7db34e59ff7p+0,
    0x1.3dea64c123422p+0, 0x1.4160a21f72e2ap+0, 0x1.44e086061892dp+0, 0x1.486a2b5c13cd0p+0,
    0x1.4bfdad5362a27p+0, 0x1.4f9b2769d2ca7p+0, 0x1.5342b569d4f82p+0, 0x1.56f4736b527dap+0,
    0x1.5ab07dd485429p+0, 0x1.5e76f15ad2148p+0, 0x1.6247eb03a5585p+0, 0x1.6623882552225p+0,
    0x1.6a09e667f3bcdp+0, 0x1.6dfb23c651a2fp+0, 0x1.71f75e8ec5f74p+0, 0x1.75feb564267c9p+0,
    0x1.7a11473eb0187p+0, 0x1.7e2f336cf4e62p+0, 0x1.82589994cce13p+0, 0x1.868d99b4492edp+0,
    0x1.8ace5422aa0dbp+0, 0x1.8f1ae99157736p+0, 0x1.93737b0cdc5e5p+0, 0x1.97d829fde4e50p+0,
    0x1.9c49182a3f090p+0, 0x1.a0c667b5de565p+0, 0x1.a5503b23e255dp+0, 0x1.a9e6b5579fdbfp+0,
    0x1.ae89f995ad3adp+0, 0x1.b33a2b84f15fbp+0, 0x1.b7f76f2fb5e47p+0, 0x1.bcc1e904bc1d2p+0,
    0x1.c199bdd85529cp+0, 0x1.c67f12e57d14bp+0, 0x1.cb720dcef9069p+0, 0x1.d072d4a07897cp+0,
    0x1.d5818dcfba487p+0, 0x1.da9e603db3285p+0, 0x1.dfc97337b9b5fp+0, 0x1.e502ee78b3ff6p+0,
    0x1.ea4afa2a490dap+0, 0x1.efa1bee615a27p+0, 0x1.f50765b6e4540p+0, 0x1.fa7c1819e90d8p+0,
};

// Consecutive elements of a row, from index `first` on.
template <int N>
struct Run {
  float x[N];
  int first;
};
// Elements (fp32 or bf16) [first, first + n) of a row, f(Run) for all of them; any alignment.
template <bool BF16>
struct Logits {
  const uint16_t* h;
  const float* f;
  int first, n;
  __device__ __forceinline__ Logits(const void* p, int64_t row, int first, int n)
      : h(static_cast<const uint16_t*>(p) + row), f(static_cast<const float*>(p) + row), first(first), n(n) {}
  __device__ __forceinline__ float at(int i) const { return BF16 ? bf16_to_f32(h[i]) : f[i]; }
  static constexpr int kPer = BF16 ? 8 : 4;  // elements of a 16-byte load
  static __device__ __forceinline__ Run<kPer> run(u32x4 r, int e) {
    Run<kPer> v;
    v.first = e;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (BF16) {
        v.x[2 * j] = bf16_lo(r[j]);
        v.x[2 * j + 1] = bf16_hi(r[j]);
      } else {
        v.x[j] = __uint_as_float(r[j]);
      }
    }
    return v;
  }
  // LOADS 16-byte loads of a thread in flight
  template <int LOADS, typename F>
  __device__ __forceinline__ void each(F&& fn) const {
    constexpr int SIZE = BF16 ? 2 : 4;
    const int tid = threadIdx.x;
    const uintptr_t p = BF16 ? reinterpret_cast<uintptr_t>(h + first) : reinterpret_cast<uintptr_t>(f + first);
    const int head = min(n, (int)((16 - (p & 15)) & 15) / SIZE);  // elements before the first 16-byte boundary
    const int nv = (n - head) / kPer, tail = head + nv * kPer;
    const u32x4* v = BF16 ? reinterpret_cast<const u32x4*>(h + first + head) : reinterpret_cast<const u32x4*>(f + first + head);
    int i0 = tid;
    for (; i0 - tid + LOADS * kThreads <= nv; i0 += LOADS * kThreads) {
      u32x4 r[LOADS];
#pragma unroll
      for (int k = 0; k < LOADS; ++k) r[k] = v[i0 + k * kThreads];
#pragma unroll
      for (int k = 0; k < LOADS; ++k) fn(run(r[k], first + head + (i0 + k * kThreads) * kPer));
    }
#pragma unroll 1
    for (; i0 < nv; i0 += kThreads) fn(run(v[i0], first + head + i0 * kPer));
    // the ragged ends: fewer than kPer elements each
    const int at = first + (tid < head ? tid : tail + tid - head);
    if (tid < head + n - tail) fn(Run<1>{{this->at(at)}, at});
  }
};

// A logit as it counts: not a number: never drawn, as -infinity; +infinity: as the largest
// finite value; -0: as 0.
__device__ __forceinline__ float clean(float x) { return x == x ? fminf(x, FLT_MAX) + 0.0f : -INFINITY; }

// Place in the descending order, as a number: larger first. (No two are the same.)
__device__ __forceinline__ u64 place_of(float x, int i) {
  const uint32_t b = __float_as_uint(x);
  return (u64)(b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u)) << 32 | (uint32_t)~i;
}
__device__ __forceinline__ float value_of(u64 place) {
  const uint32_t k = (uint32_t)(place >> 32);
  return __uint_as_float(k ^ ((uint32_t)((int32_t)~k >> 31) | 0x80000000u));
}
__device__ __forceinline__ int index_of(u64 place) { return (int)~(uint32_t)place; }

// Weights of a row, w 2^shift with w = 2^(y / 64), y = (x - max) 64 log2(e) / t: the
// power of the nearest whole step (a table, with the shift in it, and the exponent)
// times the rest's, |r| <= 1/2, by the series of exp(r ln2 / 64) to its fourth power:
// what is left out is below 2^-44 of it. |y| < 2^16 (Scale::clamp).
struct Weights {
  double max, rate;
  const double* pow2;  // in LDS
  __device__ __forceinline__ double scaled(float x) const {
    const double y = ((double)x - max) * rate, k = rint(y), r = y - k;
    const double p = fma(r, fma(r, fma(r, fma(r, 0x1.3b2ab6fba4e77p-31, 0x1.c6b08d704a0cp-23), 0x1.ebfbdff82c58fp-15),
                                0x1.62e42fefa39efp-7), 1.0);  // (ln2 / 64)^n / n!
    const int n = (int)k;
    return ldexp(p * pow2[n & (kSteps - 1)], n >> 6);
  }
  // to the nearest integer below 2^52, by the addition of 2^52
  static __device__ __forceinline__ u64 whole(double s) {
    return __double_as_longlong(s + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
  }
};

struct Least {
  __device__ __forceinline__ u64 operator()(u64 a, u64 b) const { return a < b ? a : b; }
};
struct Sum {
  __device__ __forceinline__ u64 operator()(u64 a, u64 b) const { return a + b; }
};
struct Largest {
  __device__ __forceinline__ u64 operator()(u64 a, u64 b) const { return a > b ? a : b; }
};
template <typename F>
__device__ __forceinline__ u64 wave_reduce(u64 v, F&& f) {
  v = f(v, (u64)lane_xor64<32>(v));
  v = f(v, (u64)lane_xor64<16>(v));
  v = f(v, (u64)lane_xor64<8>(v));
  v = f(v, (u64)lane_xor64<4>(v));
  v = f(v, (u64)lane_xor64<2>(v));
  return f(v, (u64)lane_xor64<1>(v));
}

// Running sums, over all threads, of a value of each. red: a word per wave, free again after the next barrier.
template <typename T>
__device__ __forceinline__ T block_scan(T v, u64* red) {
  T incl = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const T a = __shfl_up(incl, d);
    if ((int)(threadIdx.x & 63) >= d) incl += a;
  }
  if ((threadIdx.x & 63) == 63) red[threadIdx.x >> 6] = (u64)incl;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kWaves - 1; ++k)
    if (k < (int)(threadIdx.x >> 6)) incl += (T)red[k];
  return incl;
}

// The first of n > 0 places (n <= 64 * 64) at which met(i) holds, the last where it does
// nowhere; met grows with i. A wave's work, with all of its lanes.
template <typename F>
__device__ __forceinline__ int first_met(int n, F&& met) {
  const int lane = threadIdx.x & 63, step = (n + 63) / 64;
  const u64 a = __ballot(met(min(n - 1, (lane + 1) * step - 1)));
  if (a == 0) return n - 1;
  const int i0 = (__ffsll(a) - 1) * step;
  const u64 b = __ballot(lane < step && i0 + lane < n && met(min(n - 1, i0 + lane)));
  return i0 + __ffsll(b) - 1;
}

// A row's settings, its extent, and what its weights and bins are then.
struct Setting {
  float t, p, min_p, u;
  int k;
};
__device__ __forceinline__ Setting setting_of(const SampleArgs& a, int r) {
  Setting g;
  g.t = a.temperature ? a.temperature[r] : 1.f;
  const float p = a.top_p ? a.top_p[r] : 1.f;
  g.p = p < 0.f ? 0.f : p;  // (-infinity times a sum of 0 would be no number)
  g.min_p = a.min_p ? a.min_p[r] : 0.f;
  g.k = a.top_k ? a.top_k[r] : 0;
  const float u = a.u[r];
  g.u = u > 0.f ? fminf(u, 1.f - 0x1p-24f) : 0.f;
  return g;
}
// The place of the largest element, and the least finite one.
struct Extent {
  u64 top;
  float lo;
};
// Of a whole row, from its slices'.
__device__ __forceinline__ Extent row_extent(const SampleArgs& a, int r) {
  static_assert(kSampleSlices <= 64, "one a lane");
  const int i = threadIdx.x & 63;
  SampleExtent e = {0, ~0ull};
  if (i < a.slices) e = a.extents[(size_t)r * a.slices + i];
  const u64 top = wave_reduce(e.top, Largest()), lo = wave_reduce(e.lo, Least());
  return {top, value_of(lo)};
}
// Greedy rows, and those of which nothing may be drawn, need no more than that.
__device__ __forceinline__ bool no_weights(const Setting& g, const Extent& e) {
  return !(g.t > 0.f) || g.k == 1 || value_of(e.top) == -INFINITY;
}
struct Scale {
  Weights weights;
  float max, cut;  // logits below `cut` have no weight
  float per;       // bins: (max - x) per
  bool far;        // the temperature is so high that there is no such cut
  int near;        // bins that are listed while the histogram is made
  int shift;
  // A logit as its weight needs it: neither below the cut nor above the largest. (Not a number: the cut.)
  __device__ __forceinline__ float clamp(float v) const { return fminf(fmaxf(v, cut), max); }
  template <bool FAR>
  __device__ __forceinline__ u64 weight(float v) const {
    const u64 w = Weights::whole(weights.scaled(clamp(v)));
    return FAR && !(v > -INFINITY) ? 0 : w;
  }
  __device__ __forceinline__ u64 weight_of(float v) const { return far ? weight<true>(v) : weight<false>(v); }
  __device__ __forceinline__ float distance(float v) const { return fminf((max - clamp(v)) * per, kBins - 0.5f); }
  __device__ __forceinline__ int bin_of(float v) const { return (int)distance(v); }
};
__device__ __forceinline__ Scale scale_of(const Setting& g, const Extent& e, int shift, const double* pow2) {
  Scale c;
  c.max = value_of(e.top);
  // a weight of 2^-(shift + 2) rounds to none, and so does the cut's: it lies no nearer to the largest
  const float reach = (shift + 2) * 0.6931472f * g.t;
  c.cut = c.max - reach;
  if ((double)c.max - (double)c.cut < (double)reach) c.cut = value_of(place_of(c.cut, 0) - (1ull << 32));
  c.far = !(c.cut >= -FLT_MAX);
  if (c.far) c.cut = -FLT_MAX;
  // (the second rate: temperatures for which the logit next to the largest has no weight)
  c.weights = {(double)c.max, fmin(1.4426950408889634 * kSteps / (double)g.t, 65536.0 / ((double)c.max - (double)c.cut)), pow2};
  // The bins span the finite logits, as far as they have weight. (Infinite, or next to nothing:
  // one bin. A mask of a finite value counts as a logit: the bins then span the whole reach, and
  // as temperatures rise and limits lie far out, the bins looked into hold more than the list.
  // One row of 128256 unit-normal logits, top_p 0.9, t = 1: 30 us, with one logit of -1e4 86;
  // top_k 20000 too, t = 2, half of them masked: -infinity 32, -1e4 340.)
  const float used = fminf(c.max - e.lo, reach);
  c.per = used > 1e-30f ? kBins / used : 0.f;
  c.near = min(kBins, (int)fminf(kNear * g.t * c.per, (float)kBins));
  c.shift = shift;
  return c;
}
// The table, with a barrier to come before it is read.
__device__ __forceinline__ void fill_table(double* pow2, int shift) {
  if (threadIdx.x < kSteps) pow2[threadIdx.x] = ldexp(kPow2[threadIdx.x], shift);
}

// A slice of a row: its extent. (And the row's state is cleared for the next kernel.)
template <bool BF16>
__global__ __launch_bounds__(kThreads) void sample_extent_kernel(SampleArgs a) {
  __shared__ u64 red[2][kWaves];
  const int r = blockIdx.x / a.slices, s = blockIdx.x - r * a.slices;
  const int first = s * a.slice_len;
  const Logits<BF16> x(a.logits, (int64_t)(a.row0 + r) * a.stride, first, min(a.slice_len, a.vocab - first));
  // the largest, the first run that holds it, and the least finite one
  float top = -INFINITY, lo = INFINITY;
  int at = first;
  x.template each<8>([&](const auto& v) {
    constexpr int N = sizeof v.x / 4;
    float hi = v.x[0], least = v.x[0];
#pragma unroll
    for (int j = 1; j < N; ++j) {
      hi = fmaxf(hi, v.x[j]);
      least = fminf(least, v.x[j]);
    }
    hi = fminf(hi, hi == hi ? FLT_MAX : -INFINITY);
    if (hi > top || (N == 1 && hi == top && v.first < at)) {
      top = hi;
      at = v.first;
    }
    if (!(least > -INFINITY)) {  // masked ones among them
      least = INFINITY;
#pragma unroll
      for (int j = 0; j < N; ++j) least = fminf(least, v.x[j] > -INFINITY ? v.x[j] : INFINITY);
    }
    lo = fminf(lo, least);
  });
  uint32_t* state = reinterpret_cast<uint32_t*>(a.state + r);
  constexpr int words = offsetof(SampleState, near) / 4;
  for (int i = s * kThreads + threadIdx.x; i < words; i += a.slices * kThreads) state[i] = 0;
  const u64 t = wave_reduce(place_of(clean(top), at), Largest()), l = wave_reduce(place_of(clean(lo), 0), Least());
  if ((threadIdx.x & 63) == 0) {
    red[0][threadIdx.x >> 6] = t;
    red[1][threadIdx.x >> 6] = l;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  SampleExtent e = {red[0][0], red[1][0]};
  for (int w = 1; w < kWaves; ++w) e = {Largest()(e.top, red[0][w]), Least()(e.lo, red[1][w])};
  // the element itself, in its run (a run of one, before the first or behind the last whole one, stands alone)
  int i = index_of(e.top);
  const float value = value_of(e.top);
  while (i + 1 < first + x.n && clean(x.at(i)) != value) ++i;
  e.top = place_of(value, i);
  a.extents[blockIdx.x] = e;
}

// What is searched for: the first element whose running count reaches `count`, or
// (count 0) whose running weight reaches `weight`, or (strict) passes it.
struct Target {
  uint32_t count;
  double weight;
  bool strict;
  __device__ __forceinline__ bool met(uint32_t c, u64 w) const {
    if (count) return c >= count;
    return strict ? (double)w > weight : (double)w >= weight;
  }
};

// Running sums over a row's bins, in LDS.
struct Bins {
  u64 w[kBins];
  uint32_t c[kBins];
  __device__ __forceinline__ u64 w_before(int b) const { return b ? w[b - 1] : 0; }
  __device__ __forceinline__ uint32_t c_before(int b) const { return b ? c[b - 1] : 0; }
  // The bin in which a target is met, the running sums before the first of them being (c0, w0).
  __device__ __forceinline__ int met(const Target& t, uint32_t c0 = 0, u64 w0 = 0) const {
    return first_met(kBins, [&](int i) { return t.met(c0 + c[i], w0 + w[i]); });
  }
  __device__ __forceinline__ void clear() {
    for (int i = threadIdx.x; i < kBins; i += kThreads) {
      w[i] = 0;
      c[i] = 0;
    }
  }
};
constexpr int kOwnBins = kBins / kThreads;  // of a thread, one after the other
// Each thread's bins into running sums.
__device__ __forceinline__ void scan_bins(Bins& s, u64 (&w)[kOwnBins], uint32_t (&c)[kOwnBins], u64 (*red)[kWaves]) {
#pragma unroll
  for (int k = 1; k < kOwnBins; ++k) {
    w[k] += w[k - 1];
    c[k] += c[k - 1];
  }
  const u64 w0 = block_scan(w[kOwnBins - 1], red[0]) - w[kOwnBins - 1];
  const uint32_t c0 = block_scan(c[kOwnBins - 1], red[1]) - c[kOwnBins - 1];
#pragma unroll
  for (int k = 0; k < kOwnBins; ++k) {
    s.w[threadIdx.x * kOwnBins + k] = w0 + w[k];
    s.c[threadIdx.x * kOwnBins + k] = c0 + c[k];
  }
  __syncthreads();
}

// A list of places, and the running weights of their elements once it is sorted.
template <int SIZE>
struct List {
  u64 key[SIZE], sum[SIZE];
  uint32_t at[SIZE];
  uint32_t lo, hi;
};

// The n <= SIZE listed places (no two the same) into descending order: counted into SIZE
// even parts of the range of distance(logit) (which grows as the logit falls), dealt to
// their parts' places, and ranked within a part, which few share (equal logits aside). A network over the same 518
// places took 16 us with a barrier a step, 11 us by waves and a merge of theirs.
template <int SIZE, typename D>
__device__ __forceinline__ void sort_list(List<SIZE>& s, int n, u64 (*red)[kWaves], D&& distance) {
  constexpr int PER = SIZE / kThreads;
  const int tid = threadIdx.x;
  if (tid == 0) {
    s.lo = __float_as_uint(INFINITY);
    s.hi = 0;
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) s.at[tid + k * kThreads] = 0;
  __syncthreads();
  u64 v[PER];
  float f[PER], lo = INFINITY, hi = 0.f;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int i = tid + k * kThreads;
    if (i >= n) continue;
    v[k] = s.key[i];
    f[k] = distance(value_of(v[k]));
    lo = fminf(lo, f[k]);
    hi = fmaxf(hi, f[k]);
  }
  if (tid < n) {  // (none is negative: their bits are in their order)
    atomicMin(&s.lo, __float_as_uint(lo));
    atomicMax(&s.hi, __float_as_uint(hi));
  }
  __syncthreads();
  lo = __uint_as_float(s.lo);
  const float range = __uint_as_float(s.hi) - lo, per = range > 1e-20f ? SIZE / range : 0.f;
  int part[PER];
  uint32_t slot[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    if (tid + k * kThreads >= n) continue;
    part[k] = min((int)((f[k] - lo) * per), SIZE - 1);
    slot[k] = atomicAdd(&s.at[part[k]], 1u);
  }
  __syncthreads();
  uint32_t own[PER], sum = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    own[k] = sum;
    sum += s.at[tid * PER + k];
  }
  const uint32_t before = block_scan(sum, red[0]) - sum;
#pragma unroll
  for (int k = 0; k < PER; ++k) s.at[tid * PER + k] = before + own[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < PER; ++k)
    if (tid + k * kThreads < n) s.sum[s.at[part[k]] + slot[k]] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    if (tid + k * kThreads >= n) continue;
    const int first = (int)s.at[part[k]], end = part[k] + 1 < SIZE ? (int)s.at[part[k] + 1] : n;
    int rank = first;
#pragma unroll 4
    for (int i = first; i < end; ++i) rank += s.sum[i] > v[k];
    s.key[rank] = v[k];
  }
  __syncthreads();
}
// Running weights of the sorted list into s.sum; gap(i) is what stands between element i
// and the one listed before it.
template <int SIZE, typename G>
__device__ __forceinline__ void scan_list(List<SIZE>& s, int n, const Scale& c, u64 (*red)[kWaves], G&& gap) {
  const int per = (n + kThreads - 1) / kThreads, i0 = threadIdx.x * per, i1 = min(n, i0 + per);
  u64 sum = 0;
  for (int i = i0; i < i1; ++i) {
    sum += gap(i) + c.weight_of(value_of(s.key[i]));
    s.sum[i] = sum;
  }
  const u64 w0 = block_scan(sum, red[1]) - sum;
  for (int i = i0; i < i1; ++i) s.sum[i] += w0;
  __syncthreads();
}

// Where a row's searches may end, given that the weights searched for are known up to the
// bins of the searches before: bins [from, to] each, none if to < from.
struct Search {
  int k_bin, p_from, p_to, m_from, m_to, u_from, u_to;
  int k_rank;  // which of its bin's elements is the k-th, from 0
  __device__ __forceinline__ int last() const { return max(max(k_bin, p_to), max(m_to, u_to)); }
  __device__ __forceinline__ bool wanted(int b) const {
    return b == k_bin || (b >= p_from && b <= p_to) || (b >= m_from && b <= m_to) || (b >= u_from && b <= u_to);
  }
};
__device__ __forceinline__ Search search_of(const Setting& g, const Scale& c, const Bins& s) {
  Search h = {-1, 0, -1, 0, -1, 0, -1, 0};
  u64 lo = s.w[kBins - 1], hi = lo;  // of the kept weight
  if (g.k > 0 && (uint32_t)g.k < s.c[kBins - 1]) {
    h.k_bin = s.met({(uint32_t)g.k, 0.0, false});
    h.k_rank = g.k - 1 - (int)s.c_before(h.k_bin);
    lo = s.w_before(h.k_bin);
    hi = s.w[h.k_bin];
  }
  if (g.p < 1.f) {
    h.p_from = s.met({0, (double)g.p * (double)lo, false});
    h.p_to = s.met({0, (double)g.p * (double)hi, false});
    lo = s.w_before(h.p_from);
    hi = s.w[h.p_to];
  }
  if (g.min_p > 0.f) {
    // the logit at which a weight is min_p: its bin, and the next ones for what rounding does
    // (a weight is 1 in fp64 down to a distance of 2^-54 t; none is above 1)
    const float ends = g.min_p < 1.f ? logf(g.min_p) : g.min_p > 1.f ? 0.f : -0x1p-54f;
    const int b = ends < 0.f ? c.bin_of(fmaxf(c.max + g.t * ends, -FLT_MAX)) : 0;
    h.m_from = max(0, b - 1);
    h.m_to = min(kBins - 1, b + 1);
    if (s.w[h.m_to] <= lo) {  // min_p ends before the others
      h.k_bin = -1;
      h.p_from = 0;
      h.p_to = -1;
    } else if (s.w_before(h.m_from) >= hi) {  // or behind them
      h.m_from = 0;
      h.m_to = -1;
    }
    if (h.m_to >= h.m_from) {
      lo = Least()(lo, s.w_before(h.m_from));
      hi = Least()(hi, s.w[h.m_to]);
    }
  }
  h.u_from = s.met({0, (double)g.u * (double)lo, true});
  h.u_to = s.met({0, (double)g.u * (double)hi, true});
  return h;
}

struct Pick {
  u64 place, kept_w;
  bool some;  // (min_p above 1 keeps nothing but the first token)
};
__device__ __forceinline__ void answer(const SampleArgs& a, int r, const Scale& c, const Pick& f) {
  if (threadIdx.x != 0) return;
  a.tokens[r] = index_of(f.place);
  if (a.probs) a.probs[r] = f.some ? (float)(c.weights.scaled(c.clamp(value_of(f.place))) / (double)f.kept_w) : 1.f;
}
// As pick_listed, of at most 64 elements: all in the registers of a wave (every wave does
// the same).
template <int SIZE, typename W>
__device__ __forceinline__ Pick pick_few(List<SIZE>& s, int n, const Setting& g, const Scale& c, const Search& h, W&& w_before) {
  const int lane = threadIdx.x & 63;
  u64 place = lane < n ? s.key[lane] : 0;
  int rank = 0;
#pragma unroll 4
  for (int j = 0; j < n; ++j) rank += s.key[j] > place;
  __syncthreads();
  if ((int)threadIdx.x < n) s.key[rank] = place;
  __syncthreads();
  place = s.key[min(lane, n - 1)];
  const float x = value_of(place);
  const int b = c.bin_of(x);
  int before = __shfl_up(b, 1);
  if (lane == 0) before = -1;
  const u64 own = lane < n ? c.weight_of(x) : 0;
  u64 sum = own;
  if (b != before) sum += w_before(b) - w_before(before + 1);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const u64 w = __shfl_up(sum, d);
    if (lane >= d) sum += w;
  }
  // the first of the elements that does, the last where none does
  auto first = [&](bool does) {
    const u64 m = __ballot(does && lane < n);
    return m ? __ffsll(m) - 1 : n - 1;
  };
  Pick f = {0, w_before(kBins), true};
  if (h.k_bin >= 0) f.kept_w = __shfl(sum, min(first(b >= h.k_bin) + h.k_rank, n - 1));
  if (h.p_to >= h.p_from) f.kept_w = __shfl(sum, first((double)sum >= (double)g.p * (double)f.kept_w));
  if (h.m_to >= h.m_from) {
    const bool keeps = c.weights.scaled(c.clamp(x)) >= ldexp((double)g.min_p, c.shift);
    const int j = first(!keeps);
    const u64 all = w_before(h.m_to + 1), m = __shfl((int)keeps, j) ? all : Least()(all, __shfl(sum - own, j));
    f.some = m > 0;
    f.kept_w = Least()(f.kept_w, m);
  }
  f.place = __shfl(place, first((double)sum > (double)g.u * (double)f.kept_w));
  return f;
}
// The token, from the n listed elements, all of the wanted bins' among them.
// w_before(b): running weights; distance: as sort_list takes it.
template <int SIZE, typename W, typename D>
__device__ __forceinline__ Pick pick_listed(List<SIZE>& s, int n, const Setting& g, const Scale& c, const Search& h,
                                            u64 (*red)[kWaves], W&& w_before, D&& distance) {
  n = max(n, 1);  // (the element drawn is always there)
  if (n <= 64) return pick_few(s, n, g, c, h, w_before);
  sort_list(s, n, red, distance);
  auto bin_at = [&](int i) { return c.bin_of(value_of(s.key[i])); };
  scan_list(s, n, c, red, [&](int i) -> u64 {
    const int b = bin_at(i), before = i ? bin_at(i - 1) : -1;
    return b == before ? 0 : w_before(b) - w_before(before + 1);
  });
  Pick f = {0, w_before(kBins), true};
  if (h.k_bin >= 0) f.kept_w = s.sum[min(first_met(n, [&](int i) { return bin_at(i) >= h.k_bin; }) + h.k_rank, n - 1)];
  if (h.p_to >= h.p_from) {
    const double want = (double)g.p * (double)f.kept_w;
    f.kept_w = s.sum[first_met(n, [&](int i) { return (double)s.sum[i] >= want; })];
  }
  if (h.m_to >= h.m_from) {
    // the elements that min_p keeps come first
    const double least = ldexp((double)g.min_p, c.shift);
    auto keeps = [&](int i) { return c.weights.scaled(c.clamp(value_of(s.key[i]))) >= least; };
    const int j = first_met(n, [&](int i) { return !keeps(i); });
    const u64 all = w_before(h.m_to + 1), m = keeps(j) ? all : Least()(all, s.sum[j] - c.weight_of(value_of(s.key[j])));
    f.some = m > 0;
    f.kept_w = Least()(f.kept_w, m);
  }
  const double want = (double)g.u * (double)f.kept_w;
  f.place = s.key[first_met(n, [&](int i) { return (double)s.sum[i] > want; })];
  return f;
}

// Stores and loads of what another workgroup of the same launch reads or has written: past
// the L2s (agent scope), so that a ticket need only wait for them to arrive. A fence would
// write back all of an L2, 20 us of it.
template <typename T>
__device__ __forceinline__ void put(T* p, T v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename T>
__device__ __forceinline__ T get(const T* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// Whether this workgroup is the last of n to come here. With barriers.
__device__ __forceinline__ bool last_of(uint32_t n, uint32_t* tickets, uint32_t& mine) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // each wave's own stores and atomics have arrived
  __syncthreads();
  if (threadIdx.x == 0) mine = atomicAdd(tickets, 1u);
  __syncthreads();
  return mine == n - 1;
}

// A slice of a row: its weights into the row's histogram, its likely tokens into the
// row's list. The last of the row's workgroups to be done draws the token, or leaves
// what it has found out to the next kernel where the listed tokens do not tell.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void sample_weights_kernel(SampleArgs a) {
  __shared__ __attribute__((aligned(16))) Bins bins;
  __shared__ List<kSampleNear> list;
  __shared__ u64 red[2][kWaves];
  __shared__ double pow2[kSteps];
  __shared__ uint32_t n, base;
  const int r = blockIdx.x / a.slices, out = a.row0 + r, slice = blockIdx.x - r * a.slices, tid = threadIdx.x;
  const Setting g = setting_of(a, out);
  const Extent e = row_extent(a, r);
  if (no_weights(g, e)) {
    const bool none = value_of(e.top) == -INFINITY;
    if (tid == 0 && slice == 0) {
      a.tokens[out] = none ? 0 : index_of(e.top);
      if (a.probs) a.probs[out] = none ? 0.f : 1.f;
    }
    return;
  }
  bins.clear();
  if (tid == 0) n = 0;
  fill_table(pow2, a.shift);
  const Scale c = scale_of(g, e, a.shift, pow2);
  const bool count = g.k > 0 && g.k < a.vocab;
  __syncthreads();
  const int first = slice * a.slice_len;
  const Logits<BF16> x(a.logits, (int64_t)out * a.stride, first, min(a.slice_len, a.vocab - first));
  bool listing = true;  // the list has room yet
  // (a run's weights are formed together, with their reads of the table in flight together)
  auto add = [&](auto far, const auto& v) {
    constexpr int N = sizeof v.x / 4;
    u64 w[N];
    int b[N], least = kBins;
#pragma unroll
    for (int j = 0; j < N; ++j) w[j] = c.weight<decltype(far)::value>(v.x[j]);
#pragma unroll
    for (int j = 0; j < N; ++j) b[j] = c.bin_of(v.x[j]);
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (w[j]) {
        atomicAdd(&bins.w[b[j]], w[j]);
        least = min(least, b[j]);
      }
    if (count) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (w[j]) atomicAdd(&bins.c[b[j]], 1u);
    }
    if (least < c.near && listing) {
      asm volatile("" ::: "memory");  // (keeps the read of n, which waits for the additions above, in here)
      listing = n < kNearList;
      if (!listing) return;
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (w[j] && b[j] < c.near) {
          const uint32_t at = atomicAdd(&n, 1u);
          if (at < kNearList) list.key[at] = place_of(clean(v.x[j]), v.first + j);
        }
    }
  };
  if (c.far) x.template each<2>([&](const auto& v) { add(std::true_type{}, v); });
  else x.template each<4>([&](const auto& v) { add(std::false_type{}, v); });
  __syncthreads();
  SampleState& st = a.state[r];
  // (a slice whose list may have lost some counts as more than the row's list holds)
  const uint32_t mine = n < kNearList ? n : kNearList + 1;
  if (tid == 0) base = mine ? atomicAdd(&st.n_near, mine) : 0;
  for (int i = tid; i < kBins; i += kThreads) {
    if (bins.w[i]) atomicAdd(&st.w[i], bins.w[i]);
    if (bins.c[i]) atomicAdd(&st.c[i], bins.c[i]);
  }
  __syncthreads();
  if (mine <= kNearList)
    for (int i = tid; i < (int)mine; i += kThreads)
      if (base + i < kNearList) put(&st.near[base + i], list.key[i]);
  if (!last_of(a.slices, &st.slices_done, base)) return;

  u64 own_w[kOwnBins];
  uint32_t own_c[kOwnBins];
#pragma unroll
  for (int k = 0; k < kOwnBins; ++k) {
    own_w[k] = get(&st.w[tid * kOwnBins + k]);
    own_c[k] = count ? get(&st.c[tid * kOwnBins + k]) : 0;
  }
  const uint32_t listed = get(&st.n_near);
  if (tid == 0) n = 0;
  scan_bins(bins, own_w, own_c, red);
  const Search h = search_of(g, c, bins);
  if (listed > kNearList || h.last() >= c.near) {
    // running sums, for the next kernel, and where to look
#pragma unroll
    for (int k = 0; k < kOwnBins; ++k) st.w[tid * kOwnBins + k] = bins.w[tid * kOwnBins + k];
    if (tid == 0) {
      st.search[0] = h.k_bin; st.search[1] = h.p_from; st.search[2] = h.p_to; st.search[3] = h.m_from;
      st.search[4] = h.m_to;  st.search[5] = h.u_from; st.search[6] = h.u_to;  st.search[7] = h.k_rank;
      st.pending = 1;
    }
    return;
  }
  for (int i = tid; i < (int)listed; i += kThreads) {
    const u64 q = get(&st.near[i]);
    if (h.wanted(c.bin_of(value_of(q)))) list.key[atomicAdd(&n, 1u)] = q;
  }
  __syncthreads();
  const Pick f = pick_listed(
      list, (int)n, g, c, h, red, [&](int b) { return bins.w_before(b); }, [&](float v) { return c.distance(v); });
  answer(a, out, c, f);
}

// A part of a row that the kernel before left: its elements of the wanted bins. The last
// of the row's workgroups draws the token from them.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void sample_rest_kernel(SampleArgs a) {
  __shared__ union {
    List<kList> list;
    Bins bins;
  } s;
  // 0, or of which wanted bin it is, from 1 to 255 and no further. (A look-up per element,
  // in place of four ranges: half the time.)
  __shared__ uint8_t wanted[kBins];
  __shared__ u64 red[2][kWaves];
  __shared__ double pow2[kSteps];
  __shared__ uint32_t n, base;
  const int r = blockIdx.x / a.parts, out = a.row0 + r, tid = threadIdx.x;
  SampleState& st = a.state[r];
  if (!const_load(&st.pending)) return;
  const Search h = {st.search[0], st.search[1], st.search[2], st.search[3], st.search[4], st.search[5], st.search[6], st.search[7]};
  const Setting g = setting_of(a, out);
  const Extent e = row_extent(a, r);
  fill_table(pow2, a.shift);
  const Scale c = scale_of(g, e, a.shift, pow2);
  if (tid == 0) n = 0;
  uint32_t bits = 0;
  static_assert(kOwnBins <= 32, "a bit each");
#pragma unroll
  for (int k = 0; k < kOwnBins; ++k) bits |= (uint32_t)h.wanted(tid * kOwnBins + k) << k;
  uint32_t ordinal = block_scan((uint32_t)__popc(bits), red[0]) - __popc(bits);
#pragma unroll
  for (int k = 0; k < kOwnBins; ++k) {
    const bool is = bits >> k & 1;
    ordinal += is;
    wanted[tid * kOwnBins + k] = is ? (uint8_t)min(ordinal, 255u) : 0;
  }
  __syncthreads();
  // List the elements that take(value, index) and also(value) want; n (0 before) counts
  // all of them, and the first kList to arrive are there.
  auto gather = [&](const Logits<BF16>& x, auto&& take, auto&& also) {
    x.template each<8>([&](const auto& v) {
      constexpr int N = sizeof v.x / 4;
      bool any = false, takes[N];
#pragma unroll
      for (int j = 0; j < N; ++j) any |= takes[j] = take(v.x[j], v.first + j);
      if (!any) return;
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (takes[j] && also(v.x[j])) {
          const uint32_t at = atomicAdd(&n, 1u);
          if (at < kList) s.list.key[at] = place_of(clean(v.x[j]), v.first + j);
        }
    });
    __syncthreads();
  };
  // (The elements at the cut have no weight.)
  const int first = (blockIdx.x - r * a.parts) * a.part_len;
  const float least_v = c.far ? -INFINITY : c.cut;
  gather(Logits<BF16>(a.logits, (int64_t)out * a.stride, first, max(0, min(a.part_len, a.vocab - first))),
         [&](float v, int) { return wanted[c.bin_of(v)] != 0; }, [&](float v) { return v > least_v; });
  const uint32_t mine = n;
  if (tid == 0) base = mine ? atomicAdd(&st.n_list, mine) : 0;
  __syncthreads();
  for (uint32_t i = tid; i < min(mine, (uint32_t)kList); i += kThreads)
    if (base + i < kList) put(&st.list[base + i], s.list.key[i]);
  if (!last_of(a.parts, &st.parts_done, base)) return;
  const uint32_t all = get(&st.n_list);
  if (all <= kList) {
    for (int i = tid; i < (int)all; i += kThreads) s.list.key[i] = get(&st.list[i]);
    __syncthreads();
    // (distances without the bins between that are not wanted; as they are from the 255th wanted one on)
    const Pick f = pick_listed(s.list, (int)all, g, c, h, red, [&](int b) { return b ? st.w[b - 1] : 0; }, [&](float v) {
      const float d = c.distance(v);
      return wanted[(int)d] + (wanted[(int)d] < 255 ? d - truncf(d) : d);
    });
    answer(a, out, c, f);
    return;
  }
  // Bins that hold more than the list (many equal logits): each search goes to its bin by
  // the running sums, and narrows the places of that by histograms of its own until the
  // list holds what is left.
  const Logits<BF16> x(a.logits, (int64_t)out * a.stride, 0, a.vocab);
  auto w_before = [&](int b) { return b ? st.w[b - 1] : 0; };
  Pick f = {0, w_before(kBins), true};
  u64 min_w = f.kept_w;
  if (h.m_to >= h.m_from) {
    const double least = ldexp((double)g.min_p, a.shift);
    u64 sum = 0;
    x.template each<4>([&](const auto& v) {
      for (const float y : v.x) {
        const int b = c.bin_of(y);
        if (b < h.m_from || b > h.m_to) continue;
        const u64 w = c.weight_of(y);
        if (w && c.weights.scaled(c.clamp(y)) >= least) sum += w;
      }
    });
    sum = wave_reduce(sum, Sum());
    if ((tid & 63) == 0) red[0][tid >> 6] = sum;
    __syncthreads();
    min_w = w_before(h.m_from) + red[0][0] + red[0][1] + red[0][2] + red[0][3];
    f.some = min_w > 0;
  }
  for (int stage = 0; stage < 3; ++stage) {
    if (stage == 0 ? h.k_bin < 0 : stage == 1 && h.p_to < h.p_from) continue;
    if (stage == 2) f.kept_w = Least()(f.kept_w, min_w);
    const Target t = {stage == 0 ? (uint32_t)g.k : 0u, (double)(stage == 1 ? g.p : g.u) * (double)f.kept_w, stage == 2};
    const int bin = stage == 0 ? h.k_bin : first_met(kBins, [&](int i) { return t.met(0, st.w[i]); });
    u64 w0 = w_before(bin), from = ~0ull, to = 0;
    uint32_t c0 = stage == 0 ? (uint32_t)(g.k - 1 - h.k_rank) : 0u, left = kList + 1;
    x.template each<4>([&](const auto& v) {
#pragma unroll
      for (int j = 0; j < (int)(sizeof v.x / 4); ++j) {
        if (c.bin_of(v.x[j]) != bin || !(v.x[j] > least_v)) continue;
        const u64 q = place_of(clean(v.x[j]), v.first + j);
        from = Least()(from, q);
        to = Largest()(to, q);
      }
    });
    from = wave_reduce(from, Least());
    to = wave_reduce(to, Largest());
    __syncthreads();
    if ((tid & 63) == 0) {
      red[0][tid >> 6] = from;
      red[1][tid >> 6] = to;
    }
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) {
      from = Least()(from, red[0][w]);
      to = Largest()(to, red[1][w]);
    }
    while (left > kList) {
      int sh = 0;
      while (((to - from) >> sh) >= kBins) ++sh;
      __syncthreads();
      s.bins.clear();
      __syncthreads();
      x.template each<4>([&](const auto& v) {
        // (a run's elements of one bin are added together: equal logits beside each other are)
        int last = -1;
        u64 w_sum = 0;
        uint32_t c_sum = 0;
        auto add = [&] {
          atomicAdd(&s.bins.w[last], w_sum);
          atomicAdd(&s.bins.c[last], c_sum);
        };
        for (int j = 0; j < (int)(sizeof v.x / 4); ++j) {
          const u64 q = place_of(clean(v.x[j]), v.first + j);
          if (q < from || q > to) continue;
          const u64 w = c.weight_of(v.x[j]);
          if (w == 0) continue;
          const int b = (int)((to - q) >> sh);
          if (b != last && last >= 0) {
            add();
            w_sum = 0;
            c_sum = 0;
          }
          last = b;
          w_sum += w;
          ++c_sum;
        }
        if (last >= 0) add();
      });
      __syncthreads();
      u64 own_w[kOwnBins];
      uint32_t own_c[kOwnBins];
#pragma unroll
      for (int k = 0; k < kOwnBins; ++k) {
        own_w[k] = s.bins.w[tid * kOwnBins + k];
        own_c[k] = s.bins.c[tid * kOwnBins + k];
      }
      scan_bins(s.bins, own_w, own_c, red);
      const int b = s.bins.met(t, c0, w0);
      left = s.bins.c[b] - s.bins.c_before(b);
      c0 += s.bins.c_before(b);
      w0 += s.bins.w_before(b);
      to -= (u64)b << sh;
      const u64 span = ((u64)1 << sh) - 1;
      from = to - from > span ? to - span : from;
    }
    __syncthreads();
    if (tid == 0) n = 0;
    __syncthreads();
    gather(x, [&](float v, int i) {
      const u64 q = place_of(clean(v), i);
      return q >= from && q <= to;
    }, [&](float v) { return c.weight_of(v) != 0; });
    const int m = max(1, (int)min(n, (uint32_t)kList));
    sort_list(s.list, m, red, [&](float v) { return c.distance(v); });
    scan_list(s.list, m, c, red, [](int) -> u64 { return 0; });
    const int j = first_met(m, [&](int i) { return t.met(c0 + i + 1, w0 + s.list.sum[i]); });
    f.place = s.list.key[j];
    if (stage < 2) f.kept_w = w0 + s.list.sum[j];
  }
  answer(a, out, c, f);
}

}  // namespace

void launch_sample(hipStream_t s, SampleArgs a) {
  int bits = 0;
  while (((int64_t)1 << bits) < a.vocab) ++bits;
  a.shift = std::min(45, 62 - bits);
  const int rows = a.rows;
  for (a.row0 = 0; a.row0 < rows; a.row0 += kSampleRows) {
    a.rows = std::min(rows - a.row0, kSampleRows);
    sample_slices(a.rows, a.vocab, &a.slices, &a.slice_len);
    sample_parts(a.rows, a.vocab, &a.parts, &a.part_len);
    auto go = [&](auto bf16) {
      constexpr bool B = decltype(bf16)::value;
      sample_extent_kernel<B><<<a.rows * a.slices, kThreads, 0, s>>>(a);
      sample_weights_kernel<B><<<a.rows * a.slices, kThreads, 0, s>>>(a);
      sample_rest_kernel<B><<<a.rows * a.parts, kThreads, 0, s>>>(a);
    };
    a.bf16 ? go(std::true_type{}) : go(std::false_type{});
  }
}

}  // namespace hb
