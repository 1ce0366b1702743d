// Sampling from rows of logits: temperature, top-k, top-p, min-p, given random numbers.
//
// The tokens of a row stand in descending order of their logits, lower indices first
// among equals; every limit keeps a prefix of that order, and the token drawn is the
// first at which the running weight passes u times the kept weight. All of it is the
// same search -- for the k-th token, for the one that reaches p of the weight, for the
// one drawn -- in one cumulative distribution, so no row is sorted: a histogram over
// the logits' distances to their maximum tells the bin that holds an element searched
// for, and only the bins' elements (at most kList of them at a time) are sorted.
//
// Weights w = exp((x - max) / t) are formed in fp64 and summed as integers, w 2^shift
// rounded to the nearest, with a shift that keeps the sum of a row below 2^63: sums then
// do not depend on their order, and two programs that use 64 bits agree on every token
// unless u falls within some 2^-40 of a border. In fp32 they would not: 128256 even
// weights, each off by 2^-25, move some border past u in one row of 10^4 to 10^5.
#include <algorithm>
#include <cfloat>
#include <cstddef>

#include "hb_device.h"
#include "hb_kernels.h"

namespace hb {
namespace {

typedef unsigned long long u64;

constexpr int kBins = 2048;   // of a row's histogram: 1/64 of a factor e or less, over the 32 factors that have weight
constexpr int kList = 4096;   // elements sorted at a time
constexpr int kNearList = kSampleNear;
constexpr float kNear = 8.f;  // tokens whose weight is above e^-8 are listed while the histogram is made
constexpr int kSteps = 32;    // steps of an octave in the table of powers of two
constexpr int kSliceThreads = 256, kSliceList = 512, kRowThreads = 1024;
static_assert(kBins == kSampleBins, "workspace");

// The elements (fp32 or bf16) [first, first + n) of a row, f(value, index in the row) for each; any alignment.
template <bool BF16>
struct Logits {
  const uint16_t* h;
  const float* f;
  int first, n;
  __device__ __forceinline__ Logits(const void* p, int64_t row, int first, int n)
      : h(static_cast<const uint16_t*>(p) + row), f(static_cast<const float*>(p) + row), first(first), n(n) {}
  // Not a number: never drawn, as -infinity; +infinity: as the largest finite value; -0: as 0.
  static __device__ __forceinline__ float clean(float x) { return x == x ? fminf(x, FLT_MAX) + 0.0f : -INFINITY; }
  __device__ __forceinline__ float at(int i) const { return clean(BF16 ? bf16_to_f32(h[i]) : f[i]); }
  // LOADS 16-byte loads of a thread in flight
  template <int THREADS, int LOADS, typename F>
  __device__ __forceinline__ void each(F&& fn) const {
    constexpr int PER = BF16 ? 8 : 4, SIZE = BF16 ? 2 : 4;
    const int tid = threadIdx.x;
    const uintptr_t p = BF16 ? reinterpret_cast<uintptr_t>(h + first) : reinterpret_cast<uintptr_t>(f + first);
    const int head = min(n, (int)((16 - (p & 15)) & 15) / SIZE);  // elements before the first 16-byte boundary
    const int nv = (n - head) / PER, tail = head + nv * PER;
    if (tid < head) fn(at(first + tid), first + tid);
    if (tid < n - tail) fn(at(first + tail + tid), first + tail + tid);
    const u32x4* v = BF16 ? reinterpret_cast<const u32x4*>(h + first + head) : reinterpret_cast<const u32x4*>(f + first + head);
    for (int i0 = tid; i0 < nv; i0 += LOADS * THREADS) {
      u32x4 r[LOADS];
#pragma unroll
      for (int k = 0; k < LOADS; ++k)
        if (i0 + k * THREADS < nv) r[k] = v[i0 + k * THREADS];
#pragma unroll
      for (int k = 0; k < LOADS; ++k) {
        if (i0 + k * THREADS >= nv) break;
        const int e = first + head + (i0 + k * THREADS) * PER;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (BF16) {
            fn(clean(bf16_lo(r[k][j])), e + 2 * j);
            fn(clean(bf16_hi(r[k][j])), e + 2 * j + 1);
          } else {
            fn(clean(__uint_as_float(r[k][j])), e + j);
          }
        }
      }
    }
  }
};

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

// Weights of a row: w = 2^(y / 32), y = (x - max) 32 log2(e) / t, from the nearest whole
// step's power (a table and the exponent) and the rest's, |r| <= 1/2, the series of
// exp(r ln2 / 32) to its fifth power: what is left out is below 2^-48 of it.
struct Weights {
  double max, rate;
  int shift;
  const double* pow2;
  // w 2^shift, not rounded
  __device__ __forceinline__ double scaled(float x) const {
    // -infinity, and whatever is too far away: 2^-128, which rounds to none
    const double y = fmax(((double)x - max) * rate, -128.0 * kSteps);
    const double k = rint(y), a = (y - k) * (0.693147180559945309417 / kSteps);
    const double p = fma(a, fma(a, fma(a, fma(a, fma(a, 1.0 / 120, 1.0 / 24), 1.0 / 6), 0.5), 1.0), 1.0);
    const int n = (int)k;
    return ldexp(p * pow2[n & (kSteps - 1)], (n >> 5) + shift);
  }
  // to the nearest integer below 2^52, by the addition of 2^52
  static __device__ __forceinline__ u64 whole(double s) {
    return __double_as_longlong(s + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
  }
};

// f over all threads' values; every thread gets the result. red: a word per wave.
template <int THREADS, typename T, typename F>
__device__ __forceinline__ T block_reduce(T v, F&& f, u64* red) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v = f(v, (T)__shfl_xor(v, d));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = (u64)v;
  __syncthreads();
  T r = (T)red[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) r = f(r, (T)red[w]);
  __syncthreads();
  return r;
}
struct Least {
  __device__ __forceinline__ u64 operator()(u64 a, u64 b) const { return a < b ? a : b; }
};
struct Largest {
  __device__ __forceinline__ u64 operator()(u64 a, u64 b) const { return a > b ? a : b; }
};
struct Sum {
  __device__ __forceinline__ u64 operator()(u64 a, u64 b) const { return a + b; }
};

// Running sums, over all threads, of a value of each.
template <int THREADS, typename T>
__device__ __forceinline__ T block_scan(T v, u64* red) {
  T incl = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const T a = __shfl_up(incl, d);
    if ((int)(threadIdx.x & 63) >= d) incl += a;
  }
  if ((threadIdx.x & 63) == 63) red[threadIdx.x >> 6] = (u64)incl;
  __syncthreads();
  for (int k = 0; k < (int)(threadIdx.x >> 6); ++k) incl += (T)red[k];
  __syncthreads();
  return incl;
}

// A row's settings, its extent, and what its weights and bins are then.
struct Setting {
  float t, p, min_p, u;
  int k;
};
__device__ __forceinline__ Setting setting_of(const SampleArgs& a, int r) {
  Setting g;
  g.t = a.temperature ? a.temperature[r] : 1.f;
  g.p = a.top_p ? a.top_p[r] : 1.f;
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
template <int THREADS>
__device__ __forceinline__ Extent row_extent(const SampleArgs& a, int r, u64* red) {
  u64 top = 0, lo = ~0ull;
  for (int i = threadIdx.x; i < a.slices; i += THREADS) {
    const SampleExtent e = a.extents[(size_t)r * a.slices + i];
    top = Largest()(top, e.top);
    lo = Least()(lo, e.lo);
  }
  top = block_reduce<THREADS>(top, Largest(), red);
  return {top, value_of(block_reduce<THREADS>(lo, Least(), red))};
}
// Greedy rows, and those of which nothing may be drawn, need no more than that.
__device__ __forceinline__ bool no_weights(const Setting& g, const Extent& e) {
  return !(g.t > 0.f) || g.k == 1 || value_of(e.top) == -INFINITY;
}
struct Scale {
  Weights weight;
  float max, per;  // bins: (max - x) per
  double least;    // scaled weights that min_p keeps
  int near;        // bins that are listed while the histogram is made
  // (A NaN, from a scale of 0 or infinity, and the elements without weight: the last bin.)
  __device__ __forceinline__ int bin_of(float v) const { return (int)fminf((max - v) * per, (float)(kBins - 1)); }
};
__device__ __forceinline__ Scale scale_of(const Setting& g, const Extent& e, int shift, const double* pow2) {
  Scale c;
  c.max = value_of(e.top);
  // distances beyond which a weight rounds to none
  const float reach = fminf(c.max - e.lo, (shift + 2) * 0.6931472f * g.t);
  c.weight = {(double)c.max, 1.4426950408889634 * kSteps / (double)g.t, shift, pow2};
  c.per = reach > 0.f ? kBins / reach : 0.f;
  c.least = g.min_p > 0.f ? ldexp((double)g.min_p, shift) : 0.0;
  c.near = min(kBins, (int)fminf(kNear * g.t * c.per, (float)kBins));
  return c;
}
__device__ __forceinline__ void fill_table(double* pow2) {
  if (threadIdx.x < kSteps) pow2[threadIdx.x] = exp2((double)threadIdx.x / kSteps);
  __syncthreads();
}

template <bool BF16>
__device__ __forceinline__ Logits<BF16> slice_of(const SampleArgs& a, int r, int s) {
  const int first = s * a.slice_len;
  return Logits<BF16>(a.logits, (int64_t)(a.row0 + r) * a.stride, first, min(a.slice_len, a.vocab - first));
}

// A slice of a row: its extent. (And the row's state is cleared for the next kernel.)
template <bool BF16>
__global__ __launch_bounds__(kSliceThreads) void sample_extent_kernel(SampleArgs a) {
  __shared__ u64 red[kSliceThreads / 64];
  const int r = blockIdx.x / a.slices, s = blockIdx.x - r * a.slices;
  uint32_t* state = reinterpret_cast<uint32_t*>(a.state + r);
  constexpr int words = offsetof(SampleState, list) / 4;
  for (int i = s * kSliceThreads + threadIdx.x; i < words; i += a.slices * kSliceThreads) state[i] = 0;
  u64 top = 0;
  float lo = INFINITY;
  slice_of<BF16>(a, r, s).template each<kSliceThreads, 8>([&](float v, int i) {
    top = Largest()(top, place_of(v, i));
    lo = v > -INFINITY ? fminf(lo, v) : lo;
  });
  top = block_reduce<kSliceThreads>(top, Largest(), red);
  const u64 low = block_reduce<kSliceThreads>(place_of(lo, 0), Least(), red);
  if (threadIdx.x == 0) a.extents[blockIdx.x] = {top, low};
}

// A slice of a row: its weights into the row's histogram, its likely tokens into the row's list.
template <bool BF16>
__global__ __launch_bounds__(kSliceThreads) void sample_weights_kernel(SampleArgs a) {
  __shared__ u64 hist_w[kBins];
  __shared__ uint32_t hist_c[kBins];
  __shared__ u64 list[kSliceList];
  __shared__ u64 red[kSliceThreads / 64];
  __shared__ double pow2[kSteps];
  __shared__ uint32_t n, base;
  const int r = blockIdx.x / a.slices, tid = threadIdx.x;
  const Setting g = setting_of(a, a.row0 + r);
  const Extent e = row_extent<kSliceThreads>(a, r, red);
  if (no_weights(g, e)) return;
  for (int i = tid; i < kBins; i += kSliceThreads) {
    hist_w[i] = 0;
    hist_c[i] = 0;
  }
  if (tid == 0) n = 0;
  fill_table(pow2);
  const Scale c = scale_of(g, e, a.shift, pow2);
  const bool count = g.k > 0 && g.k < a.vocab;
  u64 min_w = 0;
  slice_of<BF16>(a, r, blockIdx.x - r * a.slices).template each<kSliceThreads, 4>([&](float v, int i) {
    const double ws = c.weight.scaled(v);
    const u64 w = Weights::whole(ws);
    if (w == 0) return;
    const int b = c.bin_of(v);
    atomicAdd(&hist_w[b], w);
    if (count) atomicAdd(&hist_c[b], 1u);
    if (ws >= c.least) min_w += w;
    if (b < c.near && n < kSliceList) {
      const uint32_t at = atomicAdd(&n, 1u);
      if (at < kSliceList) list[at] = place_of(v, i);
    }
  });
  min_w = block_reduce<kSliceThreads>(min_w, Sum(), red);
  SampleState& st = a.state[r];
  // (a slice whose list may have lost some counts as more than the row's list holds)
  const uint32_t listed = n < kSliceList ? n : kNearList + 1;
  if (tid == 0) {
    if (min_w) atomicAdd(&st.min_w, min_w);
    base = listed ? atomicAdd(&st.n, listed) : 0;
  }
  __syncthreads();
  for (int i = tid; i < kBins; i += kSliceThreads) {
    if (hist_w[i]) atomicAdd(&st.w[i], hist_w[i]);
    if (hist_c[i]) atomicAdd(&st.c[i], hist_c[i]);
  }
  if (listed <= kSliceList)
    for (int i = tid; i < (int)listed; i += kSliceThreads)
      if (base + i < kNearList) st.list[base + i] = list[i];
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

struct Smem {
  u64 w[kBins];
  uint32_t c[kBins];
  u64 key[kList], sum[kList];
  uint32_t cnt[kList];
  u64 red[kRowThreads / 64];
  double pow2[kSteps];
  uint32_t n, found;
};

// The histogram into running sums.
__device__ __forceinline__ void scan_hist(Smem& s) {
  __syncthreads();
  constexpr int PER = kBins / kRowThreads;
  static_assert(PER == 2, "two bins a thread");
  const int b = threadIdx.x * PER;
  const u64 w0 = s.w[b], w1 = w0 + s.w[b + 1];
  const uint32_t c0 = s.c[b], c1 = c0 + s.c[b + 1];
  const u64 w = block_scan<kRowThreads>(w1, s.red) - w1;
  const uint32_t c = block_scan<kRowThreads>(c1, s.red) - c1;
  s.w[b] = w + w0;
  s.w[b + 1] = w + w1;
  s.c[b] = c + c0;
  s.c[b + 1] = c + c1;
  __syncthreads();
}
// Running sums before bin b.
__device__ __forceinline__ u64 w_before(const Smem& s, int b) { return b ? s.w[b - 1] : 0; }
__device__ __forceinline__ uint32_t c_before(const Smem& s, int b) { return b ? s.c[b - 1] : 0; }

// The first of n > 0 places at which met(i) holds, the last where it does nowhere. (met grows with i.)
template <typename F>
__device__ __forceinline__ int first_met(Smem& s, int n, F&& met) {
  if (threadIdx.x == 0) s.found = (uint32_t)(n - 1);
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kRowThreads)
    if (met(i) && (i == 0 || !met(i - 1))) s.found = (uint32_t)i;
  __syncthreads();
  const int r = (int)s.found;
  __syncthreads();
  return r;
}
// The bin in which a target is met, the running sums before the first of them being (c0, w0).
__device__ __forceinline__ int bin_met(Smem& s, const Target& t, uint32_t c0 = 0, u64 w0 = 0) {
  return first_met(s, kBins, [&](int i) { return t.met(c0 + s.c[i], w0 + s.w[i]); });
}

// The s.n <= kList listed places into descending order.
__device__ __forceinline__ void sort_list(Smem& s) {
  const int n = (int)s.n, tid = threadIdx.x;
  int len = 2;
  while (len < n) len *= 2;
  for (int i = n + tid; i < len; i += kRowThreads) s.key[i] = 0;
  __syncthreads();
  for (int size = 2; size <= len; size *= 2)
    for (int d = size / 2; d >= 1; d /= 2) {
      for (int t = tid; t < len / 2; t += kRowThreads) {
        const int i = 2 * t - (t & (d - 1)), j = i + d;
        const u64 a = s.key[i], b = s.key[j];
        if ((a < b) == ((i & size) == 0)) {
          s.key[i] = b;
          s.key[j] = a;
        }
      }
      __syncthreads();
    }
}
// Running sums of the sorted list into s.sum and s.cnt; gap(i, w, c) adds what stands
// between element i and the one listed before it.
template <typename G>
__device__ __forceinline__ void scan_list(Smem& s, const Weights& weight, G&& gap) {
  constexpr int PER = kList / kRowThreads;
  const int n = (int)s.n, i0 = threadIdx.x * PER;
  u64 sum = 0;
  uint32_t cnt = 0;
  for (int i = i0; i < min(n, i0 + PER); ++i) {
    gap(i, sum, cnt);
    sum += Weights::whole(weight.scaled(value_of(s.key[i])));
    ++cnt;
    s.sum[i] = sum;
    s.cnt[i] = cnt;
  }
  const u64 w = block_scan<kRowThreads>(sum, s.red) - sum;
  const uint32_t c = block_scan<kRowThreads>(cnt, s.red) - cnt;
  for (int i = i0; i < min(n, i0 + PER); ++i) {
    s.sum[i] += w;
    s.cnt[i] += c;
  }
  __syncthreads();
}

// A row: the token, from its histogram and what has to be looked at of its elements.
template <bool BF16>
__global__ __launch_bounds__(kRowThreads) void sample_pick_kernel(SampleArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  Smem& s = *reinterpret_cast<Smem*>(smem);
  const int r = blockIdx.x, out = a.row0 + r, tid = threadIdx.x;
  const Setting g = setting_of(a, out);
  const Extent e = row_extent<kRowThreads>(a, r, s.red);
  if (no_weights(g, e)) {
    const bool none = value_of(e.top) == -INFINITY;
    if (tid == 0) {
      a.tokens[out] = none ? 0 : index_of(e.top);
      if (a.probs) a.probs[out] = none ? 0.f : 1.f;
    }
    return;
  }
  const SampleState& st = a.state[r];
  for (int i = tid; i < kBins; i += kRowThreads) {
    s.w[i] = st.w[i];
    s.c[i] = st.c[i];
  }
  const u64 min_w = st.min_w;
  const uint32_t listed = st.n;
  fill_table(s.pow2);
  const Scale c = scale_of(g, e, a.shift, s.pow2);
  scan_hist(s);
  // The bins that each search may end in, given that the weights searched for are
  // known up to the bins of the searches before: [from, to] each, none if to < from.
  const u64 all_w = s.w[kBins - 1];
  const bool by_k = g.k > 0 && (uint32_t)g.k < s.c[kBins - 1], by_p = g.p < 1.f;
  int k_bin = -1, p_from = 0, p_to = -1;
  u64 lo = all_w, hi = all_w;  // of the kept weight
  if (by_k) {
    k_bin = bin_met(s, {(uint32_t)g.k, 0.0, false});
    lo = w_before(s, k_bin);
    hi = s.w[k_bin];
  }
  if (by_p) {
    p_from = bin_met(s, {0, (double)g.p * (double)lo, false});
    p_to = bin_met(s, {0, (double)g.p * (double)hi, false});
    lo = w_before(s, p_from);
    hi = s.w[p_to];
  }
  if (min_w <= lo) {  // min_p ends before them
    k_bin = -1;
    p_from = 0;
    p_to = -1;
  }
  lo = Least()(lo, min_w);
  hi = Least()(hi, min_w);
  const int u_from = bin_met(s, {0, (double)g.u * (double)lo, true});
  const int u_to = bin_met(s, {0, (double)g.u * (double)hi, true});
  auto wanted = [&](int b) { return b == k_bin || (b >= p_from && b <= p_to) || (b >= u_from && b <= u_to); };
  const Logits<BF16> x(a.logits, (int64_t)out * a.stride, 0, a.vocab);
  // List the elements that take(value, index) wants and that have weight; s.n counts
  // all of them, and the first kList to arrive are there.
  auto gather = [&](auto&& take) {
    if (tid == 0) s.n = 0;
    __syncthreads();
    x.template each<kRowThreads, 8>([&](float v, int i) {
      if (!take(v, i) || Weights::whole(c.weight.scaled(v)) == 0) return;
      const uint32_t at = atomicAdd(&s.n, 1u);
      if (at < kList) s.key[at] = place_of(v, i);
    });
    __syncthreads();
  };
  const int last = max(max(k_bin, p_to), u_to);
  if (listed <= kNearList && last < c.near) {
    if (tid == 0) s.n = 0;
    __syncthreads();
    for (int i = tid; i < (int)listed; i += kRowThreads) {
      const u64 q = st.list[i];
      if (wanted(c.bin_of(value_of(q)))) s.key[atomicAdd(&s.n, 1u)] = q;
    }
    __syncthreads();
  } else {
    gather([&](float v, int) { return wanted(c.bin_of(v)); });
  }
  u64 kept_w = all_w, place = 0;
  if (s.n <= kList) {
    sort_list(s);
    auto bin_at = [&](int i) { return c.bin_of(value_of(s.key[i])); };
    scan_list(s, c.weight, [&](int i, u64& w, uint32_t& n) {
      const int b = bin_at(i), before = i ? bin_at(i - 1) : -1;
      if (b == before) return;
      w += w_before(s, b) - w_before(s, before + 1);
      n += c_before(s, b) - c_before(s, before + 1);
    });
    const int n = (int)s.n;
    if (k_bin >= 0) kept_w = s.sum[first_met(s, n, [&](int i) { return s.cnt[i] >= (uint32_t)g.k; })];
    if (p_to >= p_from) {
      const double want = (double)g.p * (double)kept_w;
      kept_w = s.sum[first_met(s, n, [&](int i) { return (double)s.sum[i] >= want; })];
    }
    kept_w = Least()(kept_w, min_w);
    const double want = (double)g.u * (double)kept_w;
    place = s.key[first_met(s, n, [&](int i) { return (double)s.sum[i] > want; })];
  } else {
    // Bins that hold more than the list (many equal logits): each search narrows the
    // places by histograms of its own until the list holds what is left.
    for (int stage = by_k ? 0 : by_p ? 1 : 2; stage < 3; ++stage) {
      if (stage == 1 && !by_p) continue;
      if (stage == 2) kept_w = Least()(kept_w, min_w);
      const Target t = {stage == 0 ? (uint32_t)g.k : 0u, (double)(stage == 1 ? g.p : g.u) * (double)kept_w, stage == 2};
      u64 to = e.top, from = place_of(e.lo, 0x7FFFFFFF), w0 = 0;
      uint32_t c0 = 0, n = kList + 1;
      while (n > kList) {
        int sh = 0;
        while (((to - from) >> sh) >= kBins) ++sh;
        __syncthreads();
        for (int i = tid; i < kBins; i += kRowThreads) {
          s.w[i] = 0;
          s.c[i] = 0;
        }
        __syncthreads();
        x.template each<kRowThreads, 8>([&](float v, int i) {
          const u64 q = place_of(v, i);
          if (q < from || q > to) return;
          const u64 w = Weights::whole(c.weight.scaled(v));
          if (w == 0) return;
          const int b = (int)((to - q) >> sh);
          atomicAdd(&s.w[b], w);
          atomicAdd(&s.c[b], 1u);
        });
        scan_hist(s);
        const int b = bin_met(s, t, c0, w0);
        n = s.c[b] - c_before(s, b);
        c0 += c_before(s, b);
        w0 += w_before(s, b);
        to -= (u64)b << sh;
        const u64 span = ((u64)1 << sh) - 1;
        from = to - from > span ? to - span : from;
      }
      gather([&](float v, int i) {
        const u64 q = place_of(v, i);
        return q >= from && q <= to;
      });
      sort_list(s);
      scan_list(s, c.weight, [](int, u64&, uint32_t&) {});
      const int j = first_met(s, (int)s.n, [&](int i) { return t.met(c0 + s.cnt[i], w0 + s.sum[i]); });
      place = s.key[j];
      kept_w = stage < 2 ? w0 + s.sum[j] : kept_w;
    }
  }
  if (tid != 0) return;
  a.tokens[out] = index_of(place);
  // (min_p above 1 keeps nothing but the first token)
  if (a.probs) a.probs[out] = min_w ? (float)(c.weight.scaled(value_of(place)) / (double)kept_w) : 1.f;
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
    auto go = [&](auto extent, auto weights, auto pick, std::atomic<uint64_t>& raised) {
      static_assert(sizeof(Smem) <= 160 * 1024, "LDS of a CU");
      raise_dynamic_lds(reinterpret_cast<const void*>(pick), sizeof(Smem), raised);
      extent<<<a.rows * a.slices, kSliceThreads, 0, s>>>(a);
      weights<<<a.rows * a.slices, kSliceThreads, 0, s>>>(a);
      pick<<<a.rows, kRowThreads, sizeof(Smem), s>>>(a);
    };
    static std::atomic<uint64_t> raised_f32{0}, raised_bf16{0};
    if (a.bf16) go(&sample_extent_kernel<true>, &sample_weights_kernel<true>, &sample_pick_kernel<true>, raised_bf16);
    else go(&sample_extent_kernel<false>, &sample_weights_kernel<false>, &sample_pick_kernel<false>, raised_f32);
  }
}

}  // namespace hb
