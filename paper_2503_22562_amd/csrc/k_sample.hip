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

#include "hb_device.h"
#include "hb_kernels.h"

namespace hb {
namespace {

typedef unsigned long long u64;

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 128, kCols = 32;  // bins of a histogram, copies of each (lane % 32), which keep lanes off each other's bins
constexpr int kList = 4096;             // elements sorted at a time
constexpr int kLoads = 8;               // 16-byte loads of a thread in flight
constexpr int kSteps = 32;              // steps of an octave in the table of powers of two

struct Smem {
  u64 hist_w[kBins * kCols];
  uint32_t hist_c[kBins * kCols];
  u64 key[kList], w[kList];
  u64 cum_w[kBins];
  uint32_t cum_c[kBins];
  u64 red[kWaves][4];
  double pow2[kSteps];
  uint32_t n, found;
};

// Elements (fp32 or bf16) of a row, f(value, index) for each; any alignment.
template <bool BF16>
struct Logits {
  const uint16_t* h;
  const float* f;
  int V;
  __device__ __forceinline__ Logits(const void* p, int64_t first, int v)
      : h(static_cast<const uint16_t*>(p) + first), f(static_cast<const float*>(p) + first), V(v) {}
  // Not a number: never drawn, as -infinity; +infinity: as the largest finite value; -0: as 0.
  static __device__ __forceinline__ float clean(float x) { return x == x ? fminf(x, FLT_MAX) + 0.0f : -INFINITY; }
  __device__ __forceinline__ float at(int i) const { return clean(BF16 ? bf16_to_f32(h[i]) : f[i]); }
  template <typename F>
  __device__ __forceinline__ void each(int first, int step, F&& fn) const {
    constexpr int PER = BF16 ? 8 : 4, SIZE = BF16 ? 2 : 4;
    const uintptr_t p = BF16 ? reinterpret_cast<uintptr_t>(h) : reinterpret_cast<uintptr_t>(f);
    const int head = min(V, (int)((16 - (p & 15)) & 15) / SIZE);  // elements before the first 16-byte boundary
    const int nv = (V - head) / PER, tail = head + nv * PER;
    if (first < head) fn(at(first), first);
    if (first < V - tail) fn(at(tail + first), tail + first);
    const u32x4* v = reinterpret_cast<const u32x4*>(p + (uintptr_t)head * SIZE);
    for (int i0 = first; i0 < nv; i0 += kLoads * step) {
      u32x4 r[kLoads];
#pragma unroll
      for (int k = 0; k < kLoads; ++k)
        if (i0 + k * step < nv) r[k] = v[i0 + k * step];
#pragma unroll
      for (int k = 0; k < kLoads; ++k) {
        if (i0 + k * step >= nv) break;
        const int e = head + (i0 + k * step) * PER;
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

// x.f(y) over all threads; every thread gets the result.
template <typename T, typename F>
__device__ __forceinline__ T block_reduce(T v, F&& f, u64 (*red)[4]) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v = f(v, (T)__shfl_xor(v, d));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6][0] = (u64)v;
  __syncthreads();
  T r = (T)red[0][0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) r = f(r, (T)red[w][0]);
  __syncthreads();
  return r;
}

__device__ __forceinline__ void clear_hist(Smem& s) {
  for (int i = threadIdx.x; i < kBins * kCols; i += kThreads) {
    s.hist_w[i] = 0;
    s.hist_c[i] = 0;
  }
  __syncthreads();
}
__device__ __forceinline__ void add_hist(Smem& s, int bin, u64 w) {
  const int at = bin * kCols + (threadIdx.x & (kCols - 1));
  atomicAdd(&s.hist_w[at], w);
  atomicAdd(&s.hist_c[at], 1u);
}
// Running sums over the bins, each with its own.
__device__ __forceinline__ void scan_hist(Smem& s) {
  __syncthreads();
  static_assert(kThreads == 8 * kBins && kCols == 4 * 8, "eight threads per bin, four copies each");
  const int b = threadIdx.x >> 3, c0 = 4 * (threadIdx.x & 7);
  u64 w = 0;
  uint32_t c = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    w += s.hist_w[b * kCols + c0 + k];
    c += s.hist_c[b * kCols + c0 + k];
  }
#pragma unroll
  for (int d = 1; d < 8; d *= 2) {
    w += __shfl_xor(w, d);
    c += __shfl_xor(c, d);
  }
  if (c0 == 0) {
    s.cum_w[b] = w;
    s.cum_c[b] = c;
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    const int l = threadIdx.x;
    const u64 w0 = s.cum_w[2 * l], w1 = s.cum_w[2 * l + 1];
    const uint32_t n0 = s.cum_c[2 * l], n1 = s.cum_c[2 * l + 1];
    u64 w2 = w0 + w1;
    uint32_t n2 = n0 + n1;
    for (int d = 1; d < 64; d *= 2) {
      const u64 a = __shfl_up(w2, d);
      const uint32_t e = __shfl_up(n2, d);
      if (l >= d) {
        w2 += a;
        n2 += e;
      }
    }
    s.cum_w[2 * l] = w2 - w1;
    s.cum_w[2 * l + 1] = w2;
    s.cum_c[2 * l] = n2 - n1;
    s.cum_c[2 * l + 1] = n2;
  }
  __syncthreads();
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
// The first of n places at which met(i) holds, n where it does nowhere. (met grows with i.)
template <typename F>
__device__ __forceinline__ int first_met(Smem& s, int n, F&& met) {
  if (threadIdx.x == 0) s.found = (uint32_t)n;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kThreads)
    if (met(i) && (i == 0 || !met(i - 1))) s.found = (uint32_t)i;
  __syncthreads();
  const int r = (int)s.found;
  __syncthreads();
  return r;
}

// The listed elements into descending order, their weights into running sums on top of `base`.
__device__ void sort_list(Smem& s, u64 base) {
  const int n = (int)s.n, tid = threadIdx.x;
  int len = 2;
  while (len < n) len *= 2;
  for (int i = n + tid; i < len; i += kThreads) {
    s.key[i] = 0;
    s.w[i] = 0;
  }
  __syncthreads();
  for (int size = 2; size <= len; size *= 2)
    for (int d = size / 2; d >= 1; d /= 2) {
      for (int t = tid; t < len / 2; t += kThreads) {
        const int i = 2 * t - (t & (d - 1)), j = i + d;
        const u64 a = s.key[i], b = s.key[j];
        if ((a < b) == ((i & size) == 0)) {
          s.key[i] = b;
          s.key[j] = a;
          const u64 w = s.w[i];
          s.w[i] = s.w[j];
          s.w[j] = w;
        }
      }
      __syncthreads();
    }
  constexpr int PER = kList / kThreads;
  u64 w[PER], sum = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int i = tid * PER + k;
    w[k] = i < n ? s.w[i] : 0;
    sum += w[k];
  }
  u64 incl = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const u64 a = __shfl_up(incl, d);
    if ((tid & 63) >= d) incl += a;
  }
  if ((tid & 63) == 63) s.red[tid >> 6][0] = incl;
  __syncthreads();
  u64 at = base + incl - sum;
  for (int k = 0; k < (tid >> 6); ++k) at += s.red[k][0];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    at += w[k];
    if (tid * PER + k < n) s.w[tid * PER + k] = at;
  }
  __syncthreads();
}

struct Found {
  u64 place, cum_w;
  uint32_t cum_c;
};

template <bool BF16>
struct Row {
  Smem& s;
  Logits<BF16> x;
  Weights weight;
  float max, scale;  // bins: (max - x) scale

  // (A NaN, from a scale of 0 or infinity, and the elements without weight: the last bin.)
  __device__ __forceinline__ int bin_of(float v) const { return (int)fminf((max - v) * scale, (float)(kBins - 1)); }

  // List the elements that take(value, index) wants and that have weight: at most kList are there.
  template <typename F>
  __device__ __forceinline__ void gather(F&& take) const {
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    x.each(threadIdx.x, kThreads, [&](float v, int i) {
      if (!take(v, i)) return;
      const u64 w = Weights::whole(weight.scaled(v));
      if (w == 0) return;
      const uint32_t at = atomicAdd(&s.n, 1u);
      if (at < kList) {
        s.key[at] = place_of(v, i);
        s.w[at] = w;
      }
    });
    __syncthreads();
    if (threadIdx.x == 0) s.n = min(s.n, (uint32_t)kList);
    __syncthreads();
  }

  // The element searched for, known to be in bin b of the first histogram, with the
  // running sums before that bin. Narrowed by histograms over the places until the
  // list holds what is left.
  __device__ Found locate(const Target& t, int b, uint32_t c0, u64 w0, uint32_t n) const {
    if (n <= kList) {
      gather([&](float v, int) { return bin_of(v) == b; });
    } else {
      u64 lo = ~0ull, hi = 0;
      x.each(threadIdx.x, kThreads, [&](float v, int i) {
        if (bin_of(v) != b || Weights::whole(weight.scaled(v)) == 0) return;
        const u64 p = place_of(v, i);
        lo = p < lo ? p : lo;
        hi = p > hi ? p : hi;
      });
      lo = block_reduce(lo, [](u64 a, u64 c) { return a < c ? a : c; }, s.red);
      hi = block_reduce(hi, [](u64 a, u64 c) { return a > c ? a : c; }, s.red);
      while (n > kList) {
        int sh = 0;
        while (((hi - lo) >> sh) >= kBins) ++sh;
        clear_hist(s);
        x.each(threadIdx.x, kThreads, [&](float v, int i) {
          const u64 p = place_of(v, i);
          if (p >= lo && p <= hi) add_hist(s, (int)((hi - p) >> sh), Weights::whole(weight.scaled(v)));
        });
        scan_hist(s);
        const int k = min(kBins - 1, first_met(s, kBins, [&](int i) { return t.met(c0 + s.cum_c[i], w0 + s.cum_w[i]); }));
        const uint32_t before_c = k ? s.cum_c[k - 1] : 0;
        n = s.cum_c[k] - before_c;
        c0 += before_c;
        w0 += k ? s.cum_w[k - 1] : 0;
        hi -= (u64)k << sh;
        const u64 span = ((u64)1 << sh) - 1;
        lo = hi - lo > span ? hi - span : lo;
        __syncthreads();
      }
      gather([&](float v, int i) {
        const u64 p = place_of(v, i);
        return p >= lo && p <= hi;
      });
    }
    sort_list(s, w0);
    const int m = (int)s.n;
    const int j = min(m - 1, first_met(s, m, [&](int i) { return t.met(c0 + i + 1, s.w[i]); }));
    const Found f = {s.key[j], s.w[j], c0 + (uint32_t)j + 1};
    __syncthreads();
    return f;
  }
};

template <bool BF16>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  Smem& s = *reinterpret_cast<Smem*>(smem);
  const int r = blockIdx.x, tid = threadIdx.x, V = a.vocab;
  const Logits<BF16> x(a.logits, (int64_t)r * a.stride, V);
  const float t = a.temperature ? a.temperature[r] : 1.f;
  const int k = a.top_k ? a.top_k[r] : 0;
  const float p = a.top_p ? a.top_p[r] : 1.f, mp = a.min_p ? a.min_p[r] : 0.f;
  float u = a.u[r];
  u = u > 0.f ? fminf(u, 1.f - 0x1p-24f) : 0.f;
  auto answer = [&](int token, double prob) {
    if (tid != 0) return;
    a.tokens[r] = token;
    if (a.probs) a.probs[r] = (float)prob;
  };
  if (tid < kSteps) s.pow2[tid] = exp2((double)tid / kSteps);
  // the largest element (of a row drawn from by its weights: its value) and the smallest finite one
  if (!(t > 0.f) || k == 1) {
    u64 best = 0;
    x.each(tid, kThreads, [&](float v, int i) {
      const u64 q = place_of(v, i);
      best = q > best ? q : best;
    });
    best = block_reduce(best, [](u64 c, u64 d) { return c > d ? c : d; }, s.red);
    const bool none = value_of(best) == -INFINITY;
    answer(none ? 0 : index_of(best), none ? 0.0 : 1.0);
    return;
  }
  float hi = -INFINITY, lo = INFINITY;
  x.each(tid, kThreads, [&](float v, int) {
    hi = fmaxf(hi, v);
    lo = v > -INFINITY ? fminf(lo, v) : lo;
  });
  hi = __uint_as_float(block_reduce(__float_as_uint(hi), [](uint32_t c, uint32_t d) {
    return __float_as_uint(fmaxf(__uint_as_float(c), __uint_as_float(d)));
  }, s.red));
  lo = __uint_as_float(block_reduce(__float_as_uint(lo), [](uint32_t c, uint32_t d) {
    return __float_as_uint(fminf(__uint_as_float(c), __uint_as_float(d)));
  }, s.red));
  if (hi == -INFINITY) {  // nothing may be drawn
    answer(0, 0.0);
    return;
  }
  // distances beyond which a weight rounds to none
  const float reach = fminf(hi - lo, (a.shift + 2) * 0.6931472f * t);
  const Weights wt = {(double)hi, 1.4426950408889634 * kSteps / (double)t, a.shift, s.pow2};
  const Row<BF16> row = {s, x, wt, hi, reach > 0.f ? kBins / reach : 0.f};
  // all weights, by distance; and those that min_p keeps
  const double least = mp > 0.f ? ldexp((double)mp, a.shift) : 0.0;
  clear_hist(s);
  u64 min_w = 0;
  uint32_t min_c = 0;
  x.each(tid, kThreads, [&](float v, int) {
    const double ws = wt.scaled(v);
    const u64 w = Weights::whole(ws);
    if (w == 0) return;
    add_hist(s, row.bin_of(v), w);
    if (ws >= least) {
      min_w += w;
      ++min_c;
    }
  });
  scan_hist(s);
  auto add = [](auto c, auto d) { return c + d; };
  const uint32_t all_c = s.cum_c[kBins - 1];
  const u64 all_w = s.cum_w[kBins - 1];
  min_w = block_reduce(min_w, add, s.red);
  min_c = block_reduce(min_c, add, s.red);
  const bool by_k = k > 0 && (uint32_t)k < all_c, by_p = p < 1.f;
  // kept: how many, and their weight
  uint32_t kept = all_c;
  u64 kept_w = all_w;
  auto find = [&](const Target& tg) {
    const int b = min(kBins - 1, first_met(s, kBins, [&](int i) { return tg.met(s.cum_c[i], s.cum_w[i]); }));
    return b;
  };
  auto locate = [&](const Target& tg) {
    const int b = find(tg);
    const uint32_t c0 = b ? s.cum_c[b - 1] : 0, n = s.cum_c[b] - c0;
    return row.locate(tg, b, c0, b ? s.cum_w[b - 1] : 0, n);
  };
  // Where all that can matter fits the list, it is read once more and sorted, and the
  // rest is looked up there.
  int last = kBins - 1;
  if (by_k) last = find({(uint32_t)k, 0.0, false});
  else if (by_p) last = find({0, (double)p * (double)all_w, false});
  if (!(by_k && by_p) && min_c > 0) last = min(last, find({min_c, 0.0, false}));
  if (s.cum_c[last] <= kList) {
    row.gather([&](float v, int) { return row.bin_of(v) <= last; });
    sort_list(s, 0);
    const int n = (int)s.n;
    kept = by_k ? min((uint32_t)k, (uint32_t)n) : (uint32_t)n;
    if (by_p) {
      const double want = (double)p * (double)(by_k ? s.w[kept - 1] : all_w);
      kept = min(kept, 1 + (uint32_t)first_met(s, n, [&](int i) { return (double)s.w[i] >= want; }));
    }
    kept = min(kept, max(min_c, 1u));
    kept_w = s.w[kept - 1];
    const double want = (double)u * (double)kept_w;
    const int j = first_met(s, (int)kept, [&](int i) { return (double)s.w[i] > want; });
    const u64 place = s.key[min(j, (int)kept - 1)];
    answer(index_of(place), wt.scaled(value_of(place)) / (double)kept_w);
    return;
  }
  // The histogram is needed for up to three searches, each of which may use it for itself.
  const u64 keep_w = tid < kBins ? s.cum_w[tid] : 0;
  const uint32_t keep_c = tid < kBins ? s.cum_c[tid] : 0;
  auto restore = [&] {
    __syncthreads();
    if (tid < kBins) {
      s.cum_w[tid] = keep_w;
      s.cum_c[tid] = keep_c;
    }
    __syncthreads();
  };
  if (by_k) {
    const Found f = locate({(uint32_t)k, 0.0, false});
    kept = f.cum_c;
    kept_w = f.cum_w;
    restore();
  }
  if (by_p) {
    const Found f = locate({0, (double)p * (double)kept_w, false});
    kept = f.cum_c;
    kept_w = f.cum_w;
    restore();
  }
  if (min_c < kept) {
    kept = min_c;
    kept_w = min_w;
  }
  if (min_c == 0) {  // min_p above 1: the first alone
    const Found f = locate({1, 0.0, false});
    answer(index_of(f.place), 1.0);
    return;
  }
  const Found f = locate({0, (double)u * (double)kept_w, true});
  answer(index_of(f.place), wt.scaled(value_of(f.place)) / (double)kept_w);
}

}  // namespace

void launch_sample(hipStream_t s, SampleArgs a) {
  if (a.rows <= 0) return;
  int bits = 0;
  while (((int64_t)1 << bits) < a.vocab) ++bits;
  a.shift = std::min(45, 62 - bits);
  auto go = [&](auto kernel, std::atomic<uint64_t>& raised) {
    raise_dynamic_lds(reinterpret_cast<const void*>(kernel), sizeof(Smem), raised);
    kernel<<<a.rows, kThreads, sizeof(Smem), s>>>(a);
  };
  static std::atomic<uint64_t> raised_f32{0}, raised_bf16{0};
  if (a.bf16) go(&sample_kernel<true>, raised_bf16);
  else go(&sample_kernel<false>, raised_f32);
}

}  // namespace hb
