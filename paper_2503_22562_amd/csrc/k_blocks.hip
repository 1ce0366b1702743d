// Copies of whole pool blocks (forked sequences' last blocks, compaction).
#include <algorithm>

#include "hb_device.h"
#include "hb_kernels.h"

namespace hb {
namespace {

// pool[dst] = pool[src], a block's n_kv heads at a time: one contiguous run of
// 32 n_kv hd bytes in the K pool and one in the V pool. A workgroup copies two
// 16-byte vectors per thread, 8 KB, of one run; its neighbours take the rest of
// the run, the block's other runs (V, then the other layers), then the next
// pair. Bound by HBM: every byte is read once and written once. Bytes moved per
// second (read + write; torch's copy of 4 GiB: 5.4 TB/s):
//   9000 pairs of 2 x 32 KB         6.0 TB/s, 195 us
//   48 pairs in 32 layers           6.6 TB/s, 30.5 us
//   4000 pairs of 2 x 4 KB          6.5 TB/s, 10.1 us
// Eight vectors per thread leave too few workgroups in flight (4.0, 3.6 and 2.7
// TB/s); four are as fast on large lists and slower on short ones (300 pairs 5.7
// against 4.8 us). Stores are non-temporal, as they displace the next pairs'
// lines otherwise (5.5 -> 6.0 TB/s); non-temporal loads cost up to a third on
// lists that fit the caches.
constexpr int kCopyThreads = 256, kCopyVecs = 2;

template <int N>
struct InlinePairs {
  int32_t s[N], d[N];
  __device__ __forceinline__ int src(int i) const { return s[i]; }
  __device__ __forceinline__ int dst(int i) const { return d[i]; }
};
struct ListedPairs {
  const int32_t *s, *d;
  __device__ __forceinline__ int src(int i) const { return const_load(s + i); }
  __device__ __forceinline__ int dst(int i) const { return const_load(d + i); }
};

struct OnePool {
  void *k[1], *v[1];
};
static_assert(sizeof(CopyPools) + sizeof(InlinePairs<kCopyInlinePairs>) + 12 <= 4096, "launch arguments");
static_assert(sizeof(OnePool) + sizeof(InlinePairs<kCopyInlineOne>) + 12 <= 4096, "launch arguments");

template <typename Pools, typename Pairs>
__global__ __launch_bounds__(kCopyThreads) void copy_blocks_kernel(Pools pools, int n_pools, Pairs pairs, int vecs,
                                                                   int parts) {
  const int run = blockIdx.x / parts, part = blockIdx.x - run * parts;
  const int pair = run / (2 * n_pools), side = run - pair * 2 * n_pools;  // K and V of layer 0, of layer 1, ...
  u32x4* pool = static_cast<u32x4*>((side & 1) ? pools.v[side >> 1] : pools.k[side >> 1]);
  const u32x4* s = pool + (size_t)pairs.src(pair) * vecs;
  u32x4* d = pool + (size_t)pairs.dst(pair) * vecs;
  const int i0 = part * kCopyThreads * kCopyVecs + threadIdx.x;
  u32x4 v[kCopyVecs];
#pragma unroll
  for (int k = 0; k < kCopyVecs; ++k)
    if (i0 + k * kCopyThreads < vecs) v[k] = s[i0 + k * kCopyThreads];
#pragma unroll
  for (int k = 0; k < kCopyVecs; ++k)
    if (i0 + k * kCopyThreads < vecs) __builtin_nontemporal_store(v[k], d + i0 + k * kCopyThreads);
}

// Launches of at most `pairs` pairs and 2^20 workgroups (a grid holds fewer than 2^32 threads).
template <typename F>
void for_pairs(int n, int pairs, int n_pools, int nkv, int hd, F&& launch) {
  const int vecs = nkv * hd * 2, parts = (vecs + kCopyThreads * kCopyVecs - 1) / (kCopyThreads * kCopyVecs);
  const int per_pair = 2 * n_pools * parts, most = std::max(1, std::min(pairs, (1 << 20) / per_pair));
  for (int i = 0; i < n; i += most) {
    const int m = std::min(most, n - i);
    launch(i, m, m * per_pair, vecs, parts);
  }
}

}  // namespace

void launch_copy_blocks(hipStream_t s, const CopyPools& pools, int n_pools, const int32_t* src, const int32_t* dst,
                        int n, int nkv, int hd) {
  for_pairs(n, n, n_pools, nkv, hd, [&](int i, int, int groups, int vecs, int parts) {
    copy_blocks_kernel<<<groups, kCopyThreads, 0, s>>>(pools, n_pools, ListedPairs{src + i, dst + i}, vecs, parts);
  });
}

void launch_copy_blocks_inline(hipStream_t s, const CopyPools& pools, int n_pools, const int32_t* src,
                               const int32_t* dst, int n, int nkv, int hd) {
  auto go = [&](const auto& to, auto pairs, int most) {
    for_pairs(n, most, n_pools, nkv, hd, [&](int i, int m, int groups, int vecs, int parts) {
      std::copy(src + i, src + i + m, pairs.s);
      std::copy(dst + i, dst + i + m, pairs.d);
      copy_blocks_kernel<<<groups, kCopyThreads, 0, s>>>(to, n_pools, pairs, vecs, parts);
    });
  };
  if (n_pools == 1) go(OnePool{{pools.k[0]}, {pools.v[0]}}, InlinePairs<kCopyInlineOne>{}, kCopyInlineOne);
  else go(pools, InlinePairs<kCopyInlinePairs>{}, kCopyInlinePairs);
}

}  // namespace hb
