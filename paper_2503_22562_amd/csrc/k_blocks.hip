// Copies of whole pool blocks (forked sequences' last blocks, compaction).
#include <algorithm>

#include "hb_device.h"
#include "hb_kernels.h"

namespace hb {
namespace {

// pool[dst] = pool[src], a block's n_kv heads at a time: one contiguous run of
// 32 n_kv hd bytes in the K pool and one in the V pool. A workgroup copies up to
// kCopyVecs 16-byte vectors per thread of one run, all of its loads in flight
// before its first store. Bound by HBM: every byte is read once and written once.
constexpr int kCopyThreads = 256, kCopyVecs = 8;

struct InlinePairs {
  int32_t s[kCopyInlinePairs], d[kCopyInlinePairs];
  __device__ __forceinline__ int src(int i) const { return s[i]; }
  __device__ __forceinline__ int dst(int i) const { return d[i]; }
};
struct ListedPairs {
  const int32_t *s, *d;
  __device__ __forceinline__ int src(int i) const { return const_load(s + i); }
  __device__ __forceinline__ int dst(int i) const { return const_load(d + i); }
};

template <typename Pairs>
__global__ __launch_bounds__(kCopyThreads) void copy_blocks_kernel(CopyPools pools, Pairs pairs, int vecs, int parts) {
  const int pair = blockIdx.x / parts, part = blockIdx.x - pair * parts;
  const int layer = blockIdx.y >> 1;
  u32x4* pool = static_cast<u32x4*>((blockIdx.y & 1) ? pools.v[layer] : pools.k[layer]);
  const u32x4* s = pool + (size_t)pairs.src(pair) * vecs;
  u32x4* d = pool + (size_t)pairs.dst(pair) * vecs;
  const int i0 = part * kCopyThreads * kCopyVecs + threadIdx.x;
  u32x4 v[kCopyVecs];
#pragma unroll
  for (int k = 0; k < kCopyVecs; ++k)
    if (i0 + k * kCopyThreads < vecs) v[k] = s[i0 + k * kCopyThreads];
#pragma unroll
  for (int k = 0; k < kCopyVecs; ++k)
    if (i0 + k * kCopyThreads < vecs) d[i0 + k * kCopyThreads] = v[k];
}

// Launches of at most 2^20 workgroups along the pairs (a grid holds fewer than 2^32 threads).
template <typename F>
void for_pairs(int n, int nkv, int hd, F&& launch) {
  const int vecs = nkv * hd * 2, parts = (vecs + kCopyThreads * kCopyVecs - 1) / (kCopyThreads * kCopyVecs);
  const int most = std::max(1, (1 << 20) / parts);
  for (int i = 0; i < n; i += most) launch(i, std::min(most, n - i) * parts, vecs, parts);
}

}  // namespace

void launch_copy_blocks(hipStream_t s, const CopyPools& pools, int n_pools, const int32_t* src, const int32_t* dst,
                        int n, int nkv, int hd) {
  for_pairs(n, nkv, hd, [&](int i, int groups, int vecs, int parts) {
    copy_blocks_kernel<<<dim3(groups, 2 * n_pools), kCopyThreads, 0, s>>>(pools, ListedPairs{src + i, dst + i}, vecs,
                                                                         parts);
  });
}

void launch_copy_blocks_inline(hipStream_t s, const CopyPools& pools, int n_pools, const int32_t* src,
                               const int32_t* dst, int n, int nkv, int hd) {
  InlinePairs p{};
  std::copy(src, src + n, p.s);
  std::copy(dst, dst + n, p.d);
  for_pairs(n, nkv, hd, [&](int i, int groups, int vecs, int parts) {
    (void)i;  // n <= kCopyInlinePairs: one launch
    copy_blocks_kernel<<<dim3(groups, 2 * n_pools), kCopyThreads, 0, s>>>(pools, p, vecs, parts);
  });
}

}  // namespace hb
