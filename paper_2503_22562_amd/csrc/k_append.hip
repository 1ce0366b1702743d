// Append of a planned batch: new queries and keys rotated to their positions, new
// keys and values put into the pool's layouts.
//
// Pair j at position p turns by p f_j: (a, b) -> m (a cos - b sin, b cos + a sin). Bytes
// bound it: each row is read once and written once, 165 MB for four prompts of 777 to
// 1500 tokens beside 8 decodes with 70B heads, 23 us at a copy's rate, in 33 us. Decodes
// are a launch and one chain of loads: 3.3 us of kernel for one, 3.6 for 64.
//
// The work is cut by pool blocks, so that a block's 128-byte lines are written by one
// workgroup, together; and by eight heads, so that one token's heads share its cosines and a
// batch of a few decodes still has a workgroup for every few heads (4 or 16 heads, 128 or
// 512 threads: no faster at any of 1 decode, 64 decodes and the 70B case). Rows and q_out
// are read and written past the caches: nothing reads them again before megabytes of others
// have passed (70B case, before the values' two ways below: neither 45 us, reads 38.6, both
// 35.2; keys stored that way too 64: a line of the pool is put together in L2 from several
// stores).
#include <algorithm>
#include <type_traits>

#include "hb_device.h"
#include "hb_kernels.h"

namespace hb {
namespace {

constexpr int kThreads = 256;
constexpr int kHeads = 8;   // query or key heads of a rotating workgroup, value heads of a copying one
constexpr int kTokens = 16;  // tokens of a unit at most: a block's slots

// cos and sin of one turn's fraction t (|t| <= 1/8): Taylor series in x = 2 pi t, |x| <= pi/4,
// whose first terms left out are below 2^-29 of 1 and 2^-28 of sin x.
__device__ __forceinline__ void cos_sin_eighth(float t, float& c, float& s) {
  const float x = t * 6.283185307179586f, z = x * x;
  c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  s = x * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
}

// cos and sin of `turns` (fp64: positions reach 2^30): whole eighths of a turn are taken off in fp64.
__device__ __forceinline__ void cos_sin_turns(double turns, float& c, float& s) {
  const double q = rint(turns * 4.0);
  float c0, s0;
  cos_sin_eighth((float)fma(q, -0.25, turns), c0, s0);
  const int quarter = (int)(q - 4.0 * floor(q * 0.25));  // 0 .. 3
  const float a = (quarter & 1) ? s0 : c0, b = (quarter & 1) ? c0 : s0;
  c = (quarter == 1 || quarter == 2) ? -a : a;
  s = (quarter & 2) ? -b : b;
}

// A workgroup takes the tokens of one unit (they go to one pool block) and eight
// heads: of queries and keys, rotating them, or of values.
//
// Rotating: a thread moves two runs of eight dimensions of one head of one token,
// which hold eight whole pairs (half layout: 8c .. and R/2 + 8c ..; interleaved and
// unrotated dimensions: 16c .. and 16c + 8 ..): both are read before either is
// written, so q_out may be q. The cosines and sines are formed once per token and
// pair, one a thread, while the rows are on their way, and shared through LDS.
// Values of a whole block: a thread moves eight dimensions of one head for eight slots,
// transposed in registers. Of a part of one, whose other slots are not touched: of one
// token, value by value. (Units of both kinds through the transposition, with a test of
// each slot: 10.4 us of kernel, with this 6.2, for a chunk of 777 tokens behind 5234 and 45
// decodes with 16 and 4 heads; so much code is read for the few units that need it. With
// the workgroups of values before the others 5.6: theirs is the longer chain.)
template <int HD, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a, int v_parts) {
  __shared__ __attribute__((aligned(16))) float cs[2][kTokens][HD / 2];
  constexpr int CH = HD / 16;  // threads of one head of one token
  const AppendUnit u = const_load(reinterpret_cast<const AppendUnit*>(a.units) + blockIdx.x / a.parts);
  const int part = blockIdx.x % a.parts, tid = threadIdx.x;
  const size_t block = (size_t)u.block * a.nkv * 16 * HD;
  if (part < v_parts) {  // values
    constexpr int VC = HD / 8, STEP = kThreads / VC;
    const int c = tid % VC, g0 = part * kHeads, heads = min(kHeads, a.nkv - g0);
    if (u.n < 16) {
      constexpr int LOADS = 4;
      for (int e0 = tid / VC; e0 < u.n * heads; e0 += LOADS * STEP) {
        u32x4 r[LOADS];
        uint16_t* to[LOADS];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          const int e = e0 + i * STEP, h = e / u.n, t = e - h * u.n, slot = (u.pos0 & 15) + t;
          to[i] = a.v_pool + block + (size_t)(g0 + h) * 16 * HD + ((slot >> 3) * HD + 8 * c) * 8 + (slot & 7);
          if (e < u.n * heads) r[i] = ld16_stream(a.v + (int64_t)(u.tok0 + t) * a.v_stride + (g0 + h) * HD + 8 * c);
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          if (e0 + i * STEP >= u.n * heads) break;
#pragma unroll
          for (int d = 0; d < 8; ++d) to[i][8 * d] = (uint16_t)(r[i][d >> 1] >> (16 * (d & 1)));
        }
      }
      return;
    }
    const int half = (tid / VC) & 1;
    for (int h = tid / (2 * VC); h < heads; h += STEP / 2) {
      const uint16_t* row = a.v + (int64_t)(u.tok0 + 8 * half) * a.v_stride + (g0 + h) * HD + 8 * c;
      u32x4 r[8];
#pragma unroll
      for (int t = 0; t < 8; ++t) r[t] = ld16_stream(row + t * a.v_stride);
      uint16_t* vb = a.v_pool + block + (size_t)(g0 + h) * 16 * HD + (half * HD + 8 * c) * 8;
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        u32x4 o;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t x = r[2 * w][d >> 1], y = r[2 * w + 1][d >> 1];
          o[w] = (d & 1) ? (x >> 16) | (y & 0xFFFF0000u) : (x & 0xFFFFu) | (y << 16);
        }
        st16(vb + 8 * d, o);
      }
    }
    return;
  }
  constexpr int ITEMS = kTokens * kHeads * CH / kThreads;  // of a full unit
  const int rot = a.rotary;
  u32x4 x0[ITEMS], x1[ITEMS];
  const int c = tid % CH;
  const bool rotated = 16 * c < rot;
  const int d0 = !INTERLEAVED && rotated ? 8 * c : 16 * c, d1 = !INTERLEAVED && rotated ? rot / 2 + 8 * c : 16 * c + 8;
  // item i of a thread: head hi, token t (heads of one token first)
  auto place = [&](int i, int& h, int& t) {
    const int e = (tid + i * kThreads) / CH;
    h = (part - v_parts) * kHeads + e % kHeads;
    t = e / kHeads;
    return t < u.n && h < a.nq + a.nkv;
  };
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    int h, t;
    if (!place(i, h, t)) continue;
    const uint16_t* row = h < a.nq ? a.q + (int64_t)(u.tok0 + t) * a.q_stride + h * HD
                                   : a.k + (int64_t)(u.tok0 + t) * a.k_stride + (h - a.nq) * HD;
    x0[i] = ld16_stream(row + d0);
    x1[i] = ld16_stream(row + d1);
  }
  const int pairs = rot / 2;
  for (int i = tid; i < u.n * pairs; i += kThreads) {
    const int t = i / pairs, j = i - t * pairs;
    float cv, sv;
    cos_sin_turns((double)(u.pos0 + t) * a.turns[j], cv, sv);
    cs[0][t][j] = cv * a.magnitude;
    cs[1][t][j] = sv * a.magnitude;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    int h, t;
    if (!place(i, h, t)) continue;
    u32x4 y0 = x0[i], y1 = x1[i];
    if (rotated) {
      const f32x4* pc = reinterpret_cast<const f32x4*>(&cs[0][t][8 * c]);
      const f32x4* ps = reinterpret_cast<const f32x4*>(&cs[1][t][8 * c]);
      const f32x4 cv[2] = {pc[0], pc[1]}, sv[2] = {ps[0], ps[1]};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if (INTERLEAVED) {  // pairs are the words: w of the first run is pair w, of the second 4 + w
          const float p0 = bf16_lo(x0[i][w]), q0 = bf16_hi(x0[i][w]), p1 = bf16_lo(x1[i][w]), q1 = bf16_hi(x1[i][w]);
          y0[w] = pack_bf16x2(p0 * cv[0][w] - q0 * sv[0][w], q0 * cv[0][w] + p0 * sv[0][w]);
          y1[w] = pack_bf16x2(p1 * cv[1][w] - q1 * sv[1][w], q1 * cv[1][w] + p1 * sv[1][w]);
        } else {
          const float c0 = cv[w >> 1][2 * (w & 1)], c1 = cv[w >> 1][2 * (w & 1) + 1];
          const float s0 = sv[w >> 1][2 * (w & 1)], s1 = sv[w >> 1][2 * (w & 1) + 1];
          const float p0 = bf16_lo(x0[i][w]), p1 = bf16_hi(x0[i][w]), q0 = bf16_lo(x1[i][w]), q1 = bf16_hi(x1[i][w]);
          y0[w] = pack_bf16x2(p0 * c0 - q0 * s0, p1 * c1 - q1 * s1);
          y1[w] = pack_bf16x2(q0 * c0 + p0 * s0, q1 * c1 + p1 * s1);
        }
      }
    }
    if (h < a.nq) {
      uint16_t* row = a.q_out + (int64_t)(u.tok0 + t) * a.q_out_stride + h * HD;
      st16_stream(row + d0, y0);
      st16_stream(row + d1, y1);
    } else {
      uint16_t* kb = a.k_pool + block + (size_t)(h - a.nq) * 16 * HD;
      const int slot = (u.pos0 + t) & 15;
      st16(kb + k_block_offset(slot, d0, HD), y0);
      st16(kb + k_block_offset(slot, d1, HD), y1);
    }
  }
}

}  // namespace

void launch_append(hipStream_t s, AppendArgs a) {
  if (a.n_units <= 0) return;
  const int v_parts = (a.nkv + kHeads - 1) / kHeads;
  a.parts = v_parts + (a.nq + a.nkv + kHeads - 1) / kHeads;
  // a grid holds fewer than 2^32 threads
  const int most = (1 << 23) / a.parts;
  for (int left = a.n_units; left > 0; left -= most, a.units += 4 * (size_t)most) {
    const int groups = std::min(left, most) * a.parts;
    auto go = [&](auto hd, auto inter) {
      append_kernel<decltype(hd)::value, decltype(inter)::value><<<groups, kThreads, 0, s>>>(a, v_parts);
    };
    auto layout = [&](auto hd) { a.interleaved ? go(hd, std::true_type{}) : go(hd, std::false_type{}); };
    if (a.hd == 128) layout(std::integral_constant<int, 128>{});
    else layout(std::integral_constant<int, 64>{});
  }
}

}  // namespace hb
