// Attention over the paged cache on its own: a plan (the work list of one
// batch, on the device) that every layer of an iteration runs against its own
// pool, with the kernels of the layer.
#include <algorithm>
#include <cstdlib>
#include <cstring>
#include <new>
#include <utility>

#include <hip/hip_runtime.h>

#include "hb.h"
#include "hb_kernels.h"
#include "hb_plan.h"
#include "hb_runtime.h"

using namespace hb;

namespace {
// Pinned copies of a plan's metadata: as many plans may be enqueued before the
// host waits for the first one's upload.
constexpr int kPlanStages = 4;
struct PlanStage {
  int32_t* host = nullptr;
  size_t cap = 0;  // int32
  hipEvent_t copied = nullptr;
  bool pending = false;
};
}  // namespace

struct hb_attention {
  Dims d;
  int num_blocks = 0, device = 0, cu_count = 0;
  hipStream_t stream = nullptr;
  PlanOptions opt;
  Plan plan, next;  // the current plan, and the one being built
  RecordPlan records, next_records;
  bool planned = false;
  // appends: the rotation, and whether and where the plan's units stand
  bool rope_set = false, can_append = false;
  int rotary = 0, rope_layout = HB_ROPE_HALF, n_append = 0, off_append = 0;
  float magnitude = 1.f;
  double turns[64] = {};
  SlotMarks marks;
  int32_t* meta = nullptr;  // the current plan's metadata; in stream order with the runs that read it
  size_t meta_cap = 0;      // int32
  float *part_o = nullptr, *part_ml = nullptr;
  int part_cap = 0;
  PlanStage stage[kPlanStages];
  int stage_next = 0;
};

namespace {

void free_attention(hb_attention* a) {
  if (!a) return;
  const DeviceGuard on(a->device);
  (void)hipStreamSynchronize(a->stream);
  for (void* p : {(void*)a->meta, (void*)a->part_o, (void*)a->part_ml})
    if (p) (void)hipFree(p);
  for (PlanStage& s : a->stage) {
    if (s.host) (void)hipHostFree(s.host);
    if (s.copied) (void)hipEventDestroy(s.copied);
  }
  delete a;
}

// Replace a device array by one of `bytes` (its contents are not kept) once no
// enqueued work uses it. Where the new one cannot be had the old one stays.
bool regrow(hb_attention* a, void** p, size_t bytes) {
  void* q = nullptr;
  if (hipMalloc(&q, bytes) != hipSuccess) {
    (void)hipGetLastError();
    return false;
  }
  if (*p) {
    (void)hipStreamSynchronize(a->stream);
    (void)hipFree(*p);
  }
  *p = q;
  return true;
}

// The plan of a checked batch of T tokens.
hb_status plan_checked(hb_attention* a, int n, const hb_request* requests, int64_t T, const PlanOptions& opt) {
  const bool can_append = a->rope_set && check_slots(a->num_blocks, requests, n, T, &a->marks) == HB_OK;
  const DeviceGuard on(a->device);
  const hb_status st = refuse_capture(a->stream);
  if (st != HB_OK) return st;
  a->planned = false;  // until the new one stands
  const hb_batch_desc desc{n, requests, nullptr, nullptr, HB_OUT_BF16};
  build_plan(a->d, &desc, a->cu_count, &a->next, opt);
  if (a->next.too_many_slots) return fail(HB_ERR_UNSUPPORTED, "more than 2^30 partial results of shared prefixes");
  build_records(a->next, &a->next_records);
  if (can_append) a->n_append = build_append(requests, n, &a->next_records.meta, &a->off_append);
  a->can_append = can_append;
  const size_t words = a->next_records.meta.size();
  PlanStage& s = a->stage[a->stage_next];
  if (s.pending) {
    if (hipEventSynchronize(s.copied) != hipSuccess) return fail(HB_ERR_HIP, "plan staging wait failed");
    s.pending = false;
  }
  // room for longer tables than this batch's: contexts grow from one plan to the next
  const size_t cap = std::max<size_t>((words + words / 4 + 3) & ~(size_t)3, 1 << 14);
  if (words > s.cap) {
    if (s.host) (void)hipHostFree(s.host);
    s.host = nullptr;
    s.cap = 0;
    if (hipHostMalloc((void**)&s.host, cap * sizeof(int32_t), hipHostMallocDefault) != hipSuccess) {
      (void)hipGetLastError();
      return fail(HB_ERR_OOM, "pinned staging of %zu B", cap * 4);
    }
    s.cap = cap;
  }
  if (a->next.n_slots > a->part_cap) {
    const int slots = std::max(a->next.n_slots, 2 * a->part_cap);
    a->part_cap = 0;
    if (!regrow(a, (void**)&a->part_o, (size_t)slots * a->d.hd * sizeof(float)) ||
        !regrow(a, (void**)&a->part_ml, (size_t)slots * 2 * sizeof(float)))
      return fail(HB_ERR_OOM, "attention split buffers for %d column slots", slots);
    a->part_cap = slots;
  }
  if (words > a->meta_cap) {
    if (!regrow(a, (void**)&a->meta, cap * sizeof(int32_t))) return fail(HB_ERR_OOM, "plan of %zu B", cap * 4);
    a->meta_cap = cap;
  }
  if (words > 0) {
    std::memcpy(s.host, a->next_records.meta.data(), words * sizeof(int32_t));
    launch_copy_words(a->stream, s.host, a->meta, words);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || hipEventRecord(s.copied, a->stream) != hipSuccess)
      return fail(HB_ERR_HIP, "plan upload: %s", hipGetErrorString(e));
    s.pending = true;
    a->stage_next = (a->stage_next + 1) % kPlanStages;
  }
  std::swap(a->plan, a->next);
  std::swap(a->records, a->next_records);
  a->planned = true;
  return HB_OK;
}

hb_status plan_attention(hb_attention* a, int n, const hb_request* requests, int window, int sinks) {
  hb_status st = check_window_args(window, sinks);
  if (st != HB_OK) return st;
  PlanOptions opt = a->opt;
  opt.window.window = window;
  opt.window.sinks = window > 0 ? sinks : 0;
  int64_t T = 0;
  st = check_requests(a->d, a->num_blocks, requests, n, opt.window, &T);
  return st != HB_OK ? st : plan_checked(a, n, requests, T, opt);
}

hb_status plan_shared(hb_attention* a, int n, const hb_request* requests, int n_groups, const hb_prefix_group* groups) {
  int64_t T = 0;
  const hb_status st = check_shared(a->d, a->num_blocks, requests, n, groups, n_groups, &T);
  if (st != HB_OK) return st;
  PlanOptions opt = a->opt;
  opt.groups = groups;
  opt.n_groups = n_groups;
  return plan_checked(a, n, requests, T, opt);
}

hb_status run_append(hb_attention* a, const hb_kv_pool* pool, const Rows& q, const Rows& k, const Rows& v,
                     const Rows& out) {
  hb_status st = check_append(a->d, a->num_blocks, a->plan.T, pool, q, k, v, out);
  if (st != HB_OK) return st;
  const DeviceGuard on(a->device);
  st = refuse_capture(a->stream);
  if (st != HB_OK) return st;
  AppendArgs g{};
  g.units = a->meta + a->off_append;
  g.n_units = a->n_append;
  g.q = (const uint16_t*)q.at; g.q_stride = q.stride;
  g.k = (const uint16_t*)k.at; g.k_stride = k.stride;
  g.v = (const uint16_t*)v.at; g.v_stride = v.stride;
  g.q_out = (uint16_t*)out.at; g.q_out_stride = out.stride;
  g.k_pool = (uint16_t*)pool->k_pool;
  g.v_pool = (uint16_t*)pool->v_pool;
  g.nq = a->d.nq; g.nkv = a->d.nkv; g.hd = a->d.hd;
  g.rotary = a->rotary;
  g.interleaved = a->rope_layout == HB_ROPE_INTERLEAVED;
  g.magnitude = a->magnitude;
  std::copy(a->turns, a->turns + 64, g.turns);
  launch_append(a->stream, g);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(HB_ERR_HIP, "append launch: %s", hipGetErrorString(e));
  return HB_OK;
}

}  // namespace

extern "C" {

hb_status hb_create_attention(const hb_layer_config* cfg, int32_t num_blocks, void* hip_stream, hb_attention** out) {
  if (!out) return fail(HB_ERR_INVALID, "null output handle");
  *out = nullptr;
  Dims d;
  hb_status st = check_config(cfg, &d);
  if (st != HB_OK) return st;
  if (num_blocks <= 0) return fail(HB_ERR_INVALID, "num_blocks %d: no pool block", num_blocks);
  return guarded([&]() -> hb_status {
    hb_attention* a = new hb_attention();
    auto bail = [&](hb_status s) { free_attention(a); return s; };
    a->d = d;
    a->num_blocks = num_blocks;
    a->opt.fit_round = true;
    a->stream = static_cast<hipStream_t>(hip_stream);
    if (hipGetDevice(&a->device) != hipSuccess ||
        hipDeviceGetAttribute(&a->cu_count, hipDeviceAttributeMultiprocessorCount, a->device) != hipSuccess)
      return bail(fail(HB_ERR_HIP, "device query failed"));
    if (const char* e = std::getenv("HB_ATTN_SPLIT_TILE")) a->opt.split_tile = std::atoi(e);
    if (const char* e = std::getenv("HB_ATTN_SPLIT_ITEM")) a->opt.split_item = std::atoi(e);
    if (const char* e = std::getenv("HB_ATTN_UNIT_BLOCK")) a->opt.unit_block = std::atoi(e);
    if (const char* e = std::getenv("HB_ATTN_SHARE_ALL")) a->opt.share_all = std::atoi(e) != 0;
    for (PlanStage& s : a->stage)
      if (hipEventCreateWithFlags(&s.copied, hipEventDisableTiming) != hipSuccess)
        return bail(fail(HB_ERR_HIP, "hipEventCreate failed"));
    *out = a;
    return HB_OK;
  });
}

void hb_destroy_attention(hb_attention* a) { free_attention(a); }

hb_status hb_plan_attention(hb_attention* a, int32_t n_requests, const hb_request* requests, int32_t window,
                            int32_t sinks) {
  if (!a) return fail(HB_ERR_INVALID, "null attention handle");
  return guarded([&] { return plan_attention(a, n_requests, requests, window, sinks); });
}

hb_status hb_plan_shared_attention(hb_attention* a, int32_t n_requests, const hb_request* requests, int32_t n_groups,
                                   const hb_prefix_group* groups) {
  if (!a) return fail(HB_ERR_INVALID, "null attention handle");
  return guarded([&] { return plan_shared(a, n_requests, requests, n_groups, groups); });
}

hb_status hb_set_attention_rope(hb_attention* a, int32_t rotary_dim, int32_t layout, const double* inv_freq,
                                double magnitude) {
  if (!a) return fail(HB_ERR_INVALID, "null attention handle");
  const hb_status st = check_rope(a->d.hd, rotary_dim, layout, inv_freq, magnitude);
  if (st != HB_OK) return st;
  for (int j = 0; j < rotary_dim / 2; ++j) a->turns[j] = inv_freq[j] / 6.283185307179586;
  a->rotary = rotary_dim;
  a->rope_layout = layout;
  a->magnitude = (float)magnitude;
  a->rope_set = true;
  return HB_OK;
}

hb_status hb_run_append(hb_attention* a, const hb_kv_pool* pool, const void* q, int64_t q_stride, const void* k,
                        int64_t k_stride, const void* v, int64_t v_stride, void* q_out, int64_t q_out_stride) {
  if (!a) return fail(HB_ERR_INVALID, "null attention handle");
  if (!a->planned) return fail(HB_ERR_INVALID, "hb_run_append before a successful plan");
  if (!a->can_append)
    return fail(HB_ERR_INVALID, "hb_run_append: the plan was made before the handle's first hb_set_attention_rope, "
                                "or two of its requests write one slot");
  if (a->plan.T == 0) return HB_OK;
  const int64_t row = (int64_t)a->d.nq * a->d.hd, kv_row = (int64_t)a->d.nkv * a->d.hd;
  return run_append(a, pool, {(uintptr_t)q, q_stride, row}, {(uintptr_t)k, k_stride, kv_row},
                    {(uintptr_t)v, v_stride, kv_row}, {(uintptr_t)q_out, q_out_stride, row});
}

hb_status hb_run_attention(hb_attention* a, const hb_kv_pool* pool, const void* q, int64_t q_stride, void* out,
                           int64_t out_stride) {
  if (!a) return fail(HB_ERR_INVALID, "null attention handle");
  if (!a->planned) return fail(HB_ERR_INVALID, "hb_run_attention before a successful hb_plan_attention");
  const Plan& p = a->plan;
  if (p.T == 0) return HB_OK;
  if (!pool || !pool->k_pool || !pool->v_pool || !q || !out) return fail(HB_ERR_INVALID, "null pool, q or out");
  if (pool->num_blocks < a->num_blocks)
    return fail(HB_ERR_INVALID, "pool of %d blocks, the plan's tables are over %d", pool->num_blocks, a->num_blocks);
  const int64_t row = (int64_t)a->d.nq * a->d.hd;
  for (int64_t s : {q_stride, out_stride})
    if (s < row || s % 8 || s > (int64_t)1 << 40)
      return fail(HB_ERR_INVALID, "row stride %lld: a multiple of 8 from %lld on", (long long)s, (long long)row);
  for (const void* x : {(const void*)pool->k_pool, (const void*)pool->v_pool, q, (const void*)out})
    if ((uintptr_t)x % 16) return fail(HB_ERR_INVALID, "pools, q and out must be 16-byte aligned");
  const uintptr_t q0 = (uintptr_t)q, q1 = q0 + ((uintptr_t)(p.T - 1) * q_stride + row) * 2;
  const uintptr_t o0 = (uintptr_t)out, o1 = o0 + ((uintptr_t)(p.T - 1) * out_stride + row) * 2;
  if (q0 < o1 && o0 < q1) return fail(HB_ERR_INVALID, "out overlaps q");
  const uintptr_t pool_bytes = (uintptr_t)pool->num_blocks * a->d.nkv * 16 * a->d.hd * 2;
  for (const void* x : {(const void*)pool->k_pool, (const void*)pool->v_pool})
    if ((uintptr_t)x < o1 && o0 < (uintptr_t)x + pool_bytes) return fail(HB_ERR_INVALID, "out overlaps a pool");
  const DeviceGuard on(a->device);
  const hb_status st = refuse_capture(a->stream);
  if (st != HB_OK) return st;
  AttnArgs at = attention_args(a->d, p, a->meta, pool->k_pool, pool->v_pool, a->part_o, a->part_ml, &a->records);
  at.q = static_cast<const uint16_t*>(q);
  at.o = static_cast<uint16_t*>(out);
  at.q_stride = q_stride;
  at.o_stride = out_stride;
  launch_attention(a->stream, at);
  launch_attn_merge(a->stream, at);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(HB_ERR_HIP, "attention launch: %s", hipGetErrorString(e));
  return HB_OK;
}

}  // extern "C"
