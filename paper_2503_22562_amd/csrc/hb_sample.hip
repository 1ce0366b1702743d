// Sampling handles: the argument checks around k_sample.hip.
#include <algorithm>
#include <new>

#include <hip/hip_runtime.h>

#include "hb.h"
#include "hb_kernels.h"
#include "hb_plan.h"
#include "hb_runtime.h"

using namespace hb;

struct hb_sampler {
  int max_rows = 0, vocab = 0, device = 0;
  hipStream_t stream = nullptr;
  SampleExtent* extents = nullptr;
  SampleState* state = nullptr;
};

namespace {
void free_sampler(hb_sampler* s) {
  if (!s) return;
  const DeviceGuard on(s->device);
  (void)hipStreamSynchronize(s->stream);
  for (void* p : {(void*)s->extents, (void*)s->state})
    if (p) (void)hipFree(p);
  delete s;
}
}  // namespace

extern "C" {

hb_status hb_create_sampler(int32_t max_rows, int32_t vocab, void* hip_stream, hb_sampler** out) {
  if (!out) return fail(HB_ERR_INVALID, "null output handle");
  *out = nullptr;
  if (max_rows < 1 || vocab < 1) return fail(HB_ERR_INVALID, "max_rows %d or vocab %d below 1", max_rows, vocab);
  if (max_rows > 1 << 20 || vocab > 1 << 20)
    return fail(HB_ERR_UNSUPPORTED, "max_rows %d or vocab %d above 2^20", max_rows, vocab);
  return guarded([&]() -> hb_status {
    int device = 0;
    if (hipGetDevice(&device) != hipSuccess) return fail(HB_ERR_HIP, "device query failed");
    hb_sampler* s = new hb_sampler();
    s->max_rows = max_rows;
    s->vocab = vocab;
    s->device = device;
    s->stream = static_cast<hipStream_t>(hip_stream);
    const size_t rows = std::min(max_rows, kSampleRows);
    if (hipMalloc((void**)&s->extents, rows * kSampleSlices * sizeof(SampleExtent)) != hipSuccess ||
        hipMalloc((void**)&s->state, rows * sizeof(SampleState)) != hipSuccess) {
      (void)hipGetLastError();
      free_sampler(s);
      return fail(HB_ERR_OOM, "sampling workspace of %d rows", (int)rows);
    }
    *out = s;
    return HB_OK;
  });
}

void hb_destroy_sampler(hb_sampler* s) { free_sampler(s); }

hb_status hb_sample(hb_sampler* s, const hb_sample_desc* d) {
  if (!s) return fail(HB_ERR_INVALID, "null sampler handle");
  const hb_status st = check_sample(s->max_rows, s->vocab, d);
  if (st != HB_OK || d->n_rows == 0) return st;
  const DeviceGuard on(s->device);
  SampleArgs a{};
  a.logits = d->logits;
  a.stride = d->row_stride;
  a.bf16 = d->logits_dtype == HB_OUT_BF16;
  a.rows = d->n_rows;
  a.vocab = s->vocab;
  a.temperature = d->temperature;
  a.top_k = d->top_k;
  a.top_p = d->top_p;
  a.min_p = d->min_p;
  a.u = d->u;
  a.tokens = d->tokens;
  a.probs = d->probs;
  a.extents = s->extents;
  a.state = s->state;
  launch_sample(s->stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(HB_ERR_HIP, "sampling launch: %s", hipGetErrorString(e));
  return HB_OK;
}

}  // extern "C"
