// Runtime entry points shared by the layer runtime and the whole-model
// driver (internal: not part of the C ABI).
#pragma once

#include <hip/hip_runtime.h>

#include <new>

#include "hb.h"
#include "hb_plan.h"

namespace hb {

// HB_ERR_HIP when the stream is under graph capture. Calls whose kernels read a
// slot of the metadata ring (or the model's row staging), and the KV append, are
// refused there before anything is enqueued; the capture itself stays valid.
hb_status refuse_capture(hipStream_t s);

// One iteration of a stack of layers that share configuration, pool size
// and stream, over one batch: the batch is validated, planned and its
// metadata uploaded once, and every layer's kernels read that upload.
// Layer l reads x_in[l] and writes x_out[l] (bf16 or fp32 per desc).
hb_status run_layer_stack(hb_layer* const* layers, int n, const hb_batch_desc* desc, const void* const* x_in,
                          void* const* x_out);

// The checks of that call alone: the batch against every layer's window.
hb_status check_layer_stack(hb_layer* const* layers, int n, const hb_batch_desc* desc);

// Copy blocks src[i] -> dst[i] in the pools of a stack of layers that share
// head shape, pool size and stream.
hb_status copy_stack_blocks(hb_layer* const* layers, int n_layers, const int32_t* src, const int32_t* dst, int n);

// The device of a handle made current for the scope of one call.
class DeviceGuard {
 public:
  explicit DeviceGuard(int device) {
    if (hipGetDevice(&before_) != hipSuccess || before_ == device) before_ = -1;
    else (void)hipSetDevice(device);
  }
  ~DeviceGuard() {
    if (before_ >= 0) (void)hipSetDevice(before_);
  }
  DeviceGuard(const DeviceGuard&) = delete;
  DeviceGuard& operator=(const DeviceGuard&) = delete;

 private:
  int before_ = -1;
};

// f(), with a failed host allocation as a status.
template <typename F>
hb_status guarded(F&& f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return host_oom();
  }
}

}  // namespace hb
