// Internal declarations of the operators around the self-attention (rotary positions, norm, cross attention): they take
// no context, so what they share -- error text, per-device facts, argument checks -- is here.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/ditango.h"

namespace dt {

// What the operators need to know of the current device, looked up on the first call on it.
struct OpsDevice {
    int ordinal, sms;
    int32_t *status;      // device status word of the operators (dt_poll_ops)
    void *encode_tiled;   // cuTensorMapEncodeTiled
};

// What a kernel needs before its first launch on a device (a shared-memory limit): done by the first call that launches it, so that
// no operator loads another's kernels.  Threads that get here at once do the same.
struct OncePerDevice {
    std::atomic<uint64_t> done{0};
    template <typename F>
    cudaError_t operator()(const OpsDevice &dev, F &&configure) {
        const uint64_t bit = 1ull << dev.ordinal;
        if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
        const cudaError_t e = configure();
        if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
        return e;
    }
};

dt_status ops_fail(dt_status s, const char *what);                 // keeps the text for dt_last_error(NULL)
dt_status ops_fail_cuda(cudaError_t e, const char *where);
dt_status ops_device(const OpsDevice **out);
const char *ops_last_error();

// B, L, H, D strides in elements: D's is 1, the others are multiples of 8 (a stride of a dimension of one entry is not
// looked at), the base is 16-byte aligned.  Inputs may repeat (stride 0) along the batch; an output's rows may not overlap.
dt_status check_blhd(const char *name, const void *base, const int64_t *s, int B, int L, int H, int D, bool output);
// An output and an input with one base: in place, which needs the same strides.
bool same_strides(const int64_t *a, const int64_t *b, int B, int L, int H);

}  // namespace dt
