// What the context-free operators share: error text, facts about the current device, argument checks.
#include <algorithm>
#include <cstdio>
#include <cstring>

#include "dt_internal.h"
#include "ops.h"

namespace dt {
namespace {

thread_local char g_error[192] = "";
__device__ int32_t g_status;   // conditions only the device can see; zero at load time, cleared by dt_poll_ops

constexpr int MAX_DEVICES = 64;   // bits of OncePerDevice::done
OpsDevice g_devices[MAX_DEVICES];
std::atomic<int> g_ready[MAX_DEVICES];
std::atomic_flag g_looking_up = ATOMIC_FLAG_INIT;

// Fills g_devices[dev] with g_looking_up held.
dt_status look_up(int dev) {
    OpsDevice d = {};
    d.ordinal = dev;
    cudaError_t e;
    int major = 0;
    if ((e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev)) != cudaSuccess ||
        (e = cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess)
        return ops_fail_cuda(e, "device attributes");
    if (major != 10) return ops_fail(DT_ERR_UNSUPPORTED, "the kernels are built for sm_100 only");
    void *word = nullptr;
    if ((e = cudaGetSymbolAddress(&word, g_status)) != cudaSuccess) return ops_fail_cuda(e, "status word");
    d.status = static_cast<int32_t *>(word);
    cudaDriverEntryPointQueryResult qres;
    e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &d.encode_tiled, cudaEnableDefault, &qres);
    if (e != cudaSuccess) return ops_fail_cuda(e, "cuTensorMapEncodeTiled");
    if (qres != cudaDriverEntryPointSuccess || !d.encode_tiled) return ops_fail(DT_ERR_CUDA, "cuTensorMapEncodeTiled not found");
    g_devices[dev] = d;
    g_ready[dev].store(1, std::memory_order_release);
    return DT_OK;
}

}  // namespace

dt_status ops_fail(dt_status s, const char *what) {
    snprintf(g_error, sizeof g_error, "%s", what);
    return s;
}

dt_status ops_fail_cuda(cudaError_t e, const char *where) {
    snprintf(g_error, sizeof g_error, "%s: %s", where, cudaGetErrorString(e));
    return DT_ERR_CUDA;
}

const char *ops_last_error() { return g_error; }

dt_status ops_device(const OpsDevice **out) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return ops_fail_cuda(e, "cudaGetDevice");
    if (dev < 0 || dev >= MAX_DEVICES) return ops_fail(DT_ERR_UNSUPPORTED, "device ordinal beyond 63");
    if (!g_ready[dev].load(std::memory_order_acquire)) {
        while (g_looking_up.test_and_set(std::memory_order_acquire)) {}   // (no call in there waits for another thread)
        const dt_status s = g_ready[dev].load(std::memory_order_acquire) ? DT_OK : look_up(dev);
        g_looking_up.clear(std::memory_order_release);
        if (s != DT_OK) return s;
    }
    // The tensor maps' encoder is of the driver: it wants the device's context current in the calling thread, which the runtime only
    // sees to in calls that need one itself.  A thread whose first CUDA call is an operator has had none.
    thread_local uint64_t bound = 0;
    if (!(bound >> dev & 1)) {
        if ((e = cudaSetDevice(dev)) != cudaSuccess) return ops_fail_cuda(e, "cudaSetDevice");
        bound |= 1ull << dev;
    }
    *out = &g_devices[dev];
    return DT_OK;
}

dt_status check_blhd(const char *name, const void *base, const int64_t *s, int B, int L, int H, int D, bool output) {
    char text[128];
    const char *why = nullptr;
    const int n[3] = {B, L, H};
    if (!base || !s) why = "null pointer or strides";
    else if (s[3] != 1) why = "stride of D must be 1";
    else if ((reinterpret_cast<uintptr_t>(base) & 15u) != 0) why = "base must be 16-byte aligned";
    else
        for (int d = 0; d < 3 && !why; ++d) {
            if (n[d] <= 1) continue;
            const bool repeats = d == 0 && s[d] == 0 && !output;
            if (!repeats && (s[d] <= 0 || s[d] % 8 != 0)) why = "strides of B, L, H must be positive multiples of 8 elements";
        }
    if (!why && output) {   // from the innermost dimension outwards, each step beyond what lies within
        int at[3] = {0, 1, 2};
        std::sort(at, at + 3, [&](int i, int j) { return s[i] < s[j]; });
        int64_t extent = D;
        for (int d : at) {
            if (n[d] <= 1) continue;
            if (s[d] < extent) why = "an output's rows must not overlap";
            extent += s[d] * (n[d] - 1);
        }
    }
    if (!why) return DT_OK;
    snprintf(text, sizeof text, "%s: %s", name, why);
    return ops_fail(DT_ERR_INVALID_ARG, text);
}

bool same_strides(const int64_t *a, const int64_t *b, int B, int L, int H) {
    return (B <= 1 || a[0] == b[0]) && (L <= 1 || a[1] == b[1]) && (H <= 1 || a[2] == b[2]);
}

}  // namespace dt

extern "C" dt_status dt_poll_ops(void) {
    const dt::OpsDevice *dev;
    dt_status s = dt::ops_device(&dev);
    if (s != DT_OK) return s;
    int32_t word = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpy(&word, dev->status, sizeof word, cudaMemcpyDeviceToHost);
    if (e == cudaSuccess && word) e = cudaMemset(dev->status, 0, sizeof word);
    if (e != cudaSuccess) return dt::ops_fail_cuda(e, "dt_poll_ops");
    if (word & dt::STATUS_WAIT_TIMEOUT) return dt::ops_fail(DT_ERR_TIMEOUT, "a bounded device-side wait expired");
    return DT_OK;
}
