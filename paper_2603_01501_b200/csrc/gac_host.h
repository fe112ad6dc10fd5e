// Host-side helpers shared by the translation units of the library: the message of the last
// failed call without a context, the current-device guard, CUDA error checks and profiler ranges.
#pragma once

#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>
#include <stdio.h>

#include "gac.h"

// What gac_last_error(NULL) returns: one buffer per host thread for the whole library.
inline thread_local char g_init_err[512] = "no error";

namespace {

struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev) {
        if (cudaGetDevice(&prev) != cudaSuccess) prev = -1;
        ok = (prev == dev) || (cudaSetDevice(dev) == cudaSuccess);
        if (prev == dev) prev = -1;   // nothing to put back
    }
    ~DeviceGuard() {
        if (prev >= 0) cudaSetDevice(prev);
    }
};

// Every failing call of the library goes through a `fail` of its translation unit.
#define GAC_CUDA(ctx, call)                                                          \
    do {                                                                             \
        cudaError_t e_ = (call);                                                     \
        if (e_ != cudaSuccess)                                                       \
            return fail((ctx), GAC_ERR_CUDA, "%s (CUDA error %lld): " #call,        \
                        cudaGetErrorString(e_), (long long)e_);                      \
    } while (0)

// Named range around the host side of a call, visible in a timeline profiler; costs one
// pointer test when no tool is attached.
struct Range {
    explicit Range(const char *name) { nvtxRangePushA(name); }
    ~Range() { nvtxRangePop(); }
};

}  // namespace
