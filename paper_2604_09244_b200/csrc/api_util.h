// What the files with public entry points share: ranges and log lines around calls, the device of a call, and what a call
// that is no prune step needs to know of its context.
#pragma once

#include "attend_plan.h"
#include "common.cuh"

#include <cstdio>
#include <cstdlib>

#include <cudaTypedefs.h>
#include <nvtx3/nvToolsExt.h>

namespace mvla {

constexpr int kMaxBatch = 64;       // samples or sequences per call (mvla_prune_create refuses more)

// Tracing and logging, both on the host and off the device's path: every public call is an NVTX range (a profiler
// shows the call and, inside mvla_prune_step, its phases around the kernels they enqueue; without a profiler
// attached a range costs a few nanoseconds), and with MVLA_LOG=1 in the environment every call prints one line
// with its arguments and its result to stderr.
struct ApiRange {
    explicit ApiRange(const char* name) { nvtxRangePushA(name); }
    ~ApiRange() { nvtxRangePop(); }
    ApiRange(const ApiRange&) = delete;
    ApiRange& operator=(const ApiRange&) = delete;
};
inline bool log_enabled()
{
    static const bool on = [] {
        const char* e = std::getenv("MVLA_LOG");
        return e && *e && *e != '0';
    }();
    return on;
}

struct DeviceGuard {
    int prev = -1;
    bool ok = false;
    explicit DeviceGuard(int dev)
    {
        if (cudaGetDevice(&prev) != cudaSuccess) return;
        ok = (prev == dev) || cudaSetDevice(dev) == cudaSuccess;
    }
    ~DeviceGuard()
    {
        if (ok && prev >= 0) cudaSetDevice(prev);
    }
};

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// A context as the calls beside the prune step see it.
struct CtxView : ServeShape {
    int device;
    int* status_dev;                    // word that a kernel whose bounded wait gave up writes
    PFN_cuTensorMapEncodeTiled_v12000 encode;
};
// Opens such a call: the sticky status.
int32_t open_call(mvla_ctx* ctx, CtxView* view);
// The call enqueues work: what the stream ran last is no longer a known prune step, and the next one with stable inputs is ordered after all of it.  (Not
// for a call that is refused or has nothing to do: the overlap of the prune steps around it stays.)
void note_work(mvla_ctx* ctx);
int32_t close_call(mvla_ctx* ctx, cudaError_t e);      // status of the call's launches

}  // namespace mvla
