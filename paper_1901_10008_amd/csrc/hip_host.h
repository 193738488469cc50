// What the entry points of the libraries of decoder steps share: errors, the device and stream that a plan's launches need, launches.
#pragma once

#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <new>
#include <string>

#include "launch_limits.h"
#include "sk_internal.h"

namespace sk {

inline sk_status hip_error(const char *what, hipError_t e) { return set_last_error(SK_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e)); }

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// Every entry point's body runs in here: no exception leaves the library.
template <class F>
sk_status guarded(F f) {
  try {
    return f();
  } catch (const std::bad_alloc &) {
    try {
      return set_last_error(SK_ERR_ALLOC, "host allocation failed");
    } catch (...) {
      return SK_ERR_ALLOC;
    }
  } catch (...) {
    return SK_ERR_INVALID_ARG;
  }
}

inline bool capturing(hipStream_t stream) {
  hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
  return hipStreamIsCapturing(stream, &cs) != hipSuccess || cs != hipStreamCaptureStatusNone;
}

// What every plan has of the device.
struct PlanOnDevice {
  int device = -1;
  bool resident = false;
  char *blob = nullptr;
  hipEvent_t last_use = nullptr;  // completes with the latest launch made outside a stream capture
  LaunchLedger ledger;            // of launches that use the plan's workspace
};

inline sk_status check_resident(const PlanOnDevice *plan) {
  if (!plan) return set_last_error(SK_ERR_INVALID_ARG, "plan is null");
  if (!plan->resident) return set_last_error(SK_ERR_STATE, "plan was created host-only; it has no device tables");
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_error("hipGetDevice", e);
  if (dev != plan->device) return set_last_error(SK_ERR_STATE, "plan belongs to another device than the current one");
  return SK_OK;
}

// As for the plans of superkernel.h: SK_ERR_BUSY while the previous launch still runs on another stream.
inline sk_status admit(PlanOnDevice *plan, hipStream_t stream, bool *in_capture) {
  const sk_status st = check_resident(plan);
  if (st != SK_OK) return st;
  *in_capture = capturing(stream);
  if (plan->ledger.before_launch((uintptr_t)stream, *in_capture) == LaunchLedger::QUERY_EVENT) {
    const hipError_t e = hipEventQuery(plan->last_use);
    if (e == hipErrorNotReady) {
      (void)hipGetLastError();
      return set_last_error(SK_ERR_BUSY, "the plan's previous launch is still running on another stream");
    }
    if (e != hipSuccess) return hip_error("hipEventQuery", e);
  }
  if (!*in_capture && !plan->last_use && hipEventCreateWithFlags(&plan->last_use, hipEventDisableTiming) != hipSuccess) {
    (void)hipGetLastError();
    plan->last_use = nullptr;
  }
  return SK_OK;
}

// Waits for what may still use the plan: `all` of the device's work, or what the ledger says.
inline hipError_t wait_for(const PlanOnDevice *plan, bool all) {
  hipError_t e = hipSuccess;
  const LaunchLedger::Wait wait = all ? LaunchLedger::DEVICE : plan->ledger.before_destroy();
  if (wait == LaunchLedger::EVENT) {
    e = hipEventSynchronize(plan->last_use);
  } else if (wait == LaunchLedger::DEVICE) {
    int cur = -1;
    e = hipGetDevice(&cur);
    if (e == hipSuccess && cur != plan->device) e = hipSetDevice(plan->device);
    if (e == hipSuccess) e = hipDeviceSynchronize();
    if (cur >= 0 && cur != plan->device) (void)hipSetDevice(cur);
  }
  return e;
}

// A launch whose completion is an event's signal (null: none).
template <class K, class A>
sk_status launch(K kernel, int64_t grid, hipStream_t stream, hipEvent_t behind, const A &args, int threads = CACHE_THREADS, size_t lds = 0) {
  const dim3 g((unsigned)grid), b((unsigned)threads);
  if (behind)
    hipExtLaunchKernelGGL(kernel, g, b, (unsigned)lds, stream, nullptr, behind, 0, args);
  else
    hipLaunchKernelGGL(kernel, g, b, lds, stream, args);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SK_OK : hip_error("kernel launch", e);
}

}  // namespace sk
