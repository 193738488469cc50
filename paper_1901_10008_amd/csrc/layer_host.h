// Plans of libsk_layer.so: what their entry points share.
#pragma once

#include <cstring>

#include "hip_host.h"
#include "layer_internal.h"

namespace sk {

// Frees a plan that nothing uses any more.
template <class Plan>
void release(Plan *plan) {
  if (plan->blob) (void)hipFree(plan->blob);
  if (plan->last_use) (void)hipEventDestroy(plan->last_use);
  delete plan;
}

template <class Plan>
sk_status destroy_plan(Plan *plan, bool wait_for_all) {
  const hipError_t e = plan->resident ? wait_for(plan, wait_for_all) : hipSuccess;
  const sk_status st = e == hipSuccess ? SK_OK : hip_error("waiting for the plan's launches", e);
  if (e != hipSuccess) plan->blob = nullptr;  // not freed under a kernel that may still run
  release(plan);
  return st;
}

// A plan on the current device (unless host_only): `check` plans, `upload` brings its tables there.
template <class Plan, class F, class G>
sk_status create_plan(const sk_layer_params *params, Plan **out, F check, G upload) {
  return guarded([&]() -> sk_status {
    if (!out) return set_last_error(SK_ERR_INVALID_ARG, "out is null");
    sk_layer_params prm{};
    if (params) prm = *params;
    if ((prm.host_only != 0 && prm.host_only != 1) || prm.workgroups < 0 || prm.workgroups > 65536 || prm.reserved[0] || prm.reserved[1])
      return set_last_error(SK_ERR_INVALID_ARG, "bad params field");
    int cus = 256, device = -1;
    if (!prm.host_only) {
      hipError_t e = hipGetDevice(&device);
      if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device);
      if (e != hipSuccess) return hip_error("hipGetDevice", e);
    }
    Plan *plan = new Plan;
    try {
      plan->device = device;
      std::string err;
      sk_status st = check(*plan, cus, prm.workgroups, err);
      if (st != SK_OK) st = set_last_error(st, err);
      if (st == SK_OK && !prm.host_only) {
        st = upload(*plan);
        plan->resident = st == SK_OK;
      }
      if (st != SK_OK) {
        release(plan);
        return st;
      }
    } catch (...) {
      release(plan);
      throw;
    }
    *out = plan;
    return SK_OK;
  });
}

// Device memory of a plan: `image` (tables and zeroed counters), and `workspace` bytes behind it, whose address goes to *ws.
inline sk_status upload_image(PlanOnDevice &plan, const std::vector<char> &image, size_t workspace, char **ws) {
  const size_t tables = align_up(image.size(), 256);
  hipError_t e = hipMalloc((void **)&plan.blob, std::max<size_t>(tables + workspace, 256));
  if (e != hipSuccess) {
    (void)hipGetLastError();
    plan.blob = nullptr;
    return set_last_error(SK_ERR_ALLOC, std::string("hipMalloc: ") + hipGetErrorString(e));
  }
  *ws = plan.blob + tables;
  return SK_OK;
}
inline sk_status copy_image(PlanOnDevice &plan, const std::vector<char> &image) {
  if (image.empty()) return SK_OK;
  const hipError_t e = hipMemcpy(plan.blob, image.data(), image.size(), hipMemcpyHostToDevice);
  return e == hipSuccess ? SK_OK : hip_error("hipMemcpy", e);
}

}  // namespace sk
