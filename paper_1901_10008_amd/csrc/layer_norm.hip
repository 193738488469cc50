// Norms before and after a block: entry points.
#include <atomic>

#include "layer_host.h"
#include "layer_norm.hip.h"

namespace sk {
#define SK_NORM_FORM(T, P)                                      \
  extern template __global__ void sk_norm<T, P, false>(NormArgs); \
  extern template __global__ void sk_norm<T, P, true>(NormArgs);
SK_NORM_FORM(16, 2)
SK_NORM_FORM(64, 2)
SK_NORM_FORM(128, 2)
SK_NORM_FORM(256, 2)
SK_NORM_FORM(512, 2)
SK_NORM_FORM(1024, 4)
#undef SK_NORM_FORM
}  // namespace sk

struct sk_norm_plan : sk::PlanOnDevice {
  sk::NormPlanHost host;
  std::atomic<bool> launched{false};  // (launches may overlap, from several threads too)
};

namespace {

sk_status upload(sk_norm_plan &plan) {
  const std::vector<sk::NormLaunch> &launches = plan.host.launches;
  if (launches.empty()) return SK_OK;
  std::vector<char> image(launches.size() * sizeof(sk::NormTable));
  for (size_t i = 0; i < launches.size(); ++i) std::memcpy(image.data() + i * sizeof(sk::NormTable), &launches[i].table, sizeof(sk::NormTable));
  char *ws = nullptr;
  const sk_status st = sk::upload_image(plan, image, 0, &ws);
  return st == SK_OK ? sk::copy_image(plan, image) : st;
}

template <int T, int P>
void (*kernel_of(bool once))(sk::NormArgs) {
  return once ? sk::sk_norm<T, P, true> : sk::sk_norm<T, P, false>;
}
void (*norm_kernel(sk::NormForm form, bool once))(sk::NormArgs) {
  switch (form) {
    case sk::NORM_SIXTEEN: return kernel_of<16, 2>(once);
    case sk::NORM_WAVE: return kernel_of<64, 2>(once);
    case sk::NORM_ROWS: return kernel_of<128, 2>(once);
    case sk::NORM_GROUP: return kernel_of<256, 2>(once);
    case sk::NORM_PAIR: return kernel_of<512, 2>(once);
    default: return kernel_of<1024, 4>(once);
  }
}

}  // namespace

extern "C" {

void sk_layer_params_default(sk_layer_params *params) {
  if (params) *params = sk_layer_params{};
}

sk_status sk_norm_plan_create(const sk_norm_problem *problems, int32_t n, const sk_layer_params *params, sk_norm_plan **out) {
  return sk::create_plan<sk_norm_plan>(params, out, [&](sk_norm_plan &plan, int32_t, int32_t, std::string &err) { return sk::plan_norm(problems, n, plan.host, err); },
                                       upload);
}

sk_status sk_norm_plan_destroy(sk_norm_plan *plan) {
  if (!plan) return SK_OK;
  return sk::guarded([&]() -> sk_status { return sk::destroy_plan(plan, plan->launched.load(std::memory_order_relaxed)); });
}

sk_status sk_norm_launch(sk_norm_plan *plan, void *hip_stream) {
  return sk::guarded([&]() -> sk_status {
    sk_status st = sk::check_resident(plan);
    if (st != SK_OK) return st;
    const sk::NormTable *table = (const sk::NormTable *)plan->blob;
    plan->launched.store(true, std::memory_order_relaxed);
    for (const sk::NormLaunch &l : plan->host.launches) {
      if (st != SK_OK) break;
      st = sk::launch(norm_kernel(l.form, l.once), l.grid, (hipStream_t)hip_stream, nullptr, sk::NormArgs{table++, l.n}, sk::norm_threads(l.form));
    }
    return st;
  });
}

}  // extern "C"
