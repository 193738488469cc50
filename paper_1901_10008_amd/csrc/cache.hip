// Entry points of libsk_cache.so: attention plans and their launches, the account of pages and its copies.
#include <cstring>

#include "cache_rows.hip.h"
#include "hip_host.h"

namespace sk {
extern template __global__ void sk_attend<false, false>(AttnArgs);
extern template __global__ void sk_attend<true, false>(AttnArgs);
extern template __global__ void sk_attend<false, true>(AttnArgs);
extern template __global__ void sk_attend<true, true>(AttnArgs);
}  // namespace sk

namespace {

using sk::admit;
using sk::align_up;
using sk::capturing;
using sk::check_resident;
using sk::guarded;
using sk::hip_error;
using sk::launch;
using sk::set_last_error;

}  // namespace

struct sk_attn_plan : sk::PlanOnDevice {
  sk::AttnPlanHost host;
  const sk::AttnDev *problems = nullptr;
  const sk::AttnSeq *seqs = nullptr;
  const uint32_t *append_first = nullptr;
  uint32_t *arrivals = nullptr;
  float *workspace = nullptr;
  bool appended = false;  // sk_attn_append has been called
};

struct sk_pages {
  sk::PageAccount account;
  // rows of the page table on their way to the device: pinned memory in turn, each with an event behind the launch that reads it
  static constexpr int SLOTS = 4;
  int32_t *rows[SLOTS] = {};
  hipEvent_t done[SLOTS] = {};
  bool used[SLOTS] = {};
  int next = 0;
  sk_pages(int32_t num_pages, int32_t page_tokens, int32_t sequences, int32_t columns) : account(num_pages, page_tokens, sequences, columns) {}
};

namespace {

void (*attend_kernel(const sk::AttnGroup &g))(sk::AttnArgs) {
  if (g.wide) return g.many ? sk::sk_attend<true, true> : sk::sk_attend<false, true>;
  return g.many ? sk::sk_attend<true, false> : sk::sk_attend<false, false>;
}

void release(sk_attn_plan *plan) {
  if (plan->blob) (void)hipFree(plan->blob);
  if (plan->last_use) (void)hipEventDestroy(plan->last_use);
  delete plan;
}

sk_status make_resident(sk_attn_plan *plan) {
  const sk::AttnPlanHost &h = plan->host;
  const size_t o_seqs = align_up(h.problems.size() * sizeof(sk::AttnDev), 256), o_first = o_seqs + align_up(h.seqs.size() * sizeof(sk::AttnSeq), 256);
  const size_t o_arrivals = o_first + align_up(h.append_first.size() * 4, 256), o_ws = o_arrivals + align_up((size_t)h.counters * 4, 256);
  const size_t bytes = o_ws + (size_t)h.workspace_floats * 4;
  hipError_t e = hipMalloc((void **)&plan->blob, bytes);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    plan->blob = nullptr;
    return set_last_error(SK_ERR_ALLOC, std::string("hipMalloc: ") + hipGetErrorString(e));
  }
  std::vector<char> image(o_ws, 0);  // counters: zero
  std::memcpy(image.data(), h.problems.data(), h.problems.size() * sizeof(sk::AttnDev));
  std::memcpy(image.data() + o_seqs, h.seqs.data(), h.seqs.size() * sizeof(sk::AttnSeq));
  std::memcpy(image.data() + o_first, h.append_first.data(), h.append_first.size() * 4);
  e = hipMemcpy(plan->blob, image.data(), o_ws, hipMemcpyHostToDevice);
  if (e != hipSuccess) return hip_error("hipMemcpy", e);
  plan->problems = (const sk::AttnDev *)plan->blob;
  plan->seqs = (const sk::AttnSeq *)(plan->blob + o_seqs);
  plan->append_first = (const uint32_t *)(plan->blob + o_first);
  plan->arrivals = (uint32_t *)(plan->blob + o_arrivals);
  plan->workspace = (float *)(plan->blob + o_ws);
  plan->resident = true;
  return SK_OK;
}

// The copies of one wave and, with the last launch, n_rows rows of the page table: in host memory that the device can read (`pinned`), or as
// `put` writes them into the launch's arguments.
template <class F>
sk_status launch_copies(const sk_page_array *arrays, int32_t n_arrays, const sk::PageMove *moves, size_t n_moves, hipStream_t stream, int32_t *table, int32_t n_rows,
                        int32_t columns, const int32_t *pinned, F put, hipEvent_t behind) {
  sk::CopyArgs a;
  a.table = table;
  a.columns = columns;
  double bytes = 0.0;
  int64_t most_chunks = 1;
  for (int32_t i = 0; i < n_arrays; ++i) {
    bytes += (double)arrays[i].page_bytes;
    most_chunks = std::max(most_chunks, (arrays[i].page_bytes + sk::COPY_CHUNK - 1) / sk::COPY_CHUNK);
  }
  const sk::CopyBatch batch = sk::copy_batch(most_chunks);
  void (*const kernel)(sk::CopyArgs) = bytes * 2.0 * (double)n_moves > (double)sk::PAST_CACHES ? sk::sk_copy_pages<true> : sk::sk_copy_pages<false>;
  for (int32_t a0 = 0;; a0 += batch.arrays) {
    a.n_arrays = n_moves ? std::max(0, std::min(n_arrays - a0, batch.arrays)) : 0;
    a.chunks = 0;
    for (int32_t i = 0; i < a.n_arrays; ++i) {
      std::memcpy(a.words + 4 * i, &arrays[a0 + i].base, 8);
      std::memcpy(a.words + 4 * i + 2, &arrays[a0 + i].page_bytes, 8);
      a.chunks = std::max(a.chunks, (arrays[a0 + i].page_bytes + sk::COPY_CHUNK - 1) / sk::COPY_CHUNK);
    }
    const bool last_arrays = n_arrays - a0 <= batch.arrays || !n_moves;
    for (size_t m0 = 0;; m0 += (size_t)batch.moves) {
      a.n_moves = a.n_arrays ? (int32_t)std::min(n_moves - m0, (size_t)batch.moves) : 0;
      if (a.n_moves) std::memcpy(a.words + 4 * a.n_arrays, moves + m0, (size_t)a.n_moves * sizeof(sk::PageMove));
      const bool last = last_arrays && m0 + (size_t)batch.moves >= n_moves;
      const int64_t copies = a.chunks * a.n_arrays * a.n_moves;
      bool with_rows = last && n_rows;
      a.rows = pinned;
      if (with_rows && !pinned) {
        const int64_t at = 4 * a.n_arrays + 2 * a.n_moves, words = n_rows * (1 + (int64_t)columns);
        if (at + words <= sk::COPY_WORDS) put(a.words + at);
        else with_rows = false;  // they get a launch of their own
      }
      a.n_rows = with_rows ? n_rows : 0;
      const bool alone = last && n_rows && !with_rows;
      if (copies + a.n_rows) {
        const sk_status st = launch(kernel, copies + std::min(a.n_rows, sk::ROW_GROUPS), stream, last && !alone ? behind : nullptr, a);
        if (st != SK_OK) return st;
      }
      if (alone) {
        a.n_arrays = a.n_moves = 0;
        a.n_rows = n_rows;
        put(a.words);
        return launch(kernel, std::min(n_rows, sk::ROW_GROUPS), stream, behind, a);
      }
      if (m0 + (size_t)batch.moves >= n_moves) break;
    }
    if (last_arrays) return SK_OK;
  }
}

sk_status check_arrays(const sk_page_array *arrays, int32_t n_arrays) {
  if (n_arrays < 0 || (n_arrays && !arrays)) return set_last_error(SK_ERR_INVALID_ARG, "arrays is null or n_arrays is negative");
  for (int32_t i = 0; i < n_arrays; ++i) {
    if (!arrays[i].base || arrays[i].page_bytes < 1) return set_last_error(SK_ERR_INVALID_ARG, "an array without memory or with empty pages");
    if (((uintptr_t)arrays[i].base | (uintptr_t)arrays[i].page_bytes) & 15) return set_last_error(SK_ERR_UNSUPPORTED, "arrays and pages must be multiples of 16 bytes");
    if (arrays[i].page_bytes > sk::COPY_PAGE) return set_last_error(SK_ERR_UNSUPPORTED, "a page of more than 2^38 bytes");
  }
  return SK_OK;
}

}  // namespace

extern "C" {

void sk_attn_params_default(sk_attn_params *params) {
  if (params) *params = sk_attn_params{};
}

sk_status sk_attn_plan_create(const sk_attn_problem *problems, int32_t n, const sk_attn_params *params, sk_attn_plan **out) {
  return guarded([&]() -> sk_status {
    if (!out) return set_last_error(SK_ERR_INVALID_ARG, "out is null");
    sk_attn_params prm{};
    if (params) prm = *params;
    if ((prm.host_only != 0 && prm.host_only != 1) || prm.workgroups < 0 || prm.workgroups > 65536 || prm.reserved[0] || prm.reserved[1])
      return set_last_error(SK_ERR_INVALID_ARG, "bad params field");
    int cus = 256, device = -1;
    if (!prm.host_only) {
      hipError_t e = hipGetDevice(&device);
      if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device);
      if (e != hipSuccess) return hip_error("hipGetDevice", e);
    }
    sk_attn_plan *plan = new sk_attn_plan;
    try {
      plan->device = device;
      std::string err;
      sk_status st = sk::plan_attn(problems, n, cus, prm.workgroups, plan->host, err);
      if (st != SK_OK) st = set_last_error(st, err);
      if (st == SK_OK && !prm.host_only) st = make_resident(plan);
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

sk_status sk_attn_plan_destroy(sk_attn_plan *plan) {
  if (!plan) return SK_OK;
  return guarded([&]() -> sk_status {
    const hipError_t e = sk::wait_for(plan, plan->appended);
    const sk_status st = e == hipSuccess ? SK_OK : hip_error("waiting for the plan's launches", e);
    if (e != hipSuccess) plan->blob = nullptr;  // not freed under a kernel that may still run
    release(plan);
    return st;
  });
}

sk_status sk_attn_append(sk_attn_plan *plan, void *hip_stream) {
  return guarded([&]() -> sk_status {
    const hipStream_t stream = (hipStream_t)hip_stream;
    sk_status st = check_resident(plan);
    if (st != SK_OK || plan->host.problems.empty()) return st;
    if (!plan->host.all_qkv) return set_last_error(SK_ERR_STATE, "a problem of the plan has no qkv");
    const sk::AppendArgs a{plan->problems, plan->append_first, (int32_t)plan->host.problems.size()};
    // It writes nothing of the plan's, so no later launch has to wait for it, only the plan's end (for the device: an event with
    // the launch makes who waits for the device behind it wait up to 10 us longer).
    st = launch(plan->host.append_once ? sk::sk_append<true> : sk::sk_append<false>, (int64_t)plan->host.append_first.back(), stream, nullptr, a);
    plan->appended = true;
    return st;
  });
}

sk_status sk_attn_launch(sk_attn_plan *plan, void *hip_stream) {
  return guarded([&]() -> sk_status {
    const hipStream_t stream = (hipStream_t)hip_stream;
    bool in_capture = false;
    sk_status st = admit(plan, stream, &in_capture);
    if (st != SK_OK || plan->host.problems.empty()) return st;
    if (!plan->host.all_out) return set_last_error(SK_ERR_STATE, "a problem of the plan has no out");
    const hipEvent_t behind = in_capture ? nullptr : plan->last_use;
    for (const sk::AttnGroup &g : plan->host.groups) {
      sk::AttnArgs a{};
      a.problems = plan->problems;
      a.seqs = plan->seqs + g.first_seq;
      a.sequences = (int32_t)g.sequences;
      a.grid = (uint32_t)g.grid;
      a.slots_many = (uint32_t)g.slots_many;
      a.slots_few = (uint32_t)g.slots_few;
      a.workgroups = (int32_t)g.workgroups;
      a.ws_many = plan->workspace;
      a.ws_few = plan->workspace + g.slots_many * sk::part_floats(sk::ROWS_MANY, g.wide ? 256 : 128);
      a.arrivals = plan->arrivals;
      st = launch(attend_kernel(g), g.grid, stream, &g == &plan->host.groups.back() ? behind : nullptr, a);
      if (st != SK_OK) break;
    }
    plan->ledger.after_launch((uintptr_t)stream, in_capture, behind && st == SK_OK);  // also after a failure: some launches may be out
    return st;
  });
}

sk_status sk_attn_plan_info(const sk_attn_plan *plan, int32_t *launches, int64_t *workspace_bytes) {
  return guarded([&]() -> sk_status {
    if (!plan) return set_last_error(SK_ERR_INVALID_ARG, "plan is null");
    if (launches) *launches = (int32_t)plan->host.groups.size();
    if (workspace_bytes) *workspace_bytes = plan->host.workspace_floats * 4;
    return SK_OK;
  });
}

sk_status sk_pages_create(int32_t num_pages, int32_t page_tokens, int32_t sequences, int32_t pages_per_sequence, sk_pages **out) {
  return guarded([&]() -> sk_status {
    if (!out || num_pages < 1 || page_tokens < 1 || sequences < 1 || pages_per_sequence < 1) return set_last_error(SK_ERR_INVALID_ARG, "out is null or a size is less than 1");
    if ((int64_t)pages_per_sequence * page_tokens >= (int64_t)1 << 31 || (int64_t)sequences * pages_per_sequence >= (int64_t)1 << 31)
      return set_last_error(SK_ERR_UNSUPPORTED, "the page table is too large");
    *out = new sk_pages(num_pages, page_tokens, sequences, pages_per_sequence);
    return SK_OK;
  });
}

sk_status sk_pages_destroy(sk_pages *pages) {
  if (!pages) return SK_OK;
  return guarded([&]() -> sk_status {
    hipError_t e = hipSuccess;
    for (int i = 0; i < sk_pages::SLOTS; ++i) {
      if (pages->used[i] && e == hipSuccess) e = hipEventSynchronize(pages->done[i]);
      if (pages->done[i]) (void)hipEventDestroy(pages->done[i]);
      if (pages->rows[i] && e == hipSuccess) (void)hipHostFree(pages->rows[i]);
    }
    delete pages;
    return e == hipSuccess ? SK_OK : hip_error("waiting for the account's launches", e);
  });
}

sk_status sk_pages_resize(sk_pages *pages, const int32_t *sequences, const int32_t *tokens, int32_t n) {
  return guarded([&]() -> sk_status {
    if (!pages || n < 0 || (n && (!sequences || !tokens))) return set_last_error(SK_ERR_INVALID_ARG, "null pointer or negative n");
    std::string err;
    const sk_status st = pages->account.resize(sequences, tokens, n, err);
    return st == SK_OK ? st : set_last_error(st, err);
  });
}

sk_status sk_pages_fork(sk_pages *pages, int32_t from, const int32_t *to, int32_t n) {
  return guarded([&]() -> sk_status {
    if (!pages || n < 0 || (n && !to)) return set_last_error(SK_ERR_INVALID_ARG, "null pointer or negative n");
    std::string err;
    const sk_status st = pages->account.fork(from, to, n, err);
    return st == SK_OK ? st : set_last_error(st, err);
  });
}

sk_status sk_pages_compact(sk_pages *pages) {
  return guarded([&]() -> sk_status {
    if (!pages) return set_last_error(SK_ERR_INVALID_ARG, "pages is null");
    return pages->account.compact();
  });
}

sk_status sk_pages_state(const sk_pages *pages, int32_t *free_pages, int32_t *pending_copies, int32_t sequence, int32_t *tokens, int32_t *row) {
  return guarded([&]() -> sk_status {
    if (!pages) return set_last_error(SK_ERR_INVALID_ARG, "pages is null");
    if ((tokens || row) && (sequence < 0 || sequence >= pages->account.sequences())) return set_last_error(SK_ERR_INVALID_ARG, "no such sequence");
    if (free_pages) *free_pages = pages->account.free_pages();
    if (pending_copies) *pending_copies = pages->account.pending();
    if (tokens) *tokens = pages->account.tokens(sequence);
    if (row) std::memcpy(row, pages->account.row(sequence), (size_t)pages->account.columns() * 4);
    return SK_OK;
  });
}

sk_status sk_pages_apply(sk_pages *pages, const sk_page_array *arrays, int32_t n_arrays, int32_t *page_table, void *hip_stream) {
  return guarded([&]() -> sk_status {
    if (!pages) return set_last_error(SK_ERR_INVALID_ARG, "pages is null");
    sk_status st = check_arrays(arrays, n_arrays);
    if (st != SK_OK) return st;
    if ((uintptr_t)page_table & 3) return set_last_error(SK_ERR_UNSUPPORTED, "the page table must be a multiple of 4 bytes");
    const hipStream_t stream = (hipStream_t)hip_stream;
    if (capturing(stream)) return set_last_error(SK_ERR_STATE, "inside a stream capture");
    sk::PageAccount &acc = pages->account;
    const std::vector<int32_t> &dirty = acc.dirty_rows();
    const int32_t n_rows = page_table ? (int32_t)dirty.size() : 0, columns = acc.columns();
    const std::vector<std::vector<sk::PageMove>> waves = acc.waves();
    if (waves.empty() && !n_rows) return SK_OK;
    auto put = [&](int32_t *to) {
      std::memcpy(to, dirty.data(), (size_t)n_rows * 4);
      for (int32_t r = 0; r < n_rows; ++r) std::memcpy(to + n_rows + (size_t)r * columns, acc.row(dirty[r]), (size_t)columns * 4);
    };
    const int i = pages->next;
    hipError_t e = hipSuccess;
    const bool pinned = n_rows && n_rows * (1 + (int64_t)columns) > sk::COPY_WORDS;  // more than a launch's arguments hold
    if (pinned) {
      if (!pages->rows[i]) {
        const size_t bytes = ((size_t)acc.sequences() * (columns + 1)) * 4;
        if ((e = hipHostMalloc((void **)&pages->rows[i], bytes, hipHostMallocDefault)) != hipSuccess) {
          (void)hipGetLastError();
          pages->rows[i] = nullptr;
          return set_last_error(SK_ERR_ALLOC, std::string("hipHostMalloc: ") + hipGetErrorString(e));
        }
      }
      if (!pages->done[i] && (e = hipEventCreateWithFlags(&pages->done[i], hipEventDisableTiming)) != hipSuccess) return hip_error("hipEventCreate", e);
      if (pages->used[i] && (e = hipEventSynchronize(pages->done[i])) != hipSuccess) return hip_error("hipEventSynchronize", e);
      pages->used[i] = false;
      put(pages->rows[i]);
    }
    const size_t launches = std::max<size_t>(waves.size(), 1);
    for (size_t w = 0; w < launches; ++w) {
      const bool last = w + 1 == launches;
      st = launch_copies(arrays, n_arrays, waves.empty() ? nullptr : waves[w].data(), waves.empty() ? 0 : waves[w].size(), stream, page_table, last ? n_rows : 0,
                         columns, pinned ? pages->rows[i] : nullptr, put, last && pinned ? pages->done[i] : nullptr);
      if (st != SK_OK) return st;
    }
    if (pinned) {
      pages->used[i] = true;
      pages->next = (i + 1) % sk_pages::SLOTS;
    }
    acc.applied(page_table != nullptr);
    return SK_OK;
  });
}

sk_status sk_pages_copy(const sk_page_array *arrays, int32_t n_arrays, int32_t num_pages, const int32_t *from, const int32_t *to, int32_t n, void *hip_stream) {
  return guarded([&]() -> sk_status {
    sk_status st = check_arrays(arrays, n_arrays);
    if (st != SK_OK) return st;
    if (num_pages < 1 || n < 0 || (n && (!from || !to))) return set_last_error(SK_ERR_INVALID_ARG, "null pointer, negative n or no pages");
    std::vector<sk::PageMove> moves((size_t)n);
    std::vector<uint8_t> seen((size_t)num_pages, 0);
    for (int32_t i = 0; i < n; ++i) {
      if (from[i] < 0 || from[i] >= num_pages || to[i] < 0 || to[i] >= num_pages) return set_last_error(SK_ERR_INVALID_ARG, "copy " + std::to_string(i) + ": no such page");
      if (seen[to[i]]) return set_last_error(SK_ERR_OVERLAP, "copy " + std::to_string(i) + ": its page is written twice");
      seen[to[i]] = 1;
      moves[(size_t)i] = sk::PageMove{from[i], to[i]};
    }
    for (int32_t i = 0; i < n; ++i)
      if (seen[from[i]]) return set_last_error(SK_ERR_OVERLAP, "copy " + std::to_string(i) + ": its page is read and written");
    if (!n || !n_arrays) return SK_OK;
    return launch_copies(arrays, n_arrays, moves.data(), moves.size(), (hipStream_t)hip_stream, nullptr, 0, 0, nullptr, [](int32_t *) {}, nullptr);
  });
}

}  // extern "C"
