// What the libraries of decoder steps know of launches, for host code and kernels.
#pragma once

#include <cstdint>

namespace sk {

constexpr int CACHE_THREADS = 256;  // of a workgroup
// Workgroups of a launch: the runtime refuses 2^32 threads and more.
constexpr int64_t MOST_GRID = (((int64_t)1 << 32) - 1) / CACHE_THREADS;
constexpr int64_t PAST_CACHES = (int64_t)160 << 20;  // bytes that a launch reads and writes (the last-level cache holds 256 MiB)

}  // namespace sk
