// What the sources behind the C ABI share on the host: the library's lock, per-kernel timing, argument checks, workspace
// layout.  Defined in meft_api.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <mutex>
#include <vector>

#include "../../include/meft.h"

namespace meft {

#pragma GCC visibility push(hidden)

// The host side of every entry point that enqueues work or touches the library's few pieces of process-wide state
// (the timing list, the side stream and events of the host-resident variant, the table of staged workspaces) runs
// under this lock, so the entry points may be called from several host threads.
extern std::mutex g_api_mutex;
#define MEFT_API_LOCK() std::lock_guard<std::mutex> api_lock_(g_api_mutex)

// ---- per-kernel timing ----------------------------------------------------------------------
struct ProfEntry {
  const char* name;
  hipEvent_t start, stop;
};
extern bool g_prof_on;
extern std::vector<ProfEntry> g_prof;

struct LaunchScope {
  hipStream_t st;
  bool on;
  hipEvent_t stop{};
  LaunchScope(const char* name, hipStream_t s) : st(s), on(g_prof_on) {
    if (!on) return;
    ProfEntry e{name, nullptr, nullptr};
    if (hipEventCreate(&e.start) != hipSuccess || hipEventCreate(&e.stop) != hipSuccess) {
      on = false;
      return;
    }
    (void)hipEventRecord(e.start, st);
    stop = e.stop;
    g_prof.push_back(e);
  }
  ~LaunchScope() {
    if (on) (void)hipEventRecord(stop, st);
  }
};

#define MEFT_LAUNCH(name, kernel, grid, block, shmem, stream, ...)            \
  do {                                                                        \
    LaunchScope scope_(name, stream);                                         \
    hipLaunchKernelGGL(kernel, grid, block, shmem, stream, __VA_ARGS__);      \
  } while (0)

// ---- checks ---------------------------------------------------------------------------------
constexpr int kMaxD = 16384, kMaxBlocks = 16384;

meft_status check_shape(const meft_shape* s);
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// MEFT_ERR_DEVICE and its description if a launch since clear_stale_error() failed.  The runtime keeps the last error of the
// thread until it is read: an entry point reads it away before its first launch, so that MEFT_ERR_DEVICE reports this call's
// own launches and not a failure some other code left behind.
meft_status launch_status();
inline void clear_stale_error() { (void)hipGetLastError(); }

// ---- workspace layout -----------------------------------------------------------------------
struct Carver {
  char* base;
  size_t off = 0;
  explicit Carver(void* b) : base(static_cast<char*>(b)) {}
  template <typename T>
  T* take(size_t n) {
    T* p = base ? reinterpret_cast<T*>(base + off) : nullptr;
    off += (n * sizeof(T) + 255) & ~(size_t)255;
    return p;
  }
};

#pragma GCC visibility pop

}  // namespace meft
