// Host-side helpers shared by the translation units of the library: device queries, buffer layout, launches and their
// bookkeeping.  The state (launch counter, trace, failed-launch flag) is one instance for the whole library.
#pragma once
#include <atomic>
#include <mutex>
#include <unordered_map>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/laplace_nystrom.h"

namespace ln {
namespace host {

// Number of SMs of the current device (asked once per device; 148 on a B200, the fallback if the query fails).
constexpr int kMaxDevices = 64;
inline int sm_count() {
  static std::atomic<int> cached[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 148;
  int v = cached[dev].load(std::memory_order_relaxed);
  if (v <= 0) {
    if (cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || v <= 0) { cudaGetLastError(); v = 148; }
    cached[dev].store(v, std::memory_order_relaxed);
  }
  return v;
}

// cudaFuncSetAttribute(MaxDynamicSharedMemorySize) once per kernel and device (again only when a larger size is
// asked for): a table keyed by the kernel's address.
template <typename K>
inline void want_smem(K kern, size_t smem) {
  static std::mutex mu;
  static std::unordered_map<const void*, int> have[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) dev = 0;
  const void* id = reinterpret_cast<const void*>(kern);
  std::lock_guard<std::mutex> lk(mu);
  auto it = have[dev].find(id);
  if (it != have[dev].end() && it->second >= (int)smem) return;
  cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  have[dev][id] = (int)smem;
}

template <typename A0, typename... R> A0 arg0(void (*)(A0, R...));   // first parameter type of a kernel (declaration only)
inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Bump allocator over a caller-provided buffer; with base == nullptr it only measures.
struct Carver {
  char* base; size_t off;
  explicit Carver(void* b) : base(static_cast<char*>(b)), off(0) {}
  float* take(size_t nfloats) {
    float* p = base ? reinterpret_cast<float*>(base + off) : nullptr;
    off += align_up(nfloats * sizeof(float), 256);
    return p;
  }
};

// A launch that fails is noticed right after it (a later successful call may otherwise hide it) and reported by the
// entry point when it returns.
inline thread_local bool g_launch_failed = false;
inline std::atomic<unsigned long long> g_launch_count{0};      // kernels launched by this library since it was loaded
inline void note_launch() {
  g_launch_count.fetch_add(1, std::memory_order_relaxed);
  if (cudaPeekAtLastError() != cudaSuccess) g_launch_failed = true;
}
inline int launch_ok() {
  const bool bad = (cudaGetLastError() != cudaSuccess) || g_launch_failed;
  g_launch_failed = false;
  return bad ? LN_ERR_CUDA : LN_OK;
}
inline unsigned cdiv(long long a, long long b) { return (unsigned)((a + b - 1) / b); }

// Profiling aid: when switched on by ln_trace_begin every launch is bracketed by two CUDA events
// on its stream.  Off by default; the product path never touches it.
constexpr int kTraceCap = 2048;
struct Trace {
  std::atomic<bool> on{false};
  int count = 0;
  cudaEvent_t ev[2 * kTraceCap];
  const char* name[kTraceCap];
};
inline Trace g_trace;
struct TraceScope {
  cudaStream_t st; int slot;
  TraceScope(const char* name, cudaStream_t s) : st(s), slot(-1) {
    if (g_trace.on && g_trace.count < kTraceCap) {
      slot = g_trace.count++;
      g_trace.name[slot] = name;
      cudaEventRecord(g_trace.ev[2 * slot], st);
    }
  }
  ~TraceScope() { if (slot >= 0) cudaEventRecord(g_trace.ev[2 * slot + 1], st); }
};
#define LN_LAUNCH(name, st, ...) do { ln::host::TraceScope ts_(name, st); __VA_ARGS__; ln::host::note_launch(); } while (0)

// Every kernel is launched as a programmatic dependent of the one before it on its stream (see pdl_wait in
// ln_common.cuh): the launch of a kernel overlaps the end of the one before.
inline cudaLaunchAttribute early_launch() {
  cudaLaunchAttribute a = {};
  a.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  a.val.programmaticStreamSerializationAllowed = 1;
  return a;
}
template <typename... KArgs, typename... Args>
void enqueue(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute at = early_launch();
  cfg.attrs = &at; cfg.numAttrs = 1;
  cudaLaunchKernelEx(&cfg, kern, KArgs(args)...);
}

}  // namespace host
}  // namespace ln
