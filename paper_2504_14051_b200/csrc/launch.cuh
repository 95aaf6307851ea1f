// What every entry point needs on the host: error text, launch counting and tracing, launches with programmatic
// serialisation, the device check, tensor maps' encoder. Shared by the library's translation units.
#pragma once

#include <cuda.h>

#include <atomic>
#include <cstdio>
#include <cstring>
#include <mutex>
#include <utility>
#include <vector>

#include "common.cuh"

namespace caote {

inline std::atomic<long long> g_launches{0};
inline thread_local char g_cuda_error[256] = "";

inline int cuda_fail(cudaError_t e, const char* what) {
  snprintf(g_cuda_error, sizeof(g_cuda_error), "%s: %s", what, cudaGetErrorString(e));
  return CAOTE_ERR_CUDA;
}
#define CAOTE_CUDA(call)                                  \
  do {                                                    \
    cudaError_t e__ = (call);                             \
    if (e__ != cudaSuccess) return cuda_fail(e__, #call); \
  } while (0)

inline int after_launch(const char* name) {
  g_launches.fetch_add(1, std::memory_order_relaxed);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return cuda_fail(e, name);
  return CAOTE_OK;
}

// ---- optional per-kernel tracing: CUDA events recorded on the launching stream around each kernel ----
struct TraceRec {
  const char* name;
  cudaEvent_t a, b;
};
inline std::atomic<bool> g_trace_on{false};
inline std::mutex g_trace_mu;
inline std::vector<TraceRec> g_trace_pending;
inline std::vector<cudaEvent_t> g_trace_pool;

inline cudaEvent_t trace_event() {
  std::lock_guard<std::mutex> lk(g_trace_mu);
  if (!g_trace_pool.empty()) {
    cudaEvent_t e = g_trace_pool.back();
    g_trace_pool.pop_back();
    return e;
  }
  cudaEvent_t e = nullptr;
  if (cudaEventCreate(&e) != cudaSuccess) return nullptr;
  return e;
}

struct TraceScope {
  const char* name;
  cudaStream_t st;
  cudaEvent_t a = nullptr, b = nullptr;
  TraceScope(const char* n, cudaStream_t s) : name(n), st(s) {
    if (!g_trace_on.load(std::memory_order_relaxed)) return;
    a = trace_event();
    b = trace_event();
    if (a && b) cudaEventRecord(a, st);
  }
  ~TraceScope() {
    if (!a || !b) return;
    cudaEventRecord(b, st);
    std::lock_guard<std::mutex> lk(g_trace_mu);
    g_trace_pending.push_back({name, a, b});
  }
};

// Launch a kernel (the statement after the stream argument), count it, trace it when tracing is on,
// and return from the calling function if the launch failed.
#define CAOTE_LAUNCH(name, st, ...)        \
  do {                                     \
    int rc__;                              \
    {                                      \
      TraceScope ts__(name, st);           \
      __VA_ARGS__;                         \
      rc__ = after_launch(name);           \
    }                                      \
    if (rc__ != CAOTE_OK) return rc__;     \
  } while (0)

// Launch with the programmatic-serialization attribute: the kernel may be scheduled while its predecessor in the
// stream is still running and waits for it in its first statement (ptx::pdl_wait). Only for kernels that do so.
// cluster > 1: in clusters of that many CTAs along x.
template <typename... KArgs, typename... Args>
inline void launch_pdl_clusters(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t st,
                                Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)cluster;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  (void)cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);  // (errors are picked up by after_launch)
}
template <typename... KArgs, typename... Args>
inline void launch_pdl(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args&&... args) {
  launch_pdl_clusters(kernel, grid, block, smem, 1, st, std::forward<Args>(args)...);
}

// The device must be a compute-capability 10.x part; checked once per device.
inline int check_device() {
  static std::atomic<int> ok[64];
  int dev = 0;
  CAOTE_CUDA(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64) return CAOTE_ERR_UNSUPPORTED;
  int st = ok[dev].load(std::memory_order_acquire);
  if (st == 0) {
    int major = 0;
    CAOTE_CUDA(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev));
    st = (major == 10) ? 1 : -1;
    ok[dev].store(st, std::memory_order_release);
  }
  return st == 1 ? CAOTE_OK : CAOTE_ERR_UNSUPPORTED;
}

// Once per device, kernel and size, not at every launch.
template <typename KernelT>
inline int allow_smem(KernelT kernel, size_t bytes) {
  if (bytes <= 48 * 1024) return CAOTE_OK;
  struct Done { int dev; const void* kernel; size_t bytes; };
  static std::mutex mu;
  static std::vector<Done> done;
  int dev = 0;
  CAOTE_CUDA(cudaGetDevice(&dev));
  std::lock_guard<std::mutex> lk(mu);
  for (Done& d : done)
    if (d.dev == dev && d.kernel == (const void*)kernel) {
      if (d.bytes >= bytes) return CAOTE_OK;
      CAOTE_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
      d.bytes = bytes;
      return CAOTE_OK;
    }
  CAOTE_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
  done.push_back({dev, (const void*)kernel, bytes});
  return CAOTE_OK;
}

typedef CUresult (*TensorMapEncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                      const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                      CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline TensorMapEncodeFn tensor_map_encoder() {
  static std::atomic<TensorMapEncodeFn> fn{nullptr};
  TensorMapEncodeFn f = fn.load(std::memory_order_acquire);
  if (!f) {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult qr;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &qr) == cudaSuccess &&
        qr == cudaDriverEntryPointSuccess)
      f = reinterpret_cast<TensorMapEncodeFn>(ptr);
    fn.store(f, std::memory_order_release);
  }
  return f;
}

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// The split heuristics of the prefill and any-shape paths look at the SM count: keep it current for this device
// (cached per device; left at its default when there is no device, e.g. when only sizes are asked for).
inline void refresh_sm_count() {
  static std::atomic<int> cached[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    (void)cudaGetLastError();
    return;
  }
  int n = cached[dev].load(std::memory_order_acquire);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) {
      (void)cudaGetLastError();
      return;
    }
    cached[dev].store(n, std::memory_order_release);
  }
  g_sm_count = n;
}

}  // namespace caote
