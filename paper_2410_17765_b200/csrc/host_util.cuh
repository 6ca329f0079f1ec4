// Host-side helpers shared by the entry points: alignment, device properties, per-stage timing, launches.
#pragma once
#include <cuda_runtime.h>
#include <cstddef>
#include <cstdint>
#include <mutex>
#include <vector>

#include "../../include/cpmtp.h"

namespace cpmtp {

constexpr size_t kAlign = 256;

inline size_t align_up(size_t v, size_t a = kAlign) { return (v + a - 1) / a * a; }

struct DeviceInfo {
  int sms = 0;
  int cc_major = 0;
  bool ok = false;
};

// One lock for the small per-process caches below (device properties, kernel attributes, tensor maps,
// the static scratch address).  Host-side only and held for microseconds; calls from several threads are safe.
inline std::mutex g_cache_mutex;

// Cached per device ordinal; filled on first use with that device current.
inline DeviceInfo* device_info() {
  static DeviceInfo infos[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
  std::lock_guard<std::mutex> lock(g_cache_mutex);
  DeviceInfo& di = infos[dev];
  if (!di.ok) {
    if (cudaDeviceGetAttribute(&di.sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return nullptr;
    if (cudaDeviceGetAttribute(&di.cc_major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess)
      return nullptr;
    di.ok = true;
  }
  return &di;
}

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// How long a wait inside a kernel may last, and the test hook that leaves out a load: of the environment knobs.
struct WaitKnobs {
  unsigned limit_us;
  int skip_load;
};
WaitKnobs wait_knobs();

// Optional per-stage timing: events bracket each launch while profiling is on.
struct Profiler {
  bool on = false;
  std::vector<cudaEvent_t> events;   // start/stop pairs
  std::vector<int> stages;
};
inline Profiler g_prof;

struct ProfScope {
  cudaStream_t st;
  bool active;
  ProfScope(int stage, cudaStream_t stream) : st(stream), active(g_prof.on) {
    if (!active) return;
    cudaEvent_t a, b;
    if (cudaEventCreate(&a) != cudaSuccess || cudaEventCreate(&b) != cudaSuccess) { active = false; return; }
    g_prof.events.push_back(a);
    g_prof.events.push_back(b);
    g_prof.stages.push_back(stage);
    cudaEventRecord(a, st);
  }
  ~ProfScope() {
    if (active) cudaEventRecord(g_prof.events.back(), st);
  }
};

// Dynamic shared memory above 48 KB has to be allowed once per kernel and device.
template <class K>
cudaError_t allow_smem(K* kernel, bool (&done)[64], int bytes) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(g_cache_mutex);
  if (done[dev]) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  done[dev] = e == cudaSuccess;
  return e;
}

// The device that the caller has made current, if this library runs on it.
inline int check_device(DeviceInfo** out) {
  DeviceInfo* di = device_info();
  if (di == nullptr) return CPMTP_ERR_LAUNCH;
  if (di->cc_major != 10) return CPMTP_ERR_ARCH;
  *out = di;
  return CPMTP_OK;
}

// The current device's number of SMs; without a device that of the one this is written for.
inline int sm_count() {
  const DeviceInfo* di = device_info();
  return di != nullptr && di->sms > 0 ? di->sms : 148;
}

// Launch with programmatic stream serialization: the kernel may be scheduled while the one before it in
// the stream drains; it calls ptx::grid_dep_wait() before it touches anything that kernel produced.
// `cluster`: blocks to a thread-block cluster.
template <class... KArgs, class... Args>
cudaError_t launch_clusters(int cluster, void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}
template <class... KArgs, class... Args>
cudaError_t launch_pdl(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream,
                       const Args&... args) {
  return launch_clusters(1, kernel, grid, block, smem, stream, args...);
}

#define CPMTP_TRY(expr)                         \
  do {                                          \
    if ((expr) != cudaSuccess) return CPMTP_ERR_LAUNCH; \
  } while (0)

}  // namespace cpmtp
