// Stands in for the CUDA runtime calls that a kernel launch makes (preloaded before the library; no GPU): two
// devices with different room for CTA pairs, and the runtime's rule that a kernel needs its shared-memory attribute on every
// device before a launch above 48 KB. Nothing is launched.
#include <cuda.h>
#include <cuda_runtime_api.h>
#include <time.h>

#include <algorithm>
#include <atomic>
#include <map>
#include <mutex>
#include <utility>

namespace {
thread_local int g_device = 0;
thread_local cudaError_t g_error = cudaSuccess;
std::mutex g_mu;
std::map<std::pair<int, const void *>, int> g_smem;
std::atomic<int> g_launches{0}, g_widest{0}, g_entry_ms{0};

cudaError_t smem_ok(const void *func, size_t bytes) {
  std::lock_guard<std::mutex> g(g_mu);
  if (bytes <= 48 * 1024) return cudaSuccess;
  auto it = g_smem.find({g_device, func});
  return it != g_smem.end() && bytes <= size_t(it->second) ? cudaSuccess : cudaErrorInvalidValue;
}
int clusters_of(int device) { return device == 0 ? 70 : 60; }

CUresult encode(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                CUtensorMapFloatOOBfill) {
  return CUDA_SUCCESS;
}
}  // namespace

extern "C" {

// The test's side: the calling thread's device; launches so far, and the most CTAs of one with clusters (both
// set back); how long a look-up of a driver function takes.
void fake_use_device(int device) { g_device = device; }
int fake_launches() { return g_launches.exchange(0); }
int fake_widest_cluster_grid() { return g_widest.exchange(0); }
int fake_clusters(int device) { return clusters_of(device); }
void fake_entry_point_ms(int ms) { g_entry_ms = ms; }

cudaError_t cudaGetDevice(int *device) {
  *device = g_device;
  return cudaSuccess;
}
cudaError_t cudaDeviceGetAttribute(int *value, cudaDeviceAttr, int) {
  *value = 152;
  return cudaSuccess;
}
cudaError_t cudaDeviceGetStreamPriorityRange(int *least, int *greatest) {
  *least = 0;
  *greatest = -5;
  return cudaSuccess;
}
cudaError_t cudaGetLastError() { return std::exchange(g_error, cudaSuccess); }
cudaError_t cudaFuncSetAttribute(const void *func, cudaFuncAttribute attr, int value) {
  std::lock_guard<std::mutex> g(g_mu);
  if (attr == cudaFuncAttributeMaxDynamicSharedMemorySize) g_smem[{g_device, func}] = value;
  return cudaSuccess;
}
cudaError_t cudaOccupancyMaxActiveClusters(int *n, const void *func, const cudaLaunchConfig_t *cfg) {
  *n = clusters_of(g_device);
  return smem_ok(func, cfg->dynamicSmemBytes);
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *cfg, const void *func, void **) {
  const cudaError_t e = smem_ok(func, cfg->dynamicSmemBytes);
  if (e != cudaSuccess) return g_error = e;
  ++g_launches;
  for (unsigned i = 0; i < cfg->numAttrs; ++i)
    if (cfg->attrs[i].id == cudaLaunchAttributeClusterDimension) g_widest = std::max(g_widest.load(), int(cfg->gridDim.x));
  return cudaSuccess;
}
cudaError_t cudaGetDriverEntryPointByVersion(const char *, void **fn, unsigned int, unsigned long long,
                                             cudaDriverEntryPointQueryResult *q) {
  timespec t{g_entry_ms / 1000, (g_entry_ms % 1000) * 1000000L};
  nanosleep(&t, nullptr);
  *fn = reinterpret_cast<void *>(encode);
  *q = cudaDriverEntryPointSuccess;
  return cudaSuccess;
}

}  // extern "C"
