// Stands in for the CUDA runtime's calls of a cluster launch, in a process without
// a GPU: two devices whose kernels' attributes are each their own, and launches
// that are looked at instead of made. Preloaded ahead of the runtime.
#include <cuda_runtime_api.h>

#include <set>
#include <utility>

namespace {
int device = 0, launches = 0, last_cluster = 0, last_grid = 0;
std::set<std::pair<int, const void *>> large;  // (device, kernel) that may use large clusters

int cluster_of(const cudaLaunchConfig_t *c) {
  for (unsigned x = 0; x < c->numAttrs; ++x)
    if (c->attrs[x].id == cudaLaunchAttributeClusterDimension)
      return (int)c->attrs[x].val.clusterDim.x;
  return 1;
}
bool refused(const cudaLaunchConfig_t *c, const void *f) {
  return cluster_of(c) > 8 && !large.count({device, f});
}
}  // namespace

extern "C" {
void fake_set_device(int d) { device = d; }
int fake_launches() { return launches; }
int fake_cluster() { return last_cluster; }
int fake_grid() { return last_grid; }

cudaError_t cudaGetDevice(int *d) {
  *d = device;
  return cudaSuccess;
}
cudaError_t cudaDeviceGetAttribute(int *v, cudaDeviceAttr attr, int) {
  *v = attr == cudaDevAttrComputeCapabilityMajor ? 10
       : attr == cudaDevAttrComputeCapabilityMinor ? 3 : 152;
  return cudaSuccess;
}
cudaError_t cudaFuncSetAttribute(const void *f, cudaFuncAttribute attr, int v) {
  if (attr == cudaFuncAttributeNonPortableClusterSizeAllowed && v) large.insert({device, f});
  return cudaSuccess;
}
cudaError_t cudaOccupancyMaxActiveClusters(int *n, const void *f, const cudaLaunchConfig_t *c) {
  if (refused(c, f)) return cudaErrorInvalidClusterSize;
  *n = device == 0 ? 9 : 2;
  return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *c, const void *f, void **) {
  if (refused(c, f)) return cudaErrorInvalidClusterSize;
  ++launches;
  last_cluster = cluster_of(c);
  last_grid = (int)c->gridDim.x;
  return cudaSuccess;
}
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaPeekAtLastError() { return cudaSuccess; }
}
