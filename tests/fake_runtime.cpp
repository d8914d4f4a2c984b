// A CUDA runtime of a test's own, for the host code of one object file without a GPU: it writes down what is launched, and says of clusters
// what the test told it.
#include <cuda_runtime.h>

#include "../paper_2503_08154_b200/csrc/s2a_launch.h"

namespace {
int g_device = 0, g_clusters[128], g_asked = 0, g_error = 0, g_count = 0;
unsigned g_grids[16];
const void* g_cluster_kernel[2];  // the kernels that a cluster was asked for
bool in_clusters(const void* f) { return f == g_cluster_kernel[0] || f == g_cluster_kernel[1]; }
}  // namespace

extern "C" {
void** __cudaRegisterFatBinary(void*) { static void* handle; return &handle; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char*, char*, const char*, int, uint3*, uint3*, dim3*, dim3*, int*) {}
void __cudaRegisterVar(void**, char*, char*, const char*, int, size_t, int, int) {}
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, void*) { return 1; }
cudaError_t __cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return cudaErrorUnknown; }
cudaError_t __cudaGetKernel(cudaKernel_t*, const void*) { return cudaErrorUnknown; }
cudaError_t __cudaLaunchKernel(cudaKernel_t, dim3, dim3, void**, size_t, cudaStream_t) { return cudaErrorUnknown; }
cudaError_t cudaLaunchKernel(const void*, dim3, dim3, void**, size_t, cudaStream_t) { return cudaErrorUnknown; }

cudaError_t cudaGetDevice(int* device) { *device = g_device; return cudaSuccess; }
cudaError_t cudaGetLastError() { const int e = g_error; g_error = 0; return (cudaError_t)e; }
// leave for clusters beyond the portable size is what tells their kernels from the others here
cudaError_t cudaFuncSetAttribute(const void* f, cudaFuncAttribute, int) {
  if (!in_clusters(f)) g_cluster_kernel[g_cluster_kernel[0] != nullptr] = f;
  return cudaSuccess;
}
cudaError_t cudaOccupancyMaxActiveClusters(int* n, const void*, const cudaLaunchConfig_t*) {
  ++g_asked;
  *n = 0;
  if (g_clusters[g_device] < 0) return (cudaError_t)(g_error = cudaErrorInvalidClusterSize);
  *n = g_clusters[g_device];
  return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* f, void**) {
  if (in_clusters(f) && g_clusters[g_device] <= 0) return (cudaError_t)(g_error = cudaErrorInvalidClusterSize);
  if (g_count < 16) g_grids[g_count++] = c->gridDim.x;
  return cudaSuccess;
}

// A gradients' norm over n_chunks single blocks on `device`, where `clusters` of them fit at once (below 0: the question fails).
// Returns the launches, whose grids are in `grids`, or below 0 the error; *asked: questions so far.
int run_grad_norm(int device, int clusters, int gdt, unsigned n_chunks, unsigned* grids, int* asked) {
  g_device = device;
  g_clusters[device] = clusters;
  g_count = 0;
  s2a::StepArgs a = {};
  a.n_chunks = n_chunks;
  a.chunk_blocks = 1;
  const cudaError_t e = s2a::launch_grad_norm(gdt, a, 1.0f, nullptr, nullptr, nullptr);
  for (int i = 0; i < g_count; ++i) grids[i] = g_grids[i];
  *asked = g_asked;
  return e != cudaSuccess ? -(int)e : (g_error ? -g_error : g_count);
}
}

namespace s2a {
int sm_count() { return 148; }
}
