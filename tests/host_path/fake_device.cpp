// A stand-in for the CUDA runtime under csrc/fp8_gemm.cu (with ask_matmul.cu): devices with given numbers of SMs and of clusters that run at once, and the last
// launch that was asked for.  Nothing runs; pointers are never followed.
#include <cuda.h>
#include <cuda_runtime_api.h>
#include <cstring>
#include <map>
#include <string>

struct Device { int sms, clusters[4]; };                    // clusters of 1, 2, 4, 8 CTAs
struct Launch { char kernel[128]; int grid, cluster, threads; };
extern "C" {
Device fake_devices[8];
int fake_device;                                            // the current one
int fake_sms() { return fake_devices[fake_device].sms; }
Launch last_launch;
long launches;
}

static std::map<const void*, std::string>& names() { static std::map<const void*, std::string> n; return n; }
static CUresult encode(CUtensorMap* m, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                       CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill) {
  std::memset(m, 0, sizeof(*m));
  return CUDA_SUCCESS;
}

extern "C" {
cudaError_t cudaGetDevice(int* d) { *d = fake_device; return cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t cudaFuncGetAttributes(cudaFuncAttributes* a, const void*) { std::memset(a, 0, sizeof(*a)); a->numRegs = 168; return cudaSuccess; }
cudaError_t cudaOccupancyMaxActiveClusters(int* n, const void*, const cudaLaunchConfig_t* c) {
  const int size = (int)c->attrs[0].val.clusterDim.x;
  *n = fake_devices[fake_device].clusters[size == 8 ? 3 : size == 4 ? 2 : size == 2 ? 1 : 0];
  return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* kernel, void**) {
  ++launches;
  last_launch = {"", (int)c->gridDim.x, 1, (int)c->blockDim.x};
  std::strncpy(last_launch.kernel, names()[kernel].c_str(), sizeof(last_launch.kernel) - 1);
  for (unsigned i = 0; i < c->numAttrs; ++i)
    if (c->attrs[i].id == cudaLaunchAttributeClusterDimension) last_launch.cluster = (int)c->attrs[i].val.clusterDim.x;
  return cudaSuccess;
}
cudaError_t cudaGetDriverEntryPoint(const char*, void** p, unsigned long long, cudaDriverEntryPointQueryResult* q) {
  *p = reinterpret_cast<void*>(encode);
  *q = cudaDriverEntryPointSuccess;
  return cudaSuccess;
}
// registration of the device code, for the kernels' names
void** __cudaRegisterFatBinary(void*) { static void* h; return &h; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterVar(void**, char*, char*, const char*, int, size_t, int, int) {}
void __cudaRegisterFunction(void**, const char* host, char*, const char* name, int, uint3*, uint3*, dim3*, dim3*, int*) { names()[host] = name; }
char __cudaInitModule(void**) { return 1; }
cudaError_t cudaLaunchKernel(const void*, dim3, dim3, void**, size_t, cudaStream_t) { return cudaErrorUnknown; }
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, cudaStream_t) { return 1; }
cudaError_t __cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return cudaErrorUnknown; }
cudaError_t __cudaLaunchKernel(void*, dim3, dim3, void**, size_t, cudaStream_t) { return cudaErrorUnknown; }
cudaError_t __cudaGetKernel(void** k, const void*) { *k = nullptr; return cudaErrorUnknown; }
}
