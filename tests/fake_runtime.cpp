// Stands in for the CUDA runtime under libfls.so's entry points, so that what they refuse and what they would launch can be
// seen on a machine without a GPU.  Nothing runs: launches and clears are written down.
//   An address says whose memory it is: bits 44..47 are the device, 15 is host memory.
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <cstring>

#include "fls_head.h"

namespace {
struct Launch { uint64_t grid[3], block[3]; };
Launch launches[1024];
int n_launches = 0, n_clears = 0, device = 0;
uint64_t cleared[64][2];
fls::HeadCall first_call;
CUresult encode(...) { return CUDA_SUCCESS; }
}  // namespace

extern "C" {

int fake_launches() { return n_launches; }
const uint64_t* fake_grid(int i) { return launches[i].grid; }
int fake_clears() { return n_clears; }
const uint64_t* fake_cleared(int i) { return cleared[i]; }
void fake_reset(int current_device) { n_launches = n_clears = 0; device = current_device; }
// of the first launch of a head's call
uint32_t fake_group_m() { return first_call.group_m; }

cudaError_t cudaGetDevice(int* d) { *d = device; return cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaPointerGetAttributes(cudaPointerAttributes* a, const void* p) {
  const int owner = int((reinterpret_cast<uintptr_t>(p) >> 44) & 15);
  a->type = owner == 15 ? cudaMemoryTypeHost : cudaMemoryTypeDevice;
  a->device = owner == 15 ? 0 : owner;
  return cudaSuccess;
}
cudaError_t cudaMemsetAsync(void* p, int, size_t bytes, cudaStream_t) {
  cleared[n_clears][0] = reinterpret_cast<uintptr_t>(p);
  cleared[n_clears++][1] = bytes;
  return cudaSuccess;
}
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t cudaOccupancyMaxActiveClusters(int* n, const void*, const cudaLaunchConfig_t*) { *n = 74; return cudaSuccess; }
#undef cudaGetDriverEntryPoint
cudaError_t cudaGetDriverEntryPoint(const char*, void** f, unsigned long long, cudaDriverEntryPointQueryResult* q) {
  *f = reinterpret_cast<void*>(&encode);
  if (q) *q = cudaDriverEntryPointSuccess;
  return cudaSuccess;
}
// The limits of a launch: 2^31 - 1 blocks along x, 65535 along y and z, 1024 threads.
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void*, void** args) {
  const dim3 g = c->gridDim, b = c->blockDim;
  if (!g.x || !g.y || !g.z || g.x > 0x7FFFFFFFu || g.y > 65535 || g.z > 65535 || b.x * b.y * b.z > 1024) return cudaErrorInvalidConfiguration;
  if (n_launches == 0 && args && b.x <= 256 && c->numAttrs == 0) std::memcpy(&first_call, args[0], sizeof first_call);
  if (n_launches == 1024) return cudaErrorUnknown;
  launches[n_launches++] = {{g.x, g.y, g.z}, {b.x, b.y, b.z}};
  return cudaSuccess;
}

}  // extern "C"
