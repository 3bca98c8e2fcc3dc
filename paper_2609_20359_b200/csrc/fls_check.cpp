// Checks of the buffers that a call is given.
#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdio>

#include "fls_internal.h"

namespace fls {

int refuse(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  set_last_error(buf);
  return code;
}

int check_spans(const Span* s, int n) {
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess) { cudaGetLastError(); device = -1; }
  for (int i = 0; i < n; ++i) {
    if (!s[i].p) {
      if (s[i].bytes) return refuse(FLS_EPTR, "%s is null", s[i].what);
      continue;
    }
    if (reinterpret_cast<uintptr_t>(s[i].p) % s[i].align)
      return refuse(FLS_EALIGN, "%s must start on a %llu-byte boundary", s[i].what, (unsigned long long)s[i].align);
    if (!s[i].bytes) continue;
    cudaPointerAttributes at{};
    const cudaError_t e = cudaPointerGetAttributes(&at, s[i].p);
    if (e != cudaSuccess) {
      cudaGetLastError();
      return refuse(FLS_ECUDA, "cudaPointerGetAttributes: %s", cudaGetErrorString(e));
    }
    if (at.type != cudaMemoryTypeDevice && at.type != cudaMemoryTypeManaged) return refuse(FLS_EPTR, "%s is not device memory", s[i].what);
    if (at.type == cudaMemoryTypeDevice && at.device != device)
      return refuse(FLS_EPTR, "%s is on device %d, not the current one", s[i].what, at.device);
  }
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < n; ++j) {
      if (i == j || !s[i].output || (s[j].output && j < i) || !s[i].bytes || !s[j].bytes) continue;
      const uintptr_t a = reinterpret_cast<uintptr_t>(s[i].p), b = reinterpret_cast<uintptr_t>(s[j].p);
      if (a < b + s[j].bytes && b < a + s[i].bytes) return refuse(FLS_EPTR, "%s overlaps %s", s[i].what, s[j].what);
    }
  return FLS_OK;
}

}  // namespace fls
