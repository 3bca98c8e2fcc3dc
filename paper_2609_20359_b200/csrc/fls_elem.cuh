// What the embedding and norm kernels share: elements of activations, weights and gradients, bf16 (as its bits) or fp32, moved
// one at a time or in cells of eight neighbouring columns (a 128-bit access of bf16, a 256-bit one of fp32; two 128-bit
// accesses 32 bytes apart from lane to lane would fetch and store every 32-byte sector twice), and their launches.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

namespace fls {

__device__ __forceinline__ void pdl_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Two fp32 operations in one instruction.
struct f2 { uint64_t v; };
__device__ __forceinline__ f2 make_f2(float a, float b) {
  f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ f2 make_f2(float a) { return make_f2(a, a); }
__device__ __forceinline__ void split(f2 x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x.v)); }
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ float sum2(f2 x) {
  float a, b;
  split(x, a, b);
  return a + b;
}
__device__ __forceinline__ void pairs_of(const float (&x)[8], f2 (&y)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = make_f2(x[2 * i], x[2 * i + 1]);
}
__device__ __forceinline__ void singles_of(const f2 (&x)[4], float (&y)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) split(x[i], y[2 * i], y[2 * i + 1]);
}

template <typename T> struct Elem;
template <> struct Elem<uint16_t> {
  __device__ static __forceinline__ float get(const uint16_t* p) { return __uint_as_float(uint32_t(*p) << 16); }
  __device__ static __forceinline__ void put(uint16_t* p, float x) { *p = __bfloat16_as_ushort(__float2bfloat16_rn(x)); }
  __device__ static __forceinline__ float round(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }
  using Raw = uint4;                                       // a cell as it lies in memory
  __device__ static __forceinline__ Raw load_raw(const uint16_t* p) { return *reinterpret_cast<const uint4*>(p); }
  __device__ static __forceinline__ void unpack(const Raw& r, float (&x)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  }
  __device__ static __forceinline__ void store8(uint16_t* p, const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <> struct Elem<float> {
  __device__ static __forceinline__ float get(const float* p) { return *p; }
  __device__ static __forceinline__ void put(float* p, float x) { *p = x; }
  __device__ static __forceinline__ float round(float x) { return x; }
  struct Raw { float4 a, b; };
  __device__ static __forceinline__ Raw load_raw(const float* p) {
    Raw r;
    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(r.a.x), "=f"(r.a.y), "=f"(r.a.z), "=f"(r.a.w), "=f"(r.b.x), "=f"(r.b.y), "=f"(r.b.z), "=f"(r.b.w)
                 : "l"(p)
                 : "memory");
    return r;
  }
  __device__ static __forceinline__ void unpack(const Raw& r, float (&x)[8]) {
    x[0] = r.a.x; x[1] = r.a.y; x[2] = r.a.z; x[3] = r.a.w;
    x[4] = r.b.x; x[5] = r.b.y; x[6] = r.b.z; x[7] = r.b.w;
  }
  __device__ static __forceinline__ void store8(float* p, const float (&x)[8]) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]),
                 "f"(x[5]), "f"(x[6]), "f"(x[7])
                 : "memory");
  }
};

// An asynchronous copy of 16 bytes to shared memory; zeros where `there` is false.
__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ uint4 shared16(uint32_t from) {
  uint4 x;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(from) : "memory");
  return x;
}

// The cells of a warp's 32 lanes on their way through shared memory: P 16-byte pieces of each, 32 P in a row.  The warp
// copies them in order, every sector once; a lane then reads its own cell, which other lanes have copied (hence the
// __syncwarp between waiting for the copies and reading, and between reading and copying again).  For P = 2 neighbouring pieces are swapped in
// every second group of eight, so that neither access meets a bank twice.
template <typename T> struct Staged {
  static constexpr int P = sizeof(T) / 2;
  static constexpr uint32_t bytes = P * 512;                // of a warp
  __device__ static __forceinline__ uint32_t place(uint32_t q) { return (P == 2 ? q ^ (q >> 3 & 1) : q) * 16; }
  // first: the column of lane 0's cell
  __device__ static __forceinline__ void copy(uint32_t to, const T* row, uint32_t first, uint32_t lane, uint32_t dim) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const uint32_t q = p * 32 + lane, col = first + q * (16 / sizeof(T));
      copy16(to + place(q), row + (col < dim ? col : 0), col < dim);
    }
  }
  __device__ static __forceinline__ void read(uint32_t from, uint32_t lane, typename Elem<T>::Raw& raw) {
#pragma unroll
    for (int p = 0; p < P; ++p) reinterpret_cast<uint4*>(&raw)[p] = shared16(from + place(lane * P + p));
  }
};

// ------------------------------------------------------------------------------------------------ host
// Whether every row starts on a boundary of eight elements, as cells ask for.
inline bool in_cells(const void* p, uint64_t stride, uint64_t elem) { return reinterpret_cast<uintptr_t>(p) % (8 * elem) == 0 && stride % 8 == 0; }

// Lets a kernel have `bytes` of dynamic shared memory, once per device and kernel.
inline cudaError_t allow_shared(const void* kernel, int bytes, std::atomic<uint64_t>& done) {
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  const uint64_t bit = device < 64 ? 1ull << device : 0;
  if (bit & done.load(std::memory_order_acquire)) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
  return e;
}

// dependent: the kernel may start before the one ahead of it is done (it waits with pdl_wait for what it needs of that one).
template <typename... P, typename... A>
cudaError_t launch_clusters(void (*kernel)(P...), dim3 grid, uint32_t cluster, uint32_t threads, uint32_t smem, bool dependent, cudaStream_t s,
                            const A&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[2] = {};
  if (dependent) {
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
  }
  if (cluster > 1) {
    at[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    at[cfg.numAttrs].val.clusterDim.x = cluster;
    at[cfg.numAttrs].val.clusterDim.y = at[cfg.numAttrs].val.clusterDim.z = 1;
    ++cfg.numAttrs;
  }
  cfg.attrs = at;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}
template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, uint32_t threads, uint32_t smem, bool dependent, cudaStream_t s, const A&... args) {
  return launch_clusters(kernel, grid, 1, threads, smem, dependent, s, args...);
}

}  // namespace fls
