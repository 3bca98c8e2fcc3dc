// fls_norm_*: layer norm and root mean square norm of rows, with the residual addition before it, and the backward pass with
// the sums of the weight's and the bias's gradient.
//
// Forward, per row s of d values: m = mean(s) in fp32, then e = mean(s - m) and q = mean((s - m)^2) in a second look at the
// values, which takes the rounding of m out of the result: mean = m + e, variance = q - e^2.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>

#include "fls.h"
#include "fls_elem.cuh"
#include "fls_internal.h"

using namespace fls;

namespace {

constexpr uint32_t kColTile = 32;          // columns of a CTA of the weight gradients' kernel
constexpr uint32_t kMaxParts = 296;        // parts of the rows whose sums are joined

constexpr uint64_t up(uint64_t x, uint64_t q) { return (x + q - 1) / q * q; }

struct NormCall {
  const void *x, *residual, *weight, *bias;
  void *y, *total;
  float *mean, *rstd;                      // forward: outputs or null
  const float *mean_in, *rstd_in;
  const void *grad_y, *grad_total;
  void *grad_x, *grad_weight, *grad_bias;
  uint64_t x_stride, residual_stride, y_stride, total_stride, grad_y_stride, grad_total_stride, grad_x_stride;
  uint64_t rows;
  uint32_t dim, dp;
  uint32_t rms, weight_f32, grad_f32, accumulate;
  float eps, inv_dim;
  float2* coef;                            // [rows]: mean(g) and mean(g xhat)
  float* part;                             // [parts][2][dp]
  uint32_t parts;
};

__device__ __forceinline__ float weight_at(const NormCall& c, const void* p, uint32_t j) {
  return c.weight_f32 ? static_cast<const float*>(p)[j] : Elem<uint16_t>::get(static_cast<const uint16_t*>(p) + j);
}

// Sums over the CTA, the same for all threads and from run to run.
__device__ __forceinline__ float2 block_sum(float2 v, float2* shared) {
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, warps = blockDim.x / 32;
#pragma unroll
  for (int o = 16; o; o /= 2) {
    v.x += __shfl_xor_sync(~0u, v.x, o);
    v.y += __shfl_xor_sync(~0u, v.y, o);
  }
  __syncthreads();
  if (lane == 0) shared[warp] = v;
  __syncthreads();
  v = lane < warps ? shared[lane] : make_float2(0.f, 0.f);
#pragma unroll
  for (int o = 16; o; o /= 2) {
    v.x += __shfl_xor_sync(~0u, v.x, o);
    v.y += __shfl_xor_sync(~0u, v.y, o);
  }
  return v;
}

// A row per CTA, read again for each step.
template <typename X, typename Y>
__global__ void __launch_bounds__(256) fls_norm_rows_kernel(const __grid_constant__ NormCall c) {
  __shared__ float2 shared[32];
  for (uint64_t n = blockIdx.x; n < c.rows; n += gridDim.x) {
    const X* x = static_cast<const X*>(c.x) + n * c.x_stride;
    if (c.residual) {
      const X* r = static_cast<const X*>(c.residual) + n * c.residual_stride;
      X* t = static_cast<X*>(c.total) + n * c.total_stride;
      for (uint32_t j = threadIdx.x; j < c.dim; j += blockDim.x) Elem<X>::put(t + j, Elem<X>::get(x + j) + Elem<X>::get(r + j));
      x = t;                                             // a thread reads back only what it wrote
    }
    float m = 0.f;
    if (!c.rms) {
      float2 v = make_float2(0.f, 0.f);
      for (uint32_t j = threadIdx.x; j < c.dim; j += blockDim.x) v.x += Elem<X>::get(x + j);
      m = block_sum(v, shared).x * c.inv_dim;
    }
    float2 v = make_float2(0.f, 0.f);
    for (uint32_t j = threadIdx.x; j < c.dim; j += blockDim.x) {
      const float a = Elem<X>::get(x + j) - m;
      v.x += a;
      v.y = fmaf(a, a, v.y);
    }
    v = block_sum(v, shared);
    const float e = c.rms ? 0.f : v.x * c.inv_dim, var = fmaf(-e, e, v.y * c.inv_dim);
    const float rstd = 1.f / sqrtf(var + c.eps);
    Y* y = static_cast<Y*>(c.y) + n * c.y_stride;
    for (uint32_t j = threadIdx.x; j < c.dim; j += blockDim.x) {
      float a = ((Elem<X>::get(x + j) - m) - e) * rstd;
      if (c.weight) a *= weight_at(c, c.weight, j);
      if (c.bias) a += weight_at(c, c.bias, j);
      Elem<Y>::put(y + j, a);
    }
    if (threadIdx.x == 0) {
      if (c.mean) c.mean[n] = m + e;
      if (c.rstd) c.rstd[n] = rstd;
    }
  }
}

// mean(g) and mean(g xhat) of every row.
template <typename X, typename Y>
__global__ void __launch_bounds__(256) fls_norm_coef_kernel(const __grid_constant__ NormCall c) {
  __shared__ float2 shared[32];
  pdl_launch();
  for (uint64_t n = blockIdx.x; n < c.rows; n += gridDim.x) {
    const X* x = static_cast<const X*>(c.x) + n * c.x_stride;
    const Y* dy = static_cast<const Y*>(c.grad_y) + n * c.grad_y_stride;
    const float m = c.rms ? 0.f : c.mean_in[n], r = c.rstd_in[n];
    float2 v = make_float2(0.f, 0.f);
    for (uint32_t j = threadIdx.x; j < c.dim; j += blockDim.x) {
      float g = Elem<Y>::get(dy + j);
      if (c.weight) g *= weight_at(c, c.weight, j);
      v.x += g;
      v.y = fmaf(g, (Elem<X>::get(x + j) - m) * r, v.y);
    }
    v = block_sum(v, shared);
    if (threadIdx.x == 0) c.coef[n] = make_float2(c.rms ? 0.f : v.x * c.inv_dim, v.y * c.inv_dim);
  }
}

// 32 columns of one part of the rows, eight rows at a time: dx, and the part's sums for the weight and the bias.
template <typename X, typename Y>
__global__ void __launch_bounds__(256) fls_norm_columns_kernel(const __grid_constant__ NormCall c) {
  __shared__ float2 shared[8][kColTile];
  const uint32_t lane = threadIdx.x % 32, group = threadIdx.x / 32, j = blockIdx.x * kColTile + lane;
  const uint64_t per = (c.rows + c.parts - 1) / c.parts, begin = blockIdx.y * per, end = min(c.rows, begin + per);
  pdl_launch();
  pdl_wait();
  float2 sum = make_float2(0.f, 0.f);
  const float w = j < c.dim && c.weight ? weight_at(c, c.weight, j) : 1.f;
  for (uint64_t n = begin + group; n < end && j < c.dim; n += 8) {
    const float m = c.rms ? 0.f : c.mean_in[n], r = c.rstd_in[n];
    const float xhat = (Elem<X>::get(static_cast<const X*>(c.x) + n * c.x_stride + j) - m) * r;
    const float dy = Elem<Y>::get(static_cast<const Y*>(c.grad_y) + n * c.grad_y_stride + j);
    sum.x = fmaf(dy, xhat, sum.x);
    sum.y += dy;
    if (c.grad_x) {
      const float2 k = c.coef[n];
      float dx = (fmaf(-xhat, k.y, dy * w) - k.x) * r;
      if (c.grad_total) dx += Elem<X>::get(static_cast<const X*>(c.grad_total) + n * c.grad_total_stride + j);
      Elem<X>::put(static_cast<X*>(c.grad_x) + n * c.grad_x_stride + j, dx);
    }
  }
  shared[group][lane] = sum;
  __syncthreads();
  if (group || j >= c.dim) return;
  for (int g = 1; g < 8; ++g) { sum.x += shared[g][lane].x; sum.y += shared[g][lane].y; }
  c.part[uint64_t(2 * blockIdx.y) * c.dp + j] = sum.x;
  c.part[uint64_t(2 * blockIdx.y + 1) * c.dp + j] = sum.y;
}

// The parts' sums, in their order inside each of eight groups, then of the groups.
__global__ void __launch_bounds__(256) fls_norm_join_kernel(const __grid_constant__ NormCall c) {
  __shared__ float shared[8][kColTile];
  const uint32_t lane = threadIdx.x % 32, group = threadIdx.x / 32, j = blockIdx.x * kColTile + lane, which = blockIdx.y;
  void* out = which ? c.grad_bias : c.grad_weight;
  pdl_wait();
  if (!out) return;
  float sum = 0.f;
  for (uint32_t p = group; p < c.parts && j < c.dim; p += 8) sum += c.part[uint64_t(2 * p + which) * c.dp + j];
  shared[group][lane] = sum;
  __syncthreads();
  if (group || j >= c.dim) return;
  for (int g = 1; g < 8; ++g) sum += shared[g][lane];
  if (c.grad_f32) {
    float* o = static_cast<float*>(out) + j;
    *o = c.accumulate ? *o + sum : sum;
  } else {
    uint16_t* o = static_cast<uint16_t*>(out) + j;
    Elem<uint16_t>::put(o, c.accumulate ? Elem<uint16_t>::get(o) + sum : sum);
  }
}

template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, uint32_t threads, bool dependent, cudaStream_t s, const A&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = s;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = dependent ? 1 : 0;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

struct Regions { uint64_t coef, part, total; };
Regions regions(const fls_norm_desc& d) {
  Regions r{};
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) { const uint64_t o = at; at += up(bytes, 256); return o; };
  if (d.grads) {
    r.coef = take(std::max<uint64_t>(d.max_rows, 1) * 8);
    r.part = take(uint64_t(2) * kMaxParts * up(d.dim, 32) * 4);
  }
  r.total = at;
  return r;
}

bool known(uint32_t dtype) { return dtype == FLS_GRAD_BF16 || dtype == FLS_GRAD_F32; }
uint64_t size_of(uint32_t dtype) { return dtype == FLS_GRAD_F32 ? 4 : 2; }
uint64_t span_bytes(uint64_t rows, uint64_t cols, uint64_t stride, uint64_t elem) { return rows ? ((rows - 1) * stride + cols) * elem : 0; }

}  // namespace

struct fls_norm {
  fls_norm_desc desc{};
  Regions reg{};
  uint64_t launches = 0;
};

namespace {

#define FLS_LAUNCH(call)                                                                            \
  do {                                                                                              \
    const cudaError_t e_ = (call);                                                                  \
    if (e_ != cudaSuccess) return refuse(FLS_ECUDA, "norm kernel: %s", cudaGetErrorString(e_));     \
    ++h->launches;                                                                                  \
  } while (0)

template <typename X, typename Y>
int run_forward(fls_norm* h, const NormCall& c, cudaStream_t s) {
  FLS_LAUNCH(launch(fls_norm_rows_kernel<X, Y>, dim3(uint32_t(std::min<uint64_t>(c.rows, 148 * 64))), 256, false, s, c));
  return FLS_OK;
}

template <typename X, typename Y>
int run_backward(fls_norm* h, NormCall& c, cudaStream_t s) {
  const uint32_t tiles = (c.dim + kColTile - 1) / kColTile;
  bool dependent = false;
  c.parts = uint32_t(std::max<uint64_t>(1, std::min<uint64_t>({kMaxParts, (c.rows + 7) / 8, std::max<uint32_t>(1, 148 * 16 / tiles)})));
  if (c.grad_x && c.rows) {
    FLS_LAUNCH(launch(fls_norm_coef_kernel<X, Y>, dim3(uint32_t(std::min<uint64_t>(c.rows, 148 * 64))), 256, false, s, c));
    dependent = true;
  }
  FLS_LAUNCH(launch(fls_norm_columns_kernel<X, Y>, dim3(tiles, c.parts), 256, dependent, s, c));
  if (c.grad_weight || c.grad_bias) FLS_LAUNCH(launch(fls_norm_join_kernel, dim3(tiles, 2), 256, true, s, c));
  return FLS_OK;
}

int check_stride(uint64_t& stride, uint32_t dim, const char* name) {
  if (!stride) stride = dim;
  if (stride < dim) return refuse(FLS_EINVAL, "%s (%llu) < dim (%u)", name, (unsigned long long)stride, dim);
  if (stride >= (1ull << 31)) return refuse(FLS_EINVAL, "%s out of range", name);
  return FLS_OK;
}

NormCall call_of(const fls_norm* h, uint64_t rows) {
  NormCall c{};
  const fls_norm_desc& d = h->desc;
  c.rows = rows;
  c.dim = d.dim;
  c.dp = uint32_t(up(d.dim, 32));
  c.rms = d.kind == FLS_NORM_RMS;
  c.weight_f32 = d.weight_dtype == FLS_GRAD_F32;
  c.grad_f32 = d.grad_dtype == FLS_GRAD_F32;
  c.eps = float(d.eps);
  c.inv_dim = float(1.0 / d.dim);
  return c;
}

}  // namespace

extern "C" {

int fls_norm_create(const fls_norm_desc* desc, fls_norm** out) {
  if (out) *out = nullptr;
  if (!desc || !out) return refuse(FLS_EINVAL, "null argument");
  if (desc->reserved) return refuse(FLS_EINVAL, "reserved must be 0");
  if (desc->max_rows > (1ull << 24)) return refuse(FLS_EINVAL, "max_rows > 2^24");
  if (desc->dim < 1 || desc->dim > 65536) return refuse(FLS_EINVAL, "dim must be in 1 .. 65536");
  if (desc->kind != FLS_NORM_LAYER && desc->kind != FLS_NORM_RMS) return refuse(FLS_EINVAL, "unknown kind %u", desc->kind);
  if (desc->grads > 1) return refuse(FLS_EINVAL, "grads must be 0 or 1");
  if (!known(desc->x_dtype)) return refuse(FLS_EINVAL, "unknown x_dtype %u", desc->x_dtype);
  if (!known(desc->y_dtype)) return refuse(FLS_EINVAL, "unknown y_dtype %u", desc->y_dtype);
  if (!known(desc->weight_dtype)) return refuse(FLS_EINVAL, "unknown weight_dtype %u", desc->weight_dtype);
  if (!known(desc->grad_dtype)) return refuse(FLS_EINVAL, "unknown grad_dtype %u", desc->grad_dtype);
  if (!(desc->eps >= 0.0 && desc->eps <= 1e30)) return refuse(FLS_EINVAL, "eps must be in 0 .. 1e30");
  fls_norm* h = new (std::nothrow) fls_norm;
  if (!h) return refuse(FLS_ESTATE, "out of host memory");
  h->desc = *desc;
  h->reg = regions(*desc);
  *out = h;
  return FLS_OK;
}

int fls_norm_query(const fls_norm* norm, fls_norm_layout* out) {
  if (!norm || !out) return refuse(FLS_EINVAL, "null argument");
  out->workspace_bytes = norm->reg.total;
  return FLS_OK;
}

int fls_norm_destroy(fls_norm* norm) {
  delete norm;
  return FLS_OK;
}

int fls_norm_forward(fls_norm* h, const fls_norm_io* io, void* cuda_stream) {
  if (!h || !io) return refuse(FLS_EINVAL, "null argument");
  const fls_norm_desc& d = h->desc;
  if (io->reserved) return refuse(FLS_EINVAL, "reserved must be 0");
  if (io->rows > d.max_rows) return refuse(FLS_EINVAL, "rows (%llu) > max_rows (%llu)", (unsigned long long)io->rows, (unsigned long long)d.max_rows);
  if (!io->residual != !io->total && io->rows) return refuse(FLS_EINVAL, "residual and total belong together");
  if (d.kind == FLS_NORM_RMS && io->mean) return refuse(FLS_EINVAL, "a root mean square norm has no mean");
  NormCall c = call_of(h, io->rows);
  c.x_stride = io->x_stride; c.residual_stride = io->residual_stride; c.y_stride = io->y_stride; c.total_stride = io->total_stride;
  if (int rc = check_stride(c.x_stride, d.dim, "x_stride")) return rc;
  if (int rc = check_stride(c.residual_stride, d.dim, "residual_stride")) return rc;
  if (int rc = check_stride(c.y_stride, d.dim, "y_stride")) return rc;
  if (int rc = check_stride(c.total_stride, d.dim, "total_stride")) return rc;
  const uint64_t n = io->rows, xs = size_of(d.x_dtype), ys = size_of(d.y_dtype), ws = size_of(d.weight_dtype);
  // total may be x or the residual themselves: every element is read before it is written, by the same thread
  const bool over_x = io->total && io->total == io->x && c.total_stride == c.x_stride;
  const bool over_r = io->total && io->total == io->residual && c.total_stride == c.residual_stride;
  const uint64_t rb = io->residual ? span_bytes(n, d.dim, c.residual_stride, xs) : 0;
  const Span s[8] = {{io->x, over_x ? 0 : span_bytes(n, d.dim, c.x_stride, xs), xs, false, "x"},
                     {io->residual, over_r ? 0 : rb, xs, false, "residual"},
                     {io->weight, n && io->weight ? d.dim * ws : 0, ws, false, "weight"},
                     {io->bias, n && io->bias ? d.dim * ws : 0, ws, false, "bias"},
                     {io->y, span_bytes(n, d.dim, c.y_stride, ys), ys, true, "y"},
                     {io->total, io->total ? span_bytes(n, d.dim, c.total_stride, xs) : 0, xs, true, "total"},
                     {io->mean, io->mean ? n * 4 : 0, 4, true, "mean"},
                     {io->rstd, io->rstd ? n * 4 : 0, 4, true, "rstd"}};
  if (int rc = check_spans(s, 8)) return rc;
  if (!n) return FLS_OK;
  c.x = io->x; c.residual = io->residual; c.weight = io->weight; c.bias = io->bias;
  c.y = io->y; c.total = io->total; c.mean = io->mean; c.rstd = io->rstd;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (d.x_dtype == FLS_GRAD_F32) return d.y_dtype == FLS_GRAD_F32 ? run_forward<float, float>(h, c, st) : run_forward<float, uint16_t>(h, c, st);
  return d.y_dtype == FLS_GRAD_F32 ? run_forward<uint16_t, float>(h, c, st) : run_forward<uint16_t, uint16_t>(h, c, st);
}

int fls_norm_backward(fls_norm* h, const fls_norm_grad_io* io, void* cuda_stream) {
  if (!h || !io) return refuse(FLS_EINVAL, "null argument");
  const fls_norm_desc& d = h->desc;
  if (io->reserved) return refuse(FLS_EINVAL, "reserved must be 0");
  if (!d.grads) return refuse(FLS_EINVAL, "the norm was created without grads");
  if (io->rows > d.max_rows) return refuse(FLS_EINVAL, "rows (%llu) > max_rows (%llu)", (unsigned long long)io->rows, (unsigned long long)d.max_rows);
  if (io->accumulate > 1) return refuse(FLS_EINVAL, "accumulate must be 0 or 1");
  if (io->grad_total && !io->grad_x && io->rows) return refuse(FLS_EINVAL, "grad_total needs grad_x");
  if (d.kind == FLS_NORM_RMS && io->mean) return refuse(FLS_EINVAL, "a root mean square norm has no mean");
  NormCall c = call_of(h, io->rows);
  c.x_stride = io->x_stride; c.grad_y_stride = io->grad_y_stride; c.grad_total_stride = io->grad_total_stride; c.grad_x_stride = io->grad_x_stride;
  if (int rc = check_stride(c.x_stride, d.dim, "x_stride")) return rc;
  if (int rc = check_stride(c.grad_y_stride, d.dim, "grad_y_stride")) return rc;
  if (int rc = check_stride(c.grad_total_stride, d.dim, "grad_total_stride")) return rc;
  if (int rc = check_stride(c.grad_x_stride, d.dim, "grad_x_stride")) return rc;
  if (io->workspace && io->workspace_bytes < h->reg.total)
    return refuse(FLS_ESIZE, "workspace has %llu bytes, %llu needed", (unsigned long long)io->workspace_bytes, (unsigned long long)h->reg.total);
  const uint64_t n = io->rows, xs = size_of(d.x_dtype), ys = size_of(d.y_dtype), ws = size_of(d.weight_dtype), gs = size_of(d.grad_dtype);
  const bool layer = d.kind == FLS_NORM_LAYER;
  // grad_x may be grad_total itself
  const bool over = io->grad_total && io->grad_total == io->grad_x && c.grad_total_stride == c.grad_x_stride;
  const Span s[11] = {{io->x, span_bytes(n, d.dim, c.x_stride, xs), xs, false, "x"},
                      {io->weight, n && io->weight ? d.dim * ws : 0, ws, false, "weight"},
                      {io->mean, layer ? n * 4 : 0, 4, false, "mean"},
                      {io->rstd, n * 4, 4, false, "rstd"},
                      {io->grad_y, span_bytes(n, d.dim, c.grad_y_stride, ys), ys, false, "grad_y"},
                      {io->grad_total, io->grad_total && !over ? span_bytes(n, d.dim, c.grad_total_stride, xs) : 0, xs, false, "grad_total"},
                      {io->grad_x, io->grad_x ? span_bytes(n, d.dim, c.grad_x_stride, xs) : 0, xs, true, "grad_x"},
                      {io->grad_weight, io->grad_weight ? d.dim * gs : 0, gs, true, "grad_weight"},
                      {io->grad_bias, io->grad_bias ? d.dim * gs : 0, gs, true, "grad_bias"},
                      {io->workspace, h->reg.total, 256, true, "workspace"}};
  if (int rc = check_spans(s, 10)) return rc;
  if (!io->grad_x && !io->grad_weight && !io->grad_bias) return FLS_OK;
  if (!n && (io->accumulate || (!io->grad_weight && !io->grad_bias))) return FLS_OK;
  c.x = io->x; c.weight = io->weight; c.mean_in = io->mean; c.rstd_in = io->rstd;
  c.grad_y = io->grad_y; c.grad_total = io->grad_total;
  c.grad_x = io->grad_x; c.grad_weight = io->grad_weight; c.grad_bias = io->grad_bias;
  c.accumulate = io->accumulate;
  char* w = static_cast<char*>(io->workspace);
  c.coef = reinterpret_cast<float2*>(w + h->reg.coef);
  c.part = reinterpret_cast<float*>(w + h->reg.part);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (d.x_dtype == FLS_GRAD_F32) return d.y_dtype == FLS_GRAD_F32 ? run_backward<float, float>(h, c, st) : run_backward<float, uint16_t>(h, c, st);
  return d.y_dtype == FLS_GRAD_F32 ? run_backward<uint16_t, float>(h, c, st) : run_backward<uint16_t, uint16_t>(h, c, st);
}

int fls_norm_get_launch_count(const fls_norm* norm, uint64_t* launches) {
  if (!norm || !launches) return refuse(FLS_EINVAL, "null argument");
  *launches = norm->launches;
  return FLS_OK;
}

}  // extern "C"
