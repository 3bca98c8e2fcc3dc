// fls_norm_*: layer norm and root mean square norm of rows, with the residual addition before it, and the backward pass with
// the sums of the weight's and the bias's gradient.
//
// Forward, per row s of d values: m = mean(s) in fp32, then e = mean(s - m) and q = mean((s - m)^2) in a second look at the
// values, which takes the rounding of m out of the result: mean = m + e, variance = q - e^2, which is not below zero but by the
// roundings of q and e (rows of equal values), about 3 (d / 32 + 16) 2^-24 (s - m)^2.
//
// Bound by memory where rows are fp32 (16384 x 2048 with residual 72 us, 6.5 TB/s, 99 % of the measured copy) or bf16 with a residual
// (44 us, 6.05 TB/s); bf16 alone by the instructions and sums between a row's load and its store (29 us, 4.6 TB/s).  Backward
// 32768 x 768 with fp32 rows 47 to 49 us, 6.1 TB/s in the loop and 7 us of start and joins; with bf16 rows 38 us, 4.0 TB/s, bound by
// latency and issue.  One row: 2.4 us forward, 5 backward.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <new>
#include <type_traits>

#include "fls.h"
#include "fls_elem.cuh"
#include "fls_internal.h"

using namespace fls;

namespace {

constexpr uint32_t kColTile = 32;          // columns of a CTA of the weight gradients' kernel
constexpr uint32_t kJoinFloats = 16384;    // of the parts' sums of one gradient that a single CTA adds up: 128 x 768 costs the device 2 us more
                                           // than a second kernel, and the host 3 us less
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
  uint32_t* ticket;                        // 0 between calls: CTAs that have left their sums
  uint32_t join;                           // the last of them adds the sums up
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

// The gradient of column `col` of the weight (which = 0) or the bias (1).
__device__ __forceinline__ void write_gradient(const NormCall& c, uint32_t which, uint32_t col, float sum) {
  void* out = which ? c.grad_bias : c.grad_weight;
  if (!out || col >= c.dim) return;
  if (c.grad_f32) {
    float* o = static_cast<float*>(out) + col;
    *o = c.accumulate ? *o + sum : sum;
  } else {
    uint16_t* o = static_cast<uint16_t*>(out) + col;
    Elem<uint16_t>::put(o, c.accumulate ? Elem<uint16_t>::get(o) + sum : sum);
  }
}

// From q and e of a row.  A comparison, not a maximum: the variance of a row that is not finite stays NaN.
__device__ __forceinline__ float rstd_of(float q, float e, float eps) {
  const float var = fmaf(-e, e, q);
  return 1.f / sqrtf((var < 0.f ? 0.f : var) + eps);
}

// ------------------------------------------------------------------------------------------------ rows in registers
// A row belongs to `tpr` neighbouring threads, each with K cells of eight columns: neighbouring columns where every row starts
// on a boundary of eight elements and holds whole cells (VEC), otherwise columns 32 apart, moved one by one.
template <bool VEC>
__device__ __forceinline__ uint32_t column(uint32_t tpr, uint32_t t, int k, int j) {
  return VEC ? (k * tpr + t) * 8 + j : (k * (tpr / 32) + t / 32) * 256 + t % 32 + 32 * j;
}

template <typename T, bool VEC> struct Cell;
template <typename T> struct Cell<T, true> {
  typename Elem<T>::Raw raw;
  __device__ __forceinline__ void load(const T* row, uint32_t col, uint32_t dim) {
    raw = typename Elem<T>::Raw{};
    if (col < dim) raw = Elem<T>::load_raw(row + col);
  }
  __device__ __forceinline__ void get(f2 (&x)[4]) const {
    float y[8];
    Elem<T>::unpack(raw, y);
    pairs_of(y, x);
  }
  __device__ static __forceinline__ void store(T* row, uint32_t col, uint32_t dim, const f2 (&x2)[4]) {
    float x[8];
    singles_of(x2, x);
    if (col < dim) Elem<T>::store8(row + col, x);
  }
};
template <typename T> struct Cell<T, false> {
  float x_[8];
  __device__ __forceinline__ void load(const T* row, uint32_t col, uint32_t dim) {
    row += col;
#pragma unroll
    for (int j = 0; j < 8; ++j) x_[j] = col + 32 * j < dim ? Elem<T>::get(row + 32 * j) : 0.f;
  }
  __device__ __forceinline__ void get(f2 (&x)[4]) const { pairs_of(x_, x); }
  __device__ static __forceinline__ void store(T* row, uint32_t col, uint32_t dim, const f2 (&x2)[4]) {
    float x[8];
    singles_of(x2, x);
    row += col;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (col + 32 * j < dim) Elem<T>::put(row + 32 * j, x[j]);
  }
};

// Eight values of the weight or the bias; `other` where there is none.  VEC asks for a boundary of eight of theirs too.
template <bool VEC>
__device__ __forceinline__ void weight_cell(const NormCall& c, const void* p, float other, uint32_t col, f2 (&x)[4]) {
  if (!p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = make_f2(other);
  } else if (c.weight_f32) {
    Cell<float, VEC> w;
    w.load(static_cast<const float*>(p), col, c.dim);
    w.get(x);
  } else {
    Cell<uint16_t, VEC> w;
    w.load(static_cast<const uint16_t*>(p), col, c.dim);
    w.get(x);
  }
}

// Sum over `width` neighbouring lanes, a power of two.
__device__ __forceinline__ float warp_sum(float x, uint32_t width) {
#pragma unroll
  for (uint32_t o = 16; o; o /= 2)
    if (o < width) x += __shfl_xor_sync(~0u, x, o);
  return x;
}
// Two sums over a warp, from the second step on one in each half: x's in lanes 0 .. 15, y's in lanes 16 .. 31.
__device__ __forceinline__ float warp_sum(float x, float y, uint32_t lane) {
  const float other = __shfl_xor_sync(~0u, lane < 16 ? y : x, 16);
  float v = (lane < 16 ? x : y) + other;
#pragma unroll
  for (int o = 8; o; o /= 2) v += __shfl_xor_sync(~0u, v, o);
  return v;
}

// Four sums over a warp: a's in lanes 0 .. 7, b's in lanes 8 .. 15, c's and d's in the other half.
__device__ __forceinline__ float warp_sum(float a, float b, float c, float d, uint32_t lane) {
  const bool low = lane < 16, even = (lane & 8) == 0;
  a = (low ? a : c) + __shfl_xor_sync(~0u, low ? c : a, 16);
  b = (low ? b : d) + __shfl_xor_sync(~0u, low ? d : b, 16);
  a = (even ? a : b) + __shfl_xor_sync(~0u, even ? b : a, 8);
#pragma unroll
  for (int o = 4; o; o /= 2) a += __shfl_xor_sync(~0u, a, o);
  return a;
}

// Sums over the `warps` warps of a row of what each has left in `shared`, V values each, in order of the warps.
template <int V>
__device__ __forceinline__ void warps_sum(const float* shared, uint32_t warps, float (&v)[V]) {
  typedef typename std::conditional<V == 4, float4, float2>::type Vec;
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = shared[i];
#pragma unroll 4
  for (uint32_t w = 1; w < warps; ++w) {
    const Vec x = reinterpret_cast<const Vec*>(shared)[w];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] += reinterpret_cast<const float*>(&x)[i];
  }
}

// One row from its cells on: the residual's addition, statistics and the result.  The row's threads meet in `meet`; shared1 and
// shared2 hold a value of each of the CTA's warps.  live: false for threads that only keep the others' barriers company.
template <typename X, typename Y, bool VEC, int K, typename Meet>
__device__ __forceinline__ void norm_row(const NormCall& c, const Cell<X, VEC> (&in)[K], const Cell<X, VEC> (&add)[K], uint64_t n, bool live,
                                         uint32_t tpr, uint32_t t, float2* shared1, float2* shared2, Meet meet) {
  const uint32_t lane = threadIdx.x % 32, width = min(tpr, 32u), warps = tpr / width, mine = threadIdx.x / 32, first = mine / warps * warps;
  f2 x[K][4], w[4], b[4];
#pragma unroll
  for (int k = 0; k < K; ++k) in[k].get(x[k]);
  if (c.residual) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      f2 r[4];
      float s[8];
      add[k].get(r);
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = add2(x[k][i], r[i]);
      singles_of(r, s);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = Elem<X>::round(s[j]);
      pairs_of(s, x[k]);
      if (live) Cell<X, VEC>::store(static_cast<X*>(c.total) + n * c.total_stride, column<VEC>(tpr, t, k, 0), c.dim, x[k]);
    }
  }
  if (K == 1) {                                             // few rows: everything on its way at once
    weight_cell<VEC>(c, c.weight, 1.f, column<VEC>(tpr, t, 0, 0), w);
    weight_cell<VEC>(c, c.bias, 0.f, column<VEC>(tpr, t, 0, 0), b);
  }
  float m = 0.f;
  if (!c.rms) {
    f2 a = make_f2(0.f);
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) a = add2(a, x[k][i]);
    m = warp_sum(sum2(a), width);
    if (warps > 1) {
      if (lane == 0) shared1[mine] = make_float2(m, 0.f);
      meet();
      float v[2];
      warps_sum<2>(&shared1[first].x, warps, v);
      m = v[0];
    }
    m *= c.inv_dim;
    const f2 less = make_f2(-m);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (VEC) {
        const f2 off = column<VEC>(tpr, t, k, 0) < c.dim ? less : make_f2(0.f);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[k][i] = add2(x[k][i], off);
      } else {
        float s[8];
        singles_of(x[k], s);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = column<VEC>(tpr, t, k, j) < c.dim ? s[j] - m : 0.f;
        pairs_of(s, x[k]);
      }
    }
  }
  f2 ones = make_f2(0.f), squares = make_f2(0.f);
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (!c.rms) ones = add2(ones, x[k][i]);
      squares = fma2(x[k][i], x[k][i], squares);
    }
  float v[2];
  if (width < 32) {
    v[0] = c.rms ? 0.f : warp_sum(sum2(ones), width);
    v[1] = warp_sum(sum2(squares), width);
  } else {
    const float half = warp_sum(sum2(ones), sum2(squares), lane);
    if (warps > 1) {
      if (lane % 16 == 0) (lane ? shared2[mine].y : shared2[mine].x) = half;
      meet();
      warps_sum<2>(&shared2[first].x, warps, v);
    } else {
      v[0] = __shfl_sync(~0u, half, 0);
      v[1] = __shfl_sync(~0u, half, 16);
    }
  }
  const float e = c.rms ? 0.f : v[0] * c.inv_dim, rstd = rstd_of(v[1] * c.inv_dim, e, c.eps);
  if (!live) return;
  const f2 scale = make_f2(rstd), shift = make_f2(-e * rstd);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if (column<VEC>(tpr, t, k, 0) >= c.dim) break;
    if (K > 1) {
      weight_cell<VEC>(c, c.weight, 1.f, column<VEC>(tpr, t, k, 0), w);
      weight_cell<VEC>(c, c.bias, 0.f, column<VEC>(tpr, t, k, 0), b);
    }
    f2 y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = fma2(fma2(x[k][i], scale, shift), w[i], b[i]);
    Cell<Y, VEC>::store(static_cast<Y*>(c.y) + n * c.y_stride, column<VEC>(tpr, t, k, 0), c.dim, y);
  }
  if (t == 0) {
    if (c.mean) c.mean[n] = m + e;
    if (c.rstd) c.rstd[n] = rstd;
  }
}

// CTAs of an SM that the registers are divided among (us of 16384 x 2048 bf16, K = 4, with 3 / 4: 32.6 / 29.4; 65536 x 512, K = 2,
// with 4 / 5: 46.3 / 43.5; 65536 x 256, K = 1, with 5 / 6: 29.4 / 27.8).
constexpr int ctas_per_sm(bool vec, int k, int size, int threads) {
  return threads != 256 ? 1 : !vec ? (k == 1 ? 5 : 1) : size == 4 ? 1 : k == 1 ? 6 : k == 2 ? 5 : 4;
}

template <typename X, typename Y, bool VEC, int K, int THREADS>
__global__ void __launch_bounds__(THREADS, ctas_per_sm(VEC, K, sizeof(X), THREADS)) fls_norm_forward_kernel(const __grid_constant__ NormCall c, uint32_t tpr) {
  __shared__ float2 shared1[32], shared2[32];
  const uint32_t t = threadIdx.x % tpr;
  const uint64_t n = uint64_t(blockIdx.x) * (blockDim.x / tpr) + threadIdx.x / tpr;
  const bool live = n < c.rows;
  const uint64_t row = live ? n : c.rows - 1;
  Cell<X, VEC> in[K], add[K];
#pragma unroll
  for (int k = 0; k < K; ++k) in[k].load(static_cast<const X*>(c.x) + row * c.x_stride, column<VEC>(tpr, t, k, 0), c.dim);
  if (c.residual)
#pragma unroll
    for (int k = 0; k < K; ++k) add[k].load(static_cast<const X*>(c.residual) + row * c.residual_stride, column<VEC>(tpr, t, k, 0), c.dim);
  norm_row<X, Y, VEC, K>(c, in, add, row, live, tpr, t, shared1, shared2, [] { __syncthreads(); });
}

// All gradients in one look at the rows.  A CTA has blockDim / tpr groups, a group a stretch of rows, B of them at a time; a
// thread keeps its columns' sums for weight and bias in registers, adds them to the other groups' at the end and leaves the
// CTA's in the workspace.  VEC: STAGES times B rows are on their way at once, copied asynchronously into shared memory, every
// warp for itself.
template <typename X, typename Y, bool VEC, int K, int B, int STAGES, int THREADS, bool RMS>
__global__ void __launch_bounds__(THREADS, 1) fls_norm_backward_kernel(const __grid_constant__ NormCall c, uint32_t tpr) {
  extern __shared__ __align__(16) float smem[];             // rows on their way, then the groups' sums
  __shared__ __align__(16) float sums[2][THREADS / 32][2 * B];
  const uint32_t t = threadIdx.x % tpr, group = threadIdx.x / tpr, groups = blockDim.x / tpr, warps = tpr / 32, lane = threadIdx.x % 32;
  const uint64_t all = uint64_t(gridDim.x) * groups, g = uint64_t(blockIdx.x) * groups + group;
  const uint64_t begin = c.rows * g / all;
  const uint32_t count = uint32_t(c.rows * (g + 1) / all - begin);
  const bool with_total = c.grad_total != nullptr;
  const uint32_t row_bytes = K * (Staged<X>::bytes + Staged<Y>::bytes + (with_total ? Staged<X>::bytes : 0));
  const uint32_t mine = uint32_t(__cvta_generic_to_shared(smem)) + threadIdx.x / 32 * (STAGES * B * row_bytes), stop = mine + STAGES * B * row_bytes;
  const X* px = static_cast<const X*>(c.x) + begin * c.x_stride;
  const Y* py = static_cast<const Y*>(c.grad_y) + begin * c.grad_y_stride;
  const X* pt = static_cast<const X*>(c.grad_total) + begin * c.grad_total_stride;
  X* pd = static_cast<X*>(c.grad_x) + begin * c.grad_x_stride;
  pdl_launch();

  uint32_t to = mine, unsent = count;
  auto send = [&] {                                         // the next B rows' copies
    if (VEC) {
#pragma unroll
      for (int b = 0; b < B; ++b) {
        if (unsent) {
          --unsent;
#pragma unroll
          for (int k = 0; k < K; ++k) {
            const uint32_t first = column<VEC>(tpr, t - lane, k, 0);
            const uint32_t q = to + k * (Staged<X>::bytes + Staged<Y>::bytes);
            Staged<X>::copy(q, px, first, lane, c.dim);
            Staged<Y>::copy(q + Staged<X>::bytes, py, first, lane, c.dim);
            if (with_total) Staged<X>::copy(to + K * (Staged<X>::bytes + Staged<Y>::bytes) + k * Staged<X>::bytes, pt, first, lane, c.dim);
          }
          px += c.x_stride;
          py += c.grad_y_stride;
          pt += c.grad_total_stride;
        }
        to += row_bytes;
      }
      if (to == stop) to = mine;
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
  };
#pragma unroll 1
  for (int i = 0; i + 1 < STAGES; ++i) send();

  f2 w[K][4], dw[K][4], db[K][4];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    weight_cell<VEC>(c, c.weight, 1.f, column<VEC>(tpr, t, k, 0), w[k]);
#pragma unroll
    for (int i = 0; i < 4; ++i) dw[k][i] = db[k][i] = make_f2(0.f);
  }
  float means = 0.f, rstds = 0.f;                           // of 32 rows, one per lane
  uint32_t from = mine, turn = 0;
  for (uint32_t i = 0; i < count; i += B) {
    if (i % 32 == 0) {
      const bool there = i + lane < count;
      means = there && !RMS ? c.mean_in[begin + i + lane] : 0.f;
      rstds = there ? c.rstd_in[begin + i + lane] : 0.f;
    }
    if (VEC) {
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES > 1 ? STAGES - 2 : 0) : "memory");
      __syncwarp();
    }
    Cell<X, VEC> dt[B][K];
    f2 xhat[B][K][4], gy[B][K][4];
    f2 scale[B];
    float rstd[B], v[2 * B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const bool there = B == 1 || i + b < count;           // the stretch may end with half of a pair, whose place holds what was there
      Cell<X, VEC> x[K];
      Cell<Y, VEC> dy[K];
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if constexpr (VEC) {
          const uint32_t q = from + b * row_bytes + k * (Staged<X>::bytes + Staged<Y>::bytes);
          Staged<X>::read(q, lane, x[k].raw);
          Staged<Y>::read(q + Staged<X>::bytes, lane, dy[k].raw);
          if (with_total) Staged<X>::read(from + b * row_bytes + K * (Staged<X>::bytes + Staged<Y>::bytes) + k * Staged<X>::bytes, lane, dt[b][k].raw);
          if (!there) { x[k] = Cell<X, VEC>{}; dy[k] = Cell<Y, VEC>{}; }
        } else {
          const uint32_t col = there ? column<VEC>(tpr, t, k, 0) : c.dim;      // nothing beyond the last column
          x[k].load(px, col, c.dim);
          dy[k].load(py, col, c.dim);
          if (with_total) dt[b][k].load(pt, col, c.dim);
        }
      }
      if (!VEC) {
        px += c.x_stride;
        py += c.grad_y_stride;
        pt += c.grad_total_stride;
      }
      const float mean = __shfl_sync(~0u, means, i + b);
      rstd[b] = __shfl_sync(~0u, rstds, i + b);             // 0 for a row that is not there
      scale[b] = make_f2(rstd[b]);
      f2 sum_g = make_f2(0.f), sum_gx = make_f2(0.f);
      const f2 less = make_f2(-mean);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        x[k].get(xhat[b][k]);
        dy[k].get(gy[b][k]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (!RMS) xhat[b][k][j] = add2(xhat[b][k][j], less);
          xhat[b][k][j] = mul2(xhat[b][k][j], scale[b]);
          dw[k][j] = fma2(gy[b][k][j], xhat[b][k][j], dw[k][j]);
          db[k][j] = add2(db[k][j], gy[b][k][j]);
          gy[b][k][j] = mul2(gy[b][k][j], w[k][j]);
          if (!RMS) sum_g = add2(sum_g, gy[b][k][j]);
          sum_gx = fma2(gy[b][k][j], xhat[b][k][j], sum_gx);
        }
      }
      v[2 * b] = sum2(sum_g);
      v[2 * b + 1] = sum2(sum_gx);
    }
    if (VEC) {
      __syncwarp();
      from += B * row_bytes;
      if (from == stop) from = mine;
      send();                                               // into the place that the rows before these had
    }
    if (!c.grad_x) continue;
    float part;
    if constexpr (B == 2) part = warp_sum(v[0], v[1], v[2], v[3], lane);
    else part = warp_sum(v[0], v[1], lane);
    if (warps > 1) {
      if (lane % (16 / B) == 0) sums[turn][threadIdx.x / 32][lane / (16 / B)] = part;
      asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(tpr) : "memory");
      warps_sum<2 * B>(sums[turn][group * warps], warps, v);
      turn ^= 1;                                            // the next rows' go elsewhere while these are read
    } else {
#pragma unroll
      for (int q = 0; q < 2 * B; ++q) v[q] = __shfl_sync(~0u, part, q * (16 / B));
    }
    // rstd (gy - mean(gy) - xhat mean(gy xhat))
#pragma unroll
    for (int b = 0; b < B; ++b) {
      if (B > 1 && i + b >= count) break;
      const f2 k1 = make_f2(RMS ? 0.f : -v[2 * b] * c.inv_dim * rstd[b]), k2 = make_f2(-v[2 * b + 1] * c.inv_dim * rstd[b]);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        f2 dx[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) dx[j] = fma2(gy[b][k][j], scale[b], fma2(xhat[b][k][j], k2, k1));
        if (with_total) {
          f2 add[4];
          dt[b][k].get(add);
#pragma unroll
          for (int j = 0; j < 4; ++j) dx[j] = add2(dx[j], add[j]);
        }
        Cell<X, VEC>::store(pd, column<VEC>(tpr, t, k, 0), c.dim, dx);
      }
      pd += c.grad_x_stride;
    }
  }
  if (!c.grad_weight && !c.grad_bias) return;
  // the groups' sums, in their order
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  f2* sh = reinterpret_cast<f2*>(smem);
  if (group) {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sh[((group - 1) * 8 * K + k * 8 + j) * tpr + t] = dw[k][j];
        sh[((group - 1) * 8 * K + k * 8 + 4 + j) * tpr + t] = db[k][j];
      }
  }
  __syncthreads();
  if (group == 0) {
#pragma unroll 1
    for (uint32_t o = 0; o + 1 < groups; ++o)
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          dw[k][j] = add2(dw[k][j], sh[(o * 8 * K + k * 8 + j) * tpr + t]);
          db[k][j] = add2(db[k][j], sh[(o * 8 * K + k * 8 + 4 + j) * tpr + t]);
        }
    float* part = c.part + uint64_t(2 * blockIdx.x) * c.dp;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      Cell<float, VEC>::store(part, column<VEC>(tpr, t, k, 0), c.dim, dw[k]);
      Cell<float, VEC>::store(part + c.dp, column<VEC>(tpr, t, k, 0), c.dim, db[k]);
    }
  }
  if (!c.join) return;
  // few sums: whoever comes last adds them up, in order of the CTAs
  __shared__ uint32_t arrived;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) arrived = atomicAdd(c.ticket, 1u);
  __syncthreads();
  if (arrived + 1 != gridDim.x) return;
  __threadfence();
  if (threadIdx.x == 0) *c.ticket = 0;
  for (uint32_t q = threadIdx.x; q < c.dp / 2; q += blockDim.x) {       // four columns of the weight's sums, then of the bias's
    const uint32_t which = q >= c.dp / 4, col = (which ? q - c.dp / 4 : q) * 4;
    const float4* from = reinterpret_cast<const float4*>(c.part + uint64_t(which) * c.dp + col);
    float4 sum = __ldcg(from);
#pragma unroll 8
    for (uint32_t p = 1; p < gridDim.x; ++p) {
      const float4 v = __ldcg(from + uint64_t(p) * (c.dp / 2));
      sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
    }
    write_gradient(c, which, col, sum.x);
    write_gradient(c, which, col + 1, sum.y);
    write_gradient(c, which, col + 2, sum.z);
    write_gradient(c, which, col + 3, sum.w);
  }
}

// ------------------------------------------------------------------------------------------------ rows of any length
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
    const float e = c.rms ? 0.f : v.x * c.inv_dim, rstd = rstd_of(v.y * c.inv_dim, e, c.eps);
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

// The parts' sums, in their order inside each of 32 groups, then of the groups.
__global__ void __launch_bounds__(1024) fls_norm_join_kernel(const __grid_constant__ NormCall c) {
  __shared__ float shared[32][kColTile + 1];
  const uint32_t lane = threadIdx.x % 32, group = threadIdx.x / 32, j = blockIdx.x * kColTile + lane, which = blockIdx.y;
  void* out = which ? c.grad_bias : c.grad_weight;
  pdl_wait();
  if (!out) return;
  float sum = 0.f;
#pragma unroll 10
  for (uint32_t p = group; p < c.parts; p += 32)
    if (j < c.dim) sum += c.part[uint64_t(2 * p + which) * c.dp + j];
  shared[group][lane] = sum;
  __syncthreads();
  sum = shared[lane][group];                                // column `group`, group `lane`
#pragma unroll
  for (int o = 16; o; o /= 2) sum += __shfl_xor_sync(~0u, sum, o);
  const uint32_t col = blockIdx.x * kColTile + group;
  if (!lane) write_gradient(c, which, col, sum);
}

struct Regions { uint64_t coef, part, total; };
Regions regions(const fls_norm_desc& d) {
  Regions r{};
  uint64_t at = d.grads ? 256 : 0;         // the ticket
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
  std::atomic<uint64_t> launches{0};      // calls that do not share a workspace may come from several host threads
};

namespace {

#define FLS_LAUNCH(call)                                                                            \
  do {                                                                                              \
    const cudaError_t e_ = (call);                                                                  \
    if (e_ != cudaSuccess) return refuse(FLS_ECUDA, "norm kernel: %s", cudaGetErrorString(e_));     \
    ++h->launches;                                                                                  \
  } while (0)

template <typename X, typename Y, bool VEC>
cudaError_t forward_rows(const NormCall& c, cudaStream_t s) {
  const uint32_t cells = (c.dim + 7) / 8;
  // Few rows: a cell per thread, for the shortest way through a row.  Many: four, which leaves the fewest sums over threads;
  // columns moved one by one are many loads on their way as it is.
  int k = VEC && c.rows * cells > 148 * 1024 ? 4 : 1;
  while (k < 4 && cells > uint32_t(k) * 1024) ++k;
  while (k > 1 && cells <= 32u * (k - 1)) --k;              // short rows: no empty cells
  uint32_t tpr = (cells + 32 * k - 1) / (32 * k) * 32;
  if (VEC && cells <= 16) tpr = cells <= 8 ? 8 : 16;        // two or four rows in a warp
  const uint32_t rows = std::max(1u, 256 / tpr);
  const dim3 grid(uint32_t((c.rows + rows - 1) / rows));
#define FLS_K(K) (tpr > 256 ? launch(fls_norm_forward_kernel<X, Y, VEC, K, 1024>, grid, tpr * rows, 0, false, s, c, tpr) \
                            : launch(fls_norm_forward_kernel<X, Y, VEC, K, 256>, grid, tpr * rows, 0, false, s, c, tpr))
  return k == 1 ? FLS_K(1) : k == 2 ? FLS_K(2) : k == 3 ? FLS_K(3) : FLS_K(4);
#undef FLS_K
}

template <typename X, typename Y>
int run_forward(fls_norm* h, NormCall& c, cudaStream_t s) {
  const uint64_t ws = c.weight_f32 ? 4 : 2;
  if (c.dim <= 32768) {
    const bool vec = c.dim % 8 == 0 && in_cells(c.weight, 0, ws) && in_cells(c.bias, 0, ws) && in_cells(c.x, c.x_stride, sizeof(X)) && in_cells(c.y, c.y_stride, sizeof(Y)) &&
                     (!c.residual || (in_cells(c.residual, c.residual_stride, sizeof(X)) && in_cells(c.total, c.total_stride, sizeof(X))));
    FLS_LAUNCH((vec ? forward_rows<X, Y, true>(c, s) : forward_rows<X, Y, false>(c, s)));
    return FLS_OK;
  }
  FLS_LAUNCH(launch(fls_norm_rows_kernel<X, Y>, dim3(uint32_t(std::min<uint64_t>(c.rows, 148 * 64))), 256, 0, false, s, c));
  return FLS_OK;
}

template <typename X, typename Y, bool VEC, int K, int B, int STAGES, int THREADS>
cudaError_t backward_rows(NormCall& c, cudaStream_t s) {
  const uint32_t cells = (c.dim + 7) / 8, tpr = (cells + 32 * K - 1) / (32 * K) * 32, groups = THREADS / tpr, threads = tpr * groups;
  c.parts = uint32_t(std::max<uint64_t>(1, std::min<uint64_t>(148, (c.rows + B * groups - 1) / (B * groups))));
  // Up to 128 KB of sums are added up by one CTA, more of them by a kernel of its own.
  c.join = c.parts * c.dp <= kJoinFloats;
  const uint32_t row_bytes = K * (Staged<X>::bytes * (c.grad_total ? 2 : 1) + Staged<Y>::bytes);
  const uint32_t smem = std::max(VEC ? STAGES * B * row_bytes * (threads / 32) : 0, (groups - 1) * tpr * 16 * K * 4);
  auto kernel = c.rms ? fls_norm_backward_kernel<X, Y, VEC, K, B, STAGES, THREADS, true> : fls_norm_backward_kernel<X, Y, VEC, K, B, STAGES, THREADS, false>;
  static std::atomic<uint64_t> done[2];
  const cudaError_t e = allow_shared(reinterpret_cast<const void*>(kernel), 226 << 10, done[c.rms]);
  if (e != cudaSuccess) return e;
  return launch(kernel, dim3(c.parts), threads, smem, false, s, c, tpr);
}

template <typename X, typename Y, bool VEC>
cudaError_t backward_of(NormCall& c, cudaStream_t s) {
  // Two rows of one cell per thread, or one row of two cells, which leaves more groups of threads for wide rows (us, two rows / two cells:
  // 32768 x 768 fp32 48 / 55, 8192 x 2560 bf16 44 / 37, fp32 56 / 60, 8192 x 4096 bf16 56 / 53, fp32 88 / 93); columns moved one by one
  // want the latter (8192 x 1001 39 / 33).  One row of one cell and 768 threads: 32768 x 768 fp32 52, 8192 x 4096 bf16 78.
  return VEC && c.dim <= (sizeof(X) == 4 ? 4096 : 2048) ? backward_rows<X, Y, VEC, 1, 2, 2, 512>(c, s) : backward_rows<X, Y, VEC, 2, 1, 2, 512>(c, s);
}

template <typename X, typename Y>
int run_backward(fls_norm* h, NormCall& c, cudaStream_t s) {
  const uint32_t tiles = (c.dim + kColTile - 1) / kColTile;
  bool dependent = false;
  const uint64_t ws = c.weight_f32 ? 4 : 2;
  if (c.dim <= 8192) {
    const bool vec = c.dim % 8 == 0 && in_cells(c.weight, 0, ws) &&
                     (!c.rows || (in_cells(c.x, c.x_stride, sizeof(X)) && in_cells(c.grad_y, c.grad_y_stride, sizeof(Y)) &&
                                 (!c.grad_x || in_cells(c.grad_x, c.grad_x_stride, sizeof(X))) &&
                                 (!c.grad_total || in_cells(c.grad_total, c.grad_total_stride, sizeof(X)))));
    FLS_LAUNCH((vec ? backward_of<X, Y, true>(c, s) : backward_of<X, Y, false>(c, s)));
  } else {
    c.parts = uint32_t(std::max<uint64_t>(1, std::min<uint64_t>({kMaxParts, (c.rows + 7) / 8, std::max<uint32_t>(1, 148 * 16 / tiles)})));
    if (c.grad_x && c.rows) {
      FLS_LAUNCH(launch(fls_norm_coef_kernel<X, Y>, dim3(uint32_t(std::min<uint64_t>(c.rows, 148 * 64))), 256, 0, false, s, c));
      dependent = true;
    }
    FLS_LAUNCH(launch(fls_norm_columns_kernel<X, Y>, dim3(tiles, c.parts), 256, 0, dependent, s, c));
  }
  if ((c.grad_weight || c.grad_bias) && !c.join) FLS_LAUNCH(launch(fls_norm_join_kernel, dim3(tiles, 2), 1024, 0, true, s, c));
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
  const Span s[10] = {{io->x, span_bytes(n, d.dim, c.x_stride, xs), xs, false, "x"},
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
  c.ticket = reinterpret_cast<uint32_t*>(w);
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
