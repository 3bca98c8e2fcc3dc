// fls_top_logits: the k largest logits of every row, ties to the lowest index, and the row's log sum exp.
//
// One pass over the logits, and a second look at few of them.  A row (or, when there are few rows, one of 2, 4 or 8 parts
// of a row, the CTAs of a cluster) belongs to a CTA of T threads.  While a thread adds up exponentials it keeps the largest
// logit it has seen, overall and in each of up to nine stretches of what it reads.  The k-th largest of the T overall
// maxima is a lower bound of the k-th largest logit, and a close one: about T ln(T / (T - k)) logits are expected to reach
// it (68 for k = 64 and T = 512).  So only stretches whose maximum reaches it, about k of them and still in L2, are read
// again.  The candidates are then ranked by counting, on 64-bit keys (value, lowest index first) that are all different,
// which makes the result independent of the order in which they were found.  Rows with so many equal logits that the
// stretches or candidates do not fit are searched bit by bit instead (fls_top_exact below).
//
// Bound by memory, 2 or 4 bytes per logit read once: 4096 x 128256 bf16, k = 64 in 206 us alone, 5.1 TB/s (79 % of the measured
// copy), 214 to 219 us among others (76 %); with k = 128 249 us.  The rest is the second look, for which 180 MB come from memory
// again, and the ranking, during which a CTA reads nothing new.  Ahead of
// the sums two fp32 operations go into one instruction (270 us without) and four 16-byte vectors per thread are on their
// way while four are added up (256 us with one thread maximum instead of stretches, 512 threads).  One row is latency:
// 11.5 us for 128256 bf16 by four CTAs, of which the load is a tenth; the 16 block-wide counts that find the bound, the
// ranking and the two cluster barriers are the rest.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "fls.h"
#include "fls_internal.h"

using namespace fls;

namespace {

constexpr uint32_t kCap = 2048;              // candidates that are ranked directly
static_assert(kCap >= 8 * FLS_HEAD_MAX_TOP, "the parts' results fit where the candidates were");
constexpr uint32_t kNegInf = 0x007FFFFFu;    // order key of -inf; larger keys may be chosen

struct TopArgs {
  const void* logits;
  uint64_t stride;
  uint32_t vocab, top;
  float c;                 // log2(e) / T
  float huge;              // logits from here on are not multiplied by c before the maximum is taken off
  double inv_temp;
  float* value;
  int32_t* index;
  float* lse;
};

// Monotone map of floats to unsigned integers; -0 equals +0, NaN ranks above everything.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0xFFFFFFFFu;
  const uint32_t u = __float_as_uint(x + 0.0f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  if (k == 0xFFFFFFFFu) return __int_as_float(0x7FC00000);
  return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}
__device__ __forceinline__ uint64_t key64(uint32_t key, uint32_t idx) { return (uint64_t(key) << 32) | (0xFFFFFFFFu - idx); }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t remote(const void* p, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(uint32_t(__cvta_generic_to_shared(p))), "r"(rank));
  return r;
}
__device__ __forceinline__ uint64_t remote_u64(uint32_t a) {
  uint64_t x;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(x) : "r"(a) : "memory");
  return x;
}
__device__ __forceinline__ float remote_f32(uint32_t a) {
  float x;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(a) : "memory");
  return x;
}
// max that lets NaN through, so that a thread that met one is known
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Two fp32 operations in one instruction.
struct f2 { uint64_t v; };
__device__ __forceinline__ f2 make_f2(float a, float b) {
  f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void split(f2 x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x.v)); }
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}

template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int n = 4;
  __device__ static __forceinline__ void unpack(const uint4& r, float (&x)[4]) {
    x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
  }
  __device__ static __forceinline__ float top(const uint4& r) {
    return max_nan(max_nan(__uint_as_float(r.x), __uint_as_float(r.y)), max_nan(__uint_as_float(r.z), __uint_as_float(r.w)));
  }
  __device__ static __forceinline__ float load(const float* p) { return *p; }
};
template <> struct Vec<uint16_t> {
  static constexpr int n = 8;
  __device__ static __forceinline__ void unpack(const uint4& r, float (&x)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  }
  __device__ static __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  __device__ static __forceinline__ float top(const uint4& r) {
    const uint32_t m = max2(max2(r.x, r.y), max2(r.z, r.w));
    return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
  }
  __device__ static __forceinline__ float load(const uint16_t* p) { return __uint_as_float(uint32_t(*p) << 16); }
};

constexpr uint32_t kStretches = 8;           // of whole steps (4 vectors per thread each), and one of what is left
template <int kTopThreads>
struct Shared {
  static constexpr int kTopWarps = kTopThreads / 32;
  uint64_t cand[kCap];                       // later, in the cluster's first CTA, all parts' results
  uint64_t best[FLS_HEAD_MAX_TOP];           // this part's result, read by the cluster's first CTA
  float stretch[kStretches + 1][kTopThreads];
  uint32_t hot[kTopThreads];                 // stretch * T + thread
  uint32_t scan[kTopWarps];
  float wm[kTopWarps], ws[kTopWarps];
  float m, s;
  uint32_t n_hot, n_cand, count[3];
};

// The part of a row that a CTA works on: `lead` single elements, whole 16-byte vectors, `trail` single elements.
template <typename T>
struct Part {
  const T* row;            // the whole row
  const uint4* vec;        // first vector of the part
  uint32_t vec0;           // index in the row of its first element
  uint32_t n_vec;
  uint32_t lead, trail;    // only the first part has `lead`, only the last `trail`
  uint32_t trail0;         // index in the row of the first trailing element
};

// (x - y) / T in powers of two.  Sums are kept relative to 2^(m c), m c rounded, while that is off by less than 2^-8 (the log
// sum exp by less than its own last digit); from |m c| = 2^16 on (masks; logits far beyond a model's) the difference is taken
// first, since 2 to the power of a rounding error of m c soon has nothing to do with 1, and m c may have no fp32.
__device__ __forceinline__ float log2_ratio(float x, float y, const TopArgs& a) {
  if (fabsf(x) < a.huge && fabsf(y) < a.huge) return __fmul_rn(x, a.c) - __fmul_rn(y, a.c);
  return (x - y) * a.c;
}

// Adds one value to a running maximum and sum of exponentials.
__device__ __forceinline__ void add_one(float x, const TopArgs& a, float& m, float& s) {
  const float n = max_nan(m, x);
  if (n == -INFINITY) return;
  s = (m == -INFINITY ? 0.f : s * ex2(log2_ratio(m, n, a))) + (x == -INFINITY ? 0.f : ex2(log2_ratio(x, n, a)));
  m = n;
}

template <int kTopThreads, typename T, typename Body>
__device__ __forceinline__ void for_each(const Part<T>& p, Body&& body) {
  for (uint32_t i = threadIdx.x; i < p.n_vec; i += kTopThreads) {
    float x[Vec<T>::n];
    Vec<T>::unpack(p.vec[i], x);
#pragma unroll
    for (int e = 0; e < Vec<T>::n; ++e) body(x[e], p.vec0 + i * Vec<T>::n + e);
  }
  if (threadIdx.x < p.lead) body(Vec<T>::load(p.row + threadIdx.x), threadIdx.x);
  if (threadIdx.x < p.trail) body(Vec<T>::load(p.row + p.trail0 + threadIdx.x), p.trail0 + threadIdx.x);
}

// For rows with more than kCap candidates (many equal logits): the k-th largest key two bits at a time, then what is
// above it, then the lowest indices of what equals it: 17 reads of the row, from L2.
template <int kTopThreads, typename T>
__device__ void fls_top_exact(const Part<T>& p, uint32_t top, Shared<kTopThreads>& sh) {
  constexpr int kTopWarps = kTopThreads / 32;
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t thr = 0;
  for (int shift = 30; shift >= 0; shift -= 2) {
    uint32_t n1 = 0, n2 = 0, n3 = 0;
    const uint32_t t1 = thr | (1u << shift), t2 = thr | (2u << shift), t3 = thr | (3u << shift);
    for_each<kTopThreads>(p, [&](float x, uint32_t) {
      const uint32_t k = order_key(x);
      if (k > kNegInf) { n1 += k >= t1; n2 += k >= t2; n3 += k >= t3; }
    });
    __syncthreads();
    if (threadIdx.x < 3) sh.count[threadIdx.x] = 0;
    __syncthreads();
    n1 = __reduce_add_sync(0xFFFFFFFFu, n1);
    n2 = __reduce_add_sync(0xFFFFFFFFu, n2);
    n3 = __reduce_add_sync(0xFFFFFFFFu, n3);
    if (lane == 0) { atomicAdd(&sh.count[0], n1); atomicAdd(&sh.count[1], n2); atomicAdd(&sh.count[2], n3); }
    __syncthreads();
    thr = sh.count[2] >= top ? t3 : sh.count[1] >= top ? t2 : sh.count[0] >= top ? t1 : thr;
  }
  // thr is the k-th largest key (or 0 when fewer than k may be chosen, and then all of them are above it)
  __syncthreads();
  if (threadIdx.x == 0) sh.n_cand = 0;
  __syncthreads();
  for_each<kTopThreads>(p, [&](float x, uint32_t idx) {
    const uint32_t k = order_key(x);
    if (k > kNegInf && k > thr) sh.cand[atomicAdd(&sh.n_cand, 1u)] = key64(k, idx);
  });
  __syncthreads();
  uint32_t have = sh.n_cand;
  __syncthreads();
  if (thr <= kNegInf) return;
  // equal keys in ascending index: lead, vectors, trail; one block-wide count per 512 vectors
  auto take = [&](uint32_t n, auto&& visit) {
    const uint32_t base = have;
    uint32_t x = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, x, o);
      if (lane >= uint32_t(o)) x += y;
    }
    __syncthreads();
    if (lane == 31) sh.scan[warp] = x;
    __syncthreads();
    uint32_t before = 0, total = 0;
    for (int w = 0; w < kTopWarps; ++w) { if (w < int(warp)) before += sh.scan[w]; total += sh.scan[w]; }
    uint32_t at = base + before + x - n;
    if (n) visit(at);
    have = min(base + total, top);
  };
  auto single = [&](uint32_t n, uint32_t first) {
    const bool mine = threadIdx.x < n;
    const bool eq = mine && order_key(Vec<T>::load(p.row + first + (mine ? threadIdx.x : 0))) == thr;
    take(eq ? 1u : 0u, [&](uint32_t at) { if (at < top) sh.cand[at] = key64(thr, first + threadIdx.x); });
  };
  single(p.lead, 0);
  for (uint32_t i0 = 0; i0 < p.n_vec && have < top; i0 += kTopThreads) {
    const uint32_t i = i0 + threadIdx.x;
    float x[Vec<T>::n];
    uint32_t mask = 0;
    if (i < p.n_vec) {
      Vec<T>::unpack(p.vec[i], x);
#pragma unroll
      for (int e = 0; e < Vec<T>::n; ++e) mask |= uint32_t(order_key(x[e]) == thr) << e;
    }
    take(__popc(mask), [&](uint32_t at) {
#pragma unroll
      for (int e = 0; e < Vec<T>::n; ++e)
        if ((mask >> e) & 1) {
          if (at < top) sh.cand[at] = key64(thr, p.vec0 + i * Vec<T>::n + e);
          ++at;
        }
    });
  }
  if (have < top) single(p.trail, p.trail0);
  __syncthreads();
  if (threadIdx.x == 0) sh.n_cand = have;
  __syncthreads();
}

template <typename T, int kTopThreads>
__global__ void __launch_bounds__(kTopThreads, kTopThreads == 512 ? 2 : 5) fls_top_logits_kernel(const __grid_constant__ TopArgs a) {
  constexpr int kTopWarps = kTopThreads / 32;
  __shared__ Shared<kTopThreads> sh;
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t rank, parts;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
  const uint64_t n = blockIdx.x / parts;
  constexpr uint32_t VN = Vec<T>::n;
  Part<T> p;
  p.row = static_cast<const T*>(a.logits) + n * a.stride;
  const uint32_t lead = min(a.vocab, uint32_t((16 - (reinterpret_cast<uintptr_t>(p.row) & 15)) & 15) / uint32_t(sizeof(T)));
  const uint32_t vecs = (a.vocab - lead) / VN;
  const uint32_t v0 = uint32_t(uint64_t(vecs) * rank / parts), v1 = uint32_t(uint64_t(vecs) * (rank + 1) / parts);
  p.vec0 = lead + v0 * VN;
  p.vec = reinterpret_cast<const uint4*>(p.row + p.vec0);
  p.n_vec = v1 - v0;
  p.lead = rank == 0 ? lead : 0;
  p.trail0 = lead + vecs * VN;
  p.trail = rank == parts - 1 ? a.vocab - p.trail0 : 0;

  // pass 1: maximum and sum of exponentials of what this thread reads
  float m = -INFINITY, s = 0.f;
  float seen = -INFINITY;                             // largest of the current stretch
  const f2 c2 = make_f2(a.c, a.c);
  auto batch = [&](const uint4* r, auto cnt) {
    constexpr int n_vec = decltype(cnt)::value;
    float t = Vec<T>::top(r[0]);
#pragma unroll
    for (int j = 1; j < n_vec; ++j) t = max_nan(t, Vec<T>::top(r[j]));
    seen = max_nan(seen, t);
    if (t > m || t != t) {                            // larger, or NaN, which stays
      s = m == -INFINITY ? 0.f : s * ex2(log2_ratio(m, t, a));
      m = t;
    }
    if (m == -INFINITY) return;
    if (!(fabsf(m) < a.huge)) {
#pragma unroll
      for (int j = 0; j < n_vec; ++j) {
        float x[VN];
        Vec<T>::unpack(r[j], x);
#pragma unroll
        for (int e = 0; e < int(VN); ++e) s += ex2((x[e] - m) * a.c);
      }
      return;
    }
    const float b = -__fmul_rn(m, a.c);
    const f2 b2 = make_f2(b, b);
    f2 sum[2] = {make_f2(0.f, 0.f), make_f2(0.f, 0.f)};
#pragma unroll
    for (int j = 0; j < n_vec; ++j) {
      float x[VN];
      Vec<T>::unpack(r[j], x);
#pragma unroll
      for (int e = 0; e < int(VN); e += 2) {
        float u, w;
        split(fma2(make_f2(x[e], x[e + 1]), c2, b2), u, w);
        sum[e / 2 % 2] = add2(sum[e / 2 % 2], make_f2(ex2(u), ex2(w)));
      }
    }
    float u, w;
    split(add2(sum[0], sum[1]), u, w);
    s += u + w;
  };
  // Four vectors are added up while the next four are on their way: 128 KB in flight per SM.
  constexpr uint32_t kStep = 4 * kTopThreads;
  const uint32_t full = p.n_vec / kStep;
  uint32_t shift = 0;                                 // 2^shift steps per stretch
  while ((full + (1u << shift) - 1) >> shift > kStretches) ++shift;
  const uint32_t stretches = (full + (1u << shift) - 1) >> shift;
  auto close = [&](uint32_t k) {                      // after step k
    if (((k + 1) & ((1u << shift) - 1)) == 0 || k + 1 == full) {
      sh.stretch[k >> shift][threadIdx.x] = seen;
      seen = -INFINITY;
    }
  };
  if (full) {
    uint4 r[4], q[4];
    auto fetch = [&](uint4* to, uint32_t k) {
#pragma unroll
      for (int j = 0; j < 4; ++j) to[j] = __ldg(p.vec + k * kStep + j * kTopThreads + threadIdx.x);
    };
    fetch(r, 0);
#pragma unroll 1
    for (uint32_t k = 0; k < full; k += 2) {
      if (k + 1 < full) fetch(q, k + 1);
      batch(r, std::integral_constant<int, 4>());
      close(k);
      if (k + 1 < full) {
        if (k + 2 < full) fetch(r, k + 2);
        batch(q, std::integral_constant<int, 4>());
        close(k + 1);
      }
    }
  }
  for (uint32_t i = full * kStep + threadIdx.x; i < p.n_vec; i += kTopThreads) {
    const uint4 r = p.vec[i];
    batch(&r, std::integral_constant<int, 1>());
  }
  sh.stretch[stretches][threadIdx.x] = seen;          // what is left: fewer than 4 vectors per thread
  const uint32_t key = order_key(m);                  // of the vectors only: the single elements are looked at below
  if (threadIdx.x < p.lead) add_one(Vec<T>::load(p.row + threadIdx.x), a, m, s);
  if (threadIdx.x < p.trail) add_one(Vec<T>::load(p.row + p.trail0 + threadIdx.x), a, m, s);
  if (threadIdx.x == 0) sh.n_hot = sh.n_cand = 0;

  // the block's maximum and sum
  float bm = m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) bm = max_nan(bm, __shfl_xor_sync(0xFFFFFFFFu, bm, o));
  if (lane == 0) sh.wm[warp] = bm;
  __syncthreads();
  bm = sh.wm[lane % kTopWarps];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) bm = max_nan(bm, __shfl_xor_sync(0xFFFFFFFFu, bm, o));
  float bs = m == -INFINITY ? 0.f : s * ex2(log2_ratio(m, bm, a));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) bs += __shfl_xor_sync(0xFFFFFFFFu, bs, o);
  if (lane == 0) sh.ws[warp] = bs;

  // the k-th largest of the 512 maxima, to 16 bits (any value that k maxima reach is a bound)
  uint32_t thr = 0;
#pragma unroll 1
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t t = thr | (1u << bit);
    if (__syncthreads_count(key >= t) >= int(a.top)) thr = t;
  }
  thr = max(thr, kNegInf + 1);
  const float low = key_value(thr);                   // NaN when only NaN may be chosen: the keys decide
  if (key >= thr)
    for (uint32_t g = 0; g <= stretches; ++g)
      if (!(sh.stretch[g][threadIdx.x] < low)) {
        const uint32_t at = atomicAdd(&sh.n_hot, 1u);
        if (at < kTopThreads) sh.hot[at] = g * kTopThreads + threadIdx.x;
      }
  __syncthreads();

  // pass 2: the hot stretches again
  auto offer = [&](float x, uint32_t idx) {
    if (x < low) return;
    const uint32_t k = order_key(x);
    if (k >= thr) {
      const uint32_t at = atomicAdd(&sh.n_cand, 1u);
      if (at < kCap) sh.cand[at] = key64(k, idx);
    }
  };
  const bool too_hot = sh.n_hot > uint32_t(kTopThreads);
  const uint32_t per = 4u << shift, items = too_hot ? 0 : sh.n_hot * per;
  for (uint32_t w = threadIdx.x; w < items; w += kTopThreads) {
    const uint32_t h = sh.hot[w / per], g = h / kTopThreads, t = h % kTopThreads;
    const bool whole = g < stretches;                 // the last one may be short
    const uint32_t v = ((whole ? g * per : full * 4) + w % per) * kTopThreads + t;
    if (v < (whole ? full * kStep : p.n_vec)) {
      const uint4 r = p.vec[v];
      if (Vec<T>::top(r) < low) continue;
      float x[VN];
      Vec<T>::unpack(r, x);
#pragma unroll
      for (int e = 0; e < int(VN); ++e) offer(x[e], p.vec0 + v * VN + e);
    }
  }
  if (threadIdx.x < p.lead) offer(Vec<T>::load(p.row + threadIdx.x), threadIdx.x);
  if (threadIdx.x < p.trail) offer(Vec<T>::load(p.row + p.trail0 + threadIdx.x), p.trail0 + threadIdx.x);
  __syncthreads();
  if (too_hot || sh.n_cand > kCap) fls_top_exact<kTopThreads>(p, a.top, sh);
  const uint32_t cands = sh.n_cand;

  // rank by counting: the keys are all different
  auto put = [&](uint32_t r, uint64_t k) {
    const bool none = k == 0;
    a.value[n * a.top + r] = none ? -INFINITY : key_value(uint32_t(k >> 32));
    a.index[n * a.top + r] = none ? -1 : int32_t(0xFFFFFFFFu - uint32_t(k));
  };
  for (uint32_t q = threadIdx.x; q < cands; q += kTopThreads) {
    const uint64_t k = sh.cand[q];
    uint32_t r = 0;
#pragma unroll 8
    for (uint32_t j = 0; j < cands; ++j) r += sh.cand[j] > k;
    if (r < a.top) { if (parts == 1) put(r, k); else sh.best[r] = k; }
  }
  for (uint32_t r = cands + threadIdx.x; r < a.top; r += kTopThreads) { if (parts == 1) put(r, 0); else sh.best[r] = 0; }
  if (threadIdx.x == 0) {
    float t = 0.f;
    for (int w = 0; w < kTopWarps; ++w) t += sh.ws[w];
    sh.m = bm;
    sh.s = t;
  }
  auto put_lse = [&](float mm, double ss) {
    a.lse[n] = mm == INFINITY ? INFINITY : mm == -INFINITY ? -INFINITY : float(double(mm) * a.inv_temp + log(ss));
  };
  if (parts == 1) {
    if (threadIdx.x == 0) put_lse(sh.m, double(sh.s));
    return;
  }
  // the cluster's first CTA joins the parts: a key's rank is the sum of its ranks in the sorted lists
  cluster_sync();
  if (rank == 0) {
    for (uint32_t q = threadIdx.x; q < parts * a.top; q += kTopThreads) {
      const uint32_t w = q / a.top;
      sh.cand[q] = remote_u64(remote(&sh.best[q - w * a.top], w));
    }
    if (threadIdx.x == 0) {
      float mm = -INFINITY;
      for (uint32_t w = 0; w < parts; ++w) mm = max_nan(mm, remote_f32(remote(&sh.m, w)));
      double ss = 0.0;
      for (uint32_t w = 0; w < parts; ++w) {
        const float pm = remote_f32(remote(&sh.m, w));
        if (pm != -INFINITY) ss += double(remote_f32(remote(&sh.s, w))) * double(exp2f(log2_ratio(pm, mm, a)));
      }
      put_lse(mm, ss);
    }
  }
  cluster_sync();
  if (rank != 0) return;
  for (uint32_t q = threadIdx.x; q < parts * a.top; q += kTopThreads) {
    const uint64_t k = sh.cand[q];
    uint32_t r = 0;
    for (uint32_t w = 0; w < parts; ++w) {
      const uint64_t* list = sh.cand + w * a.top;
      uint32_t lo = 0, len = a.top;                   // first entry not above k
      while (len) {
        const uint32_t half = len >> 1;
        if (list[lo + half] > k) { lo += half + 1; len -= half + 1; } else len = half;
      }
      r += lo;
    }
    if (k == 0)                                       // empty entries follow all others
      for (uint32_t j = 0; j < q; ++j) r += sh.cand[j] == 0;
    if (r < a.top) put(r, k);
  }
}

}  // namespace

extern "C" int fls_top_logits(const void* logits, uint32_t logit_dtype, uint64_t rows, uint64_t vocab, uint64_t stride, uint32_t top,
                              double temperature, float* value, int32_t* index, float* lse, void* cuda_stream) {
  if (logit_dtype != FLS_GRAD_BF16 && logit_dtype != FLS_GRAD_F32) return refuse(FLS_EINVAL, "unknown logit_dtype %u", logit_dtype);
  if (vocab < 1 || vocab > (1ull << 30)) return refuse(FLS_EINVAL, "vocab must be in 1 .. 2^30");
  if (rows > (1ull << 24)) return refuse(FLS_EINVAL, "rows > 2^24");
  if (top < 1 || top > FLS_HEAD_MAX_TOP) return refuse(FLS_EINVAL, "top must be in 1 .. %d", FLS_HEAD_MAX_TOP);
  if (!(std::isfinite(temperature) && temperature > 0.0)) return refuse(FLS_EINVAL, "temperature must be finite and > 0");
  if (stride == 0) stride = vocab;
  if (stride < vocab || stride >= (1ull << 36)) return refuse(FLS_EINVAL, "stride out of range");
  if (rows == 0) return FLS_OK;
  const uint64_t elem = logit_dtype == FLS_GRAD_F32 ? 4 : 2;
  const Span s[4] = {{logits, ((rows - 1) * stride + vocab) * elem, elem, false, "logits"},
                     {value, rows * top * 4, 4, true, "value"},
                     {index, rows * top * 4, 4, true, "index"},
                     {lse, rows * 4, 4, true, "lse"}};
  if (int rc = check_spans(s, 4)) return rc;
  const float c = float(std::min(1.4426950408889634 / temperature, 3e38));
  TopArgs a{logits, stride, uint32_t(vocab), top, c, 65536.f / c, 1.0 / temperature, value, index, lse};
  // Few rows: a row is shared by the CTAs of a cluster while there is an SM for each and a part has at least 64 KB (one row of
  // 128256 bf16, k = 64, in 1, 2, 4, 8 parts: 13.0, 12.4, 11.5, 12.7 us; 20 rows of 32000 fp32: 8.7, 10.1, 10.3, 14.1).
  uint32_t parts = 1;
  while (parts < 8 && rows * parts * 2 <= 148 && vocab * elem >= uint64_t(parts) * 2 * (64 << 10)) parts *= 2;
  // CTAs of 512 threads where an SM has one or two of them and the rows are not short, otherwise of 256, five to an SM, of
  // which some read while others rank (512 / 256 threads, us: 1 x 128256 bf16 13.0 / 17.0, 200 rows 21.1 / 22.7, 500 rows
  // 41.2 / 35.0, 4096 rows 247 / 204; 220 x 20000 bf16 9.8 / 11.0; 100 x 5000 bf16 6.9 / 6.4; 333 x 50257 fp32 24.6 / 19.4).
  const int threads = parts > 1 || (rows <= 222 && vocab * elem >= (16 << 10)) ? 512 : 256;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(uint32_t(rows) * parts);
  cfg.blockDim = dim3(threads);
  cfg.stream = static_cast<cudaStream_t>(cuda_stream);
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = parts;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  const bool f32 = logit_dtype == FLS_GRAD_F32;
  const cudaError_t e = threads == 512 ? (f32 ? cudaLaunchKernelEx(&cfg, fls_top_logits_kernel<float, 512>, a)
                                              : cudaLaunchKernelEx(&cfg, fls_top_logits_kernel<uint16_t, 512>, a))
                                       : (f32 ? cudaLaunchKernelEx(&cfg, fls_top_logits_kernel<float, 256>, a)
                                              : cudaLaunchKernelEx(&cfg, fls_top_logits_kernel<uint16_t, 256>, a));
  if (e != cudaSuccess) return refuse(FLS_ECUDA, "fls_top_logits: %s", cudaGetErrorString(e));
  return FLS_OK;
}
