// fls_embed_*: rows of an embedding table by token, and the gradient of that table.
//
// The gradient of row v is the sum of the output gradients of all tokens equal to v.  Sums of a fixed order need the tokens'
// positions sorted by token: a stable radix sort of (token, position), most significant key V for positions that take no
// part.  The sorted positions are cut into chunks of equal length, whatever tokens they hold, so that a token that makes up
// half of the batch is shared by many warps; a warp sums one chunk for 256 columns and writes a row of the gradient whenever
// the token changes.  Sums of a token that reaches beyond the chunk go to the workspace and are joined in ascending order.
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

constexpr int kSortThreads = 256, kSortRounds = 16;
constexpr uint32_t kSortTile = kSortThreads * kSortRounds;   // positions per CTA of the sort
constexpr uint32_t kMaxRadix = 512;
constexpr uint32_t kMaxChunks = 2048;
constexpr uint32_t kSlab = 256;                              // columns of a warp: eight per lane

constexpr uint64_t up(uint64_t x, uint64_t q) { return (x + q - 1) / q * q; }

struct EmbedCall {
  const int64_t* token;
  uint64_t tokens, vocab;
  int64_t ignore;
  uint32_t dim, dp;               // dp: floats between two rows of partial sums
  const uint16_t* weight; uint64_t weight_stride;
  void* out; uint64_t out_stride;
  const void* grad_out; uint64_t grad_out_stride;
  void* grad_weight; uint64_t grad_weight_stride;
  float scale;
  uint32_t accumulate;
  uint32_t grad_size, zero_vec;   // bytes of an element; rows of grad_weight start on 16-byte boundaries
  uint32_t chunk, chunks;
  uint2* pairs[2];                // (key, position)
  uint32_t* counts;               // [radix][tiles]
  uint32_t tiles;
  float* part;                    // [2 * chunks][dp]: of the token a chunk begins with, of the one it ends with
};

// V stands for a position that takes no part: ignored, or outside the table.
__device__ __forceinline__ uint32_t key_of(const EmbedCall& c, uint64_t i) {
  const int64_t t = c.token[i];
  return t != c.ignore && t >= 0 && uint64_t(t) < c.vocab ? uint32_t(t) : uint32_t(c.vocab);
}

// ------------------------------------------------------------------------------------------------ lookup
// A warp takes a row and 1024 of its columns.  VEC: cells of eight columns start on 16-byte boundaries on both sides.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) fls_embed_lookup_kernel(const __grid_constant__ EmbedCall c) {
  const uint64_t n = uint64_t(blockIdx.x) * 8 + threadIdx.x / 32;
  const uint32_t lane = threadIdx.x % 32, col0 = blockIdx.y * 1024;
  if (n >= c.tokens) return;
  const int64_t t = c.token[n];
  T* out = static_cast<T*>(c.out) + n * c.out_stride;
  const bool inside = t >= 0 && uint64_t(t) < c.vocab;
  const bool live = t != c.ignore && inside;
  const float other = t == c.ignore ? 0.f : __int_as_float(0x7FC00000);
  const uint16_t* w = c.weight + (live ? uint64_t(t) * c.weight_stride : 0);
  if (VEC) {
    uint4 raw[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t col = col0 + k * kSlab + lane * 8;
      raw[k] = make_uint4(0, 0, 0, 0);
      if (live && col + 8 <= c.dim) raw[k] = Elem<uint16_t>::load_raw(w + col);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t col = col0 + k * kSlab + lane * 8;
      if (col + 8 <= c.dim) {
        float x[8];
        Elem<uint16_t>::unpack(raw[k], x);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = live ? x[j] * c.scale : other;
        Elem<T>::store8(out + col, x);
      } else {
        for (uint32_t j = col; j < c.dim; ++j) Elem<T>::put(out + j, live ? Elem<uint16_t>::get(w + j) * c.scale : other);
      }
    }
  } else {
    const uint32_t end = min(c.dim, col0 + 1024);
#pragma unroll 8
    for (uint32_t j = col0 + lane; j < end; j += 32) Elem<T>::put(out + j, live ? Elem<uint16_t>::get(w + j) * c.scale : other);
  }
}

// ------------------------------------------------------------------------------------------------ sort
// One pass sorts by `bits` bits of the key from `shift` on; the first takes its keys from the tokens.
struct SortPass { uint32_t shift, bits, first, from; };

__device__ __forceinline__ uint2 sort_item(const EmbedCall& c, const SortPass& p, uint64_t i) {
  return p.first ? make_uint2(key_of(c, i), uint32_t(i)) : c.pairs[p.from][i];
}

__global__ void __launch_bounds__(kSortThreads) fls_embed_count_kernel(const __grid_constant__ EmbedCall c, const SortPass p) {
  __shared__ uint32_t count[kMaxRadix];
  const uint32_t radix = 1u << p.bits;
  for (uint32_t d = threadIdx.x; d < radix; d += kSortThreads) count[d] = 0;
  pdl_launch();
  pdl_wait();
  __syncthreads();
  for (int r = 0; r < kSortRounds; ++r) {
    const uint64_t i = uint64_t(blockIdx.x) * kSortTile + r * kSortThreads + threadIdx.x;
    if (i < c.tokens) atomicAdd(&count[(sort_item(c, p, i).x >> p.shift) & (radix - 1)], 1u);
  }
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < radix; d += kSortThreads) c.counts[uint64_t(d) * c.tiles + blockIdx.x] = count[d];
}

// Exclusive sums of counts, in place, by one CTA.
__global__ void __launch_bounds__(1024) fls_embed_scan_kernel(const __grid_constant__ EmbedCall c, const SortPass p) {
  __shared__ uint32_t warp_sum[32];
  const uint64_t n = uint64_t(c.tiles) << p.bits;
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  uint32_t before = 0;
  pdl_launch();
  pdl_wait();
  for (uint64_t base = 0; base < n; base += 1024) {
    const uint64_t i = base + threadIdx.x;
    const uint32_t own = i < n ? c.counts[i] : 0;
    uint32_t x = own;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const uint32_t y = __shfl_up_sync(~0u, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) warp_sum[warp] = x;
    __syncthreads();
    if (warp == 0) {
      uint32_t s = warp_sum[lane];
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const uint32_t y = __shfl_up_sync(~0u, s, o);
        if (lane >= o) s += y;
      }
      warp_sum[lane] = s;
    }
    __syncthreads();
    if (i < n) c.counts[i] = before + (warp ? warp_sum[warp - 1] : 0) + x - own;
    before += warp_sum[31];
    __syncthreads();
  }
}

// A warp owns kSortRounds * 32 neighbouring positions and takes them in order, so that equal digits keep it.
__global__ void __launch_bounds__(kSortThreads) fls_embed_scatter_kernel(const __grid_constant__ EmbedCall c, const SortPass p) {
  constexpr int kWarps = kSortThreads / 32;
  __shared__ uint32_t count[kWarps][kMaxRadix];
  const uint32_t radix = 1u << p.bits, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  for (uint32_t d = threadIdx.x; d < kWarps * kMaxRadix; d += kSortThreads) (&count[0][0])[d] = 0;
  pdl_launch();
  pdl_wait();
  __syncthreads();
  uint2 item[kSortRounds];
  uint32_t rank[kSortRounds];
  const uint64_t first = uint64_t(blockIdx.x) * kSortTile + warp * (kSortRounds * 32);
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const uint64_t i = first + r * 32 + lane;
    item[r] = i < c.tokens ? sort_item(c, p, i) : make_uint2(~0u, 0);
  }
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const bool in = first + r * 32 + lane < c.tokens;
    const uint32_t d = in ? (item[r].x >> p.shift) & (radix - 1) : kMaxRadix;     // not a digit: apart from all others
    const uint32_t same = __match_any_sync(~0u, d);
    rank[r] = in ? count[warp][d] + __popc(same & ((1u << lane) - 1)) : 0;
    __syncwarp();
    if (in && (same >> lane) == 1) count[warp][d] = rank[r] + 1;                  // the last of them
    __syncwarp();
  }
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < radix; d += kSortThreads) {
    uint32_t at = c.counts[uint64_t(d) * c.tiles + blockIdx.x];
    for (int w = 0; w < kWarps; ++w) {
      const uint32_t k = count[w][d];
      count[w][d] = at;
      at += k;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    if (first + r * 32 + lane >= c.tokens) continue;
    c.pairs[p.from ^ 1][count[warp][(item[r].x >> p.shift) & (radix - 1)] + rank[r]] = item[r];
  }
}

// ------------------------------------------------------------------------------------------------ rows without a token
constexpr uint32_t kFillRows = 8192;                       // rows of one look at the tokens
#ifndef FLS_FILL
#define FLS_FILL 147
#endif
constexpr uint32_t kFillCtas = FLS_FILL;

__device__ __forceinline__ uint32_t first_at_least(const uint2* pairs, uint32_t n, uint64_t key) {
  uint32_t lo = 0, len = n;
  while (len) {
    const uint32_t half = len / 2;
    if (pairs[lo + half].x < key) { lo += half + 1; len -= half + 1; } else len = half;
  }
  return lo;
}

// Zeros to the rows v0 .. v1 - 1 whose bit in `there` is not set, a warp each.
__device__ __forceinline__ void fill_rows(const EmbedCall& c, const uint32_t* there, uint64_t v0, uint64_t v1) {
  const uint32_t lane = threadIdx.x % 32, warps = blockDim.x / 32;
  for (uint64_t v = v0 + threadIdx.x / 32; v < v1; v += warps) {
    const uint32_t r = uint32_t(v - v0);
    if (there[r / 32] >> (r % 32) & 1) continue;
    char* row = static_cast<char*>(c.grad_weight) + v * c.grad_weight_stride * c.grad_size;
    const uint32_t bytes = c.dim * c.grad_size, whole = c.zero_vec ? bytes / 16 * 16 : 0;
    for (uint32_t j = lane * 16; j < whole; j += 512) __stcs(reinterpret_cast<uint4*>(row + j), make_uint4(0, 0, 0, 0));
    for (uint32_t j = whole + lane * 2; j < bytes; j += 64) *reinterpret_cast<uint16_t*>(row + j) = 0;
  }
}

__global__ void __launch_bounds__(256) fls_embed_fill_kernel(const __grid_constant__ EmbedCall c, const uint2* pairs, uint64_t rows_per_cta) {
  __shared__ uint32_t there[kFillRows / 32], range[2];
  pdl_launch();
  pdl_wait();
  const uint64_t begin = blockIdx.x * rows_per_cta, end = min(c.vocab, begin + rows_per_cta);
  for (uint64_t v0 = begin; v0 < end; v0 += kFillRows) {
    const uint64_t v1 = min(end, v0 + kFillRows);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kFillRows / 32; i += 256) there[i] = 0;
    if (threadIdx.x < 2) range[threadIdx.x] = c.tokens ? first_at_least(pairs, uint32_t(c.tokens), threadIdx.x ? v1 : v0) : 0;
    __syncthreads();
    for (uint32_t p = range[0] + threadIdx.x; p < range[1]; p += 256) {
      const uint32_t r = pairs[p].x - uint32_t(v0);
      atomicOr(&there[r / 32], 1u << (r % 32));
    }
    __syncthreads();
    fill_rows(c, there, v0, v1);
  }
}

// ------------------------------------------------------------------------------------------------ sort of up to 2^17 tokens
// The first cluster of the grid sorts while the others write zeros to the rows without a token, which they find for
// themselves by looking through the tokens.  A warp of the sort owns up to 16 * 32 neighbouring positions; per pass it ranks
// them among its own by digit, the CTA adds its warps up, and the CTAs of the cluster read each other's digit counts from
// distributed shared memory.
constexpr int kClusterThreads = 1024, kClusterRounds = 16;
constexpr uint32_t kCluster = 8;
constexpr uint32_t kOneCta = kClusterThreads * kClusterRounds;

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t remote_u32(const uint32_t* p, uint32_t rank) {
  uint32_t a, x;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(uint32_t(__cvta_generic_to_shared(p))), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(a) : "memory");
  return x;
}

struct SortShared {
  uint16_t count[kClusterThreads / 32][kMaxRadix];   // of a warp, then of the warps before it
  uint32_t total[kMaxRadix];                         // of the CTA, read by the cluster
  uint32_t base[kMaxRadix];                          // where the CTA's first item of a digit goes
  uint32_t scan[kMaxRadix / 32];
};

template <int ROUNDS>
__device__ __forceinline__ void sort_tokens(const EmbedCall& c, SortShared& sh, uint32_t bits, uint32_t passes, uint32_t ctas) {
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, rank = blockIdx.x, n = uint32_t(c.tokens);
  const uint32_t per = (bits + passes - 1) / passes;
  const uint32_t first = (rank * (kClusterThreads / 32) + warp) * (ROUNDS * 32) + lane;
  for (uint32_t pass = 0; pass < passes; ++pass) {
    const uint32_t shift = pass * per, radix = 1u << min(per, bits - shift);
    uint2 item[ROUNDS];
    uint32_t at[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      const uint32_t i = first + r * 32;
      item[r] = i >= n ? make_uint2(0, 0) : pass ? __ldcg(&c.pairs[(pass - 1) & 1][i]) : make_uint2(key_of(c, i), i);
    }
    for (uint32_t d = threadIdx.x; d < kClusterThreads / 32 * kMaxRadix / 2; d += kClusterThreads) reinterpret_cast<uint32_t*>(sh.count)[d] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      const bool in = first + r * 32 < n;
      if (__any_sync(~0u, in)) {
        const uint32_t d = in ? (item[r].x >> shift) & (radix - 1) : kMaxRadix;      // not a digit: apart from all others
        const uint32_t same = __match_any_sync(~0u, d);
        at[r] = in ? sh.count[warp][d] + __popc(same & ((1u << lane) - 1)) : 0;
        __syncwarp();
        if (in && (same >> lane) == 1) sh.count[warp][d] = uint16_t(at[r] + 1);      // the last of them
        __syncwarp();
      }
    }
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < radix; d += kClusterThreads) {
      uint32_t sum = 0;
#pragma unroll 8
      for (int w = 0; w < kClusterThreads / 32; ++w) {
        const uint32_t k = sh.count[w][d];
        sh.count[w][d] = uint16_t(sum);
        sum += k;
      }
      sh.total[d] = sum;
    }
    if (ctas > 1) cluster_sync(); else __syncthreads();
    uint32_t before = 0, all = 0, x = 0;
    if (threadIdx.x < kMaxRadix) {
      if (threadIdx.x < radix)
        for (uint32_t q = 0; q < ctas; ++q) {
          const uint32_t k = ctas > 1 ? remote_u32(&sh.total[threadIdx.x], q) : sh.total[threadIdx.x];
          all += k;
          if (q < rank) before += k;
        }
      x = all;
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const uint32_t y = __shfl_up_sync(~0u, x, o);
        if (lane >= o) x += y;
      }
      if (lane == 31) sh.scan[warp] = x;
    }
    __syncthreads();
    if (threadIdx.x < radix) {
      for (uint32_t w = 0; w < warp; ++w) before += sh.scan[w];
      sh.base[threadIdx.x] = before + x - all;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      if (first + r * 32 >= n) continue;
      const uint32_t d = (item[r].x >> shift) & (radix - 1);
      c.pairs[pass & 1][sh.base[d] + sh.count[warp][d] + at[r]] = item[r];
    }
    if (ctas > 1) cluster_sync(); else __syncthreads();
  }
}

__global__ void __launch_bounds__(kClusterThreads, 1)
    fls_embed_sort_kernel(const __grid_constant__ EmbedCall c, uint32_t bits, uint32_t passes, uint32_t ctas, uint64_t rows_per_cta) {
  __shared__ union { SortShared sort; uint32_t there[kFillRows / 32]; } sh;
  pdl_launch();
  if (blockIdx.x < ctas) {
    const uint32_t rounds = uint32_t((c.tokens + ctas * kClusterThreads - 1) / (ctas * kClusterThreads));
    if (rounds <= 1) sort_tokens<1>(c, sh.sort, bits, passes, ctas);
    else if (rounds <= 4) sort_tokens<4>(c, sh.sort, bits, passes, ctas);
    else if (rounds <= 8) sort_tokens<8>(c, sh.sort, bits, passes, ctas);
    else sort_tokens<16>(c, sh.sort, bits, passes, ctas);
    return;
  }
  const uint64_t begin = (blockIdx.x - ctas) * rows_per_cta, end = min(c.vocab, begin + rows_per_cta);
  for (uint64_t v0 = begin; v0 < end; v0 += kFillRows) {
    const uint64_t v1 = min(end, v0 + kFillRows);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kFillRows / 32; i += kClusterThreads) sh.there[i] = 0;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < uint32_t(c.tokens); i += kClusterThreads) {
      const uint32_t v = key_of(c, i);
      if (v >= v0 && v < v1) atomicOr(&sh.there[(v - uint32_t(v0)) / 32], 1u << ((v - uint32_t(v0)) % 32));
    }
    __syncthreads();
    fill_rows(c, sh.there, v0, v1);
  }
}

// ------------------------------------------------------------------------------------------------ sums
// The eight columns of a lane: neighbours (VEC) or 32 apart.
template <bool VEC>
__device__ __forceinline__ uint32_t column(uint32_t slab, uint32_t lane, int j) {
  return slab * kSlab + (VEC ? lane * 8 + j : lane + 32 * j);
}

template <typename T, bool VEC>
__device__ __forceinline__ void load_columns(const T* row, uint32_t slab, uint32_t lane, uint32_t dim, float (&x)[8]) {
  const uint32_t col = column<VEC>(slab, lane, 0);
  if (VEC && col + 8 <= dim) {
    load8(row + col, x);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t k = column<VEC>(slab, lane, j);
    x[j] = k < dim ? Elem<T>::get(row + k) : 0.f;
  }
}

template <typename G, bool VEC>
__device__ __forceinline__ void write_row(const EmbedCall& c, uint32_t key, uint32_t slab, uint32_t lane, const float (&sum)[8]) {
  G* row = static_cast<G*>(c.grad_weight) + uint64_t(key) * c.grad_weight_stride;
  float x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = sum[j] * c.scale;
  if (c.accumulate) {
    float old[8];
    load_columns<G, VEC>(row, slab, lane, c.dim, old);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] += old[j];
  }
  const uint32_t col = column<VEC>(slab, lane, 0);
  if (VEC && col + 8 <= c.dim) {
    Elem<G>::store8(row + col, x);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t k = column<VEC>(slab, lane, j);
    if (k < c.dim) Elem<G>::put(row + k, x[j]);
  }
}

template <typename T, typename G, bool VEC>
__global__ void __launch_bounds__(256) fls_embed_sum_kernel(const __grid_constant__ EmbedCall c, const uint2* pairs) {
  const uint32_t lane = threadIdx.x % 32, chunk = blockIdx.x * 8 + threadIdx.x / 32, slab = blockIdx.y;
  pdl_launch();
  pdl_wait();
  if (chunk >= c.chunks) return;
  const uint32_t n = uint32_t(c.tokens), none = uint32_t(c.vocab);
  const uint32_t begin = chunk * c.chunk, end = min(n, begin + c.chunk);
  float sum[8] = {};
  uint32_t now = pairs[begin].x;
  if (now == none) return;
  bool from_left = begin > 0 && pairs[begin - 1].x == now;
  for (uint32_t p0 = begin; p0 < end; p0 += 8) {
    uint2 pair[8];
    float x[8][8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      pair[u] = p0 + u < end ? pairs[p0 + u] : make_uint2(none, 0);
      if (pair[u].x != none) load_columns<T, VEC>(static_cast<const T*>(c.grad_out) + pair[u].y * c.grad_out_stride, slab, lane, c.dim, x[u]);
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (p0 + u >= end) break;
      if (pair[u].x != now) {
        if (from_left) {
#pragma unroll
          for (int j = 0; j < 8; ++j) c.part[uint64_t(2 * chunk) * c.dp + column<VEC>(slab, lane, j)] = sum[j];
        } else {
          write_row<G, VEC>(c, now, slab, lane, sum);
        }
        from_left = false;
        now = pair[u].x;
        if (now == none) return;                            // nothing follows
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = 0.f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] += x[u][j];
    }
  }
  const bool to_right = end < n && pairs[end].x == now;
  if (!from_left && !to_right) {
    write_row<G, VEC>(c, now, slab, lane, sum);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) c.part[uint64_t(2 * chunk + (from_left ? 0 : 1)) * c.dp + column<VEC>(slab, lane, j)] = sum[j];
}

// A CTA for every chunk whose last token begins in it and goes on in the next: the sums of that token, in order of the chunks
// inside each of eight warps, then of the warps.
template <typename G, bool VEC>
__global__ void __launch_bounds__(256) fls_embed_join_kernel(const __grid_constant__ EmbedCall c, const uint2* pairs) {
  __shared__ float sums[8][kSlab];
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, chunk = blockIdx.x, slab = blockIdx.y;
  const uint32_t n = uint32_t(c.tokens), none = uint32_t(c.vocab);
  pdl_wait();
  const uint32_t begin = chunk * c.chunk, end = begin + c.chunk;
  if (end >= n) return;
  const uint32_t key = pairs[end].x;
  if (key == none || pairs[end - 1].x != key) return;
  if (pairs[begin].x == key && begin > 0 && pairs[begin - 1].x == key) return;   // began before this chunk
  uint32_t more = 0;                                                             // chunks after this one that begin with the token
  for (;;) {
    const uint64_t p = uint64_t(end) + uint64_t(more + threadIdx.x) * c.chunk;
    const int got = __syncthreads_count(p < n && pairs[p].x == key);
    more += got;
    if (got < 256) break;
  }
  float sum[8] = {};
  for (uint32_t k = warp; k <= more; k += 8) {
    const float* row = c.part + uint64_t(k ? 2 * (chunk + k) : 2 * chunk + 1) * c.dp;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] += row[column<VEC>(slab, lane, j)];
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) sums[warp][lane + 32 * j] = sum[j];
  __syncthreads();
  if (warp) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    sum[j] = sums[0][lane + 32 * j];
    for (int w = 1; w < 8; ++w) sum[j] += sums[w][lane + 32 * j];
  }
  write_row<G, VEC>(c, key, slab, lane, sum);
}

// ------------------------------------------------------------------------------------------------ host
template <typename... P, typename... A>
cudaError_t launch_clusters(void (*kernel)(P...), dim3 grid, uint32_t cluster, uint32_t threads, bool dependent, cudaStream_t s, const A&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = s;
  cudaLaunchAttribute at[2] = {};
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = dependent ? 1 : 0;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}
template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, uint32_t threads, bool dependent, cudaStream_t s, const A&... args) {
  return launch_clusters(kernel, grid, 1, threads, dependent, s, args...);
}

struct Regions { uint64_t pairs[2], counts, part, total; };

uint32_t chunk_of(uint64_t tokens) {
  uint32_t c = 8;
  while (uint64_t(c) * kMaxChunks < tokens) c *= 2;
  return c;
}

Regions regions(const fls_embed_desc& d) {
  Regions r{};
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) { const uint64_t o = at; at += up(bytes, 256); return o; };
  if (d.grads) {
    const uint64_t n = std::max<uint64_t>(d.max_tokens, 1);
    r.pairs[0] = take(n * 8);
    r.pairs[1] = take(n * 8);
    r.counts = take(up(n, kSortTile) / kSortTile * kMaxRadix * 4);
    r.part = take(2 * std::min<uint64_t>(kMaxChunks, up(n, 8) / 8) * up(d.dim, kSlab) * 4);
  }
  r.total = at;
  return r;
}

bool known(uint32_t dtype) { return dtype == FLS_GRAD_BF16 || dtype == FLS_GRAD_F32; }
uint64_t size_of(uint32_t dtype) { return dtype == FLS_GRAD_F32 ? 4 : 2; }
// Whether every row starts on a 16-byte boundary.
bool cells(const void* p, uint64_t stride, uint64_t elem) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * elem % 16 == 0; }
uint64_t span_bytes(uint64_t rows, uint64_t cols, uint64_t stride, uint64_t elem) { return rows ? ((rows - 1) * stride + cols) * elem : 0; }

}  // namespace

struct fls_embed {
  fls_embed_desc desc{};
  Regions reg{};
  uint64_t launches = 0;
};

namespace {

int check_common(const fls_embed* e, const fls_embed_io* io) {
  if (!e || !io) return refuse(FLS_EINVAL, "null argument");
  const fls_embed_desc& d = e->desc;
  if (io->reserved) return refuse(FLS_EINVAL, "reserved must be 0");
  if (io->tokens > d.max_tokens)
    return refuse(FLS_EINVAL, "tokens (%llu) > max_tokens (%llu)", (unsigned long long)io->tokens, (unsigned long long)d.max_tokens);
  if (io->accumulate > 1) return refuse(FLS_EINVAL, "accumulate must be 0 or 1");
  if (!std::isfinite(io->scale) || std::fabs(io->scale) > 3.4028234663852886e38) return refuse(FLS_EINVAL, "scale must be finite in fp32");
  const uint64_t strides[4] = {io->weight_stride, io->out_stride, io->grad_out_stride, io->grad_weight_stride};
  static const char* const names[4] = {"weight_stride", "out_stride", "grad_out_stride", "grad_weight_stride"};
  for (int i = 0; i < 4; ++i) {
    if (strides[i] && strides[i] < d.dim) return refuse(FLS_EINVAL, "%s (%llu) < dim (%u)", names[i], (unsigned long long)strides[i], d.dim);
    if (strides[i] >= (1ull << 31)) return refuse(FLS_EINVAL, "%s out of range", names[i]);
  }
  return FLS_OK;
}

EmbedCall call_of(const fls_embed* e, const fls_embed_io* io) {
  const fls_embed_desc& d = e->desc;
  EmbedCall c{};
  c.token = io->token;
  c.tokens = io->tokens;
  c.vocab = d.vocab;
  c.ignore = io->ignore_token;
  c.dim = d.dim;
  c.dp = uint32_t(up(d.dim, kSlab));
  c.weight = static_cast<const uint16_t*>(io->weight);
  c.weight_stride = io->weight_stride ? io->weight_stride : d.dim;
  c.out = io->out;
  c.out_stride = io->out_stride ? io->out_stride : d.dim;
  c.grad_out = io->grad_out;
  c.grad_out_stride = io->grad_out_stride ? io->grad_out_stride : d.dim;
  c.grad_weight = io->grad_weight;
  c.grad_weight_stride = io->grad_weight_stride ? io->grad_weight_stride : d.dim;
  c.scale = float(io->scale);
  c.accumulate = io->accumulate;
  return c;
}

#define FLS_LAUNCH(call)                                                                                 \
  do {                                                                                                   \
    const cudaError_t e_ = (call);                                                                       \
    if (e_ != cudaSuccess) return refuse(FLS_ECUDA, "embedding kernel: %s", cudaGetErrorString(e_));     \
    ++e->launches;                                                                                       \
  } while (0)

template <typename T, typename G, bool VEC>
int run_grad(fls_embed* e, EmbedCall& c, cudaStream_t s) {
  const uint64_t n = c.tokens;
  uint32_t bits = 1, at = 0;
  const uint2* sorted = nullptr;
  while (c.vocab >> bits) ++bits;                         // of keys 0 .. V
  const uint32_t passes = (bits + 8) / 9, per = (bits + passes - 1) / passes;
  if (n && n <= uint64_t(kOneCta) * kCluster) {
    const uint32_t ctas = n <= kOneCta ? 1 : kCluster;
    uint64_t per_cta = 0;
    uint32_t fill = 0;
    if (!c.accumulate) {
      per_cta = std::max<uint64_t>(1, (c.vocab + kFillCtas - 1) / kFillCtas);
      fill = uint32_t(up((c.vocab + per_cta - 1) / per_cta, ctas));
    }
    FLS_LAUNCH(launch_clusters(fls_embed_sort_kernel, ctas + fill, ctas, kClusterThreads, false, s, c, bits, passes, ctas, per_cta));
    sorted = c.pairs[(passes - 1) & 1];
  } else {
    bool dependent = false;
    c.tiles = uint32_t((n + kSortTile - 1) / kSortTile);
    for (uint32_t p = 0; n && p < passes; ++p) {
      const SortPass sp{p * per, std::min(per, bits - p * per), p == 0, at};
      FLS_LAUNCH(launch(fls_embed_count_kernel, c.tiles, kSortThreads, dependent, s, c, sp));
      dependent = true;
      FLS_LAUNCH(launch(fls_embed_scan_kernel, 1, 1024, true, s, c, sp));
      FLS_LAUNCH(launch(fls_embed_scatter_kernel, c.tiles, kSortThreads, true, s, c, sp));
      at ^= 1;
    }
    sorted = c.pairs[at];
    if (!c.accumulate) {
      const uint64_t per_cta = std::max<uint64_t>(1, (c.vocab + 148 * 8 - 1) / (148 * 8));
      const uint32_t ctas = uint32_t((c.vocab + per_cta - 1) / per_cta);
      FLS_LAUNCH((launch(fls_embed_fill_kernel, ctas, 256, dependent, s, c, sorted, per_cta)));
    }
  }
  if (n) {
    c.chunk = chunk_of(n);
    c.chunks = uint32_t((n + c.chunk - 1) / c.chunk);
    const uint32_t slabs = (c.dim + kSlab - 1) / kSlab;
    FLS_LAUNCH((launch(fls_embed_sum_kernel<T, G, VEC>, dim3((c.chunks + 7) / 8, slabs), 256, true, s, c, sorted)));
    if (c.chunks > 1) FLS_LAUNCH((launch(fls_embed_join_kernel<G, VEC>, dim3(c.chunks - 1, slabs), 256, true, s, c, sorted)));
  }
  return FLS_OK;
}

}  // namespace

extern "C" {

int fls_embed_create(const fls_embed_desc* desc, fls_embed** out) {
  if (out) *out = nullptr;
  if (!desc || !out) return refuse(FLS_EINVAL, "null argument");
  if (desc->reserved) return refuse(FLS_EINVAL, "reserved must be 0");
  if (desc->max_tokens > (1ull << 24)) return refuse(FLS_EINVAL, "max_tokens > 2^24");
  if (desc->vocab < 1 || desc->vocab > (1ull << 30)) return refuse(FLS_EINVAL, "vocab must be in 1 .. 2^30");
  if (desc->dim < 1 || desc->dim > 65536) return refuse(FLS_EINVAL, "dim must be in 1 .. 65536");
  if (desc->grads > 1) return refuse(FLS_EINVAL, "grads must be 0 or 1");
  if (!known(desc->act_dtype)) return refuse(FLS_EINVAL, "unknown act_dtype %u", desc->act_dtype);
  if (!known(desc->grad_dtype)) return refuse(FLS_EINVAL, "unknown grad_dtype %u", desc->grad_dtype);
  fls_embed* e = new (std::nothrow) fls_embed;
  if (!e) return refuse(FLS_ESTATE, "out of host memory");
  e->desc = *desc;
  e->reg = regions(*desc);
  *out = e;
  return FLS_OK;
}

int fls_embed_query(const fls_embed* embed, fls_embed_layout* out) {
  if (!embed || !out) return refuse(FLS_EINVAL, "null argument");
  out->workspace_bytes = embed->reg.total;
  return FLS_OK;
}

int fls_embed_destroy(fls_embed* embed) {
  delete embed;
  return FLS_OK;
}

int fls_embed_lookup(fls_embed* e, const fls_embed_io* io, void* cuda_stream) {
  if (int rc = check_common(e, io)) return rc;
  const fls_embed_desc& d = e->desc;
  EmbedCall c = call_of(e, io);
  const uint64_t n = c.tokens, es = size_of(d.act_dtype);
  const Span s[3] = {{io->token, n * 8, 8, false, "token"},
                     {io->weight, n ? span_bytes(d.vocab, d.dim, c.weight_stride, 2) : 0, 2, false, "weight"},
                     {io->out, span_bytes(n, d.dim, c.out_stride, es), es, true, "out"}};
  if (int rc = check_spans(s, 3)) return rc;
  if (!n) return FLS_OK;
  const dim3 grid(uint32_t((n + 7) / 8), (d.dim + 1023) / 1024);
  const bool vec = cells(c.weight, c.weight_stride, 2) && cells(c.out, c.out_stride, es), f32 = d.act_dtype == FLS_GRAD_F32;
  auto kernel = f32 ? (vec ? fls_embed_lookup_kernel<float, true> : fls_embed_lookup_kernel<float, false>)
                    : (vec ? fls_embed_lookup_kernel<uint16_t, true> : fls_embed_lookup_kernel<uint16_t, false>);
  FLS_LAUNCH(launch(kernel, grid, 256, false, static_cast<cudaStream_t>(cuda_stream), c));
  return FLS_OK;
}

int fls_embed_grad(fls_embed* e, const fls_embed_io* io, void* cuda_stream) {
  if (int rc = check_common(e, io)) return rc;
  const fls_embed_desc& d = e->desc;
  if (!d.grads) return refuse(FLS_EINVAL, "the embedding was created without grads");
  EmbedCall c = call_of(e, io);
  const uint64_t n = c.tokens, es = size_of(d.act_dtype), gs = size_of(d.grad_dtype);
  if (io->workspace && io->workspace_bytes < e->reg.total)
    return refuse(FLS_ESIZE, "workspace has %llu bytes, %llu needed", (unsigned long long)io->workspace_bytes, (unsigned long long)e->reg.total);
  const Span s[4] = {{io->token, n * 8, 8, false, "token"},
                     {io->grad_out, span_bytes(n, d.dim, c.grad_out_stride, es), es, false, "grad_out"},
                     {io->grad_weight, span_bytes(d.vocab, d.dim, c.grad_weight_stride, gs), gs, true, "grad_weight"},
                     {io->workspace, e->reg.total, 256, true, "workspace"}};
  if (int rc = check_spans(s, 4)) return rc;
  if (!n && c.accumulate) return FLS_OK;
  char* ws = static_cast<char*>(io->workspace);
  for (int i = 0; i < 2; ++i) c.pairs[i] = reinterpret_cast<uint2*>(ws + e->reg.pairs[i]);
  c.counts = reinterpret_cast<uint32_t*>(ws + e->reg.counts);
  c.part = reinterpret_cast<float*>(ws + e->reg.part);
  c.grad_size = uint32_t(gs);
  c.zero_vec = cells(c.grad_weight, c.grad_weight_stride, gs);
  const bool vec = c.zero_vec && (!n || cells(c.grad_out, c.grad_out_stride, es));
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (d.act_dtype == FLS_GRAD_F32) {
    if (d.grad_dtype == FLS_GRAD_F32) return vec ? run_grad<float, float, true>(e, c, st) : run_grad<float, float, false>(e, c, st);
    return vec ? run_grad<float, uint16_t, true>(e, c, st) : run_grad<float, uint16_t, false>(e, c, st);
  }
  if (d.grad_dtype == FLS_GRAD_F32) return vec ? run_grad<uint16_t, float, true>(e, c, st) : run_grad<uint16_t, float, false>(e, c, st);
  return vec ? run_grad<uint16_t, uint16_t, true>(e, c, st) : run_grad<uint16_t, uint16_t, false>(e, c, st);
}

int fls_embed_get_launch_count(const fls_embed* embed, uint64_t* launches) {
  if (!embed || !launches) return refuse(FLS_EINVAL, "null argument");
  *launches = embed->launches;
  return FLS_OK;
}

}  // extern "C"
