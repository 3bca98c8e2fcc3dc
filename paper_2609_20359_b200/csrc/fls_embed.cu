// fls_embed_*: rows of an embedding table by token, and the gradient of that table.
//
// The gradient of row v is the sum of the output gradients of all tokens equal to v.  Sums of a fixed order need the tokens'
// positions sorted by token: a stable radix sort of (token, position), most significant key V for positions that take no
// part.  The sorted positions are cut into chunks of equal length, whatever tokens they hold, so that a token that makes up
// half of the batch is shared by many warps; a warp sums one chunk for 256 columns and writes a row of the gradient whenever
// the token changes.  Sums of a token that reaches beyond the chunk go to the workspace and are joined in ascending order.
//
// Bound by memory, and of that mostly by the zeros of rows without a token, which need no sums: 8191 x 2048 tokens' gradients into
// 128256 x 2048 fp32 in 174 us, 6.2 TB/s of what has to move (95 % of the measured copy).  With few
// tokens it is latency: 4096 tokens x 768 added to a gradient take 16 to 18 us on the device, 6 of sort, 5 of sums, 4 of joins.  The
// lookup is one pass: 16384 x 2048 in 17.1 us, 5.6 TB/s; one token 1.3 to 1.5 us.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
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
// Warps of the sums' kernel below which a chunk is not made longer: 16 on every SM.  (1200 / 2400 / 4800, us: 16384 tokens x 768
// 42 / 42 / 45; 65536 x 768 87 / 87 / 85; 8191 x 2048 273 / 271 / 274.)
constexpr uint64_t kWarpsWanted = 2400;
// Tokens that one CTA sorts, in fewer steps than the cluster of eight; from there on its scattered stores are what takes time (us a
// call that adds, one CTA / cluster: 1024 12.4 / 12.7, 2048 14.6 / 15.8, 4096 18.4 / 15.6).
constexpr uint64_t kOneCta = 2048;
// Tokens up to which the CTAs that write zeros look through all of them (4 us for 8192) rather than wait for the sort (11 us);
// 8192 x 768 29 us against 33, 16384 39 against 47.
constexpr uint64_t kLookThrough = 16384;
// Bytes of zeros from which on they are all the last kernel's: neither sums nor joins then wait for a zero, but CTAs that wait for
// the sums take room from those that write (us, zeros beside the sums / beside the joins: 8192 x 768 into 77 MB 29 / 33; 8191 x 2048
// into 131 MB 51 / 45, 262 MB 65 / 59, 525 MB 101 / 95, 1050 MB 181 / 174; 16384 x 2048 into 1050 MB 213 / 190).
constexpr uint64_t kManyZeros = 96 << 20;
constexpr uint64_t kZerosPerCta = 256 << 10;     // bytes: 8191 x 2048 fp32 in 179 us, with 1 MB 189; at least two CTAs per SM
constexpr uint64_t kZerosBesideJoins = 16 << 20; // bytes, at most an eighth: what the memory takes during the joins' 5 us
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

// Rows begin .. end - 1 of grad_weight, per_cta to each of `ctas` CTAs, of which a kernel sets those without a token to zero.
// wait: the CTAs take the tokens from the sort; otherwise they look through them and wait for nothing.
struct FillShare { uint64_t begin, end, per_cta; uint32_t ctas, wait; };

// V stands for a position that takes no part: ignored, or outside the table.
__device__ __forceinline__ uint32_t key_of(const EmbedCall& c, uint64_t i) {
  const int64_t t = c.token[i];
  return t != c.ignore && t >= 0 && uint64_t(t) < c.vocab ? uint32_t(t) : uint32_t(c.vocab);
}

// ------------------------------------------------------------------------------------------------ lookup
// A warp takes a row and 1024 of its columns.  VEC: rows are whole cells of eight columns and start on boundaries of eight
// elements on both sides.
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
      if (live && col < c.dim) raw[k] = Elem<uint16_t>::load_raw(w + col);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t col = col0 + k * kSlab + lane * 8;
      if (col >= c.dim) break;
      float x[8];
      Elem<uint16_t>::unpack(raw[k], x);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = live ? x[j] * c.scale : other;
      Elem<T>::store8(out + col, x);
    }
  } else {
    const uint32_t end = min(c.dim, col0 + 1024);
#pragma unroll 8
    for (uint32_t j = col0 + lane; j < end; j += 32) Elem<T>::put(out + j, live ? Elem<uint16_t>::get(w + j) * c.scale : other);
  }
}

// ------------------------------------------------------------------------------------------------ sort
// The lanes with the same digit of `bits` bits among those that take part.  (Ballots: a match instruction takes the longer the
// more different digits a warp holds.)
__device__ __forceinline__ uint32_t same_digit(bool in, uint32_t d, uint32_t bits) {
  uint32_t same = __ballot_sync(~0u, in);
#pragma unroll
  for (int b = 0; b < 9; ++b)
    if (b < bits) {
      const uint32_t set = __ballot_sync(~0u, d >> b & 1);
      same &= d >> b & 1 ? set : ~set;
    }
  return same;
}

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
    const uint32_t d = (item[r].x >> p.shift) & (radix - 1), same = same_digit(in, d, p.bits);
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

// The first of n sorted pairs whose key is at least `key`, found by a warp that looks at 32 places at once.
__device__ __forceinline__ uint32_t first_at_least(const uint2* pairs, uint32_t n, uint64_t key) {
  const uint32_t lane = threadIdx.x % 32;
  uint32_t lo = 0, len = n;                                 // the place is in lo .. lo + len
  while (len) {
    const uint32_t step = (len + 31) / 32, p = lo + lane * step;
    const uint32_t below = __popc(__ballot_sync(~0u, p < lo + len && pairs[p].x < key));   // a prefix of the lanes
    if (!below) return lo;
    const uint32_t end = lo + len;
    lo += (below - 1) * step + 1;
    len = min(step - 1, end - lo);
  }
  return lo;
}

struct FillShared { uint32_t there[kFillRows / 32]; };

// Zeros to the rows v0 .. v1 - 1 whose bit in `there` is not set, a warp each, or several short rows to a warp.
__device__ __forceinline__ void fill_rows(const EmbedCall& c, const FillShared& sh, uint64_t v0, uint64_t v1) {
  const uint32_t lane = threadIdx.x % 32, warps = blockDim.x / 32;
  const uint32_t bytes = c.dim * c.grad_size;
  if (c.zero_vec && bytes % 16 == 0 && bytes <= 256) {
    const uint32_t pieces = bytes / 16, rows = 32 / pieces, own = lane / pieces;
    char* to = static_cast<char*>(c.grad_weight) + (lane - own * pieces) * 16;
    if (own < rows)
#pragma unroll 4
      for (uint64_t v = v0 + threadIdx.x / 32 * rows + own; v < v1; v += warps * rows) {
        const uint32_t r = uint32_t(v - v0);
        if (!(sh.there[r / 32] >> (r % 32) & 1)) __stcs(reinterpret_cast<uint4*>(to + v * c.grad_weight_stride * c.grad_size), make_uint4(0, 0, 0, 0));
      }
    return;
  }
  for (uint64_t v = v0 + threadIdx.x / 32; v < v1; v += warps) {
    const uint32_t r = uint32_t(v - v0);
    if (sh.there[r / 32] >> (r % 32) & 1) continue;
    // elements up to the first 16-byte boundary, 16 bytes at a time from there, the elements behind the last boundary
    char* row = static_cast<char*>(c.grad_weight) + v * c.grad_weight_stride * c.grad_size;
    const uint32_t head = min(bytes, uint32_t(-reinterpret_cast<uintptr_t>(row)) % 16), middle = (bytes - head) / 16 * 16, tail = bytes - head - middle;
    if (lane * 2 < head) *reinterpret_cast<uint16_t*>(row + lane * 2) = 0;
#pragma unroll 4
    for (uint32_t j = lane * 16; j < middle; j += 512) __stcs(reinterpret_cast<uint4*>(row + head + j), make_uint4(0, 0, 0, 0));
    if (lane * 2 < tail) *reinterpret_cast<uint16_t*>(row + head + middle + lane * 2) = 0;
  }
}

// The rows without a token among those of one CTA of a kernel: CTA `index` of `share.ctas`.  The tokens that fall there are
// those that the sort has put side by side, or, beside the sort itself (pairs null), found by looking through all.
__device__ __forceinline__ void fill_part(const EmbedCall& c, const FillShare& share, uint32_t index, const uint2* pairs, FillShared& sh) {
  const uint64_t begin = share.begin + index * share.per_cta, end = min(share.end, begin + share.per_cta);
  for (uint64_t v0 = begin; v0 < end; v0 += kFillRows) {
    const uint64_t v1 = min(end, v0 + kFillRows);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kFillRows / 32; i += blockDim.x) sh.there[i] = 0;
    __syncthreads();
    if (pairs) {
      const uint32_t last = first_at_least(pairs, uint32_t(c.tokens), v1);
      for (uint32_t p = first_at_least(pairs, uint32_t(c.tokens), v0) + threadIdx.x; p < last; p += blockDim.x) {
        const uint32_t r = pairs[p].x - uint32_t(v0);
        atomicOr(&sh.there[r / 32], 1u << (r % 32));
      }
    } else {
      for (uint32_t base = threadIdx.x; base < uint32_t(c.tokens); base += 8 * blockDim.x) {
        uint32_t v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const uint32_t i = base + u * blockDim.x;
          v[u] = i < uint32_t(c.tokens) ? key_of(c, i) : uint32_t(c.vocab);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (v[u] >= v0 && v[u] < v1) atomicOr(&sh.there[(v[u] - uint32_t(v0)) / 32], 1u << ((v[u] - uint32_t(v0)) % 32));
      }
    }
    __syncthreads();
    fill_rows(c, sh, v0, v1);
  }
}

__global__ void __launch_bounds__(256) fls_embed_fill_kernel(const __grid_constant__ EmbedCall c, const FillShare share, const uint2* pairs) {
  __shared__ FillShared sh;
  pdl_launch();
  pdl_wait();
  fill_part(c, share, blockIdx.x, pairs, sh);
}

// ------------------------------------------------------------------------------------------------ sort of up to 2^17 tokens
// By the CTAs of one cluster.  A warp owns up to 16 * 32 neighbouring positions; per pass it ranks them among its own by digit,
// the CTA adds its warps up, and the CTAs of the cluster read each other's digit counts from distributed shared memory, into
// which they also write the items that are theirs after the pass.  65536 tokens in about 18 us, 4096 in 6.
constexpr int kClusterThreads = 1024, kClusterRounds = 16;
constexpr uint32_t kCluster = 8;
constexpr uint32_t kSortAtOnce = kCluster * kClusterThreads * kClusterRounds;

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

__device__ __forceinline__ void remote_store(const uint2* p, uint32_t rank, uint2 x) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(uint32_t(__cvta_generic_to_shared(p))), "r"(rank));
  asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(a), "r"(x.x), "r"(x.y) : "memory");
}

struct SortShared {
  uint16_t count[kClusterThreads / 32][kMaxRadix];   // of a warp, then of the warps before it
  uint32_t total[kMaxRadix];                         // of the CTA, read by the cluster
  uint32_t base[kMaxRadix];                          // where the CTA's first item of a digit goes
  uint32_t scan[kMaxRadix / 32];
};

template <int ROUNDS>
__device__ __forceinline__ void sort_tokens(const EmbedCall& c, SortShared& sh, uint2* items, uint32_t bits, uint32_t passes, uint32_t ctas) {
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
      item[r] = i >= n ? make_uint2(0, 0) : pass ? items[(warp * ROUNDS + r) * 32 + lane] : make_uint2(key_of(c, i), i);
    }
    for (uint32_t d = threadIdx.x; d < kClusterThreads / 32 * kMaxRadix / 2; d += kClusterThreads) reinterpret_cast<uint32_t*>(sh.count)[d] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      const bool in = first + r * 32 < n;
      if (__any_sync(~0u, in)) {
        const uint32_t d = (item[r].x >> shift) & (radix - 1), same = same_digit(in, d, per);
        at[r] = in ? sh.count[warp][d] + __popc(same & ((1u << lane) - 1)) : 0;
        __syncwarp();
        if (in && (same >> lane) == 1) sh.count[warp][d] = uint16_t(at[r] + 1);      // the last of them
        __syncwarp();
      }
    }
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < radix; d += kClusterThreads) {
      uint16_t k[kClusterThreads / 32];
#pragma unroll
      for (int w = 0; w < kClusterThreads / 32; ++w) k[w] = sh.count[w][d];
      uint32_t sum = 0;
#pragma unroll
      for (int w = 0; w < kClusterThreads / 32; ++w) {
        sh.count[w][d] = uint16_t(sum);
        sum += k[w];
      }
      sh.total[d] = sum;
    }
    if (ctas > 1) cluster_sync(); else __syncthreads();
    uint32_t before = 0, all = 0, x = 0;
    if (threadIdx.x < kMaxRadix) {
      if (threadIdx.x < radix && ctas == 1) {
        all = sh.total[threadIdx.x];
      } else if (threadIdx.x < radix) {
        uint32_t k[kCluster];
#pragma unroll
        for (uint32_t q = 0; q < kCluster; ++q) k[q] = remote_u32(&sh.total[threadIdx.x], q);
#pragma unroll
        for (uint32_t q = 0; q < kCluster; ++q) {
          all += k[q];
          if (q < rank) before += k[q];
        }
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
      const uint32_t to = sh.base[d] + sh.count[warp][d] + at[r];
      if (pass + 1 == passes) c.pairs[0][to] = item[r];
      else if (ctas == 1) items[to] = item[r];
      else remote_store(items + to % (ROUNDS * kClusterThreads), to / (ROUNDS * kClusterThreads), item[r]);
    }
    if (ctas > 1) cluster_sync(); else __syncthreads();
  }
}

__global__ void __launch_bounds__(kClusterThreads, 1)
    fls_embed_sort_kernel(const __grid_constant__ EmbedCall c, uint32_t bits, uint32_t passes) {
  __shared__ SortShared sh;
  extern __shared__ uint2 items[];                          // of the CTA, between two passes
  pdl_launch();
  const uint32_t ctas = gridDim.x, rounds = uint32_t((c.tokens + ctas * kClusterThreads - 1) / (ctas * kClusterThreads));
  if (rounds <= 1) sort_tokens<1>(c, sh, items, bits, passes, ctas);
  else if (rounds <= 2) sort_tokens<2>(c, sh, items, bits, passes, ctas);
  else if (rounds <= 4) sort_tokens<4>(c, sh, items, bits, passes, ctas);
  else if (rounds <= 8) sort_tokens<8>(c, sh, items, bits, passes, ctas);
  else sort_tokens<16>(c, sh, items, bits, passes, ctas);
}

// ------------------------------------------------------------------------------------------------ sums
// The eight columns of a lane are neighbours where every row starts on a boundary of eight elements and holds whole cells (VEC),
// otherwise 32 apart.

// The columns of one row as they lie in memory.
template <typename T, bool VEC> struct Piece;
template <typename T> struct Piece<T, true> {
  typename Elem<T>::Raw raw;
  __device__ __forceinline__ void load(const T* row, uint32_t col, uint32_t dim) {
    raw = typename Elem<T>::Raw{};
    if (col < dim) raw = Elem<T>::load_raw(row + col);
  }
  __device__ __forceinline__ void get(float (&x)[8]) const { Elem<T>::unpack(raw, x); }
};
template <typename T> struct Piece<T, false> {
  float x_[8];
  __device__ __forceinline__ void load(const T* row, uint32_t col, uint32_t dim) {
    row += col;
#pragma unroll
    for (int j = 0; j < 8; ++j) x_[j] = col + 32 * j < dim ? Elem<T>::get(row + 32 * j) : 0.f;
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = x_[j];
  }
};

// old: what is there, with accumulate.
template <typename G, bool VEC>
__device__ __forceinline__ void write_row(const EmbedCall& c, uint32_t key, uint32_t col, const float (&sum)[8], const Piece<G, VEC>& old) {
  if (col >= c.dim) return;
  G* row = static_cast<G*>(c.grad_weight) + uint64_t(key) * c.grad_weight_stride;
  float x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = sum[j] * c.scale;
  if (c.accumulate) {
    float o[8];
    old.get(o);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] += o[j];
  }
  if constexpr (VEC) {
    Elem<G>::store8(row + col, x);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (col + 32 * j < c.dim) Elem<G>::put(row + col + 32 * j, x[j]);
  }
}

// Partial sums of a warp's 256 columns: eight neighbours per lane.
__device__ __forceinline__ void write_part(const EmbedCall& c, uint32_t row, uint32_t slab, uint32_t lane, const float (&sum)[8]) {
  Elem<float>::store8(c.part + uint64_t(row) * c.dp + slab * kSlab + lane * 8, sum);
}

// A warp takes a chunk and 256 columns.  VEC: kAhead rows, and what is there of the rows that they finish, are on their way at
// once, copied asynchronously into shared memory (65536 x 768: 30 us for 100 MB read and 67 MB of zeros beside it; with the rows
// in registers 42).
constexpr int kAhead = 8;

template <typename T, typename G, bool VEC>
__global__ void __launch_bounds__(256, 3) fls_embed_sum_kernel(const __grid_constant__ EmbedCall c, const uint2* pairs, const FillShare share) {
  extern __shared__ uint4 rows[];
  __shared__ FillShared sh;
  pdl_launch();
  // first two CTAs of zeros for every SM, then the sums, then the other zeros
  const uint32_t ahead = min(share.ctas, 296u), sums = gridDim.x - share.ctas;
  if (blockIdx.x < ahead || blockIdx.x >= ahead + sums) {
    if (share.wait) pdl_wait();
    fill_part(c, share, blockIdx.x < ahead ? blockIdx.x : blockIdx.x - sums, share.wait ? pairs : nullptr, sh);
    return;
  }
  pdl_wait();
  const uint32_t block = blockIdx.x - ahead;
  const uint32_t lane = threadIdx.x % 32, slabs = c.dp / kSlab, unit = block * 8 + threadIdx.x / 32;
  const uint32_t chunk = unit / slabs, slab = unit - chunk * slabs;
  if (chunk >= c.chunks) return;
  const uint32_t n = uint32_t(c.tokens), none = uint32_t(c.vocab);
  const uint32_t begin = chunk * c.chunk, end = min(n, begin + c.chunk), col = slab * kSlab + (VEC ? lane * 8 : lane);
  const uint32_t row_bytes = Staged<T>::bytes + (c.accumulate ? Staged<G>::bytes : 0);
  const uint32_t place = uint32_t(__cvta_generic_to_shared(rows)) + threadIdx.x / 32 * (kAhead * row_bytes);
  float sum[8] = {};
  const uint32_t left = begin ? pairs[begin - 1].x : none, right = end < n ? pairs[end].x : none;
  bool from_left = false;
  uint32_t now = none;
  for (uint32_t base = begin; base < end; base += 64) {
    // 64 positions, two per lane, and the key behind each
    const uint32_t here = min(64u, end - base);
    const uint2 lo = lane < here ? pairs[base + lane] : make_uint2(none, 0), hi = lane + 32 < here ? pairs[base + lane + 32] : make_uint2(none, 0);
    const uint32_t behind = base + here < end ? pairs[base + here].x : right;
    uint32_t lo_next = __shfl_down_sync(~0u, lo.x, 1), hi_next = __shfl_down_sync(~0u, hi.x, 1);
    const uint32_t hi_first = __shfl_sync(~0u, hi.x, 0);
    if (lane == 31) lo_next = hi_first;
    if (lane + 1 >= here) lo_next = behind;
    if (lane + 33 >= here) hi_next = behind;
    auto key_at = [&](uint32_t i) { return __shfl_sync(~0u, i < 32 ? lo.x : hi.x, i); };
    if (base == begin) from_left = left == key_at(0);
    auto row_at = [&](uint32_t i) { return __shfl_sync(~0u, i < 32 ? lo.y : hi.y, i); };
    auto next_at = [&](uint32_t i) { return __shfl_sync(~0u, i < 32 ? lo_next : hi_next, i); };
    auto send = [&](uint32_t i) {
      if (i < here) {
        const uint32_t key = key_at(i), row = row_at(i), next = next_at(i);
        if (key != none) {
          const uint32_t to = place + i % kAhead * row_bytes;
          Staged<T>::copy(to, static_cast<const T*>(c.grad_out) + row * c.grad_out_stride, slab * kSlab, lane, c.dim);
          if (c.accumulate && key != next)
            Staged<G>::copy(to + Staged<T>::bytes, static_cast<const G*>(c.grad_weight) + uint64_t(key) * c.grad_weight_stride, slab * kSlab, lane, c.dim);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if constexpr (VEC)
      for (int i = 0; i + 1 < kAhead; ++i) send(i);
    for (uint32_t i = 0; i < here; ++i) {
      const uint32_t key = key_at(i), next = next_at(i);
      if (key == none) return;                              // nothing follows
      Piece<T, VEC> x;
      Piece<G, VEC> old;
      const uint32_t from = place + i % kAhead * row_bytes;
      if constexpr (VEC) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 2) : "memory");
        __syncwarp();
        Staged<T>::read(from, lane, x.raw);
        if (c.accumulate && key != next) Staged<G>::read(from + Staged<T>::bytes, lane, old.raw);
        __syncwarp();
      } else {
        x.load(static_cast<const T*>(c.grad_out) + row_at(i) * c.grad_out_stride, col, c.dim);
        if (c.accumulate && key != next) old.load(static_cast<const G*>(c.grad_weight) + uint64_t(key) * c.grad_weight_stride, col, c.dim);
      }
      float v[8];
      x.get(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] += v[j];
      now = key;
      if (key != next) {
        if (from_left) {
          write_part(c, 2 * chunk, slab, lane, sum);
        } else {
          write_row<G, VEC>(c, key, col, sum, old);
        }
        from_left = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = 0.f;
      }
      if constexpr (VEC) send(i + kAhead - 1);              // into the place that the row before this one had
    }
    if constexpr (VEC) asm volatile("cp.async.wait_all;" ::: "memory");
  }
  if (right != none && right == now) write_part(c, 2 * chunk + (from_left ? 0 : 1), slab, lane, sum);
}

// A CTA for every chunk whose last token begins in it and goes on in the next: the sums of that token.  Up to eight are added
// up in order, a warp for every 256 columns; more of them in order inside each of eight warps, then of the warps.
template <typename G, bool VEC>
__global__ void __launch_bounds__(256, 4) fls_embed_join_kernel(const __grid_constant__ EmbedCall c, const uint2* pairs, const FillShare share) {
  __shared__ union { float sums[8][kSlab]; FillShared fill; } sh;
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, slabs = c.dp / kSlab;
  // first two CTAs of zeros for every SM, then the joins, then the other zeros
  const uint32_t ahead = min(share.ctas, 296u), joins = gridDim.x - share.ctas;
  if (blockIdx.x < ahead || blockIdx.x >= ahead + joins) {
    if (share.wait) pdl_wait();
    fill_part(c, share, blockIdx.x < ahead ? blockIdx.x : blockIdx.x - joins, share.wait ? pairs : nullptr, sh.fill);
    return;
  }
  pdl_wait();
  const uint32_t chunk = blockIdx.x - ahead, n = uint32_t(c.tokens), none = uint32_t(c.vocab);
  const uint32_t begin = chunk * c.chunk, end = begin + c.chunk;
  if (end >= n) return;
  const uint64_t mine = uint64_t(end) + uint64_t(threadIdx.x) * c.chunk;
  uint32_t begins = mine < n ? pairs[mine].x : none;               // a token that a chunk after this one begins with
  const uint32_t key = pairs[end].x, last = pairs[end - 1].x, first = pairs[begin].x, left = begin ? pairs[begin - 1].x : none;
  if (key == none || last != key || (first == key && left == key)) return;       // nothing goes on, or began before this chunk
  uint32_t more = 0;                                                             // chunks after this one that begin with the token
  for (;;) {
    const int got = __syncthreads_count(begins == key);
    more += got;
    if (got < 256) break;
    const uint64_t p = mine + uint64_t(more) * c.chunk;
    begins = p < n ? pairs[p].x : none;
  }
  // the sums are in rows 2 chunk + 1, 2 chunk + 2, 2 chunk + 4, ... 2 (chunk + more)
  const bool few = more < 8;
  const uint32_t per = few ? more + 1 : (more + 8) / 8, k0 = few ? 0 : warp * per, k1 = min(more + 1, k0 + per);
  for (uint32_t slab = few ? warp : 0; slab < slabs; slab += few ? 8 : 1) {
    const uint32_t col = slab * kSlab + (VEC ? lane * 8 : lane);
    const float* part = c.part + slab * kSlab + lane * 8;
    Piece<G, VEC> old;
    if (c.accumulate && (few || warp == 0)) old.load(static_cast<const G*>(c.grad_weight) + uint64_t(key) * c.grad_weight_stride, col, c.dim);
    float sum[8] = {};
    for (uint32_t k = k0; k < k1; k += 4) {
      typename Elem<float>::Raw x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (k + u < k1) x[u] = Elem<float>::load_raw(part + uint64_t(k + u ? 2 * (chunk + k + u) : 2 * chunk + 1) * c.dp);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (k + u < k1) {
          float v[8];
          Elem<float>::unpack(x[u], v);
#pragma unroll
          for (int j = 0; j < 8; ++j) sum[j] += v[j];
        }
    }
    if (!few) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) sh.sums[warp][lane + 32 * j] = sum[j];
      __syncthreads();
      if (warp) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        for (int w = 1; w < 8; ++w) sum[j] += sh.sums[w][lane + 32 * j];
    }
    write_row<G, VEC>(c, key, col, sum, old);
  }
}

// ------------------------------------------------------------------------------------------------ few tokens
// As many tokens as a CTA has threads, in one kernel and without a workspace: every CTA that sums sorts all of them for itself, each
// thread counting the keys that come before its own, and takes every so many of (token, 256 columns), a warp for each, or all its
// warps where a token stands for more than 32 rows.  The other CTAs write zeros.  256 tokens x 512 of 11000 in 7.3 us on the device
// and 6 on the host, against 10 and 10 by the three kernels above; 128 x 768 of 50257 in 13.4 us, 5.8 TB/s.
constexpr uint32_t kFewTokens = 512, kLongRun = 32;
constexpr uint64_t kFewZeros = 64 << 20;

// The sum of rows b .. e - 1 of the sorted positions, eight on their way at once.
template <typename T, bool VEC>
__device__ __forceinline__ void sum_rows(const EmbedCall& c, const uint16_t* position, uint32_t b, uint32_t e, uint32_t col, float (&sum)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) sum[j] = 0.f;
  for (uint32_t p = b; p < e; p += 8) {
    Piece<T, VEC> x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (p + u < e) x[u].load(static_cast<const T*>(c.grad_out) + position[p + u] * c.grad_out_stride, col, c.dim);
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (p + u < e) {
        float v[8];
        x[u].get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += v[j];
      }
  }
}

template <typename T, typename G, bool VEC, int THREADS>
__global__ void __launch_bounds__(THREADS, 512 / THREADS) fls_embed_few_kernel(const __grid_constant__ EmbedCall c, const FillShare share, uint32_t sum_ctas) {
  __shared__ union { FillShared fill; float sums[THREADS / 32][kSlab]; } sh;
  __shared__ uint4 keys[THREADS / 4];
  __shared__ uint32_t sorted[THREADS], heads[THREADS / 32];
  __shared__ uint16_t position[THREADS], start[THREADS + 1];
  if (blockIdx.x >= sum_ctas) {
    fill_part(c, share, blockIdx.x - sum_ctas, nullptr, sh.fill);
    return;
  }
  constexpr uint32_t kWarps = THREADS / 32;
  const uint32_t n = uint32_t(c.tokens), none = uint32_t(c.vocab), tid = threadIdx.x, lane = tid % 32, warp = tid / 32, slabs = c.dp / kSlab;
  const uint32_t mine = tid < n ? key_of(c, tid) : ~0u;
  reinterpret_cast<uint32_t*>(keys)[tid] = mine;
  __syncthreads();
  // equal keys of smaller positions come before, others not: up to the own warp's keys those below mine + 1, then those below mine
  uint32_t before = 0;
  auto count = [&](uint32_t from, uint32_t to, uint32_t below) {
#pragma unroll 4
    for (uint32_t j = from; j < to; j += 4) {
      const uint4 k = keys[j / 4];
      before += uint32_t(k.x < below) + uint32_t(k.y < below) + uint32_t(k.z < below) + uint32_t(k.w < below);
    }
  };
  if (warp * 32 < n) {
    count(0, warp * 32, mine + 1);
#pragma unroll
    for (uint32_t j = 0; j < 32; ++j) before += __shfl_sync(~0u, mine, j) < mine + (j < lane ? 1 : 0);
    count(warp * 32 + 32, n, mine);                         // entries beyond n are below nothing
  }
  if (tid < n) {
    sorted[before] = mine;
    position[before] = uint16_t(tid);
  }
  __syncthreads();
  const bool live = tid < n && sorted[tid] != none, head = live && (tid == 0 || sorted[tid - 1] != sorted[tid]);
  const uint32_t mask = __ballot_sync(~0u, head), last = __syncthreads_count(live);
  if (lane == 0) heads[warp] = __popc(mask);
  __syncthreads();
  uint32_t at = __popc(mask & ((1u << lane) - 1)), runs = 0;
#pragma unroll
  for (uint32_t w = 0; w < kWarps; ++w) {
    if (w < warp) at += heads[w];
    runs += heads[w];
  }
  if (head) start[at] = uint16_t(tid);
  if (tid == 0) start[runs] = uint16_t(last);
  __syncthreads();
  float sum[8];
  Piece<G, VEC> old;
  auto what_is_there = [&](uint32_t key, uint32_t col) {
    if (c.accumulate) old.load(static_cast<const G*>(c.grad_weight) + uint64_t(key) * c.grad_weight_stride, col, c.dim);
  };
  for (uint32_t u = blockIdx.x * kWarps + warp; u < runs * slabs; u += sum_ctas * kWarps) {
    const uint32_t run = u / slabs, b = start[run], e = start[run + 1], col = (u - run * slabs) * kSlab + (VEC ? lane * 8 : lane);
    if (e - b > kLongRun) continue;
    what_is_there(sorted[b], col);
    sum_rows<T, VEC>(c, position, b, e, col, sum);
    write_row<G, VEC>(c, sorted[b], col, sum, old);
  }
  for (uint32_t u = blockIdx.x; u < runs * slabs; u += sum_ctas) {
    const uint32_t run = u / slabs, b = start[run], e = start[run + 1], col = (u - run * slabs) * kSlab + (VEC ? lane * 8 : lane);
    if (e - b <= kLongRun) continue;
    const uint32_t per = (e - b + kWarps - 1) / kWarps, from = min(e, b + warp * per);
    if (warp == 0) what_is_there(sorted[b], col);
    sum_rows<T, VEC>(c, position, from, min(e, from + per), col, sum);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) sh.sums[warp][lane + 32 * j] = sum[j];
    __syncthreads();
    if (warp) continue;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      for (uint32_t w = 1; w < kWarps; ++w) sum[j] += sh.sums[w][lane + 32 * j];
    write_row<G, VEC>(c, sorted[b], col, sum, old);
  }
}

// ------------------------------------------------------------------------------------------------ host
struct Regions { uint64_t pairs[2], counts, part, total; };

// Positions per chunk: few chunks leave few sums to join, many keep the memory busy.
uint32_t chunk_of(uint64_t tokens, uint32_t slabs) {
  uint32_t c = 8;
  while (uint64_t(c) * kMaxChunks < tokens || (c < 64 && tokens * slabs >= uint64_t(2 * c) * kWarpsWanted)) c *= 2;
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
uint64_t span_bytes(uint64_t rows, uint64_t cols, uint64_t stride, uint64_t elem) { return rows ? ((rows - 1) * stride + cols) * elem : 0; }

}  // namespace

struct fls_embed {
  fls_embed_desc desc{};
  Regions reg{};
  std::atomic<uint64_t> launches{0};      // calls that do not share a workspace may come from several host threads
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
  c.chunk = chunk_of(n, c.dp / kSlab);
  c.chunks = uint32_t((n + c.chunk - 1) / c.chunk);
  const uint32_t sums = uint32_t((uint64_t(c.chunks) * (c.dp / kSlab) + 7) / 8);
  // The zeros are written beside the sort and the sums, and some beside the joins, so that the memory is never idle.
  FillShare beside_sums{}, beside_joins{};
  uint64_t done = 0;
  auto share = [&](uint64_t bytes, uint32_t ctas) {
    FillShare f{};
    if (c.accumulate) return f;
    const uint64_t row = uint64_t(c.dim) * c.grad_size, rows = std::min(c.vocab - done, bytes / row);
    if (!rows) return f;
    f.begin = done;
    f.end = done += rows;
    f.per_cta = (rows + ctas - 1) / ctas;
    f.ctas = uint32_t((rows + f.per_cta - 1) / f.per_cta);
    f.wait = n > kLookThrough;
    return f;
  };
  // More than 256 tokens take CTAs of 512 threads, one to an SM, which are slow at writing many zeros (257 tokens x 512 of 11000: 8.4 us
  // against 10, x 4096 of 50257: 73 against 65).
  if (n && (n <= kFewTokens / 2 || (n <= kFewTokens && (c.accumulate || c.vocab * c.dim * c.grad_size <= kFewZeros)))) {
    beside_sums = share(~0ull, uint32_t(std::clamp<uint64_t>(c.vocab * c.dim * c.grad_size / kZerosPerCta, 296, 148 * 16)));
    const uint32_t threads = n <= 256 ? 256 : 512, sum_ctas = uint32_t(std::min<uint64_t>(148, (n * (c.dp / kSlab) * 32 + threads - 1) / threads));
    auto kernel = n <= 256 ? fls_embed_few_kernel<T, G, VEC, 256> : fls_embed_few_kernel<T, G, VEC, 512>;
    FLS_LAUNCH(launch(kernel, sum_ctas + beside_sums.ctas, threads, 0, false, s, c, beside_sums, sum_ctas));
    return FLS_OK;
  }
  if (n && n <= kSortAtOnce) {
    const uint32_t ctas = n <= kOneCta ? 1 : kCluster;
    // The last kernel's CTAs that wait for nothing start as soon as those of the two before it have, and so run beside all three.
    const uint64_t zeros = c.vocab * c.dim * c.grad_size;
    const uint32_t ctas_of_all = uint32_t(std::clamp<uint64_t>(zeros / kZerosPerCta, 296, 148 * 16));
    if (n <= kLookThrough && zeros >= kManyZeros) beside_joins = share(~0ull, ctas_of_all);
    else beside_joins = share(std::min<uint64_t>(zeros / 8, kZerosBesideJoins), 148);
    beside_sums = share(~0ull, ctas_of_all);
    const uint32_t rounds = uint32_t((n + ctas * kClusterThreads - 1) / (ctas * kClusterThreads));
    uint32_t room = kClusterThreads * 8;                    // as many rounds as the kernel is made for
    while (room < rounds * kClusterThreads * 8) room *= 2;
    if (room > 8 << 10) {
      static std::atomic<uint64_t> allowed{0};
      const cudaError_t err = allow_shared(reinterpret_cast<const void*>(fls_embed_sort_kernel), 128 << 10, allowed);
      if (err != cudaSuccess) return refuse(FLS_ECUDA, "embedding kernel: %s", cudaGetErrorString(err));
    }
    FLS_LAUNCH(launch_clusters(fls_embed_sort_kernel, ctas, ctas, kClusterThreads, room, false, s, c, bits, passes));
    sorted = c.pairs[0];
  } else {
    bool dependent = false;
    c.tiles = uint32_t((n + kSortTile - 1) / kSortTile);
    for (uint32_t p = 0; n && p < passes; ++p) {
      const SortPass sp{p * per, std::min(per, bits - p * per), p == 0, at};
      FLS_LAUNCH(launch(fls_embed_count_kernel, c.tiles, kSortThreads, 0, dependent, s, c, sp));
      dependent = true;
      FLS_LAUNCH(launch(fls_embed_scan_kernel, 1, 1024, 0, true, s, c, sp));
      FLS_LAUNCH(launch(fls_embed_scatter_kernel, c.tiles, kSortThreads, 0, true, s, c, sp));
      at ^= 1;
    }
    sorted = n ? c.pairs[at] : nullptr;
    const FillShare all = share(~0ull, 148 * 8);
    if (all.ctas) FLS_LAUNCH(launch(fls_embed_fill_kernel, all.ctas, 256, 0, dependent, s, c, all, sorted));
  }
  if (n) {
    auto kernel = fls_embed_sum_kernel<T, G, VEC>;
    const uint32_t smem = VEC ? kAhead * 8 * (Staged<T>::bytes + (c.accumulate ? Staged<G>::bytes : 0)) : 0;
    if (smem > 32 << 10) {
      static std::atomic<uint64_t> allowed{0};
      const cudaError_t err = allow_shared(reinterpret_cast<const void*>(kernel), 128 << 10, allowed);
      if (err != cudaSuccess) return refuse(FLS_ECUDA, "embedding kernel: %s", cudaGetErrorString(err));
    }
    FLS_LAUNCH(launch(kernel, sums + beside_sums.ctas, 256, smem, true, s, c, sorted, beside_sums));
    if (c.chunks > 1 || beside_joins.ctas)
      FLS_LAUNCH((launch(fls_embed_join_kernel<G, VEC>, beside_joins.ctas + c.chunks - 1, 256, 0, true, s, c, sorted, beside_joins)));
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
  const bool vec = d.dim % 8 == 0 && in_cells(c.weight, c.weight_stride, 2) && in_cells(c.out, c.out_stride, es), f32 = d.act_dtype == FLS_GRAD_F32;
  auto kernel = f32 ? (vec ? fls_embed_lookup_kernel<float, true> : fls_embed_lookup_kernel<float, false>)
                    : (vec ? fls_embed_lookup_kernel<uint16_t, true> : fls_embed_lookup_kernel<uint16_t, false>);
  FLS_LAUNCH(launch(kernel, grid, 256, 0, false, static_cast<cudaStream_t>(cuda_stream), c));
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
  c.zero_vec = reinterpret_cast<uintptr_t>(c.grad_weight) % 16 == 0 && c.grad_weight_stride * gs % 16 == 0;
  const bool vec = d.dim % 8 == 0 && in_cells(c.grad_weight, c.grad_weight_stride, gs) && (!n || in_cells(c.grad_out, c.grad_out_stride, es));
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
