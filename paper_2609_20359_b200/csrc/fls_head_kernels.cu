// Kernels of the language-model head: cross entropy and distillation of a linear head without kept logits.
//
//   fls_head_map_kernel    which rows take part, and where they go (compaction; ignored rows cost nothing below)
//   fls_head_pack_kernel   packed copy of their hidden states, the columns that get a value of their own, sorted
//   fls_head_gemm_kernel   the tensor-core kernel, three epilogues:
//     kStats    logits tile -> maximum and sum of exponentials per row and 128 columns
//     kDlogits  logits tile -> dL/dz in bf16 (one piece of the vocabulary)
//     kGrads    dL/dz of the piece -> rows of grad_weight, and partial sums of grad_hidden
//   fls_head_rescale_kernel, fls_head_own_kernel   dL/dz of the columns whose logits the statistics pass kept
//   fls_head_rows_kernel   joins the tile sums, losses, coefficients of dL/dz
//   fls_head_grad_hidden_kernel   sums the partial sums, rounds, puts rows back in the caller's order
#include <cuda_bf16.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <utility>

#include "fls_head.h"

namespace fls {
namespace {

constexpr uint32_t kOperandBytes = 128 * kHeadBK * 2;            // one operand of one stage of one CTA: 16 KB
constexpr uint32_t kStageBytes = 2 * kOperandBytes;
constexpr int kEpiWarps = 8;                                     // two per lane quarter of TMEM, 128 columns each
constexpr uint32_t kStoreBytes = 32 * 128;                       // one staged store of one warp: 32 rows of 128 bytes
enum { kStats = 0, kDlogits = 1, kGrads = 2 };
// Shared memory goes to pipeline stages first (row statistics of 2048 x 128256 x 2048 from idle clocks: 775 us with 7
// stages, 827 us with 5); what stores tiles keeps a 4 KB buffer per epilogue warp, or two for fp32 logits and for two
// terms of dL/dz.
template <int MODE, bool FLAG, bool KEEP>
struct Smem {
  static constexpr int kBufs = MODE == kStats ? 2 * KEEP : MODE == kDlogits && FLAG ? 2 : 1;
  static constexpr int kStages = 7 - kBufs;
  static constexpr uint32_t kBytes = kStages * kStageBytes + kEpiWarps * kBufs * kStoreBytes + 1024 + 256;
  static_assert(kBytes <= 232448, "shared memory of one CTA");
};
constexpr int kGemmThreads = 128 + 32 * kEpiWarps;               // warp 0 TMA, 1 MMA, 2 TMEM, 4..11 epilogue

// ------------------------------------------------------------------------------------------------ PTX
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return uint32_t(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ uint32_t cta_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
// Programmatic dependent launch: the next kernel of the call may start (its blocks wait in pdl_wait) / everything the
// kernels before this one wrote is visible.  Every kernel of a call waits, so completion carries over several kernels.
__device__ __forceinline__ void pdl_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Address, in the cluster's shared window, of the leader CTA's copy of a shared variable.
__device__ __forceinline__ uint32_t leader_addr(uint32_t a) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(a));
  return r;
}
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// False if the phase did not complete within `limit` polls (each poll may sleep in hardware for a while).
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, uint32_t limit) {
  for (uint32_t i = 0; i < limit; ++i) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    if (ok) return true;
  }
  return false;
}
// A tile of 64 x box-rows elements into this CTA's shared memory; the bytes are counted on the leader's barrier.
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
      ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load3(uint32_t dst, const CUtensorMap* map, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(map), "r"(0), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_prefetch(const CUtensorMap* map, int x, int y) {
  asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(map), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
// Arrives on the barrier at this offset in both CTAs when the products issued so far are done.
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
      ::"r"(bar), "h"(uint16_t(3)) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of this thread's row of an accumulator.  The wait is part of the statement: registers handed through a
// separate wait would be copied once per value.
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
        "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]),
        "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]),
        "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
      : "r"(addr) : "memory");
}
__device__ __forceinline__ void tma_store(const CUtensorMap* map, int x, int y, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
}
__device__ __forceinline__ void tma_add(const CUtensorMap* map, int x, int y, uint32_t src) {
  asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
}
__device__ __forceinline__ void tma_store3(const CUtensorMap* map, int y, int z, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(0), "r"(y), "r"(z), "r"(src) : "memory");
}
__device__ __forceinline__ void st_shared(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ void st_shared_u16(uint32_t a, uint16_t x) {
  asm volatile("st.shared.b16 [%0], %1;" ::"r"(a), "h"(x) : "memory");
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
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
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// Sums of exponentials are kept relative to 2^(m c), m c rounded (one instruction less per value), while that is off by less
// than 2^-8, the log sum exp by less than its own last digit.  From |m c| = 2^16 on (columns masked through the weight with
// -1e10 or the type's lowest value, in a stretch of nothing else) the difference to m is taken first: a rounding error of m c
// is soon a power of two beyond fp32.
constexpr float kFar = 65536.f;
// (x - m) / T in powers of two, c = log2(e) / T
struct Log2Ratio {
  float c, off, b;
  __device__ __forceinline__ Log2Ratio(float m, float cc) : c(cc) {
    b = __fmul_rn(m, c);
    const bool far = !(fabsf(b) < kFar);
    off = far ? m : 0.f;
    if (far) b = 0.f;
  }
  __device__ __forceinline__ float operator()(float x) const { return __fmul_rn(x - off, c) - b; }
};
// sum over 32 values of 2^((z - m) c)
__device__ __forceinline__ float sum_ex2(const float (&z)[32], float c, float m) {
  const float b = __fmul_rn(m, c);
  if (!(fabsf(b) < kFar)) {
    float t = 0.f;
#pragma unroll
    for (int j = 0; j < 32; ++j) t += ex2((z[j] - m) * c);
    return t;
  }
  const f2 c2 = make_f2(c, c), b2 = make_f2(-b, -b);
  f2 t0 = make_f2(0.f, 0.f), t1 = t0;
#pragma unroll
  for (int j = 0; j < 32; j += 4) {
    float u, v, x, y;
    split(fma2(make_f2(z[j], z[j + 1]), c2, b2), u, v);
    split(fma2(make_f2(z[j + 2], z[j + 3]), c2, b2), x, y);
    t0 = add2(t0, make_f2(ex2(u), ex2(v)));
    t1 = add2(t1, make_f2(ex2(x), ex2(y)));
  }
  float u, v;
  split(add2(t0, t1), u, v);
  return u + v;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Shared-memory matrix descriptor, 128-byte swizzle.  Depth-contiguous operand (K-major): rows of 64 elements = 128
// bytes, 8-row groups 1024 bytes apart (sbo).  Width-contiguous operand (MN-major): blocks of 64 columns x 64 depth
// rows; 8-row groups 1024 bytes apart (sbo), 64-column blocks 8192 bytes apart (lbo).
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr) {
  constexpr uint32_t kLbo = 8192 >> 4, kSbo = 1024 >> 4;
  const uint32_t lo = ((addr >> 4) & 0x3FFF) | (kLbo << 16);
  const uint32_t hi = kSbo | (1u << 14) | (2u << 29);
  return (uint64_t(hi) << 32) | lo;
}
// fp32 accumulator, bf16 operands, 256 x 256 over the CTA pair.
__device__ __forceinline__ uint32_t instr_desc(bool a_mn, bool b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (uint32_t(a_mn) << 15) | (uint32_t(b_mn) << 16) | ((kHeadBN >> 3) << 17) |
         ((kHeadBM >> 4) << 24);
}

// dL/dz of a piece lies in panels of 64 columns: [panel][row][64] bf16, whole 128-byte lines one after the other for a
// box of rows.  With two terms a panel is followed by that of the second term.  Kept logits lie the same way in panels of
// 32 fp32 columns; two of them become one panel of dL/dz in place, and the second one's place holds the second term's.
// (Row-major, where a store is 32 scattered lines, the statistics of 3686 x 50257 x 768 took 259 us instead of 243, the
// whole step of 8192 x 128256 x 2048 13.3 ms instead of 12.9.)
__device__ __forceinline__ int dz_panel(const HeadPiece& p, uint32_t n, uint32_t second) {
  return int(n / 64 * p.panel_step + second);
}

// ------------------------------------------------------------------------------------------------ work units
struct Unit {
  uint32_t grad_hidden;   // kGrads: which of the two products
  uint32_t m0, n0;        // first row / column of the 256 x 256 tile
  uint32_t kb0, kbn;      // depth blocks of 64
  uint32_t split;
};

// The hidden gradient's depth (a piece's columns) is cut into `s` parts, each with partial sums of its own.  A cluster
// works through units u, u + clusters, ...: first those of the hidden gradient (tiles_h * s of kb_h / s blocks), then
// those of the weight gradient (tiles_w of kb_w blocks).  Time of the busiest cluster in blocks of depth, with kUnitCost
// for what a unit costs besides its products (its epilogue's tail, the partial sums written and read again).
constexpr uint32_t kUnitCost = 12;
__device__ __forceinline__ uint32_t head_makespan(uint32_t s, uint32_t tiles_h, uint32_t kb_h, uint32_t tiles_w, uint32_t kb_w, uint32_t clusters) {
  const uint32_t units_h = tiles_h * s, units = units_h + tiles_w;
  const uint32_t len_h = (kb_h + s - 1) / s + kUnitCost, len_w = kb_w + kUnitCost;
  uint32_t worst = 0;
  for (int i = 0; i < 2; ++i) {          // the first cluster, and the first one with a unit less of the hidden gradient
    const uint32_t c = i ? units_h % clusters : 0;
    const uint32_t nh = (units_h + clusters - 1 - c) / clusters, nu = (units + clusters - 1 - c) / clusters;
    worst = max(worst, nh * len_h + (nu - nh) * len_w);
  }
  return worst;
}

template <int MODE>
struct Schedule {
  uint32_t mt, nt, kb, group, n_units, n_gh, splits, kb_gh, planes;
  __device__ __forceinline__ Schedule(const HeadCall& c, const HeadPiece& p, uint32_t count) {
    mt = (count + kHeadBM - 1) / kHeadBM;
    group = c.group_m;
    planes = c.planes;
    if constexpr (MODE == kGrads) {
      nt = (c.dim + kHeadBN - 1) / kHeadBN;
      kb = (count + kHeadBK - 1) / kHeadBK;
      kb_gh = (p.width + kHeadBK - 1) / kHeadBK;
      splits = c.state->splits;
      n_gh = c.want_gh ? mt * nt * splits : 0;
      n_units = n_gh + (c.want_gw ? (p.width + kHeadBM - 1) / kHeadBM * nt : 0);
    } else {
      nt = (p.width + kHeadBN - 1) / kHeadBN;
      kb = (c.dp + kHeadBK - 1) / kHeadBK;
      n_units = mt * nt;
      n_gh = splits = kb_gh = 0;
    }
  }
  __device__ __forceinline__ Unit at(uint32_t u) const {
    Unit w;
    w.grad_hidden = 0; w.split = 0; w.kb0 = 0;
    if constexpr (MODE == kGrads) {
      if (u < n_gh) {
        w.grad_hidden = 1;
        w.split = u / (mt * nt);
        const uint32_t r = u - w.split * (mt * nt);
        w.m0 = r / nt * kHeadBM;
        w.n0 = r % nt * kHeadBN;
        w.kb0 = uint32_t(uint64_t(kb_gh) * w.split / splits);
        w.kbn = uint32_t(uint64_t(kb_gh) * (w.split + 1) / splits) - w.kb0;
      } else {
        const uint32_t r = u - n_gh;
        w.m0 = r / nt * kHeadBM;
        w.n0 = r % nt * kHeadBN;
        w.kbn = kb * planes;
      }
    } else {
      // all column tiles of a group of row tiles before the next group: the group's hidden rows stay in L2
      const uint32_t per = group * nt, gi = u / per, r = u - gi * per;
      const uint32_t gm = min(group, mt - gi * group);
      w.n0 = r / gm * kHeadBN;
      w.m0 = (gi * group + r % gm) * kHeadBM;
      w.kbn = kb;
    }
    return w;
  }
};

// ------------------------------------------------------------------------------------------------ epilogues
// A row's own columns from some point on, ascending.  The one after the next is fetched ahead.
struct Columns {
  int32_t next = INT_MAX, after = INT_MAX;
  const int32_t* idx;
  uint32_t ptr, slots;
  __device__ __forceinline__ int32_t at(uint32_t i) const { return i < slots ? idx[i] : INT_MAX; }
  // start: the first of them not below the tile's first column
  __device__ __forceinline__ void open(const int32_t* i, uint32_t n, uint32_t start) {
    idx = i; slots = n; ptr = start;
    next = at(start);
    after = at(start + 1);
  }
  __device__ __forceinline__ void advance() {
    ++ptr;
    next = after;
    after = at(ptr + 1);
  }
};

// Maximum and sum of exponentials of one row of a tile.  Columns with a value of their own (the label, the teacher's
// list) are written down and left out of the sum, so that "everything else" is known without a cancelling difference.
template <bool TWO, bool SMOOTH>
struct StatsRow : Columns {
  float m = -INFINITY, s = 0.f, s1 = 0.f, sz = 0.f;
  float* zs;
  __device__ __forceinline__ void chunk(float (&z)[32], int32_t col0, uint32_t vocab, float cT, float c1) {
    const bool edge = uint32_t(col0) + 32 > vocab;
    if constexpr (SMOOTH) {
      float t0 = 0.f, t1 = 0.f;
#pragma unroll
      for (int j = 0; j < 32; j += 2) {
        t0 += (!edge || uint32_t(col0 + j) < vocab) ? z[j] : 0.f;
        t1 += (!edge || uint32_t(col0 + j + 1) < vocab) ? z[j + 1] : 0.f;
      }
      sz += t0 + t1;
    }
    if (edge) {
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (uint32_t(col0 + j) >= vocab) z[j] = -INFINITY;
    }
    while (next < col0 + 32) {
      const int off = next - col0;
      float v = 0.f;
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (j == off) { v = z[j]; z[j] = -INFINITY; }
      const int32_t at = next;
      do {                                            // repeated columns share the value
        zs[ptr] = v;
        advance();
      } while (next == at);
    }
    float x0 = max3(z[0], z[1], z[2]), x1 = max3(z[3], z[4], z[5]), x2 = max3(z[6], z[7], z[8]), x3 = max3(z[9], z[10], z[11]);
#pragma unroll
    for (int j = 12; j < 28; j += 8) {
      x0 = max3(x0, z[j], z[j + 1]); x1 = max3(x1, z[j + 2], z[j + 3]); x2 = max3(x2, z[j + 4], z[j + 5]); x3 = max3(x3, z[j + 6], z[j + 7]);
    }
    x0 = max3(x0, z[28], z[29]);
    x1 = max3(x1, z[30], z[31]);
    const float cm = fmaxf(max3(x0, x1, x2), x3);
    if (cm > m) {
      const float old = m;
      m = cm;
      if (old != -INFINITY) {
        s *= ex2(Log2Ratio(m, cT)(old));
        if constexpr (TWO) s1 *= ex2(Log2Ratio(m, c1)(old));
      }
    }
    const float base = m == -INFINITY ? 0.f : m;
    s += sum_ex2(z, cT, base);
    if constexpr (TWO) s1 += sum_ex2(z, c1, base);
  }
};

__device__ __forceinline__ float bf16_round(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }
__device__ __forceinline__ uint16_t bf16_bits(float x) { return __bfloat16_as_ushort(__float2bfloat16_rn(x)); }

// A warp's way out: 32 rows x 128 bytes are written to shared memory in the layout that a TMA store with 128-byte
// swizzle reads (16-byte piece q of row r at q ^ (r & 7): no bank conflicts), and leave as whole lines.
template <int BUFS>
struct Stager {
  uint32_t base, lane, next = 0;
  __device__ __forceinline__ Stager(uint32_t b, uint32_t l) : base(b), lane(l) {}
  // Buffer to write next.  Buffers take turns and every acquire is followed by one group (send or skip), so with two of
  // them all groups but the last are older than the buffer's last store.
  __device__ __forceinline__ uint32_t acquire() {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(BUFS == 2 ? 1 : 0) : "memory");
    __syncwarp();
    const uint32_t b = base + next * kStoreBytes;
    if constexpr (BUFS == 2) next ^= 1;
    return b;
  }
  // the other buffer too, before anything is sent from the first
  __device__ __forceinline__ uint32_t acquire_next() {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
    const uint32_t b = base + next * kStoreBytes;
    next ^= 1;
    return b;
  }
  __device__ __forceinline__ uint32_t piece(uint32_t buf, uint32_t q) const { return buf + lane * 128 + ((q ^ (lane & 7)) << 4); }
  __device__ __forceinline__ void send(const CUtensorMap* map, int x, int y, uint32_t buf, bool add) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
      if (add) tma_add(map, x, y, buf); else tma_store(map, x, y, buf);
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
  }
  __device__ __forceinline__ void send3(const CUtensorMap* map, int y, int z, uint32_t buf) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
      tma_store3(map, y, z, buf);
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
  }
  __device__ __forceinline__ void skip() {
    if (lane == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  }
  __device__ __forceinline__ void drain() {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    __syncwarp();
  }
  // 32 columns as bf16 into the first or second half of a buffer's 64
  __device__ __forceinline__ void put_bf16(uint32_t buf, uint32_t half, const float (&v)[32]) const {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      st_shared(piece(buf, half * 4 + q), pack_bf16(v[8 * q], v[8 * q + 1]), pack_bf16(v[8 * q + 2], v[8 * q + 3]),
                pack_bf16(v[8 * q + 4], v[8 * q + 5]), pack_bf16(v[8 * q + 6], v[8 * q + 7]));
  }
  __device__ __forceinline__ void put_f32(uint32_t buf, const float (&v)[32]) const {
#pragma unroll
    for (int q = 0; q < 8; ++q)
      st_shared(piece(buf, q), __float_as_uint(v[4 * q]), __float_as_uint(v[4 * q + 1]), __float_as_uint(v[4 * q + 2]), __float_as_uint(v[4 * q + 3]));
  }
  __device__ __forceinline__ void put_one(uint32_t buf, uint32_t col, uint16_t x) const {
    st_shared_u16(piece(buf, col >> 3) + (col & 7) * 2, x);
  }
};

// dL/dz is rounded to bf16, the type of the operands it meets in the products, whose sums are fp32: gradients are 1.8e-3 to
// 2.3e-3 off 64 bits, of which 1.7e-3 is the rounding of a bf16 result.  Two terms for the weight's product (PLANES: fp32 weight
// gradients) leave 2.6e-6 and cost 2 N V d more; a third, or two for the hidden gradient, would cost as much again each.
// dL/dz of one row of a tile: aT exp(z/T - lse_T) + a1 exp(z - lse_1) - b, then the columns with a value of their own
// (lse_T: with the tail as a class that of the columns outside the list).
template <bool TWO, bool PLANES, int BUFS>
struct DlogitsRow : Columns {
  float4 k;          // {lse_T log2(e), aT, lse_1 log2(e), a1}; without TWO {lse log2(e) , a, b, -}
  bool live;         // one of the rows that take part; those after them are zero, whatever the weight holds
  const float* val;
  // the first (half 0) or second 32 of the 64 columns from col0 on; lo: buffer of the second term (PLANES)
  __device__ __forceinline__ void chunk(float (&v)[32], int32_t col0, uint32_t half, uint32_t vocab, float cT, float c1,
                                        const Stager<BUFS>& out, uint32_t hi, uint32_t lo) {
    const int32_t c0 = col0 + int32_t(half) * 32;
    if constexpr (TWO) {
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = fmaf(k.w, ex2(fmaf(v[j], c1, -k.z)), k.y * ex2(fmaf(v[j], cT, -k.x)));
    } else {
      const f2 c2 = make_f2(cT, cT), l2 = make_f2(-k.x, -k.x), a2 = make_f2(k.y, k.y), b2 = make_f2(-k.z, -k.z);
#pragma unroll
      for (int j = 0; j < 32; j += 2) {
        float x, y;
        split(fma2(make_f2(v[j], v[j + 1]), c2, l2), x, y);
        split(fma2(a2, make_f2(ex2(x), ex2(y)), b2), v[j], v[j + 1]);
      }
    }
    if (!live || uint32_t(c0) + 32 > vocab) {
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (!live || uint32_t(c0 + j) >= vocab) v[j] = 0.f;
    }
    out.put_bf16(hi, half, v);
    if constexpr (PLANES) {
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] -= bf16_round(v[j]);
      out.put_bf16(lo, half, v);
    }
    while (next < c0 + 32) {            // same thread, same address, after the store above
      const float x = val[ptr];
      out.put_one(hi, uint32_t(next - col0), bf16_bits(x));
      if constexpr (PLANES) out.put_one(lo, uint32_t(next - col0), bf16_bits(x - bf16_round(x)));
      advance();
    }
  }
};

__device__ __forceinline__ bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename T>
__device__ __forceinline__ void store_row32(T* dst, const float (&v)[32], uint32_t n, bool add) {
  if (n >= 32 && aligned16(dst)) {
    if constexpr (sizeof(T) == 4) {
      float4* o = reinterpret_cast<float4*>(dst);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        float4 x = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
        if (add) { const float4 y = o[q]; x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w; }
        o[q] = x;
      }
    } else {
      uint4* o = reinterpret_cast<uint4*>(dst);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = v[8 * q + e];
        if (add) {
          const uint4 y = o[q];
          const uint32_t yy[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            w[2 * e] += __uint_as_float(yy[e] << 16);
            w[2 * e + 1] += __uint_as_float(yy[e] & 0xFFFF0000u);
          }
        }
        o[q] = make_uint4(pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3]), pack_bf16(w[4], w[5]), pack_bf16(w[6], w[7]));
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      if (j < int(n)) {
        if constexpr (sizeof(T) == 4) dst[j] = add ? dst[j] + v[j] : v[j];
        else dst[j] = bf16_bits(add ? __uint_as_float(uint32_t(dst[j]) << 16) + v[j] : v[j]);
      }
    }
  }
}

// Without row weights the mean's 1 / count stays out of dL/dz and goes onto the gradients in fp32: a label's entry is then
// p - 1, whose leading term in bf16 is mostly exact, and not a number with 24 bits that 8 or 16 have to hold.
__device__ __forceinline__ float mean_scale(const HeadCall& c, uint32_t count) {
  return c.row_weight || !count ? 1.f : 1.f / float(count);
}

// The first of a packed row's own columns that is not below column n (a multiple of 128).
__device__ __forceinline__ uint32_t first_slot(const HeadCall& c, uint32_t row, uint32_t n) {
  if (c.slots == 1) return c.slot_idx[row] < int32_t(n) ? 1 : 0;
  return c.slot_start[uint64_t(row) * c.tiles + n / kHeadStatCols];
}

// ------------------------------------------------------------------------------------------------ the kernel
template <int STAGES>
struct alignas(8) Barriers {
  uint64_t full[STAGES];    // leader: both CTAs' operands of a stage have landed
  uint64_t empty[STAGES];   // both: the products that read a stage are done
  uint64_t acc_full[2];      // both: an accumulator is complete
  uint64_t acc_empty[2];     // leader: both CTAs' epilogues have read an accumulator
  uint32_t tmem;
  uint32_t gave_up;
};

// The products.  A CTA pair makes 256 x 256 tiles of C = A B^T with tcgen05.mma (cta_group::2, bf16, fp32 accumulator in
// TMEM): each CTA brings 128 rows of A and 128 of B per 64 of depth by TMA, one thread of the leading CTA issues, eight
// epilogue warps (a lane quarter and 128 columns each) read one accumulator while the other is being made.  The grid is
// persistent, one pair per two SMs; a pair takes units u, u + pairs, ...
//   What bounds it: one 64-deep block takes 577 to 588 cycles where the tensor pipe needs 512 (shared memory carries 64
// bytes per cycle in by TMA and 64 out to the products, its limit; with half the loads left out 557), a unit another 500
// cycles, about 1000 more while the epilogue reads TMEM beside the products, a launch about 12000 (7 us).  With d = 4096
// the statistics of 1023 x 128256 run at 1.55 PFLOP/s from idle clocks (95 % of the measured library product); back to
// back the board's power cap holds everything to 1.25 - 1.3 (library product 1.35 - 1.39), and then shape, stages and
// split no longer show in time, only work left out does.
//   Why these choices: a pair's tile of 256 x 256 needs 64 bytes per SM and cycle from L2 where two single CTAs would need
// 96; clusters of four that share loads would leave 16 of 148 SMs idle (33 fit).  Tiles go out through shared memory and
// TMA stores because a thread owns a row: as 32-byte stores of its own the kept logits of 3686 x 50257 took 293 us
// instead of 243.  Operands whose depth is not contiguous in memory (dL/dz and hidden for the weight's gradient, the weight
// for the hidden one) are read as they are, MN-major, so nothing is transposed; measured as fast as K-major (588 cycles).
// TWO: two temperatures.  FLAG: label smoothing (kStats), dL/dz as two bf16 terms (kDlogits).  KEEP (kStats): the
// logits of the columns from c.keep_v0 on stay in the workspace.
template <int MODE, bool TWO, bool FLAG, bool KEEP>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGemmThreads, 1)
fls_head_gemm_kernel(const __grid_constant__ HeadMaps maps, const __grid_constant__ HeadCall c, const HeadPiece piece) {
  constexpr int kStages = Smem<MODE, FLAG, KEEP>::kStages, kBufs = Smem<MODE, FLAG, KEEP>::kBufs;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  auto* bars = reinterpret_cast<Barriers<kStages>*>(tiles + kStages * kStageBytes + kEpiWarps * kBufs * kStoreBytes);
  const uint32_t tile_base = smem_u32(tiles);
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cta_rank();
  const uint32_t cluster = blockIdx.x >> 1, n_clusters = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) { mbar_init(smem_u32(&bars->full[i]), 1); mbar_init(smem_u32(&bars->empty[i]), 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&bars->acc_full[i]), 1); mbar_init(smem_u32(&bars->acc_empty[i]), 2 * kEpiWarps); }
    bars->gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&bars->tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  if (MODE == kStats && threadIdx.x == 0 && c.prefetch_weight) {
    // One row tile: this cluster's first columns are known before the packed rows are, and the weight is nothing that an
    // earlier kernel of the call wrote.  It comes from memory while they are still packed.
    for (uint32_t k = 0; k < c.dp; k += kHeadBK) tma_prefetch(&maps.b0, int(k), int(cluster * kHeadBN + rank * 128));
  }
  fence_before();
  __syncthreads();
  cluster_sync();
  fence_after();
  const uint32_t tmem = bars->tmem;
  pdl_launch();
  pdl_wait();

  const uint32_t count = c.state->count;
  const Schedule<MODE> plan(c, piece, count);
  bool ok = true;

  // The two issuing threads do as little as they can per block: addresses advance, nothing is recomputed.
  const uint32_t full0 = smem_u32(&bars->full[0]), empty0 = smem_u32(&bars->empty[0]);
  if (warp == 0) {
    if (lane == 0) {
      const uint32_t full_leader = leader_addr(full0);
      const bool leader = rank == 0 && !c.hold_back;
      uint32_t stage = 0, phase = 0;
      // waits for the stage, announces both CTAs' bytes, and lets `load` fetch into it
      auto block = [&](auto&& load) {
        if (!mbar_wait(empty0 + stage * 8, phase ^ 1, c.wait_limit)) { ok = false; return; }
        if (leader) mbar_expect(full0 + stage * 8, 2 * kStageBytes);
        const uint32_t sa = tile_base + stage * kStageBytes;
        load(sa, sa + kOperandBytes, full_leader + stage * 8);
        if (++stage == kStages) { stage = 0; phase ^= 1; }
      };
      for (uint32_t u = cluster; u < plan.n_units && ok; u += n_clusters) {
        const Unit w = plan.at(u);
        const int m = int(w.m0 + rank * 128), n = int(w.n0 + rank * 128);
        if constexpr (MODE == kGrads) {
          if (w.grad_hidden) {
            int panel = dz_panel(piece, w.kb0 * kHeadBK, 0), v = int(piece.v0 + w.kb0 * kHeadBK);
            for (uint32_t i = 0; i < w.kbn && ok; ++i, panel += int(piece.panel_step), v += kHeadBK)
              block([&](uint32_t sa, uint32_t sb, uint32_t bar) {
                tma_load3(sa, &maps.a1, m, panel, bar);                  // dL/dz: 128 rows x 64 columns
                tma_load(sb, &maps.b1, n, v, bar);                       // weight: 64 rows x 2 x 64 columns
                tma_load(sb + 8192, &maps.b1, n + 64, v, bar);
              });
          } else {
            // fp32 weight gradients: the depth twice, the second time with the second term of dL/dz
            for (uint32_t second = 0; second < plan.planes; ++second) {
              const int p0 = dz_panel(piece, uint32_t(m), second), p1 = dz_panel(piece, uint32_t(m) + 64, second);
              int r = 0;
              for (uint32_t i = 0; i < plan.kb && ok; ++i, r += kHeadBK)
                block([&](uint32_t sa, uint32_t sb, uint32_t bar) {
                  tma_load3(sa, &maps.a0, r, p0, bar);                   // dL/dz: 64 rows x 2 x 64 columns
                  tma_load3(sa + 8192, &maps.a0, r, p1, bar);
                  tma_load(sb, &maps.b0, n, r, bar);                     // hidden: 64 rows x 2 x 64 columns
                  tma_load(sb + 8192, &maps.b0, n + 64, r, bar);
                });
            }
          }
        } else {
          const int v = int(piece.v0) + n;
          int k = 0;
          for (uint32_t i = 0; i < w.kbn && ok; ++i, k += kHeadBK)
            block([&](uint32_t sa, uint32_t sb, uint32_t bar) {
              tma_load(sa, &maps.a0, k, m, bar);                         // hidden: 128 rows x 64
              tma_load(sb, &maps.b0, k, v, bar);                         // weight: 128 rows x 64
            });
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0 && lane == 0) {
      const uint64_t desc0 = smem_desc(tile_base);
      uint32_t stage = 0, phase = 0, buf = 0, acc_phase = 0;
      for (uint32_t u = cluster; u < plan.n_units && ok; u += n_clusters) {
        const Unit w = plan.at(u);
        if (w.kbn == 0) continue;
        const bool a_mn = MODE == kGrads && !w.grad_hidden, b_mn = MODE == kGrads;
        const uint32_t idesc = instr_desc(a_mn, b_mn);
        const uint32_t ka = (a_mn ? 2048u : 32u) >> 4, kb = (b_mn ? 2048u : 32u) >> 4;   // 16 deep, in descriptor units
        if (!mbar_wait(smem_u32(&bars->acc_empty[buf]), acc_phase ^ 1, c.wait_limit)) { ok = false; break; }
        fence_after();
        const uint32_t acc = tmem + buf * kHeadBN;
        for (uint32_t i = 0; i < w.kbn; ++i) {
          if (!mbar_wait(full0 + stage * 8, phase, c.wait_limit)) { ok = false; break; }
          fence_after();
          const uint64_t da = desc0 + stage * (kStageBytes >> 4), db = da + (kOperandBytes >> 4);
#pragma unroll
          for (uint32_t j = 0; j < kHeadBK / 16; ++j) mma_f16(acc, da + j * ka, db + j * kb, idesc, (i | j) != 0);
          mma_commit(empty0 + stage * 8);
          if (++stage == kStages) { stage = 0; phase ^= 1; }
        }
        if (!ok) break;
        mma_commit(smem_u32(&bars->acc_full[buf]));
        if (++buf == 2) { buf = 0; acc_phase ^= 1; }
      }
    }
  } else if (warp >= 4) {
    const uint32_t quarter = warp & 3, half = (warp - 4) >> 2;    // 32 rows, 128 of the tile's columns
    const uint32_t lane_base = tmem + ((quarter * 32) << 16) + half * 128;
    Stager<kBufs> out(tile_base + kStages * kStageBytes + (warp - 4) * kBufs * kStoreBytes, lane);
    uint32_t buf = 0, phase = 0;
    const float scale = mean_scale(c, count);
    for (uint32_t u = cluster; u < plan.n_units; u += n_clusters) {
      const Unit w = plan.at(u);
      const bool empty = w.kbn == 0;
      const uint32_t row0 = w.m0 + rank * 128 + quarter * 32, row = row0 + lane;
      const uint32_t n0 = w.n0 + half * 128;
      // Rows nobody reads are left out: beyond the rows that take part, for dL/dz beyond the depth of the weight product.
      bool work = true;
      if constexpr (MODE == kStats) work = row0 < (KEEP ? (count + kHeadBK - 1) / kHeadBK * kHeadBK : count);
      if constexpr (MODE == kDlogits) work = row0 < (count + kHeadBK - 1) / kHeadBK * kHeadBK;
      if constexpr (MODE == kGrads) work = w.grad_hidden ? row0 < count : (row0 < piece.width && n0 < c.dim);
      // what the tile's rows need besides the accumulator is fetched before the wait
      StatsRow<TWO, FLAG> st;
      DlogitsRow<TWO, FLAG, kBufs> dl;
      if constexpr (MODE == kStats) {
        st.zs = c.slot_z + uint64_t(row) * c.slots;
        if (row < count) st.open(c.slot_idx + uint64_t(row) * c.slots, c.slots, first_slot(c, row, n0));
      } else if constexpr (MODE == kDlogits) {
        dl.val = c.slot_g + uint64_t(row) * c.slots;
        dl.k = make_float4(0.f, 0.f, 0.f, 0.f);
        dl.live = row < count;
        if (dl.live) {
          dl.k = c.coef[row];
          dl.open(c.slot_idx + uint64_t(row) * c.slots, c.slots, first_slot(c, row, piece.v0 + n0));
        }
      }
      if (!empty) {
        ok = mbar_wait(smem_u32(&bars->acc_full[buf]), phase, c.wait_limit);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        fence_after();
      }
      const uint32_t acc = lane_base + buf * kHeadBN;
      uint32_t hi = 0, lo = 0;
      // chunk 0..3: 32 columns each
      auto process = [&](float (&v)[32], uint32_t chunk) {
        const uint32_t n = n0 + chunk * 32;
        if constexpr (MODE == kStats) {
          if constexpr (KEEP) {
            if (n0 >= c.keep_v0) {
              hi = out.acquire();
              out.put_f32(hi, v);
              out.send3(&maps.store, int(row0), int((n - c.keep_v0) / 32), hi);
            }
          }
          st.chunk(v, int32_t(n), c.vocab, c.cT, c.c1);
        } else if constexpr (MODE == kDlogits) {
          if (!(chunk & 1)) {
            hi = out.acquire();
            if constexpr (FLAG) lo = out.acquire_next();
          }
          dl.chunk(v, int32_t(piece.v0 + n0 + (chunk & 2) * 32), chunk & 1, c.vocab, c.cT, c.c1, out, hi, lo);
          if (chunk & 1) {
            out.send3(&maps.store, int(row0), dz_panel(piece, n, 0), hi);
            if constexpr (FLAG) out.send3(&maps.store, int(row0), dz_panel(piece, n, 1), lo);
          }
        } else {
          if (!w.grad_hidden) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] *= scale;
          }
          if (w.grad_hidden) {
            // [split][rows_cap][dcap]; pieces after the first add to their split's sums, one after the other
            if (!empty || piece.first) {
              hi = out.acquire();
              out.put_f32(hi, v);
              out.send(&maps.store2, int(n), int(w.split * c.rows_cap + row0), hi, !piece.first);
            }
          } else if (c.direct_store) {
            if (row < piece.width && n < c.dim) {
              const uint64_t at = uint64_t(piece.v0 + row) * c.grad_weight_stride + n;
              const uint32_t left = c.dim - n;
              if (c.grad_f32) store_row32<float>(static_cast<float*>(c.grad_weight) + at, v, left, c.accumulate);
              else store_row32<uint16_t>(static_cast<uint16_t*>(c.grad_weight) + at, v, left, c.accumulate);
            }
          } else if (c.grad_f32) {
            hi = out.acquire();
            out.put_f32(hi, v);
            if (n < c.dim) out.send(&maps.store, int(n), int(piece.v0 + row0), hi, c.accumulate); else out.skip();
          } else {
            if (!(chunk & 1)) hi = out.acquire();
            out.put_bf16(hi, chunk & 1, v);
            if (chunk & 1) {
              if (n - 32 < c.dim) out.send(&maps.store, int(n - 32), int(piece.v0 + row0), hi, false); else out.skip();
            }
          }
        }
        __syncwarp();
      };
      if (empty) {
        if (work) {
#pragma unroll 1
          for (uint32_t chunk = 0; chunk < 4; ++chunk) {
            float v[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = 0.f;
            process(v, chunk);
          }
        }
        continue;
      }
#pragma unroll 1
      for (uint32_t chunk = 0; chunk < 4; ++chunk) {
        float v[32];
        if (work) tmem_load(acc + chunk * 32, v);
        if (chunk == 3) {                       // the accumulator is in registers: the next product may overwrite it
          fence_before();
          if (lane == 0) mbar_arrive_cluster(leader_addr(smem_u32(&bars->acc_empty[buf])));
        }
        if (work) process(v, chunk);
      }
      if constexpr (MODE == kStats) {
        if (work) {
          const uint64_t at = uint64_t(n0 / kHeadStatCols) * c.rows_cap + row;
          c.part_m[at] = st.m;
          c.part_s[at] = st.s;
          if constexpr (TWO) c.part_s1[at] = st.s1;
          if constexpr (FLAG) c.part_z[at] = st.sz;
        }
      }
      if (++buf == 2) { buf = 0; phase ^= 1; }
    }
    out.drain();
  }
  if (!ok) {
    atomicOr(&c.state->status, uint32_t(FLS_STATUS_WAIT_EXPIRED));
    bars->gave_up = 1;
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  // A role that gave up may have copies in flight: let them land (bounded) before shared memory goes away.
  if (bars->gave_up) {
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
  }
  cluster_sync();
  if (warp == 2) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// ------------------------------------------------------------------------------------------------ rows
__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  return x;
}

// Which rows take part is a bit per row, and a count per 256 rows.
constexpr uint32_t kRowChunk = 256;

// One thread per row.  Rows that take no part get their outputs here.
__device__ __forceinline__ bool row_active(const HeadCall& c, uint64_t n, bool write) {
  bool active = false, bad = false;
  if (c.use_label) {
    const int64_t y = c.labels[n];
    bad = y != c.ignore_label && (y < 0 || y >= int64_t(c.vocab));
    active = y != c.ignore_label;
  }
  for (uint32_t k0 = 0; k0 < c.top && !active; k0 += 8) {              // eight at a time: rows without any read all of them
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
      const uint64_t at = n * c.top + min(k0 + j, c.top - 1);
      const int32_t i = c.top_index[at];
      active |= i >= 0 && uint32_t(i) < c.vocab && c.top_logit[at] != -INFINITY;
    }
  }
  active = active && !bad;
  if (!active && write) {
    c.loss[n] = bad ? NAN : 0.f;
    c.lse[n] = bad ? NAN : 0.f;
  }
  return active;
}

__global__ void __launch_bounds__(kRowChunk) fls_head_map_kernel(const __grid_constant__ HeadCall c) {
  pdl_launch();
  pdl_wait();
  const uint64_t n = uint64_t(blockIdx.x) * kRowChunk + threadIdx.x;
  const bool active = n < c.rows && row_active(c, n, true);
  const uint32_t mask = __ballot_sync(0xFFFFFFFFu, active);
  if ((threadIdx.x & 31) == 0) c.row_mask[n / 32] = mask;
  const int count = __syncthreads_count(active);
  if (threadIdx.x == 0) c.row_count[blockIdx.x] = uint32_t(count);
}

// One block per row: its packed position is the number of rows before it that take part.  A row that does is copied there
// with its own columns in ascending order; block i also clears packed row i if that is one of those between the rows that
// take part and the next multiple of 256.  ONE_CHUNK: at most 256 rows; every block looks at all of them itself and the map
// kernel is not needed.
template <bool ONE_CHUNK>
__global__ void __launch_bounds__(ONE_CHUNK ? 256 : 128) fls_head_pack_kernel(const __grid_constant__ HeadCall c) {
  __shared__ int32_t s_idx[FLS_HEAD_MAX_TOP + 1];
  __shared__ int32_t s_sorted[FLS_HEAD_MAX_TOP + 1];
  __shared__ float s_t[FLS_HEAD_MAX_TOP + 1];
  __shared__ double s_z[8];
  __shared__ uint32_t s_mask[kRowChunk / 32], s_before, s_count;
  const uint32_t i = blockIdx.x, chunk = i / kRowChunk;
  if (threadIdx.x == 0) s_before = s_count = 0;
  pdl_launch();
  pdl_wait();
  __syncthreads();
  if constexpr (ONE_CHUNK) {
    const uint64_t n = threadIdx.x;
    const bool active = n < c.rows && row_active(c, n, i == 0);
    const uint32_t mask = __ballot_sync(0xFFFFFFFFu, active);
    if ((threadIdx.x & 31) == 0) s_mask[threadIdx.x / 32] = mask;
    s_count = uint32_t(__syncthreads_count(active));
  } else {
    if (threadIdx.x < kRowChunk / 32) s_mask[threadIdx.x] = chunk * kRowChunk < c.rows ? c.row_mask[chunk * (kRowChunk / 32) + threadIdx.x] : 0u;
    uint32_t before = 0, all = 0;
    for (uint32_t k = threadIdx.x; k < uint32_t((c.rows + kRowChunk - 1) / kRowChunk); k += blockDim.x) {
      const uint32_t x = c.row_count[k];
      all += x;
      before += k < chunk ? x : 0u;
    }
    before = __reduce_add_sync(0xFFFFFFFFu, before);
    all = __reduce_add_sync(0xFFFFFFFFu, all);
    if ((threadIdx.x & 31) == 0) { atomicAdd(&s_before, before); atomicAdd(&s_count, all); }
    __syncthreads();
  }
  const uint32_t count = s_count, bit = i % kRowChunk;
  uint32_t p = s_before;
  for (uint32_t w = 0; w < bit / 32; ++w) p += __popc(s_mask[w]);
  p += __popc(s_mask[bit / 32] & ((1u << (bit & 31)) - 1));
  const bool active = (s_mask[bit / 32] >> (bit & 31)) & 1;
  if (threadIdx.x == 0) {
    if (i == 0) c.state->count = count;
    if (i < c.rows) c.pos[i] = active ? int32_t(p) : -1;
    if (active) c.src[p] = int32_t(i);
  }
  if (i >= count && i < (count + kHeadBM - 1) / kHeadBM * kHeadBM) {
    uint4* out = reinterpret_cast<uint4*>(c.hp + uint64_t(i) * c.dp);
    for (uint32_t k = threadIdx.x; k < c.dp / 8; k += blockDim.x) out[k] = make_uint4(0, 0, 0, 0);
  }
  if (!active) return;
  const uint64_t n = i;
  uint16_t* out = c.hp + uint64_t(p) * c.dp;
  const uint16_t* in = c.hidden + n * c.hidden_stride;
  if (c.dim % 8 == 0 && aligned16(in)) {
    for (uint32_t k = threadIdx.x; k < c.dp / 8; k += blockDim.x) reinterpret_cast<uint4*>(out)[k] = reinterpret_cast<const uint4*>(in)[k];
  } else {
    for (uint32_t k = threadIdx.x; k < c.dp; k += blockDim.x) out[k] = k < c.dim ? in[k] : uint16_t(0);
  }
  // The label's logit, of which the loss is a small difference, from the same products summed in double: the tensor cores
  // truncate as they add (losses off 64 bits at d = 2048 and 4096: 9.2e-7 and 1.9e-6, with this 5.3e-7 and 1.1e-6).
  if (c.use_label && c.labels[n] != c.ignore_label) {
    const uint16_t* w = c.weight + uint64_t(c.labels[n]) * c.weight_stride;
    double z = 0.0;
    if (c.dim % 8 == 0 && aligned16(in) && aligned16(w)) {
      for (uint32_t k = threadIdx.x; k < c.dim / 8; k += blockDim.x) {
        const uint4 a = reinterpret_cast<const uint4*>(in)[k], b = reinterpret_cast<const uint4*>(w)[k];
        const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
        float t = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          t = fmaf(__uint_as_float(x[e] << 16), __uint_as_float(y[e] << 16), t);
          t = fmaf(__uint_as_float(x[e] & 0xFFFF0000u), __uint_as_float(y[e] & 0xFFFF0000u), t);
        }
        z += double(t);
      }
    } else {
      for (uint32_t k = threadIdx.x; k < c.dim; k += blockDim.x)
        z += double(__uint_as_float(uint32_t(in[k]) << 16) * __uint_as_float(uint32_t(w[k]) << 16));
    }
    z = warp_sum(z);
    if ((threadIdx.x & 31) == 0) s_z[threadIdx.x / 32] = z;
    __syncthreads();
    if (threadIdx.x == 0) {
      z = s_z[0];
      for (uint32_t k = 1; k < blockDim.x / 32; ++k) z += s_z[k];
      c.label_z[p] = float(z);
    }
  }
  for (uint32_t k = threadIdx.x; k < c.slots; k += blockDim.x) {
    int32_t idx = INT_MAX;
    float t = -INFINITY;
    if (k < c.top) {
      const int32_t x = c.top_index[n * c.top + k];
      const float y = c.top_logit[n * c.top + k];
      if (x >= 0 && uint32_t(x) < c.vocab && y != -INFINITY) { idx = x; t = y; }
    } else if (c.use_label) {
      const int64_t y = c.labels[n];
      if (y != c.ignore_label) idx = int32_t(y);
    }
    s_idx[k] = idx;
    s_t[k] = t;
  }
  __syncthreads();
  for (uint32_t k = threadIdx.x; k < c.slots; k += blockDim.x) {
    const int32_t x = s_idx[k];
    uint32_t rank = 0;
    for (uint32_t j = 0; j < c.slots; ++j) rank += s_idx[j] < x || (s_idx[j] == x && j < k);
    c.slot_idx[uint64_t(p) * c.slots + rank] = x;
    c.slot_t[uint64_t(p) * c.slots + rank] = s_t[k];
    s_sorted[rank] = x;
  }
  if (c.slots == 1) return;
  __syncthreads();
  for (uint32_t t = threadIdx.x; t < c.tiles; t += blockDim.x) {
    const int32_t col = int32_t(t * kHeadStatCols);
    uint32_t lo = 0, len = c.slots;
    while (len) {
      const uint32_t h = len >> 1;
      if (s_sorted[lo + h] < col) { lo += h + 1; len -= h + 1; } else len = h;
    }
    c.slot_start[uint64_t(p) * c.tiles + t] = uint8_t(lo);
  }
}

__global__ void __launch_bounds__(256) fls_head_pack_weight_kernel(const uint16_t* w, uint64_t stride, uint16_t* out, uint32_t dim, uint32_t dp) {
  pdl_launch();
  pdl_wait();
  const uint64_t v = blockIdx.x;
  for (uint32_t i = threadIdx.x; i < dp; i += blockDim.x) out[v * dp + i] = i < dim ? w[v * stride + i] : uint16_t(0);
}

__device__ __forceinline__ double warp_max(double x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = fmax(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
  return x;
}

// Eight packed rows per block.  First the partial sums of each row are joined: a warp reads four columns' worth of eight
// neighbouring rows, whole 32-byte sectors.  Then a warp takes a row: its own columns are added to the sums and give loss
// and gradient.  Sums over the row and logarithms are double: a few hundred operations beside 2 V d of the products.
// TEACHER: distillation.  Cross entropy has one own column per row and gets code without the teacher's: a call of one row
// waits for it to come from memory (1 x 50257 x 768: 27.1 us a call with it, 25.4 without).
// Blocks start where the products' kernel ends first, and as many as fit there: few of them would share a few SMs while the
// others idle.  kRowsSpread bytes of shared memory that nothing uses keep it at two per SM where all fit that way (step of
// 128 x 50257 x 768 with five, three, two per SM: 90.6, 87.0, 85.0 us).
constexpr uint32_t kRowsSpread = 85 * 1024;
constexpr uint32_t kRowsPerBlock = 8;
template <bool TEACHER>
__global__ void __launch_bounds__(256) fls_head_rows_kernel(const __grid_constant__ HeadCall c) {
  __shared__ float sh_m[32][kRowsPerBlock], sh_s[32][kRowsPerBlock], sh_s1[32][kRowsPerBlock], sh_z[32][kRowsPerBlock];
  constexpr int kSlots = TEACHER ? FLS_HEAD_MAX_TOP + 1 : 1;
  __shared__ double sh_q[kRowsPerBlock][kSlots];
  __shared__ int32_t sh_i[kRowsPerBlock][kSlots];
  __shared__ float sh_t[kRowsPerBlock][kSlots], sh_zs[kRowsPerBlock][kSlots];
  const uint32_t slots = TEACHER ? c.slots : 1;
  const bool two = TEACHER && c.two, smooth = !TEACHER && c.smooth;
  const uint32_t lane = threadIdx.x & 31, y = threadIdx.x >> 5;
  pdl_launch();
  pdl_wait();
  const uint32_t count = c.state->count, p0 = blockIdx.x * kRowsPerBlock;
  // How the gradient launches split their depth: good with and without the weight gradient, and from nothing that depends on
  // which of the two is asked for (as are the pieces), so that one gradient alone has the same bits as both together.
  if (blockIdx.x == 0 && y == 7 && c.split_cols) {
    const uint32_t nt = (c.dim + kHeadBN - 1) / kHeadBN, th = (count + kHeadBM - 1) / kHeadBM * nt, kb_h = c.split_cols / kHeadBK;
    const uint32_t tw = c.split_cols / kHeadBM * nt, kb_w = (count + kHeadBK - 1) / kHeadBK * c.terms;
    uint32_t best = 0xFFFFFFFFu;
    for (uint32_t s = lane + 1; s <= min(c.max_splits, kb_h); s += 32)
      best = min(best, min(head_makespan(s, th, kb_h, tw, kb_w, c.clusters) + head_makespan(s, th, kb_h, 0, 0, c.clusters), 0x3FFFFFFu) << 6 | (s - 1));
    best = __reduce_min_sync(0xFFFFFFFFu, best);
    if (lane == 0) c.state->splits = (best & 63) + 1;
  }
  if (p0 >= count) return;
  const uint32_t p = min(p0 + y, count - 1);
  const uint64_t n = uint64_t(c.src[p]);               // used after the sums
  const int32_t* idx = c.slot_idx + uint64_t(p) * slots;
  const float* zs = c.slot_z + uint64_t(p) * slots;
  const float* ts = c.slot_t + uint64_t(p) * slots;
  float* gs = c.slot_g + uint64_t(p) * slots;
  {
    const uint32_t r = threadIdx.x % kRowsPerBlock, t0 = threadIdx.x / kRowsPerBlock;   // packed rows to the next multiple of 256 exist
    float m = -INFINITY, s = 0.f, s1 = 0.f, z = 0.f;
    constexpr int B = 8;                               // loads in flight per thread
    for (uint32_t t = t0; t < c.tiles; t += 32 * B) {
      float tm[B], ts[B], t1[B];
#pragma unroll
      for (int j = 0; j < B; ++j) {
        const bool in = t + 32 * j < c.tiles;
        const uint64_t at = uint64_t(in ? t + 32 * j : t) * c.rows_cap + p0 + r;
        tm[j] = in ? c.part_m[at] : -INFINITY;
        ts[j] = in ? c.part_s[at] : 0.f;
        t1[j] = in && two ? c.part_s1[at] : 0.f;
        z += in && smooth ? c.part_z[at] : 0.f;
      }
      float nm = m;
#pragma unroll
      for (int j = 0; j < B; ++j) nm = fmaxf(nm, tm[j]);
      const float base = nm == -INFINITY ? 0.f : nm;
      const Log2Ratio toT(base, c.cT), to1(base, c.c1);
      s *= exp2f(toT(m));                              // an empty side has factor 2^-inf = 0
      if (two) s1 *= exp2f(to1(m));
#pragma unroll
      for (int j = 0; j < B; ++j) {
        // columns all left out: m = -inf and s = 0; NaN goes through
        s += ts[j] * (tm[j] == -INFINITY ? 1.f : exp2f(toT(tm[j])));
        if (two) s1 += t1[j] * (tm[j] == -INFINITY ? 1.f : exp2f(to1(tm[j])));
      }
      m = nm;
    }
    sh_m[t0][r] = m;
    sh_s[t0][r] = s;
    sh_s1[t0][r] = s1;
    sh_z[t0][r] = z;
  }
  // what this warp needs of its row comes while the others finish
  const int64_t label = c.use_label ? c.labels[n] : c.ignore_label;
  const double w = c.row_weight ? double(c.row_weight[n]) : 1.0;      // the mean's 1 / count: mean_scale
  float mf = -INFINITY;
  for (uint32_t i = lane; i < slots; i += 32) {
    const int32_t x = idx[i];
    sh_i[y][i] = x;
    const float z = c.use_label && int64_t(x) == label && label != c.ignore_label ? c.label_z[p] : zs[i];
    sh_t[y][i] = ts[i];
    sh_zs[y][i] = z;
    if (x != INT_MAX) mf = fmaxf(mf, z);
  }
  __syncthreads();
  {
    if (p0 + y >= count) return;
    mf = fmaxf(mf, sh_m[lane][y]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mf = fmaxf(mf, __shfl_xor_sync(0xFFFFFFFFu, mf, o));
    const float base = mf == -INFINITY ? 0.f : mf, lm = sh_m[lane][y];
    const double M = double(base);
    const double denseT = warp_sum(double(sh_s[lane][y]) * (lm == -INFINITY ? 1.0 : double(exp2f(Log2Ratio(base, c.cT)(lm)))));
    const double dense1 = !two ? denseT : warp_sum(double(sh_s1[lane][y]) * (lm == -INFINITY ? 1.0 : double(exp2f(Log2Ratio(base, c.c1)(lm)))));
    const double zsum = smooth ? warp_sum(double(sh_z[lane][y])) : 0.0;
    const bool labelled = c.use_label && label != c.ignore_label;

    // the teacher's probabilities: log q = (t - shift) / T - norm; the list's maximum goes first, so that entries at the
    // type's lowest value keep log k
    bool taught = false;
    double norm = 0.0, shift = 0.0, tmax = -INFINITY;
    if constexpr (TEACHER) {
      bool nan_t = false;
      for (uint32_t i = lane; i < slots; i += 32)
        if (sh_i[y][i] != INT_MAX && sh_t[y][i] != -INFINITY) { tmax = fmax(tmax, double(sh_t[y][i])); nan_t |= isnan(sh_t[y][i]); }
      tmax = warp_max(tmax);
      taught = __any_sync(0xFFFFFFFFu, nan_t) || tmax != -INFINITY;
    }
    if (taught) {
      if (c.tail_class) norm = double(c.teacher_lse[n]);
      else {
        shift = tmax == -INFINITY ? 0.0 : tmax;
        double a = 0.0;
        for (uint32_t i = lane; i < slots; i += 32)
          if (sh_i[y][i] != INT_MAX && sh_t[y][i] != -INFINITY) a += exp((double(sh_t[y][i]) - shift) * c.inv_temp);
        norm = log(warp_sum(a));
      }
    }
    // own columns: their exponentials, with those of the label apart from the rest
    double ownT = 0.0, own1 = 0.0, eT_label = 0.0, e1_label = 0.0, z_label = 0.0, qsum = 0.0;
    float out_z = -INFINITY;                               // the label's logit where it is not in the teacher's list
    for (uint32_t i = lane; i < slots; i += 32) {
      double qi = 0.0;
      const int32_t x = sh_i[y][i];
      if (x != INT_MAX) {
        if (TEACHER && sh_t[y][i] != -INFINITY) { qi = exp((double(sh_t[y][i]) - shift) * c.inv_temp - norm); qsum += qi; }
        const bool first = i == 0 || sh_i[y][i - 1] != x;
        if (first) {
          bool listed = false;
          for (uint32_t j = i; j < slots && sh_i[y][j] == x; ++j) listed |= sh_t[y][j] != -INFINITY;
          const double eT = exp((double(sh_zs[y][i]) - M) * c.inv_temp), e1 = two ? exp(double(sh_zs[y][i]) - M) : eT;
          if (labelled && int64_t(x) == label) { eT_label = eT; e1_label = e1; z_label = double(sh_zs[y][i]); }
          else { ownT += eT; own1 += e1; }
          if (!listed) out_z = sh_zs[y][i];    // the label outside the teacher's list belongs to the tail
        }
      }
      sh_q[y][i] = qi;
    }
    ownT = warp_sum(ownT); own1 = warp_sum(own1); qsum = warp_sum(qsum);
    eT_label = warp_sum(eT_label); e1_label = warp_sum(e1_label); z_label = warp_sum(z_label);
    __syncwarp();
    const double restT = denseT + ownT, rest1 = dense1 + own1;         // everything but the label
    const double totT = restT + eT_label, tot1 = rest1 + e1_label;
    // What is outside the list, relative to its own maximum: relative to the row's nothing of it is left where a student is sure.
    const bool class_t = taught && c.tail_class;
    double tail = 0.0, tail_m = 0.0;
    if (class_t) {
      float tm = fmaxf(lm, out_z);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) tm = fmaxf(tm, __shfl_xor_sync(0xFFFFFFFFu, tm, o));
      if (tm == -INFINITY) tm = 0.f;
      tail_m = double(tm);
      tail = double(sh_s[lane][y]) * (lm == -INFINITY ? 1.0 : double(exp2f(Log2Ratio(tm, c.cT)(lm))));
      if (out_z != -INFINITY) tail += exp((double(out_z) - tail_m) * c.inv_temp);
      tail = warp_sum(tail);
    }
    // Four logarithms, one per lane: of the sums (at least 1: the maximum's own term) at T and 1, -log p_label where the
    // label dominates and lse - z would cancel, and of the tail's sum (at least 1, or 0 where nothing is outside the list).
    const double part = log1p(lane == 0 ? totT - 1.0 : lane == 1 ? tot1 - 1.0 : lane == 2 ? rest1 / e1_label : tail - 1.0);
    const double log_T = __shfl_sync(0xFFFFFFFFu, part, 0), log_1 = __shfl_sync(0xFFFFFFFFu, part, 1), log_p = __shfl_sync(0xFFFFFFFFu, part, 2);
    const double log_tail = __shfl_sync(0xFFFFFFFFu, part, 3), lse_tail = tail_m * c.inv_temp + log_tail;
    // A log sum exp of m / T + l, where its exponentials' exponents z cc - (.) are formed.  Far from zero it is rounded up, from
    // the fp32 factor that z gets: no rounding makes a probability exceed 1.
    auto exponent = [](double m, float cc, double t, double l) {
      constexpr double kLog2e = 1.4426950408889634;
      const double e = (m * t + l) * kLog2e;
      return fabs(e) < double(kFar) ? float(e) : __double2float_ru(m * double(cc) + l * kLog2e);
    };
    const float exp_T = exponent(M, c.cT, c.inv_temp, log_T);
    const double lseT = M * c.inv_temp + log_T, lse1 = two ? M + log_1 : lseT;
    const double nll = !labelled ? 0.0 : (rest1 < e1_label ? log_p : (two ? lse1 - z_label : lseT - z_label * c.inv_temp));

    if constexpr (!TEACHER) {
      const double pl = e1_label / totT, ql = restT / totT, zl = 2.0 * c.z_loss * lseT, eps = c.smoothing;
      if (lane == 0) {
        double loss = (1.0 - eps) * nll + c.z_loss * lseT * lseT;
        if (smooth) loss += eps * (lseT - zsum / double(c.vocab));
        c.loss[n] = float(loss);
        c.lse[n] = float(lseT);
        c.coef[p] = make_float4(exp_T, float(w * (1.0 + zl)), float(w * eps / double(c.vocab)), 0.f);
        gs[0] = float(w * (-ql + zl * pl + eps - eps / double(c.vocab)));
      }
    } else {
      double kl = 0.0;
      for (uint32_t i = lane; i < slots; i += 32)
        if (sh_i[y][i] != INT_MAX && sh_t[y][i] != -INFINITY) {
          const double qi = sh_q[y][i];
          if (qi != 0.0) kl += qi * (((double(sh_t[y][i]) - shift) * c.inv_temp - norm) - (double(sh_zs[y][i]) * c.inv_temp - lseT));
        }
      kl = warp_sum(kl);
      // Outside the list dL/dz = a p (1 - q'/p') = a r (p' - q'), r = p / p' = exp(z/T - lse_tail): neither factor exceeds 1
      // however small p' is, where q'/p' would overflow and p vanish (in fp32 from 87 T between the list and the rest on).
      const bool split_tail = class_t && lse_tail != -INFINITY;
      float exp_out = exp_T;
      double lse_out = lseT, p_out = 1.0, d_out = 1.0;      // p = p_out exp(z/T - lse_out), its distillation factor d_out for p_out
      if (class_t) {
        const double qt = qsum > 1.0 ? 0.0 : 1.0 - qsum;
        if (qt > (split_tail ? 0.0 : 1e-6)) kl += qt * (log(qt) - (lse_tail - lseT));   // without a tail what is left of 1 is rounding
        if (split_tail) {
          lse_out = lse_tail;
          exp_out = exponent(tail_m, c.cT, c.inv_temp, log_tail);
          p_out = exp(lse_tail - lseT);
          d_out = p_out - qt;
        }
      }
      const double a = taught ? c.distill_weight * c.temp * w : 0.0, b = labelled ? c.label_weight * w : 0.0;
      if (lane == 0) {
        c.loss[n] = float((taught ? c.distill_weight * c.temp * c.temp * kl : 0.0) + (labelled ? c.label_weight * nll : 0.0));
        c.lse[n] = float(lseT);
        if (two) c.coef[p] = make_float4(exp_out, float(a * d_out), exponent(M, c.c1, 1.0, log_1), float(b));
        else c.coef[p] = make_float4(exp_out, float(a * d_out + b * p_out), 0.f, 0.f);
      }
      for (uint32_t i = lane; i < slots; i += 32) {
        const int32_t x = sh_i[y][i];
        if (x == INT_MAX) continue;
        double qi = 0.0;
        bool listed = false;
        for (uint32_t j = i + 1; j-- > 0 && sh_i[y][j] == x;) { qi += sh_q[y][j]; listed |= sh_t[y][j] != -INFINITY; }
        for (uint32_t j = i + 1; j < slots && sh_i[y][j] == x; ++j) { qi += sh_q[y][j]; listed |= sh_t[y][j] != -INFINITY; }
        const double zT = double(sh_zs[y][i]) * c.inv_temp, pT = exp(zT - lseT);
        double v = a * (listed ? pT - qi : exp(zT - lse_out) * d_out);
        if (labelled) v += b * (int64_t(x) == label ? -rest1 / tot1 : (two ? exp(double(sh_zs[y][i]) - lse1) : pT));
        gs[i] = float(v);
      }
    }
  }
}

// dL/dz of the kept columns, in place: reads 4 bytes and writes 2 (two terms: 4) per element instead of forming the logit
// again.  The same operations on the same fp32 logit as in the kDlogits epilogue: the same bits.  Bound by memory: 1024 x
// 128256 in 122 us, 6.5 TB/s of its 6 bytes per element.  A block takes 128 rows of 64 columns; eight threads of a warp
// share a row, so what is overwritten has been read.
constexpr uint32_t kRescaleRows = 128;
template <bool TWO, bool PLANES>
__global__ void __launch_bounds__(256) fls_head_rescale_kernel(const __grid_constant__ HeadCall c) {
  pdl_launch();
  pdl_wait();
  const uint32_t count = c.state->count, live = (count + kHeadBK - 1) / kHeadBK * kHeadBK;
  const uint32_t panels = (c.vocab - c.keep_v0 + 63) / 64, panel = blockIdx.x % panels, first = blockIdx.x / panels * kRescaleRows;
  const uint32_t row0 = first + threadIdx.x / 8, sub = threadIdx.x % 8;
  if (first >= count) return;                                          // live rows end in the same block
  const uint32_t n = c.keep_v0 + panel * 64 + sub * 8;
  const uint64_t pitch = uint64_t(c.rows_cap) * 32;                    // floats per panel of 32 columns
  float* base = c.keep_z + 2 * uint64_t(panel) * pitch;
  float4 za[4], zb[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t row = min(row0 + q * 32, count - 1);                // the last row again beyond it
    const float4* x = reinterpret_cast<const float4*>(base + (sub / 4) * pitch + uint64_t(row) * 32 + (sub % 4) * 8);
    za[q] = x[0];
    zb[q] = x[1];
  }
  uint4 hi[4], lo[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const bool in = row0 + q * 32 < count;
    const float4 k = c.coef[min(row0 + q * 32, count - 1)];
    float v[8] = {za[q].x, za[q].y, za[q].z, za[q].w, zb[q].x, zb[q].y, zb[q].z, zb[q].w};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float z = v[j];
      if constexpr (TWO) v[j] = fmaf(k.w, ex2(fmaf(z, c.c1, -k.z)), k.y * ex2(fmaf(z, c.cT, -k.x)));
      else v[j] = fmaf(k.y, ex2(fmaf(z, c.cT, -k.x)), -k.z);
      if (!in || n + j >= c.vocab) v[j] = 0.f;
    }
    hi[q] = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    if constexpr (PLANES) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] -= bf16_round(v[j]);
      lo[q] = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    }
  }
  __syncwarp();
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t row = row0 + q * 32;
    float* o = base + uint64_t(row) * 32 + sub * 4;                    // 16 bytes
    if (row < live) {
      *reinterpret_cast<uint4*>(o) = hi[q];
      if constexpr (PLANES) *reinterpret_cast<uint4*>(o + pitch) = lo[q];
    }
  }
}

// Then the rows' own columns among the kept ones.
__global__ void __launch_bounds__(128) fls_head_own_kernel(const __grid_constant__ HeadCall c) {
  pdl_launch();
  pdl_wait();
  const uint32_t i = blockIdx.x * 128 + threadIdx.x, row = i / c.slots;
  if (row >= c.state->count) return;
  const int32_t x = c.slot_idx[i] - int32_t(c.keep_v0);
  if (x < 0 || uint32_t(x) >= c.vocab - c.keep_v0) return;
  const float y = c.slot_g[i];
  uint16_t* o = c.g + (uint64_t(x / 64) * 2 * c.rows_cap + row) * 64 + x % 64;
  o[0] = bf16_bits(y);
  if (c.planes == 2) o[uint64_t(c.rows_cap) * 64] = bf16_bits(y - bf16_round(y));
}

// Bound by memory: 4 bytes per column and split in, 2 out (1024 x 2048, 9 splits: 18 us cold, 4.1 TB/s).
// One row, 256 / G groups of four columns per block; G threads share a group's split sums (each adds every G-th, then the G
// partial sums are added in order), so that with few rows and many splits the loads do not wait for one another.
template <int G>
__global__ void __launch_bounds__(256) fls_head_grad_hidden_kernel(const __grid_constant__ HeadCall c) {
  __shared__ float4 part[G > 1 ? 256 : 1];
  pdl_launch();
  pdl_wait();
  constexpr uint32_t kCols = 256 / G;
  const uint64_t n = blockIdx.x;
  const int32_t p = c.pos[n];
  uint16_t* out = c.grad_hidden + n * c.grad_hidden_stride;
  const uint32_t splits = c.state->splits, g = threadIdx.x / kCols;
  const bool vec = c.dim % 4 == 0 && (reinterpret_cast<uintptr_t>(out) & 7) == 0;
  for (uint32_t i0 = blockIdx.y * kCols * 4; i0 < c.dim; i0 += gridDim.y * kCols * 4) {
    const uint32_t i = i0 + threadIdx.x % kCols * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (p >= 0 && i < c.dim) {
      const float* x = c.dh + uint64_t(p) * c.dcap + i;
      const uint64_t step = uint64_t(c.rows_cap) * c.dcap;
#pragma unroll 8
      for (uint32_t s = g; s < splits; s += G) {
        const float4 a = *reinterpret_cast<const float4*>(x + s * step);
        v.x += a.x; v.y += a.y; v.z += a.z; v.w += a.w;
      }
    }
    if constexpr (G > 1) {
      __syncthreads();
      part[threadIdx.x] = v;
      __syncthreads();
      if (g) continue;
#pragma unroll
      for (uint32_t q = 1; q < G; ++q) {
        const float4 a = part[q * kCols + threadIdx.x];
        v.x += a.x; v.y += a.y; v.z += a.z; v.w += a.w;
      }
    }
    if (i >= c.dim) continue;
    const float scale = mean_scale(c, c.state->count);
    v.x *= scale; v.y *= scale; v.z *= scale; v.w *= scale;
    if (vec) *reinterpret_cast<uint2*>(out + i) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
    else {
      const float w[4] = {v.x, v.y, v.z, v.w};
      for (uint32_t j = 0; j < 4 && i + j < c.dim; ++j) out[i + j] = bf16_bits(w[j]);
    }
  }
}

// Kernels of a call after its first start while the one before ends (pdl_wait).
template <typename... P, typename... A>
cudaError_t launch(void (*k)(P...), dim3 grid, uint32_t block, uint32_t smem, bool first, cudaStream_t s, A&&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = first ? 0 : 1;
  return cudaLaunchKernelEx(&cfg, k, std::forward<A>(args)...);
}

template <int MODE, bool TWO, bool FLAG, bool KEEP = false>
cudaError_t launch_gemm(const HeadCall& c, const HeadMaps& m, const HeadPiece& p, cudaStream_t s) {
  auto* k = fls_head_gemm_kernel<MODE, TWO, FLAG, KEEP>;
  constexpr uint32_t kBytes = Smem<MODE, FLAG, KEEP>::kBytes;
  return launch(k, dim3(2 * c.clusters), kGemmThreads, kBytes, false, s, m, c, p);
}

}  // namespace

namespace {
template <int MODE, bool TWO, bool FLAG, bool KEEP = false>
cudaError_t allow_smem() {
  return cudaFuncSetAttribute(fls_head_gemm_kernel<MODE, TWO, FLAG, KEEP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<MODE, FLAG, KEEP>::kBytes);
}
}  // namespace

cudaError_t head_clusters(uint32_t* out) {
  for (cudaError_t e : {allow_smem<kStats, false, false>(), allow_smem<kStats, false, true>(), allow_smem<kStats, true, false>(),
                        allow_smem<kStats, false, false, true>(), allow_smem<kStats, false, true, true>(), allow_smem<kStats, true, false, true>(),
                        allow_smem<kDlogits, false, false>(), allow_smem<kDlogits, true, false>(), allow_smem<kDlogits, false, true>(),
                        allow_smem<kDlogits, true, true>(), allow_smem<kGrads, false, false>(),
                        cudaFuncSetAttribute(fls_head_rows_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRowsSpread),
                        cudaFuncSetAttribute(fls_head_rows_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRowsSpread)})
    if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(2);
  cfg.blockDim = dim3(kGemmThreads);
  cfg.dynamicSmemBytes = Smem<kStats, false, false>::kBytes;       // the variants differ little in it and not in CTAs per SM
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = 2; at.val.clusterDim.y = 1; at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  int n = 0;
  const cudaError_t e = cudaOccupancyMaxActiveClusters(&n, fls_head_gemm_kernel<kStats, false, false, false>, &cfg);
  *out = uint32_t(n > 0 ? n : 1);
  return e;
}

cudaError_t launch_head_rows_map(const HeadCall& c, cudaStream_t s) {
  return launch(fls_head_map_kernel, dim3(uint32_t((c.rows + kRowChunk - 1) / kRowChunk)), kRowChunk, 0, true, s, c);
}
cudaError_t launch_head_pack(const HeadCall& c, cudaStream_t s) {
  if (c.rows <= kRowChunk) return launch(fls_head_pack_kernel<true>, dim3(c.rows_cap), 256, 0, true, s, c);
  return launch(fls_head_pack_kernel<false>, dim3(c.rows_cap), 128, 0, false, s, c);
}
cudaError_t launch_head_pack_weight(const uint16_t* w, uint64_t stride, uint16_t* out, uint32_t vocab, uint32_t dim, uint32_t dp, cudaStream_t s) {
  return launch(fls_head_pack_weight_kernel, dim3(vocab), 256, 0, false, s, w, stride, out, dim, dp);
}
cudaError_t launch_head_stats(const HeadCall& c, const HeadMaps& m, cudaStream_t s) {
  const HeadPiece p{0, c.vocab, 0, 0};
  if (c.keep_v0 < c.vocab) {
    if (c.two) return launch_gemm<kStats, true, false, true>(c, m, p, s);
    if (c.smooth) return launch_gemm<kStats, false, true, true>(c, m, p, s);
    return launch_gemm<kStats, false, false, true>(c, m, p, s);
  }
  if (c.two) return launch_gemm<kStats, true, false>(c, m, p, s);
  if (c.smooth) return launch_gemm<kStats, false, true>(c, m, p, s);
  return launch_gemm<kStats, false, false>(c, m, p, s);
}
cudaError_t launch_head_rows(const HeadCall& c, cudaStream_t s) {
  const uint32_t blocks = c.rows_cap / kRowsPerBlock, smem = blocks <= 4 * c.clusters ? kRowsSpread : 0;      // a cluster is two SMs
  return launch(c.top ? fls_head_rows_kernel<true> : fls_head_rows_kernel<false>, dim3(blocks), 256, smem, false, s, c);
}
cudaError_t launch_head_dlogits(const HeadCall& c, const HeadMaps& m, const HeadPiece& p, cudaStream_t s) {
  if (c.planes == 2) return c.two ? launch_gemm<kDlogits, true, true>(c, m, p, s) : launch_gemm<kDlogits, false, true>(c, m, p, s);
  return c.two ? launch_gemm<kDlogits, true, false>(c, m, p, s) : launch_gemm<kDlogits, false, false>(c, m, p, s);
}
cudaError_t launch_head_own(const HeadCall& c, cudaStream_t s) {
  return launch(fls_head_own_kernel, dim3(uint32_t((std::max<uint64_t>(c.rows, 1) * c.slots + 127) / 128)), 128, 0, false, s, c);
}
cudaError_t launch_head_rescale(const HeadCall& c, cudaStream_t s) {
  const dim3 grid((c.vocab - c.keep_v0 + 63) / 64 * (c.rows_cap / kRescaleRows));      // either factor may exceed 65535
  if (c.planes == 2)
    return c.two ? launch(fls_head_rescale_kernel<true, true>, grid, 256, 0, false, s, c) : launch(fls_head_rescale_kernel<false, true>, grid, 256, 0, false, s, c);
  return c.two ? launch(fls_head_rescale_kernel<true, false>, grid, 256, 0, false, s, c) : launch(fls_head_rescale_kernel<false, false>, grid, 256, 0, false, s, c);
}
cudaError_t launch_head_grads(const HeadCall& c, const HeadMaps& m, const HeadPiece& p, cudaStream_t s) {
  return launch_gemm<kGrads, false, false>(c, m, p, s);
}
cudaError_t launch_head_grad_hidden(const HeadCall& c, cudaStream_t s) {
  // few rows have many splits and few blocks (128 x 50257 x 768, 24 splits: 10.5 us with one thread per four columns)
  if (c.rows <= 512) return launch(fls_head_grad_hidden_kernel<8>, dim3(uint32_t(c.rows), (c.dim + 127) / 128), 256, 0, false, s, c);
  return launch(fls_head_grad_hidden_kernel<1>, dim3(uint32_t(c.rows)), 256, 0, false, s, c);
}

}  // namespace fls
