// C ABI of the language-model head (see include/fls.h): argument checks, workspace layout, launch order.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "fls_head.h"
#include "fls_internal.h"

using namespace fls;

namespace {

int cuda_fail(cudaError_t e, const char* what) { return refuse(FLS_ECUDA, "%s: %s", what, cudaGetErrorString(e)); }

constexpr uint64_t up(uint64_t x, uint64_t q) { return (x + q - 1) / q * q; }
constexpr uint32_t kWaitLimit = 1u << 20;            // polls, 4 us each, of a barrier before a role of the tensor-core kernel gives up
constexpr uint64_t kMinPieceCols = 512, kMaxPieceCols = 1ull << 28;
constexpr uint64_t kDefaultPieceBytes = 1ull << 30;
constexpr uint64_t kPartialBytes = 256ull << 20;     // room for the split sums of grad_hidden: at least 2, at most 64 splits

// Keeping a logit moves 8 bytes more than forming it again, which does 2 d operations or, with few rows, waits for the
// weight (2 d bytes per column of all rows).  Measured equal at d = 896 and, below it, at about 2 d / 3 rows (us a step,
// kept / formed again; 4096 x 50257: d = 256 658 / 496, 768 1030 / 1008, 896 1262 / 1262, 1024 1307 / 1355; 1024 x 128256,
// d = 2048: 1591 / 1738; d = 768, 50257 columns: 128 rows 99 / 108, 512 184 / 186, 1024 320 / 309; d = 256: 128 rows
// 74 / 75, 256 80 / 78).
bool keeps_logits(uint64_t rows, uint64_t dim) { return dim >= 896 || 3 * rows <= 2 * dim; }

// bf16 terms of dL/dz that the weight's gradient takes.
uint64_t terms_of(const fls_head_desc& d) { return d.grad_dtype == FLS_GRAD_F32 ? 2 : 1; }

// Byte offsets of the workspace.  Sizes are those of max_rows; a smaller call uses the front of each region.
struct Regions {
  uint64_t mask, counts, pos, src, hp, slot_idx, slot_start, slot_t, slot_z, slot_g, label_z, part, coef, g, dh, wcopy, total;
  uint64_t part_bytes, g_bytes, dh_bytes;
};

Regions regions(const fls_head_desc& d) {
  const uint64_t cap = up(std::max<uint64_t>(d.max_rows, 1), kHeadBM), dp = up(d.dim, 8), dcap = up(d.dim, kHeadBN);
  const uint64_t slots = uint64_t(d.top) + 1, tiles = up(d.vocab, kHeadBN) / kHeadStatCols;
  const uint64_t planes = terms_of(d);
  Regions r{};
  uint64_t at = 256;
  auto take = [&](uint64_t bytes) { const uint64_t o = at; at += up(bytes, 256); return o; };
  r.mask = take(cap / 8);
  r.counts = take(cap / 256 * 4);
  r.pos = take(cap * 4);
  r.src = take(cap * 4);
  r.hp = take(cap * dp * 2);
  r.slot_idx = take(cap * slots * 4);
  if (d.top) r.slot_start = take(cap * tiles);
  r.slot_t = take(cap * slots * 4);
  r.slot_z = take(cap * slots * 4);
  r.slot_g = take(cap * slots * 4);
  r.label_z = take(cap * 4);
  r.part_bytes = cap * tiles * 4;
  r.part = take(3 * r.part_bytes);          // maximum, sum, and one of: sum at temperature 1, sum of logits
  r.coef = take(cap * 16);
  if (d.grads) {
    const uint64_t all = (keeps_logits(d.max_rows, d.dim) ? 4 : 2 * planes) * cap * up(d.vocab, 256);   // the whole vocabulary in one piece
    r.g_bytes = std::min(all, std::max(d.piece_bytes ? d.piece_bytes : kDefaultPieceBytes, 2 * planes * cap * kMinPieceCols));
    r.g = take(r.g_bytes);
    r.dh_bytes = std::max<uint64_t>(2, std::min<uint64_t>(kHeadMaxSplits, kPartialBytes / (cap * dcap * 4))) * cap * dcap * 4;
    r.dh = take(r.dh_bytes);
  }
  if (d.any_weight || d.dim % 8) r.wcopy = take(d.vocab * dp * 2);
  r.total = at;
  return r;
}

// How the vocabulary is taken apart.  The last columns keep the logits of the statistics pass, 4 bytes each, and get their
// dL/dz from those; the columns before them are formed again, in pieces of 2 bytes per column and term, evened out.
struct Pieces { uint32_t keep_v0, cols; };
Pieces pieces_of(const fls_head_desc& d, uint64_t g_bytes, uint64_t rows, uint64_t planes) {
  const uint64_t rows_cap = up(std::max<uint64_t>(rows, 1), kHeadBM);
  Pieces p{};
  const uint64_t keep = !keeps_logits(rows, d.dim) ? 0 : std::min(kMaxPieceCols, g_bytes / (4 * rows_cap) / 256 * 256);
  const uint64_t v0 = keep >= d.vocab ? 0 : keep ? up(d.vocab - keep, 256) : d.vocab;
  p.keep_v0 = uint32_t(std::min(v0, d.vocab));
  if (p.keep_v0) {
    const uint64_t vr = up(p.keep_v0, 256);
    const uint64_t most = std::min({vr, kMaxPieceCols, std::max<uint64_t>(256, g_bytes / (2 * planes * rows_cap) / 256 * 256)});
    const uint64_t n = (vr + most - 1) / most;
    p.cols = uint32_t(up((vr + n - 1) / n, 256));
  }
  return p;
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Row-major bf16 or fp32 matrix, boxes of 128 bytes x box_rows, 128-byte swizzle, zeros outside.
bool encode(EncodeTiled f, CUtensorMap* m, const void* base, uint64_t cols, uint64_t rows, uint64_t stride, uint32_t box_rows, bool f32 = false) {
  const cuuint64_t dims[2] = {cols, rows};
  const cuuint64_t strides[1] = {stride * (f32 ? 4 : 2)};
  const cuuint32_t box[2] = {f32 ? 32u : 64u, box_rows}, step[2] = {1, 1};
  return f(m, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, step,
           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Panels of 128 bytes x rows, boxes of box_rows rows of one panel.
bool encode_panels(EncodeTiled f, CUtensorMap* m, const void* base, uint64_t rows, uint64_t panels, uint32_t box_rows, bool f32 = false) {
  const cuuint64_t dims[3] = {f32 ? 32u : 64u, rows, panels};
  const cuuint64_t strides[2] = {128, rows * 128};
  const cuuint32_t box[3] = {f32 ? 32u : 64u, box_rows, 1}, step[3] = {1, 1, 1};
  return f(m, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, step,
           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Bytes from the first to the last element of a matrix with `stride` elements between rows.
uint64_t span_bytes(uint64_t rows, uint64_t cols, uint64_t stride, uint64_t elem) {
  return rows ? ((rows - 1) * stride + cols) * elem : 0;
}

}  // namespace

struct fls_head {
  fls_head_desc desc{};
  Regions reg{};
  int device = -1;
  uint32_t clusters = 0;
  EncodeTiled encode = nullptr;
  uint64_t launches = 0;
  uint32_t expire_polls = 0;        // test hook: the next call's waits run out after so many polls
};

namespace {

// What depends on the device is looked up at the first call on it.
int prepare_device(fls_head* h) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
  if (dev == h->device) return FLS_OK;
  void* f = nullptr;
  cudaDriverEntryPointQueryResult q{};
  e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q);
  if (e != cudaSuccess || !f) return cuda_fail(e, "cuTensorMapEncodeTiled not available");
  h->encode = reinterpret_cast<EncodeTiled>(f);
  e = head_clusters(&h->clusters);
  if (e != cudaSuccess) return cuda_fail(e, "cudaOccupancyMaxActiveClusters");
  h->device = dev;
  return FLS_OK;
}

int run(fls_head* h, const fls_head_io* io, HeadCall& c, void* cuda_stream) {
  const fls_head_desc& d = h->desc;
  const Regions& r = h->reg;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  int rc = prepare_device(h);
  if (rc) return rc;

  char* ws = static_cast<char*>(io->workspace);
  c.state = reinterpret_cast<HeadState*>(ws);
  c.row_mask = reinterpret_cast<uint32_t*>(ws + r.mask);
  c.row_count = reinterpret_cast<uint32_t*>(ws + r.counts);
  c.pos = reinterpret_cast<int32_t*>(ws + r.pos);
  c.src = reinterpret_cast<int32_t*>(ws + r.src);
  c.hp = reinterpret_cast<uint16_t*>(ws + r.hp);
  c.slot_idx = reinterpret_cast<int32_t*>(ws + r.slot_idx);
  c.slot_start = reinterpret_cast<uint8_t*>(ws + r.slot_start);
  c.slot_t = reinterpret_cast<float*>(ws + r.slot_t);
  c.slot_z = reinterpret_cast<float*>(ws + r.slot_z);
  c.slot_g = reinterpret_cast<float*>(ws + r.slot_g);
  c.label_z = reinterpret_cast<float*>(ws + r.label_z);
  c.part_m = reinterpret_cast<float*>(ws + r.part);
  c.part_s = reinterpret_cast<float*>(ws + r.part + r.part_bytes);
  c.part_s1 = c.part_z = reinterpret_cast<float*>(ws + r.part + 2 * r.part_bytes);
  c.coef = reinterpret_cast<float4*>(ws + r.coef);
  c.g = reinterpret_cast<uint16_t*>(ws + r.g);
  c.keep_z = reinterpret_cast<float*>(ws + r.g);
  c.dh = reinterpret_cast<float*>(ws + r.dh);
  c.hidden = static_cast<const uint16_t*>(io->hidden);
  c.hidden_stride = io->hidden_stride ? io->hidden_stride : d.dim;
  c.weight = static_cast<const uint16_t*>(io->weight);
  c.weight_stride = io->weight_stride ? io->weight_stride : d.dim;
  c.labels = io->labels;
  c.ignore_label = io->ignore_label;
  c.row_weight = io->row_weight;
  c.loss = io->loss;
  c.lse = io->lse;
  c.grad_hidden = static_cast<uint16_t*>(io->grad_hidden);
  c.grad_hidden_stride = io->grad_hidden_stride ? io->grad_hidden_stride : d.dim;
  c.grad_weight = io->grad_weight;
  c.grad_weight_stride = io->grad_weight_stride ? io->grad_weight_stride : d.dim;
  c.rows = io->rows;
  c.rows_cap = uint32_t(up(std::max<uint64_t>(io->rows, 1), kHeadBM));
  c.vocab = uint32_t(d.vocab);
  c.dim = d.dim;
  c.dp = uint32_t(up(d.dim, 8));
  c.dcap = uint32_t(up(d.dim, kHeadBN));
  c.slots = c.top + c.use_label;
  c.tiles = uint32_t(up(d.vocab, kHeadBN) / kHeadStatCols);
  c.grad_f32 = d.grad_dtype == FLS_GRAD_F32;
  c.accumulate = io->accumulate;
  c.want_gh = io->grad_hidden != nullptr && io->rows > 0;
  c.want_gw = io->grad_weight != nullptr;
  c.terms = uint32_t(terms_of(d));
  c.planes = c.want_gw ? c.terms : 1;
  c.clusters = h->clusters;
  // hidden rows of one group of row tiles: 32 MB, a quarter of L2, beside the weight tiles that stream past them.  No more
  // tiles than there are, so that a group's tiles of the vocabulary stay below the 2^31 that fls_head_create allows in all.
  c.group_m = std::max<uint32_t>(1, std::min(c.rows_cap / uint32_t(kHeadBM), uint32_t((32ull << 20) / (uint64_t(kHeadBM) * c.dp * 2))));
  c.hold_back = h->expire_polls != 0;
  c.wait_limit = h->expire_polls ? h->expire_polls : kWaitLimit;
  h->expire_polls = 0;
  c.c1 = 1.4426950408889634f;
  c.cT = float(1.4426950408889634 * c.inv_temp);
  const bool grads = c.want_gh || c.want_gw;
  c.keep_v0 = c.vocab;
  // A TMA store ends on a 16-byte boundary: with a row of any other length it writes into what follows the row (zeros, seen
  // in the first column after rows of 23 fp32, stride 24).
  const uint32_t we = c.grad_f32 ? 4 : 2;
  c.direct_store = reinterpret_cast<uintptr_t>(c.grad_weight) % 16 || c.grad_weight_stride * we % 16 || uint64_t(c.dim) * we % 16 ||
                   (c.accumulate && !c.grad_f32);
  if (grads) {
    const Pieces p = pieces_of(d, r.g_bytes, c.rows, terms_of(d));
    c.keep_v0 = p.keep_v0;
    c.piece_cols = p.cols;
    c.split_cols = std::max(p.cols, uint32_t(up(c.vocab - p.keep_v0, 256)));
    c.max_splits = uint32_t(std::min<uint64_t>(kHeadMaxSplits, r.dh_bytes / (uint64_t(c.rows_cap) * c.dcap * 4)));
  }
  if (io->rows == 0 && (!c.want_gw || io->accumulate)) {               // nothing to launch, but no rows took part
    const cudaError_t e = cudaMemsetAsync(&c.state->count, 0, sizeof c.state->count, s);
    return e == cudaSuccess ? FLS_OK : cuda_fail(e, "cudaMemsetAsync(rows that take part)");
  }

  const uint16_t* w = static_cast<const uint16_t*>(io->weight);
  uint64_t w_stride = io->weight_stride ? io->weight_stride : d.dim, w_cols = d.dim;
  const bool copy = d.dim % 8 || reinterpret_cast<uintptr_t>(w) % 16 || w_stride % 8;
  c.prefetch_weight = c.rows_cap == kHeadBM && !copy;
  if (copy) { w = reinterpret_cast<const uint16_t*>(ws + r.wcopy); w_stride = w_cols = c.dp; }

  // fwd: logits, and where they or their dL/dz are stored; grad: the two products of a piece, kept the same for the kept one
  const bool keeps = grads && c.keep_v0 < c.vocab, forms = grads && c.keep_v0 > 0;
  HeadMaps fwd{}, stat{}, grad{}, kept{};
  const auto f = h->encode;
  bool ok = encode(f, &fwd.a0, c.hp, c.dp, c.rows_cap, c.dp, 128) && encode(f, &fwd.b0, w, w_cols, d.vocab, w_stride, 128);
  fwd.a1 = fwd.store = fwd.store2 = fwd.a0;
  fwd.b1 = fwd.b0;
  stat = fwd;
  if (ok && grads)
    ok = encode(f, &grad.b0, c.hp, c.dp, c.rows_cap, c.dp, 64) && encode(f, &grad.b1, w, w_cols, d.vocab, w_stride, 64) &&
         encode(f, &grad.store2, c.dh, c.dcap, uint64_t(c.max_splits) * c.rows_cap, c.dcap, 32, true) &&
         (!c.want_gw || c.direct_store || encode(f, &grad.store, c.grad_weight, d.dim, d.vocab, c.grad_weight_stride, 32, c.grad_f32));
  kept = grad;
  if (ok && keeps) {
    const uint64_t n = up(d.vocab - c.keep_v0, 256) / 32;
    ok = encode_panels(f, &stat.store, c.keep_z, c.rows_cap, n, 32, true) && encode_panels(f, &kept.a0, c.g, c.rows_cap, n, 64) &&
         encode_panels(f, &kept.a1, c.g, c.rows_cap, n, 128);
  }
  if (ok && forms) {
    const uint64_t n = uint64_t(c.planes) * c.piece_cols / 64;
    ok = encode_panels(f, &fwd.store, c.g, c.rows_cap, n, 32) && encode_panels(f, &grad.a0, c.g, c.rows_cap, n, 64) &&
         encode_panels(f, &grad.a1, c.g, c.rows_cap, n, 128);
  }
  if (!ok) return refuse(FLS_ECUDA, "cuTensorMapEncodeTiled failed");

#define FLS_LAUNCH(call)                                        \
  do {                                                          \
    const cudaError_t e_ = (call);                              \
    if (e_ != cudaSuccess) return cuda_fail(e_, "head kernel"); \
    ++h->launches;                                              \
  } while (0)
  if (io->rows > 256) FLS_LAUNCH(launch_head_rows_map(c, s));
  FLS_LAUNCH(launch_head_pack(c, s));
  if (copy)
    FLS_LAUNCH(launch_head_pack_weight(static_cast<const uint16_t*>(io->weight), io->weight_stride ? io->weight_stride : d.dim,
                                       reinterpret_cast<uint16_t*>(ws + r.wcopy), c.vocab, c.dim, c.dp, s));
  FLS_LAUNCH(launch_head_stats(c, stat, s));
  FLS_LAUNCH(launch_head_rows(c, s));
  if (grads) {
    if (keeps) {
      FLS_LAUNCH(launch_head_rescale(c, s));
      FLS_LAUNCH(launch_head_own(c, s));
      FLS_LAUNCH(launch_head_grads(c, kept, HeadPiece{c.keep_v0, c.vocab - c.keep_v0, 1, 2}, s));
    }
    for (uint32_t v0 = 0; v0 < c.keep_v0; v0 += c.piece_cols) {
      const HeadPiece p{v0, std::min(c.piece_cols, c.keep_v0 - v0), !keeps && v0 == 0, c.planes};
      FLS_LAUNCH(launch_head_dlogits(c, fwd, p, s));
      FLS_LAUNCH(launch_head_grads(c, grad, p, s));
    }
    if (c.want_gh) FLS_LAUNCH(launch_head_grad_hidden(c, s));
  }
#undef FLS_LAUNCH
  return FLS_OK;
}

// Everything both losses check; `extra` / n_extra are the distillation's own buffers.
int check_io(const fls_head* h, const fls_head_io* io, bool need_labels, const Span* extra, int n_extra) {
  if (!h || !io) return refuse(FLS_EINVAL, "null argument");
  const fls_head_desc& d = h->desc;
  if (io->reserved) return refuse(FLS_EINVAL, "reserved must be 0");
  if (io->rows > d.max_rows) return refuse(FLS_EINVAL, "rows (%llu) > max_rows (%llu)", (unsigned long long)io->rows, (unsigned long long)d.max_rows);
  if (io->accumulate > 1) return refuse(FLS_EINVAL, "accumulate must be 0 or 1");
  if ((io->grad_hidden || io->grad_weight) && !d.grads) return refuse(FLS_EINVAL, "the head was created without grads");
  const uint64_t strides[4] = {io->hidden_stride, io->weight_stride, io->grad_hidden_stride, io->grad_weight_stride};
  static const char* const names[4] = {"hidden_stride", "weight_stride", "grad_hidden_stride", "grad_weight_stride"};
  for (int i = 0; i < 4; ++i) {
    if (strides[i] && strides[i] < d.dim) return refuse(FLS_EINVAL, "%s (%llu) < dim (%u)", names[i], (unsigned long long)strides[i], d.dim);
    if (strides[i] >= (1ull << 36)) return refuse(FLS_EINVAL, "%s out of range", names[i]);
  }
  auto st = [&](int i) { return strides[i] ? strides[i] : uint64_t(d.dim); };
  if (!(d.any_weight || d.dim % 8) && (reinterpret_cast<uintptr_t>(io->weight) % 16 || st(1) % 8))
    return refuse(FLS_EALIGN, "weight must start on a 16-byte boundary with a stride of a multiple of 8 elements (or create the head with any_weight)");
  const uint64_t we = d.grad_dtype == FLS_GRAD_F32 ? 4 : 2;
  Span s[16] = {
      {io->hidden, span_bytes(io->rows, d.dim, st(0), 2), 2, false, "hidden"},
      {io->weight, span_bytes(d.vocab, d.dim, st(1), 2), 2, false, "weight"},
      {io->labels, need_labels ? io->rows * 8 : 0, 8, false, "labels"},
      {io->row_weight, io->row_weight ? io->rows * 4 : 0, 4, false, "row_weight"},
      {io->loss, io->rows * 4, 4, true, "loss"},
      {io->lse, io->rows * 4, 4, true, "lse"},
      {io->grad_hidden, io->grad_hidden ? span_bytes(io->rows, d.dim, st(2), 2) : 0, 2, true, "grad_hidden"},
      {io->grad_weight, io->grad_weight ? span_bytes(d.vocab, d.dim, st(3), we) : 0, we, true, "grad_weight"},
      {io->workspace, h->reg.total, 256, true, "workspace"},
  };
  int n = 9;
  for (int i = 0; i < n_extra; ++i) s[n++] = extra[i];
  if (io->workspace && io->workspace_bytes < h->reg.total)
    return refuse(FLS_ESIZE, "workspace has %llu bytes, %llu needed", (unsigned long long)io->workspace_bytes, (unsigned long long)h->reg.total);
  return check_spans(s, n);
}

bool weight_ok(double x) { return std::isfinite(x) && x >= 0; }

}  // namespace

extern "C" {

int fls_head_create(const fls_head_desc* desc, fls_head** out) {
  if (out) *out = nullptr;
  if (!desc || !out) return refuse(FLS_EINVAL, "null argument");
  if (desc->reserved) return refuse(FLS_EINVAL, "reserved must be 0");
  if (desc->max_rows > (1ull << 24)) return refuse(FLS_EINVAL, "max_rows > 2^24");
  if (desc->vocab < 1 || desc->vocab > (1ull << 30)) return refuse(FLS_EINVAL, "vocab must be in 1 .. 2^30");
  if (desc->dim < 1 || desc->dim > 65536) return refuse(FLS_EINVAL, "dim must be in 1 .. 65536");
  if (up(desc->max_rows, 256) / 256 * (up(desc->vocab, 256) / 256) > (1ull << 31)) return refuse(FLS_EINVAL, "max_rows * vocab > 2^47");
  if (desc->top > FLS_HEAD_MAX_TOP) return refuse(FLS_EINVAL, "top > %d", FLS_HEAD_MAX_TOP);
  if (desc->grads > 1 || desc->any_weight > 1) return refuse(FLS_EINVAL, "grads and any_weight must be 0 or 1");
  if (desc->grad_dtype != FLS_GRAD_BF16 && desc->grad_dtype != FLS_GRAD_F32) return refuse(FLS_EINVAL, "unknown grad_dtype %u", desc->grad_dtype);
  if (desc->piece_bytes > (1ull << 40)) return refuse(FLS_EINVAL, "piece_bytes > 2^40");
  fls_head* h = new (std::nothrow) fls_head;
  if (!h) return refuse(FLS_ESTATE, "out of host memory");
  h->desc = *desc;
  h->reg = regions(*desc);
  *out = h;
  return FLS_OK;
}

int fls_head_query(const fls_head* head, fls_head_layout* out) {
  if (!head || !out) return refuse(FLS_EINVAL, "null argument");
  const fls_head_desc& d = head->desc;
  out->workspace_bytes = head->reg.total;
  out->piece_cols = out->pieces = out->kept_cols = 0;
  if (d.grads) {
    const Pieces p = pieces_of(d, head->reg.g_bytes, d.max_rows, terms_of(d));
    out->piece_cols = p.cols;
    out->pieces = p.cols ? (p.keep_v0 + p.cols - 1) / p.cols : 0;
    out->kept_cols = d.vocab - p.keep_v0;
  }
  return FLS_OK;
}

int fls_head_destroy(fls_head* head) {
  delete head;
  return FLS_OK;
}

int fls_head_xent(fls_head* head, const fls_head_io* io, double label_smoothing, double z_loss, void* cuda_stream) {
  if (!(label_smoothing >= 0.0 && label_smoothing < 1.0)) return refuse(FLS_EINVAL, "label_smoothing must be in [0, 1)");
  if (!weight_ok(z_loss)) return refuse(FLS_EINVAL, "z_loss must be finite and >= 0");
  int rc = check_io(head, io, true, nullptr, 0);
  if (rc) return rc;
  HeadCall c{};
  c.use_label = 1;
  c.smooth = label_smoothing > 0.0;
  c.smoothing = label_smoothing;
  c.z_loss = z_loss;
  c.temp = c.inv_temp = 1.0;
  return run(head, io, c, cuda_stream);
}

int fls_head_distill(fls_head* head, const fls_head_io* io, const fls_distill_desc* t, void* cuda_stream) {
  if (!head || !io || !t) return refuse(FLS_EINVAL, "null argument");
  if (t->reserved) return refuse(FLS_EINVAL, "reserved must be 0");
  if (head->desc.top == 0) return refuse(FLS_EINVAL, "the head was created with top = 0");
  if (t->tail != FLS_TAIL_RENORM && t->tail != FLS_TAIL_CLASS) return refuse(FLS_EINVAL, "unknown tail %u", t->tail);
  if (!(std::isfinite(t->temperature) && t->temperature > 0.0)) return refuse(FLS_EINVAL, "temperature must be finite and > 0");
  if (!weight_ok(t->distill_weight) || !weight_ok(t->label_weight)) return refuse(FLS_EINVAL, "distill_weight and label_weight must be finite and >= 0");
  const bool labels = t->label_weight > 0.0;
  const uint64_t n = io->rows, k = head->desc.top;
  const Span extra[3] = {{t->top_index, n * k * 4, 4, false, "top_index"},
                         {t->top_logit, n * k * 4, 4, false, "top_logit"},
                         {t->teacher_lse, t->tail == FLS_TAIL_CLASS ? n * 4 : 0, 4, false, "teacher_lse"}};
  int rc = check_io(head, io, labels, extra, 3);
  if (rc) return rc;
  HeadCall c{};
  c.top = head->desc.top;
  c.top_index = t->top_index;
  c.top_logit = t->top_logit;
  c.teacher_lse = t->teacher_lse;
  c.tail_class = t->tail == FLS_TAIL_CLASS;
  c.use_label = labels;
  c.temp = t->temperature;
  c.inv_temp = 1.0 / t->temperature;
  c.two = labels && t->temperature != 1.0;
  c.distill_weight = t->distill_weight;
  c.label_weight = t->label_weight;
  return run(head, io, c, cuda_stream);
}

int fls_head_get_state(const void* workspace, const uint32_t** dev_status, const uint32_t** dev_count) {
  if (!workspace) return refuse(FLS_EPTR, "workspace is null");
  const HeadState* s = static_cast<const HeadState*>(workspace);
  if (dev_status) *dev_status = &s->status;
  if (dev_count) *dev_count = &s->count;
  return FLS_OK;
}

int fls_debug_expire_next_head_wait(fls_head* head, uint32_t polls) {
  if (!head || !polls) return refuse(FLS_EINVAL, "null argument");
  head->expire_polls = polls;
  return FLS_OK;
}

int fls_head_get_launch_count(const fls_head* head, uint64_t* launches) {
  if (!head || !launches) return refuse(FLS_EINVAL, "null argument");
  *launches = head->launches;
  return FLS_OK;
}

}  // extern "C"
