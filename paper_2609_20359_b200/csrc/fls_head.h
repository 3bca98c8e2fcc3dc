// Internal declarations of the language-model head operators (cross entropy and distillation of a linear head
// without kept logits): what the host code and the kernels share.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "fls.h"

namespace fls {

constexpr int kHeadBM = 256;      // rows of C per CTA pair (128 per CTA)
constexpr int kHeadBN = 256;      // columns of C per CTA pair; both CTAs hold all of them for their own rows
constexpr int kHeadBK = 64;       // depth of one pipeline stage: 64 bf16 = one 128-byte swizzle row
constexpr int kHeadStatCols = 128; // columns per partial sum of a row
constexpr int kHeadMaxSplits = 64;

// Head of the workspace: words the device writes.
struct HeadState {
  uint32_t status;   // FLS_STATUS_* bits, sticky
  uint32_t count;    // rows of the last call that take part (label or teacher entry present)
  uint32_t splits;   // parts of the hidden gradient's depth, 1 .. kHeadMaxSplits
};

// Everything the kernels of one call share.  Packed row p stands for row src[p] of the caller.
struct HeadCall {
  HeadState* state;
  uint32_t* row_mask;        // [rows / 32]: a bit per row that takes part
  uint32_t* row_count;       // [rows / 256]: rows that take part among 256
  int32_t* pos;              // [rows]: packed row of a row, -1 if it takes no part
  int32_t* src;              // [rows_cap]: row of a packed row
  uint16_t* hp;              // [rows_cap][dp]: packed hidden rows, zero up to the next multiple of 256 rows
  int32_t* slot_idx;         // [rows_cap][slots]: columns that get a value of their own, ascending, INT32_MAX = none
  uint8_t* slot_start;       // [rows_cap][tiles]: the first of them in each 128 columns (only with a teacher's list)
  float* slot_t;             // [rows_cap][slots]: the teacher's logit of that column (-inf: label only)
  float* slot_z;             // [rows_cap][slots]: the logit of that column
  float* label_z;            // [rows_cap]: the label's logit, summed in double
  float* slot_g;             // [rows_cap][slots]: its gradient
  float* part_m;             // [tiles][rows_cap]: largest logit of 128 columns, slots left out
  float* part_s;             // [tiles][rows_cap]: sum of exp((z - m) / T)
  float* part_s1;            // same at temperature 1 (only when T != 1 and labels count)
  float* part_z;             // sum of the logits (only with label smoothing)
  float4* coef;              // [rows_cap]: see fls_head_rows_kernel
  uint16_t* g;               // d loss / d logits of one piece of the vocabulary, in panels of 64 columns (dz_panel)
  float* keep_z;             // [panels of 32 columns][rows_cap][32]: kept logits, in the bytes of g
  float* dh;                 // [splits][rows_cap][dcap]: partial sums of the hidden gradient
  // problem
  const uint16_t* hidden; uint64_t hidden_stride;
  const uint16_t* weight; uint64_t weight_stride;
  const int64_t* labels; int64_t ignore_label;
  const int32_t* top_index; const float* top_logit; const float* teacher_lse;
  const float* row_weight;
  float* loss; float* lse;
  uint16_t* grad_hidden; uint64_t grad_hidden_stride;
  void* grad_weight; uint64_t grad_weight_stride;
  uint64_t rows; uint32_t rows_cap;
  uint32_t vocab, dim, dp, dcap;
  uint32_t top, slots, tiles;
  uint32_t piece_cols;
  uint32_t terms, planes;    // bf16 terms of dL/dz that a weight gradient of this head takes; those that this call stores
  uint32_t tail_class, use_label, two, smooth, grad_f32, accumulate;
  uint32_t want_gh, want_gw;
  uint32_t direct_store;     // grad_weight cannot be a TMA store's target (alignment, length of a row, bf16 accumulation): plain stores
  uint32_t max_splits, clusters, group_m;
  uint32_t prefetch_weight;  // one row tile, and the weight is the caller's: fetched ahead of the packed rows
  uint32_t wait_limit;       // polls of a barrier before a role gives up
  uint32_t hold_back;        // tests only: the operands' arrival is never announced
  uint32_t keep_v0;          // columns from here on keep their logits, vocab: none
  uint32_t split_cols;       // columns of the widest piece, 0 without gradients
  float c1, cT;              // log2(e), log2(e) / T
  double inv_temp, temp, smoothing, z_loss, distill_weight, label_weight;
};

// Operands of the products (kGrads: 0 for the weight's, 1 for the hidden gradient) and where tiles are stored: dL/dz, or
// grad_weight (store) and the partial sums of grad_hidden (store2).
struct HeadMaps { CUtensorMap a0, b0, a1, b1, store, store2; };

// One launch of the tensor-core kernel.
struct HeadPiece {
  uint32_t v0, width;        // the columns of the vocabulary it works on
  uint32_t first;            // first piece: the hidden gradient's partial sums are stored, later ones added to
  uint32_t panel_step;       // panels from one 64 columns of dL/dz to the next
};

cudaError_t launch_head_rows_map(const HeadCall& c, cudaStream_t s);
cudaError_t launch_head_pack(const HeadCall& c, cudaStream_t s);
cudaError_t launch_head_pack_weight(const uint16_t* w, uint64_t stride, uint16_t* out, uint32_t vocab, uint32_t dim, uint32_t dp, cudaStream_t s);
cudaError_t launch_head_stats(const HeadCall& c, const HeadMaps& m, cudaStream_t s);
cudaError_t launch_head_rows(const HeadCall& c, cudaStream_t s);
cudaError_t launch_head_dlogits(const HeadCall& c, const HeadMaps& m, const HeadPiece& p, cudaStream_t s);
cudaError_t launch_head_rescale(const HeadCall& c, cudaStream_t s);
cudaError_t launch_head_own(const HeadCall& c, cudaStream_t s);
cudaError_t launch_head_grads(const HeadCall& c, const HeadMaps& m, const HeadPiece& p, cudaStream_t s);
cudaError_t launch_head_grad_hidden(const HeadCall& c, cudaStream_t s);
// Readies the kernels on the current device; clusters of two CTAs that fit on it at once.
cudaError_t head_clusters(uint32_t* out);

}  // namespace fls
