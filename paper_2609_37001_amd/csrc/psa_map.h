// Internal interface between the C ABI and the kernels of the block selection (psa_select.hip) and of the attention over
// a block map (psa_map.hip).  For hipcc only (bf16 pointers).
#pragma once

#include "psa_launch.h"
#include "psa_pieces.h"

namespace psa {

// Block selection.  Key blocks below first_k and query blocks below first_q hold no text.
struct SelectArgs {
  const __bf16 *q, *k;                // [n_bh][n_q][d]; keys by strides, rows contiguous
  int64_t kv_stride_b, kv_stride_h;
  double *mean_q, *mean_k;            // [n_bh][nbq][d], [batch * n_kv_heads][nbk][d]
  uint64_t* scores;                   // slabs of psa_select_kernel's workgroups
  uint8_t* map;                       // [n_bh][nbq][nbk]
  int32_t* kept_per_row;              // [n_bh][nbq] or null
  int32_t n_bh, n_heads, n_kv_heads, group, n_q, n_k, nbq, nbk, block, keep, first_q, first_k;
  int32_t q_blocks_all, slab;         // set by the launcher
};
struct SelectLayout {
  size_t mean_q, mean_k, scores, total;
};
// Whether the launches hold the blocks of both sides.
bool select_fits(int32_t n_bh, int32_t n_kv, int32_t nbq, int32_t nbk);
SelectLayout select_layout(int32_t n_bh, int32_t n_kv, int32_t head_dim, int32_t nbq, int32_t nbk);
hipError_t launch_select(const SelectArgs& args, int32_t head_dim, hipStream_t stream);

// Attention over a block map.
struct MapArgs {
  const __bf16 *q, *k, *v;            // q [n_bh][n_q][d]; k and v by strides, rows contiguous
  const __bf16* grad_o;               // backward
  __bf16* o;                          // [n_bh][n_q][d] (backward: an input)
  __bf16 *dq, *dk, *dv;               // backward; dk and dv [batch * kv heads][n_k][d]
  float* lse;                         // [n_bh][n_q] or null (backward: an input)
  const uint8_t* map;                 // [n_heads][nbq][nbk] per batch element
  int64_t map_stride_b, kv_stride_b, kv_stride_h;
  float* part_o;                      // forward: sums of a part of a list, [tile][block][d], and (m, l) of its rows
  float2* part_ml;
  float *neg_lse2, *neg_delta;        // backward: [n_bh][nbq][block]
  int32_t* row_counts;                // list lengths of the (head, query block) items (null: not ordered)
  int32_t *pair_counts, *pair_order;  // forward, block 64: those of pairs of query blocks, and
  int32_t* paired;                    // whether pairs run (null: they do not)
  int32_t* col_counts;                // backward: those of the (key head, key block) items
  Pieces row_pieces, col_pieces;
  int32_t n_bh, n_heads, group;       // group: query heads per key head
  float *part_q, *part_k, *part_v;    // backward: sums of a part of a list, [tile][block][d]
  int32_t n_q, n_k, nbq, nbk, block, parts;
  int32_t head_parts, list_parts;     // backward: parts of a key block's query heads, and of each one's list
  float c, scale;                     // scale log2(e), scale
  float pow2, factor;                 // forward: c = pow2 factor, a power of two with c's sign and a factor in [1, 2)
};
hipError_t launch_map_fwd(const MapArgs& a, int32_t head_dim, hipStream_t stream);
hipError_t launch_map_bwd(const MapArgs& a, int32_t head_dim, hipStream_t stream);

}  // namespace psa
