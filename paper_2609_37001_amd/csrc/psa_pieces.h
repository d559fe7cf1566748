// How the attention over a block map shares its lists out over the workgroups: the sizes that the host reserves for it,
// and the cut that the ordering kernel makes of the lists it finds.  No bf16 here, so that any host compiler takes it.
#pragma once

#include <math.h>

#include "psa_launch.h"

namespace psa {

// Order of a kernel's items (psa_map.hip, order_pieces): `grid` workgroups (0: there is none), of which at most
// `pieces` (0: the lists stay whole) take a piece of a list, of at most `splits` items.
struct Pieces {
  int2* order;
  int4* split;
  int32_t grid, pieces, splits;
};

// The lists' lengths differ: a row of text lists every key block, a key block that every row keeps (text, the first block
// of a sequence) lists the rows of every query head, and such a list can outlast all the others together.  So long
// ones go in pieces, each to a workgroup of its own that leaves its sums in the workspace, where another kernel adds them.
// With `room` workgroups sharing the work (`share` blocks each):
//   * more items than room: lists longer than 1.25 share, in pieces of half a share, 8 blocks at least (shorter ones,
//     started first, end with the others).  At most 0.8 room lists and 2.8 room pieces, whatever the map.
//   * fewer: a list of average length goes in room / items pieces and a longer one in pieces as long, 4 blocks at
//     least.  At most 4/3 room pieces.
// The kernels clamp nothing: that no map gives more pieces or cut lists than pieces_for reserves, that pieces come first
// in the order (a piece's tile of the workspace is its workgroup's number), and that a cut list has two pieces at least
// (its sums are read from there) is what keeps every access inside the workspace.  tests/test_pieces.py holds these rules.
// Whole gradients without and with pieces, in us.  Every row keeps the first block and others by chance: 12 heads x
// 32760 (D 128, blocks of 128, 8 kept) 1247 and 1031; 16 heads over 4 3815 and 1298; 12 x 16384 (D 64, blocks of 64, 12
// kept) 342 and 249; 32 over 8 x 16384 (D 128, blocks of 64, 16 kept) 2060 and 1280.  Rows of text (226 tokens): 8
// heads x 4096 (D 128, blocks of 64, 8 kept) 181 and 124.  Maps without any of these pay 0 to 2 %.
constexpr int kPieceBlocks = 8, kFewBlocks = 4;
struct Cut {
  float mean, piece, longest, up;
  __host__ __device__ inline Cut(unsigned long long work, int32_t items, int32_t room, const Pieces& to) {
    const float share = (float)work / (float)room;
    mean = (float)work / (float)items;
    const bool few = items <= room;
    piece = few ? fmaxf((float)kFewBlocks, mean / (float)(room / items)) : fmaxf((float)kPieceBlocks, 0.5f * share);
    longest = to.pieces == 0 ? __builtin_inff() : few ? 1.5f * piece : fmaxf(1.5f * kPieceBlocks, 1.25f * share);
    up = few ? 0.5f : 1.0f;
  }
  __host__ __device__ inline bool cuts(int32_t c) const { return (float)c > longest; }
  __host__ __device__ inline int32_t pieces(int32_t c) const { return (int32_t)((float)c / piece + up); }   // of such a list
};

// Workgroups that share a call's work: one of 128 rows to a CU, two of 64.
inline int32_t room_of(int32_t block) { return 256 * (128 / block); }
// Forward items up to which a call is not ordered: as many as run at once, at head dim 64 twice as many (two rounds: the
// kernel there is held to two waves per SIMD, though its registers and LDS would allow four).  Ordered and not at head
// dim 64, 8 heads x 5000 take 36 and 24 us at block 64, 44 and 36 at block 128; 8 x 8000 at block 64 67 and 52.
inline int32_t unordered(int32_t head_dim, int32_t block) { return room_of(block) * (128 / head_dim); }

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// Parts of every query block's list: as many as give every CU its workgroups where there are fewer query blocks
// (two of 64 rows to a CU, one of 128), each part at least six blocks of a full row: the parts' sums cost a kernel more, 4 us,
// and a block 0.5 to 1.3 us.
inline int32_t map_parts(int32_t n_bh, int32_t nbq, int32_t nbk, int32_t block) {
  const int64_t items = (int64_t)n_bh * nbq, room = room_of(block);
  return (int32_t)std::max<int64_t>(1, std::min<int64_t>(room / items, nbk / 6));
}

// The order of a kernel's `items`, whose lists hold at most `longest` blocks and would else go in `parts` each.  No more than
// `unordered` items are ordered too if a part may hold more than a kernel's `long_part` tokens: the
// order costs 10 to 20 us of a balanced call, a block of 128 takes 2.4 us in the gradients' kernels and 1 us in the
// forward's, one of 64 half as much.  (Gradients, D 128, blocks of 64, equal parts and the order, in us: 4 heads over 2 x
// 7791 with 226 of text, 31 kept, 337 and 228; without text 4 over 2 x 5760, 43 kept, 171 and 187; 3 heads x 2430 in a
// batch of 4, whose lists stay below, 130 and 160.  Forward: 4 x 8192 with text, 16 kept, 119 and 66; 2 x 16384
// without, 40 kept, 63 and 67.)
inline Pieces pieces_for(int64_t items, int32_t unordered, int64_t longest, int32_t parts, int32_t long_part, int32_t block) {
  Pieces p = {};
  const int64_t room = room_of(block);
  if (items <= unordered && longest / parts * block <= long_part) return p;
  p.pieces = (int32_t)std::min(3 * room, items * ((longest + kFewBlocks - 1) / kFewBlocks));
  p.splits = (int32_t)std::min(room, items);
  p.grid = (int32_t)(items + p.pieces);
  return p;
}

constexpr int32_t kLongForward = 8000, kLongBackward = 3000;
// No forward list shorter than this goes in pieces: they cost a launch more, 5 us (without and with them, 226 of text,
// blocks of 64: 20 heads x 2400 in a batch of 2 86 and 90 us; 8 x 4096 65 and 63; 4 x 8192 119 and 66; 3 x 16384 235
// and 105.  Nothing between 4096 and 8192 was measured.)
constexpr int32_t kShortForward = 6000;

struct MapLayout {
  Pieces rows;                        // sizes alone
  int32_t parts;
  size_t row_counts, row_order, row_split, pair_counts, pair_order, paired, part_o, part_ml, total;
};
inline MapLayout map_layout(int32_t n_bh, int32_t head_dim, int32_t nbq, int32_t nbk, int32_t block) {
  MapLayout l = {};
  l.parts = map_parts(n_bh, nbq, nbk, block);
  // (single query blocks, no more than `slots`: a few tokens behind a cache, lists as long as each other)
  const int64_t items = (int64_t)n_bh * nbq;
  const int32_t slots = unordered(head_dim, block);
  if (nbq > 1 || items > slots) l.rows = pieces_for(items, slots, nbk, l.parts, kLongForward, block);
  auto take = [&](size_t& at, size_t bytes) {
    at = l.total;
    l.total += up256(bytes);
  };
  if (l.rows.grid) {
    l.parts = 1;
    if ((int64_t)nbk * block < kShortForward) l.rows.pieces = l.rows.splits = 0, l.rows.grid = (int32_t)items;
    take(l.row_counts, (size_t)n_bh * nbq * sizeof(int32_t));
    take(l.row_order, l.rows.grid * sizeof(int2));
    take(l.row_split, (1 + (size_t)l.rows.splits) * sizeof(int4));
    if (block == 64 && items > slots) {
      take(l.pair_counts, (size_t)n_bh * pairs_per_head(nbq) * sizeof(int32_t));
      take(l.pair_order, (size_t)n_bh * pairs_per_head(nbq) * sizeof(int32_t));
      take(l.paired, sizeof(int32_t));
    }
  }
  const size_t tiles = l.rows.grid ? l.rows.pieces : l.parts > 1 ? (size_t)n_bh * nbq * l.parts : 0;
  take(l.part_o, tiles * block * head_dim * sizeof(float));
  take(l.part_ml, tiles * block * sizeof(float2));
  return l;
}

// Whether the launches of a forward hold its workgroups (those for pairs and for the list lengths are fewer).
inline bool map_fits(const MapLayout& l, int32_t n_bh, int32_t nbq, int32_t block) {
  const int64_t items = (int64_t)n_bh * nbq;
  return launch_fits(l.rows.grid ? items + l.rows.pieces : items * l.parts, 4 * block);
}

struct MapBwdLayout {
  Pieces rows, cols;                  // sizes alone
  int32_t parts, head_parts, list_parts;
  size_t neg_lse2, neg_delta, row_counts, row_order, row_split, col_counts, col_order, col_split, part_q, part_k, part_v, total;
};
inline MapBwdLayout map_bwd_layout(int32_t n_bh, int32_t n_kv, int32_t head_dim, int32_t nbq, int32_t nbk, int32_t block) {
  MapBwdLayout l = {};
  // dq's lists go in parts as the forward's do, dk's and dv's by the query heads of a key head first; or in pieces.
  const int32_t group = n_bh / n_kv, room = std::max(1, (int32_t)(room_of(block) / ((int64_t)n_kv * nbk)));
  l.parts = map_parts(n_bh, nbq, nbk, block);
  l.head_parts = std::min(group, room);
  l.list_parts = std::max(1, std::min(room / l.head_parts, nbq / 6));
  const int32_t kv_parts = l.head_parts * l.list_parts;
  l.rows = pieces_for((int64_t)n_bh * nbq, room_of(block), nbk, l.parts, kLongBackward, block);
  l.cols = pieces_for((int64_t)n_kv * nbk, room_of(block), (int64_t)group * nbq, kv_parts, kLongBackward, block);
  const size_t tile = (size_t)block * head_dim * sizeof(float);
  auto take = [&](size_t& at, size_t bytes) {
    at = l.total;
    l.total += up256(bytes);
  };
  take(l.neg_lse2, (size_t)n_bh * nbq * block * sizeof(float));
  take(l.neg_delta, (size_t)n_bh * nbq * block * sizeof(float));
  if (l.rows.grid) {
    take(l.row_counts, (size_t)n_bh * nbq * sizeof(int32_t));
    take(l.row_order, l.rows.grid * sizeof(int2));
    take(l.row_split, (1 + (size_t)l.rows.splits) * sizeof(int4));
  }
  if (l.cols.grid) {
    take(l.col_counts, (size_t)n_kv * nbk * sizeof(int32_t));
    take(l.col_order, l.cols.grid * sizeof(int2));
    take(l.col_split, (1 + (size_t)l.cols.splits) * sizeof(int4));
  }
  const size_t tiles_q = l.rows.grid ? l.rows.pieces : l.parts > 1 ? (size_t)n_bh * nbq * l.parts : 0;
  const size_t tiles_kv = l.cols.grid ? l.cols.pieces : kv_parts > 1 ? (size_t)n_kv * nbk * kv_parts : 0;
  take(l.part_q, tile * tiles_q);
  take(l.part_k, tile * tiles_kv);
  take(l.part_v, tile * tiles_kv);
  return l;
}

// Workgroups of a backward call that form its row values, and that count the lists of rows and of columns.
inline int64_t value_groups(int32_t n_bh, int32_t head_dim, int32_t nbq, int32_t block) {
  return ((int64_t)n_bh * nbq * block * (head_dim / 8) + 255) / 256;
}
inline int64_t row_groups(int32_t n_bh, int32_t nbq) { return ((int64_t)n_bh * pairs_per_head(nbq) + 3) / 4; }
inline int64_t col_groups(int32_t n_kv, int32_t nbk) { return (int64_t)(nbk + 63) / 64 * n_kv; }

inline bool map_bwd_fits(const MapBwdLayout& l, int32_t n_bh, int32_t n_kv, int32_t head_dim, int32_t nbq, int32_t nbk, int32_t block) {
  const int64_t rows = (int64_t)n_bh * nbq, cols = (int64_t)n_kv * nbk;
  const int64_t prepare = value_groups(n_bh, head_dim, nbq, block) + (l.rows.grid ? row_groups(n_bh, nbq) : 0) +
                          (l.cols.grid ? col_groups(n_kv, nbk) : 0);
  return launch_fits(l.rows.grid ? rows + l.rows.pieces : rows * l.parts, 4 * block) &&
         launch_fits(l.cols.grid ? cols + l.cols.pieces : cols * l.head_parts * l.list_parts, 4 * block) && launch_fits(prepare, 256);
}

}  // namespace psa
