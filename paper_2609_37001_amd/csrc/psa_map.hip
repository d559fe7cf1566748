// Attention over the kept blocks of any block map, forward and backward: HIP kernels for gfx950.
//
//   forward   S = scale q k^T over kept blocks, o = softmax(S) v, lse = log sum exp S
//   backward  P = exp(S - lse), dP = do v^T, delta = rowsum(do * o), dS = P (dP - delta)
//             dq = scale dS k,   dk = scale dS^T q,   dv = P^T do
//
// Scores are exact up to their fp32 sums, in both directions: the forward scales q by a power of two alone (no
// rounding) and multiplies every score by the rest of scale log2(e), a factor in [1, 2), before its exponential; the
// backward multiplies by the whole.  Rounding scale log2(e) q to bf16 instead would save that multiplication (3 to 6 %
// of the forward's time, 2 % of the backward's: 5 heads x 75600, 141 blocks of 128 kept, 3335 us without and 3445 with;
// gradients of 12 x 32760, 64 kept, 5210 and 5290) and move scores by up to 2^-8 of the magnitudes they add: outputs
// then are 2.9e-3 off instead of 2.35e-3, and a normaliser of rows whose scores share a large part by tenths.
//
// Rounded to bf16, as in the library's other attention kernels: the weights P and, in the backward, dS, which the matrix
// cores take as operands of the second products.  It is half a step, 2^-8 of a weight at most, and moves outputs by 1.6e-3; with
// the rounding of the output, 1.65e-3, the forward is 2.3e-3 off where weights in 32 bits would leave 1.65e-3.  The
// normaliser sums the rounded weights, so that a row's weights still add up to one.  Without it every weight
// would be two bf16 halves and P V two products for one, three in the forward for two.  Scores, statistics
// and all sums are in 32 bits.
//
// One workgroup takes one block of one side -- queries in the forward and for dq, keys for dk and dv -- holds its
// rows in registers, and streams the blocks that the map keeps of the other side through LDS, double-buffered,
// with the tile engine of psa_tile.h.  Its two groups of waves hold the same rows and take half of every streamed
// block each; their sums are added through LDS at the end.  So a block's work is spread over twice the waves, and
// no two blocks have to agree on what they keep.
//   * psa_mapped_fwd_kernel   S^T = K Q^T, O^T += V^T P^T
//   * psa_mapped_dq_kernel    S^T = K Q^T, dP^T = V dO^T, dQ^T += K^T dS^T
//   * psa_mapped_dkv_kernel   the same with the sides exchanged: S = Q K^T, dP = dO V^T, dV^T += dO^T P,
//                             dK^T += Q^T dS; key heads shared by several query heads stream all of them
// Every sum has one order, fixed by the call's sizes and its map; there are no atomics on results.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "psa_launch.h"
#include "psa_map.h"
#include "psa_tile.h"

namespace psa {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994530942f;

// The kept entries of `len` places, ascending, by all waves of the workgroup: entry(i) is what to list for place i, -1
// for nothing.  Each wave counts a run of the places and, once all counts are known, goes over it again: two
// barriers for any length.  Ends with a barrier.
template <int W, typename F>
__device__ __forceinline__ int32_t kept_list(int32_t len, uint16_t* list, int32_t* found, F entry) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int32_t run = (len + W * 64 - 1) / (W * 64) * 64, i0 = wave * run, i1 = min(len, i0 + run);
  int32_t mine = 0;
  for (int32_t i = i0; i < i1; i += 64)
    mine += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i + lane < i1 && entry(i + lane) >= 0));
  if (lane == 0) found[wave] = mine;
  __syncthreads();
  int32_t pos = 0, nu = 0;
#pragma unroll
  for (int w = 0; w < W; w++) {
    pos += w < wave ? found[w] : 0;
    nu += found[w];
  }
  for (int32_t i = i0; i < i1; i += 64) {
    const int32_t e = i + lane < i1 ? entry(i + lane) : -1;
    const uint64_t mask = __builtin_amdgcn_ballot_w64(e >= 0);
    if (e >= 0) list[pos + __builtin_popcountll(mask & ((1ull << lane) - 1))] = (uint16_t)e;
    pos += __builtin_popcountll(mask);
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(nu);
}

// Position j of a run of `len` items -> its place among workgroups that start in turn: consecutive workgroups go to the
// XCDs in turn, so XCD x gets the x-th contiguous part of the run, whose blocks stream much the same other side
// through its L2.  (The last len % 8 items follow one by one.)
__device__ __forceinline__ int32_t spread(int32_t j, int32_t len) {
  const int32_t part = len / kNumQueues;
  if (j >= part * kNumQueues) return j;
  const int32_t x = j / part;
  return (j - x * part) * kNumQueues + x;
}

// The reverse: the item that workgroup `blk` of `items` takes.
__device__ __forceinline__ int32_t item_of(int32_t blk, int32_t items) {
  const int32_t part = items / kNumQueues;
  return blk >= part * kNumQueues ? blk : blk % kNumQueues * part + blk / kNumQueues;
}

// Whether maps of 64 run on pairs of query blocks, where these outnumber the workgroups: `either` counts the key blocks
// that one block of a pair or both keep, `single` those that each keeps, over all pairs.  A wave waits while its
// neighbour's block alone is worked on, so at head dim 128 pairs pay where neighbours share enough; at head dim 64 its
// four waves per SIMD cover such waits.  Microseconds in pairs and one by one at either / single 0.87, 0.70 and 0.50:
// (one by one at head dim 64 on two waves per SIMD, what its attribute allows)
//   head dim 64   12 heads x 32760, density 0.25 (256 pairs each)  1104, 1009, 895 and 1281, 1284, 1288
//                 16 x 8000, 0.2 (63 pairs each)                   107, 94, 85     and 118, 118, 116
//                 9 x 8000, 0.2                                    90, 81, 67      and 91, 88, 87
//   head dim 128  12 x 32760, 0.25                                 2129, 1923, 1645 and 2046, 2006, 1962
//                 8 x 8000, 0.2                                    110, 96, 83     and 97, 95, 91
__device__ __forceinline__ bool pairs_pay(unsigned long long either, unsigned long long single, int32_t head_dim) {
  return head_dim == 64 || either * 10 <= single * 7;
}

// ---------------------------------------------------------------------------------------------
// Order of the items: those with long lists first.  Where the items outnumber the workgroups that run at once, a
// long one that starts late is waited for alone (a row of text, a key block that everybody keeps).  Items whose
// lists are about as long stay in their order, for the XCDs' sake.
// ---------------------------------------------------------------------------------------------

// The two query blocks of pair p of a map's head: 2 p and 2 p + 1 (-1 behind an odd number of them).
__device__ __forceinline__ int2 pair_of(int32_t p, int32_t nbq) { return make_int2(2 * p, 2 * p + 1 < nbq ? 2 * p + 1 : -1); }

// Kept key blocks of every (head, query block), and, if asked, those that either block of a pair keeps; a wave per pair.
__device__ __forceinline__ void count_rows(const MapArgs& a, int32_t group) {
  const int32_t item = group * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63, np = pairs_per_head(a.nbq);
  if (item >= a.n_bh * np) return;
  const int32_t bh = item / np, b = bh / a.n_heads, hd = bh - b * a.n_heads;
  const int2 pr = pair_of(item - bh * np, a.nbq);
  const uint8_t* first = a.map + b * a.map_stride_b + ((int64_t)hd * a.nbq + pr.x) * a.nbk;
  const uint8_t* second = pr.y < 0 ? first : first + a.nbk;
  int32_t c0 = 0, c1 = 0, both = 0;
#pragma unroll 4
  for (int32_t j = lane; j < a.nbk; j += 64) {
    const bool x = first[j] != 0, y = second[j] != 0;
    c0 += x;
    c1 += y;
    both += x || y;
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    c0 += __shfl_xor(c0, off);
    c1 += __shfl_xor(c1, off);
    both += __shfl_xor(both, off);
  }
  if (lane == 0) {
    a.row_counts[bh * a.nbq + pr.x] = c0;
    if (pr.y >= 0) a.row_counts[bh * a.nbq + pr.y] = c1;
    if (a.pair_counts) a.pair_counts[item] = both;
  }
}

// Kept (query head, query block) pairs of every (key head, key block); 64 key blocks per workgroup.
__device__ __forceinline__ void count_cols(const MapArgs& a, int32_t group) {
  __shared__ int32_t part[4][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int32_t n_kv = a.n_heads / a.group, per = (a.nbk + 63) / 64, bk = group / per, b = bk / n_kv, hk = bk - b * n_kv;
  const int32_t kb = (group - bk * per) * 64 + lane;
  // the rows of a key head's query heads lie one behind the other
  const uint8_t* col = a.map + b * a.map_stride_b + (int64_t)hk * a.group * a.nbq * a.nbk + min(kb, a.nbk - 1);
  int32_t c = 0;
#pragma unroll 8
  for (int32_t i = wave; i < a.group * a.nbq; i += 4) c += col[(int64_t)i * a.nbk] != 0;
  part[wave][lane] = c;
  __syncthreads();
  if (wave == 0 && kb < a.nbk) a.col_counts[bk * a.nbk + kb] = part[0][lane] + part[1][lane] + part[2][lane] + part[3][lane];
}

// Per query row, in blocks of `block` rows: -lse log2(e), and -delta, where the sums of dP start.  Rows behind the last
// one, and rows that keep nothing (lse = -inf), get -inf: every weight formed with it is 0.  D / 8 lanes a row.
template <int D>
__device__ __forceinline__ void form_row_values(const MapArgs& a, int32_t group) {
  constexpr int L = D / 8;
  const int64_t r = (int64_t)group * (256 / L) + threadIdx.x / L;
  const int32_t padded = a.nbq * a.block;
  if (r >= (int64_t)a.n_bh * padded) return;
  const int c = threadIdx.x % L;
  const int32_t bh = (int32_t)(r / padded), row = (int32_t)(r - (int64_t)bh * padded);
  const int64_t at = (int64_t)bh * a.n_q + min(row, a.n_q - 1);
  const f32x8 x = __builtin_convertvector(*(const bf16x8*)(a.grad_o + at * D + 8 * c), f32x8);
  const f32x8 y = __builtin_convertvector(*(const bf16x8*)(a.o + at * D + 8 * c), f32x8);
  float s = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; e++) s = fmaf(x[e], y[e], s);
#pragma unroll
  for (int off = L / 2; off > 0; off >>= 1) s += __shfl_xor(s, off);
  if (c == 0) {
    const float lse = a.lse[at];
    const bool none = row >= a.n_q || lse == -__builtin_inff();
    a.neg_lse2[r] = none ? -__builtin_inff() : -lse * kLog2e;
    a.neg_delta[r] = none ? 0.0f : -s;
  }
}

// What the main kernels need first, in one launch: the row values of a backward call and the list lengths.  (Three
// launches took 8 us more.)
template <int D>
__global__ __launch_bounds__(256) void psa_mapped_prepare_kernel(MapArgs a, int32_t value_groups, int32_t row_groups) {
  int32_t group = blockIdx.x;
  if (group < value_groups) {
    form_row_values<D>(a, group);
  } else if ((group -= value_groups) < row_groups) {
    count_rows(a, group);
  } else {
    count_cols(a, group - row_groups);
  }
}

constexpr int kOrderThreads = 1024, kOrderWaves = kOrderThreads / 64, kOrderClasses = 8, kOrderRun = 8;

struct OrderSpace {
  int32_t at[kOrderClasses * kOrderThreads * 33 / 32], waves[kOrderWaves];
  unsigned long long totals[kOrderWaves];
};

// One workgroup of kOrderThreads over a list of items; each thread takes a run of them, whose first kOrderRun counts it keeps
// (read again by every pass, their latencies were most of the kernel).
struct Items {
  const int32_t* counts;
  int32_t n, i0, i1, kept[kOrderRun];
  __device__ __forceinline__ Items(const int32_t* counts_, int32_t n_) : counts(counts_), n(n_) {
    const int32_t each = (n + kOrderThreads - 1) / kOrderThreads;
    i0 = min(n, (int32_t)threadIdx.x * each);
    i1 = min(n, i0 + each);
    read(kept, i0);
  }
  __device__ __forceinline__ void read(int32_t (&c)[kOrderRun], int32_t i) const {
#pragma unroll
    for (int u = 0; u < kOrderRun; u++) c[u] = counts[min(i + u, n - 1)];
  }
  // f(item, its count) over this thread's items.
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    int32_t c[kOrderRun];
#pragma unroll
    for (int u = 0; u < kOrderRun; u++) c[u] = kept[u];
    for (int32_t i = i0; i < i1;) {
#pragma unroll
      for (int u = 0; u < kOrderRun; u++)
        if (i + u < i1) f(i + u, c[u]);
      i += kOrderRun;
      if (i < i1) read(c, i);
    }
  }
  // Sum of the counts, in every thread.
  __device__ __forceinline__ unsigned long long sum(unsigned long long* totals) const {
    unsigned long long mine = 0, all = 0;
    each([&](int32_t, int32_t c) { mine += c; });
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) mine += __shfl_xor(mine, off);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) totals[threadIdx.x >> 6] = mine;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kOrderWaves; w++) all += totals[w];
    return all;
  }
};

// Exclusive sum of a value over the workgroup's threads; *all: of every thread's.
__device__ __forceinline__ int32_t sum_before(int32_t v, int32_t* waves, int32_t* all) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int32_t up = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int32_t y = __shfl_up(up, off);
    if (lane >= off) up += y;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = up;
  __syncthreads();
  int32_t before = up - v, sum = 0;
  for (int w = 0; w < kOrderWaves; w++) {
    before += w < wave ? waves[w] : 0;
    sum += waves[w];
  }
  *all = sum;
  return before;
}

// Places the items that cls does not skip (-1): emit(item, place), the places from 0 on.  Eight classes of list lengths,
// the longest first, each in the items' order and spread over the XCDs.
template <typename K, typename E>
__device__ __forceinline__ void place_items(const Items& items, int32_t* at, int32_t* waves, K cls, E emit) {
  const int tid = threadIdx.x;
  auto cell = [&](int p) -> int32_t& { return at[p + (p >> 5)]; };       // (a lane's eight lie in banks of their own)
  int32_t have[kOrderClasses] = {};
  items.each([&](int32_t, int32_t c) {
    const int k = cls(c);
#pragma unroll
    for (int x = 0; x < kOrderClasses; x++) have[x] += x == k;
  });
#pragma unroll
  for (int x = 0; x < kOrderClasses; x++) cell(x * kOrderThreads + tid) = have[x];
  __syncthreads();
  // exclusive sums over (class, thread): eight entries a thread, then over the threads
  int32_t v[kOrderClasses], sum = 0, all;
#pragma unroll
  for (int x = 0; x < kOrderClasses; x++) {
    v[x] = sum;
    sum += cell(tid * kOrderClasses + x);
  }
  const int32_t before = sum_before(sum, waves, &all);
#pragma unroll
  for (int x = 0; x < kOrderClasses; x++) cell(tid * kOrderClasses + x) = before + v[x];
  __syncthreads();
  int32_t next[kOrderClasses], start[kOrderClasses + 1];
#pragma unroll
  for (int x = 0; x < kOrderClasses; x++) {
    next[x] = cell(x * kOrderThreads + tid);
    start[x] = cell(x * kOrderThreads);
  }
  start[kOrderClasses] = all;
  items.each([&](int32_t i, int32_t c) {
    const int k = cls(c);
    if (k < 0) return;
    int32_t first = 0, place = 0, size = 0;       // of the class (emitting within the loop would emit eight times)
#pragma unroll
    for (int x = 0; x < kOrderClasses; x++) {
      first = x == k ? start[x] : first;
      place = x == k ? next[x] - start[x] : place;
      size = x == k ? start[x + 1] - start[x] : size;
      next[x] += x == k;
    }
    emit(i, first + spread(place, size));
  });
}

__device__ __forceinline__ int length_class(int32_t c, float mean) {
  const float x = (float)c;
  return x >= 4.0f * mean ? 0 : x >= 2.83f * mean ? 1 : x >= 2.0f * mean ? 2 : x >= 1.5f * mean ? 3 :
         x >= 1.25f * mean ? 4 : x >= 1.1f * mean ? 5 : x >= 0.9f * mean ? 6 : 7;
}

//   order[workgroup] = (item, piece << 16 | pieces): the pieces first (a piece's tile of the workspace is its workgroup's
//                      number), then the whole items by their lengths, then -1
//   split[i]         = (item, workgroup of its first piece, pieces), split[-1].x their number
__device__ __forceinline__ void order_pieces(const Items& items, const Pieces& to, int32_t room, OrderSpace& s) {
  const Cut cut(items.sum(s.totals), items.n, room, to);
  int32_t split = 0, pieces = 0, all_split = 0, all_pieces = 0;
  if (to.pieces) {
    items.each([&](int32_t, int32_t c) {
      if (!cut.cuts(c)) return;
      split++;
      pieces += cut.pieces(c);
    });
    split = sum_before(split, s.waves, &all_split);
    pieces = sum_before(pieces, s.waves, &all_pieces);
    if (threadIdx.x == 0) to.split[-1] = make_int4(all_split, 0, 0, 0);
    if (all_split)
      items.each([&](int32_t i, int32_t c) {
        if (!cut.cuts(c)) return;
        const int32_t p = cut.pieces(c);
        to.split[split++] = make_int4(i, pieces, p, 0);
        for (int32_t x = 0; x < p; x++) to.order[pieces++] = make_int2(i, x << 16 | p);
      });
  }
  place_items(items, s.at, s.waves, [&](int32_t c) { return cut.cuts(c) ? -1 : length_class(c, cut.mean); },
              [&](int32_t i, int32_t place) { to.order[all_pieces + place] = make_int2(i, 1); });
  for (int32_t i = all_pieces + items.n - all_split + threadIdx.x; i < to.grid; i += kOrderThreads)
    to.order[i] = make_int2(-1, 0);
}

// Pairs of query blocks: pair_order[workgroup] = (head, pair), and whether they run: if they pay (pairs_pay) and no list
// goes in pieces.
__device__ __forceinline__ void order_pairs(const MapArgs& a, int32_t head_dim, int32_t room, OrderSpace& s) {
  const Items rows(a.row_counts, a.n_bh * a.nbq), items(a.pair_counts, a.n_bh * pairs_per_head(a.nbq));
  const unsigned long long single = rows.sum(s.totals), either = items.sum(s.totals);
  const Cut cut(single, rows.n, room, a.row_pieces);
  int32_t any = 0;
  rows.each([&](int32_t, int32_t c) { any |= cut.cuts(c); });
  any = __syncthreads_or(any);
  if (threadIdx.x == 0) *a.paired = !any && pairs_pay(either, single, head_dim) ? 1 : 0;
  const float mean = (float)either / (float)items.n;
  place_items(items, s.at, s.waves, [&](int32_t c) { return length_class(c, mean); },
              [&](int32_t i, int32_t place) { a.pair_order[place] = i; });
}

// Up to two orders, a workgroup each: the rows', and the pairs' of a forward call or the columns' of a backward call.
enum class Order { kRows, kPairs, kCols };
__global__ __launch_bounds__(kOrderThreads) void psa_mapped_order_kernel(MapArgs a, Order first, Order second,
                                                                         int32_t head_dim, int32_t room) {
  __shared__ OrderSpace space;
  const Order which = blockIdx.x == 0 ? first : second;
  if (which == Order::kRows)
    order_pieces(Items(a.row_counts, a.n_bh * a.nbq), a.row_pieces, room, space);
  else if (which == Order::kCols)
    order_pieces(Items(a.col_counts, a.n_bh / a.group * a.nbk), a.col_pieces, room, space);
  else
    order_pairs(a, head_dim, room, space);
}

// Where this lane reads a tile of rows of D channels in LDS, in bytes from the tile's start: `rows` for the operand of
// rows_times, `lo` and `hi` for the two halves of cols_times'.  The swizzle is an exclusive or, so the address of
// a later chunk is that of the first one with bits flipped: one instruction a read.  here() hides the sum
// with the tile's address from the compiler, which would otherwise keep every flipped address of both
// buffers in registers across the loop over the blocks (116 of them, spilled: dk and dv of 12 heads x 32760 took
// 9.5 ms so).
template <int D>
struct LaneAt {
  uint32_t rows, lo, hi;
  __device__ __forceinline__ explicit LaneAt(int lane) {
    constexpr int CPR = D / 8, RB = 2 * D;
    const int h = lane >> 5, g = lane >> 4, j16 = lane & 15;
    const int kr = key_perm(lane & 31);
    rows = kr * RB + ((h ^ swz<CPR>(kr)) << 4);
    const int row = 8 * h + (j16 >> 2), dd = 16 * (g & 1) + 4 * (j16 & 3);
    lo = row * RB + (((dd >> 3) ^ swz<CPR>(row)) << 4) + (dd & 7) * 2;
    hi = (row + 4) * RB + (((dd >> 3) ^ swz<CPR>(row + 4)) << 4) + (dd & 7) * 2;
  }
  __device__ __forceinline__ static uint32_t here(uint32_t tile, uint32_t lane_at) {
    uint32_t at = tile + lane_at;
    asm volatile("" : "+v"(at));
    return at;
  }
};

// The loads of DmaPlan with one register per lane instead of one per slot: a slot is 64 / CPR rows from a multiple
// of them, so its lanes' places in the block are those of slot 0, the swizzle's row bits above them flipped (bits
// that all lanes share), 1 KB further on for each slot.  Offsets kept for every slot spill where two sets of sums
// fill the registers, and reading them back waits for every load in flight, twice a block: dk and dv of 12 heads x
// 32760 took 4.24 ms so, 3.26 this way.  Where they do not spill they are faster (the forward by 1 to 8 %).
template <int D, int BLK>
struct Stream {
  using T = Tile<D, BLK>;
  static constexpr int W = 2 * T::kWaves, S = T::BYTES / (1024 * W);
  uint32_t lane_off;
  int wave, lane;
  __device__ __forceinline__ Stream(int wave_, int lane_) : wave(wave_), lane(lane_) {
    const int row = lane / T::CPR;
    lane_off = row * T::RB + ((lane % T::CPR ^ swz<T::CPR>(row)) << 4);
  }
  // Loads block `blk` of rows x (n of them) into the tile at LDS address `lds`.  Rows behind the last one are read as
  // the last one.
  __device__ __forceinline__ void load(const __bf16* x, uint32_t lds, int blk, int n) const {
    blk = __builtin_amdgcn_readfirstlane(blk);
    const int rows = n - blk * BLK;
    const uint8_t* base = (const uint8_t*)(x + (size_t)blk * BLK * D);
    const int slot0 = __builtin_amdgcn_readfirstlane(wave * S);
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds + slot0 * 1024u);
    if (rows >= BLK) {
#pragma unroll
      for (int i = 0; i < S; i++)
        dma16(to + i * 1024u, lane_off ^ (uint32_t)(swz<T::CPR>((slot0 + i) * (64 / T::CPR)) << 4), base + (slot0 + i) * 1024u);
    } else {
      int l = lane;
      asm volatile("" : "+v"(l));         // formed here, not kept in registers for the last block
#pragma unroll
      for (int i = 0; i < S; i++) {
        const int row = (slot0 + i) * (64 / T::CPR) + l / T::CPR, chunk = l % T::CPR ^ swz<T::CPR>(row);
        dma16(to + i * 1024u, (uint32_t)(min(row, rows - 1) * T::RB + chunk * 16), base);
      }
    }
  }
};

// Loads 64 words from x on into LDS, one per lane.
__device__ __forceinline__ void dma4(uint32_t lds, int lane, const void* x) {
  asm volatile("" : "+v"(lane));          // (the offset is formed here, not kept in a register)
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(4 * lane), "s"(x)
               : "memory");
}

// One 32 x 32 tile X Y^T: 32 rows of the tile X in LDS from `at` on (in the order of key_perm), this lane's row of Y
// in registers; acc is where the sums start.
template <int D>
__device__ __forceinline__ f32x16 rows_times(const bf16x8 (&y)[D / 16], uint32_t at, f32x16 acc) {
#pragma unroll
  for (int cc = 0; cc < D / 16; cc++)
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(PSA_LDS const bf16x8*)(uintptr_t)(at ^ (cc << 5)), y[cc], acc, 0, 0, 0);
  return acc;
}

// out^T += X^T p for 16 rows of the tile X in LDS from `lo` and `hi` on; p holds this lane's eight of them.
template <int D>
__device__ __forceinline__ void cols_times(f32x16 (&out)[D / 32], uint32_t lo, uint32_t hi, bf16x8 p) {
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++) {
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PSA_LDS s16x4*)(uintptr_t)(lo ^ (dt << 6)));
    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PSA_LDS s16x4*)(uintptr_t)(hi ^ (dt << 6)));
    const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    out[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, p, out[dt], 0, 0, 0);
  }
}

template <int D>
__device__ __forceinline__ void load_rows(bf16x8 (&y)[D / 16], const __bf16* row, int h) {
#pragma unroll
  for (int cc = 0; cc < D / 16; cc++) y[cc] = *((const bf16x8*)row + h + 2 * cc);
}

// A value for every row of a tile: element e belongs to row 16 (e / 8) + e % 8 from `row` on.
__device__ __forceinline__ f32x16 row_values(const float* row) {
  f32x16 v;
#pragma unroll
  for (int e = 0; e < 16; e++) v[e] = row[16 * (e >> 3) + (e & 7)];
  return v;
}

__device__ __forceinline__ bf16x8 half_of(const f32x16& v, int j) {
  f32x8 e;
#pragma unroll
  for (int x = 0; x < 8; x++) e[x] = v[8 * j + x];
  return __builtin_convertvector(e, bf16x8);
}

// Stores 32 columns of a row: O^T accumulator `v` of column group dt.
__device__ __forceinline__ void store_cols(__bf16* dst, const f32x16& v, float f) {
#pragma unroll
  for (int a = 0; a < 4; a++) {
    const f32x4 x = {v[4 * a] * f, v[4 * a + 1] * f, v[4 * a + 2] * f, v[4 * a + 3] * f};
    *(bf16x4*)(dst + 8 * a) = __builtin_convertvector(x, bf16x4);
  }
}

// The same, unscaled, into a part's fp32 sums.
__device__ __forceinline__ void store_cols(float* dst, const f32x16& v) {
#pragma unroll
  for (int a = 0; a < 4; a++) *(f32x4*)(dst + 8 * a) = f32x4{v[4 * a], v[4 * a + 1], v[4 * a + 2], v[4 * a + 3]};
}

// How a kernel's lists are shared out: a workgroup each; the same number of parts each; or as order_pieces
// says.
enum class Share { kWhole, kParts, kOrder };

// A workgroup's item and its part of the item's list, whose sums go to `tile` of the workspace if there are several.
template <Share SHARE>
struct Piece {
  int32_t item, part = 0, parts = 1, tile;
  __device__ __forceinline__ Piece(const Pieces& order, int32_t equal_parts) {
    if constexpr (SHARE == Share::kOrder) {
      tile = blockIdx.x;
      const int2 e = order.order[tile];
      item = e.x;
      part = e.y >> 16;
      parts = e.y & 0xffff;
    } else {
      item = tile = item_of(blockIdx.x, gridDim.x);
      if constexpr (SHARE == Share::kParts) {
        parts = equal_parts;
        item = tile / parts;
        part = tile - item * parts;
      }
    }
  }
  __device__ __forceinline__ bool none() const { return SHARE == Share::kOrder && item < 0; }
  __device__ __forceinline__ bool partial() const { return SHARE != Share::kWhole && parts > 1; }
};
// Where a part of a list of n starts.
__device__ __forceinline__ int32_t part_start(int32_t n, int32_t part, int32_t parts) {
  return (int32_t)((int64_t)n * part / parts);
}

// ---------------------------------------------------------------------------------------------
// Forward.
// ---------------------------------------------------------------------------------------------

// A workgroup that takes a part of a list leaves its sums (relative to its base m, with m and l) in the workspace, where
// psa_mapped_join_kernel adds them.
template <int D, int BLK, Share SHARE>
__global__ __launch_bounds__(BLK * 4) __attribute__((amdgpu_waves_per_eu(2, 2))) void psa_mapped_fwd_kernel(MapArgs a) {
  using T = Tile<D, BLK>;
  constexpr int HK = BLK / 2, W = 2 * T::kWaves, DH = T::DT / 2;
  using H = Half<D, BLK, HK>;
  __shared__ __attribute__((aligned(1024))) uint8_t sk[2][T::BYTES];
  __shared__ __attribute__((aligned(1024))) uint8_t sv[2][T::BYTES];
  __shared__ int32_t found[W];
  __shared__ float2 stat[W][32];              // (m, l) of every wave's rows
  extern __shared__ uint16_t list[];          // nbk entries

  if (BLK == 64 && SHARE == Share::kOrder && a.paired && *a.paired) return;   // (psa_mapped_pairs_kernel runs)
  const Piece<SHARE> piece(a.row_pieces, a.parts);
  if (piece.none()) return;
  const bool partial = piece.partial();
  const int32_t bh = piece.item / a.nbq, qb = piece.item - bh * a.nbq, b = bh / a.n_heads, hd = bh - b * a.n_heads;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, gw = wave & (T::kWaves - 1);
  const int grp = __builtin_amdgcn_readfirstlane(wave / T::kWaves);
  const int h = lane >> 5, r32 = lane & 31;
  const int64_t kv_off = b * a.kv_stride_b + (hd / a.group) * a.kv_stride_h;
  const __bf16 *kh = a.k + kv_off, *vh = a.v + kv_off;
  const int32_t n = a.n_k, n_q = a.n_q;
  const int row = qb * BLK + gw * 32 + r32;
  // whether any of this wave's rows exists
  const bool rows = __builtin_amdgcn_readfirstlane(qb * BLK + gw * 32) < n_q;

  const uint8_t* kept = a.map + b * a.map_stride_b + ((int64_t)hd * a.nbq + qb) * a.nbk;
  int32_t nu = kept_list<W>(a.nbk, list, found, [&](int32_t i) { return kept[i] ? i : -1; });
  int32_t first = 0;
  if constexpr (SHARE != Share::kWhole) {
    first = part_start(nu, piece.part, piece.parts);
    nu = part_start(nu, piece.part + 1, piece.parts) - first;
  }
  auto entry = [&](int i) { return (int)__builtin_amdgcn_readfirstlane(list[first + i]); };

  DmaPlan<D, BLK> plan;
  plan.init(__builtin_amdgcn_readfirstlane(wave), lane);
  int kb = 0;
  if (nu > 0) {
    kb = entry(0);
    issue_block<D, BLK>(plan, kh, lds_address(sk[0]), kb, n);
    issue_block<D, BLK>(plan, vh, lds_address(sv[0]), kb, n);
  }
  WaveState<D, BLK> st;
  {
    load_rows<D>(st.q, a.q + ((int64_t)bh * n_q + min(row, n_q - 1)) * D, h);
#pragma unroll
    for (int cc = 0; cc < T::DC; cc++)
      st.q[cc] = __builtin_convertvector(__builtin_convertvector(st.q[cc], f32x8) * a.pow2, bf16x8);
#pragma unroll
    for (int cc = 0; cc < T::DC; cc++) asm volatile("" ::"v"(st.q[cc]));
  }
  st.m = -__builtin_inff();
  st.l = 0.0f;
  st.set_neg_max(0.0f);
  int fresh = 1;
#pragma unroll
  for (int dt = 0; dt < T::DT; dt++) st.o[dt] = (f32x16){};

  const int k0 = grp * HK;
  for (int i = 0; i < nu; i++) {
    const bool tail = (kb + 1) * BLK > n;
    wait_dma<0>();                                        // block i, issued a block ago
    __syncthreads();                                      // ... by every wave; block i-1 read
    const int cur = kb;
    const bool more = i + 1 < nu;
    if (more) {
      kb = entry(i + 1);
      issue_block<D, BLK>(plan, kh, lds_address(sk[(i + 1) & 1]), kb, n);
    }
    if (rows) {
      f32x16 s[H::KT];
      qk_half<D, BLK, HK>(st, s, sk[i & 1], k0, lane);
      if (more) issue_block<D, BLK>(plan, vh, lds_address(sv[(i + 1) & 1]), kb, n);
      softmax_pv_half<D, BLK, false, HK, true>(st, s, sv[i & 1], cur, k0, n, tail, ~0ull, ~0ull, lane, fresh, a.factor);
    } else if (more) {
      issue_block<D, BLK>(plan, vh, lds_address(sv[(i + 1) & 1]), kb, n);
    }
  }

  // Merge: both groups scale their O to the common base; group g finishes columns 32 DH g .., adding what the
  // other group holds of them.
  const float mine = pair_sum(st.l);
  if (h == 0) stat[wave][r32] = make_float2(st.m, mine);
  __syncthreads();                                        // (also: the buffers are no longer read)
  const float2 other = stat[(1 - grp) * T::kWaves + gw][r32];
  const float top = fmaxf(st.m, other.x);
  const float alpha = st.m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((st.m - top) * a.factor);
  const float beta = other.x == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((other.x - top) * a.factor);
  const float lsum = mine * alpha + other.y * beta;
  const float inv = partial ? 1.0f : lsum > 0.0f ? 1.0f / lsum : 0.0f;
  static_assert(W * DH * 4096 <= 4 * T::BYTES, "a wave's half of O fits its share of the buffers");
  constexpr int kPer = T::BYTES / (DH * 4096);            // waves per buffer
  auto slot = [&](int w) { return (f32x4*)((w / kPer < 2 ? sk[w / kPer] : sv[w / kPer - 2]) + (w % kPer) * DH * 4096) + lane; };
  f32x4* out = slot(wave);
#pragma unroll
  for (int j = 0; j < DH; j++)
#pragma unroll
    for (int x = 0; x < 4; x++) {
      const f32x16 &lo = st.o[j], &hi = st.o[DH + j];
      const int e = 4 * x;
      const f32x4 lower = {lo[e], lo[e + 1], lo[e + 2], lo[e + 3]}, upper = {hi[e], hi[e + 1], hi[e + 2], hi[e + 3]};
      out[(j * 4 + x) * 64] = (grp == 0 ? upper : lower) * alpha;
    }
  __syncthreads();
  const f32x4* in = slot((1 - grp) * T::kWaves + gw);
  const int64_t place = partial ? (int64_t)piece.tile * BLK + gw * 32 + r32 : (int64_t)bh * n_q + row;
  const int64_t at = place * D + 32 * DH * grp + 4 * h;
#pragma unroll
  for (int j = 0; j < DH; j++)
#pragma unroll
    for (int x = 0; x < 4; x++) {
      const f32x16 &lo = st.o[j], &hi = st.o[DH + j];
      const int e = 4 * x;
      const f32x4 lower = {lo[e], lo[e + 1], lo[e + 2], lo[e + 3]}, upper = {hi[e], hi[e + 1], hi[e + 2], hi[e + 3]};
      const f32x4 sum = ((grp == 0 ? lower : upper) * alpha + in[(j * 4 + x) * 64]) * inv;
      if (row < n_q) {
        if (partial)
          *(f32x4*)(a.part_o + at + 32 * j + 8 * x) = sum;
        else
          *(bf16x4*)(a.o + at + 32 * j + 8 * x) = __builtin_convertvector(sum, bf16x4);
      }
    }
  if (grp == 0 && h == 0 && row < n_q) {
    if (partial)
      a.part_ml[place] = make_float2(top, lsum);
    else if (a.lse)
      a.lse[place] = lsum > 0.0f ? (top * a.factor + __builtin_log2f(lsum)) * kLn2 : -__builtin_inff();
  }
}

// Maps of 64 on pairs: a workgroup of the pair engine (psa_tile.h) takes two neighbouring query blocks, which share one
// stream of the key blocks that either keeps; a wave works through whole blocks of 64 keys where the kernel above
// gives it 32.  Neighbours that keep much the same blocks gain by it, see pairs_pay.
template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 4 : 2, D == 64 ? 4 : 2))) void psa_mapped_pairs_kernel(MapArgs a) {
  constexpr int BLK = 64;
  using T = Tile<D, BLK>;
  constexpr int W = 2 * T::kWaves;
  __shared__ __attribute__((aligned(1024))) uint8_t sk[2][T::BYTES];
  __shared__ __attribute__((aligned(1024))) uint8_t sv[2][T::BYTES];
  __shared__ int32_t found[W];
  extern __shared__ uint16_t list[];          // nbk entries
  if (*a.paired == 0) return;
  const int32_t np = pairs_per_head(a.nbq), item = a.pair_order[blockIdx.x];
  const int32_t bh = item / np, b = bh / a.n_heads, hd = bh - b * a.n_heads;
  const int2 pr = pair_of(item - bh * np, a.nbq);
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int grp = __builtin_amdgcn_readfirstlane(wave / T::kWaves);
  const uint8_t* first = a.map + b * a.map_stride_b + ((int64_t)hd * a.nbq + pr.x) * a.nbk;
  const int32_t nu = kept_list<W>(a.nbk, list, found, [&](int32_t i) {
    const int rows = (first[i] ? 1 : 0) | (pr.y >= 0 && first[(int64_t)a.nbk + i] ? 2 : 0);
    return rows ? i | rows << kEntryRowShift : -1;
  });
  DmaPlan<D, BLK> plan;
  plan.init(__builtin_amdgcn_readfirstlane(wave), lane);
  const int64_t kv_off = b * a.kv_stride_b + (hd / a.group) * a.kv_stride_h, off = (int64_t)bh * a.n_q;
  process_pair<D, BLK, 1, true, false, true>(plan, grp, a.q + off * D, a.k + kv_off, a.v + kv_off, a.o + off * D,
                                       a.lse ? a.lse + off : nullptr, a.n_q, a.n_k,
                                       __builtin_amdgcn_readfirstlane(grp == 0 ? pr.x : pr.y), nu, 0, list, a.pow2, sk, sv,
                                       nullptr, a.factor);
}

// Adds the parts of a query row: o = sum_p 2^(f (m_p - m)) O_p / sum_p 2^(f (m_p - m)) l_p.  D / 4 lanes for a row's
// channels, G of these side by side for its parts: one where parts are few and rows many (10400 rows in three parts:
// 4 us less than with a workgroup a row), else all 256 / (D / 4) of a workgroup (one lane for all 64 parts of
// a single token took 15 us).  The lists that order_pieces cut have a lane each, a workgroup R rows.
template <int D, int BLK, Share SHARE, int G>
__global__ __launch_bounds__(256) void psa_mapped_join_kernel(MapArgs a) {
  constexpr int L = D / 4, R = 256 / (L * G);
  __shared__ f32x4 sum_o[G > 1 ? G : 1][L];
  __shared__ float2 sum_ml[G];
  const int c = threadIdx.x % L, g = threadIdx.x / L % G;
  int64_t r, first;                       // the row, its place in the first part
  int32_t parts = a.parts;
  if constexpr (SHARE == Share::kOrder) {
    if ((int32_t)blockIdx.x >= min(a.row_pieces.splits, a.row_pieces.split[-1].x)) return;
    const int4 e = a.row_pieces.split[blockIdx.x];
    const int32_t bh = e.x / a.nbq, x = blockIdx.y * R + threadIdx.x / L, row = (e.x - bh * a.nbq) * BLK + x;
    if (row >= a.n_q) return;
    r = (int64_t)bh * a.n_q + row;
    first = (int64_t)e.y * BLK + x;
    parts = e.z;
  } else {
    r = (int64_t)blockIdx.x * R + threadIdx.x / (L * G);
    if (r >= (int64_t)a.n_bh * a.n_q) return;
    const int32_t bh = (int32_t)(r / a.n_q), row = (int32_t)(r - (int64_t)bh * a.n_q), qb = row / BLK;
    first = ((int64_t)bh * a.nbq + qb) * parts * BLK + (row - qb * BLK);
  }
  float m = -__builtin_inff(), l = 0.0f;
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  auto add = [&](float pm, float pl, f32x4 po) {
    const float top = fmaxf(m, pm);
    const float was = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((m - top) * a.factor);
    const float w = pm == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((pm - top) * a.factor);
    l = l * was + pl * w;
    o = o * was + po * w;
    m = top;
  };
#pragma unroll 4
  for (int p = g; p < parts; p += G) {
    const int64_t at = first + (int64_t)p * BLK;
    const float2 ml = a.part_ml[at];
    add(ml.x, ml.y, *(const f32x4*)(a.part_o + at * D + 4 * c));
  }
  if constexpr (G > 1) {
    sum_o[g][c] = o;
    if (c == 0) sum_ml[g] = make_float2(m, l);
    __syncthreads();
    if (g > 0) return;
#pragma unroll
    for (int i = 1; i < G; i++) add(sum_ml[i].x, sum_ml[i].y, sum_o[i][c]);
  }
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  *(bf16x4*)(a.o + r * D + 4 * c) = __builtin_convertvector(o * inv, bf16x4);
  if (a.lse && c == 0) a.lse[r] = l > 0.0f ? (m * a.factor + __builtin_log2f(l)) * kLn2 : -__builtin_inff();
}

// ---------------------------------------------------------------------------------------------
// Backward.
// ---------------------------------------------------------------------------------------------

// Waves per SIMD of dq's kernel: at head dim 64 the registers allow more than two, and no unit alone bounds it (12 heads
// x 16000, a fifth kept, dq, dk and dv: block 64 659 us with two, 639 with three, 660 with four; block 128 641, 635, 630).
constexpr int dq_waves(int d, int blk) { return d == 128 ? 2 : blk == 64 ? 3 : 4; }
// ... of dk's and dv's: head dim 64 and block 64 have room for a third wave (12 heads x 16000, a fifth kept, all three
// gradients: 625 us with two, 592 with three); elsewhere another workgroup would need half the registers.
constexpr int dkv_waves(int d, int blk) { return d == 64 && blk == 64 ? 3 : 2; }

template <int D, int BLK, Share SHARE>
__global__ __launch_bounds__(BLK * 4) __attribute__((amdgpu_waves_per_eu(dq_waves(D, BLK), dq_waves(D, BLK)))) void psa_mapped_dq_kernel(MapArgs a) {
  using T = Tile<D, BLK>;
  constexpr int HK = BLK / 2, W = 2 * T::kWaves, DH = T::DT / 2;
  __shared__ __attribute__((aligned(1024))) uint8_t sk[2][T::BYTES];
  __shared__ __attribute__((aligned(1024))) uint8_t sv[2][T::BYTES];
  __shared__ int32_t found[W];
  extern __shared__ uint16_t list[];          // nbk entries

  const Piece<SHARE> piece(a.row_pieces, a.parts);
  if (piece.none()) return;
  const int32_t bh = piece.item / a.nbq, qb = piece.item - bh * a.nbq, b = bh / a.n_heads, hd = bh - b * a.n_heads;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, gw = wave & (T::kWaves - 1);
  const int grp = __builtin_amdgcn_readfirstlane(wave / T::kWaves);
  const int h = lane >> 5, r32 = lane & 31;
  const int64_t kv_off = b * a.kv_stride_b + (hd / a.group) * a.kv_stride_h;
  const __bf16 *kh = a.k + kv_off, *vh = a.v + kv_off;
  const int32_t n = a.n_k, n_q = a.n_q;
  const int row = qb * BLK + gw * 32 + r32;

  const uint8_t* kept = a.map + b * a.map_stride_b + ((int64_t)hd * a.nbq + qb) * a.nbk;
  int32_t nu = kept_list<W>(a.nbk, list, found, [&](int32_t i) { return kept[i] ? i : -1; });
  int32_t first = 0;
  if constexpr (SHARE != Share::kWhole) {
    first = part_start(nu, piece.part, piece.parts);
    nu = part_start(nu, piece.part + 1, piece.parts) - first;
  }
  auto entry = [&](int i) { return (int)__builtin_amdgcn_readfirstlane(list[first + i]); };
  DmaPlan<D, BLK> plan;
  plan.init(__builtin_amdgcn_readfirstlane(wave), lane);
  int kb = 0;
  if (nu > 0) {
    kb = entry(0);
    issue_block<D, BLK>(plan, kh, lds_address(sk[0]), kb, n);
    issue_block<D, BLK>(plan, vh, lds_address(sv[0]), kb, n);
  }
  const LaneAt<D> at_lane(lane);
  bf16x8 q[T::DC], g[T::DC];
  const int64_t at = ((int64_t)bh * n_q + min(row, n_q - 1)) * D;
  load_rows<D>(q, a.q + at, h);
  load_rows<D>(g, a.grad_o + at, h);
  const int64_t sat = (int64_t)bh * a.nbq * BLK + row;
  const float neg_lse2 = a.neg_lse2[sat], neg_delta = a.neg_delta[sat];
  f32x16 dq[T::DT];
#pragma unroll
  for (int dt = 0; dt < T::DT; dt++) dq[dt] = (f32x16){};

  for (int i = 0; i < nu; i++) {
    const bool tail = (kb + 1) * BLK > n;
    wait_dma<0>();
    __syncthreads();
    const int cur = kb;
    const bool more = i + 1 < nu;
    if (more) {
      kb = entry(i + 1);
      issue_block<D, BLK>(plan, kh, lds_address(sk[(i + 1) & 1]), kb, n);
      issue_block<D, BLK>(plan, vh, lds_address(sv[(i + 1) & 1]), kb, n);
    }
    const uint32_t tk = lds_address(sk[i & 1]) + grp * HK * T::RB, tv = lds_address(sv[i & 1]) + grp * HK * T::RB;
    const uint32_t kr = LaneAt<D>::here(tk, at_lane.rows), vr = LaneAt<D>::here(tv, at_lane.rows);
    const uint32_t klo = LaneAt<D>::here(tk, at_lane.lo), khi = LaneAt<D>::here(tk, at_lane.hi);
#pragma unroll
    for (int kt = 0; kt < HK / 32; kt++) {
      const int k0 = grp * HK + 32 * kt;
      f32x16 s = rows_times<D>(q, kr + 32 * kt * T::RB, (f32x16){});
      f32x16 dp = rows_times<D>(g, vr + 32 * kt * T::RB, (f32x16){} + neg_delta);
      if (tail) {
        // Keys behind the last one read as the last one, whose weight is finite: no gradient of theirs.
        asm volatile("" ::: "memory");        // keep the mask a branch taken only by the last block
        const int kbase = cur * BLK + k0 + 8 * h;
#pragma unroll
        for (int e = 0; e < 16; e++)
          if (kbase + 16 * (e >> 3) + (e & 7) >= n) dp[e] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < 16; e++) dp[e] *= __builtin_amdgcn_exp2f(fmaf(s[e], a.c, neg_lse2));
#pragma unroll
      for (int j = 0; j < 2; j++) {
        const int off = (32 * kt + 16 * j) * T::RB;
        cols_times<D>(dq, klo + off, khi + off, half_of(dp, j));
      }
    }
  }

  // Group g finishes columns 32 DH g .., adding what the other group holds of them.
  __syncthreads();                                        // the buffers are no longer read
  constexpr int kPer = T::BYTES / (DH * 4096);            // waves per buffer
  auto slot = [&](int w) { return (f32x4*)((w / kPer < 2 ? sk[w / kPer] : sv[w / kPer - 2]) + (w % kPer) * DH * 4096) + lane; };
  f32x4* out = slot(wave);
#pragma unroll
  for (int j = 0; j < DH; j++)
#pragma unroll
    for (int x = 0; x < 4; x++)
#pragma unroll
      for (int e = 0; e < 4; e++)
        out[(j * 4 + x) * 64][e] = grp == 0 ? dq[DH + j][4 * x + e] : dq[j][4 * x + e];
  __syncthreads();
  const f32x4* in = slot((1 - grp) * T::kWaves + gw);
  const bool partial = piece.partial();
  if (partial || row < n_q) {
    const int64_t dst = (partial ? (int64_t)piece.tile * BLK + gw * 32 + r32 : (int64_t)bh * n_q + row) * D + 32 * DH * grp + 4 * h;
#pragma unroll
    for (int j = 0; j < DH; j++) {
      f32x16 v;
#pragma unroll
      for (int x = 0; x < 4; x++)
#pragma unroll
        for (int e = 0; e < 4; e++)
          v[4 * x + e] = (grp == 0 ? dq[j][4 * x + e] : dq[DH + j][4 * x + e]) + in[(j * 4 + x) * 64][e];
      if (partial)
        store_cols(a.part_q + dst + 32 * j, v);
      else
        store_cols(a.dq + dst + 32 * j, v, a.scale);
    }
  }
}

template <int D, int BLK, Share SHARE>
__global__ __launch_bounds__(BLK * 4) __attribute__((amdgpu_waves_per_eu(dkv_waves(D, BLK), dkv_waves(D, BLK)))) void psa_mapped_dkv_kernel(MapArgs a) {
  using T = Tile<D, BLK>;
  constexpr int HQ = BLK / 2, W = 2 * T::kWaves;
  __shared__ __attribute__((aligned(1024))) uint8_t sq[2][T::BYTES];
  __shared__ __attribute__((aligned(1024))) uint8_t sg[2][T::BYTES];
  __shared__ __attribute__((aligned(16))) float stat[2][2][BLK];       // -lse log2(e) and -delta of a streamed block
  __shared__ int32_t found[W];
  extern __shared__ uint16_t list[];          // nbq entries

  const Piece<SHARE> piece(a.col_pieces, a.head_parts * a.list_parts);
  if (piece.none()) return;
  const int32_t bk = piece.item / a.nbk, kb = piece.item - bk * a.nbk, n_kv = a.n_heads / a.group;
  const int32_t b = bk / n_kv, hk = bk - b * n_kv;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, gw = wave & (T::kWaves - 1);
  const int grp = __builtin_amdgcn_readfirstlane(wave / T::kWaves);
  const int h = lane >> 5, r32 = lane & 31;
  const int32_t n_q = a.n_q, n_k = a.n_k;
  const int key = kb * BLK + gw * 32 + r32;
  bf16x8 k[T::DC], v[T::DC];
  {
    const int64_t at = b * a.kv_stride_b + hk * a.kv_stride_h + (int64_t)min(key, n_k - 1) * D;
    load_rows<D>(k, a.k + at, h);
    load_rows<D>(v, a.v + at, h);
  }
  f32x16 dk[T::DT], dv[T::DT];
#pragma unroll
  for (int dt = 0; dt < T::DT; dt++) dk[dt] = dv[dt] = (f32x16){};
  const int wave_s = __builtin_amdgcn_readfirstlane(wave);
  const Stream<D, BLK> stream(wave_s, lane);
  const LaneAt<D> at_lane(lane);

  // the query heads of this workgroup, and its part of each one's list, or of all their lists one behind the other
  int32_t hd0 = hk * a.group, hd1 = hd0 + a.group, lp = 0, lo = 0, hi = 0;
  if constexpr (SHARE == Share::kParts) {
    const int32_t hp = piece.part / a.list_parts;
    lp = piece.part - hp * a.list_parts;
    hd1 = hd0 + a.group * (hp + 1) / a.head_parts;
    hd0 += a.group * hp / a.head_parts;
  }
  if constexpr (SHARE == Share::kOrder) {
    const int32_t all = a.col_counts[piece.item];
    lo = part_start(all, piece.part, piece.parts);
    hi = part_start(all, piece.part + 1, piece.parts);
  }
  for (int32_t hd = hd0; hd < hd1; hd++) {
    if (SHARE == Share::kOrder && hi <= 0) break;
    const int64_t bh = (int64_t)b * a.n_heads + hd;
    const __bf16 *qh = a.q + bh * n_q * D, *gh = a.grad_o + bh * n_q * D;
    // This wave's 64 of the 2 BLK row values of a block (waves behind them load none).
    const int which = wave_s * 64 / BLK, place = wave_s * 64 % BLK;
    const float* sh = (which == 0 ? a.neg_lse2 : a.neg_delta) + bh * a.nbq * BLK + place;
    // (its barriers also separate the buffers from the head before)
    const uint8_t* kept = a.map + b * a.map_stride_b + (int64_t)hd * a.nbq * a.nbk + kb;
    int32_t nu = kept_list<W>(a.nbq, list, found, [&](int32_t i) { return kept[(int64_t)i * a.nbk] ? i : -1; });
    int32_t first = 0;
    if constexpr (SHARE == Share::kParts) {
      first = part_start(nu, lp, a.list_parts);
      nu = part_start(nu, lp + 1, a.list_parts) - first;
    }
    if constexpr (SHARE == Share::kOrder) {
      const int32_t len = nu;
      first = max(0, min(len, lo));
      nu = max(0, min(len, hi)) - first;
      lo -= len;
      hi -= len;
    }
    auto entry = [&](int i) { return (int)__builtin_amdgcn_readfirstlane(list[first + i]); };
    auto issue = [&](int i) {
      const int qb = entry(i);
      stream.load(qh, lds_address(sq[i & 1]), qb, n_q);
      stream.load(gh, lds_address(sg[i & 1]), qb, n_q);
      if (which < 2) dma4(lds_address(&stat[i & 1][which][place]), lane, sh + (int64_t)qb * BLK);
    };
    if (nu > 0) issue(0);
    for (int i = 0; i < nu; i++) {
      wait_dma<0>();
      __syncthreads();
      const bool more = i + 1 < nu;
      if (more) issue(i + 1);
      const uint32_t tq = lds_address(sq[i & 1]) + grp * HQ * T::RB, tg = lds_address(sg[i & 1]) + grp * HQ * T::RB;
      const uint32_t qr = LaneAt<D>::here(tq, at_lane.rows), gr = LaneAt<D>::here(tg, at_lane.rows);
      const uint32_t qlo = LaneAt<D>::here(tq, at_lane.lo), qhi = LaneAt<D>::here(tq, at_lane.hi);
      const uint32_t glo = LaneAt<D>::here(tg, at_lane.lo), ghi = LaneAt<D>::here(tg, at_lane.hi);
#pragma unroll
      for (int kt = 0; kt < HQ / 32; kt++) {
        const int q0 = grp * HQ + 32 * kt;
        __builtin_amdgcn_sched_barrier(0);      // one tile's operands at a time
        f32x16 s = rows_times<D>(k, qr + 32 * kt * T::RB, (f32x16){});
        f32x16 dp = rows_times<D>(v, gr + 32 * kt * T::RB, row_values(&stat[i & 1][1][q0 + 8 * h]));
        const f32x16 neg_lse2 = row_values(&stat[i & 1][0][q0 + 8 * h]);
#pragma unroll
        for (int e = 0; e < 16; e++) s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], a.c, neg_lse2[e]));
#pragma unroll
        for (int j = 0; j < 2; j++) {
          const int off = (32 * kt + 16 * j) * T::RB;
          cols_times<D>(dv, glo + off, ghi + off, half_of(s, j));
        }
        dp *= s;
#pragma unroll
        for (int j = 0; j < 2; j++) {
          const int off = (32 * kt + 16 * j) * T::RB;
          cols_times<D>(dk, qlo + off, qhi + off, half_of(dp, j));
        }
      }
    }
  }

  // Group 0 finishes dv, group 1 dk, adding what the other group holds.
  __syncthreads();                                        // the buffers are no longer read
  constexpr int kPer = T::BYTES / (T::DT * 4096);         // waves per buffer
  static_assert(kPer >= 1 && W <= 4 * kPer, "a wave's sums fit its share of the buffers");
  auto slot = [&](int w) { return (f32x4*)((w / kPer < 2 ? sq[w / kPer] : sg[w / kPer - 2]) + (w % kPer) * T::DT * 4096) + lane; };
  f32x4* out = slot(wave);
#pragma unroll
  for (int j = 0; j < T::DT; j++)
#pragma unroll
    for (int x = 0; x < 4; x++)
#pragma unroll
      for (int e = 0; e < 4; e++)
        out[(j * 4 + x) * 64][e] = grp == 0 ? dk[j][4 * x + e] : dv[j][4 * x + e];
  __syncthreads();
  const f32x4* in = slot((1 - grp) * T::kWaves + gw);
  const bool partial = piece.partial();
  if (partial || key < n_k) {
    const int64_t dst = (partial ? (int64_t)piece.tile * BLK + gw * 32 + r32 : (int64_t)bk * n_k + key) * D + 4 * h;
#pragma unroll
    for (int j = 0; j < T::DT; j++) {
      f32x16 t;
#pragma unroll
      for (int x = 0; x < 4; x++)
#pragma unroll
        for (int e = 0; e < 4; e++)
          t[4 * x + e] = (grp == 0 ? dv[j][4 * x + e] : dk[j][4 * x + e]) + in[(j * 4 + x) * 64][e];
      if (partial)
        store_cols((grp == 0 ? a.part_v : a.part_k) + dst + 32 * j, t);
      else
        store_cols((grp == 0 ? a.dv : a.dk) + dst + 32 * j, t, grp == 0 ? 1.0f : a.scale);
    }
  }
}

// The sums of what several workgroups left of an item, of dk, dv and dq as far as these have any; a workgroup adds 1024
// columns of 16 bytes.
struct Sums {
  const float* part;
  __bf16* out;
  const int4* split;                // the items and their parts, or null: `parts` of every item
  float scale;
  int32_t items, parts, n, nb;      // items: all of them, or at most these are split; rows: n in nb blocks per head
};
struct AllSums {
  Sums of[3];
};
template <int D, int BLK>
__global__ __launch_bounds__(256) void psa_mapped_sum_kernel(AllSums all) {
  constexpr int L = D / 4, kGroups = BLK * L / 1024;
  const Sums p = all.of[blockIdx.y / kGroups];
  const int32_t i = blockIdx.x;
  if (i >= (p.split ? min(p.items, p.split[-1].x) : p.items)) return;
  const int4 e = p.split ? p.split[i] : make_int4(i, i * p.parts, p.parts, 0);
  const int32_t head = e.x / p.nb, row0 = (e.x - head * p.nb) * BLK;
  const f32x4* src = (const f32x4*)p.part + (int64_t)e.y * (BLK * L);
  __bf16* dst = p.out + ((int64_t)head * p.n + row0) * D;
  f32x4 s[4] = {};
  const int at = blockIdx.y % kGroups * 1024 + threadIdx.x;
#pragma unroll 2
  for (int x = 0; x < e.z; x++)
#pragma unroll
    for (int u = 0; u < 4; u++) s[u] += src[(int64_t)x * (BLK * L) + at + 256 * u];
#pragma unroll
  for (int u = 0; u < 4; u++)
    if (row0 + (at + 256 * u) / L < p.n)
      *(bf16x4*)(dst + 4 * (at + 256 * u)) = __builtin_convertvector(s[u] * p.scale, bf16x4);
}

int32_t list_bytes(int32_t nb) { return (2 * nb + 15) & ~15; }

template <typename F>
hipError_t by_shape(int32_t head_dim, int32_t block, F f) {
  using I64 = std::integral_constant<int, 64>;
  using I128 = std::integral_constant<int, 128>;
  if (head_dim == 128) return block == 128 ? f(I128(), I128()) : f(I128(), I64());
  return block == 128 ? f(I64(), I128()) : f(I64(), I64());
}

}  // namespace

// What comes before the main kernels: a backward call's row values, the list lengths and the orders of the rows and columns
// that have one.
template <int D>
static hipError_t launch_prepare(const MapArgs& a, bool backward, hipStream_t stream) {
  const int32_t n_kv = a.n_bh / a.group;
  const int64_t values = backward ? value_groups(a.n_bh, D, a.nbq, a.block) : 0;
  const int64_t rows = a.row_counts ? row_groups(a.n_bh, a.nbq) : 0, cols = a.col_counts ? col_groups(n_kv, a.nbk) : 0;
  const int64_t groups = values + rows + cols;
  if (groups == 0) return hipSuccess;
  hipLaunchKernelGGL(psa_mapped_prepare_kernel<D>, dim3((uint32_t)groups), dim3(256), 0, stream, a, (int32_t)values,
                     (int32_t)rows);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || (!a.row_counts && !a.col_counts)) return e;
  const Order other = backward ? Order::kCols : Order::kPairs;
  const bool both = a.row_counts && (backward ? a.col_counts != nullptr : a.paired != nullptr);
  hipLaunchKernelGGL(psa_mapped_order_kernel, dim3(both ? 2 : 1), dim3(kOrderThreads), 0, stream, a,
                     a.row_counts ? Order::kRows : other, other, D, room_of(a.block));
  return hipGetLastError();
}

hipError_t launch_map_fwd(const MapArgs& a, int32_t head_dim, hipStream_t stream) {
  return by_shape(head_dim, a.block, [&](auto dim, auto blk) {
    constexpr int D = decltype(dim)::value, B = decltype(blk)::value;
    constexpr int kLanes = D / 4, kSide = 256 / kLanes;
    const int32_t items = a.n_bh * a.nbq, rows = a.n_bh * a.n_q, list = list_bytes(a.nbk);
    const dim3 threads(4 * B);
    hipError_t e = launch_prepare<D>(a, false, stream);
    if (e != hipSuccess) return e;
    if (a.row_pieces.grid) {
      if (B == 64 && a.paired) {
        hipLaunchKernelGGL((psa_mapped_pairs_kernel<D>), dim3(a.n_bh * pairs_per_head(a.nbq)), dim3(256), list, stream, a);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
      }
      hipLaunchKernelGGL((psa_mapped_fwd_kernel<D, B, Share::kOrder>), dim3(a.row_pieces.grid), threads, list, stream, a);
      e = hipGetLastError();
      if (e != hipSuccess || a.row_pieces.splits == 0) return e;
      hipLaunchKernelGGL((psa_mapped_join_kernel<D, B, Share::kOrder, 1>), dim3(a.row_pieces.splits, B / kSide), dim3(256), 0,
                         stream, a);
    } else if (a.parts == 1) {
      hipLaunchKernelGGL((psa_mapped_fwd_kernel<D, B, Share::kWhole>), dim3(items), threads, list, stream, a);
    } else {
      hipLaunchKernelGGL((psa_mapped_fwd_kernel<D, B, Share::kParts>), dim3(items * a.parts), threads, list, stream, a);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
      if (a.parts <= 4)
        hipLaunchKernelGGL((psa_mapped_join_kernel<D, B, Share::kParts, 1>), dim3((rows + kSide - 1) / kSide), dim3(256), 0,
                           stream, a);
      else
        hipLaunchKernelGGL((psa_mapped_join_kernel<D, B, Share::kParts, kSide>), dim3(rows), dim3(256), 0, stream, a);
    }
    return hipGetLastError();
  });
}

hipError_t launch_map_bwd(const MapArgs& a, int32_t head_dim, hipStream_t stream) {
  return by_shape(head_dim, a.block, [&](auto dim, auto blk) {
    constexpr int D = decltype(dim)::value, B = decltype(blk)::value;
    hipError_t e = launch_prepare<D>(a, true, stream);
    if (e != hipSuccess) return e;
    const int32_t n_kv = a.n_bh / a.group, rows = a.n_bh * a.nbq, cols = n_kv * a.nbk, kv_parts = a.head_parts * a.list_parts;
    const dim3 threads(4 * B);
    const bool row_order = a.row_pieces.grid > 0, col_order = a.col_pieces.grid > 0;
    if (col_order)
      hipLaunchKernelGGL((psa_mapped_dkv_kernel<D, B, Share::kOrder>), dim3(a.col_pieces.grid), threads, list_bytes(a.nbq),
                         stream, a);
    else if (kv_parts > 1)
      hipLaunchKernelGGL((psa_mapped_dkv_kernel<D, B, Share::kParts>), dim3(cols * kv_parts), threads, list_bytes(a.nbq), stream,
                         a);
    else
      hipLaunchKernelGGL((psa_mapped_dkv_kernel<D, B, Share::kWhole>), dim3(cols), threads, list_bytes(a.nbq), stream, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (row_order)
      hipLaunchKernelGGL((psa_mapped_dq_kernel<D, B, Share::kOrder>), dim3(a.row_pieces.grid), threads, list_bytes(a.nbk),
                         stream, a);
    else if (a.parts > 1)
      hipLaunchKernelGGL((psa_mapped_dq_kernel<D, B, Share::kParts>), dim3(rows * a.parts), threads, list_bytes(a.nbk), stream,
                         a);
    else
      hipLaunchKernelGGL((psa_mapped_dq_kernel<D, B, Share::kWhole>), dim3(rows), threads, list_bytes(a.nbk), stream, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    AllSums sums;
    int32_t n = 0, most = 0;
    auto sum = [&](const float* part, __bf16* out, const Pieces& p, float scale, int32_t items, int32_t parts, int32_t len,
                   int32_t nb) {
      if (!p.grid && parts == 1) return;
      sums.of[n] = {part, out, p.split, scale, p.grid ? p.splits : items, parts, len, nb};
      most = std::max(most, sums.of[n++].items);
    };
    sum(a.part_k, a.dk, a.col_pieces, a.scale, cols, kv_parts, a.n_k, a.nbk);
    sum(a.part_v, a.dv, a.col_pieces, 1.0f, cols, kv_parts, a.n_k, a.nbk);
    sum(a.part_q, a.dq, a.row_pieces, a.scale, rows, a.parts, a.n_q, a.nbq);
    if (n == 0) return hipSuccess;
    hipLaunchKernelGGL((psa_mapped_sum_kernel<D, B>), dim3(most, n * (B * D / 4096)), dim3(256), 0, stream, sums);
    return hipGetLastError();
  });
}

}  // namespace psa
