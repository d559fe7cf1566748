// Block selection by mean scores: HIP kernels for gfx950.
//
//   mq_i, mk_j = means of the queries of block i and of the keys of block j
//   s_ij = <mq_i, mk_j>;  row i keeps the `keep` highest of the key blocks before the text, of equal ones the
//   lowest index, and every block with text; a query block with text keeps everything
//
// Whether a block is kept hangs on the order of nearly equal scores, so means and scores are held in 64 bits: sums of
// up to 128 bf16 values are then exact where they lie within 2^38 of each other, and the result does not
// depend on how anything was split.  64-bit products cost little here: 2 nq nk d per head, 46 us at the 78
// TFLOP/s of the matrix cores for 40 heads of 591 x 591 blocks, next to 300 us for reading q and k once,
// which is the bound.  That call takes 460 us: the means 280 (5.5 TB/s), scores and search 175.
//
//   psa_block_mean_kernel    one pass over q and k
//   psa_select_kernel        16 query blocks of a head per workgroup: scores with v_mfma_f64_16x16x4, then
//                            per row a search for the lowest score that is kept, bit by bit
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "psa_launch.h"
#include "psa_map.h"
#include "psa_tile.h"

namespace psa {
namespace {

typedef double f64x2 __attribute__((ext_vector_type(2)));
typedef double f64x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

// Means of the blocks of one tensor, one workgroup each.  D / 8 lanes read a row; every lane adds its eight
// channels over its rows, the workgroup's rows are added through LDS.
template <int D>
__global__ __launch_bounds__(256) void psa_block_mean_kernel(SelectArgs a) {
  constexpr int L = D / 8, G = 256 / L;
  const bool keys = blockIdx.x >= a.q_blocks_all;
  const int32_t i = keys ? blockIdx.x - a.q_blocks_all : blockIdx.x;
  const int32_t nb = keys ? a.nbk : a.nbq, n = keys ? a.n_k : a.n_q;
  const int32_t bh = i / nb, blk = i - bh * nb;
  const __bf16* x = keys ? a.k + (bh / a.n_kv_heads) * a.kv_stride_b + (bh % a.n_kv_heads) * a.kv_stride_h
                         : a.q + (int64_t)bh * a.n_q * D;
  const int32_t r0 = blk * a.block, rows = min(a.block, n - r0);
  const int chunk = threadIdx.x % L, g = threadIdx.x / L;
  double sum[8] = {};
  const __bf16* src = x + (int64_t)(r0 + g) * D + 8 * chunk;
  for (int32_t r = g; r < rows; r += 4 * G) {
    f32x8 v[4];
#pragma unroll
    for (int u = 0; u < 4; u++) {
      const int32_t back = max(0, r + u * G - (rows - 1));      // (a place behind the block: its last row, not added)
      v[u] = __builtin_convertvector(*(const bf16x8*)(src + (int64_t)(r - g + u * G - back) * D), f32x8);
    }
#pragma unroll
    for (int u = 0; u < 4; u++)
      if (r + u * G < rows)
#pragma unroll
        for (int e = 0; e < 8; e++) sum[e] += (double)v[u][e];
  }
  __shared__ double part[G][D + 2];
#pragma unroll
  for (int e = 0; e < 8; e++) part[g][8 * chunk + e] = sum[e];
  __syncthreads();
  if (threadIdx.x < D) {
    double s = 0.0;
#pragma unroll
    for (int r = 0; r < G; r++) s += part[r][threadIdx.x];
    (keys ? a.mean_k : a.mean_q)[(int64_t)i * D + threadIdx.x] = s / (double)rows;
  }
}

// Scores as unsigned words of the same order; above 0 for every score.  -0 counts as 0, NaN as -inf.
__device__ __forceinline__ uint64_t ordered(double s) {
  s = s != s ? -__builtin_inf() : s + 0.0;
  const uint64_t b = __builtin_bit_cast(uint64_t, s);
  return b >> 63 ? ~b : b | (1ull << 63);
}

constexpr int kSelectRows = 16;

// LDS: the workgroup's scores are kept there, up to kSelectLds key blocks (two workgroups per CU, more where they
// are fewer).  Else they go to a slab of the workspace, which stays in the L2.  R: score words per lane and row in
// registers (0: read again for every bit).
constexpr int kSelectLds = 624;

// The means of 16 blocks as the matrix core's operand: of block j (16 of them over lane % 16) this lane's channels
// are 8 s + 2 part + {0, 1}, part = lane / 16, at element 4 s.  (Any assignment of channels to the steps of a product
// will do if both sides share it; this one reads 64 contiguous bytes of a block at a time.)
template <int D>
__device__ __forceinline__ const f64x2* mean_of(const double* mean, int32_t j, int32_t nb, int part) {
  return (const f64x2*)(mean + (int64_t)min(j, nb - 1) * D) + part;
}

// Eight waves, two workgroups per CU at 624 key blocks: the search is a chain of compares and counts that only other
// waves can fill.
constexpr int kSelectWaves = 8;

template <int D, int R, bool LDS>
__global__ __launch_bounds__(64 * kSelectWaves) __attribute__((amdgpu_waves_per_eu(4))) void psa_select_kernel(SelectArgs a) {
  constexpr int S = D / 4;                         // channels of a lane
  extern __shared__ uint64_t lds_words[];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, part = lane >> 4;
  const int32_t per_head = (a.nbq + kSelectRows - 1) / kSelectRows, items = a.n_bh * per_head;
  const int32_t cap = a.slab;
  uint64_t* const words = LDS ? lds_words : a.scores + (int64_t)blockIdx.x * kSelectRows * cap;
  // consecutive items of one XCD share the keys' means
  const int32_t share = (items + kNumQueues - 1) / kNumQueues;
  for (int32_t at = blockIdx.x / kNumQueues; at < share; at += gridDim.x / kNumQueues) {
    const int32_t item = (blockIdx.x % kNumQueues) * share + at;
    if (item >= items) break;
    const int32_t bh = item / per_head, i0 = (item - bh * per_head) * kSelectRows;
    const int32_t b = bh / a.n_heads, kv = b * a.n_kv_heads + (bh - b * a.n_heads) / a.group;
    const int32_t kept = min(a.keep, a.first_k);
    // A row that keeps all or nothing needs no scores.
    if (kept > 0 && kept < a.first_k && i0 < a.first_q) {
      const double* mk = a.mean_k + (int64_t)kv * a.nbk * D;
      const f64x2* mq = mean_of<D>(a.mean_q + (int64_t)bh * a.nbq * D, i0 + col, a.nbq, part);
      f64x2 q[S / 2];
#pragma unroll
      for (int s = 0; s < S / 2; s++) q[s] = mq[4 * s];
      for (int32_t j0 = 16 * wave; j0 < a.first_k; j0 += 16 * kSelectWaves) {
        const f64x2* k = mean_of<D>(mk, j0 + col, a.nbk, part);
        f64x4 acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
        for (int s = 0; s < S / 2; s++) {
          const f64x2 x = k[4 * s];
          acc = __builtin_amdgcn_mfma_f64_16x16x4f64(q[s][0], x[0], acc, 0, 0, 0);
          acc = __builtin_amdgcn_mfma_f64_16x16x4f64(q[s][1], x[1], acc, 0, 0, 0);
        }
        // element e: query block 4 e + part, key block col
        if (j0 + col < a.first_k)
#pragma unroll
          for (int e = 0; e < 4; e++) words[(4 * e + part) * cap + j0 + col] = ordered(acc[e]);
      }
      __syncthreads();
    }
    for (int row = wave; row < kSelectRows; row += kSelectWaves) {
      const int32_t i = i0 + row;
      if (i >= a.nbq) break;
      uint8_t* out = a.map + ((int64_t)bh * a.nbq + i) * a.nbk;
      const bool whole = i >= a.first_q;
      if (a.kept_per_row && lane == 0)
        a.kept_per_row[(int64_t)bh * a.nbq + i] = whole ? a.nbk : kept + a.nbk - a.first_k;
      // keys at or above `low` are kept, of those equal to `low` the first `ties`
      uint64_t low = 0;
      int32_t ties = a.nbk;
      const bool search = !whole && kept > 0 && kept < a.first_k;
      const uint64_t* w = words + row * cap;
      uint64_t v[R > 0 ? R : 1];
      if constexpr (R > 0) {
#pragma unroll
        for (int r = 0; r < R; r++) v[r] = search && 64 * r + lane < a.first_k ? w[64 * r + lane] : 0;
      }
      auto count = [&](uint64_t least) {
        int32_t c = 0;
        if constexpr (R > 0) {
#pragma unroll
          for (int r = 0; r < R; r++) c += __builtin_popcountll(__builtin_amdgcn_ballot_w64(v[r] >= least));
        } else {
          for (int32_t j = 0; j < a.first_k; j += 64)
            c += __builtin_popcountll(__builtin_amdgcn_ballot_w64(j + lane < a.first_k && w[j + lane] >= least));
        }
        return c;
      };
      if (search) {
        int32_t c = a.first_k, bit = 63;
        if constexpr (R > 0) {
          // the upper halves first: they nearly always decide, and compare at four times the rate
          for (; bit >= 32 && c != kept; bit--) {
            const uint32_t t = (uint32_t)(low >> 32) | (1u << (bit - 32));
            int32_t ct = 0;
#pragma unroll
            for (int r = 0; r < R; r++) ct += __builtin_popcountll(__builtin_amdgcn_ballot_w64((uint32_t)(v[r] >> 32) >= t));
            if (ct >= kept) {
              low = (uint64_t)t << 32;
              c = ct;
            }
          }
        }
        for (; bit >= 0 && c != kept; bit--) {
          const uint64_t t = low | (1ull << bit);
          const int32_t ct = count(t);
          if (ct >= kept) {
            low = t;
            c = ct;
          }
        }
        // more than `kept` at or above `low`: `low` itself is the score of the last kept and its equals
        ties = c == kept ? a.nbk : kept - count(low + 1);
      }
      auto decide = [&](int32_t j, uint64_t word) {
        bool in = whole || j >= a.first_k;
        const bool mine = !whole && j < a.first_k && (search ? word >= low : kept > 0);
        const bool tie = mine && search && ties < a.nbk && word == low;
        const uint64_t others = __builtin_amdgcn_ballot_w64(tie);
        const int32_t before = __builtin_popcountll(others & ((1ull << lane) - 1));
        in = in || (mine && (!tie || before < ties));
        if (search && ties < a.nbk) ties = max(0, ties - __builtin_popcountll(others));
        if (j < a.nbk) out[j] = in ? 1 : 0;
      };
      if constexpr (R > 0) {
#pragma unroll
        for (int r = 0; r < R; r++) decide(64 * r + lane, v[r]);
        for (int32_t j = 64 * R; j < a.nbk; j += 64) decide(j + lane, 0);     // text
      } else {
        for (int32_t j = 0; j < a.nbk; j += 64)
          decide(j + lane, search && j + lane < a.first_k ? w[j + lane] : 0);
      }
    }
    __syncthreads();                                 // the scores are no longer read
  }
}

}  // namespace

// Score words per lane and row for these key blocks (before the text): 5 or 10 from LDS, 20 through the slab, else none.
// Whole calls, this form and the next: 5 and 10 at 278 blocks (32 heads x 17776, D 64) 63 and 72 us, at 282 (40 x 36000,
// D 128) 192 and 210; 10 and 20 at 591 (40 x 75600, D 128) 460 and 506; 20 and none at 1000 (16 x 64000) 298 and 732.
static int select_regs(int32_t first_k) {
  return first_k <= 64 * 5 ? 5 : first_k <= kSelectLds ? 10 : first_k <= 64 * 20 ? 20 : 0;
}

// Workgroups that have a slab each: two per CU.
constexpr int32_t kSelectGroups = 512;

static int64_t select_items(int32_t n_bh, int32_t nbq) {
  return ((int64_t)n_bh * ((nbq + kSelectRows - 1) / kSelectRows) + kNumQueues - 1) / kNumQueues * kNumQueues;
}

bool select_fits(int32_t n_bh, int32_t n_kv, int32_t nbq, int32_t nbk) {
  return launch_fits((int64_t)n_bh * nbq + (int64_t)n_kv * nbk, 256) && launch_fits(select_items(n_bh, nbq), 64 * kSelectWaves);
}

SelectLayout select_layout(int32_t n_bh, int32_t n_kv, int32_t head_dim, int32_t nbq, int32_t nbk) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  SelectLayout l;
  l.mean_q = 0;
  l.mean_k = up((size_t)n_bh * nbq * head_dim * sizeof(double));
  l.scores = l.mean_k + up((size_t)n_kv * nbk * head_dim * sizeof(double));
  // (sized for every key block: the text may be none)
  const size_t slab = nbk <= kSelectLds ? 0 : (size_t)kSelectGroups * kSelectRows * nbk * sizeof(uint64_t);
  l.total = l.scores + up(slab);
  return l;
}

hipError_t launch_select(const SelectArgs& args, int32_t head_dim, hipStream_t stream) {
  SelectArgs a = args;
  a.q_blocks_all = a.n_bh * a.nbq;
  a.slab = std::max(a.first_k, 1);
  const int32_t items = (int32_t)select_items(a.n_bh, a.nbq);
  const int32_t slabs = std::min(kSelectGroups, items);
  const int32_t bytes = kSelectRows * a.slab * (int32_t)sizeof(uint64_t);
  const dim3 means(a.q_blocks_all + (a.n_bh / a.group) * a.nbk);
  auto go = [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    hipLaunchKernelGGL(psa_block_mean_kernel<D>, means, dim3(256), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    switch (select_regs(a.first_k)) {
      case 5: hipLaunchKernelGGL((psa_select_kernel<D, 5, true>), dim3(items), dim3(64 * kSelectWaves), bytes, stream, a); break;
      case 10: hipLaunchKernelGGL((psa_select_kernel<D, 10, true>), dim3(items), dim3(64 * kSelectWaves), bytes, stream, a); break;
      case 20: hipLaunchKernelGGL((psa_select_kernel<D, 20, false>), dim3(slabs), dim3(64 * kSelectWaves), 0, stream, a); break;
      default: hipLaunchKernelGGL((psa_select_kernel<D, 0, false>), dim3(slabs), dim3(64 * kSelectWaves), 0, stream, a);
    }
    return hipGetLastError();
  };
  return head_dim == 128 ? go(std::integral_constant<int, 128>()) : go(std::integral_constant<int, 64>());
}

}  // namespace psa
