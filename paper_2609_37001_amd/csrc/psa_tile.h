// The per-wave tile engine of the attention kernels: K/V tiles in LDS, S^T = K Q^T, online softmax and
// O^T += V^T P^T on 32 rows per wave (described at the top of psa_kernels.hip).  Device code only.
#pragma once

#include <stdint.h>

#include <type_traits>

#include <hip/hip_runtime.h>

#include "psa.h"

namespace psa {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

#define PSA_LDS __attribute__((address_space(3)))

template <int D, int BLK>
struct Tile {
  static constexpr int kWaves = BLK / 32;      // one wave per 32 query rows
  static constexpr int kThreads = 64 * kWaves;
  static constexpr int KT = BLK / 32;          // 32-key row groups of S^T
  static constexpr int DC = D / 16;            // 16-wide head-dim chunks (Q K^T contraction)
  static constexpr int DT = D / 32;            // 32-row head-dim groups of O^T
  static constexpr int KC = BLK / 16;          // 16-key chunks (P V contraction)
  static constexpr int RB = D * 2;             // LDS bytes per row
  static constexpr int CPR = D / 8;            // 16-byte chunks per row
  static constexpr int BYTES = BLK * RB;       // one K or V block in LDS
  static constexpr int LPW = BYTES / (1024 * kWaves);  // 1 KB DMA slots per wave per tensor
  static_assert(LPW >= 1 && BYTES % (1024 * kWaves) == 0, "tile shape");
};

// XOR swizzle of the 16-byte chunks of LDS row `row` (D = 128: 16 chunks per row).  K reads
// touch the 16 rows {x..x+15} (8 lanes per cycle: rows {x..x+3, x+8..x+11}) at one logical
// chunk; transposed V reads touch 4 consecutive rows r0..r0+3 at 4 consecutive chunks (16 lanes
// per cycle: 2 chunks).  Within a quad of rows, bits (1,2) and bits (2,3) of the swizzle are
// both all distinct; row bits 2 and 3 flip bits 1 and 0.  Every one of these access groups then
// hits distinct banks whether the LDS serves 128 or 256 bytes per clock.  The 8 chunks of D = 64 take
// the low three bits, for which this does not hold: half of its LDS cycles are bank conflicts.
template <int CPR>
__device__ __forceinline__ int swz(int row) {
  const int i = row & 3;
  const int s = (((i >> 1) << 3) | ((i & 1) << 2) | ((i >> 1) << 1)) ^ (((row >> 2) & 1) << 1) ^
                ((row >> 3) & 1);
  return s & (CPR - 1);
}

// Lane l supplies K row sigma(l & 31) of a 32-row group so that accumulator element i of lane l
// holds key 16*(i/8) + 8*(l/32) + (i%8).
__device__ __forceinline__ int key_perm(int r) {
  const int a = r >> 3, hh = (r >> 2) & 1, b = r & 3;
  return 16 * (a >> 1) + 8 * hh + 4 * (a & 1) + b;
}

__device__ __forceinline__ float pair_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float pair_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}


__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(const PSA_LDS void*)p;
}

__device__ __forceinline__ void dma16(uint32_t lds_addr, uint32_t voff, const void* base) {
  // One wait state separates the M0 write from the LDS DMA that reads it.
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(lds_addr), "v"(voff), "s"(base)
               : "memory");
}

// Wait until at most N of this wave's DMA loads are outstanding.
template <int N>
__device__ __forceinline__ void wait_dma() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Per-wave state: 32 query rows (lane l owns row l & 31; lanes l and l^32 split its keys).
// Scores live in the exp2 domain: Q is multiplied by scale*log2(e) once, when it is loaded, and
// the S^T accumulators start at -m instead of 0, so the MFMAs deliver S - m and the softmax needs
// no per-score multiply or subtract.
template <int D, int BLK>
struct WaveState {
  using T = Tile<D, BLK>;
  bf16x8 q[T::DC];     // (scale*log2(e) Q)^T B operands
  f32x16 o[T::DT];     // O^T accumulators
  // -m (0 while m = -inf), the initial S^T accumulators.  Head dim 128 keeps all 16 elements in
  // registers; head dim 64 needs those registers for its four waves per SIMD and broadcasts one
  // (16 moves per step; with 16 kept the block loop spills).
  static constexpr bool kScalarM = D == 64;
  using NegM = typename std::conditional<kScalarM, float, f32x16>::type;
  NegM negm;
  __device__ __forceinline__ f32x16 neg_max() const {
    if constexpr (kScalarM) {
      f32x16 z;
#pragma unroll
      for (int i = 0; i < 16; i++) z[i] = negm;
      return z;
    } else {
      return negm;
    }
  }
  __device__ __forceinline__ float base() const {
    if constexpr (kScalarM) return -negm;
    else return -negm[0];
  }
  __device__ __forceinline__ void set_neg_max(float nb) {
    if constexpr (kScalarM) {
      negm = nb;
    } else {
#pragma unroll
      for (int i = 0; i < 16; i++) negm[i] = nb;
    }
  }
  float m;             // base of the weights: at or near the running max of the scaled scores
  float l;             // running sum of the bf16-rounded P over this lane's keys
};

// A key/value block is processed in steps of HK_ keys (S^T: HK_/32 groups of 32 keys per wave): 64 in
// the pair engine (two halves at block 128, the whole block at block 64), half a block in the split
// engine.  Every step updates the online-softmax statistics on its own.
template <int D, int BLK, int HK_ = 64>
struct Half {
  static constexpr int HK = HK_;              // keys per step
  static constexpr int KT = HK / 32;          // 32-key groups of S^T per half
  static constexpr int KC = HK / 16;          // 16-key chunks per half
};

// S^T = K Q^T for keys [k0, k0 + HK) of the block (K rows from LDS).
template <int D, int BLK, int HK = 64>
__device__ __forceinline__ void qk_half(const WaveState<D, BLK>& st,
                                        f32x16 (&s)[Half<D, BLK, HK>::KT], const uint8_t* sk, int k0,
                                        int lane) {
  using T = Tile<D, BLK>;
  using H = Half<D, BLK, HK>;
  const int h = lane >> 5;
  const int krow0 = k0 + key_perm(lane & 31);
  const int ksw = swz<T::CPR>(krow0);   // identical for krow0 + 32 kt
  // The K operands of step cc + 1 are read while the MFMAs of step cc run.
  bf16x8 a[2][H::KT];
#pragma unroll
  for (int kt = 0; kt < H::KT; kt++)
    a[0][kt] = *(const bf16x8*)(sk + (krow0 + 32 * kt) * T::RB + ((h ^ ksw) << 4));
#pragma unroll
  for (int cc = 0; cc < T::DC; cc++) {
    if (cc + 1 < T::DC) {
#pragma unroll
      for (int kt = 0; kt < H::KT; kt++)
        a[(cc + 1) & 1][kt] =
            *(const bf16x8*)(sk + (krow0 + 32 * kt) * T::RB + (((2 * (cc + 1) + h) ^ ksw) << 4));
    }
    __builtin_amdgcn_sched_barrier(0);      // keep the reads ahead of this step's MFMAs
#pragma unroll
    for (int kt = 0; kt < H::KT; kt++)
      s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[cc & 1][kt], st.q[cc], cc == 0 ? st.neg_max() : s[kt], 0, 0, 0);
  }
}

// Mask (tail: the block reaches past the sequence end), online-softmax statistics, P^T chunk by
// chunk and O^T += V^T P^T, for keys [k0, k0 + HK) of block kb.
//  * The base m of the weights moves only when a weight would exceed 2^8 (then to the row's maximum),
//    at head dim 64 when one reaches 2 (then to 2^6 above the maximum).  Any base is exact up to the
//    rounding of the weights, which is relative.
//  * Accumulator elements 8*(j&1)..+7 of S^T group j/2 are keys 16j + 8h + 0..7: the B operand
//    of 16-key chunk j.
//  * V^T operand: within each 16-lane group, source lane 4r+c reads V[key0 + r][d0 + 4c .. +3];
//    the transpose read hands lane i the four keys key0..key0+3 at head-dim d0 + i.
//  * Masked keys: past the sequence end (one-dimensional blocks: only the last block), or, in
//    the PSABlock-centric layout (PAD), every position whose bit in the tile's validity words
//    (lo: positions 0..63, hi: 64..127) is clear -- 3D padding and the end of the sequence.
//  * FACTOR: the scores are in units of log2 of a weight divided by `factor`, in [1, 2), and so are the base and
//    st.m: a weight is 2^(factor (S - base)).  q then needs scaling by a power of two alone, which rounds nothing,
//    for one multiplication a score.  (The base moves when a score is 4 above it, at head dim 64 when a weight
//    reaches 2, then to 3 above the maximum.)
template <int D, int BLK, bool PAD, int HK = 64, bool FACTOR = false>
__device__ __forceinline__ void softmax_pv_half(WaveState<D, BLK>& st,
                                                f32x16 (&s)[Half<D, BLK, HK>::KT], const uint8_t* sv,
                                                int kb, int k0, int n, bool tail, uint64_t lo,
                                                uint64_t hi, int lane, int& fresh, float factor = 1.0f) {
  using T = Tile<D, BLK>;
  using H = Half<D, BLK, HK>;
  const int h = lane >> 5, g = lane >> 4, j16 = lane & 15;
  auto pow2 = [&](float x) { return __builtin_amdgcn_exp2f(FACTOR ? x * factor : x); };
  if (tail) {
    asm volatile("" ::: "memory");        // keep the mask a branch taken only by partial tiles
    int hh = h;
    if constexpr (D == 64) asm volatile("" : "+v"(hh));       // formed here, not kept in a register
    if constexpr (PAD) {
#pragma unroll
      for (int kt = 0; kt < H::KT; kt++) {
        // This lane's keys of group kt are positions r0 + {0..7, 16..23}: one 64-bit word.
        const int r0 = k0 + 32 * kt + 8 * hh;
        const uint32_t win = (uint32_t)((BLK == 64 || r0 < 64 ? lo : hi) >> (r0 & 63));
#pragma unroll
        for (int i = 0; i < 16; i++)
          if (!((win >> (16 * (i >> 3) + (i & 7))) & 1u)) s[kt][i] = -__builtin_inff();
      }
    } else {
      const int kbase = kb * BLK + k0 + 8 * hh;
#pragma unroll
      for (int kt = 0; kt < H::KT; kt++)
#pragma unroll
        for (int i = 0; i < 16; i++)
          if (kbase + kt * 32 + 16 * (i >> 3) + (i & 7) >= n) s[kt][i] = -__builtin_inff();
    }
  }

  // s holds S - base with base = -negm (m, or 0 before the first kept key).
  // The softmax and its P V form the longest dependent chain of a block; while a wave runs it,
  // it issues ahead of the other wave on its SIMD, whose Q K^T MFMAs fill the gaps (measured:
  // 3 % faster sparse, 2-4 % dense).
  __builtin_amdgcn_s_setprio(1);
  if constexpr (D == 64) {
    // Head dim 64: the weights come first and their bits tell whether the base was too low.  A
    // weight of 2 or more has bit 14 set (bf16, sign 0), so one OR over the packed weights takes
    // the place of the maximum over the scores: 10 instructions instead of 27, of 131 per step,
    // and off the dependent chain between the two products.  Only a step that trips the test, or
    // has a row without a base yet (fresh), finds the maximum; the new base is 2^6 above it, so
    // that later steps rarely trip it again.  bf16 weights keep their relative precision at any
    // base.  Measured 3-4 % faster than the maximum first (878 -> 851 us at 32 heads x 17776
    // tokens); at head dim 128 the same order is equal or up to 4 % slower.
    const int vkey = k0 + 8 * h + (j16 >> 2);
    const int vsw0 = swz<T::CPR>(vkey), vsw1 = swz<T::CPR>(vkey + 4);   // identical for vkey + 16 j
    bf16x8 va[2][T::DT];
    auto read_v = [&](int j) {
#pragma unroll
      for (int dt = 0; dt < T::DT; dt++) {
        const int dd = dt * 32 + 16 * (g & 1) + 4 * (j16 & 3);
        const int lchunk = dd >> 3, inoff = (dd & 7) * 2;
        const uint8_t* a0 = sv + (vkey + 16 * j) * T::RB + ((lchunk ^ vsw0) << 4) + inoff;
        const uint8_t* a1 = sv + (vkey + 16 * j + 4) * T::RB + ((lchunk ^ vsw1) << 4) + inoff;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PSA_LDS s16x4*)a0);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PSA_LDS s16x4*)a1);
        va[j & 1][dt] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      }
    };
    bf16x8 p[H::KC];
    auto weights = [&]() {
#pragma unroll
      for (int j = 0; j < H::KC; j++) {
        f32x8 e;
#pragma unroll
        for (int x = 0; x < 8; x++) e[x] = pow2(s[j >> 1][8 * (j & 1) + x]);
        p[j] = __builtin_convertvector(e, bf16x8);
      }
    };
    const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
    weights();
    uint32_t any = 0;
#pragma unroll
    for (int j = 0; j < H::KC; j++) {
      const u32x4 w = __builtin_bit_cast(u32x4, p[j]);
      any |= w[0] | w[1] | w[2] | w[3];
    }
    if (fresh || __builtin_amdgcn_ballot_w64((any & 0x40004000u) != 0)) {
      asm volatile("" ::: "memory");        // keep this rare path a branch
      float m4[4] = {-__builtin_inff(), -__builtin_inff(), -__builtin_inff(), -__builtin_inff()};
#pragma unroll
      for (int kt = 0; kt < H::KT; kt++)
#pragma unroll
        for (int i = 0; i < 16; i++) m4[i & 3] = fmaxf(m4[i & 3], s[kt][i]);
      const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
      const float base = st.base();
      const float ms = pair_max(mx) + base;
      const bool need = ms > st.m + 0.5f;
      const float up = ms + (FACTOR ? 3.0f : 6.0f);
      const float alpha = need ? pow2(st.m - up) : 1.0f;
      const float shift = need ? up - base : 0.0f;
      st.m = need ? up : st.m;
      st.l *= alpha;
#pragma unroll
      for (int dt = 0; dt < T::DT; dt++) st.o[dt] *= alpha;
#pragma unroll
      for (int kt = 0; kt < H::KT; kt++) s[kt] -= shift;
      st.set_neg_max(st.m == -__builtin_inff() ? 0.0f : -st.m);
      fresh = __builtin_amdgcn_ballot_w64(st.m == -__builtin_inff()) != 0;
      weights();
    }
    read_v(0);
#pragma unroll
    for (int j = 0; j < H::KC; j++) {
      if (j + 1 < H::KC) read_v(j + 1);
      __builtin_amdgcn_sched_barrier(0);      // keep the reads ahead of this chunk's MFMAs
      st.l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p[j], p[j], 0, 1), ones, st.l, false);
      st.l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p[j], p[j], 2, 3), ones, st.l, false);
      st.l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p[j], p[j], 4, 5), ones, st.l, false);
      st.l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p[j], p[j], 6, 7), ones, st.l, false);
#pragma unroll
      for (int dt = 0; dt < T::DT; dt++)
        st.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[j & 1][dt], p[j], st.o[dt], 0, 0, 0);
    }
  } else {
    // Row max as four independent chains, then combined (a short dependent chain).
    float m4[4] = {-__builtin_inff(), -__builtin_inff(), -__builtin_inff(), -__builtin_inff()};
#pragma unroll
    for (int kt = 0; kt < H::KT; kt++)
#pragma unroll
      for (int i = 0; i < 16; i++) m4[i & 3] = fmaxf(m4[i & 3], s[kt][i]);
    const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
    const float base = st.base();
    const float ms = pair_max(mx) + base;
    const bool need = ms - st.m > (FACTOR ? 4.0f : 8.0f);     // false for -inf - -inf (NaN)
    if (__builtin_amdgcn_ballot_w64(need)) {
      asm volatile("" ::: "memory");        // keep this rare path a branch
      const float alpha = need ? pow2(st.m - ms) : 1.0f;
      const float shift = need ? ms - base : 0.0f;
      st.m = need ? ms : st.m;
      st.l *= alpha;
#pragma unroll
      for (int dt = 0; dt < T::DT; dt++) st.o[dt] *= alpha;
#pragma unroll
      for (int kt = 0; kt < H::KT; kt++) s[kt] -= shift;
      const float nb = st.m == -__builtin_inff() ? 0.0f : -st.m;
      st.set_neg_max(nb);
    }

    const int vkey = k0 + 8 * h + (j16 >> 2);
    const int vsw0 = swz<T::CPR>(vkey), vsw1 = swz<T::CPR>(vkey + 4);   // identical for vkey + 16 j
    const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int j = 0; j < H::KC; j++) {
      // The V^T operands of this chunk are read ahead of its exponentials, which hide the LDS
      // latency.
      bf16x8 va[T::DT];
#pragma unroll
      for (int dt = 0; dt < T::DT; dt++) {
        const int dd = dt * 32 + 16 * (g & 1) + 4 * (j16 & 3);
        const int lchunk = dd >> 3, inoff = (dd & 7) * 2;
        const uint8_t* a0 = sv + (vkey + 16 * j) * T::RB + ((lchunk ^ vsw0) << 4) + inoff;
        const uint8_t* a1 = sv + (vkey + 16 * j + 4) * T::RB + ((lchunk ^ vsw1) << 4) + inoff;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PSA_LDS s16x4*)a0);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PSA_LDS s16x4*)a1);
        va[dt] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      }
      __builtin_amdgcn_sched_barrier(0);      // keep the reads ahead of the exponentials
      f32x8 e;
#pragma unroll
      for (int x = 0; x < 8; x++) e[x] = pow2(s[j >> 1][8 * (j & 1) + x]);
      const bf16x8 p = __builtin_convertvector(e, bf16x8);
      // Row sum of the rounded weights, two per instruction: the normaliser matches the P that
      // multiplies V.
      st.l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p, p, 0, 1), ones, st.l, false);
      st.l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p, p, 2, 3), ones, st.l, false);
      st.l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p, p, 4, 5), ones, st.l, false);
      st.l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p, p, 6, 7), ones, st.l, false);
#pragma unroll
      for (int dt = 0; dt < T::DT; dt++)
        st.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[dt], p, st.o[dt], 0, 0, 0);
    }
  }
  __builtin_amdgcn_s_setprio(0);
}

// Direct global->LDS loads of a whole K or V block by the waves of a workgroup: wave w
// loads the 1 KB slots w S .. w S + S - 1.  Slot j covers LDS bytes [1024 j, +1024) of the block;
// lane l writes bytes [1024 j + 16 l, +16): row (64 j + l) / CPR, physical chunk (64 j + l) % CPR,
// which holds logical chunk (physical ^ swz(row)).  The loads are issued from inline assembly (SGPR
// base + 32-bit lane offset, M0 = LDS destination); the compiler does not track them, so every
// consumer first waits with wait_dma<N>() and a barrier.
template <int D, int BLK>
struct DmaPlan {
  using T = Tile<D, BLK>;
  static constexpr int W = 2 * T::kWaves;              // waves of a workgroup
  static constexpr int S = T::BYTES / (1024 * W);      // slots per wave per tensor
  static_assert(S >= 1 && T::BYTES % (1024 * W) == 0, "tile shape");
  uint32_t off[S];
  int wave, lane;

  __device__ __forceinline__ void init(int wave_, int lane_) {
    wave = wave_;
    lane = lane_;
#pragma unroll
    for (int i = 0; i < S; i++) off[i] = offset(i, BLK);
  }

  // Byte offset in the block of the 16 bytes this lane loads for slot i; rows at or past `rows`
  // are clamped to row rows - 1 (their scores are masked).
  __device__ __forceinline__ uint32_t offset(int i, int rows) const {
    int l = lane;
    // Head dim 64 has no registers to keep the addresses of partial blocks in across the block
    // loop: they are formed where they are used.
    if constexpr (D == 64) asm volatile("" : "+v"(l));
    const int p = (wave * S + i) * 64 + l;
    const int row = p / T::CPR;
    const int chunk = (p % T::CPR) ^ swz<T::CPR>(row);
    return (uint32_t)(min(row, rows - 1) * T::RB + chunk * 16);
  }
};

// Loads block kb of one tensor into its LDS buffer.  Rows past the sequence end are clamped to the
// last row: their scores are masked to -inf, so they are never weighted.
template <int D, int BLK>
__device__ __forceinline__ void issue_block(const DmaPlan<D, BLK>& plan, const __bf16* xh,
                                            uint32_t lds, int kb, int n) {
  using P = DmaPlan<D, BLK>;
  kb = __builtin_amdgcn_readfirstlane(kb);
  const int rows = n - kb * BLK;
  const void* base = (const void*)(xh + (size_t)kb * BLK * D);
  const uint32_t l0 = __builtin_amdgcn_readfirstlane(lds + (uint32_t)(plan.wave * P::S) * 1024u);
  if (rows >= BLK) {
#pragma unroll
    for (int i = 0; i < P::S; i++) dma16(l0 + i * 1024u, plan.off[i], base);
  } else {
#pragma unroll
    for (int i = 0; i < P::S; i++) dma16(l0 + i * 1024u, plan.offset(i, rows), base);
  }
}

// O = O^T / l of a finished row block (rows past the end are not stored), LSE if asked.
template <int D, int BLK>
__device__ __forceinline__ void store_rows(const WaveState<D, BLK>& st, __bf16* __restrict__ oh,
                                           float* __restrict__ lseh, int row, int n, int lane) {
  using T = Tile<D, BLK>;
  const int h = lane >> 5;
  const float lsum = pair_sum(st.l);
  const float inv = lsum > 0.0f ? 1.0f / lsum : 0.0f;
  if (row < n) {
    __bf16* dst = oh + (size_t)row * D + 4 * h;
#pragma unroll
    for (int dt = 0; dt < T::DT; dt++)
#pragma unroll
      for (int a = 0; a < 4; a++) {
        const f32x4 v = {st.o[dt][4 * a] * inv, st.o[dt][4 * a + 1] * inv,
                         st.o[dt][4 * a + 2] * inv, st.o[dt][4 * a + 3] * inv};
        *(bf16x4*)(dst + dt * 32 + 8 * a) = __builtin_convertvector(v, bf16x4);
      }
    if (lseh && h == 0)
      lseh[row] = lsum > 0.0f ? (st.m + __builtin_log2f(lsum)) * 0.69314718055994530942f
                              : -__builtin_inff();
  }
}

// The same through LDS: the wave's 32 rows are staged row-major in `stage` (32 x 2D bytes of LDS
// no other wave touches; 16-byte chunks XOR-swizzled by the row), then stored as whole rows, 16
// bytes per lane, so that each store covers 64 x 16 contiguous bytes of O instead of 8 bytes in
// each of 32 rows.  row0 = the wave's first row; lane l holds row row0 + (l & 31).
// (m times `factor`: in log2 units; 1 without a factor.)
template <int D, int BLK, bool FACTOR = false>
__device__ __forceinline__ void store_rows_staged(const WaveState<D, BLK>& st, __bf16* __restrict__ oh,
                                                  float* __restrict__ lseh, int row0, int n, int lane,
                                                  uint32_t stage, float factor = 1.0f) {
  using T = Tile<D, BLK>;
  constexpr int RB = 2 * D;                   // bytes per row
  constexpr int C16 = RB / 16;                // 16-byte chunks per row
  // The lane's addresses are formed here, not hoisted out of the item loop into registers that
  // would stay live across the block loop.
  asm volatile("" : "+v"(lane));
  const int h = lane >> 5, r = lane & 31;
  const float lsum = pair_sum(st.l);
  const float inv = lsum > 0.0f ? 1.0f / lsum : 0.0f;
#pragma unroll
  for (int dt = 0; dt < T::DT; dt++)
#pragma unroll
    for (int a = 0; a < 4; a++) {
      const f32x4 v = {st.o[dt][4 * a] * inv, st.o[dt][4 * a + 1] * inv,
                       st.o[dt][4 * a + 2] * inv, st.o[dt][4 * a + 3] * inv};
      const int chunk = (4 * dt + a) ^ (r & (C16 - 1));        // columns 8 (4 dt + a) + 4 h ...
      *(PSA_LDS bf16x4*)(uintptr_t)(stage + r * RB + chunk * 16 + 8 * h) = __builtin_convertvector(v, bf16x4);
    }
#pragma unroll 2
  for (int j = 0; j < 32 * C16 / 64; j++) {
    const int idx = 64 * j + lane, rr = idx / C16, c = idx % C16;
    const u32x4 val = *(PSA_LDS u32x4*)(uintptr_t)(stage + rr * RB + ((c ^ (rr & (C16 - 1))) * 16));
    if (row0 + rr < n) *(u32x4*)(oh + (size_t)(row0 + rr) * D + 8 * c) = val;
  }
  if (lseh && h == 0 && row0 + r < n)
    lseh[row0 + r] = lsum > 0.0f ? ((FACTOR ? st.m * factor : st.m) + __builtin_log2f(lsum)) * 0.69314718055994530942f
                                 : -__builtin_inff();
}

// Entry i of a pair's block stream: key block in bits 0-12, kept by the first row (bit 13) and
// by the second row (bit 14).
constexpr int kEntryRowShift = 13;
constexpr int kEntryBlockMask = (1 << kEntryRowShift) - 1;
static_assert(PSA_MAX_BLOCKS <= (1 << kEntryRowShift), "block index fits the entry");

// One work item of the pair engine: this wave's row (block of BLK of n_q query rows, -1: none) of one
// (batch, head) and, of n keys, nu stream entries (SPARSE: in `list`; dense: every block, kept by both rows).
// Block i sits in buffer i & 1; after one barrier (its loads, issued a block earlier, have landed
// and block i - 1 is no longer read) the loads of block i + 1 go out and each row that keeps block
// i runs it: Q K^T, softmax and P V for each step of 64 keys.
// FACTOR: c is the power of two (with a sign, or 0) that q is scaled by, `factor` that of the scores, see
// softmax_pv_half.
template <int D, int BLK, int SUB, bool SPARSE, bool PAD, bool FACTOR = false>
__device__ __forceinline__ void process_pair(const DmaPlan<D, BLK>& plan, int grp,
                                             const __bf16* __restrict__ qh,
                                             const __bf16* __restrict__ kh,
                                             const __bf16* __restrict__ vh,
                                             __bf16* __restrict__ oh, float* __restrict__ lseh,
                                             int n_q, int n, int my_row, int nu, int first,
                                             const uint16_t* list, float c,
                                             uint8_t (*sk)[Tile<D, BLK>::BYTES],
                                             uint8_t (*sv)[Tile<D, BLK>::BYTES],
                                             const uint64_t* masks, float factor = 1.0f) {
  using T = Tile<D, BLK>;
  using H = Half<D, BLK>;
  const int tid = threadIdx.x, lane = tid & 63, gw = (tid >> 6) & (T::kWaves - 1);
  const int h = lane >> 5, r32 = lane & 31;
  const int row = my_row * BLK + gw * 32 + r32;

  // Entry i of the stream: list entry first + i, cyclically (SUB = 2: half i % 2 of list entry
  // first + i / 2, kept by both groups).  Dense: block i, kept by both rows, in a word that numbers any
  // number of blocks (its streams can be longer than a list).
  constexpr int kRowShift = SPARSE ? kEntryRowShift : 30;
  auto entry = [&](int i) {
    if constexpr (SPARSE) {
      int j = i / SUB + first;
      const int len = nu / SUB;
      j = j >= len ? j - len : j;
      const int x = (int)__builtin_amdgcn_readfirstlane(list[j]);
      return SUB == 1 ? x : (x & kEntryBlockMask) * SUB + i % SUB;
    } else {
      return (int)((uint32_t)i | (3u << kRowShift));
    }
  };
  auto block_of = [](int x) { return SUB == 1 ? x & ((1 << kRowShift) - 1) : x; };
  // The second half of the sequence's last block may lie past the end altogether; it is loaded
  // from the last half that does not, and masked.
  auto from = [&](int kb) { return SUB == 1 ? kb : min(kb, (n - 1) / BLK); };
  auto issue_k = [&](int buf, int kb) { issue_block<D, BLK>(plan, kh, lds_address(sk[buf]), from(kb), n); };
  auto issue_v = [&](int buf, int kb) { issue_block<D, BLK>(plan, vh, lds_address(sv[buf]), from(kb), n); };
  int e = 0;
  // Sparse: the first block's loads go out before the Q loads, so that the two latencies overlap
  // at the start of the item (dense: after them; the other order measured slower there).
  if constexpr (SPARSE) {
    if (nu > 0) {
      e = entry(0);
      issue_k(0, block_of(e));
      issue_v(0, block_of(e));
    }
  }

  WaveState<D, BLK> st;
  if (my_row >= 0) {
    const bf16x8* src = (const bf16x8*)(qh + (size_t)min(row, n_q - 1) * D) + h;
#pragma unroll
    for (int cc = 0; cc < T::DC; cc++) st.q[cc] = src[2 * cc];
#pragma unroll
    for (int cc = 0; cc < T::DC; cc++)
      st.q[cc] = __builtin_convertvector(__builtin_convertvector(st.q[cc], f32x8) * c, bf16x8);
#pragma unroll
    for (int cc = 0; cc < T::DC; cc++) asm volatile("" ::"v"(st.q[cc]));
  }
  st.m = -__builtin_inff();
  st.l = 0.0f;
  st.set_neg_max(0.0f);
  int fresh = 1;
#pragma unroll
  for (int dt = 0; dt < T::DT; dt++) st.o[dt] = (f32x16){};

  if constexpr (!SPARSE) {
    if (nu > 0) {
      e = entry(0);
      issue_k(0, block_of(e));
      issue_v(0, block_of(e));
    }
  }
  // The validity words of a block (one word per 64 positions) are read when its loads are issued, a block
  // ahead: read where they are needed they put a scalar load into the chain of every block.  Not with
  // SUB = 2, whose four waves per SIMD hide that load and have no registers left.
  uint64_t lo_next = ~0ull, hi_next = ~0ull;
  auto read_masks = [&](int kb) {
    if constexpr (PAD) {
      lo_next = masks[SUB == 1 ? 2 * kb : kb];
      if constexpr (BLK > 64) hi_next = masks[2 * kb + 1];
    }
  };
  if (SUB == 1 && nu > 0) read_masks(block_of(e));
  // Where the loop's instructions lie within the fetch lines moves the dense kernel of head dim 128 by up
  // to 1.5 % (75600 tokens, 40 heads: 98.0 to 99.3 ms over 13 offsets); this is the best one measured.
  if constexpr (!SPARSE && D == 128 && BLK == 128) asm volatile(".p2align 8\n\ts_nop 0\n\ts_nop 0\n\ts_nop 0");
  for (int i = 0; i < nu; i++) {
    const int kb = block_of(e);
    const bool mine = my_row >= 0 && (SUB > 1 || ((e >> (kRowShift + grp)) & 1));
    if constexpr (SUB > 1) read_masks(kb);
    const uint64_t lo = lo_next, hi = hi_next;
    const bool tail = PAD ? (BLK > 64 ? lo & hi : lo) != ~0ull : (kb + 1) * BLK > n;
    wait_dma<0>();                                        // block i, issued a block ago
    __syncthreads();                                      // ... by every wave; block i-1 read
    // The next block's K goes out right after the barrier and its V after this block's first
    // Q K^T half: a wave stalls while it issues, and a single burst of all its loads after the
    // barrier, where every wave issues at once, keeps the MFMA pipes idle for longer (measured:
    // sparse 0.5-1.3 % and dense 0.4-3 % faster on two boxes, same bits).
    const bool more = i + 1 < nu;
    int kbn = 0;
    if (more) {
      e = entry(i + 1);
      kbn = block_of(e);
      if constexpr (SUB == 1) read_masks(kbn);
      issue_k((i + 1) & 1, kbn);
    }
    if (mine) {
      const uint8_t* skb = sk[i & 1];
      const uint8_t* svb = sv[i & 1];
      f32x16 s[H::KT];
      qk_half<D, BLK>(st, s, skb, 0, lane);
      if (more) issue_v((i + 1) & 1, kbn);
      softmax_pv_half<D, BLK, PAD, 64, FACTOR>(st, s, svb, kb, 0, n, tail, lo, hi, lane, fresh, factor);
      if constexpr (BLK > H::HK) {
        qk_half<D, BLK>(st, s, skb, H::HK, lane);
        softmax_pv_half<D, BLK, PAD, 64, FACTOR>(st, s, svb, kb, H::HK, n, tail, lo, hi, lane, fresh, factor);
      }
    } else if (more) {
      issue_v((i + 1) & 1, kbn);
    }
  }
  if constexpr (SPARSE) {
    // The buffer of block nu - 2 (every wave passed the barrier of block nu - 1) stages the
    // output: 8 KB per wave, K half for group 0, V half for group 1.
    if (my_row >= 0) {
      static_assert(T::kWaves * 32 * 2 * D <= T::BYTES, "a wave's rows fit its share of a free buffer");
      const uint32_t stage = lds_address(grp == 0 ? sk[nu & 1] : sv[nu & 1]) + gw * (32 * 2 * D);
      store_rows_staged<D, BLK, FACTOR>(st, oh, lseh, my_row * BLK + gw * 32, n_q, lane, stage, factor);
    }
  } else {
    if (my_row >= 0) store_rows<D, BLK>(st, oh, lseh, row, n_q, lane);
  }
}


}  // namespace psa
