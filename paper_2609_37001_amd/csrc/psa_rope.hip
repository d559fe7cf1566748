// Norms of queries and keys per head with the rotation by (t, h, w) positions, forward and backward: HIP
// kernels for gfx950.
//
//   n = x r w with r = 1 / sqrt(mean(x^2) + eps), the mean over the channels of one head
//   y = R n, R turning channel pair j of an axis of d_a channels by pos_a theta^(-2j / d_a)
//   backward: g = R^T dy, t = g w, dx = r (t - x r^2 mean(t x)), dw = sum of g x r over all rows
//
// Both directions read and write each tensor once and are bound by HBM.  A row (token, head) is D / 8
// lanes of eight channels, so a row's sums are DPP steps inside a 16-lane row, and every access is 16
// bytes a lane.  A workgroup takes a tile of tokens and walks over the heads of one tensor: the angles of
// a token depend on its position alone, so their sines are taken once per lane and serve all of them.
// The input keeps the projection's strides; the output is the attention's [batch][head][token][channel],
// so the pass is the transposition as well.  Measured, queries and keys of D 128 in bf16: 24 heads x 119056 with the
// norm, slices of a fused projection, 567 us (5.16 TB/s read and written, as a plain copy); 40 x 75600 without it 604
// (5.13); the gradients of 12 x 32760 126 (4.8).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "psa_launch.h"
#include "psa_tile.h"

namespace psa {
namespace {

constexpr int kRopeThreads = 256;

__device__ __forceinline__ f32x8 load8(const __bf16* p) {
  return __builtin_convertvector(*(const bf16x8*)p, f32x8);
}
__device__ __forceinline__ f32x8 load8(const float* p) {
  const f32x4 a = ((const f32x4*)p)[0], b = ((const f32x4*)p)[1];
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ void store8(__bf16* p, f32x8 v) { *(bf16x8*)p = __builtin_convertvector(v, bf16x8); }
__device__ __forceinline__ void store8(float* p, f32x8 v) {
  ((f32x4*)p)[0] = __builtin_shufflevector(v, v, 0, 1, 2, 3);
  ((f32x4*)p)[1] = __builtin_shufflevector(v, v, 4, 5, 6, 7);
}

// Eight channels of a norm's weight (all ones without one).
__device__ __forceinline__ f32x8 load_weight(const float* w, int chunk) {
  const f32x8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
  if (!w) return ones;
  f32x8 v;
#pragma unroll
  for (int e = 0; e < 8; e++) v[e] = w[8 * chunk + e];      // (any four-byte alignment)
  return v;
}

// Sum over the L = 8 or 16 lanes of a row, in every one of them.
template <int L>
__device__ __forceinline__ float row_sum(float x) {
  auto step = [](float v, auto ctrl) {
    return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, false));
  };
  x = step(x, std::integral_constant<int, 0xb1>());        // quad_perm 1,0,3,2
  x = step(x, std::integral_constant<int, 0x4e>());        // quad_perm 2,3,0,1
  x = step(x, std::integral_constant<int, 0x141>());       // row_half_mirror: lanes l, 7 - l
  if constexpr (L == 16) x = step(x, std::integral_constant<int, 0x140>());   // row_mirror: lanes l, 15 - l
  return x;
}

// The angles of this lane's channels: pairs (2j, 2j + 1), four of them, or (HALVES) eight channels of one
// half of the head, whose partners are the same lane's of the other half.
template <int D, bool HALVES>
struct Turn {
  static constexpr int P = HALVES ? 8 : 4;
  float cos[P], sin[P];

  // Angles in turns, in 64 bits until the whole turns are gone: a position of 2^20 at full speed leaves
  // 32 bits four digits.
  __device__ __forceinline__ void at(const RopeArgs& a, int32_t token, int chunk) {
    int32_t pos[3] = {0, 0, 0};
    const bool video = token < a.n_video;
    if (video) {
      pos[0] = token / a.hw;
      const int32_t s = token - pos[0] * a.hw;
      pos[1] = s / a.width;
      pos[2] = s - pos[1] * a.width;
      pos[0] += a.origin[0];
      pos[1] += a.origin[1];
      pos[2] += a.origin[2];
    }
    const int j0 = HALVES ? 8 * chunk & (D / 2 - 1) : 4 * chunk;
#pragma unroll
    for (int e = 0; e < P; e++) {
      const int j = j0 + e;
      const double p = (double)(j < a.end[0] ? pos[0] : j < a.end[1] ? pos[1] : pos[2]);
      const double t = p * a.turns[j];
      sincospif(2.0f * (float)(t - rint(t)), &sin[e], &cos[e]);
    }
  }

  // R v, or R^T v (BACK).
  template <bool BACK>
  __device__ __forceinline__ f32x8 apply(f32x8 v, int chunk) const {
    f32x8 y;
    if constexpr (HALVES) {
      // The lane of the other half: lanes of a row are consecutive, halves D / 16 lanes apart.
      const bool upper = chunk >= D / 16;
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const float o = __uint_as_float(
            D == 128 ? __builtin_amdgcn_update_dpp(0, __float_as_uint(v[e]), 0x128, 0xf, 0xf, false)      // row_ror:8
                     : __builtin_amdgcn_ds_swizzle(__float_as_uint(v[e]), 0x101f));                        // lane ^ 4
        const float s = upper != BACK ? sin[e] : -sin[e];
        y[e] = v[e] * cos[e] + o * s;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const float s = BACK ? -sin[e] : sin[e];
        y[2 * e] = v[2 * e] * cos[e] - v[2 * e + 1] * s;
        y[2 * e + 1] = v[2 * e] * s + v[2 * e + 1] * cos[e];
      }
    }
    return y;
  }
};

// Where a workgroup's lanes stand: `wide` tokens of a tile side by side (a power of two), the other row
// places on other heads.
struct RopePlace {
  int chunk;
  int32_t token, head, step;
  __device__ __forceinline__ RopePlace(int cpr, const RopeArgs& a, int32_t tile) {
    const int g = threadIdx.x / cpr;
    chunk = threadIdx.x % cpr;
    token = tile * a.wide + (g & (a.wide - 1));
    head = g / a.wide;
    step = kRopeThreads / cpr / a.wide;
  }
};

// Rows in flight per lane.
constexpr int kRopeRows = 4;

template <typename X, int D, bool NORM, bool HALVES>
__global__ __launch_bounds__(kRopeThreads) void psa_norm_rope_kernel(RopeArgs a) {
  constexpr int L = D / 8, U = kRopeRows;
  const RopeTensor& ts = a.t[blockIdx.z % a.n_tensors];
  const int32_t b = blockIdx.z / a.n_tensors;
  const RopePlace at(L, a, blockIdx.x);
  // heads of this workgroup
  const int32_t h0 = blockIdx.y * a.heads_per_group, h1 = min(ts.n_heads, h0 + a.heads_per_group);
  if (h0 >= h1) return;
  const bool live = at.token < a.n;
  const int32_t token = min(at.token, a.n - 1);
  const X* x = (const X*)ts.x + b * ts.stride_b + token * ts.stride_n + 8 * at.chunk;
  __bf16* y = (__bf16*)ts.y + ((int64_t)b * ts.n_heads * a.n + token) * D + 8 * at.chunk;
  f32x8 w;
  if constexpr (NORM) w = load_weight(ts.weight, at.chunk);
  Turn<D, HALVES> turn;
  turn.at(a, token, at.chunk);
  for (int32_t h = h0 + at.head; h < h1; h += U * at.step) {
    f32x8 v[U];
#pragma unroll
    for (int u = 0; u < U; u++) v[u] = load8(x + min(h + u * at.step, h1 - 1) * ts.stride_h);
#pragma unroll
    for (int u = 0; u < U; u++) {
      if constexpr (NORM) {
        float ss = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; e++) ss = fmaf(v[u][e], v[u][e], ss);
        const float r = rsqrtf(row_sum<L>(ss) * (1.0f / D) + a.eps);
        v[u] = v[u] * r * w;
      }
      v[u] = turn.template apply<false>(v[u], at.chunk);
      if (live && h + u * at.step < h1) store8(y + (int64_t)(h + u * at.step) * a.n * D, v[u]);
    }
  }
}

// Backward.  A workgroup walks over token tiles, so that the partial sums of the weights' gradients are few:
// each lane sums its eight channels over its rows, the workgroup's rows are added through LDS, and
// psa_norm_rope_dw_kernel adds the workgroups, all in a fixed order.
template <typename X, int D, bool NORM, bool HALVES>
__global__ __launch_bounds__(kRopeThreads) void psa_norm_rope_bwd_kernel(RopeArgs a) {
  constexpr int L = D / 8, U = NORM ? 2 : kRopeRows, G = kRopeThreads / L;
  const int which = blockIdx.z % a.n_tensors;
  const RopeTensor& ts = a.t[which];
  const int32_t b = blockIdx.z / a.n_tensors;
  const int32_t h0 = blockIdx.y * a.heads_per_group, h1 = min(ts.n_heads, h0 + a.heads_per_group);
  const int chunk = threadIdx.x % L;
  f32x8 w = {}, dw = {};
  if constexpr (NORM) w = load_weight(ts.weight, chunk);
  for (int32_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const RopePlace at(L, a, tile);
    const bool live = at.token < a.n;
    const int32_t token = min(at.token, a.n - 1);
    const X* x = (const X*)ts.x + b * ts.stride_b + token * ts.stride_n + 8 * chunk;
    X* dx = (X*)ts.dx + b * ts.dx_stride_b + token * ts.dx_stride_n + 8 * chunk;
    const __bf16* dy = (const __bf16*)ts.dy + ((int64_t)b * ts.n_heads * a.n + token) * D + 8 * chunk;
    Turn<D, HALVES> turn;
    turn.at(a, token, chunk);
    for (int32_t h = h0 + at.head; h < h1; h += U * at.step) {
      f32x8 v[U], g[U];
#pragma unroll
      for (int u = 0; u < U; u++) {
        const int32_t hu = min(h + u * at.step, h1 - 1);
        g[u] = load8(dy + (int64_t)hu * a.n * D);
        if constexpr (NORM) v[u] = load8(x + hu * ts.stride_h);
      }
#pragma unroll
      for (int u = 0; u < U; u++) {
        const bool here = live && h + u * at.step < h1;
        g[u] = turn.template apply<true>(g[u], chunk);
        if constexpr (NORM) {
          const f32x8 t = g[u] * w;
          float ss = 0.0f, tx = 0.0f;
#pragma unroll
          for (int e = 0; e < 8; e++) {
            ss = fmaf(v[u][e], v[u][e], ss);
            tx = fmaf(t[e], v[u][e], tx);
          }
          const float r = rsqrtf(row_sum<L>(ss) * (1.0f / D) + a.eps);
          const float m = row_sum<L>(tx) * (1.0f / D) * r * r;
          // a row that is not this lane's (a place behind the last token or head) adds nothing
          if (here) dw += g[u] * v[u] * r;
          g[u] = (t - v[u] * m) * r;
        }
        if (here) store8(dx + (h + u * at.step) * ts.dx_stride_h, g[u]);
      }
    }
  }
  if constexpr (NORM) {
    __shared__ float part[G][D];
    store8(&part[threadIdx.x / L][8 * chunk], dw);
    __syncthreads();
    if (threadIdx.x < D) {
      float s = 0.0f;
#pragma unroll
      for (int g = 0; g < G; g++) s += part[g][threadIdx.x];
      const int64_t group = ((int64_t)which * a.batch + b) * gridDim.y * gridDim.x + (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
      a.partial[group * D + threadIdx.x] = s;
    }
  }
}

// dw of a tensor: the workgroups' partial sums in 64 bits, `rows` of them, 16 channels per workgroup.
__global__ __launch_bounds__(256) void psa_norm_rope_dw_kernel(const float* __restrict__ partial, int32_t rows,
                                                               int32_t d, float* __restrict__ dw0,
                                                               float* __restrict__ dw1) {
  __shared__ double part[16][17];
  const int c = threadIdx.x & 15, k = threadIdx.x >> 4;
  const float* p = partial + (int64_t)blockIdx.y * rows * d + blockIdx.x * 16 + c;
  double s = 0.0;
#pragma unroll 8
  for (int32_t i = k; i < rows; i += 16) s += (double)p[(int64_t)i * d];
  part[k][c] = s;
  __syncthreads();
  if (k == 0) {
    double t = 0.0;
#pragma unroll
    for (int i = 0; i < 16; i++) t += part[i][c];
    (blockIdx.y == 0 ? dw0 : dw1)[blockIdx.x * 16 + c] = (float)t;
  }
}

template <typename F>
void by_form(bool f32, int32_t d, bool norm, bool halves, F f) {
  auto dim = [&](auto x, auto n, auto hv) {
    if (d == 128)
      f(x, std::integral_constant<int, 128>(), n, hv);
    else
      f(x, std::integral_constant<int, 64>(), n, hv);
  };
  auto type = [&](auto n, auto hv) {
    if (f32)
      dim(0.0f, n, hv);
    else
      dim((__bf16)0.0f, n, hv);
  };
  using T = std::true_type;
  using N = std::false_type;
  if (norm)
    halves ? type(T(), T()) : type(T(), N());
  else
    halves ? type(N(), T()) : type(N(), N());
}

}  // namespace

// Tiles, and how many heads a workgroup walks over: as many as leave `groups` workgroups, so that a short
// sequence still spreads over the chip.
static void rope_split(RopeArgs& a, int32_t d, int32_t groups, int32_t* head_groups) {
  const int32_t rows = kRopeThreads / (d / 8);
  a.wide = 1;
  while (a.wide < rows && a.wide < a.n) a.wide *= 2;
  a.tiles = (a.n - 1) / a.wide + 1;
  int32_t heads = 0;
  for (int32_t i = 0; i < a.n_tensors; i++) heads = std::max(heads, a.t[i].n_heads);
  const int32_t step = rows / a.wide;                                     // heads side by side
  const int64_t have = (int64_t)a.tiles * a.batch * a.n_tensors;
  const int32_t want = (int32_t)std::max<int64_t>(1, std::min<int64_t>((heads + step - 1) / step, groups / have));
  a.heads_per_group = ((heads + want - 1) / want + step - 1) / step * step;
  *head_groups = (heads - 1) / a.heads_per_group + 1;
}

// Workgroups that a launch aims at: eight of four waves on each of 256 CUs.  Fewer start fewer waves than hide the
// latency, more form a token's sines more often: with 512, 2048 and 8192 of them 40 heads x 1560 tokens take 14.3,
// 13.3 and 23.5 us, the gradients of 12 heads x 32760 124, 126 and 139.
constexpr int32_t kRopeGroups = 2048;

bool rope_fits(int32_t n, int32_t d) {
  const int32_t rows = kRopeThreads / (d / 8);
  return launch_fits(((int64_t)n + rows - 1) / rows, kRopeThreads);
}

int64_t rope_partial_rows(RopeArgs a, int32_t d) {
  int32_t hg;
  rope_split(a, d, kRopeGroups, &hg);
  const int32_t per = std::max(1, kRopeGroups / (a.batch * a.n_tensors * hg));
  return (int64_t)a.batch * hg * std::min(a.tiles, per);
}

hipError_t launch_norm_rope(const RopeArgs& args, int32_t d, bool f32, bool norm, bool halves, hipStream_t stream) {
  RopeArgs a = args;
  int32_t hg;
  rope_split(a, d, kRopeGroups, &hg);
  by_form(f32, d, norm, halves, [&](auto x, auto dim, auto n, auto hv) {
    hipLaunchKernelGGL((psa_norm_rope_kernel<decltype(x), decltype(dim)::value, decltype(n)::value, decltype(hv)::value>),
                       dim3(a.tiles, hg, a.batch * a.n_tensors), dim3(kRopeThreads), 0, stream, a);
  });
  return hipGetLastError();
}

hipError_t launch_norm_rope_bwd(const RopeArgs& args, int32_t d, bool f32, bool norm, bool halves, float* dw0,
                                float* dw1, hipStream_t stream) {
  RopeArgs a = args;
  int32_t hg;
  rope_split(a, d, kRopeGroups, &hg);
  const int32_t rows = (int32_t)rope_partial_rows(args, d);
  by_form(f32, d, norm, halves, [&](auto x, auto dim, auto n, auto hv) {
    hipLaunchKernelGGL((psa_norm_rope_bwd_kernel<decltype(x), decltype(dim)::value, decltype(n)::value, decltype(hv)::value>),
                       dim3(rows / (a.batch * hg), hg, a.batch * a.n_tensors), dim3(kRopeThreads), 0, stream, a);
  });
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !norm) return e;
  hipLaunchKernelGGL(psa_norm_rope_dw_kernel, dim3(d / 16, a.n_tensors), dim3(256), 0, stream, a.partial, rows, d, dw0,
                     dw1);
  return hipGetLastError();
}

}  // namespace psa
