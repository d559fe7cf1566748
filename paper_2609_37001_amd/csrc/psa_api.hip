// C ABI of libpsa (declared in include/psa.h): argument validation, workspace layout and
// kernel dispatch.  All device work lives in psa_kernels.hip.
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <cmath>
#include <utility>

#include "psa_launch.h"
#include "psa_map.h"

namespace {

thread_local char g_error[512] = "";

psa_status_t fail(psa_status_t status, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_error, sizeof(g_error), fmt, ap);
  va_end(ap);
  return status;
}

// Restores the thread's error detail when it goes out of scope.
struct SavedError {
  char text[sizeof(g_error)];
  SavedError() { memcpy(text, g_error, sizeof(text)); }
  ~SavedError() { memcpy(g_error, text, sizeof(text)); }
};

psa_status_t hip_fail(hipError_t e, const char* what) {
  return fail(PSA_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// Token and block counts of a grid; false if the grid is invalid or too large for int32 indices.
bool grid_geometry(psa_grid_t grid, int32_t block, psa::Geometry* g) {
  if (grid.frames < 1 || grid.height < 1 || grid.width < 1 || grid.n_text < 0 || block < 1)
    return false;
  const int64_t hw = (int64_t)grid.height * grid.width;
  if (hw >= ((int64_t)1 << 31)) return false;             // (times the frames it may not fit 64 bits)
  const int64_t n_video = hw * grid.frames;
  const int64_t n = n_video + grid.n_text;
  if (n + 2 * (int64_t)block >= ((int64_t)1 << 31)) return false;
  *g = psa::Geometry{};
  g->hw = (int32_t)hw;
  g->n_video = (int32_t)n_video;
  g->n = (int32_t)n;
  g->n_text = grid.n_text;
  g->block = block;
  g->nb = (int32_t)((n + block - 1) / block);
  g->frames = grid.frames;
  g->height = grid.height;
  g->width = grid.width;
  return true;
}

// Geometry of the PSABlock-centric layout (3D padding, Sec. 3.2) cut into tiles of `tile`
// positions; tile = 0 only sizes the layout (PSABlock-level maps).
psa_status_t geometry_3d(psa_grid_t grid, psa_block3d_t pb, int32_t tile, psa::Geometry* g) {
  if (grid.frames < 1 || grid.height < 1 || grid.width < 1 || grid.n_text < 0)
    return fail(PSA_ERR_INVALID, "invalid grid (%d x %d x %d + %d text)", grid.frames, grid.height,
                grid.width, grid.n_text);
  if (pb.t < 1 || pb.h < 1 || pb.w < 1)
    return fail(PSA_ERR_INVALID, "PSABlock sizes must be >= 1 (got %d x %d x %d)", pb.t, pb.h, pb.w);
  const int64_t tp = (grid.frames + (int64_t)pb.t - 1) / pb.t;
  const int64_t hp = (grid.height + (int64_t)pb.h - 1) / pb.h;
  const int64_t wp = (grid.width + (int64_t)pb.w - 1) / pb.w;
  const int64_t vol = (int64_t)pb.t * pb.h * pb.w;
  const int64_t n_blk = tp * hp * wp * vol;
  const int64_t n = n_blk + grid.n_text;
  const int64_t n_video = (int64_t)grid.frames * grid.height * grid.width;
  if (vol >= ((int64_t)1 << 31) || n + 256 >= ((int64_t)1 << 31) || n_video + grid.n_text + 256 >= ((int64_t)1 << 31))
    return fail(PSA_ERR_UNSUPPORTED, "PSABlock layout of %lld tokens is too large", (long long)n);
  if (tile != 0 && vol % tile != 0)
    return fail(PSA_ERR_UNSUPPORTED, "a PSABlock of %lld tokens is not a whole number of %d-token tiles",
                (long long)vol, tile);
  *g = psa::Geometry{};
  g->hw = grid.height * grid.width;
  g->n_video = (int32_t)n_video;
  g->n = (int32_t)n;
  g->n_text = grid.n_text;
  g->block = tile;
  g->nb = tile ? (int32_t)((n + tile - 1) / tile) : 0;
  g->frames = grid.frames;
  g->height = grid.height;
  g->width = grid.width;
  g->pbt = pb.t;
  g->pbh = pb.h;
  g->pbw = pb.w;
  g->tp = (int32_t)tp;
  g->hp = (int32_t)hp;
  g->wp = (int32_t)wp;
  g->n_blk = (int32_t)n_blk;
  return PSA_OK;
}

// Alignment of a device pointer (NULL passes: optional outputs are checked for presence
// separately).
bool aligned(const void* p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// The tensors of an attention call: q, k, v and o present and 16-byte aligned (the kernels load
// and store 16-byte vectors), lse (optional) 4-byte aligned.
psa_status_t check_tensors(const void* q, const void* k, const void* v, const void* o,
                           const float* lse) {
  if (!q || !k || !v || !o) return fail(PSA_ERR_INVALID, "q, k, v and o must be non-NULL");
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(o, 16))
    return fail(PSA_ERR_INVALID, "q, k, v and o must be 16-byte aligned (%p %p %p %p)", q, k, v, o);
  if (!aligned(lse, 4)) return fail(PSA_ERR_INVALID, "lse must be 4-byte aligned (%p)", (const void*)lse);
  return PSA_OK;
}

// Optional count outputs of the map and plan calls.
psa_status_t check_counts_out(const int32_t* per_row, const int64_t* per_head) {
  if (!aligned(per_row, 4)) return fail(PSA_ERR_INVALID, "kept_per_row must be 4-byte aligned");
  if (!aligned(per_head, 8)) return fail(PSA_ERR_INVALID, "kept_per_head must be 8-byte aligned");
  return PSA_OK;
}

psa_status_t check_params(const psa_stripe_t* params, int32_t n_heads) {
  if (!params) return fail(PSA_ERR_INVALID, "params is NULL");
  if (n_heads < 1) return fail(PSA_ERR_INVALID, "n_heads must be >= 1 (got %d)", n_heads);
  for (int32_t h = 0; h < n_heads; h++) {
    const psa_stripe_t& m = params[h];
    if (m.t_w < 1 || m.s_w < 1)
      return fail(PSA_ERR_INVALID, "head %d: widths must be >= 1 (T_w=%d, S_w=%d)", h, m.t_w, m.s_w);
    if (m.t_s < 1 || m.s_s < 1)
      return fail(PSA_ERR_INVALID, "head %d: strides must be >= 1 (T_s=%d, S_s=%d)", h, m.t_s, m.s_s);
    if (m.t_o > PSA_MAX_OFFSET || m.t_o < -PSA_MAX_OFFSET || m.s_o > PSA_MAX_OFFSET ||
        m.s_o < -PSA_MAX_OFFSET)
      return fail(PSA_ERR_INVALID, "head %d: |offset| must be <= %d", h, PSA_MAX_OFFSET);
  }
  return PSA_OK;
}

psa::ParamChunk chunk_of(const psa_stripe_t* params, int32_t head0, int32_t n_heads) {
  psa::ParamChunk pc;
  pc.n = std::min(psa::kHeadsPerChunk, n_heads - head0);
  for (int32_t i = 0; i < psa::kHeadsPerChunk; i++) pc.m[i] = i < pc.n ? params[head0 + i] : params[head0];
  return pc;
}

psa_status_t check_attention_shape(int32_t batch, int32_t n_heads, int32_t head_dim,
                                   int32_t block) {
  if (batch < 1) return fail(PSA_ERR_INVALID, "batch must be >= 1 (got %d)", batch);
  if (n_heads < 1) return fail(PSA_ERR_INVALID, "n_heads must be >= 1 (got %d)", n_heads);
  if (head_dim != 64 && head_dim != 128)
    return fail(PSA_ERR_UNSUPPORTED, "head_dim must be 64 or 128 (got %d)", head_dim);
  if (block != 64 && block != 128)
    return fail(PSA_ERR_UNSUPPORTED, "block must be 64 or 128 (got %d)", block);
  return PSA_OK;
}

// Limits of the scheduler, shared by the plans and runs of both layouts.
psa_status_t check_limits(int32_t batch, int32_t n_heads, const psa::Geometry* g) {
  if (g->nb > PSA_MAX_BLOCKS)
    return fail(PSA_ERR_UNSUPPORTED, "%d blocks per sequence exceed %d", g->nb, PSA_MAX_BLOCKS);
  if ((int64_t)batch * n_heads > PSA_MAX_BATCH_HEADS)
    return fail(PSA_ERR_UNSUPPORTED, "batch*n_heads = %lld exceeds %d", (long long)batch * n_heads,
                PSA_MAX_BATCH_HEADS);
  if ((int64_t)batch * n_heads * g->nb >= ((int64_t)1 << 31))
    return fail(PSA_ERR_UNSUPPORTED, "too many work items");
  return PSA_OK;
}

// Limits of the scheduler and the workspace, shared by the plans and runs of both layouts.
psa_status_t check_work(int32_t batch, int32_t n_heads, const void* workspace,
                        size_t workspace_bytes, const psa::Geometry* g, psa::WorkspaceLayout* wl) {
  const psa_status_t s = check_limits(batch, n_heads, g);
  if (s != PSA_OK) return s;
  *wl = psa::workspace_layout(batch, n_heads, g->nb, g->pbt > 0);
  if (!workspace || workspace_bytes < wl->total)
    return fail(PSA_ERR_WORKSPACE, "workspace of %zu bytes at %p; %zu bytes required", workspace_bytes,
                workspace, wl->total);
  if (((uintptr_t)workspace & 255) != 0)
    return fail(PSA_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  return PSA_OK;
}

psa_status_t check_counts(int32_t batch, int32_t n_heads) {
  if (batch < 1) return fail(PSA_ERR_INVALID, "batch must be >= 1 (got %d)", batch);
  if (n_heads < 1) return fail(PSA_ERR_INVALID, "n_heads must be >= 1 (got %d)", n_heads);
  return PSA_OK;
}

// Sizes shared by the plan and the run of one-dimensional blocks.
psa_status_t check_plan(int32_t batch, int32_t n_heads, psa_grid_t grid, int32_t block,
                        const void* workspace, size_t workspace_bytes, psa::Geometry* g,
                        psa::WorkspaceLayout* wl) {
  psa_status_t s = check_counts(batch, n_heads);
  if (s != PSA_OK) return s;
  if (block != 64 && block != 128)
    return fail(PSA_ERR_UNSUPPORTED, "block must be 64 or 128 (got %d)", block);
  if (!grid_geometry(grid, block, g))
    return fail(PSA_ERR_INVALID, "invalid grid (%d x %d x %d + %d text)", grid.frames, grid.height,
                grid.width, grid.n_text);
  return check_work(batch, n_heads, workspace, workspace_bytes, g, wl);
}

// Sizes shared by the plan and the run of the PSABlock-centric layout.
psa_status_t check_plan_3d(int32_t batch, int32_t n_heads, psa_grid_t grid, psa_block3d_t pb,
                           int32_t tile, const void* workspace, size_t workspace_bytes,
                           psa::Geometry* g, psa::WorkspaceLayout* wl) {
  psa_status_t s = check_counts(batch, n_heads);
  if (s != PSA_OK) return s;
  if (tile != 64 && tile != 128)
    return fail(PSA_ERR_UNSUPPORTED, "tile must be 64 or 128 (got %d)", tile);
  s = geometry_3d(grid, pb, tile, g);
  if (s != PSA_OK) return s;
  return check_work(batch, n_heads, workspace, workspace_bytes, g, wl);
}

// The kernels of a plan over geometry g.
psa_status_t enqueue_plan(int32_t batch, int32_t n_heads, const psa::Geometry& g,
                          const psa_stripe_t* params, void* workspace,
                          const psa::WorkspaceLayout& wl, int32_t* kept_per_row,
                          hipStream_t stream, const char* who) {
  psa::ParamChunk chunks[(PSA_MAX_BATCH_HEADS + psa::kHeadsPerChunk - 1) / psa::kHeadsPerChunk];
  for (int32_t h0 = 0; h0 < n_heads; h0 += psa::kHeadsPerChunk)
    chunks[h0 / psa::kHeadsPerChunk] = chunk_of(params, h0, n_heads);
  const hipError_t e = psa::launch_plan(chunks, g, batch, n_heads, psa::plan_full(g, params, n_heads), workspace, wl,
                                         kept_per_row, stream);
  return e == hipSuccess ? PSA_OK : hip_fail(e, who);
}

psa_status_t check_layout_args(const void* a, const void* b, int32_t n_bh, int32_t head_dim) {
  if (!a || !b) return fail(PSA_ERR_INVALID, "tensors must be non-NULL");
  if (!aligned(a, 16) || !aligned(b, 16))
    return fail(PSA_ERR_INVALID, "tensors must be 16-byte aligned (%p %p)", a, b);
  if (n_bh < 1) return fail(PSA_ERR_INVALID, "batch_heads must be >= 1 (got %d)", n_bh);
  if (n_bh > 65535) return fail(PSA_ERR_UNSUPPORTED, "batch_heads must be <= 65535 (got %d)", n_bh);
  if (head_dim != 64 && head_dim != 128)
    return fail(PSA_ERR_UNSUPPORTED, "head_dim must be 64 or 128 (got %d)", head_dim);
  return PSA_OK;
}

// Compute units of the current device: the persistent grids are sized by them.
int32_t compute_units() {
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 128;
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus < 1)
    return 128;
  return cus;
}

// The run of a plan; right after the plan's own kernels `params` are the plan's, else null.
psa_status_t run_planned(const void* q, const void* k, const void* v, void* o, int32_t batch,
                         int32_t n_heads, int32_t head_dim, psa_grid_t grid, int32_t block,
                         float softmax_scale, void* workspace, size_t workspace_bytes, float* lse,
                         hipStream_t stream, const psa_stripe_t* params) {
  psa_status_t s = check_tensors(q, k, v, o, lse);
  if (s != PSA_OK) return s;
  s = check_attention_shape(batch, n_heads, head_dim, block);
  if (s != PSA_OK) return s;
  psa::Geometry g;
  psa::WorkspaceLayout wl;
  s = check_plan(batch, n_heads, grid, block, workspace, workspace_bytes, &g, &wl);
  if (s != PSA_OK) return s;
  const float c = softmax_scale * 1.4426950408889634f;
  hipError_t e = psa::launch_sparse(q, k, v, o, lse, batch, n_heads, head_dim, g, c, workspace, wl,
                                    compute_units(), stream,
                                    params ? (int32_t)psa::plan_full(g, params, n_heads) : -1);
  if (e != hipSuccess) return hip_fail(e, "psa_attention_run kernel launch");
  return PSA_OK;
}

constexpr int32_t kMaxRowHeads = 1 << 30;     // (the kernels step over the heads in 32 bits)

// Whether no two rows share memory: of the axes with more than one place, in the order of their strides, each
// steps over all that the smaller ones reach.
bool rows_apart(const psa_rows_t& r, int32_t batch, int64_t n, int32_t head_dim) {
  std::pair<int64_t, int64_t> axes[3] = {{r.stride_b, batch}, {r.stride_h, r.n_heads}, {r.stride_n, n}};
  std::sort(axes, axes + 3);
  __int128 reach = head_dim;
  for (const auto& a : axes) {
    if (a.second == 1) continue;
    if (a.first < reach) return false;
    reach += (__int128)a.first * (a.second - 1);
  }
  return true;
}

// One tensor of a norm-and-rotation call.  write: the rows are an output.
psa_status_t check_rows(const psa_rows_t& r, const char* what, int32_t batch, int64_t n, int32_t head_dim, int32_t type,
                        bool write) {
  const int64_t unit = type == PSA_TYPE_BF16 ? 8 : 4;       // elements of 16 bytes
  if (!r.x) return fail(PSA_ERR_INVALID, "%s is NULL", what);
  if (!aligned(r.x, 16)) return fail(PSA_ERR_INVALID, "%s must be 16-byte aligned (%p)", what, r.x);
  if (r.n_heads < 1) return fail(PSA_ERR_INVALID, "%s: n_heads must be >= 1 (got %d)", what, r.n_heads);
  if (r.n_heads > kMaxRowHeads) return fail(PSA_ERR_UNSUPPORTED, "%s: %d heads are too many", what, r.n_heads);
  if (r.stride_b % unit || r.stride_h % unit || r.stride_n % unit || r.stride_b < 0 || r.stride_h < 0 || r.stride_n < 0)
    return fail(PSA_ERR_INVALID, "%s: strides must be multiples of 16 bytes, not negative (%lld, %lld, %lld)", what,
                (long long)r.stride_b, (long long)r.stride_h, (long long)r.stride_n);
  if (write && !rows_apart(r, batch, n, head_dim))
    return fail(PSA_ERR_INVALID, "%s: an output's rows must not share memory", what);
  return PSA_OK;
}

// Bytes of partial sums of a backward with a norm; `a` holds checked sizes and heads.
size_t rope_partial_bytes(const psa::RopeArgs& a, int32_t head_dim) {
  return (size_t)(psa::rope_partial_rows(a, head_dim) * a.n_tensors * head_dim) * sizeof(float);
}

// Whether a launch can number the batch elements of all its tensors.
bool rope_batch_fits(int32_t batch, int32_t n_tensors) { return (int64_t)batch * n_tensors <= 65535; }

// Shapes and the rotation of a norm-and-rotation call; fills all of `a` but its tensors.
psa_status_t check_rope(int32_t type, int32_t batch, int32_t n_tensors, int32_t head_dim, const psa_rope_t* rope,
                        int32_t norm, const float* q_weight, const float* k_weight, float eps, psa::RopeArgs* a) {
  if (type != PSA_TYPE_BF16 && type != PSA_TYPE_FP32)
    return fail(PSA_ERR_UNSUPPORTED, "type must be PSA_TYPE_BF16 or PSA_TYPE_FP32 (got %d)", type);
  if (batch < 1) return fail(PSA_ERR_INVALID, "batch must be >= 1 (got %d)", batch);
  if (!rope_batch_fits(batch, n_tensors)) return fail(PSA_ERR_UNSUPPORTED, "batch %d is too large", batch);
  if (head_dim != 64 && head_dim != 128)
    return fail(PSA_ERR_UNSUPPORTED, "head_dim must be 64 or 128 (got %d)", head_dim);
  if (!rope) return fail(PSA_ERR_INVALID, "rope is NULL");
  psa::Geometry g;
  if (!grid_geometry(rope->grid, 1, &g))
    return fail(PSA_ERR_INVALID, "invalid grid (%d x %d x %d + %d text)", rope->grid.frames, rope->grid.height,
                rope->grid.width, rope->grid.n_text);
  const int32_t axes[3] = {rope->axis_t, rope->axis_h, rope->axis_w};
  const int32_t origin[3] = {rope->origin_t, rope->origin_h, rope->origin_w};
  const int32_t extent[3] = {rope->grid.frames, rope->grid.height, rope->grid.width};
  int64_t channels = 0;
  for (int i = 0; i < 3; i++) {
    if (axes[i] < 0 || axes[i] % 2) return fail(PSA_ERR_INVALID, "channels of an axis must be even and >= 0 (got %d)", axes[i]);
    if ((int64_t)origin[i] + extent[i] > INT32_MAX) return fail(PSA_ERR_INVALID, "positions from %d on are too large", origin[i]);
    channels += axes[i];
  }
  if (channels > head_dim) return fail(PSA_ERR_INVALID, "the axes have %lld channels, a head %d", (long long)channels, head_dim);
  if (rope->pairs != PSA_PAIRS_ADJACENT && rope->pairs != PSA_PAIRS_HALVES)
    return fail(PSA_ERR_INVALID, "pairs must be PSA_PAIRS_ADJACENT or PSA_PAIRS_HALVES (got %d)", rope->pairs);
  if (rope->pairs == PSA_PAIRS_HALVES && channels != head_dim)
    return fail(PSA_ERR_INVALID, "pairs across the halves need axes that fill the head (%lld of %d channels)",
                (long long)channels, head_dim);
  if (!(rope->theta > 0) || !std::isfinite(rope->theta)) return fail(PSA_ERR_INVALID, "theta must be positive and finite");
  if (!(eps >= 0) || !std::isfinite(eps)) return fail(PSA_ERR_INVALID, "eps must be >= 0 and finite");
  if (!norm && (q_weight || k_weight)) return fail(PSA_ERR_INVALID, "weights without a norm");
  if (!aligned(q_weight, 4) || !aligned(k_weight, 4)) return fail(PSA_ERR_INVALID, "weights must be 4-byte aligned");
  *a = psa::RopeArgs{};
  a->n_tensors = n_tensors;
  a->batch = batch;
  a->n = g.n;
  a->n_video = g.n_video;
  a->hw = g.hw;
  a->width = rope->grid.width;
  a->eps = eps;
  a->t[0].weight = q_weight;
  a->t[1].weight = k_weight;
  int pair = 0;
  for (int i = 0; i < 3; i++) {
    a->origin[i] = origin[i];
    // theta^(-2 j / d_a) by products of its first step, each right to 2^-53: 2^-47 after the 63 of a whole head.
    const double step = axes[i] > 0 ? std::pow(rope->theta, -2.0 / axes[i]) : 0.0;
    double turns = 0.15915494309189533577;                                                        // 1 / (2 pi)
    for (int j = 0; j < axes[i] / 2; j++, turns *= step) a->turns[pair++] = turns;
    if (i < 2) a->end[i] = pair;
  }
  return PSA_OK;
}

void set_rows(psa::RopeTensor* t, const psa_rows_t& r) {
  t->x = r.x;
  t->stride_b = r.stride_b;
  t->stride_h = r.stride_h;
  t->stride_n = r.stride_n;
  t->n_heads = r.n_heads;
}

// Shapes that a selection and the attention over a map share.  kv may be null (size queries).
psa_status_t check_mapped(int32_t batch, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t n_q,
                          int32_t n_k, int32_t block, int32_t* nbq, int32_t* nbk) {
  psa_status_t s = check_attention_shape(batch, n_heads, head_dim, block);
  if (s != PSA_OK) return s;
  if (n_kv_heads < 1 || n_heads % n_kv_heads)
    return fail(PSA_ERR_INVALID, "%d key heads do not divide %d query heads", n_kv_heads, n_heads);
  if (n_q < 1 || n_k < 1) return fail(PSA_ERR_INVALID, "n_q and n_k must be >= 1 (got %d, %d)", n_q, n_k);
  *nbq = (int32_t)(((int64_t)n_q + block - 1) / block);
  *nbk = (int32_t)(((int64_t)n_k + block - 1) / block);
  if (*nbq > PSA_MAX_BLOCKS || *nbk > PSA_MAX_BLOCKS)
    return fail(PSA_ERR_UNSUPPORTED, "%d x %d blocks exceed %d", *nbq, *nbk, PSA_MAX_BLOCKS);
  // (work items, and blocks of both sides together, are 32-bit numbers; of the two products the first may need 62 bits)
  const int64_t most = ((int64_t)1 << 31) - 8, n_bh = (int64_t)batch * n_heads;
  if (n_bh >= most || n_bh * ((int64_t)*nbq + *nbk) >= most)
    return fail(PSA_ERR_UNSUPPORTED, "too many work items");
  return PSA_OK;
}

// A call whose sizes are right but whose launches would not hold them.
psa_status_t check_launch(bool fits) {
  return fits ? PSA_OK : fail(PSA_ERR_UNSUPPORTED, "more blocks than a launch holds");
}

psa_status_t check_kv(const psa_kv_t* kv, bool values) {
  if (!kv || !kv->k || (values && !kv->v)) return fail(PSA_ERR_INVALID, "keys and values must be non-NULL");
  if (!aligned(kv->k, 16) || (values && !aligned(kv->v, 16)))
    return fail(PSA_ERR_INVALID, "keys and values must be 16-byte aligned (%p %p)", kv->k, kv->v);
  if (kv->stride_b < 0 || kv->stride_h < 0 || kv->stride_b % 8 || kv->stride_h % 8)
    return fail(PSA_ERR_INVALID, "strides of keys and values must be multiples of 8, not negative (%lld, %lld)",
                (long long)kv->stride_b, (long long)kv->stride_h);
  return PSA_OK;
}

// Tensors, map and shapes of an attention over a map; fills `a` but for what one direction has alone.
psa_status_t check_map_call(const void* q, const psa_kv_t* kv, const void* o, const float* lse, int32_t batch,
                            int32_t n_heads, int32_t head_dim, int32_t n_q, int32_t n_k, int32_t block,
                            const uint8_t* blockmap, int64_t map_stride_b, float softmax_scale, psa::MapArgs* a) {
  psa_status_t s = check_kv(kv, true);
  if (s != PSA_OK) return s;
  int32_t nbq, nbk;
  s = check_mapped(batch, n_heads, kv->n_heads, head_dim, n_q, n_k, block, &nbq, &nbk);
  if (s != PSA_OK) return s;
  if (!q || !o || !aligned(q, 16) || !aligned(o, 16))
    return fail(PSA_ERR_INVALID, "q and o must be non-NULL and 16-byte aligned (%p %p)", q, o);
  if (!aligned(lse, 4)) return fail(PSA_ERR_INVALID, "lse must be 4-byte aligned (%p)", (const void*)lse);
  if (!blockmap) return fail(PSA_ERR_INVALID, "blockmap is NULL");
  if (map_stride_b < 0) return fail(PSA_ERR_INVALID, "map_stride_b must not be negative (%lld)", (long long)map_stride_b);
  *a = psa::MapArgs{};
  a->q = (const __bf16*)q;
  a->k = (const __bf16*)kv->k;
  a->v = (const __bf16*)kv->v;
  a->o = (__bf16*)const_cast<void*>(o);
  a->lse = const_cast<float*>(lse);
  a->map = blockmap;
  a->map_stride_b = map_stride_b;
  a->kv_stride_b = kv->stride_b;
  a->kv_stride_h = kv->stride_h;
  a->n_bh = batch * n_heads;
  a->n_heads = n_heads;
  a->group = n_heads / kv->n_heads;
  a->n_q = n_q;
  a->n_k = n_k;
  a->nbq = nbq;
  a->nbk = nbk;
  a->block = block;
  a->scale = softmax_scale;
  const double c = (double)softmax_scale * 1.4426950408889634;
  a->c = (float)c;
  int exponent = 1;
  a->factor = c != 0.0 && std::isfinite(c) ? (float)(2.0 * std::frexp(std::fabs(c), &exponent)) : 1.0f;
  a->pow2 = c != 0.0 && std::isfinite(c) ? (float)std::copysign(std::ldexp(1.0, exponent - 1), c) : (float)c;
  return PSA_OK;
}

psa_status_t check_map_workspace(const void* workspace, size_t bytes, size_t need) {
  if (need && (!workspace || bytes < need))
    return fail(PSA_ERR_WORKSPACE, "workspace of %zu bytes at %p; %zu bytes required", bytes, workspace, need);
  if (!aligned(workspace, 256)) return fail(PSA_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  return PSA_OK;
}

}  // namespace

extern "C" {

int32_t psa_num_blocks(psa_grid_t grid, int32_t block) {
  psa::Geometry g;
  return grid_geometry(grid, block, &g) ? g.nb : -1;
}

size_t psa_workspace_size(int32_t batch, int32_t n_heads, psa_grid_t grid, int32_t block) {
  psa::Geometry g;
  if (batch < 1 || n_heads < 1 || !grid_geometry(grid, block, &g)) return 0;
  return psa::workspace_layout(batch, n_heads, g.nb, false).total;
}

int64_t psa_blocked_tokens(psa_grid_t grid, psa_block3d_t pb) {
  psa::Geometry g;
  const SavedError keep;  // a size query leaves the error detail alone
  const psa_status_t s = geometry_3d(grid, pb, 0, &g);
  return s == PSA_OK ? (int64_t)g.n : -1;
}

psa_status_t psa_to_blocks(const void* x, void* xb, int32_t batch_heads, int32_t head_dim,
                           psa_grid_t grid, psa_block3d_t pb, hipStream_t stream) {
  psa_status_t s = check_layout_args(x, xb, batch_heads, head_dim);
  if (s != PSA_OK) return s;
  psa::Geometry g;
  s = geometry_3d(grid, pb, 0, &g);
  if (s != PSA_OK) return s;
  hipError_t e = psa::launch_layout(x, xb, batch_heads, head_dim, g, true, stream);
  return e == hipSuccess ? PSA_OK : hip_fail(e, "psa_to_blocks launch");
}

psa_status_t psa_from_blocks(const void* xb, void* x, int32_t batch_heads, int32_t head_dim,
                             psa_grid_t grid, psa_block3d_t pb, hipStream_t stream) {
  psa_status_t s = check_layout_args(xb, x, batch_heads, head_dim);
  if (s != PSA_OK) return s;
  psa::Geometry g;
  s = geometry_3d(grid, pb, 0, &g);
  if (s != PSA_OK) return s;
  hipError_t e = psa::launch_layout(xb, x, batch_heads, head_dim, g, false, stream);
  return e == hipSuccess ? PSA_OK : hip_fail(e, "psa_from_blocks launch");
}

psa_status_t psa_build_blockmap_3d(const psa_stripe_t* params, int32_t n_heads, psa_grid_t grid,
                                   psa_block3d_t pb, uint8_t* blockmap, int32_t* kept_per_row,
                                   int64_t* kept_per_head, hipStream_t stream) {
  psa::Geometry g;
  psa_status_t s = geometry_3d(grid, pb, 0, &g);
  if (s != PSA_OK) return s;
  s = check_params(params, n_heads);
  if (s != PSA_OK) return s;
  s = check_counts_out(kept_per_row, kept_per_head);
  if (s != PSA_OK) return s;
  const int64_t groups = (int64_t)g.tp * g.hp * g.wp + (grid.n_text > 0 ? 1 : 0);
  if (groups * groups >= ((int64_t)1 << 40) || groups >= ((int64_t)1 << 31))
    return fail(PSA_ERR_UNSUPPORTED, "PSABlock map of %lld groups is too large", (long long)groups);
  g.nb = (int32_t)groups;
  for (int32_t h0 = 0; h0 < n_heads; h0 += psa::kHeadsPerChunk) {
    const psa::ParamChunk pc = chunk_of(params, h0, n_heads);
    hipError_t e = psa::launch_group_blockmap(pc, h0, g, blockmap, kept_per_row, kept_per_head, stream);
    if (e != hipSuccess) return hip_fail(e, "psa_build_blockmap_3d launch");
  }
  return PSA_OK;
}

size_t psa_workspace_size_3d(int32_t batch, int32_t n_heads, psa_grid_t grid, psa_block3d_t pb,
                             int32_t tile) {
  psa::Geometry g;
  const SavedError keep;
  const psa_status_t s = (tile == 64 || tile == 128) ? geometry_3d(grid, pb, tile, &g) : PSA_ERR_UNSUPPORTED;
  if (batch < 1 || n_heads < 1 || s != PSA_OK) return 0;
  return psa::workspace_layout(batch, n_heads, g.nb, true).total;
}

psa_status_t psa_attention_plan_3d(int32_t batch, int32_t n_heads, psa_grid_t grid,
                                   psa_block3d_t pb, int32_t tile, const psa_stripe_t* params,
                                   void* workspace, size_t workspace_bytes,
                                   int32_t* kept_per_tile, hipStream_t stream) {
  psa::Geometry g;
  psa::WorkspaceLayout wl;
  psa_status_t s = check_plan_3d(batch, n_heads, grid, pb, tile, workspace, workspace_bytes, &g, &wl);
  if (s != PSA_OK) return s;
  s = check_params(params, n_heads);
  if (s != PSA_OK) return s;
  s = check_counts_out(kept_per_tile, nullptr);
  if (s != PSA_OK) return s;
  return enqueue_plan(batch, n_heads, g, params, workspace, wl, kept_per_tile, stream,
                      "psa_attention_plan_3d launch");
}

psa_status_t psa_attention_run_3d(const void* q, const void* k, const void* v, void* o,
                                  int32_t batch, int32_t n_heads, int32_t head_dim,
                                  psa_grid_t grid, psa_block3d_t pb, int32_t tile,
                                  float softmax_scale, void* workspace, size_t workspace_bytes,
                                  float* lse, hipStream_t stream) {
  psa_status_t s = check_tensors(q, k, v, o, lse);
  if (s != PSA_OK) return s;
  s = check_attention_shape(batch, n_heads, head_dim, tile);
  if (s != PSA_OK) return s;
  psa::Geometry g;
  psa::WorkspaceLayout wl;
  s = check_plan_3d(batch, n_heads, grid, pb, tile, workspace, workspace_bytes, &g, &wl);
  if (s != PSA_OK) return s;
  const float c = softmax_scale * 1.4426950408889634f;
  hipError_t e = psa::launch_sparse(q, k, v, o, lse, batch, n_heads, head_dim, g, c, workspace, wl,
                                    compute_units(), stream, -1);
  if (e != hipSuccess) return hip_fail(e, "psa_attention_run_3d kernel launch");
  return PSA_OK;
}

psa_status_t psa_build_blockmap(const psa_stripe_t* params, int32_t n_heads, psa_grid_t grid,
                                int32_t block, uint8_t* blockmap, int32_t* kept_per_row,
                                int64_t* kept_per_head, hipStream_t stream) {
  psa::Geometry g;
  if (!grid_geometry(grid, block, &g))
    return fail(PSA_ERR_INVALID, "invalid grid (%d x %d x %d + %d text) or block %d", grid.frames,
                grid.height, grid.width, grid.n_text, block);
  psa_status_t s = check_params(params, n_heads);
  if (s != PSA_OK) return s;
  s = check_counts_out(kept_per_row, kept_per_head);
  if (s != PSA_OK) return s;
  if ((int64_t)g.nb * g.nb >= ((int64_t)1 << 40))
    return fail(PSA_ERR_UNSUPPORTED, "block map of %d x %d blocks is too large", g.nb, g.nb);
  for (int32_t h0 = 0; h0 < n_heads; h0 += psa::kHeadsPerChunk) {
    const psa::ParamChunk pc = chunk_of(params, h0, n_heads);
    hipError_t e = psa::launch_blockmap(pc, h0, g, blockmap, kept_per_row, kept_per_head, stream);
    if (e != hipSuccess) return hip_fail(e, "psa_build_blockmap launch");
  }
  return PSA_OK;
}

psa_status_t psa_attention_plan(int32_t batch, int32_t n_heads, psa_grid_t grid, int32_t block,
                                const psa_stripe_t* params, void* workspace,
                                size_t workspace_bytes, int32_t* kept_per_row,
                                hipStream_t stream) {
  psa::Geometry g;
  psa::WorkspaceLayout wl;
  psa_status_t s = check_plan(batch, n_heads, grid, block, workspace, workspace_bytes, &g, &wl);
  if (s != PSA_OK) return s;
  s = check_params(params, n_heads);
  if (s != PSA_OK) return s;
  s = check_counts_out(kept_per_row, nullptr);
  if (s != PSA_OK) return s;
  return enqueue_plan(batch, n_heads, g, params, workspace, wl, kept_per_row, stream,
                      "psa_attention_plan launch");
}

psa_status_t psa_attention_run(const void* q, const void* k, const void* v, void* o,
                               int32_t batch, int32_t n_heads, int32_t head_dim, psa_grid_t grid,
                               int32_t block, float softmax_scale, void* workspace,
                               size_t workspace_bytes, float* lse, hipStream_t stream) {
  return run_planned(q, k, v, o, batch, n_heads, head_dim, grid, block, softmax_scale, workspace,
                     workspace_bytes, lse, stream, nullptr);
}

psa_status_t psa_attention_fwd(const void* q, const void* k, const void* v, void* o,
                               int32_t batch, int32_t n_heads, int32_t head_dim, psa_grid_t grid,
                               int32_t block, const psa_stripe_t* params, float softmax_scale,
                               void* workspace, size_t workspace_bytes, float* lse,
                               int32_t* kept_per_row, hipStream_t stream) {
  psa_status_t s = check_tensors(q, k, v, o, lse);
  if (s != PSA_OK) return s;
  s = check_attention_shape(batch, n_heads, head_dim, block);
  if (s != PSA_OK) return s;
  s = psa_attention_plan(batch, n_heads, grid, block, params, workspace, workspace_bytes,
                         kept_per_row, stream);
  if (s != PSA_OK) return s;
  return run_planned(q, k, v, o, batch, n_heads, head_dim, grid, block, softmax_scale, workspace,
                     workspace_bytes, lse, stream, params);
}

psa_status_t psa_attention_fwd_noalloc(const void* q, const void* k, const void* v, void* o,
                                       int32_t batch, int32_t n_heads, int32_t head_dim,
                                       psa_grid_t grid, int32_t block, const psa_stripe_t* params,
                                       float softmax_scale, float* lse, int32_t* kept_per_row,
                                       hipStream_t stream) {
  // Everything is validated before the first HIP call.
  psa_status_t s = check_tensors(q, k, v, o, lse);
  if (s != PSA_OK) return s;
  s = check_attention_shape(batch, n_heads, head_dim, block);
  if (s != PSA_OK) return s;
  psa::Geometry g;
  if (!grid_geometry(grid, block, &g))
    return fail(PSA_ERR_INVALID, "invalid grid (%d x %d x %d + %d text)", grid.frames, grid.height,
                grid.width, grid.n_text);
  s = check_limits(batch, n_heads, &g);
  if (s != PSA_OK) return s;
  s = check_params(params, n_heads);
  if (s != PSA_OK) return s;
  s = check_counts_out(kept_per_row, nullptr);
  if (s != PSA_OK) return s;
  const size_t need = psa::workspace_layout(batch, n_heads, g.nb, false).total;
  if (need > PSA_NOALLOC_SCRATCH_BYTES)
    return fail(PSA_ERR_WORKSPACE, "the plan of these sizes needs %zu bytes; the static scratch holds %zu",
                need, (size_t)PSA_NOALLOC_SCRATCH_BYTES);
  void* scratch = nullptr;
  const hipError_t e = psa::scratch_pointer(&scratch);
  if (e != hipSuccess) return hip_fail(e, "psa_attention_fwd_noalloc: address of the static scratch");
  return psa_attention_fwd(q, k, v, o, batch, n_heads, head_dim, grid, block, params, softmax_scale,
                           scratch, PSA_NOALLOC_SCRATCH_BYTES, lse, kept_per_row, stream);
}

size_t psa_dense_workspace_size(void) { return psa::kDenseWorkspaceBytes; }

psa_status_t psa_dense_fwd(const void* q, const void* k, const void* v, void* o, int32_t batch,
                           int32_t n_heads, int32_t head_dim, int32_t n_tokens, int32_t block,
                           float softmax_scale, float* lse, void* workspace,
                           size_t workspace_bytes, hipStream_t stream) {
  psa_status_t s = check_tensors(q, k, v, o, lse);
  if (s != PSA_OK) return s;
  s = check_attention_shape(batch, n_heads, head_dim, block);
  if (s != PSA_OK) return s;
  if (n_tokens < 1 || (int64_t)n_tokens + 2 * block >= ((int64_t)1 << 31))
    return fail(PSA_ERR_INVALID, "n_tokens must be in [1, 2^31 - 2*block) (got %d)", n_tokens);
  const int64_t items = (int64_t)batch * n_heads * ((n_tokens + block - 1) / block);
  if (items + 8 >= ((int64_t)1 << 31)) return fail(PSA_ERR_UNSUPPORTED, "too many work items");
  if (workspace && workspace_bytes < psa::kDenseWorkspaceBytes)
    return fail(PSA_ERR_WORKSPACE, "dense workspace of %zu bytes; %zu bytes required", workspace_bytes,
                psa::kDenseWorkspaceBytes);
  if (((uintptr_t)workspace & 255) != 0)
    return fail(PSA_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  const float c = softmax_scale * 1.4426950408889634f;
  hipError_t e = psa::launch_dense(q, k, v, o, lse, batch, n_heads, head_dim, n_tokens, block, c,
                                   (int32_t*)workspace, compute_units(), stream);
  if (e != hipSuccess) return hip_fail(e, "psa_dense_fwd kernel launch");
  return PSA_OK;
}

size_t psa_l2_workspace_size(int32_t batch_heads) {
  return batch_heads < 1 ? 0 : (size_t)batch_heads * psa::kL2Chunks * 2 * sizeof(double);
}

psa_status_t psa_l2_distance(const void* o, const void* ref, int32_t batch_heads, int32_t n_tokens,
                             int32_t head_dim, double* sq_err, double* sq_ref, void* workspace,
                             size_t workspace_bytes, hipStream_t stream) {
  if (!o || !ref || !sq_err) return fail(PSA_ERR_INVALID, "o, ref and sq_err must be non-NULL");
  if (batch_heads < 1 || n_tokens < 1)
    return fail(PSA_ERR_INVALID, "batch_heads and n_tokens must be >= 1 (got %d, %d)", batch_heads,
                n_tokens);
  if (batch_heads > 65535)
    return fail(PSA_ERR_UNSUPPORTED, "batch_heads must be <= 65535 (got %d)", batch_heads);
  if (head_dim < 8 || head_dim % 8 != 0)
    return fail(PSA_ERR_UNSUPPORTED, "head_dim must be a positive multiple of 8 (got %d)", head_dim);
  if (!aligned(o, 16) || !aligned(ref, 16))
    return fail(PSA_ERR_INVALID, "o and ref must be 16-byte aligned");
  if (!aligned(sq_err, 8) || !aligned(sq_ref, 8))
    return fail(PSA_ERR_INVALID, "sq_err and sq_ref must be 8-byte aligned");
  if (!workspace || workspace_bytes < psa_l2_workspace_size(batch_heads))
    return fail(PSA_ERR_WORKSPACE, "workspace of %zu bytes; %zu bytes required", workspace_bytes,
                psa_l2_workspace_size(batch_heads));
  if (!aligned(workspace, 8)) return fail(PSA_ERR_WORKSPACE, "workspace must be 8-byte aligned");
  hipError_t e = psa::launch_l2(o, ref, batch_heads, (int64_t)n_tokens * head_dim, (double*)workspace,
                                sq_err, sq_ref, stream);
  return e == hipSuccess ? PSA_OK : hip_fail(e, "psa_l2_distance launch");
}

psa_status_t psa_qk_norm_rope_fwd(const psa_rows_t* q, const psa_rows_t* k, void* q_out, void* k_out,
                                  int32_t type, int32_t batch, int32_t head_dim, const psa_rope_t* rope,
                                  int32_t norm, const float* q_weight, const float* k_weight, float eps,
                                  hipStream_t stream) {
  psa::RopeArgs a;
  psa_status_t s = check_rope(type, batch, k ? 2 : 1, head_dim, rope, norm, q_weight, k_weight, eps, &a);
  if (s != PSA_OK) return s;
  if (!psa::rope_fits(a.n, head_dim)) return fail(PSA_ERR_UNSUPPORTED, "%d tokens are too many", a.n);
  if (!q) return fail(PSA_ERR_INVALID, "q is NULL");
  const psa_rows_t* rows[2] = {q, k};
  void* out[2] = {q_out, k_out};
  for (int i = 0; i < a.n_tensors; i++) {
    s = check_rows(*rows[i], i ? "k" : "q", batch, a.n, head_dim, type, false);
    if (s != PSA_OK) return s;
    if (!out[i] || !aligned(out[i], 16))
      return fail(PSA_ERR_INVALID, "outputs must be non-NULL and 16-byte aligned (%p)", out[i]);
    set_rows(&a.t[i], *rows[i]);
    a.t[i].y = out[i];
  }
  const hipError_t e = psa::launch_norm_rope(a, head_dim, type == PSA_TYPE_FP32, norm, rope->pairs == PSA_PAIRS_HALVES, stream);
  return e == hipSuccess ? PSA_OK : hip_fail(e, "psa_qk_norm_rope_fwd launch");
}

size_t psa_qk_norm_rope_workspace_size(int32_t batch, int32_t n_heads, int32_t n_kv_heads,
                                       int32_t head_dim, psa_grid_t grid, int32_t norm) {
  psa::Geometry g;
  const int32_t n_tensors = n_kv_heads > 0 ? 2 : 1;
  if (!norm || batch < 1 || n_heads < 1 || n_kv_heads < 0 || n_heads > kMaxRowHeads || n_kv_heads > kMaxRowHeads ||
      (head_dim != 64 && head_dim != 128) || !rope_batch_fits(batch, n_tensors) || !grid_geometry(grid, 1, &g))
    return 0;
  psa::RopeArgs a = {};
  a.batch = batch;
  a.n = g.n;
  a.n_tensors = n_tensors;
  a.t[0].n_heads = n_heads;
  a.t[1].n_heads = n_kv_heads;
  return rope_partial_bytes(a, head_dim);
}

psa_status_t psa_qk_norm_rope_bwd(const void* dq_out, const void* dk_out, const psa_rows_t* q,
                                  const psa_rows_t* k, const psa_rows_t* dq, const psa_rows_t* dk,
                                  float* dq_weight, float* dk_weight, int32_t type, int32_t batch,
                                  int32_t head_dim, const psa_rope_t* rope, int32_t norm,
                                  const float* q_weight, const float* k_weight, float eps, void* workspace,
                                  size_t workspace_bytes, hipStream_t stream) {
  psa::RopeArgs a;
  psa_status_t s = check_rope(type, batch, k ? 2 : 1, head_dim, rope, norm, q_weight, k_weight, eps, &a);
  if (s != PSA_OK) return s;
  if (!q || !dq || (k && !dk)) return fail(PSA_ERR_INVALID, "q, dq and, with k, dk must be non-NULL");
  const psa_rows_t *rows[2] = {q, k}, *grads[2] = {dq, dk};
  const void* dy[2] = {dq_out, dk_out};
  float* dw[2] = {dq_weight, dk_weight};
  for (int i = 0; i < a.n_tensors; i++) {
    if (norm) {
      s = check_rows(*rows[i], i ? "k" : "q", batch, a.n, head_dim, type, false);
      if (s != PSA_OK) return s;
      if (!dw[i] || !aligned(dw[i], 4))
        return fail(PSA_ERR_INVALID, "the weights' gradients must be non-NULL and 4-byte aligned (%p)", (void*)dw[i]);
    }
    s = check_rows(*grads[i], i ? "dk" : "dq", batch, a.n, head_dim, type, true);
    if (s != PSA_OK) return s;
    if (grads[i]->n_heads != rows[i]->n_heads)
      return fail(PSA_ERR_INVALID, "gradients of %d heads for %d", grads[i]->n_heads, rows[i]->n_heads);
    if (!dy[i] || !aligned(dy[i], 16))
      return fail(PSA_ERR_INVALID, "dq_out and dk_out must be non-NULL and 16-byte aligned (%p)", dy[i]);
    set_rows(&a.t[i], *rows[i]);
    a.t[i].dy = dy[i];
    a.t[i].dx = grads[i]->x;
    a.t[i].dx_stride_b = grads[i]->stride_b;
    a.t[i].dx_stride_h = grads[i]->stride_h;
    a.t[i].dx_stride_n = grads[i]->stride_n;
  }
  const size_t need = norm ? rope_partial_bytes(a, head_dim) : 0;
  if (norm && (!workspace || workspace_bytes < need))
    return fail(PSA_ERR_WORKSPACE, "workspace of %zu bytes at %p; %zu bytes required", workspace_bytes, workspace, need);
  if (!aligned(workspace, 256)) return fail(PSA_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  a.partial = (float*)workspace;
  const hipError_t e = psa::launch_norm_rope_bwd(a, head_dim, type == PSA_TYPE_FP32, norm,
                                                 rope->pairs == PSA_PAIRS_HALVES, dq_weight, dk_weight, stream);
  return e == hipSuccess ? PSA_OK : hip_fail(e, "psa_qk_norm_rope_bwd launch");
}

size_t psa_select_workspace_size(int32_t batch, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                 int32_t n_q, int32_t n_k, int32_t block) {
  const SavedError keep;
  int32_t nbq, nbk;
  if (check_mapped(batch, n_heads, n_kv_heads, head_dim, n_q, n_k, block, &nbq, &nbk) != PSA_OK ||
      !psa::select_fits(batch * n_heads, batch * n_kv_heads, nbq, nbk))
    return 0;
  return psa::select_layout(batch * n_heads, batch * n_kv_heads, head_dim, nbq, nbk).total;
}

psa_status_t psa_select_blocks(const void* q, const psa_kv_t* kv, int32_t batch, int32_t n_heads,
                               int32_t head_dim, int32_t n_q, int32_t n_k, int32_t block, int32_t keep,
                               int32_t q_text, int32_t k_text, uint8_t* blockmap, int32_t* kept_per_row,
                               void* workspace, size_t workspace_bytes, hipStream_t stream) {
  psa_status_t s = check_kv(kv, false);
  if (s != PSA_OK) return s;
  psa::SelectArgs a = {};
  s = check_mapped(batch, n_heads, kv->n_heads, head_dim, n_q, n_k, block, &a.nbq, &a.nbk);
  if (s != PSA_OK) return s;
  s = check_launch(psa::select_fits(batch * n_heads, batch * kv->n_heads, a.nbq, a.nbk));
  if (s != PSA_OK) return s;
  if (!q || !aligned(q, 16)) return fail(PSA_ERR_INVALID, "q must be non-NULL and 16-byte aligned (%p)", q);
  if (!blockmap) return fail(PSA_ERR_INVALID, "blockmap is NULL");
  s = check_counts_out(kept_per_row, nullptr);
  if (s != PSA_OK) return s;
  if (keep < 0) return fail(PSA_ERR_INVALID, "keep must be >= 0 (got %d)", keep);
  if (q_text < 0 || q_text > n_q || k_text < 0 || k_text > n_k)
    return fail(PSA_ERR_INVALID, "text of %d and %d tokens in %d and %d", q_text, k_text, n_q, n_k);
  const psa::SelectLayout l = psa::select_layout(batch * n_heads, batch * kv->n_heads, head_dim, a.nbq, a.nbk);
  s = check_map_workspace(workspace, workspace_bytes, l.total);
  if (s != PSA_OK) return s;
  a.q = (const __bf16*)q;
  a.k = (const __bf16*)kv->k;
  a.kv_stride_b = kv->stride_b;
  a.kv_stride_h = kv->stride_h;
  a.mean_q = (double*)((char*)workspace + l.mean_q);
  a.mean_k = (double*)((char*)workspace + l.mean_k);
  a.scores = (uint64_t*)((char*)workspace + l.scores);
  a.map = blockmap;
  a.kept_per_row = kept_per_row;
  a.n_bh = batch * n_heads;
  a.n_heads = n_heads;
  a.n_kv_heads = kv->n_heads;
  a.group = n_heads / kv->n_heads;
  a.n_q = n_q;
  a.n_k = n_k;
  a.block = block;
  a.keep = keep;
  a.first_q = q_text ? (n_q - q_text) / block : a.nbq;
  a.first_k = k_text ? (n_k - k_text) / block : a.nbk;
  const hipError_t e = psa::launch_select(a, head_dim, stream);
  return e == hipSuccess ? PSA_OK : hip_fail(e, "psa_select_blocks launch");
}

size_t psa_attention_map_workspace_size(int32_t batch, int32_t n_heads, int32_t head_dim, int32_t n_q,
                                        int32_t n_k, int32_t block) {
  const SavedError keep;
  int32_t nbq, nbk;
  if (check_mapped(batch, n_heads, 1, head_dim, n_q, n_k, block, &nbq, &nbk) != PSA_OK) return 0;
  const psa::MapLayout l = psa::map_layout(batch * n_heads, head_dim, nbq, nbk, block);
  return psa::map_fits(l, batch * n_heads, nbq, block) ? l.total : 0;
}

psa_status_t psa_attention_map_fwd(const void* q, const psa_kv_t* kv, void* o, int32_t batch,
                                   int32_t n_heads, int32_t head_dim, int32_t n_q, int32_t n_k,
                                   int32_t block, const uint8_t* blockmap, int64_t map_stride_b,
                                   float softmax_scale, float* lse, void* workspace,
                                   size_t workspace_bytes, hipStream_t stream) {
  psa::MapArgs a;
  psa_status_t s = check_map_call(q, kv, o, lse, batch, n_heads, head_dim, n_q, n_k, block, blockmap, map_stride_b,
                                  softmax_scale, &a);
  if (s != PSA_OK) return s;
  const psa::MapLayout l = psa::map_layout(a.n_bh, head_dim, a.nbq, a.nbk, block);
  s = check_launch(psa::map_fits(l, a.n_bh, a.nbq, block));
  if (s != PSA_OK) return s;
  s = check_map_workspace(workspace, workspace_bytes, l.total);
  if (s != PSA_OK) return s;
  a.parts = l.parts;
  char* ws = (char*)workspace;
  a.row_pieces = l.rows;
  if (l.rows.grid) {
    a.row_counts = (int32_t*)(ws + l.row_counts);
    a.row_pieces.order = (int2*)(ws + l.row_order);
    a.row_pieces.split = (int4*)(ws + l.row_split) + 1;
    if (l.paired) {
      a.pair_counts = (int32_t*)(ws + l.pair_counts);
      a.pair_order = (int32_t*)(ws + l.pair_order);
      a.paired = (int32_t*)(ws + l.paired);
    }
  }
  a.part_o = (float*)(ws + l.part_o);
  a.part_ml = (float2*)(ws + l.part_ml);
  const hipError_t e = psa::launch_map_fwd(a, head_dim, stream);
  return e == hipSuccess ? PSA_OK : hip_fail(e, "psa_attention_map_fwd launch");
}

size_t psa_attention_map_bwd_workspace_size(int32_t batch, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                            int32_t n_q, int32_t n_k, int32_t block) {
  const SavedError keep;
  int32_t nbq, nbk;
  if (check_mapped(batch, n_heads, n_kv_heads, head_dim, n_q, n_k, block, &nbq, &nbk) != PSA_OK) return 0;
  const psa::MapBwdLayout l = psa::map_bwd_layout(batch * n_heads, batch * n_kv_heads, head_dim, nbq, nbk, block);
  return psa::map_bwd_fits(l, batch * n_heads, batch * n_kv_heads, head_dim, nbq, nbk, block) ? l.total : 0;
}

psa_status_t psa_attention_map_bwd(const void* grad_o, const void* q, const psa_kv_t* kv, const void* o,
                                   const float* lse, int32_t batch, int32_t n_heads, int32_t head_dim,
                                   int32_t n_q, int32_t n_k, int32_t block, const uint8_t* blockmap,
                                   int64_t map_stride_b, float softmax_scale, void* dq, void* dk,
                                   void* dv, void* workspace, size_t workspace_bytes,
                                   hipStream_t stream) {
  psa::MapArgs a;
  psa_status_t s = check_map_call(q, kv, o, lse, batch, n_heads, head_dim, n_q, n_k, block, blockmap, map_stride_b,
                                  softmax_scale, &a);
  if (s != PSA_OK) return s;
  if (!lse) return fail(PSA_ERR_INVALID, "lse is NULL");
  for (const void* p : {grad_o, (const void*)dq, (const void*)dk, (const void*)dv})
    if (!p || !aligned(p, 16))
      return fail(PSA_ERR_INVALID, "grad_o, dq, dk and dv must be non-NULL and 16-byte aligned (%p)", p);
  const psa::MapBwdLayout l = psa::map_bwd_layout(a.n_bh, batch * kv->n_heads, head_dim, a.nbq, a.nbk, block);
  s = check_launch(psa::map_bwd_fits(l, a.n_bh, batch * kv->n_heads, head_dim, a.nbq, a.nbk, block));
  if (s != PSA_OK) return s;
  s = check_map_workspace(workspace, workspace_bytes, l.total);
  if (s != PSA_OK) return s;
  a.grad_o = (const __bf16*)grad_o;
  a.dq = (__bf16*)dq;
  a.dk = (__bf16*)dk;
  a.dv = (__bf16*)dv;
  char* ws = (char*)workspace;
  a.neg_lse2 = (float*)(ws + l.neg_lse2);
  a.neg_delta = (float*)(ws + l.neg_delta);
  a.row_pieces = l.rows;
  if (l.rows.grid) {
    a.row_counts = (int32_t*)(ws + l.row_counts);
    a.row_pieces.order = (int2*)(ws + l.row_order);
    a.row_pieces.split = (int4*)(ws + l.row_split) + 1;
  }
  a.col_pieces = l.cols;
  if (l.cols.grid) {
    a.col_counts = (int32_t*)(ws + l.col_counts);
    a.col_pieces.order = (int2*)(ws + l.col_order);
    a.col_pieces.split = (int4*)(ws + l.col_split) + 1;
  }
  a.part_q = (float*)(ws + l.part_q);
  a.part_k = (float*)(ws + l.part_k);
  a.part_v = (float*)(ws + l.part_v);
  a.parts = l.parts;
  a.head_parts = l.head_parts;
  a.list_parts = l.list_parts;
  const hipError_t e = psa::launch_map_bwd(a, head_dim, stream);
  return e == hipSuccess ? PSA_OK : hip_fail(e, "psa_attention_map_bwd launch");
}

const char* psa_status_string(psa_status_t status) {
  switch (status) {
    case PSA_OK: return "PSA_OK";
    case PSA_ERR_INVALID: return "PSA_ERR_INVALID: invalid argument";
    case PSA_ERR_UNSUPPORTED: return "PSA_ERR_UNSUPPORTED: unsupported shape";
    case PSA_ERR_WORKSPACE: return "PSA_ERR_WORKSPACE: workspace missing or too small";
    case PSA_ERR_HIP: return "PSA_ERR_HIP: HIP runtime error";
  }
  return "unknown psa_status_t";
}

const char* psa_last_error(void) { return g_error; }

}  // extern "C"
