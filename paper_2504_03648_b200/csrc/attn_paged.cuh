// Host side of attn_paged and attn_tree: checks, the choice of kernels and the workspace.
#pragma once

#include <float.h>
#include <math.h>

#include "attn_cols.cuh"
#include "kv_tables.cuh"

namespace aibx {

struct AttnPlan {
  int G = 0;
  int row_limit = 0;                     // rows up to which a request is the row kernel's
  bool rows = false, tiles = false;      // which kernels run
  int cols = 0, col_limit = 0;           // trees: rows of the column kernel's blocks (0: not that one) and requests
  uint64_t rows_bytes = 0, workspace = 0;
};

// Two slots of `rows` rows and one record per CTA.
inline uint64_t slot_bytes(int rows, int dim) {
  return (uint64_t)sm_count() * (2ull * rows * (dim + 2) * sizeof(float) + sizeof(JoinRecord));
}

// The row kernel alone where no request can have more than 16 rows; the tile kernel alone for a
// single request; both for a batch, each taking the requests of its kind.  The row kernel comes
// for 8 rows and for 16; beside the tile kernel it is the one for 8 where that holds a request's
// single token.
//
// Trees: the row kernel alone where no request can have more than 8 rows (at 16 it takes 206 us where
// the column kernel takes 123: twice the products, and registers spill).  The column kernel for requests of up to
// 128 rows, in blocks of 32 or 64 where none has more (fewer registers, less shared memory); over e4m3, where a
// block of 128 leaves its warps too few registers, up to 64.  The tile kernel for more: there a step costs
// less per row (bf16, 256 rows: 236 us against 291 of two blocks; e4m3, 112 rows: 532 against 569 of two,
// whose weights had 8 bits then).
inline int32_t attn_plan(const aibx_kv_cache_t* c, const aibx_kv_batch_t* b,
                         const aibx_attn_params_t* p, bool tree, AttnPlan& plan) {
  PagedPool pool;
  PagedBatch batch;
  bool work;
  const int32_t rc = paged_views(c, b, pool, batch, work);
  if (rc != AIBX_OK) return rc;
  if (!p) return AIBX_ERR_INVALID;
  const aibx_kv_layout_t& L = c->layout;
  if (p->q_type != AIBX_TYPE_BF16 && p->q_type != AIBX_TYPE_FP16) return AIBX_ERR_INVALID;
  // the scale times log2 e is a normal fp32 number: infinite it would make NaN of a score of 0, below
  // 2^-126 the kernels take it for 2^-126
  if (p->num_q_heads <= 0 || p->num_q_heads % L.num_kv_heads != 0 || p->window < 0 ||
      !(p->scale >= FLT_MIN) || !isfinite(p->scale * kLog2E))
    return AIBX_ERR_INVALID;
  const long long strides[4] = {p->q_token_stride, p->q_head_stride, p->out_token_stride,
                                p->out_head_stride};
  for (long long s : strides)
    if (s < 0 || s % 8 != 0) return AIBX_ERR_INVALID;
  if (c->type != AIBX_TYPE_E4M3 && c->type != p->q_type) return AIBX_ERR_UNSUPPORTED;
  if ((L.head_dim != 64 && L.head_dim != 128) || L.block_tokens % 8 != 0) return AIBX_ERR_UNSUPPORTED;
  plan.G = p->num_q_heads / L.num_kv_heads;
  if (plan.G > 128 || L.num_blocks > 0x7fffffffu || b->n_tokens >= (1 << 24)) return AIBX_ERR_UNSUPPORTED;
  const long long bound = b->max_new > 0 ? b->max_new : (1LL << 31);
  if (tree) {
    plan.rows = bound * plan.G <= 8;
    if (plan.rows) plan.row_limit = 8;
    const int most = c->type == AIBX_TYPE_E4M3 ? 64 : 128;
    plan.tiles = bound * plan.G > most;
    if (!plan.rows && (!plan.tiles || b->R > 1)) plan.cols = bound * plan.G <= 32 ? 32 : bound * plan.G <= 64 ? 64 : most;
    plan.col_limit = plan.cols ? most : 0;
    plan.rows_bytes = plan.rows ? slot_bytes(8, L.head_dim) : plan.cols ? slot_bytes(plan.cols, L.head_dim) : 0;
    plan.workspace = plan.rows_bytes + (plan.tiles ? slot_bytes(2 * kTileRows, L.head_dim) : 0);
    return AIBX_OK;
  }
  plan.tiles = bound * plan.G > 16;
  plan.rows = !plan.tiles || (b->R > 1 && plan.G <= 16);
  if (plan.rows) plan.row_limit = (plan.tiles ? plan.G : bound * plan.G) <= 8 ? 8 : 16;
  plan.rows_bytes = plan.rows ? slot_bytes(plan.row_limit, L.head_dim) : 0;
  plan.workspace = plan.rows_bytes + (plan.tiles ? slot_bytes(2 * kTileRows, L.head_dim) : 0);
  return AIBX_OK;
}

template <int D, bool F8, typename QT, bool TREE>
inline int32_t launch_attn_kind(AttnArgs a, int type, const AttnPlan& plan, cudaStream_t st) {
  JoinSet rows = {nullptr, nullptr, 0}, tiles = rows;
  if constexpr (TREE) {
    constexpr int kMost = F8 ? 64 : 128;
    int32_t rc = AIBX_OK;
    if (plan.rows)
      rc = launch_attn_rows<D, F8, QT, 8, true>(a, type, rows, st);
    else if (plan.cols)
      rc = plan.cols == 32   ? launch_attn_cols<D, F8, QT, 32>(a, type, rows, st)
           : plan.cols == 64 ? launch_attn_cols<D, F8, QT, 64>(a, type, rows, st)
                             : launch_attn_cols<D, F8, QT, kMost>(a, type, rows, st);
    if (rc == AIBX_OK && plan.tiles) {
      a.slots += plan.rows_bytes / sizeof(float);
      a.row_limit = plan.col_limit;
      rc = launch_attn_tiles<D, F8, QT, true>(a, type, tiles, plan.cols > 0, st);
    }
    return rc != AIBX_OK ? rc : launch_join<D, QT, true>(a, rows, tiles, st);
  }
  if (plan.rows) {
    const int32_t rc = plan.row_limit == 8 ? launch_attn_rows<D, F8, QT, 8, false>(a, type, rows, st)
                                           : launch_attn_rows<D, F8, QT, 16, false>(a, type, rows, st);
    if (rc != AIBX_OK) return rc;
    a.slots += plan.rows_bytes / sizeof(float);
  }
  if (plan.tiles) {
    const int32_t rc = launch_attn_tiles<D, F8, QT, false>(a, type, tiles, false, st);
    if (rc != AIBX_OK) return rc;
  }
  return launch_join<D, QT, false>(a, rows, tiles, st);
}

template <int D, bool TREE>
inline int32_t launch_attn_dim(const AttnArgs& a, int type, int q_type, const AttnPlan& plan,
                               cudaStream_t st) {
  if (type == AIBX_TYPE_E4M3)
    return q_type == AIBX_TYPE_BF16 ? launch_attn_kind<D, true, __nv_bfloat16, TREE>(a, type, plan, st)
                                    : launch_attn_kind<D, true, __half, TREE>(a, type, plan, st);
  return q_type == AIBX_TYPE_BF16 ? launch_attn_kind<D, false, __nv_bfloat16, TREE>(a, type, plan, st)
                                  : launch_attn_kind<D, false, __half, TREE>(a, type, plan, st);
}

template <bool TREE>
inline int32_t launch_attn(const AttnArgs& a, int type, int q_type, const AttnPlan& plan,
                           cudaStream_t st) {
  return a.pool.D == 64 ? launch_attn_dim<64, TREE>(a, type, q_type, plan, st)
                        : launch_attn_dim<128, TREE>(a, type, q_type, plan, st);
}

// Both calls: `d_mask` for trees only.
template <bool TREE>
inline int32_t attention(const aibx_kv_cache_t* cache, const aibx_kv_batch_t* batch, const aibx_attn_params_t* params,
                         const uint64_t* d_mask, int32_t mask_words, const void* d_q, void* d_out, float* d_lse,
                         void* d_workspace, uint64_t workspace_bytes, cudaStream_t st) {
  AttnPlan plan;
  int32_t rc = attn_plan(cache, batch, params, TREE, plan);
  if (rc != AIBX_OK) return rc;
  if (TREE && mask_words <= 0) return AIBX_ERR_INVALID;
  if (TREE && mask_words > kTreeMaxWords) return AIBX_ERR_UNSUPPORTED;
  AttnArgs a;
  bool work;
  rc = paged_views(cache, batch, a.pool, a.b, work);
  if (rc != AIBX_OK || !work) return rc;
  // a piece may still read queries of a row that another has written
  if (!d_q || !d_out || !d_workspace || d_q == d_out) return AIBX_ERR_INVALID;
  if ((reinterpret_cast<uintptr_t>(d_q) | reinterpret_cast<uintptr_t>(d_out) |
       reinterpret_cast<uintptr_t>(d_workspace)) & 15)
    return AIBX_ERR_INVALID;
  if ((reinterpret_cast<uintptr_t>(d_lse) & 3) || workspace_bytes < plan.workspace)
    return AIBX_ERR_INVALID;
  if (TREE && (!d_mask || (reinterpret_cast<uintptr_t>(d_mask) & 7))) return AIBX_ERR_INVALID;
  a.q = static_cast<const char*>(d_q);
  a.out = static_cast<char*>(d_out);
  a.lse = d_lse;
  a.q_tok = params->q_token_stride;
  a.q_head = params->q_head_stride;
  a.o_tok = params->out_token_stride;
  a.o_head = params->out_head_stride;
  a.scale_log2 = params->scale * kLog2E;   // never 0: hidden keys are -infinity
  a.G = plan.G;
  a.by_g = small_divisor(plan.G);
  a.by_pos = TREE ? SmallDivisor{0} : a.by_g;
  a.causal = !TREE && params->causal != 0;
  a.mask = TREE ? reinterpret_cast<const uint32_t*>(d_mask) : nullptr;
  a.mask_words = 2 * mask_words;
  a.window = params->window;
  a.box = 0;
  a.max_new = batch->max_new;
  a.row_limit = plan.row_limit;
  a.col_limit = plan.col_limit;
  a.slots = static_cast<float*>(d_workspace);
  return launch_attn<TREE>(a, cache->type, params->q_type, plan, st);
}

}  // namespace aibx
