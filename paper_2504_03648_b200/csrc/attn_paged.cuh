// Host side of attn_paged: checks, the choice of kernels and the workspace.
#pragma once

#include <float.h>
#include <math.h>

#include "attn_tiles.cuh"

namespace aibx {

struct AttnPlan {
  int G = 0;
  int row_limit = 0;                     // rows up to which a request is the row kernel's
  bool rows = false, tiles = false;      // which kernels run
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
inline int32_t attn_plan(const aibx_kv_cache_t* c, const aibx_kv_batch_t* b,
                         const aibx_attn_params_t* p, AttnPlan& plan) {
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
  plan.tiles = bound * plan.G > 16;
  plan.rows = !plan.tiles || (b->R > 1 && plan.G <= 16);
  if (plan.rows) plan.row_limit = (plan.tiles ? plan.G : bound * plan.G) <= 8 ? 8 : 16;
  plan.rows_bytes = plan.rows ? slot_bytes(plan.row_limit, L.head_dim) : 0;
  plan.workspace = plan.rows_bytes + (plan.tiles ? slot_bytes(2 * kTileRows, L.head_dim) : 0);
  return AIBX_OK;
}

template <int D, bool F8, typename QT>
inline int32_t launch_attn_kind(AttnArgs a, int type, const AttnPlan& plan, cudaStream_t st) {
  JoinSet rows = {nullptr, nullptr, 0}, tiles = rows;
  if (plan.rows) {
    const int32_t rc = plan.row_limit == 8 ? launch_attn_rows<D, F8, QT, 8>(a, type, rows, st)
                                           : launch_attn_rows<D, F8, QT, 16>(a, type, rows, st);
    if (rc != AIBX_OK) return rc;
    a.slots += plan.rows_bytes / sizeof(float);
  }
  if (plan.tiles) {
    const int32_t rc = launch_attn_tiles<D, F8, QT>(a, type, tiles, st);
    if (rc != AIBX_OK) return rc;
  }
  return launch_join<D, QT>(a, rows, tiles, st);
}

template <int D>
inline int32_t launch_attn_dim(const AttnArgs& a, int type, int q_type, const AttnPlan& plan,
                               cudaStream_t st) {
  if (type == AIBX_TYPE_E4M3)
    return q_type == AIBX_TYPE_BF16 ? launch_attn_kind<D, true, __nv_bfloat16>(a, type, plan, st)
                                    : launch_attn_kind<D, true, __half>(a, type, plan, st);
  return q_type == AIBX_TYPE_BF16 ? launch_attn_kind<D, false, __nv_bfloat16>(a, type, plan, st)
                                  : launch_attn_kind<D, false, __half>(a, type, plan, st);
}

inline int32_t launch_attn(const AttnArgs& a, int type, int q_type, const AttnPlan& plan,
                           cudaStream_t st) {
  return a.pool.D == 64 ? launch_attn_dim<64>(a, type, q_type, plan, st)
                        : launch_attn_dim<128>(a, type, q_type, plan, st);
}

}  // namespace aibx
