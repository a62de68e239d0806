// Token-wise access to a paged KV pool: the views that kv_append, kv_read and attn_paged share,
// and the kernels of the first two.
//
// append: token i of request r goes to position p = kv_len[r] - n_r + i of its sequence, that is
//   to slot p mod T of block table[r][p / T], for K and V of every KV head.  A 16-bit pool takes
//   the value rounded once to its type.  An e4m3 pool takes, per (token, head, K or V) row x,
//       e    = least integer with max|x| <= 448 * 2^e        (finite elements only)
//       y    = x * 2^-e rounded to the nearest e4m3          and the byte e + 127,
//   so a cached value is y * 2^e.  The scale is a power of two because e4m3 is a floating format:
//   any other scale buys no relative precision, and with this one reading a row back is exact in
//   every type it can go to.
// read: the same places, the other way round.
//
// One warp takes one token (or, with few tokens, a part of its 2 * heads rows, so that a decoding
// step's handful of tokens still spreads over the machine); `lanes per row` lanes hold a row in
// 8-element pieces, reduce its maximum by shuffles and store it with one access per lane.  Each
// byte crosses the memory system once in each direction: bound by HBM bandwidth for long inputs
// and by the chain offsets -> length -> table -> pool of dependent loads for short ones.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "aibx_common.cuh"
#include "kv_permute.cuh"

namespace aibx {

// One layer of a pool, as strides in bytes.
struct PagedPool {
  char* base;                      // K rows of the layer, block 0
  long long kv, block, head, slot; // K -> V, block -> block, head -> head, slot -> slot
  unsigned char* scales;           // e4m3: one byte per row, the same order with rows of one byte
  long long s_kv, s_block, s_head, s_slot;
  uint32_t num_blocks;
  int T, H, D;
};

struct PagedBatch {
  const uint32_t* table;
  const int64_t* blk_off;          // ragged table when not null
  long long table_stride;
  const int64_t* tok_off;
  const int32_t* kv_len;
  long long n_tokens;
  int R;
};

// First entry and number of entries of request r's table row.
__device__ __forceinline__ void table_row(const PagedBatch& b, int r, const uint32_t*& row,
                                          long long& entries) {
  if (b.blk_off) {
    const long long at = __ldg(b.blk_off + r);
    row = b.table + at;
    entries = __ldg(b.blk_off + r + 1) - at;
  } else {
    row = b.table + (long long)r * b.table_stride;
    entries = b.table_stride;
  }
}

// The request that holds token i, by a 32-way search of the warp; -1 behind the last one.
__device__ __forceinline__ int warp_find_request(const int64_t* tok_off, int R, long long i) {
  const int lane = threadIdx.x & 31;
  const bool behind = i >= __ldg(tok_off + R);
  int lo = 0, span = R;
  while (span > 1) {
    const int step = (span + 31) >> 5;
    const long long idx = (long long)lo + (long long)(lane + 1) * step;
    const bool le = (lane + 1) * (long long)step < span && __ldg(tok_off + idx) <= i;
    const int cnt = __popc(__ballot_sync(0xffffffffu, le));
    lo += cnt * step;
    span -= cnt * step;
    if (span > step) span = step;
  }
  return behind ? -1 : lo;
}

// ------------------------------------------------------------------------------------------
// eight elements of a row

template <typename T>
struct Row8;

template <>
struct Row8<float> {
  static constexpr int kBytes = 32;
  static __device__ __forceinline__ void load(const float* p, bool vec, float* x) {
    if (vec) {
      const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
      x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
      x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = p[i];
    }
  }
  static __device__ __forceinline__ void store(float* p, bool vec, const float* x) {
    if (vec) {
      *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
      *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = x[i];
    }
  }
};

template <typename T2>
struct Half8 {
  static __device__ __forceinline__ void unpack(uint4 v, float* x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const T2 h = *reinterpret_cast<const T2*>(&w[i]);
      const float2 f = to_float2(h);
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ float2 to_float2(__nv_bfloat162 h) { return __bfloat1622float2(h); }
  static __device__ __forceinline__ float2 to_float2(__half2 h) { return __half22float2(h); }
  static __device__ __forceinline__ uint32_t pack2(float a, float b, __nv_bfloat162*) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ uint32_t pack2(float a, float b, __half2*) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ uint4 pack(const float* x) {
    T2* tag = nullptr;
    return make_uint4(pack2(x[0], x[1], tag), pack2(x[2], x[3], tag), pack2(x[4], x[5], tag),
                      pack2(x[6], x[7], tag));
  }
};

template <typename T, typename T2>
struct Row8Half {
  static constexpr int kBytes = 16;
  static __device__ __forceinline__ void load(const T* p, bool vec, float* x) {
    if (vec) {
      Half8<T2>::unpack(*reinterpret_cast<const uint4*>(p), x);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = (float)p[i];
    }
  }
  static __device__ __forceinline__ void store(T* p, bool vec, const float* x) {
    const uint4 v = Half8<T2>::pack(x);
    if (vec) {
      *reinterpret_cast<uint4*>(p) = v;
    } else {
      const T* h = reinterpret_cast<const T*>(&v);
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = h[i];
    }
  }
};

template <>
struct Row8<__nv_bfloat16> : Row8Half<__nv_bfloat16, __nv_bfloat162> {};
template <>
struct Row8<__half> : Row8Half<__half, __half2> {};

struct E4M3 {};   // tag of a pool of e4m3 rows with scale bytes

// Scale byte of a row whose largest finite magnitude is a: e + 127 with e the least integer such
// that a <= 448 * 2^e (448 = 1.75 * 2^8: compare a's exponent and its fraction with 1.75).
__device__ __forceinline__ int scale_byte(float a) {
  if (!(a > 0.0f)) return 127;
  const unsigned int u = __float_as_uint(a);
  const int ex = (int)(u >> 23);                       // biased; 0 for subnormals: clamped below
  const int byte = ex - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return byte < 1 ? 1 : byte;                          // at most 247: a < 2^128
}

__device__ __forceinline__ float power_of_byte(int byte) {   // 2^(byte - 127), 0 <= byte <= 254
  return __uint_as_float(byte > 0 ? (unsigned int)byte << 23 : 0x00400000u);
}

__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.0f;
}

// Two e4m3 numbers; infinities become NaN (the format has none).
__device__ __forceinline__ uint32_t e4m3_pair(float a, float b) {
  a = fabsf(a) < INFINITY ? a : NAN;
  b = fabsf(b) < INFINITY ? b : NAN;
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

__device__ __forceinline__ __half2 halves_of_e4m3(uint32_t pair) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)pair, __NV_E4M3);
  return *reinterpret_cast<const __half2*>(&h);
}

struct PagedIO {
  char* k;
  char* v;
  long long k_tok, k_head, v_tok, v_head;   // strides in elements
  int lanes;                                // lanes per row, a power of two
  int parts;                                // warps per token
  int vec;                                  // every row 16-byte aligned
};

// Where row `row` (K rows of all heads, then V rows) of a token lies.
template <typename X>
__device__ __forceinline__ X* io_row(const PagedIO& io, long long i, int row, int H) {
  const bool is_v = row >= H;
  const int h = is_v ? row - H : row;
  X* b = reinterpret_cast<X*>(is_v ? io.v : io.k);
  return b + i * (is_v ? io.v_tok : io.k_tok) + h * (is_v ? io.v_head : io.k_head);
}

constexpr int kPagedThreads = 256;
constexpr int kPagedUnroll = 4;      // rows in flight per lane

// TO_POOL: append; else read.  P: pool element (E4M3 tag, __half, __nv_bfloat16), X: the caller's.
// PIECES: 8-element pieces of a row per lane (1 up to D = 256, 4 up to 1024).
template <bool TO_POOL, typename P, typename X, int PIECES>
__global__ void __launch_bounds__(kPagedThreads)
kv_token_kernel(PagedPool pool, PagedBatch b, PagedIO io) {
  constexpr bool kQuant = std::is_same<P, E4M3>::value;
  constexpr int kUnroll = PIECES == 1 ? kPagedUnroll : 1;
  const long long unit = ((long long)blockIdx.x * kPagedThreads + threadIdx.x) >> 5;
  const long long i = unit / io.parts;
  const int part = (int)(unit - i * io.parts);
  if (i >= b.n_tokens) return;
  const int lane = threadIdx.x & 31;
  const int r = warp_find_request(b.tok_off, b.R, i);
  if (r < 0) return;                                     // padding behind the last request
  const long long pos = (long long)__ldg(b.kv_len + r) - (__ldg(b.tok_off + r + 1) - i);
  if (pos < 0) return;
  const uint32_t* row;
  long long entries;
  table_row(b, r, row, entries);
  const long long at = pos / pool.T;
  const int slot = (int)(pos - at * pool.T);
  const uint32_t id = at < entries ? __ldg(row + at) : pool.num_blocks;
  if (id >= pool.num_blocks) {
    if (id != AIBX_NO_BLOCK && part == 0 && lane == 0) raise_status(AIBX_ERR_RANGE);
    return;
  }
  char* base = pool.base + (long long)id * pool.block + (long long)slot * pool.slot;
  unsigned char* sbase =
      kQuant ? pool.scales + (long long)id * pool.s_block + (long long)slot * pool.s_slot : nullptr;

  const int rows = 2 * pool.H;
  const int per_step = 32 / io.lanes;                     // rows a warp holds at once
  const int sub = lane / io.lanes, col = (lane - sub * io.lanes) * 8;
  const int per_part = (rows + io.parts - 1) / io.parts;
  const int row0 = part * per_part, row1 = min(row0 + per_part, rows);
  for (int r0 = row0; r0 < row1; r0 += per_step * kUnroll) {
    float x[kUnroll][PIECES][8];
    int byte[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int rr = r0 + u * per_step + sub;
      byte[u] = 127;
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        const int d = col + p * io.lanes * 8;
        const bool on = rr < row1 && d < pool.D;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[u][p][e] = 0.0f;
        if (!on) continue;
        if (TO_POOL) {
          Row8<X>::load(io_row<const X>(io, i, rr, pool.H) + d, io.vec, x[u][p]);
        } else {
          const int kv = rr >= pool.H, h = rr - kv * pool.H;
          const char* src = base + kv * pool.kv + h * pool.head;
          if constexpr (kQuant) {
            const uint2 w = *reinterpret_cast<const uint2*>(src + d);
            byte[u] = sbase[kv * pool.s_kv + h * pool.s_head];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t pair = ((e < 2 ? w.x : w.y) >> (16 * (e & 1))) & 0xffffu;
              const float2 f = __half22float2(halves_of_e4m3(pair));
              x[u][p][2 * e] = f.x;
              x[u][p][2 * e + 1] = f.y;
            }
          } else {
            Row8<P>::load(reinterpret_cast<const P*>(src) + d, true, x[u][p]);
          }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int rr = r0 + u * per_step + sub;
      float f = 1.0f;
      if constexpr (kQuant) {
        if (TO_POOL) {
          float a = 0.0f;
#pragma unroll
          for (int p = 0; p < PIECES; ++p)
#pragma unroll
            for (int e = 0; e < 8; ++e) a = fmaxf(a, finite_abs(x[u][p][e]));
          for (int m = io.lanes >> 1; m > 0; m >>= 1)
            a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, m));
          byte[u] = scale_byte(a);
          f = power_of_byte(254 - byte[u]);
        } else {
          f = byte[u] == 255 ? NAN : power_of_byte(byte[u]);
        }
      }
      if (rr >= row1) continue;
      const int kv = rr >= pool.H, h = rr - kv * pool.H;
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        const int d = col + p * io.lanes * 8;
        if (d >= pool.D) continue;
        if constexpr (kQuant) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[u][p][e] *= f;
        }
        if (TO_POOL) {
          char* dst = base + kv * pool.kv + h * pool.head;
          if constexpr (kQuant) {
            uint2 w;
            w.x = e4m3_pair(x[u][p][0], x[u][p][1]) | (e4m3_pair(x[u][p][2], x[u][p][3]) << 16);
            w.y = e4m3_pair(x[u][p][4], x[u][p][5]) | (e4m3_pair(x[u][p][6], x[u][p][7]) << 16);
            *reinterpret_cast<uint2*>(dst + d) = w;
            if (p == 0 && col == 0) sbase[kv * pool.s_kv + h * pool.s_head] = (unsigned char)byte[u];
          } else {
            Row8<P>::store(reinterpret_cast<P*>(dst) + d, true, x[u][p]);
          }
        } else {
          Row8<X>::store(io_row<X>(io, i, rr, pool.H) + d, io.vec, x[u][p]);
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------------------
// host side

inline int type_bytes(int t) {
  switch (t) {
    case AIBX_TYPE_BF16:
    case AIBX_TYPE_FP16: return 2;
    case AIBX_TYPE_FP32: return 4;
    case AIBX_TYPE_E4M3: return 1;
    default: return 0;
  }
}

// Checks a cache and a batch and turns them into what the kernels take.  `work` says whether
// there is anything to do.
inline int32_t paged_views(const aibx_kv_cache_t* c, const aibx_kv_batch_t* b, PagedPool& pool,
                           PagedBatch& batch, bool& work) {
  work = false;
  if (!c || !b) return AIBX_ERR_INVALID;
  const aibx_kv_layout_t& L = c->layout;
  if (L.layout < 0 || L.layout > 2 || L.num_layers <= 0 || L.num_kv_heads <= 0 ||
      L.block_tokens <= 0 || L.head_dim <= 0 || c->layer < 0 || c->layer >= L.num_layers ||
      (c->inner != AIBX_INNER_HEAD_TOKEN && c->inner != AIBX_INNER_TOKEN_HEAD))
    return AIBX_ERR_INVALID;
  if (c->type != AIBX_TYPE_BF16 && c->type != AIBX_TYPE_FP16 && c->type != AIBX_TYPE_E4M3)
    return AIBX_ERR_INVALID;
  if (L.elem_bytes != type_bytes(c->type)) return AIBX_ERR_INVALID;
  if (b->R < 0 || b->n_tokens < 0 || b->max_new < 0 || b->table_stride < 0) return AIBX_ERR_INVALID;
  if (L.num_kv_heads > 4096 || L.block_tokens > 65536) return AIBX_ERR_UNSUPPORTED;
  if (L.head_dim > 1024 || L.head_dim % 8 != 0 || ((long long)L.head_dim * L.elem_bytes) % 16 != 0)
    return AIBX_ERR_UNSUPPORTED;
  if (b->R == 0 || b->n_tokens == 0) return AIBX_OK;
  if (!c->d_pool || !b->d_block_table || !b->d_tok_off || !b->d_kv_len ||
      (c->type == AIBX_TYPE_E4M3 && !c->d_scales))
    return AIBX_ERR_INVALID;
  if (reinterpret_cast<uintptr_t>(c->d_pool) & 15) return AIBX_ERR_INVALID;
  if ((reinterpret_cast<uintptr_t>(b->d_block_table) & 3) || (reinterpret_cast<uintptr_t>(b->d_tok_off) & 7) ||
      (reinterpret_cast<uintptr_t>(b->d_kv_len) & 3) || (reinterpret_cast<uintptr_t>(b->d_blk_off) & 7))
    return AIBX_ERR_INVALID;
  const bool token_first = c->inner == AIBX_INNER_TOKEN_HEAD;
  const long long row = (long long)L.head_dim * L.elem_bytes;
  const long long rows = (long long)L.num_kv_heads * L.block_tokens;
  long long layer;
  pool_strides(&L, 2 * rows * row, rows * row, pool.block, layer, pool.kv);
  pool.base = static_cast<char*>(c->d_pool) + layer * c->layer;
  pool.head = token_first ? row : row * L.block_tokens;
  pool.slot = token_first ? row * L.num_kv_heads : row;
  pool_strides(&L, 2 * rows, rows, pool.s_block, layer, pool.s_kv);
  pool.scales = c->type == AIBX_TYPE_E4M3 ? c->d_scales + layer * c->layer : nullptr;
  pool.s_head = token_first ? 1 : L.block_tokens;
  pool.s_slot = token_first ? L.num_kv_heads : 1;
  pool.num_blocks = L.num_blocks;
  pool.T = L.block_tokens;
  pool.H = L.num_kv_heads;
  pool.D = L.head_dim;
  batch.table = b->d_block_table;
  batch.blk_off = b->d_blk_off;
  batch.table_stride = b->table_stride;
  batch.tok_off = b->d_tok_off;
  batch.kv_len = b->d_kv_len;
  batch.n_tokens = b->n_tokens;
  batch.R = b->R;
  work = true;
  return AIBX_OK;
}

template <bool TO_POOL, typename P, typename X>
inline int32_t launch_kv_token(const PagedPool& pool, const PagedBatch& b, PagedIO io,
                               cudaStream_t st) {
  const int pieces = pool.D / 8;
  int lanes = 1;
  while (lanes < pieces && lanes < 32) lanes *= 2;
  io.lanes = lanes;
  // One warp per token once there are tokens for four warps on every scheduler; with fewer, a
  // token's rows are shared out down to one step of the warp's rows.
  const int steps = (2 * pool.H + 32 / lanes - 1) / (32 / lanes);
  long long parts = (long long)sm_count() * 16 / b.n_tokens;
  io.parts = (int)(parts < 1 ? 1 : parts > steps ? steps : parts);
  const long long warps = b.n_tokens * io.parts;
  const long long blocks = (warps + kPagedThreads / 32 - 1) / (kPagedThreads / 32);
  if (blocks >= (1LL << 31)) return AIBX_ERR_UNSUPPORTED;
  if (pieces <= 32)
    kv_token_kernel<TO_POOL, P, X, 1><<<(unsigned int)blocks, kPagedThreads, 0, st>>>(pool, b, io);
  else
    kv_token_kernel<TO_POOL, P, X, 4><<<(unsigned int)blocks, kPagedThreads, 0, st>>>(pool, b, io);
  return launch_status();
}

template <bool TO_POOL>
inline int32_t kv_tokens(const aibx_kv_cache_t* c, const aibx_kv_batch_t* b, const void* k,
                         int64_t k_tok, int64_t k_head, const void* v, int64_t v_tok,
                         int64_t v_head, int32_t type, cudaStream_t st) {
  PagedPool pool;
  PagedBatch batch;
  bool work;
  const int32_t rc = paged_views(c, b, pool, batch, work);
  if (rc != AIBX_OK) return rc;
  const int size = type_bytes(type);
  if (size < 2) return AIBX_ERR_INVALID;
  if (!work) return AIBX_OK;
  if (!k || !v || k_tok < 0 || k_head < 0 || v_tok < 0 || v_head < 0) return AIBX_ERR_INVALID;
  const uintptr_t kp = reinterpret_cast<uintptr_t>(k), vp = reinterpret_cast<uintptr_t>(v);
  if ((kp | vp) & (uintptr_t)(size - 1)) return AIBX_ERR_INVALID;
  PagedIO io;
  io.k = static_cast<char*>(const_cast<void*>(k));
  io.v = static_cast<char*>(const_cast<void*>(v));
  io.k_tok = k_tok;
  io.k_head = k_head;
  io.v_tok = v_tok;
  io.v_head = v_head;
  io.vec = (((kp | vp) & 15) == 0 && (((k_tok | k_head | v_tok | v_head) * size) & 15) == 0) ? 1 : 0;
#define AIBX_TOKEN_CASE(P)                                                        \
  switch (type) {                                                                 \
    case AIBX_TYPE_BF16: return launch_kv_token<TO_POOL, P, __nv_bfloat16>(pool, batch, io, st); \
    case AIBX_TYPE_FP16: return launch_kv_token<TO_POOL, P, __half>(pool, batch, io, st);        \
    default: return launch_kv_token<TO_POOL, P, float>(pool, batch, io, st);      \
  }
  switch (c->type) {
    case AIBX_TYPE_BF16: AIBX_TOKEN_CASE(__nv_bfloat16)
    case AIBX_TYPE_FP16: AIBX_TOKEN_CASE(__half)
    default: AIBX_TOKEN_CASE(E4M3)
  }
#undef AIBX_TOKEN_CASE
}

}  // namespace aibx
