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
// A warp takes up to 32 neighbouring tokens and some of their 2 * heads planes (K or V of a head).
// Finding a token's request, length, block and slot is a chain of dependent loads; the lanes walk
// it once for all the warp's tokens together and hand the places on by shuffles, so that what is
// left per row is an address and 16 pool bytes per lane.  (A warp per token, searching for itself,
// spent 620 instructions on 1 KB: 444 us for 404,000 tokens of 4 e4m3 heads.)  With few tokens the
// groups shrink, down to one step of rows per warp.  Now 212 us, 5.9 TB/s; 35,000 tokens quantised
// in 29 us, 3.8 TB/s (ALU pipe 64 % busy, issue slots 60 %).  Every byte crosses the memory system once in
// each direction: bound by HBM for long inputs, by the chain of loads for short ones.
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
// elements of a row in registers

template <typename X>
struct Elems;
template <>
struct Elems<float> {
  static __device__ __forceinline__ float get(const uint32_t* w, int e) { return __uint_as_float(w[e]); }
  static __device__ __forceinline__ void put(uint32_t* w, int e, float a, float b) {
    w[e] = __float_as_uint(a);
    w[e + 1] = __float_as_uint(b);
  }
};
template <>
struct Elems<__nv_bfloat16> {
  static __device__ __forceinline__ float get(const uint32_t* w, int e) {
    return __uint_as_float((e & 1) ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
  }
  static __device__ __forceinline__ void put(uint32_t* w, int e, float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    w[e >> 1] = *reinterpret_cast<const uint32_t*>(&h);
  }
};
template <>
struct Elems<__half> {
  static __device__ __forceinline__ float get(const uint32_t* w, int e) {
    const __half2 h = *reinterpret_cast<const __half2*>(w + (e >> 1));
    return (e & 1) ? __high2float(h) : __low2float(h);
  }
  static __device__ __forceinline__ void put(uint32_t* w, int e, float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    w[e >> 1] = *reinterpret_cast<const uint32_t*>(&h);
  }
};

// N words from or to memory; element by element where the caller's rows are not 16-byte aligned.
template <typename X, int N>
__device__ __forceinline__ void load_words(const X* p, bool vec, uint32_t* w) {
  if (vec) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<uint4*>(w + i) = __ldg(reinterpret_cast<const uint4*>(p) + i / 4);
  } else {
    constexpr int kPer = 4 / sizeof(X);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (kPer == 1)
        w[i] = *reinterpret_cast<const uint32_t*>(p + i);
      else
        w[i] = (uint32_t)*reinterpret_cast<const uint16_t*>(p + 2 * i) |
               ((uint32_t)*reinterpret_cast<const uint16_t*>(p + 2 * i + 1) << 16);
    }
  }
}
template <typename X, int N>
__device__ __forceinline__ void store_words(X* p, bool vec, const uint32_t* w) {
  if (vec) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *(reinterpret_cast<uint4*>(p) + i / 4) = *reinterpret_cast<const uint4*>(w + i);
  } else {
    constexpr int kPer = 4 / sizeof(X);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (kPer == 1) {
        *reinterpret_cast<uint32_t*>(p + i) = w[i];
      } else {
        *reinterpret_cast<uint16_t*>(p + 2 * i) = (uint16_t)w[i];
        *reinterpret_cast<uint16_t*>(p + 2 * i + 1) = (uint16_t)(w[i] >> 16);
      }
    }
  }
}

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

// Bits of the largest magnitude among 2 or 1 numbers a word holds: magnitudes order as their bits
// do, infinities and NaN above all finite ones.
template <typename X>
__device__ __forceinline__ uint32_t max_bits(uint32_t m, uint32_t w) {
  if constexpr (sizeof(X) == 2) return __vmaxu2(m, w & 0x7fff7fffu);
  return max(m, w & 0x7fffffffu);
}
// The magnitude itself; `finite`: whether it is one.
template <typename X>
__device__ __forceinline__ float magnitude(uint32_t m, bool& finite) {
  if constexpr (sizeof(X) == 2) {
    m = max(m >> 16, m & 0xffffu);
    const uint32_t w[1] = {m};
    const float a = Elems<X>::get(w, 0);
    finite = a < INFINITY;
    return a;
  }
  finite = m < 0x7f800000u;
  return __uint_as_float(m);
}

// Two e4m3 numbers; where not all are finite (`odd`) infinities become NaN: the format has none.
__device__ __forceinline__ uint32_t e4m3_pair(float a, float b, bool odd) {
  if (odd) {
    a = fabsf(a) < INFINITY ? a : NAN;
    b = fabsf(b) < INFINITY ? b : NAN;
  }
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
  int lane_log;                             // log2 of the lanes that hold a row
  int tokens;                               // per warp: a power of two up to 32, at least 32 >> lane_log
  int parts;                                // warps that share a group's planes
  int vec;                                  // every row 16-byte aligned
};

constexpr int kPagedThreads = 256;

// TO_POOL: append; else read.  P: pool element (E4M3 tag, __half, __nv_bfloat16), X: the caller's.
// PIECES: 16-byte pool pieces of a row per lane (with 8 bytes of an e4m3 row a lane stores 16-bit rows
// in whole sectors, but does everything else twice: 286 instead of 264 us).
// Reading wants many warps (six CTAs an SM at 40 registers: 200 us, four: 252), quantising wants its
// rows in registers (four CTAs: 29 us, six: 35).
template <bool TO_POOL, typename P, typename X, int PIECES>
__global__ void __launch_bounds__(kPagedThreads, TO_POOL ? 4 : 6)
kv_token_kernel(PagedPool pool, PagedBatch b, PagedIO io) {
  constexpr bool kQuant = std::is_same<P, E4M3>::value;
  constexpr bool kCopy = std::is_same<P, X>::value;       // nothing to convert
  constexpr int kN = kQuant ? 16 : 8;                     // elements of a piece
  constexpr int kWords = kN * (int)sizeof(X) / 4;         // of the caller's side
  constexpr int kUnroll = PIECES > 1 ? 1 : 2;   // rows in flight per lane
  const long long unit = ((long long)blockIdx.x * kPagedThreads + threadIdx.x) >> 5;
  const long long group = unit / io.parts;
  const int part = (int)(unit - group * io.parts);
  const long long i0 = group * io.tokens;
  if (i0 >= b.n_tokens) return;
  const int lane = threadIdx.x & 31;

  // ---- lane t: where token i0 + t lives
  const int r0 = warp_find_request(b.tok_off, b.R, i0);
  if (r0 < 0) return;                                     // padding behind the last request
  const int t = lane & (io.tokens - 1);
  const long long i = i0 + t;
  const int behind = (int)min(__ldg(b.tok_off + min(r0 + 1 + lane, b.R)) - i0, (long long)(1 << 20));
  int r = 0;                                              // requests that end at or before i
#pragma unroll
  for (int d = 16; d > 0; d >>= 1)
    if (__shfl_sync(0xffffffffu, behind, r + d - 1) <= t) r += d;
  const int last = __shfl_sync(0xffffffffu, behind, 31);
  if (r == 31 && last <= t) r = 32;
  r += r0;
  // Past 32 requests (those without tokens count) the rest is halved: one by one, four tokens among 4,096
  // requests took 82 us, now 6.
  for (int end = r < r0 + 32 ? r : b.R; r < end;) {
    const int mid = r + (end - r) / 2;
    if (__ldg(b.tok_off + mid + 1) <= i)
      r = mid + 1;
    else
      end = mid;
  }
  long long place = -1, splace = 0;
  if (r < b.R && i < b.n_tokens) {
    const long long pos = (long long)__ldg(b.kv_len + r) - (__ldg(b.tok_off + r + 1) - i);
    if (pos >= 0) {
      const uint32_t* row;
      long long entries;
      table_row(b, r, row, entries);
      const int at = (int)pos / pool.T, slot = (int)pos - at * pool.T;
      const uint32_t id = at < entries ? __ldg(row + at) : pool.num_blocks;
      if (id < pool.num_blocks) {
        place = (long long)id * pool.block + (long long)slot * pool.slot;
        if (kQuant) splace = (long long)id * pool.s_block + (long long)slot * pool.s_slot;
      } else if (id != AIBX_NO_BLOCK && part == 0 && lane < io.tokens) {
        raise_status(AIBX_ERR_RANGE);
      }
    }
  }

  // ---- rows: `step` tokens at a time, a plane after the other
  const int lanes = 1 << io.lane_log, step = 32 >> io.lane_log;
  const int sub = lane >> io.lane_log, col = (lane & (lanes - 1)) * kN;
  const int planes = 2 * pool.H, per_part = (planes + io.parts - 1) / io.parts;
  const int y1 = min(part * per_part + per_part, planes);
  for (int y = part * per_part; y < y1; ++y) {
    const bool is_v = y >= pool.H;
    const int h = is_v ? y - pool.H : y;
    char* base = pool.base + (is_v ? pool.kv : 0) + h * pool.head;
    unsigned char* sbase = kQuant ? pool.scales + (is_v ? pool.s_kv : 0) + h * pool.s_head : nullptr;
    const long long x_tok = is_v ? io.v_tok : io.k_tok;
    X* x0 = reinterpret_cast<X*>(is_v ? io.v : io.k) + (long long)h * (is_v ? io.v_head : io.k_head) + i0 * x_tok;
    for (int t0 = 0; t0 < io.tokens; t0 += step * kUnroll) {
      uint32_t w[kUnroll][PIECES][kWords];
      uint4 q[kUnroll][PIECES];                           // the pool's side
      long long at[kUnroll], sat[kUnroll];
      int byte[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int tt = t0 + u * step + sub;
        at[u] = (long long)shfl64(0xffffffffu, (uint64_t)place, tt & 31);
        if (kQuant) sat[u] = (long long)shfl64(0xffffffffu, (uint64_t)splace, tt & 31);
        if (tt >= io.tokens) at[u] = -1;
        byte[u] = 127;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
          const int d = col + p * lanes * kN;
          const bool on = at[u] >= 0 && d < pool.D;
          if (TO_POOL) {
#pragma unroll
            for (int e = 0; e < kWords; ++e) w[u][p][e] = 0;
            if (on) load_words<X, kWords>(x0 + tt * x_tok + d, io.vec, w[u][p]);
          } else if (on) {
            q[u][p] = __ldg(reinterpret_cast<const uint4*>(base + at[u] + d * (kQuant ? 1 : 2)));
            if (kQuant) byte[u] = __ldg(sbase + sat[u]);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int tt = t0 + u * step + sub;
        float f = 1.0f;
        bool odd = false;                                  // somewhere in the warp's rows: not a finite number
        if constexpr (kQuant) {
          if (TO_POOL) {
            uint32_t top = 0;
#pragma unroll
            for (int p = 0; p < PIECES; ++p)
#pragma unroll
              for (int e = 0; e < kWords; ++e) top = max_bits<X>(top, w[u][p][e]);
            bool finite;
            float a = magnitude<X>(top, finite);
            odd = __any_sync(0xffffffffu, !finite);
            if (odd) {
              a = 0.0f;
#pragma unroll
              for (int p = 0; p < PIECES; ++p)
#pragma unroll
                for (int e = 0; e < kN; ++e) a = fmaxf(a, finite_abs(Elems<X>::get(w[u][p], e)));
            }
            for (int m = lanes >> 1; m > 0; m >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, m));
            byte[u] = scale_byte(a);
            f = power_of_byte(254 - byte[u]);
          } else {
            f = byte[u] == 255 ? NAN : power_of_byte(byte[u]);
          }
        }
        if (at[u] < 0) continue;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
          const int d = col + p * lanes * kN;
          if (d >= pool.D) continue;
          if (TO_POOL) {
            uint32_t* out = reinterpret_cast<uint32_t*>(&q[u][p]);
            if constexpr (kQuant) {
#pragma unroll
              for (int e = 0; e < kN; e += 4)
                out[e / 4] = e4m3_pair(Elems<X>::get(w[u][p], e) * f, Elems<X>::get(w[u][p], e + 1) * f, odd) |
                             (e4m3_pair(Elems<X>::get(w[u][p], e + 2) * f, Elems<X>::get(w[u][p], e + 3) * f, odd) << 16);
              if (p == 0 && col == 0) sbase[sat[u]] = (unsigned char)byte[u];
            } else if constexpr (kCopy) {
#pragma unroll
              for (int e = 0; e < 4; ++e) out[e] = w[u][p][e];
            } else {
#pragma unroll
              for (int e = 0; e < kN; e += 2)
                Elems<P>::put(out, e, Elems<X>::get(w[u][p], e), Elems<X>::get(w[u][p], e + 1));
            }
            *reinterpret_cast<uint4*>(base + at[u] + d * (kQuant ? 1 : 2)) = q[u][p];
          } else {
            const uint32_t* in = reinterpret_cast<const uint32_t*>(&q[u][p]);
            if constexpr (kQuant) {
#pragma unroll
              for (int e = 0; e < kN; e += 2) {
                const float2 y2 = __half22float2(halves_of_e4m3((in[e / 4] >> (16 * ((e >> 1) & 1))) & 0xffffu));
                Elems<X>::put(w[u][p], e, y2.x * f, y2.y * f);
              }
            } else if constexpr (kCopy) {
#pragma unroll
              for (int e = 0; e < 4; ++e) w[u][p][e] = in[e];
            } else {
#pragma unroll
              for (int e = 0; e < kN; e += 2) Elems<X>::put(w[u][p], e, Elems<P>::get(in, e), Elems<P>::get(in, e + 1));
            }
            store_words<X, kWords>(x0 + tt * x_tok + d, io.vec, w[u][p]);
          }
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
  constexpr int kN = std::is_same<P, E4M3>::value ? 16 : 8;
  const int pieces = pool.D / kN;
  io.lane_log = 0;
  while ((1 << io.lane_log) < pieces && io.lane_log < 5) ++io.lane_log;
  // Groups of 32 tokens, one warp per plane, once that gives every scheduler eight warps to switch
  // between; with fewer tokens smaller groups, down to one step of rows.
  const long long enough = (long long)sm_count() * 32;
  io.tokens = 32;
  while (io.tokens > (32 >> io.lane_log) && (b.n_tokens + io.tokens - 1) / io.tokens * 2 * pool.H < enough)
    io.tokens /= 2;
  const long long groups = (b.n_tokens + io.tokens - 1) / io.tokens;
  io.parts = 2 * pool.H;
  while (io.parts > 1 && groups * io.parts >= 64 * enough) io.parts = (io.parts + 1) / 2;
  const long long warps = groups * io.parts;
  const long long blocks = (warps + kPagedThreads / 32 - 1) / (kPagedThreads / 32);
  if (blocks >= (1LL << 31)) return AIBX_ERR_UNSUPPORTED;
  if (pieces <= 32)
    kv_token_kernel<TO_POOL, P, X, 1><<<(unsigned int)blocks, kPagedThreads, 0, st>>>(pool, b, io);
  else
    kv_token_kernel<TO_POOL, P, X, 32 / kN><<<(unsigned int)blocks, kPagedThreads, 0, st>>>(pool, b, io);
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
