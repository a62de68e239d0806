// Rotary positions: rows turned pair by pair, alone (rope) or on their way into the paged pool
// (rope_append: queries turned where they are, keys turned into their slots, values as they are).
//
//   y1 = g (x1 cos a - x2 sin a),  y2 = g (x2 cos a + x1 sin a),  a = position * frequency of the pair,
// with pairs (i, i + R/2) or (2 i, 2 i + 1) of a row's first R elements.  The angle is taken in turns, in
// 64 bits: t = position * (f / 2 pi), and t - rint(t) goes to the sine and cosine in 32 bits, so that far
// positions lose nothing (a 32-bit product would be off by 0.03 radians at position 500,000).  Products
// and sums of 32 bits, one rounding to what is stored; e4m3 rows take their scale from the turned values
// before any rounding.
//
// A warp takes some tokens and some planes (a head of Q, K or V); per token its lanes share out the sines and
// cosines, which then stay in registers for all planes.  A lane holds the two 8-element pieces of a row that
// belong to each other, so that a pair never leaves its lane.
// Bound: HBM for long inputs, each row being read once and written once (40,001 tokens of 32 fp16 heads: 109
// us, 6.0 TB/s; 26,600 tokens of 28 heads of queries and 4 of K and V into an e4m3 pool: 97 us, 4.8 TB/s, where
// the quantisation's instructions show; into a bf16 pool 92 us, 5.3 TB/s; fp32 rows 5.4 to 5.9 TB/s), the chain of
// dependent loads for few tokens (64 tokens: 6 us).
// 80 registers, for three CTAs an SM, are not enough for the pool's part beside two rows in flight: every rope_append
// keeps a stack (16-bit rows 32 to 52 bytes stored and 16 to 40 loaded per thread, fp32 rows 92 to 140 and 116 to
// 128), and so does fp32 rope alone (20 to 36 and 24 to 40); 16-bit rope keeps none.
#pragma once

#include "kv_paged.cuh"

namespace aibx {

struct RopeIO {
  char *q, *q_out, *k, *v;
  long long q_tok, q_head, o_tok, o_head, k_tok, k_head, v_tok, v_head;   // in elements
  const double* inv_freq;          // radians per position
  const int32_t* pos;              // null: the batch's positions
  float factor;
  int half;                        // rotated pairs of a row, a multiple of 8
  int q_heads, D;
  long long n_tokens;
  int lane_log;                    // log2 of the lanes that hold a row
  int tokens, parts;               // per warp; warps that share a group's planes
  int vec;                         // every row of the caller's 16-byte aligned
};

struct NoPool {};                  // tag: nothing but queries

constexpr int kRopeThreads = 256;
constexpr int kRopeMaxDim = 512;   // 32 lanes of 16 elements

// As load_words, of memory that this kernel may write (queries turned in place).
template <typename X, int N>
__device__ __forceinline__ void load_words_rw(const X* p, bool vec, uint32_t* w) {
  if (vec) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<uint4*>(w + i) = *(reinterpret_cast<const uint4*>(p) + i / 4);
  } else {
    load_words<X, N>(p, false, w);
  }
}

template <typename P, typename X, bool INTER>
__global__ void __launch_bounds__(kRopeThreads, 3)
rope_kernel(PagedPool pool, PagedBatch b, RopeIO io) {
  constexpr bool kPool = !std::is_same<P, NoPool>::value;
  constexpr bool kQuant = std::is_same<P, E4M3>::value;
  constexpr bool kCopy = std::is_same<P, X>::value;       // V needs no conversion
  constexpr int kW = 8 * (int)sizeof(X) / 4;              // words of a piece
  constexpr int kUnroll = 2;                              // rows in flight per lane
  extern __shared__ float2 s_turn[];                      // [warps][half]
  const long long unit = ((long long)blockIdx.x * kRopeThreads + threadIdx.x) >> 5;
  const long long group = unit / io.parts;
  const int part = (int)(unit - group * io.parts);
  const long long i0 = group * io.tokens;
  if (i0 >= io.n_tokens) return;
  const int lane = threadIdx.x & 31;
  float2* turn = s_turn + (threadIdx.x >> 5) * io.half;

  long long pos = kNoToken, place = -1, splace = 0;       // lane t: of token i0 + t
  if constexpr (kPool) {
    if (!warp_token_places<kQuant>(pool, b, i0, io.tokens, part == 0, pos, place, splace)) return;
    if (io.pos && pos != kNoToken) pos = __ldg(io.pos + i0 + (lane & (io.tokens - 1)));
  } else {
    const long long i = i0 + (lane & (io.tokens - 1));
    if (i < io.n_tokens) pos = __ldg(io.pos + i);
  }

  const int lanes = 1 << io.lane_log, step = 32 >> io.lane_log;
  const int sub = lane >> io.lane_log, u = lane & (lanes - 1);
  const int units = (io.D + 15) >> 4;
  const bool turns = u < io.half >> 3;                    // this lane's pieces are rotated
  const int oa = INTER || !turns ? 16 * u : 8 * u, ob = INTER || !turns ? 16 * u + 8 : io.half + 8 * u;
  const bool on_a = u < units, on_b = on_a && ob < io.D;
  const int heads = kPool ? pool.H : 0;
  const int planes = io.q_heads + 2 * heads, per_part = (planes + io.parts - 1) / io.parts;
  const int y1 = min(part * per_part + per_part, planes);

  for (int t = 0; t < io.tokens; ++t) {
    const long long p_t = (long long)shfl64(0xffffffffu, (uint64_t)pos, t);
    const long long at = kPool ? (long long)shfl64(0xffffffffu, (uint64_t)place, t) : -1;
    const long long sat = kQuant ? (long long)shfl64(0xffffffffu, (uint64_t)splace, t) : 0;
    if (p_t == kNoToken) continue;
    const long long i = i0 + t;
    float c[8], s[8];
    __syncwarp();
    for (int x = lane; x < io.half; x += 32) {
      double w = (double)p_t * (__ldg(io.inv_freq + x) * 0.15915494309189535);
      w -= rint(w);
      // what the turns lose in 32 bits is put back to first order (up to 2^-26 turns: as much as all else)
      const float near = (float)w, rest = (float)(w - near) * 6.283185307f;
      float sn, cs;
      sincospif(2.0f * near, &sn, &cs);
      turn[x] = make_float2((cs - sn * rest) * io.factor, (sn + cs * rest) * io.factor);
    }
    __syncwarp();
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float4 f = turns ? *reinterpret_cast<const float4*>(turn + 8 * u + e) : make_float4(1.0f, 0.0f, 1.0f, 0.0f);
      c[e] = f.x;
      s[e] = f.y;
      c[e + 1] = f.z;
      s[e + 1] = f.w;
    }
    // Queries and cached rows in loops of their own: what a pool of 8 bits needs would cost the queries, the
    // most of the rows, a third of their time.
    auto turn_rows = [&](auto of_q, int y0, int y_end) {
      constexpr bool kQ = decltype(of_q)::value;
      for (; y0 < y_end; y0 += step * kUnroll) {
        uint32_t a[kUnroll][kW], d[kUnroll][kW];          // the two pieces
#pragma unroll
        for (int r = 0; r < kUnroll; ++r) {
          const int y = y0 + r * step + sub;
          const X* src = reinterpret_cast<const X*>(io.q) + i * io.q_tok + (long long)y * io.q_head;
          if constexpr (!kQ)
            src = y < heads ? reinterpret_cast<const X*>(io.k) + i * io.k_tok + (long long)y * io.k_head
                            : reinterpret_cast<const X*>(io.v) + i * io.v_tok + (long long)(y - heads) * io.v_head;
#pragma unroll
          for (int e = 0; e < kW; ++e) a[r][e] = d[r][e] = 0;
          if (y < y_end && on_a) load_words_rw<X, kW>(src + oa, io.vec, a[r]);
          if (y < y_end && on_b) load_words_rw<X, kW>(src + ob, io.vec, d[r]);
        }
#pragma unroll
        for (int r = 0; r < kUnroll; ++r) {
          const int y = y0 + r * step + sub;
          const bool is_v = !kQ && y >= heads;
          const bool same = is_v || !turns;               // as it came
          float fa[8], fb[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            fa[e] = Elems<X>::get(a[r], e);
            fb[e] = Elems<X>::get(d[r], e);
          }
          if (!same) {
            if constexpr (INTER) {
#pragma unroll
              for (int e = 0; e < 8; e += 2) {
                const float xa = fa[e], xb = fb[e];
                fa[e] = xa * c[e / 2] - fa[e + 1] * s[e / 2];
                fa[e + 1] = fa[e + 1] * c[e / 2] + xa * s[e / 2];
                fb[e] = xb * c[4 + e / 2] - fb[e + 1] * s[4 + e / 2];
                fb[e + 1] = fb[e + 1] * c[4 + e / 2] + xb * s[4 + e / 2];
              }
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float x1 = fa[e], x2 = fb[e];
                fa[e] = x1 * c[e] - x2 * s[e];
                fb[e] = x2 * c[e] + x1 * s[e];
              }
            }
          }
          if constexpr (kQ) {
            if (y >= y_end || !on_a) continue;
            if (!same) {
#pragma unroll
              for (int e = 0; e < 8; e += 2) {
                Elems<X>::put(a[r], e, fa[e], fa[e + 1]);
                Elems<X>::put(d[r], e, fb[e], fb[e + 1]);
              }
            }
            X* dst = reinterpret_cast<X*>(io.q_out) + i * io.o_tok + (long long)y * io.o_head;
            store_words<X, kW>(dst + oa, io.vec, a[r]);
            if (on_b) store_words<X, kW>(dst + ob, io.vec, d[r]);
          } else if constexpr (kPool) {
            const int h = y - (is_v ? heads : 0);
            char* row = pool.base + at + (is_v ? pool.kv : 0) + h * pool.head;
            if constexpr (kQuant) {
              uint32_t top = 0;
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                top = max_bits<float>(top, __float_as_uint(fa[e]));
                top = max_bits<float>(top, __float_as_uint(fb[e]));
              }
              const bool odd = __any_sync(0xffffffffu, top >= 0x7f800000u);
              float m = __uint_as_float(top);
              if (odd) {
                m = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) m = fmaxf(m, fmaxf(finite_abs(fa[e]), finite_abs(fb[e])));
              }
              for (int x = lanes >> 1; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
              const int byte = scale_byte(m);
              const float f = power_of_byte(254 - byte);
              if (y >= y_end || !on_a) continue;
              uint32_t w[2][2];
#pragma unroll
              for (int e = 0; e < 8; e += 4) {
                w[0][e / 4] = e4m3_pair(fa[e] * f, fa[e + 1] * f, odd) | (e4m3_pair(fa[e + 2] * f, fa[e + 3] * f, odd) << 16);
                w[1][e / 4] = e4m3_pair(fb[e] * f, fb[e + 1] * f, odd) | (e4m3_pair(fb[e + 2] * f, fb[e + 3] * f, odd) << 16);
              }
              *reinterpret_cast<uint2*>(row + oa) = make_uint2(w[0][0], w[0][1]);
              if (on_b) *reinterpret_cast<uint2*>(row + ob) = make_uint2(w[1][0], w[1][1]);
              if (u == 0) pool.scales[sat + (is_v ? pool.s_kv : 0) + h * pool.s_head] = (unsigned char)byte;
            } else {
              if (y >= y_end || !on_a) continue;
              uint32_t w[2][4];
#pragma unroll
              for (int e = 0; e < 8; e += 2) {
                Elems<P>::put(w[0], e, fa[e], fa[e + 1]);
                Elems<P>::put(w[1], e, fb[e], fb[e + 1]);
              }
              if constexpr (kCopy) {
                if (same) {
#pragma unroll
                  for (int e = 0; e < 4; ++e) {
                    w[0][e] = a[r][e];
                    w[1][e] = d[r][e];
                  }
                }
              }
              *reinterpret_cast<uint4*>(row + 2 * oa) = make_uint4(w[0][0], w[0][1], w[0][2], w[0][3]);
              if (on_b) *reinterpret_cast<uint4*>(row + 2 * ob) = make_uint4(w[1][0], w[1][1], w[1][2], w[1][3]);
            }
          }
        }
      }
    };
    const int y0 = part * per_part;
    turn_rows(std::true_type(), y0, min(y1, io.q_heads));
    if constexpr (kPool)
      if (at >= 0) turn_rows(std::false_type(), max(y0 - io.q_heads, 0), y1 - io.q_heads);
  }
}

// ------------------------------------------------------------------------------------------
// host side

template <typename P, typename X, bool INTER>
inline int32_t launch_rope(const PagedPool& pool, const PagedBatch& b, RopeIO io, cudaStream_t st) {
  const int units = (io.D + 15) / 16, heads = std::is_same<P, NoPool>::value ? 0 : pool.H;
  io.lane_log = 0;
  while ((1 << io.lane_log) < units) ++io.lane_log;
  const int planes = io.q_heads + 2 * heads;
  const int rows = 2 * (32 >> io.lane_log);               // of a token that a warp has in flight
  const int most = (planes + rows - 1) / rows;
  const long long enough = (long long)sm_count() * 24;    // warps that the GPU holds at once
  io.tokens = 8;                                          // (at least two rounds of warps, or the last one shows:
  while (io.tokens > 1 && (io.n_tokens + io.tokens - 1) / io.tokens < 2 * enough) io.tokens /= 2;   // 128 instead of 109 us)
  const long long groups = (io.n_tokens + io.tokens - 1) / io.tokens;
  io.parts = 1;
  while (io.parts < most && groups * io.parts < enough) ++io.parts;
  const long long warps = groups * io.parts;
  const long long blocks = (warps + kRopeThreads / 32 - 1) / (kRopeThreads / 32);
  if (blocks >= (1LL << 31)) return AIBX_ERR_UNSUPPORTED;
  const size_t smem = (size_t)(kRopeThreads / 32) * io.half * sizeof(float2);   // at most 16 KB
  rope_kernel<P, X, INTER><<<(unsigned int)blocks, kRopeThreads, smem, st>>>(pool, b, io);
  return launch_status();
}

template <typename P>
inline int32_t launch_rope_kind(const PagedPool& pool, const PagedBatch& b, const RopeIO& io, int type, int style,
                                cudaStream_t st) {
#define AIBX_ROPE_CASE(X)                                                            \
  return style == AIBX_ROPE_INTERLEAVED ? launch_rope<P, X, true>(pool, b, io, st)   \
                                        : launch_rope<P, X, false>(pool, b, io, st);
  switch (type) {
    case AIBX_TYPE_BF16: AIBX_ROPE_CASE(__nv_bfloat16)
    case AIBX_TYPE_FP16: AIBX_ROPE_CASE(__half)
    default: AIBX_ROPE_CASE(float)
  }
#undef AIBX_ROPE_CASE
}

// What both calls check of the rotation; `work`: whether there are rows (then pointers count).
inline int32_t rope_check(const aibx_rope_t* rope, int head_dim, int type, bool work) {
  if (!rope || type_bytes(type) < 2) return AIBX_ERR_INVALID;
  if (rope->style != AIBX_ROPE_HALF && rope->style != AIBX_ROPE_INTERLEAVED) return AIBX_ERR_INVALID;
  if (rope->rotary_dim <= 0 || rope->rotary_dim > head_dim || rope->rotary_dim % 2 != 0) return AIBX_ERR_INVALID;
  if (rope->rotary_dim % 16 != 0 || head_dim > kRopeMaxDim || head_dim % 8 != 0) return AIBX_ERR_UNSUPPORTED;
  if (!work) return AIBX_OK;
  if (!rope->d_inv_freq || (reinterpret_cast<uintptr_t>(rope->d_inv_freq) & 7) ||
      (reinterpret_cast<uintptr_t>(rope->d_pos) & 3))
    return AIBX_ERR_INVALID;
  return AIBX_OK;
}

inline void rope_io(const aibx_rope_t* rope, int head_dim, RopeIO& io) {
  io.inv_freq = rope->d_inv_freq;
  io.pos = rope->d_pos;
  io.factor = rope->factor;
  io.half = rope->rotary_dim / 2;
  io.D = head_dim;
}

// Whether rows of D elements at t * tok + h * head, t < n and h < heads, lie upon one another.  Rows that follow one
// another and lists of them that do not touch are told at once; else, for a step in h, the nearest two in t.
inline bool rows_overlap(long long n, long long tok, long long heads, long long head, long long D) {
  if ((n > 1 && tok < D) || (heads > 1 && head < D)) return true;
  if (n <= 1 || heads <= 1) return false;
  if ((tok - D) / head >= heads - 1 || (head - D) / tok >= n - 1) return false;
  for (long long h = 1; h < heads; ++h) {
    const __int128 at = (__int128)h * head;
    const __int128 t = at / tok;
    if (t >= n) return false;                              // (all further ones are beyond, too)
    if (at - t * tok < D || (t + 1 < n && (t + 1) * tok - at < D)) return true;
  }
  return false;
}

// Pointers and strides of the caller's rows: whether they are usable at all, and in 16-byte pieces.
struct RopeRows {
  uintptr_t bits = 0;
  bool good = true;
  void add(const void* p, int64_t tok, int64_t head, int size) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(p);
    if (!p || tok < 0 || head < 0 || (x & (uintptr_t)(size - 1))) good = false;
    bits |= x | (uintptr_t)(tok * size) | (uintptr_t)(head * size);
  }
  int vec() const { return (bits & 15) == 0; }
};

inline int32_t rope_rows(const aibx_rope_t* rope, int64_t n, int32_t heads, int32_t head_dim, const void* x,
                         int64_t x_tok, int64_t x_head, void* y, int64_t y_tok, int64_t y_head, int32_t type,
                         cudaStream_t st) {
  if (n < 0 || heads < 0 || head_dim <= 0) return AIBX_ERR_INVALID;
  const bool work = n > 0 && heads > 0;
  const int32_t rc = rope_check(rope, head_dim, type, work);
  if (rc != AIBX_OK || !work) return rc;
  if (heads > 65536) return AIBX_ERR_UNSUPPORTED;
  if (!rope->d_pos) return AIBX_ERR_INVALID;
  RopeRows rows;
  rows.add(x, x_tok, x_head, type_bytes(type));
  rows.add(y, y_tok, y_head, type_bytes(type));
  if (!rows.good || rows_overlap(n, y_tok, heads, y_head, head_dim)) return AIBX_ERR_INVALID;
  // in place means each row onto itself
  if (x == y && ((n > 1 && x_tok != y_tok) || (heads > 1 && x_head != y_head))) return AIBX_ERR_INVALID;
  RopeIO io = {};
  rope_io(rope, head_dim, io);
  io.q = static_cast<char*>(const_cast<void*>(x));
  io.q_out = static_cast<char*>(y);
  io.q_tok = x_tok;
  io.q_head = x_head;
  io.o_tok = y_tok;
  io.o_head = y_head;
  io.q_heads = heads;
  io.n_tokens = n;
  io.vec = rows.vec();
  return launch_rope_kind<NoPool>(PagedPool{}, PagedBatch{}, io, type, rope->style, st);
}

inline int32_t rope_append(const aibx_kv_cache_t* c, const aibx_kv_batch_t* b, const aibx_rope_t* rope,
                           const aibx_rope_rows_t* r, cudaStream_t st) {
  PagedPool pool;
  PagedBatch batch;
  bool work;
  int32_t rc = paged_views(c, b, pool, batch, work);
  if (rc != AIBX_OK) return rc;
  if (!r || r->num_q_heads < 0) return AIBX_ERR_INVALID;
  rc = rope_check(rope, c->layout.head_dim, r->type, work);
  if (rc != AIBX_OK || !work) return rc;
  if (r->num_q_heads > 65536) return AIBX_ERR_UNSUPPORTED;
  const int size = type_bytes(r->type);
  RopeRows rows;
  rows.add(r->d_k, r->k_token_stride, r->k_head_stride, size);
  rows.add(r->d_v, r->v_token_stride, r->v_head_stride, size);
  if (r->num_q_heads > 0) {
    rows.add(r->d_q, r->q_token_stride, r->q_head_stride, size);
    rows.add(r->d_q_out, r->q_out_token_stride, r->q_out_head_stride, size);
    if (rows.good && rows_overlap(b->n_tokens, r->q_out_token_stride, r->num_q_heads, r->q_out_head_stride, pool.D))
      return AIBX_ERR_INVALID;
    if (r->d_q == r->d_q_out && ((b->n_tokens > 1 && r->q_token_stride != r->q_out_token_stride) ||
                                 (r->num_q_heads > 1 && r->q_head_stride != r->q_out_head_stride)))
      return AIBX_ERR_INVALID;
  }
  if (!rows.good) return AIBX_ERR_INVALID;
  RopeIO io = {};
  rope_io(rope, pool.D, io);
  io.q = static_cast<char*>(const_cast<void*>(r->d_q));
  io.q_out = static_cast<char*>(r->d_q_out);
  io.k = static_cast<char*>(const_cast<void*>(r->d_k));
  io.v = static_cast<char*>(const_cast<void*>(r->d_v));
  io.q_tok = r->q_token_stride;
  io.q_head = r->q_head_stride;
  io.o_tok = r->q_out_token_stride;
  io.o_head = r->q_out_head_stride;
  io.k_tok = r->k_token_stride;
  io.k_head = r->k_head_stride;
  io.v_tok = r->v_token_stride;
  io.v_head = r->v_head_stride;
  io.q_heads = r->num_q_heads;
  io.n_tokens = batch.n_tokens;
  io.vec = rows.vec();
  switch (c->type) {
    case AIBX_TYPE_BF16: return launch_rope_kind<__nv_bfloat16>(pool, batch, io, r->type, rope->style, st);
    case AIBX_TYPE_FP16: return launch_rope_kind<__half>(pool, batch, io, r->type, rope->style, st);
    default: return launch_rope_kind<E4M3>(pool, batch, io, r->type, rope->style, st);
  }
}

}  // namespace aibx
