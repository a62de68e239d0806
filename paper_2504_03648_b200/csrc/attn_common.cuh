// What the two kernels of attn_paged share: the call's arguments, how its work is cut and handed
// out, the tensor map of the pool, and the kernel that joins cut rows.
//
// Work is a line of KV tiles: request by request, (KV head, row block) by (KV head, row block), tile
// by tile.  CTA c of the persistent grid takes the c-th equal piece of that line, whatever
// the requests' lengths are: no CTA waits for a long request, and the host needs to know no
// length.  A piece that begins or ends inside a (request, head, row block) leaves unnormalised
// sums with their maximum in one of the CTA's two workspace slots; attn_join_kernel adds those
// up in line order, so the result does not depend on timing.
#pragma once

#include "kv_paged.cuh"

namespace aibx {

// Division of a row number n < 2^24 d by a small divisor d <= 128, as a multiplication: with
// m = ceil(2^40 / d), n m < 2^64, and n m / 2^40 exceeds n / d by less than n / 2^40 < 1 / d.
struct SmallDivisor {
  unsigned long long m;
  __device__ __forceinline__ int div(int n) const { return (int)(((unsigned long long)n * m) >> 40); }
};
// Trees: a token's mask bits from d on (d may be negative), as far as they name one of its request's n
// tokens.
__device__ __forceinline__ uint32_t tree_bits(const uint32_t* row, int words, int n, int d) {
  const int i = d >> 5;
  const uint32_t lo = i >= 0 && i < words ? __ldg(row + i) : 0u;
  const uint32_t hi = i >= -1 && i + 1 < words ? __ldg(row + i + 1) : 0u;
  const int there = min(max(n - d, 0), 32);
  return __funnelshift_r(lo, hi, d & 31) & (uint32_t)((1ull << there) - 1);
}

// How far a token stands above its request's cached ones: one less than the nodes that it sees of the tree.
__device__ __forceinline__ int tree_depth(const uint32_t* row, int words, int n) {
  int seen = 0;
  for (int i = 0; i < words && 32 * i < n; ++i) seen += __popc(tree_bits(row, words, n, 32 * i));
  return max(seen - 1, 0);
}

inline SmallDivisor small_divisor(int d) { return SmallDivisor{((1ull << 40) + d - 1) / d}; }

constexpr float kLog2E = 1.4426950408889634f;

struct AttnArgs {
  PagedPool pool;
  PagedBatch b;
  const char* q;
  char* out;
  float* lse;
  long long q_tok, q_head, o_tok, o_head;   // element strides
  float scale_log2;                         // scale * log2(e): scores in powers of two
  int G;                                    // query heads per KV head
  SmallDivisor by_g;
  int causal, window;
  SmallDivisor by_pos;                      // by_g where a row's position follows its token; 0 for trees
  const uint32_t* mask;                     // trees: 32-bit words of a token's mask, the lowest first
  int mask_words;                           // how many
  int box, box_log;                         // tokens one tensor-map box covers: a power of two
  int row_limit;                            // requests of up to so many rows (tokens * G) are the
                                            // row kernel's, 0: none
  int col_limit;                            // trees: the most rows of the requests that are the column kernel's
  int max_new;                              // bound on a request's tokens, 0: none given
  float* slots;                             // two per CTA, then a JoinRecord per CTA
};


struct AttnRequest {
  long long tok0;     // first row of the per-token tensors
  int n;              // new tokens
  int len;            // tokens in the cache
  int keys;           // of them, those the table has entries for
};

__device__ __forceinline__ AttnRequest attn_request(const PagedBatch& b, int T, int r) {
  AttnRequest q;
  q.tok0 = __ldg(b.tok_off + r);
  long long n = __ldg(b.tok_off + r + 1) - q.tok0;
  if (q.tok0 < 0) n = 0;
  if (n > b.n_tokens - q.tok0) n = b.n_tokens - q.tok0;
  q.n = n > 0 ? (int)n : 0;
  q.len = max(__ldg(b.kv_len + r), 0);
  const uint32_t* row;
  long long entries;
  table_row(b, r, row, entries);
  const long long cap = entries * T;
  q.keys = cap < q.len ? (int)max(cap, 0LL) : q.len;
  return q;
}

// Block-wide sum and exclusive prefix of one value per thread (N threads, scratch[33]).
template <int N>
__device__ __forceinline__ long long block_prefix(long long v, long long* scratch, long long& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long inc = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long up = (long long)shfl_up64((uint64_t)inc, d);
    if (lane >= d) inc += up;
  }
  if (lane == 31) scratch[warp] = inc;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < N / 32; ++w) {
    const long long s = scratch[w];
    if (w < warp) before += s;
    all += s;
  }
  __syncthreads();
  total = all;
  return before + inc - v;
}

struct WorkStart {
  long long total;      // tiles of the whole line
  long long base;       // first position of request r's part of the line
  int r;                // request in which this CTA's piece begins (-1: it is empty)
  int head, block, off; // and there: head, block of rows, tiles of it that belong to earlier pieces
  int cls, g;           // and where that stands in the request's order
};

// Finds the request that holds position `index * per` of the line, per = ceil(total / pieces).
// cost(r, on) = tiles of request r over all heads, asked by whole warps.  All N threads take part.
template <int N, typename Cost>
__device__ __forceinline__ void locate_piece(int R, unsigned int index, unsigned int pieces, long long* scratch,
                                             WorkStart* shared, const Cost& cost) {
  const int tid = threadIdx.x;
  const bool one = R <= N;                 // every request has a thread: one look at each
  long long mine = 0, total, base = 0;
  for (int r0 = 0; r0 < R; r0 += N) mine += cost(r0 + tid, r0 + tid < R);
  long long before = block_prefix<N>(mine, scratch, total);
  const long long per = (total + pieces - 1) / pieces;
  const long long target = per * index;
  if (tid == 0) {
    shared->total = total;
    shared->base = 0;
    shared->r = -1;                        // past the end: nothing to do
  }
  __syncthreads();
  if (target < total) {
    if (one) {
      if (mine > 0 && before <= target && target < before + mine) {
        shared->base = before;
        shared->r = tid;
      }
    } else {
      for (int r0 = 0; r0 < R; r0 += N) {
        const long long v = cost(r0 + tid, r0 + tid < R);
        long long sum;
        before = base + block_prefix<N>(v, scratch, sum);
        if (v > 0 && before <= target && target < before + v) {
          shared->base = before;
          shared->r = r0 + tid;
        }
        base += sum;
        if (base > target) break;
      }
    }
  }
  __syncthreads();
}

// What a CTA leaves for the join, beside its two slots: whether its first piece ends rows that an
// earlier CTA began, and which.  (Working this out again would cost the join what it cost here.)
struct alignas(16) JoinRecord {
  long long tok0;               // first token of the request
  int rows;                     // rows to join; 0: none
  int row0;                     // the first of them among the request's rows
  int head;
  int first_cta, first_slot;    // the CTA that holds the rows' first tiles, and its slot
  int pad;
};

// What one kernel leaves to be joined.  Slot of CTA x: 2 x for the piece it begins with, 2 x + 1 for
// the one it ends with, each holding `cap` maxima, `cap` sums and cap x D unnormalised outputs.
struct JoinSet {
  const float* slots;
  const JoinRecord* records;
  int cap;
};

// Waits for a phase of an mbarrier, at most two seconds; then (or once another warp has given up)
// the CTA's abort flag is set, TIMEOUT is in the device status, and every later wait returns at
// once: roles run to their end on whatever is in memory, and nobody is left at a barrier.
__device__ __forceinline__ bool ring_wait(unsigned int bar, unsigned int parity, volatile int* abort_flag) {
  if (mbar_try_wait(bar, parity)) return true;
  unsigned long long t0 = 0;
  for (unsigned int spins = 1;; ++spins) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((spins & 63u) == 0) {
      if (*abort_flag) return false;
      unsigned long long now;
      asm volatile("mov.u64 %0, %globaltimer;" : "=l"(now));
      if (t0 == 0) t0 = now;
      if (now - t0 > 2000000000ull) {
        if (!*abort_flag) raise_status(AIBX_ERR_TIMEOUT);
        *abort_flag = 1;
        return false;
      }
    }
  }
}

// The same for copies that must have landed before a CTA ends.
__device__ __forceinline__ void ring_drain(unsigned int bar, unsigned int parity) {
  for (unsigned int spins = 0; spins < (1u << 14) && !mbar_try_wait(bar, parity); ++spins) {
  }
}

// ------------------------------------------------------------------------------------------
// tensor map of a pool's layer: (element, slot, head, block, K/V)

__device__ __forceinline__ void tensor_load_5d(unsigned int dst, const CUtensorMap* map,
                                               unsigned int bar, int x, int slot, int head,
                                               int block, int kv) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(slot), "r"(head), "r"(block), "r"(kv)
      : "memory");
}

// 16-bit rows are cut into 128-byte columns whose 16-byte pieces are XORed with the row's place
// among eight (128-byte swizzle); so is a 128-byte e4m3 row.  64-byte rows stay as they are.
// dims: element of a column, slot, then three of {column, head, block, K/V}.
inline int32_t encode_pool_map(const PagedPool& p, int type, const void* base, const cuuint64_t* dims,
                               const cuuint64_t* strides, const cuuint32_t* box, CUtensorMap* map) {
  const EncodeTiledFn encode = encode_tiled_fn();
  if (!encode) return AIBX_ERR_CUDA;
  const cuuint32_t es[5] = {1, 1, 1, 1, 1};
  const CUtensorMapDataType dt = type == AIBX_TYPE_BF16   ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                 : type == AIBX_TYPE_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                          : CU_TENSOR_MAP_DATA_TYPE_UINT8;
  if (encode(map, dt, 5, const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
             p.D * type_bytes(type) >= 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
             CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return AIBX_ERR_UNSUPPORTED;
  return AIBX_OK;
}

inline int column_elems(const PagedPool& p, int type) {
  const int size = type_bytes(type);
  return p.D * size < 128 ? p.D : 128 / size;
}

// (element, slot, head, block, K/V): a box is one column of `box` slots.
inline int32_t pool_tensor_map(const PagedPool& p, int type, int box, CUtensorMap* map) {
  const cuuint64_t dims[5] = {(cuuint64_t)p.D, (cuuint64_t)p.T, (cuuint64_t)p.H, (cuuint64_t)p.num_blocks, 2};
  const cuuint64_t strides[4] = {(cuuint64_t)p.slot, (cuuint64_t)p.head, (cuuint64_t)p.block, (cuuint64_t)p.kv};
  const cuuint32_t bx[5] = {(cuuint32_t)column_elems(p, type), (cuuint32_t)box, 1, 1, 1};
  return encode_pool_map(p, type, p.base, dims, strides, bx, map);
}

// (element, slot, column, head, block) of K or of V: a box is `box` whole rows, column by column.
inline int32_t plane_tensor_map(const PagedPool& p, int type, int box, int kv, CUtensorMap* map) {
  const int col = column_elems(p, type);
  const cuuint64_t dims[5] = {(cuuint64_t)col, (cuuint64_t)p.T, (cuuint64_t)(p.D / col), (cuuint64_t)p.H,
                              (cuuint64_t)p.num_blocks};
  const cuuint64_t strides[4] = {(cuuint64_t)p.slot, 128, (cuuint64_t)p.head, (cuuint64_t)p.block};
  const cuuint32_t bx[5] = {(cuuint32_t)col, (cuuint32_t)box, (cuuint32_t)(p.D / col), 1, 1};
  return encode_pool_map(p, type, p.base + kv * p.kv, dims, strides, bx, map);
}

inline int gcd_int(int a, int b) {
  while (b) {
    const int t = a % b;
    a = b;
    b = t;
  }
  return a;
}

inline int log2_int(int power) {
  int k = 0;
  while ((1 << k) < power) ++k;
  return k;
}

// ------------------------------------------------------------------------------------------
// numbers

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <typename T>
struct Bits16;
template <>
struct Bits16<__nv_bfloat16> {
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ float2 unpack(uint32_t w) {
    return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w));
  }
};
template <>
struct Bits16<__half> {
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ float2 unpack(uint32_t w) {
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
  }
};

// Weights are held 2^kWeightHead up where they become fp16, whose normal numbers end at 2^-14: the
// running maximum m stands that much below the largest score, and follows once a score has grown by
// 2^8, so that weights reach up to 2^15 and keep all their bits down to 2^-21 of the largest.
template <typename T>
constexpr float kWeightHead = std::is_same<T, __half>::value ? 7.0f : 0.0f;

// Over e4m3 the weight that multiplies V carries V's exponent b_j beside the score, and m covers
// t_j + b_j.  b_j says little about the row's size where the scale byte is larger than its elements
// need: a row of zeros written by append has b = 0, beside b = -7 for rows of magnitude 3.  If such a
// row leads, all others' weights lie b_j (and its lead) below m, and fp16 would lose them.  So keys whose
// bytes lie more than kScaleSpread below the largest so far, or outside [kScaleLow, kScaleHigh], are
// multiplied "wide": weights as the sum of two bf16 numbers (16 bits, range 2^-126), V as bf16
// (exact: four bits).  b_j is taken within the range; the rest of it joins those bf16 numbers (the
// weights' in the row kernel, V's in the tile kernel), so that m, 2^b_j and the sum of 2^t_j stay within
// fp32 whatever the bytes are: a weight is lost below 2^-126 only, and then the key's score is 37 below
// another's (a factor of 2^37) at the least.
constexpr int kScaleLow = 79, kScaleHigh = 175, kScaleSpread = 4;

__device__ __forceinline__ int weight_byte(int byte) { return min(max(byte, kScaleLow), kScaleHigh); }

// A group of keys' V bytes, of those that a row may see: 16 + the least one (0 if one lies outside the
// range), and the largest.  255 (NaN) is outside, and not the largest.
__device__ __forceinline__ uint32_t scale_facts(uint32_t least16, uint32_t most) { return least16 | (most << 16); }
// Whether the group is multiplied wide; `most` = the largest byte so far, moved on.
__device__ __forceinline__ bool scales_wide(uint32_t facts, int& most) {
  most = max(most, (int)(facts >> 16));
  return most + 16 - (int)(facts & 0xffffu) > kScaleSpread;
}

// 2^-k and 2^k for the power k that brings a magnitude into [1, 2); k = 0 for 0, kept in range.
__device__ __forceinline__ void power_scale(float amax, float& down, float& up) {
  int k = (int)(__float_as_uint(amax) >> 23) - 127;
  if (!(amax > 0.0f)) k = 0;
  k = max(-120, min(k, 120));
  down = __uint_as_float((unsigned int)(127 - k) << 23);
  up = __uint_as_float((unsigned int)(127 + k) << 23);
}

// Joins rows that were cut: block c those that end in CTA c.  blockIdx.y takes 16 rows: the first
// y_rows of them of the row kernel's set, the others of the tile kernel's.
template <int D, typename QT>
__global__ void __launch_bounds__(256)
attn_join_kernel(const __grid_constant__ AttnArgs a, JoinSet rows, JoinSet tiles, int y_rows) {
  // Requests with more tokens than the caller's bound: looked for here, beside the kernel before,
  // where it costs the call nothing.
  if (a.max_new > 0 && blockIdx.x == 0 && blockIdx.y == 0)
    for (int r = threadIdx.x; r < a.b.R; r += 256)
      if (attn_request(a.b, a.pool.T, r).n > a.max_new) raise_status(AIBX_ERR_RANGE);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const bool of_rows = (int)blockIdx.y < y_rows;
  const int y = of_rows ? (int)blockIdx.y : (int)blockIdx.y - y_rows;
  const float* slots = of_rows ? rows.slots : tiles.slots;
  const int cap = of_rows ? rows.cap : tiles.cap;
  const JoinRecord rec = (of_rows ? rows.records : tiles.records)[blockIdx.x];
  const int c1 = (int)blockIdx.x;
  const size_t size = (size_t)cap * (D + 2);
  for (int x = threadIdx.x; x < 16 * (D / 4); x += 256) {
    const int i = y * 16 + x / (D / 4), d = (x % (D / 4)) * 4;
    if (i >= rec.rows) break;
    float top = -INFINITY, sum = 0.0f;
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int c = rec.first_cta; c <= c1; ++c) {
      const float* slot = slots + (size_t)(2 * c + (c == rec.first_cta ? rec.first_slot : 0)) * size;
      const float mc = slot[i], lc = slot[cap + i];
      const float4 o = *reinterpret_cast<const float4*>(slot + 2 * cap + (size_t)i * D + d);
      const float tn = fmaxf(top, mc);
      const float safe = tn == -INFINITY ? 0.0f : tn;
      const float f0 = exp2_fast(top - safe), f1 = exp2_fast(mc - safe);
      sum = sum * f0 + lc * f1;
      v.x = v.x * f0 + o.x * f1;
      v.y = v.y * f0 + o.y * f1;
      v.z = v.z * f0 + o.z * f1;
      v.w = v.w * f0 + o.w * f1;
      top = tn;
    }
    const int ri = rec.row0 + i, ti = a.by_g.div(ri);
    const long long tok = rec.tok0 + ti;
    const int qh = rec.head * a.G + (ri - ti * a.G);
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    QT* dst = reinterpret_cast<QT*>(a.out) + tok * a.o_tok + (long long)qh * a.o_head + d;
    *reinterpret_cast<uint2*>(dst) =
        make_uint2(Bits16<QT>::pack(v.x * inv, v.y * inv), Bits16<QT>::pack(v.z * inv, v.w * inv));
    if (a.lse && d == 0)
      a.lse[tok * (a.pool.H * a.G) + qh] = sum == 0.0f ? -INFINITY : 0.69314718056f * (top + log2f(sum));
  }
}

// The same for trees, whose rows over long contexts are cut into many pieces.  A warp takes a row or (EACH = 2)
// two: the pieces' maxima and sums a piece a lane, their outputs several at once.  blockIdx.y: 16 EACH rows of
// one set or the other.  Bound by the latency of three dependent loads and by blocks without rows: two rows a
// warp where there are the tile kernel's many (33 -> 25 us), one where latency is all (a draft of 26 nodes
// over 2,000 tokens 28.7 -> 26 us).
template <int D, typename QT, int EACH>
__global__ void __launch_bounds__(512, 2)
attn_join_tree_kernel(const __grid_constant__ AttnArgs a, JoinSet rows, JoinSet tiles, int y_rows) {
  // Requests with more tokens than the caller's bound, or than their masks can name
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int r = threadIdx.x; r < a.b.R; r += 512) {
      const int n = attn_request(a.b, a.pool.T, r).n;
      if ((a.max_new > 0 && n > a.max_new) || n > 32 * a.mask_words) raise_status(AIBX_ERR_RANGE);
    }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const bool of_rows = (int)blockIdx.y < y_rows;
  const int lane = threadIdx.x & 31, i0 = ((int)blockIdx.y - (of_rows ? 0 : y_rows)) * 16 * EACH + (int)(threadIdx.x >> 5);
  const float* slots = of_rows ? rows.slots : tiles.slots;
  const int cap = of_rows ? rows.cap : tiles.cap;
  const JoinRecord rec = (of_rows ? rows.records : tiles.records)[blockIdx.x];
  const size_t size = (size_t)cap * (D + 2);
  const int pieces = (int)blockIdx.x - rec.first_cta + 1;
  auto piece = [&](int k) { return slots + (size_t)(2 * (rec.first_cta + k) + (k == 0 ? rec.first_slot : 0)) * size; };
  if (i0 >= rec.rows) return;
  constexpr int kStep = 16;
  float top[EACH], sum[EACH], v[EACH][D / 32];
#pragma unroll
  for (int x = 0; x < EACH; ++x) {
    top[x] = -INFINITY;
    sum[x] = 0.0f;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) v[x][e] = 0.0f;
  }
  for (int k = lane; k < pieces; k += 32)
#pragma unroll
    for (int x = 0; x < EACH; ++x)
      if (i0 + x * kStep < rec.rows) top[x] = fmaxf(top[x], piece(k)[i0 + x * kStep]);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1)
#pragma unroll
    for (int x = 0; x < EACH; ++x) top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], d));
  for (int k0 = 0; k0 < pieces; k0 += 32) {
    float f[EACH];
#pragma unroll
    for (int x = 0; x < EACH; ++x) {
      const int i = i0 + x * kStep;
      f[x] = 0.0f;
      if (k0 + lane < pieces && i < rec.rows) {
        f[x] = exp2_fast(piece(k0 + lane)[i] - (top[x] == -INFINITY ? 0.0f : top[x]));
        sum[x] += piece(k0 + lane)[cap + i] * f[x];
      }
    }
    const int n = min(pieces - k0, 32);
#pragma unroll 4
    for (int k = 0; k < n; ++k) {
      const float* from = piece(k0 + k) + 2 * cap + lane * (D / 32);
#pragma unroll
      for (int x = 0; x < EACH; ++x) {
        const float w = __shfl_sync(0xffffffffu, f[x], k);
        const float* o = from + (size_t)min(i0 + x * kStep, rec.rows - 1) * D;
#pragma unroll
        for (int e = 0; e < D / 32; e += 2) {
          const float2 z = *reinterpret_cast<const float2*>(o + e);
          v[x][e] += z.x * w;
          v[x][e + 1] += z.y * w;
        }
      }
    }
  }
#pragma unroll
  for (int x = 0; x < EACH; ++x) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum[x] += __shfl_xor_sync(0xffffffffu, sum[x], d);
    const int i = i0 + x * kStep;
    if (i >= rec.rows) continue;
    const int ri = rec.row0 + i, ti = a.by_g.div(ri);
    const long long tok = rec.tok0 + ti;
    const int qh = rec.head * a.G + (ri - ti * a.G);
    const float inv = sum[x] == 0.0f ? 0.0f : 1.0f / sum[x];
    uint32_t* dst = reinterpret_cast<uint32_t*>(reinterpret_cast<QT*>(a.out) + tok * a.o_tok + (long long)qh * a.o_head) + lane * (D / 64);
#pragma unroll
    for (int e = 0; e < D / 32; e += 2) dst[e / 2] = Bits16<QT>::pack(v[x][e] * inv, v[x][e + 1] * inv);
    if (a.lse && lane == 0)
      a.lse[tok * (a.pool.H * a.G) + qh] = sum[x] == 0.0f ? -INFINITY : 0.69314718056f * (top[x] + log2f(sum[x]));
  }
}

template <int D, typename QT, bool TREE>
inline int32_t launch_join(const AttnArgs& a, const JoinSet& rows, const JoinSet& tiles, cudaStream_t st) {
  const int each = TREE && tiles.cap > 0 ? 32 : 16;        // rows of a block
  const int y_rows = (rows.cap + each - 1) / each, y_tiles = (tiles.cap + each - 1) / each;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned int)sm_count(), (unsigned int)(y_rows + y_tiles));
  cfg.blockDim = dim3(TREE ? 512 : 256);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  if constexpr (TREE) {
    if (each == 32)
      cudaLaunchKernelEx(&cfg, attn_join_tree_kernel<D, QT, 2>, a, rows, tiles, y_rows);
    else
      cudaLaunchKernelEx(&cfg, attn_join_tree_kernel<D, QT, 1>, a, rows, tiles, y_rows);
  } else {
    cudaLaunchKernelEx(&cfg, attn_join_kernel<D, QT>, a, rows, tiles, y_rows);
  }
  return launch_status();
}

}  // namespace aibx
