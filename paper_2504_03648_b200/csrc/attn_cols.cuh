// Attention of a drafted tree's nodes over a paged cache: more than 8 and up to some hundred query rows
// (nodes * query heads per KV head) of a (request, KV head), on the 5th-generation tensor cores.
//
// Few rows against many keys: the keys are the M of both products and the rows their N, so that work
// shrinks with the rows (a tile of 128 rows, filled or not, costs its softmax 128 exponentials a key; here
// a row costs one).  A block of up to N rows meets KV tiles of 128 positions:
//   S^T = K Q^T        [128 keys][rows], K and Q from shared memory, S^T in tensor memory (fp32)
//   P^T = 2^(S^T c - m)   one thread per key and a quarter or half of the rows; P^T to shared memory, 16-bit
//   O^T += V^T P^T     [dims][rows], V as it lies in the pool ([position][dim]: V^T's M-major form)
// A row's maximum runs across the threads, which is what makes this form dear; but m needs to move only
// when a score passes it by 2^8 (weights up to 2^8 are as good as weights up to 1).  So a tile costs one
// comparison per score and one vote of the warpgroup; maxima over keys are taken in the rare tile where the
// vote says so (a segment's first).  The sums l stay per key and are added up once, at the end.
//
// Visible: cached positions (window: those near enough to the row's node) and the nodes whose bit is set
// in the row's mask; a thread looks at bits only in tiles that touch the nodes.
//
// Over an e4m3 pool K of D = 128 is multiplied as it lies, 8 bits by 8 bits: a query becomes the sum of three
// e5m2 numbers, whose products with K add up in one accumulator (converting K instead, 28 rows:
// 316 us where this took 226).  K of D = 64, whose rows do not fill an operand's, two warpgroups turn into fp16 as it
// arrives, exact.  K's scales the thread that has the key applies to its scores.  V the same two turn into bf16,
// exact too; its scales go with the weights, in bf16, whose range holds them however far apart they are
// (scale bytes outside [kScaleLow, kScaleHigh] leave the rest with V).  Weights are the sum of two bf16 numbers: one
// has 8 bits, where fp16, which the tile and row kernels have, has 11.  P^T holds the first and the second side by
// side, as twice the rows; so does O^T, whose halves are added at the end.
//
// Roles: four softmax warpgroups (e4m3 and 32 rows: two), each with its part of the rows, which never wait
// for each other; a warp for S^T and one for O^T; a loader of K and one of V; over e4m3 eight that convert and
// fetch the scale bytes.  Rings of K and of V tiles of their own, S^T twice, so that S^T(j + 1) runs beside the
// softmax of tile j.  What a warp of the softmax keeps for rare paths is read again there: with all of it in
// registers the main loop spilled (32 requests of 32 nodes, 230 instead of 163 us).
//
// Bound, 16-bit: HBM, 2,740 cycles a tile of 128 keys of D = 128 (this SM's share); the products take 8 N
// cycles of the tensor pipe.  32 requests over 2k to 8k cached tokens of 8 heads: 123 us for 16 rows (5.4
// TB/s), 136 for 64, 166 for 128 (4.1 TB/s, where the softmax takes as long as the bytes); 48 requests of 4
// nodes 161 us (5.5 TB/s).  Without a segment's sums and outputs (a copy, for timing): 141 us for 128 rows.
// e4m3: 1,370 cycles would be the share of HBM, a tile takes 2,900 (8 requests over 60k to 131k tokens, 28
// rows: 260 us, 3.1 TB/s; 63 rows: 327): the conversion of V (with half the warps for it 329 us where this took
// 230) and the weights' two numbers (with one, of 8 bits, 230 and 288 us).
#pragma once

#include "attn_tiles.cuh"

namespace aibx {

// Rows cut evenly into the fewest blocks of up to MOST; every block sees the same tiles.
template <int MOST>
struct EvenBlocks {
  static __device__ __forceinline__ int size(int rows) {
    const int blocks = (int)(((long long)rows + MOST - 1) / MOST);
    return (int)(((long long)rows + blocks - 1) / blocks);
  }
  // (requests of more rows than col_limit are the tile kernel's)
  static __device__ __forceinline__ int blocks(const AttnArgs& a, const AttnRequest& q) {
    const long long rows = (long long)q.n * a.G;
    if (rows == 0 || rows > a.col_limit) return 0;
    const int each = size((int)rows);
    return (int)((rows + each - 1) / each);
  }
  static __device__ __forceinline__ TileSpan span(const AttnArgs& a, const AttnRequest& q, int) {
    const long long first = (long long)q.len - q.n;
    TileSpan s;
    s.hi = q.keys;
    const long long lo = a.window > 0 ? first - a.window + 1 : 0;
    s.lo = lo < 0 ? 0 : lo > s.hi ? s.hi : (int)lo;
    s.tile0 = s.lo / kTileKeys;
    s.tiles = max(1, (int)(((unsigned int)s.hi + kTileKeys - 1) / kTileKeys) - s.tile0);
    return s;
  }
};

// Tiles of a request over all heads.
template <typename B>
struct EvenCost {
  const AttnArgs& a;
  __device__ __forceinline__ long long operator()(int r, bool on) const {
    if (!on) return 0;
    const AttnRequest q = attn_request(a.b, a.pool.T, r);
    return (long long)B::blocks(a, q) * B::span(a, q, 0).tiles * a.pool.H;
  }
};

// By one thread: where in its request a piece begins.  As locate_block, whose order of segments it keeps, but
// with as many tiles in every segment there is nothing to search.
template <typename B>
__device__ __forceinline__ void locate_even(const AttnArgs& a, unsigned int index, unsigned int pieces, WorkStart* w) {
  if (w->r < 0) return;
  const AttnRequest q = attn_request(a.b, a.pool.T, w->r);
  const long long per = (w->total + pieces - 1) / pieces;
  const int blocks = B::blocks(a, q), tiles = B::span(a, q, 0).tiles;
  const long long segments = (long long)blocks * a.pool.H;
  long long g = (segments * tiles + per / 2) / per;        // as in request_line
  g = g < 1 ? 1 : g > segments ? segments : g;
  const long long off = per * index - w->base;
  long long k = off / tiles, cls;                          // k-th segment in the order
  const long long some = segments / g, more = segments - some * g;   // classes of some + 1 segments: `more` of them
  if (k < more * (some + 1)) {
    cls = k / (some + 1);
    k -= cls * (some + 1);
  } else {
    k -= more * (some + 1);
    cls = more + k / some;
    k -= (cls - more) * some;
  }
  const long long segment = cls + k * g;
  w->off = (int)(off - off / tiles * tiles);
  w->head = (int)(segment / blocks);
  w->block = (int)(segment - (long long)w->head * blocks);
  w->cls = (int)cls;
  w->g = (int)g;
}

template <int D, bool F8, int N>
struct ColShape {
  // Softmax warpgroups.  Over e4m3 two for 32 rows: with four the waits of twice the warps stand in the converters'
  // way (28 rows: 281 instead of 273 us at D = 64, 256 instead of 259 at 128); for 64 rows four (with two, whose
  // registers spill, 63 rows with weights of two numbers took 411 instead of 340 us; now 327).
  static constexpr int kGroups = F8 && N == 32 ? 2 : 4;
  static constexpr int kConverters = F8 ? 2 : 0;           // warpgroups that convert
  static constexpr int kThreads = 128 * (kGroups + 1 + kConverters);
  static constexpr int kCols = D / 64;                     // 128-byte columns of an operand row
  static constexpr int kColBytes = 128 * 128;
  static constexpr int kRaw = kTileKeys * D;               // a tile's e4m3 rows, as they arrive
  static constexpr int kBuf = kTileKeys * D * 2 + (F8 && D == 64 ? kRaw : 0);   // as in TileShape
  // K as it lies, if a row's 8-bit numbers fill the 128 bytes of an operand row
  static constexpr bool kPlain = F8 && D == 128;
  static constexpr int kKBuf = kPlain ? kRaw : kBuf;
  static constexpr int kParts = F8 ? 2 : 1;                // 16-bit numbers that make up a weight
  static constexpr int kPRows = kParts * N;                // rows of P^T and O^T
  static constexpr int kP = kTileKeys * 128 * ((kPRows + 63) / 64);   // P^T: 64 rows in 128 bytes a key
  static constexpr int kRoom = 216 * 1024;
};
// What is left of shared memory goes to the rings.
template <int D, bool F8, int N>
struct ColRings : ColShape<D, F8, N> {
  using B = ColShape<D, F8, N>;
  static constexpr int kPs = N <= 64 ? 2 : 1;              // P^T of that many tiles
  static constexpr int kQParts = B::kPlain ? 3 : 1;        // 8-bit numbers that make up a query's
  static constexpr int kQ = B::kPlain ? kQParts * N * 128 : B::kCols * B::kColBytes * N / 128;
  static constexpr int kLeft = B::kRoom - kQ - kPs * B::kP - 1024;
  static constexpr int kHalf = kLeft / (B::kKBuf + B::kBuf);
  static constexpr int kV = (kLeft - kHalf * B::kKBuf) / B::kBuf < 4 ? (kLeft - kHalf * B::kKBuf) / B::kBuf : 4;
  static constexpr int kK = (kLeft - kV * B::kBuf) / B::kKBuf < 4 ? (kLeft - kV * B::kBuf) / B::kKBuf : 4;
  static constexpr int kVAt = kK * B::kKBuf, kQAt = kVAt + kV * B::kBuf, kPAt = kQAt + kQ;
  static constexpr int kSmem = kPAt + kPs * B::kP + 1024;
  static constexpr int kSlot = N * (D + 2);                // floats per workspace slot
  // 16 bits: 4 * 104 + 64 = 5 * 96 (launch); e4m3: 2 * 136 + 64 + 2 * 72 = 5 * 96, or 4 * 72 + 64 + 2 * 72 < 7 * 72
  // (64 rows of e4m3 spill 8 bytes of the 72 registers)
  static constexpr int kRegsSoftmax = !F8 ? 104 : N == 32 ? 136 : 72;
  static constexpr int kRegsOther = 64, kRegsConvert = 72;
  static_assert(kK >= 2 && kV >= 2, "two tiles of each at least");
};

// fp32 accumulator, M = 128; operands as they lie (K-major), or both M- and N-major
__host__ __device__ constexpr unsigned int col_mma_desc(bool half, int n, bool major) {
  return (1u << 4) | ((half ? 0u : 1u) << 7) | ((half ? 0u : 1u) << 10) | (major ? 3u << 15 : 0u) |
         ((unsigned int)(n >> 3) << 17) | ((128u >> 4) << 24);
}

// The same of e4m3 numbers by e5m2 numbers (K = 32), both K-major.
__host__ __device__ constexpr unsigned int col_mma_desc8(int n) {
  return (1u << 4) | (1u << 10) | ((unsigned int)(n >> 3) << 17) | ((128u >> 4) << 24);
}
__device__ __forceinline__ void mma_smem8(unsigned int d, uint64_t a, uint64_t b, unsigned int idesc, unsigned int add,
                                          unsigned int leader) {
  asm volatile(
      "{\n.reg .pred p, q;\nsetp.ne.u32 p, %4, 0;\nsetp.ne.u32 q, %5, 0;\n"
      "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(add), "r"(leader)
      : "memory");
}

__device__ __forceinline__ void tmem_ld8(unsigned int addr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(addr));
}
__device__ __forceinline__ void tmem_st8(unsigned int addr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(addr)
               : "memory");
}

// Whether any thread of a warpgroup says so (named barrier `id`, 128 threads).
__device__ __forceinline__ bool group_any(int id, bool mine) {
  unsigned int any;
  asm volatile(
      "{\n.reg .pred p, q;\nsetp.ne.u32 p, %1, 0;\nbarrier.cta.red.or.pred q, %2, 128, p;\nselp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(any)
      : "r"((unsigned int)mine), "r"(id)
      : "memory");
  return any != 0;
}
__device__ __forceinline__ void group_sync(int id) { asm volatile("bar.sync %0, 128;" ::"r"(id) : "memory"); }

// Two e5m2 numbers, and as halves again: those, without the lower byte.
__device__ __forceinline__ uint32_t e5m2_pair(float a, float b) {
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E5M2);
}
__device__ __forceinline__ __half2 halves_of_e5m2(uint32_t pair) {
  const uint32_t w = __byte_perm(pair, 0, 0x1404);
  return *reinterpret_cast<const __half2*>(&w);
}

// The largest of those that are not NaN (max3 would give NaN).
__device__ __forceinline__ float max3_numbers(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// Whole numbers that order as the floats do (not for NaN).
__device__ __forceinline__ int float_order(float x) {
  const int u = __float_as_int(x);
  return u ^ ((u >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float order_float(int k) { return __int_as_float(k ^ ((k >> 31) & 0x7fffffff)); }

constexpr int kColBatch = 4, kColInfo = 4;                 // scale bytes: tiles at a time, and batches in the ring

template <int D, bool F8, typename QT, int N>
__global__ void __launch_bounds__(ColShape<D, F8, N>::kThreads, 1)
attn_cols_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ AttnArgs a) {
  using S = ColRings<D, F8, N>;
  using Blocks = EvenBlocks<N>;
  using KT = typename std::conditional<F8, __half, QT>::type;            // operands of S^T
  using VT = typename std::conditional<F8, __nv_bfloat16, QT>::type;     // and of O^T
  constexpr int kParts = S::kParts, kMine = N / S::kGroups, kChunks = kMine / 8;   // rows of a softmax warpgroup, 8 at a time
  constexpr int kQK = 4 * S::kGroups, kPV = kQK + 2, kLoadV = kQK + 3;   // warps (kQK + 1 loads K)
  extern __shared__ unsigned char s_raw[];
  __shared__ __align__(8) unsigned long long s_k_full[S::kK], s_k_empty[S::kK], s_k_raw[S::kK];
  __shared__ __align__(8) unsigned long long s_v_full[S::kV], s_v_empty[S::kV], s_v_raw[S::kV];
  __shared__ __align__(8) unsigned long long s_s_full[2], s_s_free[2], s_q_full, s_p_full[2], s_pv_done[2];
  __shared__ __align__(8) unsigned long long s_vote[S::kGroups];
  __shared__ int s_grow[S::kGroups][2];                    // a vote's outcome
  __shared__ __align__(8) unsigned long long s_info_full[kColInfo], s_info_empty[kColInfo];
  __shared__ unsigned int s_mask[kInfoRing];
  __shared__ __align__(16) float s_ref[N], s_scale[N], s_al[N];     // m (0 where no key was seen yet) and scale of each row
  __shared__ float s_top[N], s_inv[N];
  __shared__ int s_new[N], s_low[N], s_tok[N];
  __shared__ long long s_out[N];
  __shared__ float s_part[4][N];
  __shared__ __align__(4) unsigned char s_bytes[F8 ? kColInfo * kColBatch : 1][2][kTileKeys];
  __shared__ int s_odd[kColInfo * kColBatch][4];                     // whether V's bytes leave a rest with V, by 32 keys
  __shared__ long long s_scan[33];
  __shared__ WorkStart s_start;
  __shared__ TileWalk<Blocks> s_walk[S::kThreads / 32];
  __shared__ unsigned int s_tmem;
  __shared__ int s_abort;

  const unsigned int smem0 = (smem_u32(s_raw) + 1023u) & ~1023u;
  unsigned char* base = s_raw + (smem0 - smem_u32(s_raw));
  const unsigned int k0 = smem0, v0 = smem0 + S::kVAt;
  const int lane = threadIdx.x & 31;
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  volatile int* abort_flag = &s_abort;

  if (threadIdx.x == 0) {
    for (int i = 0; i < S::kK; ++i) {
      mbar_init(smem_u32(&s_k_full[i]), F8 && !S::kPlain ? 128u * S::kConverters : 1u);
      mbar_init(smem_u32(&s_k_empty[i]), 1u);
      mbar_init(smem_u32(&s_k_raw[i]), 1u);
    }
    for (int i = 0; i < S::kV; ++i) {
      mbar_init(smem_u32(&s_v_full[i]), F8 ? 128u * S::kConverters : 1u);
      mbar_init(smem_u32(&s_v_empty[i]), 1u);
      mbar_init(smem_u32(&s_v_raw[i]), 1u);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&s_s_full[i]), 1u);
      mbar_init(smem_u32(&s_s_free[i]), 4u * S::kGroups);
      mbar_init(smem_u32(&s_p_full[i]), 4u * S::kGroups);
      mbar_init(smem_u32(&s_pv_done[i]), 1u);
    }
    for (int i = 0; i < kColInfo; ++i) {
      mbar_init(smem_u32(&s_info_full[i]), 4u * (F8 ? S::kConverters : 1));
      mbar_init(smem_u32(&s_info_empty[i]), 4u * (S::kGroups + S::kConverters));
    }
    mbar_init(smem_u32(&s_q_full), 128u * S::kGroups);
    for (int i = 0; i < S::kGroups; ++i) {
      mbar_init(smem_u32(&s_vote[i]), 4u);
      s_grow[i][0] = s_grow[i][1] = 0;
    }
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == kQK) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    tmem_before();
  }
  const EvenCost<Blocks> cost{a};
  locate_piece<S::kThreads>(a.b.R, blockIdx.x, gridDim.x, s_scan, &s_start, cost);
  const long long per = (s_start.total + gridDim.x - 1) / gridDim.x;
  if (warp == 0) {
    // one thread finds the place, all warps start from copies of it
    if (lane == 0) {
      locate_even<Blocks>(a, blockIdx.x, gridDim.x, &s_start);
      s_walk[0].init(a, s_start, blockIdx.x, gridDim.x);
    }
    __syncwarp();
    constexpr int kWords = (int)(sizeof(TileWalk<Blocks>) / 4);
    const uint32_t* from = reinterpret_cast<const uint32_t*>(&s_walk[0]);
    for (int x = lane; x < (S::kThreads / 32 - 1) * kWords; x += 32)
      reinterpret_cast<uint32_t*>(&s_walk[1])[x] = from[x % kWords];
  }
  __syncthreads();
  tmem_after();
  const unsigned int tmem = s_tmem;                        // columns: S^T 0 and 128, O^T 256
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  TileWalk<Blocks>& walk = s_walk[warp];

  if (warp < kQK) {
    // ================================================================ softmax: thread = key
    regs_up<S::kRegsSoftmax>();
    const int w = warp >> 2, id = 1 + w;                   // warpgroup and its barrier
    const int tid = threadIdx.x & 127;                     // key in the tile; of O^T, the dimension
    const unsigned int lanes = (unsigned int)(warp & 3) << 21;
    const unsigned int tm_s = tmem + lanes, tm_o = tmem + lanes + 256;
    unsigned char* s_q = base + S::kQAt;
    const int c0 = w * kMine;                              // first of this warpgroup's rows in a block
    unsigned int step = 0, votes = 0, batch = 0;
    auto pv_wait = [&](unsigned int x) {                   // the product of step x is done, and so are all before
      ring_wait(smem_u32(&s_pv_done[x % S::kPs]), (x / S::kPs) & 1u, abort_flag);
      __syncwarp();
      tmem_after();
    };
    while (walk.next_warp(a, per)) {
      const int steps = walk.t1 - walk.t0;
      // (What only the rare paths need is read from the walk again where it is: a register saved.)
      auto block_row0 = [&]() { return walk.block * Blocks::size(walk.q.n * a.G); };
      // ---- what is known of each row
      const int rows = walk.rows(a), row0 = block_row0();
      if (tid < kMine) {
        const int ri = row0 + min(c0 + tid, rows - 1), ti = a.by_g.div(ri);
        s_tok[c0 + tid] = ti;
        s_out[c0 + tid] = (walk.q.tok0 + ti) * a.o_tok + (long long)(walk.head * a.G + (ri - ti * a.G)) * a.o_head;
        int low = walk.span.lo;
        if (a.window > 0) {
          const int depth = tree_depth(a.mask + (walk.q.tok0 + ti) * a.mask_words, a.mask_words, walk.q.n);
          low = (int)max((long long)low, (long long)walk.q.len - walk.q.n + depth - a.window + 1);
        }
        s_low[c0 + tid] = low;
        s_ref[c0 + tid] = 0.0f;
        s_top[c0 + tid] = -INFINITY;
        s_new[c0 + tid] = float_order(-INFINITY);
      }
      // ---- queries into shared memory (the last product that read them is done: its S^T was seen)
      {
        constexpr int kPieces = D / 8;                     // 16-byte pieces of a row
        const int c = tid % kPieces;
        unsigned char* dst = s_q + (c >> 3) * (S::kQ / S::kCols);
        constexpr int kBatch = 4;
        for (int i0 = tid / kPieces; i0 < kMine; i0 += kBatch * (128 / kPieces)) {
          uint4 batch[kBatch];
#pragma unroll
          for (int u = 0; u < kBatch; ++u) {
            const int ri = row0 + min(c0 + i0 + u * (128 / kPieces), rows - 1);
            const int ti = a.by_g.div(ri), gi = ri - ti * a.G;
            batch[u] = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const QT*>(a.q) +
                                                            (walk.q.tok0 + ti) * a.q_tok +
                                                            (long long)(walk.head * a.G + gi) * a.q_head + c * 8));
          }
#pragma unroll
          for (int u = 0; u < kBatch; ++u) {
            const int i = c0 + i0 + u * (128 / kPieces);
            const bool on = i0 + u * (128 / kPieces) < kMine;
            uint4 v = i < rows ? batch[u] : make_uint4(0, 0, 0, 0);
            if constexpr (F8) {
              uint32_t x[4] = {v.x, v.y, v.z, v.w};
              float amax = 0.0f;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float2 f = Bits16<QT>::unpack(x[e]);
                amax = fmaxf(amax, fmaxf(fabsf(f.x), fabsf(f.y)));
              }
#pragma unroll
              for (int m = 1; m < kPieces; m <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, m));
              float down, up;
              power_scale(S::kPlain ? amax * (1.0f / 128.0f) : amax, down, up);
              if constexpr (S::kPlain) {
                // The row's largest element into [128, 256), then all as the sum of e5m2 numbers: each takes three
                // bits of what the ones before have left, and its sign one more from the second on, so that three
                // make an fp16 number (of its 11 bits the first leaves at most 128 units, the second 8, which the
                // third has).  Their steps end at 2^-16: elements lose what is below 2^-24 of the largest, as where
                // queries are fp16 (two e4m3 numbers, whose steps end at 2^-9, kept 2^-17).  The power is that of
                // amax / 128, which power_scale need not cut short however large amax is; the smallest it does cut
                // short, at 2^120, and bf16's steps of 2^-133 are multiples of 2^-16 then.
                if (!(amax < INFINITY)) up = NAN;          // (saturated: these bits have no infinity)
                float2 f[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  f[e] = Bits16<QT>::unpack(x[e]);
                  f[e].x *= down;
                  f[e].y *= down;
                }
#pragma unroll
                for (int part = 0; part < S::kQParts; ++part) {
                  uint32_t y[4];
#pragma unroll
                  for (int e = 0; e < 4; ++e) {
                    y[e] = e5m2_pair(f[e].x, f[e].y);
                    const float2 g = __half22float2(halves_of_e5m2(y[e]));
                    f[e].x -= g.x;
                    f[e].y -= g.y;
                  }
                  if (on)
                    *reinterpret_cast<uint2*>(s_q + part * N * 128 + i * 128 + (((c >> 1) ^ (i & 7)) << 4) + (c & 1) * 8) =
                        make_uint2(y[0] | y[1] << 16, y[2] | y[3] << 16);
                }
              } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const float2 f = Bits16<QT>::unpack(x[e]);
                  x[e] = Bits16<KT>::pack(f.x * down, f.y * down);
                }
                v = make_uint4(x[0], x[1], x[2], x[3]);
              }
              if (on && c == 0) s_scale[i] = a.scale_log2 * up;
            }
            if (on && !S::kPlain) *reinterpret_cast<uint4*>(dst + i * 128 + (((c & 7) ^ (i & 7)) << 4)) = v;
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_arrive(smem_u32(&s_q_full));
        group_sync(id);
      }
      uint64_t l[kMine / 2];                               // sums of this thread's keys, two rows in each
#pragma unroll
      for (int i = 0; i < kMine / 2; ++i) l[i] = 0;
      bool blank = true;                                   // a row of this warpgroup has seen no key yet
      // steps [open0, open1): all of their keys are there and seen by all rows (if no block is missing)
      int open0 = 0, open1;
      {
        const int key_first = (walk.span.tile0 + walk.t0) * kTileKeys, lo = walk.span.lo;
        const int open_hi = min(walk.q.len - walk.q.n, walk.span.hi);
        const int open_lo = a.window > 0 ? max(lo, walk.q.len - a.window) : lo;
        if (open_lo > key_first) open0 = (int)(((unsigned int)(open_lo - key_first) + kTileKeys - 1) / kTileKeys);
        open1 = open_hi > key_first ? (open_hi - key_first) / kTileKeys : 0;
      }
      constexpr float kHead = kWeightHead<VT>;
      for (int j = 0; j < steps; ++j, ++step) {
        const unsigned int sb = step & 1u;
        float kf = 1.0f, vf = 1.0f;
        if constexpr (F8) {
          const unsigned int f = batch % kColInfo;
          if (j % kColBatch == 0) ring_wait(smem_u32(&s_info_full[f]), (batch / kColInfo) & 1u, abort_flag);
          const int kb = s_bytes[f * kColBatch + j % kColBatch][0][tid], vb = s_bytes[f * kColBatch + j % kColBatch][1][tid];
          kf = kb == 255 ? NAN : power_of_byte(kb);
          vf = power_of_byte(weight_byte(vb));
          if (j % kColBatch == kColBatch - 1 || j == steps - 1) {
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&s_info_empty[f]));
            ++batch;
          }
        }
        ring_wait(smem_u32(&s_s_full[sb]), (step >> 1) & 1u, abort_flag);
        __syncwarp();
        tmem_after();
        const unsigned int mask = s_mask[step % kInfoRing];
        const bool hide = mask != 0xffffffffu || j < open0 || j >= open1;
        uint32_t vis = 0xffffffffu;                        // which of its rows see this thread's key
        if (hide) {
          const int key = (walk.span.tile0 + walk.t0 + j) * kTileKeys + tid, d = key - (walk.q.len - walk.q.n);
          vis = key >= walk.span.lo && key < walk.span.hi && ((mask >> (tid >> a.box_log)) & 1u) ? 0xffffffffu : 0u;
          if (vis && d >= 0) {                             // a node: its bit, token by token
            const int t0 = s_tok[c0], t1 = s_tok[c0 + kMine - 1], left = walk.rows(a) - c0;
            const uint32_t* bits = a.mask + (walk.q.tok0 + t0) * a.mask_words + (d >> 5);
            const bool named = (d >> 5) < a.mask_words;
            vis = left < kMine ? 0xffffffffu << max(left, 0) : 0u;       // (rows that are not there see all)
            int from = t0 * a.G - block_row0() - c0;
#pragma unroll 4
            for (int t = t0; t <= t1; ++t, bits += a.mask_words, from += a.G) {
              const uint32_t bit = named ? __ldg(bits) >> (d & 31) & 1u : 0u;
              const uint32_t upto = from + a.G >= 32 ? 0xffffffffu : from + a.G > 0 ? (1u << (from + a.G)) - 1u : 0u;
              vis |= (0u - bit) & upto & (0xffffffffu << max(from, 0));
            }
          } else if (vis && a.window > 0) {
            vis = 0;
            for (int i = 0; i < kMine; ++i) vis |= (uint32_t)(key >= s_low[c0 + i]) << i;
          }
        }
        // Scores of 8 rows in powers of two, less the rows' m.
        auto scores = [&](int c, uint32_t* x, uint32_t seen) {
#pragma unroll
          for (int i = 0; i < 8; i += 4) {
            const float4 r = *reinterpret_cast<const float4*>(s_ref + c + i);
            uint64_t x0 = pair2(__uint_as_float(x[i]), __uint_as_float(x[i + 1]));
            uint64_t x1 = pair2(__uint_as_float(x[i + 2]), __uint_as_float(x[i + 3]));
            if constexpr (F8) {
              const float4 sc = *reinterpret_cast<const float4*>(s_scale + c + i);
              x0 = fma2(fma2(x0, pair2(kf, kf), pair2(0.0f, 0.0f)), pair2(sc.x, sc.y), pair2(-r.x, -r.y));
              x1 = fma2(fma2(x1, pair2(kf, kf), pair2(0.0f, 0.0f)), pair2(sc.z, sc.w), pair2(-r.z, -r.w));
            } else {
              x0 = fma2(x0, pair2(a.scale_log2, a.scale_log2), pair2(-r.x, -r.y));
              x1 = fma2(x1, pair2(a.scale_log2, a.scale_log2), pair2(-r.z, -r.w));
            }
            float y[4];
            split2(x0, y[0], y[1]);
            split2(x1, y[2], y[3]);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i + e] = __float_as_uint(y[e]);
          }
          if (hide) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (!(seen & (1u << i))) x[i] = 0xff800000u;
          }
        };
        // ---- weights.  They are taken with the m there is, while the warpgroup votes on whether that will do;
        // where it will not (and where a row has none yet) m moves first, and they are taken again.
        uint32_t z[kMine];
        bool move = blank;
        for (;;) {
          if (move) {
            // largest scores of the rows over all keys; m, l and O follow
            int best = float_order(-INFINITY);             // lane: of row `lane`, the warp's
#pragma unroll 1
            for (int ch = 0; ch < kChunks; ++ch) {
              uint32_t x[8];
              tmem_ld8(tm_s + sb * 128 + c0 + ch * 8, x);
              tmem_wait_ld();
              scores(c0 + ch * 8, x, vis >> (ch * 8));
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const int top = __reduce_max_sync(0xffffffffu, float_order(__uint_as_float(x[i])));
                if (lane == ch * 8 + i) best = top;
              }
            }
            if (lane < kMine) atomicMax(&s_new[c0 + lane], best);
            if (j > 0) pv_wait(step - 1);
            group_sync(id);
            if (tid < kMine) {
              const int c = c0 + tid;
              const float old = s_top[c], ref = s_ref[c];
              const float mn = fmaxf(old, order_float(s_new[c]) + ref - kHead);
              s_al[c] = old == -INFINITY ? 1.0f : exp2_fast(old - mn);
              s_top[c] = mn;
              s_ref[c] = mn == -INFINITY ? 0.0f : mn;
              s_new[c] = float_order(-INFINITY);
            }
            if (tid == 0) s_grow[w][0] = s_grow[w][1] = 0;
            blank = group_any(id, false);                  // (a barrier)
            for (int i = 0; i < kMine; ++i) blank |= s_top[c0 + i] == -INFINITY;
#pragma unroll
            for (int i = 0; i < kMine; i += 4) {
              const float4 al = *reinterpret_cast<const float4*>(s_al + c0 + i);
              l[i / 2] = fma2(l[i / 2], pair2(al.x, al.y), 0);
              l[i / 2 + 1] = fma2(l[i / 2 + 1], pair2(al.z, al.w), 0);
            }
            if (j > 0 && (D == 128 || (warp & 2) == 0)) {
#pragma unroll 1
              for (int x = 0; x < kParts * kChunks; ++x) {
                const int c = c0 + x % kChunks * 8, at = x / kChunks * N + c;
                uint32_t o[8];
                tmem_ld8(tm_o + at, o);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * s_al[c + i]);
                tmem_st8(tm_o + at, o);
              }
              tmem_wait_st();
            }
          }
#pragma unroll
          for (int ch = 0; ch < kChunks; ++ch)
            tmem_ld8(tm_s + sb * 128 + c0 + ch * 8, z + ch * 8);
          tmem_wait_ld();
          // (A row whose query is infinite has m = infinity after its first tile, and NaN where a score is infinite
          // again.  That is its own affair: the other rows of this thread's key have their say all the same.)
          float most = -INFINITY;
#pragma unroll
          for (int ch = 0; ch < kChunks; ++ch) {
            scores(c0 + ch * 8, z + ch * 8, vis >> (ch * 8));
#pragma unroll
            for (int i = ch * 8; i < ch * 8 + 8; i += 2)
              most = max3_numbers(most, __uint_as_float(z[i]), __uint_as_float(z[i + 1]));
          }
          if (!move) {
            const bool grow = __any_sync(0xffffffffu, most > kHead + 8.0f);
            if (lane == 0) {
              if (grow) s_grow[w][votes & 1u] = 1;
              mbar_arrive(smem_u32(&s_vote[w]));
            }
          }
#pragma unroll
          for (int ch = 0; ch < kChunks; ++ch) {
#pragma unroll
            for (int i = ch * 8; i < ch * 8 + 8; ++i) z[i] = __float_as_uint(exp2_fast(__uint_as_float(z[i])));
          }
          if (move) break;
          ring_wait(smem_u32(&s_vote[w]), votes & 1u, abort_flag);
          move = *reinterpret_cast<volatile int*>(&s_grow[w][votes & 1u]) != 0;
          ++votes;
          if (!move) break;
        }
        tmem_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_s_free[sb]));
        uint32_t pk[kParts][kMine / 2];
#pragma unroll
        for (int ch = 0; ch < kChunks; ++ch) {
#pragma unroll
          for (int i = ch * 8; i < ch * 8 + 8; i += 2) {
            float p0 = __uint_as_float(z[i]), p1 = __uint_as_float(z[i + 1]);
            l[i >> 1] = add2(l[i >> 1], pair2(p0, p1));
            if constexpr (F8) {
              p0 *= vf;
              p1 *= vf;
            }
            pk[0][i >> 1] = Bits16<VT>::pack(p0, p1);
            if constexpr (kParts == 2) {
              const float2 y = Bits16<VT>::unpack(pk[0][i >> 1]);
              pk[1][i >> 1] = Bits16<VT>::pack(p0 - y.x, p1 - y.y);
            }
          }
        }
        if (j >= S::kPs) pv_wait(step - S::kPs);           // the product that had this place has read its weights
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
          unsigned char* s_p = base + S::kPAt + (step % S::kPs) * S::kP + tid * 128;
#pragma unroll
          for (int ch = 0; ch < kChunks; ++ch) {
            const int c = part * N + c0 + ch * 8;
            *reinterpret_cast<uint4*>(s_p + (c >> 6) * S::kColBytes + ((((c >> 3) & 7) ^ (tid & 7)) << 4)) =
                make_uint4(pk[part][ch * 4], pk[part][ch * 4 + 1], pk[part][ch * 4 + 2], pk[part][ch * 4 + 3]);
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tmem_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_p_full[step % S::kPs]));
      }
      // ---- sums over the keys, 8 rows at a time, by way of tensor memory: taken from registers in a rolled
      // loop (unrolled over all rows, this part took registers from the loop above: 230 instead of 163 us for 32 drafts of 128 rows)
#pragma unroll
      for (int ch = 0; ch < kChunks; ++ch) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; i += 2) split2(l[ch * 4 + i / 2], x[i], x[i + 1]);
        tmem_st8(tm_o + 128 + c0 + ch * 8, reinterpret_cast<const uint32_t*>(x));
      }
      tmem_wait_st();
#pragma unroll 1
      for (int ch = 0; ch < kChunks; ++ch) {
        uint32_t x[8];
        tmem_ld8(tm_o + 128 + c0 + ch * 8, x);
        tmem_wait_ld();
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __uint_as_float(x[i]);
#pragma unroll
        for (int d = 4; d > 0; d >>= 1)                    // lane: of row lane mod 8
#pragma unroll
          for (int i = 0; i < d; ++i) {
            const bool up = lane & d;
            const float send = up ? y[i] : y[i + d];
            y[i] = (up ? y[i + d] : y[i]) + __shfl_xor_sync(0xffffffffu, send, d);
          }
        y[0] += __shfl_xor_sync(0xffffffffu, y[0], 8);
        y[0] += __shfl_xor_sync(0xffffffffu, y[0], 16);
        if (lane < 8) s_part[warp & 3][c0 + ch * 8 + lane] = y[0];
      }
      group_sync(id);
      const bool whole = walk.whole();
      const bool at_start = walk.pos - steps == walk.start;
      float* slot = a.slots + ((long long)blockIdx.x * 2 + (at_start ? 0 : 1)) * S::kSlot;
      const int rows_end = walk.rows(a);
      if (tid < kMine && c0 + tid < rows_end) {
        const int c = c0 + tid;
        float sum = (s_part[0][c] + s_part[1][c]) + (s_part[2][c] + s_part[3][c]);
        const float m = s_top[c];
        if (m == -INFINITY) sum = sum == sum ? 0.0f : sum; // a row that has seen no key
        s_inv[c] = sum == 0.0f ? 0.0f : 1.0f / sum;
        if (!whole) {
          slot[c] = m;
          slot[N + c] = sum;
        } else if (a.lse) {
          const int ti = s_tok[c], gi = block_row0() + c - ti * a.G;
          a.lse[(walk.q.tok0 + ti) * (a.pool.H * a.G) + walk.head * a.G + gi] =
              sum == 0.0f ? -INFINITY : 0.69314718056f * (m + log2f(sum));
        }
      }
      group_sync(id);
      // ---- O out of tensor memory
      pv_wait(step - 1);
      if (D == 128 || (warp & 2) == 0) {
#pragma unroll 1
        for (int ch = 0; ch < kChunks; ++ch) {
          uint32_t o[8];
          tmem_ld8(tm_o + c0 + ch * 8, o);
          if constexpr (kParts == 2) {
            uint32_t more[8];
            tmem_ld8(tm_o + N + c0 + ch * 8, more);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) + __uint_as_float(more[i]));
          } else {
            tmem_wait_ld();
          }
          const int c = c0 + ch * 8, left = rows_end - c;
          if (whole) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (i < left) reinterpret_cast<QT*>(a.out)[s_out[c + i] + tid] = QT(__uint_as_float(o[i]) * s_inv[c + i]);
          } else {
            float* to = slot + 2 * N + c * D + tid;
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (i < left) to[i * D] = __uint_as_float(o[i]);
          }
        }
      }
      tmem_before();
      group_sync(id);                                      // before the rows' facts change
    }
  } else if (warp < kQK + 4) {
    regs_down<S::kRegsOther>();
    const unsigned int leader = lane == 0;
    auto uniform = [](unsigned int x) { return __shfl_sync(0xffffffffu, x, 0); };
    const unsigned int tmu = uniform(tmem);
    if (warp == kQK) {
      // ============================================================== S^T = K Q^T
      unsigned int buf = 0, phase = 0, q_phase = 0, step = 0;
      const unsigned int q_low = uniform(operand_low(smem0 + S::kQAt, 16)), k_low = uniform(operand_low(k0, 16));
      while (walk.next_warp(a, per)) {
        const int steps = (int)uniform(walk.t1 - walk.t0);
        constexpr unsigned int desc = S::kPlain ? col_mma_desc8(N) : col_mma_desc(std::is_same<KT, __half>::value, N, false);
        ring_wait(smem_u32(&s_q_full), q_phase, abort_flag);
        q_phase ^= 1u;
        for (int j = 0; j < steps; ++j, ++step) {
          const unsigned int sb = step & 1u;
          ring_wait(smem_u32(&s_k_full[buf]), phase, abort_flag);
          ring_wait(smem_u32(&s_s_free[sb]), ((step >> 1) & 1u) ^ 1u, abort_flag);
          __syncwarp();
          tmem_after();
          const unsigned int low = k_low + buf * (S::kKBuf >> 4);
          if constexpr (S::kPlain) {
#pragma unroll
            for (int x = 0; x < S::kQParts * 4; ++x)       // (part x / 4, 32 dimensions from 32 (x % 4) on)
              mma_smem8(tmu + sb * 128, operand_desc(low + ((x & 3) * 32 >> 4)),
                        operand_desc(q_low + (((x >> 2) * N * 128 + (x & 3) * 32) >> 4)), desc, x > 0, leader);
          }
#pragma unroll
          for (int k = 0; k < (S::kPlain ? 0 : D / 16); ++k)
            mma_smem(tmu + sb * 128, operand_desc(low + (((k >> 2) * S::kColBytes + (k & 3) * 32) >> 4)),
                     operand_desc(q_low + (((k >> 2) * (S::kQ / S::kCols) + (k & 3) * 32) >> 4)), desc, k > 0, leader);
          mma_commit(smem_u32(&s_s_full[sb]), leader);
          mma_commit(smem_u32(&s_k_empty[buf]), leader);
          if (++buf == S::kK) {
            buf = 0;
            phase ^= 1u;
          }
        }
      }
    } else if (warp == kPV) {
      // ============================================================== O^T += V^T P^T
      unsigned int buf = 0, phase = 0, step = 0;
      if (lane == 0) {
        TileWalk<Blocks> look = walk;
        JoinRecord rec = {};
        if (look.next(a) == 1 && look.t0 > 0 && look.t1 == look.span.tiles) {
          const long long p0 = look.pos - look.t1;         // position of the rows' first tile
          rec.tok0 = look.q.tok0;
          rec.rows = look.rows(a);
          rec.row0 = look.block * Blocks::size(look.q.n * a.G);
          rec.head = look.head;
          rec.first_cta = (int)(p0 / per);
          rec.first_slot = p0 != rec.first_cta * per;
        }
        reinterpret_cast<JoinRecord*>(a.slots + 2ull * gridDim.x * S::kSlot)[blockIdx.x] = rec;
      }
      __syncwarp();
      // (at D = 64 the M of 128 reaches past V, into what lies there: lanes that nobody reads)
      const unsigned int v_low = uniform(operand_low(v0, S::kColBytes)), p_low = uniform(operand_low(smem0 + S::kPAt, S::kColBytes));
      while (walk.next_warp(a, per)) {
        const int steps = (int)uniform(walk.t1 - walk.t0);
        constexpr unsigned int desc = col_mma_desc(std::is_same<VT, __half>::value, S::kPRows, true);
        const int key_first = (int)uniform((walk.span.tile0 + walk.t0) * kTileKeys);
        const int lo = (int)uniform(walk.span.lo), hi = (int)uniform(walk.span.hi);
        for (int j = 0; j < steps; ++j, ++step) {
          const unsigned int pb = step % S::kPs;
          ring_wait(smem_u32(&s_v_full[buf]), phase, abort_flag);
          if (!F8) {
            // V rows of positions that no row sees, whatever the pool holds there, become zero (0 * NaN is NaN)
            const int key0 = key_first + j * kTileKeys;
            const int z0 = min(max(lo - key0, 0), kTileKeys), z1 = max(min(hi - key0, kTileKeys), 0);
            if (z0 > 0 || z1 < kTileKeys) {
              unsigned char* v = base + (v0 - smem0) + buf * S::kBuf;
              for (int x = lane; x < kTileKeys * 8; x += 32) {
                const int rr = x >> 3;
                if (rr < z0 || rr >= z1) {
#pragma unroll
                  for (int cc = 0; cc < S::kCols; ++cc)
                    *reinterpret_cast<uint4*>(v + cc * S::kColBytes + rr * 128 + (x & 7) * 16) = make_uint4(0, 0, 0, 0);
                }
              }
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
            }
          }
          ring_wait(smem_u32(&s_p_full[pb]), (step / S::kPs) & 1u, abort_flag);
          __syncwarp();
          tmem_after();
          const unsigned int low = v_low + buf * (S::kBuf >> 4);
#pragma unroll
          for (int k = 0; k < kTileKeys / 16; ++k)
            mma_smem(tmu + 256, operand_desc(low + k * (2048 >> 4)), operand_desc(p_low + ((pb * S::kP + k * 2048) >> 4)),
                     desc, k > 0 || j > 0, leader);
          mma_commit(smem_u32(&s_pv_done[pb]), leader);
          mma_commit(smem_u32(&s_v_empty[buf]), leader);
          if (++buf == S::kV) {
            buf = 0;
            phase ^= 1u;
          }
        }
      }
    } else {
      // ============================================================== loader warps, of K and of V
      // (A box takes its warp 75 cycles to issue: 16 of either K or V in one warp's loop took longer than
      // the bytes need.)
      const bool is_v = uniform(warp == kLoadV);
      constexpr unsigned int kBytes = F8 ? S::kRaw : S::kBuf;   // of a tile of K or V
      constexpr int kRow = F8 ? D : 128;
      unsigned long long* full = is_v ? (F8 ? s_v_raw : s_v_full) : (F8 && !S::kPlain ? s_k_raw : s_k_full);
      unsigned long long* empty = is_v ? s_v_empty : s_k_empty;
      const unsigned int ring0 = is_v ? v0 + (F8 ? S::kColBytes : 0) : k0 + (F8 && !S::kPlain ? S::kColBytes : 0);
      const unsigned int bufs = is_v ? S::kV : S::kK, each = is_v ? S::kBuf : S::kKBuf;
      const int boxes = kTileKeys >> a.box_log;
      unsigned int buf = 0, phase = 1, issued = 0;         // (a fresh barrier passes for phase 1)
      while (walk.next_warp(a, per)) {
        const uint32_t* row;
        long long entries;
        table_row(a.b, walk.r, row, entries);
        if (!is_v && walk.q.keys < walk.q.len && walk.head == 0 && walk.block == 0 && walk.t0 == 0 && lane == 0)
          raise_status(AIBX_ERR_RANGE);                    // tokens the table has no entry for
        BoxIds<kTileKeys> ids(a, row, walk.span.tile0 + walk.t0, walk.span.tile0 + walk.t1, walk.span.lo,
                              walk.span.hi);
        const int head = walk.head, tile0 = walk.span.tile0, lo = walk.span.lo, hi = walk.span.hi, t1 = walk.t1;
        for (int j = walk.t0; j < t1; ++j, ++issued) {
          uint32_t block_id;
          const bool valid = ids.give(block_id, !is_v && head == 0);
          const int slot = ids.slot;
          ids.step_slot();
          // a box that is not there, or that holds no visible key, comes as zeros from beyond the pool
          const int block = valid ? (int)block_id : (int)a.pool.num_blocks;
          const int tok = (tile0 + j) * kTileKeys + (lane & (boxes - 1)) * a.box;
          const bool missing = lane < boxes && tok < hi && tok > lo - a.box && !valid;
          const unsigned int gone = __ballot_sync(0xffffffffu, missing);
          if (!is_v && lane == 0) s_mask[issued % kInfoRing] = ~gone;
          ring_wait(smem_u32(&empty[buf]), phase, abort_flag);
          __syncwarp();
          const unsigned int bar = smem_u32(&full[buf]);
          if (__any_sync(0xffffffffu, *abort_flag)) {
            if (lane == 0) mbar_arrive(bar);
          } else {
            if (lane == 0) mbar_arrive_expect_tx(bar, kBytes);
            __syncwarp();
            if (lane < boxes) {
              const unsigned int dst = ring0 + buf * each + lane * a.box * kRow;
#pragma unroll
              for (int cc = 0; cc < (F8 ? 1 : S::kCols); ++cc)
                tensor_load_5d(dst + cc * S::kColBytes, &map, bar, cc * 64, slot, head, block, is_v ? 1 : 0);
            }
          }
          __syncwarp();
          if (++buf == bufs) {
            buf = 0;
            phase ^= 1u;
          }
        }
      }
      // nothing may still be on its way here when the CTA ends: no copy, no word of a product
      for (unsigned int i = issued > bufs ? issued - bufs : 0; i < issued; ++i) {
        ring_drain(smem_u32(&full[i % bufs]), (i / bufs) & 1u);
        ring_wait(smem_u32(&empty[i % bufs]), (i / bufs) & 1u, abort_flag);
      }
    }
  } else if constexpr (F8) {
    // ================================================================ converter warps
    regs_down<S::kRegsConvert>();
    // A thread takes one 16-byte piece of kRows neighbouring rows; a row's pieces are one warp's, which has
    // read them all before it writes over them.
    const int tid = threadIdx.x - 32 * (kQK + 4);
    constexpr int kPieces = D / 16;                        // 16-byte pieces of a raw row
    constexpr int kRows = kTileKeys * kPieces / (128 * S::kConverters);
    const int c = tid % kPieces, i0 = tid / kPieces * kRows;
    unsigned int kbuf = 0, kphase = 0, vbuf = 0, vphase = 0, batch = 0, made = 0;
    while (walk.next_warp(a, per)) {
      const int steps = walk.t1 - walk.t0;
      const int key_first = (walk.span.tile0 + walk.t0) * kTileKeys, lo = walk.span.lo, hi = walk.span.hi;
      // Scale bytes are fetched four tiles at a time, the next four while these are converted: two dependent
      // loads, which the warps wait for here once in four tiles.
      const uint32_t* row;
      long long entries;
      table_row(a.b, walk.r, row, entries);
      const unsigned char* scales = a.pool.scales + (long long)walk.head * a.pool.s_head;
      auto fetch = [&](int j0) {
        constexpr int kEach = kColBatch * kTileKeys / (128 * (F8 ? S::kConverters : 1));   // keys of a thread
        const unsigned int f = made % kColInfo;
        uint32_t block[kEach], kb[kEach], vb[kEach];
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
          const uint32_t key = (uint32_t)(key_first + tid) + (uint32_t)(j0 * kTileKeys + u * (128 * S::kConverters));
          block[u] = key >= (uint32_t)lo && key < (uint32_t)hi ? __ldg(row + key / (uint32_t)a.pool.T) : AIBX_NO_BLOCK;
          kb[u] = vb[u] = 127;
        }
#pragma unroll
        for (int u = 0; u < kEach; ++u)
          if (block[u] < a.pool.num_blocks) {
            const uint32_t key = (uint32_t)(key_first + tid) + (uint32_t)(j0 * kTileKeys + u * (128 * S::kConverters));
            const unsigned char* src = scales + (long long)block[u] * a.pool.s_block + (long long)(key % (uint32_t)a.pool.T) * a.pool.s_slot;
            kb[u] = __ldg(src);
            vb[u] = __ldg(src + a.pool.s_kv);
          }
        ring_wait(smem_u32(&s_info_empty[f]), ((made / kColInfo) & 1u) ^ 1u, abort_flag);
        __syncwarp();
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
          const int x = u * (128 * S::kConverters) + tid, t = x / kTileKeys, k = x % kTileKeys;
          const uint32_t key = (uint32_t)key_first + (uint32_t)(j0 * kTileKeys + x);   // (past 2^31 behind the last tile)
          s_bytes[f * kColBatch + t][0][k] = (unsigned char)kb[u];
          s_bytes[f * kColBatch + t][1][k] = (unsigned char)vb[u];
          // (rows outside: zeros)
          const bool odd = __any_sync(0xffffffffu, (int)vb[u] != weight_byte((int)vb[u]) || key < (uint32_t)lo || key >= (uint32_t)hi);
          if (lane == 0) s_odd[f * kColBatch + t][k >> 5] = odd;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_info_full[f]));
        ++made;
      };
      fetch(0);
      for (int j = 0; j < steps; ++j) {
        const unsigned int f = batch % kColInfo, ft = f * kColBatch + j % kColBatch;
        if (j % kColBatch == 0 && j + kColBatch < steps) fetch(j + kColBatch);
        auto convert = [&](unsigned int at, auto is_v, auto odd) {
          unsigned char* out = base + at + (c >> 2) * S::kColBytes;
          const unsigned char* src = base + at + S::kColBytes;
          uint4 v[kRows];
#pragma unroll
          for (int u = 0; u < kRows; ++u) {
            const int i = i0 + u;
            v[u] = *reinterpret_cast<const uint4*>(src + i * D + ((D == 128 ? c ^ (i & 7) : c) << 4));
          }
          __syncwarp();
#pragma unroll
          for (int u = 0; u < kRows; ++u) {
            const int i = i0 + u;
            const uint32_t wv[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
            uint32_t o[8];
            float rest = 1.0f;
            bool gone = false;
            if constexpr (decltype(odd)::value) {
              const int key = key_first + j * kTileKeys + i, vb = s_bytes[ft][1][i];
              gone = key < lo || key >= hi;              // whatever the pool holds there
              rest = vb == 255 ? NAN : power_of_byte(127 + vb - weight_byte(vb));
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const uint32_t two = (wv[e >> 1] >> (16 * (e & 1))) & 0xffffu;
              if constexpr (!decltype(is_v)::value)
                o[e] = e4m3_bits(two);
              else if constexpr (decltype(odd)::value)
                o[e] = gone ? 0u : bf16_of_e4m3(two, rest);
              else {
                const float2 y = __half22float2(halves_of_e4m3(two));
                o[e] = Bits16<__nv_bfloat16>::pack(y.x, y.y);
              }
            }
            // (pieces 2 c and 2 c + 1; the upper half of a row's lanes the other way round: with their
            // column 16 KB on they would meet the lower half's banks)
            const int p0 = (2 * c) & 7, flip = c >> 2 & 1;
            *reinterpret_cast<uint4*>(out + i * 128 + (((p0 + flip) ^ (i & 7)) << 4)) =
                flip ? make_uint4(o[4], o[5], o[6], o[7]) : make_uint4(o[0], o[1], o[2], o[3]);
            *reinterpret_cast<uint4*>(out + i * 128 + (((p0 + 1 - flip) ^ (i & 7)) << 4)) =
                flip ? make_uint4(o[0], o[1], o[2], o[3]) : make_uint4(o[4], o[5], o[6], o[7]);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        };
        if constexpr (!S::kPlain) {
          ring_wait(smem_u32(&s_k_raw[kbuf]), kphase, abort_flag);
          __syncwarp();
          convert((k0 - smem0) + kbuf * S::kKBuf, std::false_type(), std::false_type());
          mbar_arrive(smem_u32(&s_k_full[kbuf]));
          if (++kbuf == S::kK) {
            kbuf = 0;
            kphase ^= 1u;
          }
        }
        if (j % kColBatch == 0) ring_wait(smem_u32(&s_info_full[f]), (batch / kColInfo) & 1u, abort_flag);
        ring_wait(smem_u32(&s_v_raw[vbuf]), vphase, abort_flag);
        __syncwarp();
        if (s_odd[ft][0] | s_odd[ft][1] | s_odd[ft][2] | s_odd[ft][3])
          convert((v0 - smem0) + vbuf * S::kBuf, std::true_type(), std::true_type());
        else
          convert((v0 - smem0) + vbuf * S::kBuf, std::true_type(), std::false_type());
        mbar_arrive(smem_u32(&s_v_full[vbuf]));
        if (j % kColBatch == kColBatch - 1 || j == steps - 1) {
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&s_info_empty[f]));
          ++batch;
        }
        if (++vbuf == S::kV) {
          vbuf = 0;
          vphase ^= 1u;
        }
      }
    }
  }
  tmem_before();
  __syncthreads();
  if (warp == kQK) {
    tmem_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

template <int D, bool F8, typename QT, int N>
inline int32_t launch_attn_cols(AttnArgs a, int type, JoinSet& join, cudaStream_t st) {
  using S = ColRings<D, F8, N>;
  a.box = gcd_int(a.pool.T, kTileKeys);
  a.box_log = log2_int(a.box);
  CUtensorMap map;
  const int32_t rc = pool_tensor_map(a.pool, type, a.box, &map);
  if (rc != AIBX_OK) return rc;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return AIBX_ERR_CUDA;
  static size_t configured[64] = {0};
  static std::mutex lock;
  if (!ensure_dynamic_smem(attn_cols_kernel<D, F8, QT, N>, S::kSmem, dev, configured, lock)) return AIBX_ERR_CUDA;
  const unsigned int grid = (unsigned int)sm_count();
  attn_cols_kernel<D, F8, QT, N><<<grid, S::kThreads, S::kSmem, st>>>(map, a);
  join = JoinSet{a.slots, reinterpret_cast<const JoinRecord*>(a.slots + 2ull * grid * S::kSlot), N};
  return launch_status();
}

}  // namespace aibx
