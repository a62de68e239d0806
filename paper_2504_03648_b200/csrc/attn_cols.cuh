// Attention of a drafted tree's nodes over a paged cache: more than 8 and up to some hundred query rows
// (nodes * query heads per KV head) of a (request, KV head), on the 5th-generation tensor cores.
//
// Few rows against many keys: the keys are the M of both products and the rows their N, so that work
// shrinks with the rows (a tile of 128 rows, filled or not, costs its softmax 128 exponentials a key; here
// a row costs one).  A block of up to N rows meets KV tiles of 128 positions:
//   S^T = K Q^T        [128 keys][rows], K and Q from shared memory, S^T in tensor memory (fp32)
//   P^T = 2^(S^T c - m)   one thread per key and half of the rows; P^T to shared memory, 16-bit
//   O^T += V^T P^T     [dims][rows], V as it lies in the pool ([position][dim]: V^T's M-major form)
// A row's maximum runs across the threads, which is what makes this form dear; but m needs to move only
// when a score passes it by 2^8 (weights up to 2^8 are as good as weights up to 1).  So a tile costs one
// comparison per score and one vote of the warpgroup; maxima over keys are taken in the rare tile where the
// vote says so (a segment's first).  The sums l stay per key and are added up once, at the end.
//
// Visible: cached positions (window: those near enough to the row's node) and the nodes whose bit is set
// in the row's mask; a thread looks at bits only in tiles that touch the nodes.
//
// Over an e4m3 pool a warpgroup turns raw tiles into operands as they arrive: K into fp16, exact and
// without its scales, which the thread that has the key applies to its scores; V into bf16, exact too.
// V's scales go with the weights, in bf16, whose range holds them however far apart they are (scale bytes
// outside [kScaleLow, kScaleHigh] leave the rest with V).  fp16 queries get weights as the sum of two
// bf16 numbers, so that they lose nothing to the type.
//
// Roles: two softmax warpgroups, one for each half of the rows, which never wait for each other; a warp
// for S^T and one for O^T; a loader; over e4m3 a warp for the scale bytes and four that convert.  Rings of K
// and of V tiles of their own, S^T twice, so that S^T(j + 1) runs beside the softmax of tile j.
// Bound: HBM, 2,800 cycles a tile of 128 16-bit keys of D = 128 (this SM's share), 1,400 of e4m3 ones; the
// products take (4 + 4) * N cycles of the tensor pipe.
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

template <int D, bool F8, int N>
struct ColShape {
  static constexpr int kThreads = F8 ? 512 : 384;
  static constexpr int kCols = D / 64;                     // 128-byte columns of an operand row
  static constexpr int kColBytes = 128 * 128;
  static constexpr int kRaw = kTileKeys * D;               // a tile's e4m3 rows, as they arrive
  static constexpr int kBuf = kTileKeys * D * 2 + (F8 && D == 64 ? kRaw : 0);   // as in TileShape
  static constexpr int kQ = kCols * kColBytes * N / 128;
  static constexpr int kP = kTileKeys * 128 * (N / 64);    // P^T: 64 rows in 128 bytes a key
  static constexpr int kRoom = 216 * 1024;
};
// P^T as one 16-bit number or the sum of two; what is left of shared memory goes to the rings.
template <int D, bool F8, int N, int PARTS>
struct ColRings : ColShape<D, F8, N> {
  using B = ColShape<D, F8, N>;
  static constexpr int kBufs = (B::kRoom - B::kQ - PARTS * B::kP - 1024) / B::kBuf;
  static constexpr int kK = kBufs / 2 < 4 ? kBufs / 2 : 4, kV = kBufs - kBufs / 2 < 4 ? kBufs - kBufs / 2 : 4;
  static constexpr int kQAt = (kK + kV) * B::kBuf, kPAt = kQAt + B::kQ;
  static constexpr int kSmem = kPAt + PARTS * B::kP + 1024;
  static constexpr int kSlot = N * (D + 2);                // floats per workspace slot
  static constexpr int kRegsSoftmax = F8 ? 176 : 200;      // sums as in TileShape
  static constexpr int kRegsOther = F8 ? 80 : 104;
  static_assert(kK >= 2 && kV >= 2, "two tiles of each at least");
};

// fp32 accumulator, M = 128, B's N at run time; operands N- or M-major where said
__device__ __forceinline__ unsigned int col_mma_desc(bool half, int n, bool major) {
  return (1u << 4) | ((half ? 0u : 1u) << 7) | ((half ? 0u : 1u) << 10) | (major ? 3u << 15 : 0u) |
         ((unsigned int)(n >> 3) << 17) | ((128u >> 4) << 24);
}

__device__ __forceinline__ void tmem_ld16(unsigned int addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr));
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

// Whole numbers that order as the floats do (not for NaN).
__device__ __forceinline__ int float_order(float x) {
  const int u = __float_as_int(x);
  return u ^ ((u >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float order_float(int k) { return __int_as_float(k ^ ((k >> 31) & 0x7fffffff)); }

constexpr int kColInfo = 4;                                // per-tile facts of an e4m3 pool

template <int D, bool F8, typename QT, int N>
__global__ void __launch_bounds__(ColShape<D, F8, N>::kThreads, 1)
attn_cols_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ AttnArgs a) {
  constexpr int kParts = F8 && std::is_same<QT, __half>::value ? 2 : 1;
  using S = ColRings<D, F8, N, kParts>;
  using Blocks = EvenBlocks<N>;
  using KT = typename std::conditional<F8, __half, QT>::type;            // operands of S^T
  using VT = typename std::conditional<F8, __nv_bfloat16, QT>::type;     // and of O^T
  constexpr int kMine = N / 2, kChunks = kMine / 16;       // rows of a softmax warpgroup, 16 at a time
  extern __shared__ unsigned char s_raw[];
  __shared__ __align__(8) unsigned long long s_k_full[S::kK], s_k_empty[S::kK], s_k_raw[S::kK];
  __shared__ __align__(8) unsigned long long s_v_full[S::kV], s_v_empty[S::kV], s_v_raw[S::kV];
  __shared__ __align__(8) unsigned long long s_s_full[2], s_s_free[2], s_q_full, s_p_full, s_pv_done;
  __shared__ __align__(8) unsigned long long s_info_full[kColInfo], s_info_empty[kColInfo];
  __shared__ unsigned int s_mask[kInfoRing];
  __shared__ __align__(16) float s_ref[N], s_scale[N];     // m (0 where no key was seen yet) and scale of each row
  __shared__ float s_top[N], s_inv[N];
  __shared__ int s_new[N], s_low[N], s_tok[N];
  __shared__ long long s_out[N];
  __shared__ float s_part[4][N];
  __shared__ __align__(4) unsigned char s_bytes[F8 ? kColInfo : 1][2][kTileKeys];
  __shared__ int s_odd[kColInfo];                          // whether V's bytes leave a rest with V
  __shared__ long long s_scan[33];
  __shared__ WorkStart s_start;
  __shared__ TileWalk<Blocks> s_walk[S::kThreads / 32];
  __shared__ unsigned int s_tmem;
  __shared__ int s_abort;

  const unsigned int smem0 = (smem_u32(s_raw) + 1023u) & ~1023u;
  unsigned char* base = s_raw + (smem0 - smem_u32(s_raw));
  const unsigned int k0 = smem0, v0 = smem0 + S::kK * S::kBuf;
  const int lane = threadIdx.x & 31;
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  volatile int* abort_flag = &s_abort;

  if (threadIdx.x == 0) {
    for (int i = 0; i < S::kK; ++i) {
      mbar_init(smem_u32(&s_k_full[i]), F8 ? 128u : 1u);
      mbar_init(smem_u32(&s_k_empty[i]), 1u);
      mbar_init(smem_u32(&s_k_raw[i]), 1u);
    }
    for (int i = 0; i < S::kV; ++i) {
      mbar_init(smem_u32(&s_v_full[i]), F8 ? 128u : 1u);
      mbar_init(smem_u32(&s_v_empty[i]), 1u);
      mbar_init(smem_u32(&s_v_raw[i]), 1u);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&s_s_full[i]), 1u);
      mbar_init(smem_u32(&s_s_free[i]), 8u);
    }
    for (int i = 0; i < kColInfo; ++i) {
      mbar_init(smem_u32(&s_info_full[i]), 1u);
      mbar_init(smem_u32(&s_info_empty[i]), 12u);
    }
    mbar_init(smem_u32(&s_q_full), 256u);
    mbar_init(smem_u32(&s_p_full), 8u);
    mbar_init(smem_u32(&s_pv_done), 1u);
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    tmem_before();
  }
  const TileCost<Blocks> cost{a};
  locate_piece<S::kThreads>(a.b.R, blockIdx.x, gridDim.x, s_scan, &s_start, cost);
  const long long per = (s_start.total + gridDim.x - 1) / gridDim.x;
  if (warp == 0) {
    locate_block<Blocks>(a, blockIdx.x, gridDim.x, &s_start);
    __syncwarp();
    if (lane == 0) {
      TileWalk<Blocks> look;
      look.init(a, s_start, blockIdx.x, gridDim.x);
      JoinRecord rec = {};
      if (look.next(a) == 1 && look.t0 > 0 && look.t1 == look.span.tiles) {
        const long long p0 = look.pos - look.t1;           // position of the rows' first tile
        rec.tok0 = look.q.tok0;
        rec.rows = look.rows(a);
        rec.row0 = look.block * Blocks::size(look.q.n * a.G);
        rec.head = look.head;
        rec.first_cta = (int)(p0 / per);
        rec.first_slot = p0 != rec.first_cta * per;
      }
      reinterpret_cast<JoinRecord*>(a.slots + 2ull * gridDim.x * S::kSlot)[blockIdx.x] = rec;
    }
  }
  __syncthreads();
  tmem_after();
  const unsigned int tmem = s_tmem;                        // columns: S^T 0 and 128, O^T 256
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  TileWalk<Blocks>& walk = s_walk[warp];
  if (lane == 0) walk.init(a, s_start, blockIdx.x, gridDim.x);
  __syncwarp();

  if (warp < 8) {
    // ================================================================ softmax: thread = key
    regs_up<S::kRegsSoftmax>();
    const int w = warp >> 2, id = 1 + w;                   // warpgroup and its barrier
    const int tid = threadIdx.x & 127;                     // key in the tile; of O^T, the dimension
    const unsigned int lanes = (unsigned int)(warp & 3) << 21;
    const unsigned int tm_s = tmem + lanes, tm_o = tmem + lanes + 256;
    unsigned char* s_q = base + S::kQAt;
    unsigned int step = 0, pv_phase = 0;
    while (walk.next_warp(a, per)) {
      const int rows = walk.rows(a), steps = walk.t1 - walk.t0;
      const int chunks = (rows + 31) >> 5, mine = chunks * 16;           // of this warpgroup's rows
      const int c0 = w * mine;                             // its first row of the block
      const int row0 = walk.block * Blocks::size(walk.q.n * a.G);
      const int first = walk.q.len - walk.q.n;
      // ---- what is known of each row
      if (tid < mine) {
        const int ri = row0 + min(c0 + tid, rows - 1), ti = a.by_g.div(ri);
        s_tok[c0 + tid] = ti;
        s_out[c0 + tid] = (walk.q.tok0 + ti) * a.o_tok + (long long)(walk.head * a.G + (ri - ti * a.G)) * a.o_head;
        int low = walk.span.lo;
        if (a.window > 0) {
          const int depth = tree_depth(a.mask + (walk.q.tok0 + ti) * a.mask_words, a.mask_words, walk.q.n);
          low = (int)max((long long)low, (long long)first + depth - a.window + 1);
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
        for (int i0 = tid / kPieces; i0 < mine; i0 += kBatch * (128 / kPieces)) {
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
            const bool on = i0 + u * (128 / kPieces) < mine;
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
              power_scale(amax, down, up);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float2 f = Bits16<QT>::unpack(x[e]);
                x[e] = Bits16<KT>::pack(f.x * down, f.y * down);
              }
              v = make_uint4(x[0], x[1], x[2], x[3]);
              if (on && c == 0) s_scale[i] = a.scale_log2 * up;
            }
            if (on) *reinterpret_cast<uint4*>(dst + i * 128 + (((c & 7) ^ (i & 7)) << 4)) = v;
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_arrive(smem_u32(&s_q_full));
        group_sync(id);
      }
      float l[kMine];
#pragma unroll
      for (int i = 0; i < kMine; ++i) l[i] = 0.0f;
      bool blank = true;                                   // a row of this warpgroup has seen no key yet
      const int key_first = (walk.span.tile0 + walk.t0) * kTileKeys;
      const int lo = walk.span.lo, hi = walk.span.hi;
      const int open_hi = min(first, hi);
      const int open_lo = a.window > 0 ? max(lo, walk.q.len - a.window) : lo;
      constexpr float kHead = kWeightHead<VT>;
      for (int j = 0; j < steps; ++j, ++step) {
        const unsigned int sb = step & 1u;
        float kf = 1.0f, vf = 1.0f;
        if constexpr (F8) {
          const unsigned int f = step % kColInfo;
          ring_wait(smem_u32(&s_info_full[f]), (step / kColInfo) & 1u, abort_flag);
          const int kb = s_bytes[f][0][tid], vb = s_bytes[f][1][tid];
          kf = kb == 255 ? NAN : power_of_byte(kb);
          vf = power_of_byte(weight_byte(vb));
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&s_info_empty[f]));
        }
        ring_wait(smem_u32(&s_s_full[sb]), (step >> 1) & 1u, abort_flag);
        __syncwarp();
        tmem_after();
        uint32_t z[kMine];
#pragma unroll
        for (int ch = 0; ch < kChunks; ++ch)
          if (ch < chunks) tmem_ld16(tm_s + sb * 128 + c0 + ch * 16, z + ch * 16);
        tmem_wait_ld();
        tmem_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_s_free[sb]));
        // ---- scores in powers of two, less the row's m
        const int key0 = key_first + j * kTileKeys;
        const unsigned int mask = s_mask[step % kInfoRing];
        const bool hide = mask != 0xffffffffu || key0 < open_lo || key0 > open_hi - kTileKeys;   // (key0 + 128 may be 2^31)
        float most = -INFINITY;
#pragma unroll
        for (int ch = 0; ch < kChunks; ++ch) {
          if (ch >= chunks) continue;
#pragma unroll
          for (int i = ch * 16; i < ch * 16 + 16; i += 4) {
            const float4 r = *reinterpret_cast<const float4*>(s_ref + c0 + i);
            uint64_t x0 = pair2(__uint_as_float(z[i]), __uint_as_float(z[i + 1]));
            uint64_t x1 = pair2(__uint_as_float(z[i + 2]), __uint_as_float(z[i + 3]));
            if constexpr (F8) {
              const float4 sc = *reinterpret_cast<const float4*>(s_scale + c0 + i);
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
            for (int e = 0; e < 4; ++e) z[i + e] = __float_as_uint(y[e]);
          }
        }
        if (hide) {
          const int key = key0 + tid, d = key - first;
          const bool here = key >= lo && key < hi && ((mask >> (tid >> a.box_log)) & 1u);
          const uint32_t* bits = a.mask + walk.q.tok0 * a.mask_words + (d >> 5);
          const bool node = here && d >= 0 && (d >> 5) < a.mask_words;
#pragma unroll
          for (int ch = 0; ch < kChunks; ++ch) {
            if (ch >= chunks) continue;
#pragma unroll
            for (int i = ch * 16; i < ch * 16 + 16; ++i) {
              bool ok = here && d < 0 && key >= s_low[c0 + i];
              if (node) ok = (__ldg(bits + (long long)s_tok[c0 + i] * a.mask_words) >> (d & 31)) & 1u;
              if (!ok) z[i] = 0xff800000u;
            }
          }
        }
#pragma unroll
        for (int ch = 0; ch < kChunks; ++ch) {
          if (ch >= chunks) continue;
#pragma unroll
          for (int i = ch * 16; i < ch * 16 + 16; i += 2) most = max3(most, __uint_as_float(z[i]), __uint_as_float(z[i + 1]));
        }
        // ---- m, moved only when a score passes it by 2^8
        if (group_any(id, blank || most > kHead + 8.0f)) {
          if (j > 0) {
            ring_wait(smem_u32(&s_pv_done), pv_phase, abort_flag);     // (looked at once more below)
            __syncwarp();
            tmem_after();
          }
          int best[(kMine + 31) / 32];                     // lane: of row 32 k + lane, the warp's largest score
#pragma unroll
          for (int k = 0; k < (kMine + 31) / 32; ++k) best[k] = float_order(-INFINITY);
#pragma unroll
          for (int i = 0; i < kMine; ++i) {
            if (i / 16 >= chunks) continue;
            const int top = __reduce_max_sync(0xffffffffu, float_order(__uint_as_float(z[i])));
            if (lane == (i & 31)) best[i / 32] = top;
          }
#pragma unroll
          for (int k = 0; k < (kMine + 31) / 32; ++k)
            if (32 * k + lane < mine) atomicMax(&s_new[c0 + 32 * k + lane], best[k]);
          group_sync(id);
          blank = false;
#pragma unroll
          for (int ch = 0; ch < kChunks; ++ch) {
            if (ch >= chunks) continue;
            uint32_t o[16];
            const bool scale_o = j > 0 && (D == 128 || (warp & 2) == 0);
            if (scale_o) {
              tmem_ld16(tm_o + c0 + ch * 16, o);
              tmem_wait_ld();
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int c = c0 + ch * 16 + i;
              const float old = s_top[c], ref = s_ref[c];
              const float mn = fmaxf(old, order_float(s_new[c]) + ref - kHead);
              const float al = old == -INFINITY ? 1.0f : exp2_fast(old - mn);
              l[ch * 16 + i] *= al;
              blank |= mn == -INFINITY;
              z[ch * 16 + i] = __float_as_uint(__uint_as_float(z[ch * 16 + i]) + (ref - (mn == -INFINITY ? 0.0f : mn)));
              o[i] = __float_as_uint(__uint_as_float(o[i]) * al);
            }
            if (scale_o) tmem_st16(tm_o + c0 + ch * 16, o);
          }
          tmem_wait_st();
          tmem_before();
          group_sync(id);                                  // all have read what changes now
          if (tid < mine) {
            const int c = c0 + tid;
            const float mn = fmaxf(s_top[c], order_float(s_new[c]) + s_ref[c] - kHead);
            s_top[c] = mn;
            s_ref[c] = mn == -INFINITY ? 0.0f : mn;
            s_new[c] = float_order(-INFINITY);
          }
          group_sync(id);
        }
        // ---- weights
        uint32_t pk[kParts][kMine / 2];
#pragma unroll
        for (int ch = 0; ch < kChunks; ++ch) {
          if (ch >= chunks) continue;
#pragma unroll
          for (int i = ch * 16; i < ch * 16 + 16; i += 2) {
            float p0 = exp2_fast(__uint_as_float(z[i])), p1 = exp2_fast(__uint_as_float(z[i + 1]));
            l[i] += p0;
            l[i + 1] += p1;
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
        if (j > 0) {                                       // the product before has read its weights
          ring_wait(smem_u32(&s_pv_done), pv_phase, abort_flag);
          pv_phase ^= 1u;
          __syncwarp();
        }
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
          unsigned char* s_p = base + S::kPAt + part * S::kP + tid * 128;
#pragma unroll
          for (int ch = 0; ch < kChunks; ++ch) {
            if (ch >= chunks) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int c = c0 + ch * 16 + h * 8;
              *reinterpret_cast<uint4*>(s_p + (c >> 6) * S::kColBytes + ((((c >> 3) & 7) ^ (tid & 7)) << 4)) =
                  make_uint4(pk[part][ch * 8 + h * 4], pk[part][ch * 8 + h * 4 + 1], pk[part][ch * 8 + h * 4 + 2],
                             pk[part][ch * 8 + h * 4 + 3]);
            }
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_p_full));
      }
      // ---- sums over the keys: each lane ends with the warp's sum of row 32 k + lane
#pragma unroll
      for (int k = 0; k < kMine; k += 32) {
        if (k >= mine) continue;
        float x[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = k + i < kMine ? l[k + i < kMine ? k + i : 0] : 0.0f;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1)
#pragma unroll
          for (int i = 0; i < d; ++i) {
            const bool up = lane & d;
            const float send = up ? x[i] : x[i + d];
            x[i] = (up ? x[i + d] : x[i]) + __shfl_xor_sync(0xffffffffu, send, d);
          }
        if (k + lane < mine) s_part[warp & 3][c0 + k + lane] = x[0];
      }
      group_sync(id);
      const bool whole = walk.whole();
      const bool at_start = walk.pos - steps == walk.start;
      float* slot = a.slots + ((long long)blockIdx.x * 2 + (at_start ? 0 : 1)) * S::kSlot;
      if (tid < mine && c0 + tid < rows) {
        const int c = c0 + tid;
        float sum = (s_part[0][c] + s_part[1][c]) + (s_part[2][c] + s_part[3][c]);
        const float m = s_top[c];
        if (m == -INFINITY) sum = sum == sum ? 0.0f : sum; // a row that has seen no key
        s_inv[c] = sum == 0.0f ? 0.0f : 1.0f / sum;
        if (!whole) {
          slot[c] = m;
          slot[N + c] = sum;
        } else if (a.lse) {
          const int ti = s_tok[c], gi = row0 + c - ti * a.G;
          a.lse[(walk.q.tok0 + ti) * (a.pool.H * a.G) + walk.head * a.G + gi] =
              sum == 0.0f ? -INFINITY : 0.69314718056f * (m + log2f(sum));
        }
      }
      group_sync(id);
      // ---- O out of tensor memory
      ring_wait(smem_u32(&s_pv_done), pv_phase, abort_flag);
      pv_phase ^= 1u;
      __syncwarp();
      tmem_after();
      if (D == 128 || (warp & 2) == 0) {
#pragma unroll
        for (int ch = 0; ch < kChunks; ++ch) {
          if (ch >= chunks) continue;
          uint32_t o[16];
          tmem_ld16(tm_o + c0 + ch * 16, o);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int c = c0 + ch * 16 + i;
            if (c < rows) {
              if (whole)
                reinterpret_cast<QT*>(a.out)[s_out[c] + tid] = QT(__uint_as_float(o[i]) * s_inv[c]);
              else
                slot[2 * N + (long long)c * D + tid] = __uint_as_float(o[i]);
            }
          }
        }
      }
      tmem_before();
      group_sync(id);                                      // before the rows' facts change
    }
  } else if (warp < 12) {
    regs_down<S::kRegsOther>();
    const unsigned int leader = lane == 0;
    auto uniform = [](unsigned int x) { return __shfl_sync(0xffffffffu, x, 0); };
    const unsigned int tmu = uniform(tmem);
    if (warp == 8) {
      // ============================================================== S^T = K Q^T
      unsigned int buf = 0, phase = 0, q_phase = 0, step = 0;
      const unsigned int q_low = uniform(operand_low(smem0 + S::kQAt, 16)), k_low = uniform(operand_low(k0, 16));
      while (walk.next_warp(a, per)) {
        const int steps = (int)uniform(walk.t1 - walk.t0);
        const unsigned int desc = uniform(col_mma_desc(std::is_same<KT, __half>::value, (walk.rows(a) + 31) / 32 * 32, false));
        ring_wait(smem_u32(&s_q_full), q_phase, abort_flag);
        q_phase ^= 1u;
        for (int j = 0; j < steps; ++j, ++step) {
          const unsigned int sb = step & 1u;
          ring_wait(smem_u32(&s_k_full[buf]), phase, abort_flag);
          ring_wait(smem_u32(&s_s_free[sb]), ((step >> 1) & 1u) ^ 1u, abort_flag);
          __syncwarp();
          tmem_after();
          const unsigned int low = k_low + buf * (S::kBuf >> 4);
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
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
    } else if (warp == 10) {
      // ============================================================== O^T += V^T P^T
      unsigned int buf = 0, phase = 0, p_phase = 0;
      // (at D = 64 the M of 128 reaches past V, into what lies there: lanes that nobody reads)
      const unsigned int v_low = uniform(operand_low(v0, S::kColBytes)), p_low = uniform(operand_low(smem0 + S::kPAt, S::kColBytes));
      while (walk.next_warp(a, per)) {
        const int steps = (int)uniform(walk.t1 - walk.t0);
        const unsigned int desc = uniform(col_mma_desc(std::is_same<VT, __half>::value, (walk.rows(a) + 31) / 32 * 32, true));
        const int key_first = (int)uniform((walk.span.tile0 + walk.t0) * kTileKeys);
        const int lo = (int)uniform(walk.span.lo), hi = (int)uniform(walk.span.hi);
        for (int j = 0; j < steps; ++j) {
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
          ring_wait(smem_u32(&s_p_full), p_phase, abort_flag);
          p_phase ^= 1u;
          __syncwarp();
          tmem_after();
          const unsigned int low = v_low + buf * (S::kBuf >> 4);
#pragma unroll
          for (int part = 0; part < kParts; ++part)
#pragma unroll
            for (int k = 0; k < kTileKeys / 16; ++k)
              mma_smem(tmu + 256, operand_desc(low + k * (2048 >> 4)), operand_desc(p_low + ((part * S::kP + k * 2048) >> 4)),
                       desc, part > 0 || k > 0 || j > 0, leader);
          mma_commit(smem_u32(&s_pv_done), leader);
          mma_commit(smem_u32(&s_v_empty[buf]), leader);
          if (++buf == S::kV) {
            buf = 0;
            phase ^= 1u;
          }
        }
      }
    } else if (warp == 9) {
      // ============================================================== loader warp
      constexpr unsigned int kBytes = F8 ? S::kRaw : S::kBuf;
      constexpr int kRow = F8 ? D : 128;
      const int boxes = kTileKeys >> a.box_log;
      unsigned int kbuf = 0, kphase = 1, vbuf = 0, vphase = 1, issued = 0;   // (a fresh barrier passes for phase 1)
      while (walk.next_warp(a, per)) {
        const uint32_t* row;
        long long entries;
        table_row(a.b, walk.r, row, entries);
        const bool tell = walk.head == 0 && walk.block == 0;
        if (walk.q.keys < walk.q.len && tell && walk.t0 == 0 && lane == 0)
          raise_status(AIBX_ERR_RANGE);                    // tokens the table has no entry for
        BoxIds<kTileKeys> ids(a, row, walk.span.tile0 + walk.t0, walk.span.tile0 + walk.t1, walk.span.lo,
                              walk.span.hi);
        const int head = walk.head, tile0 = walk.span.tile0, lo = walk.span.lo, hi = walk.span.hi, t1 = walk.t1;
        for (int j = walk.t0; j < t1; ++j, ++issued) {
          uint32_t block_id;
          const bool valid = ids.give(block_id, head == 0);
          const int slot = ids.slot;
          ids.step_slot();
          // a box that is not there, or that holds no visible key, comes as zeros from beyond the pool
          const int block = valid ? (int)block_id : (int)a.pool.num_blocks;
          const int tok = (tile0 + j) * kTileKeys + (lane & (boxes - 1)) * a.box;
          const bool missing = lane < boxes && tok < hi && tok > lo - a.box && !valid;
          const unsigned int gone = __ballot_sync(0xffffffffu, missing);
          if (lane == 0) s_mask[issued % kInfoRing] = ~gone;
          for (int kv = 0; kv < 2; ++kv) {
            const unsigned int buf = kv ? vbuf : kbuf;
            ring_wait(smem_u32(kv ? &s_v_empty[vbuf] : &s_k_empty[kbuf]), kv ? vphase : kphase, abort_flag);
            __syncwarp();
            const unsigned int bar = smem_u32(kv ? (F8 ? &s_v_raw[vbuf] : &s_v_full[vbuf]) : (F8 ? &s_k_raw[kbuf] : &s_k_full[kbuf]));
            if (__any_sync(0xffffffffu, *abort_flag)) {
              if (lane == 0) mbar_arrive(bar);
            } else {
              if (lane == 0) mbar_arrive_expect_tx(bar, kBytes);
              __syncwarp();
              if (lane < boxes) {
                const unsigned int dst = (kv ? v0 : k0) + (F8 ? S::kColBytes : 0) + buf * S::kBuf + lane * a.box * kRow;
#pragma unroll
                for (int cc = 0; cc < (F8 ? 1 : S::kCols); ++cc)
                  tensor_load_5d(dst + cc * S::kColBytes, &map, bar, cc * 64, slot, head, block, kv);
              }
            }
            __syncwarp();
          }
          if (++kbuf == S::kK) {
            kbuf = 0;
            kphase ^= 1u;
          }
          if (++vbuf == S::kV) {
            vbuf = 0;
            vphase ^= 1u;
          }
        }
      }
      // nothing may still be on its way here when the CTA ends: no copy, no word of a product
      for (unsigned int i = issued > S::kK ? issued - S::kK : 0; i < issued; ++i) {
        ring_drain(smem_u32(F8 ? &s_k_raw[i % S::kK] : &s_k_full[i % S::kK]), (i / S::kK) & 1u);
        ring_wait(smem_u32(&s_k_empty[i % S::kK]), (i / S::kK) & 1u, abort_flag);
      }
      for (unsigned int i = issued > S::kV ? issued - S::kV : 0; i < issued; ++i) {
        ring_drain(smem_u32(F8 ? &s_v_raw[i % S::kV] : &s_v_full[i % S::kV]), (i / S::kV) & 1u);
        ring_wait(smem_u32(&s_v_empty[i % S::kV]), (i / S::kV) & 1u, abort_flag);
      }
    } else if (F8 && warp == 11) {
      // ============================================================== scale bytes, four keys a lane
      unsigned int step = 0;
      while (walk.next_warp(a, per)) {
        const uint32_t* row;
        long long entries;
        table_row(a.b, walk.r, row, entries);
        const int head = walk.head, tile0 = walk.span.tile0, lo = walk.span.lo, hi = walk.span.hi, t1 = walk.t1;
        for (int j = walk.t0; j < t1; ++j, ++step) {
          const int tok = (tile0 + j) * kTileKeys + lane * 4;   // four slots of one block
          uint32_t kb = 0x7f7f7f7fu, vb = 0x7f7f7f7fu;
          unsigned int there = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (tok + i >= lo && tok + i < hi) there |= 1u << i;
          if (there) {
            const int at = tok / a.pool.T;
            const uint32_t block = __ldg(row + at);
            if (block < a.pool.num_blocks) {
              const unsigned char* src = a.pool.scales + (long long)block * a.pool.s_block +
                                         (long long)head * a.pool.s_head +
                                         (long long)(tok - at * a.pool.T) * a.pool.s_slot;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t x = __ldg(src + i * a.pool.s_slot), y = __ldg(src + a.pool.s_kv + i * a.pool.s_slot);
                if ((there >> i) & 1u) {
                  kb = (kb & ~(255u << (8 * i))) | x << (8 * i);
                  vb = (vb & ~(255u << (8 * i))) | y << (8 * i);
                }
              }
            }
          }
          bool odd = there != 15u;                         // (rows outside: zeros)
#pragma unroll
          for (int i = 0; i < 4; ++i) odd |= (int)((vb >> (8 * i)) & 255u) != weight_byte((vb >> (8 * i)) & 255u);
          odd = __any_sync(0xffffffffu, odd);
          const unsigned int f = step % kColInfo;
          ring_wait(smem_u32(&s_info_empty[f]), ((step / kColInfo) & 1u) ^ 1u, abort_flag);
          __syncwarp();
          *reinterpret_cast<uint32_t*>(&s_bytes[f][0][lane * 4]) = kb;
          *reinterpret_cast<uint32_t*>(&s_bytes[f][1][lane * 4]) = vb;
          if (lane == 0) s_odd[f] = odd;
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&s_info_full[f]));
        }
      }
    }
  } else if constexpr (F8) {
    // ================================================================ converter warps (12 .. 15)
    regs_down<S::kRegsOther>();
    // A thread takes one 16-byte piece of kRows neighbouring rows, half of them at a time; a row's
    // pieces are one warp's, which has read them all before it writes over them.
    const int tid = threadIdx.x - 384;
    constexpr int kPieces = D / 16;                        // 16-byte pieces of a raw row
    constexpr int kRows = kTileKeys * kPieces / 128;
    const int c = tid % kPieces, i0 = tid / kPieces * kRows;
    unsigned int kbuf = 0, kphase = 0, vbuf = 0, vphase = 0, step = 0;
    while (walk.next_warp(a, per)) {
      const int steps = walk.t1 - walk.t0;
      const int key_first = (walk.span.tile0 + walk.t0) * kTileKeys, lo = walk.span.lo, hi = walk.span.hi;
      for (int j = 0; j < steps; ++j, ++step) {
        const unsigned int f = step % kColInfo;
        auto convert = [&](unsigned int at, auto is_v, auto odd) {
          unsigned char* out = base + at + (c >> 2) * S::kColBytes;
          const unsigned char* src = base + at + S::kColBytes;
          constexpr int kTurn = kRows / 2;
#pragma unroll
          for (int u0 = 0; u0 < kRows; u0 += kTurn) {
            uint4 v[kTurn];
#pragma unroll
            for (int u = 0; u < kTurn; ++u) {
              const int i = i0 + u0 + u;
              v[u] = *reinterpret_cast<const uint4*>(src + i * D + ((D == 128 ? c ^ (i & 7) : c) << 4));
            }
            __syncwarp();
#pragma unroll
            for (int u = 0; u < kTurn; ++u) {
              const int i = i0 + u0 + u;
              const uint32_t wv[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
              uint32_t o[8];
              float rest = 1.0f;
              bool gone = false;
              if constexpr (decltype(odd)::value) {
                const int key = key_first + j * kTileKeys + i, vb = s_bytes[f][1][i];
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
                else
                  o[e] = bf16_of_e4m3(two, 1.0f);
              }
              const int p0 = (2 * c) & 7;
              *reinterpret_cast<uint4*>(out + i * 128 + ((p0 ^ (i & 7)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
              *reinterpret_cast<uint4*>(out + i * 128 + (((p0 + 1) ^ (i & 7)) << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        };
        ring_wait(smem_u32(&s_k_raw[kbuf]), kphase, abort_flag);
        __syncwarp();
        convert((k0 - smem0) + kbuf * S::kBuf, std::false_type(), std::false_type());
        mbar_arrive(smem_u32(&s_k_full[kbuf]));
        if (++kbuf == S::kK) {
          kbuf = 0;
          kphase ^= 1u;
        }
        ring_wait(smem_u32(&s_info_full[f]), (step / kColInfo) & 1u, abort_flag);
        ring_wait(smem_u32(&s_v_raw[vbuf]), vphase, abort_flag);
        __syncwarp();
        if (s_odd[f])
          convert((v0 - smem0) + vbuf * S::kBuf, std::true_type(), std::true_type());
        else
          convert((v0 - smem0) + vbuf * S::kBuf, std::true_type(), std::false_type());
        mbar_arrive(smem_u32(&s_v_full[vbuf]));
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_info_empty[f]));
        if (++vbuf == S::kV) {
          vbuf = 0;
          vphase ^= 1u;
        }
      }
    }
  }
  tmem_before();
  __syncthreads();
  if (warp == 8) {
    tmem_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

template <int D, bool F8, typename QT, int N>
inline int32_t launch_attn_cols(AttnArgs a, int type, JoinSet& join, cudaStream_t st) {
  using S = ColRings<D, F8, N, F8 && std::is_same<QT, __half>::value ? 2 : 1>;
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
