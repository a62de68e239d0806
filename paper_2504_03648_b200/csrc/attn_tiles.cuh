// Attention of chunks of new tokens over a paged cache on the 5th-generation tensor cores.
//
// A CTA works on a block of 256 query rows of one (request, KV head) - row = token * G + query
// head of the group, so that the heads which share K and V share their tiles - as two tiles of
// 128 rows, against KV tiles of 128 positions:
//   S = Q K^T          tcgen05.mma, Q and K from shared memory, S in tensor memory (fp32)
//   P = 2^(S c - m)    one thread per row: S to registers, running maximum m (moved only when it
//                      grows by more than 2^8, so that O is rarely rescaled), P to tensor memory
//                      over S, as 16-bit
//   O += P V           tcgen05.mma, P from tensor memory, V from shared memory as it lies in the
//                      pool ([position][dim], the operand's N-major form), O in tensor memory
// Roles: two softmax warpgroups (one per tile), a warp per tile that issues its MMAs, one warp that
// feeds a ring of K and V tiles with tensor-map boxes (one box = the slots of one block and head that
// fall into the tile).  The MMA warps take turns, PV(j) and S(j + 1) of one tile, then of the other:
// while one tile's rows are exponentiated the other tile's MMAs run (without turns both tiles fall
// into step, softmax with softmax: 948 instead of 805 us for six chunks over cached prefixes).  A
// tile's MMAs complete in issue order, and S of step j + 1 is issued behind PV of step j: seeing
// S(j + 1) is therefore also seeing O(j), and no further barrier guards O.
//
// Over an e4m3 pool a warpgroup more turns each raw tile into fp16 as it arrives: element times
// 2^(e - E), e its row's exponent and E the tile's largest; 2^E then joins the scale of the scores (K) or
// the exponent of the weights (V: m covers S c + E, and l takes the sum of the weights times 2^-E).
// That is exact while the tile's exponents are close together.  Steps where they are far apart (see
// kKeySpread, kScaleSpread) leave K without its scales, which the softmax applies score by score, and
// turn V into bf16.  Queries become fp16 scaled to [1, 2) per row.
//
// Bound: the tensor pipe (1024 cycles per KV tile and 128 rows at D = 128, both products) and the
// special function unit (128 * 128 exponentials at 16 a cycle: 1024 cycles too), neither of them
// busy all the time: a step of both tiles takes about 3,800 cycles where both pipes need 2,048, and
// 5,300 over e4m3, where the converters share the schedulers and warps wait for instructions (the roles'
// code together exceeds what the instruction cache holds: every addition to the softmax or MMA loop
// shows).  Six chunks of 8,505 tokens over prefixes of 1k to 8k (16-bit, 32 query heads on 8): 890 us,
// 865 TFLOP/s, at the 1.67 GHz that the power cap leaves; a 1,023-token chunk over 130k e4m3 positions:
// 2,360 us, 810 TFLOP/s, at 1.9 GHz.
#pragma once

#include "attn_rows.cuh"

namespace aibx {

constexpr int kTileRows = 128;
constexpr int kTileKeys = 128;
constexpr int kKeySpread = 14;       // of K's bytes in a tile: times 2^-14, fp16's least normal number, e4m3 is exact
constexpr int kInfoRing = 16;        // per-step facts the softmax reads: far deeper than the rings

template <int D, bool F8>
struct TileShape {
  static constexpr int kThreads = F8 ? 512 : 384;
  static constexpr int kRaw = kTileKeys * D;               // a tile's e4m3 rows, as they arrive
  // One K or V tile as MMA operand.  Raw rows arrive 16 KB into the buffer: at D = 128 that is the
  // second column, and every 128-byte raw row lies where the second half of its own fp16 row goes.
  static constexpr int kBuf = kTileKeys * D * 2 + (F8 && D == 64 ? kRaw : 0);
  static constexpr int kBufs = D == 64 ? (F8 ? 6 : 8) : (F8 ? 4 : 5);
  static constexpr int kFactorRing = 4;
  static constexpr int kCols = D / 64;                     // 128-byte columns of an operand row
  static constexpr int kColBytes = 128 * 128;
  static constexpr int kQ = kTileRows * D * 2;
  static constexpr int kSmem = 2 * kQ + kBufs * kBuf +
                               (F8 ? kFactorRing * 2 * kTileKeys * 2 + 2 * kTileRows * 4 : 0) + 1024;
  static constexpr int kSlot = 2 * kTileRows * (D + 2);    // floats per workspace slot
  static constexpr int kRegsSoftmax = F8 ? 176 : 200;      // launch: 128 (512 threads), 168 (384)
  static constexpr int kRegsOther = F8 ? 80 : 104;          // 2 * 176 + 2 * 80 = 4 * 128; 2 * 200 + 104 = 3 * 168
};

// ------------------------------------------------------------------------------------------
// tensor-core wrappers

// Shared-memory operand: 128-byte swizzle, groups of 8 rows 1024 bytes apart; `lbo` bytes between
// 64-element columns (N-major operands).
__device__ __forceinline__ unsigned int operand_low(unsigned int addr, unsigned int lbo) {
  return (addr >> 4) | ((lbo >> 4) << 16);
}
__device__ __forceinline__ uint64_t operand_desc(unsigned int lo) {
  constexpr unsigned int hi = (1024u >> 4) | (1u << 14) | (2u << 29);      // version 1 at bit 46
  return ((uint64_t)hi << 32) | lo;
}

// fp32 accumulator, M = 128; `half` operands or bfloat16; B as it lies (K-major) or N-major
__host__ __device__ constexpr unsigned int mma_desc(bool half, int n, bool b_n_major) {
  return (1u << 4) | ((half ? 0u : 1u) << 7) | ((half ? 0u : 1u) << 10) | ((b_n_major ? 1u : 0u) << 16) |
         ((unsigned int)(n >> 3) << 17) | ((128u >> 4) << 24);
}

// MMAs and commits run convergent, with a predicate for the one lane that issues: everything that
// goes into a descriptor stays warp-uniform and needs no detour through vector registers (issued
// inside `if (lane == 0)` an MMA took 120 cycles to issue and 64 to execute).
__device__ __forceinline__ void mma_smem(unsigned int d, uint64_t a, uint64_t b, unsigned int idesc,
                                         unsigned int add, unsigned int leader) {
  asm volatile(
      "{\n.reg .pred p, q;\nsetp.ne.u32 p, %4, 0;\nsetp.ne.u32 q, %5, 0;\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(add), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void mma_tmem(unsigned int d, unsigned int a, uint64_t b, unsigned int idesc,
                                         unsigned int add, unsigned int leader) {
  asm volatile(
      "{\n.reg .pred p, q;\nsetp.ne.u32 p, %4, 0;\nsetp.ne.u32 q, %5, 0;\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(add), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void mma_commit(unsigned int bar, unsigned int leader) {
  asm volatile(
      "{\n.reg .pred q;\nsetp.ne.u32 q, %1, 0;\n"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(bar),
      "r"(leader)
      : "memory");
}
__device__ __forceinline__ void tmem_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void tmem_ld32(unsigned int addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_st32(unsigned int addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]),
      "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]),
      "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(unsigned int addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(
          r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr)
      : "memory");
}

// Two fp32 operations in one instruction, and the maximum of three (NaN if one is).
__device__ __forceinline__ uint64_t pair2(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ void split2(uint64_t v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// ------------------------------------------------------------------------------------------
// the line of work

// KV tiles of one block of 256 rows: the positions [lo, hi) that some row of it sees.
struct TileSpan {
  int lo, hi, tile0, tiles;
};

// How a request's rows are cut into blocks, and which tiles a block has: of 256 rows, two tiles of a CTA.
struct PairBlocks {
  static __device__ __forceinline__ int size(int) { return 2 * kTileRows; }
  static __device__ __forceinline__ int blocks(const AttnArgs& a, const AttnRequest& q) {
    const long long rows = (long long)q.n * a.G;
    return rows <= a.row_limit ? 0 : (int)((rows + 2 * kTileRows - 1) / (2 * kTileRows));
  }
  static __device__ __forceinline__ TileSpan span(const AttnArgs& a, const AttnRequest& q, int block) {
    const int rows = q.n * a.G;
    const int r0 = block * 2 * kTileRows, r1 = min(r0 + 2 * kTileRows, rows) - 1;
    const long long first = (long long)q.len - q.n;
    TileSpan s;
    long long hi = a.causal ? first + a.by_g.div(r1) + 1 : q.keys;
    hi = hi < 0 ? 0 : hi > q.keys ? q.keys : hi;
    long long lo = a.window > 0 ? first + a.by_pos.div(r0) - a.window + 1 : 0;
    lo = lo < 0 ? 0 : lo > hi ? hi : lo;
    s.hi = (int)hi;
    s.lo = (int)lo;
    s.tile0 = s.lo / kTileKeys;
    s.tiles = max(1, (int)(((unsigned int)s.hi + kTileKeys - 1) / kTileKeys) - s.tile0);
    return s;
  }
};

// Tiles of a request for one head.  Requests of many blocks of rows are summed by the whole warp,
// 32 blocks at a time (one thread over 128 blocks took tens of microseconds before the first load).
template <typename B>
struct TileCost {
  const AttnArgs& a;
  __device__ __forceinline__ int blocks(const AttnRequest& q) const { return B::blocks(a, q); }
  __device__ __forceinline__ long long operator()(int r, bool on) const {
    AttnRequest q = {};
    if (on) q = attn_request(a.b, a.pool.T, r);
    const int n = on ? blocks(q) : 0;
    long long sum = 0;
    if (n <= 4)
      for (int b = 0; b < n; ++b) sum += B::span(a, q, b).tiles;
    for (unsigned int many = __ballot_sync(0xffffffffu, n > 4); many; many &= many - 1) {
      const int src = __ffs(many) - 1, lane = threadIdx.x & 31;
      AttnRequest w;
      w.n = __shfl_sync(0xffffffffu, q.n, src);
      w.len = __shfl_sync(0xffffffffu, q.len, src);
      w.keys = __shfl_sync(0xffffffffu, q.keys, src);
      const int wn = blocks(w);
      long long part = 0;
      for (int b = lane; b < wn; b += 32) part += B::span(a, w, b).tiles;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) part += (long long)shfl_xor64(0xffffffffu, (uint64_t)part, d);
      if (lane == src) sum = part;
    }
    return sum * a.pool.H;
  }
};

// A request's part of the line: its (head, block of rows) segments, head by head, dealt out like cards
// to the g pieces that cover it: segments 0, g, 2 g .. come first, then 1, g + 1 .., and so on.  Pieces
// are worked on at the same time, so at any moment their CTAs stand at about g neighbouring segments,
// which share one or two heads' keys in L2.  (Segment after segment, every piece stood at a head of its
// own, and keys came from DRAM six times: six chunks 936 instead of 821 us from a cold L2, two whole
// prompts 1,170 instead of 1,070.)
struct RequestLine {
  int blocks, g;
};

template <typename B>
__device__ __forceinline__ RequestLine request_line(const AttnArgs& a, const AttnRequest& q, long long per) {
  RequestLine line;
  line.blocks = TileCost<B>{a}.blocks(q);
  long long tiles = 0;
  for (int b = threadIdx.x & 31; b < line.blocks; b += 32) tiles += B::span(a, q, b).tiles;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) tiles += (long long)shfl_xor64(0xffffffffu, (uint64_t)tiles, d);
  const long long g = (tiles * a.pool.H + per / 2) / per, most = (long long)line.blocks * a.pool.H;
  line.g = (int)(g < 1 ? 1 : g > most ? most : g);
  return line;
}

// By one warp: where in its request a piece begins.
template <typename B>
__device__ __forceinline__ void locate_block(const AttnArgs& a, unsigned int index, unsigned int pieces, WorkStart* w) {
  if (w->r < 0) return;
  const int lane = threadIdx.x & 31;
  const AttnRequest q = attn_request(a.b, a.pool.T, w->r);
  const long long per = (w->total + pieces - 1) / pieces;
  const RequestLine line = request_line<B>(a, q, per);
  long long off = per * index - w->base;
  const int dh = line.g / line.blocks, db = line.g - dh * line.blocks;      // g segments on
  for (int c0 = 0; c0 < line.g; c0 += 32) {
    const int c = c0 + lane;
    long long tiles = 0;                                     // of the segments c, c + g, c + 2 g ..
    if (c < line.g) {
      int h = c / line.blocks, b = c - h * line.blocks;
      while (h < a.pool.H) {
        tiles += B::span(a, q, b).tiles;
        h += dh;
        b += db;
        if (b >= line.blocks) {
          b -= line.blocks;
          ++h;
        }
      }
    }
    long long upto = tiles;                                  // and of all classes before
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long up = (long long)shfl_up64((uint64_t)upto, d);
      if (lane >= d) upto += up;
    }
    const unsigned int past = __ballot_sync(0xffffffffu, c < line.g && off < upto);
    if (past) {
      if (lane == __ffs(past) - 1) {
        long long left = off - (upto - tiles);
        int h = c / line.blocks, b = c - h * line.blocks;
        for (;;) {
          const int here = B::span(a, q, b).tiles;
          if (left < here) break;
          left -= here;
          h += dh;
          b += db;
          if (b >= line.blocks) {
            b -= line.blocks;
            ++h;
          }
        }
        w->head = h;
        w->block = b;
        w->off = (int)left;
        w->cls = c;
        w->g = line.g;
      }
      break;
    }
    off -= (long long)shfl64(0xffffffffu, (uint64_t)upto, 31);
  }
}

// Walks a CTA's piece of the line, one (request, head, block of rows) at a time.  Each warp keeps
// its own in shared memory, moved on by its first lane: as registers of 16 warps it cost the
// softmax warps spills.
template <typename B>
struct TileWalk {
  long long pos, start, end;
  AttnRequest q;
  TileSpan span;
  int r, head, block, blocks, g, cls, t0, t1;
  int fresh;                         // block not yet entered

  __device__ void init(const AttnArgs& a, const WorkStart& w, unsigned int index, unsigned int pieces) {
    const long long per = (w.total + pieces - 1) / pieces;
    pos = start = per * index;
    end = min(pos + per, w.total);
    r = w.r;
    if (r < 0) pos = end = 0;
    if (pos >= end) return;
    q = attn_request(a.b, a.pool.T, r);
    blocks = TileCost<B>{a}.blocks(q);
    head = w.head;
    block = w.block;
    cls = w.cls;
    g = w.g;
    span = B::span(a, q, block);
    t1 = w.off;                      // where next() goes on
    fresh = 0;
  }
  // To the next segment: 0 none, 1 there, 2 the request is done (then enter() the next one, and again).
  __device__ int next(const AttnArgs& a) {
    if (pos >= end) return 0;
    if (fresh == 1) {
      const int dh = g / blocks;
      head += dh;
      block += g - dh * blocks;
      if (block >= blocks) {
        block -= blocks;
        ++head;
      }
      if (head >= a.pool.H) {
        if (++cls == g) return 2;
        head = cls / blocks;
        block = cls - head * blocks;
      }
    }
    if (fresh) {
      span = B::span(a, q, block);
      t1 = 0;
    }
    t0 = t1;
    const long long left = end - pos;
    t1 = left < span.tiles - t0 ? t0 + (int)left : span.tiles;
    pos += t1 - t0;
    fresh = 1;
    return 1;
  }
  // by a whole warp: the next request with work
  __device__ __forceinline__ void enter(const AttnArgs& a, long long per) {
    int x = r;
    AttnRequest next_q;
    RequestLine line;
    do {
      ++x;
      next_q = attn_request(a.b, a.pool.T, x);
    } while (TileCost<B>{a}.blocks(next_q) == 0);
    line = request_line<B>(a, next_q, per);
    __syncwarp();
    if ((threadIdx.x & 31) == 0) {
      r = x;
      q = next_q;
      blocks = line.blocks;
      g = line.g;
      cls = head = block = 0;
      fresh = 2;                     // at its first segment
    }
    __syncwarp();
  }
  // by a whole warp
  __device__ __forceinline__ bool next_warp(const AttnArgs& a, long long per) {
    for (;;) {
      __syncwarp();
      int more = 0;
      if ((threadIdx.x & 31) == 0) more = next(a);
      more = __shfl_sync(0xffffffffu, more, 0);
      __syncwarp();                  // (a shuffle orders no memory: the other lanes read what next() wrote)
      if (more != 2) return more != 0;
      enter(a, per);
    }
  }
  __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == span.tiles; }
  __device__ __forceinline__ int rows(const AttnArgs& a) const {
    const int size = B::size(q.n * a.G);
    return min(q.n * a.G - block * size, size);
  }
};

template <int REGS>
__device__ __forceinline__ void regs_up() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS));
}
template <int REGS>
__device__ __forceinline__ void regs_down() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS));
}

// TREE: rows are a drafted tree's, and see the nodes that their masks name.
template <int D, bool F8, typename QT, bool TREE>
__global__ void __launch_bounds__(TileShape<D, F8>::kThreads, 1)
attn_tiles_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ AttnArgs a) {
  using S = TileShape<D, F8>;
  using MT = typename std::conditional<F8, __half, QT>::type;
  extern __shared__ unsigned char s_raw[];
  __shared__ __align__(8) unsigned long long s_kv_full[S::kBufs], s_kv_empty[S::kBufs];
  __shared__ __align__(8) unsigned long long s_raw_full[S::kBufs];
  __shared__ __align__(8) unsigned long long s_fac_full[S::kFactorRing], s_fac_empty[S::kFactorRing];
  __shared__ __align__(8) unsigned long long s_q_full[2], s_s_full[2], s_h_full[2], s_p_full[2], s_o_full[2], s_turn[2], s_w_full[2];
  __shared__ unsigned int s_mask[kInfoRing];
  __shared__ float s_kscale[kInfoRing], s_vexp[kInfoRing];
  __shared__ int s_wide[kInfoRing];                        // whether the step's scales are far apart, and if so
  __shared__ float s_wide_vexp[kInfoRing];                 // V's exponent and K's bytes
  __shared__ __align__(4) unsigned char s_kbytes[F8 ? kInfoRing : 1][kTileKeys];
  __shared__ long long s_scan[33];
  __shared__ WorkStart s_start;
  __shared__ TileWalk<PairBlocks> s_walk[S::kThreads / 32];
  __shared__ unsigned int s_tmem;
  __shared__ int s_abort;

  const unsigned int smem0 = (smem_u32(s_raw) + 1023u) & ~1023u;
  unsigned char* base = s_raw + (smem0 - smem_u32(s_raw));
  __half* factors = reinterpret_cast<__half*>(base + 2 * S::kQ + S::kBufs * S::kBuf);
  float* s_qup = reinterpret_cast<float*>(factors + S::kFactorRing * 2 * kTileKeys);
  const unsigned int kv0 = smem0 + 2 * S::kQ;
  const int lane = threadIdx.x & 31;
  // the same in all lanes, and known to be: role code may keep it in uniform registers
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  volatile int* abort_flag = &s_abort;

  if (threadIdx.x == 0) {
    for (int i = 0; i < S::kBufs; ++i) {
      mbar_init(smem_u32(&s_kv_full[i]), F8 ? 128u : 1u);
      mbar_init(smem_u32(&s_kv_empty[i]), 2u);
      mbar_init(smem_u32(&s_raw_full[i]), 1u);
    }
    for (int i = 0; i < S::kFactorRing; ++i) {
      mbar_init(smem_u32(&s_fac_full[i]), 1u);
      mbar_init(smem_u32(&s_fac_empty[i]), 4u);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&s_q_full[t]), 128u);
      mbar_init(smem_u32(&s_s_full[t]), 1u);
      mbar_init(smem_u32(&s_h_full[t]), 4u);
      mbar_init(smem_u32(&s_p_full[t]), 4u);
      mbar_init(smem_u32(&s_o_full[t]), 1u);
      mbar_init(smem_u32(&s_turn[t]), 1u);
      mbar_init(smem_u32(&s_w_full[t]), 1u);
    }
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    tmem_before();
  }
  const TileCost<PairBlocks> cost{a};
  locate_piece<S::kThreads>(a.b.R, blockIdx.x, gridDim.x, s_scan, &s_start, cost);
  if (warp == 0) {
    locate_block<PairBlocks>(a, blockIdx.x, gridDim.x, &s_start);
    __syncwarp();
    if (lane == 0) {
      TileWalk<PairBlocks> look;
      look.init(a, s_start, blockIdx.x, gridDim.x);
      JoinRecord rec = {};
      if (look.next(a) == 1 && look.t0 > 0 && look.t1 == look.span.tiles) {
        const long long per = (s_start.total + gridDim.x - 1) / gridDim.x;
        const long long p0 = look.pos - look.t1;           // position of the rows' first tile
        rec.tok0 = look.q.tok0;
        rec.rows = look.rows(a);
        rec.row0 = look.block * 2 * kTileRows;
        rec.head = look.head;
        rec.first_cta = (int)(p0 / per);
        rec.first_slot = p0 != rec.first_cta * per;
      }
      reinterpret_cast<JoinRecord*>(a.slots + 2ull * gridDim.x * S::kSlot)[blockIdx.x] = rec;
    }
  }
  __syncthreads();
  tmem_after();
  const unsigned int tmem = s_tmem;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const long long per = (s_start.total + gridDim.x - 1) / gridDim.x;
  TileWalk<PairBlocks>& walk = s_walk[warp];
  if (lane == 0) walk.init(a, s_start, blockIdx.x, gridDim.x);
  __syncwarp();

  if (warp < 8) {
    // ================================================================ softmax: thread = row
    regs_up<S::kRegsSoftmax>();
    const int t = warp >> 2;                               // tile
    const int row = threadIdx.x & 127;
    const unsigned int lanes = (unsigned int)(warp & 3) << 21;
    const unsigned int tm_s = tmem + lanes + t * 128;
    const unsigned int tm_o = tmem + lanes + 256 + t * D;
    unsigned int s_phase = 0, o_phase = 0, w_phase = 0, step = 0;
    while (walk.next_warp(a, per)) {
      const int rows_here = walk.rows(a) - t * kTileRows;   // rows of this tile (<= 0: none)
      const int steps = walk.t1 - walk.t0;
      if (rows_here <= 0) {
        step += steps;
        continue;
      }
      const int row0 = walk.block * 2 * kTileRows + t * kTileRows;   // in the request's rows
      if constexpr (F8) {                                  // O = 0: every product of a step adds to it
        uint32_t zero[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) zero[e] = 0;
#pragma unroll
        for (int k = 0; k < D; k += 32) tmem_st32(tm_o + k, zero);
        tmem_wait_st();
        tmem_before();
      }
      // ---- queries into shared memory
      {
        constexpr int kChunks = D / 8;                     // 16-byte pieces of a row
        const int c = row % kChunks;
        unsigned char* dst = base + t * S::kQ + (c >> 3) * S::kColBytes;
        constexpr int kBatch = 8;                          // rows on their way at once
        for (int i0 = row / kChunks; i0 < kTileRows; i0 += kBatch * (128 / kChunks)) {
          uint4 batch[kBatch];
#pragma unroll
          for (int u = 0; u < kBatch; ++u) {
            const int ri = row0 + min(i0 + u * (128 / kChunks), rows_here - 1);
            const int ti = a.by_g.div(ri), gi = ri - ti * a.G;
            batch[u] = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const QT*>(a.q) +
                                                            (walk.q.tok0 + ti) * a.q_tok +
                                                            (long long)(walk.head * a.G + gi) * a.q_head + c * 8));
          }
#pragma unroll
          for (int u = 0; u < kBatch; ++u) {
            const int i = i0 + u * (128 / kChunks);
            uint4 v = i < rows_here ? batch[u] : make_uint4(0, 0, 0, 0);
            if constexpr (F8) {
              uint32_t x[4] = {v.x, v.y, v.z, v.w};
              float amax = 0.0f;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float2 f = Bits16<QT>::unpack(x[e]);
                amax = fmaxf(amax, fmaxf(fabsf(f.x), fabsf(f.y)));
              }
#pragma unroll
              for (int m = 1; m < kChunks; m <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, m));
              float down, up;
              power_scale(amax, down, up);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float2 f = Bits16<QT>::unpack(x[e]);
                x[e] = Bits16<MT>::pack(f.x * down, f.y * down);
              }
              v = make_uint4(x[0], x[1], x[2], x[3]);
              if (c == 0) s_qup[t * kTileRows + i] = up;
            }
            *reinterpret_cast<uint4*>(dst + i * 128 + (((c & 7) ^ (i & 7)) << 4)) = v;
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_arrive(smem_u32(&s_q_full[t]));
        if (F8) asm volatile("bar.sync %0, 128;" ::"r"(1 + t) : "memory");
      }
      const float c0 = F8 ? a.scale_log2 * s_qup[t * kTileRows + row] : a.scale_log2;
      const int tok = a.by_g.div(row0 + min(row, rows_here - 1));
      const int first = walk.q.len - walk.q.n;
      const uint32_t* tree = TREE ? a.mask + (walk.q.tok0 + tok) * a.mask_words : nullptr;
      // this row's position
      const long long p = (long long)first + (!TREE ? tok : a.window > 0 ? tree_depth(tree, a.mask_words, walk.q.n) : 0);
      // positions [vis0, vis1) this row sees (of those that are there; trees: of the cached ones)
      const int vis1 = (int)max(0LL, TREE ? min((long long)first, (long long)walk.span.hi)
                                     : a.causal ? min(p + 1, (long long)walk.span.hi) : (long long)walk.span.hi);
      const int vis0 = a.window > 0 ? (int)max((long long)walk.span.lo, p - a.window + 1) : walk.span.lo;
      const int key_first = (walk.span.tile0 + walk.t0) * kTileKeys;
      float m = -INFINITY, l = 0.0f;
      for (int j = 0; j < steps; ++j, ++step) {
        ring_wait(smem_u32(&s_s_full[t]), s_phase, abort_flag);
        s_phase ^= 1u;
        __syncwarp();
        tmem_after();
        const int key0 = key_first + j * kTileKeys;
        const unsigned int mask = s_mask[step % kInfoRing];
        float c = c0, shift = 0.0f;
        bool spread = false;
        if constexpr (F8) {
          spread = s_wide[step % kInfoRing];
          c = fmaxf(c * s_kscale[step % kInfoRing], 1.2e-38f);   // (0 would make NaN of a hidden key's -infinity)
          shift = s_vexp[step % kInfoRing];
        }
        const int b0 = vis0 - key0, b1 = vis1 - key0;
        const bool hide = mask != 0xffffffffu || b1 < kTileKeys || b0 > 0;
        // what this row sees of the tile, a bit per key
        uint32_t vis[4];
        if (hide) {
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int lo = min(max(b0 - 32 * x, 0), 32), hi = min(max(b1 - 32 * x, 0), 32);
            vis[x] = (uint32_t)((1ull << hi) - 1) & ~(uint32_t)((1ull << lo) - 1);
            if (TREE) vis[x] |= tree_bits(tree, a.mask_words, walk.span.hi - first, key0 + 32 * x - first);
          }
          if (mask != 0xffffffffu) {                       // blocks that are not there
            for (int k = 0; k < kTileKeys >> a.box_log; ++k)
              if (!((mask >> k) & 1u))
                for (int e = 0; e < a.box; e += 8) vis[((k << a.box_log) + e) >> 5] &= ~(0xffu << (((k << a.box_log) + e) & 31));
          }
        }
        auto hide_keys = [&](uint32_t* x, int w) {
#pragma unroll
          for (int k = 0; k < 64; ++k)
            if (!(vis[w + (k >> 5)] & (1u << (k & 31)))) x[k] = 0xff800000u;
        };
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        auto raise_max = [&](const uint32_t* x) {
#pragma unroll
          for (int e = 0; e < 64; e += 8)
#pragma unroll
            for (int y = 0; y < 4; ++y)
              mx[y] = max3(mx[y], __uint_as_float(x[e + 2 * y]), __uint_as_float(x[e + 2 * y + 1]));
        };
        const uint64_t c2 = pair2(c, c);
        uint64_t off2, sum2;
        auto weights = [&](const uint32_t* x, uint32_t* pk) {   // of 64 scores, packed
#pragma unroll
          for (int e = 0; e < 64; e += 2) {
            float p0, p1;
            const uint64_t z = fma2(pair2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), c2, off2);
            split2(z, p0, p1);
            p0 = exp2_fast(p0);
            p1 = exp2_fast(p1);
            sum2 = add2(sum2, pair2(p0, p1));
            pk[e >> 1] = Bits16<MT>::pack(p0, p1);
          }
        };
        uint32_t s[128], pk[32];
        tmem_ld32(tm_s, s);
        tmem_ld32(tm_s + 32, s + 32);
        tmem_wait_ld();
        tmem_ld32(tm_s + 64, s + 64);
        tmem_ld32(tm_s + 96, s + 96);
        // The first half's weights are taken with the maximum so far while the second half arrives
        // and the new maximum forms; it hardly ever moves, and then they are taken again.
        if (hide) hide_keys(s, 0);
        float off = (m == -INFINITY ? 0.0f : m) - shift;
        off2 = pair2(-off, -off);
        sum2 = 0;                                          // two zeros
        weights(s, pk);
        raise_max(s);
        tmem_wait_ld();
        if (hide) hide_keys(s + 64, 2);
        raise_max(s + 64);
        const float mt = max3(max3(mx[0], mx[1], mx[2]), mx[3], mx[3]) * c + shift;
        if (!(mt < INFINITY)) l = NAN;                     // a NaN or infinite score: so is the row's result
        constexpr float kHead = kWeightHead<MT>;
        if (__any_sync(0xffffffffu, mt > m + (kHead + 8.0f))) {
          const float mn = fmaxf(m, mt - kHead);
          const float al = mn == -INFINITY ? 1.0f : exp2_fast(m - mn);
          m = mn;
          l *= al;
          if (j > 0) {
            constexpr int kUnroll = F8 ? 1 : D / 32;       // (over e4m3 the shorter code: 2,315 instead of 2,420 us)
#pragma unroll kUnroll
            for (int k = 0; k < D; k += 32) {
              uint32_t o[32];
              tmem_ld32(tm_o + k, o);
              tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * al);
              tmem_st32(tm_o + k, o);
            }
          }
          tmem_ld32(tm_s, s);
          tmem_ld32(tm_s + 32, s + 32);
          tmem_wait_ld();
          if (hide) hide_keys(s, 0);
          off = (m == -INFINITY ? 0.0f : m) - shift;
          off2 = pair2(-off, -off);
          sum2 = 0;
          weights(s, pk);
        }
        if (F8 && spread) {
          // Scales far apart.  Up to here the step had V exponent -infinity: no weights, no new maximum.
          // K is there without its scales, so every score takes its own; V is bf16, and weights are two
          // bf16 numbers, 16 columns of the first and 16 of the second in the place of 32 scores.  The
          // product is issued here, and the MMA warp's own of this step adds zeros: it knows of nothing
          // (with these 16 MMAs in its loop as well, taken or not, a 1,023-token chunk over 130k
          // positions took 2,820 us instead of 2,315; with every step like this 5,710).
          const float vexp = s_wide_vexp[step % kInfoRing];
          const unsigned char* bytes = s_kbytes[step % kInfoRing];
          float most = -INFINITY;
#pragma unroll 1
          for (int q = 0; q < 4; ++q) {
            tmem_ld32(tm_s + 32 * q, s);
            tmem_wait_ld();
            const uint32_t seen = !hide ? 0xffffffffu : q < 2 ? (q ? vis[1] : vis[0]) : (q > 2 ? vis[3] : vis[2]);
#pragma unroll
            for (int k = 0; k < 32; ++k) {
              const float z = __uint_as_float(s[k]) * power_of_byte(bytes[32 * q + k]);
              s[k] = seen & (1u << k) ? __float_as_uint(z) : 0xff800000u;
            }
#pragma unroll
            for (int k = 0; k < 32; k += 2) most = max3(most, __uint_as_float(s[k]), __uint_as_float(s[k + 1]));
            tmem_st32(tm_s + 32 * q, s);
          }
          tmem_wait_st();
          const float cw = fmaxf(c0, 1.2e-38f), mw = most * cw + vexp;
          if (!(mw < INFINITY)) l = NAN;
          if (__any_sync(0xffffffffu, mw > m + (kHead + 8.0f))) {
            const float mn = fmaxf(m, mw - kHead);
            const float al = mn == -INFINITY ? 1.0f : exp2_fast(m - mn);
            m = mn;
            l *= al;
#pragma unroll 1
            for (int k = 0; k < D; k += 32) {
              tmem_ld32(tm_o + k, s);
              tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 32; ++e) s[e] = __float_as_uint(__uint_as_float(s[e]) * al);
              tmem_st32(tm_o + k, s);
            }
          }
          const float below = vexp - (m == -INFINITY ? 0.0f : m);
          float total = 0.0f;
#pragma unroll 1
          for (int q = 0; q < 4; ++q) {
            uint32_t two[32];
            tmem_ld32(tm_s + 32 * q, s);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              const float p0 = exp2_fast(fmaf(__uint_as_float(s[e]), cw, below));
              const float p1 = exp2_fast(fmaf(__uint_as_float(s[e + 1]), cw, below));
              total += p0 + p1;
              two[e >> 1] = Bits16<__nv_bfloat16>::pack(p0, p1);
              const float2 y = Bits16<__nv_bfloat16>::unpack(two[e >> 1]);
              two[16 + (e >> 1)] = Bits16<__nv_bfloat16>::pack(p0 - y.x, p1 - y.y);
            }
            tmem_st32(tm_s + 32 * q, two);
          }
          l += total * power_of_byte(127 - (int)vexp);
          tmem_wait_st();
          tmem_before();
          asm volatile("bar.sync %0, 128;" ::"r"(1 + t) : "memory");
          if ((warp & 3) == 0) {
            constexpr unsigned int kPVWide = mma_desc(false, D, true);
            const unsigned int vbuf = (2 * step + 1) % S::kBufs;
            ring_wait(smem_u32(&s_kv_full[vbuf]), ((2 * step + 1) / S::kBufs) & 1u, abort_flag);
            __syncwarp();
            tmem_after();
            const unsigned int low = operand_low(kv0 + vbuf * S::kBuf, S::kColBytes);
#pragma unroll 1
            for (int k = 0; k < 16; ++k)                   // per 32 keys: 2 x 16 of the first part, then of the second
              mma_tmem(tmem + 256 + t * D, tmem + t * 128 + k * 8,
                       operand_desc(low + ((k >> 2) * 2 + (k & 1)) * (2048 >> 4)), kPVWide, 1u, lane == 0);
            mma_commit(smem_u32(&s_w_full[t]), lane == 0);
          }
          ring_wait(smem_u32(&s_w_full[t]), w_phase, abort_flag);
          w_phase ^= 1u;
          __syncwarp();
          tmem_after();
          // the MMA warp's own product of the step: zeros (V's bf16 bits are finite numbers as fp16, too)
#pragma unroll
          for (int e = 0; e < 32; ++e) pk[e] = 0;
          tmem_st32(tm_s, pk);
          tmem_st32(tm_s + 32, pk);
          tmem_wait_st();
          tmem_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&s_h_full[t]));
        } else {
          tmem_st32(tm_s, pk);
          tmem_wait_st();
          tmem_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&s_h_full[t]));   // the first half may be multiplied already
          weights(s + 64, pk);
          tmem_st32(tm_s + 32, pk);
          float total, other;
          split2(sum2, total, other);
          total += other;
          l += F8 ? total * power_of_byte(127 - (int)shift) : total;   // (2^-127 too: no flushing here)
        }
        tmem_wait_st();
        tmem_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_p_full[t]));
      }
      // ---- O out of tensor memory
      ring_wait(smem_u32(&s_o_full[t]), o_phase, abort_flag);
      o_phase ^= 1u;
      __syncwarp();
      tmem_after();
      const bool whole = walk.whole();
      const bool at_start = walk.pos - steps == walk.start;
      float* slot = a.slots + ((long long)blockIdx.x * 2 + (at_start ? 0 : 1)) * S::kSlot;
      const int srow = t * kTileRows + row;
      const bool on = row < rows_here;
      const long long otok = walk.q.tok0 + tok;
      const int qh = walk.head * a.G + (row0 + row - tok * a.G);
      if (m == -INFINITY) l = l == l ? 0.0f : l;           // a row that has seen no key
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
      QT* dst = reinterpret_cast<QT*>(a.out) + otok * a.o_tok + (long long)qh * a.o_head;
#pragma unroll
      for (int k = 0; k < D; k += 32) {
        uint32_t o[32];
        __syncwarp();
        tmem_ld32(tm_o + k, o);
        tmem_wait_ld();
        if (on && whole) {
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            uint4 v;
            v.x = Bits16<QT>::pack(__uint_as_float(o[e]) * inv, __uint_as_float(o[e + 1]) * inv);
            v.y = Bits16<QT>::pack(__uint_as_float(o[e + 2]) * inv, __uint_as_float(o[e + 3]) * inv);
            v.z = Bits16<QT>::pack(__uint_as_float(o[e + 4]) * inv, __uint_as_float(o[e + 5]) * inv);
            v.w = Bits16<QT>::pack(__uint_as_float(o[e + 6]) * inv, __uint_as_float(o[e + 7]) * inv);
            *reinterpret_cast<uint4*>(dst + k + e) = v;
          }
        } else if (on) {
          float* to = slot + 4 * kTileRows + (long long)srow * D + k;
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            *reinterpret_cast<uint4*>(to + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
        }
      }
      if (on) {
        if (!whole) {
          slot[srow] = m;
          slot[2 * kTileRows + srow] = l;
        } else if (a.lse) {
          a.lse[otok * (a.pool.H * a.G) + qh] = l == 0.0f ? -INFINITY : 0.69314718056f * (m + log2f(l));
        }
      }
      tmem_before();
    }
  } else if (warp < 12) {
    regs_down<S::kRegsOther>();
    if (warp == 8 || warp == 10) {
      // ============================================================== MMA warps, one per tile
      // Issuing an MMA and looking at a barrier take one warp 60 and more than 100 cycles each: while
      // one of the two looks, the other's MMAs run.
      const int t = warp == 10 ? 1 : 0;
      constexpr bool kHalf = std::is_same<MT, __half>::value;
      constexpr unsigned int kQK = mma_desc(kHalf, kTileKeys, false), kPV = mma_desc(kHalf, D, true);
      unsigned int buf = 0, buf_phase = 0;                 // next buffer of the ring to be read
      unsigned int q_phase = 0, p_phase = 0;
      unsigned int turn_phase = t == 0;                    // (the first turn is tile 0's: a fresh barrier passes for phase 1)
      unsigned int last_buf = 0, last_phase = 1;           // (a fresh barrier passes for phase 1)
      auto advance = [&]() {
        if (++buf == S::kBufs) {
          buf = 0;
          buf_phase ^= 1u;
        }
      };
      const unsigned int leader = lane == 0;
      auto uniform = [](unsigned int x) { return __shfl_sync(0xffffffffu, x, 0); };
      const unsigned int tmu = uniform(tmem);
      // low words of the operands' descriptors; the rest of them is constant
      const unsigned int q_low = uniform(operand_low(smem0, 16)), k_low = uniform(operand_low(kv0, 16));
      const unsigned int v_low = uniform(operand_low(kv0, S::kColBytes));
      auto qk = [&](unsigned int kbuf) {
        const unsigned int low = k_low + kbuf * (S::kBuf >> 4);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const unsigned int off = ((k >> 2) * S::kColBytes + (k & 3) * 32) >> 4;
          mma_smem(tmu + t * 128, operand_desc(q_low + t * (S::kQ >> 4) + off), operand_desc(low + off), kQK, k > 0,
                   leader);
        }
        mma_commit(smem_u32(&s_s_full[t]), leader);
      };
      while (walk.next_warp(a, per)) {
        const int steps = (int)uniform(walk.t1 - walk.t0);
        const bool turns = uniform(walk.rows(a) > kTileRows);     // two tiles at work
        const bool active = uniform(walk.rows(a) > t * kTileRows);   // the tile has rows; else only hands buffers on
        const int key_first = (int)uniform((walk.span.tile0 + walk.t0) * kTileKeys);
        const int lo = (int)uniform(walk.span.lo), hi = (int)uniform(walk.span.hi);
        ring_wait(smem_u32(&s_kv_full[buf]), buf_phase, abort_flag);
        if (active) {
          ring_wait(smem_u32(&s_q_full[t]), q_phase, abort_flag);
          __syncwarp();
          q_phase ^= 1u;
          tmem_after();
          qk(buf);
        }
        mma_commit(smem_u32(&s_kv_empty[buf]), leader);
        advance();
        for (int j = 0; j < steps; ++j) {
          const unsigned int vbuf = buf;
          last_buf = buf;
          last_phase = buf_phase;
          ring_wait(smem_u32(&s_kv_full[buf]), buf_phase, abort_flag);
          advance();
          if (!F8) {
            // V rows of positions nobody in the block sees: whatever the pool holds there
            // (0 * NaN is NaN) becomes zero; both warps see to it, each before its own MMAs
            const int key0 = key_first + j * kTileKeys;
            const int z0 = min(max(lo - key0, 0), kTileKeys), z1 = max(min(hi - key0, kTileKeys), 0);
            if (z0 > 0 || z1 < kTileKeys) {
              unsigned char* v = base + 2 * S::kQ + vbuf * S::kBuf;
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
          const bool more = j + 1 < steps;
          const unsigned int kbuf = buf;
          if (more) {
            ring_wait(smem_u32(&s_kv_full[buf]), buf_phase, abort_flag);
            advance();
          }
          const unsigned int low = v_low + vbuf * (S::kBuf >> 4), old = F8 || j > 0;
          if (active) {
            ring_wait(smem_u32(&s_h_full[t]), p_phase, abort_flag);
            if (turns) {
              ring_wait(smem_u32(&s_turn[t]), turn_phase, abort_flag);
              turn_phase ^= 1u;
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              if (half) ring_wait(smem_u32(&s_p_full[t]), p_phase, abort_flag);
              __syncwarp();
              tmem_after();
#pragma unroll
              for (int k = half * 4; k < half * 4 + 4; ++k)
                mma_tmem(tmu + 256 + t * D, tmu + t * 128 + k * 8, operand_desc(low + k * (2048 >> 4)), kPV,
                         k > 0 ? 1u : old, leader);
            }
            p_phase ^= 1u;
            if (more)
              qk(kbuf);
            else
              mma_commit(smem_u32(&s_o_full[t]), leader);
            if (turns && lane == 0) mbar_arrive(smem_u32(&s_turn[1 - t]));
            __syncwarp();
          }
          mma_commit(smem_u32(&s_kv_empty[vbuf]), leader);
          if (more) mma_commit(smem_u32(&s_kv_empty[kbuf]), leader);
        }
      }
      // the last commit has to arrive while its barrier is still this CTA's
      ring_wait(smem_u32(&s_kv_empty[last_buf]), last_phase, abort_flag);
    } else if (warp == 9) {
      // ============================================================== loader warp
      constexpr unsigned int kBytes = F8 ? S::kRaw : S::kBuf;
      constexpr int kRow = F8 ? D : 128;
      const unsigned int ring0 = F8 ? kv0 + S::kColBytes : kv0;
      unsigned long long* full = F8 ? s_raw_full : s_kv_full;
      const int boxes = kTileKeys >> a.box_log;
      unsigned int buf = 0, phase = 1, issued = 0, step = 0;
      while (walk.next_warp(a, per)) {
        const uint32_t* row;
        long long entries;
        table_row(a.b, walk.r, row, entries);
        if (walk.q.keys < walk.q.len && walk.head == 0 && walk.block == 0 && walk.t0 == 0 && lane == 0)
          raise_status(AIBX_ERR_RANGE);                    // tokens the table has no entry for
        BoxIds<kTileKeys> ids(a, row, walk.span.tile0 + walk.t0, walk.span.tile0 + walk.t1, walk.span.lo,
                              walk.span.hi);
        const int head = walk.head, tile0 = walk.span.tile0, lo = walk.span.lo, hi = walk.span.hi, t1 = walk.t1;
        for (int j = walk.t0; j < t1; ++j, ++step) {
          uint32_t id;
          const bool valid = ids.give(id, head == 0);
          const int slot = ids.slot;
          ids.step_slot();
          // a box that is not there, or that holds no visible key, comes as zeros from beyond the pool
          const int block = valid ? (int)id : (int)a.pool.num_blocks;
          const int tok = (tile0 + j) * kTileKeys + (lane & (boxes - 1)) * a.box;
          const bool missing = lane < boxes && tok < hi && tok > lo - a.box && !valid;
          const unsigned int gone = __ballot_sync(0xffffffffu, missing);
          if (lane == 0) s_mask[step % kInfoRing] = ~gone;
          for (int kv = 0; kv < 2; ++kv) {
            ring_wait(smem_u32(&s_kv_empty[buf]), phase, abort_flag);
            __syncwarp();
            const unsigned int bar = smem_u32(&full[buf]);
            if (__any_sync(0xffffffffu, *abort_flag)) {
              if (lane == 0) mbar_arrive(bar);
            } else {
              if (lane == 0) mbar_arrive_expect_tx(bar, kBytes);
              __syncwarp();
              if (lane < boxes) {
                const unsigned int dst = ring0 + buf * S::kBuf + lane * a.box * kRow;
#pragma unroll
                for (int cc = 0; cc < (F8 ? 1 : S::kCols); ++cc)
                  tensor_load_5d(dst + cc * S::kColBytes, &map, bar, cc * 64, slot, head, block, kv);
              }
            }
            __syncwarp();
            ++issued;
            if (++buf == S::kBufs) {
              buf = 0;
              phase ^= 1u;
            }
          }
        }
      }
      // nothing may still be on its way into this CTA's shared memory when it ends
      for (unsigned int i = issued > S::kBufs ? issued - S::kBufs : 0; i < issued; ++i)
        ring_drain(smem_u32(&full[i % S::kBufs]), (i / S::kBufs) & 1u);
    } else if (F8 && warp == 11) {
      // ============================================================== scale warp (11)
      // Per step: the factor 2^(e - E) of every position of the K and of the V tile, and E.  The
      // chain table -> scale byte is long: it runs ahead.
      unsigned int step = 0;
      while (walk.next_warp(a, per)) {
        int most = 0;                                      // largest V byte of the segment so far
        const uint32_t* row;
        long long entries;
        table_row(a.b, walk.r, row, entries);
        const int head = walk.head, tile0 = walk.span.tile0, lo = walk.span.lo, hi = walk.span.hi, t1 = walk.t1;
        for (int j = walk.t0; j < t1; ++j, ++step) {
          const int tok = (tile0 + j) * kTileKeys + lane * 4;   // four slots of one block
          int byte[2][4];
          unsigned int there = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            byte[0][i] = byte[1][i] = 0;
            if (tok + i >= lo && tok + i < hi) there |= 1u << i;
          }
          if (there) {
            const int at = tok / a.pool.T;
            const uint32_t id = __ldg(row + at);
            if (id < a.pool.num_blocks) {
              const unsigned char* src = a.pool.scales + (long long)id * a.pool.s_block +
                                         (long long)head * a.pool.s_head +
                                         (long long)(tok - at * a.pool.T) * a.pool.s_slot;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                byte[0][i] = __ldg(src + i * a.pool.s_slot);
                byte[1][i] = __ldg(src + a.pool.s_kv + i * a.pool.s_slot);
              }
            } else {
              there = 0;
            }
          }
          const unsigned int f = step % S::kFactorRing;
          ring_wait(smem_u32(&s_fac_empty[f]), ((step / S::kFactorRing) & 1u) ^ 1u, abort_flag);
          __syncwarp();
          // Bytes at most 14 (K, in the tile) or 4 (V, in the segment so far) below the largest: every
          // factor is a power of two that bits make.
          int top[2];
          bool far = false;
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            top[kv] = 27;                                  // exponents from -100: 2^-E stays finite
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (((there >> i) & 1u) && byte[kv][i] != 255) top[kv] = max(top[kv], byte[kv][i]);
            top[kv] = __reduce_max_sync(0xffffffffu, top[kv]);
          }
          most = max(most, top[1]);
          const int low[2] = {top[0] - kKeySpread, max(most - kScaleSpread, kScaleLow)};
#pragma unroll
          for (int i = 0; i < 4; ++i)
            far |= ((there >> i) & 1u) && (byte[0][i] < low[0] || byte[1][i] < low[1] || byte[1][i] > kScaleHigh);
          // (K's largest too: the scale of the scores has to stay finite)
          const bool wide = __any_sync(0xffffffffu, far) || most > kScaleHigh || top[0] > kScaleHigh;
          uint32_t out[2][4];                              // 16 bits each
          if (!wide) {
#pragma unroll
            for (int kv = 0; kv < 2; ++kv)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                out[kv][i] = byte[kv][i] == 255 ? 0x7e00u : 0x3c00u - 1024u * (uint32_t)(top[kv] - byte[kv][i]);
                if (!((there >> i) & 1u)) out[kv][i] = 0;
              }
          } else {                                         // K's rows as they are, V as bf16
            uint32_t packed = 0x7f7f7f7fu;
            top[1] = weight_byte(top[1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const bool on = (there >> i) & 1u;
              out[0][i] = !on ? 0 : byte[0][i] == 255 ? 0x7e00u : 0x3c00u;
              out[1][i] = !on ? 0 : byte[1][i] == 255 ? 0x7fc0u : (uint32_t)max(127 + byte[1][i] - top[1], 0) << 7;
              if (out[0][i] == 0x3c00u) packed ^= (uint32_t)(byte[0][i] ^ 0x7f) << (8 * i);
            }
            *reinterpret_cast<uint32_t*>(&s_kbytes[step % kInfoRing][lane * 4]) = packed;
            if (lane == 0) s_wide_vexp[step % kInfoRing] = (float)(top[1] - 127);
          }
#pragma unroll
          for (int kv = 0; kv < 2; ++kv)
            *reinterpret_cast<uint2*>(factors + (f * 2 + kv) * kTileKeys + lane * 4) =
                make_uint2(out[kv][0] | out[kv][1] << 16, out[kv][2] | out[kv][3] << 16);
          if (lane == 0) {
            s_kscale[step % kInfoRing] = wide ? 1.0f : power_of_byte(top[0]);
            s_vexp[step % kInfoRing] = wide ? -INFINITY : (float)(top[1] - 127);
            s_wide[step % kInfoRing] = wide;
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&s_fac_full[f]));
        }
      }
    }
  } else if constexpr (F8) {
    // ================================================================ converter warps (12 .. 15)
    regs_down<S::kRegsOther>();
    // A thread takes one 16-byte piece of kRows neighbouring rows, half of them at a time; a row's
    // pieces are one warp's, which has read them all before it writes over them.
    const int tid = threadIdx.x - 384;
    constexpr int kChunks = D / 16;                        // 16-byte pieces of a raw row
    constexpr int kRows = kTileKeys * kChunks / 128;
    const int c = tid % kChunks, i0 = tid / kChunks * kRows;
    unsigned int buf = 0, phase = 0, step = 0;
    while (walk.next_warp(a, per)) {
      const int steps = walk.t1 - walk.t0;
      for (int j = 0; j < steps; ++j, ++step) {
        const unsigned int f = step % S::kFactorRing;
        ring_wait(smem_u32(&s_fac_full[f]), (step / S::kFactorRing) & 1u, abort_flag);
        for (int kv = 0; kv < 2; ++kv) {
          __half x[kRows];
          const __half* fac = factors + (f * 2 + kv) * kTileKeys + i0;
          if constexpr (kRows == 8)
            *reinterpret_cast<uint4*>(x) = *reinterpret_cast<const uint4*>(fac);
          else
            *reinterpret_cast<uint2*>(x) = *reinterpret_cast<const uint2*>(fac);
          const bool wide = kv == 1 && s_wide[step % kInfoRing];
          bool gone = false;                               // rows that are not there, or too small to show
#pragma unroll
          for (int u = 0; u < kRows; ++u) gone |= __half_as_ushort(x[u]) == 0;
          ring_wait(smem_u32(&s_raw_full[buf]), phase, abort_flag);
          __syncwarp();
          unsigned char* out = base + 2 * S::kQ + buf * S::kBuf + (c >> 2) * S::kColBytes;
          const unsigned char* src = base + 2 * S::kQ + buf * S::kBuf + S::kColBytes;
          constexpr int kTurn = kRows / 2;
          auto convert = [&](auto to_bf16) {
#pragma unroll
            for (int u0 = 0; u0 < kRows; u0 += kTurn) {
              uint4 v[kTurn];
#pragma unroll
              for (int u = 0; u < kTurn; ++u) {
                const int i = i0 + u0 + u;
                v[u] = *reinterpret_cast<const uint4*>(src + i * D + ((D == 128 ? c ^ (i & 7) : c) << 4));
              }
              if (gone) {
#pragma unroll
                for (int u = 0; u < kTurn; ++u)
                  if (__half_as_ushort(x[u0 + u]) == 0) v[u] = make_uint4(0, 0, 0, 0);
              }
              __syncwarp();
#pragma unroll
              for (int u = 0; u < kTurn; ++u) {
                const int i = i0 + u0 + u;
                const uint32_t wv[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
                uint32_t o[8];
                if constexpr (decltype(to_bf16)::value) {    // the factor is one already
                  const float xf = __uint_as_float((uint32_t)__half_as_ushort(x[u0 + u]) << 16);
#pragma unroll
                  for (int e = 0; e < 8; ++e) o[e] = bf16_of_e4m3((wv[e >> 1] >> (16 * (e & 1))) & 0xffffu, xf);
                } else {
                  const __half2 x2 = __half2half2(x[u0 + u]);
#pragma unroll
                  for (int e = 0; e < 4; ++e) {
                    const __half2 lo = __hmul2(halves_of_e4m3(wv[e] & 0xffffu), x2);
                    const __half2 hi = __hmul2(halves_of_e4m3(wv[e] >> 16), x2);
                    o[2 * e] = *reinterpret_cast<const uint32_t*>(&lo);
                    o[2 * e + 1] = *reinterpret_cast<const uint32_t*>(&hi);
                  }
                }
                const int p0 = (2 * c) & 7;
                *reinterpret_cast<uint4*>(out + i * 128 + ((p0 ^ (i & 7)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
                *reinterpret_cast<uint4*>(out + i * 128 + (((p0 + 1) ^ (i & 7)) << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
              }
            }
          };
          if (wide)
            convert(std::true_type());
          else
            convert(std::false_type());
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          mbar_arrive(smem_u32(&s_kv_full[buf]));
          if (++buf == S::kBufs) {
            buf = 0;
            phase ^= 1u;
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_fac_empty[f]));
      }
    }
  }
  tmem_before();
  __syncthreads();
  if (warp == 8) {
    tmem_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
  if constexpr (TREE) asm volatile("griddepcontrol.wait;" ::: "memory");   // (the kernel before, if there is one)
}

// `behind`: a kernel of the same call runs before this one, in the same stream and on its own requests.  Its
// SMs then go on to this kernel one by one, as they come free (32 drafts of both kinds: 215 -> 206 us); at its end this kernel waits for that one, so that the join, which waits for this one alone, finds
// what both have left.
template <int D, bool F8, typename QT, bool TREE>
inline int32_t launch_attn_tiles(AttnArgs a, int type, JoinSet& join, bool behind, cudaStream_t st) {
  using S = TileShape<D, F8>;
  a.box = gcd_int(a.pool.T, kTileKeys);
  a.box_log = log2_int(a.box);
  CUtensorMap map;
  const int32_t rc = pool_tensor_map(a.pool, type, a.box, &map);
  if (rc != AIBX_OK) return rc;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return AIBX_ERR_CUDA;
  static size_t configured[64] = {0};
  static std::mutex lock;
  if (!ensure_dynamic_smem(attn_tiles_kernel<D, F8, QT, TREE>, S::kSmem, dev, configured, lock))
    return AIBX_ERR_CUDA;
  const unsigned int grid = (unsigned int)sm_count();
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(S::kThreads);
  cfg.dynamicSmemBytes = S::kSmem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = behind ? 1 : 0;
  cudaLaunchKernelEx(&cfg, attn_tiles_kernel<D, F8, QT, TREE>, map, a);
  join = JoinSet{a.slots, reinterpret_cast<const JoinRecord*>(a.slots + 2ull * grid * S::kSlot), 2 * kTileRows};
  return launch_status();
}

}  // namespace aibx
