// Attention of few query rows (new tokens * query heads per KV head <= 16) over a paged cache: a
// decoding step, or a few speculative tokens.
//
// Mathematics, per (request, KV head) with query rows i and keys j, in powers of two:
//   t_ij = scale * log2(e) * q_i . k_j,  m = running max, l = sum 2^(t - m), O = sum 2^(t - m) v_j,
//   out = O / l, lse = ln 2 * (m + log2 l).
// Over an e4m3 pool k_j = K_j 2^a_j and v_j = V_j 2^b_j with e4m3 rows K_j, V_j.  Those are exact
// in fp16, so they go to the tensor core as they are: the scores take 2^a_j afterwards, and the
// weight that multiplies V_j is w = 2^(t + b_j - m) with m the maximum of t + b_j; then
// l = sum w 2^-b_j (stages whose b_j are far apart: see kScaleSpread).  Queries are scaled to [1, 2)
// per row to fit fp16 (fp16 keeps 3 more bits than bf16; what falls below 2^-24 of the row's maximum
// is lost).
//
// Bound: HBM.  Every K and V byte is read once and meets at most 16 rows, so the legacy tensor
// path (mma.sync m16n8k16) has an order of magnitude to spare: 16 tokens of D = 128 cost 32 MMAs
// against 341 cycles of this SM's share of the bandwidth (16-bit rows).  What counts is bytes in
// flight: one warp feeds a ring of five 32 KB stages with tensor-map boxes (one box = the slots
// of one block and head), 160 KB per SM outstanding, and runs ahead over the seams between
// requests, so that the memory never idles (64 single tokens over 292,000 cached ones of 8 heads,
// bf16: 194 us, 6.2 TB/s; 32 over 131,072 each of 4 heads, e4m3: 816 us, 5.3 TB/s, with all stages'
// scales far apart a third more); eight warps consume, 16 tokens each at a time, with their own m, l
// and O, joined once per (request, head).
// The keys are the MMA's M dimension and the query rows its N of 8: S^T = K Q^T and O^T = V^T P^T,
// so that 8 rows (7 or 8 query heads of one token) waste nothing.  Fragments are read from shared
// memory without transposition: the order of the contraction index is free as long as both
// operands agree.  For K Q^T a lane's 16-byte piece of a K row serves as the k-indices of two MMAs;
// for V^T P^T a lane reads the same 16-byte column piece of its four tokens and pairs tokens with
// byte permutes; P^T goes from accumulator to operand layout with movmatrix.
#pragma once

#include "attn_common.cuh"

namespace aibx {

constexpr int kRowStages = 5;
constexpr int kRowHalfStage = 16384;                       // bytes of K (and of V) per stage
constexpr int kScaleWarps = 3;

template <int D, bool F8, int ROWS>
struct RowShape {
  static constexpr int kWarps = 8;                           // consumers (16 of them, at 96 registers
                                                             // each: 297 us against 215)
  static constexpr int kNQ = ROWS / 8;                       // MMAs across the rows
  static constexpr int kElem = F8 ? 1 : 2;
  static constexpr int kTok = kRowHalfStage / (D * kElem);   // tokens per stage
  static constexpr int kRowBytes = F8 ? D : 128;             // bytes of a shared-memory row
  static constexpr int kCols = F8 ? 1 : D / 64;              // 128-byte columns of a 16-bit row
  static constexpr int kTasks = kTok / 16;
  static constexpr int kThreads = 32 * (kWarps + 1 + (F8 ? kScaleWarps : 0));
  static constexpr int kSmem = kRowStages * 2 * kRowHalfStage + kWarps / 2 * ROWS * D * 4 +
                               (F8 ? kRowStages * 2 * kTok : 0) + 1024;
  static constexpr int kSlot = ROWS * (D + 2);               // floats per workspace slot
};

__device__ __forceinline__ void mma_16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1,
                                          __nv_bfloat16) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1,
                                          __half) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Transposes an 8x8 matrix of 16-bit numbers held as an MMA fragment.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

__device__ __forceinline__ uint32_t e4m3_bits(uint32_t pair) {
  const __half2 h = halves_of_e4m3(pair);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Two e4m3 numbers times a power of two, as bf16: exact.
__device__ __forceinline__ uint32_t bf16_of_e4m3(uint32_t pair, float f) {
  const float2 y = __half22float2(halves_of_e4m3(pair));
  return Bits16<__nv_bfloat16>::pack(y.x * f, y.y * f);
}

// The tiles of request r: first tile and how many (at least one, so that empty rows are written).
struct RowSpan {
  int tile0, tiles, lo, hi;
};

template <int TOK>
__device__ __forceinline__ RowSpan row_span(const AttnArgs& a, const AttnRequest& q) {
  RowSpan s;
  s.hi = q.keys;
  const long long lo = a.window > 0 ? (long long)q.len - q.n - a.window + 1 : 0;
  s.lo = lo < 0 ? 0 : lo > s.hi ? s.hi : (int)lo;
  s.tile0 = s.lo / TOK;
  s.tiles = max(1, (int)(((unsigned int)s.hi + TOK - 1) / TOK) - s.tile0);   // (hi may be 2^31 - 1)
  return s;
}

template <int TOK>
struct RowCost {
  const AttnArgs& a;
  __device__ __forceinline__ long long operator()(int r, bool on) const {
    if (!on) return 0;
    const AttnRequest q = attn_request(a.b, a.pool.T, r);
    if (q.n == 0 || (long long)q.n * a.G > a.row_limit) return 0;
    return (long long)row_span<TOK>(a, q).tiles * a.pool.H;
  }
};

// Walks a CTA's piece of the line, one (request, head) segment at a time.
template <int TOK>
struct RowWalk {
  const AttnArgs& a;
  long long pos, end, base;     // next position, end of the piece, first position of request r
  int r;
  AttnRequest q;
  RowSpan span;
  int head, t0, t1;             // the segment: tiles [t0, t1) of the request, counted from tile0

  __device__ __forceinline__ RowWalk(const AttnArgs& args, const WorkStart& w, unsigned int index,
                                     unsigned int pieces)
      : a(args) {
    const long long per = (w.total + pieces - 1) / pieces;
    pos = per * index;
    end = min(pos + per, w.total);
    base = w.base;
    r = w.r;
    if (r < 0) pos = end = 0;
    if (pos < end) load();
  }
  __device__ __forceinline__ void load() {
    q = attn_request(a.b, a.pool.T, r);
    span = row_span<TOK>(a, q);
  }
  __device__ __forceinline__ bool next() {
    if (pos >= end) return false;
    long long off = pos - base;
    while (off >= (long long)span.tiles * a.pool.H) {      // on to the next request with work
      base += (long long)span.tiles * a.pool.H;
      do {
        ++r;
        q = attn_request(a.b, a.pool.T, r);
      } while (q.n == 0 || (long long)q.n * a.G > a.row_limit);
      span = row_span<TOK>(a, q);
      off = pos - base;
    }
    head = (int)(off / span.tiles);
    t0 = (int)(off - (long long)head * span.tiles);
    const long long left = end - pos;
    t1 = left < span.tiles - t0 ? t0 + (int)left : span.tiles;
    pos += t1 - t0;
    return true;
  }
  __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == span.tiles; }
};

// Block ids of the boxes of a segment's tiles, in order.  A lane fetches the id of one box, 32
// boxes at a time, and the next 32 are under way while these are used: the loader never waits for
// the table (looking at an id as soon as it was asked for cost the latency of the load per tile:
// 302 instead of 285 us for 64 single tokens over 292,000 cached ones).
template <int TOK>
struct BoxIds {
  const AttnArgs& a;
  const uint32_t* row;
  int lane, boxes, per;          // boxes per tile (a power of two), tiles per 32 boxes
  int tile, end, lo, hi;         // next tile to be asked for
  uint32_t id, id_next;
  int used;                      // tiles of the current 32 boxes already given out
  int slot, slot_step;           // this lane's first slot in the next tile, and its way per tile

  __device__ __forceinline__ BoxIds(const AttnArgs& args, const uint32_t* table, int tile0, int tile1,
                                    int lo_, int hi_)
      : a(args), row(table), lane(threadIdx.x & 31), boxes(TOK >> args.box_log), per(32 / boxes), tile(tile0),
        end(tile1), lo(lo_), hi(hi_), id(0), used(0) {
    id_next = ask();
    used = per;
    slot = (int)(((long long)tile0 * TOK + lane * a.box) % a.pool.T);
    slot_step = TOK % a.pool.T;
  }
  __device__ __forceinline__ void step_slot() {
    slot += slot_step;
    if (slot >= a.pool.T) slot -= a.pool.T;
  }
  __device__ __forceinline__ uint32_t ask() {
    const int t = tile + lane / boxes;
    const long long tok = (long long)t * TOK + (lane & (boxes - 1)) * a.box;
    tile += per;
    return t < end && tok < hi && tok + a.box > lo ? __ldg(row + (int)tok / a.pool.T) : AIBX_NO_BLOCK;
  }
  // The next tile's box of this lane (lanes below `boxes`): its block, and whether it is there.
  __device__ __forceinline__ bool give(uint32_t& block, bool tell) {
    if (used == per) {
      id = id_next;
      id_next = ask();
      used = 0;
    }
    block = __shfl_sync(0xffffffffu, id, (used * boxes + lane) & 31);
    ++used;
    if (lane >= boxes || block == AIBX_NO_BLOCK) return false;
    if (block >= a.pool.num_blocks) {
      if (tell) raise_status(AIBX_ERR_RANGE);
      return false;
    }
    return true;
  }
};

template <int D, bool F8, typename QT, int ROWS, bool TREE>
__global__ void __launch_bounds__(RowShape<D, F8, ROWS>::kThreads, 1)
attn_rows_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                 const __grid_constant__ AttnArgs a) {
  using S = RowShape<D, F8, ROWS>;
  using MT = typename std::conditional<F8, __half, QT>::type;   // operand type of the MMAs
  constexpr int TOK = S::kTok, RB = S::kRowBytes, kRowWarps = S::kWarps;
  extern __shared__ unsigned char s_raw[];
  __shared__ __align__(8) unsigned long long s_full[kRowStages], s_empty[kRowStages];
  __shared__ unsigned int s_mask[kRowStages];
  __shared__ uint32_t s_facts[kRowStages];                  // of the stage's V bytes
  __shared__ float s_m[2][kRowWarps][ROWS], s_l[2][kRowWarps][ROWS];
  __shared__ long long s_scan[33];
  __shared__ WorkStart s_start;
  __shared__ int s_abort;

  const unsigned int smem0 = (smem_u32(s_raw) + 1023u) & ~1023u;
  unsigned char* ring = s_raw + (smem0 - smem_u32(s_raw));
  float* merge = reinterpret_cast<float*>(ring + kRowStages * 2 * kRowHalfStage);
  unsigned char* s_scale = reinterpret_cast<unsigned char*>(merge + kRowWarps / 2 * ROWS * D);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kRowStages; ++s) {
      mbar_init(smem_u32(&s_full[s]), F8 ? 2u : 1u);
      mbar_init(smem_u32(&s_empty[s]), (unsigned int)kRowWarps);
    }
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  const RowCost<TOK> cost{a};
  locate_piece<S::kThreads>(a.b.R, blockIdx.x, gridDim.x, s_scan, &s_start, cost);
  const WorkStart w = s_start;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  RowWalk<TOK> walk(a, w, blockIdx.x, gridDim.x);
  volatile int* abort_flag = &s_abort;

  if (threadIdx.x == 0) {
    RowWalk<TOK> look = walk;
    JoinRecord rec = {};
    if (look.next() && look.t0 > 0 && look.t1 == look.span.tiles) {
      const long long per = (w.total + gridDim.x - 1) / gridDim.x;
      const long long p0 = look.pos - look.t1;             // position of the rows' first tile
      rec.tok0 = look.q.tok0;
      rec.rows = look.q.n * a.G;
      rec.head = look.head;
      rec.first_cta = (int)(p0 / per);
      rec.first_slot = p0 != rec.first_cta * per;
    }
    reinterpret_cast<JoinRecord*>(a.slots + 2ull * gridDim.x * S::kSlot)[blockIdx.x] = rec;
  }

  if (warp == kRowWarps) {
    // ---------------------------------------------------------------- loader warp
    // Its instructions per tile are what a tile takes at least: counters instead of divisions.
    unsigned int issued = 0, s = 0, phase = 1;               // (a fresh barrier passes for phase 1)
    const unsigned int box_bytes = (unsigned int)a.box * D * S::kElem;
    while (walk.next()) {
      const uint32_t* row;
      long long entries;
      table_row(a.b, walk.r, row, entries);
      if (walk.q.keys < walk.q.len && walk.head == 0 && walk.t0 == 0 && lane == 0)
        raise_status(AIBX_ERR_RANGE);                      // tokens the table has no entry for
      BoxIds<TOK> ids(a, row, walk.span.tile0 + walk.t0, walk.span.tile0 + walk.t1, walk.span.lo, walk.span.hi);
      for (int t = walk.t0; t < walk.t1; ++t, ++issued) {
        uint32_t id;
        bool valid = ids.give(id, walk.head == 0);
        const unsigned int bar = smem_u32(&s_full[s]);
        if (!ring_wait(smem_u32(&s_empty[s]), phase, abort_flag)) valid = false;
        const unsigned int mask = __ballot_sync(0xffffffffu, valid);
        if (lane == 0) {
          s_mask[s] = mask;
          if (mask)
            mbar_arrive_expect_tx(bar, (unsigned int)__popc(mask) * 2u * box_bytes);
          else
            mbar_arrive(bar);
        }
        __syncwarp();
        if (valid) {
          const unsigned int dst = smem0 + s * 2 * kRowHalfStage + lane * box_bytes;
          tensor_load_5d(dst, &map_k, bar, 0, ids.slot, 0, walk.head, (int)id);
          tensor_load_5d(dst + kRowHalfStage, &map_v, bar, 0, ids.slot, 0, walk.head, (int)id);
        }
        ids.step_slot();
        if (++s == kRowStages) {
          s = 0;
          phase ^= 1u;
        }
      }
    }
    // what is still in flight targets this CTA's shared memory: wait for it before leaving
    for (unsigned int i = issued > kRowStages ? issued - kRowStages : 0; i < issued; ++i)
      ring_drain(smem_u32(&s_full[i % kRowStages]), (i / kRowStages) & 1u);
    return;
  }
  if (F8 && warp > kRowWarps) {
    // ---------------------------------------------------------------- scale warps
    // Warp k fetches the scale bytes of every third tile: the chain table -> byte is long, three
    // warps keep three of them under way.
    const int k = warp - kRowWarps - 1;
    constexpr int kPer = TOK / 32;
    unsigned int it = 0;
    while (walk.next()) {
      const uint32_t* row;
      long long entries;
      table_row(a.b, walk.r, row, entries);
      for (int t = walk.t0; t < walk.t1; ++t, ++it) {
        if (it % kScaleWarps != (unsigned int)k) continue;
        uint32_t kb = 0x7f7f7f7fu, vb = 0x7f7f7f7fu, kb2 = kb, vb2 = vb;
        const int tok = (walk.span.tile0 + t) * TOK + lane * kPer;     // kPer slots of one block
        bool there = false;
        if (tok < walk.span.hi) {
          const int at = tok / a.pool.T;
          const uint32_t id = __ldg(row + at);
          there = id < a.pool.num_blocks;
          if (there) {
            const unsigned char* p = a.pool.scales + (long long)id * a.pool.s_block +
                                     (long long)walk.head * a.pool.s_head +
                                     (long long)(tok - at * a.pool.T) * a.pool.s_slot;
            kb = vb = kb2 = vb2 = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              kb |= (uint32_t)__ldg(p + i * a.pool.s_slot) << (8 * i);
              vb |= (uint32_t)__ldg(p + a.pool.s_kv + i * a.pool.s_slot) << (8 * i);
            }
            if (kPer == 8) {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                kb2 |= (uint32_t)__ldg(p + (i + 4) * a.pool.s_slot) << (8 * i);
                vb2 |= (uint32_t)__ldg(p + a.pool.s_kv + (i + 4) * a.pool.s_slot) << (8 * i);
              }
            }
          }
        }
        // least and largest V byte of the positions that a row may see
        uint32_t least = 0xffffffffu, most = 0u;
#pragma unroll
        for (int w = 0; w < kPer / 4; ++w) {
          const int t0w = tok + 4 * w;
          const int n0 = min(max(walk.span.lo - t0w, 0), 4), n1 = there ? min(max(walk.span.hi - t0w, 0), 4) : 0;
          const uint32_t in = (uint32_t)((1ull << (8 * n1)) - 1) & ~(uint32_t)((1ull << (8 * n0)) - 1);
          const uint32_t b4 = w ? vb2 : vb;
          least = __vminu4(least, (b4 & ~__vcmpgtu4(b4, kScaleHigh * 0x01010101u)) | ~in);
          most = __vmaxu4(most, b4 & in & ~__vcmpeq4(b4, 0xffffffffu));
        }
        least = __vminu4(least, least >> 16 | 0xffff0000u);
        most = __vmaxu4(most, most >> 16);
        least = min(least & 255u, (least >> 8) & 255u);
        least = __reduce_min_sync(0xffffffffu, least < kScaleLow ? 0u : least + 16u);
        most = __reduce_max_sync(0xffffffffu, max(most & 255u, (most >> 8) & 255u));
        const int s = (int)(it % kRowStages);
        if (it >= kRowStages) ring_wait(smem_u32(&s_empty[s]), (it / kRowStages - 1) & 1u, abort_flag);
        if (lane == 0) s_facts[s] = scale_facts(least, most);
        uint32_t* dst = reinterpret_cast<uint32_t*>(s_scale + s * 2 * TOK);
        if (kPer == 8) {
          dst[2 * lane] = kb;
          dst[2 * lane + 1] = kb2;
          dst[TOK / 4 + 2 * lane] = vb;
          dst[TOK / 4 + 2 * lane + 1] = vb2;
        } else {
          dst[lane] = kb;
          dst[TOK / 4 + lane] = vb;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_full[s]));
      }
    }
    return;
  }

  // ------------------------------------------------------------------ consumer warps
  const int g = lane >> 2, t4 = lane & 3;
  constexpr int NQ = S::kNQ;
  constexpr int kMT = D / 16;                              // 16-dim tiles of O^T
  constexpr int kPiece = F8 ? 16 : 8;                      // elements of a lane's piece of a K row
  constexpr int kPieces = D / (4 * kPiece);
  constexpr int kSteps = kPiece / 4;                       // MMAs per piece
  // a box lies column by column, `box` rows of RB bytes each; 16 tokens are two runs of 8 rows
  const int boxes = TOK >> a.box_log;
  const int col_stride = a.box * RB;
  const int run_stride = a.box >= 16 ? 8 * RB : col_stride * S::kCols;
  int stage = 0, seg = 0;
  unsigned int phase = 0;
  int turn = warp;                                         // first task of the next stage that is this warp's
  const unsigned int all_boxes = boxes == 32 ? 0xffffffffu : (1u << boxes) - 1u;
  while (walk.next()) {
    const int n_rows = walk.q.n * a.G;
    const int first = walk.q.len - walk.q.n;
    // ---- queries: row x * 8 + g as the operand's column g; their scale for columns 2 t4, 2 t4 + 1
    uint32_t qf[NQ][kPieces][kSteps][2];
    float qscale[NQ][2];
    int prow[NQ][2];
    uint32_t tree[NQ][2];                                  // trees: the request's nodes that a row sees (at most 16)
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
      const int i = x * 8 + g;
      const int ti = a.by_g.div(min(i, n_rows - 1));
      const QT* src = reinterpret_cast<const QT*>(a.q) + (walk.q.tok0 + ti) * a.q_tok +
                      (long long)(walk.head * a.G + (i - ti * a.G)) * a.q_head;
      uint32_t raw[kPieces][kPiece / 2];
#pragma unroll
      for (int p = 0; p < kPieces; ++p)
#pragma unroll
        for (int e = 0; e < kPiece / 8; ++e) {
          uint4 v = make_uint4(0, 0, 0, 0);
          if (i < n_rows) v = *reinterpret_cast<const uint4*>(src + p * 4 * kPiece + t4 * kPiece + e * 8);
          raw[p][4 * e] = v.x;
          raw[p][4 * e + 1] = v.y;
          raw[p][4 * e + 2] = v.z;
          raw[p][4 * e + 3] = v.w;
        }
      float down = 1.0f, up = 1.0f;
      if constexpr (F8) {
        float amax = 0.0f;
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
#pragma unroll
          for (int e = 0; e < kPiece / 2; ++e) {
            const float2 f = Bits16<QT>::unpack(raw[p][e]);
            amax = fmaxf(amax, fmaxf(fabsf(f.x), fabsf(f.y)));
          }
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
        power_scale(amax, down, up);
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
#pragma unroll
          for (int e = 0; e < kPiece / 2; ++e) {
            const float2 f = Bits16<QT>::unpack(raw[p][e]);
            raw[p][e] = Bits16<MT>::pack(f.x * down, f.y * down);
          }
      }
#pragma unroll
      for (int p = 0; p < kPieces; ++p)
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          qf[x][p][s][0] = raw[p][2 * s];
          qf[x][p][s][1] = raw[p][2 * s + 1];
        }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        qscale[x][h] = __shfl_sync(0xffffffffu, up, (2 * t4 + h) * 4) * a.scale_log2;
        const int ti = a.by_g.div(min(x * 8 + 2 * t4 + h, n_rows - 1));
        prow[x][h] = first + ti;
        if constexpr (TREE) {
          tree[x][h] = tree_bits(a.mask + (walk.q.tok0 + ti) * a.mask_words, a.mask_words, walk.q.n, 0);
          prow[x][h] = first + max(__popc(tree[x][h]) - 1, 0);
        }
      }
    }
    int most = 0;                                          // largest V byte of the segment so far
    float m[NQ][2], l[NQ][2], o[NQ][kMT][4];
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
      m[x][0] = m[x][1] = -INFINITY;
      l[x][0] = l[x][1] = 0.0f;
#pragma unroll
      for (int j = 0; j < kMT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[x][j][e] = 0.0f;
    }

    // the rows' positions run from `first` to len - 1: keys from open_lo to open_hi - 1 all see
    const int open_hi = TREE ? min(walk.span.hi, first) : a.causal ? min(walk.span.hi, first + 1) : walk.span.hi;
    const int open_lo = max(walk.span.lo, a.window > 0 ? walk.q.len - a.window : 0);
    for (int t = walk.t0; t < walk.t1; ++t) {
      // Every warp waits for every stage and hands every stage back, its own or not: a phase bit
      // tells a stage from the next one in its place only to a warp that misses none.
      const int s = stage;
      ring_wait(smem_u32(&s_full[s]), phase, abort_flag);
      if (++stage == kRowStages) {
        stage = 0;
        phase ^= 1u;
      }
      __syncwarp();
      const unsigned int boxmask = s_mask[s];
      const bool wide = F8 && scales_wide(s_facts[s], most);
      const int tile_key0 = (walk.span.tile0 + t) * TOK;
      // the 16-token tasks of all stages go round the warps in turn
      for (int task = turn; task < S::kTasks; task += kRowWarps) {
        const int key0 = tile_key0 + task * 16;
        const int b0 = (task * 16) >> a.box_log;
        // all 16 keys there, and seen by all rows
        const bool open = boxmask == all_boxes && key0 >= open_lo && key0 <= open_hi - 16;
        if (!open) {
          const int b1 = (task * 16 + 15) >> a.box_log;
          const unsigned int want = ((2u << (b1 - b0)) - 1u) << b0;
          if ((boxmask & want) == 0 || key0 >= walk.span.hi || key0 + 15 < walk.span.lo) continue;
        }
        const unsigned char* kbase =
            ring + s * 2 * kRowHalfStage + ((b0 * S::kCols) << a.box_log) * RB + (task * 16 - (b0 << a.box_log)) * RB;
        const unsigned char* vbase = kbase + kRowHalfStage;
        // ---- everything the task needs, into registers
        uint4 kr[kPieces][2];
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
          const int piece = F8 ? p * 4 + t4 : (p & 1) * 4 + t4;
          const unsigned char* src = kbase + (F8 ? 0 : (p >> 1) * col_stride) + g * RB +
                                     ((RB == 128 ? piece ^ g : piece) << 4);
          kr[p][0] = *reinterpret_cast<const uint4*>(src);
          kr[p][1] = *reinterpret_cast<const uint4*>(src + run_stride);
        }
        // V: the pieces of this lane's four tokens
        constexpr int kW = F8 ? D / 32 : 4;                  // words of a piece
        constexpr int kVC = F8 ? 1 : S::kCols;
        uint32_t v[kVC][4][kW];
#pragma unroll
        for (int cc = 0; cc < kVC; ++cc)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r8 = 2 * t4 + (e & 1);
            const unsigned char* src = vbase + cc * col_stride + (e >> 1) * run_stride + r8 * RB;
            if constexpr (RB == 128) {
              const uint4 y = *reinterpret_cast<const uint4*>(src + ((g ^ r8) << 4));
              v[cc][e][0] = y.x; v[cc][e][1] = y.y; v[cc][e][2] = y.z; v[cc][e][3] = y.w;
            } else {
              const uint2 y = *reinterpret_cast<const uint2*>(src + g * 8);
              v[cc][e][0] = y.x; v[cc][e][1] = y.y;
            }
          }
        int kbyte[2] = {127, 127}, vbyte[2] = {127, 127};
        if constexpr (F8) {
          const unsigned char* sc = s_scale + s * 2 * TOK + task * 16 + g;
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            kbyte[r] = sc[r * 8];
            vbyte[r] = sc[TOK + r * 8];
          }
        }
        // ---- S^T = K Q^T, in two chains
        float c[NQ][4], c2[NQ][4];
#pragma unroll
        for (int x = 0; x < NQ; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) c[x][e] = c2[x][e] = 0.0f;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
          const uint4 lo = kr[p][0], hi = kr[p][1];
          if constexpr (F8) {
            const uint32_t wl[4] = {lo.x, lo.y, lo.z, lo.w}, wh[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int st = 0; st < 4; ++st) {
              const uint32_t af[4] = {e4m3_bits(wl[st] & 0xffffu), e4m3_bits(wh[st] & 0xffffu),
                                      e4m3_bits(wl[st] >> 16), e4m3_bits(wh[st] >> 16)};
#pragma unroll
              for (int x = 0; x < NQ; ++x)
                mma_16816((st & 1) ? c2[x] : c[x], af, qf[x][p][st][0], qf[x][p][st][1], MT());
            }
          } else {
            const uint32_t a0[4] = {lo.x, hi.x, lo.y, hi.y}, a1[4] = {lo.z, hi.z, lo.w, hi.w};
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
              mma_16816(c[x], a0, qf[x][p][0][0], qf[x][p][0][1], MT());
              mma_16816(c2[x], a1, qf[x][p][1][0], qf[x][p][1][1], MT());
            }
          }
        }
#pragma unroll
        for (int x = 0; x < NQ; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) c[x][e] += c2[x][e];
        // ---- scores in powers of two; over e4m3 with the V exponent of each key added
        float unshift[2] = {1.0f, 1.0f};                    // 2^-b_j
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float kf = 1.0f, vexp = 0.0f;
          if constexpr (F8) {
            const int kb = kbyte[r], vb = weight_byte(vbyte[r]);
            kf = kb == 255 ? NAN : power_of_byte(kb);
            vexp = (float)(vb - 127);
            unshift[r] = __uint_as_float((unsigned int)(254 - vb) << 23);
          }
#pragma unroll
          for (int x = 0; x < NQ; ++x)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float& z = c[x][2 * r + h];
              z = F8 ? fmaf(z * kf, qscale[x][h], vexp) : z * qscale[x][h];
            }
        }
        if (!open) {
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int rel = r * 8 + g, key = key0 + rel;
            const bool here = key >= walk.span.lo && key < walk.span.hi && ((boxmask >> ((task * 16 + rel) >> a.box_log)) & 1u);
#pragma unroll
            for (int x = 0; x < NQ; ++x)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                bool ok = here && (TREE || !a.causal || key <= prow[x][h]) &&
                          (a.window <= 0 || (long long)key > (long long)prow[x][h] - a.window);
                if (TREE && key >= first) ok = here && ((tree[x][h] >> (key - first)) & 1u);
                if (!ok) c[x][2 * r + h] = -INFINITY;
              }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {                      // V rows nobody sees may hold anything
            const int rel = (e >> 1) * 8 + 2 * t4 + (e & 1), key = key0 + rel;
            const bool here = key >= walk.span.lo && key < walk.span.hi && ((boxmask >> ((task * 16 + rel) >> a.box_log)) & 1u);
            if (!here) {
#pragma unroll
              for (int cc = 0; cc < kVC; ++cc)
#pragma unroll
                for (int w4 = 0; w4 < kW; ++w4) v[cc][e][w4] = 0;
            }
          }
        }
        // ---- running maximum, moved only when it grows by more than 2^8
        constexpr float kHead = kWeightHead<MT>;
        float mt[NQ][2];
        bool grow = wide;                                   // (one branch for what is rare)
#pragma unroll
        for (int x = 0; x < NQ; ++x)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float y = fmaxf(c[x][h], c[x][2 + h]);
            y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 4));
            y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 8));
            y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 16));
            mt[x][h] = y;
            grow |= y > m[x][h] + (kHead + 8.0f);           // also from -infinity
          }
        uint32_t pb[NQ][2];
        auto weights = [&](int x, int r, float& p0, float& p1) {
          const float m0 = m[x][0] == -INFINITY ? 0.0f : m[x][0], m1 = m[x][1] == -INFINITY ? 0.0f : m[x][1];
          p0 = exp2_fast(c[x][2 * r] - m0);
          p1 = exp2_fast(c[x][2 * r + 1] - m1);
          l[x][0] += F8 ? p0 * unshift[r] : p0;
          l[x][1] += F8 ? p1 * unshift[r] : p1;
        };
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
          for (int x = 0; x < NQ; ++x)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float mn = fmaxf(m[x][h], mt[x][h] - kHead);
              const float al = mn == -INFINITY ? 1.0f : exp2_fast(m[x][h] - mn);
              m[x][h] = mn;
              l[x][h] *= al;
#pragma unroll
              for (int j = 0; j < kMT; ++j) {
                o[x][j][h] *= al;
                o[x][j][2 + h] *= al;
              }
            }
          if constexpr (F8) {
            if (wide) {
              // ---- O^T += V^T P^T, V and the weights as bf16
#pragma unroll
              for (int x = 0; x < NQ; ++x)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                  float p0, p1;
                  weights(x, r, p0, p1);
                  // what the weight does not carry yet; a NaN row is one for those that see it
                  const float rest = power_of_byte(127 + vbyte[r] - weight_byte(vbyte[r]));
                  c[x][2 * r] = vbyte[r] == 255 && c[x][2 * r] != -INFINITY ? NAN : p0 * rest;
                  c[x][2 * r + 1] = vbyte[r] == 255 && c[x][2 * r + 1] != -INFINITY ? NAN : p1 * rest;
                }
#pragma unroll 1
              for (int part = 0; part < 2; ++part) {
#pragma unroll
                for (int x = 0; x < NQ; ++x)
#pragma unroll
                  for (int r = 0; r < 2; ++r) {
                    const uint32_t hi = Bits16<__nv_bfloat16>::pack(c[x][2 * r], c[x][2 * r + 1]);
                    const float2 y = Bits16<__nv_bfloat16>::unpack(hi);
                    c[x][2 * r] -= y.x;
                    c[x][2 * r + 1] -= y.y;
                    pb[x][r] = transpose8(hi);
                  }
#pragma unroll
                for (int w4 = 0; w4 < kW; ++w4) {
#pragma unroll
                  for (int half = 0; half < 2; ++half) {
                    const uint32_t y0 = __byte_perm(v[0][0][w4], v[0][1][w4], half ? 0x7362 : 0x5140);
                    const uint32_t y1 = __byte_perm(v[0][2][w4], v[0][3][w4], half ? 0x7362 : 0x5140);
                    const uint32_t af[4] = {bf16_of_e4m3(y0 & 0xffffu, 1.0f), bf16_of_e4m3(y0 >> 16, 1.0f),
                                            bf16_of_e4m3(y1 & 0xffffu, 1.0f), bf16_of_e4m3(y1 >> 16, 1.0f)};
#pragma unroll
                    for (int x = 0; x < NQ; ++x)
                      mma_16816(o[x][2 * w4 + half], af, pb[x][0], pb[x][1], __nv_bfloat16());
                  }
                }
              }
              continue;
            }
          }
        }
#pragma unroll
        for (int x = 0; x < NQ; ++x)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float p0, p1;
            weights(x, r, p0, p1);
            pb[x][r] = transpose8(Bits16<MT>::pack(p0, p1));
          }
        // ---- O^T += V^T P^T
#pragma unroll
        for (int cc = 0; cc < kVC; ++cc)
#pragma unroll
          for (int w4 = 0; w4 < kW; ++w4) {
            if constexpr (F8) {
              const uint32_t lo0 = __byte_perm(v[cc][0][w4], v[cc][1][w4], 0x5140);
              const uint32_t hi0 = __byte_perm(v[cc][0][w4], v[cc][1][w4], 0x7362);
              const uint32_t lo1 = __byte_perm(v[cc][2][w4], v[cc][3][w4], 0x5140);
              const uint32_t hi1 = __byte_perm(v[cc][2][w4], v[cc][3][w4], 0x7362);
              const uint32_t a0[4] = {e4m3_bits(lo0 & 0xffffu), e4m3_bits(lo0 >> 16), e4m3_bits(lo1 & 0xffffu),
                                      e4m3_bits(lo1 >> 16)};
              const uint32_t a1[4] = {e4m3_bits(hi0 & 0xffffu), e4m3_bits(hi0 >> 16), e4m3_bits(hi1 & 0xffffu),
                                      e4m3_bits(hi1 >> 16)};
#pragma unroll
              for (int x = 0; x < NQ; ++x) {
                mma_16816(o[x][2 * w4], a0, pb[x][0], pb[x][1], MT());
                mma_16816(o[x][2 * w4 + 1], a1, pb[x][0], pb[x][1], MT());
              }
            } else {
              const uint32_t a0[4] = {
                  __byte_perm(v[cc][0][w4], v[cc][1][w4], 0x5410), __byte_perm(v[cc][0][w4], v[cc][1][w4], 0x7632),
                  __byte_perm(v[cc][2][w4], v[cc][3][w4], 0x5410), __byte_perm(v[cc][2][w4], v[cc][3][w4], 0x7632)};
#pragma unroll
              for (int x = 0; x < NQ; ++x) mma_16816(o[x][cc * 4 + w4], a0, pb[x][0], pb[x][1], MT());
            }
          }
      }
      turn = (turn - S::kTasks % kRowWarps + kRowWarps) % kRowWarps;
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&s_empty[s]));
    }

    // ---- join the warps
    const int par = seg & 1;
    ++seg;
#pragma unroll
    for (int x = 0; x < NQ; ++x)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[x][h] += __shfl_xor_sync(0xffffffffu, l[x][h], d);
        if (g == 0) {
          s_m[par][warp][x * 8 + 2 * t4 + h] = m[x][h];
          s_l[par][warp][x * 8 + 2 * t4 + h] = l[x][h];
        }
      }
    asm volatile("bar.sync 1, %0;" ::"n"(32 * kRowWarps) : "memory");
    // the upper half of the warps hands its O to the lower half, whose sums meet in shared memory
#pragma unroll
    for (int go = 0; go < 2; ++go) {
      const bool upper = warp >= kRowWarps / 2;
#pragma unroll
      for (int x = 0; x < NQ; ++x)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int i = x * 8 + 2 * t4 + h;
          if (i >= n_rows || upper != (go == 0)) continue;
          float top = -INFINITY;
#pragma unroll
          for (int y = 0; y < kRowWarps; ++y) top = fmaxf(top, s_m[par][y][i]);
          const float f = top == -INFINITY ? 0.0f : exp2_fast(m[x][h] - top);
          float* dst = merge + ((warp % (kRowWarps / 2)) * ROWS + i) * D;
#pragma unroll
          for (int j = 0; j < kMT; ++j)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const int d = F8 ? g * (D / 8) + 2 * j + r : (j >> 2) * 64 + g * 8 + (j & 3) * 2 + r;
              const float y = o[x][j][2 * r + h] * f;
              dst[d] = go == 0 ? y : dst[d] + y;
            }
        }
      asm volatile("bar.sync 1, %0;" ::"n"(32 * kRowWarps) : "memory");
    }
    const bool whole = walk.whole();
    const bool at_start = walk.pos - (walk.t1 - walk.t0) ==
                          (w.total + gridDim.x - 1) / gridDim.x * blockIdx.x;
    float* slot = a.slots + ((long long)blockIdx.x * 2 + (at_start ? 0 : 1)) * S::kSlot;
    for (int x = threadIdx.x; x < n_rows * (D / 2); x += 32 * kRowWarps) {
      const int i = x / (D / 2), d = (x - i * (D / 2)) * 2;
      float top = -INFINITY, sum = 0.0f;
#pragma unroll
      for (int y = 0; y < kRowWarps; ++y) top = fmaxf(top, s_m[par][y][i]);
      const float safe = top == -INFINITY ? 0.0f : top;
      float v0 = 0.0f, v1 = 0.0f;
#pragma unroll
      for (int y = 0; y < kRowWarps; ++y) sum += s_l[par][y][i] * exp2_fast(s_m[par][y][i] - safe);
#pragma unroll
      for (int y = 0; y < kRowWarps / 2; ++y) {
        const float2 p = *reinterpret_cast<const float2*>(merge + (y * ROWS + i) * D + d);
        v0 += p.x;
        v1 += p.y;
      }
      if (whole) {
        const int ti = a.by_g.div(i);
        const long long tok = walk.q.tok0 + ti;
        const int qh = walk.head * a.G + (i - ti * a.G);
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        QT* dst = reinterpret_cast<QT*>(a.out) + tok * a.o_tok + (long long)qh * a.o_head + d;
        *reinterpret_cast<uint32_t*>(dst) = Bits16<QT>::pack(v0 * inv, v1 * inv);
        if (a.lse && d == 0)
          a.lse[tok * (a.pool.H * a.G) + qh] = sum == 0.0f ? -INFINITY : 0.69314718056f * (top + log2f(sum));
      } else {
        *reinterpret_cast<float2*>(slot + 2 * ROWS + i * D + d) = make_float2(v0, v1);
        if (d == 0) {
          slot[i] = top;
          slot[ROWS + i] = sum;
        }
      }
    }
  }
}

template <int D, bool F8, typename QT, int ROWS, bool TREE>
inline int32_t launch_attn_rows(AttnArgs a, int type, JoinSet& join, cudaStream_t st) {
  using S = RowShape<D, F8, ROWS>;
  a.box = gcd_int(a.pool.T, S::kTok);
  a.box_log = log2_int(a.box);
  CUtensorMap map_k, map_v;
  int32_t rc = plane_tensor_map(a.pool, type, a.box, 0, &map_k);
  if (rc == AIBX_OK) rc = plane_tensor_map(a.pool, type, a.box, 1, &map_v);
  if (rc != AIBX_OK) return rc;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return AIBX_ERR_CUDA;
  static size_t configured[64] = {0};
  static std::mutex lock;
  if (!ensure_dynamic_smem(attn_rows_kernel<D, F8, QT, ROWS, TREE>, S::kSmem, dev, configured, lock))
    return AIBX_ERR_CUDA;
  const unsigned int grid = (unsigned int)sm_count();
  attn_rows_kernel<D, F8, QT, ROWS, TREE><<<grid, S::kThreads, S::kSmem, st>>>(map_k, map_v, a);
  join = JoinSet{a.slots, reinterpret_cast<const JoinRecord*>(a.slots + 2ull * grid * S::kSlot), ROWS};
  return launch_status();
}

}  // namespace aibx
