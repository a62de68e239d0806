// Attention of few query rows (new tokens * query heads per KV head <= 16) over a paged cache: a
// decoding step, or a few speculative tokens.
//
// Mathematics, per (request, KV head) with query rows i and keys j, in powers of two:
//   t_ij = scale * log2(e) * q_i . k_j,  m = running max, l = sum 2^(t - m), O = sum 2^(t - m) v_j,
//   out = O / l, lse = ln 2 * (m + log2 l).
// Over an e4m3 pool k_j = K_j 2^a_j and v_j = V_j 2^b_j with e4m3 rows K_j, V_j.  Those are exact
// in fp16, so they go to the tensor core as they are: the scores take 2^a_j afterwards, and the
// weight that multiplies V_j is w = 2^(t + b_j - m) with m the maximum of t + b_j; then
// l = sum w 2^-b_j.  Queries are scaled to [1, 2) per row to fit fp16 (fp16 keeps 3 more bits than
// bf16; what falls below 2^-24 of the row's maximum is lost).
//
// Bound: HBM.  Every K and V byte is read once and meets at most 16 rows, so the legacy tensor
// path (mma.sync m16n8k16) has an order of magnitude to spare: 16 tokens of D = 128 cost 32 MMAs
// against 341 cycles of this SM's share of the bandwidth (16-bit rows).  What counts is bytes in
// flight: one warp feeds a ring of five 32 KB stages with tensor-map boxes (one box = the slots
// of one block and head), 160 KB per SM outstanding, and runs ahead over the seams between
// requests, so that the memory never idles; eight warps consume, 16 tokens each at a time, with
// their own m, l and O, joined once per (request, head).
// Fragments are read from shared memory without transposition: the order of the contraction index
// is free as long as both operands agree.  For Q K^T a lane's 16-byte piece of a K row serves as
// the k-indices of two MMAs; for P V a lane reads the same 16-byte column piece of its four
// tokens and pairs tokens with byte permutes.
#pragma once

#include "attn_common.cuh"

namespace aibx {

constexpr int kRowWarps = 8;
constexpr int kRowStages = 5;
constexpr int kRowHalfStage = 16384;                       // bytes of K (and of V) per stage
constexpr int kScaleWarps = 3;                            // 12 warps in all: 168 registers each

template <int D, bool F8>
struct RowShape {
  static constexpr int kElem = F8 ? 1 : 2;
  static constexpr int kTok = kRowHalfStage / (D * kElem);   // tokens per stage
  static constexpr int kRowBytes = F8 ? D : 128;             // bytes of a shared-memory row
  static constexpr int kCols = F8 ? 1 : D / 64;              // 128-byte columns of a 16-bit row
  static constexpr int kTasks = kTok / 16;
  static constexpr int kThreads = 32 * (kRowWarps + 1 + (F8 ? kScaleWarps : 0));
  static constexpr int kSmem = kRowStages * 2 * kRowHalfStage + kRowWarps / 2 * kRowsMax * D * 4 +
                               (F8 ? kRowStages * 2 * kTok : 0) + 1024;
  static constexpr int kSlot = kRowsMax * (D + 2);           // floats per workspace slot
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
  s.tiles = max(1, (s.hi + TOK - 1) / TOK - s.tile0);
  return s;
}

template <int TOK>
struct RowCost {
  const AttnArgs& a;
  __device__ __forceinline__ long long operator()(int r) const {
    const AttnRequest q = attn_request(a.b, a.pool.T, r);
    if (q.n == 0 || (long long)q.n * a.G > kRowsMax) return 0;
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
      } while (q.n == 0 || (long long)q.n * a.G > kRowsMax);
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

// Block ids of a tile's boxes, one per lane; `valid` where the box is there and holds keys.
template <int TOK>
__device__ __forceinline__ uint32_t box_block(const AttnArgs& a, const uint32_t* row, int tile,
                                              int lane, int boxes, int lo, int hi, bool tell,
                                              bool& valid, int& slot) {
  const int tok = tile * TOK + lane * a.box;
  valid = lane < boxes && tok < hi && tok + a.box > lo;
  slot = 0;
  uint32_t id = 0;
  if (valid) {
    const int at = tok / a.pool.T;
    slot = tok - at * a.pool.T;
    id = __ldg(row + at);
    if (id >= a.pool.num_blocks) {
      if (id != AIBX_NO_BLOCK && tell) raise_status(AIBX_ERR_RANGE);
      valid = false;
    }
  }
  return id;
}

template <int D, bool F8, typename QT>
__global__ void __launch_bounds__(RowShape<D, F8>::kThreads, 1)
attn_rows_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ AttnArgs a) {
  using S = RowShape<D, F8>;
  using MT = typename std::conditional<F8, __half, QT>::type;   // operand type of the MMAs
  constexpr int TOK = S::kTok, RB = S::kRowBytes;
  extern __shared__ unsigned char s_raw[];
  __shared__ __align__(8) unsigned long long s_full[kRowStages], s_empty[kRowStages];
  __shared__ unsigned int s_mask[kRowStages];
  __shared__ float s_m[2][kRowWarps][kRowsMax], s_l[2][kRowWarps][kRowsMax];
  __shared__ long long s_scan[33];
  __shared__ WorkStart s_start;
  __shared__ int s_abort;

  const unsigned int smem0 = (smem_u32(s_raw) + 1023u) & ~1023u;
  unsigned char* ring = s_raw + (smem0 - smem_u32(s_raw));
  float* merge = reinterpret_cast<float*>(ring + kRowStages * 2 * kRowHalfStage);
  unsigned char* s_scale = reinterpret_cast<unsigned char*>(merge + kRowWarps / 2 * kRowsMax * D);
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
  if (a.check_bound && blockIdx.x == 0)
    for (int r = threadIdx.x; r < a.b.R; r += S::kThreads) {
      const AttnRequest q = attn_request(a.b, a.pool.T, r);
      if ((long long)q.n * a.G > kRowsMax) raise_status(AIBX_ERR_RANGE);
    }
  const RowCost<TOK> cost{a};
  const WorkStart w = locate_piece<S::kThreads>(a.b.R, blockIdx.x, gridDim.x, s_scan, &s_start, cost);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  RowWalk<TOK> walk(a, w, blockIdx.x, gridDim.x);
  volatile int* abort_flag = &s_abort;
  const int boxes = TOK / a.box;

  if (warp == kRowWarps) {
    // ---------------------------------------------------------------- loader warp
    unsigned int it = 0;
    while (walk.next()) {
      const uint32_t* row;
      long long entries;
      table_row(a.b, walk.r, row, entries);
      if (walk.q.keys < walk.q.len && walk.head == 0 && walk.t0 == 0 && lane == 0)
        raise_status(AIBX_ERR_RANGE);                      // tokens the table has no entry for
      bool valid, valid_next = false;
      int slot, slot_next = 0;
      uint32_t id = box_block<TOK>(a, row, walk.span.tile0 + walk.t0, lane, boxes, walk.span.lo,
                                   walk.span.hi, walk.head == 0, valid, slot);
      for (int t = walk.t0; t < walk.t1; ++t, ++it) {
        uint32_t id_next = 0;
        if (t + 1 < walk.t1)
          id_next = box_block<TOK>(a, row, walk.span.tile0 + t + 1, lane, boxes, walk.span.lo,
                                   walk.span.hi, walk.head == 0, valid_next, slot_next);
        const int s = (int)(it % kRowStages);
        const unsigned int bar = smem_u32(&s_full[s]);
        if (it >= kRowStages) ring_wait(smem_u32(&s_empty[s]), (it / kRowStages - 1) & 1u, abort_flag);
        __syncwarp();
        if (*abort_flag) valid = false;
        const unsigned int mask = __ballot_sync(0xffffffffu, valid);
        if (lane == 0) {
          s_mask[s] = mask;
          if (mask)
            mbar_arrive_expect_tx(bar, (unsigned int)__popc(mask) * 2u * a.box * D * S::kElem);
          else
            mbar_arrive(bar);
        }
        __syncwarp();
        if (valid) {
          const unsigned int dst = smem0 + s * 2 * kRowHalfStage + lane * a.box * RB;
#pragma unroll
          for (int kv = 0; kv < 2; ++kv)
#pragma unroll
            for (int c = 0; c < S::kCols; ++c)
              tensor_load_5d(dst + kv * kRowHalfStage + c * TOK * RB, &map, bar, c * 64, slot,
                             walk.head, (int)id, kv);
        }
        id = id_next;
        valid = valid_next;
        slot = slot_next;
      }
    }
    // what is still in flight targets this CTA's shared memory: wait for it before leaving
    for (unsigned int i = it > kRowStages ? it - kRowStages : 0; i < it; ++i)
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
        if (tok < walk.span.hi) {
          const int at = tok / a.pool.T;
          const uint32_t id = __ldg(row + at);
          if (id < a.pool.num_blocks) {
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
        const int s = (int)(it % kRowStages);
        if (it >= kRowStages) ring_wait(smem_u32(&s_empty[s]), (it / kRowStages - 1) & 1u, abort_flag);
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
  constexpr int kNT = D / 8;                               // n-tiles of O
  constexpr int kPiece = F8 ? 16 : 8;                      // elements of a lane's piece of a K row
  constexpr int kPieces = D / (4 * kPiece);
  constexpr int kSteps = kPiece / 4;                       // MMAs per piece
  unsigned int it = 0;
  int seg = 0;
  while (walk.next()) {
    const int n_rows = walk.q.n * a.G;
    const int first = walk.q.len - walk.q.n;
    uint32_t qf[kPieces][kSteps][4];
    float qscale[2];
    int prow[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int i = g + 8 * h;
      const int ti = min(i, n_rows - 1) / a.G;
      prow[h] = first + ti;
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
      if (F8) {
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
      qscale[h] = up * a.scale_log2;
#pragma unroll
      for (int p = 0; p < kPieces; ++p)
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          qf[p][s][h] = raw[p][2 * s];
          qf[p][s][2 + h] = raw[p][2 * s + 1];
        }
    }
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
    float o[kNT][4];
#pragma unroll
    for (int j = 0; j < kNT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[j][e] = 0.0f;

    for (int t = walk.t0; t < walk.t1; ++t, ++it) {
      const int s = (int)(it % kRowStages);
      ring_wait(smem_u32(&s_full[s]), (it / kRowStages) & 1u, abort_flag);
      __syncwarp();
      const unsigned int boxmask = s_mask[s];
      // the 16-token tasks of all stages go round the warps in turn
      for (int task = (int)(((unsigned int)warp - it * S::kTasks) & (kRowWarps - 1)); task < S::kTasks; task += kRowWarps) {
        const int key0 = (walk.span.tile0 + t) * TOK + task * 16;
        if (key0 >= walk.span.hi || key0 + 15 < walk.span.lo) continue;
        const int b0 = task * 16 / a.box, b1 = (task * 16 + 15) / a.box;
        const unsigned int want = ((2u << (b1 - b0)) - 1u) << b0;
        if ((boxmask & want) == 0) continue;
        // all 16 keys seen by all rows: the rows' positions run from `first` to len - 1
        const bool open = (boxmask & want) == want && key0 + 15 < walk.span.hi &&
                          (!a.causal || key0 + 15 <= first) &&
                          (a.window <= 0 || key0 > (long long)walk.q.len - 1 - a.window);
        const unsigned char* kbase = ring + s * 2 * kRowHalfStage + task * 16 * RB;
        const unsigned char* vbase = kbase + kRowHalfStage;
        float c[2][4];
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
#pragma unroll
          for (int e = 0; e < 4; ++e) c[nt][e] = 0.0f;
          const int row = nt * 8 + g;
#pragma unroll
          for (int p = 0; p < kPieces; ++p) {
            if constexpr (F8) {
              const int piece = p * 4 + t4;
              const unsigned char* src = kbase + row * RB + ((RB == 128 ? piece ^ (row & 7) : piece) << 4);
              const uint4 v = *reinterpret_cast<const uint4*>(src);
              const uint32_t wv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
              for (int st = 0; st < 4; ++st) {
                const __half2 lo = halves_of_e4m3(wv[st] & 0xffffu), hi = halves_of_e4m3(wv[st] >> 16);
                mma_16816(c[nt], qf[p][st], *reinterpret_cast<const uint32_t*>(&lo),
                          *reinterpret_cast<const uint32_t*>(&hi), MT());
              }
            } else {
              const int piece = (p & 1) * 4 + t4;
              const unsigned char* src = kbase + (p >> 1) * TOK * 128 + row * 128 + ((piece ^ (row & 7)) << 4);
              const uint4 v = *reinterpret_cast<const uint4*>(src);
              mma_16816(c[nt], qf[p][0], v.x, v.y, MT());
              mma_16816(c[nt], qf[p][1], v.z, v.w, MT());
            }
          }
        }
        // ---- scores in powers of two; over e4m3 with the V exponent of each key added
        float unshift[2][2];                                // 2^-b_j
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float kf = 1.0f, vexp = 0.0f;
            if constexpr (F8) {
              const unsigned char* sc = s_scale + s * 2 * TOK + task * 16 + nt * 8 + 2 * t4 + e;
              const int kb = sc[0], vb = sc[TOK];
              kf = kb == 255 ? NAN : power_of_byte(kb);
              const int ve = max(vb - 127, -100);
              vexp = vb == 255 ? NAN : (float)ve;
              unshift[nt][e] = __uint_as_float((unsigned int)(127 - min(ve, 126)) << 23);
            }
            c[nt][e] = fmaf(c[nt][e] * kf, qscale[0], vexp);
            c[nt][2 + e] = fmaf(c[nt][2 + e] * kf, qscale[1], vexp);
          }
        unsigned int seen = 0xfu;                           // this lane's four tokens: V rows that count
        if (!open) {
          seen = 0;
#pragma unroll
          for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int rel = nt * 8 + 2 * t4 + e;
              const int key = key0 + rel;
              const bool here = key >= walk.span.lo && key < walk.span.hi &&
                                ((boxmask >> ((task * 16 + rel) / a.box)) & 1u);
              if (here) seen |= 1u << (nt * 2 + e);
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const bool ok = here && (!a.causal || key <= prow[h]) &&
                                (a.window <= 0 || (long long)key > (long long)prow[h] - a.window);
                if (!ok) c[nt][2 * h + e] = -INFINITY;
              }
            }
        }
        // ---- running maximum, moved only when it grows by more than 2^8
        float mt[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float x = fmaxf(fmaxf(c[0][2 * h], c[0][2 * h + 1]), fmaxf(c[1][2 * h], c[1][2 * h + 1]));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
          mt[h] = x;
        }
        const bool grow = mt[0] > m[0] + 8.0f || mt[1] > m[1] + 8.0f;   // also from -infinity
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float mn = fmaxf(m[h], mt[h]);
            const float al = mn == -INFINITY ? 1.0f : exp2_fast(m[h] - mn);
            m[h] = mn;
            l[h] *= al;
#pragma unroll
            for (int j = 0; j < kNT; ++j) {
              o[j][2 * h] *= al;
              o[j][2 * h + 1] *= al;
            }
          }
        }
        const float ms[2] = {m[0] == -INFINITY ? 0.0f : m[0], m[1] == -INFINITY ? 0.0f : m[1]};
        uint32_t pa[4];
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float p0 = exp2_fast(c[nt][2 * h] - ms[h]), p1 = exp2_fast(c[nt][2 * h + 1] - ms[h]);
            if constexpr (F8)
              l[h] += p0 * unshift[nt][0] + p1 * unshift[nt][1];
            else
              l[h] += p0 + p1;
            pa[nt * 2 + h] = Bits16<MT>::pack(p0, p1);
          }
        // ---- O += P V
        const int r0 = 2 * t4;
        if constexpr (F8) {
          constexpr int kW = D / 32;                        // words of a lane's piece of a V row
          uint32_t v[4][kW];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int row = (e >> 1) * 8 + r0 + (e & 1);
            if constexpr (RB == 128) {
              const uint4 x = *reinterpret_cast<const uint4*>(vbase + row * 128 + ((g ^ (row & 7)) << 4));
              v[e][0] = x.x; v[e][1] = x.y; v[e][2] = x.z; v[e][3] = x.w;
            } else {
              const uint2 x = *reinterpret_cast<const uint2*>(vbase + row * RB + g * 8);
              v[e][0] = x.x; v[e][1] = x.y;
            }
            if (!((seen >> e) & 1u)) {
#pragma unroll
              for (int q = 0; q < kW; ++q) v[e][q] = 0;
            }
          }
#pragma unroll
          for (int q = 0; q < kW; ++q) {
            uint32_t b[2][4];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const uint32_t lo = __byte_perm(v[2 * half][q], v[2 * half + 1][q], 0x5140);
              const uint32_t hi = __byte_perm(v[2 * half][q], v[2 * half + 1][q], 0x7362);
              const __half2 x0 = halves_of_e4m3(lo & 0xffffu), x1 = halves_of_e4m3(lo >> 16);
              const __half2 x2 = halves_of_e4m3(hi & 0xffffu), x3 = halves_of_e4m3(hi >> 16);
              b[half][0] = *reinterpret_cast<const uint32_t*>(&x0);
              b[half][1] = *reinterpret_cast<const uint32_t*>(&x1);
              b[half][2] = *reinterpret_cast<const uint32_t*>(&x2);
              b[half][3] = *reinterpret_cast<const uint32_t*>(&x3);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) mma_16816(o[4 * q + e], pa, b[0][e], b[1][e], MT());
          }
        } else {
#pragma unroll
          for (int hh = 0; hh < S::kCols; ++hh) {
            uint32_t v[4][4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int row = (e >> 1) * 8 + r0 + (e & 1);
              const uint4 x = *reinterpret_cast<const uint4*>(vbase + hh * TOK * 128 + row * 128 +
                                                              ((g ^ (row & 7)) << 4));
              v[e][0] = x.x; v[e][1] = x.y; v[e][2] = x.z; v[e][3] = x.w;
              if (!((seen >> e) & 1u)) v[e][0] = v[e][1] = v[e][2] = v[e][3] = 0;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              mma_16816(o[hh * 8 + 2 * q], pa, __byte_perm(v[0][q], v[1][q], 0x5410),
                        __byte_perm(v[2][q], v[3][q], 0x5410), MT());
              mma_16816(o[hh * 8 + 2 * q + 1], pa, __byte_perm(v[0][q], v[1][q], 0x7632),
                        __byte_perm(v[2][q], v[3][q], 0x7632), MT());
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&s_empty[s]));
    }

    // ---- join the eight warps
    const int par = seg & 1;
    ++seg;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
      if (t4 == 0) {
        s_m[par][warp][g + 8 * h] = m[h];
        s_l[par][warp][g + 8 * h] = l[h];
      }
    }
    asm volatile("bar.sync 1, %0;" ::"n"(32 * kRowWarps) : "memory");
    // the upper four warps hand their O to the lower four, whose sums meet in shared memory
#pragma unroll
    for (int turn = 0; turn < 2; ++turn) {
      const bool upper = warp >= kRowWarps / 2;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int i = g + 8 * h;
        if (i >= n_rows || upper != (turn == 0)) continue;
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < kRowWarps; ++x) top = fmaxf(top, s_m[par][x][i]);
        const float f = top == -INFINITY ? 0.0f : exp2_fast(m[h] - top);
        float* dst = merge + ((warp & (kRowWarps / 2 - 1)) * kRowsMax + i) * D;
#pragma unroll
        for (int j = 0; j < kNT; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int n = 2 * t4 + e;
            const int d = F8 ? n * (D / 8) + j : (j >> 3) * 64 + n * 8 + (j & 7);
            const float x = o[j][2 * h + e] * f;
            dst[d] = turn == 0 ? x : dst[d] + x;
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
        const float2 p = *reinterpret_cast<const float2*>(merge + (y * kRowsMax + i) * D + d);
        v0 += p.x;
        v1 += p.y;
      }
      if (whole) {
        const int ti = i / a.G;
        const long long tok = walk.q.tok0 + ti;
        const int qh = walk.head * a.G + (i - ti * a.G);
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        QT* dst = reinterpret_cast<QT*>(a.out) + tok * a.o_tok + (long long)qh * a.o_head + d;
        *reinterpret_cast<uint32_t*>(dst) = Bits16<QT>::pack(v0 * inv, v1 * inv);
        if (a.lse && d == 0)
          a.lse[tok * (a.pool.H * a.G) + qh] = sum == 0.0f ? -INFINITY : 0.69314718056f * (top + log2f(sum));
      } else {
        *reinterpret_cast<float2*>(slot + 2 * kRowsMax + i * D + d) = make_float2(v0, v1);
        if (d == 0) {
          slot[i] = top;
          slot[kRowsMax + i] = sum;
        }
      }
    }
  }
}

// Joins a (request, head) that was cut: block c takes the one whose last tile lies in CTA c and
// whose first tile lies in an earlier CTA.
template <int D, bool F8, typename QT>
__global__ void __launch_bounds__(256)
attn_rows_join_kernel(const __grid_constant__ AttnArgs a) {
  using S = RowShape<D, F8>;
  constexpr int TOK = S::kTok;
  __shared__ long long s_scan[33];
  __shared__ WorkStart s_start;
  const RowCost<TOK> cost{a};
  const WorkStart w = locate_piece<256>(a.b.R, blockIdx.x, gridDim.x, s_scan, &s_start, cost);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  RowWalk<TOK> walk(a, w, blockIdx.x, gridDim.x);
  if (!walk.next() || walk.t0 == 0 || walk.t1 != walk.span.tiles) return;
  const long long per = (w.total + gridDim.x - 1) / gridDim.x;
  const long long p0 = walk.base + (long long)walk.head * walk.span.tiles;   // its first position
  const int c0 = (int)(p0 / per), c1 = (int)blockIdx.x;
  const int n_rows = walk.q.n * a.G;
  for (int x = threadIdx.x; x < n_rows * (D / 2); x += 256) {
    const int i = x / (D / 2), d = (x - i * (D / 2)) * 2;
    float top = -INFINITY, sum = 0.0f, v0 = 0.0f, v1 = 0.0f;
    for (int c = c0; c <= c1; ++c) {
      const float* slot = a.slots + ((long long)c * 2 + (c == c0 && p0 != c0 * per ? 1 : 0)) * S::kSlot;
      const float mc = slot[i];
      const float2 p = *reinterpret_cast<const float2*>(slot + 2 * kRowsMax + i * D + d);
      const float tn = fmaxf(top, mc);
      const float safe = tn == -INFINITY ? 0.0f : tn;
      const float f0 = exp2_fast(top - safe), f1 = exp2_fast(mc - safe);
      sum = sum * f0 + slot[kRowsMax + i] * f1;
      v0 = v0 * f0 + p.x * f1;
      v1 = v1 * f0 + p.y * f1;
      top = tn;
    }
    const int ti = i / a.G;
    const long long tok = walk.q.tok0 + ti;
    const int qh = walk.head * a.G + (i - ti * a.G);
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    QT* dst = reinterpret_cast<QT*>(a.out) + tok * a.o_tok + (long long)qh * a.o_head + d;
    *reinterpret_cast<uint32_t*>(dst) = Bits16<QT>::pack(v0 * inv, v1 * inv);
    if (a.lse && d == 0)
      a.lse[tok * (a.pool.H * a.G) + qh] = sum == 0.0f ? -INFINITY : 0.69314718056f * (top + log2f(sum));
  }
}

// ------------------------------------------------------------------------------------------

template <typename Kernel>
inline int32_t launch_after(Kernel kernel, dim3 grid, unsigned int threads, cudaStream_t st,
                            const AttnArgs& a) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a) == cudaSuccess ? AIBX_OK : AIBX_ERR_CUDA;
}

template <int D, bool F8, typename QT>
inline int32_t launch_attn_rows(AttnArgs a, int type, cudaStream_t st) {
  using S = RowShape<D, F8>;
  a.box = gcd_int(a.pool.T, S::kTok);
  CUtensorMap map;
  const int32_t rc = pool_tensor_map(a.pool, type, a.box, &map);
  if (rc != AIBX_OK) return rc;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return AIBX_ERR_CUDA;
  static size_t configured[64] = {0};
  static std::mutex lock;
  if (!ensure_dynamic_smem(attn_rows_kernel<D, F8, QT>, S::kSmem, dev, configured, lock))
    return AIBX_ERR_CUDA;
  const unsigned int grid = (unsigned int)sm_count();
  attn_rows_kernel<D, F8, QT><<<grid, S::kThreads, S::kSmem, st>>>(map, a);
  const int32_t rc2 = launch_status();
  if (rc2 != AIBX_OK) return rc2;
  return launch_after(attn_rows_join_kernel<D, F8, QT>, dim3(grid), 256, st, a);
}

}  // namespace aibx
