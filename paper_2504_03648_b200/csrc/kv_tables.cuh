// What a step of an engine needs to know of its requests, from their lengths alone: block tables grown
// from a free list, offsets, positions, slots (kv_tables), and the ancestor masks of drafted trees
// (tree_masks).  Integers only.
//
// kv_tables, per request with h held and n new tokens, blocks of T slots:
//   had = ceil(h / T), need = ceil((h + n) / T); F = sum of need - had over the requests before;
//   table[had + k] = free[(head + F + k) mod capacity];  tok_off = sum of n before;  kv_len = h + n;
//   token i: position p = h + i, slot table[p / T] * T + p mod T.
// One launch: every CTA takes the prefix sums over all requests for itself, 512 at a time (they are a few
// kilobytes out of L2, and a barrier or a second launch costs more than the sums), keeps them in shared
// memory and then finds the request of each of its tokens by halving.  A new block's entry is written by
// its first token: no search of its own.  Bound: launch and the chain lengths -> sums -> entry -> slot
// for the calls that are usual (200 single tokens: 6.3 us); with many tokens the instructions of finding a
// token's block, 12 bytes being all that it writes (96 prompts of 840,000 tokens: 14.5 us, 0.78 TB/s).
//
// tree_masks, per request: mask(i) = bit i, or that and mask(parent(i)).  In shared memory, twice as far
// up each round: mask'(i) = mask(i) | mask(up(i)), up'(i) = up(up(i)), so that a chain of 512 takes nine
// rounds; all of a round's reads come before its writes.  250 requests of 300 to 512 nodes: 12.5 us (7.5 MB), of
// which rounds in shared memory and their barriers are the most; 12 of 26 nodes: 4.3 us.
#pragma once

#include <limits.h>

#include "attn_common.cuh"

namespace aibx {

// Division of 0 <= p < 2^31 by T: with 2^(s-1) < T <= 2^s and m = floor(2^(31+s) / T) + 1, m T exceeds 2^(31+s)
// by at most T <= 2^s, so p m / 2^(31+s) exceeds p / T by less than 1 / T.
struct PositionDivisor {
  uint32_t m;
  int shift;
  __device__ __forceinline__ int div(int p) const { return (int)(((uint64_t)(uint32_t)p * m) >> shift); }
};
inline PositionDivisor position_divisor(int T) {
  int s = 0;
  while ((1 << s) < T) ++s;
  return PositionDivisor{(uint32_t)((1ull << (31 + s)) / (uint64_t)T + 1), 31 + s};
}

struct TablesArgs {
  const int32_t *held, *fresh;     // tokens held, tokens new
  int R, T;
  PositionDivisor by_T;
  uint32_t num_blocks;
  const uint32_t* free_ids;
  long long capacity;
  const int64_t *head, *tail;
  int64_t* head_out;
  uint32_t* table;
  const int64_t* blk_off;
  long long stride;
  const uint32_t* match;
  const int64_t* match_off;
  int64_t* tok_off;
  int32_t* kv_len;
  int32_t* pos;
  int64_t* slots;
  long long n_tokens;
};

constexpr int kTablesThreads = 512;

// Last k in [0, n) with at[k] <= x (at[0] <= x): the request that holds x, past those without any.  In as many
// bits as X has.
template <typename X>
__device__ __forceinline__ int last_not_above(const long long* at, int n, X x) {
  int lo = 0;
  while (n > 1) {
    const int half = n >> 1;
    if ((X)at[lo + half] <= x) {
      lo += half;
      n -= half;
    } else {
      n = half;
    }
  }
  return lo;
}

// Exclusive prefixes and sums of three numbers per thread over the block.
template <int N>
__device__ __forceinline__ void block_prefix3(long long (&v)[3], long long (&scratch)[3][N / 32], long long (&total)[3]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long inc[3];
#pragma unroll
  for (int x = 0; x < 3; ++x) {
    inc[x] = v[x];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long up = (long long)shfl_up64((uint64_t)inc[x], d);
      if (lane >= d) inc[x] += up;
    }
    if (lane == 31) scratch[x][warp] = inc[x];
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < 3; ++x) {
    long long w = lane < N / 32 ? scratch[x][lane] : 0;     // warps' sums, a lane each
    const long long own = w;
#pragma unroll
    for (int d = 1; d < N / 32; d <<= 1) {
      const long long up = (long long)shfl_up64((uint64_t)w, d);
      if (lane >= d) w += up;
    }
    total[x] = (long long)shfl64(0xffffffffu, (uint64_t)w, N / 32 - 1);
    const long long before = (long long)shfl64(0xffffffffu, (uint64_t)(w - own), warp);
    v[x] = before + inc[x] - v[x];
  }
  __syncthreads();
}

struct Lengths {
  int h, n, had, need;
  bool bad;
};

__device__ __forceinline__ Lengths request_lengths(const TablesArgs& a, int r) {
  Lengths q = {0, 0, 0, 0, false};
  if (r >= a.R) return q;
  const int h = __ldg(a.held + r), n = __ldg(a.fresh + r);
  q.bad = h < 0 || n < 0 || (long long)h + n > INT_MAX;
  q.h = max(h, 0);
  q.n = q.bad ? 0 : n;
  q.had = (int)(((unsigned int)q.h + a.T - 1) / (unsigned int)a.T);
  q.need = (int)(((unsigned int)q.h + q.n + a.T - 1) / (unsigned int)a.T);
  return q;
}

// kTables: all but the two outputs that may stand in the place of inputs (kv_len, head), which need every
// CTA to have read those; kCommit: these two.  A call with one CTA, or whose outputs stand apart, does both
// at once; else a second launch of one CTA commits.
template <bool TABLES, bool COMMIT>
__global__ void __launch_bounds__(kTablesThreads, 2)
kv_tables_kernel(const __grid_constant__ TablesArgs a) {
  constexpr int N = kTablesThreads;
  __shared__ long long s_scan[3][N / 32];
  __shared__ long long s_tok[N], s_free[N], s_ent[N], s_row[N], s_match[N];
  __shared__ int s_held[N], s_had[N], s_width[N], s_matches[N];
  const int tid = threadIdx.x;
  const long long head = *a.head;
  long long left = *a.tail - head;                         // ids to be had
  left = left < 0 ? 0 : left > a.capacity ? a.capacity : left;
  long long start = head % a.capacity;
  if (start < 0) start += a.capacity;

  auto matched = [&](int k, int e) -> const uint32_t* {   // entry e of the tile's request k among the matched ids
    if (e < s_matches[k]) return a.match + s_match[k] + e;
    raise_status(AIBX_ERR_RANGE);
    return nullptr;
  };

  long long tok_base = 0, free_base = 0;
  for (int r0 = 0; r0 < a.R; r0 += N) {
    const int r = r0 + tid, rows = min(N, a.R - r0);
    const Lengths q = request_lengths(a, r);
    long long row = 0, width = 0;
    if (r < a.R) {
      row = a.blk_off ? __ldg(a.blk_off + r) : (long long)r * a.stride;
      width = a.blk_off ? __ldg(a.blk_off + r + 1) - row : a.stride;
      width = width < 0 ? 0 : width > INT_MAX ? INT_MAX : width;
    }
    const int have = min(q.had, (int)width), new_blocks = max(min(q.need, (int)width) - q.had, 0);
    long long match_at = 0, matches = 0;
    if (TABLES && a.match && r < a.R) {
      match_at = __ldg(a.match_off + r);
      matches = __ldg(a.match_off + r + 1) - match_at;
    }
    long long sums[3] = {q.n, new_blocks, a.match && r < a.R ? have : 0}, totals[3];
    block_prefix3<N>(sums, s_scan, totals);
    const long long before_tok = sums[0], before_free = sums[1], toks = totals[0], frees = totals[1], ents = totals[2];
    if (TABLES) {
      s_tok[tid] = before_tok;
      s_free[tid] = free_base + before_free;
      s_ent[tid] = sums[2];
      s_match[tid] = match_at;
      s_matches[tid] = (int)(matches < 0 ? 0 : matches > INT_MAX ? INT_MAX : matches);
      s_row[tid] = row;
      s_held[tid] = q.h;
      s_had[tid] = q.had;
      s_width[tid] = (int)width;
      if (blockIdx.x == (unsigned int)(r0 / N) % gridDim.x && r < a.R) {
        if (q.bad || q.need > width) raise_status(AIBX_ERR_RANGE);   // (without new tokens, too)
        a.tok_off[r] = tok_base + before_tok;
      }
    }
    if (COMMIT && blockIdx.x == (unsigned int)(r0 / N) % gridDim.x && r < a.R) a.kv_len[r] = q.h + q.n;
    if (TABLES) {
      __syncthreads();
      // Four tokens per thread at a time, so that their ids are on their way together: 32 apart where there are
      // many (a warp then takes 128 neighbours), else far apart, so that every thread gets its first one.
      const int all = (int)gridDim.x * N, slot = (int)blockIdx.x * N + tid;
      auto give = [&](auto wide, int apart, int from) {
        using X = decltype(wide);                          // of what counts tokens of this tile
        for (X i0 = (X)from; i0 < (X)toks; i0 += 4 * (X)all) {
          // the request of the warp's first token, which most of them share
          int k, had, width;
          X begin, next;                                   // its tokens
          int held;
          long long free_at;
          uint32_t* entries;
          auto enter = [&](int to) {
            k = to;
            begin = (X)s_tok[k];
            next = k + 1 < rows ? (X)s_tok[k + 1] : (X)toks;
            held = s_held[k];
            had = s_had[k];
            width = s_width[k];
            free_at = s_free[k] - had;
            entries = a.table + s_row[k];
          };
          enter(last_not_above<X>(s_tok, rows, apart == 32 ? i0 - (tid & 31) : i0));
          int p[4], off[4];
          uint32_t id[4];
          const uint32_t* src[4];
          uint32_t* dst[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const X i = i0 + (X)(u * apart);
            src[u] = nullptr;
            dst[u] = nullptr;
            p[u] = off[u] = 0;
            if (i >= (X)toks) continue;
            if (i >= next) enter(last_not_above<X>(s_tok, rows, i));
            p[u] = held + (int)(i - begin);
            const int blk = a.by_T.div(p[u]);
            off[u] = p[u] - blk * a.T;
            if (blk >= width) continue;
            if (blk >= had) {
              const long long f = free_at + blk;
              if (f < left) src[u] = a.free_ids + (start + f < a.capacity ? start + f : start + f - a.capacity);
              if (off[u] == 0) dst[u] = entries + blk;
            } else {
              src[u] = a.match ? matched(k, blk) : entries + blk;
            }
          }
#pragma unroll
          for (int u = 0; u < 4; ++u) id[u] = src[u] ? *src[u] : AIBX_NO_BLOCK;
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const X i = i0 + (X)(u * apart);
            const long long t = tok_base + (long long)i;
            if (i >= (X)toks) continue;
            if (dst[u]) *dst[u] = id[u];
            if (id[u] >= a.num_blocks && id[u] != AIBX_NO_BLOCK) raise_status(AIBX_ERR_RANGE);
            if (t >= a.n_tokens) continue;
            if (a.pos) a.pos[t] = p[u];
            if (a.slots) a.slots[t] = id[u] < a.num_blocks ? (int64_t)id[u] * a.T + off[u] : -1;
          }
        }
      };
      const int apart = toks > all ? 32 : all, from = toks > all ? (slot >> 5) * 128 + (slot & 31) : slot;
      if (toks < (1ll << 31) - 8ll * all)                  // (i0 goes at most 8 * all past it)
        give(0u, apart, from);
      else
        give(0ull, apart, from);
      for (long long e = slot; e < ents; e += all) {
        const int k = last_not_above<long long>(s_ent, rows, e);
        const int at = (int)(e - s_ent[k]);
        const uint32_t* from_match = matched(k, at);
        a.table[s_row[k] + at] = from_match ? *from_match : AIBX_NO_BLOCK;
      }
      __syncthreads();
    }
    tok_base += toks;
    free_base += frees;
  }
  if (blockIdx.x == 0 && tid == 0) {
    if (TABLES) {
      a.tok_off[a.R] = tok_base;
      if (free_base > left) raise_status_n(AIBX_ERR_FULL, (unsigned long long)(free_base - left));
      if ((a.pos || a.slots) && tok_base > a.n_tokens) raise_status(AIBX_ERR_RANGE);
    }
    if (COMMIT) *a.head_out = head + (free_base < left ? free_base : left);
  }
}

inline int32_t kv_tables(const aibx_kv_tables_t* t, int32_t R, cudaStream_t st) {
  if (!t || R < 0 || t->block_tokens <= 0 || t->table_stride < 0 || t->free_capacity < 0 || t->n_tokens < 0)
    return AIBX_ERR_INVALID;
  if (t->block_tokens > 65536) return AIBX_ERR_UNSUPPORTED;
  if (R == 0) return AIBX_OK;
  if (!t->d_held || !t->d_new || !t->d_free_ids || !t->d_free_head || !t->d_free_tail || !t->d_free_head_out ||
      !t->d_block_table || !t->d_tok_off || !t->d_kv_len || t->free_capacity == 0 ||
      (t->d_match_ids == nullptr) != (t->d_match_off == nullptr))
    return AIBX_ERR_INVALID;
  const uintptr_t four = reinterpret_cast<uintptr_t>(t->d_held) | reinterpret_cast<uintptr_t>(t->d_new) |
                         reinterpret_cast<uintptr_t>(t->d_free_ids) | reinterpret_cast<uintptr_t>(t->d_block_table) |
                         reinterpret_cast<uintptr_t>(t->d_kv_len) | reinterpret_cast<uintptr_t>(t->d_match_ids) |
                         reinterpret_cast<uintptr_t>(t->d_pos);
  const uintptr_t eight = reinterpret_cast<uintptr_t>(t->d_free_head) | reinterpret_cast<uintptr_t>(t->d_free_tail) |
                          reinterpret_cast<uintptr_t>(t->d_free_head_out) | reinterpret_cast<uintptr_t>(t->d_blk_off) |
                          reinterpret_cast<uintptr_t>(t->d_match_off) | reinterpret_cast<uintptr_t>(t->d_tok_off) |
                          reinterpret_cast<uintptr_t>(t->d_slots);
  if ((four & 3) || (eight & 7)) return AIBX_ERR_INVALID;
  // written by some threads while others read
  if (t->d_kv_len == t->d_new || t->d_pos == t->d_held || t->d_pos == t->d_new || t->d_block_table == t->d_match_ids ||
      t->d_block_table == t->d_free_ids || t->d_free_head_out == t->d_free_tail)
    return AIBX_ERR_INVALID;
  TablesArgs a;
  a.held = t->d_held;
  a.fresh = t->d_new;
  a.R = R;
  a.T = t->block_tokens;
  a.by_T = position_divisor(a.T);
  a.num_blocks = t->num_blocks;
  a.free_ids = t->d_free_ids;
  a.capacity = t->free_capacity;
  a.head = t->d_free_head;
  a.tail = t->d_free_tail;
  a.head_out = t->d_free_head_out;
  a.table = t->d_block_table;
  a.blk_off = t->d_blk_off;
  a.stride = t->table_stride;
  a.match = t->d_match_ids;
  a.match_off = t->d_match_off;
  a.tok_off = t->d_tok_off;
  a.kv_len = t->d_kv_len;
  a.pos = t->d_pos;
  a.slots = t->d_slots;
  a.n_tokens = t->n_tokens;
  // four tokens or matched entries per thread, as far as the host can tell
  const long long most = 2 * sm_count(), each = 4 * kTablesThreads;
  const double copies = !a.match ? 0.0 : a.blk_off ? 1e18 : (double)a.stride * R;
  const double want = ((double)a.n_tokens + copies) / each;
  const unsigned int grid = want >= (double)most ? (unsigned int)most : want > 1.0 ? (unsigned int)want + 1 : 1u;
  const bool apart = a.kv_len != a.held && a.head_out != a.head;
  if (grid == 1 || apart) {
    kv_tables_kernel<true, true><<<grid, kTablesThreads, 0, st>>>(a);
  } else {
    kv_tables_kernel<true, false><<<grid, kTablesThreads, 0, st>>>(a);
    kv_tables_kernel<false, true><<<1, kTablesThreads, 0, st>>>(a);
  }
  return launch_status();
}

// ------------------------------------------------------------------------------------------
// ancestors

struct TreeArgs {
  const int32_t* parent;
  const int64_t* tok_off;
  const int32_t* kv_len;
  unsigned long long* mask;
  int32_t* pos;
  long long n_tokens;
  int R;
};

constexpr int kTreeMaxWords = 8;
template <int W>
constexpr int kTreeThreads = W >= 6 ? 1024 : W >= 4 ? 512 : W >= 2 ? 256 : 64;

template <int W>
__global__ void __launch_bounds__(kTreeThreads<W>)
tree_masks_kernel(TreeArgs a) {
  constexpr int N = kTreeThreads<W>, kNodes = 64 * W, kV = W % 2 == 0 ? 2 : 1, kItems = W / kV;   // words at a time
  constexpr int kEach = (kNodes * kItems + N - 1) / N;     // such pieces of masks per thread
  struct alignas(8 * kV) Words {
    unsigned long long w[kV];
  };
  extern __shared__ __align__(16) unsigned long long s_mask[];   // [kNodes][W]
  short* s_up = reinterpret_cast<short*>(s_mask + kNodes * W);   // [kNodes]
  const int tid = threadIdx.x;
  for (int r = blockIdx.x; r < a.R; r += gridDim.x) {
    const long long tok0 = __ldg(a.tok_off + r);
    const long long end = min((long long)__ldg(a.tok_off + r + 1), a.n_tokens);
    if (tok0 < 0 || end <= tok0) continue;
    if (end - tok0 > kNodes) {
      if (tid == 0) raise_status(AIBX_ERR_RANGE);
      continue;
    }
    const int n = (int)(end - tok0);
    bool more = false;
    for (int i = tid; i < n; i += N) {
      const int p = __ldg(a.parent + tok0 + i);
      if (p >= i) raise_status(AIBX_ERR_RANGE);
      s_up[i] = (short)(p < 0 || p >= i ? -1 : p);
      more |= p >= 0 && p < i;
    }
    Words v[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int x = tid + e * N, i = x / kItems, w = (x - i * kItems) * kV;
#pragma unroll
      for (int y = 0; y < kV; ++y) v[e].w[y] = w + y == i >> 6 ? 1ull << (i & 63) : 0ull;
      if (x < n * kItems) *reinterpret_cast<Words*>(s_mask + x * kV) = v[e];
    }
    // A round: every node reads the mask of the one its `up` names, and that one's own; then all write.
    while (__syncthreads_or(more)) {
      int up[kEach];
      bool grown[kEach];
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int x = tid + e * N, i = x / kItems, w = x - i * kItems;
        const int j = x < n * kItems ? s_up[i] : -1;
        grown[e] = j >= 0;
        up[e] = -1;
        if (j < 0) continue;
        if (w * kV <= j >> 6) {                            // (beyond its own bit a mask is zero)
          const Words above = *reinterpret_cast<const Words*>(s_mask + (j * kItems + w) * kV);
#pragma unroll
          for (int y = 0; y < kV; ++y) v[e].w[y] |= above.w[y];
        }
        up[e] = s_up[j];
      }
      __syncthreads();
      more = false;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        if (!grown[e]) continue;
        const int x = tid + e * N, i = x / kItems;
        *reinterpret_cast<Words*>(s_mask + x * kV) = v[e];
        if (x == i * kItems) s_up[i] = (short)up[e];
        more |= up[e] >= 0;
      }
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int x = tid + e * N;
      if (x < n * kItems) {
#pragma unroll
        for (int y = 0; y < kV; ++y) a.mask[tok0 * W + x * kV + y] = v[e].w[y];
      }
    }
    if (a.pos) {
      const int base = (int)(__ldg(a.kv_len + r) - (__ldg(a.tok_off + r + 1) - tok0));
      for (int i = tid; i < n; i += N) {
        int above = -1;
#pragma unroll
        for (int w = 0; w < W; ++w) above += __popcll(s_mask[i * W + w]);
        a.pos[tok0 + i] = base + above;
      }
    }
    __syncthreads();
  }
}

template <int W>
inline int32_t launch_tree_masks(const TreeArgs& a, cudaStream_t st) {
  constexpr size_t smem = (size_t)64 * W * (8 * W + 2);    // at most 33 KB
  const long long most = (long long)sm_count() * 8;
  tree_masks_kernel<W><<<(unsigned int)(a.R < most ? a.R : most), kTreeThreads<W>, smem, st>>>(a);
  return launch_status();
}

inline int32_t tree_masks(const int32_t* parent, const int64_t* tok_off, const int32_t* kv_len, int32_t R,
                          int64_t n_tokens, int32_t words, uint64_t* mask, int32_t* pos, cudaStream_t st) {
  if (R < 0 || n_tokens < 0 || words <= 0) return AIBX_ERR_INVALID;
  if (words > kTreeMaxWords) return AIBX_ERR_UNSUPPORTED;
  if (R == 0 || n_tokens == 0) return AIBX_OK;
  if (!parent || !tok_off || !mask || (pos && !kv_len)) return AIBX_ERR_INVALID;
  if (((reinterpret_cast<uintptr_t>(parent) | reinterpret_cast<uintptr_t>(kv_len) | reinterpret_cast<uintptr_t>(pos)) & 3) ||
      ((reinterpret_cast<uintptr_t>(tok_off) | reinterpret_cast<uintptr_t>(mask)) & 7))
    return AIBX_ERR_INVALID;
  const void* in[] = {parent, tok_off, kv_len};
  for (const void* x : in)
    if (x && (x == mask || x == pos)) return AIBX_ERR_INVALID;
  const TreeArgs a = {parent, tok_off, kv_len, reinterpret_cast<unsigned long long*>(mask), pos, n_tokens, R};
  switch (words) {
    case 1: return launch_tree_masks<1>(a, st);
    case 2: return launch_tree_masks<2>(a, st);
    case 3: return launch_tree_masks<3>(a, st);
    case 4: return launch_tree_masks<4>(a, st);
    case 5: return launch_tree_masks<5>(a, st);
    case 6: return launch_tree_masks<6>(a, st);
    case 7: return launch_tree_masks<7>(a, st);
    default: return launch_tree_masks<8>(a, st);
  }
}

}  // namespace aibx
