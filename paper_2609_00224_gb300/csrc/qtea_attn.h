// Parameters and work division shared by the attention kernels.
//
// The work of a call is a sequence of units: for every sequence, cache head and tile of query rows
// (an item), the stretches of unit_keys keys that the tile sees. The grid's CTAs take equal runs of
// that sequence, whatever the lengths are, so a ragged batch loads every SM alike and a single long
// sequence is split over all of them. An item that several CTAs share is joined by the last of them
// to finish: the others leave (O, m, l) in the workspace. Which CTAs share an item follows from
// the unit numbers alone, and they are joined in that order, so results do not depend on timing.
#pragma once

#include "qtea_kv_internal.h"

namespace qtea {

constexpr int kAttnHeaderBytes = 8192;  // workspace: the status word, then one counter per CTA
constexpr int kAttnCounters = 1024;     // at most this many CTAs
constexpr int kAttnMaxGroup = 32;       // query heads of one cache head

struct AttnParams {
  KvView kv;
  KvBatchView b;
  const __half* q;
  __half* out;
  float* lse;
  long long q_ld, out_ld;
  int q_heads, group;
  float scale_log2;  // scale * log2(e)
  int window;
  int tile_tokens;  // tokens of an item: the rows of a tile / group
  int unit_shift;   // log2 of a unit's keys
  int min_units;    // the least units worth a CTA of their own
  int* status;
  unsigned* counters;
  float* slots;     // [grid][2] partial results
};

cudaError_t launch_attn_chunk(const qtea_kv* kv, const AttnParams& p, cudaStream_t st);
size_t attn_chunk_floats(int sm_count);  // of one partial result for each CTA
cudaError_t launch_attn_rows(const qtea_kv* kv, const AttnParams& p, cudaStream_t st);
size_t attn_rows_floats(int sm_count);  // of one partial result for each CTA

#ifdef __CUDACC__

// One sequence of the batch.
struct AttnSeq {
  int q0, n, base;  // first row, new tokens, position of the first
};

__device__ __forceinline__ AttnSeq attn_seq(const AttnParams& p, int s) {
  AttnSeq a;
  a.q0 = min(max(__ldg(p.b.q_start + s), 0), p.b.n_tokens);
  const int q1 = min(max(__ldg(p.b.q_start + s + 1), a.q0), p.b.n_tokens);
  a.base = kv_context(p.b, p.kv, s) - (q1 - a.q0);
  a.n = min(q1 - a.q0, p.b.max_q);
  return a;
}

// The units of tile t of a sequence: first unit and their number (at least one, for tiles that see
// nothing have zeros to write).
__device__ __forceinline__ int2 attn_tile(const AttnParams& p, const AttnSeq& a, int t) {
  const int i0 = t * p.tile_tokens, i1 = min(a.n, i0 + p.tile_tokens) - 1;
  const int hi = a.base + i1 + 1;
  const int lo = p.window > 0 ? max(0, a.base + i0 - p.window + 1) : 0;
  const int u0 = lo >> p.unit_shift;
  const int u1 = (max(hi, 0) + (1 << p.unit_shift) - 1) >> p.unit_shift;
  return make_int2(u0, max(u1 - u0, 1));
}

__device__ __forceinline__ int attn_tiles(const AttnParams& p, const AttnSeq& a) {
  return (a.n + p.tile_tokens - 1) / p.tile_tokens;
}

// Units before each sequence, into shared memory: prefix[0 .. n_seqs] (every thread of the CTA
// calls it; it ends with a barrier).
__device__ __forceinline__ void attn_prefix(const AttnParams& p, long long* prefix) {
  const int n = p.b.n_seqs, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (p.b.max_q <= p.tile_tokens) {  // one tile a sequence: a thread each
    for (int s = threadIdx.x; s < n; s += blockDim.x) {
      const AttnSeq a = attn_seq(p, s);
      prefix[s + 1] = a.n > 0 ? (long long)attn_tile(p, a, 0).y * p.kv.heads : 0;
    }
  } else {  // a warp each
    for (int s = warp; s < n; s += blockDim.x >> 5) {
      const AttnSeq a = attn_seq(p, s);
      const int tiles = attn_tiles(p, a);
      long long sum = 0;
      for (int t = lane; t < tiles; t += 32) sum += attn_tile(p, a, t).y;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (lane == 0) prefix[s + 1] = sum * p.kv.heads;
    }
  }
  __syncthreads();
  if (warp == 0) {
    long long before = 0;
    if (lane == 0) prefix[0] = 0;
    for (int s0 = 0; s0 < n; s0 += 32) {
      long long v = s0 + lane < n ? prefix[s0 + lane + 1] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
      }
      if (s0 + lane < n) prefix[s0 + lane + 1] = before + v;
      before += __shfl_sync(0xffffffffu, v, 31);
    }
  }
  __syncthreads();
}

// How the units are divided: CTA c of `ctas` takes [first(c), first(c + 1)).
struct AttnSplit {
  long long total;
  int ctas;
  __device__ __forceinline__ long long first(int c) const { return total * c / ctas; }
  __device__ __forceinline__ int cta_of(long long u) const { return (int)(((u + 1) * ctas - 1) / total); }
};

__device__ __forceinline__ AttnSplit attn_split(const AttnParams& p, const long long* prefix) {
  AttnSplit d;
  d.total = prefix[p.b.n_seqs];
  const long long worth = (d.total + p.min_units - 1) / p.min_units;
  d.ctas = (int)min((long long)gridDim.x, max(worth, 1LL));
  return d;
}

// A CTA's next stretch of one item.
struct AttnItem {
  AttnSeq seq;
  int s, head, tile;
  int unit0;            // the stretch's first unit, in units from the start of the sequence's keys
  int units;            // its units
  long long item_first; // number of the item's first unit in the call
  int item_units;       // all of the item's units
};

// The item that holds unit `cur`, and the part of it in [cur, end). Every lane of a warp calls it.
__device__ __forceinline__ AttnItem attn_item(const AttnParams& p, const long long* prefix, long long cur,
                                              long long end) {
  AttnItem it;
  int lo = 0, hi = p.b.n_seqs;
  while (hi - lo > 1) {  // the last sequence whose units start at or before cur (it is not empty)
    const int mid = (lo + hi) >> 1;
    if (prefix[mid] <= cur) lo = mid;
    else hi = mid;
  }
  it.s = lo;
  it.seq = attn_seq(p, lo);
  const long long per_head = (prefix[lo + 1] - prefix[lo]) / p.kv.heads;
  const long long in_seq = cur - prefix[lo];
  it.head = (int)(in_seq / per_head);
  long long rem = in_seq - it.head * per_head;
  int2 u = attn_tile(p, it.seq, 0);
  it.tile = 0;
  if (p.b.max_q > p.tile_tokens) {
    const int lane = threadIdx.x & 31, tiles = attn_tiles(p, it.seq);
    for (int t0 = 0;; t0 += 32) {
      const int t = t0 + lane;
      const int2 mine = t < tiles ? attn_tile(p, it.seq, t) : make_int2(0, 0);
      long long v = mine.y;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long w = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += w;
      }
      const unsigned past = __ballot_sync(0xffffffffu, v > rem);
      if (past || t0 + 32 >= tiles) {
        const int at = past ? __ffs(past) - 1 : 31;
        it.tile = t0 + at;
        u.x = __shfl_sync(0xffffffffu, mine.x, at);
        u.y = __shfl_sync(0xffffffffu, mine.y, at);
        rem -= __shfl_sync(0xffffffffu, v, at) - u.y;
        break;
      }
      rem -= __shfl_sync(0xffffffffu, v, 31);
    }
  }
  it.item_first = cur - rem;
  it.item_units = u.y;
  it.unit0 = u.x + (int)rem;
  it.units = (int)min((long long)(u.y - rem), end - cur);
  return it;
}
#endif

}  // namespace qtea
