// What the attention kernels share: the split of the work among CTAs, masks, and the join of
// what CTAs leave unfinished.
#pragma once

#include "qlin_attention.h"

namespace qlin {

namespace {

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}

// A place in the work: tile `tile` of the item (b, h, rt).
struct Cursor {
  CacheSeq s;
  int b, h, rt, tile, tiles, row_tiles;
};

template <int kRows, int kTile>
__device__ __forceinline__ CacheSeq read_seq(const AttnParams& p, int b) {
  return cache_seq(p.q_start[b], p.q_start[b + 1], p.cached[b], p.tokens, p.page_size, p.table_width);
}

template <int kRows, int kTile>
__device__ __forceinline__ void size_seq(const AttnParams& p, Cursor& c) {
  c.tiles = (int)((c.s.keys + kTile - 1) / kTile);
  c.row_tiles = (int)(((int64_t)c.s.fresh * p.group + kRows - 1) / kRows);
}

template <int kRows, int kTile>
__device__ __forceinline__ void open_seq(const AttnParams& p, Cursor& c) {
  c.s = read_seq<kRows, kTile>(p, c.b);
  size_seq<kRows, kTile>(p, c);
}

// The next tile; past the last sequence the cursor stays at its end.
template <int kRows, int kTile>
__device__ __forceinline__ void advance(const AttnParams& p, Cursor& c) {
  if (++c.tile < c.tiles) return;
  c.tile = 0;
  if (++c.rt < c.row_tiles) return;
  c.rt = 0;
  if (++c.h < p.heads) return;
  c.h = 0;
  while (++c.b < p.sequences) {
    open_seq<kRows, kTile>(p, c);
    if (c.s.fresh > 0 && c.s.keys > 0) return;
  }
}

// A sequence's units: those of an item are its tiles and behind them item_cost more, which nobody
// works on, for its begin and end.
template <int kRows, int kTile>
__device__ __forceinline__ int64_t seq_units(const AttnParams& p, const CacheSeq& s) {
  const int64_t tiles = (s.keys + kTile - 1) / kTile;
  return tiles == 0 ? 0 : ((int64_t)s.fresh * p.group + kRows - 1) / kRows * p.heads * (tiles + p.item_cost);
}

// The CTA's run of units and the cursor at its begin; the same in all threads.
struct Run {
  int64_t begin, end;
  Split split;
};
struct RunScratch {   // in shared memory
  int64_t warp_sum[32], warp_all[32];
  CacheSeq s;
  int64_t at;
  int b;
};

// Up to kThreads sequences take one pass over the counts
// and two barriers; more, a second pass.
template <int kRows, int kTile, int kThreads>
__device__ __forceinline__ Run find_run(const AttnParams& p, Cursor& c, int cta, int ctas, RunScratch& scratch) {
  constexpr int kWarps = kThreads / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Run r{0, 0, {0, 0}};
  CacheSeq mine{};
  int64_t first = 0, all = 0;
  bool bad = false;
  for (int b = threadIdx.x; b < p.sequences; b += kThreads) {
    const CacheSeq s = read_seq<kRows, kTile>(p, b);
    bad |= s.bad;
    const int64_t u = seq_units<kRows, kTile>(p, s);
    if (b < kThreads) {
      first = u;
      mine = s;
    }
    all += u;
  }
  if (bad && cta == 0) report_invalid(p.err);
  // the sequences up to this thread's, and all
  auto scan = [&](int64_t u) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t n = __shfl_up_sync(0xFFFFFFFFu, u, o);
      if (lane >= o) u += n;
    }
    return u;
  };
  int64_t incl = scan(first);
  if (lane == 31) scratch.warp_sum[warp] = incl;
  if (p.sequences > kThreads) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, o);
    if (lane == 0) scratch.warp_all[warp] = all;
  }
  __syncthreads();
  int64_t base = 0, run = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) base += scratch.warp_sum[w];
    run += scratch.warp_sum[w];
  }
  int64_t total = run;
  if (p.sequences > kThreads) {
    total = 0;
    for (int w = 0; w < kWarps; ++w) total += scratch.warp_all[w];
  }
  if (total == 0) return r;
  const int64_t working = split_ctas(total, ctas, p.least);
  if (cta >= working) return r;
  r.split = split_evenly(total, working);
  r.begin = split_begin(r.split, cta);
  r.end = split_begin(r.split, cta + 1);
  const int64_t want = r.begin;
  auto found = [&](int b, const CacheSeq& s, int64_t before) {
    scratch.b = b;
    scratch.s = s;
    scratch.at = want - before;
  };
  if (base + incl - first <= want && want < base + incl) found(threadIdx.x, mine, base + incl - first);
  for (int b0 = kThreads; run <= want; b0 += kThreads) {   // (total above want: some sequence has it)
    const int b = b0 + threadIdx.x;
    int64_t u = 0;
    if (b < p.sequences) {
      mine = read_seq<kRows, kTile>(p, b);
      u = seq_units<kRows, kTile>(p, mine);
    }
    incl = scan(u);
    __syncthreads();   // warp_sum's last readers
    if (lane == 31) scratch.warp_sum[warp] = incl;
    __syncthreads();
    base = run;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) base += scratch.warp_sum[w];
      run += scratch.warp_sum[w];
    }
    if (base + incl - u <= want && want < base + incl) found(b, mine, base + incl - u);
  }
  __syncthreads();
  c.b = scratch.b;
  c.s = scratch.s;
  size_seq<kRows, kTile>(p, c);
  const int64_t at = scratch.at, per = c.tiles + p.item_cost, item = div_small(at, per), tile = at - item * per;
  c.tile = (int)min(tile, (int64_t)(c.tiles - 1));
  c.h = (int)div_small(item, c.row_tiles);
  c.rt = (int)(item - (int64_t)c.h * c.row_tiles);
  if (tile >= c.tiles) {   // behind an item's tiles: on to the next item
    r.begin += per - tile;
    if (r.begin < r.end) advance<kRows, kTile>(p, c);
  }
  return r;
}

// The first key that not every row sees: the first new one, or where the table ends before it the one
// behind its last (counts that pass the table's room).
__device__ __forceinline__ int64_t first_unseen(const CacheSeq& s) { return min(s.cached, s.keys); }

// Whether new token t of a sequence (number `token` of the call) sees new token i.
__device__ __forceinline__ bool sees(const AttnParams& p, int64_t token, int t, int64_t i) {
  if (p.mask == nullptr) return i <= t;
  const int64_t w = i >> 6;
  return w < p.mask_words && ((p.mask[token * p.mask_token + w] >> (i & 63)) & 1u) != 0u;
}

// What a row of Q is multiplied by where its scores' factor takes the keys' scale without its sign, so
// that the maximum stays one: the sign is Q's, and a scale of infinity or NaN makes the scores NaN (not
// those of keys that the row does not see).
__device__ __forceinline__ float signed_factor(float f, float k_scale) {
  return fabsf(k_scale) < INFINITY ? copysignf(f, k_scale) : __uint_as_float(0x7FFFFFFFu);
}

__device__ __forceinline__ void store_out4(const AttnParams& p, int64_t token, int head, int d, float4 v) {
  uint16_t* const y = p.out + token * p.out_token + head * p.out_head + d;
  const uint2 w = p.fp16 ? make_uint2(pack_f16x2(v.x, v.y), pack_f16x2(v.z, v.w))
                         : make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
  *reinterpret_cast<uint2*>(y) = w;
}

__device__ __forceinline__ float log_sum(float m, float l) {   // m in powers of two
  return l > 0.0f || l != l ? fmaf(m, 0.693147181f, logf(l)) : -INFINITY;
}

// x as a condition that the compiler does not know before this place, so that it guards a few
// instructions: one that it knows before the loads became a branch for each part of a join (one token
// over 1000 keys 10.9 us, so 9.8; 64 decodes 144.2, 141.2).
__device__ __forceinline__ bool known_here(bool x) {
  uint32_t r = x ? 1u : 0u;
  asm volatile("" : "+r"(r));
  return r != 0u;
}

// An item's parts in the workspace: CTA first's is its second, all others' their first.
template <int kRows>
__device__ __forceinline__ int64_t part_row(int cta, int first, int row) {
  return (int64_t)(2 * cta + (cta == first ? 1 : 0)) * kRows + row;
}

// A part's sums lie [kD / 4][kRows] in fours: threads with a row each write and read whole lines.
template <int kRows, int kD>
__device__ __forceinline__ float4* part_sums(const AttnParams& p, int64_t part_row0, int row, int d) {
  return reinterpret_cast<float4*>(p.part + part_row0 * kD) + (int64_t)(d / 4) * kRows + row;
}

}  // namespace

}  // namespace qlin
