// What the attention kernels share: the split of the work among CTAs, masks, and the join of
// what CTAs leave unfinished.
#pragma once

#include "qlin_attention.h"

namespace qlin {

namespace {

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

// The tiles of a sequence, and its items.
struct Work {
  int64_t tiles, items;
};
template <int kRows, int kTile>
__device__ __forceinline__ Work seq_work(const AttnParams& p, const CacheSeq& s) {
  const int64_t tiles = (s.keys + kTile - 1) / kTile;
  const int64_t items = tiles > 0 ? ((int64_t)s.fresh * p.group + kRows - 1) / kRows * p.heads : 0;
  return {items * tiles, items};
}

// The CTA's run of units and the cursor at its begin; the same in all threads.  An item's units are
// its tiles and behind them `gap` more that nobody works on: what its begin and end cost.
struct Run {
  int64_t begin, end;
  Split split;
  int gap;
};
struct RunScratch {   // in shared memory
  Work warp_sum[32], warp_all[32];
  CacheSeq s;
  int64_t at;
  int b;
};

// (kLast: the cursor at its last unit.)  Up to kThreads sequences take one pass over the counts
// and two barriers; more, a second pass.
template <int kRows, int kTile, int kThreads, bool kLast = false>
__device__ __forceinline__ Run find_run(const AttnParams& p, Cursor& c, int cta, int ctas, RunScratch& scratch) {
  constexpr int kWarps = kThreads / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Run r{0, 0, {0, 0}, 0};
  CacheSeq mine{};
  Work first{0, 0}, all{0, 0};
  bool bad = false;
  for (int b = threadIdx.x; b < p.sequences; b += kThreads) {
    const CacheSeq s = read_seq<kRows, kTile>(p, b);
    bad |= s.bad;
    const Work u = seq_work<kRows, kTile>(p, s);
    if (b < kThreads) {
      first = u;
      mine = s;
    }
    all = {all.tiles + u.tiles, all.items + u.items};
  }
  if (bad && cta == 0) atomicExch(p.err, kErrInvalid);
  // the sequences up to this thread's, and all
  auto scan = [&](Work u) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t t = __shfl_up_sync(0xFFFFFFFFu, u.tiles, o), n = __shfl_up_sync(0xFFFFFFFFu, u.items, o);
      if (lane >= o) u = {u.tiles + t, u.items + n};
    }
    return u;
  };
  Work incl = scan(first);
  if (lane == 31) scratch.warp_sum[warp] = incl;
  if (p.sequences > kThreads) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      all.tiles += __shfl_xor_sync(0xFFFFFFFFu, all.tiles, o);
      all.items += __shfl_xor_sync(0xFFFFFFFFu, all.items, o);
    }
    if (lane == 0) scratch.warp_all[warp] = all;
  }
  __syncthreads();
  auto plus = [](const Work& a, const Work& b) { return Work{a.tiles + b.tiles, a.items + b.items}; };
  Work before{0, 0}, run{0, 0};
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before = plus(before, scratch.warp_sum[w]);
    run = plus(run, scratch.warp_sum[w]);
  }
  Work total = run;
  if (p.sequences > kThreads) {
    total = {0, 0};
    for (int w = 0; w < kWarps; ++w) total = plus(total, scratch.warp_all[w]);
  }
  if (total.tiles == 0) return r;
  // (with fewer tiles per CTA a gap would rather give somebody one more of them)
  r.gap = total.tiles >= (int64_t)p.item_cost * ctas ? p.item_cost : 0;
  auto units = [&](const Work& w) { return w.tiles + w.items * r.gap; };
  const int64_t working = split_ctas(units(total), ctas, p.least);
  if (cta >= working) return r;
  r.split = split_evenly(units(total), working);
  r.begin = split_begin(r.split, cta);
  r.end = split_begin(r.split, cta + 1);
  const int64_t want = kLast ? r.end - 1 : r.begin;
  // (want: in the thread's own sequence, which ends `incl` behind the units before its warp?)
  auto look = [&](int b, const Work& own) {
    const int64_t end = units(plus(before, incl)), begin = end - units(own);
    if (begin <= want && want < end) {
      scratch.b = b;
      scratch.s = mine;
      scratch.at = want - begin;
    }
  };
  look(threadIdx.x, first);
  for (int b0 = kThreads; units(run) <= want; b0 += kThreads) {   // (the total above want: some sequence has it)
    const int b = b0 + threadIdx.x;
    Work u{0, 0};
    if (b < p.sequences) {
      mine = read_seq<kRows, kTile>(p, b);
      u = seq_work<kRows, kTile>(p, mine);
    }
    incl = scan(u);
    __syncthreads();   // warp_sum's last readers
    if (lane == 31) scratch.warp_sum[warp] = incl;
    __syncthreads();
    before = run;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) before = plus(before, scratch.warp_sum[w]);
      run = plus(run, scratch.warp_sum[w]);
    }
    look(b, u);
  }
  __syncthreads();
  c.b = scratch.b;
  c.s = scratch.s;
  size_seq<kRows, kTile>(p, c);
  const int64_t at = scratch.at;
  const int64_t per = c.tiles + r.gap, item = div_small(at, per), tile = at - item * per;
  c.tile = (int)min(tile, (int64_t)(c.tiles - 1));
  c.h = (int)div_small(item, c.row_tiles);
  c.rt = (int)(item - (int64_t)c.h * c.row_tiles);
  // in a gap: on to the next item, or back to the last tile
  if (tile >= c.tiles) {
    if (kLast) {
      r.end -= tile - c.tile;
    } else {
      r.begin += per - tile;
      if (r.begin < r.end) advance<kRows, kTile>(p, c);
    }
  }
  return r;
}

// Whether new token t of a sequence (number `token` of the call) sees new token i.
__device__ __forceinline__ bool sees(const AttnParams& p, int64_t token, int t, int64_t i) {
  if (p.mask == nullptr) return i <= t;
  const int64_t w = i >> 6;
  return w < p.mask_words && ((p.mask[token * p.mask_token + w] >> (i & 63)) & 1u) != 0u;
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

// Rows row0 .. row0 + rows - 1 of an item, whose parts the CTAs first to last left in the
// workspace, joined in the order of the keys.  Called by all of kThreads threads of a CTA; stat:
// `rows` of them in shared memory.
template <int kRows, int kD, int kThreads>
__device__ __forceinline__ void join_parts(const AttnParams& p, const Cursor& c, int first, int last, float v_scale,
                                           int row0, int rows, float2* stat) {
  const int thread = (int)threadIdx.x;
  for (int i = thread; i < rows; i += kThreads) {
    float m = -INFINITY, l = 0.0f;
#pragma unroll 4
    for (int q = first; q <= last; ++q) {
      const float2 ml = __ldcg(&p.part_ml[part_row<kRows>(q, first, row0 + i)]);
      const float now = fmaxf(m, ml.x), base = now == -INFINITY ? 0.0f : now;
      l = fmaf(l, exp2_fast(m - base), ml.y * exp2_fast(ml.x - base));
      m = now;
    }
    stat[i] = make_float2(m, l);
  }
  __syncthreads();
  const int items = rows * (p.head_dim / 4);
  constexpr int kAtOnce = 4;
  for (int i0 = thread; i0 < items; i0 += kThreads * kAtOnce) {
    float4 o[kAtOnce];
    float base[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = min(i0 + k * kThreads, items - 1);
      const float m = stat[i % rows].x;
      base[k] = m == -INFINITY ? 0.0f : m;
      o[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
#pragma unroll 2
    for (int q = first; q <= last; ++q) {
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int i = min(i0 + k * kThreads, items - 1), row = row0 + i % rows;
        const float f = exp2_fast(__ldcg(&p.part_ml[part_row<kRows>(q, first, row)].x) - base[k]);
        const float4 v = __ldcg(part_sums<kRows, kD>(p, part_row<kRows>(q, first, 0), row, i / rows * 4));
        o[k] = make_float4(fmaf(v.x, f, o[k].x), fmaf(v.y, f, o[k].y), fmaf(v.z, f, o[k].z), fmaf(v.w, f, o[k].w));
      }
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = i0 + k * kThreads;
      if (i >= items) break;
      const int row = i % rows, d = i / rows * 4;
      const float2 ml = stat[row];
      const int64_t r = (int64_t)c.rt * kRows + row0 + row;
      const int64_t token = c.s.first + r / p.group;
      const int head = c.h * p.group + (int)(r % p.group);
      const float inv = ml.y == 0.0f ? 0.0f : v_scale / ml.y;
      store_out4(p, token, head, d, make_float4(o[k].x * inv, o[k].y * inv, o[k].z * inv, o[k].w * inv));
      if (p.lse != nullptr && d == 0) p.lse[token * p.lse_token + head] = log_sum(ml.x, ml.y);
    }
  }
}

}  // namespace

}  // namespace qlin
