// Attention of many rows over a paged cache of 16-bit keys and values, on the tensor cores'
// own memory (tcgen05): drafts and runs of tokens whose rows per KV head (query heads of its
// group times new tokens) make the products the work.
//
// A CTA takes 256 rows of an item and tiles of 128 keys, in two streams that take turns on
// the tensor cores: while one stream's softmax runs, the other's products do.  With more than
// 128 rows the streams are the rows' halves over the same keys; with 128 or fewer, even and
// odd tiles over the same rows, joined at the end.  Per stream and tile:
//   S = Q K^T     tcgen05 from shared memory (K's pages by TMA, 128-byte swizzle) into 128 columns
//   P = 2^(S - m) a thread per row: 128 scores in registers, P as 16-bit over S's columns
//   O += P V      A from tensor memory, V as it lies (keys x elements: an MN-major B)
// The running maximum moves only when it rises by more than 2^8, so O is rarely rescaled; P
// stays below 2^8 and the sums in fp32 (both fine in 16 bits: a P's rounding is relative).
//   Per tile of 256 rows and 128 keys of 128: 2048 cycles of MMAs, 2048 of exponentials (16 a
// cycle and SM), 64 KB of keys and values, about 2850 cycles of an SM's share of HBM.
// Roles: warp 0 loads, warp 1 issues MMAs, warps 4-7 and 8-11 are the streams' softmax.
// Tiles with new tokens are masked, and V's slots behind the last key and values that are
// not finite are zeroed in shared memory: 0 times them would reach rows that do not see them.
// (Rows that do see such a value take it at the end.)
#include "qlin_attention_work.cuh"

namespace qlin {

namespace {

constexpr int kRows = 256, kTile = 128;
constexpr int kThreads = 384, kSoftWarp0 = 4;
constexpr int kRoleRegs = 56, kSoftRegs = 224;
constexpr float kSlack = 8.0f;   // powers of two that a score may exceed the kept maximum by
constexpr int kBadRing = 16;     // tiles whose bad pages are remembered

template <int kDC>   // chunks of 64 elements of a head
struct TileCfg {
  static constexpr int kChunk = kTile * 128;          // 64 elements of 128 keys or rows
  static constexpr int kSlot = kDC * kChunk;          // a tile of K or V, or 128 rows of Q
  static constexpr int kSlots = kDC == 1 ? 10 : 5;
  static constexpr int kQBytes = 2 * kSlot;
  static constexpr int kBarrierBytes = 256;
  static constexpr int kSmem = 1024 + kQBytes + kSlots * kSlot + kBarrierBytes;
  static_assert((2 * kSlots + 8) * 8 <= kBarrierBytes && kSmem <= 232448 - 1536, "shared memory (static: 1.3 KB)");
};

struct TileParams {
  AttnParams a;
  int box_rows, boxes;   // keys of a TMA box, boxes of a tile
  uint64_t timeout_ns;
};

// O[tmem] (+)= P[tmem] V: A from tensor memory, 16-bit.
__device__ __forceinline__ void mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                           uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// V as B operand: 64 elements of a key are 128 swizzled bytes (the N direction), 8 keys a
// group of 1024 bytes, the next 64 elements a chunk further.
__device__ __forceinline__ uint64_t sdesc_v(uint32_t saddr, uint32_t chunk_bytes) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr >> 4) & 0x3FFFu);
  d |= (uint64_t)(chunk_bytes >> 4) << 16;   // between chunks of 64 elements
  d |= (uint64_t)(1024 >> 4) << 32;          // between groups of 8 keys
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// Where in the order of loads a segment's tiles lie (n tiles; K and V of each).  Rows in two
// halves: K0 V0 K1 V1 ...  Tiles in turn: K0 K1 V0 K2 V1 K3 ...: each as the MMAs take them.
__device__ __forceinline__ int k_pos(bool halves, int j) { return halves ? 2 * j : j < 2 ? j : 2 * j - 1; }
__device__ __forceinline__ int v_pos(bool halves, int j, int n) { return halves ? 2 * j + 1 : min(2 * j + 2, n + j); }

// A run's pieces: consecutive tiles of one item.
struct Segment {
  int first, n;      // tiles
  bool halves;
};
__device__ __forceinline__ Segment segment_at(const AttnParams& p, const Cursor& c, int64_t unit, int64_t end) {
  const int64_t rows = (int64_t)c.s.fresh * p.group - (int64_t)c.rt * kRows;
  return {c.tile, (int)min((int64_t)(c.tiles - c.tile), end - unit), rows > 128};
}
__device__ __forceinline__ void skip_segment(const AttnParams& p, Cursor& c, const Segment& s) {
  c.tile += s.n - 1;
  advance<kRows, kTile>(p, c);
}

// 32 bits of a row's mask from new token i on (negative ones are cached tokens: seen).
__device__ __forceinline__ uint32_t mask_window(const uint64_t* m, int words, int64_t i) {
  if (i <= -32) return 0xFFFFFFFFu;
  const int n = i < 0 ? (int)-i : 0;
  const int64_t at = i + n;
  const int64_t w = at >> 6;
  const int s = (int)(at & 63);
  uint64_t v = w < words ? m[w] >> s : 0ull;
  if (s > 32 && w + 1 < words) v |= m[w + 1] << (64 - s);
  return n == 0 ? (uint32_t)v : ((uint32_t)v << n) | ((1u << n) - 1u);
}
// The first n of 32 (n may be negative or large).
__device__ __forceinline__ uint32_t first_bits(int64_t n) {
  return n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << (int)n) - 1u;
}

// Which keys of 32 a row (new token t, number `token` of the call) sees, from key `key` on.
__device__ __forceinline__ uint32_t seen_bits(const AttnParams& p, const CacheSeq& s, int64_t token, int t, int64_t key) {
  const uint32_t in = first_bits(s.keys - key);
  if (p.mask == nullptr) return in & first_bits(s.cached + t + 1 - key);
  return in & mask_window(p.mask + token * p.mask_token, p.mask_words, key - s.cached);
}

template <bool kF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return kF16 ? pack_f16x2(lo, hi) : pack_bf16x2(lo, hi);
}

template <bool kF16, int kDC>
__global__ void __launch_bounds__(kThreads, 1)
    attn_tiles_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                      const TileParams tp) {
  using C = TileCfg<kDC>;
  constexpr int kD = 64 * kDC;
  const AttnParams& p = tp.a;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem =
      reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* const q_smem = smem;
  uint8_t* const ring = smem + C::kQBytes;
  uint64_t* const full = reinterpret_cast<uint64_t*>(ring + C::kSlots * C::kSlot);
  uint64_t* const empty = full + C::kSlots;
  uint64_t* const s_full = empty + C::kSlots;    // per stream: scores are there (and its products before done)
  uint64_t* const p_ready = s_full + 2;          // per stream: P is there
  uint64_t* const o_done = p_ready + 2;          // per stream: the segment's last product is done
  uint64_t* const q_ready = o_done + 2;
  uint64_t* const mma_done = q_ready + 1;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_word;
  __shared__ unsigned bad_pages[kBadRing];       // of K tiles in order
  __shared__ int odd_values;
  __shared__ unsigned last_flag;
  __shared__ float2 other_ml[128];

  const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kSlots; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&p_ready[i], 4);
      mbar_init(&o_done[i], 1);
    }
    mbar_init(q_ready, 8);
    mbar_init(mma_done, 1);
    abort_word = 0;
    odd_values = 0;
    mbar_fence_init();
  }
  if (warp == 0 && lane < 2) prefetch_tmap(lane == 0 ? &tmap_k : &tmap_v);
  if (warp == 1) tmem_alloc(&tmem_slot, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, tmem_slot, 0);
  const uint32_t s_tmem = tmem, o_tmem = tmem + 256;   // stream s: 128 columns further
  const WaitCtl ctl{&abort_word, p.err, tp.timeout_ns};
  grid_dep_wait();
  grid_dep_launch();
  Cursor cur;
  const Run run = find_run<kRows, kTile, kThreads>(p, cur);

  auto slot_of = [&](int64_t pos) { return (int)(pos % C::kSlots); };
  auto phase_of = [&](int64_t pos) { return (uint32_t)(pos / C::kSlots) & 1u; };

  if (warp < kSoftWarp0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRoleRegs));
    if (warp == 0) {
      // ---- loads: a lane per page of the tile ----
      int64_t base = 0, tiles_done = 0;   // loads and K tiles before this segment
      int64_t issued = 0;
      bool ok = true;
      for (int64_t unit = run.begin; unit < run.end && ok;) {
        const Segment sg = segment_at(p, cur, unit, run.end);
        // load i of the segment: tile j of K or V, and the lane's page of it
        struct Load {
          bool is_v, in;
          int j, at, page;
        };
        auto locate = [&](int i) {
          Load d{};
          if (sg.halves) {
            d.is_v = (i & 1) != 0;
            d.j = i >> 1;
          } else if (i < 2 && i < sg.n) {
            d.j = i;
          } else if (sg.n == 1) {
            d.is_v = true;
          } else {
            // V0 K2 V1 K3 ... with V alone once K is through
            d.is_v = (i & 1) == 0 || (i >> 1) + 1 >= sg.n;
            d.j = !d.is_v ? (i + 1) >> 1 : (i & 1) == 0 ? (i - 2) >> 1 : i - sg.n;
          }
          const int64_t key = (int64_t)(sg.first + d.j) * kTile + lane * tp.box_rows;
          int index = 0;
          d.in = lane < tp.boxes && key < cur.s.keys && cache_place(key, p.page_size, p.table_width, &index, &d.at);
          d.page = d.in ? p.table[cur.b * p.table_stride + index] : 0;
          return d;
        };
        Load next = locate(0);
        for (int i = 0; i < 2 * sg.n; ++i) {
          const Load d = next;
          if (i + 1 < 2 * sg.n) next = locate(i + 1);   // (the table's entry on its way while this load waits)
          const bool is_v = d.is_v;
          const int j = d.j;
          const int64_t pos = base + i;
          const int slot = slot_of(pos);
          const bool bad = d.in && (d.page < 0 || d.page >= p.pages);
          const unsigned bads = __ballot_sync(0xFFFFFFFFu, bad);
          if (bad) atomicExch(p.err, kErrInvalid);
          const int page = !d.in || bad ? p.pages : d.page;   // past the last: zeros
          const int at = !d.in || bad ? 0 : d.at;
          if (!mbar_wait_warp(&empty[slot], phase_of(pos) ^ 1u, ctl)) {
            ok = false;
            break;
          }
          if (lane == 0) {
            if (!is_v) *(volatile unsigned*)&bad_pages[(tiles_done + j) % kBadRing] = bads;
            mbar_arrive_expect_tx(&full[slot], C::kSlot);
          }
          __syncwarp();
          if (lane < tp.boxes) {
            uint8_t* const dst = ring + slot * C::kSlot + lane * tp.box_rows * 128;
#pragma unroll
            for (int c = 0; c < kDC; ++c)
              tma_load_4d(dst + c * C::kChunk, is_v ? &tmap_v : &tmap_k, smem_u32(&full[slot]), 64 * c, at, cur.h, page);
          }
          __syncwarp();
          ++issued;
        }
        base += 2 * sg.n;
        tiles_done += sg.n;
        unit += sg.n;
        if (unit < run.end) skip_segment(p, cur, sg);
      }
      if (lane == 0) {   // the last copies land before the CTA exits
        for (int64_t i = issued < C::kSlots ? 0 : issued - C::kSlots; i < issued; ++i) {
          const uint32_t bar = smem_u32(&full[slot_of(i)]);
          const uint64_t t0 = global_timer_ns();
          while (!mbar_try_wait(bar, phase_of(i)))
            if (global_timer_ns() - t0 > tp.timeout_ns) {
              atomicExch(p.err, kErrTimeout);
              break;
            }
        }
      }
    } else if (warp == 1) {
      // ---- MMAs ----
      const int k_steps = p.head_dim / 16;
      const uint32_t id = kF16 ? idesc_fp16(0) : idesc_bf16(0);
      const uint32_t id_s = id | ((uint32_t)(kTile >> 3) << 17);
      const uint32_t id_o = id | ((uint32_t)(p.head_dim >> 3) << 17) | (1u << 16);   // B is MN-major
      int64_t base = 0;
      uint32_t q_phase = 0, p_phase[2] = {0u, 0u};
      bool ok = true;
      for (int64_t unit = run.begin; unit < run.end && ok;) {
        const Segment sg = segment_at(p, cur, unit, run.end);
        const int n0 = sg.halves ? sg.n : (sg.n + 1) / 2, n1 = sg.halves ? sg.n : sg.n / 2;
        if (!mbar_wait_warp(q_ready, q_phase, ctl)) break;
        q_phase ^= 1u;
        tc_fence_after();
        auto scores = [&](int s, int j) {
          const int64_t pos = base + k_pos(sg.halves, sg.halves ? j : 2 * j + s);
          const int slot = slot_of(pos);
          if (!mbar_wait_warp(&full[slot], phase_of(pos), ctl)) return false;
          tc_fence_after();
          if (elect_one()) {
            const uint32_t qa = smem_u32(q_smem) + (sg.halves ? s * C::kSlot : 0);
            const uint32_t ka = smem_u32(ring + slot * C::kSlot);
            for (int i = 0; i < k_steps; ++i) {
              const uint32_t o = (uint32_t)(i >> 2) * C::kChunk + (uint32_t)(i & 3) * 32;
              mma_bf16(s_tmem + 128 * s, sdesc_k128(qa + o), sdesc_k128(ka + o), id_s, i > 0 ? 1u : 0u);
            }
            tc_commit(&s_full[s]);
            if (!sg.halves || s == 1) tc_commit(&empty[slot]);
          }
          __syncwarp();
          return true;
        };
        auto product = [&](int s, int j, bool last) {
          const int64_t pos = base + v_pos(sg.halves, sg.halves ? j : 2 * j + s, sg.n);
          const int slot = slot_of(pos);
          if (!mbar_wait_warp(&p_ready[s], p_phase[s], ctl) || !mbar_wait_warp(&full[slot], phase_of(pos), ctl))
            return false;
          p_phase[s] ^= 1u;
          tc_fence_after();
          if (elect_one()) {
            const uint32_t va = smem_u32(ring + slot * C::kSlot);
#pragma unroll
            for (int i = 0; i < kTile / 16; ++i)
              mma_f16_ts(o_tmem + 128 * s, s_tmem + 128 * s + 8 * i, sdesc_v(va + i * 2048, C::kChunk), id_o,
                         i > 0 || j > 0 ? 1u : 0u);
            if (!sg.halves || s == 1) tc_commit(&empty[slot]);
            if (last) tc_commit(&o_done[s]);
          }
          __syncwarp();
          return true;
        };
        ok = scores(0, 0) && (n1 == 0 || scores(1, 0));
        for (int j = 0; j < n0 && ok; ++j) {
          ok = product(0, j, j + 1 == n0) && (j + 1 >= n0 || scores(0, j + 1));
          if (ok && j < n1) ok = product(1, j, j + 1 == n1) && (j + 1 >= n1 || scores(1, j + 1));
        }
        base += 2 * sg.n;
        unit += sg.n;
        if (unit < run.end) skip_segment(p, cur, sg);
      }
      // every MMA issued finishes before tensor memory is released
      if (elect_one()) {
        tc_commit(mma_done);
        const uint32_t bar = smem_u32(mma_done);
        const uint64_t t0 = global_timer_ns();
        while (!mbar_try_wait(bar, 0))
          if (global_timer_ns() - t0 > tp.timeout_ns) {
            atomicExch(p.err, kErrTimeout);
            break;
          }
      }
    }
  } else {
    // ---- softmax: stream s, a thread per row ----
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    const int thread = threadIdx.x - kSoftWarp0 * 32;
    const int s = thread >> 7, r = thread & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t my_s = s_tmem + 128 * s + lanes, my_o = o_tmem + 128 * s + lanes;
    bool up = true;   // no wait has failed (after one, the loops run out without waiting)
    int64_t base = 0, tiles_done = 0;
    uint32_t s_phase = 0, o_phase = 0;
    for (int64_t unit = run.begin; unit < run.end;) {
      const Segment sg = segment_at(p, cur, unit, run.end);
      const int rows = (int)min((int64_t)kRows, (int64_t)cur.s.fresh * p.group - (int64_t)cur.rt * kRows);
      const int my_row = sg.halves ? 128 * s + r : r;
      const bool row_in = my_row < rows;
      const int64_t row = (int64_t)cur.rt * kRows + (row_in ? my_row : 0);
      const int t = (int)(row / p.group);
      const int64_t token = cur.s.first + t;
      const int head = cur.h * p.group + (int)(row % p.group);
      // Q into shared memory: rows of 128 swizzled bytes, 64 elements a chunk
      if (sg.halves || s == 0) {
        const uint16_t* const q = p.q + token * p.q_token + head * p.q_head;
        const uint32_t dst = smem_u32(q_smem) + (sg.halves ? s * C::kSlot : 0) + r * 128;
#pragma unroll
        for (int i = 0; i < kD / 8; ++i) {
          uint4 w = make_uint4(0u, 0u, 0u, 0u);
          if (row_in && 8 * i < p.head_dim) w = *reinterpret_cast<const uint4*>(q + 8 * i);
          st_shared_v4(dst + (i >> 3) * C::kChunk + (((i & 7) ^ (r & 7)) << 4), w.x, w.y, w.z, w.w);
        }
        fence_proxy_async_smem();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(q_ready);

      float m = -INFINITY, l = 0.0f;
      const int mine = sg.halves ? sg.n : (sg.n + 1 - s) / 2;
      for (int j = 0; j < mine; ++j) {
        const int tile = sg.halves ? j : 2 * j + s;
        const int64_t key0 = (int64_t)(sg.first + tile) * kTile;
        if (up) up = mbar_wait(&s_full[s], s_phase, ctl);
        s_phase ^= 1u;
        __syncwarp();
        tc_fence_after();
        uint32_t v[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(my_s + 32 * c, v[c]);
        tmem_ld_wait();
        const unsigned bads = *(volatile unsigned*)&bad_pages[(tiles_done + tile) % kBadRing];
        const bool tail = key0 + kTile > cur.s.cached;
        if (tail || bads != 0u) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t bits = tail ? seen_bits(p, cur.s, token, t, key0 + 32 * c) : 0xFFFFFFFFu;
            if (bads != 0u)
              for (int i = 0; i < 32; ++i)
                if ((bads >> ((32 * c + i) / tp.box_rows)) & 1u) bits &= ~(1u << i);
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (!((bits >> i) & 1u)) v[c][i] = 0xFF800000u;   // -infinity
          }
        }
        float top[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          top[c] = __uint_as_float(v[c][0]);
#pragma unroll
          for (int i = 1; i < 32; ++i) top[c] = fmaxf(top[c], __uint_as_float(v[c][i]));
        }
        const float cand = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * p.scale_log2;
        const bool rise = cand > m + kSlack || (m == -INFINITY && cand > m);
        if (__any_sync(0xFFFFFFFFu, rise)) {
          const float f = rise ? exp2_fast(m - cand) : 1.0f;
          l *= f;
          if (rise) m = cand;
          if (j > 0) {   // (the product before is done: the scores came after it)
#pragma unroll 1
            for (int c = 0; c < p.head_dim; c += 32) {
              uint32_t o[32];
              tmem_ld32(my_o + c, o);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
              tmem_st32(my_o + c, o);
            }
          }
        }
        const float2 scale2 = splat(p.scale_log2), base2 = splat(m == -INFINITY ? 0.0f : -m);
        float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t w[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const uint32_t* const x = v[2 * h + (i >> 4)];
            float2 e = fma2(make_float2(__uint_as_float(x[2 * (i & 15)]), __uint_as_float(x[2 * (i & 15) + 1])), scale2,
                            base2);
            e = make_float2(exp2_fast(e.x), exp2_fast(e.y));
            sum = add2(sum, e);
            w[i] = pack2<kF16>(e.x, e.y);
          }
          tmem_st32(my_s + 32 * h, w);
        }
        l += sum.x + sum.y;
        if (tail) {
          // V's row r of the tile: nothing but finite values may meet a P of zero
          const int64_t pos = base + v_pos(sg.halves, tile, sg.n);
          if (up) up = mbar_wait(&full[slot_of(pos)], phase_of(pos), ctl);
          const uint32_t va = smem_u32(ring + slot_of(pos) * C::kSlot) + r * 128;
          const bool in = key0 + r < cur.s.keys;
#pragma unroll 1
          for (int i = 0; i < kD / 8; ++i) {
            const uint32_t a = va + (i >> 3) * C::kChunk + (((i & 7) ^ (r & 7)) << 4);
            uint32_t x[4];
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                         : "r"(a));
            uint32_t odd = 0u;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const uint32_t hit = __vcmpgeu2(x[q] & 0x7FFF7FFFu, kF16 ? 0x7C007C00u : 0x7F807F80u);
              odd |= hit;
              x[q] = in ? x[q] & ~hit : 0u;
            }
            if (in && odd != 0u) {
              *(volatile int*)&odd_values = 1;   // before the zeros: who finds them finds this
              __threadfence_block();
            }
            if (!in || odd != 0u) st_shared_v4(a, x[0], x[1], x[2], x[3]);
          }
          fence_proxy_async_smem();
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_ready[s]);
      }

      // ---- the segment's end ----
      if (mine > 0) {
        if (up) up = mbar_wait(&o_done[s], o_phase, ctl);
        o_phase ^= 1u;
        __syncwarp();
        tc_fence_after();
      }
      const int64_t item0 = unit - sg.first, item1 = item0 + cur.tiles - 1;
      const bool whole = item0 >= run.begin && item1 < run.end;
      const bool join_streams = !sg.halves && sg.n > 1;
      // tiles in turn: the odd ones' sums through Q's place
      if (join_streams) {
        if (s == 1) {
          other_ml[r] = make_float2(m, l);
          const uint32_t dst = smem_u32(q_smem) + r * (kD * 4);
#pragma unroll 1
          for (int c = 0; c < p.head_dim; c += 32) {
            uint32_t o[32];
            tmem_ld32(my_o + c, o);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 8; ++i)
              st_shared_v4(dst + (((c / 4 + i) ^ (r & 7)) << 4), o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
          }
        }
        softmax_sync();
      }
      if (sg.halves || s == 0) {
        float f0 = 1.0f, f1 = 0.0f;
        if (join_streams) {
          const float2 b = other_ml[r];
          const float both = fmaxf(m, b.x), at = both == -INFINITY ? 0.0f : both;
          f0 = exp2_fast(m - at);
          f1 = exp2_fast(b.x - at);
          l = fmaf(l, f0, b.y * f1);
          m = both;
        }
        const int64_t part_row = (int64_t)(2 * blockIdx.x + (item0 < run.begin ? 0 : 1)) * kRows + my_row;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        const bool odd = *(volatile int*)&odd_values != 0;
        const uint32_t src = smem_u32(q_smem) + r * (kD * 4);
#pragma unroll 1
        for (int c = 0; c < p.head_dim; c += 32) {
          uint32_t o[32];
          tmem_ld32(my_o + c, o);
          tmem_ld_wait();
          float f[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(o[i]) * f0;
          if (join_streams) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float4 b;
              asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                           : "=f"(b.x), "=f"(b.y), "=f"(b.z), "=f"(b.w)
                           : "r"(src + (((c / 4 + i) ^ (r & 7)) << 4)));
              f[4 * i] = fmaf(b.x, f1, f[4 * i]);
              f[4 * i + 1] = fmaf(b.y, f1, f[4 * i + 1]);
              f[4 * i + 2] = fmaf(b.z, f1, f[4 * i + 2]);
              f[4 * i + 3] = fmaf(b.w, f1, f[4 * i + 3]);
            }
          }
          if (odd && row_in) {
            // values that were zeroed, for the rows that see them: infinities and NaN as they are
            const int64_t key_end = min(cur.s.keys, (int64_t)(sg.first + sg.n) * kTile);
            for (int64_t key = max((int64_t)sg.first * kTile, cur.s.cached / kTile * kTile); key < key_end; ++key) {
              int index, at;
              if (!(seen_bits(p, cur.s, token, t, key) & 1u) ||
                  !cache_place(key, p.page_size, p.table_width, &index, &at))
                continue;
              const int page = p.table[cur.b * p.table_stride + index];
              if (page < 0 || page >= p.pages) continue;
              const uint16_t* const x =
                  reinterpret_cast<const uint16_t*>(p.v + page * p.v_page + at * p.v_slot + cur.h * p.v_head) + c;
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                if (c + i >= p.head_dim) break;
                const uint32_t w = x[i];
                if ((w & 0x7FFFu) >= (kF16 ? 0x7C00u : 0x7F80u))
                  f[i] += kF16 ? __half2float(__ushort_as_half((unsigned short)w)) : __uint_as_float(w << 16);
              }
            }
          }
          if (row_in) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int d = c + 4 * i;
              if (d >= p.head_dim) break;
              const float4 x = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
              if (whole)
                store_out4(p, token, head, d, make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv));
              else
                *reinterpret_cast<float4*>(p.part + part_row * kD + d) = x;
            }
          }
        }
        if (row_in) {
          if (!whole)
            p.part_ml[part_row] = make_float2(m, l);
          else if (p.lse != nullptr)
            p.lse[token * p.lse_token + head] = log_sum(m, l);
        }
      }
      if (!whole) {
        const int first = (int)split_owner(item0, run.total, run.ctas), last = (int)split_owner(item1, run.total, run.ctas);
        __threadfence();
        softmax_sync();
        if (thread == 0) {
          const bool all = atomicAdd(&p.counts[first], 1u) == (unsigned)(last - first);
          if (all) p.counts[first] = 0u;   // as it was before the call
          __threadfence();
          last_flag = all ? 1u : 0u;
        }
        softmax_sync();
        if (last_flag != 0u) join_parts<kRows, kD, 256>(p, cur, first, last, 1.0f, thread);
      }
      tc_fence_before();
      softmax_sync();   // Q's place and the flags are free
      if (thread == 0) odd_values = 0;
      base += 2 * sg.n;
      tiles_done += sg.n;
      unit += sg.n;
      if (unit < run.end) skip_segment(p, cur, sg);
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <bool kF16, int kDC>
cudaError_t launch_cfg(TileParams tp, const CUtensorMap& tk, const CUtensorMap& tv, cudaStream_t s, Device dev) {
  using C = TileCfg<kDC>;
  auto kern = attn_tiles_kernel<kF16, kDC>;
  static PerDevice<cudaError_t> per_device;
  const cudaError_t e = per_device.get(dev.index, [&] {
    return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
  });
  if (e != cudaSuccess) return e;
  constexpr int64_t kPart = 2 * kRows * ((int64_t)64 * kDC * 4 + 8);
  const int ctas = (int)std::min<int64_t>(dev.num_sms, std::min<int64_t>(kMostCtas, (kWorkspaceBytes - kCountBytes) / kPart));
  AttnParams& p = tp.a;
  p.part_ml = reinterpret_cast<float2*>(reinterpret_cast<uint8_t*>(p.counts) + kCountBytes);
  p.part = reinterpret_cast<float*>(p.part_ml + (int64_t)2 * kRows * ctas);
  p.least = 2;
  return launch_pdl(kern, dim3((unsigned)ctas), kThreads, C::kSmem, s, tk, tv, tp);
}

}  // namespace

bool attention_tiles_fit(const AttnParams& p) {
  const bool pages = p.page_size % 8 == 0 && (p.page_size >= kTile ? p.page_size % kTile : kTile % p.page_size) == 0;
  return p.head_dim <= 128 && pages && p.k_slot > 0 && p.k_head > 0 && p.k_page > 0 && p.v_slot > 0 && p.v_head > 0 &&
         p.v_page > 0;
}

cudaError_t launch_attention_tiles(const AttnParams& p, bool fp16, uint64_t timeout_ns, cudaStream_t s, Device dev) {
  TileParams tp{};
  tp.a = p;
  tp.box_rows = std::min(p.page_size, kTile);
  tp.boxes = kTile / tp.box_rows;
  tp.timeout_ns = timeout_ns;
  CUtensorMap tk, tv;
  const uint64_t dims[4] = {(uint64_t)p.head_dim, (uint64_t)p.page_size, (uint64_t)p.heads, (uint64_t)p.pages};
  const uint32_t box[4] = {64u, (uint32_t)tp.box_rows, 1u, 1u};
  if (encode_tensor_map_4d16(&tk, p.k, fp16, dims, {(uint64_t)p.k_slot, (uint64_t)p.k_head, (uint64_t)p.k_page}, box) !=
          CUDA_SUCCESS ||
      encode_tensor_map_4d16(&tv, p.v, fp16, dims, {(uint64_t)p.v_slot, (uint64_t)p.v_head, (uint64_t)p.v_page}, box) !=
          CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  if (p.head_dim <= 64)
    return fp16 ? launch_cfg<true, 1>(tp, tk, tv, s, dev) : launch_cfg<false, 1>(tp, tk, tv, s, dev);
  return fp16 ? launch_cfg<true, 2>(tp, tk, tv, s, dev) : launch_cfg<false, 2>(tp, tk, tv, s, dev);
}

}  // namespace qlin
