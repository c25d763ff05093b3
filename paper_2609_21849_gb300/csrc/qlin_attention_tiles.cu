// Attention of many rows over a paged cache of 16-bit keys and values, on the tensor cores'
// own memory (tcgen05): drafts and runs of tokens whose rows per KV head (query heads of its
// group times new tokens) make the products the work.
//
// A CTA takes 256 rows of an item and tiles of 128 keys, in two streams that take turns on
// the tensor cores: while one stream's softmax runs, the other's products do.  With more than
// 128 rows the streams are the rows' halves over the same keys; with 128 or fewer, even and
// odd tiles over the same rows, joined at the end.  Per stream and tile:
//   S = Q K^T     tcgen05 from shared memory (K's pages by TMA, 128-byte swizzle) into 128 columns
//   P = 2^(S - m) a thread per row, 64 scores in registers at a time, P as 16-bit over S's columns
//   O += P V      A from tensor memory, V as it lies (keys x elements: an MN-major B)
// The running maximum moves only when it rises by more than 2^8, so O is rarely rescaled; P
// stays below 2^8 and the sums in fp32 (both fine in bf16: a P's rounding is relative).  fp16 has
// few exponents below 1: there the kept maximum is 2^7 below a row's, and P up to 2^15, so that
// weights down to 2^-32 of the largest one count.
//   Per tile of 256 rows and 128 keys of 128: 2048 cycles of MMAs (2560 where 128 bytes of shared
// memory a cycle bring a half's scores Q's rows and 64 keys), 1024 of exponentials (four cycles a warp
// measured), 64 KB of keys and values, about 2850 cycles of an SM's share of HBM.
// Roles: warps 0 and 2 load K and V, warp 1 issues MMAs, warp 3 walks the run for the softmax a
// segment ahead of it (and asks for the segment's Q), warps 4-7 and 8-11 are the streams' softmax, four
// more convert codes.
// Tiles with new tokens are masked, and V's slots behind the last key and values that are
// not finite are zeroed in shared memory: 0 times them would reach rows that do not see them.
// (Rows that do see such a value take it at the end.)
//   Heads above 128 fill tensor memory with one stream's O: tiles of 64 keys, the two halves of a
// tile's keys taking the streams' turns.  E4M3 codes land in a ring of their own, and four warps
// convert them to fp16 tiles (every code is an fp16); Q becomes fp16 after a power of two per row.
// An item that several CTAs share is joined by a second kernel, many CTAs to an item (joined by one
// of these, at one SM's rate of reading, the trees below took 40 us longer); it takes 14 of their us.
//   Measured, 16 trees of 64 tokens behind 8192-16384 keys, 8 KV heads of 128, 4 query heads each:
// 199 us (bf16; the keys and values from HBM need 126, the MMAs 106), 221 from E4M3; 288 at heads of
// 256 behind half as many keys.  About 3600 cycles a tile, of which the MMAs take 2048 to 2560, and no
// issue slot is short; what lasts is each stream's chain of scores, maximum, exponentials, P
// and products, of which two run at a time.  A segment's begin and end (Q's way in, the first scores,
// the tiles with masks, the last products, O's way out) take 10000 to 20000 cycles, many of them for
// instructions that no tile before them brought: their loops stay short.
#include <type_traits>

#include "qlin_attention_work.cuh"

namespace qlin {

namespace {

constexpr int kSoftWarp0 = 4, kConvertWarps = 4;
constexpr float kSlack = 8.0f;   // powers of two that a score may exceed the kept maximum by
constexpr float kRaise = 7.0f;   // powers of two above 1 of an fp16 P's maximum, without these
constexpr int kBadRing = 16;     // tiles whose bad pages are remembered

// A run's pieces: consecutive tiles of one item.
struct Segment {
  int first, n;      // tiles
  bool halves;
};
template <typename C>
__device__ __forceinline__ Segment segment_at(const AttnParams& p, const Cursor& c, int64_t unit, int64_t end) {
  const int64_t rows = (int64_t)c.s.fresh * p.group - (int64_t)c.rt * C::kRows;
  // (one stream: its tiles in the order of halves of the rows, of which there is one)
  return {c.tile, (int)min((int64_t)(c.tiles - c.tile), end - unit), C::kStreams == 1 || rows > 128};
}
template <typename C>
__device__ __forceinline__ void skip_segment(const AttnParams& p, Cursor& c, const Segment& s) {
  c.tile += s.n - 1;
  advance<C::kRows, C::kTile>(p, c);
}
// The unit behind a segment's, c being at its begin.
__device__ __forceinline__ int64_t unit_after(const Cursor& c, const Segment& s, int64_t unit, int item_cost) {
  return unit + s.n + (s.first + s.n == c.tiles ? item_cost : 0);
}

// A segment as the softmax threads need it, in shared memory: their registers hold scores.
struct SoftSegment {
  CacheSeq s;
  uint32_t base;         // loads before it
  int b, h, rt;
  int first, n;          // tiles; n 0: none left
  unsigned tiles_done;   // K tiles before it
  bool halves, whole, begun;   // begun: the item, before this CTA
};

// What the roles share beside tiles and barriers.
struct TileShared {
  float2 other[128];       // the odd tiles' maxima and sums
  RunScratch scratch;
  SoftSegment seg[2];
  unsigned bad_pages[kBadRing];   // of K tiles in order
  uint32_t tmem;
  int abort;
  int odd_values;
};

// kDC: chunks of 64 elements of a head.  Heads of up to 128 have two streams; longer ones take all of
// tensor memory for one stream's sums, 128 rows and tiles of 64 keys.  kCodes: an E4M3 cache.
template <int kDC, bool kCodes>
struct TileCfg {
  static constexpr int kStreams = kDC <= 2 ? 2 : 1;
  static constexpr int kRows = 128 * kStreams;
  static constexpr int kTile = kDC <= 2 ? 128 : 64, kHalf = kTile / 2;   // keys
  static constexpr int kChunk = kTile * 128, kQChunk = 128 * 128;        // 64 elements of a tile's keys, of 128 rows
  static constexpr int kSlot = kDC * kChunk;                             // a tile of K or V
  static constexpr int kQSlot = kDC * kQChunk, kQBytes = kStreams * kQSlot;
  static constexpr int kRawRow = 64 * kDC, kRawSlot = kCodes ? kTile * kRawRow : 0, kRawSlots = kCodes ? 4 : 0;
  static constexpr int kBarrierBytes = 384;
  static constexpr int kOther = kQBytes + kRawSlots * kRawSlot + kBarrierBytes + (int)sizeof(TileShared);
  static constexpr int kSlotsRaw = (232448 - kOther) / kSlot, kSlots = kSlotsRaw > 10 ? 10 : kSlotsRaw;
  static constexpr int kSmem = kOther + kSlots * kSlot;
  static constexpr int kSoftThreads = 128 * kStreams;
  static constexpr int kThreads = kSoftWarp0 * 32 + kSoftThreads + (kCodes ? kConvertWarps * 32 : 0);
  // registers: roles (and conversion), softmax
  static constexpr int kRoleRegs = kThreads == 512 ? 88 : 104, kSoftRegs = kThreads == 512 ? 152 : 200;
  static constexpr int kLaunchRegs = kThreads == 512 ? 128 : 168;
  static_assert((kThreads - kSoftThreads) * kRoleRegs + kSoftThreads * kSoftRegs <= kThreads * kLaunchRegs, "registers");
  static_assert((2 * kSlots + 2 * kRawSlots + 18) * 8 <= kBarrierBytes && kSlots >= 3, "shared memory");
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

template <int kSoftThreads>
__device__ __forceinline__ void softmax_sync() {
  asm volatile("bar.sync 1, %0;" ::"n"(kSoftThreads) : "memory");
}
// The same, and whether any thread says so.
template <int kSoftThreads>
__device__ __forceinline__ bool softmax_any(bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbar.red.or.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)x), "n"(kSoftThreads)
      : "memory");
  return r != 0u;
}

// Where in the order of loads a segment's tiles lie (n tiles; K and V of each).  Rows in two
// halves: K0 V0 K1 V1 ...  Tiles in turn: K0 K1 V0 K2 V1 K3 ...: each as the MMAs take them.
__device__ __forceinline__ int k_pos(bool halves, int j) { return halves ? 2 * j : j < 2 ? j : 2 * j - 1; }
__device__ __forceinline__ int v_pos(bool halves, int j, int n) { return halves ? 2 * j + 1 : min(2 * j + 2, n + j); }

// 32 bits of a row's mask from new token i on (negative ones are cached tokens: seen).
template <typename Words>
__device__ __forceinline__ uint32_t mask_window(const Words& m, int words, int64_t i) {
  if (i <= -32) return 0xFFFFFFFFu;
  const int n = i < 0 ? (int)-i : 0;
  const int64_t at = i + n;
  const int64_t w = at >> 6;
  const int s = (int)(at & 63);
  auto word = [&](int64_t k) -> uint64_t {
    if constexpr (std::is_array_v<Words>)
      return k >= words ? 0ull : k == 0 ? m[0] : m[1];   // (in registers: no index)
    else
      return k >= words ? 0ull : m[k];
  };
  uint64_t v = word(w) >> s;
  if (s > 32) v |= word(w + 1) << (64 - s);
  return n == 0 ? (uint32_t)v : ((uint32_t)v << n) | ((1u << n) - 1u);
}
// The first n of 32 (n may be negative or large).
__device__ __forceinline__ uint32_t first_bits(int64_t n) {
  return n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << (int)n) - 1u;
}

// Two E4M3 codes as two halves, exactly.
__device__ __forceinline__ uint32_t e4m3x2_half2(uint32_t codes) {
  uint32_t h;
  const uint16_t c = (uint16_t)codes;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(c));
  return h;
}

// Which keys of 32 a row (new token t, number `token` of the call) sees, from key `key` on.  early:
// the row's first two mask words.
__device__ __forceinline__ uint32_t seen_bits(const AttnParams& p, const CacheSeq& s, int64_t token, int t, int64_t key,
                                              const uint64_t (&early)[2]) {
  const uint32_t in = first_bits(s.keys - key);
  if (p.mask == nullptr) return in & first_bits(s.cached + t + 1 - key);
  return in & (p.mask_words <= 2 ? mask_window(early, p.mask_words, key - s.cached)
                                 : mask_window(p.mask + token * p.mask_token, p.mask_words, key - s.cached));
}

template <bool kF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return kF16 ? pack_f16x2(lo, hi) : pack_bf16x2(lo, hi);
}

// The largest, or NaN.
__device__ __forceinline__ float max_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Minus infinity for the scores of columns 32 c on that a row does not see.
__device__ __forceinline__ void hide(uint32_t bits, unsigned bads, int c, int box_rows, uint32_t (&v)[32]) {
  if (bads != 0u)
    for (int i = 0; i < 32; ++i)
      if ((bads >> ((32 * c + i) / box_rows)) & 1u) bits &= ~(1u << i);
#pragma unroll
  for (int i = 0; i < 32; ++i)
    if (!((bits >> i) & 1u)) v[i] = 0xFF800000u;
}

template <bool kF16, int kDC, bool kCodes>
__global__ void __launch_bounds__(TileCfg<kDC, kCodes>::kThreads, 1)
    attn_tiles_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                      const TileParams tp) {
  using C = TileCfg<kDC, kCodes>;
  constexpr int kD = 64 * kDC, kRows = C::kRows, kTile = C::kTile, kHalf = C::kHalf, kThreads = C::kThreads;
  static_assert(kF16 || !kCodes, "codes become fp16");
  const AttnParams& p = tp.a;
  extern __shared__ __align__(1024) uint8_t smem[];
  if ((smem_u32(smem) & 1023u) != 0u) {   // (the swizzle's atoms; no other shared memory comes before)
    atomicExch(p.err, kErrTimeout);
    if (threadIdx.x == 0) p.join[blockIdx.x].rows = 0;
    return;
  }
  uint8_t* const q_smem = smem;
  uint8_t* const ring = smem + C::kQBytes;
  uint8_t* const raw = ring + C::kSlots * C::kSlot;   // kCodes: tiles of codes as they come
  uint64_t* const full = reinterpret_cast<uint64_t*>(raw + C::kRawSlots * C::kRawSlot);
  uint64_t* const empty = full + C::kSlots;
  uint64_t* const s_full = empty + C::kSlots;    // per stream and half of a tile: scores are there
  uint64_t* const p_ready = s_full + 4;          // the same: P is there
  uint64_t* const pv_done = p_ready + 4;         // the same: its product is done
  uint64_t* const q_ready = pv_done + 4;
  uint64_t* const mma_done = q_ready + 1;
  uint64_t* const seg_full = mma_done + 1;       // of two: a segment is published, and has been worked off
  uint64_t* const seg_free = seg_full + 2;
  uint64_t* const raw_full = seg_free + 2;       // kCodes: codes have landed, and have been converted
  uint64_t* const raw_empty = raw_full + C::kRawSlots;
  TileShared& sh = *reinterpret_cast<TileShared*>(raw + C::kRawSlots * C::kRawSlot + C::kBarrierBytes);

  const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kSlots; ++i) {
      mbar_init(&full[i], kCodes ? kConvertWarps : 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < C::kRawSlots; ++i) {
      mbar_init(&raw_full[i], 1);
      mbar_init(&raw_empty[i], kConvertWarps);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&p_ready[i], 4);
      mbar_init(&pv_done[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&seg_full[i], 1);
      mbar_init(&seg_free[i], 4 * C::kStreams);
    }
    mbar_init(q_ready, 4 * C::kStreams);
    mbar_init(mma_done, 1);
    sh.abort = 0;
    sh.odd_values = 0;
    mbar_fence_init();
  }
  if (warp == 0 && lane < 2) prefetch_tmap(lane == 0 ? &tmap_k : &tmap_v);
  if (warp == 1) tmem_alloc(&sh.tmem, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, sh.tmem, 0);
  const uint32_t s_tmem = tmem, o_tmem = tmem + 256;   // stream s: 128 columns further
  const WaitCtl ctl{&sh.abort, p.err, tp.timeout_ns};
  grid_dep_wait();
  grid_dep_launch();
  Cursor cur;
  const Run run = find_run<kRows, kTile, kThreads>(p, cur, (int)blockIdx.x, (int)gridDim.x, sh.scratch);

  // (loads of a CTA are counted in 32 bits: fewer than 2^25 tiles of keys a sequence, 2^31 in all)
  auto slot_of = [&](uint32_t pos) { return (int)(pos % C::kSlots); };
  auto phase_of = [&](uint32_t pos) { return (pos / C::kSlots) & 1u; };
  constexpr uint32_t kRing = kCodes ? C::kRawSlots : 1;   // of codes

  if (warp < kSoftWarp0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRoleRegs));
    if (warp == 0 || warp == 2) {
      // ---- loads, of K or V: a lane per page of the tile ----
      const bool is_v = warp == 2;
      const CUtensorMap* const map = is_v ? &tmap_v : &tmap_k;
      uint32_t base = 0;         // loads before this segment
      unsigned tiles_done = 0;   // K tiles before it
      uint32_t used = 0u, phases = 0u;   // slots that this warp filled, and in which phase last
      bool ok = true;
      for (int64_t unit = run.begin; unit < run.end && ok;) {
        const Segment sg = segment_at<C>(p, cur, unit, run.end);
        struct Load {
          bool in;
          int at, page;
        };
        // the lane's page of tile j, and its first slot of it
        auto locate = [&](int j) {
          Load d{};
          const uint32_t key = (uint32_t)(sg.first + j) * kTile + lane * tp.box_rows;   // (below 2^31 + 128)
          const uint32_t index = key / (uint32_t)p.page_size;
          d.in = lane < tp.boxes && key < cur.s.keys;
          d.at = (int)(key - index * (uint32_t)p.page_size);
          d.page = d.in ? p.table[cur.b * p.table_stride + index] : 0;
          return d;
        };
        Load next = locate(0);
        for (int j = 0; j < sg.n; ++j) {
          const Load d = next;
          if (j + 1 < sg.n) next = locate(j + 1);   // (the table's entry on its way while this load waits)
          const uint32_t pos = base + (is_v ? v_pos(sg.halves, j, sg.n) : k_pos(sg.halves, j));
          const int slot = slot_of(pos);
          const bool bad = d.in && (d.page < 0 || d.page >= p.pages);
          const unsigned bads = __ballot_sync(0xFFFFFFFFu, bad);
          if (bad) report_invalid(p.err);
          const int page = !d.in || bad ? p.pages : d.page;   // past the last: zeros
          const int at = !d.in || bad ? 0 : d.at;
          const int rs = (int)(pos % kRing);
          uint64_t* const there = kCodes ? &raw_full[rs] : &full[slot];
          if (!(kCodes ? mbar_wait_warp(&raw_empty[rs], ((pos / kRing) & 1u) ^ 1u, ctl)
                       : mbar_wait_warp(&empty[slot], phase_of(pos) ^ 1u, ctl))) {
            ok = false;
            break;
          }
          if (lane == 0) {
            if (!is_v) *(volatile unsigned*)&sh.bad_pages[(tiles_done + j) % kBadRing] = bads;
            mbar_arrive_expect_tx(there, kCodes ? C::kRawSlot : C::kSlot);
          }
          __syncwarp();
          if (lane < tp.boxes) {
            if (kCodes) {
              tma_load_4d(raw + rs * C::kRawSlot + lane * tp.box_rows * C::kRawRow, map, smem_u32(there), 0, at, cur.h,
                          page);
            } else {
              uint8_t* const dst = ring + slot * C::kSlot + lane * tp.box_rows * 128;
#pragma unroll
              for (int c = 0; c < kDC; ++c) tma_load_4d(dst + c * C::kChunk, map, smem_u32(there), 64 * c, at, cur.h, page);
            }
          }
          __syncwarp();
          const int b = kCodes ? rs : slot;
          used |= 1u << b;
          phases = (phases & ~(1u << b)) | ((kCodes ? (pos / kRing) & 1u : phase_of(pos)) << b);
        }
        base += 2 * sg.n;
        tiles_done += sg.n;
        unit = unit_after(cur, sg, unit, p.item_cost);
        if (unit < run.end) skip_segment<C>(p, cur, sg);
      }
      // (The MMAs wait for every load.)  After a wait that gave up, copies in flight land before
      // the CTA exits, or a limit passes.
      if (!ok && lane == 0) {
        const uint64_t t0 = global_timer_ns();
        for (int i = 0; i < (kCodes ? C::kRawSlots : C::kSlots); ++i)
          while (((used >> i) & 1u) && !mbar_try_wait(smem_u32(kCodes ? &raw_full[i] : &full[i]), (phases >> i) & 1u))
            if (global_timer_ns() - t0 > tp.timeout_ns) break;
      }
    } else if (warp == 1) {
      // ---- MMAs ----
      const int k_steps = p.head_dim / 16;
      const uint32_t id = kF16 ? idesc_fp16(0) : idesc_bf16(0);
      const uint32_t id_s = id | ((uint32_t)(kHalf >> 3) << 17);
      const uint32_t id_o = id | ((uint32_t)(p.head_dim >> 3) << 17) | (1u << 16);   // B is MN-major
      uint32_t base = 0;
      uint32_t q_phase = 0, p_phase[2] = {0u, 0u};
      bool ok = true;
      for (int64_t unit = run.begin; unit < run.end && ok;) {
        // (what the descriptors depend on goes through a shuffle, so that the compiler knows it to
        // be the same in all lanes and keeps them in uniform registers, where tcgen05 takes them: an
        // MMA issued from others cost 70 cycles, more than it runs)
        Segment sg = segment_at<C>(p, cur, unit, run.end);
        sg.n = __shfl_sync(0xFFFFFFFFu, sg.n, 0);
        sg.halves = __shfl_sync(0xFFFFFFFFu, (int)sg.halves, 0) != 0;
        const int n0 = sg.halves ? sg.n : (sg.n + 1) / 2, n1 = C::kStreams == 1 ? 0 : sg.halves ? sg.n : sg.n / 2;
        if (!mbar_wait_warp(q_ready, q_phase, ctl)) break;
        q_phase ^= 1u;
        tc_fence_after();
        // (one elected lane) scores of half hf of the stream's tile in `slot`
        auto scores = [&](int s, int hf, int slot) {
          const uint32_t qa = smem_u32(q_smem) + (sg.halves ? s * C::kQSlot : 0);
          const uint32_t ka = smem_u32(ring + slot * C::kSlot) + hf * kHalf * 128;
          const uint64_t qd = sdesc_k128(qa), kd = sdesc_k128(ka);
#pragma unroll
          for (int i = 0; i < 4 * kDC; ++i) {
            constexpr uint64_t kStep = 32 >> 4;   // (in the descriptors' units)
            const uint64_t q = (uint64_t)(i >> 2) * (C::kQChunk >> 4) + (uint64_t)(i & 3) * kStep;
            const uint64_t k = (uint64_t)(i >> 2) * (C::kChunk >> 4) + (uint64_t)(i & 3) * kStep;
            if (i < k_steps) mma_bf16(s_tmem + 128 * s + kHalf * hf, qd + q, kd + k, id_s, i > 0 ? 1u : 0u);
          }
          tc_commit(&s_full[2 * s + hf]);
          if (hf == 1 && (C::kStreams == 1 || !sg.halves || s == 1)) tc_commit(&empty[slot]);
        };
        auto k_slot = [&](int s, int j, int* slot) {
          const uint32_t pos = base + k_pos(sg.halves, sg.halves ? j : 2 * j + s);
          *slot = __shfl_sync(0xFFFFFFFFu, slot_of(pos), 0);
          const bool there = mbar_wait_warp(&full[*slot], phase_of(pos), ctl);
          tc_fence_after();
          return there;
        };
        // The products of the stream's tile j, and the scores of its next one: each half's as its P
        // comes, into the columns that this frees, while the softmax works on the other half.
        auto tile = [&](int s, int j, bool last) {
          const uint32_t pos = base + v_pos(sg.halves, sg.halves ? j : 2 * j + s, sg.n);
          const int slot = __shfl_sync(0xFFFFFFFFu, slot_of(pos), 0);
          int next = 0;
          if (!mbar_wait_warp(&full[slot], phase_of(pos), ctl)) return false;
          const uint64_t vd = sdesc_v(smem_u32(ring + slot * C::kSlot), C::kChunk);
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            if (!mbar_wait_warp(&p_ready[2 * s + hf], p_phase[s], ctl)) return false;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int i = 0; i < kHalf / 16; ++i)
                mma_f16_ts(o_tmem + 128 * s, s_tmem + 128 * s + kHalf * hf + 8 * i,
                           vd + (uint64_t)((kHalf / 16 * hf + i) * (2048 >> 4)), id_o, i > 0 || hf > 0 || j > 0 ? 1u : 0u);
              tc_commit(&pv_done[2 * s + hf]);
              if (hf == 1 && (C::kStreams == 1 || !sg.halves || s == 1)) tc_commit(&empty[slot]);
            }
            __syncwarp();
            if (last) continue;
            if (hf == 0 && !k_slot(s, j + 1, &next)) return false;
            if (elect_one()) scores(s, hf, next);
            __syncwarp();
          }
          p_phase[s] ^= 1u;
          return true;
        };
        for (int s = 0; s < (n1 > 0 ? 2 : 1) && ok; ++s) {
          int slot;
          ok = k_slot(s, 0, &slot);
          if (ok && elect_one()) {
            scores(s, 0, slot);
            scores(s, 1, slot);
          }
          __syncwarp();
        }
        for (int j = 0; j < n0 && ok; ++j) {
          ok = tile(0, j, j + 1 == n0);
          if (ok && j < n1) ok = tile(1, j, j + 1 == n1);
        }
        base += 2 * sg.n;
        unit = unit_after(cur, sg, unit, p.item_cost);
        if (unit < run.end) skip_segment<C>(p, cur, sg);
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
    } else {
      // ---- the run's segments for the softmax threads, one ahead of them ----
      uint32_t base = 0;
      unsigned tiles_done = 0, phase = 0;
      int64_t unit = run.begin;
      JoinItem mine{0, 0, 0, 0, 0};
      for (int at = 0;; at ^= 1) {
        if (!mbar_wait_warp(&seg_free[at], phase ^ 1u, ctl)) break;
        phase ^= (uint32_t)at;
        const bool any = unit < run.end;
        Segment sg{0, 0, false};
        if (any) sg = segment_at<C>(p, cur, unit, run.end);
        if (lane == 0) {
          SoftSegment& g = sh.seg[at];
          const int64_t item0 = unit - sg.first;
          g.s = cur.s;
          g.base = base;
          g.b = cur.b;
          g.h = cur.h;
          g.rt = cur.rt;
          g.first = sg.first;
          g.n = sg.n;
          g.tiles_done = tiles_done;
          g.halves = sg.halves;
          g.begun = item0 < run.begin;
          g.whole = !g.begun && item0 + cur.tiles <= run.end;
          mbar_arrive(&seg_full[at]);
        }
        __syncwarp();
        if (!any) break;
        const int64_t item0 = unit - sg.first, item1 = item0 + cur.tiles - 1;
        if (item0 >= run.begin && item1 >= run.end)
          mine = {cur.s.first, cur.rt * kRows, cur.h * p.group, min(kRows, cur.s.fresh * p.group - cur.rt * kRows),
                  (int)split_owner(run.split, item1)};
        // its rows of Q towards L2
        for (int i = lane; i < kRows; i += 32) {
          const int row = cur.rt * kRows + i;
          if (row >= cur.s.fresh * p.group) break;
          const uint16_t* const q = p.q + (cur.s.first + row / p.group) * p.q_token +
                                    (int64_t)(cur.h * p.group + row % p.group) * p.q_head;
          for (int d = 0; d < p.head_dim; d += 64) asm volatile("prefetch.global.L2 [%0];" ::"l"(q + d));
        }
        base += 2 * sg.n;
        tiles_done += sg.n;
        unit = unit_after(cur, sg, unit, p.item_cost);
        if (unit < run.end) skip_segment<C>(p, cur, sg);
      }
      if (lane == 0) p.join[blockIdx.x] = mine;
    }
  } else if (kCodes && warp >= kSoftWarp0 + C::kSoftThreads / 32) {
    // ---- codes to fp16 (exactly), from the rows as they came to the MMAs' swizzled tiles ----
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRoleRegs));
    const int thread = threadIdx.x - kSoftWarp0 * 32 - C::kSoftThreads;
    uint32_t pos = 0;
    bool ok = true;
    for (int64_t unit = run.begin; unit < run.end && ok;) {
      const Segment sg = segment_at<C>(p, cur, unit, run.end);
      for (const uint32_t end = pos + 2 * sg.n; pos < end; ++pos) {
        const int rs = (int)(pos % kRing), slot = slot_of(pos);
        if (!mbar_wait_warp(&raw_full[rs], (pos / kRing) & 1u, ctl) ||
            !mbar_wait_warp(&empty[slot], phase_of(pos) ^ 1u, ctl)) {
          ok = false;
          break;
        }
        const uint32_t src = smem_u32(raw + rs * C::kRawSlot), dst = smem_u32(ring + slot * C::kSlot);
#pragma unroll 4
        for (int i = thread; i < kTile * 4 * kDC; i += kConvertWarps * 32) {   // 16 codes
          const int key = i / (4 * kDC), at = i % (4 * kDC);
          uint32_t w[4], h[8];
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                       : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                       : "r"(src + key * C::kRawRow + at * 16));
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            h[2 * k] = e4m3x2_half2(w[k]);
            h[2 * k + 1] = e4m3x2_half2(w[k] >> 16);
          }
          const uint32_t to = dst + (at >> 2) * C::kChunk + key * 128;
          const int piece = 2 * (at & 3);
          st_shared_v4(to + ((piece ^ (key & 7)) << 4), h[0], h[1], h[2], h[3]);
          st_shared_v4(to + (((piece + 1) ^ (key & 7)) << 4), h[4], h[5], h[6], h[7]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&full[slot]);
          mbar_arrive(&raw_empty[rs]);
        }
      }
      unit = unit_after(cur, sg, unit, p.item_cost);
      if (unit < run.end) skip_segment<C>(p, cur, sg);
    }
  } else {
    // ---- softmax: stream s, row r ----
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kSoftRegs));
    const int thread = threadIdx.x - kSoftWarp0 * 32;
    const int s = thread >> 7, r = thread & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t my_s = s_tmem + 128 * s + lanes, my_o = o_tmem + 128 * s + lanes;
    bool up = true;   // no wait has failed (after one, the loops run out without waiting)
    uint32_t s_phase = 0;   // of the stream's tiles
    uint32_t seg_phase = 0;
    for (int at = 0;; at ^= 1) {
      const SoftSegment& g = sh.seg[at];
      if (up) up = mbar_wait(&seg_full[at], seg_phase, ctl);
      __syncwarp();
      seg_phase ^= (uint32_t)at;
      // (after a wait that gave up, all leave together: no thread waits at a barrier for one that left)
      if (softmax_any<C::kSoftThreads>(!up)) break;
      const int n = g.n;
      if (n == 0) break;
      const bool halves = g.halves;
      // (tokens and rows below 2^31)
      const int my_row = halves ? 128 * s + r : r;
      auto row_in = [&] { return g.rt * kRows + my_row < g.s.fresh * p.group; };
      auto row_of = [&] { return row_in() ? g.rt * kRows + my_row : 0; };
      float mult = p.scale_log2;   // from scores to powers of two
      uint64_t early[2] = {0ull, 0ull};   // the row's mask, on its way before a tile needs it
      if (p.mask != nullptr && p.mask_words <= 2) {
        const uint64_t* const words = p.mask + (g.s.first + row_of() / p.group) * p.mask_token;
        early[0] = words[0];
        if (p.mask_words == 2) early[1] = words[1];
      }
      // Q into shared memory: rows of 128 swizzled bytes, 64 elements a chunk.  Each warp copies its rows,
      // asynchronously: through registers, with a store behind each load, this took 6000 to 14000 cycles.
      const bool stores_q = halves || s == 0;
      const int64_t q_row = row_in() ? (g.s.first + row_of() / p.group) * p.q_token +
                                           (int64_t)(g.h * p.group + row_of() % p.group) * p.q_head
                                     : -1;
      const uint32_t q_dst = smem_u32(q_smem) + (halves ? s * C::kQSlot : 0);
      if (stores_q) {
        constexpr int kPieces = kD / 8;   // of 16 bytes
#pragma unroll 4
        for (int i = 0; i < kPieces; ++i) {
          const int at = i * 32 + lane, row = at / kPieces, piece = at % kPieces, to = (r & ~31) + row;
          const int64_t from = __shfl_sync(0xFFFFFFFFu, q_row, row);
          const bool in = from >= 0 && 8 * piece < p.head_dim;
          cp_async16(q_dst + (piece >> 3) * C::kQChunk + to * 128 + (((piece & 7) ^ (to & 7)) << 4),
                     p.q + (in ? from + 8 * piece : 0), in);
        }
        cp_async_commit();
        cp_async_wait<0>();
        __syncwarp();
      }
      if constexpr (kCodes) {
        // fp16 after a power of two that brings the row's largest |q| into [1, 2) (a zero, infinite or
        // NaN row as it is); a stream that did not store reads its rows again
        const uint32_t dst = q_dst + r * 128;
        auto place = [&](int i) { return dst + (i >> 3) * C::kQChunk + (((i & 7) ^ (r & 7)) << 4); };
        auto piece = [&](int i) {
          if (stores_q) return lds128(place(i));
          return q_row >= 0 && 8 * i < p.head_dim ? *reinterpret_cast<const uint4*>(p.q + q_row + 8 * i)
                                                  : make_uint4(0u, 0u, 0u, 0u);
        };
        uint32_t top = 0u;
#pragma unroll 2
        for (int i = 0; i < kD / 8; ++i) {
          const uint4 w = piece(i);
          top = __vmaxu2(__vmaxu2(__vmaxu2(__vmaxu2(top, w.x & 0x7FFF7FFFu), w.y & 0x7FFF7FFFu), w.z & 0x7FFF7FFFu),
                         w.w & 0x7FFF7FFFu);
        }
        top = max(top & 0xFFFFu, top >> 16);
        const float big = p.fp16 ? __half2float(__ushort_as_half((unsigned short)top)) : __uint_as_float(top << 16);
        int e = (int)(__float_as_uint(big) >> 23);   // biased
        e = e == 0 || e == 255 ? 127 : min(e, 252);
        const float k_scale = *p.k_scale, down = signed_factor(__uint_as_float((uint32_t)(254 - e) << 23), k_scale);
        mult = fminf(fmaxf(p.scale_log2 * __uint_as_float((uint32_t)e << 23) * fabsf(k_scale), FLT_MIN), FLT_MAX);
        auto scaled = [&](uint32_t w) {
          const float2 v = p.fp16 ? __half22float2(*reinterpret_cast<const __half2*>(&w)) : make_float2(bf16_lo(w), bf16_hi(w));
          return pack_f16x2(v.x * down, v.y * down);
        };
#pragma unroll 2
        for (int i = 0; i < (stores_q ? kD / 8 : 0); ++i) {
          const uint4 w = lds128(place(i));
          st_shared_v4(place(i), scaled(w.x), scaled(w.y), scaled(w.z), scaled(w.w));
        }
      }
      if (stores_q) fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(q_ready);

      float m = -INFINITY, l = 0.0f;
      const int mine = halves ? n : (n + 1 - s) / 2;
      const int tail_from = (int)(first_unseen(g.s) / kTile - g.first);   // the first tile with new tokens or none
      for (int j2 = 0; j2 < 2 * mine; ++j2) {
        const int hf = j2 & 1, tile = halves ? j2 >> 1 : (j2 & ~1) + s;
        const bool tail = tile >= tail_from;
        const uint32_t at_s = my_s + kHalf * hf;
        if (up) up = mbar_wait(&s_full[2 * s + hf], s_phase, ctl);
        __syncwarp();
        tc_fence_after();
        constexpr int kC = kHalf / 32;
        uint32_t v[kC][32];
#pragma unroll
        for (int c = 0; c < kC; ++c) tmem_ld32(at_s + 32 * c, v[c]);
        const unsigned bads = *(volatile unsigned*)&sh.bad_pages[(g.tiles_done + tile) % kBadRing];
        tmem_ld_wait();
        if (tail || bads != 0u) {
          const int row = row_of(), t = row / p.group;
          const int64_t key = (int64_t)(g.first + tile) * kTile + kHalf * hf;
#pragma unroll
          for (int c = 0; c < kC; ++c)
            hide(tail ? seen_bits(p, g.s, g.s.first + t, t, key + 32 * c, early) : 0xFFFFFFFFu, bads, kC * hf + c, tp.box_rows,
                 v[c]);
        }
        float top[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) top[i] = __uint_as_float(v[0][i]);
#pragma unroll
        for (int i = 8; i < kHalf; i += 16)
#pragma unroll
          for (int k = 0; k < 8; ++k)
            top[k] = max_nan(top[k], __uint_as_float(v[(i + k) >> 5][(i + k) & 31]),
                             i + 8 < kHalf ? __uint_as_float(v[(i + 8 + k) >> 5][(i + 8 + k) & 31]) : top[k]);
        const float most = max_nan(max_nan(top[0], top[1], top[2]), max_nan(top[3], top[4], top[5]),
                                   max_nan(top[6], top[7], top[7]));
        // (fp16: the candidate rounded up and the limit down, so that no P passes 2^15)
        const float cand = kF16 ? __fadd_ru(__fmul_ru(most, mult), -kRaise) : most * mult;
        const bool rise = cand > (kF16 ? __fadd_rd(m, kSlack) : m + kSlack) || (m == -INFINITY && cand > m);
        if (__any_sync(0xFFFFFFFFu, rise)) {
          const float f = rise ? exp2_fast(m - cand) : 1.0f;
          l *= f;
          if (rise) m = cand;
          if (j2 > 0) {
            // the product before this half's has to be done (those before that one are: its
            // columns hold these scores): the first half's of this tile, the second's of the last
            if (up) up = mbar_wait(&pv_done[2 * s + (hf ^ 1)], hf ? s_phase : s_phase ^ 1u, ctl);
            __syncwarp();
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < p.head_dim; c += 16) {
              uint32_t o[16];
              tmem_ld16(my_o + c, o);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
              tmem_st16(my_o + c, o);
            }
          }
        }
        const float2 scale2 = splat(mult), base2 = splat(m == -INFINITY ? 0.0f : -m);
        // (with a NaN or an infinity among the scores the row is NaN)
        float2 sum = make_float2(cand < INFINITY ? 0.0f : __uint_as_float(0x7FFFFFFFu), 0.0f);
#pragma unroll
        for (int c = 0; c < kC; ++c) {
          uint32_t w[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float2 e = fma2(make_float2(__uint_as_float(v[c][2 * i]), __uint_as_float(v[c][2 * i + 1])), scale2, base2);
            e = make_float2(exp2_fast(e.x), exp2_fast(e.y));
            sum = add2(sum, e);
            w[i] = pack2<kF16>(e.x, e.y);
          }
          tmem_st16(at_s + 16 * c, w);
        }
        l += sum.x + sum.y;
        if (tail) {
          // V's rows of the half, two threads (or four) each: nothing but finite values may meet a P of zero
          const uint32_t pos = g.base + v_pos(halves, tile, n);
          if (up) up = mbar_wait(&full[slot_of(pos)], phase_of(pos), ctl);
          const int key_row = kHalf * hf + (r & (kHalf - 1));
          const uint32_t va = smem_u32(ring + slot_of(pos) * C::kSlot) + key_row * 128;
          const bool in = (int64_t)(g.first + tile) * kTile + key_row < g.s.keys;
          constexpr int kStep = 128 / kHalf, kOwn = kD / 8 / kStep, kBatch = kOwn % 4 == 0 ? 4 : 2;
#pragma unroll 1
          for (int i0 = r / kHalf; i0 < kD / 8; i0 += kBatch * kStep) {
            auto place = [&](int k) {
              const int i = i0 + k * kStep;
              return va + (i >> 3) * C::kChunk + (((i & 7) ^ (r & 7)) << 4);
            };
            uint4 x[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) x[k] = lds128(place(k));
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
              uint32_t odd = 0u;
              auto finite = [&](uint32_t w) {
                const uint32_t hit = __vcmpgeu2(w & 0x7FFF7FFFu, kF16 ? 0x7C007C00u : 0x7F807F80u);
                odd |= hit;
                return in ? w & ~hit : 0u;
              };
              const uint4 w = make_uint4(finite(x[k].x), finite(x[k].y), finite(x[k].z), finite(x[k].w));
              if (in && odd != 0u) {
                *(volatile int*)&sh.odd_values = 1;   // before the zeros: who finds them finds this
                __threadfence_block();
              }
              if (!in || odd != 0u) st_shared_v4(place(k), w.x, w.y, w.z, w.w);
            }
          }
          fence_proxy_async_smem();
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_ready[2 * s + hf]);
        s_phase ^= (uint32_t)hf;
      }

      // ---- the segment's end ----
      if (mine > 0) {
        if (up) up = mbar_wait(&pv_done[2 * s + 1], s_phase ^ 1u, ctl);
        __syncwarp();
        tc_fence_after();
      }
      const bool join_streams = !halves && n > 1;
      // tiles in turn: the odd ones' sums through Q's place
      if (join_streams) {
        if (s == 1) {
          sh.other[r] = make_float2(m, l);
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
        softmax_sync<C::kSoftThreads>();
      }
      if (halves || s == 0) {
        float f0 = 1.0f, f1 = 0.0f;
        if (join_streams) {
          const float2 b = sh.other[r];
          const float both = fmaxf(m, b.x), top = both == -INFINITY ? 0.0f : both;
          f0 = exp2_fast(m - top);
          f1 = exp2_fast(b.x - top);
          l = fmaf(l, f0, b.y * f1);
          m = both;
        }
        const bool in = row_in(), whole = g.whole;
        const int row = row_of(), t = row / p.group, head = g.h * p.group + row % p.group;
        const int64_t token = g.s.first + t;
        const int64_t at_part = (int64_t)(2 * blockIdx.x + (g.begun ? 0 : 1)) * kRows;
        const float inv = l == 0.0f ? 0.0f : (kCodes ? *p.v_scale : 1.0f) / l;
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
          if (*(volatile int*)&sh.odd_values != 0 && in) {
            // values that were zeroed, for the rows that see them: infinities and NaN as they are
            const int64_t key_end = min(g.s.keys, (int64_t)(g.first + n) * kTile);
            for (int64_t key = max((int64_t)g.first * kTile, first_unseen(g.s) / kTile * kTile); key < key_end; ++key) {
              int index, slot;
              if (!(seen_bits(p, g.s, token, t, key, early) & 1u) ||
                  !cache_place(key, p.page_size, p.table_width, &index, &slot))
                continue;
              const int page = p.table[g.b * p.table_stride + index];
              if (page < 0 || page >= p.pages) continue;
              const uint8_t* const x = p.v + page * p.v_page + slot * p.v_slot + g.h * p.v_head;
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                if (c + i >= p.head_dim) break;
                if constexpr (kCodes) {
                  if ((x[c + i] & 0x7Fu) == 0x7Fu) f[i] = __uint_as_float(0x7FFFFFFFu);
                } else {
                  const uint32_t w = reinterpret_cast<const uint16_t*>(x)[c + i];
                  if ((w & 0x7FFFu) >= (kF16 ? 0x7C00u : 0x7F80u))
                    f[i] += kF16 ? __half2float(__ushort_as_half((unsigned short)w)) : __uint_as_float(w << 16);
                }
              }
            }
          }
          if (in) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int d = c + 4 * i;
              if (d >= p.head_dim) break;
              const float4 x = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
              if (!whole) {
                *part_sums<kRows, kD>(p, at_part, my_row, d) = x;
              } else if ((i & 1) == 0) {   // (head_dim % 16 == 0: eight elements at a time)
                auto pair = [&](float a, float b) {
                  return p.fp16 ? pack_f16x2(a * inv, b * inv) : pack_bf16x2(a * inv, b * inv);
                };
                *reinterpret_cast<uint4*>(p.out + token * p.out_token + (int64_t)head * p.out_head + d) =
                    make_uint4(pair(x.x, x.y), pair(x.z, x.w), pair(f[4 * i + 4], f[4 * i + 5]),
                               pair(f[4 * i + 6], f[4 * i + 7]));
              }
            }
          }
        }
        if (in) {
          if (!whole)
            p.part_ml[at_part + my_row] = make_float2(m, l);
          else if (p.lse != nullptr)
            p.lse[token * p.lse_token + head] = log_sum(m, l);
        }
      }
      tc_fence_before();
      softmax_sync<C::kSoftThreads>();   // Q's place and the flags are free
      if (thread == 0) sh.odd_values = 0;
      if (lane == 0) mbar_arrive(&seg_free[at]);
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

// Items that end in other CTAs than they begin in, kJoinRows rows of one a CTA, their parts joined in
// the order of the keys.  What it costs is waiting for L2: a thread has four elements of kJoin parts
// and their maxima and sums on their way at a time, and meets no other.  (With the items found anew and
// the maxima and sums taken first, the trees above took 8 us longer, one short tree 31.6, not 25.7.)
constexpr int kJoinRows = 8, kJoinThreads = 256, kJoin = 4;
template <int kDC, int kRows>
__global__ void __launch_bounds__(kJoinThreads) attn_join_kernel(const __grid_constant__ AttnParams p) {
  constexpr int kD = 64 * kDC;
  grid_dep_wait();
  grid_dep_launch();
  const int first = (int)blockIdx.x, row_first = (int)blockIdx.y * kJoinRows;
  const JoinItem u = p.join[first];
  const int parts = u.last - first + 1;
  const float v_scale = p.v_scale != nullptr ? *p.v_scale : 1.0f;
#pragma unroll 1
  for (int i = threadIdx.x; i < kJoinRows * (p.head_dim / 4); i += kJoinThreads) {
    const int row = row_first + i % kJoinRows, d = i / kJoinRows * 4;
    if (row >= u.rows) continue;
    float m = -INFINITY, l = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
    for (int q0 = 0; q0 < parts; q0 += kJoin) {
      float4 v[kJoin];
      float2 ml[kJoin];
      // (past the last part its own again, with a maximum of minus infinity: no branch between the loads)
#pragma unroll
      for (int k = 0; k < kJoin; ++k) {
        const int cta = first + min(q0 + k, parts - 1);
        ml[k] = __ldcg(&p.part_ml[part_row<kRows>(cta, first, row)]);
        v[k] = __ldcg(part_sums<kRows, kD>(p, part_row<kRows>(cta, first, 0), row, d));
      }
      float now = m;
#pragma unroll
      for (int k = 0; k < kJoin; ++k) {
        if (q0 + k >= parts) ml[k].x = -INFINITY;
        now = fmaxf(now, ml[k].x);
      }
      const float base = now == -INFINITY ? 0.0f : now, keep = exp2_fast(m - base);
      l *= keep;
      o = make_float4(o.x * keep, o.y * keep, o.z * keep, o.w * keep);
#pragma unroll
      for (int k = 0; k < kJoin; ++k) {
        const float w = exp2_fast(ml[k].x - base);
        // (whatever its weight: a part of NaN scores has a weight of 0 and a NaN sum)
        if (known_here(q0 + k < parts)) {
          l = fmaf(ml[k].y, w, l);
          o = make_float4(fmaf(v[k].x, w, o.x), fmaf(v[k].y, w, o.y), fmaf(v[k].z, w, o.z), fmaf(v[k].w, w, o.w));
        }
      }
      m = now;
    }
    const int r = u.row0 + row, head = u.head0 + r % p.group;
    const int64_t token = u.token0 + r / p.group;
    const float inv = l == 0.0f ? 0.0f : v_scale / l;
    store_out4(p, token, head, d, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
    if (p.lse != nullptr && d == 0) p.lse[token * p.lse_token + head] = log_sum(m, l);
  }
}

template <bool kF16, int kDC, bool kCodes>
cudaError_t launch_cfg(TileParams tp, const CUtensorMap& tk, const CUtensorMap& tv, cudaStream_t s, Device dev) {
  using C = TileCfg<kDC, kCodes>;
  auto kern = attn_tiles_kernel<kF16, kDC, kCodes>;
  static PerDevice<cudaError_t> per_device;
  const cudaError_t e = per_device.get(dev.index, [&] {
    return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
  });
  if (e != cudaSuccess) return e;
  constexpr int64_t kPart = 2 * C::kRows * ((int64_t)64 * kDC * 4 + 8);
  const int ctas = (int)std::min<int64_t>(dev.num_sms, std::min<int64_t>(kMostCtas, (kWorkspaceBytes - kCountBytes - kJoinBytes) / kPart));
  AttnParams& p = tp.a;
  p.join = reinterpret_cast<JoinItem*>(reinterpret_cast<uint8_t*>(p.counts) + kCountBytes);
  p.part_ml = reinterpret_cast<float2*>(reinterpret_cast<uint8_t*>(p.join) + kJoinBytes);
  p.part = reinterpret_cast<float*>(p.part_ml + (int64_t)2 * C::kRows * ctas);
  p.least = 2;
  // (in us without it, with 6, 8, 11 and 15, before the join below its present form: the trees above 225, 213, 214, 213, 219; 64 of 500-1000 keys
  // 152, 135, 131, 132, 135; three of 15000-30000 keys 109, 99, 100, 95, 96; without and with 8: four of
  // 2048-4096 keys 51.6, 45.0, 16 of 250-500 52.7, 42.6)
  p.item_cost = 8;
  const cudaError_t st = launch_pdl(kern, dim3((unsigned)ctas), C::kThreads, C::kSmem, s, tk, tv, tp);
  if (st != cudaSuccess) return st;
  return launch_pdl(attn_join_kernel<kDC, C::kRows>, dim3((unsigned)ctas, C::kRows / kJoinRows), kJoinThreads, 0, s, p);
}

}  // namespace

bool attention_tiles_fit(const AttnParams& p) {
  const int tile = p.head_dim <= 128 ? 128 : 64;
  const bool pages = p.page_size % 8 == 0 && (p.page_size >= tile ? p.page_size % tile : tile % p.page_size) == 0;
  return pages && p.k_slot > 0 && p.k_head > 0 && p.k_page > 0 && p.v_slot > 0 && p.v_head > 0 && p.v_page > 0 &&
         p.tokens * p.group < (int64_t)1 << 30 && (int64_t)p.page_size * p.table_width < (int64_t)1 << 31;
}

cudaError_t launch_attention_tiles(const AttnParams& p, CacheKind kind, uint64_t timeout_ns, cudaStream_t s, Device dev) {
  const int tile = p.head_dim <= 128 ? 128 : 64, chunks = (p.head_dim + 63) / 64;
  const bool codes = kind == CacheKind::kE4m3, fp16 = kind == CacheKind::kFp16;
  TileParams tp{};
  tp.a = p;
  tp.box_rows = std::min(p.page_size, tile);
  tp.boxes = tile / tp.box_rows;
  tp.timeout_ns = timeout_ns;
  CUtensorMap tk, tv;
  const uint64_t dims[4] = {(uint64_t)p.head_dim, (uint64_t)p.page_size, (uint64_t)p.heads, (uint64_t)p.pages};
  // 16-bit: 64 elements of a box's keys, swizzled; codes: whole rows as they lie
  const uint32_t box[4] = {codes ? 64u * (uint32_t)chunks : 64u, (uint32_t)tp.box_rows, 1u, 1u};
  auto encode = [&](CUtensorMap* map, const void* base, int64_t slot, int64_t head, int64_t page) {
    return encode_tensor_map_4d(map, base, codes ? 1 : fp16 ? 3 : 2, dims, {(uint64_t)slot, (uint64_t)head, (uint64_t)page},
                                box);
  };
  if (encode(&tk, p.k, p.k_slot, p.k_head, p.k_page) != CUDA_SUCCESS ||
      encode(&tv, p.v, p.v_slot, p.v_head, p.v_page) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  auto launch = [&](auto dc) {
    constexpr int kDC = decltype(dc)::value;
    return codes  ? launch_cfg<true, kDC, true>(tp, tk, tv, s, dev)
           : fp16 ? launch_cfg<true, kDC, false>(tp, tk, tv, s, dev)
                  : launch_cfg<false, kDC, false>(tp, tk, tv, s, dev);
  };
  return chunks == 1   ? launch(std::integral_constant<int, 1>{})
         : chunks == 2 ? launch(std::integral_constant<int, 2>{})
         : chunks == 3 ? launch(std::integral_constant<int, 3>{})
                       : launch(std::integral_constant<int, 4>{});
}

}  // namespace qlin
