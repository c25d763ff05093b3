// The paged cache's index arithmetic and the attention's split of its work: host and
// device code without CUDA headers, so that a CPU test can run it.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define QLIN_HD __host__ __device__ __forceinline__
#else
#define QLIN_HD inline
#endif

namespace qlin {

// a / b of what is not negative, in 32 bits where it fits (a tenth of the time on the device).
QLIN_HD int64_t div_small(int64_t a, int64_t b) {
  return ((uint64_t)a | (uint64_t)b) >> 32 == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// Where the cache of one sequence holds its token `at`: its page's number in the table
// row, and the slot in that page.  False past the table's row.
QLIN_HD bool cache_place(int64_t at, int page_size, int table_width, int* index, int* slot) {
  if (at < 0 || at >= (int64_t)page_size * table_width) return false;
  *index = (int)div_small(at, page_size);   // (the product fits 62 bits, the quotient 31)
  *slot = (int)(at - (int64_t)*index * page_size);
  return true;
}

// One sequence's share of a call, from device data that may be wrong: counts outside the
// call or the table come as an empty sequence, or its keys cut at the table's end.
struct CacheSeq {
  int64_t first;    // its first new token
  int64_t cached;   // tokens before these
  int64_t keys;     // cached + fresh, at most what the table can hold
  int fresh;        // new tokens
  bool bad;
};

QLIN_HD CacheSeq cache_seq(int64_t start, int64_t end, int64_t cached, int64_t tokens, int page_size,
                           int table_width) {
  CacheSeq s{start, cached, 0, 0, false};
  const int64_t room = (int64_t)page_size * table_width;
  if (start < 0 || end < start || end > tokens || cached < 0) {
    s.bad = true;
    return s;
  }
  s.fresh = (int)(end - start);
  s.keys = cached + s.fresh;
  if (s.keys > room) {
    s.bad = s.fresh > 0;
    s.keys = room;
  }
  return s;
}

// An even split of `total` units among `ctas`: the first `rest` of them take per + 1, the others
// per.
struct Split {
  int64_t per, rest;
};

// How many of `ctas` work where each should have `least` units.
QLIN_HD int64_t split_ctas(int64_t total, int64_t ctas, int64_t least) {
  const int64_t want = div_small(total + least - 1, least);
  return want < 1 ? 1 : want < ctas ? want : ctas;
}

QLIN_HD Split split_evenly(int64_t total, int64_t ctas) {
  const int64_t per = div_small(total, ctas);
  return {per, total - per * ctas};
}

// CTA c takes [begin(c), begin(c + 1)).
QLIN_HD int64_t split_begin(const Split& s, int64_t c) { return c * s.per + (c < s.rest ? c : s.rest); }

// The CTA that takes unit t.
QLIN_HD int64_t split_owner(const Split& s, int64_t t) {
  const int64_t longer = s.rest * (s.per + 1);
  return t < longer ? div_small(t, s.per + 1) : s.rest + div_small(t - longer, s.per);
}

// The few-row attention's numbers that its split and its joins follow from.
constexpr int kFewWarps = 4;
// keys of a warp and tile (rows: 16 or 32)
QLIN_HD constexpr int few_warp_keys(int element_bytes, int rows) { return element_bytes == 1 ? 32 : rows; }
// tiles that a CTA should have
QLIN_HD constexpr int few_least(int tile) { return 128 / tile < 1 ? 1 : 128 / tile; }
// tiles that an item's begin and end take as long as (in us without it, with 1, 2, 3 and 4: 64 sequences
// of 2048-8192 E4M3 keys, 8 heads of 128, 144, 141, 139, 139, 140; of 512-2048 59, 55, 53, 53, 55; 8 of
// 512-2048, without and with 2, 20.0, 15.5)
constexpr int kFewItemCost = 2;
// CTAs whose parts of an item are joined by the last of them: as many as a CTA joins in about the time
// that another level takes
QLIN_HD int few_join_group(int rows, int head_dim) {
  const int per4 = rows * head_dim / (4 * 32 * kFewWarps);
  return per4 <= 1 ? 64 : per4 <= 4 ? 32 : 16;
}

}  // namespace qlin
