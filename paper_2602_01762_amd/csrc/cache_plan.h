// Launch plans, run arithmetic and scratch sizes of the long-context draft cache
// (plain C++, as plan.h, which includes this file).
#pragma once
#include "plan.h"

namespace prism {

// Attention over the long-context cache, for `units` pairs of a sequence and
// a KV head of up to `span` places: the waves that share the granules of
// CACHE_GRAN places.
constexpr int CACHE_GRAN = 64;      // whole tiles of every attention kernel
// That many are resident at once (8 on each of 256 CUs, two per SIMD; 4 where a
// row of 1024 bytes, fp32 and d = 256, takes more than half a SIMD's registers),
// and each pays its first lookups once.  32 sequences of 32768 slots, 64 query
// heads: 669 us, with 1024 waves 680, 4096 690, 8192 726; fp32 with d = 256, one
// sequence of 32768: 72 us, with 2048 waves 90.
constexpr int CACHE_WAVES = 2048;
constexpr int cache_waves(int row_bytes) { return row_bytes > 512 ? CACHE_WAVES / 2 : CACHE_WAVES; }
// A direct call gives each segment to one workgroup, which needs no join: up to
// CACHE_DIRECT places (128 segments of 512: 13.0 us, joined 14.4; 8 of 512: 10.6
// and 10.5, of 768: 14.4 and 11.2), and up to CACHE_DIRECT_MANY where CACHE_DIRECT_UNITS segments fill
// the chip (256 segments of 1024: 25.7 us, joined 30.1; of 1 .. 1024, whose
// lengths the host does not know: 23.0 and 21.9).
constexpr int CACHE_DIRECT = 512, CACHE_DIRECT_MANY = 1024, CACHE_DIRECT_UNITS = 256;
// The arithmetic of the runs, which kernels, runtime and tests share.  Granules
// of a segment (a sequence's KV head) and of a wave's run:
constexpr int cache_granules(int places) { return (places + CACHE_GRAN - 1) / CACHE_GRAN; }
constexpr int cache_run(int total, int waves) { return total > waves ? (total - 1) / waves + 1 : 1; }
struct CachePlan {
  int waves;
  bool direct;
};
inline CachePlan cache_plan(int units, int span, bool weights, int waves = CACHE_WAVES) {
  if (span <= (units >= CACHE_DIRECT_UNITS ? CACHE_DIRECT_MANY : CACHE_DIRECT) && !weights) return {units, true};
  const long granules = (long)units * cache_granules(span);
  return {(int)(granules < waves ? granules : waves), false};
}
// The part of a segment that the run with `left` granules to go begins with, at
// granule `at` of a sequence whose heads have `count` each.
struct CacheRun {
  int head, first, granules;
};
constexpr CacheRun cache_run_at(int at, int count, int left) {
  const int head = at / count, first = at - head * count;
  return {head, first, left < count - first ? left : count - first};
}
// Partial of a wave for a segment (units: segments before it): along the runs
// each step moves on one wave or one segment, so no two share one.
constexpr int cache_partial(int wave, int segment) { return wave + segment; }
constexpr int cache_partials(int waves, int units) { return waves + units; }
// The waves whose runs touch the segment of `count` granules from `begin` on.
struct CacheParts {
  int wave, n;
};
constexpr CacheParts cache_parts(int begin, int count, int run) {
  const int wave = begin / run;
  return {wave, count ? (begin + count - 1) / run - wave + 1 : 0};
}
// row length of the scores kept for the slot weights: whole granules
inline int cache_score_row(int span) { return cache_granules(span) * CACHE_GRAN; }
// Scratch bytes of an attention call over `batch` sequences with nkv KV heads of
// g query heads and d channels, shared by at most `waves` waves: two statistics and an output of each partial
// (256-byte aligned runs), and the kept scores.
inline size_t cache_attend_scratch(int batch, int nkv, int g, int d, int span, bool weights, int waves = CACHE_WAVES) {
  const CachePlan p = cache_plan(batch * nkv, span, weights, waves);
  if (p.direct) return 0;
  const size_t parts = (size_t)cache_partials(p.waves, batch * nkv) * g, pad = 255;
  size_t n = ((parts * 4 + pad) & ~pad) * 2 + ((parts * d * 4 + pad) & ~pad);
  if (weights) n += (size_t)batch * nkv * g * cache_score_row(span) * 4;
  return n;
}
// The most that any batch up to this one takes: a larger one may be direct, and
// take none, where a smaller one is not.
inline size_t cache_attend_scratch_up_to(int batch, int nkv, int g, int d, int span, bool weights,
                                         int waves = CACHE_WAVES) {
  size_t most = 0;
  for (int b = 1; b <= batch; ++b) {
    const size_t n = cache_attend_scratch(b, nkv, g, d, span, weights, waves);
    most = n > most ? n : most;
  }
  return most;
}

// Table columns per wave of the passes over the blocks of a cache (summaries,
// scores), for units * columns of them at most: about `waves` waves, a multiple
// of `step` columns (those of one load), at most `top` <= 64 (one lane looks up
// each).  Scores take fewer waves, since each has queries to convert (131071
// slots, 8 KV heads of 4 queries, the whole sparse step: 2048 waves 32.5 us,
// 4096 34.1, 8192 40.2).
constexpr int CACHE_SUM_WAVES = 4096, CACHE_SUM_COLUMNS = 8;
constexpr int CACHE_SCORE_WAVES = 2048, CACHE_SCORE_COLUMNS = 64;
inline int cache_columns_per_wave(long units, int columns, int step, int top, int waves) {
  const long steps = (units * columns + (long)waves * step - 1) / ((long)waves * step);
  const long most = top / step;
  return (int)(steps < 1 ? 1 : steps > most ? most : steps) * step;
}

// Choice of the best of many candidates: up to CHOOSE_LDS have their keys in one
// workgroup's LDS; more slots go through scratch, in segments of CHOOSE_SEG keys
// with a histogram of 1024 words, a list of the keys at the cut and four words
// of counts each.
constexpr int CHOOSE_LDS = 24576, CHOOSE_SEG = 4096;
constexpr int CHOOSE_MAX_SEGS = ATT_MAX_CHUNKS * ATT_STEP * ATT_MAX_SUB / CHOOSE_SEG;   // of a context's capacity
inline int choose_key_row(int most) { return (most + 3) / 4 * 4; }
inline int choose_segs(int most) { return most > CHOOSE_LDS ? (most + CHOOSE_SEG - 1) / CHOOSE_SEG : 0; }
inline int choose_hist_row(int most) { return choose_segs(most) * 1024; }
inline int choose_list_row(int most) { return choose_segs(most) * CHOOSE_SEG; }
inline int choose_cut_row(int most) { return choose_segs(most) ? 4 + 4 * choose_segs(most) : 0; }
inline size_t choose_scratch(size_t units, int most) {
  return units * ((size_t)choose_key_row(most) + choose_hist_row(most) + choose_list_row(most) + choose_cut_row(most)) * 4;
}

}  // namespace prism
