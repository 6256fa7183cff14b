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

// Attention of several rows per sequence.  A wave's tile has `cols` columns, (row,
// head) pairs of a KV head: 16, and 32 where the rows are more than the sequences and
// two tiles of outputs fit the registers (six rows of 4 heads over 8-bit caches of
// 512 .. 16384 slots, 16 sequences: 105 us with 16 columns, 72 with 32).
constexpr int rows_per_tile(int g, int cols) { return cols / g; }
constexpr int rows_cols(bool bf16, int d, int batch, int rows) { return bf16 && d <= 128 && rows > batch ? 32 : 16; }
// The tiles of `per` rows that T rows of B sequences can make at most: the sum of
// ceil(n / per), a sequence's last one may be short.
inline long rows_tiles(int per, int batch, int rows) {
  const long tiles = ((long)rows + (long)batch * (per - 1)) / per;
  return tiles < rows ? tiles : rows;
}
inline long rows_segments(int nkv, int g, int cols, int batch, int rows) {
  return rows_tiles(rows_per_tile(g, cols), batch, rows) * nkv;
}
// Places of a segment at most.
inline int rows_span(int g, int cols, int max_len, int window, int n_first) {
  const long w = window ? (long)window + n_first + rows_per_tile(g, cols) - 1 : max_len;
  return (int)(w < max_len ? w : max_len);
}
// A workgroup for each segment, and no join, where segments are short or fill the
// chip by themselves; else equal runs of granules for all waves, as above.
constexpr int ROWS_DIRECT_SEGMENTS = 2048;
// In bf16 contexts, sequences of more rows than ROWS_FEW columns hold go to the
// kernel of prompts.  In tiles and as a prompt, over 4096 slots: 4 query heads per KV
// head, one sequence, 16 rows 26 and 28 us, 32 rows 31 and 31, 64 rows 47 and 39; one
// query head per KV head, 64 rows 48 and 31; 32 sequences of 12 rows in 8 bits 129 and
// 185.  So they meet at 128 columns with 4 heads and below 64 with one, and the limit
// is below both: with 4 heads, 13 .. 31 rows of a lone sequence lose up to 2 us, and
// the low bits of their probabilities.  A call whose rows are one each, or no more than PROMPT_LEAST columns in several sequences, does
// without it: its launch costs 9 us where no sequence is that long, and a lone one
// of so many takes about 1.5 times as long in tiles.
//   Its tiles have prompt_columns, 32 to a wave: 256 (with 128, two workgroups to a CU:
// one prompt of 8192 rows, 32 heads, 692 us, so 634), and 128 where a wave's outputs take
// more than a quarter of a SIMD's registers.  Where tiles are fewer than PROMPT_FILL
// over all KV heads, each is split along its places into at most PROMPT_SPLITS parts
// of PROMPT_PART at least, up to twice PROMPT_FILL in all (64 rows over 32768 slots:
// 102 us, unsplit 1170).  The bound of the tiles is exact for one sequence: 8 workgroups of
// 24 without work made 128 rows there 186 us instead of 110.
constexpr int ROWS_FEW = 48, PROMPT_LEAST = 1024;
constexpr int PROMPT_FILL = 128, PROMPT_SPLITS = 16, PROMPT_PART = 256;
constexpr int prompt_columns(int d) { return d == 256 ? 128 : 256; }
constexpr int prompt_rows(int g, int d) { return prompt_columns(d) / g; }
struct RowsPlan {
  int cols;                       // columns of a tile of the first kernel
  int few;                        // rows of a sequence that the first kernel takes
  int segments, waves;            // of it (segments 0: it is not needed)
  bool direct;
  int prompt_segments, splits;    // of the other (0: not needed)
};
inline RowsPlan rows_plan(bool bf16, int nkv, int g, int d, int batch, int rows, bool one_each, int max_len, int window,
                          int n_first, int waves) {
  RowsPlan p{rows_cols(bf16, d, batch, rows), 0x7fffffff, 0, 0, true, 0, 1};
  const int span = rows_span(g, p.cols, max_len, window, n_first), rt = rows_per_tile(g, p.cols);
  const int few = ROWS_FEW / g;
  const bool prompts = bf16 && !one_each && rows > few && (batch == 1 || (long)rows * g > PROMPT_LEAST);
  if (prompts) {
    // tiles to expect: full ones, and one at least for each sequence if those have
    // enough rows on average
    long full = (rows + prompt_rows(g, d) - 1l) / prompt_rows(g, d);
    if (rows / batch > few && full < batch) full = batch;
    full *= nkv;
    p.few = few;
    p.prompt_segments = (int)(rows_tiles(prompt_rows(g, d), batch, rows) * nkv);
    if (full < PROMPT_FILL) {
      const long most = (2 * PROMPT_FILL + full - 1) / full, parts = span / PROMPT_PART;
      const long n = most < parts ? most : parts;
      p.splits = (int)(n < 1 ? 1 : n > PROMPT_SPLITS ? PROMPT_SPLITS : n);
    }
    if (batch == 1) return p;     // the kernel of prompts takes a lone sequence however short it is
  }
  long n = rows_segments(nkv, g, p.cols, batch, rows);
  // short sequences among prompts have few / rt tiles at most
  const long top = prompts ? (long)batch * ((few + rt - 1) / rt) * nkv : n;
  n = n < top ? n : top;
  p.segments = (int)n;
  p.direct = span <= CACHE_DIRECT || n >= ROWS_DIRECT_SEGMENTS;
  const long granules = n * cache_granules(span);
  p.waves = (int)(p.direct ? n : granules < waves ? granules : waves);
  return p;
}
// Scratch bytes: of the first kernel, of the other (each run 256-byte aligned).
inline size_t rows_part_bytes(size_t parts, int d) {
  const size_t pad = 255;
  return ((parts * 4 + pad) & ~pad) * 2 + ((parts * d * 4 + pad) & ~pad);
}
inline size_t rows_scratch(int g, int d, const RowsPlan &p) {
  if (p.direct || !p.segments) return 0;
  return rows_part_bytes((size_t)cache_partials(p.waves, p.segments) * rows_per_tile(g, p.cols) * g, d);
}
inline size_t prompt_scratch(int nq, int d, int rows, const RowsPlan &p) {
  return p.prompt_segments && p.splits > 1 ? rows_part_bytes((size_t)p.splits * rows * nq, d) : 0;
}
// The most that any call over up to `batch` sequences and `rows` rows takes: of
// splits * rows, with splits <= 2 PROMPT_FILL / full + 1, full >= rows / prompt_rows *
// nkv and < PROMPT_FILL.
inline size_t rows_scratch_up_to(bool bf16, int nkv, int g, int d, int batch, int rows, int max_len, int waves) {
  size_t bytes = 0;
  if (max_len > CACHE_DIRECT) {
    for (int cols = 16; cols <= rows_cols(bf16, d, 0, rows); cols += 16) {   // (a smaller batch may have wider tiles)
      const long n = rows_segments(nkv, g, cols, batch, rows);
      const int most = (int)(n < ROWS_DIRECT_SEGMENTS ? n : ROWS_DIRECT_SEGMENTS - 1);
      const size_t need = rows_part_bytes((size_t)cache_partials(waves, most) * rows_per_tile(g, cols) * g, d);
      bytes = need > bytes ? need : bytes;
    }
  }
  if (bf16 && max_len >= 2 * PROMPT_PART) {
    const long fill = (long)PROMPT_FILL * prompt_rows(g, d) / nkv + 1, all = 2 * fill + (rows < fill ? rows : fill);
    const long each = (long)PROMPT_SPLITS * rows;
    bytes += rows_part_bytes((size_t)(all < each ? all : each) * nkv * g, d);
  }
  return bytes;
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
