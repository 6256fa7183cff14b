// Declarations of the long-context draft cache, shared by its kernels
// (cache.hip) and the runtime.
#pragma once
#include "internal.h"

namespace prism {

// The sequences of one call and their paged cache.  Sequence b sees its
// context of kv.ctx_lens[b] slots plus n_new, at most max_len (<= mbps * bs).
struct CacheView {
  KvArgs kv;
  int nkv;
  int n_new, max_len;
};
struct CacheAppend {
  CacheView v;
  int rows, nq;
  const int32_t *offsets, *positions;   // [B + 1] / [B], or NULL
  const void *qkv;                      // [rows, (nq + 2 nkv) d]
  const void *q_gain, *k_gain;          // [d] or NULL
  void *q;                              // [rows, nq d]
  float *weights;                       // slot weights, or NULL
  const double *inv_freq;
  float eps;
  uint32_t *err;
};
void launch_cache_append(bool bf16, const CacheAppend &a, int d, hipStream_t s);
struct CacheAttend {
  CacheView v;
  int nq, g, d;
  const void *q;                        // [B, nq, d]
  const int32_t *blocks; int n_list;    // [B, nkv, n_list] or NULL
  int span;                             // places per sequence: max_len, or all of a list's first
                                        // mbps entries
  int waves, direct;                    // cache_plan
  float scale;                          // log2(e) / sqrt(d)
  float *pm, *pl, *po;                  // partials [waves + B * nkv][g] / [.., d]
  float *scores; int ld_scores;         // [B, nkv, ld_scores / 16, g, 16] in base 2 (weights only)
  void *out; float *lse;                // [B, nq, d] / [B, nq] or NULL
  float *weights;                       // slot weights, or NULL
  uint32_t *err;
};
void launch_cache_attend(bool bf16, const CacheAttend &a, hipStream_t s);
struct CacheSummarize {
  CacheView v;
  int span, columns;                    // last slots covered (0: all), table columns they may touch
  int per;                              // columns per wave, 1..64
  void *summary;                        // [n_blocks, nkv, 2, d]
  uint32_t *err;
};
void launch_cache_summarize(bool bf16, const CacheSummarize &a, int d, hipStream_t s);
struct CacheSelect {
  CacheView v;
  int nq, g;
  const void *q, *summary;
  int n_take, n_first, n_last, columns; // columns: table columns of max_len slots
  int per;                              // columns per wave, 1..64
  uint32_t *keys; int ld_keys;          // [B, nkv, ld_keys]
  int32_t *out;                         // [B, nkv, n_take]
  uint32_t *err;
};
void launch_cache_select(bool bf16, const CacheSelect &a, int d, hipStream_t s);
struct CacheChoose {
  CacheView v;
  const uint32_t *keys; int ld_keys;    // [B, nkv, ld_keys], ld_keys a multiple of 4
  const uint32_t *hists; int ld_hists;  // first digits per CHOOSE_SEG keys, 1024 words each, or NULL
  uint32_t *cand; int ld_cand;          // (with hists) listed keys, CHOOSE_SEG per segment
  uint32_t *cut; int ld_cut;            // (with hists)
  const float *weights;                 // slot weights to make the keys from, or NULL
  int per_block;                        // candidates are blocks (else slots)
  int n_take, n_first, n_last;          // (n_first, n_last: with weights)
  int32_t *out, *lens;                  // [B, nkv, n_take]; [B] counts taken, or NULL
  uint32_t *err;
};
struct CacheEvict {
  CacheView v;
  const int32_t *new_table;             // [B, mbps]
  float *weights;
  int n_keep, n_first, n_recent;
  uint32_t *keys; int ld_keys;          // [B, nkv, ld_keys]
  // more than CHOOSE_LDS candidates: per (sequence, KV head) the segments'
  // histograms, listed keys and cuts
  uint32_t *hists; int ld_hists;
  uint32_t *cand; int ld_cand;
  uint32_t *cut; int ld_cut;
  int32_t *kept, *new_lens;             // [B, nkv, n_keep] / [B]
  uint32_t *err;
};
void launch_cache_evict(bool bf16, const CacheEvict &a, int d, hipStream_t s);

}  // namespace prism
