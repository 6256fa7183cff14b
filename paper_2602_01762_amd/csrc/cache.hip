// Long-context draft cache: rows appended to the paged cache with per-head
// norms and rotation, attention of one token per sequence over the whole cache
// or a list of its blocks (with the weight that every slot receives), block
// summaries and the selection of blocks by them, and eviction by accumulated
// weight.
//
// Pools are [block, KV head, slot in block, d]: row (block, head, slot) of a
// pool seen as [rows, d] has a 32-bit index (the runtime refuses larger pools).
#include "cache.h"
#include "cache_device.h"
#include "rotation.h"

namespace prism {

// Inclusive maximum over the lanes below, as wave_scan.
__device__ __forceinline__ uint32_t wave_scan_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false));
  return v;
}

// ---------------------------------------------------------------- append
// One lane group of d / 16 lanes per head: lane i holds dims 8i .. 8i+7 and
// their rotation partners d/2 + 8i ...  The angles of a row are the same for
// all its heads: d / 2 threads of the workgroup compute them once.
template <typename T, int D>
__global__ __launch_bounds__(512) void k_cache_append(CacheAppend a) {
  constexpr int LPH = D / 16, HPW = 64 / LPH;      // lanes per head, heads per wave
  const int r = blockIdx.x, tid = threadIdx.x, wave = wave_id(), lane = tid & 63;
  __shared__ float cs[D / 2], sn[D / 2];
  const int nh = a.nq + 2 * a.v.nkv;
  const int h = (blockIdx.y * (blockDim.x >> 6) + wave) * HPW + lane / LPH, li = lane % LPH;
  const bool has = h < nh;
  float x1[8], x2[8];
  const T *row = (const T *)a.qkv + ((size_t)r * nh + (has ? h : 0)) * D + 8 * li;
  load8f<T>(row, x1);
  load8f<T>(row + D / 2, x2);
  // sequence of the row, at most 64 of them: one lane per sequence
  int b = r, at = 0;
  if (a.offsets) {
    const int B = a.v.kv.n_seq;
    const int lo = lane < B ? a.offsets[lane] : 0, hi = lane < B ? a.offsets[lane + 1] : 0x7fffffff;
    const bool bad = lane < B && (hi < lo || hi > a.rows || (lane == 0 && lo != 0));
    if (__ballot(bad)) {                            // the same in every wave of every workgroup
      if (tid == 0 && r == 0) atomicOr(a.err, ERRF_ROWS);
      return;
    }
    b = __popcll(__ballot(lane < B && hi <= r));
    if (b >= B) return;                             // a row behind the last sequence
    at = r - __builtin_amdgcn_readlane(lo, __builtin_amdgcn_readfirstlane(b));
  }
  const int L = a.v.kv.ctx_lens[b];
  const int pos0 = a.positions ? a.positions[b] : L;
  for (int i = tid; i < D / 2; i += blockDim.x)
    rotation_cos_sin((double)((long)pos0 + at) * a.inv_freq[i], cs[i], sn[i]);
  __syncthreads();
  if (!has) return;
  const bool is_q = h < a.nq, is_v = h >= a.nq + a.v.nkv;
  if (!is_v) {
    const T *gain = (const T *)(is_q ? a.q_gain : a.k_gain);
    if (gain) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss += x1[i] * x1[i] + x2[i] * x2[i];
#pragma unroll
      for (int m = 1; m < LPH; m *= 2) ss += __shfl_xor(ss, m, 64);
      const float rs = 1.0f / sqrtf(ss / (float)D + a.eps);
      float g1[8], g2[8];
      load8f<T>(gain + 8 * li, g1);
      load8f<T>(gain + D / 2 + 8 * li, g2);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x1[i] *= rs * g1[i];
        x2[i] *= rs * g2[i];
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float c = cs[8 * li + i], s = sn[8 * li + i], u = x1[i], w = x2[i];
      x1[i] = u * c - w * s;
      x2[i] = w * c + u * s;
    }
  }
  if (is_q) {
    T *o = (T *)a.q + ((size_t)r * a.nq + h) * D + 8 * li;
    store8f<T>(o, x1);
    store8f<T>(o + D / 2, x2);
    return;
  }
  const int j = is_v ? h - a.nq - a.v.nkv : h - a.nq;
  const long t = (long)L + at;
  uint32_t prow = NO_ROW;
  if (L < 0 || t >= (long)a.v.kv.mbps * a.v.kv.bs) {
    atomicOr(a.err, ERRF_CAPACITY);
  } else {
    const int bi = slot_block(a.v.kv, (int)t);
    prow = pool_row(a.v, a.v.kv.block_table, b, j, bi, slot_in_block(a.v.kv, (int)t, bi), a.err);
  }
  if (prow == NO_ROW) return;
  T *o = (T *)(is_v ? a.v.kv.v_pool : a.v.kv.k_pool) + (size_t)prow * D + 8 * li;
  store8f<T>(o, x1);
  store8f<T>(o + D / 2, x2);
  if (a.weights && is_v && li == 0) a.weights[prow] = 0.f;
}

template <typename T>
static void append_d(const CacheAppend &a, int d, hipStream_t s) {
  const int hpw = 64 / (d / 16), nh = a.nq + 2 * a.v.nkv;
  const int nw = min(8, (nh + hpw - 1) / hpw);
  const dim3 g(a.rows, (nh + nw * hpw - 1) / (nw * hpw)), t(64 * nw);
  if (d == 32) hipLaunchKernelGGL((k_cache_append<T, 32>), g, t, 0, s, a);
  else if (d == 64) hipLaunchKernelGGL((k_cache_append<T, 64>), g, t, 0, s, a);
  else if (d == 128) hipLaunchKernelGGL((k_cache_append<T, 128>), g, t, 0, s, a);
  else hipLaunchKernelGGL((k_cache_append<T, 256>), g, t, 0, s, a);
}
void launch_cache_append(bool bf16, const CacheAppend &a, int d, hipStream_t s) {
  if (bf16) append_d<bf16_t>(a, d, s);
  else append_d<float>(a, d, s);
}

// ---------------------------------------------------------------- attention
// A call walks sequence b's "places" p: slot p, or with a block list slot p %
// bs of block list[p / bs].  The places of one sequence and KV head are cut
// into granules of CACHE_GRAN places, the granules of all sequences and heads are
// numbered in (sequence, head, place) order, and wave w takes the w-th run of
// equally many of them.  So every wave streams the same amount whatever the
// lengths, and one long sequence among short ones fills the chip as equal
// ones do.  A run covers parts of one or more segments (sequence, KV head);
// for each it leaves, per query head, the maximum, the sum and the
// unnormalised output of the softmax in base 2 in partial w + segment (unique:
// along the runs each step moves on one wave or one segment).  The join adds a
// segment's partials in order, so the result does not depend on scheduling.
constexpr int CACHE_MAXG = 8;

// The numbering of the granules, in every lane of a wave.
struct Walk {
  int n, count, begin, end;   // lane b: visible slots; granules per head, before and through sequence b
  int total, per;             // granules in all, granules per wave
};
__device__ __forceinline__ int places_of(const CacheAttend &a, int n) { return a.blocks ? a.span : min(n, a.span); }
__device__ __forceinline__ Walk walk_of(const CacheAttend &a) {
  const int lane = threadIdx.x & 63;
  const bool has = lane < a.v.kv.n_seq;
  Walk w;
  w.n = has ? visible_slots(a.v, lane, a.err) : 0;
  w.count = has ? cache_granules(places_of(a, w.n)) : 0;
  if (a.direct && has) w.count = 1;            // an empty sequence writes its zeros itself
  w.end = w.count * a.v.nkv;
  for (int x = 1; x < a.v.kv.n_seq; x *= 2) {
    const int v = __shfl_up(w.end, x, 64);
    if (lane >= x) w.end += v;
  }
  w.total = __builtin_amdgcn_readlane(w.end, a.v.kv.n_seq - 1);
  if (!has) w.end = w.total;
  w.begin = w.end - w.count * a.v.nkv;
  w.per = cache_run(w.total, a.waves);
  return w;
}
// Where the score of place p and head h of a KV head is kept: 16 places of all
// its heads together, so that a wave's scores are one run of memory.
__device__ __forceinline__ size_t score_at(const CacheAttend &a, int b, int j, int h, int p) {
  return ((((size_t)b * a.v.nkv + j) * (a.ld_scores >> 4) + (p >> 4)) * a.g + h) * 16 + (p & 15);
}
// The part of a segment that a run starting at granule u (< w.total) and
// ending at `last` begins with.
struct Segment {
  int b, j, n, granules, p0, p1;
};
__device__ __forceinline__ Segment segment_at(const CacheAttend &a, const Walk &w, int u, int last) {
  Segment s;
  s.b = __popcll(__ballot(w.end <= u));        // wave-uniform
  const int count = __builtin_amdgcn_readlane(w.count, s.b);
  const int at = u - __builtin_amdgcn_readlane(w.begin, s.b);
  s.n = __builtin_amdgcn_readlane(w.n, s.b);
  const CacheRun run = cache_run_at(at, count, last - u);
  s.j = run.head;
  s.granules = run.granules;
  s.p0 = run.first * CACHE_GRAN;               // (0 in a direct call, whose one granule is the segment)
  s.p1 = a.direct ? places_of(a, s.n) : min(places_of(a, s.n), (run.first + s.granules) * CACHE_GRAN);
  return s;
}

// Lookup of a segment's places, in the steps that their loads allow: the
// table column of a place (from the list), the block of the column, the pool
// row.  The loads are made for every place (past the end for the last one), so
// that they can be issued early and counted.
//   An entry of a list is read if it is larger than every entry before it and
// none of them is -1, so that no block is read twice whatever the list holds.
// A wave keeps that of 64 entries at a time: begin() looks through the list up
// to them, advance() moves on (a load that is waited for, every 64 entries).
struct Lookup {
  const CacheAttend &a;
  const Segment &s;
  const int32_t *table, *list;
  int first = 0;         // entries first .. first + 63:
  uint64_t rising = 0;   // bit i: entry first + i is to be read
  uint32_t most = 0;     // lane i: the largest rank of entries up to first + i
  __device__ __forceinline__ Lookup(const CacheAttend &a_, const Segment &s_)
      : a(a_), s(s_), table(a_.v.kv.block_table + (size_t)s_.b * a_.v.kv.mbps),
        list(a_.blocks ? a_.blocks + ((size_t)s_.b * a_.v.nkv + s_.j) * a_.n_list : nullptr) {}
  __device__ __forceinline__ int entry(int p) const { return slot_block(a.v.kv, min(p, s.p1 - 1)); }
  // an entry's place in the order: nothing is larger than -1, and what is no
  // block is larger than nothing
  static __device__ __forceinline__ uint32_t rank(int id) { return id >= 0 ? (uint32_t)id + 1u : id == -1 ? ~0u : 0u; }
  __device__ __forceinline__ void window(int c, int id, uint32_t before) {
    most = max(wave_scan_max(rank(id)), before);
    const uint32_t below = __shfl_up(most, 1, 64);
    rising = __ballot(id >= 0 && rank(id) > ((threadIdx.x & 63) ? below : before));
    first = c;
  }
  // the loads of begin(), for the entries from place p on
  struct Start {
    int id, early;
  };
  __device__ __forceinline__ Start start(int p) const {
    if (!list) return {0, 0};
    const int lane = threadIdx.x & 63, c = entry(p);
    return {list[min(c + lane, entry(s.p1))], c ? list[min(lane, c - 1)] : -2};
  }
  __device__ __forceinline__ void begin(int p, const Start &st) {
    if (!list) return;
    const int lane = threadIdx.x & 63, c = entry(p);
    uint32_t v = rank(st.early);
#pragma unroll 4
    for (int i = 64; i < c; i += 64) v = max(v, rank(list[min(i + lane, c - 1)]));
    window(c, st.id, (uint32_t)__builtin_amdgcn_readlane((int)wave_scan_max(v), 63));
  }
  // the entries of places p .. p + 63 at most become those at hand (p not
  // below that of the call before)
  __device__ __forceinline__ void advance(int p, int places) {
    if (!list) return;
    const int lane = threadIdx.x & 63, c = entry(p), c1 = entry(p + places - 1), end = entry(s.p1);
    while (c >= first + 64)
      window(first + 64, list[min(first + 64 + lane, end)], (uint32_t)__builtin_amdgcn_readlane((int)most, 63));
    if (c1 >= first + 64)
      window(c, list[min(c + lane, end)], (uint32_t)__builtin_amdgcn_readlane((int)most, c - 1 - first));
  }
  __device__ __forceinline__ int column(int p) const { return list ? list[entry(p)] : entry(p); }
  __device__ __forceinline__ int block(int id) const { return table[id >= 0 && id < a.v.kv.mbps ? id : 0]; }
  __device__ __forceinline__ uint32_t row(int p, int id, int blk) const {
    const KvArgs &kv = a.v.kv;
    if (p >= s.p1 || id == -1) return NO_ROW;
    const int e = slot_block(kv, p);
    if (list && (!((rising >> (e - first)) & 1) || (long)id * kv.bs >= s.n)) {
      atomicOr(a.err, ERRF_ROWS);
      return NO_ROW;
    }
    const int off = p - e * kv.bs;
    if ((long)id * kv.bs + off >= s.n) return NO_ROW;
    if (blk < 0 || blk >= kv.n_blocks) {
      atomicOr(a.err, ERRF_CAPACITY);
      return NO_ROW;
    }
    return ((uint32_t)blk * a.v.nkv + s.j) * kv.bs + off;
  }
};

// A wave takes tiles of TS places.  K and V rows are loaded whole, 16 bytes per
// lane, so that every cache line is requested once, into registers, and pass
// through LDS into operand order: the scores are MFMAs of 16 slots x 16 heads
// (K rows as A, the queries as B), the outputs MFMAs of 16 dims x 16 heads (V
// transposed by the LDS read as A, the probabilities, straight from the score
// layout, as B).  fp32 caches use the fp32 MFMAs, which take the same 16-byte
// pieces four values at a time (on the vector units 8 heads per KV head were
// bound by arithmetic at 3.2 TB/s).
// Each lane then holds one head's softmax state and output, so nothing is
// exchanged but the maximum and the sum over the four lane rows.  The next
// tile's rows are in flight while one is computed, and the block-table
// entries of the one after it.
//   In LDS the 16-byte pieces of row s are permuted by s, so that both the
// A-operand reads (16 rows, one piece) and the transposing reads (4 rows, the
// pieces of 16 dims) spread over all banks.
//   In bf16 caches a probability is multiplied as the sum of three bf16, which
// hold its 24 bits exactly (split_bf16).

//   Scores that are kept (KEEP, for the slot weights) gather in 4 KB of LDS
// and are stored a buffer at a time, ahead of the next loads.  Stores count
// with the loads and retire in order with them, so each one delays the wait
// for a tile's rows: 16 sequences of up to 16384 slots took 109 us with a store
// per tile, 93 without any, 105 so.
//   NW > 1 (direct calls): a workgroup per segment, whose waves take its tiles
// in turn and meet in LDS.
template <typename T, int D, bool KEEP, int NW>
__global__ __launch_bounds__(64 * NW, D * sizeof(T) > 512 ? 1 : 2) void k_cache_attend(CacheAttend a) {
  using M = Tile<T, D>;
  constexpr int TS = M::TS, LPR = M::LPR, RPI = M::RPI, NI = M::NI, E = 16 / sizeof(T);   // E: values of a piece
  constexpr int NS = TS / 16, NK = LPR / 4, ND = D / 16;
  __shared__ __attribute__((aligned(16))) char sh_k[NW][TS * LPR * 16], sh_v[NW][TS * LPR * 16];
  constexpr int KEPT = 1024;                                // scores in LDS
  __shared__ __attribute__((aligned(16))) float s_s[KEEP ? KEPT : 4];
  const int wave = NW > 1 ? wave_id() : 0, lane = threadIdx.x & 63, g = a.g;
  char *s_k = sh_k[wave], *s_v = sh_v[wave];
  const int most = KEPT / (g * TS) * TS;                    // places whose scores fit (g <= 8: at least one tile)
  const int col = lane & 15, q4 = lane >> 4, grp = lane / LPR, li = lane % LPR;
  const KvArgs &kv = a.v.kv;
  const Walk wk = walk_of(a);
  int u = blockIdx.x * wk.per;
  const int last = min(wk.total, u + wk.per);
  while (u < last) {
    const Segment sg = segment_at(a, wk, u, last);
    u += sg.granules;
    Lookup lk(a, sg);
    const size_t hi = (size_t)sg.b * a.nq + sg.j * g + col;   // this lane's query head (col < g)
    u32x4 kr[NI], vr[NI];
    auto load = [&](uint32_t row) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const uint32_t r = __shfl(row, i * RPI + grp, 64);
        const size_t at = (size_t)(r == NO_ROW ? 0 : r) * D + E * li;   // a masked place reads row 0
        kr[i] = stream16((const T *)kv.k_pool + at);
        vr[i] = stream16((const T *)kv.v_pool + at);
      }
    };
    float m_run = -INFINITY, l_run = 0.f;
    f32x4 o[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    u32x4 qf[NK];
#pragma unroll
    for (int kk = 0; kk < NK; ++kk)
      qf[kk] = col < g ? *(const u32x4 *)((const T *)a.q + hi * D + (4 * kk + q4) * E) : u32x4{0, 0, 0, 0};
    int id1, b1, id2;
    uint32_t row = NO_ROW;
    int kept = sg.p0;                                       // first place whose scores are in LDS
    auto store_scores = [&](int to) {                       // places kept .. to - 1
      wave_lds_sync();
      float *ps = a.scores + score_at(a, sg.b, sg.j, 0, kept);
      for (int i = 4 * lane; i < (to - kept) * g; i += 256) *(f32x4 *)(ps + i) = *(const f32x4 *)(s_s + i);
      wave_lds_sync();
      kept = to;
    };
    constexpr int STEP = NW * TS;
    const int t0 = sg.p0 + wave * TS;
    if (t0 < sg.p1) {
      const int id0 = lk.column(t0 + lane);
      const typename Lookup::Start st = lk.start(t0);
      id1 = lk.column(t0 + STEP + lane);
      id2 = lk.column(t0 + 2 * STEP + lane);
      const int b0 = lk.block(id0);
      b1 = lk.block(id1);
      lk.begin(t0, st);
      row = lane < TS ? lk.row(t0 + lane, id0, b0) : NO_ROW;
      load(row);
    }
    for (int t = t0; t < sg.p1; t += STEP) {
      const uint64_t mask = __ballot(row != NO_ROW);   // lanes TS .. 63 hold none
      constexpr uint64_t FULL = TS == 64 ? ~0ull : (1ull << (TS & 63)) - 1;
      // rows to LDS; V rows of masked places as zeros (a NaN there must not
      // meet a probability of 0)
      if (mask != FULL) {
#pragma unroll
        for (int i = 0; i < NI; ++i)
          if (!((mask >> (i * RPI + grp)) & 1)) vr[i] = u32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        *(u32x4 *)(s_k + M::at(i * RPI + grp, li)) = kr[i];
        *(u32x4 *)(s_v + M::at(i * RPI + grp, li)) = vr[i];
      }
      if constexpr (KEEP)
        if (t - kept == most) store_scores(t);
      // the lookups of the tile after the next one, and the next one's rows
      if (t + STEP < sg.p1) {
        lk.advance(t + STEP, TS);
        row = lane < TS ? lk.row(t + STEP + lane, id1, b1) : NO_ROW;
        id1 = id2;
        b1 = lk.block(id1);
        id2 = lk.column(t + 3 * STEP + lane);
        load(row);
      }
      wave_lds_sync();
      // scores S[slot 16 st + 4 q4 + i][head col]
      f32x4 sc[NS];
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        sc[st] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < NK; ++kk)
          sc[st] = Ty<T>::mma(*(const u32x4 *)(s_k + M::at(16 * st + col, 4 * kk + q4)), qf[kk], sc[st]);
      }
      float mx = -INFINITY;
#pragma unroll
      for (int st = 0; st < NS; ++st)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sc[st][i] = ((mask >> (16 * st + 4 * q4 + i)) & 1) ? sc[st][i] * a.scale : -INFINITY;
          mx = fmaxf(mx, sc[st][i]);
        }
      if constexpr (KEEP) {
        if (col < g) {
#pragma unroll
          for (int st = 0; st < NS; ++st) *(f32x4 *)(s_s + (t - kept + 16 * st) * g + 16 * col + 4 * q4) = sc[st];
        }
      }
      mx = fmaxf(mx, xor16_f(mx));
      mx = fmaxf(mx, xor32_f(mx));
      const float mn = fmaxf(m_run, mx);
      // nothing but -inf so far: subtract 0, so that every p is 0 (a NaN score
      // still makes its p, and with it the sum and the output, NaN)
      const float ms = mn == -INFINITY ? 0.f : mn;
      const float al = __builtin_amdgcn_exp2f(m_run - ms);
      m_run = mn;
      float ls = 0.f;
#pragma unroll
      for (int st = 0; st < NS; ++st)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sc[st][i] = __builtin_amdgcn_exp2f(sc[st][i] - ms);
          ls += sc[st][i];
        }
      ls += xor16_f(ls);
      ls += xor32_f(ls);
      l_run = l_run * al + ls;
      if (__ballot(al != 1.f)) {
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) o[dt] *= al;
      }
      // O[dim 16 dt + 4 q4 + i][head col]
      constexpr int NP = sizeof(T) == 2 && NS > 1 ? 2 : 1;   // groups of 16 slots per bf16 MFMA (32 slots, or 16)
#pragma unroll
      for (int st = 0; st < NS; st += NP) {
        if constexpr (sizeof(T) == 2) {
          uint32_t hi[NP][2], mid[NP][2], lo[NP][2];
#pragma unroll
          for (int x = 0; x < NP; ++x) split_bf16(sc[st + x], hi[x], mid[x], lo[x]);
#pragma unroll
          for (int dt = 0; dt < ND; ++dt) {
            uint2 v[NP];
#pragma unroll
            for (int x = 0; x < NP; ++x) {
              const char *pv = s_v + M::at(16 * (st + x) + 4 * q4 + (col >> 2), 2 * dt + ((col & 3) >> 1)) + 8 * (col & 1);
              v[x] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)pv));
            }
            if constexpr (NP == 2) {
              // k = 8 q4 + e: slots 16 st + 4 q4 + e, then the same of st + 1, in both operands
              const u32x4 vv = {v[0].x, v[0].y, v[1].x, v[1].y};
              o[dt] = Ty<T>::mma(vv, u32x4{hi[0][0], hi[0][1], hi[1][0], hi[1][1]}, o[dt]);
              o[dt] = Ty<T>::mma(vv, u32x4{mid[0][0], mid[0][1], mid[1][0], mid[1][1]}, o[dt]);
              o[dt] = Ty<T>::mma(vv, u32x4{lo[0][0], lo[0][1], lo[1][0], lo[1][1]}, o[dt]);
            } else {
              const s16x4 vv = __builtin_bit_cast(s16x4, v[0]);
              o[dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vv, __builtin_bit_cast(s16x4, uint2{hi[0][0], hi[0][1]}), o[dt], 0, 0, 0);
              o[dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vv, __builtin_bit_cast(s16x4, uint2{mid[0][0], mid[0][1]}), o[dt], 0, 0, 0);
              o[dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vv, __builtin_bit_cast(s16x4, uint2{lo[0][0], lo[0][1]}), o[dt], 0, 0, 0);
            }
          }
        } else {
          // step i: slot 4 q4 + i of each lane row
#pragma unroll
          for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const char *pv = s_v + M::at(16 * st + 4 * q4 + i, 4 * dt + (col >> 2)) + 4 * (col & 3);
              o[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(*(const float *)pv, sc[st][i], o[dt], 0, 0, 0);
            }
        }
      }
      wave_lds_sync();                                 // reads done before the next tile's writes
    }
    if constexpr (KEEP)
      if (sg.p0 < sg.p1) store_scores(sg.p0 + (sg.p1 - sg.p0 + TS - 1) / TS * TS);
    if constexpr (NW > 1) {
      __shared__ float s_m[NW][16], s_l[NW][16];
      float *so = (float *)s_k;                        // this wave's outputs [g][D]: within its K tile
      if (col < g) {
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) *(f32x4 *)(so + col * D + 16 * dt + 4 * q4) = o[dt];
      }
      if (q4 == 0) {
        s_m[wave][col] = m_run;
        s_l[wave][col] = l_run;
      }
      __syncthreads();
      for (int e = threadIdx.x; e < g * D / 4; e += 64 * NW) {
        const int h = e / (D / 4);
        float M2 = -INFINITY, l = 0.f;
        for (int w = 0; w < NW; ++w) M2 = fmaxf(M2, s_m[w][h]);
        M2 = M2 == -INFINITY ? 0.f : M2;
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < NW; ++w) {
          const float wt = __builtin_amdgcn_exp2f(s_m[w][h] - M2);
          l += s_l[w][h] * wt;
          y += *(const f32x4 *)((const float *)sh_k[w] + 4 * e) * wt;
        }
        if (l == 0.f) y = f32x4{0.f, 0.f, 0.f, 0.f};   // (0 times a value that is not finite)
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const float z[4] = {y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv};
        store_n<T, 4>((T *)a.out + ((size_t)sg.b * a.nq + sg.j * g) * D + 4 * e, z);
        if (a.lse && e % (D / 4) == 0)
          a.lse[(size_t)sg.b * a.nq + sg.j * g + h] = l == 0.f ? -INFINITY : (M2 + log2f(l)) * LN2;
      }
      return;                                          // one segment per workgroup
    }
    if (col >= g) continue;
    const size_t part = (size_t)cache_partial(blockIdx.x, sg.b * a.v.nkv + sg.j) * g + col;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) *(f32x4 *)(a.po + part * D + 16 * dt + 4 * q4) = o[dt];
    if (q4 == 0) {
      a.pm[part] = m_run;
      a.pl[part] = l_run;
    }
  }
}

// The partials of one query head: np of them, entry i of pm / pl at at + i * g.
struct Parts {
  size_t at;
  int np;
};
__device__ __forceinline__ Parts parts_of(const CacheAttend &a, const Walk &w, int b, int j, int h) {
  const int count = __builtin_amdgcn_readlane(w.count, b);
  const CacheParts p = cache_parts(__builtin_amdgcn_readlane(w.begin, b) + j * count, count, w.per);
  return {(size_t)cache_partial(p.wave, b * a.v.nkv + j) * a.g + h, p.n};
}
// From every lane of a wave: the largest maximum M (0 if there is none) and
// the sum l of 2^(m_c - M) l_c.
__device__ __forceinline__ void join_stats(const CacheAttend &a, const Parts &p, float &M, float &l) {
  const int lane = threadIdx.x & 63;
  float m = -INFINITY;
  for (int c = lane; c < p.np; c += 64) m = fmaxf(m, a.pm[p.at + (size_t)c * a.g]);
  M = wave_max(m);
  M = M == -INFINITY ? 0.f : M;
  float s = 0.f;
  for (int c = lane; c < p.np; c += 64) s += a.pl[p.at + (size_t)c * a.g] * exp2f(a.pm[p.at + (size_t)c * a.g] - M);
  l = wave_sum(s);
}

// Join: T threads per query head add its partial outputs, each weighted by
// 2^(its maximum - the largest one), in an order that only the lengths set:
// a wave where the heads have few partials on average, so that no barrier is
// needed, a workgroup where they have many.  The first loads go out before the statistics
// are known.  Workgroups past the heads (with slot weights) take JOIN_P places
// of one KV head each: the sum over its g heads of 2^(score - log-sum) is
// added to the place's slot, which one thread owns.
constexpr int JOIN_P = 1024;
template <typename T, int D, int TH>
__global__ __launch_bounds__(256) void k_cache_join(CacheAttend a) {
  constexpr int Q = D / 4, G = TH / Q, PRE = 4;         // lanes per partial, groups of partials, early loads
  const int b = blockIdx.y, tid = threadIdx.x, wave = wave_id(), lane = tid & 63;
  const int heads = (a.nq + 256 / TH - 1) / (256 / TH);   // workgroups that join
  const Walk w = walk_of(a);                           // every wave for itself
  if ((int)blockIdx.x < heads) {
    const int h = blockIdx.x * (256 / TH) + tid / TH, t = tid % TH;
    if (TH == 64 && h >= a.nq) return;                 // whole waves
    const size_t hi = (size_t)b * a.nq + h;
    const int hw = __builtin_amdgcn_readfirstlane(h);
    const Parts p = parts_of(a, w, b, hw / a.g, hw % a.g);
    const int x = t % Q, grp = t / Q;
    f32x4 pre[PRE];
#pragma unroll
    for (int i = 0; i < PRE; ++i) {
      const int c = grp + i * G;
      pre[i] = c < p.np ? *(const f32x4 *)(a.po + (p.at + (size_t)c * a.g) * D + 4 * x) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
    float pm[PRE];
#pragma unroll
    for (int i = 0; i < PRE; ++i) {
      const int c = grp + i * G;
      pm[i] = c < p.np ? a.pm[p.at + (size_t)c * a.g] : -INFINITY;
    }
    float M, l;
    join_stats(a, p, M, l);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < PRE; ++i) o += pre[i] * exp2f(pm[i] - M);
#pragma unroll 4
    for (int c = grp + PRE * G; c < p.np; c += G) {
      const size_t i = p.at + (size_t)c * a.g;
      o += *(const f32x4 *)(a.po + i * D + 4 * x) * exp2f(a.pm[i] - M);
    }
    if constexpr (TH == 64) {
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = stride_sum(o[i], Q);
    } else {
      __shared__ float red[TH * 4];
      *(f32x4 *)(red + 4 * t) = o;
      __syncthreads();
      if (grp == 0)
        for (int y = 1; y < G; ++y) o += *(const f32x4 *)(red + 4 * (y * Q + x));
    }
    if (grp == 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = l == 0.f ? 0.f : o[i] / l;
      const float y[4] = {o[0], o[1], o[2], o[3]};
      store_n<T, 4>((T *)a.out + hi * D + 4 * x, y);
    }
    if (t == 0 && a.lse) a.lse[hi] = l == 0.f ? -INFINITY : (M + log2f(l)) * LN2;
    return;
  }
  constexpr int U = JOIN_P / 256;
  const int y = blockIdx.x - heads, j = y % a.v.nkv, g = a.g;
  const int n = __builtin_amdgcn_readlane(w.n, b), places = places_of(a, n);
  const int t0 = y / a.v.nkv * JOIN_P;
  if (t0 >= places) return;
  const Segment sg{b, j, n, 0, 0, places};
  Lookup lk(a, sg);
  const int p0 = t0 + 64 * wave;                       // this wave's places: from here, and 256 on
  int id[U], blk[U];
  const typename Lookup::Start st = lk.start(p0);
#pragma unroll
  for (int i = 0; i < U; ++i) id[i] = lk.column(t0 + i * 256 + tid);
#pragma unroll
  for (int i = 0; i < U; ++i) blk[i] = lk.block(id[i]);
  __shared__ float lse[CACHE_MAXG];
  for (int h = wave; h < g; h += 4) {
    float M, l;
    join_stats(a, parts_of(a, w, b, j, h), M, l);
    if (lane == 0) lse[h] = l == 0.f ? INFINITY : M + log2f(l);   // nothing seen: every weight 0
  }
  uint32_t row[U];
  float old[U];
  lk.begin(p0, st);
#pragma unroll
  for (int i = 0; i < U; ++i) {
    lk.advance(p0 + i * 256, 64);
    row[i] = lk.row(t0 + i * 256 + tid, id[i], blk[i]);
    old[i] = a.weights[row[i] == NO_ROW ? 0 : row[i]];
  }
  __syncthreads();
  float sum[U] = {};
  for (int h = 0; h < g; ++h) {
    const float *sc = a.scores + score_at(a, b, j, h, t0 + tid);
    float s[U];
#pragma unroll
    for (int i = 0; i < U; ++i) s[i] = t0 + i * 256 + tid < places ? sc[i * 256 * g] : 0.f;
#pragma unroll
    for (int i = 0; i < U; ++i) sum[i] += exp2f(s[i] - lse[h]);
  }
#pragma unroll
  for (int i = 0; i < U; ++i)
    if (row[i] != NO_ROW) a.weights[row[i]] = old[i] + sum[i];
}
template <typename T, int D>
static void join_d(const CacheAttend &a, hipStream_t s) {
  // partials of a head on average (a wave adds 64 / (D / 4) at a time; the host
  // does not know the lengths).  A wave each: 32 sequences of 32768 slots 665 us,
  // by workgroups 671; but one of 131072 among 63 of 256, whose heads have
  // hundreds where the average is 4, 120 and 113
  const bool few = a.waves / (a.v.nkv * a.v.kv.n_seq) <= 16;
  const int per = few ? 4 : 1;
  const dim3 g((a.nq + per - 1) / per + (a.weights ? a.v.nkv * ((a.span + JOIN_P - 1) / JOIN_P) : 0), a.v.kv.n_seq);
  if (few) hipLaunchKernelGGL((k_cache_join<T, D, 64>), g, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_cache_join<T, D, 256>), g, dim3(256), 0, s, a);
}
template <typename T, int D>
static void attend_d(const CacheAttend &a, hipStream_t s) {
  constexpr int NW = D * sizeof(T) > 512 ? 2 : 4;      // 64 KB of LDS
  const dim3 g(a.waves);
  if (a.direct) {
    hipLaunchKernelGGL((k_cache_attend<T, D, false, NW>), g, dim3(64 * NW), 0, s, a);
    return;
  }
  if (a.weights) hipLaunchKernelGGL((k_cache_attend<T, D, true, 1>), g, dim3(64), 0, s, a);
  else hipLaunchKernelGGL((k_cache_attend<T, D, false, 1>), g, dim3(64), 0, s, a);
  join_d<T, D>(a, s);
}
template <typename T>
static void attend_t(const CacheAttend &a, hipStream_t s) {
  if (a.d == 32) attend_d<T, 32>(a, s);
  else if (a.d == 64) attend_d<T, 64>(a, s);
  else if (a.d == 128) attend_d<T, 128>(a, s);
  else attend_d<T, 256>(a, s);
}
void launch_cache_attend(bool bf16, const CacheAttend &a, hipStream_t s) {
  if (bf16) attend_t<bf16_t>(a, s);
  else attend_t<float>(a, s);
}

// ---------------------------------------------------------------- summaries
// Channelwise minimum and maximum of the keys of a.per consecutive table
// columns of one sequence and KV head per wave, in steps of 4 rows per lane
// group; two steps are in flight while one is compared.  fminf and fmaxf pass
// over NaN.  The lane groups of a wave meet by swaps of half waves and of rows:
// one exchange and one comparison reduce two channels, after which each half
// keeps its own.
__device__ __forceinline__ void swap32(float &x, float &y) {   // x: low halves of both, y: high halves
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
  x = __uint_as_float(r[0]);
  y = __uint_as_float(r[1]);
}
__device__ __forceinline__ void swap16(float &x, float &y) {   // the same of even and odd rows of 16 lanes
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
  x = __uint_as_float(r[0]);
  y = __uint_as_float(r[1]);
}
template <typename T, int D>
__global__ __launch_bounds__(256) void k_cache_summarize(CacheSummarize a) {
  constexpr int LPR = D / 8, RPI = 64 / LPR, NI = 4, P = sizeof(T) / 2;   // P: 16-byte pieces of 8 values
  const int lane = threadIdx.x & 63, j = blockIdx.y * (blockDim.x >> 6) + wave_id(), b = blockIdx.z, bs = a.v.kv.bs;
  const int grp = lane / LPR, li = lane % LPR;
  const int n = visible_slots(a.v, b, a.err);
  const int nblk = (int)(((long)n + bs - 1) / bs);
  const int first = a.span > 0 && a.span < n ? (n - a.span) / bs : 0;
  const int c0 = first + blockIdx.x * a.per, c1 = min(nblk, c0 + a.per);
  if (c0 >= c1 || j >= a.v.nkv) return;             // whole waves
  // lane i < a.per: pool block and KV head of column c0 + i
  const uint32_t blks = lane < c1 - c0 ? pool_block(a.v, a.v.kv.block_table, b, j, c0 + lane, a.err) : NO_ROW;
  // step t of the wave: rows (t % spb) NI RPI .. of column c0 + t / spb (rows
  // past the visible ones: the last of them again; past the last step: pool
  // block 0).  The loads are made always, so that they can be counted.
  const int spb = (bs + NI * RPI - 1) / (NI * RPI), steps = (c1 - c0) * spb;
  int lt = 0, lc = c0, ls = 0;                      // the next step to load
  auto load = [&](u32x4 (&k)[NI][P]) {
    const bool in = lt < steps;
    const uint32_t blk = in ? (uint32_t)__builtin_amdgcn_readlane((int)blks, lc - c0) : NO_ROW;
    const uint32_t base = blk == NO_ROW ? 0u : blk;
    const int top = in ? min(bs, n - lc * bs) - 1 : 0;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int r = min(ls + i * RPI + grp, top);
      const T *p = (const T *)a.v.kv.k_pool + ((size_t)base * bs + r) * D + 8 * li;
#pragma unroll
      for (int x = 0; x < P; ++x) k[i][x] = stream16((const u32x4 *)p + x);
    }
    ++lt;
    ls += NI * RPI;
    const bool over = ls >= bs;
    ls = over ? 0 : ls;
    lc += over;
  };
  float v[16];                                      // minima and maxima of 8 channels
  int c = c0, left = spb;                           // the step at hand: its column, steps left of it
  auto compare = [&](const u32x4 (&k)[NI][P]) {
    if (left == spb) {
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        v[x] = INFINITY;
        v[8 + x] = -INFINITY;
      }
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      float y[8];
      unpack8<T>(k[i], y);
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        v[x] = fminf(v[x], y[x]);
        v[8 + x] = fmaxf(v[8 + x], y[x]);
      }
    }
  };
  auto finish = [&]() {
    if (--left || c >= c1) return;
    left = spb;
    const uint32_t blk = (uint32_t)__builtin_amdgcn_readlane((int)blks, c - c0);
    ++c;
    T *o = (T *)a.summary + (size_t)(blk == NO_ROW ? 0u : blk) * 2 * D;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      if constexpr (LPR <= 4) {
        v[x] = fminf(v[x], dpp_f32<DPP_ROW_ROR4>(v[x]));
        v[8 + x] = fmaxf(v[8 + x], dpp_f32<DPP_ROW_ROR4>(v[8 + x]));
      }
      if constexpr (LPR <= 8) {
        v[x] = fminf(v[x], dpp_f32<DPP_ROW_ROR8>(v[x]));
        v[8 + x] = fmaxf(v[8 + x], dpp_f32<DPP_ROW_ROR8>(v[8 + x]));
      }
    }
    // halves: lanes below 32 keep channels 0 .. 3, the others 4 .. 7
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      swap32(v[x], v[4 + x]);
      v[x] = fminf(v[x], v[4 + x]);
      swap32(v[8 + x], v[12 + x]);
      v[8 + x] = fmaxf(v[8 + x], v[12 + x]);
    }
    constexpr int W = LPR <= 16 ? 2 : 4;            // channels that a lane keeps
    if constexpr (W == 2) {                         // rows: the first two of those four, or the others
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        swap16(v[x], v[2 + x]);
        v[x] = fminf(v[x], v[2 + x]);
        swap16(v[8 + x], v[10 + x]);
        v[8 + x] = fmaxf(v[8 + x], v[10 + x]);
      }
    }
    // into channel order, so that the stores fill their lines: lane l takes
    // channels W l .. from the lane of column l / (8 / W) that keeps them
    const int from = lane / (8 / W) % LPR + lane % (8 / W) * (64 / (8 / W));
#pragma unroll
    for (int x = 0; x < W; ++x) {
      v[x] = __shfl(v[x], from, 64);
      v[8 + x] = __shfl(v[8 + x], from, 64);
    }
    if (blk != NO_ROW && lane < D / W) {
      store_n<T, W>(o + W * lane, v);
      store_n<T, W>(o + D + W * lane, v + 8);
    }
  };
  u32x4 k0[NI][P], k1[NI][P];
  // (the loads in this order on every path, so that a wait for one set leaves
  // the other in flight)
  load(k0);
  __builtin_amdgcn_sched_barrier(0);
  load(k1);
  __builtin_amdgcn_sched_barrier(0);
  for (int t = 0; t < steps; t += 2) {              // (an odd last step is followed by an idle one)
    compare(k0);
    load(k0);
    __builtin_amdgcn_sched_barrier(0);
    finish();
    compare(k1);
    load(k1);
    __builtin_amdgcn_sched_barrier(0);
    finish();
  }
}

template <typename T>
static void summarize_d(const CacheSummarize &a, int d, hipStream_t s) {
  // the waves of a workgroup take different heads of the same columns, whose
  // rows lie next to each other in the pool
  const int nw = min(4, a.v.nkv);
  const dim3 g((a.columns + a.per - 1) / a.per, (a.v.nkv + nw - 1) / nw, a.v.kv.n_seq), t(64 * nw);
  if (d == 32) hipLaunchKernelGGL((k_cache_summarize<T, 32>), g, t, 0, s, a);
  else if (d == 64) hipLaunchKernelGGL((k_cache_summarize<T, 64>), g, t, 0, s, a);
  else if (d == 128) hipLaunchKernelGGL((k_cache_summarize<T, 128>), g, t, 0, s, a);
  else hipLaunchKernelGGL((k_cache_summarize<T, 256>), g, t, 0, s, a);
}
void launch_cache_summarize(bool bf16, const CacheSummarize &a, int d, hipStream_t s) {
  if (bf16) summarize_d<bf16_t>(a, d, s);
  else summarize_d<float>(a, d, s);
}

// ---------------------------------------------------------------- choice
// Order key of a choice's candidate: larger value first, NaN after every
// number, forced candidates before all.
constexpr uint32_t KEY_FORCED = 0xffffffffu;
__device__ __forceinline__ uint32_t choice_key(float v) { return (uint32_t)(cand_key(v, 0) >> 32); }

// Scores of the blocks: for every query head of the group the sum over the
// channels of q_c * (q_c >= 0 ? max_c : min_c), an upper bound of q.k over the
// block's keys; the block's score is the largest of them.  Products of stored
// values are exact in fp64 and their sum is as good as exact, so the order of
// the blocks does not depend on the order of the sum.
//   A lane group of d / 8 lanes per block; a wave takes a.per blocks, with the
// queries in registers (G of them: the heads of a KV head, rounded up to a
// power of two; the missing ones repeat the last) and four steps of summaries
// in flight.  The sums of the G heads meet pairwise, so that each exchange
// halves what is left to add.  Bound by instructions, some 250 per step (d =
// 128, 4 heads): 147,000 summaries (75 MB) of 16 sequences take 20 us.

// v of the lane whose index differs in bit 2^X (X < 4: DPP within 16 lanes,
// where the mirrors pair lanes of equal sums; else permlane swaps)
template <int X>
__device__ __forceinline__ double xor_f64(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  uint32_t l = (uint32_t)u, h = (uint32_t)(u >> 32);
  if constexpr (X == 0) { l = dpp_u32<DPP_QUAD_XOR1>(l); h = dpp_u32<DPP_QUAD_XOR1>(h); }
  else if constexpr (X == 1) { l = dpp_u32<DPP_QUAD_XOR2>(l); h = dpp_u32<DPP_QUAD_XOR2>(h); }
  else if constexpr (X == 2) {                      // lane ^ 4: the half-row mirror (^ 7), then ^ 3
    l = dpp_u32<0x1B>(dpp_u32<DPP_HALF_MIRROR>(l)); h = dpp_u32<0x1B>(dpp_u32<DPP_HALF_MIRROR>(h));
  } else if constexpr (X == 3) { l = dpp_u32<DPP_ROW_ROR8>(l); h = dpp_u32<DPP_ROW_ROR8>(h); }
  else { l = __float_as_uint(xor16_f(__uint_as_float(l))); h = __float_as_uint(xor16_f(__uint_as_float(h))); }
  return __builtin_bit_cast(double, ((uint64_t)h << 32) | l);
}
template <int X>
__device__ __forceinline__ float xor_f32(float v) {
  if constexpr (X == 0) return dpp_f32<DPP_QUAD_XOR1>(v);
  else if constexpr (X == 1) return dpp_f32<DPP_QUAD_XOR2>(v);
  else return dpp_f32<0x1B>(dpp_f32<DPP_HALF_MIRROR>(v));
}
// Sums of s[0 .. N - 1] over the lane groups of 2^(SH - X) lanes; lane l ends
// with the sum of entry bits of l (the first exchanges halve N, the others add).
template <int N, int X, int SH>
__device__ __forceinline__ double group_sums(double (&s)[N]) {
  if constexpr (X == SH) {
    return s[0];
  } else if constexpr (N > 1) {
    const bool odd = (threadIdx.x >> X) & 1;
    double t[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const double keep = odd ? s[N / 2 + i] : s[i], give = odd ? s[i] : s[N / 2 + i];
      t[i] = keep + xor_f64<X>(give);
    }
    return group_sums<N / 2, X + 1, SH>(t);
  } else {
    s[0] += xor_f64<X>(s[0]);
    return group_sums<N, X + 1, SH>(s);
  }
}
// the larger one, NaN if either is
__device__ __forceinline__ float nan_max(float a, float b) { return __builtin_elementwise_maximum(a, b); }
// A bf16 value as a double has no low word.
__device__ __forceinline__ uint32_t high_word(float x) {
  return (uint32_t)(__builtin_bit_cast(uint64_t, (double)x) >> 32);
}

template <typename T, int D, int G>
__global__ __launch_bounds__(256, G > 4 ? 2 : 3) void k_cache_score(CacheSelect a) {
  constexpr int LPR = D / 8, RPI = 64 / LPR, P = sizeof(T) / 2, DEPTH = 4;
  constexpr int SH = D == 32 ? 2 : D == 64 ? 3 : D == 128 ? 4 : 5;   // log2 LPR
  // with fewer lanes than heads (d = 32, 8 heads) two rounds of 4
  constexpr int N = G > LPR ? LPR : G;
  const int lane = threadIdx.x & 63, j = blockIdx.y * (blockDim.x >> 6) + wave_id(), b = blockIdx.z, bs = a.v.kv.bs;
  const int grp = lane / LPR, li = lane % LPR;
  const int n = visible_slots(a.v, b, a.err);
  const int nblk = (int)(((long)n + bs - 1) / bs);
  const int c0 = blockIdx.x * a.per, c1 = min(nblk, c0 + a.per);
  if (c0 >= c1 || j >= a.v.nkv) return;             // whole waves
  u32x4 raw[G][P];
#pragma unroll
  for (int h = 0; h < G; ++h)
#pragma unroll
    for (int y = 0; y < P; ++y)
      raw[h][y] = *((const u32x4 *)((const T *)a.q + ((size_t)b * a.nq + j * a.g + min(h, a.g - 1)) * D + 8 * li) + y);
  // lane i < a.per: pool block and KV head of column c0 + i
  const uint32_t blks = lane < c1 - c0 ? pool_block(a.v, a.v.kv.block_table, b, j, c0 + lane, a.err) : NO_ROW;
  u32x4 mn[DEPTH][P], mx[DEPTH][P];
  auto load = [&](int x, int c) {
    const uint32_t blk = (uint32_t)__shfl((int)blks, min(c + grp - c0, 63), 64);
    const T *p = (const T *)a.summary + (size_t)(blk == NO_ROW ? 0 : blk) * 2 * D + 8 * li;
#pragma unroll
    for (int y = 0; y < P; ++y) {
      mn[x][y] = stream16((const u32x4 *)p + y);
      mx[x][y] = stream16((const u32x4 *)(p + D) + y);
    }
  };
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int x = 0; x < DEPTH; ++x) {                 // in this order: a wait for one leaves the others in flight
    load(x, c0 + x * RPI);
    __builtin_amdgcn_sched_barrier(0);
  }
  double q[G][8];
#pragma unroll
  for (int h = 0; h < G; ++h) {
    float x[8];
    unpack8<T>(raw[h], x);
#pragma unroll
    for (int i = 0; i < 8; ++i) q[h][i] = (double)x[i];
  }
  float mine = 0.f;                                 // score of column c0 + li * RPI + grp (a.per <= 64)
  int step = 0;
  for (int cc = c0; cc < c1; cc += DEPTH * RPI)
#pragma unroll
    for (int x = 0; x < DEPTH; ++x, ++step) {
      const int c = cc + x * RPI;
      float lo[8], hi[8];                           // (of pool block 0 past the last column: not kept)
      unpack8<T>(mn[x], lo);
      unpack8<T>(mx[x], hi);
      uint32_t lo_w[8], hi_w[8];                    // bf16: high words as doubles
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          lo_w[i] = high_word(lo[i]);
          hi_w[i] = high_word(hi[i]);
        }
      }
      load(x, c + DEPTH * RPI);                     // always, so that the loads can be counted
      __builtin_amdgcn_sched_barrier(0);
      float best = -INFINITY;
#pragma unroll
      for (int h0 = 0; h0 < G; h0 += N) {
        double s[N];
#pragma unroll
        for (int h = 0; h < N; ++h) {
          s[h] = 0.0;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const double x = q[h0 + h][i];
            double m;
            if constexpr (sizeof(T) == 2)
              m = __builtin_bit_cast(double, (uint64_t)(x >= 0.0 ? hi_w[i] : lo_w[i]) << 32);
            else
              m = (double)(x >= 0.0 ? hi[i] : lo[i]);
            s[h] += x * m;
          }
        }
        best = nan_max(best, (float)group_sums<N, 0, SH>(s));
      }
      if constexpr (N > 1) best = nan_max(best, xor_f32<0>(best));
      if constexpr (N > 2) best = nan_max(best, xor_f32<1>(best));
      if constexpr (N > 4) best = nan_max(best, xor_f32<2>(best));
      if (li == step) mine = best;
    }
  const int bi = c0 + li * RPI + grp;
  const bool bad = (uint32_t)__shfl((int)blks, bi - c0, 64) == NO_ROW;
  if (bi < c1) {
    const bool forced = bi < a.n_first || bi >= nblk - a.n_last;
    a.keys[((size_t)b * a.v.nkv + j) * a.ld_keys + bi] = bad ? 0u : forced ? KEY_FORCED : choice_key(mine);
  }
}

// the smallest of the wave, in every lane
__device__ __forceinline__ uint32_t wave_least(uint32_t v) {
  v = min(v, dpp_u32<DPP_QUAD_XOR1>(v));
  v = min(v, dpp_u32<DPP_QUAD_XOR2>(v));
  v = min(v, dpp_u32<DPP_HALF_MIRROR>(v));
  v = min(v, dpp_u32<DPP_ROW_MIRROR>(v));
  const uint32_t a = min((uint32_t)__builtin_amdgcn_readlane((int)v, 0), (uint32_t)__builtin_amdgcn_readlane((int)v, 16));
  return min(a, min((uint32_t)__builtin_amdgcn_readlane((int)v, 32), (uint32_t)__builtin_amdgcn_readlane((int)v, 48)));
}
// sum of v[0 .. w - 1] (LDS, at most 64 entries), w wave-uniform
__device__ __forceinline__ uint32_t sum_before(const uint32_t *v, int entries, int w) {
  const int lane = threadIdx.x & 63;
  return (uint32_t)__builtin_amdgcn_readlane((int)wave_scan(lane < entries && lane < w ? v[lane] : 0u), 63);
}

// The n_take candidates of largest key of one (sequence, KV head), ties to
// the lowest index, in index order, then -1.  A radix descent over digits of
// 11 bits with an LDS histogram finds the key of the last one taken, and ends
// where a whole digit is taken; the candidates left after the first digit are
// listed in LDS if at most CHOOSE_LIST are.  Each wave then owns a run
// of candidates, so a prefix over the waves gives every taken one its place.
// Candidates are padded with keys of 0 to groups of 256: behind all others,
// and never reached, since fewer are taken than there are.
//   LDS: the keys fit CHOOSE_LDS and are read once, and the digits start at the
// highest bit in which they differ (scores share their exponents, and lanes
// that add to one counter queue); else every pass streams
// them (from the L2 after the first).  WEIGHTS (with LDS): the keys are made
// here from the slot weights.
//   One workgroup's instructions and its barriers bound it: 8 of 256 CUs are at
// work for 8 heads.  128 of 8192 blocks 8.7 us, 1024 of 4096 slots (keys from
// the weights) 9.8.
constexpr int CHOOSE_T = 1024, CHOOSE_W = CHOOSE_T / 64;
constexpr int CHOOSE_LIST = 8192;
// One key's digit counted.  Many lanes with one digit (equal keys: unweighted
// slots) would queue for its counter: one addition for all of them.
__device__ __forceinline__ void count_digit(uint32_t *hg, uint32_t dg, bool in) {
  const uint32_t d0 = __builtin_amdgcn_readfirstlane(dg);
  const uint64_t same = __ballot(in && dg == d0);
  if (__popcll(same) >= 16) {
    if ((int)(threadIdx.x & 63) == __builtin_ctzll(same)) atomicAdd(&hg[d0], (uint32_t)__popcll(same));
    in &= dg != d0;
  }
  if (in) atomicAdd(&hg[dg], 1u);
}
// Of 2048 counters (complete: behind a barrier), the digit in which the
// need-th largest lies, the number above it and its own count.  Whole workgroup
// of CHOOSE_T threads; `clear` zeroes the counters.
struct Digit {
  uint32_t digit, above, count;
};
struct DigitWs {
  uint32_t wsum[CHOOSE_W];
  Digit d;
};
__device__ __forceinline__ Digit digit_of(uint32_t *hg, uint32_t need, bool clear, DigitWs &ws) {
  const int tid = threadIdx.x, wave = wave_id(), lane = tid & 63;
  // thread t owns the digits 2047 - 2t and 2046 - 2t: a sum over the threads
  // before it counts the digits above
  const uint32_t h1 = hg[2047 - 2 * tid], h0 = hg[2046 - 2 * tid];
  const uint32_t scan = wave_scan(h0 + h1);
  if (lane == 63) ws.wsum[wave] = scan;
  if (clear) {
    hg[2047 - 2 * tid] = 0;
    hg[2046 - 2 * tid] = 0;
  }
  __syncthreads();
  const uint32_t above = sum_before(ws.wsum, CHOOSE_W, wave) + scan - h0 - h1;
  if (above < need && above + h1 >= need) ws.d = {2047u - 2 * tid, above, h1};
  else if (above + h1 < need && above + h1 + h0 >= need) ws.d = {2046u - 2 * tid, above + h1, h0};
  __syncthreads();
  return ws.d;
}
template <bool WEIGHTS, bool LDS>
__global__ __launch_bounds__(CHOOSE_T) void k_cache_choose(CacheChoose a) {
  const int j = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, wave = wave_id(), lane = tid & 63;
  extern __shared__ __attribute__((aligned(16))) uint32_t s_keys[];
  __shared__ uint32_t hist[2][2048], list[CHOOSE_LIST];
  __shared__ uint32_t wgt[CHOOSE_W], weq[CHOOSE_W], wmin[CHOOSE_W], wmax[CHOOSE_W], s_listed;
  __shared__ DigitWs dws;
  const int n_vis = visible_slots(a.v, b, a.err);
  const int bs = a.per_block ? a.v.kv.bs : 1;
  const int n = (int)(((long)n_vis + bs - 1) / bs);
  const size_t u = (size_t)b * a.v.nkv + j;
  const uint32_t *keys = a.keys + u * a.ld_keys;
  int32_t *out = a.out + u * a.n_take;
  if (a.lens && j == 0 && tid == 0) a.lens[b] = min(n, a.n_take);
  if (n <= a.n_take) {
    for (int i = tid; i < a.n_take; i += CHOOSE_T) out[i] = i < n ? i : -1;
    return;
  }
  // a run of groups of 256 candidates per wave; lane l holds candidates
  // 4 l .. 4 l + 3 of a group
  const int groups = (n + 255) / 256, per = (groups + CHOOSE_W - 1) / CHOOSE_W;
  const int g0 = wave * per, g1 = min(groups, g0 + per);
  for (int i = tid; i < 4096; i += CHOOSE_T) (&hist[0][0])[i] = 0;
  if (tid == 0) s_listed = 0;
  // a key counts as its distance from `base`, in digits from bit top_shift + 10
  // down; forced ones, the largest of all, in the first digit's last counter
  uint32_t base = 0;
  int top_shift = 21;
  if constexpr (LDS) {
    uint32_t least = KEY_FORCED, most = 0;
    constexpr int U = 4;                            // loads in flight per thread
    for (int i0 = 0; i0 < 256 * groups; i0 += U * CHOOSE_T) {
      uint32_t k[U];
      if constexpr (WEIGHTS) {
        uint32_t row[U];
#pragma unroll
        for (int x = 0; x < U; ++x) {
          const int i = i0 + x * CHOOSE_T + tid, bi = slot_block(a.v.kv, i);
          row[x] = i < n ? pool_row(a.v, a.v.kv.block_table, b, j, bi, slot_in_block(a.v.kv, i, bi), a.err) : NO_ROW;
        }
        float w[U];
#pragma unroll
        for (int x = 0; x < U; ++x) w[x] = a.weights[row[x] == NO_ROW ? 0 : row[x]];
#pragma unroll
        for (int x = 0; x < U; ++x) {
          const int i = i0 + x * CHOOSE_T + tid;
          k[x] = row[x] == NO_ROW ? 0u : i < a.n_first || i >= n - a.n_last ? KEY_FORCED : choice_key(w[x]);
        }
      } else {
#pragma unroll
        for (int x = 0; x < U; ++x) {
          const int i = i0 + x * CHOOSE_T + tid;
          k[x] = i < n ? keys[i] : 0u;
        }
      }
#pragma unroll
      for (int x = 0; x < U; ++x) {
        const int i = i0 + x * CHOOSE_T + tid;
        if (i < 256 * groups) s_keys[i] = k[x];
        least = i < n ? min(least, k[x]) : least;
        most = i < n && k[x] != KEY_FORCED ? max(most, k[x]) : most;
      }
    }
    least = wave_least(least);
    most = ~wave_least(~most);
    if (lane == 0) {
      wmin[wave] = least;
      wmax[wave] = most;
    }
    __syncthreads();
    base = wave_least(lane < CHOOSE_W ? wmin[lane] : KEY_FORCED);
    most = ~wave_least(lane < CHOOSE_W ? ~wmax[lane] : KEY_FORCED);
    // the largest distance that is not forced fits below the last counter
    top_shift = most > base ? max(0, 22 - __clz((int)(most - base))) : 0;
    if (top_shift && ((most - base) >> (top_shift - 1)) < 2047u) --top_shift;
  }
  __syncthreads();
  auto load4 = [&](int gr) -> u32x4 {
    const int i = gr * 256 + 4 * lane;
    if constexpr (LDS) {
      u32x4 k = *(const u32x4 *)(s_keys + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) k[e] = max(k[e], base) - base;   // (padding is below the base)
      return k;
    } else {
      if (gr * 256 + 256 <= n) return *(const u32x4 *)(keys + i);
      u32x4 k;
#pragma unroll
      for (int e = 0; e < 4; ++e) k[e] = i + e < n ? keys[i + e] : 0u;
      return k;
    }
  };
  constexpr int UG = LDS ? 2 : 8;                   // groups in flight per wave
  uint32_t prefix = 0, mask = 0, need = a.n_take;
  bool listed = false;
#pragma unroll 1
  for (int p = 0; p < 3; ++p) {
    const int shift = max(0, top_shift - 11 * p);
    // digits of 11 bits, the last one of what is left
    const uint32_t dm = p == 0 || top_shift - 11 * p >= 0 ? 2047u : (1u << (top_shift - 11 * p + 11)) - 1;
    uint32_t *hg = hist[p & 1];
    auto add = [&](uint32_t k, bool in) {
      count_digit(hg, p == 0 ? min(k >> shift, 2047u) : (k >> shift) & dm, in);
    };
    if (listed) {
      for (int i = tid; i < (int)s_listed; i += CHOOSE_T) add(list[i], (list[i] & mask) == prefix);
    } else {
#pragma unroll 1
      for (int gr = g0; gr < g1; gr += UG) {
        u32x4 k[UG];
#pragma unroll
        for (int x = 0; x < UG; ++x) k[x] = load4(min(gr + x, g1 - 1));
#pragma unroll
        for (int x = 0; x < UG; ++x) {
          if (gr + x >= g1) break;
          bool in[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) in[e] = (k[x][e] & mask) == prefix;
          if (!__ballot(in[0] | in[1] | in[2] | in[3])) continue;
#pragma unroll
          for (int e = 0; e < 4; ++e) add(k[x][e], in[e]);
        }
      }
    }
    __syncthreads();
    const Digit dg = digit_of(hg, need, p == 0, dws);   // (the third pass counts here again)
    prefix |= dg.digit << shift;
    mask = ~0u << shift;
    need -= dg.above;
    if (need == dg.count || shift == 0) break;      // the whole digit, or no digit left (uniform)
    if (p == 0 && dg.count <= CHOOSE_LIST) {        // (uniform) in any order: only counted
      listed = true;
#pragma unroll 1
      for (int gr = g0; gr < g1; gr += UG) {
        u32x4 k[UG];
#pragma unroll
        for (int x = 0; x < UG; ++x) k[x] = load4(min(gr + x, g1 - 1));
#pragma unroll
        for (int x = 0; x < UG; ++x) {
          if (gr + x >= g1) break;
          uint64_t m[4];
          uint32_t all = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            m[e] = __ballot((k[x][e] & mask) == prefix);
            all += __popcll(m[e]);
          }
          if (!all) continue;
          uint32_t to = 0;
          if (lane == 0) to = atomicAdd(&s_listed, all);
          to = __builtin_amdgcn_readfirstlane(to);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if ((k[x][e] & mask) == prefix) list[to + __popcll(m[e] & ((1ull << lane) - 1))] = k[x][e];
            to += __popcll(m[e]);
          }
        }
      }
      __syncthreads();
    }
  }
  // taken: key & mask > prefix, and the first `need` of those equal to it
  uint32_t gt = 0, eq = 0;
#pragma unroll 1
  for (int gr = g0; gr < g1; gr += UG) {
    u32x4 k[UG];
#pragma unroll
    for (int x = 0; x < UG; ++x) k[x] = load4(min(gr + x, g1 - 1));
#pragma unroll
    for (int x = 0; x < UG; ++x) {
      if (gr + x >= g1) break;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        gt += (k[x][e] & mask) > prefix;
        eq += (k[x][e] & mask) == prefix;
      }
    }
  }
  gt = wave_scan(gt);
  eq = wave_scan(eq);
  if (lane == 63) {
    wgt[wave] = gt;
    weq[wave] = eq;
  }
  __syncthreads();
  uint32_t eq0 = sum_before(weq, CHOOSE_W, wave), to = sum_before(wgt, CHOOSE_W, wave) + min(eq0, need);
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll 1
  for (int gr = g0; gr < g1; gr += UG) {
    u32x4 k[UG];
#pragma unroll
    for (int x = 0; x < UG; ++x) k[x] = load4(min(gr + x, g1 - 1)) & mask;
#pragma unroll
    for (int x = 0; x < UG; ++x) {
      if (gr + x >= g1) break;
      bool any = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) any |= k[x][e] >= prefix;
      if (!__ballot(any)) continue;
      bool take[4], some_eq = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        take[e] = k[x][e] > prefix;
        some_eq |= k[x][e] == prefix;
      }
      if (__ballot(some_eq)) {
        uint32_t ahead = eq0;                       // equal ones before this lane's next candidate
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint64_t m = __ballot(k[x][e] == prefix);
          ahead += __popcll(m & below);
          eq0 += __popcll(m);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          take[e] |= k[x][e] == prefix && ahead < need;
          ahead += k[x][e] == prefix;
        }
      }
      uint32_t pos = to;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint64_t t = __ballot(take[e]);
        pos += __popcll(t & below);
        to += __popcll(t);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (take[e]) out[pos++] = gr * 256 + x * 256 + 4 * lane + e;
    }
  }
}
// at most CHOOSE_LDS candidates have their keys in LDS (96 KB beside the 48
// of histograms and list; a workgroup may take 160)

// The same choice for more slots than fit one CU's LDS, spread over the chip in
// segments of CHOOSE_SEG keys: k_cache_keys makes the keys and the segments'
// histograms of the first digit; a workgroup per segment (k_cache_collect)
// finds the digit of the cut from all of them, counts its keys above and lists
// those in it; one workgroup per (sequence, KV head) (k_cache_cut) descends
// through the listed keys, or through all where they are too many, and leaves
// the cut and each segment's place in the output; a workgroup per segment
// (k_cache_emit) writes its indices there.  16384 of 131000 slots of 8 heads:
// 27 us, by one workgroup per head 53.
//   cut of unit u (words): prefix, mask, need, -, then per segment the number
// taken before it and the number equal to the prefix before it, then per
// segment its keys above the first digit's cut and in it.
constexpr int CUT_SEG = 4;
__device__ __forceinline__ int wide_count(const CacheChoose &a, int b) { return visible_slots(a.v, b, a.err); }
// the segments' histograms summed into hg
__device__ __forceinline__ void sum_hists(const CacheChoose &a, size_t u, int segs, uint32_t *hg) {
  const uint32_t *h = a.hists + u * a.ld_hists + threadIdx.x;
  uint32_t lo = 0, hi = 0;
#pragma unroll 8
  for (int x = 0; x < segs; ++x) {
    const uint32_t v = h[x * 1024];
    lo += v & 0xffffu;
    hi += v >> 16;
  }
  hg[2 * threadIdx.x] = lo;
  hg[2 * threadIdx.x + 1] = hi;
  __syncthreads();
}
// 4 keys of this thread in a segment (0 past the end: behind all, never taken)
__device__ __forceinline__ u32x4 seg_keys(const uint32_t *keys, int i, int n) {
  if (i + 4 <= n) return *(const u32x4 *)(keys + i);
  u32x4 k;
#pragma unroll
  for (int e = 0; e < 4; ++e) k[e] = i + e < n ? keys[i + e] : 0u;
  return k;
}
__global__ __launch_bounds__(CHOOSE_T) void k_cache_collect(CacheChoose a) {
  static_assert(CHOOSE_SEG == 4 * CHOOSE_T, "4 keys per thread");
  const int sg = blockIdx.x, j = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, wave = wave_id(), lane = tid & 63;
  __shared__ uint32_t hg[2048], wgt[CHOOSE_W], weq[CHOOSE_W];
  __shared__ DigitWs dws;
  const int n = wide_count(a, b);
  if (n <= a.n_take || sg * CHOOSE_SEG >= n) return;
  const size_t u = (size_t)b * a.v.nkv + j;
  const int segs = (n + CHOOSE_SEG - 1) / CHOOSE_SEG;
  const u32x4 k = seg_keys(a.keys + u * a.ld_keys, sg * CHOOSE_SEG + 4 * tid, n);
  sum_hists(a, u, segs, hg);
  const uint32_t d = digit_of(hg, a.n_take, false, dws).digit;
  uint32_t gt = 0, eq = 0;
  uint64_t m[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bool in = sg * CHOOSE_SEG + 4 * tid + e < n;
    gt += __popcll(__ballot(in && (k[e] >> 21) > d));
    m[e] = __ballot(in && (k[e] >> 21) == d);
    eq += __popcll(m[e]);
  }
  if (lane == 0) {
    wgt[wave] = gt;
    weq[wave] = eq;
  }
  __syncthreads();
  uint32_t to = sum_before(weq, CHOOSE_W, wave);
  uint32_t *cand = a.cand + u * a.ld_cand + (size_t)sg * CHOOSE_SEG;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if ((m[e] >> lane) & 1) cand[to + __popcll(m[e] & ((1ull << lane) - 1))] = k[e];
    to += __popcll(m[e]);
  }
  if (wave == 0) {
    const uint32_t g = sum_before(wgt, CHOOSE_W, CHOOSE_W), q = sum_before(weq, CHOOSE_W, CHOOSE_W);
    uint32_t *c = a.cut + u * a.ld_cut + CUT_SEG + 2 * ((size_t)a.ld_cand / CHOOSE_SEG + sg);
    if (lane == 0) {
      c[0] = g;
      c[1] = q;
    }
  }
}
// exclusive sums over up to CHOOSE_MAX_SEGS entries (LDS), by one wave; the
// total in v[n]
__device__ __forceinline__ void scan_segs(uint32_t *v, int n) {
  const int lane = threadIdx.x & 63;
  uint32_t run = 0;
  for (int i = 0; i < n; i += 64) {
    const uint32_t x = i + lane < n ? v[i + lane] : 0u, t = wave_scan(x);
    if (i + lane < n) v[i + lane] = run + t - x;
    run += (uint32_t)__builtin_amdgcn_readlane((int)t, 63);
  }
  if (lane == 0) v[n] = run;
}
__global__ __launch_bounds__(CHOOSE_T) void k_cache_cut(CacheChoose a) {
  const int j = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, wave = wave_id(), lane = tid & 63;
  __shared__ uint32_t hist[2][2048], list[CHOOSE_LIST];
  __shared__ uint32_t s_gt[CHOOSE_MAX_SEGS + 1], s_eq[CHOOSE_MAX_SEGS + 1];
  __shared__ DigitWs dws;
  const int n = wide_count(a, b);
  if (j == 0 && tid == 0) a.lens[b] = min(n, a.n_take);
  if (n <= a.n_take) return;
  const size_t u = (size_t)b * a.v.nkv + j;
  const int segs = (n + CHOOSE_SEG - 1) / CHOOSE_SEG;
  const uint32_t *keys = a.keys + u * a.ld_keys, *cand = a.cand + u * a.ld_cand;
  uint32_t *cut = a.cut + u * a.ld_cut, *counts = cut + CUT_SEG + 2 * (a.ld_cand / CHOOSE_SEG);
  for (int i = tid; i < segs; i += CHOOSE_T) s_eq[i] = counts[2 * i + 1];
  hist[1][tid] = 0;
  hist[1][tid + CHOOSE_T] = 0;
  sum_hists(a, u, segs, hist[0]);
  Digit dg = digit_of(hist[0], a.n_take, true, dws);
  uint32_t prefix = dg.digit << 21, mask = ~0u << 21, need = a.n_take - dg.above;
  const bool listed = dg.count <= CHOOSE_LIST;
  if (wave == 0) scan_segs(s_eq, segs);                // places in the list
  __syncthreads();
  // f(key, segment) for every listed key, or every key; a wave per segment
  auto each = [&](auto f) {
    for (int sg = wave; sg < segs; sg += CHOOSE_W) {
      if (listed) {
        const int l0 = s_eq[sg], l1 = s_eq[sg + 1];
        for (int i = l0; i < l1; i += 64) f(i + lane < l1 ? list[i + lane] : 0u, i + lane < l1, sg);
      } else {
        const int k1 = min(n, (sg + 1) * CHOOSE_SEG);
#pragma unroll 4
        for (int i = sg * CHOOSE_SEG; i < k1; i += 64) f(i + lane < k1 ? keys[i + lane] : 0u, i + lane < k1, sg);
      }
    }
  };
  if (need < dg.count) {
    if (listed) {
      for (int sg = wave; sg < segs; sg += CHOOSE_W) {
        const int l0 = s_eq[sg], l1 = s_eq[sg + 1];
        for (int i = lane; i < l1 - l0; i += 64) list[l0 + i] = cand[(size_t)sg * CHOOSE_SEG + i];
      }
      __syncthreads();
    }
#pragma unroll 1
    for (int p = 1; p < 3; ++p) {
      const int shift = p == 1 ? 10 : 0;
      const uint32_t dm = p == 1 ? 2047u : 1023u;
      uint32_t *hg = hist[p & 1];
      each([&](uint32_t k, bool in, int) { count_digit(hg, (k >> shift) & dm, in && (k & mask) == prefix); });
      __syncthreads();
      dg = digit_of(hg, need, false, dws);
      prefix |= dg.digit << shift;
      mask = ~0u << shift;
      need -= dg.above;
      if (need == dg.count) break;
    }
  }
  // per segment: its keys above the cut and equal to it
  const bool refined = mask != ~0u << 21;
  for (int sg = wave; sg < segs; sg += CHOOSE_W) {
    uint32_t gt = counts[2 * sg], eq = counts[2 * sg + 1];
    if (refined) {
      // (of all keys, or of the listed ones beside those above the first digit)
      gt = listed ? gt : 0u;
      eq = 0;
      const int l0 = listed ? (int)s_eq[sg] : sg * CHOOSE_SEG;
      const int l1 = listed ? (int)s_eq[sg + 1] : min(n, (sg + 1) * CHOOSE_SEG);
      for (int i = l0; i < l1; i += 64) {
        const uint32_t k = i + lane < l1 ? (listed ? list[i + lane] : keys[i + lane]) & mask : 0u;
        gt += __popcll(__ballot(i + lane < l1 && k > prefix));
        eq += __popcll(__ballot(i + lane < l1 && k == prefix));
      }
    }
    if (lane == 0) {
      s_gt[sg] = gt;
      hist[0][sg] = eq;                                // (s_eq is still read)
    }
  }
  __syncthreads();
  for (int i = tid; i < segs; i += CHOOSE_T) s_eq[i] = hist[0][i];
  __syncthreads();
  if (wave == 0) scan_segs(s_gt, segs);
  if (wave == 1) scan_segs(s_eq, segs);
  __syncthreads();
  for (int i = tid; i < segs; i += CHOOSE_T) {
    cut[CUT_SEG + 2 * i] = s_gt[i] + min(s_eq[i], need);
    cut[CUT_SEG + 2 * i + 1] = s_eq[i];
  }
  if (tid == 0) {
    cut[0] = prefix;
    cut[1] = mask;
    cut[2] = need;
  }
}
__global__ __launch_bounds__(CHOOSE_T) void k_cache_emit(CacheChoose a) {
  const int sg = blockIdx.x, j = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, wave = wave_id(), lane = tid & 63;
  __shared__ uint32_t wgt[CHOOSE_W], weq[CHOOSE_W];
  const int n = wide_count(a, b);
  const size_t u = (size_t)b * a.v.nkv + j;
  int32_t *out = a.out + u * a.n_take;
  if (n <= a.n_take) {                                 // all of them, in the segments there are
    for (int i = sg * CHOOSE_T + tid; i < a.n_take; i += (int)gridDim.x * CHOOSE_T) out[i] = i < n ? i : -1;
    return;
  }
  if (sg * CHOOSE_SEG >= n) return;
  const int i0 = sg * CHOOSE_SEG + 4 * tid;
  const uint32_t *cut = a.cut + u * a.ld_cut;
  const uint32_t prefix = cut[0], mask = cut[1], need = cut[2];
  const u32x4 k = seg_keys(a.keys + u * a.ld_keys, i0, n) & mask;
  uint32_t gt = 0, eq = 0;
  uint64_t mg[4], me[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    mg[e] = __ballot(i0 + e < n && k[e] > prefix);
    me[e] = __ballot(i0 + e < n && k[e] == prefix);
    gt += __popcll(mg[e]);
    eq += __popcll(me[e]);
  }
  if (lane == 0) {
    wgt[wave] = gt;
    weq[wave] = eq;
  }
  __syncthreads();
  const uint32_t seg_eq = cut[CUT_SEG + 2 * sg + 1];
  const uint32_t eq0 = seg_eq + sum_before(weq, CHOOSE_W, wave);   // equal ones before this wave
  const uint64_t below = (1ull << lane) - 1;
  // the place of this wave's first taken one, of this lane's
  uint32_t to = cut[CUT_SEG + 2 * sg] + sum_before(wgt, CHOOSE_W, wave) + min(eq0, need) - min(seg_eq, need);
  uint32_t ahead = eq0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    to += __popcll(mg[e] & below);
    ahead += __popcll(me[e] & below);
  }
  to += min(ahead, need) - min(eq0, need);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bool is_eq = (me[e] >> lane) & 1;
    if (((mg[e] >> lane) & 1) || (is_eq && ahead < need)) out[to++] = i0 + e;
    ahead += is_eq;
  }
}
static void choose(const CacheChoose &a, int most, hipStream_t s) {
  if (most > CHOOSE_LDS && a.hists) {
    const dim3 gs((most + CHOOSE_SEG - 1) / CHOOSE_SEG, a.v.nkv, a.v.kv.n_seq);
    hipLaunchKernelGGL(k_cache_collect, gs, dim3(CHOOSE_T), 0, s, a);
    hipLaunchKernelGGL(k_cache_cut, dim3(a.v.nkv, a.v.kv.n_seq), dim3(CHOOSE_T), 0, s, a);
    hipLaunchKernelGGL(k_cache_emit, gs, dim3(CHOOSE_T), 0, s, a);
    return;
  }
  const dim3 g(a.v.nkv, a.v.kv.n_seq), t(CHOOSE_T);
  const size_t lds = (size_t)((most + 255) / 256) * 1024;
  if (most > CHOOSE_LDS) hipLaunchKernelGGL((k_cache_choose<false, false>), g, t, 0, s, a);
  else if (a.weights) hipLaunchKernelGGL((k_cache_choose<true, true>), g, t, lds, s, a);
  else hipLaunchKernelGGL((k_cache_choose<false, true>), g, t, lds, s, a);
}

template <typename T, int D>
static void score_g(const CacheSelect &a, hipStream_t s) {
  // the waves of a workgroup take different heads of the same blocks, whose
  // summaries lie next to each other
  const int nw = min(4, a.v.nkv);
  const dim3 g((a.columns + a.per - 1) / a.per, (a.v.nkv + nw - 1) / nw, a.v.kv.n_seq), t(64 * nw);
  if (a.g == 1) hipLaunchKernelGGL((k_cache_score<T, D, 1>), g, t, 0, s, a);
  else if (a.g == 2) hipLaunchKernelGGL((k_cache_score<T, D, 2>), g, t, 0, s, a);
  else if (a.g <= 4) hipLaunchKernelGGL((k_cache_score<T, D, 4>), g, t, 0, s, a);
  else if constexpr (D < 256) hipLaunchKernelGGL((k_cache_score<T, D, 8>), g, t, 0, s, a);   // g * d <= 1024
}
template <typename T>
static void score_d(const CacheSelect &a, int d, hipStream_t s) {
  if (d == 32) score_g<T, 32>(a, s);
  else if (d == 64) score_g<T, 64>(a, s);
  else if (d == 128) score_g<T, 128>(a, s);
  else score_g<T, 256>(a, s);
}
void launch_cache_select(bool bf16, const CacheSelect &a, int d, hipStream_t s) {
  if (bf16) score_d<bf16_t>(a, d, s);
  else score_d<float>(a, d, s);
  choose({a.v, a.keys, a.ld_keys, nullptr, 0, nullptr, 0, nullptr, 0, nullptr, 1, a.n_take, 0, 0, a.out, nullptr, a.err}, a.columns, s);
}

// ---------------------------------------------------------------- eviction
// Order keys of the slots of one sequence and KV head (those that do not fit
// the choice's LDS), and the histogram of their first digits, two to a word.
__global__ __launch_bounds__(CHOOSE_T) void k_cache_keys(CacheEvict a) {
  constexpr int U = CHOOSE_SEG / CHOOSE_T;
  const int t0 = blockIdx.x * CHOOSE_SEG, j = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  __shared__ uint32_t hist[CHOOSE_T];
  const int n = visible_slots(a.v, b, a.err);
  if (t0 >= n) return;
  hist[tid] = 0;
  __syncthreads();
  const size_t u = (size_t)b * a.v.nkv + j;
  uint32_t row[U];
#pragma unroll
  for (int x = 0; x < U; ++x) {
    const int t = t0 + x * CHOOSE_T + tid, bi = slot_block(a.v.kv, t);
    row[x] = t < n ? pool_row(a.v, a.v.kv.block_table, b, j, bi, slot_in_block(a.v.kv, t, bi), a.err) : NO_ROW;
  }
  float w[U];
#pragma unroll
  for (int x = 0; x < U; ++x) w[x] = a.weights[row[x] == NO_ROW ? 0 : row[x]];
#pragma unroll
  for (int x = 0; x < U; ++x) {
    const int t = t0 + x * CHOOSE_T + tid;
    if (t >= n) break;
    const uint32_t k = row[x] == NO_ROW ? 0u : t < a.n_first || t >= n - a.n_recent ? KEY_FORCED : choice_key(w[x]);
    a.keys[u * a.ld_keys + t] = k;
    atomicAdd(&hist[k >> 22], (k >> 21) & 1 ? 0x10000u : 1u);   // at most CHOOSE_SEG < 2^16 each
  }
  __syncthreads();
  a.hists[u * a.ld_hists + blockIdx.x * 1024 + tid] = hist[tid];
}

// Keys, values and weight of the kept slots to the new blocks: a lane group
// of d / 8 lanes per slot.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_cache_copy(CacheEvict a) {
  constexpr int LPR = D / 8, RPI = 64 / LPR;
  const int lane = threadIdx.x & 63, j = blockIdx.y, b = blockIdx.z;
  const int i = (blockIdx.x * 4 + wave_id()) * RPI + lane / LPR, li = lane % LPR;
  if (i >= a.n_keep) return;
  const int t = a.kept[((size_t)b * a.v.nkv + j) * a.n_keep + i];
  if (t < 0) return;
  const int sb = slot_block(a.v.kv, t), db = slot_block(a.v.kv, i);
  const uint32_t src = pool_row(a.v, a.v.kv.block_table, b, j, sb, slot_in_block(a.v.kv, t, sb), a.err);
  const uint32_t dst = pool_row(a.v, a.new_table, b, j, db, slot_in_block(a.v.kv, i, db), a.err);
  if (src == NO_ROW || dst == NO_ROW) return;
  constexpr int U = sizeof(T) / 2;                 // 16-byte pieces per lane
  const size_t so = (size_t)src * D + 8 * li, to = (size_t)dst * D + 8 * li;
  u32x4 k[U], v[U];
#pragma unroll
  for (int x = 0; x < U; ++x) {
    k[x] = stream16((const u32x4 *)((const T *)a.v.kv.k_pool + so) + x);
    v[x] = stream16((const u32x4 *)((const T *)a.v.kv.v_pool + so) + x);
  }
#pragma unroll
  for (int x = 0; x < U; ++x) {
    ((u32x4 *)((T *)a.v.kv.k_pool + to))[x] = k[x];
    ((u32x4 *)((T *)a.v.kv.v_pool + to))[x] = v[x];
  }
  if (li == 0) a.weights[dst] = a.weights[src];
}

template <typename T>
static void copy_d(const CacheEvict &a, int d, hipStream_t s) {
  const int rpi = 64 / (d / 8);
  const dim3 g((a.n_keep + 4 * rpi - 1) / (4 * rpi), a.v.nkv, a.v.kv.n_seq);
  if (d == 32) hipLaunchKernelGGL((k_cache_copy<T, 32>), g, dim3(256), 0, s, a);
  else if (d == 64) hipLaunchKernelGGL((k_cache_copy<T, 64>), g, dim3(256), 0, s, a);
  else if (d == 128) hipLaunchKernelGGL((k_cache_copy<T, 128>), g, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_cache_copy<T, 256>), g, dim3(256), 0, s, a);
}
void launch_cache_evict(bool bf16, const CacheEvict &a, int d, hipStream_t s) {
  if (a.v.max_len > CHOOSE_LDS)
    hipLaunchKernelGGL(k_cache_keys, dim3((a.v.max_len + CHOOSE_SEG - 1) / CHOOSE_SEG, a.v.nkv, a.v.kv.n_seq),
                       dim3(CHOOSE_T), 0, s, a);
  choose({a.v, a.keys, a.ld_keys, a.hists, a.ld_hists, a.cand, a.ld_cand, a.cut, a.ld_cut, a.weights, 0, a.n_keep,
          a.n_first, a.n_recent, a.kept, a.new_lens, a.err},
         a.v.max_len, s);
  if (bf16) copy_d<bf16_t>(a, d, s);
  else copy_d<float>(a, d, s);
}

}  // namespace prism
