// Attention of several rows per sequence over the paged draft cache, in the
// context's type or in 8 bits: the tokens of a decoding step, drafts to be
// scored, prompts.  Row i of a sequence sees the slots below v = L + n_new + i;
// with a window W those from v - W on and the first n_first.
//
// The rows of a sequence are cut into tiles whose (row, head) pairs of one KV head
// are the 16 columns of a matrix-core tile, or of two.  A segment is a tile of one KV head;
// it walks the slots that any of its rows sees as "places": the first ones, then
// those from the first row's window on.
#include "cache.h"
#include "cache_device.h"

namespace prism {

constexpr int NO_SLOTS = -(1 << 30);       // slots before row 0 of a sequence that sees none

// Per lane b of a wave: the rows of sequence b, its segments, and their place in
// the numbering of granules (in a direct call each segment counts as one).
struct RowWalk {
  int r0, n, v0;              // first row, rows, slots that row 0 sees
  int tiles, count;           // tiles, granules of a segment (at least its places)
  int begin, end, seg_end;    // granules before and through b, segments through b
  int total, per;
  bool bad;
};
__device__ __forceinline__ int visible_of(int v0, int i, int max_len) { return max(0, min(v0 + i, max_len)); }
__device__ __forceinline__ RowWalk row_walk(const RowsAttend &a) {
  const int lane = threadIdx.x & 63, B = a.v.kv.n_seq;
  const bool has = lane < B;
  RowWalk w;
  w.r0 = lane;
  w.n = has;
  w.bad = false;
  if (a.offsets) {
    const int lo = has ? a.offsets[lane] : 0, hi = has ? a.offsets[lane + 1] : 0;
    w.r0 = lo;
    w.n = hi - lo;
    w.bad = __ballot(has && (hi < lo || hi > a.rows || (lane == 0 && lo != 0))) != 0;
    if (w.bad) {
      if (lane == 0) atomicOr(a.err, ERRF_ROWS);
      w.n = 0;
    }
  }
  const int L = has ? a.v.kv.ctx_lens[lane] : 0;
  const long v0 = (long)L + a.v.n_new;
  if (w.n > 0 && (L < 0 || v0 + w.n - 1 > a.v.max_len)) atomicOr(a.err, ERRF_CAPACITY);
  w.v0 = L < 0 ? NO_SLOTS : (int)min(v0, (long)a.v.max_len);
  const int rt = rows_per_tile(a.g, a.cols);
  w.tiles = w.n > a.few ? 0 : (w.n + rt - 1) / rt;   // (k_rows_prompt's)
  if (a.direct) {
    w.count = 1;                           // an empty segment writes its zeros itself
  } else {
    // the last rows see the most, but for a window that tiles of fewer rows overhang less
    const int v = visible_of(w.v0, w.n - 1, a.v.max_len);
    w.count = cache_granules(a.window ? (int)min((long)v, (long)a.n_first + a.window + rt - 1) : v);
  }
  w.end = w.tiles * a.v.nkv * w.count;
  w.seg_end = w.tiles * a.v.nkv;
  const int mine = w.end;
  for (int x = 1; x < B; x *= 2) {
    const int e = __shfl_up(w.end, x, 64), s = __shfl_up(w.seg_end, x, 64);
    if (lane >= x) {
      w.end += e;
      w.seg_end += s;
    }
  }
  w.total = __builtin_amdgcn_readlane(w.end, B - 1);
  w.begin = has ? w.end - mine : w.total;
  if (!has) {
    w.end = w.total;
    w.seg_end = 0x7fffffff;                // no segment lies there
  }
  w.per = cache_run(w.total, a.waves);
  return w;
}
// The part of a segment that a run at granule u (< w.total), ending at `last`,
// begins with; sink, lo: places 0 .. sink - 1 are slots 0 .. sink - 1, the others
// slots from lo on.
struct RowSegment {
  int b, j, tile, index;      // index: segments before it
  int r, i0, rows, v0;        // its first row in q, and in the sequence; its rows; what row 0 of the sequence sees
  int sink, lo, p0, p1, granules;
};
__device__ __forceinline__ void segment_places(const RowsAttend &a, RowSegment &s, int &places) {
  const int first = visible_of(s.v0, s.i0, a.v.max_len), last = visible_of(s.v0, s.i0 + s.rows - 1, a.v.max_len);
  s.lo = a.window ? max(0, first - a.window) : 0;
  s.sink = min(a.n_first, s.lo);
  places = last - s.lo + s.sink;
}
__device__ __forceinline__ RowSegment row_segment_at(const RowsAttend &a, const RowWalk &w, int u, int last) {
  RowSegment s;
  s.b = __popcll(__ballot(w.end <= u));
  const int count = __builtin_amdgcn_readlane(w.count, s.b), tiles = __builtin_amdgcn_readlane(w.tiles, s.b);
  const CacheRun run = cache_run_at(u - __builtin_amdgcn_readlane(w.begin, s.b), count, last - u);
  s.index = __builtin_amdgcn_readlane(w.seg_end, s.b) - tiles * a.v.nkv + run.head;
  s.j = run.head / tiles;
  s.tile = run.head - s.j * tiles;
  const int rt = rows_per_tile(a.g, a.cols);
  s.i0 = s.tile * rt;
  s.rows = min(rt, __builtin_amdgcn_readlane(w.n, s.b) - s.i0);
  s.r = __builtin_amdgcn_readlane(w.r0, s.b) + s.i0;
  s.v0 = __builtin_amdgcn_readlane(w.v0, s.b);
  int places;
  segment_places(a, s, places);
  s.granules = run.granules;
  s.p0 = a.direct ? 0 : min(places, run.first * CACHE_GRAN);
  s.p1 = a.direct ? places : min(places, (run.first + run.granules) * CACHE_GRAN);
  return s;
}

// Rows of the pools in LDS, from 16-byte pieces of them: as they are, or codes
// turned into values by the scale of their block (exactly: e4m3 times a power of
// two is a bf16).
template <typename T, int D, bool Q8>
struct Loader {
  static constexpr int SZ = Q8 ? 1 : (int)sizeof(T);                    // bytes of a stored value
  static constexpr int LPR = D * SZ / 16, RPI = 64 / LPR;               // lanes per row, rows per load
  static constexpr int NI = Tile<T, D>::TS / RPI;                       // loads per tile
  // byte of piece c of row s of the values' tile: in bf16 the transposing read takes
  // two pieces of 8 rows at a time, which this puts in all 64 banks
  __device__ static int v_at(int s, int c) {
    constexpr int L = Tile<T, D>::LPR;
    if constexpr (sizeof(T) == 4) return Tile<T, D>::at(s, c);
    return (s * L + (c ^ (L >= 16 ? 2 * (s & 7) : L == 8 ? s & 6 : (s >> 1) & 2))) * 16;
  }
  // whether one of the values of a piece is an infinity or a NaN
  __device__ static bool odd(u32x4 x) {
    bool r = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (Q8) {
        // a byte of seven ones: adding 1 to the seven carries into the eighth
        r |= (((x[i] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
      } else if constexpr (sizeof(T) == 2) {
        r |= (((x[i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u) != 0;
      } else {
        r |= (x[i] & 0x7f800000u) == 0x7f800000u;
      }
    }
    return r;
  }
  // piece li of row s of a tile to LDS
  template <bool V>
  __device__ static void put(char *tile, int s, int li, u32x4 x, float scale) {
    auto at = [](int s, int c) { return V ? v_at(s, c) : Tile<T, D>::at(s, c); };
    if constexpr (!Q8) {
      *(u32x4 *)(tile + at(s, li)) = x;
    } else if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 y;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          y[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x[2 * h + i], scale, false));
          y[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x[2 * h + i], scale, true));
        }
        *(u32x4 *)(tile + at(s, 2 * li + h)) = y;
      }
    } else {
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)x[h], scale, false);
        const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)x[h], scale, true);
        *(f32x4 *)(tile + at(s, 4 * li + h)) = f32x4{lo[0], lo[1], hi[0], hi[1]};
      }
    }
  }
};
// A value that is not finite must not meet the probability 0 of a column that does
// not see it (0 times it is NaN).  Of a masked tile that holds one, the values that
// are not finite become 0 in LDS, and masks keep their places, for each dim those of
// +inf, -inf and NaN; what a column sees of them is added to its outputs behind the
// product.
typedef uint64_t OddMask[3];
template <typename T>
__device__ __forceinline__ void take_odd(T *v, OddMask &m, int s) {
  const float x = Ty<T>::ld(v, 0);
  if (fabsf(x) < INFINITY) return;
  atomicOr((unsigned long long *)&m[x != x ? 2 : x < 0.f], 1ull << s);
  *v = 0;
}
__device__ __forceinline__ float odd_sum(const OddMask &m, uint64_t see) {
  const bool pos = m[0] & see, neg = m[1] & see, nan = m[2] & see;
  return nan || (pos && neg) ? NAN : pos ? INFINITY : neg ? -INFINITY : 0.f;
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}
// Four probabilities as hi + lo: the first 8 bits, cut off, and what is left rounded to
// 8 (2^-16 of the value at most), neither negative, nor 0 but for p = 0, as in
// split_bf16.
__device__ __forceinline__ void pair_bf16(const f32x4 &p, uint32_t (&hi)[2], uint32_t (&lo)[2]) {
  float l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    l[i] = fmaxf(p[i] - __uint_as_float(__float_as_uint(p[i]) & 0xffff0000u), fminf(p[i], 0x1p-126f));
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    hi[i] = pack_upper(p[2 * i], p[2 * i + 1]);
    lo[i] = pack_bf16(l[2 * i], l[2 * i + 1]);
  }
}

// A wave takes tiles of TS places, as in the attention of one row per sequence
// (cache.hip): rows loaded whole, into operand order through LDS, scores as MFMAs of
// 16 places x 16 columns, outputs as MFMAs of 16 dims x 16 columns, each lane
// holding one column's softmax state.  A column is a (row, head) pair, so a tile's
// rows share what is loaded; where not every row sees every place of a tile, the
// scores are masked place by place.
//   32 sequences of 32768 slots of 8 heads in 8 bits: 2.1 GB in 325 us, 6.6 TB/s (a
// plain stream reads 7.1), bound by memory with the vector units 47% busy; six rows of
// 4 heads of each of 16 sequences: 66 us for 39 us of bytes, bound by the softmax.
template <typename T, int D, bool Q8, int NT, int NW>
__global__ __launch_bounds__(64 * NW, D * sizeof(T) > 512 ? 1 : 2) void k_rows_attend(RowsAttend a) {
  using M = Tile<T, D>;
  using Ld = Loader<T, D, Q8>;
  constexpr int TS = M::TS, LPR = Ld::LPR, RPI = Ld::RPI, NI = Ld::NI, E = 16 / sizeof(T);
  constexpr int NS = TS / 16, NK = M::LPR / 4, ND = D / 16;
  constexpr int TILE = TS * M::LPR * 16;                    // bytes
  __shared__ __attribute__((aligned(16))) char sh[NW][2 * TILE];
  const int wave = NW > 1 ? wave_id() : 0, lane = threadIdx.x & 63, g = a.g;
  char *s_k = sh[wave], *s_v = s_k + TILE;
  const int col = lane & 15, q4 = lane >> 4, grp = lane / LPR, li = lane % LPR;
  const KvArgs &kv = a.v.kv;
  const RowWalk wk = row_walk(a);
  if (wk.bad) return;
  constexpr int NC = 16 * NT;                                // columns of the tile: n * 16 + col
  const int columns = NC / g * g;
  int crow[NT], chead[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    crow[n] = (16 * n + col) / g;
    chead[n] = 16 * n + col - crow[n] * g;
  }
  int u = blockIdx.x * wk.per;
  const int last = min(wk.total, u + wk.per);
  while (u < last) {
    const RowSegment sg = row_segment_at(a, wk, u, last);
    u += sg.granules;
    // of this lane's columns: whether there is a row, and what it sees: slots below
    // vis, from win on or below n_first
    bool used[NT];
    int vis[NT], win[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      used[n] = 16 * n + col < columns && crow[n] < sg.rows;
      vis[n] = used[n] ? visible_of(sg.v0, sg.i0 + crow[n], a.v.max_len) : 0;
      win[n] = a.window ? vis[n] - a.window : 0;
    }
    const int vis_min = visible_of(sg.v0, sg.i0, a.v.max_len);           // slots below it every row sees, if
    const int win_max = a.window ? visible_of(sg.v0, sg.i0 + sg.rows - 1, a.v.max_len) - a.window : 0;   // from here on
    const int32_t *table = kv.block_table + (size_t)sg.b * kv.mbps;
    auto slot_of = [&](int p) { return p < sg.sink ? p : p - sg.sink + sg.lo; };
    // the block of place p (past the end: of the last one), and the pool row and
    // scales of a place
    auto column = [&](int p) { return slot_block(kv, slot_of(min(p, sg.p1 - 1))); };
    auto block = [&](int c) { return c < kv.mbps ? table[c] : -1; };
    struct Row {
      uint32_t row;
      float ks, vs;
    };
    auto row_of = [&](int p, int c, int blk) {
      Row r{NO_ROW, 1.f, 1.f};
      if (p >= sg.p1) return r;
      if (blk < 0 || blk >= kv.n_blocks) {
        atomicOr(a.err, ERRF_CAPACITY);
        return r;
      }
      const uint32_t hb = (uint32_t)blk * a.v.nkv + sg.j;
      r.row = hb * kv.bs + (slot_of(p) - c * kv.bs);
      if constexpr (Q8) {
        const float2 s = *(const float2 *)(a.scales + 2 * (size_t)hb);
        r.ks = s.x;
        r.vs = s.y;
      }
      return r;
    };
    u32x4 kr[NI], vr[NI];
    // nontemporal: where tiles of a sequence share its slots that costs at most 3%
    // (1000 fp32 rows of 32 heads), where each slot is read once it gives 3 to 8
    auto load = [&](uint32_t row) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const uint32_t r = __shfl(row, i * RPI + grp, 64);
        const size_t at = (size_t)(r == NO_ROW ? 0 : r) * (D * Ld::SZ) + 16 * li;   // a masked place reads row 0
        kr[i] = stream16((const char *)kv.k_pool + at);
        vr[i] = stream16((const char *)kv.v_pool + at);
      }
    };
    float m_run[NT], l_run[NT];
    f32x4 o[NT][ND];
    u32x4 qf[NT][NK];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      m_run[n] = -INFINITY;
      l_run[n] = 0.f;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) o[n][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
      const size_t hi = (size_t)(sg.r + crow[n]) * a.nq + sg.j * g + chead[n];
#pragma unroll
      for (int kk = 0; kk < NK; ++kk)
        qf[n][kk] = used[n] ? *(const u32x4 *)((const T *)a.q + hi * D + (4 * kk + q4) * E) : u32x4{0, 0, 0, 0};
    }
    constexpr int STEP = NW * TS;
    const int t0 = sg.p0 + wave * TS;
    int c1 = 0, b1 = 0;
    Row row{NO_ROW, 1.f, 1.f};
    if (t0 < sg.p1) {
      const int c0 = column(t0 + lane), b0 = block(c0);
      c1 = column(t0 + STEP + lane);
      b1 = block(c1);
      if (lane < TS) row = row_of(t0 + lane, c0, b0);
      load(row.row);
    }
    for (int t = t0; t < sg.p1; t += STEP) {
      const uint64_t mask = __ballot(row.row != NO_ROW);
      constexpr uint64_t FULL = TS == 64 ? ~0ull : (1ull << (TS & 63)) - 1;
      if (mask != FULL) {
        const uint64_t mine = mask >> grp;
#pragma unroll
        for (int i = 0; i < NI; ++i)
          if (!((uint32_t)(mine >> (i * RPI)) & 1)) vr[i] = u32x4{0, 0, 0, 0};
      }
      // whether every row sees every place of the tile that has a row
      const int top = slot_of(t + TS - 1);
      const bool whole = sg.rows == 1 ||
                         (min(top, slot_of(sg.p1 - 1)) < vis_min &&
                          (!a.window || slot_of(t) >= win_max || t + TS <= sg.sink));
      bool odd = false;
      if (!whole) {
#pragma unroll
        for (int i = 0; i < NI; ++i) odd |= Ld::odd(vr[i]);
        odd = __ballot(odd) != 0;
      }
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int s = i * RPI + grp;
        Ld::template put<false>(s_k, s, li, kr[i], Q8 ? __shfl(row.ks, s, 64) : 1.f);
        Ld::template put<true>(s_v, s, li, vr[i], Q8 ? __shfl(row.vs, s, 64) : 1.f);
      }
      if (t + STEP < sg.p1) {
        row = Row{NO_ROW, 1.f, 1.f};
        if (lane < TS) row = row_of(t + STEP + lane, c1, b1);
        c1 = column(t + 2 * STEP + lane);
        b1 = block(c1);
        load(row.row);
      }
      wave_lds_sync();
      // scores S[place 16 st + 4 q4 + i][column 16 n + col]
      f32x4 sc[NT][NS];
#pragma unroll
      for (int st = 0; st < NS; ++st) {
#pragma unroll
        for (int n = 0; n < NT; ++n) sc[n][st] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (sizeof(T) == 4) {
          // four sums of a quarter of the dims each: a single one of d terms in fp32 is
          // twice as far off (1.2e-6 of the outputs with d = 256)
          f32x4 part[3] = {};
#pragma unroll
          for (int kk = 0; kk < NK; ++kk) {
            const f32x4 kf = *(const f32x4 *)(s_k + M::at(16 * st + col, 4 * kk + q4)), q = __builtin_bit_cast(f32x4, qf[0][kk]);
            sc[0][st] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[0], q[0], sc[0][st], 0, 0, 0);
#pragma unroll
            for (int x = 0; x < 3; ++x) part[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[x + 1], q[x + 1], part[x], 0, 0, 0);
          }
          sc[0][st] = (sc[0][st] + part[0]) + (part[1] + part[2]);
        } else {
#pragma unroll
          for (int kk = 0; kk < NK; ++kk) {
            const u32x4 kf = *(const u32x4 *)(s_k + M::at(16 * st + col, 4 * kk + q4));
#pragma unroll
            for (int n = 0; n < NT; ++n) sc[n][st] = Ty<T>::mma(kf, qf[n][kk], sc[n][st]);
          }
        }
      }
      uint32_t sees[NT];                                   // bit 4 st + i: the column sees that place
      const uint64_t mine = mask >> (4 * q4);              // from this lane's first place on
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        sees[n] = ~0u;
        if (!whole || mask != FULL) {
          sees[n] = 0;
#pragma unroll
          for (int st = 0; st < NS; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int slot = slot_of(t + 4 * q4 + 16 * st + i);
              const bool see = ((uint32_t)(mine >> (16 * st)) & (1u << i)) && slot < vis[n] && (slot >= win[n] || slot < a.n_first);
              sees[n] |= (uint32_t)see << (4 * st + i);
              sc[n][st][i] = see ? sc[n][st][i] : -INFINITY;
            }
        }
        float mx = -INFINITY;
#pragma unroll
        for (int st = 0; st < NS; ++st)
#pragma unroll
          for (int i = 0; i < 4; ++i) mx = fmaxf(mx, sc[n][st][i]);
        mx = fmaxf(mx, xor16_f(mx));
        mx = fmaxf(mx, xor32_f(mx)) * a.scale;
        const float mn = fmaxf(m_run[n], mx);
        // nothing but -inf so far: subtract 0, so that every p is 0 (a NaN score
        // still makes its p, and with it the sum and the output, NaN)
        const float ms = mn == -INFINITY ? 0.f : mn;
        const float al = __builtin_amdgcn_exp2f(m_run[n] - ms);
        m_run[n] = mn;
        float ls = 0.f;
#pragma unroll
        for (int st = 0; st < NS; ++st)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            sc[n][st][i] = __builtin_amdgcn_exp2f(fmaf(sc[n][st][i], a.scale, -ms));
            ls += sc[n][st][i];
          }
        ls += xor16_f(ls);
        ls += xor32_f(ls);
        l_run[n] = l_run[n] * al + ls;
        if (__ballot(al != 1.f)) {
#pragma unroll
          for (int dt = 0; dt < ND; ++dt) o[n][dt] *= al;
        }
      }
      // O[dim 16 dt + 4 q4 + i][column 16 n + col]
      constexpr int NP = sizeof(T) == 2 && NS > 1 ? 2 : 1;   // groups of 16 places per bf16 MFMA (32 places, or 16)
      OddMask *masks = (OddMask *)s_k;                     // [D], over the keys, whose scores are done
      static_assert(D * sizeof(OddMask) <= TILE, "masks fit the K tile");
      if (odd) {
        wave_lds_sync();
        for (int i = lane; i < 3 * D; i += 64) masks[i / 3][i % 3] = 0;
        wave_lds_sync();
        for (int i = lane; i < TS * D; i += 64) {
          const int p = i / D, dim = i % D;
          take_odd((T *)(s_v + Ld::v_at(p, dim / E)) + dim % E, masks[dim], p);
        }
        wave_lds_sync();
      }
#pragma unroll
      for (int st = 0; st < NS; st += NP) {
        if constexpr (sizeof(T) == 2) {
          uint32_t hi[NT][2 * NP], mid[NT][2 * NP], lo[NT][2 * NP];
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int x = 0; x < NP; ++x) {
              uint32_t h[2], m[2], l[2];
              if constexpr (NT == 1) split_bf16(sc[n][st + x], h, m, l);
              else pair_bf16(sc[n][st + x], h, m);
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                hi[n][2 * x + y] = h[y];
                mid[n][2 * x + y] = m[y];
                if constexpr (NT == 1) lo[n][2 * x + y] = l[y];
              }
            }
#pragma unroll
          for (int dt = 0; dt < ND; ++dt) {
            uint32_t v[2 * NP];
#pragma unroll
            for (int x = 0; x < NP; ++x) {
              const char *pv = s_v + Ld::v_at(16 * (st + x) + 4 * q4 + (col >> 2), 2 * dt + ((col & 3) >> 1)) + 8 * (col & 1);
              const uint2 r = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)pv));
              v[2 * x] = r.x;
              v[2 * x + 1] = r.y;
            }
            // k = 8 q4 + e: places 16 st + 4 q4 + e, then the same of st + 1, in both operands
            auto mma = [&](const uint32_t(&x)[2 * NP], const uint32_t(&y)[2 * NP], f32x4 acc) {
              if constexpr (NP == 2)
                return Ty<T>::mma(u32x4{x[0], x[1], x[2], x[3]}, u32x4{y[0], y[1], y[2], y[3]}, acc);
              else
                return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, uint2{x[0], x[1]}),
                                                                __builtin_bit_cast(s16x4, uint2{y[0], y[1]}), acc, 0, 0, 0);
            };
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              o[n][dt] = mma(v, hi[n], o[n][dt]);
              o[n][dt] = mma(v, mid[n], o[n][dt]);
              if constexpr (NT == 1) o[n][dt] = mma(v, lo[n], o[n][dt]);
            }
          }
        } else {
          // step i: place 4 q4 + i of each lane row
#pragma unroll
          for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const char *pv = s_v + Ld::v_at(16 * st + 4 * q4 + i, 4 * dt + (col >> 2)) + 4 * (col & 3);
              const float v = *(const float *)pv;
#pragma unroll
              for (int n = 0; n < NT; ++n) o[n][dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, sc[n][st][i], o[n][dt], 0, 0, 0);
            }
        }
      }
      if (odd) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          // the places that this column sees, those of its four lanes
          uint64_t see = 0;
#pragma unroll
          for (int st = 0; st < NS; ++st) see |= (uint64_t)((sees[n] >> (4 * st)) & 15) << (16 * st + 4 * q4);
          see |= __shfl_xor(see, 16, 64);
          see |= __shfl_xor(see, 32, 64);
#pragma unroll
          for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              o[n][dt][i] += odd_sum(masks[16 * dt + 4 * q4 + i], see);
              __builtin_amdgcn_sched_barrier(0);            // few registers rather than overlap
            }
        }
      }
      wave_lds_sync();                                 // reads done before the next tile's writes
    }
    if constexpr (NW > 1) {
      __shared__ float s_m[NW][NC], s_l[NW][NC];
      float *so = (float *)s_k;                        // this wave's outputs [NC][D]: within its K and V tiles
      static_assert(2 * TILE >= NC * D * (int)sizeof(float), "outputs of a wave fit its tiles");
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        if (used[n]) {
#pragma unroll
          for (int dt = 0; dt < ND; ++dt) *(f32x4 *)(so + (16 * n + col) * D + 16 * dt + 4 * q4) = o[n][dt];
        }
        if (q4 == 0) {
          s_m[wave][16 * n + col] = m_run[n];
          s_l[wave][16 * n + col] = l_run[n];
        }
      }
      __syncthreads();
      for (int e = threadIdx.x; e < sg.rows * g * D / 4; e += 64 * NW) {
        const int c = e / (D / 4);
        float M2 = -INFINITY, l = 0.f;
        for (int w = 0; w < NW; ++w) M2 = fmaxf(M2, s_m[w][c]);
        M2 = M2 == -INFINITY ? 0.f : M2;
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < NW; ++w) {
          const float wt = __builtin_amdgcn_exp2f(s_m[w][c] - M2);
          l += s_l[w][c] * wt;
          y += *(const f32x4 *)((const float *)sh[w] + 4 * e) * wt;
        }
        if (l == 0.f) y = f32x4{0.f, 0.f, 0.f, 0.f};   // (0 times a value that is not finite)
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const float z[4] = {y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv};
        const size_t at = (size_t)(sg.r + c / g) * a.nq + sg.j * g + c % g;
        store_n<T, 4>((T *)a.out + at * D + 4 * (e % (D / 4)), z);
        if (a.lse && e % (D / 4) == 0) a.lse[at] = l == 0.f ? -INFINITY : (M2 + log2f(l)) * LN2;
      }
      return;                                          // one segment per workgroup
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (!used[n]) continue;
      const size_t part = (size_t)cache_partial(blockIdx.x, sg.index) * columns + 16 * n + col;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) *(f32x4 *)(a.po + part * D + 16 * dt + 4 * q4) = o[n][dt];
      if (q4 == 0) {
        a.pm[part] = m_run[n];
        a.pl[part] = l_run[n];
      }
    }
  }
}

// Join: T threads per column add its partial outputs, each weighted by 2^(its
// maximum - the largest one), in an order that only the lengths set.
template <typename T, int D, int TH>
__global__ __launch_bounds__(256) void k_rows_join(RowsAttend a) {
  constexpr int Q = D / 4, G = TH / Q, PRE = 4;
  const int tid = threadIdx.x, lane = tid & 63;
  const RowWalk w = row_walk(a);
  if (w.bad) return;
  const int rt = rows_per_tile(a.g, a.cols), columns = rt * a.g;
  // the column of this group of threads (whole waves), the same in each of its lanes
  const int id = __builtin_amdgcn_readfirstlane(blockIdx.x * (256 / TH) + tid / TH), t = tid % TH;
  const int seg = id / columns, col = id - seg * columns;
  const int b = __popcll(__ballot(w.seg_end <= seg));
  if (b >= a.v.kv.n_seq) return;
  const int tiles = __builtin_amdgcn_readlane(w.tiles, b), count = __builtin_amdgcn_readlane(w.count, b);
  const int x = seg - (__builtin_amdgcn_readlane(w.seg_end, b) - tiles * a.v.nkv), j = x / tiles;
  const int i = (x - j * tiles) * rt + col / a.g;
  if (i >= __builtin_amdgcn_readlane(w.n, b)) return;
  const size_t hi = (size_t)(__builtin_amdgcn_readlane(w.r0, b) + i) * a.nq + j * a.g + col % a.g;
  const CacheParts p = cache_parts(__builtin_amdgcn_readlane(w.begin, b) + x * count, count, w.per);
  const size_t at = (size_t)cache_partial(p.wave, seg) * columns + col;
  const int q = t % Q, grp = t / Q;
  f32x4 pre[PRE];
  float pm[PRE];
#pragma unroll
  for (int k = 0; k < PRE; ++k) {
    const int c = grp + k * G;
    pre[k] = c < p.n ? *(const f32x4 *)(a.po + (at + (size_t)c * columns) * D + 4 * q) : f32x4{0.f, 0.f, 0.f, 0.f};
  }
#pragma unroll
  for (int k = 0; k < PRE; ++k) {
    const int c = grp + k * G;
    pm[k] = c < p.n ? a.pm[at + (size_t)c * columns] : -INFINITY;
  }
  float m = -INFINITY, l = 0.f;
  for (int c = lane; c < p.n; c += 64) m = fmaxf(m, a.pm[at + (size_t)c * columns]);
  float top = wave_max(m);
  top = top == -INFINITY ? 0.f : top;
  for (int c = lane; c < p.n; c += 64) l += a.pl[at + (size_t)c * columns] * exp2f(a.pm[at + (size_t)c * columns] - top);
  l = wave_sum(l);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < PRE; ++k) o += pre[k] * exp2f(pm[k] - top);
#pragma unroll 4
  for (int c = grp + PRE * G; c < p.n; c += G) {
    const size_t k = at + (size_t)c * columns;
    o += *(const f32x4 *)(a.po + k * D + 4 * q) * exp2f(a.pm[k] - top);
  }
  if constexpr (TH == 64) {
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = stride_sum(o[k], Q);
  } else {
    __shared__ float red[TH * 4];
    *(f32x4 *)(red + 4 * t) = o;
    __syncthreads();
    if (grp == 0)
      for (int y = 1; y < G; ++y) o += *(const f32x4 *)(red + 4 * (y * Q + q));
  }
  if (grp == 0) {
    const float z[4] = {l == 0.f ? 0.f : o[0] / l, l == 0.f ? 0.f : o[1] / l, l == 0.f ? 0.f : o[2] / l,
                        l == 0.f ? 0.f : o[3] / l};
    store_n<T, 4>((T *)a.out + hi * D + 4 * q, z);
  }
  if (t == 0 && a.lse) a.lse[hi] = l == 0.f ? -INFINITY : (top + log2f(l)) * LN2;
}

// ---------------------------------------------------------------- prompts
// Sequences of more than a.few rows in bf16 contexts.  A workgroup takes a tile of
// prompt_columns (row, head) pairs of one KV head, 32 columns a wave, and walks its
// places BN at a time: S = K Q^T and O = V^T P as MFMAs of 32 x 32, so that a lane
// holds one column's probabilities just where the second product takes them.
// Probabilities are rounded to bf16 for it (2^-9 of each on average over a sum of
// many, as much as the rounding of the output; the sum of a row takes them
// unrounded): in three parts they would double the work of the larger product.
//   What is subtracted from the scores lies up to 2^8 above the largest so far and
// follows only a score that passes it, so that outputs are seldom rescaled and no
// probability is above 1: as in the tiles of rows, sums leave fp32's range where the
// values times the slots do.  Below 2^-118 of the largest a probability may be 0.
// Each column decides for itself, so that no other row's scores change how its
// probabilities are rounded.
//   Rows of K and V go through registers (8-bit ones become bf16 on the way) to one
// of two LDS buffers, one tile ahead of the products, their loads two tiles ahead
// and block-table lookups three: one barrier per tile.
//   8192 rows of 32 heads: 630 us, 873 TFLOP/s, 72% of what a large product of the
// vendor's library reaches here; the matrix units are busy 33% of the cycles, the
// vector units 40%, and a wave waits 36% of its time, so their overlap bounds it.
typedef float f32x16 __attribute__((ext_vector_type(16)));
constexpr float PROMPT_SLACK = 8.f;
// LDS written by the workgroup is there, with global loads still in flight
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
template <int D>
struct PromptTile {
  static constexpr int BN = D == 256 ? 32 : 64;             // places
  static constexpr int LPR = D / 8;                         // 16-byte pieces of a row
  static constexpr int BYTES = BN * D * 2;
  // byte of piece c of row s: permuted so that what is read together lies in all 64
  // banks (keys: one piece of 16 rows; values: four pieces of 4 rows).  At rows and
  // pieces 16 further it is the same by step(), so a lane keeps few addresses.
  __device__ static int k_at(int s, int c) { return (s * LPR + (c ^ (LPR >= 16 ? s & 15 : LPR == 8 ? (s >> 1) & 7 : (s >> 2) & 3))) * 16; }
  __device__ static int v_at(int s, int c) { return (s * LPR + (c ^ (LPR >= 16 ? 4 * (s & 3) : LPR == 8 ? 4 * ((s >> 1) & 1) : 0))) * 16; }
  __device__ static constexpr int step(int rows, int pieces) { return (rows * LPR + pieces) * 16; }
};
template <int D, bool Q8>
__global__ __launch_bounds__(2 * prompt_columns(D), D == 256 ? 1 : 2) void k_rows_prompt(RowsAttend a) {
  using PT = PromptTile<D>;
  constexpr int BN = PT::BN, NS = BN / 32, NK = D / 16, ND = D / 32;
  constexpr int LPR = Q8 ? D / 16 : D / 8, RPI = 2 * prompt_columns(D) / LPR, NI = (BN + RPI - 1) / RPI;   // lanes per stored row, rows per load, loads
  __shared__ __attribute__((aligned(16))) char s_k[2][PT::BYTES], s_v[2][PT::BYTES];
  __shared__ OddMask s_mask[D];
  __shared__ int s_odd[3];                                  // of the tiles in turn: whether a masked one holds
                                                            // what is not finite
  const int tid = threadIdx.x, wave = wave_id(), lane = tid & 63, half = lane >> 5, g = a.g, nkv = a.v.nkv;
  const KvArgs &kv = a.v.kv;
  // the segment: KV heads fastest (workgroups of one head meet in the XCDs' L2
  // where there are 8 of them), the tiles that see most first
  int b, j, tile;
  RowSegment sg;
  {
    const RowWalk w = row_walk(a);
    if (w.bad) return;
    const int tiles = w.n > a.few ? (w.n + prompt_rows(g, D) - 1) / prompt_rows(g, D) : 0;
    const uint32_t end = wave_scan((uint32_t)(lane < kv.n_seq ? tiles * nkv : 0));
    b = __popcll(__ballot(end <= blockIdx.x));
    if (b >= kv.n_seq) return;
    const int nt = __builtin_amdgcn_readlane(tiles, b);
    const int at = (int)blockIdx.x - ((int)__builtin_amdgcn_readlane(end, b) - nt * nkv);
    tile = nt - 1 - at / nkv;
    j = at % nkv;
    sg.v0 = __builtin_amdgcn_readlane(w.v0, b);
    sg.i0 = tile * prompt_rows(g, D);
    sg.rows = min(prompt_rows(g, D), __builtin_amdgcn_readlane(w.n, b) - sg.i0);
    sg.r = __builtin_amdgcn_readlane(w.r0, b) + sg.i0;
  }
  int places;
  segment_places(a, sg, places);
  const int granules = (places + BN - 1) / BN;
  const int p_begin = (int)((long)granules * blockIdx.y / gridDim.y) * BN;
  const int p_end = min(places, (int)((long)granules * (blockIdx.y + 1) / gridDim.y) * BN);
  const int sink = sg.sink, shift = sg.lo - sink;
  auto slot_of = [&](int p) { return p < sink ? p : p + shift; };

  // this lane's column, and what the wave's columns see
  const int cid = 32 * wave + (lane & 31), crow = cid / g, chead = cid - crow * g;
  const bool used = crow < sg.rows && crow < prompt_rows(g, D);
  const size_t hi = (size_t)(sg.r + crow) * a.nq + j * g + chead;
  const int vis = used ? visible_of(sg.v0, sg.i0 + crow, a.v.max_len) : 0, win = a.window ? vis - a.window : 0;
  const int row_a = 32 * wave / g, row_b = min(sg.rows, prompt_rows(g, D)) - 1;
  const bool some = row_a <= row_b;
  const int vis_a = visible_of(sg.v0, sg.i0 + row_a, a.v.max_len);
  const int vis_b = visible_of(sg.v0, sg.i0 + min(row_b, (32 * wave + 31) / g), a.v.max_len);
  const int seg_a = visible_of(sg.v0, sg.i0, a.v.max_len), seg_b = visible_of(sg.v0, sg.i0 + row_b, a.v.max_len);
  // whether rows that see va .. vb slots all see every place of the tile at t
  auto whole_for = [&](int t, int va, int vb) {
    return t + BN <= p_end && slot_of(t + BN - 1) < va && (!a.window || slot_of(t) >= vb - a.window || t + BN <= sink);
  };

  u32x4 qf[NK];
  {
    const bf16_t *q = (const bf16_t *)a.q + (used ? hi : 0) * D + 8 * half;   // (a column of no row: another's)
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) qf[kk] = *(const u32x4 *)(q + 16 * kk);
  }
  f32x16 o[ND];
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  float m_run = -INFINITY;                                  // what is subtracted
  float l_run = 0.f;                                        // over this lane's half of the places

  // Loads: a lane of each wave looks up one place of a tile, and takes piece li of
  // row grp of each pass.
  const int32_t *table = kv.block_table + (size_t)b * kv.mbps;
  const int grp = tid / LPR, li = tid % LPR;
  const bool loads = RPI <= BN || grp < BN;                 // a load may cover more than a tile (d = 32, 8 bits)
  const float inv_bs = 1.f / (float)kv.bs;
  // table column of a slot (below 2^20): the quotient by way of fp32 is off by one at
  // most
  auto column = [&](int slot) {
    int c = (int)((float)slot * inv_bs);
    c -= c * kv.bs > slot;
    return c + ((c + 1) * kv.bs <= slot);
  };
  u32x4 kr[NI], vr[NI];
  uint32_t exps[Q8 ? NI : 1];                               // scales of keys and values: their upper halves
  int col_next, blk_next;                                   // of this lane's place of the tile to be loaded
  uint64_t m_load = 0;                                      // places of the loaded tile with a row
  auto look_up = [&](int t) {
    col_next = column(slot_of(min(t + lane, p_end - 1)));
    blk_next = table[min(col_next, kv.mbps - 1)];
  };
  auto load = [&](int t) {
    const int p = t + lane;
    const bool due = lane < BN && p < p_end, there = due && blk_next >= 0 && blk_next < kv.n_blocks;
    m_load = __ballot(there);
    if (__ballot(due && !there)) atomicOr(a.err, ERRF_CAPACITY);
    const uint32_t hb = there ? (uint32_t)blk_next * nkv + j : 0u;
    const uint32_t row = there ? hb * kv.bs + (uint32_t)(slot_of(p) - col_next * kv.bs) : 0u;   // (row 0: masked)
    uint32_t ex = 0;
    if constexpr (Q8) {
      const uint2 sc = *(const uint2 *)(a.scales + 2 * (size_t)hb);
      ex = there ? (sc.x >> 16) | (sc.y & 0xffff0000u) : 0x3f803f80u;   // (a scale of 1: the 0 of a masked place stays 0)
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int from = i * RPI + grp;
      const size_t at = (size_t)__shfl(row, from, 64) * (D * (Q8 ? 1 : 2)) + 16 * li;
      kr[i] = *(const u32x4 *)((const char *)kv.k_pool + at);
      vr[i] = *(const u32x4 *)((const char *)kv.v_pool + at);
      if constexpr (Q8) exps[i] = __shfl(ex, from, 64);
    }
  };
  constexpr int PP = Q8 ? 2 : 1, PR = RPI % 16 ? 2 : 1;      // pieces in LDS of a loaded one; loads per 16 rows
  static_assert(RPI % 8 == 0, "a thread's rows repeat modulo 16");
  int put_k[PR][PP], put_v[PP];
#pragma unroll
  for (int h = 0; h < PP; ++h) {
#pragma unroll
    for (int i = 0; i < PR; ++i) put_k[i][h] = PT::k_at(grp + i * RPI, PP * li + h) - PT::step(i * RPI, 0);
    put_v[h] = PT::v_at(grp, PP * li + h);
  }
  // the operands' pieces: keys of place lane % 32, values of the places and dims
  // that the transposing read takes from this lane
  constexpr int KA = NK < 8 ? NK : 8, VA = ND < 4 ? ND : 4;
  int get_k[KA], get_v[VA];
#pragma unroll
  for (int x = 0; x < KA; ++x) get_k[x] = PT::k_at(lane & 31, 2 * x + half);
#pragma unroll
  for (int x = 0; x < VA; ++x) {
    const int c = lane & 15;
    get_v[x] = PT::v_at(4 * half + (c >> 2), 4 * x + 2 * ((lane >> 4) & 1) + ((c & 3) >> 1)) + 8 * (c & 1);
  }
  constexpr uint64_t FULL = BN == 64 ? ~0ull : (1ull << (BN & 63)) - 1;
  auto put = [&](int t, int buf, int turn) {
    if (m_load != FULL) {
      const uint64_t mine = m_load >> (grp & 63);
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (!((uint32_t)(mine >> (i * RPI & 63)) & 1)) vr[i] = u32x4{0, 0, 0, 0};
    }
    if (!whole_for(t, seg_a, seg_b)) {
      bool odd = false;
#pragma unroll
      for (int i = 0; i < NI; ++i) odd |= Loader<bf16_t, D, Q8>::odd(vr[i]);
      if (odd) s_odd[turn] = 1;
    }
    if (!loads) return;
    char *bk = s_k[buf], *bv = s_v[buf];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      if constexpr (Q8) {
        const float ks = __uint_as_float(exps[i] << 16), vs = __uint_as_float(exps[i] & 0xffff0000u);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          u32x4 x, y;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            x[2 * k] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)kr[i][2 * h + k], ks, false));
            x[2 * k + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)kr[i][2 * h + k], ks, true));
            y[2 * k] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)vr[i][2 * h + k], vs, false));
            y[2 * k + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)vr[i][2 * h + k], vs, true));
          }
          *(u32x4 *)(bk + put_k[i % PR][h] + PT::step(i * RPI, 0)) = x;
          *(u32x4 *)(bv + put_v[h] + PT::step(i * RPI, 0)) = y;
        }
      } else {
        *(u32x4 *)(bk + put_k[i % PR][0] + PT::step(i * RPI, 0)) = kr[i];
        *(u32x4 *)(bv + put_v[0] + PT::step(i * RPI, 0)) = vr[i];
      }
    }
  };

  if (tid < 3) s_odd[tid] = 0;
  __syncthreads();
  uint64_t m_tile = 0;
  if (p_begin < p_end) {
    look_up(p_begin);
    load(p_begin);
    look_up(p_begin + BN);
    put(p_begin, 0, 0);
    m_tile = m_load;
    if (p_begin + BN < p_end) {
      load(p_begin + BN);
      look_up(p_begin + 2 * BN);
    }
  }
  int buf = 0, turn = 0;                                    // tile / BN modulo 2 and 3
  for (int t = p_begin; t < p_end; t += BN, buf ^= 1, turn = turn == 2 ? 0 : turn + 1) {
    lds_barrier();
    const int next = turn == 2 ? 0 : turn + 1, after = next == 2 ? 0 : next + 1;
    if (tid == 0) s_odd[after] = 0;                         // of the tile before; set again behind the next barrier
    const uint64_t held = m_tile;                           // places of this tile with a row
    if (t + BN < p_end) {
      put(t + BN, buf ^ 1, next);
      m_tile = m_load;
      if (t + 2 * BN < p_end) {
        load(t + 2 * BN);
        look_up(t + 3 * BN);
      }
    }
    const bool odd = s_odd[turn] != 0;
    const char *bk = s_k[buf], *bv = s_v[buf];
    if (odd) {                                              // the same for the workgroup
      for (int i = tid; i < 3 * D; i += 2 * prompt_columns(D)) s_mask[i / 3][i % 3] = 0;
      lds_barrier();
      for (int i = tid; i < BN * D; i += 2 * prompt_columns(D)) {
        const int s = i / D, dim = i % D;
        take_odd((bf16_t *)(s_v[buf] + PT::v_at(s, dim >> 3)) + (dim & 7), s_mask[dim], s);
      }
      lds_barrier();
    }
    const int first = slot_of(t), last_slot = slot_of(min(t + BN, p_end) - 1);
    const bool skip = !some || first >= vis_b || (a.window && last_slot < vis_a - a.window && first >= a.n_first);
    const bool whole = whole_for(t, vis_a, vis_b) && held == FULL;
    if (!skip) {
      // scores S[place 32 st + 8 jj + 4 half + i][column lane % 32]
      f32x16 sc[NS];
#pragma unroll
      for (int st = 0; st < NS; ++st)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[st][i] = 0.f;
#pragma unroll
      for (int kk = 0; kk < NK; ++kk)
#pragma unroll
        for (int st = 0; st < NS; ++st)
          sc[st] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              __builtin_bit_cast(bf16x8, *(const u32x4 *)(bk + get_k[kk % KA] + PT::step(32 * st, 16 * (kk / KA)))),
              __builtin_bit_cast(bf16x8, qf[kk]), sc[st], 0, 0, 0);
      uint32_t sees = ~0u;                                  // bit 16 st + i
      if (!whole) {
        sees = 0;
        const uint64_t mine = held >> (4 * half);           // from this lane's first place on
        const int p0 = t + 4 * half;
#pragma unroll
        for (int st = 0; st < NS; ++st)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int x = 8 * (i >> 2) + (i & 3), slot = slot_of(p0 + 32 * st + x);
            const bool see = ((uint32_t)(mine >> (32 * st)) & (1u << x)) && slot < vis && (slot >= win || slot < a.n_first);
            sees |= (uint32_t)see << (16 * st + i);
            sc[st][i] = see ? sc[st][i] : -INFINITY;
          }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int st = 0; st < NS; ++st)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[st][i]);
      mx = fmaxf(mx, xor32_f(mx)) * a.scale;
      const bool up = mx > m_run;                           // (from -inf: any score that is not)
      if (__ballot(up)) {
        const float ms = mx + PROMPT_SLACK, al = up ? __builtin_amdgcn_exp2f(m_run - ms) : 1.f;
        m_run = up ? ms : m_run;
        l_run *= al;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[dt][i] *= al;
      }
      const float ms = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
      for (int st = 0; st < NS; ++st)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          sc[st][i] = __builtin_amdgcn_exp2f(fmaf(sc[st][i], a.scale, -ms));
          l_run += sc[st][i];
        }
      // O[dim 32 dt + 8 jj + 4 half + i][column lane % 32]
#pragma unroll
      for (int x = 0; x < 2 * NS; ++x) {                    // places 16 x .. 16 x + 15
        u32x4 pb;
#pragma unroll
        for (int k = 0; k < 4; ++k) pb[k] = pack_bf16(sc[x >> 1][8 * (x & 1) + 2 * k], sc[x >> 1][8 * (x & 1) + 2 * k + 1]);
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
          uint2 v[2];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const char *pv = bv + get_v[dt % VA] + PT::step(16 * x + 8 * y, 16 * (dt / VA));
            v[y] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)pv));
          }
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              __builtin_bit_cast(bf16x8, u32x4{v[0].x, v[0].y, v[1].x, v[1].y}), __builtin_bit_cast(bf16x8, pb), o[dt], 0, 0, 0);
        }
      }
      if (odd) {
        // the places that this column sees, those of both halves of the lanes
        uint64_t see = 0;
#pragma unroll
        for (int st = 0; st < NS; ++st)
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) see |= (uint64_t)((sees >> (16 * st + 4 * jj)) & 15) << (32 * st + 8 * jj + 4 * half);
        see |= __shfl_xor(see, 32, 64);
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            o[dt][i] += odd_sum(s_mask[32 * dt + 8 * (i >> 2) + 4 * half + (i & 3)], see);
            __builtin_amdgcn_sched_barrier(0);              // few registers rather than overlap
          }
      }
    }
  }
  const float l = l_run + xor32_f(l_run);
  if (!used) return;
  if (gridDim.y > 1) {
    const size_t part = (size_t)blockIdx.y * a.rows * a.nq + hi;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int jj = 0; jj < 4; ++jj)
        *(f32x4 *)(a.po2 + part * D + 32 * dt + 8 * jj + 4 * half) =
            f32x4{o[dt][4 * jj], o[dt][4 * jj + 1], o[dt][4 * jj + 2], o[dt][4 * jj + 3]};
    if (half == 0) {
      a.pm2[part] = m_run;
      a.pl2[part] = l;
    }
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) {
      // (an output is not finite with l = 0 where a value is not)
      const float z[4] = {l == 0.f ? 0.f : o[dt][4 * jj] * inv, l == 0.f ? 0.f : o[dt][4 * jj + 1] * inv,
                          l == 0.f ? 0.f : o[dt][4 * jj + 2] * inv, l == 0.f ? 0.f : o[dt][4 * jj + 3] * inv};
      store_n<bf16_t, 4>((bf16_t *)a.out + hi * D + 32 * dt + 8 * jj + 4 * half, z);
    }
  if (a.lse && half == 0) a.lse[hi] = l == 0.f ? -INFINITY : (m_run + log2f(l)) * LN2;
}
// Join of a prompt's splits: D / 4 threads per (row, head), in the order of the
// splits.
template <int D>
__global__ __launch_bounds__(256) void k_prompt_join(RowsAttend a, int splits) {
  const RowWalk w = row_walk(a);
  if (w.bad) return;
  const long id = (long)blockIdx.x * (256 / (D / 4)) + threadIdx.x / (D / 4);
  const int q = threadIdx.x % (D / 4);
  const long row = id / a.nq;
  // rows of sequences with more than a.few
  bool mine = false;
  for (int b = 0; b < a.v.kv.n_seq; ++b) {
    const int r0 = __builtin_amdgcn_readlane(w.r0, b), n = __builtin_amdgcn_readlane(w.n, b);
    mine |= n > a.few && row >= r0 && row < (long)r0 + n;
  }
  if (!mine) return;
  float top = -INFINITY;
  for (int c = 0; c < splits; ++c) top = fmaxf(top, a.pm2[(size_t)c * a.rows * a.nq + id]);
  top = top == -INFINITY ? 0.f : top;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
  for (int c = 0; c < splits; ++c) {
    const size_t part = (size_t)c * a.rows * a.nq + id;
    const float wt = exp2f(a.pm2[part] - top);
    l += a.pl2[part] * wt;
    o += *(const f32x4 *)(a.po2 + part * D + 4 * q) * wt;
  }
  const float z[4] = {l == 0.f ? 0.f : o[0] / l, l == 0.f ? 0.f : o[1] / l, l == 0.f ? 0.f : o[2] / l, l == 0.f ? 0.f : o[3] / l};
  store_n<bf16_t, 4>((bf16_t *)a.out + (size_t)id * D + 4 * q, z);
  if (q == 0 && a.lse) a.lse[id] = l == 0.f ? -INFINITY : (top + log2f(l)) * LN2;
}

template <typename T, int D, bool Q8>
static void rows_d(const RowsAttend &a, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (a.prompt_segments) {
      RowsAttend p = a;
      p.few = a.segments ? a.few : 0;                      // alone it takes every sequence
      hipLaunchKernelGGL((k_rows_prompt<D, Q8>), dim3(p.prompt_segments, p.splits), dim3(2 * prompt_columns(D)), 0, s, p);
      if (p.splits > 1) {
        const long per = 256 / (D / 4), n = (long)p.rows * p.nq;
        hipLaunchKernelGGL((k_prompt_join<D>), dim3((n + per - 1) / per), dim3(256), 0, s, p, p.splits);
      }
    }
  }
  if (!a.segments) return;
  constexpr int NW = D * sizeof(T) > 512 ? 2 : 4;      // 64 KB of LDS
  const dim3 g(a.waves);
  const bool wide = a.cols == 32;
  if constexpr (sizeof(T) == 2 && D <= 128) {
    if (wide && a.direct) hipLaunchKernelGGL((k_rows_attend<T, D, Q8, 2, NW>), g, dim3(64 * NW), 0, s, a);
    else if (wide) hipLaunchKernelGGL((k_rows_attend<T, D, Q8, 2, 1>), g, dim3(64), 0, s, a);
  }
  if (!wide && a.direct) hipLaunchKernelGGL((k_rows_attend<T, D, Q8, 1, NW>), g, dim3(64 * NW), 0, s, a);
  else if (!wide) hipLaunchKernelGGL((k_rows_attend<T, D, Q8, 1, 1>), g, dim3(64), 0, s, a);
  if (a.direct) return;
  // partials of a segment on average: few, and a wave adds a column's
  const bool few = a.waves / a.segments <= 16;
  const long columns = (long)a.segments * rows_per_tile(a.g, a.cols) * a.g;
  if (few) hipLaunchKernelGGL((k_rows_join<T, D, 64>), dim3((columns + 3) / 4), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_rows_join<T, D, 256>), dim3(columns), dim3(256), 0, s, a);
}
template <typename T, bool Q8>
static void rows_t(const RowsAttend &a, hipStream_t s) {
  if (a.d == 32) rows_d<T, 32, Q8>(a, s);
  else if (a.d == 64) rows_d<T, 64, Q8>(a, s);
  else if (a.d == 128) rows_d<T, 128, Q8>(a, s);
  else rows_d<T, 256, Q8>(a, s);
}
void launch_rows_attend(bool bf16, const RowsAttend &a, hipStream_t s) {
  if (bf16) {
    if (a.scales) rows_t<bf16_t, true>(a, s);
    else rows_t<bf16_t, false>(a, s);
  } else {
    if (a.scales) rows_t<float, true>(a, s);
    else rows_t<float, false>(a, s);
  }
}

}  // namespace prism
