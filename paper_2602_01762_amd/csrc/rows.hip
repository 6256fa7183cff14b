// Attention of several rows per sequence over the paged draft cache, in the
// context's type or in 8 bits: the tokens of a decoding step, drafts to be
// scored, prompts.  Row i of a sequence sees the slots below v = L + n_new + i;
// with a window W those from v - W on and the first n_first.
//
// The rows of a sequence are cut into tiles whose (row, head) pairs of one KV head
// are the 16 columns of a matrix-core tile.  A segment is a tile of one KV head;
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
  const int rt = rows_per_tile(a.g);
  w.tiles = (w.n + rt - 1) / rt;
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
  const int rt = rows_per_tile(a.g);
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
  __device__ static void put(char *tile, int s, int li, u32x4 x, float scale) {
    using M = Tile<T, D>;
    if constexpr (!Q8) {
      *(u32x4 *)(tile + M::at(s, li)) = x;
    } else if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 y;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          y[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x[2 * h + i], scale, false));
          y[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x[2 * h + i], scale, true));
        }
        *(u32x4 *)(tile + M::at(s, 2 * li + h)) = y;
      }
    } else {
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)x[h], scale, false);
        const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)x[h], scale, true);
        *(f32x4 *)(tile + M::at(s, 4 * li + h)) = f32x4{lo[0], lo[1], hi[0], hi[1]};
      }
    }
  }
};
template <typename T>
__device__ __forceinline__ float lds_value(const char *p) {
  if constexpr (sizeof(T) == 2) return bf2f(*(const uint16_t *)p);
  else return *(const float *)p;
}

// A wave takes tiles of TS places, as in the attention of one row per sequence
// (cache.hip): rows loaded whole, into operand order through LDS, scores as MFMAs of
// 16 places x 16 columns, outputs as MFMAs of 16 dims x 16 columns, each lane
// holding one column's softmax state.  A column is a (row, head) pair, so a tile's
// rows share what is loaded; where not every row sees every place of a tile, the
// scores are masked place by place.
//   A value that is not finite must not meet a probability of 0 of a column that
// does not see it; tiles that hold one and are masked take their outputs on the
// vector units.
template <typename T, int D, bool Q8, int NW>
__global__ __launch_bounds__(64 * NW, D * sizeof(T) > 512 ? 1 : 2) void k_rows_attend(RowsAttend a) {
  using M = Tile<T, D>;
  static_assert(M::LPR * 16 >= 64, "a row of 16 probabilities fits a row of the K tile");
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
  const int rt = rows_per_tile(g), columns = rt * g, crow = col / g, chead = col - crow * g;
  int u = blockIdx.x * wk.per;
  const int last = min(wk.total, u + wk.per);
  while (u < last) {
    const RowSegment sg = row_segment_at(a, wk, u, last);
    u += sg.granules;
    const bool used = col < columns && crow < sg.rows;
    const size_t hi = (size_t)(sg.r + crow) * a.nq + sg.j * g + chead;   // this column's row of q and out (used)
    // what this column sees: slots below vis, from win on or below n_first
    const int vis = used ? visible_of(sg.v0, sg.i0 + crow, a.v.max_len) : 0;
    const int win = a.window ? vis - a.window : 0;
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
    auto load = [&](uint32_t row) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const uint32_t r = __shfl(row, i * RPI + grp, 64);
        const size_t at = (size_t)(r == NO_ROW ? 0 : r) * (D * Ld::SZ) + 16 * li;   // a masked place reads row 0
        kr[i] = *(const u32x4 *)((const char *)kv.k_pool + at);
        vr[i] = *(const u32x4 *)((const char *)kv.v_pool + at);
      }
    };
    float m_run = -INFINITY, l_run = 0.f;
    f32x4 o[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    u32x4 qf[NK];
#pragma unroll
    for (int kk = 0; kk < NK; ++kk)
      qf[kk] = used ? *(const u32x4 *)((const T *)a.q + hi * D + (4 * kk + q4) * E) : u32x4{0, 0, 0, 0};
    constexpr int STEP = NW * TS;
    const int t0 = sg.p0 + wave * TS;
    int c1 = 0, b1 = 0;
    Row row{NO_ROW, 1.f, 1.f};
    if (t0 < sg.p1) {
      const int c0 = column(t0 + lane);
      const int b0 = block(c0);
      c1 = column(t0 + STEP + lane);
      b1 = block(c1);
      if (lane < TS) row = row_of(t0 + lane, c0, b0);
      load(row.row);
    }
    for (int t = t0; t < sg.p1; t += STEP) {
      const uint64_t mask = __ballot(row.row != NO_ROW);
      constexpr uint64_t FULL = TS == 64 ? ~0ull : (1ull << (TS & 63)) - 1;
      if (mask != FULL) {
#pragma unroll
        for (int i = 0; i < NI; ++i)
          if (!((mask >> (i * RPI + grp)) & 1)) vr[i] = u32x4{0, 0, 0, 0};
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
        Ld::put(s_k, s, li, kr[i], Q8 ? __shfl(row.ks, s, 64) : 1.f);
        Ld::put(s_v, s, li, vr[i], Q8 ? __shfl(row.vs, s, 64) : 1.f);
      }
      if (t + STEP < sg.p1) {
        row = Row{NO_ROW, 1.f, 1.f};
        if (lane < TS) row = row_of(t + STEP + lane, c1, b1);
        c1 = column(t + 2 * STEP + lane);
        b1 = block(c1);
        load(row.row);
      }
      wave_lds_sync();
      // scores S[place 16 st + 4 q4 + i][column col]
      f32x4 sc[NS];
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        sc[st] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < NK; ++kk)
          sc[st] = Ty<T>::mma(*(const u32x4 *)(s_k + M::at(16 * st + col, 4 * kk + q4)), qf[kk], sc[st]);
      }
      uint32_t sees = 0;                                   // bit 4 st + i: this column sees that place
      float mx = -INFINITY;
#pragma unroll
      for (int st = 0; st < NS; ++st)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int p = 16 * st + 4 * q4 + i;
          bool see = (mask >> p) & 1;
          if (!whole) {
            const int slot = slot_of(t + p);
            see &= slot < vis && (slot >= win || slot < a.n_first);
          }
          sees |= (uint32_t)see << (4 * st + i);
          sc[st][i] = see ? sc[st][i] * a.scale : -INFINITY;
          mx = fmaxf(mx, sc[st][i]);
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
      // O[dim 16 dt + 4 q4 + i][column col]
      if (odd) {
        // the probabilities by way of the K tile, whose scores are done; -1: not seen
        float *ps = (float *)s_k;
        wave_lds_sync();
#pragma unroll
        for (int st = 0; st < NS; ++st)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            ps[(16 * st + 4 * q4 + i) * 16 + col] = (sees >> (4 * st + i)) & 1 ? sc[st][i] : -1.f;
        wave_lds_sync();
#pragma unroll 1
        for (int p = 0; p < TS; ++p) {
          const float w = ps[p * 16 + col];
#pragma unroll
          for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int dim = 16 * dt + 4 * q4 + e;
              const float v = lds_value<T>(s_v + M::at(p, dim / E) + dim % E * sizeof(T));
              o[dt][e] += w < 0.f ? 0.f : w * v;
            }
        }
        wave_lds_sync();
        continue;
      }
      constexpr int NP = sizeof(T) == 2 && NS > 1 ? 2 : 1;
#pragma unroll
      for (int st = 0; st < NS; st += NP) {
        if constexpr (sizeof(T) == 2) {
          uint32_t hi3[NP][2], mid[NP][2], lo[NP][2];
#pragma unroll
          for (int x = 0; x < NP; ++x) split_bf16(sc[st + x], hi3[x], mid[x], lo[x]);
#pragma unroll
          for (int dt = 0; dt < ND; ++dt) {
            uint2 v[NP];
#pragma unroll
            for (int x = 0; x < NP; ++x) {
              const char *pv = s_v + M::at(16 * (st + x) + 4 * q4 + (col >> 2), 2 * dt + ((col & 3) >> 1)) + 8 * (col & 1);
              v[x] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)pv));
            }
            if constexpr (NP == 2) {
              const u32x4 vv = {v[0].x, v[0].y, v[1].x, v[1].y};
              o[dt] = Ty<T>::mma(vv, u32x4{hi3[0][0], hi3[0][1], hi3[1][0], hi3[1][1]}, o[dt]);
              o[dt] = Ty<T>::mma(vv, u32x4{mid[0][0], mid[0][1], mid[1][0], mid[1][1]}, o[dt]);
              o[dt] = Ty<T>::mma(vv, u32x4{lo[0][0], lo[0][1], lo[1][0], lo[1][1]}, o[dt]);
            } else {
              const s16x4 vv = __builtin_bit_cast(s16x4, v[0]);
              o[dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vv, __builtin_bit_cast(s16x4, uint2{hi3[0][0], hi3[0][1]}), o[dt], 0, 0, 0);
              o[dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vv, __builtin_bit_cast(s16x4, uint2{mid[0][0], mid[0][1]}), o[dt], 0, 0, 0);
              o[dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vv, __builtin_bit_cast(s16x4, uint2{lo[0][0], lo[0][1]}), o[dt], 0, 0, 0);
            }
          }
        } else {
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
    if constexpr (NW > 1) {
      __shared__ float s_m[NW][16], s_l[NW][16];
      float *so = (float *)s_k;                        // this wave's outputs [16][D]: within its K and V tiles
      static_assert(2 * TILE >= 16 * D * (int)sizeof(float), "outputs of a wave fit its tiles");
      if (used) {
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) *(f32x4 *)(so + col * D + 16 * dt + 4 * q4) = o[dt];
      }
      if (q4 == 0) {
        s_m[wave][col] = m_run;
        s_l[wave][col] = l_run;
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
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const float z[4] = {y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv};
        const size_t at = (size_t)(sg.r + c / g) * a.nq + sg.j * g + c % g;
        store_n<T, 4>((T *)a.out + at * D + 4 * (e % (D / 4)), z);
        if (a.lse && e % (D / 4) == 0) a.lse[at] = l == 0.f ? -INFINITY : (M2 + log2f(l)) * LN2;
      }
      return;                                          // one segment per workgroup
    }
    if (!used) continue;
    const size_t part = (size_t)cache_partial(blockIdx.x, sg.index) * columns + col;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) *(f32x4 *)(a.po + part * D + 16 * dt + 4 * q4) = o[dt];
    if (q4 == 0) {
      a.pm[part] = m_run;
      a.pl[part] = l_run;
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
  const int rt = rows_per_tile(a.g), columns = rt * a.g;
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

template <typename T, int D, bool Q8>
static void rows_d(const RowsAttend &a, hipStream_t s) {
  constexpr int NW = D * sizeof(T) > 512 ? 2 : 4;      // 64 KB of LDS
  const dim3 g(a.waves);
  if (a.direct) {
    hipLaunchKernelGGL((k_rows_attend<T, D, Q8, NW>), g, dim3(64 * NW), 0, s, a);
    return;
  }
  hipLaunchKernelGGL((k_rows_attend<T, D, Q8, 1>), g, dim3(64), 0, s, a);
  // partials of a segment on average: few, and a wave adds a column's
  const bool few = a.waves / a.segments <= 16;
  const long columns = (long)a.segments * rows_per_tile(a.g) * a.g;
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
