// The draft cache in 8 bits: rows appended to it, and the cache of the context's
// type written to it and read back.
//
// Values are held as e4m3 codes (1 sign, 4 exponent, 3 fraction bits; subnormals
// down to 2^-9, largest 448, no infinity) over one scale per pool block, KV head
// and pool, 2^e with the least e in -110 .. 119 for which the block's largest
// finite magnitude is at most 448 * 2^e.  With a power of two, value / scale and
// code * scale are exact, so a value is rounded once, to its code; and when later
// rows need a larger scale, the codes that a block holds follow it without
// another rounding, but for those that become subnormal.  (With a scale of
// amax / 448 every larger row would round the whole block again.)  A value that
// is not finite is held as NaN.
#include "cache.h"
#include "cache_device.h"
#include "rotation.h"

namespace prism {

constexpr int E8_MIN = -110, E8_MAX = 119;   // both 2^e and 2^-e are normal fp32, 448 * 2^e finite
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// Least e with amax <= 448 * 2^e.  448 = 1.75 * 2^8: from amax = m * 2^x, 1 <= m <
// 2, that is x - 8, or x - 7 where m > 1.75.  (0 and subnormals: E8_MIN.)
__device__ __forceinline__ int scale_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
  return min(max(e, E8_MIN), E8_MAX);
}
// Exponent of a scale that a block holds.
__device__ __forceinline__ int held_exponent(float scale) {
  return min(max((int)((__float_as_uint(scale) >> 23) & 0xff) - 127, E8_MIN), E8_MAX);
}
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}
// x / 2^e (inv = 2^-e) as the conversion takes it
__device__ __forceinline__ float scaled8(float x, float inv) {
  const float y = fminf(fmaxf(x * inv, -448.f), 448.f);
  return fabsf(x) < INFINITY ? y : NAN;
}
// Codes of four values: rounded to the nearest, ties to the even code.
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float inv) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(scaled8(a, inv), scaled8(b, inv), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(scaled8(c, inv), scaled8(d, inv), r, true);
}
// Four codes times f <= 1 (a power of two), rounded again.
__device__ __forceinline__ uint32_t shrink4(uint32_t c, float f) {
  const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)c, f, false);
  const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)c, f, true);
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0], lo[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(hi[0], hi[1], r, true);
}
// The first n rows of a block of one head, from scale 2^old to 2^e > 2^old: the
// wave's lanes take 16 codes each.  2^-20 already takes every code to 0.
__device__ __forceinline__ void shrink_rows(uint8_t *codes, int n, int d, int old, int e) {
  const float f = pow2f(max(old - e, -20));
  for (int i = threadIdx.x & 63; i < n * d / 16; i += 64) {
    u32x4 c = *(u32x4 *)(codes + 16 * (size_t)i);
#pragma unroll
    for (int k = 0; k < 4; ++k) c[k] = shrink4(c[k], f);
    *(u32x4 *)(codes + 16 * (size_t)i) = c;
  }
}
// fp64 to fp32, cut off, and the last bit set where anything was: a rounding of
// that to fewer bits is the rounding of the fp64 value.  A finite value beyond fp32
// is cut off to its largest one (whose last bit is set), which has the same scale
// and code.
__device__ __forceinline__ float to_odd(double x) {
  const float f = (float)x;
  uint32_t u = __float_as_uint(f);
  if ((double)f == x || x != x) return f;
  if (fabs((double)f) > fabs(x)) --u;        // cut off (f is not 0 then; the one below infinity is the largest)
  return __uint_as_float(u | 1u);
}

// ---------------------------------------------------------------- append
// A workgroup takes the new rows of one cache block, 16 at a time, and a share of
// the heads, a wave a head: the scale of a block needs all its rows.  LPH = d / 16
// lanes hold a head of a row as the rotation pairs it: dims 8i .. 8i+7 and d/2 +
// 8i ...  Keys are normalised and rotated in fp64, as the angles are, so that a key
// next to the border of two codes takes the nearer one; the rounding to fp32 in
// between keeps the side (to_odd).  Queries, which have no such borders, in fp32.  Up to 16 new rows of a block stay in registers
// between the maximum and the codes; of more (larger blocks), the rows are read
// twice.
//   6640 rows of 48 heads, 150 MB: 50 us, 3 TB/s, where a copy takes 31: bound by
// latency, since the fp64 values and the angles' constants take 217 registers, two
// waves to a SIMD.  Four waves to a workgroup (59 us a call, with eight 62); heads
// over workgroups up to APPEND8_FILL of them.
constexpr int APPEND8_ROWS = 16, APPEND8_FILL = 1024;
template <typename T, int D>
__global__ __launch_bounds__(256) void k_cache8_append(Cache8Append a) {
  constexpr int LPH = D / 16, HPW = 64 / LPH, IT = (APPEND8_ROWS + HPW - 1) / HPW;
  const int tid = threadIdx.x, wave = wave_id(), lane = tid & 63, NW = blockDim.x >> 6;
  __shared__ double cs[APPEND8_ROWS][D / 2], sn[APPEND8_ROWS][D / 2];
  __shared__ __attribute__((aligned(16))) float cq[APPEND8_ROWS][D / 2], sq[APPEND8_ROWS][D / 2];   // of the queries
  const KvArgs &kv = a.v.kv;
  const int bs = kv.bs, nkv = a.v.nkv, nh = a.nq + 2 * nkv, B = kv.n_seq;
  // the sequence and the block of this workgroup, from one lane per sequence
  int lo = 0, n = 0;
  if (a.offsets) {
    const int hi = lane < B ? a.offsets[lane + 1] : 0;
    lo = lane < B ? a.offsets[lane] : 0;
    if (__ballot(lane < B && (hi < lo || hi > a.rows || (lane == 0 && lo != 0)))) {
      if (tid == 0 && blockIdx.x == 0) atomicOr(a.err, ERRF_ROWS);
      return;
    }
    n = hi - lo;
  } else if (lane < B) {
    lo = lane;
    n = 1;
  }
  const int len = lane < B ? kv.ctx_lens[lane] : 0;
  // where the rows of a sequence begin in its first block (of a negative length: 0)
  const int in = len > 0 ? slot_in_block(kv, len, slot_block(kv, len)) : 0;
  const int count = n > 0 ? (int)(((long)in + n - 1) / bs) + 1 : 0;
  const uint32_t end = wave_scan((uint32_t)count);
  const int b = __popcll(__ballot(end <= blockIdx.x));
  if (b >= B) return;                              // fewer blocks than the launch allows for
  const int i_blk = blockIdx.x - (int)(__builtin_amdgcn_readlane(end, b) - (uint32_t)__builtin_amdgcn_readlane(count, b));
  const int L = __builtin_amdgcn_readlane(len, b), at0 = __builtin_amdgcn_readlane(in, b);
  const int r_seq = __builtin_amdgcn_readlane(lo, b), n_seq = __builtin_amdgcn_readlane(n, b);
  const int first = i_blk ? i_blk * bs - at0 : 0;            // new rows of the block: first .. first + rows - 1
  const int s0 = i_blk ? 0 : at0, rows = min(n_seq - first, bs - s0);
  const long col = (long)(L > 0 ? slot_block(kv, L) : 0) + i_blk;   // table column
  uint32_t blk = NO_ROW;                                     // block * heads
  if (L < 0 || col >= kv.mbps) {
    if (tid == 0) atomicOr(a.err, ERRF_CAPACITY);
  } else {
    blk = pool_block(a.v, kv.block_table, b, 0, (int)col, a.err);
  }
  const long pos0 = (long)(a.positions ? a.positions[b] : L) + first;
  const bool once = rows <= APPEND8_ROWS;
  const int grp = lane / LPH, li = lane % LPH;
  constexpr int JOBS = 8;                                    // heads of a wave whose maxima are kept at once
  for (int h0 = blockIdx.y * NW + wave; ; h0 += gridDim.y * NW * JOBS) {
    // the same trips for every wave of the workgroup (barriers inside)
    if (h0 - wave >= nh) break;
    float amax[JOBS] = {};
    for (int pass = 0; pass < (once ? 1 : 2); ++pass) {
      for (int c0 = 0; c0 < rows; c0 += APPEND8_ROWS) {
        const int nr = min(rows - c0, APPEND8_ROWS);
        __syncthreads();
        for (int i = tid; i < nr * (D / 2); i += blockDim.x) {
          const int r = i / (D / 2), k = i % (D / 2);
          rotation_cos_sin64((double)(pos0 + c0 + r) * a.inv_freq[k], cs[r][k], sn[r][k]);
          cq[r][k] = (float)cs[r][k];
          sq[r][k] = (float)sn[r][k];
        }
        __syncthreads();
#pragma unroll 1
        for (int job = 0; job < JOBS; ++job) {
          const int h = h0 + job * gridDim.y * NW;
          if (h >= nh) break;
          const bool is_q = h < a.nq, is_v = h >= a.nq + nkv;
          if (is_q && pass) continue;
          if (!is_q && blk == NO_ROW) continue;
          float x[IT][16];
          float top = 0.f;
#pragma unroll
          for (int it = 0; it < IT; ++it) {
            const int r = it * HPW + grp;
            const bool has = r < nr;
            const size_t row = (size_t)r_seq + first + c0 + (has ? r : 0);
            const T *src = (const T *)a.qkv + (row * nh + h) * D + 8 * li;
            float x1[8], x2[8];
            load8f<T>(src, x1);
            load8f<T>(src + D / 2, x2);
            const int rc = has ? r : 0;
            if (is_q) {
              if (a.q_gain) {
                float ss = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) ss += x1[i] * x1[i] + x2[i] * x2[i];
                ss = group_sum(ss, LPH == 2 ? 1 : LPH == 4 ? 2 : LPH == 8 ? 3 : 4);
                const float rs = 1.0f / sqrtf(ss / (float)D + a.eps);
                float g1[8], g2[8];
                load8f<T>((const T *)a.q_gain + 8 * li, g1);
                load8f<T>((const T *)a.q_gain + D / 2 + 8 * li, g2);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                  x1[i] *= rs * g1[i];
                  x2[i] *= rs * g2[i];
                }
              }
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float c = cq[rc][8 * li + i], s = sq[rc][8 * li + i], u = x1[i], w = x2[i];
                x1[i] = u * c - w * s;
                x2[i] = w * c + u * s;
              }
            } else if (!is_v) {
              double y1[8], y2[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                y1[i] = x1[i];
                y2[i] = x2[i];
              }
              if (a.k_gain) {
                double ss = 0.0;
#pragma unroll
                for (int i = 0; i < 8; ++i) ss += y1[i] * y1[i] + y2[i] * y2[i];
#pragma unroll
                for (int m = 1; m < LPH; m *= 2) ss += __shfl_xor(ss, m, 64);
                const double rs = 1.0 / sqrt(ss / D + (double)a.eps);
                float g1[8], g2[8];
                load8f<T>((const T *)a.k_gain + 8 * li, g1);
                load8f<T>((const T *)a.k_gain + D / 2 + 8 * li, g2);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                  y1[i] *= rs * g1[i];
                  y2[i] *= rs * g2[i];
                }
              }
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const double c = cs[rc][8 * li + i], s = sn[rc][8 * li + i];
                x1[i] = to_odd(y1[i] * c - y2[i] * s);
                x2[i] = to_odd(y2[i] * c + y1[i] * s);
              }
            }
            if (is_q) {
              if (has) {
                T *o = (T *)a.q + (row * a.nq + h) * D + 8 * li;
                store8f<T>(o, x1);
                store8f<T>(o + D / 2, x2);
              }
              continue;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              x[it][i] = x1[i];
              x[it][8 + i] = x2[i];
              if (has) top = fmaxf(top, fmaxf(finite_abs(x1[i]), finite_abs(x2[i])));
            }
          }
          if (is_q) continue;
          if (!pass) {
            top = wave_max(top);
#pragma unroll
            for (int k = 0; k < JOBS; ++k) amax[k] = k == job ? fmaxf(amax[k], top) : amax[k];
            if (!once) continue;
          }
          float whole = 0.f;
#pragma unroll
          for (int k = 0; k < JOBS; ++k) whole = k == job ? amax[k] : whole;
          const int j = is_v ? h - a.nq - nkv : h - a.nq;
          uint8_t *codes = (uint8_t *)(is_v ? kv.v_pool : kv.k_pool) + (size_t)(blk + j) * bs * D;
          float *scale = a.scales + 2 * (size_t)(blk + j) + is_v;
          int e = scale_exponent(whole);
          if (s0) {                                          // the block holds rows
            const int old = held_exponent(*scale);
            if (e <= old) e = old;
            else if (c0 + APPEND8_ROWS >= rows) shrink_rows(codes, s0, D, old, e);   // (once, with the last rows)
          }
          const float inv = pow2f(-e);
#pragma unroll
          for (int it = 0; it < IT; ++it) {
            const int r = it * HPW + grp;
            if (r >= nr) continue;
            uint8_t *o = codes + (size_t)(s0 + c0 + r) * D + 8 * li;
            const float(&y)[16] = x[it];
            *(uint2 *)o = uint2{encode4(y[0], y[1], y[2], y[3], inv), encode4(y[4], y[5], y[6], y[7], inv)};
            *(uint2 *)(o + D / 2) = uint2{encode4(y[8], y[9], y[10], y[11], inv), encode4(y[12], y[13], y[14], y[15], inv)};
          }
          if (lane == 0 && c0 + APPEND8_ROWS >= rows) *scale = pow2f(e);
        }
      }
    }
  }
}

template <typename T>
static void append8_d(const Cache8Append &a, int d, hipStream_t s) {
  const int nh = a.nq + 2 * a.v.nkv, bs = a.v.kv.bs, B = a.v.kv.n_seq;
  // blocks that can receive rows: each row one, each sequence ceil((at + n) / bs)
  long blocks = a.rows;
  if (a.offsets) blocks = min(blocks, (long)a.rows / bs + 2 * B);
  const int nw = min(4, nh);
  const int share = (int)max(1l, min((long)(nh + nw - 1) / nw, APPEND8_FILL / max(1l, blocks)));
  const dim3 g(blocks, share), t(64 * nw);
  if (d == 32) hipLaunchKernelGGL((k_cache8_append<T, 32>), g, t, 0, s, a);
  else if (d == 64) hipLaunchKernelGGL((k_cache8_append<T, 64>), g, t, 0, s, a);
  else if (d == 128) hipLaunchKernelGGL((k_cache8_append<T, 128>), g, t, 0, s, a);
  else hipLaunchKernelGGL((k_cache8_append<T, 256>), g, t, 0, s, a);
}
void launch_cache8_append(bool bf16, const Cache8Append &a, int d, hipStream_t s) {
  if (bf16) append8_d<bf16_t>(a, d, s);
  else append8_d<float>(a, d, s);
}

// ---------------------------------------------------------------- pack, unpack
// The slots of table column c of sequence b that a call moves, and its blocks in
// both caches (as block * heads).
struct Moved {
  int from, to;                 // slots in the block (none: from >= to)
  uint32_t blk8, blk;
};
__device__ __forceinline__ Moved moved_slots(const Cache8Move &a, int b, int c) {
  const KvArgs &kv = a.v.kv;
  const int n = visible_slots(a.v, b, a.err);
  int start = a.start ? a.start[b] : 0;
  if (start < 0) {
    atomicOr(a.err, ERRF_ROWS);
    start = n;
  }
  const long s0 = (long)c * kv.bs;
  Moved m{(int)max(0l, min((long)start - s0, (long)kv.bs)), (int)max(0l, min((long)n - s0, (long)kv.bs)), NO_ROW, NO_ROW};
  if (m.from >= m.to) return m;
  m.blk8 = pool_block(a.v, kv.block_table, b, 0, c, a.err);
  CacheView o = a.v;
  o.kv = a.kv;
  m.blk = pool_block(o, a.kv.block_table, b, 0, c, a.err);
  if (m.blk8 == NO_ROW || m.blk == NO_ROW) m.to = m.from;
  return m;
}

// Pack: a wave takes a head's keys or values of one block: 8 values per lane, in
// registers between the maximum and the codes up to KEEP rows, read twice beyond.
// Memory bounds it: 1.0 GB in 208 us, the rate of a copy.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_cache8_pack(Cache8Move a) {
  constexpr int LPR = D / 8, RPI = 64 / LPR, KEEP = 16, IT = (KEEP + RPI - 1) / RPI;
  const int b = blockIdx.y, lane = threadIdx.x & 63, grp = lane / LPR, li = lane % LPR;
  const int nkv = a.v.nkv, bs = a.v.kv.bs;
  const Moved m = moved_slots(a, b, blockIdx.x);
  if (m.from >= m.to) return;
  const bool once = m.to - m.from <= KEEP;
  for (int job = 4 * blockIdx.z + wave_id(); job < 2 * nkv; job += 4 * gridDim.z) {
    const int j = job >> 1, is_v = job & 1;
    const T *src = (const T *)(is_v ? a.kv.v_pool : a.kv.k_pool) + (size_t)(m.blk + j) * bs * D + 8 * li;
    uint8_t *codes = (uint8_t *)(is_v ? a.v.kv.v_pool : a.v.kv.k_pool) + (size_t)(m.blk8 + j) * bs * D;
    float *scale = a.scales + 2 * (size_t)(m.blk8 + j) + is_v;
    const int old = m.from ? held_exponent(*scale) : E8_MIN;
    float top = 0.f;
    float x[IT][8];
    int e = old;
    for (int pass = 0; pass < (once ? 1 : 2); ++pass) {
      for (int r0 = m.from; r0 < m.to; r0 += IT * RPI) {
#pragma unroll
        for (int it = 0; it < IT; ++it) {
          const int r = min(r0 + it * RPI + grp, m.to - 1);
          load8f<T>(src + (size_t)r * D, x[it]);
        }
        if (!pass) {
#pragma unroll
          for (int it = 0; it < IT; ++it)
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, finite_abs(x[it][i]));
          if (!once) continue;
        }
        if (once) e = max(old, scale_exponent(wave_max(top)));
        const float inv = pow2f(-e);
#pragma unroll
        for (int it = 0; it < IT; ++it) {
          const int r = r0 + it * RPI + grp;
          if (r >= m.to) continue;
          const float(&y)[8] = x[it];
          *(uint2 *)(codes + (size_t)r * D + 8 * li) =
              uint2{encode4(y[0], y[1], y[2], y[3], inv), encode4(y[4], y[5], y[6], y[7], inv)};
        }
      }
      if (!once && !pass) e = max(old, scale_exponent(wave_max(top)));
    }
    if (m.from && e > old) shrink_rows(codes, m.from, D, old, e);
    if (lane == 0) *scale = pow2f(e);
  }
}

// Unpack: a share of the heads of a block, which both pools hold in one piece, per
// workgroup; a thread turns as many codes as make 16 bytes, so that loads and stores
// of a wave are one run of memory each (16 codes a thread, whose stores lie 32 bytes
// apart: 950 us for 2.0 GB, so 401, the rate of a copy).
template <typename T, int D>
__global__ __launch_bounds__(256) void k_cache8_unpack(Cache8Move a) {
  constexpr int N = 16 / sizeof(T), LPR = D / N;             // codes of a thread, threads of a row
  const int b = blockIdx.y, nkv = a.v.nkv, bs = a.v.kv.bs;
  const Moved m = moved_slots(a, b, blockIdx.x);
  if (m.from >= m.to) return;
  const int per = (m.to - m.from) * LPR;                     // pieces of a head
  for (int j = blockIdx.z; j < nkv; j += gridDim.z) {
    const float2 sc = *(const float2 *)(a.scales + 2 * (size_t)(m.blk8 + j));
    const size_t from = ((size_t)(m.blk8 + j) * bs + m.from) * D, to = ((size_t)(m.blk + j) * bs + m.from) * D;
    const uint8_t *ck = (const uint8_t *)a.v.kv.k_pool + from, *cv = (const uint8_t *)a.v.kv.v_pool + from;
    T *ok = (T *)a.kv.k_pool + to, *ov = (T *)a.kv.v_pool + to;
    for (int p = threadIdx.x; p < per; p += 256) {
      uint32_t c[2][N / 4];
#pragma unroll
      for (int i = 0; i < N / 4; ++i) {
        c[0][i] = *(const uint32_t *)(ck + (size_t)p * N + 4 * i);
        c[1][i] = *(const uint32_t *)(cv + (size_t)p * N + 4 * i);
      }
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const float f = w ? sc.y : sc.x;
        u32x4 y;
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            y[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c[w][i], f, false));
            y[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c[w][i], f, true));
          }
        } else {
          const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)c[w][0], f, false);
          const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)c[w][0], f, true);
          y = u32x4{__float_as_uint(lo[0]), __float_as_uint(lo[1]), __float_as_uint(hi[0]), __float_as_uint(hi[1])};
        }
        *(u32x4 *)((w ? ov : ok) + (size_t)p * N) = y;
      }
    }
  }
}

// Workgroups over which the heads of few blocks are spread (4096 slots of 32 heads
// packed: 20.5 us, one workgroup per block 33.5; 2048 of 8 unpacked 4.7 and 11.6).
constexpr int MOVE_FILL = 4096;
template <typename T>
static void pack_d(const Cache8Move &a, int d, bool unpack, hipStream_t s) {
  const int columns = (a.v.max_len + a.v.kv.bs - 1) / a.v.kv.bs, nkv = a.v.nkv;
  const long fill = MOVE_FILL / ((long)columns * a.v.kv.n_seq) + 1;
  const dim3 g(columns, a.v.kv.n_seq, (int)min(fill, unpack ? (long)nkv : (nkv + 1l) / 2)), t(256);
#define PRISM_MOVE(D)                                                             \
  if (unpack) hipLaunchKernelGGL((k_cache8_unpack<T, D>), g, t, 0, s, a);         \
  else hipLaunchKernelGGL((k_cache8_pack<T, D>), g, t, 0, s, a)
  if (d == 32) { PRISM_MOVE(32); }
  else if (d == 64) { PRISM_MOVE(64); }
  else if (d == 128) { PRISM_MOVE(128); }
  else { PRISM_MOVE(256); }
#undef PRISM_MOVE
}
void launch_cache8_pack(bool bf16, const Cache8Move &a, int d, hipStream_t s) {
  if (bf16) pack_d<bf16_t>(a, d, false, s);
  else pack_d<float>(a, d, false, s);
}
void launch_cache8_unpack(bool bf16, const Cache8Move &a, int d, hipStream_t s) {
  if (bf16) pack_d<bf16_t>(a, d, true, s);
  else pack_d<float>(a, d, true, s);
}

}  // namespace prism
