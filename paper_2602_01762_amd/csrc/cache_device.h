// Device code that the kernels over the paged draft cache share: slots and pool
// rows, loads and stores of rows, tiles of rows in LDS.
#pragma once
#include "cache.h"
#include "device.h"

namespace prism {

constexpr float LN2 = 0.6931471805599453f;
constexpr uint32_t NO_ROW = 0xffffffffu;   // a slot without storage

// Slots of sequence b that a call sees: its context plus n_new, at most
// max_len.  With a negative context it sees none; a longer one is cut.  Both flag.
__device__ __forceinline__ int visible_slots(const CacheView &v, int b, uint32_t *err) {
  const int L = v.kv.ctx_lens[b];
  const long n = (long)L + v.n_new;
  if (L < 0 || n > v.max_len) {
    atomicOr(err, ERRF_CAPACITY);
    return L < 0 ? 0 : v.max_len;
  }
  return (int)n;
}
// Pool block and KV head of table column bi of sequence b, as block * heads + j.
__device__ __forceinline__ uint32_t pool_block(const CacheView &v, const int32_t *table, int b, int j, int bi,
                                               uint32_t *err) {
  const int blk = bi < v.kv.mbps ? table[(size_t)b * v.kv.mbps + bi] : -1;
  if (blk < 0 || blk >= v.kv.n_blocks) {
    atomicOr(err, ERRF_CAPACITY);
    return NO_ROW;
  }
  return (uint32_t)blk * v.nkv + j;
}
// Pool row of slot s of that block.
__device__ __forceinline__ uint32_t pool_row(const CacheView &v, const int32_t *table, int b, int j,
                                             int bi, int s, uint32_t *err) {
  const uint32_t blk = pool_block(v, table, b, j, bi, err);
  return blk == NO_ROW ? NO_ROW : blk * v.kv.bs + s;
}

// 16 bytes that the call reads once: a nontemporal load.  Read rates of a plain
// streaming kernel over 4.3 GB: 6.3 TB/s, with nontemporal loads 7.1.
__device__ __forceinline__ u32x4 stream16(const void *p) { return __builtin_nontemporal_load((const u32x4 *)p); }
// N values of a row (N * sizeof(T) a multiple of 4)
template <typename T, int N>
__device__ __forceinline__ void store_n(T *p, const float *x) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < N; i += 2) ((uint32_t *)p)[i / 2] = f2bf(x[i]) | (f2bf(x[i + 1]) << 16);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = x[i];
  }
}
// 8 values of a row <-> fp32
template <typename T>
__device__ __forceinline__ void load8f(const T *p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const u32x4 r = *(const u32x4 *)p;
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else {
    const f32x4 a = *(const f32x4 *)p, b = *(const f32x4 *)(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = a[i];
      x[4 + i] = b[i];
    }
  }
}
// the same from the 16-byte pieces of 8 values
template <typename T>
__device__ __forceinline__ void unpack8(const u32x4 (&p)[sizeof(T) / 2], float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      x[2 * i] = __uint_as_float(p[0][i] << 16);
      x[2 * i + 1] = __uint_as_float(p[0][i] & 0xffff0000u);
    } else {
      x[i] = __uint_as_float(p[0][i]);
      x[4 + i] = __uint_as_float(p[sizeof(T) / 2 - 1][i]);
    }
  }
}
template <typename T>
__device__ __forceinline__ void store8f(T *p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = f2bf(x[2 * i]) | (f2bf(x[2 * i + 1]) << 16);
    *(u32x4 *)p = r;
  } else {
    *(f32x4 *)p = f32x4{x[0], x[1], x[2], x[3]};
    *(f32x4 *)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
  }
}

// Inclusive sum over the lanes below, in a wave (DPP: within rows of 16
// lanes, then the last lane of a row to the next row, then of the first half
// to the second).
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, true);    // row_shr:1
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, true);    // row_shr:2
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, true);    // row_shr:4
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, true);    // row_shr:8
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false);   // row_bcast:15
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false);   // row_bcast:31
  return v;
}
typedef short s16x4 __attribute__((ext_vector_type(4)));
// The upper halves of two fp32: their bf16 values cut off.
__device__ __forceinline__ uint32_t pack_upper(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
// Four probabilities as hi + mid + lo, each the next 8 bits of the value, cut
// off: no part is negative, and a part is 0 only where p is (what would be 0 is
// 2^-126, below every rounding of a sum), so that an infinite value times the
// parts is that infinity and no NaN.
__device__ __forceinline__ void split_bf16(const f32x4 &p, uint32_t (&hi)[2], uint32_t (&mid)[2], uint32_t (&lo)[2]) {
  float m[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float least = fminf(p[i], 0x1p-126f);
    const float r = p[i] - __uint_as_float(__float_as_uint(p[i]) & 0xffff0000u);
    m[i] = fmaxf(r, least);
    l[i] = fmaxf(r - __uint_as_float(__float_as_uint(m[i]) & 0xffff0000u), least);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    hi[i] = pack_upper(p[2 * i], p[2 * i + 1]);
    mid[i] = pack_upper(m[2 * i], m[2 * i + 1]);
    lo[i] = pack_upper(l[2 * i], l[2 * i + 1]);
  }
}

template <typename T, int D>
struct Tile {
  static constexpr int LPR = D * (int)sizeof(T) / 16, RPI = 64 / LPR;   // lanes (pieces) per row, rows per load
  static constexpr int TS = LPR >= 32 ? 16 : LPR >= 16 ? 32 : 64;       // places per tile
  static constexpr int NI = TS / RPI;
  __device__ static int swz(int s) {
    return LPR >= 16 ? s & 15 : LPR == 8 ? (s >> 1) & 7 : (s >> 2) & 3;
  }
  // byte of 16-byte piece c of row s
  __device__ static int at(int s, int c) { return (s * LPR + (c ^ swz(s))) * 16; }
};

}  // namespace prism
