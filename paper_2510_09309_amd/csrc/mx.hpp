// The cache in 4 bits: a group of 32 neighbours along the head dimension has one power of two 2^e (byte e + 127) and a code of
// four bits each, sign and one of the sizes 0, 0.5, 1, 1.5, 2, 3, 4, 6.
//
// gfx950 converts two elements an instruction, both ways, with the scale as an fp32 of which the exponent counts: over every code, scale
// byte, bf16 and four million fp32 values the instructions give the nearest size times 2^e with ties to the even code, what is
// beyond the largest size as that, and NaN for the scale byte 255.
#pragma once

#include "kernels.hpp"

namespace maskkv {

typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

constexpr int kMxGroup = 32;

// A launch has fewer than 2^32 threads along a dimension; a workgroup for every few rows of a cache may be more: those beyond
// 2^20 go on along the second dimension, and the last ones may lie behind the last row.
constexpr int kGridBits = 20;
inline dim3 grid_of(int64_t groups) {
  return groups <= 1 << kGridBits ? dim3((unsigned)groups) : dim3(1u << kGridBits, (unsigned)((groups + (1 << kGridBits) - 1) >> kGridBits));
}
__device__ __forceinline__ uint32_t group_number() { return blockIdx.x + (blockIdx.y << kGridBits); }
constexpr uint32_t kMxLeast = 3, kMxMost = 252, kMxNan = 255;

// The scale byte of a group from the largest of its elements' magnitudes (their bits as fp32): the smallest 2^e with most <= 6 * 2^e.
// 6 * 2^e has the mantissa 1.5 and an exponent of e + 2: a mantissa above 1.5 carries into the next one.  Below 2^-124 even the smallest size
// would be no normal bf16, and above 2^125 the largest none at all.
__device__ __forceinline__ uint32_t mx_scale(uint32_t most) {
  if (most >= 0x7F800000u) return kMxNan;
  const uint32_t up = (most + 0x003FFFFFu) >> 23;
  return min(max(up, kMxLeast + 2) - 2, kMxMost);
}

__device__ __forceinline__ float mx_unit(uint32_t scale) { return as_f32(scale << 23); }

// Eight (four) codes of a lane's 16 bytes of bf16 (fp32).  (A group of NaN has codes of 0.)
template <typename T>
__device__ __forceinline__ uint32_t mx_encode(const u32x4& x, uint32_t scale);
template <>
__device__ __forceinline__ uint32_t mx_encode<bf16_t>(const u32x4& x, uint32_t scale) {
  const float unit = mx_unit(scale);
  const uint32_t w0 = x[0], w1 = x[1], w2 = x[2], w3 = x[3];
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w0), unit, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w1), unit, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w2), unit, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w3), unit, 3);
  return scale == kMxNan ? 0u : c;
}
template <>
__device__ __forceinline__ uint32_t mx_encode<float>(const u32x4& x, uint32_t scale) {
  const float unit = mx_unit(scale);
  const uint32_t w0 = x[0], w1 = x[1], w2 = x[2], w3 = x[3];
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, as_f32(w0), as_f32(w1), unit, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, as_f32(w2), as_f32(w3), unit, 1);
  return scale == kMxNan ? 0u : c;
}

// The values of eight codes: as four words of bf16, or as floats.
__device__ __forceinline__ u32x4 mx_decode_bf16(uint32_t codes, float unit) {
  u32x4 x;
  x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 0));
  x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 1));
  x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 2));
  x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 3));
  return x;
}
__device__ __forceinline__ void mx_decode_f32(uint32_t codes, float unit, float (&x)[8]) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 1),
              c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 3);
  x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1], x[4] = c[0], x[5] = c[1], x[6] = d[0], x[7] = d[1];
}

// The head that a packed row belongs to, the largest with cu[head] <= row (row < cu[BH]); found by a wave for a row that its lanes
// share, 64 ways at a time.
__device__ __forceinline__ int head_of_row(const int32_t* cu, int BH, int row) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = BH;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64;
    const int probe = min(lo + (lane + 1) * step, hi);
    const int n = __popcll(__ballot(cu[probe] <= row));  // true for a prefix of the lanes
    const int from = n == 0 ? lo : min(lo + n * step, hi);
    hi = n == 64 ? hi : min(lo + (n + 1) * step, hi);
    lo = from;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// The sum of a value over the lanes up to this one (rows of 16 lanes by shifts, then row ends into the rows behind).
template <int CTRL, int ROWS>
__device__ __forceinline__ int plus_dpp(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int wave_prefix(int v) {
  v = plus_dpp<0x111, 0xf>(v);
  v = plus_dpp<0x112, 0xf>(v);
  v = plus_dpp<0x114, 0xf>(v);
  v = plus_dpp<0x118, 0xf>(v);
  v = plus_dpp<0x142, 0xa>(v);
  return plus_dpp<0x143, 0xc>(v);
}

// Rows that are read once: those of an array larger than the memory-side cache come from HBM, and go past the cache.
constexpr int64_t kSideCache = 256 << 20;
template <bool ONCE>
__device__ __forceinline__ u32x4 read_piece(const char* from) {
  const u32x4* p = reinterpret_cast<const u32x4*>(from);
  if constexpr (ONCE)
    return __builtin_nontemporal_load(p);
  else
    return *p;
}

// The head of a unit of work when a head of n cached rows has units_of(n) units, which is its first and how many it has, and where its rows
// lie (behind the last one: bh -1, and all heads' units before `first_unit`).  Found by a wave, which asks for 256 heads at a time and counts 64.
struct UnitHead {
  int bh, first_unit, units;
  int first, rows;
};
template <typename F>
__device__ __forceinline__ UnitHead head_of_unit(const int32_t* cu, int BH, int capacity, int unit, F units_of) {
  constexpr int kSets = 4;
  const int lane = threadIdx.x & 63;
  UnitHead x = {-1, 0, 0, 0, 0};
  int before = 0;
  for (int base = 0; base < BH; base += 64 * kSets) {
    int from[kSets], to[kSets];
#pragma unroll
    for (int i = 0; i < kSets; ++i) {
      const int bh = min(base + i * 64 + lane, BH - 1);
      from[i] = cu[bh];
      to[i] = cu[bh + 1];
    }
#pragma unroll
    for (int i = 0; i < kSets; ++i) {
      if (base + i * 64 >= BH) break;
      const int first = min(from[i], capacity), rows = max(min(to[i], capacity) - first, 0);
      const int own = base + i * 64 + lane < BH ? units_of(rows) : 0;
      const int upto = wave_prefix(own);
      const uint64_t over = __ballot(before + upto > unit);
      if (over) {
        const int at = __builtin_ctzll(over);
        x.units = __builtin_amdgcn_readlane(own, at);
        x.first_unit = before + __builtin_amdgcn_readlane(upto, at) - x.units;
        x.first = __builtin_amdgcn_readlane(first, at);
        x.rows = __builtin_amdgcn_readlane(rows, at);
        x.bh = __builtin_amdgcn_readfirstlane(base + i * 64 + at);
        return x;
      }
      before += __builtin_amdgcn_readlane(upto, 63);
    }
  }
  x.first_unit = before;
  return x;
}

// The sum of units_of(rows) over the heads before one; found by a wave.
template <typename F>
__device__ __forceinline__ int sum_before(const int32_t* cu, int bh, int capacity, F units_of) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int base = 0; base < bh; base += 64) {
    const int i = min(base + lane, bh - 1), first = min(cu[i], capacity), rows = max(min(cu[i + 1], capacity) - first, 0);
    before += __builtin_amdgcn_readlane(wave_prefix(base + lane < bh ? units_of(rows) : 0), 63);
  }
  return before;
}

}  // namespace maskkv
