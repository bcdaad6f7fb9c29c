// Rows of layer values in 8-bit integers, as the int8 products read them (the
// definition is in quant.hip).
#pragma once

#include "common.hpp"
#include "validate.hpp"

namespace moe {

// Bytes between quantised rows of n values: whole 16-byte vectors, the bytes
// behind the values zero, so that products may contract over the whole width.
inline int quantized_width(int n) { return (n + 15) / 16 * 16; }

// Quantises rows of n values (x, ldx elements apart) to q (quantized_width(n)
// apart) and scale.  offsets, region_rows (with E regions): only the rows
// [offsets[e], offsets[e] + region_rows[e]) below rows; the others keep what
// they held.
moe_status quantize_launch(hipStream_t s, moe_dtype dt, int64_t rows, int n, const void* x,
                           int64_t ldx, int8_t* q, float* scale, int E, const int32_t* offsets,
                           const int32_t* region_rows);

// ---- device ---------------------------------------------------------------------
namespace {

template <typename T> struct Unit;   // 8 values
template <> struct Unit<uint16_t> {
  uint4 v;
  __device__ __forceinline__ void load(const uint16_t* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float* f) const { unpack8(v, f); }
  __device__ __forceinline__ void set(const float* f) { v = pack8(f); }   // rounds
  __device__ __forceinline__ void store(uint16_t* p) const { *reinterpret_cast<uint4*>(p) = v; }
};
template <> struct Unit<float> {
  uint4 lo, hi;
  __device__ __forceinline__ void load(const float* p) {
    lo = reinterpret_cast<const uint4*>(p)[0];
    hi = reinterpret_cast<const uint4*>(p)[1];
  }
  __device__ __forceinline__ void get(float* f) const {
    Elem<float>::load(lo, f);
    Elem<float>::load(hi, f + 4);
  }
  __device__ __forceinline__ void set(const float* f) {
    lo = Elem<float>::store(f);
    hi = Elem<float>::store(f + 4);
  }
  __device__ __forceinline__ void store(float* p) const {
    reinterpret_cast<uint4*>(p)[0] = lo;
    reinterpret_cast<uint4*>(p)[1] = hi;
  }
};

// Largest |value| of a unit as bits: NaNs order above infinity and infinity
// above every number, which a maximum of floats would lose.
__device__ __forceinline__ uint32_t abs_bits_max(const float (&f)[8], uint32_t m) {
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(f[e]) & 0x7FFFFFFFu);
  return m;
}
template <typename T>
__device__ __forceinline__ uint32_t abs_bits_max(const Unit<T>& u, uint32_t m) {
  float f[8];
  u.get(f);
  return abs_bits_max(f, m);
}

// How a row is divided: pre (1, or 2^64 where the row's values are so small
// that 1 / scale would overflow; a power of two, so exact), and the scale,
// half of it and its reciprocal, all times pre.
struct RowScale {
  float pre, s, half, inv;
};
__device__ __forceinline__ RowScale row_scale(uint32_t amax, float& scale) {
  const float a = __uint_as_float(amax);
  scale = a < INFINITY ? a * (1.f / 127.f) : NAN;
  const float pre = a < 0x1p-60f ? 0x1p64f : 1.f;
  const float s = scale * pre;
  const bool none = !(scale > 0.f);
  return {none ? 0.f : pre, none ? 1.f : s, none ? 0.5f : 0.5f * s, none ? 0.f : 1.f / s};
}

// q for eight values.  x times the rounded reciprocal is within 2^-16 of the
// quotient, so its rounding is off by one at the most, and only where the
// quotient lies next to a half.  r = x - q s is exact in fp32 (it is a multiple of
// half the last place of s and at most about s / 2), so comparing it with
// s / 2 settles those cases; they are rare enough to branch on.
__device__ __forceinline__ uint2 quantize8(float (&f)[8], const RowScale& rs) {
  float q[8];
  bool border = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    f[e] = rs.pre != 0.f ? f[e] * rs.pre : 0.f;
    q[e] = __builtin_rintf(f[e] * rs.inv);
    border |= __builtin_fabsf(__builtin_fmaf(-q[e], rs.s, f[e])) >= rs.half;
  }
  if (border) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float r = __builtin_fmaf(-q[e], rs.s, f[e]), a = __builtin_fabsf(r);
      const bool odd = static_cast<int>(q[e]) & 1;
      if (a > rs.half || (a == rs.half && odd)) q[e] += r > 0.f ? 1.f : -1.f;
    }
  }
  uint32_t b[8];
#pragma unroll
  for (int e = 0; e < 8; ++e)
    b[e] = static_cast<uint32_t>(static_cast<int>(fminf(fmaxf(q[e], -127.f), 127.f))) & 255u;
  return make_uint2(b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24,
                    b[4] | b[5] << 8 | b[6] << 16 | b[7] << 24);
}
template <typename T>
__device__ __forceinline__ uint2 quantize8(const Unit<T>& u, const RowScale& rs) {
  float f[8];
  u.get(f);
  return quantize8(f, rs);
}

}  // namespace
}  // namespace moe
