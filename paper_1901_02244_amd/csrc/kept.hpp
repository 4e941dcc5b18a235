// kept.hpp -- the 8-bit form of activations, shared by the kernels that write
// and read it.
//
// A row of d values is cut into groups of 32 neighbouring columns (the last
// may be short).  A group is held as whole numbers q in [-127, 127] and one
// power of two 2^e, the least with max|x| <= 127 * 2^e:  x ~ q * 2^e, off by
// at most 2^e / 2.  A power of two and not max|x|/127: the division, and the
// product that undoes it, are then exact, every q * 2^e is a number of any of
// the three types (8 significant bits), and the matrix cores take it without
// another rounding; it costs at most one bit of the eight.
//   - e is at least -126 (fp16: -24), where q * 2^e is still exact.
//   - In the topmost group exponent (fp32, bf16: 122; fp16: 10) 64 * 2^e is
//     past the type's largest value: q stops at 63 there.
//   - A group that holds an infinity or a NaN stands for 32 NaNs.
// Storage: [rows][dp] bytes of q, dp = d up to a multiple of 32 (zeros in
// the padding), then [rows][dp/32] bytes e + 127 (255: a group of NaNs).
#pragma once
#include "lm.hpp"

namespace cbk {

constexpr int KEPT_GROUP = 32;
__host__ __device__ constexpr int64_t kept_dp(int64_t d) {
  return (d + KEPT_GROUP - 1) / KEPT_GROUP * KEPT_GROUP;
}

template <class T>
__device__ __forceinline__ float to_f32(T v) {
  return (float)v;
}

// 2^e for e in [-126, 127].
__device__ __forceinline__ float pow2(int e) {
  return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
}

// The group byte for the largest |x| of a group (bits of a non-negative
// float; NaN and infinity are the largest of all).
template <class T>
__device__ __forceinline__ int kept_byte(uint32_t most) {
  constexpr int LOW = __is_same(T, _Float16) ? -24 : -126;
  if (most >= 0x7f800000u) return 255;
  // most = 1.m * 2^(E-127) <= 127 * 2^e = 1.984375 * 2^(e+6)
  const int e = (int)(most >> 23) - 127 - 6 + ((most & 0x7fffffu) > 0x7e0000u ? 1 : 0);
  return (e < LOW ? LOW : e) + 127;
}

// Eight values to eight bytes, given their group's byte.
template <class T>
__device__ __forceinline__ uint64_t kept_pack8(const float (&x)[8], int byte) {
  if (byte == 255) return 0;
  constexpr int TOP = __is_same(T, _Float16) ? 10 : 122;
  const float lim = byte == TOP + 127 ? 63.f : 127.f;
  const float inv = pow2(127 - byte);  // byte >= 1
  uint64_t q = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float v = fminf(fmaxf(__builtin_rintf(x[i] * inv), -lim), lim);
    q |= (uint64_t)(uint8_t)(int8_t)(int)v << (8 * i);
  }
  return q;
}

__device__ __forceinline__ float kept_scale(int byte) {
  return byte == 255 ? __builtin_nanf("") : pow2(byte - 127);
}

// The bits of |x| as a whole number that orders like |x| (NaN on top).
__device__ __forceinline__ uint32_t abs_bits(float x) {
  return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu;
}

// Eight neighbouring values of a row, as they lie in memory.  Rows start
// anywhere: global loads and stores of 16 bytes need no more than their
// element's alignment on this card, and a row that is not on 16 bytes costs
// one more cache line a wave, where single elements cost eight loads.
template <class T>
struct Raw8 {
  static constexpr int WORDS = 2 * (int)sizeof(T);
  uint32_t w[WORDS];
  __device__ __forceinline__ float at(int i) const {
    if constexpr (__is_same(T, float)) return __builtin_bit_cast(float, w[i]);
    const uint32_t h = i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
    if constexpr (__is_same(T, _Float16)) return (float)__builtin_bit_cast(_Float16, (uint16_t)h);
    return __builtin_bit_cast(float, i % 2 ? w[i / 2] & 0xffff0000u : h << 16);
  }
};
// WHOLE: d is a multiple of 8, so that no row ends inside an eight; the
// other form's ends cost registers that the larger kernels feel.
template <class T, bool WHOLE>
__device__ __forceinline__ Raw8<T> load_raw8(const T* row, int c, int d) {
  Raw8<T> r;
  if (WHOLE ? c < d : c + 8 <= d) {
    __builtin_memcpy(r.w, row + c, sizeof(r.w));
    return r;
  }
#pragma unroll
  for (int i = 0; i < Raw8<T>::WORDS; ++i) r.w[i] = 0;
  if constexpr (!WHOLE) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < d) {
        if constexpr (sizeof(T) == 4)
          r.w[i] = __builtin_bit_cast(uint32_t, row[c + i]);
        else
          r.w[i / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, row[c + i]) << (i % 2 * 16);
      }
  }
  return r;
}
// The same as floats; zeros past the row's end.
template <class T, bool WHOLE>
__device__ __forceinline__ void load8(const T* row, int c, int d, float (&x)[8]) {
  const Raw8<T> r = load_raw8<T, WHOLE>(row, c, d);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = r.at(i);
}
template <class T, bool WHOLE>
__device__ __forceinline__ void store8(T* row, int c, int d, const float (&x)[8]) {
  T v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (T)x[i];
  if (WHOLE ? c < d : c + 8 <= d) {
    __builtin_memcpy(row + c, v, sizeof(v));
  } else if constexpr (!WHOLE) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < d) row[c + i] = v[i];
  }
}

}  // namespace cbk
