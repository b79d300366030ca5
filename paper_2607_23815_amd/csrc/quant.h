// A block of the quantised cache, and the conversions between its codes and bf16 (gfx950).
//
// A slab holds the 16 tokens of one (block, kv head): key codes, key scales, value codes, value scales.
// Codes are e4m3 (8 bits) or e2m1 (4 bits), whose largest values are M = 448 and M = 6; the layouts are
// the matrix cores' operands, so that attention takes its codes in 16-byte loads that are contiguous
// across the wave and converts them in registers:
//   key codes   [D * bits / 128 units][16 slots][16 bytes]: lane (slot, grp) of a 16x16x32 product holds
//               dims D / 4 * grp .. of its slot, all in one group of 32 dims, and so under one scale;
//   key scales  [16 slots][D / 32] bytes: the power of two 2^(byte - 127), which the conversion
//               instruction multiplies by (255: NaN);
//   value codes [lane = 16 q + b][D / 16][4]: dim 16 a + b of slots 4 q .. 4 q + 3 is entry a of lane
//               16 q + b; with 32 bytes a lane (8 bits, D = 128) the lanes' first 16 bytes come before
//               their second;
//   value scales [16 slots] float, 4 significant bits: a value is code x scale, exact in bf16, and the
//               scale may as well multiply the weight of the token.
#pragma once

#include "device_utils.h"
#include "wave_utils.h"

namespace pkv {
namespace qnt {

template <int D, int BITS>
struct Slab {
  static constexpr int kCodes = 2 * D * BITS;       // bytes of key codes, and of value codes
  static constexpr int kKeyScales = kCodes;         // offsets
  static constexpr int kValues = kCodes + D / 2;
  static constexpr int kValueScales = kValues + kCodes;
  static constexpr int kBytes = kValueScales + 4 * kBlockSize;
  static constexpr int kLane = D * BITS / 32;       // bytes of a lane's codes: 8, 16 or 32
  static constexpr int kWords = kLane / 4;
  static constexpr float kMost = BITS == 8 ? 448.f : 6.f;
};

constexpr uint32_t kTiny = 27u << 23;       // 2^-100: what stays below it is stored as zeros
constexpr uint32_t kInfinite = 0x7F800000u;

#if __HIP_DEVICE_COMPILE__
template <int kByte>
__device__ __forceinline__ uint32_t two_bf16_of_4(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, kByte));
}
template <int kHalf>
__device__ __forceinline__ uint32_t two_bf16_of_8(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t,
                            __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, kHalf != 0));
}
#else
template <int kByte>
__device__ __forceinline__ uint32_t two_bf16_of_4(uint32_t, float) { return 0u; }
template <int kHalf>
__device__ __forceinline__ uint32_t two_bf16_of_8(uint32_t, float) { return 0u; }
#endif

// Eight codes (two words of 8 bits, one of 4) times a power of two, as bf16.
template <int BITS>
__device__ __forceinline__ u32x4 eight_bf16(const uint32_t* w, float scale) {
  if constexpr (BITS == 4)
    return u32x4{two_bf16_of_4<0>(w[0], scale), two_bf16_of_4<1>(w[0], scale),
                 two_bf16_of_4<2>(w[0], scale), two_bf16_of_4<3>(w[0], scale)};
  else
    return u32x4{two_bf16_of_8<0>(w[0], scale), two_bf16_of_8<1>(w[0], scale),
                 two_bf16_of_8<0>(w[1], scale), two_bf16_of_8<1>(w[1], scale)};
}
// The four slots' codes of a lane's dim 16 kA + b, as bf16.
template <int BITS, int kA>
__device__ __forceinline__ u32x2 four_bf16(const uint32_t* w) {
  if constexpr (BITS == 4)
    return u32x2{two_bf16_of_4<(kA & 1) * 2>(w[kA / 2], 1.f),
                 two_bf16_of_4<(kA & 1) * 2 + 1>(w[kA / 2], 1.f)};
  else
    return u32x2{two_bf16_of_8<0>(w[kA], 1.f), two_bf16_of_8<1>(w[kA], 1.f)};
}

// The four slots' codes of a lane's dim 16 kA + b times the slots' scales, as bf16 (exact).
template <int BITS, int kA>
__device__ __forceinline__ u32x2 four_scaled(const uint32_t* w, const u32x4 scale) {
#if __HIP_DEVICE_COMPILE__
  const float s[4] = {__uint_as_float(scale[0]), __uint_as_float(scale[1]), __uint_as_float(scale[2]),
                      __uint_as_float(scale[3])};
  if constexpr (BITS == 4) {
    const auto x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[kA / 2], 1.f, (kA & 1) * 2);
    const auto y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[kA / 2], 1.f, (kA & 1) * 2 + 1);
    return u32x2{pack_bf16x2(x[0] * s[0], x[1] * s[1]), pack_bf16x2(y[0] * s[2], y[1] * s[3])};
  } else {
    const auto x = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[kA], false);
    const auto y = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[kA], true);
    return u32x2{pack_bf16x2(x[0] * s[0], x[1] * s[1]), pack_bf16x2(y[0] * s[2], y[1] * s[3])};
  }
#else
  return u32x2{0u, 0u};
#endif
}

// Two floats of at most M as codes, to nearest even: 4 bits into byte kPart of `into`, 8 bits into half
// kPart (the others stay).
template <int BITS, int kPart>
__device__ __forceinline__ uint32_t two_codes(uint32_t into, float x, float y) {
#if __HIP_DEVICE_COMPILE__
  if constexpr (BITS == 4)
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(into, x, y, 1.f, kPart);
  else
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, y, (int)into, kPart != 0);
#else
  return into;
#endif
}

// The magnitude bits of two packed bf16 as floats' bits, the larger of them and `top`. (As whole numbers
// they are ordered as the magnitudes are, infinities and NaN above all.)
__device__ __forceinline__ uint32_t top_of(uint32_t pair, uint32_t top) {
  return max(max(pair << 16 & 0x7FFF0000u, pair & 0x7FFF0000u), top);
}

// A key group's scale byte and what its values are multiplied by, from its largest magnitude's bits: the
// least e with top <= M 2^e, M = 1.5 2^2 or 1.75 2^8, is the exponent of top over M's, one more where top's
// fraction is above M's. Never past 2^125 (2^119), so that no code stands for an infinity.
template <int BITS>
__device__ __forceinline__ void key_scale(uint32_t top, uint32_t& byte, float& inverse) {
  constexpr uint32_t kAbove = BITS == 8 ? 0x1FFFFFu : 0x3FFFFFu;
  constexpr uint32_t kMostByte = BITS == 8 ? 119 + 127 : 125 + 127;
  byte = min(((top + kAbove) >> 23) - (BITS == 8 ? 8 : 2), kMostByte);
  inverse = __uint_as_float((254u - byte) << 23);
  if (top < kTiny) byte = 127;
  if (top >= kInfinite) byte = 255;
}
// A token's value scale, the least number of 4 significant bits that is not below top / M (the quotient
// is exact where it is such a number, and 2^-12 of itself away from one otherwise). Never past the largest
// whose M-fold is finite; quotients above M then become M by the conversion (6.4 and 455 at most).
template <int BITS>
__device__ __forceinline__ float value_scale(uint32_t top) {
  const float s = __uint_as_float(top) / Slab<128, BITS>::kMost;
  constexpr float kTop = BITS == 8 ? 0x1.2p119f : 0x1.4p125f;
  const float up = fminf(__uint_as_float((__float_as_uint(s) + 0xFFFFFu) & 0xFFF00000u), kTop);
  return top >= kInfinite ? __uint_as_float(0x7FC00000u) : top < kTiny ? 1.f : up;
}
// x / s for the rounding to a code, from an approximate 1 / s. A border between codes has 5 significant bits,
// s has 4 and x 8, so that a quotient is on a border or 2^-9 of itself away from any; the product is off by
// 2^-21 and finds back to the border when it is rounded to 16 bits.
__device__ __forceinline__ float over_scale(float x, float inverse) {
  return __uint_as_float((__float_as_uint(x * inverse) + 0x80u) & ~0xFFu);
}
__device__ __forceinline__ bool stored(uint32_t top) { return top >= kTiny && top < kInfinite; }
__device__ __forceinline__ float clamp_code(float x, float most) {
  return __builtin_amdgcn_fmed3f(x, -most, most);
}


typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(16))) uint32_t u32x16;
typedef __attribute__((ext_vector_type(32))) __bf16 bf16x32;

// 4-bit keys go into the matrix cores as they are, beside queries in e2m3 (products and sums come out as in
// 32 bits; beside e4m3 they are off by 2^-11 of the largest product).
constexpr int kParts = 3;

// A group of 32 queries (16 words of bf16) in kParts parts of e2m3 and their scale bytes (byte i: part i's). The
// group's largest magnitude is brought to 4 .. 8 by a power of two; a part is the nearest code to what the
// parts before it leave, times 16^i. A code has 4 significant bits above 1 and steps of 1/8 below, so the parts'
// sum is the query if that is at least 2^-6 of the group's largest, and within 2^-14 of the largest otherwise. (Scales
// end at 2^-118: of a group whose largest is below 2^-116 every query is within 2^-130.)
// Where a query is not finite the bytes are 255, which makes the products NaN.
__device__ __forceinline__ uint32_t query_parts(u32x16 x, i32x8 (&part)[kParts]) {
#if __HIP_DEVICE_COMPILE__
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 16; ++e) top = top_of(x[e], top);
  const uint32_t byte = max((int)(top >> 23) - 2, 9);
#pragma unroll
  for (int i = 0; i < kParts; ++i) {
    const float scale = __uint_as_float((byte - 4 * i) << 23);
    const auto code = __builtin_amdgcn_cvt_scalef32_pk32_fp6_bf16(__builtin_bit_cast(bf16x32, x), scale);
#pragma unroll
    for (int e = 0; e < 6; ++e) part[i][e] = (int)code[e];
    part[i][6] = part[i][7] = 0;
    const u32x16 back = __builtin_bit_cast(u32x16, __builtin_amdgcn_cvt_scalef32_pk32_bf16_fp6(code, scale));
#pragma unroll
    for (int e = 0; e < 16; ++e)  // (exact)
      x[e] = pack_bf16x2(__uint_as_float(x[e] << 16) - __uint_as_float(back[e] << 16),
                         __uint_as_float(x[e] & 0xFFFF0000u) - __uint_as_float(back[e] & 0xFFFF0000u));
  }
  return top >= kInfinite ? 0xFFFFFFu : byte | (byte - 4) << 8 | (byte - 8) << 16;
#else
  return 0u;
#endif
}

}  // namespace qnt
}  // namespace pkv
