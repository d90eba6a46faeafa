// Microscaled 4-bit floating point on the device: conversions shared by the
// producers of codes (mx4.hip, resid_norm.hip).
//
// A block of 32 channels has the step 2^s, s = floor(log2 max|y|) - 2 clamped to
// [-127, 127], held as the byte s + 127; its codes are y / 2^s rounded to the
// nearest e2m1 value (ties to the even code, past 6: 6).  A block with an
// infinity or a NaN has byte 255 and codes 0.
//
// Eight channels of a row (16 bytes in, 4 bytes of codes out) are a thread's
// piece, so a block is a quad of lanes and its maximum two DPP exchanges.
//
// Codes are those of the formula in 64 bits: a producer either computes in
// double (whose adds and multiplies run at the rate of float ones here), or in
// float with a bound on its error, and repeats in double what lies within it of
// a border between two codes.
#pragma once
#include "common.h"

namespace oq {
namespace {

typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), CTRL, 0xF, 0xF, true));
}
constexpr int kQuadXor1 = 0xB1, kQuadXor2 = 0x4E;  // quad_perm [1, 0, 3, 2] and [2, 3, 0, 1]

__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, dpp<kQuadXor1>(x));
  return max(x, dpp<kQuadXor2>(x));
}

// 2^s for the byte s + 127 (0 is the subnormal 2^-127).
__device__ __forceinline__ float step_of(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }

// The byte of a block whose largest magnitude has the float exponent field `field` (0 .. 254).
__device__ __forceinline__ uint32_t step_byte(uint32_t field) { return field < 2 ? 0u : field - 2; }

// Codes of eight floats at 2^s, channel 0 in the low nibble.
__device__ __forceinline__ uint32_t codes8(const float (&v)[8], float step) {
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], step, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], step, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], step, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], step, 3);
}

// |v| as the high word of a double, its last bit set where the low word is not
// 0: what decides a rounding to one or two bits is kept.
__device__ __forceinline__ uint32_t high_word(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  return (static_cast<uint32_t>(b >> 32) & 0x7FFFFFFFu) | min(static_cast<uint32_t>(b), 1u);
}

// The byte of a block whose largest high word is `top`; 255: not finite.
__device__ __forceinline__ uint32_t step_byte64(uint32_t top) {
  const int field = static_cast<int>(top >> 20);           // exponent + 1023
  if (field == 2047) return 255u;
  return static_cast<uint32_t>(min(max(field - 1023 - 2 + 127, 0), 254));
}

// v / 2^s as a float that rounds to the same code (below 2^-126: 0).
__device__ __forceinline__ float ratio64(double v, uint32_t byte) {
  const int bias = (896 + static_cast<int>(byte) - 127) << 20;
  const uint32_t t = static_cast<uint32_t>(max(static_cast<int>(high_word(v)) - bias, 0)) ;
  const uint32_t sign = static_cast<uint32_t>(__builtin_bit_cast(uint64_t, v) >> 32) & 0x80000000u;
  // (A ratio past the largest float, of a step clamped at 2^127, is that float.)
  return __uint_as_float((t > 0x0FEFFFFFu ? 0x7F7FFFFFu : t << 3) | sign);
}

// Codes of eight doubles of a block whose byte is given.
__device__ __forceinline__ uint32_t codes8(const double (&v)[8], uint32_t byte) {
  if (byte == 255) return 0;
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = ratio64(v[e], byte);
  return codes8(r, 1.0f);
}

// Codes and byte of a quad's block of doubles.
__device__ __forceinline__ uint32_t quad_codes(const double (&v)[8], uint32_t* byte) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, high_word(v[e]));
  *byte = step_byte64(quad_max(top));
  return codes8(v, *byte);
}

// Element e of eight 16-bit values.
template <bool BF>
__device__ __forceinline__ float half8(const uint4& q, int e) {
  const uint32_t w = e < 2 ? q.x : e < 4 ? q.y : e < 6 ? q.z : q.w;
  const uint16_t h = static_cast<uint16_t>(e & 1 ? w >> 16 : w);
  if constexpr (BF) return __uint_as_float(static_cast<uint32_t>(h) << 16);
  else return static_cast<float>(__builtin_bit_cast(_Float16, h));
}

// (Round to nearest even; a NaN stays one.)
template <bool BF>
__device__ __forceinline__ uint16_t to_half(float f) {
  if constexpr (BF) return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f));
  else return __builtin_bit_cast(uint16_t, static_cast<_Float16>(f));
}
template <bool BF>
__device__ __forceinline__ uint4 pack_half8(const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = to_half<BF>(v[2 * e]) | static_cast<uint32_t>(to_half<BF>(v[2 * e + 1])) << 16;
  return make_uint4(w[0], w[1], w[2], w[3]);
}

}  // namespace

// Bytes from one row's steps to the next.
inline int64_t mx4_step_bytes(int64_t K) { return 16 * ((K + 511) / 512); }

}  // namespace oq
