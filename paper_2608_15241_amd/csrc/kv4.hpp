// The 4-bit KV pool: layout of a tile, rounding to 4 bits and back.
//
// Values are 4-bit floats (a sign and a magnitude of 0, 0.5, 1, 1.5, 2, 3, 4 or 6)
// times a power of two shared by 32 neighbouring dims of one token, the formats that
// gfx950 converts by itself: one v_cvt_scalef32_pk_bf16_fp4 makes two scaled bf16
// values, exactly (a magnitude has 2 significant bits), so reading the pool costs
// half a vector instruction a value and no rounding.
//
// A (block, KV head) owns one tile of 17 * D bytes: the codes of K, the codes of V,
// the scales of K, the scales of V. Codes lie in the order in which the 64 lanes of a
// wave hold the operands of the matrix instructions: lane l (k-group l / 16, column
// l % 16) finds its D/8 bytes of K at l * D/8 (token l % 16, D/4 neighbouring dims)
// and its D/8 bytes of V at 8 D + l * D/8 (the 4 tokens of its k-group one after the
// other, D/16 neighbouring dims each).
#pragma once

#include "common.hpp"

namespace localk {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <int D>
struct Kv4 {
  static constexpr int kGroups = D / 32;      // scales of a token
  static constexpr int kLane = D / 8;         // bytes of codes a lane holds of K, and of V
  static constexpr int kTokenV = D / 32;      // of them, bytes of one token of V
  static constexpr int kV = 8 * D;            // byte offsets in a tile
  static constexpr int kKs = 16 * D;
  static constexpr int kVs = 16 * D + D / 2;
  static constexpr int kTile = 17 * D;
  // Scale bytes: of K by (group, token), of V by (token / 4, group, token % 4).
  static __device__ __forceinline__ int k_scale(int group, int tok) {
    return kKs + group * kBlockSize + tok;
  }
  static __device__ __forceinline__ int v_scale(int group, int tok) {
    return kVs + ((tok / 4) * kGroups + group) * 4 + tok % 4;
  }
  // Group of a lane's dims: K by k-group, V by column.
  static __device__ __forceinline__ int k_group(int kgrp) { return kgrp * kGroups / 4; }
  static __device__ __forceinline__ int v_group(int col) { return col * kGroups / 16; }
};

// Scale byte -> 2^(byte - 127) (255, the mark of a group with an infinity or a NaN,
// gives a float whose exponent the conversions read as NaN).
__device__ __forceinline__ float scale4(uint32_t byte) { return __uint_as_float(byte << 23); }

// Byte i of a dword of scales.
template <int I>
__device__ __forceinline__ float scale4_of(uint32_t w) {
  return __uint_as_float((w >> (8 * I) & 0xffu) << 23);
}

// Byte SEL of a dword of codes -> two scaled bf16 values (low = low nibble).
template <int SEL>
__device__ __forceinline__ uint32_t unpack4(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
}

// Scale byte of a group: E = the least with amax <= 6 * 2^E, from amax's exponent and
// whether its mantissa is above 1.5, within [-125, 125]: below, the smallest value
// (0.5 * 2^E) would not be a normal bf16; above, the largest (6 * 2^E) would overflow
// (values beyond it round to it). 255 for an amax that is not finite.
__device__ __forceinline__ uint32_t scale_byte(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = static_cast<int>(u >> 23) - 2 + ((u & 0x007fffffu) > 0x00400000u ? 1 : 0);
  return u >= 0x7f800000u ? 255u : static_cast<uint32_t>(min(max(e, 2), 252));
}

// max(|a|, |b|) of values' bits: NaN (its magnitude bits are the largest) stays.
__device__ __forceinline__ float amax_bits(float m, float x) {
  return __uint_as_float(max(__float_as_uint(m), __float_as_uint(x) & 0x7fffffffu));
}

// Two values -> byte SEL of codes: nearest, ties to the even code, beyond 6 to 6 (what
// the conversion does for every finite value and scale; checked over all of bf16). A
// group without a finite amax has codes 0.
template <int SEL>
__device__ __forceinline__ uint32_t pack4(uint32_t w, float a, float b, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a, b, scale, SEL);
}

// 8 values of one group -> a dword of codes.
__device__ __forceinline__ uint32_t pack4x8(const float (&x)[8], uint32_t byte) {
  const float s = scale4(byte);
  uint32_t w = 0u;
  w = pack4<0>(w, x[0], x[1], s);
  w = pack4<1>(w, x[2], x[3], s);
  w = pack4<2>(w, x[4], x[5], s);
  w = pack4<3>(w, x[6], x[7], s);
  return byte == 255u ? 0u : w;
}

__device__ __forceinline__ float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t w) {
  return __uint_as_float(w & 0xffff0000u);
}

__device__ __forceinline__ void split8(u32x4 v, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = lo_bf16(v[i]);
    x[2 * i + 1] = hi_bf16(v[i]);
  }
}

// Codes of token e (of the lane's 4) of V: D = 128 a dword, D = 64 half of one.
template <int D>
__device__ __forceinline__ uint32_t v_token(const uint32_t (&v)[D / 32], int e) {
  return D == 128 ? v[e % (D / 32)] : v[e / 2] >> (16 * (e % 2));
}

// The lane's dims of one token of V, as bf16 pairs: x[i] = dims 2i, 2i + 1.
template <int D>
__device__ __forceinline__ void unpack_token(uint32_t w, float s, uint32_t (&x)[D / 32]) {
  x[0] = unpack4<0>(w, s);
  x[1] = unpack4<1>(w, s);
  if constexpr (D == 128) {
    x[2] = unpack4<2>(w, s);
    x[3] = unpack4<3>(w, s);
  }
}

// V of a lane's 4 tokens of one block -> per tile t (dim t of the lane's D/16) two
// dwords of token pairs, the A operand of the value product.
template <int D>
__device__ __forceinline__ void unpack_v(const uint32_t (&v)[D / 32], uint32_t vs,
                                         u32x2 (&o)[D / 16]) {
  uint32_t x[4][D / 32];
  unpack_token<D>(v_token<D>(v, 0), scale4_of<0>(vs), x[0]);
  unpack_token<D>(v_token<D>(v, 1), scale4_of<1>(vs), x[1]);
  unpack_token<D>(v_token<D>(v, 2), scale4_of<2>(vs), x[2]);
  unpack_token<D>(v_token<D>(v, 3), scale4_of<3>(vs), x[3]);
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    o[2 * i] = u32x2{__builtin_amdgcn_perm(x[1][i], x[0][i], 0x05040100u),
                     __builtin_amdgcn_perm(x[3][i], x[2][i], 0x05040100u)};
    o[2 * i + 1] = u32x2{__builtin_amdgcn_perm(x[1][i], x[0][i], 0x07060302u),
                         __builtin_amdgcn_perm(x[3][i], x[2][i], 0x07060302u)};
  }
}

// Maximum of a nonnegative float's bits over lanes l ^ mask.
__device__ __forceinline__ float amax_xor(float v, int mask) {
  return amax_bits(v, __shfl_xor(v, mask));
}

// A lane's D/4 dims of one token of K (bf16 pairs; k-group lane / 16) -> codes; returns
// the scale byte of their group.
template <int D>
__device__ __forceinline__ uint32_t round_k(const u32x4 (&kv)[D / 32], uint32_t (&code)[D / 32]) {
  float x[D / 32][8], amax = 0.f;
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    split8(kv[c], x[c]);
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = amax_bits(amax, x[c][i]);
  }
  if constexpr (D == 64) amax = amax_xor(amax, 16);  // the group's other 16 dims
  const uint32_t s = scale_byte(amax);
#pragma unroll
  for (int c = 0; c < D / 32; ++c) code[c] = pack4x8(x[c], s);
  return s;
}

// A lane's D/16 dims of one token of V (bf16 pairs; column lane % 16; D = 64: the first
// two dwords) -> codes (D = 64: the low half); returns the scale byte of their group.
template <int D>
__device__ __forceinline__ uint32_t round_v(u32x4 v, uint32_t& code) {
  float x[8], amax = 0.f;
  split8(v, x);
#pragma unroll
  for (int i = 0; i < D / 16; ++i) amax = amax_bits(amax, x[i]);
  amax = amax_xor(amax, 1);
  amax = amax_xor(amax, 2);
  if constexpr (D == 64) amax = amax_xor(amax, 4);
  const uint32_t s = scale_byte(amax);
  code = pack4x8(x, s);
  return s;
}

// Softmax scale in log2 units, kept positive so that the largest raw score is the
// largest score: a negative scale flips q's signs, a zero one (every visible key then
// weighs the same) clears q.
struct Scale4 {
  float log2;
  uint32_t q_xor, q_and;
};

inline Scale4 scale_of(float sm_scale) {
  const float l = sm_scale * kLog2e;
  if (l == 0.f) return {1.f, 0u, 0u};
  return {l < 0.f ? -l : l, l < 0.f ? 0x80008000u : 0u, 0xffffffffu};
}

// Bytes of the pool that an alignment check asks for: lanes read 16 bytes.
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace
}  // namespace localk
