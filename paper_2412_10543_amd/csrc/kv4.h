// The 4-bit page (internal): 16 tokens of one kv head in 9 D bytes.
//
// Each group of 64 channels of a token's row has a scale s (bf16) and a zero
// point z in 0..15; code c in 0..15 stands for s (c - z).
//   K codes  u32 [16 tokens][4][D/64][2]: word (i, g, w) holds the channels 64 g +
//            16 i + 8 w + e, e = 0..7: channel e in nibble e/2, + 4 where e is odd.
//            A lane of the matrix product K Q^T (key l % 16, i = l / 16) has its
//            operands in one load, and (word >> 4 p) & 0x000f000f are the two
//            neighbours 2 p and 2 p + 1 of a bf16 register.
//   V codes  u16 [16][16 tokens][D/64]: the unit (i, g) of a token holds the
//            channels 64 g + 4 i + e, e = 0..3, in nibble e.  A lane of V^T P^T
//            (rows i = l % 16, keys 4 (l / 16) ..) has its four keys in one load.
//   params   u32 [D/64][16 tokens] at byte 8 D: the bits of s above those of bf16
//            128 + z (both are floats by one shift or mask; bf16 holds 128 + z and,
//            as 0x4300 | c, 128 + c exactly).
#pragma once

#include "common.h"

namespace rag {

constexpr uint32_t kKv4Ones = 0x000f000f;
constexpr uint32_t kKv4Magic = 0x43004300;     // two bf16 128s

template <int D>
struct Kv4Page {
  static constexpr int kGroups = D / 64;
  static constexpr int kBytes = 9 * D;
  static constexpr int kParams = 8 * D;
  // byte of the word that holds channels 8 j .. 8 j + 7 of a token's K row
  static __device__ __forceinline__ int k_word(int token, int j) {
    return token * (D / 2) + (j % 8 / 2) * (D / 8) + (j / 8) * 8 + (j % 2) * 4;
  }
  // byte of V unit i of a token, group g
  static __device__ __forceinline__ int v_unit(int token, int i, int g) {
    return (i * 16 + token) * (D / 32) + 2 * g;
  }
  static __device__ __forceinline__ int param(int token, int g) {
    return kParams + (g * 16 + token) * 4;
  }
};

__device__ __forceinline__ float kv4_scale(uint32_t p) { return __uint_as_float(p & 0xffff0000u); }
__device__ __forceinline__ float kv4_zero(uint32_t p) { return __uint_as_float(p << 16); }   // 128 + z

// The bf16 pair 128 + (nibbles p of both halves).
__device__ __forceinline__ uint32_t kv4_pair(uint32_t w, int p) {
  return ((w >> (4 * p)) & kKv4Ones) | kKv4Magic;
}
// The same as a shift and one v_and_or_b32, for loops: that takes one constant from a scalar
// register, so that the other one has to be in a vector register.
struct Kv4Unpack {
  uint32_t ones = kKv4Ones, magic = kKv4Magic;
  __device__ __forceinline__ Kv4Unpack() { asm("" : "+s"(ones), "+v"(magic)); }
  __device__ __forceinline__ uint32_t operator()(uint32_t w, int p) const {
    return ((w >> (4 * p)) & ones) | magic;
  }
};

// Scale and zero point of a group from its lowest and highest value (0 counted in):
// s = (hi - lo) / 15 rounded to bf16 (formed from halves, which do not overflow),
// z = -lo / s rounded.  A group with a NaN or an infinity has s = NaN, and reads back as
// NaN throughout.
struct Kv4Scale {
  float s, z;
  __device__ __forceinline__ Kv4Scale(float lo, float hi, bool finite) {
    s = (float)(__bf16)((0.5f * hi - 0.5f * lo) / 7.5f);
    z = s > 0.f ? fminf(__builtin_rintf(-lo / s), 15.f) : 0.f;
    if (!finite) {
      s = __builtin_nanf("");
      z = 0.f;
    }
  }
  __device__ __forceinline__ uint32_t param() const {
    const uint32_t zz = __float_as_uint(128.f + z) >> 16;
    return (__float_as_uint(s) & 0xffff0000u) | zz;
  }
  // Codes of N values, as whole floats.  x / s is rounded to fp32 before it is rounded to a whole
  // number; both are bf16, so that a quotient that is no tie is at least 2^-10 away from one, and
  // one that is comes out exact (x times 1 / s and one step that makes good what is left of x).
  template <int N>
  __device__ __forceinline__ void codes(const float (&x)[N], float (&c)[N]) const {
    const bool near = s > 1e-30f && s < 1e30f;       // (the reciprocal and the step in range)
    const float r = 1.f / s;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float q = x[i] * r;
      q = __builtin_fmaf(__builtin_fmaf(-q, s, x[i]), r, q);
      if (!near) q = s > 0.f ? x[i] / s : 0.f;
      c[i] = __builtin_amdgcn_fmed3f(__builtin_rintf(q) + z, 0.f, 15.f);
    }
  }
};

}  // namespace rag
