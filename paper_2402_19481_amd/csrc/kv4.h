// Keys and values held in 4 bits: layout and conversion (kv4.hip, qattn.hip).
//
// A row (token, head) of d values is held as e2m1 codes (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives) and one scale, a sixth of the row's
// largest magnitude rounded to six significant bits.  Level times scale has at most eight significant bits, so what a row stands for is exact in
// bf16: a matrix operand made from codes and scale carries no further rounding.
//   K codes  [B][kv_heads][Lp][d / 2]           value i of a row in nibble i (low nibble first)
//   V codes  [B][kv_heads][Lp / 64][d][32]      64 keys of a value: nibble j is key j of the tile (a matrix operand takes consecutive keys)
//   K scales [B][kv_heads][Lp] bf16, V scales the same;  Lp = L rounded up to 64
#pragma once
#include "kernels.h"

namespace df {

__host__ __device__ inline long long kv4_pitch(long long L) { return (L + 63) / 64 * 64; }
struct Kv4View {
  unsigned char *kc, *vc;                      // of batch item 0, head 0
  bf16_t *ks, *vs;
  long long pitch;                             // rows of a head
};
inline size_t kv4_bytes(long long B, long long L, long long kv_heads, long long d) {
  return (size_t)(B * kv_heads * kv4_pitch(L) * (d + 4));
}
inline Kv4View kv4_view(const void* cache, long long B, long long L, long long kv_heads, long long d) {
  Kv4View v;
  const long long rows = B * kv_heads * kv4_pitch(L);
  v.kc = (unsigned char*)const_cast<void*>(cache);
  v.vc = v.kc + rows * (d / 2);
  v.ks = (bf16_t*)(v.vc + rows * (d / 2));
  v.vs = v.ks + rows;
  v.pitch = kv4_pitch(L);
  return v;
}

// Scale of a row from the bits of its largest magnitude (bits of magnitudes order like the magnitudes, infinities and NaN above all).
// Rows with either are NaN as a whole; rows below 2^-100 are zeros (no denormal numbers arise); the largest scale keeps 6 * scale finite.
__device__ __forceinline__ float kv4_scale(unsigned int most) {
  if (most >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
  if (most < 0x0d800000u) return 0.f;
  const unsigned int q = __float_as_uint(__fdiv_rn(__uint_as_float(most), 6.0f));
  const float s = __uint_as_float((q + 0x1ffffu + ((q >> 18) & 1u)) & 0xfffc0000u);   // to nearest, ties to even: no quotient of a float lies
  return fminf(s, 1.3125f * 0x1p125f);                                              // so near a tie that its own rounding decides
}

// Codes of x0, x1 in byte `SEL` of `old`.  x / s correctly rounded (product, remainder, correction; inv = 1 / s rounded): it is equal to a
// border between two levels exactly where x is, since s has six bits; the conversion rounds to nearest even.
template <int SEL>
__device__ __forceinline__ unsigned int kv4_codes(unsigned int old, float x0, float x1, float s, float inv) {
  const float q0 = x0 * inv, q1 = x1 * inv;
  const float r0 = fmaf(fmaf(-q0, s, x0), inv, q0), r1 = fmaf(fmaf(-q1, s, x1), inv, q1);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, r0, r1, 1.0f, SEL);
}

// Levels of byte SEL
template <int SEL>
__device__ __forceinline__ f32x2 kv4_levels(unsigned int w) { return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, SEL); }

// 8 x 8 nibbles turn: nibble j of a[i] becomes nibble i of a[j] (halves, bytes, nibbles change places: 32 instructions)
__device__ __forceinline__ void kv4_turn(unsigned int (&a)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned int t = a[i], u = a[i + 4];
    a[i] = __builtin_amdgcn_perm(u, t, 0x05040100u);
    a[i + 4] = __builtin_amdgcn_perm(u, t, 0x07060302u);
  }
#pragma unroll
  for (int i = 0; i < 8; i += i % 4 == 1 ? 3 : 1) {
    const unsigned int t = a[i], u = a[i + 2];
    a[i] = __builtin_amdgcn_perm(u, t, 0x06020400u);
    a[i + 2] = __builtin_amdgcn_perm(u, t, 0x07030501u);
  }
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const unsigned int t = a[i], u = a[i + 1];
    a[i] = (t & 0x0f0f0f0fu) | ((u << 4) & 0xf0f0f0f0u);
    a[i + 1] = ((t >> 4) & 0x0f0f0f0fu) | (u & 0xf0f0f0f0u);
  }
}

// What eight codes stand for
__device__ __forceinline__ void kv4_values(unsigned int w, float s, float* o) {
  const f32x2 a[4] = {kv4_levels<0>(w), kv4_levels<1>(w), kv4_levels<2>(w), kv4_levels<3>(w)};
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = a[i >> 1][i & 1] * s;
}

}  // namespace df
