// Norm of queries and keys per head with the position rotation in the same pass (what a diffusion transformer does to its fused projection
// before the attention of a patch, Section 4, Sparse operations: per-token work on the fresh tokens alone).
//
// A head's row x of d values: y = x / sqrt(mean(x^2) + eps) * gamma, then pairs (a, b) of the first rot_dim values turn by the token's
// angles: (a cos - b sin, b cos + a sin).  Everything in float, rounded once at the end.
#include "kernels.h"

namespace df {

namespace {

struct RopeParams {
  const void *q, *k;
  void *qo, *ko;
  const float *qg, *kg, *rot;
  const int* pos;
  long long ldq, bsq, ldk, bsk, ldqo, bsqo, ldko, bsko;
  int T, hq, heads, d, half, rot_len;      // heads: of queries and keys; half = rot_dim / 2
  unsigned int waves, per_token, per_token_recip, T_recip;
  int steps;                               // steps of 64 / G heads per wave
  float eps, inv_d;
};

// Sum over the G lanes that share a row, the same in each of them; added in a fixed order
template <int G>
__device__ __forceinline__ float group_sum(float v) {
  auto dpp = [&](auto ctrl) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  if constexpr (G >= 2) v += dpp(std::integral_constant<int, 0xb1>{});      // quad_perm 1 0 3 2
  if constexpr (G >= 4) v += dpp(std::integral_constant<int, 0x4e>{});      // quad_perm 2 3 0 1
  if constexpr (G >= 8) v += dpp(std::integral_constant<int, 0x141>{});     // row_half_mirror
  if constexpr (G >= 16) v += dpp(std::integral_constant<int, 0x140>{});    // row_mirror
  if constexpr (G >= 32) v += __shfl_xor(v, 16, 64);
  if constexpr (G >= 64) v += __shfl_xor(v, 32, 64);
  return v;
}

__device__ __forceinline__ void ld_n(const float* p, float (&v)[4]) { ld_vec(p, v); }
__device__ __forceinline__ void ld_n(const bf16_t* p, float (&v)[8]) { ld_vec(p, v); }
__device__ __forceinline__ void ld_n(const bf16_t* p, float (&v)[4]) {
  const u32x2 t = *reinterpret_cast<const u32x2*>(p);
  v[0] = __uint_as_float(t.x << 16); v[1] = __uint_as_float(t.x & 0xffff0000u);
  v[2] = __uint_as_float(t.y << 16); v[3] = __uint_as_float(t.y & 0xffff0000u);
}
__device__ __forceinline__ void st_n(float* p, const float (&v)[4]) { st_vec(p, v); }
__device__ __forceinline__ void st_n(bf16_t* p, const float (&v)[8]) { st_vec(p, v); }
__device__ __forceinline__ void st_n(bf16_t* p, const float (&v)[4]) {
  *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3])};
}

// G lanes share a head's row, V values each; a wave takes `steps` (at most four) times 64 / G heads of one token, so the token's angles and the scales are
// read once.  HALVES: value i turns with value i + half, which another lane of the row has normed; else with its neighbour.
// Bound by memory: 14401 tokens, 20 + 4 heads of 128 in float 62 - 65 us (5.6 TB/s); one token 2.8 - 3.2 us, 2400 tokens of 20 heads of 64 in bf16 by
// halves 5.7 - 6.2, the latency of one wave's reads and writes.
template <typename T, int V, int G, bool NORM, bool HALVES>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(RopeParams p) {
  constexpr int U = 4;                                     // rows of a lane, at most
  const unsigned int w = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (w >= p.waves) return;
  const int lane = threadIdx.x & 63, sub = lane / G, e0 = (lane % G) * V;
  const unsigned int tok = quotient_u32(w, p.per_token, p.per_token_recip);
  const int first = (int)(w - tok * p.per_token) * p.steps;
  const unsigned int b = quotient_u32(tok, (unsigned int)p.T, p.T_recip);
  const long long t = tok - b * (unsigned int)p.T;
  const bool in = e0 < p.d;
  const int n = 2 * p.half;
  const int at = p.pos ? p.pos[tok] : (int)t;
  const bool turns = e0 < n && at >= 0;                    // (a token that does not turn keeps its values whatever their partners are)

  // angles of this lane's values, sign of the partner's share included: y = y * c + partner * s
  float c[V], s[V];
#pragma unroll
  for (int i = 0; i < V; ++i) { c[i] = 1.f; s[i] = 0.f; }
  if (p.rot && turns) {
    if (at >= p.rot_len) {                                 // no such angles: the result must not pass for one
#pragma unroll
      for (int i = 0; i < V; ++i) c[i] = __uint_as_float(0x7fc00000u);
    } else {
      const bool second = HALVES && e0 >= p.half;
      const float* r = p.rot + (long long)at * n + (HALVES ? 2 * (second ? e0 - p.half : e0) : e0);
#pragma unroll
      for (int i = 0; i < (HALVES ? 2 * V : V); i += 4) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(r + i);
        if constexpr (HALVES) {
          c[i / 2] = a.x; c[i / 2 + 1] = a.z;
          s[i / 2] = second ? a.y : -a.y; s[i / 2 + 1] = second ? a.w : -a.w;
        } else {
          c[i] = a.x; c[i + 1] = a.x; c[i + 2] = a.z; c[i + 3] = a.z;
          s[i] = -a.y; s[i + 1] = a.y; s[i + 2] = -a.w; s[i + 3] = a.w;
        }
      }
    }
  }
  const int partner = HALVES && turns ? 4 * (lane + (e0 >= p.half ? -p.half : p.half) / V) : 4 * lane;   // the lane of the other half's values

  // all that the wave reads is requested at once
  float x[U][V], gx[NORM ? U : 1][V];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int h = (first + u) * (64 / G) + sub;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      x[u][i] = 0.f;
      if constexpr (NORM) gx[u][i] = 1.f;
    }
    if (u < p.steps && in && h < p.heads) {
      const bool isq = h < p.hq;
      const T* src = isq ? (const T*)p.q + b * p.bsq + t * p.ldq + (long long)h * p.d : (const T*)p.k + b * p.bsk + t * p.ldk + (long long)(h - p.hq) * p.d;
      ld_n(src + e0, x[u]);
      if constexpr (NORM) {
        const float* g = isq ? p.qg : p.kg;
        if (g) {
#pragma unroll
          for (int i = 0; i < V; i += 4) ld_vec(g + e0 + i, gx[u] + i);
        }
      }
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (u >= p.steps) break;
    const int h = (first + u) * (64 / G) + sub;
    if constexpr (NORM) {
      float sq = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i) sq = fmaf(x[u][i], x[u][i], sq);
      float v = fmaf(group_sum<G>(sq), p.inv_d, p.eps);
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(v >= 0x1p-96f && v < INFINITY)) != 0, 0)) {
        // Squares that left float's range, or are about to (what a square loses below 2^-126 is nothing beside 2^-96): the sum is that of the values
        // times a power of two, f.  1 / sqrt(v) is then too small by f, which the values of a small row take on, and those of a large one, in halves
        // with their scales, give up.
        const float f = v < 0x1p-96f ? 0x1p100f : v < INFINITY ? 1.f : 0x1p-100f, half = f < 1.f ? 0x1p-50f : 1.f;
        sq = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float y = x[u][i] * f;
          sq = fmaf(y, y, sq);
          x[u][i] = f > 1.f ? y : x[u][i] * half;
          gx[u][i] *= half;
        }
        v = fmaf(group_sum<G>(sq), p.inv_d, p.eps * f * f);
      }
      float r = __builtin_amdgcn_rsqf(v);
      r = fmaf(0.5f * r, fmaf(-v * r, r, 1.f), r);         // (the instruction is off by one unit in the last place)
#pragma unroll
      for (int i = 0; i < V; ++i) x[u][i] *= r * gx[u][i];
    }
    float o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float other = HALVES ? __int_as_float(__builtin_amdgcn_ds_bpermute(partner, __float_as_int(x[u][i]))) : x[u][i ^ 1];
      o[i] = turns ? fmaf(x[u][i], c[i], other * s[i]) : x[u][i];
    }
    if (in && h < p.heads) {
      T* dst = h < p.hq ? (T*)p.qo + b * p.bsqo + t * p.ldqo + (long long)h * p.d : (T*)p.ko + b * p.bsko + t * p.ldko + (long long)(h - p.hq) * p.d;
      st_n(dst + e0, o);
    }
  }
}

template <typename T, int V, int G>
void launch_rope(const RopeParams& p, bool norm, bool halves, hipStream_t st) {
  const dim3 grid((p.waves + 3) / 4);
  if (norm && halves) hipLaunchKernelGGL((qk_norm_rope_kernel<T, V, G, true, true>), grid, dim3(256), 0, st, p);
  else if (norm) hipLaunchKernelGGL((qk_norm_rope_kernel<T, V, G, true, false>), grid, dim3(256), 0, st, p);
  else if (halves) hipLaunchKernelGGL((qk_norm_rope_kernel<T, V, G, false, true>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((qk_norm_rope_kernel<T, V, G, false, false>), grid, dim3(256), 0, st, p);
}

}  // namespace

int launch_qk_norm_rope(const RopeArgs& a, hipStream_t st) {
  const bool bf = a.dtype == DF_BF16;
  // V values per lane, 16 bytes where everything allows it (bf16: else 8 bytes; partners of a rotation by halves lie half a rot_dim apart)
  const void* ptrs[] = {a.q, a.k, a.q_out, a.k_out};
  const long long strides[] = {a.ldq, a.bsq, a.ldk, a.bsk, a.ldqo, a.bsqo, a.ldko, a.bsko};
  int V = bf ? 8 : 4;
  if (bf && !a.interleaved && a.rot && (a.rot_dim / 2) % 8) V = 4;
  for (const void* x : ptrs) if (bf && (uintptr_t)x % 16) V = 4;
  for (long long s : strides) if (bf && s % 8) V = 4;
  for (const void* x : ptrs) if ((uintptr_t)x % (V * (bf ? 2 : 4))) return DF_EINVAL;
  for (long long s : strides) if (s % V) return DF_EINVAL;
  if (((uintptr_t)a.q_gamma | (uintptr_t)a.k_gamma | (uintptr_t)a.rot) % 16) return DF_EINVAL;
  int G = 2;
  while (G * V < a.d) G *= 2;
  RopeParams p = {};
  p.q = a.q; p.k = a.k; p.qo = a.q_out; p.ko = a.k_out; p.qg = a.q_gamma; p.kg = a.k_gamma; p.rot = a.rot; p.pos = a.pos;
  p.ldq = a.ldq; p.bsq = a.bsq; p.ldk = a.ldk; p.bsk = a.bsk; p.ldqo = a.ldqo; p.bsqo = a.bsqo; p.ldko = a.ldko; p.bsko = a.bsko;
  p.T = a.T; p.hq = a.heads; p.heads = a.heads + a.kv_heads; p.d = a.d; p.half = a.rot ? a.rot_dim / 2 : 0; p.rot_len = a.rot_len;
  p.eps = a.eps; p.inv_d = 1.0f / (float)a.d;
  const int all = cdiv(p.heads, 64 / G);                   // steps of a token, split evenly into waves of at most four
  p.per_token = (unsigned int)cdiv(all, 4);
  p.steps = cdiv(all, p.per_token);
  const long long waves = (long long)a.B * a.T * p.per_token;
  if (waves > (1LL << 26) - 4) return DF_ESHAPE;          // (a launch counts its work items in 32 bits)
  p.waves = (unsigned int)waves;
  p.per_token_recip = reciprocal_u32(p.per_token);
  p.T_recip = reciprocal_u32((unsigned int)a.T);
  const bool halves = a.rot && !a.interleaved, norm = a.norm != 0;
#define DF_ROPE(TYPE, VV)                                      \
  switch (G) {                                                 \
    case 2: launch_rope<TYPE, VV, 2>(p, norm, halves, st); break;   \
    case 4: launch_rope<TYPE, VV, 4>(p, norm, halves, st); break;   \
    case 8: launch_rope<TYPE, VV, 8>(p, norm, halves, st); break;   \
    case 16: launch_rope<TYPE, VV, 16>(p, norm, halves, st); break; \
    case 32: launch_rope<TYPE, VV, 32>(p, norm, halves, st); break; \
    default: launch_rope<TYPE, VV, 64>(p, norm, halves, st); break; \
  }
  if (!bf) { DF_ROPE(float, 4) }
  else if (V == 8) { DF_ROPE(bf16_t, 8) }
  else { DF_ROPE(bf16_t, 4) }
#undef DF_ROPE
  DF_LAUNCH_CHECK();
  return DF_OK;
}

}  // namespace df
