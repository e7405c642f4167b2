// Refresh of a patch's rows of a 4-bit key / value cache, and the cache read back (Section 4: the stale buffers hold the keys and values of
// the whole image between the steps; in 4 bits they are a quarter of their size, and so is what devices would exchange).
#include "kv4.h"

namespace df {

namespace {

struct Kv4Params {
  const void *k, *v;                           // refresh: fresh rows; read: unused
  void *ko, *vo;                               // read: [B, L, kv_heads, d]
  long long ldk, bsk, ldv, bsv;
  Kv4View c;
  int L, kv_heads, tile0;
  int own_lo, own_n, own_period;               // as AttnArgs
  unsigned int period_recip;
};

// Largest bits over the G lanes of a row
template <int G>
__device__ __forceinline__ unsigned int group_max(unsigned int v) {
  auto dpp = [&](auto ctrl) { return (unsigned int)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xf, 0xf, true); };
  auto up = [&](unsigned int o) { v = v > o ? v : o; };
  up(dpp(std::integral_constant<int, 0xb1>{}));            // quad_perm 1 0 3 2
  up(dpp(std::integral_constant<int, 0x4e>{}));            // quad_perm 2 3 0 1
  up(dpp(std::integral_constant<int, 0x141>{}));           // row_half_mirror
  if constexpr (G >= 16) up(dpp(std::integral_constant<int, 0x140>{}));   // row_mirror
  return v;
}

__device__ __forceinline__ void ld8(const bf16_t* p, float* v) { ld_vec(p, v); }
__device__ __forceinline__ void ld8(const float* p, float* v) { ld_vec(p, v); ld_vec(p + 4, v + 4); }
__device__ __forceinline__ void st8(bf16_t* p, const float* v) { st_vec(p, v); }
__device__ __forceinline__ void st8(float* p, const float* v) { st_vec(p, v); st_vec(p + 4, v + 4); }

__device__ __forceinline__ unsigned int encode8(const float* x, float s, float inv) {
  if (!(s > 0.f)) return 0u;                               // zeros, or NaN (which the scale holds)
  unsigned int w = kv4_codes<0>(0u, x[0], x[1], s, inv);
  w = kv4_codes<1>(w, x[2], x[3], s, inv);
  w = kv4_codes<2>(w, x[4], x[5], s, inv);
  return kv4_codes<3>(w, x[6], x[7], s, inv);
}

// Where key j is among the fresh rows, or -1
__device__ __forceinline__ long long own_row(const Kv4Params& p, int j) {
  if (j >= p.L) return -1;
  if (p.own_period > 0) {
    const int r = (int)quotient_u32((unsigned int)j, (unsigned int)p.own_period, p.period_recip), rel = j - r * p.own_period - p.own_lo;
    return rel >= 0 && rel < p.own_n ? (long long)r * p.own_n + rel : -1;
  }
  const int rel = j - p.own_lo;
  return rel >= 0 && rel < p.own_n ? rel : -1;
}

// A workgroup per tile of 64 keys of a head; D / 8 lanes share a row, eight values each.  The codes of a value's 64 keys lie side by side, so
// the values' codes cross LDS.  Rows that are not the patch's keep their bytes; a byte that holds one key of the patch and one that is not is
// read and written by one lane, every other byte is written whole.  Bound by the conversion as it is
// dealt out: each lane of a row divides twice and rounds a quotient per value, and a wave with one row of the patch converts all of its.  A
// strip of 31 of 124 columns, 128 rows, 10 heads of 128 (20 MB read, about a quarter of the rows its own): 15 - 17 us, where the bytes take 5; 300 rows of
// 20 heads of 64: 4.4 - 4.8 us, the latency of a launch.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv4_refresh_kernel(Kv4Params p) {
  constexpr int G = D / 8, ROWS = 256 / G, PASS = 64 / ROWS, PITCH = G + 1;
  __shared__ unsigned int vw[64 * PITCH];
  __shared__ __attribute__((aligned(8))) unsigned char mine[64];
  const int tid = threadIdx.x, sub = tid % G, row = tid / G;
  const int tile = p.tile0 + blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const long long head = (long long)b * p.kv_heads + h;
  const T *k = (const T*)p.k + (long long)b * p.bsk + (long long)h * D + 8 * sub, *v = (const T*)p.v + (long long)b * p.bsv + (long long)h * D + 8 * sub;
  long long from[PASS];
  float x[PASS][2][8];
#pragma unroll
  for (int i = 0; i < PASS; ++i) {
    from[i] = own_row(p, tile * 64 + i * ROWS + row);
    if (from[i] >= 0) {
      ld8(k + from[i] * p.ldk, x[i][0]);
      ld8(v + from[i] * p.ldv, x[i][1]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][0][e] = x[i][1][e] = 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < PASS; ++i) {
    const int r = i * ROWS + row;
    if (sub == 0) mine[r] = from[i] >= 0;
    if (__builtin_amdgcn_ballot_w64(from[i] >= 0) == 0) continue;          // a strip of columns: most waves' rows are another patch's
    const long long at = head * p.c.pitch + (long long)tile * 64 + r;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      unsigned int m = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const unsigned int a = __float_as_uint(x[i][kv][e]) & 0x7fffffffu;
        m = m > a ? m : a;
      }
      const float s = kv4_scale(group_max<G>(m));
      const unsigned int w = encode8(x[i][kv], s, __fdiv_rn(1.0f, s));
      if (kv == 0 && from[i] >= 0) *reinterpret_cast<unsigned int*>(p.c.kc + at * (D / 2) + 4 * sub) = w;
      if (kv == 1) vw[r * PITCH + sub] = w;
      if (sub == 0 && from[i] >= 0) (kv ? p.c.vs : p.c.ks)[at] = (bf16_t)(__float_as_uint(s) >> 16);
    }
  }
  __syncthreads();
  unsigned char* vt = p.c.vc + (head * (p.c.pitch / 64) + tile) * (D * 32);
  if (tid >= D) return;
  const int g = tid >> 3, o = tid & 7;                     // values 8 g .., keys 8 o ..
  const u32x2 of = *reinterpret_cast<const u32x2*>(mine + 8 * o);
  if (!(of.x | of.y)) return;
  unsigned int w[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = vw[(8 * o + j) * PITCH + g];
  kv4_turn(w);
  if ((of.x & of.y) == 0x01010101u) {
#pragma unroll
    for (int e = 0; e < 8; ++e) *reinterpret_cast<unsigned int*>(vt + (8 * g + e) * 32 + o * 4) = w[e];
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {                            // keys 2 j and 2 j + 1
    const unsigned int o2 = ((j < 2 ? of.x : of.y) >> (16 * (j & 1))) & 0x101u, keep = o2 == 0x101u ? 0u : o2 == 1u ? 0xf0u : 0x0fu;
    if (!o2) continue;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      unsigned char* dst = vt + (8 * g + e) * 32 + o * 4 + j;
      *dst = (unsigned char)((((w[e] >> (8 * j)) & 0xffu) & ~keep) | (keep ? *dst & keep : 0u));
    }
  }
}

// A tile of V codes -> dwords of eight values of a key, at [key][D / 8 + 1]: 8 x 8 nibbles turn per eight values and eight keys
template <int D>
__device__ __forceinline__ void turn_values(const unsigned char* vt, unsigned int* vw, int tid) {
  for (int idx = tid; idx < D; idx += 256) {
    const int g = idx >> 3, o = idx & 7;
    unsigned int src[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) src[e] = *reinterpret_cast<const unsigned int*>(vt + (8 * g + e) * 32 + o * 4);
    kv4_turn(src);
#pragma unroll
    for (int j = 0; j < 8; ++j) vw[(8 * o + j) * (D / 8 + 1) + g] = src[j];
  }
}

// A tile of a head per workgroup; bound by memory: 15872 rows of 10 heads of 128 (21 MB of codes to 81 MB): 14.2 - 15.9 us, 6.5 TB/s
template <typename T, int D>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4Params p) {
  constexpr int G = D / 8, ROWS = 256 / G, PASS = 64 / ROWS, PITCH = G + 1;
  __shared__ unsigned int vw[64 * PITCH];
  const int tid = threadIdx.x, sub = tid % G, row = tid / G;
  const int tile = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const long long head = (long long)b * p.kv_heads + h;
  const unsigned char* vt = p.c.vc + (head * (p.c.pitch / 64) + tile) * (D * 32);
  unsigned int kw[PASS];
  float s[PASS][2];
#pragma unroll
  for (int i = 0; i < PASS; ++i) {
    const long long at = head * p.c.pitch + (long long)tile * 64 + i * ROWS + row;
    kw[i] = *reinterpret_cast<const unsigned int*>(p.c.kc + at * (D / 2) + 4 * sub);
    s[i][0] = bf2f(p.c.ks[at]);
    s[i][1] = bf2f(p.c.vs[at]);
  }
  turn_values<D>(vt, vw, tid);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PASS; ++i) {
    const int r = i * ROWS + row, j = tile * 64 + r;
    if (j >= p.L) continue;
    const long long to = (((long long)b * p.L + j) * p.kv_heads + h) * D + 8 * sub;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      float o[8];
      kv4_values(kv ? vw[r * PITCH + sub] : kw[i], s[i][kv], o);
      st8((T*)(kv ? p.vo : p.ko) + to, o);
    }
  }
}

// The rows that are not the patch's as bf16, side by side per head: what attention with many queries reads (qattn.hip), the conversion
// once for all blocks of rows.  8400 rows of 10 heads of 64: 7.8 - 8.5 us, 50400: 26 (168 MB, 6.4 TB/s)
template <int D>
__global__ __launch_bounds__(256) void kv4_expand_kernel(Kv4Params p, const int* lens, long long rows) {
  constexpr int G = D / 8, ROWS = 256 / G, PASS = 64 / ROWS, PITCH = G + 1;
  __shared__ unsigned int vw[64 * PITCH];
  const int tid = threadIdx.x, sub = tid % G, row = tid / G;
  const int tile = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  if (lens && tile * 64 >= lens[b]) return;
  const long long head = (long long)b * p.kv_heads + h;
  const unsigned char* vt = p.c.vc + (head * (p.c.pitch / 64) + tile) * (D * 32);
  unsigned int kw[PASS];
  float s[PASS][2];
#pragma unroll
  for (int i = 0; i < PASS; ++i) {
    const long long at = head * p.c.pitch + (long long)tile * 64 + i * ROWS + row;
    kw[i] = *reinterpret_cast<const unsigned int*>(p.c.kc + at * (D / 2) + 4 * sub);
    s[i][0] = bf2f(p.c.ks[at]);
    s[i][1] = bf2f(p.c.vs[at]);
  }
  turn_values<D>(vt, vw, tid);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PASS; ++i) {
    const int r = i * ROWS + row, j = tile * 64 + r;
    if (j >= p.L || own_row(p, j) >= 0) continue;
    int before = j - p.own_lo;                             // of the patch's rows, how many come before row j
    if (p.own_period > 0) {
      const int q = (int)quotient_u32((unsigned int)j, (unsigned int)p.own_period, p.period_recip);
      before = q * p.own_n + (j - q * p.own_period >= p.own_lo ? p.own_n : 0);
    } else {
      before = before >= 0 ? p.own_n : 0;
    }
    const long long to = ((head * rows) + j - before) * D + 8 * sub;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      float o[8];
      kv4_values(kv ? vw[r * PITCH + sub] : kw[i], s[i][kv], o);
      st_vec((bf16_t*)(kv ? p.vo : p.ko) + to, o);
    }
  }
}

}  // namespace

int launch_kv4_expand(const Kv4Args& a, const int* lens, long long rows, void* k, void* v, hipStream_t st) {
  Kv4Params p = {};
  p.ko = k; p.vo = v;
  p.c = kv4_view(a.cache, a.B, a.L, a.kv_heads, a.d);
  p.L = a.L; p.kv_heads = a.kv_heads; p.own_lo = a.own_lo; p.own_n = a.own_n; p.own_period = a.own_period;
  p.period_recip = a.own_period > 0 ? reciprocal_u32((unsigned int)a.own_period) : 0u;
  const dim3 grid((unsigned)(p.c.pitch / 64), (unsigned)a.kv_heads, (unsigned)a.B);
  if (a.d == 64) hipLaunchKernelGGL(kv4_expand_kernel<64>, grid, dim3(256), 0, st, p, lens, rows);
  else hipLaunchKernelGGL(kv4_expand_kernel<128>, grid, dim3(256), 0, st, p, lens, rows);
  DF_LAUNCH_CHECK();
  return DF_OK;
}

int launch_kv4_refresh(const Kv4Args& a, hipStream_t st) {
  Kv4Params p = {};
  p.k = a.k; p.v = a.v; p.ldk = a.ldk; p.bsk = a.bsk; p.ldv = a.ldv; p.bsv = a.bsv;
  p.c = kv4_view(a.cache, a.B, a.L, a.kv_heads, a.d);
  p.L = a.L; p.kv_heads = a.kv_heads; p.own_lo = a.own_lo; p.own_n = a.own_n; p.own_period = a.own_period;
  p.period_recip = a.own_period > 0 ? reciprocal_u32((unsigned int)a.own_period) : 0u;
  const int last = a.own_period > 0 ? a.L - 1 : a.own_lo + a.own_n - 1;
  p.tile0 = a.own_period > 0 ? 0 : a.own_lo / 64;
  const dim3 grid((unsigned)(last / 64 - p.tile0 + 1), (unsigned)a.kv_heads, (unsigned)a.B);
  if (a.dtype == DF_BF16 && a.d == 64) hipLaunchKernelGGL((kv4_refresh_kernel<bf16_t, 64>), grid, dim3(256), 0, st, p);
  else if (a.dtype == DF_BF16) hipLaunchKernelGGL((kv4_refresh_kernel<bf16_t, 128>), grid, dim3(256), 0, st, p);
  else if (a.d == 64) hipLaunchKernelGGL((kv4_refresh_kernel<float, 64>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((kv4_refresh_kernel<float, 128>), grid, dim3(256), 0, st, p);
  DF_LAUNCH_CHECK();
  return DF_OK;
}

int launch_kv4_read(const Kv4Args& a, void* k, void* v, hipStream_t st) {
  Kv4Params p = {};
  p.ko = k; p.vo = v;
  p.c = kv4_view(a.cache, a.B, a.L, a.kv_heads, a.d);
  p.L = a.L; p.kv_heads = a.kv_heads;
  const dim3 grid((unsigned)(p.c.pitch / 64), (unsigned)a.kv_heads, (unsigned)a.B);
  if (a.dtype == DF_BF16 && a.d == 64) hipLaunchKernelGGL((kv4_read_kernel<bf16_t, 64>), grid, dim3(256), 0, st, p);
  else if (a.dtype == DF_BF16) hipLaunchKernelGGL((kv4_read_kernel<bf16_t, 128>), grid, dim3(256), 0, st, p);
  else if (a.d == 64) hipLaunchKernelGGL((kv4_read_kernel<float, 64>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((kv4_read_kernel<float, 128>), grid, dim3(256), 0, st, p);
  DF_LAUNCH_CHECK();
  return DF_OK;
}

}  // namespace df
