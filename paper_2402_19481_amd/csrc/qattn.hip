// Attention of a patch's queries to rows of another length (an encoder's states) and to a 4-bit cache with the patch's own rows fresh
// (Section 4, Sparse operations: the keys and values are a scatter output; softmax does not ask for their order, so the cache's rows without
// the patch's own, and the fresh ones, are two segments of one sum).
//
//   out = softmax(q k^T * scale) v per head, one pass over the keys with the running maximum and sum.  `group` query heads share a key head;
//   they are rows of one problem: row r of a key head is query r / group, head r % group of the group, so shared keys are read once.
//
// bf16: S^T = K Q^T and O^T = V^T P^T on v_mfma_f32_32x32x16_bf16 (a lane owns one row of queries; the exponentiated accumulators of S^T are,
// by the order in which keys are assigned to its rows, the operand P^T without any data movement).  P is rounded to bf16 as the matrix
// instruction takes it (2^-9 of each weight, averaged over the keys); sums, maxima and O are float, the row sums are those of the float weights.
// float: the same on v_mfma_f32_32x32x2_f32, for the small full-precision networks.
#include "kv4.h"

namespace df {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

struct Seg {
  const void *k, *v;                           // rows of d values
  long long ldk, ldv, bsk, bsv;                // elements between rows and batch items
  long long hsk, hsv;                          // and between heads
  int n;
};
struct QParams {
  const void* q;
  long long ldq, bsq;
  Seg seg[2];
  const unsigned char* mask;                   // [B, n of segment 0], 0: not a key; or nullptr
  const int* lens;                             // [B] rows of segment 0 that are keys, or nullptr
  Kv4View c;                                   // the cache, where segment 0 is one (its n rows but the own ones)
  int own_lo, own_n, own_period;
  void* out;                                   // [B, Lq, heads, d]
  float *part_o, *part_ml;                     // [nsplit][B * kv_heads][rows][d], [..][2] (nsplit > 1)
  int B, Lq, group, kv_heads, d, rows;         // rows = Lq * group
  unsigned int group_recip;
  int nsplit, tiles_per_split;
  float sc;                                    // scale * log2(e)
};

__device__ __forceinline__ int seg0_rows(const QParams& p, int b) {
  if (!p.lens) return p.seg[0].n;
  const int n = p.lens[b];
  return n < 0 ? 0 : n < p.seg[0].n ? n : p.seg[0].n;
}
__device__ __forceinline__ unsigned long long low_bits(int n) { return n >= 64 ? ~0ULL : n <= 0 ? 0ULL : (1ULL << n) - 1ULL; }

// Offset of row r of a key head's problem in [B, Lq, heads, d], heads * d = ld
__device__ __forceinline__ long long row_offset(const QParams& p, int b, int kh, int r, long long bs, long long ld) {
  const unsigned int i = quotient_u32((unsigned int)r, (unsigned int)p.group, p.group_recip);
  return (long long)b * bs + (long long)i * ld + (long long)(kh * p.group + (r - (int)i * p.group)) * p.d;
}

// Workgroup -> (block of rows, key head, batch item, split); an XCD takes a contiguous range, so a head's keys are read into few L2s
__device__ __forceinline__ void place(const QParams& p, int nrb, int& rb, int& kh, int& b, int& split) {
  int t = blockIdx.x;
  const int nwg = gridDim.x, xcd = t & 7, base = nwg >> 3, rem = nwg & 7;
  t = xcd * base + (xcd < rem ? xcd : rem) + (t >> 3);
  rb = t % nrb;
  t /= nrb;
  split = t % p.nsplit;
  t /= p.nsplit;
  kh = t % p.kv_heads;
  b = t / p.kv_heads;
}

// Tiles of 64 keys that a workgroup sums over: those of segment 0 that have a key, then segment 1's
constexpr int kListTiles = 1024;               // tiles of one split whose words are kept (masks)

// ---- bf16 rows ----
template <int D, int NW, bool MASK>
__global__ __launch_bounds__(64 * NW, 2) void rows_attn(QParams p) {
  constexpr int TK = 64, TILE = TK * D * 2, CH = D / 8, KS = D / 16, DB = D / 32, LPT = TILE / 1024 / NW, RPI = 1024 / (D * 2);
  static_assert(LPT >= 1, "a wave loads a part of each tile");
  extern __shared__ __attribute__((aligned(16))) char smem[];             // three slots of a K and a V tile; MASK: words and tiles
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, c = lane & 31, csig = (c & 0x13) | ((c & 4) << 1) | ((c & 8) >> 1);
  int rb, kh, b, split;
  place(p, (p.rows + 32 * NW - 1) / (32 * NW), rb, kh, b, split);
  const int n0 = seg0_rows(p, b), n1 = p.seg[1].n, tiles0 = (n0 + 63) >> 6;
  const int lo = split * p.tiles_per_split;
  int hi = lo + p.tiles_per_split;
  if (hi > tiles0 + ((n1 + 63) >> 6)) hi = tiles0 + ((n1 + 63) >> 6);
  int nt = hi > lo ? hi - lo : 0;

  unsigned long long* words = (unsigned long long*)(smem + 6 * TILE);     // MASK: of the tiles that have a key
  unsigned short* list = (unsigned short*)(words + kListTiles);
  if constexpr (MASK) {
    for (int i = wave; i < nt; i += NW) {
      const int key = (lo + i) * 64 + lane;
      const unsigned long long w = __builtin_amdgcn_ballot_w64(key < n0 && p.mask[(long long)b * p.seg[0].n + key] != 0);
      if (lane == 0) words[i] = w;
    }
    __syncthreads();
    // the tiles with a key move to the front (wave 0; every chunk is read before it is written, in front of itself)
    if (wave == 0) {
      int at = 0;
      for (int i = 0; i < nt; i += 64) {
        const unsigned long long w = i + lane < nt ? words[i + lane] : 0ULL;
        const unsigned long long some = __builtin_amdgcn_ballot_w64(w != 0);
        const int to = at + __popcll(some & low_bits(lane));
        if (w) { words[to] = w; list[to] = (unsigned short)(i + lane); }
        at += __popcll(some);
      }
      if (lane == 0) *(int*)(list + kListTiles) = at;
    }
    __syncthreads();
    nt = *(volatile int*)(list + kListTiles);
  }
  nt = __builtin_amdgcn_readfirstlane(nt);

  const int row = rb * 32 * NW + wave * 32 + c;
  const bool have = row < p.rows;
  const bool idle = __builtin_amdgcn_readfirstlane(rb * 32 * NW + wave * 32) >= p.rows;
  bf16x8 qreg[KS];
  {
    const bf16_t* qp = (const bf16_t*)p.q + row_offset(p, b, kh, have ? row : 0, p.bsq, p.ldq);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u32x4 t = {0u, 0u, 0u, 0u};
      if (have && 16 * s + 8 * g < p.d) t = *reinterpret_cast<const u32x4*>(qp + 16 * s + 8 * g);
      qreg[s] = __builtin_bit_cast(bf16x8, t);
    }
  }

  auto tile_of = [&](int i) { return MASK ? (int)list[i] : i; };
  auto word_of = [&](int i, int t) {
    if constexpr (MASK) return words[i];
    else return t < tiles0 ? low_bits(n0 - t * 64) : low_bits(n1 - (t - tiles0) * 64);
  };
  // Direct loads of tile i to slot: keys that are none are read as one that is (their weight is 0, the value must be finite where the others
  // are); values beyond d are read as the first ones (Q is 0 there, those of O are dropped)
  auto load = [&](int i, int slot) {
    const int t = lo + tile_of(i);
    const unsigned long long w = word_of(i, t);
    const bool second = !MASK && t >= tiles0;
    const Seg& s = p.seg[second ? 1 : 0];
    const int key0 = (second ? t - tiles0 : t) * 64, some = __builtin_ctzll(w);
    const bf16_t* k = (const bf16_t*)s.k + (long long)b * s.bsk + (long long)kh * s.hsk + (long long)key0 * s.ldk;
    const bf16_t* v = (const bf16_t*)s.v + (long long)b * s.bsv + (long long)kh * s.hsv + (long long)key0 * s.ldv;
#pragma unroll
    for (int j = 0; j < LPT; ++j) {
      const int r = (wave * LPT + j) * RPI + lane / CH, at = lane % CH;
      const int from = (w >> r) & 1 ? r : some;
      const int kc = (at ^ (D == 64 ? (r >> 1) & 7 : r & 15)) * 8;
      const int vc = (at ^ (D == 64 ? ((r >> 1) & 1) * 2 ^ ((r >> 3) & 1) * 4 : (r & 3) * 4)) * 8;
      char* to = smem + slot * 2 * TILE + (wave * LPT + j) * 1024;
      lds_load16(k + (long long)from * s.ldk + (kc < p.d ? kc : 0), to);
      lds_load16(v + (long long)from * s.ldv + (vc < p.d ? vc : 0), to + TILE);
    }
  };

  f32x16 o[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  float m = -1e30f, l = 0.f;
  const int tri = lane & 15;

  if (nt > 0) {
    load(0, 0);
    load(nt > 1 ? 1 : 0, 1);
    for (int i = 0, slot = 0; i < nt; ++i, slot = slot == 2 ? 0 : slot + 1) {
      // tile i has landed for every wave, and every wave has read tile i - 1, whose slot takes tile i + 2
      __builtin_amdgcn_s_waitcnt(((2 * LPT) & 0xF) | (((2 * LPT) >> 4) << 14) | (0x7 << 4) | (0 << 8));
      block_sync();
      load(i + 2 < nt ? i + 2 : nt - 1, slot == 0 ? 2 : slot - 1);
      if (idle) continue;
      const char* kt = smem + slot * 2 * TILE;
      const char* vt = kt + TILE;
      f32x16 s[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const int r = 32 * kb + csig;
          const u32x4 a = *reinterpret_cast<const u32x4*>(kt + r * (D * 2) + (((2 * ks + g) ^ (D == 64 ? (r >> 1) & 7 : r & 15)) * 16));
          s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), qreg[ks], s[kb], 0, 0, 0);
        }
      }
      const unsigned long long w = word_of(i, lo + tile_of(i));
      if (w != ~0ULL) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (!((w >> (32 * kb + 16 * (e >> 3) + 8 * g + (e & 7))) & 1)) s[kb][e] = -INFINITY;
      }
      float top = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, s[kb][e]);
      top = fmaxf(top, __shfl_xor(top, 32, 64)) * p.sc;
      if (__builtin_amdgcn_ballot_w64(top > m + 8.f)) {
        const float mn = fmaxf(m, top), alpha = __builtin_amdgcn_exp2f(m - mn);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[db][e] *= alpha;
        l *= alpha;
        m = mn;
      }
      u32x4 pk[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] = __builtin_amdgcn_exp2f(fmaf(s[u >> 1][8 * (u & 1) + e], p.sc, -m));
          l += x[e];
        }
        pk[u] = u32x4{pack_bf2(x[0], x[1]), pack_bf2(x[2], x[3]), pack_bf2(x[4], x[5]), pack_bf2(x[6], x[7])};
      }
#pragma unroll
      for (int ts = 0; ts < 4; ++ts)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const int key = 16 * ts + 8 * g + (tri >> 2);
          const int chunk = 4 * db + 2 * ((lane >> 4) & 1) + (tri & 1);
          const int pc = D == 64 ? chunk ^ (2 * ((key >> 1) & 1)) ^ (4 * ((key >> 3) & 1)) : chunk ^ ((key & 3) * 4);
          const char* at = vt + key * (D * 2) + pc * 16 + ((tri >> 1) & 1) * 8;
          typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
          const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(at));
          // keys 4 .. 7 of the eight; their swizzle (by key & 3 or by bits 1 and 3) is the same
          const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(at + 4 * D * 2));
          const bf16x8 a = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, pk[ts]), o[db], 0, 0, 0);
        }
    }
    __builtin_amdgcn_s_waitcnt(0xf70);         // no direct load outlives the wave
    l += __shfl_xor(l, 32, 64);
    if (l == 0.f) l = __uint_as_float(0x7fc00000u);        // keys, and every score -inf: no softmax
  } else {
    m = -INFINITY;
  }
  if (!have) return;
  if (p.nsplit == 1) {
    const float inv = nt > 0 ? 1.0f / l : 0.f;             // no key: zeros
    bf16_t* op = (bf16_t*)p.out + row_offset(p, b, kh, row, (long long)p.Lq * p.kv_heads * p.group * p.d, (long long)p.kv_heads * p.group * p.d);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const int at = 32 * db + 16 * f + 8 * g;
        if (at >= p.d) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = o[db][8 * f + e] * inv;
        st_vec(op + at, v);
      }
  } else {
    const long long at0 = ((long long)split * p.B * p.kv_heads + (long long)b * p.kv_heads + kh) * p.rows + row;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const int at = 32 * db + 16 * f + 8 * g;
        if (at >= p.d) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = o[db][8 * f + e];
        st_vec(p.part_o + at0 * p.d + at, v);
        st_vec(p.part_o + at0 * p.d + at + 4, v + 4);
      }
    if (g == 0) { p.part_ml[2 * at0] = m; p.part_ml[2 * at0 + 1] = l; }
  }
}

// ---- merge ----
// Partial results of the splits, eight values of a row per lane, in the order of the splits
template <typename T>
__global__ __launch_bounds__(256) void merge_splits(QParams p, unsigned int per_row, unsigned int per_row_recip, unsigned int total, unsigned int rows_recip,
                                                    unsigned int heads_recip) {
  const unsigned int idx = blockIdx.x * 256 + threadIdx.x;
  if (idx >= total) return;
  const unsigned int row = quotient_u32(idx, per_row, per_row_recip);
  const int at = (int)(idx - row * per_row) * 8;
  const unsigned int all = (unsigned int)(p.B * p.kv_heads) * (unsigned int)p.rows;
  float m = -INFINITY, l = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < p.nsplit; ++s) m = fmaxf(m, p.part_ml[2 * ((long long)s * all + row)]);
  for (int s = 0; s < p.nsplit; ++s) {
    const long long r = (long long)s * all + row;
    const float ms = p.part_ml[2 * r], w = ms == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ms - m);
    float v[8];
    ld_vec(p.part_o + r * p.d + at, v);
    ld_vec(p.part_o + r * p.d + at + 4, v + 4);
    if (ms == -INFINITY) continue;
    l = fmaf(w, p.part_ml[2 * r + 1], l);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = fmaf(w, v[e], o[e]);
  }
  const float inv = m == -INFINITY ? 0.f : 1.0f / l;       // no key in any split: zeros
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] *= inv;
  const unsigned int bh = quotient_u32(row, (unsigned int)p.rows, rows_recip), b = quotient_u32(bh, (unsigned int)p.kv_heads, heads_recip);
  const long long ld = (long long)p.kv_heads * p.group * p.d;
  T* op = (T*)p.out + row_offset(p, (int)b, (int)(bh - b * p.kv_heads), (int)(row - bh * p.rows), (long long)p.Lq * ld, ld) + at;
  st_vec(op, o);
  if constexpr (sizeof(T) == 4) st_vec(op + 4, o + 4);
}

// ---- float ----
// Four waves of 32 rows each share a tile of 32 keys in LDS.  KV4: segment 0 is the cache (own rows masked out), segment 1 rows of floats.
template <int D, bool KV4>
__global__ __launch_bounds__(256) void float_attn(QParams p) {
  constexpr int PK = D + 4, PV = D + 8, DB = D / 32, PER = D / 8;
  __shared__ __attribute__((aligned(16))) float kt[32 * PK], vt[32 * PV];
  __shared__ float bias[32];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, c = lane & 31;
  int rb, kh, b, split;
  place(p, (p.rows + 127) / 128, rb, kh, b, split);
  const int n0 = seg0_rows(p, b), n1 = p.seg[1].n, tiles0 = (n0 + 31) >> 5, all = tiles0 + ((n1 + 31) >> 5);
  const int lo = split * p.tiles_per_split, hi = lo + p.tiles_per_split < all ? lo + p.tiles_per_split : all;
  const int row = rb * 128 + wave * 32 + c;
  const bool have = row < p.rows, idle = rb * 128 + wave * 32 >= p.rows;
  float q[D / 2];                                          // values 8 j + 4 g + i at 4 j + i
  {
    const float* qp = (const float*)p.q + row_offset(p, b, kh, have ? row : 0, p.bsq, p.ldq);
#pragma unroll
    for (int j = 0; j < D / 8; ++j) {
      f32x4 t = {0.f, 0.f, 0.f, 0.f};
      if (have && 8 * j + 4 * g < p.d) t = *reinterpret_cast<const f32x4*>(qp + 8 * j + 4 * g);
      q[4 * j] = t.x; q[4 * j + 1] = t.y; q[4 * j + 2] = t.z; q[4 * j + 3] = t.w;
    }
  }
  f32x16 o[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  float m = -1e30f, l = 0.f;
  bool any = false;                                        // a key so far
  for (int t = lo; t < hi; ++t) {
    const bool second = t >= tiles0;
    const Seg& s = p.seg[second ? 1 : 0];
    const int key0 = (second ? t - tiles0 : t) * 32, n = second ? n1 : n0;
    const int r = tid >> 3, part = (tid & 7) * PER, key = key0 + r;
    bool valid = key < n;
    if (valid && !second && p.mask) valid = p.mask[(long long)b * p.seg[0].n + key] != 0;
    if (KV4 && valid && !second && p.own_n > 0) {
      const int rel = (p.own_period > 0 ? key % p.own_period : key) - p.own_lo;
      valid = !(rel >= 0 && rel < p.own_n);
    }
    if (!__syncthreads_or(valid)) continue;                // (also: the last tile's reads are done)
    any = true;
    if (!KV4 || second) {
      const float* k = (const float*)s.k + (long long)b * s.bsk + (long long)kh * s.hsk + (long long)key * s.ldk;
      const float* v = (const float*)s.v + (long long)b * s.bsv + (long long)kh * s.hsv + (long long)key * s.ldv;
#pragma unroll
      for (int i = 0; i < PER; i += 4) {
        f32x4 a = {0.f, 0.f, 0.f, 0.f}, w = a;
        if (valid && part + i < p.d) {
          a = *reinterpret_cast<const f32x4*>(k + part + i);
          w = *reinterpret_cast<const f32x4*>(v + part + i);
        }
        *reinterpret_cast<f32x4*>(kt + r * PK + part + i) = a;
        *reinterpret_cast<f32x4*>(vt + r * PV + part + i) = w;
      }
    } else {
      const long long head = (long long)b * p.kv_heads + kh, base = head * p.c.pitch;
      const float sk = valid ? bf2f(p.c.ks[base + key]) : 0.f;
#pragma unroll
      for (int i = 0; i < PER; i += 8) {
        const unsigned int w = *reinterpret_cast<const unsigned int*>(p.c.kc + (base + key) * (D / 2) + (part + i) / 2);
        const f32x2 a0 = kv4_levels<0>(w), a1 = kv4_levels<1>(w), a2 = kv4_levels<2>(w), a3 = kv4_levels<3>(w);
        float* to = kt + r * PK + part + i;
        *reinterpret_cast<f32x4*>(to) = f32x4{a0.x * sk, a0.y * sk, a1.x * sk, a1.y * sk};
        *reinterpret_cast<f32x4*>(to + 4) = f32x4{a2.x * sk, a2.y * sk, a3.x * sk, a3.y * sk};
      }
      for (int idx = tid; idx < D * 4; idx += 256) {       // eight keys of a value
        const int e = idx >> 2, k8 = (key0 & 32) + 8 * (idx & 3);
        const unsigned int w = *reinterpret_cast<const unsigned int*>(p.c.vc + (head * (p.c.pitch / 64) + (key0 >> 6)) * (D * 32) + e * 32 + k8 / 2);
        const f32x2 a[4] = {kv4_levels<0>(w), kv4_levels<1>(w), kv4_levels<2>(w), kv4_levels<3>(w)};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int kk = 8 * (idx & 3) + j;
          const float x = a[j >> 1][j & 1] * bf2f(p.c.vs[base + key0 + kk]);
          vt[kk * PV + e] = x;
        }
      }
    }
    if ((tid & 7) == 0) bias[r] = valid ? 0.f : -INFINITY;
    __syncthreads();
    if (idle) continue;
    f32x16 sa;
#pragma unroll
    for (int e = 0; e < 16; ++e) sa[e] = 0.f;
#pragma unroll
    for (int j = 0; j < D / 8; ++j) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(kt + c * PK + 8 * j + 4 * g);
#pragma unroll
      for (int i = 0; i < 4; ++i) sa = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], q[4 * j + i], sa, 0, 0, 0);
    }
    float top = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      if (bias[8 * (e >> 2) + 4 * g + (e & 3)] != 0.f) sa[e] = -INFINITY;
      top = fmaxf(top, sa[e]);
    }
    top = fmaxf(top, __shfl_xor(top, 32, 64)) * p.sc;
    const float mn = fmaxf(m, top), alpha = __builtin_amdgcn_exp2f(m - mn);
    m = mn;
    l *= alpha;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[db][e] *= alpha;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int kk = 8 * (e >> 2) + 4 * g + (e & 3);
      const float x = __builtin_amdgcn_exp2f(fmaf(sa[e], p.sc, -m));
      l += x;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        float v = vt[kk * PV + 32 * db + c];
        if (KV4 && bias[kk] != 0.f) v = 0.f;               // (a row that is none may hold a scale that is none)
        o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, x, o[db], 0, 0, 0);
      }
    }
  }
  l += __shfl_xor(l, 32, 64);
  if (any && l == 0.f) l = __uint_as_float(0x7fc00000u);
  if (!any) m = -INFINITY;
  if (!have) return;
  const long long at0 = ((long long)split * p.B * p.kv_heads + (long long)b * p.kv_heads + kh) * p.rows + row;
  float* to;
  float f = 1.f;
  if (p.nsplit == 1) {
    to = (float*)p.out + row_offset(p, b, kh, row, (long long)p.Lq * p.kv_heads * p.group * p.d, (long long)p.kv_heads * p.group * p.d);
    f = any ? 1.0f / l : 0.f;
  } else {
    to = p.part_o + at0 * p.d;
    if (g == 0) { p.part_ml[2 * at0] = m; p.part_ml[2 * at0 + 1] = l; }
  }
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int at = 32 * db + 2 * e + 4 * g;
      if (at >= p.d) continue;
      *reinterpret_cast<f32x4*>(to + at) = f32x4{o[db][e] * f, o[db][e + 1] * f, o[db][e + 2] * f, o[db][e + 3] * f};
    }
}

// ---- 4-bit cache, few rows ----
// NQ * 16 rows of queries against tiles of 64 keys that a wave reads into registers as they lie in the cache, the next tile while this one is
// summed; every wave takes every fourth tile.  A lane's dword of codes is eight values of a key (K) or eight keys of a value (V): an operand of
// v_mfma_f32_16x16x32_bf16 once its levels, which are exact in bf16, are converted.  The scales are those of keys: they multiply the scores and
// the weights, in float.  Score register (kb, r) of lane group gg is key 16 gg + 4 kb + r.
template <int D, int NQ>
__global__ __launch_bounds__(256, 2) void few_rows_kv4(QParams p) {
  constexpr int KS = D / 32, DB = D / 16, CPL = D / 4;     // k-steps, blocks of 16 values, values of a key per lane
  typedef __attribute__((ext_vector_type(KS))) unsigned int KVec;
  constexpr int ROW = D + 4;
  __shared__ __attribute__((aligned(16))) float red[4 * 16 * ROW];
  __shared__ float red_ml[4][16][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), rho = lane & 15, gg = lane >> 4;
  int rb, kh, b, split;
  place(p, (p.rows + 16 * NQ - 1) / (16 * NQ), rb, kh, b, split);
  const int n0 = seg0_rows(p, b), tiles = (n0 + 63) >> 6;
  const int lo = split * p.tiles_per_split, hi = lo + p.tiles_per_split < tiles ? lo + p.tiles_per_split : tiles;
  const long long head = (long long)b * p.kv_heads + kh, base = head * p.c.pitch;
  const unsigned char* kc = p.c.kc + (base + 16 * (rho >> 2) + (rho & 3)) * (D / 2) + gg * (D / 8);
  const unsigned char* vc = p.c.vc + base * (D / 2) + rho * 32 + gg * 8;
  const bf16_t *ks = p.c.ks + base + 16 * gg, *vs = p.c.vs + base + 16 * gg;
  bf16x8 q[NQ][KS];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int row = rb * 16 * NQ + 16 * n + rho;
    const bf16_t* qp = (const bf16_t*)p.q + row_offset(p, b, kh, row < p.rows ? row : 0, p.bsq, p.ldq) + CPL * gg;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u32x4 t = {0u, 0u, 0u, 0u};
      if (row < p.rows) t = *reinterpret_cast<const u32x4*>(qp + 8 * s);
      q[n][s] = __builtin_bit_cast(bf16x8, t);
    }
  }
  struct Tile { KVec k[4]; u32x2 v[DB]; u32x4 sk[2], sv[2]; };
  auto load = [&](Tile& t, int i) {
    const long long key = (long long)i * 64;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) t.k[kb] = *reinterpret_cast<const KVec*>(kc + (key + 8 * (kb >> 1) + 4 * (kb & 1)) * (D / 2));
#pragma unroll
    for (int i2 = 0; i2 < 2; ++i2) {
      t.sk[i2] = *reinterpret_cast<const u32x4*>(ks + key + 8 * i2);
      t.sv[i2] = *reinterpret_cast<const u32x4*>(vs + key + 8 * i2);
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) t.v[db] = *reinterpret_cast<const u32x2*>(vc + key * (D / 2) + db * 16 * 32);
  };
  auto operand = [&](unsigned int w) {                     // eight codes as bf16
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0), b2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1);
    const bf16x2 c2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2), d2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3);
    return bf16x8{a[0], a[1], b2[0], b2[1], c2[0], c2[1], d2[0], d2[1]};
  };
  f32x4 o[NQ][DB];
  float m[NQ], l[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
#pragma unroll
    for (int i = 0; i < DB; ++i) o[n][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    m[n] = -1e30f; l[n] = 0.f;
  }
  const bool any = lo + wave < hi;
  Tile cur, nxt;
  if (any) load(cur, lo + wave);
  for (int t = lo + wave; t < hi; t += 4) {
    load(nxt, t + 4 < hi ? t + 4 : t);
    f32x4 s[NQ][4];
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) s[n][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks2 = 0; ks2 < KS; ++ks2) {
        const bf16x8 a = operand(cur.k[kb][ks2]);
#pragma unroll
        for (int n = 0; n < NQ; ++n) s[n][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[n][ks2], s[n][kb], 0, 0, 0);
      }
    }
    const int left = n0 - t * 64 - 16 * gg;                // of the lane's 16 keys
    float fk[16], fv[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const unsigned int wk = cur.sk[j >> 3][(j & 7) >> 1], wv = cur.sv[j >> 3][(j & 7) >> 1];
      fk[j] = __uint_as_float(j & 1 ? wk & 0xffff0000u : wk << 16) * p.sc;
      fv[j] = __uint_as_float(j & 1 ? wv & 0xffff0000u : wv << 16);
    }
    const bool ragged = (t + 1) * 64 > n0;
    bf16x8 pf[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float x[16], top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 16; ++j) x[j] = s[n][j >> 2][j & 3] * fk[j];
      if (ragged) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          if (j >= left) { x[j] = -INFINITY; fv[j] = 0.f; }
        }
      }
#pragma unroll
      for (int j = 0; j < 16; ++j) top = fmaxf(top, x[j]);
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      if (__builtin_amdgcn_ballot_w64(top > m[n] + 8.f)) {
        const float mn = fmaxf(m[n], top), alpha = __builtin_amdgcn_exp2f(m[n] - mn);
#pragma unroll
        for (int db = 0; db < DB; ++db) o[n][db] *= alpha;
        l[n] *= alpha;
        m[n] = mn;
      }
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        x[j] = __builtin_amdgcn_exp2f(x[j] - m[n]);
        l[n] += x[j];
        x[j] *= fv[j];
      }
#pragma unroll
      for (int ts = 0; ts < 2; ++ts)
        pf[n][ts] = __builtin_bit_cast(bf16x8, u32x4{pack_bf2(x[8 * ts], x[8 * ts + 1]), pack_bf2(x[8 * ts + 2], x[8 * ts + 3]),
                                                     pack_bf2(x[8 * ts + 4], x[8 * ts + 5]), pack_bf2(x[8 * ts + 6], x[8 * ts + 7])});
    }
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int ts = 0; ts < 2; ++ts) {
        const bf16x8 a = operand(cur.v[db][ts]);
#pragma unroll
        for (int n = 0; n < NQ; ++n) o[n][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pf[n][ts], o[n][db], 0, 0, 0);
      }
    cur = nxt;
  }
  // the four waves' parts
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    float ln = l[n] + __shfl_xor(l[n], 16, 64);
    ln += __shfl_xor(ln, 32, 64);
    if (any && ln == 0.f) ln = __uint_as_float(0x7fc00000u);
    if (n) __syncthreads();
#pragma unroll
    for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(red + (wave * 16 + rho) * ROW + 16 * db + 4 * gg) = o[n][db];
    if (gg == 0) { red_ml[wave][rho][0] = any ? m[n] : -INFINITY; red_ml[wave][rho][1] = ln; }
    __syncthreads();
    const int r = tid >> 4, row = rb * 16 * NQ + 16 * n + r;
    if (row >= p.rows) continue;
    float mw[4], mt = -INFINITY, lt = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) { mw[w] = red_ml[w][r][0]; mt = fmaxf(mt, mw[w]); }
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      mw[w] = mw[w] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw[w] - mt);
      if (mw[w] != 0.f) lt = fmaf(mw[w], red_ml[w][r][1], lt);
    }
    const float f = p.nsplit > 1 ? 1.f : mt == -INFINITY ? 0.f : 1.0f / lt;
    const long long at0 = ((long long)split * p.B * p.kv_heads + head) * p.rows + row;
    const long long ld = (long long)p.kv_heads * p.group * D;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const int at = 64 * i + 4 * (tid & 15);
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w) v += mw[w] * *reinterpret_cast<const f32x4*>(red + (w * 16 + r) * ROW + at);
      v *= f;
      if (p.nsplit > 1) *reinterpret_cast<f32x4*>(p.part_o + at0 * D + at) = v;
      else *reinterpret_cast<u32x2*>((bf16_t*)p.out + row_offset(p, b, kh, row, (long long)p.Lq * ld, ld) + at) = u32x2{pack_bf2(v.x, v.y), pack_bf2(v.z, v.w)};
    }
    if (p.nsplit > 1 && (tid & 15) == 0) { p.part_ml[2 * at0] = mt; p.part_ml[2 * at0 + 1] = lt; }
  }
}

// ---- choice of kernel and splits, all from the arguments' sizes ----
enum { kRows, kFewKv4, kFloat };
struct Plan {
  int kind, nq;                                // nq: blocks of 16 rows (kFewKv4)
  int block, tile;                             // rows of a workgroup, keys of a tile
  int nsplit, tiles_per_split;
  size_t expand, parts;                        // bytes of the workspace: the cache's rows in bf16, the splits' parts
};

// `keys`: of both segments; `cached`: segment 0 is a 4-bit cache of whose rows `other` are not the patch's
Plan plan_of(int B, long long rows, int kv_heads, int d, long long keys0, long long keys1, bool cached, bool masked, int dtype) {
  Plan r = {};
  const long long heads = (long long)B * kv_heads;
  if (dtype == DF_F32) { r.kind = kFloat; r.block = 128; r.tile = 32; }
  else if (cached && keys1 == 0 && rows <= 64) { r.kind = kFewKv4; r.nq = rows > 16 ? 2 : 1; r.block = 16 * r.nq; r.tile = 64; }
  else { r.kind = kRows; r.block = d <= 64 ? 128 : 256; r.tile = 64; }
  const long long tiles = (keys0 + r.tile - 1) / r.tile + (keys1 + r.tile - 1) / r.tile;
  const long long blocks = heads * ((rows + r.block - 1) / r.block);
  long long ns = 1;
  const long long want = r.kind == kFewKv4 ? 768 : r.kind == kRows && d > 64 ? 256 : 512, least = r.kind == kFewKv4 ? 4 : 4;
  if (blocks < want) ns = want / blocks;
  if (ns > tiles / least) ns = tiles / least;
  if (ns < 1) ns = 1;
  if (ns > 64) ns = 64;
  if (masked && r.kind == kRows && ns < (tiles + kListTiles - 1) / kListTiles) ns = (tiles + kListTiles - 1) / kListTiles;
  r.tiles_per_split = (int)((tiles + ns - 1) / ns);
  r.nsplit = (int)((tiles + r.tiles_per_split - 1) / r.tiles_per_split);
  if (cached && r.kind == kRows) r.expand = (size_t)(heads * keys0 * d * 4 + 255) / 256 * 256;
  if (r.nsplit > 1) r.parts = (size_t)r.nsplit * heads * rows * (d + 2) * sizeof(float);
  return r;
}

template <int D, int NW>
int launch_rows(const QParams& p, bool masked, dim3 grid, hipStream_t st) {
  constexpr int smem = 6 * 64 * D * 2, list = kListTiles * 10 + 16;
  static const hipError_t set = [] {
    const hipError_t e = hipFuncSetAttribute((const void*)rows_attn<D, NW, true>, hipFuncAttributeMaxDynamicSharedMemorySize, smem + list);
    return e != hipSuccess ? e : hipFuncSetAttribute((const void*)rows_attn<D, NW, false>, hipFuncAttributeMaxDynamicSharedMemorySize, smem);
  }();
  if (set != hipSuccess) return DF_EHIP;
  if (masked) hipLaunchKernelGGL((rows_attn<D, NW, true>), grid, dim3(64 * NW), smem + list, st, p);
  else hipLaunchKernelGGL((rows_attn<D, NW, false>), grid, dim3(64 * NW), smem, st, p);
  return DF_OK;
}

}  // namespace

size_t qattn_workspace(int B, long long rows, int kv_heads, int d, long long keys0, long long keys1, bool cached, bool masked, int dtype) {
  const Plan r = plan_of(B, rows, kv_heads, d, keys0, keys1, cached, masked, dtype);
  return r.expand + r.parts;
}

int launch_qattn(const QAttnArgs& a, hipStream_t st) {
  const bool cached = a.cache != nullptr;
  const long long rows = (long long)a.Lq * (a.heads / a.kv_heads), own = a.own_period > 0 ? (long long)a.own_n * (a.L / a.own_period) : a.own_n;
  const long long keys0 = cached ? a.L - own : a.L;
  const Plan r = plan_of(a.B, rows, a.kv_heads, a.d, keys0, own, cached, a.mask != nullptr, a.dtype);
  if (rows > 0x7fffffffLL - 256 || (long long)a.B * a.kv_heads * rows * (a.d / 8) >= (1LL << 32) - 256) return DF_ESHAPE;
  if (a.workspace_bytes < r.expand + r.parts || (r.expand + r.parts && !a.workspace)) return DF_ENOMEM;
  QParams p = {};
  p.q = a.q; p.ldq = a.ldq; p.bsq = a.bsq; p.out = a.out;
  p.B = a.B; p.Lq = a.Lq; p.group = a.heads / a.kv_heads; p.kv_heads = a.kv_heads; p.d = a.d; p.rows = (int)rows;
  p.group_recip = reciprocal_u32((unsigned int)p.group);
  p.sc = a.scale * kLog2e;
  p.nsplit = r.nsplit; p.tiles_per_split = r.tiles_per_split;
  p.mask = a.mask; p.lens = a.lens;
  p.part_o = (float*)((char*)a.workspace + r.expand);
  p.part_ml = p.part_o + (size_t)r.nsplit * a.B * a.kv_heads * rows * a.d;
  if (cached) {
    p.c = kv4_view(a.cache, a.B, a.L, a.kv_heads, a.d);
    p.own_lo = a.own_lo; p.own_n = a.own_n; p.own_period = a.own_period;
    p.seg[0].n = r.kind == kRows ? (int)keys0 : a.L;
  } else {
    p.seg[0].n = a.L;
  }
  Seg& rows_seg = p.seg[cached ? 1 : 0];                   // the caller's rows: fresh ones beside a cache, else all
  rows_seg.k = a.k; rows_seg.v = a.v; rows_seg.ldk = a.ldk; rows_seg.ldv = a.ldv; rows_seg.bsk = a.bsk; rows_seg.bsv = a.bsv;
  rows_seg.hsk = rows_seg.hsv = a.d;
  if (cached) rows_seg.n = (int)own;
  const long long nwg = (rows + r.block - 1) / r.block * a.kv_heads * a.B * r.nsplit;
  if (nwg > 0x7fffffffLL) return DF_ESHAPE;
  const dim3 grid((unsigned)nwg);
  if (r.expand) {
    Kv4Args e = {};
    e.cache = const_cast<void*>(a.cache); e.B = a.B; e.L = a.L; e.kv_heads = a.kv_heads; e.d = a.d; e.dtype = DF_BF16;
    e.own_lo = a.own_lo; e.own_n = a.own_n; e.own_period = a.own_period;
    bf16_t *k = (bf16_t*)a.workspace, *v = k + (size_t)a.B * a.kv_heads * keys0 * a.d;
    const int rc = keys0 > 0 ? launch_kv4_expand(e, a.lens, keys0, k, v, st) : DF_OK;
    if (rc != DF_OK) return rc;
    Seg& s = p.seg[0];
    s.k = k; s.v = v; s.ldk = s.ldv = a.d; s.hsk = s.hsv = keys0 * a.d; s.bsk = s.bsv = keys0 * a.d * a.kv_heads;
  }
  if (r.kind == kFloat) {
    // (tiles of 32 keys; the cache's own rows stay among segment 0's and are masked)
    if (cached) {
      const long long tiles = cdiv(a.L, 32) + cdiv(own, 32);
      p.tiles_per_split = (int)((tiles + r.nsplit - 1) / r.nsplit);
    }
    if (cached && a.d == 64) hipLaunchKernelGGL((float_attn<64, true>), grid, dim3(256), 0, st, p);
    else if (cached) hipLaunchKernelGGL((float_attn<128, true>), grid, dim3(256), 0, st, p);
    else if (a.d <= 32) hipLaunchKernelGGL((float_attn<32, false>), grid, dim3(256), 0, st, p);
    else if (a.d <= 64) hipLaunchKernelGGL((float_attn<64, false>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((float_attn<128, false>), grid, dim3(256), 0, st, p);
  } else if (r.kind == kFewKv4) {
    if (a.d == 64 && r.nq == 1) hipLaunchKernelGGL((few_rows_kv4<64, 1>), grid, dim3(256), 0, st, p);
    else if (a.d == 64) hipLaunchKernelGGL((few_rows_kv4<64, 2>), grid, dim3(256), 0, st, p);
    else if (r.nq == 1) hipLaunchKernelGGL((few_rows_kv4<128, 1>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((few_rows_kv4<128, 2>), grid, dim3(256), 0, st, p);
  } else {
    const int rc = a.d <= 64 ? launch_rows<64, 4>(p, a.mask != nullptr, grid, st) : launch_rows<128, 8>(p, a.mask != nullptr, grid, st);
    if (rc != DF_OK) return rc;
  }
  DF_LAUNCH_CHECK();
  if (r.nsplit > 1) {
    const unsigned int per_row = (unsigned int)(a.d / 8), total = (unsigned int)((long long)a.B * a.kv_heads * rows * per_row);
    const dim3 g((total + 255) / 256);
    if (a.dtype == DF_F32) hipLaunchKernelGGL(merge_splits<float>, g, dim3(256), 0, st, p, per_row, reciprocal_u32(per_row), total, reciprocal_u32((unsigned int)rows), reciprocal_u32((unsigned int)a.kv_heads));
    else hipLaunchKernelGGL(merge_splits<bf16_t>, g, dim3(256), 0, st, p, per_row, reciprocal_u32(per_row), total, reciprocal_u32((unsigned int)rows), reciprocal_u32((unsigned int)a.kv_heads));
    DF_LAUNCH_CHECK();
  }
  return DF_OK;
}

}  // namespace df
