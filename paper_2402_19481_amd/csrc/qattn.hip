// Attention of a patch's queries to rows of another length (an encoder's states) and to a 4-bit cache with the patch's own rows fresh
// (Section 4, Sparse operations: the keys and values are a scatter output; softmax does not ask for their order, so the cache's rows without
// the patch's own, and the fresh ones, are two segments of one sum).
//
//   out = softmax(q k^T * scale) v per head, one pass over the keys with the running maximum and sum.  `group` query heads share a key head;
//   they are rows of one problem: row r of a key head is query r / group, head r % group of the group, so shared keys are read once.
//
// bf16: S^T = K Q^T and O^T = V^T P^T on v_mfma_f32_32x32x16_bf16 (a lane owns one row of queries; the exponentiated accumulators of S^T are,
// by the order in which keys are assigned to its rows, the operand P^T without any data movement).  P is rounded to bf16 as the matrix
// instruction takes it (by 2^-8 of a weight at most, averaged over the keys); sums, maxima and O are float, the row sums are those of the float weights.
// float: the same on v_mfma_f32_32x32x2_f32, for the small full-precision networks.
#include <cstring>

#include "kv4.h"

namespace df {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLow = -3.0e38f;               // a running maximum before the first score: finite, so that -inf scores have weight 0
#define DF_INLINE __attribute__((always_inline))

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

// ---- bf16 rows ----
// A workgroup is four waves of QB * 32 rows.  The work is a line of tiles of 64 keys, block of rows by block of rows; workgroup w takes the w-th of
// equal shares of it (`Share`), so all end together whatever the number of blocks: a share that covers a block writes its result, one that
// begins or ends inside a block leaves a part (running maximum, sum, O in float) for merge_shares.
struct Share {
  unsigned int tiles, count, per, more, all;   // tiles of a block; shares; each `per` tiles, the first `more` one more, the last what is left of all
};
__host__ __device__ inline unsigned int share_begin(const Share& s, unsigned int w) {
  const unsigned int t = w * s.per + (w < s.more ? w : s.more);
  return t < s.all ? t : s.all;
}
__host__ __device__ inline unsigned int share_of(const Share& s, unsigned int tile) {
  const unsigned int big = s.more * (s.per + 1);
  return tile < big ? tile / (s.per + 1) : s.more + (tile - big) / s.per;
}

// Where lengths (or the number of rows that a mask leaves) are known on the device only, the shares are those of the longest batch item: as many as
// planned, of the keys there are.
__device__ __forceinline__ Share share_of_keys(const QParams& p, Share s, int nrb) {
  if (!p.lens || p.B > 1024) return s;                     // (of many batch items some have work while others have none)
  int longest = 0;
  for (int b = threadIdx.x & 63; b < p.B; b += 64) longest = max(longest, seg0_rows(p, b));
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) longest = max(longest, __shfl_xor(longest, o, 64));
  longest = __builtin_amdgcn_readfirstlane(longest);
  const unsigned int tiles = (unsigned int)(((longest + 63) >> 6) + ((p.seg[1].n + 63) >> 6)), planned = s.tiles;
  s.tiles = tiles > 0 ? tiles : 1;
  s.all = s.tiles * (unsigned int)(nrb * p.kv_heads * p.B);
  if (s.more == 0 && s.per % planned == 0) s.per = s.per / planned * s.tiles;      // whole blocks
  else { s.per = s.all / s.count; s.more = s.all % s.count; }
  return s;
}

// The loop is software-pipelined inside the wave, since matrix instructions and the softmax's vector instructions of a SIMD overlap only where one
// wave's stream mixes them: iteration t issues S_{t+1} = K_{t+1} Q^T and O += V_{t-1} P_{t-1} between the exponentials of tile t, whose registers
// take S_{t+1} as they come free.  K and V tiles go memory -> LDS by direct loads, K_{t+3} and V_{t+1} in iteration t, to rings of four slots (so
// that K_t is there to the end of iteration t, and all slots follow from one number).  With one wave on a SIMD every instruction takes its time
// slot, scalar ones too: runs of whole tiles of one segment go through a loop that only moves its pointers on.
// Many keys: bound by instruction issue: of a tile's 1460 cycles (64 values; 215 instructions) the matrix unit works 512, and a second workgroup on the
// unit adds 16 %.  7200 queries, 10 heads of 64: 5120 keys 124 us (0.76 PFLOP/s), 57600 rows of a cache 1065 - 1220 (0.87 - 1.0); 16384 queries, 16 heads
// of 128 on 2048 keys 300 us (0.92), on 512 keys with a mask 112 - 114 (six or seven tiles a block, whose beginning and end take the time of five).
// With fewer keys that is not all of it: 1200 queries on 9600 rows, 10 heads of 64, take 49 - 51 us (two workgroups on every unit, equal shares,
// ending after 30 - 33 and 40 - 44), attn_pipe_d64 on as many rows of bf16 37.  That one has V transposed in memory (8 plain reads of LDS a tile for 16
// transposing ones, a third of whose cycles are conflicts here) and its queries scaled, which saves 32 of the vector instructions.
// The running maximum is that of the first tile and moves when a row's weights of a tile sum to more than 2^13 (the sums are needed anyway; the
// maximum of every tile would be 22 instructions more): by the power of two above the sum, which scales the packed weights exactly, or, beyond 2^100,
// to the tile's own maximum, with the tile done again from its K in LDS.
template <int D, int QB>
__global__ __launch_bounds__(256, D == 64 && QB == 1 ? 2 : 1) void rows_attn(QParams p, Share planned) {
  constexpr int TILE = 64 * D * 2, CH = D / 8, KS = D / 16, DB = D / 32, LPT = TILE / 4096, RPI = 1024 / (D * 2), M = D / 64, BLK = 128 * QB;
  extern __shared__ __attribute__((aligned(16))) char smem[];             // four K tiles, four V tiles
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, c = lane & 31, csig = (c & 0x13) | ((c & 4) << 1) | ((c & 8) >> 1), tri = lane & 15;
  const int nrb = (p.rows + BLK - 1) / BLK;
  const Share sh = share_of_keys(p, planned, nrb);
  unsigned int w;
  {
    const unsigned int t = blockIdx.x, xcd = t & 7, base = sh.count >> 3, rem = sh.count & 7;   // an XCD takes shares side by side: the same keys
    w = xcd * base + (xcd < rem ? xcd : rem) + (t >> 3);
  }
  unsigned int pos = share_begin(sh, w);
  const unsigned int end = share_begin(sh, w + 1);
  if (pos >= end) return;                                  // fewer tiles than shares were planned: no block, and no batch item, is its
  // Direct load j of the wave covers tile rows (LPT wave + j) * RPI + lane / CH; the chunks of a row are swizzled by it.  (K and V have D
  // values a row; where d is less they are zeros, Q is too, those of O are dropped.)
  unsigned int kch[LPT], vch[LPT];
  int trow[LPT];
#pragma unroll
  for (int j = 0; j < LPT; ++j) {
    const int r = (wave * LPT + j) * RPI + lane / CH, at = lane % CH;
    const int kc = (at ^ (D == 64 ? (r >> 1) & 7 : r & 15)) * 8;
    const int vc = (at ^ (D == 64 ? ((r >> 1) & 1) * 2 ^ ((r >> 3) & 1) * 4 : (r & 3) * 4)) * 8;
    trow[j] = r;
    kch[j] = 2 * kc;
    vch[j] = 2 * vc;
  }
  auto slot_of = [&](int i) DF_INLINE { return (i & 3) * TILE; };
  constexpr int VR = 4 * TILE;                             // the ring of V
  const int wofs = 1024 * LPT * wave;
  // LDS offsets of this lane's operands in a tile: chunk 2 s + g of MFMA row c, which is key csig (the second block of keys is 32 rows on); four keys
  // of 16 values for the transposing reads (the lane's chunks 1 and 2 exchanged, so that O's rows come out in the order of csig too)
  const int kof = csig * (D * 2) + ((g ^ (D == 64 ? (csig >> 1) & 7 : csig & 15)) * 16);
  int vof[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    const int key = 8 * g + (tri >> 2), chunk = 4 * db + 2 * ((lane >> 4) & 1) + (tri & 1);
    const int pc = D == 64 ? chunk ^ (2 * ((key >> 1) & 1)) ^ (4 * ((key >> 3) & 1)) : chunk ^ ((key & 3) * 4);
    vof[db] = key * (D * 2) + pc * 16 + ((tri >> 1) & 1) * 8;
  }
  auto kfrag = [&](int at, int s, int kb) DF_INLINE { return *reinterpret_cast<const u32x4*>(smem + (at + (kof ^ (32 * s))) + kb * 32 * D * 2); };
  auto vfrag = [&](int slot, int ts, int db) DF_INLINE {
    typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
    const char* at = smem + (slot + vof[db]) + VR + ts * 16 * D * 2;
    const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(at));
    const bf16x4 z = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(at + 4 * D * 2));
    const u32x2 a2 = __builtin_bit_cast(u32x2, a), z2 = __builtin_bit_cast(u32x2, z);
    return u32x4{a2.x, a2.y, z2.x, z2.y};
  };
  auto sync_tile = [&]() DF_INLINE {                                   // all but the last iteration's loads have landed, and its reads are done, for every wave
    __builtin_amdgcn_s_waitcnt((2 * LPT) | (0x7 << 4) | (0 << 8));
    block_sync();
  };

  // A block of rows (or the share's part of one)
  struct Block { int kh, b, row0, lo, nt, n0, tiles0; bool whole; };
  int lo0 = (int)(pos % sh.tiles), rb, kh0, b0, n00;       // of the next one: its first tile, place, keys of segment 0
  {
    const unsigned int block = pos / sh.tiles, bh = block / (unsigned int)nrb;
    rb = (int)(block - bh * nrb);
    b0 = (int)(bh / (unsigned int)p.kv_heads);
    kh0 = (int)(bh - (unsigned int)b0 * p.kv_heads);
    n00 = b0 < p.B ? seg0_rows(p, b0) : 0;
  }
  auto open = [&]() DF_INLINE {
    Block r;
    r.lo = lo0;
    int hi = (int)(r.lo + end - pos < sh.tiles ? r.lo + end - pos : sh.tiles);
    pos += hi - r.lo;
    r.whole = r.lo == 0 && hi == (int)sh.tiles;
    r.row0 = rb * BLK + wave * 32 * QB;
    r.b = b0;
    r.kh = kh0;
    r.n0 = n00;
    r.tiles0 = (r.n0 + 63) >> 6;
    if (hi > r.tiles0 + ((p.seg[1].n + 63) >> 6)) hi = r.tiles0 + ((p.seg[1].n + 63) >> 6);
    r.nt = hi > r.lo ? hi - r.lo : 0;
    lo0 = 0;
    if (++rb == nrb) {
      rb = 0;
      if (++kh0 == p.kv_heads) {
        kh0 = 0;
        ++b0;
        if (pos < end) n00 = seg0_rows(p, b0);
      }
    }
    return r;
  };
  bf16x8 qreg[QB][KS], qnext[QB][KS];
  auto queries = [&](const Block& k) DF_INLINE {           // the wave's rows of Q -> qnext (behind the last row it is read again, and not used)
#pragma unroll
    for (int n = 0; n < QB; ++n) {
      const int row = k.row0 + 32 * n + c;
      const bf16_t* qp = (const bf16_t*)p.q + row_offset(p, k.b, k.kh, row < p.rows ? row : p.rows - 1, p.bsq, p.ldq);
#pragma unroll
      for (int s = 0; s < KS; ++s)
        qnext[n][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qp + (p.d == D || 16 * s + 8 * g < p.d ? 16 * s + 8 * g : 0)));
    }
  };
  // What is loaded next: the rows of a tile's K and V, the keys and the tiles from it on in its segment (and the block's tiles in segment 1 behind
  // it), all in scalar registers; and what was loaded before: the keys (and 256 if segment 1's) of tiles t .. t + 2 of an iteration, V of t + 1, t + 2.
  const char *fk = nullptr, *fv = nullptr, *v1 = nullptr, *v2 = nullptr;
  long long kstep = 0, vstep = 0;
  int left = 0, tiles = 0, rest = 0, w0 = 0, w1 = 0, w2 = 0, kw = 0, vw = 0;
  bool second = false, beyond = false;                     // ... is segment 1's; is in the next block
  unsigned int kofs[LPT], vofs[LPT];                       // a lane's offsets in a tile of kw and vw keys
  auto feed = [&](int kh, int b, int z, int tile, int n, int count) DF_INLINE {
    const Seg& s = p.seg[z];
    kstep = 128 * s.ldk; vstep = 128 * s.ldv;
    fk = (const char*)s.k + 2 * ((long long)b * s.bsk + (long long)kh * s.hsk) + tile * kstep;
    fv = (const char*)s.v + 2 * ((long long)b * s.bsv + (long long)kh * s.hsv) + tile * vstep;
    left = n - tile * 64; tiles = count; second = z;
  };
  auto feed_block = [&](const Block& k) DF_INLINE {
    const int kh = k.kh, b = k.b, lo = k.lo, nt = k.nt, n0 = k.n0, tiles0 = k.tiles0;
    if (lo < tiles0) {
      const int some = tiles0 - lo < nt ? tiles0 - lo : nt;
      feed(kh, b, 0, lo, n0, some);
      rest = nt - some;
    } else {
      feed(kh, b, 1, lo - tiles0, p.seg[1].n, nt);
      rest = 0;
    }
  };
  auto offsets = [&](auto isv, int word, unsigned int (&ofs)[LPT]) DF_INLINE {
    constexpr bool V = decltype(isv)::value;
    const Seg& s = p.seg[word >> 8];
    const int ld = (int)(V ? s.ldv : s.ldk), last = (word & 255) - 1;
#pragma unroll
    for (int j = 0; j < LPT; ++j) {                        // behind the last key its row is read again: the weight is 0, the value must be finite
      ofs[j] = 2u * (unsigned int)((trow[j] < last ? trow[j] : last) * ld) + (V ? vch[j] : kch[j]);   // where the others are
      asm volatile("" : "+v"(ofs[j]));
    }
  };
  auto load = [&](const char* base, const unsigned int (&ofs)[LPT], int j, int to) DF_INLINE { lds_load16(base, ofs[j], smem + to + 1024 * j); };
  using IsK = std::false_type;
  using IsV = std::true_type;

  Block blk = open(), after = blk;
  bool primed = false;                                     // the last block's final iterations have requested this one's first tiles and Q
  int s0 = 0;                                              // slot of its tile 0
  for (bool more = true; more;) {
    more = pos < end;
    if (more) after = open();
    if (!primed) queries(blk);
    const int nt = blk.nt, ant = after.nt;
    // The next block's first tiles follow this one's last (of which a block that was itself begun ahead has three at least: the slots behind a
    // shorter one hold its last tile again)
    const bool ahead = more && nt > 0 && ant > 0 && (!primed || nt >= 3);
    const int lo = blk.lo, n0 = blk.n0, n1 = p.seg[1].n, tiles0 = blk.tiles0, b = blk.b, kh = blk.kh, row0 = blk.row0;
    const bool whole = blk.whole, idle = row0 >= p.rows;
    const unsigned int slot = 2 * w + (lo == 0 ? 1 : 0);
    f32x16 o[QB][DB], sa[QB][2];
    u32x4 pk[QB][4];
    float m[QB], l[QB];
#pragma unroll
    for (int n = 0; n < QB; ++n) {
#pragma unroll
      for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[n][i][e] = 0.f;
      m[n] = kLow; l[n] = 0.f;
    }
    auto s_mfma = [&](u32x4 k, int s, int kb, int n) DF_INLINE {
      if (s == 0) {
#pragma unroll
        for (int e = 0; e < 16; ++e) sa[n][kb][e] = 0.f;
      }
      sa[n][kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), qreg[n][s], sa[n][kb], 0, 0, 0);
    };
    auto pv_mfma = [&](u32x4 v, int ts, int db, int n) DF_INLINE {
      o[n][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, pk[n][ts]), o[n][db], 0, 0, 0);
    };
    auto scores = [&](int i) DF_INLINE {
      const int kt = slot_of(s0 + i);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const u32x4 k = kfrag(kt, s, kb);
#pragma unroll
          for (int n = 0; n < QB; ++n) s_mfma(k, s, kb, n);
        }
    };
    auto hide = [&](int word) DF_INLINE {                            // scores behind the last key
      if ((word & 255) == 64) return;
      const unsigned long long bits = low_bits(word & 255);
      const unsigned long long mine = bits >> (8 * g);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const bool off = !((mine >> (32 * kb + 16 * (e >> 3) + (e & 7))) & 1);
#pragma unroll
          for (int n = 0; n < QB; ++n)
            if (off) sa[n][kb][e] = -INFINITY;
        }
    };
    auto scale_by = [&](int n, float f) DF_INLINE {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[n][db][e] *= f;
      l[n] *= f;
    };
    auto settle = [&](int n) DF_INLINE {                             // the maximum that covers the scores in sa too; the factor for what came before
      float top = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, sa[n][kb][e]);
      top = fmaxf(top, __shfl_xor(top, 32, 64)) * p.sc;
      const float mn = fmaxf(m[n], top), alpha = __builtin_amdgcn_exp2f(m[n] - mn);
      m[n] = mn;
      return alpha;
    };

    // Iteration t: weights of tile t from the scores in sa, O += V P of tile t - 1 (PV), S of tile t + 1.  Sixteen slots of M * QB matrix
    // instructions and their share of the vector instructions; operands are read from LDS some slots ahead.
    const char *ka = nullptr, *va = nullptr;               // of K_{t+3} and V_{t+1}
    float tsum[QB];
    int x = 0;                                             // slot of tile t + 1; tile t - 1's, which tile t + 3 takes, is two from it
    auto tile = [&](auto pvc) DF_INLINE {
      constexpr bool PV = decltype(pvc)::value;
      constexpr int A = M == 1 ? 4 : 3;
      //                          slot: 0  1  2  3  4  5  6  7  8  9 10 11 12 13 14 15; of S (kb, quarter), of O (key step, half)
      constexpr int kIsS[16] =       {0, 0, 0, 0, 0, 0, 1, 0, 1, 0, 1, 1, 1, 1, 1, 1};
      constexpr int kFirst[16] =     {0, 0, 1, 1, 2, 2, 0, 3, 0, 3, 0, 0, 1, 1, 1, 1};
      constexpr int kSecond[16] =    {0, 1, 0, 1, 0, 1, 0, 0, 1, 1, 2, 3, 0, 1, 2, 3};
      const int kt = x, vt = x ^ (2 * TILE), kd = (x ^ (2 * TILE)) + wofs, vd = VR + x + wofs;
      u32x4 f[16][M];
      float ex[QB][2][8];
      auto fetch = [&](int i) DF_INLINE {
#pragma unroll
        for (int k = 0; k < M; ++k) {
          if (kIsS[i]) f[i][k] = kfrag(kt, kSecond[i] * M + k, kFirst[i]);
          else if (PV) f[i][k] = vfrag(vt, kFirst[i], kSecond[i] * M + k);
        }
      };
      auto E = [&](int u, int h) DF_INLINE {                         // four exponentials of key step u
#pragma unroll
        for (int n = 0; n < QB; ++n)
#pragma unroll
          for (int q = 0; q < 4; ++q) ex[n][u & 1][4 * h + q] = __builtin_amdgcn_exp2f(fmaf(sa[n][u >> 1][8 * (u & 1) + 4 * h + q], p.sc, -m[n]));
      };
      auto C = [&](int u) DF_INLINE {                                // packing, behind the matrix instructions that read the old pk[u]
#pragma unroll
        for (int n = 0; n < QB; ++n) {
          const float* x = ex[n][u & 1];
          pk[n][u] = u32x4{pack_bf2(x[0], x[1]), pack_bf2(x[2], x[3]), pack_bf2(x[4], x[5]), pack_bf2(x[6], x[7])};
          asm volatile("" : "+v"(pk[n][u]));
        }
      };
      auto S = [&](int u) DF_INLINE {                                // row sums
#pragma unroll
        for (int n = 0; n < QB; ++n) {
          const float* x = ex[n][u & 1];
          const float s = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
          tsum[n] = u == 0 ? s : tsum[n] + s;
          asm volatile("" : "+v"(tsum[n]));
        }
      };
#pragma unroll
      for (int i = 0; i < A; ++i) fetch(i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
#pragma unroll
        for (int k = 0; k < M; ++k)
#pragma unroll
          for (int n = 0; n < QB; ++n) {
            if (kIsS[i]) s_mfma(f[i][k], kSecond[i] * M + k, kFirst[i], n);
            else if (PV) pv_mfma(f[i][k], kFirst[i], kSecond[i] * M + k, n);
          }
        if (i + A < 16) fetch(i + A);
        switch (i) {
          case 0: E(0, 0); break;
          case 1: E(0, 1); load(ka, kofs, 0, kd); break;
          case 2: C(0); load(ka, kofs, 1, kd); break;
          case 3: E(1, 0); break;
          case 4: E(1, 1); break;
          case 5: C(1); S(0); break;
          case 6: E(2, 0); if constexpr (LPT > 2) load(ka, kofs, 2, kd); break;
          case 7: E(2, 1); S(1); break;
          case 8: C(2); load(va, vofs, 0, vd); break;
          case 9: E(3, 0); break;
          case 10: E(3, 1); load(va, vofs, 1, vd); break;
          case 11: S(2); if constexpr (LPT > 2) load(ka, kofs, 3, kd); break;
          case 12: C(3); if constexpr (LPT > 2) load(va, vofs, 2, vd); break;
          case 13: S(3); break;
          case 14: if constexpr (LPT > 2) load(va, vofs, 3, vd); break;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    constexpr float kMove = 0x1p13f, kRedo = 0x1p100f;
    auto large = [&](int t) DF_INLINE {                              // a tile whose sums are far above 1 somewhere
      bool redo = false;
#pragma unroll
      for (int n = 0; n < QB; ++n) redo |= __builtin_amdgcn_ballot_w64(tsum[n] > kRedo) != 0;
      if (redo) {
        scores(t);
        hide(w0);
#pragma unroll
        for (int n = 0; n < QB; ++n) {
          scale_by(n, settle(n));
          tsum[n] = 0.f;
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              x[e] = __builtin_amdgcn_exp2f(fmaf(sa[n][u >> 1][8 * (u & 1) + e], p.sc, -m[n]));
              tsum[n] += x[e];
            }
            pk[n][u] = u32x4{pack_bf2(x[0], x[1]), pack_bf2(x[2], x[3]), pack_bf2(x[4], x[5]), pack_bf2(x[6], x[7])};
          }
        }
        scores(t + 1);
        return;
      }
#pragma unroll
      for (int n = 0; n < QB; ++n) {
        const float both = fmaxf(tsum[n], __shfl_xor(tsum[n], 32, 64));
        const int k = both > kMove ? __builtin_amdgcn_frexp_expf(both) : 0;
        const float f = __builtin_amdgcn_ldexpf(1.0f, -k);
        m[n] += (float)k;
        scale_by(n, f);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float a = __uint_as_float(pk[n][u][q] << 16) * f, z = __uint_as_float(pk[n][u][q] & 0xffff0000u) * f;
            pk[n][u][q] = (__float_as_uint(a) >> 16) | (__float_as_uint(z) & 0xffff0000u);
          }
        tsum[n] *= f;
      }
    };

    if (nt > 0) {
      // The next tile to load; past the block's end the next block's, or the last one again, which keeps the counts of loads in flight uniform
      int w3 = 0;
      const char* v3 = nullptr;
      auto take = [&]() DF_INLINE {
        if (tiles == 0) {
          if (rest > 0) {
            const Block& of = beyond ? after : blk;
            const int kh1 = of.kh, b1 = of.b, some = rest;
            feed(kh1, b1, 1, 0, n1, some);
            rest = 0;
          } else if (!beyond && ahead) {
            feed_block(after);
            beyond = true;
          }
        }
        if (tiles > 0) {
          ka = fk; v3 = fv;
          w3 = (left < 64 ? left : 64) | (second ? 256 : 0);
          fk += kstep; fv += vstep;
          left -= 64; --tiles;
        } else {
          ka = fk - kstep; v3 = v2; w3 = w2;
        }
        if (w3 != kw) { kw = w3; offsets(IsK{}, w3, kofs); }
      };
      auto next = [&]() DF_INLINE { w0 = w1; w1 = w2; w2 = w3; v1 = v2; v2 = v3; };
      if (!primed) {
        s0 = 0;
        kw = vw = 0;
        beyond = false;
        feed_block(blk);
        block_sync();                                      // (every wave's reads of the last block are done: they were waited for)
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          take();
#pragma unroll
          for (int j = 0; j < LPT; ++j) load(ka, kofs, j, slot_of(i) + wofs);
          if (i == 0) {
            va = v3;
            vw = w3;
            offsets(IsV{}, vw, vofs);
          }
          next();
        }
#pragma unroll
        for (int j = 0; j < LPT; ++j) load(va, vofs, j, VR + wofs);
        sync_tile();
      }
#pragma unroll
      for (int n = 0; n < QB; ++n)
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          qreg[n][s] = qnext[n][s];
          asm volatile("" : "+v"(qreg[n][s]));             // Q has arrived: the loop does not wait for it, with the direct loads
          if (p.d != D && 16 * s + 8 * g >= p.d) qreg[n][s] = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
        }
      // an iteration's loads, and at the last one the next block's Q
      auto begin = [&](int t) DF_INLINE {
        take();
        va = v1;
        if (w1 != vw) { vw = w1; offsets(IsV{}, vw, vofs); }
        if (t == nt - 1 && ahead) queries(after);
      };
      if (idle) {
        for (int t = 0; t < nt; ++t) {
          begin(t);
#pragma unroll
          for (int j = 0; j < LPT; ++j) load(ka, kofs, j, slot_of(s0 + t + 3) + wofs);
#pragma unroll
          for (int j = 0; j < LPT; ++j) load(va, vofs, j, VR + slot_of(s0 + t + 1) + wofs);
          next();
          sync_tile();
        }
      } else {
        auto finish = [&](int t) DF_INLINE {               // of an iteration
          float most = tsum[0];
          if constexpr (QB == 2) most = fmaxf(most, tsum[1]);
          if (__builtin_expect(__builtin_amdgcn_ballot_w64(most > kMove) != 0, 0)) large(t);
#pragma unroll
          for (int n = 0; n < QB; ++n) l[n] += tsum[n];
          x = (x + TILE) & (3 * TILE);
          sync_tile();
        };
        scores(0);
        hide(w0);
#pragma unroll
        for (int n = 0; n < QB; ++n) settle(n);
        begin(0);
        x = slot_of(s0 + 1);
        tile(std::false_type{});
#pragma unroll
        for (int n = 0; n < QB; ++n) l[n] += tsum[n];      // (weights of at most 1)
        x = slot_of(s0 + 2);
        next();
        sync_tile();
        int t = 1;
        while (t < nt) {
          // Tiles t .. t + 3 whole and of one segment: as long as that holds.  (Without a scope of their own its values spill.)
          {
            int run = tiles < left >> 6 ? tiles : left >> 6;
            if (run > nt - 1 - t) run = nt - 1 - t;
            const int whole = second ? 320 : 64;
            if (run > 0 && w0 == whole && w1 == whole && w2 == whole && kw == whole && vw == whole) {
              left -= 64 * run; tiles -= run;
              const int to = t + run;
              do {
                ka = fk; va = v1;
                tile(std::true_type{});
                v1 = v2; v2 = fv;
                fk += kstep; fv += vstep;
                finish(t);
                ++t;
              } while (t < to);
              continue;
            }
          }
          begin(t);
          hide(w0);
          tile(std::true_type{});
          finish(t);
          next();
          ++t;
        }
        const int vt = slot_of(s0 + nt - 1);
#pragma unroll
        for (int ts = 0; ts < 4; ++ts)
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            const u32x4 v = vfrag(vt, ts, db);
#pragma unroll
            for (int n = 0; n < QB; ++n) pv_mfma(v, ts, db, n);
          }
      }
      // V has been read; no direct load outlives the wave, or its slot's part in the ring where the next block starts one of its own
      if (ahead) __builtin_amdgcn_s_waitcnt(0xc07f);
      else __builtin_amdgcn_s_waitcnt(0x0070);
      s0 = (s0 + nt) & 3;
    }
    primed = ahead;
    beyond = false;
#pragma unroll
    for (int n = 0; n < QB; ++n) {
      if (row0 + 32 * n + c >= p.rows) continue;
      const float lt = l[n] + __shfl_xor(l[n], 32, 64);
      const float inv = !whole ? 1.f : nt > 0 ? 1.0f / lt : 0.f;          // no key: zeros (all scores -inf: 0 / 0, as the formula)
      const int at0 = wave * 32 * QB + 32 * n + c;
      bf16_t* op = (bf16_t*)p.out + row_offset(p, b, kh, row0 + 32 * n + c, (long long)p.Lq * p.kv_heads * p.group * p.d, (long long)p.kv_heads * p.group * p.d);
      float* po = p.part_o + ((long long)slot * BLK + at0) * p.d;
      auto store = [&](auto wholec, auto fullc) DF_INLINE {  // (branches outside: straight code; of 256 rows two forms, with three the loop has 16 moves more)
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int f = 0; f < 2; ++f) {
            const int at = 32 * db + 16 * f + 8 * g;
            if (!decltype(fullc)::value && at >= p.d) continue;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = o[n][db][8 * f + e] * inv;
            if (decltype(wholec)::value) {
              st_vec(op + at, v);
            } else {
              st_vec(po + at, v);
              st_vec(po + at + 4, v + 4);
            }
          }
      };
      if (QB == 1 && whole && p.d == D) store(std::true_type{}, std::true_type{});
      else if (whole) store(std::true_type{}, std::false_type{});
      else store(std::false_type{}, std::false_type{});
      if (!whole && g == 0) {
        float* ml = p.part_ml + 2 * ((long long)slot * BLK + at0);
        ml[0] = nt > 0 ? m[n] : -INFINITY;
        ml[1] = lt;
      }
    }
    blk = after;
  }
}

// n parts of a row, in order, eight values of it from `at` on; part i lies in row where(i).  Four at a time are requested at once: one after the other
// each waits for memory.
template <typename F>
__device__ __forceinline__ void merge_parts(const QParams& p, int n, int at, F where, float& m, float& l, float (&o)[8]) {
  for (int i0 = 0; i0 < n; i0 += 4) {
    f32x2 ml[4];
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long r = where(i0 + i < n ? i0 + i : n - 1);
      ml[i] = *reinterpret_cast<const f32x2*>(p.part_ml + 2 * r);
      ld_vec(p.part_o + r * p.d + at, v[i]);
      ld_vec(p.part_o + r * p.d + at + 4, v[i] + 4);
    }
    float mn = m;
#pragma unroll
    for (int i = 0; i < 4; ++i) mn = fmaxf(mn, ml[i].x);   // (the last one again where there are fewer: no other maximum)
    if (mn == -INFINITY) continue;
    const float f = __builtin_amdgcn_exp2f(m - mn);        // 0 at first
    m = mn;
    l *= f;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] *= f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i0 + i >= n || ml[i].x == -INFINITY) continue;   // (a part without keys)
      const float w = __builtin_amdgcn_exp2f(ml[i].x - m);
      l = fmaf(w, ml[i].y, l);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = fmaf(w, v[i][e], o[e]);
    }
  }
}

// The parts of a block that shares cut: its first share's (slot 2 w + 1), then those of the shares that begin inside it (slot 2 w), in that order.
// Eight values of a row per lane.  1200 rows of 10 heads of 64, 512 shares: 5.6 us.
__global__ __launch_bounds__(256) void merge_shares(QParams p, Share planned, int blk, unsigned int per_row) {
  const unsigned int nrb = (unsigned int)(p.rows + blk - 1) / blk, block = blockIdx.x;
  const Share sh = share_of_keys(p, planned, (int)nrb);
  const unsigned int w0 = share_of(sh, block * sh.tiles), w1 = share_of(sh, block * sh.tiles + sh.tiles - 1);
  if (w0 == w1) return;
  const unsigned int idx = blockIdx.y * 256 + threadIdx.x;
  const int r = (int)(idx / per_row), at = (int)(idx - r * per_row) * 8;
  const int bh = (int)(block / nrb), b = bh / p.kv_heads, kh = bh - b * p.kv_heads, row = (int)(block % nrb) * blk + r;
  if (r >= blk || row >= p.rows) return;
  float m = -INFINITY, l = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  merge_parts(p, (int)(w1 - w0 + 1), at, [&](int i) DF_INLINE { return (long long)(i == 0 ? 2 * w0 + 1 : 2 * (w0 + i)) * blk + r; }, m, l, o);
  const float inv = m == -INFINITY ? 0.f : 1.0f / l;       // no key in any part: zeros
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] *= inv;
  const long long ld = (long long)p.kv_heads * p.group * p.d;
  st_vec((bf16_t*)p.out + row_offset(p, b, kh, row, (long long)p.Lq * ld, ld) + at, o);
}

// Rows of segment 0 that the mask (and the length) leaves, side by side per head, with zeros behind their d values, and how many they are per batch
// item: the pipelined loop then has whole tiles of keys, and none for what is masked (its own words and biases per tile cost it 20 us of 150 at 7200
// queries, 5120 keys, 10 heads of 64, with every key there).  A workgroup copies those of 64 rows of a head; it counts the ones before them itself.
// Bound by memory: 512 rows of 8 heads of 128 take 5.5 us (the launch is 3 of them).  The counting grows with the square of the rows: one query, 100000
// keys, 8 heads of 64: 146 - 161 us with a mask, 53 without.
__global__ __launch_bounds__(256) void keep_rows(QParams p, int tiles, bf16_t* ko, bf16_t* vo, int* counts) {
  __shared__ int before[4];
  __shared__ unsigned long long word;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tile = (int)(blockIdx.x % tiles), bh = (int)(blockIdx.x / tiles), b = bh / p.kv_heads, kh = bh - b * p.kv_heads;
  const int n = p.seg[0].n, n0 = seg0_rows(p, b);
  const unsigned char* mask = p.mask ? p.mask + (long long)b * n : nullptr;
  const int row0 = tile * 64, upto = row0 < n0 ? row0 : n0;
  int mine = 0;
  if (mask) {
    for (int i = tid * 16; i + 16 <= upto; i += 4096) {
      unsigned int x[4];
      __builtin_memcpy(x, mask + i, 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) mine += __popc((((x[e] & 0x7f7f7f7fu) + 0x7f7f7f7fu) | x[e]) & 0x80808080u);      // bytes that are not 0
    }
    if (tid < (upto & 15)) mine += mask[(upto & ~15) + tid] != 0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o, 64);
  }
  if (lane == 0) before[wave] = mine;
  if (wave == 0) {
    const unsigned long long w = __builtin_amdgcn_ballot_w64(row0 + lane < n0 && (!mask || mask[row0 + lane] != 0));
    if (lane == 0) word = w;
  }
  __syncthreads();
  const int first = mask ? before[0] + before[1] + before[2] + before[3] : upto;
  const unsigned long long w = word;
  if (tile == tiles - 1 && kh == 0 && tid == 0) counts[b] = first + __popcll(w);
  const Seg& s = p.seg[0];
  const bf16_t* k = (const bf16_t*)s.k + (long long)b * s.bsk + (long long)kh * s.hsk;
  const bf16_t* v = (const bf16_t*)s.v + (long long)b * s.bsv + (long long)kh * s.hsv;
  const long long to0 = ((long long)b * p.kv_heads + kh) * n + first;
  const int D = p.d <= 64 ? 64 : 128;
  for (int i = tid; i < 8 * D; i += 256) {
    const int r = i / (D / 8), at = (i - r * (D / 8)) * 8;
    if (!((w >> r) & 1)) continue;
    const long long to = (to0 + __popcll(w & low_bits(r))) * D + at;
    u32x4 a = {0u, 0u, 0u, 0u}, z = a;
    if (at < p.d) {
      a = *reinterpret_cast<const u32x4*>(k + (row0 + r) * s.ldk + at);
      z = *reinterpret_cast<const u32x4*>(v + (row0 + r) * s.ldv + at);
    }
    *reinterpret_cast<u32x4*>(ko + to) = a;
    *reinterpret_cast<u32x4*>(vo + to) = z;
  }
}

// ---- few keys ----
// The keys of a split, at most kHeldBytes of them, are brought to LDS once (every load in flight at a time) and stay there; each wave then takes
// blocks of 32 rows on its own, without barriers.  For short prompts, for patches whose keys are few, and, with the keys split over workgroups, for
// few rows against more keys.  300 queries, 77 keys, 2 x 20 heads of 64: 5.6 us, of which a launch is 3; 300 queries, 2560 keys, 20 heads: 21 us
// (pipelined 23); 300 queries beside a cache of 2400 rows, 20 heads: 24 us with the merge (attn_displaced on rows of bf16: 18).  KV4: segment 0 is the 4-bit cache itself, converted on its way to LDS (levels times scale is exact in bf16), V
// transposed as it is held; the patch's own rows of it are no keys.
constexpr int kHeldBytes = 128 * 1024;
__device__ const u32x4 kZeros[1] = {};
template <int D, int NW, bool MASK, bool KV4>
__global__ __launch_bounds__(64 * NW, 2) void held_attn(QParams p, int row_groups, int own_tiles) {
  constexpr int TILE = 64 * D * 2, CH = D / 8, KS = D / 16, DB = D / 32, RPI = 1024 / (D * 2), NI = TILE / 1024;
  extern __shared__ __attribute__((aligned(16))) char smem[];             // K and V tile of each; where their scores start; their words
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, c = lane & 31, csig = (c & 0x13) | ((c & 4) << 1) | ((c & 8) >> 1), tri = lane & 15;
  int rg, kh, b, split;
  place(p, row_groups, rg, kh, b, split);
  const int n0 = seg0_rows(p, b), n1 = p.seg[1].n;
  // tiles of segment 0 (without the `own_tiles` in the middle that hold nothing but the patch's rows), then of segment 1
  const int first_own = (p.own_lo + 63) >> 6, tiles0 = ((n0 + 63) >> 6) - own_tiles, all = tiles0 + ((n1 + 63) >> 6);
  const int lo = split * p.tiles_per_split, hi = lo + p.tiles_per_split < all ? lo + p.tiles_per_split : all, nt = hi > lo ? hi - lo : 0;
  float* const start = (float*)(smem + 2 * TILE * p.tiles_per_split);
  unsigned long long* const words = (unsigned long long*)(start + 64 * p.tiles_per_split);

  auto queries = [&](int row0, u32x4 (&q)[KS]) DF_INLINE {
    const bool have = row0 + c < p.rows;
    const bf16_t* qp = (const bf16_t*)p.q + row_offset(p, b, kh, have ? row0 + c : 0, p.bsq, p.ldq);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      q[s] = u32x4{0u, 0u, 0u, 0u};
      if (have && 16 * s + 8 * g < p.d) q[s] = *reinterpret_cast<const u32x4*>(qp + 16 * s + 8 * g);
    }
  };
  int row0 = (rg * NW + wave) * 32;
  const int step = row_groups * NW * 32;
  u32x4 q[KS];
  if (row0 < p.rows) queries(row0, q);

  // A wave takes whole tiles of K or V
  for (int u = wave; u < 2 * nt; u += NW) {
    const int i = u >> 1, isv = u & 1;
    int t = lo + i;
    const bool second = t >= tiles0;
    t = second ? t - tiles0 : t < first_own ? t : t + own_tiles;
    const int key = t * 64 + lane, n = second ? n1 : n0;
    bool valid = key < n;
    if (MASK && valid) valid = p.mask[(long long)b * p.seg[0].n + key] != 0;
    if (KV4 && !second && p.own_n > 0) {
      const int rel = (p.own_period > 0 ? key % p.own_period : key) - p.own_lo;
      if (rel >= 0 && rel < p.own_n) valid = false;
    }
    const unsigned long long bits = __builtin_amdgcn_ballot_w64(valid);
    if (!isv) {
      start[64 * i + lane] = valid ? 0.f : -INFINITY;
      if (lane == 0) words[i] = bits;
    }
    if (bits == 0) continue;
    char* const to = smem + (2 * i + isv) * TILE;
    if (!KV4 || second) {
      const Seg& s = p.seg[second ? 1 : 0];
      const long long ld = isv ? s.ldv : s.ldk;
      const bf16_t* src = (const bf16_t*)(isv ? s.v : s.k) + (long long)b * (isv ? s.bsv : s.bsk) + (long long)kh * (isv ? s.hsv : s.hsk) + (long long)t * 64 * ld;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int r = j * RPI + lane / CH, at = lane % CH;
        const int kc = (at ^ (D == 64 ? (r >> 1) & 7 : r & 15)) * 8, vc = (at ^ (D == 64 ? ((r >> 1) & 1) * 2 ^ ((r >> 3) & 1) * 4 : (r & 3) * 4)) * 8;
        const int ch = isv ? vc : kc;
        const bool there = (bits >> r) & 1 && ch < p.d;    // else zeros: a weight of 0 times what else is read there need not be 0
        lds_load16(there ? (const void*)(src + (long long)r * ld + ch) : (const void*)kZeros, to + j * 1024);
      }
    } else {
      const long long base = ((long long)b * p.kv_heads + kh) * p.c.pitch + (long long)t * 64;
      if (!isv) {                                          // a key per lane
        const float s = valid ? bf2f(p.c.ks[base + lane]) : 0.f;
        const u32x4* src = reinterpret_cast<const u32x4*>(p.c.kc + (base + lane) * (D / 2));
        u32x4 w[D / 32];
#pragma unroll
        for (int j = 0; j < D / 32; ++j) w[j] = src[j];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
          float x[8];
          kv4_values(w[j >> 2][j & 3], s, x);
          st_vec((bf16_t*)(to + lane * (D * 2) + ((j ^ (D == 64 ? (lane >> 1) & 7 : lane & 15)) * 16)), x);
        }
      } else {                                             // values of all keys: rows of V^T
#pragma unroll
        for (int e0 = 0; e0 < D; e0 += 8) {                // eight values, eight keys a lane
          const int e = e0 + (lane >> 3), o = lane & 7;
          const unsigned int w = *reinterpret_cast<const unsigned int*>(p.c.vc + (base >> 6) * (D * 32) + e * 32 + o * 4);
          const u32x4 sv = *reinterpret_cast<const u32x4*>(p.c.vs + base + 8 * o);
          const f32x2 a[4] = {kv4_levels<0>(w), kv4_levels<1>(w), kv4_levels<2>(w), kv4_levels<3>(w)};
          float x[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float s = __uint_as_float(k & 1 ? sv[k >> 1] & 0xffff0000u : sv[k >> 1] << 16);
            x[k] = (bits >> (8 * o + k)) & 1 ? a[k >> 1][k & 1] * s : 0.f;
          }
          st_vec((bf16_t*)(to + e * 128 + ((o ^ ((e >> 1) & 7)) * 16)), x);
        }
      }
    }
  }
  __builtin_amdgcn_s_waitcnt(0x0070);                      // the wave's loads have landed
  __syncthreads();

  for (; row0 < p.rows; row0 += step) {
    u32x4 qn[KS];
    const bool more = row0 + step < p.rows;
    if (more) queries(row0 + step, qn);
    f32x16 o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
    float m = kLow, l = 0.f;
    bool any = false;
    for (int i = 0; i < nt; ++i) {
      if (MASK || KV4) {
        const unsigned long long bits = words[i];
        if (__builtin_amdgcn_readfirstlane((int)bits | (int)(bits >> 32)) == 0) continue;
      }
      any = true;
      const char *kt = smem + 2 * i * TILE, *vt = kt + TILE;
      f32x16 s[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(start + 64 * i + 32 * kb + 16 * (j >> 1) + 8 * g + 4 * (j & 1));
          s[kb][4 * j] = v.x; s[kb][4 * j + 1] = v.y; s[kb][4 * j + 2] = v.z; s[kb][4 * j + 3] = v.w;
        }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const int r = 32 * kb + csig;
          const u32x4 a = *reinterpret_cast<const u32x4*>(kt + r * (D * 2) + (((2 * ks + g) ^ (D == 64 ? (r >> 1) & 7 : r & 15)) * 16));
          s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, q[ks]), s[kb], 0, 0, 0);
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
        for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_exp2f(fmaf(s[u >> 1][8 * (u & 1) + e], p.sc, -m));
        l += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
        pk[u] = u32x4{pack_bf2(x[0], x[1]), pack_bf2(x[2], x[3]), pack_bf2(x[4], x[5]), pack_bf2(x[6], x[7])};
      }
      if (KV4 && lo + i < tiles0) {                        // V^T as the cache holds it
#pragma unroll
        for (int ts = 0; ts < 4; ++ts)
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            const int r = 32 * db + csig;
            const u32x4 a = *reinterpret_cast<const u32x4*>(vt + r * 128 + (((2 * ts + g) ^ ((r >> 1) & 7)) * 16));
            o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, pk[ts]), o[db], 0, 0, 0);
          }
      } else {
#pragma unroll
        for (int ts = 0; ts < 4; ++ts)
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            const int key = 16 * ts + 8 * g + (tri >> 2), chunk = 4 * db + 2 * ((lane >> 4) & 1) + (tri & 1);
            const int pc = D == 64 ? chunk ^ (2 * ((key >> 1) & 1)) ^ (4 * ((key >> 3) & 1)) : chunk ^ ((key & 3) * 4);
            const char* at = vt + key * (D * 2) + pc * 16 + ((tri >> 1) & 1) * 8;
            typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
            const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(at));
            const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(at + 4 * D * 2));
            const bf16x8 a = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
            o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, pk[ts]), o[db], 0, 0, 0);
          }
      }
    }
    l += __shfl_xor(l, 32, 64);
    const int row = row0 + c;
    if (row < p.rows) {
      const float inv = p.nsplit > 1 ? 1.f : any ? 1.0f / l : 0.f;        // no key: zeros
      bf16_t* op = (bf16_t*)p.out + row_offset(p, b, kh, row, (long long)p.Lq * p.kv_heads * p.group * p.d, (long long)p.kv_heads * p.group * p.d);
      const long long at0 = ((long long)split * p.B * p.kv_heads + (long long)b * p.kv_heads + kh) * p.rows + row;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          const int at = 32 * db + 16 * f + 8 * g;
          if (at >= p.d) continue;
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = o[db][8 * f + e] * inv;
          if (p.nsplit == 1) {
            st_vec(op + at, v);
          } else {
            st_vec(p.part_o + at0 * p.d + at, v);
            st_vec(p.part_o + at0 * p.d + at + 4, v + 4);
          }
        }
      if (p.nsplit > 1 && g == 0) { p.part_ml[2 * at0] = any ? m : -INFINITY; p.part_ml[2 * at0 + 1] = l; }
    }
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = qn[s];
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
  merge_parts(p, p.nsplit, at, [&](int s) DF_INLINE { return (long long)s * all + row; }, m, l, o);
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
// A wave takes 32 rows and every kw-th tile of 32 keys, the workgroup's four 128 / kw rows; the kw sums of a row are joined in LDS at the end.  There
// are no barriers: lane c's operands are rows of K and values of V as they lie in memory, so they go to registers, V of a tile while its scores are
// summed and K of the next one during O += V P (2048 cycles of matrix instructions per tile at 32 values; waves with the same keys find them in
// L1).  KV4: segment 0 is the cache (own rows masked out), segment 1 rows of floats.  1200 queries, 333 keys, 8 heads of 32: 14.2 us, where a tile
// staged in LDS between barriers took 19.2.
template <int D, bool KV4>
__global__ __launch_bounds__(256) void float_attn(QParams p, int kw) {
  constexpr int DB = D / 32;
  __shared__ float red[3][16 * DB + 2][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, c = lane & 31;
  const int kg = wave & (kw - 1), group = wave / kw, block = 128 / kw;
  int rb, kh, b, split;
  place(p, (p.rows + block - 1) / block, rb, kh, b, split);
  const int n0 = seg0_rows(p, b), n1 = p.seg[1].n, tiles0 = (n0 + 31) >> 5, all = tiles0 + ((n1 + 31) >> 5);
  const int lo = split * p.tiles_per_split, hi = lo + p.tiles_per_split < all ? lo + p.tiles_per_split : all;
  const int row = rb * block + group * 32 + c;
  const bool have = row < p.rows;
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
  f32x16 o[DB], sa;
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  float m = kLow, l = 0.f;
  bool any = false;                                        // a key so far
  auto is_key = [&](int key, int n, bool first) DF_INLINE {
    bool valid = key < n;
    if (valid && first && p.mask) valid = p.mask[(long long)b * p.seg[0].n + key] != 0;
    if (KV4 && valid && first && p.own_n > 0) {
      const int rel = (p.own_period > 0 ? key % p.own_period : key) - p.own_lo;
      valid = !(rel >= 0 && rel < p.own_n);
    }
    return valid;
  };
  // scores of the keys that count -> weights; the keys of element e are 8 (e / 4) + 4 g + e % 4
  auto weights = [&](unsigned int bits) DF_INLINE {
    const unsigned int mine = bits >> (4 * g);
    float top = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      if (!(mine >> (8 * (e >> 2) + (e & 3)) & 1)) sa[e] = -INFINITY;
      top = fmaxf(top, sa[e]);
    }
    top = fmaxf(top, __shfl_xor(top, 32, 64)) * p.sc;
    const float mn = fmaxf(m, top), alpha = __builtin_amdgcn_exp2f(m - mn);
    if (__builtin_amdgcn_ballot_w64(mn > m)) {
      l *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[db][e] *= alpha;
    }
    m = mn;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      sa[e] = __builtin_amdgcn_exp2f(fmaf(sa[e], p.sc, -m));
      l += sa[e];
    }
    any = true;
  };
  auto scores = [&](const f32x4 (&k)[D / 8]) DF_INLINE {
#pragma unroll
    for (int e = 0; e < 16; ++e) sa[e] = 0.f;
#pragma unroll
    for (int j = 0; j < D / 8; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) sa = __builtin_amdgcn_mfma_f32_32x32x2f32(k[j][i], q[4 * j + i], sa, 0, 0, 0);
  };
  int t = lo + kg;
  if constexpr (KV4) {                                     // the cache: codes to registers, levels times scale (exact) before their use
    const long long head = (long long)b * p.kv_heads + kh, base = head * p.c.pitch;
    const int end = hi < tiles0 ? hi : tiles0;
    u32x4 kc[D / 32], vc[DB];
    u32x2 vs[4];
    bf16_t ks;
    bool valid = false;
    auto load_k = [&](int t) DF_INLINE {
      valid = is_key(t * 32 + c, n0, true);
      ks = p.c.ks[base + t * 32 + c];
#pragma unroll
      for (int i = 0; i < D / 32; ++i) kc[i] = *reinterpret_cast<const u32x4*>(p.c.kc + (base + t * 32 + c) * (D / 2) + 16 * i);
    };
    if (t < end) load_k(t);
    for (; t < end; t += kw) {
      const unsigned int bits = (unsigned int)__builtin_amdgcn_ballot_w64(valid);
#pragma unroll
      for (int db = 0; db < DB; ++db)
        vc[db] = *reinterpret_cast<const u32x4*>(p.c.vc + (head * (p.c.pitch / 64) + (t >> 1)) * (D * 32) + (32 * db + c) * 32 + (t & 1) * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) vs[i] = *reinterpret_cast<const u32x2*>(p.c.vs + base + t * 32 + 8 * i + 4 * g);
      f32x4 k[D / 8];
      const float sk = valid ? bf2f(ks) : 0.f;
#pragma unroll
      for (int j = 0; j < D / 8; ++j) {
        const unsigned int w = kc[j >> 2][j & 3] >> (16 * g);
        const f32x2 x = kv4_levels<0>(w), z = kv4_levels<1>(w);
        k[j] = f32x4{x.x * sk, x.y * sk, z.x * sk, z.y * sk};
      }
      if (bits) scores(k);
      __builtin_amdgcn_sched_barrier(0);
      if (t + kw < end) load_k(t + kw);
      if (!bits) continue;
      weights(bits);
      const unsigned int mine = bits >> (4 * g);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float sv[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sv[e] = mine >> (8 * i + e) & 1 ? __uint_as_float(e & 1 ? vs[i][e >> 1] & 0xffff0000u : vs[i][e >> 1] << 16) : 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const unsigned int w = vc[db][i] >> (16 * g);
          const f32x2 x = kv4_levels<0>(w), z = kv4_levels<1>(w);
          o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.x * sv[0], sa[4 * i], o[db], 0, 0, 0);
          o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.y * sv[1], sa[4 * i + 1], o[db], 0, 0, 0);
          o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(z.x * sv[2], sa[4 * i + 2], o[db], 0, 0, 0);
          o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(z.y * sv[3], sa[4 * i + 3], o[db], 0, 0, 0);
        }
      }
    }
  }
  {                                                        // rows of floats; behind the last one it is read again, and what is no key counts as 0
    constexpr bool first = !KV4;
    const Seg& s = p.seg[KV4 ? 1 : 0];
    const int n = KV4 ? n1 : n0, t0 = KV4 ? tiles0 : 0;
    const float* kp = (const float*)s.k + (long long)b * s.bsk + (long long)kh * s.hsk;
    const float* vp = (const float*)s.v + (long long)b * s.bsv + (long long)kh * s.hsv;
    f32x4 k[D / 8];
    bool valid = false;
    auto load_k = [&](int t) DF_INLINE {
      const int key = (t - t0) * 32 + c;
      valid = is_key(key, n, first);
      const float* from = kp + (key < n ? key : n - 1) * s.ldk;
#pragma unroll
      for (int j = 0; j < D / 8; ++j) k[j] = *reinterpret_cast<const f32x4*>(from + (8 * j + 4 * g < p.d ? 8 * j + 4 * g : 0));
    };
    if (t < hi) load_k(t);
    for (; t < hi; t += kw) {
      const unsigned int bits = (unsigned int)__builtin_amdgcn_ballot_w64(valid);
      float v[DB][16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = (t - t0) * 32 + 8 * (e >> 2) + 4 * g + (e & 3);
        const float* from = vp + (key < n ? key : n - 1) * s.ldv;
#pragma unroll
        for (int db = 0; db < DB; ++db) v[db][e] = from[32 * db + c < p.d ? 32 * db + c : 0];
      }
      __builtin_amdgcn_sched_barrier(0);
      if (bits != 0xffffffffu || p.d != D) {
#pragma unroll
        for (int j = 0; j < D / 8; ++j)
          if (!valid || 8 * j + 4 * g >= p.d) k[j] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      scores(k);
      __builtin_amdgcn_sched_barrier(0);
      if (t + kw < hi) load_k(t + kw);
      __builtin_amdgcn_sched_barrier(0);
      if (!bits) continue;
      weights(bits);
      if (bits != 0xffffffffu) {
        const unsigned int mine = bits >> (4 * g);
#pragma unroll
        for (int e = 0; e < 16; ++e)
#pragma unroll
          for (int db = 0; db < DB; ++db)
            if (!(mine >> (8 * (e >> 2) + (e & 3)) & 1)) v[db][e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e)
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[db][e], sa[e], o[db], 0, 0, 0);
    }
  }
  l += __shfl_xor(l, 32, 64);
  if (!any) m = -INFINITY;
  if (kw > 1) {                                            // the sums of a row: the first wave's, then the others in order
    if (kg) {
      float(*to)[64] = red[group * (kw - 1) + kg - 1];
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) to[16 * db + e][lane] = o[db][e];
      to[16 * DB][lane] = m;
      to[16 * DB + 1][lane] = l;
    }
    __syncthreads();
    if (kg) return;
    for (int i = 0; i + 1 < kw; ++i) {
      const float(*from)[64] = red[group * (kw - 1) + i];
      const float mi = from[16 * DB][lane], mn = fmaxf(m, mi);
      if (mi == -INFINITY) continue;                       // (no key)
      const float f = __builtin_amdgcn_exp2f(m - mn), w = __builtin_amdgcn_exp2f(mi - mn);
      l = l * f + from[16 * DB + 1][lane] * w;
      m = mn;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[db][e] = o[db][e] * f + from[16 * db + e][lane] * w;
    }
  }
  if (!have) return;
  const long long at0 = ((long long)split * p.B * p.kv_heads + (long long)b * p.kv_heads + kh) * p.rows + row;
  float* to;
  float f = 1.f;
  if (p.nsplit == 1) {
    to = (float*)p.out + row_offset(p, b, kh, row, (long long)p.Lq * p.kv_heads * p.group * p.d, (long long)p.kv_heads * p.group * p.d);
    f = m != -INFINITY ? 1.0f / l : 0.f;                   // no key: zeros (all scores -inf: 0 / 0, as the formula)
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
// the weights, in float.  Score register (kb, r) of lane group gg is key 16 gg + 4 kb + r.  Bound by memory: one query on 57600 keys, 4 x 20 heads of
// 64 (313 MB of codes and scales): 57 - 59 us, 5.4 TB/s; on 1037 keys, 4 x 5 heads: 5.0 - 5.3 us.
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
    m[n] = kLow; l[n] = 0.f;
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
enum { kRows, kHeld, kFewKv4, kFloat };
struct Plan {
  int kind, nq;                                // nq: blocks of 16 (kFewKv4) or of 32 rows a wave (kRows), waves (kHeld), waves on the same rows (kFloat)
  int block;                                   // rows of a workgroup
  int nsplit, tiles_per_split;                 // all but kRows
  int row_groups, own_tiles;                   // kHeld
  Share share;                                 // kRows
  bool ok;
  size_t expand, parts;                        // bytes of the workspace: the cache's, or a mask's, rows in bf16, the parts of the splits or shares
};

// What an attention is to be planned for: `own` of `L` keys are fresh rows beside a cache, in a row from own_lo on (or not: own_period)
struct Task {
  int B, kv_heads, d, dtype;
  long long rows, L, own, own_lo;
  bool cached, masked, period;
};

constexpr long long kMostGroups = (1LL << 24) - 1;         // of 256 work items: a launch counts those in 32 bits

// Microseconds of writing and merging `parts` rows of partial results
double merge_us(double parts, int d) { return 3.3 + parts * (d + 2) * 8.0 / 3.5e6; }

// The held form with `ns` splits and `nw` waves: its plan, and its predicted microseconds.  A wave takes 0.7 us for 32 rows and a tile of 64 keys of 64
// values where it has its SIMD to itself, two 1.2; 128 values 1.15 and 2.1; a tile of codes 0.3 more to convert.
double plan_held(const Task& k, long long ns, int nw, Plan& r) {
  r = Plan{};
  r.ok = true;
  const long long heads = (long long)k.B * k.kv_heads;
  const int D = k.d <= 64 ? 64 : 128, held = 2 * 64 * D * 2, most = kHeldBytes / held;
  r.kind = kHeld;
  if (k.cached && k.own > 0 && !k.period) {
    const long long first = (k.own_lo + 63) / 64, last = (k.own_lo + k.own) / 64;
    if (last > first) r.own_tiles = (int)(last - first);
  }
  const long long tiles = (k.L + 63) / 64 - r.own_tiles + (k.cached ? (k.own + 63) / 64 : 0), blocks = (k.rows + 31) / 32;
  r.tiles_per_split = (int)((tiles + ns - 1) / ns);
  if (r.tiles_per_split > most) return 1e30;
  r.nsplit = (int)((tiles + r.tiles_per_split - 1) / r.tiles_per_split);
  r.nq = nw;
  r.block = 32 * nw;
  const long long groups = (blocks + nw - 1) / nw, by_lds = 160 * 1024 / (r.tiles_per_split * (held + 264)), cap = by_lds < 8 / nw ? by_lds : 8 / nw;
  const long long fit = 256 * cap / (heads * r.nsplit);                    // workgroups along the rows for one round
  const long long each = fit < 1 ? groups : (groups + fit - 1) / fit;      // blocks of a wave
  r.row_groups = (int)((groups + each - 1) / each);
  const long long wgs = r.row_groups * heads * r.nsplit, rounds = (wgs + 256 * cap - 1) / (256 * cap);
  if (wgs > kMostGroups / 2) return 1e30;
  const long long on_cu = rounds > 1 ? cap : (wgs + 255) / 256;
  const bool two = on_cu * nw > 4;
  const double tile = D == 64 ? (two ? 1.2 : 0.7) : (two ? 2.1 : 1.15);
  if (r.nsplit > 1) r.parts = (size_t)r.nsplit * heads * k.rows * (k.d + 2) * sizeof(float);
  return 3.6 + (D == 64 ? 0.0 : 0.5) + (double)(rounds * each) * r.tiles_per_split * tile + (k.cached ? 0.3 * (double)rounds * r.tiles_per_split : 0.0) +
         (r.nsplit > 1 ? merge_us((double)r.nsplit * heads * k.rows, k.d) : 0.0);
}

// The pipelined form with `qb` blocks of 32 rows a wave.  A tile takes a workgroup 0.85 us, two on a unit 1.16 (128 values 1.1; 256 rows 1.1, one on a
// unit, and beginning and end of a block cost more: 1200 queries on 10240 keys 55 us with 128 rows, 57 with 256; 7200 on 1280 49 and 52, on 5120 124
// and 125, on 57600 of a cache 1260 and 1185); its code is long, the first pass over it costs.
double plan_rows(const Task& k, int qb, Plan& r) {
  r = Plan{};
  r.ok = true;
  const long long heads = (long long)k.B * k.kv_heads, keys0 = k.cached ? k.L - k.own : k.L, keys1 = k.cached ? k.own : 0;
  r.kind = kRows; r.nq = qb; r.block = 128 * qb;
  const long long tiles0 = (keys0 + 63) / 64 + (keys1 + 63) / 64, tiles = tiles0 > 0 ? tiles0 : 1;
  const long long blocks = heads * ((k.rows + r.block - 1) / r.block), all = blocks * tiles;
  const int D = k.d <= 64 ? 64 : 128;
  const bool copied = k.cached || k.masked || k.d != D;
  if (copied) r.expand = ((size_t)heads * keys0 * D * 4 + 255) / 256 * 256 + (k.cached ? 0 : ((size_t)k.B * 4 + 255) / 256 * 256);
  if (blocks > kMostGroups || (copied && (k.cached ? 1 : heads) * tiles > kMostGroups)) return 1e30;
  // Whole blocks, the same number each, where that takes hardly longer than cutting the line into as many equal shares as workgroups fit the chip
  // (the parts and their merge cost about as much as kCut tiles); shares of four tiles or more.
  constexpr long long kCut = 10;
  const long long fit = k.d <= 64 && qb == 1 ? 512 : 256, rounds = (blocks + fit - 1) / fit;
  r.ok = all < (1LL << 31) - (1LL << 20);
  if (!r.ok) return 1e30;
  Share& s = r.share;
  s.tiles = (unsigned int)tiles; s.all = (unsigned int)all;
  if (rounds * tiles <= (all + fit - 1) / fit + kCut) {
    s.per = (unsigned int)(rounds * tiles);
    s.count = (unsigned int)((blocks + rounds - 1) / rounds);
  } else {
    long long n = all / 4 < fit ? all / 4 : fit;
    if (n < 1) n = 1;
    s.count = (unsigned int)n; s.per = (unsigned int)(all / n); s.more = (unsigned int)(all % n);
    r.parts = (size_t)n * 2 * r.block * (k.d + 2) * sizeof(float);
  }
  const bool two = fit == 512 && s.count > 256;
  const double tile = k.d > 64 ? 1.1 : qb == 2 ? 1.1 : two ? 1.16 : 0.85;
  return (qb == 2 ? 12.0 : k.d > 64 ? 7.7 : 6.2) + tile * (double)(s.per + 1) * (double)((s.count + fit - 1) / fit) +
         (r.parts ? merge_us(1.2 * (double)s.count * r.block, k.d) : 0.0) + (copied ? 4.0 + (double)(heads * keys0) * D * (k.cached ? 4.5 : 8.0) / 4e6 : 0.0);
}

// Full precision: `kw` waves of a workgroup on the same rows.  A tile of 32 keys takes a wave 1.55 us at 32 values, 2.6 at 64 and 4.6 at 128 (1200
// queries, 8 heads of 64 on 2048 keys: kw = 1 with 3 splits 69 us, kw = 2 with one 92, kw = 4 with one 104; 333 keys of 32: 15.1, 14.1, 15.1).
double plan_float(const Task& k, int kw, long long ns, Plan& r) {
  r = Plan{};
  r.ok = true;
  const long long heads = (long long)k.B * k.kv_heads, own = k.cached ? k.own : 0, tiles = (k.L + 31) / 32 + (own + 31) / 32;
  r.kind = kFloat; r.nq = kw; r.block = 128 / kw;
  r.tiles_per_split = (int)((tiles + ns - 1) / ns);
  r.nsplit = (int)((tiles + r.tiles_per_split - 1) / r.tiles_per_split);
  const long long wgs = heads * ((k.rows + r.block - 1) / r.block) * r.nsplit, each = (r.tiles_per_split + kw - 1) / kw;
  if (wgs > kMostGroups) return 1e30;
  if (r.nsplit > 1) r.parts = (size_t)r.nsplit * heads * k.rows * (k.d + 2) * sizeof(float);
  const double tile = (0.5 + 1.03 * (k.d <= 32 ? 1 : k.d <= 64 ? 2 : 4)) * (wgs > 256 ? 1.15 : 1.0);
  return 4.5 + tile * (double)(((wgs + 255) / 256) * each) + (r.nsplit > 1 ? merge_us((double)r.nsplit * heads * k.rows, k.d) : 0.0);
}

// Few rows against the cache as it is: 1.05 us per 1000 tiles and blocks of 32 rows (128 values 1.2).  10 heads of 64, 57600 keys: 64 rows 35 us
// (held 75), 128 rows 47 (78), 256 rows 76 (94), 512 rows 153 (pipelined 138); 4 x 20 heads, 1024 keys: 128 rows 18 (21), 512 rows 26 (40).
double plan_few(const Task& k, Plan& r) {
  r = Plan{};
  r.ok = true;
  const long long heads = (long long)k.B * k.kv_heads, tiles = (k.L + 63) / 64;
  r.kind = kFewKv4; r.nq = k.rows > 16 ? 2 : 1; r.block = 16 * r.nq;
  const long long blocks = heads * ((k.rows + r.block - 1) / r.block);
  long long ns = 1;
  if (blocks < 768) ns = 768 / blocks;
  if (ns > tiles / 4) ns = tiles / 4;
  if (ns < 1) ns = 1;
  if (ns > 64) ns = 64;
  r.tiles_per_split = (int)((tiles + ns - 1) / ns);
  r.nsplit = (int)((tiles + r.tiles_per_split - 1) / r.tiles_per_split);
  if (blocks * r.nsplit > kMostGroups) return 1e30;
  if (r.nsplit > 1) r.parts = (size_t)r.nsplit * heads * k.rows * (k.d + 2) * sizeof(float);
  return 6.0 + (k.d == 64 ? 1.05e-3 : 1.2e-3) * (double)(blocks * tiles) + (r.nsplit > 1 ? merge_us((double)r.nsplit * heads * k.rows, k.d) : 0.0);
}

Plan choose(const Task& k) {
  Plan r = {};
  r.ok = true;
  const long long heads = (long long)k.B * k.kv_heads, rows = k.rows, own = k.cached ? k.own : 0;
  double best = 1e30;
  auto offer = [&](double us, const Plan& q) {
    if (us < best - 1e-9) { best = us; r = q; }
  };
  Plan q;
  if (k.dtype == DF_F32) {
#ifdef DF_TUNING
    if (const char* f = tune_env("DF_FLOAT")) {            // waves on the same rows, a colon, splits
      plan_float(k, f[0] - '0', atoi(f + 2), q);
      return q;
    }
#endif
    for (int kw = 1; kw <= 4; kw *= 2)
      for (long long ns = 1; ns <= 32; ++ns)
        if (ns == 1 || ns * kw * 2 <= (k.L + 31) / 32 + (own + 31) / 32) offer(plan_float(k, kw, ns, q), q);
    if (best >= 1e29) r.ok = false;
    return r;
  }
  const char* form = tune_env("DF_QATTN");
  if (k.cached && own == 0 && (form ? !strcmp(form, "few") : rows <= 64)) {
    r.ok = plan_few(k, q) < 1e29;
    return r.ok ? q : r;
  }
  // The form that is predicted to take least
#ifdef DF_TUNING
  if (form && !strcmp(form, "rows1")) { plan_rows(k, 1, q); return q; }
  if (form && !strcmp(form, "rows2")) { plan_rows(k, k.d <= 64 ? 2 : 1, q); return q; }
#endif
  const long long keys = (k.L + 63) / 64 + (own + 63) / 64;
  for (int tps = k.d <= 64 ? 8 : 4; tps >= 1; --tps) {    // tiles that a workgroup holds
    if (tps > keys && tps > 1) continue;
    const long long ns = (keys + tps - 1) / tps;
    if (ns > 48) break;
    offer(plan_held(k, ns, 4, q), q);
    if (rows > 128) offer(plan_held(k, ns, 8, q), q);
  }
#ifdef DF_TUNING
  if (form && !strcmp(form, "held") && best < 1e29) return r;
#endif
  if (k.cached && own == 0) offer(plan_few(k, q), q);
  offer(plan_rows(k, 1, q), q);
  if (k.d <= 64) offer(plan_rows(k, 2, q), q);
  if (best >= 1e29) r.ok = false;
  return r;
}

// The choice takes 1.5 us; a call asks twice (its workspace, then itself) and a program for the same sizes again and again, so a thread keeps its last.
const Plan& plan_of(const Task& k) {
  thread_local Task last = {};
  thread_local Plan plan = {};
  if (last.B != k.B || last.kv_heads != k.kv_heads || last.d != k.d || last.dtype != k.dtype || last.rows != k.rows || last.L != k.L || last.own != k.own ||
      last.own_lo != k.own_lo || last.cached != k.cached || last.masked != k.masked || last.period != k.period || tune_env("DF_QATTN") || tune_env("DF_FLOAT")) {
    plan = choose(k);
    last = k;
  }
  return plan;
}

template <int D, int QB>
int launch_rows(const QParams& p, const Plan& r, hipStream_t st) {
  constexpr int smem = 8 * 64 * D * 2;
  static const hipError_t set = hipFuncSetAttribute((const void*)rows_attn<D, QB>, hipFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (set != hipSuccess) return DF_EHIP;
  hipLaunchKernelGGL((rows_attn<D, QB>), dim3(r.share.count), dim3(256), smem, st, p, r.share);
  if (r.parts) {
    DF_LAUNCH_CHECK();
    const unsigned int per_row = (unsigned int)(p.d / 8), blocks = (unsigned int)((p.rows + r.block - 1) / r.block * (long long)p.kv_heads * p.B);
    hipLaunchKernelGGL(merge_shares, dim3(blocks, (unsigned)((r.block * per_row + 255) / 256)), dim3(256), 0, st, p, r.share, r.block, per_row);
  }
  return DF_OK;
}

}  // namespace

size_t qattn_workspace(int B, long long rows, int kv_heads, int d, long long L, long long own, long long own_lo, bool period, bool cached, bool masked,
                       int dtype) {
  const Plan r = plan_of(Task{B, kv_heads, d, dtype, rows, L, own, own_lo, cached, masked, period});
  return r.expand + r.parts;
}

template <int D, int NW>
int launch_held(const QParams& p, const Plan& r, bool masked, bool cached, hipStream_t st) {
  const int smem = r.tiles_per_split * (2 * 64 * D * 2 + 64 * 4 + 8);
  static const hipError_t set = [] {
    constexpr int most = kHeldBytes + kHeldBytes / (2 * 64 * D * 2) * (64 * 4 + 8);
    hipError_t e = hipFuncSetAttribute((const void*)held_attn<D, NW, false, false>, hipFuncAttributeMaxDynamicSharedMemorySize, most);
    if (e == hipSuccess) e = hipFuncSetAttribute((const void*)held_attn<D, NW, true, false>, hipFuncAttributeMaxDynamicSharedMemorySize, most);
    if (e == hipSuccess) e = hipFuncSetAttribute((const void*)held_attn<D, NW, false, true>, hipFuncAttributeMaxDynamicSharedMemorySize, most);
    return e;
  }();
  if (set != hipSuccess) return DF_EHIP;
  const dim3 grid((unsigned)((long long)r.row_groups * r.nsplit * p.kv_heads * p.B)), wg(64 * NW);
  if (cached) hipLaunchKernelGGL((held_attn<D, NW, false, true>), grid, wg, smem, st, p, r.row_groups, r.own_tiles);
  else if (masked) hipLaunchKernelGGL((held_attn<D, NW, true, false>), grid, wg, smem, st, p, r.row_groups, r.own_tiles);
  else hipLaunchKernelGGL((held_attn<D, NW, false, false>), grid, wg, smem, st, p, r.row_groups, r.own_tiles);
  return DF_OK;
}

int launch_qattn(const QAttnArgs& a, hipStream_t st) {
  const bool cached = a.cache != nullptr;
  const long long rows = (long long)a.Lq * (a.heads / a.kv_heads), own = a.own_period > 0 ? (long long)a.own_n * (a.L / a.own_period) : a.own_n;
  const long long keys0 = cached ? a.L - own : a.L;
  const Plan r = plan_of(Task{a.B, a.kv_heads, a.d, a.dtype, rows, a.L, own, a.own_lo, cached, a.mask != nullptr, a.own_period > 0});
  if (!r.ok || rows > 0x7fffffffLL - 256 || (long long)a.B * a.kv_heads * rows * (a.d / 8) >= (1LL << 32) - 256) return DF_ESHAPE;
  if (a.workspace_bytes < r.expand + r.parts || (r.expand + r.parts && !a.workspace)) return DF_ENOMEM;
  QParams p = {};
  p.q = a.q; p.ldq = a.ldq; p.bsq = a.bsq; p.out = a.out;
  p.B = a.B; p.Lq = a.Lq; p.group = a.heads / a.kv_heads; p.kv_heads = a.kv_heads; p.d = a.d; p.rows = (int)rows;
  p.group_recip = reciprocal_u32((unsigned int)p.group);
  p.sc = a.scale * kLog2e;
  p.nsplit = r.nsplit; p.tiles_per_split = r.tiles_per_split;
  p.mask = a.mask; p.lens = a.lens;
  p.part_o = (float*)((char*)a.workspace + r.expand);
  p.part_ml = p.part_o + (r.kind == kRows ? (size_t)r.share.count * 2 * r.block : (size_t)r.nsplit * a.B * a.kv_heads * rows) * a.d;
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
  const long long nwg = r.kind == kRows ? r.share.count : r.kind == kHeld ? (long long)r.row_groups * a.kv_heads * a.B * r.nsplit : (rows + r.block - 1) / r.block * a.kv_heads * a.B * r.nsplit;
  if (nwg > 0x7fffffffLL) return DF_ESHAPE;
  const dim3 grid((unsigned)nwg);
  if (r.expand && !cached) {                               // the rows that count, and their number
    const int D = a.d <= 64 ? 64 : 128, tiles = (int)((keys0 + 63) / 64);
    bf16_t *k = (bf16_t*)a.workspace, *v = k + (size_t)a.B * a.kv_heads * keys0 * D;
    int* const counts = (int*)((char*)a.workspace + ((size_t)a.B * a.kv_heads * keys0 * D * 4 + 255) / 256 * 256);
    hipLaunchKernelGGL(keep_rows, dim3((unsigned)((long long)tiles * a.kv_heads * a.B)), dim3(256), 0, st, p, tiles, k, v, counts);
    DF_LAUNCH_CHECK();
    Seg& s = p.seg[0];
    s.k = k; s.v = v; s.ldk = s.ldv = D; s.hsk = s.hsv = keys0 * D; s.bsk = s.bsv = keys0 * D * a.kv_heads;
    p.lens = counts;
  }
  if (r.expand && cached) {
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
    if (cached && a.d == 64) hipLaunchKernelGGL((float_attn<64, true>), grid, dim3(256), 0, st, p, r.nq);
    else if (cached) hipLaunchKernelGGL((float_attn<128, true>), grid, dim3(256), 0, st, p, r.nq);
    else if (a.d <= 32) hipLaunchKernelGGL((float_attn<32, false>), grid, dim3(256), 0, st, p, r.nq);
    else if (a.d <= 64) hipLaunchKernelGGL((float_attn<64, false>), grid, dim3(256), 0, st, p, r.nq);
    else hipLaunchKernelGGL((float_attn<128, false>), grid, dim3(256), 0, st, p, r.nq);
  } else if (r.kind == kFewKv4) {
    if (a.d == 64 && r.nq == 1) hipLaunchKernelGGL((few_rows_kv4<64, 1>), grid, dim3(256), 0, st, p);
    else if (a.d == 64) hipLaunchKernelGGL((few_rows_kv4<64, 2>), grid, dim3(256), 0, st, p);
    else if (r.nq == 1) hipLaunchKernelGGL((few_rows_kv4<128, 1>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((few_rows_kv4<128, 2>), grid, dim3(256), 0, st, p);
  } else if (r.kind == kHeld) {
    const bool masked = a.mask != nullptr;
    const int rc = a.d <= 64 ? (r.nq == 8 ? launch_held<64, 8>(p, r, masked, cached, st) : launch_held<64, 4>(p, r, masked, cached, st))
                             : (r.nq == 8 ? launch_held<128, 8>(p, r, masked, cached, st) : launch_held<128, 4>(p, r, masked, cached, st));
    if (rc != DF_OK) return rc;
  } else {
    const int rc = a.d <= 64 ? (r.nq == 1 ? launch_rows<64, 1>(p, r, st) : launch_rows<64, 2>(p, r, st)) : launch_rows<128, 1>(p, r, st);
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
