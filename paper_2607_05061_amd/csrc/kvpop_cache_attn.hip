// gfx950 attention of new queries over the compact cache's page lists of 8-bit keys and
// values (include/kvpop_cache.h):
//
//   l(i, j) = scale <q_i, k_j>,  k_j = code 2^ke,  v_j = code 2^ve,
//   lse_i   = log sum_j exp l(i, j),   o_i = sum_j exp(l(i, j) - lse_i) v_j.
//
// One pass with a running reference. A value's power of two goes into the exponent of its
// probability: with x = l log2(e) + ve, the numerators p' = 2^(x - M) multiply the bare codes,
// and the normaliser in the same units is sum p' 2^-ve. So codes enter the products as they
// are, exact in 16 bits, whatever scales a list's pages have. Numerators are f16 there (the
// normaliser sums them in 32 bits): M lies below the running maximum of x, so that a numerator far
// below the largest one keeps its 11 bits: the largest is at least 2^7, so they reach down to
// 2^-21 of it (2^-14 is f16's least normal number), and below that what is lost is 2^-32 of it at
// most. (With M = max x, a sink's 2^27 times larger probability, or a scale 2^24 times another
// page's, took the other keys out of o and left them in the normaliser.)

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kvpop_cache.h"
#include "kvpop_cache_codes.h"
#include "kvpop_internal.h"

namespace kvpop {
namespace {

// Where M moves, the largest numerator becomes 2^kRoom. (A reference 7 below the maximum, rounded to 32 bits, is
// at most 8 below it, whatever its size, and no numerator passes f16's range; 9 and more can become 16.)
constexpr float kRoom = 7.f;
constexpr int kNoPage = 0x7FFF7FFF;  // in the place of a page's exponents
constexpr int kRows = 16;        // (token, head) rows per workgroup
constexpr int kTile = 32;        // keys per step of a wave
constexpr int kMinTiles = 1;     // least tiles per wave of a split list
constexpr int kMaxSplits = 64;
constexpr int kFewParts = 4;     // fewer parts are joined by one group of threads a row

// Bytes 2 k and 2 k + 1 (k 0 or 1) of two keys' dwords, in 16 bits: a is byte 2 k of
// (w0, w1), b byte 2 k + 1.
template <int FMT, int K>
__device__ __forceinline__ void widen_pair(uint32_t w0, uint32_t w1, f16x2& a, f16x2& b) {
  if constexpr (FMT == KVPOP_CACHE_INT8) {
    constexpr uint32_t s0 = 0x0C000C00u | (2 * K) | ((4 + 2 * K) << 16), s1 = s0 + 0x00010001u;
    const f16x2 off = {(_Float16)1152.f, (_Float16)1152.f};
    a = as_h2(__builtin_amdgcn_perm(w1, w0, s0) ^ 0x64806480u) - off;
    b = as_h2(__builtin_amdgcn_perm(w1, w0, s1) ^ 0x64806480u) - off;
  } else {
    constexpr uint32_t s = (2 * K) | ((4 + 2 * K) << 8) | ((2 * K + 1) << 16) | ((5 + 2 * K) << 24);
    const uint32_t w = __builtin_amdgcn_perm(w1, w0, s);
    a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true);
  }
}

// What a list's splits hold: the tiles of each (at least `least`), for a list of n tiles.
__device__ __forceinline__ int split_tiles(int n, int splits, int least) {
  return max(least, (n + splits - 1) / splits);
}

// One workgroup: 16 rows (query tokens times the G heads of a KV head, tokens slowest)
// against a run of a list's tiles, which its waves divide. S^T = K Q^T puts keys on
// the accumulator's rows and queries on its columns, so a lane holds 4 keys of each 16 for
// the query lane % 16; with two such blocks the lane's 8 probabilities are the B operand of
// O^T += V^T P^T as they stand, its contraction index running over the keys
// {4 g .. 4 g + 3, 16 + 4 g ..} of lane group g. A lane loads the D / 16 bytes at D / 16 (lane %
// 16) of each of these keys, so that byte t of its 8 loads is its A operand of the
// product for the head dims t, t + D / 16, ...: no value passes through LDS.
// HBM bounds it: 8 KB of a tile are on their way while one is multiplied. 32 x 8 lists of 16384
// tokens of 128 dims (1.07 GB) take 185-195 us, 5.5-5.8 TB/s (part of the pool stays in
// the 256 MB cache), 128 x 8 of 2276 113-115 us, 5.2 TB/s. For D = 128 the form of 8 waves takes 142
// registers (3 waves a SIMD), that of 4 waves 140 and 36 accumulator registers (2 waves). Two tiles on
// their way (172 registers): 113 us, but 9.1 instead of 7.6 us for 64 x 8 lists of 100.
template <int D, int FMT, int W>
__global__ __launch_bounds__(64 * W) void cache_attn_kernel(CacheAttnLaunch a, int row_blocks, int splits) {
  constexpr int KS = D / 32;  // k-steps of the logits
  constexpr int VB = D / 16;  // bytes of a key's value per lane; tiles of 16 head dims
  constexpr int KW = D / 16;  // dwords of a key per lane (D / 4 bytes)
  constexpr int VW = VB / 4;
  __shared__ float o_sh[W][kRows][D + 4];
  __shared__ float m_sh[W][kRows], s_sh[W][kRows];

  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int g = lane >> 4, c = lane & 15;
  int blk = blockIdx.x;
  const int split = blk % splits;
  blk /= splits;
  const int rb = blk % row_blocks, list = blk / row_blocks;
  const int b = list / a.c.H, h = list % a.c.H, G = a.Hq / a.c.H, R = G * a.N;
  const int lgP = 31 - __builtin_clz(a.c.P);

  const int L = clampi(a.held[list], 0, a.c.max_pages * a.c.P);
  const int nq = a.q_lens ? clampi(a.q_lens[b], 0, a.N) : a.N;
  const int tiles = (L + kTile - 1) / kTile, per = split_tiles(tiles, splits, kMinTiles * W);
  if (split > 0 && split * per >= tiles) return;
  const int active = max(1, (tiles + per - 1) / per);

  const int end_wg = min(tiles, (split + 1) * per);
  const int share = (end_wg - split * per + W - 1) / W;
  // Nothing to read where no row of the workgroup has a query.
  const int t0 = split * per + wave * share, t1 = rb * kRows / G < nq ? min(end_wg, t0 + share) : t0;

  struct Tile {
    Words<4> k[2][KW / 4];
    Words<VW> v[2][4];
  };

  // Pages 64 at a time, one per lane.
  int ids = -1, exps = 0, page_base = 0;
  auto load_pages = [&](int first) __attribute__((always_inline)) {
    page_base = first;
    const int at = first + lane;
    ids = at < a.c.max_pages && (at << lgP) < L ? a.c.table[(int64_t)list * a.c.max_pages + at] : -1;
    if ((unsigned)ids >= (unsigned)a.c.n_pages) ids = -1;
    if (ids >= 0)
      exps = (clampi(a.c.ke[ids], kExpMin, kExpMax) & 0xFFFF) | (clampi(a.c.ve[ids], kExpMin, kExpMax) << 16);
  };
  auto load = [&](Tile& x, int t) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int key = kTile * t + 16 * s, at = (key >> lgP) - page_base;
      const int64_t base = ((int64_t)max(__builtin_amdgcn_readlane(ids, at), 0) << lgP) + (key & (a.c.P - 1));
      const uint8_t* kp = a.c.k + base * D + c * D + (D / 4) * g;
#pragma unroll
      for (int i = 0; i < KW / 4; ++i) x.k[s][i] = *reinterpret_cast<const Words<4>*>(kp + 16 * i);
      const uint8_t* vp = a.c.v + base * D + 4 * g * D + VB * c;
#pragma unroll
      for (int i = 0; i < 4; ++i) x.v[s][i] = *reinterpret_cast<const Words<VW>*>(vp + i * D);
    }
  };
  Tile x;
  if (t0 < t1) {
    load_pages((kTile * t0) >> lgP);
    load(x, t0);
  }

  // This lane's query. Rows without one go along with every key in sight.
  const int row = rb * kRows + c, qi = row / G, qg = row % G;
  const bool some = row < R && qi < nq;
  const int seen = some ? max(0, L - (nq - 1 - qi)) : L;
  f16x8 qf[KS];
  float cq;
  {
    float x[KS][8], big = 0.f;
#pragma unroll
    for (int m = 0; m < KS; ++m) {
      uint4 w = {0, 0, 0, 0};
      if (some)
        w = *reinterpret_cast<const uint4*>(a.q.ptr + b * a.q.sb + (h * G + qg) * a.q.sh + qi * a.q.st + (D / 4) * g +
                                            8 * m);
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[m][2 * i] = __uint_as_float(u[i] << 16);
        x[m][2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) big = fmaxf(big, __builtin_fabsf(x[m][i]));
    }
    big = max_groups(big);
    // Queries in f16: their largest element in [2^14, 2^15), so that elements down to
    // 2^-28 of it keep their 8 bits.
    const int e = big > 0.f ? __builtin_amdgcn_frexp_expf(big) - 15 : 0;
    cq = __builtin_ldexpf(a.scale * kLog2e, e);
#pragma unroll
    for (int m = 0; m < KS; ++m)
#pragma unroll
      for (int i = 0; i < 8; ++i) qf[m][i] = (_Float16)__builtin_ldexpf(x[m][i], -e);
  }
  const int least_seen = -(int)max_groups(-(float)seen);  // exact: below 2^24
  int sure = least_seen;                                   // keys that every column sees
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) sure = min(sure, __shfl_xor(sure, o));
  sure = __builtin_amdgcn_readfirstlane(sure);

  f32x4 o[VB];
#pragma unroll
  for (int t = 0; t < VB; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  float M = neg_inf(), S = 0.f;

  auto step = [&](Tile& x, int t) __attribute__((always_inline)) {
    float l[2][4];
    int id[2], e[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int at = ((kTile * t + 16 * s) >> lgP) - page_base;
      id[s] = __builtin_amdgcn_readlane(ids, at);
      e[s] = __builtin_amdgcn_readlane(exps, at);
    }
    const bool whole = kTile * (t + 1) <= sure && id[0] >= 0 && id[1] >= 0;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int m = 0; m < KS; ++m) {
        H8 k;
        widen4<FMT>(x.k[s][m / 2].w[2 * (m % 2)], k.h[0], k.h[1]);
        widen4<FMT>(x.k[s][m / 2].w[2 * (m % 2) + 1], k.h[2], k.h[3]);
        acc = mfma16(k.v, qf[m], acc);
      }
      const float kc = __builtin_ldexpf(cq, (int16_t)e[s]), ve = (float)(e[s] >> 16);
#pragma unroll
      for (int r = 0; r < 4; ++r) l[s][r] = __builtin_fmaf(acc[r], kc, ve);
      if (!whole) {
        const int key = kTile * t + 16 * s + 4 * g;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          l[s][r] = id[s] >= 0 && key + r < seen ? l[s][r] : neg_inf();
          if (id[s] < 0 || key + r >= L)
#pragma unroll
            for (int i = 0; i < VW; ++i) x.v[s][r].w[i] = 0;
        }
      }
    }
    float mx = fmaxf(fmaxf(fmaxf(l[0][0], l[0][1]), fmaxf(l[0][2], l[0][3])),
                     fmaxf(fmaxf(l[1][0], l[1][1]), fmaxf(l[1][2], l[1][3])));
    mx = max_groups(mx) - kRoom;
    if (__builtin_amdgcn_ballot_w64(mx > M) != 0) {
      const float m = fmaxf(M, mx);
      const float f = __builtin_amdgcn_exp2f(M - (m == neg_inf() ? 0.f : m));
#pragma unroll
      for (int i = 0; i < VB; ++i) o[i] *= f;
      S *= f;
      M = m;
    }
    const float mu = M == neg_inf() ? 0.f : M;
    H8 p;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const float w = __builtin_ldexpf(1.f, -(e[s] >> 16));
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float y = __builtin_amdgcn_exp2f(l[s][r] - mu);
        S = __builtin_fmaf(y, w, S);
        p.v[4 * s + r] = (_Float16)y;
      }
    }
#pragma unroll
    for (int i = 0; i < VW; ++i) {
      H8 v[4];
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const uint32_t w0 = x.v[s][2 * r].w[i], w1 = x.v[s][2 * r + 1].w[i];
          widen_pair<FMT, 0>(w0, w1, v[0].h[2 * s + r], v[1].h[2 * s + r]);
          widen_pair<FMT, 1>(w0, w1, v[2].h[2 * s + r], v[3].h[2 * s + r]);
        }
#pragma unroll
      for (int j = 0; j < 4; ++j) o[4 * i + j] = mfma16(v[j].v, p.v, o[4 * i + j]);
    }
  };

  for (int t = t0; t < t1;) {
    const int64_t last_key = (int64_t)(page_base + 64) << lgP;  // of these 64 pages
    const int stop = (int)min((int64_t)t1, last_key / kTile);
    for (; t < stop; ++t) {
      Tile nx;
      if (t + 1 < stop) load(nx, t + 1);
      step(x, t);
      x = nx;
    }
    if (t < t1) {
      load_pages((kTile * t) >> lgP);
      load(x, t);
    }
  }

  // The waves' parts: columns of 16 rows, head dims VB (4 g + r) + t.
  S = sum_groups(S);
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int t = 0; t < VB; ++t) o_sh[wave][c][VB * (4 * g + r) + t] = o[t][r];
  if (g == 0) m_sh[wave][c] = M, s_sh[wave][c] = S;
  __syncthreads();
  if (W > 4 && tid >= 256) return;
  const int wr = tid / 16, d0 = (tid % 16) * VB;
  const int orow = rb * kRows + wr, oi = orow / G;
  if (orow >= R) return;
  const bool has = oi < nq && L - (nq - 1 - oi) > 0;
  float m = neg_inf();
#pragma unroll
  for (int w = 0; w < W; ++w) m = fmaxf(m, m_sh[w][wr]);
  const float mu = m == neg_inf() ? 0.f : m;
  float z = 0.f, y[VB];
#pragma unroll
  for (int t = 0; t < VB; ++t) y[t] = 0.f;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const float f = __builtin_amdgcn_exp2f(m_sh[w][wr] - mu);
    z = __builtin_fmaf(f, s_sh[w][wr], z);
#pragma unroll
    for (int t = 0; t < VB; ++t) y[t] = __builtin_fmaf(f, o_sh[w][wr][d0 + t], y[t]);
  }
  if (!has) m = neg_inf(), z = 0.f;
  if (active == 1) {
    const int64_t out = ((int64_t)b * a.Hq + h * G + orow % G) * a.N + oi;
    const float f = has && z != 0.f ? 1.f / z : 0.f;
    typedef __bf16 bf16v __attribute__((ext_vector_type(VB)));
    typedef float f32v __attribute__((ext_vector_type(VB)));
    f32v v;
#pragma unroll
    for (int t = 0; t < VB; ++t) v[t] = has ? y[t] * f : 0.f;
    *reinterpret_cast<bf16v*>(a.o + out * D + d0) = __builtin_convertvector(v, bf16v);
    if (d0 == 0) a.lse[out] = z > 0.f || z != z ? (m + __builtin_amdgcn_logf(z)) * kLn2 : neg_inf();
  } else {
    const int64_t at = ((int64_t)list * R + orow) * splits + split;
    float* po = a.workspace + at * D + d0;
#pragma unroll
    for (int t = 0; t < VB; ++t) po[t] = has ? y[t] : 0.f;
    float* ms = a.workspace + (int64_t)a.c.B * a.c.H * R * splits * D + 2 * at;
    if (d0 == 0) ms[0] = m, ms[1] = z;
  }
}

// The same for chunks of queries, whose work is the matrix products: 256 rows (32 a wave, tokens times
// heads, tokens slowest) against a run of a list's tiles of 64 keys (128 for D = 64). A tile is widened to
// 16 bits once, by all waves, into LDS, in the order in which the products' operands are
// read (16 bytes a lane, a wave's 1 KB in one piece):
//   S^T = K Q^T    v_mfma_f32_32x32x16_f16, keys on the accumulator's rows, queries on its
//                  columns: a lane owns one query, with the other half of its keys in lane ^ 32;
//   O^T += V^T P^T the numerators are the B operand as they stand, contraction slot (hi, j) of
//                  16 keys being key 4 hi + j % 4 + 8 (j / 4), so V's piece for (16 keys, 32
//                  head dims, hi) holds those 8 keys of each dim. A thread widens 4 bytes of
//                  4 keys, half a piece; dim 4 t + i of a block of 32 sits at place 8 i + t, so that
//                  neighbouring threads write neighbouring places.
// Three tile buffers: while one is multiplied, with the next one's first logits, the one after
// is widened, and the bytes of the following one are on their way in registers.
//
// 1024 queries of 32 heads over 8 lists of 32768 tokens, a workgroup for each CU: 0.55-0.60 ms, 910-980
// TFLOP/s (36-39% of the dense peak), D = 64 0.38-0.39 ms; other numbers of queries reach 550-810 (the
// times beside `plan`). Matrix cores are busy on 43% of the cycles, the vector ALU (exponential, its
// argument and sum per pair, the widening) on 54%, LDS on 31%. With the numerators of 64 keys after
// all their logits, and two buffers: 0.70 ms; with the masks of the last tiles as selects in every
// block, 0.63 ms; with a maximum per block instead of the sums' test 3-5% more; with a raised
// priority around the products, the same. With M moved for all queries of a wave as soon as one asks for it 1-3%
// less (D = 64 5%), but then what a query gets depends on the others.
constexpr int kChunkWaves = 8, kChunkThreads = 64 * kChunkWaves, kChunkRows = 32 * kChunkWaves;
constexpr float kSlack = 12.f;  // how far x may pass M, in powers of two, in a block that a query sees a part of

typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 mfma32(const f16x8& a, const f16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ float max_pair(float x) {
  const int i = __float_as_int(x);
  const auto r = __builtin_amdgcn_permlane32_swap(i, i, false, false);
  return fmaxf(__int_as_float(r[0]), __int_as_float(r[1]));
}

constexpr int chunk_tile(int D) { return 8192 / D; }  // keys: 16 KB a widened side

template <int D, int FMT>
__global__ __attribute__((amdgpu_flat_work_group_size(kChunkThreads, kChunkThreads), amdgpu_waves_per_eu(2, 2))) void cache_attn_chunk_kernel(CacheAttnLaunch a, int row_blocks,
                                                                            int splits) {
  constexpr int KS = D / 16, DB = D / 32;                        // k-steps, blocks of 32 dims
  constexpr int TILE = chunk_tile(D), NB = TILE / 32, NE = TILE / 16;  // blocks of 32 keys; of 16, with exponents
  constexpr int kSide = TILE * D * 2;                             // bytes of a widened side
  __shared__ __attribute__((aligned(16))) uint8_t sm[3][2][kSide];

  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int hi = lane >> 5, col = lane & 31;
  // Later rows see more keys: they go first.
  const int lists = a.c.B * a.c.H, list = (int)(blockIdx.x % (unsigned)lists);
  const int part = (int)(blockIdx.x / (unsigned)lists), split = part % splits, rb = row_blocks - 1 - part / splits;
  const int b = list / a.c.H, h = list % a.c.H, G = a.Hq / a.c.H, R = G * a.N;
  const int P = a.c.P, lgP = 31 - __builtin_clz(P);

  const int L = clampi(a.held[list], 0, a.c.max_pages * P);
  const int nq = a.q_lens ? clampi(a.q_lens[b], 0, a.N) : a.N;
  const int tiles = (L + TILE - 1) / TILE, per = split_tiles(tiles, splits, 1);
  if (split > 0 && split * per >= tiles) return;
  const int active = max(1, (tiles + per - 1) / per);

  // This lane's query; rows without one go along with every key in sight.
  const int row = rb * kChunkRows + 32 * wave + col, qi = row / G, qg = row % G;
  const bool some = row < R && qi < nq;
  const int seen = some ? max(0, L - (nq - 1 - qi)) : L;
  f16x8 qf[KS];
  float cq;
  {
    uint4 w[KS];
    float big = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      w[s] = uint4{0, 0, 0, 0};
      if (some)
        w[s] = *reinterpret_cast<const uint4*>(a.q.ptr + b * a.q.sb + (h * G + qg) * a.q.sh + qi * a.q.st + 16 * s +
                                               8 * hi);
      const uint32_t u[4] = {w[s].x, w[s].y, w[s].z, w[s].w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        big = fmaxf(big, fmaxf(__builtin_fabsf(__uint_as_float(u[i] << 16)),
                               __builtin_fabsf(__uint_as_float(u[i] & 0xFFFF0000u))));
    }
    big = max_pair(big);
    const int e = big > 0.f ? __builtin_amdgcn_frexp_expf(big) - 15 : 0;
    cq = __builtin_ldexpf(a.scale * kLog2e, e);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const uint32_t u[4] = {w[s].x, w[s].y, w[s].z, w[s].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        qf[s][2 * i] = (_Float16)__builtin_ldexpf(__uint_as_float(u[i] << 16), -e);
        qf[s][2 * i + 1] = (_Float16)__builtin_ldexpf(__uint_as_float(u[i] & 0xFFFF0000u), -e);
      }
    }
  }
  // Keys that every column of the wave sees, and that any does; the last key any row of
  // the workgroup sees (its last row's token sees most).
  int sure = seen, any = some ? seen : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    sure = min(sure, __shfl_xor(sure, o));
    any = max(any, __shfl_xor(any, o));
  }
  sure = __builtin_amdgcn_readfirstlane(sure);
  any = __builtin_amdgcn_readfirstlane(any);
  const int last_qi = min(min(R - 1, rb * kChunkRows + kChunkRows - 1) / G, nq - 1);
  const int most = rb * kChunkRows / G < nq ? max(0, L - (nq - 1 - last_qi)) : 0;
  const int t0 = split * per, t1 = min(min(tiles, t0 + per), (most + TILE - 1) / TILE);

  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = f32x16{};
  float M = neg_inf(), S = 0.f;

  // Pages 64 at a time, one per lane; -1: none.
  int ids = -1, exps = 0, page_base = 0;
  auto load_pages = [&](int first) __attribute__((always_inline)) {
    page_base = first;
    const int at = first + lane;
    ids = at < a.c.max_pages && (at << lgP) < L ? a.c.table[(int64_t)list * a.c.max_pages + at] : -1;
    if ((unsigned)ids >= (unsigned)a.c.n_pages) ids = -1;
    exps = kNoPage;
    if (ids >= 0)
      exps = (clampi(a.c.ke[ids], kExpMin, kExpMax) & 0xFFFF) | (clampi(a.c.ve[ids], kExpMin, kExpMax) << 16);
  };
  // A tile on its way: 16 bytes of each side a thread, and its pages' exponents per 16 keys.
  // K: 16 bytes of one key. V: 4 bytes of 4 keys (slots j of one half of a piece).
  struct Raw {
    uint32_t k[4], v[4];
    int e[NE];
  };
  const int kkey = tid % TILE, kpart = tid / TILE;
  const int vquad = tid % (D / 4), vgrp = tid / (D / 4), v16 = vgrp >> 2, vhi = vgrp & 1, vhalf = (vgrp >> 1) & 1;
  const int vkey = 16 * v16 + 4 * vhi + 8 * vhalf;
  auto load = [&](Raw& x, int t) __attribute__((always_inline)) {
    if (((TILE * (t + 1) - 1) >> lgP) >= page_base + 64) load_pages((TILE * t) >> lgP);
#pragma unroll
    for (int i = 0; i < NE; ++i) x.e[i] = __builtin_amdgcn_readlane(exps, ((TILE * t + 16 * i) >> lgP) - page_base);
    // Values past the list's end are those of its last slot: their numerators are 0, and their
    // bytes could be anything.
    const int kk = TILE * t + kkey, vk = TILE * t + vkey, vl = min(vk, L - 1);
    const int kid = max(__shfl(ids, (kk >> lgP) - page_base), 0), vid = max(__shfl(ids, (vl >> lgP) - page_base), 0);
    const uint4 u = *reinterpret_cast<const uint4*>(a.c.k + (((int64_t)kid << lgP) + (kk & (P - 1))) * D + 16 * kpart);
    x.k[0] = u.x, x.k[1] = u.y, x.k[2] = u.z, x.k[3] = u.w;
    const uint8_t* p = a.c.v + (((int64_t)vid << lgP) + (vl & (P - 1))) * D + 4 * vquad;
    const int top = max(0, min(3, L - 1 - vk));
#pragma unroll
    for (int j = 0; j < 4; ++j) x.v[j] = *reinterpret_cast<const uint32_t*>(p + min(j, top) * D);
  };
  auto widen = [&](const Raw& x, int buf) __attribute__((always_inline)) {
    uint8_t* p = sm[buf][0] + (((kkey >> 5) * KS * 2 + kpart * 2) * 32 + (kkey & 31)) * 16;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      H8 k;
      widen4<FMT>(x.k[2 * i], k.h[0], k.h[1]);
      widen4<FMT>(x.k[2 * i + 1], k.h[2], k.h[3]);
      *reinterpret_cast<f16x8*>(p + i * 512) = k.v;
    }
    H8 v[2];
    widen_pair<FMT, 0>(x.v[0], x.v[1], v[0].h[0], v[0].h[2]);
    widen_pair<FMT, 0>(x.v[2], x.v[3], v[0].h[1], v[0].h[3]);
    widen_pair<FMT, 1>(x.v[0], x.v[1], v[1].h[0], v[1].h[2]);
    widen_pair<FMT, 1>(x.v[2], x.v[3], v[1].h[1], v[1].h[3]);
    p = sm[buf][1] + (((v16 * DB + (vquad >> 3)) * 2 + vhi) * 32 + (vquad & 7)) * 16 + 8 * vhalf;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<uint2*>(p + i * 128) = uint2{v[i / 2].u[2 * (i & 1)], v[i / 2].u[2 * (i & 1) + 1]};
  };
  // Values of 16 keys without a page become 0.
  auto blank = [&](const int (&e)[NE], int buf) __attribute__((always_inline)) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < NE; ++i) bad = bad || e[i] == kNoPage;
    if (!bad) return;
#pragma unroll
    for (int i = 0; i < NE; ++i)
      if (e[i] == kNoPage && v16 == i) {
        uint8_t* p = sm[buf][1] + (((v16 * DB + (vquad >> 3)) * 2 + vhi) * 32 + (vquad & 7)) * 16 + 8 * vhalf;
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<uint2*>(p + j * 128) = uint2{0, 0};
      }
  };
  // The logits of 32 keys (block n of a tile).
  auto logits = [&](int n, int buf) __attribute__((always_inline)) {
    f32x16 x = f32x16{};
    const uint8_t* kt = sm[buf][0] + n * KS * 1024 + lane * 16;
#pragma unroll
    for (int s = 0; s < KS; ++s) x = mfma32(*reinterpret_cast<const f16x8*>(kt + s * 1024), qf[s], x);
    return x;
  };
  // Numerators 2^(x - M) of a block of 32 keys from its bare products, summed and in 16 bits. The
  // usual block is all seen, and none of its numerators passes f16's range or is NaN: their sums
  // show it. For a query that does not see all of a block, or whose own sums pass the range,
  // it is done over without the keys that are not seen, and with M moved where one passes it by
  // more than kSlack. The wave's other queries keep what they have: a query's bits follow
  // from its own products alone.
  auto numerators = [&](const f32x16& x, int e0, int e1, int key0, f16x8 (&p)[2]) __attribute__((always_inline)) {
    const float kc0 = __builtin_ldexpf(cq, (int16_t)e0), kc1 = __builtin_ldexpf(cq, (int16_t)e1);
    const float v0 = (float)(e0 >> 16), v1 = (float)(e1 >> 16), m0 = v0 - M, m1 = v1 - M;
    const float w0 = __builtin_ldexpf(1.f, -(e0 >> 16)), w1 = __builtin_ldexpf(1.f, -(e1 >> 16));
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const float y0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], kc0, m0));
      const float y1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r + 8], kc1, m1));
      s0 += y0, s1 += y1;
      p[0][r] = (_Float16)y0, p[1][r] = (_Float16)y1;
    }
    const bool pages = e0 != kNoPage && e1 != kNoPage, whole = key0 + 32 <= sure && pages;
    const uint64_t over = __builtin_amdgcn_ballot_w64(!(s0 <= 65504.f && s1 <= 65504.f));
    if (!whole || over != 0) {
      f32x16 y;
      float mx = neg_inf();
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        y[r] = __builtin_fmaf(x[r], r < 8 ? kc0 : kc1, r < 8 ? v0 : v1);
      }
      if (!whole) {
        int key = key0 + 4 * hi;
        asm volatile("" : "+v"(key));  // the comparisons stay in this branch
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if ((r < 8 ? e0 : e1) == kNoPage || key + 8 * (r >> 2) + (r & 3) >= seen) y[r] = neg_inf();
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, y[r]);
      mx = max_pair(mx);
      const bool asks = ((uint32_t)(over | over >> 32) >> col & 1) != 0;  // in either of the query's lanes
      const bool keep = key0 + 32 <= seen && pages && !asks;
      // (The difference is exact where it matters; M + kSlack can round to M + 16, whose numerator is infinite.)
      const float m = !keep && mx - M > kSlack ? mx - kRoom : M, mu = m == neg_inf() ? 0.f : m;
      if (__builtin_amdgcn_ballot_w64(m != M) != 0) {
        const float f = __builtin_amdgcn_exp2f(M - mu);
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] *= f;
        S *= f;
        M = m;
      }
      if (!keep) {
        s0 = s1 = 0.f;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const float y0 = __builtin_amdgcn_exp2f(y[r] - mu), y1 = __builtin_amdgcn_exp2f(y[r + 8] - mu);
          s0 += y0, s1 += y1;
          p[0][r] = (_Float16)y0, p[1][r] = (_Float16)y1;
        }
      }
    }
    S = __builtin_fmaf(s0, w0, __builtin_fmaf(s1, w1, S));
  };
  auto weigh = [&](const f16x8 (&p)[2], int n, int buf) __attribute__((always_inline)) {
    const uint8_t* vt_ = sm[buf][1] + n * 2 * DB * 1024 + lane * 16;
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
      for (int d = 0; d < DB; ++d)
        o[d] = mfma32(*reinterpret_cast<const f16x8*>(vt_ + (k2 * DB + d) * 1024), p[k2], o[d]);
  };

  if (t0 < t1) {
    Raw x, y;
    int e[NE], en[NE];
    load_pages((TILE * t0) >> lgP);
    load(x, t0);
    if (t0 + 1 < t1)
      load(y, t0 + 1);
    else
      y = x;
    widen(x, 0);
    blank(x.e, 0);
    widen(y, 1);
    blank(y.e, 1);
#pragma unroll
    for (int i = 0; i < NE; ++i) e[i] = x.e[i], en[i] = y.e[i];
    if (t0 + 2 < t1) load(x, t0 + 2);
    __syncthreads();
    f32x16 l = logits(0, 0);
    int buf = 0;
    for (int t = t0; t < t1; ++t) {
      const int b1 = buf == 2 ? 0 : buf + 1, b2 = buf == 0 ? 2 : buf - 1;
      // Matrix products stand beside vector work that does not wait for them: a block's product
      // with V and the logits of the block after the next beside the next one's
      // numerators, the last ones beside the widening. Past the last tile, what is
      // widened and multiplied is not used.
      if (TILE * t < any) {
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          f16x8 p[2];
          const f32x16 ln = n + 1 < NB ? logits(n + 1, buf) : logits(0, b1);
          numerators(l, e[2 * n], e[2 * n + 1], TILE * t + 32 * n, p);
          weigh(p, n, buf);
          l = ln;
        }
        widen(x, b2);
        asm volatile("; beside the last products");  // not merged with the other copy
      } else {
        widen(x, b2);
        asm volatile("; alone");
      }
#pragma unroll
      for (int i = 0; i < NE; ++i) e[i] = en[i];
      if (t + 2 < t1) {
        blank(x.e, b2);
#pragma unroll
        for (int i = 0; i < NE; ++i) en[i] = x.e[i];
        if (t + 3 < t1) load(x, t + 3);
      }
      __syncthreads();  // the tile after next is in place, and this one's readers are done
      buf = b1;
    }
  }

  {
    const int s = __float_as_int(S);
    const auto r = __builtin_amdgcn_permlane32_swap(s, s, false, false);
    S = __int_as_float(r[0]) + __int_as_float(r[1]);
  }
  if (row >= R) return;
  const bool has = some && seen > 0;
  if (!has) M = neg_inf(), S = 0.f;
  if (active == 1) {
    const int64_t out = ((int64_t)b * a.Hq + h * G + qg) * a.N + qi;
    const float f = S != 0.f ? 1.f / S : 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        f32x8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = has ? o[d][4 * (i & 3) + 2 * n + (i >> 2)] * f : 0.f;
        *reinterpret_cast<bf16x8*>(a.o + out * D + 32 * d + 16 * hi + 8 * n) = __builtin_convertvector(v, bf16x8);
      }
    if (hi == 0) a.lse[out] = S > 0.f || S != S ? (M + __builtin_amdgcn_logf(S)) * kLn2 : neg_inf();
  } else {
    const int64_t at = ((int64_t)list * R + row) * splits + split;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        f32x8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = has ? o[d][4 * (i & 3) + 2 * n + (i >> 2)] : 0.f;
        *reinterpret_cast<f32x8*>(a.workspace + at * D + 32 * d + 16 * hi + 8 * n) = v;
      }
    float* ms = a.workspace + (int64_t)a.c.B * a.c.H * R * splits * D + 2 * at;
    if (hi == 0) ms[0] = M, ms[1] = S;
  }
}

// Joins a row's splits: J groups of D / 8 threads a row, each with every J-th split.
template <int D, int J>
__global__ __launch_bounds__(256) void cache_attn_join_kernel(CacheAttnLaunch a, int splits, int tile, int least) {
  constexpr int C = D / 8, ROWS = 256 / C / J;
  __shared__ float y_sh[ROWS][J][D], m_sh[ROWS][J], z_sh[ROWS][J];
  const int G = a.Hq / a.c.H, R = G * a.N;
  const int d0 = 8 * (threadIdx.x % C), j = threadIdx.x / C % J, rr = threadIdx.x / C / J;
  const int64_t row = (int64_t)blockIdx.x * ROWS + rr;
  const bool there = row < (int64_t)a.c.B * a.c.H * R;
  const int list = there ? (int)(row / R) : 0, r = (int)(row % R);
  // Every part's sums are asked for before it is known which of them the list has: the time is
  // the latency of these loads. Parts that are not there are left out below.
  constexpr int K = J > 1 ? kMaxSplits / J : kFewParts - 1;
  const float* ms = a.workspace + (int64_t)a.c.B * a.c.H * R * splits * D + 2 * row * splits;
  const float* po = a.workspace + row * splits * D + d0;
  f32x2 mz[K];
  f32x8 part[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int s = j + J * k;
    if (there && s < splits) {
      mz[k] = *reinterpret_cast<const f32x2*>(ms + 2 * s);
      part[k] = *reinterpret_cast<const f32x8*>(po + (int64_t)s * D);
    }
  }
  const int L = clampi(a.held[list], 0, a.c.max_pages * a.c.P);
  const int tiles = (L + tile - 1) / tile, per = split_tiles(tiles, splits, least), active = (tiles + per - 1) / per;
  const bool work = there && active > 1;  // else the workgroup of the only part wrote the row
  float m = neg_inf(), z = 0.f;
  f32x8 y = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (work) {
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (j + J * k < active) m = fmaxf(m, mz[k][0]);
    const float mu = m == neg_inf() ? 0.f : m;
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (j + J * k < active) {
        const float f = __builtin_amdgcn_exp2f(mz[k][0] - mu);
        z = __builtin_fmaf(f, mz[k][1], z);
#pragma unroll
        for (int t = 0; t < 8; ++t) y[t] = __builtin_fmaf(f, part[k][t], y[t]);
      }
  }
  if constexpr (J > 1) {
    *reinterpret_cast<f32x8*>(&y_sh[rr][j][d0]) = y;
    if (d0 == 0) m_sh[rr][j] = m, z_sh[rr][j] = z;
    __syncthreads();
    if (j != 0 || !work) return;
#pragma unroll
    for (int i = 1; i < J; ++i) m = fmaxf(m, m_sh[rr][i]);
    const float mu = m == neg_inf() ? 0.f : m;
    z = 0.f;
    y = f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < J; ++i) {
      const float f = __builtin_amdgcn_exp2f(m_sh[rr][i] - mu);
      z = __builtin_fmaf(f, z_sh[rr][i], z);
#pragma unroll
      for (int t = 0; t < 8; ++t) y[t] = __builtin_fmaf(f, y_sh[rr][i][d0 + t], y[t]);
    }
  } else if (!work) {
    return;
  }
  const float f = z != 0.f ? 1.f / z : 0.f;
  const int64_t out = ((int64_t)(list / a.c.H) * a.Hq + (list % a.c.H) * G + r % G) * a.N + r / G;
  y *= f;
  *reinterpret_cast<bf16x8*>(a.o + out * D + d0) = __builtin_convertvector(y, bf16x8);
  if (d0 == 0) a.lse[out] = z > 0.f || z != z ? (m + __builtin_amdgcn_logf(z)) * kLn2 : neg_inf();
}

// Which kernel, and how many workgroups share a list (us on one MI355X, D = 128, int8, 64
// tokens a page, G = 4 unless said).
//
// The chunk kernel costs a wave's worth of matrix products per 32 rows but widens a tile once per
// 256; the other one reads a list once per 16 rows. Lists of 4096 tokens, (lists, rows), chunk
// and other: (8, 80) 19.8 and 17.1, (16, 80) 24.1 and 23.5; (32, 48) 24.8 and 25.8, (32, 32)
// 23.1 and 20.8; (64, 48) 36.6 and 36.6, (128, 48) 57.5 and 69.3, (128, 32) 55.6 and 43.9; of
// 8192, (8, 96) 26.0 and 28.1. It gets one workgroup per CU, parts of at least 4 tiles. The number
// of parts is rounded down, so that a call whose workgroups are not a divisor of 256 leaves CUs without
// work: 32 heads over 8 lists of 32768, 1024 queries (128 workgroups x 2 parts) 559, 2048 1051, 4096 2000,
// but 700 (88 x 2) 525, 1025 (136) 990, 1536 (192) 998, 2304 (288) 1995; 512 (64 x 4, more to join) 353.
//
// The other kernel's time is the lists' bytes. With at most one workgroup per CU it takes 8 waves
// (lists of 2276 tokens: 256 of them 27.7, 4 waves 32.0; 136 22.6 and 29.8); beyond, as
// many workgroups of 4 waves as fit: at D = 128 a second one of 8 waves does not fit a CU's registers
// (320 lists 40.5, 8 waves 45.7), at D = 64 it does (384 28.5, 8 waves 25.4; 640 35.7 and
// 38.1). Fewer lists than CUs are split until each CU has a part, which costs a
// second launch: not for lists of up to 512 tokens (8 of 384: 8.6, split 9.7-10.1; 512 9.7 and 9.7;
// 640 10.8 and 9.8). Parts of less than 2 tiles a wave go to workgroups of 4 waves with at least
// one each (8 lists of 2276: 18 parts 10.2, 9 of 8 waves 10.7; 32 of 4096, 8 parts: 8
// waves 14.4, 4 waves 15.3).
struct Plan {
  bool chunk;
  int row_blocks, waves, splits;
};
constexpr int kCus = 256;
Plan plan(const CacheAttnLaunch& L) {
  Plan p;
  const int64_t lists = (int64_t)L.c.B * L.c.H, R = (int64_t)(L.Hq / L.c.H) * L.N;
  const int64_t room = (int64_t)L.c.max_pages * L.c.P;
  p.chunk = R > 80 || (R > 32 && lists >= 32);
  if (p.chunk) {
    p.waves = kChunkWaves;
    p.row_blocks = (int)((R + kChunkRows - 1) / kChunkRows);
    const int64_t blocks = lists * p.row_blocks, tiles = (room + chunk_tile(L.c.D) - 1) / chunk_tile(L.c.D);
    int64_t s = blocks < kCus ? kCus / blocks : 1;
    s = s < tiles / 4 ? s : tiles / 4;
    p.splits = (int)(s < 1 ? 1 : s > kMaxSplits ? kMaxSplits : s);
    return p;
  }
  p.row_blocks = (int)((R + kRows - 1) / kRows);
  const int64_t blocks = lists * p.row_blocks, tiles = (room + kTile - 1) / kTile;
  p.splits = 1;
  p.waves = 4;
  if (tiles <= 16 || blocks > (L.c.D == 64 ? 2 : 1) * kCus) return p;
  int64_t s = blocks < kCus ? kCus / blocks : 1;
  if (tiles >= 16 * s)
    p.waves = 8;
  else
    s = s < tiles / 4 ? s : tiles / 4;
  p.splits = (int)(s < kMaxSplits ? s : kMaxSplits);
  return p;
}

template <int D, int FMT>
int launch_attn(const CacheAttnLaunch& L) {
  const Plan p = plan(L);
  const dim3 grid((unsigned)(L.c.B * L.c.H * p.row_blocks * p.splits)), block(64 * p.waves);
  const hipStream_t st = (hipStream_t)L.stream;
  if (p.chunk)
    hipLaunchKernelGGL((cache_attn_chunk_kernel<D, FMT>), grid, block, 0, st, L, p.row_blocks, p.splits);
  else if (p.waves == 8)
    hipLaunchKernelGGL((cache_attn_kernel<D, FMT, 8>), grid, block, 0, st, L, p.row_blocks, p.splits);
  else
    hipLaunchKernelGGL((cache_attn_kernel<D, FMT, 4>), grid, block, 0, st, L, p.row_blocks, p.splits);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess || p.splits == 1) return (int)e;
  // Several parts are read by 8 groups of threads each row, two or three by one.
  const int64_t rows = (int64_t)L.c.B * L.Hq * L.N;
  const int tile = p.chunk ? chunk_tile(D) : kTile, least = p.chunk ? 1 : kMinTiles * p.waves;
  constexpr int kMost = 2048 / D;  // rows a workgroup with one group a row
  if (p.splits >= kFewParts)
    hipLaunchKernelGGL((cache_attn_join_kernel<D, 8>), dim3((unsigned)((8 * rows + kMost - 1) / kMost)), dim3(256), 0, st,
                       L, p.splits, tile, least);
  else
    hipLaunchKernelGGL((cache_attn_join_kernel<D, 1>), dim3((unsigned)((rows + kMost - 1) / kMost)), dim3(256), 0, st, L,
                       p.splits, tile, least);
  return (int)hipGetLastError();
}

}  // namespace

int64_t cache_attn_threads(const CacheAttnLaunch& L) {
  const Plan p = plan(L);
  return (int64_t)L.c.B * L.c.H * p.row_blocks * p.splits * (64 * p.waves);
}

int64_t cache_attn_workspace_floats(const CacheAttnLaunch& L) {
  const Plan p = plan(L);
  return p.splits == 1 ? 0 : (int64_t)L.c.B * L.Hq * L.N * p.splits * (L.c.D + 2);
}

int launch_cache_attn(const CacheAttnLaunch& L) {
  const bool i8 = L.c.format == KVPOP_CACHE_INT8;
  if (L.c.D == 64) return i8 ? launch_attn<64, KVPOP_CACHE_INT8>(L) : launch_attn<64, KVPOP_CACHE_E4M3>(L);
  return i8 ? launch_attn<128, KVPOP_CACHE_INT8>(L) : launch_attn<128, KVPOP_CACHE_E4M3>(L);
}

}  // namespace kvpop
