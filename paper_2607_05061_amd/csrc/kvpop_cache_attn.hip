// gfx950 attention of new queries over the compact cache's page lists of 8-bit keys and
// values (include/kvpop_cache.h):
//
//   l(i, j) = scale <q_i, k_j>,  k_j = code 2^ke,  v_j = code 2^ve,
//   lse_i   = log sum_j exp l(i, j),   o_i = sum_j exp(l(i, j) - lse_i) v_j.
//
// One pass with a running maximum. A value's power of two goes into the exponent of its
// probability: with x = l log2(e) + ve and M the running maximum of x, the numerators
// p' = 2^(x - M) <= 1 multiply the bare codes, and the normaliser in the same units is
// sum p' 2^-ve. So codes enter the products as they are, exact in 16 bits, whatever
// scales a list's pages have.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kvpop_cache.h"
#include "kvpop_internal.h"

namespace kvpop {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kExpMin = -32, kExpMax = 32;
constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kRows = 16;        // (token, head) rows per workgroup
constexpr int kTile = 32;        // keys per step of a wave
constexpr int kMinTiles = 4;     // least tiles per workgroup of a split list
constexpr int kMaxSplits = 64;
constexpr int kWantBlocks = 1024;

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }
__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }

__device__ __forceinline__ f32x4 mfma16(const f16x8& a, const f16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// The larger of the four lanes l % 16 + 16 k, on all of them.
__device__ __forceinline__ float max_groups(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_groups(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

union H8 {
  f16x8 v;
  f16x2 h[4];
  uint32_t u[4];
};

__device__ __forceinline__ f16x2 as_h2(uint32_t u) {
  union { uint32_t u; f16x2 h; } x;
  x.u = u;
  return x.h;
}

// Four codes of one dword, in 16 bits. A signed byte b as 1024 + (b + 128) is the f16
// with bits 0x6400 | (b ^ 0x80); the difference is exact.
template <int FMT>
__device__ __forceinline__ void widen4(uint32_t w, f16x2& a, f16x2& b) {
  if constexpr (FMT == KVPOP_CACHE_INT8) {
    const uint32_t u = w ^ 0x80808080u;
    const f16x2 off = {(_Float16)1152.f, (_Float16)1152.f};
    a = as_h2(__builtin_amdgcn_perm(u, 0x64646464u, 0x00050004u)) - off;
    b = as_h2(__builtin_amdgcn_perm(u, 0x64646464u, 0x00070006u)) - off;
  } else {
    a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true);
  }
}

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

template <int N>
struct alignas(4 * N) Words {
  uint32_t w[N];
};

// What a list's splits hold: the tiles of each, for a list of n tiles.
__device__ __forceinline__ int split_tiles(int n, int splits) { return max(kMinTiles, (n + splits - 1) / splits); }

// One workgroup: 16 rows (query tokens times the G heads of a KV head, tokens slowest)
// against a run of a list's tiles, which its four waves divide. S^T = K Q^T puts keys on
// the accumulator's rows and queries on its columns, so a lane holds 4 keys of each 16 for
// the query lane % 16; with two such blocks the lane's 8 probabilities are the B operand of
// O^T += V^T P^T as they stand, its contraction index running over the keys
// {4 g .. 4 g + 3, 16 + 4 g ..} of lane group g. A lane loads the D / 16 bytes at D / 16 (lane %
// 16) of each of these keys, so that byte t of its 8 loads is its A operand of the
// product for the head dims t, t + D / 16, ...: no value passes through LDS.
template <int D, int FMT>
__global__ __launch_bounds__(kThreads) void cache_attn_kernel(CacheAttnLaunch a, int row_blocks, int splits) {
  constexpr int KS = D / 32;  // k-steps of the logits
  constexpr int VB = D / 16;  // bytes of a key's value per lane; tiles of 16 head dims
  constexpr int KW = D / 16;  // dwords of a key per lane (D / 4 bytes)
  constexpr int VW = VB / 4;
  __shared__ float o_sh[kWaves][kRows][D + 4];
  __shared__ float m_sh[kWaves][kRows], s_sh[kWaves][kRows];

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
  const int tiles = (L + kTile - 1) / kTile, per = split_tiles(tiles, splits);
  if (split > 0 && split * per >= tiles) return;
  const int active = max(1, (tiles + per - 1) / per);

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

  const int end_wg = min(tiles, (split + 1) * per);
  const int share = (end_wg - split * per + kWaves - 1) / kWaves;
  const int t0 = split * per + wave * share, t1 = min(end_wg, t0 + share);

  struct Tile {
    Words<4> k[2][KW / 4];
    Words<VW> v[2][4];
    int id[2];  // pages, -1: none
    int e[2];   // exponents: key's in the low half, value's in the high half
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
      x.id[s] = __builtin_amdgcn_readlane(ids, at);
      x.e[s] = __builtin_amdgcn_readlane(exps, at);
      const int64_t base = ((int64_t)max(x.id[s], 0) << lgP) + (key & (a.c.P - 1));
      const uint8_t* kp = a.c.k + base * D + c * D + (D / 4) * g;
#pragma unroll
      for (int i = 0; i < KW / 4; ++i) x.k[s][i] = *reinterpret_cast<const Words<4>*>(kp + 16 * i);
      const uint8_t* vp = a.c.v + base * D + 4 * g * D + VB * c;
#pragma unroll
      for (int i = 0; i < 4; ++i) x.v[s][i] = *reinterpret_cast<const Words<VW>*>(vp + i * D);
    }
  };
  auto step = [&](Tile& x, int t) __attribute__((always_inline)) {
    float l[2][4];
    const bool whole = kTile * (t + 1) <= sure && x.id[0] >= 0 && x.id[1] >= 0;
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
      const float kc = __builtin_ldexpf(cq, (int16_t)x.e[s]), ve = (float)(x.e[s] >> 16);
#pragma unroll
      for (int r = 0; r < 4; ++r) l[s][r] = __builtin_fmaf(acc[r], kc, ve);
      if (!whole) {
        const int key = kTile * t + 16 * s + 4 * g;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          l[s][r] = x.id[s] >= 0 && key + r < seen ? l[s][r] : neg_inf();
          if (x.id[s] < 0 || key + r >= L)
#pragma unroll
            for (int i = 0; i < VW; ++i) x.v[s][r].w[i] = 0;
        }
      }
    }
    float mx = fmaxf(fmaxf(fmaxf(l[0][0], l[0][1]), fmaxf(l[0][2], l[0][3])),
                     fmaxf(fmaxf(l[1][0], l[1][1]), fmaxf(l[1][2], l[1][3])));
    mx = max_groups(mx);
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
      const float w = __builtin_ldexpf(1.f, -(x.e[s] >> 16));
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float e = __builtin_amdgcn_exp2f(l[s][r] - mu);
        S = __builtin_fmaf(e, w, S);
        p.v[4 * s + r] = (_Float16)e;
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
    const int first = (kTile * t) >> lgP;
    load_pages(first);
    const int64_t last_key = (int64_t)(first + 64) << lgP;  // of these 64 pages
    const int stop = (int)min((int64_t)t1, last_key / kTile);
    Tile x;
    load(x, t);
    for (; t < stop; ++t) {
      Tile nx;
      if (t + 1 < stop) load(nx, t + 1);
      step(x, t);
      x = nx;
    }
  }

  // The four waves' parts: columns of 16 rows, head dims VB (4 g + r) + t.
  S = sum_groups(S);
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int t = 0; t < VB; ++t) o_sh[wave][c][VB * (4 * g + r) + t] = o[t][r];
  if (g == 0) m_sh[wave][c] = M, s_sh[wave][c] = S;
  __syncthreads();
  const int wr = tid / 16, d0 = (tid % 16) * VB;
  const int orow = rb * kRows + wr, oi = orow / G;
  if (orow >= R) return;
  const bool has = oi < nq && L - (nq - 1 - oi) > 0;
  float m = neg_inf();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) m = fmaxf(m, m_sh[w][wr]);
  const float mu = m == neg_inf() ? 0.f : m;
  float z = 0.f, y[VB];
#pragma unroll
  for (int t = 0; t < VB; ++t) y[t] = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
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

// Joins a row's splits, D / 8 threads a row.
template <int D>
__global__ __launch_bounds__(64) void cache_attn_join_kernel(CacheAttnLaunch a, int splits) {
  const int G = a.Hq / a.c.H, R = G * a.N;
  const int64_t row = (int64_t)blockIdx.x * (512 / D) + threadIdx.x / (D / 8);
  const int d0 = 8 * (threadIdx.x % (D / 8));
  if (row >= (int64_t)a.c.B * a.c.H * R) return;
  const int list = (int)(row / R), r = (int)(row % R);
  const int L = clampi(a.held[list], 0, a.c.max_pages * a.c.P);
  const int tiles = (L + kTile - 1) / kTile, per = split_tiles(tiles, splits), active = (tiles + per - 1) / per;
  if (active <= 1) return;  // the workgroup of the only part wrote the row
  const float* ms = a.workspace + (int64_t)a.c.B * a.c.H * R * splits * D + 2 * row * splits;
  const float* po = a.workspace + row * splits * D + d0;
  float m = neg_inf(), z = 0.f;
  for (int s = 0; s < active; ++s) m = fmaxf(m, ms[2 * s]);
  const float mu = m == neg_inf() ? 0.f : m;
  f32x8 y = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < active; ++s) {
    const float f = __builtin_amdgcn_exp2f(ms[2 * s] - mu);
    z = __builtin_fmaf(f, ms[2 * s + 1], z);
#pragma unroll
    for (int t = 0; t < 8; ++t) y[t] = __builtin_fmaf(f, po[(int64_t)s * D + t], y[t]);
  }
  const float f = z != 0.f ? 1.f / z : 0.f;
  const int64_t out = ((int64_t)(list / a.c.H) * a.Hq + (list % a.c.H) * G + r % G) * a.N + r / G;
  y *= f;
  *reinterpret_cast<bf16x8*>(a.o + out * D + d0) = __builtin_convertvector(y, bf16x8);
  if (d0 == 0) a.lse[out] = z > 0.f || z != z ? (m + __builtin_amdgcn_logf(z)) * kLn2 : neg_inf();
}

struct Plan {
  int row_blocks, splits;
};
Plan plan(const CacheAttnLaunch& L) {
  Plan p;
  const int64_t lists = (int64_t)L.c.B * L.c.H, R = (int64_t)(L.Hq / L.c.H) * L.N;
  p.row_blocks = (int)((R + kRows - 1) / kRows);
  const int64_t blocks = lists * p.row_blocks;
  const int64_t tiles = ((int64_t)L.c.max_pages * L.c.P + kTile - 1) / kTile;
  int64_t s = (kWantBlocks + blocks - 1) / blocks;
  s = s < (tiles + kMinTiles - 1) / kMinTiles ? s : (tiles + kMinTiles - 1) / kMinTiles;
  p.splits = (int)(s < 1 ? 1 : s > kMaxSplits ? kMaxSplits : s);
  return p;
}

template <int D, int FMT>
int launch_attn(const CacheAttnLaunch& L) {
  const Plan p = plan(L);
  hipLaunchKernelGGL((cache_attn_kernel<D, FMT>), dim3((unsigned)cache_attn_blocks(L)), dim3(kThreads), 0,
                     (hipStream_t)L.stream, L, p.row_blocks, p.splits);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess || p.splits == 1) return (int)e;
  const int64_t rows = (int64_t)L.c.B * L.Hq * L.N;
  hipLaunchKernelGGL((cache_attn_join_kernel<D>), dim3((unsigned)((rows + 512 / D - 1) / (512 / D))), dim3(64), 0,
                     (hipStream_t)L.stream, L, p.splits);
  return (int)hipGetLastError();
}

}  // namespace

int64_t cache_attn_blocks(const CacheAttnLaunch& L) {
  const Plan p = plan(L);
  return (int64_t)L.c.B * L.c.H * p.row_blocks * p.splits;
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
