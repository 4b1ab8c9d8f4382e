// gfx950 kernels of eviction by accumulated attention weight (include/kvpop_mass.h):
//
//   mass_j <- decay mass_j + sum_i exp(scale <q_i, k_j> - lse_i)   over the compact cache's lists,
//   the tokens that a prompt keeps by their masses, and the slot for a new token.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kvpop_cache.h"
#include "kvpop_cache_codes.h"
#include "kvpop_internal.h"

namespace kvpop {
namespace {

// The order of masses: that of desc_key, NaN of either sign above +inf (which sign a sum's NaN has
// is not defined).
__device__ __forceinline__ uint32_t mass_key(float x) { return x != x ? 0u : desc_key(x); }

constexpr int kWaves = 4;
constexpr int kQueries = 128;  // (token, head) rows that a workgroup shares at a time

// 16 keys of a list, widened to 16 bits, and what is known of them.
template <int D, int FMT>
struct Keys {
  Words<4> w[D / 64];
  H8 k[D / 32];
  float e;
  bool page;
  // Their page (uniform), -1 for none, then their codes.
  static __device__ __forceinline__ int page_of(const CacheMassLaunch& a, int list, int key, int L, int lgP) {
    const int id = key < L ? a.c.table[(int64_t)list * a.c.max_pages + (key >> lgP)] : -1;
    return (unsigned)id < (unsigned)a.c.n_pages ? id : -1;
  }
  __device__ __forceinline__ void load(const CacheMassLaunch& a, int id, int key, int lgP, int g, int c) {
    page = id >= 0;
    id = max(id, 0);
    e = (float)clampi(a.c.ke[id], kExpMin, kExpMax);
    const uint8_t* p = a.c.k + (((int64_t)id << lgP) + (key & (a.c.P - 1)) + c) * D + (D / 4) * g;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) w[i] = *reinterpret_cast<const Words<4>*>(p + 16 * i);
  }
  __device__ __forceinline__ void widen() {
#pragma unroll
    for (int m = 0; m < D / 32; ++m) {
      widen4<FMT>(w[m / 2].w[2 * (m % 2)], k[m].h[0], k[m].h[1]);
      widen4<FMT>(w[m / 2].w[2 * (m % 2) + 1], k[m].h[2], k[m].h[3]);
    }
  }
};

// N elements of a query from `at` on: their largest magnitude, then f16 with e taken out.
template <int N>
struct QueryPart {
  float x[N];
  __device__ __forceinline__ float load(const uint16_t* at, bool some) {
    float big = 0.f;
#pragma unroll
    for (int m = 0; m < N / 8; ++m) {
      uint4 w = {0, 0, 0, 0};
      if (some) w = *reinterpret_cast<const uint4*>(at + 8 * m);
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[8 * m + 2 * i] = __uint_as_float(u[i] << 16);
        x[8 * m + 2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) big = fmaxf(big, __builtin_fabsf(x[i]));
    return big;
  }
  __device__ __forceinline__ void half(H8* to, int e) const {
#pragma unroll
    for (int i = 0; i < N; ++i) to[i / 8].v[i % 8] = (_Float16)__builtin_ldexpf(x[i], -e);
  }
};
// Queries in f16: their largest element in [2^14, 2^15), so that elements down to 2^-28 of it keep their 8
// bits (as in the attention that made lse).
__device__ __forceinline__ int query_exponent(float big) {
  return big > 0.f ? __builtin_amdgcn_frexp_expf(big) - 15 : 0;
}
// lse in units of log2; a query that saw nothing gives nothing.
__device__ __forceinline__ float lse2(float x) { return x == neg_inf() ? -neg_inf() : x * kLog2e; }

// One workgroup: 4 waves of 16 KT keys each, which stay in registers, against all queries of the KV head
// ((token, head) rows, tokens slowest). S = K Q^T puts keys on the accumulator's rows and queries on its
// columns; a lane adds up its column's probabilities and the 16 lanes of a row join at the end. Nothing is
// shared between workgroups, and a mass has one writer.
// MANY: rows pass through LDS in f16, 128 at a time, widened once, and 8 waves take them: two for
// each 16 KT keys, with half of the rows each (a lane's chain of sums is the time; twice the waves hide it).
// Else (16 rows at most) each wave takes them from memory.
// Few rows: codes are read once, and the waits for length, page and codes, one after the other, bound it: 64 x 8 lists
// of up to 2276 tokens of 128 in e4m3 23 us. Many rows: the chain of a workgroup's rows, 128 after 128, with two waves a SIMD
// on as many CUs as there are blocks of 128 keys: 500 queries of 7 heads on 6 lists of up to 9001 (D = 64, int8; 163 such blocks see them) 67 us,
// where the exponentials and their sums (about 6 vector instructions a pair) would take 13-17 spread over all CUs.
template <int D, int FMT, int KT, bool MANY>
__global__ __launch_bounds__(64 * kWaves * (MANY ? 2 : 1)) void cache_mass_kernel(CacheMassLaunch a, int blocks) {
  constexpr int KS = D / 32, QS = D + 8;
  __shared__ __align__(16) uint16_t q_sh[MANY ? kQueries * QS : 8];
  __shared__ float c_sh[MANY ? kQueries : 1], lse_sh[MANY ? kQueries : 1], half_sh[MANY ? kWaves * 16 * KT : 1];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane((tid >> 6) % kWaves), half = __builtin_amdgcn_readfirstlane(tid / (64 * kWaves));
  const int g = lane >> 4, c = lane & 15;
  const int list = blockIdx.x / blocks, key0 = ((blockIdx.x % blocks) * kWaves + wave) * 16 * KT;
  const int b = list / a.c.H, h = list % a.c.H, G = a.Hq / a.c.H;
  const int lgP = 31 - __builtin_clz(a.c.P);
  const int L = clampi(a.held[list], 0, a.c.max_pages * a.c.P), end = min(L, a.S);
  if ((blockIdx.x % blocks) * kWaves * 16 * KT >= end) return;
  if (!MANY && key0 >= end) return;
  const int nq = a.q_lens ? clampi(a.q_lens[b], 0, a.N) : a.N, R = G * nq;

  Keys<D, FMT> k[KT];
  int id[KT];
#pragma unroll
  for (int s = 0; s < KT; ++s) id[s] = k[s].page_of(a, list, key0 + 16 * s, L, lgP);
#pragma unroll
  for (int s = 0; s < KT; ++s) k[s].load(a, id[s], key0 + 16 * s, lgP, g, c);

  // The old masses are on their way meanwhile. Lane c < 4 of a group has its key 4 g + c.
  float* mass = a.mass + (int64_t)list * a.S;
  float old[KT];
#pragma unroll
  for (int s = 0; s < KT; ++s) old[s] = a.decay > 0.f ? mass[min(key0 + 16 * s + 4 * g + (c & 3), end - 1)] : 0.f;

  float sum[KT][4] = {};
  // 16 rows from r0 on against the wave's keys; `edge`: some row may not see some key, or a page is missing.
  auto add = [&](const H8 (&q)[KS], float cq, float lse, int row, bool edge) __attribute__((always_inline)) {
    const int seen = row < R ? L - (nq - 1 - row / G) : 0;
#pragma unroll
    for (int s = 0; s < KT; ++s) {
      if (!MANY) k[s].widen();
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int m = 0; m < KS; ++m) acc = mfma16(k[s].k[m].v, q[m].v, acc);
      const float kc = __builtin_ldexpf(cq, (int)k[s].e);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[r], kc, -lse));
        sum[s][r] += !edge || (k[s].page && key0 + 16 * s + 4 * g + r < seen) ? p : 0.f;
      }
    }
  };
  if constexpr (!MANY) {
    const int qi = c / G, qh = h * G + c % G;
    const bool some = c < R;
    QueryPart<D / 4> x;
    const float big = max_groups(x.load(a.q.ptr + b * a.q.sb + qh * a.q.sh + qi * a.q.st + (D / 4) * g, some));
    const int e = query_exponent(big);
    H8 q[KS];
    x.half(q, e);
    const float lse = some ? lse2(a.lse[((int64_t)b * a.Hq + qh) * a.N + qi]) : 0.f;
    add(q, __builtin_ldexpf(a.scale * kLog2e, e), lse, c, true);
  } else {
#pragma unroll
    for (int s = 0; s < KT; ++s) k[s].widen();
    bool pages = true;
#pragma unroll
    for (int s = 0; s < KT; ++s) pages = pages && id[s] >= 0;
    // Four threads a row.
    const int mine = tid >> 2, part = (tid & 3) * (D / 4);
    QueryPart<D / 4> x;
    float big, lse;
    auto fetch = [&](int r0) __attribute__((always_inline)) {
      const int row = r0 + mine, qi = row / G, qh = h * G + row % G;
      const bool some = row < R;
      big = x.load(a.q.ptr + b * a.q.sb + qh * a.q.sh + qi * a.q.st + part, some);
      lse = some ? a.lse[((int64_t)b * a.Hq + qh) * a.N + qi] : 0.f;
    };
    if (R > 0) fetch(0);
    for (int r0 = 0; r0 < R; r0 += kQueries) {
      big = fmaxf(big, __shfl_xor(big, 1));
      big = fmaxf(big, __shfl_xor(big, 2));
      const int e = query_exponent(big);
      H8 y[D / 32];
      x.half(y, e);
      __syncthreads();
#pragma unroll
      for (int m = 0; m < D / 32; ++m) *reinterpret_cast<f16x8*>(q_sh + mine * QS + part + 8 * m) = y[m].v;
      if ((tid & 3) == 0) c_sh[mine] = __builtin_ldexpf(a.scale * kLog2e, e), lse_sh[mine] = lse2(lse);
      __syncthreads();
      if (r0 + kQueries < R) fetch(r0 + kQueries);
      // All of these rows see all of the wave's keys (the first sees the fewest).
      const bool whole = pages && r0 + kQueries <= R && key0 + 16 * KT <= L - (nq - 1 - r0 / G);
#pragma unroll
      for (int x = 0; x < kQueries / 2; x += 16) {
        const int i = half * (kQueries / 2) + x;
        H8 q[KS];
#pragma unroll
        for (int m = 0; m < KS; ++m) q[m].v = *reinterpret_cast<const f16x8*>(q_sh + (i + c) * QS + (D / 4) * g + 8 * m);
        if (whole)
          add(q, c_sh[i + c], lse_sh[i + c], r0 + i + c, false);
        else
          add(q, c_sh[i + c], lse_sh[i + c], r0 + i + c, true);
      }
    }
  }
  // The sum over a row's 16 lanes: pairs exchange what the other keeps, so that lane c ends with its key 4 g + (c & 3).
  float mine[KT];
#pragma unroll
  for (int s = 0; s < KT; ++s) {
    const bool odd = c & 1, high = c & 2;
    const float x = (odd ? sum[s][1] : sum[s][0]) + __shfl_xor(odd ? sum[s][0] : sum[s][1], 1);
    const float y = (odd ? sum[s][3] : sum[s][2]) + __shfl_xor(odd ? sum[s][2] : sum[s][3], 1);
    float z = (high ? y : x) + __shfl_xor(high ? x : y, 2);
    z += __shfl_xor(z, 4);
    mine[s] = z + __shfl_xor(z, 8);
  }
  if constexpr (MANY) {
#pragma unroll
    for (int s = 0; s < KT; ++s)
      if (half && c < 4) half_sh[(wave * KT + s) * 16 + 4 * g + c] = mine[s];
    __syncthreads();
    if (half) return;
  }
#pragma unroll
  for (int s = 0; s < KT; ++s) {
    const float more = mine[s] + (MANY ? half_sh[MANY ? (wave * KT + s) * 16 + 4 * g + (c & 3) : 0] : 0.f);
    const int key = key0 + 16 * s + 4 * g + c;
    if (c < 4 && key < end) mass[key] = a.decay > 0.f ? __builtin_fmaf(a.decay, old[s], more) : more;
  }
}

// 64 keys a wave for few rows: more codes on their way at once (64 x 8 lists above 24.2 us, with 32 26.2). 32 for many, where the
// keys and their sums have to stay in registers and the CUs need waves (500 queries above 67.7 us, with 64 96, with 16
// 66-68 at twice the reads of rows from LDS).
bool many_rows(const CacheMassLaunch& L) { return (int64_t)L.Hq / L.c.H * L.N > 16; }
int mass_keys(const CacheMassLaunch& L) { return kWaves * (many_rows(L) ? 32 : 64); }
int mass_blocks(const CacheMassLaunch& L) {
  const int64_t slots = (int64_t)L.c.max_pages * L.c.P < L.S ? (int64_t)L.c.max_pages * L.c.P : L.S;
  return (int)((slots + mass_keys(L) - 1) / mass_keys(L));
}

template <int D, int FMT>
int launch_mass(const CacheMassLaunch& L) {
  const int blocks = mass_blocks(L);
  const dim3 grid((unsigned)(L.c.B * L.c.H * blocks)), block(64 * kWaves);
  if (many_rows(L))
    hipLaunchKernelGGL((cache_mass_kernel<D, FMT, 2, true>), grid, dim3(128 * kWaves), 0, (hipStream_t)L.stream, L, blocks);
  else
    hipLaunchKernelGGL((cache_mass_kernel<D, FMT, 4, false>), grid, block, 0, (hipStream_t)L.stream, L, blocks);
  return (int)hipGetLastError();
}

// ---------------------------------------------------------------------------
// What a prompt keeps
// ---------------------------------------------------------------------------

constexpr int kSumThreads = 1024;

// A KV head's masses: its group's summed in 64 bits, in the heads' order.
__global__ __launch_bounds__(kSumThreads) void mass_sum_kernel(MassPromptLaunch a, int parts) {
  const int list = blockIdx.x / parts, b = list / a.H, h = list % a.H, G = a.Hq / a.H;
  const int t = (blockIdx.x % parts) * kSumThreads + threadIdx.x;
  const int n = a.lens ? clampi(a.lens[b], 0, a.T) : a.T;
  if (t >= n) return;
  const float* x = a.mass + ((int64_t)b * a.Hq + h * G) * a.T + t;
  double s = x[0];
  for (int g = 1; g < G; ++g) s += x[(int64_t)g * a.T];
  a.workspace[(int64_t)list * a.T + t] = (float)s;
}

constexpr int kPickThreads = 1024, kPickWaves = kPickThreads / 64;
constexpr int kBins = 2048;  // 11 bits of a key: the first of them spread masses over some tens of bins
constexpr int kMostEach = 32;  // tokens per thread that stay in registers

// A list's keys (mass_key; kNoKey outside [lo, hi), which is behind every key): EACH tokens of a thread in registers, whose
// masses are read and summed once, or (EACH = 0) from memory in every pass. Token `i` of a thread is
// t0 + 64 i; each wave has a run of the tokens.
constexpr uint32_t kNoKey = 0xFFFFFFFFu;
__device__ __forceinline__ float key_mass(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k : ~k & 0x7FFFFFFFu); }

template <int EACH>
struct ListKeys {
  uint32_t k[EACH > 0 ? EACH : 1];
  const float* at;
  int t0, lo, hi, steps;
  // `edge` gets the tokens of [0, lo) and [hi, n) with their masses.
  template <class F>
  __device__ __forceinline__ ListKeys(const MassPromptLaunch& a, int list, int n, int lo_, int hi_, int wave, int lane, F&& edge)
      : lo(lo_), hi(hi_) {
    if constexpr (EACH > 0) {
      steps = EACH;
      t0 = wave * EACH * 64 + lane;
      const int b = list / a.H, h = list % a.H, G = a.Hq / a.H;
      const float* p = a.mass + ((int64_t)b * a.Hq + h * G) * a.T;
      constexpr int W = EACH < 8 ? EACH : 8;  // tokens of 4 heads whose loads are on their way at once
#pragma unroll
      for (int i0 = 0; i0 < EACH; i0 += W) {
        double s[W] = {};
        for (int g0 = 0; g0 < G; g0 += 4) {
          float y[4][W];
#pragma unroll
          for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int i = 0; i < W; ++i) y[g][i] = p[(int64_t)min(g0 + g, G - 1) * a.T + min(t0 + 64 * (i0 + i), a.T - 1)];
#pragma unroll
          for (int g = 0; g < 4; ++g)
            if (g0 + g < G)
#pragma unroll
              for (int i = 0; i < W; ++i) s[i] = g0 + g == 0 ? (double)y[g][i] : s[i] + y[g][i];
        }
#pragma unroll
        for (int i = 0; i < W; ++i) k[i0 + i] = key(t0 + 64 * (i0 + i), (float)s[i], n, edge);
      }
    } else {
      at = a.sums + (int64_t)list * a.T;
      steps = (n + kPickThreads - 1) / kPickThreads;
      t0 = wave * steps * 64 + lane;
      for (int i = 0; i < steps; ++i)
        if (t0 + 64 * i < n) key(t0 + 64 * i, at[t0 + 64 * i], n, edge);
    }
  }
  template <class F>
  __device__ __forceinline__ uint32_t key(int t, float x, int n, F&& edge) const {
    if (t >= lo && t < hi) return mass_key(x);
    if (t < n) edge(t, x);
    return kNoKey;
  }
  template <class F>
  __device__ __forceinline__ void each(F&& f) const {
    if constexpr (EACH > 0) {
#pragma unroll
      for (int i = 0; i < EACH; ++i) f(t0 + 64 * i, k[i]);
    } else {
      for (int i = 0; i < steps; ++i) {
        const int t = t0 + 64 * i;
        f(t, t >= lo && t < hi ? mass_key(at[t]) : kNoKey);
      }
    }
  }
};

// One workgroup per list: the topk-th key 11, 11 and 10 bits at a time, from counts in LDS, then a stable compaction
// of what is at or before it. The sinks' and the window's slots are known before. The latency of its passes on one CU
// bounds it: prompts of 4096 tokens 8.6 us, of 32768 of 4 heads 26 us.
template <int EACH>
__global__ __launch_bounds__(kPickThreads) void mass_pick_kernel(MassPromptLaunch a) {
  __shared__ __align__(16) int hist[kBins];
  __shared__ int total_sh[kPickWaves], keep_sh[kPickWaves], equal_sh[kPickWaves];
  __shared__ uint32_t prefix_sh;
  __shared__ int need_sh;
  const int list = blockIdx.x, b = list / a.H, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int n = a.lens ? clampi(a.lens[b], 0, a.T) : a.T;
  int32_t* pos = a.pos + (int64_t)list * a.S;
  float* prio = a.prio + (int64_t)list * a.S;
  const int lo = min(a.sinks, n), hi = max(lo, (int)max((int64_t)n - a.window, (int64_t)lo));
  const int middle = min(a.topk, hi - lo), held = lo + middle + (n - hi);
  const ListKeys<EACH> x(a, list, n, lo, hi, wave, lane, [&](int t, float v) {
    const int slot = t < lo ? t : lo + middle + (t - hi);
    pos[slot] = t;
    prio[slot] = v;
  });
  // Keys before `cut` are kept, and of those that are it the first `need`.
  uint32_t cut = kNoKey;
  int need = 0;
  if (hi - lo > a.topk) {
    cut = 0, need = a.topk;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, above = pass == 1 ? 21 : 10;
      const uint32_t bins = pass == 2 ? 1023u : 2047u;
      reinterpret_cast<int2*>(hist)[tid] = int2{0, 0};
      __syncthreads();
      x.each([&](int, uint32_t k) __attribute__((always_inline)) {
        if (pass == 0 ? k != kNoKey : (k >> above) == (cut >> above)) atomicAdd(&hist[(k >> shift) & bins], 1);
      });
      __syncthreads();
      // Two bins a thread: the one where the counts reach `need`.
      const int2 c = reinterpret_cast<const int2*>(hist)[tid];
      const int mine = c.x + c.y;
      int upto = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(upto, o);
        if (lane >= o) upto += y;
      }
      if (lane == 63) total_sh[wave] = upto;
      __syncthreads();
      for (int w = 0; w < wave; ++w) upto += total_sh[w];
      const int before = upto - mine;
      if (before < need && need <= upto) {
        const bool second = need > before + c.x;
        prefix_sh = cut | ((uint32_t)(2 * tid + (second ? 1 : 0)) << shift);
        need_sh = need - before - (second ? c.x : 0);
      }
      __syncthreads();
      cut = prefix_sh, need = need_sh;
    }
  }
  int kept = 0, equal = 0;
  x.each([&](int, uint32_t k) __attribute__((always_inline)) {
    kept += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k < cut));
    equal += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k == cut));
  });
  if (need == 0) equal = 0;
  if (lane == 0) keep_sh[wave] = kept, equal_sh[wave] = equal;
  __syncthreads();
  int at = lo, eq = 0;
  for (int w = 0; w < wave; ++w) {
    at += keep_sh[w] + max(0, min(need - eq, equal_sh[w]));
    eq += equal_sh[w];
  }
  auto below = [&](uint64_t m) __attribute__((always_inline)) {
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
  };
  x.each([&](int t, uint32_t k) __attribute__((always_inline)) {
    bool keep = k < cut;
    const uint64_t ties = __builtin_amdgcn_ballot_w64(k == cut);
    if (ties != 0 && need > 0) {
      keep = keep || (k == cut && eq + below(ties) < need);
      eq += __builtin_popcountll(ties);
    }
    const uint64_t m = __builtin_amdgcn_ballot_w64(keep);
    if (keep) {
      pos[at + below(m)] = t;
      prio[at + below(m)] = key_mass(k);
    }
    at += __builtin_popcountll(m);
  });
  for (int i = held + tid; i < a.S; i += kPickThreads) {
    pos[i] = -1;
    prio[i] = 0.f;
  }
  if (tid == 0) a.held[list] = held;
}

int sum_parts(int T) { return (T + kSumThreads - 1) / kSumThreads; }

// ---------------------------------------------------------------------------
// The slot for a new token
// ---------------------------------------------------------------------------

constexpr int kStepThreads = 256;

// One workgroup per list. A full one reads every slot's position and mass once; the least
// mass that may go is the largest of (key, position) pairs, then the first slot that holds it. One with
// room reads none. 8 lists 6.4 us (latency), 2048 lists of 2276 slots (37 MB) 12.4 us; 512 threads a list, or a
// thread's slots loaded several at a time, are no faster.
__global__ __launch_bounds__(kStepThreads) void mass_step_kernel(RetainLaunch a) {
  __shared__ unsigned long long best_sh[kStepThreads / 64];
  __shared__ int slot_sh[kStepThreads / 64];
  const int list = blockIdx.x, b = list / a.H, tid = threadIdx.x;
  const int q = a.q_pos[b];
  const int held = clampi(a.held[list], 0, a.S);
  if (q < 0) {
    if (tid == 0) a.slot[list] = -1;
    return;
  }
  __syncthreads();  // all have read held before one writes it
  int32_t* pos = a.pos + (int64_t)list * a.S;
  float* mass = a.prio + (int64_t)list * a.S;
  if (held < a.sinks + a.window + a.topk) {
    if (tid == 0) {
      pos[held] = q;
      mass[held] = 0.f;
      a.held[list] = held + 1;
      a.slot[list] = held;
    }
    return;
  }
  const int64_t newest = (int64_t)q - a.window;
  unsigned long long best = 0;  // 0: none (a position is at least 0: its pair is stored + 1)
  int slot = a.S;
  for (int i = tid; i < held; i += kStepThreads) {
    const int p = pos[i];
    const float v = mass[i];
    if (p >= a.sinks && p <= newest) {
      const unsigned long long k = (((unsigned long long)mass_key(v) << 32) | (unsigned)p) + 1;
      if (k > best) best = k, slot = i;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const unsigned long long k = __shfl_xor(best, o);
    const int s = __shfl_xor(slot, o);
    if (k > best || (k == best && s < slot)) best = k, slot = s;
  }
  if ((tid & 63) == 0) best_sh[tid >> 6] = best, slot_sh[tid >> 6] = slot;
  __syncthreads();
  if (tid != 0) return;
  for (int w = 0; w < kStepThreads / 64; ++w)
    if (best_sh[w] > best || (best_sh[w] == best && slot_sh[w] < slot)) best = best_sh[w], slot = slot_sh[w];
  if (best == 0) {
    slot = -1;
  } else {
    pos[slot] = q;
    mass[slot] = 0.f;
  }
  a.slot[list] = slot;
}

}  // namespace

int64_t cache_mass_threads(const CacheMassLaunch& L) { return (int64_t)L.c.B * L.c.H * mass_blocks(L) * 128 * kWaves; }

int launch_cache_mass(const CacheMassLaunch& L) {
  const bool i8 = L.c.format == KVPOP_CACHE_INT8;
  if (L.c.D == 64) return i8 ? launch_mass<64, KVPOP_CACHE_INT8>(L) : launch_mass<64, KVPOP_CACHE_E4M3>(L);
  return i8 ? launch_mass<128, KVPOP_CACHE_INT8>(L) : launch_mass<128, KVPOP_CACHE_E4M3>(L);
}

// Longer prompts are summed first, into the workspace.
constexpr int64_t kLongPrompt = (int64_t)kPickThreads * kMostEach;

int64_t mass_prompt_workspace_floats(int64_t B, int64_t H, int64_t Hq, int64_t T) {
  return Hq == H || T <= kLongPrompt ? 0 : B * H * T;
}

int64_t mass_prompt_threads(const MassPromptLaunch& L) {
  const int64_t lists = (int64_t)L.B * L.H;
  return L.Hq == L.H || L.T <= kLongPrompt ? lists * kPickThreads : lists * sum_parts(L.T) * kSumThreads;
}

int launch_mass_prompt(const MassPromptLaunch& in) {
  MassPromptLaunch L = in;
  const hipStream_t st = (hipStream_t)L.stream;
  const dim3 lists((unsigned)(L.B * L.H)), block(kPickThreads);
  if (L.T <= kPickThreads * 4) {
    hipLaunchKernelGGL((mass_pick_kernel<4>), lists, block, 0, st, L);
  } else if (L.T <= kPickThreads * 8) {
    hipLaunchKernelGGL((mass_pick_kernel<8>), lists, block, 0, st, L);
  } else if (L.T <= kPickThreads * 16) {
    hipLaunchKernelGGL((mass_pick_kernel<16>), lists, block, 0, st, L);
  } else if (L.T <= kLongPrompt) {
    hipLaunchKernelGGL((mass_pick_kernel<kMostEach>), lists, block, 0, st, L);
  } else {
    L.sums = L.mass;
    if (L.Hq != L.H) {
      const int parts = sum_parts(L.T);
      hipLaunchKernelGGL(mass_sum_kernel, dim3((unsigned)(L.B * L.H * parts)), dim3(kSumThreads), 0, st, L, parts);
      const int e = (int)hipGetLastError();
      if (e != 0) return e;
      L.sums = L.workspace;
    }
    hipLaunchKernelGGL((mass_pick_kernel<0>), lists, block, 0, st, L);
  }
  return (int)hipGetLastError();
}

int64_t mass_step_threads(const RetainLaunch& L) { return (int64_t)L.B * L.H * kStepThreads; }

int launch_mass_step(const RetainLaunch& L) {
  hipLaunchKernelGGL(mass_step_kernel, dim3((unsigned)(L.B * L.H)), dim3(kStepThreads), 0, (hipStream_t)L.stream, L);
  return (int)hipGetLastError();
}

}  // namespace kvpop
