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

constexpr int kTile = 32;   // keys per wave
constexpr int kWaves = 4;

// One wave: 32 keys of a list, which stay in registers, against all queries of the KV head,
// 16 (token, head) rows at a time (tokens slowest). S = K Q^T puts keys on the accumulator's rows and
// queries on its columns; a lane adds up its column's probabilities and the 16 lanes of a row join
// at the end. Nothing is shared between waves, and a mass has one writer.
template <int D, int FMT>
__global__ __launch_bounds__(64 * kWaves) void cache_mass_kernel(CacheMassLaunch a, int blocks) {
  constexpr int KS = D / 32, KW = D / 16;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int g = lane >> 4, c = lane & 15;
  const int list = blockIdx.x / blocks, t = (blockIdx.x % blocks) * kWaves + wave;
  const int b = list / a.c.H, h = list % a.c.H, G = a.Hq / a.c.H;
  const int lgP = 31 - __builtin_clz(a.c.P);
  const int L = clampi(a.held[list], 0, a.c.max_pages * a.c.P);
  const int key0 = kTile * t;
  if (key0 >= min(L, a.S)) return;
  const int nq = a.q_lens ? clampi(a.q_lens[b], 0, a.N) : a.N;

  int id[2];
  float ke[2];
  H8 k[2][KS];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int key = key0 + 16 * s, at = key >> lgP;
    id[s] = key < L ? a.c.table[(int64_t)list * a.c.max_pages + at] : -1;
    if ((unsigned)id[s] >= (unsigned)a.c.n_pages) id[s] = -1;
    const int page = max(id[s], 0);
    ke[s] = (float)clampi(a.c.ke[page], kExpMin, kExpMax);
    const uint8_t* kp = a.c.k + (((int64_t)page << lgP) + (key & (a.c.P - 1)) + c) * D + (D / 4) * g;
    Words<4> w[KW / 4];
#pragma unroll
    for (int i = 0; i < KW / 4; ++i) w[i] = *reinterpret_cast<const Words<4>*>(kp + 16 * i);
#pragma unroll
    for (int m = 0; m < KS; ++m) {
      widen4<FMT>(w[m / 2].w[2 * (m % 2)], k[s][m].h[0], k[s][m].h[1]);
      widen4<FMT>(w[m / 2].w[2 * (m % 2) + 1], k[s][m].h[2], k[s][m].h[3]);
    }
  }

  float sum[2][4] = {};
  const int R = G * nq;
  for (int r0 = 0; r0 < R; r0 += 16) {
    const int row = r0 + c, qi = row / G, qh = h * G + row % G;
    const bool some = row < R;
    const int seen = some ? L - (nq - 1 - qi) : 0;
    float lse = some ? a.lse[((int64_t)b * a.Hq + qh) * a.N + qi] : 0.f;
    lse = lse == neg_inf() ? -neg_inf() : lse * kLog2e;
    float x[KS][8], big = 0.f;
#pragma unroll
    for (int m = 0; m < KS; ++m) {
      uint4 w = {0, 0, 0, 0};
      if (some)
        w = *reinterpret_cast<const uint4*>(a.q.ptr + b * a.q.sb + qh * a.q.sh + qi * a.q.st + (D / 4) * g + 8 * m);
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
    // Queries in f16: their largest element in [2^14, 2^15), so that elements down to 2^-28 of it
    // keep their 8 bits (as in the attention that made lse).
    const int e = big > 0.f ? __builtin_amdgcn_frexp_expf(big) - 15 : 0;
    const float cq = __builtin_ldexpf(a.scale * kLog2e, e);
    H8 q[KS];
#pragma unroll
    for (int m = 0; m < KS; ++m)
#pragma unroll
      for (int i = 0; i < 8; ++i) q[m].v[i] = (_Float16)__builtin_ldexpf(x[m][i], -e);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int m = 0; m < KS; ++m) acc = mfma16(k[s][m].v, q[m].v, acc);
      const float kc = __builtin_ldexpf(cq, (int)ke[s]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const bool in = id[s] >= 0 && key0 + 16 * s + 4 * g + r < seen;
        sum[s][r] += in ? __builtin_amdgcn_exp2f(__builtin_fmaf(acc[r], kc, -lse)) : 0.f;
      }
    }
  }
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) sum[s][r] += __shfl_xor(sum[s][r], o);
  // Lane c < 4 of a group has its key 4 g + c.
  float* mass = a.mass + (int64_t)list * a.S;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const float add = c == 0 ? sum[s][0] : c == 1 ? sum[s][1] : c == 2 ? sum[s][2] : sum[s][3];
    const int key = key0 + 16 * s + 4 * g + c;
    if (c < 4 && key < min(L, a.S)) mass[key] = a.decay > 0.f ? __builtin_fmaf(a.decay, mass[key], add) : add;
  }
}

int mass_blocks(const CacheMassLaunch& L) {
  const int64_t slots = (int64_t)L.c.max_pages * L.c.P < L.S ? (int64_t)L.c.max_pages * L.c.P : L.S;
  return (int)((slots + kTile * kWaves - 1) / (kTile * kWaves));
}

template <int D, int FMT>
int launch_mass(const CacheMassLaunch& L) {
  const int blocks = mass_blocks(L);
  hipLaunchKernelGGL((cache_mass_kernel<D, FMT>), dim3((unsigned)(L.c.B * L.c.H * blocks)), dim3(64 * kWaves), 0,
                     (hipStream_t)L.stream, L, blocks);
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

// One workgroup per list: the topk-th key (in the order of mass_key) digit by digit, 8 bits at a time, from counts
// in LDS, then a stable compaction of what is at or before it; each wave has a run of the tokens.
__global__ __launch_bounds__(kPickThreads) void mass_pick_kernel(MassPromptLaunch a) {
  __shared__ __align__(16) int hist[256];
  __shared__ int keep_sh[kPickWaves], equal_sh[kPickWaves];
  __shared__ uint32_t prefix_sh;
  __shared__ int need_sh;
  const int list = blockIdx.x, b = list / a.H, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int n = a.lens ? clampi(a.lens[b], 0, a.T) : a.T;
  const float* x = a.sums + (int64_t)list * a.T;
  int32_t* pos = a.pos + (int64_t)list * a.S;
  float* prio = a.prio + (int64_t)list * a.S;
  const int lo = min(a.sinks, n), hi = max(lo, (int)max((int64_t)n - a.window, (int64_t)lo));
  const bool all = hi - lo <= a.topk;
  uint32_t prefix = 0;
  int need = min(a.topk, hi - lo);  // how many of those that begin with `prefix` are kept
  if (!all)
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int t = lo + tid; t < hi; t += kPickThreads) {
        const uint32_t k = mass_key(x[t]);
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1);
      }
      __syncthreads();
      if (wave == 0) {  // four bins a lane: the one where the counts reach `need`
        const int4 c = *reinterpret_cast<const int4*>(hist + 4 * lane);
        const int mine = c.x + c.y + c.z + c.w;
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const int y = __shfl_up(upto, o);
          if (lane >= o) upto += y;
        }
        const int before = upto - mine;
        if (before < need && need <= upto) {
          int rest = need - before, d = 0;
          const int each[3] = {c.x, c.y, c.z};
#pragma unroll
          for (int i = 0; i < 3; ++i)
            if (d == i && rest > each[i]) rest -= each[i], ++d;
          prefix_sh = prefix | ((uint32_t)(4 * lane + d) << shift);
          need_sh = rest;
        }
      }
      __syncthreads();
      prefix = prefix_sh, need = need_sh;
    }

  // Tokens before the cutoff key are kept, and of those that have it the first `need`.
  const int span = ((n + kPickThreads - 1) / kPickThreads) * 64;
  const int t0 = min(n, wave * span), t1 = min(n, t0 + span);
  int kept = 0, equal = 0;
  for (int t = t0 + lane; t < t1; t += 64) {
    const bool mid = t >= lo && t < hi && !all;
    const uint32_t k = mid ? mass_key(x[t]) : 0u;
    kept += !mid || k < prefix;
    equal += mid && k == prefix;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    kept += __shfl_xor(kept, o);
    equal += __shfl_xor(equal, o);
  }
  if (lane == 0) keep_sh[wave] = kept, equal_sh[wave] = equal;
  __syncthreads();
  int at = 0, eq = 0;
  for (int w = 0; w < wave; ++w) {
    at += keep_sh[w] + max(0, min(need - eq, equal_sh[w]));
    eq += equal_sh[w];
  }
  auto below = [&](uint64_t m) __attribute__((always_inline)) {
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
  };
  for (int first = t0; first < t1; first += 64) {
    const int t = first + lane;
    const bool in = t < t1, mid = in && t >= lo && t < hi && !all;
    const float v = in ? x[t] : 0.f;
    const uint32_t k = mid ? mass_key(v) : 0u;
    const uint64_t ties = __builtin_amdgcn_ballot_w64(mid && k == prefix);
    const bool keep = in && (!mid || k < prefix || (k == prefix && eq + below(ties) < need));
    const uint64_t m = __builtin_amdgcn_ballot_w64(keep);
    if (keep) {
      pos[at + below(m)] = t;
      prio[at + below(m)] = v;
    }
    at += __builtin_popcountll(m);
    eq += __builtin_popcountll(ties);
  }
  const int held = lo + (n - hi) + min(a.topk, hi - lo);
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
// room reads none.
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

int64_t cache_mass_threads(const CacheMassLaunch& L) { return (int64_t)L.c.B * L.c.H * mass_blocks(L) * 64 * kWaves; }

int launch_cache_mass(const CacheMassLaunch& L) {
  const bool i8 = L.c.format == KVPOP_CACHE_INT8;
  if (L.c.D == 64) return i8 ? launch_mass<64, KVPOP_CACHE_INT8>(L) : launch_mass<64, KVPOP_CACHE_E4M3>(L);
  return i8 ? launch_mass<128, KVPOP_CACHE_INT8>(L) : launch_mass<128, KVPOP_CACHE_E4M3>(L);
}

int64_t mass_prompt_workspace_floats(int64_t B, int64_t H, int64_t Hq, int64_t T) { return Hq == H ? 0 : B * H * T; }

int64_t mass_prompt_threads(const MassPromptLaunch& L) {
  const int64_t lists = (int64_t)L.B * L.H;
  return L.Hq == L.H ? lists * kPickThreads : lists * sum_parts(L.T) * kSumThreads;
}

int launch_mass_prompt(const MassPromptLaunch& in) {
  MassPromptLaunch L = in;
  const hipStream_t st = (hipStream_t)L.stream;
  L.sums = L.mass;
  if (L.Hq != L.H) {
    const int parts = sum_parts(L.T);
    hipLaunchKernelGGL(mass_sum_kernel, dim3((unsigned)(L.B * L.H * parts)), dim3(kSumThreads), 0, st, L, parts);
    const int e = (int)hipGetLastError();
    if (e != 0) return e;
    L.sums = L.workspace;
  }
  hipLaunchKernelGGL(mass_pick_kernel, dim3((unsigned)(L.B * L.H)), dim3(kPickThreads), 0, st, L);
  return (int)hipGetLastError();
}

int64_t mass_step_threads(const RetainLaunch& L) { return (int64_t)L.B * L.H * kStepThreads; }

int launch_mass_step(const RetainLaunch& L) {
  hipLaunchKernelGGL(mass_step_kernel, dim3((unsigned)(L.B * L.H)), dim3(kStepThreads), 0, (hipStream_t)L.stream, L);
  return (int)hipGetLastError();
}

}  // namespace kvpop
