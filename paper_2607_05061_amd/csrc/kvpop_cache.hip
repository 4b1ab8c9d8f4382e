// gfx950 kernels that keep the compact cache of a KVpop model: the append of new keys
// and values to the per-head page lists (rotated, in 8 bits), and the retention that
// says which slot a token takes (include/kvpop_cache.h has the definitions).

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kvpop_cache.h"
#include "kvpop_internal.h"

namespace kvpop {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

constexpr int kExpMin = -32, kExpMax = 32;

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }

__device__ __forceinline__ void unpack8(const uint4& w, float (&x)[8]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = bf16_lo(u[i]);
    x[2 * i + 1] = bf16_hi(u[i]);
  }
}

// ---------------------------------------------------------------------------
// Codes
// ---------------------------------------------------------------------------

// The least e with a <= qmax 2^e, into [kExpMin, kExpMax]; a >= 0 and finite. With a =
// m 2^x, m in [1/2, 1): 127 2^e = (127/128) 2^(e+7) and 448 2^e = (7/8) 2^(e+9).
template <int FMT>
__device__ __forceinline__ int needed_exponent(double a) {
  if (a == 0.0) return kExpMin;
  const double m = __builtin_amdgcn_frexp_mant(a);
  const int x = __builtin_amdgcn_frexp_exp(a);
  const int e = FMT == KVPOP_CACHE_INT8 ? x - (m <= 127.0 / 128.0 ? 7 : 6) : x - (m <= 0.875 ? 9 : 8);
  return clampi(e, kExpMin, kExpMax);
}

// y in 32 bits, rounded to odd where that is inexact, so that a rounding to fewer bits
// that follows is the one rounding of y.
__device__ __forceinline__ float to_odd(double y) {
  const float f = (float)y;
  const double d = (double)f;
  uint32_t b = __float_as_uint(f);
  if (d != y) b = (b - (__builtin_fabs(d) > __builtin_fabs(y) ? 1u : 0u)) | 1u;
  return __uint_as_float(b);
}

// Four codes of y[0..3] (already divided by the scale); NaN gives 0.
template <int FMT>
__device__ __forceinline__ uint32_t codes4(const double* y) {
  if constexpr (FMT == KVPOP_CACHE_INT8) {
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double c = y[i] == y[i] ? __builtin_fmin(__builtin_fmax(y[i], -127.0), 127.0) : 0.0;
      r |= ((uint32_t)(int)__builtin_rint(c) & 0xFFu) << (8 * i);
    }
    return r;
  } else {
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      f[i] = to_odd(y[i] == y[i] ? __builtin_fmin(__builtin_fmax(y[i], -448.0), 448.0) : 0.0);
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], r, true);
  }
}

// Four codes moved to a scale 2^-shift times coarser (shift < 0).
template <int FMT>
__device__ __forceinline__ uint32_t moved4(uint32_t w, int shift) {
  if constexpr (FMT == KVPOP_CACHE_INT8) {
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float c = __builtin_rintf(__builtin_ldexpf((float)(int8_t)(w >> (8 * i)), shift));
      r |= ((uint32_t)(int)c & 0xFFu) << (8 * i);
    }
    return r;
  } else {
    const float f0 = __builtin_ldexpf(__builtin_amdgcn_cvt_f32_fp8(w, 0), shift);
    const float f1 = __builtin_ldexpf(__builtin_amdgcn_cvt_f32_fp8(w, 1), shift);
    const float f2 = __builtin_ldexpf(__builtin_amdgcn_cvt_f32_fp8(w, 2), shift);
    const float f3 = __builtin_ldexpf(__builtin_amdgcn_cvt_f32_fp8(w, 3), shift);
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(f0, f1, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f2, f3, r, true);
  }
}

// ---------------------------------------------------------------------------
// Append
// ---------------------------------------------------------------------------

// Elements 8 c .. 8 c + 7 of R(p) applied to a row, F = float or double. row: the row's
// first element; cs, sn: the position's table rows.
template <class F>
__device__ __forceinline__ void rotated8(const uint16_t* row, int c, int rot, int adjacent, const float* cs,
                                         const float* sn, F (&y)[8]) {
  float x[8];
  unpack8(*reinterpret_cast<const uint4*>(row + 8 * c), x);
  if (8 * c >= rot) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (F)x[i];
  } else if (adjacent) {
    const float4 co = *reinterpret_cast<const float4*>(cs + 4 * c), si = *reinterpret_cast<const float4*>(sn + 4 * c);
    const float cc[4] = {co.x, co.y, co.z, co.w}, ss[4] = {si.x, si.y, si.z, si.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const F a = x[2 * i], b = x[2 * i + 1];
      y[2 * i] = a * (F)cc[i] - b * (F)ss[i];
      y[2 * i + 1] = b * (F)cc[i] + a * (F)ss[i];
    }
  } else {
    const int half = rot / 16;  // chunks per half
    const bool second = c >= half;
    const int j = 8 * (second ? c - half : c);
    float z[8];
    unpack8(*reinterpret_cast<const uint4*>(row + 8 * (second ? c - half : c + half)), z);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const F s = second ? (F)sn[j + i] : -(F)sn[j + i];
      y[i] = (F)x[i] * (F)cs[j + i] + (F)z[i] * s;
    }
  }
}

// One workgroup per (list, page that may get tokens, side): the rows of a page stay in
// registers between the maximum, which needs all of them, and the codes. D / 8 threads
// hold one row, 8 elements each. The workgroups after those turn the queries.
template <int D, int FMT, int ITER>
__global__ __launch_bounds__(512) void cache_append_kernel(AppendLaunch a, int pages, int64_t kv_blocks) {
  constexpr int C = D / 8;
  const int tid = threadIdx.x, c = tid % C, r0 = tid / C, rows = blockDim.x / C;
  if ((int64_t)blockIdx.x >= kv_blocks) {
    const int64_t row = ((int64_t)blockIdx.x - kv_blocks) * rows + r0;  // (b, head, token)
    if (row >= (int64_t)a.c.B * a.Hq * a.N) return;
    const int n = (int)(row % a.N);
    const int64_t bh = row / a.N;
    const int h = (int)(bh % a.Hq), b = (int)(bh / a.Hq);
    const int64_t p = (a.pos0 ? a.pos0[b] : 0) + (int64_t)n;
    float y[8];
    if (a.rot == 0 || (p >= 0 && p < a.n_positions)) {
      const int64_t t = a.rot ? p * (a.rot / 2) : 0;
      rotated8(a.q.ptr + b * a.q.sb + h * a.q.sh + n * a.q.st, c, a.rot, a.adjacent, a.cos + t, a.sin + t, y);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = 0.f;
    }
    f32x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = y[i];
    *reinterpret_cast<bf16x8*>(a.q_out + row * D + 8 * c) = __builtin_convertvector(v, bf16x8);
    return;
  }
  __shared__ int need_sh[8];
  const int P = a.c.P;
  const int side = (int)(blockIdx.x & 1);
  const int list = (int)((blockIdx.x >> 1) / (unsigned)pages), nth = (int)((blockIdx.x >> 1) % (unsigned)pages);
  const int b = list / a.c.H, h = list % a.c.H;
  const int64_t held = a.held[list];
  const int cnt = a.count ? clampi(a.count[list], 0, a.M) : a.M;
  const int64_t start = a.start ? (int64_t)a.start[list] : held - cnt;
  if (start < 0) return;
  const int64_t page0 = start / P + nth;
  if (page0 >= a.c.max_pages) return;
  const int64_t first = page0 * P;
  const int64_t lo = max(start, first), hi = min(start + cnt, first + P);
  if (lo >= hi) return;
  const int page = a.c.table[(int64_t)list * a.c.max_pages + page0];
  if ((unsigned)page >= (unsigned)a.c.n_pages) return;
  uint8_t* codes = (side ? a.c.v : a.c.k) + (int64_t)page * P * D;
  int8_t* exps = side ? a.c.ve : a.c.ke;
  // Rows of the page that other tokens use: below lo and from hi on, of the list's held.
  const int before = (int)(min(lo, held) - first), after = (int)(min(held, first + P) - hi);
  const bool others = before > 0 || after > 0;
  const int was = others ? clampi(exps[page], kExpMin, kExpMax) : kExpMin;

  const Rows x = side ? a.v : a.k;
  const uint16_t* base = x.ptr + b * x.sb + h * x.sh;
  const int rot = side ? 0 : a.rot;
  const int n_rows = (int)(hi - lo);
  double y[ITER][8];
  double big = 0.0;
#pragma unroll
  for (int it = 0; it < ITER; ++it) {
    const int r = it * rows + r0;
    bool ok = r < n_rows;
    int64_t n = 0, t = 0;
    if (ok) {
      const int64_t i = lo - start + r;
      n = a.src ? (int64_t)a.src[(int64_t)list * a.M + i] : i;
      ok = n >= 0 && n < a.N;
      if (rot) {
        const int64_t p = (a.pos0 ? a.pos0[b] : 0) + n;
        ok = ok && p >= 0 && p < a.n_positions;
        t = p * (rot / 2);
      }
    }
    if (ok) {
      rotated8(base + n * x.st, c, rot, a.adjacent, a.cos + t, a.sin + t, y[it]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[it][i] = 0.0;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double v = __builtin_fabs(y[it][i]);
      big = v < __builtin_inf() ? __builtin_fmax(big, v) : big;
    }
  }
  int need = needed_exponent<FMT>(big);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) need = max(need, __shfl_xor(need, o));
  if ((tid & 63) == 0) need_sh[tid >> 6] = need;
  __syncthreads();
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) need = max(need, need_sh[w]);
  const int e = max(need, was);
#pragma unroll
  for (int it = 0; it < ITER; ++it) {
    const int r = it * rows + r0;
    if (r < n_rows) {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[it][i] = __builtin_ldexp(y[it][i], -e);
      uint2 w;
      w.x = codes4<FMT>(y[it]);
      w.y = codes4<FMT>(y[it] + 4);
      *reinterpret_cast<uint2*>(codes + (lo - first + r) * D + 8 * c) = w;
    }
  }
  if (tid == 0) exps[page] = (int8_t)e;
  if (others && e > was) {
    const int n_old = max(before, 0) + max(after, 0);
    for (int i = r0; i < n_old; i += rows) {
      const int64_t r = i < before ? i : hi - first + (i - max(before, 0));
      uint2* at = reinterpret_cast<uint2*>(codes + r * D + 8 * c);
      uint2 w = *at;
      w.x = moved4<FMT>(w.x, was - e);
      w.y = moved4<FMT>(w.y, was - e);
      *at = w;
    }
  }
}

// Pages of a list that M consecutive slots can touch.
int append_pages(const AppendLaunch& L) { return (L.M + L.c.P - 2) / L.c.P + 1; }

// Threads per workgroup: four rows' worth of 8 elements per thread at most (up to 512
// threads for the largest page), or one wave for a few tokens.
struct AppendShape {
  int threads, iter;
};
AppendShape append_shape(const AppendLaunch& L) {
  const int chunks = (L.M < L.c.P ? L.M : L.c.P) * (L.c.D / 8);
  if (chunks <= 64) return {64, 1};
  int threads = 64;
  while (4 * threads < chunks) threads *= 2;
  return {threads, 4};
}

template <int D, int FMT>
int launch_append(const AppendLaunch& L) {
  const AppendShape s = append_shape(L);
  const int pages = append_pages(L);
  const int64_t kv = 2LL * L.c.B * L.c.H * pages;
  const dim3 grid((unsigned)cache_append_blocks(L)), block(s.threads);
  const hipStream_t st = (hipStream_t)L.stream;
  if (s.iter == 1)
    hipLaunchKernelGGL((cache_append_kernel<D, FMT, 1>), grid, block, 0, st, L, pages, kv);
  else
    hipLaunchKernelGGL((cache_append_kernel<D, FMT, 4>), grid, block, 0, st, L, pages, kv);
  return (int)hipGetLastError();
}

// ---------------------------------------------------------------------------
// Retention
// ---------------------------------------------------------------------------

// The order of kvpop_running_topk: larger keys are lower priorities, -0 = +0.
__device__ __forceinline__ uint32_t desc_key(float f) {
  uint32_t u = __float_as_uint(f);
  if (u == 0x80000000u) u = 0u;
  return (u & 0x80000000u) ? u : ~(u | 0x80000000u);
}

// fl(r - fl(t * lg)): two roundings, never fused.
__device__ __forceinline__ float static_priority(float r, float t, float lg) {
#pragma clang fp contract(off)
  const float d = t * lg;
  return r - d;
}

constexpr int kStepThreads = 256;

// One workgroup per list: every slot's position and priority is read once, the token
// that leaves the window gets its priority on the way, and the least eligible one is
// the largest of (key, position) pairs, then the first slot that holds it.
__global__ __launch_bounds__(kStepThreads) void retain_step_kernel(RetainLaunch a) {
  __shared__ unsigned long long best_sh[kStepThreads / 64];
  __shared__ int slot_sh[kStepThreads / 64];
  const int list = blockIdx.x, b = list / a.H, h = list % a.H, tid = threadIdx.x;
  const int q = a.q_pos[b];
  if (q < 0) {
    if (tid == 0) a.slot[list] = -1;
    return;
  }
  const int64_t fresh = (int64_t)q - a.window;  // the token that leaves the window
  const int held = clampi(a.held[list], 0, a.S);
  const bool room = held < a.sinks + a.window + a.topk;
  int32_t* pos = a.pos + (int64_t)list * a.S;
  float* prio = a.prio + (int64_t)list * a.S;
  const float p_new = static_priority(a.scores[list], (float)fresh, a.log_gamma ? a.log_gamma[h] : 0.f);
  unsigned long long best = 0;  // 0: none (a position is at least 0: its pair is stored + 1)
  int slot = a.S;
  for (int i = tid; i < held; i += kStepThreads) {
    const int p = pos[i];
    float v = prio[i];
    if (p == fresh) prio[i] = v = p_new;
    if (p >= a.sinks && p <= fresh) {
      const unsigned long long k = (((unsigned long long)desc_key(v) << 32) | (unsigned)p) + 1;
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
  if (room) {
    slot = held;
    a.held[list] = held + 1;
  } else if (best == 0) {
    slot = -1;
  } else if (a.window == 0 && q >= a.sinks) {
    // The new token takes part, and is the latest of its equals.
    if (desc_key(p_new) >= (uint32_t)((best - 1) >> 32)) slot = -1;
  }
  if (slot >= 0) {
    pos[slot] = q;
    prio[slot] = a.window == 0 ? p_new : 0.f;
  }
  a.slot[list] = slot;
}

constexpr int kPromptThreads = 1024;

// One workgroup per list: a stable compaction in steps of 1024 positions.
__global__ __launch_bounds__(kPromptThreads) void retain_prompt_kernel(RetainLaunch a) {
  constexpr int W = kPromptThreads / 64;
  __shared__ int n_sh[2][W];
  const int list = blockIdx.x, b = list / a.H, h = list % a.H, tid = threadIdx.x;
  const int n = a.lens ? clampi(a.lens[b], 0, a.T) : a.T;
  const int32_t* evict = a.evict + (int64_t)list * a.T;
  const float* r = a.scores + (int64_t)list * a.T;
  int32_t* pos = a.pos + (int64_t)list * a.S;
  float* prio = a.prio + (int64_t)list * a.S;
  const float lg = a.log_gamma ? a.log_gamma[h] : 0.f;
  int held = 0, turn = 0;
  for (int t0 = 0; t0 < n; t0 += kPromptThreads) {
    const int t = t0 + tid;
    const bool keep = t < n && evict[t] >= n;
    const uint64_t m = __builtin_amdgcn_ballot_w64(keep);
    if ((tid & 63) == 0) n_sh[turn][tid >> 6] = __builtin_popcountll(m);
    __syncthreads();
    int at = held + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
    for (int w = 0; w < W; ++w) {
      if (w < (tid >> 6)) at += n_sh[turn][w];
      held += n_sh[turn][w];
    }
    turn ^= 1;
    if (keep && at < a.S) {
      pos[at] = t;
      prio[at] = static_priority(r[t], (float)t, lg);
    }
  }
  held = min(held, a.S);
  for (int i = held + tid; i < a.S; i += kPromptThreads) {
    pos[i] = -1;
    prio[i] = -__builtin_inff();
  }
  if (tid == 0) a.held[list] = held;
}

}  // namespace

int64_t cache_append_blocks(const AppendLaunch& L) {
  const AppendShape s = append_shape(L);
  const int64_t kv = 2LL * L.c.B * L.c.H * append_pages(L);
  const int64_t q_rows = L.q.ptr ? (int64_t)L.c.B * L.Hq * L.N : 0, per = s.threads / (L.c.D / 8);
  return kv + (q_rows + per - 1) / per;
}

int launch_cache_append(const AppendLaunch& L) {
  const bool i8 = L.c.format == KVPOP_CACHE_INT8;
  if (L.c.D == 64)
    return i8 ? launch_append<64, KVPOP_CACHE_INT8>(L) : launch_append<64, KVPOP_CACHE_E4M3>(L);
  return i8 ? launch_append<128, KVPOP_CACHE_INT8>(L) : launch_append<128, KVPOP_CACHE_E4M3>(L);
}

int launch_retain_prompt(const RetainLaunch& L) {
  hipLaunchKernelGGL(retain_prompt_kernel, dim3((unsigned)(L.B * L.H)), dim3(kPromptThreads), 0, (hipStream_t)L.stream,
                     L);
  return (int)hipGetLastError();
}

int launch_retain_step(const RetainLaunch& L) {
  hipLaunchKernelGGL(retain_step_kernel, dim3((unsigned)(L.B * L.H)), dim3(kStepThreads), 0, (hipStream_t)L.stream, L);
  return (int)hipGetLastError();
}

}  // namespace kvpop
