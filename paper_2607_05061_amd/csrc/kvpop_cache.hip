// gfx950 kernels that keep the compact cache of a KVpop model: the append of new keys
// and values to the per-head page lists (rotated, in 8 bits), and the retention that
// says which slot a token takes (include/kvpop_cache.h has the definitions).

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kvpop_cache.h"
#include "kvpop_cache_codes.h"
#include "kvpop_internal.h"

namespace kvpop {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }

// ---------------------------------------------------------------------------
// Codes
// ---------------------------------------------------------------------------

// The least e with a <= qmax 2^e, into [kExpMin, kExpMax]; a >= 0 and finite. With a =
// m 2^x, m in [1/2, 1): 127 2^e = (127/128) 2^(e+7) and 448 2^e = (7/8) 2^(e+9).
template <int FMT, class F>
__device__ __forceinline__ int needed_exponent(F a) {
  if (a == 0) return kExpMin;
  int x;
  bool low;
  if constexpr (sizeof(F) == 8) {
    x = __builtin_amdgcn_frexp_exp(a);
    low = __builtin_amdgcn_frexp_mant(a) <= (FMT == KVPOP_CACHE_INT8 ? 127.0 / 128.0 : 0.875);
  } else {
    x = __builtin_amdgcn_frexp_expf(a);
    low = __builtin_amdgcn_frexp_mantf(a) <= (FMT == KVPOP_CACHE_INT8 ? 127.f / 128.f : 0.875f);
  }
  const int e = FMT == KVPOP_CACHE_INT8 ? x - (low ? 7 : 6) : x - (low ? 9 : 8);
  return clampi(e, kExpMin, kExpMax);
}

__device__ __forceinline__ double larger(double m, double y) { return __builtin_fmax(m, __builtin_fabs(y)); }
__device__ __forceinline__ float larger(float m, float y) { return __builtin_fmaxf(m, __builtin_fabsf(y)); }

// y saturated; NaN gives 0.
__device__ __forceinline__ double saturated(double y, double q) {
  return y == y ? __builtin_fmin(__builtin_fmax(y, -q), q) : 0.0;
}
__device__ __forceinline__ float saturated(float y, float q) {
  return y == y ? __builtin_fminf(__builtin_fmaxf(y, -q), q) : 0.f;
}

// The nearest whole number of y inv (inv a power of two, the product within the codes' range), in
// the low byte: one fma with 1.5 2^52 (2^23) rounds it into the last bits of a number.
__device__ __forceinline__ uint32_t whole(double y, double inv) {
  return (uint32_t)__double_as_longlong(__builtin_fma(y, inv, 0x1.8p52));
}
__device__ __forceinline__ uint32_t whole(float y, float inv) { return __float_as_uint(__builtin_fmaf(y, inv, 0x1.8p23f)); }

// y inv in 32 bits, with every nearer half-way point of the codes on its side: 20 bits of the
// mantissa, the last one set if more follow (rounded to odd), so that a rounding to 4 bits that follows
// is the one rounding of y.
__device__ __forceinline__ float to_odd(double y, double inv) {
  const uint64_t b = (uint64_t)__double_as_longlong(y * inv);
  const uint32_t hi = (uint32_t)(b >> 32) | ((uint32_t)b != 0 ? 1u : 0u);
  return (float)__longlong_as_double((long long)((uint64_t)hi << 32));
}
__device__ __forceinline__ float to_odd(float y, float inv) { return y * inv; }

// Four codes of y[0..3] inv, within the codes' range.
template <int FMT, class F>
__device__ __forceinline__ uint32_t codes4(const F* y, F inv) {
  if constexpr (FMT == KVPOP_CACHE_INT8) {
    const uint32_t lo = __builtin_amdgcn_perm(whole(y[1], inv), whole(y[0], inv), 0x0C0C0400u);
    const uint32_t hi = __builtin_amdgcn_perm(whole(y[3], inv), whole(y[2], inv), 0x04000C0Cu);
    return lo | hi;
  } else {
    const int r = __builtin_amdgcn_cvt_pk_fp8_f32(to_odd(y[0], inv), to_odd(y[1], inv), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(to_odd(y[2], inv), to_odd(y[3], inv), r, true);
  }
}

// Largest magnitudes of 64-bit values by their high words, doubled (the sign falls out): integers
// that order as the values do, up to the low words. frac: the 20 high bits of the mantissa.
__device__ __forceinline__ uint32_t high_key(double y) {
  return (uint32_t)((uint64_t)__double_as_longlong(y) >> 32) << 1;
}
// needed_exponent from the largest key; sure: false where the low words would decide.
template <int FMT>
__device__ __forceinline__ int needed_exponent_of_key(uint32_t key, bool& sure) {
  constexpr uint32_t border = FMT == KVPOP_CACHE_INT8 ? 0xFC000u : 0xC0000u;  // 127/64 - 1, 7/4 - 1
  const int x = (int)(key >> 21) - 1022;
  const uint32_t frac = key >> 1 & 0xFFFFFu;
  sure = frac != border;
  const int e = FMT == KVPOP_CACHE_INT8 ? x - (frac < border ? 7 : 6) : x - (frac < border ? 9 : 8);
  return clampi(e, kExpMin, kExpMax);
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

// A thread holds two pieces of 8 elements of a row. Pieces that turn into each other (halves)
// go together, so that a row and its angles are read once: piece j with j + R / 16 below
// the R / 16 pairs, neighbours (2 j, 2 j + 1) otherwise.
struct Pieces {
  int a, b;     // element offsets of the two pieces
  bool turn;    // by the 8 angles from t on
  int t;
};
__device__ __forceinline__ Pieces pieces(int j, int rot, int adjacent) {
  const bool halves = !adjacent && 16 * j < rot;
  const int half = rot / 2;
  if (halves) return {8 * j, 8 * j + half, true, 8 * j};
  return {16 * j, 16 * j + 8, 16 * j < rot, 8 * j};
}

struct Words8 {
  u32x4 a, b;
};
__device__ __forceinline__ Words8 load_pieces(const uint16_t* row, const Pieces& pc) {
  return {*reinterpret_cast<const u32x4*>(row + pc.a), *reinterpret_cast<const u32x4*>(row + pc.b)};
}

struct Angles {
  f32x4 c[2], s[2];
};
__device__ __forceinline__ Angles load_angles(const float* cs, const float* sn, const Pieces& pc) {
  return {{*reinterpret_cast<const f32x4*>(cs + pc.t), *reinterpret_cast<const f32x4*>(cs + pc.t + 4)},
          {*reinterpret_cast<const f32x4*>(sn + pc.t), *reinterpret_cast<const f32x4*>(sn + pc.t + 4)}};
}

// The first and second elements of the 8 pairs.
__device__ __forceinline__ void paired(const Words8& w, int adjacent, float (&a)[8], float (&b)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t u0 = i < 2 ? w.a[2 * i] : w.b[2 * i - 4], u1 = i < 2 ? w.a[2 * i + 1] : w.b[2 * i - 3];
    const uint32_t p = adjacent ? __builtin_amdgcn_perm(u1, u0, 0x05040100u) : w.a[i];
    const uint32_t q = adjacent ? __builtin_amdgcn_perm(u1, u0, 0x07060302u) : w.b[i];
    a[2 * i] = bf16_lo(p), a[2 * i + 1] = bf16_hi(p);
    b[2 * i] = bf16_lo(q), b[2 * i + 1] = bf16_hi(q);
  }
}

// The pairs turned, F = float or double (where products of bf16 and fp32 are exact).
template <class F>
__device__ __forceinline__ void turned(const float (&a)[8], const float (&b)[8], bool turn, const Angles& g, F (&x)[8],
                                       F (&y)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const F c = g.c[i / 4][i % 4], s = g.s[i / 4][i % 4], p = a[i], q = b[i];
    x[i] = turn ? p * c - q * s : p;
    y[i] = turn ? q * c + p * s : q;
  }
}

// 0, or NaN if a turned value may be NaN or infinite: what goes into it, times 0 (products of
// bf16 and fp32 do not pass the range of 64 bits).
__device__ __forceinline__ float not_finite(const float (&a)[8], const float (&b)[8], const Angles& g) {
  float r = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    r = __builtin_fmaf(a[i], 0.f, r);
    r = __builtin_fmaf(b[i], 0.f, r);
    r = __builtin_fmaf(g.c[i / 4][i % 4], 0.f, r);
    r = __builtin_fmaf(g.s[i / 4][i % 4], 0.f, r);
  }
  return r;
}

constexpr int kQHeads = 4;  // query heads a thread turns by the same angles

// The queries' part: D / 16 threads per token and kQHeads heads.
template <int D>
__device__ __forceinline__ void turn_queries(const AppendLaunch& a, int64_t blk) {
  constexpr int C = D / 16;
  const int groups = (a.Hq + kQHeads - 1) / kQHeads;
  const int64_t item = blk * (blockDim.x / C) + threadIdx.x / C;  // (b, token, heads)
  if (item >= (int64_t)a.c.B * a.N * groups) return;
  const int hg = (int)(item % groups), n = (int)(item / groups % a.N), b = (int)(item / groups / a.N);
  const Pieces pc = pieces(threadIdx.x % C, a.rot, a.adjacent);
  const int64_t p = (a.pos0 ? a.pos0[b] : 0) + (int64_t)n;
  const bool ok = a.rot == 0 || (p >= 0 && p < a.n_positions);
  const uint16_t* x = a.q.ptr + b * a.q.sb + n * a.q.st;
  Words8 w[kQHeads] = {};
  Angles g = {};
  if (ok) {
#pragma unroll
    for (int i = 0; i < kQHeads; ++i)
      w[i] = load_pieces(x + min(hg * kQHeads + i, a.Hq - 1) * a.q.sh, pc);
    if (pc.turn) g = load_angles(a.cos + p * (a.rot / 2), a.sin + p * (a.rot / 2), pc);
  }
#pragma unroll
  for (int i = 0; i < kQHeads; ++i) {
    const int h = hg * kQHeads + i;
    if (h < a.Hq) {
      float p[8], q[8], x[8], y[8];
      paired(w[i], a.adjacent, p, q);
      turned(p, q, pc.turn, g, x, y);
      union {
        bf16x8 h;
        u32x4 u;
      } u, v;
      f32x8 f0, f1;
#pragma unroll
      for (int k = 0; k < 8; ++k) f0[k] = x[k], f1[k] = y[k];
      u.h = __builtin_convertvector(f0, bf16x8);
      v.h = __builtin_convertvector(f1, bf16x8);
      u32x4 lo = u.u, hi = v.u;
      if (a.adjacent) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          lo[2 * k] = __builtin_amdgcn_perm(v.u[k], u.u[k], 0x05040100u);
          lo[2 * k + 1] = __builtin_amdgcn_perm(v.u[k], u.u[k], 0x07060302u);
          hi[2 * k] = __builtin_amdgcn_perm(v.u[k + 2], u.u[k + 2], 0x05040100u);
          hi[2 * k + 1] = __builtin_amdgcn_perm(v.u[k + 2], u.u[k + 2], 0x07060302u);
        }
      }
      uint16_t* out = a.q_out + (((int64_t)b * a.Hq + h) * a.N + n) * D;
      *reinterpret_cast<u32x4*>(out + pc.a) = lo;
      *reinterpret_cast<u32x4*>(out + pc.b) = hi;
    }
  }
}

// What one workgroup writes: rows lo - first .. hi - first - 1 of a page, from the list's
// entries lo - start on.
struct PageJob {
  int list, b, h, nth, n_rows, first_row, entry;  // nth: the page's place in the list
  int before, after;  // rows other tokens use: the first ones, and those behind the written ones
};

template <int D, int FMT, int ITER, class F>
__device__ __forceinline__ void write_page(const AppendLaunch& a, const PageJob& job, const Rows& x, int rot,
                                           uint8_t* pool, int8_t* exps, int* need_sh) {
  constexpr int C = D / 16;
  const int tid = threadIdx.x, r0 = tid / C, rows = blockDim.x / C;
  const Pieces pc = pieces(tid % C, rot, a.adjacent);
  const uint16_t* base = x.ptr + job.b * x.sb + job.h * x.sh;
  const int pos0 = a.pos0 ? a.pos0[job.b] : 0;
  Words8 w[ITER];
  Angles g[ITER];
#pragma unroll
  for (int it = 0; it < ITER; ++it) {
    const int r = it * rows + r0;
    w[it] = Words8{};  // a row that is not there is zeros
    g[it] = Angles{};
    if (r < job.n_rows) {
      const int i = job.entry + r;
      const int64_t n = a.src ? (int64_t)a.src[(int64_t)job.list * a.M + i] : i, p = pos0 + n;
      if (n >= 0 && n < a.N && (rot == 0 || (p >= 0 && p < a.n_positions))) {
        w[it] = load_pieces(base + n * x.st, pc);
        if (pc.turn) g[it] = load_angles(a.cos + p * (rot / 2), a.sin + p * (rot / 2), pc);
      }
    }
  }
  // The page is looked up while the rows are on their way.
  const int page = a.c.table[(int64_t)job.list * a.c.max_pages + job.nth];
  if ((unsigned)page >= (unsigned)a.c.n_pages) return;
  uint8_t* codes = pool + (int64_t)page * a.c.P * D;
  const int was = job.before > 0 || job.after > 0 ? clampi(exps[page], kExpMin, kExpMax) : kExpMin;
  F y[ITER][2][8], big = 0;
  uint32_t key = 0;
  float odd = 0.f;  // NaN if a value may be NaN or infinite
#pragma unroll
  for (int it = 0; it < ITER; ++it) {
    float p[8], q[8];
    paired(w[it], a.adjacent, p, q);
    turned(p, q, pc.turn && rot, g[it], y[it][0], y[it][1]);
    odd += not_finite(p, q, g[it]);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if constexpr (sizeof(F) == 8)
        key = max(key, high_key(y[it][i / 8][i % 8]));
      else
        big = larger(big, y[it][i / 8][i % 8]);  // passes over NaN
    }
  }
  bool sure = sizeof(F) == 4;
  int need = 0;
  if constexpr (sizeof(F) == 8) need = needed_exponent_of_key<FMT>(key, sure);
  if (odd != odd || !sure) {
    big = 0;
#pragma unroll
    for (int it = 0; it < ITER; ++it)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const F v = larger(0, y[it][i / 8][i % 8]);
        big = v < (F)__builtin_inff() ? larger(big, v) : big;
      }
    need = needed_exponent<FMT>(big);
  } else if constexpr (sizeof(F) == 4) {
    need = needed_exponent<FMT>(big);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) need = max(need, __shfl_xor(need, o));
  if ((tid & 63) == 0) need_sh[tid >> 6] = need;
  __syncthreads();
  for (int i = 0; i < (int)(blockDim.x >> 6); ++i) need = max(need, need_sh[i]);
  const int e = max(need, was);
  const F inv = (F)__builtin_ldexpf(1.f, -e);
  // Within the codes' range, unless a value is not finite or the largest scale does not hold it.
  if (odd != odd || e == kExpMax) {
    const F most = (F)(FMT == KVPOP_CACHE_INT8 ? 127 : 448) * (F)__builtin_ldexpf(1.f, e);
#pragma unroll
    for (int it = 0; it < ITER; ++it)
#pragma unroll
      for (int i = 0; i < 16; ++i) y[it][i / 8][i % 8] = saturated(y[it][i / 8][i % 8], most);
  }
#pragma unroll
  for (int it = 0; it < ITER; ++it) {
    const int r = it * rows + r0;
    u32x2 lo = {codes4<FMT>(y[it][0], inv), codes4<FMT>(y[it][0] + 4, inv)};
    u32x2 hi = {codes4<FMT>(y[it][1], inv), codes4<FMT>(y[it][1] + 4, inv)};
    if (a.adjacent) {
      const u32x2 u = lo, v = hi;
      lo = u32x2{__builtin_amdgcn_perm(v.x, u.x, 0x05010400u), __builtin_amdgcn_perm(v.x, u.x, 0x07030602u)};
      hi = u32x2{__builtin_amdgcn_perm(v.y, u.y, 0x05010400u), __builtin_amdgcn_perm(v.y, u.y, 0x07030602u)};
    }
    if (r < job.n_rows) {
      uint8_t* at = codes + (job.first_row + r) * D;
      *reinterpret_cast<u32x2*>(at + pc.a) = lo;
      *reinterpret_cast<u32x2*>(at + pc.b) = hi;
    }
  }
  if (tid == 0) exps[page] = (int8_t)e;
  const int n_before = job.before, n_old = n_before + job.after;
  if (n_old > 0 && e > was) {
    for (int i = r0; i < n_old; i += rows) {
      const int r = i < n_before ? i : job.first_row + job.n_rows + (i - n_before);
      u32x4* at = reinterpret_cast<u32x4*>(codes + r * D + 16 * (tid % C));
      u32x4 v = *at;
      v.x = moved4<FMT>(v.x, was - e);
      v.y = moved4<FMT>(v.y, was - e);
      v.z = moved4<FMT>(v.z, was - e);
      v.w = moved4<FMT>(v.w, was - e);
      *at = v;
    }
  }
}

// One workgroup per (list, page that may get tokens, side): the rows of a page stay in
// registers between the maximum, which needs all of them, and the codes; nothing is shared between
// workgroups, so nothing depends on their order. Keys that turn are held in
// 64 bits, others in 32, where bf16 is exact. The workgroups after those turn the queries.
// HBM bounds large calls: 3 ragged chunks of 20001 tokens (28 query heads, 4 lists each, 1.05 GB)
// 217-221 us, 4.8 TB/s; 4 x 8 lists of 8192 with as many query heads 76-89 us (0.31 GB). Small
// ones are the latency of one page's loads: 5 us for one token of 8 lists, 6 us for one of 1024.
// With the angles read per element and head instead: 455 us for the chunks, 52 instead of 14 us
// for 16 lists that gather 2276 of 32768 tokens.
template <int D, int FMT, int ITER>
__global__ __launch_bounds__(512) void cache_append_kernel(AppendLaunch a, int pages, int64_t kv_blocks) {
  __shared__ int need_sh[8];
  if ((int64_t)blockIdx.x >= kv_blocks) {
    turn_queries<D>(a, (int64_t)blockIdx.x - kv_blocks);
    return;
  }
  const int P = a.c.P;
  const int side = (int)(blockIdx.x & 1);
  PageJob job;
  job.list = (int)((blockIdx.x >> 1) / (unsigned)pages);
  job.b = job.list / a.c.H, job.h = job.list % a.c.H;
  const int64_t held = a.held[job.list];
  const int cnt = a.count ? clampi(a.count[job.list], 0, a.M) : a.M;
  const int64_t start = a.start ? (int64_t)a.start[job.list] : held - cnt;
  if (start < 0) return;
  const int64_t nth = start / P + (blockIdx.x >> 1) % (unsigned)pages;
  if (nth >= a.c.max_pages) return;
  const int64_t first = nth * P, lo = max(start, first), hi = min(start + cnt, first + P);
  if (lo >= hi) return;
  job.n_rows = (int)(hi - lo), job.first_row = (int)(lo - first), job.entry = (int)(lo - start);
  // held is any number: these fit 32 bits only once they are within the page.
  job.before = (int)max(min(lo, held) - first, (int64_t)0);
  job.after = (int)max(min(held, first + P) - hi, (int64_t)0);
  job.nth = (int)nth;
  if (side == 0 && a.rot)
    write_page<D, FMT, ITER, double>(a, job, a.k, a.rot, a.c.k, a.c.ke, need_sh);
  else
    write_page<D, FMT, ITER, float>(a, job, side ? a.v : a.k, 0, side ? a.c.v : a.c.k, side ? a.c.ve : a.c.ke, need_sh);
}

// Pages of a list that M consecutive slots can touch.
int append_pages(const AppendLaunch& L) { return (L.M + L.c.P - 2) / L.c.P + 1; }

// Threads per workgroup: two rows' worth of 16 elements per thread at most (up to 512
// threads for the largest page), or one wave for a few tokens.
struct AppendShape {
  int threads, iter;
};
AppendShape append_shape(const AppendLaunch& L) {
  const int items = (L.M < L.c.P ? L.M : L.c.P) * (L.c.D / 16);
  if (items <= 64) return {64, 1};
  int threads = 64;
  while (2 * threads < items) threads *= 2;
  return {threads, 2};
}

int64_t append_blocks(const AppendLaunch& L) {
  const int64_t kv = 2LL * L.c.B * L.c.H * append_pages(L);
  const int64_t items = L.q.ptr ? (int64_t)L.c.B * L.N * ((L.Hq + kQHeads - 1) / kQHeads) : 0;
  const int64_t per = append_shape(L).threads / (L.c.D / 16);
  return kv + (items + per - 1) / per;
}

template <int D, int FMT>
int launch_append(const AppendLaunch& L) {
  const AppendShape s = append_shape(L);
  const int pages = append_pages(L);
  const int64_t kv = 2LL * L.c.B * L.c.H * pages;
  const dim3 grid((unsigned)append_blocks(L)), block(s.threads);
  const hipStream_t st = (hipStream_t)L.stream;
  if (s.iter == 1)
    hipLaunchKernelGGL((cache_append_kernel<D, FMT, 1>), grid, block, 0, st, L, pages, kv);
  else
    hipLaunchKernelGGL((cache_append_kernel<D, FMT, 2>), grid, block, 0, st, L, pages, kv);
  return (int)hipGetLastError();
}

// ---------------------------------------------------------------------------
// Retention
// ---------------------------------------------------------------------------

// fl(r - fl(t * lg)): two roundings, never fused.
__device__ __forceinline__ float static_priority(float r, float t, float lg) {
#pragma clang fp contract(off)
  const float d = t * lg;
  return r - d;
}

constexpr int kStepThreads = 256;

// One workgroup per list: every slot's position and priority is read once, the token
// that leaves the window gets its priority on the way, and the least eligible one is
// the largest of (key, position) pairs, then the first slot that holds it. The time is that of
// reading 8 bytes a slot: 2048 lists of 2276 slots (37 MB) 10 us, 8 lists 5.5 us (latency).
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

constexpr int kPromptThreads = 1024, kPromptEach = 4, kPromptPart = kPromptThreads * kPromptEach;

// A stable compaction: one workgroup per list and 4096 positions. It counts the kept tokens
// before its part (a list's lifetimes are read from L2 by its later workgroups: at most T / 4096
// times) and writes its own; the last one also clears the slots that are left. 32 lists of 32768
// positions 9 us, 8 of 131072 13 us (one workgroup per list: 23 and 83 us).
__global__ __launch_bounds__(kPromptThreads) void retain_prompt_kernel(RetainLaunch a, int parts) {
  constexpr int W = kPromptThreads / 64;
  __shared__ int n_sh[W], own_sh[W];
  const int list = blockIdx.x / parts, part = blockIdx.x % parts, b = list / a.H, h = list % a.H;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int n = a.lens ? clampi(a.lens[b], 0, a.T) : a.T;
  const int begin = part * kPromptPart;
  if (begin >= n && part > 0) return;
  const bool last = begin + kPromptPart >= n;
  const int32_t* evict = a.evict + (int64_t)list * a.T;
  const float* r = a.scores + (int64_t)list * a.T;
  int32_t* pos = a.pos + (int64_t)list * a.S;
  float* prio = a.prio + (int64_t)list * a.S;
  const float lg = a.log_gamma ? a.log_gamma[h] : 0.f;
  // A wave's own positions are 4 runs of 64 after each other.
  uint64_t m[kPromptEach];
  int own = 0;
#pragma unroll
  for (int i = 0; i < kPromptEach; ++i) {
    const int t = begin + (wave * kPromptEach + i) * 64 + lane;
    m[i] = __builtin_amdgcn_ballot_w64(t < n && evict[min(t, a.T - 1)] >= n);
    own += __builtin_popcountll(m[i]);
  }
  int before = 0;
#pragma unroll 8
  for (int t = tid; t < begin; t += kPromptThreads) before += evict[t] >= n;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) before += __shfl_xor(before, o);
  if (lane == 0) n_sh[wave] = before, own_sh[wave] = own;
  __syncthreads();
  int at = 0, held = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    at += n_sh[w] + (w < wave ? own_sh[w] : 0);
    held += n_sh[w] + own_sh[w];
  }
#pragma unroll
  for (int i = 0; i < kPromptEach; ++i) {
    const int t = begin + (wave * kPromptEach + i) * 64 + lane;
    const int slot = at + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m[i] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m[i], 0u));
    if ((m[i] >> lane & 1) && slot < a.S) {
      pos[slot] = t;
      prio[slot] = static_priority(r[t], (float)t, lg);
    }
    at += __builtin_popcountll(m[i]);
  }
  if (!last) return;
  held = min(held, a.S);
  for (int i = held + tid; i < a.S; i += kPromptThreads) {
    pos[i] = -1;
    prio[i] = -__builtin_inff();
  }
  if (tid == 0) a.held[list] = held;
}

int prompt_parts(const RetainLaunch& L) { return (L.T + kPromptPart - 1) / kPromptPart; }

}  // namespace

int64_t cache_append_threads(const AppendLaunch& L) { return append_blocks(L) * append_shape(L).threads; }

int launch_cache_append(const AppendLaunch& L) {
  const bool i8 = L.c.format == KVPOP_CACHE_INT8;
  if (L.c.D == 64)
    return i8 ? launch_append<64, KVPOP_CACHE_INT8>(L) : launch_append<64, KVPOP_CACHE_E4M3>(L);
  return i8 ? launch_append<128, KVPOP_CACHE_INT8>(L) : launch_append<128, KVPOP_CACHE_E4M3>(L);
}

int64_t retain_prompt_threads(const RetainLaunch& L) { return (int64_t)L.B * L.H * prompt_parts(L) * kPromptThreads; }

int launch_retain_prompt(const RetainLaunch& L) {
  const int parts = prompt_parts(L);
  hipLaunchKernelGGL(retain_prompt_kernel, dim3((unsigned)(L.B * L.H * parts)), dim3(kPromptThreads), 0,
                     (hipStream_t)L.stream, L, parts);
  return (int)hipGetLastError();
}

int64_t retain_step_threads(const RetainLaunch& L) { return (int64_t)L.B * L.H * kStepThreads; }

int launch_retain_step(const RetainLaunch& L) {
  hipLaunchKernelGGL(retain_step_kernel, dim3((unsigned)(L.B * L.H)), dim3(kStepThreads), 0, (hipStream_t)L.stream, L);
  return (int)hipGetLastError();
}

}  // namespace kvpop
