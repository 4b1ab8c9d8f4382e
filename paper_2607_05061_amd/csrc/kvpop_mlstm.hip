// gfx950 kernels of the mLSTM scorer's recurrence (include/kvpop_mlstm.h): read-outs of whole
// sequences, their gradients, one token at a time.
//
// Chunks of 64 tokens. With b the running sum of log f since the chunk's start, a token's weight in a
// later read-out of the chunk is exp(b_u - b_t + ig_t): a factor of the row times one of the column.
// So a chunk is
//   out = (far o (A S)) + (W o (A B^T)) C,   S <- keep S + B^T (w o C),
// one product with what is held (S, D x D, in registers), a masked product within the chunk, and the
// update. All four sweeps are this: the read-outs (A, B, C = q, k, v), dq (do, v, k) forwards,
// dv (k, q, do) and dk (v, do, q) backwards in time, where what is held is the gradient of C_t.
// Exponents are sums of 64-bit running sums in units of log2, which no gate makes larger than 2^31 (kForget): no
// weight loses bits to a large |b|.
//
// Sequences are cut into segments for parallelism: a first sweep finds what each segment adds to
// what is held, a scan over the segments what each one starts from, then every segment runs alone.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kvpop_internal.h"

namespace kvpop {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef double f64x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

constexpr double kLog2e = 1.4426950408889634074, kLog2eInv = 0.69314718055994530942;
constexpr int kChunk = 64;       // tokens of a chunk
constexpr int kBlock = 4;        // chunks whose gates are worked out at once, one by each wave
constexpr int kGates = kChunk * kBlock;

enum { kFwd = 0, kDq = 1, kDkv = 2 };

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }
__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }
__device__ __forceinline__ bool gone(double x) { return x == -__builtin_inf(); }
__device__ __forceinline__ float bf16_value(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ uint16_t bf16_bits(float x) {
  union { __bf16 h; uint16_t u; } y;
  y.h = (__bf16)x;
  return y.u;
}
// 2^x of a sum of 64-bit exponents; 0 where one of them is -inf and none NaN.
__device__ __forceinline__ float pow2(double x) { return __builtin_amdgcn_exp2f((float)x); }

__device__ __forceinline__ f32x4 mfma(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// The sum over the lanes l % 16 + 16 k, on all of them.
__device__ __forceinline__ float sum_groups(float x) {
  // Swapped with itself, x becomes its two halves (its even and odd rows of 16) on all lanes.
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// A lane's value from lanes before it, without LDS: row_shr within 16 lanes, then the last lane of the row (of the
// two rows) before. CTRL 0x110 + n: n lanes back; 0x142, 0x143: the broadcasts. Lanes without a source get `none`.
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double x, double none) {
  union { double d; int i[2]; } a, b;
  a.d = x, b.d = none;
  a.i[0] = __builtin_amdgcn_update_dpp(b.i[0], a.i[0], CTRL, ROWS, 0xf, false);
  a.i[1] = __builtin_amdgcn_update_dpp(b.i[1], a.i[1], CTRL, ROWS, 0xf, false);
  return a.d;
}
// Running sum over the wave.
__device__ __forceinline__ double wave_sums(double x) {
  x += moved<0x111, 0xf>(x, 0.0);
  x += moved<0x112, 0xf>(x, 0.0);
  x += moved<0x114, 0xf>(x, 0.0);
  x += moved<0x118, 0xf>(x, 0.0);
  x += moved<0x142, 0xa>(x, 0.0);
  return x + moved<0x143, 0xc>(x, 0.0);
}
// Running maximum over the wave.
__device__ __forceinline__ double wave_maxima(double x) {
  const double none = -__builtin_inf();
  x = fmax(x, moved<0x111, 0xf>(x, none));
  x = fmax(x, moved<0x112, 0xf>(x, none));
  x = fmax(x, moved<0x114, 0xf>(x, none));
  x = fmax(x, moved<0x118, 0xf>(x, none));
  x = fmax(x, moved<0x142, 0xa>(x, none));
  return fmax(x, moved<0x143, 0xc>(x, none));
}
__device__ __forceinline__ double last_lane(double x) {
  union { double d; int i[2]; } a;
  a.d = x;
  a.i[0] = __builtin_amdgcn_readlane(a.i[0], 63);
  a.i[1] = __builtin_amdgcn_readlane(a.i[1], 63);
  return a.d;
}

// A gate below this forgets everything, as -inf does. Its logarithm has no bits of other gates in fp32, in which m and
// lse are held; and a running sum that holds it keeps fewer of them the larger it is (64 bits have none beside 2^53),
// where 64 sums of at most 2^24 keep 22 below the point.
constexpr float kForget = -16777216.f;
__device__ __forceinline__ bool forgets(float fg) { return fg < kForget; }

// log2 sigmoid(x); 0 for +inf.
__device__ __forceinline__ double log2_sigmoid(float x) {
  return -(double)(fmaxf(-x, 0.f) + log1pf(expf(-fabsf(x)))) * kLog2e;
}

union Frag {
  bf16x8 v;
  bf16x4 h[2];
  u32x2 d[2];
  u32x4 u;
};

// 8 elements of a row, 16 bytes.
__device__ __forceinline__ bf16x8 row8(const uint16_t* at) { return *reinterpret_cast<const bf16x8*>(at); }
// Elements at, at + 1 .. + 3 and at + 16 .. + 19: the order of two accumulator tiles' rows.
__device__ __forceinline__ bf16x8 row4x2(const uint16_t* at) {
  Frag f;
  f.d[0] = *reinterpret_cast<const u32x2*>(at);
  f.d[1] = *reinterpret_cast<const u32x2*>(at + 16);
  return f.v;
}
// Column c (of 16) of the 8 rows 8 g .. 8 g + 7 at `at` (a row of `stride` elements), lane = 16 g + c:
// a transposed load gives lane c of a group the elements c of the four rows that its lanes name.
__device__ __forceinline__ bf16x8 column8(const uint16_t* at, int stride, int g, int c) {
  const uint16_t* p = at + (8 * g + (c >> 2)) * stride + 4 * (c & 3);
  Frag f;
  f.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)p);
  f.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(p + 4 * stride));
  return f.v;
}

// ---------------------------------------------------------------------------
// Gates
// ---------------------------------------------------------------------------

// Of kBlock chunks, in units of log2, running sums from each chunk's start.
struct __align__(16) Gates {
  double u[kGates];    // ig - b
  double r[kGates];    // kFwd: the largest u since the last reset; else b - lse (-inf: not read)
  double b[kGates];
  int rid[kGates];     // resets (gates that forget everything) up to here
  float d[kGates];     // backward: d_u, of the query that reads here
  double sum[kBlock];  // b at the chunk's end
  double top[kBlock];  // the largest exponent that the chunk adds to what is held
  int resets[kBlock];
  int odd_k[kBlock], odd_q[kBlock];  // tokens whose k, v (q, do) have no weight
};

// A token's gates on their way (and, backward, what its query's read-out left).
template <int MODE>
struct RawGates {
  uint16_t ig, fg;
  float lse, dot;
  // The wave's chunk; any token that is there stands for those outside [0, n).
  __device__ __forceinline__ void load(const MlstmLaunch& a, int b, int h, int n, int chunk, int lane) {
    const int t = min(chunk * kChunk + lane, n - 1);
    ig = a.ig.ptr[b * a.ig.sb + h * a.ig.sh + t * a.ig.st];
    fg = a.fg.ptr[b * a.fg.sb + h * a.fg.sh + t * a.fg.st];
    if (MODE != kFwd) {
      const int64_t row = ((int64_t)b * a.H + h) * a.T + max(t - a.delay, 0);
      lse = a.lse[row];
      dot = a.dots[row];
    }
  }
};

// The wave's chunk into place `slot`.
template <int MODE>
__device__ __forceinline__ void chunk_gates(const MlstmLaunch& a, Gates& G, const RawGates<MODE>& raw, int n, int chunk,
                                            int slot, int lane) {
  const int t = chunk * kChunk + lane, i = slot * kChunk + lane;
  const bool in = t < n, read = in && t >= a.delay;
  const float ig = in ? bf16_value(raw.ig) : neg_inf(), fg = in ? bf16_value(raw.fg) : -neg_inf();
  const bool reset = forgets(fg);
  const uint64_t resets = __builtin_amdgcn_ballot_w64(reset), mine = resets & ((2ull << lane) - 1);
  const int rid = __builtin_popcountll(mine), all = __builtin_popcountll(resets);
  const double s = wave_sums(reset ? 0.0 : log2_sigmoid(fg));
  const double u = (double)ig * kLog2e - s;
  double r, top;
  if (MODE == kFwd) {
    if (all == 0) {
      r = wave_maxima(u);
    } else {  // since the last reset
      const int first = mine ? 63 - __builtin_clzll(mine) : 0;
      r = u;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double y = __shfl_up(r, o);
        if (lane - o >= first) r = fmax(r, y);
      }
    }
    top = last_lane(r);
  } else {
    const float lse = read ? raw.lse : neg_inf();
    r = lse == neg_inf() ? -__builtin_inf() : s - (double)lse * kLog2e;
    top = MODE == kDq ? (rid == all ? u : -__builtin_inf()) : (rid == 0 ? r : -__builtin_inf());
    top = last_lane(wave_maxima(top));
    G.d[i] = a.normalize && !gone(r) ? -raw.dot : 0.f;
  }
  G.u[i] = u;
  G.r[i] = r;
  G.b[i] = s;
  G.rid[i] = rid;
  const uint64_t odd_k = __builtin_amdgcn_ballot_w64(in && gone(u));
  const uint64_t odd_q = __builtin_amdgcn_ballot_w64(MODE != kFwd && read && gone(r));
  if (lane == 63) {
    G.sum[slot] = s;
    G.top[slot] = top;
    G.resets[slot] = all;
    G.odd_k[slot] = odd_k != 0;
    G.odd_q[slot] = odd_q != 0;
  }
}

// ---------------------------------------------------------------------------
// What is held between chunks
// ---------------------------------------------------------------------------

// A segment's part of the workspace: a matrix [D, D], a vector [D], then these.
struct SegmentScalars {
  double add;   // the exponent of what the segment adds
  double sum;   // log f over the segment, -inf with a reset
  double from;  // the exponent of what it starts from
  double top;   // forwards: what m is after the segment alone
};
__host__ __device__ constexpr int segment_floats(int D) { return D * D + D + 8; }
__device__ __forceinline__ SegmentScalars* scalars(float* part, int D) {
  return reinterpret_cast<SegmentScalars*>(part + D * D + D);
}

// One array's chunks of rows, on their way to LDS. Rows at times outside [shift, n) are zeros; their
// loads go to a row that is there, so that no load waits for a comparison.
template <int D, int THREADS>
struct Tile {
  static constexpr int kPer = kChunk * D / 8 / THREADS;
  static constexpr int kStride = D + 8;  // elements of a row in LDS: 16 rows spread over all banks
  u32x4 x[kPer];
  __device__ __forceinline__ void load(const Rows& a, int b, int h, int t0, int shift, int n, int tid) {
    const uint16_t* p = a.ptr + b * a.sb + h * a.sh + 8 * (tid % (D / 8));
    const int first = t0 - shift + tid / (D / 8);
    if (t0 >= shift && t0 + kChunk <= n) {
      p += first * a.st;
#pragma unroll
      for (int i = 0; i < kPer; ++i) x[i] = *reinterpret_cast<const u32x4*>(p + i * (THREADS * 8 / D) * a.st);
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        x[i] = *reinterpret_cast<const u32x4*>(p + min(max(first + i * (THREADS * 8 / D), 0), n - 1) * a.st);
    }
  }
  __device__ __forceinline__ void store(uint16_t* sh, int t0, int shift, int n, int tid) const {
    const int row = tid / (D / 8);
    uint16_t* to = sh + row * kStride + 8 * (tid % (D / 8));
    if (t0 >= shift && t0 + kChunk <= n) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) *reinterpret_cast<u32x4*>(to + i * (THREADS * 8 / D) * kStride) = x[i];
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int t = t0 + row + i * (THREADS * 8 / D);
        *reinterpret_cast<u32x4*>(to + i * (THREADS * 8 / D) * kStride) = t >= shift && t < n ? x[i] : u32x4{0, 0, 0, 0};
      }
    }
  }
};

// Rows of a chunk that have no weight become zeros, so that nothing in them (NaN) matters.
template <int D>
__device__ __forceinline__ void clear_rows(uint16_t* sh, const double* weight, int tid, int threads) {
  for (int i = tid; i < kChunk * D; i += threads)
    if (gone(weight[i / D])) sh[(i / D) * (D + 8) + i % D] = 0;
}

// What is held carries a power of two, 2^m. It moves with the gates, and beyond that only where a chunk's
// weights would pass 2^kRoom beside it: bf16 and fp32 have the room, and 64 registers are not multiplied
// in every chunk.
constexpr double kRoom = 24.0;

// The exponents of a chunk's update: what is held before (m), after (next), and a token's.
template <bool REV>
struct Update {
  double next, shift;
  float keep;
  int want;
  __device__ __forceinline__ Update(const Gates& G, int slot, double m) {
    const int all = G.resets[slot];
    const double old = all == 0 ? m + G.sum[slot] : -__builtin_inf();
    const double top = added(G, slot);
    next = gone(old) || top > old + kRoom ? top : old;
    keep = gone(old) ? 0.f : next == old ? 1.f : pow2(old - next);
    shift = gone(next) ? 0.0 : (REV ? -next : G.sum[slot] - next);
    want = REV ? 0 : all;
  }
  // The largest exponent that the chunk adds.
  static __device__ __forceinline__ double added(const Gates& G, int slot) {
    return REV ? G.top[slot] : G.top[slot] + G.sum[slot];
  }
  __device__ __forceinline__ float weight(const Gates& G, int i) const {
    return G.rid[i] == want ? pow2((REV ? G.r[i] : G.u[i]) + shift) : 0.f;
  }
};

// m as the header defines it: after a chunk or a segment.
__device__ __forceinline__ double held_m(double m, double sum, double top) { return fmax(m + sum, top); }

// S <- keep S + B^T (w o C) on this wave's NT * 16 columns of C. w o C is taken as the sum of two bf16
// (16 bits), so that what is held is good for more than the read-outs that are made from it; rounded once, it
// would be off by as much as they are.
template <int D, int NT>
__device__ __forceinline__ void update_state(f32x4 (&S)[D / 16][NT], float keep, const uint16_t* b_sh,
                                             const bf16x8 (&cf)[2][NT], const float* w_sh, int g, int c) {
  constexpr int LS = D + 8;
  Frag hi[2][NT], lo[2][NT];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    float w[8];
    *reinterpret_cast<f32x4*>(w) = *reinterpret_cast<const f32x4*>(w_sh + 32 * s + 8 * g);
    *reinterpret_cast<f32x4*>(w + 4) = *reinterpret_cast<const f32x4*>(w_sh + 32 * s + 8 * g + 4);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      Frag v;
      v.v = cf[s][t];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = __uint_as_float(v.u[i] << 16) * w[2 * i], y = __uint_as_float(v.u[i] & 0xFFFF0000u) * w[2 * i + 1];
        const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
        hi[s][t].u[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);  // cut off, not rounded: the rest is the low part
        lo[s][t].v[2 * i] = (__bf16)(x - __uint_as_float(a & 0xFFFF0000u));
        lo[s][t].v[2 * i + 1] = (__bf16)(y - __uint_as_float(b & 0xFFFF0000u));
      }
    }
  }
  if (keep != 1.f) {  // what is forgotten may be anything
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int t = 0; t < NT; ++t) S[i][t] = keep == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : S[i][t] * keep;
  }
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    bf16x8 bf[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) bf[s] = column8(b_sh + 32 * s * LS + 16 * i, LS, g, c);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        S[i][t] = mfma(bf[s], hi[s][t].v, S[i][t]);
        S[i][t] = mfma(bf[s], lo[s][t].v, S[i][t]);
      }
    }
  }
}

// Weights as an operand of two columns: the high and the low bf16 part.
struct Weights {
  static constexpr int kStride = kChunk + 8;
  uint16_t part[2 * kStride];
  __device__ __forceinline__ void set(int i, float w) {
    const float hi = (float)(__bf16)w;
    part[i] = bf16_bits(w);
    part[kStride + i] = bf16_bits(w - hi);
  }
  __device__ __forceinline__ bf16x8 frag(int s, int g, int c) const { return row8(part + (c & 1) * kStride + 32 * s + 8 * g); }
};

// The two columns' sum, in lanes of even c.
__device__ __forceinline__ f32x4 both_columns(f32x4 z) {
#pragma unroll
  for (int r = 0; r < 4; ++r)  // lanes 1, 0, 3, 2 of each four
    z[r] += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(z[r]), 0xB1, 0xf, 0xf, true));
  return z;
}

// sum_t w_t b_t over the 16 columns of B at b_sh: rows 4 g + r of them.
template <int D>
__device__ __forceinline__ f32x4 weighted_rows(const uint16_t* b_sh, const Weights& w, int g, int c) {
  f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < 2; ++s) z = mfma(column8(b_sh + 32 * s * (D + 8), D + 8, g, c), w.frag(s, g, c), z);
  return both_columns(z);
}

__device__ __forceinline__ f32x4 scaled(f32x4 x, float keep) {
  return keep == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : x * keep;
}

// ---------------------------------------------------------------------------
// First sweep: what each segment adds to what is held
// ---------------------------------------------------------------------------

// One workgroup per segment of a head and direction (blockIdx.y, from a.direction on: 0 forwards, k and v; 1
// backwards, q and do). Wave w holds columns [w D / 4, (w + 1) D / 4) of the matrix. Each row is read once and HBM bounds it:
// k and v of 4 x 8 x 32768 tokens of 128 (537 MB) 125 us, 4.3 TB/s. 256 threads, so that two workgroups a CU
// fill each other's waits.
template <int D>
__global__ __launch_bounds__(256, 2) void mlstm_segment_kernel(MlstmLaunch a) {
  constexpr int NT = D / 64, LS = D + 8, NZ = D / 64;
  __shared__ __align__(16) uint16_t b_sh[kChunk * LS], c_sh[kChunk * LS];
  __shared__ Gates G;
  __shared__ __align__(16) float w_sh[kChunk];
  __shared__ __align__(16) Weights wz;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int seg = blockIdx.x % a.segs, list = blockIdx.x / a.segs, b = list / a.H, h = list % a.H;
  const int n = a.lens ? clampi(a.lens[b], 0, a.T) : a.T, chunks = (n + kChunk - 1) / kChunk;
  const bool rev = a.direction + blockIdx.y != 0;
  const int first = min(seg * a.seg_chunks, chunks), count = min((seg + 1) * a.seg_chunks, chunks) - first;
  const Rows& rb = rev ? a.q : a.k;
  const Rows& rc = rev ? a.go : a.v;
  const int shift = rev ? a.delay : 0;

  f32x4 S[D / 16][NT];
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t) S[i][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  f32x4 z[NZ];
#pragma unroll
  for (int j = 0; j < NZ; ++j) z[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  double m = -__builtin_inf(), sum = 0.0, top = -__builtin_inf();
  auto chunk_at = [&](int i) { return rev ? first + count - 1 - i : first + i; };

  RawGates<kDkv> raw;
  RawGates<kFwd> forward;
  auto load_gates = [&](int chunk) __attribute__((always_inline)) {
    if (rev)
      raw.load(a, b, h, n, chunk, lane);
    else
      forward.load(a, b, h, n, chunk, lane);
  };
  if (wave < count) load_gates(chunk_at(wave));
  Tile<D, 256> tb, tc;
  if (count > 0) {
    tb.load(rb, b, h, chunk_at(0) * kChunk, shift, n, tid);
    tc.load(rc, b, h, chunk_at(0) * kChunk, shift, n, tid);
  }
  for (int i = 0; i < count; ++i) {
    const int slot = i % kBlock;
    if (slot == 0) {
      if (i + wave < count) {
        if (rev)
          chunk_gates<kDkv>(a, G, raw, n, chunk_at(i + wave), wave, lane);
        else
          chunk_gates<kFwd>(a, G, forward, n, chunk_at(i + wave), wave, lane);
      }
      if (i + kBlock + wave < count) load_gates(chunk_at(i + kBlock + wave));
    }
    tb.store(b_sh, chunk_at(i) * kChunk, shift, n, tid);
    tc.store(c_sh, chunk_at(i) * kChunk, shift, n, tid);
    __syncthreads();
    if (rev ? G.odd_q[slot] : G.odd_k[slot]) {
      clear_rows<D>(b_sh, (rev ? G.r : G.u) + slot * kChunk, tid, 256);
      clear_rows<D>(c_sh, (rev ? G.r : G.u) + slot * kChunk, tid, 256);
      __syncthreads();
    }
    if (i + 1 < count) {
      tb.load(rb, b, h, chunk_at(i + 1) * kChunk, shift, n, tid);
      tc.load(rc, b, h, chunk_at(i + 1) * kChunk, shift, n, tid);
    }
    double next;
    float keep;
    if (rev) {
      const Update<true> up(G, slot, m);
      next = up.next, keep = up.keep;
      if (tid < kChunk) {
        const float w = up.weight(G, slot * kChunk + tid);
        w_sh[tid] = w;
        wz.set(tid, w * G.d[slot * kChunk + tid]);
      }
    } else {
      const Update<false> up(G, slot, m);
      next = up.next, keep = up.keep;
      if (tid < kChunk) {
        const float w = up.weight(G, slot * kChunk + tid);
        w_sh[tid] = w;
        wz.set(tid, w);
      }
      top = held_m(top, G.resets[slot] ? -__builtin_inf() : G.sum[slot], up.added(G, slot));
    }
    sum = G.resets[slot] ? -__builtin_inf() : sum + G.sum[slot];
    __syncthreads();
    bf16x8 cf[2][NT];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int t = 0; t < NT; ++t) cf[s][t] = column8(c_sh + 32 * s * LS + (wave * NT + t) * 16, LS, g, c);
    update_state<D, NT>(S, keep, b_sh, cf, w_sh, g, c);
#pragma unroll
    for (int j = 0; j < NZ; ++j) {
      const f32x4 add = weighted_rows<D>(b_sh + (wave * NZ + j) * 16, wz, g, c);
      z[j] = scaled(z[j], keep) + add;
    }
    m = next;
    __syncthreads();
  }

  float* part = a.parts + ((int64_t)(rev ? 1 : 0) * a.B * a.H * a.segs + blockIdx.x) * segment_floats(D);
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) part[(16 * i + 4 * g + r) * D + (wave * NT + t) * 16 + c] = S[i][t][r];
#pragma unroll
  for (int j = 0; j < NZ; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (c == 0) part[D * D + (wave * NZ + j) * 16 + 4 * g + r] = z[j][r];
  if (tid == 0) {
    scalars(part, D)->add = m;
    scalars(part, D)->sum = sum;
    scalars(part, D)->top = top;
    if (seg == (rev ? a.segs - 1 : 0)) scalars(part, D)->from = !rev && a.C ? (double)a.m_in[list] * kLog2e : -__builtin_inf();
  }
}

// ---------------------------------------------------------------------------
// What each segment starts from
// ---------------------------------------------------------------------------

// One thread per 4 elements of a head's matrix and vector, which it carries over the segments: a part is
// replaced by what its segment starts from. Forwards, a given state is where it starts and ends. The
// exponents' chain is worked out first, by every workgroup; then kAhead parts are on their way. Memory
// bounds it, with the start of a launch: 32 heads of 16 parts (34 MB, read and written) 12 us.
constexpr int kScanSegments = 512;  // the most that plan() makes
template <int D>
__global__ __launch_bounds__(256) void mlstm_scan_kernel(MlstmLaunch a, int blocks) {
  __shared__ double add_sh[kScanSegments], sum_sh[kScanSegments], top_sh[kScanSegments], from_sh[kScanSegments];
  __shared__ float keep_sh[kScanSegments], put_sh[kScanSegments];
  __shared__ double last_sh[2];
  const int list = blockIdx.x / blocks, e = ((blockIdx.x % blocks) * 256 + threadIdx.x) * 4, tid = threadIdx.x;
  const bool rev = a.direction + blockIdx.y != 0, mine = e < D * D + D;
  float* parts = a.parts + ((int64_t)(rev ? 1 : 0) * a.B * a.H + list) * a.segs * segment_floats(D);
  auto part = [&](int i) { return parts + (int64_t)(rev ? a.segs - 1 - i : i) * segment_floats(D); };
  float* held = nullptr;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  if (!rev && a.C && mine) {
    held = e < D * D ? a.C + (int64_t)list * D * D + e : a.z + (int64_t)list * D + (e - D * D);
    x = *reinterpret_cast<const f32x4*>(held);
  }
  double m = scalars(part(0), D)->from, defined = m;
  constexpr int kAhead = 8;
  f32x4 next[kAhead];
  auto fetch = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) next[j] = *reinterpret_cast<const f32x4*>(part(min(i0 + j, a.segs - 1)) + (mine ? e : 0));
  };
  fetch(0);
  const int count = a.segs;
  for (int i = tid; i < count; i += 256) {
    const SegmentScalars* s = scalars(part(i), D);
    add_sh[i] = s->add, sum_sh[i] = s->sum, top_sh[i] = s->top;
  }
  __syncthreads();
  if (tid < 64)  // m -> max(m + sum, add), a wave's segments at a time: such steps compose to one
    for (int i0 = 0; i0 < count; i0 += 64) {
      const int i = min(i0 + tid, count - 1);
      const double none = -__builtin_inf();
      const bool in = i0 + tid < count;
      double sum = in ? sum_sh[i] : 0.0, add = in ? add_sh[i] : none, top = in ? top_sh[i] : none;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double s = __shfl_up(sum, o), x = __shfl_up(add, o), y = __shfl_up(top, o);
        if (tid >= o) add = fmax(x + sum, add), top = fmax(y + sum, top), sum += s;
      }
      const double after = fmax(m + sum, add), end = fmax(defined + sum, top);
      const double before = __shfl_up(after, 1);
      if (in) from_sh[i] = tid ? before : m;
      m = last_lane(after), defined = last_lane(end);
    }
  if (tid == 0) last_sh[0] = m, last_sh[1] = defined;
  __syncthreads();
  m = last_sh[0], defined = last_sh[1];
  for (int i = tid; i < count; i += 256) {
    const double old = from_sh[i] + sum_sh[i], now = i + 1 < count ? from_sh[i + 1] : m;
    keep_sh[i] = gone(old) ? 0.f : pow2(old - now);
    put_sh[i] = gone(add_sh[i]) ? 0.f : pow2(add_sh[i] - now);
    if (blockIdx.x % blocks == 0 && i > 0) scalars(part(i), D)->from = from_sh[i];
  }
  __syncthreads();
  for (int i0 = 0; i0 < count; i0 += kAhead) {
    f32x4 now[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) now[j] = next[j];
    if (i0 + kAhead < count) fetch(i0 + kAhead);
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (i0 + j < count) {
        if (mine) *reinterpret_cast<f32x4*>(part(i0 + j) + e) = x;
        x = scaled(x, keep_sh[i0 + j]) + now[j] * put_sh[i0 + j];
      }
  }
  if (held) {
    *reinterpret_cast<f32x4*>(held) = gone(m) ? x : x * pow2(m - defined);
    if (e == 0) a.m[list] = (float)(defined * kLog2eInv);
  }
}

// ---------------------------------------------------------------------------
// The sweeps
// ---------------------------------------------------------------------------

template <int D, int MODE>
struct Shared {
  static constexpr int kTiles = MODE == kDkv ? 4 : 3, kRoles = MODE == kDkv ? 2 : 1;
  __align__(16) uint16_t tile[kTiles][kChunk * (D + 8)];
  __align__(16) uint16_t p[kRoles][kChunk * (kChunk + 8)];
  Gates G;
  __align__(16) float w[kChunk];
  __align__(16) Weights wz;
  __align__(16) uint16_t zrow[MODE == kFwd ? 2 * (D + 8) : 8];  // z's high and low bf16 parts
  __align__(16) float far[kRoles][kChunk], far_z[kRoles][kChunk], out[kChunk];
  __align__(16) float z[kRoles][D];
  float dig[4][kChunk];  // backward: the waves' parts of x . dx (of what is held), of k . dk
  float dig_z[MODE == kDq ? 4 : 1][kChunk];  // kDq: of x . z
};

// One workgroup per segment of a head. 4 waves (for dk and dv 4 each, over the same tiles): wave w takes
// rows [16 w, 16 w + 16) of the masked product, which it leaves in LDS, and columns [w D / 4, (w + 1) D / 4) of
// what is held, of the output and of the update. Products are transposed throughout, so that what is held
// serves as an operand from the registers that accumulate it (its rows are the contraction, in the
// order of two accumulator tiles' rows) and a lane's outputs are 4 neighbours of a row.
//
// Chunks follow each other, and the phases of one wait for each other: two waves a SIMD (256 registers a lane; two
// workgroups a CU, of dk and dv one) fill part of the waits, and neither the products nor HBM are busy
// all the time. D = 128: read-outs of 4 x 8 x 32768 tokens 266 us (1.07 GB: 4.0 TB/s), of 2 x 8 x 16384 76 us; dq there
// 118 us, dk and dv 161 us. Twice the waves with 16 columns each needed more registers than they have: read-outs
// 493 us where 4 waves took 277.
template <int D, int MODE>
__global__ __launch_bounds__(MODE == kDkv ? 512 : 256, 2) void mlstm_kernel(MlstmLaunch a) {
  constexpr bool REV = MODE == kDkv;
  constexpr int NT = D / 64, LS = D + 8, PS = kChunk + 8, NZ = D / 64, THREADS = REV ? 512 : 256;
  __shared__ Shared<D, MODE> sh;
  Gates& G = sh.G;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane((tid >> 6) & 3), role = REV ? __builtin_amdgcn_readfirstlane(tid >> 8) : 0;
  // The first sweep went over the heads in order: the read-outs and dq begin with its last ones, whose rows the
  // memory-side cache still has, and dk and dv where dq ended.
  const int block = REV ? blockIdx.x : gridDim.x - 1 - blockIdx.x;
  const int seg = block % a.segs, list = block / a.segs, b = list / a.H, h = list % a.H;
  const int n = a.lens ? clampi(a.lens[b], 0, a.T) : a.T, chunks = (n + kChunk - 1) / kChunk;
  const int first = min(seg * a.seg_chunks, chunks), count = min((seg + 1) * a.seg_chunks, chunks) - first;
  auto chunk_at = [&](int i) { return REV ? first + count - 1 - i : first + i; };
  // kFwd: q, k, v. kDq: do, v, k. kDkv: k, v, q, do.
  const Rows& r0 = MODE == kFwd ? a.q : MODE == kDq ? a.go : a.k;
  const Rows& r1 = MODE == kFwd ? a.k : a.v;
  const Rows& r2 = MODE == kFwd ? a.v : MODE == kDq ? a.k : a.q;
  const int late0 = REV ? 0 : a.delay, late2 = REV ? a.delay : 0;
  const uint16_t* a_sh = sh.tile[REV && role ? 1 : 0];
  const uint16_t* b_sh = sh.tile[!REV ? 1 : role ? 3 : 2];
  const uint16_t* c_sh = sh.tile[!REV ? 2 : role ? 2 : 3];
  // What multiplies with the vector that is held beside the matrix: nothing for dv.
  const bool with_z = MODE != kDkv || role;
  // The state's rows are C's dk and its columns dv, or the other way round.
  const bool turned = MODE == kDq || (REV && role);
  uint16_t* out = MODE == kFwd ? a.o : MODE == kDq ? a.dq : role ? a.dk : a.dv;

  // What the segment starts from.
  f32x4 S[D / 16][NT];
  double m = -__builtin_inf();
  const float* from_S = nullptr;
  const float* from_z = nullptr;
  if (a.segs > 1) {
    float* part = a.parts + (((int64_t)(REV ? a.B * a.H : 0) + list) * a.segs + seg) * segment_floats(D);
    from_S = part, from_z = part + D * D;
    m = scalars(part, D)->from;
  } else if (MODE == kFwd && a.C) {
    from_S = a.C + (int64_t)list * D * D, from_z = a.z + (int64_t)list * D;
    m = (double)a.m_in[list] * kLog2e;
  }
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * i + 4 * g + r, col = (wave * NT + t) * 16 + c;
        S[i][t][r] = from_S ? from_S[turned ? col * D + row : row * D + col] : 0.f;
      }
  auto set_zrow = [&](int i, float z) __attribute__((always_inline)) {
    const float hi = (float)(__bf16)z;
    sh.zrow[i] = bf16_bits(z);
    sh.zrow[LS + i] = bf16_bits(z - hi);
  };
  if ((tid & 255) < D) {
    const float z = from_z ? from_z[tid & 255] : 0.f;
    sh.z[role][tid & 255] = z;
    if (MODE == kFwd) set_zrow(tid, z);
  }
  double defined = m;

  if (REV) {
    // At the end of the segment: what is held there times its gradient.
    float dot = 0.f;
    const bool inner = seg + 1 < a.segs;
    const float* held = a.parts + ((int64_t)list * a.segs + (inner ? seg + 1 : 0)) * segment_floats(D);
    if (inner && !role) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) dot += S[i][t][r] * held[(16 * i + 4 * g + r) * D + (wave * NT + t) * 16 + c];
      if (tid < D) dot += from_z[tid] * held[D * D + tid];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) dot += __shfl_xor(dot, o);
    if (lane == 0 && !role) sh.dig[wave][0] = dot;
    __syncthreads();
    if (tid == 0) {
      const double e = inner ? m + scalars(const_cast<float*>(held), D)->from : -__builtin_inf();
      const double all = ((double)sh.dig[0][0] + sh.dig[1][0] + sh.dig[2][0] + sh.dig[3][0]) * a.scale;
      a.edges[(int64_t)list * a.segs + seg] = gone(e) ? 0.0 : all * (double)pow2(e);
    }
    __syncthreads();
  }
  Tile<D, THREADS> t0, t1, t2, t3;
  auto load = [&](int chunk, int tid) __attribute__((always_inline)) {
    t0.load(r0, b, h, chunk * kChunk, late0, n, tid);
    t1.load(r1, b, h, chunk * kChunk, 0, n, tid);
    t2.load(r2, b, h, chunk * kChunk, late2, n, tid);
    if (REV) t3.load(a.go, b, h, chunk * kChunk, a.delay, n, tid);
  };
  RawGates<MODE> raw;
  if (role == 0 && wave < count) raw.load(a, b, h, n, chunk_at(wave), lane);
  if (count > 0) load(chunk_at(0), tid);

  for (int it = 0; it < count; ++it) {
    // Addresses are made anew in every chunk (kDq, and D = 64): held over them all, they took so many registers that
    // others went to memory, whose waits are those of the tiles on their way (dq of 2 x 8 x 16384 of 128 187 us, 118 so; a training
    // step of 4 x 8 x 4096 of 64 170 us, 155 so).
    int tid_now = tid;
    if (MODE == kDq || D == 64) asm volatile("" : "+v"(tid_now));
    const int tid = tid_now, lane = tid & 63, g = lane >> 4, c = lane & 15;
    const int chunk = chunk_at(it), slot = it % kBlock, at = slot * kChunk;
    if (slot == 0 && role == 0) {
      if (it + wave < count) chunk_gates<MODE>(a, G, raw, n, chunk_at(it + wave), wave, lane);
      if (it + kBlock + wave < count) raw.load(a, b, h, n, chunk_at(it + kBlock + wave), lane);
    }
    t0.store(sh.tile[0], chunk * kChunk, late0, n, tid);
    t1.store(sh.tile[1], chunk * kChunk, 0, n, tid);
    t2.store(sh.tile[2], chunk * kChunk, late2, n, tid);
    if (REV) t3.store(sh.tile[REV ? 3 : 0], chunk * kChunk, a.delay, n, tid);
    __syncthreads();
    if (G.odd_k[slot] | (MODE != kFwd ? G.odd_q[slot] : 0)) {
      if (MODE == kFwd) {
        clear_rows<D>(sh.tile[1], G.u + at, tid, THREADS);
        clear_rows<D>(sh.tile[2], G.u + at, tid, THREADS);
      } else if (MODE == kDq) {
        clear_rows<D>(sh.tile[0], G.r + at, tid, THREADS);
        clear_rows<D>(sh.tile[1], G.u + at, tid, THREADS);
        clear_rows<D>(sh.tile[2], G.u + at, tid, THREADS);
      } else {
        clear_rows<D>(sh.tile[0], G.u + at, tid, THREADS);
        clear_rows<D>(sh.tile[1], G.u + at, tid, THREADS);
        clear_rows<D>(sh.tile[2], G.r + at, tid, THREADS);
        clear_rows<D>(sh.tile[REV ? 3 : 0], G.r + at, tid, THREADS);
      }
      __syncthreads();
    }
    if (it + 1 < count) load(chunk_at(it + 1), tid);

    f32x4 weighted[4];  // kDq: the masked product in 32 bits, and its weights
    bf16x4 weight[4];
    {  // The masked product, transposed: this lane has row j and columns 4 g + r of each 16.
      const int j = 16 * wave + c, rid = G.rid[at + j];
      double rho;   // the row's exponent within the chunk
      float far;    // its factor of what is held
      if (MODE == kFwd) {
        const double M = rid == 0 ? fmax(m, G.r[at + j]) : G.r[at + j];
        rho = gone(M) ? 0.0 : -M;
        far = rid == 0 && !gone(m) ? pow2(m + rho) : 0.f;
      } else if (MODE == kDq) {
        rho = G.r[at + j];
        far = rid == 0 && !gone(m) ? pow2(rho + m) : 0.f;
      } else {
        rho = G.u[at + j];
        far = rid == G.resets[slot] && !gone(m) ? pow2(rho + G.sum[slot] + m) : 0.f;
      }
      const float alpha = MODE == kDq ? G.d[at + j] : 0.f;
      bf16x8 af[D / 32];
#pragma unroll
      for (int s = 0; s < D / 32; ++s) af[s] = row8(a_sh + j * LS + 32 * s + 8 * g);
      float den = 0.f, rounded = 0.f;
      uint32_t bits = 0;
      const bool plain = G.resets[slot] == 0;
      // Two tiles of 16 columns at a time: all that the product with C takes, the further ones as zeros.
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (REV ? half < wave / 2 : half > wave / 2) continue;
        f32x4 acc[2], w[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int kt = 2 * half + x, key = 16 * kt + 4 * g;
          const f64x2* ex = reinterpret_cast<const f64x2*>((REV ? G.r : G.u) + at + key);
          const f64x2 e0 = ex[0], e1 = ex[1];
          acc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < D / 32; ++s) acc[x] = mfma(row8(b_sh + (16 * kt + c) * LS + 32 * s + 8 * g), af[s], acc[x]);
          w[x] = f32x4{pow2(e0.x + rho), pow2(e0.y + rho), pow2(e1.x + rho), pow2(e1.y + rho)};
          if (MODE == kDq) acc[x] += alpha;
          if (REV && role) acc[x] += *reinterpret_cast<const f32x4*>(G.d + at + key);
          acc[x] *= w[x];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const bool in = REV ? key + r >= j : key + r <= j;
            acc[x][r] = in ? acc[x][r] : 0.f;
            if (MODE == kDq) w[x][r] = in ? w[x][r] : 0.f;
          }
        }
        if (!plain)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const i32x4 other = *reinterpret_cast<const i32x4*>(G.rid + at + 32 * half + 16 * x + 4 * g);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              acc[x][r] = other[r] == rid ? acc[x][r] : 0.f;
              if (MODE == kDq) w[x][r] = other[r] == rid ? w[x][r] : 0.f;
            }
          }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          bf16x4 p;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            p[r] = (__bf16)acc[x][r];
            if (MODE == kFwd) den += acc[x][r], rounded += (float)p[r], bits |= __float_as_uint(acc[x][r]);
          }
          if (MODE != kDq) *reinterpret_cast<bf16x4*>(sh.p[role] + j * PS + 32 * half + 16 * x + 4 * g) = p;
          if (MODE == kDq) {
            weighted[2 * half + x] = acc[x];
#pragma unroll
            for (int r = 0; r < 4; ++r) weight[2 * half + x][r] = (__bf16)w[x][r];
          }
        }
      }
      if (MODE == kFwd) {
        f32x4 qz = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < D / 32; ++s) qz = mfma(row8(sh.zrow + (c & 1) * LS + 32 * s + 8 * g), af[s], qz);
        const float held = far == 0.f ? 0.f : far * (qz[0] + qz[1]);
        den = (sum_groups(den) + held) * a.scale;
        // o is divided by the sum of the rounded weights that it is made with: what rounding leaves weighs v - o then, not
        // v, and is nothing where a query sees one token. do . (v - o) of few tokens needs that. Not where a weight or
        // the held part is negative: such sums cancel, and their roundings are no longer small beside them. (NaN then,
        // which is not > 0.) 2-norm error of o of signed features, 64 tokens: 2.1e-1 with the rounded sum, 2.5e-3 so.
        rounded = (int32_t)bits < 0 || held < 0.f ? __builtin_nanf("") : rounded;
        rounded = (sum_groups(rounded) + held) * a.scale;
        const double e = G.b[at + j] - rho;  // that of the row's common factor
        float fac, lse;
        if (a.normalize) {
          const bool some = den > 0.f;
          fac = some ? a.scale / (rounded > 0.f ? rounded : den) : 0.f;
          lse = some ? logf(den) + (float)(e * kLog2eInv) : neg_inf();
          if (den != den) fac = lse = den;
        } else {
          fac = a.scale * pow2(e);
          lse = 0.f;
        }
        const int t = chunk * kChunk + j;
        if (g == 0) {
          sh.out[j] = fac;
          if (a.lse_out && t >= a.delay && t < n) a.lse_out[((int64_t)b * a.H + h) * a.T + t - a.delay] = lse;
        }
      }
      if (g == 0) {
        sh.far[role][j] = far;
        if (REV) sh.far_z[role][j] = far;
      }
    }
    if (role == 0 && wave == (REV ? 3 : 0)) {  // the wave that has the least of it
      const Update<REV> up(G, slot, m);
      const float w = up.weight(G, at + lane);
      sh.w[lane] = w;
      sh.wz.set(lane, REV ? w * G.d[at + lane] : w);
    }
    __syncthreads();
    const Update<REV> up(G, slot, m);
    const double added = up.added(G, slot), gates_sum = G.resets[slot] ? -__builtin_inf() : G.sum[slot];

    const int t_0 = chunk * kChunk;
    // dq's rows of q (dk's rows of k are in LDS): this wave's columns of all of them on their way.
    auto q_row = [&](int j) __attribute__((always_inline)) { return min(max(t_0 + j - a.delay, 0), n - 1); };
    bf16x4 rows_q[MODE == kDq ? 4 : 1][NT];
    if (MODE == kDq) {
      const uint16_t* from = a.q.ptr + b * a.q.sb + h * a.q.sh;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint16_t* p = from + q_row(16 * q + c) * a.q.st + wave * NT * 16 + 4 * g;
#pragma unroll
        for (int t = 0; t < NT; ++t) rows_q[MODE == kDq ? q : 0][t] = *reinterpret_cast<const bf16x4*>(p + 16 * t);
      }
    }
    f32x4 acc[4][NT];
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[q][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    // What is held, rounded to bf16 for the product (its terms' errors are independent; out is rounded too). For dq it
    // is two bf16: x . dx, which corrects do . o and makes dfg, is taken from its products.
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      bf16x8 sf[NT], low[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = S[2 * s + i / 4][t][i % 4];
          sf[t][i] = (__bf16)x;
          if (MODE == kDq) low[t][i] = (__bf16)(x - (float)sf[t][i]);
        }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const bf16x8 af = row4x2(a_sh + (16 * q + c) * LS + 32 * s + 4 * g);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          acc[q][t] = mfma(sf[t], af, acc[q][t]);
          if (MODE == kDq) acc[q][t] = mfma(low[t], af, acc[q][t]);
        }
      }
    }
    bf16x8 cf[2][NT];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int t = 0; t < NT; ++t) cf[s][t] = column8(c_sh + 32 * s * LS + (wave * NT + t) * 16, LS, g, c);
    // Columns 16 t + 4 g + 0 .. 3 of the wave's of row 16 q + c.
    auto result = [&](int q, int t, float far, float far_z, float fac) __attribute__((always_inline)) {
      f32x4 y = MODE == kDq ? acc[q][t] : scaled(acc[q][t], far);
      if (MODE != kFwd && with_z) y += scaled(*reinterpret_cast<const f32x4*>(sh.z[role] + (wave * NT + t) * 16 + 4 * g), far_z);
#pragma unroll
      for (int s = 0; s < 2; ++s)
        if (REV ? 32 * s + 31 >= 16 * q : 32 * s <= 16 * q)
          y = mfma(cf[s][t], row8(sh.p[role] + (16 * q + c) * PS + 32 * s + 8 * g), y);
      return y * fac;
    };
    // A normalised read-out does not change with the size of x, so x . dx = 0, and what comes out for it is the error of
    // do . o: of the rounding of o, which is not small beside do . (v - o) where a query sees few tokens, by whatever gates and
    // features. So x . dx is taken first, from the masked product in 32 bits and <x, k> (its rounded elements would leave more than
    // the error where features of either sign cancel), and do . v - do . o corrected with it. What is rounded then gives
    // the x . dx that the forget gates' gradients are made of.
    if (MODE == kDq) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int j = 16 * q + c;
        const float far = sh.far[role][j];
        float dot = 0.f, dot_z = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          acc[q][t] = scaled(acc[q][t], far);
          const f32x4 z = *reinterpret_cast<const f32x4*>(sh.z[role] + (wave * NT + t) * 16 + 4 * g);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float x = (float)rows_q[MODE == kDq ? q : 0][t][r];
            dot += acc[q][t][r] * x, dot_z += z[r] * x;
          }
        }
        dot = sum_groups(dot), dot_z = sum_groups(dot_z);
        asm volatile("" : "+v"(dot), "+v"(dot_z));
        if (g == 0) sh.dig[wave][j] = dot, sh.dig_z[MODE == kDq ? wave : 0][j] = far == 0.f ? 0.f : far * dot_z;
      }
      bf16x8 row_q[D / 32];  // all of the wave's own rows, which the caches have by now
      const uint16_t* p = a.q.ptr + b * a.q.sb + h * a.q.sh + q_row(16 * wave + c) * a.q.st + 8 * g;
#pragma unroll
      for (int s = 0; s < D / 32; ++s) row_q[s] = row8(p + 32 * s);
      f32x4 score[4];
      float in = 0.f;
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) {
        if (kt / 2 > wave / 2) continue;
        score[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < D / 32; ++s) score[kt] = mfma(row8(c_sh + (16 * kt + c) * LS + 32 * s + 8 * g), row_q[s], score[kt]);
#pragma unroll
        for (int r = 0; r < 4; ++r) in += weighted[kt][r] * score[kt][r];
      }
      in = sum_groups(in);
      __syncthreads();
      const int j = 16 * wave + c, t = t_0 + j;
      const bool read = !gone(G.r[at + j]);
      float held = 0.f, held_z = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) held += sh.dig[w][j], held_z += sh.dig_z[MODE == kDq ? w : 0][j];
      float d = G.d[at + j], x = 0.f;
      if (a.normalize && read) x = a.scale * (held + d * held_z + in);
      if (x != x) x = 0.f;
      d -= x;
      in = 0.f;
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) {
        if (kt / 2 > wave / 2) continue;
        bf16x4 p;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          p[r] = (__bf16)(weighted[kt][r] - x * (float)weight[kt][r]);
          in += (float)p[r] * score[kt][r];
        }
        *reinterpret_cast<bf16x4*>(sh.p[role] + j * PS + 16 * kt + 4 * g) = p;
      }
      in = sum_groups(in);
      if (g == 0) {
        sh.far_z[role][j] = sh.far[role][j] * d;
        if (t < n) {
          const bool mine = t >= a.delay;
          // A row that is not read has dx = 0, whatever q holds.
          a.xdx[(int64_t)list * a.T + t] = mine && read ? a.scale * (held + d * held_z + in) : 0.f;
          if (a.normalize && mine) a.dots[(int64_t)list * a.T + t - a.delay] = -d;
        }
      }
      __syncthreads();
    }
    {
      const int late = REV ? 0 : a.delay;
      uint16_t* to = out + ((int64_t)list * a.T + c - late + t_0) * D + wave * NT * 16 + 4 * g;
#pragma unroll
      for (int q0 = 0; q0 < 4; q0 += 2) {
        bf16x4 y[2][NT];
        float dot[2] = {0.f, 0.f};
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int q = q0 + x, j = 16 * q + c;
          const float far = sh.far[role][j], fac = MODE == kFwd ? sh.out[j] : a.scale;
          const float far_z = MODE != kFwd && with_z ? sh.far_z[role][j] : 0.f;
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            acc[q][t] = result(q, t, far, far_z, fac);
            bf16x4 with;
            if (REV) with = *reinterpret_cast<const bf16x4*>(sh.tile[0] + j * LS + (wave * NT + t) * 16 + 4 * g);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              y[x][t][r] = (__bf16)acc[q][t][r];
              if (REV) dot[x] += acc[q][t][r] * (float)with[r];
            }
          }
          if (REV) dot[x] = sum_groups(dot[x]);
        }
        // The values are made before the branch: where the products' results were first read behind one, the
        // compiler had left out the wait that they need.
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int t = 0; t < NT; ++t) asm volatile("" : "+v"(y[x][t]), "+v"(dot[x]));
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int j = 16 * (q0 + x) + c;
          if (t_0 + j >= late && t_0 + j < n)
#pragma unroll
            for (int t = 0; t < NT; ++t) *reinterpret_cast<bf16x4*>(to + 16 * (q0 + x) * D + 16 * t) = y[x][t];
          if (REV && g == 0 && role) sh.dig[wave][j] = dot[x];
        }
      }
    }

    f32x4 add[NT];
    if (MODE == kFwd) {
#pragma unroll
      for (int i = 0; i < NZ; ++i) add[i] = weighted_rows<D>(b_sh + (wave * NZ + i) * 16, sh.wz, g, c);
    } else if (with_z) {  // a vector over this wave's own columns: sum w_t c_t
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        add[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < 2; ++s) add[t] = mfma(cf[s][t], sh.wz.frag(s, g, c), add[t]);
        add[t] = both_columns(add[t]);
      }
    }
    update_state<D, NT>(S, up.keep, b_sh, cf, sh.w, g, c);
    if (MODE == kFwd) {
#pragma unroll
      for (int i = 0; i < NZ; ++i) {
        const int at_z = (wave * NZ + i) * 16 + 4 * g;
        f32x4* z = reinterpret_cast<f32x4*>(sh.z[0] + at_z);
        if (c == 0) {
          const f32x4 y = scaled(*z, up.keep) + add[i];
          *z = y;
#pragma unroll
          for (int r = 0; r < 4; ++r) set_zrow(at_z + r, y[r]);
        }
      }
      defined = held_m(defined, gates_sum, added);
    } else if (with_z) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        f32x4* z = reinterpret_cast<f32x4*>(sh.z[role] + (wave * NT + t) * 16 + 4 * g);
        if (c == 0) *z = scaled(*z, up.keep) + add[t];
      }
    }
    m = up.next;
    __syncthreads();
    if (REV && tid < kChunk) {
      const int t = chunk * kChunk + tid;
      if (t < n) {
        const float x = sh.dig[0][tid] + sh.dig[1][tid] + sh.dig[2][tid] + sh.dig[3][tid];
        a.dig32[(int64_t)list * a.T + t] = x;
        a.dig[(int64_t)list * a.T + t] = bf16_bits(x);
      }
    }
  }

  // Rows that nothing reads, and tokens past the sequence's end.
  const int c0 = seg * a.seg_chunks, c1 = min((seg + 1) * a.seg_chunks, (a.T + kChunk - 1) / kChunk);
  const int z0 = max(c0 * kChunk, max(0, REV ? n : n - a.delay)), z1 = min(c1 * kChunk, a.T);
  for (int64_t i = (int64_t)z0 * (D / 8) + (tid & 255); i < (int64_t)z1 * (D / 8); i += 256)
    *reinterpret_cast<u32x4*>(out + (int64_t)list * a.T * D + i * 8) = u32x4{0, 0, 0, 0};
  for (int i = z0 + tid; i < z1; i += THREADS) {
    if (MODE == kFwd && a.lse_out) a.lse_out[(int64_t)list * a.T + i] = neg_inf();
    if (REV) a.dig[(int64_t)list * a.T + i] = 0;
  }

  if (MODE == kFwd && a.segs == 1 && a.C) {
    const float out_scale = gone(m) ? 1.f : pow2(m - defined);
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          a.C[(int64_t)list * D * D + (16 * i + 4 * g + r) * D + (wave * NT + t) * 16 + c] = S[i][t][r] * out_scale;
    if (tid < D) a.z[(int64_t)list * D + tid] = sh.z[0][tid] * out_scale;
    if (tid == 0) a.m[list] = (float)(defined * kLog2eInv);
  }
}

// ---------------------------------------------------------------------------
// The rest of the backward pass
// ---------------------------------------------------------------------------

// do . o of each row: D / 8 threads a row. 2 x 8 x 16384 rows of 128 (134 MB) 25 us, 5.4 TB/s: HBM.
template <int D>
__global__ __launch_bounds__(256) void mlstm_dots_kernel(MlstmLaunch a, int64_t rows) {
  constexpr int W = D / 8;
  const int64_t row = (int64_t)blockIdx.x * (256 / W) + threadIdx.x / W;
  if (row >= rows) return;
  const int list = (int)(row / a.T), t = (int)(row % a.T), b = list / a.H, h = list % a.H, i = threadIdx.x % W;
  const int n = a.lens ? clampi(a.lens[b], 0, a.T) : a.T;
  float s = 0.f;
  if (t < n - a.delay) {
    Frag x, y;
    x.u = *reinterpret_cast<const u32x4*>(a.go.ptr + b * a.go.sb + h * a.go.sh + t * a.go.st + 8 * i);
    y.u = *reinterpret_cast<const u32x4*>(a.o_in + row * D + 8 * i);
#pragma unroll
    for (int j = 0; j < 8; ++j) s += (float)x.v[j] * (float)y.v[j];
  }
#pragma unroll
  for (int o = 1; o < W; o <<= 1) s += __shfl_xor(s, o);
  if (i == 0) a.dots[row] = s;
}

__device__ __forceinline__ double block_sum(double x, double* sh) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  return sh[0] + sh[1] + sh[2] + sh[3];
}

// The forget gates' gradients, one workgroup per segment. d log f_t is the sum over the pairs s < t <= u
// that t lies between. At a segment's start that is the product of what is held there and its gradient,
// and from token to token it changes by x . dx - k . dk of the token. Both of these hold the pairs of their chunk
// with the same rounded weights, which cancel in the running sum; it is made to end in the next
// product, in proportion, so that what rounding is left does not pile up along the sequence.
// 2 x 8 x 16384 tokens 7 us: the latency of two passes over a segment's few KB.
__global__ __launch_bounds__(256) void mlstm_forget_kernel(MlstmLaunch a) {
  __shared__ double sum_sh[4], edge_sh[4];
  __shared__ int reset_sh[4];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int seg = blockIdx.x % a.segs, list = blockIdx.x / a.segs, b = list / a.H, h = list % a.H;
  const int n = a.lens ? clampi(a.lens[b], 0, a.T) : a.T;
  const int t0 = min(seg * a.seg_chunks * kChunk, a.T), t1 = min((seg + 1) * a.seg_chunks * kChunk, a.T), end = min(t1, n);
  const double* edges = a.edges + (int64_t)list * a.segs;
  const double start = seg > 0 ? edges[seg - 1] : 0.0, stop = edges[seg];
  // a token's step: x . dx - k . dk
  auto step = [&](int t) -> double {
    if (t >= end) return 0.0;
    return (double)a.xdx[(int64_t)list * a.T + t] - a.dig32[(int64_t)list * a.T + t];
  };
  auto fg = [&](int t) { return bf16_value(a.fg.ptr[b * a.fg.sb + h * a.fg.sh + t * a.fg.st]); };
  double total = 0.0, resets = 0.0;
  for (int t = t0 + tid; t < end; t += 256) {
    total += step(t);
    resets += forgets(fg(t));
  }
  total = block_sum(total, sum_sh);
  resets = block_sum(resets, sum_sh);
  const double drift = resets > 0.0 || end <= t0 ? 0.0 : (start - total - stop) / (end - t0);
  double carry = start;  // before this block's tokens
  for (int base = t0; base < end; base += 256) {
    const int t = base + tid;
    const bool in = t < end;
    const float f = in ? fg(t) : 0.f;
    const bool reset = in && forgets(f);
    const double mine = step(t);
    // the running sum of steps before t, since the last reset at or before t
    double s = mine;
    const uint64_t r = __builtin_amdgcn_ballot_w64(reset), upto = r & ((2ull << lane) - 1);
    const int first = upto ? 63 - __builtin_clzll(upto) : -1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double y = __shfl_up(s, o);
      if (lane - o >= max(first, 0)) s += y;
    }
    __syncthreads();
    if (lane == 63) edge_sh[wave] = s, reset_sh[wave] = r != 0;
    __syncthreads();
    double before = carry;  // at this wave's start
    for (int w = 0; w < wave; ++w) before = (reset_sh[w] ? 0.0 : before) - edge_sh[w];
    const double d = (first >= 0 ? 0.0 : before) - (s - mine) - drift * (t - t0);
    if (in) a.dfg[(int64_t)list * a.T + t] = bf16_bits(reset ? 0.f : (float)d / (1.f + expf(f)));
    for (int w = wave; w < 4; ++w) before = (reset_sh[w] ? 0.0 : before) - edge_sh[w];
    carry = before;
  }
  for (int t = max(t0, n) + tid; t < t1; t += 256) a.dfg[(int64_t)list * a.T + t] = 0;
}

// ---------------------------------------------------------------------------
// One token
// ---------------------------------------------------------------------------

constexpr int kStepThreads = 512;

// One workgroup per head: the matrix is read, updated, written and multiplied with q in one pass. D = 128:
// 8 heads 6 us (the latency of one read and write), 1024 heads 19-20 us (134 MB: what HBM and the memory-side cache give).
template <int D>
__global__ __launch_bounds__(kStepThreads) void mlstm_step_kernel(MlstmLaunch a) {
  constexpr int COLS = D / 4, ROWS = kStepThreads / COLS, PER = D / ROWS, W = kStepThreads / 64;
  __shared__ __align__(16) float num_sh[W][D];
  __shared__ float den_sh[W];
  const int list = blockIdx.x, b = list / a.H, h = list % a.H, tid = threadIdx.x, wave = tid >> 6;
  uint16_t* o = a.o + (int64_t)list * D;
  if (a.lens && a.lens[b] <= 0) {
    if (tid < D) o[tid] = 0;
    return;
  }
  const int col = 4 * (tid % COLS), row0 = tid / COLS;
  float* C = a.C + (int64_t)list * D * D + col;
  f32x4 x[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) x[i] = *reinterpret_cast<const f32x4*>(C + (row0 + i * ROWS) * D);
  const float ig = bf16_value(a.ig.ptr[b * a.ig.sb + h * a.ig.sh]), fg = bf16_value(a.fg.ptr[b * a.fg.sb + h * a.fg.sh]);
  const uint16_t* q = a.q.ptr + b * a.q.sb + h * a.q.sh;
  const uint16_t* k = a.k.ptr + b * a.k.sb + h * a.k.sh;
  const uint16_t* v = a.v.ptr + b * a.v.sb + h * a.v.sh;
  const float m = a.m_in[list];
  const double old = forgets(fg) ? -__builtin_inf() : (double)m * kLog2e + log2_sigmoid(fg), put = (double)ig * kLog2e;
  // C and z go with m as it is stored, so that what its rounding loses (up to 2^-25 |m| a token, all of a slow decay beside a
  // large m) is theirs. Below fp32's range nothing is held.
  const float m_out = (float)(fmax(old, put) * kLog2eInv);
  const double now = (double)m_out * kLog2e;
  const bool masked = ig == neg_inf();
  const float keep = gone(old) || gone(now) ? 0.f : pow2(old - now), in = masked || gone(now) ? 0.f : pow2(put - now);
  float vi[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) vi[j] = masked ? 0.f : in * bf16_value(v[col + j]);
  f32x4 num = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int row = row0 + i * ROWS;
    const float kr = masked ? 0.f : bf16_value(k[row]), qr = bf16_value(q[row]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[i][j] = (keep == 0.f ? 0.f : keep * x[i][j]) + kr * vi[j];
      num[j] += qr * x[i][j];
    }
    *reinterpret_cast<f32x4*>(C + row * D) = x[i];
  }
  float den = 0.f;
  if (tid < D) {
    float* z = a.z + (int64_t)list * D + tid;
    const float zr = (keep == 0.f ? 0.f : keep * *z) + (masked ? 0.f : in * bf16_value(k[tid]));
    *z = zr;
    den = bf16_value(q[tid]) * zr;
  }
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) den += __shfl_xor(den, s);
#pragma unroll
  for (int s = COLS; s < 64; s <<= 1)
#pragma unroll
    for (int j = 0; j < 4; ++j) num[j] += __shfl_xor(num[j], s);
  if ((tid & 63) < COLS) *reinterpret_cast<f32x4*>(&num_sh[wave][col]) = num;
  if ((tid & 63) == 0) den_sh[wave] = den;
  __syncthreads();
  if (tid == 0) a.m[list] = m_out;
  if (tid >= D) return;
  float y = 0.f;
#pragma unroll
  for (int w = 0; w < W; ++w) y += num_sh[w][tid];
  if (a.normalize) {
    den = den_sh[0] + (D > 64 ? den_sh[1] : 0.f);
    y = den > 0.f ? y / den : den != den ? den : 0.f;
  } else {
    y *= a.scale * pow2(now);
  }
  o[tid] = bf16_bits(y);
}

// ---------------------------------------------------------------------------
// Plans
// ---------------------------------------------------------------------------

int chunk_count(const MlstmLaunch& L) { return (L.T + kChunk - 1) / kChunk; }

// Segments: enough for two workgroups a CU: each adds a matrix that is written and read twice, and not all of more run
// at once. Few chunks are one segment, since two launches more cost as much as they do. Read-outs + gradients, us, D = 128, wanting 256, 512,
// 1024 workgroups: 8 heads of 16384 tokens 83 + 245, 76 + 241, 103 + 329; 32 of them 264 + 779, 220 + 692, 232 + 771; 64 heads of 1024
// 52 + 150, 53 + 164, 78 + 238. One segment up to 2, 4, 8 chunks: 8 heads of 3 chunks 22 + 68, 20 + 60, 20 + 60, of 4 23 + 69, 25 + 75,
// 25 + 75, of 5 23 + 71, 23 + 71, 30 + 91; 64 heads of 4 32 + 86, 25 + 78, 25 + 78. Off the line: one head of 32768 would take 74 + 181
// with 256 (117 + 281 so), 304 heads of 8 chunks 61 + 232 as one segment (101 + 333 so).
constexpr int kWantGroups = 512, kFewChunks = 4;
static_assert(kWantGroups <= kScanSegments, "a head's segments");
void plan(MlstmLaunch& L) {
  const int chunks = chunk_count(L);
  const int64_t lists = (int64_t)L.B * L.H;
  int64_t segs = lists >= kWantGroups || chunks <= kFewChunks ? 1 : (kWantGroups + lists - 1) / lists;
  if (segs > chunks) segs = chunks;
  L.seg_chunks = (int)((chunks + segs - 1) / segs);
  L.segs = (chunks + L.seg_chunks - 1) / L.seg_chunks;
}

template <int D>
int launch_states(MlstmLaunch L, int first, int directions) {
  L.direction = first;
  const hipStream_t st = (hipStream_t)L.stream;
  const unsigned lists = (unsigned)L.B * L.H;
  hipLaunchKernelGGL((mlstm_segment_kernel<D>), dim3(lists * L.segs, directions), dim3(256), 0, st, L);
  int e = (int)hipGetLastError();
  if (e != 0) return e;
  const int blocks = (D * D + D + 1023) / 1024;
  hipLaunchKernelGGL((mlstm_scan_kernel<D>), dim3(lists * blocks, directions), dim3(256), 0, st, L, blocks);
  return (int)hipGetLastError();
}

template <int D>
int launch_fwd(const MlstmLaunch& L) {
  if (L.segs > 1) {
    const int e = launch_states<D>(L, 0, 1);
    if (e != 0) return e;
  }
  hipLaunchKernelGGL((mlstm_kernel<D, kFwd>), dim3((unsigned)(L.B * L.H * L.segs)), dim3(256), 0, (hipStream_t)L.stream, L);
  return (int)hipGetLastError();
}

template <int D>
int launch_bwd(const MlstmLaunch& L) {
  const hipStream_t st = (hipStream_t)L.stream;
  const unsigned groups = (unsigned)(L.B * L.H * L.segs);
  const int64_t rows = (int64_t)L.B * L.H * L.T, per = 256 / (D / 8);
  int e;
  hipLaunchKernelGGL((mlstm_dots_kernel<D>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, st, L, rows);
  if ((e = (int)hipGetLastError()) != 0) return e;
  // The backward direction sums do . o, which dq's sweep corrects where it is normalised.
  if (L.segs > 1 && (e = launch_states<D>(L, 0, L.normalize ? 1 : 2)) != 0) return e;
  hipLaunchKernelGGL((mlstm_kernel<D, kDq>), dim3(groups), dim3(256), 0, st, L);
  if ((e = (int)hipGetLastError()) != 0) return e;
  if (L.segs > 1 && L.normalize && (e = launch_states<D>(L, 1, 1)) != 0) return e;
  hipLaunchKernelGGL((mlstm_kernel<D, kDkv>), dim3(groups), dim3(512), 0, st, L);
  if ((e = (int)hipGetLastError()) != 0) return e;
  hipLaunchKernelGGL(mlstm_forget_kernel, dim3(groups), dim3(256), 0, st, L);
  return (int)hipGetLastError();
}

// Floats of a direction's parts, rounded up to 16 bytes by segment_floats' own size.
int64_t part_floats(const MlstmLaunch& L) {
  return L.segs > 1 ? (int64_t)L.B * L.H * L.segs * segment_floats(L.D) : 0;
}
int64_t edge_floats(const MlstmLaunch& L) { return ((int64_t)L.B * L.H * L.segs * 2 + 3) / 4 * 4; }
int64_t row_floats(const MlstmLaunch& L) { return ((int64_t)L.B * L.H * L.T + 3) / 4 * 4; }

}  // namespace

int64_t mlstm_threads(const MlstmLaunch& L) { return (int64_t)L.B * L.H * chunk_count(L) * 1024; }

int64_t mlstm_fwd_workspace_floats(MlstmLaunch L) {
  plan(L);
  return part_floats(L);
}
int64_t mlstm_bwd_workspace_floats(MlstmLaunch L) {
  plan(L);
  return 2 * part_floats(L) + 3 * row_floats(L) + edge_floats(L);
}

int launch_mlstm_fwd(MlstmLaunch L) {
  plan(L);
  L.parts = L.workspace;
  return L.D == 64 ? launch_fwd<64>(L) : launch_fwd<128>(L);
}

int launch_mlstm_bwd(MlstmLaunch L) {
  plan(L);
  L.dots = L.workspace;
  L.dig32 = L.dots + row_floats(L);
  L.xdx = L.dig32 + row_floats(L);
  L.edges = reinterpret_cast<double*>(L.xdx + row_floats(L));
  L.parts = L.xdx + row_floats(L) + edge_floats(L);
  return L.D == 64 ? launch_bwd<64>(L) : launch_bwd<128>(L);
}

int launch_mlstm_step(const MlstmLaunch& L) {
  const dim3 grid((unsigned)(L.B * L.H)), block(kStepThreads);
  if (L.D == 64)
    hipLaunchKernelGGL((mlstm_step_kernel<64>), grid, block, 0, (hipStream_t)L.stream, L);
  else
    hipLaunchKernelGGL((mlstm_step_kernel<128>), grid, block, 0, (hipStream_t)L.stream, L);
  return (int)hipGetLastError();
}

}  // namespace kvpop
