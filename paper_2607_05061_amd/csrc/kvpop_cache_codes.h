// What the kernels of the compact cache and of its lists share (kvpop_cache.hip,
// kvpop_cache_attn.hip, kvpop_mass.hip): codes to 16 bits, products, sums over lane groups, the order of priorities.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kvpop_cache.h"

namespace kvpop {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kExpMin = -32, kExpMax = 32;

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

// The order of kvpop_running_topk: larger keys are lower priorities, -0 = +0.
__device__ __forceinline__ uint32_t desc_key(float f) {
  uint32_t u = __float_as_uint(f);
  if (u == 0x80000000u) u = 0u;
  return (u & 0x80000000u) ? u : ~(u | 0x80000000u);
}

template <int N>
struct alignas(4 * N) Words {
  uint32_t w[N];
};

}  // namespace
}  // namespace kvpop
