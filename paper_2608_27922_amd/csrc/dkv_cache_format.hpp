// Row formats of the paged window cache on gfx950: quantising and reading 8-bit
// (e4m3) and 4-bit (e2m1) groups of 32 elements with a power-of-two scale.
#pragma once

#include <hip/hip_runtime.h>

#include "dkv_cache.hpp"
#include "dkv_internal.hpp"

namespace dkv {

typedef short cs16x2 __attribute__((ext_vector_type(2)));

constexpr int kGroup = 32;          // elements per scale
constexpr int kScaleBias = 127;
constexpr int kScaleFirst = -100;   // smallest exponent written: no value of a group is subnormal in bf16
constexpr int kScaleNan = 255;      // group that held a NaN or an infinity

// A launch has less than 2^32 threads.
inline bool grid_fits(int64_t workgroups, int threads) { return workgroups <= 0xffffffffLL / threads; }

// Sequence that packed row t belongs to (the last that begins at or before it: -1 if none does), found by groups of N
// lanes, 64 / N of them a wave.
template <int N>
__device__ __forceinline__ int seq_of(const Pages &c, int t) {
  const int l = threadIdx.x & 63, lane = l % N;
  return last_at_most<N>(c.S, [&](int lo, int step, int hi) {
    const int s = lo + lane * step;
    const bool ok = s < hi && bound(c.start[s], 0, c.T) <= t;
    const uint64_t bits = (__ballot(ok) >> (l - lane)) & (~0ull >> (64 - N));
    return 63 - __clzll((long long)bits);
  });
}

// Scale code of a group whose largest magnitude is amax: the smallest exponent e with
// amax <= F 2^e.  F = 1.75 * 2^8 (e4m3) or 1.5 * 2^2 (e2m1), so with amax = 1.f * 2^a
// e is a - 8 (a - 2), and one more where 1.f exceeds 1.75 (1.5): a comparison of the
// fraction bits.  A subnormal amax has exponent field 0 and ends at the clamp.
template <int FMT>
__device__ __forceinline__ int scale_code(float amax) {
  const uint32_t u = __float_as_uint(amax);
  constexpr uint32_t frac = FMT == DKV_CACHE_FP8 ? 0x600000u : 0x400000u;
  constexpr int emax = FMT == DKV_CACHE_FP8 ? 8 : 2;
  const int code = (int)(u >> 23) - emax + ((u & 0x7fffffu) > frac ? 1 : 0);
  return u >= 0x7f800000u ? kScaleNan : max(code, kScaleBias + kScaleFirst);
}
// A group of the largest scale code holds values next to 2^128, which would round up to it: they take the largest value
// below, 1.875 x 2^127 (e4m3: off by at most 2^-4 of the value) or 1.5 x 2^127 (e2m1: 2^-2), and stay finite.
template <int FMT>
__device__ __forceinline__ void below_infinity(float *x, int code) {
  constexpr int top = kScaleBias + (FMT == DKV_CACHE_FP8 ? 120 : 126);
  constexpr float most = FMT == DKV_CACHE_FP8 ? 0x1.ep127f : 0x1.8p127f;
  if (code != top) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = fminf(fmaxf(x[j], -most), most);
}
__device__ __forceinline__ float scale_of(int code) { return __uint_as_float((uint32_t)code << 23); }

// Eight elements of a group -> 8 bytes (FP8) or 4 bytes (FP4): x / scale rounded to
// nearest even by the conversion instructions, which divide by the scale exactly.
__device__ __forceinline__ uint2 quantise_fp8(const float *x, float scale) {
  cs16x2 a = {0, 0}, b = {0, 0};
  a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, x[0], x[1], scale, false);
  a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, x[2], x[3], scale, true);
  b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, x[4], x[5], scale, false);
  b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, x[6], x[7], scale, true);
  return uint2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
}
__device__ __forceinline__ uint32_t quantise_fp4(const float *x, float scale) {
  uint32_t a = 0;
  a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(a, x[0], x[1], scale, 0);
  a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(a, x[2], x[3], scale, 1);
  a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(a, x[4], x[5], scale, 2);
  a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(a, x[6], x[7], scale, 3);
  return a;
}

// Eight elements as four packed bf16 pairs (exact: at most four significant bits).  A scale
// with all exponent bits set makes every result NaN.
__device__ __forceinline__ uint4 bf16_of_fp8(uint2 q, int code) {
  const float s = scale_of(code);
  return uint4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q.x, s, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q.x, s, true)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q.y, s, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q.y, s, true))};
}
__device__ __forceinline__ uint4 bf16_of_fp4(uint32_t q, int code) {
  const float s = scale_of(code);
  return uint4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, s, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, s, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, s, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, s, 3))};
}
__device__ __forceinline__ void unpack_bf16x8(uint4 p, float *x) {
  const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// Elements 8 c .. 8 c + 7 of a pool row as packed bf16 (bf16 caches) or floats.
template <int FMT, int D>
__device__ __forceinline__ uint4 load_bf16x8(const unsigned char *pool, const uint8_t *scale, size_t row, int c) {
  if constexpr (FMT == DKV_CACHE_FULL) {
    return *reinterpret_cast<const uint4 *>(pool + row * (2 * D) + 16 * c);
  } else {
    const int code = scale[row * (D / kGroup) + c / 4];
    if constexpr (FMT == DKV_CACHE_FP8) return bf16_of_fp8(*reinterpret_cast<const uint2 *>(pool + row * D + 8 * c), code);
    else return bf16_of_fp4(*reinterpret_cast<const uint32_t *>(pool + row * (D / 2) + 4 * c), code);
  }
}
template <int DT, int FMT, int D>
__device__ __forceinline__ void load_f32x8(const unsigned char *pool, const uint8_t *scale, size_t row, int c, float *x) {
  if constexpr (FMT == DKV_CACHE_FULL && DT == DKV_F32) {
    const float4 *p = reinterpret_cast<const float4 *>(pool + row * (4 * D) + 32 * c);
    const float4 a = p[0], b = p[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  } else {
    unpack_bf16x8(load_bf16x8<FMT, D>(pool, scale, row, c), x);
  }
}

}  // namespace dkv
