// Device view and number formats of the 8-bit KV cache.
#pragma once
#include "common.hpp"
#include "kernels.hpp"

namespace tri {

template <int N>
struct Int {
  static constexpr int value = N;
};
// f(Int<0>{}) ... f(Int<N - 1>{})
template <int N, int I = 0, typename F>
__device__ __forceinline__ void each(F&& f) {
  if constexpr (I < N) {
    f(Int<I>{});
    each<N, I + 1>(f);
  }
}

constexpr int kKv8LeastExp = -100;  // exponent of the smallest scale

// First scale of (panel, head), and the first row's index in mass / stamp.
__device__ __forceinline__ int64_t kv8_scale_at(const Kv8Dev& c, int Hkv, int panel, int h, int prow) {
  return ((int64_t)panel * Hkv + h) * c.scales_per_panel() + (prow >> c.scale_shift);
}
__device__ __forceinline__ int64_t kv8_row_at(const Kv8Dev& c, int Hkv, int panel, int h, int prow) {
  return ((int64_t)panel * Hkv + h) * c.kv.panel_rows() + prow;
}

// The sequence's new tokens [q0, q0 + n), cached rows and slot; false where it has
// none or is to be skipped (s < n_seqs by the grid).
__device__ __forceinline__ bool kv8_seq(const BatchDev& b, const Kv8Dev& c, int s, int& q0, int& n,
                                        int& ctx, int& sl) {
  q0 = b.cu_q[s];
  const int q1 = b.cu_q[s + 1];
  ctx = b.ctx_len[s];
  sl = b.slot[s];
  n = q1 - q0;
  return q0 >= 0 && n >= 0 && q1 <= b.n_tokens && ctx >= 0 && sl >= 0 && sl < c.kv.n_slots &&
         n <= c.kv.max_seq && ctx <= c.kv.max_seq - n;
}

// The least power of two s >= 2^-100 with amax <= top * s, from the bits of amax
// (127 = 1.984375 * 2^6, 448 = 1.75 * 2^8: one comparison of mantissas decides); NaN
// where amax is not finite.  Magnitudes as integers: a NaN is the largest.
template <bool FP8>
__device__ __forceinline__ float kv8_scale_of(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
  int e = (int)(amax_bits >> 23) - 127 - (FP8 ? 8 : 6);
  if ((amax_bits & 0x7fffffu) > (FP8 ? 0x600000u : 0x7e0000u)) ++e;
  return __uint_as_float((uint32_t)(max(e, kKv8LeastExp) + 127) << 23);
}
// The larger of two scales; NaN if either is (the bits of a NaN are the larger).
__device__ __forceinline__ float kv8_scale_max(float a, float b) {
  return __uint_as_float(max(__float_as_uint(a) & 0x7fffffffu, __float_as_uint(b) & 0x7fffffffu));
}
// 1 / s of a power of two; 0 for NaN (whose codes are all zero).
__device__ __forceinline__ float kv8_inverse(float s) {
  return s == s ? __uint_as_float((254u << 23) - __float_as_uint(s)) : 0.f;
}

// Four codes in a dword <-> floats.  Values are finite and within the type.
template <bool FP8>
__device__ __forceinline__ f32x4 kv8_decode4(uint32_t w) {
  if constexpr (FP8) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
    const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return f32x4{a[0], a[1], b[0], b[1]};
  } else {
    return f32x4{(float)(int8_t)w, (float)(int8_t)(w >> 8), (float)(int8_t)(w >> 16),
                 (float)(int8_t)(w >> 24)};
  }
}
template <bool FP8>
__device__ __forceinline__ uint32_t kv8_encode4(f32x4 v) {
  if constexpr (FP8) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w, true);
  } else {
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) w |= ((uint32_t)(int)rintf(v[e]) & 0xffu) << (8 * e);
    return w;
  }
}
// Sixteen codes times `f` (a power of two <= 1, or 0), rounded again.
template <bool FP8>
__device__ __forceinline__ u32x4 kv8_rescale16(u32x4 c, float f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = kv8_encode4<FP8>(kv8_decode4<FP8>(c[i]) * f);
  return c;
}

}  // namespace tri
