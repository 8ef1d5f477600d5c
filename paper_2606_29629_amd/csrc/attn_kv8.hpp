// Shared by the attention kernels over the 8-bit cache: codes and queries as float16.
#pragma once
#include "kv8.hpp"

namespace tri {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef f16 f16x2 __attribute__((ext_vector_type(2)));

// Splits of a sequence's rows: how many, rows of each (a multiple of the tile); and a bound
// on those of all sequences that never falls as the rows or the sequences grow.
struct Kv8Splits {
  int n, rows;
  int64_t most;
};
size_t attn_kv8_decode_bytes(const BatchDev& b, const Kv8Dev& c, int n_q_heads, int n_kv_heads,
                             int head_dim);
// The sequences of one new token; ws: attn_kv8_decode_bytes.
hipError_t launch_attn_kv8_decode(const BatchDev& b, const Kv8Dev& c, bool fp8, int n_q_heads,
                                  int n_kv_heads, int head_dim, const void* q, int64_t q_stride,
                                  void* out, float* ws, hipStream_t s);

// Eight codes (two dwords, in order) as float16, exact.  int8: with the sign bit flipped
// the byte b = code + 128 under the exponent of 1024 is 1024 + b; minus 1152.
template <bool FP8>
__device__ __forceinline__ f16x8 codes_to_f16(uint32_t a, uint32_t b) {
  union {
    f16x2 h[4];
    f16x8 v;
  } u;
  if constexpr (FP8) {
    u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false);
    u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
    u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false);
    u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
  } else {
    const f16x2 off = {(f16)-1152.f, (f16)-1152.f};
    a ^= 0x80808080u;
    b ^= 0x80808080u;
    u.h[0] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, a, 0x04010400u)) + off;
    u.h[1] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u)) + off;
    u.h[2] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u)) + off;
    u.h[3] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u)) + off;
  }
  return u.v;
}

// A head's bf16 query values, 8 N of them in each of the lanes that differ in the bits
// SHARE, as float16 times a power of two that brings the largest to [2^14, 2^15); returns
// the power of two that takes products back.  (A row that is not finite stays as it is.)
template <int SHARE, int N>
__device__ __forceinline__ float q_to_f16(const Pack8 (&x)[N], f16x8 (&o)[N]) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(bf2f(x[j].e[e])) & 0x7fffffffu);
#pragma unroll
  for (int bit = 1; bit < 64; bit <<= 1)
    if (SHARE & bit) m = max(m, (uint32_t)__shfl_xor((int)m, bit, 64));
  const int exp = (int)(m >> 23) - 127;  // (-127: zero or subnormal)
  const int up = m >= 0x7f800000u ? 0 : min(14 - exp, 126);
  const float f = __uint_as_float((uint32_t)(up + 127) << 23);
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) o[j][e] = (f16)(bf2f(x[j].e[e]) * f);
  return __uint_as_float((uint32_t)(127 - up) << 23);
}

// Largest of a lane's 16 scores.
__device__ __forceinline__ float tree_max16(const f32x16& s) {
  float m[5];
#pragma unroll
  for (int i = 0; i < 5; ++i) m[i] = max3f(s[3 * i], s[3 * i + 1], s[3 * i + 2]);
  return max3f(max3f(m[0], m[1], m[2]), max3f(m[3], m[4], s[15]), m[4]);
}

__device__ __forceinline__ float readlane_f(float v, int lane) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane));
}
// log2 of a power of two (NaN of NaN), and its inverse.
__device__ __forceinline__ float scale_log2(float s) {
  return s == s ? (float)((int)(__float_as_uint(s) >> 23) - 127) : s;
}
__device__ __forceinline__ float scale_inverse(float s) {
  return s == s ? __uint_as_float((254u << 23) - __float_as_uint(s)) : s;
}

}  // namespace tri
