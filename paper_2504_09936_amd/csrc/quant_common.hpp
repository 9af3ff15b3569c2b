// e4m3 codes and their scales: what the kernels on caches of codes share.
#pragma once

#include <type_traits>

#include "kk_common.hpp"

namespace kk {

constexpr int kQBlock = KEEPKV_QUANT_BLOCK;      // slots that share a scale
constexpr int kScaleLow = -110, kScaleHigh = 120;

inline __host__ __device__ int quant_blocks(int capacity) { return (capacity + kQBlock - 1) / kQBlock; }

typedef __attribute__((ext_vector_type(2))) float f32x2_t;

// The bits of the scale for a largest finite magnitude with bits `amax` (sign clear): the smallest 2^e with amax <= 448 * 2^e.
// 448 = 1.75 * 2^8, so with amax = m * 2^x, 1 <= m < 2, e is x - 8 if m <= 1.75 and x - 7 otherwise.
__device__ __forceinline__ uint32_t scale_bits(uint32_t amax) {
  const int e = (int)(amax >> 23) - 127 - 8 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return (uint32_t)(min(max(e, kScaleLow), kScaleHigh) + 127) << 23;
}
// 1 / scale, exact
__device__ __forceinline__ float inverse_scale(uint32_t bits) { return __builtin_bit_cast(float, (254u << 23) - bits); }

// Bits of |x| if x is finite, else 0: ordered like the magnitudes.
__device__ __forceinline__ uint32_t finite_magnitude(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu;
  return u < 0x7F800000u ? u : 0u;
}

// Four f32 (already divided by the scale) as codes, to nearest even; encode4: an infinity becomes NaN, encode4_no_inf: there is none.
__device__ __forceinline__ uint32_t encode4_no_inf(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  auto nan_if_inf = [](float x) { return __builtin_fabsf(x) == INFINITY ? __builtin_nanf("") : x; };
  return encode4_no_inf(nan_if_inf(a), nan_if_inf(b), nan_if_inf(c), nan_if_inf(d));
}
// Four codes as f32.
__device__ __forceinline__ void decode4(uint32_t w, float (&x)[4]) {
  const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = lo[0];
  x[1] = lo[1];
  x[2] = hi[0];
  x[3] = hi[1];
}

// Four codes under a scale that is larger by 1 / ratio (ratio a power of two below 1).
__device__ __forceinline__ uint32_t shift_codes(uint32_t w, float ratio) {
  float x[4];
  decode4(w, x);
  return encode4_no_inf(x[0] * ratio, x[1] * ratio, x[2] * ratio, x[3] * ratio);
}

// Maximum over the wavefront, in every lane: register moves, where six exchanges through LDS cost 0.2 us of a short launch (quantising 8 heads x
// 800 slots 5.56 / 5.34 us, appending 8000 tokens to 8 heads 13.14 / 12.88).
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  auto dpp = [](uint32_t v, auto ctrl) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xF, 0xF, true); };
  x = max(x, dpp(x, std::integral_constant<int, 0x121>{}));      // row_ror:1, 2, 4, 8
  x = max(x, dpp(x, std::integral_constant<int, 0x122>{}));
  x = max(x, dpp(x, std::integral_constant<int, 0x124>{}));
  x = max(x, dpp(x, std::integral_constant<int, 0x128>{}));
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  const uint32_t r0 = r[0], r1 = r[1];
  x = max(r0, r1);
  const auto h = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  const uint32_t h0 = h[0], h1 = h[1];
  return max(h0, h1);
}

// 16 / sizeof(T) elements of a row from 16 bytes
__device__ __forceinline__ void to_f32(uint4 u, float (&x)[4]) {
  x[0] = __builtin_bit_cast(float, u.x);
  x[1] = __builtin_bit_cast(float, u.y);
  x[2] = __builtin_bit_cast(float, u.z);
  x[3] = __builtin_bit_cast(float, u.w);
}
__device__ __forceinline__ void to_f32(uint4 u, float (&x)[8]) {
  x[0] = bf16_lo(u.x); x[1] = bf16_hi(u.x);
  x[2] = bf16_lo(u.y); x[3] = bf16_hi(u.y);
  x[4] = bf16_lo(u.z); x[5] = bf16_hi(u.z);
  x[6] = bf16_lo(u.w); x[7] = bf16_hi(u.w);
}

inline bool quant_cache_ok(const keepkv_quant_cache* c) { return c && cache_ok(&c->c) && c->k_scale && c->v_scale; }

}  // namespace kk
