// 8-bit codes of the paged cache and their exact 16-bit values.
#pragma once
#include "common.h"
#include "paged.h"

namespace sparq {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// Two floats as a pair of 16-bit values, rounded to nearest-even; infinities and NaN stay what they are.
template <class T> __device__ __forceinline__ uint32_t narrow2(float a, float b);
template <> __device__ __forceinline__ uint32_t narrow2<F16>(float a, float b) {
  return __builtin_bit_cast(uint32_t, half2_t{(_Float16)a, (_Float16)b});
}
template <> __device__ __forceinline__ uint32_t narrow2<BF16>(float a, float b) {
  return __builtin_bit_cast(uint32_t, bf16x2_t{(__bf16)a, (__bf16)b});
}

// Four codes (bytes of `w`) as fp16, which holds every one of them exactly (8 bits of an integer, 4 of an e4m3 value).
template <int PT> __device__ __forceinline__ uint2 codes_to_half(uint32_t w) {
  if constexpr (PT == kPagesE4M3) {
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, true)));
  } else {
    // 0x6400 | u is 1024 + u: with u = code + 128 the code is what is left above 1152
    const uint32_t u = w ^ 0x80808080u;
    const half2_t off = {(_Float16)1152.0f, (_Float16)1152.0f};
    const half2_t lo = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - off;
    const half2_t hi = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - off;
    return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
  }
}

// Four values, already divided by the row's scale, as codes.
template <int PT> __device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d) {
  constexpr float most = PT == kPagesI8 ? kMaxI8 : kMaxE4M3;
  const float x[4] = {__builtin_amdgcn_fmed3f(a, -most, most), __builtin_amdgcn_fmed3f(b, -most, most),
                      __builtin_amdgcn_fmed3f(c, -most, most), __builtin_amdgcn_fmed3f(d, -most, most)};
  if constexpr (PT == kPagesE4M3) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
  } else {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= ((uint32_t)(int)rintf(x[i]) & 0xffu) << (8 * i);
    return w;
  }
}

}  // namespace sparq
