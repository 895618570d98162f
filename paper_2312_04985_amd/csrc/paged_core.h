// What the two attention kernels over the paged cache share.
#pragma once
#include <type_traits>

#include "paged_codes.h"

namespace sparq {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// The products' type: the rows' own, and fp16 for 8-bit pages, which holds every code exactly.
template <class T, int PT> using Product = std::conditional_t<PT == kPages16, T, F16>;

// Four 16-bit elements of a column: each group of 16 lanes reads 4 rows of 16 elements (lanes 4 r .. 4 r + 3 point at the
// four 8-byte pieces of row r), lane i of the group gets column i.
__device__ __forceinline__ uint2 lds_read_transposed(uint16_t* p) {
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
}

// whether one of eight 16-bit values is an infinity or NaN
template <class T> __device__ __forceinline__ bool has_special(const uint4& v) {
  constexpr uint32_t e = std::is_same_v<T, F16> ? 0x7c00u : 0x7f80u;
  bool found = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = (&v.x)[i];
    found = found || (w & e) == e || ((w >> 16) & e) == e;
  }
  return found;
}

// A value's scale as the attention uses it: a scale of 0 (rows of zeros that another program wrote) has no logarithm; NaN stays.
__device__ __forceinline__ float value_scale(float s) { return s < kLeastMagnitude / 1024.0f ? kLeastMagnitude / 1024.0f : s; }

// bf16 queries for products of fp16 (8-bit pages): a row, whose pieces lie in the lanes l ^ X, l ^ 2 X .. l ^ 32, is multiplied by a power
// of 2, the inverse of which is returned: 1 where its largest finite magnitude lies in [2^-4, 2^15), as those of most rows do, otherwise
// what brings it into [2^14, 2^15).  fp16 then holds every bf16 value of 2^-17 and more exactly, the others to within 2^-25: 2^-21 of the row's
// largest, less than the sums' own roundings.
template <int X, int N> __device__ __forceinline__ float query_to_half(uint4 (&q)[N]) {
  uint32_t top = 0;
#pragma unroll
  for (int s = 0; s < N; ++s)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = (&q[s].x)[i], x0 = w & 0x7f80u, x1 = (w >> 16) & 0x7f80u;
      if (x0 < 0x7f80u && x0 > top) top = x0;
      if (x1 < 0x7f80u && x1 > top) top = x1;
    }
#pragma unroll
  for (int o = X; o < kWave; o <<= 1) { const uint32_t other = __shfl_xor(top, o); top = other > top ? other : top; }
  int e = (int)(top >> 7) - 127;                               // exponent of the largest finite magnitude
  e = e < -112 ? -112 : e;                                     // (2^(14 - e) stays a float)
  const int lift = e >= -4 && e < 15 ? 0 : 14 - e;
  const float up = __uint_as_float((uint32_t)(lift + 127) << 23);
#pragma unroll
  for (int s = 0; s < N; ++s) {
    float f[8];
    unpack8<BF16>(q[s], f);
    q[s] = make_uint4(narrow2<F16>(f[0] * up, f[1] * up), narrow2<F16>(f[2] * up, f[3] * up), narrow2<F16>(f[4] * up, f[5] * up), narrow2<F16>(f[6] * up, f[7] * up));
  }
  return __uint_as_float((uint32_t)(127 - lift) << 23);
}

// n / d for results that fit an int (64-bit divisions are long)
__device__ __forceinline__ int quotient(int64_t n, int64_t d) { return n <= UINT32_MAX && d <= UINT32_MAX ? (int)((uint32_t)n / (uint32_t)d) : (int)(n / d); }

// The positions [lo, hi) that row t of a sequence sees.  Both rise with t.
struct Seen { int lo, hi; };
__device__ __forceinline__ Seen seen_by(const PagedAttendArgs& a, const SeqRows& r, int t) {
  const int pos = r.S - r.n + t;
  return Seen{a.window > 0 && pos - a.window + 1 > 0 ? pos - a.window + 1 : 0, a.all ? r.S : pos + 1};
}

// Where a row's logarithm of the denominator goes.
__device__ __forceinline__ int64_t lse_place(const PagedAttendArgs& a, const SeqRows& r, int b, int head, int t) {
  return a.p.row_start ? (int64_t)head * a.p.n_rows + r.row0 + t : ((int64_t)b * a.p.H + head) * a.p.n + t;
}
constexpr float kLn2 = 0.6931471805599453f;

}  // namespace sparq
