// Rows into pages and back: sparq_paged_append, sparq_paged_read.
//
// A row is the d_h values of one position and KV head.  In 8 bits it is stored as code * scale with scale = a / qmax, a its
// largest magnitude (fp32 division), and code = the nearest code to x (qmax / a): one multiplication by a quotient that is
// rounded once, so that the codes are those of the same three operations anywhere.
// Bound by HBM: every byte is moved once, nothing is kept.  d_h / 8 lanes share a row (16 bytes each of the 16-bit side), and
// a thread has its part of the K row and of the V row in flight together.  Rows that are read back are stored past the caches, which
// leaves these to the pages: 31 777 rows of 8 KV heads from e4m3 pages (197 MB) 32.5 us (6.1 TB/s; 45.4 with ordinary stores, 41.7 with
// loads past the caches too).  16 sequences of up to 512 rows of 8 KV heads into e4m3 pages: 8.8 us (2.7 TB/s), of which a launch that
// waits for its length, page and row takes 3.4.
#include "paged_codes.h"

namespace sparq {
namespace {

constexpr int RT = 256;            // threads per workgroup

// What a thread does: 8 channels of one row, and whether the row is to be moved.
struct Item { int b, t, head, c0, pos; SeqRows r; bool on; };

template <int DH>
__device__ __forceinline__ Item item_of(const PagedRowsArgs& a, bool reads) {
  constexpr int LPR = DH / 8;
  const PagedArgs& p = a.p;
  Item it;
  const uint32_t n_items = (uint32_t)p.B * p.n * p.H_kv;               // (checked to fit by the host)
  const uint32_t i = blockIdx.x * (RT / LPR) + threadIdx.x / LPR;
  it.on = i < n_items;
  const int j = it.on ? (int)i : 0;
  const int row = divided(j, p.by_H_kv);
  it.head = j - row * p.H_kv;                                           // heads vary fastest: rows of a token lie together
  it.b = divided(row, p.by_n);
  it.t = row - it.b * p.n;
  it.c0 = threadIdx.x % LPR * 8;
  it.r = seq_rows(p.seq_lens[it.b], p.bound, p.n, p.n_per_seq, p.row_start, p.n_rows, it.b);
  if (reads) {
    const int64_t at = (int64_t)(a.first ? a.first[it.b] : 0) + it.t;
    it.pos = at >= 0 && at < it.r.S ? (int)at : -1;
    if (it.t < it.r.n && it.pos < 0) it.r.err |= kErrBadSeqLen;
  } else {
    if (it.r.n > it.r.S) { it.r.n = 0; it.r.err |= kErrBadSeqLen; }
    it.pos = it.r.S - it.r.n + it.t;
  }
  if (it.on && it.t == 0 && it.head == 0 && it.c0 == 0 && it.r.err) atomicOr(p.err, it.r.err);
  it.on = it.on && it.t < it.r.n && it.pos >= 0;
  return it;
}

// The row's number in the pool; -1 (and the error bit) where the table names no page.
__device__ __forceinline__ int64_t place_of(const PagedArgs& p, const Item& it) {
  const int index = divided(it.pos, p.by_page), page = page_at(p, it.b, index);
  if (page < 0) { atomicOr(p.err, kErrBadPage); return -1; }
  return pool_row(p, page, it.head, it.pos - index * p.page_size);
}

template <class T, int PT, int DH>
__device__ __forceinline__ void store_row(void* pool, float* scales, int64_t row, int c0, const uint4& x) {
  if constexpr (PT == kPages16) {
    *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(pool) + row * DH + c0) = x;
  } else {
    constexpr float qmax = PT == kPagesI8 ? kMaxI8 : kMaxE4M3;
    float f[8];
    unpack8<T>(x, f);
    uint32_t top = 0;              // magnitudes compare as their bits; infinities and NaN are the largest
#pragma unroll
    for (int i = 0; i < 8; ++i) { const uint32_t u = __float_as_uint(f[i]) & 0x7fffffffu; top = u > top ? u : top; }
#pragma unroll
    for (int o = 1; o < DH / 8; o <<= 1) { const uint32_t u = __shfl_xor(top, o); top = u > top ? u : top; }
    const bool finite = top < 0x7f800000u;
    const float a = fminf(fmaxf(__uint_as_float(top), kLeastMagnitude), kMostMagnitude);
    const float inv = qmax / a;
    uint2 codes;
    codes.x = codes_of<PT>(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv);
    codes.y = codes_of<PT>(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv);
    if (!finite) codes = make_uint2(0u, 0u);
    *reinterpret_cast<uint2*>(reinterpret_cast<uint8_t*>(pool) + row * DH + c0) = codes;
    if (c0 == 0) scales[row] = finite ? a / qmax : __uint_as_float(0x7fc00000u);
  }
}

template <class T, int PT, int DH>
__global__ __launch_bounds__(RT) void paged_append(const PagedRowsArgs a) {
  const Item it = item_of<DH>(a, false);
  // (the lanes of a row share everything that decides whether it is written)
  if (!it.on) return;
  const int64_t from = row_offset(a.s, a.p.row_start != nullptr, it.b, it.r.row0, it.head, it.t) + it.c0;
  const uint4 k = load16(reinterpret_cast<const uint16_t*>(a.k) + from), v = load16(reinterpret_cast<const uint16_t*>(a.v) + from);
  const int64_t row = place_of(a.p, it);
  if (row < 0) return;
  store_row<T, PT, DH>(a.p.K, a.p.K_scale, row, it.c0, k);
  store_row<T, PT, DH>(a.p.V, a.p.V_scale, row, it.c0, v);
}

template <class T, int PT, int DH>
__device__ __forceinline__ uint4 load_row(const void* pool, const float* scales, int64_t row, int c0) {
  if constexpr (PT == kPages16) {
    return load16(reinterpret_cast<const uint16_t*>(pool) + row * DH + c0);
  } else {
    const uint2 w = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint8_t*>(pool) + row * DH + c0);
    const float s = scales[row];
    const uint2 lo = codes_to_half<PT>(w.x), hi = codes_to_half<PT>(w.y);
    float f[8];
    unpack8<F16>(make_uint4(lo.x, lo.y, hi.x, hi.y), f);
    return make_uint4(narrow2<T>(f[0] * s, f[1] * s), narrow2<T>(f[2] * s, f[3] * s), narrow2<T>(f[4] * s, f[5] * s), narrow2<T>(f[6] * s, f[7] * s));
  }
}

template <class T, int PT, int DH>
__global__ __launch_bounds__(RT) void paged_read(const PagedRowsArgs a) {
  const Item it = item_of<DH>(a, true);
  if (!it.on) return;
  const int64_t row = place_of(a.p, it);
  if (row < 0) return;
  const uint4 k = load_row<T, PT, DH>(a.p.K, a.p.K_scale, row, it.c0), v = load_row<T, PT, DH>(a.p.V, a.p.V_scale, row, it.c0);
  const int64_t to = row_offset(a.s, a.p.row_start != nullptr, it.b, it.r.row0, it.head, it.t) + it.c0;
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4, k), reinterpret_cast<u32x4*>(reinterpret_cast<uint16_t*>(a.k) + to));
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<u32x4*>(reinterpret_cast<uint16_t*>(a.v) + to));
}

template <class T, int PT, int DH>
hipError_t launch_rows(const PagedRowsArgs& a, bool reads, hipStream_t s) {
  const int64_t items = (int64_t)a.p.B * a.p.n * a.p.H_kv, per = RT / (DH / 8);
  const dim3 grid((uint32_t)((items + per - 1) / per));
  if (reads) hipLaunchKernelGGL((paged_read<T, PT, DH>), grid, dim3(RT), 0, s, a);
  else hipLaunchKernelGGL((paged_append<T, PT, DH>), grid, dim3(RT), 0, s, a);
  return hipGetLastError();
}
template <class T, int PT>
hipError_t launch_d(const PagedRowsArgs& a, bool reads, hipStream_t s) {
  switch (a.p.d_h) {
    case 64: return launch_rows<T, PT, 64>(a, reads, s);
    case 128: return launch_rows<T, PT, 128>(a, reads, s);
    case 256: return launch_rows<T, PT, 256>(a, reads, s);
    default: return hipErrorInvalidValue;
  }
}
hipError_t launch(const PagedRowsArgs& a, bool reads, int dtype, int page_type, hipStream_t s) {
  const bool bf = dtype == 1;
  switch (page_type) {
    case kPages16: return launch_d<F16, kPages16>(a, reads, s);          // (moved as they are)
    case kPagesI8: return bf ? launch_d<BF16, kPagesI8>(a, reads, s) : launch_d<F16, kPagesI8>(a, reads, s);
    case kPagesE4M3: return bf ? launch_d<BF16, kPagesE4M3>(a, reads, s) : launch_d<F16, kPagesE4M3>(a, reads, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_paged_append(const PagedRowsArgs& a, int dtype, int page_type, hipStream_t s) { return launch(a, false, dtype, page_type, s); }
hipError_t launch_paged_read(const PagedRowsArgs& a, int dtype, int page_type, hipStream_t s) { return launch(a, true, dtype, page_type, s); }

}  // namespace sparq
