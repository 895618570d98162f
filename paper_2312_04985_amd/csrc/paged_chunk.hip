// Attention of many rows per (sequence, KV head) over a paged cache: chunks of new tokens, whole prompts.
//
// A workgroup serves 32 rows per wave of one (sequence, KV head): row m stands for token m / g and query head m % g of the
// group, so that the heads of a group share what is read of the cache.  It walks the positions that its rows see in tiles
// of 64 through LDS, one pass, with the running maximum and sum of the softmax.
//   scores   S^T[position][row] = K Q^T by 32x32x16 matrix instructions: a lane then holds 32 scores of ONE row, so that
//            maximum and sum are taken inside the lane (and once across the two halves of the wave)
//   weights  P^T[position][row]: the lane's weights are, as they stand, the right operand of the next product if its
//            contraction runs over the positions in the order (8 a + 4 h + j), a = 0, 1, j = 0 .. 3 of lane half h
//   output   O^T[channel][row] += V^T P^T; V^T comes out of LDS by the transposing load, in the same order of positions.
// 8-bit pages: every code is a 16-bit float, so the products are those of 16-bit pages; a key's scale multiplies its scores.
// A value's scale goes into the exponent: w_j = 2^(x_j + log2 s_j - m) <= 1 is what multiplies the codes, and w_j / s_j what
// is summed.  Neither needs a rounding that 16-bit pages do not have.
#include "paged_core.h"

namespace sparq {
namespace {

constexpr int kTile = 64;               // positions per tile

// c[m][n] += sum_k a[m][k] b[n][k] over 16 k: lane l holds a[l % 32], b[l % 32] at k = 8 (l / 32) .. + 7 and
// c[8 (i / 4) + 4 (l / 32) + i % 4][l % 32]
template <class T> __device__ __forceinline__ f32x16 mfma_32x32x16(const uint4& a, const uint4& b, f32x16 c);
template <> __device__ __forceinline__ f32x16 mfma_32x32x16<F16>(const uint4& a, const uint4& b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x16 mfma_32x32x16<BF16>(const uint4& a, const uint4& b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Rows of DH elements in LDS in pieces of 8 (16 bytes).  Keys are read by 32 rows at one piece, values by 8 rows at 4
// neighbouring pieces: both are spread over the banks by changing the pieces' places with the row.
template <int DH> __device__ __forceinline__ int key_piece(int row, int piece) { return row * DH + ((piece ^ (row & (DH / 8 - 1) & 15)) << 3); }
template <int DH> __device__ __forceinline__ int value_piece(int row, int piece) {
  const int turn = DH == 64 ? ((row & 1) << 2) | ((row >> 1) & 3) : ((row & 3) << 2) | ((row >> 2) & 3);
  return row * DH + ((piece ^ turn) << 3);
}

template <class T, int PT, int DH, int NW>
__global__ __launch_bounds__(NW * 64) void paged_chunk(const PagedAttendArgs a) {
  using E = Product<T, PT>;
  constexpr int NT = NW * 64, ROWS = NW * 32, PIECES = DH / 8;
  __shared__ __align__(16) uint16_t Kt[kTile * DH], Vt[kTile * DH];
  __shared__ __align__(16) float s_k[kTile], s_log[kTile], s_inv[kTile];   // 8-bit pages: scale of the key, log2 and inverse of the value's
  const PagedArgs& p = a.p;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, half = lane >> 5;

  // Workgroups are dealt round-robin to the 8 XCDs: eight (sequence, KV head) units at a time, so that the workgroups that
  // share rows of the cache share an XCD's L2; a unit's last row tiles, which see most, first.
  const int units = p.B * p.H_kv, chunk = blockIdx.x / (8 * a.n_tiles), in_chunk = blockIdx.x - chunk * 8 * a.n_tiles;
  const int width = units - chunk * 8 < 8 ? units - chunk * 8 : 8;
  const int tile_up = in_chunk / width, unit = chunk * 8 + in_chunk - tile_up * width, tile = a.n_tiles - 1 - tile_up;
  const int b = divided(unit, p.by_H_kv), hk = unit - b * p.H_kv;
  const SeqRows r = seq_rows(p.seq_lens[b], p.bound, p.n, p.n_per_seq, p.row_start, p.n_rows, b);
  if (r.err && tid == 0 && hk == 0 && tile == 0) atomicOr(p.err, r.err);
  const int M = r.n * a.group, m0 = tile * ROWS;
  if (m0 >= M || M <= a.skip_rows) return;
  const bool packed = p.row_start != nullptr;

  const int m_w = m0 + wave * 32, m_last = M - 1;
  const bool live = m_w < M;                                   // a wave without rows only helps to load
  const int m = m_w + col < M ? m_w + col : m_last;
  const int t = divided(m, a.by_group), head = hk * a.group + m - t * a.group;
  const auto row_sees = [&](int m) { return seen_by(a, r, divided(m < M ? m : m_last, a.by_group)); };
  const Seen mine = seen_by(a, r, t), wg_first = row_sees(m0), wg_last = row_sees(m0 + ROWS - 1), w_first = row_sees(m_w), w_last = row_sees(m_w + 31);
  const int lo = mine.lo;
  const uint32_t len = mine.hi > lo ? (uint32_t)(mine.hi - lo) : 0u;

  // the lane's part of its row of Q: channels 16 s + 8 half .. + 7
  uint4 qf[DH / 16];
  const uint16_t* qp = reinterpret_cast<const uint16_t*>(a.q) + row_offset(a.qs, packed, b, r.row0, head, t) + half * 8;
#pragma unroll
  for (int s = 0; s < DH / 16; ++s) qf[s] = *reinterpret_cast<const uint4*>(qp + s * 16);
  float c_row = kLog2e / sqrtf((float)DH);                     // scores to exponents of 2
  if constexpr (PT != kPages16 && std::is_same_v<T, BF16>) query_to_half<32>(qf, c_row);

  f32x16 O[DH / 32];
#pragma unroll
  for (int j = 0; j < DH / 32; ++j)
#pragma unroll
    for (int i = 0; i < 16; ++i) O[j][i] = 0.0f;
  float m_ref = -INFINITY, l = 0.0f;

  const int begin = wg_first.lo / kTile * kTile;
  for (int p0 = begin; p0 < wg_last.hi; p0 += kTile) {
    // ---- the tile into LDS: 16 rows of a page per turn of a wave ----
    for (int g = wave; g < kTile / 16; g += NW) {
      const int pos0 = p0 + g * 16;
      const int at = pos0 < r.S ? pos0 : 0;                    // (behind the last position: any row, its values are not used)
      const int index = divided(at, p.by_page);
      int page = page_at(p, b, index);
      if (page < 0) { if (lane == 0) atomicOr(p.err, kErrBadPage); page = 0; }
      const int64_t row = pool_row(p, page, hk, at - index * p.page_size);
      if constexpr (PT == kPages16) {
        const uint16_t* kp = reinterpret_cast<const uint16_t*>(p.K) + row * DH;
        const uint16_t* vp = reinterpret_cast<const uint16_t*>(p.V) + row * DH;
#pragma unroll
        for (int i = 0; i < 16 * PIECES / 64; ++i) {
          const int e = i * 64 + lane, rr = e / PIECES, piece = e % PIECES;
          const uint4 k = *reinterpret_cast<const uint4*>(kp + e * 8);
          uint4 v = *reinterpret_cast<const uint4*>(vp + e * 8);
          if (pos0 + rr >= r.S) v = make_uint4(0, 0, 0, 0);
          *reinterpret_cast<uint4*>(&Kt[key_piece<DH>(g * 16 + rr, piece)]) = k;
          *reinterpret_cast<uint4*>(&Vt[value_piece<DH>(g * 16 + rr, piece)]) = v;
        }
      } else {
        const uint8_t* kp = reinterpret_cast<const uint8_t*>(p.K) + row * DH;
        const uint8_t* vp = reinterpret_cast<const uint8_t*>(p.V) + row * DH;
#pragma unroll
        for (int i = 0; i < 16 * PIECES / 64; ++i) {
          const int e = i * 64 + lane, rr = e / PIECES, piece = e % PIECES;
          const uint2 k = *reinterpret_cast<const uint2*>(kp + e * 8);
          uint2 v = *reinterpret_cast<const uint2*>(vp + e * 8);
          uint2 x = codes_to_half<PT>(k.x), y = codes_to_half<PT>(k.y);
          *reinterpret_cast<uint4*>(&Kt[key_piece<DH>(g * 16 + rr, piece)]) = make_uint4(x.x, x.y, y.x, y.y);
          x = codes_to_half<PT>(v.x); y = codes_to_half<PT>(v.y);
          uint4 w = make_uint4(x.x, x.y, y.x, y.y);
          if (pos0 + rr >= r.S) w = make_uint4(0, 0, 0, 0);
          *reinterpret_cast<uint4*>(&Vt[value_piece<DH>(g * 16 + rr, piece)]) = w;
        }
        if (lane < 16) {
          const float sk = p.K_scale[row + lane], sv = p.V_scale[row + lane];
          const float v = value_scale(sv);
          s_k[g * 16 + lane] = sk;
          s_log[g * 16 + lane] = log2_normal(v);
          s_inv[g * 16 + lane] = 1.0f / v;
        }
      }
    }
    __syncthreads();

    // ---- scores, exponents, weights ----
    // (a row's exponent of 2 at position j is x_j = c q . K_j, with 8-bit pages plus log2 s_j)
    const bool active = live && p0 < w_last.hi && p0 + kTile > w_first.lo;
    f32x16 S[2];
    if (active) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int e = 0; e < 16; ++e) S[i][e] = 0.0f;
#pragma unroll
        for (int s = 0; s < DH / 16; ++s)
          S[i] = mfma_32x32x16<E>(*reinterpret_cast<const uint4*>(&Kt[key_piece<DH>(i * 32 + col, 2 * s + half)]), qf[s], S[i]);
      }
      const bool masked = p0 < w_last.lo || p0 + kTile > w_first.hi;
      const uint32_t from = (uint32_t)(p0 + 4 * half - lo);
      f32x16 inv[2];
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int j = 32 * i + 8 * (e / 4) + e % 4, at = j + 4 * half;
          float x;
          if constexpr (PT == kPages16) x = S[i][e] * c_row;
          else { x = fmaf(S[i][e], s_k[at] * c_row, s_log[at]); inv[i][e] = s_inv[at]; }
          if (masked && from + j >= len) { x = -INFINITY; if constexpr (PT != kPages16) inv[i][e] = 0.0f; }
          S[i][e] = x;
          mx = fmaxf(mx, x);
        }
      float m_a, m_b;
      lane_pair<32>(mx, m_a, m_b);
      const float m_new = fmaxf(fmaxf(m_a, m_b), m_ref);
      if (__ballot(m_new > m_ref)) {
        const float w = weight_exp2(m_ref, m_new);
        m_ref = m_new;
        l *= w;
#pragma unroll
        for (int j = 0; j < DH / 32; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e) O[j][e] *= w;
      }
      const float m_use = m_ref == -INFINITY ? 0.0f : m_ref;     // (nothing seen yet: every weight is 2^-inf)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          S[i][e] = exp2_weight(S[i][e] - m_use);
          if constexpr (PT == kPages16) l += S[i][e];
          else l = fmaf(S[i][e], inv[i][e], l);
        }
    }

    // ---- infinities and NaN among the values of positions that some rows of the tile do not see: a weight of 0 would
    // still make NaN of them.  They are added to the rows that see them, and zeros take their places. ----
    if constexpr (PT == kPages16) {
      if (p0 < wg_last.lo || p0 + kTile > wg_first.hi) {
        bool found = false;
        for (int e = tid; e < kTile * PIECES; e += NT) found = found || has_special<T>(*reinterpret_cast<const uint4*>(&Vt[e * 8]));
        if (__syncthreads_or(found)) {
          if (active)
            for (int j = 0; j < kTile; ++j) {
              if ((uint32_t)(p0 + j - lo) >= len) continue;
#pragma unroll
              for (int jj = 0; jj < DH / 32; ++jj)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                  const int d = 32 * jj + 8 * (e / 4) + 4 * half + e % 4;
                  const float v = T::widen(Vt[value_piece<DH>(j, d / 8) + d % 8]);
                  if (!(fabsf(v) < INFINITY)) O[jj][e] += v;
                }
            }
          __syncthreads();
          for (int e = tid; e < kTile * DH; e += NT)
            if (!(fabsf(T::widen(Vt[e])) < INFINITY)) Vt[e] = 0;
          __syncthreads();
        }
      }
    }

    // ---- output ----
    if (active) {
#pragma unroll
      for (int sl = 0; sl < 4; ++sl) {
        const int e0 = sl % 2 * 8;
        const f32x16& w = S[sl / 2];
        const uint4 pw = make_uint4(narrow2<E>(w[e0], w[e0 + 1]), narrow2<E>(w[e0 + 2], w[e0 + 3]), narrow2<E>(w[e0 + 4], w[e0 + 5]), narrow2<E>(w[e0 + 6], w[e0 + 7]));
        const int row = sl * 16 + 4 * half + (lane & 15) / 4;
#pragma unroll
        for (int j = 0; j < DH / 32; ++j) {
          const int piece = 4 * j + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1), sub = (lane & 1) * 4;
          const uint2 v0 = lds_read_transposed(&Vt[value_piece<DH>(row, piece) + sub]), v1 = lds_read_transposed(&Vt[value_piece<DH>(row + 8, piece) + sub]);
          O[j] = mfma_32x32x16<E>(make_uint4(v0.x, v0.y, v1.x, v1.y), pw, O[j]);
        }
      }
    }
    __syncthreads();                                             // the next tile overwrites this one
  }

  // ---- a row's two halves have summed half of its weights each ----
  float l_a, l_b;
  lane_pair<32>(l, l_a, l_b);
  l = l_a + l_b;
  if (!live || m_w + col >= M) return;
  const bool none = l == 0.0f;                                   // nothing seen: zeros (a sum that is NaN stays NaN)
  const float inv_l = none ? 0.0f : 1.0f / l;
  uint16_t* op = reinterpret_cast<uint16_t*>(a.out) + row_offset(a.os, packed, b, r.row0, head, t);
#pragma unroll
  for (int j = 0; j < DH / 32; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint2 w = make_uint2(narrow2<T>(O[j][4 * q] * inv_l, O[j][4 * q + 1] * inv_l), narrow2<T>(O[j][4 * q + 2] * inv_l, O[j][4 * q + 3] * inv_l));
      *reinterpret_cast<uint2*>(op + 32 * j + 8 * q + 4 * half) = none ? make_uint2(0u, 0u) : w;
    }
  if (a.lse && half == 0) {
    a.lse[lse_place(a, r, b, head, t)] = none ? -INFINITY : (m_ref + log2f(l)) * kLn2;
  }
}

template <class T, int PT, int DH>
hipError_t launch_one(const PagedAttendArgs& args, hipStream_t s) {
  constexpr int NW = 4;
  PagedAttendArgs a = args;
  a.n_tiles = (int)(((int64_t)a.p.n * a.group + NW * 32 - 1) / (NW * 32));
  const int64_t blocks = (int64_t)a.p.B * a.p.H_kv * a.n_tiles;
  hipLaunchKernelGGL((paged_chunk<T, PT, DH, NW>), dim3((uint32_t)blocks), dim3(NW * 64), 0, s, a);
  return hipGetLastError();
}
template <class T, int PT>
hipError_t launch_d(const PagedAttendArgs& a, hipStream_t s) {
  switch (a.p.d_h) {
    case 64: return launch_one<T, PT, 64>(a, s);
    case 128: return launch_one<T, PT, 128>(a, s);
    case 256: return launch_one<T, PT, 256>(a, s);
    default: return hipErrorInvalidValue;
  }
}
template <class T>
hipError_t launch_t(const PagedAttendArgs& a, int page_type, hipStream_t s) {
  switch (page_type) {
    case kPages16: return launch_d<T, kPages16>(a, s);
    case kPagesI8: return launch_d<T, kPagesI8>(a, s);
    case kPagesE4M3: return launch_d<T, kPagesE4M3>(a, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_paged_chunk(const PagedAttendArgs& a, int dtype, int page_type, hipStream_t s) {
  return dtype == 1 ? launch_t<BF16>(a, page_type, s) : launch_t<F16>(a, page_type, s);
}

}  // namespace sparq
