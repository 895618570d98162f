// Attention of few rows per (sequence, KV head) over a paged cache: single tokens, and a handful of them.
//
// Bound by HBM: every key and value is read once for all rows of its KV head (tokens x query heads of the group, up to 16 NT), and
// there is nothing to share between workgroups.  So the waves divide the positions, not the rows, and the work of the whole
// batch is one line of runs of 128 positions, (sequence, KV head, run) in order, cut into equal parts, one per workgroup:
// sequences of different lengths, few long ones and many short ones all load the chip evenly, whatever the table has room for.
// A unit (sequence, KV head) that several workgroups share is put together by the last of them to finish.
//
// A wave takes 32 positions at a time.  Scores S^T[position][row] = K Q^T by 16x16x32 matrix instructions straight from the
// registers that the keys were loaded into; a lane then holds 8 scores of one row.  O^T[channel][row] += V^T P^T: the weights are, as
// they stand, the right operand, with the contraction over the positions in the order (16 a + 4 quarter + j); the values go
// through LDS (each wave its own part, no barriers) for the transposing load.  8-bit codes become fp16 in registers.
//
// us (GB/s of keys and values, of the 7.07 TB/s that plain reads reach): 64 sequences of 8192 positions, 8 KV heads of 4 heads, 128 channels,
// int8 pages 176 (6270); 32 of 1024 to 16 384, 16 heads of 256 channels, bf16 685 (6400).  What is left of it is the line's ends and the clock
// of the first microseconds.  One sequence is bound by latency: the start of the workgroups, a chain of length, page, row and ticket, and the merge;
// 3981 positions of 8 KV heads, 16 bits 12.5, 32 768 positions of e4m3 pages 23.3 (2970).
#include "paged_core.h"

namespace sparq {
namespace {

constexpr int TT = 256, TW = TT / kWave;       // threads and waves per workgroup
constexpr int kPos = 32;                       // positions per wave and turn
constexpr int kRun = kPos * TW;                // ... per workgroup and turn

// Rows of DH elements in LDS in pieces of 8: 16 rows are read at 2 neighbouring pieces at a time, which the row spreads over the banks.
template <int DH> __device__ __forceinline__ int piece_place(int row, int piece) {
  const int turn = DH == 64 ? (row >> 1) & 3 : row & 7;
  return row * DH + ((piece ^ (turn << 1)) << 3);
}

template <class T, int PT, int DH, int NT>
struct TokensGeometry {
  static constexpr int ROWS = 16 * NT;
  static constexpr int KK = DH / 32;                          // products per 16 positions
  static constexpr int EB = PT == kPages16 ? 2 : 1;           // bytes of a stored element
  static constexpr int PER16 = 16 / EB;                       // elements of 16 bytes
  static constexpr int KL = KK * EB / 2 > 0 ? KK * EB / 2 : 1;   // loads of 16 bytes per lane and 16 positions
  static constexpr int STRIDE = DH + 4;                       // floats per row of a partial result: DH numerators, maximum, denominator
  static constexpr size_t lds = (size_t)TW * (ROWS * STRIDE * 4 > kPos * DH * 2 ? ROWS * STRIDE * 4 : kPos * DH * 2);
};

// this lane's part of 32 positions: 16 bytes at a time of keys and values, and the scales of positions 4 quarter + i, + 16
template <int KL, int PT> struct Stage {
  uint4 k[2][KL], v[2][KL];
  float4 sk[2], sv[2];
};

template <class T, int PT, int DH, int NT>
__global__ __launch_bounds__(TT, tokens_per_cu(DH, 16 * NT)) void paged_tokens(const PagedAttendArgs a, const int max_rows, const int G, const Divider by_G, float* partials, int32_t* tickets) {
  using E = Product<T, PT>;
  using Geo = TokensGeometry<T, PT, DH, NT>;
  constexpr int ROWS = Geo::ROWS, KK = Geo::KK, KL = Geo::KL, STRIDE = Geo::STRIDE, NJ = DH / 16;
  __shared__ __align__(16) unsigned char lds[Geo::lds];
  __shared__ int64_t sum_w[TW];
  __shared__ int s_begin[4];
  __shared__ int flag;
  const PagedArgs& p = a.p;
  const int thread = threadIdx.x;
  const bool packed = p.row_start != nullptr;

  // ---- this workgroup's part of the line ----
  // Runs of sequence b: one per KV head and 128 positions that some row sees, one at least (a row that sees nothing is written
  // too); none where the sequence has no rows, or more than this kernel takes.
  auto rows_of = [&](int b) { return seq_rows(p.seq_lens[b], p.bound, p.n, p.n_per_seq, p.row_start, p.n_rows, b); };
  auto range_of = [&](const SeqRows& r, int& from, int& to) {      // positions that some row sees, from a multiple of 16 on
    from = seen_by(a, r, 0).lo & ~15;
    to = seen_by(a, r, r.n - 1).hi;
  };
  auto runs_of = [&](int b) -> int {
    const SeqRows r = rows_of(b);
    if (r.err && blockIdx.x == 0) atomicOr(p.err, r.err);
    if (r.n == 0 || r.n * a.group > max_rows) return 0;
    int from, to;
    range_of(r, from, to);
    return to - from <= kRun ? 1 : (to - from + kRun - 1) / kRun;
  };
  const int lane0 = thread & 63, wave0 = thread >> 6;
  const int per = (p.B + TT - 1) / TT, b_first = thread * per, b_last = b_first + per < p.B ? b_first + per : p.B;
  int64_t mine = 0;
  for (int b = b_first; b < b_last; ++b) mine += runs_of(b);
  int64_t upto = mine;                                             // inclusive prefix sum over the wave
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int64_t x = __shfl_up(upto, o);
    if (lane0 >= o) upto += x;
  }
  if (lane0 == 63) sum_w[wave0] = upto;
  __syncthreads();
  int64_t before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < TW; ++w) { before += w < wave0 ? sum_w[w] : 0; total += sum_w[w]; }
  before += upto - mine;
  total *= p.H_kv;
  const int64_t share = total < INT32_MAX - G ? (int64_t)divided((int)total + G - 1, by_G) : (total + G - 1) / G;
  const int64_t begin = (int64_t)blockIdx.x * share, end = begin + share < total ? begin + share : total;
  if (begin >= end) return;
  if (before * p.H_kv <= begin && begin < (before + mine) * p.H_kv) {        // one thread
    int64_t at = before * p.H_kv;
    int b = b_first;
    for (; b < b_last - 1; ++b) {
      const int64_t c = (int64_t)runs_of(b) * p.H_kv;
      if (begin < at + c) break;
      at += c;
    }
    const int runs = per == 1 ? (int)mine : runs_of(b), c = runs > 0 ? runs : 1;
    const int64_t off = begin - at;
    s_begin[0] = b;
    s_begin[1] = quotient(off, c);                                 // KV head
    s_begin[2] = (int)(off - (int64_t)s_begin[1] * c);             // run
  }
  __syncthreads();
  int b = __builtin_amdgcn_readfirstlane(s_begin[0]), hk = __builtin_amdgcn_readfirstlane(s_begin[1]), run = __builtin_amdgcn_readfirstlane(s_begin[2]);

  for (int64_t at = begin; at < end;) {
    int tid = thread;
    asm volatile("" : "+v"(tid));                                  // (what follows from it is not to be kept in registers from one unit to the next: 75 of them)
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, quarter = lane >> 4;
    const int runs = runs_of(b);
    if (runs == 0) {                                               // (a later sequence has runs: at < end <= total)
      if (++b >= p.B) return;
      continue;
    }
    const SeqRows r = rows_of(b);
    int from, to;
    range_of(r, from, to);
    const int todo = (int)(end - at < runs - run ? end - at : runs - run);
    const int64_t unit_at = at - run;                              // of the unit's first run
    const int M = r.n * a.group;

    const int lo_last = seen_by(a, r, r.n - 1).lo, hi_first = seen_by(a, r, 0).hi;
    uint16_t* Vt = reinterpret_cast<uint16_t*>(lds) + wave * (kPos * DH);

    using St = Stage<KL, PT>;
    // The pages of the wave's next 32 turns, two groups of 16 positions each, one per lane: a turn's loads do not wait for a page's.
    int pages = 0, pages_from = 0;
    auto group_at = [&](int pos) { return pos < to ? pos : from; };   // (behind the last position: any row, its values are not used)
    auto load_pages = [&](int p0) {
      pages_from = p0;
      const int turn = lane / 2 < (to - p0) / kRun + 1 ? lane / 2 : 0;
      pages = page_at(p, b, divided(group_at(p0 + turn * kRun + lane % 2 * 16), p.by_page));
      if (pages < 0) { atomicOr(p.err, kErrBadPage); pages = 0; }
    };
    auto place = [&](int p0, int i) -> int64_t {                   // row in the pool of a group of 16 positions
      const int x = group_at(p0 + 16 * i), index = divided(x, p.by_page);
      return pool_row(p, __builtin_amdgcn_readlane(pages, (p0 - pages_from) / kRun * 2 + i), hk, x - index * p.page_size);
    };
    auto load = [&](St& s, int p0) {
      if (p0 - pages_from >= 32 * kRun) load_pages(p0);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t row = place(p0, i);
        const char* kp = reinterpret_cast<const char*>(p.K) + row * (DH * Geo::EB) + (col * DH * Geo::EB + quarter * 16);
        const char* vp = reinterpret_cast<const char*>(p.V) + row * (DH * Geo::EB) + lane * 16;
#pragma unroll
        for (int e = 0; e < KL; ++e) s.k[i][e] = load16(kp + e * 64);
#pragma unroll
        for (int e = 0; e < KL; ++e) s.v[i][e] = load16(vp + e * 1024);
        if constexpr (PT != kPages16) {
          s.sk[i] = *reinterpret_cast<const float4*>(p.K_scale + row + 4 * quarter);
          s.sv[i] = *reinterpret_cast<const float4*>(p.V_scale + row + 4 * quarter);
        }
      }
    };
    const int p1 = from + (run + todo) * kRun < to ? from + (run + todo) * kRun : to;
    St s;
    int p0 = from + run * kRun + wave * kPos;
    bool more = p0 < p1;
    if (more) {
      load_pages(p0);
      load(s, p0);
    }

    // ---- the lane's rows ----
    uint4 qf[NT][KK];
    float c_row[NT], m_ref[NT], l[NT];
    int lo[NT];
    uint32_t len[NT];
    f32x4 O[NT][NJ];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int m = nt * 16 + col < M ? nt * 16 + col : M - 1, t = divided(m, a.by_group), head = hk * a.group + m - t * a.group;
      const Seen s = seen_by(a, r, t);
      lo[nt] = s.lo;
      len[nt] = s.hi > s.lo ? (uint32_t)(s.hi - s.lo) : 0u;
      // channels of a product: 32 kk + 8 quarter .. + 7; of 8-bit keys, whose lane loads 16 of them, 64 (kk / 2) + 16 quarter + 8 (kk % 2) .. + 7
      const uint16_t* qp = reinterpret_cast<const uint16_t*>(a.q) + row_offset(a.qs, packed, b, r.row0, head, t) + quarter * Geo::PER16;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) qf[nt][kk] = *reinterpret_cast<const uint4*>(qp + (PT == kPages16 ? kk * 32 : kk / 2 * 64 + kk % 2 * 8));
      c_row[nt] = kLog2e / sqrtf((float)DH);
      if constexpr (PT != kPages16 && std::is_same_v<T, BF16>) c_row[nt] *= query_to_half<16>(qf[nt]);
      m_ref[nt] = -INFINITY; l[nt] = 0.0f;
#pragma unroll
      for (int j = 0; j < NJ; ++j) O[nt][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // ---- the positions: the next ones are loaded once this turn's are out of their registers ----
    while (more) {
      more = p0 + kRun < p1;
      // values into LDS
      const bool masked = p0 < lo_last || p0 + kPos > hi_first;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < KL; ++e) {
          constexpr int LPR = DH * Geo::EB / 16;                   // lanes per row
          const int at16 = e * 64 + lane, rr = 16 * i + at16 / LPR, piece = at16 % LPR;
          const uint4& v = s.v[i][e];
          if constexpr (PT == kPages16) {
            *reinterpret_cast<uint4*>(&Vt[piece_place<DH>(rr, piece)]) = v;
          } else {
            const uint2 x0 = codes_to_half<PT>(v.x), x1 = codes_to_half<PT>(v.y), x2 = codes_to_half<PT>(v.z), x3 = codes_to_half<PT>(v.w);
            *reinterpret_cast<uint4*>(&Vt[piece_place<DH>(rr, 2 * piece)]) = make_uint4(x0.x, x0.y, x1.x, x1.y);
            *reinterpret_cast<uint4*>(&Vt[piece_place<DH>(rr, 2 * piece + 1)]) = make_uint4(x2.x, x2.y, x3.x, x3.y);
          }
        }
      // scores
      f32x4 S[NT][2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) S[nt][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          uint4 k;
          if constexpr (PT == kPages16) k = s.k[i][kk];
          else {
            const uint4& w = s.k[i][kk / 2];
            const uint2 x = codes_to_half<PT>(kk % 2 ? w.z : w.x), y = codes_to_half<PT>(kk % 2 ? w.w : w.y);
            k = make_uint4(x.x, x.y, y.x, y.y);
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) S[nt][i] = E::mfma_16x16x32(k, qf[nt][kk], S[nt][i]);
        }
      }
      float s_key[2][4], s_log[2][4], s_inv[2][4];
      if constexpr (PT != kPages16) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float v = value_scale((&s.sv[i].x)[e]);
            s_key[i][e] = (&s.sk[i].x)[e];
            s_log[i][e] = log2_normal(v);
            s_inv[i][e] = __builtin_amdgcn_rcpf(v);                // (1 ulp)
          }
      }
      if (more) load(s, p0 + kRun);                                // in flight during the rest of this turn
      uint4 w16[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const uint32_t at = (uint32_t)(p0 + 4 * quarter - lo[nt]);
        float inv[2][4], mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x;
            if constexpr (PT == kPages16) x = S[nt][i][e] * c_row[nt];
            else { x = fmaf(S[nt][i][e], s_key[i][e] * c_row[nt], s_log[i][e]); inv[i][e] = s_inv[i][e]; }
            S[nt][i][e] = x;
          }
        if (masked) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (at + (16 * i + e) >= len[nt]) { S[nt][i][e] = -INFINITY; inv[i][e] = 0.0f; }   // (0: whatever the scale of a position that is not seen)
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx = fmaxf(mx, S[nt][i][e]);
        float x, y;
        lane_pair<16>(mx, x, y);
        lane_pair<32>(fmaxf(x, y), x, y);
        const float m_new = fmaxf(fmaxf(x, y), m_ref[nt]);
        if (__ballot(m_new > m_ref[nt])) {
          const float w = weight_exp2(m_ref[nt], m_new);
          m_ref[nt] = m_new;
          l[nt] *= w;
#pragma unroll
          for (int j = 0; j < NJ; ++j) O[nt][j] *= w;
        }
        const float m_use = m_ref[nt] == -INFINITY ? 0.0f : m_ref[nt];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            S[nt][i][e] = exp2_weight(S[nt][i][e] - m_use);
            if constexpr (PT == kPages16) l[nt] += S[nt][i][e];
            else l[nt] = fmaf(S[nt][i][e], inv[i][e], l[nt]);
          }
        w16[nt] = make_uint4(narrow2<E>(S[nt][0][0], S[nt][0][1]), narrow2<E>(S[nt][0][2], S[nt][0][3]), narrow2<E>(S[nt][1][0], S[nt][1][1]), narrow2<E>(S[nt][1][2], S[nt][1][3]));
      }
      wave_lds_fence();
      if (masked) {
        // values behind the last position that some row sees: zeros
        for (int e = (to - p0) * (DH / 8) + lane; e < kPos * (DH / 8); e += kWave) *reinterpret_cast<uint4*>(&Vt[e * 8]) = make_uint4(0, 0, 0, 0);
        wave_lds_fence();
        if constexpr (PT == kPages16) {
          // infinities and NaN among values that some rows do not see (a weight of 0 would make NaN of them): added to the
          // rows that see them, zeros in their places
          bool special = false;
          for (int e = lane; e < kPos * (DH / 8); e += kWave) special = special || has_special<T>(*reinterpret_cast<const uint4*>(&Vt[e * 8]));
          if (__ballot(special)) {
#pragma unroll 1
            for (int j = 0; j < kPos; ++j)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                if ((uint32_t)(p0 + j - lo[nt]) >= len[nt]) continue;
#pragma unroll
                for (int jj = 0; jj < NJ; ++jj)
#pragma unroll
                  for (int e = 0; e < 4; ++e) {
                    const int d = 16 * jj + 4 * quarter + e;
                    const float v = T::widen(Vt[piece_place<DH>(j, d / 8) + d % 8]);
                    if (!(fabsf(v) < INFINITY)) O[nt][jj][e] += v;
                  }
              }
            wave_lds_fence();
            for (int e = lane; e < kPos * DH; e += kWave)
              if (!(fabsf(T::widen(Vt[e])) < INFINITY)) Vt[e] = 0;
            wave_lds_fence();
          }
        }
      }
      const int row = 4 * quarter + (lane & 15) / 4;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const int piece = 2 * j + ((lane >> 1) & 1), sub = (lane & 1) * 4;
        const uint2 v0 = lds_read_transposed(&Vt[piece_place<DH>(row, piece) + sub]), v1 = lds_read_transposed(&Vt[piece_place<DH>(row + 16, piece) + sub]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) O[nt][j] = E::mfma_16x16x32(make_uint4(v0.x, v0.y, v1.x, v1.y), w16[nt], O[nt][j]);
      }
      wave_lds_fence();                                            // the next values take these places
      p0 += kRun;
    }

    // ---- the four waves' results together ----
    __syncthreads();                                               // (the parts of LDS are used anew)
    float* part = reinterpret_cast<float*>(lds);                   // [TW][ROWS][STRIDE]
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float x, y;
      lane_pair<16>(l[nt], x, y);
      lane_pair<32>(x + y, x, y);
      float* dst = part + ((size_t)wave * ROWS + nt * 16 + col) * STRIDE;
#pragma unroll
      for (int j = 0; j < NJ; ++j) *reinterpret_cast<f32x4*>(dst + 16 * j + 4 * quarter) = O[nt][j];
      if (quarter == 0) { dst[DH] = m_ref[nt]; dst[DH + 1] = x + y; }
    }
    __syncthreads();
    const int n_slots = M * (DH / 4);                              // 4 channels of a row each
    const int64_t unit_end = unit_at + runs;
    const bool whole = run == 0 && todo == runs;
    const int first_wg = run == 0 ? (int)blockIdx.x : quotient(unit_at, share), last_wg = unit_end <= end ? (int)blockIdx.x : quotient(unit_end - 1, share);
    auto slot_of = [&](int wg) { return partials + ((size_t)wg * 2 + (wg == first_wg ? 1 : 0)) * (ROWS * STRIDE); };
    auto finish = [&](int m, int c, const float4& y, float m_all, float l_all) {
      const int t = divided(m, a.by_group), head = hk * a.group + m - t * a.group;
      const bool none = l_all == 0.0f;                             // nothing seen: zeros (a sum that is NaN stays NaN)
      const float inv = none ? 0.0f : 1.0f / l_all;
      uint16_t* op = reinterpret_cast<uint16_t*>(a.out) + row_offset(a.os, packed, b, r.row0, head, t) + c;
      *reinterpret_cast<uint2*>(op) = none ? make_uint2(0u, 0u) : make_uint2(narrow2<T>(y.x * inv, y.y * inv), narrow2<T>(y.z * inv, y.w * inv));
      if (a.lse && c == 0) a.lse[lse_place(a, r, b, head, t)] = none ? -INFINITY : (m_all + log2f(l_all)) * kLn2;
    };
    for (int slot = tid; slot < n_slots; slot += TT) {
      const int m = slot / (DH / 4), c = slot % (DH / 4) * 4;
      float m_all = -INFINITY, l_all = 0.0f;
      float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < TW; ++w) m_all = fmaxf(m_all, part[((size_t)w * ROWS + m) * STRIDE + DH]);
#pragma unroll
      for (int w = 0; w < TW; ++w) {
        const float* src = part + ((size_t)w * ROWS + m) * STRIDE;
        const float f = weight_exp2(src[DH], m_all);
        const float4 o = *reinterpret_cast<const float4*>(src + c);
        l_all += src[DH + 1] * f;
        y.x += o.x * f; y.y += o.y * f; y.z += o.z * f; y.w += o.w * f;
      }
      if (whole) finish(m, c, y, m_all, l_all);
      else {
        float* dst = slot_of(blockIdx.x);
        store_agent4(dst, (uint32_t)(m * STRIDE + c) * 4, y);
        if (c == 0) store_agent4(dst, (uint32_t)(m * STRIDE + DH) * 4, make_float4(m_all, l_all, 0.0f, 0.0f));
      }
    }
    if (!whole && last_to_arrive(tickets + first_wg, last_wg - first_wg + 1, &flag)) {
      // The parts of a unit in an order of their own, so that the sums do not depend on who comes last: threads that are left over by
      // the slots share the parts of a slot, eight of them in flight each.
      const int grps = n_slots < TT ? TT / n_slots : 1;
      auto add = [](float4& y, float& m_all, float& l_all, const float4& o, float m_o, float l_o) {
        const float m_new = fmaxf(m_all, m_o);
        const float f = weight_exp2(m_all, m_new), g = weight_exp2(m_o, m_new);
        l_all = l_all * f + l_o * g;
        y.x = y.x * f + o.x * g; y.y = y.y * f + o.y * g; y.z = y.z * f + o.z * g; y.w = y.w * f + o.w * g;
        m_all = m_new;
      };
      const int grp = grps > 1 ? tid / n_slots : 0;
      float4* sum = reinterpret_cast<float4*>(lds);                // [TT] numerators, then [TT] (maximum, denominator)
      for (int slot = grps > 1 ? tid - grp * n_slots : tid; slot < n_slots && grp < grps; slot += TT) {
        const int m = slot / (DH / 4), c = slot % (DH / 4) * 4;
        float m_all = -INFINITY, l_all = 0.0f;
        float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int wg = first_wg + grp; wg <= last_wg; wg += 8 * grps) {
          float4 o[8], st[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint32_t at_wg = (uint32_t)((wg + i * grps <= last_wg ? wg + i * grps : wg) - first_wg), off = (at_wg * 2 - (at_wg ? 1 : 0)) * (ROWS * STRIDE * 4);
            o[i] = load_agent4(slot_of(first_wg), off + (uint32_t)(m * STRIDE + c) * 4);
            st[i] = load_agent4(slot_of(first_wg), off + (uint32_t)(m * STRIDE + DH) * 4);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (wg + i * grps <= last_wg) add(y, m_all, l_all, o[i], st[i].x, st[i].y);
        }
        if (grps == 1) finish(m, c, y, m_all, l_all);
        else { sum[tid] = y; sum[TT + tid] = make_float4(m_all, l_all, 0.0f, 0.0f); }
      }
      if (grps > 1) {
        __syncthreads();
        if (tid < n_slots) {
          float4 y = sum[tid], st = sum[TT + tid];
          for (int k = 1; k < grps; ++k) { const float4 s2 = sum[TT + k * n_slots + tid]; add(y, st.x, st.y, sum[k * n_slots + tid], s2.x, s2.y); }
          finish(tid / (DH / 4), tid % (DH / 4) * 4, y, st.x, st.y);
        }
      }
    }
    at += todo;
    run = 0;
    if (unit_end <= end && ++hk == p.H_kv) { hk = 0; ++b; }
    __syncthreads();                                               // (LDS is used anew)
  }
}

template <class T, int PT, int DH, int NT>
hipError_t launch_one(const PagedAttendArgs& a, const TokensPlan& t, hipStream_t s) {
  hipLaunchKernelGGL((paged_tokens<T, PT, DH, NT>), dim3(t.workgroups), dim3(TT), 0, s, a, t.max_rows, t.workgroups, make_divider(t.workgroups), t.partials, t.tickets);
  return hipGetLastError();
}
template <class T, int PT, int DH>
hipError_t launch_nt(const PagedAttendArgs& a, const TokensPlan& t, hipStream_t s) {
  if (t.max_rows <= 16) return launch_one<T, PT, DH, 1>(a, t, s);
  if constexpr (DH <= 128) { if (t.max_rows <= 32) return launch_one<T, PT, DH, 2>(a, t, s); }
  return hipErrorInvalidValue;
}
template <class T, int PT>
hipError_t launch_d(const PagedAttendArgs& a, const TokensPlan& t, hipStream_t s) {
  switch (a.p.d_h) {
    case 64: return launch_nt<T, PT, 64>(a, t, s);
    case 128: return launch_nt<T, PT, 128>(a, t, s);
    case 256: return launch_nt<T, PT, 256>(a, t, s);
    default: return hipErrorInvalidValue;
  }
}
template <class T>
hipError_t launch_t(const PagedAttendArgs& a, const TokensPlan& t, int page_type, hipStream_t s) {
  switch (page_type) {
    case kPages16: return launch_d<T, kPages16>(a, t, s);
    case kPagesI8: return launch_d<T, kPagesI8>(a, t, s);
    case kPagesE4M3: return launch_d<T, kPagesE4M3>(a, t, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_paged_tokens(const PagedAttendArgs& a, const TokensPlan& t, int dtype, int page_type, hipStream_t s) {
  return dtype == 1 ? launch_t<BF16>(a, t, page_type, s) : launch_t<F16>(a, t, page_type, s);
}

}  // namespace sparq
