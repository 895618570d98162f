// Attention of many rows per (sequence, KV head) over a paged cache: chunks of new tokens, whole prompts.
//
// A workgroup's row tile is 32 rows per wave of one (sequence, KV head): row m stands for token m / g and query head m % g of the
// group, so that the heads of a group share what is read of the cache.  It walks the positions that its rows see in tiles
// of 64 through LDS, one pass, with the running maximum and sum of the softmax.
//   scores   S^T[position][row] = K Q^T by 32x32x16 matrix instructions: a lane then holds 32 scores of ONE row, so that
//            maximum and sum are taken inside the lane (and once across the two halves of the wave)
//   weights  P^T[position][row]: the lane's weights are, as they stand, the right operand of the next product if its
//            contraction runs over the positions in the order (8 a + 4 h + j), a = 0, 1, j = 0 .. 3 of lane half h
//   output   O^T[channel][row] += V^T P^T; V^T comes out of LDS by the transposing load, in the same order of positions.
// 8-bit pages: every code is a 16-bit float, so the products are those of 16-bit pages; a key's scale multiplies its scores.
// A value's scale goes into the exponent: w_j = 2^(x_j + log2 s_j - m) is what multiplies the codes, and w_j / s_j what
// is summed.  Neither needs a rounding that 16-bit pages do not have.
//
// Two ways to divide the work.  Where the host knows that there are row tiles enough, a workgroup serves one of them; the
// dispatcher levels their sizes out, and the workgroups of a KV head, which read the same rows, run next to each other on one XCD.
// Otherwise the work of the whole batch is one line of (sequence, KV head, row tile, tile of 64 positions) in order, cut into equal
// parts, one per workgroup: chunks of different lengths and few rows over a long cache load the chip evenly as well; where the lengths allow it, the
// cuts are those of row tiles into parts of their own.  A row tile that several workgroups share is put together by the last of them to finish.
// us, row tiles / the line, 16 bits (row tiles of all KV heads): 128 channels, 32 heads of 512 rows behind 8192 positions, 256 row tiles 216 / 194,
// 384 278 / 311, 512 318 / 321, 640 474 / 515, 768 514 / 592, 1024 642 / 732, 1536 914 / 1117; prompts of 1024, 2048, 4096 and 8192, 256 35.5 / 40,
// 512 75.6 / 71, 1024 212 / 215, 2048 622 / 680; 8 KV heads of 4 heads, prompts of 4096, 1024 162 / 180.  64 channels behind 8192 positions, 256 134 / 108,
// 384 178 / 151, 512 191 / 187, 640 227 / 223, 1024 299 / 298; prompts, 512 51 / 44, 640 62 / 61, 1024 126 / 125, 2048 400 / 415; 8 KV heads of 4
// heads 1024 110 / 128; 1024 of int8 pages 420 / 371 behind 8192 positions, 156 / 171 with the 8 KV heads.
//
// What bounds it: a prompt of 8192 (32 heads of 128 channels, f16) takes 585 us, 0.94 PFLOP/s, of which a large library product of the same
// numbers reaches 1.31.  The matrix instructions fill 54 % of the SIMDs' cycles: two waves share a SIMD, and while the tile's reads, exponents and roundings
// of one overlap with the products of the other, their turns do not always meet; LDS has no bank conflicts.  The clock is 1.8 GHz of 2.4 under this load
// (zeros instead of numbers run faster), so that whatever fills the SIMDs better gains less than its share.  512 rows over 32 768 positions (8 KV heads
// of 4 heads, bf16): 275 us, 0.99 PFLOP/s.
#include "paged_tiles.h"

namespace sparq {
namespace {

constexpr int kWaves = chunk_rows / 32; // waves of a workgroup

template <class T, int PT, int DH>
__global__ __launch_bounds__(kWaves * 64, chunk_per_cu(DH)) void paged_chunk(const PagedAttendArgs a, const ChunkPlan plan, const Divider by_G) {
  using E = Product<T, PT>;
  constexpr int NW = kWaves, NTH = NW * 64, ROWS = NW * 32, PIECES = DH / 8, ND = DH / 32;
  constexpr int LOADS = 16 * PIECES / 64;                      // 16-bit pages: loads of 1 KB per wave, keys and values each
  constexpr int CL = PT == kPages16 ? 1 : DH / 64;             // 8-bit pages: loads of 16 codes per lane
  static_assert(NW * 16 == kTile, "a wave loads 16 positions of a tile");
  // One object: of several, the compiler lets reads of one wait for loads into another.
  struct Lds {
    uint16_t Kt[2][kTile * DH], Vt[2][kTile * DH];
    float s_k[2][kTile], s_log[2][kTile], s_inv[2][kTile];     // 8-bit pages: scale of the key, log2 and inverse of the value's
    LineLds<NW> line;
    int found[NW], flag;
  };
  __shared__ __align__(16) Lds lds;
  const PagedArgs& p = a.p;
  const int thread = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
  const bool packed = p.row_start != nullptr;
  const int G = plan.workgroups;
  float* const partials = plan.partials;

  const Line<ROWS, NW> line{a, plan};
  Part part;
  if (!line.find(lds.line, by_G, part)) return;
  const int me = part.me;
  const int64_t share = part.share, end = part.end;
  int b = part.b, hk = part.hk, tile = part.tile, skip = part.skip;

  for (int64_t at = part.begin; at < end;) {
    int tid = thread;
    asm volatile("" : "+v"(tid));                              // (what follows from it is not to be kept in registers from one row tile to the next)
    const int lane = tid & 63, col = lane & 31, half = lane >> 5;
    const SeqRows r = line.rows_of(b);
    const int n_tiles = line.tiles_of(r);
    if (tile >= n_tiles) {                                     // the next KV head or sequence (one with rows follows: at < end <= total)
      tile = 0;
      if (n_tiles == 0 || ++hk == p.H_kv) { hk = 0; if (++b >= p.B) return; }
      continue;
    }
    int from, to;
    const int steps = line.steps_of(r, tile, from, to);
    const int todo = (int)(end - at < steps - skip ? end - at : steps - skip);
    const int64_t tile_at = at - skip;
    const int k0 = skip > kStart ? skip - kStart : 0, k1 = skip + todo - kStart;   // its tiles of positions here
    if (k1 <= k0) {                                            // (the start alone is no part of a row tile)
      at += todo; skip = 0; ++tile;
      continue;
    }

    // ---- the lane's row ----
    const int M = r.n * a.group, m0 = tile * ROWS, m_w = m0 + wave * 32, m_last = M - 1;
    const bool live = m_w < M;                                 // a wave without rows only helps to load
    const int m = m_w + col < M ? m_w + col : m_last;
    const int t = divided(m, a.by_group), head = hk * a.group + m - t * a.group;
    const auto row_sees = [&](int x) { return seen_by(a, r, divided(x < M ? x : m_last, a.by_group)); };
    const Seen mine_sees = seen_by(a, r, t), wg_first = row_sees(m0), wg_last = row_sees(m0 + ROWS - 1), w_first = row_sees(m_w), w_last = row_sees(m_w + 31);
    const int lo = mine_sees.lo;
    const uint32_t len = mine_sees.hi > lo ? (uint32_t)(mine_sees.hi - lo) : 0u;

    // its part of the row of Q: channels 16 s + 8 half .. + 7
    uint4 qf[DH / 16];
    const uint16_t* qp = reinterpret_cast<const uint16_t*>(a.q) + row_offset(a.qs, packed, b, r.row0, head, t) + half * 8;
#pragma unroll
    for (int s = 0; s < DH / 16; ++s) qf[s] = *reinterpret_cast<const uint4*>(qp + s * 16);
    const float c = kLog2e / sqrtf((float)DH);                 // scores to exponents of 2
    float lift = 1.0f;
    if constexpr (PT != kPages16 && std::is_same_v<T, BF16>) lift = query_to_half<32>(qf);
    const bool lifted = __ballot(lift != 1.0f) != 0;           // some row of the wave

    f32x16 O[ND];
#pragma unroll
    for (int j = 0; j < ND; ++j)
#pragma unroll
      for (int i = 0; i < 16; ++i) O[j][i] = 0.0f;
    float m_ref = -INFINITY, l = 0.0f;

    // ---- loads: a wave's part of a tile is 16 positions, which share a page ----
    const int p_begin = from + k0 * kTile, p_end = from + k1 * kTile < to ? from + k1 * kTile : to;
    // The pages of the next 64 tiles' parts, one per lane: a tile's loads do not wait for a page's.
    int pages = 0, pages_from = 0;
    auto part_at = [&](int p0) { const int x = p0 + wave * 16; return x < to ? x : from; };   // (behind the last position: any row, its values are not used)
    auto load_pages = [&](int p0) {
      pages_from = p0;
      pages = page_at(p, b, divided(part_at(lane < (to - p0) / kTile + 1 ? p0 + lane * kTile : p0), p.by_page));
      if (pages < 0) { atomicOr(p.err, kErrBadPage); pages = 0; }
    };
    auto place = [&](int p0) -> int64_t {
      if (p0 - pages_from >= kWave * kTile) load_pages(p0);
      const int x = part_at(p0), index = divided(x, p.by_page);
      return pool_row(p, __builtin_amdgcn_readlane(pages, (p0 - pages_from) / kTile), hk, x - index * p.page_size);
    };
    uint4 ck[CL], cv[CL];                                      // 8-bit pages: the next tile's codes and scales
    float csk = 0.0f, csv = 0.0f;
    auto issue = [&](int64_t row, int buf) {
      if constexpr (PT == kPages16) {
        const char* kp = reinterpret_cast<const char*>(p.K) + row * (DH * 2);
        const char* vp = reinterpret_cast<const char*>(p.V) + row * (DH * 2);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          const int first = i * 64, e = first + lane, rr = wave * 16 + e / PIECES, slot = e % PIECES, at8 = (wave * 16 * PIECES + first) * 8;
          load_to_lds(kp, (uint32_t)((e / PIECES) * (DH * 2) + (slot ^ key_turn<DH>(rr)) * 16), &lds.Kt[buf][at8]);
          load_to_lds(vp, (uint32_t)((e / PIECES) * (DH * 2) + (slot ^ value_turn<DH>(rr)) * 16), &lds.Vt[buf][at8]);
        }
      } else {
        const uint8_t* kp = reinterpret_cast<const uint8_t*>(p.K) + row * DH;
        const uint8_t* vp = reinterpret_cast<const uint8_t*>(p.V) + row * DH;
#pragma unroll
        for (int i = 0; i < CL; ++i) {
          const int e = i * 64 + lane;                         // 16 codes each
          ck[i] = *reinterpret_cast<const uint4*>(kp + e * 16);
          cv[i] = *reinterpret_cast<const uint4*>(vp + e * 16);
        }
        csk = p.K_scale[row + (lane & 15)];
        csv = p.V_scale[row + (lane & 15)];
      }
    };
    auto settle = [&](int p0, int buf) {                       // 8-bit pages: codes that have arrived go to LDS as fp16
      if constexpr (PT != kPages16) {
        auto put = [&](uint16_t* dst0, uint16_t* dst1, const uint4& w, bool on) {
          const uint2 x0 = codes_to_half<PT>(on ? w.x : 0u), x1 = codes_to_half<PT>(on ? w.y : 0u), x2 = codes_to_half<PT>(on ? w.z : 0u), x3 = codes_to_half<PT>(on ? w.w : 0u);
          *reinterpret_cast<uint4*>(dst0) = make_uint4(x0.x, x0.y, x1.x, x1.y);
          *reinterpret_cast<uint4*>(dst1) = make_uint4(x2.x, x2.y, x3.x, x3.y);
        };
#pragma unroll
        for (int i = 0; i < CL; ++i) {
          const int e = i * 64 + lane, rr = wave * 16 + e / (DH / 16), piece = e % (DH / 16) * 2;
          put(&lds.Kt[buf][key_piece<DH>(rr, piece)], &lds.Kt[buf][key_piece<DH>(rr, piece + 1)], ck[i], true);
          put(&lds.Vt[buf][value_piece<DH>(rr, piece)], &lds.Vt[buf][value_piece<DH>(rr, piece + 1)], cv[i], p0 + rr < to);
        }
        if (lane < 16) {
          const float v = value_scale(csv);
          lds.s_k[buf][wave * 16 + lane] = csk * c;
          lds.s_log[buf][wave * 16 + lane] = log2_normal(v);
          // (a scale that is no number makes NaN of what sees it by its logarithm; its inverse must leave the 0 of what does not)
          lds.s_inv[buf][wave * 16 + lane] = v < INFINITY ? 1.0f / v : 0.0f;
        }
      }
    };

    if (p_begin < p_end) {
      load_pages(p_begin);
      issue(place(p_begin), 0);
      settle(p_begin, 0);
    }
    for (int p0 = p_begin, buf = 0; p0 < p_end; p0 += kTile, buf ^= 1) {
      tile_barrier();                                          // this tile is there; nobody reads the other buffer
      const bool more = p0 + kTile < p_end;
      if (more) issue(place(p0 + kTile), buf ^ 1);
      uint16_t* const kt = lds.Kt[buf];
      uint16_t* const vt = lds.Vt[buf];
      if constexpr (PT == kPages16) {
        if (p0 + kTile > to) {                                 // values behind the last position: zeros
          for (int e = tid; e < (p0 + kTile - to) * PIECES; e += NTH) *reinterpret_cast<uint4*>(&vt[(to - p0) * DH + e * 8]) = make_uint4(0, 0, 0, 0);
          __syncthreads();
        }
      }

      // ---- scores, exponents, weights ----
      // (a row's exponent of 2 at position j is x_j = c q . K_j, with 8-bit pages plus log2 s_j)
      const bool active = live && p0 < w_last.hi && p0 + kTile > w_first.lo;
      f32x16 S[2];
      if (active) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) S[i][e] = 0.0f;
        // (the next four reads are on their way before these four products begin)
        uint4 kf[2][4];
        auto fetch = [&](int s) {
#pragma unroll
          for (int e = 0; e < 4; ++e) kf[s / 2 % 2][e] = *reinterpret_cast<const uint4*>(&kt[key_piece<DH>(e % 2 * 32 + col, 2 * (s + e / 2) + half)]);
        };
        fetch(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int s = 0; s < DH / 16; s += 2) {
          if (s + 2 < DH / 16) fetch(s + 2);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int e = 0; e < 4; ++e) S[e % 2] = mfma_32x32x16<E>(kf[s / 2 % 2][e], qf[s + e / 2], S[e % 2]);
          __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        if constexpr (PT != kPages16) {
          if (std::is_same_v<T, BF16> && lifted) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int e = 0; e < 16; ++e) S[i][e] *= lift;
          }
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int j = 32 * i + 8 * (e / 4) + e % 4 + 4 * half;
              S[i][e] = fmaf(S[i][e], lds.s_k[buf][j], lds.s_log[buf][j]);
            }
        }
        const bool masked = p0 < w_last.lo || p0 + kTile > w_first.hi;
        const uint32_t at0 = (uint32_t)(p0 + 4 * half - lo);
        if (masked) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (at0 + (32 * i + 8 * (e / 4) + e % 4) >= len) S[i][e] = -INFINITY;
        }
        const float c_max = PT == kPages16 ? c : 1.0f;         // (8-bit pages: in the exponents already)
        float mx = fmaxf(S[0][0], S[1][0]);
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(fmaxf(mx, S[0][e]), S[1][e]);
        float m_a, m_b;
        lane_pair<32>(mx, m_a, m_b);
        const float m_new = fmaxf(m_a, m_b) * c_max;
        // the maximum is followed only when it rises by more than 8: weights are at most 2^8 then, and most tiles rescale nothing
        if (__ballot(m_new > m_ref + 8.0f)) {
          const float m_to = fmaxf(m_new, m_ref);
          const float w = weight_exp2(m_ref, m_to);
          m_ref = m_to;
          l *= w;
#pragma unroll
          for (int j = 0; j < ND; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) O[j][e] *= w;
        }
        const float m_use = m_ref == -INFINITY ? 0.0f : m_ref; // (nothing seen yet: every weight is 2^-inf)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) S[i][e] = exp2_weight(PT == kPages16 ? fmaf(S[i][e], c, -m_use) : S[i][e] - m_use);
        if constexpr (PT == kPages16) {
          float l0 = 0.0f, l1 = 0.0f;
#pragma unroll
          for (int e = 0; e < 16; ++e) { l0 += S[0][e]; l1 += S[1][e]; }
          l += l0 + l1;
        } else {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) l = fmaf(S[i][e], lds.s_inv[buf][32 * i + 8 * (e / 4) + e % 4 + 4 * half], l);
        }
      }

      // ---- infinities and NaN among the values of positions that some rows of the tile do not see: a weight of 0 would
      // still make NaN of them.  They are added to the rows that see them, and zeros take their places. ----
      if constexpr (PT == kPages16) {
        if (p0 < wg_last.lo || p0 + kTile > wg_first.hi) {
          bool found = false;
          for (int e = tid; e < kTile * PIECES; e += NTH) found = found || has_special<T>(*reinterpret_cast<const uint4*>(&vt[e * 8]));
          if (lane == 0) lds.found[wave] = 0;
          if (found) lds.found[wave] = 1;                      // (the same word by the lanes that found some, behind the 0 of lane 0)
          __syncthreads();
          int any = 0;
#pragma unroll
          for (int w = 0; w < NW; ++w) any |= lds.found[w];
          if (__builtin_amdgcn_readfirstlane(any)) {
            if (active)
#pragma unroll 1
              for (int j = 0; j < kTile; ++j) {
                if ((uint32_t)(p0 + j - lo) >= len) continue;
#pragma unroll
                for (int jj = 0; jj < ND; ++jj)
#pragma unroll
                  for (int e = 0; e < 16; ++e) {
                    const int d = 32 * jj + 8 * (e / 4) + 4 * half + e % 4;
                    const float v = T::widen(vt[value_piece<DH>(j, d / 8) + d % 8]);
                    if (!(fabsf(v) < INFINITY)) O[jj][e] += v;
                  }
              }
            __syncthreads();
            for (int e = tid; e < kTile * DH; e += NTH)
              if (!(fabsf(T::widen(vt[e])) < INFINITY)) vt[e] = 0;
            __syncthreads();
          }
        }
      }

      // ---- output ----
      if (active) {
        // the values of 16 positions and of the next 16 (8-bit pages: the next tile's codes are in the registers for those)
        constexpr int AHEAD = PT == kPages16 ? 1 : 0;
        uint4 vf[1 + AHEAD][ND];
        auto fetch = [&](int sl) {
          const int row = sl * 16 + 4 * half + (lane & 15) / 4;
#pragma unroll
          for (int j = 0; j < ND; ++j) {
            const int piece = 4 * j + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1), sub = (lane & 1) * 4;
            const uint2 v0 = lds_read_transposed(&vt[value_piece<DH>(row, piece) + sub]), v1 = lds_read_transposed(&vt[value_piece<DH>(row + 8, piece) + sub]);
            vf[sl % (1 + AHEAD)][j] = make_uint4(v0.x, v0.y, v1.x, v1.y);
          }
        };
        if (AHEAD) fetch(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int sl = 0; sl < 4; ++sl) {
          if (sl + AHEAD < 4) fetch(sl + AHEAD);
          const int e0 = sl % 2 * 8;
          const f32x16& w = S[sl / 2];
          const uint4 pw = make_uint4(narrow2<E>(w[e0], w[e0 + 1]), narrow2<E>(w[e0 + 2], w[e0 + 3]), narrow2<E>(w[e0 + 4], w[e0 + 5]), narrow2<E>(w[e0 + 6], w[e0 + 7]));
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int j = 0; j < ND; ++j) O[j] = mfma_32x32x16<E>(vf[sl % (1 + AHEAD)][j], pw, O[j]);
          __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
      }
      if (more) settle(p0 + kTile, buf ^ 1);
    }

    // ---- a row tile that several workgroups share: partial results in the order of registers ----
    const int64_t tile_end = tile_at + steps;
    bool write = true;
    if (k0 != 0 || k1 != steps - kStart) {
      const int first_wg = share == 0 ? part.first : (k0 == 0 ? me : quotient(tile_at + kStart, share)), last_wg = share == 0 ? part.last : (tile_end <= end ? me : quotient(tile_end - 1, share));
      constexpr int SLOT = NTH * (DH / 2 + 4);                 // floats: a lane's DH / 2 numerators, its maximum and its part of the denominator
      auto slot_of = [&](int wg) { return partials + ((size_t)wg * 2 + (wg == first_wg ? 1 : 0)) * SLOT; };
      auto store = [&](float* dst) {
#pragma unroll
        for (int j = 0; j < ND; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) store_agent4(dst, (uint32_t)((j * 4 + q) * NTH + tid) * 16, make_float4(O[j][4 * q], O[j][4 * q + 1], O[j][4 * q + 2], O[j][4 * q + 3]));
        store_agent4(dst, (uint32_t)(ND * 4 * NTH + tid) * 16, make_float4(m_ref, l, 0.0f, 0.0f));
      };
      // the results of every `step`-th workgroup from wg on, in the order of the line, whoever is last
      auto gather = [&](int wg, int step, int to_wg) {
        m_ref = -INFINITY; l = 0.0f;
#pragma unroll
        for (int j = 0; j < ND; ++j)
#pragma unroll
          for (int i = 0; i < 16; ++i) O[j][i] = 0.0f;
        constexpr int AT_ONCE = DH <= 128 ? 2 : 1;             // results in flight
#pragma unroll 1
        for (; wg <= to_wg; wg += AT_ONCE * step) {
          float4 st[AT_ONCE], o[AT_ONCE][ND * 4 / (3 - AT_ONCE)];
          auto fetch = [&](int i, int q0) {
            const float* src = slot_of(wg + i * step <= to_wg ? wg + i * step : wg);
            if (q0 == 0) st[i] = load_agent4(src, (uint32_t)(ND * 4 * NTH + tid) * 16);
#pragma unroll
            for (int q = 0; q < ND * 4 / (3 - AT_ONCE); ++q) o[i][q] = load_agent4(src, (uint32_t)((q0 + q) * NTH + tid) * 16);
          };
#pragma unroll
          for (int i = 0; i < AT_ONCE; ++i) fetch(i, 0);
#pragma unroll
          for (int i = 0; i < AT_ONCE; ++i) {
            if (wg + i * step > to_wg) break;
            const float m_to = fmaxf(m_ref, st[i].x), f = weight_exp2(m_ref, m_to), g = weight_exp2(st[i].x, m_to);
            m_ref = m_to;
            l = l * f + st[i].y * g;
#pragma unroll
            for (int q = 0; q < ND * 4; ++q) {
              if (q > 0 && q % (ND * 4 / (3 - AT_ONCE)) == 0) fetch(i, q);
              f32x16& x = O[q / 4];
              const float4& y = o[i][q % (ND * 4 / (3 - AT_ONCE))];
              const int e = q % 4 * 4;
              x[e] = x[e] * f + y.x * g; x[e + 1] = x[e + 1] * f + y.y * g; x[e + 2] = x[e + 2] * f + y.z * g; x[e + 3] = x[e + 3] * f + y.w * g;
            }
          }
        }
      };
      // The last of eight neighbours puts theirs together, the last of those that did so puts these together: one workgroup takes 2 us for a result
      // (128 rows over 32 768 positions, 64 workgroups to each row tile: 133 us by one of them).
      // (A counter per group at its first workgroup: a group of one, which another row tile's may share its workgroup with, needs none.)
      const int group0 = first_wg + (me - first_wg) / kGather * kGather, group1 = group0 + kGather - 1 < last_wg ? group0 + kGather - 1 : last_wg;
      store(slot_of(me));
      write = group0 == group1 || last_to_arrive(plan.tickets + group0, group1 - group0 + 1, &lds.flag);
      if (write && group0 != group1) gather(group0, 1, group1);
      if (write && last_wg - first_wg >= kGather) {
        if (group0 != group1) store(slot_of(group0));
        write = last_to_arrive(plan.tickets + G + first_wg, (last_wg - first_wg) / kGather + 1, &lds.flag);
        if (write) gather(first_wg, kGather, last_wg);
      }
    }

    // ---- a row's two halves have summed half of its weights each ----
    float l_a, l_b;
    lane_pair<32>(l, l_a, l_b);
    l = l_a + l_b;
    if (write && live && m_w + col < M) {
      const bool none = l == 0.0f;                             // nothing seen: zeros (a sum that is NaN stays NaN)
      const float inv_l = none ? 0.0f : 1.0f / l;
      uint16_t* op = reinterpret_cast<uint16_t*>(a.out) + row_offset(a.os, packed, b, r.row0, head, t);
#pragma unroll
      for (int j = 0; j < ND; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint2 w = make_uint2(narrow2<T>(O[j][4 * q] * inv_l, O[j][4 * q + 1] * inv_l), narrow2<T>(O[j][4 * q + 2] * inv_l, O[j][4 * q + 3] * inv_l));
          *reinterpret_cast<uint2*>(op + 32 * j + 8 * q + 4 * half) = none ? make_uint2(0u, 0u) : w;
        }
      if (a.lse && half == 0) a.lse[lse_place(a, r, b, head, t)] = none ? -INFINITY : (m_ref + log2f(l)) * kLn2;
    }
    at += todo;
    skip = 0;
    ++tile;
    __syncthreads();                                           // (LDS is used anew)
  }
}

template <class T, int PT, int DH>
hipError_t launch_one(const PagedAttendArgs& a, const ChunkPlan& c, hipStream_t s) {
  hipLaunchKernelGGL((paged_chunk<T, PT, DH>), dim3(c.workgroups), dim3(kWaves * 64), 0, s, a, c, make_divider(c.workgroups));
  return hipGetLastError();
}
template <class T, int PT>
hipError_t launch_d(const PagedAttendArgs& a, const ChunkPlan& c, hipStream_t s) {
  switch (a.p.d_h) {
    case 64: return launch_one<T, PT, 64>(a, c, s);
    case 128: return launch_one<T, PT, 128>(a, c, s);
    case 256: return launch_one<T, PT, 256>(a, c, s);
    default: return hipErrorInvalidValue;
  }
}
template <class T>
hipError_t launch_t(const PagedAttendArgs& a, const ChunkPlan& c, int page_type, hipStream_t s) {
  switch (page_type) {
    case kPages16: return launch_d<T, kPages16>(a, c, s);
    case kPagesI8: return launch_d<T, kPagesI8>(a, c, s);
    case kPagesE4M3: return launch_d<T, kPagesE4M3>(a, c, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_paged_chunk(const PagedAttendArgs& a, const ChunkPlan& c, int dtype, int page_type, hipStream_t s) {
  return dtype == 1 ? launch_t<BF16>(a, c, page_type, s) : launch_t<F16>(a, c, page_type, s);
}

}  // namespace sparq
