// What the two kernels have in common whose waves divide the rows: tiles of positions in LDS, and how the work is divided.
#pragma once
#include "paged_core.h"

namespace sparq {

constexpr int kTile = 64;               // positions per tile
// What a row tile costs besides its tiles of positions (queries, first loads, results), in tiles.
constexpr int kStart = 4;
constexpr int kGather = 8;              // results that a workgroup puts together at a time

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
template <int DH> __device__ __forceinline__ int key_turn(int row) { return row & (DH / 8 - 1) & 15; }
template <int DH> __device__ __forceinline__ int value_turn(int row) { return DH == 64 ? ((row & 1) << 2) | ((row >> 1) & 3) : ((row & 3) << 2) | ((row >> 2) & 3); }
template <int DH> __device__ __forceinline__ int key_piece(int row, int piece) { return row * DH + ((piece ^ key_turn<DH>(row)) << 3); }
template <int DH> __device__ __forceinline__ int value_piece(int row, int piece) { return row * DH + ((piece ^ value_turn<DH>(row)) << 3); }

// 16 bytes per lane from memory (base + the lane's offset) into LDS at `to` + 16 lane, without a way through registers: the
// instruction has no result but what tile_barrier waits for.  (The builtin for it makes every transposing read wait for all
// such loads, those into the other buffer too: the prompt of 8192 took 820 us with it.)
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t off, void* to) {
  typedef __attribute__((address_space(3))) void lvoid;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"((uint32_t)(uintptr_t)(lvoid*)to), "v"(off), "s"(base) : "memory");
}

// All of this wave's loads have arrived and its LDS accesses are done; then all waves' have.
__device__ __forceinline__ void tile_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070);                          // vmcnt(0) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ---- the division of the work ----
// ROWS rows per row tile.  The line is counted in tiles of 64 positions: those that a row tile sees (one at least: rows that see
// nothing are written too), behind kStart that stand for its start and end.
template <int NW> struct LineLds { int64_t sum_w[NW]; int begin[4]; };
// A workgroup's part: [begin, end) of the line, whose first step is step `skip` of row tile `tile` of (sequence b, KV head hk); with `plan.tiles` one
// row tile whole.  `share`: steps per workgroup, of which this is number `me`; 0 where a row tile is cut into parts of its own, which the
// workgroups `first` to `last` have.
struct Part { int64_t begin, end, share; int me, b, hk, tile, skip, first, last; };

template <int ROWS, int NW> struct Line {
  const PagedAttendArgs& a;
  const ChunkPlan& plan;

  __device__ __forceinline__ SeqRows rows_of(int b) const {
    const PagedArgs& p = a.p;
    return seq_rows(p.seq_lens[b], p.bound, p.n, p.n_per_seq, p.row_start, p.n_rows, b);
  }
  __device__ __forceinline__ int tiles_of(const SeqRows& r) const {
    const int M = r.n * a.group;
    return M <= a.skip_rows ? 0 : (M + ROWS - 1) / ROWS;
  }
  // positions [from, to) of row tile k, from a multiple of 64 on
  __device__ __forceinline__ int steps_of(const SeqRows& r, int k, int& from, int& to) const {
    const int M = r.n * a.group, m0 = k * ROWS, m1 = m0 + ROWS < M ? m0 + ROWS : M;
    from = seen_by(a, r, divided(m0, a.by_group)).lo & ~(kTile - 1);
    to = seen_by(a, r, divided(m1 - 1, a.by_group)).hi;
    return kStart + (to - from <= kTile ? 1 : (to - from + kTile - 1) / kTile);
  }
  // ... of `size` steps or a rest of them
  __device__ __forceinline__ int parts_of(const SeqRows& r, int k, int size) const {
    int from, to;
    const int steps = steps_of(r, k, from, to);
    return size == 1 ? steps : (int)((uint32_t)(steps + size - 1) / (uint32_t)size);
  }
  __device__ __forceinline__ int64_t parts_of_unit(const SeqRows& r, int size, int lane) const {   // by all lanes of a wave together
    const int n_tiles = tiles_of(r);
    int64_t sum = 0;
    for (int k = lane; k < n_tiles; k += kWave) sum += parts_of(r, k, size);
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) sum += __shfl_xor(sum, o);
    return sum;
  }

  // by all threads; false where there is nothing to do
  __device__ __forceinline__ bool find(LineLds<NW>& lds, const Divider& by_G, Part& part) const {
    const PagedArgs& p = a.p;
    const int thread = threadIdx.x, lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6), G = plan.workgroups;
    part.me = blockIdx.x; part.share = 1; part.begin = 0;
    if (plan.tiles) {
      // Workgroups are dealt round-robin to the 8 XCDs: eight (sequence, KV head) units at a time, the last row tiles, which see most, first.
      const int units = p.B * p.H_kv, eight = blockIdx.x / (8 * plan.tiles), in_eight = blockIdx.x - eight * 8 * plan.tiles;
      const int width = units - eight * 8 < 8 ? units - eight * 8 : 8, up = in_eight / width, unit = eight * 8 + in_eight - up * width;
      part.b = divided(unit, p.by_H_kv);
      part.hk = unit - part.b * p.H_kv;
      part.tile = plan.tiles - 1 - up;
      part.skip = 0;
      const SeqRows r = rows_of(part.b);
      if (r.err && part.tile == 0 && part.hk == 0 && thread == 0) atomicOr(p.err, r.err);
      if (part.tile >= tiles_of(r)) return false;
      int from, to;
      part.end = steps_of(r, part.tile, from, to);
      return true;
    }
    const int per = (p.B + NW - 1) / NW, b_first = wave * per, b_last = b_first + per < p.B ? b_first + per : p.B;
    int64_t mine, before, total;
    auto count = [&](int size) {
      mine = 0;
      for (int b = b_first; b < b_last; ++b) mine += parts_of_unit(rows_of(b), size, lane);
      if (lane == 0) lds.sum_w[wave] = mine;
      __syncthreads();
      before = 0; total = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) { before += w < wave ? lds.sum_w[w] : 0; total += lds.sum_w[w]; }
      before *= p.H_kv; total *= p.H_kv;
      __syncthreads();
    };
    if (blockIdx.x == 0)
      for (int b = b_first; b < b_last; ++b) { const int err = rows_of(b).err; if (err && lane == 0) atomicOr(p.err, err); }
    count(1);
    part.share = total < INT32_MAX - G ? (int64_t)divided((int)total + G - 1, by_G) : (total + G - 1) / G;
    // Where the workgroups can be dealt out to the row tiles, each cut into equal parts of at most 9/8 of a share, they are: those of a KV head then go
    // through the same positions at the same time and find them in their L2.  us, shares of the line / such parts, 16 bits, 8 KV heads of 4 heads of 128
    // channels: 512 rows over 32 768 positions (128 row tiles, 4 parts each) 345 / 321, 1273 / 176 MB fetched; 256 rows 186 / 166, 512 over 20 000 204 / 199; 32 heads of
    // 512 rows over 8192 183 / 185, 4 sequences of 256 rows over 8192 192 / 184.
    int size = 1;
    if (part.share >= 8 && part.share < INT32_MAX / 2) {
      const int64_t keep_mine = mine, keep_before = before, keep_total = total;
      size = (int)part.share + (int)part.share / 8;
      count(size);
      if (total > G) { size = 1; mine = keep_mine; before = keep_before; total = keep_total; }
      else part.share = 0;
    }
    // Consecutive parts share rows of the cache; so that they share an L2 too, each XCD takes an eighth of them.
    const int used = size == 1 ? G : (int)total, eighth = (used + 7) / 8;
    if (G % 8 == 0) {
      if ((int)blockIdx.x / 8 >= eighth) return false;
      part.me = (int)(blockIdx.x % 8) * eighth + (int)blockIdx.x / 8;
    }
    part.begin = size == 1 ? (int64_t)part.me * part.share : part.me;
    part.end = size == 1 && part.begin + part.share < total ? part.begin + part.share : total;
    if (part.begin >= total) return false;
    if (before <= part.begin && part.begin < before + mine * p.H_kv) {   // one wave
      int64_t at = before, c = 1;
      int b = b_first;
      for (; b < b_last; ++b) {
        c = parts_of_unit(rows_of(b), size, lane);
        if (part.begin < at + c * p.H_kv || b == b_last - 1) break;
        at += c * p.H_kv;
      }
      const int64_t off = part.begin - at;
      const int hk = quotient(off, c > 0 ? c : 1);
      int64_t rest = off - hk * c;
      const SeqRows r = rows_of(b);
      const int n_tiles = tiles_of(r);
      for (int k0 = 0; k0 < n_tiles; k0 += kWave) {
        const uint32_t cnt = k0 + lane < n_tiles ? (uint32_t)parts_of(r, k0 + lane, size) : 0u;
        uint32_t upto = cnt;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) { const uint32_t x = __shfl_up(upto, o); if (lane >= o) upto += x; }
        const uint64_t past = __ballot((int64_t)upto > rest);
        if (past) {
          if (lane == __builtin_ctzll(past)) { lds.begin[0] = b; lds.begin[1] = hk; lds.begin[2] = k0 + lane; lds.begin[3] = (int)(rest - (upto - cnt)); }
          break;
        }
        rest -= __shfl(upto, 63);
      }
    }
    __syncthreads();
    part.b = __builtin_amdgcn_readfirstlane(lds.begin[0]); part.hk = __builtin_amdgcn_readfirstlane(lds.begin[1]);
    part.tile = __builtin_amdgcn_readfirstlane(lds.begin[2]); part.skip = __builtin_amdgcn_readfirstlane(lds.begin[3]);
    if (size > 1) {                                            // part `skip` of the row tile
      int from, to;
      const int mine_is = part.skip, steps = steps_of(rows_of(part.b), part.tile, from, to), tiles = steps - kStart;
      const int parts = (int)((uint32_t)(steps + size - 1) / (uint32_t)size), each = (tiles + parts - 1) / parts, needed = (tiles + each - 1) / each;
      if (mine_is >= needed) return false;
      part.first = part.me - mine_is;
      part.last = part.first + needed - 1;
      part.skip = mine_is ? kStart + mine_is * each : 0;
      part.begin = part.skip;
      part.end = kStart + (mine_is + 1) * each < steps ? kStart + (mine_is + 1) * each : steps;
    }
    return true;
  }
};

}  // namespace sparq
