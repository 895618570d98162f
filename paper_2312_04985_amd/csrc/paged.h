// The paged cache: argument blocks, the arithmetic of rows and pages (also compiled for the host), launcher prototypes.
#pragma once
#include "params.h"

namespace sparq {

enum PageType { kPages16 = 0, kPagesI8 = 1, kPagesE4M3 = 2 };

// Largest code of an 8-bit page type; the largest magnitude of a row lies on it.
constexpr float kMaxI8 = 127.0f, kMaxE4M3 = 448.0f;
// What a row's largest magnitude is taken as, at least and at most: with scales from 2^-69 to 2^94 the exponents of the
// attention's sums stay in fp32's range whatever mixture of rows a query sees.
constexpr float kLeastMagnitude = 0x1p-60f, kMostMagnitude = 0x1p100f;

struct RowStrides { int64_t seq, head, row; };          // elements

// The rows of a call (see sparq_rows) and the cache that they stand in.
struct PagedArgs {
  void* K; void* V; float* K_scale; float* V_scale;
  const int32_t* page_table; const int32_t* seq_lens;
  const int32_t* n_per_seq; const int32_t* row_start;
  int32_t* err;
  int32_t B, H, H_kv, d_h, page_size, n_pages, max_pages, bound;   // bound: no length may pass it
  int32_t n, n_rows;
  Divider by_page, by_H_kv, by_n;
};

struct PagedRowsArgs {                                  // append and read
  PagedArgs p;
  void* k; void* v;                                     // k_new, v_new; K_out, V_out
  const int32_t* first;                                 // read: position of every sequence's first row, or null
  RowStrides s;
};

struct PagedAttendArgs {
  PagedArgs p;
  const void* q; void* out; float* lse;
  RowStrides qs, os;
  int32_t window, all;                                  // all: not causal
  int32_t group;                                        // query heads per KV head
  int32_t skip_rows;                                    // sequences of up to this many rows (times group) are another launch's
  Divider by_group;
};

// Rows of one sequence in a call: its length (the new rows included), how many rows, the first one's number along the row
// stride, and what is wrong with what the caller's arrays say (SPARQ_ERR_* bits).
struct SeqRows { int S, n, row0, err; };

constexpr int kErrBadSeqLen = 8, kErrBadRows = 32, kErrBadPage = 64;

// A length outside [0, bound] counts as 0; a row count outside [0, n], or rows outside the packed buffers, as none.
__host__ __device__ inline SeqRows seq_rows(int len, int bound, int n_max, const int32_t* n_per_seq, const int32_t* row_start, int n_rows, int b) {
  SeqRows r{len, n_max, 0, 0};
  if (len < 0 || len > bound) { r.S = 0; r.err |= kErrBadSeqLen; }
  if (row_start) {
    const int r0 = row_start[b], r1 = row_start[b + 1];
    r.row0 = r0;
    r.n = r1 - r0;
    if (r0 < 0 || r1 < r0 || r1 > n_rows || r.n > n_max) { r.n = 0; r.row0 = 0; r.err |= kErrBadRows; }
  } else if (n_per_seq) {
    r.n = n_per_seq[b];
    if (r.n < 0 || r.n > n_max) { r.n = 0; r.err |= kErrBadRows; }
  }
  return r;
}

// Element offset of row t of sequence b and head h.
__host__ __device__ inline int64_t row_offset(const RowStrides& s, bool packed, int b, int row0, int h, int t) {
  return (packed ? (int64_t)0 : (int64_t)b * s.seq) + (int64_t)h * s.head + ((int64_t)row0 + t) * s.row;
}

// The pool's page of position `pos` of sequence b: -1 where the table names none.  0 <= pos < max_pages * page_size.
__host__ __device__ inline int page_at(const PagedArgs& a, int b, int index) {
  const int page = a.page_table[(int64_t)b * a.max_pages + index];
  return (uint32_t)page < (uint32_t)a.n_pages ? page : -1;
}
// Row number in the pool [n_pages, H_kv, page_size].
__host__ __device__ inline int64_t pool_row(const PagedArgs& a, int page, int head, int slot) {
  return ((int64_t)page * a.H_kv + head) * a.page_size + slot;
}

// Few rows per (sequence, KV head): the launch's workgroups and what they leave for each other.
struct TokensPlan {
  int workgroups, max_rows;                             // max_rows: tokens times group, 0: no sequence is served that way
  float* partials;                                      // [workgroups][2][16 or 32][d_h + 4]
  int32_t* tickets;                                     // [workgroups], 0 between launches
};
// The most rows, tokens times group, for which it is faster than the other kernel, or whose sums registers hold next to the positions in flight (us, this
// kernel / the other; f16 rows of 8 KV heads over 32 768 positions: 16 bits, 64 channels, 4 rows 19.5 / 35, 32 31.5 / 35, 40 43 / 37, 64 50 / 38; 128
// channels, 4 and 32 rows 32 / 55 and 53 / 56; 256 channels, 4 and 16 rows 57 / 103 and 76 / 103; int8 pages, 64 channels, 32 and 40 rows 33 / 39 and 45 / 41;
// 16 sequences of 4096 positions, 128 channels, 4 rows 53 / 63, of int8 pages 23 / 43).
constexpr int tokens_rows(int d_h) { return d_h == 256 ? 16 : 32; }
// Workgroups per CU by what they are built for: with 4096 sums a wave's registers are those of two.
constexpr int tokens_per_cu(int d_h, int tile_rows) { return d_h * tile_rows >= 4096 ? 1 : 2; }
constexpr int kTokensWorkgroups = 512;                  // at most

// Many rows per (sequence, KV head): row tiles of chunk_rows rows.
constexpr int chunk_rows = 128;
// Workgroups per CU: what the registers of a wave with d_h sums per row allow.
constexpr int chunk_per_cu(int d_h) { return d_h == 256 ? 1 : (d_h == 64 ? 3 : 2); }
struct ChunkPlan {
  int workgroups;
  int tiles;                                            // row tiles per (sequence, KV head), each by a workgroup of its own; 0: equal parts of the work
  float* partials;                                      // ... which leave [workgroups][2][2 chunk_rows lanes][d_h / 2 + 4] for each other
  int32_t* tickets;                                     // [2][workgroups], 0 between launches
};

hipError_t launch_paged_append(const PagedRowsArgs& a, int dtype, int page_type, hipStream_t s);
hipError_t launch_paged_read(const PagedRowsArgs& a, int dtype, int page_type, hipStream_t s);
hipError_t launch_paged_chunk(const PagedAttendArgs& a, const ChunkPlan& c, int dtype, int page_type, hipStream_t s);
hipError_t launch_paged_tokens(const PagedAttendArgs& a, const TokensPlan& t, int dtype, int page_type, hipStream_t s);

}  // namespace sparq
