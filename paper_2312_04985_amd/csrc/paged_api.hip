// C ABI of the paged cache (include/sparq.h): argument validation, launch planning, enqueue.
#include "../../include/sparq.h"

#include <hip/hip_runtime.h>

#include "paged.h"

static_assert((int)sparq::kPages16 == SPARQ_PAGES_16 && (int)sparq::kPagesI8 == SPARQ_PAGES_I8 && (int)sparq::kPagesE4M3 == SPARQ_PAGES_E4M3, "page types");
static_assert(sparq::kErrBadSeqLen == SPARQ_ERR_BAD_SEQ_LEN && sparq::kErrBadRows == SPARQ_ERR_BAD_ROWS && sparq::kErrBadPage == SPARQ_ERR_BAD_PAGE, "error bits");

namespace {

using namespace sparq;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_paged_shape(const sparq_paged_shape* s) {
  if (!s) return SPARQ_EINVAL;
  if (s->B < 1 || s->H < 1 || s->H_kv < 1 || s->d_h < 1 || s->H % s->H_kv != 0) return SPARQ_EINVAL;
  if (s->page_size < 16 || s->page_size % 16 != 0 || s->n_pages < 1 || s->max_pages < 1) return SPARQ_EINVAL;
  const int64_t capacity = (int64_t)s->max_pages * s->page_size;
  if (capacity > INT32_MAX - (1 << 16)) return SPARQ_EINVAL;      // (positions are counted up in steps behind the last one)
  if (s->dtype != SPARQ_F16 && s->dtype != SPARQ_BF16) return SPARQ_EINVAL;
  if (s->page_type != SPARQ_PAGES_16 && s->page_type != SPARQ_PAGES_I8 && s->page_type != SPARQ_PAGES_E4M3) return SPARQ_EINVAL;
  if (s->flags & ~(uint32_t)SPARQ_FLAG_PAGED_ALL) return SPARQ_EINVAL;
  if (s->window < 0 || s->S_bound < 0 || s->S_bound > capacity) return SPARQ_EINVAL;
  if (s->d_h != 64 && s->d_h != 128 && s->d_h != 256) return SPARQ_EUNSUPPORTED;
  if ((int64_t)s->B * s->H > (int64_t)1 << 30) return SPARQ_EUNSUPPORTED;
  return SPARQ_OK;
}

int check_rows(const sparq_paged_shape* s, const sparq_rows* r) {
  if (!r || r->n < 1 || (r->n_per_seq && r->row_start)) return SPARQ_EINVAL;
  if (r->row_start && r->n_rows < 1) return SPARQ_EINVAL;
  // (row numbers of a launch, B n H, are formed in 32 bits)
  if ((int64_t)s->B * r->n > INT32_MAX / s->H) return SPARQ_EUNSUPPORTED;
  return SPARQ_OK;
}

// The strides that a call steps along: those of extents of one are not looked at.
RowStrides strides_of(const sparq_paged_shape* s, const sparq_rows* r, const sparq_strides* t, int heads) {
  return RowStrides{!r->row_start && s->B > 1 ? t->seq : 0, heads > 1 ? t->head : 0, (r->row_start ? r->n_rows : r->n) > 1 ? t->row : 0};
}

// `written`: rows must not lie on top of each other
int check_strides(const sparq_paged_shape* s, const sparq_rows* r, const sparq_strides* t, int heads, bool written) {
  if (!t) return SPARQ_EINVAL;
  const RowStrides u = strides_of(s, r, t, heads);
  if (u.seq < 0 || u.head < 0 || u.row < 0 || u.seq % 8 || u.head % 8 || u.row % 8) return SPARQ_EINVAL;
  if (!written) return SPARQ_OK;
  if (!r->row_start && s->B > 1 && u.seq < s->d_h) return SPARQ_EINVAL;
  if (heads > 1 && u.head < s->d_h) return SPARQ_EINVAL;
  if ((r->row_start ? r->n_rows : r->n) > 1 && u.row < s->d_h) return SPARQ_EINVAL;
  return SPARQ_OK;
}

int check_paged_cache(const sparq_paged_shape* s, const sparq_paged_cache* c) {
  if (!c || !c->K || !c->V || !c->page_table || !c->seq_lens) return SPARQ_EINVAL;
  if (!aligned16(c->K) || !aligned16(c->V)) return SPARQ_EINVAL;
  if (s->page_type != SPARQ_PAGES_16 && (!c->K_scale || !c->V_scale || !aligned16(c->K_scale) || !aligned16(c->V_scale))) return SPARQ_EINVAL;
  return SPARQ_OK;
}

// How an attention call is served: by the kernel whose waves divide the positions where the rows of a KV head (tokens times
// group) are few (tokens_rows), by the kernel whose waves divide the rows otherwise; by both where only the
// device knows how many rows each sequence has: single tokens then go to the first, longer chunks to the second.
struct AttendPlan { int tokens_rows, chunk; };   // rows that the first kernel takes at most (0: not launched); whether the second is launched

AttendPlan attend_plan(const sparq_paged_shape* s, int n, bool counted) {
  const int64_t g = s->H / s->H_kv, most = tokens_rows(s->d_h);
  if (n * g <= most) return {(int)(n * g), 0};
  if (!counted) return {0, 1};
  const int64_t single = (g + 15) / 16 * 16;
  return {single <= most ? (int)single : 0, 1};
}

int tokens_tile(int rows) { return rows <= 16 ? 16 : 32; }

// Workgroups of the first kernel: what runs at once, but no more than 32 for a unit, whose last one puts their results together, or 64 while
// that keeps to one per CU (us, 32 / 64 for each, 32 768 positions of 128 channels: 8 units of e4m3 pages 25.2 / 28.3, of 16 bits 32.3 / 36.0;
// 30 000 of 64, 4 units of int8 pages 23.7 / 19.4).
int tokens_workgroups(const sparq_paged_shape* s, int tile) {
  const int64_t units = (int64_t)s->B * s->H_kv, most = 256 * tokens_per_cu(s->d_h, tile);
  const int64_t one_per_cu = units * 64 < 256 ? units * 64 : 256, want = units * 32 > one_per_cu ? units * 32 : one_per_cu;
  return (int)(want < most ? want : most);
}

// Row tiles of the second kernel per (sequence, KV head) if a workgroup serves each, 0 if they are cut into equal parts of the work: where the host
// cannot know how many there are, and where they are fewer than three quarters of the workgroups that run at once (128 and 256 channels), or than
// four per CU (64; both sides are in paged_chunk.hip).
int chunk_tiles(const sparq_paged_shape* s, int n, bool counted) {
  const int64_t rows = (int64_t)n * (s->H / s->H_kv), tiles = (rows + chunk_rows - 1) / chunk_rows;
  const int64_t enough = s->d_h == 64 ? 4 * 256 : 3 * 256 * chunk_per_cu(s->d_h) / 4;
  return !counted && tiles * s->B * s->H_kv >= enough && tiles * s->B * s->H_kv <= UINT32_MAX / 256 ? (int)tiles : 0;   // (threads of a launch: 32 bits)
}

// Workgroups of the second kernel for equal parts: what runs at once, and no more than could have work (a row tile, and 4 tiles of positions of one).
// With 64 channels three fit a CU; where little falls to each, two do it sooner, because fewer results are put together (us, two / three: 512 rows of
// 4 heads over 32 768 positions, 8 KV heads, 16 bits 215 / 207, e4m3 270 / 256; up to 301 rows of 8 heads that see 1000 positions, 8 sequences
// of 2 KV heads, int8 34.5 / 37).
int chunk_workgroups(const sparq_paged_shape* s, int n) {
  const int64_t rows = (int64_t)n * (s->H / s->H_kv), bound = s->S_bound > 0 ? s->S_bound : (int64_t)s->max_pages * s->page_size;
  const int64_t tiles = (int64_t)s->B * s->H_kv * ((rows + chunk_rows - 1) / chunk_rows);
  const int64_t seen = s->window > 0 && s->window + (int64_t)chunk_rows < bound ? s->window + (int64_t)chunk_rows : bound;   // positions of a row tile, at most
  const int64_t could = tiles * (seen / 256 + 1);
  const int per_cu = chunk_per_cu(s->d_h) > 2 && could < 4 * 3 * 256 ? 2 : chunk_per_cu(s->d_h);
  return (int)(could < 256 * per_cu ? could : 256 * per_cu);
}

// Scratch behind the control block; the two kernels of a call follow each other and share it.
size_t tokens_scratch(const sparq_paged_shape* s, int rows) {
  size_t most = 0;
  for (int tile = 16; tile <= tokens_tile(rows); tile *= 2) {
    const size_t need = (size_t)tokens_workgroups(s, tile) * 2 * tile * (s->d_h + 4) * sizeof(float);
    most = need > most ? need : most;
  }
  return most;
}
size_t chunk_scratch(const sparq_paged_shape* s, int n) { return (size_t)chunk_workgroups(s, n) * 2 * (2 * chunk_rows) * (s->d_h / 2 + 4) * sizeof(float); }

// (calls of fewer rows than n need no more: they have at most as many rows per KV head, and row tiles, as are counted here)
size_t paged_workspace(const sparq_paged_shape* s, int n) {
  const int64_t rows = (int64_t)n * (s->H / s->H_kv), most = tokens_rows(s->d_h);
  const size_t first = tokens_scratch(s, (int)(rows < most ? rows : most)), second = rows > most ? chunk_scratch(s, n) : 0;
  return (size_t)kControlBytes + (first > second ? first : second);
}

// everything that the calls have in common
int check_call(const sparq_paged_shape* s, const sparq_paged_cache* c, const sparq_rows* r, const void* ws, size_t ws_bytes) {
  int rc = check_paged_shape(s);
  if (rc == SPARQ_OK) rc = check_paged_cache(s, c);
  if (rc == SPARQ_OK) rc = check_rows(s, r);
  if (rc != SPARQ_OK) return rc;
  if (!ws || !aligned16(ws) || ws_bytes < paged_workspace(s, r->n)) return SPARQ_EWORKSPACE;
  return SPARQ_OK;
}

static_assert(kTokensWorkgroups <= kTickets && 2 * 256 * chunk_per_cu(64) <= kTickets, "the workgroups' counters");

PagedArgs paged_args(const sparq_paged_shape* s, const sparq_paged_cache* c, const sparq_rows* r, void* ws) {
  PagedArgs p{};
  p.K = c->K; p.V = c->V; p.K_scale = c->K_scale; p.V_scale = c->V_scale; p.page_table = c->page_table; p.seq_lens = c->seq_lens;
  p.n_per_seq = r->n_per_seq; p.row_start = r->row_start; p.err = static_cast<int32_t*>(ws);
  p.B = s->B; p.H = s->H; p.H_kv = s->H_kv; p.d_h = s->d_h; p.page_size = s->page_size; p.n_pages = s->n_pages; p.max_pages = s->max_pages;
  p.bound = s->S_bound > 0 ? s->S_bound : s->max_pages * s->page_size;
  p.n = r->n; p.n_rows = r->row_start ? r->n_rows : 0;
  p.by_page = make_divider(s->page_size); p.by_H_kv = make_divider(s->H_kv); p.by_n = make_divider(r->n);
  return p;
}

int move_rows(const sparq_paged_shape* shape, const sparq_paged_cache* cache, const sparq_rows* rows, const int32_t* first, void* k, void* v,
              const sparq_strides* strides, void* workspace, size_t workspace_bytes, void* hip_stream, bool reads) {
  int rc = check_call(shape, cache, rows, workspace, workspace_bytes);
  // (a thread for 8 channels, and no more than 2^32 of them)
  if (rc == SPARQ_OK && (int64_t)shape->B * rows->n * shape->H_kv > UINT32_MAX / (shape->d_h / 8) - 256) rc = SPARQ_EUNSUPPORTED;
  if (rc == SPARQ_OK && (!k || !v || !aligned16(k) || !aligned16(v))) rc = SPARQ_EINVAL;
  if (rc == SPARQ_OK) rc = check_strides(shape, rows, strides, shape->H_kv, reads);
  if (rc != SPARQ_OK) return rc;
  PagedRowsArgs a{};
  a.p = paged_args(shape, cache, rows, workspace);
  a.k = k; a.v = v; a.first = first; a.s = strides_of(shape, rows, strides, shape->H_kv);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = reads ? launch_paged_read(a, shape->dtype, shape->page_type, s) : launch_paged_append(a, shape->dtype, shape->page_type, s);
  return e == hipSuccess ? SPARQ_OK : SPARQ_ELAUNCH;
}

}  // namespace

extern "C" {

int sparq_paged_workspace_bytes(const sparq_paged_shape* shape, int32_t n, size_t* out_bytes) {
  const int rc = check_paged_shape(shape);
  if (rc != SPARQ_OK) return rc;
  if (n < 1 || !out_bytes) return SPARQ_EINVAL;
  *out_bytes = paged_workspace(shape, n);
  return SPARQ_OK;
}

int sparq_paged_append(const sparq_paged_shape* shape, const sparq_paged_cache* cache, const sparq_rows* rows, const void* k_new, const void* v_new,
                       const sparq_strides* strides, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return move_rows(shape, cache, rows, nullptr, const_cast<void*>(k_new), const_cast<void*>(v_new), strides, workspace, workspace_bytes, hip_stream, false);
}

int sparq_paged_read(const sparq_paged_shape* shape, const sparq_paged_cache* cache, const sparq_rows* rows, const int32_t* first, void* K_out, void* V_out,
                     const sparq_strides* strides, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return move_rows(shape, cache, rows, first, K_out, V_out, strides, workspace, workspace_bytes, hip_stream, true);
}

int sparq_paged_attention(const sparq_paged_shape* shape, const sparq_paged_cache* cache, const sparq_rows* rows, const void* q, const sparq_strides* q_strides,
                          void* out, const sparq_strides* out_strides, float* lse_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int rc = check_call(shape, cache, rows, workspace, workspace_bytes);
  if (rc == SPARQ_OK && (!q || !out || !aligned16(q) || !aligned16(out))) rc = SPARQ_EINVAL;
  if (rc == SPARQ_OK) rc = check_strides(shape, rows, q_strides, shape->H, false);
  if (rc == SPARQ_OK) rc = check_strides(shape, rows, out_strides, shape->H, true);
  if (rc != SPARQ_OK) return rc;
  PagedAttendArgs a{};
  a.p = paged_args(shape, cache, rows, workspace);
  a.q = q; a.out = out; a.lse = lse_out; a.qs = strides_of(shape, rows, q_strides, shape->H); a.os = strides_of(shape, rows, out_strides, shape->H);
  a.window = shape->window; a.all = (shape->flags & SPARQ_FLAG_PAGED_ALL) != 0;
  a.group = shape->H / shape->H_kv; a.by_group = make_divider(a.group);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const AttendPlan plan = attend_plan(shape, rows->n, rows->n_per_seq || rows->row_start);
  hipError_t e = hipSuccess;
  if (plan.tokens_rows) {
    const TokensPlan t{tokens_workgroups(shape, tokens_tile(plan.tokens_rows)), plan.tokens_rows, reinterpret_cast<float*>(static_cast<char*>(workspace) + kControlBytes),
                       reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + kTicketOffset)};
    e = launch_paged_tokens(a, t, shape->dtype, shape->page_type, s);
  }
  a.skip_rows = plan.tokens_rows;
  if (e == hipSuccess && plan.chunk) {
    const int tiles = chunk_tiles(shape, rows->n, rows->n_per_seq || rows->row_start);
    const ChunkPlan c{tiles ? tiles * shape->B * shape->H_kv : chunk_workgroups(shape, rows->n), tiles, reinterpret_cast<float*>(static_cast<char*>(workspace) + kControlBytes),
                      reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + kTicketOffset)};
    e = launch_paged_chunk(a, c, shape->dtype, shape->page_type, s);
  }
  return e == hipSuccess ? SPARQ_OK : SPARQ_ELAUNCH;
}

}  // extern "C"
