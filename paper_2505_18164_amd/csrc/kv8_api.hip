// The entry points of the 8-bit cache (mdi_kv8_* of mdi.h): checks on the host, then the launches (two at most, but for packed rows of very many samples).
#include "kv8_internal.h"

using namespace mdi;

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

mdi_status take_cache(const mdi_kv8* k, Kv8Cache* c) {
  if (!k || !k->codes || !k->scales || !k->tables || !aligned16(k->codes) || !aligned16(k->scales)) return MDI_ERR_ARG;
  if (!kv8_geometry(k->n_pages, k->n_kv_head, k->head_dim, k->page_tokens, k->n_tables, k->table_stride, c)) return MDI_ERR_ARG;
  c->codes = k->codes; c->scales = k->scales; c->tables = k->tables; c->err = k->err;
  return MDI_OK;
}

mdi_status take_rows(const mdi_kv8* k, const mdi_kv8_rows* g, Kv8Rows* r) {
  if (!g || (g->n && g->n_rows && !g->pos)) return MDI_ERR_ARG;
  if (g->n > INT32_MAX / 2 || g->n_rows > 1u << 24 || (!g->start && g->n_rows != g->n)) return MDI_ERR_ARG;
  if (!g->max_ctx || g->max_ctx > (uint64_t)k->table_stride * k->page_tokens) return MDI_ERR_ARG;
  *r = Kv8Rows{g->table, g->start, g->pos, (int)g->n, (int)g->n_rows, (int)g->max_ctx};
  return MDI_OK;
}

mdi_status take(const mdi_kv8* k, const mdi_kv8_rows* g, Kv8Cache* c, Kv8Rows* r) {
  const mdi_status st = take_cache(k, c);
  return st != MDI_OK ? st : take_rows(k, g, r);
}

// Query rows of the call: heads that the kv heads divide.  A launch has fewer than 2^32 threads, 256 a row and head (kv8_prompt.hip,
// which counts otherwise, takes several launches); the tiles of all units, and kKv8Begin more each, are counted in 32 bits.
bool good_heads(const Kv8Cache& c, const Kv8Rows& r, uint32_t n_head) {
  return n_head && n_head <= 4096 && n_head % (uint32_t)c.K == 0 && (uint64_t)r.n_rows * n_head < (1ull << 24) &&
         (uint64_t)r.n * n_head * ((unsigned)r.max_ctx / kKv8Tile + 3) < (1ull << 30);
}

mdi_status hip_status() { return hipGetLastError() == hipSuccess ? MDI_OK : MDI_ERR_HIP; }

mdi_status rows_io(const mdi_kv8* k, const mdi_kv8_rows* g, void* kp, void* vp, uint32_t dtype, uint64_t row_stride, uint64_t head_stride,
                   Kv8Cache* c, Kv8Rows* r, Kv8RowsIO* io) {
  const mdi_status st = take(k, g, c, r);
  if (st != MDI_OK) return st;
  if (dtype > MDI_BF16) return MDI_ERR_ARG;
  const uint64_t unit = dtype == MDI_BF16 ? 8 : 4;               // elements of 16 bytes
  if ((r->n && r->n_rows && (!kp || !vp)) || !aligned16(kp) || !aligned16(vp) || row_stride % unit || head_stride % unit) return MDI_ERR_ARG;
  if ((uint64_t)r->n_rows * c->K * c->h >= 1ull << 33) return MDI_ERR_ARG;       // a launch has fewer than 2^32 threads
  if (row_stride > 1ull << 38 || head_stride > 1ull << 38) return MDI_ERR_ARG;   // offsets stay within 64 bits
  *io = Kv8RowsIO{kp, vp, (long)row_stride, (long)head_stride};
  return MDI_OK;
}

}  // namespace

extern "C" {

mdi_status mdi_kv8_write(const mdi_kv8* cache, const mdi_kv8_rows* rows, const void* k, const void* v, uint32_t dtype, uint64_t row_stride,
                         uint64_t head_stride, void* hip_stream) {
  Kv8Cache c; Kv8Rows r; Kv8RowsIO io;
  const mdi_status st = rows_io(cache, rows, const_cast<void*>(k), const_cast<void*>(v), dtype, row_stride, head_stride, &c, &r, &io);
  if (st != MDI_OK || !r.n || !r.n_rows) return st;
  launch_kv8_write((hipStream_t)hip_stream, (int)dtype, c, r, io);
  return hip_status();
}

mdi_status mdi_kv8_read(const mdi_kv8* cache, const mdi_kv8_rows* rows, void* k, void* v, uint32_t dtype, uint64_t row_stride,
                        uint64_t head_stride, void* hip_stream) {
  Kv8Cache c; Kv8Rows r; Kv8RowsIO io;
  const mdi_status st = rows_io(cache, rows, k, v, dtype, row_stride, head_stride, &c, &r, &io);
  if (st != MDI_OK || !r.n || !r.n_rows) return st;
  launch_kv8_read((hipStream_t)hip_stream, (int)dtype, c, r, io);
  return hip_status();
}

mdi_status mdi_kv8_attn_bytes(const mdi_kv8* cache, const mdi_kv8_rows* rows, uint32_t n_head, size_t* workspace_bytes) {
  if (!workspace_bytes) return MDI_ERR_ARG;
  Kv8Cache c; Kv8Rows r;
  const mdi_status st = take(cache, rows, &c, &r);
  if (st != MDI_OK) return st;
  if (!good_heads(c, r, n_head)) return MDI_ERR_ARG;
  *workspace_bytes = r.n && r.n_rows ? kv8_part_bytes(kv8_plan(c, r, (int)n_head), c, r, (int)n_head) : 0;
  return MDI_OK;
}

mdi_status mdi_kv8_attn(const mdi_kv8* cache, const mdi_kv8_rows* rows, const void* q, uint64_t q_stride, uint32_t n_head, float scale, void* out,
                        uint64_t out_stride, void* workspace, size_t workspace_bytes, void* hip_stream) {
  Kv8Cache c; Kv8Rows r;
  const mdi_status st = take(cache, rows, &c, &r);
  if (st != MDI_OK) return st;
  if ((r.n && r.n_rows && (!q || !out)) || !aligned16(q) || !aligned16(out) || !good_heads(c, r, n_head)) return MDI_ERR_ARG;
  const uint64_t width = (uint64_t)n_head * c.h;
  if (q_stride < width || out_stride < width || q_stride % 8 || out_stride % 8 || q_stride > 1ull << 38 || out_stride > 1ull << 38) return MDI_ERR_ARG;
  const float scale2 = scale * 1.44269504f;                      // scores are exponents of two
  if (!(scale2 - scale2 == 0.f)) return MDI_ERR_ARG;              // finite
  if (!r.n || !r.n_rows) return MDI_OK;
  const Kv8Plan plan = kv8_plan(c, r, (int)n_head);
  const size_t need = kv8_part_bytes(plan, c, r, (int)n_head);
  if (need && (!workspace || !aligned16(workspace))) return MDI_ERR_ARG;
  if (need > workspace_bytes) return MDI_ERR_NOMEM;
  if (!kv8_allow_lds()) return MDI_ERR_HIP;
  launch_kv8_attn((hipStream_t)hip_stream, c, r,
                  Kv8Attn{(const bf16_t*)q, (long)q_stride, (bf16_t*)out, (long)out_stride, (int)n_head, scale2, (float*)workspace, plan});
  return hip_status();
}

}  // extern "C"
