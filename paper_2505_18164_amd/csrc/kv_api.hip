// The entry points of the cache in the storage type (mdi_kv_* of mdi.h): checks on the host, then the launches: one or two, of very many samples a few.
#include <algorithm>

#include "kv_plan.h"

using namespace mdi;

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
constexpr uint64_t kMostStride = 1ull << 38;                     // offsets stay within 64 bits

mdi_status take(const mdi_kv* k, const mdi_kv8_rows* g, KvCache* c, KvRows* r) {
  if (!k || !k->data || !k->tables || !aligned16(k->data) || k->dtype > MDI_BF16) return MDI_ERR_ARG;
  if (!kv8_geometry(k->n_pages, k->n_kv_head, k->head_dim, k->page_tokens, k->n_tables, k->table_stride, c)) return MDI_ERR_ARG;
  c->data = k->data; c->dtype = (int)k->dtype; c->tables = k->tables; c->err = k->err;
  if (!g || (g->n && g->n_rows && !g->pos)) return MDI_ERR_ARG;
  if (g->n > INT32_MAX / 2 || g->n_rows > 1u << 24 || (!g->start && g->n_rows != g->n)) return MDI_ERR_ARG;
  if (!g->max_ctx || g->max_ctx > (uint64_t)k->table_stride * k->page_tokens) return MDI_ERR_ARG;
  *r = KvRows{g->table, g->start, g->pos, (int)g->n, (int)g->n_rows, (int)g->max_ctx};
  return MDI_OK;
}

// Query rows of an attention call: heads that the kv heads divide.  A launch has fewer than 2^32 threads, 256 a row and head; tiles of
// all samples and heads are counted in 32 bits.
bool good_heads(const KvCache& c, const KvRows& r, uint32_t n_head) {
  return n_head && n_head <= 4096 && n_head % (uint32_t)c.K == 0 && (uint64_t)r.n_rows * n_head < (1ull << 24) &&
         (uint64_t)r.n * n_head * ((unsigned)r.max_ctx / kKv8Tile + 3) < (1ull << 30);
}

KvSight sight_of(uint32_t window, uint32_t sinks) {
  constexpr uint32_t all = 1u << 30;                             // positions are below it
  return KvSight{(int)(window && window < all ? window : all), (int)(window ? std::min(sinks, all) : 0)};
}

bool good_stride(uint64_t stride, uint64_t unit) { return stride % unit == 0 && stride <= kMostStride; }
mdi_status hip_status() { return hipGetLastError() == hipSuccess ? MDI_OK : MDI_ERR_HIP; }

}  // namespace

extern "C" {

mdi_status mdi_kv_append(const mdi_kv* cache, const mdi_kv8_rows* rows, const mdi_qk_prep* prep, const void* k, const void* v, uint64_t row_stride,
                         uint64_t head_stride, const void* q, uint64_t q_row_stride, uint64_t q_head_stride, uint32_t n_head, void* q_out,
                         uint64_t q_out_stride, void* hip_stream) {
  KvCache c; KvRows r;
  const mdi_status st = take(cache, rows, &c, &r);
  if (st != MDI_OK) return st;
  const uint64_t unit = c.dtype == MDI_BF16 ? 8 : 4;             // elements of 16 bytes
  const bool some = r.n && r.n_rows;
  if ((some && (!k || !v)) || !aligned16(k) || !aligned16(v) || !good_stride(row_stride, unit) || !good_stride(head_stride, unit)) return MDI_ERR_ARG;
  if (n_head) {
    if (n_head > 4096 || n_head % (uint32_t)c.K || (some && (!q || !q_out)) || !aligned16(q) || !aligned16(q_out)) return MDI_ERR_ARG;
    if (!good_stride(q_row_stride, unit) || !good_stride(q_head_stride, unit) || !good_stride(q_out_stride, unit) || q_out_stride < (uint64_t)n_head * c.h)
      return MDI_ERR_ARG;
    if (some && q == q_out && ((r.n_rows > 1 && q_row_stride != q_out_stride) || (n_head > 1 && q_head_stride != (uint64_t)c.h))) return MDI_ERR_ARG;
  } else if (q || q_out) {
    return MDI_ERR_ARG;
  }
  if ((uint64_t)r.n_rows * (n_head + 2 * c.K) * c.h >= 1ull << 33) return MDI_ERR_ARG;   // a launch has fewer than 2^32 threads
  KvAppend a{q, k, v, q_out, (long)q_row_stride, (long)q_head_stride, (long)row_stride, (long)head_stride, (long)q_out_stride,
             nullptr, nullptr, nullptr, nullptr, nullptr, 0.f, (int)n_head, 0, 0};
  if (prep) {
    if (prep->norm_kind > MDI_NORM_RMSNORM || prep->rot > cache->head_dim || prep->rot % 8 || (prep->rot && !prep->freq)) return MDI_ERR_ARG;
    if (!(prep->eps >= 0.f) || !(prep->eps - prep->eps == 0.f) || (prep->q_b && !prep->q_g) || (prep->k_b && !prep->k_g)) return MDI_ERR_ARG;
    if ((uintptr_t)prep->freq & 7u) return MDI_ERR_ARG;
    for (const float* p : {prep->q_g, prep->q_b, prep->k_g, prep->k_b}) if (!aligned16(p)) return MDI_ERR_ARG;
    a.q_g = prep->q_g; a.q_b = prep->q_b; a.k_g = prep->k_g; a.k_b = prep->k_b; a.freq = prep->freq;
    a.eps = prep->eps; a.rot = (int)prep->rot; a.rms = prep->norm_kind == MDI_NORM_RMSNORM;
  }
  if (!some) return MDI_OK;
  launch_kv_append((hipStream_t)hip_stream, c, r, a);
  return hip_status();
}

mdi_status mdi_kv_attn_bytes(const mdi_kv* cache, const mdi_kv8_rows* rows, uint32_t n_head, uint32_t window, uint32_t sinks, size_t* workspace_bytes) {
  if (!workspace_bytes) return MDI_ERR_ARG;
  KvCache c; KvRows r;
  const mdi_status st = take(cache, rows, &c, &r);
  if (st != MDI_OK) return st;
  if (!good_heads(c, r, n_head)) return MDI_ERR_ARG;
  *workspace_bytes = r.n && r.n_rows ? kv_part_bytes(kv_plan(c, r, (int)n_head, sight_of(window, sinks)), c, r, (int)n_head) : 0;
  return MDI_OK;
}

mdi_status mdi_kv_attn(const mdi_kv* cache, const mdi_kv8_rows* rows, const void* q, uint64_t q_stride, uint32_t n_head, float scale, uint32_t window,
                       uint32_t sinks, void* out, uint64_t out_stride, void* workspace, size_t workspace_bytes, void* hip_stream) {
  KvCache c; KvRows r;
  const mdi_status st = take(cache, rows, &c, &r);
  if (st != MDI_OK) return st;
  if ((r.n && r.n_rows && (!q || !out)) || !aligned16(q) || !aligned16(out) || !good_heads(c, r, n_head)) return MDI_ERR_ARG;
  const uint64_t width = (uint64_t)n_head * c.h, unit = c.dtype == MDI_BF16 ? 8 : 4;
  if (q_stride < width || out_stride < width || !good_stride(q_stride, unit) || !good_stride(out_stride, unit)) return MDI_ERR_ARG;
  const float scale2 = scale * 1.44269504f;                      // scores are exponents of two
  if (!(scale2 - scale2 == 0.f)) return MDI_ERR_ARG;              // finite
  if (!r.n || !r.n_rows) return MDI_OK;
  const KvSight sight = sight_of(window, sinks);
  const KvPlan plan = kv_plan(c, r, (int)n_head, sight);
  const size_t need = kv_part_bytes(plan, c, r, (int)n_head);
  if (need && (!workspace || !aligned16(workspace))) return MDI_ERR_ARG;
  if (need > workspace_bytes) return MDI_ERR_NOMEM;
  if (q == out) return MDI_ERR_ARG;                              // (queries are read until the last results are written)
  if (!kv_allow_lds()) return MDI_ERR_HIP;
  launch_kv_attn((hipStream_t)hip_stream, c, r, KvAttn{q, (long)q_stride, out, (long)out_stride, (int)n_head, scale2, sight, (float*)workspace, plan});
  return hip_status();
}

}  // extern "C"
