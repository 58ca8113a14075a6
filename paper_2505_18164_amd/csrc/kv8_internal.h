// Key/value cache in 8 bits (mdi_kv8_* of mdi.h): what its entry points, the partition and the kernels share.
//
// A row - one position of one kv head, its key or its value - is kept as head_dim codes of 8 bits and one scale:
//   top = max |x|, c = 127 / top and scale = top / 127 (each rounded to fp32),
//   code = the whole number nearest to x c, ties to even, value = code * scale.
// A value is off by at most half a scale.  One scale a row, because it then stands outside both sums of the attention: a score is
// scale_k (q . codes_k), the weighted sum takes (weight * scale_v) codes_v, and codes are exact in bf16, so the matrix
// cores multiply what the cache holds without another rounding.
#pragma once

#include "mdi_internal.h"

namespace mdi {

struct KvPages {                     // how a paged cache lies, whatever its rows are: of 8 bits here, of the storage type in kv_internal.h
  const int32_t* tables; int32_t* err;
  int n_pages, K, h, pt;
  unsigned pt_magic, pt_one;         // page of a position: the high word of pos * pt_magic, or (pages of one) the position & pt_one
  int n_tables, table_stride;
};
struct Kv8Cache : KvPages {          // mdi_kv8 as the kernels take it
  int8_t* codes; float* scales;      // [n_pages][K][2][pt][h], [n_pages][K][2][pt]
};
struct Kv8Rows {                     // mdi_kv8_rows
  const int32_t *table, *start, *pos;
  int n, n_rows, max_ctx;            // max_ctx <= table_stride * pt
};

struct Kv8RowsIO {                   // rows in or out: element (row, kv head, channel) at row * row_stride + head * head_stride + channel
  void *k, *v; long row_stride, head_stride;
};
void launch_kv8_write(hipStream_t s, int dtype, const Kv8Cache& c, const Kv8Rows& r, const Kv8RowsIO& io);
void launch_kv8_read(hipStream_t s, int dtype, const Kv8Cache& c, const Kv8Rows& r, const Kv8RowsIO& io);

// How an attention call is divided: a row's visible positions go to workgroups in pieces of `chunk`, at most `splits` of them.
// A row with one piece is finished where it is computed; of the others, every piece leaves its h weighted sums and, behind all of
// those, its reference and its sum of weights (kv8_part_sums, kv8_part_marks in kv8_device.h); a second launch adds them.
// wgs > 0 (kv8_decode.hip): the cut is another, all samples' positions in equal shares for so many workgroups, of at least `chunk`.
constexpr int kKv8Tile = 128;        // positions that shares are counted in
struct Kv8Plan { int chunk, splits, wgs, groups; };   // groups: kv8_prompt.hip's, of wavefronts in a workgroup
__host__ __device__ inline int kv8_groups(const KvPages& c, int H) { return (H / c.K + 15) / 16; }   // sets of up to sixteen query heads of a kv head
Kv8Plan kv8_plan(const Kv8Cache& c, const Kv8Rows& r, int H, size_t part_limit = SIZE_MAX);   // part_limit: room for the pieces' sums
inline size_t kv8_part_bytes(const Kv8Plan& p, const Kv8Cache& c, const Kv8Rows& r, int H) {
  return p.splits > 1 ? (size_t)r.n_rows * H * p.splits * (c.h + 2) * sizeof(float) : 0;
}
struct Kv8Attn {
  const bf16_t* q; long q_stride;    // [n_rows][H][h], rows q_stride elements apart
  bf16_t* out; long out_stride;
  int H; float scale;                // scores are scale * (q . k) in powers of two: the softmax's scale times log2 e
  float* part; Kv8Plan plan;
};
// One new token per sample with heads of 64 or 128: on the matrix cores (kv8_decode.hip).
bool kv8_decode_supported(const Kv8Cache& c, const Kv8Rows& r);
Kv8Plan kv8_decode_plan(const Kv8Cache& c, const Kv8Rows& r, int H);
void launch_kv8_decode(hipStream_t s, const Kv8Cache& c, const Kv8Rows& r, const Kv8Attn& a);
// Packed rows with heads of 64 or 128: on the matrix cores (kv8_prompt.hip).  kv8_allow_lds: before the first launch on the current device.
bool kv8_prompt_supported(const Kv8Cache& c, const Kv8Rows& r);
bool kv8_allow_lds();
Kv8Plan kv8_prompt_plan(const Kv8Cache& c, const Kv8Rows& r, int H, size_t part_limit);
void launch_kv8_prompt(hipStream_t s, const Kv8Cache& c, const Kv8Rows& r, const Kv8Attn& a);
void launch_kv8_attn(hipStream_t s, const Kv8Cache& c, const Kv8Rows& r, const Kv8Attn& a);

// What a call of a partition with an 8-bit cache sets up on the device before its layers run (kv8_visit.hip): which rows are whose, at
// which position, and where a new page starts; optionally the rows' angles and inputs, one after the other.
constexpr int kMaxVisits = 64;       // samples one pass over the weights can take
struct Kv8Setup {
  int n, rows;
  int first[kMaxVisits + 1], pos[kMaxVisits], seq[kMaxVisits];
  long page_at[kMaxVisits]; int page[kMaxVisits];   // entry of `tables` to fill (there may be more than 2^31), or -1
  int32_t *start, *at, *table, *row_pos, *zero, *tables;
  const float2* rope; float2* rope_rows; int half;   // rope_rows[row] = rope[its position], `half` pairs each; nullptr: not needed
  const void* in[kMaxVisits]; void* in_rows; int in_bytes;   // in_rows[i] = the in_bytes of in[i]; nullptr: the rows are together already
};
void launch_kv8_setup(hipStream_t s, const Kv8Setup& a);
struct Kv8Handoff { const void* rows; void* out[kMaxVisits]; int n, bytes; };   // out[i] = row i
void launch_kv8_handoff(hipStream_t s, const Kv8Handoff& a);

// The geometry of a cache; false when its positions or sizes are beyond what the kernels count with.
inline bool kv8_geometry(uint64_t n_pages, uint64_t n_kv_head, uint64_t head_dim, uint64_t page_tokens, uint64_t n_tables, uint64_t table_stride, KvPages* c) {
  if (!n_pages || !n_kv_head || !head_dim || !page_tokens || !n_tables || !table_stride) return false;
  if (head_dim % 8 || head_dim > 256 || n_kv_head > 1024 || n_pages > INT32_MAX || n_tables > INT32_MAX) return false;
  // a position is divided by the page size with one multiplication, exact below the second bound
  if (table_stride * page_tokens > 1u << 30 || table_stride * page_tokens * page_tokens >= (1ull << 32)) return false;
  c->n_pages = (int)n_pages; c->K = (int)n_kv_head; c->h = (int)head_dim; c->pt = (int)page_tokens;
  c->pt_magic = page_tokens == 1 ? 0u : 0xFFFFFFFFu / (unsigned)page_tokens + 1u;
  c->pt_one = page_tokens == 1 ? ~0u : 0u;
  c->n_tables = (int)n_tables; c->table_stride = (int)table_stride;
  return true;
}

}  // namespace mdi
