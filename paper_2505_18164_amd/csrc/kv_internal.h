// Key/value cache in the storage type, bf16 or fp32 (mdi_kv_* of mdi.h): what its entry points and kernels share.
//
// It lies like the 8-bit one, [page][kv head][key, value][position of the page][channel], so a head's keys of one page are one
// stretch of memory, and its values the next.
#pragma once

#include <algorithm>

#include "kv8_internal.h"

namespace mdi {

struct KvCache : KvPages { void* data; int dtype; };             // mdi_kv as the kernels take it
typedef Kv8Rows KvRows;

// Rows into the cache, query and key heads normalised and rotated on the way (kv_append.hip).  Element (row, head, channel) of q at
// row * q_row + head * q_head + channel, of k and v with kv_row and kv_head.
struct KvAppend {
  const void *q, *k, *v; void* q_out;
  long q_row, q_head, kv_row, kv_head, out_row;
  const float *q_g, *q_b, *k_g, *k_b; const double* freq;        // [h], [rot / 2]; no gain: not normalised
  float eps; int H, rot, rms;                                    // H = 0: keys and values only
};
void launch_kv_append(hipStream_t s, const KvCache& c, const KvRows& r, const KvAppend& a);

// What a row at position p sees: the positions up to p that are less than `window` behind it, and the first `sinks`.
struct KvSight { int window, sinks; };                           // both at most 2^30, window at least 1
// How many positions a row sees at most, and 32 for where the two parts begin and end (KvSpan).
inline int kv_most_seen(const KvSight& w, int max_ctx) { return (int)std::min<long>(max_ctx, (long)w.window + w.sinks + 32); }

// How an attention call is divided: what a row sees goes to workgroups in pieces, at most `splits` of them.  A row with one piece is
// finished where it is computed; of the others every piece leaves its h weighted sums, its reference and its sum of
// weights, which a second launch adds.  How many pieces a row and head has is left by whoever computes the first one.
// wgs > 0 (kv_decode.hip): the cut is another, all samples' places in equal shares for so many workgroups, of at least `chunk`.
enum KvKernel { kKvDecode, kKvPrompt, kKvAny };
struct KvPlan { KvKernel kernel; int chunk, splits, wgs, groups, rows; };   // chunk: places, or (kv_prompt.hip) blocks of 64; groups: kv_prompt.hip's, of wavefronts in a workgroup; kv_any.hip's, of sixteen rows; rows: kv_prompt.hip's, of a workgroup
inline size_t kv_part_bytes(const KvPlan& p, const KvCache& c, const KvRows& r, int H) {
  return p.splits > 1 ? (size_t)r.n_rows * H * (p.splits * (size_t)(c.h + 2) + 1) * sizeof(float) : 0;
}
struct KvAttn {
  const void* q; long q_stride;      // [n_rows][H][h], rows q_stride elements apart, in the cache's type
  void* out; long out_stride;
  int H; float scale;                // the softmax's scale times log2 e: scores are exponents of two
  KvSight sight;
  float* part; KvPlan plan;
};
// One new token per sample in bf16 with heads of 64 or 128: on the matrix cores (kv_decode.hip).
void launch_kv_decode(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a);
// Packed rows in bf16 with heads of 64 or 128: on the matrix cores (kv_prompt.hip).  kv_allow_lds: before the first launch on the current device.
bool kv_allow_lds();
void launch_kv_prompt(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a);
// Any other, also on the matrix cores, and few packed rows (kv_any.hip).
void launch_kv_any(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a);
// Whichever of them a.plan names (kv_plan.h), and the launch that adds the pieces.
void launch_kv_attn(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a);

}  // namespace mdi
