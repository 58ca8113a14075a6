// Device-side parts of the 8-bit cache that its kernels share: which sample and position a row is, and where that lies.
#pragma once

#include "device_utils.h"
#include "kv8_internal.h"

namespace mdi {

__device__ __forceinline__ void kv8_report(const Kv8Cache& c) {
  if (c.err) __hip_atomic_store(c.err, 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Quotient of a position and the page size (exact: table_stride * pt * pt < 2^32 is checked on the host).
__device__ __forceinline__ int kv8_page_of(const Kv8Cache& c, int pos) {
  return c.pt_sh >= 0 ? pos >> c.pt_sh : (int)__umulhi((unsigned)pos, c.pt_magic);
}

// The sample that `row` belongs to, or -1; `row` is the same in all lanes.  The samples' ends are looked at 64 at a time: one
// round trip instead of a search's chain of them.
__device__ __forceinline__ int kv8_sample_of(const Kv8Rows& r, int row) {
  if (!r.start) return row < r.n ? row : -1;
  const int lane = threadIdx.x & 63;
  int s = 0;
  for (int base = 0; base < r.n; base += 64) {
    const bool past = base + lane < r.n && r.start[base + lane + 1] <= row;
    const unsigned long long m = __ballot(past);
    s += __popcll(m);
    if (m != ~0ull) break;
  }
  return s < r.n && r.start[s] <= row ? s : -1;
}

// A sample's page table, or nullptr when the row of `tables` it names is not there.
__device__ __forceinline__ const int32_t* kv8_table(const Kv8Cache& c, const Kv8Rows& r, int sample) {
  const int t = r.table ? r.table[sample] : sample;
  if ((unsigned)t >= (unsigned)c.n_tables) { kv8_report(c); return nullptr; }
  return c.tables + (long)t * c.table_stride;
}

// A page number that is not of this cache is reported and page 0 read in its place.
__device__ __forceinline__ int kv8_checked_page(const Kv8Cache& c, int page) {
  if ((unsigned)page < (unsigned)c.n_pages) return page;
  kv8_report(c);
  return 0;
}

// What a row of an attention call attends to: its sample and the positions it sees (its own and the earlier ones).
struct Kv8View {
  int sample, seen;                  // sample < 0: no sample's row, its output is left alone; seen = 0: its output is zeros
};
__device__ __forceinline__ Kv8View kv8_view(const Kv8Cache& c, const Kv8Rows& r, int row) {
  Kv8View v{kv8_sample_of(r, row), 0};
  if (v.sample < 0) return v;
  const int p0 = r.pos[v.sample];
  if (p0 < 0) return v;
  const long seen = (long)p0 + (r.start ? row - r.start[v.sample] : 0) + 1;
  if (seen > r.max_ctx) kv8_report(c);
  v.seen = (int)max(0l, min(seen, (long)r.max_ctx));
  return v;
}

constexpr float kKv8None = -3e38f;   // reference of a softmax that has seen nothing

}  // namespace mdi
