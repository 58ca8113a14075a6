// Device-side parts of the 8-bit cache that its kernels share: which sample and position a row is, and where that lies.
#pragma once

#include "device_utils.h"
#include "kv8_internal.h"

namespace mdi {

__device__ __forceinline__ void kv8_report(const KvPages& c) {
  if (c.err) __hip_atomic_store(c.err, 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Quotient of a position and the page size (exact: table_stride * pt * pt < 2^32 is checked on the host).
__device__ __forceinline__ int kv8_page_of(const KvPages& c, int pos) {
  return (int)(__umulhi((unsigned)pos, c.pt_magic) | ((unsigned)pos & c.pt_one));
}

// The key of position pos in `page`, as a row of codes or an index of scales; its value is c.pt further.
__device__ __forceinline__ long kv8_row(const KvPages& c, unsigned page, int kv, int pos) {
  return (long)((uint64_t)page * (unsigned)(2 * c.K * c.pt) + (unsigned)(2 * kv * c.pt + pos - kv8_page_of(c, pos) * c.pt));
}

// Where the last of n samples stands that `begun` holds for, one that holds for no sample behind it: a window of at most 64
// samples, or none (len 0).  A round looks at 64 samples, one a lane, so 64 samples take none, 4096 one, 2^24 three; what a wavefront
// does for every row or workgroup may not grow with the number of samples.
struct Kv8Window { int base, len; };
template <typename Begun> __device__ __forceinline__ Kv8Window kv8_window(int n, Begun&& begun) {
  const int lane = threadIdx.x & 63;
  int base = 0, len = n;
  while (len > 64) {
    const int step = (len + 63) >> 6, at = lane * step, k = __popcll(__ballot(at < len && begun(base + min(at, len - 1))));
    if (k == 0) return Kv8Window{0, 0};
    base += (k - 1) * step;
    len = min(step, len - (k - 1) * step);
  }
  return Kv8Window{base, len};
}

// The sample that `row` belongs to, or -1; `row` is the same in all lanes.  Of the window all ends are looked at at once: one round trip
// instead of a search's chain of them.
__device__ __forceinline__ int kv8_sample_of(const Kv8Rows& r, int row) {
  if (!r.start) return row < r.n ? row : -1;
  const Kv8Window w = kv8_window(r.n, [&](int i) { return r.start[i] <= row; });
  const int lane = threadIdx.x & 63, i = w.base + min(lane, max(w.len - 1, 0));
  const int s = w.base + __popcll(__ballot(lane < w.len && r.start[i + 1] <= row));
  return s < w.base + w.len && r.start[s] <= row ? s : -1;
}

// A row of `tables`, or -1 when it is not there.
__device__ __forceinline__ int kv8_checked_row(const KvPages& c, int t) {
  if ((unsigned)t < (unsigned)c.n_tables) return t;
  kv8_report(c);
  return -1;
}

// The row of `tables` that is a sample's, or -1 when the one it names is not there.
__device__ __forceinline__ int kv8_table_row(const KvPages& c, const Kv8Rows& r, int sample) {
  return kv8_checked_row(c, r.table ? r.table[sample] : sample);
}

// A page number that is not of this cache is reported and page 0 read in its place.
__device__ __forceinline__ int kv8_checked_page(const KvPages& c, int page) {
  if ((unsigned)page < (unsigned)c.n_pages) return page;
  kv8_report(c);
  return 0;
}

// What a row of an attention call attends to: its sample and the positions it sees (its own and the earlier ones).
struct Kv8View {
  int sample, seen;                  // sample < 0: no sample's row, its output is left alone; seen = 0: its output is zeros
};
__device__ __forceinline__ Kv8View kv8_view(const KvPages& c, const Kv8Rows& r, int row) {
  Kv8View v{kv8_sample_of(r, row), 0};
  if (v.sample < 0) return v;
  const int p0 = r.pos[v.sample];
  if (p0 < 0) return v;
  const long seen = (long)p0 + (r.start ? row - r.start[v.sample] : 0) + 1;
  if (seen > r.max_ctx) kv8_report(c);
  v.seen = (int)max(0l, min(seen, (long)r.max_ctx));
  return v;
}

// Item (row * H + head)'s piece in the workspace.
__device__ __forceinline__ float* kv8_part_sums(const Kv8Attn& a, const Kv8Cache& c, int item, int piece) {
  return a.part + ((long)item * a.plan.splits + piece) * c.h;
}
__device__ __forceinline__ float2* kv8_part_marks(const Kv8Attn& a, const Kv8Cache& c, const Kv8Rows& r, int item, int piece) {
  return reinterpret_cast<float2*>(a.part + (long)r.n_rows * a.H * a.plan.splits * c.h) + (long)item * a.plan.splits + piece;
}

// The cut of kv8_decode.hip.  The tiles of all samples' units follow one another - sample by sample, a sample's units side by
// side, kKv8Begin more for every unit, what it costs to begin one - and workgroup w has w * per .. + per - 1 of them.  Every
// wavefront works this out for itself, 64 samples at a time; `seen` is what the first 64 see, one a lane.
constexpr int kKv8Begin = 2;         // (1, 2, 4: 30.2, 29.8, 32.1 us for 8 samples of 1 .. 4096 positions of the 7B shape)
__device__ __forceinline__ int kv8_seen(const KvPages& c, const Kv8Rows& r, int sample) { return sample < r.n ? kv8_view(c, r, sample).seen : 0; }
__device__ __forceinline__ int kv8_tiles(int seen) { return (seen + kKv8Tile - 1) / kKv8Tile; }
__device__ __forceinline__ int kv8_cost(const Kv8Rows& r, int sample, int seen) { return sample < r.n ? kv8_tiles(seen) + kKv8Begin : 0; }

struct Kv8Stream { int cost, per, before; };                     // of one unit of every sample; a share; of those before `sample`
template <typename Seen>                                         // seen_of(i): what sample i sees (0: none), `seen` that of the first 64, one a lane
__device__ __forceinline__ Kv8Stream kv8_stream_of(const Kv8Rows& r, int chunk, int wgs, int units, int sample, int seen, Seen&& seen_of) {
  int sum = 0, before = 0;
  for (int i = threadIdx.x & 63; i < r.n; i += 64) {
    const int t = kv8_cost(r, i, i < 64 ? seen : seen_of(i));
    sum += t;
    if (i < sample) before += t;
  }
  for (int off = 32; off >= 1; off >>= 1) { sum += __shfl_xor(sum, off, 64); before += __shfl_xor(before, off, 64); }
  sum = __builtin_amdgcn_readfirstlane(sum);
  return Kv8Stream{sum, max(chunk / kKv8Tile, (int)(((long)sum * units + wgs - 1) / wgs)), __builtin_amdgcn_readfirstlane(before)};
}
__device__ __forceinline__ Kv8Stream kv8_stream(const Kv8Cache& c, const Kv8Rows& r, const Kv8Plan& p, int units, int sample, int seen) {
  return kv8_stream_of(r, p.chunk, p.wgs, units, sample, seen, [&](int i) { return kv8_seen(c, r, i); });
}
struct Kv8Found { int sample, start, seen; };                    // the sample in whose unit `x` lies, and where that unit starts
template <typename Seen>
__device__ __forceinline__ Kv8Found kv8_find_of(const Kv8Rows& r, int x, int seen, Seen&& seen_of) {
  const int lane = threadIdx.x & 63;
  for (int base = 0, sum = 0;; base += 64) {
    if (base) seen = seen_of(base + lane);
    const int t = kv8_cost(r, base + lane, seen);
    int up = t;
    for (int off = 1; off < 64; off <<= 1) { const int o = __shfl_up(up, off, 64); if (lane >= off) up += o; }
    const unsigned long long past = __ballot(sum + up > x);
    if (past || base + 64 >= r.n) {
      const int at = past ? __ffsll(past) - 1 : 0;
      return Kv8Found{__builtin_amdgcn_readfirstlane(base + at), __builtin_amdgcn_readfirstlane(sum + __shfl(up - t, at, 64)),
                      __builtin_amdgcn_readfirstlane(__shfl(seen, at, 64))};
    }
    sum += __shfl(up, 63, 64);
  }
}
__device__ __forceinline__ Kv8Found kv8_find(const Kv8Cache& c, const Kv8Rows& r, int x, int seen) {
  return kv8_find_of(r, x, seen, [&](int i) { return kv8_seen(c, r, i); });
}

constexpr float kKv8None = -3e38f;   // reference of a softmax that has seen nothing

// One row and head by a wavefront, for any head: L lanes hold eight channels each of a position (`ch` on, `live` where the head has
// them), the lane groups take positions from, from + 1 .. and `step` further, up to hi.  A lane group keeps its own running (reference,
// sum, output), which are folded at the end: every lane then has the sums of its eight channels.  Everything is binary32, with no
// other reference than the largest score so far: no size of scores or values is out of its reach that is not out of binary32's.
struct Kv8Sums { float m, l, o[8]; };
__device__ __forceinline__ float kv8_sum_of(float v, int L) {
  for (int off = 1; off < L; off <<= 1) v += __shfl_xor(v, off, 64);
  return v;
}
__device__ __forceinline__ Kv8Sums kv8_attend(const Kv8Cache& c, const int32_t* table, int kv, const float (&q)[8], int L, int ch, bool live,
                                              int from, int step, int hi) {
  const int sub = (threadIdx.x & 63) / L, h = c.h;
  Kv8Sums r{kKv8None, 0.f, {}};
  for (int t0 = from; t0 < hi; t0 += step) {
    const int pos = min(t0 + sub, hi - 1), at = kv8_page_of(c, pos);
    const long rk = kv8_row(c, kv8_checked_page(c, table[at]), kv, pos), rv = rk + c.pt;
    const uint2 kc = live ? *reinterpret_cast<const uint2*>(c.codes + rk * h + ch) : make_uint2(0, 0);
    const uint2 vc = live ? *reinterpret_cast<const uint2*>(c.codes + rv * h + ch) : make_uint2(0, 0);
    const float ks = c.scales[rk], vs = c.scales[rv];
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(q[j], (float)(int8_t)((j < 4 ? kc.x : kc.y) >> (8 * (j & 3))), s);
    s = kv8_sum_of(s, L) * ks;
    if (t0 + sub >= hi) continue;
    const float to = fmaxf(r.m, s), alpha = exp2f(r.m - to), p = exp2f(s - to), w = p * vs;
    r.m = to;
    r.l = r.l * alpha + p;
#pragma unroll
    for (int j = 0; j < 8; ++j) r.o[j] = r.o[j] * alpha + w * (float)(int8_t)((j < 4 ? vc.x : vc.y) >> (8 * (j & 3)));
  }
  for (int off = L; off < 64; off <<= 1) {
    const float m1 = __shfl_xor(r.m, off, 64), l1 = __shfl_xor(r.l, off, 64), to = fmaxf(r.m, m1), a0 = exp2f(r.m - to), a1 = exp2f(m1 - to);
    r.l = r.l * a0 + l1 * a1;
#pragma unroll
    for (int j = 0; j < 8; ++j) r.o[j] = r.o[j] * a0 + __shfl_xor(r.o[j], off, 64) * a1;
    r.m = to;
  }
  return r;
}

}  // namespace mdi
