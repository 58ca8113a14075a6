// Device-side parts of the cache in the storage type that its kernels share: what a row sees, where the pieces of a row lie.
#pragma once

#include "kv8_device.h"
#include "kv_internal.h"

namespace mdi {

template <typename T> struct KvType;
template <> struct KvType<bf16_t> {
  __device__ static __forceinline__ void load8(const bf16_t* p, float (&x)[8]) { Storage<bf16_t>::load(p, x); }
};
template <> struct KvType<float> {
  __device__ static __forceinline__ void load8(const float* p, float (&x)[8]) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
};

// The positions that a row at position end - 1 sees, [0, sinks) and [from, end), counted without the gap between: place c is position
// c of the first sinks16, then c + shift.  Both parts begin at multiples of 16, so that sixteen places from such a multiple
// on are positions next to each other; places that are no visible position lie only in front of `from` and behind `sinks`.
struct KvSpan {
  int sinks, sinks16, shift, from, end;
  __device__ __forceinline__ int places() const { return end - shift; }
  __device__ __forceinline__ int position(int c) const { return c + (c >= sinks16 ? shift : 0); }
  __device__ __forceinline__ bool sees(int pos) const { return pos < sinks || (pos >= from && pos < end); }
};
__device__ __forceinline__ KvSpan kv_span(const KvSight& w, int end) {   // end: at most 2^30
  KvSpan s;
  s.end = end;
  s.from = max(end - w.window, 0);
  s.sinks = min(w.sinks, s.from);
  const int s16 = (s.sinks + 15) & ~15, b16 = s.from & ~15;
  const bool apart = s16 < b16;
  s.sinks16 = apart ? s16 : 0;
  s.shift = apart ? b16 - s16 : 0;
  return s;
}

// The workspace: sums of every item (row * H + head) and piece, then their references and sums of weights, then how many pieces an item has.
__device__ __forceinline__ float* kv_part_sums(const KvAttn& a, const KvPages& c, int item, int piece) {
  return a.part + ((long)item * a.plan.splits + piece) * c.h;
}
__device__ __forceinline__ float2* kv_part_marks(const KvAttn& a, const KvPages& c, const KvRows& r, int item, int piece) {
  return reinterpret_cast<float2*>(a.part + (long)r.n_rows * a.H * a.plan.splits * c.h) + (long)item * a.plan.splits + piece;
}
__device__ __forceinline__ int* kv_part_counts(const KvAttn& a, const KvPages& c, const KvRows& r) {
  return reinterpret_cast<int*>(a.part + (long)r.n_rows * a.H * a.plan.splits * (c.h + 2));
}

// How many places the newest row of a sample sees (one new token per sample); 0: it takes no part.
__device__ __forceinline__ int kv_places(const KvPages& c, const KvRows& r, const KvSight& w, int sample) {
  const int seen = kv8_seen(c, r, sample);
  return seen ? kv_span(w, seen).places() : 0;
}

constexpr float kKvNone = -3e38f;    // reference of a softmax that has seen nothing

// One row and head by a wavefront, for any head: L lanes hold eight channels each of a position (`ch` on, `live` where the head has
// them), the lane groups take places lo + first, + 1 .. and `step` further, up to hi.  A lane group keeps its own running (reference,
// sum, output), which are folded at the end: every lane then has the sums of its eight channels.  Everything is binary32, with no
// other reference than the largest score so far, and nothing is multiplied that the row does not see.
struct KvSums { float m, l, o[8]; };
template <typename T>
__device__ __forceinline__ KvSums kv_attend(const KvCache& c, const int32_t* table, int kv, const KvSpan& span, const float (&q)[8], int L, int ch,
                                            bool live, int from, int step, int hi) {
  const int sub = (threadIdx.x & 63) / L, h = c.h;
  KvSums r{kKvNone, 0.f, {}};
  for (int t0 = from; t0 < hi; t0 += step) {
    const int place = t0 + sub, pos = span.position(min(place, hi - 1));
    const bool seen = place < hi && span.sees(pos);
    float s = 0.f, v[8] = {};
    if (seen) {
      const long row = kv8_row(c, kv8_checked_page(c, table[kv8_page_of(c, pos)]), kv, pos);
      if (live) {
        float k[8];
        KvType<T>::load8((const T*)c.data + row * h + ch, k);
        KvType<T>::load8((const T*)c.data + (row + c.pt) * h + ch, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) s = fmaf(q[j], k[j], s);
      }
    }
    s = kv8_sum_of(s, L);
    if (!seen) continue;
    const float to = fmaxf(r.m, s), alpha = exp2f(r.m - to), p = exp2f(s - to);
    r.m = to;
    r.l = r.l * alpha + p;
#pragma unroll
    for (int j = 0; j < 8; ++j) r.o[j] = r.o[j] * alpha + p * v[j];
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
