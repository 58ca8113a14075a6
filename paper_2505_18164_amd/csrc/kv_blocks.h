// Packed rows of many samples in blocks of workgroups (kv8_prompt.hip, kv_prompt.hip): which sample's rows a workgroup has, worked out from
// `start` on the device, so the host knows only a bound of the grid.
#pragma once

#include "kv8_device.h"
#include "kv_plan.h"

namespace mdi {

// Rows of sample i, 0 <= first <= end <= n_rows whatever `start` holds.
struct Span { int first, end; };
__device__ __forceinline__ Span kv_rows_of(const Kv8Rows& r, int i) {
  const int first = min(max(r.start[i], 0), r.n_rows);
  return Span{first, min(max(r.start[i + 1], first), r.n_rows)};
}

// The sample that has block x, counting bp positions a block, a power of two, and which of its blocks that is; sample < 0: nobody's.
// Up to kInOrder samples' blocks follow one another without a gap, which takes a sum over the samples before.  Of more, sample i's
// start at first_i / bp + min(i, first_i) - rows before it, and samples that may have rows -, which leaves each as many as its
// rows need and up to one over; there the sample is searched for.  Dense / searched, us: 257 samples of up to 64 rows of 20 heads on
// one 70 / 75, 300 of up to 30 of the 8B shape 107 / 108, 600 of up to 20 of TinyLlama 101 / 78, 2000 of up to 10 of the 8B shape
// 1101 / 601.  (What is over costs where the chip is just full: 4 pieces of 64 behind 8000 of the 8B shape, 256 workgroups, 60 us, with as
// many empty ones between them 96.  Two kernels, because in one that has both the long prompts take 427 us instead of 414.)
struct BlockPlace { int sample, block, first, rows, pos, table; };
template <bool kMany> __device__ __forceinline__ BlockPlace place_of(const Kv8Rows& r, int x, int bp) {
  const int lane = threadIdx.x & 63;
  if constexpr (!kMany) {
    for (int base = 0, sum = 0; base < r.n; base += 64) {
      const int i = min(base + lane, r.n - 1), pos = r.pos[i], table = r.table ? r.table[i] : i;   // (asked for along with the rows)
      const Span s = base + lane < r.n ? kv_rows_of(r, i) : Span{0, 0};
      const int t = (s.end - s.first + bp - 1) / bp;
      int up = t;
      for (int off = 1; off < 64; off <<= 1) { const int o = __shfl_up(up, off, 64); if (lane >= off) up += o; }
      const unsigned long long past = __ballot(sum + up > x);
      if (past) {
        const int at = __ffsll(past) - 1;
        return BlockPlace{__builtin_amdgcn_readfirstlane(base + at), __builtin_amdgcn_readfirstlane(x - (sum + __shfl(up - t, at, 64))),
                          __builtin_amdgcn_readfirstlane(__shfl(s.first, at, 64)), __builtin_amdgcn_readfirstlane(__shfl(s.end - s.first, at, 64)),
                          __builtin_amdgcn_readfirstlane(__shfl(pos, at, 64)), __builtin_amdgcn_readfirstlane(__shfl(table, at, 64))};
      }
      sum += __shfl(up, 63, 64);
    }
  } else {
    auto starts = [&](int i, int first) { return first / bp + min(i, first); };
    const Kv8Window w = kv8_window(r.n, [&](int i) { return starts(i, kv_rows_of(r, i).first) <= x; });
    const int i = w.base + min(lane, max(w.len - 1, 0)), pos = r.pos[i], table = r.table ? r.table[i] : i;
    const Span s = kv_rows_of(r, i);
    const int from = starts(i, s.first), at = __popcll(__ballot(lane < w.len && from <= x)) - 1;
    if (at >= 0) {
      const int block = __builtin_amdgcn_readfirstlane(x - __shfl(from, at, 64)), rows = __builtin_amdgcn_readfirstlane(__shfl(s.end - s.first, at, 64));
      if (block >= 0 && block < (rows + bp - 1) / bp)
        return BlockPlace{__builtin_amdgcn_readfirstlane(w.base + at), block, __builtin_amdgcn_readfirstlane(__shfl(s.first, at, 64)), rows,
                          __builtin_amdgcn_readfirstlane(__shfl(pos, at, 64)), __builtin_amdgcn_readfirstlane(__shfl(table, at, 64))};
    }
  }
  return BlockPlace{-1, 0, 0, 0, 0, 0};
}

}  // namespace mdi
