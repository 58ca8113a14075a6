// What the kernels of packed rows over the bf16 cache share (kv_prompt.hip, kv_prompt_wide.hip).
#pragma once

#include "kv8_mfma.h"
#include "kv_blocks.h"
#include "kv_device.h"
#include "kv_prompt_wide.h"

namespace mdi {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4* lds_i16x4;
typedef __attribute__((address_space(3))) u32x4* lds_u32x4;

constexpr int BK = 64;               // keys of a step
// Weights are counted from a reference of their row, the largest score of the first block that the row sees; it is raised only
// when a block's weights sum to more than this: weights of any size keep their digits in their operands and in the sums, which are divided
// out at the end.  So no maximum is looked for where nothing is raised.
constexpr float kMostSum = 0x1p16f;
// Weights above the reference make sums larger than values are.  From 2^118 on they are not taken: two groups and 32 pieces of smaller ones stay
// within the range, and kv_attend's weights are at most 1.
constexpr float kTooLarge = 0x1p10f;

__device__ __forceinline__ u32x2 read_transposed(uint32_t at) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(uintptr_t)at));
}
__device__ __forceinline__ u32x4 read_lds(uint32_t at) { return *(lds_u32x4)(uintptr_t)at; }
// 64 x 16 bytes global -> LDS: lane l's piece lands at lds + 16 l.
__device__ __forceinline__ void dma(uint32_t lds, const void* base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "m0", "memory");
}
__device__ __forceinline__ void dma(uint32_t lds, const void* p) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p) : "m0", "memory");
}
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// The blocks of 64 positions that some row of a workgroup sees, its first row at position `at`, `end` behind its last: those
// of the first positions, then from the one that the first row's window begins in.
struct KvBlocks { int sinks, n_sinks, first, from, end, n; };
__device__ __forceinline__ KvBlocks kv_blocks(const KvSight& w, int at, int end) {
  KvBlocks b;
  b.end = end;
  b.from = max(at + 1 - w.window, 0);
  b.sinks = min(w.sinks, b.from);
  const int s64 = (b.sinks + 63) >> 6, f64 = b.from >> 6;
  b.n_sinks = s64 < f64 ? s64 : 0;
  b.first = b.n_sinks || b.sinks == 0 ? f64 << 6 : 0;
  b.n = b.n_sinks + ((end - b.first + 63) >> 6);
  return b;
}



// What a row at distance `up_to` behind the first of 32 keys sees of them, a bit a key; `stay` of them are among the first positions.
__device__ __forceinline__ uint32_t lowest(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }
__device__ __forceinline__ uint32_t seen_keys(int up_to, int window, int stay) { return lowest(up_to + 1) & (~lowest(up_to - window + 1) | lowest(stay)); }
// A score, or -inf where bit `key` says so.
__device__ __forceinline__ float masked(float s, uint32_t seen, int key) {
  const uint32_t all = (uint32_t)__builtin_amdgcn_sbfe((int)seen, key, 1);
  return __uint_as_float((__float_as_uint(s) & all) | (0xFF800000u & ~all));
}

// A lane's weights of 16 N keys as two operands of the second product each: rounded to bf16, and what that leaves, rounded again, which
// is sixteen digits of a weight.  (One alone would be off by as much as the rounding of the result.)
template <int N> struct PromptWeights {
  u32x4 upper[N], lower[N];
  __device__ __forceinline__ void put(int e, float w0, float w1) {   // weights e and e + 1, e even
    uint32_t up = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)w0, (__bf16)w1});
    asm("" : "+v"(up));                                          // (else each half is worked out once more)
    upper[e >> 3][(e & 7) >> 1] = up;
    lower[e >> 3][(e & 7) >> 1] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)(w0 - __uint_as_float(up << 16)), (__bf16)(w1 - __uint_as_float(up & 0xFFFF0000u))});
  }
};

// What a workgroup's rows are, and the blocks they see.
struct PromptRows {
  BlockPlace at;
  int g_sh, head0, kv, q0, p0;       // heads side by side: 2^g_sh from head0 on; the first row, counted in its sample; the sample's first position
  const int32_t* table;
  KvBlocks kb;
  int piece, b_lo, b_hi, pieces;
};

// Rows whose sums were spoiled, each by a wavefront by itself.
template <int HD>
__device__ __forceinline__ void prompt_again(const KvCache& c, const KvRows& r, const KvAttn& a, const PromptRows& w, int rows, int waves) {
  constexpr int L = HD / 8;
  const int lane = threadIdx.x & 63, ch = 8 * (lane & (L - 1));
  for (int i = threadIdx.x >> 6; i < rows; i += waves) {         // a wavefront takes a row and head
    const int row = w.q0 + (i >> w.g_sh), head = w.head0 + (i & ((1 << w.g_sh) - 1)), item = (w.at.first + row) * a.H + head;
    if (row >= w.at.rows) continue;
    const int end = (int)min((long)w.p0 + row + 1, (long)r.max_ctx), from = max(end - a.sight.window, 0), shift = w.kb.first - 64 * w.kb.n_sinks;
    const KvSpan span{min(a.sight.sinks, from), 64 * w.kb.n_sinks, shift, from, end};
    float q[8];
    KvType<bf16_t>::load8((const bf16_t*)a.q + (long)(w.at.first + row) * a.q_stride + (long)head * HD + ch, q);
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] *= a.scale;
    const KvSums sums = kv_attend<bf16_t>(c, w.table, w.kv, span, q, L, ch, true, 64 * w.b_lo, 64 / L, min(64 * w.b_hi, end - shift));
    if (lane >= L) continue;
    bf16_t* const out = (bf16_t*)a.out + (long)(w.at.first + row) * a.out_stride + (long)head * HD + ch;
    float* const part = kv_part_sums(a, c, item, w.piece) + ch;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (w.pieces == 1) out[e] = f32_to_bf16(sums.o[e] / sums.l);
      else part[e] = sums.o[e];
    if (lane == 0 && w.pieces > 1) *kv_part_marks(a, c, r, item, w.piece) = make_float2(sums.m, sums.l);
    if (lane == 0 && w.piece == 0 && a.plan.splits > 1) kv_part_counts(a, c, r)[item] = w.pieces;
  }
}

// A lane's row and head, channels 32 i + 8 g + 4 (lane / 32) + 0..3 in o[i][4 g ..]: the result, or a piece of it.
template <int HT>
__device__ __forceinline__ void prompt_store(const KvCache& c, const KvRows& r, const KvAttn& a, const PromptRows& w, int row, int head, const f32x16 (&o)[HT], float m, float l) {
  const int half = (threadIdx.x >> 5) & 1, item = (w.at.first + row) * a.H + head;
  if (a.plan.splits > 1 && w.piece == 0 && half == 0) kv_part_counts(a, c, r)[item] = w.pieces;
  if (w.pieces == 1) {
    bf16_t* const out = (bf16_t*)a.out + (long)(w.at.first + row) * a.out_stride + (long)head * (32 * HT);
    const float inv = 1.f / l;
#pragma unroll
    for (int i = 0; i < HT; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const uint32_t w0 = (uint32_t)f32_to_bf16(o[i][4 * g] * inv) | ((uint32_t)f32_to_bf16(o[i][4 * g + 1] * inv) << 16);
        const uint32_t w1 = (uint32_t)f32_to_bf16(o[i][4 * g + 2] * inv) | ((uint32_t)f32_to_bf16(o[i][4 * g + 3] * inv) << 16);
        *reinterpret_cast<u32x2*>(out + 32 * i + 8 * g + 4 * half) = u32x2{w0, w1};
      }
  } else {
    float* const part = kv_part_sums(a, c, item, w.piece);
#pragma unroll
    for (int i = 0; i < HT; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(part + 32 * i + 8 * g + 4 * half) = f32x4{o[i][4 * g], o[i][4 * g + 1], o[i][4 * g + 2], o[i][4 * g + 3]};
    if (half == 0) *kv_part_marks(a, c, r, item, w.piece) = make_float2(m, l);
  }
}

// A lane's row of a sample that takes no part.
template <int HT>
__device__ __forceinline__ void prompt_zeros(const KvCache& c, const KvRows& r, const KvAttn& a, const BlockPlace& at, int row, int head) {
  const int half = (threadIdx.x >> 5) & 1;
  bf16_t* const out = (bf16_t*)a.out + (long)(at.first + row) * a.out_stride + (long)head * (32 * HT);
#pragma unroll
  for (int i = 0; i < HT; ++i)
#pragma unroll
    for (int g = 0; g < 4; ++g) *reinterpret_cast<u32x2*>(out + 32 * i + 8 * g + 4 * half) = u32x2{0, 0};
  if (a.plan.splits > 1 && half == 0) kv_part_counts(a, c, r)[(at.first + row) * a.H + head] = 1;
}

}  // namespace
}  // namespace mdi
