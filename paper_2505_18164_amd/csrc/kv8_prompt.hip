// Causal attention of packed rows - prompts, or the next pieces of prompts, of several samples - over the 8-bit cache, on the
// matrix cores.
//
// A workgroup takes 32 rows of (position, query head) for each of its wavefronts, the heads of one kv head side by side, and passes
// over the keys they see 64 at a time.  A wavefront computes S^T = K Q^T with v_mfma_f32_32x32x16 (codes are exact in bf16; a key's
// scale, the softmax's and log2 e multiply the scores in fp32), weighs them against a reference that is near the row's largest
// score, and adds O^T += V^T P^T: the scores of a query lie in the lane, and in the order, in which the second product takes weights,
// so they never leave the registers.  The workgroup turns each block's codes into bf16 keys and fp16 values once, in the LDS.
// Which sample a workgroup belongs to it works out from `start`, 64 samples at a time, so the host knows only a bound of the grid.
//
// What bounds it, long prompts: 6000 + 2000 + 500 rows of the 8B shape take 410 to 440 us = 0.75 to 0.81 PFLOP/s, where a large matrix product
// reaches 1.19 on the same card.  A block of 128 channels takes 2.15 us, some 4700 cycles, in which a SIMD's matrix core works 2048
// for its two wavefronts; the vector unit works a little longer on their 4096 scores (product with the scale, largest, exponential,
// conversion: four and a half instructions each, on 64 at a time, of 4.5 cycles) and on the codes, and the LDS delivers
// 32 KB of operands to each wavefront.  Counted: of the time that a compute unit has work its matrix cores are busy 38 %, its vector
// units 45 %, its LDS 34 % (14 % of that bank conflicts).  No one of them is the limit; that two turns do not overlap further is.  Three choices follow.  The wavefronts of a SIMD take turns - one multiplies and stages
// while the other takes exponentials -, with two barriers a block.  Operands are read one set of four ahead of their products.  A
// block's codes are asked for a whole block before they are staged.  More wavefronts on a SIMD instead, which have to do with 128
// registers, cost more in spills than they hide (8 prompts of TinyLlama 56 -> 82 us).
// Short prompts: a block after the other.  1024 rows of the 7B shape are 256 workgroups, one for each compute unit, of which the
// longest passes over 16 blocks: two groups of wavefronts take half of the blocks each (45 -> 32 us); six us are the way to the first
// block - rows, page numbers, codes, each behind the one before.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kv8_mfma.h"
#include "kv_blocks.h"
#include "once_per_device.h"

namespace mdi {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int BK = 64;               // keys of a step
// Weights and values are multiplied as fp16, which has three more digits than bf16 (with bf16 the results were off by 0.0026 of
// their size, of which their own rounding is 0.0017) and a smaller range.  Weights are counted so that the largest of a row's first
// block is 2^kTop, and counted anew when one would exceed 2^kRaise; one below 2^-14 keeps the digits down to 2^-24, 2^-30 of the
// largest.  Values are multiplied by a power of two, so far that a row's largest magnitude is at most 2^13 where that is
// chosen, and up to 2^15 before it is chosen anew.  That serves rows of values whose sizes are within 2^20 of each other: the smallest
// has a scale of 2^-14 then, so that every value is a normal fp16.  The unit is that of whatever the workgroup has met, seen by
// all of its rows or by a few; so a workgroup that meets sizes further apart (scale below kLeastScale) computes its rows over
// again, each by itself, in binary32 (kv8_attend): 1024 rows of the 7B shape of which one value is 2^40 times the others' size 2.4 ms
// instead of 34 us.
constexpr float kTop = 6.f, kFromTop = 0x1p-6f, kRaise = 14.f;
constexpr float kUnitFirst = 0x1p100f;                           // scales are zero, or 2^-107 and more
constexpr float kLeastScale = 0x1p-14f;
// Scores are rounded as distances from the row's reference.  When that is raised the block's own are rounded at its distance: up to
// kFar, by 2^-15 at most.  From further below (keys that count for nothing before those that decide) they would lose their digits,
// 11 % of a weight at 10^7, so there too the workgroup computes its rows over again.
constexpr float kFar = 1024.f;

__device__ __forceinline__ float reciprocal(float power_of_two) { return __uint_as_float(0x7F000000u - __float_as_uint(power_of_two)); }

__device__ __forceinline__ u32x2 read_transposed(const bf16_t* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)p));
}

struct PromptGeo { int n_blocks, sets, g_sh, from; };            // bound of the blocks of all samples; sets of 2^g_sh query heads; of the launch's first workgroup

// A workgroup is eight wavefronts: NG groups of WQ, which work on the same 32 WQ rows; group g takes the key blocks NG i + g.
// kWhole: pages of a multiple of 64 positions, so that a block of keys lies in one.  kMany: of more than kInOrder samples.
template <int HD, int NG, bool kWhole, bool kMany>
__global__ __launch_bounds__(512, 2) void k_kv8_prompt(Kv8Cache c, Kv8Rows r, Kv8Attn a, PromptGeo geo) {
  constexpr int WQ = 8 / NG, BQ = 32 * WQ, GT = 64 * WQ;         // rows of a workgroup - (position, head) pairs -, threads of a group
  constexpr int KS = HD + 8, VR = HD + 32, HT = HD / 32;
  constexpr int UB = 64 * HD / GT < 16 ? 64 * HD / GT : 16;      // codes a thread moves at a time
  constexpr int KU = 64 * HD / (GT * UB), PER = HD / UB;         // ... and how often; threads a key
  constexpr int NB = 2;                                          // buffers of keys, and of values
  constexpr int KV = NB * BK * (KS + VR) + 8 * BK + 8;           // 16-bit elements of a group: keys, values, scales of four blocks of keys, units of four blocks of values
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  __shared__ int again[NG];                                      // a group met what these numbers do not hold

  const int tid = threadIdx.x & (GT - 1), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = NG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / GT), late = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
  bf16_t* const Kb = (bf16_t*)smem + grp * KV;
  bf16_t* const Vb = Kb + NB * BK * KS;
  float* const Sc = (float*)(Vb + NB * BK * VR);                 // [4][64]
  float* const Un = Sc + 4 * BK;                                 // [4]
  // A sample's longest rows first, and of those all sets.  (Workgroups are handed to the eight compute dies, each with an L2 of its
  // own, in turn: with a multiple of eight sets, a set stays on its die.)
  const int x = kMany ? geo.from + blockIdx.x : blockIdx.x, block = x / geo.sets, set = x - block * geo.sets;
  const BlockPlace at = place_of<kMany>(r, block, BQ >> geo.g_sh);
  if (at.sample < 0) return;
  const int g_sh = geo.g_sh, bp = BQ >> g_sh, head0 = set << g_sh, kv = head0 / (a.H / c.K);
  const int q0 = ((at.rows + bp - 1) / bp - 1 - at.block) * bp;  // first row of the sample in this block
  const int p0 = at.pos, which = p0 < 0 ? -1 : kv8_checked_row(c, at.table);
  const int32_t* table = c.tables + (long)max(which, 0) * c.table_stride;
  const int col = lane & 31, half = lane >> 5;
  const int row = q0 + ((32 * wave + col) >> g_sh), head = head0 + (col & ((1 << g_sh) - 1));   // (32 is a multiple of 2^g_sh)
  const bool live = row < at.rows;
  bf16_t* out = a.out + (long)(at.first + row) * a.out_stride + (long)head * HD;
  if (which < 0) {                                               // takes no part
    if (blockIdx.y == 0 && grp == 0 && live)
#pragma unroll
      for (int i = 0; i < HT; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) *reinterpret_cast<u32x2*>(out + 32 * i + 8 * g + 4 * half) = u32x2{0, 0};
    return;
  }
  // positions up to `pos` are seen by this lane's row; n_keys: what the block's last row sees
  const long far = (long)p0 + min(q0 + bp, at.rows);
  if (far > r.max_ctx) kv8_report(c);
  const int n_seen = (int)min(far, (long)r.max_ctx), pos = (int)min((long)p0 + min(row, at.rows - 1), (long)r.max_ctx - 1);
  const int lo = blockIdx.y * a.plan.chunk, hi = (int)min((long)n_seen, (long)lo + a.plan.chunk);
  if (lo >= hi) return;

  bf16x8 qf[HD / 16];
  f32x16 o[HT];
#pragma unroll
  for (int i = 0; i < HT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  float m = 0.f, l = 0.f;
  bool first = true;                                             // no block yet: scores are counted from zero
  const int wave_pos = (int)min((long)p0 + q0 + ((32 * wave) >> g_sh), (long)r.max_ctx - 1);   // of the wavefront's first row

  // Staging.  A thread moves UB channels of KU keys: those of block j along with the values of block j - 1.
  const int n_kb = (hi - lo + BK - 1) / BK, n_it = (n_kb + NG - 1) / NG;
  u32x4 kreg[KU], vreg[KU];
  float vs[KU], sk = 0.f, sv = 0.f;
  float unit = kUnitFirst, made = kUnitFirst, mine = kUnitFirst;  // of the block whose values are staged; newest that was chosen; of o
  float least = INFINITY;                                        // of the scales that this lane has met, but zeros (the group's first wavefront looks at them)
  unsigned worst = 0;                                            // a page that is not of the cache is looked for at the end, the last one read in its place
  auto checked = [&](int page) __attribute__((always_inline)) {
    worst = max(worst, (unsigned)page);
    return min((unsigned)page, (unsigned)c.n_pages - 1);
  };
  auto block_at = [&](int j) __attribute__((always_inline)) { return lo + (NG * j + grp) * BK; };
  auto take = [&](const char* codes, uint32_t off) __attribute__((always_inline)) {
    if constexpr (UB == 16) return *reinterpret_cast<const u32x4*>(codes + off);
    const u32x2 x = *reinterpret_cast<const u32x2*>(codes + off);
    return u32x4{x.x, x.y, 0, 0};
  };
  // fetch(j) asks for block j's keys and block j - 1's values (whose places it was left by the one before) and for block j + 1's page numbers.
  int pg[kWhole ? 1 : KU + 1];
  long k_row[kWhole ? 1 : KU] = {};                              // rows of the cache
  int k_last = 0;                                                // positions of the block but the first
  auto pages = [&](int j) __attribute__((always_inline)) {
    if constexpr (kWhole) {
      int at = kv8_page_of(c, min(block_at(j), hi - 1));
      asm volatile("" : "+v"(at));                               // a vector load: behind a scalar one every read of LDS would have to wait for it
      pg[0] = table[at];
    } else {
#pragma unroll
      for (int u = 0; u <= KU; ++u) pg[u] = table[kv8_page_of(c, min(block_at(j) + (u < KU ? (tid + u * GT) / PER : lane), hi - 1))];
    }
  };
  auto fetch = [&](int j) __attribute__((always_inline)) {
    const int k0 = min(block_at(j), hi - 1);                     // keys past the last repeat it
    if constexpr (kWhole) {
      const long v_row = k_row[0] + c.pt;
      const int v_last = k_last;
      k_row[0] = kv8_row(c, __builtin_amdgcn_readfirstlane((int)checked(pg[0])), kv, k0);
      k_last = min(BK, hi - k0) - 1;
      const char* const kp = (const char*)c.codes + k_row[0] * HD;
      const char* const vp = (const char*)c.codes + v_row * HD;
#pragma unroll
      for (int u = 0; u < KU; ++u) {
        const int at = tid + u * GT, key = at / PER, ch = UB * (at % PER);
        kreg[u] = take(kp, (uint32_t)(min(key, k_last) * HD + ch));
        if (j > 0) {
          vreg[u] = take(vp, (uint32_t)(min(key, v_last) * HD + ch));
          vs[u] = *reinterpret_cast<const float*>((const char*)(c.scales + v_row) + 4u * min(key, v_last));
        }
      }
      if (wave == 0) {
        const char* const sp = (const char*)(c.scales + k_row[0]);
        const uint32_t off = 4u * min(lane, k_last);
        sk = *reinterpret_cast<const float*>(sp + off);
        sv = *reinterpret_cast<const float*>(sp + 4l * c.pt + off);
      }
    } else {
#pragma unroll
      for (int u = 0; u < KU; ++u) {
        const int at = tid + u * GT, ch = UB * (at % PER);
        const long v_row = k_row[u] + c.pt;
        k_row[u] = kv8_row(c, checked(pg[u]), kv, min(block_at(j) + at / PER, hi - 1));
        kreg[u] = take((const char*)c.codes + k_row[u] * HD, ch);
        if (j > 0) {
          vreg[u] = take((const char*)c.codes + v_row * HD, ch);
          vs[u] = c.scales[v_row];
        }
      }
      if (wave == 0) {
        const long row = kv8_row(c, checked(pg[KU]), kv, min(block_at(j) + lane, hi - 1));
        sk = c.scales[row];
        sv = c.scales[row + c.pt];
      }
    }
    pages(j + 1);
  };
  // What has been asked for is looked at here and not before: a shift that is moved up to the load waits for it there.
  auto here = [](uint32_t w) __attribute__((always_inline)) { asm volatile("" : "+v"(w)); return w; };
  constexpr int kUnits = UB / 8 * KU;                            // eight codes of a key each
  auto stash_keys = [&](int j, int n) __attribute__((always_inline)) {
    const int u = n / (UB / 8), h = n % (UB / 8), at = tid + u * GT;
    const uint32_t w0 = here(kreg[u][2 * h]), w1 = here(kreg[u][2 * h + 1]);
    *reinterpret_cast<u32x4*>(Kb + (j & 1) * BK * KS + at / PER * KS + UB * (at % PER) + 8 * h) =
        u32x4{high_halves(code_of<0>(w0), code_of<1>(w0)), high_halves(code_of<2>(w0), code_of<3>(w0)),
              high_halves(code_of<0>(w1), code_of<1>(w1)), high_halves(code_of<2>(w1), code_of<3>(w1))};
  };
  auto stash_values = [&](int j, int n) __attribute__((always_inline)) {
    const int u = n / (UB / 8), h = n % (UB / 8), at = tid + u * GT;
    const float f = __uint_as_float(here(__float_as_uint(vs[u]))), by = f - f == 0.f ? f * unit : 0.f;
    const uint32_t w0 = here(vreg[u][2 * h]), w1 = here(vreg[u][2 * h + 1]);
    *reinterpret_cast<f16x8*>(Vb + ((j - 1) & 1) * BK * VR + at / PER * VR + UB * (at % PER) + 8 * h) =
        f16x8{(_Float16)(code_of<0>(w0) * by), (_Float16)(code_of<1>(w0) * by), (_Float16)(code_of<2>(w0) * by), (_Float16)(code_of<3>(w0) * by),
              (_Float16)(code_of<0>(w1) * by), (_Float16)(code_of<1>(w1) * by), (_Float16)(code_of<2>(w1) * by), (_Float16)(code_of<3>(w1) * by)};
  };
  auto stash_scales = [&](int j) __attribute__((always_inline)) {
    const float v = __uint_as_float(here(__float_as_uint(sv)));
    if (wave == 0) {
      const bool fine = v - v == 0.f;
      Sc[64 * (j & 3) + lane] = fine ? sk * a.scale : __uint_as_float(0x7FC00000u);   // a value that is not finite makes its weight NaN (and is staged as zeros)
      if (__builtin_expect(__any(v * made > 256.f), 0)) {
        float top = fine ? v : 0.f;
        for (int off = 32; off; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
        if (top * made > 256.f) made = __uint_as_float((127 + 5 + 127 - (__float_as_uint(top) >> 23)) << 23);   // top is less than 2^6 of these
      }
      if (v > 0.f) least = fminf(least, v);
      if (lane == 0) Un[j & 3] = made;
    }
  };

  const int v_lane = (4 * half + ((lane & 15) >> 2)) * VR + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  const int last_pos = min(wave_pos + (31 >> g_sh), n_seen - 1);
  auto sees = [&](int j) __attribute__((always_inline)) { return NG * j + grp < n_kb && lo + (NG * j + grp) * BK <= last_pos; };   // some row of the wavefront, some key of the block
  f32x16 s[2];
  u32x4 pf[4] = {};                                              // weights, two a word
  // The products of a step: the values of block j - 1 with its weights, the keys of block j with the queries.  Four operands are
  // on their way from the LDS while the four before them are multiplied.
  auto products = [&](int j, auto keys) __attribute__((always_inline)) {
    constexpr int kSets = decltype(keys)::value ? 2 * HT : HT;   // sets of four operands: HT of values, HT of keys
    const bf16_t* const V = Vb + ((j - 1) & 1) * BK * VR + v_lane;
    const bf16_t* const K = Kb + (j & 1) * BK * KS + col * KS + 8 * half;
    if constexpr (decltype(keys)::value) unit = Un[j & 3];
    u32x4 f[2][4];
    auto read = [&](int n) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if (n < HT) {
          const bf16_t* const at = V + 16 * ((4 * n + x) / HT) * VR + 32 * (x % HT);
          const u32x2 b0 = read_transposed(at), b1 = read_transposed(at + 8 * VR);
          f[n & 1][x] = u32x4{b0.x, b0.y, b1.x, b1.y};
        } else {
          f[n & 1][x] = *reinterpret_cast<const u32x4*>(K + 32 * (x & 1) * KS + 16 * (2 * (n - HT) + (x >> 1)));
        }
      }
    };
    read(0);
#pragma unroll
    for (int n = 0; n < kSets; ++n) {
      if (n + 1 < kSets) read(n + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if (n < HT) {
          o[x % HT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, f[n & 1][x]), __builtin_bit_cast(f16x8, pf[(4 * n + x) / HT]), o[x % HT], 0, 0, 0);
        } else {
          const int k = 2 * (n - HT) + (x >> 1);
          s[x & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f[n & 1][x]), qf[k], k ? s[x & 1] : f32x16{}, 0, 0, 0);
        }
      }
      if constexpr (decltype(keys)::value) {                     // staging, in between
        constexpr int kPer = (kUnits + HT - 1) / HT;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const int x = n % HT * kPer + i;
          if (x < kUnits) { if (n < HT) stash_keys(j + 1, x); else stash_values(j + 1, x); }
        }
        if (n == 2 * HT - 1) { stash_scales(j + 1); fetch(j + 2); }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // The weights of block j from its scores.  They are counted from m, the row's reference, which is the largest score of the first
  // block and is raised - in both lanes of a row alike - when a weight would exceed 2^kRaise: the sum is divided out at
  // the end, so any reference near the largest score does.  The sum takes the weights as they are multiplied, cut to
  // fp16 (by the conversion that is 2 us of 58 faster than the one to the nearest: eight prompts of TinyLlama).
  float alpha = 1.f, rise = 0.f;                                 // rise: the furthest a reference was raised (kept here: a store where it is raised costs 3 % of a long call)
  bool raised = false;
  auto weigh = [&](int j, auto mask) __attribute__((always_inline)) {
    constexpr bool kMask = decltype(mask)::value;                // some of these keys are not for some of the rows
    const int pos_in = min(pos, hi - 1) - (lo + (NG * j + grp) * BK) - 4 * half;   // what the lane's row sees of the block
    const float* const sc = Sc + 64 * (j & 3) + 4 * half;
    float top = kKv8None;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 k = *reinterpret_cast<const f32x4*>(sc + 32 * t + 8 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = 4 * g + i;
          s[t][e] = fmaf(s[t][e], k[i], -m);
          if (kMask && 32 * t + 8 * g + i > pos_in) s[t][e] = -INFINITY;
          top = fmaxf(top, s[t][e]);
        }
      }
    if (__builtin_expect(first || __any(top > kRaise), 0)) {
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float by = first ? top - kTop : fmaxf(top - kTop, 0.f);
      rise = fmaxf(rise, first ? 0.f : by);
      alpha = first ? 1.f : exp2_raw(-by);
      raised = !first;
      m += by;
      first = false;
      l *= alpha;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[t][e] -= by;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const f16x2 w = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(exp2_raw(s[t][e]), exp2_raw(s[t][e + 1])));
        l = __builtin_amdgcn_fdot2(w, f16x2{(_Float16)1.f, (_Float16)1.f}, l, false);
        pf[2 * t + (e >> 3)][(e & 7) >> 1] = __builtin_bit_cast(uint32_t, w);
      }
  };
  auto soften = [&](int j) __attribute__((always_inline)) {
    if (!sees(j)) {
#pragma unroll
      for (int t = 0; t < 4; ++t) pf[t] = u32x4{0, 0, 0, 0};
      return;
    }
    const int k0 = lo + (NG * j + grp) * BK;
    if (first) mine = unit;                                      // (the sums are zeros)
    if (k0 + BK - 1 > wave_pos || k0 + BK > hi) weigh(j, std::true_type()); else weigh(j, std::false_type());
    if (__builtin_expect(unit != mine, 0)) {                     // the block's values are counted in another unit than the sums
      alpha = (raised ? alpha : 1.f) * (unit * reciprocal(mine));
      raised = true;
      mine = unit;
    }
  };

  // The wavefronts of a SIMD, w and w + 4, take turns: while one multiplies and stages, the other takes exponentials; so the later
  // four are one turn behind.  Block j + 1's keys and block j's values, which both stage in turn j, go over blocks that both have left.
  pages(0);
  fetch(0);
  {                                                              // (behind the way to the first codes, which is the longer one)
    const bf16_t* qp = a.q + (long)(at.first + min(row, at.rows - 1)) * a.q_stride + (long)head * HD + 8 * half;
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(qp + 16 * ks);
  }
#pragma unroll
  for (int n = 0; n < kUnits; ++n) stash_keys(0, n);
  stash_scales(0);
  fetch(1);
  // (the first step has no values yet: its weights are zeros, and so is what they multiply)
  for (int i = tid; i < BK * VR / 8; i += GT) *reinterpret_cast<u32x4*>(Vb + BK * VR + 8 * i) = u32x4{0, 0, 0, 0};
  if (tid == 0) again[grp] = 0;
  __syncthreads();
  if (late) __syncthreads();
  for (int j = 0; j < n_it; ++j) {
    products(j, std::true_type());
    __syncthreads();
    soften(j);
    if (__builtin_expect(raised, 0)) {
#pragma unroll
      for (int i = 0; i < HT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float x = o[i][e] * alpha;
          asm volatile("" : "+v"(x));                            // (one after the other, in place: else they are copied, and others spilled)
          o[i][e] = x;
        }
      raised = false;
    }
    __syncthreads();
  }
  if (__any(rise > kFar || least * made < kLeastScale)) again[grp] = 1;   // (least and made only fall; a barrier before it is read)
  products(n_it, std::false_type());
  if (!late) __syncthreads();
  __syncthreads();
  if (worst >= (unsigned)c.n_pages) kv8_report(c);
  int over = again[0];
  if constexpr (NG > 1) over |= again[1];
  over = __builtin_amdgcn_readfirstlane(over);
  if (__builtin_expect(over != 0, 0)) {
    constexpr int L = HD / 8;
    const int ch = 8 * (lane & (L - 1));
    for (int i = threadIdx.x >> 6; i < BQ; i += 8) {             // a wavefront takes a row and head
      const int row1 = q0 + (i >> g_sh), head1 = head0 + (i & ((1 << g_sh) - 1));
      if (row1 >= at.rows) continue;
      const int pos1 = (int)min((long)p0 + row1, (long)r.max_ctx - 1);
      if (pos1 < lo) continue;
      const bf16_t* const q1 = a.q + (long)(at.first + row1) * a.q_stride + (long)head1 * HD + ch;
      float q[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) q[e] = bf16_to_f32(q1[e]) * a.scale;
      const Kv8Sums x = kv8_attend(c, table, kv, q, L, ch, true, lo, 64 / L, min(pos1 + 1, hi));
      if (lane >= L) continue;
      if (pos1 < a.plan.chunk) {
        bf16_t* const out1 = a.out + (long)(at.first + row1) * a.out_stride + (long)head1 * HD + ch;
#pragma unroll
        for (int e = 0; e < 8; e += 2)
          *reinterpret_cast<uint32_t*>(out1 + e) = (uint32_t)f32_to_bf16(x.o[e] / x.l) | ((uint32_t)f32_to_bf16(x.o[e + 1] / x.l) << 16);
      } else {
        const int item = (at.first + row1) * a.H + head1;
        float* const part = kv8_part_sums(a, c, item, blockIdx.y) + ch;
#pragma unroll
        for (int e = 0; e < 8; ++e) part[e] = x.o[e];
        if (lane == 0) *kv8_part_marks(a, c, r, item, blockIdx.y) = make_float2(x.m, x.l);
      }
    }
    return;
  }
  // the largest weights count as one again, and the sums in the values' own unit
  m = first ? kKv8None : m + kTop;                               // (first: saw nothing)
  l *= kFromTop;
  const float own = kFromTop * reciprocal(mine);

#pragma unroll
  for (int i = 0; i < HT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] *= own;

  if constexpr (NG > 1) {
    float* fold = (float*)smem + (grp > 0 ? grp - 1 : 0) * (HT * 16 + 2) * GT;
    if (grp > 0) {
#pragma unroll
      for (int i = 0; i < HT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) fold[(i * 16 + e) * GT + tid] = o[i][e];
      fold[(HT * 16) * GT + tid] = m;
      fold[(HT * 16 + 1) * GT + tid] = l;
    }
    __syncthreads();
    if (grp > 0) return;
    for (int g = 1; g < NG; ++g, fold += (HT * 16 + 2) * GT) {
      const float m1 = fold[(HT * 16) * GT + tid], l1 = fold[(HT * 16 + 1) * GT + tid];
      const float to = fmaxf(m, m1), a0 = exp2_raw(m - to), a1 = exp2_raw(m1 - to);
      l = l * a0 + l1 * a1;
      m = to;
#pragma unroll
      for (int i = 0; i < HT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] = o[i][e] * a0 + fold[(i * 16 + e) * GT + tid] * a1;
    }
  }

  l += __shfl_xor(l, 32, 64);
  if (!live || pos < lo) return;                                 // (a row that sees nothing of this piece has no such piece)
  if (pos < a.plan.chunk) {
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
    const int item = (at.first + row) * a.H + head;
    float* part = kv8_part_sums(a, c, item, blockIdx.y);
#pragma unroll
    for (int i = 0; i < HT; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(part + 32 * i + 8 * g + 4 * half) = f32x4{o[i][4 * g], o[i][4 * g + 1], o[i][4 * g + 2], o[i][4 * g + 3]};
    if (half == 0) *kv8_part_marks(a, c, r, item, blockIdx.y) = make_float2(m, l);
  }
}

template <int HD, int NG>
constexpr size_t prompt_lds() {
  const size_t kv = (size_t)NG * (2 * BK * (HD + 8 + HD + 32) + 8 * BK + 8) * sizeof(bf16_t);
  const size_t fold = (size_t)(NG - 1) * (HD / 2 + 2) * (512 / NG) * sizeof(float);
  return kv > fold ? kv : fold;
}
template <int HD, int NG, bool kWhole, bool kMany>
bool allow_one() {                                               // 64 KiB is what a kernel gets by default
  constexpr size_t lds = prompt_lds<HD, NG>();
  return lds <= 64 * 1024 ||
         hipFuncSetAttribute((const void*)k_kv8_prompt<HD, NG, kWhole, kMany>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) == hipSuccess;
}
template <int HD, int NG>
bool allow_groups() {
  return allow_one<HD, NG, true, false>() && allow_one<HD, NG, false, false>() && allow_one<HD, NG, true, true>() && allow_one<HD, NG, false, true>();
}
template <int HD>
bool allow_heads() { return allow_groups<HD, 1>() && allow_groups<HD, 2>(); }

PromptGeo geo_of(const Kv8Cache& c, const Kv8Rows& r, int H, int WQ) {
  const int sh = kv_heads_shift(c, H), bp = 32 * WQ >> sh;
  return PromptGeo{r.n_rows / bp + std::min(r.n, r.n_rows), H >> sh, sh, 0};
}
// Groups of a workgroup and pieces of a row's positions.  A step of 64 NG keys takes `step` us, a workgroup six or seven more to begin
// and end; what is divided is added by a second launch, a wavefront per row and head.  How long the single samples are is on the
// device: they are taken for equal.  Whole calls, us, undivided with 1 / 2 groups: a prompt of 512, 1024, 2048 of the 7B shape
// 28.3/21.8, 45.5/33.8, 81.8/69.9, four of 512 32.5/40.8, sixteen of 64 20.8/24.1, eight of 333 of TinyLlama 27.1/32.4, one of 1500
// 43.9/31.3; four pieces of 64 behind 8000 of the 8B shape 263/161, in 2 parts 144/94, in 4 84/61, in 8 60/74, in 16 77/102; four
// of 128 behind 2000 79/53, 60/50, 47/62; the prompt of 1024 in two parts 43/49.  Of 25 such shapes the rule takes the best of
// these ways for all but four short ones, which it misses by up to 11 % (one us).
struct PromptPlan { int groups, splits; };
PromptPlan prompt_plan(const Kv8Cache& c, const Kv8Rows& r, int H, size_t part_limit) {
  const int n = std::max(1, std::min(r.n, r.n_rows)), rows = (r.n_rows + n - 1) / n;   // of a sample
  const double heads = (double)r.n_rows * H, seen = r.max_ctx - 0.5 * std::min(r.max_ctx, rows);   // what a row sees, on average
  PromptPlan best{1, 1};
  double best_us = 1e30;
  for (int ng = 1; ng <= 2; ++ng) {
    const int sh = kv_heads_shift(c, H), bp = 256 / ng >> sh;
    const double items = (double)n * ((rows + bp - 1) / bp) * (H >> sh), step = c.h == 128 ? (ng == 1 ? 2.15 : 2.65) : (ng == 1 ? 1.45 : 1.65);
    for (int s = 1; s <= 32; s *= 2) {
      if (s > 1 && (r.max_ctx < 256 * s || kv8_part_bytes(Kv8Plan{0, s, 0, 0}, c, r, H) > part_limit)) break;
      const double longest = std::ceil(r.max_ctx / (64. * ng * s)), all = items * seen / (64. * ng * 256);
      double us = std::max(longest * step + 6, all * step + items * s / 256 * (5 + ng));
      if (s > 1) us += 2 + heads / 2000 + heads * s * c.h / 4e6;
      if (us < best_us) { best_us = us; best = PromptPlan{ng, s}; }
    }
  }
  return best;
}

// A launch has fewer than 2^32 threads.  n_rows * H is below 2^24, so the workgroups of up to kInOrder samples, at most 2^24 / 128 for
// the rows and H for each sample, are far below that; one for each of very many samples and heads may not be, and go out in several.
constexpr int kMostWgs = 1 << 22;
template <int HD, int NG, bool kWhole>
void launch_pages(hipStream_t s, const Kv8Cache& c, const Kv8Rows& r, const Kv8Attn& a) {
  PromptGeo g = geo_of(c, r, a.H, 8 / NG);
  const int total = g.n_blocks * g.sets;                         // (at most 2^24 + 2^17)
  if (r.n <= kInOrder) {
    hipLaunchKernelGGL((k_kv8_prompt<HD, NG, kWhole, false>), dim3(total, a.plan.splits), dim3(512), (prompt_lds<HD, NG>()), s, c, r, a, g);
    return;
  }
  for (; g.from < total; g.from += kMostWgs)
    hipLaunchKernelGGL((k_kv8_prompt<HD, NG, kWhole, true>), dim3(std::min(kMostWgs, total - g.from), a.plan.splits), dim3(512), (prompt_lds<HD, NG>()), s, c, r, a, g);
}
template <int HD, int NG>
void launch_groups(hipStream_t s, const Kv8Cache& c, const Kv8Rows& r, const Kv8Attn& a) {
  if (c.pt % BK == 0) launch_pages<HD, NG, true>(s, c, r, a); else launch_pages<HD, NG, false>(s, c, r, a);
}
template <int HD>
void launch_heads(hipStream_t s, const Kv8Cache& c, const Kv8Rows& r, const Kv8Attn& a) {
  if (a.plan.groups == 1) launch_groups<HD, 1>(s, c, r, a); else launch_groups<HD, 2>(s, c, r, a);
}

}  // namespace

bool kv8_prompt_supported(const Kv8Cache& c, const Kv8Rows& r) { return r.start && (c.h == 64 || c.h == 128); }
bool kv8_allow_lds() {
  static OncePerDevice done;
  int dev = -1;
  return hipGetDevice(&dev) == hipSuccess && done.run(dev, []() { return allow_heads<64>() && allow_heads<128>(); });
}

Kv8Plan kv8_prompt_plan(const Kv8Cache& c, const Kv8Rows& r, int H, size_t part_limit) {
  const PromptPlan p = prompt_plan(c, r, H, part_limit);
  const int chunk = ((r.max_ctx + p.splits - 1) / p.splits + BK - 1) / BK * BK;
  return Kv8Plan{chunk, (r.max_ctx + chunk - 1) / chunk, 0, p.groups};
}

void launch_kv8_prompt(hipStream_t s, const Kv8Cache& c, const Kv8Rows& r, const Kv8Attn& a) {
  if (c.h == 128) launch_heads<128>(s, c, r, a); else launch_heads<64>(s, c, r, a);
}

}  // namespace mdi
