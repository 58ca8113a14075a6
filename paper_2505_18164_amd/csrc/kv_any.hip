// Attention over the cache in the storage type on the matrix cores, for what the other kernels do not serve: fp32, and bf16 heads of other
// than 64 or 128 channels, single tokens and packed rows; and for packed rows that are too few for kv_prompt.hip (kv_plan.h).
//
// A workgroup takes sixteen rows of (position, query head) of a kv head, or two times sixteen, and its four wavefronts (two) a share each of
// the keys they see, sixteen at a time (bf16: two times sixteen), straight from the pages into registers; their sums are added
// through the LDS.  Both products are computed transposed, as in kv_decode.hip: S^T = K Q^T leaves scores of keys 4 g + r (g = lane / 16)
// of row lane % 16 in a lane, which is what O^T = V^T P^T takes as its second operand - for fp32 v_mfma_f32_16x16x4_f32, whose
// products and sums are fp32's, register by register; for bf16 v_mfma_f32_16x16x32_bf16 with a weight as two operands, its upper digits
// and what they leave.  Channels and keys may be named in any order that both operands share, so a lane reads 16 bytes of a key and
// 16 channels' worth of a value at a time.  The keys of the next step are asked for when those of this one are multiplied,
// the values when the step begins.  Heads are padded to HD channels with zeros in keys and queries; the padding is not written.
//
// 5 ragged fp32 prompts, 2462 rows of 16 heads of 64 with a window of 300: 49 to 52 us, of which the matrix instructions are 18 (at 154
// TFLOP/s).  A step of a wavefront takes 1.35 times its matrix instructions' time, and 20 us go before the first: the chain from
// the samples' starts over page numbers and addresses to the first keys, twice, as each compute unit is given five workgroups and
// holds three.  A wavefront for every sixteen rows (and no sums to add) took 57, 32 rows of it 60, VALU products 240 to 263.  16 tokens
// behind 3000 of the 7B shape in fp32: 263 us, 6.0 TB/s.
#include <algorithm>
#include <cmath>

#include "kv8_mfma.h"
#include "kv_blocks.h"
#include "kv_device.h"

namespace mdi {
namespace {

constexpr float kRaise = 8.f;        // how far (in powers of two) a score may exceed its row's reference before that is raised

// The operands of a step.  K: what a lane has of key `col` of each sixteen; V: channels VB col .. + VB - 1 of keys 4 g + 0..3.
template <typename T, int HD> struct Step;
template <int HD> struct Step<float, HD> {
  static constexpr int kGroups = 1, VB = HD / 16, KU = HD / 16;
  f32x4 k[KU];
  float v[4][VB];
};
template <int HD> struct Step<bf16_t, HD> {
  static constexpr int kGroups = 2, VB = HD / 16, KU = HD / 32;
  u32x4 k[2][KU];
  uint32_t v[2][4][VB / 2];
};
template <typename T, int HD> struct Query;
template <int HD> struct Query<float, HD> { f32x4 q[HD / 16]; };
template <int HD> struct Query<bf16_t, HD> { u32x4 q[HD / 32]; };

struct AnyGeo { int n_blocks, sets, g_sh, from; };

// What the rows of a workgroup see, at positions at .. end - 1: the first sinks and from .. end - 1, counted in steps of T positions without
// the steps between: place c is position c of the first `apart`, then c + shift (as KvSpan of one row).  64 places are a block.
struct AnySpan { int sinks, apart, shift, from, end, steps; };
template <int T>
__device__ __forceinline__ AnySpan any_span(const KvSight& w, int at, int end) {
  AnySpan b;
  b.end = end;
  b.from = max(at + 1 - w.window, 0);
  b.sinks = min(w.sinks, b.from);
  const int first = (b.sinks + T - 1) & -T, second = b.from & -T;
  b.apart = first < second ? first : 0;
  b.shift = first < second ? second - first : 0;
  b.steps = (end - b.shift + T - 1) / T;
  return b;
}

// kTokens: one row a sample, the columns are up to sixteen query heads of a kv head; else the columns are (position, head) pairs.
template <typename T, int HD, int S, bool kTokens, bool kMany>
__global__ __launch_bounds__(64 * kv_waves_of(HD), HD > 128 ? 1 : 2) void k_kv_any(KvCache c, KvRows r, KvAttn a, AnyGeo geo) {
  typedef Step<T, HD> St;
  constexpr int kKeyStep = 64 / sizeof(T);                       // channels of a key that the four lanes with it read at once
  constexpr int VB = St::VB, KU = St::KU, NG = St::kGroups, KT = 16 * NG, kSteps = 64 / KT;
  constexpr int kWaves = kv_waves_of(HD);
  constexpr int VP = VB < 4 ? VB : 4, kRow = 16 * VP + 4;         // channels of a lane's VB that are added at a time
  __shared__ long list[kWaves][2][64];                           // rows of the cache of 64 places, and of the next ones
  __shared__ float sums[kWaves][16 * S][kRow];
  __shared__ float2 marks[kWaves][16 * S];
  __shared__ int items[16 * S];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4, h = c.h;
  const T* const data = (const T*)c.data;
  int sample_row[S], head[S], pos[S];                            // of this lane's column: row of the call, query head, position
  bool live[S];
  int which, kv, first_pos, last_pos;                            // of the workgroup's rows
  bool none = false;                                             // the sample takes no part
  if constexpr (kTokens) {
    const int G = a.H / c.K, groups = kv8_groups(c, a.H), unit = blockIdx.x, sample = unit / (c.K * groups), rest = unit - sample * (c.K * groups);
    kv = rest / groups;
    const int head0 = kv * G + 16 * (rest - kv * groups), heads = min(16, kv * G + G - head0);
    const int seen = __builtin_amdgcn_readfirstlane(kv8_seen(c, r, sample));
    which = seen ? __builtin_amdgcn_readfirstlane(kv8_table_row(c, r, sample)) : -1;
    none = which < 0;
    first_pos = last_pos = seen - 1;
    sample_row[0] = sample; head[0] = head0 + min(col, heads - 1); pos[0] = seen - 1; live[0] = col < heads;
  } else {
    const int x = kMany ? geo.from + blockIdx.x : blockIdx.x, block = x / geo.sets, set = x - block * geo.sets, g_sh = geo.g_sh, bp = 16 * S >> g_sh;
    const BlockPlace at = place_of<kMany>(r, block, bp);
    if (at.sample < 0) return;
    // (a sample's longest rows first)
    const int q0 = ((at.rows + bp - 1) / bp - 1 - at.block) * bp, head0 = set << g_sh, end = min(q0 + bp, at.rows);
    kv = head0 / (a.H / c.K);
    which = at.pos < 0 ? -1 : kv8_checked_row(c, at.table);
    none = which < 0;
    const long far = (long)at.pos + end;
    if (!none && far > r.max_ctx) kv8_report(c);
    auto pos_of = [&](int row) { return (int)min((long)at.pos + min(row, at.rows - 1), (long)r.max_ctx - 1); };
    first_pos = pos_of(q0);
    last_pos = pos_of(end - 1);
#pragma unroll
    for (int u = 0; u < S; ++u) {
      const int row = q0 + ((16 * u + col) >> g_sh);
      live[u] = row < at.rows;
      pos[u] = pos_of(row);
      sample_row[u] = at.first + min(row, at.rows - 1);
      head[u] = head0 + (col & ((1 << g_sh) - 1));
    }
  }
  auto item_of = [&](int u) { return sample_row[u] * a.H + head[u]; };
  if (none) {
    if (blockIdx.y == 0 && wave == 0)
#pragma unroll
      for (int u = 0; u < S; ++u) {
        if (!live[u]) continue;
        T* const out = (T*)a.out + (long)sample_row[u] * a.out_stride + (long)head[u] * h;
        for (int ch = g; ch < h; ch += 4) Storage<T>::put(out + ch, 0.f);
        if (a.plan.splits > 1 && g == 0) kv_part_counts(a, c, r)[item_of(u)] = 1;
      }
    return;
  }
  const int32_t* const table = c.tables + (long)which * c.table_stride;
  const AnySpan kb = any_span<KT>(a.sight, first_pos, last_pos + 1);
  const int blocks = (kb.steps + kSteps - 1) / kSteps, pieces = (blocks + a.plan.chunk - 1) / a.plan.chunk;
  const int p_lo = kSteps * blockIdx.y * a.plan.chunk, p_hi = (int)min((long)kb.steps, (long)p_lo + kSteps * (long)a.plan.chunk);   // of the piece
  if (p_lo >= p_hi) return;
  const int lo = p_lo + (int)((long)(p_hi - p_lo) * wave / kWaves), hi = p_lo + (int)((long)(p_hi - p_lo) * (wave + 1) / kWaves);   // of the wavefront

  // queries: channels 16 s + 4 g + 0..3 (bf16: 32 s + 8 g + 0..7), as the keys'
  Query<T, HD> q[S];
#pragma unroll
  for (int u = 0; u < S; ++u) {
    const T* const p = (const T*)a.q + (long)sample_row[u] * a.q_stride + (long)head[u] * h;
#pragma unroll
    for (int s = 0; s < KU; ++s) {
      if constexpr (sizeof(T) == 4) q[u].q[s] = 16 * s + 4 * g < h ? *reinterpret_cast<const f32x4*>(p + 16 * s + 4 * g) : f32x4{};
      else q[u].q[s] = 32 * s + 8 * g < h ? *reinterpret_cast<const u32x4*>(p + 32 * s + 8 * g) : u32x4{};
    }
  }
  f32x4 o[S][VB];
  float m[S], l[S];
#pragma unroll
  for (int u = 0; u < S; ++u) {
    m[u] = kKvNone;
    l[u] = 0.f;
#pragma unroll
    for (int b = 0; b < VB; ++b) o[u][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // A position that no row of the workgroup sees stands for one near it that some row sees; lane i looks up place i of 64 from step lo on.
  auto position = [&](int place) __attribute__((always_inline)) { return place + (place >= kb.apart ? kb.shift : 0); };
  auto key_at = [&](int b) __attribute__((always_inline)) {
    const int place = KT * lo + 64 * b + lane, p = position(place);
    return min(p < kb.sinks || p >= kb.from ? p : place < kb.apart ? kb.sinks - 1 : kb.from, kb.end - 1);
  };
  auto page_at = [&](int b) __attribute__((always_inline)) { return table[kv8_page_of(c, key_at(b))]; };
  auto note = [&](int b, int page) __attribute__((always_inline)) { list[wave][b & 1][lane] = kv8_row(c, kv8_checked_page(c, page), kv, key_at(b)) * h; };
  // (a wavefront's LDS accesses are made in order)
  auto wrote = [&]() __attribute__((always_inline)) { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); __builtin_amdgcn_wave_barrier(); };
  St st;
  // Channels behind the head's: others of the same row are read, which count for nothing (keys: set to zero when they are used; values:
  // their sums are not written).
  int key_ch[KU], value_ch[VB * sizeof(T) / 4 < 4 ? 1 : VB * sizeof(T) / 16];
#pragma unroll
  for (int s = 0; s < KU; ++s) key_ch[s] = min(kKeyStep * s + kKeyStep / 4 * g, h - kKeyStep / 4);
#pragma unroll
  for (int w = 0; w < (int)(sizeof(value_ch) / sizeof(int)); ++w) value_ch[w] = min(VB * col + kKeyStep / 4 * w, h - min(VB, kKeyStep / 4));
  auto ask_keys = [&](int b, int t) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      const T* const p = data + list[wave][b & 1][KT * t + 16 * n + col];
#pragma unroll
      for (int s = 0; s < KU; ++s) {
        if constexpr (sizeof(T) == 4) st.k[s] = *reinterpret_cast<const f32x4*>(p + key_ch[s]);
        else st.k[n][s] = *reinterpret_cast<const u32x4*>(p + key_ch[s]);
      }
    }
  };
  auto ask_values = [&](int b, int t) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NG; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const T* const p = data + (list[wave][b & 1][KT * t + 16 * n + 4 * g + j] + (long)c.pt * h);
        if constexpr (sizeof(T) == 4) {
          if constexpr (VB % 4 == 0) {
#pragma unroll
            for (int w = 0; w < VB; w += 4) {
              const f32x4 x = *reinterpret_cast<const f32x4*>(p + value_ch[w / 4]);
              st.v[j][w] = x.x; st.v[j][w + 1] = x.y; st.v[j][w + 2] = x.z; st.v[j][w + 3] = x.w;
            }
          } else {
            const float2 x = *reinterpret_cast<const float2*>(p + value_ch[0]);
            st.v[j][0] = x.x; st.v[j][1] = x.y;
          }
        } else if constexpr (VB % 8 == 0) {
#pragma unroll
          for (int w = 0; w < VB / 2; w += 4) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(p + value_ch[w / 4]);
            st.v[n][j][w] = x.x; st.v[n][j][w + 1] = x.y; st.v[n][j][w + 2] = x.z; st.v[n][j][w + 3] = x.w;
          }
        } else {
#pragma unroll
          for (int w = 0; w < VB / 2; ++w) st.v[n][j][w] = *reinterpret_cast<const uint32_t*>(p + value_ch[0] + 2 * w);
        }
      }
  };

  if (lo < hi) {
    note(0, page_at(0));
    int page = page_at(1);
    wrote();
    ask_keys(0, 0);
    for (int b = 0; lo + kSteps * b < hi; ++b) {
      note(b + 1, page);
      page = page_at(b + 2);
      wrote();
      const int steps = min(kSteps, hi - lo - kSteps * b);
      for (int t = 0; t < steps; ++t) {
        const int kt = position(KT * lo + 64 * b + KT * t);
        ask_values(b, t);
        __builtin_amdgcn_sched_barrier(0);
        if (h != HD)
#pragma unroll
          for (int s = 0; s < KU; ++s)
            if (kKeyStep * s + kKeyStep / 4 * g >= h)
#pragma unroll
              for (int n = 0; n < NG; ++n) {
                if constexpr (sizeof(T) == 4) st.k[s] = f32x4{}; else st.k[n][s] = u32x4{};
              }
        f32x4 s[S][NG];
#pragma unroll
        for (int u = 0; u < S; ++u)
#pragma unroll
          for (int n = 0; n < NG; ++n) s[u][n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KU; ++i)
          if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int u = 0; u < S; ++u) s[u][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(st.k[i][e], q[u].q[i][e], s[u][0], 0, 0, 0);
          } else {
#pragma unroll
            for (int n = 0; n < NG; ++n)
#pragma unroll
              for (int u = 0; u < S; ++u)
                s[u][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, st.k[n][i]), __builtin_bit_cast(bf16x8, q[u].q[i]), s[u][n], 0, 0, 0);
          }
        __builtin_amdgcn_sched_barrier(0);
        // (behind the last step's keys nothing that is used)
        ask_keys(t + 1 < steps ? b : b + 1, t + 1 < steps ? t + 1 : 0);
        __builtin_amdgcn_sched_barrier(0);
        float weight[S][4 * NG];
        const bool whole = kt + KT - 1 <= first_pos && (kt > last_pos - a.sight.window || kt + KT <= a.sight.sinks);   // all keys are for all rows
#pragma unroll
        for (int u = 0; u < S; ++u) {
          // (from here on scalars: hipcc lost elements of a vector of which one was replaced under a condition)
          float x[4 * NG], top;
#pragma unroll
          for (int i = 0; i < 4 * NG; ++i) x[i] = s[u][i >> 2][i & 3] * a.scale;
          if (!whole) {
#pragma unroll
            for (int i = 0; i < 4 * NG; ++i) {
              const int key = kt + 16 * (i >> 2) + 4 * g + (i & 3);
              x[i] = (key <= pos[u]) & ((key > pos[u] - a.sight.window) | (key < a.sight.sinks)) ? x[i] : -INFINITY;
            }
          }
          top = x[0];
#pragma unroll
          for (int i = 1; i < 4 * NG; ++i) top = fmaxf(top, x[i]);
          // Weights are relative to m, which is raised - for all four lanes of a row alike - only when a score exceeds it by
          // 2^kRaise: the sum is divided out at the end, so any reference near the largest score does.
          if (__any(top > m[u] + kRaise)) {
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float to = fmaxf(m[u], top), alpha = exp2_raw(m[u] - to);
            m[u] = to;
            l[u] *= alpha;
#pragma unroll
            for (int v = 0; v < VB; ++v) o[u][v] *= alpha;
          }
#pragma unroll
          for (int i = 0; i < 4 * NG; ++i) {
            weight[u][i] = exp2_raw(x[i] - m[u]);
            l[u] += weight[u][i];
          }
        }
        if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int v = 0; v < VB; ++v)
#pragma unroll
              for (int u = 0; u < S; ++u) o[u][v] = __builtin_amdgcn_mfma_f32_16x16x4f32(st.v[j][v], weight[u][j], o[u][v], 0, 0, 0);
        } else {
          u32x4 hi_w[S];
          bf16x8 lo_w[S];
#pragma unroll
          for (int u = 0; u < S; ++u)
#pragma unroll
            for (int n = 0; n < NG; ++n)
#pragma unroll
              for (int j = 0; j < 4; j += 2) {
                const float w0 = weight[u][4 * n + j], w1 = weight[u][4 * n + j + 1];
                hi_w[u][2 * n + j / 2] = high_halves(w0, w1);
                lo_w[u][4 * n + j] = (__bf16)(w0 - __uint_as_float(__float_as_uint(w0) & 0xFFFF0000u));
                lo_w[u][4 * n + j + 1] = (__bf16)(w1 - __uint_as_float(__float_as_uint(w1) & 0xFFFF0000u));
              }
#pragma unroll
          for (int w = 0; w < VB / 2; ++w) {
            u32x4 f[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {                           // keys 4 g + 2 (i % 2), + 1 of group i / 2
              const uint32_t lo_row = st.v[i >> 1][2 * (i & 1)][w], hi_row = st.v[i >> 1][2 * (i & 1) + 1][w];
              f[0][i] = __builtin_amdgcn_perm(hi_row, lo_row, 0x05040100u);
              f[1][i] = __builtin_amdgcn_perm(hi_row, lo_row, 0x07060302u);
            }
#pragma unroll
            for (int u = 0; u < S; ++u)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                f32x4& x = o[u][2 * w + e];
                x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f[e]), __builtin_bit_cast(bf16x8, hi_w[u]), x, 0, 0, 0);
                x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f[e]), lo_w[u], x, 0, 0, 0);
              }
          }
        }
      }
    }

  }
  // A value that is not finite spoils the sums of rows that do not see it, too: a zero weight times infinity is no number.  Then all rows
  // are computed once more, each by itself.  (Weights that are no numbers are what they should be.)
  float odd = 0.f;
  bool spoiled = false;
#pragma unroll
  for (int u = 0; u < S; ++u) {
    l[u] += __shfl_xor(l[u], 16, 64);
    l[u] += __shfl_xor(l[u], 32, 64);
    odd = 0.f;
#pragma unroll
    for (int v = 0; v < VB; ++v)
#pragma unroll
      for (int j = 0; j < 4; ++j) odd = fmaf(o[u][v][j], 0.f, odd);
    spoiled |= !(odd == 0.f) && l[u] - l[u] == 0.f;
  }
  if (wave == 0 && g == 0)
#pragma unroll
    for (int u = 0; u < S; ++u) {
      items[16 * u + col] = live[u] ? item_of(u) : -1;
      if (live[u] && a.plan.splits > 1 && blockIdx.y == 0) kv_part_counts(a, c, r)[item_of(u)] = pieces;
    }
  if (__builtin_expect(__syncthreads_or(spoiled), 0)) {
    int L = 1;
    while (8 * L < h) L *= 2;
    const int ch = 8 * (lane & (L - 1));
#pragma unroll
    for (int u = 0; u < S; ++u)
      for (int i = wave; i < 16; i += kWaves) {
        if (!__shfl((int)live[u], i, 64)) continue;
        const int row1 = __shfl(sample_row[u], i, 64), head1 = __shfl(head[u], i, 64), end1 = __shfl(pos[u], i, 64) + 1, from1 = max(end1 - a.sight.window, 0),
                  item1 = row1 * a.H + head1;
        const KvSpan span{min(a.sight.sinks, from1), kb.apart, kb.shift, from1, end1};
        float x[8] = {};
        if (ch < h) KvType<T>::load8((const T*)a.q + (long)row1 * a.q_stride + (long)head1 * h + ch, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= a.scale;
        const KvSums one = kv_attend<T>(c, table, kv, span, x, L, ch, ch < h, KT * p_lo, 64 / L, min(KT * p_hi, end1 - kb.shift));
        if (lane >= L || ch >= h) continue;
        T* const out = (T*)a.out + (long)row1 * a.out_stride + (long)head1 * h + ch;
        float* const part = kv_part_sums(a, c, item1, blockIdx.y) + ch;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (pieces == 1) Storage<T>::put(out + e, one.o[e] / one.l);
          else part[e] = one.o[e];
        if (lane == 0 && pieces > 1) *kv_part_marks(a, c, r, item1, blockIdx.y) = make_float2(one.m, one.l);
      }
    return;
  }
  // Lane (col, g) has channels VB (4 g + j) + v of its rows in o[v][j].  The wavefronts' sums are added, VP of the VB at a time, always in
  // the same order.
#pragma unroll
  for (int v0 = 0; v0 < VB; v0 += VP) {
    if (v0) __syncthreads();
#pragma unroll
    for (int u = 0; u < S; ++u) {
      if (v0 == 0 && g == 0) marks[wave][16 * u + col] = make_float2(m[u], l[u]);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int v = 0; v < VP; ++v) sums[wave][16 * u + col][VP * (4 * g + j) + v] = o[u][v0 + v][j];
    }
    __syncthreads();
#pragma unroll
    for (int row = threadIdx.x >> 4; row < 16 * S; row += 4 * kWaves) {
      const int ch = VB * (threadIdx.x & 15) + v0, item = items[row];
      float f[kWaves], to = kKvNone, sum = 0.f, x[VP] = {};
#pragma unroll
      for (int i = 0; i < kWaves; ++i) to = fmaxf(to, marks[i][row].x);
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        f[i] = exp2_raw(marks[i][row].x - to);
        sum += marks[i][row].y * f[i];
#pragma unroll
        for (int v = 0; v < VP; ++v) x[v] = fmaf(sums[i][row][VP * (threadIdx.x & 15) + v], f[i], x[v]);
      }
      if (item < 0) continue;
      if (pieces == 1) {
        const int at = item / a.H;
        T* const out = (T*)a.out + (long)at * a.out_stride + (long)(item - at * a.H) * h + ch;
        const float inv = 1.f / sum;
#pragma unroll
        for (int v = 0; v < VP; ++v)
          if (ch + v < h) Storage<T>::put(out + v, x[v] * inv);
      } else {
        float* const part = kv_part_sums(a, c, item, blockIdx.y) + ch;
#pragma unroll
        for (int v = 0; v < VP; ++v)
          if (ch + v < h) part[v] = x[v];
        if (ch == 0) *kv_part_marks(a, c, r, item, blockIdx.y) = make_float2(to, sum);
      }
    }
  }
}

AnyGeo geo_of(const KvCache& c, const KvRows& r, int H, int sets) {
  const int rows = 16 * sets, sh = std::min(kv_heads_shift(c, H), 4), bp = rows >> sh;   // (a wavefront's sixteen are a multiple of 2^sh)
  return AnyGeo{r.n_rows / bp + std::min(r.n, r.n_rows), H >> sh, sh, 0};
}

constexpr int kMostWgs = 1 << 22;    // of a launch: it has fewer than 2^32 threads
template <typename T, int HD, int S>
void launch_sets(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a) {
  AnyGeo g = geo_of(c, r, a.H, S);
  const int total = g.n_blocks * g.sets;
  if (r.n <= kInOrder) {
    hipLaunchKernelGGL((k_kv_any<T, HD, S, false, false>), dim3(total, a.plan.splits), dim3(64 * kv_waves_of(HD)), 0, s, c, r, a, g);
    return;
  }
  for (; g.from < total; g.from += kMostWgs)
    hipLaunchKernelGGL((k_kv_any<T, HD, S, false, true>), dim3(std::min(kMostWgs, total - g.from), a.plan.splits), dim3(64 * kv_waves_of(HD)), 0, s, c, r, a, g);
}
template <typename T, int HD>
void launch_heads(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a) {
  if (!r.start) {
    const long units = (long)r.n * c.K * kv8_groups(c, a.H);     // (below 2^24: n_rows * H is)
    hipLaunchKernelGGL((k_kv_any<T, HD, 1, true, false>), dim3((unsigned)units, a.plan.splits), dim3(64 * kv_waves_of(HD)), 0, s, c, r, a, AnyGeo{});
    return;
  }
  if constexpr (kv_most_sets(HD, sizeof(T)) == 2) if (a.plan.groups == 2) return launch_sets<T, HD, 2>(s, c, r, a);
  launch_sets<T, HD, 1>(s, c, r, a);
}
template <typename T>
void launch_type(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a) {
  switch (kv_padded(c.h)) {
    case 32: return launch_heads<T, 32>(s, c, r, a);
    case 64: return launch_heads<T, 64>(s, c, r, a);
    case 128: return launch_heads<T, 128>(s, c, r, a);
    default: return launch_heads<T, 256>(s, c, r, a);
  }
}

}  // namespace

void launch_kv_any(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a) {
  if (c.dtype == MDI_BF16) launch_type<bf16_t>(s, c, r, a); else launch_type<float>(s, c, r, a);
}

}  // namespace mdi
