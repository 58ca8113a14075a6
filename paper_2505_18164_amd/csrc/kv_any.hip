// Attention over the cache in the storage type on the matrix cores, for what the other two kernels do not serve: fp32, and bf16 heads of
// other than 64 or 128 channels; single tokens and packed rows.
//
// A wavefront takes sixteen rows of (position, query head) of a kv head, or S times as many, and passes over the keys they see,
// sixteen at a time (bf16: two times sixteen), straight from the pages into registers.  Both products are computed transposed, as in
// kv_decode.hip: S^T = K Q^T leaves scores of keys 4 g + r (g = lane / 16) of row lane % 16 in a lane, which is what O^T = V^T P^T
// takes as its second operand - for fp32 v_mfma_f32_16x16x4_f32, whose products and sums are fp32's, register by register; for bf16
// v_mfma_f32_16x16x32_bf16 with a weight as two operands, its upper digits and what they leave.  Channels and keys may be named in any
// order that both operands share, so a lane reads 16 bytes of a key and 16 channels' worth of a value at a time.
// The keys of the next step are asked for when those of this one are multiplied, the values when the scores are, so that either has half
// a step to arrive, without other registers.  Heads are padded to HD channels, the padding is neither read nor written.
#include <algorithm>
#include <cmath>

#include "kv8_mfma.h"
#include "kv_blocks.h"
#include "kv_device.h"

namespace mdi {
namespace {

constexpr int kWaves = 4;
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

// What a wavefront's rows see, 64 positions a block: as in kv_prompt_device.h.
struct AnyBlocks { int sinks, n_sinks, first, from, end, n; };
__device__ __forceinline__ AnyBlocks any_blocks(const KvSight& w, int at, int end) {
  AnyBlocks b;
  b.end = end;
  b.from = max(at + 1 - w.window, 0);
  b.sinks = min(w.sinks, b.from);
  const int s64 = (b.sinks + 63) >> 6, f64 = b.from >> 6;
  b.n_sinks = s64 < f64 ? s64 : 0;
  b.first = b.n_sinks || b.sinks == 0 ? f64 << 6 : 0;
  b.n = b.n_sinks + ((end - b.first + 63) >> 6);
  return b;
}

// kTokens: one row a sample, the columns are up to sixteen query heads of a kv head; else the columns are (position, head) pairs.
template <typename T, int HD, int S, bool kTokens, bool kMany>
__global__ __launch_bounds__(64 * kWaves, HD > 128 ? 1 : 2) void k_kv_any(KvCache c, KvRows r, KvAttn a, AnyGeo geo) {
  typedef Step<T, HD> St;
  constexpr int kKeyStep = 64 / sizeof(T);                       // channels of a key that the four lanes with it read at once
  constexpr int VB = St::VB, KU = St::KU, NG = St::kGroups, KT = 16 * NG, kTiles = 64 / KT;
  __shared__ long list[kWaves][2][64];                           // rows of the cache of a block's keys, and of the next one's

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4, h = c.h;
  const T* const data = (const T*)c.data;
  int sample_row[S], head[S], pos[S];                            // of this lane's column: row of the call, query head, position
  bool live[S];
  int which, kv, first_pos, last_pos;                            // of the wavefront's rows
  bool none = false;                                             // the sample takes no part
  if constexpr (kTokens) {
    const int G = a.H / c.K, groups = kv8_groups(c, a.H), unit = blockIdx.x * kWaves + wave, sample = unit / (c.K * groups), rest = unit - sample * (c.K * groups);
    if (sample >= r.n) return;
    kv = rest / groups;
    const int head0 = kv * G + 16 * (rest - kv * groups), heads = min(16, kv * G + G - head0);
    const int seen = __builtin_amdgcn_readfirstlane(kv8_seen(c, r, sample));
    which = __builtin_amdgcn_readfirstlane(kv8_table_row(c, r, sample));
    none = !seen || which < 0;
    first_pos = last_pos = seen - 1;
    sample_row[0] = sample; head[0] = head0 + min(col, heads - 1); pos[0] = seen - 1; live[0] = col < heads;
  } else {
    const int x = kMany ? geo.from + blockIdx.x : blockIdx.x, block = x / geo.sets, set = x - block * geo.sets, g_sh = geo.g_sh, bp = 16 * S * kWaves >> g_sh;
    const BlockPlace at = place_of<kMany>(r, block, bp);
    if (at.sample < 0) return;
    // (a sample's longest rows first)
    const int q0 = ((at.rows + bp - 1) / bp - 1 - at.block) * bp + (16 * S * wave >> g_sh), head0 = set << g_sh, end = min(q0 + (16 * S >> g_sh), at.rows);
    if (q0 >= at.rows) return;
    kv = head0 / (a.H / c.K);
    which = kv8_checked_row(c, at.table);
    none = at.pos < 0 || which < 0;
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
    if (blockIdx.y == 0)
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
  const AnyBlocks kb = any_blocks(a.sight, first_pos, last_pos + 1);
  const int b_lo = blockIdx.y * a.plan.chunk, b_hi = (int)min((long)kb.n, (long)b_lo + a.plan.chunk), pieces = (kb.n + a.plan.chunk - 1) / a.plan.chunk;
  if (b_lo >= b_hi) return;

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

  // A position that no row of the wavefront sees stands for one near it that some row sees; lane i looks up key i of a block.
  auto start_of = [&](int b) __attribute__((always_inline)) { return b < kb.n_sinks ? b << 6 : kb.first + ((b - kb.n_sinks) << 6); };
  auto key_at = [&](int b) __attribute__((always_inline)) {
    const int k0 = start_of(min(b, b_hi - 1)), p = k0 + lane;
    return min(p < kb.sinks || p >= kb.from ? p : k0 < kb.sinks ? kb.sinks - 1 : kb.from, kb.end - 1);
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

  note(b_lo, page_at(b_lo));
  int page = page_at(b_lo + 1);
  wrote();
  ask_keys(b_lo, 0);
  for (int b = b_lo; b < b_hi; ++b) {
    note(b + 1, page);
    page = page_at(b + 2);
    wrote();
    const int k0 = start_of(b);
    for (int t = 0; t < kTiles; ++t) {
      const int kt = k0 + KT * t;
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
      ask_keys(t + 1 < kTiles ? b : b + 1, t + 1 < kTiles ? t + 1 : 0);
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
  if (__builtin_expect(__any(spoiled), 0)) {
    int L = 1;
    while (8 * L < h) L *= 2;
    const int ch = 8 * (lane & (L - 1)), shift = kb.first - 64 * kb.n_sinks;
    for (int u = 0; u < S; ++u)
      for (int i = 0; i < 16; ++i) {
        if (!__shfl((int)(u == 0 ? live[0] : live[S - 1]), i, 64)) continue;
        const int row1 = __shfl(u == 0 ? sample_row[0] : sample_row[S - 1], i, 64), head1 = __shfl(u == 0 ? head[0] : head[S - 1], i, 64),
                  end1 = __shfl(u == 0 ? pos[0] : pos[S - 1], i, 64) + 1, from1 = max(end1 - a.sight.window, 0), item1 = row1 * a.H + head1;
        const KvSpan span{min(a.sight.sinks, from1), 64 * kb.n_sinks, shift, from1, end1};
        float x[8] = {};
        if (ch < h) KvType<T>::load8((const T*)a.q + (long)row1 * a.q_stride + (long)head1 * h + ch, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= a.scale;
        const KvSums sums = kv_attend<T>(c, table, kv, span, x, L, ch, ch < h, 64 * b_lo, 64 / L, min(64 * b_hi, end1 - shift));
        if (lane >= L || ch >= h) continue;
        T* const out = (T*)a.out + (long)row1 * a.out_stride + (long)head1 * h + ch;
        float* const part = kv_part_sums(a, c, item1, blockIdx.y) + ch;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (pieces == 1) Storage<T>::put(out + e, sums.o[e] / sums.l);
          else part[e] = sums.o[e];
        if (lane == 0 && pieces > 1) *kv_part_marks(a, c, r, item1, blockIdx.y) = make_float2(sums.m, sums.l);
        if (lane == 0 && blockIdx.y == 0 && a.plan.splits > 1) kv_part_counts(a, c, r)[item1] = pieces;
      }
    return;
  }
  // lane (col, g) has channels VB (4 g + j) + v of its column in o[v][j]
#pragma unroll
  for (int u = 0; u < S; ++u) {
    if (!live[u]) continue;
    const int item = item_of(u);
    if (a.plan.splits > 1 && blockIdx.y == 0 && g == 0) kv_part_counts(a, c, r)[item] = pieces;
    const float inv = 1.f / l[u];
    T* const out = (T*)a.out + (long)sample_row[u] * a.out_stride + (long)head[u] * h;
    float* const part = kv_part_sums(a, c, item, blockIdx.y);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int v = 0; v < VB; ++v) {
        const int ch = VB * (4 * g + j) + v;
        if (ch >= h) continue;
        if (pieces == 1) Storage<T>::put(out + ch, o[u][v][j] * inv);
        else part[ch] = o[u][v][j];
      }
    if (pieces > 1 && g == 0) *kv_part_marks(a, c, r, item, blockIdx.y) = make_float2(m[u], l[u]);
  }
}

// Rows of a workgroup: S sets of sixteen for each of four wavefronts; two sets where they fit into the registers of two wavefronts a SIMD.
template <typename T> constexpr int sets_of(int padded) { return padded * sizeof(T) <= 256 ? 2 : 1; }
int padded(int h) { return h <= 32 ? 32 : h <= 64 ? 64 : h <= 128 ? 128 : 256; }

int sets_of(const KvCache& c) { return c.dtype == MDI_BF16 ? sets_of<bf16_t>(padded(c.h)) : sets_of<float>(padded(c.h)); }

AnyGeo geo_of(const KvCache& c, const KvRows& r, int H) {
  const int rows = 16 * sets_of(c) * kWaves, sh = std::min(kv_heads_shift(c, H), 4), bp = rows >> sh;   // (a wavefront's sixteen are a multiple of 2^sh)
  return AnyGeo{r.n_rows / bp + std::min(r.n, r.n_rows), H >> sh, sh, 0};
}

constexpr int kMostWgs = 1 << 22;    // of a launch: it has fewer than 2^32 threads
template <typename T, int HD>
void launch_heads(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a) {
  constexpr int S = sets_of<T>(HD);
  if (!r.start) {
    const long units = (long)r.n * c.K * kv8_groups(c, a.H);     // (below 2^24: n_rows * H is)
    hipLaunchKernelGGL((k_kv_any<T, HD, 1, true, false>), dim3((unsigned)((units + kWaves - 1) / kWaves), a.plan.splits), dim3(64 * kWaves), 0, s, c, r, a, AnyGeo{});
    return;
  }
  AnyGeo g = geo_of(c, r, a.H);
  const int total = g.n_blocks * g.sets;
  if (r.n <= kInOrder) {
    hipLaunchKernelGGL((k_kv_any<T, HD, S, false, false>), dim3(total, a.plan.splits), dim3(64 * kWaves), 0, s, c, r, a, g);
    return;
  }
  for (; g.from < total; g.from += kMostWgs)
    hipLaunchKernelGGL((k_kv_any<T, HD, S, false, true>), dim3(std::min(kMostWgs, total - g.from), a.plan.splits), dim3(64 * kWaves), 0, s, c, r, a, g);
}
template <typename T>
void launch_type(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a) {
  switch (padded(c.h)) {
    case 32: return launch_heads<T, 32>(s, c, r, a);
    case 64: return launch_heads<T, 64>(s, c, r, a);
    case 128: return launch_heads<T, 128>(s, c, r, a);
    default: return launch_heads<T, 256>(s, c, r, a);
  }
}

}  // namespace

// Pieces of a row's blocks: so many wavefronts that every SIMD has two, if there are blocks for them; more pieces than that have to be
// added again.
KvPlan kv_any_plan(const KvCache& c, const KvRows& r, int H, const KvSight& w) {
  const int S = r.start ? sets_of(c) : 1, sh = std::min(kv_heads_shift(c, H), 4), bp = 16 * S >> sh;   // positions of a wavefront
  const int n = std::max(1, std::min(r.n, r.n_rows)), rows = (r.n_rows + n - 1) / n;
  const double waves = r.start ? (double)n * ((rows + bp - 1) / bp) * (H >> sh) : (double)r.n * c.K * kv8_groups(c, H);
  const long most = std::min<long>(((long)r.max_ctx + 63) / 64, ((long)w.window + (r.start ? bp : 1) + 62) / 64 + 1 + ((long)w.sinks + 63) / 64);   // blocks of a wavefront
  const int want = (int)std::min(64., std::max(1., std::min(most / 2., std::ceil(2048. / waves))));
  const int chunk = (int)((most + want - 1) / want);
  return KvPlan{chunk, (int)((most + chunk - 1) / chunk), 0, 0};
}

void launch_kv_any(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a) {
  if (c.dtype == MDI_BF16) launch_type<bf16_t>(s, c, r, a); else launch_type<float>(s, c, r, a);
}

}  // namespace mdi
