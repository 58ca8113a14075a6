// Attention of one new token per sample over the bf16 cache, on the matrix cores.
//
// A workgroup takes one kv head of one sample and up to sixteen of its query heads (a unit), or a piece of the places they see (see
// KvSpan); its four wavefronts take 32 places in turn, straight from the pages into registers.  Both products are computed
// transposed: S^T = K Q^T leaves, with v_mfma_f32_16x16x32_bf16, places 4 g + r (g = lane / 16) of query lane % 16 in a lane, and two
// groups of 16 places side by side are just what O^T = V^T P^T takes as its second operand, if the places that lane
// group g contracts are named 4 g .. 4 g + 3 of either.  The sum over places is in no order, so any naming does; likewise the
// channels of K and Q.  So a key is read 16 bytes a lane (four lanes a row, 64 bytes of it next to each other), a value HD / 8 bytes a
// lane, a whole row by sixteen lanes, and what the first operand of the second product wants - one channel of eight places - is a
// byte permutation of two registers for every two of them.
//
// Memory bounds it: one token of the 8B shape behind 120001, 492 MB, 81.6 us and 5.4 to join the pieces, 6.0 TB/s (a plain read reaches
// 6.3 to 6.5); 8 tokens of the 7B shape behind 1 to 4096, 259 MB, 47.3 and 4.6; 16 of the 8B shape with a window of 4096, 264 MB,
// 47.9 and 4.6.  Of the 47 us some 5 are the way to the first keys: positions, shares, page numbers, each behind the one before.
// Dot products in vector instructions took 107, 366 and 200 us for the three.
#include <algorithm>

#include "kv8_mfma.h"
#include "kv_device.h"
#include "kv_plan.h"

namespace mdi {
namespace {

constexpr int kWaves = 4;
constexpr float kRaise = 8.f;        // how far (in powers of two) a score may exceed its query's reference before that is raised
constexpr int kList = 1024;          // rows of a piece that the LDS holds at a time: one for every 16 places, or for every one

template <int HD> struct Tile {      // 32 places of a wavefront
  u32x4 k[2][HD / 32];
  uint32_t v[2][4][HD / 32];
};

// A cache that no later call finds in the last cache is read without a place in it.
template <bool kOnce, typename T> __device__ __forceinline__ T load_rows(const void* p) {
  if constexpr (kOnce) return __builtin_nontemporal_load((const T*)p); else return *(const T*)p;
}

// kWhole16: pages of a multiple of 16 positions, so 16 aligned positions lie in one page, next to each other.
template <int HD, bool kWhole16, bool kOnce>
__global__ __launch_bounds__(64 * kWaves, 3) void k_kv_decode(KvCache c, KvRows r, KvAttn a, int groups) {
  constexpr int KI = HD / 32, VB = HD / 16;                      // 16-byte units of a key a lane has; channels of a value (= channel blocks)
  constexpr int OS = HD + 4, kGrain = kWhole16 ? 16 : 1;
  __shared__ __attribute__((aligned(16))) float fold[kWaves * 16 * OS];
  __shared__ float fold_m[kWaves][16], fold_l[kWaves][16];
  __shared__ long list[kList];
  __shared__ int again;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
  const bf16_t* const data = (const bf16_t*)c.data;
  const int units = c.K * groups, G = a.H / c.K;                  // units of a sample: a kv head's sixteen query heads
  int x0 = blockIdx.x, x1 = x0 + 1, per = 1, seen64 = 0;
  auto places_of = [&](int i) __attribute__((always_inline)) { return kv_places(c, r, a.sight, i); };
  if (a.plan.wgs) {
    seen64 = places_of(lane);
    const Kv8Stream all = kv8_stream_of(r, a.plan.chunk, a.plan.wgs, units, 0, seen64, places_of);
    per = all.per;
    x0 = min(x0 * per, all.cost * units);
    x1 = min(x0 + per, all.cost * units);
  }
  while (x0 < x1) {
    int sample, unit, n_places, piece = 0, pieces = 1, lo = 0, end;
    if (a.plan.wgs) {
      const Kv8Found f = kv8_find_of(r, x0 / units, seen64, places_of);
      sample = f.sample;
      n_places = f.seen;
      const int tiles = kv8_tiles(n_places), cost = tiles + kKv8Begin, in = x0 - f.start * units;
      unit = in / cost;
      // this share has x0 .. next - 1, the unit's tiles are from .. from + tiles - 1
      const int start = f.start * units + unit * cost, from = start + kKv8Begin, next = min(x1, start + cost), first_wg = from / per;
      lo = max(x0 - from, 0) * kKv8Tile;
      end = min(n_places, max(next - from, 0) * kKv8Tile);
      piece = (int)blockIdx.x - first_wg;
      pieces = max(from + tiles - 1, from) / per - first_wg + 1;
      x0 = next;
      if (n_places && lo >= end) continue;                       // only what it costs to begin: the tiles are another share's
    } else {
      sample = x0 / units;
      unit = x0 - sample * units;
      n_places = end = __builtin_amdgcn_readfirstlane(places_of(sample));
      x0 = x1;
    }
    const int kv = unit / groups, head0 = kv * G + 16 * (unit - kv * groups), heads = min(16, kv * G + G - head0);
    const int which = n_places ? __builtin_amdgcn_readfirstlane(kv8_table_row(c, r, sample)) : -1;   // (who takes no part may have any table)
    const int32_t* table = c.tables + (long)max(which, 0) * c.table_stride;
    const KvSpan span = kv_span(a.sight, __builtin_amdgcn_readfirstlane(kv8_seen(c, r, sample)));
    bf16_t* out = (bf16_t*)a.out + (long)sample * a.out_stride + (long)head0 * HD;
    if (a.plan.splits > 1 && piece <= 0 && threadIdx.x < heads) kv_part_counts(a, c, r)[sample * a.H + head0 + threadIdx.x] = which >= 0 ? pieces : 1;
    if (which < 0) {
      if (piece <= 0) for (int e = threadIdx.x; e < heads * HD; e += 64 * kWaves) out[e] = 0;
      continue;
    }
    // this lane's query: channels 32 s + 8 g + 0..7 for step s, as the keys' units have them
    bf16x8 qf[KI];
    const bf16_t* const q0 = (const bf16_t*)a.q + (long)sample * a.q_stride + (long)head0 * HD;
#pragma unroll
    for (int i = 0; i < KI; ++i) qf[i] = *reinterpret_cast<const bf16x8*>(q0 + (long)min(col, heads - 1) * HD + 32 * i + 8 * g);
    f32x4 o[VB];
#pragma unroll
    for (int b = 0; b < VB; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kKvNone, l = 0.f;
    const int begin = lo;
    int hi = lo;

    // A place that is no visible position stands for a visible one near it, the same page's where 16 are read together; its weight is zero.
    auto visible = [&](int pos, int low) __attribute__((always_inline)) { return min(pos < span.sinks || pos >= span.from ? pos : low, span.end - 1); };
    auto fetch = [&](Tile<HD>& t, int base) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int c16 = min(base + 16 * u, (hi - 1) & ~15);
        if constexpr (kWhole16) {
          const int p16 = span.position(c16), low = p16 < span.sinks ? span.sinks - 1 : span.from;
          const long row = list[(c16 - lo) >> 4];
          const char* const kp = (const char*)(data + row * HD);
          const char* const vp = kp + (long)c.pt * (2 * HD);
          const bool inside = p16 + 15 < span.sinks || (p16 >= span.from && p16 + 15 < span.end);
          unsigned k_at = col, v_at[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) v_at[j] = 4 * g + j;
          if (!inside) {
            k_at = visible(p16 + col, low) - p16;
#pragma unroll
            for (int j = 0; j < 4; ++j) v_at[j] = visible(p16 + 4 * g + j, low) - p16;
          }
#pragma unroll
          for (int i = 0; i < KI; ++i) t.k[u][i] = load_rows<kOnce, u32x4>(kp + (k_at * (2 * HD) + 16 * g + 64u * i));
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const char* const w = vp + (v_at[j] * (2 * HD) + 2 * VB * col);
            if constexpr (KI == 4) { const u32x4 x = load_rows<kOnce, u32x4>(w); t.v[u][j][0] = x.x; t.v[u][j][1] = x.y; t.v[u][j][2] = x.z; t.v[u][j][3] = x.w; }
            else { const u32x2 x = load_rows<kOnce, u32x2>(w); t.v[u][j][0] = x.x; t.v[u][j][1] = x.y; }
          }
        } else {
          const int last = hi - 1 - lo, at = base + 16 * u - lo;
          const bf16_t* const kp = data + list[min(at + col, last)] * HD + 8 * g;
#pragma unroll
          for (int i = 0; i < KI; ++i) t.k[u][i] = load_rows<kOnce, u32x4>(kp + 32 * i);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const bf16_t* const w = data + (list[min(at + 4 * g + j, last)] + c.pt) * HD + VB * col;
            if constexpr (KI == 4) { const u32x4 x = load_rows<kOnce, u32x4>(w); t.v[u][j][0] = x.x; t.v[u][j][1] = x.y; t.v[u][j][2] = x.z; t.v[u][j][3] = x.w; }
            else { const u32x2 x = load_rows<kOnce, u32x2>(w); t.v[u][j][0] = x.x; t.v[u][j][1] = x.y; }
          }
        }
      }
    };
    auto use = [&](Tile<HD>& t, int base) __attribute__((always_inline)) {
      float s[2][4], p[2][4];                                     // (scalars: hipcc has lost elements of a vector of which one was replaced under a condition)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KI; ++i) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t.k[u][i]), qf[i], x, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[u][j] = x[j] * a.scale;
      }
      const int p0 = span.position(base);                         // (32 places from here on lie next to each other, or the second 16 behind the gap)
      if (!(p0 + 31 < span.sinks || (base >= span.sinks16 && p0 >= span.from && p0 + 31 < span.end))) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            s[u][j] = span.sees(span.position(base + 16 * u) + 4 * g + j) ? s[u][j] : -INFINITY;
      }
      float top = -INFINITY;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, s[u][j]);
      // Weights are relative to m, which is raised - for all four lanes of a query alike - only when a score exceeds it by
      // 2^kRaise: the sum is divided out at the end, so any reference near the largest score does.
      if (__any(top > m + kRaise)) {
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float to = fmaxf(m, top), alpha = exp2_raw(m - to);
        m = to;
        l *= alpha;
#pragma unroll
        for (int b = 0; b < VB; ++b) o[b] *= alpha;
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          p[u][j] = exp2_raw(s[u][j] - m);
          l += p[u][j];
        }
      // A weight as two bf16 operands, its upper digits and what they leave, which is sixteen digits of it: one alone
      // would be off by as much as the rounding of the result.
      u32x4 hi_w;
      bf16x8 lo_w;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
          hi_w[2 * u + j / 2] = high_halves(p[u][j], p[u][j + 1]);
          lo_w[4 * u + j] = (__bf16)(p[u][j] - __uint_as_float(__float_as_uint(p[u][j]) & 0xFFFF0000u));
          lo_w[4 * u + j + 1] = (__bf16)(p[u][j + 1] - __uint_as_float(__float_as_uint(p[u][j + 1]) & 0xFFFF0000u));
        }
#pragma unroll
      for (int w = 0; w < VB / 2; ++w) {                          // two channel blocks of a word of the values
        u32x4 f[2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {                             // places 4 g + 2 (i % 2), + 1 of group i / 2
          const uint32_t lo_row = t.v[i >> 1][2 * (i & 1)][w], hi_row = t.v[i >> 1][2 * (i & 1) + 1][w];
          f[0][i] = __builtin_amdgcn_perm(hi_row, lo_row, 0x05040100u);
          f[1][i] = __builtin_amdgcn_perm(hi_row, lo_row, 0x07060302u);
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) o[2 * w + b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f[b]), __builtin_bit_cast(bf16x8, hi_w), o[2 * w + b], 0, 0, 0);
#pragma unroll
        for (int b = 0; b < 2; ++b) o[2 * w + b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f[b]), lo_w, o[2 * w + b], 0, 0, 0);
      }
    };

    // as many places at a time as the LDS holds rows of
    for (; lo < end; lo = hi) {
      hi = (int)min((long)end, (long)lo + kList * kGrain);
      const int n_list = (hi - lo + kGrain - 1) / kGrain;
      __syncthreads();                                             // the rows before are no longer needed
      if (threadIdx.x == 0) again = 0;
      for (int i = threadIdx.x; i < n_list; i += 64 * kWaves) {
        int pos = span.position(lo + kGrain * i);
        if constexpr (!kWhole16) pos = visible(pos, pos < span.from && lo + i < span.sinks16 ? max(span.sinks - 1, 0) : span.from);
        list[i] = kv8_row(c, kv8_checked_page(c, table[kv8_page_of(c, pos)]), kv, pos);
      }
      __syncthreads();
      // places lo + 32 (wave + kWaves i)
      for (int base = lo + 32 * wave; base < hi; base += 32 * kWaves) {
        Tile<HD> t;
        fetch(t, base);
        use(t, base);
      }
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    // lane (col, g) has channels VB (4 g + j) + b of query col in o[b][j]
    if (col < heads) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int w = 0; w < VB / 4; ++w)
          *reinterpret_cast<f32x4*>(fold + (wave * 16 + col) * OS + VB * (4 * g + j) + 4 * w) = f32x4{o[4 * w][j], o[4 * w + 1][j], o[4 * w + 2][j], o[4 * w + 3][j]};
      if (g == 0) { fold_m[wave][col] = m; fold_l[wave][col] = l; }
    }
    __syncthreads();
    bool strange = false;
    for (int e = 2 * threadIdx.x; e < heads * HD; e += 2 * 64 * kWaves) {
      const int q = e / HD, ch = e % HD;
      float to = kKvNone, ls = 0.f, s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) to = fmaxf(to, fold_m[w][q]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = exp2_raw(fold_m[w][q] - to);
        const float* x = fold + (w * 16 + q) * OS + ch;
        ls += fold_l[w][q] * f; s0 += x[0] * f; s1 += x[1] * f;
      }
      strange |= !(s0 - s0 == 0.f && s1 - s1 == 0.f) && ls - ls == 0.f;
      if (pieces == 1) {
        const float inv = 1.f / ls;
        *reinterpret_cast<uint32_t*>(out + e) = (uint32_t)f32_to_bf16(s0 * inv) | ((uint32_t)f32_to_bf16(s1 * inv) << 16);
      } else {
        float* part = kv_part_sums(a, c, sample * a.H + head0 + q, piece);
        part[ch] = s0; part[ch + 1] = s1;
        if (ch == 0) *kv_part_marks(a, c, r, sample * a.H + head0 + q, piece) = make_float2(to, ls);
      }
    }
    // Values that are not finite: a zero weight, or the lower digits of one, times infinity is no number here.  Once more by itself.
    if (__any(strange)) again = 1;
    __syncthreads();
    if (__builtin_expect(again, 0)) {
      constexpr int L = HD / 8;
      const int ch = 8 * (lane & (L - 1));
      for (int i = wave; i < heads; i += kWaves) {
        float q[8];
        KvType<bf16_t>::load8(q0 + (long)i * HD + ch, q);
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] *= a.scale;
        const KvSums x = kv_attend<bf16_t>(c, table, kv, span, q, L, ch, true, begin, 64 / L, end);
        if (lane >= L) continue;
        float* const part = kv_part_sums(a, c, sample * a.H + head0 + i, piece) + ch;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (pieces == 1) out[i * HD + ch + e] = f32_to_bf16(x.o[e] / x.l);
          else part[e] = x.o[e];
        }
        if (pieces > 1 && lane == 0) *kv_part_marks(a, c, r, sample * a.H + head0 + i, piece) = make_float2(x.m, x.l);
      }
    }
  }
}

template <int HD, bool kOnce>
void launch_decode(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a) {
  const int groups = kv8_groups(c, a.H);
  const dim3 grid((unsigned)(a.plan.wgs ? a.plan.wgs : r.n * c.K * groups)), block(64 * kWaves);
  if (c.pt % 16 == 0) hipLaunchKernelGGL((k_kv_decode<HD, true, kOnce>), grid, block, 0, s, c, r, a, groups);
  else hipLaunchKernelGGL((k_kv_decode<HD, false, kOnce>), grid, block, 0, s, c, r, a, groups);
}
template <int HD>
void launch_heads(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a) {
  if (kv_decode_once(c, r, a.sight)) launch_decode<HD, true>(s, c, r, a); else launch_decode<HD, false>(s, c, r, a);
}

}  // namespace

void launch_kv_decode(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a) {
  if (c.h == 128) launch_heads<128>(s, c, r, a); else launch_heads<64>(s, c, r, a);
}

}  // namespace mdi
