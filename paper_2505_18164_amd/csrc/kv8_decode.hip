// Attention of one new token per sample over the 8-bit cache, on the matrix cores.
//
// A workgroup takes one kv head of one sample and up to sixteen of its query heads (a unit), or a piece of its positions; its
// four wavefronts take 32 positions in turn, straight from the pages into registers.  Both products are computed transposed:
// S^T = K Q^T leaves, with v_mfma_f32_16x16x32_bf16, positions 4 g + r (g = lane / 16) of query lane % 16 in a lane, and two
// tiles of 16 positions side by side are just what O^T = V^T P^T takes as its second operand, if the positions that lane
// group g contracts are named 4 g .. 4 g + 3 of either tile.  The sum over positions is in no order, so any naming does; likewise
// the channels of K and Q.  So a key's codes are read 16 bytes a lane (four lanes a row, 64 bytes of it next to each other),
// a value's HD / 16 bytes a lane (sixteen lanes a row), and nothing has to be transposed: a code becomes bf16 by itself,
// whichever byte of whichever row's word it is (one conversion, and one byte permutation for two of them).
//
// What bounds it: memory.  A code takes 1.5 vector instructions, a score about ten; a wavefront spends 0.7 us on 32 positions,
// 40 % of the time that twelve of them on a compute unit have until the memory has answered, so that a second product for the lower
// digits of the weights (error of the results 0.0024 -> 0.0017 of their size, which is their own rounding) costs 0.7 us of 30.  Nothing is fetched ahead inside a
// wavefront: a second tile of registers (217 of them, two workgroups a compute unit) only made every load wait longer, the first ones of
// a unit - page numbers, query - included (8 samples of the 7B shape 42 us, 16 of the 8B shape 55).
// Shares instead of pieces of one length: 8 samples of 1 .. 4096 positions 41 -> 29.8 us at that step (a piece is as long as the longest
// sample's, and few of them are); what a unit costs to begin has to count, or 32 short ones after the other are one workgroup's (69 us).
// 16 samples of 8100 positions of the 8B shape: 47.9 us = 5.7 TB/s of codes and scales, 8 of the 7B shape 28.2 us = 4.7 TB/s.
#include <algorithm>
#include <type_traits>

#include "kv8_mfma.h"

namespace mdi {
namespace {

constexpr int kWaves = 4;
constexpr float kRaise = 8.f;        // how far (in powers of two) a score may exceed its query's reference before that is raised
constexpr int kPages = 1024;         // page numbers of a piece: chunk / pt + 2 at most

template <int HD> struct Tile {      // 32 positions of a wavefront
  u32x4 k[2][HD / 64];
  uint32_t v[2][4][HD / 64];
  f32x4 ks[2], vs[2];
};

// A cache that no later call finds in the last cache is read without a place in it.
template <bool kOnce, typename T> __device__ __forceinline__ T load_codes(const void* p) {
  if constexpr (kOnce) return __builtin_nontemporal_load((const T*)p); else return *(const T*)p;
}

// kWhole16: pages of a multiple of 16 positions, so 16 aligned positions lie in one page, next to each other.
template <int HD, bool kWhole16, bool kOnce>
__global__ __launch_bounds__(64 * kWaves, 3) void k_kv8_decode(Kv8Cache c, Kv8Rows r, Kv8Attn a, int groups) {
  constexpr int KI = HD / 64, VB = HD / 16;                      // 16-byte units of a key a lane has; bytes of a value (= channel blocks)
  constexpr int OS = HD + 4;
  __shared__ __attribute__((aligned(16))) float fold[kWaves * 16 * OS];
  __shared__ float fold_m[kWaves][16], fold_l[kWaves][16];
  __shared__ int pages[kPages];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
  const unsigned k_off = col * HD + 16 * g, v_off = 4 * g * HD + VB * col, s_off = 16 * g;
  const int units = c.K * groups, G = a.H / c.K;                  // units of a sample: a kv head's sixteen query heads
  int x0 = blockIdx.x, x1 = x0 + 1, per = 1, seen64 = 0;
  if (a.plan.wgs) {
    seen64 = kv8_seen(c, r, lane);
    const Kv8Stream all = kv8_stream(c, r, a.plan, units, 0, seen64);
    per = all.per;
    x0 = min(x0 * per, all.cost * units);
    x1 = min(x0 + per, all.cost * units);
  }
  while (x0 < x1) {
    int sample, unit, seen, piece = 0, pieces = 1, lo = 0, end;
    if (a.plan.wgs) {
      const Kv8Found f = kv8_find(c, r, x0 / units, seen64);
      sample = f.sample;
      seen = f.seen;
      const int tiles = kv8_tiles(seen), cost = tiles + kKv8Begin, in = x0 - f.start * units;
      unit = in / cost;
      // this share has x0 .. next - 1, the unit's tiles are from .. from + tiles - 1
      const int start = f.start * units + unit * cost, from = start + kKv8Begin, next = min(x1, start + cost), first_wg = from / per;
      lo = max(x0 - from, 0) * kKv8Tile;
      end = min(seen, max(next - from, 0) * kKv8Tile);
      piece = (int)blockIdx.x - first_wg;
      pieces = max(from + tiles - 1, from) / per - first_wg + 1;
      x0 = next;
      if (seen && lo >= end) continue;                           // only what it costs to begin: the tiles are another share's
    } else {
      sample = x0 / units;
      unit = x0 - sample * units;
      seen = end = __builtin_amdgcn_readfirstlane(kv8_seen(c, r, sample));
      x0 = x1;
    }
    const int kv = unit / groups, head0 = kv * G + 16 * (unit - kv * groups), heads = min(16, kv * G + G - head0);
    const int which = seen ? __builtin_amdgcn_readfirstlane(kv8_table_row(c, r, sample)) : -1;   // (who takes no part may have any table)
    const int32_t* table = c.tables + (long)max(which, 0) * c.table_stride;
    int at0 = kv8_page_of(c, lo);
    const int first = at0 + (int)threadIdx.x < c.table_stride ? table[at0 + threadIdx.x] : 0;
    bf16_t* out = a.out + (long)sample * a.out_stride + (long)head0 * HD;
    if (which < 0) {
      if (piece <= 0) for (int e = threadIdx.x; e < heads * HD; e += 64 * kWaves) out[e] = 0;
      continue;
    }
    // this lane's query: channels 64 i + 16 g + 8 s + 0..7 for steps 2 i + s, as the keys' units have them
    bf16x8 qf[2 * KI];
    {
      const bf16_t* q = a.q + (long)sample * a.q_stride + (long)(head0 + min(col, heads - 1)) * HD + 16 * g;
#pragma unroll
      for (int i = 0; i < KI; ++i)
#pragma unroll
        for (int s = 0; s < 2; ++s) qf[2 * i + s] = *reinterpret_cast<const bf16x8*>(q + 64 * i + 8 * s);
    }
    f32x4 o[VB];
#pragma unroll
    for (int b = 0; b < VB; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kKv8None, l = 0.f;
    int hi = lo;

    auto row_of = [&](int pos) __attribute__((always_inline)) {     // the key's row; the value's is pt further
      return kv8_row(c, pages[kv8_page_of(c, pos) - at0], kv, pos);
    };
    auto fetch = [&](Tile<HD>& t, int base) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if constexpr (kWhole16) {
          const int p16 = min(base + 16 * u, (hi - 1) & ~15);
          const long row = kv8_row(c, __builtin_amdgcn_readfirstlane(pages[kv8_page_of(c, p16) - at0]), kv, p16);
          // one uniform address each and 32-bit offsets of the lanes
          const char* kp = (const char*)c.codes + row * HD;
          const char* vp = kp + (long)c.pt * HD;
          const char* sk = (const char*)(c.scales + row);
          const char* sv = sk + 4l * c.pt;
#pragma unroll
          for (int i = 0; i < KI; ++i) t.k[u][i] = load_codes<kOnce, u32x4>(kp + (k_off + 64u * i));
          t.ks[u] = *reinterpret_cast<const f32x4*>(sk + s_off);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const char* w = vp + (v_off + (unsigned)(j * HD));
            if constexpr (KI == 2) { const u32x2 x = load_codes<kOnce, u32x2>(w); t.v[u][j][0] = x.x; t.v[u][j][1] = x.y; }
            else t.v[u][j][0] = load_codes<kOnce, uint32_t>(w);
          }
          t.vs[u] = *reinterpret_cast<const f32x4*>(sv + s_off);
        } else {
          const int8_t* kp = c.codes + row_of(min(base + 16 * u + col, hi - 1)) * HD;
#pragma unroll
          for (int i = 0; i < KI; ++i) t.k[u][i] = load_codes<kOnce, u32x4>(kp + 64 * i + 16 * g);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const long row = row_of(min(base + 16 * u + 4 * g + j, hi - 1));
            const uint32_t* w = reinterpret_cast<const uint32_t*>(c.codes + (row + c.pt) * HD + VB * col);
            if constexpr (KI == 2) { const u32x2 x = load_codes<kOnce, u32x2>(w); t.v[u][j][0] = x.x; t.v[u][j][1] = x.y; }
            else t.v[u][j][0] = load_codes<kOnce, uint32_t>(w);
            t.ks[u][j] = c.scales[row];
            t.vs[u][j] = c.scales[row + c.pt];
          }
        }
      }
    };
    auto use = [&](Tile<HD>& t, int base) __attribute__((always_inline)) {
      // What has been asked for is looked at from here on: a product or a shift that is moved up to a load waits for it there
      // (pages of 40 positions, one sample of 120001 of the 8B shape: 50 -> 69 us).
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float ks = t.ks[u][j], vs = t.vs[u][j];
          asm volatile("" : "+v"(ks), "+v"(vs));
          t.ks[u][j] = ks; t.vs[u][j] = vs;
#pragma unroll
          for (int w = 0; w < KI; ++w) asm volatile("" : "+v"(t.v[u][j][w]));
        }
      f32x4 s[2];
      float p[2][4];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        s[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KI; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t a0 = t.k[u][i][2 * h], a1 = t.k[u][i][2 * h + 1];
            const u32x4 f = {high_halves(code_of<0>(a0), code_of<1>(a0)), high_halves(code_of<2>(a0), code_of<3>(a0)),
                             high_halves(code_of<0>(a1), code_of<1>(a1)), high_halves(code_of<2>(a1), code_of<3>(a1))};
            s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), qf[2 * i + h], s[u], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);                     // (else every step's operands are made first, and spilled)
          }
        t.ks[u] *= a.scale;
      }
      if (base + 32 > hi) {                                        // what lies behind the last position counts for nothing, whatever it holds
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (base + 16 * u + 4 * g + j >= hi) { s[u][j] = -INFINITY; t.ks[u][j] = 1.f; t.vs[u][j] = 0.f; }
      }
      float top = -INFINITY;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, s[u][j] * t.ks[u][j]);
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
          p[u][j] = exp2_raw(fmaf(s[u][j], t.ks[u][j], -m));
          l += p[u][j];
          p[u][j] *= t.vs[u][j];
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
      for (int w = 0; w < KI; ++w) {
        auto operand = [&](auto byte) __attribute__((always_inline)) {
          constexpr int N = decltype(byte)::value;
          return __builtin_bit_cast(bf16x8, u32x4{high_halves(code_of<N>(t.v[0][0][w]), code_of<N>(t.v[0][1][w])), high_halves(code_of<N>(t.v[0][2][w]), code_of<N>(t.v[0][3][w])),
                                                  high_halves(code_of<N>(t.v[1][0][w]), code_of<N>(t.v[1][1][w])), high_halves(code_of<N>(t.v[1][2][w]), code_of<N>(t.v[1][3][w]))});
        };
        auto blocks = [&](auto byte) __attribute__((always_inline)) {   // two: a product waits for the one before it on the same sums
          constexpr int N = decltype(byte)::value;
          const bf16x8 f0 = operand(std::integral_constant<int, N>()), f1 = operand(std::integral_constant<int, N + 1>());
          f32x4 &o0 = o[4 * w + N], &o1 = o[4 * w + N + 1];
          o0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f0, __builtin_bit_cast(bf16x8, hi_w), o0, 0, 0, 0);
          o1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f1, __builtin_bit_cast(bf16x8, hi_w), o1, 0, 0, 0);
          o0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f0, lo_w, o0, 0, 0, 0);
          o1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f1, lo_w, o1, 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        };
        blocks(std::integral_constant<int, 0>());
        blocks(std::integral_constant<int, 2>());
      }
    };

    // as many positions at a time as the LDS holds page numbers of
    const int span = (kPages - 2) * c.pt / kKv8Tile * kKv8Tile;
    for (bool fresh = true; lo < end; lo = hi, fresh = false) {
      hi = (int)min((long)end, (long)lo + span);
      at0 = kv8_page_of(c, lo);
      const int n_at = kv8_page_of(c, hi - 1) - at0 + 1;
      __syncthreads();                                             // the numbers before are no longer needed
      for (int i = threadIdx.x; i < n_at; i += 64 * kWaves) pages[i] = kv8_checked_page(c, fresh && i < 64 * kWaves ? first : table[at0 + i]);
      __syncthreads();
      // tiles lo + 32 (wave + kWaves i)
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
        for (int w = 0; w < KI; ++w)
          *reinterpret_cast<f32x4*>(fold + (wave * 16 + col) * OS + VB * (4 * g + j) + 4 * w) = f32x4{o[4 * w][j], o[4 * w + 1][j], o[4 * w + 2][j], o[4 * w + 3][j]};
      if (g == 0) { fold_m[wave][col] = m; fold_l[wave][col] = l; }
    }
    __syncthreads();
    for (int e = 2 * threadIdx.x; e < heads * HD; e += 2 * 64 * kWaves) {
      const int q = e / HD, ch = e % HD;
      float to = kKv8None, ls = 0.f, s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) to = fmaxf(to, fold_m[w][q]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = exp2_raw(fold_m[w][q] - to);
        const float* x = fold + (w * 16 + q) * OS + ch;
        ls += fold_l[w][q] * f; s0 += x[0] * f; s1 += x[1] * f;
      }
      if (pieces == 1) {
        const float inv = 1.f / ls;
        *reinterpret_cast<uint32_t*>(out + e) = (uint32_t)f32_to_bf16(s0 * inv) | ((uint32_t)f32_to_bf16(s1 * inv) << 16);
      } else {
        float* part = kv8_part_sums(a, c, sample * a.H + head0 + q, piece);
        part[ch] = s0; part[ch + 1] = s1;
        if (ch == 0) *kv8_part_marks(a, c, r, sample * a.H + head0 + q, piece) = make_float2(to, ls);
      }
    }
  }
}

// Read once: more than half of what the last cache holds (256 MB), counting every sample as long as the longest may be.  16 samples of
// 8192 positions of the 8B shape 51.7 -> 47.9 us, one of 120001 51.0 -> 47.3, 8 of up to 4096 of the 7B shape 28.9 -> 28.2; but the same 4 samples of 8000 again and
// again, 68 MB, 22.2 -> 23.7, and 8 of 1000 of the 7B shape, 68 MB, 22.6 -> 23.3.
template <int HD, bool kOnce>
void launch_decode(hipStream_t s, const Kv8Cache& c, const Kv8Rows& r, const Kv8Attn& a) {
  const int groups = kv8_groups(c, a.H);
  const dim3 grid((unsigned)(a.plan.wgs ? a.plan.wgs : r.n * c.K * groups)), block(64 * kWaves);
  if (c.pt % 16 == 0) hipLaunchKernelGGL((k_kv8_decode<HD, true, kOnce>), grid, block, 0, s, c, r, a, groups);
  else hipLaunchKernelGGL((k_kv8_decode<HD, false, kOnce>), grid, block, 0, s, c, r, a, groups);
}
template <int HD>
void launch_heads(hipStream_t s, const Kv8Cache& c, const Kv8Rows& r, const Kv8Attn& a) {
  const bool once = (double)r.n * r.max_ctx * c.K * 2 * (HD + 4) > 128e6;
  if (once) launch_decode<HD, true>(s, c, r, a); else launch_decode<HD, false>(s, c, r, a);
}

}  // namespace

bool kv8_decode_supported(const Kv8Cache& c, const Kv8Rows& r) { return !r.start && (c.h == 64 || c.h == 128); }

// Workgroups of a call that is cut into shares: two on each of 256 compute units.  (Every one keeps 32 KiB on their way, and more of
// them only make each wait longer: 512 / 768 workgroups, 16 samples of 8100 positions of the 8B shape 53.3 / 54.4 us, 8 of 1 to
// 4096 of the 7B shape 29.8 / 30.8.)
constexpr int kShares = 512;
constexpr int kLeast = 2;            // tiles of a share, at least

// With many units, or short samples, a unit is a workgroup's.  Else the tiles of all units are cut into equal shares.
Kv8Plan kv8_decode_plan(const Kv8Cache& c, const Kv8Rows& r, int H) {
  const int each = c.K * kv8_groups(c, H);                       // units of a sample
  if ((long)r.n * each >= 4 * kShares || r.max_ctx <= kLeast * kKv8Tile) return Kv8Plan{r.max_ctx, 1, 0, 0};
  // a unit of t tiles in shares of at least kLeast, and of at least t * each / kShares (it is one of `each` alike)
  const int tiles = (r.max_ctx + kKv8Tile - 1) / kKv8Tile;
  return Kv8Plan{kLeast * kKv8Tile, std::min(tiles / kLeast, (kShares + each - 1) / each) + 2, kShares, 0};
}

void launch_kv8_decode(hipStream_t s, const Kv8Cache& c, const Kv8Rows& r, const Kv8Attn& a) {
  if (c.h == 128) launch_heads<128>(s, c, r, a); else launch_heads<64>(s, c, r, a);
}

}  // namespace mdi
