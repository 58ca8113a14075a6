// Attention of one new token per sample over the 8-bit cache, on the matrix cores.
//
// A workgroup takes one kv head of one sample, up to sixteen of its query heads and a piece of its positions; its four wavefronts
// take tiles of 32 positions in turn, straight from the pages into registers.  Both products are computed transposed:
// S^T = K Q^T leaves, with v_mfma_f32_16x16x32_bf16, positions 4 g + r (g = lane / 16) of query lane % 16 in a lane, and two
// tiles of 16 positions side by side are just what O^T = V^T P^T takes as its second operand, if the sixteen positions that lane
// group g contracts are named 4 g .. 4 g + 3 of either tile.  The sum over positions is in no order, so any naming does; likewise
// the channels of K and Q.  So a key's codes are read 16 bytes a lane (four lanes a row, 64 bytes of it next to each other),
// a value's HD / 16 bytes a lane (sixteen lanes a row), and the transposition of V costs nothing: a code becomes bf16 by itself, whichever byte
// of whichever row's word it is.
#include <algorithm>
#include <type_traits>

#include "kv8_mfma.h"

namespace mdi {
namespace {

constexpr int kWaves = 4;
constexpr int kPages = 1024;         // page numbers of a piece: chunk / pt + 2 at most

template <int HD> struct Tile {      // 32 positions of a wavefront
  u32x4 k[2][HD / 64];
  uint32_t v[2][4][HD / 64];
  f32x4 ks[2], vs[2];
};

// kWhole16: pages of a multiple of 16 positions, so 16 aligned positions lie in one page, next to each other.
template <int HD, bool kWhole16>
__global__ __launch_bounds__(64 * kWaves, 2) void k_kv8_decode(Kv8Cache c, Kv8Rows r, Kv8Attn a, int groups) {
  constexpr int KI = HD / 64, VB = HD / 16;                      // 16-byte units of a key a lane has; bytes of a value (= channel blocks)
  constexpr int OS = HD + 4;
  __shared__ __attribute__((aligned(16))) float fold[kWaves * 16 * OS];
  __shared__ float fold_m[kWaves][16], fold_l[kWaves][16];
  int* pages = (int*)fold;                                       // (done with before the fold begins)
  static_assert(kPages <= kWaves * 16 * OS, "page numbers fit");

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
  const int piece = blockIdx.x % a.plan.splits, unit = blockIdx.x / a.plan.splits;
  const int sample = unit / (c.K * groups), kvg = unit - sample * (c.K * groups), kv = kvg / groups, G = a.H / c.K;
  const int head0 = kv * G + 16 * (kvg - kv * groups), heads = min(16, kv * G + G - head0);
  const Kv8View view = kv8_view(c, r, sample);
  const int lo = piece * a.plan.chunk, hi = min(view.seen, lo + a.plan.chunk);
  if (lo >= hi && piece > 0) return;
  const int32_t* table = view.seen ? kv8_table(c, r, sample) : nullptr;
  bf16_t* out = a.out + (long)sample * a.out_stride + (long)head0 * HD;
  if (!table) {
    if (piece == 0) for (int e = threadIdx.x; e < heads * HD; e += 64 * kWaves) out[e] = 0;
    return;
  }

  const int at0 = kv8_page_of(c, lo), n_at = kv8_page_of(c, hi - 1) - at0 + 1;
  for (int i = threadIdx.x; i < n_at; i += 64 * kWaves) pages[i] = kv8_checked_page(c, table[at0 + i]);
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
  __syncthreads();

  auto row_of = [&](int pos) __attribute__((always_inline)) {     // the key's row; the value's is pt further
    const int at = kv8_page_of(c, pos);
    return ((long)pages[at - at0] * c.K + kv) * 2 * c.pt + (pos - at * c.pt);
  };
  auto fetch = [&](Tile<HD>& t, int base) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if constexpr (kWhole16) {
        const int p16 = min(base + 16 * u, (hi - 1) & ~15), at = kv8_page_of(c, p16);
        const int page = __builtin_amdgcn_readfirstlane(pages[at - at0]);
        const long row = ((long)page * c.K + kv) * 2 * c.pt + (p16 - at * c.pt);
        const int8_t* kp = c.codes + row * HD;
        const int8_t* vp = kp + (long)c.pt * HD;
#pragma unroll
        for (int i = 0; i < KI; ++i) t.k[u][i] = *reinterpret_cast<const u32x4*>(kp + col * HD + 64 * i + 16 * g);
        const float* sp = c.scales + row + 4 * g;
        t.ks[u] = *reinterpret_cast<const f32x4*>(sp);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t* w = reinterpret_cast<const uint32_t*>(vp + (4 * g + j) * HD + VB * col);
          if constexpr (KI == 2) { const u32x2 x = *reinterpret_cast<const u32x2*>(w); t.v[u][j][0] = x.x; t.v[u][j][1] = x.y; }
          else t.v[u][j][0] = *w;
        }
        t.vs[u] = *reinterpret_cast<const f32x4*>(sp + c.pt);
      } else {
        const int8_t* kp = c.codes + row_of(min(base + 16 * u + col, hi - 1)) * HD;
#pragma unroll
        for (int i = 0; i < KI; ++i) t.k[u][i] = *reinterpret_cast<const u32x4*>(kp + 64 * i + 16 * g);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const long row = row_of(min(base + 16 * u + 4 * g + j, hi - 1));
          const uint32_t* w = reinterpret_cast<const uint32_t*>(c.codes + (row + c.pt) * HD + VB * col);
          if constexpr (KI == 2) { const u32x2 x = *reinterpret_cast<const u32x2*>(w); t.v[u][j][0] = x.x; t.v[u][j][1] = x.y; }
          else t.v[u][j][0] = *w;
          t.ks[u][j] = c.scales[row];
          t.vs[u][j] = c.scales[row + c.pt];
        }
      }
    }
  };
  auto use = [&](Tile<HD>& t, int base) __attribute__((always_inline)) {
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
        }
      t.ks[u] *= a.scale;
    }
    __builtin_amdgcn_sched_barrier(0);
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
    // 2^kKv8Raise: the sum is divided out at the end, so any reference near the largest score does.
    if (__any(top > m + kKv8Raise)) {
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
    bf16x8 pf;                                                   // the one rounding of a weight: to the matrix cores' operand
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) pf[4 * u + j] = (__bf16)p[u][j];
#pragma unroll
    for (int w = 0; w < KI; ++w) {
      auto block = [&](auto byte) __attribute__((always_inline)) {
        constexpr int N = decltype(byte)::value;
        const u32x4 f = {high_halves(code_of<N>(t.v[0][0][w]), code_of<N>(t.v[0][1][w])), high_halves(code_of<N>(t.v[0][2][w]), code_of<N>(t.v[0][3][w])),
                         high_halves(code_of<N>(t.v[1][0][w]), code_of<N>(t.v[1][1][w])), high_halves(code_of<N>(t.v[1][2][w]), code_of<N>(t.v[1][3][w]))};
        o[4 * w + N] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), pf, o[4 * w + N], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);                       // (else every block's operands are made first, and spilled)
      };
      block(std::integral_constant<int, 0>());
      block(std::integral_constant<int, 1>());
      block(std::integral_constant<int, 2>());
      block(std::integral_constant<int, 3>());
    }
  };

  // tiles lo + 32 (wave + kWaves i), the next one on its way while one is used
  int base = lo + 32 * wave;
  if (base < hi) {
    Tile<HD> t0, t1;
    fetch(t0, base);
    for (;;) {
      const int next = base + 32 * kWaves, after = next + 32 * kWaves;
      if (next < hi) fetch(t1, next);
      use(t0, base);
      if (next >= hi) break;
      if (after < hi) fetch(t0, after);
      use(t1, next);
      if (after >= hi) break;
      base = after;
    }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  __syncthreads();                                               // the page numbers are no longer needed
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
  const bool whole = view.seen <= a.plan.chunk;
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
    if (whole) {
      const float inv = 1.f / ls;
      *reinterpret_cast<uint32_t*>(out + e) = (uint32_t)f32_to_bf16(s0 * inv) | ((uint32_t)f32_to_bf16(s1 * inv) << 16);
    } else {
      float* part = a.part + (((long)sample * a.H + head0 + q) * a.plan.splits + piece) * (HD + 4);
      part[ch] = s0; part[ch + 1] = s1;
      if (ch == 0) { part[HD] = to; part[HD + 1] = ls; }
    }
  }
}

template <int HD>
void launch_decode(hipStream_t s, const Kv8Cache& c, const Kv8Rows& r, const Kv8Attn& a) {
  const int groups = (a.H / c.K + 15) / 16;
  const dim3 grid((unsigned)((long)r.n * c.K * groups * a.plan.splits)), block(64 * kWaves);
  if (c.pt % 16 == 0) hipLaunchKernelGGL((k_kv8_decode<HD, true>), grid, block, 0, s, c, r, a, groups);
  else hipLaunchKernelGGL((k_kv8_decode<HD, false>), grid, block, 0, s, c, r, a, groups);
}

}  // namespace

bool kv8_decode_supported(const Kv8Cache& c, const Kv8Rows& r) { return !r.start && (c.h == 64 || c.h == 128); }

Kv8Plan kv8_decode_plan(const Kv8Cache& c, const Kv8Rows& r, int H) {
  const long units = (long)r.n * c.K * ((H / c.K + 15) / 16);
  const int want = (int)std::max<long>(1, std::min<long>(256, 2048 / units));
  int chunk = std::max(256, (r.max_ctx + want - 1) / want);
  chunk = std::min(chunk, std::min(4096, (kPages - 2) * c.pt));
  chunk = std::max(128, chunk / 128 * 128);
  return Kv8Plan{chunk, (r.max_ctx + chunk - 1) / chunk};
}

void launch_kv8_decode(hipStream_t s, const Kv8Cache& c, const Kv8Rows& r, const Kv8Attn& a) {
  if (c.h == 128) launch_decode<128>(s, c, r, a); else launch_decode<64>(s, c, r, a);
}

}  // namespace mdi
