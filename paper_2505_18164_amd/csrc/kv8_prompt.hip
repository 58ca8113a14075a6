// Causal attention of packed rows - prompts, or the next pieces of prompts, of several samples - over the 8-bit cache, on the
// matrix cores.
#include <algorithm>
#include <cstdlib>

#include "kv8_mfma.h"

namespace mdi {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr int BK = 64;               // keys of a step

__device__ __forceinline__ u32x2 read_transposed(const bf16_t* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)p));
}

// Rows of sample i, 0 <= first <= end <= n_rows whatever `start` holds.
struct Span { int first, end; };
__device__ __forceinline__ Span rows_of(const Kv8Rows& r, int i) {
  const int first = min(max(r.start[i], 0), r.n_rows);
  return Span{first, min(max(r.start[i + 1], first), r.n_rows)};
}

// The sample that has block x, counting BP positions a block, and which of its blocks that is; sample < 0: there are fewer.
struct BlockPlace { int sample, block, first, rows; };
template <int BQ>
__device__ __forceinline__ BlockPlace place_of(const Kv8Rows& r, int x, int g_sh) {
  const int lane = threadIdx.x & 63, bp = BQ >> g_sh;
  for (int base = 0, sum = 0; base < r.n; base += 64) {
    const Span s = base + lane < r.n ? rows_of(r, base + lane) : Span{0, 0};
    const int t = (s.end - s.first + bp - 1) / bp;
    int up = t;
    for (int off = 1; off < 64; off <<= 1) { const int o = __shfl_up(up, off, 64); if (lane >= off) up += o; }
    const unsigned long long past = __ballot(sum + up > x);
    if (past) {
      const int at = __ffsll(past) - 1;
      return BlockPlace{__builtin_amdgcn_readfirstlane(base + at), __builtin_amdgcn_readfirstlane(x - (sum + __shfl(up - t, at, 64))),
                        __builtin_amdgcn_readfirstlane(__shfl(s.first, at, 64)), __builtin_amdgcn_readfirstlane(__shfl(s.end - s.first, at, 64))};
    }
    sum += __shfl(up, 63, 64);
  }
  return BlockPlace{-1, 0, 0, 0};
}

struct PromptGeo { int n_blocks, sets, g_sh; };                  // bound of the blocks of all samples; sets of 2^g_sh query heads

template <int HD, int NG, int WQ>
__global__ __launch_bounds__(WQ * 64 * NG, 2) void k_kv8_prompt(Kv8Cache c, Kv8Rows r, Kv8Attn a, PromptGeo geo) {
  constexpr int BQ = 32 * WQ, GT = 64 * WQ;                      // rows of a workgroup - (position, head) pairs -, threads of a group
  constexpr int KS = HD + 8, VR = HD + 32, HT = HD / 32;
  constexpr int UB = 64 * HD / GT < 16 ? 64 * HD / GT : 16;      // codes a thread moves at a time
  constexpr int KU = 64 * HD / (GT * UB), PER = HD / UB;         // ... and how often; threads a key
  constexpr int KV = BK * KS + BK * VR + 4 * BK;                 // bf16 elements of a buffer: keys, values, their scales
  constexpr int NB = NG == 4 ? 1 : 2;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];

  const int tid = threadIdx.x & (GT - 1), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = NG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / GT);
  bf16_t* bufs = (bf16_t*)smem + grp * NB * KV;
  // Workgroups are handed to the eight compute dies in turn, each with an L2 of its own: a die takes sets that follow each
  // other (sets share keys), a sample's longest rows first.
  const int total = geo.n_blocks * geo.sets, per_die = (total + 7) >> 3, idx = (blockIdx.x & 7) * per_die + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per_die || idx >= total) return;
  const int set = idx / geo.n_blocks;
  const BlockPlace at = place_of<BQ>(r, idx - set * geo.n_blocks, geo.g_sh);
  if (at.sample < 0) return;
  const int g_sh = geo.g_sh, bp = BQ >> g_sh, head0 = set << g_sh, kv = head0 / (a.H / c.K);
  const int q0 = ((at.rows + bp - 1) / bp - 1 - at.block) * bp;  // first row of the sample in this block
  const int which = __builtin_amdgcn_readfirstlane(kv8_table_row(c, r, at.sample)), p0 = __builtin_amdgcn_readfirstlane(r.pos[at.sample]);
  const int32_t* table = c.tables + (long)max(which, 0) * c.table_stride;
  const int col = lane & 31, half = lane >> 5;
  const int row = q0 + ((32 * wave + col) >> g_sh), head = head0 + (col & ((1 << g_sh) - 1));   // (32 is a multiple of 2^g_sh)
  const bool live = row < at.rows;
  bf16_t* out = a.out + (long)(at.first + row) * a.out_stride + (long)head * HD;
  if (p0 < 0 || which < 0) {                                     // takes no part
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
  {
    const bf16_t* qp = a.q + (long)(at.first + min(row, at.rows - 1)) * a.q_stride + (long)head * HD + 8 * half;
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(qp + 16 * ks);
  }
  f32x16 o[HT];
#pragma unroll
  for (int i = 0; i < HT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  float m = kKv8None, l = 0.f;
  const int wave_pos = (int)min((long)p0 + q0 + ((32 * wave) >> g_sh), (long)r.max_ctx - 1);   // of the wavefront's first row

  const int n_kb = (hi - lo + BK - 1) / BK, n_it = (n_kb + NG - 1) / NG;
  u32x4 kreg[KU], vreg[KU];
  int pg[KU], pgs;
  float sreg;
  auto key_of = [&](int kb, int in) __attribute__((always_inline)) { return min(lo + kb * BK + in, hi - 1); };   // keys past the last repeat it
  auto pages = [&](int kb) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < KU; ++j) pg[j] = table[kv8_page_of(c, key_of(kb, (tid + j * GT) / PER))];
    pgs = table[kv8_page_of(c, key_of(kb, tid & 63))];
  };
  auto row_at = [&](int page, int key) __attribute__((always_inline)) {
    return ((long)kv8_checked_page(c, page) * c.K + kv) * 2 * c.pt + (key - kv8_page_of(c, key) * c.pt);
  };
  auto fetch = [&](int kb) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < KU; ++j) {
      const int u = tid + j * GT;
      const int8_t* kp = c.codes + row_at(pg[j], key_of(kb, u / PER)) * HD + UB * (u % PER);
      const int8_t* vp = kp + (long)c.pt * HD;
      if constexpr (UB == 16) {
        kreg[j] = *reinterpret_cast<const u32x4*>(kp);
        vreg[j] = *reinterpret_cast<const u32x4*>(vp);
      } else {
        const u32x2 x = *reinterpret_cast<const u32x2*>(kp), y = *reinterpret_cast<const u32x2*>(vp);
        kreg[j] = u32x4{x.x, x.y, 0, 0};
        vreg[j] = u32x4{y.x, y.y, 0, 0};
      }
    }
    sreg = tid < 128 ? c.scales[row_at(pgs, key_of(kb, tid & 63)) + (tid < 64 ? 0 : c.pt)] : 0.f;
    pages(kb + NG);
  };
  auto widen = [&](bf16_t* to, const u32x4& x) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < UB / 8; ++h) {
      const uint32_t w0 = x[2 * h], w1 = x[2 * h + 1];
      *reinterpret_cast<u32x4*>(to + 8 * h) = u32x4{high_halves(code_of<0>(w0), code_of<1>(w0)), high_halves(code_of<2>(w0), code_of<3>(w0)),
                                                    high_halves(code_of<0>(w1), code_of<1>(w1)), high_halves(code_of<2>(w1), code_of<3>(w1))};
    }
  };
  auto stash = [&](bf16_t* Ks) __attribute__((always_inline)) {
    bf16_t* Vs = Ks + BK * KS;
    float* sc = (float*)(Vs + BK * VR);
#pragma unroll
    for (int j = 0; j < KU; ++j) {
      const int u = tid + j * GT, key = u / PER, ch = UB * (u % PER);
      widen(Ks + key * KS + ch, kreg[j]);
      widen(Vs + key * VR + ch, vreg[j]);
    }
    if (tid < 128) sc[tid] = tid < 64 ? sreg * a.scale : sreg;
  };

  const int v_lane = (4 * half + ((lane & 15) >> 2)) * VR + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  pages(grp);
  fetch(grp);
  stash(bufs);
  __syncthreads();
  for (int it = 0; it < n_it; ++it) {
    const int kb = NG * it + grp;
    const bf16_t* Ks = bufs + (NB == 2 ? it & 1 : 0) * KV;
    const bf16_t* Vs = Ks + BK * KS;
    const float* sc = (const float*)(Vs + BK * VR);
    if (it + 1 < n_it) fetch(kb + NG);
    const int k0 = lo + kb * BK;
    const int last_pos = min(wave_pos + (31 >> g_sh), n_seen - 1);
    if (kb < n_kb && k0 <= last_pos) {                           // else: no block, or this wavefront's rows see none of these keys
      f32x16 s[2], x[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
        const bf16_t* kr = Ks + (32 * t + col) * KS + 8 * half;
#pragma unroll
        for (int ks = 0; ks < HD / 16; ++ks)
          s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(kr + 16 * ks), qf[ks], s[t], 0, 0, 0);
      }
      const bool masked = k0 + BK - 1 > wave_pos || k0 + BK > hi;
      auto count = [&]() __attribute__((always_inline)) {        // scores counted from m, and the largest
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const f32x4 ks = *reinterpret_cast<const f32x4*>(sc + 32 * t + 8 * g + 4 * half);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[t][4 * g + j] = fmaf(s[t][4 * g + j], ks[j], -m);
          }
        if (masked)
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int key = k0 + 32 * t + 8 * (e >> 2) + 4 * half + (e & 3);
              if (key > pos || key >= hi) x[t][e] = -INFINITY;
            }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) top = fmaxf(top, x[t][e]);
        return top;
      };
      float top = count();
      if (__any(top > kKv8Raise)) {
        // the largest score itself, not counted from an m that may lie far from it
        const float was = m;
        m = 0.f;
        top = count();
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        m = fmaxf(was, top);
        const float alpha = exp2_raw(was - m);
        l *= alpha;
#pragma unroll
        for (int i = 0; i < HT; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[i][e] *= alpha;
        count();
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int pp = 0; pp < 2; ++pp) {
          bf16x8 pf;
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const f32x4 vs = *reinterpret_cast<const f32x4*>(sc + BK + 32 * t + 16 * pp + 8 * g + 4 * half);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int e = 8 * pp + 4 * g + j;
              const float p = exp2_raw(x[t][e]);
              l += p;
              float w = p * vs[j];
              if (masked) {
                const int key = k0 + 32 * t + 8 * (e >> 2) + 4 * half + (e & 3);
                if (key > pos || key >= hi) w = 0.f;             // whatever its scale is
              }
              pf[4 * g + j] = (__bf16)w;
            }
          }
#pragma unroll
          for (int i = 0; i < HT; ++i) {
            const bf16_t* vr = Vs + v_lane + (32 * t + 16 * pp) * VR + 32 * i;
            const u32x2 b0 = read_transposed(vr), b1 = read_transposed(vr + 8 * VR);
            const u32x4 vf = {b0.x, b0.y, b1.x, b1.y};
            o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf), pf, o[i], 0, 0, 0);
          }
        }
    }
    if (NB == 1) __syncthreads();
    if (it + 1 < n_it) stash(bufs + (NB == 2 ? (it + 1) & 1 : 0) * KV);
    __syncthreads();
  }

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

template <int HD, int NG, int WQ>
constexpr size_t prompt_lds() {
  const size_t kv = (size_t)NG * (NG == 4 ? 1 : 2) * (BK * (HD + 8 + HD + 32) + 4 * BK) * sizeof(bf16_t);
  const size_t fold = NG > 1 ? (size_t)(NG - 1) * (HD / 2 + 2) * 64 * WQ * sizeof(float) : 0;
  return kv > fold ? kv : fold;
}
template <int HD, int NG, int WQ>
bool allow_one() {                                               // 64 KiB is what a kernel gets by default
  constexpr size_t lds = prompt_lds<HD, NG, WQ>();
  return lds <= 64 * 1024 || hipFuncSetAttribute((const void*)k_kv8_prompt<HD, NG, WQ>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) == hipSuccess;
}
template <int HD>
bool allow_heads() { return allow_one<HD, 1, 8>() && allow_one<HD, 2, 4>() && allow_one<HD, 4, 2>() && allow_one<HD, 1, 4>(); }

// Query heads of a kv head that a workgroup's rows take together: the largest power of two that divides their number, up to 32.
int heads_shift(const Kv8Cache& c, int H) {
  const int G = H / c.K;
  int sh = 0;
  while (sh < 5 && G % (2 << sh) == 0) ++sh;
  return sh;
}
PromptGeo geo_of(const Kv8Cache& c, const Kv8Rows& r, int H, int WQ) {
  const int sh = heads_shift(c, H), bp = 32 * WQ >> sh;
  return PromptGeo{r.n_rows / bp + std::min(r.n, r.n_rows), H >> sh, sh};
}
struct Shape { int groups, waves; };
Shape shape_of(const Kv8Cache& c, const Kv8Rows& r, int H) {
  if (const char* e = getenv("KV8_SHAPE")) return Shape{e[0] - '0', e[1] - '0'};
  return Shape{1, 8};
}

template <int HD, int NG, int WQ>
void launch_shape(hipStream_t s, const Kv8Cache& c, const Kv8Rows& r, const Kv8Attn& a) {
  const PromptGeo g = geo_of(c, r, a.H, WQ);
  const long total = (long)g.n_blocks * g.sets;
  hipLaunchKernelGGL((k_kv8_prompt<HD, NG, WQ>), dim3((unsigned)(8 * ((total + 7) / 8)), a.plan.splits), dim3(64 * WQ * NG), (prompt_lds<HD, NG, WQ>()), s, c, r, a, g);
}
template <int HD>
void launch_heads(hipStream_t s, const Kv8Cache& c, const Kv8Rows& r, const Kv8Attn& a) {
  const Shape p = shape_of(c, r, a.H);
  if (p.groups == 1 && p.waves == 8) launch_shape<HD, 1, 8>(s, c, r, a);
  else if (p.groups == 1) launch_shape<HD, 1, 4>(s, c, r, a);
  else if (p.groups == 2) launch_shape<HD, 2, 4>(s, c, r, a);
  else launch_shape<HD, 4, 2>(s, c, r, a);
}

}  // namespace

bool kv8_prompt_supported(const Kv8Cache& c, const Kv8Rows& r) { return r.start && (c.h == 64 || c.h == 128); }
bool kv8_prompt_allow_lds() { return allow_heads<64>() && allow_heads<128>(); }

Kv8Plan kv8_prompt_plan(const Kv8Cache& c, const Kv8Rows& r, int H) {
  const char* e = getenv("KV8_SPLIT");
  const int want = e ? atoi(e) : 1;
  const int chunk = ((r.max_ctx + want - 1) / want + BK - 1) / BK * BK;
  return Kv8Plan{chunk, (r.max_ctx + chunk - 1) / chunk, 0};
}

void launch_kv8_prompt(hipStream_t s, const Kv8Cache& c, const Kv8Rows& r, const Kv8Attn& a) {
  if (c.h == 128) launch_heads<128>(s, c, r, a); else launch_heads<64>(s, c, r, a);
}

}  // namespace mdi
