// Attention of packed rows - prompts, or the next pieces of prompts, of several samples - over the bf16 cache, on the matrix cores: heads
// of 64, and the launches of these and of heads of 128 (kv_prompt_wide.hip).  Few rows are kv_any.hip's.
//
// A workgroup is one group of eight wavefronts or two of four; a group's wavefronts take 32 rows of (position, query head) each, the heads of
// one kv head side by side, and pass over the keys they see 64 at a time (KvBlocks), two groups over every other 64 of the same rows' keys.  A wavefront computes S^T = K Q^T with v_mfma_f32_32x32x16_bf16, weighs the scores
// against a reference of its row, and adds O^T += V^T P^T: the scores of a query lie in the lane, and in the order, in which the second
// product takes weights, so they never leave the registers.  Keys and values travel from the pages to the LDS without passing
// registers, a block ahead, 16 bytes a lane; the 16-byte units of a row are permuted by the row's number (the permutation is
// applied to the address in memory, the LDS then holds it for free), which spreads both kinds of reads over all banks.
//
// A weight is two operands of the second product, sixteen digits of it (PromptWeights), half as many matrix instructions again; as one it would be
// off by up to 2^-8, and results by 0.0020 of their size instead of the 0.0017 that are their own rounding.
// 8 prompts of 333 rows of TinyLlama 28 us, one of 4000 127, 0.51 PFLOP/s (weights of one operand: 25 and 98): a step of 64 keys takes
// 1.7 us, the matrix instructions of it 0.84, exponentials of one wavefront of a SIMD beside the products of the other.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kv_prompt_device.h"
#include "once_per_device.h"

namespace mdi {
namespace {

// A workgroup is eight wavefronts: NG groups of WQ, which work on the same 32 WQ rows; group g takes the key blocks NG i + g.
// kWhole: pages of a multiple of 64 positions, so that a block of keys lies in one.  kMany: of more than kInOrder samples.
template <int NG, bool kWhole, bool kMany>
__global__ __launch_bounds__(512, 2) void k_kv_prompt(KvCache c, KvRows r, KvAttn a, PromptGeo geo) {
  constexpr int HD = 64, WQ = 8 / NG, BQ = 32 * WQ, GT = 64 * WQ;   // rows of a workgroup - (position, head) pairs -, threads of a group
  constexpr int HT = HD / 32, RB = 2 * HD, UN = HD / 8;          // bytes and 16-byte units of a key
  constexpr int BB = BK * RB;                                    // bytes of a block of keys, or of values
  constexpr int KP = 64 / UN, NI = BK / KP / WQ;                 // keys of an instruction that loads, instructions of a wavefront
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  __shared__ int again;

  const int tid = threadIdx.x & (GT - 1), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = NG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / GT), late = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
  const uint32_t Kb = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)smem + grp * 4 * BB, Vb = Kb + 2 * BB;
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
  if (which < 0) {                                               // takes no part
    if (blockIdx.y == 0 && grp == 0 && live) prompt_zeros<HT>(c, r, a, at, row, head);
    return;
  }
  // positions up to `pos` are seen by this lane's row; the block's rows end before `far`
  const long far = (long)p0 + min(q0 + bp, at.rows);
  if (far > r.max_ctx) kv8_report(c);
  const int pos = (int)min((long)p0 + min(row, at.rows - 1), (long)r.max_ctx - 1);
  const KvBlocks kb = kv_blocks(a.sight, (int)min((long)p0 + q0, (long)r.max_ctx - 1), (int)min(far, (long)r.max_ctx));
  const int b_lo = blockIdx.y * a.plan.chunk, b_hi = (int)min((long)kb.n, (long)b_lo + a.plan.chunk), pieces = (kb.n + a.plan.chunk - 1) / a.plan.chunk;
  if (b_lo >= b_hi) return;
  const PromptRows mine{at, g_sh, head0, kv, q0, p0, table, kb, (int)blockIdx.y, b_lo, b_hi, pieces};

  bf16x8 qf[HD / 16];
  f32x16 o[HT];
#pragma unroll
  for (int i = 0; i < HT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  float m = kKvNone, l = 0.f;
  const float scale = a.scale == 0.f ? 1.f : fabsf(a.scale);
  const int wave_pos = (int)min((long)p0 + min(q0 + ((32 * wave) >> g_sh), at.rows - 1), (long)r.max_ctx - 1);   // of the wavefront's first row
  const int last_pos = (int)min((long)p0 + min(q0 + ((32 * wave + 31) >> g_sh), at.rows - 1), (long)r.max_ctx - 1);

  // Loading.  Stage j: the keys of block j and the values of block j - 1.  A position that no row of the workgroup sees is not read, one
  // near it in its place.
  const int n_it = (b_hi - b_lo + NG - 1) / NG;
  auto block_of = [&](int j) __attribute__((always_inline)) { return min(b_lo + NG * j + grp, b_hi - 1); };
  auto start_of = [&](int b) __attribute__((always_inline)) { return b < kb.n_sinks ? b << 6 : kb.first + ((b - kb.n_sinks) << 6); };
  auto visible = [&](int p, int k0) __attribute__((always_inline)) {
    return min(p < kb.sinks || p >= kb.from ? p : k0 < kb.sinks ? kb.sinks - 1 : kb.from, kb.end - 1);
  };
  // lane's key of instruction n, and where in it the 16 bytes are that land at its place
  auto key_of = [&](int n) __attribute__((always_inline)) { return (wave * NI + n) * KP + lane / UN; };
  auto unit_of = [&](int key) __attribute__((always_inline)) {
    return (lane % UN) ^ ((((key >> 1) & 1) << 2) | ((key >> 2) & 3));
  };
  unsigned worst = 0;                                            // a page that is not of the cache is looked for at the end, the last one read in its place
  auto checked = [&](int page) __attribute__((always_inline)) {
    worst = max(worst, (unsigned)page);
    return min((unsigned)page, (unsigned)c.n_pages - 1);
  };
  int pg[kWhole ? 1 : NI];
  uint32_t v_off[kWhole ? NI : 1] = {};
  const char* v_at[kWhole ? 1 : NI] = {};
  const long v_by = (long)c.pt * RB;                             // from a key to its value
  auto pages = [&](int j) __attribute__((always_inline)) {
    const int k0 = start_of(block_of(j));
    if constexpr (kWhole) {
      int p = kv8_page_of(c, k0);
      asm volatile("" : "+v"(p));                                // a vector load: behind a scalar one every read of LDS would have to wait for it
      pg[0] = table[p];
    } else {
#pragma unroll
      for (int n = 0; n < NI; ++n) pg[n] = table[kv8_page_of(c, visible(k0 + key_of(n), k0))];
    }
  };
  auto issue = [&](int j) __attribute__((always_inline)) {
    const int k0 = start_of(block_of(j));
    const uint32_t k_lds = Kb + (j & 1) * BB + wave * NI * 1024, v_lds = Vb + ((j - 1) & 1) * BB + wave * NI * 1024;
    if constexpr (kWhole) {
      // (the page's number is looked at before anything else is asked for: whoever waits for it waits for that, too)
      unsigned page = __builtin_amdgcn_readfirstlane((int)checked(pg[0]));
      asm volatile("" : "+s"(page));
      pages(j + 1);
      if (j > 0)
#pragma unroll
        for (int n = 0; n < NI; ++n) dma(v_lds + 1024 * n, v_at[0], v_off[n]);
      const int in_page = k0 - kv8_page_of(c, k0) * c.pt;
      const char* const kp = (const char*)c.data + ((long)((uint64_t)page * (unsigned)(2 * c.K * c.pt)) + 2 * kv * c.pt + in_page) * RB;
      const bool inside = (k0 >= kb.from && k0 + BK <= kb.end) || k0 + BK <= kb.sinks;
#pragma unroll
      for (int n = 0; n < NI; ++n) {
        int key = key_of(n);
        const int unit = unit_of(key);
        if (!inside) key = visible(k0 + key, k0) - k0;
        v_off[n] = (uint32_t)(key * RB + 16 * unit);
        dma(k_lds + 1024 * n, kp, v_off[n]);
      }
      v_at[0] = kp + v_by;
    } else {
      const char* kp[NI];
#pragma unroll
      for (int n = 0; n < NI; ++n) {
        const int key = key_of(n);
        kp[n] = (const char*)c.data + kv8_row(c, checked(pg[n]), kv, visible(k0 + key, k0)) * RB + 16 * unit_of(key);
        asm volatile("" : "+v"(kp[n]));
      }
      pages(j + 1);
#pragma unroll
      for (int n = 0; n < NI; ++n) {
        if (j > 0) dma(v_lds + 1024 * n, v_at[n]);
        dma(k_lds + 1024 * n, kp[n]);
        v_at[n] = kp[n] + v_by;
      }
    }
  };

  // what this lane reads: keys `col` and col + 32, 16 bytes at channels 16 ks + 8 half; values 4 half + kk and 8 further, of every 16 keys,
  // 8 bytes at channels 32 i + 16 ((lane / 16) mod 2) + 4 (lane mod 4)
  const int kk = (lane & 15) >> 2;
  const uint32_t k_lane = col * RB + 16 * (half ^ ((((col >> 1) & 1) << 2) | ((col >> 2) & 3)));
  const uint32_t v_lane = (4 * half + kk) * RB + 64 * (kk >> 1) + 16 * ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ half) + 8 * (lane & 1);

  auto sees = [&](int j) __attribute__((always_inline)) {        // some row of the wavefront, some key of the block
    if (b_lo + NG * j + grp >= b_hi) return false;
    const int k0 = start_of(block_of(j));
    return k0 <= last_pos && (k0 + BK - 1 > wave_pos - a.sight.window || k0 < a.sight.sinks);
  };
  f32x16 s[2];
  PromptWeights<4> pf = {};
  // The products of a step: the values of block j - 1 with its weights, the keys of block j with the queries.  Four operands are
  // on their way from the LDS while the four before them are multiplied.
  auto products = [&](int j, auto keys) __attribute__((always_inline)) {
    constexpr int kSets = decltype(keys)::value ? 2 * HT : HT;   // sets of four operands: HT of values, HT of keys
    const uint32_t V = Vb + ((j - 1) & 1) * BB + v_lane, K = Kb + (j & 1) * BB + k_lane;
    u32x4 f[2][4];
    auto read = [&](int n) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if (n < HT) {
          const uint32_t p = (V ^ (64 * (x % HT))) + 16 * ((4 * n + x) / HT) * RB;
          const u32x2 b0 = read_transposed(p), b1 = read_transposed((p ^ 32) + 8 * RB);
          f[n & 1][x] = u32x4{b0.x, b0.y, b1.x, b1.y};
        } else {
          f[n & 1][x] = read_lds((K ^ (32 * (2 * (n - HT) + (x >> 1)))) + 32 * (x & 1) * RB);
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
          o[x % HT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f[n & 1][x]), __builtin_bit_cast(bf16x8, pf.upper[(4 * n + x) / HT]), o[x % HT], 0, 0, 0);
          if (x % HT == HT - 1)
#pragma unroll
            for (int y = x + 1 - HT; y <= x; ++y)
              o[y % HT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f[n & 1][y]), __builtin_bit_cast(bf16x8, pf.lower[(4 * n + y) / HT]), o[y % HT], 0, 0, 0);
        } else {
          const int k = 2 * (n - HT) + (x >> 1);
          s[x & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f[n & 1][x]), qf[k], k ? s[x & 1] : f32x16{}, 0, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // The weights of block j from its scores.
  float alpha = 1.f;
  bool raised = false;
  auto weigh = [&](const float (&x)[2][16]) __attribute__((always_inline)) {
    float sum;
    auto weights = [&]() __attribute__((always_inline)) {
      sum = 0.f;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const float w0 = exp2_raw(fmaf(x[t][e], scale, -m)), w1 = exp2_raw(fmaf(x[t][e + 1], scale, -m));
          sum += w0;
          sum += w1;
          pf.put(16 * t + e, w0, w1);
        }
    };
    weights();
    if (__builtin_expect(__any(!(sum < kMostSum)), 0)) {         // (the first block that a row sees, too)
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, x[t][e]);
      top = fmaxf(top, __shfl_xor(top, 32, 64)) * scale;         // both lanes of a row raise alike
      const float to = fmaxf(m, top);
      alpha = exp2_raw(m - to);
      raised = true;
      m = to;
      l *= alpha;
      weights();
    }
    l += sum;
  };
  auto soften = [&](int j) __attribute__((always_inline)) {
    if (!sees(j)) {
#pragma unroll
      for (int t = 0; t < 4; ++t) { pf.upper[t] = u32x4{0, 0, 0, 0}; pf.lower[t] = u32x4{0, 0, 0, 0}; }
      return;
    }
    const int k0 = start_of(block_of(j));
    float x[2][16];                                              // (from here on scalars: hipcc lost elements of a vector of which one was replaced under a condition)
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) x[t][e] = s[t][e];
    if (k0 + BK - 1 > wave_pos || (k0 <= last_pos - a.sight.window && k0 + BK > a.sight.sinks)) {   // some of these keys are not for some of the rows
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint32_t seen = seen_keys(pos - k0 - 32 * t, a.sight.window, a.sight.sinks - k0 - 32 * t) >> (4 * half);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[t][e] = masked(x[t][e], seen, 8 * (e >> 2) + (e & 3));
      }
    }
    weigh(x);
  };

  // Of the wavefronts of a SIMD, w and w + 4, one multiplies while the other takes exponentials: in a step the early four multiply and
  // then weigh the new scores, the late four weigh those of the step before and then multiply.  Stage j + 1 is asked for at the
  // beginning of step j, over blocks that all have left, and waited for at its end.
  pages(0);
  issue(0);
  {                                                              // (behind the way to the first keys, which is the longer one)
    const bf16_t* qp = (const bf16_t*)a.q + (long)(at.first + min(row, at.rows - 1)) * a.q_stride + (long)head * HD + 8 * half;
    u32x4 w[HD / 16];
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks) w[ks] = *reinterpret_cast<const u32x4*>(qp + 16 * ks);
    // (scores are multiplied by a positive number: a masked one is -inf before that)
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u, keep = a.scale == 0.f ? 0u : ~0u;
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t x = (w[ks][i] ^ flip) & keep;
        asm volatile("" : "+v"(x));                              // (looked at here: else the loop waits for them, and for all that it has asked for)
        w[ks][i] = x;
      }
      qf[ks] = __builtin_bit_cast(bf16x8, w[ks]);
    }
  }
  // (the first step has no values yet: its weights are zeros, and so is what they multiply)
  for (int i = tid; i < BB / 16; i += GT) *(lds_u32x4)(uintptr_t)(Vb + BB + 16 * i) = u32x4{0, 0, 0, 0};
  if (threadIdx.x == 0) again = 0;
  wait_loads();
  __syncthreads();
  auto rescale = [&]() __attribute__((always_inline)) {
    if (__builtin_expect(raised, 0)) {
#pragma unroll
      for (int i = 0; i < HT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float v = o[i][e] * alpha;
          asm volatile("" : "+v"(v));                            // (one after the other, in place: else they are copied, and others spilled)
          o[i][e] = v;
        }
      raised = false;
    }
  };
  auto turns = [&](auto second) __attribute__((always_inline)) {
    constexpr bool kLate = decltype(second)::value;
    for (int j = 0; j < n_it; ++j) {
      issue(j + 1);
      if (kLate && j > 0) { soften(j - 1); rescale(); }
      products(j, std::true_type());
      if constexpr (!kLate) { soften(j); rescale(); }
      wait_loads();
      __syncthreads();
    }
    if constexpr (kLate) { soften(n_it - 1); rescale(); }
    products(n_it, std::false_type());
  };
  if (late) turns(std::true_type()); else turns(std::false_type());
  if (worst >= (unsigned)c.n_pages) kv8_report(c);
  l += __shfl_xor(l, 32, 64);
  // A value that is not finite spoils the sums of rows that do not see it, too: a zero weight times infinity is no number.  Then all rows
  // are computed once more, each by itself, and where sums are so large that adding the groups' or pieces' might exceed binary32's
  // range (kTooLarge).  (Weights that are no numbers are what they should be.)
  {
    float odd = 0.f;
#pragma unroll
    for (int i = 0; i < HT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) odd = fmaf(o[i][e] * kTooLarge, 0.f, odd);
    if (__any(!(odd == 0.f) && l - l == 0.f)) again = 1;
  }
  __syncthreads();
  if (__builtin_expect(__builtin_amdgcn_readfirstlane(again), 0)) {
    prompt_again<HD>(c, r, a, mine, BQ, 8);
    return;
  }

  if constexpr (NG > 1) {
    float* fold = (float*)smem;
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
    const float m1 = fold[(HT * 16) * GT + tid], l1 = fold[(HT * 16 + 1) * GT + tid];
    const float to = fmaxf(m, m1), a0 = exp2_raw(m - to), a1 = exp2_raw(m1 - to);
    l = l * a0 + l1 * a1;
    m = to;
#pragma unroll
    for (int i = 0; i < HT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[i][e] = o[i][e] * a0 + fold[(i * 16 + e) * GT + tid] * a1;
  }

  if (live) prompt_store<HT>(c, r, a, mine, row, head, o, m, l);
}

template <int NG>
constexpr size_t prompt_lds() {
  const size_t kv = (size_t)NG * 4 * BK * 128, fold = (size_t)(NG - 1) * 34 * (512 / NG) * sizeof(float);
  return kv > fold ? kv : fold;
}
template <int NG, bool kWhole, bool kMany>
bool allow_one() {                                               // 64 KiB is what a kernel gets by default
  return hipFuncSetAttribute((const void*)k_kv_prompt<NG, kWhole, kMany>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)prompt_lds<NG>()) == hipSuccess;
}

PromptGeo geo_of(const KvCache& c, const KvRows& r, int H, int rows) {
  const int sh = kv_heads_shift(c, H), bp = rows >> sh;
  return PromptGeo{r.n_rows / bp + std::min(r.n, r.n_rows), H >> sh, sh, 0};
}
// A launch has fewer than 2^32 threads.  n_rows * H is below 2^24, so the workgroups of up to kInOrder samples, at most 2^24 / 128 for
// the rows and H for each sample, are far below that; one for each of very many samples and heads may not be, and go out in several.
constexpr int kMostWgs = 1 << 22;
template <int NG, bool kWhole>
void launch_pages(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a, const PromptGeo& g, int wgs) {
  if (r.n <= kInOrder) hipLaunchKernelGGL((k_kv_prompt<NG, kWhole, false>), dim3(wgs, a.plan.splits), dim3(512), prompt_lds<NG>(), s, c, r, a, g);
  else hipLaunchKernelGGL((k_kv_prompt<NG, kWhole, true>), dim3(wgs, a.plan.splits), dim3(512), prompt_lds<NG>(), s, c, r, a, g);
}

}  // namespace

bool kv_allow_lds() {
  static OncePerDevice done;
  int dev = -1;
  return hipGetDevice(&dev) == hipSuccess && done.run(dev, []() { return allow_one<2, true, false>() && allow_one<2, false, false>() && allow_one<2, true, true>() && allow_one<2, false, true>() && kv_wide_allow_lds(); });
}

void launch_kv_prompt(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a) {
  PromptGeo g = geo_of(c, r, a.H, a.plan.rows);
  const int total = g.n_blocks * g.sets;                         // (at most 2^24 + 2^17)
  const bool many = r.n > kInOrder, whole = c.pt % BK == 0;
  for (; g.from < total; g.from += kMostWgs) {
    const int wgs = many ? std::min(kMostWgs, total - g.from) : total;
    if (c.h == 128) launch_kv_wide(s, c, r, a, g, wgs, many);
    else if (a.plan.groups == 1) { if (whole) launch_pages<1, true>(s, c, r, a, g, wgs); else launch_pages<1, false>(s, c, r, a, g, wgs); }
    else { if (whole) launch_pages<2, true>(s, c, r, a, g, wgs); else launch_pages<2, false>(s, c, r, a, g, wgs); }
    if (!many) break;
  }
}

}  // namespace mdi
