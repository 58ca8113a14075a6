// Attention of packed rows over the bf16 cache, heads of 128: 64 rows of (position, query head) a wavefront, one wavefront a SIMD, two or four a workgroup.
//
// The products of kv_prompt.hip read an operand of every matrix instruction from the LDS, 1 KiB in 32 cycles for each of the four SIMDs of
// a compute unit: all that its LDS delivers.  Here an operand serves two of them, for the wavefront's two sets of 32 rows, and values four:
// a weight is two operands (PromptWeights).  What a second wavefront on the SIMD did, exponentials while the first multiplies, the
// wavefront does itself: in step i, of 32 keys, it multiplies the keys of step i + 1 and the values of step i - 1 and in between
// weighs the scores of step i, some five vector instructions behind every matrix instruction.  Everything of a step is in registers
// (operands are read into them shortly before they are multiplied), some 420 of them.
//
// Matrix instructions bound it: prompts of 6000, 2000 and 500 of the 8B shape take 470 to 485 us, 0.7 PFLOP/s of useful products and 1.05 with those
// of the weights' lower digits, where a large product of the library reaches 1.21; with a window of 1024 of the 7B shape 250, where
// a workgroup passes over 1152 keys for rows that see 1024 each.  (Weights of one operand: 351 and 197; in vector instructions 25 ms and 9 ms.)
// A workgroup begins and ends in some 6 us, most of them its queries, first keys and results on their way.
#include <utility>

#include "kv_prompt_device.h"
#include "kv_prompt_wide.h"

namespace mdi {
namespace {

constexpr float kFarSum = 0x1p30f;

// Four times 64 x 16 bytes global -> LDS, the places 1024 bytes apart: an instruction's offset counts for both addresses.
__device__ __forceinline__ void dma4(uint32_t lds, const char* base, const uint32_t* off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\tglobal_load_lds_dwordx4 %2, %5 offset:0x400\n\t"
               "global_load_lds_dwordx4 %3, %5 offset:0x800\n\tglobal_load_lds_dwordx4 %4, %5 offset:0xc00"
               ::"s"(lds), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base) : "m0", "memory");
}
__device__ __forceinline__ void dma4(uint32_t lds, const char* const* p) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\tglobal_load_lds_dwordx4 %2, off offset:0x400\n\t"
               "global_load_lds_dwordx4 %3, off offset:0x800\n\tglobal_load_lds_dwordx4 %4, off offset:0xc00"
               ::"s"(lds), "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]) : "m0", "memory");
}

// f(0) .. f(N - 1), numbers that the compiler knows: a loop whose body takes this much is not unrolled.
template <typename F, int... N> __device__ __forceinline__ void each(F&& f, std::integer_sequence<int, N...>) { (f(std::integral_constant<int, N>()), ...); }

// A workgroup is W wavefronts, four or two: NG groups of WQ, which work on the same 64 WQ rows; group g takes the key blocks NG i + g.
template <int W, int NG, bool kWhole, bool kMany>
__global__ __launch_bounds__(64 * W, 1) void k_kv_prompt_wide(KvCache c, KvRows r, KvAttn a, PromptGeo geo) {
  constexpr int HD = 128, WQ = W / NG, BQ = 64 * WQ, GT = 64 * WQ;   // rows of a workgroup - (position, head) pairs -, threads of a group
  constexpr int HT = HD / 32, KS = HD / 16, RB = 2 * HD, UN = HD / 8;   // bytes and 16-byte units of a key
  constexpr int BB = BK * RB;                                    // bytes of a block of keys, or of values
  constexpr int KP = 64 / UN, NI = BK / KP / WQ;                 // keys of an instruction that loads, instructions of a wavefront
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];

  const int tid = threadIdx.x & (GT - 1), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = NG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / GT);
  const uint32_t Kb = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)smem + grp * 5 * BB, Vb = Kb + 2 * BB;   // two blocks of keys, three of values
  const int x = kMany ? geo.from + blockIdx.x : blockIdx.x, block = x / geo.sets, set = x - block * geo.sets;   // (as in kv_prompt.hip)
  const BlockPlace at = place_of<kMany>(r, block, BQ >> geo.g_sh);
  if (at.sample < 0) return;
  const int g_sh = geo.g_sh, bp = BQ >> g_sh, head0 = set << g_sh, kv = head0 / (a.H / c.K);
  const int q0 = ((at.rows + bp - 1) / bp - 1 - at.block) * bp;  // first row of the sample in this block
  const int p0 = at.pos, which = p0 < 0 ? -1 : kv8_checked_row(c, at.table);
  const int32_t* table = c.tables + (long)max(which, 0) * c.table_stride;
  const int col = lane & 31, half = lane >> 5, head = head0 + (col & ((1 << g_sh) - 1));   // (32 is a multiple of 2^g_sh)
  int row[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) row[u] = q0 + ((64 * wave + 32 * u + col) >> g_sh);
  if (which < 0) {                                               // takes no part
#pragma unroll
    for (int u = 0; u < 2; ++u)
      if (blockIdx.y == 0 && grp == 0 && row[u] < at.rows) prompt_zeros<HT>(c, r, a, at, row[u], head);
    return;
  }
  const long far = (long)p0 + min(q0 + bp, at.rows);             // behind the workgroup's last position
  if (far > r.max_ctx) kv8_report(c);
  const int cap = r.max_ctx - 1;
  auto pos_of = [&](int row1) __attribute__((always_inline)) { return (int)min((long)p0 + min(row1, at.rows - 1), (long)cap); };
  const KvBlocks kb = kv_blocks(a.sight, pos_of(q0), (int)min(far, (long)r.max_ctx));
  const int b_lo = blockIdx.y * a.plan.chunk, b_hi = (int)min((long)kb.n, (long)b_lo + a.plan.chunk), pieces = (kb.n + a.plan.chunk - 1) / a.plan.chunk;
  if (b_lo >= b_hi) return;
  const PromptRows mine{at, g_sh, head0, kv, q0, p0, table, kb, (int)blockIdx.y, b_lo, b_hi, pieces};

  f32x16 o[2][HT];
  float m[2], l[2];
  int pos[2];                                                    // a lane's rows see positions up to these
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    pos[u] = pos_of(row[u]);
    m[u] = kKvNone;
  }
  const float scale = a.scale == 0.f ? 1.f : fabsf(a.scale);
  const int wave_pos = pos_of(q0 + ((64 * wave) >> g_sh)), last_pos = pos_of(q0 + ((64 * wave + 63) >> g_sh));   // of the wavefront's first and last rows

  // Loading, as in kv_prompt.hip: stage j is the keys of block j and the values of block j - 1.
  const int n_it = (b_hi - b_lo + NG - 1) / NG, gap = kb.first - (kb.n_sinks << 6);
  auto block_of = [&](int j) __attribute__((always_inline)) { return min(b_lo + NG * j + grp, b_hi - 1); };
  auto start_of = [&](int b) __attribute__((always_inline)) { return (b << 6) + (b < kb.n_sinks ? 0 : gap); };
  // Blocks whose positions are all seen by some row of the workgroup, and by all rows of the wavefront (of those behind the first positions).
  auto first_from = [&](int pos) __attribute__((always_inline)) { return max(kb.n_sinks, (pos - gap + 63) >> 6); };   // that starts at or behind pos
  auto step_from = [&](int b) __attribute__((always_inline)) { return max(b - b_lo - grp + NG - 1, 0) / NG; };   // the group's first whose block is b or behind it
  // steps whose block is the wavefront's rows' as a whole; stages whose keys and values all are
  const int all_lo = step_from(first_from(max(last_pos - a.sight.window + 1, 0))), all_hi = step_from(min((wave_pos + 1 - gap) >> 6, b_hi));
  const int rare_lo = step_from(first_from(kb.from)), rare_hi = step_from(min((kb.end - gap) >> 6, b_hi));
  auto visible = [&](int p, int k0) __attribute__((always_inline)) {
    return min(p < kb.sinks || p >= kb.from ? p : k0 < kb.sinks ? kb.sinks - 1 : kb.from, kb.end - 1);
  };
  auto key_of = [&](int n) __attribute__((always_inline)) { return (wave * NI + n) * KP + lane / UN; };
  auto unit_of = [&](int key) __attribute__((always_inline)) {
    return (lane % UN) ^ (((key & 3) << 2) | ((key >> 2) & 3));
  };
  auto by_of = [](int n) __attribute__((always_inline)) { return 4096 - 1024 * (n & 3); };   // (dma4 adds what is missing)
  unsigned worst = 0;                                            // a page that is not of the cache is looked for at the end, the last one read in its place
  auto checked = [&](int page) __attribute__((always_inline)) {
    worst = max(worst, (unsigned)page);
    return min((unsigned)page, (unsigned)c.n_pages - 1);
  };
  constexpr int kPages = kWhole ? 1 : NI;
  int pg[kPages];
  uint32_t at_off[NI];                                           // of a block whose positions are all seen by some row
#pragma unroll
  for (int n = 0; n < NI; ++n) at_off[n] = (uint32_t)(key_of(n) * RB + 16 * unit_of(key_of(n)) + by_of(n));
  const char *k_at[kPages] = {}, *v_at = nullptr;                // the stage's keys (kWhole: and its values)
  const long v_by = (long)c.pt * RB;                             // from a key to its value
  const char* const heads_at = (const char*)c.data + 2 * kv * v_by;
  const uint64_t page_bytes = 2ull * c.K * v_by;
  auto pages = [&](int j, int (&pg)[kPages]) __attribute__((always_inline)) {
    const int k0 = start_of(block_of(kWhole ? j + lane : j));
#pragma unroll
    for (int n = 0; n < kPages; ++n) pg[n] = table[kv8_page_of(c, kWhole ? k0 : visible(k0 + key_of(n), k0))];
  };
  // Pages that blocks lie in whole: lane i of `list` has the address of the keys of stage 64 n + i, worked out for 64 stages at a time, from
  // page numbers that were asked for 64 stages before.
  uint32_t list[2] = {};
  auto fill = [&](int j, int (&pg)[kPages]) __attribute__((always_inline)) {
    const int k0 = start_of(block_of(j + lane));
    const uint64_t k = (uint64_t)(heads_at - 4096) + (checked(pg[0]) * page_bytes + (unsigned)((k0 - kv8_page_of(c, k0) * c.pt) * RB));   // (4096: see dma4)
    list[0] = (uint32_t)k;
    list[1] = (uint32_t)(k >> 32);
    asm volatile("" : "+v"(list[0]), "+v"(list[1]));
  };
  // Pages that hold blocks as a whole: where stage j is, its keys, and its values from the keys of the stage before.  (Page numbers are
  // looked at before anything else is asked for: whoever waits for them waits for that, too.)
  auto find = [&](int j, int (&pg)[kPages]) __attribute__((always_inline)) {
    if constexpr (kWhole) {
      v_at = k_at[0] + v_by;
      if ((j & 63) == 0) {
        fill(j, pg);
        pages(j + 64, pg);
      }
      k_at[0] = (const char*)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)list[1], j & 63) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)list[0], j & 63));
    }
  };
  // Instructions 4 n .. + 3 of stage j; lds: the wavefront's part of the block.  Other pages: the values' before the same of the keys,
  // whose addresses are the next stage's values'.
  auto ask_block = [&](uint32_t lds, const char* at, int n, int j, bool rare) __attribute__((always_inline)) {
    if (__builtin_expect(rare, 0)) {
      const int k0 = start_of(block_of(j));
      uint32_t off[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = key_of(4 * n + i);
        off[i] = (uint32_t)((visible(k0 + key, k0) - k0) * RB + 16 * unit_of(key) + by_of(i));
      }
      dma4(lds + 4096 * n, at, off);
    } else {
      dma4(lds + 4096 * n, at, &at_off[4 * n]);
    }
  };
  auto ask_keys = [&](uint32_t lds, int n, int j, int (&pg)[kPages]) __attribute__((always_inline)) {
    if constexpr (kWhole) {
      ask_block(lds, k_at[0], n, j, j < rare_lo || j >= rare_hi);
    } else {
      const int k0 = start_of(block_of(j));
#pragma unroll
      for (int i = 4 * n; i < 4 * n + 4; ++i) {
        const int key = key_of(i);
        k_at[i] = (const char*)c.data + kv8_row(c, checked(pg[i]), kv, visible(k0 + key, k0)) * RB + 16 * unit_of(key) + by_of(i) - 4096;
      }
      dma4(lds + 4096 * n, &k_at[4 * n]);
    }
  };
  auto ask_values = [&](uint32_t lds, int n, int j) __attribute__((always_inline)) {
    if constexpr (kWhole) {
      ask_block(lds, v_at, n, max(j - 1, 0), j <= rare_lo || j > rare_hi);
    } else {
      const char* p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = k_at[4 * n + i] + v_by;
      dma4(lds + 4096 * n, p);
    }
  };
  // (behind a wait for all loads: else the first that looks at them waits for what has been asked for since)
  auto loaded = [&](int (&pg)[kPages]) __attribute__((always_inline)) {
    if constexpr (!kWhole)
#pragma unroll
      for (int n = 0; n < NI; ++n) asm volatile("" : "+v"(pg[n]));
  };
  const uint32_t w_lds = wave * NI * 1024;

  const int kk = (lane & 15) >> 2;                               // what this lane reads: as in kv_prompt.hip
  const uint32_t k_lane = col * RB + 16 * (half ^ (((col & 3) << 2) | ((col >> 2) & 3)));
  const uint32_t v_lane = (4 * half + kk) * RB + 64 * kk + 16 * ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ half) + 8 * (lane & 1);
  u32x4 kf[KS], vf[HT];                                          // operands: keys of a step; values of 16 of its keys
  bf16x8 qf[2][KS];
  auto read_key = [&](uint32_t K, int ks) __attribute__((always_inline)) { kf[ks] = read_lds(K ^ (32 * ks)); };
  auto read_value = [&](uint32_t V, int n) __attribute__((always_inline)) {   // n: channel block and half of the operand
    const uint32_t p = V ^ (64 * (n >> 1));
    const u32x2 w = read_transposed(n & 1 ? (p ^ 32) + 8 * RB : p);
    vf[n >> 1][2 * (n & 1)] = w.x;
    vf[n >> 1][2 * (n & 1) + 1] = w.y;
  };

  // A row's reference is the largest score of the first keys that it sees.  Where later ones would have weights of more than
  // kFarSum the reference is raised, but not the sums so far: then all is done once more, from the references that the first time
  // ended with, which nothing exceeds as far.  (A rescaling would have the sums in registers that vector instructions reach, and copied
  // there and back around every step.)
  typedef PromptWeights<2> Weights;                               // of a row and 32 keys
  auto keep = [](Weights& w, int pp) __attribute__((always_inline)) { asm volatile("" : "+a"(w.upper[pp]), "+a"(w.lower[pp])); };   // (as kf and vf)
  bool once_more = false;
  // Step i = 2 j + t: scores sn of step i + 1 (operands there), weights pn of step i from its scores sc, and the values of step i - 1
  // times its weights pc.  K: where the keys of step i + 2 are; V: the values of step i - 1.
  // ask(n): what is asked for behind matrix instruction n.  Of three of these instructions two have an exponential behind them, the third
  // divides the two weights into their operands.
  auto step = [&](bool whole, int k0, f32x16 (&sc)[2], f32x16 (&sn)[2], Weights (&pc)[2], Weights (&pn)[2], uint32_t K, uint32_t V, auto&& ask) __attribute__((always_inline)) {
    float x[2][16];                                              // (from here on scalars: hipcc lost elements of a vector of which one was replaced under a condition)
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) x[u][e] = sc[u][e];
    if (!whole) {                                                // some of these keys are not for some of the rows
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint32_t seen = k0 < 0 ? 0u : seen_keys(pos[u] - k0, a.sight.window, a.sight.sinks - k0) >> (4 * half);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[u][e] = masked(x[u][e], seen, 8 * (e >> 2) + (e & 3));
      }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) asm volatile("" : "+v"(x[0][e]), "+v"(x[1][e]));   // (not in the accumulation registers)
    float sum[2] = {0.f, 0.f}, w0 = 0.f, w1 = 0.f;
    __builtin_amdgcn_sched_barrier(0);
    each([&](auto index) __attribute__((always_inline)) {
      constexpr int n = decltype(index)::value;
      if constexpr (n < 2 * KS) {
        constexpr int ks = n >> 1, u = n & 1;
        if (u == 0) asm volatile("" : "+a"(kf[ks]));
        sn[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[ks]), qf[u][ks], ks ? sn[u] : f32x16{}, 0, 0, 0);
      } else {
        constexpr int q = n - 2 * KS, pp = q / (4 * HT), h = (q >> 2) % HT, part = (q >> 1) & 1, u = q & 1;
        if ((q & 3) == 0) asm volatile("" : "+a"(vf[h]));
        o[u][h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[h]), __builtin_bit_cast(bf16x8, part ? pc[u].lower[pp] : pc[u].upper[pp]), o[u][h], 0, 0, 0);
      }
      // (operands are asked for when their registers are free, and those of the products before are no longer needed)
      if (n < 2 * HT) read_value(V, n);
      else if (n >= 2 * KS + 4 && n < 2 * KS + 4 + 4 * HT && n % 4 < 2) read_value(V + 16 * RB, (n - 2 * KS - 4) / 4 * 2 + n % 4);
      else if (n >= 48 - KS) read_key(K, n - 48 + KS);
      ask(index);
      constexpr int u = n / 24, e = 2 * (n % 24 / 3) + n % 3;    // weight e of set u, or the two before
      if constexpr (n % 3 < 2) {
        const float w = exp2_raw(fmaf(x[u][e & 15], scale, -m[u]));
        sum[u] += w;
        if (n % 3) w1 = w; else w0 = w;
      } else {
        pn[u].put(e - 2, w0, w1);
        if constexpr (e % 8 == 0) keep(pn[u], e / 8 - 1);
      }
      __builtin_amdgcn_sched_barrier(0);
    }, std::make_integer_sequence<int, 48>());
    if (__builtin_expect(__any(!(sum[0] < kFarSum) || !(sum[1] < kFarSum)), 0)) {   // (the first keys that a row sees, too)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, x[u][e]);
        top = fmaxf(top, __shfl_xor(top, 32, 64)) * scale;       // both lanes of a row raise alike
        const float to = top > m[u] + 25.f ? top : m[u];         // (32 weights of up to 2^25 are no more than kFarSum: other rows' references stay)
        once_more |= to > m[u] && m[u] != kKvNone;
        m[u] = to;
        sum[u] = 0.f;
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const float a0 = exp2_raw(fmaf(x[u][e], scale, -to)), a1 = exp2_raw(fmaf(x[u][e + 1], scale, -to));
          sum[u] += a0;
          sum[u] += a1;
          pn[u].put(e, a0, a1);
          if (e % 8 == 6) keep(pn[u], e / 8);
        }
      }
    }
    l[0] += sum[0];
    l[1] += sum[1];
  };

  {
    // (scores are multiplied by a positive number: a masked one is -inf before that)
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u, keep = a.scale == 0.f ? 0u : ~0u;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const bf16_t* qp = (const bf16_t*)a.q + (long)(at.first + min(row[u], at.rows - 1)) * a.q_stride + (long)head * HD + 8 * half;
      u32x4 w[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) w[ks] = *reinterpret_cast<const u32x4*>(qp + 16 * ks);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t y = (w[ks][i] ^ flip) & keep;
          asm volatile("" : "+v"(y));                            // (looked at here: else the loop waits for them, and for all that it has asked for)
          w[ks][i] = y;
        }
        qf[u][ks] = __builtin_bit_cast(bf16x8, w[ks]);
      }
    }
  }
  int again;                                                     // 1: once more with other references; 2: a value that is not finite
  do {
  {
    int pg0[kPages];
    pages(0, pg0);
    if constexpr (!kWhole) pages(1, pg);
    find(0, pg0);
#pragma unroll
    for (int n = 0; n < NI / 4; ++n) ask_keys(Kb + w_lds, n, 0, pg0);
    find(1, pg0);
#pragma unroll
    for (int n = 0; n < NI / 4; ++n) { ask_values(Vb + w_lds, n, 1); ask_keys(Kb + BB + w_lds, n, 1, kWhole ? pg0 : pg); }
    if constexpr (kWhole) pg[0] = pg0[0]; else pages(2, pg);
  }
  // (the first step has no values yet: its weights are zeros, and so is what they multiply)
  for (int i = tid; i < BB / 16; i += GT) *(lds_u32x4)(uintptr_t)(Vb + 2 * BB + 16 * i) = u32x4{0, 0, 0, 0};
  wait_loads();
  loaded(pg);
  __syncthreads();

#pragma unroll
  for (int u = 0; u < 2; ++u) {
    l[u] = 0.f;
#pragma unroll
    for (int i = 0; i < HT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[u][i][e] = 0.f;
  }
  f32x16 s0[2], s1[2];
  Weights w0[2] = {}, w1[2] = {};
  // scores of step 0, and the keys of step 1
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) read_key(Kb + k_lane, ks);
#pragma unroll
  for (int n = 0; n < 2 * KS; ++n)
    s0[n & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[n >> 1]), qf[n & 1][n >> 1], n > 1 ? s0[n & 1] : f32x16{}, 0, 0, 0);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) read_key(Kb + k_lane + 32 * RB, ks);
  __syncthreads();                                               // (the first step loads over these)

  uint32_t v_before = Vb + 2 * BB, v_now = Vb;
  for (int j = 0; j < n_it; ++j) {
    find(j + 2, pg);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+a"(qf[u][ks]));   // (operands: in the accumulation registers, which vector instructions do not reach)
    const bool mine_too = NG == 1 || b_lo + NG * j + grp < b_hi;            // (a group's last step may have no block)
    const bool whole = j >= all_lo && j < all_hi;
    const int k0 = whole ? 0 : mine_too ? start_of(block_of(j)) : -(1 << 30);
    const uint32_t K = Kb + ((j + 1) & 1) * BB + k_lane, v_next = v_now == Vb + 2 * BB ? Vb : v_now + BB, k_lds = Kb + (j & 1) * BB + w_lds;
    step(whole, k0, s0, s1, w1, w0, K, v_before + v_lane + 32 * RB, [&](auto index) __attribute__((always_inline)) {
      constexpr int n = decltype(index)::value;
      if constexpr (n % 4 == 0 && n / 4 < NI / 2) { if constexpr (n & 4) ask_keys(k_lds, n / 8, j + 2, pg); else ask_values(v_next + w_lds, n / 8, j + 2); }
    });
    if constexpr (!kWhole) pages(j + 3, pg);
    step(whole, k0 + (mine_too ? 32 : 0), s1, s0, w0, w1, K + 32 * RB, v_now + v_lane, [](auto) {});
    v_before = v_now;
    v_now = v_next;
    wait_loads();
    loaded(pg);
    __syncthreads();
  }
  // the values of the last step
#pragma unroll
  for (int n = 0; n < 8 * HT; ++n) {
    const int pp = n / (4 * HT), h = (n >> 2) % HT, part = (n >> 1) & 1, u = n & 1;
    if ((n & 3) == 0) { read_value(v_before + v_lane + (32 + 16 * pp) * RB, 2 * h); read_value(v_before + v_lane + (32 + 16 * pp) * RB, 2 * h + 1); }
    o[u][h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[h]), __builtin_bit_cast(bf16x8, part ? w1[u].lower[pp] : w1[u].upper[pp]), o[u][h], 0, 0, 0);
  }
  __syncthreads();
  // A value that is not finite spoils the sums of rows that do not see it, too: a zero weight times infinity is no number.  Then all rows
  // are computed once more, each by itself, and where sums are so large that adding the groups' or pieces' might exceed binary32's
  // range (kTooLarge).  (Weights that are no numbers are what they should be.)
  int* const flag = (int*)smem;
  if (threadIdx.x == 0) *flag = 0;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    l[u] += __shfl_xor(l[u], 32, 64);
    float odd = 0.f;
#pragma unroll
    for (int i = 0; i < HT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) odd = fmaf(o[u][i][e] * kTooLarge, 0.f, odd);
    if (__any(!(odd == 0.f) && l[u] - l[u] == 0.f)) atomicOr(flag, 2);
  }
  if (__any(once_more)) atomicOr(flag, 1);
  once_more = false;
  __syncthreads();
  again = __builtin_amdgcn_readfirstlane(*flag);
  __syncthreads();
  } while (__builtin_expect(again & 1, 0));
  if (worst >= (unsigned)c.n_pages) kv8_report(c);
  if (__builtin_expect(again, 0)) {
    prompt_again<HD>(c, r, a, mine, BQ, W);
    return;
  }
  if constexpr (NG > 1) {
    __syncthreads();
    float* fold = (float*)smem;
#pragma unroll
    for (int u = 0; u < 2; ++u) {                                // (element j of thread t at [j][t])
      if (grp > 0) {
#pragma unroll
        for (int i = 0; i < HT; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) fold[(u * (HT * 16 + 2) + i * 16 + e) * GT + tid] = o[u][i][e];
        fold[(u * (HT * 16 + 2) + HT * 16) * GT + tid] = m[u];
        fold[(u * (HT * 16 + 2) + HT * 16 + 1) * GT + tid] = l[u];
      }
    }
    __syncthreads();
    if (grp > 0) return;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float* f = fold + u * (HT * 16 + 2) * GT + tid;
      const float m1 = f[HT * 16 * GT], l1 = f[(HT * 16 + 1) * GT], to = fmaxf(m[u], m1), a0 = exp2_raw(m[u] - to), a1 = exp2_raw(m1 - to);
      l[u] = l[u] * a0 + l1 * a1;
      m[u] = to;
#pragma unroll
      for (int i = 0; i < HT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[u][i][e] = o[u][i][e] * a0 + f[(i * 16 + e) * GT] * a1;
    }
  }
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (row[u] < at.rows) prompt_store<HT>(c, r, a, mine, row[u], head, o[u], m[u], l[u]);
}

template <int NG> constexpr size_t wide_lds() { return (size_t)NG * 5 * BK * 256; }
template <int W, int NG>
bool allow() {                                                   // 64 KiB is what a kernel gets by default
  auto one = [](const void* k) { return hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)wide_lds<NG>()) == hipSuccess; };
  return one((const void*)k_kv_prompt_wide<W, NG, true, false>) && one((const void*)k_kv_prompt_wide<W, NG, false, false>) &&
         one((const void*)k_kv_prompt_wide<W, NG, true, true>) && one((const void*)k_kv_prompt_wide<W, NG, false, true>);
}
template <int W, int NG>
void launch(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a, const PromptGeo& g, int wgs, bool many) {
  const dim3 grid(wgs, a.plan.splits), block(64 * W);
  const size_t lds = wide_lds<NG>();
  if (c.pt % BK == 0) {
    if (many) hipLaunchKernelGGL((k_kv_prompt_wide<W, NG, true, true>), grid, block, lds, s, c, r, a, g);
    else hipLaunchKernelGGL((k_kv_prompt_wide<W, NG, true, false>), grid, block, lds, s, c, r, a, g);
  } else {
    if (many) hipLaunchKernelGGL((k_kv_prompt_wide<W, NG, false, true>), grid, block, lds, s, c, r, a, g);
    else hipLaunchKernelGGL((k_kv_prompt_wide<W, NG, false, false>), grid, block, lds, s, c, r, a, g);
  }
}

}  // namespace

bool kv_wide_allow_lds() { return allow<4, 1>() && allow<4, 2>() && allow<2, 1>(); }
void launch_kv_wide(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a, const PromptGeo& g, int wgs, bool many) {
  if (a.plan.groups == 2) launch<4, 2>(s, c, r, a, g, wgs, many);
  else if (a.plan.rows == 256) launch<4, 1>(s, c, r, a, g, wgs, many);
  else launch<2, 1>(s, c, r, a, g, wgs, many);
}

}  // namespace mdi
