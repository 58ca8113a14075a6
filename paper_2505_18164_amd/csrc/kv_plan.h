// Which kernels an attention call over the cache in the storage type runs on, and how it is divided.  Host code without launches, so that tests
// can ask which ones a set of sizes reaches.
#pragma once

#include <algorithm>
#include <cmath>

#include "kv_internal.h"

namespace mdi {

// Packed rows of up to so many samples are divided in order (kv_blocks.h).
constexpr int kInOrder = 384;

// Query heads of a kv head that a workgroup's rows take together: the largest power of two that divides their number, up to 32.
inline int kv_heads_shift(const KvPages& c, int H) {
  const int G = H / c.K;
  int sh = 0;
  while (sh < 5 && G % (2 << sh) == 0) ++sh;
  return sh;
}

// ---- One new token per sample in bf16 with heads of 64 or 128 (kv_decode.hip).
inline bool kv_decode_supported(const KvCache& c, const KvRows& r) { return !r.start && c.dtype == MDI_BF16 && (c.h == 64 || c.h == 128); }
// A cache that no later call finds in the last cache is read without a place in it.
inline bool kv_decode_once(const KvCache& c, const KvRows& r, const KvSight& w) {
  return (double)r.n * kv_most_seen(w, r.max_ctx) * c.K * 4 * c.h > 128e6;
}
// (384, 512, 768, 1024 shares: the 8 tokens 62.0, 52.9, 53.2, 55.9 us, the one 110.9, 89.6, 89.2, 91.9, 32 of the 7B shape behind 600 73.1,
// 63.4, 66.3, 63.5)
constexpr int kKvShares = 512;
constexpr int kKvLeast = 2;          // tiles of a share, at least

// With many units, or short samples, a unit is a workgroup's.  Else the tiles of all units are cut into equal shares.
inline KvPlan kv_decode_plan(const KvCache& c, const KvRows& r, int H, const KvSight& w) {
  const int each = c.K * kv8_groups(c, H), most = kv_most_seen(w, r.max_ctx);   // units of a sample
  if ((long)r.n * each >= 4 * kKvShares || most <= kKvLeast * kKv8Tile) return KvPlan{kKvDecode, most, 1, 0, 0, 0};
  // a unit of t tiles in shares of at least kKvLeast, and of at least t * each / kKvShares (it is one of `each` alike)
  const int tiles = (most + kKv8Tile - 1) / kKv8Tile;
  return KvPlan{kKvDecode, kKvLeast * kKv8Tile, std::min(tiles / kKvLeast, (kKvShares + each - 1) / each) + 2, kKvShares, 0, 0};
}

// ---- Any other, and few packed rows (kv_any.hip).  us: what the call should take, without its launches; of single tokens it is not asked for.
// Wavefronts of a workgroup.  (Of heads of more than 128 channels a SIMD holds one: two workgroups of two are busy when one of four waits: three
// prompts of 2633 rows of 8 heads of 256 in bf16 111 -> 95 us, in fp32 204 -> 198; the 2462 fp32 rows of kv_any.hip with 8, 4 and 2: 67, 52, 52, 2633
// of TinyLlama's shape in fp32 211, 179, 189.)
constexpr int kv_waves_of(int padded) { return padded > 128 ? 2 : 4; }
inline int kv_padded(int h) { return h <= 32 ? 32 : h <= 64 ? 64 : h <= 128 ? 128 : 256; }
// How many sets of sixteen rows a wavefront may have: two where they fit into the registers of two wavefronts a SIMD.
constexpr int kv_most_sets(int padded, int size) { return padded * size <= 256 ? 2 : 1; }
inline int kv_most_sets(const KvCache& c) { return kv_most_sets(kv_padded(c.h), c.dtype == MDI_BF16 ? 2 : 4); }
// Two sets of sixteen rows a workgroup read the keys and values half as often, one set is twice as many workgroups: two from 512
// workgroups on (fp32, 12 heads of 64: 1600 rows 47 against 50 us, 800 rows 29 against 22; bf16 heads of 96: 1600 rows 31 against 34, 800
// rows 18 against 17).  Pieces only while there is no workgroup for every compute unit, of four blocks or more: 16 fp32 tokens behind
// 3000 of the TinyLlama shape in 1 piece 40 us, in 2 28, in 4 - a workgroup for each - 23, in 16 26; 2633 rows of it in 1 piece 170, in 2 181.
inline KvPlan kv_any_plan(const KvCache& c, const KvRows& r, int H, const KvSight& w, double* us) {
  const int n = std::max(1, std::min(r.n, r.n_rows)), rows = (r.n_rows + n - 1) / n, sh = std::min(kv_heads_shift(c, H), 4);
  auto wgs_of = [&](int sets) { const int bp = 16 * sets >> sh; return (double)n * ((rows + bp - 1) / bp) * (H >> sh); };
  const int sets = r.start && kv_most_sets(c) == 2 && rows << sh > 16 && wgs_of(2) >= 512. ? 2 : 1;
  const double wgs = r.start ? wgs_of(sets) : (double)r.n * c.K * kv8_groups(c, H);
  const int reach = (int)std::min<long>(r.max_ctx, (long)w.window + (r.start ? 16 * sets >> sh : 1) + w.sinks + 4 * 31);   // places of a workgroup
  const int most = (reach + 63) / 64;
  const int want = (int)std::min(64., std::max(1., std::min(most / 4., std::ceil(1024. / kv_waves_of(kv_padded(c.h)) / wgs)))), chunk = (most + want - 1) / want, splits = (most + chunk - 1) / chunk;
  // 128 keys of a workgroup's rows take `step` us of a compute unit, a workgroup some more to begin and end
  const bool wide = c.h > 64;
  const double seen = std::min<double>(reach, r.max_ctx - 0.5 * std::min(r.max_ctx, rows)), step = sets == 2 ? (wide ? 1.35 : 0.8) : (wide ? 0.9 : 0.5);
  *us = std::max(3 + std::ceil(reach / (128. * splits)), wgs * (seen / 128 * step + splits * (wide ? 3.5 : 2.2)) / 256);
  if (splits > 1) *us += 2 + (double)r.n_rows * H * (1 / 2000. + splits * (double)c.h / 4e6);
  return KvPlan{kKvAny, chunk, splits, 0, sets, 0};
}

// ---- Packed rows in bf16 with heads of 64 (kv_prompt.hip) or 128 (kv_prompt_wide.hip).
inline bool kv_prompt_supported(const KvCache& c, const KvRows& r) { return r.start && c.dtype == MDI_BF16 && (c.h == 64 || c.h == 128); }
// Rows and groups of a workgroup and pieces of a row's blocks.  A step of 64 keys (of 128, with two groups) takes `step` us, a workgroup
// some more to begin and end; what is divided is added by a second launch.  How long the single samples are is on the device: they are
// taken for equal, all as long as the longest, so `us` is more than such a call takes (6000 + 2000 + 500 of the 8B shape: 485 us, taken for
// 800), and serves to compare.  `step` and the rest are fitted to 29 calls with one and two groups and 1 to 16 pieces.
// Two groups against one: 1024 rows of the 7B shape 31 and 48 us, 2048 68 and 85, 1500 of TinyLlama 30 and 47, 4000 of it 137 and 127, 6000 + 2000 +
// 500 of the 8B shape 522 and 485.  4 pieces of 64 rows behind 8000 of the 8B shape, two groups in 1, 2, 4 and 8 pieces: 152, 92, 68 and 80 us.
// Heads of 128 also by workgroups of two wavefronts, two at a time on a compute unit: each reads what four read, but begins and ends beside
// the other, and 128 rows see fewer keys between them.  Against four: 6000 + 2000 + 500 of the 7B shape with windows of 512, 1024 and
// 2048 185 and 208, 248 and 266, 353 and 365 us, 8 of 1024 148 and 162; of the 8B shape 487 and 485, 2048 of the 7B shape 83 and 85.
struct KvPromptPlan { int rows, groups, splits; double us; };
inline KvPromptPlan kv_prompt_forms(const KvCache& c, const KvRows& r, int H, const KvSight& w) {
  const int n = std::max(1, std::min(r.n, r.n_rows)), n_rows = (r.n_rows + n - 1) / n, sh = kv_heads_shift(c, H);   // rows of a sample
  const double heads = (double)r.n_rows * H;
  struct Form { int rows, groups, at_once; double step, ends; };  // workgroups of a compute unit; us of a step and of a workgroup's beginning and end
  const Form forms[] = {{256, 1, 1, c.h == 128 ? 2.55 : 1.7, 6}, {128, 2, 1, c.h == 128 ? 2.85 : 1.95, 7}, {128, 1, 2, 2.8, 4}};
  KvPromptPlan best{256, 1, 1, 1e30};
  for (const Form& f : forms) {
    if (f.at_once == 2 && c.h != 128) continue;
    const int bp = f.rows >> sh, most = (int)std::min<long>(r.max_ctx, (long)w.window + w.sinks + std::min(bp, n_rows) + 64);
    const double items = (double)n * ((n_rows + bp - 1) / bp) * (H >> sh), slots = 256 * f.at_once;
    const double seen = std::min<double>(most, r.max_ctx - 0.5 * std::min(r.max_ctx, n_rows));   // what a workgroup sees, on average
    for (int s = 1; s <= 32; s *= 2) {
      if (s > 1 && most < 256 * s) break;
      double us = std::max(std::ceil(most / (64. * f.groups * s)) * f.step + 6, items / slots * (seen / (64. * f.groups) * f.step + s * f.ends));
      if (s > 1) us += 2 + heads / 2000 + heads * s * c.h / 4e6;
      if (us < best.us) best = KvPromptPlan{f.rows, f.groups, s, us};
    }
  }
  return best;
}
inline KvPlan kv_prompt_plan(const KvCache& c, const KvRows& r, int H, const KvSight& w, double* us) {
  const KvPromptPlan p = kv_prompt_forms(c, r, H, w);
  // blocks that a workgroup of up to `bp` positions may have: of the first ones, and of a window that begins inside one
  const int bp = p.rows >> kv_heads_shift(c, H);
  const long most = std::min<long>(((long)r.max_ctx + 63) / 64, ((long)w.window + bp + 62) / 64 + 1 + ((long)w.sinks + 63) / 64);
  const int chunk = (int)((most + p.splits - 1) / p.splits);
  *us = p.us;
  return KvPlan{kKvPrompt, chunk, (int)((most + chunk - 1) / chunk), 0, p.groups, p.rows};
}

// Packed rows in bf16 with heads of 64 or 128 are kv_prompt.hip's (256 or 128 rows of position and head to a workgroup) or kv_any.hip's (16
// or 32), whichever should take less time by their plans: 64 samples of 2 rows behind 500 of the 8B shape 33 against 26 us, 512 rows of
// the 7B shape 21.4 against 16.5, 512 of 12 heads of 64 14.9 against 9.5, but 24 prompts of 40 rows of the 8B shape 14.5 against 20.5, 8 of 333
// rows of TinyLlama's 28 against 33.
inline KvPlan kv_plan(const KvCache& c, const KvRows& r, int H, const KvSight& w) {
  if (kv_decode_supported(c, r)) return kv_decode_plan(c, r, H, w);
  double any_us, us;
  const KvPlan any = kv_any_plan(c, r, H, w, &any_us);
  if (!kv_prompt_supported(c, r)) return any;
  const KvPlan prompt = kv_prompt_plan(c, r, H, w, &us);
  return any_us < us ? any : prompt;
}

}  // namespace mdi
