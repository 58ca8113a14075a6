// Attention over the 8-bit cache: the form for any head, and the launch that adds the pieces of rows which were divided.
#include <algorithm>

#include "kv8_device.h"

namespace mdi {
namespace {

// One workgroup per row, head and piece of the positions, its wavefronts' sums folded at the end.  It serves heads of other than 64
// or 128 channels, reads the cache once for every query head, and is bound by vector instructions: 16 tokens of 8100 positions of the
// 8B shape would take it 374 us (kv8_decode.hip: 48), a prompt of 1024 of the 7B shape 710 (kv8_prompt.hip: 32).
__global__ __launch_bounds__(kBlock) void k_kv8_attn(Kv8Cache c, Kv8Rows r, Kv8Attn a, int L) {
  __shared__ float sm[4][8 * 32 + 2];
  const int row = blockIdx.x / a.H, head = blockIdx.x - row * a.H, kv = head / (a.H / c.K), piece = blockIdx.y;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = c.h;
  const Kv8View v = kv8_view(c, r, row);
  if (v.sample < 0) return;
  bf16_t* out = a.out + (long)row * a.out_stride + (long)head * h;
  const int t = v.seen ? kv8_table_row(c, r, v.sample) : -1;
  const int32_t* table = c.tables + (long)max(t, 0) * c.table_stride;
  if (t < 0) {
    if (piece == 0) for (int e = threadIdx.x; e < h; e += kBlock) out[e] = 0;
    return;
  }
  const int lo = piece * a.plan.chunk, hi = min(v.seen, lo + a.plan.chunk);
  if (lo >= hi) return;
  const int ch = 8 * (lane & (L - 1)), sub = lane / L, tpw = 64 / L;
  const bool live = ch < h;
  float q[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) q[j] = live ? bf16_to_f32(a.q[(long)row * a.q_stride + (long)head * h + ch + j]) * a.scale : 0.f;
  const Kv8Sums mine = kv8_attend(c, table, kv, q, L, ch, live, lo + wave * tpw, 4 * tpw, hi);
  if (sub == 0) {
    if (live)
#pragma unroll
      for (int j = 0; j < 8; ++j) sm[wave][ch + j] = mine.o[j];
    if (lane == 0) { sm[wave][h] = mine.m; sm[wave][h + 1] = mine.l; }
  }
  __syncthreads();
  float to = kKv8None;
  for (int w = 0; w < 4; ++w) to = fmaxf(to, sm[w][h]);
  const bool whole = v.seen <= a.plan.chunk;
  float* part = kv8_part_sums(a, c, row * a.H + head, piece);
  for (int e = threadIdx.x; e < h; e += kBlock) {
    float sum = 0.f, ls = 0.f;
    for (int w = 0; w < 4; ++w) { const float f = exp2f(sm[w][h] - to); sum += sm[w][e] * f; ls += sm[w][h + 1] * f; }
    if (whole) out[e] = f32_to_bf16(sum / ls);
    else { part[e] = sum; if (e == 0) *kv8_part_marks(a, c, r, row * a.H + head, piece) = make_float2(to, ls); }
  }
}

// Pieces of equal length, 64 at most: a wavefront per row and head adds them, 64 / (h / 4) at a time, a float4 a lane.  (As
// k_kv8_join, a workgroup each: 256 rows of 32 heads of 128, four pieces: 19.0 us instead of 8.2.)
__global__ __launch_bounds__(kBlock) void k_kv8_join_few(Kv8Cache c, Kv8Rows r, Kv8Attn a) {
  const int lane = threadIdx.x & 63, h = c.h, item = __builtin_amdgcn_readfirstlane(blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6)), row = item / a.H;
  if (row >= r.n_rows) return;
  const Kv8View v = kv8_view(c, r, row);
  if (v.sample < 0 || v.seen <= a.plan.chunk) return;            // finished where it was computed
  if (kv8_table_row(c, r, v.sample) < 0) return;                 // its zeros are written
  const int n = (v.seen + a.plan.chunk - 1) / a.plan.chunk;
  const float2 mark = lane < n ? *kv8_part_marks(a, c, r, item, lane) : make_float2(kKv8None, 0.f);
  float to = mark.x;
  for (int off = 32; off >= 1; off >>= 1) to = fmaxf(to, __shfl_xor(to, off, 64));
  const float f = exp2f(mark.x - to), l = wave_sum(mark.y * f);
  const int per = h / 4, at_once = 64 / per, slot = lane / per, ch = 4 * (lane - slot * per);
  const float* sums = kv8_part_sums(a, c, item, 0) + ch;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p0 = 0; p0 < n; p0 += at_once) {
    const int p = p0 + slot;
    const float w = __shfl(f, min(p, 63), 64);
    if (slot >= at_once || p >= n) continue;
    const float4 x = *reinterpret_cast<const float4*>(sums + (long)p * h);
    acc.x += x.x * w; acc.y += x.y * w; acc.z += x.z * w; acc.w += x.w * w;
  }
  float4 all = acc;
  for (int i = 1; i < at_once; ++i) {
    const int from = min(i * per + lane, 63);
    all.x += __shfl(acc.x, from, 64); all.y += __shfl(acc.y, from, 64); all.z += __shfl(acc.z, from, 64); all.w += __shfl(acc.w, from, 64);
  }
  if (slot) return;
  bf16_t* out = a.out + (long)row * a.out_stride + (long)(item - row * a.H) * h + ch;
  const float inv = 1.f / l;
  *reinterpret_cast<uint2*>(out) = make_uint2((uint32_t)f32_to_bf16(all.x * inv) | ((uint32_t)f32_to_bf16(all.y * inv) << 16),
                                              (uint32_t)f32_to_bf16(all.z * inv) | ((uint32_t)f32_to_bf16(all.w * inv) << 16));
}

// Shares of the stream of tiles, any number of them: a workgroup per row and head, always in the same order: 256 / (h / 4) pieces at a
// time, a float4 a thread.
// References and sums of weights are looked at 256 pieces at a time.  (One wavefront that took piece after piece: 237 us for 313
// pieces of 32 heads, 16 us for 16 pieces of 512.)
__global__ __launch_bounds__(kBlock) void k_kv8_join(Kv8Cache c, Kv8Rows r, Kv8Attn a) {
  __shared__ float weight[kBlock], red[8];
  __shared__ float4 fold[kBlock];
  const int item = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = c.h;
  const int row = item / a.H;
  const Kv8View v = kv8_view(c, r, row);
  if (v.sample < 0 || v.seen == 0) return;
  if (kv8_table_row(c, r, v.sample) < 0) return;                 // its zeros are written
  const int groups = kv8_groups(c, a.H), head = item - row * a.H, G = a.H / c.K;
  const Kv8Stream all = kv8_stream(c, r, a.plan, c.K * groups, row, kv8_seen(c, r, lane));
  const int tiles = kv8_tiles(v.seen), from = all.before * c.K * groups + (head / G * groups + head % G / 16) * (tiles + kKv8Begin) + kKv8Begin;
  const int n = (from + tiles - 1) / all.per - from / all.per + 1;   // the row's pieces
  if (n == 1) return;                                            // finished where it was computed
  const int per = h / 4, at_once = kBlock / per, slot = tid / per, ch = 4 * (tid - slot * per);
  const float* sums = kv8_part_sums(a, c, item, 0) + ch;
  const float2* marks = kv8_part_marks(a, c, r, item, 0);
  float m = kKv8None, l = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p0 = 0; p0 < n; p0 += kBlock) {
    const int k = min(kBlock, n - p0);
    const float2 mark = tid < k ? marks[p0 + tid] : make_float2(kKv8None, 0.f);
    float to = mark.x;
    for (int off = 32; off >= 1; off >>= 1) to = fmaxf(to, __shfl_xor(to, off, 64));
    if (lane == 0) red[wave] = to;
    __syncthreads();
    to = fmaxf(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])), m);
    const float f = exp2f(mark.x - to), alpha = exp2f(m - to);
    const float ls = wave_sum(mark.y * f);
    weight[tid] = f;
    if (lane == 0) red[4 + wave] = ls;
    __syncthreads();
    m = to;
    l = l * alpha + (red[4] + red[5] + red[6] + red[7]);
    acc.x *= alpha; acc.y *= alpha; acc.z *= alpha; acc.w *= alpha;
    if (slot < at_once)
#pragma unroll 4
      for (int p = slot; p < k; p += at_once) {
        const float4 x = *reinterpret_cast<const float4*>(sums + (long)(p0 + p) * h);
        const float w = weight[p];
        acc.x += x.x * w; acc.y += x.y * w; acc.z += x.z * w; acc.w += x.w * w;
      }
    __syncthreads();
  }
  fold[tid] = acc;
  __syncthreads();
  if (slot) return;
  for (int i = 1; i < at_once; ++i) {
    const float4 x = fold[i * per + tid];
    acc.x += x.x; acc.y += x.y; acc.z += x.z; acc.w += x.w;
  }
  bf16_t* out = a.out + (long)row * a.out_stride + (long)(item - row * a.H) * h + ch;
  const float inv = 1.f / l;
  *reinterpret_cast<uint2*>(out) = make_uint2((uint32_t)f32_to_bf16(acc.x * inv) | ((uint32_t)f32_to_bf16(acc.y * inv) << 16),
                                              (uint32_t)f32_to_bf16(acc.z * inv) | ((uint32_t)f32_to_bf16(acc.w * inv) << 16));
}

}  // namespace

Kv8Plan kv8_plan(const Kv8Cache& c, const Kv8Rows& r, int H, size_t part_limit) {
  Kv8Plan p{};
  if (kv8_decode_supported(c, r)) {
    p = kv8_decode_plan(c, r, H);
  } else if (kv8_prompt_supported(c, r)) {
    p = kv8_prompt_plan(c, r, H, part_limit);
  } else {
    const int want = (int)std::max<long>(1, std::min<long>(64, 1024 / ((long)r.n_rows * H)));
    p.chunk = std::max(256, ((r.max_ctx + want - 1) / want + 63) / 64 * 64);
    p.splits = (r.max_ctx + p.chunk - 1) / p.chunk;
  }
  return kv8_part_bytes(p, c, r, H) <= part_limit ? p : Kv8Plan{r.max_ctx, 1, 0, 1};
}

void launch_kv8_attn(hipStream_t s, const Kv8Cache& c, const Kv8Rows& r, const Kv8Attn& a) {
  if (kv8_decode_supported(c, r)) {
    launch_kv8_decode(s, c, r, a);
  } else if (kv8_prompt_supported(c, r)) {
    launch_kv8_prompt(s, c, r, a);
  } else {
    int L = 1;
    while (8 * L < c.h) L *= 2;
    hipLaunchKernelGGL(k_kv8_attn, dim3((unsigned)(r.n_rows * a.H), a.plan.splits), dim3(kBlock), 0, s, c, r, a, L);
  }
  const unsigned items = (unsigned)(r.n_rows * a.H);
  if (a.plan.wgs) hipLaunchKernelGGL(k_kv8_join, dim3(items), dim3(kBlock), 0, s, c, r, a);
  else if (a.plan.splits > 1) hipLaunchKernelGGL(k_kv8_join_few, dim3((items + kBlock / 64 - 1) / (kBlock / 64)), dim3(kBlock), 0, s, c, r, a);
}

}  // namespace mdi
