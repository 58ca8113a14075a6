// Attention over the cache in the storage type: the simple form, for any head and type, and the launch that adds the pieces of rows
// which were divided.
#include <algorithm>

#include "kv_device.h"

namespace mdi {
namespace {

// One workgroup per row, head and piece of what the row sees, its wavefronts' sums folded at the end.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_kv_attn(KvCache c, KvRows r, KvAttn a, int L) {
  __shared__ float sm[4][8 * 32 + 2];
  const int row = blockIdx.x / a.H, head = blockIdx.x - row * a.H, kv = head / (a.H / c.K), piece = blockIdx.y;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = c.h;
  const Kv8View v = kv8_view(c, r, row);
  if (v.sample < 0) return;
  T* out = (T*)a.out + ((long)row * a.out_stride + (long)head * h);
  const int t = v.seen ? kv8_table_row(c, r, v.sample) : -1, item = row * a.H + head;
  if (t < 0) {
    if (piece) return;
    for (int e = threadIdx.x; e < h; e += kBlock) Storage<T>::put(out + e, 0.f);
    if (a.plan.splits > 1 && threadIdx.x == 0) kv_part_counts(a, c, r)[item] = 1;
    return;
  }
  const int32_t* table = c.tables + (long)t * c.table_stride;
  const KvSpan span = kv_span(a.sight, v.seen);
  const int n = span.places(), lo = piece * a.plan.chunk, hi = min(n, lo + a.plan.chunk), pieces = (n + a.plan.chunk - 1) / a.plan.chunk;
  if (lo >= hi) return;
  const int ch = 8 * (lane & (L - 1)), sub = lane / L, tpw = 64 / L;
  const bool live = ch < h;
  float q[8] = {};
  if (live) KvType<T>::load8((const T*)a.q + ((long)row * a.q_stride + (long)head * h + ch), q);
#pragma unroll
  for (int j = 0; j < 8; ++j) q[j] *= a.scale;
  const KvSums mine = kv_attend<T>(c, table, kv, span, q, L, ch, live, lo + wave * tpw, 4 * tpw, hi);
  if (sub == 0) {
    if (live)
#pragma unroll
      for (int j = 0; j < 8; ++j) sm[wave][ch + j] = mine.o[j];
    if (lane == 0) { sm[wave][h] = mine.m; sm[wave][h + 1] = mine.l; }
  }
  __syncthreads();
  float to = kKvNone;
  for (int w = 0; w < 4; ++w) to = fmaxf(to, sm[w][h]);
  for (int e = threadIdx.x; e < h; e += kBlock) {
    float sum = 0.f, ls = 0.f;
    for (int w = 0; w < 4; ++w) { const float f = exp2f(sm[w][h] - to); sum += sm[w][e] * f; ls += sm[w][h + 1] * f; }
    if (pieces == 1) Storage<T>::put(out + e, sum / ls);
    else { kv_part_sums(a, c, item, piece)[e] = sum; if (e == 0) *kv_part_marks(a, c, r, item, piece) = make_float2(to, ls); }
  }
  if (piece == 0 && a.plan.splits > 1 && threadIdx.x == 0) kv_part_counts(a, c, r)[item] = pieces;
}

// Up to 64 pieces of every row and head, always in the same order: a wavefront each, 64 / (h / 4) pieces at a time, a float4 a lane.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_kv_join_few(KvCache c, KvRows r, KvAttn a) {
  const int lane = threadIdx.x & 63, h = c.h, item = __builtin_amdgcn_readfirstlane(blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6)), row = item / a.H;
  if (row >= r.n_rows || kv8_sample_of(r, row) < 0) return;      // nobody's: nothing was left
  const int n = __builtin_amdgcn_readfirstlane(min(kv_part_counts(a, c, r)[item], a.plan.splits));
  if (n <= 1) return;                                            // finished where it was computed
  const float2 mark = lane < n ? *kv_part_marks(a, c, r, item, lane) : make_float2(kKvNone, 0.f);
  float to = mark.x;
  for (int off = 32; off >= 1; off >>= 1) to = fmaxf(to, __shfl_xor(to, off, 64));
  const float f = exp2f(mark.x - to), l = wave_sum(mark.y * f);
  const int per = h / 4, at_once = 64 / per, slot = lane / per, ch = 4 * (lane - slot * per);
  const float* sums = kv_part_sums(a, c, item, 0) + ch;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
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
  T* out = (T*)a.out + ((long)row * a.out_stride + (long)(item - row * a.H) * h + ch);
  const float inv = 1.f / l;
  Storage<T>::put(out, all.x * inv); Storage<T>::put(out + 1, all.y * inv); Storage<T>::put(out + 2, all.z * inv); Storage<T>::put(out + 3, all.w * inv);
}

// More of them: a workgroup each, 256 / (h / 4) pieces at a time, a float4 a thread.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_kv_join(KvCache c, KvRows r, KvAttn a) {
  __shared__ float weight[kBlock], red[8];
  __shared__ float4 fold[kBlock];
  const int item = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = c.h, row = item / a.H;
  if (kv8_sample_of(r, row) < 0) return;                         // nobody's: nothing was left
  const int n = min(kv_part_counts(a, c, r)[item], a.plan.splits);
  if (n <= 1) return;                                            // finished where it was computed
  const int per = h / 4, at_once = kBlock / per, slot = tid / per, ch = 4 * (tid - slot * per);
  const float* sums = kv_part_sums(a, c, item, 0) + ch;
  const float2* marks = kv_part_marks(a, c, r, item, 0);
  float m = kKvNone, l = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p0 = 0; p0 < n; p0 += kBlock) {
    const int k = min(kBlock, n - p0);
    const float2 mark = tid < k ? marks[p0 + tid] : make_float2(kKvNone, 0.f);
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
  T* out = (T*)a.out + ((long)row * a.out_stride + (long)(item - row * a.H) * h + ch);
  const float inv = 1.f / l;
  Storage<T>::put(out, acc.x * inv); Storage<T>::put(out + 1, acc.y * inv); Storage<T>::put(out + 2, acc.z * inv); Storage<T>::put(out + 3, acc.w * inv);
}

template <typename T>
void launch(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a) {
  int L = 1;
  while (8 * L < c.h) L *= 2;
  const unsigned items = (unsigned)(r.n_rows * a.H);
  if (kv_decode_supported(c, r)) launch_kv_decode(s, c, r, a);
  else if (kv_prompt_supported(c, r)) launch_kv_prompt(s, c, r, a);
  else hipLaunchKernelGGL((k_kv_attn<T>), dim3(items, a.plan.splits), dim3(kBlock), 0, s, c, r, a, L);
  if (a.plan.splits > 1 && a.plan.splits <= 64) hipLaunchKernelGGL((k_kv_join_few<T>), dim3((items + kBlock / 64 - 1) / (kBlock / 64)), dim3(kBlock), 0, s, c, r, a);
  else if (a.plan.splits > 1) hipLaunchKernelGGL((k_kv_join<T>), dim3(items), dim3(kBlock), 0, s, c, r, a);
}

}  // namespace

KvPlan kv_plan(const KvCache& c, const KvRows& r, int H, const KvSight& w) {
  if (kv_decode_supported(c, r)) return kv_decode_plan(c, r, H, w);
  if (kv_prompt_supported(c, r)) return kv_prompt_plan(c, r, H, w);
  const int most = kv_most_seen(w, r.max_ctx);
  const int want = (int)std::max<long>(1, std::min<long>(64, 1024 / ((long)r.n_rows * H)));
  KvPlan p{};
  p.chunk = std::max(256, ((most + want - 1) / want + 63) / 64 * 64);
  p.splits = (most + p.chunk - 1) / p.chunk;
  return p;
}

void launch_kv_attn(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a) {
  if (c.dtype == MDI_BF16) launch<bf16_t>(s, c, r, a); else launch<float>(s, c, r, a);
}

}  // namespace mdi
