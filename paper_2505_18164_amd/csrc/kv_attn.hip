// Attention over the cache in the storage type: which kernel serves a call, and the launch that adds the pieces of rows that were divided.
#include <algorithm>

#include "kv_device.h"
#include "kv_plan.h"

namespace mdi {
namespace {

// Up to 64 pieces of every row and head, always in the same order.  Most of it is a launch behind another: 4 to 5 us for 128 to 512 rows and heads,
// 8 for 8192 with four pieces.  A wavefront each (a workgroup each took 19 for those), 64 / (h / 4) pieces at a time, a float4 a lane.
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

// More of them (of single tokens in bf16): a workgroup each, 256 / (h / 4) pieces at a time, a float4 a thread.
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
  bf16_t* out = (bf16_t*)a.out + ((long)row * a.out_stride + (long)(item - row * a.H) * h + ch);
  const float inv = 1.f / l;
  Storage<bf16_t>::put(out, acc.x * inv); Storage<bf16_t>::put(out + 1, acc.y * inv); Storage<bf16_t>::put(out + 2, acc.z * inv); Storage<bf16_t>::put(out + 3, acc.w * inv);
}

void launch_join(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a) {
  const unsigned items = (unsigned)(r.n_rows * a.H);
  const dim3 grid((items + kBlock / 64 - 1) / (kBlock / 64)), block(kBlock);
  if (a.plan.splits > 64) hipLaunchKernelGGL(k_kv_join, dim3(items), block, 0, s, c, r, a);   // (kv_decode.hip's alone may have more than 64)
  else if (c.dtype == MDI_BF16) hipLaunchKernelGGL((k_kv_join_few<bf16_t>), grid, block, 0, s, c, r, a);
  else hipLaunchKernelGGL((k_kv_join_few<float>), grid, block, 0, s, c, r, a);
}

}  // namespace

void launch_kv_attn(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a) {
  if (a.plan.kernel == kKvDecode) launch_kv_decode(s, c, r, a);
  else if (a.plan.kernel == kKvPrompt) launch_kv_prompt(s, c, r, a);
  else launch_kv_any(s, c, r, a);
  if (a.plan.splits > 1) launch_join(s, c, r, a);
}

}  // namespace mdi
