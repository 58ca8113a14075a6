// Attention over the 8-bit cache: the form for any head, and the launch that adds the pieces of rows which were divided.
#include <algorithm>

#include "kv8_device.h"

namespace mdi {
namespace {

__device__ __forceinline__ float sum_of(float v, int L) {
  for (int off = 1; off < L; off <<= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// One workgroup per row, head and piece of the positions.  L lanes hold eight channels each of a position; a lane group keeps
// its own running (reference, sum, output), which are folded at the end.
__global__ __launch_bounds__(kBlock) void k_kv8_attn(Kv8Cache c, Kv8Rows r, Kv8Attn a, int L) {
  __shared__ float sm[4][8 * 32 + 2];
  const int row = blockIdx.x / a.H, head = blockIdx.x - row * a.H, kv = head / (a.H / c.K), piece = blockIdx.y;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = c.h;
  const Kv8View v = kv8_view(c, r, row);
  if (v.sample < 0) return;
  bf16_t* out = a.out + (long)row * a.out_stride + (long)head * h;
  const int32_t* table = v.seen ? kv8_table(c, r, v.sample) : nullptr;
  if (!table) {
    if (piece == 0) for (int e = threadIdx.x; e < h; e += kBlock) out[e] = 0;
    return;
  }
  const int lo = piece * a.plan.chunk, hi = min(v.seen, lo + a.plan.chunk);
  if (lo >= hi) return;
  const int ch = 8 * (lane & (L - 1)), sub = lane / L, tpw = 64 / L;
  const bool live = ch < h;
  float q[8], o[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) { q[j] = live ? bf16_to_f32(a.q[(long)row * a.q_stride + (long)head * h + ch + j]) * a.scale : 0.f; o[j] = 0.f; }
  float m = kKv8None, l = 0.f;
  for (int t0 = lo + wave * tpw; t0 < hi; t0 += 4 * tpw) {
    const int pos = min(t0 + sub, hi - 1), at = kv8_page_of(c, pos);
    const long rk = ((long)kv8_checked_page(c, table[at]) * c.K + kv) * 2 * c.pt + (pos - at * c.pt), rv = rk + c.pt;
    const uint2 kc = live ? *reinterpret_cast<const uint2*>(c.codes + rk * h + ch) : make_uint2(0, 0);
    const uint2 vc = live ? *reinterpret_cast<const uint2*>(c.codes + rv * h + ch) : make_uint2(0, 0);
    const float ks = c.scales[rk], vs = c.scales[rv];
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(q[j], (float)(int8_t)((j < 4 ? kc.x : kc.y) >> (8 * (j & 3))), s);
    s = sum_of(s, L) * ks;
    if (t0 + sub >= hi) continue;
    const float to = fmaxf(m, s), alpha = exp2f(m - to), p = exp2f(s - to), w = p * vs;
    m = to;
    l = l * alpha + p;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = o[j] * alpha + w * (float)(int8_t)((j < 4 ? vc.x : vc.y) >> (8 * (j & 3)));
  }
  for (int off = L; off < 64; off <<= 1) {
    const float m1 = __shfl_xor(m, off, 64), l1 = __shfl_xor(l, off, 64), to = fmaxf(m, m1), a0 = exp2f(m - to), a1 = exp2f(m1 - to);
    l = l * a0 + l1 * a1;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = o[j] * a0 + __shfl_xor(o[j], off, 64) * a1;
    m = to;
  }
  if (sub == 0) {
    if (live)
#pragma unroll
      for (int j = 0; j < 8; ++j) sm[wave][ch + j] = o[j];
    if (lane == 0) { sm[wave][h] = m; sm[wave][h + 1] = l; }
  }
  __syncthreads();
  float to = kKv8None;
  for (int w = 0; w < 4; ++w) to = fmaxf(to, sm[w][h]);
  const bool whole = v.seen <= a.plan.chunk;
  float* part = a.part + (((long)row * a.H + head) * a.plan.splits + piece) * (h + 4);
  for (int e = threadIdx.x; e < h; e += kBlock) {
    float sum = 0.f, ls = 0.f;
    for (int w = 0; w < 4; ++w) { const float f = exp2f(sm[w][h] - to); sum += sm[w][e] * f; ls += sm[w][h + 1] * f; }
    if (whole) out[e] = f32_to_bf16(sum / ls);
    else { part[e] = sum; if (e == 0) { part[h] = to; part[h + 1] = ls; } }
  }
}

// A wavefront per row and head: adds the pieces, in their order.
__global__ __launch_bounds__(kBlock) void k_kv8_join(Kv8Cache c, Kv8Rows r, Kv8Attn a) {
  const int item = __builtin_amdgcn_readfirstlane(blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6)), lane = threadIdx.x & 63, h = c.h;
  const int row = item / a.H;
  if (row >= r.n_rows) return;
  const Kv8View v = kv8_view(c, r, row);
  if (v.sample < 0 || v.seen <= a.plan.chunk) return;            // no sample's, or finished in its only piece
  const int t = r.table ? r.table[v.sample] : v.sample;
  if ((unsigned)t >= (unsigned)c.n_tables) return;               // its zeros are written
  const int n = (v.seen + a.plan.chunk - 1) / a.plan.chunk;
  const float* part = a.part + (long)item * a.plan.splits * (h + 4);
  float to = kKv8None;
  for (int i = lane; i < n; i += 64) to = fmaxf(to, part[(long)i * (h + 4) + h]);
  for (int off = 32; off >= 1; off >>= 1) to = fmaxf(to, __shfl_xor(to, off, 64));
  float sum[4] = {0.f, 0.f, 0.f, 0.f}, ls = 0.f;
  for (int i = 0; i < n; ++i) {
    const float* p = part + (long)i * (h + 4);
    const float f = exp2f(p[h] - to);
    ls += p[h + 1] * f;
#pragma unroll
    for (int j = 0; j < 4; ++j) if (lane + 64 * j < h) sum[j] += p[lane + 64 * j] * f;
  }
  bf16_t* out = a.out + (long)row * a.out_stride + (long)(item - row * a.H) * h;
#pragma unroll
  for (int j = 0; j < 4; ++j) if (lane + 64 * j < h) out[lane + 64 * j] = f32_to_bf16(sum[j] / ls);
}

}  // namespace

Kv8Plan kv8_plan(const Kv8Cache& c, const Kv8Rows& r, int H) {
  if (kv8_decode_supported(c, r)) return kv8_decode_plan(c, r, H);
  const long items = (long)r.n_rows * H;
  const int want = (int)std::max<long>(1, std::min<long>(64, 1024 / items));
  int chunk = std::max(256, ((r.max_ctx + want - 1) / want + 63) / 64 * 64);
  return Kv8Plan{chunk, (r.max_ctx + chunk - 1) / chunk};
}

void launch_kv8_attn(hipStream_t s, const Kv8Cache& c, const Kv8Rows& r, const Kv8Attn& a) {
  if (kv8_decode_supported(c, r)) {
    launch_kv8_decode(s, c, r, a);
  } else {
    int L = 1;
    while (8 * L < c.h) L *= 2;
    hipLaunchKernelGGL(k_kv8_attn, dim3((unsigned)(r.n_rows * a.H), a.plan.splits), dim3(kBlock), 0, s, c, r, a, L);
  }
  if (a.plan.splits > 1)
    hipLaunchKernelGGL(k_kv8_join, dim3((unsigned)(((long)r.n_rows * a.H + 3) / 4)), dim3(kBlock), 0, s, c, r, a);
}

}  // namespace mdi
