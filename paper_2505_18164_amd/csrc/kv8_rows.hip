// Rows into the 8-bit cache and back out of it.
#include "kv8_device.h"

namespace mdi {
namespace {

constexpr int kUnits = 4;                                        // head rows a lane takes one after the other

__device__ __forceinline__ unsigned group_max(unsigned v, int L) {   // over aligned groups of L lanes
  auto step = [&](unsigned o) { v = max(v, o); };
  if (L >= 2) step(__builtin_amdgcn_update_dpp(0, v, kDppXor1, 0xF, 0xF, false));
  if (L >= 4) step(__builtin_amdgcn_update_dpp(0, v, kDppXor2, 0xF, 0xF, false));
  if (L >= 8) step(__builtin_amdgcn_update_dpp(0, v, kDppHalfMirror, 0xF, 0xF, false));
  if (L >= 16) step(__builtin_amdgcn_update_dpp(0, v, kDppMirror, 0xF, 0xF, false));
  if (L >= 32) step(__shfl_xor(v, 16, 64));
  return v;
}

// What is written into the cache is read once: without a place in the caches for it, 8192 rows of the 7B shape take 46 us instead of
// 60 (and reading them back 71 instead of 73; there, written values without a place take 92).
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <typename T> __device__ __forceinline__ void load8(const T* p, float (&x)[8]);
template <> __device__ __forceinline__ void load8<bf16_t>(const bf16_t* p, float (&x)[8]) {
  const u32x4 w = __builtin_nontemporal_load((const u32x4*)p);
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
}
template <> __device__ __forceinline__ void load8<float>(const float* p, float (&x)[8]) {
  const u32x4 a = __builtin_nontemporal_load((const u32x4*)p), b = __builtin_nontemporal_load((const u32x4*)p + 1);
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[i] = __uint_as_float(a[i]); x[4 + i] = __uint_as_float(b[i]); }
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&x)[8]);
template <> __device__ __forceinline__ void store8<bf16_t>(bf16_t* p, const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f32_to_bf16(x[2 * i]) | ((uint32_t)f32_to_bf16(x[2 * i + 1]) << 16);
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
template <> __device__ __forceinline__ void store8<float>(float* p, const float (&x)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}

// Where position `pos` of a sample lies: its page and slot; false when the position or the page is not of this cache.
__device__ __forceinline__ bool place(const Kv8Cache& c, const Kv8Rows& r, int row, int* page, int* slot) {
  const int s = kv8_sample_of(r, row);
  if (s < 0) return false;
  const int p0 = r.pos[s];
  if (p0 < 0) return false;                                      // a sample that takes no part
  const long far = (long)p0 + (r.start ? row - r.start[s] : 0);
  const int t = kv8_table_row(c, r, s);
  if (t < 0) return false;
  if (far < 0 || far >= r.max_ctx) { kv8_report(c); return false; }
  const int pos = (int)far, at = kv8_page_of(c, pos);
  *page = c.tables[(long)t * c.table_stride + at];
  *slot = pos - at * c.pt;
  if ((unsigned)*page >= (unsigned)c.n_pages) { kv8_report(c); return false; }
  return true;
}

// A wavefront takes 64 / L head rows (keys of all heads, then values of all heads) of one row of the call at a time, kUnits
// times; L lanes hold eight channels each of one.  What bounds it: memory - 8192 rows of the 7B shape, bf16, are quantised in 46 us
// (134 MB in, 69 out: 4.4 TB/s) and read back as fp32 in 71 (69 in, 268 out: 4.8 TB/s) -, and for few rows
// the way to the page: sample, table, page, each behind the one before, 4.5 us.  (Workgroups of sixteen rows that follow one another,
// whose scales and codes then lie together in a page, are slower to write: 70 us when that was 61.)
// (The code is x c + 1.5 2^23: one addition whose rounding is the one to a whole number, and whose low byte is the code.)
template <typename T, bool kWrite>
__global__ __launch_bounds__(kBlock) void k_kv8_rows(Kv8Cache c, Kv8Rows r, Kv8RowsIO io, int L, int l_sh, int pieces) {
  const int lane = threadIdx.x & 63;
  const unsigned item = __builtin_amdgcn_readfirstlane(blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6));
  const int row = (int)(item / (unsigned)pieces), piece = (int)(item - (unsigned)row * (unsigned)pieces);
  if (row >= r.n_rows) return;
  int page, slot;
  if (!place(c, r, row, &page, &slot)) return;
  const int ch = 8 * (lane & (L - 1));
  const int hr0 = (piece * kUnits << (6 - l_sh)) + (lane >> l_sh), step = 64 >> l_sh;
  float x[kUnits][8];
  uint2 code[kUnits];
  float scale[kUnits];
  bool live[kUnits];
  long at[kUnits], row_at[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int hr = hr0 + u * step, side = hr >= c.K, kv = hr - (side ? c.K : 0);
    live[u] = hr < 2 * c.K && ch < c.h;
    row_at[u] = (((long)page * c.K + kv) * 2 + side) * c.pt + slot;
    at[u] = (long)row * io.row_stride + (long)kv * io.head_stride + ch;
    if (!live[u]) continue;
    if constexpr (kWrite) {
      load8<T>((const T*)(side ? io.v : io.k) + at[u], x[u]);
    } else {
      code[u] = *reinterpret_cast<const uint2*>(c.codes + row_at[u] * c.h + ch);
      scale[u] = c.scales[row_at[u]];
    }
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    if constexpr (kWrite) {
      unsigned top = 0;                                          // bits of a magnitude: they order like it, infinities and NaN on top
      if (live[u])
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[u][j]) & 0x7FFFFFFFu);
      top = group_max(top, L);
      if (!live[u]) continue;
      const bool fine = top < 0x7F800000u, some = fine && top >= 0x0D800000u;   // finite; at least 2^-100
      const float t = some ? __uint_as_float(top) : 1.f, m = 127.f / t;
      unsigned w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = some ? __float_as_uint(fmaf(x[u][j], m, 12582912.f)) & 0xFFu : 0u;
      *reinterpret_cast<uint2*>(c.codes + row_at[u] * c.h + ch) =
          make_uint2(w[0] | w[1] << 8 | w[2] << 16 | w[3] << 24, w[4] | w[5] << 8 | w[6] << 16 | w[7] << 24);
      if (ch == 0) c.scales[row_at[u]] = some ? t / 127.f : fine ? 0.f : __uint_as_float(0x7FC00000u);
    } else {
      if (!live[u]) continue;
      const bool side = hr0 + u * step >= c.K;
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = (float)(int8_t)((j < 4 ? code[u].x : code[u].y) >> (8 * (j & 3)) & 0xFFu) * scale[u];
      store8<T>((T*)(side ? io.v : io.k) + at[u], y);
    }
  }
}

template <bool kWrite>
void launch_rows(hipStream_t s, int dtype, const Kv8Cache& c, const Kv8Rows& r, const Kv8RowsIO& io) {
  int L = 1, l_sh = 0;
  while (8 * L < c.h) { L *= 2; ++l_sh; }
  const int per = kUnits * (64 / L), pieces = (2 * c.K + per - 1) / per;
  const dim3 grid((unsigned)(((long)r.n_rows * pieces + kBlock / 64 - 1) / (kBlock / 64))), block(kBlock);
  if (dtype == MDI_BF16) hipLaunchKernelGGL((k_kv8_rows<bf16_t, kWrite>), grid, block, 0, s, c, r, io, L, l_sh, pieces);
  else hipLaunchKernelGGL((k_kv8_rows<float, kWrite>), grid, block, 0, s, c, r, io, L, l_sh, pieces);
}

}  // namespace

void launch_kv8_write(hipStream_t s, int dtype, const Kv8Cache& c, const Kv8Rows& r, const Kv8RowsIO& io) { launch_rows<true>(s, dtype, c, r, io); }
void launch_kv8_read(hipStream_t s, int dtype, const Kv8Cache& c, const Kv8Rows& r, const Kv8RowsIO& io) { launch_rows<false>(s, dtype, c, r, io); }

}  // namespace mdi
