// Rows of the fused QKV product into the cache in the storage type: query and key heads are normalised and rotated on the way.
//
// Norm of a head x [h]: (x - mean) / sqrt(variance + eps) * g + b, or x / sqrt(mean of x^2 + eps) * g + b.  Rotation of the first
// `rot` channels at position p: channels i and i + rot / 2 turn by p * freq[i].  The angle is taken in 64 bits, in turns, and
// reduced there: in 32 it would be off by 2^-24 of itself, 0.007 at position 120000.  Everything else is binary32, rounded once.
//
// Memory bounds it, every row is read and written once: 8192 rows of the 7B shape with norms and rotation, 403 MB, 92 us, 4.4 TB/s (a large
// copy reaches 4.9); 4514 rows of TinyLlama in fp32 with norms, 92 MB, 23 to 24 us.  16 rows of the 8B shape take 5.3 us of the
// GPU, most of them the way from a row to its sample, its page and the page's place, and 6.6 of the host.
#include "kv_device.h"

namespace mdi {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Rows are read once: without a place in the caches.
template <int N> __device__ __forceinline__ void load(const bf16_t* p, float* x) {
  if constexpr (N == 8) {
    const u32x4 w = __builtin_nontemporal_load((const u32x4*)p);
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  } else {
    const u32x2 w = __builtin_nontemporal_load((const u32x2*)p);
#pragma unroll
    for (int i = 0; i < 2; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  }
}
template <int N> __device__ __forceinline__ void load(const float* p, float* x) {
#pragma unroll
  for (int n = 0; n < N; n += 4) {
    const u32x4 w = __builtin_nontemporal_load((const u32x4*)(p + n));
#pragma unroll
    for (int i = 0; i < 4; ++i) x[n + i] = __uint_as_float(w[i]);
  }
}
__device__ __forceinline__ uint32_t pair_of(float lo, float hi) { return (uint32_t)f32_to_bf16(lo) | ((uint32_t)f32_to_bf16(hi) << 16); }
template <int N> __device__ __forceinline__ void store(bf16_t* p, const float* x) {
  if constexpr (N == 8) *reinterpret_cast<u32x4*>(p) = u32x4{pair_of(x[0], x[1]), pair_of(x[2], x[3]), pair_of(x[4], x[5]), pair_of(x[6], x[7])};
  else *reinterpret_cast<u32x2*>(p) = u32x2{pair_of(x[0], x[1]), pair_of(x[2], x[3])};
}
template <int N> __device__ __forceinline__ void store(float* p, const float* x) {
#pragma unroll
  for (int n = 0; n < N; n += 4) *reinterpret_cast<float4*>(p + n) = make_float4(x[n], x[n + 1], x[n + 2], x[n + 3]);
}

// Inputs come in past the caches (through them 101 instead of 93 us for the 8192 rows) and results go out through them: past them it would
// be 86, but the rows and the attention that reads them together 213 instead of 204.  A head's gains and biases are read once a workgroup, into the LDS (from
// memory by every wavefront: 126 instead of 92 us for the 8192 rows).  fp32 rows are read 16 bytes a lane, lanes next to each
// other: 32 bytes a lane, lanes 64 bytes apart, took 38 instead of 24 us for the 4514 rows.
//
// A wavefront takes the head rows - queries, then keys, then values - of one row of the call, 64 / L at a time and U times.  A
// lane holds 2 V channels of one: V that are rotated and their V partners, so that no other lane is needed, or 2 V that are not.  The
// angles are the same for all heads: each is worked out by one lane and read by the others from LDS.
template <typename T, int V, int U>
__global__ __launch_bounds__(kBlock) void k_kv_append(KvCache c, KvRows r, KvAppend a, int l_sh, int pieces) {
  __shared__ __attribute__((aligned(16))) float turn[kBlock / 64][2][128];   // cosines, sines
  __shared__ __attribute__((aligned(16))) float gains[2][2][256];            // of queries and keys: gains, biases
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), L = 1 << l_sh;
  const unsigned item = blockIdx.x * (kBlock / 64) + wave;
  const int row = (int)(item / (unsigned)pieces), piece = (int)(item - (unsigned)row * (unsigned)pieces);
  const bool norms = a.q_g || a.k_g;
  if (row >= r.n_rows && !norms) return;

  const int j = lane & (L - 1), half = a.rot >> 1, heads = a.H + 2 * c.K;
  const bool turns = V * j < half;
  // (half is a multiple of V: lanes past it hold what is not rotated, in two parts as well, so that neighbours are next to each other)
  const int ch0 = turns ? V * j : half + V * j, ch1 = ch0 + (turns ? half : (c.h - a.rot) >> 1);
  const int hr0 = (piece * U << (6 - l_sh)) + (lane >> l_sh), step = 64 >> l_sh;
  float x[U][2 * V];
  bool live[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int hr = hr0 + u * step, kv = hr - a.H;
    live[u] = row < r.n_rows && hr < heads && 2 * V * j < c.h;
    if (!live[u]) {
#pragma unroll
      for (int i = 0; i < 2 * V; ++i) x[u][i] = 0.f;
      continue;
    }
    const T* p = kv < 0 ? (const T*)a.q + ((long)row * a.q_row + (long)hr * a.q_head)
                        : (const T*)(kv < c.K ? a.k : a.v) + ((long)row * a.kv_row + (long)(kv < c.K ? kv : kv - c.K) * a.kv_head);
    load<V>(p + ch0, x[u]);
    load<V>(p + ch1, x[u] + V);
  }

  if (norms) {                                                   // (behind the rows' loads: read once a workgroup)
    for (int i = threadIdx.x; i < c.h; i += kBlock) {
      gains[0][0][i] = a.q_g ? a.q_g[i] : 0.f;
      gains[0][1][i] = a.q_b ? a.q_b[i] : 0.f;
      gains[1][0][i] = a.k_g ? a.k_g[i] : 0.f;
      gains[1][1][i] = a.k_b ? a.k_b[i] : 0.f;
    }
    __syncthreads();
    if (row >= r.n_rows) return;
  }

  // Where the row goes.
  const int s = kv8_sample_of(r, row);
  if (s < 0) return;
  const int p0 = r.pos[s];
  if (p0 < 0) return;                                            // a sample that takes no part
  const long far = (long)p0 + (r.start ? row - r.start[s] : 0);
  const int t = kv8_table_row(c, r, s);
  if (t < 0) return;
  if (far < 0 || far >= r.max_ctx) { kv8_report(c); return; }
  const int pos = (int)far, at = kv8_page_of(c, pos), page = c.tables[(long)t * c.table_stride + at];
  for (int i = lane; i < half; i += 64) {
    const double turns_of = (double)pos * a.freq[i] * 0.15915494309189533577;   // 1 / (2 pi)
    const float f = 2.f * (float)(turns_of - rint(turns_of));
    turn[wave][0][i] = cospif(f);
    turn[wave][1][i] = sinpif(f);
  }
  if ((unsigned)page >= (unsigned)c.n_pages) { kv8_report(c); return; }
  __builtin_amdgcn_wave_barrier();                               // (a wavefront's LDS accesses are made in order)
  float cs[V], sn[V];
#pragma unroll
  for (int i = 0; i < V; ++i) { cs[i] = turns ? turn[wave][0][V * j + i] : 1.f; sn[i] = turns ? turn[wave][1][V * j + i] : 0.f; }

#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int hr = hr0 + u * step, kv = hr - a.H;
    if (norms) {                                                 // (all lanes: the sums go over neighbours)
      float mean = 0.f, sum = 0.f;
      if (!a.rms) {
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) mean += x[u][i];
        mean = group_sum(mean, L) / c.h;
      }
#pragma unroll
      for (int i = 0; i < 2 * V; ++i) { const float d = x[u][i] - mean; sum = live[u] ? fmaf(d, d, sum) : 0.f; }
      const float by = 1.f / sqrtf(group_sum(sum, L) / c.h + a.eps);
      if (live[u] && (kv < 0 ? a.q_g != nullptr : kv < c.K && a.k_g)) {
        const float* const g = gains[kv < 0 ? 0 : 1][0];
#pragma unroll
        for (int i = 0; i < 2 * V; i += 4) {
          const int ch = i < V ? ch0 + i : ch1 + i - V;
          const float4 gain = *reinterpret_cast<const float4*>(g + ch), bias = *reinterpret_cast<const float4*>(g + 256 + ch);
          x[u][i] = fmaf((x[u][i] - mean) * by, gain.x, bias.x);
          x[u][i + 1] = fmaf((x[u][i + 1] - mean) * by, gain.y, bias.y);
          x[u][i + 2] = fmaf((x[u][i + 2] - mean) * by, gain.z, bias.z);
          x[u][i + 3] = fmaf((x[u][i + 3] - mean) * by, gain.w, bias.w);
        }
      }
    }
    if (!live[u]) continue;
    if (kv < c.K && turns)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float lo = x[u][i], hi = x[u][V + i];
        x[u][i] = lo * cs[i] - hi * sn[i];
        x[u][V + i] = hi * cs[i] + lo * sn[i];
      }
    T* to;
    if (kv < 0) to = (T*)a.q_out + ((long)row * a.out_row + (long)hr * c.h);
    else to = (T*)c.data + (kv8_row(c, page, kv < c.K ? kv : kv - c.K, pos) + (kv < c.K ? 0 : c.pt)) * c.h;
    store<V>(to + ch0, x[u]);
    store<V>(to + ch1, x[u] + V);
  }
}

template <typename T, int V, int U>
void launch_units(hipStream_t s, const KvCache& c, const KvRows& r, const KvAppend& a, int l_sh) {
  const int per = U * (64 >> l_sh), pieces = (a.H + 2 * c.K + per - 1) / per;
  const dim3 grid((unsigned)(((long)r.n_rows * pieces + kBlock / 64 - 1) / (kBlock / 64)));
  hipLaunchKernelGGL((k_kv_append<T, V, U>), grid, dim3(kBlock), 0, s, c, r, a, l_sh, pieces);
}
// Units of a wavefront: of 4, 3 and 2 the one that leaves the fewest of them without a head, of equals the larger.  (4 for all: 4514 rows
// of 40 fp32 heads of 64 25.6 instead of 24.4 us, 8192 rows of 48 heads of 128 with norms 53.8 instead of 52.)
template <typename T, int V>
void launch(hipStream_t s, const KvCache& c, const KvRows& r, const KvAppend& a) {
  int l_sh = 0;
  while ((2 * V << l_sh) < c.h) ++l_sh;
  const int need = (a.H + 2 * c.K + (64 >> l_sh) - 1) >> (6 - l_sh);       // units of a row
  auto idle = [&](int u) { return (need + u - 1) / u * u - need; };
  if (idle(4) <= idle(3) && idle(4) <= idle(2)) launch_units<T, V, 4>(s, c, r, a, l_sh);
  else if (idle(3) <= idle(2)) launch_units<T, V, 3>(s, c, r, a, l_sh);
  else launch_units<T, V, 2>(s, c, r, a, l_sh);
}

}  // namespace

void launch_kv_append(hipStream_t s, const KvCache& c, const KvRows& r, const KvAppend& a) {
  const bool eight = c.h % 16 == 0 && a.rot % 16 == 0;           // 16 bytes a load: sixteen channels a lane, of fp32 eight; else 8 bytes
  if (c.dtype == MDI_BF16) { if (eight) launch<bf16_t, 8>(s, c, r, a); else launch<bf16_t, 4>(s, c, r, a); }
  else launch<float, 4>(s, c, r, a);
}

}  // namespace mdi
