// What a pass of a partition with an 8-bit cache needs on the device before its layers run, and the hand-off of its rows afterwards.
#include "device_utils.h"
#include "kv8_internal.h"

namespace mdi {
namespace {

// One row by a workgroup: 16 bytes a thread where both lie so, else two (a caller's rows may lie anywhere), eight of them on their way.
__device__ __forceinline__ void copy_row(void* to, const void* from, int bytes) {
  if ((((uintptr_t)to | (uintptr_t)from | (unsigned)bytes) & 15) == 0) {
    for (int e = threadIdx.x; e < bytes / 16; e += kBlock) ((uint4*)to)[e] = ((const uint4*)from)[e];
    return;
  }
  const int n = bytes / 2;
  for (int e0 = threadIdx.x; e0 < n; e0 += 8 * kBlock) {
    uint16_t x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = ((const uint16_t*)from)[min(e0 + i * kBlock, n - 1)];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (e0 + i * kBlock < n) ((uint16_t*)to)[e0 + i * kBlock] = x[i];
  }
}

// Workgroup 0 writes who has which rows; workgroup i + 1 brings row i's angles and input.
__global__ __launch_bounds__(kBlock) void k_kv8_setup(Kv8Setup a) {
  if (blockIdx.x == 0) {
    for (int i = threadIdx.x; i < a.n; i += kBlock) {
      a.start[i] = a.first[i];
      a.at[i] = a.pos[i];
      a.table[i] = a.seq[i];
      if (a.page_at[i] >= 0) a.tables[a.page_at[i]] = a.page[i];
    }
    if (threadIdx.x == 0) { a.start[a.n] = a.rows; *a.zero = 0; }
    return;
  }
  const int row = blockIdx.x - 1;
  // the row's sample: at most 64 ends, looked at together
  const int lane = threadIdx.x & 63, s = __popcll(__ballot(lane + 1 < a.n && a.first[min(lane + 1, a.n)] <= row));
  const int pos = a.pos[s] + row - a.first[s];
  if (threadIdx.x == 0) a.row_pos[row] = pos;
  if (a.rope_rows)
    for (int e = threadIdx.x; e < a.half; e += kBlock) a.rope_rows[(long)row * a.half + e] = a.rope[(long)pos * a.half + e];
  if (a.in_rows) copy_row((char*)a.in_rows + (long)row * a.in_bytes, a.in[s], a.in_bytes);   // (one row each)
}

__global__ __launch_bounds__(kBlock) void k_kv8_handoff(Kv8Handoff a) {
  copy_row(a.out[blockIdx.x], (const char*)a.rows + (long)blockIdx.x * a.bytes, a.bytes);
}

}  // namespace

void launch_kv8_setup(hipStream_t s, const Kv8Setup& a) {
  const int rows = a.n > 1 || a.in_rows ? a.rows : 0;            // a lone sample's rows are where they are wanted
  hipLaunchKernelGGL(k_kv8_setup, dim3(rows + 1), dim3(kBlock), 0, s, a);
}
void launch_kv8_handoff(hipStream_t s, const Kv8Handoff& a) { hipLaunchKernelGGL(k_kv8_handoff, dim3(a.n), dim3(kBlock), 0, s, a); }

}  // namespace mdi
