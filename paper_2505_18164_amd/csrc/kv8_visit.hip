// What a pass of a partition with an 8-bit cache needs on the device before its layers run, and the hand-off of its rows afterwards.
#include "device_utils.h"
#include "kv8_internal.h"

namespace mdi {
namespace {

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
  int s = 0;
  while (s + 1 < a.n && a.first[s + 1] <= row) ++s;
  const int pos = a.pos[s] + row - a.first[s];
  if (threadIdx.x == 0) a.row_pos[row] = pos;
  if (a.rope_rows)
    for (int e = threadIdx.x; e < a.half; e += kBlock) a.rope_rows[(long)row * a.half + e] = a.rope[(long)pos * a.half + e];
  if (a.in_rows)                                                 // (one row each; pieces of two bytes: an input may lie anywhere)
    for (int e = threadIdx.x; e < a.in_bytes / 2; e += kBlock) ((uint16_t*)a.in_rows)[(long)row * (a.in_bytes / 2) + e] = ((const uint16_t*)a.in[s])[e];
}

__global__ __launch_bounds__(kBlock) void k_kv8_handoff(Kv8Handoff a) {
  const int row = blockIdx.x;
  for (int e = threadIdx.x; e < a.bytes / 2; e += kBlock) ((uint16_t*)a.out[row])[e] = ((const uint16_t*)a.rows)[(long)row * (a.bytes / 2) + e];
}

}  // namespace

void launch_kv8_setup(hipStream_t s, const Kv8Setup& a) {
  const int rows = a.n > 1 || a.in_rows ? a.rows : 0;            // a lone sample's rows are where they are wanted
  hipLaunchKernelGGL(k_kv8_setup, dim3(rows + 1), dim3(kBlock), 0, s, a);
}
void launch_kv8_handoff(hipStream_t s, const Kv8Handoff& a) { hipLaunchKernelGGL(k_kv8_handoff, dim3(a.n), dim3(kBlock), 0, s, a); }

}  // namespace mdi
