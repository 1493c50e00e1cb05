// Rows of experts whose offsets lie on the device, cut into chunks: every block finds its tiles by itself.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "sq_internal.h"

namespace sq {

// Exclusive scan of v over the block's threads; `warp_sums`: 33 ints.  Returns the sum before this thread; total in warp_sums[32].
__device__ __forceinline__ int block_scan(int v, int* warp_sums) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xFFFFFFFFu, s, o);
    if (lane >= o) s += u;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = s;
  __syncthreads();
  if (warp == 0) {
    const int nw = blockDim.x >> 5;
    int w = lane < nw ? warp_sums[lane] : 0;
    const int own = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xFFFFFFFFu, w, o);
      if (lane >= o) w += u;
    }
    if (lane == 31) warp_sums[32] = w;
    warp_sums[lane] = w - own;
  }
  __syncthreads();
  return warp_sums[warp] + s - v;
}

// Rows [lo, hi) of expert e, within [0, M).
__device__ __forceinline__ void expert_rows(const GsArgs& a, int e, long long& lo, long long& hi) {
  const long long M = a.M, b = a.offsets[e], d = a.offsets[e + 1];
  lo = b < 0 ? 0 : (b < M ? b : M);
  hi = d < lo ? lo : (d < M ? d : M);
}

// The experts' rows cut into chunks of `rows` each: first[e] = chunks of the experts before e, first[E] = all.  All threads.
__device__ __forceinline__ void expert_chunks(const GsArgs& a, int rows, int* first) {
  __shared__ int sums[33];
  int carry = 0;
  for (int e0 = 0; e0 < a.E; e0 += static_cast<int>(blockDim.x)) {
    const int e = e0 + static_cast<int>(threadIdx.x);
    int c = 0;
    if (e < a.E) {
      long long lo, hi;
      expert_rows(a, e, lo, hi);
      c = static_cast<int>((hi - lo + rows - 1) / rows);
    }
    const int off = carry + block_scan(c, sums);
    if (e < a.E) first[e] = off;
    carry += sums[32];
    __syncthreads();
  }
  if (threadIdx.x == 0) first[a.E] = carry;
  __syncthreads();
}
// The expert of a chunk: the last e with first[e] <= chunk (an expert without chunks has the same first as the next).
__device__ __forceinline__ int chunk_expert(const int* first, int E, int chunk) {
  int lo = 0, hi = E;
  while (lo + 1 < hi) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= chunk) lo = mid;
    else hi = mid;
  }
  return lo;
}

}  // namespace sq
