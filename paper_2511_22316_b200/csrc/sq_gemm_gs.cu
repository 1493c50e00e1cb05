// Weight-only products with group scales:
//   w[c, k] = code[c, k] * sg[k / group, c] + bg[k / group, c],   Y[r, c] = fp16(sum_k Z16[token(r), k] * w_e(r)[c, k])
// for one matrix of weights (dense) or for the experts of a sparse block, whose rows the router sorted on the device.
#include <cuda_fp16.h>

#include <algorithm>

#include "sq_internal.h"
#include "sq_ptx.cuh"

namespace sq {
namespace {

// First index i in offsets[0 .. E] (clamped to [0, M]) with offsets[i] > r, minus one: the expert of row r, or -1 / E outside.
__device__ __forceinline__ int expert_of_row(const int32_t* __restrict__ offsets, int E, long long r) {
  int lo = 0, hi = E + 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (offsets[mid] > r) hi = mid;
    else lo = mid + 1;
  }
  return lo - 1;
}

// Any shape with K % 8 == 0: a thread per channel and row, fp32 throughout, weights in the order of the channels.
__global__ void __launch_bounds__(128)
gs_simple_kernel(const GsArgs a) {
  griddep_launch_dependents();
  griddep_wait();
  const long long c = blockIdx.x * 128ll + threadIdx.x;
  if (c >= a.N) return;
  const long long G = (a.K + a.group - 1) / a.group;
  for (long long r = blockIdx.y; r < a.M; r += gridDim.y) {
    const int e = a.E > 0 ? expert_of_row(a.offsets, a.E, r) : 0;
    if (a.E > 0 && (e < 0 || e >= a.E)) continue;
    const long long tok = a.row_token ? a.row_token[r] : r;
    float acc = 0.0f;
    if (tok >= 0 && tok < a.T) {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(a.Wq + (static_cast<size_t>(e) * a.N + c) * (a.K / 2));
      const __half* z = a.Z + static_cast<size_t>(tok) * a.K;
      for (int g = 0; g < a.K / 8; ++g) {
        const size_t gi = (static_cast<size_t>(e) * G + (8 * g) / a.group) * a.N + c;
        const float s = __half2float(a.sg[gi]), b = a.bg ? __half2float(a.bg[gi]) : 0.0f;
        const uint32_t word = w[g];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c0 = (static_cast<int>(word << (28 - 4 * i))) >> 28;          // nibble position i: channel 2i
          const int c1 = (static_cast<int>(word << (12 - 4 * i))) >> 28;          // position i + 4: channel 2i + 1
          acc = fmaf(__half2float(z[8 * g + 2 * i]), fmaf(static_cast<float>(c0), s, b), acc);
          acc = fmaf(__half2float(z[8 * g + 2 * i + 1]), fmaf(static_cast<float>(c1), s, b), acc);
        }
      }
    }
    a.Y[static_cast<size_t>(r) * a.N + c] = __float2half_rn(acc);
  }
}

// Rows of fp16 or fp32 values -> codes in the weight-only order, scales and offsets per group.  A thread takes a word of eight
// channels, group / 8 neighbouring lanes a group; rows are padded to whole groups, so that every lane of a group is here.
template <typename V>
__global__ void __launch_bounds__(256)
quant_groups_kernel(const V* __restrict__ X, long long rows, long long row0, long long N, int K, int group, int bits,
                    uint32_t* __restrict__ Wq, __half* __restrict__ sg, __half* __restrict__ bg) {
  const int lpg = group / 8, words = K / 8, padded = (words + lpg - 1) / lpg * lpg;
  const int cmin = -(1 << (bits - 1)), cmax = -cmin - 1;
  const long long total = rows * padded, stride = static_cast<long long>(gridDim.x) * blockDim.x;
  const long long rounds = (total + stride - 1) / stride;
  for (long long it = 0; it < rounds; ++it) {
    const long long i = it * stride + blockIdx.x * static_cast<long long>(blockDim.x) + threadIdx.x;
    const long long row = i / padded;
    const int w = static_cast<int>(i - row * padded);
    const bool in = i < total && w < words;
    float x[8], lo = __int_as_float(0x7F800000), hi = -lo;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = in ? static_cast<float>(X[static_cast<size_t>(row) * K + 8 * w + j]) : 0.0f;
      if (in) {
        lo = fminf(lo, x[j]);
        hi = fmaxf(hi, x[j]);
      }
    }
    for (int o = lpg / 2; o > 0; o >>= 1) {
      lo = fminf(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, o));
      hi = fmaxf(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, o));
    }
    if (!in) continue;
    __half step, off = __ushort_as_half(0);
    if (bg != nullptr) {
      step = __float2half_rn(__fdiv_rn(__fsub_rn(hi, lo), static_cast<float>(cmax - cmin)));
      off = __float2half_rn(__fsub_rn(lo, __fmul_rn(static_cast<float>(cmin), __half2float(step))));
    } else {
      step = __float2half_rn(__fdiv_rn(fmaxf(fabsf(lo), fabsf(hi)), static_cast<float>(cmax)));
    }
    const float d = __half2float(step), b = __half2float(off);
    const float inv = d > 0.0f ? __fdiv_rn(1.0f, d) : 0.0f;
    uint32_t word = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float t = __fadd_rn(__fmul_rn(__fsub_rn(x[j], b), inv), 0.5f);
      const int code = max(cmin, min(cmax, static_cast<int>(floorf(t))));
      word |= static_cast<uint32_t>(code & 15) << (4 * ((j >> 1) + 4 * (j & 1)));
    }
    Wq[(row0 + row) * words + w] = word;
    if (w % lpg == 0) {
      const size_t gi = static_cast<size_t>(w / lpg) * N + row0 + row;
      sg[gi] = step;
      if (bg != nullptr) bg[gi] = off;
    }
  }
}

}  // namespace

sq_status_t launch_quant_groups(const void* X, bool f32, int64_t rows, int64_t row0, int64_t N, int K, int group, int bits, void* Wq,
                                void* sg, void* bg, cudaStream_t s) {
  const int sms = sm_count();
  if (sms <= 0) return SQ_ERR_CUDA;
  const int lpg = group / 8;
  const long long total = rows * static_cast<long long>((K / 8 + lpg - 1) / lpg * lpg);
  const unsigned grid = static_cast<unsigned>(std::min<long long>((total + 255) / 256, static_cast<long long>(sms) * 8));
  uint32_t* w = static_cast<uint32_t*>(Wq);
  __half *sh = static_cast<__half*>(sg), *bh = static_cast<__half*>(bg);
  if (f32) quant_groups_kernel<float><<<grid, 256, 0, s>>>(static_cast<const float*>(X), rows, row0, N, K, group, bits, w, sh, bh);
  else quant_groups_kernel<__half><<<grid, 256, 0, s>>>(static_cast<const __half*>(X), rows, row0, N, K, group, bits, w, sh, bh);
  count_launch();
  return cudaGetLastError() == cudaSuccess ? SQ_OK : SQ_ERR_CUDA;
}

sq_status_t launch_gemm_gs(const GsArgs& a, void* workspace, cudaStream_t s) {
  (void)workspace;
  const dim3 grid(static_cast<unsigned>((a.N + 127) / 128), static_cast<unsigned>(std::min<long long>(a.M, 65535)));
  const cudaError_t err = launch_maybe_pdl(gs_simple_kernel, grid, dim3(128), 0, s, a);
  count_launch();
  return err == cudaSuccess ? SQ_OK : SQ_ERR_CUDA;
}

}  // namespace sq
