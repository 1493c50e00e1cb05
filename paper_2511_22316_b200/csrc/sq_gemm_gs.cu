// Weight-only products with group scales:
//   w[c, k] = code[c, k] * sg[k / group, c] + bg[k / group, c],   Y[r, c] = fp16(sum_k Z16[token(r), k] * w_e(r)[c, k])
// for one matrix of weights (dense) or for the experts of a sparse block, whose rows the router sorted on the device.
#include <cuda_fp16.h>

#include <algorithm>

#include "sq_internal.h"
#include "sq_groups.cuh"
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

// ---------------------------------------------------------------------------------------------
// Few tokens: a stream of weights through warp-level MMAs
// ---------------------------------------------------------------------------------------------
// Up to 8 or 16 rows at a time (NT = 1, 2): what counts is the weights' trip through the chip.  A tile is up to 16 RB output
// channels; the eight warps of a block split K, in steps of 128 channels dealt out in turn.  Two blocks share an SM, so that one
// streams while the other adds up, and so that the next kernel's first weights are on their way before this one ends.
//
// Every thread copies from global memory what it alone will read: lane 4 g + t takes the 16-byte piece t of the rows 2 g and 2 g + 1
// of a block of 16 (an MMA's rows g and g + 8, in whatever order of k as long as weights and tokens agree), and the fp16 pair of
// their scales.  So a warp's ring needs no barrier, only the thread's own wait for its copies, and it runs on from tile to tile.
// The tokens come straight from L2 into the MMA's layout, a step ahead: each warp needs another part of K, nothing is shared.
//
// The weight is code * scale + offset in one fp16 fused multiply-add (one rounding, 2^-11 of the weight); sums are fp32.  With
// steps of one group (128) the scale could follow the MMAs in fp32, but not with 32 or 64, whose pieces meet in one MMA.
constexpr int GS_WARPS = 8, GS_THREADS = GS_WARPS * 32;

template <int RB, int NT, bool BIAS>
struct GsStream {
  static constexpr int SLOT = 1024 + (BIAS ? 256 : 128);      // 16 channels x 128 codes, their scales (and offsets), per lane
  static constexpr int DEPTH = RB == 1 ? 8 : (RB == 2 ? 4 : (RB == 3 ? 3 : 2));
  static constexpr int RING = DEPTH * RB * SLOT;              // of a warp
  static constexpr int PITCH = 16 * RB + 8;                   // of the sums: 2 pitch = 16 banks
  static constexpr int PART = 8 * NT * PITCH;                 // floats of one warp's sums
  static constexpr int BYTES = GS_WARPS * (RING + 4 * PART);
  static_assert(BYTES <= 112 * 1024, "two blocks to an SM");
};

__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src, bool take) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(take ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ uint4 lds128_at(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}

template <int RB, int NT, bool BIAS, bool EXPERTS>
__global__ void __launch_bounds__(GS_THREADS, 2)
gs_stream_kernel(const __grid_constant__ GsArgs a, int R, int splits) {
  using L = GsStream<RB, NT, BIAS>;
  griddep_launch_dependents();
  extern __shared__ __align__(16) unsigned char gs_smem[];
  __shared__ int first[EXPERTS ? 1025 : 1];
  float* part = reinterpret_cast<float*>(gs_smem + GS_WARPS * L::RING);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int K = a.K, N = static_cast<int>(a.N), group = a.group;
  const int G = (K + group - 1) / group;
  const int crank = splits > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int cid = static_cast<int>(blockIdx.x) / splits, ncl = static_cast<int>(gridDim.x) / splits;
  const int nks = (K + 127) / 128;
  const int ks0 = crank * nks / splits + warp, ks1 = (crank + 1) * nks / splits;
  const int cw = ks1 > ks0 ? (ks1 - ks0 + GS_WARPS - 1) / GS_WARPS : 0;      // this warp's steps of a tile
  const int ctiles = (N + R - 1) / R;
  int tiles = ctiles;
  if constexpr (EXPERTS) {
    griddep_wait();                                  // the offsets come from the router
    expert_chunks(a, 8 * NT, first);
    tiles = first[a.E] * ctiles;
  }
  const int my_tiles = cid < tiles ? (tiles - cid + ncl - 1) / ncl : 0;
  const int total = my_tiles * cw;
  const uint32_t ring = smem_u32(gs_smem) + warp * L::RING + lane * 16;
  const uint32_t ring_s = smem_u32(gs_smem) + warp * L::RING + 1024 + lane * 4;

  // Cursor of the copies: step `iq` of the sequence, its tile's weights.
  int iq = 0, iks = ks0, itile = cid, islot = 0;
  const uint8_t* iw = nullptr;
  const __half *is = nullptr, *ib = nullptr;
  int irows = 0;
  auto aim = [&]() {
    const int chunk = EXPERTS ? itile / ctiles : 0;
    const int e = EXPERTS ? chunk_expert(first, a.E, chunk) : 0;
    const int row0 = (itile - chunk * ctiles) * R;
    irows = min(R, N - row0);
    iw = a.Wq + (static_cast<size_t>(e) * N + row0 + 2 * g) * (K / 2) + 16 * t;
    is = a.sg + static_cast<size_t>(e) * G * N + row0;
    if (BIAS) ib = a.bg + static_cast<size_t>(e) * G * N + row0;
  };
  auto issue = [&]() {
    if (iq < total) {
      if (iks == ks0) aim();
      const int k = iks * 128 + 32 * t;
      const size_t gi = static_cast<size_t>(min(k, K - 1) / group) * N;
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        const int r = 16 * b + 2 * g;
        const bool ok = r < irows && k < K;
        const uint8_t* w = ok ? iw + static_cast<size_t>(16 * b) * (K / 2) + iks * 64 : a.Wq;
        const uint32_t d = (islot * RB + b) * L::SLOT;
        cp_async_16(ring + d, w, ok);
        cp_async_16(ring + d + 512, ok ? w + K / 2 : a.Wq, ok);
        const size_t si = gi + min(r, irows - 2);
        cp_async_4(ring_s + d, is + si);
        if (BIAS) cp_async_4(ring_s + d + 128, ib + si);
      }
      iks += GS_WARPS;
      if (iks >= ks1) {
        iks = ks0;
        itile += ncl;
      }
      ++iq;
      if (++islot == L::DEPTH) islot = 0;
    }
    cp_async_commit();
  };
#pragma unroll
  for (int d = 0; d < L::DEPTH; ++d) issue();
  if constexpr (!EXPERTS) griddep_wait();            // Z16 may come from the kernel before, which may still read Y

  // Cursor of the tokens, a step ahead of the products.
  int xq = 0, xks = ks0, xtile = cid;
  const __half* xrow[NT];
  uint4 xn[NT][4];
  auto fetch = [&]() {
    if (xq < total) {
      if (xks == ks0 && (EXPERTS || xq == 0)) {
        long long lo = 0, hi = a.M;
        if constexpr (EXPERTS) {
          const int chunk = xtile / ctiles, e = chunk_expert(first, a.E, chunk);
          expert_rows(a, e, lo, hi);
          lo += static_cast<long long>(chunk - first[e]) * (8 * NT);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const long long r = lo + 8 * n + g;
          long long tok = -1;
          if (r < hi) tok = EXPERTS && a.row_token != nullptr ? a.row_token[r] : r;
          xrow[n] = tok >= 0 && tok < a.T ? a.Z + static_cast<size_t>(tok) * K + 32 * t : nullptr;
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          xn[n][i] = xrow[n] != nullptr && xks * 128 + 32 * t < K ? __ldg(reinterpret_cast<const uint4*>(xrow[n] + xks * 128) + i)
                                                                  : make_uint4(0u, 0u, 0u, 0u);
      xks += GS_WARPS;
      if (xks >= ks1) {
        xks = ks0;
        xtile += ncl;
      }
      ++xq;
    }
  };
  fetch();

  const WidenConsts wk = widen_consts();
  int slot = 0;
  for (int tl = 0, tile = cid; tl < my_tiles; ++tl, tile += ncl) {
    float acc[RB][NT][4];
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[b][n][e] = 0.0f;
    for (int i = 0; i < cw; ++i) {
      uint4 x[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) x[n][j] = xn[n][j];
      fetch();
      cp_async_wait<L::DEPTH - 1>();
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        const uint32_t d = (slot * RB + b) * L::SLOT;
        const uint4 u = lds128_at(ring + d), v = lds128_at(ring + d + 512);
        const uint32_t sw = lds32(ring_s + d), bw = BIAS ? lds32(ring_s + d + 128) : 0u;
        const __half2 sh = *reinterpret_cast<const __half2*>(&sw), bh = *reinterpret_cast<const __half2*>(&bw);
        const __half2 s0 = __low2half2(sh), s1 = __high2half2(sh), b0 = __low2half2(bh), b1 = __high2half2(bh);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint4 p = scaled_word<BIAS>(word_of(u, j), wk, s0, b0), q = scaled_word<BIAS>(word_of(v, j), wk, s1, b1);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            mma_f16(acc[b][n], p.x, q.x, p.y, q.y, x[n][j].x, x[n][j].y);
            mma_f16(acc[b][n], p.z, q.z, p.w, q.w, x[n][j].z, x[n][j].w);
          }
        }
      }
      if (++slot == L::DEPTH) slot = 0;
      issue();
    }
    // The warps' sums over K, added up in a fixed order.
    float* mine = part + warp * L::PART;
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        *reinterpret_cast<float2*>(mine + (8 * n + 2 * t) * L::PITCH + 16 * b + 2 * g) = make_float2(acc[b][n][0], acc[b][n][2]);
        *reinterpret_cast<float2*>(mine + (8 * n + 2 * t + 1) * L::PITCH + 16 * b + 2 * g) = make_float2(acc[b][n][1], acc[b][n][3]);
      }
    __syncthreads();
    const int chunk = EXPERTS ? tile / ctiles : 0;
    long long r0 = 0, r1 = a.M;
    if constexpr (EXPERTS) {
      const int e = chunk_expert(first, a.E, chunk);
      expert_rows(a, e, r0, r1);
      r0 += static_cast<long long>(chunk - first[e]) * (8 * NT);
    }
    const int row0 = (tile - chunk * ctiles) * R, rows = min(R, N - row0);
    for (int o = threadIdx.x; o < 64 * RB * NT; o += GS_THREADS) {
      const int tok = o / (8 * RB), c = 2 * (o % (8 * RB));
      float* p = part + tok * L::PITCH + c;
      float2 v = make_float2(0.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < GS_WARPS; ++w) {
        const float2 u = *reinterpret_cast<const float2*>(p + w * L::PART);
        v.x += u.x;
        v.y += u.y;
      }
      if (splits > 1) *reinterpret_cast<float2*>(p) = v;       // the first warp's place: this thread alone reads it here
      else if (c < rows && r0 + tok < r1)
        *reinterpret_cast<__half2*>(a.Y + static_cast<size_t>(r0 + tok) * N + row0 + c) = __floats2half2_rn(v.x, v.y);
    }
    if (splits > 1) {
      // One tile per cluster then.  Block r of it finishes every splits-th pair of channels.
      __syncwarp();
      cluster_sync_all();
      for (int o = threadIdx.x; o < 64 * RB * NT; o += GS_THREADS) {
        const int tok = o / (8 * RB), c = 2 * (o % (8 * RB));
        if ((c >> 1) % splits != crank || c >= rows || tok >= a.M) continue;
        const float* p = part + tok * L::PITCH + c;
        float2 v = make_float2(0.0f, 0.0f);
        for (int r = 0; r < splits; ++r) {
          float2 u;
          asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(u.x), "=f"(u.y)
                       : "r"(cluster_map(p, static_cast<uint32_t>(r))) : "memory");
          v.x += u.x;
          v.y += u.y;
        }
        *reinterpret_cast<__half2*>(a.Y + static_cast<size_t>(tok) * N + row0 + c) = __floats2half2_rn(v.x, v.y);
      }
      __syncwarp();
      cluster_sync_all();                            // the others have read this block's sums
    } else if (tl + 1 < my_tiles) {
      __syncthreads();                               // the sums have been read
    }
  }
  cp_async_wait<0>();
}

// out[r] = Z[row_token[r]], zeros for a token that does not exist; rows of no expert are not needed.
__global__ void __launch_bounds__(256)
gs_gather_kernel(const __grid_constant__ GsArgs a, uint4* __restrict__ out) {
  griddep_launch_dependents();
  griddep_wait();
  const int per_row = a.K / 8;
  const long long rows = max(0ll, min(static_cast<long long>(a.offsets[a.E]), static_cast<long long>(a.M)));
  const uint4* Z = reinterpret_cast<const uint4*>(a.Z);
  for (long long i = blockIdx.x * 256ll + threadIdx.x; i < rows * per_row; i += gridDim.x * 256ll) {
    const long long r = i / per_row, tok = a.row_token[r];
    out[i] = tok >= 0 && tok < a.T ? __ldg(Z + tok * per_row + (i - r * per_row)) : make_uint4(0u, 0u, 0u, 0u);
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

namespace {

template <int RB, int NT, bool BIAS, bool EXPERTS>
sq_status_t launch_stream_as(const GsArgs& a, int R, int splits, int grid, cudaStream_t s) {
  using L = GsStream<RB, NT, BIAS>;
  auto kern = gs_stream_kernel<RB, NT, BIAS, EXPERTS>;
  if (!ensure_dyn_smem(reinterpret_cast<const void*>(kern), L::BYTES)) return SQ_ERR_CUDA;
  const cudaError_t err = launch_cluster_maybe_pdl(kern, dim3(static_cast<unsigned>(grid)), dim3(GS_THREADS), static_cast<size_t>(L::BYTES),
                                                   s, static_cast<unsigned>(splits), a, R, splits);
  count_launch();
  return err == cudaSuccess ? SQ_OK : SQ_ERR_CUDA;
}
template <int NT, bool BIAS, bool EXPERTS>
sq_status_t launch_stream_rows(const GsArgs& a, int R, int splits, int grid, cudaStream_t s) {
  if (R <= 16) return launch_stream_as<1, NT, BIAS, EXPERTS>(a, R, splits, grid, s);
  if (R <= 32) return launch_stream_as<2, NT, BIAS, EXPERTS>(a, R, splits, grid, s);
  if constexpr (NT == 1) {
    if (R <= 48) return launch_stream_as<3, NT, BIAS, EXPERTS>(a, R, splits, grid, s);
    return launch_stream_as<4, NT, BIAS, EXPERTS>(a, R, splits, grid, s);
  }
  return SQ_ERR_UNSUPPORTED;
}
template <bool EXPERTS>
sq_status_t launch_stream_any(const GsArgs& a, int nt, int R, int splits, int grid, cudaStream_t s) {
  if (nt == 1) return a.bg ? launch_stream_rows<1, true, EXPERTS>(a, R, splits, grid, s) : launch_stream_rows<1, false, EXPERTS>(a, R, splits, grid, s);
  return a.bg ? launch_stream_rows<2, true, EXPERTS>(a, R, splits, grid, s) : launch_stream_rows<2, false, EXPERTS>(a, R, splits, grid, s);
}

int even_rows(int64_t N, int64_t tiles) { return static_cast<int>(std::max<int64_t>(2, (N + 2 * tiles - 1) / (2 * tiles) * 2)); }

sq_status_t launch_stream(const GsArgs& a, cudaStream_t s) {
  const int sms = sm_count();
  if (sms <= 0) return SQ_ERR_CUDA;
  const int slots = 2 * sms, nks = (a.K + 127) / 128;
  if (a.E > 0) {
    // Chunks of rows: one for each expert that has any, and a few more; the tiles are dealt out to all blocks.
    const int nt = a.M > 8 * static_cast<int64_t>(a.E) && a.T > 8 ? 2 : 1;
    const int64_t chunks = std::min<int64_t>(a.E, a.M);
    const int cap = nt == 1 ? 64 : 32;
    const int R = std::min<int>(cap, std::max<int>(16, even_rows(a.N, std::max<int64_t>(1, slots / chunks))));
    return launch_stream_any<true>(a, nt, R, 1, slots, s);
  }
  const int nt = a.M <= 8 ? 1 : 2, cap = nt == 1 ? 64 : 32;
  // A block's bytes, weights and tokens, with K in 1, 2, 4 or 8 parts.
  int best_r = 0, best_s = 1, best_grid = 0;
  double best = 0.0;
  for (int sp = 1; sp <= 8 && nks / sp >= (sp == 1 ? 1 : 4); sp *= 2) {
    const int R = std::min(cap, even_rows(a.N, slots / sp));
    const int64_t tiles = (a.N + R - 1) / R;
    if (sp > 1 && tiles * sp > slots) continue;
    const int64_t waves = (tiles * sp + slots - 1) / slots;
    const double cost = static_cast<double>(waves) * ((nks + sp - 1) / sp) * (R * 64.0 + a.M * 256.0) + (sp > 1 ? 20000.0 : 0.0);
    if (best_r == 0 || cost < best) {
      best = cost;
      best_r = R;
      best_s = sp;
      best_grid = static_cast<int>(std::min<int64_t>(tiles * sp, slots));
    }
  }
  return launch_stream_any<false>(a, nt, best_r, best_s, best_grid, s);
}

// Rows of a token tile of the CTA-pair kernel for experts (a multiple of 32 up to 256), as for a dense product: waves of tiles,
// each of a time of about width + 70, with every expert's last tile half full.
int gs_tile_m(const GsArgs& a) {
  const int pairs = std::max(1, sm_count() / 2);
  const double ch_tiles = static_cast<double>((a.N + 255) / 256), experts = static_cast<double>(std::min<int64_t>(a.E, a.M));
  int best = 256;
  double best_cost = 0.0;
  for (int w = 256; w >= 32; w -= 32) {
    const double load = ch_tiles * (experts * (a.M / experts / w + 0.5)) / pairs;
    const double cost = std::max(1.0, load) * (w + 70);
    if (w == 256 || cost < best_cost) {
      best = w;
      best_cost = cost;
    }
  }
  return best;
}

}  // namespace

sq_status_t launch_gemm_gs(const GsArgs& a, void* workspace, cudaStream_t s) {
  const bool few = a.E > 0 ? a.M <= 16 * static_cast<int64_t>(a.E) : a.M <= 16;
  if (a.K % 32 == 0 && a.N % 2 == 0 && few) return launch_stream(a, s);
  // (32-bit coordinates of a tile in the weights and in the rows)
  const int64_t kMax = (1ll << 31) - 1024;
  if (a.K % 32 == 0 && a.M <= kMax && a.N * std::max(a.E, 1) <= kMax) {
    if (a.E == 0) return launch_wo_gemm_groups(a, 0, s);
    GsArgs b = a;
    if (a.row_token) {
      // The rows in their order, so that a tile of them is one TMA box.
      const int64_t pieces = a.M * (a.K / 8);
      const unsigned grid = static_cast<unsigned>(std::min<int64_t>((pieces + 255) / 256, static_cast<int64_t>(std::max(sm_count(), 1)) * 8));
      const cudaError_t err = launch_maybe_pdl(gs_gather_kernel, dim3(grid), dim3(256), 0, s, a, static_cast<uint4*>(workspace));
      count_launch();
      if (err != cudaSuccess) return SQ_ERR_CUDA;
      b.Z = static_cast<const __half*>(workspace);
      b.row_token = nullptr;
      b.T = a.M;
    }
    return launch_wo_gemm_groups(b, gs_tile_m(a), s);
  }
  const dim3 grid(static_cast<unsigned>((a.N + 127) / 128), static_cast<unsigned>(std::min<long long>(a.M, 65535)));
  const cudaError_t err = launch_maybe_pdl(gs_simple_kernel, grid, dim3(128), 0, s, a);
  count_launch();
  return err == cudaSuccess ? SQ_OK : SQ_ERR_CUDA;
}

}  // namespace sq
