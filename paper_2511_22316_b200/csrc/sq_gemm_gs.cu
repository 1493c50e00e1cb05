// Weight-only products with group scales:
//   w[c, k] = code[c, k] * sg[k / group, c] + bg[k / group, c],   Y[r, c] = fp16(sum_k Z16[token(r), k] * w_e(r)[c, k])
// for one matrix of weights (dense) or for the experts of a sparse block, whose rows the router sorted on the device.
#include <cuda.h>
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
// Each warp has a ring of its own in shared memory, filled by its own TMA loads (16 RB rows x 64 bytes): no barriers between warps,
// and it runs on from tile to tile.  The tokens come straight from L2 into the MMA's layout, eight rows ahead: each warp needs
// another part of K.  (With 16-byte asynchronous copies in place of TMA a step of 16 x 128 weights took 169 instructions.)
//
// The MMA multiplies the codes themselves, widened to fp16 exactly (widen_word: nine operations for eight weights); the pairs that
// the widening makes of low and of high bits go to accumulators of their own, two chains, and behind each group, in fp32,
//   sum += scale (lo + hi) + offset sum(x),
// with the group's sum of the tokens, where there are offsets, from an MMA with ones, once for all channels of the warp.  No weight is
// rounded, and a code of zero adds nothing, whatever its token.  (Masked out of its word a nibble is an fp16 subnormal, code + 8,
// that the MMA would take as it is, five operations in place of nine; but 8 sum(x) has to come off again, whose rounding showed where
// a token is large and its code zero, and the chain for sum(x) stands before all others: groups of 128, 1 x 8192 -> 28672 26.7 us and 27.2
// with the codes, 1 x 4096 -> 14336 8.8 both, 1 x 4096 -> 4096 5.6 and 4.7; 8 x 4096 -> 14336, groups of 64, 10.5 and 9.5.)  With
// each weight made fp16(code scale + offset) beforehand, 1 x 4096 -> 14336 took 10.7 us.
//
// 1 x 4096 -> 14336 in 8.8 us is 3.4 TB/s, 1 x 8192 -> 28672 in 27.2 us 4.5 TB/s (graph replays): by the two some 2.6 us of a call are its
// start and end, and the rest runs at 4.9 TB/s, 75 % of the copy rate.
//
// So that an MMA stays within a group of 32, 64 or 128, lane 4 g + t takes word t, words 2 t, 2 t + 1 or piece t (four words) of
// the group: the MMA's order of k is whatever weights and tokens agree on.
constexpr int GS_WARPS = 8, GS_THREADS = GS_WARPS * 32;

template <int RB, int NT, int GROUP>
struct GsStream {
  static constexpr int CHUNKS = 128 / GROUP;                  // groups of a step
  static constexpr int WPL = GROUP / 32;                      // words of a group that a lane takes
  static constexpr int ROWS = 16 * RB;
  static constexpr int DEPTH = RB == 1 ? 8 : (RB == 2 ? 4 : 2);
  static constexpr int W_SLOT = ROWS * 64;                    // 128 codes of each row
  static constexpr int S_SLOT = CHUNKS * ROWS * 2;            // the groups' scales, and as much for the offsets
  static constexpr int OFF_S = DEPTH * W_SLOT;
  static constexpr int RING = (OFF_S + 2 * DEPTH * S_SLOT + 511) / 512 * 512;       // of a warp (SWIZZLE_64B repeats after 512 bytes)
  static constexpr int PITCH = ROWS + 4;                      // of the sums: 8 banks from a token pair to the next
  static constexpr int PART = 8 * NT * PITCH;                 // floats of one warp's sums
  static constexpr int OFF_PART = GS_WARPS * RING;
  static constexpr int OFF_BAR = OFF_PART + GS_WARPS * 4 * PART;
  static constexpr int BYTES = OFF_BAR + GS_WARPS * DEPTH * 8 + 512;                // slack for the alignment
  static_assert(BYTES + (1025 + 33) * 4 <= 113 * 1024, "two blocks to an SM, with the experts' chunks and the scan in static memory");
};
enum GsSite : uint32_t { GS_FULL = 112 };

__device__ __forceinline__ void cp_async_4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ float lds_half(uint32_t a) {
  unsigned short v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a) : "memory");
  return __half2float(__ushort_as_half(v));
}
// D = A B: sums that begin.
__device__ __forceinline__ void mma_f16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}
template <int W>
__device__ __forceinline__ void lds_words(uint32_t a, uint32_t (&w)[W]) {
  if constexpr (W == 4) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(a) : "memory");
  else if constexpr (W == 2) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(a) : "memory");
  else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(a) : "memory");
}

__device__ const uint4 g_zero_words[4] = {};

template <int RB, int NT, int GROUP, bool BIAS, bool EXPERTS>
__global__ void __launch_bounds__(GS_THREADS, 2)
gs_stream_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ GsArgs a, int splits) {
  using L = GsStream<RB, NT, GROUP>;
  constexpr int CHUNKS = L::CHUNKS, WPL = L::WPL, R = L::ROWS;
  griddep_launch_dependents();
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 511) & ~uintptr_t(511));
  __shared__ int first[EXPERTS ? 1025 : 1];
  float* part = reinterpret_cast<float*>(smem + L::OFF_PART);

  const int warp = __shfl_sync(0xFFFFFFFFu, static_cast<int>(threadIdx.x) >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int K = a.K, N = static_cast<int>(a.N);
  const int G = (K + GROUP - 1) / GROUP;
  const int crank = splits > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int cid = static_cast<int>(blockIdx.x) / splits, ncl = static_cast<int>(gridDim.x) / splits;
  const int nks = (K + 127) / 128;
  const int ks0 = crank * nks / splits + warp, ks1 = (crank + 1) * nks / splits;
  const int cw = ks1 > ks0 ? (ks1 - ks0 + GS_WARPS - 1) / GS_WARPS : 0;      // this warp's steps of a tile
  // The step whose channels end before 128 of them, if it is this warp's: always the last of its steps.
  const bool ragged = (K & 127) != 0 && cw > 0 && ks0 + (cw - 1) * GS_WARPS == nks - 1;
  unsigned char* ring = smem + warp * L::RING;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::OFF_BAR) + warp * L::DEPTH;
  if (lane == 0) {
#pragma unroll
    for (int d = 0; d < L::DEPTH; ++d) mbar_init(&full[d], 1);
    mbar_fence_init();
  }
  __syncwarp();
  // Tiles of blocks of 16 channels.  Dense: a run of them for every thread block, as even as can be, cut into tiles of up to RB (1 x
  // 8192 -> 28672 29.2 -> 26.9 us against whole tiles dealt out in turn).  Experts: the tiles of R channels of all chunks of rows in
  // one list, dealt out in turn.
  const int nb = (N + 15) / 16, ctiles = (N + R - 1) / R;
  int my_tiles = 0, run0 = 0, run1 = 0;              // experts: how many tiles; dense: a run of blocks
  if constexpr (EXPERTS) {
    griddep_wait();                                  // the offsets come from the router
    expert_chunks(a, 8 * NT, first);
    const int tiles = first[a.E] * ctiles;           // (the launcher has seen to it that they fit 32 bits)
    my_tiles = cid < tiles ? (tiles - cid + ncl - 1) / ncl : 0;
  } else {
    run0 = static_cast<int>(static_cast<long long>(nb) * cid / ncl);
    run1 = static_cast<int>(static_cast<long long>(nb) * (cid + 1) / ncl);
    my_tiles = (run1 - run0 + RB - 1) / RB;
  }
  auto dense_size = [&](int from, int left) { return (run1 - from + left - 1) / left; };      // of the first of `left` tiles
  const uint32_t limit = wait_limit();

  // Where this lane reads its words of row g of a block, by group: 16-byte piece p of row r lies at p ^ (r >> 1 & 3).
  uint32_t take[CHUNKS];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int word = c * (GROUP / 8) + t * WPL;      // of the row's sixteen
    take[c] = smem_u32(ring) + g * 64 + (((word >> 2) ^ (g >> 1 & 3)) << 4) + (word & 3) * 4;
  }
  const uint32_t take_s = smem_u32(ring) + L::OFF_S + g * 2;

  // Cursor of the copies: the steps left of its tile, and the tile's weights and scales (of this lane's pair of channels).
  int ileft = 0, itiles = cw > 0 ? my_tiles : 0, itile = EXPERTS ? cid : run0, isize = 0, islot = 0, ix = 0, iy = 0;
  const __half *is = nullptr, *ib = nullptr;
  const size_t step_s = static_cast<size_t>(GS_WARPS * CHUNKS) * N;
  const uint32_t put_s = smem_u32(ring) + L::OFF_S + lane * 4;
  auto issue = [&]() {
    if (ileft == 0 && itiles > 0) {
      const int chunk = EXPERTS ? itile / ctiles : 0;
      const int e = EXPERTS ? chunk_expert(first, a.E, chunk) : 0;
      if (!EXPERTS) isize = dense_size(itile, itiles);
      const int row0 = EXPERTS ? (itile - chunk * ctiles) * R : 16 * itile;
      iy = e * N + row0 + (EXPERTS ? 0 : 16 * lane);           // dense: lane b < isize loads block b
      const size_t so = (static_cast<size_t>(e) * G + ks0 * CHUNKS) * N + row0 + min(2 * lane, min(EXPERTS ? R : 16 * isize, N - row0) - 2);
      is = a.sg + so;
      if (BIAS) ib = a.bg + so;
      ix = ks0 * 64;
      ileft = cw;
      itile += EXPERTS ? ncl : isize;
      --itiles;
    }
    if (ileft > 0) {
      --ileft;
      if constexpr (EXPERTS) {                       // one box of a whole tile's rows
        if (lane == 0) {
          mbar_arrive_expect_tx(&full[islot], L::W_SLOT);
          tma_load_2d(ring + islot * L::W_SLOT, &tmap_w, &full[islot], ix, iy);
        }
      } else {
        if (lane == 0) mbar_arrive_expect_tx(&full[islot], static_cast<uint32_t>(isize * 1024));
        __syncwarp();
        if (lane < isize) tma_load_2d(ring + islot * L::W_SLOT + lane * 1024, &tmap_w, &full[islot], ix, iy);
      }
      if (RB == 4 || lane < 8 * RB) {
        const uint32_t d = put_s + islot * (2 * L::S_SLOT);
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
          // A group behind the last one takes the last one's: its tokens are zeros, its scales have to be finite.
          size_t o = static_cast<size_t>(c) * N;
          if (CHUNKS > 1 && c > 0 && ragged && ileft == 0) o = static_cast<size_t>(min(c, G - 1 - (nks - 1) * CHUNKS)) * N;
          cp_async_4(d + c * (2 * L::ROWS), is + o);
          if (BIAS) cp_async_4(d + c * (2 * L::ROWS) + L::S_SLOT, ib + o);
        }
      }
      is += step_s;
      if (BIAS) ib += step_s;
      ix += GS_WARPS * 64;
      islot = islot + 1 == L::DEPTH ? 0 : islot + 1;
    }
    cp_async_commit();
  };
#pragma unroll
  for (int d = 0; d < L::DEPTH; ++d) issue();
  if constexpr (!EXPERTS) griddep_wait();            // Z16 may come from the kernel before, which may still read Y

  // Cursor of the tokens, eight rows ahead of the products.  Columns of an MMA that are no row of the tile repeat another row (its
  // sums are not stored).
  int xleft = 0, xtiles = cw > 0 ? my_tiles : 0, xtile = cid;
  bool xaimed = false;
  const __half *xrow[NT], *xat[NT];
  uint4 xn[4];
  auto fetch = [&](int n) {
    if (n == 0 && xleft == 0) {
      if (xtiles == 0) return;
      if (EXPERTS || !xaimed) {
        xaimed = true;
        long long lo = 0, hi = a.M;
        if constexpr (EXPERTS) {
          const int chunk = xtile / ctiles, e = chunk_expert(first, a.E, chunk);
          expert_rows(a, e, lo, hi);
          lo += static_cast<long long>(chunk - first[e]) * (8 * NT);
        }
#pragma unroll
        for (int m = 0; m < NT; ++m) {
          long long tok = lo + 8 * m + g;
          tok = tok < hi ? tok : hi - 1;
          if (EXPERTS && a.row_token != nullptr) tok = a.row_token[tok];
          tok = tok < 0 ? 0 : (tok < a.T ? tok : a.T - 1);       // (no such token: zeros are stored, see below)
          xrow[m] = a.Z + static_cast<size_t>(tok) * K + ks0 * 128 + 8 * WPL * t;
        }
      }
#pragma unroll
      for (int m = 0; m < NT; ++m) xat[m] = xrow[m];
      xleft = cw;
      xtile += ncl;
      --xtiles;
    }
    // Channels behind the last are read as zeros.
    const bool last = ragged && xleft == 1;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const uint4* p = reinterpret_cast<const uint4*>(xat[n] + c * GROUP);
      if (last && (nks - 1) * 128 + c * GROUP + 8 * WPL * t >= K) p = g_zero_words;
#pragma unroll
      for (int j = 0; j < WPL; ++j) xn[c * WPL + j] = __ldg(p + j);
    }
    xat[n] += GS_WARPS * 128;
    if (n == NT - 1) --xleft;
  };
  fetch(0);

  const WidenConsts wk = widen_consts();
  const uint32_t ones = 0x3C003C00u;
  int slot = 0;
  uint32_t phase = 0;
  bool ok = true;
  for (int tl = 0, tile = EXPERTS ? cid : run0; tl < my_tiles; ++tl) {
    const int chunk = EXPERTS ? tile / ctiles : 0;
    const int size = EXPERTS ? RB : dense_size(tile, my_tiles - tl);
    const int row0 = EXPERTS ? (tile - chunk * ctiles) * R : 16 * tile, rows = min(EXPERTS ? R : 16 * size, N - row0);
    tile += EXPERTS ? ncl : size;
    float acc[RB][NT][4];
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[b][n][e] = 0.0f;
    for (int i = 0; i < cw; ++i) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {                 // (16 rows: the codes are widened twice, which costs less than 32 more registers)
        // Channel pairs (0, 1) and (4, 5) of each word, then (2, 3) and (6, 7): as the MMAs take them.
        uint2 xl[4], xh[4];
        float2 sx[CHUNKS];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          xl[j] = make_uint2(xn[j].x, xn[j].z);
          xh[j] = make_uint2(xn[j].y, xn[j].w);
        }
        fetch((n + 1) % NT);
        if constexpr (BIAS) {
#pragma unroll
          for (int c = 0; c < CHUNKS; ++c) {
            float d[4];
#pragma unroll
            for (int j = 0; j < WPL; ++j) {
              const uint2 vl = xl[c * WPL + j], vh = xh[c * WPL + j];
              if (j == 0) mma_f16_first(d, ones, ones, ones, ones, vl.x, vl.y);
              else mma_f16(d, ones, ones, ones, ones, vl.x, vl.y);
              mma_f16(d, ones, ones, ones, ones, vh.x, vh.y);
            }
            sx[c] = make_float2(d[0], d[1]);
          }
        }
        if (n == 0) {
          cp_async_wait<L::DEPTH - 1>();
          // (After a time-out nothing is requested any more, and what is on its way gets a little longer.  The lanes agree on it: what
          // follows is the whole warp's.)
          ok = __all_sync(0xFFFFFFFFu, mbar_wait(&full[slot], phase, GS_FULL, ok ? limit : 65536u) && ok) != 0;
          __syncwarp();                              // the other lanes' scales
        }
        // A tile of experts has all its blocks of channels but for an expert's last (what lies behind the channels is not stored), and
        // without a way out of the loop the compiler mixes the blocks: 16 tokens on eight experts, 4096 -> 14336, groups of 128 55.7 -> 55.1
        // us (two blocks side by side: 57.4); groups of 32 71.9 -> 67.8, with offsets 86.8 -> 82.5.  The other forms run out of registers by
        // it: groups of 64 63.8 -> 65.0, 128 with offsets 67.1 -> 69.3.
        constexpr bool WHOLE = EXPERTS && (GROUP == 32 || (GROUP == 128 && !BIAS));
#pragma unroll
        for (int b = 0; b < RB; ++b) {
          if (!WHOLE && (EXPERTS ? 16 * b >= rows : RB > 1 && b >= size)) break;
          const uint32_t d = slot * L::W_SLOT + b * 1024, ds = take_s + slot * 2 * L::S_SLOT + b * 32;
#pragma unroll
          for (int c = 0; c < CHUNKS; ++c) {
            uint32_t u[WPL], v[WPL];
            lds_words<WPL>(take[c] + d, u);
            lds_words<WPL>(take[c] + d + 512, v);
            const uint32_t sa = ds + c * (2 * L::ROWS);
            const float2 s = make_float2(lds_half(sa), lds_half(sa + 16));
            float2 o = make_float2(0.0f, 0.0f);
            if (BIAS) o = make_float2(lds_half(sa + L::S_SLOT), lds_half(sa + L::S_SLOT + 16));
            float lo[4], hi[4];
#pragma unroll
            for (int j = 0; j < WPL; ++j) {
              const uint2 p = xl[c * WPL + j], q = xh[c * WPL + j];
              const uint4 uc = widen_word(u[j], wk), vc = widen_word(v[j], wk);
              if (j == 0) {
                mma_f16_first(lo, uc.x, vc.x, uc.z, vc.z, p.x, p.y);
                mma_f16_first(hi, uc.y, vc.y, uc.w, vc.w, q.x, q.y);
              } else {
                mma_f16(lo, uc.x, vc.x, uc.z, vc.z, p.x, p.y);
                mma_f16(hi, uc.y, vc.y, uc.w, vc.w, q.x, q.y);
              }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {              // e & 1: token 2 t or 2 t + 1, e >> 1: channel g or g + 8
              float& sum = acc[b][n][e];
              sum = fmaf(e < 2 ? s.x : s.y, lo[e] + hi[e], sum);
              if (BIAS) sum = fmaf(e < 2 ? o.x : o.y, (e & 1) ? sx[c].y : sx[c].x, sum);
            }
          }
        }
      }
      if (++slot == L::DEPTH) {
        slot = 0;
        phase ^= 1;
      }
      __syncwarp();                                  // every lane has read the slot
      if (ok) issue();
    }
    // The warps' sums over K, added up in a fixed order.
    float* mine = part + warp * L::PART;
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float* p = mine + (8 * n + 2 * t) * L::PITCH + 16 * b + g;
        p[0] = acc[b][n][0];
        p[L::PITCH] = acc[b][n][1];
        p[8] = acc[b][n][2];
        p[L::PITCH + 8] = acc[b][n][3];
      }
    __syncthreads();
    long long r0 = 0, r1 = a.M;
    if constexpr (EXPERTS) {
      const int e = chunk_expert(first, a.E, chunk);
      expert_rows(a, e, r0, r1);
      r0 += static_cast<long long>(chunk - first[e]) * (8 * NT);
    }
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
      else if (c < rows && r0 + tok < r1) {
        if (EXPERTS && a.row_token != nullptr) {
          const long long id = a.row_token[r0 + tok];
          if (id < 0 || id >= a.T) v = make_float2(0.0f, 0.0f);
        }
        *reinterpret_cast<__half2*>(a.Y + static_cast<size_t>(r0 + tok) * N + row0 + c) = __floats2half2_rn(v.x, v.y);
      }
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

template <int RB, int NT, int GROUP, bool BIAS, bool EXPERTS>
sq_status_t launch_stream_as(const GsArgs& a, int splits, int grid, cudaStream_t s) {
  using L = GsStream<RB, NT, GROUP>;
  auto kern = gs_stream_kernel<RB, NT, GROUP, BIAS, EXPERTS>;
  if (!ensure_dyn_smem(reinterpret_cast<const void*>(kern), L::BYTES)) return SQ_ERR_CUDA;
  EncodeTiledFn enc = get_encode_fn();
  if (!enc) return SQ_ERR_CUDA;
  CUtensorMap mw;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(a.K / 2), static_cast<cuuint64_t>(a.N * std::max(a.E, 1))};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(a.K / 2)};
  const cuuint32_t box[2] = {64, EXPERTS ? L::ROWS : 16};
  const cuuint32_t estr[2] = {1, 1};
  if (enc(&mw, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(a.Wq), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
          CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return SQ_ERR_CUDA;
  const cudaError_t err = launch_cluster_maybe_pdl(kern, dim3(static_cast<unsigned>(grid)), dim3(GS_THREADS), static_cast<size_t>(L::BYTES),
                                                   s, static_cast<unsigned>(splits), mw, a, splits);
  count_launch();
  return err == cudaSuccess ? SQ_OK : SQ_ERR_CUDA;
}
// `rb`: blocks of 16 channels that a tile has to hold (experts take eight rows at a time and the largest tiles).
template <int GROUP, bool BIAS, bool EXPERTS>
sq_status_t launch_stream_rows(const GsArgs& a, int nt, int rb, int splits, int grid, cudaStream_t s) {
  if constexpr (!EXPERTS) {
    if (rb == 1 && nt == 1) return launch_stream_as<1, 1, GROUP, BIAS, EXPERTS>(a, splits, grid, s);
    if (rb == 2 && nt == 1) return launch_stream_as<2, 1, GROUP, BIAS, EXPERTS>(a, splits, grid, s);
    if (rb == 1) return launch_stream_as<1, 2, GROUP, BIAS, EXPERTS>(a, splits, grid, s);
    if (nt == 2) return launch_stream_as<2, 2, GROUP, BIAS, EXPERTS>(a, splits, grid, s);
  }
  return launch_stream_as<4, 1, GROUP, BIAS, EXPERTS>(a, splits, grid, s);
}
template <bool EXPERTS>
sq_status_t launch_stream_any(const GsArgs& a, int nt, int rb, int splits, int grid, cudaStream_t s) {
  if (a.group == 128)
    return a.bg ? launch_stream_rows<128, true, EXPERTS>(a, nt, rb, splits, grid, s) : launch_stream_rows<128, false, EXPERTS>(a, nt, rb, splits, grid, s);
  if (a.group == 64)
    return a.bg ? launch_stream_rows<64, true, EXPERTS>(a, nt, rb, splits, grid, s) : launch_stream_rows<64, false, EXPERTS>(a, nt, rb, splits, grid, s);
  return a.bg ? launch_stream_rows<32, true, EXPERTS>(a, nt, rb, splits, grid, s) : launch_stream_rows<32, false, EXPERTS>(a, nt, rb, splits, grid, s);
}

sq_status_t launch_stream(const GsArgs& a, cudaStream_t s) {
  const int sms = sm_count();
  if (sms <= 0) return SQ_ERR_CUDA;
  const int slots = 2 * sms, nks = (a.K + 127) / 128;
  // Experts: eight rows and 64 channels make a tile (sixteen tokens on eight experts, 4096 -> 14336, with 16 / 32 / 64 channels: 120 /
  // 80 / 58 us).
  if (a.E > 0) return launch_stream_any<true>(a, 1, 4, 1, slots, s);
  const int nt = a.M <= 8 ? 1 : 2, cap = nt == 1 ? 4 : 2;
  const int64_t nb = (a.N + 15) / 16;
  // Time of a call in us, fitted to one to eight rows of five shapes, 4096 x 4096 to 8192 x 28672, with K in 1 to 8 parts (10 % off; the
  // codes were subnormals then, see above, and the times have moved by -17 to +4 % since; the choices are those of the fit): a
  // step of 128 channels costs something by itself, something for its rows and something for its blocks of 16 channels, more with
  // small groups, and a third less where an SM has one block.  K over a cluster costs 1.5 us and has to fit the chip at once: 5 x
  // 14336 -> 4096 with K in 1 / 2 / 4 parts 16.2 / 12.5 / 12.4 us, but 17.7 with 74 clusters of four.
  const double unit = a.group == 128 ? 0.36 : (a.group == 64 ? 0.45 : 0.54);
  int best_rb = 0, best_s = 1, best_grid = 0;
  double best = 0.0;
  for (int sp = 1; sp <= 8 && nks / sp >= (sp == 1 ? 1 : 8); sp *= 2) {
    const int room = sp == 1 ? slots : (sp == 2 ? slots - slots / 16 : slots - slots / 8);       // blocks that clusters find place for
    for (int half = 0; half < 2; ++half) {           // two blocks per SM, or one
      const int64_t ncl = std::min<int64_t>(nb, (half ? room / 2 : room) / sp), per = (nb + ncl - 1) / ncl;
      if (sp > 1 && per > cap) continue;             // one tile for a cluster
      const int64_t cuts = (per + cap - 1) / cap;
      const double cost = (((nks + sp - 1) / sp + GS_WARPS - 1) / GS_WARPS) * (unit * nt * per + cuts * (0.31 + 0.024 * a.M)) *
                              (ncl * sp <= sms ? 0.67 : 1.0) + (sp > 1 ? 1.5 : 0.0);
      if (best_rb == 0 || cost < best) {
        best = cost;
        best_rb = per == 1 ? 1 : (per == 2 || nt == 2 ? 2 : 4);
        best_s = sp;
        best_grid = static_cast<int>(ncl * sp);
      }
    }
  }
  return launch_stream_any<false>(a, nt, best_rb, best_s, best_grid, s);
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
  // Rows for the stream: up to 8 (an expert: on average); up to 16 of a small layer, where the other kernel starts slowly: 12 x 4096
  // -> 4096 7.5 us and 9.3, but 16 x 4096 -> 14336 19.4 and 14.9.
  const bool few = a.E > 0 ? a.M <= 8 * static_cast<int64_t>(a.E) : a.M <= 8 || (a.M <= 16 && a.N * a.K <= 30000000);
  const int64_t kMax = (1ll << 31) - 1024;           // 32-bit coordinates of a tile in the weights and in the rows
  if (a.K % 32 == 0 && a.N % 2 == 0 && few && a.N * std::max(a.E, 1) <= kMax &&
      (a.N / 16 + 1) * (a.E + a.M / 8 + 1) <= kMax)
    return launch_stream(a, s);
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
