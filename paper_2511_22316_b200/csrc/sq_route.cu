// The router of a sparse block and the way back from its experts' rows to tokens.
//   route_kernel / route_finish_kernel   softmax, top-k, gates, rows sorted by expert, per-expert counts, balance loss
//   route_backward_kernel                the gradient with respect to the logits
//   combine_kernel / combine_backward_kernel
//
// With p = softmax(l): gates g_j = p of the j-th largest logit, or p_j over the sum of the selected ones; loss =
// E sum_e f_e P_e with f_e = counts_e / (k n), P_e = sum_t p_te / n.  With c_e = dloss E f_e / n:
//   dl = p (d - sum_e p_e d_e),  d_e = c_e  (+ dgates_j where e is the token's j-th expert, gates over all experts)
//   dl_{e_j} += g_j (dgates_j - sum_i g_i dgates_i)   (gates over the selected experts)
//
// Few tokens are bound by latency (16 tokens, 2 of 8 experts: 3.8 us), many by the instructions of softmax and selection (16384 tokens, 8
// of 256 experts: 26.6 us, 0.4 TB/s; their gradient 11.3 us; graph replays), the combination by memory (80 % of the copy rate).  A token
// belongs to LPT lanes of
// a warp (8, 16 or 32), EPL neighbouring experts to each of them: a row is one vector load per lane, stays in registers, and
// ties go to the lowest lane and so to the lowest index.  Every group of LPT lanes takes a contiguous run of tokens, and every
// block a run of groups: the row that a slot gets is the number of slots of the same expert before it, and that is the sum of
// counts per block, per group and within the group, with no atomics whose order could matter.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <type_traits>

#include "sq_internal.h"
#include "sq_groups.cuh"
#include "sq_ptx.cuh"

namespace sq {
namespace {

constexpr int RT_MAX_BLOCKS = 148;                   // the second kernel reads every block's counts, five to a lane
constexpr int RT_STAGED = 4096;                      // slots of a block whose expert and rank stay in shared memory
constexpr int RT_FLUSH = 64;                         // tokens whose probabilities are added up in a register before they join the sums
constexpr uint32_t RT_KEY_NINF = 0x007FFFFFu;        // route_key(-inf): not above it is not usable
constexpr float RT_NINF = -__builtin_huge_valf();

struct RouteArgs {
  const void* logits;
  int dtype;
  int E, k;
  long long T, ld;
  int renorm;
  int vec;                                           // a lane's experts may be read as whole 4, 8 or 16-byte pieces
  const uint8_t* mask;
};

__device__ __forceinline__ float bits_to_float(uint32_t h, int dtype) {
  return dtype == SQ_F16 ? __half2float(__ushort_as_half(static_cast<unsigned short>(h))) : __uint_as_float(h << 16);
}

// The EPL logits of this lane: experts lane * EPL .. + EPL - 1; -inf behind the last expert and for NaN.
template <int LPT, int EPL>
__device__ __forceinline__ void route_load(const RouteArgs& a, long long t, int sub, float (&x)[EPL]) {
  const int e0 = sub * EPL;
  const bool mine = e0 < a.E;
  if (a.dtype == SQ_F32) {
    const float* row = static_cast<const float*>(a.logits) + t * a.ld + e0;
    if (EPL % 4 == 0 && a.vec) {
#pragma unroll
      for (int i = 0; i < EPL / 4; ++i) {
        const float4 v = mine ? *reinterpret_cast<const float4*>(row + 4 * i) : make_float4(RT_NINF, RT_NINF, RT_NINF, RT_NINF);
        x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
      }
    } else if (EPL == 2 && a.vec) {
      const float2 v = mine ? *reinterpret_cast<const float2*>(row) : make_float2(RT_NINF, RT_NINF);
      x[0] = v.x; x[EPL - 1] = v.y;
    } else {
#pragma unroll
      for (int i = 0; i < EPL; ++i) x[i] = e0 + i < a.E ? row[i] : RT_NINF;
    }
  } else {
    const unsigned short* row = static_cast<const unsigned short*>(a.logits) + t * a.ld + e0;
    if (EPL % 8 == 0 && a.vec) {
#pragma unroll
      for (int i = 0; i < EPL / 8; ++i) {
        const uint4 v = mine ? *reinterpret_cast<const uint4*>(row + 8 * i) : make_uint4(0u, 0u, 0u, 0u);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[8 * i + 2 * j] = mine ? bits_to_float(w[j] & 0xFFFFu, a.dtype) : RT_NINF;
          x[8 * i + 2 * j + 1] = mine ? bits_to_float(w[j] >> 16, a.dtype) : RT_NINF;
        }
      }
    } else if (EPL == 4 && a.vec) {
      const uint2 v = mine ? *reinterpret_cast<const uint2*>(row) : make_uint2(0u, 0u);
      const uint32_t w[2] = {v.x, v.y};
#pragma unroll
      for (int j = 0; j < EPL / 2; ++j) {
        x[2 * j] = mine ? bits_to_float(w[j & 1] & 0xFFFFu, a.dtype) : RT_NINF;
        x[2 * j + 1] = mine ? bits_to_float(w[j & 1] >> 16, a.dtype) : RT_NINF;
      }
    } else if (EPL == 2 && a.vec) {
      const uint32_t v = mine ? *reinterpret_cast<const uint32_t*>(row) : 0u;
      x[0] = mine ? bits_to_float(v & 0xFFFFu, a.dtype) : RT_NINF;
      x[EPL - 1] = mine ? bits_to_float(v >> 16, a.dtype) : RT_NINF;
    } else {
#pragma unroll
      for (int i = 0; i < EPL; ++i) x[i] = e0 + i < a.E ? bits_to_float(row[i], a.dtype) : RT_NINF;
    }
  }
#pragma unroll
  for (int i = 0; i < EPL; ++i) x[i] = x[i] != x[i] ? RT_NINF : x[i];
}

// Order of the selection as unsigned integers; 0 is below every logit's.  (+ 0: -0 and 0 are equal.)
__device__ __forceinline__ uint32_t route_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}
// exp(x - m) for x <= m: 1 at x == m, infinite or not.  (__expf: 2 + 1.2 |x - m| ulp, as much as rounding x - m costs.)
__device__ __forceinline__ float route_exp(float x, float m) { return x == m ? 1.0f : __expf(x - m); }
// Logits of 16 bits and their place in one key: larger logits first, then lower places, and no two alike.
__device__ __forceinline__ uint32_t route_key16(float x, int e) { return (route_key(x) & 0xFFFFE000u) | static_cast<uint32_t>(0x1FFF - e); }

constexpr float RT_LOG2E = 1.44269504088896340736f;
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <int LPT>
__device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int o = LPT / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
  return v;
}
template <int LPT>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = LPT / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}

// p of this lane's experts, and whether the token counts (a usable logit; the mask is the caller's).  All lanes of the warp.
template <int LPT, int EPL>
__device__ __forceinline__ bool route_softmax(const float (&x)[EPL], float (&p)[EPL], float& m, float& inv) {
  m = x[0];
#pragma unroll
  for (int i = 1; i < EPL; ++i) m = fmaxf(m, x[i]);
  m = group_max<LPT>(m);
  const bool usable = m > RT_NINF;
  float s = 0.0f;
  if (__all_sync(0xFFFFFFFFu, m < -RT_NINF)) {
    const float from = usable ? m : 0.0f;            // (all -inf: zeros)
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      p[i] = exp2_fast((x[i] - from) * RT_LOG2E);
      s += p[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      p[i] = usable && x[i] > RT_NINF ? route_exp(x[i], m) : 0.0f;
      s += p[i];
    }
  }
  s = group_sum<LPT>(s);
  inv = usable ? 1.0f / s : 0.0f;
#pragma unroll
  for (int i = 0; i < EPL; ++i) p[i] *= inv;
  return usable;
}

__device__ __forceinline__ double block_sum(double v, double* sums) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  __syncthreads();
  if (lane == 0) sums[warp] = v;
  __syncthreads();
  v = 0.0;
  for (int w = 0; w < static_cast<int>(blockDim.x >> 5); ++w) v += sums[w];
  return v;
}

// The k largest of the group's logits: lane j < k gets the j-th's expert (-1: none left) and value.  All lanes of the warp.
// KEY16: the logits have 16 bits, so that one 32-bit maximum finds the logit and its expert; else the lowest of the lanes that
// hold the maximum wins, and in it the lowest place.
template <int LPT, int EPL, bool KEY16>
__device__ __forceinline__ void route_select(const float (&x)[EPL], int sub, int k, int& my_id, float& my_x) {
  uint32_t key[EPL];
#pragma unroll
  for (int i = 0; i < EPL; ++i) key[i] = KEY16 ? route_key16(x[i], sub * EPL + i) : route_key(x[i]);
  uint32_t mine = 0;
  int where = 0;
  if (KEY16 && EPL >= 4 && EPL <= 8) {
    // A lane's keys in order, largest first (odd-even transposition); the largest of the heads goes, and its lane's keys move up.
#pragma unroll
    for (int r = 0; r < EPL; ++r)
#pragma unroll
      for (int i = r & 1; i + 1 < EPL; i += 2) {
        const uint32_t hi = max(key[i], key[i + 1]), lo = min(key[i], key[i + 1]);
        key[i] = hi;
        key[i + 1] = lo;
      }
    for (int j = 0; j < k; ++j) {
      const uint32_t top = __reduce_max_sync(0xFFFFFFFFu, key[0]);
      const bool pop = key[0] == top;
#pragma unroll
      for (int i = 0; i + 1 < EPL; ++i) key[i] = pop ? key[i + 1] : key[i];
      key[EPL - 1] = pop ? 0u : key[EPL - 1];
      if (sub == j) mine = top;
    }
  } else
  for (int j = 0; j < k; ++j) {
    uint32_t best = key[0];
#pragma unroll
    for (int i = 1; i < EPL; ++i) best = max(best, key[i]);
    uint32_t top = best;
    if (LPT == 32) {
      top = __reduce_max_sync(0xFFFFFFFFu, best);
    } else {
#pragma unroll
      for (int o = LPT / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    }
    if (KEY16) {
#pragma unroll
      for (int i = 0; i < EPL; ++i) key[i] = key[i] == top ? 0u : key[i];
      if (sub == j) mine = top;
    } else {
      const uint32_t who = __ballot_sync(0xFFFFFFFFu, best == top) >> (LPT == 32 ? 0 : (threadIdx.x & 31 & ~(LPT - 1)));
      const int winner = __ffs(who & (LPT == 32 ? 0xFFFFFFFFu : (1u << (LPT & 31)) - 1u)) - 1;
      bool open = sub == winner;
      int at = 0;
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        const bool hit = open && key[i] == top;
        if (hit) { key[i] = 0; at = i; }
        open = open && !hit;
      }
      at = __shfl_sync(0xFFFFFFFFu, at, winner, LPT);
      if (sub == j) {
        mine = top;
        where = winner * EPL + at;
      }
    }
  }
  if (KEY16) {
    where = 0x1FFF - static_cast<int>(mine & 0x1FFFu);
    mine &= 0xFFFFE000u;
    const bool usable = mine > (RT_KEY_NINF & 0xFFFFE000u);
    my_id = usable ? where : -1;
  } else {
    my_id = mine > RT_KEY_NINF ? where : -1;
  }
  my_x = __uint_as_float(mine & 0x80000000u ? mine ^ 0x80000000u : ~mine & (KEY16 ? 0xFFFFE000u : 0xFFFFFFFFu));
}

// Shared memory: counters [groups][E], sums of p [groups][E], base [E], partial sums over groups [2][threads], and the block's slots
// as (expert, rank) where they fit (staged).
template <int LPT, int EPL, int THREADS, bool KEY16>
__global__ void __launch_bounds__(THREADS)
route_kernel(const RouteArgs a, long long chunk, int staged, int32_t* __restrict__ ids, float* __restrict__ gates, int32_t* pos,
             int32_t* __restrict__ hist, float* __restrict__ psum, int32_t* __restrict__ counts, int32_t* __restrict__ offsets,
             int32_t* __restrict__ row_token, float* __restrict__ loss) {
  constexpr int GROUPS = THREADS / LPT;
  griddep_launch_dependents();
  extern __shared__ __align__(16) unsigned char rt_smem[];
  const int E = a.E, k = a.k;
  int* cnt = reinterpret_cast<int*>(rt_smem);                            // [GROUPS][E]
  float* ps = reinterpret_cast<float*>(cnt + GROUPS * E);                // [GROUPS][E]
  int* base = reinterpret_cast<int*>(ps + GROUPS * E);                   // [E]
  int* part_c = base + E;                                                // [THREADS]
  float* part_p = reinterpret_cast<float*>(part_c + THREADS);            // [THREADS]
  int* slot_id = reinterpret_cast<int*>(part_p + THREADS);               // [RT_STAGED], [RT_STAGED]
  int* slot_rank = slot_id + RT_STAGED;
  __shared__ int warp_sums[33];
  __shared__ double sums[32];
  __shared__ int live_of[GROUPS];

  const int grp = threadIdx.x / LPT, sub = threadIdx.x % LPT;
  for (int i = threadIdx.x; i < GROUPS * E; i += THREADS) cnt[i] = 0;
  __syncthreads();
  griddep_wait();                                    // the logits come from, and the outputs may be read by, the kernel before

  const long long first = blockIdx.x * chunk, last = first + chunk < a.T ? first + chunk : a.T;
  const int run = static_cast<int>((chunk + GROUPS - 1) / GROUPS);         // (a 148th of 2^31 tokens)
  const long long t0 = first + static_cast<long long>(grp) * run, t1 = t0 + run < last ? t0 + run : last;
  int* my_cnt = cnt + grp * E;
  float acc[EPL], x[EPL], next[EPL];
  bool next_live = false;
#pragma unroll
  for (int i = 0; i < EPL; ++i) { acc[i] = 0.0f; next[i] = RT_NINF; }
  int live = 0;
  auto load = [&](long long t) {
    route_load<LPT, EPL>(a, t, sub, next);
    next_live = a.mask == nullptr || a.mask[t] != 0;
  };
  if (t0 < t1) load(t0);
  // A run's probabilities are added up by 64 tokens at a time, so that no sum has more than 64 and a 64th of the run's roundings.
  int it = 0;
  do {
    const bool begun = it > 0;
    const int end = min(it + RT_FLUSH, run);
    for (; it < end; ++it) {                         // every group of a warp: the shuffles below are the warp's
      const long long t = t0 + it;
      const bool in = t < t1;
#pragma unroll
      for (int i = 0; i < EPL; ++i) x[i] = in && next_live ? next[i] : RT_NINF;
      if (t + 1 < t1) load(t + 1);
      float p[EPL], m, inv;
      live += route_softmax<LPT, EPL>(x, p, m, inv) ? 1 : 0;
#pragma unroll
      for (int i = 0; i < EPL; ++i) acc[i] += p[i];
      int my_id;
      float my_x;
      route_select<LPT, EPL, KEY16>(x, sub, k, my_id, my_x);
      if (sub >= k) my_id = -1;
      const float ev = my_id >= 0 ? route_exp(my_x, m) : 0.0f;
      const float scale = a.renorm ? 1.0f / group_sum<LPT>(ev) : inv;
      if (in && sub < k) {
        const long long o = t * k + sub;
        ids[o] = my_id;
        gates[o] = my_id >= 0 ? ev * scale : 0.0f;
        int r = -1;
        if (my_id >= 0) {                              // the token's experts differ: no two lanes share a counter
          r = my_cnt[my_id];
          my_cnt[my_id] = r + 1;
        }
        if (staged) {
          slot_id[o - first * k] = my_id;
          slot_rank[o - first * k] = r;
        } else {
          pos[o] = r;                                  // within the group, for now
        }
      }
      __syncwarp();
    }
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (sub * EPL + i < E) {
        float* sum = ps + grp * E + sub * EPL + i;
        *sum = begun ? *sum + acc[i] : acc[i];
        acc[i] = 0.0f;
      }
  } while (it < run);
  if (sub == 0) live_of[grp] = live;
  __syncthreads();

  // Counts of the groups before, and the block's own: a thread takes an expert and one of `parts` runs of groups.
  const bool only = gridDim.x == 1;
  const int parts = max(1, min(THREADS / E, 16)), per = (GROUPS + parts - 1) / parts;
  double part = 0.0;
  int n = 0;
  if (threadIdx.x < 32) {
    for (int g = threadIdx.x; g < GROUPS; g += 32) n += live_of[g];
    n = __reduce_add_sync(0xFFFFFFFFu, n);
  }
  int carry = 0;
  for (int e0 = 0; e0 < E; e0 += THREADS / parts) {  // (uniform: the barriers are the whole block's; one round where E <= THREADS)
    const int width = min(E - e0, THREADS / parts);
    const int q = threadIdx.x / width, e = e0 + threadIdx.x % width;
    const bool on = q < parts;
    int c = 0;
    float s = 0.0f;
    if (on) {
#pragma unroll 4
      for (int g = q * per; g < min(GROUPS, (q + 1) * per); ++g) {
        c += cnt[g * E + e];
        s += ps[g * E + e];
      }
      part_c[q * width + e - e0] = c;
      part_p[q * width + e - e0] = s;
    }
    __syncthreads();
    int before = 0, total = 0;
    float psum_e = 0.0f;
    if (on) {
      for (int r = 0; r < parts; ++r) {
        const int v = part_c[r * width + e - e0];
        before += r < q ? v : 0;
        total += v;
        psum_e += part_p[r * width + e - e0];
      }
#pragma unroll 4
      for (int g = q * per; g < min(GROUPS, (q + 1) * per); ++g) {
        const int v = cnt[g * E + e];
        cnt[g * E + e] = before;
        before += v;
      }
    }
    const bool mine = on && q == 0;
    if (only) {
      const int off = carry + block_scan(mine ? total : 0, warp_sums);
      carry += warp_sums[32];
      if (mine) {
        base[e] = off;
        counts[e] = total;
        offsets[e] = off;
        part += static_cast<double>(total) * psum_e;
      }
    } else if (mine) {
      hist[static_cast<size_t>(e) * gridDim.x + blockIdx.x] = total;
      psum[static_cast<size_t>(e) * gridDim.x + blockIdx.x] = psum_e;
      base[e] = 0;
    }
    __syncthreads();
  }
  if (only) {
    const double all = block_sum(part, sums);
    if (threadIdx.x == 0) {
      counts[E] = n;
      offsets[E] = carry;
      if (loss != nullptr) *loss = n > 0 ? static_cast<float>(all * E / (static_cast<double>(k) * n * n)) : 0.0f;
    }
  } else if (threadIdx.x == 0) {
    hist[static_cast<size_t>(E) * gridDim.x + blockIdx.x] = n;
  }
  // The slots' rows within the block (or for good, and then the rows' tokens too).
  for (long long i = t0 * k + sub; i < t1 * k; i += LPT) {
    const int id = staged ? slot_id[i - first * k] : ids[i];
    int r = -1;
    if (id >= 0) {
      r = (staged ? slot_rank[i - first * k] : pos[i]) + cnt[grp * E + id] + base[id];
      if (only) row_token[r] = static_cast<int32_t>(i / k);
    }
    pos[i] = r;
  }
}

// Blocks 0 .. B - 1: the final rows of the tokens of a block of the first kernel.  The last block: counts, offsets and the loss.
// Shared memory: base [E], total [E], sum of p [E].
__global__ void __launch_bounds__(1024)
route_finish_kernel(int B, int E, int k, long long T, long long chunk, const int32_t* __restrict__ hist,
                    const float* __restrict__ psum, const int32_t* __restrict__ ids, int32_t* pos, int32_t* __restrict__ counts,
                    int32_t* __restrict__ offsets, int32_t* __restrict__ row_token, float* __restrict__ loss) {
  griddep_launch_dependents();
  extern __shared__ __align__(16) unsigned char rt_smem[];
  int* base = reinterpret_cast<int*>(rt_smem);
  int* total = base + E;
  float* prob = reinterpret_cast<float*>(total + E);
  __shared__ int warp_sums[33];
  __shared__ double sums[32];
  griddep_wait();

  const int mine = static_cast<int>(blockIdx.x);     // B: the sums
  const bool summing = mine == B;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int PER = (RT_MAX_BLOCKS + 31) / 32;
  for (int e = warp; e < E; e += 32) {               // a warp takes an expert: every block's count of it
    int v[PER];
    float q[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int b = lane + 32 * i;
      v[i] = b < B ? hist[static_cast<size_t>(e) * B + b] : 0;
      q[i] = summing && b < B ? psum[static_cast<size_t>(e) * B + b] : 0.0f;
    }
    int all = 0, before = 0;
    float p = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      all += v[i];
      p += q[i];
      before += lane + 32 * i < mine ? v[i] : 0;
    }
    all = __reduce_add_sync(0xFFFFFFFFu, all);
    if (summing) {
      p = group_sum<32>(p);
      if (lane == 0) prob[e] = p;
    } else {
      before = __reduce_add_sync(0xFFFFFFFFu, before);
      if (lane == 0) base[e] = before;
    }
    if (lane == 0) total[e] = all;
  }
  __syncthreads();
  const int e = threadIdx.x;                         // E <= 1024
  const int all = e < E ? total[e] : 0;
  const int off = block_scan(all, warp_sums);
  if (summing) {
    const int rows = warp_sums[32];
    if (e < E) {
      counts[e] = all;
      offsets[e] = off;
    }
    int live = 0;
    for (int o = threadIdx.x; o < B; o += blockDim.x) live += hist[static_cast<size_t>(E) * B + o];
    block_scan(live, warp_sums);
    const double n = warp_sums[32];
    const double sum = block_sum(e < E ? static_cast<double>(all) * prob[e] : 0.0, sums);
    if (threadIdx.x == 0) {
      counts[E] = static_cast<int32_t>(n);
      offsets[E] = rows;
      if (loss != nullptr) *loss = n > 0.0 ? static_cast<float>(sum * E / (static_cast<double>(k) * n * n)) : 0.0f;
    }
    return;
  }
  if (e < E) base[e] += off;
  __syncthreads();
  const long long first = mine * chunk, last = first + chunk < T ? first + chunk : T;
  for (long long i = first * k + threadIdx.x; i < last * k; i += blockDim.x) {
    const int id = ids[i];
    if (id >= 0) {
      const int r = pos[i] + base[id];
      pos[i] = r;
      row_token[r] = static_cast<int32_t>(first + static_cast<unsigned>(i - first * k) / static_cast<unsigned>(k));
    }
  }
}

__device__ __forceinline__ uint32_t pack16(float a, float b, int dtype) {
  if (dtype == SQ_F16) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// What the slots of a group's token add to its logits' gradients, from the lanes that hold the slots to those that hold the logits,
// through a row that is all zeros before and after.  The last barrier is for the next token, whose slot of the same expert
// another lane may hold: its value must not be cleared by this one.  All lanes of the warp.
template <int EPL>
__device__ __forceinline__ void route_spread(float* row, bool put, int id, float add, int sub, float (&extra)[EPL]) {
  if (put) row[id] = add;                            // the token's experts differ: no two lanes write one place
  __syncwarp();
#pragma unroll
  for (int i = 0; i < EPL; ++i) extra[i] = row[sub * EPL + i];
  __syncwarp();
  if (put) row[id] = 0.0f;
  __syncwarp();
}

template <int LPT, int EPL>
__global__ void __launch_bounds__(256)
route_backward_kernel(const RouteArgs a, const int32_t* __restrict__ ids, const float* __restrict__ gates,
                      const int32_t* __restrict__ counts, const float* __restrict__ dgates, const float* __restrict__ dloss,
                      void* dlogits, long long ld_d, int vec_d) {
  griddep_launch_dependents();
  // A group's row of what its slots add to the logits' gradients: all zeros between tokens.
  __shared__ __align__(16) float rows[256 / LPT][LPT * EPL];
  float* add_row = rows[threadIdx.x / LPT];
#pragma unroll
  for (int i = 0; i < EPL; ++i) add_row[(threadIdx.x % LPT) * EPL + i] = 0.0f;
  __syncwarp();
  griddep_wait();
  const int sub = threadIdx.x % LPT, E = a.E, k = a.k;
  const long long groups = static_cast<long long>(gridDim.x) * (blockDim.x / LPT);
  const long long g0 = blockIdx.x * static_cast<long long>(blockDim.x / LPT) + threadIdx.x / LPT;
  float c[EPL];
  {
    const double n = counts[E];
    const double w = dloss != nullptr && n > 0.0 ? static_cast<double>(*dloss) * E / (k * n * n) : 0.0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) c[i] = sub * EPL + i < E ? static_cast<float>(w * counts[sub * EPL + i]) : 0.0f;
  }
  const long long rounds = (a.T + groups - 1) / groups;
  for (long long r = 0; r < rounds; ++r) {           // every group of a warp: the shuffles are the warp's
    const long long t = g0 + r * groups;
    const bool in = t < a.T;
    float x[EPL], p[EPL], d[EPL], m, inv;
    const bool live = in && (a.mask == nullptr || a.mask[t] != 0);
    if (live) {
      route_load<LPT, EPL>(a, t, sub, x);
    } else {
#pragma unroll
      for (int i = 0; i < EPL; ++i) x[i] = RT_NINF;
    }
    int id = -1;
    float dg = 0.0f, g = 0.0f;
    if (in && sub < k) {
      id = ids[t * k + sub];
      if (id >= 0) {
        dg = dgates != nullptr ? dgates[t * k + sub] : 0.0f;
        g = gates[t * k + sub];
      }
    }
    const bool counts_in = route_softmax<LPT, EPL>(x, p, m, inv);
#pragma unroll
    for (int i = 0; i < EPL; ++i) d[i] = counts_in ? c[i] : 0.0f;         // (p = 0 times a loss that overflowed)
    float add = dg;
    if (a.renorm) add = g * (dg - group_sum<LPT>(g * dg));
    float extra[EPL];
    route_spread<EPL>(add_row, id >= 0 && id < E, id, add, sub, extra);
    if (!a.renorm) {
#pragma unroll
      for (int i = 0; i < EPL; ++i) { d[i] += extra[i]; extra[i] = 0.0f; }
    }
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < EPL; ++i) dot += p[i] * d[i];
    dot = group_sum<LPT>(dot);
#pragma unroll
    for (int i = 0; i < EPL; ++i) d[i] = p[i] * (d[i] - dot) + extra[i];
    if (!in) continue;
    const int e0 = sub * EPL;
    if (a.dtype == SQ_F32) {
      float* row = static_cast<float*>(dlogits) + t * ld_d + e0;
      if (EPL % 4 == 0 && vec_d) {
        if (e0 < E) {
#pragma unroll
          for (int i = 0; i < EPL / 4; ++i)
            *reinterpret_cast<float4*>(row + 4 * i) = make_float4(d[4 * i], d[4 * i + 1 < EPL ? 4 * i + 1 : 0], d[4 * i + 2 < EPL ? 4 * i + 2 : 0],
                                                                  d[4 * i + 3 < EPL ? 4 * i + 3 : 0]);
        }
      } else if (EPL == 2 && vec_d) {
        if (e0 < E) *reinterpret_cast<float2*>(row) = make_float2(d[0], d[EPL - 1]);
      } else {
#pragma unroll
        for (int i = 0; i < EPL; ++i)
          if (e0 + i < E) row[i] = d[i];
      }
    } else {
      unsigned short* row = static_cast<unsigned short*>(dlogits) + t * ld_d + e0;
      if (EPL % 2 == 0 && vec_d) {
        if (e0 < E) {
#pragma unroll
          for (int i = 0; i < EPL / 2; ++i)
            *reinterpret_cast<uint32_t*>(row + 2 * i) = pack16(d[2 * i], d[2 * i + 1 < EPL ? 2 * i + 1 : 0], a.dtype);
        }
      } else {
#pragma unroll
        for (int i = 0; i < EPL; ++i)
          if (e0 + i < E) row[i] = static_cast<unsigned short>(pack16(d[i], 0.0f, a.dtype) & 0xFFFFu);
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Combination
// ---------------------------------------------------------------------------------------------
// VEC: eight channels a thread and piece (N % 8 == 0), else one.  A block takes 256 PIECES pieces of one token after the other; SLOTS
// rows of each are requested at once, and where the next token's rows are is known before this one's are added: what counts is
// how many bytes are on their way (2048 tokens of 4096 channels: 12.2 us with one piece of two slots, 9.7
// with two; 4001 tokens, six slots, 2048 channels: 31.7 us without looking ahead, 22.5 with).
template <bool VEC, int SLOTS, int PIECES>
__global__ void __launch_bounds__(256)
combine_kernel(const __half* __restrict__ Y, long long M, const int32_t* __restrict__ pos, const float* __restrict__ gates,
               long long T, int k, long long N, __half* __restrict__ out) {
  griddep_launch_dependents();
  griddep_wait();
  constexpr int W = VEC ? 8 : 1;
  const long long c = (blockIdx.x * (256ll * PIECES) + threadIdx.x) * W;
  if (c >= N) return;
  int row[SLOTS];
  float gate[SLOTS];
  auto look = [&](long long t, int j0) {
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
      row[j] = -1;
      gate[j] = 0.0f;
      if (j0 + j < k) {
        row[j] = pos[t * k + j0 + j];
        gate[j] = gates[t * k + j0 + j];
      }
    }
  };
  if (blockIdx.y < T) look(blockIdx.y, 0);
  for (long long t = blockIdx.y; t < T; t += gridDim.y) {
    float acc[PIECES][W];
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int w = 0; w < W; ++w) acc[p][w] = 0.0f;
    for (int j0 = 0; j0 < k; j0 += SLOTS) {
      float g[SLOTS];
      uint4 v[SLOTS][PIECES];
#pragma unroll
      for (int j = 0; j < SLOTS; ++j) {
        const bool there = row[j] >= 0 && row[j] < M;
        g[j] = there ? gate[j] : 0.0f;
        const __half* y = Y + static_cast<size_t>(there ? row[j] : 0) * N + c;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
          v[j][p] = make_uint4(0u, 0u, 0u, 0u);
          if (there && c + p * 256 * W < N) {
            if constexpr (VEC) v[j][p] = __ldg(reinterpret_cast<const uint4*>(y + p * 256 * W));
            else v[j][p].x = __half_as_ushort(y[p * 256]);
          }
        }
      }
      if (j0 + SLOTS < k) look(t, j0 + SLOTS);
      else if (t + gridDim.y < T) look(t + gridDim.y, 0);
#pragma unroll
      for (int j = 0; j < SLOTS; ++j)
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
          if constexpr (VEC) {
            const uint32_t u[4] = {v[j][p].x, v[j][p].y, v[j][p].z, v[j][p].w};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[w]));
              acc[p][2 * w] = fmaf(g[j], f.x, acc[p][2 * w]);
              acc[p][2 * w + 1] = fmaf(g[j], f.y, acc[p][2 * w + 1]);
            }
          } else {
            acc[p][0] = fmaf(g[j], __half2float(__ushort_as_half(static_cast<unsigned short>(v[j][p].x))), acc[p][0]);
          }
        }
    }
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const long long cp = c + p * 256 * W;
      if (cp >= N) continue;
      if constexpr (VEC) {
        uint4 o;
        uint32_t* ow = reinterpret_cast<uint32_t*>(&o);
#pragma unroll
        for (int w = 0; w < 4; ++w) ow[w] = pack16(acc[p][2 * w], acc[p][2 * w + 1], SQ_F16);
        *reinterpret_cast<uint4*>(out + t * N + cp) = o;
      } else {
        out[t * N + cp] = __float2half_rn(acc[p][0]);
      }
    }
  }
}

// A block takes a token: its dout is read once for up to four of its rows at a time, whose products with it are added up over
// the block in a fixed order.
template <bool VEC>
__global__ void __launch_bounds__(256)
combine_backward_kernel(const __half* __restrict__ dout, const __half* __restrict__ Y, long long M, const int32_t* __restrict__ pos,
                        const float* __restrict__ gates, long long T, int k, long long N, __half* __restrict__ dY,
                        float* __restrict__ dgates) {
  griddep_launch_dependents();
  griddep_wait();
  constexpr int W = VEC ? 8 : 1;
  __shared__ float part[4][8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (long long t = blockIdx.x; t < T; t += gridDim.x) {
    for (int j0 = 0; j0 < k; j0 += 4) {
      int r[4];
      float g[4], s[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        r[j] = j0 + j < k ? pos[t * k + j0 + j] : -1;
        if (r[j] >= M) r[j] = -1;
        g[j] = r[j] >= 0 ? gates[t * k + j0 + j] : 0.0f;
        s[j] = 0.0f;
      }
      for (long long c = threadIdx.x * W; c < N; c += 256 * W) {
        if constexpr (VEC) {
          const uint4 dv = __ldg(reinterpret_cast<const uint4*>(dout + t * N + c));
          uint4 yv[4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            yv[j] = r[j] >= 0 && dgates != nullptr ? __ldg(reinterpret_cast<const uint4*>(Y + static_cast<size_t>(r[j]) * N + c))
                                                   : make_uint4(0u, 0u, 0u, 0u);
          float d[8];
          const uint32_t du[4] = {dv.x, dv.y, dv.z, dv.w};
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&du[w]));
            d[2 * w] = f.x;
            d[2 * w + 1] = f.y;
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (r[j] < 0) continue;
            const uint32_t yu[4] = {yv[j].x, yv[j].y, yv[j].z, yv[j].w};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&yu[w]));
              s[j] = fmaf(d[2 * w], f.x, s[j]);
              s[j] = fmaf(d[2 * w + 1], f.y, s[j]);
            }
            if (dY != nullptr) {
              uint4 o;
              uint32_t* ow = reinterpret_cast<uint32_t*>(&o);
#pragma unroll
              for (int w = 0; w < 4; ++w) ow[w] = pack16(g[j] * d[2 * w], g[j] * d[2 * w + 1], SQ_F16);
              *reinterpret_cast<uint4*>(dY + static_cast<size_t>(r[j]) * N + c) = o;
            }
          }
        } else {
          const float d = __half2float(dout[t * N + c]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (r[j] < 0) continue;
            const size_t o = static_cast<size_t>(r[j]) * N + c;
            if (dgates != nullptr) s[j] = fmaf(d, __half2float(Y[o]), s[j]);
            if (dY != nullptr) dY[o] = __float2half_rn(g[j] * d);
          }
        }
      }
      if (dgates != nullptr) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float v = group_sum<32>(s[j]);
          if (lane == 0) part[j][warp] = v;
        }
        __syncthreads();
        if (threadIdx.x < 4 && j0 + static_cast<int>(threadIdx.x) < k) {
          float v = 0.0f;
#pragma unroll
          for (int w = 0; w < 8; ++w) v += part[threadIdx.x][w];
          dgates[t * k + j0 + threadIdx.x] = v;
        }
        __syncthreads();
      }
    }
  }
}

int route_lanes(int E) { return E <= 8 ? 8 : (E <= 16 ? 16 : 32); }

// Blocks of the first kernel: one, of 256 threads, while a group of lanes has no more than four tokens (the second launch costs
// more than what more SMs would save); else as many as give every group of 1024 threads (512: more registers) one.
int route_threads(int64_t T, int E) {
  if (T <= 4 * (256 / route_lanes(E))) return 256;
  return E <= 256 ? 1024 : 512;
}
int route_blocks(int64_t T, int E) {
  const int threads = route_threads(T, E);
  if (threads == 256) return 1;
  const int64_t groups = threads / route_lanes(E);
  return static_cast<int>(std::min<int64_t>(RT_MAX_BLOCKS, std::max<int64_t>(2, (T + groups - 1) / groups)));
}

size_t elem_bytes(int dtype) { return dtype == SQ_F32 ? 4 : 2; }

// Whether a lane's EPL experts may be read or written as one or more whole pieces of up to 16 bytes.
int route_vec(const void* p, int dtype, int E, long long ld, int epl) {
  const size_t piece = std::min<size_t>(16, epl * elem_bytes(dtype));
  return E % epl == 0 && (ld * elem_bytes(dtype)) % piece == 0 && reinterpret_cast<uintptr_t>(p) % piece == 0;
}

template <typename F>
sq_status_t with_shape(int E, F f) {
  if (E <= 8) return f(std::integral_constant<int, 8>(), std::integral_constant<int, 1>());
  if (E <= 16) return f(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
  if (E <= 32) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 1>());
  if (E <= 64) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 2>());
  if (E <= 128) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 4>());
  if (E <= 256) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 8>());
  if (E <= 512) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 16>());
  return f(std::integral_constant<int, 32>(), std::integral_constant<int, 32>());
}

}  // namespace

size_t route_workspace_bytes(int64_t T, int32_t E) {
  const size_t B = route_blocks(T, E);
  if (B == 1) return 0;
  return (B * (E + 1) * 4 + 255) / 256 * 256 + (B * E * 4 + 255) / 256 * 256;
}

sq_status_t launch_route(const void* logits, int dtype, int64_t T, int E, int64_t ld, int k, bool renorm, const void* mask, void* ids,
                         void* gates, void* counts, void* offsets, void* row_token, void* pos, void* loss, void* workspace,
                         cudaStream_t s) {
  const int B = route_blocks(T, E);
  const long long chunk = (T + B - 1) / B;
  int32_t* hist = static_cast<int32_t*>(workspace);
  float* psum = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + (static_cast<size_t>(B) * (E + 1) * 4 + 255) / 256 * 256);
  int32_t *idsp = static_cast<int32_t*>(ids), *posp = static_cast<int32_t*>(pos), *cnt = static_cast<int32_t*>(counts),
          *off = static_cast<int32_t*>(offsets), *rt = static_cast<int32_t*>(row_token);
  const sq_status_t st = with_shape(E, [&](auto lpt, auto epl) -> sq_status_t {
    constexpr int LPT = decltype(lpt)::value, EPL = decltype(epl)::value;
    const RouteArgs a = {logits, dtype, E, k, T, ld, renorm ? 1 : 0, route_vec(logits, dtype, E, ld, EPL), static_cast<const uint8_t*>(mask)};
    constexpr int BIG = EPL <= 8 ? 1024 : 512;
    const int threads = route_threads(T, E);
    auto kern = dtype == SQ_F32 ? (threads == 256 ? route_kernel<LPT, EPL, 256, false> : route_kernel<LPT, EPL, BIG, false>)
                                : (threads == 256 ? route_kernel<LPT, EPL, 256, true> : route_kernel<LPT, EPL, BIG, true>);
    const int staged = chunk * k <= RT_STAGED;
    const int smem = ((2 * (threads / LPT) + 1) * E + 2 * threads + (staged ? 2 * RT_STAGED : 0)) * 4;
    // The kernel's static shared memory, below 2 KB, counts towards the 48 KB that need no asking.
    if (!ensure_dyn_smem(reinterpret_cast<const void*>(kern), smem > 46 * 1024 ? std::max(smem, 48 * 1024 + 16) : smem)) return SQ_ERR_CUDA;
    const cudaError_t err = launch_maybe_pdl(kern, dim3(static_cast<unsigned>(B)), dim3(static_cast<unsigned>(threads)), static_cast<size_t>(smem), s, a, chunk,
                                             staged, idsp, static_cast<float*>(gates), posp, hist, psum, cnt, off, rt, static_cast<float*>(loss));
    count_launch();
    return err == cudaSuccess ? SQ_OK : SQ_ERR_CUDA;
  });
  if (st != SQ_OK || B == 1) return st;
  const int smem = 3 * E * 4;
  const cudaError_t err = launch_dependent(route_finish_kernel, dim3(static_cast<unsigned>(B + 1)), dim3(1024), static_cast<size_t>(smem), s, B,
                                           E, k, static_cast<long long>(T), chunk, static_cast<const int32_t*>(hist),
                                           static_cast<const float*>(psum), static_cast<const int32_t*>(idsp), posp, cnt, off, rt,
                                           static_cast<float*>(loss));
  count_launch();
  return err == cudaSuccess ? SQ_OK : SQ_ERR_CUDA;
}

sq_status_t launch_route_backward(const void* logits, int dtype, int64_t T, int E, int64_t ld, int k, bool renorm, const void* mask,
                                  const void* ids, const void* gates, const void* counts, const void* dgates, const void* dloss,
                                  void* dlogits, int64_t ld_d, cudaStream_t s) {
  const int sms = sm_count();
  if (sms <= 0) return SQ_ERR_CUDA;
  return with_shape(E, [&](auto lpt, auto epl) -> sq_status_t {
    constexpr int LPT = decltype(lpt)::value, EPL = decltype(epl)::value;
    const RouteArgs a = {logits, dtype, E, k, T, ld, renorm ? 1 : 0, route_vec(logits, dtype, E, ld, EPL), static_cast<const uint8_t*>(mask)};
    const long long blocks = (T + 256 / LPT - 1) / (256 / LPT);
    const unsigned grid = static_cast<unsigned>(std::min<long long>(blocks, static_cast<long long>(sms) * 8));
    const cudaError_t err = launch_maybe_pdl(route_backward_kernel<LPT, EPL>, dim3(grid), dim3(256), 0, s, a, static_cast<const int32_t*>(ids),
                                             static_cast<const float*>(gates), static_cast<const int32_t*>(counts),
                                             static_cast<const float*>(dgates), static_cast<const float*>(dloss), dlogits,
                                             static_cast<long long>(ld_d), route_vec(dlogits, dtype, E, ld_d, EPL));
    count_launch();
    return err == cudaSuccess ? SQ_OK : SQ_ERR_CUDA;
  });
}

sq_status_t launch_combine(const void* Y, int64_t M, const void* pos, const void* gates, int64_t T, int k, int64_t N, void* out,
                           cudaStream_t s) {
  const bool vec = N % 8 == 0;
  const int pieces = k <= 2 && N > 2048 ? 2 : 1;
  const int64_t width = 256 * pieces * (vec ? 8 : 1), across = (N + width - 1) / width;
  const int64_t down = std::min<int64_t>(T, std::max<int64_t>(1, 8 * std::max(sm_count(), 1) / across));
  const dim3 grid(static_cast<unsigned>(across), static_cast<unsigned>(down));
  auto kern = pieces == 2 ? (vec ? combine_kernel<true, 2, 2> : combine_kernel<false, 2, 2>)
                          : (vec ? combine_kernel<true, 4, 1> : combine_kernel<false, 4, 1>);
  const cudaError_t err = launch_maybe_pdl(kern, grid, dim3(256), 0, s,
                                           static_cast<const __half*>(Y), static_cast<long long>(M), static_cast<const int32_t*>(pos),
                                           static_cast<const float*>(gates), static_cast<long long>(T), k, static_cast<long long>(N),
                                           static_cast<__half*>(out));
  count_launch();
  return err == cudaSuccess ? SQ_OK : SQ_ERR_CUDA;
}

sq_status_t launch_combine_backward(const void* dout, const void* Y, int64_t M, const void* pos, const void* gates, int64_t T, int k,
                                    int64_t N, void* dY, void* dgates, cudaStream_t s) {
  const int sms = sm_count();
  if (sms <= 0) return SQ_ERR_CUDA;
  const unsigned grid = static_cast<unsigned>(std::min<long long>(T, static_cast<long long>(sms) * 8));
  const cudaError_t err = launch_maybe_pdl(N % 8 == 0 ? combine_backward_kernel<true> : combine_backward_kernel<false>, dim3(grid), dim3(256),
                                           0, s, static_cast<const __half*>(dout), static_cast<const __half*>(Y), static_cast<long long>(M),
                                           static_cast<const int32_t*>(pos), static_cast<const float*>(gates), static_cast<long long>(T), k,
                                           static_cast<long long>(N), static_cast<__half*>(dY), static_cast<float*>(dgates));
  count_launch();
  return err == cudaSuccess ? SQ_OK : SQ_ERR_CUDA;
}

}  // namespace sq
