// Choice of the blocks of a block-sparse decode step: bounds of each block's keys,
// kept in 8 bits, and for each KV head the blocks whose bounds score highest
// against the step's queries.
//
// A block is 32 cached rows.  With hi_c and lo_c the largest and smallest value of
// channel c over its keys (a NaN counts as 0, an infinity as the largest bf16
// number) and 2^t the power of two that brings max_c max(|hi_c|, |lo_c|) into
// (63.5, 127] (t in [-60, 50]), the bounds are held as H_c = ceil(hi_c / 2^t) and
// L_c = floor(lo_c / 2^t), rounded outwards so that they still bound the keys.
// A query row is brought to Q_c = rint(q_c / 2^u) likewise, and
//   score = max over the group's queries of 2^(t+u) * sum_c max(Q_c H_c, Q_c L_c),
// an upper bound of its products with the block's keys but for Q's rounding.  The
// sums are of integers and exact, and so is the power of two in fp32: the choice does
// not depend on the order of anything.
#include <algorithm>

#include "block_choice.h"
#include "select.h"

namespace ra {
namespace {

struct BoundsBatch {
  int n;                      // ranges
  BoundsRange r[kBoundsBatch];
  int layer[kBoundsBatch];
};

typedef int16_t i16x2 __attribute__((ext_vector_type(2)));

// Two bf16 numbers as integers of the same order, and back.
__device__ __forceinline__ i16x2 bf16_order(uint32_t w) {
  i16x2 x;
  __builtin_memcpy(&x, &w, 4);
  return x ^ ((x >> 15) & int16_t(0x7fff));
}
__device__ __forceinline__ float bf16_of_order(int16_t x) {
  const int16_t b = x ^ ((x >> 15) & 0x7fff);
  return __uint_as_float(static_cast<uint32_t>(static_cast<uint16_t>(b)) << 16);
}

// Two codes (the low or the high ones of w) times their row's scale, as bf16.
template <bool HIGH>
__device__ __forceinline__ uint32_t bf16_pair(uint32_t w, float scale) {
  const auto x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HIGH);
  uint32_t r;
  __builtin_memcpy(&r, &x, 4);
  return r;
}

// x joined over the lanes with the same lane & 15.
template <typename F>
__device__ __forceinline__ void over_groups(i16x2& x, F&& join) {
  uint32_t u;
  const auto step = [&](auto pair) {
    i16x2 a, b;
    const uint32_t p = pair[0], q = pair[1];
    __builtin_memcpy(&a, &p, 4);
    __builtin_memcpy(&b, &q, 4);
    x = join(a, b);
  };
  __builtin_memcpy(&u, &x, 4);
  step(__builtin_amdgcn_permlane16_swap(u, u, false, false));
  __builtin_memcpy(&u, &x, 4);
  step(__builtin_amdgcn_permlane32_swap(u, u, false, false));
}

// One wavefront per block: lane (c8, r4) folds eight channels of eight rows as packed
// 16-bit integers, the four row groups join by lane swaps; rows with an infinity or a NaN
// are folded again without them.  Bound by HBM, the key rows once per row that an event
// or a write has changed: 256 heads of 9,216 rows 108 us in bf16 (5.8 TB/s, the bounds
// written included), 63 in e4m3 (5.1; folded in fp32 with shuffles 71).  Two, four or eight blocks to a wavefront, the
// next one's rows prefetched, and for e4m3 16-byte units of four rows, took 5 to 60%
// longer.  Grid: (ceil(blocks / 4), Hkv, ranges x layers).
template <bool E4M3, bool PAGED>
__global__ __launch_bounds__(256) void block_bounds_kernel(
    const SeqMeta* __restrict__ meta, const void* __restrict__ kpool,
    const uint8_t* __restrict__ k_scale, int8_t* __restrict__ bounds, int8_t* __restrict__ units,
    int Hkv, Paging pg, BoundsBatch batch) {
  const BoundsRange range = batch.r[blockIdx.z % batch.n];
  const int layer = batch.layer[blockIdx.z / batch.n];
  const int b = range.from + static_cast<int>(blockIdx.x) * 4 +
                __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (b >= range.to) return;
  const SeqMeta& M = meta[range.slot];
  const RowMap rm = row_map(M, range.slot, layer * Hkv + static_cast<int>(blockIdx.y), pg);
  const int64_t row0 = pool_row<PAGED>(rm, b * kBlockRows);
  const int lane = threadIdx.x & 63, c8 = lane & 15, r4 = lane >> 4;
  uint32_t w[8][4];                            // eight rows, pairs of channels in bf16
  if constexpr (E4M3) {
    uint2 codes[8];
    uint32_t scale[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int64_t row = row0 + r4 + 4 * e;
      codes[e] = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(kpool) +
                                                 row * kHeadDim + 8 * c8);
      scale[e] = k_scale[row];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = e4m3_scale(scale[e]);
      w[e][0] = bf16_pair<false>(codes[e].x, x);
      w[e][1] = bf16_pair<true>(codes[e].x, x);
      w[e][2] = bf16_pair<false>(codes[e].y, x);
      w[e][3] = bf16_pair<true>(codes[e].y, x);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const u32x4 x =
          ld16(static_cast<const uint16_t*>(kpool) + (row0 + r4 + 4 * e) * kHeadDim + 8 * c8);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[e][i] = x[i];
    }
  }
  i16x2 most[4], least[4];
  bool odd = false;                            // infinities or NaNs among the rows
  const auto fold = [&] {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      most[i] = least[i] = bf16_order(w[0][i]);
#pragma unroll
      for (int e = 1; e < 8; ++e) {
        const i16x2 x = bf16_order(w[e][i]);
        most[i] = __builtin_elementwise_max(most[i], x);
        least[i] = __builtin_elementwise_min(least[i], x);
      }
      over_groups(most[i], [](i16x2 x, i16x2 y) { return __builtin_elementwise_max(x, y); });
      over_groups(least[i], [](i16x2 x, i16x2 y) { return __builtin_elementwise_min(x, y); });
#pragma unroll
      for (int h = 0; h < 2; ++h)
        odd = odd || most[i][h] >= 0x7f80 || least[i][h] <= -0x7f81;
    }
  };
  fold();
  if (__any(odd)) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[e][i] = bf16_pack_exact(finite_bf16(bf16_low(w[e][i])), finite_bf16(bf16_high(w[e][i])));
    fold();
  }
  float hi[8], lo[8];
  uint32_t amax = 0;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    hi[c] = bf16_of_order(most[c / 2][c & 1]);
    lo[c] = bf16_of_order(least[c / 2][c & 1]);
    amax = max(amax, max(__float_as_uint(fabsf(hi[c])), __float_as_uint(fabsf(lo[c]))));
  }
  const int t = unit_exponent(max_over_row16(amax));
  const float inv = pow2(-t);
  if (r4 < 2) {
    float v[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) v[c] = r4 == 0 ? ceilf(hi[c] * inv) : floorf(lo[c] * inv);
    uint2 w;
    w.x = pack_int8(v[0], v[1], v[2], v[3]);
    w.y = pack_int8(v[4], v[5], v[6], v[7]);
    *reinterpret_cast<uint2*>(bounds + row0 / kBlockRows * kBoundsBytes + kHeadDim * r4 + 8 * c8) =
        w;
  }
  if (lane == 0) units[row0 / kBlockRows] = static_cast<int8_t>(t);
}

// Choice among the candidates of long heads (shorter ones: choose_few in the
// attention kernel): workgroups of a head score kChunkBlocks candidates each and leave
// the scores in memory; the last to finish selects (select.h; as in merge_if_last,
// nothing waits for another workgroup).  One workgroup per head took 40 us for 8 heads
// of 4,096 candidates, whose bounds it read at 27 GB/s; with 512 candidates to a
// workgroup a step took 38 to 40 us, with 256 36, with 128 37.  Scores of a head share
// their sign and most of their exponent, so the select works on their distance from the
// lowest, shifted to 32 bits: on the scores themselves its first passes counted nearly all
// of them into a bin or two (16.9 and 12.8 us for 8 heads of 4,096 candidates; a step of
// 12,500 60 and 46).
constexpr int kChooseThreads = 512;
constexpr int kChunkBlocks = 256;

template <int KPT, bool PAGED>
__global__ __launch_bounds__(kChooseThreads) void choose_blocks_kernel(
    const SeqMeta* __restrict__ meta, const uint16_t* __restrict__ q, int layer, int Hq, int Hkv,
    int G, Paging pg, BlockChoice ch, uint32_t* __restrict__ scores, int score_stride,
    int* __restrict__ arrivals) {
  constexpr int NT = kChooseThreads;
  __shared__ uint32_t keys[kChunkBlocks];
  __shared__ SelectShared sel_sh;
  __shared__ uint32_t span[2][NT / 64];
  __shared__ int last;
  const int g = blockIdx.y, slot = blockIdx.z, head = slot * Hkv + g;
  const SeqMeta& M = meta[slot];
  if (!M.active) return;
  const int cand = candidate_blocks(M.len, ch.recent);
  const int lo = static_cast<int>(blockIdx.x) * kChunkBlocks;
  if (cand <= ch.n_blocks || cand <= kFusedBlocks || lo >= cand) return;
  const int n = min(cand - lo, kChunkBlocks);
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const RowMap rm = row_map(M, slot, layer * Hkv + g, pg);
  score_blocks<NT>(keys, lo, n, [&](int b) { return pool_row<PAGED>(rm, b * kBlockRows); },
                   ch.bounds, ch.units, q + (static_cast<int64_t>(slot) * Hq + g * G) * kHeadDim, G);
  __syncthreads();
  uint32_t* all = scores + static_cast<int64_t>(head) * score_stride;
  if (t < n)
    __hip_atomic_store(all + lo + t, keys[t], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (t == 0) {
    const int chunks = (cand + kChunkBlocks - 1) / kChunkBlocks;
    const int prev = __hip_atomic_fetch_add(arrivals + head, 1, __ATOMIC_RELAXED,
                                            __HIP_MEMORY_SCOPE_AGENT);
    last = prev == chunks - 1;
    if (last) __hip_atomic_store(arrivals + head, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!last) return;
  uint32_t x[KPT], low = 0xffffffffu, high = 0;
#pragma unroll
  for (int i = 0; i < KPT; i += 2) {     // (as many words as a head has, all of them there)
    const uint64_t two =
        __hip_atomic_load(reinterpret_cast<const uint64_t*>(all + t * KPT + i), __ATOMIC_RELAXED,
                          __HIP_MEMORY_SCOPE_AGENT);
    x[i] = static_cast<uint32_t>(two);
    x[i + 1] = static_cast<uint32_t>(two >> 32);
  }
#pragma unroll
  for (int i = 0; i < KPT; ++i) {
    if (t * KPT + i >= cand) break;
    low = min(low, x[i]);
    high = max(high, x[i]);
  }
  // the scores of a head share their leading bits: the radix passes see the others
  low = ~max_over_groups(max_over_row16(~low));
  high = max_over_groups(max_over_row16(high));
  if (lane == 0) {
    span[0][wave] = low;
    span[1][wave] = high;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    low = min(low, span[0][w]);
    high = max(high, span[1][w]);
  }
  const int shift = high > low ? __clz(static_cast<int>(high - low)) : 0;
  uint64_t key[KPT];
  uint32_t tie[KPT], valid = 0;
#pragma unroll
  for (int i = 0; i < KPT; ++i) {
    const int b = t * KPT + i;
    tie[i] = static_cast<uint32_t>(b);
    key[i] = (x[i] - low) << shift;
    if (b < cand) valid |= 1u << i;
  }
  const uint32_t chosen = select_smallest<NT, KPT, 32>(key, tie, valid, ch.n_blocks, sel_sh);
  const int mine = __popc(chosen), incl = wave_inclusive_scan(mine);
  if (lane == 63) sel_sh.wave_tot[wave] = incl;
  __syncthreads();
  int k = incl - mine;
  for (int w = 0; w < wave; ++w) k += sel_sh.wave_tot[w];
  int32_t* dst = ch.list + static_cast<int64_t>(head) * ch.stride;
#pragma unroll
  for (int i = 0; i < KPT; ++i)
    if ((chosen >> i) & 1) dst[k++] = t * KPT + i;
}

template <int KPT>
void launch_choose(const Shape& sh, const SeqMeta* meta, const void* q, int layer, int max_seqs,
                   const BlockChoice& ch, uint32_t* scores, int score_stride, int* arrivals,
                   int max_candidates, hipStream_t s) {
  const auto kernel = sh.pg.tables ? choose_blocks_kernel<KPT, true>
                                   : choose_blocks_kernel<KPT, false>;
  const dim3 grid((max_candidates + kChunkBlocks - 1) / kChunkBlocks, sh.Hkv, max_seqs);
  hipLaunchKernelGGL(kernel, grid, dim3(kChooseThreads), 0, s, meta,
                     static_cast<const uint16_t*>(q), layer, sh.Hq, sh.Hkv, sh.G, sh.pg, ch, scores,
                     score_stride, arrivals);
}

}  // namespace

hipError_t launch_block_bounds(const Shape& sh, const SeqMeta* meta, const void* kpool,
                               int8_t* bounds, int64_t pool_rows, const int* layers, int n_layers,
                               const BoundsRange* ranges, int n, hipStream_t s) {
  int8_t* units = bounds + pool_rows / kBlockRows * kBoundsBytes;
  const auto kernel =
      sh.dtype == 2 ? (sh.pg.tables ? block_bounds_kernel<true, true>
                                    : block_bounds_kernel<true, false>)
                    : (sh.pg.tables ? block_bounds_kernel<false, true>
                                    : block_bounds_kernel<false, false>);
  for (int l0 = 0; l0 < n_layers; l0 += kBoundsBatch) {
    for (int i0 = 0; i0 < n; i0 += kBoundsBatch) {
      BoundsBatch b{};
      b.n = std::min(kBoundsBatch, n - i0);
      const int nl = std::min(kBoundsBatch, n_layers - l0);
      std::copy(ranges + i0, ranges + i0 + b.n, b.r);
      std::copy(layers + l0, layers + l0 + nl, b.layer);
      int most = 0;
      for (int i = 0; i < b.n; ++i) most = std::max(most, b.r[i].to - b.r[i].from);
      hipLaunchKernelGGL(kernel, dim3((most + 3) / 4, sh.Hkv, b.n * nl), dim3(256), 0, s, meta,
                         kpool, sh.k_scale, bounds, units, sh.Hkv, sh.pg, b);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

hipError_t launch_choose_blocks(const Shape& sh, const SeqMeta* meta, const void* q, int layer,
                                int max_seqs, const BlockChoice& ch, uint32_t* scores,
                                int score_stride, int* arrivals, int max_candidates,
                                hipStream_t s) {
  if (max_candidates <= kFusedBlocks) return hipSuccess;
#define RA_CHOOSE(KPT)                                                                       \
  launch_choose<KPT>(sh, meta, q, layer, max_seqs, ch, scores, score_stride, arrivals,       \
                     max_candidates, s)
  if (max_candidates <= 4 * kChooseThreads) RA_CHOOSE(4);
  else if (max_candidates <= 8 * kChooseThreads) RA_CHOOSE(8);
  else if (max_candidates <= 32 * kChooseThreads) RA_CHOOSE(32);
  else return hipErrorInvalidValue;
#undef RA_CHOOSE
  static_assert(32 * kChooseThreads == kMaxBlocks, "the largest build chooses from any head");
  return hipGetLastError();
}

}  // namespace ra
