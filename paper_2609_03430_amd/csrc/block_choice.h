// Scores of a head's candidate blocks, and the choice among few of them: device code
// of the block-sparse step (the definition is in blocks.hip).
#pragma once

#include "attn_parts.h"
#include "e4m3.h"

namespace ra {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// Candidates of a head that its attention's workgroups choose from themselves, each
// all of them: a launch of its own for the choice costs more than scoring the head
// once per split (bf16 rows, microseconds per layer, here and by a launch: one request
// of 9,000 rows 17.7 and 20.5, of 16,000 20.5 and 20.9, 8 of 16,000 28 and 31, 32 of
// 16,000 44 and 52; but one of 24,000 25 and 21, where 32 of 24,000 take 50 and 52 to 55).
constexpr int kFusedBlocks = 512;

constexpr float kMaxBf16 = 3.3895313892515355e38f;

__device__ __forceinline__ float finite_bf16(float x) {
  x = x == x ? x : 0.f;
  return fminf(fmaxf(x, -kMaxBf16), kMaxBf16);
}

// t of a largest magnitude: its fp32 exponent less 6 where its fraction is at most
// 127/64, else less 5 (the sum carries), within [-60, 50].
__device__ __forceinline__ int unit_exponent(uint32_t amax_bits) {
  const int t = static_cast<int>((amax_bits + 0x01ffffu) >> 23) - 127 - 6;
  return min(max(t, -60), 50);
}

__device__ __forceinline__ float pow2(int e) { return __uint_as_float((e + 127) << 23); }

__device__ __forceinline__ uint32_t pack_int8(float a, float b, float c, float d) {
  const auto byte = [](float x) {
    return static_cast<uint32_t>(static_cast<int>(fminf(fmaxf(x, -127.f), 127.f))) & 255u;
  };
  return byte(a) | byte(b) << 8 | byte(c) << 16 | byte(d) << 24;
}

// A group's queries in 8 bits: lane (r, grp) holds channels 64 s + 16 grp .. + 15 of
// query r, the positive and the negative parts apart, and the row's exponent.
struct BlockQuery {
  i32x4 pos[2], neg[2];
  int u;
  static __device__ __forceinline__ int channel(int i, int grp) {
    return 64 * (i >> 1) + 16 * grp + 8 * (i & 1);
  }
  __device__ __forceinline__ void set(const u32x4 (&raw)[4]) {
    float x[32];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t w = raw[i >> 2][i & 3];
      x[2 * i] = finite_bf16(bf16_low(w));
      x[2 * i + 1] = finite_bf16(bf16_high(w));
      amax = max(amax, max(__float_as_uint(fabsf(x[2 * i])), __float_as_uint(fabsf(x[2 * i + 1]))));
    }
    u = unit_exponent(max_over_groups(amax));
    const float inv = pow2(-u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = rintf(x[4 * i + j] * inv);
      pos[i >> 2][i & 3] = static_cast<int>(pack_int8(fmaxf(y[0], 0.f), fmaxf(y[1], 0.f),
                                                      fmaxf(y[2], 0.f), fmaxf(y[3], 0.f)));
      neg[i >> 2][i & 3] = static_cast<int>(pack_int8(fminf(y[0], 0.f), fminf(y[1], 0.f),
                                                      fminf(y[2], 0.f), fminf(y[3], 0.f)));
    }
  }
};

// K tiles of sixteen blocks, their bounds loaded together: tile first + k * STRIDE of
// the n candidates from block lo on (in a last tile the last candidate's again past
// them, scored and not stored).
template <int K, int STRIDE>
struct ScoreTiles {
  i32x4 h[K][4];
  int unit[K];
  template <typename RowOf>
  __device__ __forceinline__ void load(int first, int lo, int n, const RowOf& row_of,
                                       const int8_t* bounds, const int8_t* units) {
    const int lane = threadIdx.x & 63, r = lane & 15, grp = lane >> 4;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (16 * (first + k * STRIDE) >= n) break;
      const int b = lo + min(16 * (first + k * STRIDE) + r, n - 1);
      const int64_t at = row_of(b) >> kBlockShift;
      const int8_t* src = bounds + at * kBoundsBytes + 16 * grp;
#pragma unroll
      for (int s = 0; s < 4; ++s) h[k][s] = *reinterpret_cast<const i32x4*>(src + 64 * s);
      unit[k] = units[at];
    }
  }
  __device__ __forceinline__ void score(uint32_t* keys, int first, int n, const BlockQuery& q,
                                        int G) const {
    const int lane = threadIdx.x & 63, r = lane & 15, grp = lane >> 4;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (16 * (first + k * STRIDE) >= n) break;
      i32x4 sum = {0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < 4; ++s)
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(h[k][s], s < 2 ? q.pos[s] : q.neg[s - 2], sum,
                                                    0, 0, 0);
      // lane (query r, grp): blocks 4 grp + i of the tile; a block's exponent is the
      // same for every query and joins after the maximum
      const int e = __shfl(unit[k], 4 * grp + (r & 3), 64);
      float best[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        best[i] = __uint_as_float(over_row16(
            __float_as_uint(r < G ? ldexpf(static_cast<float>(sum[i]), q.u) : kNegInf),
            [](uint32_t a, uint32_t b) {
              return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
            }));
      const int b = 16 * (first + k * STRIDE) + 4 * grp + r;
      const float x = ldexpf(r == 0 ? best[0] : r == 1 ? best[1] : r == 2 ? best[2] : best[3], e);
      const uint32_t bits = __float_as_uint(x);        // descending order of the scores
      if (r < 4 && b < n) keys[b] = bits >> 31 ? bits : ~(bits | 0x80000000u);
    }
  }
};

// Scores of n candidate blocks from block lo of a head on into keys[0, n), as words
// that ascend from the best: the wavefronts of the workgroup (NT threads, all of them
// call) take sixteen blocks at a time (v_mfma_i32_16x16x64_i8: blocks x [H | L] against
// [max(Q, 0); min(Q, 0)]); the first bounds are on their way while the queries are
// rounded.  row_of: the pool row at which a block of the head begins.
template <int NT, typename RowOf>
__device__ __forceinline__ void score_blocks(uint32_t* keys, int lo, int n, const RowOf& row_of,
                                             const int8_t* bounds, const int8_t* units,
                                             const uint16_t* queries, int G) {
  constexpr int kWaves = NT / 64;
  const int lane = threadIdx.x & 63, r = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  u32x4 raw[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    raw[i] = ld16(queries + (r < G ? r : 0) * kHeadDim + BlockQuery::channel(i, grp));
  ScoreTiles<4, kWaves> t;
  t.load(wave, lo, n, row_of, bounds, units);
  BlockQuery q;
  q.set(raw);
  for (int first = wave;;) {
    t.score(keys, first, n, q, G);
    first += 4 * kWaves;
    if (16 * first >= n) break;
    t.load(first, lo, n, row_of, bounds, units);
  }
}

// The want (< n) smallest of n <= 64 * kPer keys, the lowest index first among
// equals, as ascending indices: one wavefront halves the range of the keys until a
// bound has exactly `want` of them at or below it, or until it is a key that several
// share.  Called by one whole wavefront; the bounds are the same in every lane.
template <int kPer>
__device__ __forceinline__ void choose_in_wave(const uint32_t* keys, int n, int want,
                                               int32_t* dst) {
  const int lane = threadIdx.x & 63;
  uint32_t k[kPer], low = 0xffffffffu, high = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    // past the candidates: worse than any (a score is finite, its key not all ones)
    k[j] = 64 * j + lane < n ? keys[64 * j + lane] : 0xffffffffu;
    low = min(low, k[j]);
    high = max(high, 64 * j + lane < n ? k[j] : 0u);
  }
  low = ~max_over_groups(max_over_row16(~low));
  high = max_over_groups(max_over_row16(high));
  uint32_t lo = __builtin_amdgcn_readfirstlane(low), hi = __builtin_amdgcn_readfirstlane(high);
  const auto count = [&](uint32_t bound) {
    int c = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) c += __popcll(__ballot(k[j] <= bound));
    return c;
  };
  // at the end hi has at least `want` keys at or below it, hi - 1 fewer if lo == hi
  bool exact = false;
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2;
    const int c = count(mid);
    if (c >= want) hi = mid; else lo = mid + 1;
    exact = c == want;
    if (exact) break;
  }
  // every key below hi, and as many of those equal to it as are wanted
  int at = 0, equal = exact ? want : want - (hi ? count(hi - 1) : 0);
  const uint64_t below_lane = (uint64_t(1) << lane) - 1;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const uint64_t eq = __ballot(k[j] == hi), lt = __ballot(k[j] < hi);
    const bool take = (lt >> lane & 1) || ((eq >> lane & 1) && __popcll(eq & below_lane) < equal);
    const uint64_t taken = __ballot(take);
    if (take) dst[at + __popcll(taken & below_lane)] = 64 * j + lane;
    at += __popcll(taken);
    equal -= min(equal, static_cast<int>(__popcll(eq)));
  }
}

// .. of n <= kFusedBlocks keys: the fewer keys a lane holds, the shorter every step.
__device__ __forceinline__ void choose_few(const uint32_t* keys, int n, int want, int32_t* dst) {
  static_assert(kFusedBlocks == 512, "eight keys to a lane");
  if (n <= 64) choose_in_wave<1>(keys, n, want, dst);
  else if (n <= 128) choose_in_wave<2>(keys, n, want, dst);
  else if (n <= 256) choose_in_wave<4>(keys, n, want, dst);
  else choose_in_wave<8>(keys, n, want, dst);
}

}  // namespace
}  // namespace ra
