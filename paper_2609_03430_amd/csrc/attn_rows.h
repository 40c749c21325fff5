// Cached rows of each dtype as the attention kernels take them, blocks of 32 at a time: a
// lane's loads of a block, the step's new pair in its place, the scores of the block's
// keys (x[e]: key 8 * (lane >> 4) + e) and its values weighed by them (a difference of two
// scores times `unit` is one in log2 units; -inf: a masked key).
#pragma once

#include "attn_parts.h"
#include "e4m3.h"

namespace ra {
namespace {

// Pools and scales of a launch.
struct Pools {
  const void* k;
  const void* v;
  const uint8_t* k_scale;
  const uint8_t* v_scale;
};

// What this wavefront's lanes have written to LDS is there for its other lanes.
__device__ __forceinline__ void staged_in_wave() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// 2^x, a result below 2^-126 flushed to zero: nothing beside a weight of 1.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// What turns a difference of two scores into log2 units: hi, and what its rounding left, which
// fp32 rows take, too.
struct Unit {
  float hi, rest;
};
// 2^(x unit), of the product to 48 bits: its rounding to 24 would be an error of |x unit| 2^-24
// of the result, more than those of the exponential itself from |x unit| = 2 on.
__device__ __forceinline__ float exp2_exact(float x, Unit unit) {
  const float y = x * unit.hi;
  // (past fp32's range nothing is left, or infinity: any number will do beside an exponential
  // of 0)
  const float left =
      __builtin_amdgcn_fmed3f(fmaf(x, unit.rest, fmaf(x, unit.hi, -y)), -1.f, 1.f);
  const float e = exp2_fast(y);
  return fmaf(e, left * 0.693147180559945309f, e);
}

// ---- bf16 rows -----------------------------------------------------------------

struct Bf16Rows {
  static constexpr int kWaves = 2;    // per SIMD: up to 256 registers each
  using Elem = uint16_t;
  using Block = BlockRegs;
  using Channels = RowChannels;
  struct Query {
    static constexpr int kLoads = 4;
    bf16x8 q[4];
    static __device__ __forceinline__ int channel(int i, int grp) { return 32 * i + 8 * grp; }
    __device__ __forceinline__ void set(const u32x4 (&raw)[4], bool real) {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const u32x4 z = {0u, 0u, 0u, 0u};
        q[s] = as_bf16x8(real ? raw[s] : z);
      }
    }
  };

  static __device__ __forceinline__ void load(Block& b, const Pools& p, int64_t row,
                                              const LaneMap& lm) {
    load_block(b, static_cast<const uint16_t*>(p.k) + row * kHeadDim,
               static_cast<const uint16_t*>(p.v) + row * kHeadDim, 0, lm);
  }
  // The step's pair, as bf16 in LDS: a lane's two channels of each (called by one whole
  // wavefront, which reads the other lanes' once they are staged_in_wave).
  struct New {
    uint16_t k[kHeadDim], v[kHeadDim];
    using Two = uint32_t;      // a lane's two channels
    __device__ __forceinline__ void stage(uint32_t wk, uint32_t wv) {
      const int lane = threadIdx.x & 63;
      __builtin_memcpy(k + 2 * lane, &wk, 4);
      __builtin_memcpy(v + 2 * lane, &wv, 4);
    }
    // .. at row `at` of the block, zeros above it
    __device__ __forceinline__ void patch(Block& b, int at, const LaneMap& lm) const {
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (lm.krow[t] == at) {
#pragma unroll
          for (int s = 0; s < 4; ++s) b.k[t][s] = ld16(k + lm.kcol + 32 * s);
        }
      const int r = at - lm.vrow;
      if (r < 8) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          uint16_t e8[8];
          __builtin_memcpy(e8, &b.v[u], 16);
          const uint16_t x = v[16 * u + lm.vch];
#pragma unroll
          for (int e = 0; e < 8; ++e) e8[e] = e < r ? e8[e] : e == r ? x : uint16_t(0);
          __builtin_memcpy(&b.v[u], e8, 16);
        }
      }
    }
    __device__ __forceinline__ void append(const AttnLaunch& a, int64_t row,
                                           uint8_t*, uint8_t*) const {
      const int lane = threadIdx.x & 63;
      uint16_t* kp = static_cast<uint16_t*>(a.kpool);
      uint16_t* vp = static_cast<uint16_t*>(a.vpool);
      for (int c = lane; c < kHeadDim; c += 64) {
        kp[row * kHeadDim + c] = k[c];
        vp[(row & ~int64_t(7)) * kHeadDim + c * 8 + (row & 7)] = v[c];
      }
    }
  };
  // compute_block in two: what is done to the scores stands between
  static __device__ __forceinline__ void scores(const Block& b, const Query& q, float (&x)[8]) {
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(b.k[0][s]), q.q[s], s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(b.k[1][s]), q.q[s], s1, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = s0[i];
      x[4 + i] = s1[i];
    }
  }
  static __device__ __forceinline__ void attend(Softmax& st, const Block& b, const float (&x)[8],
                                                Unit by) {
    const float unit = by.hi;
    float bm = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) bm = fmaxf(bm, x[e]);
    const float mn = fmaxf(st.m, max_over_groups(bm));
    const float alpha = exp2_fast((st.m - mn) * unit);
    // P = hi + lo, both bf16, so the weights keep ~16 significant bits through
    // the bf16 MFMA (the remainder of a bf16 rounding is exact in fp32)
    bf16x8 p_hi, p_lo;
    float psum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float pf = exp2_fast((x[e] - mn) * unit);
      const __bf16 hi = static_cast<__bf16>(pf);
      p_hi[e] = hi;
      p_lo[e] = static_cast<__bf16>(pf - static_cast<float>(hi));
      psum += pf;
    }
    st.l = st.l * alpha + psum;
    st.m = mn;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      st.acc[u] *= alpha;
      st.acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(b.v[u]), p_hi, st.acc[u], 0, 0, 0);
      st.acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(b.v[u]), p_lo, st.acc[u], 0, 0, 0);
    }
  }
  static __device__ __forceinline__ void compute(Softmax& st, const Block& b, const Query& q,
                                                 float scale_log2, int limit) {
    compute_block(st, b, q.q, scale_log2, limit);
  }
  // The values of the keys whose bit is set in `hidden` (of the lane's eight) as zeros.
  static __device__ __forceinline__ void hide(Block& b, uint32_t hidden) {
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      uint16_t e8[8];
      __builtin_memcpy(e8, &b.v[u], 16);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if ((hidden >> e) & 1u) e8[e] = 0;
      __builtin_memcpy(&b.v[u], e8, 16);
    }
  }
};

// ---- e4m3 rows -------------------------------------------------------------------

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// A lane's 16-byte loads hold 16 channels of a key row, and two channels of a value
// tile, the operands of two output tiles: output tile 2u + h is channels 32u + 2 *
// (its row) + h.
struct E4m3Block {
  u32x4 k[2][2];     // [S tile][64 channels]
  u32x4 v[4];        // [32 channels]
  uint64_t vs;       // scale bytes of the lane's eight values' rows
  uint64_t ks;       // .. of eight key rows, its two among them (key_byte, + 4)
};

struct E4m3Rows {
  static constexpr int kWaves = 3;    // per SIMD: up to 168 registers each
  using Elem = uint16_t;
  using Block = E4m3Block;
  struct Channels {
    static __device__ __forceinline__ int first(int u, int grp) {
      return 32 * (u >> 1) + 8 * grp + 4 * (u & 1);
    }
  };

  // The query as it is, but for infinities, which count as the largest bf16 number.
  struct Query {
    static constexpr int kLoads = 4;
    bf16x8 q[4];
    static __device__ __forceinline__ int channel(int i, int grp) {
      return 64 * (i >> 1) + 16 * grp + 8 * (i & 1);
    }
    __device__ __forceinline__ void set(const u32x4 (&raw)[4], bool real) {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t u = real ? raw[s][i] : 0u;
          if ((u & 0x7fffu) == 0x7f80u) u -= 1u;
          if ((u & 0x7fff0000u) == 0x7f800000u) u -= 0x10000u;
          w[i] = u;
        }
        q[s] = as_bf16x8(w);
      }
    }
  };

  // bit of a lane's first key row's byte in Block::ks
  static __device__ __forceinline__ int key_shift() { return 8 * (threadIdx.x & 3); }

  static __device__ __forceinline__ void load(Block& b, const Pools& p, int64_t row,
                                              const LaneMap& lm) {
    const uint8_t* K = static_cast<const uint8_t*>(p.k) + row * kHeadDim;
    const uint8_t* V = static_cast<const uint8_t*>(p.v) + row * kHeadDim;
    b.ks = *reinterpret_cast<const uint64_t*>(p.k_scale + row + (lm.krow[0] & ~7));
    b.vs = *reinterpret_cast<const uint64_t*>(p.v_scale + row + lm.vrow);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < 2; ++s)
        b.k[t][s] = ld16(K + lm.krow[t] * kHeadDim + 2 * lm.kcol + 64 * s);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      b.v[u] = ld16_stream(V + lm.vrow * kHeadDim + (32 * u + 2 * lm.vch) * 8);
  }

  struct New {
    uint8_t k[kHeadDim], v[kHeadDim];
    using Two = uint32_t;      // a lane's two channels
    uint32_t ks, vs;
    // quantised as it is written, and attended as it is held
    __device__ __forceinline__ void stage(uint32_t wk, uint32_t wv) {
      const int lane = threadIdx.x & 63;
      uint32_t mk = max(row_magnitude(bf16_low(wk)), row_magnitude(bf16_high(wk)));
      uint32_t mv = max(row_magnitude(bf16_low(wv)), row_magnitude(bf16_high(wv)));
      const uint32_t bk = e4m3_scale_byte(max_over_groups(max_over_row16(mk)));
      const uint32_t bv = e4m3_scale_byte(max_over_groups(max_over_row16(mv)));
      const float ik = e4m3_inverse(bk), iv = e4m3_inverse(bv);
      const uint32_t ck = e4m3_pack2<false>(e4m3_clamp(bf16_low(wk) * ik, bk),
                                            e4m3_clamp(bf16_high(wk) * ik, bk), 0u);
      const uint32_t cv = e4m3_pack2<false>(e4m3_clamp(bf16_low(wv) * iv, bv),
                                            e4m3_clamp(bf16_high(wv) * iv, bv), 0u);
      __builtin_memcpy(k + 2 * lane, &ck, 2);
      __builtin_memcpy(v + 2 * lane, &cv, 2);
      if (lane == 0) {
        ks = bk;
        vs = bv;
      }
    }
    __device__ __forceinline__ void patch(Block& b, int at, const LaneMap& lm) const {
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (lm.krow[t] == at) {
          const int bit = key_shift() + 32 * t;
          b.ks = (b.ks & ~(uint64_t(255) << bit)) | static_cast<uint64_t>(ks) << bit;
#pragma unroll
          for (int s = 0; s < 2; ++s) b.k[t][s] = ld16(k + 2 * lm.kcol + 64 * s);
        }
      const int r = at - lm.vrow;
      if (r < 8) {
        const int n = r < 0 ? 0 : r;                     // cached rows of the tile
        const uint64_t below = (uint64_t(1) << (8 * n)) - 1;
        b.vs = (b.vs & below) | (r >= 0 ? static_cast<uint64_t>(vs) << (8 * n) : 0);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          uint64_t w[2];
          __builtin_memcpy(w, &b.v[u], 16);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint64_t x = v[32 * u + 2 * lm.vch + h];
            w[h] = (w[h] & below) | (r >= 0 ? x << (8 * n) : 0);
          }
          __builtin_memcpy(&b.v[u], w, 16);
        }
      }
    }
    __device__ __forceinline__ void append(const AttnLaunch& a, int64_t row,
                                           uint8_t* k_scale, uint8_t* v_scale) const {
      const int lane = threadIdx.x & 63;
      uint8_t* kp = static_cast<uint8_t*>(a.kpool);
      uint8_t* vp = static_cast<uint8_t*>(a.vpool);
      uint16_t two;
      __builtin_memcpy(&two, k + 2 * lane, 2);
      __builtin_memcpy(kp + row * kHeadDim + 2 * lane, &two, 2);
      for (int c = lane; c < kHeadDim; c += 64)
        vp[(row & ~int64_t(7)) * kHeadDim + c * 8 + (row & 7)] = v[c];
      if (lane == 0) {
        k_scale[row] = static_cast<uint8_t>(ks);
        v_scale[row] = static_cast<uint8_t>(vs);
      }
    }
  };

  // Eight codes times a power of two as bf16 numbers.
  static __device__ __forceinline__ bf16x8 to_bf16(uint32_t w0, uint32_t w1, float scale) {
    union {
      bf16x2 h[4];
      bf16x8 v;
    } r;
    r.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false);
    r.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true);
    r.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false);
    r.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true);
    return r.v;
  }

  // compute_block over the values that the rows stand for, which bf16 holds: a key's
  // scale goes into its conversion, a value's into its weight.
  // The scores take bf16 products, not the matrix cores' 8-bit ones (with the query in
  // three E4M3 parts), since those cut the products of a group off about 2^-12 below the
  // largest: sums of 128 random ones were off by up to 2.9e-4 of the largest product (bf16
  // products 7e-7), the weights of equal scores by up to 7e-4.  Nor were they faster
  // (microseconds per layer in a graph, 8-bit products and these: 2 heads of 200 rows 6.4
  // and 5.7, 8 of 2,200 10.5 and 9.7, 64 of 9,000 34.9 and 34.6, 512 of 9,000 209 both).
  static __device__ __forceinline__ void scores(const Block& b, const Query& q, float (&x)[8]) {
    f32x4 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float scale =
          e4m3_scale(static_cast<uint32_t>(b.ks >> (32 * t)) >> key_shift() & 255u);
      s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x4 w = b.k[t][i >> 1];
        const bf16x8 k = i & 1 ? to_bf16(w.z, w.w, scale) : to_bf16(w.x, w.y, scale);
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q.q[i], s[t], 0, 0, 0);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = s[0][i];
      x[4 + i] = s[1][i];
    }
  }
  static __device__ __forceinline__ void attend(Softmax& st, const Block& b, const float (&x)[8],
                                                Unit by) {
    const float unit = by.hi;
    float bm = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) bm = fmaxf(bm, x[e]);
    const float mn = fmaxf(st.m, max_over_groups(bm));
    const float alpha = exp2_fast((st.m - mn) * unit);
    // weights times their values' scales as hi + lo, both bf16 (16 significant bits)
    bf16x8 p_hi, p_lo;
    float psum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float pf = exp2_fast((x[e] - mn) * unit);
      const uint32_t w = static_cast<uint32_t>(b.vs >> (32 * (e >> 2)));
      const float pv = pf * e4m3_scale(w >> (8 * (e & 3)) & 255u);
      const __bf16 hi = static_cast<__bf16>(pv);
      p_hi[e] = hi;
      p_lo[e] = static_cast<__bf16>(pv - static_cast<float>(hi));
      psum += pf;
    }
    st.l = st.l * alpha + psum;
    st.m = mn;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const u32x4 w = b.v[u >> 1];
      const bf16x8 v = u & 1 ? to_bf16(w.z, w.w, 1.f) : to_bf16(w.x, w.y, 1.f);
      st.acc[u] *= alpha;
      st.acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p_hi, st.acc[u], 0, 0, 0);
      st.acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p_lo, st.acc[u], 0, 0, 0);
    }
  }
  static __device__ __forceinline__ void compute(Softmax& st, const Block& b, const Query& q,
                                                 float scale_log2, int limit) {
    float x[8];
    scores(b, q, x);
    const int grp = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= scale_log2;
    if (limit < 32) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (8 * grp + e >= limit) x[e] = kNegInf;
    }
    attend(st, b, x, Unit{1.f, 0.f});
  }
  // The values of the keys whose bit is set in `hidden` (of the lane's eight) as zeros.
  static __device__ __forceinline__ void hide(Block& b, uint32_t hidden) {
    uint64_t kept = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (!((hidden >> e) & 1u)) kept |= uint64_t(255) << (8 * e);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      uint64_t w[2];
      __builtin_memcpy(w, &b.v[u], 16);
      w[0] &= kept;
      w[1] &= kept;
      __builtin_memcpy(&b.v[u], w, 16);
    }
  }

  // tiles 2u and 2u + 1 hold alternate channels: to runs of four
  static __device__ __forceinline__ void gather_channels(Softmax& st) {
#pragma unroll
    for (int u = 0; u < 8; u += 2) {
      const f32x4 a = st.acc[u], b = st.acc[u + 1];
      st.acc[u] = f32x4{a[0], b[0], a[1], b[1]};
      st.acc[u + 1] = f32x4{a[2], b[2], a[3], b[3]};
    }
  }
};

// ---- fp32 rows -------------------------------------------------------------------

// The lanes' keys are those of the bf16 rows (LaneMap); every product is an fp32 one,
// four channels, or four keys, to an instruction.
struct F32Block {
  u32x4 k[2][8];     // [S tile][16 channels]: the lane's four of them
  u32x4 v[8][2];     // [16-channel tile][four of the lane's eight keys]
};

struct F32Rows {
  static constexpr int kWaves = 1;    // per SIMD: up to 512 registers each
  using Elem = float;
  using Block = F32Block;
  using Channels = RowChannels;
  struct Query {
    static constexpr int kLoads = 8;
    f32x4 q[8];
    static __device__ __forceinline__ int channel(int i, int grp) { return 16 * i + 4 * grp; }
    __device__ __forceinline__ void set(const u32x4 (&raw)[8], bool real) {
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        const u32x4 w = real ? raw[s] : u32x4{0u, 0u, 0u, 0u};
        __builtin_memcpy(&q[s], &w, 16);
      }
    }
  };

  static __device__ __forceinline__ void load(Block& b, const Pools& p, int64_t row,
                                              const LaneMap& lm) {
    const float* K = static_cast<const float*>(p.k) + row * kHeadDim;
    const float* V = static_cast<const float*>(p.v) + row * kHeadDim;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < 8; ++s)
        b.k[t][s] = ld16(K + lm.krow[t] * kHeadDim + 16 * s + lm.kcol / 2);
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        b.v[u][h] = ld16_stream(V + lm.vrow * kHeadDim + (16 * u + lm.vch) * 8 + 4 * h);
  }

  struct New {
    float k[kHeadDim], v[kHeadDim];
    using Two = uint64_t;      // a lane's two channels
    __device__ __forceinline__ void stage(Two wk, Two wv) {
      const int lane = threadIdx.x & 63;
      __builtin_memcpy(k + 2 * lane, &wk, 8);
      __builtin_memcpy(v + 2 * lane, &wv, 8);
    }
    __device__ __forceinline__ void patch(Block& b, int at, const LaneMap& lm) const {
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (lm.krow[t] == at) {
#pragma unroll
          for (int s = 0; s < 8; ++s) b.k[t][s] = ld16(k + 16 * s + lm.kcol / 2);
        }
      const int r = at - lm.vrow;
      if (r < 8) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const uint32_t x = __float_as_uint(v[16 * u + lm.vch]);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            uint32_t& w = reinterpret_cast<uint32_t(&)[4]>(b.v[u][e >> 2])[e & 3];
            w = e < r ? w : e == r ? x : 0u;
          }
        }
      }
    }
    __device__ __forceinline__ void append(const AttnLaunch& a, int64_t row, uint8_t*,
                                           uint8_t*) const {
      const int lane = threadIdx.x & 63;
      float* kp = static_cast<float*>(a.kpool);
      float* vp = static_cast<float*>(a.vpool);
      for (int c = lane; c < kHeadDim; c += 64) {
        kp[row * kHeadDim + c] = k[c];
        vp[(row & ~int64_t(7)) * kHeadDim + c * 8 + (row & 7)] = v[c];
      }
    }
  };

  static __device__ __forceinline__ float word(const u32x4& w, int i) {
    return __uint_as_float(w[i]);
  }
  // Eight sums of 16 channels each, then theirs in pairs: a chain of all 128 rounds partial
  // sums as large as the score 128 times, and left outputs and weights off by 1.6 to 3.6 times
  // what torch's sums in fp32 do, these by 0.8 to 1.3 times.  Bound by the matrix cores and by
  // latency (microseconds per layer in a captured step, the chain and the eight sums: 2 heads of
  // 200 rows 9.8 and 9.9, 8 of 600 13.6 and 13.9, of 2,200 16.9 and 17.4, 64 of 600 19.3 and 19.8,
  // of 2,000 33.8 and 34.5, 256 of 900 51.6 and 52.5; of 4,000 the same).
  static __device__ __forceinline__ void scores(const Block& b, const Query& q, float (&x)[8]) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x4 s[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          s[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(word(b.k[t][i], e), q.q[i][e], s[i], 0, 0, 0);
      const f32x4 sum = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * t + i] = sum[i];
    }
  }
  static __device__ __forceinline__ void attend(Softmax& st, const Block& b, const float (&x)[8],
                                                Unit unit) {
    float bm = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) bm = fmaxf(bm, x[e]);
    const float mn = fmaxf(st.m, max_over_groups(bm));
    const float alpha = exp2_fast((st.m - mn) * unit.hi);
    float p[8], psum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      p[e] = exp2_exact(x[e] - mn, unit);
      psum += p[e];
    }
    st.l = st.l * alpha + psum;
    st.m = mn;
    // product e takes key 8 * grp + e of each group of lanes; a block's sum is made by itself, so
    // that the running one is rounded once a block
    f32x4 sum[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) sum[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int u = 0; u < 8; ++u)
        sum[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(word(b.v[u][e >> 2], e & 3), p[e], sum[u], 0,
                                                      0, 0);
#pragma unroll
    for (int u = 0; u < 8; ++u) st.acc[u] = st.acc[u] * alpha + sum[u];
  }
  static __device__ __forceinline__ void hide(Block& b, uint32_t hidden) {
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if ((hidden >> e) & 1u) b.v[u][e >> 2][e & 3] = 0u;
  }
};

}  // namespace
}  // namespace ra
