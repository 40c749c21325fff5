// Decode attention over blocks of 32 cached rows: every block of an e4m3 cache, or
// in a block-sparse step the blocks chosen for each KV head and the recent ones, of
// a bf16 or an e4m3 cache.  The mathematics is that of attention.hip: one pass with
// an online softmax, S^T = K Q^T and O^T += V^T P^T on the matrix cores, the weights
// in two bf16 parts, the step's new pair attended and appended.
//
// The blocks that a (sequence, KV head) attends to are numbered 0 .. n - 1
// (attended_blocks); a workgroup takes a run of them, its W wavefronts a W-th of the
// run each.  The last block holds the step's new row: it is read like any other (it
// lies inside the head's region or page), and the wavefront that owns it puts the
// new pair in its place and zeros above it.
#include "attn_parts.h"
#include "block_choice.h"
#include "e4m3.h"

namespace ra {
namespace {

struct BlockWork : Work {
  int b0, b1;        // the workgroup's attended blocks
  int n;             // attended blocks of the head
  int cand;          // candidate blocks
  int chosen;        // the first `chosen` come from the list ..
  int shift;         // .. and block i after them is cached block i + shift
};

template <bool LIST>
__device__ __forceinline__ BlockWork locate_blocks(const AttnLaunch& a, const BlockChoice& ch,
                                                   const SlotOrder& order, int Hkv,
                                                   const Paging& pg) {
  BlockWork w;
  w.split = blockIdx.x;
  w.g = blockIdx.y;
  w.slot = order.n ? order.slot[blockIdx.z] : blockIdx.z;
  const SeqMeta& M = a.meta[w.slot];
  w.valid = false;
  if (!M.active) return w;
  w.len = M.len;
  w.n_keys = w.len + 1;
  w.cand = w.chosen = w.shift = 0;
  if constexpr (LIST) {
    w.cand = candidate_blocks(w.len, ch.recent);
    if (w.cand > ch.n_blocks) {
      w.chosen = ch.n_blocks;
      w.shift = w.cand - ch.n_blocks;
    }
  }
  w.n = w.len / kBlockRows + 1 - w.shift;
  const int per = a.split_keys / kBlockRows;
  w.b0 = w.split * per;
  if (w.b0 >= w.n) return w;
  w.b1 = min(w.b0 + per, w.n);
  w.nsplit = (w.n + per - 1) / per;
  w.rm = row_map(M, w.slot, a.layer * Hkv + w.g, pg);
  w.valid = true;
  return w;
}

// Splits of a head, for the merge.
struct BlockSplits {
  int recent, n_blocks, at;
  __device__ __forceinline__ int slot() const { return at; }
  __device__ __forceinline__ int operator()(const AttnLaunch& a, int slot) const {
    const int per = a.split_keys / kBlockRows;
    return (attended_blocks(a.meta[slot].len, recent, n_blocks) + per - 1) / per;
  }
};

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

// ---- bf16 rows -----------------------------------------------------------------

struct Bf16Rows {
  static constexpr int kWaves = 2;    // per SIMD: up to 256 registers each
  using Block = BlockRegs;
  using Channels = RowChannels;
  struct Query {
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
  static __device__ __forceinline__ void compute(Softmax& st, const Block& b, const Query& q,
                                                 float scale_log2, int limit) {
    compute_block(st, b, q.q, scale_log2, limit);
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
  using Block = E4m3Block;
  struct Channels {
    static __device__ __forceinline__ int first(int u, int grp) {
      return 32 * (u >> 1) + 8 * grp + 4 * (u & 1);
    }
  };

  // The query as it is, but for infinities, which count as the largest bf16 number.
  struct Query {
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
  static __device__ __forceinline__ void compute(Softmax& st, const Block& b, const Query& q,
                                                 float scale_log2, int limit) {
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
    const int grp = (threadIdx.x & 63) >> 4;
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = s[0][i] * scale_log2;
      x[4 + i] = s[1][i] * scale_log2;
    }
    if (limit < 32) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (8 * grp + e >= limit) x[e] = kNegInf;
    }
    float bm = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) bm = fmaxf(bm, x[e]);
    const float mn = fmaxf(st.m, max_over_groups(bm));
    const float alpha = exp2_fast(st.m - mn);
    // weights times their values' scales as hi + lo, both bf16 (16 significant bits)
    bf16x8 p_hi, p_lo;
    float psum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float pf = exp2_fast(x[e] - mn);
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

// W wavefronts (four) per workgroup, two register buffers of a block each (three and
// four, and eight or twelve wavefronts, measured no faster), within 168 registers for
// e4m3 rows, so that three workgroups fit a CU.  Bound by HBM where the rows are many:
// 256 heads of 9,216 e4m3 rows 94 to 99 us (6.2 to 6.5 TB/s), of 8,250 in a decode window
// 88 us, where the bf16 launch takes 167; 256 heads attending to 38 of 288 bf16 blocks 28 us
// (5.7 TB/s) and 8 us for the choice.  Bound by latency where they are few: 8 heads of
// 2,200 rows 9.3 us (slot record, rows, partials out, counter, partials in), two of 200
// 5.7.
template <typename R, int W, int MINW, bool PAGED, bool LIST>
__global__ __launch_bounds__(64 * W, MINW) void attn_blocks_kernel(
    AttnLaunch a, BlockChoice ch, SlotOrder order, Paging pg, uint8_t* k_scale, uint8_t* v_scale,
    int G, int Hq, int Hkv, float scale_log2) {
  __shared__ float s_m[W][kMaxGroup];
  __shared__ float s_l[W][kMaxGroup];
  __shared__ float s_o[W][kMaxGroup][kHeadDim];
  __shared__ __align__(16) typename R::New s_new;
  const BlockWork w = locate_blocks<LIST>(a, ch, order, Hkv, pg);
  if (!w.valid) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, qi = lane & 15, grp = lane >> 4;
  const LaneMap lm = lane_map();
  const Pools pools{a.kpool, a.vpool, k_scale, v_scale};
  const int per = (w.b1 - w.b0 + W - 1) / W;
  const int b0 = __builtin_amdgcn_readfirstlane(w.b0 + wave * per);
  const int b1 = __builtin_amdgcn_readfirstlane(min(b0 + per, w.b1));
  const bool has = b0 < b1;
  const bool owns_last = has && b1 == w.n;
  // the chosen blocks: of few candidates, chosen here (by every split, alike), else by
  // the launch before
  int32_t* list = nullptr;
  __shared__ uint32_t s_keys[LIST ? kFusedBlocks : 1];
  __shared__ int32_t s_list[LIST ? kFusedBlocks : 1];
  __shared__ int32_t s_table[LIST && PAGED ? kFusedBlocks : 1];   // the candidates' pages
  const bool fused = LIST && w.chosen > 0 && w.cand <= kFusedBlocks;
  // first pool row of a candidate block
  const auto candidate_row = [&](int b) -> int64_t {
    if constexpr (PAGED) {
      const int shift = w.rm.page_shift - kBlockShift;
      return s_table[b >> shift] * w.rm.group_rows + w.rm.head_off +
             ((b & ((1 << shift) - 1)) << kBlockShift);
    } else {
      return w.rm.region + b * kBlockRows;
    }
  };
  if constexpr (LIST) {
    list = ch.list + (static_cast<int64_t>(w.slot) * Hkv + w.g) * ch.stride;
    if (fused) {
      if constexpr (PAGED) {
        const int pages = ((w.cand - 1) >> (w.rm.page_shift - kBlockShift)) + 1;
        for (int i = threadIdx.x; i < pages; i += 64 * W) s_table[i] = w.rm.table[i];
        __syncthreads();
      }
      score_blocks<64 * W>(s_keys, 0, w.cand, candidate_row, ch.bounds, ch.units,
                           static_cast<const uint16_t*>(a.q) +
                               (static_cast<int64_t>(w.slot) * Hq + w.g * G) * kHeadDim, G);
      __syncthreads();
      if (wave == 0) choose_few(s_keys, w.cand, w.chosen, s_list);
      __syncthreads();
      if (w.split == 0)
        for (int i = threadIdx.x; i < w.chosen; i += 64 * W) list[i] = s_list[i];
    }
  }
  const auto load = [&](typename R::Block& b, int i) {
    int64_t row;
    if (fused && i < w.chosen) {
      row = candidate_row(__builtin_amdgcn_readfirstlane(s_list[i]));
    } else {
      int cached = i + w.shift;
      if constexpr (LIST) {
        if (i < w.chosen) cached = __builtin_amdgcn_readfirstlane(list[i]);
      }
      row = pool_row<PAGED>(w.rm, cached * kBlockRows);
    }
    R::load(b, pools, row, lm);
  };

  Softmax st;
  st.m = kNoScore;
  st.l = 0.f;
#pragma unroll
  for (int u = 0; u < 8; ++u) st.acc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (has) {
    // the queries and the new pair first: they are made ready while the rows arrive
    const uint16_t* qrow = static_cast<const uint16_t*>(a.q) +
                           (static_cast<int64_t>(w.slot) * Hq + w.g * G + (qi < G ? qi : 0)) * kHeadDim;
    u32x4 raw[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) raw[s] = ld16(qrow + R::Query::channel(s, grp));
    uint32_t new_k = 0, new_v = 0;
    if (owns_last) {
      const int64_t src = (static_cast<int64_t>(w.slot) * Hkv + w.g) * (kHeadDim / 2) + lane;
      new_k = static_cast<const uint32_t*>(a.k_new)[src];
      new_v = static_cast<const uint32_t*>(a.v_new)[src];
    }
    const int last = b1 - 1;
    typename R::Block x0, x1;
    load(x0, b0);
    load(x1, min(b0 + 1, last));
    typename R::Query q;
    q.set(raw, qi < G);
    if (owns_last) {
      s_new.stage(new_k, new_v);
      staged_in_wave();
    }
    // two register buffers in turn; every prefetch is issued (the last block's again
    // once there is none left), so that the wait for a block leaves the next one's
    // loads in flight
    int i = b0;
    for (; i + 1 < last; i += 2) {
      R::compute(st, x0, q, scale_log2, 32);
      load(x0, min(i + 2, last));
      R::compute(st, x1, q, scale_log2, 32);
      load(x1, min(i + 3, last));
    }
    if (i < last) {
      R::compute(st, x0, q, scale_log2, 32);
      x0 = x1;
    }
    int limit = 32;
    if (owns_last) {
      const int at = w.len % kBlockRows;
      s_new.patch(x0, at, lm);
      limit = at + 1;
    }
    R::compute(st, x0, q, scale_log2, limit);
    st.l += __shfl_xor(st.l, 16, 64);
    st.l += __shfl_xor(st.l, 32, 64);
  }
  if constexpr (!std::is_same_v<R, Bf16Rows>) R::gather_channels(st);
  finish_item<uint16_t, W, true, BlockSplits, typename R::Channels>(
      a, w, wave, qi, grp, st, G, Hq, Hkv, s_m, s_l, s_o,
      LIST ? BlockSplits{ch.recent, ch.n_blocks, w.slot} : BlockSplits{0, 1 << 30, w.slot});
  if (owns_last) {
    const int64_t row = pool_row<PAGED>(w.rm, w.len);
    s_new.append(a, row, k_scale, v_scale);
    if (lane == 0) a.pos[row] = a.meta[w.slot].prompt_len + a.meta[w.slot].step;
  }
}

template <typename R, bool PAGED, bool LIST>
void launch_blocks(const Shape& sh, const AttnLaunch& a, const BlockChoice& ch, hipStream_t s) {
  const SlotOrder order = sh.order ? *sh.order : SlotOrder{};
  const dim3 grid(a.max_splits, sh.Hkv, order.n ? order.n : a.max_seqs);
  const float scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(kHeadDim));
  hipLaunchKernelGGL((attn_blocks_kernel<R, 4, R::kWaves, PAGED, LIST>), grid, dim3(256), 0, s, a,
                     ch, order, sh.pg, sh.k_scale, sh.v_scale, sh.G, sh.Hq, sh.Hkv, scale_log2);
}

}  // namespace

hipError_t launch_attention_e4m3(const Shape& sh, const AttnLaunch& a, hipStream_t s) {
  const BlockChoice none{};
  if (sh.pg.tables) launch_blocks<E4m3Rows, true, false>(sh, a, none, s);
  else launch_blocks<E4m3Rows, false, false>(sh, a, none, s);
  return hipGetLastError();
}

hipError_t launch_block_attention(const Shape& sh, const AttnLaunch& a, const BlockChoice& ch,
                                  hipStream_t s) {
  if (sh.dtype == 2) {
    if (sh.pg.tables) launch_blocks<E4m3Rows, true, true>(sh, a, ch, s);
    else launch_blocks<E4m3Rows, false, true>(sh, a, ch, s);
  } else {
    if (sh.pg.tables) launch_blocks<Bf16Rows, true, true>(sh, a, ch, s);
    else launch_blocks<Bf16Rows, false, true>(sh, a, ch, s);
  }
  return hipGetLastError();
}

}  // namespace ra
