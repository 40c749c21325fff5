// Decode attention whose scores follow a rule (ra_score_rule), and the accumulated weights
// of the rows it attends to.  The attention is that of attn_blocks.hip, over the blocks
// that may hold rows within the window:
//   s = scale q.k;  s = cap tanh(s / cap);  s -= slope * (p_new - p_j);
//   s = -inf where p_new - p_j >= window and p_j >= prefix
// with p the cached positions, so the rule means the same before and after evictions.
// A weight p_hj = exp(s_hj - m_h) / l_h needs the head's maximum and sum, which are known
// after its last row, so the scores are kept until then: in LDS where a workgroup takes a
// whole head, as many as fit, else in the workspace (G floats per row, 20 bytes beside the 512
// of a bf16 row at G = 5).  Those of a head in splits are added up by add_weights_kernel.
#include "attn_rows.h"

namespace ra {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

struct BiasedWork : Work {
  int b0, b1;          // the workgroup's blocks of those attended
  WindowBlocks win;
  int now;             // position of the new row
};

__device__ __forceinline__ BiasedWork locate_biased(const AttnLaunch& a, const BiasLaunch& bias,
                                                    const SlotOrder& order, int Hkv,
                                                    const Paging& pg) {
  BiasedWork w;
  w.split = blockIdx.x;
  w.g = blockIdx.y;
  w.slot = order.n ? order.slot[blockIdx.z] : blockIdx.z;
  const SeqMeta& M = a.meta[w.slot];
  w.valid = false;
  if (!M.active) return w;
  w.len = M.len;
  w.n_keys = w.len + 1;
  w.now = M.prompt_len + M.step;
  w.win = window_blocks(w.len, bias.ordered ? bias.window : 0, bias.prefix);
  const int per = a.split_keys / kBlockRows;
  w.b0 = w.split * per;
  if (w.b0 >= w.win.n) return w;
  w.b1 = min(w.b0 + per, w.win.n);
  w.nsplit = (w.win.n + per - 1) / per;
  w.rm = row_map(M, w.slot, a.layer * Hkv + w.g, pg);
  w.valid = true;
  return w;
}

// Splits of a head, for the merge.
struct BiasedSplits {
  int at, n;
  __device__ __forceinline__ int slot() const { return at; }
  __device__ __forceinline__ int operator()(const AttnLaunch&, int) const { return n; }
};

// What becomes of the weights: not kept, added up by a launch of its own, or at once, from
// scores in LDS or in LDS and the workspace both.
constexpr int kNoWeights = 0, kWeighAfter = 1, kWeighHere = 2, kWeighBoth = 3;

// The units of the scores; with KEEP each query's maximum and sum of a head.
template <bool KEEP, bool EXACT>
struct RuleEnds {
  static constexpr bool kKeeps = KEEP;
  Unit unit;
  float* to;       // [G][2]
  __device__ __forceinline__ float exp2(float x) const {
    return EXACT ? exp2_exact(x, unit) : exp2f(x * unit.hi);
  }
  __device__ __forceinline__ void keep(int q, float m, float l) const {
    to[2 * q] = m;
    to[2 * q + 1] = l;
  }
};

// tanh y, to about an ulp: up to 1 as y less a correction of at most a quarter of it,
// tanh y = y - y^3 (45045 + 2772 y^2 + 27 y^4) / (135135 + 62370 y^2 + 3150 y^4 + 28 y^6)
// (the convergent of its continued fraction y / (1 + y^2 / (3 + y^2 / (5 + ..))) that ends
// with 13), past it as 1 - 2 / (1 + e^2y), where the quotient is a quarter at most.  Both are
// made and one is taken: the empty asm keeps the compiler from branching around either,
// sixteen times a block.
__device__ __forceinline__ float tanh_of(float y) {
  const float a = fabsf(y), y2 = y * y;
  const float num = 45045.f + y2 * (2772.f + y2 * 27.f);
  const float den = 135135.f + y2 * (62370.f + y2 * (3150.f + y2 * 28.f));
  float near = y - y * y2 * num * __builtin_amdgcn_rcpf(den);
  float far = 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + exp2_fast(a * (2.f * kLog2e)));
  asm("" : "+v"(near), "+v"(far));
  return a > 1.f ? copysignf(far, y) : near;
}

// First pool row of a cached block.  The tables do not change while the kernel runs, and
// their entries come by scalar loads: a vector load, which the compiler takes because the
// kernel also stores, would wait for every row in flight (192 heads of 6,200 paged e4m3
// rows, with weights: 154 us).
template <bool PAGED>
__device__ __forceinline__ int64_t block_row(const RowMap& m, int block) {
  if constexpr (PAGED) {
    typedef const int32_t __attribute__((address_space(4)))* ConstantTable;
    const int j = __builtin_amdgcn_readfirstlane(block) * kBlockRows;
    const int64_t page = ((ConstantTable)(reinterpret_cast<uintptr_t>(m.table)))[j >> m.page_shift];
    return page * m.group_rows + m.head_off + (j & ((1 << m.page_shift) - 1));
  } else {
    return m.region + block * kBlockRows;
  }
}

// 16 bytes at an offset of a buffer, dropped past its end.
__device__ __forceinline__ void store16(__amdgpu_buffer_rsrc_t to, uint32_t offset, float a,
                                        float b, float c, float d) {
  const u32x4 v = {__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d)};
  __builtin_amdgcn_raw_buffer_store_b128(v, to, static_cast<int>(offset), 0, 0);
}

// w_j += sum over the group's queries of exp(s_j - m) / l for the four attended rows from
// `at` on, the new row's weight set.  A row's sum is made by one thread, in the order of the
// queries: the same on every run.  score4(q): their scores; stats [G][2].
struct FourRows {
  int64_t row;       // pool row of the first
  int j;             // its index; past the cached rows: nothing to do
};
template <bool PAGED>
__device__ __forceinline__ FourRows four_rows(const WindowBlocks& win, const RowMap& rm, int len,
                                              int at) {
  const int i = at / kBlockRows;
  if (i >= win.n) return {0, len + 1};
  const int j = (i < win.head ? i : i + win.shift) * kBlockRows + at % kBlockRows;
  return {j > len ? 0 : pool_row<PAGED>(rm, j), j};
}
template <bool EXACT, typename Score4>
__device__ __forceinline__ void weigh_rows(f32x4* to, f32x4 w, int j, int len, int G,
                                           const float* stats, Unit unit, Score4&& score4) {
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int q = 0; q < G; ++q) {
    const f32x4 x = score4(q);
    const float m = stats[2 * q], inv = 1.f / stats[2 * q + 1];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      sum[e] += (EXACT ? exp2_exact(x[e] - m, unit) : exp2_fast((x[e] - m) * unit.hi)) * inv;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = j + e < len ? w[e] + sum[e] : j + e == len ? sum[e] : w[e];
  *to = w;
}

// The four wavefronts of a workgroup and their register buffers as in attn_blocks_kernel.
// BYPOS: the rule has slopes or a window, and the positions are read with the rows (e4m3
// rows then take up to 256 registers, two workgroups to a CU).
template <typename R, int W, int MINW, bool PAGED, bool BYPOS, int WEIGH>
__global__ __launch_bounds__(64 * W, MINW) void attn_biased_kernel(
    AttnLaunch a, BiasLaunch bias, SlotOrder order, Paging pg, uint8_t* k_scale, uint8_t* v_scale,
    int G, int Hq, int Hkv) {
  using E = typename R::Elem;
  using Two = typename R::New::Two;
  constexpr bool kExact = std::is_same_v<R, F32Rows>;
  const Unit unit{bias.unit, bias.unit_rest};
  __shared__ float s_m[W][kMaxGroup];
  __shared__ float s_l[W][kMaxGroup];
  __shared__ __align__(16) float s_o[W][kMaxGroup][kHeadDim];
  __shared__ __align__(16) typename R::New s_new;
  constexpr bool kHere = WEIGH >= kWeighHere;
  __shared__ float s_stats[kHere ? kMaxGroup : 1][2];
  // kHere: [G][lds_stride], of each wavefront's blocks the first lds_blocks
  extern __shared__ __align__(16) float s_scores[];
  const BiasedWork w = locate_biased(a, bias, order, Hkv, pg);
  if (!w.valid) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, qi = lane & 15, grp = lane >> 4;
  const LaneMap lm = lane_map();
  const Pools pools{a.kpool, a.vpool, k_scale, v_scale};
  const int per = (w.b1 - w.b0 + W - 1) / W;
  const int b0 = __builtin_amdgcn_readfirstlane(w.b0 + wave * per);
  const int b1 = __builtin_amdgcn_readfirstlane(min(b0 + per, w.b1));
  const bool has = b0 < b1;
  const bool owns_last = has && b1 == w.win.n;
  const float slope = BYPOS && bias.slopes && qi < G ? bias.slopes[w.g * G + qi] : 0.f;

  struct Buffer {
    typename R::Block rows;
    int p[BYPOS ? 8 : 1];   // positions of the lane's eight keys
  };
  const auto load = [&](Buffer& b, int i) {
    const int cached = i < w.win.head ? i : i + w.win.shift;
    const int64_t row = block_row<PAGED>(w.rm, cached);
    R::load(b.rows, pools, row, lm);
    if constexpr (BYPOS) {
      const u32x4 lo = ld16(a.pos + row + lm.vrow), hi = ld16(a.pos + row + lm.vrow + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        b.p[e] = static_cast<int>(lo[e]);
        b.p[4 + e] = static_cast<int>(hi[e]);
      }
    }
  };
  // the scores of the head's queries, [block][G][32]
  const auto scores = __builtin_amdgcn_make_buffer_rsrc(
      bias.scores + (static_cast<int64_t>(w.slot) * Hq + w.g * G) * bias.score_stride, 0,
      static_cast<int>(4u * static_cast<uint32_t>(G * bias.score_stride)), 0x00020000);
  const uint32_t q_offset = 4u * static_cast<uint32_t>(kBlockRows * qi + 8 * grp);

  Softmax st;
  st.m = kNoScore;
  st.l = 0.f;
#pragma unroll
  for (int u = 0; u < 8; ++u) st.acc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (has) {
    // the queries and the new pair first: they are made ready while the rows arrive
    const E* qrow = static_cast<const E*>(a.q) +
                    (static_cast<int64_t>(w.slot) * Hq + w.g * G + (qi < G ? qi : 0)) * kHeadDim;
    u32x4 raw[R::Query::kLoads];
#pragma unroll
    for (int s = 0; s < R::Query::kLoads; ++s) raw[s] = ld16(qrow + R::Query::channel(s, grp));
    Two new_k = 0, new_v = 0;
    if (owns_last) {
      const int64_t src = (static_cast<int64_t>(w.slot) * Hkv + w.g) * (kHeadDim / 2) + lane;
      new_k = static_cast<const Two*>(a.k_new)[src];
      new_v = static_cast<const Two*>(a.v_new)[src];
    }
    const int last = b1 - 1;
    Buffer x0, x1;
    load(x0, b0);
    load(x1, min(b0 + 1, last));
    typename R::Query q;
    q.set(raw, qi < G);
    if (owns_last) {
      s_new.stage(new_k, new_v);
      staged_in_wave();
    }
    // block i; keys from `limit` on are masked out
    const auto step = [&](Buffer& b, int i, int limit) {
      float x[8];
      R::scores(b.rows, q, x);
      if (bias.cap > 0.f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = tanh_of(x[e] * bias.before);
      }
      if constexpr (BYPOS) {
        if (bias.slopes) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            x[e] = x[e] * bias.after - slope * static_cast<float>(w.now - b.p[e]);
        }
        uint32_t hidden = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int dist = w.now - b.p[e];
          if (bias.window > 0 && dist >= bias.window && b.p[e] >= bias.prefix) {
            x[e] = kNegInf;
            hidden |= 1u << e;
          }
        }
        // a hidden row's value has no part in the products, not even as 0 times it
        if (__ballot(hidden != 0)) R::hide(b.rows, hidden);
      }
      if (limit < 32) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (8 * grp + e >= limit) x[e] = kNegInf;
      }
      const bool in_lds = WEIGH == kWeighHere || (WEIGH == kWeighBoth && i - b0 < bias.lds_blocks);
      if constexpr (kHere) {
        if (in_lds && qi < G) {
          const int at = kBlockRows * (wave * bias.lds_blocks + i - b0) + 8 * grp;
          f32x4* to = reinterpret_cast<f32x4*>(s_scores + qi * bias.lds_stride + at);
          to[0] = f32x4{x[0], x[1], x[2], x[3]};
          to[1] = f32x4{x[4], x[5], x[6], x[7]};
        }
      }
      if constexpr (WEIGH == kWeighAfter || WEIGH == kWeighBoth) {
        // (lanes of no query write past the buffer's end, which drops them: a store that some
        // of them branched around would leave the loads in flight behind it uncounted)
        const uint32_t at = qi < G && !in_lds ? q_offset + 4u * (kBlockRows * G * i) : ~31u;
        store16(scores, at, x[0], x[1], x[2], x[3]);
        store16(scores, at + 16u, x[4], x[5], x[6], x[7]);
      }
      R::attend(st, b.rows, x, unit);
    };
    // two register buffers in turn; every prefetch is issued (the last block's again
    // once there is none left), so that the wait for a block leaves the next one's
    // loads in flight
    int i = b0;
    for (; i + 1 < last; i += 2) {
      step(x0, i, 32);
      load(x0, min(i + 2, last));
      step(x1, i + 1, 32);
      load(x1, min(i + 3, last));
    }
    if (i < last) {
      step(x0, i, 32);
      x0 = x1;
    }
    int limit = 32;
    if (owns_last) {
      const int at = w.len % kBlockRows;
      s_new.patch(x0.rows, at, lm);
      limit = at + 1;
      if constexpr (BYPOS) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (8 * grp + e >= at) x0.p[e] = w.now;
      }
    }
    step(x0, last, limit);
    st.l += __shfl_xor(st.l, 16, 64);
    st.l += __shfl_xor(st.l, 32, 64);
  }
  if constexpr (std::is_same_v<R, E4m3Rows>) R::gather_channels(st);
  const BiasedSplits splits{w.slot, w.nsplit};
  // a whole head: its first rows' weights come while the wavefronts merge
  const int first = static_cast<int>(threadIdx.x) * 4;
  FourRows rows{0, 0};
  f32x4 weights = {0.f, 0.f, 0.f, 0.f};
  RuleEnds<WEIGH != kNoWeights, kExact> ends{unit, nullptr};
  if constexpr (WEIGH == kWeighAfter)
    ends.to = bias.stats + 2 * (static_cast<int64_t>(w.slot) * Hq + w.g * G);
  if constexpr (kHere) {
    ends.to = &s_stats[0][0];
    rows = four_rows<PAGED>(w.win, w.rm, w.len, first);
    if (rows.j <= w.len) weights = *reinterpret_cast<const f32x4*>(bias.weights + rows.row);
  }
  finish_item<E, W, true, BiasedSplits, typename R::Channels>(
      a, w, wave, qi, grp, st, G, Hq, Hkv, s_m, s_l, s_o, splits, ends);
  if constexpr (kHere) {
    // (a barrier after which the workgroup's own stores are there to read, too)
    __syncthreads();
    const float* far = bias.scores + (static_cast<int64_t>(w.slot) * Hq + w.g * G) * bias.score_stride;
    for (int at = first; at < w.win.n * kBlockRows;) {
      if (rows.j <= w.len) {
        const int i = at / kBlockRows, in_block = at % kBlockRows, owner = i / per;
        const bool in_lds = WEIGH == kWeighHere || i - owner * per < bias.lds_blocks;
        const float* near =
            s_scores + kBlockRows * (owner * bias.lds_blocks + i - owner * per) + in_block;
        const float* from = far + static_cast<int64_t>(i) * G * kBlockRows + in_block;
        weigh_rows<kExact>(
            reinterpret_cast<f32x4*>(bias.weights + rows.row), weights, rows.j, w.len, G,
            &s_stats[0][0], unit, [&](int q) {
              if (in_lds) return *reinterpret_cast<const f32x4*>(near + q * bias.lds_stride);
              return *reinterpret_cast<const f32x4*>(from + q * kBlockRows);
            });
      }
      at += 4 * 64 * W;
      rows = four_rows<PAGED>(w.win, w.rm, w.len, at);
      if (rows.j <= w.len) weights = *reinterpret_cast<const f32x4*>(bias.weights + rows.row);
    }
  }
  if (owns_last) {
    const int64_t row = pool_row<PAGED>(w.rm, w.len);
    s_new.append(a, row, k_scale, v_scale);
    if (lane == 0) a.pos[row] = w.now;
  }
}

// The weights of a launch whose scores went to the workspace.  Grid: (runs of 1,024 attended
// rows, KV heads, slots), four rows to a thread.
constexpr int kWeighThreads = 256, kWeighRows = 4;
template <bool PAGED, bool EXACT>
__global__ __launch_bounds__(kWeighThreads) void add_weights_kernel(const SeqMeta* meta, int layer,
                                                                    BiasLaunch bias, Paging pg,
                                                                    int G, int Hq, int Hkv) {
  const int g = blockIdx.y, slot = blockIdx.z;
  const SeqMeta& M = meta[slot];
  if (!M.active) return;
  const int len = M.len;
  const WindowBlocks win = window_blocks(len, bias.ordered ? bias.window : 0, bias.prefix);
  const int at = (blockIdx.x * kWeighThreads + threadIdx.x) * kWeighRows;
  const FourRows rows = four_rows<PAGED>(win, row_map(M, slot, layer * Hkv + g, pg), len, at);
  if (rows.j > len) return;
  const int64_t head = static_cast<int64_t>(slot) * Hq + g * G;
  const float* s = bias.scores + head * bias.score_stride +
                   static_cast<int64_t>(at / kBlockRows) * G * kBlockRows + at % kBlockRows;
  f32x4* to = reinterpret_cast<f32x4*>(bias.weights + rows.row);
  weigh_rows<EXACT>(to, *to, rows.j, len, G, bias.stats + 2 * head,
                    Unit{bias.unit, bias.unit_rest}, [&](int q) {
                      return *reinterpret_cast<const f32x4*>(s + q * kBlockRows);
                    });
}

template <typename R, bool PAGED, bool BYPOS, int WEIGH>
void launch_biased(const Shape& sh, const AttnLaunch& a, const BiasLaunch& b, hipStream_t s) {
  constexpr int kMinWaves = BYPOS && R::kWaves > 2 ? 2 : R::kWaves;
  const SlotOrder order = sh.order ? *sh.order : SlotOrder{};
  const dim3 grid(a.max_splits, sh.Hkv, order.n ? order.n : a.max_seqs);
  hipLaunchKernelGGL((attn_biased_kernel<R, 4, kMinWaves, PAGED, BYPOS, WEIGH>), grid, dim3(256),
                     WEIGH >= kWeighHere ? sh.G * b.lds_stride * sizeof(float) : 0, s, a, b, order,
                     sh.pg, sh.k_scale, sh.v_scale, sh.G, sh.Hq, sh.Hkv);
}

template <typename R, bool PAGED>
void launch_rows(const Shape& sh, const AttnLaunch& a, const BiasLaunch& b, hipStream_t s) {
  const bool by_position = b.slopes || b.window > 0;
  if (!b.weights) {
    if (by_position) launch_biased<R, PAGED, true, kNoWeights>(sh, a, b, s);
    else launch_biased<R, PAGED, false, kNoWeights>(sh, a, b, s);
  } else if (b.lds_stride && 4 * kBlockRows * b.lds_blocks >= b.rows) {
    if (by_position) launch_biased<R, PAGED, true, kWeighHere>(sh, a, b, s);
    else launch_biased<R, PAGED, false, kWeighHere>(sh, a, b, s);
  } else if (b.lds_stride) {
    if (by_position) launch_biased<R, PAGED, true, kWeighBoth>(sh, a, b, s);
    else launch_biased<R, PAGED, false, kWeighBoth>(sh, a, b, s);
  } else {
    if (by_position) launch_biased<R, PAGED, true, kWeighAfter>(sh, a, b, s);
    else launch_biased<R, PAGED, false, kWeighAfter>(sh, a, b, s);
  }
}

template <typename R>
void launch_layout(const Shape& sh, const AttnLaunch& a, const BiasLaunch& b, hipStream_t s) {
  if (sh.pg.tables) launch_rows<R, true>(sh, a, b, s);
  else launch_rows<R, false>(sh, a, b, s);
}

}  // namespace

hipError_t launch_biased_attention(const Shape& sh, const AttnLaunch& a, const BiasLaunch& given,
                                   hipStream_t s) {
  BiasLaunch b = given;
  // whole heads keep what fits of a CU's 160 KB beside the 38 KB of the merge: of one workgroup
  // where there are no more heads than CUs, or of as many as its registers hold, one for fp32
  // rows, two for bf16, three for e4m3, where that is all of them (microseconds per layer in a
  // captured step, weights after and at once: bf16, 2 heads of 200 rows 9.6 and 7.8, 128 of 700
  // 18.2 and 16.0, 256 of 900 33.1 and 27.5, of 4,000 120 and 100, 512 of 1,100 73.0 and 64.7;
  // e4m3, 8 of 300 10.0 and 8.5, 256 of 200 13.3 and 10.9, of 7,400 119 and 104; fp32, 256 of
  // 900 65.2 and 56.0); part of them, the rest through the workspace, gain less (256 of 9,216, G
  // = 5, 260 and 234, of 12,000, G = 8, 357 and 348), and under half of 16 queries' nothing (160
  // e4m3 heads of 6,000 88 and 96)
  const bool alone = sh.dtype == 0 || b.heads <= 256;
  const int64_t room = (alone ? 118 : sh.dtype == 2 ? 15 : 24) * 256 / sh.G;   // floats a query
  const int blocks = b.rows / kBlockRows, per_wave = (blocks + 3) / 4;
  const int fit = static_cast<int>((room - 4) / (4 * kBlockRows));
  if (b.weights && a.max_splits == 1 && fit > 0 &&
      (per_wave <= fit || (alone && (sh.G <= 8 || per_wave <= 2 * fit)))) {
    b.lds_blocks = per_wave < fit ? per_wave : fit;
    b.lds_stride = 4 * kBlockRows * b.lds_blocks + 4;   // (queries start in different banks)
  }
  if (sh.dtype == 2) launch_layout<E4m3Rows>(sh, a, b, s);
  else if (sh.dtype == 1) launch_layout<Bf16Rows>(sh, a, b, s);
  else launch_layout<F32Rows>(sh, a, b, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !b.weights || b.lds_stride) return e;
  const int rows = a.max_splits * a.split_keys;
  const int per = kWeighThreads * kWeighRows;
  const dim3 grid((rows + per - 1) / per, sh.Hkv, a.max_seqs);
  const bool paged = sh.pg.tables, exact = sh.dtype == 0;
  const auto kernel =
      paged ? (exact ? add_weights_kernel<true, true> : add_weights_kernel<true, false>)
            : (exact ? add_weights_kernel<false, true> : add_weights_kernel<false, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(kWeighThreads), 0, s, a.meta, a.layer, b, sh.pg, sh.G,
                     sh.Hq, sh.Hkv);
  return hipGetLastError();
}

}  // namespace ra
