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
#include "attn_rows.h"
#include "block_choice.h"

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
