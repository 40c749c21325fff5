// Grouped-query decode attention over the compressed per-KV-head cache, with
// the step's append fused in (Section 2, "Notation": o = sum_i alpha_i v_i,
// alpha = softmax_i(q . k_i / sqrt(d)); Appendix F: the G query heads of a
// group read their KV head's cache).
//
// Work decomposition: one workgroup of W wavefronts per (sequence, KV head,
// split of `split_keys` keys); wavefront v streams the v-th W-th of the
// split.  Each wavefront reads its keys and values exactly once for all G
// query heads of the group and keeps an online softmax (running max and sum,
// combined across lanes with wavefront shuffles); the W states merge in LDS.
// A head with one split writes its normalised output directly; otherwise
// every split writes an unnormalised partial, and the last one to finish
// merges them (the contiguous 12-wavefront build: a second kernel).  The
// step's new key/value is read from the input buffers by
// the wavefront that owns the last key, which also stores it into the cache
// after its reads, so no wavefront of the launch reads a row that is being
// written.  Value tiles are read with nontemporal loads, key rows with
// ordinary ones.
//
// bf16 path (MFMA, v_mfma_f32_16x16x32_bf16, 16x16 output tiles):
//   S^T[key][query] = K . Q^T   A = 16 key rows x 32 channels, B = Q^T with
//                               the group's G queries on the N side (padded
//                               to 16 with zeros);
//   O^T[ch][query] += V^T . P^T A = 16 channels x 32 keys from the
//                               transposed value tiles, B = P^T split into
//                               two bf16 parts (hi + lo) for precision.
// A lane's 8 operand elements come from one 16-byte global load: key rows
// are row-major and value rows are stored as transposed 8-row tiles.  The
// key rows are assigned to the two 16-row S tiles so that each lane's
// 8 softmax weights are exactly the 8 keys its P^T operand needs (tile t
// row 4a+i holds key 8a+4t+i), so no data moves between lanes except the
// two shuffles of the row maximum.
// fp32 path (MFMA, v_mfma_f32_16x16x4_f32): the same two products over
// 16-key blocks, the softmax weights kept in fp32.
#include <mutex>

#include "attn_parts.h"

namespace ra {
namespace {

// Merge the split partials of one (sequence, KV head) into the output, for
// the 12-wavefront contiguous bf16 build (heads of one split write their
// output themselves).
// One workgroup per head, launched after the attention kernel (the kernel
// boundary makes every partial visible).  Partial layout:
//   ws_o[((head * split_stride + split) * G + q) * 128 + c]  numerator / 2^m
//   ws_ml[((head * split_stride + split) * G + q) * 2 + {0,1}] = (m, l)
// with m the running max of the scores in log2 units and l the sum of
// 2^(s - m) over the split's keys.
__global__ __launch_bounds__(256) void combine_kernel(AttnLaunch a, int G, int Hq, int Hkv) {
  __shared__ float sm[kMaxSplits * kMaxGroup];   // split maxima, then weights
  __shared__ float sl[kMaxSplits * kMaxGroup];   // split sums
  __shared__ float inv_l[kMaxGroup];
  const int g = blockIdx.x, slot = blockIdx.y;
  const SeqMeta& M = a.meta[slot];
  if (!M.active) return;
  const int t = threadIdx.x;
  const int n_keys = M.len + 1;
  const int nsplit = (n_keys + a.split_keys - 1) / a.split_keys;
  if (nsplit == 1) return;
  const int head = slot * Hkv + g;
  const float* ml = a.ws_ml + static_cast<int64_t>(head) * a.split_stride * G * 2;
  const float* po = a.ws_o + static_cast<int64_t>(head) * a.split_stride * G * kHeadDim;
  for (int i = t; i < nsplit * G; i += blockDim.x) {
    sm[i] = ml[2 * i];
    sl[i] = ml[2 * i + 1];
  }
  __syncthreads();
  // per query: global max, split weights 2^(m_s - max) and the total sum
  if (t < G) {
    float mx = kNegInf;
    for (int s = 0; s < nsplit; ++s) mx = fmaxf(mx, sm[s * G + t]);
    float lsum = 0.f;
    for (int s = 0; s < nsplit; ++s) {
      const float w = exp2f(sm[s * G + t] - mx);
      sm[s * G + t] = w;
      lsum += w * sl[s * G + t];
    }
    inv_l[t] = 1.f / lsum;
  }
  __syncthreads();
  uint16_t* out = static_cast<uint16_t*>(a.out);
  // one thread per (query, 4 channels)
  for (int item = t; item < G * (kHeadDim / 4); item += blockDim.x) {
    const int q = item / (kHeadDim / 4), c4 = (item % (kHeadDim / 4)) * 4;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int s = 0; s < nsplit; ++s) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(
          po + static_cast<int64_t>(s * G + q) * kHeadDim + c4);
      acc += v * sm[s * G + q];
    }
    acc *= inv_l[q];
    const int64_t orow = (static_cast<int64_t>(slot) * Hq + g * G + q) * kHeadDim + c4;
#pragma unroll
    for (int j = 0; j < 4; ++j) out[orow + j] = f32_to_bf16(acc[j]);
  }
}


// ---------------------------------------------------------------------------
// bf16, MFMA
// ---------------------------------------------------------------------------

// W wavefronts per workgroup share one (sequence, KV head, split) work item:
// wavefront v takes the v-th W-th of the split's keys, and the wavefronts
// merge their online-softmax states in LDS at the end.  When the
// head needs a single split, the workgroup writes the normalised output
// itself and no merge kernel runs.  MINW is the number of wavefronts per
// SIMD the build must allow (1 lets the accumulators live in the
// accumulation registers, 2 keeps each wavefront within 256 registers).
template <int W, int MINW, bool PAGED>
__global__ __launch_bounds__(64 * W, MINW) void attn_bf16_kernel(
    AttnLaunch a, Paging pg, int G, int Hq, int Hkv, float scale_log2) {
  constexpr int kNBuf = 2;   // register buffers (3 or 4 measured no faster)
  // heads of several splits merged by their last split (merge_if_last); the
  // contiguous 12-wavefront build has no registers to spare for it, and its
  // multi-split heads are merged by combine_kernel
  constexpr bool kFusedMerge = W != 12 || PAGED;
  __shared__ float s_m[W][kMaxGroup];
  __shared__ float s_l[W][kMaxGroup];
  __shared__ float s_o[W][kMaxGroup][kHeadDim];
  const Work w = locate(a.meta, a.layer, Hkv, a.split_keys, pg);
  if (!w.valid) return;
  const int wave = threadIdx.x >> 6;
  const int lane = threadIdx.x & 63, qi = lane & 15, grp = lane >> 4;
  const LaneMap lm = lane_map();
  const uint16_t* kpool = static_cast<const uint16_t*>(a.kpool);
  const uint16_t* vpool = static_cast<const uint16_t*>(a.vpool);
  const uint16_t* Kr = kpool + w.rm.region * kHeadDim;
  const uint16_t* Vr = vpool + w.rm.region * kHeadDim;
  // key block kb (a multiple of 32): its 32 rows lie in one page of the paged
  // layout, found through the block table; contiguous layouts index the region
  auto load = [&](BlockRegs& b, int kb) {
    if constexpr (PAGED) {
      const int64_t br = pool_row<true>(w.rm, kb);
      load_block(b, kpool + br * kHeadDim, vpool + br * kHeadDim, 0, lm);
    } else {
      load_block(b, Kr, Vr, kb, lm);
    }
  };
  const uint16_t* kn = static_cast<const uint16_t*>(a.k_new) +
                       (static_cast<int64_t>(w.slot) * Hkv + w.g) * kHeadDim;
  const uint16_t* vn = static_cast<const uint16_t*>(a.v_new) +
                       (static_cast<int64_t>(w.slot) * Hkv + w.g) * kHeadDim;

  // Q^T operand: query qi of the group, channels 32*s + 8*grp + [0, 8) at
  // k-step s (the key operand uses the same channel order, so a row's four
  // lane groups read 64 contiguous bytes per load)
  bf16x8 qop[4];
  {
    const uint16_t* qrow = static_cast<const uint16_t*>(a.q) +
        (static_cast<int64_t>(w.slot) * Hq + w.g * G + qi) * kHeadDim + 8 * grp;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const u32x4 z = {0u, 0u, 0u, 0u};
      qop[s] = as_bf16x8(qi < G ? ld16(qrow + 32 * s) : z);
    }
  }

  Softmax st;
  st.m = kNoScore;
  st.l = 0.f;
#pragma unroll
  for (int u = 0; u < 8; ++u) st.acc[u] = f32x4{0.f, 0.f, 0.f, 0.f};

  // this wavefront's keys: [k0, k1) within the split (a multiple of 32 long
  // except where it ends at the new key)
  const int kpw = a.split_keys / W;
  // the same in every lane of the wavefront; in the paged builds of up to 8
  // wavefronts, made scalar, so that block-table entries are scalar loads
  // and block bases scalar sums (the 12-wavefront build has no registers to
  // spare for it and looks the table up per lane)
  constexpr bool kScalarTable = PAGED && W <= 8;
  const int k0 = kScalarTable ? __builtin_amdgcn_readfirstlane(w.k0 + wave * kpw)
                              : w.k0 + wave * kpw;
  const int k1 = min(k0 + kpw, w.k1);
  const bool has = k0 < k1;
  const bool owns_last = has && k1 == w.n_keys;
  const int nfull = !has ? 0 : (owns_last ? (w.len - k0) / 32 : (k1 - k0) / 32);
  if (nfull > 0) {
    // register buffers in rotation; every prefetch is unconditional (clamped
    // to the last block, whose repeated loads hit in cache) and the loop body
    // has no conditional code, so the loads it issues are consumed by the
    // next iteration and the compiler can neither sink them nor make the wait
    // before a block's compute also wait for later blocks' loads
    const int last = nfull - 1;
    BlockRegs buf[kNBuf];
#pragma unroll
    for (int j = 0; j < kNBuf; ++j) load(buf[j], k0 + 32 * min(j, last));
    int i = 0;
    for (; i + kNBuf - 1 < nfull; i += kNBuf) {
#pragma unroll
      for (int j = 0; j < kNBuf; ++j) {
        compute_block(st, buf[j], qop, scale_log2, 32);
        load(buf[j], k0 + 32 * min(i + kNBuf + j, last));
      }
    }
#pragma unroll
    for (int j = 0; j < kNBuf - 1; ++j)
      if (i + j < nfull) compute_block(st, buf[j], qop, scale_log2, 32);
  }
  if (owns_last) {
    // tail block: cached rows below len, the new pair at len, masked above
    const int kb = k0 + 32 * nfull;
    const int limit = w.n_keys - kb;       // 1..32 valid keys
    // rows of this block below len lie in one page of the paged layout (only
    // rows below len are read from the pools: the page of row len may not be
    // in the table yet when len is a multiple of 32)
    const uint16_t* Kb = Kr + static_cast<int64_t>(kb) * kHeadDim;
    const uint16_t* Vb = Vr + static_cast<int64_t>(kb) * kHeadDim;
    if constexpr (PAGED) {
      const int64_t br = kb < w.len ? pool_row<true>(w.rm, kb) : 0;
      Kb = kpool + br * kHeadDim;
      Vb = vpool + br * kHeadDim;
    }
    BlockRegs b;
    const u32x4 z = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int key = kb + lm.krow[t];
      const uint16_t* row = key < w.len ? Kb + lm.krow[t] * kHeadDim : kn;
#pragma unroll
      for (int s = 0; s < 4; ++s)
        b.k[t][s] = key <= w.len ? ld16(row + lm.kcol + 32 * s) : z;
    }
    const int key0 = kb + lm.vrow;         // first key of this lane's tile
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int ch = 16 * u + lm.vch;
      u32x4 v = key0 < w.len ? ld16(Vb + lm.vrow * kHeadDim + ch * 8) : z;
      uint16_t e8[8];
      __builtin_memcpy(e8, &v, 16);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (key0 + e == w.len) e8[e] = vn[ch];
        else if (key0 + e > w.len) e8[e] = 0;
      }
      __builtin_memcpy(&v, e8, 16);
      b.v[u] = v;
    }
    compute_block(st, b, qop, scale_log2, limit);
  }

  // lane sums of the same query -> the wavefront's sum
  st.l += __shfl_xor(st.l, 16, 64);
  st.l += __shfl_xor(st.l, 32, 64);

  if (owns_last)
    append_row<uint16_t, PAGED>(w, a.meta, Hkv, static_cast<const uint16_t*>(a.k_new),
                         static_cast<const uint16_t*>(a.v_new),
                         static_cast<uint16_t*>(a.kpool),
                         static_cast<uint16_t*>(a.vpool), a.pos);

  finish_item<uint16_t, W, kFusedMerge>(a, w, wave, qi, grp, st, G, Hq, Hkv, s_m, s_l, s_o);
}

// A block of 32 rows for the short build, rows at or past len included: row
// len is the step's new pair, rows past it are read from some cached row and
// masked by the caller (keys) or replaced by zero in patch_values.  Every
// lane issues the same sixteen loads whatever the block holds.
__device__ __forceinline__ void load_block_any(BlockRegs& b, const uint16_t* Kb,
                                               const uint16_t* Vb, const uint16_t* kn, int kb,
                                               int len, const LaneMap& lm) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint16_t* row = (kb + lm.krow[t] < len ? Kb + lm.krow[t] * kHeadDim : kn) + lm.kcol;
#pragma unroll
    for (int s = 0; s < 4; ++s) b.k[t][s] = ld16(row + 32 * s);
  }
  // an 8-row tile with no row below len reads the block's first tile instead
  const uint16_t* vt = Vb + (kb + lm.vrow < len ? lm.vrow * kHeadDim : 0) + lm.vch * 8;
#pragma unroll
  for (int u = 0; u < 8; ++u) b.v[u] = ld16_stream(vt + 16 * 8 * u);
}

// The new value at row len, zeros above it (vn: the lane's channel of each
// 16-channel tile).
__device__ __forceinline__ void patch_values(BlockRegs& b, const uint16_t (&vn)[8], int kb,
                                             int len, const LaneMap& lm) {
  const int at = len - kb - lm.vrow;         // the new row within the lane's tile
  if (at < 8) {
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      uint16_t e8[8];
      __builtin_memcpy(e8, &b.v[u], 16);
#pragma unroll
      for (int e = 0; e < 8; ++e) e8[e] = e < at ? e8[e] : e == at ? vn[u] : uint16_t(0);
      __builtin_memcpy(&b.v[u], e8, 16);
    }
  }
}

// Decode attention where the launch is bound by latency, not by bytes: at
// most 64 keys per wavefront (see plan_for).  A wavefront issues the loads of
// all its keys, the step's new pair among them, before it uses any: one round
// trip to memory, where the streaming build takes one for its full blocks and
// another for the block of the new pair, and reads its last block again for
// every prefetch that runs out of blocks.
template <int W, bool PAGED>
__global__ __launch_bounds__(64 * W, 1) void attn_bf16_short_kernel(
    AttnLaunch a, Paging pg, int G, int Hq, int Hkv, float scale_log2) {
  __shared__ float s_m[W][kMaxGroup];
  __shared__ float s_l[W][kMaxGroup];
  __shared__ float s_o[W][kMaxGroup][kHeadDim];
  const Work w = locate(a.meta, a.layer, Hkv, a.split_keys, pg);
  if (!w.valid) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, qi = lane & 15, grp = lane >> 4;
  const LaneMap lm = lane_map();
  const uint16_t* kpool = static_cast<const uint16_t*>(a.kpool);
  const uint16_t* vpool = static_cast<const uint16_t*>(a.vpool);
  const int64_t new_row = (static_cast<int64_t>(w.slot) * Hkv + w.g) * kHeadDim;
  const uint16_t* kn = static_cast<const uint16_t*>(a.k_new) + new_row;
  const uint16_t* vn = static_cast<const uint16_t*>(a.v_new) + new_row;
  const int kpw = a.split_keys / W;            // 32 or 64
  const int k0 = w.k0 + wave * kpw;
  const int k1 = min(k0 + kpw, w.k1);
  const bool has = k0 < k1, two = k0 + 32 < k1;
  const bool owns_last = has && k1 == w.n_keys;
  auto load = [&](BlockRegs& b, int kb) {
    // the block's first row; a block that starts at row len holds no cached
    // row and reads (and does not use) the pool's first rows
    const int64_t br = kb < w.len ? pool_row<PAGED>(w.rm, kb) : 0;
    load_block_any(b, kpool + br * kHeadDim, vpool + br * kHeadDim, kn, kb, w.len, lm);
  };

  Softmax st;
  st.m = kNoScore;
  st.l = 0.f;
#pragma unroll
  for (int u = 0; u < 8; ++u) st.acc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (has) {
    bf16x8 qop[4];
    const uint16_t* qrow = static_cast<const uint16_t*>(a.q) +
        (static_cast<int64_t>(w.slot) * Hq + w.g * G + (qi < G ? qi : 0)) * kHeadDim + 8 * grp;
    uint16_t vnew[8];
    if (owns_last) {
#pragma unroll
      for (int u = 0; u < 8; ++u) vnew[u] = vn[16 * u + lm.vch];
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const u32x4 z = {0u, 0u, 0u, 0u};
      const u32x4 x = ld16(qrow + 32 * s);
      qop[s] = as_bf16x8(qi < G ? x : z);
    }
    BlockRegs b0;
    load(b0, k0);
    if (two) {
      BlockRegs b1;
      load(b1, k0 + 32);
      compute_block(st, b0, qop, scale_log2, 32);
      if (owns_last) patch_values(b1, vnew, k0 + 32, w.len, lm);
      compute_block(st, b1, qop, scale_log2, min(32, k1 - k0 - 32));
    } else {
      if (owns_last) patch_values(b0, vnew, k0, w.len, lm);
      compute_block(st, b0, qop, scale_log2, k1 - k0);
    }
    st.l += __shfl_xor(st.l, 16, 64);
    st.l += __shfl_xor(st.l, 32, 64);
  }
  finish_item<uint16_t, W, true>(a, w, wave, qi, grp, st, G, Hq, Hkv, s_m, s_l, s_o);
  if (owns_last)
    append_row<uint16_t, PAGED>(w, a.meta, Hkv, static_cast<const uint16_t*>(a.k_new),
                                static_cast<const uint16_t*>(a.v_new),
                                static_cast<uint16_t*>(a.kpool),
                                static_cast<uint16_t*>(a.vpool), a.pos);
}

// ---------------------------------------------------------------------------
// bf16, MFMA, moving the rows of a deferred eviction on the way
// ---------------------------------------------------------------------------

// The last block of a head's source rows, kb .. kb+31, reaching past the
// cached rows: it is loaded as a full block (rows past the region's end read
// its row 0, so every lane issues the same sixteen loads as for any block and
// the loads in flight stay countable) and, once the data has arrived, row
// n_rows becomes the step's new pair (staged in LDS: nk, nv) and the rows
// above it zero.
__device__ __forceinline__ void load_block_clamped(BlockRegs& b, const uint16_t* Kr,
                                                   const uint16_t* Vr, int kb, int n_rows,
                                                   const LaneMap& lm) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int key = kb + lm.krow[t];
    const uint16_t* row = Kr + static_cast<int64_t>(key < n_rows ? key : 0) * kHeadDim + lm.kcol;
#pragma unroll
    for (int s = 0; s < 4; ++s) b.k[t][s] = ld16(row + 32 * s);
  }
  const int key0 = kb + lm.vrow;                      // a tile's first row (8-aligned)
  const uint16_t* vt = Vr + static_cast<int64_t>(key0 < n_rows ? key0 : 0) * kHeadDim + lm.vch * 8;
#pragma unroll
  for (int u = 0; u < 8; ++u) b.v[u] = ld16_stream(vt + 16 * 8 * u);
}

__device__ __forceinline__ void patch_block_tail(BlockRegs& b, const uint16_t* nk,
                                                 const uint16_t* nv, int kb, int n_rows,
                                                 const LaneMap& lm) {
  const u32x4 z = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int key = kb + lm.krow[t];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (key == n_rows) b.k[t][s] = *reinterpret_cast<const u32x4*>(nk + lm.kcol + 32 * s);
      else if (key > n_rows) b.k[t][s] = z;
    }
  }
  const int key0 = kb + lm.vrow;
  if (key0 + 8 > n_rows) {
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      uint16_t e8[8];
      __builtin_memcpy(e8, &b.v[u], 16);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (key0 + e == n_rows) e8[e] = nv[16 * u + lm.vch];
        else if (key0 + e > n_rows) e8[e] = 0;
      }
      __builtin_memcpy(&b.v[u], e8, 16);
    }
  }
}

// Decode attention for the step after a deferred eviction (contiguous
// chronological layout, bf16, one workgroup of W wavefronts per (sequence,
// KV head), the whole head).  A sequence whose event deferred its row moves
// (due == kDueMovePending) holds its key/value rows in the order before the
// event, rows [0, plan_len), and the event's drop slots; its positions are
// already compacted and len = plan_len - m.  Attention runs over the
// surviving rows and the step's new pair (the dropped rows are masked), and
// every surviving row j after the first drop moves down to its compacted
// slot j - #{drops below j}, so the rows end as a full event would leave
// them, without reading them a second time.  The blocks are dealt in rounds,
// block r * W + v to wavefront v; every wavefront's loads of a round have
// returned (the round's softmax consumed them) before the barrier that
// precedes the round's moves.  A row moves only down, into a block of its
// own round or of an earlier one, which was read before that barrier, and
// no round reads a row that an earlier round wrote; the next round's loads,
// issued before the barrier, read only rows above every destination of the
// round, except that loads of blocks past the last key, and of tail rows
// past the cached ones, read the region's row 0 (which a round may be
// writing when the prompt is empty): those values are never used, being
// replaced by the new pair or zero, or belonging to no block.  The new pair
// is stored at len after the last round.  Sequences with nothing to move
// take the same path without moves.
template <int W>
__global__ __launch_bounds__(64 * W, 1) void attn_bf16_move_kernel(
    AttnLaunch a, int L, int G, int Hq, int Hkv, float scale_log2) {
  __shared__ float s_m[W][kMaxGroup];
  __shared__ float s_l[W][kMaxGroup];
  __shared__ float s_o[W][kMaxGroup][kHeadDim];
  __shared__ int s_drop[kMaxEvery];
  // a round's surviving value rows in destination order, per channel, offset
  // by the round's first destination row mod 8 so that destination tiles
  // start on 16-byte boundaries
  constexpr int kStage = W * 32 + 16;
  __shared__ __align__(16) uint16_t s_v[kHeadDim][kStage];
  __shared__ __align__(16) uint16_t s_new[2][kHeadDim];  // the step's key, value
  const int g = blockIdx.y, slot = blockIdx.z;
  const SeqMeta& M = a.meta[slot];
  if (!M.active) return;
  const bool moving = M.due == kDueMovePending;
  const int len = M.len;                              // rows once compacted
  const int n_rows = moving ? M.plan_len : len;       // rows in the region now
  const int m = min(n_rows - len, kMaxEvery);        // <= evict_every (host)
  const int lg = a.layer * Hkv + g;
  const int64_t region = M.base + static_cast<int64_t>(lg) * M.cap;
  // wavefront-uniform (the block indices and the drop scans below are scalar)
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, qi = lane & 15, grp = lane >> 4;
  if (moving) {
    const int32_t* d = a.drops + (static_cast<int64_t>(slot) * L * Hkv + lg) * a.drop_stride;
    for (int k = threadIdx.x; k < min(m, kMaxEvery); k += 64 * W) s_drop[k] = d[k];
  }
  {
    const uint16_t* src = threadIdx.x < kHeadDim ? static_cast<const uint16_t*>(a.k_new)
                                                 : static_cast<const uint16_t*>(a.v_new);
    if (threadIdx.x < 2 * kHeadDim)
      (&s_new[0][0])[threadIdx.x] =
          src[(static_cast<int64_t>(slot) * Hkv + g) * kHeadDim + (threadIdx.x & (kHeadDim - 1))];
  }
  __syncthreads();
  const LaneMap lm = lane_map();
  uint16_t* kpool = static_cast<uint16_t*>(a.kpool);
  uint16_t* vpool = static_cast<uint16_t*>(a.vpool);
  const uint16_t* Kr = kpool + region * kHeadDim;
  const uint16_t* Vr = vpool + region * kHeadDim;

  bf16x8 qop[4];
  {
    const uint16_t* qrow = static_cast<const uint16_t*>(a.q) +
        (static_cast<int64_t>(slot) * Hq + g * G + qi) * kHeadDim + 8 * grp;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const u32x4 z = {0u, 0u, 0u, 0u};
      qop[s] = as_bf16x8(qi < G ? ld16(qrow + 32 * s) : z);
    }
  }
  Softmax st;
  st.m = kNoScore;
  st.l = 0.f;
#pragma unroll
  for (int u = 0; u < 8; ++u) st.acc[u] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int n_keys = n_rows + 1;                      // the region's rows + the new pair
  const int nblk = (n_keys + 31) / 32;
  const int rounds = (nblk + W - 1) / W;
  auto load = [&](BlockRegs& b, int blk) {
    const int kb = blk * 32;
    if (kb + 32 <= n_rows) load_block(b, Kr, Vr, kb, lm);
    else load_block_clamped(b, Kr, Vr, kb, n_rows, lm);
  };
  // two register buffers, each named (an array indexed by the round's parity
  // would live in scratch memory): the loop below runs two rounds per pass
  // every round issues its sixteen prefetch loads, also for blocks past the
  // last key (they read the region's row 0 and are never used): with a fixed
  // count of loads after each block's, the wait for a block leaves the next
  // block's loads in flight
  BlockRegs buf0, buf1;
  load(buf0, wave);
  int di = 0;                 // drops below the current block (wavefront-uniform)
  auto round = [&](int r, BlockRegs& cur, BlockRegs& nxt) {
    const int blk = r * W + wave;
    const int kb = blk * 32;
    const bool have = blk < nblk;
    load(nxt, blk + W);
    uint32_t dropped = 0;
    if (have) {
      if (kb + 32 > n_rows) patch_block_tail(cur, s_new[0], s_new[1], kb, n_rows, lm);
      while (di < m && s_drop[di] < kb) ++di;
      for (int k = di; k < m && s_drop[k] < kb + 32; ++k) dropped |= 1u << (s_drop[k] - kb);
      compute_block<true>(st, cur, qop, scale_log2, min(32, n_keys - kb), dropped);
    }
    __syncthreads();          // every load of the round has been consumed
    if (moving && have) {
      const BlockRegs& b = cur;
      // key rows: this lane's two rows, four 16-byte chunks each
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int rr = lm.krow[t], j = kb + rr;
        if (j < n_rows && !((dropped >> rr) & 1u)) {
          const int dst = j - di - __popc(__builtin_amdgcn_ubfe(dropped, 0, rr));
          if (dst != j) {
            uint16_t* row = kpool + (region + dst) * kHeadDim + lm.kcol;
#pragma unroll
            for (int s = 0; s < 4; ++s) *reinterpret_cast<u32x4*>(row + 32 * s) = b.k[t][s];
          }
        }
      }
    }
    if (moving) {
      // values: the round's survivors go to LDS in destination order, then the
      // workgroup writes whole destination tiles (16 bytes per channel); only
      // the round's first and last tiles, shared with the neighbouring rounds,
      // are written element by element
      const int r0 = r * W * 32;                                 // round's first source row
      int fr = 0;                                                // drops below r0
      while (fr < m && s_drop[fr] < r0) ++fr;
      const int r1 = min(r0 + W * 32, n_rows);                   // round's source rows [r0, r1)
      int fe = fr;
      while (fe < m && s_drop[fe] < r1) ++fe;
      const int d_lo = r0 - fr, d_hi = r1 - fe;                  // destinations [d_lo, d_hi)
      const int off = d_lo & 7;
      if (have && kb < n_rows) {
        const BlockRegs& b = cur;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int rr = lm.vrow + e, j = kb + rr;
          if (j < n_rows && !((dropped >> rr) & 1u)) {
            const int dst = j - di - __popc(__builtin_amdgcn_ubfe(dropped, 0, rr));
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              uint16_t e8[8];
              __builtin_memcpy(e8, &b.v[u], 16);
              s_v[16 * u + lm.vch][off + dst - d_lo] = e8[e];
            }
          }
        }
      }
      __syncthreads();
      if (d_hi > d_lo && r1 > s_drop[0]) {
        const int t_lo = d_lo >> 3, t_hi = (d_hi - 1) >> 3;       // destination tiles
        const int items = (t_hi - t_lo + 1) * kHeadDim;
        for (int it = threadIdx.x; it < items; it += 64 * W) {
          const int tile = t_lo + it / kHeadDim, ch = it % kHeadDim;
          const int lo = max(tile * 8, d_lo), hi = min(tile * 8 + 8, d_hi);
          const int64_t row0 = region + tile * 8;                // 8-aligned (region is)
          uint16_t* dstp = vpool + row0 * kHeadDim + ch * 8;
          const uint16_t* src = &s_v[ch][off + tile * 8 - d_lo];
          if (lo == tile * 8 && hi == tile * 8 + 8) {
            *reinterpret_cast<u32x4*>(dstp) = *reinterpret_cast<const u32x4*>(src);
          } else {
            for (int x = lo; x < hi; ++x) dstp[x - tile * 8] = src[x - tile * 8];
          }
        }
      }
    }
  };
  for (int r = 0; r < rounds; r += 2) {
    round(r, buf0, buf1);
    if (r + 1 < rounds) round(r + 1, buf1, buf0);
  }
  st.l += __shfl_xor(st.l, 16, 64);
  st.l += __shfl_xor(st.l, 32, 64);
  // lane indices taken afresh (kept from before the rounds, they would be
  // spilled: the rounds hold every register)
  const int lane_e = __lane_id(), qe = lane_e & 15, ge = lane_e >> 4;
  const int tid = wave * 64 + lane_e;
  __syncthreads();            // every move is done: the new pair goes to row len
  if (wave == 0) {
    const int64_t row = region + len;
    for (int c = lane_e; c < kHeadDim; c += 64) {
      kpool[row * kHeadDim + c] = s_new[0][c];
      vpool[(row & ~int64_t(7)) * kHeadDim + c * 8 + (row & 7)] = s_new[1][c];
    }
    if (lane_e == 0) a.pos[row] = M.prompt_len + M.step;
  }

  // merge the W wavefronts in LDS and write the normalised output
  if (qe < G) {
#pragma unroll
    for (int u = 0; u < 8; ++u)
      *reinterpret_cast<f32x4*>(&s_o[wave][qe][16 * u + 4 * ge]) = st.acc[u];
    if (ge == 0) {
      s_m[wave][qe] = st.m;
      s_l[wave][qe] = st.l;
    }
  }
  __syncthreads();
  uint16_t* out = static_cast<uint16_t*>(a.out);
  for (int idx = tid; idx < G * kHeadDim; idx += 64 * W) {
    const int q = idx / kHeadDim, c = idx % kHeadDim;
    float mx = kNegInf;
#pragma unroll
    for (int v = 0; v < W; ++v) mx = fmaxf(mx, s_m[v][q]);
    float lsum = 0.f, o = 0.f;
#pragma unroll
    for (int v = 0; v < W; ++v) {
      const float sc = exp2f(s_m[v][q] - mx);
      lsum += s_l[v][q] * sc;
      o += s_o[v][q][c] * sc;
    }
    out[(static_cast<int64_t>(slot) * Hq + g * G + q) * kHeadDim + c] = f32_to_bf16(o / lsum);
  }
}

// ---------------------------------------------------------------------------
// fp32, MFMA
// ---------------------------------------------------------------------------

// A block of 16 keys in the operand registers of v_mfma_f32_16x16x4_f32
// (lane r = lane & 15, group = lane >> 4).
struct BlockF32 {
  f32x4 k[8];   // key row r, channels 16t + 4*group + [0, 4)
  f32x4 v[8];   // channel 16u + r, rows 4*group + [0, 4)
};

// The block whose `rows` first rows are cached (key rows at Kb, value tiles at
// Vb).  Rows past them read the block's first row or tile instead, so that
// every lane issues the same loads whatever the block holds.
__device__ __forceinline__ void load_block(BlockF32& b, const float* Kb, const float* Vb,
                                           int rows) {
  const int r = threadIdx.x & 15, grp = (threadIdx.x & 63) >> 4, tile = 8 * (grp >> 1);
  const int k = (r < rows ? r * kHeadDim : 0) + 4 * grp;
  const int v = (tile < rows ? tile * kHeadDim : 0) + r * 8 + 4 * (grp & 1);
#pragma unroll
  for (int t = 0; t < 8; ++t) b.k[t] = *reinterpret_cast<const f32x4*>(Kb + k + 16 * t);
#pragma unroll
  for (int u = 0; u < 8; ++u)
    b.v[u] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(Vb + v + 16 * 8 * u));
}

// One 16-key block at row kb.  S^T[key][query] = K . Q^T leaves each lane the
// scores of keys 4*group + i of query r, which is the P^T operand of
// O^T[channel][query] += V^T . P^T at key step i: no lane exchange but the
// two shuffles of the row maximum.  Keys at `limit` and above are masked.
__device__ __forceinline__ void compute_block(Softmax& st, const BlockF32& b,
                                              const f32x4 (&qop)[8], float scale_log2,
                                              int limit) {
  // four accumulators: short sums (and independent products)
  f32x4 sp[4] = {};
#pragma unroll
  for (int t = 0; t < 8; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      sp[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(b.k[t][i], qop[t][i], sp[i], 0, 0, 0);
  float x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    x[i] = ((sp[0][i] + sp[1][i]) + (sp[2][i] + sp[3][i])) * scale_log2;
  if (limit < 16) {
    const int grp = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (4 * grp + i >= limit) x[i] = kNegInf;
  }
  float bm = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
  bm = fmaxf(bm, __shfl_xor(bm, 16, 64));
  bm = fmaxf(bm, __shfl_xor(bm, 32, 64));
  const float mn = fmaxf(st.m, bm);
  const float alpha = exp2f(st.m - mn);
  float p[4], psum = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    p[i] = exp2f(x[i] - mn);
    psum += p[i];
  }
  st.l = st.l * alpha + psum;
  st.m = mn;
  // the block's own sum first, then one addition per block: the running sum
  // rounds once per 16 keys
#pragma unroll
  for (int u0 = 0; u0 < 8; u0 += 2) {
    f32x4 o[2] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        o[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(b.v[u0 + u][i], p[i], o[u], 0, 0, 0);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        st.acc[u0 + u][i] = fmaf(st.acc[u0 + u][i], alpha, o[u][i]);
  }
}

// fp32 decode attention: a workgroup of W wavefronts (four; one for many heads
// of few keys, see plan_f32) per (sequence, KV
// head, split), each streaming a W-th of the split's keys in 16-key blocks, two
// blocks in flight.  Bound by HBM where the rows are many and by latency where
// they are few; the group's queries are padded to 16, which the matrix cores
// still do in a third of the time the rows take to arrive (64 products of 32
// cycles per 16 KB block).  8 sequences of 8 heads, 2,900 rows: 40 us per
// launch (4.7 TB/s) where single wavefronts on the vector ALU, one key per
// lane, took 81 us (2.4 TB/s); 256 heads of 3,000 rows: 6.0 TB/s.
template <int W, bool PAGED>
__global__ __launch_bounds__(64 * W, 2) void attn_f32_kernel(AttnLaunch a, Paging pg, int G, int Hq,
                                                             int Hkv, float scale_log2) {
  __shared__ float s_m[W][kMaxGroup];
  __shared__ float s_l[W][kMaxGroup];
  __shared__ float s_o[W][kMaxGroup][kHeadDim];
  __shared__ __align__(16) float s_new[2][kHeadDim];   // the new pair, for its wavefront
  const Work w = locate(a.meta, a.layer, Hkv, a.split_keys, pg);
  if (!w.valid) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, qi = lane & 15, grp = lane >> 4;
  const float* kpool = static_cast<const float*>(a.kpool);
  const float* vpool = static_cast<const float*>(a.vpool);
  const int64_t new_row = (static_cast<int64_t>(w.slot) * Hkv + w.g) * kHeadDim;
  const int kpw = a.split_keys / W;            // a multiple of 16
  const int k0 = __builtin_amdgcn_readfirstlane(w.k0 + wave * kpw);
  const int k1 = min(k0 + kpw, w.k1);
  const bool has = k0 < k1;
  const bool owns_last = has && k1 == w.n_keys;
  auto load = [&](BlockF32& b, int kb) {
    // a block that starts at row len holds no cached row: it reads (and does
    // not use) the block before it
    const int64_t br = pool_row<PAGED>(w.rm, min(kb, max(0, w.len - 1) & ~15));
    load_block(b, kpool + br * kHeadDim, vpool + br * kHeadDim, w.len - kb);
  };

  Softmax st;
  st.m = kNoScore;
  st.l = 0.f;
#pragma unroll
  for (int u = 0; u < 8; ++u) st.acc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (has) {
    const float2 kn = reinterpret_cast<const float2*>(static_cast<const float*>(a.k_new) + new_row)[lane];
    const float2 vn = reinterpret_cast<const float2*>(static_cast<const float*>(a.v_new) + new_row)[lane];
    // Q^T operand: query qi, channels as the key rows' (zero past G)
    f32x4 qop[8];
    const float* qrow = static_cast<const float*>(a.q) +
        (static_cast<int64_t>(w.slot) * Hq + w.g * G + (qi < G ? qi : 0)) * kHeadDim + 4 * grp;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(qrow + 16 * t);
      qop[t] = qi < G ? x : f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int last = (k1 - k0 - 1) / 16;       // blocks 0 .. last
    BlockF32 b0, b1;
    load(b0, k0);
    load(b1, k0 + 16 * min(1, last));
    if (owns_last) {
      reinterpret_cast<float2*>(s_new[0])[lane] = kn;
      reinterpret_cast<float2*>(s_new[1])[lane] = vn;
    }
    int i = 0;
    for (; i + 1 < last; i += 2) {
      // (the loads stay where they are: moved up among the products, they
      // would need registers of their own)
      compute_block(st, b0, qop, scale_log2, 16);
      __builtin_amdgcn_sched_barrier(0);
      load(b0, k0 + 16 * (i + 2));
      __builtin_amdgcn_sched_barrier(0);
      compute_block(st, b1, qop, scale_log2, 16);
      __builtin_amdgcn_sched_barrier(0);
      load(b1, k0 + 16 * min(i + 3, last));
      __builtin_amdgcn_sched_barrier(0);
    }
    if (i < last) {
      compute_block(st, b0, qop, scale_log2, 16);
      b0 = b1;
    }
    if (owns_last) {
      // row len takes the new pair, the values past it zero
      const int at_row = w.len - (k0 + 16 * last), at = at_row - 4 * grp;
      if (qi == at_row) {
#pragma unroll
        for (int t = 0; t < 8; ++t)
          b0.k[t] = *reinterpret_cast<const f32x4*>(&s_new[0][16 * t + 4 * grp]);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) b0.v[u][e] = e < at ? b0.v[u][e] : e == at ? s_new[1][16 * u + qi] : 0.f;
    }
    compute_block(st, b0, qop, scale_log2, k1 - (k0 + 16 * last));
    st.l += __shfl_xor(st.l, 16, 64);
    st.l += __shfl_xor(st.l, 32, 64);
  }
  finish_item<float, W, true>(a, w, wave, qi, grp, st, G, Hq, Hkv, s_m, s_l, s_o);
  if (owns_last)
    append_row<float, PAGED>(w, a.meta, Hkv, static_cast<const float*>(a.k_new),
                             static_cast<const float*>(a.v_new), static_cast<float*>(a.kpool),
                             static_cast<float*>(a.vpool), a.pos);
}

template <bool PAGED>
hipError_t launch_attention_t(const Shape& sh, const AttnLaunch& a, hipStream_t s) {
  const dim3 grid(a.max_splits, sh.Hkv, a.max_seqs);
  // scores in log2 units: q.k / sqrt(d) * log2(e)
  const float scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(kHeadDim));
  const dim3 cgrid(sh.Hkv, a.max_seqs);
  if (sh.dtype == 1 && a.move) {
    // one workgroup per head (max_splits == 1), rows of deferred events moved;
    // eight wavefronts (256 registers each: two per SIMD; a four-wavefront
    // build needs more than 256 and would run one per SIMD)
    const dim3 mgrid(1, sh.Hkv, a.max_seqs);
    hipLaunchKernelGGL((attn_bf16_move_kernel<8>), mgrid, dim3(512), 0, s, a, sh.L, sh.G,
                       sh.Hq, sh.Hkv, scale_log2);
  } else if (sh.dtype == 1) {
    if (a.short_runs && a.waves == 4)
      hipLaunchKernelGGL((attn_bf16_short_kernel<4, PAGED>), grid, dim3(256), 0, s, a, sh.pg,
                         sh.G, sh.Hq, sh.Hkv, scale_log2);
    else if (a.short_runs && a.waves == 8)
      hipLaunchKernelGGL((attn_bf16_short_kernel<8, PAGED>), grid, dim3(512), 0, s, a, sh.pg,
                         sh.G, sh.Hq, sh.Hkv, scale_log2);
    else if (a.waves == 12)
      hipLaunchKernelGGL((attn_bf16_kernel<12, 1, PAGED>), grid, dim3(768), 0, s, a, sh.pg,
                         sh.G, sh.Hq, sh.Hkv, scale_log2);
    else if (a.waves == 8)
      hipLaunchKernelGGL((attn_bf16_kernel<8, 1, PAGED>), grid, dim3(512), 0, s, a, sh.pg,
                         sh.G, sh.Hq, sh.Hkv, scale_log2);
    else if (a.waves == 4 && a.wide_regs)
      hipLaunchKernelGGL((attn_bf16_kernel<4, 1, PAGED>), grid, dim3(256), 0, s, a, sh.pg,
                         sh.G, sh.Hq, sh.Hkv, scale_log2);
    else if (a.waves == 4)
      hipLaunchKernelGGL((attn_bf16_kernel<4, 2, PAGED>), grid, dim3(256), 0, s, a, sh.pg,
                         sh.G, sh.Hq, sh.Hkv, scale_log2);
    else
      return hipErrorInvalidConfiguration;
    // a head with several splits is merged by its last split (merge_if_last),
    // except in the contiguous 12-wavefront build
    if (a.max_splits > 1 && a.waves == 12 && !PAGED)
      hipLaunchKernelGGL(combine_kernel, cgrid, dim3(256), 0, s, a, sh.G, sh.Hq, sh.Hkv);
  } else {
    if (a.waves == 4)
      hipLaunchKernelGGL((attn_f32_kernel<4, PAGED>), grid, dim3(256), 0, s, a, sh.pg, sh.G,
                         sh.Hq, sh.Hkv, scale_log2);
    else if (a.waves == 1)
      hipLaunchKernelGGL((attn_f32_kernel<1, PAGED>), grid, dim3(64), 0, s, a, sh.pg, sh.G,
                         sh.Hq, sh.Hkv, scale_log2);
    else
      return hipErrorInvalidConfiguration;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attention(const Shape& sh, const AttnLaunch& a, hipStream_t s) {
  if (sh.dtype == 2) return launch_attention_e4m3(sh, a, s);
  return sh.pg.tables ? launch_attention_t<true>(sh, a, s) : launch_attention_t<false>(sh, a, s);
}

// Partials of the allocation-free attention entry point.  Every GPU the
// library runs on holds its own copy until the process ends.  In host code
// `scratch` names a host-side stand-in, not device memory: host code uses
// only the address scratch_address returns.
static __device__ __align__(256) float scratch[kNoAllocScratchBytes / sizeof(float)];

hipError_t scratch_address(void** out) {
  static std::mutex mu;
  static void* addr[64] = {};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(mu);
  if (!addr[dev]) {
    void* p = nullptr;
    e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
    if (e != hipSuccess) return e;
    addr[dev] = p;
  }
  *out = addr[dev];
  return hipSuccess;
}

}  // namespace ra
