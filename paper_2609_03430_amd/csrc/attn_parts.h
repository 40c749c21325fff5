// Device code shared by the attention kernels: the work of a workgroup, the
// online softmax's state, and the merge of a head's wavefronts and splits.
#pragma once

#include <type_traits>

#include "ra_internal.h"

namespace ra {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kNegInf = -__builtin_huge_valf();

// The largest score of a state that has seen none but -inf (masked keys, or rows
// that score so): finite, so that the weights of such keys and the rescale come
// out 0 and 1, where the difference of two infinities would make them NaN.
constexpr float kNoScore = -3.4028234663852886e38f;

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) {
  bf16x8 r;
  __builtin_memcpy(&r, &v, 16);
  return r;
}

__device__ __forceinline__ u32x4 ld16(const void* p) {
  return *reinterpret_cast<const u32x4*>(p);
}

// Streaming load (nontemporal): the cached rows are read once per launch, so
// they are fetched without being kept in the caches.  Used where a load
// instruction covers whole 128-byte lines (the value tiles); a key load
// covers half lines of 16 rows, whose other halves the next load reads.
__device__ __forceinline__ u32x4 ld16_stream(const void* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
}

__device__ __forceinline__ uint16_t f32_to_bf16(float x) {
  __bf16 b = static_cast<__bf16>(x);   // round to nearest even
  uint16_t h;
  __builtin_memcpy(&h, &b, 2);
  return h;
}

struct Work {
  int slot, g, split;
  int len, n_keys, k0, k1, nsplit;
  RowMap rm;       // where the rows of the (slot, layer, g) cache live
  bool valid;
};

__device__ __forceinline__ Work locate(const SeqMeta* meta, int layer, int Hkv,
                                       int split_keys, const Paging& pg) {
  Work w;
  w.split = blockIdx.x;
  w.g = blockIdx.y;
  w.slot = blockIdx.z;
  const SeqMeta& M = meta[w.slot];
  w.valid = false;
  if (!M.active) return w;
  w.len = M.len;
  w.n_keys = w.len + 1;
  w.k0 = w.split * split_keys;
  if (w.k0 >= w.n_keys) return w;
  w.k1 = min(w.k0 + split_keys, w.n_keys);
  w.nsplit = (w.n_keys + split_keys - 1) / split_keys;
  w.rm = row_map(M, w.slot, layer * Hkv + w.g, pg);
  w.valid = true;
  return w;
}

// Store the step's new pair into the cache (row `len` of the head).
template <typename E, bool PAGED>
__device__ __forceinline__ void append_row(const Work& w, const SeqMeta* meta,
                                           int Hkv, const E* k_new,
                                           const E* v_new, E* kpool, E* vpool,
                                           int32_t* pos) {
  const int lane = threadIdx.x & 63;   // called by one whole wavefront
  const int64_t src = (static_cast<int64_t>(w.slot) * Hkv + w.g) * kHeadDim;
  const int64_t row = pool_row<PAGED>(w.rm, w.len);
  for (int c = lane; c < kHeadDim; c += 64) {
    kpool[row * kHeadDim + c] = k_new[src + c];
    vpool[(row & ~int64_t(7)) * kHeadDim + c * 8 + (row & 7)] = v_new[src + c];
  }
  if (lane == 0) pos[row] = meta[w.slot].prompt_len + meta[w.slot].step;
}

// Partials of a head merged inside the attention kernel travel through
// device-coherent accesses (agent-scope relaxed atomics: stores written
// through to the level the chip's dies share, loads served from it), so the
// merge needs no whole-cache write-back or invalidation, which would stall
// every workgroup still streaming on the same die.
__device__ __forceinline__ void store_shared_level(float* p, float v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void load_shared_level(const float* p, float& x, float& y) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
  x = __uint_as_float(static_cast<uint32_t>(v));
  y = __uint_as_float(static_cast<uint32_t>(v >> 32));
}

// One softmax state of two channels: running max, sum and numerators.
struct Partial {
  float m, l, o0, o1;
};

// Splits of a head whose every cached row is attended.
struct DenseSplits {
  __device__ __forceinline__ int slot() const { return blockIdx.z; }
  __device__ __forceinline__ int operator()(const AttnLaunch& a, int slot) const {
    return (a.meta[slot].len + 1 + a.split_keys - 1) / a.split_keys;
  }
};

// The split partials of one head merged by the last of its splits to finish
// (outputs of element type E: bf16 bits or float).  Every split stores its
// partials with store_shared_level and waits until they are written; then one
// thread counts the split on the head's arrival counter.  The split that
// brings the count to nsplit reads every split's partials with
// load_shared_level, merges them and resets the counter for the next launch.
// Nothing waits on another workgroup: the other splits simply end.  Called by
// every thread of the workgroup after its partials are stored; the head and
// its split count are taken afresh from the grid position and the slot record
// (kept from before the key loop, they would take registers the loop needs).
//
// Bound by the latency of the shared level: a thread owns two channels of one
// query, and its splits' numerators, maxima and sums come as batches of
// 8-byte loads all in flight together (4 or 16 splits per round trip), merged
// by the thread itself with no exchange.  A thread with several items (more
// channel pairs than threads) takes 5 to 12 splits without the four loads past
// them (25 heads of 5,190 rows in 10 splits, G = 16: 27.6 -> 25.4 us).  Where the
// workgroup has more threads than the head has channel pairs, the splits are
// dealt to `parts` groups of threads, which merge in LDS in split order.
//
// `ends` says what the maxima are in (exp2(x): 2 to the difference x of two), and where it
// keeps them is told the head's maximum and sum of each query.
struct Log2Ends {
  static constexpr bool kKeeps = false;
  __device__ __forceinline__ float exp2(float x) const { return exp2f(x); }
  __device__ __forceinline__ void keep(int, float, float) const {}
};
template <typename E, int NT, typename Splits = DenseSplits, typename Ends = Log2Ends>
__device__ void merge_if_last(const AttnLaunch& a, int G, int Hq, int Hkv,
                              const Splits& splits = Splits(), const Ends& ends = Ends()) {
  __shared__ Partial s_part[NT];
  __shared__ int last;
  const int slot = splits.slot(), g = blockIdx.y, head = slot * Hkv + g;
  const int nsplit = splits(a, slot);
  // This thread's partial stores are written before the workgroup counts
  // itself: the wait is issued as an asm statement that clobbers memory, so
  // the compiler cannot move the stores (relaxed atomics) past it either.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const int prev = __hip_atomic_fetch_add(a.arrivals + head, 1, __ATOMIC_RELAXED,
                                            __HIP_MEMORY_SCOPE_AGENT);
    last = prev == nsplit - 1;
    if (last)
      __hip_atomic_store(a.arrivals + head, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!last) return;
  const int t = threadIdx.x;
  const float* ml = a.ws_ml + static_cast<int64_t>(head) * a.split_stride * G * 2;
  const float* po = a.ws_o + static_cast<int64_t>(head) * a.split_stride * G * kHeadDim;
  E* out = static_cast<E*>(a.out) + (static_cast<int64_t>(slot) * Hq + g * G) * kHeadDim;
  const int pairs = G * (kHeadDim / 2);
  const int parts = max(1, min(NT / pairs, (nsplit + 3) / 4));
  const int per = (nsplit + parts - 1) / parts;
  const auto gather_by = [&](auto batch, int item, int lo, int hi) {
    constexpr int kBatch = decltype(batch)::value;
    const int q = item / (kHeadDim / 2), c = 2 * (item % (kHeadDim / 2));
    Partial p{kNoScore, 0.f, 0.f, 0.f};
    for (int s0 = lo; s0 < hi; s0 += kBatch) {
      float m[kBatch], l[kBatch], x[kBatch], y[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int row = min(s0 + j, hi - 1) * G + q;
        load_shared_level(ml + 2 * row, m[j], l[j]);
        load_shared_level(po + row * kHeadDim + c, x[j], y[j]);
      }
      float mx = p.m;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) mx = fmaxf(mx, m[j]);
      const float keep = ends.exp2(p.m - mx);
      p.m = mx;
      p.l *= keep;
      p.o0 *= keep;
      p.o1 *= keep;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const float w = s0 + j < hi ? ends.exp2(m[j] - mx) : 0.f;
        p.l += w * l[j];
        p.o0 += w * x[j];
        p.o1 += w * y[j];
      }
    }
    return p;
  };
  const auto gather = [&](int item, int lo, int hi) {
    return hi - lo <= 4 ? gather_by(std::integral_constant<int, 4>{}, item, lo, hi)
                        : gather_by(std::integral_constant<int, 16>{}, item, lo, hi);
  };
  const auto put = [&](int item, const Partial& p) {
    const float inv = 1.f / p.l;
    if constexpr (Ends::kKeeps) {
      if (item % (kHeadDim / 2) == 0) ends.keep(item / (kHeadDim / 2), p.m, p.l);
    }
    if constexpr (sizeof(E) == 2) {
      *reinterpret_cast<uint32_t*>(out + 2 * item) =
          f32_to_bf16(p.o0 * inv) | static_cast<uint32_t>(f32_to_bf16(p.o1 * inv)) << 16;
    } else {
      *reinterpret_cast<float2*>(out + 2 * item) = make_float2(p.o0 * inv, p.o1 * inv);
    }
  };
  if (pairs > NT && nsplit > 4 && nsplit <= 12) {
    for (int item = t; item < pairs; item += NT)
      put(item, gather_by(std::integral_constant<int, 12>{}, item, 0, nsplit));
    return;
  }
  if (parts == 1) {
    for (int item = t; item < pairs; item += NT) put(item, gather(item, 0, nsplit));
    return;
  }
  const int part = t / pairs;
  if (part < parts && part * per < nsplit)
    s_part[t] = gather(t % pairs, part * per, min(part * per + per, nsplit));
  __syncthreads();
  if (t < pairs) {
    Partial p = s_part[t];
    for (int k = 1; k < parts && k * per < nsplit; ++k) {
      const Partial r = s_part[k * pairs + t];
      const float mx = fmaxf(p.m, r.m);
      const float wp = ends.exp2(p.m - mx), wr = ends.exp2(r.m - mx);
      p = Partial{mx, p.l * wp + r.l * wr, p.o0 * wp + r.o0 * wr, p.o1 * wp + r.o1 * wr};
    }
    put(t, p);
  }
}

struct BlockRegs {
  u32x4 k[2][4];  // [S tile][k-step]
  u32x4 v[8];     // [16-channel tile]
};

// Offsets (in elements) of this lane's operand loads within a 32-key block.
struct LaneMap {
  int krow[2];   // key row within the block for S tile 0 / 1
  int kcol;      // first channel of the lane's 16-byte chunk at k-step 0
  int vrow;      // first key row of the lane's value tile
  int vch;       // channel within each 16-channel tile
};

__device__ __forceinline__ LaneMap lane_map() {
  const int lane = threadIdx.x & 63, r = lane & 15, grp = lane >> 4;
  LaneMap m;
  m.krow[0] = 8 * (r >> 2) + (r & 3);
  m.krow[1] = 8 * (r >> 2) + 4 + (r & 3);
  m.kcol = 8 * grp;
  m.vrow = 8 * grp;
  m.vch = r;
  return m;
}

// Rows kb .. kb+31 from the key rows at Kr and the value tiles at Vr (the
// head's region; in the paged layout the block's page, with kb = 0).
__device__ __forceinline__ void load_block(BlockRegs& b, const uint16_t* Kr,
                                           const uint16_t* Vr, int kb,
                                           const LaneMap& lm) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint16_t* row = Kr + static_cast<int64_t>(kb + lm.krow[t]) * kHeadDim + lm.kcol;
#pragma unroll
    for (int s = 0; s < 4; ++s) b.k[t][s] = ld16(row + 32 * s);
  }
  const uint16_t* vt = Vr + static_cast<int64_t>(kb + lm.vrow) * kHeadDim + lm.vch * 8;
#pragma unroll
  for (int u = 0; u < 8; ++u) b.v[u] = ld16_stream(vt + 16 * 8 * u);
}

struct Softmax {
  float m;      // running max of the scores (log2 units, unless said otherwise), per query
  float l;      // this lane's share of the running sum
  f32x4 acc[8]; // O^T tile u: channels 16u + 4*grp + i, query lane & 15
};

// One 32-key block.  `limit`: keys with index >= limit (block-relative) are
// masked out (32 for a full block); with MASKED, so are the keys whose bit is
// set in `dropped`.
template <bool MASKED = false>
__device__ __forceinline__ void compute_block(Softmax& st, const BlockRegs& b,
                                              const bf16x8 (&qop)[4],
                                              float scale_log2, int limit,
                                              uint32_t dropped = 0) {
  f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(b.k[0][s]), qop[s], s0, 0, 0, 0);
    s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(b.k[1][s]), qop[s], s1, 0, 0, 0);
  }
  const int grp = (threadIdx.x & 63) >> 4;
  float x[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = s0[i] * scale_log2;
    x[4 + i] = s1[i] * scale_log2;
  }
  if (limit < 32) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (8 * grp + e >= limit) x[e] = kNegInf;
  }
  if constexpr (MASKED) {
    if (dropped) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if ((dropped >> (8 * grp + e)) & 1u) x[e] = kNegInf;
    }
  }
  float bm = x[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) bm = fmaxf(bm, x[e]);
  bm = fmaxf(bm, __shfl_xor(bm, 16, 64));
  bm = fmaxf(bm, __shfl_xor(bm, 32, 64));
  const float mn = fmaxf(st.m, bm);
  const float alpha = exp2f(st.m - mn);
  // P = hi + lo, both bf16, so the weights keep ~16 significant bits through
  // the bf16 MFMA (the remainder of a bf16 rounding is exact in fp32)
  bf16x8 p_hi, p_lo;
  float psum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float pf = exp2f(x[e] - mn);
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

// First of the four channels that vector u of the accumulators holds.
struct RowChannels {
  static __device__ __forceinline__ int first(int u, int grp) { return 16 * u + 4 * grp; }
};

// The W wavefronts of a work item merge their states in LDS; an item that is
// a whole head writes the normalised output, another one its partial (merged
// by the head's last item, or with FUSED false by combine_kernel).
template <typename E, int W, bool FUSED, typename Splits = DenseSplits,
          typename Channels = RowChannels, typename Ends = Log2Ends>
__device__ __forceinline__ void finish_item(const AttnLaunch& a, const Work& w, int wave,
                                            int qi, int grp, const Softmax& st, int G, int Hq, int Hkv,
                                            float (&s_m)[W][kMaxGroup],
                                            float (&s_l)[W][kMaxGroup],
                                            float (&s_o)[W][kMaxGroup][kHeadDim],
                                            const Splits& splits = Splits(),
                                            const Ends& ends = Ends()) {
  const int head = w.slot * Hkv + w.g;
  const int64_t item = static_cast<int64_t>(head) * a.split_stride + w.split;
  E* out = static_cast<E*>(a.out);
  // merge the W wavefronts in LDS
  if (qi < G) {
#pragma unroll
    for (int u = 0; u < 8; ++u)
      *reinterpret_cast<f32x4*>(&s_o[wave][qi][Channels::first(u, grp)]) = st.acc[u];
    if (grp == 0) {
      s_m[wave][qi] = st.m;
      s_l[wave][qi] = st.l;
    }
  }
  __syncthreads();
  for (int idx = threadIdx.x; idx < G * kHeadDim; idx += 64 * W) {
    const int q = idx / kHeadDim, c = idx % kHeadDim;
    float mx = kNegInf;
#pragma unroll
    for (int v = 0; v < W; ++v) mx = fmaxf(mx, s_m[v][q]);
    float lsum = 0.f, o = 0.f;
#pragma unroll
    for (int v = 0; v < W; ++v) {
      const float sc = ends.exp2(s_m[v][q] - mx);
      lsum += s_l[v][q] * sc;
      o += s_o[v][q][c] * sc;
    }
    if (w.nsplit == 1) {
      if constexpr (Ends::kKeeps) {
        if (c == 0) ends.keep(q, mx, lsum);
      }
      const int64_t idx_out = (static_cast<int64_t>(w.slot) * Hq + w.g * G + q) * kHeadDim + c;
      if constexpr (sizeof(E) == 2) out[idx_out] = f32_to_bf16(o / lsum);
      else out[idx_out] = o / lsum;
    } else if constexpr (FUSED) {
      store_shared_level(a.ws_o + (item * G + q) * kHeadDim + c, o);
      if (c == 0) {
        store_shared_level(a.ws_ml + (item * G + q) * 2, mx);
        store_shared_level(a.ws_ml + (item * G + q) * 2 + 1, lsum);
      }
    } else {
      a.ws_o[(item * G + q) * kHeadDim + c] = o;
      if (c == 0) {
        a.ws_ml[(item * G + q) * 2] = mx;
        a.ws_ml[(item * G + q) * 2 + 1] = lsum;
      }
    }
  }
  if constexpr (FUSED) {
    if (w.nsplit > 1) merge_if_last<E, 64 * W>(a, G, Hq, Hkv, splits, ends);
  }
}

}  // namespace
}  // namespace ra
