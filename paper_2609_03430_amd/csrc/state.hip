// Device-side sequence state and row transfer kernels.
//
// The per-slot metadata lives in device memory so that a decode step's
// kernels need no host round trip: the end-of-step kernel advances the step
// counter and applies the periodic trigger (Appendix F: every evict_every
// steps, once the evictable rows exceed the budget) by writing an eviction
// plan that the eviction kernel consumes.  The host library replays the
// same integer rules on its mirror to decide which launches to issue.
#include "e4m3.h"
#include "ra_internal.h"

namespace ra {
namespace {

using u32x4 = uint32_t __attribute__((ext_vector_type(4)));

__global__ void zero_words_kernel(uint32_t* p, int64_t n) {
  for (int64_t i = blockIdx.x * int64_t(blockDim.x) + threadIdx.x; i < n;
       i += int64_t(gridDim.x) * blockDim.x)
    p[i] = 0u;
}

__global__ void seq_set_kernel(SeqMeta* meta, int slot, SeqMeta v) {
  if (threadIdx.x == 0) meta[slot] = v;
}

// Applies the trigger rule to a sequence that has just completed `n_steps`
// more steps (n_steps never crosses a multiple of `every` before its end).
__device__ __forceinline__ void plan(SeqMeta& M, int r, bool at_trigger) {
  M.due = 0;
  if (at_trigger && M.len - M.prompt_len - r > M.k_keep) {
    M.due = 1;
    M.plan_len = M.len;
    M.plan_event = M.event;
    M.len = M.prompt_len + M.k_keep + r;
    M.event += 1;
  }
}

__global__ void advance_kernel(SeqMeta* meta, int lo, int hi, int n_steps,
                               int r, int every) {
  const int s = lo + blockIdx.x * blockDim.x + threadIdx.x;
  if (s >= hi) return;
  SeqMeta M = meta[s];
  if (!M.active) return;
  M.step += n_steps;
  M.len += n_steps;
  plan(M, r, every > 0 && M.step % every == 0);   // every = 0: never triggers
  meta[s] = M;
}

// advance_kernel over the runs between triggers that n_steps steps hold.
__global__ void replay_steps_kernel(SeqMeta* meta, int lo, int hi, int n_steps, int r,
                                    int every) {
  const int s = lo + blockIdx.x * blockDim.x + threadIdx.x;
  if (s >= hi) return;
  SeqMeta M = meta[s];
  if (!M.active) return;
  for (int left = n_steps; left > 0;) {
    const int run = min(left, every - M.step % every);
    M.step += run;
    M.len += run;
    plan(M, r, M.step % every == 0);
    left -= run;
  }
  meta[s] = M;
}

// The plan rule applied now to every active slot of [lo, hi).
__global__ void plan_range_kernel(SeqMeta* meta, int lo, int hi, int r) {
  const int s = lo + blockIdx.x * blockDim.x + threadIdx.x;
  if (s >= hi) return;
  SeqMeta M = meta[s];
  if (!M.active) return;
  plan(M, r, true);
  meta[s] = M;
}

__global__ void plan_now_kernel(SeqMeta* meta, int slot, int r) {
  if (threadIdx.x != 0) return;
  SeqMeta M = meta[slot];
  if (!M.active) return;
  plan(M, r, true);
  meta[slot] = M;
}

__global__ void mark_pending_kernel(SeqMeta* meta, int lo, int hi) {
  const int s = lo + blockIdx.x * blockDim.x + threadIdx.x;
  if (s >= hi) return;
  if (meta[s].active && meta[s].due == 1) meta[s].due = kDueMovePending;
}

__global__ void clear_pending_kernel(SeqMeta* meta, int lo, int hi) {
  const int s = lo + blockIdx.x * blockDim.x + threadIdx.x;
  if (s >= hi) return;
  if (meta[s].due == kDueMovePending) meta[s].due = 0;
}

// Positions lp+step .. lp+step+run-1 into rows len .. len+run-1 of every
// head of every active slot (rows themselves are not touched).
// Grid: (slots, L * Hkv).
template <bool PAGED>
__global__ void append_positions_kernel(const SeqMeta* meta, int32_t* pos, int lo,
                                        int run, Paging pg) {
  const int slot = lo + blockIdx.x;
  const SeqMeta& M = meta[slot];
  if (!M.active) return;
  const RowMap rm = row_map(M, slot, blockIdx.y, pg);
  for (int i = threadIdx.x; i < run; i += blockDim.x)
    pos[pool_row<PAGED>(rm, M.len + i)] = M.prompt_len + M.step + i;
}

// Row-major source rows [L*Hkv][len][128] into the cache layout of rows
// [0, len) of each head; rows of a partly filled last value tile are
// zeroed.  Grid: (ceil(len/64), L*Hkv).  A 64-row chunk may straddle two
// pages of 32 rows, so rows are mapped one by one (value tiles of 8 rows
// never straddle a page).
template <typename E, bool PAGED>
__global__ void write_rows_kernel(SeqMeta M, int slot, int len, Paging pg,
                                  const E* __restrict__ k_src,
                                  const E* __restrict__ v_src,
                                  const int32_t* __restrict__ pos_src,
                                  E* __restrict__ kpool, E* __restrict__ vpool,
                                  int32_t* __restrict__ pos) {
  constexpr int kEpu = 16 / sizeof(E);
  const int lg = blockIdx.y;
  const int j0 = blockIdx.x * 64;
  const RowMap rm = row_map(M, slot, lg, pg);
  const int64_t src0 = static_cast<int64_t>(lg) * len;
  if (pos) {
    for (int i = threadIdx.x; i < 64; i += blockDim.x) {
      const int j = j0 + i;
      if (j < len) pos[pool_row<PAGED>(rm, j)] = pos_src ? pos_src[src0 + j] : j;
    }
  }
  if (!k_src) return;
  constexpr int kUnitsRow = kHeadDim / kEpu;
  for (int u = threadIdx.x; u < 64 * kUnitsRow; u += blockDim.x) {
    const int j = j0 + u / kUnitsRow, col = u % kUnitsRow;
    if (j < len)
      *reinterpret_cast<u32x4*>(kpool + pool_row<PAGED>(rm, j) * kHeadDim + col * kEpu) =
          *reinterpret_cast<const u32x4*>(k_src + (src0 + j) * kHeadDim + col * kEpu);
  }
  // values: each output 16-byte unit holds kEpu consecutive rows of one channel
  constexpr int kUnitsCh = 8 / kEpu;
  for (int u = threadIdx.x; u < 8 * kHeadDim * kUnitsCh; u += blockDim.x) {
    const int tile = u / (kHeadDim * kUnitsCh);
    const int rem = u % (kHeadDim * kUnitsCh);
    const int ch = rem / kUnitsCh, part = rem % kUnitsCh;
    const int jt = j0 + tile * 8;
    if (jt >= len) continue;
    E e[kEpu];
#pragma unroll
    for (int x = 0; x < kEpu; ++x) {
      const int j = jt + part * kEpu + x;
      e[x] = j < len ? v_src[(src0 + j) * kHeadDim + ch] : E(0);
    }
    u32x4 w;
    __builtin_memcpy(&w, e, 16);
    *reinterpret_cast<u32x4*>(vpool + pool_row<PAGED>(rm, jt) * kHeadDim + ch * 8 +
                              part * kEpu) = w;
  }
}

// Rows [0, len) of heads lg, lg + 1, .. to row-major outputs [heads][len][128].
// Grid: (ceil(len/32), 2, heads): keys, values; 128 threads.  One head is a short
// copy (1.6 MB at 3,136 bf16 rows), so its time is the latency of a load and a
// store: every thread issues all its loads before its stores, in 16-byte units
// (outputs are 16-byte aligned, as all device pointers of the interface).  A thread takes kEpu channels x kEpu rows
// of a value tile and transposes them in registers.  Element by element it
// took 23 us per 3,136-row head, in 16-byte units 5.5, keys and values side by
// side 4.5.
constexpr int kReadRows = 32;
template <typename E, bool PAGED>
__global__ __launch_bounds__(128) void read_rows_kernel(SeqMeta M, int slot, int lg, int len,
                                                        Paging pg, const E* __restrict__ kpool,
                                                        const E* __restrict__ vpool,
                                                        E* __restrict__ k_out,
                                                        E* __restrict__ v_out) {
  constexpr int kEpu = 16 / sizeof(E);
  constexpr int kUnitsRow = kHeadDim / kEpu;
  constexpr int kPer = kReadRows * kUnitsRow / 128;       // key units per thread
  const RowMap rm = row_map(M, slot, lg + blockIdx.z, pg);
  const int64_t out0 = static_cast<int64_t>(blockIdx.z) * len;
  const int j0 = blockIdx.x * kReadRows;                  // 32 rows lie in one page
  const int64_t row0 = pool_row<PAGED>(rm, j0);
  if (blockIdx.y == 0) {
    if (!k_out) return;
    u32x4 k[kPer];
    const u32x4* src = reinterpret_cast<const u32x4*>(kpool + row0 * kHeadDim);
    u32x4* dst = reinterpret_cast<u32x4*>(k_out + (out0 + j0) * kHeadDim);
    const int n = min(kReadRows, len - j0) * kUnitsRow;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int u = threadIdx.x + i * 128;
      if (u < n) k[i] = src[u];
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int u = threadIdx.x + i * 128;
      if (u < n) dst[u] = k[i];
    }
    return;
  }
  if (!v_out) return;
  for (int u = threadIdx.x; u < kReadRows / kEpu * kUnitsRow; u += 128) {
    const int ch = u % kUnitsRow * kEpu, r = u / kUnitsRow * kEpu, j = j0 + r;
    if (j >= len) continue;
    // channel ch + c: rows r .. r + kEpu - 1 (of one 8-row tile)
    E in[kEpu][kEpu];
    const E* src = vpool + (row0 + (r & ~7)) * kHeadDim + ch * 8 + (r & 7);
#pragma unroll
    for (int c = 0; c < kEpu; ++c) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(src + c * 8);
      __builtin_memcpy(in[c], &x, 16);
    }
#pragma unroll
    for (int e = 0; e < kEpu; ++e) {
      E out[kEpu];
#pragma unroll
      for (int c = 0; c < kEpu; ++c) out[c] = in[c][e];
      u32x4 x;
      __builtin_memcpy(&x, out, 16);
      if (j + e < len)
        *reinterpret_cast<u32x4*>(v_out + (out0 + j + e) * kHeadDim + ch) = x;
    }
  }
}

// ---- e4m3 rows (e4m3.h) ------------------------------------------------------------

// Sixteen lanes take an 8-row tile of keys or of values, eight channels each: the
// largest magnitude of a row is joined over the sixteen lanes, and the codes are
// packed in the order in which they are stored, along the channels for keys and along
// the rows for values, so that the values' transposition costs nothing; four lanes
// exchange 16-byte units so that their stores are contiguous.
// Bound by HBM, 256 B read and 129 written per row, while the conversions stay few: the
// largest magnitudes are found on packed 16-bit words, and rows whose codes may need
// their range enforced (no finite row below 2^127 does) take a branch of their own.
constexpr int kTileLanes = 16;
constexpr int kQuantRows = 256 / kTileLanes * 8;   // rows per workgroup of 256 threads

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Eight bf16 magnitudes' largest (its bits; a NaN's are the largest of all).
__device__ __forceinline__ uint32_t largest_magnitude(u32x4 w) {
  u16x2 m[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = w[i] & 0x7fff7fffu;
    __builtin_memcpy(&m[i], &a, 4);
  }
  const u16x2 x = __builtin_elementwise_max(__builtin_elementwise_max(m[0], m[1]),
                                            __builtin_elementwise_max(m[2], m[3]));
  return max(static_cast<uint32_t>(x[0]), static_cast<uint32_t>(x[1]));
}

// Four lanes' 16-byte units transposed: lane b's unit i becomes lane i's unit b.
template <int XOR, int CTRL>
__device__ __forceinline__ void exchange_units(u32x4& a, u32x4& b) {
  const bool upper = threadIdx.x & XOR;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const uint32_t give = upper ? a[d] : b[d];
    const uint32_t got = static_cast<uint32_t>(
        __builtin_amdgcn_update_dpp(0, static_cast<int>(give), CTRL, 0xf, 0xf, false));
    a[d] = upper ? got : a[d];
    b[d] = upper ? b[d] : got;
  }
}
__device__ __forceinline__ void transpose_units(u32x4 (&u)[4]) {
  exchange_units<1, 0xB1>(u[0], u[1]);
  exchange_units<1, 0xB1>(u[2], u[3]);
  exchange_units<2, 0x4E>(u[0], u[2]);
  exchange_units<2, 0x4E>(u[1], u[3]);
}

// Row-major bf16 rows [L * Hkv][len][128] into rows [0, len) of each head.
// Grid: (ceil(len / 128), L * Hkv, 2): keys (and positions), values.
template <bool PAGED>
__global__ __launch_bounds__(256) void write_rows_e4m3_kernel(
    SeqMeta M, int slot, int len, Paging pg, const uint16_t* __restrict__ k_src,
    const uint16_t* __restrict__ v_src, const int32_t* __restrict__ pos_src,
    uint8_t* __restrict__ kpool, uint8_t* __restrict__ vpool, uint8_t* __restrict__ kscale,
    uint8_t* __restrict__ vscale, int32_t* __restrict__ pos) {
  const int lg = blockIdx.y;
  const bool keys = blockIdx.z == 0;
  const RowMap rm = row_map(M, slot, lg, pg);
  const int64_t src0 = static_cast<int64_t>(lg) * len;
  if (pos && keys) {
    for (int i = threadIdx.x; i < kQuantRows; i += 256) {
      const int j = static_cast<int>(blockIdx.x) * kQuantRows + i;
      if (j < len) pos[pool_row<PAGED>(rm, j)] = pos_src ? pos_src[src0 + j] : j;
    }
  }
  const uint16_t* src = keys ? k_src : v_src;
  if (!src) return;
  const int c8 = threadIdx.x % kTileLanes;
  const int jt = static_cast<int>(blockIdx.x) * kQuantRows + threadIdx.x / kTileLanes * 8;
  if (jt >= len) return;                       // (all sixteen lanes of the tile)
  src += (src0 + jt) * kHeadDim + 8 * c8;
  u32x4 in[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    in[e] = u32x4{0u, 0u, 0u, 0u};
    if (jt + e < len)
      in[e] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + e * kHeadDim));
  }
  uint32_t amax[8], top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    amax[e] = max_over_row16(largest_magnitude(in[e]));
    top = max(top, amax[e]);
  }
  // rows past 1.75 * 2^127, infinities or NaNs
  const bool enforce = top > 0x7f60u;
  uint32_t byte[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    uint32_t m = amax[e] << 16;
    if (enforce) {
      m = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        m = max(m, max(row_magnitude(bf16_low(in[e][i])), row_magnitude(bf16_high(in[e][i]))));
      m = max_over_row16(m);
    }
    byte[e] = e4m3_scale_byte(m);
  }
  const int64_t row0 = pool_row<PAGED>(rm, jt);          // a tile lies in one page
  if (c8 == 0) {
    uint64_t scales = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) scales |= static_cast<uint64_t>(byte[e]) << (8 * e);
    *reinterpret_cast<uint64_t*>((keys ? kscale : vscale) + row0) = scales;
  }
  if (keys) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint2 w;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t a = in[e][2 * h], b = in[e][2 * h + 1];
        uint32_t c;
        if (enforce) {
          const float inv = e4m3_inverse(byte[e]);
          c = e4m3_pack2<true>(
              e4m3_clamp(bf16_low(b) * inv, byte[e]), e4m3_clamp(bf16_high(b) * inv, byte[e]),
              e4m3_pack2<false>(e4m3_clamp(bf16_low(a) * inv, byte[e]),
                                e4m3_clamp(bf16_high(a) * inv, byte[e]), 0u));
        } else {
          const float scale = e4m3_scale(byte[e]);
          bf16x2 x, y;
          __builtin_memcpy(&x, &a, 4);
          __builtin_memcpy(&y, &b, 4);
          i16x2 r = {0, 0};
          r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, x, scale, false);
          r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, y, scale, true);
          __builtin_memcpy(&c, &r, 4);
        }
        (h ? w.y : w.x) = c;
      }
      if (jt + e < len)
        *reinterpret_cast<uint2*>(kpool + (row0 + e) * kHeadDim + 8 * c8) = w;
    }
    return;
  }
  u32x4 units[4];                              // two channels of eight rows each
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float y[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const uint32_t w = in[e + x][i];
          y[x] = (h ? bf16_high(w) : bf16_low(w)) * e4m3_inverse(byte[e + x]);
          if (enforce) y[x] = e4m3_clamp(y[x], byte[e + x]);
        }
        units[i][2 * h + e / 4] = e4m3_pack2<true>(y[2], y[3], e4m3_pack2<false>(y[0], y[1], 0u));
      }
    }
  }
  // rows past len are zero codes
  transpose_units(units);
  uint8_t* dst = vpool + row0 * kHeadDim + 64 * (c8 & ~3) + 16 * (c8 & 3);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *reinterpret_cast<u32x4*>(dst + 64 * i) = units[i];
}

// Rows [0, len) of heads lg, lg + 1, .. to row-major bf16 outputs [heads][len][128],
// the values that the rows stand for.  Grid: (ceil(len / 128), 2, heads).
template <bool PAGED>
__global__ __launch_bounds__(256) void read_rows_e4m3_kernel(
    SeqMeta M, int slot, int lg, int len, Paging pg, const uint8_t* __restrict__ kpool,
    const uint8_t* __restrict__ vpool, const uint8_t* __restrict__ kscale,
    const uint8_t* __restrict__ vscale, uint16_t* __restrict__ k_out,
    uint16_t* __restrict__ v_out) {
  const bool keys = blockIdx.y == 0;
  uint16_t* out = keys ? k_out : v_out;
  const int c8 = threadIdx.x % kTileLanes;
  const int jt = static_cast<int>(blockIdx.x) * kQuantRows + threadIdx.x / kTileLanes * 8;
  if (!out || jt >= len) return;
  const RowMap rm = row_map(M, slot, lg + blockIdx.z, pg);
  const int64_t row0 = pool_row<PAGED>(rm, jt);
  out += (static_cast<int64_t>(blockIdx.z) * len + jt) * kHeadDim + 8 * c8;
  const uint64_t scales = *reinterpret_cast<const uint64_t*>((keys ? kscale : vscale) + row0);
  const auto scale_of = [&](int e) {
    return e4m3_scale(static_cast<uint32_t>(scales >> (8 * e)) & 255u);
  };
  if (keys) {
    uint2 w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (jt + e < len)
        w[e] = *reinterpret_cast<const uint2*>(kpool + (row0 + e) * kHeadDim + 8 * c8);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (jt + e >= len) continue;
      const float s = scale_of(e);
      u32x4 o;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t c = i ? w[e].y : w[e].x;
        const f32x2 a = e4m3_unpack2<false>(c), b = e4m3_unpack2<true>(c);
        o[2 * i] = bf16_pack_exact(a[0] * s, a[1] * s);
        o[2 * i + 1] = bf16_pack_exact(b[0] * s, b[1] * s);
      }
      *reinterpret_cast<u32x4*>(out + e * kHeadDim) = o;
    }
    return;
  }
  u32x4 w[4];                                  // two channels of eight rows each
  const u32x4* src = reinterpret_cast<const u32x4*>(vpool + row0 * kHeadDim + 64 * c8);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = src[i];
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const float s0 = scale_of(e), s1 = scale_of(e + 1);
    f32x2 x[8];                                // rows e, e + 1 of the eight channels
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const uint32_t word = w[c / 2][c % 2 * 2 + e / 4];
      x[c] = e & 2 ? e4m3_unpack2<true>(word) : e4m3_unpack2<false>(word);
    }
    u32x4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = bf16_pack_exact(x[2 * i][0] * s0, x[2 * i + 1][0] * s0);
      b[i] = bf16_pack_exact(x[2 * i][1] * s1, x[2 * i + 1][1] * s1);
    }
    if (jt + e < len) *reinterpret_cast<u32x4*>(out + e * kHeadDim) = a;
    if (jt + e + 1 < len) *reinterpret_cast<u32x4*>(out + (e + 1) * kHeadDim) = b;
  }
}

template <bool PAGED>
__global__ void export_positions_kernel(SeqMeta M, int slot, int len, Paging pg,
                                        const int32_t* __restrict__ pos,
                                        int32_t* __restrict__ out) {
  const int lg = blockIdx.y;
  const int j = blockIdx.x * blockDim.x + threadIdx.x;
  const RowMap rm = row_map(M, slot, lg, pg);
  if (j < len) out[static_cast<int64_t>(lg) * len + j] = pos[pool_row<PAGED>(rm, j)];
}

struct TableBatch {
  TableEntry e[kTableBatch];
};

// Block-table entries chosen by the host's page allocator.
__global__ void table_set_kernel(int32_t* tables, int pages_per_seq, TableBatch b, int n) {
  const int i = threadIdx.x;
  if (i < n)
    tables[static_cast<int64_t>(b.e[i].slot) * pages_per_seq + b.e[i].index] = b.e[i].group;
}

}  // namespace

hipError_t launch_zero_words(uint32_t* p, int64_t n_words, hipStream_t s) {
  if (n_words <= 0) return hipSuccess;
  const int64_t blocks = std::min<int64_t>((n_words + 255) / 256, 4096);
  hipLaunchKernelGGL(zero_words_kernel, dim3(blocks), dim3(256), 0, s, p, n_words);
  return hipGetLastError();
}

hipError_t launch_seq_set(SeqMeta* meta, int slot, const SeqMeta& v, hipStream_t s) {
  hipLaunchKernelGGL(seq_set_kernel, dim3(1), dim3(64), 0, s, meta, slot, v);
  return hipGetLastError();
}

hipError_t launch_advance(SeqMeta* meta, int slot_lo, int slot_hi, int n_steps,
                          int r, int every, hipStream_t s) {
  const int n = slot_hi - slot_lo;
  if (n <= 0) return hipSuccess;
  hipLaunchKernelGGL(advance_kernel, dim3((n + 255) / 256), dim3(256), 0, s,
                     meta, slot_lo, slot_hi, n_steps, r, every);
  return hipGetLastError();
}

hipError_t launch_replay_steps(SeqMeta* meta, int slot_lo, int slot_hi, int n_steps, int r,
                               int every, hipStream_t s) {
  const int n = slot_hi - slot_lo;
  if (n <= 0) return hipSuccess;
  hipLaunchKernelGGL(replay_steps_kernel, dim3((n + 255) / 256), dim3(256), 0, s, meta, slot_lo,
                     slot_hi, n_steps, r, every);
  return hipGetLastError();
}

hipError_t launch_plan_now(SeqMeta* meta, int slot, int r, hipStream_t s) {
  hipLaunchKernelGGL(plan_now_kernel, dim3(1), dim3(64), 0, s, meta, slot, r);
  return hipGetLastError();
}

hipError_t launch_plan_range(SeqMeta* meta, int slot_lo, int slot_hi, int r, hipStream_t s) {
  if (slot_hi <= slot_lo) return hipSuccess;
  const int n = slot_hi - slot_lo;
  hipLaunchKernelGGL(plan_range_kernel, dim3((n + 255) / 256), dim3(256), 0, s, meta,
                     slot_lo, slot_hi, r);
  return hipGetLastError();
}

hipError_t launch_append_positions(const Shape& sh, const SeqMeta* meta, int32_t* pos,
                                   int slot_lo, int slot_hi, int run, hipStream_t s) {
  if (slot_hi <= slot_lo || run <= 0) return hipSuccess;
  const dim3 grid(slot_hi - slot_lo, sh.L * sh.Hkv);
  if (sh.pg.tables)
    hipLaunchKernelGGL(append_positions_kernel<true>, grid, dim3(256), 0, s, meta, pos,
                       slot_lo, run, sh.pg);
  else
    hipLaunchKernelGGL(append_positions_kernel<false>, grid, dim3(256), 0, s, meta, pos,
                       slot_lo, run, sh.pg);
  return hipGetLastError();
}

template <typename E>
void write_rows_t(const Shape& sh, const SeqMeta& M, int slot, int len, const void* k_src,
                  const void* v_src, const int32_t* pos_src, void* kpool, void* vpool,
                  int32_t* pos, hipStream_t s) {
  const dim3 grid((len + 63) / 64, sh.L * sh.Hkv);
  const E* k = static_cast<const E*>(k_src);
  const E* v = static_cast<const E*>(v_src);
  if (sh.pg.tables)
    hipLaunchKernelGGL((write_rows_kernel<E, true>), grid, dim3(256), 0, s, M, slot, len,
                       sh.pg, k, v, pos_src, static_cast<E*>(kpool), static_cast<E*>(vpool),
                       pos);
  else
    hipLaunchKernelGGL((write_rows_kernel<E, false>), grid, dim3(256), 0, s, M, slot, len,
                       sh.pg, k, v, pos_src, static_cast<E*>(kpool), static_cast<E*>(vpool),
                       pos);
}

void write_rows_e4m3(const Shape& sh, const SeqMeta& M, int slot, int len, const void* k_src,
                     const void* v_src, const int32_t* pos_src, void* kpool, void* vpool,
                     int32_t* pos, hipStream_t s) {
  const dim3 grid((len + kQuantRows - 1) / kQuantRows, sh.L * sh.Hkv, 2);
  const auto kernel = sh.pg.tables ? write_rows_e4m3_kernel<true> : write_rows_e4m3_kernel<false>;
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, M, slot, len, sh.pg,
                     static_cast<const uint16_t*>(k_src), static_cast<const uint16_t*>(v_src),
                     pos_src, static_cast<uint8_t*>(kpool), static_cast<uint8_t*>(vpool),
                     sh.k_scale, sh.v_scale, pos);
}

hipError_t launch_write_rows(const Shape& sh, const SeqMeta& M, int slot, int len,
                             const void* k_src, const void* v_src,
                             const int32_t* pos_src, void* kpool, void* vpool,
                             int32_t* pos, hipStream_t s) {
  if (len <= 0) return hipSuccess;
  if (sh.dtype == 2)
    write_rows_e4m3(sh, M, slot, len, k_src, v_src, pos_src, kpool, vpool, pos, s);
  else if (sh.dtype == 1)
    write_rows_t<uint16_t>(sh, M, slot, len, k_src, v_src, pos_src, kpool, vpool, pos, s);
  else
    write_rows_t<float>(sh, M, slot, len, k_src, v_src, pos_src, kpool, vpool, pos, s);
  return hipGetLastError();
}

template <typename E>
void read_rows_t(const Shape& sh, const SeqMeta& M, int slot, int lg, int heads, int len,
                 const void* kpool, const void* vpool, void* k_out, void* v_out,
                 hipStream_t s) {
  const dim3 grid((len + kReadRows - 1) / kReadRows, 2, heads);
  const E* k = static_cast<const E*>(kpool);
  const E* v = static_cast<const E*>(vpool);
  if (sh.pg.tables)
    hipLaunchKernelGGL((read_rows_kernel<E, true>), grid, dim3(128), 0, s, M, slot, lg, len,
                       sh.pg, k, v, static_cast<E*>(k_out), static_cast<E*>(v_out));
  else
    hipLaunchKernelGGL((read_rows_kernel<E, false>), grid, dim3(128), 0, s, M, slot, lg, len,
                       sh.pg, k, v, static_cast<E*>(k_out), static_cast<E*>(v_out));
}

// Heads lg .. lg + heads - 1 (at most 65,535 of them: a grid's z).
hipError_t read_heads(const Shape& sh, const SeqMeta& M, int slot, int lg, int heads, int len,
                      const void* kpool, const void* vpool, void* k_out, void* v_out,
                      hipStream_t s) {
  if (len <= 0) return hipSuccess;
  if (sh.dtype == 2) {
    const dim3 grid((len + kQuantRows - 1) / kQuantRows, 2, heads);
    const auto kernel = sh.pg.tables ? read_rows_e4m3_kernel<true> : read_rows_e4m3_kernel<false>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, M, slot, lg, len, sh.pg,
                       static_cast<const uint8_t*>(kpool), static_cast<const uint8_t*>(vpool),
                       sh.k_scale, sh.v_scale, static_cast<uint16_t*>(k_out),
                       static_cast<uint16_t*>(v_out));
  } else if (sh.dtype == 1) {
    read_rows_t<uint16_t>(sh, M, slot, lg, heads, len, kpool, vpool, k_out, v_out, s);
  } else {
    read_rows_t<float>(sh, M, slot, lg, heads, len, kpool, vpool, k_out, v_out, s);
  }
  return hipGetLastError();
}

hipError_t launch_read_rows(const Shape& sh, const SeqMeta& M, int slot, int lg, int len,
                            const void* kpool, const void* vpool, void* k_out,
                            void* v_out, hipStream_t s) {
  return read_heads(sh, M, slot, lg, 1, len, kpool, vpool, k_out, v_out, s);
}

hipError_t launch_export_rows(const Shape& sh, const SeqMeta& M, int slot, int len,
                              const void* kpool, const void* vpool, void* k_out, void* v_out,
                              hipStream_t s) {
  constexpr int kMost = 32768;
  const size_t head_bytes = static_cast<size_t>(len) * kHeadDim * (sh.dtype == 0 ? 4 : 2);
  for (int lg = 0; lg < sh.L * sh.Hkv; lg += kMost) {
    const auto at = [&](void* p) {
      return p ? static_cast<void*>(static_cast<char*>(p) + lg * head_bytes) : nullptr;
    };
    const hipError_t e = read_heads(sh, M, slot, lg, std::min(kMost, sh.L * sh.Hkv - lg), len,
                                    kpool, vpool, at(k_out), at(v_out), s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_export_positions(const Shape& sh, const SeqMeta& M, int slot, int len,
                                   const int32_t* pos, int32_t* out, hipStream_t s) {
  if (len <= 0) return hipSuccess;
  const dim3 grid((len + 255) / 256, sh.L * sh.Hkv);
  if (sh.pg.tables)
    hipLaunchKernelGGL(export_positions_kernel<true>, grid, dim3(256), 0, s, M, slot, len,
                       sh.pg, pos, out);
  else
    hipLaunchKernelGGL(export_positions_kernel<false>, grid, dim3(256), 0, s, M, slot, len,
                       sh.pg, pos, out);
  return hipGetLastError();
}

hipError_t launch_mark_pending(SeqMeta* meta, int slot_lo, int slot_hi, hipStream_t s) {
  if (slot_hi <= slot_lo) return hipSuccess;
  const int n = slot_hi - slot_lo;
  hipLaunchKernelGGL(mark_pending_kernel, dim3((n + 255) / 256), dim3(256), 0, s, meta,
                     slot_lo, slot_hi);
  return hipGetLastError();
}

hipError_t launch_clear_pending(SeqMeta* meta, int slot_lo, int slot_hi, hipStream_t s) {
  if (slot_hi <= slot_lo) return hipSuccess;
  const int n = slot_hi - slot_lo;
  hipLaunchKernelGGL(clear_pending_kernel, dim3((n + 255) / 256), dim3(256), 0, s, meta,
                     slot_lo, slot_hi);
  return hipGetLastError();
}

hipError_t launch_table_set(const Shape& sh, const TableEntry* entries, int n,
                            hipStream_t s) {
  for (int i0 = 0; i0 < n; i0 += kTableBatch) {
    TableBatch b{};
    const int k = std::min(kTableBatch, n - i0);
    for (int i = 0; i < k; ++i) b.e[i] = entries[i0 + i];
    hipLaunchKernelGGL(table_set_kernel, dim3(1), dim3(kTableBatch), 0, s,
                       const_cast<int32_t*>(sh.pg.tables), sh.pg.pages_per_seq, b, k);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace ra
