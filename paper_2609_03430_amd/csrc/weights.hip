// Eviction by accumulated attention weight: a float per cached row, kept beside the
// positions in a buffer of the caller's.
//
// An event drops, of each head's candidates (the rows between the prompt and the r most
// recent), the m of least weight, the earliest first among equal ones (select.h, on the
// weights' bits).  One workgroup per head selects and compacts positions and weights, and
// leaves its drop list in the m rows of positions that the compaction frees; the key and
// value rows move in a second launch (launch_weighed_moves), so the selection's registers
// and the moves' do not add up.
#include "ra_internal.h"
#include "select.h"

namespace ra {
namespace {

// Weights as integers of the same order; -0 as 0, and a NaN below every number.
__device__ __forceinline__ uint32_t weight_key(uint32_t bits) {
  if ((bits & 0x7fffffffu) > 0x7f800000u) return 0u;
  if (bits == 0x80000000u) bits = 0u;
  return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

// Pool row of row j, through the sequence's table in LDS where it is paged.
template <bool PAGED>
struct HeadRows {
  int64_t region;
  const int* table;
  int64_t group_rows, head_off;
  int shift;
  __device__ __forceinline__ int64_t operator()(int j) const {
    if constexpr (PAGED)
      return static_cast<int64_t>(table[j >> shift]) * group_rows + head_off +
             (j & ((1 << shift) - 1));
    else
      return region + j;
  }
};

// KPT consecutive candidates to a thread.  Positions and weights are read again after the
// selection, into registers that the keys have left, and written past a barrier: a
// survivor moves down by the drops below it.
template <int NT, int KPT, bool PAGED>
__global__ __launch_bounds__(NT) void weight_event_kernel(const SeqMeta* __restrict__ meta,
                                                          int32_t* pos, float* weights, int L,
                                                          int Hkv, int r, int slot_lo, Paging pg,
                                                          DueList due) {
  __shared__ SelectShared sel_sh;
  __shared__ int f[kMaxEvery];
  __shared__ int tbl[PAGED ? kMaxPagesLds : 1];
  const int per_seq = L * Hkv;
  const int at = static_cast<int>(blockIdx.x) / per_seq;
  const int slot = due.n ? due.slot[at] : slot_lo + at;
  const int lg = static_cast<int>(blockIdx.x) % per_seq;
  const SeqMeta& M = meta[slot];
  if (!M.active || !M.due) return;
  const int lp = M.prompt_len, old_len = M.plan_len;
  const int C = old_len - lp - r, m = C - M.k_keep, new_len = old_len - m;
  if (m <= 0 || m > kMaxEvery || C > NT * KPT) return;
  const int t = threadIdx.x;
  HeadRows<PAGED> row{M.base + static_cast<int64_t>(lg) * M.cap, tbl, pg.group_rows,
                      static_cast<int64_t>(lg) << pg.page_shift, pg.page_shift};
  if constexpr (PAGED) {
    const int32_t* table = pg.tables + static_cast<int64_t>(slot) * pg.pages_per_seq;
    const int n_pages = (old_len + (1 << pg.page_shift) - 1) >> pg.page_shift;
    for (int i = t; i < n_pages; i += NT) tbl[i] = table[i];
    __syncthreads();
  }
  uint32_t key[KPT], tie[KPT];
  uint32_t valid = 0;
#pragma unroll
  for (int i = 0; i < KPT; ++i) {
    const int c = t * KPT + i;
    key[i] = 0;
    tie[i] = static_cast<uint32_t>(c);
    if (c < C) {
      key[i] = weight_key(__float_as_uint(weights[row(lp + c)]));
      valid |= 1u << i;
    }
  }
  const uint32_t drop = select_smallest<NT, KPT, 32>(key, tie, valid, m, sel_sh);
  int k = drop_list<NT, KPT>(drop, lp, f, sel_sh);
  int32_t p[KPT];
  float w[KPT];
#pragma unroll
  for (int i = 0; i < KPT; ++i) {
    if ((valid >> i) & 1u) {
      const int64_t from = row(lp + t * KPT + i);
      p[i] = pos[from];
      w[i] = weights[from];
    }
  }
  // every load has returned before any thread writes
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
#pragma unroll
  for (int i = 0; i < KPT; ++i) {
    if (!((valid >> i) & 1u)) continue;
    if ((drop >> i) & 1u) {
      ++k;
    } else if (k) {
      const int64_t to = row(lp + t * KPT + i - k);
      pos[to] = p[i];
      weights[to] = w[i];
    }
  }
  // the r most recent rows follow, NT at a time: their sources lie above every row
  // written so far, and those of later turns above the destinations of this one
  for (int j0 = lp + C; j0 < old_len; j0 += NT) {
    const int j = j0 + t;
    int32_t pj = 0;
    float wj = 0.f;
    if (j < old_len) {
      const int64_t from = row(j);
      pj = pos[from];
      wj = weights[from];
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (j < old_len) {
      const int64_t to = row(j - m);
      pos[to] = pj;
      weights[to] = wj;
    }
  }
  // the drop list, and a word for the moves to order themselves by, in rows that every thread
  // has read by now
  __syncthreads();
  if (t == 0) weights[row(new_len)] = 0.f;
  for (int i = t; i < m; i += NT) pos[row(new_len + i)] = f[i] + i;
}

// Rows [from, from + n) of every head: their weights set from src [L * Hkv][n] (null: 0),
// or with out, copied there.  A row to a thread: a copy's time is the latency of a load and a
// store.  Grid: (runs of 256 rows, L * Hkv).
constexpr int kCopyRows = 256;
template <bool PAGED>
__global__ __launch_bounds__(kCopyRows) void copy_weights_kernel(
    SeqMeta M, int slot, int from, int n, Paging pg, const float* src, float* weights, float* out) {
  const int j = blockIdx.x * kCopyRows + threadIdx.x;
  if (j >= n) return;
  const RowMap rm = row_map(M, slot, blockIdx.y, pg);
  const int64_t at = static_cast<int64_t>(blockIdx.y) * n + j;
  const int64_t row = pool_row<PAGED>(rm, from + j);
  if (out) out[at] = weights[row];
  else weights[row] = src ? src[at] : 0.f;
}

hipError_t copy_weights(const Shape& sh, const SeqMeta& M, int slot, int from, int n,
                        const float* src, float* weights, float* out, hipStream_t s) {
  if (n <= 0) return hipSuccess;
  const dim3 grid((n + kCopyRows - 1) / kCopyRows, sh.L * sh.Hkv);
  if (sh.pg.tables)
    hipLaunchKernelGGL((copy_weights_kernel<true>), grid, dim3(kCopyRows), 0, s, M, slot, from,
                       n, sh.pg, src, weights, out);
  else
    hipLaunchKernelGGL((copy_weights_kernel<false>), grid, dim3(kCopyRows), 0, s, M, slot, from,
                       n, sh.pg, src, weights, out);
  return hipGetLastError();
}

template <int NT, int KPT>
void launch_select(const Shape& sh, const SeqMeta* meta, int32_t* pos, float* weights, int slot_lo,
                   int slot_hi, hipStream_t s) {
  const DueList due = sh.due ? *sh.due : DueList{};
  const dim3 grid((due.n ? due.n : slot_hi - slot_lo) * sh.L * sh.Hkv);
  if (sh.pg.tables)
    hipLaunchKernelGGL((weight_event_kernel<NT, KPT, true>), grid, dim3(NT), 0, s, meta, pos,
                       weights, sh.L, sh.Hkv, sh.r, slot_lo, sh.pg, due);
  else
    hipLaunchKernelGGL((weight_event_kernel<NT, KPT, false>), grid, dim3(NT), 0, s, meta, pos,
                       weights, sh.L, sh.Hkv, sh.r, slot_lo, sh.pg, due);
}

}  // namespace

hipError_t launch_weight_event(const Shape& sh, const SeqMeta* meta, void* kpool, void* vpool,
                               int32_t* pos, float* weights, int slot_lo, int slot_hi,
                               int max_candidates, bool positions_only, hipStream_t s) {
  if (slot_hi <= slot_lo) return hipSuccess;
  // the smallest build that holds the candidates (as the random events'); the largest's keys
  // are 32 bits for its registers' sake (2 heads of 17,000 and of 30,000 candidates 60 and
  // 95 us, with keys of 64 bits, in scratch memory, 98 and 158; 64 of 30,000 110 and 168)
#define RA_SELECT(KPT)                  \
  if (max_candidates <= 1024 * KPT)     \
  launch_select<1024, KPT>(sh, meta, pos, weights, slot_lo, slot_hi, s)
  RA_SELECT(1);
  else RA_SELECT(2);
  else RA_SELECT(3);
  else RA_SELECT(5);
  else RA_SELECT(9);
  else RA_SELECT(16);
  else RA_SELECT(32);
  else return hipErrorInvalidValue;
#undef RA_SELECT
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || positions_only) return e;
  return launch_weighed_moves(sh, meta, kpool, vpool, pos, weights, slot_lo, slot_hi, max_candidates, s);
}

hipError_t launch_set_weights(const Shape& sh, const SeqMeta& M, int slot, int from, int to,
                              const float* src, float* weights, hipStream_t s) {
  return copy_weights(sh, M, slot, from, to - from, src, weights, nullptr, s);
}

hipError_t launch_export_weights(const Shape& sh, const SeqMeta& M, int slot, int len,
                                 const float* weights, float* out, hipStream_t s) {
  return copy_weights(sh, M, slot, 0, len, nullptr, const_cast<float*>(weights), out, s);
}

}  // namespace ra
