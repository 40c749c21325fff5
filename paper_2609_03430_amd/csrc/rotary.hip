// Rotary positions: the pairs of a row's leading channels turned by the row's position.
//   a' = m (a cos - b sin),  b' = m (b cos + a sin),  angle = position * quarters[pair], in quarter turns
// The angle of a far position has more whole turns than fp32 has digits to spare: the
// product and its remainder are taken in 64 bits, the sine and cosine of the rest in 32.
#include "attn_parts.h"

namespace ra {
namespace {

struct SinCos {
  float s, c;
};

// Of an angle in quarter turns: the nearest whole quarter, whose sine and cosine swap and
// negate those of what is left, an eighth of a turn at most to either side.  There the series
// of sine and cosine end with the ninth and the tenth power (what is cut off is below 2^-28).
__device__ __forceinline__ SinCos turned(double quarters, float magnitude) {
  const double whole = rint(quarters);
  const float x = static_cast<float>(quarters - whole) * 1.57079632679489662f, y = x * x;
  const float s =
      x + x * y * (-1.f / 6 + y * (1.f / 120 + y * (-1.f / 5040 + y * (1.f / 362880))));
  const float c =
      1.f + y * (-0.5f + y * (1.f / 24 + y * (-1.f / 720 + y * (1.f / 40320 - y * (1.f / 3628800)))));
  const int q = static_cast<int>(whole);
  const float a = q & 1 ? c : s, b = q & 1 ? s : c;
  return {magnitude * (q & 2 ? -a : a), magnitude * ((q + 1) & 2 ? -b : b)};
}

__device__ __forceinline__ float to_f32(uint16_t x) {
  return __uint_as_float(static_cast<uint32_t>(x) << 16);
}
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ void put(uint16_t& to, float x) { to = f32_to_bf16(x); }
__device__ __forceinline__ void put(float& to, float x) { to = x; }

// A thread's part of a row: with PACKED the pairs of two 16-byte units (eight of bf16, four
// of fp32: half is a multiple of that), otherwise one pair; past them as many of the channels
// that stay.
template <typename E, bool ADJACENT, bool PACKED>
struct Part {
  static constexpr int kPairs = PACKED ? 16 / static_cast<int>(sizeof(E)) : 1;
  static constexpr int kLanes = kHeadDim / 2 / kPairs;
  int ca, cb;          // first channels of the two sides
  int pair;            // first pair
  bool turns;
  __device__ __forceinline__ Part(int lane, int half) {
    pair = lane * kPairs;
    turns = pair < half;
    if (ADJACENT || !turns) {
      // (the channels that stay lie as adjacent pairs do, past 2 * half)
      ca = 2 * pair;
      cb = ca + kPairs;
    } else {
      ca = pair;
      cb = half + pair;
    }
  }
  struct Regs {
    E a[kPairs], b[kPairs];
  };
  __device__ __forceinline__ void load(Regs& x, const E* row) const {
    if constexpr (PACKED) {
      const u32x4 a = ld16(row + ca), b = ld16(row + cb);
      __builtin_memcpy(x.a, &a, 16);
      __builtin_memcpy(x.b, &b, 16);
    } else {
      x.a[0] = row[ca];
      x.b[0] = row[cb];
    }
  }
  __device__ __forceinline__ void store(const Regs& x, E* row) const {
    if constexpr (PACKED) {
      u32x4 a, b;
      __builtin_memcpy(&a, x.a, 16);
      __builtin_memcpy(&b, x.b, 16);
      *reinterpret_cast<u32x4*>(row + ca) = a;
      *reinterpret_cast<u32x4*>(row + cb) = b;
    } else {
      row[ca] = x.a[0];
      row[cb] = x.b[0];
    }
  }
  __device__ __forceinline__ void angles(SinCos (&sc)[kPairs], const RotaryLaunch& r,
                                         int position) const {
    if (!turns) return;
#pragma unroll
    for (int i = 0; i < kPairs; ++i)
      sc[i] = turned(static_cast<double>(position) * r.quarters[pair + i], r.magnitude);
  }
  __device__ __forceinline__ void rotate(Regs& x, const SinCos (&sc)[kPairs]) const {
    if (!turns) return;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      E& ea = ADJACENT && PACKED ? (2 * i < kPairs ? x.a[(2 * i) % kPairs] : x.b[(2 * i) % kPairs])
                                 : x.a[i];
      E& eb = ADJACENT && PACKED
                  ? (2 * i < kPairs ? x.a[(2 * i + 1) % kPairs] : x.b[(2 * i + 1) % kPairs])
                  : x.b[i];
      const float a = to_f32(ea), b = to_f32(eb);
      put(ea, a * sc[i].c - b * sc[i].s);
      put(eb, b * sc[i].c + a * sc[i].s);
    }
  }
};

constexpr int kThreads = 256;

// Workgroups of a launch, which go over more in turn: a grid holds 2^32 threads.
unsigned workgroups(int64_t n) { return static_cast<unsigned>(n < (1 << 20) ? n : 1 << 20); }

// A step's queries and keys, [max_seqs][Hq][128] and [max_seqs][Hkv][128], at the next
// position of each active slot, which the slot records hold.
template <typename E, bool ADJACENT, bool PACKED>
__global__ __launch_bounds__(kThreads) void rotate_step_kernel(const SeqMeta* meta, int max_seqs,
                                                               int Hq, int Hkv, RotaryLaunch r,
                                                               const E* q, const E* k, E* q_out,
                                                               E* k_out) {
  using P = Part<E, ADJACENT, PACKED>;
  const int heads = Hq + Hkv;
  const P part(threadIdx.x % P::kLanes, r.half);
  const int64_t items = static_cast<int64_t>(max_seqs) * heads;
  constexpr int kPer = kThreads / P::kLanes;
  for (int64_t item = static_cast<int64_t>(blockIdx.x) * kPer + threadIdx.x / P::kLanes;
       item < items; item += static_cast<int64_t>(gridDim.x) * kPer) {
    const int slot = static_cast<int>(item / heads), h = static_cast<int>(item % heads);
    const bool is_q = h < Hq;
    const E* src = is_q ? q : k;
    if (!src) continue;
    const int64_t row = is_q ? static_cast<int64_t>(slot) * Hq + h
                             : static_cast<int64_t>(slot) * Hkv + h - Hq;
    typename P::Regs x;
    part.load(x, src + row * kHeadDim);
    const SeqMeta& M = meta[slot];
    if (!M.active) continue;
    SinCos sc[P::kPairs];
    part.angles(sc, r, M.prompt_len + M.step);
    part.rotate(x, sc);
    part.store(x, (is_q ? q_out : k_out) + row * kHeadDim);
  }
}

// Rows x [heads][rows][128] at positions first + j, or positions [heads][rows].  The heads
// share the angles of a position: a workgroup takes `per` heads of its rows in turn.
template <typename E, bool ADJACENT, bool PACKED>
__global__ __launch_bounds__(kThreads) void rotate_rows_kernel(RotaryLaunch r, const E* x, E* out,
                                                               int64_t heads, int rows, int first,
                                                               const int32_t* positions,
                                                               int per) {
  using P = Part<E, ADJACENT, PACKED>;
  constexpr int kPer = kThreads / P::kLanes;
  const P part(threadIdx.x % P::kLanes, r.half);
  SinCos sc[P::kPairs];
  for (int64_t at = static_cast<int64_t>(blockIdx.x) * kPer + threadIdx.x / P::kLanes; at < rows;
       at += static_cast<int64_t>(gridDim.x) * kPer) {
    const int j = static_cast<int>(at);
    if (!positions) part.angles(sc, r, first + j);
    for (int64_t h0 = static_cast<int64_t>(blockIdx.y) * per; h0 < heads;
         h0 += static_cast<int64_t>(gridDim.y) * per) {
      const int64_t end = h0 + per < heads ? h0 + per : heads;
      for (int64_t h = h0; h < end; ++h) {
        const int64_t row = h * rows + j;
        typename P::Regs v;
        part.load(v, x + row * kHeadDim);
        if (positions) part.angles(sc, r, positions[row]);
        part.rotate(v, sc);
        part.store(v, out + row * kHeadDim);
      }
    }
  }
}

// f(Part): the build for the rows' type, the pairs' layout and their number.
template <typename E, typename F>
void with_part(const RotaryLaunch& r, F&& f) {
  if (r.half % (16 / static_cast<int>(sizeof(E))) == 0) {
    if (r.adjacent) f(std::true_type{}, std::true_type{});
    else f(std::false_type{}, std::true_type{});
  } else {
    if (r.adjacent) f(std::true_type{}, std::false_type{});
    else f(std::false_type{}, std::false_type{});
  }
}

template <typename E>
void rotate_step(const SeqMeta* meta, int max_seqs, int Hq, int Hkv, const RotaryLaunch& r,
                 const void* q, const void* k, void* q_out, void* k_out, hipStream_t s) {
  with_part<E>(r, [&](auto adjacent, auto packed) {
    constexpr bool kAdjacent = decltype(adjacent)::value, kPacked = decltype(packed)::value;
    const int64_t threads =
        static_cast<int64_t>(max_seqs) * (Hq + Hkv) * Part<E, kAdjacent, kPacked>::kLanes;
    hipLaunchKernelGGL((rotate_step_kernel<E, kAdjacent, kPacked>),
                       dim3(workgroups((threads + kThreads - 1) / kThreads)),
                       dim3(kThreads), 0, s, meta, max_seqs, Hq, Hkv, r, static_cast<const E*>(q),
                       static_cast<const E*>(k), static_cast<E*>(q_out), static_cast<E*>(k_out));
  });
}

template <typename E>
void rotate_rows(const RotaryLaunch& r, const void* x, void* out, int64_t heads, int rows,
                 int first, const int32_t* positions, hipStream_t s) {
  with_part<E>(r, [&](auto adjacent, auto packed) {
    constexpr bool kAdjacent = decltype(adjacent)::value, kPacked = decltype(packed)::value;
    const int tile = kThreads / Part<E, kAdjacent, kPacked>::kLanes;
    const unsigned tiles = workgroups((static_cast<int64_t>(rows) + tile - 1) / tile);
    // heads to a workgroup: up to eight, which share their angles, while the workgroups are many
    // (50 fp32 heads of 2,113 rows, positions of their own: 8 heads 27 us)
    const int64_t all = heads * tiles / 4096;
    const int per = positions || all < 1 ? 1 : all < 8 ? static_cast<int>(all) : 8;
    const int64_t runs = (heads + per - 1) / per;
    hipLaunchKernelGGL((rotate_rows_kernel<E, kAdjacent, kPacked>),
                       dim3(tiles, static_cast<unsigned>(runs < 65535 ? runs : 65535)),
                       dim3(kThreads), 0, s, r, static_cast<const E*>(x), static_cast<E*>(out),
                       heads, rows, first, positions, per);
  });
}

}  // namespace

hipError_t launch_rotate_step(const SeqMeta* meta, int max_seqs, int dtype, int Hq, int Hkv,
                              const RotaryLaunch& r, const void* q, const void* k, void* q_out,
                              void* k_out, hipStream_t s) {
  if (dtype == 0) rotate_step<float>(meta, max_seqs, Hq, Hkv, r, q, k, q_out, k_out, s);
  else rotate_step<uint16_t>(meta, max_seqs, Hq, Hkv, r, q, k, q_out, k_out, s);
  return hipGetLastError();
}

hipError_t launch_rotate_rows(int dtype, const RotaryLaunch& r, const void* x, void* out,
                              int64_t heads, int rows, int first, const int32_t* positions,
                              hipStream_t s) {
  if (dtype == 0) rotate_rows<float>(r, x, out, heads, rows, first, positions, s);
  else rotate_rows<uint16_t>(r, x, out, heads, rows, first, positions, s);
  return hipGetLastError();
}

}  // namespace ra
