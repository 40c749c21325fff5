// The order in which an attention launch over blocks takes the slots (test
// infrastructure): api.cpp and api_blocks.cpp with the stand-ins of
// stub_launchers.cpp and, here, of the launches that api_blocks.cpp makes.  The
// dense launch is wrapped by the linker (--wrap), so that its order is seen too.
//
// Checked at every launch: an order holds each active slot once and no other, the
// longest first.  Steps mix dense and sparse layers while slots come and go.
//
// Usage: slot_order SEED DTYPE LAYOUT SLOTS OPS
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include <hip/hip_runtime.h>

#include "ra_internal.h"
#include "randattn.h"

extern "C" void stub_configure(int64_t pool_rows, int64_t n_groups, int max_seqs, int page_rows);

namespace {

constexpr int L = 3, Hkv = 1, kPromptMax = 400;
ra_cache* g_cache = nullptr;
int g_slots = 0, g_ordered = 0, g_after_dense = 0;
bool g_dense_first = false;

[[noreturn]] void fail(const char* what, long long a, long long b) {
  std::fprintf(stderr, "check failed: %s (%lld, %lld)\n", what, a, b);
  std::abort();
}

ra_seq_info info_of(int s) {
  ra_seq_info i;
  if (ra_get_seq_info(g_cache, s, &i) != RA_OK) fail("info", s, 0);
  return i;
}

void check_order(const ra::Shape& sh, const ra::AttnLaunch& a) {
  if (!sh.order) return;
  ++g_ordered;
  g_after_dense += g_dense_first;
  const ra::SlotOrder& o = *sh.order;
  if (o.n < 2 || o.n > ra::kOrderMax) fail("order of", o.n, a.layer);
  std::vector<int> seen(g_slots, 0);
  for (int i = 0; i < o.n; ++i) {
    const int s = o.slot[i];
    if (s >= g_slots || !info_of(s).active) fail("ordered slot is not active", s, a.layer);
    if (seen[s]++) fail("slot ordered twice", s, a.layer);
    if (i && info_of(o.slot[i - 1]).len < info_of(s).len) fail("a longer slot follows", s, a.layer);
  }
  for (int s = 0; s < g_slots; ++s)
    if (info_of(s).active && !seen[s]) fail("active slot left out", s, a.layer);
}

}  // namespace

extern "C" hipError_t hipGetLastError() { return hipSuccess; }

extern "C" hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* out) {
  *out = hipStreamCaptureStatusNone;
  return hipSuccess;
}

// ra::launch_attention, as the linker's --wrap names it
extern "C" hipError_t
__real__ZN2ra16launch_attentionERKNS_5ShapeERKNS_10AttnLaunchEP12ihipStream_t(
    const ra::Shape& sh, const ra::AttnLaunch& a, hipStream_t s);
extern "C" hipError_t
__wrap__ZN2ra16launch_attentionERKNS_5ShapeERKNS_10AttnLaunchEP12ihipStream_t(
    const ra::Shape& sh, const ra::AttnLaunch& a, hipStream_t s) {
  if (sh.dtype != 2 && sh.order) fail("an order for rows that are not in 8 bits", sh.dtype, a.layer);
  check_order(sh, a);
  return __real__ZN2ra16launch_attentionERKNS_5ShapeERKNS_10AttnLaunchEP12ihipStream_t(sh, a, s);
}

namespace ra {

hipError_t launch_export_rows(const Shape&, const SeqMeta&, int, int, const void*, const void*,
                              void*, void*, hipStream_t) {
  return hipSuccess;
}

hipError_t launch_block_bounds(const Shape&, const SeqMeta*, const void*, int8_t*, int64_t,
                               const int*, int, const BoundsRange*, int, hipStream_t) {
  return hipSuccess;
}

hipError_t launch_choose_blocks(const Shape&, const SeqMeta*, const void*, int, int,
                                const BlockChoice&, uint32_t*, int, int*, int, hipStream_t) {
  return hipSuccess;
}

hipError_t launch_block_attention(const Shape& sh, const AttnLaunch& a, const BlockChoice&,
                                  hipStream_t) {
  check_order(sh, a);
  return hipSuccess;
}

}  // namespace ra

int main(int argc, char** argv) {
  if (argc != 6) return 2;
  std::mt19937 rng(std::atoi(argv[1]));
  const auto pick = [&](int n) { return static_cast<int>(rng() % static_cast<unsigned>(n)); };
  g_slots = std::atoi(argv[4]);
  ra_config c{};
  c.num_layers = L;
  c.num_q_heads = 2 * Hkv;
  c.num_kv_heads = Hkv;
  c.head_dim = 128;
  c.budget_k = 40 + pick(100);
  c.recent_r = pick(20);
  c.evict_every = 1 + pick(30);
  c.dtype = std::atoi(argv[2]);
  c.layout = std::atoi(argv[3]);
  c.max_seqs = g_slots;
  c.policy_block = 1;
  c.page_rows = 32;
  c.max_prompt_len = kPromptMax;
  const int64_t group = static_cast<int64_t>(L) * Hkv * c.page_rows;
  const int64_t rows = (ra_seq_rows(&c, kPromptMax) * g_slots + group - 1) / group * group;
  stub_configure(rows, rows / group, g_slots, c.page_rows);
  const auto aligned = [](std::vector<char>& v) {
    return v.data() + (16 - reinterpret_cast<uintptr_t>(v.data()) % 16) % 16;
  };
  std::vector<char> pool(32), pos(rows * 4 + 16), meta(ra_meta_bytes(&c) + 16),
      bounds(ra_sparse_bytes(&c, rows) + 16);
  constexpr int kBlocks = 4;
  std::vector<char> ws(ra_sparse_workspace_bytes(&c, kBlocks) + 16);
  if (ra_cache_create(&c, aligned(pool), aligned(pool), reinterpret_cast<int32_t*>(aligned(pos)),
                      rows, aligned(meta), ra_meta_bytes(&c), nullptr, &g_cache) != RA_OK)
    fail("create", 0, 0);
  if (ra_sparse_attach(g_cache, aligned(bounds), bounds.size() - 16, nullptr) != RA_OK)
    fail("attach", 0, 0);
  const size_t row = 128 * 4;
  std::vector<char> q(g_slots * 2 * Hkv * row), kv(g_slots * Hkv * row),
      many(static_cast<size_t>(L) * Hkv * (kPromptMax + 400) * row);
  int steps = 0;
  for (int op = 0, ops = std::atoi(argv[5]); op < ops; ++op) {
    const int s = pick(g_slots);
    switch (pick(6)) {
      case 0:
      case 1:
        ra_seq_begin(g_cache, s, pick(kPromptMax + 1), 1, op, many.data(), many.data(), nullptr);
        break;
      case 2:
        if (pick(2)) ra_seq_end(g_cache, s, nullptr);
        break;
      case 3:
        ra_seq_fast_forward(g_cache, s, pick(30), nullptr);
        break;
      default: {
        for (int l = 0; l < L; ++l) {
          const bool sparse = pick(2);
          g_dense_first = l == 0 ? !sparse : g_dense_first;
          const ra_status st =
              sparse ? ra_sparse_attention(g_cache, l, kBlocks, pick(60), q.data(), kv.data(),
                                           kv.data(), q.data(), aligned(ws), ws.size() - 16, nullptr)
                     : ra_decode_attention(g_cache, l, q.data(), kv.data(), kv.data(), q.data(),
                                           aligned(ws), ws.size() - 16, nullptr);
          if (st != RA_OK) fail("step", st, l);
        }
        if (ra_end_step(g_cache, nullptr, nullptr) != RA_OK) fail("end", 0, 0);
        ++steps;
      }
    }
  }
  ra_cache_destroy(g_cache);
  std::printf("{\"steps\":%d,\"ordered\":%d,\"after_dense\":%d}\n", steps, g_ordered, g_after_dense);
  return 0;
}
