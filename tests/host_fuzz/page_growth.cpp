// Steps of a paged cache while host memory runs out (test infrastructure): api.cpp
// and api_blocks.cpp with the stand-ins of stub_launchers.cpp and, here, of the launches
// that api_blocks.cpp makes.
//
// Checked: a step that needs pages either goes on or is refused with RA_ERR_CAPACITY,
// with nothing launched and no page taken, at each of the allocations that it makes;
// nothing throws.  With memory again the step and the ones after it go on.
//
// Usage: page_growth DTYPE SPARSE
#include <cstdio>
#include <cstdlib>
#include <new>
#include <vector>

#include <hip/hip_runtime.h>

#include "ra_internal.h"
#include "randattn.h"

extern "C" void stub_configure(int64_t pool_rows, int64_t n_groups, int max_seqs, int page_rows);
extern "C" int stub_check_tables(const int* active, const int* caps, int n);

namespace {

int g_allow = -1;          // allocations until memory runs out; -1: plenty
int g_launches = 0;

[[noreturn]] void fail(const char* what, long long a, long long b) {
  std::fprintf(stderr, "check failed: %s (%lld, %lld)\n", what, a, b);
  std::abort();
}

}  // namespace

void* operator new(size_t n) {
  if (g_allow == 0) throw std::bad_alloc();
  if (g_allow > 0) --g_allow;
  void* p = std::malloc(n ? n : 1);
  if (!p) throw std::bad_alloc();
  return p;
}
void* operator new(size_t n, const std::nothrow_t&) noexcept { return std::malloc(n ? n : 1); }
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }

extern "C" hipError_t hipGetLastError() { return hipSuccess; }
extern "C" hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* out) {
  *out = hipStreamCaptureStatusNone;
  return hipSuccess;
}

// ra::launch_attention and ra::launch_table_set, as the linker's --wrap names them
extern "C" hipError_t
__real__ZN2ra16launch_attentionERKNS_5ShapeERKNS_10AttnLaunchEP12ihipStream_t(
    const ra::Shape& sh, const ra::AttnLaunch& a, hipStream_t s);
extern "C" hipError_t
__wrap__ZN2ra16launch_attentionERKNS_5ShapeERKNS_10AttnLaunchEP12ihipStream_t(
    const ra::Shape& sh, const ra::AttnLaunch& a, hipStream_t s) {
  ++g_launches;
  return __real__ZN2ra16launch_attentionERKNS_5ShapeERKNS_10AttnLaunchEP12ihipStream_t(sh, a, s);
}

namespace ra {

hipError_t launch_export_rows(const Shape&, const SeqMeta&, int, int, const void*, const void*,
                              void*, void*, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_block_bounds(const Shape&, const SeqMeta*, const void*, int8_t*, int64_t,
                               const int*, int, const BoundsRange*, int, hipStream_t) {
  ++g_launches;
  return hipSuccess;
}
hipError_t launch_choose_blocks(const Shape&, const SeqMeta*, const void*, int, int,
                                const BlockChoice&, uint32_t*, int, int*, int, hipStream_t) {
  ++g_launches;
  return hipSuccess;
}
hipError_t launch_block_attention(const Shape&, const AttnLaunch&, const BlockChoice&,
                                  hipStream_t) {
  ++g_launches;
  return hipSuccess;
}

}  // namespace ra

int main(int argc, char** argv) {
  if (argc != 3) return 2;
  const bool sparse = std::atoi(argv[2]);
  constexpr int kSlots = 3, L = 2, kBlocks = 2;
  ra_config c{};
  c.num_layers = L;
  c.num_q_heads = 4;
  c.num_kv_heads = 2;
  c.head_dim = 128;
  c.budget_k = 300;
  c.recent_r = 8;
  c.evict_every = 50;
  c.dtype = std::atoi(argv[1]);
  c.layout = RA_LAYOUT_PAGED;
  c.max_seqs = kSlots;
  c.policy_block = 1;
  c.page_rows = 32;
  c.max_prompt_len = 128;
  const int64_t group = static_cast<int64_t>(L) * 2 * 32;
  const int64_t rows = (ra_seq_rows(&c, 128) * kSlots + group - 1) / group * group;
  stub_configure(rows, rows / group, kSlots, 32);
  const auto aligned = [](std::vector<char>& v) {
    return v.data() + (16 - reinterpret_cast<uintptr_t>(v.data()) % 16) % 16;
  };
  std::vector<char> pool(32), pos(rows * 4 + 16), meta(ra_meta_bytes(&c) + 16),
      bounds(ra_sparse_bytes(&c, rows) + 16), ws(ra_sparse_workspace_bytes(&c, kBlocks) + 16),
      io(kSlots * 4 * 512), many(static_cast<size_t>(L) * 2 * 128 * 512);
  char* const ws_at = aligned(ws);
  ra_cache* h = nullptr;
  if (ra_cache_create(&c, aligned(pool), aligned(pool), reinterpret_cast<int32_t*>(aligned(pos)),
                      rows, aligned(meta), ra_meta_bytes(&c), nullptr, &h) != RA_OK)
    fail("create", 0, 0);
  if (ra_sparse_attach(h, aligned(bounds), bounds.size() - 16, nullptr) != RA_OK)
    fail("attach", 0, 0);
  const int prompts[kSlots] = {64, 95, 128};
  for (int s = 0; s < kSlots; ++s)
    if (ra_seq_begin(h, s, prompts[s], 1, s, many.data(), many.data(), nullptr) != RA_OK)
      fail("begin", s, 0);
  int refused = 0;
  for (int t = 0; t < 120; ++t) {
    for (int l = 0; l < L; ++l) {
      for (int allow = 0;; ++allow) {        // memory for `allow` allocations
        int64_t before = 0, after = 0;
        ra_pool_info(h, nullptr, &before);
        const int mark = g_launches;
        g_allow = allow;
        ra_status st;
        try {
          st = sparse ? ra_sparse_attention(h, l, kBlocks, 8, io.data(), io.data(), io.data(),
                                            io.data(), ws_at, ws.size() - 16, nullptr)
                      : ra_decode_attention(h, l, io.data(), io.data(), io.data(), io.data(),
                                            ws_at, ws.size() - 16, nullptr);
        } catch (const std::bad_alloc&) {
          g_allow = -1;
          fail("an exception crossed the interface", t, l);
        }
        g_allow = -1;
        if (st == RA_OK) break;
        ra_pool_info(h, nullptr, &after);
        if (st != RA_ERR_CAPACITY) fail("step", st, t);
        if (g_launches != mark) fail("launched and refused", t, l);
        if (after != before) fail("pages taken and refused", t, l);
        ++refused;
        if (allow > 16) fail("refused with memory", t, l);
      }
    }
    if (ra_end_step(h, nullptr, nullptr) != RA_OK) fail("end", t, 0);
    int active[kSlots], caps[kSlots];
    for (int s = 0; s < kSlots; ++s) {
      ra_seq_info i;
      ra_get_seq_info(h, s, &i);
      active[s] = i.active;
      caps[s] = i.cap;
    }
    if (stub_check_tables(active, caps, kSlots)) fail("tables", t, 0);
  }
  ra_cache_destroy(h);
  std::printf("%d\n", refused);
  return 0;
}
