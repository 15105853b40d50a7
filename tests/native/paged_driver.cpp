// Drives the host side of the sampling phase's C ABI (include/paged_attn.h) through host-only plans: argument checks, and the division of
// calls among workgroups for lengths of every kind.  Built with -fsanitize=address,undefined against paged_api.cpp and the stand-ins
// below by tests/test_sampling_sanitizers.py; exits non-zero on the first surprise.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "paged.h"

// Host-only plans never reach a launch (rope_axes_* has no plan and is called with nothing to do).
namespace pa {
int launch_rope(const RopeArgs&, void*) { return 1; }
int launch_append(const RopeArgs&, void*) { return 1; }
int launch_paged_rows(const PagedArgs&, void*) { return 1; }
int launch_paged_chunk(const PagedArgs&, void*) { return 1; }
int launch_paged_merge(const PagedArgs&, void*) { return 1; }
}  // namespace pa

#define CHECK(cond)                                                                  \
  do {                                                                               \
    if (!(cond)) {                                                                   \
      std::fprintf(stderr, "paged_driver: %s failed at line %d\n", #cond, __LINE__); \
      std::exit(1);                                                                  \
    }                                                                                \
  } while (0)

namespace {

uint64_t state = 0x9E3779B97F4A7C15ull;
uint32_t rnd(uint32_t n) {
  state = state * 6364136223846793005ull + 1442695040888963407ull;
  return (uint32_t)(state >> 33) % n;
}
int32_t any_value() {
  static const int32_t odd[] = {0, 1, -1, 2147483647, -2147483647 - 1, 1 << 30, -(1 << 30), 4096, 65535, 1 << 24};
  return rnd(2) ? odd[rnd(10)] : (int32_t)rnd(5000);
}

void exercise(bool sane) {
  static const int32_t groups[] = {1, 4, 7, 20, 512}, pages[] = {16, 64, 1024}, widths[] = {1, 40, 4096, 1 << 20};
  paged_attn_desc_t d{};
  d.num_kv_heads = 1 + (int32_t)rnd(8);
  d.num_q_heads = d.num_kv_heads * groups[rnd(5)];
  d.head_dim = rnd(2) ? 128 : 64;
  d.page_size = pages[rnd(3)];
  d.num_pages = 1 + rnd(1 << 20);
  d.max_pages_per_seq = widths[rnd(4)];
  d.max_seqs = 1 + (int32_t)rnd(300);
  d.max_tokens = 1 + rnd(rnd(2) ? 600 : 100000);
  d.softmax_scale = 0.1f;
  d.dtype = rnd(2) ? PA_BF16 : PA_F32;
  d.device = -1;
  paged_attn_plan_t* plan = nullptr;
  size_t ws = 0;
  CHECK(paged_attn_plan(&d, &plan, &ws) == PA_OK && plan && ws > 0);
  const int32_t seqs = 1 + (int32_t)rnd((uint32_t)d.max_seqs);
  const int64_t tokens = 1 + rnd((uint32_t)d.max_tokens);
  std::vector<int32_t> lens((size_t)seqs), cu((size_t)seqs + 1, 0);
  for (int32_t b = 0; b < seqs; ++b) {
    lens[(size_t)b] = sane ? (int32_t)rnd(100000) : any_value();
    cu[(size_t)b + 1] = sane ? cu[(size_t)b] + (int32_t)rnd((uint32_t)(tokens / seqs + 1)) : any_value();
  }
  if (!sane && rnd(2)) cu[0] = any_value();
  const int32_t shared = rnd(2) ? -1 : sane ? (int32_t)rnd(50000) : any_value();
  int32_t workgroups = 0, rows = 0, keys = 0;
  CHECK(paged_attn_schedule_shape(plan, seqs, tokens, shared >= 0, &workgroups, &rows, &keys) == PA_OK);
  const int64_t n = paged_attn_schedule(plan, lens.data(), cu.data(), seqs, tokens, shared, nullptr, 0);
  CHECK(n >= 0);
  std::vector<int32_t> out((size_t)n * 8);
  CHECK(paged_attn_schedule(plan, lens.data(), cu.data(), seqs, tokens, shared, out.data(), n) == n);
  const int64_t cap = (int64_t)d.max_pages_per_seq * d.page_size, group = d.num_q_heads / d.num_kv_heads;
  for (int64_t i = 0; i < n; ++i) {
    const int32_t* p = &out[(size_t)i * 8];
    CHECK(p[0] >= 0 && p[0] < workgroups && p[1] >= -1 && p[1] < seqs && p[2] >= 0 && p[2] < d.num_kv_heads);
    CHECK(p[3] >= 0 && p[4] >= 1 && p[4] <= rows && (int64_t)p[3] + p[4] <= tokens * group);
    CHECK(p[5] >= 0 && p[6] <= cap + 1);
  }
  // a call on a host-only plan is refused after its other checks
  const int32_t word = 0;
  alignas(16) static char block[16];
  CHECK(paged_attn_forward(plan, block, (int64_t)d.num_q_heads * d.head_dim, block, block, &word, &word, &word, seqs, tokens, nullptr, block, nullptr, block,
                           ws, nullptr) == PA_ERR_UNSUPPORTED);
  CHECK(paged_kv_append(plan, block, (int64_t)d.num_kv_heads * d.head_dim, block, (int64_t)d.num_kv_heads * d.head_dim, block, block, &word, &word, &word, seqs,
                        tokens, nullptr) == PA_ERR_UNSUPPORTED);
  paged_attn_destroy(plan);
}

}  // namespace

int main() {
  for (int i = 0; i < 3000; ++i) exercise(i % 2 == 0);
  paged_attn_destroy(nullptr);
  paged_attn_plan_t* plan = nullptr;
  size_t ws = 0;
  paged_attn_desc_t bad{};
  CHECK(paged_attn_plan(nullptr, &plan, &ws) == PA_ERR_NULL && paged_attn_plan(&bad, &plan, &ws) == PA_ERR_SHAPE && !plan);
  CHECK(paged_attn_schedule(nullptr, nullptr, nullptr, 1, 1, -1, nullptr, 0) == -PA_ERR_NULL);
  rope_axes_desc_t r{};
  CHECK(rope_axes_forward(&r, PA_BF16, nullptr, 0, nullptr, 0, 0, 1, 0, nullptr, nullptr, nullptr, 0, nullptr, 0, nullptr) == PA_ERR_SHAPE);
  r.head_dim = r.rotary_dim = 256;
  r.num_axes = 1;
  CHECK(rope_axes_forward(&r, PA_BF16, nullptr, 0, nullptr, 0, 0, 1, 0, nullptr, nullptr, nullptr, 0, nullptr, 0, nullptr) == PA_OK);
  std::puts("paged_driver: ok");
  return 0;
}
