// Exercises the C entry points of the 8-bit cache (csrc/kv8_host.cpp) with
// random sizes, extreme ones among them, under AddressSanitizer and
// UndefinedBehaviorSanitizer.  The launchers below stand in for the kernels:
// they check that what validation lets through fits the launches.  Exits
// non-zero on the first failed check.  Test infrastructure only.
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "jfkv.h"
#include "jfkv_internal.h"

static long g_launches = 0, g_checks = 0;
#define CHECK(c)                                                                          \
  do {                                                                                    \
    ++g_checks;                                                                           \
    if (!(c)) {                                                                           \
      std::fprintf(stderr, "%s:%d: check failed: %s\n", __FILE__, __LINE__, #c);          \
      std::exit(1);                                                                       \
    }                                                                                     \
  } while (0)

static bool one_launch(int64_t blocks, int64_t threads) { return blocks * threads < (int64_t)1 << 32; }
static bool grid_yz(int64_t y, int64_t z) { return y <= 65535 && z <= 65535; }

namespace jfkv {
hipError_t launch_kv8_append(const jf_kv_layout& L, const jf_kv_pool_ptrs&, bool, const void*,
                             const void*, const int32_t*, const int32_t*, const int32_t*, int32_t B,
                             int32_t max_pages, int32_t total, hipStream_t) {
  ++g_launches;
  CHECK(total > 0 && (int64_t)max_pages * L.page_size <= INT32_MAX);
  CHECK(one_launch(total / L.group_size + 2 * (int64_t)B, 256) && grid_yz(L.num_kv_heads, 2));
  return hipSuccess;
}
hipError_t launch_kv8_decode(const jf_kv_layout& L, const jf_kv_pool_ptrs&, bool, const void*,
                             int32_t B, int32_t sq, int32_t Hq, const int32_t*, int32_t max_pages,
                             const int32_t*, float scale, int32_t splits, void*, void*, float* weights,
                             int64_t stride, hipStream_t) {
  ++g_launches;
  const int64_t pairs = (int64_t)Hq / L.num_kv_heads * sq;
  CHECK(B >= 1 && sq >= 1 && sq <= 4 && splits >= 1 && std::isfinite(scale * 1.4426951f));
  CHECK(grid_yz(L.num_kv_heads, B) && one_launch((256 + L.num_kv_heads) * ((pairs + 15) / 16), 256));
  CHECK(one_launch(pairs, 256));
  CHECK(!weights || stride >= (int64_t)max_pages * L.page_size);
  return hipSuccess;
}
int kv8_prefill_splits(const jf_kv_layout&, int32_t T, int32_t, int32_t) { return T % 64 + 1; }
size_t kv8_prefill_bytes(const jf_kv_layout& L, int32_t T, int32_t Hq, int splits) {
  return splits <= 1 ? 0 : (size_t)splits * T * Hq * (L.head_dim + 4) * sizeof(float);
}
static void chunk(const jf_kv_layout& L, int32_t T, int32_t Hq, int32_t prefix, float scale) {
  ++g_launches;
  const int64_t cols = (int64_t)T * (Hq / L.num_kv_heads);
  CHECK(T > 0 && prefix >= 0 && std::isfinite(scale * 1.4426951f));
  CHECK(cols <= INT32_MAX && (int64_t)prefix + T + 16384 <= INT32_MAX);
  CHECK(one_launch((cols + 127) / 128 * L.num_kv_heads, 512) || cols < 128);
  CHECK(one_launch(((int64_t)prefix + T + 127) / 128 * L.num_kv_heads, 256));
  CHECK(cols * L.num_kv_heads * (L.head_dim / 4) < (int64_t)1 << 32);
}
hipError_t launch_kv8_prefill(const jf_kv_layout& L, const jf_kv_pool_ptrs&, bool, const void*,
                              int32_t T, int32_t Hq, const int32_t*, int32_t prefix, float scale, int,
                              void*, void*, float*, hipStream_t) {
  chunk(L, T, Hq, prefix, scale);
  return hipSuccess;
}
hipError_t launch_kv8_weights(const jf_kv_layout& L, const jf_kv_pool_ptrs&, bool, const void*,
                              const float*, int32_t T, int32_t Hq, const int32_t*, int32_t prefix,
                              float scale, float*, int64_t stride, hipStream_t) {
  chunk(L, T, Hq, prefix, scale);
  CHECK(stride >= (int64_t)prefix + T);
  return hipSuccess;
}
size_t kv8_evict_bytes(const jf_kv_layout& L, int32_t B, int32_t max_pages) {
  return (size_t)B * L.num_kv_heads * max_pages * 64;
}
hipError_t launch_kv8_evict(const jf_kv_layout& L, const jf_kv_pool_ptrs&, int32_t B, const int32_t*,
                            int32_t max_pages, const int32_t*, const float*, int64_t stride,
                            int32_t keep, int32_t recent, const int32_t*, int32_t dst_pages, void*,
                            int32_t*, float*, hipStream_t) {
  ++g_launches;
  const int64_t cap = (int64_t)max_pages * L.page_size, most = keep < cap ? keep : cap;
  CHECK(cap <= INT32_MAX && stride >= cap && recent >= 0 && recent <= keep);
  CHECK(keep <= (int64_t)dst_pages * L.page_size && grid_yz(L.num_kv_heads, B));
  CHECK(one_launch(2 * ((most + L.group_size - 1) / L.group_size), 256));
  CHECK(one_launch((int64_t)B * L.num_kv_heads, 256));
  // (strides of the loops that count to keep: at most a thread for 16 positions)
  CHECK((int64_t)keep + (cap + 16383) / 16 <= INT32_MAX);
  return hipSuccess;
}
}  // namespace jfkv

static std::mt19937 g_rng(1);
static int32_t pick(std::initializer_list<int32_t> v) { return v.begin()[g_rng() % v.size()]; }
static int32_t any_size() {  // mostly small, sometimes at the ends
  switch (g_rng() % 8) {
    case 0: return pick({INT32_MIN, -1, 0, INT32_MAX, INT32_MAX - 1, INT32_MAX - 16384});
    case 1: return 1 << (g_rng() % 31);
    case 2: return (int32_t)(g_rng() >> (1 + g_rng() % 30));
    default: return 1 + (int32_t)(g_rng() % 300);
  }
}
static float any_scale() {
  const float v[] = {1.0f, 0.0f, -0.1f, INFINITY, NAN, 3e38f, -1e38f, 1e-40f};
  return v[g_rng() % 8];
}

int main() {
  alignas(16) static uint8_t mem[64];
  void* const at = mem;
  int32_t* const i32 = reinterpret_cast<int32_t*>(mem);
  float* const f32 = reinterpret_cast<float*>(mem);
  const jf_kv_pool_ptrs pool = {mem, mem, mem, mem};
  for (int turn = 0; turn < 400000; ++turn) {
    jf_kv_layout L = {};
    L.page_size = g_rng() % 8 ? 64 << (g_rng() % 7) : any_size();
    L.num_kv_heads = g_rng() % 4 ? pick({1, 2, 8, 16}) : any_size();
    L.head_dim = pick({64, 128, 256, 64, 128, 256, 96});
    L.group_size = pick({16, 32, 64, 128, 16, 32, 64, 8});
    L.num_pages = any_size();
    const int32_t hq = g_rng() % 4 && L.num_kv_heads < 65536 && L.num_kv_heads > 0
                           ? L.num_kv_heads * pick({1, 4, 6, 8}) : any_size();
    const int32_t B = any_size(), pages = any_size(), n = any_size(), m = any_size(), k = any_size();
    const int32_t dtype = pick({0, 1, 0, 1, 2});
    const size_t bytes = g_rng() % 4 ? SIZE_MAX / 2 : g_rng();
    const int64_t stride = g_rng() % 4 ? INT64_MAX / 2 : any_size();
    size_t a = 0, b = 0;
    jf_kv8_pool_bytes(&L, &a, &b);
    jf_kv8_append(&L, &pool, dtype, at, at, i32, i32, i32, B, pages, n, nullptr);
    jf_kv8_decode_attn(&L, &pool, dtype, at, B, pick({1, 1, 2, 3, 4, 5, 0}), hq, i32, pages, i32,
                       any_scale(), any_size(), at, bytes, at, g_rng() % 2 ? f32 : nullptr, stride,
                       nullptr);
    jf_kv8_prefill_workspace_bytes(&L, n, hq, m, &a);
    jf_kv8_prefill_attn(&L, &pool, dtype, at, n, hq, i32, pages, m, any_scale(),
                        g_rng() % 2 ? at : nullptr, bytes, at, f32, nullptr);
    jf_kv8_attn_weights(&L, &pool, dtype, at, f32, n, hq, i32, pages, m, any_scale(), f32, stride,
                        nullptr);
    jf_kv8_evict(&L, &pool, B, i32, pages, i32, f32, stride, n, g_rng() % 2 ? 0 : m, i32, k, at, bytes,
                 i32, f32, nullptr);
  }
  CHECK(g_launches > 100000);
  std::printf("%ld checks passed, %ld launches\n", g_checks, g_launches);
  return 0;
}
