// Exercises the C entry points of the rotary positions and of the attention of
// requests that share prefixes (csrc/rope_host.cpp, csrc/kv8_shared_host.cpp) with
// random sizes, extreme ones among them, under AddressSanitizer and
// UndefinedBehaviorSanitizer.  The launchers below stand in for the kernels: they
// check that what validation lets through fits the launches.  Exits non-zero on the
// first failed check.  Test infrastructure only.
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "jfkv.h"
#include "jfkv_internal.h"

static long g_launches[4], g_checks = 0;
#define CHECK(c)                                                                          \
  do {                                                                                    \
    ++g_checks;                                                                           \
    if (!(c)) {                                                                           \
      std::fprintf(stderr, "%s:%d: check failed: %s\n", __FILE__, __LINE__, #c);          \
      std::exit(1);                                                                       \
    }                                                                                     \
  } while (0)

static bool one_launch(int64_t blocks, int64_t threads) { return blocks * threads < (int64_t)1 << 32; }
static void angles(const jf_rope& r, int32_t D, int32_t total) {
  CHECK(r.table && r.rot_dim >= 2 && r.rot_dim % 2 == 0 && r.rot_dim <= D);
  CHECK(r.table_rows > 0 && (r.rows || r.table_rows >= total));
}

namespace jfkv {
hipError_t launch_rope_table(const int32_t*, int32_t n, const float*, int32_t rot, float m, float*, hipStream_t) {
  ++g_launches[0];
  CHECK(n > 0 && rot >= 2 && std::isfinite(m) && one_launch(((int64_t)n * (rot / 2) + 255) / 256, 256));
  return hipSuccess;
}
hipError_t launch_rope_rotate(const jf_rope& r, bool, bool, int32_t D, const RopeRows& q, const RopeRows& k,
                              int32_t total, hipStream_t) {
  ++g_launches[1];
  angles(r, D, total);
  CHECK(total > 0 && q.heads + k.heads > 0 && D % 2 == 0);
  // a wave for a token, or as many as reach 4,096 tokens
  CHECK(one_launch(((int64_t)(total > 4096 ? total : 4096) + 3) / 4, 256));
  // items of a token, counted in 32 bits
  CHECK(((int64_t)q.heads + k.heads) * D / 2 + 64 <= INT32_MAX);
  for (const RopeRows* x : {&q, &k})
    if (x->heads) {
      CHECK(x->from && x->to);
      CHECK(total == 1 || (x->from_stride >= (int64_t)x->heads * D && x->to_stride >= (int64_t)x->heads * D));
      CHECK(x->from_stride <= INT64_MAX / 2 / total && x->to_stride <= INT64_MAX / 2 / total);
    }
  return hipSuccess;
}
hipError_t launch_kv8_rope_append(const jf_kv_layout& L, const jf_kv_pool_ptrs&, bool, const jf_rope& r,
                                  const void*, int64_t ks, const void*, int64_t vs, const void* q, int64_t qs,
                                  void* q_out, int32_t Hq, const int32_t*, const int32_t*, const int32_t*,
                                  int32_t B, int32_t max_pages, int32_t total, hipStream_t) {
  ++g_launches[2];
  angles(r, L.head_dim, total);
  CHECK(r.rot_dim % 16 == 0 && total > 0 && (int64_t)max_pages * L.page_size <= INT32_MAX);
  CHECK(one_launch(total / L.group_size + 2 * (int64_t)B, 256) && L.num_kv_heads <= 65535);
  CHECK(ks >= 0 && vs >= 0 && ks % 8 == 0 && vs % 8 == 0 && !q == !q_out && (q ? Hq > 0 : Hq == 0));
  if (q) CHECK(qs % 8 == 0 && (int64_t)Hq * L.head_dim <= 1 << 24 && Hq % L.num_kv_heads == 0);
  return hipSuccess;
}
size_t kv8_shared_bytes(const jf_kv_layout& L, int32_t B, int32_t G, int32_t sq, int32_t Hq) {
  const int64_t pairs = (int64_t)Hq / L.num_kv_heads * sq;
  // columns, units of groups and of requests, and their record slots, in 32 bits
  CHECK((int64_t)B * pairs <= INT32_MAX && ((int64_t)B * pairs / 128 + G + 1) * L.num_kv_heads <= INT32_MAX / 64);
  CHECK((int64_t)B * ((pairs + 15) / 16) * L.num_kv_heads <= INT32_MAX / 64);
  return (size_t)B * Hq * sq * (L.head_dim + 4) * sizeof(float);
}
hipError_t launch_kv8_shared(const jf_kv_layout& L, const jf_kv_pool_ptrs&, bool, const void*, int32_t B,
                             int32_t sq, int32_t Hq, const int32_t*, int32_t max_pages, const int32_t*,
                             const int32_t*, const int32_t*, int32_t G, float scale, void*, void*, float*,
                             hipStream_t) {
  ++g_launches[3];
  CHECK(B >= 1 && B <= 65535 && G >= 1 && G <= B && sq >= 1 && sq <= 4 && Hq % L.num_kv_heads == 0);
  CHECK((int64_t)B * Hq * sq <= 65536 && L.num_kv_heads <= 65535);
  CHECK((int64_t)max_pages * L.page_size <= INT32_MAX && std::isfinite(scale * 1.4426951f));
  return hipSuccess;
}
}  // namespace jfkv

static std::mt19937 g_rng(1);
static int32_t pick(std::initializer_list<int32_t> v) { return v.begin()[g_rng() % v.size()]; }
static int32_t any_size() {  // mostly small, sometimes at the ends
  switch (g_rng() % 8) {
    case 0: return pick({INT32_MIN, -1, 0, INT32_MAX, INT32_MAX - 1, 65536});
    case 1: return 1 << (g_rng() % 31);
    case 2: return (int32_t)(g_rng() >> (1 + g_rng() % 30));
    default: return 1 + (int32_t)(g_rng() % 300);
  }
}
static int64_t any_stride(int64_t row) {
  switch (g_rng() % 8) {
    case 0: return INT64_MAX;
    case 1: return -row;
    case 2: return (int64_t)any_size();
    case 3: return INT64_MIN;
    default: return row + 8 * (g_rng() % 3);
  }
}
static float any_float() {
  const float v[] = {1.0f, 0.1f, -0.1f, INFINITY, NAN, 3e38f, 1.0f, 1e-40f};
  return v[g_rng() % 8];
}
static double any_double() {
  const double v[] = {1e4, 5e5, 8.0, 1.0, 0.0, -2.0, INFINITY, NAN, 1e300, 1e-300, 32.0, 1.5};
  return v[g_rng() % 12];
}

int main() {
  alignas(16) static uint8_t mem[64];
  void* const at = mem;
  int32_t* const i32 = reinterpret_cast<int32_t*>(mem);
  float* const f32 = reinterpret_cast<float*>(mem);
  const jf_kv_pool_ptrs pool = {mem, mem, mem, mem};
  long formed = 0;
  for (int turn = 0; turn < 300000; ++turn) {
    jf_kv_layout L = {};
    L.page_size = g_rng() % 8 ? 64 << (g_rng() % 7) : any_size();
    L.num_kv_heads = g_rng() % 4 ? pick({1, 2, 8, 16}) : any_size();
    L.head_dim = pick({64, 128, 256, 64, 128, 256, 96});
    L.group_size = pick({16, 32, 64, 128, 16, 32, 64, 8});
    L.num_pages = any_size();
    const int32_t hq = g_rng() % 4 && L.num_kv_heads < 65536 && L.num_kv_heads > 0
                           ? L.num_kv_heads * pick({1, 4, 6, 8}) : any_size();
    const int32_t B = any_size(), pages = any_size(), n = any_size(), sq = pick({1, 1, 2, 3, 4, 5, 0});
    const int32_t G = g_rng() % 2 ? 1 : any_size(), dtype = pick({0, 1, 0, 1, 2});
    const size_t bytes = g_rng() % 4 ? SIZE_MAX / 2 : g_rng();
    size_t need = 0;
    jf_kv8_shared_workspace_bytes(&L, B, G, sq, hq, &need);
    jf_kv8_shared_attn(&L, &pool, dtype, at, B, sq, hq, i32, pages, i32, i32, i32, G, any_float(), at, bytes,
                       at, g_rng() % 2 ? f32 : nullptr, nullptr);

    jf_rope r = {};
    r.table = g_rng() % 16 ? f32 : nullptr;
    r.rows = g_rng() % 2 ? i32 : nullptr;
    r.table_rows = g_rng() % 2 ? INT32_MAX : any_size();
    r.rot_dim = g_rng() % 4 ? pick({16, 32, 64, 128}) : any_size();
    r.order = pick({0, 1, 0, 1, 2});
    const int64_t kv_row = (int64_t)L.num_kv_heads * L.head_dim, q_row = (int64_t)hq * L.head_dim;
    const bool with_q = g_rng() % 2;
    jf_kv8_rope_append(&L, &pool, dtype, &r, at, any_stride(kv_row), at, any_stride(kv_row), with_q ? at : nullptr,
                       any_stride(q_row), with_q ? at : nullptr, hq, i32, i32, i32, B, pages, n, nullptr);
    const int32_t D = g_rng() % 2 ? pick({64, 128, 256, 10}) : any_size();
    const int32_t h1 = g_rng() % 2 ? pick({0, 1, 8}) : any_size(), h2 = g_rng() % 2 ? pick({0, 1, 8}) : any_size();
    jf_rope_rotate(&r, dtype, D, g_rng() % 2, at, any_stride((int64_t)h1 * D), mem + 2 * (g_rng() % 2),
                   any_stride((int64_t)h1 * D), h1, at, any_stride((int64_t)h2 * D), mem + 2 * (g_rng() % 2),
                   any_stride((int64_t)h2 * D), h2, n, nullptr);
    jf_rope_table(i32, n, f32, r.rot_dim, any_float(), f32, nullptr);

    const int32_t rot = g_rng() % 4 ? pick({2, 4, 64, 128, 65536}) : any_size();
    std::vector<float> freq(rot > 0 && rot <= 65536 ? rot / 2 : 0);  // (as long as it has to be, and no longer)
    float magnitude = 0.0f;
    formed += !jf_rope_frequencies(rot, any_double(), pick({0, 1, 2, 3, 4, -1}), any_double(), any_size(),
                                   any_double(), any_double(), freq.data() ? freq.data() : f32, &magnitude);
  }
  for (long n : g_launches) CHECK(n > 1000);
  CHECK(formed > 1000);
  std::printf("%ld checks passed, %ld, %ld, %ld, %ld launches, %ld sets of frequencies\n", g_checks, g_launches[0],
              g_launches[1], g_launches[2], g_launches[3], formed);
  return 0;
}
