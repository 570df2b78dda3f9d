// The 4-bit cache's and the pages' calls on the CPU, built with AddressSanitizer and
// UndefinedBehaviorSanitizer by tests/test_host_streams.py: what they refuse, and what
// they launch: every pair of pages in every layer once, every sequence once, fewer than 2^32
// threads each.  HIP's calls are fake_hip.h's; no launch touches the memory that it is given.
#include <climits>
#include <cstdint>
#include <cstdio>
#include <set>
#include <utility>
#include <vector>

#include "fake_hip.h"
#include "hh.h"
#include "hh_kv.h"

static int failures = 0;
#define CHECK(cond)                                                                 \
  do {                                                                              \
    if (!(cond)) {                                                                  \
      if (failures < 20) std::fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #cond); \
      ++failures;                                                                   \
    }                                                                               \
  } while (0)

struct PairArgs { int n; int src[480], dst[480]; };

static std::set<std::pair<int, int>> copied;  // (pair's destination, layer)
static std::vector<int> seqs;                 // launches of each sequence
static std::vector<int> source_of;            // by destination
static unsigned char* pool_at = nullptr;
static int64_t stride = 0;
static int joins = 0;

static void run_kernel(const std::string& k, dim3 grid, dim3 block, void** a) {
  CHECK(grid.x > 0 && grid.y > 0 && grid.z == 1 && (uint64_t)grid.x * block.x < (1ull << 32) && grid.y < 65536);
  auto is = [&](const char* name) { return k.find(name) != std::string::npos; };
  if (is("k_copy_pages")) {
    const auto p = arg<hh::PagePool>(a, 0);
    const int pieces = arg<int>(a, 1);
    const PairArgs& v = *static_cast<PairArgs*>(a[2]);
    CHECK(v.n >= 1 && v.n <= 480 && pieces == (p.bytes + 2047) / 2048);
    CHECK((uint64_t)grid.x * 4 >= (uint64_t)v.n * pieces * p.n_layers);  // a wave a piece
    const int l0 = stride ? (int)((p.pool - pool_at) / stride) : 0;
    for (int l = 0; l < p.n_layers; ++l)
      for (int i = 0; i < v.n; ++i) {
        CHECK(copied.insert({v.dst[i], l0 + l}).second);
        CHECK(source_of[v.dst[i]] == v.src[i]);
      }
  } else if (is("k_kv4_join")) {
    ++joins;
  } else if (is("k_kv4_")) {
    const auto r = arg<hh::Kv4Rows>(a, 1);
    CHECK(r.seq0 >= 0 && r.n_seqs >= 1);
    for (int s = r.seq0; s < r.seq0 + r.n_seqs; ++s) {
      CHECK(s < (int)seqs.size());
      if (s < (int)seqs.size()) ++seqs[s];
    }
  }
}

static void check_copies() {
  unsigned char* const at = pool_at = reinterpret_cast<unsigned char*>((uintptr_t)1 << 40);
  const int32_t bad[] = {-1, 64, INT_MAX, INT_MIN};
  const int32_t ok = 0, end = 63;
  stride = 64 * 1152;
  source_of.assign(64, -1);
  for (int32_t x : bad) {
    CHECK(hh_kv_copy_pages(at, 2, stride, 1152, 64, 1, &x, &ok, nullptr) == HH_ERR_INVALID_ARG);
    CHECK(hh_kv_copy_pages(at, 2, stride, 1152, 64, 1, &ok, &x, nullptr) == HH_ERR_INVALID_ARG);
  }
  CHECK(copied.empty());
  source_of[63] = 0;
  CHECK(hh_kv_copy_pages(at, 2, stride, 1152, 64, 1, &ok, &end, nullptr) == HH_OK && copied.size() == 2);
  copied.clear();
  source_of[0] = 63;
  CHECK(hh_kv_copy_pages(at, 2, stride, 1152, 64, 1, &end, &ok, nullptr) == HH_OK && copied.size() == 2);
  // Pairs and layers over several launches.
  const struct { int layers, n; int64_t bytes; } cases[] = {{1, 1, 16}, {3, 480, 1152}, {3, 481, 1152}, {2, 2000, 2064},
                                                             {65536, 3, 64 << 10}, {7, 1201, 64 << 20}, {65536, 2, 64 << 20}};
  for (const auto& c : cases) {
    copied.clear();
    const int pages = 2 * c.n + 3;
    stride = c.bytes * pages + 32;
    source_of.assign(pages, -1);
    std::vector<int32_t> src(c.n), dst(c.n);
    for (int i = 0; i < c.n; ++i) {
      dst[i] = pages - 1 - i;
      src[i] = i / 2;  // some sources twice
      source_of[dst[i]] = src[i];
    }
    CHECK(hh_kv_copy_pages(at, c.layers, stride, c.bytes, pages, c.n, src.data(), dst.data(), nullptr) == HH_OK);
    CHECK(copied.size() == (size_t)c.layers * c.n);
    dst.back() = src[0];
    CHECK(hh_kv_copy_pages(at, c.layers, stride, c.bytes, pages, c.n, src.data(), dst.data(), nullptr) == HH_ERR_INVALID_ARG);
  }
}

static void check_rows() {
  void* const at = reinterpret_cast<void*>((uintptr_t)1 << 40);
  const int32_t* const ints = static_cast<const int32_t*>(at);
  const struct { int n_seqs, max_rows, hkv, heads, max_pages; } cases[] = {
      {1, 1, 1, 1, 1},       {1, 1, 8, 32, 8192},    {300, 1, 8, 32, 400},         {5, 700, 3, 9, 80},   {1100, 1 << 20, 1, 1, 2},
      {40000, 9000, 8, 32, 600}, {3, (1 << 28) - 4000, 1, 1, 64}, {7, 1 << 20, 4, 1024, 8}, {2, 5, 1024, 4096, 300}};
  for (const auto& c : cases) {
    const hh_kv4_pool pool{at, ints, 1000, c.hkv, c.max_pages, 9};
    const hh_kv4_rows rows{ints, ints, nullptr, c.n_seqs, 1000, c.max_rows};
    auto once = [&](hh_status rc) {
      bool all = true;
      for (int n : seqs) all = all && n == 1;
      CHECK(rc == HH_ERR_UNSUPPORTED || (rc == HH_OK && all));
      return rc == HH_OK;
    };
    seqs.assign(c.n_seqs, 0);
    once(hh_kv4_append(&pool, &rows, at, at, HH_F16, c.hkv * 64, c.hkv * 64, nullptr, 0, nullptr));
    seqs.assign(c.n_seqs, 0);
    once(hh_kv4_read(&pool, &rows, at, at, HH_F16, c.hkv * 64, c.hkv * 64, nullptr));
    size_t need = 0;
    const hh_status asked = hh_kv4_attention_workspace(&pool, &rows, c.heads, &need);
    CHECK(asked == HH_OK ? need <= HH_KV4_WORKSPACE_MOST : asked == HH_ERR_UNSUPPORTED);
    for (int type : {(int)HH_F32, (int)HH_F16}) {
      seqs.assign(c.n_seqs, 0);
      joins = 0;
      const hh_status rc = hh_kv4_attention(&pool, &rows, at, type, c.heads * 64, c.heads, 1.f, nullptr, 0, at, type, c.heads * 64,
                                            at, need, nullptr);
      CHECK(rc == asked);
      if (once(rc)) CHECK((need > 0) == (joins > 0));
      // A launch that fails is reported, and nothing is launched after it.
      if (rc != HH_OK) continue;
      const int before = launches;
      fail_in = 0;
      CHECK(hh_kv4_attention(&pool, &rows, at, type, c.heads * 64, c.heads, 1.f, nullptr, 0, at, type, c.heads * 64, at, need,
                             nullptr) == HH_ERR_HIP);
      CHECK(launches == before + 1);
    }
  }
  (void)hipGetLastError();
}

static void check_nulls() {
  size_t n = 0;
  void* const at = reinterpret_cast<void*>((uintptr_t)1 << 40);
  hh_kv4_pool pool{at, static_cast<int32_t*>(at), 9, 2, 4, 3};
  hh_kv4_rows rows{nullptr, static_cast<int32_t*>(at), nullptr, 3, 3, 1};
  CHECK(hh_kv4_append(nullptr, &rows, at, at, HH_F16, 128, 128, nullptr, 0, nullptr) == HH_ERR_INVALID_ARG);
  CHECK(hh_kv4_append(&pool, nullptr, at, at, HH_F16, 128, 128, nullptr, 0, nullptr) == HH_ERR_INVALID_ARG);
  CHECK(hh_kv4_read(nullptr, &rows, at, at, HH_F16, 128, 128, nullptr) == HH_ERR_INVALID_ARG);
  CHECK(hh_kv4_attention_workspace(&pool, nullptr, 4, &n) == HH_ERR_INVALID_ARG);
  CHECK(hh_kv4_attention(&pool, nullptr, at, HH_F16, 256, 4, 1.f, nullptr, 0, at, HH_F16, 256, at, 0, nullptr) == HH_ERR_INVALID_ARG);
  CHECK(hh_kv_compact_workspace(8, nullptr) == HH_ERR_INVALID_ARG);
  CHECK(hh_kv_compact_workspace(INT_MIN, &n) == HH_ERR_INVALID_ARG);
  CHECK(hh_kv_compact_workspace(INT_MAX, &n) == HH_ERR_UNSUPPORTED);
  CHECK(hh_kv_copy_pages(nullptr, 1, 0, 16, 1, 0, nullptr, nullptr, nullptr) == HH_ERR_INVALID_ARG);
  CHECK(hh_kv_copy_pages(at, INT_MAX, LLONG_MAX, 16, INT_MAX, 0, nullptr, nullptr, nullptr) == HH_ERR_INVALID_ARG);
  CHECK(hh_kv_compact(at, 1, 0, 16, 8, nullptr, 1, 1, nullptr, nullptr, at, 1 << 20, nullptr) == HH_ERR_INVALID_ARG);
  for (int32_t x : {INT_MIN, INT_MAX, -1, 0}) {
    pool.n_kv_heads = x;
    CHECK(hh_kv4_attention_workspace(&pool, &rows, 4, &n) == HH_ERR_INVALID_ARG);
    pool.n_kv_heads = 2;
    rows.max_rows = x;
    CHECK(hh_kv4_append(&pool, &rows, at, at, HH_F16, 128, 128, nullptr, 0, nullptr) == HH_ERR_INVALID_ARG);
    rows.max_rows = 1;
    CHECK(hh_kv4_append(&pool, &rows, at, at, x == 0 ? 3 : x, 128, 128, nullptr, 0, nullptr) == HH_ERR_INVALID_ARG);
  }
  CHECK(hh_kv4_append(&pool, &rows, at, at, HH_F16, LLONG_MAX, 128, nullptr, 0, nullptr) == HH_ERR_INVALID_ARG);
  CHECK(hh_kv4_append(&pool, &rows, at, at, HH_F16, LLONG_MIN, 128, nullptr, 0, nullptr) == HH_ERR_INVALID_ARG);
}

int main() {
  check_nulls();
  check_copies();
  check_rows();
  if (failures) {
    std::fprintf(stderr, "%d checks of the cache's calls failed\n", failures);
    return 1;
  }
  std::printf("cache checks passed (%d launches)\n", launches);
  return 0;
}
