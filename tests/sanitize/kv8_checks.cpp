// The 8-bit cache's calls on the CPU, built with AddressSanitizer and UndefinedBehaviorSanitizer
// by tests/test_host_kv8.py: what they refuse, and that their launches cover every sequence,
// row, kv head and split once, with fewer than 2^32 threads each and no more LDS than the kernel
// may have; and that split outputs are joined, on the 4-bit cache too.  HIP's calls are
// fake_hip.h's, but for the limit of a kernel's LDS, which is kept here; no launch touches the
// memory that it is given.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <climits>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <string>
#include <vector>

#define hipFuncSetAttribute without_a_limit
#define hipLaunchKernel without_lds
#include "fake_hip.h"
#undef hipFuncSetAttribute
#undef hipLaunchKernel
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

struct Div { unsigned mul, shift, d; };
static unsigned over(unsigned x, Div v) { return (unsigned)(((uint64_t)x * v.mul) >> 31 >> v.shift); }

// A call's limit holds for every launch of the kernel in the process, other threads' too: it may
// not fall below what another call has asked for.
static std::map<std::string, int> limits;
extern "C" hipError_t hipFuncSetAttribute(const void* f, hipFuncAttribute what, int value) {
  CHECK(what == hipFuncAttributeMaxDynamicSharedMemorySize);
  int& limit = limits[kernels.at(f)];
  CHECK(value >= limit && value <= 160 << 10);
  limit = value;
  return hipSuccess;
}

static size_t lds = 0;  // bytes that a launch asks for
extern "C" hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t bytes, hipStream_t st) {
  lds = bytes;
  return without_lds(f, grid, block, args, bytes, st);
}

static std::vector<int> seqs;  // launches of each sequence, of the call's first kernel
static int joins = 0, scores = 0, limited = 0;
static std::map<std::string, int> seen;

static void run_kernel(const std::string& k, dim3 grid, dim3 block, void** a) {
  CHECK(grid.x > 0 && grid.y > 0 && (uint64_t)grid.x * block.x < (1ull << 32) && grid.y < 65536);
  CHECK(lds <= 64 << 10 || (int)lds <= limits[k]);
  limited += lds > 64 << 10;
  auto is = [&](const char* name) { return k.find(name) != std::string::npos; };
  const auto p = arg<hh::Kv4Pool>(a, 0);
  const auto r = arg<hh::Kv4Rows>(a, 1);
  CHECK(r.seq0 >= 0 && r.n_seqs >= 1);
  if (is("k_kv_join")) {
    ++joins;
    const auto at = arg<hh::Kv4Attend>(a, 2);
    const int64_t outs = (int64_t)r.n_seqs * r.max_rows * at.hq;
    CHECK(is("k_kv_join_rows") ? (int64_t)grid.x * 16 >= outs : grid.x == outs);
    CHECK(is("k_kv_join_rows") ? arg<int>(a, 4) <= 16 : arg<int>(a, 4) <= 64);
    return;
  }
  if (is("k_kv4_attend")) return;  // (kv_checks.cpp's)
  CHECK(grid.x % r.n_seqs == 0);
  const int64_t each = grid.x / r.n_seqs, page_tiles = (r.max_rows + 14) / 16 + 1;
  auto divides = [&](Div d, unsigned by) { return d.d == by && over(grid.x - 1, d) == (grid.x - 1) / by; };
  if (is("k_kv8_append") || is("k_kv8_read")) {
    CHECK(each == page_tiles && arg<int>(a, is("k_kv8_read") ? 7 : 8) == page_tiles);
    CHECK((int)(grid.y * (block.x / 64)) >= p.hkv && block.x % 64 == 0 && grid.z == (is("k_kv8_append") ? 2u : 1u));
  } else if (is("k_kv8_few") || is("k_kv8_attend")) {
    const auto at = arg<hh::Kv4Attend>(a, 2);
    const int group = at.hq / p.hkv, i = is("k_kv8_few") ? 4 : 3;
    const auto heads = arg<Div>(a, i), splits = arg<Div>(a, i + 1), tiles = arg<Div>(a, i + 2), of = arg<Div>(a, i + 3);
    CHECK(each == (int64_t)heads.d * splits.d * tiles.d && divides(heads, p.hkv));
    CHECK(splits.d >= 1 && splits.d <= 64 && divides(splits, splits.d) && divides(tiles, tiles.d) && of.d == (unsigned)group);
    const int64_t columns = (int64_t)r.max_rows * group;
    CHECK(over((unsigned)columns - 1, of) == (columns - 1) / group);
    if (is("k_kv8_attend")) {
      const int nq = std::atoi(k.c_str() + k.find("k_kv8_attendILi") + 15);
      CHECK((nq == 1 || nq == 2 || nq == 4) && (int64_t)tiles.d * 16 * nq >= columns && ((int64_t)tiles.d - 1) * 16 * nq < columns);
      CHECK(block.x == 256);
    } else {
      const int side = std::atoi(k.c_str() + k.find("k_kv8_fewILi") + 12), waves = block.x / 64;
      const auto list = arg<hh::Kv8List>(a, 3);
      const auto row_tiles = arg<Div>(a, 8);
      CHECK(is((std::string("k_kv8_fewILi") + std::to_string(side) + "ELi" + std::to_string(waves) + "ELb").c_str()));
      CHECK(is("ELb1ELb0E") == (list.blocks != nullptr));
      if (list.blocks) {
        CHECK((int)row_tiles.d * 16 >= group && ((int)row_tiles.d - 1) * 16 < group && (int64_t)tiles.d == (int64_t)r.max_rows * row_tiles.d);
        CHECK(over(tiles.d - 1, row_tiles) == (tiles.d - 1) / row_tiles.d && side == (group <= 8 ? 2 : 1));
      } else {
        CHECK(tiles.d == 1 && columns <= 16 && side == (columns <= 8 ? 2 : 1) && waves >= 4);
      }
    }
  } else if (is("k_kv8_score")) {
    ++scores;
    const auto tiles = arg<Div>(a, 4), chunks = arg<Div>(a, 5);
    CHECK(tiles.d == (unsigned)r.max_rows && (int64_t)chunks.d * 256 >= p.max_pages);
    CHECK(each == (int64_t)p.hkv * tiles.d * chunks.d && divides(arg<Div>(a, 3), p.hkv) && divides(tiles, tiles.d) && divides(chunks, chunks.d));
    return;  // (the search's launch counts)
  } else if (is("k_kv8_select")) {
    const int rows = arg<int>(a, 3), scores_each = std::atoi(k.c_str() + k.find("k_kv8_selectILi") + 15);
    const auto tiles = arg<Div>(a, 5);
    CHECK(each == (int64_t)p.hkv * tiles.d && (int64_t)tiles.d * rows >= r.max_rows && divides(arg<Div>(a, 4), p.hkv) && divides(tiles, tiles.d));
    // A row's scores: a run of an odd number in each thread that searches it.
    const int threads = is("ELb1E") ? block.x : 64, run = ((p.max_pages + threads - 1) / threads) | 1;
    CHECK(run <= scores_each && (size_t)rows * run * threads * 4 <= lds && rows <= 16);
  } else {
    CHECK(!"a kernel of another call");
  }
  ++seen[k];
  for (int s = r.seq0; s < r.seq0 + r.n_seqs; ++s) {
    CHECK(s < (int)seqs.size());
    if (s < (int)seqs.size()) ++seqs[s];
  }
}

static void* const at = reinterpret_cast<void*>((uintptr_t)1 << 40);
static int32_t* const ints = static_cast<int32_t*>(at);

// A call: all of its sequences once, or refused; and one whose launch fails reports it and
// launches nothing more.
template <typename F>
static bool once(int n_seqs, F call) {
  seqs.assign(n_seqs, 0);
  joins = scores = 0;
  const hh_status rc = call();
  bool all = true;
  for (int n : seqs) all = all && n == (rc == HH_OK ? 1 : 0);
  CHECK((rc == HH_OK || rc == HH_ERR_UNSUPPORTED) && all);
  if (rc != HH_OK) return false;
  const int before = launches, j = joins, s = scores;
  for (int n : {0, 1}) {
    const int start = launches;
    fail_in = n;
    const hh_status failed = call();
    CHECK(fail_in >= 0 ? failed == HH_OK && launches - start <= n : failed == HH_ERR_HIP && launches == start + n + 1);
    fail_in = -1;
  }
  (void)before;
  joins = j;
  scores = s;
  return true;
}

static void check_launches() {
  const struct { int n_seqs, max_rows, hkv, heads, max_pages; } cases[] = {
      {1, 1, 1, 1, 1},       {1, 1, 8, 32, 8192},      {1, 1, 8, 32, 32768},   {300, 1, 8, 32, 400},      {32, 1, 8, 32, 1400},
      {5, 700, 3, 9, 80},    {3, 9, 2, 80, 2048},      {2, 2000, 8, 32, 437},  {1100, 1 << 20, 1, 1, 2},  {40000, 9000, 8, 32, 600},
      {7, 1 << 20, 4, 1024, 8}, {3, (1 << 28) - 4000, 1, 1, 64}, {2, 5, 1024, 4096, 300}, {64, 1, 8, 64, 5000}, {400, 3, 8, 32, 20000},
      {9000, 4000, 8, 32, 30000}, {1, 500, 8, 32, 512}, {2, 1, 8, 32, 2049}, {1, 1, 8, 32, 10000}, {1, 64, 8, 32, 1024},
      {1, 1, 8, 128, 3000}, {100, 3, 8, 32, 400}, {128, 1, 8, 96, 60}, {30, 1, 4, 64, 500}, {100, 1, 8, 128, 30}, {2, 100, 8, 96, 200}, {1000, 2, 4, 48, 30}, {1, 40, 8, 32, 3}, {4, 30, 8, 32, 501}};
  for (const auto& c : cases) {
    const hh_kv8_pool pool{at, ints, 1000, c.hkv, c.max_pages, 9};
    const int n_rows = (int)std::min<int64_t>((int64_t)c.n_seqs * c.max_rows, 1 << 22);
    const hh_kv8_rows rows{ints, ints, nullptr, c.n_seqs, n_rows, c.max_rows};
    const int64_t kv = c.hkv * 64, q = c.heads * 64;
    once(c.n_seqs, [&] { return hh_kv8_append(&pool, &rows, at, at, HH_F16, kv, kv, nullptr, 0, nullptr); });
    once(c.n_seqs, [&] { return hh_kv8_read(&pool, &rows, at, at, HH_F16, kv, kv, nullptr); });
    for (int type : {(int)HH_F32, (int)HH_F16}) {
      size_t need = 0;
      hh_status asked = hh_kv8_attention_workspace(&pool, &rows, c.heads, &need);
      CHECK(asked == HH_OK ? need <= HH_KV8_WORKSPACE_MOST : asked == HH_ERR_UNSUPPORTED);
      bool ran = once(c.n_seqs, [&] {
        return hh_kv8_attention(&pool, &rows, at, type, q, c.heads, 1.f, nullptr, 0, at, type, q, at, need, nullptr);
      });
      CHECK(ran == (asked == HH_OK) && (!ran || (need > 0) == (joins > 0)));
      for (int n : {1, 2, 7, 32, 129, 1000, 32768}) {
        asked = hh_kv8_attention_blocks_workspace(&pool, &rows, c.heads, n, &need);
        CHECK(asked == HH_OK ? need <= HH_KV8_WORKSPACE_MOST : asked == HH_ERR_UNSUPPORTED);
        ran = once(c.n_seqs, [&] {
          return hh_kv8_attention_blocks(&pool, &rows, ints, n, at, type, q, c.heads, 1.f, nullptr, 0, at, type, q, at, need, nullptr);
        });
        CHECK(ran == (asked == HH_OK) && (!ran || (need > 0) == (joins > 0)));
      }
    }
    size_t need = 0;
    const hh_status asked = hh_kv8_select_workspace(&pool, &rows, c.heads, 32, &need);
    CHECK(asked == HH_OK ? need <= HH_KV8_WORKSPACE_MOST : asked == HH_ERR_UNSUPPORTED);
    const bool ran = once(c.n_seqs, [&] {
      return hh_kv8_select(&pool, &rows, at, HH_F16, q, c.heads, nullptr, 0, 32, 1, 2, ints, at, need, nullptr);
    });
    CHECK(ran == (asked == HH_OK) && (!ran || (need > 0) == (scores > 0)));
  }
  CHECK(limited > 0);
  // Every kernel was some call's.
  for (const auto& f : kernels)
    if (f.second.find("k_kv8_") != std::string::npos && f.second.find("k_kv8_score") == std::string::npos) {
      if (!seen.count(f.second)) std::fprintf(stderr, "never launched: %s\n", f.second.c_str());
      CHECK(seen.count(f.second));
    }
}

// Tables of falling widths, whose rows' scores need less and less LDS.
static void check_limits() {
  for (int pages : {32768, 20000, 8193, 8192, 5000, 2049, 2048, 1500, 600})
    for (int max_rows : {1, 300}) {
      const hh_kv8_pool pool{at, ints, 1000, 8, pages, 9};
      const hh_kv8_rows rows{ints, ints, nullptr, 200, 1000, max_rows};
      once(200, [&] { return hh_kv8_select(&pool, &rows, at, HH_F16, 2048, 32, nullptr, 0, 32, 1, 2, ints, at, 16 << 20, nullptr); });
    }
}

// The kernels that join split outputs are both caches'.
static void check_4_bit_joins() {
  const struct { int n_seqs, max_rows, max_pages; bool split; } cases[] = {
      {1, 1, 8192, true}, {1, 1, 300, true}, {32, 1, 8192, true}, {3, 150, 450, true}, {1, 128, 8192, true}, {1, 1, 20, false}, {64, 300, 20, false}};
  for (const auto& c : cases)
    for (int type : {(int)HH_F32, (int)HH_F16}) {
      const hh_kv4_pool pool{at, ints, 1000, 8, c.max_pages, 70};
      const hh_kv4_rows rows{ints, ints, nullptr, c.n_seqs, c.n_seqs * c.max_rows, c.max_rows};
      size_t need = 0;
      CHECK(hh_kv4_attention_workspace(&pool, &rows, 32, &need) == HH_OK && (need > 0) == c.split);
      joins = 0;
      CHECK(hh_kv4_attention(&pool, &rows, at, type, 2048, 32, 1.f, nullptr, 0, at, type, 2048, at, need, nullptr) == HH_OK);
      CHECK(joins == (c.split ? 1 : 0));
    }
}

static void check_refusals() {
  size_t n = 0;
  hh_kv8_pool pool{at, ints, 9, 2, 4, 3};
  hh_kv8_rows rows{nullptr, ints, nullptr, 3, 3, 1};
  const int before = launches;
  auto attend = [&](const hh_kv8_pool* p, const hh_kv8_rows* r, const void* q, int64_t stride, float scale, void* out) {
    return hh_kv8_attention(p, r, q, HH_F16, stride, 4, scale, nullptr, 0, out, HH_F16, 256, at, 16 << 20, nullptr);
  };
  auto listed = [&](const int32_t* blocks, int count, int64_t stride, float scale) {
    return hh_kv8_attention_blocks(&pool, &rows, blocks, count, at, HH_F16, stride, 4, scale, nullptr, 0, at, HH_F16, 256, at, 16 << 20, nullptr);
  };
  auto select = [&](int32_t* blocks, int count, int first, int last) {
    return hh_kv8_select(&pool, &rows, at, HH_F16, 256, 4, nullptr, 0, count, first, last, blocks, at, 16 << 20, nullptr);
  };
  CHECK(hh_kv8_append(nullptr, &rows, at, at, HH_F16, 128, 128, nullptr, 0, nullptr) == HH_ERR_INVALID_ARG);
  CHECK(hh_kv8_append(&pool, nullptr, at, at, HH_F16, 128, 128, nullptr, 0, nullptr) == HH_ERR_INVALID_ARG);
  CHECK(hh_kv8_read(nullptr, &rows, at, at, HH_F16, 128, 128, nullptr) == HH_ERR_INVALID_ARG);
  CHECK(hh_kv8_attention_workspace(&pool, nullptr, 4, &n) == HH_ERR_INVALID_ARG);
  CHECK(hh_kv8_select_workspace(&pool, &rows, 4, 5, nullptr) == HH_ERR_INVALID_ARG);
  CHECK(hh_kv8_attention_blocks_workspace(nullptr, &rows, 4, 5, &n) == HH_ERR_INVALID_ARG);
  CHECK(attend(nullptr, &rows, at, 256, 1.f, at) == HH_ERR_INVALID_ARG);
  CHECK(attend(&pool, &rows, nullptr, 256, 1.f, at) == HH_ERR_INVALID_ARG && attend(&pool, &rows, at, 256, 1.f, nullptr) == HH_ERR_INVALID_ARG);
  for (float s : {0.f, -1.f, 0x1.000002p100f, __builtin_inff(), __builtin_nanf("")}) {
    CHECK(attend(&pool, &rows, at, 256, s, at) == HH_ERR_INVALID_ARG);
    CHECK(listed(ints, 5, 256, s) == HH_ERR_INVALID_ARG);
  }
  for (int64_t s : {(int64_t)0, (int64_t)-256, (int64_t)LLONG_MAX, (int64_t)LLONG_MIN, (int64_t)255, (int64_t)260}) {
    CHECK(attend(&pool, &rows, at, s, 1.f, at) == HH_ERR_INVALID_ARG);
    CHECK(listed(ints, 5, s, 1.f) == HH_ERR_INVALID_ARG);
  }
  for (int c : {0, -1, INT_MIN}) CHECK(listed(ints, c, 256, 1.f) == HH_ERR_INVALID_ARG && select(ints, c, 0, 1) == HH_ERR_INVALID_ARG);
  for (int c : {32769, INT_MAX}) CHECK(listed(ints, c, 256, 1.f) == HH_ERR_UNSUPPORTED && select(ints, c, 0, 1) == HH_ERR_UNSUPPORTED);
  CHECK(listed(nullptr, 5, 256, 1.f) == HH_ERR_INVALID_ARG && select(nullptr, 5, 0, 1) == HH_ERR_INVALID_ARG);
  CHECK(select(ints, 5, -1, 1) == HH_ERR_INVALID_ARG && select(ints, 5, 0, 0) == HH_ERR_INVALID_ARG);
  CHECK(select(ints, 5, 3, 3) == HH_ERR_INVALID_ARG && select(ints, 5, INT_MAX, INT_MAX) == HH_ERR_INVALID_ARG);
  pool.max_pages = 32769;
  CHECK(select(ints, 5, 0, 1) == HH_ERR_UNSUPPORTED && hh_kv8_select_workspace(&pool, &rows, 4, 5, &n) == HH_ERR_UNSUPPORTED);
  for (int32_t x : {INT_MIN, INT_MAX, -1, 0}) {
    pool = hh_kv8_pool{at, ints, 9, 2, x, 3};
    CHECK(hh_kv8_attention_workspace(&pool, &rows, 4, &n) == HH_ERR_INVALID_ARG && select(ints, 5, 0, 1) == HH_ERR_INVALID_ARG);
    pool = hh_kv8_pool{at, ints, 9, x, 4, 3};
    CHECK(hh_kv8_attention_workspace(&pool, &rows, 4, &n) == HH_ERR_INVALID_ARG && listed(ints, 5, 256, 1.f) == HH_ERR_INVALID_ARG);
    pool = hh_kv8_pool{at, ints, 9, 2, 4, 3};
    rows.max_rows = x;
    CHECK(hh_kv8_append(&pool, &rows, at, at, HH_F16, 128, 128, nullptr, 0, nullptr) == HH_ERR_INVALID_ARG);
    rows.max_rows = 1;
  }
  CHECK(launches == before);
}

int main() {
  check_refusals();
  check_launches();
  check_limits();
  check_4_bit_joins();
  if (failures) {
    std::fprintf(stderr, "%d checks of the 8-bit cache's calls failed\n", failures);
    return 1;
  }
  std::printf("8-bit cache checks passed (%d launches)\n", launches);
  return 0;
}
