// A context's streams on the CPU, built with AddressSanitizer and
// UndefinedBehaviorSanitizer by tests/test_host_streams.py: forks, cuts, compaction, resets,
// prompts and steps in any order, with launches that fail.  HIP's calls are fake_hip.h's: a
// launch of a kernel that keeps the streams' books does on host memory what the kernel
// does, any other launch nothing.  Every position of a stream is
// stamped with its token in its KV page as the device's page table gives it, so that
// a page that is lost, shared by mistake or moved without its entry shows.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <new>
#include <random>
#include <string>
#include <vector>

#include "fake_hip.h"
#include "hh.h"

static int failures = 0;
static const char* at_op = "";
#define CHECK(cond)                                                                       \
  do {                                                                                    \
    if (!(cond)) {                                                                        \
      if (failures < 20) std::fprintf(stderr, "check failed at line %d (%s): %s\n", __LINE__, at_op, #cond); \
      ++failures;                                                                         \
    }                                                                                     \
  } while (0)

// ------------------------------------------------------------------ launches

struct IntArgs { int n; int v[62]; };
struct PairArgs { int n; int src[480], dst[480]; };
struct ForkArgs { int n, has_last; int ids[62], last[62]; };
struct PagePool { unsigned char* pool; int64_t layer_stride, bytes; int n_layers, n_pages; };

// What the launches tell: where the books are.
static struct Books {
  int *table = nullptr, *pos = nullptr, *pending = nullptr, *hist = nullptr;
  int max_pages = 0, max_ctx = 0;
  PagePool pool{};
  const int* feed = nullptr;
} dev;

static void move_page(const PagePool& p, int from, int to) {
  for (int l = 0; l < p.n_layers; ++l)
    std::memcpy(p.pool + l * p.layer_stride + to * p.bytes, p.pool + l * p.layer_stride + from * p.bytes, (size_t)p.bytes);
}

static void run_kernel(const std::string& k, dim3 grid, dim3, void** a) {
  auto is = [&](const char* name) { return k.find(name) != std::string::npos; };
  if (is("k_put_ints")) {
    const IntArgs& v = *static_cast<IntArgs*>(a[1]);
    std::memcpy(arg<int*>(a, 0), v.v, (size_t)v.n * sizeof(int));
  } else if (is("k_reset_streams")) {
    dev.pos = arg<int*>(a, 2);
    dev.pending = arg<int*>(a, 3);
    for (int s = arg<int>(a, 0); s < arg<int>(a, 0) + arg<int>(a, 1); ++s) dev.pos[s] = dev.pending[s] = 0;
  } else if (is("k_prep_embed")) {
    const int s = arg<int>(a, 0);
    dev.feed = arg<const int*>(a, 1);
    int *rs = arg<int*>(a, 2), *rp = arg<int*>(a, 3), *pos = arg<int*>(a, 4);
    for (int r = 0; s != -2 && r < (int)grid.x; ++r) {
      rp[r] = s >= 0 ? pos[s] + r : pos[rs[r]];
      if (s >= 0) rs[r] = s;
    }
  } else if (is("10k_finalize")) {
    const int r0 = arg<int>(a, 0), n = arg<int>(a, 1);
    dev.hist = arg<int*>(a, 6);
    dev.max_ctx = arg<int>(a, 8);
    for (int r = r0; r < r0 + n; ++r) {
      const int s = arg<int*>(a, 2)[r], p = arg<int*>(a, 3)[r];
      if (arg<void*>(a, 4)) arg<int*>(a, 5)[s] = dev.hist[(size_t)s * dev.max_ctx + p] = dev.feed[r];
      arg<int*>(a, 7)[s] = p + 1;
    }
  } else if (is("k_copy_pages")) {
    dev.pool = arg<PagePool>(a, 0);
    const PairArgs& v = *static_cast<PairArgs*>(a[2]);
    for (int i = 0; i < v.n; ++i) move_page(dev.pool, v.src[i], v.dst[i]);
  } else if (is("k_fork_streams")) {
    const int src = arg<int>(a, 0), len = arg<int>(a, 1), ctx = arg<int>(a, 2), mp = arg<int>(a, 3), full = len / 16;
    const ForkArgs& v = *static_cast<ForkArgs*>(a[4]);
    int *table = arg<int*>(a, 5), *pos = arg<int*>(a, 6), *pending = arg<int*>(a, 7), *hist = arg<int*>(a, 9);
    dev.table = table;
    dev.max_pages = mp;
    for (int i = 0; i < v.n; ++i) {
      const int s = v.ids[i];
      std::copy(hist + (size_t)src * ctx, hist + (size_t)src * ctx + len, hist + (size_t)s * ctx);
      std::copy(table + (size_t)src * mp, table + (size_t)src * mp + full, table + (size_t)s * mp);
      if (v.has_last) table[(size_t)s * mp + full] = v.last[i];
      pos[s] = len;
      pending[s] = pending[src];
    }
  } else if (is("k_truncate_stream")) {
    const int s = arg<int>(a, 0), len = arg<int>(a, 1), ctx = arg<int>(a, 2);
    arg<int*>(a, 3)[s] = len;
    arg<int*>(a, 4)[s] = arg<int*>(a, 5)[(size_t)s * ctx + len - 1];
#ifndef TWO_LAUNCHES
    if (int* entry = arg<int*>(a, 6)) *entry = arg<int>(a, 7);
#endif
  } else if (is("k_compact_move")) {
    const PagePool p = arg<PagePool>(a, 0);
    int* table = arg<int*>(a, 4);
    const int rows = arg<int>(a, 5), mp = arg<int>(a, 6);
    const int* lens = arg<int*>(a, 7);
    std::vector<int> used(p.n_pages, 0), to(p.n_pages);
    for (int r = 0; r < rows; ++r)
      for (int i = 0; i < (lens[r] + 15) / 16; ++i) used[table[(size_t)r * mp + i]] = 1;
    const int live = (int)std::count(used.begin(), used.end(), 1);
    int hole = 0;
    for (int i = 0; i < p.n_pages; ++i) {
      to[i] = i;
      if (i < live || !used[i]) continue;
      while (used[hole]) ++hole;
      move_page(p, i, hole);
      to[i] = hole++;
    }
    for (int r = 0; r < rows; ++r)
      for (int i = 0; i < (lens[r] + 15) / 16; ++i) table[(size_t)r * mp + i] = to[table[(size_t)r * mp + i]];
  }
}

// ------------------------------------------------------------------ host memory

static int no_memory_in = -1;  // allocations before the one that fails; < 0: none does
static int asked = 0;
void* operator new(size_t n) {
  ++asked;
  if (no_memory_in == 0) throw std::bad_alloc();
  if (no_memory_in > 0) --no_memory_in;
  if (void* p = std::malloc(n ? n : 1)) return p;
  throw std::bad_alloc();
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }

// ------------------------------------------------------------------ streams

constexpr int kStreams = 5, kContext = 128;

struct Streams {
  hh_ctx* ctx = nullptr;
  void* arena = nullptr;
  std::vector<int> held[kStreams];      // each stream's tokens
  std::vector<char> recorded[kStreams];  // positions whose argmax was recorded
  std::mt19937 rng;
  int rand(int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); }

  hh_config config{};
  size_t bytes = 0;

  explicit Streams(unsigned seed, int max_prefill = 0) : rng(seed) {
    dev = Books();
    hh_config& c = config;
    c.n_layers = 2; c.d_model = 64; c.n_heads = 2; c.n_kv_heads = 1; c.head_dim = 64; c.ffn_dim = 64; c.vocab = 4096;
    c.rms_eps = 1e-5f; c.rope_theta = 10000.f; c.tied_embeddings = 1; c.dtype = HH_F32;
    c.max_streams = kStreams; c.max_context = kContext; c.page_size = 16; c.weight_format = HH_WF_DTYPE;
    c.max_prefill = max_prefill;
    CHECK(hh_workspace_size(&c, &bytes) == HH_OK);
    arena = std::aligned_alloc(256, (bytes + 255) / 256 * 256);
    std::memset(arena, 0, bytes);
    CHECK(hh_create(&c, arena, bytes, reinterpret_cast<void*>(256), &ctx) == HH_OK);
    const std::vector<float> w((size_t)4096 * 64, 0.f);
    const std::vector<const void*> tensors(1 + 9 * 2 + 1, w.data());
    CHECK(hh_load_weights(ctx, tensors.data(), (int)tensors.size()) == HH_OK);
    // Launches that tell where the books are.
    CHECK(feed(0, 17) == HH_OK);
    const int one = 1;
    CHECK(hh_fork(ctx, 0, 1, &one) == HH_OK);
    CHECK(hh_reset(ctx, -1) == HH_OK);
    held[0].clear();
    recorded[0].clear();
  }
  ~Streams() {
    hh_destroy(ctx);
    std::free(arena);
  }

  int* stamp(int s, int p, int layer) {
    const int page = dev.table[(size_t)s * dev.max_pages + p / 16];
    return reinterpret_cast<int*>(dev.pool.pool + layer * dev.pool.layer_stride + page * dev.pool.bytes) + p % 16;
  }
  // What the layers' kernels do: the rows' keys and values go into their pages.
  void added(int s, const std::vector<int>& t) {
    for (int x : t) {
      held[s].push_back(x);
      recorded[s].push_back(0);
      if (dev.table)
        for (int l = 0; l < 2; ++l) *stamp(s, (int)held[s].size() - 1, l) = x;
    }
    recorded[s].back() = 1;
  }
  std::vector<int> tokens(int n) {
    std::vector<int> t(n);
    for (int& x : t) x = rand(0, 4095);
    return t;
  }
  hh_status feed(int s, int n) {
    const std::vector<int> t = tokens(n);
    const hh_status rc = hh_prefill(ctx, s, t.data(), n, HH_LOGITS_NONE, nullptr, nullptr);
    if (rc == HH_OK) added(s, t);
    return rc;
  }
  hh_status step(int s) {
    const std::vector<int> t = tokens(1);
    const hh_status rc = hh_decode_step(ctx, 1, &s, t.data(), nullptr, nullptr);
    if (rc == HH_OK) added(s, t);
    return rc;
  }
  hh_status fork(int s, const std::vector<int>& dst) {
    const hh_status rc = hh_fork(ctx, s, (int)dst.size(), dst.data());
    for (int d : dst) {
      // After an error a listed stream is a fork, or as it was, or empty.
      int32_t n = -1;
      CHECK(hh_stream_length(ctx, d, &n) == HH_OK);
      if (rc == HH_OK || same(d, held[s])) {
        held[d] = held[s];
        recorded[d] = recorded[s];
      } else if (!same(d, held[d]) || n != (int)held[d].size()) {
        CHECK(n == 0);
        held[d].clear();
        recorded[d].clear();
      }
    }
    return rc;
  }
  hh_status cut(int s, int n) {
    const hh_status rc = hh_truncate(ctx, s, n);
    if (rc == HH_OK) {
      held[s].resize(n);
      recorded[s].resize(n);
    }
    return rc;
  }
  hh_status reset(int s) {
    const hh_status rc = hh_reset(ctx, s);
    if (rc == HH_OK) {
      held[s].clear();
      recorded[s].clear();
    }
    return rc;
  }
  bool same(int s, const std::vector<int>& t) {
    int32_t n = -1;
    if (hh_stream_length(ctx, s, &n) != HH_OK || n != (int)t.size() || dev.pos[s] != n) return false;
    for (int p = 0; p < n; ++p)
      for (int l = 0; l < 2; ++l)
        if (*stamp(s, p, l) != t[p]) return false;
    return true;
  }
  // Host, device and content agree.
  void check() {
    for (int s = 0; s < kStreams; ++s) {
      int32_t n = -1;
      CHECK(hh_stream_length(ctx, s, &n) == HH_OK && n == (int)held[s].size());
      CHECK(dev.pos[s] == n);
      CHECK(same(s, held[s]));
      if (n > 0 && recorded[s][n - 1]) {
        int32_t x = -1;
        CHECK(dev.pending[s] == held[s].back());
        CHECK(hh_read_argmax(ctx, s, n - 1, 1, &x) == HH_OK && x == held[s].back());
      }
    }
  }
  // No page is lost or held twice: the pool can be filled to its last page.
  void refill() {
    CHECK(hh_reset(ctx, -1) == HH_OK);
    for (int s = 0; s < kStreams; ++s) {
      held[s].clear();
      recorded[s].clear();
    }
    int32_t n = -1;
    CHECK(hh_compact(ctx, &n) == HH_OK && n == 0);
    for (int s = 0; s < kStreams; ++s) CHECK(feed(s, kContext) == HH_OK);
    check();
    CHECK(hh_compact(ctx, &n) == HH_OK && n == kStreams * kContext / 16);
    check();
  }
};

// One call whose k-th launch fails, for every k: nothing has happened, and the same call works then.
static void check_errors() {
  for (int what = 0; what < 4; ++what)
    for (int k = 0; k < 8; ++k) {
      Streams t(100 + what);
      at_op = what == 0 ? "cut" : what == 1 ? "fork" : what == 2 ? "compact" : "reset";
      CHECK(t.feed(2, 50) == HH_OK && t.feed(0, 45) == HH_OK && t.fork(0, {1, 3}) == HH_OK && t.reset(2) == HH_OK);
      t.check();
      auto call = [&] {
        int32_t n = 0;
        return what == 0 ? t.cut(1, 20) : what == 1 ? t.fork(0, {4, 3}) : what == 2 ? hh_compact(t.ctx, &n) : t.reset(3);
      };
      fail_in = k;
      const hh_status rc = call();
      const bool failed = fail_in < 0;
      fail_in = -1;
      CHECK(rc == (failed ? HH_ERR_HIP : HH_OK));
      (void)hipGetLastError();
      t.check();
      // Other streams take free pages; what the call left must not be among them.
      CHECK(t.feed(2, 30) == HH_OK);
      t.check();
      CHECK(call() == HH_OK);
      t.check();
      for (int s = 0; s < kStreams; ++s) CHECK(t.step(s) == HH_OK);
      t.check();
      t.refill();
    }
}

// The launch that uploads a prompt's or a step's new page-table entries fails: the stream is as it
// was, and the same call works then.
static void check_new_pages() {
  for (int what = 0; what < 3; ++what) {
    at_op = what == 0 ? "prompt" : what == 1 ? "batch of prompts" : "step";
    Streams t(20);
    CHECK(t.feed(0, 32) == HH_OK && t.fork(0, {2}) == HH_OK);
    const std::vector<int> a = t.tokens(20);
    const int ids[2] = {0, 1}, lens[2] = {20, 20};
    std::vector<int> both = a;
    both.insert(both.end(), a.begin(), a.end());
    auto call = [&] {
      if (what == 0) return hh_prefill(t.ctx, 0, a.data(), 20, HH_LOGITS_NONE, nullptr, nullptr);
      if (what == 1) return hh_prefill_batch(t.ctx, 2, ids, lens, both.data(), nullptr);
      return hh_decode_step(t.ctx, 1, ids, a.data(), nullptr, nullptr);
    };
    fail_in = 0;
    CHECK(call() == HH_ERR_HIP);
    CHECK(fail_in == -1);
    fail_in = -1;
    (void)hipGetLastError();
    t.check();
    CHECK(t.feed(3, 40) == HH_OK);
    t.check();
    CHECK(call() == HH_OK);
    t.added(0, what == 2 ? std::vector<int>(a.begin(), a.begin() + 1) : a);
    if (what == 1) t.added(1, a);
    if (what == 1) t.recorded[0].back() = t.recorded[1].back() = 0;  // (their argmaxes are not played here)
    t.check();
    for (int s : {2, 4}) CHECK(t.feed(s, 30) == HH_OK);
    t.check();
    t.refill();
  }
}

// Host memory runs out at the k-th allocation of a call (and stays out): HH_ERR_OOM, nothing thrown and
// nothing changed, or the call needed no more.
static void check_no_memory() {
  static const char* const names[] = {"prompt", "step", "steps", "batch", "fork", "cut", "compact", "reset", "create"};
  for (int what = 0; what < 9; ++what) {
    at_op = names[what];
    bool done = false;
    for (int k = 0; k < 200 && !done; ++k) {
      Streams t(30, 24);
      CHECK(t.feed(0, 30) == HH_OK && t.feed(1, 40) == HH_OK && t.fork(1, {2}) == HH_OK);
      const std::vector<int> a = t.tokens(60);
      const int ids[2] = {0, 1}, lens[2] = {30, 30}, dst[2] = {3, 4};
      int32_t n = 0;
      hh_ctx* made = nullptr;
      auto call = [&]() -> hh_status {
        switch (what) {
          case 0: return hh_prefill(t.ctx, 0, a.data(), 30, HH_LOGITS_NONE, nullptr, nullptr);
          case 1: return hh_decode_step(t.ctx, 1, ids, a.data(), nullptr, nullptr);
          case 2: return hh_decode_step(t.ctx, 2, ids, a.data(), nullptr, nullptr);
          case 3: return hh_prefill_batch(t.ctx, 2, ids, lens, a.data(), nullptr);
          case 4: return hh_fork(t.ctx, 1, 2, dst);
          case 5: return hh_truncate(t.ctx, 2, 35);
          case 6: return hh_compact(t.ctx, &n);
          case 7: return hh_reset(t.ctx, 2);
          default: return hh_create(&t.config, t.arena, t.bytes, reinterpret_cast<void*>(256), &made);
        }
      };
      asked = 0;
      no_memory_in = k;
      hh_status rc = HH_OK;
      bool thrown = false;
      try {
        rc = call();
      } catch (...) {
        thrown = true;
      }
      done = asked <= k;
      no_memory_in = -1;
      CHECK(!thrown);
      if (thrown) return;
      CHECK(rc == (done ? HH_OK : HH_ERR_OOM));
      if (what == 8) {
        if (made) hh_destroy(made);
        continue;
      }
      if (rc == HH_OK) {
        if (what == 0) t.added(0, {a.begin(), a.begin() + 30});
        if (what == 1 || what == 2) t.added(0, {a[0]});
        if (what == 2) t.added(1, {a[1]});
        if (what == 3) {
          t.added(0, {a.begin(), a.begin() + 30});
          t.added(1, {a.begin() + 30, a.end()});
          t.recorded[0].back() = t.recorded[1].back() = 0;
        }
        for (int d : dst)
          if (what == 4) t.held[d] = t.held[1], t.recorded[d] = t.recorded[1];
        if (what == 5) t.held[2].resize(35), t.recorded[2].resize(35);
        if (what == 7) t.held[2].clear(), t.recorded[2].clear();
      }
      t.check();
      CHECK(t.step(1) == HH_OK);
      t.check();
      t.refill();
    }
    CHECK(done);
  }
}

// A full pool: the forks' copies take pages that their streams held.
static void check_full_pool() {
  for (int k = -1; k < 8; ++k) {
    at_op = "fork in a full pool";
    Streams t(7);
    CHECK(t.feed(0, kContext - 5) == HH_OK);
    for (int s = 1; s < kStreams; ++s) CHECK(t.feed(s, kContext) == HH_OK);
    fail_in = k;
    const hh_status rc = t.fork(0, {1, 2, 3, 4});
    CHECK(rc == (k >= 0 && fail_in < 0 ? HH_ERR_HIP : HH_OK));
    fail_in = -1;
    (void)hipGetLastError();
    t.check();
    CHECK(t.fork(0, {4, 3, 2, 1}) == HH_OK);
    t.check();
    for (int s = 0; s < kStreams; ++s) CHECK(t.feed(s, 5) == HH_OK);
    t.check();
    t.refill();
  }
}

// An error that another call left is neither taken nor reported.
static void check_pending_error() {
  Streams t(9);
  at_op = "pending error";
  CHECK(t.feed(0, 45) == HH_OK);
  last_error = hipErrorInvalidDevice;
  CHECK(t.fork(0, {1, 2}) == HH_OK && t.cut(1, 20) == HH_OK && t.cut(2, 40) == HH_OK && t.reset(0) == HH_OK);
  int32_t n = 0;
  CHECK(hh_compact(t.ctx, &n) == HH_OK && n == 4);
  CHECK(last_error == hipErrorInvalidDevice);
  (void)hipGetLastError();
  t.check();
  // Prompts and steps (no new page, and with one) report it and do nothing.
  CHECK(t.cut(2, 31) == HH_OK);
  for (int i = 0; i < 6; ++i) {
    at_op = i % 3 == 0 ? "prompt after an error" : i % 3 == 1 ? "step after an error" : "batch after an error";
    const std::vector<int> a = t.tokens(1);
    const int id = 2, one = 1;
    auto call = [&] {
      if (i % 3 == 2) return hh_prefill_batch(t.ctx, 1, &id, &one, a.data(), nullptr);
      return i % 3 == 1 ? hh_decode_step(t.ctx, 1, &id, a.data(), nullptr, nullptr)
                        : hh_prefill(t.ctx, id, a.data(), 1, HH_LOGITS_NONE, nullptr, nullptr);
    };
    last_error = hipErrorInvalidDevice;
    CHECK(call() == HH_ERR_HIP);
    CHECK(last_error == hipSuccess);
    t.check();
    CHECK(call() == HH_OK);
    t.added(id, a);
    if (i % 3 == 2) t.recorded[id].back() = 0;
    t.check();
  }
}

static void check_any_order() {
  for (unsigned seed = 0; seed < 60; ++seed) {
    Streams t(seed);
    for (int i = 0; i < 150; ++i) {
      const int s = t.rand(0, kStreams - 1), what = t.rand(0, 9), len = (int)t.held[s].size();
      if (what >= 4 && t.rand(0, 3) == 0) fail_in = t.rand(0, 3);
      if (what <= 2 && len < kContext) {
        at_op = "prompt";
        CHECK(t.feed(s, t.rand(1, std::min(40, kContext - len))) == HH_OK);
      } else if (what == 3 && len < kContext) {
        at_op = "step";
        CHECK(t.step(s) == HH_OK);
      } else if (what <= 6) {
        at_op = "fork";
        std::vector<int> all = {0, 1, 2, 3, 4};
        all.erase(all.begin() + s);
        std::shuffle(all.begin(), all.end(), t.rng);
        all.resize(t.rand(1, kStreams - 1));
        t.fork(s, all);
      } else if (what <= 7) {
        at_op = "cut";
        t.cut(s, t.rand(0, len));
      } else if (what == 8) {
        at_op = "compact";
        hh_compact(t.ctx, nullptr);
      } else {
        at_op = "reset";
        t.reset(s);
      }
      fail_in = -1;
      (void)hipGetLastError();
      t.check();
      if (failures) {
        std::fprintf(stderr, "(seed %u, call %d)\n", seed, i);
        return;
      }
    }
    t.refill();
  }
}

int main() {
  check_pending_error();
  check_errors();
  check_new_pages();
  check_no_memory();
  check_full_pool();
  check_any_order();
  if (failures) {
    std::fprintf(stderr, "%d stream checks failed\n", failures);
    return 1;
  }
  std::printf("stream checks passed (%d launches)\n", launches);
  return 0;
}
