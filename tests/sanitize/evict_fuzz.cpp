// Randomised evictions under AddressSanitizer and UndefinedBehaviorSanitizer
// (built by tests/test_host_sanitize_evict.py with g++; no GPU code): the KV
// block allocator's seq_evict and seq_undo_evict among the other operations,
// valid and invalid, with its invariants after every step, and the positions of
// the batches that evicted sequences are in.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <string>
#include <vector>

#include "../../paper_2609_37062_amd/csrc/alloc.hpp"

using namespace vsk;

#define CHECK(c)                                                          \
  do {                                                                    \
    if (!(c)) {                                                           \
      std::fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #c); \
      std::exit(2);                                                       \
    }                                                                     \
  } while (0)

struct Want {
  int32_t len = 0, dropped = 0;
};

static void check(const BlockAllocator& a, const std::map<int64_t, Want>& live) {
  std::vector<int32_t> refs(a.n_blocks(), 0);
  for (const auto& kv : live) {
    const SeqState* s = a.find(kv.first);
    CHECK(s != nullptr && s->len == kv.second.len && s->dropped == kv.second.dropped);
    CHECK(static_cast<int64_t>(s->blocks.size()) * a.block() >= s->len);
    std::set<int32_t> seen;
    for (int32_t b : s->blocks) {
      CHECK(b >= 0 && b < a.n_blocks() && seen.insert(b).second);
      ++refs[b];
    }
  }
  int32_t free_blocks = 0;
  for (int32_t b = 0; b < a.n_blocks(); ++b) {
    free_blocks += refs[b] == 0;
    CHECK(a.shared(b) == (refs[b] > 1));
  }
  CHECK(free_blocks == a.free_count());
}

int main(int argc, char** argv) {
  const int rounds = argc > 1 ? std::atoi(argv[1]) : 100;
  int done = 0, undone = 0, refused = 0, batches = 0;
  std::string err;
  for (int round = 0; round < rounds; ++round) {
    std::mt19937 rng(1000 + round);
    auto below = [&](int n) { return static_cast<int>(rng() % static_cast<unsigned>(n)); };
    BlockAllocator a(20 + below(100));
    std::map<int64_t, Want> live;
    int64_t next = 0;
    auto any = [&]() -> int64_t {
      if (live.empty() || below(12) == 0) return 1000000 + below(3);  // unknown
      auto it = live.begin();
      std::advance(it, below(static_cast<int>(live.size())));
      return it->first;
    };
    for (int step = 0; step < 120; ++step) {
      const int what = below(10);
      if (what < 2 || live.empty()) {
        CHECK(a.seq_create(next, err) == kOk);
        live[next++] = Want{};
      } else if (what < 4) {
        const int64_t s = any();
        const int32_t n = below(90);
        const int st = a.reserve(s, n, nullptr, err);
        if (st == kOk) live.at(s).len += n;
      } else if (what < 5) {
        const int64_t s = any();
        if (a.seq_release(s, err) == kOk) live.erase(s);
      } else if (what < 6) {
        const int64_t d = any(), s = any();
        const int32_t n = 16 * below(4);
        const SeqState* src = a.find(s);
        const bool evicted = src != nullptr && src->dropped != 0;
        const int st = a.seq_share_prefix(d, s, n, err);
        CHECK(!(st == kOk && evicted));
        if (st == kOk) live.at(d).len = n;
      } else if (what < 7) {
        std::vector<int64_t> seqs;
        std::vector<int32_t> q;
        for (const auto& kv : live)
          if (kv.second.len > 0 && below(2)) {
            seqs.push_back(kv.first);
            q.push_back(1 + below(kv.second.len));
          }
        BatchHost b;
        if (!seqs.empty() && build_batch(a, seqs.data(), q.data(), static_cast<int32_t>(seqs.size()), b, err) == kOk) {
          ++batches;
          bool evicted = false;
          int32_t top = 0, r = 0;
          for (size_t i = 0; i < seqs.size(); ++i) {
            const Want& x = live.at(seqs[i]);
            evicted = evicted || x.dropped != 0;
            for (int32_t p = x.len - q[i]; p < x.len; ++p, ++r) {
              CHECK(b.pos[r] == p && b.rot[r] == p + x.dropped);
              top = b.rot[r] > top ? b.rot[r] : top;
            }
          }
          CHECK(b.evicted == evicted && b.max_position == top);
        }
      } else {
        const int n = 1 + below(4);
        std::vector<int64_t> dst(n), src(n);
        std::vector<int32_t> keep(n);
        for (int i = 0; i < n; ++i) {
          dst[i] = any();
          if (below(8)) {
            CHECK(a.seq_create(next, err) == kOk);
            live[next] = Want{};
            dst[i] = next++;
          }
          src[i] = any();
          const SeqState* s = a.find(src[i]);
          keep[i] = s != nullptr && s->len > 0 && below(10) ? 1 + below(s->len) : below(200) - 50;
        }
        const int32_t free_before = a.free_count();
        const int st = a.seq_evict(dst.data(), src.data(), keep.data(), n, err);
        if (st != kOk) {
          ++refused;
          CHECK(a.free_count() == free_before);
        } else if (below(5) == 0) {
          ++undone;
          a.seq_undo_evict(dst.data(), n);
          CHECK(a.free_count() == free_before);
        } else {
          ++done;
          for (int i = 0; i < n; ++i) {
            const Want s = live.at(src[i]);
            CHECK(keep[i] >= 1 && keep[i] <= s.len);
            live.at(dst[i]) = Want{keep[i], s.dropped + s.len - keep[i]};
            for (int32_t b : a.find(dst[i])->blocks) CHECK(!a.shared(b));
          }
        }
      }
      check(a, live);
    }
  }
  std::printf("passed: %d evictions, %d undone, %d refused, %d batches\n", done, undone, refused, batches);
  return 0;
}
