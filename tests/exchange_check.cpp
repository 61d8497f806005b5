// Host check of the agreement on a launch's start (csrc/plan.h: start_of, moved_term): launches are
// played work-group by work-group, as check_xcd does, over random starts, sizes and strays.
// Prints "failures 0".
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "plan.h"

namespace {

// What a launch leaves in LaunchStatus::moved, and the start it reports (-1: none).
struct Left {
  uint64_t moved;
  int reported;
};

// xcd[b]: where work-group b ran; known: StepArgs::l2_start.
Left play(const std::vector<uint32_t>& xcd, uint32_t n, uint32_t known, int32_t seq) {
  Left r{0, -1};
  for (uint32_t b = 0; b < xcd.size(); ++b) {
    if (seq > 0 && xcd[b] == (b + known) % n) continue;
    const uint32_t start = infs::start_of(xcd[b], b, n);
    if (b == 0) r.reported = (int)start;
    r.moved += infs::moved_term(seq, seq > 0 ? start : start + b, b, (uint32_t)xcd.size());
  }
  return r;
}

std::vector<uint32_t> round_robin(uint32_t blocks, uint32_t n, uint32_t start) {
  std::vector<uint32_t> xcd(blocks);
  for (uint32_t b = 0; b < blocks; ++b) xcd[b] = (start + b) % n;
  return xcd;
}

}  // namespace

int main(int argc, char** argv) {
  const int rounds = argc > 1 ? std::atoi(argv[1]) : 1000;
  std::mt19937_64 rng(7);
  auto below = [&](uint32_t m) { return (uint32_t)(rng() % m); };
  int failures = 0;
  auto expect = [&](bool ok, const char* what, int r) {
    if (!ok && ++failures < 10) std::printf("%s, round %d\n", what, r);
  };
  uint64_t all = 0;  // over every launch with strays: never 0 again
  for (int r = 0; r < rounds; ++r) {
    const uint32_t n = r % 3 == 0 ? 8 : 1 + below(15), blocks = r % 5 == 0 ? 1 + below(9) : 1 + below(3000);
    const uint32_t start = below(n), known = r % 2 == 0 ? start : below(n);
    const int32_t seq = r % 7 == 0 ? INT32_MAX - r : 1 + r;
    std::vector<uint32_t> xcd = round_robin(blocks, n, start);
    const Left same = play(xcd, n, known, seq);
    expect(same.moved == 0, "agreeing work-groups leave a sum", r);
    expect(same.reported == (start == known ? -1 : (int)start), "reported start", r);
    if (blocks > 1) {
      expect(play(xcd, n, known, -seq).moved != 0, "a failing check leaves no sum", r);
      // all of the known start but the first, which the others cannot see (and the other way round)
      if (n > 1) {
        std::vector<uint32_t> first = round_robin(blocks, n, known), last = xcd;
        first[0] = (known + 1 + below(n - 1)) % n;
        expect(play(first, n, known, seq).moved != 0, "a stray first work-group passes", r);
        last[0] = known;
        expect(start == known || play(last, n, known, seq).moved != 0, "a first work-group of the known start passes", r);
        // strays on any place, one to all
        std::vector<uint32_t> some = xcd;
        for (uint32_t k = 1 + below(r % 4 == 0 ? 3 : blocks); k > 0; --k) some[below(blocks)] = below(n);
        bool agree = true;
        for (uint32_t b = 0; b < blocks; ++b)
          agree = agree && infs::start_of(some[b], b, n) == infs::start_of(some[0], 0, n);
        const uint64_t left = play(some, n, known, seq).moved;
        expect((left == 0) == agree, "strays", r);
        all += left;
        expect(all != 0 || left == 0, "launches cancel each other", r);
      }
    }
  }
  std::printf("failures %d\n", failures);
  return failures != 0;
}
