// Rings of barriers as the products fill and empty them, with everything stopped at a random
// point, to check what the kernels then wait for (csrc/ring.cuh).  Plain host code.
#include <cstdint>
#include <random>
#include <vector>

#include "ring.cuh"

namespace {

// A barrier of `count` arrivals a phase, whose phase ends once its bytes are here too.
struct Barrier {
  uint32_t count = 1, arrived = 0;
  int64_t bytes = 0;  // still expected
  uint64_t phases = 0;
  void step() {
    if (arrived == count && bytes == 0) {
      ++phases;
      arrived = 0;
    }
  }
  void arrive(int64_t expect) {
    bytes += expect;
    ++arrived;
    step();
  }
  void land(int64_t n) {
    bytes -= n;
    step();
  }
  // what mbarrier.try_wait.parity answers
  bool done(uint32_t parity) const { return (phases & 1) != parity; }
};

struct Copy {
  uint32_t stage;
  int64_t bytes;
};

}  // namespace

// One run: `threads` threads fill `n` stages in turn, a reader frees them in turn, copies land in any
// order, and all stop after `steps` steps.  0, or what went wrong: 1 a wait that nothing
// ends, 2 a copy on its way after the waits, 3 (checks the model) a phase that ended too often.
extern "C" int ring_run(uint32_t n, uint32_t threads, uint32_t steps, uint32_t seed) {
  std::mt19937 rng(seed);
  auto pick = [&](uint32_t k) { return (uint32_t)(rng() % k); };
  std::vector<Barrier> bar(n);
  for (auto& b : bar) b.count = threads;
  std::vector<Copy> flying;
  std::vector<uint64_t> fills(threads, 0);
  uint64_t read = 0;
  gleam::Ring at;  // the reader's position
  auto land = [&](size_t k) {
    const Copy c = flying[k];
    flying.erase(flying.begin() + k);
    bar[c.stage].land(c.bytes);
  };
  for (uint32_t s = 0; s < steps; ++s) {
    const uint32_t what = pick(threads + 2);
    if (what < threads) {
      if (fills[what] < read + n) {  // the stage has been freed as often as it was filled
        const uint32_t i = (uint32_t)(fills[what] % n);
        const int64_t bytes = pick(4) == 0 ? 0 : 16 * (1 + (int64_t)pick(8));
        bar[i].arrive(bytes);
        if (bytes != 0) flying.push_back({i, bytes});
        ++fills[what];
      }
    } else if (what == threads) {
      if (bar[at.i].done(at.phase)) {
        if (bar[at.i].phases != read / n + 1) return 3;
        ++read;
        at.next(n);
      }
    } else if (!flying.empty()) {
      land(pick((uint32_t)flying.size()));
    }
  }
  int bad = 0;
  gleam::settle_ring(
      fills.data(), threads, n, [&](uint32_t i) { bar[i].arrive(0); },
      [&](uint32_t i, uint32_t parity) {
        while (!bar[i].done(parity)) {
          std::vector<size_t> mine;
          for (size_t k = 0; k < flying.size(); ++k)
            if (flying[k].stage == i) mine.push_back(k);
          if (mine.empty()) {
            bad = 1;
            return;
          }
          land(mine[pick((uint32_t)mine.size())]);
        }
      });
  if (bad) return bad;
  return flying.empty() ? 0 : 2;
}
