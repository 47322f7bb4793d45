// Test-only host program: the end of a pair of CTAs (pair_open, pair_step in muon.h) played through with copies that land in any
// order and roles that stop at any time.  Arguments: stages, seed, rounds.  Says "ok", or what went wrong.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "muon.h"

using namespace mpadam;

namespace {

constexpr int kHalf = 32;  // bytes of a CTA's half of a step

// A barrier of one arrival: a phase is over when that has come and no announced byte is missing (bytes may come first).
struct Barrier {
  int over = 0, pending = 1, bytes = 0;
  void look() {
    if (pending == 0 && bytes == 0) ++over, pending = 1;
  }
  bool announce(int n) {
    if (pending == 0) return false;
    bytes += n, --pending;
    look();
    return true;
  }
  void land(int n) { bytes -= n, look(); }
  bool passed(int parity) const { return (over & 1) != parity; }  // of the last phases, as the hardware's wait sees it
};

struct Copy {
  int step;
};

int fail(const char* what, unsigned seed) {
  std::printf("%s (seed %u)\n", what, seed);
  return 1;
}

int play(int stages, unsigned seed, int* uneven) {
  std::mt19937 rng(seed);
  auto pick = [&](int n) { return (int)(rng() % n); };
  std::vector<Barrier> full(stages);
  std::vector<Copy> flying;
  const int steps = pick(4 * stages + 2);
  int asked[2] = {0, 0}, taken = 0;  // taken: steps that the issuer has multiplied
  bool on[3] = {true, true, true};   // the producers, the issuer
  auto land = [&] {
    const int i = pick((int)flying.size());
    full[flying[i].step % stages].land(kHalf);
    flying.erase(flying.begin() + i);
  };
  const int stops = pick(3) ? 40 : 1000000;  // some runs go to their end
  while (on[0] || on[1] || on[2]) {
    const int who = pick(4);
    if (who < 3 && pick(stops) == 0) on[who] = false;
    if (who < 2 && on[who]) {
      if (asked[who] == steps) {
        on[who] = false;
      } else if (asked[who] < taken + stages) {  // its stage has been given back
        const int at = asked[who] % stages;
        if (who == 0 && !full[at].announce(2 * kHalf)) return fail("announced twice", seed);
        flying.push_back({asked[who]++});
      } else if (!on[2]) {
        on[who] = false;  // a wait that gives up
      }
    } else if (who == 2 && on[2]) {
      if (taken == steps) on[2] = false;
      else if (full[taken % stages].passed(taken / stages & 1)) {
        for (const Copy& c : flying)
          if (c.step == taken) return fail("a step was taken before it was whole", seed);
        ++taken;
      } else if (!on[0] || !on[1]) {
        if (pick(8) == 0) on[2] = false;
      }
    } else if (who == 3 && !flying.empty() && pick(2)) {
      land();
    }
  }
  *uneven += asked[0] != asked[1];
  const int end = pair_end(asked[0], asked[1]), open = pair_open(asked[0], asked[1], stages);
  for (const Copy& c : flying)
    if (c.step < open || c.step >= end) return fail("a copy of a step that nobody waits for", seed);
  for (int i = open; i < end; ++i) {
    const PairStep what = pair_step(i, asked[0], asked[1]);
    if (what == PairStep::kNoPeer) full[i % stages].land(kHalf);
    if (what == PairStep::kNoLeader && !full[i % stages].announce(kHalf)) return fail("announced twice at the end", seed);
  }
  auto whole = [&] {
    for (int i = open; i < end; ++i)
      if (!full[i % stages].passed(i / stages & 1)) return false;
    return true;
  };
  while (!flying.empty()) {
    if (whole()) return fail("the waits end while a copy is in flight", seed);
    land();
  }
  if (!whole()) return fail("the waits do not end", seed);
  for (const Barrier& b : full)
    if (b.pending != 1 || b.bytes != 0) return fail("a barrier is left within a phase", seed);
  return 0;
}

}  // namespace

int main(int argc, char** argv) {
  const int stages = std::atoi(argv[1]), rounds = std::atoi(argv[3]);
  int uneven = 0;
  for (int i = 0; i < rounds; ++i)
    if (play(stages, (unsigned)std::atoi(argv[2]) + i, &uneven)) return 1;
  if (uneven < rounds / 20) return fail("the CTAs hardly ever stopped apart", 0);
  std::printf("ok\n");
}
