// Test-only host program: newton_schedule's tiles for matrices given on the command line (steps, then r and c of each), one a
// line: matrix, which product, tm, tn, steps of k, need, from, adds, keep_lo, and its matrix's rows of tiles.
#include <cstdio>
#include <cstdlib>

#include "muon_schedule.h"

int main(int argc, char** argv) {
  using namespace mpadam;
  const int steps = std::atoi(argv[1]);
  std::vector<NewtonMatrix> matrices;
  for (int i = 2; i + 1 < argc; i += 2) {
    NewtonMatrix q{};
    q.r = std::atoi(argv[i]), q.c = std::atoi(argv[i + 1]);
    matrices.push_back(q);
  }
  std::vector<NewtonTile> tiles;
  newton_schedule(matrices, 0, (int32_t)matrices.size(), steps, kNewtonPairs, &tiles);
  for (const NewtonTile& t : tiles)
    std::printf("%d %d %d %d %d %u %d %d %d\n", t.matrix, t.which(), t.tm, t.tn, t.steps_k(), t.need, t.from(), (int)t.adds(), (int)t.keep_lo());
}
