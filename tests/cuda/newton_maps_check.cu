// Test-only host program: the tensor maps that tile_map gives for every product and either X, by their names; one line each,
// "which from name name ...".
#include <cstdio>

#include "muon.h"

int main() {
  using namespace mpadam;
  static NewtonMatrix q;
  const std::pair<const char*, const CUtensorMap*> maps[] = {
      {"x0", &q.x[0]}, {"x1", &q.x[1]}, {"a", &q.a}, {"b", &q.b}, {"x_along0", &q.x_along[0]}, {"x_along1", &q.x_along[1]},
      {"a_along", &q.a_along}, {"b_along", &q.b_along}, {"x_patch0", &q.x_patch[0]}, {"x_patch1", &q.x_patch[1]},
      {"lo_patch", &q.lo_patch}, {"a_patch", &q.a_patch}, {"b_patch", &q.b_patch}};
  static_assert(kTileMaps <= 32 && sizeof(maps) / sizeof(maps[0]) == kNewtonMaps, "a lane each; all maps");
  for (int which = 1; which <= 3; ++which)
    for (int from = 0; from < 2; ++from) {
      std::printf("%d %d", which, from);
      for (int i = 0; i < kTileMaps; ++i) {
        const char* found = "none";
        for (const auto& [name, map] : maps)
          if (newton_map(&q, tile_map(which, from, i)) == map) found = name;
        std::printf(" %s", found);
      }
      std::printf("\n");
    }
}
