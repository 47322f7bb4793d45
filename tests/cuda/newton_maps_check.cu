// Test-only host program: which of the tensor maps of a list newton_map reaches by the numbers of matrices [first, first +
// members), and how often; one line a map, "matrix name times".
#include <cstdio>
#include <cstdlib>
#include <map>
#include <vector>

#include "muon.h"

int main(int argc, char** argv) {
  using namespace mpadam;
  const int all = std::atoi(argv[1]), first = std::atoi(argv[2]), members = std::atoi(argv[3]);
  std::vector<NewtonMatrix> list(all);
  std::map<const CUtensorMap*, int> times;
  for (int64_t i = 0; i < (int64_t)kNewtonMaps * members; ++i) ++times[newton_map(list.data() + first, i)];
  for (int m = 0; m < all; ++m) {
    const NewtonMatrix& q = list[m];
    const std::pair<const char*, const CUtensorMap*> maps[] = {
        {"x0", &q.x[0]}, {"x1", &q.x[1]}, {"a", &q.a}, {"b", &q.b}, {"x_along0", &q.x_along[0]}, {"x_along1", &q.x_along[1]},
        {"a_along", &q.a_along}, {"b_along", &q.b_along}, {"x_patch0", &q.x_patch[0]}, {"x_patch1", &q.x_patch[1]},
        {"lo_patch", &q.lo_patch}, {"a_patch", &q.a_patch}, {"b_patch", &q.b_patch}};
    for (const auto& [name, map] : maps) {
      std::printf("%d %s %d\n", m, name, times.count(map) ? times[map] : 0);
      times.erase(map);
    }
  }
  std::printf("others %zu\n", times.size());
}
