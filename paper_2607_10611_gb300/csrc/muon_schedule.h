// muon_schedule.h -- the order in which the tiles of all Newton-Schulz products
// of a list are taken (muon_products.cu), made on the host once a list (internal
// to the CUDA library).
#pragma once

#include <algorithm>
#include <cstdint>
#include <queue>
#include <vector>

#include "muon.h"

namespace mpadam {

inline int32_t newton_across(int32_t n) { return (n + kNewtonTile - 1) / kNewtonTile; }
inline int32_t newton_steps_k(int32_t n) { return (n + kNewtonStepK - 1) / kNewtonStepK; }
// Tiles of a matrix's products 1 and 2 (on and below the diagonal), and of 3.
inline int64_t newton_tiles(int which, int32_t r, int32_t c) {
  const int64_t a = newton_across(r);
  return which == 3 ? a * newton_across(c) : a * (a + 1) / 2;
}

// Appends the tiles of matrices [first, last) to `tiles`, each behind those that
// it waits for.  The list is what a run would do with `pairs` pairs of CTAs whose
// tiles take their steps' time and some more: a free pair goes on with the started
// matrix that has the longest way to go, and starts another one, the longest first,
// where no started one has a tile that can be made.  So few matrices are under way at
// once, and what they hold stays in L2.
inline void newton_schedule(const std::vector<NewtonMatrix>& matrices, int32_t first, int32_t last, int32_t newton_steps, int pairs,
                            std::vector<NewtonTile>* tiles) {
  // Of a tile, in steps of k: until its pair is free, and until its result can be used.  The second is more than the tile's own
  // way (about 20 steps): pairs take tiles ahead.  A Muon step of a 1.5B-width layer takes 1690 us with 20 (in a long run), 1640 to
  // 1665 with 48, 72 and 96; half of GPT-2's matrices and 4096 x 11008 alone the same with all of them.
  constexpr int64_t kBetween = 1, kLatency = 72;
  struct Tile {
    int64_t way;     // of the matrix from this product on
    int32_t chain;
    int32_t product; // 3 a Newton-Schulz step
    int64_t order;   // in the product
    int32_t tm, tn;
    bool operator<(const Tile& o) const {  // later
      if (way != o.way) return way < o.way;
      if (chain != o.chain) return chain > o.chain;
      if (product != o.product) return product > o.product;
      return order > o.order;
    }
  };
  struct Chain {
    int32_t matrix;
    std::vector<int64_t> stored;    // tiles, of every 256 rows
    std::vector<int32_t> products;  // whose operands these rows have all
  };
  struct Done {
    int64_t when;
    int32_t chain, which, tm, tn;
    bool operator<(const Done& o) const { return when > o.when; }
  };
  auto steps_of = [&](int32_t m, int which) { return newton_steps_k(which == 1 ? matrices[m].c : matrices[m].r); };
  // The way to go before product `product` is done, at best.
  auto way = [&](int32_t m, int32_t product) {
    const int64_t one = steps_of(m, 1) + kLatency, other = steps_of(m, 2) + kLatency;
    const int32_t left = 3 * newton_steps - product;
    return left / 3 * (one + 2 * other) + left % 3 * other;
  };
  // Tiles that were stored in any 256 rows before product `product` can use these.
  auto need = [&](int32_t m, int32_t product) {
    const int64_t d = newton_across(matrices[m].r);
    return product / 3 * (2 * d + newton_across(matrices[m].c)) + product % 3 * d;
  };
  std::vector<Chain> chains;
  for (int32_t m = first; m < last; ++m) chains.push_back({m, {}, {}});
  std::stable_sort(chains.begin(), chains.end(), [&](const Chain& a, const Chain& b) { return way(a.matrix, 0) > way(b.matrix, 0); });
  std::priority_queue<Tile> ready;
  std::priority_queue<Done> coming;
  using Pair = std::pair<int64_t, int>;
  std::priority_queue<Pair, std::vector<Pair>, std::greater<Pair>> free;
  for (int i = 0; i < pairs; ++i) free.push({0, i});
  int32_t started = 0;

  // Rows i of a chain are ready for one more product: the tiles that this completes the operands of.
  auto advance = [&](int32_t c, int32_t i) {
    Chain& chain = chains[c];
    const NewtonMatrix& q = matrices[chain.matrix];
    const int32_t product = chain.products[i]++;
    if (product >= 3 * newton_steps) return;
    const int64_t w = way(chain.matrix, product), down = newton_across(q.r), across = newton_across(q.c);
    if (product % 3 == 2) {  // 8 rows of tiles at a time, so that neighbours in time meet in L2
      for (int32_t n = 0; n < across; ++n) ready.push({w, c, product, (i / 8 * across + n) * 8 + i % 8, i, n});
    } else {  // column by column, which has its first rows complete first
      for (int32_t j = 0; j < down; ++j)
        if (chain.products[j] > product) ready.push({w, c, product, std::min(i, j) * down + std::max(i, j), std::max(i, j), std::min(i, j)});
    }
  };
  while (true) {
    const auto [now, pair] = free.top();
    while (!coming.empty() && coming.top().when <= now) {
      const Done t = coming.top();
      coming.pop();
      Chain& chain = chains[t.chain];
      for (int32_t row : {t.tm, t.tn}) {
        if (++chain.stored[row] == need(chain.matrix, chain.products[row])) advance(t.chain, row);
        if (t.which == 3 || t.tm == t.tn) break;
      }
    }
    if (ready.empty() && started < (int32_t)chains.size()) {
      Chain& chain = chains[started];
      const int32_t down = newton_across(matrices[chain.matrix].r);
      chain.stored.assign(down, 0);
      chain.products.assign(down, 0);
      for (int32_t i = 0; i < down; ++i) advance(started, i);
      ++started;
    }
    if (ready.empty()) {
      if (coming.empty()) return;
      free.pop();
      free.push({coming.top().when, pair});
      continue;
    }
    const Tile t = ready.top();
    ready.pop();
    const int32_t m = chains[t.chain].matrix, step = t.product / 3, which = t.product % 3 + 1, k = steps_of(m, which);
    // X's second part is for the sum a X of all steps but the last, in which it no longer matters.
    const bool adds = which == 2 || (which == 3 && step + 1 < newton_steps), keep_lo = which == 3 && step + 2 < newton_steps;
    tiles->push_back(NewtonTile::make(m, t.tm, t.tn, k, which, step & 1, adds, keep_lo, (uint32_t)(kSignals * need(m, t.product))));
    free.pop();
    free.push({now + k + kBetween, pair});
    coming.push({now + k + kLatency, t.chain, which, t.tm, t.tn});
  }
}

}  // namespace mpadam
