// Every order in which a row tile's issuer and the warps of its two streams can take the steps of a piece in the chunk kernel, with the
// waits that kv_handoff.h names, for test_kv_handoff.py.  Prints how many states were met and in how many
// of them a product with V wrote O before both streams had read the maxima that lie there, and in how many nobody could go on.
//   kv_handoff_check key_tiles
#include <array>
#include <cstdio>
#include <cstdlib>
#include <set>

#include "../paper_2512_04939_b200/csrc/kv_handoff.h"

namespace {

// A stream's warp: 0 stores its maximum, 1 waits for the other one's, 2 reads both, then per key tile: waits for its scores, takes
// them and hands over its probabilities.  The issuer: the first scores of both streams, then per key tile and stream: waits, the product
// with V, the next scores.
using State = std::array<int, 7>;  // issuer's step, per stream: step, probabilities handed over, score tiles issued

int tiles;
std::set<State> met;
int early = 0, stuck = 0;

int issuer(const State& s) { return s[0]; }
int step(const State& s, int c) { return s[1 + c]; }
int given(const State& s, int c) { return s[3 + c]; }
int scores(const State& s, int c) { return s[5 + c]; }

void visit(const State& s) {
  if (!met.insert(s).second) return;
  bool moved = false;
  if (issuer(s) == 0) {
    State n = s;
    n[0] = 1, n[5] = n[6] = 1;
    moved = true;
    visit(n);
  } else if (issuer(s) <= 2 * tiles) {
    const int j = (issuer(s) - 1) / 2, c = (issuer(s) - 1) % 2;
    bool go = true;
    for (int other = 0; other < 2; ++other) go = go && (!lv::kv_awaits(j, c, other) || given(s, other) > j);
    if (go) {
      for (int other = 0; other < 2; ++other) early += step(s, other) <= 2 ? 1 : 0;
      State n = s;
      ++n[0];
      if (j + 1 < tiles) ++n[5 + c];
      moved = true;
      visit(n);
    }
  }
  for (int c = 0; c < 2; ++c) {
    State n = s;
    const int at = step(s, c);
    if (at == 0) {
      if (scores(s, c) < 1) continue;  // the maximum is of the first scores
      n[1 + c] = 1;
    } else if (at == 1) {
      if (step(s, 1 - c) < 1) continue;
      n[1 + c] = 2;
    } else if (at == 2) {
      n[1 + c] = 3;
    } else {
      if (given(s, c) >= tiles || scores(s, c) <= given(s, c)) continue;
      ++n[3 + c];
    }
    moved = true;
    visit(n);
  }
  if (!moved && !(issuer(s) == 2 * tiles + 1 && given(s, 0) == tiles && given(s, 1) == tiles)) ++stuck;
}

}  // namespace

int main(int, char** argv) {
  tiles = atoi(argv[1]);
  visit(State{});
  printf("%zu %d %d\n", met.size(), early, stuck);
  return 0;
}
