// A producer's walk over segments whose queries are loaded onto one barrier, given up at every wait in turn: whether the copy that is
// then in flight is waited for.  Prints how many of the walks leave one behind, with the count and with a count of whole segments.
#include <cstdio>

#include "bd_copies.h"

struct Barrier {                       // as an mbarrier that each copy completes a phase of
  int landed = 0;
  bool returns_at_once(uint32_t parity) const { return ((uint32_t)landed & 1u) != parity; }
};

struct Outcome {
  bool left_count, left_segments, waits_for_nothing;
};

// Gives up at wait `stop`; `landed`: whether the last copy has landed by then.  tiles, early: of a segment, and before which the queries come.
static Outcome walk(int segments, int tiles, int early, int stop, bool landed, bool* reached) {
  bd::CopyCount queries{1};            // the first segment's, by another warp
  int waits = 0, whole = 0;
  bool up = true;
  for (int s = 0; s < segments && up; ++s) {
    for (int i = 0; i <= tiles && up; ++i) {
      if (s > 0 && i == (early < tiles ? early : tiles)) {
        if (waits++ == stop) up = false;
        else queries.add();            // (its predecessor was read, so it has landed)
      }
      if (up && i < tiles && waits++ == stop) up = false;
    }
    if (up) ++whole;
  }
  *reached = !up;
  Barrier b;
  b.landed = queries.issued - (landed ? 0 : 1);
  auto missed = [&](bool any, uint32_t parity) { return !landed && (!any || b.returns_at_once(parity)); };
  return {missed(queries.any(), queries.last_parity()), missed(whole > 0, (uint32_t)(whole - 1) & 1u),
          landed && !b.returns_at_once(queries.last_parity())};
}

int main() {
  int count = 0, segments = 0, nothing = 0, walks = 0;
  for (int segs = 1; segs <= 5; ++segs)
    for (int tiles = 1; tiles <= 6; ++tiles)
      for (int early = 1; early <= 4; ++early)
        for (int landed = 0; landed < 2; ++landed)
          for (int stop = 0;; ++stop) {
            bool reached = false;
            const Outcome o = walk(segs, tiles, early, stop, landed, &reached);
            if (!reached) break;
            ++walks;
            count += o.left_count;
            segments += o.left_segments;
            nothing += o.waits_for_nothing;
          }
  const bd::CopyCount none{0};
  std::printf("%d %d %d %d %d\n", walks, count, segments, nothing, none.any() ? 1 : 0);
  return 0;
}
