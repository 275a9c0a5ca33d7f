// How the paged decode step cuts its work into runs, and which of them a CTA takes.  Plain C++, so that it can be checked on a host.
#pragma once
#include <cstdint>

#include "paged.cuh"

namespace purekv {

// The tiles of a head, over all requests one after the other, are cut into n_long long runs and n_short short ones, each head's alike; run b
// is the (b / v_heads)th of head b % v_heads, the long ones first.  Three quarters of a CTA's share make a long run; the rest is cut
// into short ones of four tiles at least, which go to whichever CTA asks next.  Up to eight tiles per CTA all go into long runs: short
// ones would be as long as those.  The last runs may have no tiles.
struct RunCuts {
  static constexpr int kShortest = 4, kFew = 8;
  int64_t all, long_tiles, short_tiles;  // of a head; of a long and of a short run
  int32_t v_heads, n_long, n_short;

  static PK_HD RunCuts of(int64_t all, int32_t v_heads, int32_t at_once, int32_t n_long, int32_t n_short) {
    int64_t lt;
    if (all * v_heads <= (int64_t)kFew * at_once) {
      lt = (all + n_long - 1) / n_long;
    } else {
      lt = all * v_heads * 3 / 4 / at_once;
      lt = lt < 1 ? 1 : lt < all ? lt : all;
    }
    const int64_t rest = all - n_long * lt, st = rest > 0 ? (rest + n_short - 1) / n_short : 0;
    return {all, lt, st > kShortest ? st : kShortest, v_heads, n_long, n_short};
  }
  PK_HD int32_t piece_of(int32_t run) const { return run / v_heads; }
  PK_HD int64_t starts_at(int32_t piece) const {
    const int64_t t = piece <= n_long ? piece * long_tiles : n_long * long_tiles + (piece - n_long) * short_tiles;
    return t < all ? t : all;
  }
  // the runs before this one have tiles, it and those behind it none
  PK_HD int32_t first_empty() const { return all > 0 ? (piece_with(all - 1) + 1) * v_heads : 0; }
  PK_HD int64_t tiles(int32_t run) const { return starts_at(piece_of(run) + 1) - starts_at(piece_of(run)); }
  // the piece of a head that has tile `tile`
  PK_HD int32_t piece_with(int64_t tile) const {
    return (int32_t)(tile < n_long * long_tiles ? tile / long_tiles : n_long + (tile - n_long * long_tiles) / short_tiles);
  }
};

// Takes runs that no CTA has started, in whatever order they come, until one has tiles; -1 once there are none.  `ask` asks for one,
// `answer` returns it, or -1, and `taken` is told of each.
template <typename Ask, typename Answer, typename Taken>
PK_HD int32_t next_run(const RunCuts& cuts, Ask ask, Answer answer, Taken taken) {
  ask();
  const int32_t empty = cuts.first_empty();  // (while the answer is under way)
  for (int32_t b; (b = answer()) >= 0; ask()) {
    taken(b);
    if (b < empty) return b;
  }
  return -1;
}

}  // namespace purekv
