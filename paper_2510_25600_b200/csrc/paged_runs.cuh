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
    const int64_t share = all * v_heads * 3 / 4 / at_once;
    const int64_t lt = all * v_heads <= (int64_t)kFew * at_once ? (all + n_long - 1) / n_long : share < 1 ? 1 : share < all ? share : all;
    const int64_t rest = all - n_long * lt, st = rest > 0 ? (rest + n_short - 1) / n_short : 0;
    return {all, lt, st > kShortest ? st : kShortest, v_heads, n_long, n_short};
  }
  PK_HD int32_t piece_of(int32_t run) const { return run / v_heads; }
  PK_HD int64_t starts_at(int32_t piece) const {
    const int64_t t = piece <= n_long ? piece * long_tiles : n_long * long_tiles + (piece - n_long) * short_tiles;
    return t < all ? t : all;
  }
  PK_HD int64_t tiles(int32_t run) const { return starts_at(piece_of(run) + 1) - starts_at(piece_of(run)); }
  // the piece of a head that has tile `tile`
  PK_HD int32_t piece_with(int64_t tile) const {
    return (int32_t)(tile < n_long * long_tiles ? tile / long_tiles : n_long + (tile - n_long * long_tiles) / short_tiles);
  }
};

// Takes runs that no CTA has started, in whatever order they come, until one has tiles; -1 once there are none.  `take` returns a run
// or -1, `taken` is told of each.
template <typename Take, typename Taken>
PK_HD int32_t next_run(const RunCuts& cuts, Take take, Taken taken) {
  int32_t b;
  while ((b = take()) >= 0) {
    taken(b);
    if (cuts.tiles(b) > 0) return b;
  }
  return -1;
}

}  // namespace purekv
