"""How the paged decode step's work reaches its CTAs, on the host: every tile is taken once, whatever order CTAs start in and runs are
handed out in."""
import os
import subprocess

import pytest

import paper_2510_25600_b200

CSRC = os.path.join(os.path.dirname(paper_2510_25600_b200.__file__), "csrc")
# CTAs take runs as the kernel's do: the one that they start with (or, if that has no tiles, one that next_run finds), then what they ask
# for, until one without tiles or none comes; after one without tiles, what next_run finds.  `order`: 0 as numbered, 1 backwards, 2 at random.
# `discard`: after a run without tiles the rest is thrown away unlooked at, which is right only in the order of their numbers.
MAIN = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "paged_runs.cuh"
using namespace purekv;
int main(int, char** v) {
  const int64_t all = atoll(v[1]);
  const int32_t v_heads = atoi(v[2]), at_once = atoi(v[3]), n_long = atoi(v[4]), n_short = atoi(v[5]);
  const int order = atoi(v[6]), discard = atoi(v[7]);
  const RunCuts cuts = RunCuts::of(all, v_heads, at_once, n_long, n_short);
  const int32_t runs = v_heads * (n_long + n_short);
  int64_t at = 0;
  for (int32_t j = 0; j < n_long + n_short; ++j) {  // the pieces lie one after the other, and hold their tiles
    if (cuts.starts_at(j) != at || cuts.tiles(j * v_heads) < 0) return printf("piece %d", j), 0;
    for (const int64_t end = at + cuts.tiles(j * v_heads); at < end; ++at)
      if (cuts.piece_with(at) != j) return printf("tile %lld", (long long)at), 0;
  }
  if (at != all) return printf("%lld tiles of %lld", (long long)at, (long long)all), 0;
  std::vector<int32_t> pending, taken(runs), told(runs);
  for (int32_t b = 0; b < runs; ++b) {
    if ((b < cuts.first_empty()) != (cuts.tiles(b) > 0)) return printf("tiles of run %d", b), 0;
    pending.push_back(b);
  }
  uint32_t x = 12345;
  auto any = [&] {
    if (pending.empty()) return -1;
    x = x * 1664525u + 1013904223u;
    const size_t i = order == 0 ? 0 : order == 1 ? pending.size() - 1 : (x >> 8) % pending.size();
    const int32_t b = pending[i];
    pending.erase(pending.begin() + i);
    ++told[b];
    return b;
  };
  auto find = [&] {
    if (discard) { while (any() >= 0) {} return -1; }
    return next_run(cuts, [] {}, any, [](int32_t) {});
  };
  struct Cta { int32_t run; bool more, empty; };
  std::vector<Cta> ctas;
  while (!pending.empty() || !ctas.empty()) {
    while ((int32_t)ctas.size() < at_once && !pending.empty()) {
      int32_t b = any();
      if (cuts.tiles(b) == 0) b = find();
      if (b >= 0) ctas.push_back({b, true, false});
    }
    if (ctas.empty()) break;
    x = x * 1664525u + 1013904223u;
    const size_t i = (x >> 8) % ctas.size();  // a CTA that comes to the end of its run
    Cta& c = ctas[i];
    ++taken[c.run];
    c.run = -1;
    if (c.more) {
      const int32_t b = any();
      if (b >= 0 && cuts.tiles(b) > 0) c.run = b;
      else c.more = false, c.empty = b >= 0;
    }
    if (c.run < 0 && c.empty && (c.run = find()) >= 0) c.more = true, c.empty = false;
    if (c.run < 0) ctas.erase(ctas.begin() + i);
  }
  for (int32_t b = 0; b < runs; ++b)
    if (told[b] != 1 || taken[b] != (cuts.tiles(b) > 0)) return printf("run %d", b), 0;
  printf("ok");
}
"""
# tiles of a head, heads, CTAs at work, long and short runs of a head
WORK = [(0, 4, 296, 74, 222), (1, 4, 296, 74, 222), (5, 8, 444, 55, 167), (590, 4, 296, 74, 222), (593, 4, 296, 74, 222), (700, 4, 296, 74, 222), (700, 4, 296, 74, 1),
        (4001, 4, 296, 74, 222), (16000, 1, 296, 296, 888), (3, 400, 296, 1, 3), (50, 400, 296, 1, 3), (250, 3, 12, 4, 12)]


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("runs")
    (d / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=address,undefined", "-I", CSRC, str(d / "main.cpp"), "-o", str(d / "main")], check=True)
    return lambda *a: subprocess.check_output([str(d / "main"), *map(str, a)]).decode().strip()


@pytest.mark.parametrize("order", [0, 1, 2])
@pytest.mark.parametrize("work", WORK)
def test_every_tile_is_taken_once(program, work, order):
    assert program(*work, order, 0) == "ok"


def test_runs_thrown_away_unlooked_at_are_missed(program):
    work = (700, 4, 296, 74, 222)   # short runs with tiles, and many without
    assert program(*work, 0, 1) == "ok"
    assert program(*work, 1, 1).startswith("run") and program(*work, 2, 1).startswith("run")
