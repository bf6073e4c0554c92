"""Where the wide attention kernels' loop leaves out its conditions (csrc/wide_schedule.h, the kernels' own
functions), on a model of the copies of every kind of wave, built for the host."""

import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_00814_amd", "csrc")

# A copy that is asked for is (K or V, tile); what a barrier leaves on its way are the youngest.  window: tiles whose
# addresses are taken together; first: how many the item's first window holds.
PROGRAM = r"""
#define __host__
#define __device__
#define __forceinline__ inline
#include <stdio.h>
#include <algorithm>
#include <set>
#include <utility>
#include <vector>
#include "wide_schedule.h"
enum Wave { kA, kB, kIdle };
struct Item {
  int tiles, seen, full, first, window;
  bool guard;  // false: without the rule for items of two and three tiles
  std::vector<std::pair<char, int>> asked, missing;
  int edge, wrong = 0, plain = 0;
  void put(char kind, int n, bool careful) {
    if (careful && n >= tiles) return;  // the plain body asks for the last tile again
    const int at = std::min(n, tiles - 1);
    if (kind == 'K' && careful)
      while (at >= edge) edge += window;
    if (at >= edge || (!careful && at >= full)) ++wrong;  // no address, or keys that do not exist
    asked.push_back({kind, n});
  }
  void barrier(int m, int left) {
    const size_t here = asked.size() - std::min<size_t>(left, asked.size());
    for (auto x : {std::pair<char, int>{'K', m}, {'V', m - 1}})
      if (x.second >= 0 && x.second < tiles &&
          std::find(asked.begin(), asked.begin() + here, x) == asked.begin() + here)
        missing.push_back(x);
  }
  void careful(int m) { barrier(m, ooo::copies_left(m, tiles)); }
  int end() const {
    if (guard) return ooo::plain_end(tiles, seen, full, edge);
    const int care = std::min(full, edge), e = std::min(seen, tiles);
    return care < tiles ? std::min(e, care - 5) : e;
  }
  void run(Wave w) {
    edge = first;
    put('K', 0, true), put('K', 1, true), put('V', 0, true), put('K', 2, true);
    careful(0);
    if (w == kIdle) {
      for (int m = 1; m <= tiles + 1; ++m) put('V', m, true), put('K', m + 2, true), careful(m);
      return;
    }
    put('V', 1, true), put('K', 3, true);
    careful(1);
    if (w == kB) put('V', 2, true);
    put('K', 4, true);
    const auto tile = [&](int n, bool p) {
      plain += p;
      const auto turn = [&] { p ? barrier(n + 2, 2) : careful(n + 2); };
      if (w == kB) turn();
      put('V', n + 2 + (w == kB), !p);
      if (w == kA) turn();
      put('K', n + 5, !p);
    };
    for (int n = 0; n < tiles; ++n) {
      const int e = end();
      for (; n < e; ++n) tile(n, true);
      if (n < tiles) tile(n, false);
    }
  }
};
int main() {
  long long items = 0, missing = 0, wrong = 0;
  std::set<int> without;
  std::set<int> runs;  // tiles of items that go through the plain body whole
  for (int window : {16, 64, 128})
    for (int first : {window, window - 1, window - 3})
      for (int tiles = 1; tiles <= 2 * window + 9 && tiles <= 160; ++tiles)
        for (int full : {tiles, tiles - 1})
          for (int seen = 0; seen <= full; seen += tiles < 40 ? 1 : 1 + tiles / 13)
            for (Wave w : {kA, kB, kIdle})
              for (bool guard : {true, false}) {
                Item x{tiles, seen, full, first, window, guard};
                x.run(w);
                if (!guard) {
                  if (!x.missing.empty()) without.insert(tiles);
                  for (auto& m : x.missing)
                    if (m != std::pair<char, int>{'V', 1}) ++wrong;
                  continue;
                }
                ++items;
                missing += x.missing.size();
                wrong += x.wrong;
                if (w == kIdle) wrong += x.plain;
                else if (x.plain == tiles) runs.insert(tiles);
              }
  printf("%lld %lld %lld\n", items, missing, wrong);
  for (int t : without) printf("%d ", t);
  printf("\n");
  for (int t = 1; t <= 12; ++t)
    if (runs.count(t)) printf("%d ", t);
  printf("\n");
}
"""


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    d = tmp_path_factory.mktemp("wide")
    src, exe = d / "wide.cpp", d / "wide"
    src.write_text(PROGRAM)
    try:
        subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", f"-I{CSRC}", str(src), "-o", str(exe)], check=True)
    except FileNotFoundError:
        pytest.skip("no host compiler")
    lines = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines()
    return [[int(x) for x in line.split()] for line in lines]


def test_every_copy_has_landed_and_exists(model):
    items, missing, wrong = model[0]
    assert items > 30_000 and missing == 0 and wrong == 0


def test_two_and_three_tiles_need_the_rule_and_no_others_have_it(model):
    assert model[1] == [2, 3]
    assert model[2] == [1] + list(range(4, 13))
