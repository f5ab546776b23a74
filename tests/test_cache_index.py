"""Index arithmetic of the 8-bit context cache's kernels (csrc/cache_index.h),
compiled for the host."""
import os
import shutil
import subprocess

import pytest

from paper_2609_34170_gb300.build import CSRC

HEAD = "#include <cstdio>\n#include <cstdint>\n#include <cstdlib>\n#include \"cache_index.h\"\nusing namespace ravel;\n"


@pytest.fixture
def run(tmp_path):
    """Compiles a program against the header and returns its output's lines."""
    def go(source, *args):
        if not shutil.which("g++"):
            pytest.skip("needs g++")
        (tmp_path / "main.cpp").write_text(HEAD + source)
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=signed-integer-overflow",
                        "-fno-sanitize-recover=all", "-I", CSRC, str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")],
                       check=True)
        out = subprocess.run([str(tmp_path / "main"), *map(str, args)], capture_output=True, text=True)
        assert out.returncode == 0, out.stdout + out.stderr
        return out.stdout.split()
    return go


# A warp reads `loads` units through a ring; the wait for unit `at` runs out.  Barriers as the
# hardware has them: a wait for a parity ends once the current phase has the other one.
RING = r"""
struct Bar {
  unsigned completed = 0;
  int armed = 0;   // loads into the current phase
  bool passes(unsigned parity) const { return (completed & 1u) != parity; }
};
#define NEED(x) do { if (!(x)) { printf("slots %d loads %d at %d landed %x: %s\n", slots, loads, at, landed, #x); return 1; } } while (0)
int main() {
  int cases = 0;
  for (int slots = 1; slots <= 8; ++slots)
    for (int loads = 1; loads <= 3 * slots; ++loads)
      for (int at = 0; at < loads; ++at)
        for (unsigned landed = 0; landed < 1u << slots; ++landed) {   // of those on their way
          Bar bar[8];
          int issued = 0;
          auto issue = [&](int k) { ++bar[k % slots].armed; ++issued; };
          auto land = [&](int k) { --bar[k % slots].armed; ++bar[k % slots].completed; };
          for (int k = 0; k < slots && k < loads; ++k) issue(k);
          for (int k = 0; k < at; ++k) {
            land(k);
            NEED(bar[k % slots].passes(load_parity(k, slots)));
            if (k + slots < loads) issue(k + slots);
          }
          const LoadsLeft left = loads_left(at, loads, slots);
          NEED(left.first == at && left.end == issued && left.end - left.first <= slots);
          for (int k = left.first; k < left.end; ++k) NEED(bar[k % slots].armed == 1);
          for (int k = left.first; k < left.end; ++k)
            if (landed >> (k - left.first) & 1u) land(k);
          // a wait passes exactly where the load has landed, and all of them once all have
          for (int k = left.first; k < left.end; ++k)
            NEED(bar[k % slots].passes(load_parity(k, slots)) == (landed >> (k - left.first) & 1u));
          for (int k = left.first; k < left.end; ++k)
            if (!(landed >> (k - left.first) & 1u)) land(k);
          for (int k = left.first; k < left.end; ++k) NEED(bar[k % slots].passes(load_parity(k, slots)));
          ++cases;
        }
  printf("%d\n", cases);
  return 0;
}
"""


def test_loads_on_their_way_when_a_wait_runs_out(run):
    assert int(run(RING)[0]) > 10000


def test_the_kernel_for_few_rows_issues_nothing_after_a_wait_ran_out():
    """A failed wait leaves the unit loop, after the loads that are left, in front of the next load's issue."""
    with open(os.path.join(CSRC, "cache_attn.cu")) as f:
        body = f.read().split("for (; u < u1; u += RW)")[1]
    wait, issue = body.index("if (!wait_phase(&arrived[warp][slot], phase))"), body.index("fetch(u + RW * D, slot)")
    drain = body.index("loads_left((u - u0 - warp) / RW")
    assert wait < drain < body.index("break;", drain) < issue and body.count("wait_phase(") == 1


# Against each row's own definition, in 64 bits.
ROWS = r"""
struct Case { int len, count, G, causal, window, sinks; };
int main() {
  const int big = 2147483647 - 65536 - 128, half = 1 << 30;
  const Case cases[] = {
      {300, 200, 8, 1, 0, 0}, {300, 300, 1, 1, 50, 4}, {300, 40, 20, 0, 0, 0}, {130, 130, 3, 1, 1, 0}, {130, 7, 64, 1, 130, 9},
      {half + 5, 300, 4, 1, half, 4}, {big, 200, 8, 1, big, 0}, {big, 129, 1, 1, big - 1, 4}, {big, 1, 1000, 1, 3, big},
      {big, 1, half, 1, big, 0}, {2 * (half / 2) + 77, 64, 16, 1, half / 2 + 9, 20}, {big, 300, 2, 0, 0, 0}};
  srand(1);
  long long checks = 0;
  for (const Case& c : cases) {
    const int p0 = c.len - c.count, end_row = c.count * c.G;
    for (int t = 0; t < 4000; ++t) {
      // tokens at the ends, at the window's edges and anywhere (up to the end of the last tile)
      const int near = rand() % 300 - 150;
      long long jj = t % 5 == 0 ? near : t % 5 == 1 ? (long long)c.len + near : t % 5 == 2 ? (long long)p0 + near
                   : t % 5 == 3 ? (long long)p0 - c.window + near : (long long)rand() % c.len;
      if (jj < 0 || jj >= (long long)c.len + 127) continue;
      const int j = (int)jj, first = end_row > 64 ? rand() % end_row / 64 * 64 : 0;
      const RowsThatSee got = rows_that_see(j, c.len, p0, c.G, end_row, c.causal, c.window, c.sinks, first);
      if (got.lo < -1 || got.lo > 64 || got.hi < 0 || got.hi > 64) return printf("range"), 1;
      for (int k = 0; k < 64; ++k) {
        const long long r = (long long)first + k, p = p0 + r / c.G;
        bool see = r < end_row && j < c.len;
        if (c.causal) see = see && j <= p && (c.window == 0 || j > p - c.window || j < c.sinks);
        if (see != (k >= got.lo && k < got.hi)) {
          printf("len %d count %d G %d window %d sinks %d: token %d row %lld\n", c.len, c.count, c.G, c.window, c.sinks, j, r);
          return 1;
        }
        ++checks;
      }
    }
  }
  printf("%lld\n", checks);
  return 0;
}
"""


def test_rows_that_see_a_token_at_any_position(run):
    assert int(run(ROWS)[0]) > 1000000


# What is prefetched is what is read: the longest run of the units that an item walks.
RUN = r"""
int main() {
  int cases = 0;
  for (int from = 0; from < 9; ++from)
    for (int sinks = 0; sinks <= from; ++sinks)
      for (int window = 0; window < 6; ++window)
        for (int t0 = 0; t0 < sinks + window; ++t0)
          for (int n = 1; t0 + n <= sinks + window; ++n) {
            int best = 0, begin = 0;
            for (int i = 0; i < n; ++i) {
              const int at = unit_place(t0 + i, sinks, from);
              if (at != (t0 + i < sinks ? t0 + i : from + t0 + i - sinks)) return printf("place"), 1;
              if (i == 0 || at != unit_place(t0 + i - 1, sinks, from) + 1) begin = i;
              best = i - begin + 1 > best ? i - begin + 1 : best;
            }
            const UnitRun run = longest_run(t0, n, sinks, from);
            bool found = false;
            for (int i = 0; i + run.units <= n; ++i) {
              bool same = true;
              for (int k = 0; k < run.units; ++k) same = same && unit_place(t0 + i + k, sinks, from) == run.at + k;
              found = found || same;
            }
            if (run.units != best || !found) {
              printf("sinks %d from %d t0 %d n %d: %d units at %d, longest %d\n", sinks, from, t0, n, run.units, run.at, best);
              return 1;
            }
            ++cases;
          }
  printf("%d\n", cases);
  return 0;
}
"""


def test_the_longest_run_of_an_items_units(run):
    assert int(run(RUN)[0]) > 500
