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
