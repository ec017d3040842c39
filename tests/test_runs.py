"""Runs of rows whose weight gradients are summed apart (csrc/runs.cuh), on the host: subgraphs of any length, no tensor is made."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "runs.cuh"
// runs <SMs> <most rows of a run, 0: no limit> <rows of subgraph 0> ..; prints the longest run, the runs and the slots
int main(int argc, char** argv) {
  const int S = argc - 3;
  std::vector<int32_t> ptr(S + 1, 0);
  for (int s = 0; s < S; ++s) ptr[s + 1] = ptr[s] + atoi(argv[3 + s]);
  int64_t rows = run_rows(ptr[S], atoi(argv[1]));
  const int64_t most = atoll(argv[2]);
  if (most && rows > most) rows = most;
  HostRuns all, some;
  cut_runs(ptr, S, rows, nullptr, all);
  int32_t at = 0, longest = 0, slot = 0;
  size_t multi = 0, k = 0;
  for (int s = 0; s < S; ++s) {
    const int32_t first = slot;
    int32_t pieces = 0;
    do {                                                 // a subgraph without rows has one run of none
      if (k >= all.wb.size() || all.wb[k] != at || all.we[k] < at || all.we[k] > ptr[s + 1]) return printf("run %zu\n", k), 1;
      if (all.we[k] - at > longest) longest = all.we[k] - at;
      const bool whole = at == ptr[s] && all.we[k] == ptr[s + 1];
      if (all.wsl[k] != (whole ? -(s + 1) : slot)) return printf("slot of run %zu\n", k), 1;
      if (!whole) ++slot, ++pieces;
      at = all.we[k++];
    } while (at < ptr[s + 1]);
    if (!pieces) continue;
    if (multi >= all.mp.size() || all.mp[multi] != s || all.mf[multi] != first || all.mc[multi] != pieces) return printf("subgraph %d\n", s), 1;
    ++multi;
  }
  if (k != all.wb.size() || k != all.we.size() || k != all.wsl.size() || multi != all.mp.size() || all.n_wg_slots != slot) return printf("ends\n"), 1;
  // a choice of subgraphs keeps runs and slots of the ones that are chosen
  std::vector<uint8_t> on(S);
  for (int s = 0; s < S; ++s) on[s] = s % 2;
  cut_runs(ptr, S, rows, on.data(), some);
  size_t j = 0;
  for (size_t i = 0; i < all.wb.size(); ++i) {
    bool chosen = false;
    for (int s = 1; s < S; s += 2) chosen |= all.wsl[i] == -(s + 1) || (all.wsl[i] >= 0 && all.wb[i] >= ptr[s] && all.wb[i] < ptr[s + 1]);
    if (!chosen) continue;
    if (j >= some.wb.size() || some.wb[j] != all.wb[i] || some.we[j] != all.we[i] || some.wsl[j] != all.wsl[i]) return printf("choice %zu\n", i), 1;
    ++j;
  }
  if (j != some.wb.size() || some.n_wg_slots != all.n_wg_slots) return printf("choice ends\n"), 1;
  printf("%d %zu %d\n", longest, all.wb.size(), slot);
  return 0;
}
"""


@pytest.fixture(scope="module")
def runs(tmp_path_factory):
    at = tmp_path_factory.mktemp("runs")
    (at / "runs.cpp").write_text(PROGRAM)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2511_09261_b200", "csrc"), str(at / "runs.cpp"), "-o", str(at / "runs")])

    def call(sizes, most=65536, sms=148):
        r = subprocess.run([str(at / "runs"), str(sms), str(most), *map(str, sizes)], capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stdout
        return tuple(map(int, r.stdout.split()))
    return call


@pytest.mark.parametrize("sizes", [[1], [0, 5, 0], [2048, 2049, 4096, 0], [1000] * 50, [1_130_000], [38_797_312], [40_000_000, 3, 0, 70_000],
                                   [100_000_000, 65_536, 65_537], [2_147_483_390]])
@pytest.mark.parametrize("most", [0, 65536])
def test_every_row_in_one_run_and_every_slot_once(runs, sizes, most):
    longest, count, slots = runs(sizes, most)
    assert not most or longest <= most
    # what the load reserves for them: runs are no shorter than 2,048 rows, and 65,536 long where the limit cuts them
    assert count <= len(sizes) + sum(sizes) // (65536 if most and sum(sizes) > 4 * 148 * 65536 else 2048)


def test_long_subgraphs_would_have_longer_runs_without_the_limit(runs):
    """100 M rows on 148 SMs: 592 runs of 168,960 rows, whose sums the tensor core would cut off 10,560 times."""
    assert runs([100_000_000], 0)[0] == 168_960 and runs([100_000_000])[0] == 65_536


def test_shorter_graphs_keep_their_runs(runs):
    for sizes in ([1_130_000], [2_500_000, 10_000], [20_000_000, 18_000_000]):
        assert runs(sizes, 0) == runs(sizes)
