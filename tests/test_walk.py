"""How the blocks of a grid share a long array (csrc/walk.cuh), run on the host: no array of these lengths is made."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "walk.cuh"
// every element of [0, count) exactly once over the blocks, in no more pieces than there are
int main(int argc, char** argv) {
  const int64_t count = atoll(argv[1]), blocks = atoll(argv[2]), piece = atoll(argv[3]);
  int64_t seen = 0, pieces = 0;
  const int64_t most = (count + piece - 1) / piece;
  for (int64_t b = 0; b < blocks; ++b) {
    int64_t expect = b * piece;
    for (PieceWalk w(count, b, blocks, piece); w.more(); w.next()) {
      if (++pieces > most) { printf("block %lld goes on for ever\n", (long long)b); return 1; }
      if (w.at != expect) { printf("block %lld at %lld, not %lld\n", (long long)b, (long long)w.at, (long long)expect); return 1; }
      seen += count - w.at < piece ? count - w.at : piece;
      expect += blocks * piece;
    }
  }
  if (seen != count) { printf("%lld of %lld elements\n", (long long)seen, (long long)count); return 1; }
  return 0;
}
"""


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    at = tmp_path_factory.mktemp("walk")
    (at / "walk.cpp").write_text(PROGRAM)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2511_09261_b200", "csrc"),
                           str(at / "walk.cpp"), "-o", str(at / "walk")])
    return str(at / "walk")


# 128 x (2^24 - 128): the largest matrix of an orthogonalised update; 32,896 x 65,280 and 32,640 x 65,792: large and nearly square
@pytest.mark.parametrize("count", [128 * (2 ** 24 - 128), 32896 * 65280, 32640 * 65792, 2 ** 31 - 262144, 2 ** 31 - 262145,
                                   0, 1, 1023, 1024, 1025, 262143, 262144, 262145, 1537000])
@pytest.mark.parametrize("blocks", [256, 1, 17])
def test_every_element_once(walk, count, blocks):
    r = subprocess.run([walk, str(count), str(blocks), "1024"], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
