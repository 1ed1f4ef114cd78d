"""What the launches of the calls over continuations ask for (host only)."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_33503_b200", "csrc")

MAIN = r"""
#include "continuation_splits.cuh"
#include <cmath>
#include <cstdio>
#include <random>
using namespace relaxkv;
int main() {
  std::mt19937 r(1);
  const int most = 8192;
  for (int it = 0; it < 100000; ++it) {
    const int n = 1 + r() % 8, n_select = 1 + (int)std::pow(2.0, std::uniform_real_distribution<>(0, 14)(r));
    int cu[9] = {0};
    for (int b = 0; b < n; ++b) cu[b + 1] = cu[b] + (r() % 4 ? (int)std::pow(2.0, std::uniform_real_distribution<>(0, 15)(r)) : most - 2 + (int)(r() % 5));
    const int kept = kept_scores(cu, n, n_select, most);
    if (kept < 0 || kept > most) { std::printf("room for %d\n", kept); return 1; }
    for (int b = 0; b < n; ++b) {
      const int nb = cu[b + 1] - cu[b];
      // a context that competes keeps its scores exactly where they are few enough, whatever stands beside it
      if (nb > n_select && (nb <= kept) != (nb <= most)) { std::printf("%d blocks, room for %d of %d\n", nb, kept, most); return 1; }
    }
  }
  return 0;
}
"""


def test_every_context_has_room_for_the_scores_it_keeps(tmp_path):
    src, exe = tmp_path / "main.cpp", tmp_path / "main"
    src.write_text(MAIN)
    subprocess.check_call([os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-I", CSRC, str(src), "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_the_selection_looks_at_the_room_that_its_launch_gave_it():
    """The kernel decides by the launch's number, not by the constant that bounds it."""
    with open(os.path.join(CSRC, "block_select.cu")) as f:
        text = f.read()
    kernel = text[text.index("block_topk_kernel(const"):text.index("}  // namespace relaxkv")]
    assert "nb <= a.kept" in kernel and "kTopKept" not in kernel
