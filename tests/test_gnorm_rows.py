"""How group norm deals rows and columns to chunks and threads (csrc/gnorm_rows.cuh), on the host: the header is
compiled into a small program and run over every width."""
import os
import shutil
import subprocess


ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_23169_gb300", "csrc")

CHUNKS = r"""
#include <cstdio>
#include <cstring>
#include "gnorm_rows.cuh"
using namespace ut;

// every row and column of a full chunk belongs to exactly one thread and step
template <int kThreads, int kPer>
int check(int widest) {
  static unsigned char seen[kThreads * kPer * kThreads];
  int wrong = 0;
  for (int cv = 1; cv <= widest; ++cv) {
    const Chunks<kThreads, kPer> ck(cv);
    int cols = 0;
    for (int slab = 0; slab < ck.slabs; ++slab) {
      const int sc = ck.slab_cols(slab);
      cols += sc;
      memset(seen, 0, sizeof(seen));
      for (int t = 0; t < kThreads; ++t) {
        const Layout<kThreads, kPer> L(ck, slab, t);
        if (!L.on) continue;
        for (int k = 0; k < kPer; ++k) {
          const int row = L.lane + k * L.lanes, col = L.col - slab * kThreads;
          if (row < 0 || row >= ck.rows || col < 0 || col >= sc || L.cols != sc || seen[row * kThreads + col]++) ++wrong;
        }
      }
      for (int row = 0; row < ck.rows; ++row)
        for (int col = 0; col < sc; ++col) wrong += !seen[row * kThreads + col];
    }
    wrong += cols != cv || ck.rows < 1;
  }
  return wrong;
}

int main() {  // up to 8,192 channels: 1,024 16-byte columns in bf16, 2,048 in fp32
  printf("%d %d\n", check<kFwdThreads, kFwdPer>(2048), check<kBwdThreads, kBwdPer>(2048));
}
"""


def run(source: str, where) -> str:
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    src, exe = os.path.join(where, "host.cu"), os.path.join(where, "host")
    with open(src, "w") as f:
        f.write(source)
    subprocess.run([nvcc, "-O1", "-std=c++17", "-arch=sm_103a", "-I", CSRC, src, "-o", exe], check=True)
    return subprocess.run([exe], check=True, capture_output=True, text=True).stdout


def test_threads_cover_a_chunk_once_in_every_slab(tmp_path):
    assert run(CHUNKS, str(tmp_path)).split() == ["0", "0"]


PIECES = r"""
#include <algorithm>
#include <cstdio>
#include <random>
#include <tuple>
#include <vector>
#include "gnorm_rows.cuh"
using namespace ut;

int main() {
  std::mt19937 g(1);
  auto below = [&](int n) { return (int)(g() % (unsigned)n); };
  int unequal = 0, outside = 0, uncovered = 0, shared = 0;
  for (int t = 0; t < 40000; ++t) {
    const int n = below(90), B = 1 + below(7), blocks = 1 + below(5);
    const bool right = t & 1;
    std::vector<int32_t> cu(B + 1);
    for (auto& c : cu) c = below(8) ? below(n + 20) - 10 : (int)g();
    if (right) {
      for (auto& c : cu) c = std::max(0, std::min(n, c));
      cu[0] = 0;
      cu[B] = n;
      std::sort(cu.begin(), cu.end());
    }
    GnormParams p{};
    p.n = n;
    p.B = B;
    p.cu = cu.data();
    const Shares sh(p, blocks);
    std::vector<int> seen(n, 0), slot(blocks + B, 0);
    for (int b = 0; b < blocks; ++b) {
      const Pieces pieces(p, sh.first(b), sh.first(b + 1));
      std::vector<std::tuple<int, int, int>> x, y;
      pieces.forward(p, [&](int s, int lo, int hi) { x.emplace_back(s, lo, hi); });
      pieces.backward(p, [&](int s, int lo, int hi) { y.emplace_back(s, lo, hi); });
      std::reverse(y.begin(), y.end());
      unequal += x != y;
      for (auto [s, lo, hi] : x) {
        outside += lo < 0 || hi > n || lo >= hi || s < 0 || s >= B || sh.owner(lo) < 0 || sh.owner(hi - 1) >= blocks;
        if (!right) continue;
        shared += slot[b + s]++ > 0 || sh.owner(lo) != b || sh.owner(hi - 1) != b || lo < cu[s] || hi > cu[s + 1];
        for (int r = lo; r < hi; ++r) ++seen[r];
      }
    }
    if (right)
      for (int c : seen) uncovered += c != 1;
  }
  printf("%d %d %d %d\n", unequal, outside, uncovered, shared);
}
"""


def test_both_passes_list_the_same_pieces_whatever_the_prefix(tmp_path):
    """Right prefixes: every row in one piece, every piece with a place of its own for its sums.  Wrong ones: both passes
    still go over the same pieces, all of them inside the rows."""
    assert run(PIECES, str(tmp_path)).split() == ["0", "0", "0", "0"]
