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
