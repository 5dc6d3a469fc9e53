"""Which head a lane of the cache kernels takes: every one once, none outside the list, up to the largest call that is accepted."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1805_07941_b200", "csrc")

# The kernels' walk: slots are looked up for the first two rounds, then two rounds ahead of the one that is worked on.
PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "cache_items.cuh"

static long long wrong = 0;

template <typename Visit>
void walk(int items, int G, int blocks, int from_base, Visit visit) {
  const int per_warp = 32 / G, per_block = 8 * per_warp, step = blocks * per_block;
  for (int block = 0; block < blocks; ++block)
    for (int warp = 0; warp < 8; ++warp) {
      const int first = block * per_block + warp * per_warp;
      for (int j = 0; j < 2; ++j)
        for (int l = 0; l < 32; ++l) visit(qc::cache_unit(first + j * step, qc::cache_mine(l, G)), l, G);
      // (of a long list the last rounds)
      int base = first + static_cast<int>(static_cast<long long>(from_base > first ? from_base - first : 0) / (2 * step) * (2 * step));
      for (; base < items; base += 2 * step)
        for (int j = 0; j < 2; ++j)
          for (int l = 0; l < 32; ++l) visit(qc::cache_unit(base + (2 + j) * step, qc::cache_mine(l, G)), l, G);
    }
}

int main() {
  for (int G = 1; G <= 32; ++G) {
    for (int items : {1, 2, 31, 32, 33, 1000, 4097}) {
      std::vector<int> seen(items, 0);
      walk(items, G, 3, 0, [&](unsigned int u, int l, int g) {
        const bool has = qc::cache_has(u, items);
        wrong += has && (l >= 32 / g * g || u >= static_cast<unsigned int>(items));
        if (has && l % g == 0) ++seen[u];
      });
      for (int n : seen) wrong += n != 1;
    }
    if (G == 3 || G == 5 || G == 7 || G == 32)
      for (int items : {1 << 30, (1 << 30) - 142000}) {
        auto check = [&](unsigned int u, int l, int g) {
          wrong += qc::cache_has(u, items) && (l >= 32 / g * g || u >= static_cast<unsigned int>(items));
        };
        walk(items, G, 148 * 8, items - 400000, check);
      }
  }
  std::printf("%lld\n", wrong);
  return wrong != 0;
}
"""


def test_every_head_once_and_none_outside_the_list(tmp_path):
    source, binary = tmp_path / "items.cpp", tmp_path / "items"
    source.write_text(PROGRAM)
    # (signed overflow, if there were any, ends the program)
    subprocess.run(["g++", "-std=c++17", "-O1", "-ftrapv", "-I", CSRC, "-o", str(binary), str(source)], check=True)
    r = subprocess.run([str(binary)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
