"""The checked build's test of an access by address, and that the codec, norm and cache kernels ask it: their accesses are pointers
moved by strides, whose rows alone say nothing about where they end."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1805_07941_b200", "csrc")

PROGRAM = r"""
#include "extent.cuh"

int main() {
  static float t[100];
  const qc::Extent e = qc::Extent::of(t + 10, 50);
  const char* lo = reinterpret_cast<const char*>(t + 10);
  int wrong = 0;
  for (int from = -40; from < 240; ++from)
    for (int count = 1; count <= 32; ++count)
      wrong += e.has(lo + from, count) != (from >= 0 && from + count <= 200);
  wrong += e.has(nullptr, 4) || !e.has(lo, 200) || e.has(lo, 201) || e.has(lo + 200, 1) || qc::Extent::of(t, 0).has(t, 1);
  return wrong;
}
"""


def test_all_bytes_of_an_access_are_the_tensors(tmp_path):
    source, binary = tmp_path / "extent.cpp", tmp_path / "extent"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-x", "c++", "-I", CSRC, "-o", str(binary), str(source)], check=True)
    assert subprocess.run([str(binary)], timeout=60).returncode == 0


def function(text, name):
    """The text of a function or kernel from its name to the brace that closes it."""
    start = re.search(r"\b%s\(" % name, text).start()
    depth = 0
    for i in range(text.index("{", start), len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if not depth:
            return text[start:i]


def test_what_moves_values_and_codes_asks():
    files = {n: open(os.path.join(CSRC, n)).read() for n in ("mx_format.cuh", "kernels_mx.cuh", "kernels_norm.cuh", "kernels_cache.cuh")}
    asked = {"mx_format.cuh": {"store_bytes": 3, "load_bytes": 3, "load_dealt": 2, "store_dealt": 2, "group_load": 1, "group_store": 1,
                               "mx_store_codes": 1, "store_scale_word": 1},
             "kernels_mx.cuh": {"mx_dequantize_kernel": 1}, "kernels_norm.cuh": {"norm_scale": 1, "norm_store_i8": 1},
             "kernels_cache.cuh": {"cache_write_kernel": 3, "cache_read_kernel": 4}}
    for name, functions in asked.items():
        for f, count in functions.items():
            assert function(files[name], f).count("QC_AT(") == count, f
    assert "QC_IN(row, cache_rows(a))" in function(files["kernels_cache.cuh"], "cache_slot")
    # no test that the condition before it implies
    for text in files.values():
        assert "QC_IN(at.row, a.rows) ?" not in text and "QC_IN(slot, a.num_slots)" not in text
