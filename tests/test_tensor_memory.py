"""Clusters of different streams never wait for each other's tensor memory: CTAs that fit an SM by the shared memory they ask for
fit by their columns."""
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1805_07941_b200", "csrc")

# Every mix of CTAs (columns a power of two from 32, whatever they need themselves) whose shared memory fits an SM.
PROGRAM = r"""
#include <initializer_list>
#include "tensor_memory.cuh"

static int most(int room, int least) {
  int best = 0;
  for (int columns = least; columns <= qc::kSmTmemColumns; columns *= 2) {
    const int bytes = static_cast<int>(qc::cluster_smem(0, columns) + qc::kCtaReservedBytes);
    if (bytes > room) continue;
    const int with = columns + most(room - bytes, columns);
    best = with > best ? with : best;
  }
  return best;
}

int main() {
  int wrong = most(static_cast<int>(qc::kSmSharedBytes), 32) > qc::kSmTmemColumns;
  for (int columns = 32; columns <= 512; columns *= 2)
    for (size_t needed : {0ul, 50344ul, 62632ul, 87208ul, 159894ul, 232448ul}) {
      const size_t asked = qc::cluster_smem(needed, columns);
      wrong += asked < needed || asked > 227 * 1024 || (asked > needed && needed >= qc::cluster_smem(0, columns));
    }
  return wrong;
}
"""


def test_what_fits_in_shared_memory_fits_in_tensor_memory(tmp_path):
    source, binary = tmp_path / "columns.cpp", tmp_path / "columns"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-x", "c++", "-I", CSRC, "-o", str(binary), str(source)], check=True)
    assert subprocess.run([str(binary)], timeout=120).returncode == 0


def test_every_cluster_is_launched_with_its_part_of_shared_memory():
    """One function sets the cluster attribute, and its caller names the columns; no kernel has cluster dimensions of its own."""
    for name in (n for n in os.listdir(CSRC) if n.endswith((".cu", ".cuh"))):
        text = open(os.path.join(CSRC, name)).read()
        assert text.count("cudaLaunchAttributeClusterDimension") == (name == "library.cuh"), name
        assert "__cluster_dims__" not in text, name
    text = open(os.path.join(CSRC, "library.cuh")).read()
    body = text[text.index("cudaError_t launch_clusters("):]
    assert "dynamicSmemBytes = cluster_smem(smem, columns)" in body[:body.index("cudaLaunchKernelEx")]


@pytest.mark.gpu
def test_the_numbers_are_this_devices():
    import torch
    p = torch.cuda.get_device_properties(0)
    assert p.shared_memory_per_multiprocessor == 228 * 1024 and p.shared_memory_per_block_optin == 227 * 1024


@pytest.mark.gpu
def test_products_ask_for_their_part():
    import torch
    from paper_1805_07941_b200 import binding
    forms = set()
    for T, N, K in [(1, 300, 700), (20, 640, 1024), (40, 512, 600), (60, 200, 4096), (100, 256, 2000), (128, 512, 4096), (384, 8192, 8192),
                    (1000, 4999, 512)]:
        wc, ws = binding.qmx_quantize(torch.randn((N, K), device="cuda"))
        xc, xs = binding.qmx_quantize(torch.randn((T, K), device="cuda"))
        lin = binding.QMXLinear(wc, ws, N, K, dtype=torch.float32)
        lin.run(xc, xs)
        assert lin.status() == 0
        form = {k: int(v) for k, v in re.findall(r"(\w+)=(\d+)(?= |$)", lin.describe())}
        if form["split"] > 1 or form["pair"]:
            assert (form["smem"] + 1024) * 512 >= form["columns"] * 228 * 1024, lin.describe()
        forms.add("pair" if form["pair"] else "split" if form["split"] > 1 else "one")
    assert {"pair", "split"} <= forms


@pytest.mark.gpu
def test_clusters_of_two_streams_at_once():
    """Products of pairs whose rows are anywhere, on one stream, beside products that share a contraction, on the other."""
    import torch
    from paper_1805_07941_b200 import binding
    gen = torch.Generator(device="cuda").manual_seed(5)
    runs = []
    for T, N, K in ((1000, 4999, 512), (20, 640, 1024), (60, 200, 4096)):
        wc, ws = binding.qmx_quantize(torch.randn((N, K), generator=gen, device="cuda"))
        x = binding.qmx_quantize(torch.randn((T, K), generator=gen, device="cuda"))
        lin = binding.QMXLinear(wc, ws, N, K, dtype=torch.float32)
        runs.append((lin, x, lin.run(*x)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    got = [[] for _ in runs]
    for _ in range(30):
        for (lin, x, _), stream, outs in zip(runs, streams, got):
            with torch.cuda.stream(stream):
                outs.append(lin.run(*x))
    torch.cuda.synchronize()
    for (lin, _, want), outs in zip(runs, got):
        assert lin.status() == 0 and all(torch.equal(y, want) for y in outs)
