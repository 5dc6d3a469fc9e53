"""Products whose waits give up at any point: after a few polls some roles of a kernel have finished what others no longer wait for.
The run ends, its status tells, a run that reports nothing is right, and so is the next one."""
import pytest

from paper_1805_07941_b200 import binding

pytestmark = pytest.mark.gpu

# one tile a CTA, contractions shared by a cluster, many tiles on single SMs, pairs with bulk stores of both kinds and without
CASES = [(20, 640, 512, "float32"), (100, 256, 300, "bfloat16"), (4, 256, 4096, "float32"), (60, 200, 4096, "float16"), (256, 256, 6000, "float32"),
         (40, 19000, 2500, "float32"), (300, 600, 1024, "float32"), (2000, 2048, 2048, "float32"), (2000, 2048, 2048, "bfloat16"),
         (2000, 2047, 2048, "float32"), (5000, 1100, 130, "bfloat16")]


@pytest.mark.parametrize("T,N,K,dtype", CASES)
def test_any_limit(T, N, K, dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(T + N + K)
    wc, ws = binding.qmx_quantize(torch.randn((N, K), generator=gen, device="cuda"))
    xc, xs = binding.qmx_quantize(torch.randn((T, K), generator=gen, device="cuda"))
    lin = binding.QMXLinear(wc, ws, N, K, dtype=getattr(torch, dtype))
    want = lin.run(xc, xs)
    assert lin.status() == 0
    y = torch.empty_like(want)
    for limit in (0, 1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 64, 128, 1024):
        for _ in range(3):
            lin.set_wait_limit(limit)
            lin.run(xc, xs, y)
            status = lin.status()
            assert status in (0, binding.ERR_TIMEOUT)
            assert limit > 0 or status == binding.ERR_TIMEOUT
            if status == 0:
                assert torch.equal(y, want), limit
        lin.set_wait_limit(1 << 22)
        lin.run(xc, xs, y)
        assert lin.status() == 0 and torch.equal(y, want), limit
