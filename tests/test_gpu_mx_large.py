"""Tensors whose element or byte offsets pass 32 bits: the last rows equal those of a call on them alone."""
import pytest

from paper_1805_07941_b200 import binding

pytestmark = pytest.mark.gpu

ROWS, C, TAIL = 4096 * 130, 8192, 256                         # 4.4 G values, codes of 2.2 and 4.4 GB


def big(seed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty((ROWS, C), dtype=torch.bfloat16, device="cuda")
    x[:TAIL].normal_(generator=gen)
    x[TAIL:-TAIL] = 1.0
    x[-TAIL:].normal_(generator=gen)
    return x


def test_codec():
    import torch
    x = big(1)
    codes, scales = binding.qmx_quantize(x)
    for part in (slice(0, TAIL), slice(ROWS - TAIL, ROWS)):
        c, s = binding.qmx_quantize(x[part])
        n = s.numel()
        assert torch.equal(codes[part], c) and torch.equal(scales[:n] if part.start == 0 else scales[-n:], s)
    want = binding.qmx_dequantize(c, s, C, dtype=torch.bfloat16)
    x.zero_()
    binding.qmx_dequantize(codes, scales, C, out=x)
    assert torch.equal(x[-TAIL:], want) and bool((x[TAIL:TAIL + 5] == 1.0).all())


def test_norm():
    import torch
    x, gain = big(2), torch.ones((C,), dtype=torch.bfloat16, device="cuda")
    for out in (binding.NORM_I8_ROWS, binding.NORM_MX):
        codes, scales = binding.qrmsnorm(x, gain, 1e-6, out=out)
        c, s = binding.qrmsnorm(x[-TAIL:], gain, 1e-6, out=out)
        assert torch.equal(codes[-TAIL:], c) and torch.equal(scales[-s.numel():], s)
        c, s = binding.qrmsnorm(x[:TAIL], gain, 1e-6, out=out)
        assert torch.equal(codes[:TAIL], c) and torch.equal(scales[:s.numel()], s)
        del codes, scales


def test_linear():
    import torch
    T, N, K = 128 * 1100, 16384, 96                           # y has 2.3 G values
    x, w = torch.randn((T, K), device="cuda"), torch.randn((N, K), device="cuda")
    xc, xs = binding.qmx_quantize(x)
    wc, ws = binding.qmx_quantize(w)
    lin = binding.QMXLinear(wc, ws, N, K, dtype=torch.float16)
    for ld in (N, N + 1):                                     # in bulk stores, and by the lanes
        flat = torch.zeros((T, ld), dtype=torch.float16, device="cuda")
        y = lin.run(xc, xs, flat[:, :N])
        assert lin.status() == 0
        tail = lin.run(xc[-TAIL:], xs[-xs.numel() * TAIL // T:])
        assert torch.equal(y[-TAIL:], tail) and not flat[:, N:].any()
        assert torch.equal(y[:TAIL], lin.run(xc[:TAIL], xs[:xs.numel() * TAIL // T]))
        del flat, y
