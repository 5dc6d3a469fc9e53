"""Residual addition + root-mean-square norm + conversion on the GPU against the oracle: codes and scale bytes equal those
of the definition (r and the products rounded to float32), and stay within half a step of the norm in float64."""
import numpy as np
import pytest

from oracle import mx_ref
from paper_1805_07941_b200 import binding

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]
EPS = 1e-6


def make(rng, rows, C, dtype):
    import torch
    tdt = getattr(torch, dtype)
    loud = np.where(rng.random(C) < 0.02, 20.0, 1.0)
    x = torch.from_numpy((rng.standard_normal((rows, C)) * loud).astype(np.float32)).to(tdt)
    res = torch.from_numpy((rng.standard_normal((rows, C)) * 2).astype(np.float32)).to(tdt)
    gain = torch.from_numpy((1 + 0.3 * rng.standard_normal(C)).astype(np.float32)).to(tdt)
    return x, res, gain


def as64(t):
    return t.double().numpy()


def check(out, codes, scales, h, gain, e=0, eps=EPS, layout=binding.MX_TILES):
    """h: the sum as kept (CPU tensor); codes, scales as the call gave them."""
    y, y64 = mx_ref.rmsnorm(as64(h), as64(gain), eps)
    rows, C = y.shape
    codes = codes.cpu().numpy()
    # y in float32 is off by the rounding of r and of two products: 3 * 2^-24 of it, and a rounding to nearest adds half a step
    slack = np.abs(y64) * 2.0**-22
    if out == binding.NORM_MX:
        want, s = mx_ref.mx_quantize(y)
        got = scales.cpu().numpy().reshape(-1)
        assert np.array_equal(got, mx_ref.to_tiles(s) if layout == binding.MX_TILES else s.reshape(-1))
        assert np.array_equal(codes, mx_ref.pack(want))
        step = np.repeat(np.ldexp(1.0, s.astype(int) - 127), 32, axis=1)[:, :C]      # the largest step is 2, between 4 and 6
        assert (np.abs(mx_ref.mx_values(want, s, C) - y64) <= step + slack).all()
        return
    if out == binding.NORM_I8_ROWS:
        ee = np.array([mx_ref.i8_exponent(r) for r in y])
        assert np.array_equal(scales.cpu().numpy(), (ee + 127).astype(np.uint8))
    else:
        assert scales is None
        ee = np.full(rows, e)
    want = np.stack([mx_ref.i8_codes(y[r], int(ee[r])) for r in range(rows)])
    assert np.array_equal(codes, want)
    value, step = want * np.ldexp(1.0, ee)[:, None], np.ldexp(1.0, ee)[:, None]
    near = np.abs(value - y64) <= step / 2 + slack
    assert (near | (np.abs(y64) > 127 * step - slack)).all()


# lengths on either side of every form: one warp, blocks of 4 to 32 warps, rows longer than the registers
LENGTHS = [1, 7, 8, 32, 255, 256, 257, 1000, 1024, 1025, 2049, 4096, 4097, 5001, 8192, 8200, 16384, 16385, 20008, 33001]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C", LENGTHS)
def test_lengths(C, dtype):
    import torch
    rng = np.random.default_rng(C)
    x, res, gain = make(rng, 3, C, dtype)
    h = (x.double() + res.double()).to(x.dtype)
    for out in (binding.NORM_I8, binding.NORM_I8_ROWS, binding.NORM_MX):
        kept = torch.zeros_like(x).cuda()
        codes, scales = binding.qrmsnorm(x.cuda(), gain.cuda(), EPS, residual=res.cuda(), sum_out=kept, out=out, e=-5)
        assert torch.equal(kept.cpu(), h)
        check(out, codes, scales, h, gain, e=-5)
        codes, scales = binding.qrmsnorm(x.cuda(), gain.cuda(), EPS, out=out, e=-4, layout=binding.MX_ROWS)
        check(out, codes, scales, x, gain, e=-4, layout=binding.MX_ROWS)


@pytest.mark.parametrize("rows,C", [(1, 64), (127, 96), (129, 40), (300, 257), (1030, 1024), (1500, 600), (600, 4096), (520, 5000)])
def test_row_counts(rows, C):
    rng = np.random.default_rng(rows + C)
    x, res, gain = make(rng, rows, C, "bfloat16")
    h = (x.double() + res.double()).to(x.dtype)
    for out in (binding.NORM_I8, binding.NORM_I8_ROWS, binding.NORM_MX):
        codes, scales = binding.qrmsnorm(x.cuda(), gain.cuda(), EPS, residual=res.cuda(), out=out, e=-4)
        check(out, codes, scales, h, gain, e=-4)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C", [200, 3000, 20000])
@pytest.mark.parametrize("place", ["x", "residual"])
def test_sum_in_place_and_strided_rows(place, C, dtype):
    import torch
    rng = np.random.default_rng(C + 1)
    x, res, gain = make(rng, 4, C + 9, dtype)
    for start, width in ((0, C), (1, C)):
        xd, rd = x.cuda(), res.cuda()
        xv, rv = xd[:, start:start + width], rd[:, start:start + width]
        g = gain[:width].contiguous()
        h = (x.double() + res.double()).to(x.dtype)
        codes, scales = binding.qrmsnorm(xv, g.cuda(), EPS, residual=rv, sum_out=xv if place == "x" else rv, out=binding.NORM_I8_ROWS)
        check(binding.NORM_I8_ROWS, codes, scales, h[:, start:start + width], g)
        kept, other = (xd, rd) if place == "x" else (rd, xd)
        assert torch.equal(kept.cpu()[:, start:start + width], h[:, start:start + width])
        before = x if place == "x" else res
        assert torch.equal(kept.cpu()[:, start + width:], before[:, start + width:]), "written behind the row"
        assert torch.equal(other.cpu(), res if place == "x" else x)


@pytest.mark.parametrize("out", [binding.NORM_I8, binding.NORM_I8_ROWS, binding.NORM_MX])
@pytest.mark.parametrize("C", [96, 3000, 20000])
def test_rows_that_are_zero_or_not_finite(C, out):
    import torch
    rng = np.random.default_rng(9)
    x, _, gain = make(rng, 6, C, "float32")
    x[0] = 0
    x[1, 3] = float("nan")
    x[2, 5] = float("inf")
    x[3] *= 1e-30
    x[4] *= 1e30
    for eps in (EPS, 0.0):
        codes, scales = binding.qrmsnorm(x.cuda(), gain.cuda(), eps, out=out, e=-5)
        check_rows = [3, 4, 5] if eps == 0.0 else [0, 3, 4, 5]
        for r in (0, 1, 2):                                      # 0 / 0, NaN everywhere, Inf * 0 and 0: nothing but zeros
            assert not codes[r].any()
        if out == binding.NORM_I8_ROWS:
            assert (scales[:3].cpu() == 127).all()
        if out == binding.NORM_MX:
            s = scales.cpu().view(-1, 32, 4, 4)[:, :3, 0]
            assert (s == 127).all()
        for r in check_rows:
            c, s = binding.qrmsnorm(x[r:r + 1].cuda(), gain.cuda(), eps, out=out, e=-5)
            check(out, c, s, x[r:r + 1], gain, e=-5, eps=eps)
            assert torch.equal(c[0], codes[r])


def test_codes_saturate_at_a_fixed_exponent():
    import torch
    x = torch.randn((5, 500))
    gain = torch.full((500,), 40.0)
    codes, _ = binding.qrmsnorm(x.cuda(), gain.cuda(), EPS, out=binding.NORM_I8, e=-3)
    check(binding.NORM_I8, codes, None, x, gain, e=-3)
    assert codes.max() == 127 and codes.min() == -127
    for e in (-126, 126):
        codes, _ = binding.qrmsnorm(x.cuda(), gain.cuda(), EPS, out=binding.NORM_I8, e=e)
        check(binding.NORM_I8, codes, None, x, gain, e=e)


def test_capture_replays_on_new_values():
    import torch
    x, res = (torch.randn((40, 777), device="cuda", dtype=torch.float16) for _ in range(2))
    gain = torch.rand((777,), device="cuda", dtype=torch.float16)
    codes = torch.zeros((40, 777), dtype=torch.int8, device="cuda")
    scales = torch.zeros((40,), dtype=torch.uint8, device="cuda")
    kept = torch.zeros_like(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.qrmsnorm(x, gain, EPS, residual=res, sum_out=kept, out=binding.NORM_I8_ROWS, codes=codes, scales=scales)
    for _ in range(3):
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        want = binding.qrmsnorm(x, gain, EPS, residual=res, out=binding.NORM_I8_ROWS)
        assert torch.equal(codes, want[0]) and torch.equal(scales, want[1]) and torch.equal(kept, x + res)


def test_refused_tensors():
    import torch
    x, g = torch.zeros((4, 64), device="cuda"), torch.ones((64,), device="cuda")
    for kw in (dict(residual=x.half()), dict(residual=x[:3]), dict(sum_out=x.cpu()), dict(codes=torch.zeros((4, 63), dtype=torch.int8, device="cuda")),
               dict(out=binding.NORM_MX, scales=torch.zeros((100,), dtype=torch.uint8, device="cuda"))):
        with pytest.raises(ValueError):
            binding.qrmsnorm(x, g, EPS, **kw)
    with pytest.raises(ValueError):
        binding.qrmsnorm(x, g[:60], EPS)
    with pytest.raises(ValueError):
        binding.qrmsnorm(x, g.half(), EPS)
    with pytest.raises(binding.QconvError):
        binding.qrmsnorm(x, g, -1.0)
    assert binding.qrmsnorm(x[:0], g, EPS)[0].shape == (0, 64)
