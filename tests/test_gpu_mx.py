"""Microscaled 4-bit conversion on the GPU against the oracle: every code and scale byte equal, every value exact."""
import numpy as np
import pytest

from oracle import mx_ref
from paper_1805_07941_b200 import binding

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]
LAYOUTS = {"rows": binding.MX_ROWS, "tiles": binding.MX_TILES}
RULES = {"cover": binding.MX_COVER, "floor": binding.MX_FLOOR}
GUARD = 64


def make(rng, rows, K, dtype, wild=True):
    """Values of the type with blocks of very different sizes, ties, and (wild) what is not a finite number."""
    import torch
    x = rng.standard_normal((rows, K))
    span = 6 if dtype == "float16" else 120 if wild else 30
    x *= np.exp2(rng.integers(-span, span // 2, (rows, -(-K // 32)))).repeat(32, axis=1)[:, :K]
    x[rng.random((rows, K)) < 0.3] *= 0.125
    grid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    tie = rng.random((rows, K)) < 0.1
    x[tie] = (rng.choice(grid, (rows, K)) * rng.choice([-1, 1], (rows, K)))[tie]
    if wild:
        for v in (np.nan, np.inf, -np.inf, 0.0, -0.0):
            x[rng.random((rows, K)) < 0.01] = v
        x[rng.random(rows) < 0.1] = 0
        if dtype != "float16":
            x[rng.random((rows, K)) < 0.005] = 3e38
    return torch.from_numpy(x.astype(np.float32)).to(getattr(torch, dtype))


def quantize_checked(x, rule, layout):
    """qmx_quantize into buffers with guards behind them."""
    import torch
    rows, K = x.shape
    n, m = binding.lib().qmx_code_bytes(rows, K), binding.lib().qmx_scale_bytes(rows, K, LAYOUTS[layout])
    codes = torch.full((n + GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((m + GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
    binding.qmx_quantize(x, rule=RULES[rule], layout=LAYOUTS[layout], codes=codes, scales=scales)
    codes, scales = codes.cpu().numpy(), scales.cpu().numpy()
    assert (codes[n:] == 0xA5).all() and (scales[m:] == 0xA5).all(), "written past the end"
    return codes[:n].reshape(rows, -1), scales[:m]


def check_quantize(x, rule, layout):
    codes, scales = quantize_checked(x.cuda() if not x.is_cuda else x, rule, layout)
    want, s = mx_ref.mx_quantize(x.float().cpu().numpy(), rule)
    assert np.array_equal(scales, mx_ref.to_tiles(s) if layout == "tiles" else s.reshape(-1))
    assert np.array_equal(codes, mx_ref.pack(want))


SHAPES = [(1, 1), (1, 31), (3, 32), (5, 33), (2, 128), (7, 130), (130, 257), (129, 64), (33, 1000), (1, 5000), (40, 96)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("rule", RULES)
@pytest.mark.parametrize("rows,K", SHAPES)
def test_quantize(rows, K, rule, layout, dtype):
    rng = np.random.default_rng(rows * 1000 + K)
    check_quantize(make(rng, rows, K, dtype), rule, layout)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("start,ld", [(0, 160), (1, 160), (8, 160), (3, 157)])
def test_quantize_strided_rows(start, ld, dtype):
    import torch
    rng = np.random.default_rng(start * 7 + ld)
    base = make(rng, 9, ld, dtype).cuda()
    x = torch.as_strided(base, (8, 140), (ld, 1), start)
    check_quantize(x, "cover", "tiles")


def test_quantize_the_smallest_and_largest_float32():
    import torch
    x = np.zeros((6, 32), np.float32)
    x[0, 0] = 2.0**-149
    x[1, :3] = [2.0**-126, 2.0**-130, -2.0**-128]
    x[2, :2] = [np.finfo(np.float32).max, -1e38]
    x[3, :2] = [np.inf, 1.0]
    x[4, :] = np.nan
    x[5, :2] = [-np.inf, np.nan]
    for rule in RULES:
        check_quantize(torch.from_numpy(x), rule, "rows")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
def test_dequantize_every_code_at_every_scale(layout, dtype):
    import torch
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))                # 512 codes, 16 blocks a row
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 16, axis=1)
    want = mx_ref.mx_values(mx_ref.unpack(codes), scales, 512)
    s = mx_ref.to_tiles(scales) if layout == "tiles" else scales
    tdt = getattr(torch, dtype)
    got = binding.qmx_dequantize(torch.from_numpy(codes).cuda(), torch.from_numpy(s).cuda(), 512, layout=LAYOUTS[layout], dtype=tdt)
    want = torch.from_numpy(want).to(torch.float32).to(tdt)                  # (exact in float32 wherever it is in range)
    assert torch.equal(torch.nan_to_num(got.cpu(), nan=7.0), torch.nan_to_num(want, nan=7.0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,K", SHAPES)
def test_dequantize_shapes(rows, K, dtype):
    import torch
    rng = np.random.default_rng(rows + K)
    codes = rng.integers(0, 16, (rows, -(-K // 32) * 32)).astype(np.uint8)
    scales = rng.integers(115, 135, (rows, -(-K // 32))).astype(np.uint8)
    want = mx_ref.mx_values(codes, scales, K)
    tdt = getattr(torch, dtype)
    for layout in LAYOUTS:
        s = torch.from_numpy(mx_ref.to_tiles(scales) if layout == "tiles" else scales).cuda()
        c = torch.from_numpy(mx_ref.pack(codes)).cuda()
        flat = torch.full((rows * (K + 3) + GUARD,), 9.0, dtype=tdt, device="cuda")
        out = torch.as_strided(flat, (rows, K), (K + 3, 1), 1)               # rows apart, misaligned
        binding.qmx_dequantize(c, s, K, layout=LAYOUTS[layout], out=out)
        assert np.array_equal(out.float().cpu().numpy(), want)
        left = flat.clone()
        torch.as_strided(left, (rows, K), (K + 3, 1), 1).fill_(9.0)
        assert (left == 9.0).all(), "written between the rows"
        assert np.array_equal(binding.qmx_dequantize(c, s, K, layout=LAYOUTS[layout], dtype=tdt).float().cpu().numpy(), want)


def test_large_tensor_agrees_with_itself_in_pieces():
    import torch
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((4096, 8200), generator=gen, device="cuda", dtype=torch.bfloat16)
    codes, scales = binding.qmx_quantize(x, layout=binding.MX_ROWS)
    y = binding.qmx_dequantize(codes, scales, 8200, layout=binding.MX_ROWS, dtype=torch.bfloat16)
    for r in (0, 127, 2048, 4095):
        c, s = mx_ref.mx_quantize(x[r:r + 1].float().cpu().numpy())
        assert np.array_equal(codes[r:r + 1].cpu().numpy(), mx_ref.pack(c)) and np.array_equal(scales[r:r + 1].cpu().numpy(), s)
        assert np.array_equal(y[r:r + 1].float().cpu().numpy(), mx_ref.mx_values(c, s, 8200))
    # nearest: half a step of the largest code at most (values up to 6 * 2^e, steps up to 2 * 2^e), so a third of the block's top
    top = torch.nn.functional.pad(x.float(), (0, -8200 % 32)).unflatten(-1, (-1, 32)).abs().amax(-1).repeat_interleave(32, -1)[:, :8200]
    assert ((x.float() - y.float()).abs() <= top / 3).all()


def test_capture_and_another_stream():
    import torch
    x = torch.randn((70, 300), device="cuda")
    want = binding.qmx_quantize(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    codes, scales = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    y = torch.zeros((70, 300), device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        binding.qmx_quantize(x, codes=codes, scales=scales)
        binding.qmx_dequantize(codes, scales, 300, out=y)
    for k in range(3):
        x.copy_(torch.randn((70, 300), device="cuda") * 10.0**k)
        graph.replay()
        torch.cuda.synchronize()
        again = binding.qmx_quantize(x)
        assert torch.equal(codes, again[0]) and torch.equal(scales, again[1])
        assert torch.equal(y, binding.qmx_dequantize(*again, 300))


def test_refused_tensors():
    import torch
    x = torch.zeros((4, 64), device="cuda")
    with pytest.raises(ValueError):
        binding.qmx_quantize(x.double())
    with pytest.raises(ValueError):
        binding.qmx_quantize(x.t())
    with pytest.raises(ValueError):
        binding.qmx_quantize(x.cpu())
    with pytest.raises(ValueError):
        binding.qmx_quantize(x, codes=torch.zeros((4, 16), dtype=torch.uint8, device="cuda"))
    codes, scales = binding.qmx_quantize(x)
    with pytest.raises(ValueError):
        binding.qmx_dequantize(codes, scales[:100], 64)
    with pytest.raises(ValueError):
        binding.qmx_dequantize(codes, scales, 64, out=torch.zeros((4, 60), device="cuda"))
    empty = binding.qmx_quantize(torch.zeros((0, 64), device="cuda"))
    assert empty[0].shape == (0, 32) and binding.qmx_dequantize(*empty, 64).shape == (0, 64)
