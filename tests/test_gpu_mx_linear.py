"""Inner-product layers on microscaled 4-bit operands against float64."""
import numpy as np
import pytest

from oracle import mx_ref
from paper_1805_07941_b200 import binding

pytestmark = pytest.mark.gpu

# (tokens, N, K): every column width, one to many tiles, split and whole contractions, ragged everything
SHAPES = [(1, 1, 1), (1, 128, 256), (3, 130, 33), (16, 256, 512), (17, 384, 1000), (33, 64, 4096), (64, 1024, 2048), (65, 100, 130),
          (128, 640, 257), (129, 200, 300), (300, 513, 700), (1, 4096, 4096), (8, 20000, 320), (200, 2100, 4100),
          # (on single SMs: few tiles and a long contraction, shared by eight, four, two; rings that go round many times)
          (256, 256, 6000), (130, 500, 7000), (100, 8000, 4000), (70, 16000, 1100), (40, 19000, 2500)]


def operand(rng, rows, K, low=126, high=129):
    """Random codes and scales: (values float64, packed codes, scales in tiles) on the GPU."""
    import torch
    blocks = -(-K // 32)
    codes = rng.integers(0, 16, (rows, blocks * 32)).astype(np.uint8)
    codes[codes == 8] = 0
    codes[:, K:] = 0
    scales = rng.integers(low, high, (rows, blocks)).astype(np.uint8)
    r, b = np.arange(rows)[:, None], np.arange(blocks)[None]
    tiles = np.full(-(-rows // 128) * -(-blocks // 4) * 512, 127, np.uint8)
    tiles[((r // 128) * -(-blocks // 4) + b // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + b % 4] = scales
    return mx_ref.mx_values(codes, scales, K), torch.from_numpy(mx_ref.pack(codes)).cuda(), torch.from_numpy(tiles).cuda()


def layer(rng, T, N, K, dtype, bias=False, relu=False, low=126, high=129):
    import torch
    x, xc, xs = operand(rng, T, K, low, high)
    w, wc, ws = operand(rng, N, K, low, high)
    b = rng.integers(-400, 400, N).astype(np.float32) / 4 if bias else None
    lin = binding.QMXLinear(wc, ws, N, K, bias=torch.from_numpy(b).cuda() if bias else None, relu=int(relu), dtype=getattr(torch, dtype))
    return lin, xc, xs, mx_ref.linear(x, w, b, relu), x, w


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("T,N,K", SHAPES)
def test_exact_sums(T, N, K, dtype):
    """With scales 2^-1 .. 2^1 every product is a multiple of 2^-4 and at most 144, so that for K <= 7000 every partial
    sum is a multiple of 2^-4 below 2^20: 24 bits hold it, whatever the order.  The output is then the sum rounded once."""
    import torch
    rng = np.random.default_rng(T * 7 + N * 3 + K)
    lin, xc, xs, want, _, _ = layer(rng, T, N, K, dtype, bias=N % 2 == 0, relu=K % 2 == 0)
    tdt = getattr(torch, dtype)
    flat = torch.full((T * (N + 5) + 64,), 77.0, dtype=tdt, device="cuda")
    y = torch.as_strided(flat, (T, N), (N + 5, 1), 1)
    lin.run(xc, xs, y)
    assert lin.status() == 0, lin.describe()
    want = torch.from_numpy(want).to(torch.float32).to(tdt)      # exact in float32
    assert torch.equal(y.cpu(), want), lin.describe()
    torch.as_strided(flat, (T, N), (N + 5, 1), 1).fill_(77.0)
    assert (flat == 77.0).all(), "written outside the output"


@pytest.mark.parametrize("T,N,K", [(2048, 2560, 256), (2000, 2500, 1000), (1900, 4800, 130), (5000, 1100, 2050), (257, 19000, 96), (2600, 9999, 640)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_exact_sums_on_pairs_of_sms(T, N, K, dtype):
    """Many tiles: several to a pair (both accumulators, the walk's groups) and ragged ends."""
    import torch
    rng = np.random.default_rng(T + N + K)
    lin, xc, xs, _, x, w = layer(rng, T, N, K, dtype, bias=True, relu=True)
    want = torch.from_numpy(x).cuda() @ torch.from_numpy(w).cuda().T + lin._keep[2].double()
    want = want.clamp(min=0).float().to(lin.dtype)
    for start, ld in ((0, N), (16, -(-N // 8) * 8 + 16), (1, N + 3)):       # as it comes, rows at 16 bytes, rows anywhere
        flat = torch.full((T * ld + 64,), 77.0, dtype=lin.dtype, device="cuda")
        y = lin.run(xc, xs, torch.as_strided(flat, (T, N), (ld, 1), start))
        assert lin.status() == 0 and "pair=1" in lin.describe()
        per_16_bytes = 4 if dtype == "float32" else 8
        assert ("staged=1" in lin.describe()) == (start % per_16_bytes == 0 and ld % per_16_bytes == 0 and N % per_16_bytes == 0)
        assert torch.equal(y, want)
        y.fill_(77.0)
        assert (flat == 77.0).all(), "written outside the output"


@pytest.mark.parametrize("T,N,K", [(1, 300, 5000), (40, 200, 2000), (150, 300, 1024)])
def test_real_operands(T, N, K):
    """Quantized normal values: scales of any size.  Every one of the sum's additions is off by at most 2^-23 of what is
    being added up, which sum |x w| bounds, and there are at most K of them; the rounding to float32 is another 2^-24."""
    import torch
    rng = np.random.default_rng(N + K)
    x = torch.from_numpy((rng.standard_normal((T, K)) * np.exp2(rng.integers(-8, 8, (T, K)))).astype(np.float32))
    w = torch.from_numpy(rng.standard_normal((N, K)).astype(np.float32) * 0.03)
    xc, xs = binding.qmx_quantize(x.cuda())
    wc, ws = binding.qmx_quantize(w.cuda())
    y = binding.QMXLinear(wc, ws, N, K, dtype=torch.float32).run(xc, xs).double().cpu().numpy()
    xq, wq = (binding.qmx_dequantize(c, s, K).double().cpu().numpy() for c, s in ((xc, xs), (wc, ws)))
    want = xq @ wq.T
    bound = K * 2.0**-23 * (np.abs(xq) @ np.abs(wq).T) + 2.0**-24 * np.abs(want)
    assert (np.abs(y - want) <= bound).all()
    # and in the mean far nearer: the errors' signs vary (a wrong scale or a lost block is off by percents)
    assert np.abs(y - want).sum() <= 2.0**-16 * (np.abs(xq) @ np.abs(wq).T).sum()


def test_extreme_scales_and_overflow():
    import torch
    rng = np.random.default_rng(11)
    T, N, K = 20, 140, 96
    xv, xc, xs = operand(rng, T, K, 30, 31)                      # 2^-97
    wv, wc, ws = operand(rng, N, K, 250, 251)                    # 2^123
    y = binding.QMXLinear(wc, ws, N, K, dtype=torch.float32).run(xc, xs)
    assert np.array_equal(y.cpu().numpy(), (xv @ wv.T).astype(np.float32))
    y = binding.QMXLinear(wc, ws, N, K, dtype=torch.float16).run(xc, xs)
    with np.errstate(over="ignore"):
        assert np.array_equal(y.cpu().numpy(), (xv @ wv.T).astype(np.float32).astype(np.float16))


def test_the_same_call_gives_the_same_bits_and_rows_do_not_depend_on_their_neighbours():
    import torch
    rng = np.random.default_rng(12)
    lin, xc, xs, _, x, _ = layer(rng, 16, 512, 4096, "float32", low=115, high=135)
    y = lin.run(xc, xs)
    for _ in range(5):
        assert torch.equal(lin.run(xc, xs), y)
    # scale bytes behind the last token are whatever they are: also NaN
    tiles = xs.clone().view(1, -1, 32, 4, 4)
    tiles[:, :, 16:] = 255
    tiles[:, :, :, 1:] = 255
    assert torch.equal(lin.run(xc, tiles.view(-1)), y)


def test_many_tokens_reuse_the_handle():
    import torch
    rng = np.random.default_rng(13)
    _, wc, ws = operand(rng, 96, 160)
    w = binding.qmx_dequantize(wc, ws, 160).double().cpu().numpy()
    lin = binding.QMXLinear(wc, ws, 96, 160, dtype=torch.float32)
    for T in (5, 700, 1, 64, 5):
        x, xc, xs = operand(rng, T, 160)
        assert np.array_equal(lin.run(xc, xs).cpu().numpy(), (x @ w.T).astype(np.float32)), T


def test_capture_streams_and_freshly_written_operands():
    import torch
    T, N, K = 24, 300, 640
    w = torch.randn((N, K), device="cuda")
    x = torch.randn((T, K), device="cuda")
    wc, ws = binding.qmx_quantize(w)
    xc, xs = binding.qmx_quantize(x)
    lin = binding.QMXLinear(wc, ws, N, K, dtype=torch.float32)
    y = torch.zeros((T, N), device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        binding.qmx_quantize(w, codes=wc, scales=ws)             # the weights too are written just before they are read
        binding.qmx_quantize(x, codes=xc, scales=xs)
        lin.run(xc, xs, y)
    for _ in range(4):
        w.copy_(torch.randn((N, K), device="cuda"))
        x.copy_(torch.randn((T, K), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        a, b = binding.qmx_dequantize(xc, xs, K).double(), binding.qmx_dequantize(wc, ws, K).double()
        assert torch.equal(a.float(), binding.qmx_dequantize(*binding.qmx_quantize(x), K))
        assert (y.double() - a @ b.T).abs().max() <= K * 2.0**-23 * (a.abs() @ b.abs().T).max()
    # two streams at once on one handle
    outs = [torch.zeros((T, N), device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for s, o in zip(streams, outs):
            with torch.cuda.stream(s):
                lin.run(xc, xs, o)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], y) and torch.equal(outs[1], y) and lin.status() == 0


def test_a_wait_that_runs_out_is_reported_and_the_context_survives():
    import torch
    rng = np.random.default_rng(14)
    for T, N, K in ((4, 256, 4096), (300, 600, 1024), (2000, 2048, 2048)):
        lin, xc, xs, want, _, _ = layer(rng, T, N, K, "float32")
        lin.set_wait_limit(0)
        lin.run(xc, xs)
        assert lin.status() == binding.ERR_TIMEOUT
        lin.set_wait_limit(1 << 22)
        y = lin.run(xc, xs)
        assert lin.status() == 0 and np.array_equal(y.cpu().numpy(), want.astype(np.float32))


def test_refused_tensors():
    import torch
    rng = np.random.default_rng(15)
    lin, xc, xs, _, _, _ = layer(rng, 4, 64, 64, "bfloat16")
    for bad in (torch.zeros((4, 64), device="cuda"), torch.zeros((4, 63), dtype=torch.bfloat16, device="cuda"),
                torch.zeros((64, 4), dtype=torch.bfloat16, device="cuda").t()):
        with pytest.raises(ValueError):
            lin.run(xc, xs, bad)
    with pytest.raises(ValueError):
        lin.run(xc, xs[:256])
    with pytest.raises(ValueError):
        lin.run(torch.zeros((4, 48), dtype=torch.uint8, device="cuda"), xs)
    with pytest.raises(ValueError):
        lin.run(xc.cpu(), xs)
    with pytest.raises(ValueError):
        binding.QMXLinear(xc, xs, 64, 64)
    with pytest.raises(ValueError):
        binding.QMXLinear(xc, xs, 4, 64, bias=torch.zeros(3, device="cuda"))
    with pytest.raises(ValueError):
        binding.QMXLinear(xc, xs, 4, 64, dtype=torch.float64)
    assert lin.run(xc[:0], xs).shape == (0, 64)
