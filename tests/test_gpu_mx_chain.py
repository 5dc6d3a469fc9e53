"""The operators for quantized language models run together, as a model's block uses them: residual addition and norm into
the library's operand types, products on them, keys and values into a quantized cache and back."""
import numpy as np
import pytest

from oracle import mx_ref, ref
from paper_1805_07941_b200 import binding

pytestmark = pytest.mark.gpu

EPS = 1e-5


def expected_operand(x, res, gain):
    """(sum kept, values of the 4-bit operand) of a norm, in float64."""
    h = (x.double() + res.double()).to(x.dtype)
    y, _ = mx_ref.rmsnorm(h.double().cpu().numpy(), gain.double().cpu().numpy(), EPS)
    codes, scales = mx_ref.mx_quantize(y)
    return h, mx_ref.mx_values(codes, scales, y.shape[1])


@pytest.mark.parametrize("tokens", [1, 5, 130])
def test_norm_products_and_cache(tokens):
    """x + residual -> norm in 4 bits -> joint projection -> keys and values into the cache -> read back, also captured."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    C, heads, D, slots_n = 512, 4, 64, 256
    dt = torch.bfloat16
    x, res = (torch.randn((tokens, C), generator=gen, device="cuda", dtype=dt) for _ in range(2))
    gain = (1 + 0.1 * torch.randn((C,), generator=gen, device="cuda")).to(dt)
    w = torch.randn((3 * heads * D, C), generator=gen, device="cuda") * C**-0.5
    wc, ws = binding.qmx_quantize(w)
    lin = binding.QMXLinear(wc, ws, 3 * heads * D, C, dtype=dt)
    cache = binding.QCache.empty(slots_n, heads, D, binding.CACHE_I8)
    slots = torch.randperm(slots_n, generator=gen, device="cuda")[:tokens]
    kept, y = torch.empty_like(x), torch.empty((tokens, 3 * heads * D), dtype=dt, device="cuda")
    pitch, size = binding._mx_size(tokens, C, binding.MX_TILES)
    codes, scales = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in ((tokens, pitch), (size,)))
    back = torch.zeros((2, tokens, heads, D), dtype=dt, device="cuda")

    def block():
        binding.qrmsnorm(x, gain, EPS, residual=res, sum_out=kept, out=binding.NORM_MX, codes=codes, scales=scales)
        lin.run(codes, scales, y)
        k, v = (y[:, a * heads * D:(a + 1) * heads * D].unflatten(1, (heads, D)) for a in (1, 2))
        cache.write(slots, k, v)
        cache.read(slots, back[0], back[1])

    def check():
        h, operand = expected_operand(x, res, gain)
        assert torch.equal(kept, h)
        assert np.array_equal(binding.qmx_dequantize(codes, scales, C).double().cpu().numpy(), operand)
        wq = binding.qmx_dequantize(wc, ws, C).double().cpu().numpy()
        want, reach = operand @ wq.T, np.abs(operand) @ np.abs(wq).T
        # C additions in float32 (2^-23 of what is summed up each), then half a step of bfloat16
        assert (np.abs(y.double().cpu().numpy() - want) <= C * 2.0**-23 * reach + 2.0**-8 * np.abs(want)).all()
        for a, got in ((1, back[0]), (2, back[1])):
            kv = y[:, a * heads * D:(a + 1) * heads * D].double().cpu().numpy().reshape(-1, D)
            e = np.array([mx_ref.i8_exponent(r) for r in kv])
            values = np.stack([mx_ref.i8_codes(r, int(n)) for r, n in zip(kv, e)]) * np.ldexp(1.0, e)[:, None]
            assert np.array_equal(got.double().cpu().numpy().reshape(-1, D), values)

    block()
    torch.cuda.synchronize()
    assert lin.status() == 0
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block()
    for _ in range(2):
        x.normal_()
        slots.copy_(torch.randperm(slots_n, device="cuda")[:tokens])
        graph.replay()
        torch.cuda.synchronize()
        check()


def test_norm_into_an_int8_inner_product_layer():
    """The int8 norm at a calibrated exponent is the input of the library's own inner-product layer."""
    import torch
    rng = np.random.default_rng(3)
    tokens, C, N, e_x = 24, 256, 96, -5
    x = rng.standard_normal((tokens, C)).astype(np.float32)
    gain = (1 + 0.1 * rng.standard_normal(C)).astype(np.float32)
    codes, _ = binding.qrmsnorm(torch.from_numpy(x).cuda(), torch.from_numpy(gain).cuda(), EPS, out=binding.NORM_I8, e=e_x)
    y, _ = mx_ref.rmsnorm(x.astype(np.float64), gain.astype(np.float64), EPS)
    want_codes = mx_ref.i8_codes(y, e_x)
    assert np.array_equal(codes.cpu().numpy(), want_codes)
    wq, e_w = binding.qquantize_weights(rng.standard_normal((N, 1, 1, C)).astype(np.float32) * 0.06, N, 1, 1, C)
    acc_exp = binding.qacc_exponents(e_x, e_w)
    layer = binding.QConv(wq, None, None, None, acc_exp, N=tokens, H=1, W=1, C=C, K=N, R=1, S=1, out_mode=binding.OUT_FLOAT)
    out = torch.empty((tokens, 1, 1, N), dtype=torch.float32, device="cuda")
    layer.run(codes.view(tokens, 1, 1, C), out)
    assert layer.status() == 0
    want = ref.qconv(want_codes.reshape(tokens, 1, 1, C), wq, None, None, None, None, acc_exp, R=1, S=1, out_mode=2)
    assert np.array_equal(out.cpu().numpy(), want)


def test_the_codec_is_the_np_codec_block_by_block():
    """A block's codes are those of the library's (4, 1) codec at the block's exponent (whose integers are twice the values
    here)."""
    import torch
    x = torch.randn((8, 64), device="cuda") * torch.logspace(-3, 3, 8, device="cuda")[:, None]
    codes, scales = binding.qmx_quantize(x, layout=binding.MX_ROWS)
    flat = mx_ref.unpack(codes.cpu().numpy())
    for r in range(8):
        for b in range(2):
            e = int(scales[r, b]) - 127
            want = binding.qquantize_f32_np(x[r, 32 * b:32 * b + 32].contiguous(), e - 1, 4, 1).cpu().numpy()
            assert np.array_equal(flat[r, 32 * b:32 * b + 32], want)


def test_two_streams_at_once():
    """The same calls from two streams on tensors of their own: nothing is shared between them."""
    import torch
    streams = [torch.cuda.Stream() for _ in range(2)]
    w = torch.randn((384, 320), device="cuda")
    wc, ws = binding.qmx_quantize(w)
    lins = [binding.QMXLinear(wc, ws, 384, 320, dtype=torch.float32) for _ in range(2)]
    xs = [torch.randn((n, 320), device="cuda", dtype=torch.float16) for n in (40, 300)]
    gain = torch.ones((320,), device="cuda", dtype=torch.float16)
    want = []
    for x, lin in zip(xs, lins):
        c, s = binding.qrmsnorm(x, gain, EPS, out=binding.NORM_MX)
        want.append(lin.run(c, s).clone())
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                c, s = binding.qrmsnorm(xs[i], gain, EPS, out=binding.NORM_MX)
                got[i].append(lins[i].run(c, s))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i]) for i in range(2) for y in got[i])
    assert all(lin.status() == 0 for lin in lins)
