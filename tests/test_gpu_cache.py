"""Quantized caches on the GPU against the oracle: codes, scale bytes and values equal, every other byte left alone."""
import numpy as np
import pytest

from oracle import mx_ref
from paper_1805_07941_b200 import binding

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]
FORMATS = {"i8": binding.CACHE_I8, "mx": binding.CACHE_MX}


def expect(x, fmt):
    """[rows, heads, D] float64 -> (codes, scales, values) as the cache holds them and gives them back."""
    rows, heads, D = x.shape
    flat = x.reshape(rows * heads, D)
    if fmt == "mx":
        c, s = mx_ref.mx_quantize(flat)
        return mx_ref.pack(c).reshape(rows, heads, -1), s.reshape(rows, heads, -1), mx_ref.mx_values(c, s, D).reshape(x.shape)
    e = np.array([mx_ref.i8_exponent(v) for v in flat])
    c = np.stack([mx_ref.i8_codes(v, int(k)) for v, k in zip(flat, e)])
    return (c.view(np.uint8).reshape(rows, heads, D), (e + 127).astype(np.uint8).reshape(rows, heads, 1),
            (c * np.ldexp(1.0, e)[:, None]).reshape(x.shape))


def values(rng, shape, dtype, wild=True):
    import torch
    x = rng.standard_normal(shape) * np.exp2(rng.integers(-6, 6, shape[:2] + (1,)))
    if wild:
        for v in (np.nan, np.inf, -np.inf, 0.0):
            x[rng.random(shape) < 0.01] = v
        x[rng.random(shape[:2]) < 0.1] = 0
    return torch.from_numpy(x.astype(np.float32)).to(getattr(torch, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("heads,D", [(1, 1), (3, 7), (2, 32), (8, 64), (5, 80), (1, 100), (8, 128), (2, 200), (3, 256), (2, 300), (1, 1024)])
def test_write_and_read(heads, D, fmt, dtype):
    import torch
    rng = np.random.default_rng(heads * 100 + D)
    slots_n, rows = 50, 21
    cache = binding.QCache.empty(slots_n, heads, D, FORMATS[fmt])
    for t in cache._keep:
        t.fill_(0x35)
    k, v = values(rng, (rows, heads, D), dtype), values(rng, (rows, heads, D), dtype)
    slots = rng.permutation(slots_n)[:rows].astype(np.int64)
    slots[[2, 9]] = [-1, slots_n]                            # padding: skipped
    slots[15] = -(1 << 40)
    kept = (slots >= 0) & (slots < slots_n)
    cache.write(torch.from_numpy(slots).cuda(), k.cuda(), v.cuda())
    for x, codes, scales in ((k, cache.k_codes, cache.k_scales), (v, cache.v_codes, cache.v_scales)):
        c, s, _ = expect(x.double().numpy(), fmt)
        want_c, want_s = np.full(codes.shape, 0x35, np.uint8), np.full(scales.shape, 0x35, np.uint8)
        want_c[slots[kept]], want_s[slots[kept]] = c[kept], s[kept]
        assert np.array_equal(scales.cpu().numpy(), want_s)
        assert np.array_equal(codes.cpu().numpy(), want_c)
    ko, vo = torch.full((rows, heads, D), 5.0, dtype=k.dtype, device="cuda"), torch.full((rows, heads, D), 5.0, dtype=k.dtype, device="cuda")
    cache.read(torch.from_numpy(slots).cuda(), ko, vo)
    for x, got in ((k, ko), (v, vo)):
        want = expect(x.double().numpy(), fmt)[2]
        want[~kept] = 5.0                                    # rows without a slot stay as they are
        assert np.array_equal(got.double().cpu().numpy(), want)
    again = torch.from_numpy(np.repeat(slots[kept][:1], 3)).cuda()           # one slot several times
    ko, vo = torch.zeros((3, heads, D), dtype=k.dtype, device="cuda"), torch.zeros((3, heads, D), dtype=k.dtype, device="cuda")
    cache.read(again, ko, vo)
    assert torch.equal(ko[0], ko[1]) and torch.equal(vo[0], vo[2])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D", [64, 77])
def test_views_of_a_joint_projection(D, fmt):
    """Keys and values as parts of one row [queries | keys | values], and a cache of one tensor."""
    import torch
    rng = np.random.default_rng(D)
    heads, rows = 2, 13
    joint = values(rng, (rows, 1, 8 * D), "bfloat16")[:, 0].cuda()
    k, v = (joint[:, a * D:(a + heads) * D].unflatten(1, (heads, D)) for a in (4, 6))
    slots = torch.from_numpy(rng.permutation(40)[:rows].astype(np.int64)).cuda()
    cache = binding.QCache.empty(40, heads, D, FORMATS[fmt])
    cache.write(slots, k, v)
    out = torch.zeros((rows, 8 * D), dtype=torch.bfloat16, device="cuda")
    ko, vo = (out[:, a * D:(a + heads) * D].unflatten(1, (heads, D)) for a in (4, 6))
    cache.read(slots, ko, vo)
    for x, got in ((k, ko), (v, vo)):
        assert np.array_equal(got.double().cpu().numpy(), expect(x.double().cpu().numpy(), fmt)[2])
    assert not out[:, :4 * D].any(), "written beside the heads"
    one = binding.QCache.empty(40, heads, D, FORMATS[fmt], values=False)
    one.write(slots, k.transpose(0, 1).contiguous().transpose(0, 1))         # heads far apart, tokens near
    got = torch.zeros((rows, heads, D), dtype=torch.float32, device="cuda")
    one.read(slots, got)
    assert np.array_equal(got.double().cpu().numpy(), expect(k.double().cpu().numpy(), fmt)[2])


@pytest.mark.parametrize("fmt", FORMATS)
def test_offsets_beyond_32_bits(fmt):
    import torch
    D = 1024
    heads = 8 if fmt == "i8" else 16
    slots_n = (1 << 32) // (heads * (D if fmt == "i8" else D // 2)) + 5
    cache = binding.QCache.empty(slots_n, heads, D, FORMATS[fmt], values=False)
    slots = torch.tensor([slots_n - 1, 0, slots_n // 2, slots_n], device="cuda")
    x = values(np.random.default_rng(1), (4, heads, D), "float32", wild=False)
    cache.write(slots, x.cuda())
    got = torch.zeros((4, heads, D), device="cuda")
    cache.read(slots, got)
    want = expect(x.double().numpy(), fmt)[2]
    want[3] = 0
    assert np.array_equal(got.double().cpu().numpy(), want)
    assert int((cache.k_scales != 0).any(-1).any(-1).sum()) == 3


def test_more_rows_than_one_pass_of_the_grid():
    import torch
    gen = torch.Generator(device="cuda").manual_seed(4)
    rows, heads, D = 9000, 4, 128
    x = torch.randn((rows, heads, D), generator=gen, device="cuda", dtype=torch.float16)
    slots = torch.randperm(10000, generator=gen, device="cuda")[:rows]
    cache = binding.QCache.empty(10000, heads, D, binding.CACHE_I8)
    cache.write(slots, x, 2 * x)
    k, v = torch.zeros_like(x), torch.zeros_like(x)
    cache.read(slots, k, v)
    assert torch.equal(v, 2 * k)
    pick = [0, 1, 4095, 8999]
    assert np.array_equal(k[pick].double().cpu().numpy(), expect(x[pick].double().cpu().numpy(), "i8")[2])
    # nearest of steps 2^e with 127 * 2^e at most twice the head's top: off by at most top / 127
    assert ((x.float() - k.float()).abs() <= x.float().abs().amax(-1, keepdim=True) / 127).all()


def test_capture_with_slots_that_change():
    import torch
    cache = binding.QCache.empty(64, 2, 96, binding.CACHE_MX)
    k, v = (torch.randn((5, 2, 96), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    slots = torch.arange(5, device="cuda")
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.write(slots, k, v)
        cache.read(slots, ko, vo)
    for n in range(3):
        k.normal_()
        slots.copy_(torch.randperm(64, device="cuda")[:5])
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(ko.double().cpu().numpy(), expect(k.double().cpu().numpy(), "mx")[2])


def test_refused_tensors():
    import torch
    cache = binding.QCache.empty(16, 2, 64)
    x = torch.zeros((3, 2, 64), device="cuda")
    slots = torch.arange(3, device="cuda")
    for s, k, v in ((slots.int(), x, x), (slots.cpu(), x, x), (slots, x, None), (slots, x[:2], x), (slots, x, x.half()), (slots, x.double(), x.double()),
                    (slots, torch.zeros((3, 64, 2), device="cuda").transpose(1, 2), x), (slots[::2], x[:2], x[:2])):
        with pytest.raises(ValueError):
            cache.write(s, k, v)
        with pytest.raises(ValueError):
            cache.read(s, k, v)
    with pytest.raises(ValueError):
        binding.QCache(cache.k_codes, cache.k_scales[:10], cache.v_codes, cache.v_scales)
    with pytest.raises(ValueError):
        binding.QCache(cache.k_codes, cache.k_scales, cache.v_codes)
    cache.write(slots[:0], x[:0], x[:0])
