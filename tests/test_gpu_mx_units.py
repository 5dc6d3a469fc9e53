"""Rows that can be reached in units of 2 to 32 bytes, int8 codes from any address on, and cache heads that fill part of a
power of two of lanes: every code, scale byte and value equal to the oracle's, nothing around them written."""
import numpy as np
import pytest

from oracle import mx_ref
from paper_1805_07941_b200 import binding
from tests.test_gpu_cache import FORMATS, expect, values
from tests.test_gpu_mx import check_quantize, make as make_blocks
from tests.test_gpu_norm import EPS, check, make as make_rows

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]
MARK = 77.0


def placed(x, unit):
    """x on the device as a view whose rows start `unit` bytes (and no more) aligned, and the storage around it."""
    import torch
    rows, width = x.shape
    step = unit // x.element_size()
    if step == 0:
        return None, None
    start = step if unit < 32 else 0
    pitch = -(-width // step) * step
    pitch += step if pitch // step % 2 == 0 else 2 * step
    flat = torch.full((start + rows * pitch + 32,), MARK, dtype=x.dtype, device="cuda")
    view = torch.as_strided(flat, (rows, width), (pitch, 1), start)
    view.copy_(x)
    assert (view.data_ptr() | pitch * x.element_size()) % (2 * unit if unit < 32 else unit) in ((unit,) if unit < 32 else (0,))
    return view, flat


def around(view, flat):
    """The storage's elements that are not the view's."""
    import torch
    mask = torch.ones_like(flat, dtype=torch.bool)
    torch.as_strided(mask, view.shape, view.stride(), view.storage_offset()).fill_(False)
    return flat[mask]


UNITS = [2, 4, 8, 16, 32]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("unit", UNITS)
@pytest.mark.parametrize("rows,K", [(1, 1), (3, 30), (5, 129), (131, 258), (40, 515), (9, 1031), (70, 2050)])
def test_codec(rows, K, unit, dtype):
    import torch
    x = make_blocks(np.random.default_rng(rows + K), rows, K, dtype)
    view, flat = placed(x, unit)
    if view is None:
        pytest.skip("below the type's size")
    for layout in ("rows", "tiles"):
        check_quantize(view, "cover", layout)
    codes, scales = mx_ref.mx_quantize(x.float().numpy())
    want = torch.from_numpy(mx_ref.mx_values(codes, scales, K)).to(x.dtype)
    y, flat = placed(torch.zeros_like(x), unit)
    binding.qmx_dequantize(torch.from_numpy(mx_ref.pack(codes)).cuda(), torch.from_numpy(scales).cuda(), K, layout=binding.MX_ROWS, out=y)
    assert torch.equal(y.cpu(), want)
    assert (around(y, flat) == MARK).all()


# lengths on either side of the forms: part of a warp, one to nine warps with one piece or two, rows longer than the registers
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("unit", UNITS)
@pytest.mark.parametrize("rows,C", [(5, 3), (9, 62), (7, 258), (3, 515), (520, 516), (515, 1030), (530, 1542), (3, 2051), (514, 4100), (513, 4612), (513, 5125), (2, 33001)])
def test_norm(rows, C, unit, dtype):
    import torch
    x, res, gain = make_rows(np.random.default_rng(C + unit), rows, C, dtype)
    h = (x.double() + res.double()).to(x.dtype)
    xv, x_flat = placed(x, unit)
    if xv is None:
        pytest.skip("below the type's size")
    rv, _ = placed(res, unit)
    sample = slice(None) if rows < 100 else slice(rows - 20, None)
    for i, out in enumerate((binding.NORM_I8, binding.NORM_I8_ROWS, binding.NORM_MX)):
        sv, s_flat = placed(torch.zeros_like(x), unit)
        codes = None
        if out != binding.NORM_MX:                           # from an odd address on
            store = torch.full((rows * C + 16,), 99, dtype=torch.int8, device="cuda")
            codes = store[1 + i:1 + i + rows * C].view(rows, C)
        got, scales = binding.qrmsnorm(xv, gain.cuda(), EPS, residual=rv, sum_out=sv, out=out, e=-5, codes=codes, layout=binding.MX_ROWS)
        assert torch.equal(sv.cpu(), h)
        assert (around(sv, s_flat) == MARK).all()
        if codes is not None:
            assert (store[:1 + i] == 99).all() and (store[1 + i + rows * C:] == 99).all()
        check(out, got[sample], None if scales is None else scales.view(rows, -1)[sample] if out == binding.NORM_MX else scales[sample],
              h[sample], gain, e=-5, layout=binding.MX_ROWS)
    assert (around(xv, x_flat) == MARK).all()


@pytest.mark.parametrize("start", [1, 2, 3])
@pytest.mark.parametrize("rows,C", [(1, 5), (9, 64), (700, 101), (3, 1023), (600, 1025), (2, 40001)])
def test_norm_codes_from_any_address(rows, C, start):
    """Aligned rows, int8 codes that are not."""
    import torch
    width = -(-C // 32) * 32
    x, _, gain = make_rows(np.random.default_rng(C), rows, width, "bfloat16")
    x, gain = x[:, :C], gain[:C].contiguous()
    xd = torch.zeros((rows, width), dtype=x.dtype, device="cuda")
    xd[:, :C] = x
    store = torch.full((rows * C + 16,), 99, dtype=torch.int8, device="cuda")
    codes, scales = binding.qrmsnorm(xd[:, :C], gain.cuda(), EPS, out=binding.NORM_I8_ROWS, codes=store[start:start + rows * C].view(rows, C))
    assert (store[:start] == 99).all() and (store[start + rows * C:] == 99).all()
    check(binding.NORM_I8_ROWS, codes[-20:], scales[-20:], x[-20:], gain)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("heads,D", [(3, 16), (2, 40), (3, 48), (5, 72), (3, 80), (7, 96), (5, 112), (1, 160), (3, 176), (2, 208), (1, 400), (1, 496)])
@pytest.mark.parametrize("unit", [2, 4, 8, 32])
def test_cache_heads(heads, D, unit, fmt, dtype):
    import torch
    rng = np.random.default_rng(heads * 1000 + D)
    rows, slots_n = 70, 90
    k, v = values(rng, (rows, heads, D), dtype), values(rng, (rows, heads, D), dtype)
    slots = rng.permutation(slots_n)[:rows].astype(np.int64)
    slots[[0, 33, 69]] = [-1, slots_n, -5]
    kept = (slots >= 0) & (slots < slots_n)
    kv, _ = placed(k.view(rows, -1), unit)
    vv, _ = placed(v.view(rows, -1), unit)
    if kv is None:
        pytest.skip("below the type's size")
    cache = binding.QCache.empty(slots_n, heads, D, FORMATS[fmt])
    for t in cache._keep:
        t.fill_(0x35)
    cache.write(torch.from_numpy(slots).cuda(), kv.unflatten(1, (heads, D)), vv.unflatten(1, (heads, D)))
    ko, k_flat = placed(torch.full((rows, heads * D), 5.0, dtype=k.dtype), unit)
    vo, v_flat = placed(torch.full((rows, heads * D), 5.0, dtype=k.dtype), unit)
    cache.read(torch.from_numpy(slots).cuda(), ko.unflatten(1, (heads, D)), vo.unflatten(1, (heads, D)))
    for x, codes, scales, out, flat in ((k, cache.k_codes, cache.k_scales, ko, k_flat), (v, cache.v_codes, cache.v_scales, vo, v_flat)):
        c, s, want = expect(x.double().numpy(), fmt)
        want_c, want_s = np.full(codes.shape, 0x35, np.uint8), np.full(scales.shape, 0x35, np.uint8)
        want_c[slots[kept]], want_s[slots[kept]] = c[kept], s[kept]
        assert np.array_equal(scales.cpu().numpy(), want_s)
        assert np.array_equal(codes.cpu().numpy(), want_c)
        want[~kept] = 5.0
        assert np.array_equal(out.double().cpu().numpy(), want.reshape(rows, -1))
        assert (around(out, flat) == MARK).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D", [5, 40, 77, 100])
def test_cache_heads_of_padded_rows(D, fmt, dtype):
    """Aligned heads whose codes are not."""
    import torch
    rng = np.random.default_rng(D)
    rows, heads = 40, 3
    k = values(rng, (rows, heads, D), dtype)
    padded = torch.full((rows, heads, 128), 5.0, dtype=k.dtype, device="cuda")
    padded[:, :, :D] = k.cuda()
    cache = binding.QCache.empty(rows, heads, D, FORMATS[fmt])
    slots = torch.from_numpy(rng.permutation(rows)).cuda()
    cache.write(slots, padded[:, :, :D], padded[:, :, :D])
    c, s, want = expect(k.double().numpy(), fmt)
    for codes, scales in ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales)):
        assert np.array_equal(codes[slots].cpu().numpy(), c)
        assert np.array_equal(scales[slots].cpu().numpy(), s)
    out = torch.full((2, rows, heads, 128), 7.0, dtype=k.dtype, device="cuda")
    cache.read(slots, out[0, :, :, :D], out[1, :, :, :D])
    for got in out:
        assert np.array_equal(got[:, :, :D].double().cpu().numpy(), want)
        assert (got[:, :, D:] == 7.0).all()
