"""Sizes that do not fit the interface's 32-bit fields are refused in Python: ctypes would cut them, and the call would work on a part
of the tensor.  (CPU: tensors without memory on a device that calls itself current; the library is never reached.)"""
import pytest
import torch

from paper_1805_07941_b200 import binding

WIDE = (1 << 32) + 64                                       # 64 in 32 bits


class Unreachable:
    def __getattr__(self, name):
        raise AssertionError("%s was called" % name)


@pytest.fixture(autouse=True)
def on_meta(monkeypatch):
    monkeypatch.setattr(binding, "_lib", Unreachable())
    monkeypatch.setattr(binding, "_types", {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    monkeypatch.setattr(binding, "_BYTES", (torch.uint8, torch.int8))
    monkeypatch.setattr(binding, "_INT64", torch.int64)
    monkeypatch.setattr(binding, "_empty", torch.empty)
    monkeypatch.setattr(binding, "_current_device", lambda: torch.empty(0, device="meta").get_device())
    monkeypatch.setattr(binding, "_raw_stream", lambda device: 0)


def meta(*shape, dtype=torch.uint8):
    return torch.empty(shape, dtype=dtype, device="meta")


def test_rows_of_more_values_than_an_int_holds():
    with pytest.raises(ValueError):
        binding.qmx_quantize(meta(1, WIDE, dtype=torch.float16))
    with pytest.raises(ValueError):
        binding.qmx_dequantize(meta(1, WIDE // 2), meta(WIDE // 32 * 128), WIDE, dtype=torch.float16)
    for out in (binding.NORM_I8, binding.NORM_I8_ROWS, binding.NORM_MX):
        with pytest.raises(ValueError):
            binding.qrmsnorm(meta(1, WIDE, dtype=torch.float16), meta(WIDE, dtype=torch.float16), 1e-6, out=out)


@pytest.mark.parametrize("change", [dict(e=1 << 40), dict(e=0.5), dict(eps="1"), dict(layout=1 << 33)])
def test_arguments_that_the_structure_cannot_hold(change):
    kw = dict(eps=1e-6, e=0, layout=1)
    kw.update(change)
    with pytest.raises(ValueError):
        binding.qrmsnorm(meta(4, 64, dtype=torch.float32), meta(64, dtype=torch.float32), kw.pop("eps"), out=binding.NORM_I8, **kw)


def test_products():
    with pytest.raises(ValueError):
        binding.QMXLinear(meta(1, WIDE // 2), meta(WIDE // 128 * 512), 1, WIDE)
    with pytest.raises(ValueError):
        binding.QMXLinear(meta(WIDE, 16), meta(WIDE // 128 * 512 + 512), WIDE, 32)
    lin = object.__new__(binding.QMXLinear)
    lin.N, lin.K, lin.dtype, lin._pitch, lin._tiles, lin.handle, lin._run = 8, 32, torch.float16, 16, 512, None, binding._lib.__getattr__
    with pytest.raises(ValueError):
        lin.run(meta(WIDE, 16), meta((WIDE + 127) // 128 * 512), meta(WIDE, 8, dtype=torch.float16))


def test_caches():
    for shape, D in (((2, WIDE, 64), 64), ((2, 1, WIDE), WIDE)):
        with pytest.raises(ValueError):
            binding.QCache(meta(*shape), meta(*shape[:2]), D=D)


def test_a_cache_of_4_bit_codes_needs_the_values_of_a_head():
    """The codes' width is their bytes: taken for D it would be a cache of half as many values, in another layout."""
    with pytest.raises(ValueError, match="needs D"):
        binding.QCache(meta(2, 1, 64), meta(2, 1, 4), fmt=binding.CACHE_MX)
