"""Pins of the oracle for microscaled tensors (CPU): against the (n, p) codec's oracle, against torch's float types, and
against properties of the definitions."""
import numpy as np
import pytest

from oracle import dynfloat as df
from oracle import mx_ref


def test_values_are_the_four_one_type_in_halves():
    assert mx_ref.VALUES.tolist() == [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


@pytest.mark.parametrize("rule", ["cover", "floor"])
def test_a_block_is_the_np_codec_at_its_scale(rule):
    rng = np.random.default_rng(5)
    x = (rng.standard_normal((40, 96)) * np.exp2(rng.integers(-20, 20, (40, 1)))).astype(np.float32)
    x[3, 5], x[4, 6], x[5, 40] = np.nan, np.inf, -np.inf
    x[7] = 0
    codes, scales = mx_ref.mx_quantize(x, rule)
    for r in range(40):
        for b in range(3):
            e = int(scales[r, b]) - 127
            block = x[r, 32 * b:32 * b + 32]
            # the (4, 1) type's integers are twice the values here
            assert np.array_equal(codes[r, 32 * b:32 * b + 32], df.quantize_np(block, e - 1, 4, 1))
            top = np.abs(block[np.isfinite(block)]).max()
            if top == 0:
                assert e == 0
            elif rule == "cover":
                assert 6 * 2.0**e >= top > 6 * 2.0**(e - 1)
            else:
                assert 4 * 2.0**e <= top < 8 * 2.0**e


def test_scale_bytes_of_torch_agree():
    import torch
    s = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(s).view(torch.float8_e8m0fnu).to(torch.float32).numpy()
    got = mx_ref.mx_values(np.full((256, 32), 2, np.uint8), s[:, None], 1)[:, 0]
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[:255], want[:255].astype(np.float64))


def test_ties_and_borders():
    x = np.zeros((1, 32))
    x[0, :8] = [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    codes, scales = mx_ref.mx_quantize(x)
    assert scales[0, 0] == 127 and codes[0, :8].tolist() == [7, 0, 2, 2, 4, 4, 6, 6]
    for top, e in ((6.0, 0), (np.nextafter(6.0, 7), 1), (3.0, -1), (2.0**-149, -127), (1.0, -2)):
        assert mx_ref.mx_exponent([top], "cover") == e
    for top, e in ((127.0, 0), (127.5, 1), (1.0, -6), (2.0**-149, -126)):
        assert mx_ref.i8_exponent([top]) == e


def test_tiles_and_packing_round_trip():
    rng = np.random.default_rng(6)
    codes = rng.integers(0, 16, (5, 64)).astype(np.uint8)
    assert np.array_equal(mx_ref.unpack(mx_ref.pack(codes)), codes)
    s = rng.integers(0, 255, (200, 7)).astype(np.uint8)
    t = mx_ref.to_tiles(s).reshape(2, 2, 32, 4, 4)
    back = t.transpose(0, 3, 2, 1, 4).reshape(256, 8)
    assert np.array_equal(back[:200, :7], s) and (back[200:] == 127).all() and (back[:, 7:] == 127).all()
