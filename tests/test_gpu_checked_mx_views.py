"""The checked build over the codec, norm and cache kernels on views: parts of a joint projection, heads far apart and repeated
(strides of 0), sums in place, gains at odd addresses, outputs at odd addresses.  A process of its own, as it loads another library."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = r'''
import sys
sys.path.insert(0, %r)
import numpy as np, torch
from oracle import mx_ref
from paper_1805_07941_b200 import binding
binding.LIB_PATH = binding.CHECKED_LIB_PATH
assert binding.qconv_checked_faults()[0] == 0
rng = np.random.default_rng(9)
types = (torch.float32, torch.bfloat16, torch.float16)
def make(shape, dt):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dt).cuda()
for heads, D in ((1, 48), (2, 80), (3, 96), (2, 112), (4, 128), (1, 33), (2, 520)):
    for dt in types:
        for fmt in (0, 1):
            for shift in (0, 1):
                joint = make((9, 4 * heads * D + 1), dt)[:, shift:shift + 4 * heads * D].unflatten(1, (4, heads, D))
                cache = binding.QCache.empty(16, heads, D, fmt)
                slots = torch.from_numpy(rng.permutation(16)[:9].astype(np.int64)).cuda()
                cache.write(slots, joint[:, 1], joint[:, 3])
                out = torch.zeros((9, 2 * heads * D + 1), dtype=dt, device="cuda")[:, shift:shift + 2 * heads * D].unflatten(1, (2, heads, D))
                cache.read(slots, out[:, 0], out[:, 1])
                plain = binding.QCache.empty(16, heads, D, fmt)
                plain.write(slots, joint[:, 1].contiguous(), joint[:, 3].contiguous())
                assert torch.equal(plain.k_codes, cache.k_codes) and torch.equal(plain.v_scales, cache.v_scales)
                want = torch.zeros((9, heads, D), dtype=dt, device="cuda"), torch.zeros((9, heads, D), dtype=dt, device="cuda")
                plain.read(slots, *want)
                assert torch.equal(want[0], out[:, 0]) and torch.equal(want[1], out[:, 1])
                alone = binding.QCache.empty(16, heads, D, fmt, values=False)
                alone.write(slots, joint[:1, 0, :1].expand(9, heads, D))        # one head for all
                assert (alone.k_codes[slots] == alone.k_codes[slots[0], 0]).all()
for rows, C in ((1, 4096), (5, 1155), (40, 640), (3, 16384), (2, 20001), (600, 1026), (130, 30)):
    for dt in types:
        x, r = make((rows, C), dt), make((rows, C), dt)
        gain = (1 + 0.1 * make((C + 1,), dt))[1:]
        for out in (0, 1, 2):
            want_sum = torch.empty_like(x)
            want = binding.qrmsnorm(x, gain, 1e-6, residual=r, sum_out=want_sum, out=out, e=-5)
            a, b = x.clone(), r.clone()
            got = [binding.qrmsnorm(a, gain, 1e-6, residual=r, sum_out=a, out=out, e=-5), binding.qrmsnorm(x, gain, 1e-6, residual=b, sum_out=b, out=out, e=-5)]
            assert torch.equal(a, want_sum) and torch.equal(b, want_sum)
            for c, s in got:
                assert torch.equal(c, want[0]) and (s is None or torch.equal(s, want[1]))
            if out != 2:
                codes = torch.zeros((rows * C + 3,), dtype=torch.int8, device="cuda")[3:]
                binding.qrmsnorm(x, gain, 1e-6, residual=r, out=out, e=-5, codes=codes)
                assert torch.equal(codes.view(rows, C), want[0])
for rows, K in ((7, 257), (130, 96), (1, 4095)):
    for dt in types:
        x = make((rows, 3 * K + 1), dt)[:, K + 1:2 * K + 1]
        for layout in (0, 1):
            c, s = binding.qmx_quantize(x, layout=layout, rule=binding.MX_FLOOR)
            want, sw = binding.qmx_quantize(x.contiguous(), layout=layout, rule=binding.MX_FLOOR)
            assert torch.equal(c, want) and torch.equal(s, sw)
            y = torch.zeros((rows, 3 * K + 1), dtype=dt, device="cuda")
            binding.qmx_dequantize(c, s, K, layout=layout, out=y[:, K + 1:2 * K + 1])
            assert torch.equal(y[:, K + 1:2 * K + 1], binding.qmx_dequantize(c, s, K, layout=layout, dtype=dt)) and not y[:, :K + 1].any()
n, line = binding.qconv_checked_faults()
assert n == 0, "index test failed at kernels line %%d (%%d failures)" %% (line, n)
print("checked build: no index test failed")
''' % ROOT


@pytest.mark.gpu
def test_checked_build_sees_no_out_of_range_access():
    from paper_1805_07941_b200 import binding
    binding.build_library(checked=True)
    r = subprocess.run([sys.executable, "-c", SCRIPT], capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "no index test failed" in r.stdout
