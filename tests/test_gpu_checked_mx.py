"""The checked build (every computed global access of the CUDA-core kernels tests its index first) over the codec, norm and
cache kernels: odd, ragged, strided and padded calls of every form.  A process of its own, as it loads another library."""
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
rng = np.random.default_rng(8)
types = (torch.float32, torch.bfloat16, torch.float16)
for rows, K in ((1, 1), (3, 33), (5, 128), (129, 257), (2, 5001), (40, 640)):
    for dt in types:
        base = torch.from_numpy(rng.standard_normal((rows, K + 3)).astype(np.float32)).to(dt).cuda()
        for x in (base[:, :K], base[:, 1:K + 1], base[:, :K].contiguous()):
            want, s = mx_ref.mx_quantize(x.float().cpu().numpy())
            for layout in (0, 1):
                c, sc = binding.qmx_quantize(x, layout=layout)
                assert np.array_equal(c.cpu().numpy(), mx_ref.pack(want))
                assert np.array_equal(sc.cpu().numpy().reshape(-1), mx_ref.to_tiles(s) if layout else s.reshape(-1))
                out = torch.zeros((rows, K + 1), dtype=dt, device="cuda")[:, 1:]
                binding.qmx_dequantize(c, sc, K, layout=layout, out=out)
                assert np.array_equal(out.double().cpu().numpy(), mx_ref.mx_values(want, s, K))
for rows, C in ((1, 7), (9, 100), (130, 256), (3, 1025), (2, 4096), (2, 16400), (2, 33000), (600, 1100)):
    for dt in types:
        x, r = (torch.from_numpy(rng.standard_normal((rows, C + 1)).astype(np.float32)).to(dt).cuda() for _ in range(2))
        g = torch.ones(C, dtype=dt, device="cuda")
        for a, b in ((x[:, :C], r[:, 1:]), (x[:, :C].contiguous(), r[:, 1:].contiguous())):
            y, _ = mx_ref.rmsnorm((a.double() + b.double()).to(dt).double().cpu().numpy(), np.ones(C), 1e-6)
            for out in (0, 1, 2):
                kept = torch.zeros((rows, C), dtype=dt, device="cuda")
                c, s = binding.qrmsnorm(a, g, 1e-6, residual=b, sum_out=kept, out=out, e=-5)
                if out == 0: assert np.array_equal(c.cpu().numpy(), mx_ref.i8_codes(y, -5))
                if out == 2 and C < 2000:
                    want, sw = mx_ref.mx_quantize(y)
                    assert np.array_equal(c.cpu().numpy(), mx_ref.pack(want)) and np.array_equal(s.cpu().numpy(), mx_ref.to_tiles(sw))
for heads, D in ((1, 1), (3, 7), (2, 64), (8, 80), (3, 200), (1, 1024)):
    for dt in types:
        for fmt in (0, 1):
            cache = binding.QCache.empty(30, heads, D, fmt)
            k, v = (torch.from_numpy(rng.standard_normal((12, heads, D)).astype(np.float32)).to(dt).cuda() for _ in range(2))
            slots = torch.from_numpy(rng.permutation(30)[:12].astype(np.int64)).cuda()
            slots[3], slots[7] = -1, 30
            cache.write(slots, k, v)
            ko, vo = torch.zeros_like(k), torch.zeros_like(v)
            cache.read(slots, ko, vo)
            assert not ko[3].any() and not vo[7].any() and ko[0].any()
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
