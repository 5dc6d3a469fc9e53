"""Limits of an int8 layer's waits: 0 gives up at once, any other one leaves what was issued the time to end, so that a sound run
never gives up."""
import numpy as np
import pytest

from tests.helpers import oracle_conv, rand_layer

pytestmark = pytest.mark.gpu


# a 3x3 layer, one on pairs of SMs, one that splits its contraction
@pytest.mark.parametrize("shape,hints", [((2, 28, 28, 64, 64, 3), {}), ((4, 28, 28, 256, 256, 1), dict(pair_tiles=1)), ((1, 7, 7, 512, 512, 3), dict(split_k=4))])
def test_small_limits(shape, hints):
    import torch
    from paper_1805_07941_b200 import binding
    N, H, W, C, K, R = shape
    pad = (R // 2, R // 2)
    x, w, bias, shift, _, _ = rand_layer(np.random.default_rng(sum(shape)), N, H, W, C, K, R, R, pad=pad)
    want = torch.from_numpy(oracle_conv(x, w, bias, shift, None, None, R=R, S=R, pad=pad)).cuda()
    xd, y = torch.from_numpy(x).cuda(), torch.empty_like(want)
    with binding.plan_hints(**hints):
        conv = binding.QConv(w, bias, shift, None, None, N=N, H=H, W=W, C=C, K=K, R=R, S=R, pad_h=pad[0], pad_w=pad[1])
    for limit in (1, 2, 5, 40, 1 << 16, 0, 1, 1 << 22):
        conv.set_wait_limit(limit)
        y.fill_(77)
        conv.run(xd, y)
        if limit == 0:
            assert conv.status() == binding.ERR_TIMEOUT
        else:
            assert conv.status() == 0 and torch.equal(y, want), (limit, conv.describe())
