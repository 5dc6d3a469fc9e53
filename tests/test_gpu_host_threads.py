"""Calls from host threads of their own, whose first CUDA call they are: handles made, run and dropped there, and run there when
they were made elsewhere."""
import threading

import numpy as np
import pytest

from paper_1805_07941_b200 import binding

pytestmark = pytest.mark.gpu


def in_threads(*works):
    """Each of `works` in a new thread: their results; the first exception is raised here."""
    results, errors = [None] * len(works), []

    def call(i):
        try:
            results[i] = works[i]()
        except BaseException as e:                           # (handed on: a thread's exceptions are warnings otherwise)
            errors.append(e)

    threads = [threading.Thread(target=call, args=(i,)) for i in range(len(works))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    if errors:
        raise errors[0]
    return results


def product(T, N, K):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(T + N + K)
    wc, ws = binding.qmx_quantize(torch.randn((N, K), generator=gen, device="cuda"))
    xc, xs = binding.qmx_quantize(torch.randn((T, K), generator=gen, device="cuda"))
    want = binding.QMXLinear(wc, ws, N, K, dtype=torch.float32).run(xc, xs)
    torch.cuda.synchronize()
    return wc, ws, xc, xs, want


def test_an_exception_of_a_thread_comes_back():
    with pytest.raises(ZeroDivisionError):
        in_threads(lambda: 1, lambda: 1 // 0)


# (on single SMs, shared by a cluster, on pairs with and without bulk stores)
@pytest.mark.parametrize("T,N,K", [(20, 200, 96), (1, 512, 4096), (1000, 5000, 512), (1000, 4999, 512)])
def test_a_products_first_call_is_a_threads_first(T, N, K):
    import torch
    wc, ws, xc, xs, want = product(T, N, K)
    lin = binding.QMXLinear(wc, ws, N, K, dtype=torch.float32)
    y = torch.zeros_like(want)
    torch.cuda.synchronize()
    in_threads(lambda: lin.run(xc, xs, y))
    assert lin.status() == 0 and torch.equal(y, want)

    def made_there():
        mine = binding.QMXLinear(wc, ws, N, K, dtype=torch.float32)
        mine.run(xc, xs, y)
        return mine.status()

    y.zero_()
    torch.cuda.synchronize()
    assert in_threads(made_there) == [0] and torch.equal(y, want)


def test_a_handle_made_in_a_thread_that_is_gone():
    import torch
    wc, ws, xc, xs, want = product(20, 200, 96)
    lin, = in_threads(lambda: binding.QMXLinear(wc, ws, 200, 96, dtype=torch.float32))
    assert torch.equal(lin.run(xc, xs), want) and lin.status() == 0


def test_handles_made_and_dropped_in_four_threads():
    import torch
    wc, ws, xc, xs, want = product(20, 200, 96)
    done = []

    def work():
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                lin = binding.QMXLinear(wc, ws, 200, 96, dtype=torch.float32)
                y = lin.run(xc, xs)
                assert lin.status() == 0 and torch.equal(y, want)
                lin.destroy()
                done.append(1)

    in_threads(*[work] * 4)
    assert len(done) == 80


def test_the_other_operators_first_calls():
    import torch
    x = torch.randn((5, 256), device="cuda")
    gain = torch.ones((256,), device="cuda")
    want = binding.qmx_quantize(x), binding.qrmsnorm(x, gain, 1e-6, out=binding.NORM_I8_ROWS)
    k = x.view(5, 2, 128)
    slots = torch.arange(5, device="cuda")
    torch.cuda.synchronize()

    def cached():
        cache = binding.QCache.empty(8, 2, 128, values=False)
        cache.write(slots, k)
        return cache.read(slots, torch.empty_like(k))[0]

    codec, norm, values = in_threads(lambda: binding.qmx_quantize(x), lambda: binding.qrmsnorm(x, gain, 1e-6, out=binding.NORM_I8_ROWS), cached)
    torch.cuda.synchronize()
    for got, expected in zip(codec + norm, want[0] + want[1]):
        assert torch.equal(got, expected)
    assert torch.equal(values, cached())


def test_a_status_is_waited_for_on_the_handles_device():
    """From another device: the default stream that is waited for is the one of the handle's."""
    import torch
    if torch.cuda.device_count() < 2:
        pytest.skip("needs two devices")
    T, N, K = 8192, 8192, 8192
    wc, ws, xc, xs, want = product(T, N, K)
    lin = binding.QMXLinear(wc, ws, N, K, dtype=torch.float32)
    y = torch.empty_like(want)
    for _ in range(20):
        lin.run(xc, xs, y)
    after = torch.cuda.Event()
    after.record()
    with torch.cuda.device(1):
        assert lin.status() == 0 and after.query()
        assert torch.cuda.current_device() == 1
        with pytest.raises(ValueError):
            lin.run(xc, xs, y)
        lin.destroy()
        assert torch.cuda.current_device() == 1


def test_an_int8_layer_in_a_thread():
    """Made and run there; and a layer made here that first runs there, on an input that it has no tensor map of."""
    import torch
    from tests.helpers import oracle_conv, rand_layer
    rng = np.random.default_rng(4)
    N, H, W, C, K = 2, 14, 14, 64, 64
    x, w, bias, shift, _, _ = rand_layer(rng, N, H, W, C, K, 3, 3, pad=(1, 1))
    want = torch.from_numpy(oracle_conv(x, w, bias, shift, None, None, R=3, S=3, pad=(1, 1))).cuda()
    xd = torch.from_numpy(x).cuda()
    make = lambda: binding.QConv(w, bias, shift, None, None, N=N, H=H, W=W, C=C, K=K, R=3, S=3, pad_h=1, pad_w=1)
    conv = make()
    outs = [torch.zeros_like(want) for _ in range(2)]
    torch.cuda.synchronize()
    in_threads(lambda: conv.run(xd, outs[0]))
    there, = in_threads(make)
    in_threads(lambda: there.run(xd, outs[1]))
    assert conv.status() == 0 and there.status() == 0
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
