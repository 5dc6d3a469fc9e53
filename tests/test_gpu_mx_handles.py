"""Handles of microscaled products: many at once, dropped in any order, made and dropped from several threads."""
import threading

import pytest

from paper_1805_07941_b200 import binding

pytestmark = pytest.mark.gpu


def test_more_handles_than_there_are_status_words():
    import torch
    w, x = torch.randn((32, 64), device="cuda"), torch.randn((3, 64), device="cuda")
    wc, ws = binding.qmx_quantize(w)
    xc, xs = binding.qmx_quantize(x)
    lins = [binding.QMXLinear(wc, ws, 32, 64, dtype=torch.float32) for _ in range(1100)]
    want = lins[0].run(xc, xs)
    for i in (1, 500, 1023, 1024, 1099):
        assert torch.equal(lins[i].run(xc, xs), want) and lins[i].status() == 0
    # a status belongs to its handle alone, and a word that is taken again starts clean
    lins[1023].set_wait_limit(0)
    lins[1023].run(xc, xs)
    assert lins[1022].status() == 0 and lins[1024].status() == 0
    for lin in lins[::-2] + lins[::2]:
        lin.destroy()
    again = [binding.QMXLinear(wc, ws, 32, 64, dtype=torch.float32) for _ in range(1100)]
    assert all(lin.status() == 0 for lin in again)
    assert torch.equal(again[700].run(xc, xs), want)


def test_a_handle_describes_itself_before_its_first_run():
    import torch
    wc, ws = binding.qmx_quantize(torch.randn((32, 64), device="cuda"))
    assert "N=32 K=64" in binding.QMXLinear(wc, ws, 32, 64).describe()


def test_threads():
    import torch
    wc, ws = binding.qmx_quantize(torch.randn((200, 96), device="cuda"))
    xc, xs = binding.qmx_quantize(torch.randn((20, 96), device="cuda"))
    want = binding.QMXLinear(wc, ws, 200, 96, dtype=torch.float32).run(xc, xs)
    torch.cuda.synchronize()
    wrong = []

    def work():
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                lin = binding.QMXLinear(wc, ws, 200, 96, dtype=torch.float32)
                y = lin.run(xc, xs)
                if lin.status() != 0 or not torch.equal(y, want):
                    wrong.append(lin.describe())

    threads = [threading.Thread(target=work) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
