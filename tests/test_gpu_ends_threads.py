"""Two host threads, each with a context and a stream of its own, in the same kernels with launches of different size: what a
kernel is allowed (its dynamic shared memory) belongs to the function, so no call may set it to what that call alone needs.
"""
import sys
import threading

import pytest
import torch

import paper_2607_01125_gb300 as zo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rnd(seed, *shape, dt=torch.float32):
    return torch.randn(*shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV).to(dt)


def _at_once(make, calls):
    """For each of `make`, a thread with a stream and a context of its own that calls fn(*args) = make(context) `calls` times.
    Arguments are as the C ABI takes them, so that the threads are in the library for most of the time.  Returns the statuses
    that were not 0, by thread."""
    raised, bad, start = [], [[] for _ in make], threading.Barrier(len(make))

    def work(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                c = zo.Context(0)
                fn, args = make[k](c)
                bad[k].append(fn(*args))                 # its scratch
                torch.cuda.synchronize()
                start.wait(60)
                for i in range(calls):
                    bad[k].append(fn(*args))
                    if i % 200 == 199:
                        torch.cuda.synchronize()
                torch.cuda.synchronize()
                bad[k].append(c.device_status())
                c.close()
        except Exception as e:                           # noqa: BLE001  (given to the test's thread)
            start.abort()
            raised.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(len(make))]
    interval = sys.getswitchinterval()
    sys.setswitchinterval(1e-5)
    try:
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(interval)
    assert raised == []
    return [sorted({s for s in b if s != 0}) for b in bad]


def test_layer_norm_gradients_of_two_widths_at_once():
    fn, rows, keep = zo.load().zoact_layer_norm_grad, 4, []

    def case(n):
        X, dY = rnd(n, rows, n, dt=torch.bfloat16), rnd(n + 1, rows, n, dt=torch.bfloat16)
        mean, rstd = torch.zeros(rows, device=DEV), torch.ones(rows, device=DEV)
        dX, want = torch.empty_like(X), torch.empty_like(X)
        keep.append((X, dY, mean, rstd, dX, want))

        def args(c, out):
            return (c.handle, dY.data_ptr(), n, X.data_ptr(), zo.DT_BF16, rows, n, n, None, zo.DT_FP32, mean.data_ptr(),
                    rstd.data_ptr(), out.data_ptr(), None, None)

        c = zo.Context(0)
        assert fn(*args(c, want)) == 0
        torch.cuda.synchronize()
        c.close()
        return lambda c: (fn, args(c, dX))

    assert _at_once([case(n) for n in (1024, 2048, 1024, 2048)], 20000) == [[]] * 4
    assert all(torch.equal(k[-1], k[-2]) for k in keep)


def test_embedding_gradients_of_short_and_long_lists_at_once():
    fn, vocab, d, keep = zo.load().zoact_embed_grad, 50, 8, []

    def case(n):
        ids = torch.randint(0, vocab, (n,), generator=torch.Generator(DEV).manual_seed(n), device=DEV)
        dY, dE, want = rnd(n, n, d), torch.empty(vocab, d, device=DEV), torch.empty(vocab, d, device=DEV)
        keep.append((ids, dY, dE, want))

        def args(c, out):
            return (c.handle, dY.data_ptr(), zo.DT_FP32, n, d, ids.data_ptr(), zo.ID_INT64, vocab, 1.0, out.data_ptr(),
                    zo.DT_FP32, 0)

        c = zo.Context(0)
        assert fn(*args(c, want)) == 0
        torch.cuda.synchronize()
        c.close()
        return lambda c: (fn, args(c, dE))

    assert _at_once([case(n) for n in (40, 10000, 50, 9000)], 4000) == [[]] * 4
    assert all(torch.equal(k[-1], k[-2]) for k in keep)
