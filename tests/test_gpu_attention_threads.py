"""Two and more host threads, each with a context and a stream of its own, in the attention kernels and the rotation with calls of
different sizes and types at once: results are those of the calls alone."""
import threading

import pytest
import torch

import paper_2607_01125_gb300 as zo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
CASES = [(torch.bfloat16, 8, 2, 128, [300, 70]), (torch.float16, 4, 4, 64, [1, 513]), (torch.float32, 2, 1, 32, [40, 90]),
         (torch.bfloat16, 2, 2, 200, [130])]


def operands(dt, heads, kv, d, lens):
    n = sum(lens)
    g = torch.Generator(DEV).manual_seed(n)
    qkv = torch.randn(n, (heads + 2 * kv) * d, generator=g, device=DEV).to(dt)
    dO = torch.randn(n, heads * d, generator=g, device=DEV).to(dt)
    return qkv, dO, torch.arange(n, device=DEV), zo.attention_spans(lens).to(DEV)


def chain(ctx, data, case):
    """Rotation, attention and the gradient of one batch; all outputs."""
    dt, heads, kv, d, lens = case
    qkv, dO, pos, spans = data
    n, turned = qkv.shape[0], torch.empty_like(qkv)
    turned.copy_(qkv)
    qk = turned[:, :(heads + kv) * d]
    zo.zoact_rope_apply(ctx, qk, pos, zo.rope(d // 4 * 2), qk, heads + kv)
    q, k, v = turned[:, :heads * d], turned[:, heads * d:(heads + kv) * d], turned[:, (heads + kv) * d:]
    shape = zo.attention_shape(n, n, len(lens), heads, kv, d)
    plan = torch.empty(zo.zoact_attention_plan_bytes(ctx, shape, grad=True), dtype=torch.uint8, device=DEV)
    zo.zoact_attention_plan(ctx, shape, spans, plan, grad=True)
    O, lse, grads = torch.empty_like(dO), torch.empty(n, heads, device=DEV), torch.empty_like(qkv)
    zo.zoact_attention(ctx, shape, plan, q, k, v, O, lse=lse)
    zo.zoact_attention_grad(ctx, shape, plan, dO, q, k, v, O, lse, grads[:, :heads * d], grads[:, heads * d:(heads + kv) * d],
                            grads[:, (heads + kv) * d:])
    return O, lse, grads


def test_contexts_of_several_threads_at_once():
    data = [operands(*c) for c in CASES]
    alone = zo.Context(0)
    want = [chain(alone, x, c) for x, c in zip(data, CASES)]
    torch.cuda.synchronize()
    assert alone.device_status() == 0
    alone.close()
    raised, same = [], [True] * len(CASES)
    start = threading.Barrier(len(CASES))

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                c = zo.Context(0)
                chain(c, data[i], CASES[i])                  # its scratch
                torch.cuda.current_stream().synchronize()
                start.wait(60)
                for _ in range(150):
                    got = chain(c, data[i], CASES[i])
                    same[i] &= all(torch.equal(a, b) for a, b in zip(got, want[i]))
                same[i] &= c.device_status() == 0
                c.close()
        except Exception as e:                               # noqa: BLE001  (given to the test's thread)
            start.abort()
            raised.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(CASES))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert raised == [] and same == [True] * len(CASES)


def test_two_graphs_of_one_context_one_after_another():
    """Graphs of calls of different sizes share the context's scratch; replayed in turn they give what the calls give."""
    ctx = zo.Context(0)
    data = [operands(*c) for c in CASES[:2]]
    want = [chain(ctx, x, c) for x, c in zip(data, CASES)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for x, c in zip(data, CASES):
        g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(g, stream=side):
            ctx.sync_stream()
            outs.append(chain(ctx, x, c))
        graphs.append(g)
    ctx.sync_stream()
    for order in ((0, 1), (1, 0), (0, 0, 1, 1)):
        for o in outs:
            for t in o:
                t.fill_(float("nan"))
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for o, w in zip(outs, want) for a, b in zip(o, w))
    assert ctx.device_status() == 0
    ctx.close()
