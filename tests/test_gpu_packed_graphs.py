"""Captured passes of packed stacks (ZOStep.pack): a replay takes the sequences that the last pack() gave, or is refused; it never
runs through a plan whose memory has gone to something else."""
import pytest
import torch

import paper_2607_01125_gb300 as zo
from synth import normal
from test_gpu_packed_stack import D, DEV, HEAD, TYPES, stack

pytestmark = pytest.mark.gpu
T = 150


def clutter():
    """Takes and fills whatever small blocks the allocator has to give."""
    return [torch.full((n,), 0x7F, dtype=torch.uint8, device=DEV) for n in (512, 8192, 40000, 70000, 200000) for _ in range(20)]


def captured(ctx, s, x):
    s.forward(x, 3, 5)                                    # buffers and scratch
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        ctx.sync_stream()
        Y = s.forward(x, 3, 5)
    ctx.sync_stream()
    return graph, Y


def test_plans_stay_where_they_are():
    ctx = zo.Context(0)
    s = stack(ctx, "bf16", T)
    where = set()
    for lengths in ([75, 75], [100, 50], [1, 0], [0, 0]):
        s.pack(lengths)
        where.add(s._attention[1].data_ptr())
    assert len(where) == 1
    for n in range(1, 30):                                # plans that no graph holds are not kept
        s.pack([n] * 3 + [1] * n)
    assert len(s._plans) == 1
    ctx.close()


@pytest.mark.parametrize("dt,n_queries", [("bf16", None), ("bf16", 2), ("fp16", None), ("fp32", None)])
@pytest.mark.parametrize("turned", [True, False])
def test_replays_take_the_last_sequences(dt, n_queries, turned):
    ctx = zo.Context(0)
    s = stack(ctx, dt, T, n_queries=n_queries)
    x = normal((T, D), 7, DEV).to(TYPES[dt])
    rope = zo.rope(HEAD, base=500.0) if turned else None
    s.pack([75, 75], rope)
    graph, Y = captured(ctx, s, x)
    first = s.forward(x, 3, 5).clone()
    for lengths in ([100, 50], [30, 20], [0, 150], [149, 0], [75, 75]):
        s.pack(lengths, rope)
        junk = clutter()
        want = s.forward(x, 3, 5).clone()
        attn = s._bufs["attn"].clone()
        Y.fill_(float("nan"))
        s._bufs["attn"][:sum(lengths)].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert ctx.device_status() == 0
        assert torch.equal(Y, want) and torch.equal(s._bufs["attn"], attn)
        for b in range(s.nb):
            assert (attn[b * T + sum(lengths):(b + 1) * T] == 0).all()
        del junk
    assert torch.equal(want, first)
    ctx.close()


def test_replays_with_other_numbers_of_sequences_are_refused():
    ctx = zo.Context(0)
    s = stack(ctx, "bf16", T)
    x = normal((T, D), 7, DEV).to(torch.bfloat16)
    s.pack([75, 75])
    graph, Y = captured(ctx, s, x)
    first = s.forward(x, 3, 5).clone()
    for again in (lambda: s.pack([50, 50, 50]), lambda: s.pack([75, 75], causal=False), lambda: s.pack([])):
        again()
        junk = clutter()
        s._bufs["attn"].fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert ctx.device_status() == -1
        assert (s._bufs["attn"] == 5.0).all()
        s.pack([75, 75])                                  # its own number: taken again
        graph.replay()
        torch.cuda.synchronize()
        assert ctx.device_status() == 0 and torch.equal(Y, first)
        del junk
    # the synthetic mixer beside it, and the graph still packed
    s.pack(None)
    mixer = s.forward(x, 3, 5).clone()
    junk = clutter()
    graph.replay()
    torch.cuda.synchronize()
    assert ctx.device_status() == 0 and torch.equal(Y, first) and not torch.equal(mixer, first)
    assert len(junk) and torch.equal(s.forward(x, 3, 5), mixer)
    ctx.close()


def test_two_graphs_of_two_numbers_of_sequences():
    """Each is taken while the last call had its number, and both plans are kept."""
    ctx = zo.Context(0)
    s = stack(ctx, "bf16", T)
    x = normal((T, D), 7, DEV).to(torch.bfloat16)
    graphs = []
    for lengths in ([75, 75], [50, 50, 50]):
        s.pack(lengths)
        want = s.forward(x, 3, 5).clone()
        graphs.append((lengths, *captured(ctx, s, x), want))
    s.pack([T])
    assert len(s._plans) == 3
    for lengths, graph, Y, want in graphs + graphs[::-1]:
        s.pack(lengths)
        junk = clutter()
        graph.replay()
        torch.cuda.synchronize()
        assert ctx.device_status() == 0 and torch.equal(Y, want)
        del junk
    assert len(s._plans) == 2
    ctx.close()
