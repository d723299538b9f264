"""A language model on tokens (model.TokenStep): embedding, adapted stack, layer norm and the head's cross entropy as one ZO
step, and the exact gradient of the ends, against the oracle's parts chained in fp64.

Tolerances: the parity bar of the step tests.  fp32 toy graph: L within 1e-4 and a within 1e-3 relative; 16-bit stacks, from
the device's own stack output on: L and a within 2e-2.  The targets are the entries that each row's perturbation raises most,
so that every row's loss moves one way and D is resolvable; that is asserted before a is compared.
"""
import numpy as np
import pytest
import torch

import paper_2607_01125_gb300 as zo
from paper_2607_01125_gb300.model import AdaptedLinear, TokenStep, ZOStep, coefficient_offsets
from oracle import ends, graphs, optim, philox
from synth import normal, random_orthonormal, tensor_seed, workload

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F = 2.0 ** -24


def n64(t):
    return t.detach().cpu().double().numpy()


def _stack(w, n_queries=None):
    dt = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[w.act_dtype]
    specs, lins, bases = w.linears(), [], {}
    for s, off in zip(specs, coefficient_offsets(specs, w.r)):
        key = s.name[:-1] + "q" if s.name[-2:] in (".k", ".v") else s.name
        if key not in bases:
            bases[key] = random_orthonormal(s.d_in, w.r, tensor_seed(w, "U", key), DEV)
        W = normal((s.d_out, s.d_in), tensor_seed(w, "W", s.name), DEV, std=w.weight_std, dtype=dt)
        lins.append(AdaptedLinear(s.name, W, bases[key], s.layer_id, off, w.r))
    step = ZOStep(zo.Context(0), w.kind, lins, w.T, w.act_dtype, eps=w.eps, lr=w.lr, n_queries=n_queries)
    step.C.copy_(normal(tuple(step.C.shape), tensor_seed(w, "C0"), DEV, std=0.05))
    return step


def _ends(w, vocab, tied):
    d = w.d_model
    dt = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[w.act_dtype]
    table = normal((vocab, d), 5, DEV, dtype=dt)
    head = None if tied else normal((vocab, d), 6, DEV, std=2.0 / np.sqrt(d), dtype=dt)
    gain, bias = 1 + 0.2 * normal((d,), 7, DEV), 0.1 * normal((d,), 8, DEV)
    ids = np.random.default_rng(9).integers(0, vocab, w.T)
    ids[3] = -1
    return table, head, gain, bias, torch.as_tensor(ids, device=DEV)


def _raised(H, W, T, b):
    """The entries whose logits block b raises most over the other block."""
    z = H @ W.T
    return (z[:T] - z[T:2 * T] if b == 0 else z[b * T:(b + 1) * T] - z[:T]).argmax(axis=1)


@pytest.mark.parametrize("n_queries", [None, 3])
def test_token_step_of_the_toy_graph(n_queries):
    w = workload("toy_fp32", eps=0.05)
    step = _stack(w, n_queries)
    vocab, scale = 700, 0.5
    table, head, gain, bias, ids = _ends(w, vocab, tied=False)
    model = TokenStep(step, table, head=head, gain=gain, bias=bias, scale=scale)
    seed, query = 11, 2
    C0 = n64(step.C)
    lay = [dict(W=n64(l.W), U=n64(l.U), C=C0[l.offset:l.offset + l.d_out * l.r].reshape(l.d_out, l.r), layer_id=l.layer_id)
           for l in step.linears]
    blocks = None if n_queries is None else [(0.0, 0)] + [(w.eps, q) for q in step.query_ids(query)]
    Yo = graphs.toy_forward(lay, ends.embed(n64(table), ids.tolist(), scale), w.eps, seed, query, store="fp32", blocks=blocks)
    Ho, _, _ = ends.layer_norm(Yo, n64(gain), n64(bias), model.norm_eps)
    t = _raised(Ho, n64(head), w.T, 0 if n_queries is None else 1)
    t[[0, 5]] = -100
    loss, _, L = ends.cross_entropy(Ho, n64(head), t, step.nb)
    out = model.step(ids, torch.as_tensor(t, device=DEV), 1, seed, query)
    torch.cuda.synchronize()
    assert step.ctx.device_status() == 0
    o = n64(out)
    assert np.abs(n64(model.normed) - Ho).max() <= 1e-4 * np.abs(Ho).max()
    assert np.abs(o[:step.nb] - L).max() <= 1e-4 * L.max()
    if n_queries is None:
        want = ends.pair(L, loss, t, w.eps)
        assert abs(want[2]) > 2e-2 * L.max()
        assert abs(o[2] - want[2]) <= 1e-3 * abs(want[2]) and abs(o[3] - want[3]) <= 1e-3 * abs(want[3])
        a, ids_q = [want[3]], [query]
    else:
        a, ids_q = (L[1:] - L[0]) / w.eps, step.query_ids(query)
        assert abs(L[1] - L[0]) > 2e-2 * L.max() / 2
        assert np.abs(o[step.nb:] - a).max() <= 1e-3 * np.abs(a).max()
    # Adam's first step from m = v = 0 carries (1 - beta1) times the mean of a_j Z^(j)
    for l in step.linears:
        g = sum(aj * philox.perturbation(seed, l.layer_id, q, l.d_out, l.r) for aj, q in zip(a, ids_q)) / len(a)
        m = n64(step.m[l.offset:l.offset + l.d_out * l.r]).reshape(l.d_out, l.r)
        assert np.abs(m - (1 - w.beta1) * g).max() <= 2e-3 * (1 - w.beta1) * np.abs(a).max() * 6
    step.ctx.close()


@pytest.mark.parametrize("name,n_queries,tied", [("llama_stack_bf16", None, False), ("opt_stack_fp16", 2, True)])
def test_token_step_of_a_stack(name, n_queries, tied):
    w = workload(name, T=48, n_decoder=1, eps=0.05)
    step = _stack(w, n_queries)
    vocab = 900
    table, head, gain, bias, ids = _ends(w, vocab, tied)
    model = TokenStep(step, table, head=head, gain=gain, bias=bias, scale=0.02 if tied else 1.0)
    W = n64(model.head)
    seed, query = 13, 4
    Hg = n64(model.forward(ids, seed, query))
    Ho, _, _ = ends.layer_norm(n64(model.hidden), n64(gain), n64(bias), model.norm_eps)
    assert np.abs(n64(model._bufs["x"])[3]).max() == 0
    assert np.abs(Hg - Ho).max() <= 1e-2 * np.abs(Ho).max()
    t = _raised(Hg, W, w.T, 0 if n_queries is None else 1)
    t[[1, 2]] = -1
    targets = torch.as_tensor(t.astype(np.int32), device=DEV)
    loss, _, L = ends.cross_entropy(Hg, W, t, step.nb)
    before = step.loss_out
    out = model.loss(targets)
    assert out.data_ptr() != before.data_ptr()                 # the vectors take turns
    step.update(1, seed, query)
    torch.cuda.synchronize()
    assert step.ctx.device_status() == 0
    o = n64(out)
    assert np.abs(o[:step.nb] - L).max() <= 1e-4 * L.max()      # from the same bits: fp32 sums
    a = [(L[0] - L[1]) / (2 * w.eps)] if n_queries is None else (L[1:] - L[0]) / w.eps
    assert abs(a[0]) * w.eps > 1e-2 * L.max()
    assert np.abs(o[3:] - a).max() <= 2e-2 * np.abs(a).max()
    assert torch.isfinite(step.m).all() and float(step.m.abs().max()) > 0

    # the ends' gradient at the first block, from the same forward pass: the head's input as stored
    mean = model.ends_grad(ids, targets)
    dH, dW = ends.cross_entropy_grad(Hg[:w.T], W, t)
    _, dg, db = ends.layer_norm_grad(dH, n64(model.hidden)[:w.T], n64(gain), n64(model._bufs["mean"])[:w.T],
                                     n64(model._bufs["rstd"])[:w.T])
    assert abs(n64(mean)[0] - L[0]) <= 1e-4 * L[0]
    for got, want in ((model.dhead, dW), (model.dgain, dg), (model.dbias, db)):
        assert np.abs(n64(got) - want).max() <= 1e-2 * np.abs(want).max()
    assert (model.dtable is model.dhead) if tied else model.dtable is None
    step.ctx.close()


@pytest.mark.parametrize("tied", [False, True])
def test_gradient_of_the_ends_against_the_formula_and_differences(tied):
    w = workload("toy_fp32")
    vocab, scale = 300, 0.7
    table, head, gain, bias, ids = _ends(w, vocab, tied)
    ctx = zo.Context(0)
    if tied:
        table.mul_(0.1)
    model = TokenStep(None, table, head=head, gain=gain, bias=bias, scale=scale, ctx=ctx)
    t = np.random.default_rng(2).integers(0, vocab, w.T)
    t[7] = -5
    targets = torch.as_tensor(t, device=DEV)
    model.forward(ids)
    mean = model.ends_grad(ids, targets)
    assert torch.equal(mean, model.loss(targets))
    torch.cuda.synchronize()
    assert ctx.device_status() == 0

    E, g, b = n64(table), n64(gain), n64(bias)
    Hd = E if tied else n64(head)
    idl = ids.tolist()

    def L(E, Hd, g, b):
        return ends.cross_entropy(ends.layer_norm(ends.embed(E, idl, scale), g, b, model.norm_eps)[0], Hd, t)[2][0]

    X = ends.embed(E, idl, scale)
    H, m, s = ends.layer_norm(X, g, b, model.norm_eps)
    assert abs(n64(mean)[0] - L(E, Hd, g, b)) <= 1e-5 * L(E, Hd, g, b)
    dH, dW = ends.cross_entropy_grad(H, Hd, t)
    dX, dg, db = ends.layer_norm_grad(dH, X, g, m, s)
    dE = ends.embed_grad(dX, idl, vocab, scale, start=dW if tied else None)
    grads = [(model.dtable, dE), (model.dgain, dg), (model.dbias, db)] + ([] if tied else [(model.dhead, dW)])
    for got, want in grads:
        assert np.abs(n64(got) - want).max() <= 1e-4 * np.abs(want).max()
    # along a direction for each parameter: central differences of the oracle's loss, exact to h^2
    rng, h = np.random.default_rng(3), 1e-5
    dirs = [rng.standard_normal(E.shape), rng.standard_normal(g.shape), rng.standard_normal(b.shape)]

    def moved(k, x):
        P = [E, g, b]
        P[k] = P[k] + x * dirs[k]
        return L(P[0], P[0] if tied else Hd, P[1], P[2])

    for k, got in enumerate((model.dtable, model.dgain, model.dbias)):
        slope = (moved(k, h) - moved(k, -h)) / (2 * h)
        size = np.sqrt((n64(got) ** 2).sum())
        assert abs((n64(got) * dirs[k]).sum() - slope) <= 1e-4 * (abs(slope) + size), k
    ctx.close()


def test_token_step_refuses_what_does_not_fit():
    ctx = zo.Context(0)
    table = torch.zeros(8, 256, device=DEV)
    with pytest.raises(ValueError):
        TokenStep(None, table)
    with pytest.raises(ValueError):
        TokenStep(None, table, head=torch.zeros(9, 256, device=DEV), ctx=ctx)
    step = _stack(workload("toy_fp32"))
    with pytest.raises(ValueError):
        TokenStep(step, table.to(torch.bfloat16))
    with pytest.raises(ValueError):
        TokenStep(step, table).forward(torch.zeros(3, dtype=torch.int64, device=DEV))
    step.ctx.close()
    ctx.close()


def test_the_example_learns():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "token_steps.py")
    spec = importlib.util.spec_from_file_location("token_steps", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    first, second = mod.main()
    assert first[-1] < 0.9 * first[0], (first[0], first[-1])
    assert sum(second[-10:]) / 10 < second[0], (second[0], second[-10:])
