"""What the operators at the two ends of a language model are measured on: the work around the adapted stack of a ZO step
on tokens, and the exact gradients of the parts that are trained first-order (embedding, final norm, head).

Six kinds of case:

* ``loss``        softmax cross entropy of hidden states against a head over the vocabulary, without keeping the logits:
                  the rows' losses and log-sum-exps and the mean of each evaluation block (a ZO step evaluates the
                  same targets in both signs, so H holds n_blocks * T rows).
* ``loss_grad``   the same for one block, with the gradient of the mean loss by the hidden states and by the head.
* ``norm``        layer norm with gain and bias, and the rows' statistics.
* ``norm_grad``   its gradient by the input, the gain and the bias.
* ``embed``       scaled rows of the embedding table by token id.
* ``embed_grad``  the table's gradient: every row's tokens summed (dense), or added to a gradient that is there already
                  (a tied head's).

Widths are those of the workloads in ``synth/configs.py`` (256, 4096, 5120) and generic ones; the vocabularies are
those of the models these workloads are shaped like, and generic ones down to a few hundred entries.
"""
import math

import torch

own = False

DEV = "cuda:0"
TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-5


def listed():
    return [
        # the toy graph's width with a small odd vocabulary in fp32, both signs: launches and latency count
        dict(name="loss_toy_fp32", kind="loss", dtype="fp32", T=64, n_blocks=2, d=256, vocab=1009, ignored=0.1),
        # one short sequence in both signs: the head is read once for 32 rows
        dict(name="loss_t16", kind="loss", dtype="bf16", T=16, n_blocks=2, d=4096, vocab=128256, ignored=0.0),
        # the loss pair of a ZO step on 2048 tokens
        dict(name="loss_t2048", kind="loss", dtype="bf16", T=2048, n_blocks=2, d=4096, vocab=128256, ignored=0.1),
        # the head and the final norm trained first-order on an odd batch, in fp16
        dict(name="loss_grad_fp16_t333", kind="loss_grad", dtype="fp16", T=333, n_blocks=1, d=5120, vocab=50272,
             ignored=0.05),
        # the same on 2048 tokens of the wide vocabulary
        dict(name="loss_grad_t2048", kind="loss_grad", dtype="bf16", T=2048, n_blocks=1, d=4096, vocab=128256,
             ignored=0.1),
        # the final norm of the toy width
        dict(name="norm_toy_fp32", kind="norm", dtype="fp32", rows=128, n=256),
        # the final norm of both signs of a full step
        dict(name="norm_fp16_t4096", kind="norm", dtype="fp16", rows=8192, n=5120),
        # its gradient on a ragged width
        dict(name="norm_grad_odd", kind="norm_grad", dtype="bf16", rows=777, n=1001),
        # its gradient on a batch of the full width
        dict(name="norm_grad_t4096", kind="norm_grad", dtype="bf16", rows=4096, n=4096),
        # the tokens of a full step
        dict(name="embed_t4096", kind="embed", dtype="bf16", T=4096, d=4096, vocab=128256, padded=0.02),
        # the embedding's own gradient: all of the table is written
        dict(name="embed_grad_t4096", kind="embed_grad", dtype="bf16", T=4096, d=4096, vocab=128256, padded=0.02,
             accumulate=False),
        # a tied table of a small vocabulary: an odd number of tokens, added to the head's gradient
        dict(name="embed_grad_tied_t9001", kind="embed_grad", dtype="fp16", T=9001, d=5120, vocab=8192, padded=0.02,
             accumulate=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["loss", "loss", "loss_grad", "loss_grad", "norm", "norm_grad", "embed", "embed_grad"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if kind in ("loss", "loss_grad"):
        d = rng.choice([256, 4096, 4096, 5120, 8 * rng.randint(16, 640)])
        vocab = rng.choice([128256, 50272, _log(rng, 300, 128256), _log(rng, 300, 128256)])
        rows = _log(rng, 1, 4096 if kind == "loss" else 2048)
        if dtype == "fp32":            # the toy's range
            d, vocab, rows = min(d, 1024), min(vocab, 20000), min(rows, 1024)
        most = 2048 * 128256 * 4096    # the largest listed gradient
        rows = max(1, min(rows, most * (2 if kind == "loss" else 1) // (vocab * d)))
        n_blocks = rng.choice([1, 2, 2, 5]) if kind == "loss" else 1
        return dict(kind=kind, dtype=dtype, T=max(1, rows // n_blocks), n_blocks=n_blocks, d=d, vocab=vocab,
                    ignored=rng.choice([0.0, 0.1, 0.5]))
    if kind in ("norm", "norm_grad"):
        n = rng.choice([256, 4096, 5120, _log(rng, 64, 8192), _log(rng, 64, 8192)])
        rows = min(_log(rng, 1, 8192), 8192 * 5120 // n)
        return dict(kind=kind, dtype=dtype, rows=rows, n=n)
    d = rng.choice([256, 4096, 5120, _log(rng, 64, 5120)])
    c = dict(kind=kind, dtype=dtype, T=_log(rng, 1, 16384), d=d, vocab=rng.choice([128256, 50272, _log(rng, 300, 128256)]),
             padded=rng.choice([0.0, 0.02, 0.3]))
    if kind == "embed_grad":
        c["accumulate"] = rng.random() < 0.5
    return c


# ---- inputs ----
def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + salt) & 0x7FFFFFFFFFFFFFFF)
    return g


def _randn(g, *shape, std=1.0):
    return torch.randn(*shape, generator=g, device=DEV).mul_(std)


def _uniform(g, n):
    return torch.rand(n, generator=g, device=DEV)


def _ids(g, n, vocab, out):
    """Token ids with the frequencies of text (about 1 / rank), a share `out` of them marked -100 (no token)."""
    rank = torch.exp(_uniform(g, n).double() * math.log(vocab + 1)).long() - 1     # 0 .. vocab - 1, density 1 / (1 + rank)
    ids = (rank.clamp_(0, vocab - 1) * 7919 + 13) % vocab                          # frequent ids spread over the table
    return torch.where(_uniform(g, n) < out, torch.full_like(ids, -100), ids)


def prepare(case, seed):
    kind, dt = case["kind"], TORCH[case["dtype"]]
    g = _gen(seed, 11)
    s = {"case": case}
    if kind in ("loss", "loss_grad"):
        T, nb, d, V = case["T"], case["n_blocks"], case["d"], case["vocab"]
        std = 1.25 / math.sqrt(d)                  # logits of an unrelated row have a spread of about 1.25
        W = _randn(g, V, d, std=std).to(dt)
        s["targets"] = _ids(g, T, V, case["ignored"])
        # hidden states of unit RMS that lean towards their target's row to a degree that differs by token, so that
        # losses reach from near log(vocab) to near 0; the blocks differ slightly, as perturbed passes do
        lean = 0.3 * _uniform(g, T)[:, None]
        h = _randn(g, T, d) * torch.sqrt(1 - lean * lean) + lean / std * W[s["targets"].clamp(min=0)].float()
        s["H"] = (h[None] + 0.01 * _randn(g, nb, T, d)).reshape(nb * T, d).to(dt)
        s["W"] = W
        s["loss"] = torch.empty(nb * T, device=DEV)
        s["lse"] = torch.empty(nb * T, device=DEV)
        s["mean"] = torch.empty(nb, dtype=torch.float64, device=DEV)
        if kind == "loss_grad":
            s["dH"], s["dW"] = torch.empty_like(s["H"]), torch.empty_like(W)
    elif kind in ("norm", "norm_grad"):
        rows, n = case["rows"], case["n"]
        scale = torch.exp(0.5 * _randn(g, rows, 1))
        s["X"] = ((_randn(g, rows, n) + 0.3 * _randn(g, 1, n) + 0.1) * scale).to(dt)
        s["gain"], s["bias"] = 1 + 0.1 * _randn(g, n), 0.1 * _randn(g, n)
        s["mean"], s["rstd"] = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        if kind == "norm":
            s["Y"] = torch.empty_like(s["X"])
        else:
            # the statistics that the forward pass kept
            x = s["X"].double()
            m = x.mean(dim=1, keepdim=True)
            s["mean"].copy_(m[:, 0])
            s["rstd"].copy_(1 / torch.sqrt((x - m).square().mean(dim=1) + EPS))
            s["dY"] = (_randn(g, rows, n) + 0.1 * _randn(g, 1, n)).to(dt)
            s["dX"], s["dgain"], s["dbias"] = torch.empty_like(s["X"]), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    else:
        T, d, V = case["T"], case["d"], case["vocab"]
        s["ids"] = _ids(g, T, V, case["padded"])
        s["scale"] = math.sqrt(d)
        if kind == "embed":
            s["E"] = _randn(g, V, d, std=1 / math.sqrt(d)).to(dt)
            s["Y"] = torch.empty(T, d, dtype=dt, device=DEV)
        else:
            s["dY"] = _randn(g, T, d, std=0.01).to(dt)
            s["dE0"] = _randn(g, V, d, std=0.1).to(dt) if case["accumulate"] else None
            s["dE"] = torch.empty(V, d, dtype=dt, device=DEV)
    return s


# ---- the plain forms ----
def _plain_loss(s):
    c = s["case"]
    T, nb = c["T"], c["n_blocks"]
    z = s["H"].float() @ s["W"].float().t()
    top = z.max(dim=1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    t = s["targets"].repeat(nb)
    counted = t >= 0
    row = torch.where(counted, lse - z.gather(1, t.clamp(min=0)[:, None])[:, 0], torch.zeros_like(lse))
    count = counted[:T].sum().clamp(min=1)
    return e, total, t, counted, count, {"loss": row, "lse": lse, "mean": row.view(nb, T).sum(dim=1) / count}


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "loss":
        return _plain_loss(s)[-1]
    if kind == "loss_grad":
        e, total, t, counted, count, out = _plain_loss(s)
        p = e / total
        at = torch.arange(p.shape[0], device=DEV)
        p[at, t.clamp(min=0)] -= 1
        p = p * (counted.float() / count)[:, None]
        out["dH"] = (p @ s["W"].float()).to(s["H"].dtype)
        out["dW"] = (p.t() @ s["H"].float()).to(s["W"].dtype)
        return out
    if kind == "norm":
        x = s["X"].float()
        m = x.mean(dim=1, keepdim=True)
        rstd = 1 / torch.sqrt((x - m).square().mean(dim=1, keepdim=True) + EPS)
        return {"Y": ((x - m) * rstd * s["gain"] + s["bias"]).to(s["X"].dtype), "mean": m[:, 0], "rstd": rstd[:, 0]}
    if kind == "norm_grad":
        x, dy = s["X"].float(), s["dY"].float()
        rstd = s["rstd"][:, None]
        xh = (x - s["mean"][:, None]) * rstd
        u = dy * s["gain"]
        dx = (u - u.mean(dim=1, keepdim=True) - xh * (u * xh).mean(dim=1, keepdim=True)) * rstd
        return {"dX": dx.to(s["X"].dtype), "dgain": (dy * xh).sum(dim=0), "dbias": dy.sum(dim=0)}
    ids = s["ids"]
    if kind == "embed":
        y = s["E"][ids.clamp(min=0)].float() * s["scale"]
        return {"Y": torch.where((ids >= 0)[:, None], y, torch.zeros_like(y)).to(s["E"].dtype)}
    dE = s["dE0"].float() if s["dE0"] is not None else torch.zeros(c["vocab"], c["d"], device=DEV)
    rows = s["dY"].float() * ((ids >= 0).float() * s["scale"])[:, None]
    return {"dE": dE.index_add_(0, ids.clamp(min=0), rows).to(s["dY"].dtype)}


# ---- the framework's operators ----
_CTX = []


def _ctx(zo):
    """The one library context a program keeps."""
    if not _CTX:
        _CTX.append(zo.Context(0))
    return _CTX[0]


def _run_own(s):
    import paper_2607_01125_gb300 as zo

    c = s["case"]
    kind, ctx = c["kind"], _ctx(zo)
    if kind == "loss":
        zo.zoact_ce_loss(ctx, s["H"], s["W"], s["targets"], n_blocks=c["n_blocks"], loss=s["loss"], lse=s["lse"],
                         mean=s["mean"])
        return {"loss": s["loss"], "lse": s["lse"], "mean": s["mean"].float()}
    if kind == "loss_grad":
        zo.zoact_ce_grad(ctx, s["H"], s["W"], s["targets"], dH=s["dH"], dW=s["dW"], loss=s["loss"], lse=s["lse"],
                         mean=s["mean"])
        return {"loss": s["loss"], "lse": s["lse"], "mean": s["mean"].float(), "dH": s["dH"], "dW": s["dW"]}
    if kind == "norm":
        zo.zoact_layer_norm(ctx, s["X"], s["gain"], s["bias"], s["Y"], eps=EPS, mean=s["mean"], rstd=s["rstd"])
        return {"Y": s["Y"], "mean": s["mean"], "rstd": s["rstd"]}
    if kind == "norm_grad":
        zo.zoact_layer_norm_grad(ctx, s["dY"], s["X"], s["gain"], s["mean"], s["rstd"], dX=s["dX"], dgain=s["dgain"],
                                 dbias=s["dbias"])
        return {"dX": s["dX"], "dgain": s["dgain"], "dbias": s["dbias"]}
    if kind == "embed":
        zo.zoact_embed(ctx, s["E"], s["ids"], s["Y"], scale=s["scale"])
        return {"Y": s["Y"]}
    if c["accumulate"]:
        s["dE"].copy_(s["dE0"])        # the same gradient to add to on every pass
    zo.zoact_embed_grad(ctx, s["dY"], s["ids"], s["dE"], scale=s["scale"], accumulate=c["accumulate"])
    return {"dE": s["dE"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without ----
def work(case):
    e = 4 if case["dtype"] == "fp32" else 2
    kind = case["kind"]
    if kind in ("loss", "loss_grad"):
        rows, d, V = case["T"] * case["n_blocks"], case["d"], case["vocab"]
        data, small = (rows + V) * d * e, 8 * case["T"] + 8 * rows + 4 * case["n_blocks"]
        if kind == "loss":
            return {"bytes": data + small, "flops": 2 * rows * V * d}
        return {"bytes": 2 * data + small, "flops": 6 * rows * V * d}
    if kind == "norm":
        rows, n = case["rows"], case["n"]
        return {"bytes": 2 * rows * n * e + 8 * n + 8 * rows, "flops": 7 * rows * n}
    if kind == "norm_grad":
        rows, n = case["rows"], case["n"]
        return {"bytes": 3 * rows * n * e + 12 * n + 8 * rows, "flops": 14 * rows * n}
    T, d, V = case["T"], case["d"], case["vocab"]
    if kind == "embed":
        # a row that several tokens take has to be read once; the expected number of distinct rows
        return {"bytes": (min(T, _distinct(T, V)) + T) * d * e + 8 * T, "flops": T * d}
    if case["accumulate"]:
        # run() begins with a copy of the gradient that is added to; the add itself touches the tokens' rows
        return {"bytes": 2 * V * d * e + T * d * e + 8 * T, "flops": 2 * T * d}
    return {"bytes": V * d * e + T * d * e + 8 * T, "flops": T * d}


def _distinct(T, V):
    """The expected number of distinct ids among T drawn as in _ids: ranks taken together in steps of a twentieth."""
    total, steps = math.log(V + 1), int(math.log(V + 1) / math.log(1.05)) + 1
    edges = [math.exp(total * k / steps) for k in range(steps + 1)]
    return int(sum((b - a) * (1 - math.exp(-T * math.log(b / a) / total / (b - a))) for a, b in zip(edges, edges[1:])))


# ---- in 64 bits ----
def exact(case, seed):
    kind = case["kind"]
    if kind in ("loss", "loss_grad"):
        flops = work(case)["flops"]
        if flops > 8e12:
            return None
    s = prepare(case, seed)
    if kind in ("loss", "loss_grad"):
        T, nb, d, V = case["T"], case["n_blocks"], case["d"], case["vocab"]
        W = s["W"].double()
        t = torch.cat([s["targets"]] * nb)
        keep = t != -100
        count = max(1, int(keep[:T].sum()))
        loss, lse, dH = [], [], []
        dW = torch.zeros(V, d, dtype=torch.float64, device=DEV) if kind == "loss_grad" else None
        for r in range(0, nb * T, 512):
            h, tr, kr = s["H"][r:r + 512].double(), t[r:r + 512], keep[r:r + 512]
            logp = torch.log_softmax(torch.einsum("rd,vd->rv", h, W), dim=1)
            first = torch.einsum("rd,d->r", h, W[0])
            lse.append(first - logp[:, 0])
            pick = torch.nn.functional.one_hot(tr * kr, V) if kind == "loss_grad" else None
            loss.append(-logp[torch.arange(len(tr), device=DEV), tr * kr] * kr)
            if kind == "loss_grad":
                gz = (logp.exp() - pick) * kr[:, None] / count
                dH.append(torch.einsum("rv,vd->rd", gz, W))
                dW += torch.einsum("rv,rd->vd", gz, h)
        loss, lse = torch.cat(loss), torch.cat(lse)
        out = {"loss": loss, "lse": lse, "mean": torch.stack([b.sum() / count for b in loss.chunk(nb)])}
        if kind == "loss_grad":
            out["dH"], out["dW"] = torch.cat(dH), dW
        return out
    if kind in ("norm", "norm_grad"):
        x = s["X"].double()
        n = case["n"]
        gain, bias = s["gain"].double(), s["bias"].double()
        if kind == "norm":
            var, m = torch.var_mean(x, dim=1, correction=0)
            return {"Y": torch.nn.functional.layer_norm(x, (n,), gain, bias, EPS), "mean": m, "rstd": (var + EPS) ** -0.5}
        # the gradient for the statistics as given: those of the rows, rounded
        m, r = s["mean"].double()[:, None], s["rstd"].double()[:, None]
        dy = s["dY"].double()
        xh = r * (x - m)
        c1 = torch.einsum("rn,n->r", dy, gain)[:, None] / n
        c2 = torch.einsum("rn,n,rn->r", dy, gain, xh)[:, None] / n
        return {"dX": r * (dy * gain - c1 - xh * c2), "dgain": torch.einsum("rn,rn->n", dy, xh),
                "dbias": torch.einsum("rn->n", dy)}
    ids = s["ids"]
    real = ids != -100
    if kind == "embed":
        Y = torch.zeros(case["T"], case["d"], dtype=torch.float64, device=DEV)
        Y[real] = s["E"].double()[ids[real]] * s["scale"]
        return {"Y": Y}
    dE = s["dE0"].double() if s["dE0"] is not None else torch.zeros(case["vocab"], case["d"], dtype=torch.float64, device=DEV)
    order = torch.argsort(ids[real], stable=True)
    uniq, counts = torch.unique_consecutive(ids[real][order], return_counts=True)
    sums = torch.cumsum(s["dY"].double()[real][order], dim=0)
    ends = sums[torch.cumsum(counts, 0) - 1] if len(uniq) else sums[:0]
    dE[uniq] += s["scale"] * torch.diff(ends, dim=0, prepend=torch.zeros_like(ends[:1]))
    return {"dE": dE}
