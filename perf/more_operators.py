"""What the operators inside a decoder are measured on: rotary positions, and attention over packed sequences with its
gradient -- the work between the adapted linears of a ZO step on tokens, the first-order gradients beside it, and the single
tokens that an adapted model answers with.

Three kinds of case:

* ``rope``       the rotation of the q and k columns of a q/k/v output by each row's position (or back: the gradient), for
                 both signs of a ZO step (the same positions for every evaluation block).
* ``attention``  softmax(scale q k^T) v over packed sequences, causal or not, query heads in groups that share a key and
                 value head; with fewer queries than keys, the new tokens of sequences whose keys lie in the slots of a cache.
* ``grad``       its gradient by q, k and v from the output and the log-sum-exps that the forward pass kept.

Head counts and widths are those of the workloads in ``synth/configs.py`` (32 query heads on 8, 40 on 40, all of 128) and
generic ones.
"""
import math

import torch

own = False

DEV = "cuda:0"
TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BASE = 500000.0
PARTS = (8.0, 1.0, 4.0, 8192)      # factor, low, high, original length


def listed():
    return [
        # q and k of a toy batch: launches and latency count
        dict(name="rope_toy_fp32", kind="rope", dtype="fp32", T=64, n_blocks=2, heads=4, kv_heads=4, head_dim=64, rot=64,
             layout="half", scaling="none", first=0, inverse=False),
        # q and k of both signs of a ZO step on 4096 tokens, long-context frequencies
        dict(name="rope_step", kind="rope", dtype="bf16", T=4096, n_blocks=2, heads=32, kv_heads=8, head_dim=128, rot=128,
             layout="half", scaling="parts", first=0, inverse=False),
        # the gradient of neighbouring pairs in a part of an odd batch's heads, far into a context
        dict(name="rope_back_part", kind="rope", dtype="fp16", T=3001, n_blocks=1, heads=40, kv_heads=40, head_dim=80, rot=32,
             layout="interleaved", scaling="linear", first=100000, inverse=True),
        # a toy batch in fp32
        dict(name="attn_toy_fp32", kind="attention", dtype="fp32", n_seq=2, q_len=64, k_len=64, ragged=False, heads=4,
             kv_heads=4, head_dim=64, causal=True),
        # both signs of a ZO step on 16 sequences of 256 tokens
        dict(name="attn_step", kind="attention", dtype="bf16", n_seq=32, q_len=256, k_len=256, ragged=False, heads=32,
             kv_heads=8, head_dim=128, causal=True),
        # one long prompt
        dict(name="attn_prompt", kind="attention", dtype="bf16", n_seq=1, q_len=8192, k_len=8192, ragged=False, heads=32,
             kv_heads=8, head_dim=128, causal=True),
        # packed sequences of different odd lengths, every head with its own keys
        dict(name="attn_ragged_fp16", kind="attention", dtype="fp16", n_seq=9, q_len=1501, k_len=1501, ragged=True, heads=40,
             kv_heads=40, head_dim=128, causal=True),
        # one new token of one short sequence
        dict(name="attn_token", kind="attention", dtype="bf16", n_seq=1, q_len=1, k_len=300, ragged=False, heads=32,
             kv_heads=8, head_dim=128, causal=True),
        # one new token of each of 48 sequences that differ in length
        dict(name="attn_tokens", kind="attention", dtype="bf16", n_seq=48, q_len=1, k_len=16384, ragged=True, heads=32,
             kv_heads=8, head_dim=128, causal=True),
        # the gradient over 16 sequences of 256 tokens
        dict(name="grad_step", kind="grad", dtype="bf16", n_seq=16, q_len=256, k_len=256, ragged=False, heads=32, kv_heads=8,
             head_dim=128, causal=True),
        # the gradient over one long sequence
        dict(name="grad_prompt", kind="grad", dtype="bf16", n_seq=1, q_len=4096, k_len=4096, ragged=False, heads=32,
             kv_heads=8, head_dim=128, causal=True),
        # the gradient over ragged sequences that see all of themselves, narrow heads
        dict(name="grad_ragged_fp16", kind="grad", dtype="fp16", n_seq=7, q_len=777, k_len=777, ragged=True, heads=16,
             kv_heads=16, head_dim=80, causal=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _span(case):
    """Sequence lengths (queries, keys): with `ragged`, shares of the longest that spread evenly over 0.05 .. 1."""
    n, lq, lk = case["n_seq"], case["q_len"], case["k_len"]
    if not case["ragged"]:
        return [lq] * n, [lk] * n
    share = [0.05 + 0.95 * ((i + 1) * 0.6180339887 % 1.0) for i in range(n)]
    ks = [max(1, round(lk * s)) for s in share]
    return ([max(1, round(lq * s)) for s in share] if lq == lk else [min(lq, k) for k in ks]), ks


def _pairs(case):
    """Visible (query, key) pairs of one head."""
    total = 0
    for q, k in zip(*_span(case)):
        total += sum(max(0, min(k, k - q + i + 1)) for i in range(q)) if case["causal"] else q * k
    return total


def draw(rng):
    kind = rng.choice(["rope", "rope", "attention", "attention", "attention", "grad", "grad"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp16", "fp16", "fp32"])
    if kind == "rope":
        head_dim = rng.choice([128, 64, 80, 96, 2 * rng.randint(8, 128)])
        kv = rng.choice([1, 4, 8, rng.randint(1, 40)])
        heads = kv * rng.choice([1, 1, 4, 5])
        nb = rng.choice([1, 2, 2, 5])
        most = 8192 * 40 * 128                       # the largest listed one
        T = max(1, min(_log(rng, 1, 8192), most // (nb * (heads + kv) * head_dim)))
        rot = head_dim if rng.random() < 0.6 else 2 * rng.randint(1, head_dim // 2)
        return dict(kind=kind, dtype=dtype, T=T, n_blocks=nb, heads=heads, kv_heads=kv, head_dim=head_dim, rot=rot,
                    layout=rng.choice(["half", "interleaved"]), scaling=rng.choice(["none", "linear", "base", "parts"]),
                    first=rng.choice([0, 0, _log(rng, 1, 1000000)]), inverse=rng.random() < 0.4)
    head_dim = rng.choice([128, 128, 64, 96, 8 * rng.randint(2, 16)])
    kv = rng.choice([1, 2, 8, 8, rng.randint(1, 16)])
    heads = kv * rng.choice([1, 1, 4, 4, 5, 8])
    if dtype == "fp32":                              # the toy's range
        head_dim, kv, heads = min(head_dim, 64), min(kv, 4), min(kv, 4) * rng.choice([1, 2])
    c = dict(kind=kind, dtype=dtype, n_seq=0, q_len=0, k_len=0, ragged=rng.random() < 0.6, heads=heads, kv_heads=kv,
             head_dim=head_dim, causal=rng.random() < 0.75)
    form = rng.choice(["packed", "packed", "tokens", "chunk"]) if kind == "attention" else "packed"
    if form == "packed":
        top = 1024 if dtype == "fp32" else 4096
        c["q_len"] = c["k_len"] = _log(rng, 1, top)
        c["n_seq"] = max(1, min(_log(rng, 1, 64), 8192 // c["q_len"]))
        work = 2 ** 37 if kind == "attention" else 2 ** 35         # the largest listed ones
        while _pairs(c) * heads * head_dim > work:
            c["q_len"] = c["k_len"] = c["q_len"] * 3 // 4
    else:
        c["k_len"] = _log(rng, 1, 16384)
        c["q_len"] = 1 if form == "tokens" else min(_log(rng, 2, 300), c["k_len"])
        if c["q_len"] == c["k_len"]:
            c["ragged"] = False
        size = kv * head_dim * (4 if dtype == "fp32" else 2) * 2
        c["n_seq"] = max(1, min(_log(rng, 1, 48), 48 * 8192 * 4096 // (size * c["k_len"])))
        while _pairs(c) * heads * head_dim > 2 ** 36 and c["n_seq"] > 1:
            c["n_seq"] = c["n_seq"] // 2
    return c


# ---- inputs ----
def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + salt) & 0x7FFFFFFFFFFFFFFF)
    return g


def _randn(g, *shape, std=1.0):
    return torch.randn(*shape, generator=g, device=DEV).mul_(std)


def _data(g, rows, heads, d, dt, std=1.0):
    """[rows, heads d]: channels of different size, and a part that all of a head's rows share."""
    x = torch.empty(rows, heads * d, dtype=dt, device=DEV)
    size = std * torch.exp(0.4 * _randn(g, heads * d))
    common = 0.3 * _randn(g, heads * d)
    step = max(1, (1 << 27) // (heads * d))
    for r in range(0, rows, step):
        n = min(step, rows - r)
        x[r:r + n] = ((_randn(g, n, heads * d) + common) * size).to(dt)
    return x


def _layout(case):
    """(first query row, queries, first key row, keys) of every sequence, and the numbers of rows."""
    qs, ks = _span(case)
    slots = case["q_len"] != case["k_len"]           # new tokens against a cache: slots of one capacity
    out, q0, k0 = [], 0, 0
    for q, k in zip(qs, ks):
        out.append((q0, q, k0, k))
        q0 += q
        k0 += case["k_len"] + 16 if slots else k
    return out, q0, k0


def prepare(case, seed):
    dt = TORCH[case["dtype"]]
    g = _gen(seed, 23)
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    s = {"case": case}
    if case["kind"] == "rope":
        rows = case["T"] * case["n_blocks"]
        s["qkv"] = _data(g, rows, h + 2 * hk, d, dt)
        # sequences packed one after another, each counted from its own first position
        n = case["T"]
        s["pos"] = case["first"] + torch.arange(n, device=DEV) % max(1, int(1 + 0.7 * n))
        s["Y"] = torch.empty(rows, (h + hk) * d, dtype=dt, device=DEV)
        if own:
            import paper_2607_01125_gb300 as zo

            s["ctx"] = _ctx(zo)
            factor, low, high, length = PARTS
            s["rope"] = zo.rope(case["rot"], base=BASE, layout=case["layout"], scaling=case["scaling"], factor=factor, low=low,
                                high=high, original=length)
        return s
    spans, nq, nk = _layout(case)
    s["spans"] = spans
    std = 1.0 if case["kind"] == "attention" else 0.8
    if nq == nk:                                     # columns of one q/k/v output
        qkv = _data(g, nq, h + 2 * hk, d, dt, std)
        s["q"], s["k"], s["v"] = qkv[:, :h * d], qkv[:, h * d:(h + hk) * d], qkv[:, (h + hk) * d:]
    else:
        s["q"], s["k"], s["v"] = _data(g, nq, h, d, dt, std), _data(g, nk, hk, d, dt, std), _data(g, nk, hk, d, dt, std)
    s["O"] = torch.empty(nq, h * d, dtype=dt, device=DEV)
    s["lse"] = torch.empty(nq, h, device=DEV)
    if case["kind"] == "grad":
        # what the forward pass kept
        o, lse = _forward(s, torch.float32)
        s["O"].copy_(o)
        s["lse"].copy_(lse)
        s["dO"] = _data(g, nq, h, d, dt, 0.1)
        s["grads"] = torch.empty(nq, (h + 2 * hk) * d, dtype=dt, device=DEV)
    if own:
        import paper_2607_01125_gb300 as zo

        s["ctx"] = _ctx(zo)
        grad = case["kind"] == "grad"
        s["shape"] = zo.attention_shape(nq, nk, len(spans), h, hk, d, causal=case["causal"])
        s["plan"] = torch.empty(zo.zoact_attention_plan_bytes(s["ctx"], s["shape"], grad=grad), dtype=torch.uint8, device=DEV)
        zo.zoact_attention_plan(s["ctx"], s["shape"], torch.tensor(spans, dtype=torch.int32, device=DEV), s["plan"], grad=grad)
    return s


# ---- the plain forms ----
def _frequencies(case):
    """Radians a position, of each pair."""
    rot = case["rot"]
    factor, low, high, length = PARTS
    base = BASE
    if case["scaling"] == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "parts":
        turns = length * f / (2 * math.pi)
        keep = ((turns - low) / (high - low)).clamp(0, 1)
        f = f * (keep + (1 - keep) / factor)
    return f


def _plain_rope(s):
    c = s["case"]
    rows, d, rot = c["T"] * c["n_blocks"], c["head_dim"], c["rot"]
    angle = s["pos"].double()[:, None] * _frequencies(c)      # far positions: 64 bits until the sine
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    if c["inverse"]:
        sin = -sin
    x = s["qkv"][:, :(c["heads"] + c["kv_heads"]) * d].float().view(c["n_blocks"], c["T"], -1, d)
    if c["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    cos, sin = cos[:, None], sin[:, None]
    y = x.clone()
    p, q = a * cos - b * sin, a * sin + b * cos
    if c["layout"] == "half":
        y[..., :rot // 2], y[..., rot // 2:rot] = p, q
    else:
        y[..., 0:rot:2], y[..., 1:rot:2] = p, q
    return {"Y": y.view(rows, -1).to(s["Y"].dtype)}


def _scores(c, q, k):
    """[kv heads, queries x group, keys] scaled products of one sequence, minus infinity where a key is not seen."""
    lq, lk, d = q.shape[0], k.shape[0], c["head_dim"]
    hk, rep = c["kv_heads"], c["heads"] // c["kv_heads"]
    qh = q.view(lq, hk, rep, d).permute(1, 2, 0, 3).reshape(hk, rep * lq, d)
    z = torch.matmul(qh, k.view(lk, hk, d).permute(1, 2, 0)) * (1 / math.sqrt(d))
    if c["causal"]:
        hidden = torch.arange(lk, device=DEV) > torch.arange(lq, device=DEV)[:, None] + (lk - lq)
        z.view(hk, rep, lq, lk).masked_fill_(hidden, -math.inf)
    return qh, z


def _rows(c, x, lq):
    """[kv heads, queries x group, n] back to [queries, heads n]."""
    hk, rep = c["kv_heads"], c["heads"] // c["kv_heads"]
    return x.view(hk, rep, lq, -1).permute(2, 0, 1, 3).reshape(lq, -1)


def _forward(s, t):
    c = s["case"]
    hk, d = c["kv_heads"], c["head_dim"]
    O = torch.zeros(s["q"].shape[0], c["heads"] * d, dtype=t, device=DEV)
    lse = torch.empty(s["q"].shape[0], c["heads"], dtype=t, device=DEV)
    for q0, lq, k0, lk in s["spans"]:
        _, z = _scores(c, s["q"][q0:q0 + lq].to(t), s["k"][k0:k0 + lk].to(t))
        top = z.max(dim=2, keepdim=True).values
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        z = torch.exp(z - top)
        total = z.sum(dim=2, keepdim=True)
        v = s["v"][k0:k0 + lk].to(t).view(lk, hk, d).transpose(0, 1)
        o = torch.matmul(z, v) / torch.where(total > 0, total, torch.ones_like(total))
        O[q0:q0 + lq] = _rows(c, o, lq)
        lse[q0:q0 + lq] = _rows(c, top + torch.log(total), lq)
    return O, lse


def _plain_grad(s):
    c = s["case"]
    h, hk, d = c["heads"], c["kv_heads"], c["head_dim"]
    rep = h // hk
    out = torch.zeros(s["q"].shape[0], (h + 2 * hk) * d, device=DEV)
    for q0, lq, k0, lk in s["spans"]:
        k, v = s["k"][k0:k0 + lk].float(), s["v"][k0:k0 + lk].float()
        qh, z = _scores(c, s["q"][q0:q0 + lq].float(), k)

        def heads(x, n):
            return x.float().view(lq, hk, rep, n).permute(1, 2, 0, 3).reshape(hk, rep * lq, n)

        lse = heads(s["lse"][q0:q0 + lq], 1)
        p = torch.where(z == -math.inf, torch.zeros_like(z), torch.exp(z - lse))
        dO, O = heads(s["dO"][q0:q0 + lq], d), heads(s["O"][q0:q0 + lq], d)
        vh, kh = v.view(lk, hk, d).transpose(0, 1), k.view(lk, hk, d).transpose(0, 1)
        dz = p * (torch.matmul(dO, vh.transpose(1, 2)) - (dO * O).sum(dim=2, keepdim=True)) * (1 / math.sqrt(d))
        out[q0:q0 + lq, :h * d] = _rows(c, torch.matmul(dz, kh), lq)
        out[k0:k0 + lk, h * d:(h + hk) * d] = torch.matmul(dz.transpose(1, 2), qh).transpose(0, 1).reshape(lk, -1)
        out[k0:k0 + lk, (h + hk) * d:] = torch.matmul(p.transpose(1, 2), dO).transpose(0, 1).reshape(lk, -1)
    return _split(c, out.to(s["dO"].dtype))


def _split(c, grads):
    a, b = c["heads"] * c["head_dim"], (c["heads"] + c["kv_heads"]) * c["head_dim"]
    return {"dq": grads[:, :a], "dk": grads[:, a:b], "dv": grads[:, b:]}


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "rope":
        return _plain_rope(s)
    if kind == "grad":
        return _plain_grad(s)
    O, lse = _forward(s, torch.float32)
    return {"O": O.to(s["O"].dtype), "lse": lse}


# ---- the framework's operators ----
_CTX = []


def _ctx(zo):
    """The one library context a program keeps."""
    if not _CTX:
        _CTX.append(zo.Context(0))
    return _CTX[0]


def _run_own(s):
    import paper_2607_01125_gb300 as zo

    c, ctx = s["case"], s["ctx"]
    if c["kind"] == "rope":
        heads = c["heads"] + c["kv_heads"]
        zo.zoact_rope_apply(ctx, s["qkv"][:, :heads * c["head_dim"]], s["pos"], s["rope"], s["Y"], heads, inverse=c["inverse"])
        return {"Y": s["Y"]}
    if c["kind"] == "attention":
        zo.zoact_attention(ctx, s["shape"], s["plan"], s["q"], s["k"], s["v"], s["O"], lse=s["lse"])
        return {"O": s["O"], "lse": s["lse"]}
    out = _split(c, s["grads"])
    zo.zoact_attention_grad(ctx, s["shape"], s["plan"], s["dO"], s["q"], s["k"], s["v"], s["O"], s["lse"], out["dq"],
                            out["dk"], out["dv"])
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without ----
def work(case):
    e = 4 if case["dtype"] == "fp32" else 2
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    if case["kind"] == "rope":
        n = case["T"] * case["n_blocks"] * (h + hk)
        return {"bytes": 2 * n * d * e + 8 * case["T"], "flops": 3 * n * case["rot"]}
    qs, ks = _span(case)
    nq, nk, pairs = sum(qs), sum(ks), _pairs(case)
    if case["kind"] == "attention":
        return {"bytes": (2 * nq * h + 2 * nk * hk) * d * e + 4 * nq * h, "flops": 4 * pairs * h * d}
    return {"bytes": (4 * nq * h + 4 * nk * hk) * d * e + 4 * nq * h, "flops": 10 * pairs * h * d}


# ---- in 64 bits ----
def exact(case, seed):
    s = prepare(case, seed)
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    if case["kind"] == "rope":
        # pairs as complex numbers times exp(i angle)
        rot, n = case["rot"], (h + hk) * case["head_dim"]
        x = s["qkv"][:, :n].double().view(case["n_blocks"], case["T"], h + hk, d)
        turn = torch.polar(torch.ones_like(s["pos"], dtype=torch.float64)[:, None].expand(-1, rot // 2),
                           torch.outer(s["pos"].double(), _frequencies(case)) * (-1 if case["inverse"] else 1))[:, None]
        y = x.clone()
        if case["layout"] == "half":
            z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * turn
            y[..., :rot] = torch.cat([z.real, z.imag], dim=-1)
        else:
            z = torch.view_as_complex(x[..., :rot].reshape(*x.shape[:-1], rot // 2, 2)) * turn
            y[..., :rot] = torch.view_as_real(z).flatten(-2)
        return {"Y": y.view(-1, n)}
    if work(case)["flops"] > 6e12:
        return None
    rep, scale = h // hk, d ** -0.5
    grad = case["kind"] == "grad"
    nq = s["q"].shape[0]
    O = torch.zeros(nq, h, d, dtype=torch.float64, device=DEV)
    lse = torch.full((nq, h), -math.inf, dtype=torch.float64, device=DEV)
    dq, dk, dv = (torch.zeros(nq, m, d, dtype=torch.float64, device=DEV) for m in (h, hk, hk)) if grad else (None,) * 3
    for q0, lq, k0, lk in s["spans"]:
        mask = torch.ones(lq, lk, dtype=torch.bool, device=DEV)
        if case["causal"]:
            mask = mask.tril(lk - lq)
        for head in range(h):
            g = head // rep
            q, k, v = (s[n][r:r + m, i * d:(i + 1) * d].double() for n, r, m, i in
                       (("q", q0, lq, head), ("k", k0, lk, g), ("v", k0, lk, g)))
            z = torch.einsum("qd,kd->qk", q, k) * scale
            if not grad:
                z = z.masked_fill(~mask, -math.inf)
                lse[q0:q0 + lq, head] = torch.logsumexp(z, dim=1)
                O[q0:q0 + lq, head] = torch.einsum("qk,kd->qd", torch.nan_to_num(torch.softmax(z, dim=1)), v)
                continue
            # the gradient for the output and the log-sum-exps as given
            p = torch.exp(z - s["lse"][q0:q0 + lq, head:head + 1].double()) * mask
            do, o = (s[n][q0:q0 + lq, head * d:(head + 1) * d].double() for n in ("dO", "O"))
            dz = p * (torch.einsum("qd,kd->qk", do, v) - torch.einsum("qd,qd->q", do, o)[:, None]) * scale
            dq[q0:q0 + lq, head] = torch.einsum("qk,kd->qd", dz, k)
            dk[k0:k0 + lk, g] += torch.einsum("qk,qd->kd", dz, q)
            dv[k0:k0 + lk, g] += torch.einsum("qk,qd->kd", p, do)
    if grad:
        return {"dq": dq.flatten(1), "dk": dk.flatten(1), "dv": dv.flatten(1)}
    return {"O": O.flatten(1), "lse": lse}
