"""The trainer-side operators around the flat shard, as cases to measure:

  embed        scaled rows of the embedding table for a list of tokens;
  embed_grad   the table's gradient, rows summed by token;
  ce           per-token loss -log softmax(scale * h W^T)[target] over a large
               vocabulary, with the log-sum-exp that its gradient needs;
  ce_both      the same and then the gradients of h and W for one weight per
               token's loss (the form of a policy gradient);
  orth         a batch of matrices orthogonalised by Newton-Schulz products;
  muon         one Muon step of a batch of matrices: momentum, the
               orthogonalised update, the weights.

Tokens outside the vocabulary and targets outside it are padding: they give a
zero row, no loss and no gradient, whatever their states hold.

Vocabulary, hidden and matrix sizes are those of the workloads in `synth` and
of the framework's tests (151936 x 4096 and x 2048, 6002 x 1001, 1000 x 256;
matrices 4096 x 4096, 12288 x 4096, 768 x 2048, 704 x 256).
"""
import math

import torch

own = False

# the quintic of the Muon optimiser, x -> a x + b x^3 + c x^5 on the singular
# values, the same in every iteration
QUINTIC = (3.4445, -4.7750, 2.0315)
STEPS, EPS = 5, 1e-7

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # rows for the tokens of one decoding step of the smallest model
        dict(name="embed_decode", op="embed", tokens=16, vocab=1000, hidden=256, dtype="bf16",
             scale=1.0, padding=0.0),
        # a training batch of 16384 tokens, rows scaled by sqrt(hidden)
        dict(name="embed_8b", op="embed", tokens=16384, vocab=151936, hidden=4096, dtype="bf16",
             scale=64.0, padding=0.02),
        # an odd table in 32 bits: rows begin at any 4-byte address; the
        # gradient of a second micro-batch is added to that of the first
        dict(name="embed_grad_odd", op="embed_grad", tokens=3001, vocab=6002, hidden=1001,
             dtype="f32", out="f32", scale=31.6, padding=0.1, accumulate=True),
        # the training batch's gradient, written densely for the optimizer
        dict(name="embed_grad_8b", op="embed_grad", tokens=16384, vocab=151936, hidden=4096,
             dtype="bf16", out="f32", scale=64.0, padding=0.02, accumulate=False),
        # log-probability of one sampled token: the smallest call, all of it
        # reading the weights
        dict(name="ce_one_token", op="ce", tokens=1, vocab=151936, hidden=4096, scale=1.0,
             padding=0.0),
        # log-probabilities of a decoding batch at a sampling temperature
        dict(name="ce_decode_64", op="ce", tokens=64, vocab=151936, hidden=2048, scale=1.25,
             padding=0.0),
        # odd everything, a third of the tokens padding
        dict(name="ce_both_odd", op="ce_both", tokens=301, vocab=6002, hidden=1001, scale=1.0,
             padding=0.33, out="f32", accumulate=True),
        # a micro-batch of the 2048-wide model, the weight's gradient in 32 bits
        dict(name="ce_both_30b", op="ce_both", tokens=2048, vocab=151936, hidden=2048, scale=1.0,
             padding=0.1, out="f32", accumulate=False),
        # the largest: a training batch of the 4096-wide model
        dict(name="ce_both_8b", op="ce_both", tokens=8192, vocab=151936, hidden=4096, scale=1.0,
             padding=0.1, out="bf16", accumulate=False),
        # one MLP matrix of the smallest model, taller than wide: launches
        dict(name="orth_small", op="orth", batch=1, rows=704, cols=256, dtype="f32", rank=0.25),
        # one layer's 128 expert matrices
        dict(name="orth_experts", op="orth", batch=128, rows=768, cols=2048, dtype="bf16",
             rank=0.5),
        # the whole optimizer step of one attention projection
        dict(name="muon_q_proj", op="muon", batch=1, rows=4096, cols=4096, rank=0.25,
             nesterov=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size between lo and hi, odd ones and multiples of 64 among them."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.35 else max(64, n // 64 * 64)


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "ce", "ce_both", "ce_both", "orth", "orth", "muon"])
    if op in ("embed", "embed_grad"):
        c = dict(op=op, tokens=_log_int(rng, 1, 16384), vocab=_log_int(rng, 1000, 151936),
                 hidden=_size(rng, 256, 4096), dtype=rng.choice(["bf16", "f32"]),
                 scale=rng.choice([1.0, 22.6]), padding=rng.choice([0.0, 0.1]))
        if op == "embed_grad":
            c.update(accumulate=rng.random() < 0.5)
            c.update(out="f32" if c["accumulate"] else rng.choice(["bf16", "f32"]))
        return c
    if op in ("ce", "ce_both"):
        c = dict(op=op, tokens=_log_int(rng, 1, 8192), vocab=_log_int(rng, 1000, 151936),
                 hidden=_size(rng, 256, 4096), scale=rng.choice([1.0, 1.25]),
                 padding=rng.choice([0.0, 0.1, 0.5]))
        if op == "ce_both":
            c.update(out=rng.choice(["bf16", "bf16", "f32"]))
            c.update(accumulate=c["out"] == "f32" and rng.random() < 0.5)
        return c
    rows, cols = _size(rng, 128, 4096), _size(rng, 128, 4096)
    most = max(1, int(2.0e12 / _orth_flops(1, rows, cols)))
    c = dict(op=op, batch=_log_int(rng, 1, min(128, most)), rows=rows, cols=cols,
             rank=rng.choice([0.1, 0.5]))
    if op == "orth":
        c.update(dtype=rng.choice(["bf16", "f32"]))
    else:
        c.update(nesterov=rng.random() < 0.5)
    return c


# ---- inputs ------------------------------------------------------------------

def _tokens(gen, n, vocab, padding):
    """Token ids as text has them: frequency about 1 / rank (ranks spread over
    the vocabulary), a share of them padding (-1)."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    rank = (vocab ** u).long().clamp(1, vocab) - 1
    ids = (rank * 7919 + 13) % vocab
    pad = torch.rand(n, generator=gen, device="cuda") < padding
    return torch.where(pad, torch.full_like(ids, -1), ids)


def _matrices(gen, batch, rows, cols, rank, dtype):
    """Momentum as training leaves it: a few strong directions over noise."""
    r = max(1, int(rank * min(rows, cols)))
    kw = dict(generator=gen, device="cuda")
    decay = torch.arange(1, r + 1, device="cuda", dtype=torch.float32) ** -0.5
    left = torch.randn(batch, rows, r, **kw) * decay
    x = torch.bmm(left, torch.randn(batch, r, cols, **kw))
    x = x + 0.3 * torch.randn(batch, rows, cols, **kw)
    return (x * 1e-4).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1000003 * int(seed) + 17)
    kw = dict(generator=gen, device="cuda")
    s = dict(case)
    op = case["op"]
    if op in ("embed", "embed_grad"):
        s["ids"] = _tokens(gen, case["tokens"], case["vocab"], case["padding"])
        if op == "embed":
            s["table"] = (0.02 * torch.randn(case["vocab"], case["hidden"], **kw)).to(
                TYPES[case["dtype"]])
            return s
        s["grad"] = (1e-3 * torch.randn(case["tokens"], case["hidden"], **kw)).to(
            TYPES[case["dtype"]])
        s["sum"] = (1e-2 * torch.randn(case["vocab"], case["hidden"], **kw)
                    if case["accumulate"] else
                    torch.empty(case["vocab"], case["hidden"], device="cuda",
                                dtype=TYPES[case["out"]]))
        return s
    if op in ("ce", "ce_both"):
        T, V, d = case["tokens"], case["vocab"], case["hidden"]
        w = torch.empty(V, d, device="cuda", dtype=torch.bfloat16)
        for b in range(0, V, 16384):
            w[b:b + 16384] = 0.02 * torch.randn(min(16384, V - b), d, **kw)
        target = _tokens(gen, T, V, case["padding"])
        # normed states that lean towards their target, by anything from
        # nothing (a surprising token) to nearly all of the probability
        lean = 0.25 * torch.rand(T, 1, **kw) * math.sqrt(4096.0 / d)
        h = torch.randn(T, d, **kw) + lean * w[target.clamp(min=0)].float() / 0.02
        h[target < 0] = float("nan")  # what padding holds is nobody's business
        s.update(weight=w, target=target, hidden=h.bfloat16())
        if op == "ce_both":
            s["grad_loss"] = torch.randn(T, **kw) / T  # advantage of each token
            s["sum"] = (1e-5 * torch.randn(V, d, **kw) if case["accumulate"] else
                        torch.empty(V, d, device="cuda", dtype=TYPES[case["out"]]))
        return s
    dims = (case["batch"], case["rows"], case["cols"])
    if op == "orth":
        s["x"] = _matrices(gen, *dims, case["rank"], TYPES[case["dtype"]])
        return s
    s["momentum"] = _matrices(gen, *dims, case["rank"], torch.float32)
    s["grad"] = 1e-4 * torch.randn(*dims, **kw)
    s["p"] = 0.02 * torch.randn(*dims, **kw)
    s.update(lr=1e-5, mu=0.95, weight_decay=0.01,
             update_scale=0.2 * math.sqrt(max(case["rows"], case["cols"])))
    return s


# ---- one pass ----------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2608_00455_amd import train

    op = s["op"]
    if op == "embed":
        return train.embedding(s["table"], s["ids"], scale=s["scale"])
    if op == "embed_grad":
        return train.embedding_grad(s["grad"], s["ids"], s["sum"], scale=s["scale"],
                                    accumulate=s["accumulate"])
    if op == "orth":
        return train.orthogonalise(s["x"], steps=STEPS, coefficients=QUINTIC, eps=EPS)
    if op == "muon":
        hp = train.MuonStep(lr=s["lr"], momentum=s["mu"], nesterov=s["nesterov"],
                            weight_decay=s["weight_decay"], update_scale=s["update_scale"],
                            steps=STEPS, coefficients=QUINTIC, eps=EPS)
        update = train.muon_forward(s["p"], s["momentum"], s["grad"], hp)
        return {"p": s["p"], "momentum": s["momentum"], "update": update}
    loss, lse = train.linear_ce(s["hidden"], s["weight"], s["target"], scale=s["scale"])
    if op == "ce":
        return {"loss": loss, "lse": lse}
    dh, dw = train.linear_ce_grad(s["hidden"], s["weight"], s["target"], lse, s["grad_loss"],
                                  s["sum"], scale=s["scale"], accumulate=s["accumulate"])
    return {"loss": loss, "lse": lse, "grad_hidden": dh, "grad_weight": dw}


def _run_plain(s):
    op = s["op"]
    if op == "embed":
        ids, table = s["ids"], s["table"]
        ok = (ids >= 0) & (ids < table.shape[0])
        rows = table[torch.where(ok, ids, 0)].float() * s["scale"]
        return torch.where(ok[:, None], rows, 0.0).to(table.dtype)
    if op == "embed_grad":
        ids, out = s["ids"], s["sum"]
        ok = (ids >= 0) & (ids < out.shape[0])
        rows = torch.where(ok[:, None], s["grad"].float() * s["scale"], 0.0)
        acc = out if s["accumulate"] else torch.zeros(out.shape, device=out.device)
        acc.index_add_(0, torch.where(ok, ids, 0), rows)
        return acc if acc.dtype == out.dtype else out.copy_(acc)
    if op == "orth":
        return _plain_orth(s["x"].float()).bfloat16()
    if op == "muon":
        mom, g, p = s["momentum"], s["grad"], s["p"]
        mom.copy_(mom * s["mu"] + g)
        o = _plain_orth(g + mom * s["mu"] if s["nesterov"] else mom).bfloat16()
        p.copy_(p * (1.0 - s["lr"] * s["weight_decay"]) -
                o.float() * (s["lr"] * s["update_scale"]))
        return {"p": p, "momentum": mom, "update": o}
    target, W = s["target"], s["weight"].float()
    V = W.shape[0]
    ok = (target >= 0) & (target < V)
    h = torch.where(ok[:, None], s["hidden"].float(), 0.0)
    z = torch.matmul(h, W.t()) * s["scale"]
    top = z.max(dim=1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    at = torch.where(ok, target, 0)[:, None]
    loss = torch.where(ok, lse - z.gather(1, at)[:, 0], 0.0)
    out = {"loss": loss, "lse": torch.where(ok, lse, 0.0)}
    if op == "ce":
        return out
    # the logits' gradient: softmax minus the target's one, by each token's
    # weight
    G = e.div_(total)
    G.scatter_add_(1, at, torch.full_like(at, -1, dtype=torch.float32))
    G.mul_(torch.where(ok, s["grad_loss"], 0.0)[:, None] * s["scale"])
    dw = torch.matmul(G.t(), h)
    out["grad_hidden"] = torch.matmul(G, W).bfloat16()
    out["grad_weight"] = s["sum"].add_(dw) if s["accumulate"] else s["sum"].copy_(dw)
    return out


def _plain_orth(x):
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    a, b, c = QUINTIC
    x = x / (x.square().sum(dim=(1, 2), keepdim=True).sqrt() + EPS)
    for _ in range(STEPS):
        m = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * m + c * torch.bmm(m, m), x)
    return x.transpose(1, 2).contiguous() if tall else x


# ---- the definition in 64 bits -------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        out = torch.zeros(case["tokens"], case["hidden"], device="cuda", dtype=torch.float64)
        at = ((s["ids"] >= 0) & (s["ids"] < case["vocab"])).nonzero()[:, 0]
        out[at] = s["table"][s["ids"][at]].double() * s["scale"]
        return out
    if op == "embed_grad":
        out = (s["sum"].double() if case["accumulate"] else
               torch.zeros(s["sum"].shape, device="cuda", dtype=torch.float64))
        at = ((s["ids"] >= 0) & (s["ids"] < case["vocab"])).nonzero()[:, 0]
        return out.index_add_(0, s["ids"][at], s["grad"][at].double() * s["scale"])
    if op == "orth":
        return _exact_orth(s["x"])
    if op == "muon":
        mom = s["mu"] * s["momentum"].double() + s["grad"].double()
        o = _exact_orth(s["grad"].double() + s["mu"] * mom if case["nesterov"] else mom)
        p = (1.0 - s["lr"] * s["weight_decay"]) * s["p"].double()
        return {"p": p - s["lr"] * s["update_scale"] * o, "momentum": mom, "update": o}
    T, V, d = case["tokens"], case["vocab"], case["hidden"]
    f64 = dict(device="cuda", dtype=torch.float64)
    W = s["weight"].double()
    out = {"loss": torch.zeros(T, **f64), "lse": torch.zeros(T, **f64)}
    both = op == "ce_both"
    if both:
        out["grad_hidden"] = torch.zeros(T, d, **f64)
        out["grad_weight"] = s["sum"].double() if case["accumulate"] else torch.zeros(V, d, **f64)
    rows = ((s["target"] >= 0) & (s["target"] < V)).nonzero()[:, 0]
    for at in rows.split(1024):
        h, t = s["hidden"][at].double(), s["target"][at]
        z = s["scale"] * (h @ W.T)
        lse = torch.logsumexp(z, dim=1)
        out["lse"][at] = lse
        out["loss"][at] = lse - z[torch.arange(len(at), device="cuda"), t]
        if both:
            g = torch.exp(z - lse[:, None])
            g[torch.arange(len(at), device="cuda"), t] -= 1.0
            g *= s["scale"] * s["grad_loss"][at].double()[:, None]
            out["grad_hidden"][at] = g @ W
            out["grad_weight"] += g.T @ h
    return out


def _exact_orth(x):
    """One matrix at a time, the polynomial by Horner's rule on the smaller
    product."""
    a, b, c = QUINTIC
    out = torch.empty(x.shape, device="cuda", dtype=torch.float64)
    for k in range(x.shape[0]):
        y = x[k].double()
        y = y / (torch.linalg.vector_norm(y) + EPS)
        eye = torch.eye(min(y.shape), device="cuda", dtype=torch.float64)
        for _ in range(STEPS):
            q = y @ y.T if y.shape[0] <= y.shape[1] else y.T @ y
            q = a * eye + q @ (b * eye + c * q)
            y = q @ y if y.shape[0] <= y.shape[1] else y @ q
        out[k] = y
    return out


# ---- what a pass cannot do without ---------------------------------------------

def _orth_flops(batch, rows, cols):
    # each iteration: a symmetric product over the long side, a symmetric
    # square, and the full product (a symmetric one costs half)
    m, n = min(rows, cols), max(rows, cols)
    return float(batch) * STEPS * (m * m * n + m * m * m + 2 * m * m * n)


def work(case):
    op = case["op"]
    if op in ("embed", "embed_grad"):
        n, V, d = case["tokens"], case["vocab"], case["hidden"]
        size = 4 if case["dtype"] == "f32" else 2
        if op == "embed":
            return {"bytes": n * (8 + 2 * d * size), "flops": n * d}
        touched = V * (1.0 - (1.0 - 1.0 / V) ** n)  # at most; repeated tokens make it less
        table = 2 * 4 * touched * d if case["accumulate"] else (
            V * d * (4 if case["out"] == "f32" else 2))
        return {"bytes": n * (8 + d * size) + table, "flops": 2 * n * d}
    if op in ("ce", "ce_both"):
        T, V, d = case["tokens"], case["vocab"], case["hidden"]
        if op == "ce":
            return {"bytes": 2 * (T + V) * d + 16 * T, "flops": 2.0 * T * V * d}
        out = V * d * (2 if case["out"] == "bf16" else 8 if case["accumulate"] else 4)
        return {"bytes": 2 * (T + V) * d + 2 * T * d + out + 20 * T, "flops": 6.0 * T * V * d}
    n = case["batch"] * case["rows"] * case["cols"]
    flops = _orth_flops(case["batch"], case["rows"], case["cols"])
    if op == "orth":
        return {"bytes": n * ((4 if case["dtype"] == "f32" else 2) + 2), "flops": flops}
    return {"bytes": n * (5 * 4 + 2), "flops": flops + 8 * n}
