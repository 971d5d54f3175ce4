"""What the operators between the router and the loss are measured on.

The router says which experts each token goes to. From there a training step of an MoE gathers the tokens'
rows by expert and brings them back (``Dispatch``), multiplies each expert's rows with its matrix, and takes the
gradients of rows and matrices (``Experts``), and ends in the softmax cross entropy over the vocabulary of the output
head, which shares the embedding's table (``HeadLoss``). A pass is what a layer's forward or backward
calls of one of them.

A case names its operator (``op``):

* ``spread``: tokens ordered by expert, and their rows written in that order. ``combine``: the rows' weighted sums,
  token by token. ``combine_grad``: the gradients of the rows and of the weights. ``drop``: a share of the
  choices is -1 (no expert); the rows that are left over at the end are zeros.
* ``product``, ``grad_rows``, ``grad``: ``rows`` rows over ``experts`` matrices of n x m, of loads as routers make them; ``drop``: a share of the rows, at the end,
  has no expert. ``base``: the matrices' gradient adds to one that is there.
* ``loss``: the loss of each token. ``head_grad``: that, and the gradients of the activations and of the table.
  ``pad``: a share of the targets is -1, a padded place, without a loss.
"""
import math

import numpy as np
import torch

own = False


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def _tokens(name, op, **kw):
    return {"name": name, "op": op, "tokens": 32768, "k": 2, "experts": 128, "d": 4096, "token32": False, "row32": False, "drop": 0.0, **kw}


def _experts(name, op, **kw):
    return {"name": name, "op": op, "rows": 65536, "experts": 128, "n": 4096, "m": 4096, "out32": False, "base": False, "drop": 0.0, **kw}


def _head(name, op, **kw):
    return {"name": name, "op": op, "tokens": 8192, "vocab": 50304, "d": 4096, "scale": 1.0, "ids64": True, "pad": 0.0, "base": False, **kw}


def listed():
    return [
        # the toy MoE's 8 sequences of 128 tokens: latency
        _tokens("spread_toy", "spread", tokens=1024, experts=8, d=64),
        # the full model's layer: 256 sequences of 128 tokens
        _tokens("spread_full", "spread"),
        # fine-grained experts: 8 of 256
        _tokens("combine_256", "combine", k=8, experts=256, d=2048),
        # an fp32 residual stream of an odd width, an odd number of experts, some choices dropped
        _tokens("combine_grad_127", "combine_grad", tokens=4096, k=4, experts=127, d=1001, token32=True, drop=0.05),
        # eight tokens, two experts each, of the full model: the experts' matrices are read for a row or two
        _experts("product_few", "product", rows=16),
        # the full model's layer, forward
        _experts("product_full", "product"),
        # experts of 4096 x 1024, some rows without an expert: the gradient of the rows
        _experts("grad_rows_slice", "grad_rows", rows=16384, m=1024, drop=0.03),
        # the full model's layer: the gradient of the matrices
        _experts("grad_full", "grad"),
        # an odd matrix, fp32 gradients accumulated over microbatches
        _experts("grad_odd", "grad", rows=5000, experts=9, n=1000, m=511, out32=True, base=True),
        # the toy's head: latency
        _head("loss_toy", "loss", tokens=1024, vocab=512, d=64),
        # width 768, an odd vocabulary, padded sequences: evaluation
        _head("loss_768", "loss", tokens=4096, vocab=50257, d=768, scale=0.5, ids64=False, pad=0.1),
        # the full model's head, 64 sequences of 128 tokens: loss and gradients
        _head("head_grad_full", "head_grad"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    w = _log(rng, lo, hi)
    return w if rng.random() < 0.25 else -(-w // 8) * 8


def draw(rng):
    kind = rng.randrange(3)
    if kind == 0:
        d, experts = _width(rng, 16, 8192), _log(rng, 2, 512)
        k = min(_log(rng, 1, 16), experts)
        return {"op": rng.choice(("spread", "combine", "combine_grad")), "tokens": max(1, min(_log(rng, 1, 131072), (1 << 28) // (d * k))), "k": k,
                "experts": experts, "d": d, "token32": rng.random() < 0.3, "row32": rng.random() < 0.2, "drop": rng.choice((0.0, 0.0, 0.1))}
    if kind == 1:
        n, m = _width(rng, 32, 5000), _width(rng, 32, 5000)
        experts = min(_log(rng, 1, 256), max(1, (1 << 30) // (n * m)))
        op = rng.choice(("product", "grad_rows", "grad"))
        return {"op": op, "rows": _log(rng, 1, 65536), "experts": experts, "n": n, "m": m, "out32": rng.random() < 0.2,
                "base": op == "grad" and rng.random() < 0.4, "drop": rng.choice((0.0, 0.0, 0.1))}
    op = rng.choice(("loss", "head_grad"))
    return {"op": op, "tokens": _log(rng, 1, 8192), "vocab": _log(rng, 256, 50304), "d": _width(rng, 32, 4096), "scale": rng.choice((1.0, 0.5, 2.0)),
            "ids64": rng.random() < 0.6, "pad": rng.choice((0.0, 0.0, 0.1)), "base": op == "head_grad" and rng.random() < 0.4}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
class _State:
    pass


def _dtype(f32):
    return torch.float32 if f32 else torch.bfloat16


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _normal(shape, gen, sigma, f32):
    return torch.empty(shape, dtype=_dtype(f32), device="cuda").normal_(0.0, sigma, generator=gen)


def _ordered(chosen, E):
    """(offsets, places): the choices sorted by expert, stably; -1 where there is none."""
    at = chosen.reshape(-1)
    there = (at >= 0) & (at < E)
    key = torch.where(there, at, E).long()
    by = torch.sort(key, stable=True).indices
    place = torch.empty_like(by).scatter_(0, by, torch.arange(by.numel(), device="cuda"))
    counts = torch.zeros(E + 1, dtype=torch.long, device="cuda").scatter_add_(0, key, torch.ones_like(key))
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.cumsum(counts[:E], 0)
    return offsets, torch.where(there, place, -1).int().view(chosen.shape)


def _token_inputs(c, seed):
    gen, s = _generator(seed), _State()
    T, k, E, d = c["tokens"], c["k"], c["experts"], c["d"]
    liked = torch.randn(E, device="cuda", generator=gen) * 0.5  # some experts draw more tokens
    s.chosen = torch.topk(torch.randn((T, E), device="cuda", generator=gen) + liked, k, dim=-1).indices.int()
    if c["drop"]:
        s.chosen[torch.rand((T, k), device="cuda", generator=gen) < c["drop"]] = -1
    if c["op"] == "spread":
        s.x = _normal((T, d), gen, 1.0, c["token32"])
        return s
    s.order = _ordered(s.chosen, E)
    s.rows = _normal((T * k, d), gen, 1.0, c["row32"])
    w = torch.rand((T, k), device="cuda", generator=gen) + 0.1
    s.weights = w / w.sum(-1, keepdim=True)
    if c["op"] == "combine_grad":
        s.dy = _normal((T, d), gen, 1e-3, c["token32"])
    return s


def _loads(c, seed):
    """Rows of each expert, on the host: some experts draw more."""
    r = np.random.RandomState(int(seed) % (1 << 31))
    p = np.exp(0.5 * r.randn(c["experts"]))
    return r.multinomial(c["rows"] - int(c["rows"] * c["drop"]), p / p.sum())


def _expert_inputs(c, seed):
    gen, s = _generator(seed), _State()
    R, E, n, m = c["rows"], c["experts"], c["n"], c["m"]
    loads = _loads(c, seed)
    s.most = max(1, int(loads.max()))
    s.offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(loads)])).int().cuda()
    s.x = s.w = s.dy = s.base = None
    if c["op"] != "grad_rows":
        s.x = _normal((R, n), gen, 1.0, False)
    if c["op"] != "grad":
        s.w = _normal((E, n, m), gen, 0.02, False)
    if c["op"] != "product":
        s.dy = _normal((R, m), gen, 1e-3, False)
    if c["base"]:
        s.base = _normal((E, n, m), gen, 1e-3, c["out32"])
    return s


def _head_inputs(c, seed):
    gen, s = _generator(seed), _State()
    T, V, d = c["tokens"], c["vocab"], c["d"]
    s.table = _normal((V, d), gen, 0.02, False)
    targets = torch.exp(torch.rand(T, device="cuda", dtype=torch.float64, generator=gen) * math.log(V + 1.0)).long().sub_(1).clamp_(0, V - 1)
    # activations that have learnt something: the target's logit stands out, more for some tokens
    told = torch.rand((T, 1), device="cuda", generator=gen) * (10.0 / (c["scale"] * d * 0.02 ** 2))
    s.h = (torch.randn((T, d), device="cuda", generator=gen) + told * s.table[targets]).to(torch.bfloat16)
    if c["pad"]:
        targets[torch.rand(T, device="cuda", generator=gen) < c["pad"]] = -1
    s.targets = targets if c["ids64"] else targets.int()
    there = s.targets >= 0
    s.dloss = there.float() / there.sum().clamp(min=1)  # the loss's mean over the tokens that have one
    s.base = _normal((V, d), gen, 1e-5, False) if c["base"] else None
    return s


def _inputs(c, seed):
    if c["op"] in ("spread", "combine", "combine_grad"):
        return _token_inputs(c, seed)
    return (_expert_inputs if c["op"] in ("product", "grad_rows", "grad") else _head_inputs)(c, seed)


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    s.c = c
    if own:
        from paper_2607_19058_gb300 import skewadam as S
        if c["op"] in ("spread", "combine", "combine_grad"):
            s.op = S.Dispatch(c["experts"], c["k"], token_dtype=_dtype(c["token32"]), row_dtype=_dtype(c["row32"]))
        elif c["op"] in ("product", "grad_rows", "grad"):
            s.op = S.Experts(c["experts"], c["n"], c["m"], row_dtype=_dtype(c["out32"]), grad_dtype=_dtype(c["out32"]))
        else:
            s.op = S.HeadLoss(c["vocab"], c["d"], scale=c["scale"])
    return s


# ---------------------------------------------------------------------------
# A pass
# ---------------------------------------------------------------------------
def run(state):
    s, c = state, state.c
    op = c["op"]
    if own:
        if op == "spread":
            order = s.op.order(s.chosen)
            return [*order, s.op.spread(s.x, order)]
        if op == "combine":
            return s.op.combine(s.rows, s.weights, s.order)
        if op == "combine_grad":
            return s.op.combine_grad(s.dy, s.rows, s.weights, s.order)
        if op == "product":
            return s.op.product(s.x, s.w, s.offsets)
        if op == "grad_rows":
            return s.op.grad_rows(s.dy, s.w, s.offsets)
        if op == "grad":
            return s.op.grad(s.x, s.dy, s.offsets, base=s.base)
        loss, lse = s.op.loss(s.h, s.table, s.targets)
        if op == "loss":
            return [loss, lse]
        return [loss, lse, *s.op.grad(s.h, s.table, s.targets, lse, s.dloss, base=s.base)]
    if op in ("spread", "combine", "combine_grad"):
        return _plain_tokens(s, c)
    return (_plain_experts if op in ("product", "grad_rows", "grad") else _plain_head)(s, c)


def _plain_tokens(s, c):
    T, k, d = c["tokens"], c["k"], c["d"]
    tok, row = _dtype(c["token32"]), _dtype(c["row32"])
    offsets, places = _ordered(s.chosen, c["experts"]) if c["op"] == "spread" else s.order
    there = (places >= 0)[:, :, None]
    to = torch.where(places >= 0, places, T * k).long().reshape(-1)  # what has no expert goes to a row of its own, which is cut off
    if c["op"] == "spread":
        out = torch.zeros((T * k + 1, d), dtype=row, device="cuda")
        out[to] = s.x.float()[:, None, :].expand(T, k, d).reshape(T * k, d).to(row)
        return [offsets, places, out[:-1]]
    mine = torch.where(there, s.rows[places.clamp(min=0).long()].float(), 0.0)
    if c["op"] == "combine":
        return (mine * s.weights[:, :, None]).sum(1).to(tok)
    dy = s.dy.float()
    dw = (mine * dy[:, None, :]).sum(-1)
    out = torch.zeros((T * k + 1, d), dtype=row, device="cuda")
    out[to] = (s.weights[:, :, None] * dy[:, None, :]).reshape(T * k, d).to(row)
    return out[:-1], dw


def _padded(s, c, x):
    """(experts, most, width) fp32: each expert's rows, and zeros behind them."""
    at = s.offsets[:-1, None].long() + torch.arange(s.most, device="cuda")
    return torch.where((at < s.offsets[1:, None])[:, :, None], x[at.clamp(max=c["rows"] - 1)].float(), 0.0)


def _unpadded(s, c, y):
    r = torch.arange(c["rows"], device="cuda")
    e = torch.searchsorted(s.offsets[1:].long(), r, right=True)
    there = e < c["experts"]
    e = e.clamp(max=c["experts"] - 1)
    return torch.where(there[:, None], y[e, torch.where(there, r - s.offsets[e], 0)], 0.0)


def _plain_experts(s, c):
    out = _dtype(c["out32"])
    if c["op"] == "product":
        return _unpadded(s, c, torch.matmul(_padded(s, c, s.x), s.w.float())).to(out)
    if c["op"] == "grad_rows":
        return _unpadded(s, c, torch.matmul(_padded(s, c, s.dy), s.w.float().transpose(1, 2))).to(out)
    dw = torch.matmul(_padded(s, c, s.x).transpose(1, 2), _padded(s, c, s.dy))
    if s.base is not None:
        dw = dw + s.base.float()
    return dw.to(out)


def _plain_head(s, c):
    h, w = s.h.float(), s.table.float()
    there = (s.targets >= 0) & (s.targets < c["vocab"])
    at = torch.where(there, s.targets, 0).long()[:, None]
    logits = torch.matmul(h, w.t()) * c["scale"]
    top = logits.amax(-1, keepdim=True)
    lse = top + torch.log(torch.exp(logits - top).sum(-1, keepdim=True))
    loss = torch.where(there, (lse - torch.gather(logits, 1, at))[:, 0], 0.0)
    if c["op"] == "loss":
        return [loss, lse[:, 0]]
    p = torch.exp(logits - lse)
    p.scatter_add_(1, at, torch.full_like(lse, -1.0))
    p = p * torch.where(there, s.dloss, 0.0)[:, None]
    dw = torch.matmul(p.t(), h) * c["scale"]
    if s.base is not None:
        dw = dw + s.base.float()
    return [loss, lse[:, 0], (torch.matmul(p, w) * c["scale"]).to(torch.bfloat16), dw.to(torch.bfloat16)]


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    c = case
    op = c["op"]
    if op in ("spread", "combine", "combine_grad"):
        T, k, d = c["tokens"], c["k"], c["d"]
        tok, row, kept = T * d * (4 if c["token32"] else 2), T * k * d * (4 if c["row32"] else 2), 1.0 - c["drop"]
        if op == "spread":  # tokens read once, all rows written
            return {"bytes": tok + row + 8 * T * k + 4 * (c["experts"] + 1), "flops": 4 * T * k}
        if op == "combine":
            return {"bytes": int(kept * row) + tok + 8 * T * k, "flops": int(2 * kept * T * k * d)}
        return {"bytes": tok + int(kept * row) + row + 12 * T * k, "flops": int(3 * kept * T * k * d)}
    if op in ("product", "grad_rows", "grad"):
        R, E, n, m, o = c["rows"], c["experts"], c["n"], c["m"], 4 if c["out32"] else 2
        real = R - int(R * c["drop"])
        # the experts that have a row, for loads that are as even as they can be: what is read of the matrices
        used = E * -math.expm1(real * math.log1p(-1.0 / E)) if E > 1 else min(1, real)
        by = {"product": 2 * real * n + R * m * o + used * 2 * n * m, "grad_rows": 2 * real * m + R * n * o + used * 2 * n * m,
              "grad": 2 * real * (n + m) + E * n * m * o * (2 if c["base"] else 1)}[op]
        return {"bytes": int(by), "flops": 2 * real * n * m}
    T, V, d = c["tokens"], c["vocab"], c["d"]
    by = 2 * T * d + 2 * V * d + 8 * T + T * (8 if c["ids64"] else 4)
    if op == "loss":
        return {"bytes": by, "flops": 2 * T * V * d}
    # logits, and the two gradients' products; a program that does not keep the logits makes them twice, which is not counted
    return {"bytes": by + 4 * T + 2 * T * d + 2 * V * d * (2 if c["base"] else 1), "flops": 6 * T * V * d}


# ---------------------------------------------------------------------------
# In 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    c = case
    op = c["op"]
    s = _inputs(c, seed)
    if op in ("spread", "combine", "combine_grad"):
        T, k, d = c["tokens"], c["k"], c["d"]
        if op == "spread":
            flat = s.chosen.reshape(-1)
            kept = torch.nonzero((flat >= 0) & (flat < c["experts"])).reshape(-1)
            kept = kept[torch.sort(flat[kept].long() * (T * k) + kept).indices]  # by expert, then by place: all keys differ
            rows = torch.zeros((T * k, d), dtype=torch.float64, device="cuda")
            rows[: kept.numel()] = s.x.double()[kept // k]
            return [None, None, rows]
        y, dw, dx = torch.zeros((T, d), dtype=torch.float64, device="cuda"), torch.zeros((T, k), dtype=torch.float64, device="cuda"), None
        if op == "combine_grad":
            dx = torch.zeros((T * k, d), dtype=torch.float64, device="cuda")
        for j in range(k):
            t = torch.nonzero(s.order[1][:, j] >= 0).reshape(-1)
            p = s.order[1][t, j].long()
            if op == "combine":
                y[t] += s.weights[t, j].double()[:, None] * s.rows[p].double()
            else:
                g = s.dy[t].double()
                dw[t, j] = (g * s.rows[p].double()).sum(1)
                dx[p] = s.weights[t, j].double()[:, None] * g
        return y if op == "combine" else (dx, dw)
    if op in ("product", "grad_rows", "grad"):
        R, E, n, m = c["rows"], c["experts"], c["n"], c["m"]
        ends = s.offsets.tolist()
        if 2.0 * R * n * m > 1.2e13:
            return None
        if op == "grad":
            out = torch.empty((E, n, m), dtype=torch.float64, device="cuda")
            for e in range(E):
                a, b = ends[e], ends[e + 1]
                out[e] = torch.mm(s.x[a:b].double().t(), s.dy[a:b].double())
            return out if s.base is None else out.add_(s.base)
        out = torch.zeros((R, m if op == "product" else n), dtype=torch.float64, device="cuda")
        for e in range(E):
            a, b = ends[e], ends[e + 1]
            if b > a:
                out[a:b] = torch.mm(s.x[a:b].double(), s.w[e].double()) if op == "product" else torch.mm(s.dy[a:b].double(), s.w[e].double().t())
        return out
    T, V, d = c["tokens"], c["vocab"], c["d"]
    if 6.0 * T * V * d > 1.2e13:
        return None
    h, w = s.h.double(), s.table.double()
    lse, loss = (torch.zeros(T, dtype=torch.float64, device="cuda") for _ in range(2))
    dh = torch.zeros((T, d), dtype=torch.float64, device="cuda")
    dw = torch.zeros((V, d), dtype=torch.float64, device="cuda")
    for a in range(0, T, 1024):  # some tokens at a time
        x = torch.mm(h[a:a + 1024], w.t()) * c["scale"]
        t = s.targets[a:a + 1024].long()
        at = torch.nonzero(t >= 0).reshape(-1)
        lse[a:a + 1024] = torch.logsumexp(x, 1)
        loss[a + at] = lse[a + at] - x[at, t[at]]
        if op == "head_grad":
            p = torch.softmax(x, 1)
            p[at, t[at]] -= 1.0
            p *= s.dloss[a:a + 1024].double()[:, None]
            dh[a:a + 1024] = torch.mm(p, w) * c["scale"]
            dw += torch.mm(p.t(), h[a:a + 1024]) * c["scale"]
    if op == "loss":
        return [loss, lse]
    return [loss, lse, dh, dw if s.base is None else dw.add_(s.base)]
