"""What the operators around the optimizer step are measured on.

A trainer that steps an MoE with this library hands it gradients and a clip factor. The
operators here make them: the global gradient norm and clipping (``GradClip``), the embedding
lookup and its gradient (``Embedding``), and the routing of tokens to experts and its gradient
(``Router``). A pass is one call of one of them, on the inputs a training step has in hand.

A case names its operator (``op``):

* ``norm``, ``clip``: a parameter set's gradients, as one tensor for each parameter, some fp32.
  ``clip`` writes the clipped gradients to tensors of their own; with ``cast`` the gradients are
  fp32 accumulators over microbatches, and what is written is the bf16 that the step reads.
* ``lookup``, ``lookup_grad``: token ids as text has them (frequent ids are low ids, falling off
  as 1 / rank), a share of them padding (-1). ``base``: the gradient adds to one that the tied output head left.
* ``route``, ``route_grad``: one router's logits for a batch of tokens.
"""
import math

import numpy as np
import torch

own = False

ALIGN = 256       # elements: a tensor starts as an allocation of its own would
MAX_NORM = 1.0    # the trainer's limit
TINY = 1e-6       # added to the norm in the factor's divisor
SIGMA_G = 1e-3


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def _model(name, op, **kw):
    return {"name": name, "op": op, "set": "model", "vocab": 0, "d": 4096, "kv": 4096, "dense": 0, "blocks": 1, "experts": 0,
            "ffn": 4096, "router": 128, "fp32": False, "cast": False, **kw}


def _embed(name, op, **kw):
    return {"name": name, "op": op, "vocab": 50304, "d": 4096, "tokens": 32768, "table32": False, "act32": False,
            "ids64": True, "scale": 1.0, "pad": 0.0, "base": False, **kw}


def _route(name, op, **kw):
    return {"name": name, "op": op, "experts": 128, "k": 2, "tokens": 65536, "score": "softmax", "renorm": True, "bias": False,
            "groups": 1, "top_groups": 1, "group_top": 1, "scale": 1.0, "bf16": False, **kw}


def listed():
    return [
        # a toy MoE's 33 tensors: latency
        _model("norm_toy", "norm", vocab=512, d=64, kv=64, dense=256, experts=8, ffn=128, router=8),
        # the full 6.78B-parameter set: one read of 13.6 GB
        _model("norm_full", "norm", vocab=50304, kv=1024, dense=4096, blocks=2, experts=128),
        # a small MoE model of width 768, router and norms fp32: a little more than L2 holds
        _model("clip_768", "clip", vocab=50257, d=768, kv=768, dense=3072, blocks=2, experts=8, ffn=1536, router=8, fp32=True),
        # fp32 accumulators of one MoE layer with 16 experts, clipped into the bf16 gradients that the step reads
        _model("clip_accumulated", "clip", experts=16, ffn=1024, cast=True),
        # the toy model's lookup for 8 sequences of 128 tokens, scaled by sqrt(width): latency
        _embed("lookup_toy", "lookup", vocab=512, d=64, tokens=1024, scale=8.0),
        # the full model's: 256 sequences of 128 tokens
        _embed("lookup_full", "lookup"),
        # its gradient: every row of the table's gradient is written, rows without tokens as zeros
        _embed("lookup_grad_full", "lookup_grad"),
        # width 768, fp32 activations, padded sequences, on top of the output head's gradient
        _embed("lookup_grad_768", "lookup_grad", vocab=50257, d=768, tokens=4096, act32=True, ids64=False, scale=0.5, pad=0.1, base=True),
        # the paper's router (128 experts, top 2) for 8 sequences of 128 tokens: latency
        _route("route_128", "route", tokens=1024),
        # fine-grained experts: 8 of 256, the best 4 of 8 groups, sigmoid scores with a balance bias
        _route("route_grouped_256", "route", experts=256, k=8, score="sigmoid", bias=True, groups=8, top_groups=4, group_top=2, scale=2.5),
        # the paper's router, the gradient of a large batch
        _route("route_grad_128", "route_grad"),
        # an odd number of experts, bf16 logits, weights that are not renormalised
        _route("route_grad_127", "route_grad", experts=127, k=4, tokens=8192, renorm=False, bf16=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.randrange(3)
    if kind == 0:
        return {"op": rng.choice(("norm", "clip")), "set": "ragged", "tensors": _log(rng, 1, 600), "total": _log(rng, 1 << 10, 1 << 28),
                "layout": rng.randrange(1 << 20), "cast": rng.random() < 0.3}
    if kind == 1:
        d = _log(rng, 32, 8192)
        d = d if rng.random() < 0.3 else -(-d // 8) * 8
        vocab = min(_log(rng, 256, 131072), (1 << 28) // d)
        return {"op": rng.choice(("lookup", "lookup_grad")), "vocab": vocab, "d": d, "tokens": min(_log(rng, 1, 131072), (1 << 27) // d),
                "table32": rng.random() < 0.2, "act32": rng.random() < 0.4, "ids64": rng.random() < 0.6,
                "scale": rng.choice((1.0, 0.5, math.sqrt(d))), "pad": rng.choice((0.0, 0.0, 0.1)), "base": rng.random() < 0.4}
    groups = rng.choice((1, 1, 1, 2, 4, 8))
    experts = groups * max(2, _log(rng, 4, 512) // groups)
    top_groups = max(1, groups // 2)
    score = rng.choice(("softmax", "sigmoid"))
    return {"op": rng.choice(("route", "route_grad")), "experts": experts, "k": min(_log(rng, 1, 16), experts // groups * top_groups),
            "tokens": min(_log(rng, 1, 131072), (1 << 24) // experts), "score": score, "renorm": rng.random() < 0.7,
            "bias": score == "sigmoid" and rng.random() < 0.7, "groups": groups, "top_groups": top_groups,
            "group_top": rng.choice((1, 2)), "scale": rng.choice((1.0, 2.5)), "bf16": rng.random() < 0.3}


# ---------------------------------------------------------------------------
# Gradients of a parameter set
# ---------------------------------------------------------------------------
def _tensors(c):
    """[(elements, fp32, offset in elements of its type's buffer)] and {fp32: the buffer's length}."""
    sizes = []
    if c["set"] == "ragged":
        r = np.random.RandomState(c["layout"])
        share = r.exponential(size=c["tensors"]) ** 2
        for k, n in enumerate(np.maximum(1, share / share.sum() * c["total"]).astype(int)):
            sizes.append((int(n), bool(c["cast"] or r.randint(0, 5) == 0), int(r.randint(1, 8)) if r.randint(0, 4) == 0 else 0))
    else:
        d, F, E, v32 = c["d"], c["ffn"], c["experts"], c["fp32"]
        shapes = [(c["vocab"] * d, False)] if c["vocab"] else []
        for b in range(c["blocks"]):
            shapes += [(d * d, False), (c["kv"] * d, False), (c["kv"] * d, False), (d * d, False)] + [(d, v32)] * 4
            if c["dense"] and (b == 0 or c["blocks"] > 2):
                shapes += [(c["dense"] * d, False)] * 3
            if E and (b == c["blocks"] - 1 or c["blocks"] > 2):
                shapes += [(d * c["router"], v32)] + [(d * F, False)] * (3 * E)
        shapes += [(d, v32)] * 2
        sizes = [(n, bool(c["cast"] or f32), 0) for n, f32 in shapes]
    out, end = [], {False: 0, True: 0}
    for n, f32, skew in sizes:  # `skew`: a view that starts off a 16-byte boundary
        out.append((n, f32, end[f32] + skew))
        end[f32] += -(-(n + skew) // ALIGN) * ALIGN
    return out, end


def _gradients(c, seed):
    """{fp32: a buffer}: every tensor's gradient at its place, zeros between them."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    tensors, end = _tensors(c)
    flat = {f32: torch.zeros(n, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda") for f32, n in end.items() if n}
    r = np.random.RandomState(seed % (1 << 31))
    for n, f32, at in tensors:
        g = flat[f32][at: at + n].normal_(0.0, 1.0, generator=gen)
        g.mul_(SIGMA_G * math.exp(0.5 * r.randn()))  # tensors differ in the size of their gradients
    return flat


# ---------------------------------------------------------------------------
# Tokens and logits
# ---------------------------------------------------------------------------
def _frequencies(V):
    p = 1.0 / (np.arange(V, dtype=np.float64) + 2.7)
    return p / p.sum()


def _ids(c, gen):
    cdf = torch.from_numpy(np.cumsum(_frequencies(c["vocab"]))).cuda()
    u = torch.rand(c["tokens"], dtype=torch.float64, device="cuda", generator=gen)
    ids = torch.searchsorted(cdf, u).clamp_(max=c["vocab"] - 1)
    if c["pad"]:
        ids[torch.rand(c["tokens"], device="cuda", generator=gen) < c["pad"]] = -1
    return ids if c["ids64"] else ids.int()


def _dtype(f32):
    return torch.float32 if f32 else torch.bfloat16


class _State:
    pass


def _embed_inputs(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = _State()
    V, d, T = c["vocab"], c["d"], c["tokens"]
    s.ids = _ids(c, gen)
    s.table = s.base = s.dy = None
    if c["op"] == "lookup":
        s.table = torch.empty((V, d), dtype=_dtype(c["table32"]), device="cuda").normal_(0.0, 0.02, generator=gen)
    else:
        s.dy = torch.empty((T, d), dtype=_dtype(c["act32"]), device="cuda").normal_(0.0, SIGMA_G, generator=gen)
        if c["base"]:
            s.base = torch.empty((V, d), dtype=_dtype(c["table32"]), device="cuda").normal_(0.0, SIGMA_G, generator=gen)
    return s


def _route_inputs(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = _State()
    T, E = c["tokens"], c["experts"]
    liked = torch.randn(E, device="cuda", generator=gen) * 0.5  # some experts draw more tokens
    s.logits = (torch.randn((T, E), device="cuda", generator=gen) * 1.5 + liked).to(_dtype(not c["bf16"]))
    s.bias = s.chosen = s.dw = None
    if c["op"] == "route":
        if c["bias"]:
            s.bias = -0.1 * liked + 0.01 * torch.randn(E, device="cuda", generator=gen)
    else:
        s.chosen = torch.topk(s.logits.float(), c["k"], dim=-1).indices.int()
        s.dw = torch.randn((T, c["k"]), device="cuda", generator=gen) * SIGMA_G
    return s


def prepare(case, seed):
    c = case
    if c["op"] in ("norm", "clip"):
        s = _State()
        s.flat = _gradients(c, seed)
        tensors, _ = _tensors(c)
        s.out = None
        if c["op"] == "clip":
            s.out = {f32: torch.zeros_like(g, dtype=torch.bfloat16 if c["cast"] else g.dtype) for f32, g in s.flat.items()}
    elif c["op"] in ("lookup", "lookup_grad"):
        s = _embed_inputs(c, seed)
    else:
        s = _route_inputs(c, seed)
    s.c = c
    if own:
        from paper_2607_19058_gb300 import skewadam as S
        if c["op"] in ("norm", "clip"):
            cut = lambda bufs: [bufs[f32][at: at + n] for n, f32, at in tensors]  # noqa: E731
            s.op = S.GradClip(cut(s.flat), out=cut(s.out) if s.out else None)
        elif c["op"] in ("lookup", "lookup_grad"):
            s.op = S.Embedding(c["vocab"], c["d"], _dtype(c["table32"]), _dtype(c["act32"]), scale=c["scale"])
        else:
            s.op = S.Router(c["experts"], c["k"], score=c["score"], renorm=c["renorm"], groups=c["groups"], top_groups=c["top_groups"],
                            group_top=c["group_top"], scale=c["scale"])
    return s


# ---------------------------------------------------------------------------
# A pass
# ---------------------------------------------------------------------------
def run(state):
    s, c = state, state.c
    op = c["op"]
    if own:
        if op == "norm":
            return s.op.norm(MAX_NORM)
        if op == "clip":
            return [s.op.clip(MAX_NORM), list(s.out.values())]
        if op == "lookup":
            return s.op.lookup(s.table, s.ids)
        if op == "lookup_grad":
            return s.op.grad(s.ids, s.dy, base=s.base)
        if op == "route":
            return s.op.route(s.logits, bias=s.bias)
        return s.op.grad(s.logits, s.chosen, s.dw)
    if op in ("norm", "clip"):
        return _plain_clip(s, c)
    if op == "lookup":
        there = (s.ids >= 0) & (s.ids < c["vocab"])
        y = s.table[torch.where(there, s.ids, 0)].float() * c["scale"]
        return torch.where(there[:, None], y, 0.0).to(_dtype(c["act32"]))
    if op == "lookup_grad":
        return _plain_lookup_grad(s, c)
    if op == "route":
        return _plain_route(s, c)
    return _plain_route_grad(s, c)


def _plain_clip(s, c):
    norm = torch.stack([g.float().square().sum() for g in s.flat.values()]).sum().sqrt()
    gamma = torch.clamp(MAX_NORM / (norm + TINY), max=1.0)
    result = torch.stack([norm, gamma])
    if c["op"] == "norm":
        return result
    return [result, [(g.float() * gamma).to(s.out[f32].dtype) for f32, g in s.flat.items()]]


def _plain_lookup_grad(s, c):
    there = (s.ids >= 0) & (s.ids < c["vocab"])
    dw = torch.zeros((c["vocab"] + 1, c["d"]), dtype=torch.float32, device="cuda")  # padding adds to the last row
    dw.index_add_(0, torch.where(there, s.ids, c["vocab"]), s.dy.float())
    dw = dw[:-1] * c["scale"]
    if s.base is not None:
        dw = dw + s.base.float()
    return dw.to(_dtype(c["table32"]))


def _best(v, k):
    """The k largest of each row, the lowest index first among equals: values and indices."""
    v, i = torch.sort(v, dim=-1, descending=True, stable=True)
    return v[..., :k], i[..., :k]


def _plain_route(s, c):
    x = s.logits.float()
    T, E = x.shape
    if c["score"] == "softmax":
        e = torch.exp(x - x.amax(-1, keepdim=True))
        score, shown = e / e.sum(-1, keepdim=True), e  # the row's sum changes no order
    else:
        score = shown = 1.0 / (1.0 + torch.exp(-x))
    choice = x
    if s.bias is not None:
        choice = shown = score + s.bias
    if c["groups"] > 1:
        by = (choice if c["group_top"] == 1 else shown).view(T, c["groups"], -1)
        by = _best(by, c["group_top"])[0].sum(-1)
        keep = torch.zeros_like(by, dtype=torch.bool).scatter_(1, _best(by, c["top_groups"])[1], True)
        choice = torch.where(keep.repeat_interleave(E // c["groups"], dim=1), choice, -math.inf)
    chosen = _best(choice, c["k"])[1]
    w = torch.gather(score, 1, chosen)
    if c["renorm"]:
        w = w / w.sum(-1, keepdim=True)
    counts = (chosen.reshape(-1, 1) == torch.arange(E, device="cuda")).sum(0) if T * E * c["k"] < 1 << 28 else torch.bincount(chosen.reshape(-1), minlength=E)
    return chosen.int(), w * c["scale"], counts.int()


def _plain_route_grad(s, c):
    x, at = s.logits.float(), s.chosen.long()
    if c["score"] == "softmax":
        e = torch.exp(x - x.amax(-1, keepdim=True))
        score = e / e.sum(-1, keepdim=True)
    else:
        score = 1.0 / (1.0 + torch.exp(-x))
    g, p = s.dw * c["scale"], torch.gather(score, 1, at)
    if c["renorm"]:
        total = p.sum(-1, keepdim=True)
        g = (g - (g * p).sum(-1, keepdim=True) / total) / total
    ds = torch.zeros_like(x).scatter_(1, at, g)
    if c["score"] == "softmax":
        dx = score * (ds - (ds * score).sum(-1, keepdim=True))
    else:
        dx = ds * score * (1.0 - score)
    return dx.to(s.logits.dtype)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    c = case
    op = c["op"]
    if op in ("norm", "clip"):
        by = fl = 0
        for n, f32, _ in _tensors(c)[0]:
            by += n * (4 if f32 else 2)
            fl += 2 * n
            if op == "clip":
                by += n * (4 if f32 and not c["cast"] else 2)
                fl += n
        return {"bytes": by + 8, "flops": fl}
    if op in ("lookup", "lookup_grad"):
        V, d, T = c["vocab"], c["d"], c["tokens"]
        row, act = d * (4 if c["table32"] else 2), d * (4 if c["act32"] else 2)
        T_real = T * (1.0 - c["pad"])
        ids = T * (8 if c["ids64"] else 4)
        if op == "lookup":  # the rows that some token asks for, each once
            asked = float(np.sum(-np.expm1(T_real * np.log1p(-_frequencies(V)))))
            return {"bytes": int(asked * row + T * act + ids), "flops": T * d}
        return {"bytes": int(T_real * act + V * row * (2 if c["base"] else 1) + ids), "flops": int(T_real * d + V * d)}
    T, E, k, x = c["tokens"], c["experts"], c["k"], 2 if c["bf16"] else 4
    if op == "route":
        return {"bytes": T * E * x + 8 * T * k + 4 * E + (4 * E if c["bias"] else 0), "flops": 4 * T * E}
    # the chosen logits alone, unless the softmax's other entries have a gradient too
    read = T * E * x if c["score"] == "softmax" and not c["renorm"] else T * k * x
    return {"bytes": read + 8 * T * k + T * E * x, "flops": 4 * T * E}


# ---------------------------------------------------------------------------
# In 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    c = case
    op = c["op"]
    if op in ("norm", "clip"):
        flat = _gradients(c, seed)
        total = 0.0
        for g in flat.values():
            for part in g.split(1 << 28):
                total += float(torch.dot(part.double(), part.double()))
        norm = math.sqrt(total)
        gamma = min(1.0, MAX_NORM / (norm + TINY))
        result = torch.tensor([norm, gamma], dtype=torch.float64)
        return result if op == "norm" else [result, [g.double() * gamma for g in flat.values()]]
    if op == "lookup":
        s = _embed_inputs(c, seed)
        y = torch.zeros((c["tokens"], c["d"]), dtype=torch.float64, device="cuda")
        at = torch.nonzero((s.ids >= 0) & (s.ids < c["vocab"])).reshape(-1)
        y[at] = s.table.index_select(0, s.ids[at]).double() * c["scale"]
        return y
    if op == "lookup_grad":
        s = _embed_inputs(c, seed)
        dw = torch.zeros((c["vocab"], c["d"]), dtype=torch.float64, device="cuda")
        at = torch.nonzero((s.ids >= 0) & (s.ids < c["vocab"])).reshape(-1)
        dw.index_put_((s.ids[at].long(),), s.dy[at].double() * c["scale"], accumulate=True)
        return dw if s.base is None else dw.add_(s.base)
    s = _route_inputs(c, seed)
    x = s.logits.double()
    T, E = x.shape
    p = torch.softmax(x, -1) if c["score"] == "softmax" else torch.sigmoid(x)
    if op == "route":
        choice = p if s.bias is None else p + s.bias.double()
        if c["groups"] > 1:
            by = choice.view(T, c["groups"], E // c["groups"]).topk(c["group_top"], dim=-1).values.sum(-1)
            out = torch.ones((T, c["groups"]), dtype=torch.bool, device="cuda")
            out.scatter_(1, by.topk(c["top_groups"], dim=-1).indices, False)
            choice = choice.masked_fill(out[:, :, None].expand(-1, -1, E // c["groups"]).reshape(T, E), -math.inf)
        w = p.gather(1, choice.topk(c["k"], dim=-1).indices)
        if c["renorm"]:
            w = w / w.sum(1, keepdim=True)
        return None, w * c["scale"], None
    with torch.enable_grad():  # by differentiation
        x.requires_grad_(True)
        p = torch.softmax(x, -1) if c["score"] == "softmax" else torch.sigmoid(x)
        w = p.gather(1, s.chosen.long())
        if c["renorm"]:
            w = w / w.sum(1, keepdim=True)
        dx, = torch.autograd.grad(w * c["scale"], x, s.dw.double())
    return dx
