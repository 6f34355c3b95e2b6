"""What is measured of the operators around the layers whose weights depend on the pattern: the router
by scores, embeddings, the residual stream between blocks, and the clipping of many changes.

A case is a dict of plain values:
  op         "route"     bp_route_scored (and, with train, bp_route_scored_backward): the experts of each
                         pattern by softmax or sigmoid scores and a bias, within its best groups of experts;
             "embed"     bp_embed (and, with train, bp_embed_backward): rows of a table by token, and the
                         pooled change of every token's row;
             "residual"  bp_residual_forward (and, with train, bp_residual_backward): a block's output, normed,
                         gated and scaled, joins the stream, and is normed again for the next block;
             "clip"      bp_clip: the norm of all changes of a model together, and the changes scaled
                         down to a bound.
  dtype      "f32" or "bf16" (of the rows; changes, gates, biases and the norms' weights are float32 in both);
             of "clip" also "both": two thirds of the changes float32, a third bfloat16
  n          patterns, ids or rows
  E, k       experts, and those of a pattern; groups, open, top: groups of experts, those that stay open, and
             how many of a group's largest scores are its value; renorm: gates add up to the scale;
             masked: some experts are closed to a pattern
  tokens     rows of the table; width: units of a row
  norms      of the block's output and of the next block's input: "none", "rms" or "layer" each;
  gates      0: none; 1: one gate a unit; more: one gate a unit and sequence, of ragged lengths
  tensors    how many changes there are, of total values together, skew: how uneven their sizes are;
             clips: whether the norm is above the bound (else the changes stay as they are)
"""
import math

import torch

own = False
DEV = "cuda"
EPS = 1e-5


def _route(n, E, k, dtype="f32", scores="sigmoid", groups=1, open_=1, top=2, renorm=True, scale=1.0, train=False,
           masked=False):
    return dict(op="route", n=n, E=E, k=k, dtype=dtype, scores=scores, groups=groups, open=open_, top=top, renorm=renorm,
                scale=scale, train=train, masked=masked)


def _embed(n, tokens, width, dtype="bf16", train=False, scale=1.0):
    return dict(op="embed", n=n, tokens=tokens, width=width, dtype=dtype, train=train, scale=scale)


def _residual(n, width, dtype="bf16", norms=("rms", "rms"), gates=1, scale=1.0, train=False):
    return dict(op="residual", n=n, width=width, dtype=dtype, norm_out=norms[0], norm_in=norms[1], gates=gates,
                scale=scale, train=train)


def _clip(tensors, total, dtype="f32", skew=2.0, clips=True):
    return dict(op="clip", tensors=tensors, total=total, dtype=dtype, skew=skew, clips=clips)


def listed():
    return [
        # one pattern asks an interactive program's router, experts in eight groups
        dict(_route(1, 64, 6, groups=8, open_=3), name="route_1"),
        # a moderate step over softmax scores, some experts closed to some patterns, an odd number of experts a group
        dict(_route(777, 60, 4, scores="softmax", groups=12, open_=5, top=1, renorm=False, scale=2.0, train=True, masked=True),
             name="route_train_777"),
        # a long step over many experts, balanced by a bias
        dict(_route(16384, 256, 8, "bf16", groups=8, open_=4, scale=2.5, train=True), name="route_train_16384"),
        # one token of an answer under way
        dict(_embed(1, 50001, 2048), name="embed_1"),
        # 512 windows of seven letters, few tokens that each come often, odd float32 rows
        dict(_embed(3584, 29, 15, "f32", train=True), name="embed_letters_train"),
        # a step over a moderate vocabulary
        dict(_embed(40001, 32003, 1024, train=True, scale=32.0), name="embed_train_40001"),
        # a step over a large one: most rows' changes are zeros
        dict(_embed(16384, 100003, 4096, train=True, scale=64.0), name="embed_train_16384"),
        # one row of an answer under way, between two blocks
        dict(_residual(1, 2048, scale=0.5), name="residual_1"),
        # sequences of different lengths with gates of their own, layer norms, odd float32 rows
        dict(_residual(513, 203, "f32", ("layer", "layer"), gates=5, train=True), name="residual_train_513"),
        # a wide model's step
        dict(_residual(16384, 4096, scale=0.25, train=True), name="residual_train_16384"),
        # the changes of a small net, above the bound
        dict(_clip(6, 27626), name="clip_27626"),
        # the changes of a large model
        dict(_clip(211, 300_000_007, "both"), name="clip_300000007"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Sizes over the listed cases' ranges; no more work than the largest of them."""
    while True:
        op = rng.choice(["route", "embed", "residual", "clip"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        train = rng.random() < 0.6
        if op == "route":
            groups = rng.choice([1, 1, 2, 4, 8, 10])
            E = groups * max(1, _log(rng, 8, 256) // groups)
            open_ = groups if groups == 1 else rng.randint(1, groups)
            k = min(E // groups * open_, rng.randint(1, 8))
            return _route(_log(rng, 1, 16384), E, k, dtype, rng.choice(["softmax", "sigmoid"]), groups, open_, rng.choice([1, 2]),
                          k > 1 and rng.random() < 0.5, round(rng.uniform(0.5, 3.0), 2), train, rng.random() < 0.3)
        if op == "embed":
            width = 8 * _log(rng, 4, 512) if dtype == "bf16" else _log(rng, 3, 2048)
            c = _embed(_log(rng, 1, 65536), _log(rng, 27, 131072), width, dtype, train, round(rng.uniform(0.5, 64.0), 2))
        elif op == "residual":
            width = 8 * _log(rng, 8, 1024) if dtype == "bf16" else _log(rng, 16, 4096)
            norms = rng.choice([("rms", "rms"), ("rms", "rms"), ("layer", "layer"), ("none", "rms"), ("rms", "none"),
                                ("none", "layer")])
            c = _residual(_log(rng, 1, 16384), width, dtype, norms, rng.choice([0, 1, 1, 3, 17]), round(rng.uniform(0.1, 1.0), 2), train)
        else:
            c = _clip(_log(rng, 1, 400), _log(rng, 5000, 300_000_000), rng.choice(["f32", "bf16", "both"]),
                      round(rng.uniform(0.0, 4.0), 2), rng.random() < 0.7)
        if work(c)["bytes"] <= 2.5e9:
            return c


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# ------------------------------------------------------------------ inputs
def _ends(n, parts, skew, g):
    """`parts` + 1 ascending whole numbers from 0 to n, the parts the more uneven the larger skew is."""
    w = torch.rand(parts, generator=g, device=DEV).double().add(1e-3).pow(skew)
    at = torch.zeros(parts + 1, dtype=torch.int64, device=DEV)
    at[1:] = (w.cumsum(0) / w.sum() * n).round().long().clamp(0, n)
    at[-1] = n
    return at


def _inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    t, op = _type(case), case["op"]

    def normal(*shape, scale=1.0, dtype=t):
        return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)

    if op == "route":
        n, E, k = case["n"], case["E"], case["k"]
        z = torch.randn(n, E, generator=g, device=DEV) * 1.5 + torch.randn(E, generator=g, device=DEV) * 0.7
        if case["masked"]:   # experts closed to a pattern; some patterns are left with none
            closed = torch.rand(n, E, generator=g, device=DEV) < 0.3
            closed |= torch.rand(n, 1, generator=g, device=DEV) < 0.01
            z = z.masked_fill(closed, -math.inf)
        # what keeps the experts balanced: of the size of the scores' own differences
        bias = normal(E, scale=0.1 if case["scores"] == "sigmoid" else 0.5 / E, dtype=torch.float32)
        return dict(logits=z.to(t), bias=bias, dgate=normal(n, k, dtype=torch.float32))
    if op == "embed":
        n, V, w = case["n"], case["tokens"], case["width"]
        # the i-th most frequent token comes about 1 / (i + 1) as often as the first; their numbers are in no order
        often = torch.rand(n, generator=g, device=DEV, dtype=torch.float64).mul(math.log(V + 1)).exp().long().sub(1)
        order = torch.randperm(V, generator=g, device=DEV)
        ids = order[often.clamp(0, V - 1)].int()
        return dict(table=normal(V, w, scale=w ** -0.5), ids=ids, D=normal(n, w) if case["train"] else None)
    if op == "residual":
        n, w, gates = case["n"], case["width"], case["gates"]
        s = dict(X=normal(n, w, scale=2.0), F=normal(n, w, scale=0.7))
        if case["norm_out"] != "none":
            s["wo"] = 1 + normal(w, scale=0.2, dtype=torch.float32)
        if case["norm_in"] != "none":
            s["wi"] = 1 + normal(w, scale=0.2, dtype=torch.float32)
        if case["norm_out"] == "layer":
            s["bo"] = normal(w, scale=0.1, dtype=torch.float32)
        if case["norm_in"] == "layer":
            s["bi"] = normal(w, scale=0.1, dtype=torch.float32)
        if gates:
            s["gate"] = normal(gates, w, dtype=torch.float32)
        if gates > 1:
            s["offsets"] = _ends(n, gates, 2.0, g).int()
        if case["train"]:
            s.update(dY=normal(n, w), dH=normal(n, w) if case["norm_in"] != "none" else None)
        return s
    total, parts = case["total"], case["tensors"]
    # a model's sizes are its own, whatever its changes are
    ends = _ends(total, parts, case["skew"], torch.Generator(device=DEV).manual_seed(parts)).tolist()
    sixteen = [case["dtype"] == "bf16" or (case["dtype"] == "both" and i % 3 == 2) for i in range(parts)]
    sizes = [b - a for a, b in zip(ends, ends[1:])]
    # one piece of memory for each type, the changes side by side in it; some are much smaller than others
    amount = (2.0 if case["clips"] else 0.5) * total ** -0.5
    flat = {}
    for name, dtype, wide in (("f32", torch.float32, False), ("bf16", torch.bfloat16, True)):
        count = sum(s for s, w in zip(sizes, sixteen) if w == wide)
        if count:
            flat[name] = torch.randn(count, generator=g, device=DEV).mul_(amount).to(dtype)
            flat[name][: count // 5] *= 0.01
    return dict(flat=flat, sizes=sizes, sixteen=sixteen)


def _views(flat, sizes, sixteen):
    """The changes as tensors, in order, out of the memory of their type."""
    at = dict(f32=0, bf16=0)
    views = []
    for size, wide in zip(sizes, sixteen):
        name = "bf16" if wide else "f32"
        if size:
            views.append(flat[name][at[name]:at[name] + size])
            at[name] += size
    return views


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    op, t = case["op"], _type(case)
    if op == "clip":
        s["grads"] = _views(s["flat"], s["sizes"], s["sixteen"])
    if op == "residual" and case["gates"]:
        s["lengths"] = (s["offsets"][1:] - s["offsets"][:-1]).long() if case["gates"] > 1 else torch.tensor([case["n"]], device=DEV)
    if not own:
        return s
    from paper_1801_01554_gb300 import bp

    bt = bp.BP_BF16 if case["dtype"] == "bf16" else bp.BP_F32

    def empty(*shape, dtype=t):
        return torch.empty(*shape, dtype=dtype, device=DEV)

    if op == "route":
        n, E, k = case["n"], case["E"], case["k"]
        s["router"] = bp.ScoredRouter(E, k, bt, max_patterns=n,
                                      scores=bp.BP_SCORES_SIGMOID if case["scores"] == "sigmoid" else bp.BP_SCORES_SOFTMAX,
                                      n_groups=case["groups"], open_groups=case["open"], group_top=case["top"],
                                      renormalise=case["renorm"], scale=case["scale"])
        s.update(expert=empty(n, k, dtype=torch.int32), gate=empty(n, k, dtype=torch.float32),
                 offsets=empty(E + 1, dtype=torch.int32), source=empty(n * k, dtype=torch.int32),
                 place=empty(n, k, dtype=torch.int32), dlogits=empty(n, E))
    elif op == "embed":
        n, V, w = case["n"], case["tokens"], case["width"]
        s["layer"] = bp.Embedding(V, w, bt, max_ids=n)
        s["Y"] = empty(n, w)
        if case["train"]:
            s["G"] = empty(V, w, dtype=torch.float32)
    elif op == "residual":
        n, w = case["n"], case["width"]
        kind = dict(none=bp.BP_NORM_NONE, rms=bp.BP_NORM_RMS, layer=bp.BP_NORM_LAYER)
        s["layer"] = bp.Residual(w, bt, max_rows=n, norm_out=kind[case["norm_out"]], norm_in=kind[case["norm_in"]], eps=EPS,
                                 max_gates=max(1, case["gates"]))
        s.update(Y=empty(n, w), stats=empty(n, 4, dtype=torch.float32))
        s["H"] = empty(n, w) if case["norm_in"] != "none" else None
        if case["train"]:
            s.update(dX=empty(n, w), dF=empty(n, w))
            for name in ("wo", "bo", "wi", "bi", "gate"):
                s["G" + name] = empty(*s[name].shape, dtype=torch.float32) if name in s else None
    else:
        s["out"] = {name: torch.empty_like(x) for name, x in s["flat"].items()} if case["clips"] else s["flat"]
        s["clip"] = bp.Clip(s["grads"], _views(s["out"], s["sizes"], s["sixteen"]) if case["clips"] else None)
        s["norm"] = empty(1, dtype=torch.float32)
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    c = s["case"]
    op = c["op"]
    if op == "route":
        n, names = c["n"], ("expert", "gate", "offsets", "source", "place")
        s["router"].forward(s["logits"], s["bias"], n, *(s[x] for x in names))
        out = {x: s[x] for x in names}
        if c["train"]:
            s["router"].backward(s["logits"], n, s["expert"], s["dgate"], s["dlogits"])
            out["dlogits"] = s["dlogits"]
        return out
    if op == "embed":
        s["layer"].forward(s["table"], s["ids"], c["n"], s["Y"], scale=c["scale"])
        if not c["train"]:
            return dict(Y=s["Y"])
        s["layer"].backward(s["ids"], c["n"], s["D"], s["G"], scale=c["scale"])
        return dict(Y=s["Y"], G=s["G"])
    if op == "residual":
        way = dict(wo=s.get("wo"), bo=s.get("bo"), gate=s.get("gate"), offsets=s.get("offsets"), n_gates=c["gates"],
                   scale=c["scale"], wi=s.get("wi"))
        s["layer"].forward(s["X"], s["F"], c["n"], s["Y"], s["H"], s["stats"] if c["train"] else None, bi=s.get("bi"), **way)
        out = dict(Y=s["Y"], H=s["H"])
        if c["train"]:
            s["layer"].backward(s["Y"], s["F"], c["n"], s["stats"], s["dY"], s["dH"], s["dX"], s["dF"], Gwo=s["Gwo"],
                                Gbo=s["Gbo"], Ggate=s["Ggate"], Gwi=s["Gwi"], Gbi=s["Gbi"], **way)
            out.update({x: s[x] for x in ("dX", "dF", "Gwo", "Gbo", "Ggate", "Gwi", "Gbi")})
        return out
    s["clip"].run(1.0, s["norm"])
    return dict(norm=s["norm"], out=s["out"])


def _run_plain(s):
    return dict(route=_plain_route, embed=_plain_embed, residual=_plain_residual, clip=_plain_clip)[s["case"]["op"]](s)


def _plain_route(s):
    c = s["case"]
    n, E, k, G = c["n"], c["E"], c["k"], c["groups"]
    z = s["logits"].double()   # scores next to one another are told apart in 64 bits
    none = -math.inf
    open_ = z > none
    if c["scores"] == "sigmoid":
        p = 1 / (1 + torch.exp(-z))
    else:
        peak = z.max(1, keepdim=True).values
        up = torch.exp(z - torch.where(peak > none, peak, torch.zeros_like(peak)))
        total = up.sum(1, keepdim=True)
        p = up / torch.where(total > 0, total, torch.ones_like(total))
    value = torch.where(open_, p + s["bias"].double(), torch.full_like(p, none))
    if G > 1:
        best = torch.sort(value.view(n, G, E // G), dim=2, descending=True).values[:, :, :c["top"]]
        worth = torch.where(best > none, best, torch.zeros_like(best)).sum(2)
        worth = torch.where(best[:, :, 0] > none, worth, torch.full_like(worth, none))
        shut = torch.sort(worth, dim=1, descending=True, stable=True).indices[:, c["open"]:]
        value = value.view(n, G, E // G).scatter(1, shut.unsqueeze(2).expand(-1, -1, E // G), none).view(n, E)
    top, expert = torch.sort(value, dim=1, descending=True, stable=True)   # ties: the lowest index first
    top, at = top[:, :k], expert[:, :k]
    chosen = top > none
    expert = torch.where(chosen, at, torch.full_like(at, -1)).int()
    score = torch.where(chosen, p.gather(1, at), torch.zeros_like(top))
    sum_ = score.sum(1, keepdim=True)
    share = score / torch.where(sum_ > 0, sum_, torch.ones_like(sum_)) if c["renorm"] else score
    # rows by expert
    flat = expert.view(-1).long()
    rows = torch.sort(torch.where(flat < 0, torch.full_like(flat, E), flat), stable=True).indices
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=DEV)
    offsets[1:] = torch.bincount(flat + 1, minlength=E + 1)[1:].cumsum(0)
    place = torch.empty_like(flat)
    every = torch.arange(n * k, device=DEV)
    place[rows] = every
    out = dict(expert=expert, gate=(c["scale"] * share).float(), offsets=offsets.int(),
               source=torch.where(every < offsets[E], rows // k, torch.full_like(rows, -1)).int(),
               place=torch.where(flat < 0, torch.full_like(place, -1), place).view(n, k).int())
    if c["train"]:
        u = torch.where(chosen, c["scale"] * s["dgate"].double(), torch.zeros_like(score))
        pull = (share * u).sum(1, keepdim=True)
        if c["scores"] == "sigmoid":
            d = share * ((u - pull) if c["renorm"] else u) * (1 - p.gather(1, at))
            dz = torch.zeros_like(z).scatter_add_(1, at, d)
        elif c["renorm"]:
            dz = torch.zeros_like(z).scatter_add_(1, at, share * (u - pull))
        else:
            dz = (-p * pull).scatter_add_(1, at, share * u)
        out["dlogits"] = dz.to(s["logits"].dtype)
    return out


def _plain_embed(s):
    c, ids = s["case"], s["ids"].long()
    y = (s["table"][ids].float() * c["scale"]).to(s["table"].dtype)
    if not c["train"]:
        return dict(Y=y)
    g = torch.zeros(c["tokens"], c["width"], device=DEV)
    return dict(Y=y, G=g.index_add_(0, ids, s["D"].float() * c["scale"]))


def _normed(x, kind):
    """x with its mean taken off ("layer") over its root mean square, and one over that root."""
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    r = 1 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    return x * r, r


def _through(d, hat, r, kind):
    """The gradient of a norm's input from that of its normed values."""
    d = d - hat * (d * hat).mean(1, keepdim=True) - (d.mean(1, keepdim=True) if kind == "layer" else 0)
    return d * r


def _plain_residual(s):
    c, t = s["case"], s["X"].dtype
    x, f = s["X"].float(), s["F"].float()
    fhat, rf = (f, None) if c["norm_out"] == "none" else _normed(f, c["norm_out"])
    u = fhat * s["wo"] if "wo" in s else fhat
    u = u + s["bo"] if "bo" in s else u
    g = torch.repeat_interleave(s["gate"], s["lengths"], 0, output_size=c["n"]) if c["gates"] > 1 else s.get("gate", 1.0)
    y = (x + c["scale"] * g * u).to(t)
    out = dict(Y=y, H=None)
    if c["norm_in"] != "none":
        yhat, ry = _normed(y.float(), c["norm_in"])
        h = yhat * s["wi"]
        out["H"] = (h + s["bi"] if "bi" in s else h).to(t)
    if not c["train"]:
        return out
    dy = s["dY"].float()
    out.update(Gwo=None, Gbo=None, Ggate=None, Gwi=None, Gbi=None)
    if c["norm_in"] != "none":
        dh = s["dH"].float()
        dy = dy + _through(dh * s["wi"], yhat, ry, c["norm_in"])
        out["Gwi"] = (dh * yhat).sum(0)
        out["Gbi"] = dh.sum(0) if "bi" in s else None
    du = c["scale"] * g * dy
    if c["gates"]:
        of = torch.repeat_interleave(torch.arange(c["gates"], device=DEV), s["lengths"], output_size=c["n"])
        dgate = c["scale"] * dy * u
        out["Ggate"] = dgate.sum(0, keepdim=True) if c["gates"] == 1 else torch.zeros_like(s["gate"]).index_add_(0, of, dgate)
    df = du
    if c["norm_out"] != "none":
        out["Gwo"] = (du * fhat).sum(0)
        out["Gbo"] = du.sum(0) if "bo" in s else None
        df = _through(du * s["wo"], fhat, rf, c["norm_out"])
    out.update(dX=dy.to(t), dF=df.to(t))
    return out


def _plain_clip(s):
    squares = torch.stack([x.float().square().sum(dtype=torch.float64) for x in s["grads"]])
    norm = squares.sum().sqrt()
    by = torch.where(norm > 1.0, 1.0 / norm, torch.ones_like(norm)).float()
    if s["case"]["clips"]:
        out = {name: (x.float() * by).to(x.dtype) for name, x in s["flat"].items()}
    else:
        out = s["flat"]
    return dict(norm=norm.float().view(1), out=out)


# ------------------------------------------------------------------ what a pass cannot do without
def _distinct(n, tokens):
    """How many tokens n ids name, on average."""
    i = torch.arange(tokens, dtype=torch.float64)
    p = torch.log1p(1 / (i + 1)) / math.log(tokens + 1)
    return float((1 - torch.exp(n * torch.log1p(-p.clamp(max=1 - 1e-12)))).sum())


def work(case):
    op, e = case["op"], 2 if case["dtype"] == "bf16" else 4
    if op == "route":
        n, E, rows = case["n"], case["E"], case["n"] * case["k"]
        b, f = n * E * e + 4 * E + 4 * (4 * rows + E + 1), 6 * n * E
        if case["train"]:
            b, f = b + 4 * rows + n * E * e, f + 2 * n * E
        return dict(bytes=b, flops=f)
    if op == "embed":
        n, w = case["n"], case["width"]
        b, f = 4 * n + (_distinct(n, case["tokens"]) + n) * w * e, n * w
        if case["train"]:
            b, f = b + n * w * e + 4 * case["tokens"] * w, f + 2 * n * w
        return dict(bytes=int(b), flops=f)
    if op == "residual":
        n, w = case["n"], case["width"]
        norms = (case["norm_out"] != "none") + (case["norm_in"] != "none")
        rows = 3 + (case["norm_in"] != "none")           # X, F, Y and H
        f = n * w * (3 + 4 * norms)
        columns = case["gates"] + sum(dict(none=0, rms=1, layer=2)[case[x]] for x in ("norm_out", "norm_in"))
        if case["train"]:   # dY, dH, dX and dF; the forward pass's Y and F are there
            rows, f, columns = rows + 3 + (case["norm_in"] != "none"), f + n * w * (4 + 8 * norms), 2 * columns
        return dict(bytes=rows * n * w * e + 4 * columns * w, flops=f)
    e = dict(f32=4, bf16=2, both=10 / 3)[case["dtype"]]
    return dict(bytes=int(case["total"] * e * (2 if case["clips"] else 1)), flops=case["total"] * (3 if case["clips"] else 2))


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    return dict(route=_exact_route, embed=_exact_embed, residual=_exact_residual, clip=_exact_clip)[case["op"]](case, s)


def _exact_route(c, s):
    """Gates and gradient for the experts that the definition chooses, one choice after another."""
    n, E, k, G = c["n"], c["E"], c["k"], c["groups"]
    z = s["logits"].double().requires_grad_(c["train"])
    closed = z.detach() == -math.inf
    safe = torch.where(closed, torch.zeros_like(z), z)
    if c["scores"] == "sigmoid":
        p = torch.sigmoid(safe).masked_fill(closed, 0.0)
    else:
        p = torch.exp(safe - safe.detach().amax(1, keepdim=True)).masked_fill(closed, 0.0)
        p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
    left = (p.detach() + s["bias"].double()).masked_fill(closed, -math.inf)

    def pick(values):
        """Where each row's largest value is (the first of them), and whether there is one."""
        m = values.amax(1, keepdim=True)
        return (values == m).to(torch.int8).argmax(1, keepdim=True), m > -math.inf

    if G > 1:
        worth, rest = torch.zeros(n, G, dtype=torch.float64, device=DEV), left.clone().view(n * G, E // G)
        some = (rest.amax(1) > -math.inf).view(n, G)
        for _ in range(min(c["top"], E // G)):
            at, ok = pick(rest)
            worth += torch.where(ok, rest.gather(1, at), torch.zeros_like(rest[:, :1])).view(n, G)
            rest = rest.scatter(1, at, -math.inf)
        worth = worth.masked_fill(~some, -math.inf)
        stays = torch.zeros(n, G, dtype=torch.bool, device=DEV)
        for _ in range(c["open"]):
            at, ok = pick(worth)
            stays.scatter_(1, at, stays.gather(1, at) | ok)
            worth = worth.scatter(1, at, -math.inf)
        left = left.masked_fill(~stays.repeat_interleave(E // G, 1), -math.inf)
    scores = []
    for _ in range(k):
        at, ok = pick(left)
        scores.append(torch.where(ok, p.gather(1, at), torch.zeros_like(p[:, :1])))
        left = left.scatter(1, at, -math.inf)
    gate = torch.cat(scores, 1)
    if c["renorm"]:
        gate = gate / gate.sum(1, keepdim=True).clamp(min=1e-300)
    gate = c["scale"] * gate
    out = dict(expert=None, gate=gate.detach(), offsets=None, source=None, place=None)
    if c["train"]:
        out["dlogits"] = torch.autograd.grad((gate * s["dgate"].double()).sum(), z)[0]
    return out


def _exact_embed(c, s):
    order = torch.sort(s["ids"].long(), stable=True)
    y = s["table"].double().mul_(c["scale"]).index_select(0, s["ids"].long())
    if not c["train"]:
        return dict(Y=y)
    g = torch.zeros(c["tokens"], c["width"], dtype=torch.float64, device=DEV)
    some, count = torch.unique_consecutive(order.values, return_counts=True)
    sums = torch.segment_reduce(s["D"].double()[order.indices], "sum", lengths=count, axis=0)
    g[some] = c["scale"] * sums
    return dict(Y=y, G=g)


def _exact_residual(c, s):
    names = [x for x in ("X", "F", "wo", "bo", "wi", "bi", "gate") if x in s]
    v = {x: s[x].double().requires_grad_(c["train"]) for x in names}

    def norm(x, kind, w, b):
        if kind == "none":
            return x
        if kind == "layer":
            var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
            return (x - mean) * torch.rsqrt(var + EPS) * v[w] + v[b]
        return x * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS) * v[w]

    u = norm(v["F"], c["norm_out"], "wo", "bo")
    if c["gates"]:
        of = torch.zeros(c["n"], dtype=torch.int64, device=DEV)
        for i in range(1, c["gates"]):
            of += torch.arange(c["n"], device=DEV) >= s["offsets"][i]
        u = v["gate"][of] * u if c["gates"] > 1 else v["gate"] * u
    y = v["X"] + c["scale"] * u
    out = dict(Y=y.detach(), H=None)
    loss = (y * s["dY"].double()).sum() if c["train"] else None
    if c["norm_in"] != "none":   # of the stream as it is stored
        h = norm(y + (y.detach().to(s["X"].dtype).double() - y.detach()), c["norm_in"], "wi", "bi")
        out["H"] = h.detach()
        if c["train"]:
            loss = loss + (h * s["dH"].double()).sum()
    if c["train"]:
        grads = dict(zip(names, torch.autograd.grad(loss, [v[x] for x in names])))
        out.update(dX=grads["X"], dF=grads["F"], **{"G" + x: grads.get(x) for x in ("wo", "bo", "gate", "wi", "bi")})
    return out


def _exact_clip(c, s):
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(x.double()) for x in s["flat"].values()]))
    by = min(1.0, 1.0 / float(norm))
    return dict(norm=norm.view(1), out={name: x.double() * by for name, x in s["flat"].items()})
