"""What is measured of the layers whose weights depend on the pattern: a mixture of experts
(router, products grouped by expert, the mix of the chosen experts' outputs) and low-rank
adapters of many requests beside a shared layer.

A case is a dict of plain values:
  op         "route"    bp_route (and, with train, bp_route_backward): the k experts of each
                        pattern, their gates, and the order of the rows by expert;
             "mix"      bp_mix (and, with train, bp_mix_backward): each pattern's gated sum of
                        its experts' outputs;
             "experts"  bp_experts_forward, or bp_experts_backward with back: rows times the
                        weights of their expert, the changes of every expert's weights;
             "adapters" bp_adapters_forward, or bp_adapters_backward with back: a shared layer
                        plus the low-rank change of each request's adapter.
  dtype      "f32" or "bf16" (operands; changes and biases are float32 in both)
  n          patterns (rows over all requests for "adapters");  k: experts per pattern
  E          experts, or adapters;  n_in, n_out: units of the layer;  rank: of the adapters
  requests   requests that share the n rows;  gates: "chosen" (softmax over the chosen experts'
             logits) or "all" (over all experts');  squash: the logistic on the outputs, or the
             factor a (1 - a) of the layer's inputs on the way back
  gather     the inputs are patterns read through the router's order (else rows in that order)
  skew       how unevenly experts are asked for, or rows are spread over requests
"""
import math

import torch

own = False
DEV = "cuda"


def _route(n, E, k, dtype="f32", gates="chosen", train=False, masked=False):
    return dict(op="route", n=n, E=E, k=k, dtype=dtype, gates=gates, train=train, masked=masked)


def _mix(n, k, n_out, dtype="bf16", train=False):
    return dict(op="mix", n=n, k=k, n_out=n_out, dtype=dtype, train=train)


def _experts(n, k, E, n_in, n_out, dtype="bf16", back=False, squash=False, gather=True, skew=0.5):
    return dict(op="experts", n=n, k=k, E=E, n_in=n_in, n_out=n_out, dtype=dtype, back=back, squash=squash,
                gather=gather, skew=skew)


def _adapters(n, requests, E, n_in, n_out, rank, dtype="bf16", back=False, squash=False, skew=1.0):
    return dict(op="adapters", n=n, requests=requests, E=E, n_in=n_in, n_out=n_out, rank=rank, dtype=dtype,
                back=back, squash=squash, skew=skew)


def listed():
    return [
        # one pattern asks an interactive program's router
        dict(_route(1, 16, 2), name="route_1"),
        # a training step's routing, gates over all experts, some experts closed to some patterns
        dict(_route(16384, 64, 4, "bf16", "all", True, True), name="route_train_16384"),
        # a few patterns' answers put together
        dict(_mix(9, 2, 512), name="mix_9"),
        # the same in a training step of wide experts, with its gradients
        dict(_mix(16384, 2, 2048, train=True), name="mix_train_16384"),
        # small float32 experts on letter windows: odd widths, a group of 512
        dict(_experts(512, 2, 8, 203, 120, "f32", squash=True), name="experts_f32_512"),
        # five patterns served: each chosen expert's weights are read for a row or two
        dict(_experts(5, 2, 16, 1024, 2048, squash=True), name="experts_few_5"),
        # a whole set's outputs from wide experts
        dict(_experts(16384, 2, 16, 2048, 2048, squash=True), name="experts_16384"),
        # a training step of many moderate experts, small ragged groups
        dict(_experts(1001, 2, 32, 1024, 512, back=True, skew=1.0), name="experts_back_1001"),
        # the widest experts' training step, hidden deltas and pooled changes
        dict(_experts(8192, 2, 8, 4096, 4096, back=True, squash=True, gather=False), name="experts_back_8192"),
        # one row each of 61 requests, each with its own adapter, out of 200
        dict(_adapters(61, 61, 200, 4096, 4096, 16, squash=True, skew=0.0), name="adapters_61"),
        # requests of very different lengths in one pass
        dict(_adapters(8192, 11, 6, 2048, 2048, 32, squash=True, skew=1.5), name="adapters_8192"),
        # a training step of several adapters at once
        dict(_adapters(16384, 7, 5, 4096, 4096, 64, back=True), name="adapters_back_16384"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Sizes over the listed cases' ranges; no more work than the largest of them."""
    top = 1.0e12
    while True:
        op = rng.choice(["route", "mix", "experts", "experts", "experts", "adapters", "adapters", "adapters"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if op == "route":
            E = _log(rng, 2, 128)
            return _route(_log(rng, 1, 16384), E, min(E, rng.randint(1, 6)), dtype, rng.choice(["chosen", "all"]),
                          rng.random() < 0.6, rng.random() < 0.4)
        if op == "mix":
            n_out = 8 * _log(rng, 4, 512) if dtype == "bf16" else _log(rng, 3, 1024)
            return _mix(_log(rng, 1, 16384), rng.randint(1, 4), n_out, dtype, rng.random() < 0.6)
        if dtype == "bf16":
            n_in, n_out = 8 * _log(rng, 8, 512), 8 * _log(rng, 4, 512)
        else:
            n_in, n_out = _log(rng, 16, 1024), _log(rng, 3, 1024)
        n, back, squash = _log(rng, 1, 16384), rng.random() < 0.45, rng.random() < 0.5
        if op == "experts":
            E = _log(rng, 2, 64)
            c = _experts(n, min(E, rng.randint(1, 4)), E, n_in, n_out, dtype, back, squash, rng.random() < 0.6,
                         round(rng.uniform(0.0, 1.5), 2))
        else:
            c = _adapters(n, min(n, _log(rng, 1, 256)), _log(rng, 1, 200), n_in, n_out, _log(rng, 1, 64), dtype, back,
                          squash, round(rng.uniform(0.0, 1.5), 2))
        w = work(c)
        if w["flops"] <= (top if dtype == "bf16" else 1.0e11) and w["bytes"] <= 4e9:
            return c


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# ------------------------------------------------------------------ inputs
def _lengths(n, parts, skew, g):
    """`parts` whole numbers that add up to n, spread the more unevenly the larger skew is."""
    w = torch.rand(parts, generator=g, device=DEV).double().add(1e-3).pow(skew * 2)
    ends = (w.cumsum(0) / w.sum() * n).round().long().clamp(0, n)
    ends[-1] = n
    return ends


def _order(expert, E):
    """The rows by expert: offsets, the pattern of each row, and each choice's row."""
    n, k = expert.shape
    flat = expert.reshape(-1).long()
    key = torch.where(flat < 0, torch.full_like(flat, E), flat)
    rows = torch.sort(key, stable=True).indices
    count = (flat.unsqueeze(1) == torch.arange(E, device=flat.device)).sum(0)
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=flat.device)
    offsets[1:] = count.cumsum(0)
    place = torch.empty_like(flat)
    place[rows] = torch.arange(n * k, device=flat.device)
    place = torch.where(flat < 0, torch.full_like(place, -1), place)
    used = torch.arange(n * k, device=flat.device) < offsets[-1]
    source = torch.where(used, rows // k, torch.full_like(rows, -1))
    return offsets.int(), source.int(), place.view(n, k).int()


def _inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = _type(case)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device=DEV) * scale).to(t)

    op, n = case["op"], case["n"]
    if op == "route":
        E, k = case["E"], case["k"]
        logits = torch.randn(n, E, generator=g, device=DEV) * 2 + torch.randn(E, generator=g, device=DEV)
        if case["masked"]:   # experts closed to a pattern; some patterns are left with none
            closed = torch.rand(n, E, generator=g, device=DEV) < 0.3
            closed |= torch.rand(n, 1, generator=g, device=DEV) < 0.01
            logits = logits.masked_fill(closed, float("-inf"))
        return dict(logits=logits.to(t), dgate=torch.randn(n, k, generator=g, device=DEV))
    if op == "mix":
        k, n_out = case["k"], case["n_out"]
        place = torch.randperm(n * k, generator=g, device=DEV).view(n, k).int()
        gate = torch.softmax(torch.randn(n, k, generator=g, device=DEV), 1)
        return dict(H=normal(n * k, n_out), place=place, gate=gate, D=normal(n, n_out))
    E, n_in, n_out = case["E"], case["n_in"], case["n_out"]
    if op == "experts":
        k = case["k"]
        logits = torch.randn(n, E, generator=g, device=DEV) + 2 * case["skew"] * torch.randn(E, generator=g, device=DEV)
        expert = torch.topk(logits, k, 1).indices
        offsets, source, _ = _order(expert, E)
        rows = n if case["gather"] else n * k
        x = torch.randn(rows, n_in, generator=g, device=DEV)
        x = (torch.sigmoid(x) if case["back"] and case["squash"] else x).to(t)
        s = dict(X=x, W=normal(E, n_out, n_in, scale=n_in ** -0.5), offsets=offsets,
                 source=source if case["gather"] else None)
        if case["back"]:
            s["D"] = normal(n * k, n_out, scale=0.25)
        else:
            s["b"] = torch.randn(E, n_out, generator=g, device=DEV) * 0.1
        return s
    R, r = case["requests"], case["rank"]
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), _lengths(n, R, case["skew"], g)]).int()
    adapter = torch.randint(0, E, (R,), generator=g, device=DEV).int()
    if R > 3:   # some requests ask the shared layer alone
        adapter[torch.rand(R, generator=g, device=DEV) < 0.1] = -1
    x = torch.randn(n, n_in, generator=g, device=DEV)
    x = (torch.sigmoid(x) if case["back"] and case["squash"] else x).to(t)
    s = dict(X=x, W=normal(n_out, n_in, scale=n_in ** -0.5), A=normal(E, r, n_in, scale=n_in ** -0.5),
             B=normal(E, r, n_out, scale=0.5 * r ** -0.5), offsets=offsets, adapter=adapter,
             scale=torch.rand(E, generator=g, device=DEV) + 0.5)
    if case["back"]:
        s["D"] = normal(n, n_out, scale=0.25)
        s["U"] = torch.zeros(n, r, device=DEV)
        for a, lo, hi in _spans(offsets, adapter):
            s["U"][lo:hi] = s["X"][lo:hi].float() @ s["A"][a].float().t()
    else:
        s["b"] = torch.randn(n_out, generator=g, device=DEV) * 0.1
    return s


def _spans(offsets, adapter):
    """(adapter, first row, end) of the requests that have an adapter and rows."""
    o = offsets.tolist()
    return [(a, o[i], o[i + 1]) for i, a in enumerate(adapter.tolist()) if a >= 0 and o[i + 1] > o[i]]


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    op, n, t = case["op"], case["n"], _type(case)
    if op == "adapters":   # a server keeps its requests' rows on the host too
        s["spans"] = _spans(s["offsets"], s["adapter"])
    elif op == "experts":
        s["counts"] = s["offsets"].tolist()
    if not own:
        return s
    from paper_1801_01554_gb300 import bp

    bt = bp.BP_BF16 if case["dtype"] == "bf16" else bp.BP_F32

    def empty(*shape, dtype=t):
        return torch.empty(*shape, dtype=dtype, device=DEV)

    if op == "route":
        E, k = case["E"], case["k"]
        s["router"] = bp.Router(E, k, dtype=bt, max_patterns=n,
                                gates=bp.BP_GATES_CHOSEN if case["gates"] == "chosen" else bp.BP_GATES_ALL)
        s.update(expert=empty(n, k, dtype=torch.int32), gate=empty(n, k, dtype=torch.float32),
                 offsets=empty(E + 1, dtype=torch.int32), source=empty(n * k, dtype=torch.int32),
                 place=empty(n, k, dtype=torch.int32), dlogits=empty(n, E))
    elif op == "mix":
        s.update(Y=empty(n, case["n_out"]), dH=empty(n * case["k"], case["n_out"]),
                 dgate=empty(n, case["k"], dtype=torch.float32))
    elif op == "experts":
        rows = n * case["k"]
        s["layer"] = bp.Experts(case["E"], case["n_in"], case["n_out"], dtype=bt, max_rows=rows)
        if case["back"]:
            s.update(dX=empty(rows, case["n_in"]), GW=empty(case["E"], case["n_out"], case["n_in"], dtype=torch.float32),
                     Gb=empty(case["E"], case["n_out"], dtype=torch.float32))
        else:
            s["Y"] = empty(rows, case["n_out"])
    else:
        s["layer"] = bp.Adapters(case["E"], case["rank"], case["n_in"], case["n_out"], dtype=bt, max_rows=n,
                                 max_requests=case["requests"])
        if case["back"]:
            s.update(dX=empty(n, case["n_in"]), GA=empty(case["E"], case["rank"], case["n_in"], dtype=torch.float32),
                     GB=empty(case["E"], case["rank"], case["n_out"], dtype=torch.float32))
        else:
            s.update(U=empty(n, case["rank"], dtype=torch.float32), Y=empty(n, case["n_out"]))
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_1801_01554_gb300 import bp

    c = s["case"]
    op, n = c["op"], c["n"]
    if op == "route":
        s["router"].forward(s["logits"], n, s["expert"], s["gate"], s["offsets"], s["source"], s["place"])
        out = {key: s[key] for key in ("expert", "gate", "offsets", "source", "place")}
        if c["train"]:
            s["router"].backward(s["logits"], n, s["expert"], s["gate"], s["dgate"], s["dlogits"])
            out["dlogits"] = s["dlogits"]
        return out
    if op == "mix":
        bt = bp.BP_BF16 if c["dtype"] == "bf16" else bp.BP_F32
        bp.bp_mix(s["H"], n * c["k"], s["place"], s["gate"], n, c["k"], c["n_out"], bt, s["Y"])
        if not c["train"]:
            return dict(Y=s["Y"])
        bp.bp_mix_backward(s["D"], s["H"], n * c["k"], s["place"], s["gate"], n, c["k"], c["n_out"], bt, s["dH"],
                           s["dgate"])
        return dict(Y=s["Y"], dH=s["dH"], dgate=s["dgate"])
    layer = s["layer"]
    if op == "experts":
        rows, n_x = n * c["k"], s["X"].shape[0]
        if c["back"]:
            layer.backward(s["W"], s["X"], n_x, s["source"], s["offsets"], rows, s["D"], dX=s["dX"], GW=s["GW"],
                           Gb=s["Gb"], squash=c["squash"])
            return dict(dX=s["dX"], GW=s["GW"], Gb=s["Gb"])
        layer.forward(s["W"], s["b"], s["X"], n_x, s["source"], s["offsets"], rows, s["Y"], squash=c["squash"])
        return dict(Y=s["Y"])
    if c["back"]:
        layer.backward(s["W"], s["A"], s["B"], s["scale"], s["X"], s["U"], s["offsets"], s["adapter"], c["requests"], n,
                       s["D"], dX=s["dX"], GA=s["GA"], GB=s["GB"], squash=c["squash"])
        return dict(dX=s["dX"], GA=s["GA"], GB=s["GB"])
    layer.forward(s["W"], s["b"], s["A"], s["B"], s["scale"], s["X"], s["offsets"], s["adapter"], c["requests"], n,
                  s["U"], s["Y"], squash=c["squash"])
    return dict(Y=s["Y"], U=s["U"])


def _run_plain(s):
    c, t = s["case"], _type(s["case"])
    op, n = c["op"], c["n"]
    if op == "route":
        E, k = c["E"], c["k"]
        z = s["logits"].float()
        top, expert = torch.sort(z, dim=1, descending=True, stable=True)   # ties: the lowest index first
        top, expert = top[:, :k], expert[:, :k].int()
        chosen = top > float("-inf")
        expert = torch.where(chosen, expert, torch.full_like(expert, -1))
        peak = torch.where(chosen[:, :1], top[:, :1], torch.zeros_like(top[:, :1]))
        up = torch.where(chosen, torch.exp(top - peak), torch.zeros_like(top))
        every = torch.exp(z - peak)
        total = (up if c["gates"] == "chosen" else every).sum(1, keepdim=True)
        total = torch.where(chosen[:, :1], total, torch.ones_like(total))
        gate = up / total
        offsets, source, place = _order(expert, E)
        out = dict(expert=expert, gate=gate, offsets=offsets, source=source, place=place)
        if c["train"]:
            dg = s["dgate"] * gate
            pull = dg.sum(1, keepdim=True)
            p = every / total if c["gates"] == "all" else torch.zeros_like(z)
            d = -p * pull
            at = expert.clamp(min=0).long()
            d = d.scatter_add(1, at, dg if c["gates"] == "all" else dg - gate * pull)
            out["dlogits"] = d.to(t)
        return out
    if op == "mix":
        rows = s["H"].float()[s["place"].long()]
        y = (rows * s["gate"].unsqueeze(2)).sum(1).to(t)
        if not c["train"]:
            return dict(Y=y)
        d = s["D"].float()
        dh = torch.empty(s["H"].shape, dtype=t, device=DEV)
        dh[s["place"].long().view(-1)] = (s["gate"].unsqueeze(2) * d.unsqueeze(1)).view(-1, d.shape[1]).to(t)
        return dict(Y=y, dH=dh, dgate=(rows * d.unsqueeze(1)).sum(2))
    x, w = s["X"].float(), s["W"].float()
    if op == "experts":
        o = s["counts"]
        if s["source"] is not None:
            x = x[s["source"].long()]
        groups = [(e, o[e], o[e + 1]) for e in range(c["E"]) if o[e + 1] > o[e]]
        if not c["back"]:
            y = torch.empty(n * c["k"], c["n_out"], device=DEV)
            for e, lo, hi in groups:
                y[lo:hi] = x[lo:hi] @ w[e].t() + s["b"][e]
            return dict(Y=(1 / (1 + torch.exp(-y)) if c["squash"] else y).to(t))
        d = s["D"].float()
        dx = torch.empty_like(x)
        gw = torch.zeros(c["E"], c["n_out"], c["n_in"], device=DEV)
        gb = torch.zeros(c["E"], c["n_out"], device=DEV)
        for e, lo, hi in groups:
            dx[lo:hi] = d[lo:hi] @ w[e]
            gw[e] = d[lo:hi].t() @ x[lo:hi]
            gb[e] = d[lo:hi].sum(0)
        return dict(dX=(dx * x * (1 - x) if c["squash"] else dx).to(t), GW=gw, Gb=gb)
    a, b, scale = s["A"].float(), s["B"].float(), s["scale"]
    if not c["back"]:
        y = x @ w.t() + s["b"]
        u = torch.zeros(n, c["rank"], device=DEV)
        for i, lo, hi in s["spans"]:
            u[lo:hi] = x[lo:hi] @ a[i].t()
            y[lo:hi] += scale[i] * (u[lo:hi] @ b[i])
        return dict(Y=(1 / (1 + torch.exp(-y)) if c["squash"] else y).to(t), U=u)
    d = s["D"].float()
    dx = d @ w
    ga, gb = torch.zeros_like(a), torch.zeros_like(b)
    for i, lo, hi in s["spans"]:
        du = scale[i] * (d[lo:hi] @ b[i].t())
        dx[lo:hi] += du @ a[i]
        ga[i] += du.t() @ x[lo:hi]
        gb[i] += scale[i] * (s["U"][lo:hi].t() @ d[lo:hi])
    return dict(dX=(dx * x * (1 - x) if c["squash"] else dx).to(t), GA=ga, GB=gb)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op, n = case["op"], case["n"]
    e = 2 if case["dtype"] == "bf16" else 4
    if op == "route":
        E, k = case["E"], case["k"]
        rows = n * k
        b, f = n * E * e + 4 * (4 * rows + E + 1), 4 * n * E
        if case["train"]:
            b, f = b + 4 * rows + n * E * e, f + 4 * n * E
        return dict(bytes=b, flops=f)
    if op == "mix":
        rows, o = n * case["k"], case["n_out"]
        b, f = (rows + n) * o * e + 8 * rows, 2 * rows * o
        if case["train"]:
            b, f = b + (n + rows) * o * e + 4 * rows, f + 3 * rows * o
        return dict(bytes=b, flops=f)
    i, o = case["n_in"], case["n_out"]
    if op == "experts":
        rows, E = n * case["k"], case["E"]
        x = (n if case["gather"] else rows) * i * e + (4 * rows if case["gather"] else 0)
        w = min(E, rows) * i * o * e   # the experts that have rows
        if case["back"]:
            return dict(bytes=x + w + rows * (i + o) * e + 4 * E * (i + 1) * o, flops=4 * rows * i * o)
        return dict(bytes=x + w + rows * o * e + 4 * min(E, rows) * o, flops=2 * rows * i * o)
    r, R = case["rank"], case["requests"]
    pairs = min(case["E"], R) * r * (i + o) * e + 8 * R
    if case["back"]:
        return dict(bytes=n * (2 * i + o) * e + 4 * n * r + i * o * e + pairs + 4 * case["E"] * r * (i + o),
                    flops=2 * n * i * o + 4 * n * r * (i + o))
    return dict(bytes=n * (i + o) * e + 4 * n * r + i * o * e + 4 * o + pairs, flops=2 * n * i * o + 2 * n * r * (i + o))


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    if work(case)["flops"] > 8e12:
        return None
    s = _inputs(case, seed)
    op, n = case["op"], case["n"]
    sig = torch.sigmoid
    if op == "route":
        z, k, E = s["logits"].double(), case["k"], case["E"]
        gate = torch.zeros(n, k, dtype=torch.float64, device=DEV)
        weight = torch.zeros(n, E, dtype=torch.float64, device=DEV)   # of the chosen experts alone
        left = z.clone()
        picks = []
        for j in range(k):
            best = left.max(1, keepdim=True).values
            pick = (left == best).to(torch.int8).argmax(1, keepdim=True)
            picks.append((pick, best > -math.inf))
            left = left.scatter(1, pick, -math.inf)
        # log of the total over the gates' experts; a pattern with none has no gates
        logs = torch.cat([torch.where(ok, z.gather(1, p), torch.full_like(z[:, :1], -math.inf)) for p, ok in picks], 1)
        total = torch.logsumexp(z if case["gates"] == "all" else logs, 1, keepdim=True)
        for j, (p, ok) in enumerate(picks):
            gate[:, j:j + 1] = torch.where(ok, torch.exp(z.gather(1, p) - total), torch.zeros_like(total))
        out = dict(expert=None, gate=gate, offsets=None, source=None, place=None)
        if case["train"]:
            dg = s["dgate"].double()
            mean = (gate * dg).sum(1, keepdim=True)
            for j, (p, ok) in enumerate(picks):
                weight.scatter_add_(1, p, torch.where(ok, gate[:, j:j + 1] * dg[:, j:j + 1], torch.zeros_like(mean)))
            if case["gates"] == "all":
                spread = torch.exp(z - total)
            else:
                spread = torch.zeros_like(z)
                for j, (p, ok) in enumerate(picks):
                    spread.scatter_add_(1, p, gate[:, j:j + 1])
            none = ~picks[0][1]
            out["dlogits"] = torch.where(none, torch.zeros_like(z), weight - spread * mean)
        return out
    if op == "mix":
        h, gate, place = s["H"].double(), s["gate"].double(), s["place"].long()
        y = torch.zeros(n, case["n_out"], dtype=torch.float64, device=DEV)
        for j in range(case["k"]):
            y += gate[:, j:j + 1] * h[place[:, j]]
        if not case["train"]:
            return dict(Y=y)
        d = s["D"].double()
        dh, dgate = torch.empty_like(h), torch.empty_like(gate)
        for j in range(case["k"]):
            dh[place[:, j]] = gate[:, j:j + 1] * d
            dgate[:, j] = torch.einsum("no,no->n", h[place[:, j]], d)
        return dict(Y=y, dH=dh, dgate=dgate)
    i, o = case["n_in"], case["n_out"]
    x = s["X"].double()
    if op == "experts":
        rows, ends = n * case["k"], s["offsets"].tolist()
        if s["source"] is not None:
            x = x.index_select(0, s["source"].long())
        if not case["back"]:
            y = torch.zeros(rows, o, dtype=torch.float64, device=DEV)
            for e in range(case["E"]):
                part = slice(ends[e], ends[e + 1])
                y[part] = torch.addmm(s["b"][e].double(), x[part], s["W"][e].double().t())
            return dict(Y=sig(y) if case["squash"] else y)
        d = s["D"].double()
        out = dict(dX=torch.zeros(rows, i, dtype=torch.float64, device=DEV),
                   GW=torch.zeros(case["E"], o, i, dtype=torch.float64, device=DEV),
                   Gb=torch.zeros(case["E"], o, dtype=torch.float64, device=DEV))
        for e in range(case["E"]):
            part = slice(ends[e], ends[e + 1])
            slope = x[part] * (1 - x[part]) if case["squash"] else 1.0
            out["dX"][part] = torch.mm(d[part], s["W"][e].double()) * slope
            out["GW"][e] = torch.mm(d[part].t(), x[part])
            out["Gb"][e] = d[part].sum(0)
        return out
    w, a, b, scale = s["W"].double(), s["A"].double(), s["B"].double(), s["scale"].double()
    at, r = s["offsets"].tolist(), case["rank"]
    u = torch.zeros(n, r, dtype=torch.float64, device=DEV)
    if not case["back"]:
        y = torch.empty(n, o, dtype=torch.float64, device=DEV)
        for q, g in enumerate(s["adapter"].tolist()):   # the request's own dense weights
            part, full = slice(at[q], at[q + 1]), w
            if at[q + 1] == at[q]:
                continue
            if g >= 0:
                u[part] = x[part] @ a[g].t()
                if at[q + 1] - at[q] > 64:
                    full = w + scale[g] * (b[g].t() @ a[g])
            y[part] = x[part] @ full.t() + s["b"].double()
            if g >= 0 and full is w:
                y[part] += scale[g] * (u[part] @ b[g])
        return dict(Y=sig(y) if case["squash"] else y, U=u)
    d = s["D"].double()
    u = s["U"].double()
    out = dict(dX=torch.mm(d, w), GA=torch.zeros_like(a), GB=torch.zeros_like(b))
    for q, g in enumerate(s["adapter"].tolist()):
        if g < 0:
            continue
        part = slice(at[q], at[q + 1])
        v = d[part] @ (scale[g] * b[g]).t()
        out["dX"][part] += v @ a[g]
        out["GA"][g] += v.t() @ x[part]
        out["GB"][g] += (scale[g] * u[part]).t() @ d[part]
    if case["squash"]:
        out["dX"] *= x * (1 - x)
    return out
