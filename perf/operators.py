"""The operators around an ensemble's answer, as cases to be timed.

A gate chooses members for each row (route), their softmax outputs are combined with the row's own weights (combine), the best classes
of a row are kept (top), and a student learns from kept classes (distill).  A case is one pass through one of them, from the tensors a
program holds to the tensors it goes on with.  Where `own` is false a pass is written in elementary tensor operations, where it is
true it calls the library.

Fields of a case:
  op        "route", "combine", "top" or "distill"
  rows      rows of the call: images, or positions of text
  members   route, combine: members of the ensemble (the gate's columns)
  classes   combine, top, distill: length of a row
  k         members chosen for a row (route, combine), classes kept of a row (top, distill)
  dtype     type of the gate's values or of the logits: "fp32", "bf16" or "fp16"
  way       "forward"; "backward": forward and then backward, as two calls; "gradient" (distill): the loss and the gradient of the
            weighted sum of losses in one call
  score     route: "softmax" or "sigmoid"
  balance   route: whether a bias for balance is added to the scores when members are chosen
  groups, kept   route: the members stand in `groups` groups, of which `kept` stay
  form      top: "value", "log" or "log_softmax"
  tail      distill: whether what the teacher gave to the classes that it did not keep counts as one class more
  warm      top, distill: temperature
"""
import math

import torch

own = False                     # set from outside: whether run() calls the library

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
NO = float("-inf")


def _route(name, rows, members, k, dtype, way, score, balance, groups=1, kept=1):
    return dict(name=name, op="route", rows=rows, members=members, k=k, dtype=dtype, way=way, score=score, balance=balance, groups=groups, kept=kept)


def _combine(name, rows, members, classes, k, dtype, way):
    return dict(name=name, op="combine", rows=rows, members=members, classes=classes, k=k, dtype=dtype, way=way)


def _top(name, rows, classes, k, dtype, form, warm=1.0):
    return dict(name=name, op="top", rows=rows, classes=classes, k=k, dtype=dtype, way="forward", form=form, warm=warm)


def _distill(name, rows, classes, k, dtype, way, tail, warm):
    return dict(name=name, op="distill", rows=rows, classes=classes, k=k, dtype=dtype, way=way, tail=tail, warm=warm)


def listed():
    return [
        # one image in front of the twelve-member ensemble: which two members answer it
        _route("route_one", 1, 12, 2, "fp32", "forward", "softmax", False),
        # a training step of a gate over as many members as a handle holds, in groups, balanced by a bias
        _route("route_groups_train", 4097, 64, 6, "bf16", "backward", "sigmoid", True, 8, 3),
        # a gate over many experts, for the positions of a large batch of text
        _route("route_wide_train", 32768, 256, 8, "bf16", "backward", "softmax", False),
        # the chosen two of twelve members for one image
        _combine("combine_one", 1, 12, 1000, 2, "fp32", "forward"),
        # an offline request through a routed ensemble of twelve classifiers
        _combine("combine_bulk", 8100, 12, 1000, 3, "fp32", "forward"),
        # a training step through four members over a vocabulary, gradients of the gate's weights and of every member's logits
        _combine("combine_train", 1023, 4, 32001, 2, "bf16", "backward"),
        # the candidates for one next token
        _top("top_one", 1, 128000, 50, "bf16", "log_softmax", 0.7),
        # the five best classes of every image of an offline request
        _top("top_bulk", 8100, 1000, 5, "fp32", "log"),
        # a teacher's record for distillation
        _top("top_record", 1500, 50001, 100, "fp16", "log_softmax", 2.0),
        # a classifier's batch against an ensemble's five best classes, the two directions as calls of their own
        _distill("distill_batch", 64, 1000, 5, "fp32", "backward", False, 2.0),
        # a ragged batch of positions, what the teacher did not keep as one class more
        _distill("distill_tail", 1021, 50001, 64, "bf16", "gradient", True, 1.0),
        # a training step's positions over a large vocabulary
        _distill("distill_large", 4096, 128000, 50, "bf16", "gradient", False, 1.5),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(("route", "combine", "top", "distill"))
    dtype = rng.choice(("fp32", "bf16", "fp16"))
    if op == "route":
        groups = rng.choice((1, 1, 2, 4, 8))
        members = groups * _spread(rng, 2, 256 // groups)
        kept = rng.randint(1, groups)
        k = rng.randint(1, min(16, members // groups * kept))
        c = _route("", _spread(rng, 1, 32768), members, k, dtype, rng.choice(("forward", "backward")), rng.choice(("softmax", "sigmoid")),
                   rng.random() < 0.5, groups, kept)
    elif op == "combine":
        members = rng.randint(1, 24)
        k, classes = rng.randint(1, min(members, 6)), _spread(rng, 2, 65000)
        rows = _spread(rng, 1, max(1, min(16384, 100_000_000 // (members * classes))))
        c = _combine("", rows, members, classes, k, dtype, rng.choice(("forward", "backward")))
    elif op == "top":
        classes = _spread(rng, 128, 200_000)
        rows = _spread(rng, 1, max(1, min(16384, 75_000_000 // classes)))
        form = rng.choice(("value", "log", "log_softmax"))
        c = _top("", rows, classes, _spread(rng, 1, 128), dtype, form, rng.choice((0.7, 1.0, 2.0)) if form == "log_softmax" else 1.0)
    else:
        classes = _spread(rng, 256, 200_000)
        rows = _spread(rng, 1, max(1, min(16384, 150_000_000 // classes)))
        c = _distill("", rows, classes, _spread(rng, 1, 128), dtype, rng.choice(("forward", "backward", "gradient")), rng.random() < 0.5,
                     rng.choice((1.0, 1.5, 2.0, 4.0)))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------- inputs

def _some(n, total, k, g):
    """k different numbers below `total` for each of n rows, in no order."""
    step = total // k
    first = torch.randint(0, total, (n, 1), device="cuda", generator=g)
    return (first + step * torch.arange(k, device="cuda") + torch.randint(0, step, (n, k), device="cuda", generator=g)) % total


def _ragged(n, k, g):
    """Which entries of n records of k are there: most records are whole, some hold fewer."""
    whole = torch.rand((n, 1), device="cuda", generator=g) < 0.95
    return whole | (torch.rand((n, k), device="cuda", generator=g) < 0.6)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n, k, t = case["rows"], case["k"], TYPES[case["dtype"]]
    s = dict(case)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return torch.randn(shape, device="cuda", dtype=dtype, generator=g).mul_(scale)

    if case["op"] == "route":
        s["gates"] = normal(n, case["members"], scale=1.5, dtype=t)
        s["bias"] = normal(case["members"], scale=0.05) if case["balance"] else None
        s["d_weights"] = normal(n, k)
    elif case["op"] == "combine":
        s["logits"] = normal(case["members"], n, case["classes"], scale=2.0, dtype=t)
        here = _ragged(n, k, g)
        members = _some(n, case["members"], k, g)
        s["chosen"] = torch.where(here, members, -1).int()
        weights = torch.rand((n, k), device="cuda", generator=g) + 0.05
        s["weights"] = torch.where(here, weights / weights.sum(1, keepdim=True), 0.0)
        s["d_probs"] = normal(n, case["classes"]) if case["way"] == "backward" else None
    elif case["op"] == "top":
        values = normal(n, case["classes"], scale=3.0, dtype=t)
        s["values"] = torch.softmax(values.float(), 1).to(t) if case["form"] == "log" else values
    else:
        s["logits"] = normal(n, case["classes"], scale=2.0, dtype=t)
        index = _some(n, case["classes"], k, g)
        # the student has learnt something: what the teacher kept stands out among its logits
        s["logits"].scatter_add_(1, index, (4.0 * torch.rand((n, k), device="cuda", generator=g)).to(t))
        here = _ragged(n, k, g)
        s["index"] = torch.where(here, index, -1).int()
        kept = 0.5 + 0.45 * torch.rand((n, 1), device="cuda", generator=g)
        s["log_probs"] = torch.log_softmax(normal(n, k, scale=2.0), 1) + kept.log()
        # padding has no weight
        s["row_weights"] = (2.0 * torch.rand((n,), device="cuda", generator=g) - 0.1).clamp(min=0.0)
    return s


# ------------------------------------------------------------------------------------- passes

def run(s):
    return {"route": _run_route, "combine": _run_combine, "top": _run_top, "distill": _run_distill}[s["op"]](s)


def _library():
    import paper_2208_14049_amd as ens
    return ens


def _run_route(s):
    gates, backward, members, k = s["gates"], s["way"] == "backward", s["members"], s["k"]
    if own:
        ens = _library()
        load = torch.zeros(members, dtype=torch.int32, device=gates.device)
        chosen, weights = ens.ens_route(gates, k, score=s["score"], bias=s["bias"], groups=s["groups"], groups_kept=s["kept"], load=load)
        out = [chosen, weights, load]
        if backward:
            out.append(ens.ens_route_backward(gates, chosen, s["d_weights"], score=s["score"]))
        return out
    # members are chosen next to borders between nearly equal scores: in 64 bits
    x = gates.double()
    n = x.shape[0]
    e = torch.exp(x - x.amax(1, keepdim=True))
    score = e / e.sum(1, keepdim=True) if s["score"] == "softmax" else 1 / (1 + torch.exp(-x))
    choice = x if s["bias"] is None and s["groups"] == 1 else score if s["bias"] is None else score + s["bias"].double()
    if s["groups"] > 1:
        parts = choice.view(n, s["groups"], -1)
        best = torch.sort(parts, dim=2, descending=True).values[:, :, :2].sum(2)
        kept = torch.sort(best, dim=1, descending=True, stable=True).indices[:, : s["kept"]]
        mask = torch.zeros_like(best, dtype=torch.bool).scatter_(1, kept, True)
        choice = torch.where(mask.unsqueeze(2), parts, NO).view(n, -1)
    chosen = torch.sort(choice, dim=1, descending=True, stable=True).indices[:, :k]
    picked = score.gather(1, chosen)
    share = picked / picked.sum(1, keepdim=True)
    load = torch.zeros(members, dtype=torch.int32, device=x.device).index_add_(0, chosen.reshape(-1), torch.ones_like(chosen, dtype=torch.int32).reshape(-1))
    out = [chosen.int(), share.float(), load]
    if backward:
        d = s["d_weights"].double()
        d = share * (d - (share * d).sum(1, keepdim=True))
        if s["score"] == "sigmoid":
            d = d * (1 - picked)
        out.append(torch.zeros_like(x).scatter_(1, chosen, d).to(gates.dtype))
    return out


def _run_combine(s):
    logits, chosen, weights, backward = s["logits"], s["chosen"], s["weights"], s["way"] == "backward"
    if own:
        ens = _library()
        probs, lse = ens.ens_combine_routed(logits, chosen, weights)
        if not backward:
            return [probs]
        d_weights, d_logits = ens.ens_combine_routed_backward(logits, chosen, weights, lse, s["d_probs"])
        return [probs, d_weights, d_logits]
    here = chosen >= 0
    rows = torch.arange(chosen.shape[0], device=chosen.device).unsqueeze(1)
    member = chosen.clamp(min=0).long()
    z = logits[member, rows].float()                             # row, choice, class
    e = torch.exp(z - z.amax(2, keepdim=True))
    p = e / e.sum(2, keepdim=True)
    w = (weights * here).unsqueeze(2)
    probs = (w * p).sum(1)
    if not backward:
        return [probs]
    g = s["d_probs"].unsqueeze(1)
    d_weights = (p * g).sum(2) * here
    d = (w * p * (g - d_weights.unsqueeze(2))).to(logits.dtype)
    # a choice that is not there goes to a place of its own behind the members
    d_logits = torch.zeros((logits.shape[0] + 1,) + tuple(logits.shape[1:]), dtype=logits.dtype, device=logits.device)
    d_logits[torch.where(here, member, logits.shape[0]), rows] = d
    return [probs, d_weights, d_logits[:-1]]


def _run_top(s):
    if own:
        return list(_library().ens_top(s["values"], s["k"], form=s["form"], temperature=s["warm"]))
    x = s["values"].float()
    found = torch.sort(x, dim=1, descending=True, stable=True)
    value, index = found.values[:, : s["k"]], found.indices[:, : s["k"]].int()
    if s["form"] == "log":
        value = value.log()
    if s["form"] == "log_softmax":
        z = x / s["warm"]
        m = z.amax(1, keepdim=True)
        value = value / s["warm"] - m - torch.exp(z - m).sum(1, keepdim=True).log()
    return [index, value]


def _run_distill(s):
    logits, index, t, tail, warm = s["logits"], s["index"], s["log_probs"], s["tail"], s["warm"]
    w = s["row_weights"]
    if own:
        ens = _library()
        if s["way"] == "gradient":
            loss, lse, d = ens.ens_distill(logits, index, t, temperature=warm, tail=tail, row_weights=w, gradient=True)
            return [loss, d]
        loss, lse = ens.ens_distill(logits, index, t, temperature=warm, tail=tail)
        if s["way"] == "forward":
            return [loss]
        return [loss, ens.ens_distill_backward(logits, index, t, lse, d_loss=w, temperature=warm, tail=tail)]
    here = index >= 0
    some = here.any(1, keepdim=True)
    at = index.clamp(min=0).long()
    if tail:
        q = torch.where(here, t.exp(), 0.0)
        q0 = (1 - q.sum(1, keepdim=True)).clamp(min=0)
    else:
        q = torch.where(here, torch.exp(t - t.masked_fill(~here, NO).amax(1, keepdim=True)), 0.0)
        q = torch.where(some, q / q.sum(1, keepdim=True), 0.0)
    z = logits.float() / warm
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    log_p = z.gather(1, at) - m - total.log()
    loss = torch.where(q > 0, q * (torch.log(q) - log_p), 0.0).sum(1, keepdim=True)
    if tail:
        # what is not there has no place in the row: it is marked in one more column
        listed_ = torch.zeros((z.shape[0], z.shape[1] + 1), dtype=torch.bool, device=z.device)
        listed_ = listed_.scatter_(1, torch.where(here, at, z.shape[1]), True)[:, :-1]
        rest = e.masked_fill(listed_, 0.0).sum(1, keepdim=True)
        loss = loss + torch.where(q0 > 0, q0 * (torch.log(q0) - torch.log(rest / total)), 0.0)
    loss = (loss * warm * warm).squeeze(1)
    if s["way"] == "forward":
        return [loss]
    scale = w.unsqueeze(1) * warm
    mass = q.sum(1, keepdim=True) + (q0 if tail else 0.0)
    d = e * (mass / total)
    if tail:
        d = d - (e * (q0 / rest)).masked_fill(listed_, 0.0)
    d.scatter_add_(1, at, -q)
    return [loss, (d * scale).to(logits.dtype)]


# ------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    n, k, b, op = case["rows"], case["k"], BYTES[case["dtype"]], case["op"]
    backward = case["way"] != "forward"
    if op == "route":
        e = case["members"]
        return {"bytes": n * e * b + 8 * n * k + 4 * e + (2 * n * e * b + 8 * n * k if backward else 0), "flops": 8 * n * e}
    c = case["classes"]
    if op == "combine":
        forward = n * k * c * b + 4 * n * c + 8 * n * k
        return {"bytes": forward + (n * k * c * b + 4 * n * c + case["members"] * n * c * b + 4 * n * k if backward else 0),
                "flops": 4 * n * k * c * (2 if backward else 1)}
    if op == "top":
        return {"bytes": n * c * b + 8 * n * k, "flops": n * c * (4 if case["form"] == "log_softmax" else 1)}
    reads, writes = {"forward": (1, 0), "gradient": (1, 1), "backward": (2, 1)}[case["way"]]
    return {"bytes": (reads + writes) * n * c * b + 8 * n * k + 8 * n, "flops": 4 * n * c * (reads + writes)}


# ------------------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"route": _exact_route, "combine": _exact_combine, "top": _exact_top, "distill": _exact_distill}[case["op"]](s)


def _log_score(s, x):
    """Logarithm of the gate's scores."""
    if s["score"] == "softmax":
        return torch.log_softmax(x, 1)
    return -torch.logaddexp(torch.zeros_like(x), -x)


def _exact_route(s):
    x = s["gates"].double().requires_grad_(s["way"] == "backward")
    log_score = _log_score(s, x)
    with torch.no_grad():
        rank = log_score.exp() + (0.0 if s["bias"] is None else s["bias"].double())
        if s["bias"] is None and s["groups"] == 1:
            rank = s["gates"].double()
        size = s["members"] // s["groups"]
        if s["groups"] > 1:
            best = rank.unflatten(1, (s["groups"], size)).topk(min(2, size), dim=2).values.sum(2)
            order = (-best).argsort(dim=1, stable=True).argsort(dim=1)
            rank = rank.masked_fill((order >= s["kept"]).repeat_interleave(size, 1), NO)
        chosen = (-rank).argsort(dim=1, stable=True)[:, : s["k"]]
    weights = torch.softmax(log_score.gather(1, chosen), 1)
    out = [chosen.int(), weights.detach(), torch.bincount(chosen.flatten(), minlength=s["members"]).int()]
    if s["way"] == "backward":
        out.append(torch.autograd.grad(weights, x, s["d_weights"].double())[0])
    return out


def _exact_combine(s):
    members, n, classes = s["logits"].shape
    backward = s["way"] == "backward"
    weights = s["weights"].double()
    probs = torch.zeros((n, classes), dtype=torch.float64, device=weights.device)
    d_weights = torch.zeros_like(weights)
    d_logits = torch.zeros((members, n, classes), dtype=torch.float64, device=weights.device) if backward else None
    for m in range(members):                                     # the mixture, member by member
        hit = s["chosen"] == m
        row = hit.any(1).nonzero().squeeze(1)
        share = (weights * hit).sum(1)[row].unsqueeze(1)
        p = torch.softmax(s["logits"][m, row].double(), 1)
        probs[row] += share * p
        if backward:
            g = s["d_probs"][row].double()
            dot = (g * p).sum(1, keepdim=True)
            d_weights[row] += hit[row] * dot
            d_logits[m, row] = share * (p * g - p * dot)
    return [probs, d_weights, d_logits] if backward else [probs]


def _exact_top(s):
    x = s["values"].double()
    index = (-x).argsort(dim=1, stable=True)[:, : s["k"]]
    if s["form"] == "log":
        x = x.log()
    if s["form"] == "log_softmax":
        x = torch.log_softmax(x / s["warm"], 1)
    return [index.int(), x.gather(1, index)]


def _exact_distill(s):
    """The divergence between two whole distributions and its derivative, some rows at a time."""
    n, classes = s["logits"].shape
    warm, outs = s["warm"], []
    for a in range(0, n, 512):
        index, t = s["index"][a:a + 512].long(), s["log_probs"][a:a + 512].double()
        there = index >= 0
        slot = torch.where(there, index, classes)
        log_p = torch.log_softmax(s["logits"][a:a + 512].double() / warm, 1)
        q = t.exp() * there
        if not s["tail"]:
            q = q / q.sum(1, keepdim=True).clamp(min=1e-300)
        dense = torch.zeros((q.shape[0], classes + 1), dtype=torch.float64, device=q.device).scatter_add_(1, slot, q)[:, :-1]
        loss = (torch.xlogy(dense, dense) - torch.where(dense > 0, dense * log_p, 0.0)).sum(1)
        d = log_p.exp() * dense.sum(1, keepdim=True) - dense
        if s["tail"]:
            free = torch.ones((q.shape[0], classes + 1), dtype=torch.bool, device=q.device).scatter_(1, slot, False)[:, :-1]
            q0 = (1 - q.sum(1)).clamp(min=0)
            log_rest = torch.logsumexp(log_p.masked_fill(~free, NO), 1)
            loss = loss + torch.xlogy(q0, q0) - q0 * log_rest
            inside = torch.where(free, (log_p - log_rest.unsqueeze(1)).exp(), 0.0)
            d = d + q0.unsqueeze(1) * (log_p.exp() - inside)
        w = s["row_weights"][a:a + 512].double()
        outs.append((warm * warm * loss, (warm * w).unsqueeze(1) * d if s["way"] != "forward" else None))
    if s["way"] == "forward":
        return [torch.cat([o[0] for o in outs])]
    return [torch.cat([o[i] for o in outs]) for i in range(2)]
