"""The operators around a row of logits that a policy or a classifier acts and
learns with: drawing actions (temperature, top-k, top-p, min-p) from given
random numbers, the top logits of a teacher with their log-probabilities, and
the loss and gradient of a student that is taught by them.

`listed()` and `draw(rng)` give their workloads, `run(state)` one call of one
of them: the plain form in elementary torch operations, or, where `own` is
true, the library's kernels.
"""
import math

import torch

own = False  # False: the plain forms; True: the library's entry points

MOST = 256  # top logits of a row


def listed():
    return [
        # a policy acts on one small graph's nodes, 7 actions: latency counts
        dict(name="act_small", op="sample", n=256, C=7, ld=7, mask=0.0, skip=0.0,
             T=1.0, top_k=0, top_p=1.0, min_p=0.0),
        # an 8,000-node subgraph, 41 classes, the Trainer's padded rows, nucleus
        dict(name="act_8k", op="sample", n=8000, C=41, ld=44, mask=0.0, skip=0.0,
             T=0.7, top_k=0, top_p=0.9, min_p=0.0),
        # a large batch over 121 classes at an odd stride, a tenth of the rows
        # padding (NaN logits), everything switched on
        dict(name="act_ragged", op="sample", n=50001, C=121, ld=121, mask=0.0, skip=0.1,
             T=1.3, top_k=20, top_p=0.95, min_p=0.02),
        # 16,384 rows of 2,048 actions, nucleus
        dict(name="act_wide", op="sample", n=16384, C=2048, ld=2048, mask=0.0, skip=0.0,
             T=1.0, top_k=0, top_p=0.9, min_p=0.0),
        # 64 graphs, each drawing one of a full graph's 131,071 nodes, a third
        # of them not allowed (-inf)
        dict(name="act_nodes", op="sample", n=64, C=131071, ld=131072, mask=0.33, skip=0.0,
             T=0.8, top_k=1000, top_p=0.95, min_p=0.0),
        # a teacher's answers for a subgraph of 8,000 nodes
        dict(name="top_8k", op="top", n=8000, C=41, ld=44, mask=0.0, skip=0.0, k=8, T=2.0),
        # 64 of 2,048, and 128 of an odd number that fills a block
        dict(name="top_wide", op="top", n=16384, C=2048, ld=2048, mask=0.0, skip=0.0, k=64, T=1.0),
        dict(name="top_long", op="top", n=2000, C=20011, ld=20011, mask=0.0, skip=0.0, k=128,
             T=1.0),
        # a student taught by four of seven classes: latency
        dict(name="distill_small", op="distill", n=256, C=7, ld=7, mask=0.0, skip=0.0, k=4,
             T=2.0, rest=True),
        # the large ragged batch, rows without a teacher among them
        dict(name="distill_ragged", op="distill", n=50001, C=121, ld=121, mask=0.0, skip=0.1,
             k=16, T=2.0, rest=True),
        # 64 of 2,048, without the rest
        dict(name="distill_wide", op="distill", n=16384, C=2048, ld=2048, mask=0.0, skip=0.0,
             k=64, T=1.0, rest=False),
        # one distribution over a full graph's nodes for each of 64 graphs
        dict(name="distill_nodes", op="distill", n=64, C=131071, ld=131072, mask=0.33, skip=0.0,
             k=256, T=1.0, rest=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["sample", "sample", "top", "distill"])
    C = _log_int(rng, 2, 131072)
    n = _log_int(rng, 1, min(200000, 33000000 // C))
    c = dict(op=op, n=n, C=C, ld=rng.choice([C, (C + 3) // 4 * 4, C + rng.randint(1, 9)]),
             mask=round(rng.choice([0.0, 0.0, 0.5 * rng.random()]), 2),
             skip=round(rng.choice([0.0, 0.0, 0.9 * rng.random()]), 2),
             T=round(0.3 * 10.0 ** rng.random(), 3))
    if op == "sample":
        c["T"] = rng.choice([c["T"], 1.0, 0.0, c["T"]])
        c["top_k"] = rng.choice([0, 0, _log_int(rng, 1, C)])
        c["top_p"] = rng.choice([1.0, round(1.0 - 0.7 * rng.random() ** 2, 3)])
        c["min_p"] = rng.choice([0.0, 0.0, round(0.3 * rng.random(), 3)])
        return c
    c["k"] = _log_int(rng, 1, min(MOST, C))
    if op == "distill":
        c["rest"] = c["k"] < C and rng.random() < 0.5
    return c


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _logits(case, g):
    n, C = case["n"], case["C"]
    Z = torch.randn((n, case["ld"]), device="cuda", generator=g)[:, :C].mul_(2.0)
    if case["mask"]:  # actions that are not allowed
        Z.masked_fill_(torch.rand((n, C), device="cuda", generator=g) < case["mask"], -math.inf)
        Z[:, 0] = 0.0  # one always is
    return Z


def prepare(case, seed):
    g = _gen(seed)
    n, C, op = case["n"], case["C"], case["op"]
    Z = _logits(case, g)
    s = dict(case=case, Z=Z)
    skip = torch.rand(n, device="cuda", generator=g) < case["skip"]
    if op == "sample":
        s["u"] = torch.rand(n, device="cuda", generator=g)
        s["action"] = torch.empty(n, dtype=torch.int32, device="cuda")
        s["logp"] = torch.empty(n, device="cuda")
    elif op == "top":
        k = case["k"]
        s["index"] = torch.empty((n, k), dtype=torch.int32, device="cuda")
        s["logq"] = torch.empty((n, k), device="cuda")
        s["rest"] = torch.empty(n, device="cuda")
    else:
        # the teacher: the student's logits and what it has still to learn
        t = (Z + 0.7 * torch.randn((n, C), device="cuda", generator=g)) / case["T"]
        top, index = torch.topk(t, case["k"], 1)
        lse = torch.logsumexp(t, 1, keepdim=True)
        s["rest"] = None
        if case["rest"]:
            s["rest"] = torch.exp(t.scatter_(1, index, -math.inf) - lse).sum(1)
        s["logq"], s["index"] = top - lse, index.int()
        del t, top, index, lse
        s["index"][skip] = -1  # rows without a teacher
        if case["rest"]:
            s["rest"][skip] = 0.0
        s["weight"] = (0.5 + torch.rand(n, device="cuda", generator=g)) / n
        s["out"] = torch.empty(1, device="cuda")
        s["kl"] = torch.empty(n, device="cuda")
        s["dZ"] = torch.empty((n, case["ld"]), device="cuda")[:, :C]
    if case["skip"]:  # padding: whatever logits, nothing that may spread
        Z[skip] = math.nan
    if own:
        from paper_2010_03166_amd import gnnprop as G
        need = G.gnn_sample_workspace_bytes(n, C) if op == "sample" else \
            G.gnn_top_workspace_bytes(n, C, case["k"]) if op == "top" else \
            G.gnn_distill_workspace_bytes(n, C, case["k"])
        s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------ plain forms

def _plain_sample(s):
    """Kept sets and their sums in 64 bits: an action next to a border of the
    kept set or of the random number must fall on its own side of it."""
    c, Z = s["case"], s["Z"]
    C = c["C"]
    top = Z.amax(1, keepdim=True)
    ok = torch.isfinite(top)
    Z, top = torch.where(ok, Z, 0.0), torch.where(ok, top, 0.0)
    if c["T"] == 0.0:  # the best one, the first of equals
        at = torch.arange(C, device=Z.device, dtype=torch.int32)
        action = torch.where(Z == top, at, C).amin(1)
    else:
        d = Z.double() - top.double()
        e = torch.exp(d / c["T"])
        if c["min_p"] > 0.0:
            kept = d >= c["T"] * math.log(c["min_p"])
        else:
            kept = torch.ones_like(Z, dtype=torch.bool)
        if 0 < c["top_k"] < C or c["top_p"] < 1.0:
            order = torch.sort(Z, dim=1, descending=True, stable=True)[1]
            w = e.gather(1, order)
            first = torch.ones_like(kept)
            if 0 < c["top_k"] < C:
                w[:, c["top_k"]:] = 0.0
                first[:, c["top_k"]:] = False
            if c["top_p"] < 1.0:
                before = torch.cumsum(w, 1) - w
                first &= before < c["top_p"] * w.sum(1, keepdim=True)
            kept &= torch.zeros_like(kept).scatter_(1, order, first)
        cum = torch.cumsum(torch.where(kept, e, 0.0), 1)
        action = (cum <= s["u"].double()[:, None] * cum[:, -1:]).sum(1)
    action = action.clamp(max=C - 1)
    lp = Z.gather(1, action[:, None].long()).double() - top.double() - \
        torch.log(torch.exp((Z - top).float()).double().sum(1, keepdim=True))
    return {"action": torch.where(ok[:, 0], action, -1).int(),
            "logp": torch.where(ok, lp, 0.0)[:, 0].float()}


def _plain_top(s):
    c, Z = s["case"], s["Z"]
    k, T = c["k"], c["T"]
    top = Z.amax(1, keepdim=True)
    ok = torch.isfinite(top)
    top = torch.where(ok, top, 0.0)
    z, index = torch.sort(torch.where(ok, Z, -math.inf), dim=1, descending=True, stable=True)
    d = (z - top) / T
    e = torch.exp(d)
    total = e.double().sum(1, keepdim=True)
    logq = d[:, :k].double() - torch.log(total)
    there = z[:, :k] > -math.inf
    return {"index": torch.where(there, index[:, :k], -1).int(),
            "logq": torch.where(there, logq, -math.inf).float(),
            "rest": torch.where(ok, e[:, k:].double().sum(1, keepdim=True) / total, 0.0)[:, 0]
            .float()}


def _plain_distill(s):
    c, Z, logq = s["case"], s["Z"], s["logq"]
    T, C = c["T"], c["C"]
    there = (s["index"] >= 0) & (s["index"] < C)
    ok = there.any(1, keepdim=True)
    index = torch.where(there, s["index"], 0).long()
    q = torch.where(there, torch.exp(logq), 0.0)
    rest = s["rest"][:, None] if c["rest"] else torch.zeros_like(q[:, :1])
    norm = torch.where(ok, q.sum(1, keepdim=True) + rest, 1.0)
    q, rest = q / norm, rest / norm
    z = torch.where(ok, Z, 0.0)
    x = (z - z.amax(1, keepdim=True)) / T
    e = torch.exp(x)
    total = e.double().sum(1, keepdim=True)
    logp = x.gather(1, index).double() - torch.log(total)
    kl = torch.where(q > 0.0, q * (torch.log(q) - logp), 0.0).sum(1, keepdim=True)
    p = (e / total).float()
    share = torch.ones_like(norm)  # of p in the gradient outside the teacher's choice
    if c["rest"]:
        left = torch.where(ok, p.scatter(1, index, 0.0).double().sum(1, keepdim=True), 1.0)
        kl = kl + torch.where(rest > 0.0, rest * (torch.log(rest) - torch.log(left)), 0.0)
        share = torch.where(rest > 0.0, 1.0 - rest / left, 1.0)
    w = torch.where(ok, s["weight"][:, None], 0.0)
    kl = torch.where(ok, T * T * kl, 0.0)
    dZ = (w * T * share).float() * p
    dZ.scatter_(1, index, (w * T) * (p.gather(1, index) - q))
    return {"out": (w * kl).double().sum().float().reshape(1), "kl": kl[:, 0].float(), "dZ": dZ}


# --------------------------------------------------------------- one pass

def _run_own(s):
    from paper_2010_03166_amd import gnnprop as G
    c = s["case"]
    n, C = c["n"], c["C"]
    if c["op"] == "sample":
        G.gnn_sample_actions(n, C, s["Z"], c["ld"], s["u"], c["T"], c["top_k"], c["top_p"],
                             c["min_p"], s["action"], s["logp"], s["ws"])
        return {"action": s["action"], "logp": s["logp"]}
    if c["op"] == "top":
        G.gnn_top_logits(n, C, s["Z"], c["ld"], c["k"], c["T"], s["index"], s["logq"], s["rest"],
                         s["ws"])
        return {"index": s["index"], "logq": s["logq"], "rest": s["rest"]}
    G.gnn_distill_loss(n, C, s["Z"], c["ld"], c["k"], s["index"], s["logq"], s["rest"],
                       s["weight"], c["T"], s["out"], s["kl"], s["dZ"], c["ld"], s["ws"])
    return {"out": s["out"], "kl": s["kl"], "dZ": s["dZ"]}


def run(state):
    if own:
        return _run_own(state)
    return {"sample": _plain_sample, "top": _plain_top,
            "distill": _plain_distill}[state["case"]["op"]](state)


# -------------------------------------------------------------------- work

def work(case):
    n, C, op = case["n"], case["C"], case["op"]
    if op == "sample":  # logits and random numbers read, actions and logp written
        return {"bytes": 4 * n * C + 12 * n, "flops": 4 * n * C}
    if op == "top":
        return {"bytes": 4 * n * C + 8 * n * case["k"] + 4 * n, "flops": 4 * n * C}
    return {"bytes": 8 * n * C + 8 * n * case["k"] + 8 * n + 4 * n * case["rest"] + 4,
            "flops": 6 * n * C + 6 * n * case["k"]}


# ---------------------------------------------- the definitions, in 64 bits

def _live(Z):
    """Rows whose largest logit is a finite number."""
    return torch.nonzero(torch.isfinite(Z.amax(1)))[:, 0]


def _exact_sample(case, s):
    n, C, T = case["n"], case["C"], case["T"]
    live = _live(s["Z"])
    z = s["Z"][live].double()
    action = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    logp = torch.zeros(n, dtype=torch.float64, device="cuda")
    order = torch.argsort(z.neg(), dim=1, stable=True)
    if T == 0.0:
        a = order[:, 0]
    else:
        p = torch.softmax(z / T, 1)
        ranked = p.gather(1, order)
        most = case["top_k"] if 0 < case["top_k"] < C else C
        length = torch.full((len(live), 1), most, device="cuda")
        if case["top_p"] < 1.0:
            cdf = torch.cumsum(ranked[:, :most], 1)
            length = torch.searchsorted(cdf, cdf[:, -1:] * case["top_p"]) + 1
        if case["min_p"] > 0.0:
            near = z >= z.amax(1, keepdim=True) + T * math.log(case["min_p"])
            length = torch.minimum(length, near.sum(1, keepdim=True))
        ranked.masked_fill_(torch.arange(C, device="cuda") >= length, 0.0)
        cdf = torch.cumsum(torch.empty_like(p).scatter_(1, order, ranked), 1)
        a = torch.searchsorted(cdf, cdf[:, -1:] * s["u"][live].double()[:, None], right=True)[:, 0]
    action[live] = a.int()
    logp[live] = torch.log_softmax(z, 1).gather(1, a[:, None])[:, 0]
    return {"action": action, "logp": logp}


def _exact_top(case, s):
    n, k = case["n"], case["k"]
    live = _live(s["Z"])
    lq = torch.log_softmax(s["Z"][live].double() / case["T"], 1)
    at = torch.argsort(s["Z"][live].neg(), dim=1, stable=True)[:, :k]
    best = lq.gather(1, at)
    index = torch.full((n, k), -1, dtype=torch.int32, device="cuda")
    logq = torch.full((n, k), -math.inf, dtype=torch.float64, device="cuda")
    rest = torch.zeros(n, dtype=torch.float64, device="cuda")
    index[live] = at.int().masked_fill_(best == -math.inf, -1)
    logq[live] = best
    rest[live] = lq.scatter_(1, at, -math.inf).exp_().sum(1)
    return {"index": index, "logq": logq, "rest": rest}


def _exact_distill(case, s):
    n, C, T = case["n"], case["C"], case["T"]
    live = torch.nonzero(s["index"][:, 0] >= 0)[:, 0]
    at = s["index"][live].long()
    lq = s["logq"][live].double()
    if case["rest"]:
        lq = torch.cat([lq, torch.log(s["rest"][live].double())[:, None]], 1)
    lq = torch.log_softmax(lq, 1)
    q = lq.exp()
    L = torch.log_softmax(s["Z"][live].double() / T, 1)
    k = case["k"]
    lp = L.gather(1, at)
    d = L.exp()
    if case["rest"]:
        others = torch.logsumexp(L.scatter(1, at, -math.inf), 1, keepdim=True)
        lp = torch.cat([lp, others], 1)
        d -= torch.exp(L + torch.where(q[:, k:] > 0.0, lq[:, k:] - others, -math.inf))
    d.scatter_(1, at, lp[:, :k].exp() - q[:, :k])
    kl = torch.zeros(n, dtype=torch.float64, device="cuda")
    kl[live] = T * T * (q * lq - q * lp).nansum(1)  # (0 times a logarithm of 0)
    w = s["weight"].double()
    dZ = torch.zeros((n, C), dtype=torch.float64, device="cuda")
    dZ[live] = d.mul_(T * w[live][:, None])
    return {"out": (w * kl).sum().reshape(1), "kl": kl, "dZ": dZ}


def exact(case, seed):
    return {"sample": _exact_sample, "top": _exact_top,
            "distill": _exact_distill}[case["op"]](case, prepare(case, seed))
