"""The operators of a training step beyond cross-entropy and plain Adam:
log-probabilities of chosen actions, the clipped policy loss with a KL term
and its gradient, the norm of all gradients and the AdamW update of many
tensors with states in 32 or in 8 bits.

`listed()` and `draw(rng)` give their workloads, `run(state)` one call of one
of them: the plain form in elementary torch operations, or, where `own` is
true, the library's kernels.
"""
import math

import numpy as np
import torch

own = False  # False: the plain forms; True: the library's entry points

LR, B1, B2, EPS, DECAY, STEP, MAX_NORM = 1e-3, 0.9, 0.999, 1e-8, 0.01, 7, 1.0
CLIP_LO, CLIP_HI, BETA = 0.2, 0.28, 0.04
BLOCK = 256                  # elements that share a scale of 8-bit states
M_TOP, V_TOP = 448.0, 57344.0  # largest e4m3 and e5m2 values
TINY = 2.0 ** -126
GOLDEN = 0x9E3779B97F4A7C15
MASK64 = (1 << 64) - 1


def listed():
    return [
        # one small graph's nodes choosing among 7 actions: latency counts
        dict(name="policy_small", op="policy", n=256, C=7, ld=7, mask=0.0, skip=0.0),
        # a large batch of nodes over 121 classes at an odd row stride, a tenth
        # of the rows padding (no action, NaN logits)
        dict(name="policy_ragged", op="policy", n=50001, C=121, ld=121, mask=0.0, skip=0.1),
        # 16,384 rows of 2,048 actions, a power of two, aligned rows
        dict(name="policy_wide", op="policy", n=16384, C=2048, ld=2048, mask=0.0, skip=0.0),
        # 64 graphs, each choosing one of a full graph's 131,071 nodes, a
        # third of them not allowed (-inf)
        dict(name="policy_nodes", op="policy", n=64, C=131071, ld=131072, mask=0.33, skip=0.0),
        # acting: the log-probabilities of an 8,000-node subgraph, 41 classes
        dict(name="logp_8k", op="logp", n=8000, C=41, ld=44, mask=0.0, skip=0.0),
        # a reference network's log-probabilities over many actions
        dict(name="logp_long", op="logp", n=2000, C=20011, ld=20011, mask=0.0, skip=0.0),
        # gradients of the two-layer 602 -> 2 x 512 network with biases
        dict(name="norm_sage", op="norm", f=602, h=512, layers=2, C=41, bias=True),
        # eight layers of 2 x 2,048: 120 million gradients
        dict(name="norm_deep", op="norm", f=602, h=2048, layers=8, C=121, bias=True),
        # their updates, states in 32 bits
        dict(name="adamw_sage", op="adamw", bits=32, f=602, h=512, layers=2, C=41, bias=True),
        dict(name="adamw_deep", op="adamw", bits=32, f=602, h=2048, layers=8, C=121, bias=True),
        # and in 8 bits; odd widths, so that blocks end inside a wavefront
        dict(name="adamw8_odd", op="adamw", bits=8, f=199, h=301, layers=3, C=41, bias=True),
        dict(name="adamw8_deep", op="adamw", bits=8, f=602, h=2048, layers=8, C=121, bias=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["policy", "policy", "logp", "norm", "adamw", "adamw"])
    if op in ("policy", "logp"):
        C = _log_int(rng, 2, 131072)
        n = _log_int(rng, 1, min(200000, 33000000 // C))
        ld = rng.choice([C, (C + 3) // 4 * 4, C + rng.randint(1, 9)])
        return dict(op=op, n=n, C=C, ld=ld, mask=round(rng.choice([0.0, 0.0, 0.5 * rng.random()]), 2),
                    skip=round(rng.choice([0.0, 0.0, 0.9 * rng.random()]), 2))
    c = dict(op=op, f=_log_int(rng, 16, 700), h=_log_int(rng, 16, 2048), layers=rng.randint(1, 5),
             C=rng.randint(2, 121), bias=rng.random() < 0.5)
    if op == "adamw":
        c["bits"] = rng.choice([32, 8])
    return c


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _shapes(case):
    """Weights of a GraphSAGE stack with its classifier: W_MLP, then W_self,
    W_neigh (and the biases) of each layer."""
    f, h = case["f"], case["h"]
    out = [(2 * h, case["C"])]
    for _ in range(case["layers"]):
        out += [(f, h), (f, h)] + ([(h,), (h,)] if case["bias"] else [])
        f = 2 * h
    return out


def _offsets(shapes):
    """Where each tensor starts in one flat buffer (whole blocks of 256)."""
    offs, total = [], 0
    for s in shapes:
        offs.append(total)
        total += -(-math.prod(s) // BLOCK) * BLOCK
    return offs, total


def _prepare_policy(case, seed):
    g = _gen(seed)
    n, C = case["n"], case["C"]
    Z = torch.randn((n, case["ld"]), device="cuda", generator=g)[:, :C].mul_(2.0)
    if case["mask"]:  # actions that are not allowed
        Z.masked_fill_(torch.rand((n, C), device="cuda", generator=g) < case["mask"], -math.inf)
        Z[:, 0] = 0.0  # one always is
    u = torch.rand((n, C), device="cuda", generator=g).clamp_(1e-7, 1 - 1e-7)
    action = (Z - torch.log(-torch.log(u))).argmax(1)  # drawn from the policy itself
    del u
    lp = torch.log_softmax(Z.double(), 1).gather(1, action[:, None])[:, 0]
    s = dict(case=case, Z=Z,
             adv=torch.randn(n, device="cuda", generator=g),
             old=(lp + 0.1 * torch.randn(n, device="cuda", generator=g)).float(),
             ref=(lp + 0.3 * torch.randn(n, device="cuda", generator=g)).float(),
             weight=(0.5 + torch.rand(n, device="cuda", generator=g)) / n)
    action = action.int()
    if case["skip"]:  # padding: no action, whatever logits, nothing that may spread
        skip = torch.rand(n, device="cuda", generator=g) < case["skip"]
        action[skip] = -1
        Z[skip] = math.nan
    s["action"] = action
    s["logp"] = torch.empty(n, device="cuda")
    s["out"] = torch.empty(3, device="cuda")
    s["dZ"] = torch.empty((n, case["ld"]), device="cuda")[:, :C] if case["op"] == "policy" else None
    if own:
        from paper_2010_03166_amd import gnnprop as G
        s["ws"] = torch.empty(max(G.gnn_policy_workspace_bytes(n, C), 256), dtype=torch.uint8,
                              device="cuda")
    return s


def _prepare_params(case, seed):
    g = _gen(seed)
    shapes = _shapes(case)
    offs, total = _offsets(shapes)
    sizes = [math.prod(x) for x in shapes]
    live = torch.zeros(total, device="cuda")
    decay = torch.zeros(total // BLOCK, 1, device="cuda")
    for x, o, c in zip(shapes, offs, sizes):
        live[o: o + c] = 1.0
        decay[o // BLOCK: -(-(o + c) // BLOCK)] = DECAY if len(x) == 2 else 0.0
    # a gradient's size differs from one tensor and one weight to the next
    G_ = torch.randn(total, device="cuda", generator=g).mul_(live)
    G_.view(-1, BLOCK).mul_(1e-3 * torch.exp(torch.randn(total // BLOCK, 1, device="cuda",
                                                         generator=g)))
    s = dict(case=case, shapes=shapes, offs=offs, sizes=sizes, G=G_, decay=decay,
             norm=torch.empty(1, device="cuda"))
    if case["op"] == "adamw":
        s["W"] = torch.randn(total, device="cuda", generator=g).mul_(live).mul_(0.05)
        m = torch.randn(total, device="cuda", generator=g).mul_(G_.abs()).mul_(0.3)
        v = torch.rand(total, device="cuda", generator=g).mul_(1.5).add_(0.5).mul_(G_ * G_)
        s["norm"].copy_(G_.double().square().sum().sqrt())
        s["seed"] = 12345 + seed
        if case["bits"] == 32:
            s["m"], s["v"] = m, v
        else:
            r = torch.full((total // BLOCK, BLOCK), 1 << 15, device="cuda")
            s["m"], s["m_scale"] = _store(m.double().view(-1, BLOCK), 3, -6, M_TOP, r)
            s["v"], s["v_scale"] = _store(v.double().view(-1, BLOCK), 2, -14, V_TOP, r)
        del m, v
    if own:
        from paper_2010_03166_amd import gnnprop as G
        bits = case.get("bits", 32)
        tensors = []
        for x, o, c in zip(shapes, offs, sizes):
            t = [s.get("W", G_)[o: o + c], G_[o: o + c]] if case["op"] == "adamw" else \
                [None, G_[o: o + c]]
            if case["op"] == "adamw":
                b0, b1 = o // BLOCK, -(-(o + c) // BLOCK)
                t += [s["m"].view(-1)[o: o + c], s["v"].view(-1)[o: o + c]]
                t += [s["m_scale"][b0:b1], s["v_scale"][b0:b1]] if bits == 8 else [None, None]
                t.append(DECAY if len(x) == 2 else 0.0)
            tensors.append(tuple(t))
        ps = G.make_params(tensors, bits)
        s["plan"] = torch.empty(G.gnn_params_plan_bytes(ps), dtype=torch.uint8, device="cuda")
        ps.plan = s["plan"].data_ptr()
        G.gnn_params_build_plan(ps, s["plan"])
        s["params"] = ps
        s["ws"] = torch.empty(max(G.gnn_grad_norm_workspace_bytes(ps), 256), dtype=torch.uint8,
                              device="cuda")
    return s


def prepare(case, seed):
    return (_prepare_policy if case["op"] in ("policy", "logp") else _prepare_params)(case, seed)


# ------------------------------------------------------------ plain forms

def _row_stats(s):
    """(rows that count, exp(z - max), its row sums, log-probabilities), the
    sums and logarithms in 64 bits: a ratio next to the clip's border must
    fall on its own side of it."""
    Z, a = s["Z"], s["action"].long()
    ok = (a >= 0) & (a < Z.shape[1])
    z = torch.where(ok[:, None], Z, 0.0)
    a = torch.where(ok, a, 0)
    top = z.amax(1)
    e = torch.exp(z.double() - top.double()[:, None])
    tot = e.sum(1)
    lp = z.gather(1, a[:, None])[:, 0].double() - top.double() - torch.log(tot)
    return ok, a, e, tot, torch.where(ok, lp, 0.0)


def _plain_logp(s):
    return _row_stats(s)[4].float()


def _plain_policy(s):
    ok, a, e, tot, lp = _row_stats(s)
    A = s["adv"].double()
    w = torch.where(ok, s["weight"].double(), 0.0)
    rho = torch.exp(lp - s["old"].double())
    cl = torch.clamp(rho, 1.0 - CLIP_LO, 1.0 + CLIP_HI)
    inside = rho * A <= cl * A
    d = s["ref"].double() - lp
    kl = torch.exp(d) - d - 1.0
    each = -torch.where(inside, rho * A, cl * A) + BETA * kl
    out = torch.stack([(w * each).sum(), (w * kl).sum(), (w * (~inside)).sum()])
    c = (w * (torch.where(inside, -A * rho, 0.0) + BETA * (1.0 - torch.exp(d)))).float()
    dZ = (e / tot[:, None]).float() * -c[:, None]
    dZ.scatter_add_(1, a[:, None], c[:, None])
    return {"out": out.float(), "logp": lp.float(), "dZ": dZ}


def _plain_norm(s):
    g = s["G"].double()
    return torch.sqrt((g * g).sum()).float().reshape(1)


def _mix64(z):
    """SplitMix64's output function on int64 tensors (two's complement)."""
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * (0xBF58476D1CE4E5B9 - (1 << 64))
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * (0x94D049BB133111EB - (1 << 64))
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _splitmix_int(state, k):
    z = (state + (k + 1) * GOLDEN) & MASK64
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & MASK64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & MASK64
    return z ^ (z >> 31)


def _signed(x):
    return x - (1 << 64) if x >> 63 else x


def _random32(seed, t, count, device):
    """32 random bits for each of `count` elements: output i // 2 of the
    generator started at output t of the one started at `seed`, its lower
    half for even elements."""
    base = _splitmix_int(seed & MASK64, t)
    k = torch.arange(1, count // 2 + 1, device=device)
    h = _mix64(k * _signed(GOLDEN) + _signed(base))
    return torch.stack([h & 0xFFFFFFFF, (h >> 32) & 0xFFFFFFFF], 1).view(-1)


def _load(code, scale, bits, emin):
    """Values that 8-bit codes stand for: `bits` bits of mantissa."""
    mag = (code & 127).int()
    ex = (mag >> bits).clamp(min=1)
    man = (mag & ((1 << bits) - 1)) + torch.where((mag >> bits) > 0, 1 << bits, 0)
    x = torch.ldexp(man.double(), ex - 1 + emin - bits)
    return torch.where(code > 127, -x, x) * scale.double()[:, None]


def _store(x, bits, emin, top, r):
    """Codes and scales of blocks (rows): stochastic rounding by r / 2^16."""
    scale = (x.abs().amax(1) / top).float().clamp(min=TINY)
    y = x.abs() / scale.double()[:, None]
    ex = torch.where(y > 0, torch.frexp(y)[1] - 1, emin).clamp(min=emin)
    k = torch.floor(torch.ldexp(y, bits - ex) + (r.double() + 0.5) / 65536.0)
    most = 126 if bits == 3 else 123
    code = ((ex - emin) * (1 << bits) + k.int()).clamp(max=most)
    if bits == 2:  # a second moment that is not zero is not stored as zero
        code = torch.where(y > 0, code.clamp(min=1), code)
    return torch.where(x < 0, code + 128, code).to(torch.uint8), scale


def _plain_adamw(s):
    norm = s["norm"]
    k = torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0)
    c1, c2 = 1.0 - B1 ** STEP, 1.0 - B2 ** STEP
    W, g = s["W"].view(-1, BLOCK), s["G"].view(-1, BLOCK)
    if s["case"]["bits"] == 32:
        g = g * k
        m, v = s["m"].view(-1, BLOCK), s["v"].view(-1, BLOCK)
        m.copy_(B1 * m + (1.0 - B1) * g)
        v.copy_(B2 * v + (1.0 - B2) * g * g)
    else:
        g = g.double() * torch.where(norm > MAX_NORM, MAX_NORM / norm.double(), 1.0)
        m = B1 * _load(s["m"], s["m_scale"], 3, -6) + (1.0 - B1) * g
        v = B2 * _load(s["v"], s["v_scale"], 2, -14) + (1.0 - B2) * g * g
        r = _random32(s["seed"], STEP, g.numel(), g.device).view(-1, BLOCK)
        for name, x, bits, emin, top, rr in (("m", m, 3, -6, M_TOP, r & 0xFFFF),
                                             ("v", v, 2, -14, V_TOP, r >> 16)):
            code, scale = _store(x, bits, emin, top, rr)
            s[name].copy_(code)
            s[name + "_scale"].copy_(scale)
        m, v = m.float(), v.float()
    W.copy_((1.0 - LR * s["decay"]) * W - LR * (m / c1) / (torch.sqrt(v / c2) + EPS))
    return _updated(s)


def _updated(s):
    if s["case"]["bits"] == 32:
        return {"W": s["W"], "m": s["m"], "v": s["v"]}
    return {"W": s["W"], "m": s["m"].view(torch.float8_e4m3fn), "m_scale": s["m_scale"],
            "v": s["v"].view(torch.float8_e5m2), "v_scale": s["v_scale"]}


# --------------------------------------------------------------- one pass

def _run_own(s):
    from paper_2010_03166_amd import gnnprop as G
    case = s["case"]
    if case["op"] == "logp":
        G.gnn_action_logp(case["n"], case["C"], s["Z"], case["ld"], s["action"], s["logp"], s["ws"])
        return s["logp"]
    if case["op"] == "policy":
        G.gnn_policy_loss(case["n"], case["C"], s["Z"], case["ld"], s["action"], s["adv"], s["old"],
                          s["ref"], s["weight"], CLIP_LO, CLIP_HI, BETA, s["out"], s["logp"],
                          s["dZ"], case["ld"], s["ws"])
        return {"out": s["out"], "logp": s["logp"], "dZ": s["dZ"]}
    if case["op"] == "norm":
        G.gnn_grad_norm(s["params"], s["norm"], s["ws"])
        return s["norm"]
    G.gnn_adamw_step(s["params"], LR, B1, B2, EPS, STEP, s["norm"], MAX_NORM, s["seed"])
    return _updated(s)


def run(state):
    if own:
        return _run_own(state)
    return {"logp": _plain_logp, "policy": _plain_policy, "norm": _plain_norm,
            "adamw": _plain_adamw}[state["case"]["op"]](state)


# -------------------------------------------------------------------- work

def _count(case):
    return sum(math.prod(x) for x in _shapes(case))


def work(case):
    op = case["op"]
    if op in ("policy", "logp"):
        n, C = case["n"], case["C"]
        if op == "logp":
            return {"bytes": 4 * n * C + 8 * n, "flops": 4 * n * C}
        return {"bytes": 8 * n * C + 24 * n + 12, "flops": 7 * n * C}
    P = _count(case)
    if op == "norm":
        return {"bytes": 4 * P + 4, "flops": 2 * P}
    # W, m, v read and written, G read; a pair of scales for 256 weights
    return {"bytes": 28 * P if case["bits"] == 32 else 16 * P + 16 * (P // BLOCK), "flops": 16 * P}


# ---------------------------------------------- the definitions, in 64 bits

def _exact_policy(case, seed):
    s = _prepare_policy(case, seed)
    a = s["action"].long()
    live = torch.nonzero((a >= 0) & (a < case["C"]))[:, 0]
    a = a[live]
    logp = torch.zeros(case["n"], dtype=torch.float64, device="cuda")
    L = torch.log_softmax(s["Z"][live].double(), 1)
    lp = L.gather(1, a[:, None])[:, 0]
    logp[live] = lp
    if case["op"] == "logp":
        return logp
    A, w = s["adv"][live].double(), s["weight"][live].double()
    ratio, gap = (lp - s["old"][live].double()).exp(), s["ref"][live].double() - lp
    low = torch.minimum(torch.maximum(ratio, torch.full_like(ratio, 1 - CLIP_LO)),
                        torch.full_like(ratio, 1 + CLIP_HI))
    cut = (ratio * A) > (low * A)
    kl = torch.expm1(gap) - gap
    loss = -torch.minimum(ratio * A, low * A) + BETA * kl
    slope = w * (-(ratio * A).masked_fill(cut, 0.0) - BETA * torch.expm1(gap))
    d = L.exp_().mul_(-slope[:, None])
    d[torch.arange(len(a), device="cuda"), a] += slope
    dZ = torch.zeros((case["n"], case["C"]), dtype=torch.float64, device="cuda")
    dZ[live] = d
    return {"out": torch.stack([(w * loss).sum(), (w * kl).sum(), w[cut].sum()]), "logp": logp,
            "dZ": dZ}


def _grid(bits, emin, count, device):
    """The values of codes 0, 1, ... of one sign, ascending."""
    v = [(c % (1 << bits)) * 2.0 ** (emin - bits) if c < (1 << bits) else
         (1 + (c % (1 << bits)) / (1 << bits)) * 2.0 ** ((c >> bits) - 1 + emin)
         for c in range(count)]
    return torch.tensor(v, dtype=torch.float64, device=device)


def _exact_draws(seed, count):
    """The 32 random bits of every element, from the generator's definition."""
    def mixed(z):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))

    step, first = np.uint64(GOLDEN), np.array([seed], np.uint64)
    start = mixed(first + np.array([((STEP + 1) * GOLDEN) & MASK64], np.uint64))
    words = mixed(start + np.arange(1, count // 2 + 1, dtype=np.uint64) * step)
    return torch.from_numpy(words.view(np.uint32).astype(np.int64)).cuda()  # low half first


def _exact_rounded(x, grid, r):
    """(values in units of the scale, scales) after stochastic rounding."""
    top = grid[-1]
    scale = torch.maximum((x.abs().amax(1) / top).float(), torch.tensor(TINY, device=x.device))
    y = (x.abs() / scale.double()[:, None]).clamp_(max=float(top))
    at = torch.searchsorted(grid, y.contiguous(), right=True).sub_(1).clamp_(max=len(grid) - 2)
    lo, hi = grid[at], grid[at + 1]
    up = (y - lo) / (hi - lo) + (r.double() + 0.5) / 65536.0 >= 1.0
    q = torch.where(up, hi, lo)
    if len(grid) == 124:
        q = torch.where((y > 0) & (q == 0), grid[1], q)
    return torch.copysign(q, x), scale


def _exact_params(case, seed):
    s = _prepare_params(case, seed)
    if case["op"] == "norm":
        return torch.linalg.vector_norm(s["G"].double()).reshape(1)
    g = s["G"].double()
    norm = float(s["norm"])
    if norm > MAX_NORM:
        g = g * (MAX_NORM / norm)
    if case["bits"] == 32:
        m0, v0 = s["m"].double(), s["v"].double()
    else:
        gm = _grid(3, -6, 127, "cuda")
        gv = _grid(2, -14, 124, "cuda")
        c = s["m"].long()
        m0 = (gm[c & 127] * (1 - 2 * (c >> 7)) * s["m_scale"].double()[:, None]).view(-1)
        v0 = (gv[s["v"].long()] * s["v_scale"].double()[:, None]).view(-1)
        del c
    m = torch.lerp(g, m0, B1)
    v = torch.lerp(g.square(), v0, B2)
    decay = s["decay"].double().expand(-1, BLOCK).reshape(-1)
    W = s["W"].double()
    W = W - LR * decay * W - LR * (m / (1 - B1 ** STEP)) / ((v / (1 - B2 ** STEP)).sqrt() + EPS)
    if case["bits"] == 32:
        return {"W": W, "m": m, "v": v}
    r = _exact_draws(s["seed"], m.numel()).view(-1, BLOCK)
    qm, sm = _exact_rounded(m.view(-1, BLOCK), gm, r & 0xFFFF)
    qv, sv = _exact_rounded(v.view(-1, BLOCK), gv, r >> 16)
    return {"W": W, "m": qm, "m_scale": sm.double(), "v": qv, "v_scale": sv.double()}


def exact(case, seed):
    return (_exact_policy if case["op"] in ("policy", "logp") else _exact_params)(case, seed)
