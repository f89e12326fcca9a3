"""The oracle of the policy loss and AdamW pinned to closed forms, finite
differences and brute force, and the host-side refusals of their entry
points.  No GPU needed."""
import ctypes

import numpy as np
import pytest

from oracle import frontier as F
from oracle import oracle as O
from oracle import policy as P
from paper_2010_03166_amd import gnnprop as G
from paper_2010_03166_amd import runtime


# ------------------------------------------------------------- policy loss

def _case(n, C, seed):
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((n, C)) * 2
    a = rng.integers(0, C, n)
    lp, _ = P.action_logp(z, a)
    return (z, a, rng.standard_normal(n), lp + 0.3 * rng.standard_normal(n),
            lp + 0.5 * rng.standard_normal(n), rng.random(n))


def test_logp_closed_forms():
    lp, live = P.action_logp(np.zeros((2, 8)), np.array([3, -1]))
    assert np.isclose(lp[0], -np.log(8)) and lp[1] == 0 and list(live) == [True, False]
    z = np.array([[0.0, -np.inf, 0.0], [-np.inf] * 3])
    lp, live = P.action_logp(z, np.array([2, 0]))
    assert np.isclose(lp[0], -np.log(2)) and lp[1] == -np.inf and list(live) == [True, False]


@pytest.mark.parametrize("beta", [0.0, 0.3])
def test_policy_gradient_by_differences(beta):
    z, a, A, old, ref, w = _case(40, 6, 1)
    f = lambda y: P.policy_loss(y, a, A, old, ref, w, 0.2, 0.3, beta)["out"][0]
    r = P.policy_loss(z, a, A, old, ref, w, 0.2, 0.3, beta)
    assert 0 < r["cut"].sum() < 40  # both sides of the clip
    h = 1e-5
    for i in range(40):
        for j in range(6):
            y = z.copy()
            y[i, j] += h
            up = f(y)
            y[i, j] -= 2 * h
            # central differences: h^2 of the third derivative, cancellation 1e-16 / h
            assert abs((up - f(y)) / (2 * h) - r["dZ"][i, j]) < 1e-8


def test_policy_closed_forms():
    z, a, A, old, ref, w = _case(30, 5, 2)
    r = P.policy_loss(z, a, A, weight=w)  # on-policy: -sum w A, slope -w A
    assert np.isclose(r["out"][0], -(w * A).sum()) and r["out"][2] == 0
    assert np.allclose(r["slope"], -w * A)
    r = P.policy_loss(z, a, A, old, r["logp"], w, beta=0.5)  # reference = policy: no KL
    assert np.allclose(r["kl"], 0)
    # expected kl under the policy is KL(policy || reference)
    p, q = np.array([0.2, 0.5, 0.3]), np.array([0.4, 0.1, 0.5])
    k = [P.policy_loss(np.log(p)[None], [j], [0.0], None, [np.log(q[j])], [1.0])["kl"][0]
         for j in range(3)]
    assert np.isclose((p * k).sum(), (p * np.log(p / q)).sum())


# ------------------------------------------------------------------- AdamW

def test_adamw_without_decay_is_adam():
    rng = np.random.default_rng(3)
    w, g, m = (rng.standard_normal(50) for _ in range(3))
    v = rng.random(50)
    for got, want in zip(P.adamw(w, g, m, v, 0.01, 0.9, 0.99, 1e-8, 4, 0.0),
                         O.adam(w, g, m, v, 0.01, 0.9, 0.99, 1e-8, 4)):
        assert np.allclose(got, want, rtol=1e-12)
    w1 = P.adamw(w, 0 * g, 0 * m, 0 * v, 0.1, 0.9, 0.99, 1e-8, 1, 0.5)[0]
    assert np.allclose(w1, 0.95 * w)  # decay alone


def test_eight_bit_grids():
    import torch
    for grid, kind in ((P.E4M3, torch.float8_e4m3fn), (P.E5M2, torch.float8_e5m2)):
        codes = torch.arange(len(grid), dtype=torch.uint8).view(kind)
        assert np.array_equal(codes.float().numpy(), grid)
    assert P.E4M3[-1] == 448 and P.E5M2[-1] == 57344


def test_rounding_is_unbiased_and_to_neighbours():
    rng = np.random.default_rng(4)
    x = rng.standard_normal(256) * np.exp(rng.standard_normal(256) * 3)
    s = P.scales(x, P.E4M3)
    assert len(s) == 1 and s[0] == np.abs(x).max() / 448
    total = np.zeros(256)
    r = (np.arange(512) * 128 + 64)  # evenly spread draws
    for k in r:
        c, _ = P.encode(x, s, P.E4M3, np.full(256, k), False)
        d = P.decode(c, s, P.E4M3)
        y, at = np.abs(x) / s[0], c & 127
        assert np.all(P.E4M3[np.maximum(at - 1, 0)] <= y * (1 + 1e-12))
        assert np.all(y * (1 - 1e-12) <= P.E4M3[np.minimum(at + 1, 126)])
        total += d
    # 512 evenly spread draws find every fraction to 1 / 512 of a step
    top = np.searchsorted(P.E4M3, np.abs(x) / s[0], side="right").clip(1, 126)
    step = (P.E4M3[top] - P.E4M3[top - 1]) * s[0]
    assert np.all(np.abs(total / 512 - x) <= step / 512 * (1 + 1e-9))
    c, _ = P.encode(np.full(256, 1e-9), [1.0], P.E5M2, np.zeros(256), True)
    assert np.all(c == 1)  # a positive second moment is never stored as 0


def test_random_bits_are_the_generator():
    base = F.splitmix_output(77, 5)
    b = P.random_bits(77, 5, 3, 9)
    for e in range(9):
        word = F.splitmix_output(base, (3 * 256 + e) // 2)
        assert b[e] == (word >> (32 * (e & 1))) & 0xFFFFFFFF


# --------------------------------------------------------------- refusals
# Host addresses stand in for device pointers: these calls must fail before
# dereferencing or launching anything.

VP = ctypes.c_void_p


def _logp(n=4, C=3, Z=0x1000, ld=3, action=0x2000, logp=0x3000, ws=0x4000, bytes_=1 << 20):
    return G.lib().gnn_action_logp(n, C, VP(Z), ld, VP(action), VP(logp), VP(ws), bytes_, None)


def _loss(n=4, C=3, Z=0x1000, ld=3, action=0x2000, adv=0x2100, old=0x2200, ref=0x2300, w=0x2400,
          lo=0.2, hi=0.2, beta=0.0, out=0x3000, logp=0x3100, dZ=0x3200, ld_dz=3, ws=0x4000,
          bytes_=1 << 20):
    return G.lib().gnn_policy_loss(n, C, VP(Z), ld, VP(action), VP(adv), VP(old), VP(ref), VP(w),
                                   lo, hi, beta, VP(out), VP(logp), VP(dZ), ld_dz, VP(ws),
                                   bytes_, None)


def test_policy_refusals():
    for f in (_logp, _loss):
        assert f(n=-1) == -2 and f(C=0) == -2 and f(ld=2) == -2
        assert f(C=2 ** 24 + 1, ld=2 ** 24 + 1) == -2
        assert f(Z=None) == -1 and f(action=None) == -1
        assert f(ws=0x4004) == -4
        assert f(logp=0x1004) == -7 and f(logp=0x2000) == -7
    assert _loss(bytes_=8) == -5 and _loss(ws=None) == -5
    # log-probabilities need a workspace for rows that are cut into chunks
    long = dict(n=1, C=40000, ld=40000, Z=0x100000, action=0x2000)
    assert _logp(bytes_=8, **long) == -5 and _logp(ws=None, **long) == -5
    assert _logp(logp=None) == -1
    assert _logp(n=0, Z=None) == 0
    assert _loss(adv=None) == -1 and _loss(out=None) == -1
    assert _loss(beta=0.1, ref=None) == -1
    assert _loss(ld_dz=2) == -2
    nan = float("nan")
    for kw in (dict(lo=-0.1), dict(lo=1.1), dict(lo=nan), dict(hi=-0.1), dict(hi=nan),
               dict(beta=-1.0), dict(beta=nan), dict(beta=float("inf"))):
        assert _loss(**kw) == -2, kw
    for kw in (dict(out=0x1000), dict(out=0x2104), dict(dZ=0x1000), dict(dZ=0x2400),
               dict(logp=0x3008), dict(dZ=0x3100), dict(ws=0x2200)):
        assert _loss(**kw) == -7, kw
    assert G.gnn_policy_workspace_bytes(-1, 3) == 0 == G.gnn_policy_workspace_bytes(3, 0)
    assert G.gnn_policy_workspace_bytes(3, 2 ** 24 + 1) == 0
    assert G.gnn_policy_workspace_bytes(2 ** 31 - 1, 2 ** 24) > 2 ** 31 * 4096


def _set(bits=32, n=1, count=1000, **kw):
    """A gnn_params of n tensors at made-up addresses 1 MiB apart."""
    p = (G.gnn_param * max(n, 1))()
    for k in range(n):
        b = 0x10000000 + k * 0x1000000
        p[k] = G.gnn_param(count, b, b + 0x100000, b + 0x200000, b + 0x300000, b + 0x400000,
                           b + 0x500000, 0.01)
    for key, val in kw.items():
        setattr(p[n - 1], key, val)
    s = G.gnn_params(n, bits, ctypes.cast(p, ctypes.POINTER(G.gnn_param)), 0x8000000)
    s._keep = p
    return s


def _build(s, plan=0x8000000, bytes_=None):
    need = G.gnn_params_plan_bytes(s) if bytes_ is None else bytes_
    return G.lib().gnn_params_build_plan(ctypes.byref(s) if s else None, VP(plan), need, None)


@pytest.mark.parametrize("bits", [32, 8])
def test_plan_refusals(bits):
    L = G.lib()
    assert L.gnn_params_build_plan(None, VP(0x10), 1 << 20, None) == -1
    assert _build(_set(bits, n=-1), bytes_=1 << 20) == -2
    assert _build(_set(16), bytes_=1 << 20) == -4
    assert _build(_set(bits, count=-1), bytes_=1 << 20) == -2
    assert _build(_set(bits, count=(1 << 40) + 1), bytes_=1 << 20) == -2
    for bad in (float("nan"), float("inf")):
        assert _build(_set(bits, weight_decay=bad), bytes_=1 << 20) == -2
    assert _build(_set(bits, G=None), bytes_=1 << 20) == -1
    s = _set(bits)
    assert _build(s, plan=None) == -1 and _build(s, plan=0x8000008) == -4
    assert _build(s, bytes_=G.gnn_params_plan_bytes(s) - 1) == -5
    for kw in (dict(W=0x10000002), dict(G=0x10100001), dict(m_scale=0x10400002)):
        assert _build(_set(bits, **kw)) == -4, kw
    if bits == 32:
        assert _build(_set(bits, m=0x10200002)) == -4
    # whatever is written overlaps nothing, in the same tensor or another
    for kw in (dict(W=0x10100000 - 4), dict(m=0x10000000 + 3996), dict(v=0x10200000 + 996),
               dict(W=0x8000000)):
        assert _build(_set(bits, **kw)) == -7, kw
    assert _build(_set(bits, n=3, W=0x11100000)) == -7   # the second tensor's gradient
    assert _build(_set(bits, n=3, m=0x10300000)) == -7   # the first one's v
    if bits == 8:
        assert _build(_set(bits, v_scale=0x10400000)) == -7
    neg = _set(bits, n=-1)
    assert G.gnn_params_plan_bytes(neg) == 0 == G.gnn_grad_norm_workspace_bytes(neg)


@pytest.mark.parametrize("bits", [32, 8])
def test_norm_and_step_refusals(bits):
    L = G.lib()

    def norm(s, out=0x7000000, ws=0x7100000, b=1 << 20):
        return L.gnn_grad_norm(ctypes.byref(s) if s else None, VP(out), VP(ws), b, None)

    def step(s, lr=0.1, b1=0.9, b2=0.99, eps=1e-8, t=1, nrm=0x7000000, top=1.0):
        return L.gnn_adamw_step(ctypes.byref(s) if s else None, lr, b1, b2, eps, t, VP(nrm), top,
                                0, None)

    s = _set(bits)
    assert norm(None) == -1 and norm(s, out=None) == -1
    assert norm(s, ws=0x7100004) == -4 and norm(s, ws=None) == -5 and norm(s, b=4) == -5
    assert norm(s, out=0x10100000) == -7 and norm(s, ws=0x10100000 - 16) == -7
    assert norm(s, out=0x7100000) == -7 and norm(s, out=0x8000000) == -7
    assert step(None) == -1
    nan, inf = float("nan"), float("inf")
    for kw in (dict(t=0), dict(b1=1.0), dict(b1=-0.1), dict(b1=nan), dict(b2=1.0), dict(b2=nan),
               dict(eps=-1.0), dict(eps=nan), dict(eps=inf), dict(lr=nan), dict(lr=inf),
               dict(top=0.0), dict(top=nan)):
        assert step(s, **kw) == -2, kw
    for kw in (dict(W=None), dict(m=None), dict(v=None)):
        assert step(_set(bits, **kw)) == -1, kw
    if bits == 8:
        assert step(_set(bits, m_scale=None)) == -1 and step(_set(bits, v_scale=None)) == -1
    assert step(s, nrm=0x10000000) == -7 and step(s, nrm=0x10200000) == -7
    if bits == 8:
        assert step(s, nrm=0x10500000) == -7  # a scale
    s.plan = None
    assert norm(s) == -1 and step(s) == -1
    s.plan = 0x8000004
    assert norm(s) == -4 and step(s) == -4
    none = _set(bits, n=0)
    assert step(none) == 0  # nothing to do, nothing launched


def test_trainer_refusals():
    import torch
    w = torch.zeros(4)
    with pytest.raises(ValueError):
        runtime.ParamSet([w], [w.clone()], [0.0])  # not on the device
    with pytest.raises(ValueError):
        runtime.ParamSet([w], [], [0.0])
    with pytest.raises(ValueError):
        runtime.ParamSet([w], [w], [0.0], state_bits=16)
    for kw in (dict(optimizer="lion"), dict(optimizer="adam", weight_decay=0.1),
               dict(optimizer="sgd", max_norm=1.0), dict(optimizer="adam", state_bits=8),
               dict(optimizer="adamw", max_norm=0.0)):
        with pytest.raises(ValueError):
            runtime.Trainer(None, [], 4, None, False, **kw)
