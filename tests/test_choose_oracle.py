"""The oracle of drawn actions, top logits and the student's loss on closed
forms, by brute force and by differences, and the refusals of their entry
points (no GPU)."""
import ctypes
import itertools

import numpy as np
import pytest

from oracle import choose as O
from paper_2010_03166_amd import gnnprop as G

VP = ctypes.c_void_p


def test_order_is_by_logits_then_columns():
    z = [1.0, 3.0, -np.inf, 3.0, -0.0, 0.0, -2.0]
    assert O.order(z).tolist() == [1, 3, 0, 4, 5, 6]
    assert O.left_out([1.0, np.nan]) and O.left_out([-np.inf] * 2) and O.left_out([np.inf, 0.0])
    assert not O.left_out([-np.inf, -5.0])


def test_kept_columns_closed_forms():
    z = np.log(np.array([0.5, 0.2, 0.05, 0.25]))
    keep = lambda *a: O.kept_columns(z, *a)[0].tolist()
    assert keep(1.0) == [0, 3, 1, 2] and keep(1.0, 2) == [0, 3] and keep(1.0, 9) == [0, 3, 1, 2]
    assert keep(1.0, 0, 0.4) == [0] and keep(1.0, 0, 0.6) == [0, 3] and keep(1.0, 0, 0.8) == [0, 3, 1]
    # top_p is a share of the first top_k: 0.5 / 0.75
    assert keep(1.0, 2, 0.66) == [0] and keep(1.0, 2, 0.67) == [0, 3]
    assert keep(1.0, 0, 1.0, 0.45) == [0, 3] and keep(1.0, 0, 1.0, 0.55) == [0]
    # at temperature 1/2 the shares are squares
    assert keep(0.5, 0, 0.7) == [0] and keep(0.5, 0, 0.74) == [0, 3]


@pytest.mark.parametrize("T,top_k,top_p", [(1.0, 0, 1.0), (0.7, 3, 0.8), (2.0, 0, 0.5)])
def test_draws_have_the_shares_of_the_definition(T, top_k, top_p):
    rng = np.random.default_rng(0)
    z = rng.standard_normal(6).astype(np.float32)
    m = 4096
    u = ((np.arange(m) + 0.5) / m).astype(np.float32)
    a, lp, _ = O.sample(np.tile(z, (m, 1)), u, T, top_k, top_p)
    kept, _ = O.kept_columns(z, T, top_k, top_p)
    p = np.zeros(6)
    p[kept] = np.exp(z[kept].astype(np.float64) / T)
    p /= p.sum()
    assert np.all(np.abs(np.bincount(a, minlength=6) / m - p) <= 2.0 / m)
    assert np.all(np.diff(a) >= 0)  # by columns
    full = np.exp(z.astype(np.float64))
    assert np.allclose(np.exp(lp), (full / full.sum())[a], rtol=1e-12)


def test_top_logits_closed_forms():
    z = np.log(np.array([[0.5, 0.2, 0.05, 0.25], [1.0, 1.0, 1.0, 1.0]]))
    z = np.concatenate([z, np.full((1, 4), -np.inf)]).astype(np.float32)
    i, q, r = O.top_logits(z, 2, 1.0)
    assert i.tolist() == [[0, 3], [0, 1], [-1, -1]]
    assert np.allclose(np.exp(q[0]), [0.5, 0.25], rtol=1e-6) and np.allclose(r, [0.25, 0.5, 0], rtol=1e-6)
    i, q, r = O.top_logits(z, 6, 0.5)
    assert i[0].tolist() == [0, 3, 1, 2, -1, -1] and np.all(r == 0)
    assert np.allclose(np.exp(q[0, :4]).sum(), 1.0)


def test_student_loss_closed_forms():
    # a student that agrees: nothing to learn
    z = np.random.default_rng(1).standard_normal((3, 7)).astype(np.float32)
    for T, k in itertools.product((1.0, 3.0), (1, 4, 7)):
        i, q, r = O.top_logits(z, k, T)
        d = O.distill(z, i, q, r, None, T)
        assert abs(d["out"]) < 1e-14 and np.abs(d["dZ"]).max() < 1e-15
    # one column: the cross-entropy, its softmax gradient
    i = np.array([[2], [0], [6]])
    d = O.distill(z, i, np.zeros((3, 1)), None, None, 1.0)
    p = np.exp(z.astype(np.float64))
    p /= p.sum(1, keepdims=True)
    assert np.allclose(d["kl"], -np.log(p[np.arange(3), i[:, 0]]))
    p[np.arange(3), i[:, 0]] -= 1
    assert np.allclose(d["dZ"], p / 3)
    # the gradient of a shift of all logits is 0
    i, q, r = O.top_logits(z[::-1], 3, 2.0)
    assert np.abs(O.distill(z, i, q, r, None, 2.0)["dZ"].sum(1)).max() < 1e-15
    # repeated and unused places
    i2 = np.concatenate([i, i[:, :1], np.full((3, 1), -1)], 1)
    q2 = np.concatenate([q, q[:, :1] + 3, np.zeros((3, 1))], 1)
    a, b = O.distill(z, i, q, r, None, 2.0), O.distill(z, i2, q2, r, None, 2.0)
    assert a["out"] == b["out"] and np.array_equal(a["dZ"], b["dZ"])


@pytest.mark.parametrize("rest", [True, False])
def test_student_gradient_by_differences(rest):
    rng = np.random.default_rng(2)
    z = rng.standard_normal((2, 9))
    i, q, r = O.top_logits(z + rng.standard_normal((2, 9)), 3, 1.7)
    args = (i, q, r if rest else None, np.array([0.3, 0.9]), 1.7)
    d = O.distill(z, *args)
    h = 1e-6
    for a, j in itertools.product(range(2), range(9)):
        up, down = z.copy(), z.copy()
        up[a, j] += h
        down[a, j] -= h
        assert abs((O.distill(up, *args)["out"] - O.distill(down, *args)["out"]) / (2 * h) -
                   d["dZ"][a, j]) < 1e-8


# --------------------------------------------------------------- refusals

def _sample(n=4, C=3, Z=0x1000, ld=3, u=0x2000, T=1.0, k=0, p=1.0, m=0.0, action=0x3000,
            logp=0x3100, ws=0x4000, bytes_=1 << 30):
    return G.lib().gnn_sample_actions(n, C, VP(Z), ld, VP(u), T, k, p, m, VP(action), VP(logp),
                                      VP(ws), bytes_, None)


def _top(n=4, C=3, Z=0x1000, ld=3, k=2, T=1.0, index=0x2000, logq=0x2100, rest=0x2200, ws=0x4000,
         bytes_=1 << 30):
    return G.lib().gnn_top_logits(n, C, VP(Z), ld, k, T, VP(index), VP(logq), VP(rest), VP(ws),
                                  bytes_, None)


def _distill(n=4, C=3, Z=0x1000, ld=3, k=2, index=0x2000, logq=0x2100, rest=0x2200, w=0x2300, T=1.0,
             out=0x3000, kl=0x3100, dZ=0x3200, ld_dz=3, ws=0x4000, bytes_=1 << 30):
    return G.lib().gnn_distill_loss(n, C, VP(Z), ld, k, VP(index), VP(logq), VP(rest), VP(w), T,
                                    VP(out), VP(kl), VP(dZ), ld_dz, VP(ws), bytes_, None)


NAN, INF = float("nan"), float("inf")


def test_refusals_of_all():
    for f in (_sample, _top, _distill):
        assert f(n=-1) == -2 and f(C=0) == -2 and f(ld=2) == -2
        assert f(C=2 ** 24 + 1, ld=2 ** 24 + 1) == -2
        for T in (-1.0, 1e-7, 1e7, NAN, INF):
            assert f(T=T) == -2, T
        assert f(Z=None) == -1
        assert f(ws=0x4004) == -4


def test_sample_refusals():
    for kw in (dict(k=-1), dict(p=0.0), dict(p=-0.1), dict(p=1.1), dict(p=NAN), dict(m=-0.1),
               dict(m=1.1), dict(m=NAN)):
        assert _sample(**kw) == -2, kw
    assert _sample(u=None) == -1 and _sample(action=None) == -1
    for kw in (dict(action=0x1004), dict(action=0x2004), dict(logp=0x1000), dict(logp=0x2008),
               dict(logp=0x3008)):
        assert _sample(**kw) == -7, kw
    assert _sample(n=0, Z=None, u=None, action=None, logp=None) == 0
    long = dict(n=1, C=40000, ld=40000, Z=0x100000)
    need = G.gnn_sample_workspace_bytes(1, 40000)
    if need:
        assert _sample(bytes_=need - 1, **long) == -5 and _sample(ws=None, **long) == -5
    assert G.gnn_sample_workspace_bytes(-1, 3) == 0 == G.gnn_sample_workspace_bytes(3, 0)
    assert G.gnn_sample_workspace_bytes(3, 2 ** 24 + 1) == 0


def test_top_refusals():
    assert _top(T=0.0) == -2 and _top(k=0) == -2 and _top(k=257) == -2 and _top(k=-1) == -2
    assert _top(index=None) == -1 and _top(logq=None) == -1
    for kw in (dict(index=0x1004), dict(logq=0x1000), dict(rest=0x1000), dict(logq=0x2010),
               dict(rest=0x2108)):
        assert _top(**kw) == -7, kw
    assert _top(n=0, Z=None, index=None, logq=None) == 0
    long = dict(n=1, C=40000, ld=40000, Z=0x100000)
    need = G.gnn_top_workspace_bytes(1, 40000, 2)
    if need:
        assert _top(bytes_=need - 1, **long) == -5 and _top(ws=None, **long) == -5
    assert G.gnn_top_workspace_bytes(3, 3, 257) == 0 == G.gnn_top_workspace_bytes(-1, 3, 2)


def test_distill_refusals():
    assert _distill(T=0.0) == -2 and _distill(k=0) == -2 and _distill(k=257) == -2
    assert _distill(ld_dz=2) == -2
    assert _distill(index=None) == -1 and _distill(logq=None) == -1 and _distill(out=None) == -1
    assert _distill(bytes_=4) == -5 and _distill(ws=None) == -5
    for kw in (dict(out=0x1000), dict(out=0x2000), dict(kl=0x2104), dict(kl=0x2200), dict(dZ=0x1000),
               dict(dZ=0x2300), dict(dZ=0x3100), dict(kl=0x3000), dict(ws=0x2200)):
        assert _distill(**kw) == -7, kw
    assert G.gnn_distill_workspace_bytes(-1, 3, 2) == 0 == G.gnn_distill_workspace_bytes(3, 3, 0)
    assert G.gnn_distill_workspace_bytes(3, 2 ** 24 + 1, 2) == 0
    assert G.gnn_distill_workspace_bytes(2 ** 31 - 1, 2 ** 24, 8) > 2 ** 31 * 4096


def test_workspace_of_the_most_rows_serves_fewer():
    rows = [0, 1, 2, 63, 64, 255, 256, 511, 512, 1023, 1024, 2047, 2049, 8191, 8193, 16385, 32769,
            65535, 65536, 200000]
    for C in (1, 3, 7, 16, 17, 121, 500, 1025, 2049, 5000, 16384, 16385, 32769):
        for k in (1, 5, 64, 256):
            for f in (lambda n: G.gnn_sample_workspace_bytes(n, C),
                      lambda n: G.gnn_top_workspace_bytes(n, C, k),
                      lambda n: G.gnn_distill_workspace_bytes(n, C, k)):
                need = [f(n) for n in rows]
                assert need == sorted(need), (C, k)
            assert need == [G.gnn_distill_workspace_bytes(n, C, 256) for n in rows], (C, k)
