"""Drawn actions, top logits and the student's loss where a border, a NaN or
the order of a sum decides (through the C ABI and the Trainer; tolerances as in
test_gpu_choose.py)."""
import math

import numpy as np
import pytest
import torch

import test_gpu_choose as base

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("C", [7, 20, 41, 121, 600, 3000, 5000, 9000, 20011, 33000, 70001])
def test_min_p_where_the_largest_logit_and_the_cut_cancel(C):
    """A largest logit that is -T ln(min_p) itself: the border lies next to 0, where
    the differences of 6e8 floats are rounded to the cut.  Logits just around 0."""
    rng = np.random.default_rng(C)
    n = 40 if C <= 3000 else 6
    around = [0.0, -0.0] + [s * 2.0 ** e for s in (1, -1) for e in (-149, -126, -60, -54, -53, -52, -30)]
    for T, m in ((1.0, 1), (1.0, 2), (0.5, 2), (2.0, 5), (1.0, 10)):
        min_p = math.exp(-m)
        z = rng.choice(around, (n, C)).astype(np.float32)
        z[:, C // 3] = T * m
        z[1::3, :] += np.where(np.arange(C) == C // 3, 0.0, rng.standard_normal((n, C)))[1::3]
        z[1::3] = np.minimum(z[1::3], T * m)
        u = rng.random(n).astype(np.float32)
        for top_k, top_p in ((0, 1.0), (0, 0.9), (C // 2, 1.0), (5, 0.95), (C // 2, 0.9)):
            a, lp = base.run_sample(z, u, T, top_k, top_p, min_p)
            base.check_sample(z, u, T, top_k, top_p, min_p, a, lp)


@pytest.mark.parametrize("C", [2, 4, 7, 16, 41, 121, 600, 3000, 9000, 20011, 70001])
def test_student_that_is_nan_everywhere(C):
    """A row without a single number is not a row left out: its NaN shows in its kl
    and gradient, whether the list names a NaN, -inf or nothing but them."""
    n = 6
    for k in sorted({1, min(C, 3), min(C, 200)}):
        z, index, logq, rest, w = base._taught(n, C, k, 8, 1.0)
        w[:] = 1.0 / n
        z[0] = np.nan
        z[1] = -np.inf
        z[1, index[1, 0]] = np.nan                # named, all else is not there
        z[2] = -np.inf
        z[2, np.setdiff1d(np.arange(C), index[2])] = np.nan  # the others, where there are any
        z[3] = np.nan
        w[3] = 0.0                                # adds nothing
        z[4] = np.nan
        index[4] = -1                             # left out
        shows = [0, 1] + ([2] if k < C else [])
        for left in (rest, None):
            want = base.O.distill(z, index, logq, left, w, 1.0)
            r = base.run_distill(z, index, logq, left, w, 1.0)
            assert np.isnan(r["out"]) and np.isnan(want["out"])
            for i in shows:
                assert np.isnan(r["kl"][i]) and np.isnan(want["kl"][i]), i
                assert np.isnan(r["dZ"][i]).all() and np.isnan(want["dZ"][i]).all(), i
            if k == C:
                assert r["kl"][2] == 0 and np.all(r["dZ"][2] == 0)
            assert np.isnan(r["kl"][3]) and np.all(r["dZ"][3:5] == 0) and r["kl"][4] == 0
            assert np.isfinite(r["kl"][5]) and np.isfinite(r["dZ"][5]).all()


@pytest.mark.parametrize("C,k", [(16385, 3), (20011, 128), (70001, 256)])
def test_long_rows_parts_are_listed_in_one_order(C, k):
    """What the parts of a long row hand on, which later sums go over, lies in the
    same order in every call."""
    n = 60
    Z = torch.randn((n, C), device="cuda", generator=torch.Generator("cuda").manual_seed(C))
    need = base.G.gnn_top_workspace_bytes(n, C, k)
    first = None
    for _ in range(12):
        ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
        i, q = torch.empty((n, k), dtype=torch.int32, device="cuda"), torch.empty((n, k), device="cuda")
        rest = torch.empty(n, device="cuda")
        base.G.gnn_top_logits(n, C, Z, C, k, 1.0, i, q, rest, ws)
        got = (i, q, rest, ws)
        first = first or got
        for a, b in zip(first, got):
            assert torch.equal(a, b)


def test_policy_steps_keep_no_workspace_of_draws():
    """What drawing and teaching work in is not held for policy steps: the shared
    workspace is the policy's and the products', before those calls and after, and
    its memory stays where it is (a captured step goes on using it)."""
    n, C, f_in, h = 3000, 33000, 24, 16
    rng, S, G = np.random.default_rng(3), base.synth, base.G
    params = [S.LayerParams(S.glorot(f_in, h, rng), S.glorot(f_in, h, rng))]
    f = 2 * h
    tr = base.runtime.Trainer(base.prepared(S.power_law_graph(n, 2.1, 8.0, seed=7)), params, f_in,
                              rng.standard_normal((f, C)).astype(np.float32), False, "sgd", lr=1e-3)
    X = base.to_dev(rng.standard_normal((n, f_in)).astype(np.float32), 28)
    assert G.gnn_sample_workspace_bytes(n, C) > 2 * max(
        G.gnn_gemm_workspace_bytes(*x) for x in ((n, C, f), (f, C, n), (n, f, C)))
    u = torch.rand(n, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    tr.policy_step(X, torch.zeros(n, dtype=torch.int32, device="cuda"), torch.ones(n, device="cuda"))
    held = (tr.policy_ws.numel(), tr.policy_ws.data_ptr())
    assert held[0] == max(G.gnn_policy_workspace_bytes(n, C), G.gnn_gemm_workspace_bytes(n, C, f),
                          G.gnn_gemm_workspace_bytes(f, C, n), G.gnn_gemm_workspace_bytes(n, f, C), 256)
    s = torch.cuda.Stream()
    for stream in (None, s.cuda_stream):
        torch.cuda.synchronize()
        a, lp = tr.act(X, u, 0.9, 50, 0.9, 0.01, stream=stream)
        index, logq, rest = tr.top_logits(X, 3, stream=stream)
        torch.cuda.synchronize()
        Z = tr._Z.view(n)[-9:].cpu().numpy()
        last = lambda *ts: [t[-9:].cpu().numpy() for t in ts]
        base.check_sample(Z, *last(u), 0.9, 50, 0.9, 0.01, *last(a, lp))
        base.check_top(Z, 3, 1.0, last(index, logq, rest))
        tr.distill_step(X, index, logq, rest, stream=stream)
        torch.cuda.synchronize()
        assert held == (tr.policy_ws.numel(), tr.policy_ws.data_ptr())


@pytest.mark.parametrize("C", [1 << 20, (1 << 22) + 3, 1 << 24])
def test_entries_that_count_only_together(C):
    """One entry of weight 1 and all others below 2^(log C - 63), which is half of
    what a sum as large as C would leave as a unit: together they are 2^-23 to 2^-15
    of the sum, and numbers past the first entry's share draw them.  A weight is
    off by 2^-52 and 1e-13 of itself, so what lies before an action by C 2^-52 +
    2e-13 at most."""
    half = 2.0 ** (math.ceil(math.log2(C)) - 63)
    at, tol = C // 2, C * 2.0 ** -52 + 2e-13
    u = np.array([0.0, 0.5, 1 - 2.0 ** -24, 1 - 2.0 ** -23], np.float32)
    for T in (1.0, 0.7):
        z = np.full((1, C), T * math.log(0.9 * half), np.float32)
        z[0, at] = 0.0
        t = math.exp(float(z[0, 0]) / T)
        lse = math.log(1 + (C - 1) * math.exp(float(z[0, 0])))
        z = np.broadcast_to(z, (len(u), C))
        tail = (C - 1) * t
        p = 1 - tail / 4           # a quarter of the others left out
        for top_k, top_p, min_p, others in ((0, 1.0, 0.0, C - 1), (C - 5, 1.0, 0.0, C - 6),
                                            (0, p, 0.0, None), (0, 1.0, t / 2, C - 1),
                                            (C - 5, p, 0.0, None), (0, 1.0, 2 * t, 0)):
            if others is None:     # (a share of the first C - 5 where they are asked for)
                others = math.ceil((p * (1 + (top_k - 1 if top_k else C - 1) * t) - 1) / t)
            a, lp = base.run_sample(z, u, T, top_k, top_p, min_p)
            kept = 1 + others * t
            if others == 0:
                assert np.all(a == at)
                continue
            assert a.max() <= others + tol / t  # (those kept are the first)
            for i in range(len(u)):
                before = a[i] * t if a[i] <= at else 1 + (a[i] - 1) * t
                own = 1.0 if a[i] == at else t
                assert before - 2 * tol <= float(u[i]) * kept <= before + own + 2 * tol, (i, a[i])
            want = np.where(a == at, 0.0, float(z[0, 0])) - lse
            assert np.all(np.abs(lp - want) <= (20 + math.log(C)) * base.U + base.U * np.abs(want))


def test_as_many_equal_logits_as_a_row_has():
    """Sums of 2^24 largest weights fit: an action is a random number's 2^24th."""
    C = 1 << 24
    k = np.array([0, 1, 12345678, C - 1], np.int64)
    z = np.broadcast_to(np.float32(-3.5), (4, C))
    u = (k / C).astype(np.float32)
    for T in (1.0, 5.0):
        a, _ = base.run_sample(z, u, T)
        assert np.array_equal(a, k)
    a, _ = base.run_sample(z, u, 1.0, 0, 0.5)
    assert np.array_equal(a, k // 2)


@pytest.mark.parametrize("n,C", [
    (66000, 9), (66000, 13), (66000, 16), (66000, 17), (66000, 21), (66000, 24), (66000, 25),
    (66000, 32), (66000, 33), (20000, 50), (20000, 121), (9000, 250), (2100, 1000), (1100, 1300),
    (1100, 1537), (1100, 2048), (600, 2049), (300, 3000), (600, 4096), (300, 5000), (600, 6001),
    (600, 8192), (300, 8193), (300, 12289), (300, 16384), (300, 20011), (100, 30000)])
def test_rows_enough_for_every_shape(n, C):
    """Rows as many as other shapes take (lanes alone, wavefronts alone, fewer
    wavefronts): some of them against the oracle, all calls."""
    z, rng = base._logits(n, C, 900, mask=0.2, skip=0.02)
    u = rng.random(n).astype(np.float32)
    some = np.unique(np.concatenate([np.arange(12), n - 1 - np.arange(12), rng.integers(0, n, 16)]))
    for T, top_k, top_p, min_p in base.SETTINGS + [(0.8, C // 3 + 1, 0.9, 0.0)]:
        a, lp = base.run_sample(z, u, T, top_k, top_p, min_p, pad=1, shift=3)
        base.check_sample(z[some], u[some], T, top_k, top_p, min_p, a[some], lp[some])
    for k in (1, 8, 70, 256):
        got = base.run_top(z, k, 1.3, pad=1, shift=1)
        base.check_top(z[some], k, 1.3, tuple(x[some] for x in got))
        t = z + np.float32(0.3) * (np.arange(C) % 5).astype(np.float32)
        index, logq, rest = base.run_top(t, k, 1.3)
        left = np.setdiff1d(np.arange(n), some)
        w = np.zeros(n, np.float32)      # (the loss is then of the rows looked at)
        w[some] = 1.0 / len(some)
        r = base.run_distill(z, index, logq, rest, w, 1.3, pad=2)
        assert np.all(r["dZ"][left] == 0)
        picked = dict(out=r["out"], kl=r["kl"][some], dZ=r["dZ"][some])
        base.check_distill(picked, z[some], index[some], logq[some], rest[some], w[some], 1.3)
