"""Edges of the policy loss, the gradient norm and AdamW on the GPU: long rows
with whole chunks of masked actions, borders of the clip, factors and gradients
at the ends of fp32, other streams.  Tolerances as counted in
test_gpu_policy.py, or beside the test."""
import numpy as np
import pytest
import torch

from oracle import policy as P
from paper_2010_03166_amd import gnnprop as G
from paper_2010_03166_amd import runtime

from test_gpu_policy import (SHAPES, U, _case, _f, _host, _params, _room, _tensors, _trainer, _ws,
                             check_logp, check_loss, check_step, run_logp, run_loss)

pytestmark = pytest.mark.gpu

LOW = float(np.finfo(np.float32).min)


# ----------------------------------------------------------- masked chunks

@pytest.mark.parametrize("top", [-100.0, -700.0, -720.0, -1e3, -1e9, LOW, 1e9])
@pytest.mark.parametrize("n,C", SHAPES + [(8, 70000)])
def test_masked_ranges_and_far_logits(n, C, top):
    """The first half of the columns not allowed (many whole 4,096s of them
    in the longer rows), the other logits around `top`."""
    rng = np.random.default_rng([n, C, 31])
    half = C // 2
    z = np.full((n, C), -np.inf, np.float32)
    spread = 2.0 if abs(top) < 1e6 else 0.0  # (fp32's steps are coarser than that there)
    z[:, half:] = top + spread * rng.standard_normal((n, C - half))
    a = rng.integers(half, C, n)
    lp, _ = P.action_logp(z, a)
    adv = rng.standard_normal(n).astype(np.float32)
    old = (lp + 0.25 * rng.standard_normal(n)).astype(np.float32)
    ref = (lp + 0.4 * rng.standard_normal(n)).astype(np.float32)
    w = (rng.random(n) / n).astype(np.float32)
    want = P.policy_loss(z, a, adv, old, ref, w, 0.2, 0.3, 0.05)
    assert np.isfinite(want["out"]).all() and np.isfinite(want["dZ"]).all()
    check_logp(run_logp(z, a), want["logp"], C)
    check_loss(run_loss(z, a, adv, old, ref, w, beta=0.05), want, z, a, adv, old, ref, 0.05)


# ------------------------------------------------------- borders of the clip

@pytest.mark.parametrize("n,C", SHAPES)
def test_ratio_of_zero_is_not_at_a_border(n, C):
    """clip_lo = 1 puts the lower border at 0, where a ratio that underflows
    lies: such rows are as those of a border that no ratio is near."""
    z, a, adv, old, ref, w = _case(n, C, 40)
    old = (P.action_logp(z, a)[0] + 800.0).astype(np.float32)
    at = run_loss(z, a, adv, old, ref, w, lo=1.0, beta=0.05)
    off = run_loss(z, a, adv, old, ref, w, lo=1.0 - 2.0 ** -20, beta=0.05)
    assert np.array_equal(at["dZ"], off["dZ"]) and np.array_equal(at["logp"], off["logp"])
    want = P.policy_loss(z, a, adv, old, ref, w, 1.0, 0.3, 0.05)
    check_loss(at, want, z, a, adv, old, ref, 0.05)


# ------------------------------------------------------------------- AdamW

@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("top", [-1.0, 0.0, float("nan"), float("-inf"), float("inf")])
def test_adamw_without_a_norm_has_no_clipping(bits, top):
    sets = []
    for _ in range(2):
        ts = _tensors([5000, 41], bits, 12)
        sets.append((ts,) + _params(ts, bits))
    G.gnn_adamw_step(sets[0][1], 1e-3, 0.9, 0.999, 1e-8, 3, None, 1.0, 4)
    G.gnn_adamw_step(sets[1][1], 1e-3, 0.9, 0.999, 1e-8, 3, None, top, 4)
    torch.cuda.synchronize()
    for x, y in zip(sets[0][0], sets[1][0]):
        hx, hy = _host(x), _host(y)
        for k in hx:
            assert np.array_equal(hx[k], hy[k]), k
        assert np.isfinite(hx["W"]).all()
