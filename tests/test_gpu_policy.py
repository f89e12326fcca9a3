"""Log-probabilities of actions, the policy loss with its gradient, the
gradient norm and AdamW on the GPU against the oracle's doubles (through the
C ABI), and a training step of them together.

Tolerances, with u = 2^-24 (half a step of fp32), derived from the roundings
a kernel may make:
  lp      exp of a rounded difference: the term of x_j = top - z_j is off by
          x_j u + 4 u (expf within 2 ulp = 4 u) relative; the terms' weighted
          mean of x_j is at most ln C, and up to 16 terms may be added in fp32
          before they are added in double: (20 + ln C) u absolute in lp (E
          below), u |lp| for its own rounding.
  slope   rho and exp(d) are off by E relative: w (|A| rho + beta e^d) E, and
          u |slope| for its rounding.
  dZ      p_j is off by (x_j + 24 + ln C) u relative, three more roundings in
          the product; the slope's error times (1[j = a] + p_j).
  out     w (|A| rho + beta e^d) E summed, one rounding.
"""
import numpy as np
import pytest
import torch

from oracle import policy as P
from paper_2010_03166_amd import gnnprop as G
from paper_2010_03166_amd import runtime, synth

from gpu_helpers import prepared, to_dev

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SENTINEL = 12345.0


def _ws(nbytes):
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device="cuda")


def _rows(z, ld, shift):
    """(n, C) view at row stride ld, `shift` floats past a 16-byte boundary,
    in a buffer of NaNs."""
    n, C = z.shape
    buf = torch.full((n * ld + 16,), float("nan"), device="cuda")
    v = buf[shift: shift + n * ld].view(n, ld)[:, :C]
    v.copy_(torch.from_numpy(np.ascontiguousarray(z, np.float32)))
    return v


def _f(x):
    return None if x is None else torch.from_numpy(np.asarray(x, np.float32)).cuda()


def _case(n, C, seed, mask=0.0, skip=0.0):
    rng = np.random.default_rng([n, C, seed])
    z = (rng.standard_normal((n, C)) * 2.5).astype(np.float32)
    a = rng.integers(0, C, n)
    if mask:
        z[rng.random((n, C)) < mask] = -np.inf
        z[np.arange(n), a] = rng.standard_normal(n)
    lp, _ = P.action_logp(z, a)
    adv = rng.standard_normal(n).astype(np.float32)
    old = (lp + 0.25 * rng.standard_normal(n)).astype(np.float32)
    ref = (lp + 0.4 * rng.standard_normal(n)).astype(np.float32)
    w = (rng.random(n) / n).astype(np.float32)
    if skip:
        out = rng.random(n) < skip
        a = np.where(out, rng.choice([-1, C, 2 ** 31 - 1, -2 ** 31], n), a)
        z[out] = np.nan
    return z, a, adv, old, ref, w


def run_loss(z, a, adv, old=None, ref=None, w=None, lo=0.2, hi=0.3, beta=0.0, pad=0, shift=0,
             want_dz=True, want_logp=True, stream=None):
    n, C = z.shape
    ld = C + pad
    Z = _rows(z, ld, shift)
    dbuf = torch.full((n * ld + 16,), SENTINEL, device="cuda")
    dZ = dbuf[shift: shift + n * ld].view(n, ld)
    lbuf = torch.full((n + 8,), SENTINEL, device="cuda")
    out = torch.full((8,), SENTINEL, device="cuda")
    act = torch.from_numpy(np.asarray(a).astype(np.int32)).cuda()
    G.gnn_policy_loss(n, C, Z, ld, act, _f(adv), _f(old), _f(ref), _f(w), lo, hi, beta, out,
                      lbuf if want_logp else None, dZ if want_dz else None, ld,
                      _ws(G.gnn_policy_workspace_bytes(n, C)), stream)
    torch.cuda.synchronize()
    # nothing outside the outputs is written
    assert torch.all(out[3:] == SENTINEL) and torch.all(lbuf[n if want_logp else 0:] == SENTINEL)
    assert torch.all(dbuf[:shift] == SENTINEL) and torch.all(dbuf[shift + n * ld:] == SENTINEL)
    assert torch.all(dZ[:, C if want_dz else 0:] == SENTINEL)
    return dict(out=out[:3].cpu().numpy(), logp=lbuf[:n].cpu().numpy(),
                dZ=dZ[:, :C].cpu().numpy().copy())


def run_logp(z, a, pad=0, shift=0):
    n, C = z.shape
    lbuf = torch.full((n + 8,), SENTINEL, device="cuda")
    G.gnn_action_logp(n, C, _rows(z, C + pad, shift), C + pad,
                      torch.from_numpy(np.asarray(a).astype(np.int32)).cuda(), lbuf,
                      _ws(G.gnn_policy_workspace_bytes(n, C)))
    torch.cuda.synchronize()
    assert torch.all(lbuf[n:] == SENTINEL)
    return lbuf[:n].cpu().numpy()


def check_logp(got, want, C):
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine])
    got, want = got[fine], want[fine]
    assert np.all(np.abs(got - want) <= (20 + np.log(C)) * U + U * np.abs(want))


def check_loss(r, ref, z, a, adv, old, refp, beta):
    n, C = z.shape
    E = (20 + np.log(C)) * U
    check_logp(r["logp"], ref["logp"], C)
    live = ref["live"] & (ref["w"] != 0)
    d = np.zeros(n) if refp is None else np.where(live, refp - ref["logp"], 0.0)
    sens = np.where(live, ref["w"] * (np.abs(adv) * ref["rho"] + beta * np.exp(d)), 0.0)
    kls = np.where(live, ref["w"] * np.abs(np.expm1(d)), 0.0) if refp is not None else sens
    o, want = r["out"], ref["out"]
    assert abs(o[0] - want[0]) <= (sens.sum() + beta * kls.sum()) * E + 2 * U * abs(want[0])
    assert abs(o[1] - want[1]) <= kls.sum() * E + 2 * U * abs(want[1])
    assert abs(o[2] - want[2]) <= 2 * U * abs(want[2])
    with np.errstate(all="ignore"):
        zz = z.astype(np.float64)
        top = np.max(zz, 1, keepdims=True, initial=-np.inf, where=~np.isnan(zz))
        x = np.where(np.isfinite(zz), top - zz, 0.0)
        p = np.where(live[:, None], np.exp(zz - top) /
                     np.sum(np.exp(zz - top), 1, keepdims=True), 0.0)
    one = np.zeros((n, C))
    one[live, np.asarray(a)[live]] = 1.0
    tol = (sens * E + U * np.abs(ref["slope"]))[:, None] * (one + p) + \
        np.abs(ref["slope"])[:, None] * (p * (x + 27 + np.log(C)) + one * 3) * U
    assert np.all(np.abs(r["dZ"] - ref["dZ"]) <= tol)
    assert np.all(r["dZ"][~live] == 0)


WIDTHS = [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 32, 33, 41, 63, 64, 65, 100, 121, 127, 128, 129,
          255, 256, 257, 500, 511, 512, 513, 1000, 1023, 1024, 1025, 2047, 2048, 2049, 4095,
          4096, 4097]


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("n", [1, 37, 700])
def test_policy_widths(n, C):
    n = min(n, max(1, 1_000_000 // C))
    pad, shift = (C % 3, C % 4)
    z, a, adv, old, ref, w = _case(n, C, 0, mask=0.2 if C % 2 else 0.0, skip=0.2)
    beta = 0.0 if n == 37 else 0.07
    want = P.policy_loss(z, a, adv, old, ref, w, 0.2, 0.3, beta)
    r = run_loss(z, a, adv, old, ref, w, beta=beta, pad=pad, shift=shift)
    check_loss(r, want, z, a, adv, old, ref, beta)
    check_logp(run_logp(z, a, pad, shift), want["logp"], C)


@pytest.mark.parametrize("n,C", [(1, 8191), (3, 8192), (40, 9000), (5, 16384), (2, 16385),
                                 (300, 16390), (1, 32768), (2, 32769), (70, 33000), (1, 100003),
                                 (3, 131072), (1, 1000003), (6000, 300), (20000, 41), (70001, 7), (9001, 515)])
@pytest.mark.parametrize("aligned", [True, False])
def test_policy_long_rows_and_many(n, C, aligned):
    pad = -C % 4 if aligned else 1 + C % 2
    z, a, adv, old, ref, w = _case(n, C, 1, mask=0.1, skip=0.1 if n > 2 else 0.0)
    want = P.policy_loss(z, a, adv, old, ref, w, 0.2, 0.3, 0.05)
    r = run_loss(z, a, adv, old, ref, w, beta=0.05, pad=pad, shift=0 if aligned else 1)
    check_loss(r, want, z, a, adv, old, ref, 0.05)
    check_logp(run_logp(z, a, pad, 0 if aligned else 1), want["logp"], C)


SHAPES = [(300, 9), (40, 700), (6, 20000), (2, 70000)]  # every way of taking rows


@pytest.mark.parametrize("n,C", SHAPES)
def test_policy_optional_arguments(n, C):
    z, a, adv, old, ref, w = _case(n, C, 2)
    full = run_loss(z, a, adv, old, ref, w, beta=0.1)
    for kw in (dict(want_dz=False), dict(want_logp=False), dict(want_dz=False, want_logp=False)):
        r = run_loss(z, a, adv, old, ref, w, beta=0.1, **kw)
        assert np.array_equal(r["out"], full["out"])
    for o, rf, ww in ((None, ref, w), (old, None, w), (old, ref, None), (None, None, None)):
        want = P.policy_loss(z, a, adv, o, rf, ww, 0.2, 0.3, 0.0)
        r = run_loss(z, a, adv, o, rf, ww)
        check_loss(r, want, z, a, adv, o, rf, 0.0)
        if o is None:
            assert r["out"][2] == 0
        if rf is None:
            assert r["out"][1] == 0
    # no clip above, all of the ratio cut below
    want = P.policy_loss(z, a, adv, old, ref, w, 1.0, np.inf, 0.1)
    r = run_loss(z, a, adv, old, ref, w, lo=1.0, hi=float("inf"), beta=0.1)
    check_loss(r, want, z, a, adv, old, ref, 0.1)


@pytest.mark.parametrize("n,C", SHAPES)
def test_policy_masked_and_extreme_rows(n, C):
    """Rows without any action, masks of the lowest value, a row's only
    action, weights of 0 over garbage, huge logits."""
    z, a, adv, old, ref, w = _case(n, C, 3)
    low = np.finfo(np.float32).min
    z[0] = -np.inf                             # nothing to choose: left out
    z[1, :] = -np.inf
    z[1, a[1]] = 3.0                           # one action: lp = 0
    old[1], ref[1] = -0.1, 0.1
    if n > 5:
        z[2, :] = low                          # uniform
        old[2] = ref[2] = -np.log(C)
        z[3, :] = low
        z[3, a[3]] = -low                      # all the weight on the action
        old[3] = ref[3] = 0.0
        w[4] = 0.0
        z[4] = np.nan                          # weight 0: whatever the logits
    lp, _ = P.action_logp(z, a)
    assert lp[0] == -np.inf and lp[1] == 0
    want = P.policy_loss(z, a, adv, old, ref, w, 0.2, 0.3, 0.05)
    r = run_loss(z, a, adv, old, ref, w, beta=0.05)
    if n > 5:
        assert np.isnan(r["logp"][4])
        r["logp"][4] = want["logp"][4] = 0.0
        assert abs(r["logp"][2] + np.log(C)) <= (20 + np.log(C)) * U * 2 and r["logp"][3] == 0
    assert np.all(r["dZ"][1] == 0) or abs(r["dZ"][1, a[1]]) <= 4 * U * abs(want["slope"][1])
    check_loss(r, want, np.nan_to_num(z, nan=0.0, neginf=-np.inf, posinf=np.inf), a, adv, old,
               ref, 0.05)
    # every row left out
    r = run_loss(z, np.full(n, -1), adv, old, ref, w, beta=0.05)
    assert np.all(r["out"] == 0) and np.all(r["dZ"] == 0) and np.all(r["logp"] == 0)


@pytest.mark.parametrize("n,C", SHAPES)
def test_policy_not_finite_rows_stay_alone(n, C):
    z, a, adv, old, ref, w = _case(n, C, 4)
    clean = run_loss(z, a, adv, old, ref, w, beta=0.05)
    z[0, C // 2] = np.nan
    z[1, C - 1] = np.inf
    r = run_loss(z, a, adv, old, ref, w, beta=0.05)
    assert np.isnan(r["out"][0]) and np.isnan(r["dZ"][0]).all()
    assert np.isnan(r["dZ"][1]).any() and not np.isfinite(r["logp"][0])
    assert np.array_equal(r["dZ"][2:], clean["dZ"][2:])
    assert np.array_equal(r["logp"][2:], clean["logp"][2:])
    r = run_loss(z, a, adv, None, None, w)  # on-policy: a NaN shows as well
    assert np.isnan(r["out"][0]) and np.isnan(r["dZ"][0]).all()
    # a chosen action without probability: lp = -inf, no slope without beta
    z, a, adv, old, ref, w = _case(n, C, 4)
    z[0, a[0]] = -np.inf
    r = run_loss(z, a, adv, old, None, w)
    assert r["logp"][0] == -np.inf and np.all(r["dZ"][0] == 0) and np.isfinite(r["out"]).all()
    r = run_loss(z, a, adv, old, ref, w, beta=0.05)
    assert r["out"][0] == np.inf and r["out"][1] == np.inf


@pytest.mark.parametrize("n,C", SHAPES)
def test_policy_ratios_without_bound(n, C):
    """Old log-probabilities of -inf and far below: a ratio that is infinite,
    or beyond fp32, is clipped for a positive advantage, counts for nothing
    with an advantage of 0 and shows for a negative one."""
    z, a, adv, old, ref, w = _case(n, C, 9)
    lp, _ = P.action_logp(z, a)
    w[:] = 1.0 / n
    old[:2] = [-np.inf, lp[1] - 120.0][: 2]
    adv[:2] = 1.0
    want = P.policy_loss(z, a, adv, old, ref, w, 0.2, 0.3, 0.05)
    assert want["cut"][:2].all() and np.isfinite(want["out"]).all()
    r = run_loss(z, a, adv, old, ref, w, beta=0.05)
    with np.errstate(all="ignore"):
        want["rho"][:2] = 1.3  # clipped there: that is what the loss depends on
    check_loss(r, want, z, a, adv, np.where(np.isinf(old), 0, old), ref, 0.05)
    adv[1] = 0.0  # e^120 times nothing
    r = run_loss(z, a, adv, old, ref, w, beta=0.0)
    assert np.isfinite(r["out"]).all() and np.all(r["dZ"][1] == 0)
    adv[0] = -1.0
    r = run_loss(z, a, adv, old, ref, w, beta=0.0)
    assert r["out"][0] == np.inf and not np.isfinite(r["dZ"][0]).all()
    assert np.isfinite(r["dZ"][1:]).all()


@pytest.mark.parametrize("n,C", SHAPES + [(5000, 41)])
def test_policy_clip_of_nothing(n, C):
    """clip = (0, 0) at the old policy: every ratio is next to both borders."""
    z, a, adv, old, ref, w = _case(n, C, 10)
    lp, _ = P.action_logp(z, a)
    old = lp.astype(np.float32)
    r = run_loss(z, a, adv, old, ref, w, lo=0.0, hi=0.0, beta=0.05)
    want = P.policy_loss(z, a, adv, old, ref, w, 0.0, 0.0, 0.05)
    near = np.abs(want["rho"] - 1) < 1e-10
    assert near.mean() < 0.2 or n < 10
    if not near.any():
        check_loss(r, want, z, a, adv, old, ref, 0.05)
    # by rows: those that are decided, on their side
    keep = np.where(near, -1, a)
    want = P.policy_loss(z, keep, adv, old, ref, w, 0.0, 0.0, 0.05)
    r = run_loss(z, keep, adv, old, ref, w, lo=0.0, hi=0.0, beta=0.05)
    check_loss(r, want, z, keep, adv, old, ref, 0.05)


@pytest.mark.parametrize("n,C", [(4096, 41), (600, 1000), (40, 20000), (2, 131072)])
def test_policy_next_to_the_border(n, C):
    """Ratios that round to the clip's border, just inside and just outside:
    each row is decided as in doubles, or lies within 1e-10 of the border."""
    z, a, adv, old, ref, w = _case(n, C, 5)
    lp, _ = P.action_logp(z, a)
    rng = np.random.default_rng(8)
    side = np.where(rng.random(n) < 0.5, 0.8, 1.3)
    old = (lp - np.log(side)).astype(np.float32)
    r = run_loss(z, a, adv, old, ref, w)
    want = P.policy_loss(z, a, adv, old, ref, w, 0.2, 0.3, 0.0)
    near = np.abs(want["rho"] - side) < 1e-10
    assert near.mean() < 0.1 and np.abs(want["rho"] / side - 1).max() < 1e-5
    cut = np.all(r["dZ"] == 0, axis=1)
    assert np.array_equal(cut[~near], want["cut"][~near])
    # a row is cut where its advantage has the side's sign (one in two) and
    # old rounded to the outside (one in two): n / 4, give or take four
    # standard deviations of sqrt(n 3 / 16)
    assert abs(want["cut"].sum() - n / 4) <= np.sqrt(3 * n)


@pytest.mark.parametrize("n,C", SHAPES + [(9000, 41)])
def test_policy_same_bits_and_other_streams(n, C):
    z, a, adv, old, ref, w = _case(n, C, 6)
    one = run_loss(z, a, adv, old, ref, w, beta=0.05)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for stream in (None, s.cuda_stream, s):
        if stream is not None:
            torch.cuda.synchronize()
        two = run_loss(z, a, adv, old, ref, w, beta=0.05, stream=stream)
        for k in one:
            assert np.array_equal(one[k], two[k]), k


def test_policy_no_rows():
    out = torch.full((3,), SENTINEL, device="cuda")
    G.gnn_policy_loss(0, 5, None, 5, None, None, None, None, None, 0.2, 0.2, 0.0, out, None, None,
                      5, None)
    G.gnn_action_logp(0, 5, None, 5, None, None, None)
    torch.cuda.synchronize()
    assert torch.all(out == 0)


def test_policy_offsets_past_32_bits():
    """Rows whose offsets pass 2^31 elements (and 2^32 bytes long before)."""
    n, C, ld = 70000, 41, 40000
    Z = torch.empty((n, ld), device="cuda")[:, :C]
    dZ = torch.empty((n, ld), device="cuda")[:, :C]
    g = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn((n, C), device="cuda", generator=g)
    Z.copy_(z)
    act = torch.randint(0, C, (n,), device="cuda", generator=g, dtype=torch.int32)
    adv = torch.randn(n, device="cuda", generator=g)
    res = []
    for zz, lz, dd, ldd in ((z, C, torch.empty_like(z), C), (Z, ld, dZ, ld)):
        out, logp = torch.empty(3, device="cuda"), torch.empty(n, device="cuda")
        G.gnn_policy_loss(n, C, zz, lz, act, adv, None, None, None, 0.2, 0.2, 0.0, out, logp, dd,
                          ldd, _ws(G.gnn_policy_workspace_bytes(n, C)))
        torch.cuda.synchronize()
        res.append((out, logp, dd))
    for x, y in zip(*res):
        assert torch.equal(x, y)


def _random_cases(count=60, seed=77):
    rng = np.random.default_rng(seed)
    out = []
    for i in range(count):
        C = int(round(2.0 ** rng.uniform(0, 15.6)))
        n = int(round(2.0 ** rng.uniform(0, np.log2(min(4000, max(2, 600000 // C))))))
        out.append((i, n, C, int(rng.integers(0, 9)), int(rng.integers(0, 4)),
                    float(rng.choice([0.0, 0.4])), float(rng.choice([0.0, 0.3])),
                    tuple(bool(b) for b in rng.integers(0, 2, 3)),
                    float(rng.choice([0.0, 0.02, 1.0])),
                    float(rng.choice([0.0, 0.1, 1.0])), float(rng.choice([0.0, 0.3, 10.0]))))
    return out


@pytest.mark.parametrize("case", _random_cases(), ids=lambda c: "case%d" % c[0])
def test_policy_random_calls(case):
    """Seeded random rows, columns, strides, alignments, masks, optional
    arrays, clips and KL weights."""
    i, n, C, pad, shift, mask, skip, has, beta, lo, hi = case
    z, a, adv, old, ref, w = _case(n, C, 1000 + i, mask=mask, skip=skip)
    old, w = old if has[0] else None, w if has[1] else None
    if not has[2] and beta == 0.0:
        ref = None
    want = P.policy_loss(z, a, adv, old, ref, w, lo, hi, beta)
    r = run_loss(z, a, adv, old, ref, w, lo=lo, hi=hi, beta=beta, pad=pad, shift=shift)
    check_loss(r, want, z, a, adv, old, ref, beta)
    check_logp(run_logp(z, a, pad, shift), want["logp"], C)


def _room(nbytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < nbytes:
        pytest.skip("needs %d GB of free device memory" % (nbytes >> 30))


def test_policy_more_blocks_than_one_launch():
    """2^21 + 50 rows of a block each (two launches): the same rows in calls
    of one launch give the same bits."""
    n, C, cut = 2 ** 21 + 50, 520, 2 ** 21 - 100
    _room(30 << 30)
    g = torch.Generator(device="cuda").manual_seed(2)
    Z = torch.randn((n, C), device="cuda", generator=g)
    act = torch.randint(0, C, (n,), device="cuda", generator=g, dtype=torch.int32)
    adv, old, w = (torch.randn(n, device="cuda", generator=g) for _ in range(3))
    old.sub_(7.0)
    w.abs_().div_(n)
    ws = _ws(G.gnn_policy_workspace_bytes(n, C))
    dZ = torch.empty_like(Z)
    res = []
    for parts in ([(0, n)], [(0, cut), (cut, n)]):
        dZ.fill_(SENTINEL)
        logp = torch.empty(n, device="cuda")
        outs = []
        for b, e in parts:
            out = torch.empty(3, device="cuda")
            G.gnn_policy_loss(e - b, C, Z[b:e], C, act[b:e], adv[b:e], old[b:e], old[b:e], w[b:e],
                              0.2, 0.2, 0.1, out, logp[b:e], dZ[b:e], C, ws)
            outs.append(out)
        torch.cuda.synchronize()
        res.append((torch.stack(outs).double().sum(0), logp, dZ[::7].clone(), dZ[-2000:].clone()))
    # one rounding of each output, of two in the second case
    assert bool(((res[0][0] - res[1][0]).abs() <= 4 * U * res[0][0].abs().clamp(min=1e-3)).all())
    for x, y in zip(res[0][1:], res[1][1:]):
        assert torch.equal(x, y)


def test_policy_two_calls_at_once():
    """Two streams, each with its own workspace, call after call."""
    cases = [_case(3000, 121, 20), _case(40, 20000, 21), _case(3, 70000, 22), _case(9000, 7, 23)]
    alone = [run_loss(*c, beta=0.05) for c in cases]
    args, streams = [], [torch.cuda.Stream() for _ in cases]
    for z, a, adv, old, ref, w in cases:
        n, C = z.shape
        args.append([n, C, to_dev(z), C, torch.from_numpy(a.astype(np.int32)).cuda(), _f(adv),
                     _f(old), _f(ref), _f(w), 0.2, 0.3, 0.05, torch.zeros(3, device="cuda"),
                     torch.zeros(n, device="cuda"), torch.zeros((n, C), device="cuda"), C,
                     _ws(G.gnn_policy_workspace_bytes(n, C))])
    torch.cuda.synchronize()
    for _ in range(20):
        for x, s in zip(args, streams):
            G.gnn_policy_loss(*x, stream=s)
    torch.cuda.synchronize()
    for x, one in zip(args, alone):
        assert np.array_equal(x[12].cpu().numpy(), one["out"])
        assert np.array_equal(x[13].cpu().numpy(), one["logp"])
        assert np.array_equal(x[14].cpu().numpy(), one["dZ"])


@pytest.mark.parametrize("n,C", SHAPES)
def test_policy_graph_replay(n, C):
    """Captured and replayed between eager calls, its inputs changed."""
    z, a, adv, old, ref, w = _case(n, C, 7)
    Z, act = to_dev(z), torch.from_numpy(a.astype(np.int32)).cuda()
    A, o, rf, ww = _f(adv), _f(old), _f(ref), _f(w)
    bufs = [[torch.zeros(3, device="cuda"), torch.zeros(n, device="cuda"),
             torch.zeros((n, C), device="cuda"), _ws(G.gnn_policy_workspace_bytes(n, C))]
            for _ in range(2)]

    def call(b, stream=None):
        G.gnn_policy_loss(n, C, Z, C, act, A, o, rf, ww, 0.2, 0.3, 0.05, b[0], b[1], b[2], C, b[3],
                          stream)

    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call(bufs[0], s.cuda_stream)
    for it in range(3):
        Z.add_(0.1 * torch.randn_like(Z))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        call(bufs[1])
        torch.cuda.synchronize()
        for x, y in zip(bufs[0][:3], bufs[1][:3]):
            assert torch.equal(x, y), it


# ------------------------------------------------- sets of tensors: helpers

def _tensors(counts, bits, seed, shift=0, zero_state=False):
    """Weights, gradients and moments at `shift` elements past alignment, in
    buffers with guards: list of dicts of (view, buffer, start)."""
    rng = np.random.default_rng(seed)
    out = []

    def put(x, dtype):
        x = np.asarray(x)
        buf = torch.full((len(x) + 40,), 77, dtype=dtype, device="cuda")
        v = buf[16 + shift: 16 + shift + len(x)]
        v.copy_(torch.from_numpy(x))
        return v, buf, 16 + shift

    for c in counts:
        size = np.exp(2 * rng.standard_normal(c))
        g = (rng.standard_normal(c) * size * 1e-2).astype(np.float32)
        t = dict(W=put(rng.standard_normal(c).astype(np.float32) * 0.1, torch.float32),
                 G=put(g, torch.float32))
        m = np.zeros(c) if zero_state else 0.5 * g * rng.standard_normal(c)
        v = np.zeros(c) if zero_state else g.astype(np.float64) ** 2 * (0.5 + rng.random(c))
        if bits == 32:
            t["m"], t["v"] = put(m.astype(np.float32), torch.float32), \
                put(v.astype(np.float32), torch.float32)
        else:
            for k, x, grid in (("m", m, P.E4M3), ("v", v, P.E5M2)):
                s = P.scales(x, grid).astype(np.float32)
                code, _ = P.encode(x, s, grid, np.full(c, 32768), k == "v")
                t[k] = put(code.astype(np.uint8), torch.uint8)
                t[k + "_scale"] = put(s, torch.float32)
        out.append(t)
    return out


def _host(t):
    return {k: v[0].cpu().numpy().copy() for k, v in t.items()}


def _params(ts, bits, decay=None):
    tuples = []
    for i, t in enumerate(ts):
        tuples.append((t["W"][0], t["G"][0], t["m"][0], t["v"][0]) +
                      ((t["m_scale"][0], t["v_scale"][0]) if bits == 8 else (None, None)) +
                      (0.1 * (i % 3) if decay is None else decay,))
    ps = G.make_params(tuples, bits)
    plan = torch.empty(G.gnn_params_plan_bytes(ps), dtype=torch.uint8, device="cuda")
    ps.plan = plan.data_ptr()
    ps._plan = plan
    G.gnn_params_build_plan(ps, plan)
    return ps, [x[6] for x in tuples]


def _guards_intact(ts):
    for t in ts:
        for k, (v, buf, at) in t.items():
            assert torch.all(buf[:at] == 77) and torch.all(buf[at + v.numel():] == 77), k


def check_step(before, ts, bits, decays, lr, b1, b2, eps, t, k, seed=0):
    """Weights and moments after a step against the oracle.  Roundings (u each,
    relative): 32-bit moments: the coefficient, the factor k, the product and
    the sum, of b1 |m| + (1 - b1) |k g| for m (5 u) and of v (8 u: g twice).
    The update lr (m / c1) / (sqrt(v / c2) + eps): m's error, half of v's, its
    own five operations and coefficients (8 u); the weight's product and sum
    (3 u)."""
    first = 0
    for h, tt, d in zip(before, ts, decays):
        now = _host(tt)
        c = len(h["W"])
        assert np.array_equal(h["G"], now["G"])
        if bits == 32:
            m0, v0 = h["m"].astype(np.float64), h["v"].astype(np.float64)
        else:
            m0, v0 = P.decode(h["m"], h["m_scale"], P.E4M3), P.decode(h["v"], h["v_scale"], P.E5M2)
        W, m, v = P.adamw(h["W"], h["G"], m0, v0, lr, b1, b2, eps, t, d, k)
        size = b1 * np.abs(m0) + (1 - b1) * np.abs(k * h["G"].astype(np.float64))
        den = np.sqrt(v / (1 - b2 ** t)) + eps
        upd = lr * np.abs(m) / (1 - b1 ** t) / den
        tol_w = 3 * U * np.abs(h["W"]) + lr * 6 * U * size / (1 - b1 ** t) / den + 14 * U * upd
        # an underflowing second moment: half a step of the smallest fp32
        tiny = 2.0 ** -149
        tol_w = np.where(v < 2.0 ** -120, upd + lr * 1e3 * U, tol_w)
        assert np.all(np.abs(now["W"] - W) <= tol_w)
        if bits == 32:
            assert np.all(np.abs(now["m"] - m) <= 5 * U * size + 4 * tiny)
            assert np.all(np.abs(now["v"] - v) <= 8 * U * v + 4 * tiny)
        else:
            r = P.random_bits(seed, t, first, c)
            for name, x, grid, rr in (("m", m, P.E4M3, r & 0xFFFF), ("v", v, P.E5M2, r >> 16)):
                s = now[name + "_scale"]
                exact = P.scales(x, grid)
                assert np.all(np.abs(s - exact) <= U * exact * (1 + 1e-9))
                code, room = P.encode(x, s, grid, rr, name == "v")
                # decided alike, unless the decision lies within the rounding
                # of doubles (a few 2^-53, times 8 steps to a power of two)
                differ = code != now[name]
                assert np.all(room[differ] < 1e-13), name
        first += -(-c // P.BLOCK)
    _guards_intact(ts)


COUNTS = [[1], [3, 0, 5], [255, 256, 257], [2047, 2048, 2049], [100000, 7],
          [602 * 128, 602 * 128, 128, 128, 256 * 41],
          [((i * 37) % 50) * 41 + i % 3 for i in range(100)]]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [0, 1, 2, 4])
@pytest.mark.parametrize("case", range(len(COUNTS)))
def test_adamw_steps(case, shift, bits):
    ts = _tensors(COUNTS[case], bits, case, shift)
    ps, decays = _params(ts, bits)
    for t in (5, 6):
        before = [_host(x) for x in ts]
        G.gnn_adamw_step(ps, 1e-2, 0.9, 0.99, 1e-8, t, seed=99)
        torch.cuda.synchronize()
        check_step(before, ts, bits, decays, 1e-2, 0.9, 0.99, 1e-8, t, 1.0, 99)


@pytest.mark.parametrize("seed", range(12))
def test_adamw_random_sets(seed):
    """Seeded random sets: tensors of any length at any alignment, random
    hyperparameters, steps and clipping."""
    rng = np.random.default_rng(500 + seed)
    bits = 8 if seed % 2 else 32
    counts = [int(2.0 ** rng.uniform(0, 15)) for _ in range(int(rng.integers(1, 40)))]
    ts = _tensors(counts, bits, seed, int(rng.integers(0, 5)))
    ps, decays = _params(ts, bits)
    norm = torch.zeros(1, device="cuda")
    b1, b2 = float(rng.choice([0.0, 0.5, 0.9])), float(rng.choice([0.0, 0.95, 0.999]))
    lr, eps = float(rng.choice([0.0, 1e-4, 0.1])), float(rng.choice([1e-12, 1e-8, 1e-3]))
    for _ in range(2):
        t = int(rng.integers(1, 100000))
        G.gnn_grad_norm(ps, norm, _ws(G.gnn_grad_norm_workspace_bytes(ps)))
        n = float(norm)
        want = P.grad_norm([x["G"][0].cpu().numpy() for x in ts])
        assert abs(n - want) <= U * want * (1 + 1e-6)
        top = n * float(rng.choice([0.01, 0.9, 5.0]))
        before = [_host(x) for x in ts]
        G.gnn_adamw_step(ps, lr, b1, b2, eps, t, norm, top, seed * 7919)
        torch.cuda.synchronize()
        check_step(before, ts, bits, decays, lr, b1, b2, eps, t, min(1.0, top / n), seed * 7919)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_from_zero_moments(bits):
    ts = _tensors([5000, 300], bits, 3, zero_state=True)
    ps, decays = _params(ts, bits)
    ts[0]["G"][0][1000:2000].zero_()  # blocks without any gradient
    for t in (1, 2, 3):
        before = [_host(x) for x in ts]
        G.gnn_adamw_step(ps, 1e-3, 0.9, 0.999, 1e-8, t, seed=2 ** 64 - 1)
        torch.cuda.synchronize()
        check_step(before, ts, bits, decays, 1e-3, 0.9, 0.999, 1e-8, t, 1.0, 2 ** 64 - 1)
    if bits == 8:
        now = _host(ts[0])
        v = P.decode(now["v"], now["v_scale"], P.E5M2)
        assert np.all((now["G"] == 0) | (v > 0))


@pytest.mark.parametrize("counts", [[], [0], [1], [5, 0, 300], [2048 * 3000 + 17], COUNTS[6]])
@pytest.mark.parametrize("shift", [0, 1])
def test_grad_norm(counts, shift):
    ts = _tensors(counts, 32, 11, shift)
    ps, _ = _params(ts, 32)
    ws = _ws(G.gnn_grad_norm_workspace_bytes(ps))
    norm = torch.full((4,), SENTINEL, device="cuda")
    for _ in range(2):
        G.gnn_grad_norm(ps, norm, ws)
        torch.cuda.synchronize()
        want = P.grad_norm([t["G"][0].cpu().numpy() for t in ts])
        assert abs(float(norm[0]) - want) <= U * want * (1 + 1e-6)
        assert torch.all(norm[1:] == SENTINEL)
        for t in ts:  # squares that fp32 cannot hold
            t["G"][0].mul_(1e25)
    _guards_intact(ts)


def test_grad_norm_needs_gradients_only():
    g = [torch.full((1000,), 2.0, device="cuda"), torch.full((9,), 3.0, device="cuda")]
    ps = G.make_params([(None, x) for x in g] + [(None, g[0])])  # one of them shared
    plan = torch.empty(G.gnn_params_plan_bytes(ps), dtype=torch.uint8, device="cuda")
    ps.plan = plan.data_ptr()
    G.gnn_params_build_plan(ps, plan)
    norm = torch.zeros(1, device="cuda")
    G.gnn_grad_norm(ps, norm, _ws(G.gnn_grad_norm_workspace_bytes(ps)))
    assert float(norm) == np.float32(np.sqrt(8000 + 81))
    with pytest.raises(G.GnnError):
        G.gnn_adamw_step(ps, 0.1, 0.9, 0.99, 1e-8, 1)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_clipped_and_skipped(bits):
    ts = _tensors([4000, 300, 41], bits, 5)
    ps, decays = _params(ts, bits)
    norm = torch.zeros(1, device="cuda")
    G.gnn_grad_norm(ps, norm, _ws(G.gnn_grad_norm_workspace_bytes(ps)))
    n = float(norm)
    for top in (n / 3, n, 2 * n, float("inf")):
        before = [_host(x) for x in ts]
        G.gnn_adamw_step(ps, 1e-3, 0.9, 0.999, 1e-8, 3, norm, top, 4)
        torch.cuda.synchronize()
        check_step(before, ts, bits, decays, 1e-3, 0.9, 0.999, 1e-8, 3, min(1.0, top / n), 4)
    # a norm that is not finite: nothing is changed
    for bad in (float("nan"), float("inf"), float("-inf")):
        ts[0]["G"][0][7] = bad
        G.gnn_grad_norm(ps, norm, _ws(G.gnn_grad_norm_workspace_bytes(ps)))
        before = [_host(x) for x in ts]
        assert not np.isfinite(float(norm))
        G.gnn_adamw_step(ps, 1e-3, 0.9, 0.999, 1e-8, 3, norm, 1.0, 4)
        torch.cuda.synchronize()
        for h, x in zip(before, ts):
            for k, v in _host(x).items():
                assert np.array_equal(v, h[k], equal_nan=v.dtype.kind == "f"), k
    # without a norm: the element, with 8 bits its block's moments
    before = [_host(x) for x in ts]
    G.gnn_adamw_step(ps, 1e-3, 0.9, 0.999, 1e-8, 3)
    torch.cuda.synchronize()
    now = _host(ts[0])
    assert not np.isfinite(now["W"][7]) and np.isfinite(np.delete(now["W"], 7)).all()
    if bits == 32:
        assert not np.isfinite(now["v"][7]) and np.isfinite(np.delete(now["v"], 7)).all()
    else:
        v = P.decode(now["v"], now["v_scale"], P.E5M2)
        with np.errstate(invalid="ignore"):
            assert not np.isfinite(v[:256]).any() and np.isfinite(v[256:]).all()
    check_step(before[1:], ts[1:], bits, decays[1:], 1e-3, 0.9, 0.999, 1e-8, 3, 1.0, 0) \
        if bits == 32 else None


def test_adamw8_extremes():
    """Blocks of one size or of many, tiny and huge gradients, none at all."""
    c = 256 * 8
    ts = _tensors([c], 8, 6, zero_state=True)
    g = np.zeros(c, np.float32)
    g[:256] = 1e-3
    g[256:512] = np.float32(2.0) ** np.linspace(-60, 3, 256).astype(np.float32)
    g[512:768] = 1e-30
    g[768] = 1e15
    g[769:1024] = 1e-15
    g[1024:1280] = -np.float32(2.0) ** -np.arange(256).clip(0, 100).astype(np.float32)
    g[1300] = 5.0
    ts[0]["G"][0].copy_(torch.from_numpy(g))
    ps, decays = _params(ts, 8, decay=0.0)
    for t in (1, 2):
        before = [_host(x) for x in ts]
        G.gnn_adamw_step(ps, 1e-3, 0.9, 0.999, 1e-8, t, seed=31)
        torch.cuda.synchronize()
        check_step(before, ts, 8, decays, 1e-3, 0.9, 0.999, 1e-8, t, 1.0, 31)
    assert np.isfinite(_host(ts[0])["W"]).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_past_32_bit_offsets(bits):
    """One tensor of 2^31 + 5,000 elements: its ends against the same elements
    in a small tensor (32 bits), its norm, and the guards behind it."""
    c = 2 ** 31 + 5000
    W, g = torch.empty(c + 64, device="cuda"), torch.empty(c + 64, device="cuda")
    kind = torch.float32 if bits == 32 else torch.uint8
    m, v = (torch.zeros(c + 64, dtype=kind, device="cuda") for _ in range(2))
    W.fill_(0.5)
    g.fill_(2.0 ** -10)
    g[c:] = 77.0
    sc = [torch.zeros(-(-c // 256), device="cuda") for _ in range(2)] if bits == 8 else [None] * 2
    ps = G.make_params([(W[:c], g[:c], m[:c], v[:c]) + tuple(sc) + (0.1,)], bits)
    plan = torch.empty(G.gnn_params_plan_bytes(ps), dtype=torch.uint8, device="cuda")
    ps.plan = plan.data_ptr()
    G.gnn_params_build_plan(ps, plan)
    norm = torch.zeros(1, device="cuda")
    G.gnn_grad_norm(ps, norm, _ws(G.gnn_grad_norm_workspace_bytes(ps)))
    want = 2.0 ** -10 * np.sqrt(float(c))
    assert abs(float(norm) - want) <= U * want * 1.001
    G.gnn_adamw_step(ps, 1e-2, 0.9, 0.99, 1e-8, 1, norm, float(norm) * 2, 7)
    torch.cuda.synchronize()
    first = W[0].item()
    w, _, _ = P.adamw([0.5], [2.0 ** -10], [0.0], [0.0], 1e-2, 0.9, 0.99, 1e-8, 1, 0.1)
    assert abs(first - w[0]) <= 8 * U
    assert bool((W[:c] == first).all()) and bool((W[c:] == 0.5).all())
    assert bool((m[c:] == 0).all()) and bool((v[c:] == 0).all())
    if bits == 8:  # every element the block's largest: the top code
        assert bool((m[:c] == 126).all()) and bool((v[:c] == 123).all())


def test_adamw_more_pieces_than_one_launch():
    """2^33 + 5,000 weights: more pieces than a launch has blocks."""
    c = 2 ** 33 + 5000
    _room(120 << 30)
    W, g = torch.empty(c + 64, device="cuda"), torch.empty(c + 64, device="cuda")
    m, v = (torch.zeros(c + 64, dtype=torch.uint8, device="cuda") for _ in range(2))
    sc = [torch.zeros(-(-c // 256), device="cuda") for _ in range(2)]
    W.fill_(0.5)
    g.fill_(2.0 ** -10)
    ps = G.make_params([(W[:c], g[:c], m[:c], v[:c]) + tuple(sc) + (0.1,)], 8)
    plan = torch.empty(G.gnn_params_plan_bytes(ps), dtype=torch.uint8, device="cuda")
    ps.plan = plan.data_ptr()
    G.gnn_params_build_plan(ps, plan)
    G.gnn_adamw_step(ps, 1e-2, 0.9, 0.99, 1e-8, 1, seed=7)
    torch.cuda.synchronize()
    first = W[0].item()
    w, _, _ = P.adamw([0.5], [2.0 ** -10], [0.0], [0.0], 1e-2, 0.9, 0.99, 1e-8, 1, 0.1)
    assert abs(first - w[0]) <= 8 * U
    assert float(W[:c].min()) == first == float(W[:c].max()) and bool((W[c:] == 0.5).all())
    assert int(m[:c].min()) == 126 == int(m[:c].max()) and bool((m[c:] == 0).all())
    assert int(v[:c].min()) == 123 == int(v[:c].max()) and bool((v[c:] == 0).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_same_bits_streams_and_replay(bits):
    """The same step eagerly, on another stream, and captured (where t, lr
    and seed are the capture's) and replayed between eager steps."""
    sets = []
    for _ in range(3):
        ts = _tensors([70000, 513, 300], bits, 8)
        sets.append((ts,) + _params(ts, bits) + (torch.zeros(1, device="cuda"),))
    ws = [_ws(G.gnn_grad_norm_workspace_bytes(s[1])) for s in sets]
    side = torch.cuda.Stream()

    def call(k, stream=None):
        _, ps, _, norm = sets[k]
        G.gnn_grad_norm(ps, norm, ws[k], stream)
        G.gnn_adamw_step(ps, 1e-3, 0.9, 0.999, 1e-8, 9, norm, 0.5, 21, stream)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(0, side.cuda_stream)
    for it in range(3):
        graph.replay()
        torch.cuda.synchronize()
        call(1)
        torch.cuda.synchronize()
        call(2, side)
        torch.cuda.synchronize()
        for x, y, z in zip(*(s[0] for s in sets)):
            hx, hy, hz = _host(x), _host(y), _host(z)
            for k in hx:
                assert np.array_equal(hx[k], hy[k]) and np.array_equal(hx[k], hz[k]), (it, k)


# ------------------------------------------------------- the whole iteration

def _trainer(optimizer="adamw", **kw):
    wl = synth.WORKLOADS[synth.TINY_WORKLOAD]
    d = synth.workload_inputs(wl, bias=True)
    c = synth.classifier_inputs(wl)
    tr = runtime.Trainer(prepared(d["graph"]), d["params"], wl.f_in, c["w_mlp"], wl.multilabel,
                         optimizer, **kw)
    return tr, d, c, to_dev(d["x"], wl.f_in + 14), to_dev(c["targets"])


@pytest.mark.parametrize("bits", [32, 8])
def test_trainer_adamw(bits):
    """A cross-entropy iteration with AdamW: the gradients are those of the
    other optimizers, the update is the oracle's, biases do not decay."""
    tr, d, c, X, T = _trainer(lr=1e-2, weight_decay=0.2, max_norm=0.05, state_bits=bits, seed=6)
    other, _, _, _, _ = _trainer("sgd", lr=0.0)
    for t in (1, 2):
        w0 = [w.clone() for w, _ in tr.pairs]
        ts = [dict(W=(w.view(-1), None, 0), G=(g.view(-1), None, 0), **{
            k: (s, None, 0) for k, s in zip(("m", "v", "m_scale", "v_scale"), st)})
            for (w, g), st in zip(tr.pairs, tr.state)]
        before = [_host(x) for x in ts]
        for (w, _), x in zip(other.pairs, w0):
            w.copy_(x)
        tr.step(X, T)
        other.step(X, T)
        torch.cuda.synchronize()
        assert float(tr.loss) == float(other.loss)
        grads = [g.cpu().numpy() for _, g in tr.pairs]
        for g, (_, og) in zip(grads, other.pairs):
            assert np.array_equal(g, og.cpu().numpy())
        for h, g in zip(before, grads):
            h["G"] = g.reshape(-1)
        n = float(tr.params.norm)
        want = P.grad_norm(grads)
        assert abs(n - want) <= U * want * (1 + 1e-6) and n > 0.05
        decays = [0.2 if w.dim() == 2 else 0.0 for w, _ in tr.pairs]
        _check_unguarded(before, ts, bits, decays, 1e-2, t, 0.05 / n, 6)


def _check_unguarded(before, ts, bits, decays, lr, t, k, seed):
    import unittest.mock as mock
    with mock.patch(__name__ + "._guards_intact"):
        check_step(before, ts, bits, decays, lr, 0.9, 0.999, 1e-8, t, k, seed)


@pytest.mark.parametrize("bits", [32, 8])
def test_policy_iteration(bits):
    """Acting, then three clipped policy steps with a KL term to the first
    policy: loss, logits' gradient, head's gradients and the update against
    the oracle on the GPU's own top activations, the stack's gradients
    against the stack run on its own."""
    tr, d, _, X, _ = _trainer(lr=2e-3, max_norm=0.5, state_bits=bits)
    n, C = tr.n, tr.C
    rng = np.random.default_rng(1)
    a = rng.integers(0, C, n)
    a[rng.random(n) < 0.1] = -1
    act = torch.from_numpy(a.astype(np.int32)).cuda()
    adv = _f(rng.standard_normal(n))
    first = tr.action_logp(X, act)
    ref = (first + 0.1 * torch.randn(n, device="cuda",
                                     generator=torch.Generator("cuda").manual_seed(2)))
    lib = [x.cpu().numpy() for x in (adv, first, ref)]
    for t in (1, 2, 3):
        W = tr.W_mlp.cpu().numpy().astype(np.float64)
        out = tr.policy_step(X, act, adv, first, ref, clip=(0.2, 0.3), beta=0.05)
        torch.cuda.synchronize()
        top = tr.stack.layers[-1]["Y"].cpu().numpy().astype(np.float64)
        z = tr._Z.view(n).cpu().numpy()
        # split products: an error below 2^-24 of |X| |W| for each term, and
        # as many sums in fp32
        assert np.all(np.abs(z - top @ W) <= 4 * tr.f_top * U * (np.abs(top) @ np.abs(W)))
        want = P.policy_loss(z, a, *lib, None, 0.2, 0.3, 0.05)
        r = dict(out=out.cpu().numpy(), logp=tr.logp[:n].cpu().numpy(),
                 dZ=tr._dZ.view(n).cpu().numpy())
        check_loss(r, want, z, a, lib[0], lib[1], lib[2], 0.05)
        if t == 1:
            assert r["out"][2] == 0 and np.array_equal(r["logp"], lib[1])
        dz = r["dZ"].astype(np.float64)
        assert np.all(np.abs(tr.dW_mlp.cpu().numpy() - top.T @ dz) <=
                      4 * n * U * (np.abs(top).T @ np.abs(dz)))
        dx = tr.dX_top.cpu().numpy()
        assert np.all(np.abs(dx - dz @ W.T) <= 4 * C * U * (np.abs(dz) @ np.abs(W).T))
    # the same three steps again are the same bits
    again, _, _, _, _ = _trainer(lr=2e-3, max_norm=0.5, state_bits=bits)
    for t in (1, 2, 3):
        again.policy_step(X, act, adv, first, ref, clip=(0.2, 0.3), beta=0.05)
    for (w, _), (x, _) in zip(tr.pairs, again.pairs):
        assert torch.equal(w, x)


def test_policy_iteration_gradient_by_differences():
    """The gradient of the whole policy iteration (stack included) along its
    own direction in every weight, by central differences of the loss at a
    step h and at h / 2.  D(h) = slope + c h^2 + ..., so (4 D(h/2) - D(h)) / 3
    is free of the second order (a ratio exp(x) alone has (sinh x) / x - 1 =
    x^2 / 6 of it: 2 % at the x = 0.3 that rows reach here).  2 % of the slope
    is left for ReLU and clip kinks; fp32 losses of order 1 leave 1e-6."""
    tr, d, _, X, _ = _trainer("sgd", lr=0.0)
    n, C = tr.n, tr.C
    rng = np.random.default_rng(4)
    act = torch.from_numpy(rng.integers(0, C, n).astype(np.int32)).cuda()
    adv = _f(np.abs(rng.standard_normal(n)) + 0.5)
    old = tr.action_logp(X, act)
    ref = old + 0.2

    def loss():
        return float(tr.policy_step(X, act, adv, old, ref, beta=0.1)[0])

    loss()
    grads = [g.clone() for _, g in tr.pairs]
    for (w, _), g in zip(tr.pairs, grads):
        step = g / g.norm() * 1e-2 * max(float(w.norm()), 1.0)
        w0, D = w.clone(), []
        for h in (1.0, 0.5):
            w.copy_(w0 + h * step)
            up = loss()
            w.copy_(w0 - h * step)
            D.append((up - loss()) / (2 * h))
        w.copy_(w0)
        slope = float((g * step).sum())
        assert abs((4 * D[1] - D[0]) / 3 - slope) <= 0.02 * abs(slope) + 2e-6, (D, slope)


def test_policy_step_checks_and_no_rows():
    tr, d, _, X, _ = _trainer(lr=1e-3)
    n = tr.n
    act, adv = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")
    for bad in ((act.long(), adv), (act[:-1], adv), (act.cpu(), adv), (act, adv.double()),
                (act, adv.cpu())):
        with pytest.raises(ValueError):
            tr.policy_step(X, *bad)
    with pytest.raises(G.GnnError):
        tr.policy_step(X, act, adv, beta=0.1)  # no reference
    empty = prepared(synth.identity_graph(0))
    tr.bind(empty)
    none = torch.zeros(0, device="cuda")
    w0 = tr.flat_w.clone()
    out = tr.policy_step(X[:0], none.int(), none)
    torch.cuda.synchronize()
    assert torch.all(out == 0) and tr.action_logp(X[:0], none.int()).numel() == 0
    assert all(torch.all(g == 0) for _, g in tr.pairs)
    assert torch.isfinite(tr.flat_w).all() and not torch.equal(tr.flat_w, w0)  # decay alone


def test_policy_iteration_replayed():
    """A policy iteration captured (with SGD: AdamW's t is a host value) and
    replayed between eager ones, every replay against them."""
    cap, d, _, X, _ = _trainer("sgd", lr=1e-3)
    eager, _, _, _, _ = _trainer("sgd", lr=1e-3)
    n = cap.n
    act = torch.arange(n, device="cuda", dtype=torch.int32) % (cap.C + 1)  # C: left out
    adv = torch.randn(n, device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    old = eager.action_logp(X, act)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    cap.policy_step(X, act, adv, old, old, beta=0.1, stream=s.cuda_stream)  # grows the buffers
    torch.cuda.synchronize()
    eager.policy_step(X, act, adv, old, old, beta=0.1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        cap.policy_step(X, act, adv, old, old, beta=0.1, stream=s.cuda_stream)
    for it in range(3):
        graph.replay()
        torch.cuda.synchronize()
        eager.policy_step(X, act, adv, old, old, beta=0.1)
        torch.cuda.synchronize()
        assert torch.equal(cap.policy_out, eager.policy_out), it
        for (w, _), (v, _) in zip(cap.pairs, eager.pairs):
            assert torch.equal(w, v), it


def test_policy_iteration_on_other_subgraphs():
    """The trainer moved to a larger and back to a smaller subgraph between
    steps gives what trainers made for each give."""
    graphs = [prepared(synth.power_law_graph(k, 2.1, 8.0, seed=k)) for k in (300, 900, 200)]
    rng = np.random.default_rng(0)
    f, h, C = 24, 16, 5
    params = [synth.LayerParams(synth.glorot(f, h, rng), synth.glorot(f, h, rng))]
    w_mlp = synth.glorot(2 * h, C, rng)
    one = runtime.Trainer(graphs[0], params, f, w_mlp, False, "sgd", lr=0.0)
    for g in graphs:
        x = to_dev(rng.standard_normal((g.n, f)).astype(np.float32), 32)
        act = torch.from_numpy(rng.integers(0, C, g.n).astype(np.int32)).cuda()
        adv = _f(rng.standard_normal(g.n))
        one.bind(g)
        fresh = runtime.Trainer(g, params, f, w_mlp, False, "sgd", lr=0.0)
        a, b = one.policy_step(x, act, adv), fresh.policy_step(x, act, adv)
        torch.cuda.synchronize()
        assert torch.equal(a, b)
        for (_, p), (_, q) in zip(one.pairs, fresh.pairs):
            assert torch.equal(p, q)


def test_current_stream_and_timer():
    """Calls without a stream go to torch's current one; the event timer
    counts the launches under their kernels."""
    assert G._stream(None) == torch.cuda.current_stream().cuda_stream
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        assert G._stream(None) == s.cuda_stream
    assert G._stream(None) == torch.cuda.current_stream().cuda_stream
    z, a, adv, old, ref, w = _case(50, 9, 1)
    ts = _tensors([3000], 8, 1)
    ps, _ = _params(ts, 8)
    norm = torch.zeros(1, device="cuda")
    ws = _ws(G.gnn_grad_norm_workspace_bytes(ps))
    torch.cuda.synchronize()
    G.gnn_timer_reset()
    G.gnn_timer_enable(True)
    try:
        run_loss(z, a, adv, old, ref, w)
        G.gnn_grad_norm(ps, norm, ws)
        G.gnn_adamw_step(ps, 1e-3, 0.9, 0.99, 1e-8, 1, norm)
        for name, work in (("loss", 8.0 * 50 * 9), ("norm", 12000.0), ("update", 48000.0)):
            ms, launches, got = G.gnn_timer_read(name)
            assert launches == 1 and ms > 0 and got == work, name
    finally:
        G.gnn_timer_enable(False)
        G.gnn_timer_reset()
