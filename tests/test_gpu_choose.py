"""Drawn actions, top logits and the student's loss with its gradient on the
GPU against the oracle's doubles (through the C ABI).

Tolerances, with u = 2^-24 (half a step of fp32), x_j = (top - z_j) / T:
  action  a weight is off by 1e-13 of itself (the series left out, roundings
          in double) and by half a unit: at most 2^-52 of the largest, or
          2^(ceil(log2 C) - 63).  A draw whose distance to the nearest border,
          relative to the sum, is more than C units and 2e-13 must agree.
  logp    (20 + ln C) u, as for the policy loss's log-probabilities.
  sums    the arguments of the exponentials take three roundings (difference,
          1 / T, product) of relative u, expf 4 u, at most four are added in
          fp32, and the logarithm is good to 1.7 u; the weighted mean of x_j is
          at most ln C: E = (3 ln C + 12) u relative in a row's sum.
  rest    the same sum over the entries left out, over the whole sum.
  kl      T^2 (E + E of the others' sum), one rounding.
  dZ      an exponential (3 x_j + 4) u, the sums E each, four roundings.
"""
import numpy as np
import pytest
import torch

from oracle import choose as O
from paper_2010_03166_amd import gnnprop as G
from paper_2010_03166_amd import runtime, synth

from gpu_helpers import prepared, to_dev

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SENTINEL = 12345.0
WIDTHS = [1, 2, 3, 4, 5, 7, 8, 9, 12, 13, 16, 17, 31, 32, 33, 41, 63, 64, 65, 121, 127, 128, 129,
          255, 256, 257, 511, 513, 769, 1023, 1025, 1537, 2047, 2048, 2049, 4097, 8193, 16385,
          24577, 32768, 32769, 40001]


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


def _logits(n, C, seed, mask=0.0, skip=0.0, steps=0):
    rng = np.random.default_rng([n, C, seed])
    z = (rng.standard_normal((n, C)) * 2.5).astype(np.float32)
    if steps:  # few different values: many equal ones
        z = np.round(z * steps) / steps
    if mask:
        z[rng.random((n, C)) < mask] = -np.inf
        z[np.arange(n), rng.integers(0, C, n)] = 0.5
    if skip:
        z[rng.random(n) < skip] = np.nan
    return z.astype(np.float32), rng


def run_sample(z, u, T=1.0, top_k=0, top_p=1.0, min_p=0.0, pad=0, shift=0, want_logp=True,
               stream=None):
    n, C = z.shape
    abuf = torch.full((n + 8,), 77, dtype=torch.int32, device="cuda")
    lbuf = torch.full((n + 8,), SENTINEL, device="cuda")
    G.gnn_sample_actions(n, C, _rows(z, C + pad, shift), C + pad, _f(u), T, top_k, top_p, min_p,
                         abuf, lbuf if want_logp else None,
                         _ws(G.gnn_sample_workspace_bytes(n, C)), stream)
    torch.cuda.synchronize()
    assert torch.all(abuf[n:] == 77) and torch.all(lbuf[n if want_logp else 0:] == SENTINEL)
    return abuf[:n].cpu().numpy(), lbuf[:n].cpu().numpy()


def units(C):
    bits = min(51, 62 - int(np.ceil(np.log2(C)))) if C > 1 else 51
    return 2.0 ** -bits


def check_sample(z, u, T, top_k, top_p, min_p, got, logp=None):
    C = z.shape[1]
    want, lp, near = O.sample(z, u, T, top_k, top_p, min_p)
    clear = near > 2e-13 + C * units(C)
    assert np.mean(clear) > 0.99 or len(z) < 100
    assert np.array_equal(got[clear], want[clear])
    if logp is not None:
        assert np.all(np.abs(logp - lp)[clear] <= ((20 + np.log(C)) * U + U * np.abs(lp))[clear])
    return want, clear


SETTINGS = [(1.0, 0, 1.0, 0.0), (0.6, 0, 0.9, 0.0), (1.7, 5, 1.0, 0.0), (1.0, 40, 0.8, 0.05),
            (0.0, 3, 0.5, 0.1), (2.5, 0, 1.0, 0.02), (1.0, 1, 0.3, 0.0), (0.05, 0, 0.999, 0.0)]


@pytest.mark.parametrize("C", WIDTHS)
def test_sample_widths(C):
    n = 130 if C <= 2049 else 7
    for k, (T, top_k, top_p, min_p) in enumerate(SETTINGS):
        z, rng = _logits(n, C, k, mask=0.3 if k % 3 == 1 else 0.0, skip=0.1 if k % 2 else 0.0)
        u = rng.random(n).astype(np.float32)
        a, lp = run_sample(z, u, T, top_k, top_p, min_p, pad=k % 5, shift=k % 4)
        check_sample(z, u, T, top_k, top_p, min_p, a, lp)


@pytest.mark.parametrize("C", [3, 16, 20, 60, 121, 300, 700, 2000, 5000, 33000])
def test_sample_equal_logits(C):
    """Many equal logits: ties are cut by columns, and weights are equal."""
    n = 70 if C <= 2000 else 5
    for k, (T, top_k, top_p, min_p) in enumerate(SETTINGS):
        for steps in (1, 4):
            z, rng = _logits(n, C, 50 + k, mask=0.2 if k % 2 else 0.0, steps=steps)
            u = rng.random(n).astype(np.float32)
            a, _ = run_sample(z, u, T, top_k, top_p, min_p, want_logp=False)
            check_sample(z, u, T, top_k, top_p, min_p, a)
    # all alike: the action is floor(u m) of the m kept
    z = np.full((64, C), 1.25, np.float32)
    u = (np.arange(64) / 64).astype(np.float32)
    for top_k in (0, 1, 2, 3, min(C, 64)):
        m = top_k or C
        a, _ = run_sample(z, u, 0.7, top_k)
        assert np.array_equal(a, (np.arange(64) * m) // 64)
    for p in (0.25, 0.5, 0.75):
        m = int(np.ceil(p * C))
        a, _ = run_sample(z, u, 0.7, 0, p)
        assert np.array_equal(a, (np.arange(64) * m) // 64)


def test_sample_borders_of_u():
    z = np.zeros((9, 4), np.float32)
    u = np.array([0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24, 1.0, 7.0, -1.0, np.nan], np.float32)
    a, lp = run_sample(z, u)
    assert a.tolist() == [0, 1, 2, 3, 3, 3, 3, 0, 0]
    assert np.allclose(lp, -np.log(4), atol=2 * U * 2)


@pytest.mark.parametrize("C", [1, 5, 41, 121, 600, 3000, 33000])
def test_sample_rows_left_out(C):
    z, rng = _logits(40, C, 3)
    z[0] = np.nan
    z[1] = -np.inf
    z[2, C // 2] = np.nan
    z[3, C - 1] = np.inf
    z[4] = np.inf
    z[5] = np.finfo(np.float32).min       # the type's lowest value: allowed, and equal
    z[6] = np.where(np.arange(C) % 3 == 0, z[6], np.finfo(np.float32).min)
    z[7] = np.where(np.arange(C) % 2 == 0, 3e38, -3e38)
    z[8] = -np.inf
    z[8, C - 1] = -7.0
    z[9] = np.where(np.arange(C) % 2 == 0, 0.0, -0.0)
    u = rng.random(40).astype(np.float32)
    for T, top_k, top_p, min_p in SETTINGS:
        a, lp = run_sample(z, u, T, top_k, top_p, min_p, shift=1, pad=1)
        assert np.all(a[:5] == -1) and np.all(lp[:5] == 0) and a[8] == C - 1 and lp[8] == 0
        check_sample(z, u, T, top_k, top_p, min_p, a)


def test_sample_far_apart():
    """Temperatures at their limits, logits far apart."""
    z, rng = _logits(200, 50, 9)
    u = rng.random(200).astype(np.float32)
    for T in (1e-6, 1e-3, 1e3, 1e6):
        for top_p in (1.0, 0.5):
            a, _ = run_sample(z, u, T, 0, top_p)
            check_sample(z, u, T, 0, top_p, 0.0, a)
    z = (z * 1e30).astype(np.float32)
    a, _ = run_sample(z, u, 1.0, 7, 0.9, 0.1)
    assert np.array_equal(a, z.argmax(1))


def test_sample_follows_the_distribution():
    """200,000 draws from one row: each action as often as its share says, to
    five standard deviations."""
    z, _ = _logits(1, 41, 11)
    n = 200000
    Z = torch.from_numpy(z).cuda().expand(n, 41).contiguous()
    u = torch.rand(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    a = torch.empty(n, dtype=torch.int32, device="cuda")
    G.gnn_sample_actions(n, 41, Z, 41, u, 1.0, 10, 0.95, 0.0, a, None, _ws(0))
    kept, _ = O.kept_columns(z[0], 1.0, 10, 0.95)
    p = np.zeros(41)
    p[kept] = np.exp(z[0][kept].astype(np.float64))
    p /= p.sum()
    f = torch.bincount(a.long(), minlength=41).cpu().numpy() / n
    assert np.all(f[p == 0] == 0)
    assert np.all(np.abs(f - p) <= 5 * np.sqrt(p * (1 - p) / n))


# ------------------------------------------------------------- top logits

def run_top(z, k, T=1.0, pad=0, shift=0, want_rest=True, stream=None):
    n, C = z.shape
    ibuf = torch.full((n * k + 8,), 77, dtype=torch.int32, device="cuda")
    qbuf = torch.full((n * k + 8,), SENTINEL, device="cuda")
    rbuf = torch.full((n + 8,), SENTINEL, device="cuda")
    G.gnn_top_logits(n, C, _rows(z, C + pad, shift), C + pad, k, T, ibuf, qbuf,
                     rbuf if want_rest else None, _ws(G.gnn_top_workspace_bytes(n, C, k)), stream)
    torch.cuda.synchronize()
    assert torch.all(ibuf[n * k:] == 77) and torch.all(qbuf[n * k:] == SENTINEL)
    assert torch.all(rbuf[n if want_rest else 0:] == SENTINEL)
    return (ibuf[:n * k].view(n, k).cpu().numpy(), qbuf[:n * k].view(n, k).cpu().numpy(),
            rbuf[:n].cpu().numpy())


def check_top(z, k, T, got):
    n, C = z.shape
    index, logq, rest = got
    wi, wq, wr = O.top_logits(z, k, T)
    assert np.array_equal(index, wi)
    there = wi >= 0
    assert np.all(logq[~there] == -np.inf)
    E = (3 * np.log(C) + 12) * U
    assert np.all(np.abs(logq - wq)[there] <= (E + U * np.abs(wq))[there])
    for i in range(n):
        if wr[i] == 0:
            assert rest[i] <= 1e-37
            continue
        zi = z[i].astype(np.float64)
        x = (zi.max() - zi) / T
        out = np.ones(C, bool)
        out[wi[i][there[i]]] = False
        out &= zi > -np.inf
        p = np.exp(-x[out]) / np.exp(-x[np.isfinite(x)]).sum()
        tol = np.sum(p * (3 * x[out] + 8)) * U + wr[i] * (E + U) + C * 1e-38
        assert abs(rest[i] - wr[i]) <= tol


@pytest.mark.parametrize("C", WIDTHS)
def test_top_widths(C):
    n = 130 if C <= 2049 else 7
    for i, k in enumerate([1, 2, 5, 16, 63, 64, 128, 256]):
        if k > 4 * C + 8:
            continue
        z, _ = _logits(n, C, i, mask=0.4 if i % 3 == 1 else 0.0, skip=0.1 if i % 2 else 0.0)
        T = [1.0, 2.0, 0.5][i % 3]
        check_top(z, k, T, run_top(z, k, T, pad=i % 3, shift=i % 4))


@pytest.mark.parametrize("C", [3, 16, 20, 60, 121, 300, 700, 2000, 5000, 33000])
def test_top_equal_logits(C):
    n = 40 if C <= 2000 else 5
    for steps in (0.2, 1, 4):
        z, _ = _logits(n, C, 70, steps=steps)
        for k in (1, 7, 100, 256):
            check_top(z, k, 1.5, run_top(z, k, 1.5, want_rest=True))
    z = np.full((3, C), -2.0, np.float32)
    index, logq, rest = run_top(z, 8, 3.0, want_rest=False)
    m = min(8, C)
    assert np.array_equal(index[:, :m], np.tile(np.arange(m), (3, 1))) and np.all(index[:, m:] == -1)


@pytest.mark.parametrize("C", [1, 5, 41, 121, 600, 3000, 33000])
def test_top_rows_left_out(C):
    z, _ = _logits(12, C, 3)
    z[0] = np.nan
    z[1] = -np.inf
    z[2, C // 2] = np.nan
    z[3, C - 1] = np.inf
    z[4] = np.finfo(np.float32).min
    z[5] = np.where(np.arange(C) % 3 == 0, z[5], np.finfo(np.float32).min)
    z[6] = -np.inf
    z[6, C - 1] = -7.0
    for k in (1, 4, 200):
        got = run_top(z, k, 1.0, pad=1)
        assert np.all(got[0][:4] == -1) and np.all(got[2][:4] == 0)
        assert got[0][6, 0] == C - 1 and got[1][6, 0] == 0
        check_top(z, k, 1.0, got)


# ---------------------------------------------------------------- student

def run_distill(z, index, logq, rest, w, T=1.0, pad=0, shift=0, want_kl=True, want_dz=True,
                stream=None):
    n, C = z.shape
    k, ld = index.shape[1], C + pad
    dbuf = torch.full((n * ld + 16,), SENTINEL, device="cuda")
    dZ = dbuf[shift: shift + n * ld].view(n, ld)
    kbuf = torch.full((n + 8,), SENTINEL, device="cuda")
    out = torch.full((8,), SENTINEL, device="cuda")
    G.gnn_distill_loss(n, C, _rows(z, ld, shift), ld, k,
                       torch.from_numpy(np.ascontiguousarray(index, np.int32)).cuda(), _f(logq),
                       _f(rest), _f(w), T, out, kbuf if want_kl else None,
                       dZ if want_dz else None, ld,
                       _ws(G.gnn_distill_workspace_bytes(n, C, k)), stream)
    torch.cuda.synchronize()
    assert torch.all(out[1:] == SENTINEL) and torch.all(kbuf[n if want_kl else 0:] == SENTINEL)
    assert torch.all(dbuf[:shift] == SENTINEL) and torch.all(dbuf[shift + n * ld:] == SENTINEL)
    assert torch.all(dZ[:, C if want_dz else 0:] == SENTINEL)
    return dict(out=float(out[0]), kl=kbuf[:n].cpu().numpy(),
                dZ=dZ[:, :C].cpu().numpy().copy())


def _taught(n, C, k, seed, T, mask=0.0, skip=0.0, rest=True, lists=0.0):
    """A student's logits and a teacher's list of them and something more.
    lists: share of places not used, and of indices there twice."""
    z, rng = _logits(n, C, seed, mask=mask)
    t = z + rng.standard_normal((n, C)).astype(np.float32)
    index, logq, left = O.top_logits(t, k, T)
    if lists:
        far = rng.choice([-1, C, 2 ** 31 - 1, -2 ** 31], index.shape)
        index = np.where(rng.random(index.shape) < lists, far, index)
        twice = rng.random(index.shape) < lists
        index = np.where(twice, index[np.arange(n)[:, None], rng.integers(0, k, index.shape)], index)
        logq = np.where(np.isfinite(logq), logq, -3.0)
    if skip:
        out = rng.random(n) < skip
        index[out] = rng.choice([-1, C])
        z[out] = np.nan
    w = (rng.random(n) / n).astype(np.float32)
    w[rng.random(n) < 0.1] = 0.0
    return (z, index, logq.astype(np.float32), left.astype(np.float32) if rest else None, w)


def check_distill(r, z, index, logq, rest, w, T, kl=True, dz=True):
    n, C = z.shape
    want = O.distill(z, index, logq, rest, w, T)
    E = (3 * np.log(C) + 12) * U
    tol = T * T * 2 * E + 2 * U * np.abs(want["kl"])
    fine = np.isfinite(want["kl"])
    if kl:
        assert np.array_equal(r["kl"][~fine], want["kl"][~fine].astype(np.float32))
        assert np.all(np.abs(r["kl"] - want["kl"])[fine] <= tol[fine])
        assert np.all(r["kl"][~want["live"]] == 0)
    ww = np.full(n, 1.0 / n) if w is None else w.astype(np.float64)
    if np.all(fine | (ww == 0)):
        # (in one row's difference twice: the formula's is summed without them)
        assert abs(r["out"] - want["out"]) <= np.sum(ww * np.where(fine, tol, 0)) + \
            2 * U * abs(want["out"])
    if not dz:
        return want
    with np.errstate(all="ignore"):
        zz = z.astype(np.float64)
        x = np.where(np.isfinite(zz), (np.nanmax(zz, 1, keepdims=True) - zz) / T, 0.0)
        p = np.where(np.isfinite(zz), np.exp(-x), 0.0)
        p = np.where(want["live"][:, None], p / p.sum(1, keepdims=True), 0.0)
    g = np.zeros((n, C))
    for i in range(n):
        if not want["live"][i] or ww[i] == 0:
            continue
        other = np.ones(C, bool)
        other[[c for c in index[i] if 0 <= c < C]] = False
        p0 = p[i][other].sum()
        q0 = 0.0 if rest is None else float(rest[i])
        scale = p[i] * (1 + (q0 / p0 if p0 > 0 else 0.0) * other)
        g[i] = ww[i] * T * (scale * ((3 * x[i] + 8) * U + 2 * E)) + 1e-37
    assert np.all(np.abs(r["dZ"] - want["dZ"]) <= g + 2 * U * np.abs(want["dZ"]))
    assert np.all(r["dZ"][~want["live"]] == 0) and np.all(r["dZ"][ww == 0] == 0)
    return want


@pytest.mark.parametrize("C", WIDTHS)
def test_distill_widths(C):
    n = 130 if C <= 2049 else 6
    for i, k in enumerate([1, 2, 4, 16, 64, 100, 256]):
        if k > 4 * C + 8:
            continue
        T = [1.0, 2.0, 0.5][i % 3]
        case = _taught(n, C, k, i, T, mask=0.3 if i % 3 == 1 else 0.0, skip=0.1 if i % 2 else 0.0,
                       rest=i % 2 == 0, lists=0.2 if i % 4 == 3 else 0.0)
        r = run_distill(*case, T, pad=i % 3, shift=i % 4)
        check_distill(r, *case, T)


def test_distill_options():
    case = _taught(60, 100, 8, 5, 1.5)
    full = run_distill(*case, 1.5)
    assert run_distill(*case, 1.5, want_kl=False, want_dz=False)["out"] == full["out"]
    z, index, logq, rest, _ = case
    check_distill(run_distill(z, index, logq, rest, None, 1.5), z, index, logq, rest, None, 1.5)
    # without a rest the teacher's logits may be shifted
    a = run_distill(z, index, logq + 5, None, None, 1.5)
    check_distill(a, z, index, logq + np.float32(5), None, None, 1.5)


@pytest.mark.parametrize("C", [2, 7, 41, 121, 600, 3000, 33000])
def test_distill_edges(C):
    k = min(C - 1, 5) if C < 33000 else 5
    z, index, logq, rest, w = _taught(12, C, k, 8, 1.0)
    w[:] = 1.0 / 12
    z[0, index[0, 0]] = -np.inf              # the teacher's best is not allowed
    z[1] = -np.inf                           # left out
    z[2] = np.finfo(np.float32).min
    logq[3] = -np.inf
    rest[3] = 0.0                            # nothing that the teacher says
    other = np.setdiff1d(np.arange(C), index[4])
    z[4, other] = -300.0                     # the others' share below fp32
    z[5, other] = -np.inf                    # and none at all
    z[6] = np.nan
    index[6] = -1
    z[7, index[7]] = -400.0                  # the teacher's choices far down
    rest[8] = 0.0
    rest[9] = 1e-30
    logq[10, 0] = 0.0
    r = run_distill(z, index, logq, rest, w, 1.0)
    want = check_distill(r, z, index, logq, rest, w, 1.0)
    assert r["kl"][0] == np.inf and want["kl"][0] == np.inf
    assert np.all(r["kl"][[1, 3, 6]] == 0) and np.all(r["dZ"][[1, 3, 6]] == 0)
    assert np.isfinite(r["kl"][4]) and r["out"] == np.inf
    assert np.all(np.isfinite(r["dZ"]))
    z, index, logq, rest, w = _taught(4, C, k, 9, 1.0)
    z[0, 0] = np.nan                         # shows
    logq[1, 0] = np.nan
    w[:] = 0.25
    w[3] = 0.0
    z[3] = np.nan
    r = run_distill(z, index, logq, rest, w, 1.0)
    assert np.isnan(r["out"]) and np.isnan(r["kl"][0]) and np.isnan(r["kl"][1])
    assert np.isnan(r["dZ"][0]).any() and np.isnan(r["dZ"][1]).any()
    assert np.all(r["dZ"][3] == 0)


def test_distill_gradient_by_differences():
    """Central differences of the loss itself (in the oracle's doubles)."""
    T = 1.3
    z, index, logq, rest, w = _taught(6, 23, 4, 2, T)
    w[:] = 1.0 / 6
    r = run_distill(z, index, logq, rest, w, T)
    h = 1e-5
    for i in range(6):
        for j in range(23):
            up, down = z.astype(np.float64), z.astype(np.float64)
            up[i, j] += h
            down[i, j] -= h
            d = (O.distill(up, index, logq, rest, w, T)["out"] -
                 O.distill(down, index, logq, rest, w, T)["out"]) / (2 * h)
            assert abs(r["dZ"][i, j] - d) <= 1e-6


def test_no_rows():
    z = torch.zeros((0, 5), device="cuda")
    out = torch.full((1,), SENTINEL, device="cuda")
    G.gnn_sample_actions(0, 5, z, 5, None, 1.0, 0, 1.0, 0.0, None, None, _ws(0))
    G.gnn_top_logits(0, 5, z, 5, 2, 1.0, None, None, None, _ws(0))
    G.gnn_distill_loss(0, 5, z, 5, 2, None, None, None, None, 1.0, out, None, None, 5,
                       _ws(G.gnn_distill_workspace_bytes(0, 5, 2)))
    assert float(out) == 0.0


def test_many_blocks():
    """Many rows of a lane each against torch's own sums, and the same results in
    every call."""
    n, C = 300001, 3
    gen = torch.Generator(device="cuda").manual_seed(1)
    Z = torch.randn((n, C), device="cuda", generator=gen)
    u = torch.rand(n, device="cuda", generator=gen)
    a = [torch.empty(n, dtype=torch.int32, device="cuda") for _ in range(2)]
    for x in a:
        G.gnn_sample_actions(n, C, Z, C, u, 1.0, 0, 1.0, 0.0, x, None, _ws(0))
    assert torch.equal(a[0], a[1])
    cum = torch.cumsum(torch.softmax(Z.double(), 1), 1)
    cum[:, -1] = 2.0
    want = (cum <= u.double()[:, None]).sum(1)
    near = ((cum - u.double()[:, None]).abs() < 1e-12).any(1)
    assert int(near.sum()) < 10 and torch.equal(a[0].long()[~near], want[~near])


# ----------------------------------------- the Trainer, streams and graphs

def _trainer(optimizer="sgd", seed=0, **kw):
    wl = synth.WORKLOADS[synth.TINY_WORKLOAD]
    d = synth.workload_inputs(wl, bias=True)
    c = synth.classifier_inputs(wl)
    w_mlp = c["w_mlp"] + 0.3 * np.random.default_rng(seed).standard_normal(c["w_mlp"].shape)
    tr = runtime.Trainer(prepared(d["graph"]), d["params"], wl.f_in, w_mlp.astype(np.float32),
                         wl.multilabel, optimizer, **kw)
    return tr, to_dev(d["x"], wl.f_in + 14)


def test_acting_and_a_policy_step():
    """Actions drawn by the Trainer are the oracle's on the Trainer's logits, and
    with their log-probabilities as old_logp nothing is clipped."""
    tr, X = _trainer(lr=1e-3)
    n, C = tr.n, tr.C
    u = torch.rand(n, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    for T, top_k, top_p, min_p in ((1.0, 0, 1.0, 0.0), (0.8, 3, 0.9, 0.01)):
        a, lp = tr.act(X, u, T, top_k, top_p, min_p)
        Z = tr._Z.view(n).cpu().numpy()
        check_sample(Z, u.cpu().numpy(), T, top_k, top_p, min_p, a.cpu().numpy(), lp.cpu().numpy())
        assert torch.allclose(lp, tr.action_logp(X, a), rtol=0, atol=(40 + 2 * np.log(C)) * U)
    out = tr.policy_step(X, a, torch.ones(n, device="cuda"), lp)
    assert float(out[2]) == 0.0 and torch.isfinite(out).all()


@pytest.mark.parametrize("T,rest", [(1.0, True), (2.0, True), (2.0, False)])
def test_teaching(T, rest):
    """A teacher's top logits, a student's iteration with them: loss and the
    head's gradient against the oracle, the stack's against the stack's own
    backward pass."""
    teacher, X = _trainer(seed=1)
    tr, _ = _trainer(seed=2, lr=0.0)
    n, C, k = tr.n, tr.C, min(4, tr.C)
    index, logq, left = teacher.top_logits(X, k, T)
    check_top(teacher._Z.view(n).cpu().numpy(), k, T,
              (index.cpu().numpy(), logq.cpu().numpy(), left.cpu().numpy()))
    loss = tr.distill_step(X, index, logq, left if rest else None, temperature=T)
    torch.cuda.synchronize()
    Z = tr._Z.view(n).cpu().numpy()
    args = (Z, index.cpu().numpy(), logq.cpu().numpy(), left.cpu().numpy() if rest else None, None, T)
    r = dict(out=float(loss), dZ=tr._dZ.view(n).cpu().numpy())
    check_distill(r, *args, kl=False)
    top = tr.stack.forward(X).cpu().numpy().astype(np.float64)
    want = top.T @ r["dZ"].astype(np.float64)
    assert np.abs(tr.dW_mlp.cpu().numpy() - want).max() <= 1e-5 * np.abs(want).max()
    grads = [g.clone() for _, g in tr.pairs]
    tr.stack.forward(X)
    tr.stack.backward(tr.dX_top, want_dx_first=False)
    for g, (_, again) in zip(grads, tr.pairs):
        assert torch.equal(g, again)


def test_teaching_lowers_the_loss_along_its_gradient():
    """The loss after a small step is the loss less lr |gradient|^2, to second
    order: what the whole iteration's gradient says."""
    teacher, X = _trainer(seed=1)
    index, logq, left = teacher.top_logits(X, 3)
    losses = []
    tr, _ = _trainer(seed=2, lr=1e-3)
    for _ in range(2):
        losses.append(float(tr.distill_step(X, index, logq, left)))
        if len(losses) == 1:
            g2 = sum(float((g.double() ** 2).sum()) for _, g in tr.pairs)
    assert abs((losses[0] - losses[1]) / (1e-3 * g2) - 1) < 0.05


def test_trainer_refuses_lists_that_do_not_fit():
    tr, X = _trainer()
    n = tr.n
    i, q = torch.zeros((n, 3), dtype=torch.int32, device="cuda"), torch.zeros((n, 3), device="cuda")
    for bad in ((i.long(), q), (i, q.double()), (i[1:], q), (i, q[:, :2]), (i[0], q[0]),
                (i.t().contiguous().t(), q), (i.cpu(), q)):
        with pytest.raises(ValueError):
            tr.distill_step(X, *bad)
    with pytest.raises(ValueError):
        tr.distill_step(X, i, q, torch.zeros(n + 1, device="cuda"))
    with pytest.raises(ValueError):
        tr.act(X, torch.zeros(n - 1, device="cuda"))
    with pytest.raises(G.GnnError):
        tr.act(X, torch.zeros(n, device="cuda"), top_p=0.0)
    with pytest.raises(G.GnnError):
        tr.top_logits(X, 300)


def test_trainer_captured_and_replayed():
    """Acting, a policy step, teaching: captured on another stream, replayed
    between eager iterations of a second trainer, everything equal."""
    teacher, X = _trainer(seed=1)
    cap, _ = _trainer(seed=2, lr=1e-3)
    eager, _ = _trainer(seed=2, lr=1e-3)
    n = cap.n
    gen = torch.Generator("cuda").manual_seed(3)
    u, adv = torch.rand(n, device="cuda", generator=gen), torch.randn(n, device="cuda", generator=gen)
    cap.act(X, u)
    teacher.top_logits(X, 3)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()

    def once(tr, stream):
        a, lp = tr.act(X, u, 0.9, 4, 0.95, 0.01, stream=stream)
        out = tr.policy_step(X, a, adv, lp, stream=stream).clone()
        i, q, r = teacher.top_logits(X, 3, 2.0, stream=stream)
        return a, lp, out, i, q, r, tr.distill_step(X, i, q, r, temperature=2.0, stream=stream)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = once(cap, s.cuda_stream)
    for it in range(4):
        u.copy_(torch.rand(n, device="cuda", generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        want = once(eager, None)
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y), it
        for (w, _), (v, _) in zip(cap.pairs, eager.pairs):
            assert torch.equal(w, v), it


@pytest.mark.parametrize("n,C", [(300, 7), (100, 121), (20, 2048), (6, 5000), (4, 20011), (3, 70001)])
def test_calls_at_once_and_replayed(n, C):
    """The same calls on the default stream, on two others at once and from a
    graph: the same bits."""
    z, rng = _logits(n, C, 4, mask=0.2, skip=0.1)
    k = min(9, C)
    Z, u = _rows(z, C, 0), _f(rng.random(n))
    i0, q0, r0 = (_f(x) for x in O.top_logits(z + rng.standard_normal(z.shape).astype(np.float32),
                                              k, 1.0))
    i0 = i0.int()

    def calls(stream=None):
        a = torch.empty(n, dtype=torch.int32, device="cuda")
        i, q = torch.empty((n, k), dtype=torch.int32, device="cuda"), torch.empty((n, k), device="cuda")
        lp, r, kl, out = (torch.empty(m, device="cuda") for m in (n, n, n, 1))
        dZ = torch.empty((n, C), device="cuda")
        w = [_ws(G.gnn_sample_workspace_bytes(n, C)), _ws(G.gnn_top_workspace_bytes(n, C, k)),
             _ws(G.gnn_distill_workspace_bytes(n, C, k))]
        def run(stream=None):
            G.gnn_sample_actions(n, C, Z, C, u, 0.9, 50, 0.9, 0.01, a, lp, w[0], stream)
            G.gnn_top_logits(n, C, Z, C, k, 2.0, i, q, r, w[1], stream)
            G.gnn_distill_loss(n, C, Z, C, k, i0, q0, r0, None, 2.0, out, kl, dZ, C, w[2], stream)
        return run, (a, lp, i, q, r, kl, out, dZ)

    run, want = calls()
    run()
    streams = [torch.cuda.Stream() for _ in range(2)]
    both = [calls() for _ in streams]
    torch.cuda.synchronize()
    for _ in range(5):
        for (go, _), s in zip(both, streams):
            go(s.cuda_stream)
    torch.cuda.synchronize()
    graph_run, graph_out = calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        graph_run(streams[0].cuda_stream)
    for _ in range(3):
        for x in graph_out:
            x.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        for outs in (both[0][1], both[1][1], graph_out):
            for x, y in zip(outs, want):
                assert torch.equal(torch.nan_to_num(x.float(), 3.0), torch.nan_to_num(y.float(), 3.0))


def test_timer_counts_the_calls():
    z, _ = _logits(10, 20, 1)
    G.gnn_timer_enable()
    G.gnn_timer_reset()
    try:
        run_sample(z, np.zeros(10))
        run_top(z, 3)
        ms, launches, work = G.gnn_timer_read("sample")
    finally:
        G.gnn_timer_enable(False)
    assert launches == 2 and ms > 0


def test_temperature_0_needs_no_random_numbers():
    z, _ = _logits(50, 300, 6)
    a = torch.full((50,), 7, dtype=torch.int32, device="cuda")
    G.gnn_sample_actions(50, 300, _rows(z, 300, 0), 300, None, 0.0, 0, 1.0, 0.0, a, None, _ws(0))
    assert np.array_equal(a.cpu().numpy(), z.argmax(1))


def test_more_blocks_than_a_launch_has():
    """2^29 and some rows of one column: 256 to a block, 2^21 blocks to a
    launch."""
    n = (1 << 29) + 300
    Z = torch.zeros((n, 1), device="cuda")
    Z[n - 1] = float("nan")
    a = torch.full((n,), 7, dtype=torch.int32, device="cuda")
    u = torch.zeros(n, device="cuda")
    G.gnn_sample_actions(n, 1, Z, 1, u, 1.0, 0, 0.5, 0.0, a, None, _ws(0))
    assert int((a[:-1] != 0).sum()) == 0 and int(a[-1]) == -1
    q = u.fill_(3.0)
    G.gnn_top_logits(n, 1, Z, 1, 1, 1.0, a, q, None, _ws(0))
    assert int((a[:-1] != 0).sum()) == 0 and int(a[-1]) == -1
    assert int((q[:-1] != 0).sum()) == 0 and float(q[-1]) == -np.inf
    del q, u
    a.zero_()
    a[5] = -1
    logq, dZ, out = torch.zeros((n, 1), device="cuda"), torch.ones((n, 1), device="cuda"), \
        torch.ones(1, device="cuda")
    Z[n - 1] = 2.0
    G.gnn_distill_loss(n, 1, Z, 1, 1, a, logq, None, None, 1.0, out, None, dZ, 1,
                       _ws(G.gnn_distill_workspace_bytes(n, 1, 1)))
    assert int((dZ != 0).sum()) == 0 and float(out) == 0.0


@pytest.mark.parametrize("n,C", [(80000, 30011), (40000, 60013)])
def test_offsets_past_32_bits(n, C):
    """2.4e9 logits: the last rows as in a call of their own."""
    gen = torch.Generator("cuda").manual_seed(8)
    Z = torch.randn((n, C), device="cuda", generator=gen)
    u = torch.rand(n, device="cuda", generator=gen)
    k, m = 5, 3
    a, i = torch.empty(n, dtype=torch.int32, device="cuda"), \
        torch.empty((n, k), dtype=torch.int32, device="cuda")
    q, r, lp = torch.empty((n, k), device="cuda"), torch.empty(n, device="cuda"), \
        torch.empty(n, device="cuda")
    G.gnn_sample_actions(n, C, Z, C, u, 0.8, 100, 0.9, 0.0, a, lp,
                         _ws(G.gnn_sample_workspace_bytes(n, C)))
    G.gnn_top_logits(n, C, Z, C, k, 1.0, i, q, r, _ws(G.gnn_top_workspace_bytes(n, C, k)))
    z = Z[-m:].cpu().numpy()
    check_sample(z, u[-m:].cpu().numpy(), 0.8, 100, 0.9, 0.0, a[-m:].cpu().numpy(),
                 lp[-m:].cpu().numpy())
    check_top(z, k, 1.0, (i[-m:].cpu().numpy(), q[-m:].cpu().numpy(), r[-m:].cpu().numpy()))
    i[:, 0] = (i[:, 0] + 1) % C  # something to learn
    dZ, out, kl = torch.empty((n, C), device="cuda"), torch.empty(1, device="cuda"), \
        torch.empty(n, device="cuda")
    G.gnn_distill_loss(n, C, Z, C, k, i, q, r, None, 1.0, out, kl, dZ, C,
                       _ws(G.gnn_distill_workspace_bytes(n, C, k)))
    w = np.full(m, 1.0 / n)
    got = dict(out=0.0, kl=kl[-m:].cpu().numpy(), dZ=dZ[-m:].cpu().numpy())
    want = O.distill(z, i[-m:].cpu().numpy(), q[-m:].cpu().numpy(), r[-m:].cpu().numpy(), w, 1.0)
    got["out"] = want["out"]
    check_distill(got, z, i[-m:].cpu().numpy(), q[-m:].cpu().numpy(), r[-m:].cpu().numpy(),
                  w.astype(np.float32), 1.0)


@pytest.mark.parametrize("C", [200000, 1 << 20])
def test_very_long_rows(C):
    z, rng = _logits(3, C, 12, mask=0.1)
    z[2] = np.round(z[2])  # many equal ones: a crowded bin
    u = rng.random(3).astype(np.float32)
    for T, top_k, top_p, min_p in ((1.0, 0, 0.9, 0.0), (0.7, 5000, 0.95, 0.001), (1.0, 0, 1.0, 0.01),
                                   (1.0, 70000, 1.0, 0.0), (0.0, 0, 1.0, 0.0)):
        a, lp = run_sample(z, u, T, top_k, top_p, min_p)
        check_sample(z, u, T, top_k, top_p, min_p, a, lp)
    check_top(z, 200, 1.0, run_top(z, 200, 1.0))
    zero = np.zeros((2, C), np.float32)
    a, _ = run_sample(zero, np.array([0.25, 0.75]), 1.0, 0, 0.5)
    half = int(np.ceil(0.5 * C))
    assert a.tolist() == [half // 4, 3 * half // 4]


@pytest.mark.parametrize("C", [33000, 70001])
def test_long_rows_first_entries(C):
    """As many first entries as a list holds and more, of rows spread out, of few
    levels and of one, of rows with fewer entries than are asked for."""
    n = 6
    for k, top_k in enumerate((2, 127, 128, 129, 1000, 1023, 1024, 1025, 2049, 5000)):
        for j, (steps, mask) in enumerate(((0, 0.0), (60, 0.4), (3, 0.0), (1, 0.5), (0, 0.99))):
            z, rng = _logits(n, C, 300 + k, mask=mask, skip=0.1, steps=steps)
            for T, top_p, min_p in ((1.0, 0.9, 0.0), ((0.7, 1.0, 0.0), (1.4, 0.6, 0.01))[(k + j) % 2]):
                u = rng.random(n).astype(np.float32)
                a, lp = run_sample(z, u, T, top_k, top_p, min_p, pad=k % 3, shift=k % 4)
                check_sample(z, u, T, top_k, top_p, min_p, a, lp)


def test_a_million_columns_first_entries():
    z, rng = _logits(2, 1 << 20, 400)
    z[1] = np.where(np.arange(1 << 20) >= (1 << 20) - 1500, z[1], -np.inf)  # next to each other
    for top_k, top_p in ((700, 0.95), (1024, 0.999), (60, 1.0)):
        u = rng.random(2).astype(np.float32)
        a, lp = run_sample(z, u, 0.9, top_k, top_p, 0.0)
        check_sample(z, u, 0.9, top_k, top_p, 0.0, a, lp)
