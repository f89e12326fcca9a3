"""Edges of the policy loss, the gradient norm and AdamW on the GPU: long rows
with whole chunks of masked actions, borders of the clip, factors and gradients
at the ends of fp32, other streams.  Tolerances as counted in
test_gpu_policy.py, or beside the test."""
import numpy as np
import pytest
import torch

from oracle import policy as P
from paper_2010_03166_amd import gnnprop as G
from paper_2010_03166_amd import runtime, synth

from gpu_helpers import prepared, to_dev
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


def _near(n, C, seed, share=1.0):
    """Rows whose ratios round to a border of clip = (0.2, 0.3)."""
    z, a, adv, old, ref, w = _case(n, C, seed)
    lp, _ = P.action_logp(z, a)
    rng = np.random.default_rng([seed, 8])
    side = np.where(rng.random(n) < 0.5, 0.8, 1.3)
    pick = rng.random(n) < share
    old = np.where(pick, lp - np.log(side), old).astype(np.float32)
    return z, a, adv, old, ref, w


def _ms(call):
    """Least time of five calls."""
    call()
    best = np.inf
    for _ in range(5):
        x, y = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        x.record()
        call()
        y.record()
        y.synchronize()
        best = min(best, x.elapsed_time(y))
    return best


def test_row_at_a_border_costs_no_multiple_of_itself():
    """One row of 2^22 logits with its ratio at the clip's border and away
    from it: the sums in doubles are formed once, not by each of the row's
    1,024 chunks (which took 200 times the call's time)."""
    C = 1 << 22
    g = torch.Generator(device="cuda").manual_seed(5)
    Z = torch.randn((1, C), device="cuda", generator=g)
    act = torch.full((1,), 77, dtype=torch.int32, device="cuda")
    lp = torch.log_softmax(Z.double(), 1)[:, 77]
    adv, w = torch.ones(1, device="cuda"), torch.ones(1, device="cuda")
    dZ, out, logp = torch.empty_like(Z), torch.empty(3, device="cuda"), torch.empty(1, device="cuda")
    ws = _ws(G.gnn_policy_workspace_bytes(1, C))
    ms = {}
    for name, ratio in (("away", 1.0), ("at", 1.3)):
        old = (lp - np.log(ratio)).float()
        ms[name] = _ms(lambda: G.gnn_policy_loss(1, C, Z, C, act, adv, old, old, w, 0.2, 0.3, 0.05,
                                                 out, logp, dZ, C, ws))
    print(ms)
    assert ms["at"] < 10 * ms["away"] + 0.1


@pytest.mark.parametrize("n,C", [(3, 40000), (70, 33000), (1, 131072), (600, 32770)])
@pytest.mark.parametrize("share", [1.0, 0.3])
def test_long_rows_at_a_border(n, C, share):
    """Rows at and away from a border of the clip in one call: decided as in
    doubles, with the gradients and sums of their side."""
    z, a, adv, old, ref, w = _near(n, C, 41, share)
    first = P.policy_loss(z, a, adv, old, ref, w, 0.2, 0.3, 0.05)
    with np.errstate(divide="ignore"):
        unsure = np.minimum(np.abs(first["rho"] - 0.8), np.abs(first["rho"] - 1.3)) < 1e-10
    keep = np.where(unsure, -1, a)
    assert unsure.mean() < 0.1 or n < 10
    want = P.policy_loss(z, keep, adv, old, ref, w, 0.2, 0.3, 0.05)
    r = run_loss(z, keep, adv, old, ref, w, beta=0.05, pad=C % 3, shift=1)
    check_loss(r, want, z, keep, adv, old, ref, 0.05)
    again = run_loss(z, keep, adv, old, ref, w, beta=0.05, pad=C % 3, shift=1)
    no_dz = run_loss(z, keep, adv, old, ref, w, beta=0.05, want_dz=False)
    for k in r:
        assert np.array_equal(r[k], again[k]), k
    check_loss(dict(r, out=no_dz["out"], logp=no_dz["logp"]), want, z, keep, adv, old, ref, 0.05)
    # without the KL term a cut row has no gradient at all
    r = run_loss(z, keep, adv, old, None, w)
    cut = np.all(r["dZ"] == 0, axis=1)
    assert np.array_equal(cut, want["cut"] | (keep < 0))


def test_many_long_rows_at_a_border():
    """More rows than one block adds up, a fifth of them at a border: the same
    bits as in two calls of fewer rows."""
    n, C, cut = 8300, 32769, 4100
    _room(8 << 30)
    g = torch.Generator(device="cuda").manual_seed(6)
    Z = torch.randn((n, C), device="cuda", generator=g)
    act = torch.randint(0, C, (n,), device="cuda", generator=g, dtype=torch.int32)
    adv, w = (torch.randn(n, device="cuda", generator=g) for _ in range(2))
    w.abs_().div_(n)
    lp = torch.cat([torch.log_softmax(z.double(), 1).gather(1, a[:, None].long())[:, 0]
                    for z, a in zip(Z.split(1000), act.split(1000))])
    pick = torch.rand(n, device="cuda", generator=g)
    ratio = torch.where(pick < 0.1, 0.8, torch.where(pick < 0.2, 1.3, 1.0)).double()
    old = (lp - torch.log(ratio)).float()
    ws = _ws(G.gnn_policy_workspace_bytes(n, C))
    dZ = torch.empty_like(Z)
    res = []
    for parts in ([(0, n)], [(0, cut), (cut, n)]):
        ws.fill_(255)
        dZ.fill_(7.0)
        logp, outs = torch.empty(n, device="cuda"), []
        for b, e in parts:
            out = torch.empty(3, device="cuda")
            G.gnn_policy_loss(e - b, C, Z[b:e], C, act[b:e], adv[b:e], old[b:e], None, w[b:e], 0.2,
                              0.3, 0.0, out, logp[b:e], dZ[b:e], C, ws)
            outs.append(out)
        torch.cuda.synchronize()
        none = (dZ == 0).all(1)
        res.append((torch.stack(outs).double().sum(0), logp, none, dZ[::7].clone()))
    assert bool(((res[0][0] - res[1][0]).abs() <= 4 * U * res[0][0].abs().clamp(min=1e-3)).all())
    for x, y in zip(res[0][1:], res[1][1:]):
        assert torch.equal(x, y)
    rho = (lp - old.double()).exp()
    want = rho * adv.double() > rho.clamp(0.8, 1.3) * adv.double()
    sure = ((rho - 0.8).abs() > 1e-10) & ((rho - 1.3).abs() > 1e-10)
    assert torch.equal(res[0][2][sure], want[sure]) and int(want.sum()) > 100


@pytest.mark.parametrize("n,C", [(300, 9), (40, 700), (6, 20000), (70, 33000)])
def test_captured_away_from_borders_and_replayed_at_them(n, C):
    """Which rows are at a border is decided on the device: a call captured
    with none of them there, replayed with some, with all and with none, gives
    an eager call's bits."""
    z, a, adv, away, ref, w = _case(n, C, 42)
    at = [_near(n, C, 42, share)[3] for share in (0.0, 0.4, 1.0, 0.0, 1.0)]
    Z, act = to_dev(z), torch.from_numpy(a.astype(np.int32)).cuda()
    A, o, rf, ww = _f(adv), _f(away), _f(ref), _f(w)
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
    for old in at:
        o.copy_(_f(old))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        call(bufs[1])
        torch.cuda.synchronize()
        for x, y in zip(bufs[0][:3], bufs[1][:3]):
            assert torch.equal(x, y)


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


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("size,top", [(1e30, 1.0), (1e36, 1e-3), (1e37, 1e-4), (1e-30, 1e-38)])
def test_adamw_clipping_factors_at_the_ends(bits, size, top):
    """Factors down to 1e-42, which fp32 holds with a few bits only."""
    ts = _tensors([600], bits, 13, zero_state=True)
    rng = np.random.default_rng(2)
    g = (size * rng.uniform(0.5, 2.0, 600) * rng.choice([-1.0, 1.0], 600)).astype(np.float32)
    ts[0]["G"][0].copy_(torch.from_numpy(g))
    ps, decays = _params(ts, bits, decay=0.0)
    norm = torch.zeros(1, device="cuda")
    G.gnn_grad_norm(ps, norm, _ws(G.gnn_grad_norm_workspace_bytes(ps)))
    n = float(norm)
    assert np.isfinite(n) and n > top
    before = [_host(x) for x in ts]
    G.gnn_adamw_step(ps, 1e-3, 0.9, 0.999, 1e-12, 1, norm, top, 4)
    torch.cuda.synchronize()
    check_step(before, ts, bits, decays, 1e-3, 0.9, 0.999, 1e-12, 1, top / n, 4)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("size", [2.0 ** -100, 1e-24, 1e-19, 1e-12, 1e-4])
def test_adamw_tiny_gradients_from_weights_of_zero(bits, size):
    """The update alone (weights 0, no decay), so that it is seen to its own
    last bits.  Roundings, u each: m 5 of its size, v 8 of v and with 32-bit
    moments half a step of 2^-149 for each of its three operations, which the
    root carries into the update's bounds; 14 for the update's own."""
    ts = _tensors([1000, 41], bits, 14, zero_state=True)
    rng = np.random.default_rng(3)
    for t in ts:
        c = t["W"][0].numel()
        t["W"][0].zero_()
        t["G"][0].copy_(torch.from_numpy((size * rng.uniform(0.5, 2.0, c) *
                                          rng.choice([-1.0, 1.0], c)).astype(np.float32)))
    ps, _ = _params(ts, bits, decay=0.0)
    before = [_host(x) for x in ts]
    lr, b1, b2, eps = 1e-3, 0.9, 0.999, 0.1 * size
    G.gnn_adamw_step(ps, lr, b1, b2, eps, 1, seed=8)
    torch.cuda.synchronize()
    for h, x in zip(before, ts):
        _, m, v = P.adamw(h["W"], h["G"], 0 * h["W"], 0 * h["W"], lr, b1, b2, eps, 1, 0.0)
        verr = 8 * U * v + (1.5 * 2.0 ** -149 if bits == 32 else 0.0)
        now = -_host(x)["W"].astype(np.float64) * np.sign(m)
        for err, side in ((verr, -1), (-verr, 1)):
            den = np.sqrt(np.maximum(v + err, 0) / (1 - b2)) + eps
            bound = lr * np.abs(m) / (1 - b1) / den
            assert np.all(side * (now - bound) <= 20 * U * bound)


def test_adamw8_neighbours_of_a_broken_block():
    """A NaN and an infinity break their own blocks of 256; every other block,
    in the same tensor and in others, is as if they were not there."""
    ts = _tensors([256 * 6 + 100, 300], 8, 15)
    ps, decays = _params(ts, 8)
    sound = [_host(x) for x in ts]
    ts[0]["G"][0][256 + 7] = float("nan")
    ts[0]["G"][0][256 * 4 + 255] = float("inf")
    G.gnn_adamw_step(ps, 1e-3, 0.9, 0.999, 1e-8, 3, seed=5)
    torch.cuda.synchronize()
    now = [_host(x) for x in ts]
    other = _tensors([256 * 6 + 100, 300], 8, 15)
    ps2, _ = _params(other, 8)
    G.gnn_adamw_step(ps2, 1e-3, 0.9, 0.999, 1e-8, 3, seed=5)
    torch.cuda.synchronize()
    check_step(sound, other, 8, decays, 1e-3, 0.9, 0.999, 1e-8, 3, 1.0, 5)
    want = [_host(x) for x in other]
    broken = [1, 4]
    fine = np.repeat([b not in broken for b in range(7)], 256)[: 256 * 6 + 100]
    for k in ("W", "m", "v"):
        assert np.array_equal(now[0][k][fine], want[0][k][fine]), k
        assert np.array_equal(now[1][k], want[1][k]), k
    for k in ("m_scale", "v_scale"):
        ok = np.array([b not in broken for b in range(7)])
        assert np.array_equal(now[0][k][ok], want[0][k][ok]) and np.isnan(now[0][k][~ok]).all()
    at = np.zeros(256 * 6 + 100, bool)
    at[[256 + 7, 256 * 4 + 255]] = True
    assert np.array_equal(now[0]["W"][~at], want[0]["W"][~at])
    assert not np.isfinite(now[0]["W"][at]).any()


# ----------------------------------------------------------------- streams

def _busy(stream=None, times=30):
    """Work of some tens of ms on a stream."""
    with torch.cuda.stream(stream or torch.cuda.current_stream()):
        x = torch.randn((4096, 4096), device="cuda")
        for _ in range(times):
            x = (x @ x).mul_(1e-3)
    return x


def test_param_set_is_ready_for_any_stream():
    """The plan and the moments are there when the constructor returns: a
    first step may be on a stream that does not wait for the present one."""
    _busy(times=1)
    torch.cuda.synchronize()
    keep = _busy()
    w = [torch.randn(5000, device="cuda"), torch.randn((30, 41), device="cuda")]
    ps = runtime.ParamSet(w, [torch.ones_like(x) for x in w], [0.1, 0.0], 8)
    assert torch.cuda.current_stream().query()
    s = torch.cuda.Stream()
    before = [x.clone() for x in w]
    torch.cuda.synchronize()
    ps.step(1, 1e-2, max_norm=1.0, stream=s)
    s.synchronize()
    assert all(not torch.equal(x, y) for x, y in zip(w, before)) and keep is not None


def test_trainer_allocates_on_the_stream_it_works_on():
    """With stream= the tensors that a call makes come from that stream's
    memory: not from a block that the present stream freed a moment ago and
    may still be writing."""
    tr, d, _, X, _ = _trainer("sgd", lr=0.0)
    act = torch.zeros(tr.n, dtype=torch.int32, device="cuda")
    want = tr.action_logp(X, act)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    freed = [torch.empty(tr.n, device="cuda") for _ in range(4)]
    at = {x.data_ptr() for x in freed}
    del freed
    for stream in (s, s.cuda_stream):
        lp = tr.action_logp(X, act, stream=stream)
        assert lp.data_ptr() not in at
        s.synchronize()
        assert torch.equal(lp, want)
    assert torch.equal(tr.action_logp(X, act, stream=0), want)  # the default stream


def test_trainer_buffers_outlive_the_streams_that_use_them():
    """Buffers that a larger subgraph replaces while another stream still
    works in them are not handed out again before it is done."""
    small, large = (prepared(synth.power_law_graph(k, 2.1, 8.0, seed=k)) for k in (900, 2000))
    rng = np.random.default_rng(0)
    f, h, C = 24, 16, 700
    params = [synth.LayerParams(synth.glorot(f, h, rng), synth.glorot(f, h, rng))]
    tr = runtime.Trainer(small, params, f, synth.glorot(2 * h, C, rng), False, "sgd", lr=0.0)
    X = to_dev(rng.standard_normal((2000, f)).astype(np.float32), 32)
    act = torch.zeros(2000, dtype=torch.int32, device="cuda")
    tr.action_logp(X[:900], act[:900])  # made in the current stream's memory
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    keep = _busy(s, 100)
    tr.action_logp(X[:900], act[:900], stream=s)
    size = tr._Z.buf.numel()
    old = {t.data_ptr() for t in (tr._Z.buf, tr._dZ.buf)}
    tr.bind(large)
    tr.action_logp(X, act)  # replaces them
    more = [torch.empty(size, device="cuda") for _ in range(8)] + [tr._Z.buf, tr._dZ.buf]
    if not s.query():  # (else they may well be)
        assert not old & {t.data_ptr() for t in more}
    torch.cuda.synchronize()
    del keep


def test_trainer_logp_is_of_the_present_rows():
    """`logp` after a step has the present subgraph's rows, whatever subgraphs
    the trainer was on before."""
    graphs = [prepared(synth.power_law_graph(k, 2.1, 8.0, seed=k)) for k in (900, 300)]
    rng = np.random.default_rng(0)
    f, h, C = 24, 16, 5
    params = [synth.LayerParams(synth.glorot(f, h, rng), synth.glorot(f, h, rng))]
    tr = runtime.Trainer(graphs[0], params, f, synth.glorot(2 * h, C, rng), False, "sgd", lr=0.0)
    for g in graphs:
        tr.bind(g)
        X = to_dev(rng.standard_normal((g.n, f)).astype(np.float32), 32)
        act = torch.from_numpy(rng.integers(0, C, g.n).astype(np.int32)).cuda()
        tr.policy_step(X, act, torch.ones(g.n, device="cuda"))
        assert tr.logp.shape == (g.n,)
        assert torch.equal(tr.logp, tr.action_logp(X, act))


def test_trainer_captured_on_a_stream_that_it_was_not_on():
    """Buffers made on the current stream, then acting and a step captured on
    another one and replayed between eager iterations of a second trainer."""
    cap, d, _, X, _ = _trainer("sgd", lr=1e-3)
    eager, _, _, _, _ = _trainer("sgd", lr=1e-3)
    n = cap.n
    act = torch.arange(n, device="cuda", dtype=torch.int32) % cap.C
    adv = torch.randn(n, device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    cap.action_logp(X, act)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        old = cap.action_logp(X, act, stream=s.cuda_stream)
        cap.policy_step(X, act, adv, old, old, beta=0.1, stream=s.cuda_stream)
    for it in range(3):
        graph.replay()
        torch.cuda.synchronize()
        want = eager.action_logp(X, act)
        eager.policy_step(X, act, adv, want, want, beta=0.1)
        torch.cuda.synchronize()
        assert torch.equal(old, want) and torch.equal(cap.policy_out, eager.policy_out), it
        assert torch.equal(cap.logp, eager.logp)
        for (w, _), (v, _) in zip(cap.pairs, eager.pairs):
            assert torch.equal(w, v), it


@pytest.mark.parametrize("C", [5, 700, 20000, 70000])
def test_policy_of_no_rows_at_every_width(C):
    out, dZ = torch.full((3,), 7.0, device="cuda"), torch.full((C,), 7.0, device="cuda")
    for d in (None, dZ):
        out.fill_(7.0)
        G.gnn_policy_loss(0, C, None, C, None, None, None, None, None, 0.2, 0.2, 0.0, out, None, d,
                          C, None)
        torch.cuda.synchronize()
        assert torch.all(out == 0) and torch.all(dZ == 7.0)
