"""Token losses against the float64 oracle, through the C ABI.

Tolerances count the kernel's fp32 roundings (e = 2^-24 each).  With u_j = (y_j - max) * scale * log2(e), U = max |u_j|:
  - exp2(u): the difference, the product and the constant's own rounding move the argument by 3 e |u|, the approximation is good to 2 ulp
    (4 e): each term is off by e (3 U + 4) relative; adding n terms in any order used here, at most n / 32 + 64 deep, adds e per level
  - lp = ln 2 (u_t - log2 s): the sum's error, e (3 |u_t| + 2) for the first term, 2 ulp of the log, one rounding of the difference and the product
  - the gradient: c's error times ([j = t] + p) plus |c| times p's error, rounded once more to the storage type.
Values below 2^-126 may be flushed to 0.
"""
import numpy as np
import pytest
import torch

import paper_2312_14227_b200 as et
from oracle import token_oracle as tok

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = 2.0 ** -24
TINY = 2.0 ** -120


class Stack:
    """A stack whose output has the wanted width, bound with guard words round its workspace regions."""

    def __init__(self, M, width, dtype):
        et.et_debug_guard_regions(True)
        self.s = et.et_stack_create([(8, width, 0, 1, -1)], M, dtype)
        et.et_debug_guard_regions(False)
        self.tdt = torch.bfloat16 if dtype == et.ET_BF16 else torch.float32
        self.W = torch.zeros(8, width, dtype=self.tdt, device=DEV)
        self.b = torch.zeros(width, dtype=self.tdt, device=DEV)
        self.ws = torch.empty(et.et_stack_workspace_bytes(self.s), dtype=torch.uint8, device=DEV)
        et.et_stack_bind(self.s, [self.W], [self.b], self.ws)

    def check(self):
        torch.cuda.synchronize()
        st, bad = et.et_debug_check_guards(self.s)
        assert st == et.ET_OK, bad


class Case:
    def __init__(self, M, width, vocab, dtype, scale=1.0, seed=0, spread=2.0, masked=0.2, edge=True):
        self.M, self.width, self.vocab, self.dtype, self.scale = M, width, vocab, dtype, scale
        rng = self.rng = np.random.default_rng(seed)
        self.st = Stack(M, width, dtype)
        y = torch.from_numpy((rng.normal(size=(M, width)) * spread).astype(np.float32)).to(self.st.tdt)
        self.targets = rng.integers(0, vocab, M).astype(np.int32)
        for i in range(M):
            y[i, self.targets[i]] += 4
        self.weights = (rng.random(M) * (rng.random(M) >= masked)).astype(np.float32)
        self.weights[0] = 0.5
        if edge and M > 6:
            self.weights[1] = 0.0
            self.targets[2] = -100
            self.targets[3] = vocab                      # outside
            self.targets[4], self.targets[5] = 0, vocab - 1
            y[1] = float("nan")                          # rows that are left out may hold anything
            y[2] = float("inf")
            y[6, :vocab - 1] = float("-inf")             # all the mass on one token
            self.targets[6] = vocab - 1
            y[6, vocab - 1] = 0.5
        y[:, vocab:] = float("nan")                      # padding columns too
        self.y_host = y.to(torch.float64).numpy()
        self.y = y.to(DEV)
        self.live = tok.live_rows(self.targets, self.weights, vocab)

    def dev(self, a, dt=np.float32):
        return None if a is None else torch.from_numpy(np.ascontiguousarray(a).astype(dt)).to(DEV)

    def errors(self, live=None):
        """Absolute error bound of lp per row, relative error bound of p per row."""
        live = self.live if live is None else live
        lp_tol, p_tol = np.zeros(self.M), np.zeros(self.M)
        depth = self.vocab / 32 + 64
        for i in np.flatnonzero(live):
            z = self.y_host[i, :self.vocab] * self.scale
            u = (z - z.max()) / np.log(2)
            p = np.exp2(u)
            p /= p.sum()
            f = np.isfinite(u) & (p > 1e-40)
            sum_tol = E * ((p[f] * (3 * np.abs(u[f]) + 4)).sum() + depth)     # the terms' errors weigh as the terms do
            ut, ls = abs(u[self.targets[i]]), np.log2(np.exp2(u[f]).sum())
            lp_tol[i] = np.log(2) * (sum_tol / np.log(2) + E * (3 * ut + 2 + 4 * abs(ls) + 3 * abs(ut + ls)))
            p_tol[i] = sum_tol + E * (3 * np.abs(u[f]).max() + 8)
        return lp_tol, p_tol

    def check_logp(self, got, want, live=None):
        live = self.live if live is None else live
        got = got.cpu().numpy().astype(np.float64)
        assert (np.abs(got - want)[live] <= self.errors(live)[0][live]).all()
        assert (got[~live] == 0).all()

    def check_grad(self, got, want, coef, coef_tol):
        got = got.to(torch.float64).cpu().numpy()
        assert (got[~self.live] == 0).all() and (got[:, self.vocab:] == 0).all()
        half = torch.finfo(self.st.tdt).eps / 2
        _, p_tol = self.errors()
        for i in np.flatnonzero(self.live):
            z = self.y_host[i, :self.vocab] * self.scale
            p = np.exp(z - z.max())
            p /= p.sum()
            hit = np.zeros(self.vocab)
            hit[self.targets[i]] = 1
            g = want[i, :self.vocab]
            tol = self.scale * (coef_tol[i] * (p + hit) + abs(coef[i]) * (p * p_tol[i] + 4 * E * (p + hit)))
            tol = tol + half * (np.abs(g) + tol) + TINY
            bad = np.abs(got[i, :self.vocab] - g) > tol
            assert not bad.any(), (i, np.flatnonzero(bad)[:5], got[i, :self.vocab][bad][:5], g[bad][:5], tol[bad][:5])


F, B = et.ET_F32, et.ET_BF16
SHAPES = [(1, 8, 8, F), (9, 1, 1, F), (5, 7, 3, F), (33, 1000, 997, F), (17, 4099, 4099, F), (12, 33001, 33001, F), (7, 140003, 140001, F),
          (1, 8, 5, B), (40, 264, 257, B), (64, 1000, 1000, B), (21, 8200, 8195, B), (19, 32008, 32003, B), (9, 50264, 50257, B),
          (10, 131072, 131072, B), (7, 262152, 262147, B)]


@pytest.mark.parametrize("M,width,vocab,dtype", SHAPES)
def test_token_logp(M, width, vocab, dtype):
    c = Case(M, width, vocab, dtype, scale=0.8, seed=M, edge=vocab > 2)
    live = tok.live_rows(c.targets, np.ones(M), vocab)
    if M > 6 and vocab > 2:                              # no weights here: a row of NaN is a row of NaN
        c.y_host[1, :] = 0.25
        c.y[1, :] = 0.25
    out = torch.full((M,), float("nan"), device=DEV)
    et.et_token_logp(c.st.s, c.y, c.dev(c.targets, np.int32), out, vocab=vocab, logit_scale=0.8)
    c.st.check()
    want, _ = tok.log_probs(c.y_host, c.targets, vocab, float(np.float32(0.8)), live)
    c.scale = float(np.float32(0.8))
    c.check_logp(out, want, live)


def _policy(c, beta, use_old=True, use_ref=True, in_place=False, weights=True, lo=0.2, hi=0.3, stream=None):
    rng = np.random.default_rng(99)
    w = c.weights if weights else np.full(c.M, np.float32(1.0 / c.M))
    if not weights:
        c.live = tok.live_rows(c.targets, w, c.vocab)
    lp, _ = tok.log_probs(c.y_host, c.targets, c.vocab, c.scale, c.live)
    # log ratios off the borders log(0.8) = -0.223 and log(1.3) = 0.262 by far more than lp's error
    delta = rng.choice([-0.6, -0.25, -0.2, -0.05, 0.0, 0.04, 0.24, 0.28, 0.7], c.M)
    old = (lp - delta).astype(np.float32) if use_old else None
    ref = (lp + 0.4 * rng.normal(size=c.M)).astype(np.float32) if use_ref else None
    adv = rng.normal(size=c.M).astype(np.float32)
    dY = c.y.clone() if in_place else torch.full_like(c.y, float("nan"))
    src = dY if in_place else c.y
    logp = torch.full((c.M,), float("nan"), device=DEV)
    stats = torch.full((4,), float("nan"), device=DEV)
    et.et_loss_policy_grad(c.st.s, src, c.dev(c.targets, np.int32), c.dev(adv), dY, weights=c.dev(c.weights) if weights else None,
                           logp_old=c.dev(old), logp_ref=c.dev(ref), logp=logp, loss_dev=stats,
                           vocab=0 if c.vocab == c.width else c.vocab, logit_scale=c.scale, clip_low=lo, clip_high=hi, kl_coef=beta, stream=stream)
    c.st.check()
    lo, hi, beta = float(np.float32(lo)), float(np.float32(hi)), float(np.float32(beta))
    want = tok.policy(c.y_host, c.targets, w, adv, old, ref, c.vocab, c.scale, lo, hi, beta)
    # c = w (-A r - beta expm1(d)): lp's error moves r by r lp_tol and expm1(d) by exp(d) lp_tol; each is rounded a few times (expf, expm1f: 2 ulp)
    lp_tol, _ = c.errors()
    r = np.exp(np.where(c.live, lp - (lp if old is None else old), 0.0))
    ed = np.exp(np.where(c.live, ref - lp, 0.0)) if use_ref else np.zeros(c.M)
    slack = 8 * E
    grow = lp_tol + E * np.abs(lp)                        # the differences lp - old, ref - lp round once more
    moved = (0 if old is None else 1) * grow
    coef_tol = np.abs(w) * (np.abs(adv) * r * (moved + slack) + beta * (ed * grow + (ed + 1) * slack))
    return want, logp, stats, dY, coef_tol, (w, adv, r, ed, grow, moved, slack, beta)


def _check_policy(c, got):
    (stats_w, lp_w, dY_w, coef), logp, stats, dY, coef_tol, (w, adv, r, ed, grow, moved, slack, beta) = got
    c.check_logp(logp, lp_w)
    c.check_grad(dY, dY_w, coef, coef_tol)
    s = stats.cpu().numpy().astype(np.float64)
    t1 = (np.abs(w) * np.abs(adv) * np.maximum(r, 1.3) * (moved + slack))[c.live].sum()
    t2 = (np.abs(w) * (np.abs(ed - 1) * grow + slack * (ed + 1 + np.abs(np.log(np.maximum(ed, 1e-30))))))[c.live].sum()
    for k, t in enumerate((t1 + beta * t2, t1, t2, 0.0)):
        assert abs(s[k] - stats_w[k]) <= t + 2 * E * abs(stats_w[k]), (k, s, stats_w)


@pytest.mark.parametrize("M,width,vocab,dtype", SHAPES)
def test_policy_loss(M, width, vocab, dtype):
    c = Case(M, width, vocab, dtype, scale=1.0, seed=M + 1, edge=vocab > 2)
    _check_policy(c, _policy(c, 0.1))


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("opts", [dict(use_old=False), dict(use_ref=False, beta=0.0), dict(beta=0.0), dict(in_place=True),
                                  dict(use_old=False, use_ref=False, beta=0.0)])
def test_policy_variants(dtype, opts):
    c = Case(37, 2056, 2051, dtype, scale=1.25, seed=11)
    _check_policy(c, _policy(c, **{"beta": 0.05, **opts}))


@pytest.mark.parametrize("M,width,dtype", [(6, 40000, F), (6, 262152, B), (33, 70000, B)])
def test_policy_in_place_long_rows(M, width, dtype):
    c = Case(M, width, width - 5, dtype, seed=12)
    _check_policy(c, _policy(c, 0.05, in_place=True))


def test_policy_default_weights():
    c = Case(24, 520, 520, F, seed=13, edge=False, masked=0.0)
    c.targets[3] = -1
    _check_policy(c, _policy(c, 0.05, weights=False))


def test_policy_everything_left_out():
    c = Case(8, 264, 264, B, seed=14)
    c.weights[:] = 0
    c.live[:] = False
    c.y[:] = float("nan")
    want, logp, stats, dY, _, _ = _policy(c, 0.1)
    assert (dY == 0).all() and (logp == 0).all() and (stats == 0).all()


def test_policy_forward_only_and_gradient_only():
    c = Case(20, 1000, 1000, B, seed=15)
    adv = c.dev(c.rng.normal(size=20))
    t, w = c.dev(c.targets, np.int32), c.dev(c.weights)
    dY, stats, logp = torch.empty_like(c.y), torch.empty(4, device=DEV), torch.empty(20, device=DEV)
    et.et_loss_policy_grad(c.st.s, c.y, t, adv, dY, weights=w, logp=logp, loss_dev=stats)
    s2, l2, d2 = torch.empty_like(stats), torch.empty_like(logp), torch.empty_like(dY)
    et.et_loss_policy_grad(c.st.s, c.y, t, adv, None, weights=w, logp=l2, loss_dev=s2)
    et.et_loss_policy_grad(c.st.s, c.y, t, adv, d2, weights=w)
    c.st.check()
    assert torch.equal(stats, s2) and torch.equal(logp, l2) and torch.equal(dY, d2)


@pytest.mark.parametrize("dtype", [F, B])
def test_lowest_values_and_flat_rows(dtype):
    """Logits of the type's lowest value are tokens of probability 0; a row of them alone is uniform."""
    c = Case(3, 1024, 1024, dtype, seed=16, edge=False)
    low = float(torch.finfo(c.st.tdt).min)
    c.y[0, :512] = low
    c.y[1, :] = low
    c.y[2, :] = 3.0
    c.targets[:] = [700, 5, 9]
    out = torch.empty(3, device=DEV)
    et.et_token_logp(c.st.s, c.y, c.dev(c.targets, np.int32), out)
    live = np.ones(3, dtype=bool)
    c.y_host = c.y.to(torch.float64).cpu().numpy()
    want, _ = tok.log_probs(c.y_host, c.targets, 1024, 1.0, live)
    # 1024 equal terms add up exactly; only the log and its product round
    assert abs(float(out[1]) + np.log(1024)) <= 4 * E * np.log(1024) and abs(float(out[2]) + np.log(1024)) <= 4 * E * np.log(1024)
    c.check_logp(out, want, live)


def test_rows_without_a_value_give_nan():
    c = Case(4, 264, 264, F, seed=17, edge=False)
    c.y[0, :] = float("-inf")
    c.y[1, 7] = float("inf")
    c.y[2, 7] = float("nan")
    out = torch.zeros(4, device=DEV)
    et.et_token_logp(c.st.s, c.y, c.dev(c.targets, np.int32), out)
    assert torch.isnan(out[:3]).all() and torch.isfinite(out[3])
    dY = torch.zeros_like(c.y)
    et.et_loss_policy_grad(c.st.s, c.y, c.dev(c.targets, np.int32), c.dev(np.ones(4)), dY)
    assert torch.isnan(dY[:3]).any(1).all() and torch.isfinite(dY[3]).all()


# ---- preference -------------------------------------------------------------------------------------
def _pref(c, begin, ref, kind, eps=0.0, beta=0.1, weights=True, in_place=False, dY=True):
    P = (len(begin) - 1) // 2
    out = (c.y.clone() if in_place else torch.full_like(c.y, float("nan"))) if dY else None
    seq = torch.full((2 * P,), float("nan"), device=DEV)
    stats = torch.full((4,), float("nan"), device=DEV)
    et.et_loss_preference_grad(c.st.s, out if in_place else c.y, c.dev(c.targets, np.int32), c.dev(begin, np.int32), out,
                               weights=c.dev(c.weights) if weights else None, ref_logp=c.dev(ref), seq_logp=seq, loss_dev=stats, kind=kind,
                               vocab=0 if c.vocab == c.width else c.vocab, logit_scale=c.scale, beta=beta, label_smoothing=eps)
    c.st.check()
    beta, eps = float(np.float32(beta)), float(np.float32(eps))
    want = tok.preference(c.y_host, c.targets, c.weights if weights else None, begin, ref, c.vocab, c.scale, kind, beta, eps)
    return want, out, seq, stats, (P, beta)


def _check_pref(c, begin, ref, kind, **k):
    (stats_w, S, dY_w, coef), dY, seq, stats, (P, beta) = _pref(c, begin, ref, kind, **k)
    w = c.weights.astype(np.float64) if k.get("weights", True) else np.ones(c.M)
    inside = np.zeros(c.M, dtype=bool)
    b = np.clip(begin, 0, c.M)
    s_tol = np.zeros(2 * P)
    c.live = tok.live_rows(c.targets, w, c.vocab)
    lp_tol, _ = c.errors()
    lp, _ = tok.log_probs(c.y_host, c.targets, c.vocab, c.scale, c.live)
    coef_tol = np.zeros(c.M)
    for q in range(2 * P):
        rows = np.arange(b[q], max(b[q], b[q + 1]))
        inside[rows] = True
        s_tol[q] = (np.abs(w[rows]) * (lp_tol[rows] + E * np.abs(lp[rows])))[c.live[rows]].sum()
    c.live &= inside
    got = seq.cpu().numpy().astype(np.float64)
    assert (np.abs(got - S) <= s_tol + E * np.abs(S)).all(), (got, S, s_tol)
    # the slope in x changes by at most |dx''| |x error|: 1/4 (sigmoid), 2 / beta^2 (IPO), 0 (hinge, x is not near 1 here)
    second = {0: 0.25, 1: 2 / beta ** 2, 2: 0.0}[kind]
    for p in range(P):
        x_tol = beta * (s_tol[2 * p] + s_tol[2 * p + 1])
        for q in (2 * p, 2 * p + 1):
            rows = np.arange(b[q], max(b[q], b[q + 1]))
            coef_tol[rows] = np.abs(w[rows]) * beta / P * second * x_tol + 2 * E * np.abs(coef[rows])
    if dY is not None:
        c.check_grad(dY, dY_w, coef, coef_tol)
    s = stats.cpu().numpy().astype(np.float64)
    r_tol = beta * s_tol.sum() / P
    slope = {0: 1.0, 2: 1.0, 1: 2 / beta * np.sqrt(max(stats_w[0], 1e-12) * P)}[kind]
    assert abs(s[0] - stats_w[0]) <= slope * r_tol + (r_tol / beta) ** 2 * (kind == 1) * P + 2 * E * abs(stats_w[0]), (s, stats_w)
    assert abs(s[1] - stats_w[1]) <= r_tol + 2 * E * abs(stats_w[1]) and abs(s[2] - stats_w[2]) <= r_tol + 2 * E * abs(stats_w[2])
    assert s[3] == np.float32(stats_w[3])


def _near(c, begin, seed, spread=4.0, weights=True):
    """Reference sums near the policy's, so that the margins are ordinary ones."""
    w = c.weights if weights else None
    _, S, _, _ = tok.preference(c.y_host, c.targets, w, begin, None, c.vocab, c.scale, 0, 0.1, 0.0)
    return (S + np.random.default_rng(seed).normal(size=len(S)) * spread).astype(np.float32)


@pytest.mark.parametrize("kind,eps", [(0, 0.0), (0, 0.2), (1, 0.0), (2, 0.0)])
@pytest.mark.parametrize("M,width,vocab,dtype", [(40, 1003, 1001, F), (40, 1032, 1027, B), (30, 33000, 32999, B)])
def test_preference_loss(kind, eps, M, width, vocab, dtype):
    c = Case(M, width, vocab, dtype, scale=0.9, seed=21)
    c.scale = float(np.float32(0.9))
    begin = [0, 7, 12, 12, 20, 27, M - 2]                # one empty sequence, two rows behind the last
    _check_pref(c, begin, _near(c, begin, 5), kind, eps=eps)


@pytest.mark.parametrize("begin", [[0, 1, 2], [0, 0, 0], [3, 3, 20], [0, 20, 20], [-5, 8, 400], [2, 10, 18], [0, 10, 20, 20, 20]])
def test_preference_bounds(begin):
    c = Case(20, 520, 515, F, seed=22)
    _check_pref(c, begin, None, 0)


def test_preference_bounds_that_decrease_stay_in_range():
    c = Case(20, 520, 515, F, seed=23)
    want, dY, seq, stats, _ = _pref(c, [15, 3, 1 << 30, -(1 << 31), 7], None, 0)
    torch.cuda.synchronize()
    assert torch.isfinite(dY).all()


@pytest.mark.parametrize("dtype", [F, B])
def test_preference_in_place_and_default_weights(dtype):
    c = Case(24, 2056, 2056, dtype, seed=24, edge=False)
    begin = [0, 6, 11, 17, 24]
    _check_pref(c, begin, _near(c, begin, 6, weights=False), 0, weights=False, in_place=True)


def test_preference_without_gradient():
    c = Case(24, 2056, 2056, B, seed=25)
    begin = [0, 6, 11, 17, 24]
    _check_pref(c, begin, None, 0, dY=False)


def test_preference_many_pairs():
    c = Case(600, 264, 259, F, seed=26)
    begin = np.sort(np.random.default_rng(3).integers(0, 601, 2 * 250 + 1)).astype(np.int64)
    _check_pref(c, list(begin), _near(c, list(begin), 7), 0)


# ---- how the calls behave ----------------------------------------------------------------------------
@pytest.mark.parametrize("M,width,dtype", [(50, 4099, F), (50, 32008, B), (3, 131072, B)])
def test_same_inputs_same_bits(M, width, dtype):
    c = Case(M, width, width, dtype, seed=31)
    a, b = _policy(c, 0.1), _policy(c, 0.1)
    for x, y in zip(a[1:4], b[1:4]):
        assert torch.equal(x, y)
    begin = [0, M // 3, M]
    a, b = _pref(c, begin, None, 0), _pref(c, begin, None, 0)
    for x, y in zip(a[1:4], b[1:4]):
        assert torch.equal(x, y)


def test_captured_and_replayed_on_another_stream():
    c = Case(40, 8200, 8195, B, seed=32)
    t, w = c.dev(c.targets, np.int32), c.dev(c.weights)
    adv, old = c.dev(c.rng.normal(size=40)), c.dev(c.rng.normal(size=40) - 8)
    begin, ref = c.dev([0, 9, 20, 30, 40], np.int32), c.dev(c.rng.normal(size=4))
    d1, d2 = torch.empty_like(c.y), torch.empty_like(c.y)
    s1, s2, lp = torch.empty(4, device=DEV), torch.empty(4, device=DEV), torch.empty(40, device=DEV)

    def calls(st):
        et.et_token_logp(c.st.s, c.y, t, lp, vocab=c.vocab, stream=st)
        et.et_loss_policy_grad(c.st.s, c.y, t, adv, d1, weights=w, logp_old=old, loss_dev=s1, vocab=c.vocab, stream=st)
        et.et_loss_preference_grad(c.st.s, c.y, t, begin, d2, weights=w, ref_logp=ref, loss_dev=s2, vocab=c.vocab, stream=st)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        calls(side)
    c.y.copy_(torch.where(torch.isfinite(c.y), c.y * 0.5, c.y))             # new logits in the captured buffers
    for x in (d1, d2, s1, s2, lp):
        x.fill_(float("nan"))
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    got = [x.clone() for x in (d1, d2, s1, s2, lp)]
    calls(None)
    torch.cuda.synchronize()
    for a, b in zip(got, (d1, d2, s1, s2, lp)):
        assert torch.equal(a, b) or torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))
    del g


@pytest.mark.parametrize("width,vocab,dtype", [(4096, 100, F), (4096, 100, B), (40000, 3001, B), (9000, 4, F), (300000, 70, B)])
def test_few_logits_in_a_wide_row(width, vocab, dtype):
    """Whole vectors, whole rounds and whole slices of padding behind the vocabulary."""
    c = Case(24, width, vocab, dtype, seed=41, edge=False)
    _check_policy(c, _policy(c, 0.05))
    begin = [0, 6, 11, 17, 22]
    _check_pref(c, begin, _near(c, begin, 8), 0)


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("rows", [1, 3, 147, 149, 300, 1000, 5000])
def test_any_number_of_rows(dtype, rows):
    """Fewer rows than blocks, one more, many rounds; one or two warps a row and one block a row."""
    for width in (200, 1504, 3000):
        c = Case(rows, width, width - 3, dtype, seed=42 + rows, edge=rows > 6, masked=0.5)
        _check_policy(c, _policy(c, 0.05))


@pytest.mark.parametrize("scale", [1e-6, 1e-3, 30.0])
def test_logit_scales(scale):
    s = float(np.float32(scale))
    c = Case(30, 1000, 997, F, scale=s, seed=43, spread=2.0 / max(s, 1.0))
    _check_policy(c, _policy(c, 0.05))


def test_values_far_from_zero():
    """Rows whose largest value is large either way: the terms go by differences."""
    for dtype in (F, B):
        for off in (-3e4, 3e4, 1e30, -1e30):
            c = Case(12, 2056, 2056, dtype, seed=44, edge=False, masked=0.0)
            c.y += off
            c.y[:, 5] = off
            c.targets[:] = 5
            c.y_host = c.y.to(torch.float64).cpu().numpy()
            out = torch.empty(12, device=DEV)
            et.et_token_logp(c.st.s, c.y, c.dev(c.targets, np.int32), out)
            c.st.check()
            want, _ = tok.log_probs(c.y_host, c.targets, 2056, 1.0, c.live)
            c.check_logp(out, want)
            if abs(off) < 1e6:
                _check_policy(c, _policy(c, 0.05))


def test_logits_beyond_32_bit_offsets():
    M, V = 20000, 131072                                # 2.6e9 logits
    st = Stack(M, V, B)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    y = torch.randn(M, V, generator=g, device=DEV, dtype=torch.bfloat16)
    t = torch.randint(0, V, (M,), generator=g, device=DEV, dtype=torch.int32)
    adv = torch.randn(M, generator=g, device=DEV)
    lp, lp2, dY = torch.empty(M, device=DEV), torch.empty(M, device=DEV), torch.empty_like(y)
    et.et_loss_policy_grad(st.s, y, t, adv, dY, logp=lp)
    et.et_token_logp(st.s, y, t, lp2)
    st.check()
    for i in (0, 1, 16383, 16384, M - 1):
        z = y[i].double()
        want = z[t[i].long()] - torch.logsumexp(z, 0)
        for got in (lp[i], lp2[i]):
            assert abs(float(got) - float(want)) <= 64 * E * abs(float(want))
        p = torch.softmax(z, 0)
        p[t[i].long()] -= 1
        w = float(adv[i]) / M * p
        assert ((dY[i].double() - w).abs() <= (2.0 ** -8 + 1e-5) * w.abs() + TINY).all()
    begin = torch.tensor([0, M // 2, M - 1], dtype=torch.int32, device=DEV)
    et.et_loss_preference_grad(st.s, y, t, begin, dY, beta=1e-6)
    st.check()
    i, j = M - 2, M - 1
    p = torch.softmax(y[i].double(), 0)
    p[t[i].long()] -= 1
    ratio = (dY[i].double() / p)[p.abs() > 1e-7]
    assert (dY[j] == 0).all() and float(ratio.std() / ratio.mean().abs()) < 2.0 ** -8


def test_two_stacks_at_once():
    """Two stacks, each on a stream of its own, at the same time: what they give one after the other."""
    cs = [Case(700, 8200, 8195, B, seed=51), Case(300, 4099, 4099, F, seed=52)]
    want, args = [], []
    for c in cs:
        t, w, adv = c.dev(c.targets, np.int32), c.dev(c.weights), c.dev(c.rng.normal(size=c.M))
        old = c.dev(c.rng.normal(size=c.M) - 8)
        dY, stats = torch.empty_like(c.y), torch.empty(4, device=DEV)
        args.append((t, w, adv, old, dY, stats))
        et.et_loss_policy_grad(c.st.s, c.y, t, adv, dY, weights=w, logp_old=old, loss_dev=stats, vocab=c.vocab)
        c.st.check()
        want.append((dY.clone(), stats.clone()))
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, (t, w, adv, old, dY, stats), s in zip(cs, args, streams):
            et.et_loss_policy_grad(c.st.s, c.y, t, adv, dY, weights=w, logp_old=old, loss_dev=stats, vocab=c.vocab, stream=s)
    torch.cuda.synchronize()
    for c, a, (dY, stats) in zip(cs, args, want):
        c.st.check()
        assert torch.equal(a[4], dY) and torch.equal(a[5], stats)
