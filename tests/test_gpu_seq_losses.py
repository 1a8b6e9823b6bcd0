"""The losses of whole sequences on the GPU against the fp64 oracle: the clipped policy loss and the preference loss, their
gradients, masks and lengths where they can go wrong, refusals, streams and graphs, and model steps that end in them.

Tolerances follow the arithmetic: a rounding to fp32 is off by 2^-24 of its value, expf by 2^-22 of it, and a sum of four terms
in fp32 (the rest is in 64 bits) by 3 x 2^-24 of their magnitudes."""
import itertools

import numpy as np
import pytest
import torch

from oracle import losses_oracle as S
from paper_2601_05732_b200 import binding
from paper_2601_05732_b200 import layer as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    c = binding.MhcLite(4, 64, 0)
    yield c
    assert c.lib.mhclite_device_status(c._h) == binding.OK


def dev(a, dtype=F32):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(dtype).to(DEV)


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def empty(*shape, dtype=F32):
    return torch.full(shape, float("nan"), dtype=dtype, device=DEV)


def close(name, got, ref, tol):
    got = f64(got)
    assert got.shape == ref.shape, name
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got - ref) - tol):.3e} over"


def cut(r, T, S_, kind="even"):
    """Starts of S_ sequences over T tokens."""
    if kind == "all":
        return np.array([0] + [T] * S_)
    if kind == "ones":
        return np.minimum(np.arange(S_ + 1), T)
    a = np.sort(r.integers(0, T + 1, S_ + 1))
    if kind == "steps":
        a = a // 128 * 128
    if kind == "empties":
        a = np.sort(r.choice(a[:: max(1, S_ // 3)], S_ + 1))
    return a


class Case:
    def __init__(self, T, S_, kind="even", ref=True, token_adv=False, dead=0.3, seed=0):
        r = np.random.default_rng(seed + T + S_)
        f = lambda a: a.astype(np.float32).astype(np.float64)
        self.T, self.S, self.token_adv = T, S_, token_adv
        self.nll = f(r.exponential(size=T))
        self.old, self.ref = f(self.nll + 0.2 * r.normal(size=T)), f(self.nll + 0.6 * r.normal(size=T)) if ref else None
        self.target = np.where(r.random(T) < dead, -100, r.integers(0, 1000, T))
        self.starts = cut(r, T, S_, kind)
        self.adv, self.dloss = f(r.normal(size=T if token_adv else S_)), f(r.normal(size=S_))
        self.dpair = self.dloss[: S_ // 2]

    def tensors(self):
        i64 = torch.int64
        return {"nll": dev(self.nll), "old": dev(self.old), "ref": dev(self.ref), "target": dev(self.target, i64), "starts": dev(self.starts, i64),
                "adv": dev(self.adv), "dloss": dev(self.dloss), "dpair": dev(self.dpair)}


def run_policy(c, k, t, mean, grad=True, lo=0.2, hi=0.3, b=0.1):
    out = empty(k.S), empty(k.S, 3), empty(k.T) if grad else None
    c.policy_loss(t["nll"], t["old"], t["ref"], t["target"], t["starts"], t["adv"], k.token_adv, lo, hi, b, mean, out[0], out[1],
                  t["dloss"] if grad else None, out[2])
    return out


def check_policy(c, k, mean, grad=True, lo=0.2, hi=0.3, b=0.1, t=None):
    out = loss, stats, dnll = run_policy(c, k, t or k.tensors(), mean, grad, lo, hi, b)
    rl, rs, rd = S.policy_loss(k.nll, k.old, k.ref, k.target, k.starts, k.adv, k.token_adv, lo, hi, b, mean, k.dloss)
    tl, tk, td = np.zeros(k.S), np.zeros(k.S), np.zeros(k.T)
    with np.errstate(over="ignore"):
        for s, (x, y) in enumerate(S.tokens_of(k.starts, k.T)):
            at = x + np.flatnonzero(k.target[x:y] >= 0)
            if len(at) == 0:
                continue
            w = 1.0 / len(at) if mean else 1.0
            A = np.abs(k.adv[at]) if k.token_adv else np.abs(k.adv[s])
            q = k.old[at] - k.nll[at]
            r = np.exp(q)
            er = 2.0 ** -22 + U * np.abs(q) + 2 * U                     # of r and its product with A
            each, kl, slope = A * np.maximum(r, 1) * 1.3 * (er + 3 * U), 0.0, A * r * er
            if k.ref is not None:
                d = k.nll[at] - k.ref[at]
                v, e = np.expm1(d) - d, np.abs(np.expm1(d))
                far = np.abs(d) >= 0.499
                # the series: d rounded (twice in d^2), seven steps and two products; the difference: expf, then two roundings.
                # d is a difference rounded to fp32, off by up to 2^-24 |d|, which moves e^d by 2^-24 |d| e^d
                moved = U * np.abs(d) * np.exp(d)
                kl = np.where(far, 2.0 ** -22 * (np.exp(d) + np.abs(d) + 1) + moved, 12 * U * v) + 3 * U * v
                slope = slope + b * (np.where(far, 2.0 ** -22 * (np.exp(d) + 1) + moved, 8 * U * e) + 3 * U * e)
            tl[s] = w * (each + b * kl).sum() + U * abs(rl[s])
            tk[s] = w * np.sum(kl) + U * rs[s, 2]
            td[at] = np.abs(k.dloss[s]) * w * slope + 4 * U * np.abs(rd[at])
    close("loss", loss, rl, tl)
    assert np.array_equal(f64(stats)[:, :2], rs[:, :2])
    close("kl", stats[:, 2], rs[:, 2], tk)
    if grad:
        close("dnll", dnll, rd, td)
    return out


def run_pair(c, k, t, mean, grad=True, beta=0.3, margin=0.2, e=0.1):
    P = k.S // 2
    out = empty(P), empty(P, 2), empty(k.T) if grad else None
    c.preference_loss(t["nll"], t["ref"], t["target"], t["starts"], beta, margin, e, mean, out[0], out[1], t["dpair"] if grad else None, out[2])
    return out


def check_pair(c, k, mean, grad=True, beta=0.3, margin=0.2, e=0.1, t=None):
    out = loss, reward, dnll = run_pair(c, k, t or k.tensors(), mean, grad, beta, margin, e)
    rl, rr, rd = S.preference_loss(k.nll, k.ref, k.target, k.starts, beta, margin, e, mean, k.dpair)
    tr, td, spans = np.zeros_like(rr), 4 * U * np.abs(rd), S.tokens_of(k.starts, k.T)
    for p, j in itertools.product(range(k.S // 2), (0, 1)):
        x, y = spans[2 * p + j]
        at = x + np.flatnonzero(k.target[x:y] >= 0)
        n = len(at)
        each = np.abs((0 if k.ref is None else k.ref[at]) - k.nll[at])
        tr[p, j] = abs(beta) * 4 * U * each.sum() / (max(n, 1) if mean else 1)     # a difference and a sum of four
    tx = tr.sum(1)
    for p, j in itertools.product(range(k.S // 2), (0, 1)):                        # the slope of a sigmoid is 1/4 at most
        x, y = spans[2 * p + j]
        n = max((k.target[x:y] >= 0).sum(), 1) if mean else 1
        td[x:y] += np.where(k.target[x:y] >= 0, abs(beta) / n * abs(k.dpair[p]) * tx[p] / 4, 0)
    close("reward", reward, rr, tr + U * np.abs(rr))
    close("loss", loss, rl, tx + U * np.abs(rl))
    if grad:
        close("dnll", dnll, rd, td)
    return out


SHAPES = [  # T, S, kind
    (1, 2, "all"), (1, 2, "ones"), (2, 2, "ones"), (3, 4, "ones"), (127, 2, "even"), (128, 4, "even"), (129, 6, "empties"), (300, 300, "ones"), (600, 600, "ones"), (2048, 510, "even"), (2048, 512, "empties"), (2049, 20, "even"), (32768, 6, "even"), (32769, 100, "even"),
    (1000, 8, "even"), (4095, 40, "even"), (4096, 2, "all"), (4096, 32, "steps"), (4097, 10, "even"), (5000, 4000, "even"), (20000, 3000, "empties"),
    (33333, 2, "even"), (65536, 64, "steps"), (100001, 12, "even"), (700001, 6, "even"), (700001, 2, "all"), (1300000, 300, "empties"),
    (30000, 20000, "even"), (700001, 60000, "even"), (50000, 12000, "empties"), (1500, 400, "even"),
]


@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("T,S_,kind", SHAPES)
def test_policy(ctx, T, S_, kind, mean):
    check_policy(ctx, Case(T, S_, kind, ref=T % 2 == 1 or T > 50000, token_adv=T % 3 == 0), mean)


@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("T,S_,kind", SHAPES)
def test_preference(ctx, T, S_, kind, mean):
    check_pair(ctx, Case(T, S_, kind, ref=T % 3 != 0), mean)


@pytest.mark.parametrize("T,S_", [(700, 6), (9000, 30)])
@pytest.mark.parametrize("ref,token_adv,mean", list(itertools.product([False, True], repeat=3)))
def test_policy_variants(ctx, T, S_, ref, token_adv, mean):
    k = Case(T, S_, ref=ref, token_adv=token_adv)
    with_grad = check_policy(ctx, k, mean)
    without = check_policy(ctx, k, mean, grad=False)
    assert torch.equal(with_grad[0], without[0]) and torch.equal(with_grad[1], without[1])


@pytest.mark.parametrize("T,S_", [(700, 6), (9000, 30)])
@pytest.mark.parametrize("ref,mean,e", list(itertools.product([False, True], [False, True], [0.0, 0.5, 1.0])))
def test_preference_variants(ctx, T, S_, ref, mean, e):
    k = Case(T, S_, ref=ref)
    with_grad = check_pair(ctx, k, mean, e=e, beta=0.1 if e else -0.2)
    without = check_pair(ctx, k, mean, grad=False, e=e, beta=0.1 if e else -0.2)
    assert torch.equal(with_grad[0], without[0]) and torch.equal(with_grad[1], without[1])


@pytest.mark.parametrize("lo,hi", [(0.0, 0.0), (1.0, float("inf")), (0.2, 0.28), (0.5, 3.0)])
def test_ratios_next_to_the_borders(ctx, lo, hi):
    """Log ratios a few steps of fp32 around each border, and on it: which side decides between 0 and the whole slope."""
    k = Case(4096, 16)
    r = np.random.default_rng(5)
    with np.errstate(divide="ignore"):
        edge = np.array([v for v in (np.log1p(-lo), np.log1p(hi)) if np.isfinite(v)] or [0.0])
    k.nll = (np.floor(r.random(k.T) * 3) * 0.5).astype(np.float32).astype(np.float64)
    want = k.nll + edge[r.integers(0, len(edge), k.T)]
    k.old = want.astype(np.float32)
    for _ in range(3):
        step = r.integers(-1, 2, k.T)
        k.old = np.where(step == 0, k.old, np.nextafter(k.old, np.where(step > 0, np.float32(np.inf), np.float32(-np.inf)))).astype(np.float32)
    k.old = k.old.astype(np.float64)
    _, stats, _ = check_policy(ctx, k, False, lo=lo, hi=hi)
    assert np.isinf(hi) or 0 < stats[:, 1].sum() < stats[:, 0].sum()


@pytest.mark.parametrize("T", [500, 30000])
def test_small_and_large_divergences(ctx, T):
    """e^d - 1 - d from d of 1e-4, where the difference would be all rounding, to 80."""
    k = Case(T, 4)
    r = np.random.default_rng(1)
    d = np.exp(r.uniform(np.log(1e-4), np.log(80), T)) * np.where(r.random(T) < 0.5, -1, 1)
    k.nll = k.nll + 100
    k.ref = (k.nll - d).astype(np.float32).astype(np.float64)
    k.nll = k.nll.astype(np.float32).astype(np.float64)
    k.old = k.nll + 0.0
    check_policy(ctx, k, True)
    k.ref = np.where(np.abs(d) < 1, k.ref, k.nll)                       # the small ones alone
    check_policy(ctx, k, True)


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("T,S_", [(900, 12), (900, 200), (20000, 12), (20000, 3000), (50000, 12), (50000, 9000), (700001, 60)])
def test_advantages_that_no_token_takes_may_be_anything(ctx, T, S_, value):
    """A group of one answer normalised by its deviation has 0/0 for an advantage; an answer of which no token counts has no part
    in anything.  At every way of adding up: one block, the cluster, many launches, with few and many ends in a step."""
    k = Case(T, S_, dead=0.3)
    for s in range(2, S_, 5):
        k.target[k.starts[s]:k.starts[s + 1]] = -100
        k.adv[s] = value
    each = Case(T, S_, token_adv=True, dead=0.3)
    each.adv[each.target < 0] = value
    for mean in (False, True):
        assert all(torch.isfinite(o).all() for c in (k, each) for o in check_policy(ctx, c, mean))


def give_advantages(k, values):
    """To single tokens, or to whole sequences; a quarter of the sequences and more stay as they are."""
    for i, v in enumerate(values):
        if k.token_adv:
            k.adv[(np.searchsorted(k.starts, np.arange(k.T), side="right") % 4 == i) & (np.arange(k.T) % 5 == 0)] = v
        else:
            k.adv[i + 1::9] = v


def same_where_not_finite(c, k, mean):
    """Losses, counts and gradients as the oracle has them, infinities and NaN in the same places; returns the oracle's."""
    loss, stats, dnll = (f64(o) for o in run_policy(c, k, k.tensors(), mean))
    with np.errstate(invalid="ignore", over="ignore"):
        rl, rs, rd = S.policy_loss(k.nll, k.old, k.ref, k.target, k.starts, k.adv, k.token_adv, 0.2, 0.3, 0.1, mean, k.dloss)
    assert np.array_equal(stats[:, :2], rs[:, :2]) and np.isfinite(stats).all()
    for got, ref in ((loss, rl), (dnll, rd)):
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        assert np.array_equal(np.where(np.isinf(got), got, 0), np.where(np.isinf(ref), ref, 0))
    return rl, rs, rd


WAYS = [(900, 12), (900, 200), (20000, 12), (20000, 3000), (50000, 12), (50000, 9000), (700001, 60)]     # T, S: each way of adding up


@pytest.mark.parametrize("T,S_", WAYS)
@pytest.mark.parametrize("mean,token_adv", list(itertools.product([False, True], repeat=2)))
def test_infinite_advantages(ctx, T, S_, mean, token_adv):
    """Infinities where the formula has them and nowhere else, and no NaN: a clipped token's gradient is 0 under an infinite
    advantage too."""
    k = Case(T, S_, token_adv=token_adv, dead=0.3)
    give_advantages(k, (np.inf, -np.inf))
    rl, rs, rd = same_where_not_finite(ctx, k, mean)
    live = (k.target >= 0) & np.isinf(k.adv if token_adv else k.adv[np.clip(np.searchsorted(k.starts, np.arange(T), side="right") - 1, 0, S_ - 1)])
    assert np.isinf(rl).any() and np.isfinite(rl).any() and np.isinf(rd).any() and not np.isnan(rd).any() and np.isfinite(rd[live]).any()


@pytest.mark.parametrize("T,S_", WAYS)
@pytest.mark.parametrize("mean,token_adv", list(itertools.product([False, True], repeat=2)))
def test_nan_advantages(ctx, T, S_, mean, token_adv):
    """NaN stays with the tokens whose advantage it is, and their sequences; next to it no term is the larger, so no token of
    theirs counts as clipped."""
    k = Case(T, S_, token_adv=token_adv, dead=0.3)
    give_advantages(k, (np.nan,))
    rl, rs, rd = same_where_not_finite(ctx, k, mean)
    assert np.isnan(rl).any() and np.isfinite(rl).any() and np.isnan(rd).any() and not np.isinf(rd).any()


@pytest.mark.parametrize("T,S_", WAYS)
@pytest.mark.parametrize("mean,token_adv", list(itertools.product([False, True], repeat=2)))
def test_log_ratios_of_any_size(ctx, T, S_, mean, token_adv):
    """Finite log ratios from 1e7 to the largest fp32, as masked log probabilities of -1e9 or -1e30 make them: ratios of infinity
    and 0, never below 0."""
    k, r = Case(T, S_, token_adv=token_adv, dead=0.3), np.random.default_rng(T)
    f = lambda a: a.astype(np.float32).astype(np.float64)
    far = (np.searchsorted(k.starts, np.arange(T), side="right") % 3 == 0) & (r.random(T) < 0.1)
    x = np.where(r.random(T) < 0.5, np.exp(r.uniform(np.log(1e7), np.log(1e11), T)), r.choice([1e8, 1e9, 1e10, 1e30, 3e38, np.finfo(np.float32).max], T))
    up = far & (r.random(T) < 0.7)
    k.old, k.nll = f(np.where(up, x, k.old)), f(np.where(far & ~up, x, k.nll))
    k.old, k.ref = np.where(far & ~up, 1.0, k.old), np.where(far & ~up, k.nll, k.ref)
    rl, rs, rd = same_where_not_finite(ctx, k, mean)
    assert np.isposinf(rl).any() and not np.isneginf(rl).any() and np.isfinite(rl).any() and np.isinf(rd).any()
    assert (run_policy(ctx, k, k.tensors(), mean)[2][torch.from_numpy(far & ~up).to(DEV)] == 0).all()


@pytest.mark.parametrize("T", [310_000, 700_003, 1_300_001])
@pytest.mark.parametrize("ref,token_adv", [(False, False), (False, True), (True, True)])
def test_several_steps_a_warp(ctx, T, ref, token_adv):
    """Ranges of several steps, which go round the ring in shared memory: every set of tensors in it, targets on 16 bytes and on 8."""
    k = Case(T, 46, "empties" if T == 700_003 else "even", ref=ref, token_adv=token_adv)
    t = k.tensors()
    shifted = {**t, "target": inside(t["target"])}
    for mean in (False, True):
        for check, run in ((check_policy, run_policy), (check_pair, run_pair)):
            assert all(torch.equal(a, b) for a, b in zip(check(ctx, k, mean, t=t), run(ctx, k, shifted, mean)))


@pytest.mark.parametrize("T,S_", [(900, 6), (50000, 20)])
def test_tokens_that_do_not_count_may_hold_anything(ctx, T, S_):
    k = Case(T, S_, dead=0.5)
    a, b = k.starts[0], k.starts[-1]
    k.starts[0], k.starts[-1] = a + 3, max(b - 5, k.starts[-2])          # some tokens before and behind all sequences
    k.target[k.starts[2]:k.starts[3]] = -1                               # a sequence of which no token counts
    clean_policy, clean_pair = check_policy(ctx, k, True), check_pair(ctx, k, True)
    dead = k.target < 0
    dead[: k.starts[0]] = dead[k.starts[-1]:] = True
    t = k.tensors()
    for name, v in (("nll", np.nan), ("old", np.inf), ("ref", -np.inf)):
        t[name][torch.from_numpy(dead).to(DEV)] = v
    for got, want in zip((*run_policy(ctx, k, t, True), *run_pair(ctx, k, t, True)), (*clean_policy, *clean_pair)):
        assert torch.equal(got, want) and torch.isfinite(got).all()
    assert (clean_policy[2][torch.from_numpy(dead).to(DEV)] == 0).all() and (clean_policy[1][2] == 0).all() and clean_policy[0][2] == 0


@pytest.mark.parametrize("T", [300, 20000])
def test_no_token_counts(ctx, T):
    k = Case(T, 6, dead=1.0)
    loss, stats, dnll = check_policy(ctx, k, True)
    assert (loss == 0).all() and (stats == 0).all() and (dnll == 0).all()
    loss, reward, dnll = check_pair(ctx, k, True)
    assert (reward == 0).all() and (dnll == 0).all()


@pytest.mark.parametrize("T", [300, 20000])
def test_nan_stays_in_its_sequence(ctx, T):
    k = Case(T, 6, dead=0.0)
    k.starts = np.linspace(0, T, 7).astype(np.int64)
    t = k.tensors()
    t["nll"][int(k.starts[2]) + 1] = float("nan")
    loss, _, dnll = run_policy(ctx, k, t, True)
    bad = torch.arange(6, device=DEV) == 2
    assert loss[bad].isnan().all() and torch.isfinite(loss[~bad]).all() and int(dnll.isnan().sum()) == 1
    loss, _, dnll = run_pair(ctx, k, t, True)
    assert loss[1].isnan() and torch.isfinite(loss[[0, 2]]).all() and torch.isfinite(dnll[: int(k.starts[2])]).all()


def test_sure_pairs(ctx):
    """Log ratios of thousands either way: losses of 0 and of their size, not NaN."""
    k = Case(8192, 4, dead=0.0)
    k.starts = np.array([0, 2048, 4096, 6144, 8192])
    k.ref = k.nll + np.where(np.arange(8192) // 2048 % 3 == 0, 1.0, -1.0)
    k.ref = k.ref.astype(np.float32).astype(np.float64)
    loss, _, dnll = check_pair(ctx, k, False, beta=1.0, margin=0.0, e=0.0)
    assert loss[0] == 0 and loss[1] > 4000 and torch.isfinite(dnll).all() and (dnll[:4096] == 0).all() and (dnll[4096:] != 0).all()


def test_offsets_beyond_32_bits(ctx):
    """1.1 G tokens: 4.4 GB a tensor, 8.8 GB of targets.  The last sequences give what they give alone."""
    T, m = 1_100_000_000, 5001
    g = torch.Generator(device=DEV).manual_seed(1)
    nll = torch.empty(T, device=DEV).exponential_(generator=g)
    old, ref, dnll = nll * 1.01, nll * 0.98, torch.empty(T, device=DEV)
    target = torch.ones(T, dtype=torch.int64, device=DEV)
    target[-m::3] = -1
    starts = torch.tensor([7, 1000, 900_000_000, T - m, T - m + 2000, T - 1, T - 1], device=DEV)
    adv, dloss, few = torch.tensor([1.0, -1.0, 0.5, 2.0, -0.5, 1.0], device=DEV), torch.ones(6, device=DEV), slice(3, 6)
    loss, pair, stats, reward = empty(6), empty(3), empty(6, 3), empty(3, 2)
    own = lambda t: t[T - m:].clone()
    small = [own(t) for t in (nll, old, ref, target)]
    l2, s2, d2 = empty(4), empty(4, 3), empty(m)
    at = torch.cat((torch.zeros(2, dtype=torch.int64, device=DEV), starts[4:] - (T - m)))
    args = (0.2, 0.3, 0.1, True)
    ctx.policy_loss(nll, old, ref, target, starts, adv, False, *args, loss, stats, dloss, dnll)
    ctx.policy_loss(*small, at, adv[2:].clone(), False, *args, l2, s2, dloss[:4], d2)
    assert torch.equal(stats[few][:, :2], s2[1:, :2]) and torch.allclose(loss[few], l2[1:], rtol=1e-5) and torch.allclose(stats[few], s2[1:], rtol=1e-5)
    assert torch.equal(dnll[T - m:], d2) and torch.isfinite(loss).all() and abs(int(stats[2, 0]) - (T - m - 900_000_000)) <= 8      # half a step of fp32 there
    assert (dnll[:7] == 0).all() and (dnll[7:T - m] != 0).any()
    ctx.preference_loss(nll, ref, target, starts, 0.1, 0.0, 0.0, True, pair, reward, dloss[:3], dnll)
    R = (small[2].double() - small[0].double()) * (small[3] >= 0)
    n = (small[3][2000:m - 1] >= 0).sum()
    assert reward[2, 0].item() == pytest.approx(0.1 * (R[2000:m - 1].sum() / n).item(), rel=1e-4, abs=1e-7) and reward[2, 1] == 0
    assert (dnll[T - m + 2000:T - 1][small[3][2000:m - 1] < 0] == 0).all() and (dnll[T - m + 2000:T - 1][small[3][2000:m - 1] >= 0] != 0).all()


def test_bad_starts_are_reported_and_harmless():
    r = np.random.default_rng(2)
    for T in (300, 30000):
        for starts in ([5, 100, 90, 250, 200], [-7, 10, 2**40, 20, T + 1], r.integers(-2 * T, 2 * T, 5), r.integers(-2**62, 2**62, 5)):
            c = binding.MhcLite(2, 64, 0)                                # a context of its own: the report stays
            k = Case(T, 4)
            k.starts = np.array(starts)
            t = k.tensors()
            run_policy(c, k, t, True), run_pair(c, k, t, False)
            with pytest.raises(binding.MhcLiteError) as e:
                c.device_status()
            assert e.value.status == binding.ERR_INDEX
    c = binding.MhcLite(2, 64, 0)                                        # many of them, so that the search runs through several rounds
    k = Case(100000, 40000)
    k.starts = r.integers(-10, 110000, 40001)
    run_policy(c, k, k.tensors(), True), run_pair(c, k, k.tensors(), True)
    with pytest.raises(binding.MhcLiteError):
        c.device_status()


@pytest.mark.parametrize("T,S_", [(100, 600), (100, 40000), (40000, 90000)])
def test_far_more_sequences_than_tokens(ctx, T, S_):
    k = Case(T, S_, "even")
    check_policy(ctx, k, True), check_pair(ctx, k, False)


@pytest.mark.parametrize("T", [300, 20000, 50000])
def test_impossible_tokens(ctx, T):
    """A token of probability 0 under the model, or under the one that sampled it: infinities where the formula has them."""
    k = Case(T, 6, dead=0.0, ref=False)
    k.starts = np.linspace(0, T, 7).astype(np.int64)
    k.adv = np.array([1.0, 1.0, -1.0, -1.0, 1.0, -1.0])
    a = [int(v) + 3 for v in k.starts[:4]]
    k.nll[[a[0], a[2]]], k.old[[a[1], a[3]]] = np.inf, np.inf          # ratios of 0, and infinite ones
    loss, stats, dnll = run_policy(ctx, k, k.tensors(), False)
    with np.errstate(invalid="ignore", over="ignore"):
        rl, rs, rd = S.policy_loss(k.nll, k.old, None, k.target, k.starts, k.adv, False, 0.2, 0.3, 0.0, False, k.dloss)
    assert np.array_equal(f64(stats)[:, 1], rs[:, 1]) and np.isinf(rl[3]) and np.isfinite(np.delete(rl, 3)).all()
    assert np.array_equal(np.isinf(f64(loss)), np.isinf(rl)) and not np.isnan(f64(loss)).any()
    for i in a[:3]:
        assert rd[i] == 0 and dnll[i] == 0
    k.ref = np.where(np.isinf(k.nll), 1.0, k.nll)                      # the divergence of such a token is infinite
    k.nll[a[2]], k.old[[a[1], a[3]]] = 1.0, 1.0
    loss, stats, _ = run_policy(ctx, k, k.tensors(), True)
    assert torch.isposinf(loss[0]) and torch.isposinf(stats[0, 2]) and torch.isfinite(loss[1:]).all()


@pytest.mark.parametrize("T", [1500, 9000, 60000])
@pytest.mark.parametrize("token_adv", [False, True])
def test_short_sequences_between_long_ones(ctx, T, token_adv):
    """Runs of sequences of no, one and a few tokens, hundreds of empty ones at one place, long ones and gaps between: every way
    of adding up a step, next to each other."""
    k, r = Case(T, 2, token_adv=token_adv, dead=0.2), np.random.default_rng(T)
    at, starts = 5, []
    while at < T:
        kind = r.integers(0, 5)
        for _ in range([40, 300, 1, 3, 25][kind]):
            starts.append(at)
            at += int([r.integers(0, 4), 0, r.integers(100, 1000), r.integers(20, 60), r.integers(1, 12)][kind])
    starts = np.minimum(np.array(starts + [T - 2]), T - 2)
    k.starts = starts[: len(starts) // 2 * 2 - 1]                       # an even number of sequences
    k.S = len(k.starts) - 1
    k.dloss = r.normal(size=k.S).astype(np.float32).astype(np.float64)
    k.dpair = k.dloss[: k.S // 2]
    if not token_adv:
        k.adv = r.normal(size=k.S).astype(np.float32).astype(np.float64)
    for mean in (False, True):
        check_policy(ctx, k, mean), check_pair(ctx, k, mean)


def test_no_tokens_and_no_sequences(ctx):
    for n in (4, 3000, 40000):
        k = Case(0, n)
        k.starts[:] = 0
        loss, stats, _ = check_policy(ctx, k, True)
        assert (loss == 0).all() and (stats == 0).all()
        loss, reward, _ = check_pair(ctx, k, True, margin=0.5, e=0.0)
        assert (reward == 0).all() and torch.allclose(loss, torch.full_like(loss, float(np.log1p(np.exp(0.5)))))
    k = Case(50, 0)
    k.starts = np.array([0])
    t, before = k.tensors(), ctx.kernel_launches()
    assert (run_policy(ctx, k, t, True)[2] == 0).all() and (run_pair(ctx, k, t, True)[2] == 0).all()
    assert ctx.kernel_launches() == before


@pytest.mark.parametrize("n", [1, 4, 510, 512, 40000])
def test_no_tokens_and_none_of_their_tensors(ctx, n):
    """Through the C entries, which take NULL for what no token asks for: one block, the cluster and the launches of many."""
    lib, ws = ctx.lib, torch.empty(max(1, ctx.lib.mhclite_policy_scratch_bytes(0, n)), dtype=torch.uint8, device=DEV)
    starts, loss, stats, reward = torch.zeros(n + 1, dtype=torch.int64, device=DEV), empty(n), empty(n, 3), empty(n // 2, 2)
    torch.cuda.synchronize()
    for each in (0, 1):
        for ptr in (loss, stats):
            ptr.fill_(float("nan"))
        assert lib.mhclite_policy_loss(ctx._h, 0, n, None, None, None, None, starts.data_ptr(), None, each, 0.2, 0.2, 0.1, 1, None, loss.data_ptr(),
                                       stats.data_ptr(), None, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == binding.OK
        assert (loss == 0).all() and (stats == 0).all()
    if n > 1:
        assert lib.mhclite_preference_loss(ctx._h, 0, n // 2, None, None, None, starts.data_ptr(), 0.1, 0.0, 0.0, 1, None, loss.data_ptr(),
                                           reward.data_ptr(), None, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == binding.OK
        assert (reward == 0).all() and torch.allclose(loss[: n // 2], torch.full_like(loss[: n // 2], float(np.log(2.0))))


def test_refusals(ctx):
    k = Case(100, 4)
    t = k.tensors()
    bad, nan, inf = binding.MhcLiteError, float("nan"), float("inf")
    for kw in ({"lo": -0.1}, {"lo": 1.1}, {"lo": nan}, {"hi": -0.1}, {"hi": nan}, {"b": nan}, {"b": inf}):
        with pytest.raises(bad):
            run_policy(ctx, k, t, True, **kw)
    for kw in ({"beta": nan}, {"beta": inf}, {"margin": nan}, {"e": -0.1}, {"e": 1.1}, {"e": nan}):
        with pytest.raises(bad):
            run_pair(ctx, k, t, True, **kw)
    for name, v in (("nll", t["nll"][:50]), ("old", t["old"].double()), ("ref", t["ref"].to(BF)), ("target", t["target"].int()), ("starts", t["starts"][:4]),
                    ("starts", t["starts"].float()), ("adv", t["nll"]), ("dloss", t["dloss"][:3]), ("nll", t["nll"].cpu()),
                    ("nll", torch.zeros(100, 2, device=DEV)[:, 0])):
        with pytest.raises(ValueError):
            run_policy(ctx, k, {**t, name: v}, True)
        if name not in ("old", "adv", "dloss"):
            with pytest.raises(ValueError):
                run_pair(ctx, k, {**t, name: v}, True)
    loss, stats, reward, dnll = empty(4), empty(4, 3), empty(2, 2), empty(100)
    head = (t["nll"], t["old"], t["ref"], t["target"], t["starts"], t["adv"], False, 0.2, 0.2, 0.1, True)
    for tail in ((loss, stats, t["dloss"], None), (loss, stats, None, dnll)):
        with pytest.raises(ValueError):
            ctx.policy_loss(*head, *tail)
    for out in (t["nll"], t["old"], t["ref"]):
        with pytest.raises(bad):
            ctx.policy_loss(*head, loss, stats, t["dloss"], out)         # the gradient in place of an input
    for out in (t["adv"], t["dloss"]):
        with pytest.raises(bad):
            ctx.policy_loss(*head, out, stats, t["dloss"], dnll)
    with pytest.raises(bad):
        ctx.preference_loss(t["nll"], t["ref"], t["target"], t["starts"], 0.1, 0.0, 0.0, False, loss[:2], reward, t["dpair"], t["ref"])
    with pytest.raises(bad):
        run_policy(ctx, k, {**t, "nll": torch.zeros(101, device=DEV)[1:]}, True)      # not on 16 bytes
    big = Case(5000, 4)
    b, need = big.tensors(), ctx.lib.mhclite_policy_scratch_bytes(5000, 4)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    args = [b[n].data_ptr() for n in ("nll", "old", "ref", "target", "starts", "adv")]
    assert ctx.lib.mhclite_policy_loss(ctx._h, 5000, 4, *args, 0, 0.2, 0.2, 0.1, 1, None, loss.data_ptr(), stats.data_ptr(), None, ws.data_ptr(),
                                       need - 1, None) == binding.ERR_WORKSPACE
    check_policy(ctx, k, True)                                           # a refused call leaves the context usable


def test_losses_and_statistics_in_place_of_token_losses_are_refused(ctx):
    k = Case(60, 60, "ones")                                             # as many sequences as tokens, so that the shapes fit
    t, loss, stats, reward = k.tensors(), empty(60), empty(60, 3), empty(30, 2)
    tail = (t["target"], t["starts"], t["adv"], False, 0.2, 0.2, 0.1, True)
    for out in (t["nll"], t["old"], t["ref"]):
        with pytest.raises(binding.MhcLiteError, match="alias"):
            ctx.policy_loss(t["nll"], t["old"], t["ref"], *tail, out, stats)
    long = torch.zeros(180, device=DEV)                                  # 180 floats: statistics, or the first tokens' losses
    for i in range(3):
        with pytest.raises(binding.MhcLiteError, match="alias"):
            ctx.policy_loss(*(long[:60] if j == i else t[n] for j, n in enumerate(("nll", "old", "ref"))), *tail, loss, long.view(60, 3))
    for out in (t["nll"][:30], t["ref"][:30]):
        with pytest.raises(binding.MhcLiteError, match="alias"):
            ctx.preference_loss(t["nll"], t["ref"], t["target"], t["starts"], 0.1, 0.0, 0.0, False, out, reward)
    for out in (t["nll"].view(30, 2), t["ref"].view(30, 2)):
        with pytest.raises(binding.MhcLiteError, match="alias"):
            ctx.preference_loss(t["nll"], t["ref"], t["target"], t["starts"], 0.1, 0.0, 0.0, False, loss[:30], out)
    check_policy(ctx, k, True), check_pair(ctx, k, True)


def inside(t):
    """The same values in a view 16 bytes (one element, for int64: 8) into a buffer: the least alignment the calls allow."""
    if t is None:
        return None
    k = max(1, 16 // t.element_size()) if t.dtype != torch.int64 else 1
    v = torch.empty(t.numel() + 2 * k, dtype=t.dtype, device=DEV)[k:k + t.numel()].view(t.shape)
    assert v.data_ptr() % 32 in (8, 16)
    return v.copy_(t)


@pytest.mark.parametrize("T,S_", [(777, 6), (30001, 14)])
def test_inner_views(ctx, T, S_):
    k = Case(T, S_, token_adv=True)
    t = {n: inside(v) for n, v in k.tensors().items()}
    for mean in (False, True):
        for got, want in zip((*check_policy(ctx, k, mean, t=t), *check_pair(ctx, k, mean, t=t)), (*run_policy(ctx, k, k.tensors(), mean), *run_pair(ctx, k, k.tensors(), mean))):
            assert torch.equal(got, want)
    loss, stats, dnll = inside(empty(S_)), inside(empty(S_, 3)), inside(empty(T + 1))[:T]
    ctx.policy_loss(t["nll"], t["old"], t["ref"], t["target"], t["starts"], t["adv"], True, 0.2, 0.3, 0.1, True, loss, stats, t["dloss"], dnll)
    want = run_policy(ctx, k, t, True)
    assert torch.equal(loss, want[0]) and torch.equal(stats, want[1]) and torch.equal(dnll, want[2])


@pytest.mark.parametrize("T", [1001, 5001, 700001])
def test_rows_behind_the_last_token_stay(ctx, T):
    k = Case(T, 6)
    t, room = k.tensors(), torch.full((T + 8,), 7.0, device=DEV)
    for f in (lambda d: ctx.policy_loss(t["nll"], t["old"], t["ref"], t["target"], t["starts"], t["adv"], False, 0.2, 0.3, 0.1, True, empty(6), empty(6, 3), t["dloss"], d),
              lambda d: ctx.preference_loss(t["nll"], t["ref"], t["target"], t["starts"], 0.1, 0.0, 0.0, False, empty(3), empty(3, 2), t["dpair"], d)):
        f(room[:T])
        assert (room[T:] == 7).all() and torch.isfinite(room).all()


def test_two_streams_at_once_and_bitwise_repeats(ctx):
    ks = [Case(2000, 12), Case(20001, 30), Case(200001, 40)]
    ts = [k.tensors() for k in ks]
    torch.cuda.synchronize()
    outs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams * 3:
        with torch.cuda.stream(s):
            outs.append([o for k, t in zip(ks, ts) for o in (*run_policy(ctx, k, t, True), *run_pair(ctx, k, t, True))])
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))


def test_captured_and_replayed_with_new_inputs(ctx):
    """Two graphs, each with scratch of its own; between replays the tokens, the masks and the starts change."""
    ks = [Case(2000, 12), Case(20001, 30), Case(50001, 40)]
    ts = [k.tensors() for k in ks]
    step = lambda: [o for k, t in zip(ks, ts) for m in (False, True) for o in (*run_policy(ctx, k, t, m), *run_pair(ctx, k, t, m))]
    side, graphs = torch.cuda.Stream(), []
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            out = step()
        graphs.append((gr, out))
    for i in range(3):
        for k, t in zip(ks, ts):
            new = Case(k.T, k.S, ("even", "empties", "steps")[i], dead=0.2 * i, seed=50 + i).tensors()
            for n in t:
                t[n].copy_(new[n])
        torch.cuda.synchronize()
        for gr, _ in graphs:
            gr.replay()
        torch.cuda.synchronize()
        want = step()
        for _, got in graphs:
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_inputs_that_another_stream_writes(ctx):
    """A kernel that may start beside the one before it still waits for what its stream waits for."""
    k, side = Case(30000, 8), torch.cuda.Stream()
    t, new = k.tensors(), k.tensors()
    want, done = [o.clone() for o in (*run_policy(ctx, k, t, True), *run_pair(ctx, k, t, True))], torch.cuda.Event()
    torch.cuda.synchronize()
    for _ in range(3):
        t["nll"].zero_()
        t["target"].fill_(-1)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(5_000_000)
            t["nll"].copy_(new["nll"])
            t["target"].copy_(new["target"])
            done.record()
        run_policy(ctx, k, new, True)                                    # the kernel before, which lets the next one begin
        torch.cuda.current_stream().wait_event(done)
        got = (*run_policy(ctx, k, t, True), *run_pair(ctx, k, t, True))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


# ---- model steps that end in these losses ---------------------------------------------------------------------------------
def test_the_last_step_of_a_model_against_the_oracle():
    """From the token losses that model_fwd leaves, policy_loss and preference_loss are the oracle's at the tolerances of fp32, and
    so are the gradients that model_bwd takes; the token losses are those of a plain restatement of the head on the activations
    that the library left."""
    n, C, T, V = 4, 64, 150, 300
    c, r = binding.MhcLite(n, C, 0), np.random.default_rng(3)
    mk = lambda *s, std=1.0, mean=0.0: (r.normal(size=s) * std + mean).astype(np.float32)
    Ps = [L.LayerParams(mk(n * C, 32, std=0.02), mk(32, std=0.1), np.full(3, 0.5, np.float32), mk(n * C, std=0.1, mean=1.0), DEV)]
    Bs = [L.LayerBuffers(c, T)]
    M = L.ModelEnds(c, T, dev(mk(V, C, std=0.5)), 1.3, dev(mk(C, std=0.1, mean=1.0)), dev(mk(V, C, std=0.3), BF), 1.0)
    k = Case(T, 6)
    k.starts = np.array([0, 40, 40, 77, 120, 131, 148])
    target, ids = torch.from_numpy(np.where(k.target < 0, -100, k.target % V)).to(DEV), dev(r.integers(0, V, T), torch.int64)
    k.target = target.cpu().numpy()
    nll = L.model_fwd(c, M, Ps, Bs, ids, target, lambda l, u: torch.tanh(u.float()).to(BF))
    # the logits from h as the library left it: 64 products, a sum over 300 words, a logarithm, each of fp32
    x = M.h.double() @ M.W.double().T
    want = (torch.logsumexp(x, 1) - x.gather(1, target.clamp(min=0)[:, None])[:, 0]) * (target >= 0)
    size = (M.h.double().abs() @ M.W.double().abs().T).amax(1)
    assert ((nll.double() - want).abs() <= 2 * (C / 16 + 4) * 2.0 ** -23 * size + (V / 256 + 64) * U + 2.0 ** -20 * (1 + want.abs())).all()
    # and h from the streams: their mean, its norm, both rounded to bf16 (2^-8 each, and as much of the norm's sum)
    top = M.x_top.double().mean(1)
    h = top * torch.rsqrt(top.pow(2).mean(1, keepdim=True) + 1e-6) * M.w.double()
    assert ((M.h.double() - h).abs() <= 3 * 2.0 ** -8 * (h.abs() + h.abs().mean())).all()
    k.nll = f64(nll)
    k.old, k.ref = ((k.nll + s * r.normal(size=T)).astype(np.float32).astype(np.float64) for s in (0.3, 0.4))
    t = {**k.tensors(), "target": target}
    A = L.Answers(t["starts"], T)
    L.policy_loss(c, A, nll, t["old"], t["ref"], target, t["adv"], t["dloss"], clip_low=0.2, clip_high=0.3, kl_weight=0.1)
    assert all(torch.equal(a, b) for a, b in zip((A.loss, A.stats, A.dnll), check_policy(c, k, True, t=t)))
    B = L.Answers(t["starts"], T, pairs=True)
    L.preference_loss(c, B, nll, t["ref"], target, t["dpair"], beta=0.3, margin=0.2, smoothing=0.1)
    assert all(torch.equal(a, b) for a, b in zip((B.loss, B.reward, B.dnll), check_pair(c, k, False, t=t)))
    c.device_status()


@pytest.mark.parametrize("kind", ["distill", "policy", "preference"])
def test_model_step_and_its_gradients_against_differences(kind):
    """ids -> loss through two mixing layers, and back.  The activations between the calls are bf16, so a difference of two
    losses is only as fine as their roundings: the loss is computed in fp64 by a plain restatement of the model without them,
    and differenced there along the library's own gradient."""
    n, C, T, V, layers, K = 4, 64, 120, 200, 2, 12
    c = binding.MhcLite(n, C, 0)
    r = np.random.default_rng(0)
    mk = lambda *s, std=1.0, mean=0.0: (r.normal(size=s) * std + mean).astype(np.float32)
    Ps = [L.LayerParams(mk(n * C, 32, std=0.02), mk(32, std=0.1), np.full(3, 0.5, np.float32), mk(n * C, std=0.1, mean=1.0), DEV) for _ in range(layers)]
    Bs = [L.LayerBuffers(c, T) for _ in range(layers)]
    E, wf = dev(mk(V, C, std=0.5)), dev(mk(C, std=0.1, mean=1.0))
    M = L.ModelEnds(c, T, E, 1.3, wf, dev(mk(V, C, std=0.3), BF), 1.0)
    ids, target = dev(r.integers(0, V, T), torch.int64), r.integers(0, V, T)
    target[::5] = -100
    target = dev(target, torch.int64)
    f, fb = (lambda l, u: torch.tanh(u.float()).to(BF)), (lambda l, u, dy: (dy.float() * (1 - torch.tanh(u.float()) ** 2)).to(BF))
    perms = torch.tensor(list(itertools.permutations(range(n))), device=DEV)

    def plain_logits(q):
        rms = lambda x: torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + 1e-6)
        x = (q["E"][ids] * 1.3)[:, None, :].expand(T, n, C)
        for P in Ps:
            xf = x.reshape(T, n * C)
            z = (xf * rms(xf) * P.gain.double()) @ P.W.double() * 0.5 + P.b.double()
            a, pre, post = torch.softmax(z[:, :24], 1), torch.sigmoid(z[:, 24:28]), 2 * torch.sigmoid(z[:, 28:])
            H = torch.zeros(T, n, n, dtype=torch.float64, device=DEV)
            for k in range(24):
                H[:, torch.arange(n), perms[k]] += a[:, k, None]
            x = torch.einsum("tij,tjc->tic", H, x) + post[:, :, None] * torch.tanh(torch.einsum("tj,tjc->tc", pre, x))[:, None, :]
        m = x.mean(1)
        return (m * rms(m) * q["wf"]) @ q["W"].T
    q = {"E": E.double(), "wf": wf.double(), "W": M.W.double()}
    starts = np.array([0, 30, 30, 62, 97, 110, 118])
    if kind == "distill":
        tid = np.stack([r.permutation(V)[:K] for _ in range(T)])
        tid[r.random((T, K)) < 0.2] = -1
        te = L.Teacher(dev(tid, torch.int64), dev(mk(T, K, std=2.0)), 2.0)
        w = r.random(T)
        loss = L.model_fwd(c, M, Ps, Bs, ids, None, f, teacher=te)
        L.model_bwd(c, M, Ps, Bs, ids, None, dev(w), fb, teacher=te)
        p, log_p, _ = S.teacher_weights(tid, f64(te.logits), 2.0, V)
        p, log_p, at = dev(p, torch.float64), dev(np.where(p > 0, log_p, 0), torch.float64), dev(np.maximum(tid, 0), torch.int64)

        def plain(q):
            return (p * (log_p - torch.log_softmax(plain_logits(q) / 2, 1).gather(1, at))).sum(1)
    else:
        A = L.Answers(dev(starts, torch.int64), T, kind == "preference")
        nll = L.model_fwd(c, M, Ps, Bs, ids, target, f)
        w = np.full(len(A.loss), 0.5)
        old, ref = (f64(nll) + 0.3 * r.normal(size=T)).astype(np.float32), (f64(nll) + 0.4 * r.normal(size=T)).astype(np.float32)
        seq = np.searchsorted(starts, np.arange(T), side="right") - 1
        live = (target.cpu().numpy() >= 0) & (seq < 6)
        one = dev(np.stack([(seq == s) & live for s in range(6)]), torch.float64)
        if kind == "policy":
            adv = mk(6)
            loss = L.policy_loss(c, A, nll, dev(old), dev(ref), target, dev(adv), dev(w), clip_low=0.2, clip_high=0.2, kl_weight=0.1)
            share = one / one.sum(1, keepdim=True).clamp(min=1)
            At, o, rf = dev(np.where(seq < 6, adv[np.minimum(seq, 5)], 0), torch.float64), dev(old, torch.float64), dev(ref, torch.float64)
            # which tokens are clipped is the library's choice at its own rounded losses: the restatement takes it as it is
            cut = np.exp(old.astype(np.float64) - f64(nll))
            cut = dev((np.where(f64(At) > 0, cut > 1.2, cut < 0.8)), torch.bool)

            def plain_from(x):
                d = x - rf
                return share @ (torch.where(cut, -At * torch.where(At > 0, 1.2, 0.8), -At * torch.exp(o - x)) + 0.1 * (torch.expm1(d) - d))
        else:
            loss = L.preference_loss(c, A, nll, dev(ref), target, dev(w), beta=0.3, smoothing=0.1)
            rf = dev(ref, torch.float64)

            def plain_from(x):
                R = 0.3 * (one @ (rf - x)).view(3, 2)
                y = R[:, 0] - R[:, 1]
                return -0.9 * torch.nn.functional.logsigmoid(y) - 0.1 * torch.nn.functional.logsigmoid(-y)
        L.model_bwd(c, M, Ps, Bs, ids, target, A.dnll, fb)

        def plain(q):
            x = plain_logits(q)
            return plain_from((torch.logsumexp(x, 1) - x.gather(1, target.clamp(min=0)[:, None])[:, 0]) * (target >= 0))
    torch.cuda.synchronize()
    c.device_status()
    ref_loss, weight = plain(q), dev(w, torch.float64)
    # about eight bf16 tensors lie between the ids and a logit: each moves a logit of size ~1 to 3 by some 2^-8.  A pair's loss
    # takes 0.3 of a sum over up to 35 tokens of them, independent in their signs: six times one token's
    scale = {"distill": 1.0, "policy": 2.0, "preference": 0.3 * 6 * 2}[kind]
    assert (loss.double() - ref_loss).abs().max() <= scale * 10 * 2.0 ** -8 * (3 + ref_loss.abs().max())
    for name, g in {"E": M.dE, "wf": M.dw, "W": M.dW}.items():
        d = g.double() / g.double().norm()
        h = 1e-4
        up, down = dict(q), dict(q)
        up[name], down[name] = q[name] + h * d, q[name] - h * d
        diff = (((plain(up) - plain(down)) * weight).sum() / (2 * h)).item()
        # along its own direction a gradient with relative error e (2-norm) differences to its norm within e: some
        # twenty bf16 roundings of half a step each on the longest way back
        assert diff == pytest.approx(g.double().norm().item(), rel=20 * 2.0 ** -8), name
