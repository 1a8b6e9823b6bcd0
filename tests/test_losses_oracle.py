"""The fp64 oracle of the losses behind a first training: closed forms, hand cases, and every gradient against central
differences."""
import numpy as np
import pytest

from oracle import losses_oracle as S
from oracle import stack_ends_oracle as E


def _diff(f, x, d, h=1e-5):
    """Central difference of the scalar f along d at x."""
    return (f(x + h * d) - f(x - h * d)) / (2 * h)


def _rows(seed=0, T=6, C=8, V=20, K=4):
    r = np.random.default_rng(seed)
    ids = np.stack([r.permutation(V)[:K] for _ in range(T)])
    return r, r.normal(size=(T, C)), r.normal(size=(V, C)), ids, 2 * r.normal(size=(T, K))


def test_one_entry_is_cross_entropy():
    r, h, W, ids, z = _rows(K=1)
    loss, lse, logp = S.linear_distill_fwd(h, W, ids, z, 0.7, 1.0)
    ce, ref = E.linear_ce_fwd(h, W, ids[:, 0], 0.7)
    assert np.allclose(loss, ce, rtol=1e-12) and np.allclose(lse, ref, rtol=1e-12) and np.allclose(logp[:, 0], -ce, rtol=1e-12)
    dl = r.normal(size=6)
    a, b = S.linear_distill_bwd(h, W, ids, z, 0.7, 1.0, dl), E.linear_ce_bwd(h, W, ids[:, 0], 0.7, dl)
    assert np.allclose(a[0], b[0], rtol=1e-10, atol=1e-12) and np.allclose(a[1], b[1], rtol=1e-10, atol=1e-12)


def test_the_student_as_its_own_teacher():
    """All of the student's logits as the teacher's: no divergence, no gradient, at any temperature; a constant added to a
    row of the teacher changes nothing."""
    r, h, W, _, _ = _rows()
    ids = np.stack([r.permutation(20) for _ in range(6)])
    z = np.take_along_axis(0.7 * h @ W.T, ids, 1) + r.normal(size=(6, 1))
    for tau in (1.0, 3.0):
        loss, _, logp = S.linear_distill_fwd(h, W, ids, z, 0.7, tau)
        assert np.abs(loss).max() < 1e-12 and np.allclose(np.exp(logp).sum(1), 1)
        dh, dW, *_ = S.linear_distill_bwd(h, W, ids, z, 0.7, tau, np.ones(6))
        assert np.abs(dh).max() < 1e-12 and np.abs(dW).max() < 1e-12


def test_absent_entries_and_rows_count_for_nothing():
    r, h, W, ids, z = _rows()
    ids[1], ids[2, 1:], z[1] = -1, -1, np.nan
    z[2, 1:], z[3], ids[4, 2] = np.nan, -np.inf, 20
    h[1], h[3] = np.nan, np.inf
    dl = r.normal(size=6)
    loss, lse, logp = S.linear_distill_fwd(h, W, ids, z, 1.0, 2.0)
    dh, dW, *_ = S.linear_distill_bwd(h, W, ids, z, 1.0, 2.0, dl)
    for a in (loss, lse, logp, dh, dW):
        assert np.isfinite(a).all()
    assert (loss[[1, 3]] == 0).all() and (lse[[1, 3]] == 0).all() and (logp[[1, 3]] == 0).all() and (dh[[1, 3]] == 0).all()
    assert np.isclose(loss[2], -logp[2, 0]) and (logp[2, 1:] == 0).all() and logp[4, 2] == 0


def test_an_id_twice_has_both_weights():
    r, h, W, ids, z = _rows()
    twice, zt = np.concatenate((ids, ids[:, :1]), 1), np.concatenate((z, z[:, :1]), 1)
    once = z.copy()
    once[:, 0] += 2.0 * np.log(2.0)                      # at temperature 2: twice the weight
    dl = r.normal(size=6)
    a, b = S.linear_distill_bwd(h, W, twice, zt, 1.0, 2.0, dl), S.linear_distill_bwd(h, W, ids, once, 1.0, 2.0, dl)
    assert np.allclose(a[0], b[0]) and np.allclose(a[1], b[1])


@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_distill_gradients_against_differences(tau):
    r, h, W, ids, z = _rows(3)
    ids[0, 1] = ids[0, 2]
    ids[1, 3] = -1
    dl, d_h, d_W = r.normal(size=6), r.normal(size=h.shape), r.normal(size=W.shape)
    L = lambda h=h, W=W: (dl * S.linear_distill_fwd(h, W, ids, z, 0.6, tau)[0]).sum()
    dh, dW, *_ = S.linear_distill_bwd(h, W, ids, z, 0.6, tau, dl)
    assert _diff(lambda x: L(h=x), h, d_h) == pytest.approx((dh * d_h).sum(), rel=1e-6, abs=1e-7)
    assert _diff(lambda x: L(W=x), W, d_W) == pytest.approx((dW * d_W).sum(), rel=1e-6, abs=1e-7)


def _tokens(seed=0, T=40):
    r = np.random.default_rng(seed)
    nll = r.exponential(size=T) + 0.05
    target = r.integers(0, 9, T)
    target[r.random(T) < 0.2] = -1
    return r, nll, nll + 0.3 * r.normal(size=T), nll + 0.5 * r.normal(size=T), target, np.array([1, 9, 9, 10, 24, 31, 38])


def test_policy_by_hand():
    ln = np.log
    nll, old = np.array([1.0, 1.0, 1.0, 1.0]), np.array([1.0, 1.0 + ln(2), 1.0 - ln(2), 1.0 + ln(2)])
    one, at = np.zeros(4, dtype=int), np.array([0, 4])
    # ratios 1, 2, 1/2, 2 with advantages 1, 1, -1, -1 and borders 0.8, 1.2: the second and third are cut
    loss, stats, d = S.policy_loss(nll, old, None, one, at, np.array([1.0, 1.0, -1.0, -1.0]), True, 0.2, 0.2, 0.0, False, np.ones(1))
    assert loss[0] == pytest.approx(-1 - 1.2 + 0.8 + 2) and (stats[0] == [4, 2, 0]).all() and np.allclose(d, [1, 0, 0, -2])
    loss, stats, d = S.policy_loss(nll, nll, nll - ln(2), one, at, np.array([3.0]), False, 0.2, 0.2, 0.5, True, np.ones(1))
    assert loss[0] == pytest.approx(-3 + 0.5 * (1 - ln(2))) and stats[0, 2] == pytest.approx(1 - ln(2)) and np.allclose(d, (3 + 0.5) / 4)


@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("token_adv", [False, True])
@pytest.mark.parametrize("ref", [False, True])
def test_policy_gradient_against_differences(mean, token_adv, ref):
    r, nll, old, nll_ref, target, starts = _tokens(1)
    S_ = len(starts) - 1
    adv, dl, d = r.normal(size=40 if token_adv else S_), r.normal(size=S_), r.normal(size=40)
    f = lambda x: S.policy_loss(x, old, nll_ref if ref else None, target, starts, adv, token_adv, 0.2, 0.3, 0.1, mean, dl)
    loss, stats, dnll = f(nll)
    assert _diff(lambda x: (dl * f(x)[0]).sum(), nll, d, 1e-6) == pytest.approx((dnll * d).sum(), rel=1e-6, abs=1e-7)
    assert 0 < stats[:, 1].sum() < stats[:, 0].sum() and (dnll[target < 0] == 0).all() and dnll[0] == 0 and (dnll[38:] == 0).all()
    assert loss[1] == 0 and (stats[1] == 0).all()        # an empty sequence


def test_preference_by_hand():
    nll, ref = np.array([1.0, 2.0, 3.0]), np.array([1.5, 2.5, 2.0])
    loss, reward, d = S.preference_loss(nll, ref, np.zeros(3, dtype=int), np.array([0, 2, 3]), 0.5, 0.0, 0.0, False, np.ones(1))
    assert np.allclose(reward, [[0.5, -0.5]]) and loss[0] == pytest.approx(np.log1p(np.exp(-1.0)))
    g = 0.5 / (1 + np.exp(1.0))
    assert np.allclose(d, [g, g, -g])
    loss, reward, _ = S.preference_loss(nll, None, np.array([0, 0, -1]), np.array([0, 2, 3]), 1.0, 0.25, 0.1, True)
    assert np.allclose(reward, [[-1.5, 0.0]])            # the rejected sequence has no token that counts
    assert loss[0] == pytest.approx(0.9 * np.log1p(np.exp(1.75)) + 0.1 * np.log1p(np.exp(-1.75)))


@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("ref", [False, True])
def test_preference_gradient_against_differences(mean, ref):
    r, nll, _, nll_ref, target, starts = _tokens(2)
    dl, d = r.normal(size=3), r.normal(size=40)
    f = lambda x: S.preference_loss(x, nll_ref if ref else None, target, starts, 0.4, 0.2, 0.1, mean, dl)
    dnll = f(nll)[2]
    assert _diff(lambda x: (dl * f(x)[0]).sum(), nll, d) == pytest.approx((dnll * d).sum(), rel=1e-6, abs=1e-7)
    assert (dnll[target < 0] == 0).all() and dnll[0] == 0 and (dnll[38:] == 0).all() and np.abs(dnll).sum() > 0
