"""The fp64 oracle of the operators around the stack: published vectors of the generator, hand cases, and every gradient
against central differences."""
import numpy as np
import pytest

from oracle import stack_ends_oracle as S


@pytest.mark.parametrize("counter,key,words", [
    # known-answer vectors of Philox4x32-10 published with the generator
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_philox_known_answers(counter, key, words):
    assert tuple(S.philox4x32(counter, key)) == words


def test_keep_mask_share_and_prefix():
    m = S.keep_mask(20000, 0.3, 123456789012345, 7)
    # 20000 draws: six standard deviations of the share are 6 sqrt(0.21 / 20000) < 0.02
    assert abs(m.mean() - 0.7) < 0.02
    assert (S.keep_mask(77, 0.3, 123456789012345, 7) == m[:77]).all()          # a mask does not depend on the count
    assert (S.keep_mask(64, 0.0, 5, 0)).all()
    assert (S.keep_mask(512, 0.3, 123456789012345, 8) != m[:512]).any()


def test_embed_by_hand():
    E = np.arange(6.0).reshape(3, 2)
    x = S.embed_fwd(np.array([2, 0, 5, -1]), E, 2.0, 3)
    assert x.shape == (4, 3, 2) and (x[0] == [8, 10]).all() and (x[1] == [0, 2]).all() and (x[2:] == 0).all()
    g = np.ones((4, 3, 2))
    dE, mag = S.embed_bwd(np.array([2, 0, 2, -1]), g, 0.5, 3)
    assert (dE == [[1.5, 1.5], [0, 0], [3, 3]]).all() and (mag == dE).all()


def _diff(f, x, d, h=1e-5):
    """Central difference of the scalar f along d at x."""
    return (f(x + h * d) - f(x - h * d)) / (2 * h)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("p", [0.0, 0.4])
def test_block_gradients_against_differences(gated, p):
    r = np.random.default_rng(3)
    T, C, eps, s = 5, 16, 1e-6, 0.7
    o, w, dy = r.normal(size=(T, C)), 1 + 0.2 * r.normal(size=C), r.normal(size=(T, C))
    gate = r.normal(size=(T, C)) if gated else None
    keep, factor = (S.keep_mask(T * C, p, 11, 3).reshape(T, C), S.drop_factor(p)) if p else (None, 1.0)
    L = lambda o=o, g=gate, w=w, s=s: (dy * S.block_out_fwd(o, g, w, s, eps, keep, factor)[0]).sum()
    b = S.block_out_bwd(o, gate, w, s, eps, dy, keep, factor)
    # differences of step 1e-5 in fp64: truncation ~1e-10, rounding ~1e-11 / 1e-5 of the sum
    do, dw = r.normal(size=o.shape), r.normal(size=C)
    assert _diff(lambda x: L(o=x), o, do) == pytest.approx((b["d_o"] * do).sum(), rel=1e-6, abs=1e-7)
    assert _diff(lambda x: L(w=x), w, dw) == pytest.approx((b["dw"] * dw).sum(), rel=1e-6, abs=1e-7)
    assert _diff(lambda x: L(s=x), s, 1.0) == pytest.approx(b["dscale"], rel=1e-6, abs=1e-7)
    if gated:
        assert _diff(lambda x: L(g=x), gate, do) == pytest.approx((b["dgate"] * do).sum(), rel=1e-6, abs=1e-7)


def test_linear_ce_by_hand_and_differences():
    loss, lse = S.linear_ce_fwd(np.array([[1.0, 0.0]]), np.array([[0.0, 5.0], [np.log(3.0), 1.0]]), np.array([1]), 1.0)
    assert lse[0] == pytest.approx(np.log(4.0)) and loss[0] == pytest.approx(np.log(4.0 / 3.0))
    r = np.random.default_rng(5)
    T, C, V, scale = 6, 8, 11, 0.8
    h, W, d = r.normal(size=(T, C)), r.normal(size=(V, C)), r.normal(size=T)
    target = np.array([0, 10, -100, 3, 11, 5])                       # two rows without a target
    L = lambda h=h, W=W: (d * S.linear_ce_fwd(h, W, target, scale)[0]).sum()
    dh, dW, G = S.linear_ce_bwd(h, W, target, scale, d)
    eh, eW = r.normal(size=h.shape), r.normal(size=W.shape)
    assert _diff(lambda x: L(h=x), h, eh) == pytest.approx((dh * eh).sum(), rel=1e-6, abs=1e-7)
    assert _diff(lambda x: L(W=x), W, eW) == pytest.approx((dW * eW).sum(), rel=1e-6, abs=1e-7)
    assert (dh[[2, 4]] == 0).all() and (G[[2, 4]] == 0).all()
