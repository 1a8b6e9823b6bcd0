"""Distillation from a teacher's top logits on the GPU against the fp64 oracle: losses, gradients, rows and entries that count
for nothing, refusals, streams and graphs.

Tolerances follow the arithmetic.  A bf16 output is off by at most half a step, 2^-8 of its value, on top of the fp32
arithmetic before it.  An fp32 sum is off by at most (number of additions on the longest path) x 2^-24 x the sum of its
terms' magnitudes."""
import numpy as np
import pytest
import torch

from oracle import losses_oracle as S
from paper_2601_05732_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
HALF = 2.0 ** -8                    # half a step of bf16, relative


@pytest.fixture(scope="module")
def ctx_of():
    made = {}

    def get(C):
        if C not in made:
            made[C] = binding.MhcLite(4, C, 0)
        return made[C]
    yield get
    for c in made.values():
        assert c.lib.mhclite_device_status(c._h) == binding.OK


def randn(seed, *shape, std=1.0, dtype=BF):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype).to(DEV)


def f64(t):
    return t.detach().double().cpu().numpy()


def empty(*shape, dtype=BF):
    return torch.full(shape, float("nan"), dtype=dtype, device=DEV)


def close(name, got, ref, tol):
    got = f64(got)
    assert got.shape == ref.shape, name
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got - ref) - tol):.3e} over"


def case(T, K, C, V, bf=False, absent=0.2, seed=0):
    """Rows whose ids are distinct where the vocabulary has enough, some entries absent, some rows without any."""
    h, W = randn(seed + 1, T, C), randn(seed + 2, V, C, std=2.0 / np.sqrt(C))
    r = np.random.default_rng(seed + 3)
    ids = np.stack([r.permutation(V)[:K] if K <= V else r.integers(0, V, K) for _ in range(T)])
    ids[r.random((T, K)) < absent] = -1
    if absent:
        ids[r.random(T) < absent] = -100
    return h, W, torch.from_numpy(ids).to(DEV), randn(seed + 4, T, K, std=2.0, dtype=BF if bf else F32), randn(seed + 5, T, dtype=F32)


def run(c, h, W, ids, z, scale, tau, dloss):
    T, K = ids.shape
    out = empty(T, dtype=F32), empty(T, dtype=F32), empty(T, K, dtype=F32), torch.empty_like(h).fill_(float("nan")), torch.empty_like(W).fill_(float("nan"))
    c.linear_distill_fwd(h, W, ids, z, scale, tau, *out[:3])
    c.linear_distill_bwd(h, W, ids, z, scale, tau, out[1], out[2], dloss, *out[3:])
    return out


def check(c, h, W, ids, z, scale, tau, dloss):
    (T, C), V, K = h.shape, W.shape[0], ids.shape[1]
    out = loss, lse, logp, dh, dW = run(c, h, W, ids, z, scale, tau, dloss)
    n, zd, Wd = ids.cpu().numpy(), f64(z), f64(W)
    p, log_p, live = S.teacher_weights(n, zd, tau, V)
    H = np.where(live[:, None], np.nan_to_num(f64(h)), 0.0)
    s = scale / tau
    rl, rs, rq = S.linear_distill_fwd(H, Wd, n, zd, scale, tau)
    # a logit: products exact, C / 16 steps of 16 added in fp32 with up to a unit in the last place each
    el = abs(s) * (C / 16 + 4) * 2.0 ** -23 * (np.abs(H) @ np.abs(Wd).T).max(1)
    # exp2 / log2 approximations: 2^-22 of each factor, and V / 256 + 64 additions of one sign
    es = (V / 256 + 64) * 2.0 ** -24 + 2.0 ** -21 * (1 + np.abs(rs))
    # a log probability is a difference of a logit and lse, each rounded a few times
    eq = np.where(live, 2 * el + es, 0)[:, None] + np.where(rq != 0, 2.0 ** -21 * (1 + np.abs(rq)), 0)
    close("lse", lse, rs, np.where(live, el + es, 0))
    close("logp", logp, rq, np.where((n >= 0) & (n < V) & live[:, None], eq, 0))
    # a teacher's log weight: difference, scale, the logarithm of a sum of up to 256 terms of one sign; its exponential
    lp = np.where(p > 0, log_p, 0.0)
    ep = 2.0 ** -21 * (2 + np.abs(lp)) + (K / 32 + 8) * 2.0 ** -24
    gap = np.abs(np.where(p > 0, lp - rq, 0.0))
    close("loss", loss, rl, np.where(live, (p * (eq + ep + (ep + (K / 32 + 8) * 2.0 ** -24) * gap)).sum(1), 0))
    rh, rW, a, q, share = S.linear_distill_bwd(H, Wd, n, zd, scale, tau, np.where(live, f64(dloss), 0))
    # the bracket: either probability off by its errors above, then rounded to bf16; the output rounded to bf16
    B, both = np.abs(q - share), q + share
    eG = np.abs(a)[:, None] * (HALF * B + (2 * el + 2 * es + ep.max(1) + 2.0 ** -20 * (1 + np.abs(rs)))[:, None] * both)
    # below 2^-126 a value may become 0, at the exponential, at the product with dloss and at one with an element of W or h
    tiny = 2.0 ** -126
    eG = eG + tiny * (1 + np.abs(a))[:, None]
    P = np.abs(a)[:, None] * B
    close("dh", dh, rh, HALF * np.abs(rh) + (1 + HALF) * (eG @ np.abs(Wd)) + (V / 16 + 4) * 2.0 ** -23 * (P @ np.abs(Wd)) + (V + 1) * tiny)
    close("dW", dW, rW, HALF * np.abs(rW) + (1 + HALF) * (eG.T @ np.abs(H)) + (T / 16 + 4) * 2.0 ** -23 * (P.T @ np.abs(H)) + (T + 1) * tiny)
    # the roundings are independent: in the 2-norm they add up as a random walk.  Four times its length is allowed.
    for name, got, ref, e, w in (("dh", dh, rh, (P ** 2) @ (Wd ** 2), both @ np.abs(Wd) * np.abs(a)[:, None]),
                                 ("dW", dW, rW, (P ** 2).T @ (H ** 2), (both * np.abs(a)[:, None]).T @ np.abs(H))):
        slack = (2 * el + 2 * es + ep.max(1) + 2.0 ** -20 * (1 + np.abs(rs))).max() * np.linalg.norm(w)
        assert np.linalg.norm(f64(got) - ref) <= HALF * np.linalg.norm(ref) + 4 * HALF * np.sqrt(e.sum()) + slack, name
    return out


CASES = [  # T, K, C, V, scale, temperature, bf16 teacher
    (1, 1, 8, 1, 1.0, 1.0, False), (1, 64, 64, 500, 1.0, 2.0, False), (1, 256, 2048, 5001, 1.0, 1.0, True), (3, 7, 72, 257, 0.5, 3.0, False),
    (17, 33, 4096, 777, 1.0, 1.0, True), (32, 20, 264, 4099, 1.0, 0.5, False), (33, 50, 128, 3000, 1.0, 2.0, True),
    (40, 4, 64, 2, 1.0, 1.0, False), (127, 256, 64, 256, 1.0, 2.0, False), (129, 31, 200, 1000, -0.7, 1.0, False),
    (300, 64, 1024, 2001, 1.0, 2.0, False), (257, 100, 1536, 515, 1.0, 1.0, True), (700, 8, 520, 3333, 0.7, 4.0, False),
    (600, 255, 64, 900, 1.0, 1.0, False), (2, 3, 8, 70001, 1.0, 1.0, False),
]


@pytest.mark.parametrize("T,K,C,V,scale,tau,bf", CASES)
def test_distill(ctx_of, T, K, C, V, scale, tau, bf):
    check(ctx_of(C), *case(T, K, C, V, bf, 0.0 if T == 1 else 0.2)[:4], scale, tau, randn(9, T, dtype=F32))


@pytest.mark.parametrize("T", [20, 300])
def test_absent_entries_and_rows_may_hold_anything(ctx_of, T):
    h, W, ids, z, dloss = case(T, 12, 64, 700, absent=0.4)
    ids[5] = torch.arange(12, device=DEV)
    z[ids < 0] = float("nan")
    z[3], z[5, :6] = -float("inf"), -float("inf")                 # a row without weight, a row with half of its entries
    dead = (ids < 0).all(1) | (z == -float("inf")).logical_or(ids < 0).all(1)
    assert dead.any() and not dead[5]
    h[dead], dloss[dead] = float("nan"), float("inf")
    loss, lse, logp, dh, dW = check(ctx_of(64), h, W, ids, z, 1.0, 2.0, torch.where(dead, 0.0, dloss))
    again = run(ctx_of(64), h, W, ids, z, 1.0, 2.0, dloss)
    for a, b in zip(again, (loss, lse, logp, dh, dW)):
        assert torch.equal(a, b) and torch.isfinite(a).all()
    assert (dh[dead] == 0).all() and (loss[dead] == 0).all() and (logp[dead] == 0).all() and (logp[5] < 0).all()


@pytest.mark.parametrize("T", [20, 300])
def test_nan_in_a_present_entry_stays_in_its_row(ctx_of, T):
    h, W, ids, z, dloss = case(T, 12, 64, 700, absent=0.0)
    z[5, 7] = float("nan")
    loss, lse, logp, dh, _ = run(ctx_of(64), h, W, ids, z, 1.0, 2.0, dloss)
    rest = torch.arange(T, device=DEV) != 5
    assert loss[5].isnan() and dh[5].isnan().all() and torch.isfinite(loss[rest]).all() and torch.isfinite(dh[rest]).all()
    assert torch.isfinite(lse).all() and torch.isfinite(logp).all()


@pytest.mark.parametrize("T", [20, 300])
@pytest.mark.parametrize("bf,tau", [(False, 0.5), (False, 2.0), (True, 0.5)])
def test_masks_of_the_lowest_value(ctx_of, T, bf, tau):
    """Teacher logits masked with the type's lowest value instead of -inf: weights of 0, equal ones where a row has no others, and
    a largest value next to which all others vanish."""
    h, W, ids, z, dloss = case(T, 40, 64, 700, bf, absent=0.2)
    lowest = torch.finfo(z.dtype).min
    z[torch.rand(T, 40, generator=torch.Generator().manual_seed(1)).to(DEV) < 0.4] = lowest
    z[3], z[5, 2:], z[6, 7] = lowest, lowest, -lowest
    out = check(ctx_of(64), h, W, ids, z, 1.0, tau, dloss)
    assert all(torch.isfinite(o).all() for o in out)


@pytest.mark.parametrize("T", [1, 200])
def test_no_row_has_a_teacher(ctx_of, T):
    h, W, ids, z, dloss = case(T, 5, 64, 300)
    ids.fill_(-1)
    for t in run(ctx_of(64), h * float("nan"), W, ids, z, 1.0, 1.0, dloss):
        assert (t == 0).all()


def test_only_the_last_row_has_a_teacher(ctx_of):
    h, W, ids, z, dloss = case(1000, 9, 64, 300, absent=0.0)
    ids[:-1] = -1
    ids[-1] = torch.arange(291, 300, device=DEV)
    check(ctx_of(64), h, W, ids, z, 1.0, 1.0, dloss)


@pytest.mark.parametrize("T", [9, 300])
def test_the_same_id_several_times(ctx_of, T):
    h, W, ids, z, dloss = case(T, 40, 64, 500, absent=0.1)
    ids[:, 20:] = ids[:, :20]
    ids[0], ids[1, :] = 499, 0
    check(ctx_of(64), h, W, ids, z, 1.0, 1.0, dloss)


@pytest.mark.parametrize("T", [5, 300])
def test_one_entry_is_cross_entropy(ctx_of, T):
    h, W, ids, z, dloss = case(T, 1, 128, 1000)
    c = ctx_of(128)
    loss, lse, logp, dh, dW = check(c, h, W, ids, z, 1.0, 1.0, dloss)
    other = empty(T, dtype=F32), empty(T, dtype=F32)
    c.linear_ce_fwd(h, W, ids[:, 0].contiguous(), 1.0, *other)
    # the same logits and partial sums, joined in another order: two sums of 32 ranges, off by 37 additions of one sign each,
    # and two logarithms and roundings of a number below 16: 2 x 37 x 2^-24 + 4 x 16 x 2^-23 < 2^-16.  The loss also takes
    # its logit's sum in another order: C / 16 + 4 = 12 steps of 2^-23 of a sum of magnitudes below 128 at either side.
    assert (lse - other[1]).abs().max() < 2.0 ** -16 and (loss - other[0]).abs().max() < 2.0 ** -16 + 2 * 12 * 2.0 ** -23 * 128


@pytest.mark.parametrize("T,shift", [(7, 0.0), (300, 0.0), (300, 60.0)])
def test_a_teacher_near_the_student_keeps_the_digits(ctx_of, T, shift):
    """The student's own logits as the teacher's, over the whole vocabulary: the loss is 0 but for rounding, and so are the
    gradients, whatever the size of the logits."""
    C, V = 64, 200
    h, W = randn(1, T, C), randn(2, V, C, std=0.3)
    h[:, 0], W[:, 0] = 8.0, shift / 8.0
    ids = torch.from_numpy(np.stack([np.random.default_rng(t).permutation(V) for t in range(T)])).to(DEV)
    z = (h.double() @ W.double().T).gather(1, ids).float()
    loss, lse, logp, dh, dW = check(ctx_of(C), h, W, ids, z, 1.0, 1.0, torch.ones(T, device=DEV))
    # either log probability is off by some 2^-20 of the logits' size, as in check; the second order of it is the loss
    assert loss.max() < 2.0 ** -12 and dh.abs().max() < 2.0 ** -8


def test_sharp_logits(ctx_of):
    h, W, ids, z, dloss = case(60, 16, 64, 300, absent=0.0)
    check(ctx_of(64), h * 16, W * 4, ids, z * 20, 1.0, 1.0, dloss)


def test_distill_in_several_pieces(ctx_of):
    """16384 tokens and 20001 columns do not fit one piece: dh adds up over three, and a row's entries fall into all of them."""
    T, K, C, V = 16384, 24, 64, 20001
    c = ctx_of(C)
    h, W = randn(1, T, C), randn(2, V, C, std=2.0 / np.sqrt(C))
    g = torch.Generator(device=DEV).manual_seed(3)
    ids = torch.randint(0, V, (T, K), generator=g, device=DEV)
    ids[::9], ids[5, 3:] = -1, -1
    z, dloss = randn(4, T, K, std=2.0, dtype=F32), randn(5, T, dtype=F32)
    loss, lse, logp, dh, dW = run(c, h, W, ids, z, 1.0, 2.0, dloss)
    there, live = ids >= 0, (ids >= 0).any(1)
    hd, Wd, at = h.double() * live[:, None], W.double(), ids.clamp(min=0)
    x = 0.5 * hd @ Wd.T
    rs = torch.logsumexp(x, 1)
    rq = torch.where(there, x.gather(1, at) - rs[:, None], 0.0)
    log_p = torch.log_softmax(torch.where(there, z.double() / 2, -float("inf")), 1)
    p = torch.where(there, log_p.exp(), 0.0)
    rl = torch.where(there, p * (log_p - rq), 0.0).sum(1)
    G = torch.softmax(x, 1).scatter_add_(1, at, -p) * (0.5 * dloss.double() * live)[:, None]
    el = 0.5 * (C / 16 + 4) * 2.0 ** -23 * (hd.abs() @ Wd.abs().T).amax(1) + (V / 256 + 64) * 2.0 ** -24 + 2.0 ** -20 * (1 + rs.abs())
    assert ((lse - rs * live).abs() <= el).all()
    eq = 2 * el + 2.0 ** -21 * (1 + rq.abs().amax(1))
    assert ((logp - rq).abs() <= eq[:, None]).all() and (logp[~there] == 0).all()
    assert ((loss - rl).abs() <= 2 * eq + 2.0 ** -18 * (1 + rl)).all()
    for got, ref, e in ((dh, G @ Wd, (G ** 2) @ (Wd ** 2)), (dW, G.T @ hd, (G ** 2).T @ (hd ** 2))):
        assert (got.double() - ref).norm() <= HALF * ref.norm() + 4 * HALF * e.sum().sqrt()
    assert (dh[~live] == 0).all()


def test_offsets_beyond_32_bits(ctx_of):
    """A head of 1.1 M rows x 2048: the last rows lie beyond 2^31 elements."""
    C, V = 2048, 1_100_000
    c = ctx_of(C)
    W = torch.empty(V, C, dtype=BF, device=DEV).normal_(std=0.02, generator=torch.Generator(device=DEV).manual_seed(1))
    for T in (3, 40):                                             # the streaming kernel and the tiles
        h, z = randn(7, T, C), randn(8, T, 4, dtype=F32)
        ids = torch.tensor([V - 1, 5, V - 2, 600_000], device=DEV).expand(T, 4).contiguous()
        loss, lse, logp = empty(T, dtype=F32), empty(T, dtype=F32), empty(T, 4, dtype=F32)
        c.linear_distill_fwd(h, W, ids, z, 1.0, 1.0, loss, lse, logp)
        parts = [torch.logsumexp(h.double() @ W[v:v + 100_000].double().T, 1) for v in range(0, V, 100_000)]
        ref = torch.logsumexp(torch.stack(parts, 1), 1)
        rq = (h.double()[:, None] * W[ids[0]].double()).sum(2) - ref[:, None]
        # logits of about 1: 128 steps of 16 products, V / 256 sums; as in check
        assert (lse - ref).abs().max() < 1e-4 and (logp - rq).abs().max() < 1e-4


def test_vocabularies_beyond_23_bits(ctx_of):
    """More rows than a row's entries are sorted by in 32 bits: ids near both ends, one of them twice, gradients with them."""
    C, V, T = 8, (1 << 23) + 77, 40
    c = ctx_of(C)
    W = torch.empty(V, C, dtype=BF, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(1))
    h, z, dloss = randn(7, T, C), randn(8, T, 5, dtype=F32), randn(9, T, dtype=F32)
    ids = torch.tensor([V - 1, 5, (1 << 23) - 1, 5, V - 2], device=DEV).expand(T, 5).contiguous()
    ids[3], ids[4, 2:] = -1, -1
    loss, lse, logp, dh, dW = run(c, h, W, ids, z, 1.0, 1.0, dloss)
    live, there = (ids >= 0).any(1), ids >= 0
    hd, Wd = h.double() * live[:, None], W.double()
    x = hd @ Wd.T
    ref = torch.logsumexp(x, 1)
    rq = torch.where(there, x.gather(1, ids.clamp(min=0)) - ref[:, None], 0.0)
    # one step of 16 products, V / 256 sums of one sign in the longest chain: 2^-24 x V / 256 = 0.002 at most
    assert ((lse - ref * live).abs() <= V / 256 * 2.0 ** -24).all() and ((logp - rq).abs() <= V / 256 * 2.0 ** -24).all()
    p = torch.where(there, torch.softmax(torch.where(there, z.double(), -float("inf")), 1), 0.0)
    G = torch.softmax(x, 1).scatter_add_(1, ids.clamp(min=0), -p) * (dloss.double() * live)[:, None]
    for got, want, e in ((dh, G @ Wd, (G ** 2) @ (Wd ** 2)), (dW, G.T @ hd, (G ** 2).T @ (hd ** 2))):
        assert (got.double() - want).norm() <= HALF * want.norm() + 4 * HALF * e.sum().sqrt() + V / 256 * 2.0 ** -24 * (G.abs() @ Wd.abs()).norm()
    assert (dW[[5, V - 1]].double() - (G.T @ hd)[[5, V - 1]]).abs().max() <= HALF * 2 * (G.T @ hd)[[5, V - 1]].abs().max() + 1e-3


def test_ids_beyond_the_table_are_reported():
    for T in (20, 50):
        c = binding.MhcLite(2, 64, 0)                             # a context of its own: the report stays
        h, W, ids, z, dloss = case(T, 6, 64, 100, absent=0.0)
        ids[7, 2], ids[9, :] = 100, 2 ** 40
        _, _, logp, dh, _ = check(c, h, W, ids, z, 1.0, 1.0, dloss)
        assert logp[7, 2] == 0 and (dh[9] == 0).all()
        with pytest.raises(binding.MhcLiteError) as e:
            c.device_status()
        assert e.value.status == binding.ERR_INDEX


def test_refusals(ctx_of):
    c, T, K, C, V = ctx_of(64), 20, 6, 64, 100
    h, W, ids, z, dloss = case(T, K, C, V)
    loss, lse, logp, dh, dW = (empty(T, dtype=F32), empty(T, dtype=F32), empty(T, K, dtype=F32), empty(T, C), empty(V, C))
    bad = binding.MhcLiteError
    for tau in (0.0, -1.0, float("nan"), float("inf"), 1e-45):
        with pytest.raises(bad):
            c.linear_distill_fwd(h, W, ids, z, 1.0, tau, loss, lse, logp)
    for s in (float("nan"), float("inf"), 3e38):                  # the last overflows with the temperature in it
        with pytest.raises(bad):
            c.linear_distill_fwd(h, W, ids, z, s, 0.5, loss, lse, logp)
    wide = torch.zeros(T, 257, dtype=torch.int64, device=DEV)
    with pytest.raises(bad):
        c.linear_distill_fwd(h, W, wide, wide.float(), 1.0, 1.0, loss, lse, wide.float())
    none = ids[:, :0].contiguous()
    with pytest.raises(bad):
        c.linear_distill_fwd(h, W, none, none.float(), 1.0, 1.0, loss, lse, none.float())
    for args in ((h, W.float(), ids, z), (h, W, ids.int(), z), (h, W, ids, z.half()), (h, W, ids, z[:, :3]), (h, W, ids[:, 0], z),
                 (h, W, ids.t().contiguous().t(), z), (h[:, :32], W, ids, z), (h, W, ids[:3], z)):
        with pytest.raises(ValueError):
            c.linear_distill_fwd(*args, 1.0, 1.0, loss, lse, logp)
    with pytest.raises(bad):
        c.linear_distill_fwd(h, W, ids, z, 1.0, 1.0, loss, loss, logp)
    with pytest.raises(bad):
        c.linear_distill_fwd(h, W, ids, z, 1.0, 1.0, loss, lse, z)
    c.linear_distill_fwd(h, W, ids, z, 1.0, 1.0, loss, lse, logp)
    with pytest.raises(bad):
        c.linear_distill_bwd(h, W, ids, z, 1.0, 1.0, lse, logp, dloss, h, dW)
    need = c.lib.mhclite_linear_distill_scratch_bytes(C, T, V, K, 0)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    assert c.lib.mhclite_linear_distill_fwd(c._h, T, V, K, h.data_ptr(), W.data_ptr(), ids.data_ptr(), z.data_ptr(), 1, 1.0, 1.0, loss.data_ptr(),
                                            lse.data_ptr(), logp.data_ptr(), ws.data_ptr(), need - 1, None) == binding.ERR_WORKSPACE
    before = c.kernel_launches()
    c.linear_distill_fwd(h[:0], W, ids[:0], z[:0], 1.0, 1.0, loss[:0], lse[:0], logp[:0])
    c.linear_distill_bwd(h[:0], W, ids[:0], z[:0], 1.0, 1.0, lse[:0], logp[:0], dloss[:0], dh[:0], dW)
    assert (dW == 0).all() and c.kernel_launches() == before


def inside(t):
    """The same values in a view 16 bytes (one element, for int64: 8) into a buffer: the least alignment the calls allow."""
    k = max(1, 16 // t.element_size()) if t.dtype != torch.int64 else 1
    v = torch.empty(t.numel() + 2 * k, dtype=t.dtype, device=DEV)[k:k + t.numel()].view(t.shape)
    assert v.data_ptr() % 32 in (8, 16)
    return v.copy_(t)


@pytest.mark.parametrize("T,K,C,V,bf", [(40, 7, 64, 200, True), (300, 31, 72, 2001, False), (3, 5, 64, 500, True), (1, 64, 1024, 300, False)])
def test_inner_views(ctx_of, T, K, C, V, bf):
    c, (h, W, ids, z, dloss) = ctx_of(C), case(T, K, C, V, bf)
    want = run(c, h, W, ids, z, 1.0, 2.0, dloss)
    h, W, ids, z, dloss = (inside(t) for t in (h, W, ids, z, dloss))
    got = [inside(t) for t in want]
    for t in got:
        t.fill_(float("nan"))
    c.linear_distill_fwd(h, W, ids, z, 1.0, 2.0, *got[:3])
    c.linear_distill_bwd(h, W, ids, z, 1.0, 2.0, got[1], got[2], dloss, *got[3:])
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_streams_at_once_and_bitwise_repeats(ctx_of):
    c, (h, W, ids, z, dloss) = ctx_of(256), case(500, 40, 256, 3001)
    few = [t[:20].contiguous() for t in (h, ids, z, dloss)]
    torch.cuda.synchronize()
    outs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams * 3:
        with torch.cuda.stream(s):
            outs.append((*run(c, h, W, ids, z, 1.0, 2.0, dloss), *run(c, few[0], W, few[1], few[2], 1.0, 2.0, few[3])))
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))


def test_captured_and_replayed_with_new_inputs(ctx_of):
    """Two graphs, each with scratch of its own; between replays the inputs change, and with them which rows count."""
    c = ctx_of(256)
    cases = [case(200, 30, 256, 1000), case(20, 30, 256, 1000, seed=50)]
    step = lambda k: [run(c, h, W, ids, z, 1.0, 2.0, dloss) for h, W, ids, z, dloss in cases]
    side, graphs = torch.cuda.Stream(), []
    with torch.cuda.stream(side):
        step(0)
    torch.cuda.synchronize()
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            out = step(0)
        graphs.append((gr, out))
    for k in range(3):
        for (h, W, ids, z, dloss), n in zip(cases, (200, 20)):
            new = case(n, 30, 256, 1000, absent=0.1 * k, seed=100 + k)
            h.copy_(new[0]), ids.copy_(new[2]), z.copy_(new[3])
        torch.cuda.synchronize()
        for gr, _ in graphs:
            gr.replay()
        torch.cuda.synchronize()
        want = step(0)
        for _, got in graphs:
            assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))
