"""The operators around the stack on the GPU against the fp64 oracle: lookup, block norms, dropout and cross entropy, their
gradients, their refusals, and a whole model step made of them.

Tolerances follow the arithmetic.  A bf16 output is off by at most half a step, 2^-8 of its value, on top of the fp32
arithmetic before it.  An fp32 sum is off by at most (number of additions on the longest path) x 2^-24 x the sum of its
terms' magnitudes."""
import numpy as np
import pytest
import torch

from oracle import stack_ends_oracle as S
from paper_2601_05732_b200 import binding
from paper_2601_05732_b200 import layer as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
HALF = 2.0 ** -8                    # half a step of bf16, relative


@pytest.fixture(scope="module")
def ctx_of():
    made = {}

    def get(n, C):
        if (n, C) not in made:
            made[n, C] = binding.MhcLite(n, C, 0)
        return made[n, C]
    yield get
    for c in made.values():
        assert c.lib.mhclite_device_status(c._h) == binding.OK


def randn(seed, *shape, std=1.0, mean=0.0, dtype=BF):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std + mean).to(dtype).to(DEV)


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def empty(*shape, dtype=BF):
    return torch.full(shape, float("nan"), dtype=dtype, device=DEV)


def close(name, got, ref, tol):
    got = f64(got)
    assert got.shape == ref.shape, name
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got - ref) - tol):.3e} over"


def rng_of(seed, offset):
    return torch.tensor([seed, offset], dtype=torch.int64, device=DEV)


# ---- dropout -----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("count,p", [(1, 0.5), (7, 0.5), (8, 0.25), (4099, 0.1), (30000, 0.9), (513, 0.0)])
def test_dropout(ctx_of, count, p):
    c, x, y = ctx_of(4, 64), randn(count, count), empty(count)
    c.dropout(x, p, rng_of(987654321987, 42 + (1 << 40)), y)
    keep = S.keep_mask(count, p, 987654321987, 42 + (1 << 40))
    ref = np.where(keep, f64(x) * S.drop_factor(p), 0.0)
    close("y", y, ref, (HALF + 2.0 ** -20) * np.abs(ref))
    assert (f64(y)[~keep] == 0).all()


def test_dropout_of_infinities_and_a_negative_seed(ctx_of):
    c, x, y = ctx_of(4, 64), randn(1, 6, 5, 8), empty(6, 5, 8)
    keep = S.keep_mask(240, 0.5, -3, 9).reshape(6, 5, 8)
    x[torch.from_numpy(~keep).to(DEV)] = float("inf")
    x.view(-1)[int(np.flatnonzero(~keep)[0])] = float("nan")
    c.dropout(x, 0.5, rng_of(-3, 9), y)
    assert torch.isfinite(y).all() and (f64(y)[~keep] == 0).all()


def test_dropout_refusals(ctx_of):
    c, x, y, r = ctx_of(4, 64), randn(1, 16), empty(16), rng_of(1, 2)
    for p in (-0.1, 1.0, 1.5, float("nan"), 1 - 2.0 ** -18):
        with pytest.raises(binding.MhcLiteError):
            c.dropout(x, p, r, y)
    with pytest.raises(binding.MhcLiteError):
        c.dropout(x, 0.1, r, x)                                   # in place
    with pytest.raises(ValueError):
        c.dropout(x, 0.1, r, empty(15))
    with pytest.raises(ValueError):
        c.dropout(x.float(), 0.1, r, y)
    c.dropout(empty(0), 0.1, r, empty(0))
    c.dropout(x, 0.1, r, y)
    assert torch.isfinite(y).all()                                # a refused call leaves the context usable


# ---- the norms around a sublayer ---------------------------------------------------------------------------------------
BLOCKS = [  # T, C, gate, p
    (1, 8, False, 0.0), (1, 4096, True, 0.0), (3, 64, True, 0.3), (130, 256, False, 0.1), (37, 264, True, 0.1), (65, 520, True, 0.0),
    (700, 1536, False, 0.1), (257, 2048, True, 0.1), (9, 5000, True, 0.2), (5, 8192, False, 0.5), (3, 16384, True, 0.1), (2500, 72, True, 0.05),
]


@pytest.mark.parametrize("T,C,gated,p", BLOCKS)
def test_block_out(ctx_of, T, C, gated, p):
    c = ctx_of(4, C)
    o, gate = randn(1, T, C, std=3.0), randn(2, T, C, std=1.5) if gated else None
    w, s, dy = randn(3, C, std=0.2, mean=1.0, dtype=F32), torch.full((1,), 0.4, device=DEV), randn(4, T, C, std=1e-2)
    seed, off = 77, 5
    rng = rng_of(seed, off) if p else None
    y, r = empty(T, C), empty(T, dtype=F32)
    c.block_out_fwd(o, gate, w, s, 1e-6, p, rng, y, r)
    keep = S.keep_mask(T * C, p, seed, off).reshape(T, C) if p else None
    fac, sv = S.drop_factor(p), float(s.double())
    ref, rref = S.block_out_fwd(f64(o), f64(gate), f64(w), sv, 1e-6, keep, fac)
    # rstd: C squares of one sign added in fp32, at most C / 32 + 16 in a row; sigmoid: |a| < 10 in __expf, some 2^-18
    rel = (C / 32 + 32) * 2.0 ** -24
    fine = rel + (2.0 ** -16 if gated else 2.0 ** -20)
    close("rstd", r, rref, 2 * rel * rref)
    close("y", y, ref, (HALF + fine) * np.abs(ref))
    d_o, dg, dw, ds = empty(T, C), empty(T, C) if gated else None, empty(C, dtype=F32), empty(1, dtype=F32)
    c.block_out_bwd(o, gate, w, s, r, p, rng, dy, d_o, dg, dw, ds)
    b = S.block_out_bwd(f64(o), f64(gate), f64(w), sv, 1e-6, f64(dy), keep, fac)
    close("d_o", d_o, b["d_o"], HALF * np.abs(b["d_o"]) + 4 * fine * b["mag_d_o"])
    if gated:
        close("dgate", dg, b["dgate"], (HALF + 4 * fine) * np.abs(b["dgate"]))
    depth = (64 + T / 64) * 2.0 ** -24
    close("dw", dw, b["dw"], (depth + 2 * fine) * b["mag_dw"])
    close("dscale", ds, np.array([b["dscale"]]), (C / 32 * 2.0 ** -24 + 2 * fine) * b["mag_dscale"])
    dw2, ds2 = dw.clone(), ds.clone()
    c.block_out_bwd(o, gate, w, s, r, p, rng, dy, d_o, dg, dw2, ds2, accumulate_params=True)
    assert torch.equal(dw2, dw + dw) and torch.equal(ds2, ds + ds)          # doubling is exact


@pytest.mark.parametrize("T,C,gated,p", [(300, 10000, True, 0.0), (19, 16384, True, 0.2), (150, 8200, False, 0.0)])
def test_block_out_long_rows_over_several_blocks(ctx_of, T, C, gated, p):
    test_block_out(ctx_of, T, C, gated, p)


@pytest.mark.parametrize("C,p", [(64, 0.0), (520, 0.25), (9000, 0.0)])
def test_block_gates_far_open_and_shut(ctx_of, C, p):
    """1 - sigmoid(a) keeps its digits however far the gate is open; infinite gates give zeros, not NaN."""
    T, inf = 24, float("inf")
    c, rng = ctx_of(4, C), rng_of(5, 6) if p else None
    o, dy, w = randn(1, T, C), randn(2, T, C), randn(3, C, std=0.2, mean=1.0, dtype=F32)
    gate = torch.linspace(-30, 30, T * C).reshape(T, C)
    gate.view(-1)[:16] = torch.tensor([inf, -inf, 100, -100, 88.5, -88.5, 87, -87, 60, -60, 45, -45, 3e38, -3e38, 0, -0.0])
    gate = gate.view(-1)[torch.randperm(T * C, generator=torch.Generator().manual_seed(4))].reshape(T, C).to(BF).to(DEV)
    y, r, d_o, dg, dw = empty(T, C), empty(T, dtype=F32), empty(T, C), empty(T, C), empty(C, dtype=F32)
    c.block_out_fwd(o, gate, w, None, 1e-6, p, rng, y, r)
    c.block_out_bwd(o, gate, w, None, r, p, rng, dy, d_o, dg, dw, None)
    keep, fac = (S.keep_mask(T * C, p, 5, 6).reshape(T, C), S.drop_factor(p)) if p else (None, 1.0)
    ref, _ = S.block_out_fwd(f64(o), f64(gate), f64(w), 1.0, 1e-6, keep, fac)
    b = S.block_out_bwd(f64(o), f64(gate), f64(w), 1.0, 1e-6, f64(dy), keep, fac)
    # the row's sum as in test_block_out; e^-a for |a| <= 100: its argument in base 2 is rounded once, 145 x 2^-24 x ln 2 < 2^-17
    fine = (C / 32 + 32) * 2.0 ** -24 + 2.0 ** -16
    # below 2^-126 e^-a, the sigmoid and the products after them may each become 0: 2^-126 at most, times the factors that follow
    oh = np.abs(f64(o)) / np.sqrt((f64(o) ** 2).mean(1, keepdims=True))
    tiny = 4 * 2.0 ** -126 * (1 + fac * np.abs(f64(dy))) * (1 + np.abs(f64(w))) * (1 + oh)
    close("y", y, ref, (HALF + fine) * np.abs(ref) + tiny)
    close("dgate", dg, b["dgate"], (HALF + 4 * fine) * np.abs(b["dgate"]) + tiny)
    close("d_o", d_o, b["d_o"], HALF * np.abs(b["d_o"]) + 4 * fine * b["mag_d_o"] + tiny)


@pytest.mark.parametrize("T,C", [(1, 8), (1, 2048), (300, 1536), (33, 4096), (4100, 256)])
def test_block_in(ctx_of, T, C):
    c = ctx_of(2, C)
    u, w, dv = randn(1, T, C), randn(2, C, std=0.2, mean=1.0, dtype=F32), randn(3, T, C)
    v, r = empty(T, C), empty(T, dtype=F32)
    c.block_in_fwd(u, w, 1e-5, v, r)
    ref, _ = S.block_out_fwd(f64(u), None, f64(w), 1.0, 1e-5)
    fine = (C / 32 + 32) * 2.0 ** -24 + 2.0 ** -20
    close("v", v, ref, (HALF + fine) * np.abs(ref))
    du, dw = empty(T, C), empty(C, dtype=F32)
    c.block_in_bwd(u, w, r, dv, du, dw)
    b = S.block_out_bwd(f64(u), None, f64(w), 1.0, 1e-5, f64(dv))
    close("du", du, b["d_o"], HALF * np.abs(b["d_o"]) + 4 * fine * b["mag_d_o"])
    close("dw", dw, b["dw"], ((64 + T / 64) * 2.0 ** -24 + 2 * fine) * b["mag_dw"])


def test_block_mask_is_the_dropout_mask(ctx_of):
    """block_out drops exactly the elements that mhclite_dropout drops, and their gradients with them."""
    c, T, C, rng = ctx_of(4, 264), 19, 264, rng_of(3, 4)
    o, gate, w = randn(1, T, C), randn(2, T, C), torch.ones(C, device=DEV)
    y, r, m = empty(T, C), empty(T, dtype=F32), empty(T, C)
    c.block_out_fwd(o, gate, w, None, 1e-6, 0.3, rng, y, r)
    c.dropout(torch.ones(T, C, dtype=BF, device=DEV), 0.3, rng, m)
    assert torch.equal(m == 0, y == 0)
    gate[m == 0] = float("nan")                                   # what a dropped element holds does not matter
    c.block_out_fwd(o, gate, w, None, 1e-6, 0.3, rng, y, r)
    assert torch.isfinite(y).all()
    dy = randn(4, T, C)
    dy[m == 0] = float("inf")                                     # nor what its gradient holds
    d_o, dg, dw = empty(T, C), empty(T, C), empty(C, dtype=F32)
    c.block_out_bwd(o, gate, w, None, r, 0.3, rng, dy, d_o, dg, dw, None)
    assert torch.isfinite(d_o).all() and torch.isfinite(dw).all() and (dg[m == 0] == 0).all() and torch.isfinite(dg).all()


def test_block_large_and_zero_rows(ctx_of):
    """A row of zeros is normalised by eps alone; bf16's largest values square beyond fp32 and give zeros, as the formula
    1 / sqrt(inf) does, never a trap."""
    c, C = ctx_of(4, 256), 256
    o = randn(1, 3, C)
    o[0] = 0
    o[1] = 1e30
    w, y, r = torch.ones(C, device=DEV), empty(3, C), empty(3, dtype=F32)
    c.block_in_fwd(o, w, 1e-6, y, r)
    assert (y[0] == 0).all() and r[0].item() == pytest.approx(1e3, rel=1e-5)
    assert r[1].item() == 0 and (y[1] == 0).all()
    ref, _ = S.block_out_fwd(f64(o[2:]), None, f64(w), 1.0, 1e-6)
    close("row", y[2:], ref, (HALF + 2.0 ** -18) * np.abs(ref))


def test_block_refusals(ctx_of):
    c, C, T = ctx_of(4, 64), 64, 4
    o, w, y, r, dy = randn(1, T, C), torch.ones(C, device=DEV), empty(T, C), empty(T, dtype=F32), randn(2, T, C)
    rng, g = rng_of(1, 2), randn(3, T, C)
    bad = binding.MhcLiteError
    with pytest.raises(bad):
        c.block_out_fwd(o, None, w, None, -1.0, 0.0, None, y, r)
    with pytest.raises(bad):
        c.block_out_fwd(o, None, w, None, 1e-6, 0.5, None, y, r)         # dropout without a generator state
    with pytest.raises(bad):
        c.block_out_fwd(o, None, w, None, 1e-6, 1.0, rng, y, r)
    with pytest.raises(bad):
        c.block_in_fwd(o, w, 1e-6, o, r)                                 # in place
    with pytest.raises(bad):
        c.block_out_bwd(o, g, w, None, r, 0.0, None, dy, y, None, empty(C, dtype=F32), None)   # gate without dgate
    with pytest.raises(ValueError):
        c.block_in_fwd(o, w[:32], 1e-6, y, r)
    with pytest.raises(ValueError):
        c.block_in_fwd(o.t().contiguous().t(), w, 1e-6, y, r)
    big = ctx_of(2, 16392)
    with pytest.raises(bad):
        big.block_in_fwd(randn(1, 1, 16392), torch.ones(16392, device=DEV), 1e-6, empty(1, 16392), empty(1, dtype=F32))
    z = torch.ones(C, device=DEV)
    c.block_in_bwd(o[:0], w, r[:0], dy[:0], y[:0], z)
    assert (z == 0).all()                                                # no rows: the sum is zero
    z.fill_(1)
    c.block_in_bwd(o[:0], w, r[:0], dy[:0], y[:0], z, accumulate_params=True)
    assert (z == 1).all()


def test_no_tokens_at_all(ctx_of):
    """T = 0 launches nothing and leaves the outputs alone, forward; the backward's zero sums are tested with the refusals."""
    c, C = ctx_of(4, 64), 64
    none, nof, noi = empty(0, C), empty(0, dtype=F32), torch.empty(0, dtype=torch.int64, device=DEV)
    w, W, before = torch.ones(C, device=DEV), randn(1, 10, C), c.kernel_launches()
    c.block_in_fwd(none, w, 1e-6, none, nof)
    c.block_out_fwd(none, none, w, None, 1e-6, 0.5, rng_of(1, 2), none, nof)
    c.embed_fwd(noi, W, 1.0, empty(0, 4, C))
    c.linear_ce_fwd(none, W, noi, 1.0, nof, nof)
    assert c.kernel_launches() == before


# ---- lookup ------------------------------------------------------------------------------------------------------------
def some_ids(seed, T, V, kind):
    r = np.random.default_rng(seed)
    if kind == "one":
        return np.full(T, V - 1)
    if kind == "text":
        return np.minimum(np.floor((V + 1.0) ** r.random(T)).astype(np.int64) - 1, V - 1)
    return r.integers(0, V, T)


@pytest.mark.parametrize("T,n,C,V,f32", [(1, 4, 2048, 50257, False), (7, 2, 8, 3, True), (100, 3, 72, 1000, True),
                                         (33, 5, 1536, 257, False), (1025, 4, 264, 4096, True)])
def test_embed_fwd(ctx_of, T, n, C, V, f32):
    c = ctx_of(n, C)
    E, ids = randn(1, V, C, dtype=F32 if f32 else BF), torch.from_numpy(some_ids(2, T, V, "even")).to(DEV)
    x0 = empty(T, n, C)
    c.embed_fwd(ids, E, 3.5, x0)
    assert torch.equal(x0, (E[ids].float() * 3.5).to(BF)[:, None, :].expand(T, n, C))     # one rounding: bit for bit


EMBEDS = [  # T, n, C, V, ids
    (1, 4, 64, 9, "even"), (5, 2, 8, 1, "even"), (31, 3, 72, 300, "even"), (1000, 4, 256, 70, "even"), (5003, 3, 264, 5000, "text"),
    (4096, 4, 64, 100, "one"), (2500, 5, 1536, 70000, "text"), (70000, 2, 16, 1000, "text"), (33, 4, 520, 255, "one"), (256, 4, 64, 256, "even"),
    (64, 4, 2048, 500, "text"), (64, 2, 24, 3, "one"), (65, 2, 24, 3, "even"), (192, 3, 520, 2000, "text"), (192, 2, 24, 3, "one"), (193, 2, 24, 3, "even"), (6144, 2, 64, 300, "text"), (6145, 2, 64, 300000, "text"), (20000, 2, 8, 64, "even"),
]


@pytest.mark.parametrize("T,n,C,V,kind", EMBEDS)
def test_embed_bwd(ctx_of, T, n, C, V, kind):
    c = ctx_of(n, C)
    ids = some_ids(T, T, V, kind)
    g, dE = randn(3, T, n, C), empty(V, C, dtype=F32)
    t = torch.from_numpy(ids).to(DEV)
    c.embed_bwd(t, g, 0.75, dE)
    ref, mag = S.embed_bwd(ids, f64(g), 0.75, V)
    # additions in a row: 32 tokens of n streams in a chunk, an eighth of the chunks (4 tokens at least), 16 to join
    depth = (32 * n + T / 32 + 32) * 2.0 ** -24
    close("dE", dE, ref, depth * mag)
    again = empty(V, C, dtype=F32)
    c.embed_bwd(t, g, 0.75, again)
    assert torch.equal(dE, again)
    again.fill_(0)
    c.embed_bwd(t, g, 0.75, again, accumulate=True)
    assert torch.equal(dE, again)
    c.embed_bwd(t, g, 0.75, again, accumulate=True)
    close("dE twice", again, 2 * ref, 2 * depth * mag + 2.0 ** -23 * np.abs(ref))


def test_embed_leaves_other_rows_when_accumulating(ctx_of):
    c, V, C = ctx_of(2, 16), 50, 16
    dE = torch.full((V, C), 5.0, device=DEV)
    c.embed_bwd(torch.tensor([3, 7, 3], device=DEV), torch.ones(3, 2, C, dtype=BF, device=DEV), 1.0, dE, accumulate=True)
    ref = torch.full((V, C), 5.0, device=DEV)
    ref[3], ref[7] = 9.0, 7.0
    assert torch.equal(dE, ref)


def test_embed_out_of_range_ids_are_reported():
    c = binding.MhcLite(2, 16, 0)                                        # a context of its own: the report stays
    E, x0 = randn(1, 10, 16, dtype=F32), empty(4, 2, 16)
    ids = torch.tensor([1, 10, -5, 9], device=DEV)
    c.embed_fwd(ids, E, 1.0, x0)
    assert (x0[1:3] == 0).all() and torch.equal(x0[3, 1], E[9].to(BF))
    with pytest.raises(binding.MhcLiteError) as e:
        c.device_status()
    assert e.value.status == binding.ERR_INDEX
    c = binding.MhcLite(2, 16, 0)
    g, dE = torch.ones(4, 2, 16, dtype=BF, device=DEV), empty(10, 16, dtype=F32)
    c.embed_bwd(ids, g, 1.0, dE)
    ref = torch.zeros(10, 16, device=DEV)
    ref[1], ref[9] = 2.0, 2.0
    assert torch.equal(dE, ref)
    with pytest.raises(binding.MhcLiteError):
        c.device_status()


def test_embed_refusals(ctx_of):
    c, E, ids, x0 = ctx_of(2, 16), randn(1, 10, 16, dtype=F32), torch.tensor([1, 2], device=DEV), empty(2, 2, 16)
    with pytest.raises(ValueError):
        c.embed_fwd(ids.int(), E, 1.0, x0)
    with pytest.raises(ValueError):
        c.embed_fwd(ids, E.half(), 1.0, x0)
    with pytest.raises(ValueError):
        c.embed_fwd(ids, E, 1.0, empty(2, 3, 16))
    with pytest.raises(ValueError):
        c.embed_fwd(ids.cpu(), E, 1.0, x0)
    ids = torch.zeros(1000, dtype=torch.int64, device=DEV)
    lib, g, dE = c.lib, randn(2, 1000, 2, 16), empty(10, 16, dtype=F32)
    need = lib.mhclite_embed_scratch_bytes(16, 1000, 10)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    args = (c._h, 1000, 10, ids.data_ptr(), g.data_ptr(), 1.0, dE.data_ptr(), 0)
    assert lib.mhclite_embed_bwd(*args, ws.data_ptr(), need - 1, None) == binding.ERR_WORKSPACE
    assert lib.mhclite_embed_bwd(*args, None, need, None) == binding.ERR_WORKSPACE
    assert lib.mhclite_embed_bwd(*args, ws.data_ptr() + 8, need, None) == binding.ERR_BAD_ARG
    c.embed_bwd(ids[:0], g[:0], 1.0, dE)
    assert (dE == 0).all()


# ---- cross entropy -----------------------------------------------------------------------------------------------------
LOSSES = [  # T, C, V, scale
    (1, 8, 1, 1.0), (1, 64, 50, 1.0), (1, 2048, 5001, 1.0), (3, 72, 257, 0.5), (127, 64, 256, 1.0), (128, 128, 255, 2.0), (129, 200, 1000, 1.0),
    (300, 1024, 2001, 1.0), (700, 520, 3333, 0.7), (257, 1536, 515, 1.0),
    (8, 64, 33, 1.0), (9, 72, 100, 1.0), (16, 1536, 20001, 1.0), (17, 4096, 777, 1.0), (31, 264, 5000, 0.5), (32, 1000, 4099, 1.0), (32, 4096, 600, 1.0),
    (33, 128, 3000, 1.0), (2, 8, 70001, 1.0),
]


def loss_case(T, C, V, ignored=0.2, seed=0):
    h, W = randn(seed + 1, T, C), randn(seed + 2, V, C, std=2.0 / np.sqrt(C))
    r = np.random.default_rng(seed + 3)
    target = r.integers(0, V, T)
    target[r.random(T) < ignored] = -100
    return h, W, torch.from_numpy(target).to(DEV), randn(seed + 4, T, dtype=F32)


def check_loss(c, h, W, target, scale, dloss):
    (T, C), V = h.shape, W.shape[0]
    loss, lse = empty(T, dtype=F32), empty(T, dtype=F32)
    c.linear_ce_fwd(h, W, target, scale, loss, lse)
    tg = target.cpu().numpy()
    H, Wd = np.nan_to_num(f64(h)), f64(W)
    rl, rs = S.linear_ce_fwd(H, Wd, tg, scale)
    # a logit: products exact, C / 16 steps of 16 added in fp32 with up to a unit in the last place each
    el = abs(scale) * (C / 16 + 4) * 2.0 ** -23 * (np.abs(H) @ np.abs(Wd).T).max(1)
    # exp2 / log2 approximations: 2^-22 of each factor, and V / 256 + 64 additions of one sign
    es = (V / 256 + 64) * 2.0 ** -24 + 2.0 ** -21 * (1 + np.abs(rs))
    ok = (tg >= 0) & (tg < V)
    close("lse", lse, rs, np.where(ok, el + es, 0))
    close("loss", loss, rl, np.where(ok, 2 * el + es, 0))
    dh, dW = empty(T, C), empty(V, C)
    c.linear_ce_bwd(h, W, target, scale, lse, dloss, dh, dW)
    rh, rW, G = S.linear_ce_bwd(H, Wd, tg, scale, f64(dloss))
    # G: exp(l - lse) off by the errors above, then rounded to bf16; the output rounded to bf16
    P = np.where(ok[:, None], np.abs(G) + 0, 0)
    hot = np.zeros_like(P)
    hot[np.flatnonzero(ok), tg[ok]] = np.abs(scale * f64(dloss))[ok]
    eG = HALF * P + (2 * el + 2 * es)[:, None] * (P + hot)
    # below 2^-126, the smallest normal number of fp32 and of bf16, a value may become 0: exp2 flushes, then the product
    # with dloss, then the product with an element of W or h.  Each flush is off by at most 2^-126 (times what follows).
    tiny = 2.0 ** -126
    eG += tiny * (1 + np.abs(scale * f64(dloss)))[:, None]
    Hz = np.where(ok[:, None], H, 0)
    close("dh", dh, rh, HALF * np.abs(rh) + (1 + HALF) * (eG @ np.abs(Wd)) + (V / 16 + 4) * 2.0 ** -23 * (P @ np.abs(Wd)) + (V + 1) * tiny)
    close("dW", dW, rW, HALF * np.abs(rW) + (1 + HALF) * (eG.T @ np.abs(Hz)) + (T / 16 + 4) * 2.0 ** -23 * (P.T @ np.abs(Hz)) + (T + 1) * tiny)
    # the roundings are independent: in the 2-norm they add up as a random walk.  Four times its length is allowed.
    for name, got, ref, e in (("dh", dh, rh, (P ** 2) @ (Wd ** 2)), ("dW", dW, rW, (P ** 2).T @ (Hz ** 2))):
        off = np.linalg.norm(f64(got) - ref)
        slack = (2 * el + 2 * es).max() * np.linalg.norm((P + hot) @ np.abs(Wd) if name == "dh" else (P + hot).T @ np.abs(Hz))
        assert off <= HALF * np.linalg.norm(ref) + 4 * HALF * np.sqrt(e.sum()) + slack, name
    return loss, lse, dh, dW


@pytest.mark.parametrize("T,C,V,scale", LOSSES)
def test_linear_ce(ctx_of, T, C, V, scale):
    h, W, target, dloss = loss_case(T, C, V, 0.0 if T == 1 else 0.2)
    check_loss(ctx_of(4, C), h, W, target, scale, dloss)


def test_linear_ce_rows_without_target_may_hold_anything(ctx_of):
    h, W, target, dloss = loss_case(300, 64, 700, 0.3)
    h[target < 0] = float("nan")
    dloss[target < 0] = float("inf")
    _, _, dh, _ = check_loss(ctx_of(4, 64), h, W, target, 1.0, torch.nan_to_num(dloss, posinf=0.0))
    c, (T, C), V = ctx_of(4, 64), h.shape, W.shape[0]
    loss, lse, dh2, dW2 = empty(T, dtype=F32), empty(T, dtype=F32), empty(T, C), empty(V, C)
    c.linear_ce_fwd(h, W, target, 1.0, loss, lse)
    c.linear_ce_bwd(h, W, target, 1.0, lse, dloss, dh2, dW2)
    assert torch.equal(dh, dh2) and torch.isfinite(dW2).all()


@pytest.mark.parametrize("T", [1, 200])
def test_linear_ce_no_row_has_a_target(ctx_of, T):
    h, W, target, dloss = loss_case(T, 64, 300)
    target.fill_(-1)
    loss, lse, dh, dW = check_loss(ctx_of(4, 64), h, W, target, 1.0, dloss)
    assert (loss == 0).all() and (lse == 0).all() and (dh == 0).all() and (dW == 0).all()


def test_linear_ce_only_the_last_row_has_a_target(ctx_of):
    h, W, target, dloss = loss_case(1000, 64, 300)
    target[:-1] = -1
    target[-1] = 299
    check_loss(ctx_of(4, 64), h, W, target, 1.0, dloss)


def test_linear_ce_in_several_pieces(ctx_of):
    """16384 tokens and 20000 columns do not fit one piece: dh adds up over three."""
    T, C, V = 16384, 64, 20001
    c = ctx_of(4, C)
    assert binding.load().mhclite_linear_ce_scratch_bytes(C, T, V, 1) < T * V * 2
    h, W, target, dloss = loss_case(T, C, V, 0.1)
    loss, lse, dh, dW = empty(T, dtype=F32), empty(T, dtype=F32), empty(T, C), empty(V, C)
    c.linear_ce_fwd(h, W, target, 1.0, loss, lse)
    c.linear_ce_bwd(h, W, target, 1.0, lse, dloss, dh, dW)
    hd, Wd, ok = h.double(), W.double(), target >= 0
    l = hd @ Wd.T
    rs = torch.logsumexp(l, 1)
    G = torch.softmax(l, 1)
    rl = rs - l.gather(1, target.clamp(min=0)[:, None])[:, 0]
    G.scatter_add_(1, target.clamp(min=0)[:, None], torch.full((T, 1), -1.0, dtype=torch.float64, device=DEV))
    G *= (dloss.double() * ok)[:, None]
    el = (C / 16 + 4) * 2.0 ** -23 * (hd.abs() @ Wd.abs().T).amax(1) + (V / 256 + 64) * 2.0 ** -24 + 2.0 ** -21 * (1 + rs.abs())
    assert ((lse - rs * ok).abs() <= el).all() and ((loss - rl * ok).abs() <= 2 * el).all()
    for got, ref, e in ((dh, G @ Wd, (G ** 2) @ (Wd ** 2)), (dW, G.T @ hd, (G ** 2).T @ (hd ** 2))):
        assert (got.double() - ref).norm() <= HALF * ref.norm() + 4 * HALF * e.sum().sqrt()
    assert (dh[~ok] == 0).all()


def test_linear_ce_sharp_logits_and_ties(ctx_of):
    """Logits of hundreds: the largest is taken out before exp.  Equal rows of W give equal probabilities."""
    c, C, V = ctx_of(4, 64), 64, 300
    h, W, target, dloss = loss_case(40, C, V, 0.0)
    check_loss(c, h * 16, W * 4, target, 1.0, dloss)
    W[:] = W[0]
    loss, lse = empty(40, dtype=F32), empty(40, dtype=F32)
    c.linear_ce_fwd(h, W, target, 1.0, loss, lse)
    assert torch.allclose(loss, torch.full_like(loss, float(np.log(V))), rtol=0, atol=2e-5)


@pytest.mark.parametrize("T,V,scale", [(1, 1, 1.0), (7, 1, 1.0), (20, 301, 1.0), (60, 1, 1.0), (60, 700, 1.0), (60, 300, -0.7), (20, 300, -0.7)])
def test_linear_ce_of_likely_targets_keeps_its_digits(ctx_of, T, V, scale):
    """Logits around 60 whose largest is the target's: the loss is a small difference of large numbers.  A logit is one
    product of two bf16 numbers here, exact in fp32 before the scale."""
    c, C = ctx_of(4, 64), 64
    h, W = torch.zeros(T, C, dtype=BF, device=DEV), torch.zeros(V, C, dtype=BF, device=DEV)
    r = np.random.default_rng(T + V)
    h[:, 3] = torch.from_numpy(r.uniform(50, 70, T)).to(BF).to(DEV)
    target = torch.from_numpy(r.integers(0, V, T)).to(DEV)
    W[:, 3] = torch.from_numpy(r.uniform(0.5, 0.8, V)).to(BF).to(DEV)
    likely = int(target[0])
    W[likely, 3] = 1.0625
    W[:, 3] *= -1 if scale < 0 else 1
    target[: T // 2 + 1] = likely
    loss, lse = empty(T, dtype=F32), empty(T, dtype=F32)
    c.linear_ce_fwd(h, W, target, scale, loss, lse)
    rl, _ = S.linear_ce_fwd(f64(h), f64(W), target.cpu().numpy(), float(np.float32(scale)))
    # exp2 and log2 to 2^-22 each, up to V terms of one sign; the exponents, up to 150, are rounded once to fp32 and the base's
    # constant once: 2^-23 of them, which moves a term by 150 x 2^-23 x ln 2 < 2^-16 of itself
    close("loss", loss, rl, 2.0 ** -20 + 2.0 ** -16 * rl)
    assert (loss >= 0).all() and rl.min() < 1e-3


def test_linear_ce_targets_beyond_the_table_are_reported():
    c = binding.MhcLite(2, 64, 0)
    h, W, target, dloss = loss_case(50, 64, 100, 0.0)
    target[7] = 100
    check_loss(c, h, W, target, 1.0, dloss)
    with pytest.raises(binding.MhcLiteError) as e:
        c.device_status()
    assert e.value.status == binding.ERR_INDEX


def test_linear_ce_refusals(ctx_of):
    c = ctx_of(4, 64)
    h, W, target, dloss = loss_case(20, 64, 100)
    loss, lse, dh, dW = empty(20, dtype=F32), empty(20, dtype=F32), empty(20, 64), empty(100, 64)
    bad = binding.MhcLiteError
    for s in (float("nan"), float("inf")):
        with pytest.raises(bad):
            c.linear_ce_fwd(h, W, target, s, loss, lse)
    with pytest.raises(ValueError):
        c.linear_ce_fwd(h, W.float(), target, 1.0, loss, lse)
    with pytest.raises(ValueError):
        c.linear_ce_fwd(h, W, target.int(), 1.0, loss, lse)
    with pytest.raises(ValueError):
        c.linear_ce_fwd(h, W[:, :32], target, 1.0, loss, lse)
    with pytest.raises(bad):
        c.linear_ce_fwd(h, W, target, 1.0, loss, loss)
    c.linear_ce_fwd(h, W, target, 1.0, loss, lse)
    with pytest.raises(bad):
        c.linear_ce_bwd(h, W, target, 1.0, lse, dloss, h, dW)
    with pytest.raises(bad):
        c.linear_ce_bwd(h, W, target, 1.0, lse, dloss, dh, W)
    need = c.lib.mhclite_linear_ce_scratch_bytes(64, 20, 100, 0)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    assert c.lib.mhclite_linear_ce_fwd(c._h, 20, 100, h.data_ptr(), W.data_ptr(), target.data_ptr(), 1.0, loss.data_ptr(),
                                       lse.data_ptr(), ws.data_ptr(), need - 1, None) == binding.ERR_WORKSPACE
    c.linear_ce_bwd(h[:0], W, target[:0], 1.0, lse[:0], dloss[:0], dh[:0], dW)
    assert (dW == 0).all()


# ---- tensors that begin 16 bytes into their buffers ---------------------------------------------------------------------
def inside(t):
    """The same values in a view 16 bytes (one element, for int64: 8) into a buffer: the least alignment the calls allow."""
    k = max(1, 16 // t.element_size()) if t.dtype != torch.int64 else 1
    v = torch.empty(t.numel() + 2 * k, dtype=t.dtype, device=DEV)[k:k + t.numel()].view(t.shape)
    assert v.data_ptr() % 32 in (8, 16)
    return v.copy_(t)


class InnerViews:
    """A context whose calls get every tensor as such a view; what they wrote is copied back to the caller's tensors."""

    def __init__(self, c):
        self.c, self.n, self.C = c, c.n, c.C

    def __getattr__(self, name):
        def call(*args, **kw):
            views = [inside(a) if torch.is_tensor(a) else a for a in args]
            getattr(self.c, name)(*views, **kw)
            for a, v in zip(args, views):
                if torch.is_tensor(a) and a.dtype != torch.int64:
                    a.copy_(v)
        return call


# (up to 256 columns the product dh = G W is not split, and its tiles go straight to dh)
@pytest.mark.parametrize("T,C,V", [(40, 64, 200), (300, 72, 256), (300, 128, 2001), (3, 64, 500), (1, 1024, 300)])
def test_linear_ce_on_inner_views(ctx_of, T, C, V):
    h, W, target, dloss = loss_case(T, C, V, 0.0 if T == 1 else 0.2)
    check_loss(InnerViews(ctx_of(4, C)), h, W, target, 1.0, dloss)


@pytest.mark.parametrize("T,C,V,f32", [(5, 64, 40, True), (300, 72, 300, False), (7000, 16, 50, True)])
def test_embed_on_inner_views(ctx_of, T, C, V, f32):
    c = ctx_of(3, C)
    E, ids = randn(1, V, C, dtype=F32 if f32 else BF), torch.from_numpy(some_ids(2, T, V, "text")).to(DEV)
    x0, x1, dE, dE1, g = empty(T, 3, C), empty(T, 3, C), empty(V, C, dtype=F32), empty(V, C, dtype=F32), randn(3, T, 3, C)
    for k, x, d in ((c, x0, dE), (InnerViews(c), x1, dE1)):
        k.embed_fwd(ids, E, 1.5, x)
        k.embed_bwd(ids, g, 1.5, d)
    assert torch.isfinite(x0).all() and torch.equal(x0, x1) and torch.isfinite(dE).all() and torch.equal(dE, dE1)


@pytest.mark.parametrize("T,C,gated,p", [(2, 64, True, 0.2), (700, 1536, False, 0.1), (300, 1040, True, 0.0)])
def test_block_and_dropout_on_inner_views(ctx_of, T, C, gated, p):
    c, rng = ctx_of(4, C), rng_of(8, 9)
    o, gate, dy = randn(1, T, C), randn(2, T, C) if gated else None, randn(3, T, C)
    w, s, outs = randn(4, C, mean=1.0, dtype=F32), torch.full((1,), 0.3, device=DEV), []
    for k in (c, InnerViews(c)):
        y, r, d_o, dg = empty(T, C), empty(T, dtype=F32), empty(T, C), empty(T, C) if gated else None
        dw, ds, z = empty(C, dtype=F32), empty(1, dtype=F32), empty(T, C)
        k.block_out_fwd(o, gate, w, s, 1e-6, p, rng, y, r)
        k.block_out_bwd(o, gate, w, s, r, p, rng, dy, d_o, dg, dw, ds)
        k.dropout(o, 0.4, rng, z)
        outs.append([t for t in (y, r, d_o, dg, dw, ds, z) if t is not None])
    for a, b in zip(*outs):
        assert torch.isfinite(a).all() and torch.equal(a, b)


# ---- offsets beyond 32 bits --------------------------------------------------------------------------------------------
def test_offsets_beyond_32_bits_rows(ctx_of):
    """1.1 M rows of 2048 channels: more than 2^31 elements, 4.5 GB of bf16.  The last rows give what they give alone."""
    c, C, T, m = ctx_of(2, 2048), 2048, 1_100_000, 7
    x = torch.empty(T, C, dtype=BF, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(1))
    w, y, r = randn(2, C, std=0.2, mean=1.0, dtype=F32), torch.empty(T, C, dtype=BF, device=DEV), torch.empty(T, device=DEV)
    c.block_in_fwd(x, w, 1e-6, y, r)
    y2, r2 = empty(m, C), empty(m, dtype=F32)
    c.block_in_fwd(x[-m:].clone(), w, 1e-6, y2, r2)
    assert torch.equal(y[-m:], y2) and torch.equal(r[-m:], r2)
    rng = rng_of(4, 2)
    c.dropout(x, 0.5, rng, y)
    g0 = (T - m) * C // 8                                       # the mask of the last rows, from the oracle's counter
    keep = np.array([[((S.philox4x32((g & 0xFFFFFFFF, g >> 32, 2, 0), (4, 0))[e // 2] >> (16 * (e % 2))) & 0xFFFF) >= 32768
                      for e in range(8)] for g in range(g0, g0 + m * C // 8)]).reshape(m, C)
    ref = np.where(keep, f64(x[-m:]) * 2.0, 0.0)
    close("dropout", y[-m:], ref, HALF * np.abs(ref))
    du, dw = y, empty(C, dtype=F32)
    c.block_in_bwd(x, w, r, x, du, dw)
    du2, dw2 = empty(m, C), empty(C, dtype=F32)
    c.block_in_bwd(x[-m:].clone(), w, r[-m:].clone(), x[-m:].clone(), du2, dw2)
    assert torch.equal(du[-m:], du2)


def test_offsets_beyond_32_bits_tables(ctx_of):
    """A table and a head of 1.1 M rows x 2048: the last rows lie beyond 2^31 elements."""
    c, C, V, n = ctx_of(2, 2048), 2048, 1_100_000, 2
    W = torch.empty(V, C, dtype=BF, device=DEV).normal_(std=0.02, generator=torch.Generator(device=DEV).manual_seed(1))
    ids = torch.tensor([V - 1, 5, V - 2, V - 1], device=DEV)
    x0 = empty(4, n, C)
    c.embed_fwd(ids, W, 2.0, x0)
    assert torch.equal(x0, (W[ids].float() * 2.0).to(BF)[:, None, :].expand(4, n, C))
    dE = torch.full((V, C), 3.0, device=DEV)
    c.embed_bwd(ids, torch.ones(4, n, C, dtype=BF, device=DEV), 0.5, dE)
    assert (dE[V - 1] == 2.0).all() and (dE[V - 2] == 1.0).all() and (dE[5] == 1.0).all()
    dE[[5, V - 1, V - 2]] = 0
    assert not dE.any()
    del dE
    for T in (3, 40):                                           # the streaming kernel and the tiles
        h, target = randn(7, T, C), torch.full((T,), V - 1, device=DEV)
        target[1] = 12
        loss, lse, dl = empty(T, dtype=F32), empty(T, dtype=F32), torch.ones(T, device=DEV)
        c.linear_ce_fwd(h, W, target, 1.0, loss, lse)
        parts = [h.double() @ W[v:v + 100_000].double().T for v in range(0, V, 100_000)]
        ref = torch.logsumexp(torch.cat([torch.logsumexp(p, 1)[:, None] for p in parts], 1), 1)
        tl = (h.double() * W[target].double()).sum(1)
        # logits of about 1: 128 steps of 16 products, V / 256 sums; as in check_loss
        assert (lse - ref).abs().max() < 1e-4 and (loss - (ref - tl)).abs().max() < 1e-4
        dh, dW = empty(T, C), torch.empty(V, C, dtype=BF, device=DEV)
        c.linear_ce_bwd(h, W, target, 1.0, lse, dl, dh, dW)
        p = torch.exp(parts[-1] - ref[:, None])                 # the last piece of 100 000 rows
        p[:, -1] -= (target == V - 1).double()
        want = p.T @ h.double()
        assert (dW[-100_000:].double() - want).norm() <= 2 * HALF * want.norm()
        del dW, parts


# ---- marshalling -------------------------------------------------------------------------------------------------------
def test_scratch_that_cannot_be_had_is_an_error_not_an_abort(ctx_of):
    c, T, V = ctx_of(4, 64), 4096, 60000
    h, W, target, dloss = loss_case(T, 64, V, 0.0)
    lse, dh, dW = torch.zeros(T, device=DEV), empty(T, 64), empty(V, 64)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    total = torch.cuda.get_device_properties(0).total_memory
    torch.cuda.set_per_process_memory_fraction((torch.cuda.memory_reserved() + (8 << 20)) / total)
    try:
        with pytest.raises(torch.OutOfMemoryError):
            c.linear_ce_bwd(h, W, target, 1.0, lse, dloss, dh, dW)
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    check_loss(c, h[:40], W[:300].contiguous(), target[:40] % 300, 1.0, dloss[:40].contiguous())


def test_arguments_of_other_kinds_are_refused(ctx_of):
    c, x, r = ctx_of(4, 64), randn(1, 4, 64), rng_of(1, 2)
    for bad in (None, 3, "x", [1.0]):
        with pytest.raises(TypeError):
            c.dropout(bad, 0.1, r, x)
    with pytest.raises(TypeError):
        c.dropout(x, "much", r, empty(4, 64))
    with pytest.raises(ValueError):
        c.dropout(x.cpu(), 0.1, r, empty(4, 64))
    with pytest.raises(ValueError):
        c.block_in_fwd(torch.zeros((), dtype=BF, device=DEV), r, 1e-6, x, x)


# ---- streams, graphs, repeated runs ------------------------------------------------------------------------------------
def test_two_streams_at_once_and_bitwise_repeats(ctx_of):
    c = ctx_of(4, 256)
    h, W, target, dloss = loss_case(500, 256, 3001)
    ids, g = torch.from_numpy(some_ids(1, 500, 3001, "text")).to(DEV), randn(9, 500, 4, 256)
    loss, lse, _, _ = check_loss(c, h, W, target, 1.0, dloss)
    torch.cuda.synchronize()
    outs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams * 3:
        with torch.cuda.stream(s):
            o = [empty(500, 256), empty(3001, 256), empty(3001, 256, dtype=F32), empty(500, dtype=F32), empty(500, dtype=F32)]
            c.linear_ce_fwd(h, W, target, 1.0, o[3], o[4])
            c.linear_ce_bwd(h, W, target, 1.0, o[4], dloss, o[0], o[1])
            c.embed_bwd(ids, g, 1.0, o[2])
            outs.append(o)
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))
    assert torch.equal(outs[0][3], loss) and torch.equal(outs[0][4], lse)


def test_captured_and_replayed_with_new_inputs(ctx_of):
    """Two graphs, each with scratch of its own; between replays the inputs and the dropout offset change."""
    c, T, C, V = ctx_of(4, 256), 200, 256, 1000
    h, W, target, dloss = loss_case(T, C, V)
    w, rng, gate = randn(5, C, std=0.2, mean=1.0, dtype=F32), rng_of(5, 0), randn(6, T, C)
    s = torch.full((1,), 0.5, device=DEV)

    def step(buf):
        c.block_out_fwd(h, gate, w, s, 1e-6, 0.2, rng, buf["y"], buf["r"])
        c.linear_ce_fwd(buf["y"], W, target, 1.0, buf["loss"], buf["lse"])
        c.linear_ce_bwd(buf["y"], W, target, 1.0, buf["lse"], dloss, buf["dh"], buf["dW"])
        c.block_out_bwd(h, gate, w, s, buf["r"], 0.2, rng, buf["dh"], buf["d_o"], buf["dg"], buf["dw"], buf["ds"])

    def buffers():
        return {"y": empty(T, C), "r": empty(T, dtype=F32), "loss": empty(T, dtype=F32), "lse": empty(T, dtype=F32), "dh": empty(T, C),
                "dW": empty(V, C), "d_o": empty(T, C), "dg": empty(T, C), "dw": empty(C, dtype=F32), "ds": empty(1, dtype=F32)}
    bufs, graphs, side = [buffers(), buffers()], [], torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(bufs[0])
    torch.cuda.synchronize()
    for b in bufs:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            step(b)
        graphs.append(gr)
    for k in range(3):
        rng[1] = k
        h.copy_(randn(100 + k, T, C))
        target.copy_(torch.from_numpy(some_ids(k, T, V, "even")).to(DEV))
        target[k::7] = -1
        torch.cuda.synchronize()
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        ref = buffers()
        step(ref)
        for b in bufs:
            for name in ref:
                assert torch.equal(b[name], ref[name]), (k, name)


def test_inputs_that_another_stream_writes(ctx_of):
    """A kernel that may start beside the one before it still waits for what its stream waits for."""
    c, T, C, side = ctx_of(4, 256), 300, 256, torch.cuda.Stream()
    x, w = torch.zeros(T, C, dtype=BF, device=DEV), torch.ones(C, device=DEV)
    new, rng = randn(1, T, C), rng_of(1, 2)
    y, v, r, z = empty(T, C), empty(T, C), empty(T, dtype=F32), empty(T, C)
    c.dropout(new, 0.5, rng, z)
    c.block_in_fwd(new, w, 1e-6, v, r)
    want, torch_done = (v.clone(), z.clone()), torch.cuda.Event()
    torch.cuda.synchronize()
    for _ in range(3):
        x.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(5_000_000)
            x.copy_(new)
            torch_done.record()
        c.dropout(new, 0.5, rng, y)                                      # the kernel before, which lets the next one begin
        torch.cuda.current_stream().wait_event(torch_done)
        c.block_in_fwd(x, w, 1e-6, v, r)
        c.dropout(x, 0.5, rng, z)
        torch.cuda.synchronize()
        assert torch.equal(v, want[0]) and torch.equal(z, want[1])


def test_captured_behind_copies_and_joined_streams(ctx_of):
    """In a graph a call may follow a copy, a clearing, or several nodes of joined streams, not only a kernel."""
    c, T, C, V, rows, n = ctx_of(4, 256), 7000, 256, 3000, 40000, 4      # a table of which part is cleared beside the sort
    src, g, ids = randn(1, T, n, C), torch.zeros(T, n, C, dtype=BF, device=DEV), torch.from_numpy(some_ids(2, T, rows, "text")).to(DEV)
    none, w, side = ids[:0], torch.ones(C, device=DEV), torch.cuda.Stream()
    h, W, target, dloss = loss_case(T, C, V)
    b = {"dE": empty(rows, C, dtype=F32), "dE2": empty(rows, C, dtype=F32), "v": empty(T, C), "r": empty(T, dtype=F32), "z": empty(T, C), "loss": empty(T, dtype=F32),
         "lse": empty(T, dtype=F32), "dh": empty(T, C), "dW": empty(V, C)}
    x, rng = torch.zeros(T, C, dtype=BF, device=DEV), rng_of(3, 4)

    def step():
        g.copy_(src)                                                     # a copy
        c.embed_bwd(ids, g, 0.5, b["dE"])
        c.embed_bwd(none, g[:0], 0.5, b["dE"])                           # no tokens: a clearing
        c.embed_bwd(ids, g, 0.5, b["dE"], accumulate=True)
        b["dE2"].copy_(b["dE"])                                          # read before the next call clears it
        c.embed_bwd(ids, g, 2.0, b["dE"])
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        with torch.cuda.stream(side):
            x.copy_(h)
            c.block_in_fwd(x, w, 1e-6, b["v"], b["r"])
        c.linear_ce_fwd(h, W, target, 1.0, b["loss"], b["lse"])
        main.wait_stream(side)
        c.dropout(b["v"], 0.25, rng, b["z"])                             # two nodes before it
        c.linear_ce_bwd(b["z"], W, target, 1.0, b["lse"], dloss, b["dh"], b["dW"])
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        src.copy_(randn(10 + k, T, n, C))
        h.copy_(randn(20 + k, T, C))
        torch.cuda.synchronize()
        step()
        torch.cuda.synchronize()
        want = {name: t.clone() for name, t in b.items()}
        assert torch.equal(want["dE"], 4 * want["dE2"])                  # powers of two: exact
        for t in (*b.values(), x):
            t.fill_(float("nan"))
        g.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in b:
            assert torch.isfinite(want[name]).all() and torch.equal(b[name], want[name]), name


# ---- status words ------------------------------------------------------------------------------------------------------
BUSY = 100_000_000                  # cycles a stream is kept busy: some 50 ms


def test_status_words_are_cleared_behind_work_on_other_streams():
    """What is queued on any stream when the words are attached has no part in what they say afterwards."""
    c, side = binding.MhcLite(2, 16, 0), torch.cuda.Stream()
    words = torch.zeros(8, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
        words.fill_(binding.ERR_INDEX)
    assert c.lib.mhclite_set_status_words(c._h, words.data_ptr()) == binding.OK
    assert (words == 0).all()
    c.device_status()
    # cleared once the call is back: a report that follows at once, on another stream, stays
    torch.cuda._sleep(BUSY)
    assert c.lib.mhclite_set_status_words(c._h, words.data_ptr()) == binding.OK
    with torch.cuda.stream(side):
        c.embed_fwd(torch.tensor([99], device=DEV), randn(1, 10, 16), 1.0, empty(1, 2, 16))
    torch.cuda.synchronize()
    assert words[0] == binding.ERR_INDEX


def test_context_made_on_a_side_stream_starts_clean():
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        last = torch.empty(8, dtype=torch.int32, device=DEV)
        torch.cuda._sleep(BUSY)
        last.fill_(binding.ERR_INDEX)
        del last                                                         # the next allocation of this size gets its memory
        c = binding.MhcLite(2, 16, 0)
    torch.cuda.synchronize()
    c.device_status()


def test_status_waits_for_work_on_other_streams():
    c, side, E, x0 = binding.MhcLite(2, 16, 0), torch.cuda.Stream(), randn(1, 10, 16), empty(1, 2, 16)
    ids = torch.tensor([99], device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
        c.embed_fwd(ids, E, 1.0, x0)
    with pytest.raises(binding.MhcLiteError) as e:
        c.device_status()
    assert e.value.status == binding.ERR_INDEX


def test_a_report_hides_no_other():
    """The words, as kernels leave them: an index in 0 to 4, a wait that gave up in 5 to 7 (kernel, wait and block in one)."""
    c, words = binding.MhcLite(2, 16, 0), torch.zeros(8, dtype=torch.int32, device=DEV)
    assert c.lib.mhclite_set_status_words(c._h, words.data_ptr()) == binding.OK
    c.embed_fwd(torch.tensor([1, 99], device=DEV), randn(1, 10, 16), 1.0, empty(2, 2, 16))
    torch.cuda.synchronize()
    assert words.tolist() == [binding.ERR_INDEX, 20, 99, 0, 1, 0, 0, 0]
    words[5], words[6], words[7] = binding.ERR_TIMEOUT, 122 | 4 << 12 | 147 << 16, 77
    with pytest.raises(binding.MhcLiteError, match="kernel 122, wait 4, block 147, index 77") as e:
        c.device_status()
    assert e.value.status == binding.ERR_TIMEOUT
    words[5] = 0
    with pytest.raises(binding.MhcLiteError, match="index 99 .* at token 1$") as e:
        c.device_status()
    assert e.value.status == binding.ERR_INDEX


def test_reports_can_be_cleared():
    c, E, x0 = binding.MhcLite(2, 16, 0), randn(1, 10, 16), empty(3, 2, 16)
    c.premix_fwd(randn(2, 3, 2, 16), torch.full((3, 2), 0.5, device=DEV), empty(3, 16))
    c.ensure_workspace(64)
    for ids, at in (([1, 99, 2], 1), ([1, 2, -4], 2)):
        c.embed_fwd(torch.tensor(ids, device=DEV), E, 1.0, x0)
        with pytest.raises(binding.MhcLiteError, match="at token %d$" % at):
            c.device_status()
        with pytest.raises(binding.MhcLiteError):
            c.device_status()                                            # it stays until it is cleared
        c.clear_device_status()
        c.device_status()


def test_graph_that_outlives_its_context_writes_to_no_other_tensor():
    E, x0, ids = randn(1, 10, 16), empty(2, 2, 16), torch.tensor([1, 2], device=DEV)
    c = binding.MhcLite(2, 16, 0)
    c.embed_fwd(ids, E, 1.0, x0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.embed_fwd(ids, E, 1.0, x0)
    del c
    others = [torch.zeros(8, dtype=torch.int32, device=DEV) for _ in range(4000)]
    ids.fill_(99)
    graph.replay()
    torch.cuda.synchronize()
    assert (x0 == 0).all() and not any(t.any().item() for t in others)


# ---- a whole model step ------------------------------------------------------------------------------------------------
def test_model_step_runs_and_its_gradients_match_differences():
    """ids -> loss through two mixing layers with a gated sublayer, dropout on, and back.  The activations between the
    calls are bf16, so a difference of two losses is only as fine as their roundings: the loss is computed in fp64 by a
    plain restatement of the model without them, and differenced there along the library's own gradient."""
    n, C, T, V, layers, p = 4, 64, 96, 200, 2, 0.1
    c = binding.MhcLite(n, C, 0)
    r = np.random.default_rng(0)
    mk = lambda *s, std=1.0, mean=0.0: (r.normal(size=s) * std + mean).astype(np.float32)
    Ps = [L.LayerParams(mk(n * C, 32, std=0.02), mk(32, std=0.1), np.full(3, 0.5, np.float32), mk(n * C, std=0.1, mean=1.0), DEV) for _ in range(layers)]
    Ks = [L.BlockParams(mk(C, std=0.1, mean=1.0), mk(C, std=0.1, mean=1.0), [0.7], DEV, p) for _ in range(layers)]
    Bs, KBs = [L.LayerBuffers(c, T) for _ in range(layers)], [L.BlockBuffers(c, T, True) for _ in range(layers)]
    E, wf = torch.from_numpy(mk(V, C, std=0.5)).to(DEV), torch.from_numpy(mk(C, std=0.1, mean=1.0)).to(DEV)
    M = L.ModelEnds(c, T, E, 1.3, wf, randn(5, V, C, std=0.1), 1.0)
    ids = torch.from_numpy(some_ids(3, T, V, "text")).to(DEV)
    target = torch.from_numpy(some_ids(4, T, V, "even")).to(DEV)
    target[::5] = -100
    live = int((target >= 0).sum())
    dloss = torch.full((T,), 1.0 / live, device=DEV)
    rng = torch.tensor([[9, 0], [9, 1]], dtype=torch.int64, device=DEV)
    inner = lambda l, v: (torch.tanh(v.float()).to(BF), (0.5 * v.float()).to(BF))

    def inner_bwd(l, v, d_o, dgate):
        v = v.float()
        return (d_o.float() * (1 - torch.tanh(v) ** 2) + 0.5 * dgate.float()).to(BF).contiguous()
    f = L.block_sublayer(c, Ks, KBs, inner, rng)
    fb = L.block_sublayer_bwd(c, Ks, KBs, inner_bwd, rng)
    loss = L.model_fwd(c, M, Ps, Bs, ids, target, f)
    L.model_bwd(c, M, Ps, Bs, ids, target, dloss, fb)
    torch.cuda.synchronize()
    assert c.device_status() in (None, 0)

    import itertools
    perms = torch.tensor(list(itertools.permutations(range(n))), device=DEV)
    keeps = [torch.from_numpy(S.keep_mask(T * C, p, 9, l).reshape(T, C)).to(DEV) for l in range(layers)]

    def plain(q):
        rms = lambda x: torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + 1e-6)
        x = (q["E"][ids] * 1.3)[:, None, :].expand(T, n, C)
        for l in range(layers):
            P = Ps[l]
            xf = x.reshape(T, n * C)
            z = (xf * rms(xf) * P.gain.double()) @ P.W.double() * 0.5 + P.b.double()
            a, pre, post = torch.softmax(z[:, :24], 1), torch.sigmoid(z[:, 24:28]), 2 * torch.sigmoid(z[:, 28:])
            H = torch.zeros(T, n, n, dtype=torch.float64, device=DEV)
            for k in range(24):
                H[:, torch.arange(n), perms[k]] += a[:, k, None]
            u = torch.einsum("tj,tjc->tc", pre, x)
            v = u * rms(u) * q["w_in%d" % l]
            o = torch.tanh(v)
            y = o * rms(o) * q["w_out%d" % l] * torch.sigmoid(0.5 * v) * keeps[l] * S.drop_factor(p) * q["s%d" % l]
            x = torch.einsum("tij,tjc->tic", H, x) + post[:, :, None] * y[:, None, :]
        m = x.mean(1)
        logits = (m * rms(m) * q["wf"]) @ q["W"].T
        t = target.clamp(min=0)
        return (torch.logsumexp(logits, 1) - logits.gather(1, t[:, None])[:, 0]) * (target >= 0)
    q = {"E": E.double(), "wf": wf.double(), "W": M.W.double()}
    grads = {"E": M.dE, "wf": M.dw, "W": M.dW}
    for l in range(layers):
        q.update({"w_in%d" % l: Ks[l].w_in.double(), "w_out%d" % l: Ks[l].w_out.double(), "s%d" % l: Ks[l].scale.double()})
        grads.update({"w_in%d" % l: KBs[l].dw_in, "w_out%d" % l: KBs[l].dw_out, "s%d" % l: KBs[l].dscale})
    ref = plain(q)
    # about ten bf16 tensors lie between the ids and a logit: each moves a logit of size ~1 by some 2^-8
    assert (loss.double() - ref).abs().max() <= 10 * HALF * (1 + ref.abs().max())
    for name, g in grads.items():
        g = g.double()
        d = g / g.norm()
        h = 1e-4
        up, down = dict(q), dict(q)
        up[name], down[name] = q[name] + h * d, q[name] - h * d
        diff = ((plain(up) - plain(down)).sum() / live / (2 * h)).item()
        # along its own direction a gradient with relative error e (2-norm) differences to its norm within e: some
        # twenty bf16 roundings of half a step each on the longest way back
        assert diff == pytest.approx(g.norm().item(), rel=20 * HALF), name
