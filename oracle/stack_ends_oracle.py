"""fp64 definitions of the operators around a stack of mixing layers, in plain numpy: the lookup into the residual streams,
the norms that enclose a sublayer, dropout from a counter-based generator, and the cross entropy of the last hidden rows.
Written from the formulas, without code of the library."""
import numpy as np

PHILOX_M = (0xD2511F53, 0xCD9E8D57)
PHILOX_W = (0x9E3779B9, 0xBB67AE85)


def philox4x32(counter, key, rounds=10):
    """One block of Philox4x32 (Salmon et al. 2011) in Python integers: four 32-bit words."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        a, b = PHILOX_M[0] * c[0], PHILOX_M[1] * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[i] + PHILOX_W[i]) & 0xFFFFFFFF for i in (0, 1)]
    return c


def drop_threshold(p):
    return int(np.floor(p * 65536.0 + 0.5))


def keep_mask(count, p, seed, offset):
    """Which of `count` elements stay: 16 bits of group i // 8, half-word i % 8, at least round(65536 p)."""
    seed, offset = int(seed) & (2**64 - 1), int(offset) & (2**64 - 1)
    key = (seed & 0xFFFFFFFF, seed >> 32)
    out = np.zeros(count, dtype=bool)
    for g in range((count + 7) // 8):
        w = philox4x32((g & 0xFFFFFFFF, g >> 32, offset & 0xFFFFFFFF, offset >> 32), key)
        for e in range(min(8, count - 8 * g)):
            out[8 * g + e] = ((w[e // 2] >> (16 * (e % 2))) & 0xFFFF) >= drop_threshold(p)
    return out


def drop_factor(p):
    return 65536.0 / (65536 - drop_threshold(p))


def embed_fwd(ids, E, scale, n):
    V = E.shape[0]
    x = np.zeros((len(ids), E.shape[1]))
    ok = (ids >= 0) & (ids < V)
    x[ok] = E[ids[ok]] * scale
    return np.repeat(x[:, None, :], n, axis=1)


def embed_bwd(ids, g, scale, V):
    """(dE, sum of absolute terms): the second bounds what fp32 sums may be off."""
    dE, mag = np.zeros((V, g.shape[2])), np.zeros((V, g.shape[2]))
    for t, v in enumerate(ids):
        if 0 <= v < V:
            dE[v] += scale * g[t].sum(0)
            mag[v] += abs(scale) * np.abs(g[t]).sum(0)
    return dE, mag


def sigmoid(a):
    return np.exp(-np.logaddexp(0.0, -a))


def block_out_fwd(o, gate, w, s, eps, keep=None, factor=1.0):
    """y = s drop(sigmoid(gate) o rstd w); gate may be None, keep the mask of the elements that stay."""
    r = 1.0 / np.sqrt((o * o).mean(1) + eps)
    z = o * r[:, None] * w
    if gate is not None:
        z = z * sigmoid(gate)
    if keep is not None:
        z = np.where(keep, z * factor, 0.0)
    return s * z, r


def block_out_bwd(o, gate, w, s, eps, dy, keep=None, factor=1.0):
    """Gradients and, for each, the magnitude of the terms that are added up in it."""
    r = 1.0 / np.sqrt((o * o).mean(1) + eps)[:, None]
    oh = o * r
    sg = np.ones_like(o) if gate is None else sigmoid(gate)
    d = dy if keep is None else np.where(keep, dy * factor, 0.0)
    z = d * s
    e = z * sg * w
    res = {
        "d_o": r * (e - oh * (e * oh).mean(1, keepdims=True)), "dw": (z * sg * oh).sum(0), "dscale": (d * sg * oh * w).sum(),
        "mag_d_o": r * (np.abs(e) + np.abs(oh) * np.abs(e * oh).mean(1, keepdims=True)), "mag_dw": np.abs(z * sg * oh).sum(0),
        "mag_dscale": np.abs(d * sg * oh * w).sum(),
    }
    if gate is not None:
        res["dgate"] = z * oh * w * sg * sigmoid(-gate)
    return res


def linear_ce_fwd(h, W, target, scale):
    """(loss, lse); rows without a target (negative, or V and more) have 0 in both."""
    V, T = W.shape[0], h.shape[0]
    loss, lse = np.zeros(T), np.zeros(T)
    ok = (target >= 0) & (target < V)
    l = scale * h[ok] @ W.T
    top = l.max(1) if l.size else np.zeros(0)
    lse[ok] = top + np.log(np.exp(l - top[:, None]).sum(1))
    loss[ok] = lse[ok] - l[np.arange(l.shape[0]), target[ok]]
    return loss, lse


def linear_ce_bwd(h, W, target, scale, dloss):
    """dh, dW and the bracket G = scale dloss (softmax - onehot) that both are products of."""
    V, T = W.shape[0], h.shape[0]
    ok = (target >= 0) & (target < V)
    G = np.zeros((T, V))
    l = scale * h[ok] @ W.T
    p = np.exp(l - l.max(1, keepdims=True)) if l.size else l
    p = p / p.sum(1, keepdims=True) if l.size else p
    p[np.arange(p.shape[0]), target[ok]] -= 1.0
    G[ok] = scale * dloss[ok][:, None] * p
    hz = np.where(ok[:, None], h, 0.0)
    return G @ W, G.T @ hz, G
