"""fp64 definitions of the losses behind a first training, in plain numpy: distillation from a teacher's top logits, the
clipped policy loss with a KL term, and the preference loss of paired sequences.  Written from the formulas, without code of
the library."""
import numpy as np


# ---- distillation ------------------------------------------------------------------------------------------------------
def teacher_weights(ids, z, tau, V):
    """(p, log p) [T, K] over the present entries of each row, and which rows have an entry of weight.  log p is -inf where
    the weight is 0."""
    there = (ids >= 0) & (ids < V)
    a = np.where(there, np.where(there, z, 0.0) / tau, -np.inf)
    live = (a != -np.inf).any(1)                         # an entry that is NaN makes its row NaN
    top = np.where(live, a.max(1, initial=-np.inf), 0.0)[:, None]
    with np.errstate(divide="ignore", invalid="ignore"):
        log_p = a - top - np.log(np.exp(a - top).sum(1, keepdims=True))
    log_p = np.where(live[:, None] & there, log_p, -np.inf)
    return np.exp(log_p), log_p, live


def log_softmax(x):
    top = x.max(1, keepdims=True)
    return x - top - np.log(np.exp(x - top).sum(1, keepdims=True))


def linear_distill_fwd(h, W, ids, z, scale, tau):
    """(loss [T], lse [T], logp [T, K]); 0 in rows without a teacher, logp 0 at absent entries."""
    V = W.shape[0]
    p, log_p, live = teacher_weights(ids, z, tau, V)
    x = (scale / tau) * np.where(live[:, None], h, 0.0) @ W.T
    lq = log_softmax(x)
    there = (ids >= 0) & (ids < V) & live[:, None]
    logp = np.where(there, np.take_along_axis(lq, np.where(there, ids, 0), 1), 0.0)
    with np.errstate(invalid="ignore"):
        loss = np.where(p != 0, p * (log_p - logp), 0.0).sum(1)
    return np.where(live, loss, 0.0), np.where(live, (x - lq)[:, 0], 0.0), logp


def linear_distill_bwd(h, W, ids, z, scale, tau, dloss):
    """dh, dW, the bracket's factor a = dloss scale / tau (0 without a teacher), q and the teacher's weights over the vocabulary."""
    T, V = h.shape[0], W.shape[0]
    p, _, live = teacher_weights(ids, z, tau, V)
    hz = np.where(live[:, None], h, 0.0)
    q = np.exp(log_softmax((scale / tau) * hz @ W.T))
    share = np.zeros((T, V))
    for k in range(ids.shape[1]):
        ok = np.flatnonzero((ids[:, k] >= 0) & (ids[:, k] < V) & live)
        share[ok, ids[ok, k]] += p[ok, k]
    a = np.where(live, np.where(live, dloss, 0.0) * scale / tau, 0.0)
    G = a[:, None] * (q - share)
    return G @ W, G.T @ hz, a, q, share


# ---- losses of sequences -----------------------------------------------------------------------------------------------
def tokens_of(starts, T):
    """The token range of each sequence: starts as they are, cut to [0, T]."""
    e = np.clip(starts, 0, T)
    return [(int(a), int(max(a, b))) for a, b in zip(e[:-1], e[1:])]


def policy_loss(nll, nll_old, nll_ref, target, starts, adv, token_adv, clip_low, clip_high, kl_weight, mean, dloss=None):
    """(loss [S], stats [S, 3] = tokens that count, clipped ones, divergence; dnll [T])."""
    T, S = len(nll), len(starts) - 1
    loss, stats, dnll = np.zeros(S), np.zeros((S, 3)), np.zeros(T)
    for s, (a, b) in enumerate(tokens_of(starts, T)):
        at = a + np.flatnonzero(target[a:b] >= 0)
        n = len(at)
        if n == 0:
            continue
        A = adv[at] if token_adv else np.full(n, adv[s])
        x = nll_old[at] - nll[at]
        r = np.exp(x)
        free, held = -A * r, -A * np.clip(r, 1 - clip_low, 1 + clip_high)
        # e^x is above 1 + c where x is above log(1 + c): the exponential of an x below 2^-53 would be rounded to 1
        with np.errstate(divide="ignore"):
            cut = ((x > np.log1p(clip_high)) & (A > 0)) | ((x < np.log1p(-clip_low)) & (A < 0))
        l, g = np.where(cut, held, free), np.where(cut, 0.0, A * r)
        kl = np.zeros(n)
        if nll_ref is not None:
            d = nll[at] - nll_ref[at]
            kl = np.expm1(d) - d
            l, g = l + kl_weight * kl, g + kl_weight * np.expm1(d)
        w = 1.0 / n if mean else 1.0
        loss[s], stats[s] = w * l.sum(), (n, cut.sum(), w * kl.sum())
        if dloss is not None:
            dnll[at] = dloss[s] * w * g
    return loss, stats, dnll


def softplus(x):
    return np.logaddexp(0.0, x)


def preference_loss(nll, nll_ref, target, starts, beta, margin, smoothing, mean, dloss=None):
    """(loss [P], reward [P, 2], dnll [T]) of the pairs of sequences 2 p (chosen) and 2 p + 1 (rejected)."""
    T, P = len(nll), (len(starts) - 1) // 2
    loss, reward, dnll = np.zeros(P), np.zeros((P, 2)), np.zeros(T)
    spans = tokens_of(starts, T)
    for p in range(P):
        ats, ws = [], []
        for j in (0, 1):
            a, b = spans[2 * p + j]
            at = a + np.flatnonzero(target[a:b] >= 0)
            ats.append(at)
            ws.append(1.0 / max(len(at), 1) if mean else 1.0)
            reward[p, j] = beta * ws[j] * ((0.0 if nll_ref is None else nll_ref[at]) - nll[at]).sum()
        x = reward[p, 0] - reward[p, 1] - margin
        loss[p] = (1 - smoothing) * softplus(-x) + smoothing * softplus(x)
        if dloss is not None:
            dx = dloss[p] * (smoothing - np.exp(-softplus(x)))
            for j, sign in ((0, -1.0), (1, 1.0)):
                dnll[ats[j]] = sign * beta * ws[j] * dx
    return loss, reward, dnll
