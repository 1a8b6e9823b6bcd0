"""What is timed of the losses that train a stack after its first training: distillation from a teacher's top logits, the
clipped policy loss with a KL term, and the preference loss of paired sequences.

Each pass runs either the plain form (elementary torch operations, 32 bits, 64 where 32 lose what matters, rounded once at
the end) or, with ``own`` set, the calls that a program makes of the library.  Activations and the head are bf16; log
probabilities, advantages and losses are fp32, as the library's cross entropy leaves and takes them.
"""
import math

import torch

own = False

_EPS_LOW, _EPS_HIGH, _KL = 0.2, 0.28, 0.04


# ---- the cases ------------------------------------------------------------------------------------------------------
def listed():
    return [
        # the divergence of one scored token from its teacher: one pass over the head's weights
        {"name": "distill_one", "op": "distill", "dir": "fwd", "T": 1, "K": 20, "C": 2048, "V": 50257, "teacher": "f32", "ragged": False},
        # a held-out batch is scored, no gradients
        {"name": "distill_eval", "op": "distill", "dir": "fwd", "T": 4099, "K": 256, "C": 1536, "V": 50257, "teacher": "f32", "ragged": False},
        # loss and gradients of a ragged batch: rows without a teacher, rows with fewer entries, entries in bf16
        {"name": "distill_odd", "op": "distill", "dir": "train", "T": 2047, "K": 50, "C": 1024, "V": 32001, "teacher": "bf16", "ragged": True},
        # loss and gradients of a training batch
        {"name": "distill_batch", "op": "distill", "dir": "train", "T": 16384, "K": 64, "C": 2048, "V": 50257, "teacher": "f32", "ragged": False},
        # a handful of short answers, with an advantage for each token: latency
        {"name": "policy_small", "op": "policy", "T": 1500, "S": 8, "ref": True, "token_adv": True, "mean": True, "grad": True},
        # a ragged batch, loss and gradients
        {"name": "policy_odd", "op": "policy", "T": 100003, "S": 61, "ref": True, "token_adv": False, "mean": True, "grad": True},
        # a few very long answers, summed over their tokens, without the KL term
        {"name": "policy_long", "op": "policy", "T": 2097169, "S": 3, "ref": False, "token_adv": False, "mean": False, "grad": True},
        # a large batch of sampled answers
        {"name": "policy_batch", "op": "policy", "T": 16777216, "S": 2048, "ref": True, "token_adv": False, "mean": True, "grad": True},
        # two pairs: latency
        {"name": "pair_small", "op": "pair", "T": 900, "P": 2, "ref": True, "mean": False, "margin": 0.0, "smooth": 0.0, "grad": True},
        # a ragged batch of pairs, with smoothed labels
        {"name": "pair_odd", "op": "pair", "T": 60001, "P": 37, "ref": True, "mean": False, "margin": 0.0, "smooth": 0.1, "grad": True},
        # many pairs, per-token means with a margin, without a reference model
        {"name": "pair_batch", "op": "pair", "T": 8388608, "P": 4096, "ref": False, "mean": True, "margin": 0.5, "smooth": 0.0, "grad": True},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["distill", "distill", "policy", "pair"])
    if op == "distill":
        C, V = 8 * _log(rng, 8, 512), _log(rng, 1000, 131072)
        T = min(_log(rng, 1, 16384), max(1, 16384 * 2048 * 50257 // (C * V)))
        return {"op": op, "dir": rng.choice(["fwd", "train"]), "T": T, "K": _log(rng, 1, 256), "C": C, "V": V,
                "teacher": rng.choice(["f32", "bf16"]), "ragged": rng.random() < 0.5}
    T = _log(rng, 1, 16777216)
    n = _log(rng, 1, max(1, min(T // 2, 65536)))
    if op == "policy":
        return {"op": op, "T": T, "S": n, "ref": rng.random() < 0.6, "token_adv": rng.random() < 0.4, "mean": rng.random() < 0.6, "grad": rng.random() < 0.8}
    return {"op": op, "T": T, "P": max(1, n // 2), "ref": rng.random() < 0.6, "mean": rng.random() < 0.4, "margin": rng.choice([0.0, 0.5]),
            "smooth": rng.choice([0.0, 0.1]), "grad": rng.random() < 0.8}


# ---- inputs ---------------------------------------------------------------------------------------------------------
class _Rng:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(self, *shape, std=1.0, mean=0.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=self.g, device="cuda") * std + mean).to(dtype)

    def uniform(self, *shape, dtype=torch.float32):
        return torch.rand(*shape, generator=self.g, device="cuda", dtype=dtype)

    def top_ids(self, T, K, V):
        """K distinct ids a row in no order, as unevenly spread as those of text: the density falls with 1 / (id + 1)."""
        u = self.uniform(T, K, dtype=torch.float64)
        ids = (torch.exp(u * math.log(V - K + 1)).long() - 1).clamp_(0, V - K)
        ids = ids.sort(1).values + torch.arange(K, device="cuda")
        return ids.gather(1, self.uniform(T, K).argsort(1))

    def starts(self, T, S):
        """T tokens cut into S sequences of uneven length, the last few tokens (padding) in none."""
        cuts = (self.uniform(S, dtype=torch.float64) + 0.25).cumsum(0)
        used = T - T // 64
        cuts = (cuts / cuts[-1] * used).long()
        cuts[-1] = used
        return torch.cat((torch.zeros(1, dtype=torch.int64, device="cuda"), cuts))


def _out(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device="cuda")


def _answers(s, r, T, S):
    """The tokens of S sampled answers: where each begins, which tokens count (not the prompt's), their log probabilities
    under the model in training and others near it."""
    s["starts"] = r.starts(T, S)
    at = torch.arange(T, device="cuda")
    seq = (torch.searchsorted(s["starts"], at, right=True) - 1).clamp_(0, S - 1)
    length = s["starts"][1:] - s["starts"][:-1]
    prompt = (length.double() * 0.5 * r.uniform(S, dtype=torch.float64)).long()
    s["target"] = torch.randint(0, 50257, (T,), generator=r.g, device="cuda")
    s["target"][at - s["starts"][seq] < prompt[seq]] = -100
    u = r.uniform(T)
    s["nll"] = -torch.log(1 - 0.999 * u * u)
    if s["op"] == "policy":
        s["old"] = (s["nll"] + r.normal(T, std=0.15)).clamp_(min=0)
    s["nll_ref"] = (s["nll"] + r.normal(T, std=0.3)).clamp_(min=0) if s["ref"] else None


def prepare(case, seed):
    r, s = _Rng(seed), dict(case)
    op, T = case["op"], case["T"]
    if op == "distill":
        C, V, K, bf = case["C"], case["V"], case["K"], torch.bfloat16
        s["h"], s["W"] = r.normal(T, C, dtype=bf), r.normal(V, C, std=0.02, dtype=bf)
        s["ids"] = r.top_ids(T, K, V)
        s["z"] = r.normal(T, K, std=2.0, mean=12.0, dtype=torch.float32 if case["teacher"] == "f32" else bf)
        live = T
        if case["ragged"]:
            have = 1 + (r.uniform(T) * K).long()
            have[torch.randperm(T, generator=r.g, device="cuda")[: T // 8]] = 0
            s["ids"][torch.arange(K, device="cuda") >= have[:, None]] = -1
            live = T - T // 8
        s["scale"], s["tau"] = 1.0, 2.0
        s["loss"], s["lse"], s["logp"] = _out(T), _out(T), _out(T, K)
        if case["dir"] == "train":
            s["dloss"] = torch.full((T,), s["tau"] ** 2 / live, device="cuda")
            s["dh"], s["dW"] = _out(T, C, dtype=bf), _out(V, C, dtype=bf)
        return s
    S = case["S"] if op == "policy" else 2 * case["P"]
    _answers(s, r, T, S)
    if op == "policy":
        s["adv"] = r.normal(T if case["token_adv"] else S)
        s["loss"], s["stats"] = _out(S), _out(S, 3)
        n = S if case["mean"] else T
    else:
        s["beta"] = 2.0 if case["mean"] else 0.1
        s["loss"], s["reward"] = _out(case["P"]), _out(case["P"], 2)
        n = case["P"]
    s["dloss"] = torch.full((S if op == "policy" else n,), 1.0 / n, device="cuda") if case["grad"] else None
    s["dnll"] = _out(T) if case["grad"] else None
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------
_contexts = {}


def _context(C):
    """The library's context, which a program makes once for its model."""
    from paper_2601_05732_b200.binding import MhcLite
    if C not in _contexts:
        _contexts[C] = MhcLite(4, C, torch.cuda.current_device())
    return _contexts[C]


def _run_own(s):
    op = s["op"]
    if op == "distill":
        c = _context(s["C"])
        c.linear_distill_fwd(s["h"], s["W"], s["ids"], s["z"], s["scale"], s["tau"], s["loss"], s["lse"], s["logp"])
        got = {"loss": s["loss"], "lse": s["lse"], "logp": s["logp"]}
        if s["dir"] == "train":
            c.linear_distill_bwd(s["h"], s["W"], s["ids"], s["z"], s["scale"], s["tau"], s["lse"], s["logp"], s["dloss"], s["dh"], s["dW"])
            got.update(dh=s["dh"], dW=s["dW"])
        return got
    c = _context(1024)
    if op == "policy":
        c.policy_loss(s["nll"], s["old"], s["nll_ref"], s["target"], s["starts"], s["adv"], s["token_adv"], _EPS_LOW, _EPS_HIGH, _KL, s["mean"],
                      s["loss"], s["stats"], s["dloss"], s["dnll"])
        got = {"loss": s["loss"], "stats": s["stats"]}
    else:
        c.preference_loss(s["nll"], s["nll_ref"], s["target"], s["starts"], s["beta"], s["margin"], s["smooth"], s["mean"],
                          s["loss"], s["reward"], s["dloss"], s["dnll"])
        got = {"loss": s["loss"], "reward": s["reward"]}
    if s["grad"]:
        got["dnll"] = s["dnll"]
    return got


def _plain_distill(s):
    f32, bf = torch.float32, torch.bfloat16
    h, W = s["h"].to(f32), s["W"].to(f32)
    there = s["ids"] >= 0
    live = there.any(1)
    at = s["ids"].clamp(min=0)
    x = (h @ W.T) * (s["scale"] / s["tau"])
    top = x.amax(1, keepdim=True)
    log_sum = torch.log(torch.exp(x - top).sum(1, keepdim=True))
    z = torch.where(there, s["z"].to(f32) / s["tau"], -torch.inf)
    z = z - torch.where(live[:, None], z.amax(1, keepdim=True), 0.0)
    total = torch.exp(z).sum(1, keepdim=True)
    p = torch.where(there, torch.exp(z) / total, 0.0)
    logp = torch.where(there, (x.gather(1, at) - top) - log_sum, 0.0)
    got = {"loss": torch.where(there, p * (z - torch.log(total) - logp), 0.0).sum(1), "lse": (top + log_sum)[:, 0] * live, "logp": logp}
    if s["dir"] == "train":
        G = torch.exp(x - (top + log_sum))
        G.scatter_add_(1, at, -p)
        G *= (s["dloss"] * live * (s["scale"] / s["tau"]))[:, None]
        got["dh"], got["dW"] = (G @ W).to(bf), (G.T @ h).to(bf)
    return got


def _sequence_of(s, S):
    """Each token's sequence, and whether it counts: it has a target and belongs to a sequence."""
    at = torch.arange(s["T"], device="cuda")
    seq = torch.searchsorted(s["starts"], at, right=True) - 1
    counts = (s["target"] >= 0) & (seq >= 0) & (seq < S)
    return seq.clamp(0, S - 1), counts


def _sum_by(values, seq, S):
    return torch.zeros(S, dtype=torch.float64, device="cuda").index_add_(0, seq, values.double())


def _plain_policy(s):
    S, f32 = s["S"], torch.float32
    seq, counts = _sequence_of(s, S)
    A = s["adv"] if s["token_adv"] else s["adv"][seq]
    x = s["old"].double() - s["nll"].double()           # in 64 bits: which side of the border a ratio is on
    over, under = x > math.log1p(_EPS_HIGH), x < math.log1p(-_EPS_LOW)
    cut = (over & (A > 0)) | (under & (A < 0))
    r = torch.exp(x.to(f32))
    held = torch.where(over, 1 + _EPS_HIGH, torch.where(under, 1 - _EPS_LOW, r))
    each = -A * torch.where(cut, held, r)
    if s["ref"]:
        d = s["nll"].double() - s["nll_ref"].double()
        kl = (torch.expm1(d) - d).to(f32)
        each = each + _KL * kl
    else:
        kl = torch.zeros_like(each)
    n = _sum_by(counts, seq, S)
    per = torch.where(n > 0, 1 / n.clamp(min=1), 0.0) if s["mean"] else torch.ones_like(n)
    total, clipped, kls = (_sum_by(torch.where(counts, v, 0.0), seq, S) for v in (each, cut.to(f32), kl))
    got = {"loss": (total * per).to(f32), "stats": torch.stack((n, clipped, kls * per), 1).to(f32)}
    if s["grad"]:
        g = torch.where(cut, 0.0, A * r)
        if s["ref"]:
            g = g + _KL * torch.expm1(d).to(f32)
        got["dnll"] = torch.where(counts, g * (s["dloss"] * per).to(f32)[seq], 0.0)
    return got


def _plain_pair(s):
    S, f32 = 2 * s["P"], torch.float32
    seq, counts = _sequence_of(s, S)
    ratio = -s["nll"].double() if s["nll_ref"] is None else s["nll_ref"].double() - s["nll"].double()
    R = _sum_by(torch.where(counts, ratio, 0.0), seq, S)
    per = torch.ones_like(R)
    if s["mean"]:
        n = _sum_by(counts, seq, S)
        per = torch.where(n > 0, 1 / n.clamp(min=1), 0.0)
    reward = (s["beta"] * R * per).view(-1, 2)
    x, e = reward[:, 0] - reward[:, 1] - s["margin"], s["smooth"]
    soft = torch.clamp(-x, min=0) + torch.log1p(torch.exp(-x.abs()))          # -log sigmoid(x)
    got = {"loss": (soft + e * x).to(f32), "reward": reward.to(f32)}
    if s["grad"]:
        dx = s["dloss"].double() * (e - 1 / (1 + torch.exp(x)))
        each = (-s["beta"] * torch.stack((dx, -dx), 1).reshape(-1) * per).to(f32)
        got["dnll"] = torch.where(counts, each[seq], 0.0)
    return got


def run(state):
    if own:
        return _run_own(state)
    return {"distill": _plain_distill, "policy": _plain_policy, "pair": _plain_pair}[state["op"]](state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    op, T = case["op"], case["T"]
    if op == "distill":
        C, V, K = case["C"], case["V"], case["K"]
        live = T - (T // 8 if case["ragged"] else 0)
        fwd = 2 * (live + V) * C + T * K * (8 + (4 if case["teacher"] == "f32" else 2)) + 8 * T + 4 * T * K
        if case["dir"] == "fwd":
            return {"bytes": fwd, "flops": 2 * live * V * C}
        return {"bytes": fwd + 2 * (live + V) * C + 4 * T, "flops": 6 * live * V * C}
    if op == "policy":
        S = case["S"]
        per_token = 8 + 4 + 4 + (4 if case["ref"] else 0) + (4 if case["token_adv"] else 0) + (4 if case["grad"] else 0)
        return {"bytes": T * per_token + S * (8 + 16 + (0 if case["token_adv"] else 4) + (4 if case["grad"] else 0)), "flops": 20 * T}
    P = case["P"]
    per_token = 8 + 4 + (4 if case["ref"] else 0) + (4 if case["grad"] else 0)
    return {"bytes": T * per_token + P * (16 + 12 + (4 if case["grad"] else 0)), "flops": 4 * T}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------
def _exact_distill(s):
    f64, T, K, V, C = torch.float64, s["T"], s["K"], s["V"], s["C"]
    W, train = s["W"].to(f64), s["dir"] == "train"
    zeros = lambda *n: torch.zeros(*n, dtype=f64, device="cuda")
    got = {"loss": zeros(T), "lse": zeros(T), "logp": zeros(T, K)}
    if train:
        got["dh"], got["dW"] = zeros(T, C), zeros(V, C)
    for rows in torch.split(torch.nonzero((s["ids"] >= 0).any(1))[:, 0], 4096):
        ids, h = s["ids"][rows], s["h"][rows].to(f64)
        x = torch.einsum("tc,vc->tv", h, W) * s["scale"] / s["tau"]
        log_q = torch.log_softmax(x, 1)
        there = ids >= 0
        log_p = torch.log_softmax((s["z"][rows].to(f64) / s["tau"]).masked_fill(~there, -math.inf), 1)
        p = torch.exp(log_p)
        at = torch.gather(log_q, 1, ids * there)
        got["lse"][rows] = torch.logsumexp(x, 1)
        got["logp"][rows] = at * there
        got["loss"][rows] = torch.nansum(p * (log_p - at), 1)            # an absent entry is 0 x -inf
        if train:
            wanted = torch.zeros_like(x).scatter_add_(1, ids * there, p)
            G = (torch.exp(log_q) - wanted) * (s["dloss"][rows].to(f64) * s["scale"] / s["tau"])[:, None]
            got["dh"][rows] = torch.einsum("tv,vc->tc", G, W)
            got["dW"] += torch.einsum("tv,tc->vc", G, h)
    return got


def _exact_sums(values, starts):
    """Sums between successive starts."""
    run = torch.cat((torch.zeros(1, dtype=torch.float64, device="cuda"), values.cumsum(0)))
    return run[starts[1:]] - run[starts[:-1]]


def _exact_policy(s):
    f64, S, starts = torch.float64, s["S"], s["starts"]
    used = int(starts[-1])
    length = starts[1:] - starts[:-1]
    spread = lambda v: torch.repeat_interleave(v, length, output_size=used)
    live = (s["target"][:used] >= 0).to(f64)
    nll, old = s["nll"][:used].to(f64).requires_grad_(s["grad"]), s["old"][:used].to(f64)
    A = s["adv"][:used].to(f64) if s["token_adv"] else spread(s["adv"].to(f64))
    ratio = torch.exp(old - nll)
    free, held = -A * ratio, -A * torch.clamp(ratio, 1 - _EPS_LOW, 1 + _EPS_HIGH)
    loss = torch.where(held > free, held, free)                           # alike inside the borders: the free one's slope
    kl = torch.zeros_like(nll)
    if s["ref"]:
        gap = nll - s["nll_ref"][:used].to(f64)
        kl = torch.special.expm1(gap) - gap
    n = _exact_sums(live, starts)
    share = 1 / torch.clamp(n, min=1) if s["mean"] else torch.ones_like(n)
    weight = spread(share) * live
    each = (loss + _KL * kl) * weight
    got = {"loss": _exact_sums(each.detach(), starts),
           "stats": torch.stack((n, _exact_sums((held > free).to(f64) * live, starts), _exact_sums((kl * weight).detach(), starts)), 1)}
    if s["grad"]:
        (each * spread(s["dloss"].to(f64))).sum().backward()
        got["dnll"] = torch.nn.functional.pad(nll.grad, (0, s["T"] - used))
    return got


def _exact_pair(s):
    f64, starts = torch.float64, s["starts"]
    used = int(starts[-1])
    length = starts[1:] - starts[:-1]
    live = (s["target"][:used] >= 0).to(f64)
    ratio = (-s["nll"][:used].to(f64) + (s["nll_ref"][:used].to(f64) if s["ref"] else 0.0)) * live
    share = torch.ones(2 * s["P"], dtype=f64, device="cuda")
    if s["mean"]:
        share = 1 / torch.clamp(_exact_sums(live, starts), min=1)
    R = (_exact_sums(ratio, starts) * share).requires_grad_(s["grad"])
    won, lost = s["beta"] * R[0::2], s["beta"] * R[1::2]
    x = won - lost - s["margin"]
    loss = -(1 - s["smooth"]) * torch.nn.functional.logsigmoid(x) - s["smooth"] * torch.nn.functional.logsigmoid(-x)
    got = {"loss": loss.detach(), "reward": torch.stack((won, lost), 1).detach()}
    if s["grad"]:
        (loss * s["dloss"].to(f64)).sum().backward()
        each = torch.repeat_interleave(-R.grad * share, length, output_size=used) * live
        got["dnll"] = torch.nn.functional.pad(each, (0, s["T"] - used))
    return got


def exact(case, seed):
    return {"distill": _exact_distill, "policy": _exact_policy, "pair": _exact_pair}[case["op"]](prepare(case, seed))
