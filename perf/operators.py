"""What is timed of the operators around a stack of mixing layers: the lookup that fills the residual streams, the norms,
gate, scale and dropout that enclose a sublayer, dropout on its own, and the loss at the end of the stack.

Each pass runs either the plain form (elementary torch operations, 32 bits, rounded once at the end) or, with ``own`` set,
the calls that a program makes of the library.  Activations are bf16 and parameters fp32, as everywhere in the library; the
table of the lookup is fp32 or bf16, the weights of the loss are bf16.
"""
import math

import numpy as np
import torch

own = False

_EPS = 1e-6
_M32 = 0xFFFFFFFF


# ---- the cases ------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one decoded token enters the stack: latency
        {"name": "embed_one", "op": "embed", "dir": "fwd", "T": 1, "n": 4, "C": 2048, "V": 50257, "table": "bf16"},
        # a training batch enters the stack, master weights in fp32
        {"name": "embed_batch", "op": "embed", "dir": "fwd", "T": 16384, "n": 4, "C": 2048, "V": 32000, "table": "f32"},
        # its gradient with an odd number of tokens, three streams, a large table of which few rows are met
        {"name": "embed_grad_odd", "op": "embed", "dir": "bwd", "T": 5003, "n": 3, "C": 1536, "V": 50257, "table": "f32"},
        # the gradient of a large batch: tokens as unevenly spread as in text
        {"name": "embed_grad_large", "op": "embed", "dir": "bwd", "T": 65536, "n": 4, "C": 1024, "V": 100000, "table": "f32"},
        # the two norms around the sublayer of one decoded token
        {"name": "block_one", "op": "block", "dir": "fwd", "T": 1, "C": 4096, "gate": True, "p": 0.0},
        # a ragged batch, no gate, with dropout, forward and backward
        {"name": "block_odd", "op": "block", "dir": "train", "T": 4099, "C": 1536, "gate": False, "p": 0.1},
        # a training batch with the gate and dropout, forward and backward
        {"name": "block_batch", "op": "block", "dir": "train", "T": 16384, "C": 2048, "gate": True, "p": 0.1},
        # dropout of a small activation with an odd number of elements
        {"name": "dropout_small", "op": "dropout", "count": 100003, "p": 0.2},
        # dropout of a large batch's activations
        {"name": "dropout_large", "op": "dropout", "count": 65536 * 2048, "p": 0.1},
        # the log probability of one token: one pass over the weights
        {"name": "loss_one", "op": "loss", "dir": "fwd", "T": 1, "C": 2048, "V": 50257, "ignored": False},
        # loss and gradients of a ragged batch, an eighth of it without a target
        {"name": "loss_odd", "op": "loss", "dir": "train", "T": 2047, "C": 1024, "V": 32001, "ignored": True},
        # loss and gradients of a training batch
        {"name": "loss_batch", "op": "loss", "dir": "train", "T": 16384, "C": 2048, "V": 50257, "ignored": False},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["embed", "block", "dropout", "loss"])
    C = 8 * _log(rng, 8, 512)
    if op == "embed":
        n, way = rng.randint(2, 5), rng.choice(["fwd", "bwd"])
        V = min(_log(rng, 1000, 131072), 100000 * 1024 // C)
        T = min(_log(rng, 1, 131072), 65536 * 4 * 1024 // (n * C))
        return {"op": op, "dir": way, "T": T, "n": n, "C": C, "V": V, "table": rng.choice(["f32", "bf16"])}
    if op == "block":
        T = min(_log(rng, 1, 65536), 16384 * 2048 // C)
        return {"op": op, "dir": rng.choice(["fwd", "train"]), "T": T, "C": C, "gate": rng.random() < 0.6, "p": rng.choice([0.0, 0.05, 0.1, 0.5])}
    if op == "dropout":
        return {"op": op, "count": _log(rng, 1, 65536 * 2048), "p": rng.choice([0.05, 0.1, 0.2, 0.5, 0.9])}
    V = _log(rng, 1000, 131072)
    T = min(_log(rng, 1, 16384), max(1, 16384 * 2048 * 50257 // (C * V)))
    return {"op": op, "dir": rng.choice(["fwd", "train"]), "T": T, "C": C, "V": V, "ignored": rng.random() < 0.5}


# ---- inputs ---------------------------------------------------------------------------------------------------------
class _Rng:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(self, *shape, std=1.0, mean=0.0, dtype=torch.bfloat16):
        return (torch.randn(*shape, generator=self.g, device="cuda") * std + mean).to(dtype)

    def tokens(self, T, V):
        """Ids as unevenly spread as those of text: the density falls with 1 / (id + 1)."""
        u = torch.rand(T, generator=self.g, device="cuda", dtype=torch.float64)
        return (torch.exp(u * math.log(V + 1)).long() - 1).clamp_(0, V - 1)

    def key(self):
        """(seed, offset) of the dropout generator, as the program keeps it on the device."""
        return torch.randint(0, 1 << 62, (2,), generator=self.g, device="cuda", dtype=torch.int64)


def _out(*shape, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=dtype, device="cuda")


def prepare(case, seed):
    r, s, f32 = _Rng(seed), dict(case), torch.float32
    op, T, C, V = case["op"], case.get("T"), case.get("C"), case.get("V")
    if op == "embed":
        n = case["n"]
        s["ids"], s["scale"] = r.tokens(T, V), math.sqrt(C)
        if case["dir"] == "fwd":
            s["E"] = r.normal(V, C, std=0.02, dtype=f32 if case["table"] == "f32" else torch.bfloat16)
            s["x0"] = _out(T, n, C)
        else:
            s["g"], s["dE"] = r.normal(T, n, C, std=1e-2), _out(V, C, dtype=f32)
    elif op == "block":
        s["u"], s["o"] = r.normal(T, C), r.normal(T, C, std=3.0)
        s["w_in"], s["w_out"] = r.normal(C, std=0.2, mean=1.0, dtype=f32), r.normal(C, std=0.2, mean=1.0, dtype=f32)
        s["scale"] = torch.full((1,), 0.4, device="cuda")
        s["a"] = r.normal(T, C, std=1.5) if case["gate"] else None
        s["rng"] = r.key() if case["p"] > 0 else None
        s["v"], s["y"], s["r_in"], s["r_out"] = _out(T, C), _out(T, C), _out(T, dtype=f32), _out(T, dtype=f32)
        if case["dir"] == "train":
            s["dv"] = r.normal(T, C, std=1e-2)
            # a gradient that leans on the block's output, as one does while training lowers or raises the scale
            s["dy"] = (r.normal(T, C, std=1e-2, dtype=f32) + 3e-3 * s["o"].float()).to(torch.bfloat16)
            s["du"], s["d_o"], s["da"] = _out(T, C), _out(T, C), _out(T, C) if case["gate"] else None
            s["dw_in"], s["dw_out"], s["dscale"] = _out(C, dtype=f32), _out(C, dtype=f32), _out(1, dtype=f32)
    elif op == "dropout":
        s["x"], s["rng"], s["y"] = r.normal(case["count"]), r.key(), _out(case["count"])
    else:
        s["h"], s["W"] = r.normal(T, C), r.normal(V, C, std=0.02)
        s["target"] = r.tokens(T, V)
        if case["ignored"]:
            s["target"][torch.randperm(T, generator=r.g, device="cuda")[: T // 8]] = -100
        s["loss"], s["lse"] = _out(T, dtype=f32), _out(T, dtype=f32)
        if case["dir"] == "train":
            s["dloss"] = torch.full((T,), 1.0 / (T - (T // 8 if case["ignored"] else 0)), device="cuda")
            s["dh"], s["dW"] = _out(T, C), _out(V, C)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------
_contexts = {}


def _context(n, C):
    """The library's context, which a program makes once for its model."""
    from paper_2601_05732_b200.binding import MhcLite
    if (n, C) not in _contexts:
        _contexts[n, C] = MhcLite(n, C, torch.cuda.current_device())
    return _contexts[n, C]


def _run_own(s):
    op = s["op"]
    if op == "embed":
        c = _context(s["n"], s["C"])
        if s["dir"] == "fwd":
            c.embed_fwd(s["ids"], s["E"], s["scale"], s["x0"])
            return {"x0": s["x0"]}
        c.embed_bwd(s["ids"], s["g"], s["scale"], s["dE"])
        return {"dE": s["dE"]}
    if op == "block":
        c = _context(4, s["C"])
        c.block_in_fwd(s["u"], s["w_in"], _EPS, s["v"], s["r_in"])
        c.block_out_fwd(s["o"], s["a"], s["w_out"], s["scale"], _EPS, s["p"], s["rng"], s["y"], s["r_out"])
        got = {"v": s["v"], "y": s["y"]}
        if s["dir"] == "train":
            c.block_out_bwd(s["o"], s["a"], s["w_out"], s["scale"], s["r_out"], s["p"], s["rng"], s["dy"], s["d_o"], s["da"], s["dw_out"], s["dscale"])
            c.block_in_bwd(s["u"], s["w_in"], s["r_in"], s["dv"], s["du"], s["dw_in"])
            got.update(d_o=s["d_o"], dw_out=s["dw_out"], dscale=s["dscale"], du=s["du"], dw_in=s["dw_in"])
            if s["a"] is not None:
                got["da"] = s["da"]
        return got
    if op == "dropout":
        _context(4, 1024).dropout(s["x"], s["p"], s["rng"], s["y"])
        return {"y": s["y"]}
    c = _context(4, s["C"])
    c.linear_ce_fwd(s["h"], s["W"], s["target"], 1.0, s["loss"], s["lse"])
    got = {"loss": s["loss"], "lse": s["lse"]}
    if s["dir"] == "train":
        c.linear_ce_bwd(s["h"], s["W"], s["target"], 1.0, s["lse"], s["dloss"], s["dh"], s["dW"])
        got.update(dh=s["dh"], dW=s["dW"])
    return got


def _threshold(p):
    return int(math.floor(p * 65536.0 + 0.5))


def _philox(groups, rng):
    """Philox4x32-10 (Salmon et al. 2011) of the counters (group, offset) under the key `seed`: four words a group."""
    c0, c1 = groups & _M32, groups >> 32
    c2, c3 = (rng[1] & _M32).expand_as(groups), ((rng[1] >> 32) & _M32).expand_as(groups)
    k0, k1 = rng[0] & _M32, (rng[0] >> 32) & _M32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57           # the 64-bit products, wrapped
        c0, c1, c2, c3 = ((b >> 32) & _M32) ^ c1 ^ k0, b & _M32, ((a >> 32) & _M32) ^ c3 ^ k1, a & _M32
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    return torch.stack((c0, c1, c2, c3), -1)


def _keep(count, p, rng):
    """Which of `count` elements stay: element i takes 16 bits of the word (i % 8) / 2 of group i / 8, the low half first."""
    words = _philox(torch.arange((count + 7) // 8, device="cuda"), rng)
    halves = torch.stack((words & 0xFFFF, words >> 16), -1).reshape(-1)
    return halves[:count] >= _threshold(p)


def _dropped(x, p, rng):
    """x / (1 - p) where the element stays, 0 where not; p counts as rounded to 1 / 65536."""
    if p == 0:
        return x
    keep = _keep(x.numel(), p, rng).view_as(x)
    return torch.where(keep, x * (65536.0 / (65536 - _threshold(p))), torch.zeros((), device="cuda"))


def _run_plain(s):
    op, f32, bf = s["op"], torch.float32, torch.bfloat16
    if op == "embed":
        if s["dir"] == "fwd":
            x = s["E"][s["ids"]].to(f32) * s["scale"]
            return {"x0": x.to(bf)[:, None, :].expand(-1, s["n"], -1).contiguous()}
        rows = s["g"].to(f32).sum(1) * s["scale"]
        return {"dE": torch.zeros(s["V"], s["C"], device="cuda").index_add_(0, s["ids"], rows)}
    if op == "block":
        u, o, w_in, w_out = s["u"].to(f32), s["o"].to(f32), s["w_in"], s["w_out"]
        r_in = torch.rsqrt((u * u).mean(1, keepdim=True) + _EPS)
        r_out = torch.rsqrt((o * o).mean(1, keepdim=True) + _EPS)
        uh, oh = u * r_in, o * r_out
        sig = 1.0 if s["a"] is None else 1 / (1 + torch.exp(-s["a"].to(f32)))
        z = oh * w_out * sig
        d = _dropped(z, s["p"], s["rng"])
        got = {"v": (uh * w_in).to(bf), "y": (s["scale"] * d).to(bf)}
        if s["dir"] == "train":
            dy, dv = s["dy"].to(f32), s["dv"].to(f32)
            dz = _dropped(dy, s["p"], s["rng"]) * s["scale"]
            e, i = dz * sig * w_out, dv * w_in
            got["dscale"] = (dy.double() * d).sum().reshape(1).to(f32)
            got["dw_out"], got["dw_in"] = (dz * sig * oh).sum(0), (dv * uh).sum(0)
            got["d_o"] = (r_out * (e - oh * (e * oh).mean(1, keepdim=True))).to(bf)
            got["du"] = (r_in * (i - uh * (i * uh).mean(1, keepdim=True))).to(bf)
            if s["a"] is not None:
                got["da"] = (dz * oh * w_out * sig * (1 - sig)).to(bf)
        return got
    if op == "dropout":
        return {"y": _dropped(s["x"].to(f32), s["p"], s["rng"]).to(bf)}
    h, W, valid = s["h"].to(f32), s["W"].to(f32), s["target"] >= 0
    rows, at = torch.arange(s["T"], device="cuda"), s["target"].clamp(min=0)
    logits = h @ W.T
    top = logits.amax(1, keepdim=True)
    lse = top[:, 0] + torch.log(torch.exp(logits - top).sum(1))
    got = {"loss": (lse - logits[rows, at]) * valid, "lse": lse * valid}
    if s["dir"] == "train":
        G = torch.exp(logits - lse[:, None])
        G[rows, at] -= 1
        G *= (s["dloss"] * valid)[:, None]
        got["dh"], got["dW"] = (G @ W).to(bf), (G.T @ h).to(bf)
    return got


def run(state):
    if own:
        return _run_own(state)
    return _run_plain(state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def _rows_met(T, V):
    """Rows of the table that T tokens meet, on average."""
    p = np.diff(np.log(np.arange(1, V + 2, dtype=np.float64))) / math.log(V + 1)
    return float(-np.expm1(T * np.log1p(-np.minimum(p, 1 - 1e-12))).sum())


def work(case):
    op, T, C, V = case["op"], case.get("T"), case.get("C"), case.get("V")
    if op == "embed":
        n = case["n"]
        if case["dir"] == "fwd":
            return {"bytes": 8 * T + _rows_met(T, V) * C * (4 if case["table"] == "f32" else 2) + 2 * T * n * C, "flops": T * C}
        return {"bytes": 8 * T + 2 * T * n * C + 4 * V * C, "flops": T * n * C}
    if op == "block":
        gate = 1 if case["gate"] else 0
        fwd = 2 * T * C * (4 + gate) + 8 * C + 8 * T
        if case["dir"] == "fwd":
            return {"bytes": fwd, "flops": 10 * T * C}
        # the gradients read u, dv, o, dy and the gate again: the sublayer runs in between
        return {"bytes": fwd + 2 * T * C * (6 + 2 * gate) + 16 * C + 8 * T, "flops": 34 * T * C}
    if op == "dropout":
        return {"bytes": 4 * case["count"], "flops": case["count"]}
    live = T - (T // 8 if case["ignored"] else 0)
    if case["dir"] == "fwd":
        return {"bytes": 2 * (live + V) * C + 16 * T, "flops": 2 * live * V * C}
    return {"bytes": 4 * (live + V) * C + 20 * T, "flops": 6 * live * V * C}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------
def _mul_hi_lo(a, m):
    """High and low words of the product of 32-bit a and m, by 16-bit halves."""
    al, ah, ml, mh = a % 65536, a // 65536, m % 65536, m // 65536
    low, mid = al * ml, ah * ml
    mid2 = al * mh + low // 65536 + mid % 65536
    return ah * mh + mid // 65536 + mid2 // 65536, (mid2 % 65536) * 65536 + low % 65536


def _exact_keep(count, p, rng):
    seed, offset = (int(v) for v in rng.tolist())
    group = torch.arange(-(-count // 8), device="cuda")
    key = [seed % 2**32, seed // 2**32]
    ctr = [group % 2**32, group // 2**32, torch.full_like(group, offset % 2**32), torch.full_like(group, offset // 2**32)]
    for k in range(10):
        h0, l0 = _mul_hi_lo(ctr[0], 0xD2511F53)
        h1, l1 = _mul_hi_lo(ctr[2], 0xCD9E8D57)
        ka, kb = (key[0] + k * 0x9E3779B9) % 2**32, (key[1] + k * 0xBB67AE85) % 2**32
        ctr = [h1 ^ ctr[1] ^ ka, l1, h0 ^ ctr[3] ^ kb, l0]
    keep = torch.empty(group.numel(), 8, dtype=torch.bool, device="cuda")
    for e in range(8):
        keep[:, e] = (ctr[e // 2] // 65536 ** (e % 2)) % 65536 >= _threshold(p)
    return keep.reshape(-1)[:count]


def exact(case, seed):
    s = prepare(case, seed)
    f64, op = torch.float64, case["op"]
    if op == "embed":
        if case["dir"] == "fwd":
            return {"x0": torch.stack([s["E"].to(f64)[s["ids"]] * s["scale"]] * s["n"], 1)}
        total = torch.zeros(s["V"], s["C"], dtype=f64, device="cuda")
        for j in range(s["n"]):
            total.index_add_(0, s["ids"], s["g"][:, j].to(f64), alpha=s["scale"])
        return {"dE": total}
    if op == "block":
        names = ["u", "o", "w_in", "w_out", "scale"] + (["a"] if case["gate"] else [])
        x = {k: s[k].to(f64).requires_grad_(case["dir"] == "train") for k in names}
        v = x["u"] / torch.sqrt(x["u"].pow(2).mean(-1, keepdim=True) + _EPS) * x["w_in"]
        z = x["o"] / torch.sqrt(x["o"].pow(2).mean(-1, keepdim=True) + _EPS) * x["w_out"]
        if case["gate"]:
            z = z * torch.sigmoid(x["a"])
        if case["p"] > 0:
            z = z * _exact_keep(z.numel(), case["p"], s["rng"]).view_as(z) / (1 - _threshold(case["p"]) / 65536)
        y = x["scale"] * z
        got = {"v": v.detach(), "y": y.detach()}
        if case["dir"] == "train":
            torch.autograd.backward([v, y], [s["dv"].to(f64), s["dy"].to(f64)])
            got.update(d_o=x["o"].grad, dw_out=x["w_out"].grad, dscale=x["scale"].grad, du=x["u"].grad, dw_in=x["w_in"].grad)
            if case["gate"]:
                got["da"] = x["a"].grad
        return got
    if op == "dropout":
        keep = _exact_keep(case["count"], case["p"], s["rng"])
        return {"y": s["x"].to(f64) * keep / (1 - _threshold(case["p"]) / 65536)}
    T, V, C = case["T"], case["V"], case["C"]
    W = s["W"].to(f64)
    got = {"loss": torch.zeros(T, dtype=f64, device="cuda"), "lse": torch.zeros(T, dtype=f64, device="cuda")}
    train = case["dir"] == "train"
    if train:
        got["dh"], got["dW"] = torch.zeros(T, C, dtype=f64, device="cuda"), torch.zeros(V, C, dtype=f64, device="cuda")
    live = torch.nonzero(s["target"] >= 0)[:, 0]
    for rows in torch.split(live, 4096):
        h, t = s["h"][rows].to(f64), s["target"][rows]
        z = torch.einsum("tc,vc->tv", h, W)
        got["lse"][rows] = torch.logsumexp(z, 1)
        got["loss"][rows] = -torch.log_softmax(z, 1).gather(1, t[:, None])[:, 0]
        if train:
            G = (torch.softmax(z, 1) - torch.zeros_like(z).scatter_(1, t[:, None], 1.0)) * s["dloss"][rows, None].to(f64)
            got["dh"][rows] = torch.einsum("tv,vc->tc", G, W)
            got["dW"] += torch.einsum("tv,tc->vc", G, h)
    return got
