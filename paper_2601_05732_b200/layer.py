"""Device buffers of one Hyper-Connections layer and the call sequences around the caller's sublayer.

Plumbing only: tensors are allocated with PyTorch and handed to the C ABI through
:class:`~paper_2601_05732_b200.binding.MhcLite`; every step of the path runs in the
library's kernels.

Forward (paper Eq. (1), (4), (5)):   pre  -> [sublayer f: the caller's] -> post
Backward:                            post_bwd -> [f's backward]        -> tail

A model (``model_fwd`` / ``model_bwd``) is a stack with its two ends, token lookup and loss, and with the norms, gate,
scale and dropout around each sublayer (``block_sublayer``); what lies between the norms stays the caller's.
"""
from __future__ import annotations

import numpy as np
import torch

from .binding import MhcLite


def to_device_bf16(bits: np.ndarray, device) -> torch.Tensor:
    """uint16 bf16 bit patterns -> bf16 tensor on the device (no value conversion)."""
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).to(device).view(torch.bfloat16)


def bf16_to_host_f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().float().cpu().numpy().astype(np.float64)


class LayerParams:
    def __init__(self, W, b, alpha, gain, device):
        f = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(device)
        self.W, self.b, self.alpha, self.gain = f(W), f(b), f(alpha), f(gain)


class LayerBuffers:
    """Outputs and saved tensors of one layer for T tokens (kind 'lite' or 'sk')."""

    def __init__(self, ctx: MhcLite, T: int, kind: str = "lite"):
        n, C, dev = ctx.n, ctx.C, f"cuda:{ctx.device}"
        self.kind = kind
        N = ctx.n_cols(0 if kind == "lite" else 1)
        f32 = lambda *s: torch.empty(*s, dtype=torch.float32, device=dev)
        bf = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=dev)
        self.H_res, self.H_pre, self.H_post = f32(T, n, n), f32(T, n), f32(T, n)
        self.a_saved = f32(T, ctx.nfact) if kind == "lite" else None
        self.p_saved, self.rstd = f32(T, N), f32(T)
        self.u, self.x_next = bf(T, C), bf(T, n, C)
        self.dy, self.dx = bf(T, C), bf(T, n, C)
        self.dH_res, self.dH_post, self.dH_pre = f32(T, n, n), f32(T, n), f32(T, n)
        self.dW, self.db, self.dalpha, self.dgain = f32(n * C, N), f32(N), f32(4)[:3], f32(n * C)
        ctx.ensure_workspace(T, 0 if kind == "lite" else 1)


def pre_fwd(ctx: MhcLite, P: LayerParams, B: LayerBuffers, x, eps=1e-6, fused=True, iters=20, u_rstd=None, eps_u=1e-6):
    """Mappings + stream pre-mix: everything before the sublayer. Result: B.u (and the coefficients).  With u_rstd
    (fp32 [T], fused lite path only) the call also leaves the RMSNorm row statistic of the stored u there."""
    if u_rstd is not None:
        if B.kind != "lite" or not fused:
            raise ValueError("u_rstd is produced by the fused mHC-lite call only")
        ctx.pre_fwd_fused_ustat(x, P.W, P.b, P.alpha, P.gain, eps, B.H_res, B.H_pre, B.H_post, B.a_saved, B.p_saved,
                                B.rstd, B.u, u_rstd, eps_u)
        return
    if B.kind == "sk" and fused:
        ctx.sk20_pre_fwd_fused(x, P.W, P.b, P.alpha, P.gain, eps, iters, B.H_res, B.H_pre, B.H_post, B.p_saved, B.rstd,
                               B.u)
    elif B.kind == "sk":
        ctx.sk20_coeffs_fwd(x, P.W, P.b, P.alpha, P.gain, eps, iters, B.H_res, B.H_pre, B.H_post, B.p_saved, B.rstd)
        ctx.premix_fwd(x, B.H_pre, B.u)
    elif fused:
        ctx.pre_fwd_fused(x, P.W, P.b, P.alpha, P.gain, eps, B.H_res, B.H_pre, B.H_post, B.a_saved, B.p_saved,
                          B.rstd, B.u)
    else:
        ctx.coeffs_fwd(x, P.W, P.b, P.alpha, P.gain, eps, B.H_res, B.H_pre, B.H_post, B.a_saved, B.p_saved, B.rstd)
        ctx.premix_fwd(x, B.H_pre, B.u)


def post_fwd(ctx: MhcLite, B: LayerBuffers, x, y):
    """Residual mixing + merge of the sublayer output: B.x_next."""
    ctx.postres_fwd(x, y, B.H_res, B.H_post, B.x_next)


def post_bwd(ctx: MhcLite, B: LayerBuffers, x, y, g, fused=True):
    """Backward of the merge: B.dy, B.dH_res, B.dH_post (and, unfused, the H_res^T g part of B.dx)."""
    skip_dx = fused                                # the fused tail recomputes H_res^T g from g
    ctx.postres_bwd(x, y, B.H_res, B.H_post, g, B.dy, B.dH_res, B.dH_post, None if skip_dx else B.dx, False)


def tail_bwd(ctx: MhcLite, P: LayerParams, B: LayerBuffers, x, g, du, eps=1e-6, fused=True, iters=20,
             accumulate_params=False):
    """Everything after the sublayer's backward: B.dx and the parameter gradients."""
    if B.kind == "sk" and fused:
        ctx.sk20_tail_bwd_fused(x, P.W, P.b, P.alpha, P.gain, eps, iters, B.p_saved, B.rstd, B.H_res, B.H_pre, B.H_post,
                                g, du, B.dH_res, B.dH_post, B.dx, B.dW, B.db, B.dalpha, B.dgain, accumulate_params)
    elif B.kind == "sk":
        ctx.premix_bwd(x, B.H_pre, du, B.dH_pre, B.dx, True)
        ctx.sk20_coeffs_bwd(x, P.W, P.b, P.alpha, P.gain, eps, iters, B.p_saved, B.rstd, B.H_pre, B.H_post,
                            B.dH_res, B.dH_pre, B.dH_post, B.dx, True, B.dW, B.db, B.dalpha, B.dgain,
                            accumulate_params)
    elif fused:
        ctx.tail_bwd_fused(x, P.W, P.alpha, P.gain, eps, B.a_saved, B.p_saved, B.rstd, B.H_res, B.H_pre, B.H_post,
                           g, du, B.dH_res, B.dH_post, B.dx, B.dW, B.db, B.dalpha, B.dgain, accumulate_params)
    else:
        ctx.premix_bwd(x, B.H_pre, du, B.dH_pre, B.dx, True)
        ctx.coeffs_bwd(x, P.W, P.alpha, P.gain, eps, B.a_saved, B.p_saved, B.rstd, B.H_pre, B.H_post,
                       B.dH_res, B.dH_pre, B.dH_post, B.dx, True, B.dW, B.db, B.dalpha, B.dgain, accumulate_params)


def stack_fwd(ctx: MhcLite, Ps, Bs, x0, sublayer, eps=1e-6, fuse_layers=True):
    """Forward through len(Ps) layers (the paper's models are 6, 12 or 24 of them back to back): layer l reads the
    x_next of layer l - 1.  `sublayer(l, u)` is the caller's f and returns y [T,C] bf16.  Each layer's input, y
    and outputs stay in its LayerBuffers for the backward.  With fuse_layers the merge of layer l also produces the
    projection of layer l + 1 (mhclite_postres_fwd_next_proj / mhclite_pre_fwd_resume), so x_{l+1} is read once less.
    The sublayer must not call workspace-using entry points of `ctx` in between.  Returns the last layer's x_next."""
    x = x0
    resumed = False
    for l, (P, B) in enumerate(zip(Ps, Bs)):
        B.x_in = x
        if resumed:       # this layer's projection came out of the merge kernel of the layer before
            ctx.pre_fwd_resume(x, P.b, P.alpha, eps, B.H_res, B.H_pre, B.H_post, B.a_saved, B.p_saved, B.rstd, B.u)
        else:
            pre_fwd(ctx, P, B, x, eps, True)
        B.y = sublayer(l, B.u)
        resumed = fuse_layers and l + 1 < len(Ps) and B.kind == "lite"
        if resumed:
            ctx.postres_fwd_next_proj(x, B.y, B.H_res, B.H_post, B.x_next, Ps[l + 1].W, Ps[l + 1].gain)
        else:
            post_fwd(ctx, B, x, B.y)
        x = B.x_next
    return x


def stack_bwd(ctx: MhcLite, Ps, Bs, g_top, sublayer_bwd, eps=1e-6):
    """Backward through the stack: `sublayer_bwd(l, u, dy)` is the caller's backward of f and returns du [T,C] bf16.
    Returns dL/dx_0; each layer's parameter gradients are in its LayerBuffers."""
    g = g_top
    for l in reversed(range(len(Ps))):
        P, B = Ps[l], Bs[l]
        B.g_in = g
        post_bwd(ctx, B, B.x_in, B.y, g, True)
        B.du = sublayer_bwd(l, B.u, B.dy)
        tail_bwd(ctx, P, B, B.x_in, g, B.du, eps, True)
        g = B.dx
    return g


class BlockParams:
    """What encloses one sublayer: norm weights w_in, w_out [C] and the residual scale [1], fp32; p_drop of its output."""

    def __init__(self, w_in, w_out, scale, device, p_drop=0.0):
        f = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(device)
        self.w_in, self.w_out, self.scale, self.p_drop = f(w_in), f(w_out), f(np.reshape(scale, (1,))), float(p_drop)


class BlockBuffers:
    """Outputs, saved tensors and gradients of one sublayer's enclosure for T tokens."""

    def __init__(self, ctx: MhcLite, T: int, gated: bool):
        C, dev = ctx.C, f"cuda:{ctx.device}"
        f32 = lambda *s: torch.empty(*s, dtype=torch.float32, device=dev)
        bf = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=dev)
        self.v, self.y, self.r_in, self.r_out = bf(T, C), bf(T, C), f32(T), f32(T)
        self.du, self.d_o, self.dgate = bf(T, C), bf(T, C), bf(T, C) if gated else None
        self.dw_in, self.dw_out, self.dscale = f32(C), f32(C), f32(1)
        self.o = self.gate = None              # what the caller's inner function returned


def block_sublayer(ctx: MhcLite, Ks, KBs, inner, rng=None, eps=1e-6):
    """The `sublayer` of stack_fwd: norm, the caller's `inner(l, v)` -> (o, gate or None), then norm, gate, dropout and
    residual scale.  rng: int64 [layers, 2] on the device, (seed, offset) of each layer's dropout; the caller gives a layer
    an offset of its own and moves the offsets on from step to step."""
    def f(l, u):
        K, B = Ks[l], KBs[l]
        ctx.block_in_fwd(u, K.w_in, eps, B.v, B.r_in)
        B.o, B.gate = inner(l, B.v)
        ctx.block_out_fwd(B.o, B.gate, K.w_out, K.scale, eps, K.p_drop, None if rng is None else rng[l], B.y, B.r_out)
        return B.y
    return f


def block_sublayer_bwd(ctx: MhcLite, Ks, KBs, inner_bwd, rng=None, accumulate_params=False):
    """The `sublayer_bwd` of stack_bwd; `inner_bwd(l, v, d_o, dgate)` is the caller's backward of `inner` and returns dv.
    rng holds what it held in the forward."""
    def f(l, u, dy):
        K, B = Ks[l], KBs[l]
        ctx.block_out_bwd(B.o, B.gate, K.w_out, K.scale, B.r_out, K.p_drop, None if rng is None else rng[l], dy, B.d_o, B.dgate,
                          B.dw_out, B.dscale, accumulate_params)
        dv = inner_bwd(l, B.v, B.d_o, B.dgate)
        ctx.block_in_bwd(u, K.w_in, B.r_in, dv, B.du, B.dw_in, accumulate_params)
        return B.du
    return f


class ModelEnds:
    """The two ends of a model for T tokens: the table E [V,C] (fp32 or bf16) with its scale, the last norm w [C], the
    head W [V,C] bf16, and their buffers.  The last hidden row of a token is the mean over its streams."""

    def __init__(self, ctx: MhcLite, T: int, E: torch.Tensor, embed_scale: float, w: torch.Tensor, W: torch.Tensor,
                 logit_scale: float = 1.0):
        n, C, dev = ctx.n, ctx.C, f"cuda:{ctx.device}"
        f32 = lambda *s: torch.empty(*s, dtype=torch.float32, device=dev)
        bf = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=dev)
        self.E, self.embed_scale, self.w, self.W, self.logit_scale = E, float(embed_scale), w, W, float(logit_scale)
        self.x0, self.top, self.h = bf(T, n, C), bf(T, C), bf(T, C)
        self.mix, self.r = torch.full((T, n), 1.0 / n, device=dev), f32(T)
        self.loss, self.lse = f32(T), f32(T)
        self.dh, self.dtop, self.dx, self.dmix = bf(T, C), bf(T, C), bf(T, n, C), f32(T, n)
        self.dE, self.dw, self.dW = f32(*E.shape), f32(C), bf(*W.shape)


class Teacher:
    """A teacher's top entries of each token: ids [T,K] int64 (negative: absent), logits [T,K] fp32 or bf16, the temperature
    of both distributions, and the student's log probabilities at the entries, which the forward leaves."""

    def __init__(self, ids: torch.Tensor, logits: torch.Tensor, temperature: float = 1.0):
        self.ids, self.logits, self.temperature = ids, logits, float(temperature)
        self.logp = torch.empty(ids.shape, dtype=torch.float32, device=ids.device)


class Answers:
    """S sequences (with `pairs`: S / 2 pairs of a chosen and a rejected one) over the T tokens of a step: where they begin
    (starts [S+1] int64), their losses and what goes with them, and the gradient that model_bwd takes as dloss."""

    def __init__(self, starts: torch.Tensor, T: int, pairs: bool = False):
        f32 = lambda *s: torch.empty(*s, dtype=torch.float32, device=starts.device)
        S = starts.numel() - 1
        self.starts, self.pairs, self.dnll = starts, pairs, f32(T)
        self.loss = f32(S // 2 if pairs else S)
        self.reward, self.stats = (f32(S // 2, 2), None) if pairs else (None, f32(S, 3))


def policy_loss(ctx: MhcLite, A: Answers, nll, nll_old, nll_ref, target, adv, dloss, token_adv=False, clip_low=0.2, clip_high=0.2,
                kl_weight=0.0, mean=True):
    """Clipped policy loss of each sequence from the token losses of model_fwd (nll), of the policy that sampled them
    (nll_old) and of the reference (nll_ref, None: no KL term).  Leaves A.loss, A.stats and, with dloss [S], A.dnll."""
    ctx.policy_loss(nll, nll_old, nll_ref, target, A.starts, adv, token_adv, clip_low, clip_high, kl_weight, mean, A.loss, A.stats,
                    dloss, None if dloss is None else A.dnll)
    return A.loss


def preference_loss(ctx: MhcLite, A: Answers, nll, nll_ref, target, dloss, beta=0.1, margin=0.0, smoothing=0.0, mean=False):
    """Preference loss of each pair from the token losses of model_fwd (nll) and of the reference (nll_ref, or None).  Leaves
    A.loss, A.reward and, with dloss [S / 2], A.dnll."""
    ctx.preference_loss(nll, nll_ref, target, A.starts, beta, margin, smoothing, mean, A.loss, A.reward, dloss,
                        None if dloss is None else A.dnll)
    return A.loss


def model_fwd(ctx: MhcLite, M: ModelEnds, Ps, Bs, ids, target, sublayer, eps=1e-6, fuse_layers=True, teacher: Teacher | None = None):
    """Token ids [T] to the loss of each token [T] (0 where target is negative): lookup into the streams, the stack, the
    mean of the streams, the last norm, cross entropy; with a teacher the divergence from its entries instead (target is not
    used).  Everything the backward needs stays in M, Bs, the teacher and the sublayer's buffers."""
    ctx.embed_fwd(ids, M.E, M.embed_scale, M.x0)
    M.x_top = stack_fwd(ctx, Ps, Bs, M.x0, sublayer, eps, fuse_layers)
    ctx.premix_fwd(M.x_top, M.mix, M.top)
    ctx.block_in_fwd(M.top, M.w, eps, M.h, M.r)
    if teacher is None:
        ctx.linear_ce_fwd(M.h, M.W, target, M.logit_scale, M.loss, M.lse)
    else:
        ctx.linear_distill_fwd(M.h, M.W, teacher.ids, teacher.logits, M.logit_scale, teacher.temperature, M.loss, M.lse, teacher.logp)
    return M.loss


def model_bwd(ctx: MhcLite, M: ModelEnds, Ps, Bs, ids, target, dloss, sublayer_bwd, eps=1e-6, accumulate_params=False,
              teacher: Teacher | None = None):
    """Backward of model_fwd from dloss [T] fp32 (of a loss of sequences: Answers.dnll): M.dW, M.dw, M.dE, and the layers'
    gradients in Bs.  accumulate_params concerns the fp32 gradients M.dw and M.dE; M.dW is overwritten, and the layers'
    gradients are as stack_bwd leaves them."""
    if teacher is None:
        ctx.linear_ce_bwd(M.h, M.W, target, M.logit_scale, M.lse, dloss, M.dh, M.dW)
    else:
        ctx.linear_distill_bwd(M.h, M.W, teacher.ids, teacher.logits, M.logit_scale, teacher.temperature, M.lse, teacher.logp, dloss,
                               M.dh, M.dW)
    ctx.block_in_bwd(M.top, M.w, M.r, M.dh, M.dtop, M.dw, accumulate_params)
    ctx.premix_bwd(M.x_top, M.mix, M.dtop, M.dmix, M.dx, False)
    g0 = stack_bwd(ctx, Ps, Bs, M.dx, sublayer_bwd, eps)
    ctx.embed_bwd(ids, g0, M.embed_scale, M.dE, accumulate_params)
    return M.dE
