"""The gated pair of FCs, the head's log probabilities and the clipping of gradients in 64 bits, written from their definitions
(include/canvas_gated.h, canvas_head.h, canvas_clip.h): what the tests compare the kernels with, and how far these may be off.

Bounds are worst cases, element by element.  u = 2^-24 is half a step of fp32, `half` half a step of the plan's type (bf16 2^-8, fp32 2^-24).  A
sum of n products in fp32 is off by at most n u times the sum of their magnitudes (first order in u), in any order; fp32 plans add 6 n products of
pieces, leave out 3 of 9 below 2^-24 of a product each, 2^-22 in all, and cut a value into pieces exactly.
"""
import math

import torch

U = 2.0 ** -24


def half_of(f32):
    return U if f32 else 2.0 ** -8


def sum_bound(n, f32):
    """Of a sum of n products, relative to the sum of their magnitudes."""
    return (6 * n + 8) * U if f32 else (n + 2) * U


def act(kind, g):
    """(act, act') of one kind: 0 sigmoid, 1 silu, 2 gelu."""
    if kind == 2:
        cdf = 0.5 * torch.special.erfc(-g / math.sqrt(2))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(g)
    return (s, s * torch.sigmoid(-g)) if kind == 0 else (g * s, s * (1 + g * torch.sigmoid(-g)))


def gated(kind, x, wg, wu, dy=None, f32=True):
    """(values, bounds) by name."""
    half, n = half_of(f32), x.shape[1]
    g, u = x @ wg.T, x @ wu.T
    eg, eu = (sum_bound(n, f32) * (x.abs() @ w.T.abs()) for w in (wg, wu))
    a, da = act(kind, g)
    # |act'| <= 1.13 and |act''| <= 0.8 for all three; the kernel's own act and slope are good to 16 u of their largest terms
    ea = 1.13 * eg + 16 * U * a.abs() + 16 * U * (1 + g.abs()) * torch.exp(-g.abs())
    ed = 0.8 * eg + 16 * U * (1 + da.abs())
    val = {"y": a * u}
    bound = {"y": ea * (u.abs() + eu) + a.abs() * eu + 2 * half * (a * u).abs()}
    if dy is not None:
        du, dg = dy * a, dy * u * da
        rounded = half if not f32 else 4 * U
        if not f32:      # what is kept of g and u has 20 bits: half a step is 2^-12 of the value
            eg, eu = eg + 2.0 ** -12 * (g.abs() + eg), eu + 2.0 ** -12 * (u.abs() + eu)
            ea = 1.13 * eg + 16 * U * a.abs() + 16 * U * (1 + g.abs()) * torch.exp(-g.abs())
            ed = 0.8 * eg + 16 * U * (1 + da.abs())
        edu = dy.abs() * ea + rounded * du.abs()
        edg = dy.abs() * (ed * (u.abs() + eu) + da.abs() * eu) + rounded * dg.abs()
        f, t = wg.shape[0], x.shape[0]
        val["dx"] = dg @ wg + du @ wu
        bound["dx"] = (edg @ wg.abs() + edu @ wu.abs()) + sum_bound(2 * f, f32) * (dg.abs() @ wg.abs() + du.abs() @ wu.abs()) + 2 * half * val["dx"].abs()
        for name, d, e in (("dw_gate", dg, edg), ("dw_up", du, edu)):
            val[name] = d.T @ x
            bound[name] = e.T @ x.abs() + sum_bound(t, f32) * (d.T.abs() @ x.abs()) + 2 * half * val[name].abs()
    return val, bound


def head(x, w, tokens, it=1.0, mask=None, dlogprob=None, dentropy=None, f32=True, grads=True):
    """(values, bounds) by name; rows and classes whatever they hold.  mask: truth values [classes] or None."""
    half, n = half_of(f32), x.shape[1]
    t, v = x.shape[0], w.shape[0]
    keep = torch.ones(v, dtype=torch.bool, device=x.device) if mask is None else mask.bool()
    wk = torch.where(keep[:, None], w, torch.zeros_like(w))
    logits = x @ wk.T
    z = torch.where(keep[None], logits * it, torch.full_like(logits, -math.inf))
    ez = it * sum_bound(n, f32) * (x.abs() @ wk.T.abs())
    worst = torch.where(keep[None], ez, torch.zeros_like(ez)).amax(1)          # of a logit of the row
    known = (tokens >= 0) & (tokens < v)
    at = torch.where(known, tokens, torch.zeros_like(tokens))
    empty = (z == -math.inf).all(1)
    most = torch.where(empty, torch.zeros_like(worst), z.amax(1))
    d = z - most[:, None]
    lse = torch.log(torch.exp(d).sum(1))
    logp = torch.where(torch.isinf(d), d, d - lse[:, None])
    p = torch.where(empty[:, None], torch.zeros_like(z), torch.exp(logp))
    plogp = torch.where(p > 0, p * logp, torch.zeros_like(p))
    entropy = torch.where(empty, torch.zeros_like(worst), -plogp.sum(1))
    chosen = logp.gather(1, at[:, None])[:, 0]
    chosen = torch.where(empty, torch.full_like(chosen, -math.inf), chosen)
    val = {"logprob": torch.where(known, chosen, torch.zeros_like(chosen)), "entropy": entropy}
    # exponentials of differences x: their arguments are rounded a few times, (|x| + 2) 4 u; sums over v classes grow pairwise in tiles: 64 + log v terms
    far = 4 * U * (torch.where(torch.isinf(chosen), torch.zeros_like(chosen), chosen).abs() + 2 + 3 * math.log(v + 1)) + (64 + v / 64 / 16 + 20) * U
    bound = {"logprob": 2 * worst + far, "entropy": (2 * worst + (64 + v / 64 / 16 + 20) * U + 8 * U * (1 + math.log(v + 1))) * (2 + math.log(v + 1))}
    if grads:
        g = torch.where(known, dlogprob, torch.zeros_like(worst))[:, None] * it if dlogprob is not None else torch.zeros_like(z[:, :1])
        h = dentropy[:, None] * it if dentropy is not None else torch.zeros_like(z[:, :1])
        dz = -g * p - h * (plogp + p * entropy[:, None])
        if dlogprob is not None:
            dz = dz.scatter_add(1, at[:, None], g)
        live = keep[None] & ~empty[:, None] & ((g != 0) | (h != 0))
        dz = torch.where(live, dz, torch.zeros_like(dz))
        size = torch.where(torch.isinf(logp), torch.zeros_like(logp), logp.abs())
        off = (2 * worst + (64 + v / 64 / 16 + 20) * U)[:, None] + 4 * U * (size + 2 + 3 * math.log(v + 1))
        edz = p * ((g.abs() + h.abs() * (size + entropy[:, None] + 1)) * off + h.abs() * (off + bound["entropy"][:, None])) + (half if not f32 else 4 * U) * dz.abs()
        # exponentials below 2^-126 are zero in fp32, and so is what is left of products with numbers that small
        edz = edz + 2.0 ** -125 * (1 + g.abs() + h.abs() * (size + entropy[:, None] + 1))
        if dlogprob is not None:
            edz = edz.scatter_add(1, at[:, None], 4 * U * g.abs())
        edz = torch.where(live, edz, torch.zeros_like(edz))
        xl = torch.where(live.any(1)[:, None], x, torch.zeros_like(x))
        val["dx"], val["dweight"] = dz @ wk, dz.T @ xl
        bound["dx"] = edz @ wk.abs() + sum_bound(v, f32) * (dz.abs() @ wk.abs()) + 2 * half * val["dx"].abs()
        bound["dweight"] = edz.T @ xl.abs() + sum_bound(t, f32) * (dz.T.abs() @ xl.abs()) + 2 * half * val["dweight"].abs()
    return val, bound


def clip(grads, most):
    """norm, scale and the scaled tensors, in 64 bits."""
    norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    scale = 1.0 if norm == 0 or most == math.inf else min(1.0, most / norm)
    return norm, scale, [g.double() * scale for g in grads]
