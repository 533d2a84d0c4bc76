"""The operators around a block in 64 bits on the CPU, written from their definitions (include/canvas_norm.h,
canvas_logprob.h, canvas_ortho.h): what the tests compare the kernels with."""
import math

import torch


def act(gate, g):
    """(act, act') of one gate kind: 0 none, 1 sigmoid, 2 silu."""
    if gate == 0:
        return 1.0, 0.0
    s = torch.sigmoid(g)
    return (s, s * (1 - s)) if gate == 1 else (g * s, s * (1 + g * (1 - s)))


def norm_forward(x, z, g, w_post, scale, w_pre, gate, eps):
    """x' and u; z None: without POST, w_pre None: without PRE.  Maps are [N, C, P]."""
    col = lambda w: w[None, :, None]  # noqa: E731
    y = x
    if z is not None:
        r2 = ((z * z).mean(1, keepdim=True) + eps) ** -0.5
        y = x + col(scale) * act(gate, g)[0] * (z * r2 * col(w_post))
    u = None
    if w_pre is not None:
        u = y * ((y * y).mean(1, keepdim=True) + eps) ** -0.5 * col(w_pre)
    return y, u


def norm_backward(y, z, g, w_post, scale, w_pre, gate, eps, dy, du):
    """Gradients by name; y is x' (x without POST), dy may be None with PRE."""
    col = lambda w: w[None, :, None]  # noqa: E731
    out = {}
    D = dy if dy is not None else torch.zeros_like(y)
    if w_pre is not None:
        r1 = ((y * y).mean(1, keepdim=True) + eps) ** -0.5
        yh, dyh = y * r1, du * col(w_pre)
        D = D + r1 * (dyh - yh * (dyh * yh).mean(1, keepdim=True))
        out["dw_pre"] = (du * yh).sum((0, 2))
        out["dx"] = D
    if z is not None:
        r2 = ((z * z).mean(1, keepdim=True) + eps) ** -0.5
        zh, (a, da) = z * r2, act(gate, g)
        q = D * a * col(scale * w_post)
        out["dz"] = r2 * (q - zh * (q * zh).mean(1, keepdim=True))
        if gate:
            out["dgate"] = D * da * col(scale * w_post) * zh
        k = (D * a * zh).sum((0, 2))
        out["dw_post"], out["dscale"] = scale * k, w_post * k
    return out


def logprob_forward(logits, it, mask, tokens, top):
    """Row by row, as the header says.  mask: truth values [rows, classes] or None."""
    rows, classes = logits.shape
    out = {"logprob": [], "entropy": [], "top_logprob": [], "top_index": []}
    for r in range(rows):
        v = logits[r].clone()
        if mask is not None:
            v[~mask[r]] = -math.inf
        alive = (v != -math.inf).nonzero()[:, 0]
        t = int(tokens[r])
        if len(alive) == 0:
            out["logprob"].append(-math.inf if 0 <= t < classes else 0.0)
            out["entropy"].append(0.0)
            out["top_logprob"].append([-math.inf] * top)
            out["top_index"].append([-1] * top)
            continue
        bad = bool(torch.isnan(v).any() or (v == math.inf).any())
        finite = v[alive]
        if bad:
            lp, entropy = torch.full_like(v, math.nan), math.nan
        else:
            lp = (v - finite.max()) * it
            lp = lp - torch.log(torch.exp(lp).sum())
            p = torch.exp(lp[alive])
            entropy = float(-torch.where(p > 0, p * lp[alive], torch.zeros_like(p)).sum())
        out["logprob"].append(float(lp[t]) if 0 <= t < classes else 0.0)
        out["entropy"].append(entropy)
        order = torch.where(torch.isnan(finite), torch.full_like(finite, math.inf), finite)
        first = torch.isnan(finite).to(torch.int64)
        pick = sorted(range(len(alive)), key=lambda k: (-int(first[k]), -float(order[k]), int(alive[k])))[:top]
        out["top_logprob"].append([float(lp[alive[k]]) for k in pick] + [-math.inf] * (top - len(pick)))
        out["top_index"].append([int(alive[k]) for k in pick] + [-1] * (top - len(pick)))
    res = {k: torch.tensor(out[k], dtype=torch.float64) for k in ("logprob", "entropy", "top_logprob")}
    res["top_index"] = torch.tensor(out["top_index"], dtype=torch.int64)
    return res


def logprob_backward(logits, it, mask, tokens, dlogprob, dentropy):
    rows, classes = logits.shape
    grad = torch.zeros_like(logits)
    for r in range(rows):
        v = logits[r].clone()
        if mask is not None:
            v[~mask[r]] = -math.inf
        alive = v != -math.inf
        if not bool(alive.any()):
            continue
        t = int(tokens[r])
        given = 0 <= t < classes
        g = float(dlogprob[r]) if dlogprob is not None and given else 0.0
        h = float(dentropy[r]) if dentropy is not None else 0.0
        zs = (v - v[alive].max()) * it
        logp = zs - torch.log(torch.exp(zs[alive]).sum())
        p = torch.exp(logp)
        plogp = torch.where(p > 0, p * logp, torch.zeros_like(p))
        entropy = -plogp.sum()
        d = -g * p - h * (plogp + p * entropy)
        if given:
            d[t] += g
        if mask is not None:
            d[~mask[r]] = 0
        grad[r] = d * it
    return grad


COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def newton_schulz(v, steps):
    """Of one matrix [R, K]."""
    a, b, c = COEFFICIENTS
    x = v / (torch.sqrt((v * v).sum()) + 1e-7)
    if v.shape[0] > v.shape[1]:
        x = x.T
    for _ in range(steps):
        q = x @ x.T
        x = a * x + (b * q + c * (q @ q)) @ x
    return x.T if v.shape[0] > v.shape[1] else x


def ortho_step(grad, momentum, mu, nesterov, steps, master=None, lr=0.0, decay=0.0):
    out = {}
    v = grad
    if momentum is not None:
        out["momentum"] = mu * momentum + grad
        v = grad + mu * out["momentum"] if nesterov else out["momentum"]
    out["update"] = torch.stack([newton_schulz(m, steps) for m in v])
    if master is not None:
        out["master"] = (1 - lr * decay) * master - lr * out["update"]
    return out
