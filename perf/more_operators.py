"""Measured cases of the operators that end a network of micro-DAG blocks and its training step:

  gated     a gated pair of FCs: act(x Wg^T) * (x Wu^T), and the gradients of x and of both weights
  head      log probabilities of given tokens with the entropy, from features and the head's weight without keeping the logits,
            and the gradients of both
  clip      the norm over all gradients of a network, and the gradients scaled down to a largest norm

`run` makes one pass: the calls of the package where `own` is true, and the same in elementary torch operations in 32 bits
where it is not.  mode "train" is forward and backward, "infer" the forward pass of an inference plan.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

# The largest listed case of each operator: a drawn one stays below.
MOST_FLOPS = {"gated": 12.0 * 4096 * 2048 * 8192, "head": 6.0 * 4096 * 1024 * 32768}
MOST_LOGITS = 4096 * 32768
MOST_ELEMENTS = 1 << 28


def listed():
    return [
        # Training on 64 pooled images of 64 channels: the smallest products, where launches count.
        {"name": "gated_images", "op": "gated", "mode": "train", "dtype": "f32", "rows": 64, "features": 64, "width": 256, "act": "gelu"},
        # Serving: the next token of four sequences; both weights are read for four rows.
        {"name": "gated_decode", "op": "gated", "mode": "infer", "dtype": "bf16", "rows": 4, "features": 2048, "width": 8192, "act": "silu"},
        # Training on tokens: the largest products.
        {"name": "gated_tokens", "op": "gated", "mode": "train", "dtype": "bf16", "rows": 4096, "features": 2048, "width": 8192, "act": "silu"},
        # Training in fp32 on ragged sizes: no tile divides them.
        {"name": "gated_ragged", "op": "gated", "mode": "train", "dtype": "f32", "rows": 1500, "features": 1000, "width": 2731, "act": "sigmoid"},
        # Training a classifier: 256 pooled images of 512 features, 1000 classes, fp32.
        {"name": "head_classes", "op": "head", "mode": "train", "dtype": "f32", "rows": 256, "features": 512, "classes": 1000, "masked": False, "entropy": False},
        # Serving: four sequences scored over a large vocabulary with classes that are not allowed; the weight is read for four rows.
        {"name": "head_decode", "op": "head", "mode": "infer", "dtype": "bf16", "rows": 4, "features": 2048, "classes": 131072, "masked": True, "entropy": True},
        # Training on tokens with an entropy term: the largest products.
        {"name": "head_tokens", "op": "head", "mode": "train", "dtype": "bf16", "rows": 4096, "features": 1024, "classes": 32768, "masked": False, "entropy": True},
        # Scoring a prompt: an odd vocabulary.
        {"name": "head_prompt", "op": "head", "mode": "infer", "dtype": "bf16", "rows": 1500, "features": 1000, "classes": 50021, "masked": False, "entropy": True},
        # The gradients of a network of two blocks of 64 channels: a dozen small tensors, where launches count.
        {"name": "clip_blocks", "op": "clip", "tensors": 12, "elements": 60000, "dtypes": "f32", "out": "f32", "sizes": 1, "clipped": True},
        # The weights of a residual network in both types, odd sizes among them; an update takes the clipped ones in fp32.
        {"name": "clip_mixed", "op": "clip", "tensors": 55, "elements": 25500000, "dtypes": "mixed", "out": "f32", "sizes": 2, "clipped": True},
        # A large model's gradients in bf16: more than any cache holds.
        {"name": "clip_large", "op": "clip", "tensors": 24, "elements": 1 << 28, "dtypes": "bf16", "out": "bf16", "sizes": 3, "clipped": True},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["gated", "head", "clip"])
    if op == "clip":
        elements = _log_int(rng, 1000, MOST_ELEMENTS)
        return {"op": "clip", "tensors": _log_int(rng, 1, 60), "elements": elements, "dtypes": rng.choice(["f32", "bf16", "mixed"]),
                "out": "f32" if elements > MOST_ELEMENTS // 2 else rng.choice(["f32", "bf16", "same"]), "sizes": rng.randrange(1 << 20), "clipped": rng.random() < 0.75}
    mode, dtype = rng.choice(["train", "infer"]), rng.choice(["bf16", "bf16", "f32"])
    while True:
        rows = rng.choice([rng.randint(1, 32), _log_int(rng, 32, 8192), _log_int(rng, 32, 8192)])
        features = rng.choice([_log_int(rng, 16, 4096), 8 * _log_int(rng, 2, 512)])
        if op == "gated":
            width = rng.choice([_log_int(rng, 16, 16384), 8 * _log_int(rng, 2, 2048)])
            if (12.0 if mode == "train" else 4.0) * rows * features * width <= MOST_FLOPS["gated"]:
                return {"op": "gated", "mode": mode, "dtype": dtype, "rows": rows, "features": features, "width": width, "act": rng.choice(["silu", "gelu", "sigmoid"])}
        else:
            classes = _log_int(rng, 100, 200000)
            if (6.0 if mode == "train" else 2.0) * rows * features * classes <= MOST_FLOPS["head"] and rows * classes <= MOST_LOGITS:
                return {"op": "head", "mode": mode, "dtype": dtype, "rows": rows, "features": features, "classes": classes,
                        "masked": rng.random() < 0.4, "entropy": rng.random() < 0.6}


def _sizes(case):
    """How many elements each tensor of a clip case has, and its type: spread over three orders of magnitude, `elements` in all."""
    r = random.Random(case["sizes"])
    shares = [math.exp(r.uniform(0, 6.9)) for _ in range(case["tensors"])]
    counts = [max(1, int(case["elements"] * s / sum(shares))) for s in shares]
    return [(n, r.choice(["f32", "bf16"]) if case["dtypes"] == "mixed" else case["dtypes"]) for n in counts]


def _out_type(case, dtype):
    return dtype if case["out"] == "same" else case["out"]


def work(case):
    if case["op"] == "clip":
        e = {"f32": 4, "bf16": 2}
        sizes = _sizes(case)
        return {"bytes": float(sum(n * (e[t] + e[_out_type(case, t)]) for n, t in sizes)), "flops": 3.0 * sum(n for n, _ in sizes)}
    e = 2 if case["dtype"] == "bf16" else 4
    t, c, train = case["rows"], case["features"], case["mode"] == "train"
    if case["op"] == "gated":
        f = case["width"]
        moved = t * c + 2 * f * c + t * f
        return {"bytes": float(e * (moved * 2 if train else moved)), "flops": (12.0 if train else 4.0) * t * c * f}
    v = case["classes"]
    moved = t * c + v * c
    return {"bytes": float(e * (moved * 2 if train else moved) + 24 * t + (v if case["masked"] else 0)), "flops": (6.0 if train else 2.0) * t * c * v}


# ---------------------------------------------------------------- inputs

def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype)

    if case["op"] == "clip":
        # every tensor has a size of gradient of its own
        grads = [normal(n, std=1e-3 * (1 + i % 7), dtype=DTYPES[t]) for i, (n, t) in enumerate(_sizes(case))]
        expected = 1e-3 * math.sqrt(sum(n * (1 + i % 7) ** 2 for i, (n, _) in enumerate(_sizes(case))))
        return {"grads": grads, "max_norm": expected * (0.3 if case["clipped"] else 3.0)}
    dt, t, c = DTYPES[case["dtype"]], case["rows"], case["features"]
    x = normal(t, c, dtype=dt)
    if case["op"] == "gated":
        f = case["width"]
        s = {"x": x, "w_gate": normal(f, c, std=1.5 / math.sqrt(c), dtype=dt), "w_up": normal(f, c, std=1 / math.sqrt(c), dtype=dt)}
        if case["mode"] == "train":
            s["dy"] = normal(t, f, dtype=dt)
        return s
    v = case["classes"]
    w = normal(v, c, std=2.5 / math.sqrt(c), dtype=dt)
    s = {"x": x, "weight": w, "mask": None, "inv_temperature": 1.0 if case["mode"] == "train" else 1.25}
    logits = torch.matmul(x.float(), w.float().t())
    if case["masked"]:
        mask = torch.rand(v, generator=g, device="cuda") < 0.9
        mask[: min(v, 16)] = True
        s["mask"] = mask.to(torch.uint8)
        logits = torch.where(mask, logits, torch.full((), -math.inf, device="cuda"))
    # a model gives most of its tokens a high probability; some positions of a padded batch have no target
    tokens = torch.randint(0, v, (t,), generator=g, device="cuda")
    tokens = torch.where(torch.rand(t, generator=g, device="cuda") < 0.6, logits.max(1).indices, tokens)
    if s["mask"] is not None:
        tokens = torch.where(s["mask"][tokens] != 0, tokens, torch.zeros_like(tokens))
    if t >= 16:
        tokens = torch.where(torch.rand(t, generator=g, device="cuda") < 0.05, torch.full_like(tokens, -1), tokens)
    s["tokens"] = tokens
    if case["mode"] == "train":
        s |= {"dlogprob": normal(t, std=0.3, mean=-1.0) / t, "dentropy": normal(t, std=0.05) / t if case["entropy"] else None}
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=dict(case))
    if own:
        from paper_2304_07741_amd import binding as B
        from paper_2304_07741_amd import harness

        flags = B.CANVAS_OPT_INFERENCE if case.get("mode") == "infer" else 0
        if case["op"] == "gated":
            act = {"silu": B.CANVAS_GATED_SILU, "gelu": B.CANVAS_GATED_GELU, "sigmoid": B.CANVAS_GATED_SIGMOID}[case["act"]]
            s["runner"] = harness.GatedRunner(case["rows"], case["features"], case["width"], case["dtype"], act, flags=flags)
        elif case["op"] == "head":
            s["runner"] = harness.HeadRunner(case["rows"], case["features"], case["classes"], case["dtype"], flags=flags)
        else:
            sizes = _sizes(case)
            s["runner"] = harness.ClipRunner([(n,) for n, _ in sizes], [t for _, t in sizes], [_out_type(case, t) for _, t in sizes])
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    op = s["case"]["op"]
    if own:
        return {"gated": _own_gated, "head": _own_head, "clip": _own_clip}[op](s)
    return {"gated": _plain_gated, "head": _plain_head, "clip": _plain_clip}[op](s)


def _own_gated(s):
    r = s["runner"]
    out = dict(r.forward(s["x"], s["w_gate"], s["w_up"]))
    if "dy" in s:
        out |= r.backward(s["x"], s["w_gate"], s["w_up"], s["dy"])
    return out


def _own_head(s):
    r = s["runner"]
    how = {"mask": s["mask"], "inv_temperature": s["inv_temperature"]}
    out = dict(r.forward(s["x"], s["weight"], s["tokens"], **how))
    if "dlogprob" in s:
        out |= r.backward(s["x"], s["weight"], s["tokens"], s["dlogprob"], s["dentropy"], **how)
    return out


def _own_clip(s):
    return s["runner"].step(s["grads"], s["max_norm"])


def _sigmoid(v):
    return 1 / (1 + torch.exp(-v))


def _plain_gated(s):
    act, dt = s["case"]["act"], s["x"].dtype
    x, wg, wu = s["x"].float(), s["w_gate"].float(), s["w_up"].float()
    g, u = torch.matmul(x, wg.t()), torch.matmul(x, wu.t())
    if act == "gelu":
        cdf = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        a, da = g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    else:
        sig = _sigmoid(g)
        a, da = (sig, sig * (1 - sig)) if act == "sigmoid" else (g * sig, sig * (1 + g * (1 - sig)))
    out = {"y": (a * u).to(dt)}
    if "dy" in s:
        dy = s["dy"].float()
        du, dg = dy * a, dy * u * da
        out["dx"] = (torch.matmul(dg, wg) + torch.matmul(du, wu)).to(dt)
        out["dw_gate"], out["dw_up"] = torch.matmul(dg.t(), x).to(dt), torch.matmul(du.t(), x).to(dt)
    return out


def _plain_head(s):
    it, dt, v = s["inv_temperature"], s["x"].dtype, s["weight"].shape[0]
    x, w = s["x"].float(), s["weight"].float()
    z = torch.matmul(x, w.t()) * it
    if s["mask"] is not None:
        z = torch.where(s["mask"] != 0, z, torch.full((), -math.inf, device=z.device))
    known = (s["tokens"] >= 0) & (s["tokens"] < v)
    at = torch.where(known, s["tokens"], torch.zeros_like(s["tokens"]))[:, None]
    d = z - z.amax(1, keepdim=True)
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    logp = d - torch.log(total)
    p = e / total
    plogp = torch.where(p > 0, p * logp, torch.zeros((), device=p.device))
    entropy = -plogp.sum(1)
    zero = torch.zeros((), device=p.device)
    out = {"logprob": torch.where(known, logp.gather(1, at)[:, 0], zero), "entropy": entropy}
    if "dlogprob" in s:
        g = torch.where(known, s["dlogprob"], zero)[:, None]
        dz = -g * p
        if s["dentropy"] is not None:
            dz = dz - s["dentropy"][:, None] * (plogp + p * entropy[:, None])
        dz = dz.scatter_add(1, at, g) * it
        out["dx"], out["dweight"] = torch.matmul(dz, w).to(dt), torch.matmul(dz.t(), x).to(dt)
    return out


def _plain_clip(s):
    case = s["case"]
    norm = torch.sqrt(torch.stack([g.float().square().sum() for g in s["grads"]]).sum())
    scale = torch.clamp(s["max_norm"] / norm, max=1.0)
    types = {torch.float32: "f32", torch.bfloat16: "bf16"}
    return {"norm": norm, "scale": scale, "grads": [(g.float() * scale).to(DTYPES[_out_type(case, types[g.dtype])]) for g in s["grads"]]}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "clip":
        total = 0.0
        for g in s["grads"]:
            total = total + torch.linalg.vector_norm(g.double()) ** 2
        norm = total ** 0.5
        scale = torch.minimum(s["max_norm"] / norm, torch.ones_like(norm))
        return {"norm": norm, "scale": scale, "grads": [g.double() * scale for g in s["grads"]]}
    s = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in s.items()}
    return _exact_gated(case, s) if case["op"] == "gated" else _exact_head(case, s)


def _exact_gated(case, s):
    x, wg, wu = s["x"], s["w_gate"], s["w_up"]
    g, u = x @ wg.T, x @ wu.T
    if case["act"] == "sigmoid":
        a = torch.sigmoid(g)
        slope = a - a ** 2
    elif case["act"] == "silu":
        h = torch.tanh(g / 2)
        a = g * (1 + h) / 2
        slope = (1 + h) / 2 + g * (1 - h ** 2) / 4
    else:
        cdf = torch.special.ndtr(g)
        a = g * cdf
        slope = cdf + g * torch.exp(-g ** 2 / 2) / math.sqrt(2 * math.pi)
    out = {"y": a * u}
    if case["mode"] == "train":
        both = torch.cat([s["dy"] * u * slope, s["dy"] * a], 1)
        out["dx"] = both @ torch.cat([wg, wu], 0)
        dw = both.T @ x
        out["dw_gate"], out["dw_up"] = dw[: case["width"]], dw[case["width"]:]
    return out


def _exact_head(case, s):
    z = (s["x"] @ s["weight"].T) * s["inv_temperature"]
    if s["mask"] is not None:
        z = z.masked_fill(s["mask"] == 0, -math.inf)
    rows = torch.nonzero(s["tokens"] >= 0)[:, 0]
    tokens = s["tokens"][rows]
    lse = torch.logsumexp(z, 1)
    z -= lse[:, None]
    p = torch.exp(z)
    out = {"logprob": torch.zeros_like(lse), "entropy": torch.special.entr(p).sum(1)}
    out["logprob"][rows] = z[rows, tokens]
    if case["mode"] == "train":
        g = torch.zeros_like(lse)
        g[rows] = s["dlogprob"][rows]
        dz = -p * g[:, None]
        dz[rows, tokens] += g[rows]
        if s["dentropy"] is not None:
            dz += s["dentropy"][:, None] * (torch.special.entr(p) - p * out["entropy"][:, None])
        dz *= s["inv_temperature"]
        out["dx"], out["dweight"] = dz @ s["weight"], dz.T @ s["x"]
    return out
