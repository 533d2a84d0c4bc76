"""Measured cases of the operators that a training step of micro-DAG blocks has around the DAGs themselves:

  norm      the norm behind a block, its gate and residual scale, and the norm in front of the next block, in one pass
  logprob   log probabilities of given tokens with the entropy and the top alternatives, and the gradient of both
  ortho     the update of an FC weight: its momentum orthogonalised by Newton-Schulz products

`run` makes one pass: the calls of the package where `own` is true, and the same in elementary torch operations in 32 bits
where it is not.  mode "train" is forward and backward, "infer" the forward pass of an inference plan.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6                                   # of the norms
NS_EPS = 1e-7                                # of the division by the Frobenius norm
NS_COEFFICIENTS = (3.4445, -4.7750, 2.0315)  # of x + x^3 + x^5 in one Newton-Schulz step
MU, LR, DECAY = 0.95, 0.02, 0.01

# The largest listed case of each operator: a drawn one stays below.
MOST_ELEMENTS = {"norm": 64 * 64 * 56 * 56, "logprob": 4096 * 32768}
MOST_FLOPS = 5 * (4.0 * 2048 * 2048 * 8192 + 2.0 * 2048 ** 3)


def listed():
    return [
        # Serving: the join between two blocks for eight single tokens.  One launch and the host's part of it.
        {"name": "norm_decode", "op": "norm", "mode": "infer", "dtype": "bf16", "N": 8, "C": 1024, "H": 1, "W": 1, "gate": "silu"},
        # Training at the stage-1 map of the default benchmark: long planes, few channels, the largest tensors.
        {"name": "norm_stage1", "op": "norm", "mode": "train", "dtype": "bf16", "N": 64, "C": 64, "H": 56, "W": 56, "gate": "sigmoid"},
        # Training at stage 4: planes of 49 pixels that no wide access divides, many channels.
        {"name": "norm_stage4", "op": "norm", "mode": "train", "dtype": "bf16", "N": 128, "C": 512, "H": 7, "W": 7, "gate": "silu"},
        # Training on rows of tokens (planes of one pixel) in fp32, without a gate.
        {"name": "norm_tokens", "op": "norm", "mode": "train", "dtype": "f32", "N": 4096, "C": 2048, "H": 1, "W": 1, "gate": "none"},
        # Serving: four sequences, a large vocabulary under a mask of allowed tokens, the 20 best alternatives of each.
        {"name": "logprob_decode", "op": "logprob", "mode": "infer", "dtype": "bf16", "rows": 4, "classes": 131072, "pad": 0, "top": 20, "masked": True},
        # Training a classifier head: 256 images, 1000 classes, fp32.
        {"name": "logprob_classes", "op": "logprob", "mode": "train", "dtype": "f32", "rows": 256, "classes": 1000, "pad": 0, "top": 0, "masked": False},
        # Training on tokens with an entropy term: the largest tensors.
        {"name": "logprob_tokens", "op": "logprob", "mode": "train", "dtype": "bf16", "rows": 4096, "classes": 32768, "pad": 0, "top": 0, "masked": False},
        # Scoring a prompt with its five best alternatives: an odd vocabulary, rows that begin at odd addresses.
        {"name": "logprob_prompt", "op": "logprob", "mode": "infer", "dtype": "bf16", "rows": 1500, "classes": 50021, "pad": 2, "top": 5, "masked": False},
        # The grouped FC behind a 3x3 window of 64 channels: eight matrices of 8 x 72, the smallest work.
        {"name": "ortho_groups", "op": "ortho", "dtype": "f32", "G": 8, "R": 8, "K": 72, "master": False},
        # A 3x3 convolution of 256 channels with fp32 master weights and bf16 weights.
        {"name": "ortho_conv", "op": "ortho", "dtype": "bf16", "G": 1, "R": 256, "K": 2304, "master": True},
        # Two matrices with more rows than columns: an FC that widens 512 channels four times.
        {"name": "ortho_tall", "op": "ortho", "dtype": "f32", "G": 2, "R": 2048, "K": 512, "master": False},
        # The largest weight: 2048 x 8192 with master weights.
        {"name": "ortho_large", "op": "ortho", "dtype": "bf16", "G": 1, "R": 2048, "K": 8192, "master": True},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "logprob", "ortho"])
    if op == "norm":
        # maps of whole networks and rows of tokens, from a single one to a training batch
        h, w = rng.choice([(1, 1), (1, 1), (7, 7), (14, 14), (28, 28), (56, 56), (_log_int(rng, 2, 64), _log_int(rng, 2, 64))])
        c = _log_int(rng, 16, 4096) if h * w < 200 else _log_int(rng, 16, 512)
        most = MOST_ELEMENTS["norm"] // (c * h * w)
        n = _log_int(rng, 1, max(1, min(8192, most)))
        return {"op": "norm", "mode": rng.choice(["train", "train", "infer"]), "dtype": rng.choice(["bf16", "bf16", "f32"]),
                "N": n, "C": c, "H": h, "W": w, "gate": rng.choice(["none", "sigmoid", "silu"])}
    if op == "logprob":
        v = _log_int(rng, 100, 200000)
        mode = rng.choice(["train", "infer"])
        most = MOST_ELEMENTS["logprob"] // v
        if mode == "infer":
            most //= 2                       # (its plain form sorts whole rows)
        return {"op": "logprob", "mode": mode, "dtype": rng.choice(["bf16", "f32"]) if v * most < 1 << 26 else "bf16",
                "rows": _log_int(rng, 1, max(1, min(8192, most))), "classes": v, "pad": rng.choice([0, 0, 1, 8, 27]),
                "top": rng.randint(1, 32) if mode == "infer" else 0, "masked": rng.random() < 0.4}
    while True:
        g = rng.choice([1, 1, 1, 2, 4, 8, 32])
        r, k = _log_int(rng, 8, 2048), _log_int(rng, 8, 8192)
        if g * _ns_flops(min(r, k), max(r, k)) <= MOST_FLOPS and g * r * k <= 2048 * 8192:
            return {"op": "ortho", "dtype": rng.choice(["bf16", "f32"]), "G": g, "R": r, "K": k, "master": rng.random() < 0.5}


def _ns_flops(m, n, steps=5):
    """What `steps` products X X^T, A A and B X need, the first two only on one side of their diagonal (both are symmetric)."""
    return steps * (m * (m + 1.0) * n + m * (m + 1.0) * m + 2.0 * m * m * n)


def work(case):
    if case["op"] == "norm":
        e = 2 if case["dtype"] == "bf16" else 4
        maps = case["N"] * case["C"] * case["H"] * case["W"]
        gate = case["gate"] != "none"
        moved = 2 + gate + 2                                 # x, z, gate -> x', u
        flops = 12.0 * maps
        if case["mode"] == "train":
            moved += 4 + gate + 2 + gate                     # x', z, gate, dx', du -> dx, dz, dgate
            flops += 30.0 * maps
        return {"bytes": float(e * maps * moved + 4 * 6 * case["C"]), "flops": flops}
    if case["op"] == "logprob":
        e = 2 if case["dtype"] == "bf16" else 4
        n = case["rows"] * case["classes"]
        train = case["mode"] == "train"
        b = n * e * (3 if train else 1) + (n * (2 if train else 1) if case["masked"] else 0) + case["rows"] * (16 + 8 * case["top"])
        return {"bytes": float(b), "flops": float(n * (12 if train else 5))}
    n = case["G"] * case["R"] * case["K"]
    e = 2 if case["dtype"] == "bf16" else 4
    b = n * (4 * 3 + e) + (n * (4 * 2 + e) if case["master"] else 0)
    return {"bytes": float(b), "flops": case["G"] * _ns_flops(min(case["R"], case["K"]), max(case["R"], case["K"]))}


# ---------------------------------------------------------------- inputs

def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype)

    dt = DTYPES[case["dtype"]]
    if case["op"] == "norm":
        shape = (case["N"], case["C"], case["H"], case["W"])
        s = {"x": normal(*shape, std=2.0, dtype=dt), "z": normal(*shape, std=0.7, mean=0.1, dtype=dt),
             "gate": normal(*shape, dtype=dt) if case["gate"] != "none" else None,
             "w_post": normal(case["C"], std=0.1, mean=1.0), "scale": normal(case["C"], std=0.05, mean=0.2),
             "w_pre": normal(case["C"], std=0.1, mean=1.0)}
        if case["mode"] == "train":
            s |= {"dx_out": normal(*shape, dtype=dt), "du": normal(*shape, dtype=dt)}
        return s
    if case["op"] == "logprob":
        t, v = case["rows"], case["classes"]
        logits = normal(t, v + case["pad"], std=2.5, dtype=dt)[:, :v]
        tokens = torch.randint(0, v, (t,), generator=g, device="cuda")
        best = logits.max(1).indices                         # a model gives most of its tokens a high probability
        tokens = torch.where(torch.rand(t, generator=g, device="cuda") < 0.6, best, tokens)
        s = {"logits": logits, "tokens": tokens, "mask": None, "inv_temperature": 1.0 if case["mode"] == "train" else 1.25}
        if case["masked"]:
            mask = torch.rand(t, v, generator=g, device="cuda") < 0.7
            mask[torch.arange(t, device="cuda"), tokens] = True
            mask[:, : min(v, 40)] = True
            s["mask"] = mask.to(torch.uint8)
        if case["mode"] == "train":
            s |= {"dlogprob": normal(t, std=0.3, mean=-1.0) / t, "dentropy": normal(t, std=0.05) / t}
        return s
    G, R, K = case["G"], case["R"], case["K"]
    rank = max(1, min(R, K) // 4)                            # gradients are sums of few strong directions and noise
    grad = torch.matmul(normal(G, R, rank) * (1.0 / (1 + torch.arange(rank, device="cuda"))), normal(G, rank, K)) + normal(G, R, K, std=0.3)
    grad *= 1e-3
    return {"grad": grad, "momentum": normal(G, R, K, std=2e-3) + 3 * grad,
            "master": normal(G, R, K, std=1.0 / math.sqrt(K)) if case["master"] else None}


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=dict(case))
    if own:
        from paper_2304_07741_amd import binding as B
        from paper_2304_07741_amd import harness

        flags = B.CANVAS_OPT_INFERENCE if case.get("mode") == "infer" else 0
        if case["op"] == "norm":
            gate = {"none": B.CANVAS_GATE_NONE, "sigmoid": B.CANVAS_GATE_SIGMOID, "silu": B.CANVAS_GATE_SILU}[case["gate"]]
            s["runner"] = harness.NormRunner((case["N"], case["C"], case["H"], case["W"]), case["dtype"],
                                             B.CANVAS_NORM_POST | B.CANVAS_NORM_PRE, gate=gate, eps=EPS, flags=flags)
        elif case["op"] == "logprob":
            s["runner"] = harness.LogprobRunner(case["rows"], case["classes"], case["dtype"], top_k=case["top"], flags=flags)
        else:
            s["runner"] = harness.OrthoRunner((case["G"], case["R"], case["K"]), case["dtype"], flags=B.CANVAS_ORTHO_NESTEROV)
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    op = s["case"]["op"]
    if own:
        return {"norm": _own_norm, "logprob": _own_logprob, "ortho": _own_ortho}[op](s)
    return {"norm": _plain_norm, "logprob": _plain_logprob, "ortho": _plain_ortho}[op](s)


def _own_norm(s):
    r = s["runner"]
    out = dict(r.forward(s["x"], s["z"], s["gate"], s["w_post"], s["scale"], s["w_pre"]))
    if "du" in s:
        out |= r.backward(out["x_out"], s["z"], s["gate"], s["w_post"], s["scale"], s["w_pre"], s["dx_out"], s["du"])
    return out


def _own_logprob(s):
    r = s["runner"]
    out = dict(r.forward(s["logits"], s["tokens"], mask=s["mask"], inv_temperature=s["inv_temperature"]))
    if "dlogprob" in s:
        out |= r.backward(s["logits"], s["tokens"], s["dlogprob"], s["dentropy"], mask=s["mask"], inv_temperature=s["inv_temperature"])
    return out


def _own_ortho(s):
    return s["runner"].step(s["grad"], s["momentum"], s["master"], mu=MU, lr=LR, decay=DECAY)


def _columns(w):
    return w[None, :, None, None]


def _plain_norm(s):
    gate, dt = s["case"]["gate"], s["x"].dtype
    x, z = s["x"].float(), s["z"].float()
    w2, sc, w1 = _columns(s["w_post"]), _columns(s["scale"]), _columns(s["w_pre"])
    r2 = torch.rsqrt((z * z).mean(1, keepdim=True) + EPS)
    zn = z * r2
    if gate == "none":
        a, da = torch.ones((), device=x.device), None
    else:
        g = s["gate"].float()
        sig = 1 / (1 + torch.exp(-g))
        a = sig if gate == "sigmoid" else g * sig
        da = sig * (1 - sig) if gate == "sigmoid" else sig * (1 + g * (1 - sig))
    y = x + sc * a * (zn * w2)
    r1 = torch.rsqrt((y * y).mean(1, keepdim=True) + EPS)
    yn = y * r1
    out = {"x_out": y.to(dt), "u": (yn * w1).to(dt)}
    if "du" not in s:
        return out
    du = s["du"].float()
    dyn = du * w1
    dy = s["dx_out"].float() + r1 * (dyn - yn * (dyn * yn).mean(1, keepdim=True))
    t = dy * a * zn
    dzn = dy * a * (sc * w2)
    out["dx"] = dy.to(dt)
    out["dz"] = (r2 * (dzn - zn * (dzn * zn).mean(1, keepdim=True))).to(dt)
    if da is not None:
        out["dgate"] = (dy * da * zn * (sc * w2)).to(dt)
    k = t.sum((0, 2, 3))
    out["dw_post"], out["dscale"] = k * s["scale"], k * s["w_post"]
    out["dw_pre"] = (du * yn).sum((0, 2, 3))
    return out


def _plain_logprob(s):
    k, it = s["case"]["top"], s["inv_temperature"]
    raw = s["logits"].float()
    if s["mask"] is not None:
        raw = torch.where(s["mask"] != 0, raw, torch.full((), -math.inf, device=raw.device))
    z = raw * it
    d = z - z.amax(1, keepdim=True)
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    logp = d - log_total
    p = e / total
    tiny = torch.where(p > 0, p * logp, torch.zeros((), device=p.device))
    entropy = -tiny.sum(1)
    out = {"logprob": logp.gather(1, s["tokens"][:, None])[:, 0], "entropy": entropy}
    if k:
        index = torch.sort(raw, dim=1, descending=True, stable=True).indices[:, :k]
        out["top_logprob"] = logp.gather(1, index)
        out["top_index"] = index.to(torch.int32)
    if "dlogprob" in s:
        g, h = s["dlogprob"][:, None], s["dentropy"][:, None]
        dz = -g * p - h * (tiny + p * entropy[:, None])
        dz = dz.scatter_add(1, s["tokens"][:, None], g)
        out["dlogits"] = (dz * it).to(s["logits"].dtype)
    return out


def _plain_ortho(s):
    a, b, c = NS_COEFFICIENTS
    dt = DTYPES[s["case"]["dtype"]]
    m = MU * s["momentum"] + s["grad"]
    v = s["grad"] + MU * m
    x = v / (torch.sqrt((v * v).sum((1, 2), keepdim=True)) + NS_EPS)
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    for _ in range(5):
        q = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * q + c * torch.bmm(q, q), x)
    if tall:
        x = x.transpose(1, 2).contiguous()
    out = {"update": x.to(dt), "momentum": m}
    if s["master"] is not None:
        w = (1 - LR * DECAY) * s["master"] - LR * x
        out["master"], out["weights"] = w, w.to(dt)
    return out


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    s = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in s.items()}
    if case["op"] == "norm":
        return _exact_norm(case, s)
    if case["op"] == "logprob":
        return _exact_logprob(case, s)
    return _exact_ortho(case, s)


def _exact_norm(case, s):
    n, c = case["N"], case["C"]
    rows = {k: s[k].reshape(n, c, -1) for k in ("x", "z", "gate", "dx_out", "du") if s.get(k) is not None}
    w2, sc, w1 = (s[k].reshape(1, c, 1) for k in ("w_post", "scale", "w_pre"))
    z = rows["z"]
    inv_z = ((z ** 2).sum(1, keepdim=True) / c + EPS) ** -0.5
    act = slope = 1.0
    if case["gate"] != "none":
        sg = torch.sigmoid(rows["gate"])
        act, slope = (sg, sg - sg ** 2) if case["gate"] == "sigmoid" else (rows["gate"] * sg, sg + rows["gate"] * (sg - sg ** 2))
    branch = sc * w2 * z * inv_z
    y = rows["x"] + branch * act
    inv_y = ((y ** 2).sum(1, keepdim=True) / c + EPS) ** -0.5
    shape = s["x"].shape
    out = {"x_out": y.reshape(shape), "u": (y * inv_y * w1).reshape(shape)}
    if case["mode"] == "train":
        du = rows["du"]
        along = (du * w1 * y).sum(1, keepdim=True) / c
        dy = rows["dx_out"] + inv_y * du * w1 - inv_y ** 3 * y * along
        dbranch = dy * act
        dzh = dbranch * sc * w2
        along = (dzh * z).sum(1, keepdim=True) / c
        out["dx"] = dy.reshape(shape)
        out["dz"] = (inv_z * dzh - inv_z ** 3 * z * along).reshape(shape)
        if case["gate"] != "none":
            out["dgate"] = (dy * branch * slope).reshape(shape)
        out["dw_post"] = (dbranch * sc * z * inv_z).sum((0, 2))
        out["dscale"] = (dbranch * w2 * z * inv_z).sum((0, 2))
        out["dw_pre"] = (du * y * inv_y).sum((0, 2))
    return out


def _exact_logprob(case, s):
    raw = s["logits"]
    if s["mask"] is not None:
        raw = raw.masked_fill(s["mask"] == 0, -math.inf)
    z = raw * s["inv_temperature"]
    lse = torch.logsumexp(z, 1)
    logp = z - lse[:, None]
    p = torch.exp(logp)
    plogp = torch.xlogy(p, p) if s["mask"] is None else torch.where(p > 0, p * logp, torch.zeros_like(p))
    out = {"logprob": logp[torch.arange(case["rows"], device=z.device), s["tokens"]], "entropy": -plogp.sum(1)}
    if case["top"]:
        out["top_logprob"] = logp.topk(case["top"], 1).values
        out["top_index"] = None
    if case["mode"] == "train":
        g, h = s["dlogprob"], s["dentropy"]
        dz = -p * g[:, None] - (plogp + p * out["entropy"][:, None]) * h[:, None]
        dz[torch.arange(case["rows"], device=z.device), s["tokens"]] += g
        out["dlogits"] = dz * s["inv_temperature"]
    return out


def _exact_ortho(case, s):
    a, b, c = NS_COEFFICIENTS
    m = MU * s["momentum"] + s["grad"]
    v = s["grad"] + MU * m
    update = []
    for x in v:
        x = x / (x.norm() + NS_EPS)
        wide = x if case["R"] <= case["K"] else x.T.contiguous()
        eye = torch.eye(wide.shape[0], dtype=x.dtype, device=x.device)
        for _ in range(5):
            q = wide @ wide.T
            wide = (a * eye + b * q + c * (q @ q)) @ wide
        update.append(wide if case["R"] <= case["K"] else wide.T)
    update = torch.stack(update)
    out = {"update": update, "momentum": m}
    if case["master"]:
        out["master"] = (1 - LR * DECAY) * s["master"] - LR * update
        out["weights"] = out["master"]
    return out
