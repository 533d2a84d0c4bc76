"""Device-memory plumbing around the C-ABI binding: allocates torch tensors, uploads a workload,
calls forward/backward and downloads results.  No arithmetic of the method happens here."""
import math

import numpy as np
import torch

from . import binding as B


class DagRunner:
    """Owns one compiled micro-DAG plus the device buffers of one workload."""

    def __init__(self, blob, shape, dtype, flags=0, device="cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU: the micro-DAG executor has no CPU path")
        self.device = torch.device(device)
        self.bf16 = dtype == "bf16"
        self.tdtype = torch.bfloat16 if self.bf16 else torch.float32
        self.handle = B.canvas_dag_compile(blob, shape, B.CANVAS_BF16 if self.bf16 else B.CANVAS_F32, flags)
        self.info = B.canvas_dag_query(self.handle)
        self.shape = tuple(int(v) for v in shape)
        self.out_shape = tuple(int(v) for v in self.info.out_shape)
        self.wshapes = [tuple(int(v) for v in self.info.weight_shape[k]) for k in range(self.info.n_weights)]
        self.ws = torch.empty(max(16, int(self.info.workspace_bytes)), dtype=torch.uint8, device=self.device)
        self.x = torch.empty(self.shape, dtype=self.tdtype, device=self.device)
        self.y = torch.empty(self.out_shape, dtype=self.tdtype, device=self.device)
        self.dy = torch.empty(self.out_shape, dtype=self.tdtype, device=self.device)
        self.dx = torch.empty(self.shape, dtype=self.tdtype, device=self.device)
        self.w = [torch.empty(s, dtype=self.tdtype, device=self.device) for s in self.wshapes]
        self.dw = [torch.empty(s, dtype=torch.float32, device=self.device) for s in self.wshapes]

    def close(self):
        if self.handle is not None:
            B.canvas_dag_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _up(self, dst, a):
        dst.copy_(torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).reshape(dst.shape).to(self.tdtype))

    def load(self, x, weights, dy=None):
        self._up(self.x, x)
        for t, a in zip(self.w, weights):
            self._up(t, a)
        if dy is not None:
            self._up(self.dy, dy)

    def prepare(self):
        B.canvas_dag_prepare(self.handle, self.w, self.ws)

    def forward(self):
        B.canvas_dag_forward(self.handle, self.x, self.w, self.y, self.ws)

    def backward(self):
        B.canvas_dag_backward(self.handle, self.x, self.w, self.dy, self.dx, self.dw, self.ws)

    def poison_outputs(self):
        """Fill outputs with NaN so that an element no kernel writes is caught."""
        for t in [self.y, self.dx, *self.dw]:
            t.fill_(float("nan"))

    def results(self):
        torch.cuda.synchronize()
        out = {"y": self.y.float().cpu().numpy(), "dx": self.dx.float().cpu().numpy(),
               "dw": [t.cpu().numpy() for t in self.dw]}
        if out["y"].shape[2] == 1:
            out["y"] = out["y"].reshape(out["y"].shape[0], out["y"].shape[1], *out["y"].shape[3:])
        return out

    def launches(self, backward):
        n = self.info.n_launches_bwd if backward else self.info.n_launches_fwd
        return [B.canvas_dag_launch_desc(self.handle, backward, i) for i in range(n)]


class BlockRunner:
    """Owns one compiled block (a template composed for C_in != C_out) plus the device buffers of one workload."""

    def __init__(self, blob, shape, c_out, dtype, flags=0, device="cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU: the micro-DAG executor has no CPU path")
        self.device = torch.device(device)
        self.bf16 = dtype == "bf16"
        self.tdtype = torch.bfloat16 if self.bf16 else torch.float32
        self.handle = B.canvas_block_compile(blob, shape, c_out, B.CANVAS_BF16 if self.bf16 else B.CANVAS_F32, flags)
        self.info = B.canvas_block_query(self.handle)
        n, _, h, w = (int(v) for v in shape)
        self.m = int(self.info.instances)
        wshapes = [tuple(int(v) for v in self.info.plan.weight_shape[k]) for k in range(self.info.n_weights)]
        self.ws = torch.empty(max(16, int(self.info.workspace_bytes)), dtype=torch.uint8, device=self.device)
        self.x = torch.empty(tuple(int(v) for v in shape), dtype=self.tdtype, device=self.device)
        self.y = torch.empty((n, int(c_out), h, w), dtype=self.tdtype, device=self.device)
        self.dy = torch.empty_like(self.y)
        self.dx = torch.empty_like(self.x)
        self.w = [torch.empty(s, dtype=self.tdtype, device=self.device) for _ in range(self.m) for s in wshapes]
        self.dw = [torch.empty(s, dtype=torch.float32, device=self.device) for _ in range(self.m) for s in wshapes]

    def close(self):
        if self.handle is not None:
            B.canvas_block_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _up(self, dst, a):
        dst.copy_(torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).reshape(dst.shape).to(self.tdtype))

    def load(self, x, weights, dy):
        """weights: m lists (one per instance) of arrays."""
        self._up(self.x, x)
        flat = [a for inst in weights for a in inst]
        for t, a in zip(self.w, flat):
            self._up(t, a)
        self._up(self.dy, dy)

    def run(self):
        for t in [self.y, self.dx, *self.dw]:
            t.fill_(float("nan"))
        self.ws.fill_(0xFF)  # (bf16 / fp32 NaN patterns: nothing may be read before it is written)
        B.canvas_block_forward(self.handle, self.x, self.w, self.y, self.ws)
        B.canvas_block_backward(self.handle, self.x, self.w, self.dy, self.dx, self.dw, self.ws)
        torch.cuda.synchronize()
        nw = int(self.info.n_weights)
        dw = [t.cpu().numpy() for t in self.dw]
        return {"y": self.y.float().cpu().numpy(), "dx": self.dx.float().cpu().numpy(),
                "dw": [dw[j * nw:(j + 1) * nw] for j in range(self.m)]}


def _check_tensor(name, t, shape, dtype, device):
    """The library takes addresses: what a runner hands on has to be what its plan was compiled for."""
    if t is None or t.shape != shape or t.dtype is not dtype or t.device != device or not t.is_contiguous():
        got = "None" if t is None else f"{tuple(t.shape)} {t.dtype} on {t.device}, strides {t.stride()}"
        raise ValueError(f"{name}: a contiguous {shape} tensor of {dtype} on {device} is needed, got {got}")


def _check_last(passed, given):
    """backward() reads what the last forward() has left in the workspace: it takes the same arguments (tensors: the same memory, which the runner keeps alive)."""
    same = lambda a, b: a.data_ptr() == b.data_ptr() if torch.is_tensor(a) and torch.is_tensor(b) else a is b or (not torch.is_tensor(a) and a == b)  # noqa: E731
    if passed is None or not all(same(a, b) for a, b in zip(passed, given)):
        raise ValueError("not the arguments of this runner's last forward()")


# (no part of torch's interface, so it may be missing; current_device() takes 0.3 us longer)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


class _PlanRunner:
    """One compiled plan, its workspace and the buffers it writes; close() releases the plan."""

    handle = None

    def _open(self, dtype, device):
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU: the library has no CPU path")
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device(self.device.type, torch.cuda.current_device())
        self.tdtype = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        self.cdtype = B.CANVAS_BF16 if dtype == "bf16" else B.CANVAS_F32

    def _call(self, f, *args):
        """On the runner's device, on torch's current stream of it, whichever device is the current one."""
        if _current_device() == self.device.index:
            return f(*args)
        with torch.cuda.device(self.device):
            return f(*args)

    def _workspace(self, n):
        return torch.empty(max(16, int(n)), dtype=torch.uint8, device=self.device)

    def _empty(self, shape, dtype=None):
        return torch.empty(shape, dtype=dtype or self.tdtype, device=self.device)

    def close(self):
        if self.handle is not None:
            self._destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class NormRunner(_PlanRunner):
    """The norms between two blocks (include/canvas_norm.h): x' = x + scale act(gate) norm(z) w_post, u = norm(x') w_pre.

    forward() and backward() take the caller's tensors and return the runner's own buffers, which the next call overwrites:
    backward() is of the last forward(), and knows it by the x_out that this returned.  Between the two the caller leaves x as it is.
    """

    _destroy = staticmethod(B.canvas_norm_destroy)

    def __init__(self, shape, dtype, parts, gate=B.CANVAS_GATE_NONE, eps=1e-6, flags=0, device="cuda:0"):
        self._open(dtype, device)
        self.shape = tuple(int(v) for v in shape)
        self.handle = B.canvas_norm_compile(self.shape, self.cdtype, parts, gate, eps, flags)
        self.info = B.canvas_norm_query(self.handle)
        self.post, self.pre, self.gate = bool(parts & B.CANVAS_NORM_POST), bool(parts & B.CANVAS_NORM_PRE), gate != B.CANVAS_GATE_NONE
        self.ws = self._workspace(self.info.workspace_bytes)
        self.x = self.passed = None
        self.out = {}
        if self.post:
            self.out["x_out"] = self._empty(self.shape)
        if self.pre:
            self.out["u"] = self._empty(self.shape)
        self.grads = {}
        if not flags & B.CANVAS_OPT_INFERENCE:
            c = self.shape[1:2]
            if self.pre:
                self.grads |= {"dx": self._empty(self.shape), "dw_pre": self._empty(c, torch.float32)}
            if self.post:
                self.grads |= {"dz": self._empty(self.shape), "dw_post": self._empty(c, torch.float32), "dscale": self._empty(c, torch.float32)}
            if self.gate:
                self.grads["dgate"] = self._empty(self.shape)

    def _map(self, name, t):
        _check_tensor(name, t, self.shape, self.tdtype, self.device)

    def _of_the_block(self, z, gate, w_post, scale, w_pre):
        c = self.shape[1:2]
        if self.post:
            self._map("z", z)
            _check_tensor("w_post", w_post, c, torch.float32, self.device)
            _check_tensor("scale", scale, c, torch.float32, self.device)
        if self.gate:
            self._map("gate", gate)
        if self.pre:
            _check_tensor("w_pre", w_pre, c, torch.float32, self.device)

    def forward(self, x, z=None, gate=None, w_post=None, scale=None, w_pre=None):
        self._of_the_block(z, gate, w_post, scale, w_pre)
        self._map("x", x)
        self._call(B.canvas_norm_forward, self.handle, x, z, gate, w_post, scale, w_pre, self.out.get("x_out"), self.out.get("u"), self.ws)
        self.x, self.passed = x, self.out["x_out"] if self.post else x
        if not (self.post and self.grads):
            return self.out
        # every pass that may have a backward() hands out a tensor object of its own over the one buffer: those of earlier passes are told apart by it
        self.passed = self.out["x_out"].detach()
        return {**self.out, "x_out": self.passed}

    def backward(self, x_out, z=None, gate=None, w_post=None, scale=None, w_pre=None, dx_out=None, du=None):
        """Of the runner's last forward(), whose x it has kept.  x_out: what that very call returned under that name (x itself in a
        plan without POST); what an earlier one returned is refused.  The kernel computes its values again in fp32."""
        if self.x is None or x_out is not self.passed:
            raise ValueError("x_out: not the result of this runner's last forward()")
        self._of_the_block(z, gate, w_post, scale, w_pre)
        if self.pre:
            self._map("du", du)
        if dx_out is not None or not self.pre:
            self._map("dx_out", dx_out)
        g = self.grads
        self._call(B.canvas_norm_backward, self.handle, self.x, z, gate, w_post, scale, w_pre, dx_out, du, g.get("dx"), g.get("dz"), g.get("dgate"),
                   g.get("dw_post"), g.get("dscale"), g.get("dw_pre"), self.ws)
        return g


class LogprobRunner(_PlanRunner):
    """Log probabilities of tokens with entropy and top alternatives (include/canvas_logprob.h), and their gradient.

    logits: [rows, classes] with any row pitch; mask: [rows, classes] or [classes] bytes, zero where a class is not allowed.
    """

    _destroy = staticmethod(B.canvas_logprob_destroy)

    def __init__(self, rows, classes, dtype, top_k=0, flags=0, device="cuda:0"):
        self._open(dtype, device)
        self.rows, self.classes, self.top = int(rows), int(classes), int(top_k)
        self.handle = B.canvas_logprob_compile(rows, classes, self.cdtype, top_k, flags)
        self.info = B.canvas_logprob_query(self.handle)
        self.ws = self._workspace(self.info.workspace_bytes)
        self.out = {"logprob": self._empty(self.rows, torch.float32), "entropy": self._empty(self.rows, torch.float32)}
        if self.top:
            self.out |= {"top_logprob": self._empty((self.rows, self.top), torch.float32), "top_index": self._empty((self.rows, self.top), torch.int32)}
        self.grads = {} if flags & B.CANVAS_OPT_INFERENCE else {"dlogits": self._empty((self.rows, self.classes))}

    def _arguments(self, logits, tokens, mask):
        """(pitch, mask pitch) of tensors that were checked."""
        if logits.shape != (self.rows, self.classes) or logits.dtype is not self.tdtype or logits.device != self.device \
                or (logits.stride(1) != 1 and self.classes > 1):
            raise ValueError(f"logits: a {(self.rows, self.classes)} tensor of {self.tdtype} on {self.device} with dense rows is needed")
        _check_tensor("tokens", tokens, (self.rows,), torch.int64, self.device)
        pitch = logits.stride(0) if self.rows > 1 else self.classes
        if mask is None:
            return pitch, 0
        if mask.dtype not in (torch.uint8, torch.bool) or mask.device != self.device or (mask.stride(-1) != 1 and self.classes > 1) \
                or tuple(mask.shape) not in ((self.classes,), (self.rows, self.classes)):
            raise ValueError(f"mask: bytes or truth values of {(self.rows, self.classes)} or {(self.classes,)} on {self.device} are needed")
        return pitch, mask.stride(0) if mask.dim() == 2 and self.rows > 1 else 0

    def forward(self, logits, tokens, mask=None, inv_temperature=1.0):
        pitch, mask_pitch = self._arguments(logits, tokens, mask)
        o = self.out
        self._call(B.canvas_logprob_forward, self.handle, logits, pitch, inv_temperature, mask, mask_pitch, tokens, o["logprob"], o["entropy"],
                   o.get("top_logprob"), o.get("top_index"), self.ws)
        return o

    def backward(self, logits, tokens, dlogprob=None, dentropy=None, mask=None, inv_temperature=1.0):
        pitch, mask_pitch = self._arguments(logits, tokens, mask)
        for name, t in (("dlogprob", dlogprob), ("dentropy", dentropy)):
            if t is not None:
                _check_tensor(name, t, (self.rows,), torch.float32, self.device)
        self._call(B.canvas_logprob_backward, self.handle, logits, pitch, inv_temperature, mask, mask_pitch, tokens, dlogprob, dentropy,
                   self.grads["dlogits"], self.classes, self.ws)
        return self.grads


class OrthoRunner(_PlanRunner):
    """Orthogonalised update of an FC weight (include/canvas_ortho.h): shape [G, R, K] as the DAG's weight_shape."""

    _destroy = staticmethod(B.canvas_ortho_destroy)

    def __init__(self, shape, dtype, steps=5, flags=0, device="cuda:0"):
        self._open(dtype, device)
        self.shape = tuple(int(v) for v in shape)
        self.handle = B.canvas_ortho_compile(self.shape, self.cdtype, steps, flags)
        self.info = B.canvas_ortho_query(self.handle)
        self.ws = self._workspace(self.info.workspace_bytes)
        self.out = {"update": self._empty(self.shape)}

    def _buffer(self, name, dtype=None):
        if name not in self.out:
            self.out[name] = self._empty(self.shape, dtype)
        return self.out[name]

    def step(self, grad, momentum=None, master=None, mu=0.95, lr=0.0, decay=0.0):
        """Returns update, and momentum and master / weights where they were given: buffers of the runner, the arguments stay as
        they are."""
        for name, t in (("grad", grad), ("momentum", momentum), ("master", master)):
            if t is not None or name == "grad":
                _check_tensor(name, t, self.shape, torch.float32, self.device)
        names = ["update"]
        m = w = p = None
        if momentum is not None:
            m = self._buffer("momentum", torch.float32)
            names.append("momentum")
        if master is not None:
            w, p = self._buffer("master", torch.float32), self._buffer("weights")
            names += ["master", "weights"]
        self._call(B.canvas_ortho_step, self.handle, grad, momentum, m, mu, master, w, lr, decay, p, self.out["update"], self.ws)
        return {k: self.out[k] for k in names}


class GatedRunner(_PlanRunner):
    """A gated pair of FCs (include/canvas_gated.h): y = act(x w_gate^T) (x w_up^T); x [rows, features], weights [width, features].

    forward() and backward() return the runner's own buffers, which the next call overwrites; backward() is of the last forward(), whose
    tensors it is given again.
    """

    _destroy = staticmethod(B.canvas_gated_destroy)
    passed = None

    def __init__(self, rows, features, width, dtype, act=B.CANVAS_GATED_SILU, flags=0, device="cuda:0"):
        self._open(dtype, device)
        self.shape, self.wshape = (int(rows), int(features)), (int(width), int(features))
        self.handle = B.canvas_gated_compile(rows, features, width, self.cdtype, act, flags)
        self.info = B.canvas_gated_query(self.handle)
        self.ws = self._workspace(self.info.workspace_bytes)
        self.out = {"y": self._empty((self.shape[0], self.wshape[0]))}
        self.grads = {}
        if not flags & B.CANVAS_OPT_INFERENCE:
            self.grads = {"dx": self._empty(self.shape), "dw_gate": self._empty(self.wshape), "dw_up": self._empty(self.wshape)}

    def _arguments(self, x, w_gate, w_up):
        _check_tensor("x", x, self.shape, self.tdtype, self.device)
        _check_tensor("w_gate", w_gate, self.wshape, self.tdtype, self.device)
        _check_tensor("w_up", w_up, self.wshape, self.tdtype, self.device)

    def forward(self, x, w_gate, w_up):
        self._arguments(x, w_gate, w_up)
        self._call(B.canvas_gated_forward, self.handle, x, w_gate, w_up, self.out["y"], self.ws)
        self.passed = (x, w_gate, w_up)
        return self.out

    def backward(self, x, w_gate, w_up, dy):
        self._arguments(x, w_gate, w_up)
        _check_last(self.passed, (x, w_gate, w_up))
        _check_tensor("dy", dy, self.out["y"].shape, self.tdtype, self.device)
        g = self.grads
        self._call(B.canvas_gated_backward, self.handle, x, w_gate, w_up, dy, g.get("dx"), g.get("dw_gate"), g.get("dw_up"), self.ws)
        return g


class HeadRunner(_PlanRunner):
    """Log probabilities of tokens with entropy from features and the head's weight (include/canvas_head.h), and the gradients of both.

    x [rows, features], weight [classes, features]; mask: [classes] bytes or truth values, zero where a class is not allowed.
    forward() and backward() return the runner's own buffers, which the next call overwrites; backward() is of the last forward(), whose
    x, weight, mask and temperature it is given again.
    """

    _destroy = staticmethod(B.canvas_head_destroy)
    passed = None

    def __init__(self, rows, features, classes, dtype, flags=0, device="cuda:0"):
        self._open(dtype, device)
        self.rows, self.classes = int(rows), int(classes)
        self.shape, self.wshape = (self.rows, int(features)), (self.classes, int(features))
        self.handle = B.canvas_head_compile(rows, features, classes, self.cdtype, flags)
        self.info = B.canvas_head_query(self.handle)
        self.ws = self._workspace(self.info.workspace_bytes)
        self.out = {"logprob": self._empty(self.rows, torch.float32), "entropy": self._empty(self.rows, torch.float32)}
        self.grads = {} if flags & B.CANVAS_OPT_INFERENCE else {"dx": self._empty(self.shape), "dweight": self._empty(self.wshape)}

    def _arguments(self, x, weight, tokens, mask):
        _check_tensor("x", x, self.shape, self.tdtype, self.device)
        _check_tensor("weight", weight, self.wshape, self.tdtype, self.device)
        _check_tensor("tokens", tokens, (self.rows,), torch.int64, self.device)
        if mask is not None:
            _check_tensor("mask", mask, (self.classes,), torch.bool if mask.dtype is torch.bool else torch.uint8, self.device)

    def forward(self, x, weight, tokens, mask=None, inv_temperature=1.0):
        self._arguments(x, weight, tokens, mask)
        self._call(B.canvas_head_forward, self.handle, x, weight, inv_temperature, mask, tokens, self.out["logprob"], self.out["entropy"], self.ws)
        self.passed = (x, weight, mask, inv_temperature)
        return self.out

    def backward(self, x, weight, tokens, dlogprob=None, dentropy=None, mask=None, inv_temperature=1.0):
        self._arguments(x, weight, tokens, mask)
        _check_last(self.passed, (x, weight, mask, inv_temperature))
        for name, t in (("dlogprob", dlogprob), ("dentropy", dentropy)):
            if t is not None:
                _check_tensor(name, t, (self.rows,), torch.float32, self.device)
        g = self.grads
        self._call(B.canvas_head_backward, self.handle, x, weight, inv_temperature, mask, tokens, dlogprob, dentropy, g.get("dx"), g.get("dweight"), self.ws)
        return g


class ClipRunner(_PlanRunner):
    """The norm over all gradients and their scaling to a largest norm (include/canvas_clip.h).

    shapes, dtypes ("f32" or "bf16") and out_dtypes (the dtypes themselves if they are not given): one for each tensor.
    """

    _destroy = staticmethod(B.canvas_clip_destroy)

    def __init__(self, shapes, dtypes, out_dtypes=None, device="cuda:0"):
        kinds = {"f32": (torch.float32, B.CANVAS_F32), "bf16": (torch.bfloat16, B.CANVAS_BF16)}
        out_dtypes = list(dtypes) if out_dtypes is None else list(out_dtypes)
        self._open("f32", device)
        self.shapes = [tuple(int(v) for v in s) for s in shapes]
        self.dtypes, self.out_dtypes = [kinds[t][0] for t in dtypes], [kinds[t][0] for t in out_dtypes]
        counts = [math.prod(s) for s in self.shapes]
        self.handle = B.canvas_clip_compile(counts, [kinds[t][1] for t in dtypes], [kinds[t][1] for t in out_dtypes])
        self.info = B.canvas_clip_query(self.handle)
        self.ws = self._workspace(self.info.workspace_bytes)
        self.norm, self.scale = self._empty((), torch.float32), self._empty((), torch.float32)
        self.outs = None

    def step(self, grads, max_norm, in_place=False):
        """Returns norm, scale and grads, the scaled ones: buffers of the runner, or with in_place the arguments themselves."""
        if len(grads) != len(self.shapes):
            raise ValueError(f"grads: {len(self.shapes)} tensors are needed, got {len(grads)}")
        for i, (t, s, d) in enumerate(zip(grads, self.shapes, self.dtypes)):
            if t is None or t.shape != s or t.dtype is not d or t.device != self.device or not t.is_contiguous():
                _check_tensor(f"grads[{i}]", t, s, d, self.device)
        if in_place:
            outs = grads
        else:
            if self.outs is None:
                self.outs = [self._empty(s, d) for s, d in zip(self.shapes, self.out_dtypes)]
            outs = self.outs
        self._call(B.canvas_clip_step, self.handle, grads, outs, max_norm, self.norm, self.scale, self.ws)
        return {"norm": self.norm, "scale": self.scale, "grads": list(outs)}


def run_case(case, flags=0, dy=None):
    """Upload a workload (see workloads.py), run forward + backward, return (results, runner)."""
    from . import workloads as wl

    r = DagRunner(case["blob"], case["shape"], case["dtype"], flags)
    if dy is None:
        shp = r.out_shape if r.out_shape[2] != 1 else (r.out_shape[0], r.out_shape[1], *r.out_shape[3:])
        dy = wl.make_dy(case, shp)
    r.load(case["x"], case["weights"], dy)
    r.poison_outputs()
    r.forward()
    r.backward()
    return r.results(), r, dy
