"""Gradient norms and clipping of K replicas, as timed cases: the operators in plain torch, and the framework's calls.

A case is a model's parameter list, a replica count, a storage type and one of the operators:

  norms    each replica's gradient norm over its whole parameter list
  clip     new gradients arrive in the bound buffers and are scaled in place to a norm of at most max_norm
  step     a local step with clipped gradients, which stay as they are
  cycle    what a training loop issues between two global updates, every step clipped
  sgd_ar   the synchronous comparator: one step of all replicas with the clipped mean gradient
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False
DEV = "cuda:0"
MU, WD = 0.9, 1e-4             # momentum and weight decay of the workloads in use
EPS = 1e-6                     # the coefficient is max_norm / (norm + EPS), at most 1


# ---- parameter lists: element counts in module order ---------------------------------------------------------------
def _resnet(blocks, wide):
    out, width = [64 * 3 * 49, 64, 64], 64
    for stage, count in enumerate(blocks):
        p = 64 << stage
        for b in range(count):
            convs = [(p, width, 1), (p, p, 9), (4 * p, p, 1)] if wide else [(p, width, 9), (p, p, 9)]
            end = convs[-1][0]
            if b == 0 and width != end:
                convs.append((end, width, 1))
            for o, i, k in convs:
                out += [o * i * k, o, o]
            width = end
    return out + [1000 * width, 1000]


def _mobilenet_v2():
    out, width = [32 * 3 * 9, 32, 32], 32
    for t, c, n in ((1, 16, 1), (6, 24, 2), (6, 32, 3), (6, 64, 4), (6, 96, 3), (6, 160, 3), (6, 320, 1)):
        for _ in range(n):
            h = t * width
            if t != 1:
                out += [h * width, h, h]
            out += [h * 9, h, h, c * h, c, c]
            width = c
    return out + [1280 * width, 1280, 1280, 1000 * 1280, 1000]


def _numels(c):
    if c["list"] == "flat":                                 # one vector: a flattened model
        return [int(c["n"])]
    if c["list"] == "small":                                # the framework's own ragged little list
        return [5, 1024, 1, 4099, 260, 64]
    if c["list"] == "ragged":                               # `tensors` tensors of very unlike, odd sizes, about n elements
        r = random.Random(int(c["lseed"]))
        w = [math.exp(r.uniform(0.0, 8.0)) for _ in range(int(c["tensors"]))]
        return [max(1, int(c["n"] * a / sum(w))) for a in w]
    if c["list"] == "mobilenetv2":
        return _mobilenet_v2()
    return _resnet((2, 2, 2, 2), False) if c["list"] == "resnet18" else _resnet((3, 4, 6, 3), True)


def _offsets(c):
    """Where each tensor starts in a replica's flat buffer: on 256 elements, or (`tight`) on the 16 bytes that are required."""
    align = 8 if c.get("tight") else 256
    off = [0]
    for n in _numels(c):
        off.append(off[-1] + (n + align - 1) // align * align)
    return off


# ---- the cases -------------------------------------------------------------------------------------------------------
def listed():
    return [
        # the smallest call: a handful of short, odd tensors whose norms are logged every step; latency is all
        dict(name="norms-small-k3", op="norms", list="small", K=3, storage="f32"),
        # norms alone over the largest gradients, 16 bits each
        dict(name="norms-resnet50-bf16-k32", op="norms", list="resnet50", K=32, storage="bf16"),
        # a flattened model of a million parameters, clipped for an update of the caller's own
        dict(name="clip-flat-1m-k4", op="clip", list="flat", n=1 << 20, K=4, storage="f32"),
        # many small tensors, 16 bits
        dict(name="clip-mobilenetv2-bf16-k16", op="clip", list="mobilenetv2", K=16, storage="bf16"),
        # gradients far beyond any cache, scaled in place
        dict(name="clip-resnet50-k8", op="clip", list="resnet50", K=8, storage="f32"),
        # a short clipped step: a head or an adapter being tuned
        dict(name="step-small-k3", op="step", list="small", K=3, storage="f32"),
        # the ordinary size; one replica's gradients hold an infinity, and it sits the step out
        dict(name="step-resnet18-k8", op="step", list="resnet18", K=8, storage="f32", skip=True, bad=1),
        # the largest: bf16 parameters and gradients with fp32 masters
        dict(name="step-resnet50-bf16-k32", op="step", list="resnet50", K=32, storage="bf16"),
        # a global update every second step, some replicas without a local step in it (replicas at their own pace)
        dict(name="cycle-mobilenetv2-k16", op="cycle", list="mobilenetv2", K=16, m=2, storage="f32", rseed=5, skip=True),
        # the headline cycle, every step clipped, the mean on a second stream
        dict(name="cycle-resnet50-k8", op="cycle", list="resnet50", K=8, m=4, storage="f32"),
        # the synchronous comparator on a small model and on the headline's
        dict(name="sgdar-flat-1m-k4", op="sgd_ar", list="flat", n=1 << 20, K=4, storage="f32"),
        dict(name="sgdar-resnet50-k8", op="sgd_ar", list="resnet50", K=8, storage="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = dict(op=rng.choice(["norms", "clip", "step", "step", "cycle", "sgd_ar"]),
             list=rng.choice(["flat", "ragged", "ragged", "mobilenetv2", "resnet18", "resnet50"]))
    if c["list"] in ("flat", "ragged"):
        c["n"] = _log(rng, 1000, 3.0e7)
    if c["list"] == "ragged":
        c["tensors"] = _log(rng, 2, 250)
        c["lseed"] = rng.randrange(1 << 20)
    c["K"] = _log(rng, 1, max(1, min(64, int(2.0e8 / sum(_numels(c))))))
    c["storage"] = rng.choice(["f32", "f32", "bf16"])
    c["tight"] = rng.random() < 0.3
    if c["op"] == "cycle":
        c["m"] = rng.choice([1, 2, 3, 4])
    if c["op"] != "sgd_ar" and rng.random() < 0.4:
        c["rseed"] = rng.randrange(1 << 20)
    if c["op"] != "norms":
        c["skip"] = rng.random() < 0.5
    if c.get("skip") and c["op"] != "sgd_ar" and rng.random() < 0.5:
        c["bad"] = rng.randrange(c["K"])
    return c


def _lr(c):
    return {"flat": 0.1, "small": 0.05, "ragged": 0.1, "mobilenetv2": 0.4, "resnet18": 0.4, "resnet50": 0.8}[c["list"]]


def _members(c):
    """Which replicas take part (of a cycle: which take the local step of its last call): all, or about two thirds."""
    if "rseed" not in c:
        return [True] * c["K"]
    r = random.Random(int(c["rseed"]))
    m = [r.random() < 0.67 for _ in range(c["K"])]
    return m if any(m) else [True] * c["K"]


def _mask(members):
    return sum(1 << k for k, m in enumerate(members) if m)


def _max_norm(c):
    """About the middle of the replicas' norms: some are clipped and some are not."""
    n = sum(_numels(c))
    return float(np.float32(1e-3 * math.sqrt(n) / (math.sqrt(c["K"]) if c["op"] == "sgd_ar" else 1.0)))


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _inputs(c, seed):
    """(x [K, total], g [K, total]) on the GPU in the storage type; gaps between tensors hold zeros. Replicas have drifted apart,
    and their gradients differ in scale by up to e either way, as those of different mini-batches do."""
    off, numels = _offsets(c), _numels(c)
    dt = torch.bfloat16 if c["storage"] == "bf16" else torch.float32
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    scale = random.Random(int(seed))
    runs = torch.tensor([v for n, a, b in zip(numels, off, off[1:]) for v in (n, b - a - n)])         # a tensor, the gap behind it, ...
    gap = torch.repeat_interleave(torch.tensor([1.0, 0.0]).repeat(len(numels)), runs).to(DEV)
    x0 = torch.randn(off[-1], generator=gen, device=DEV) * 0.05
    x = torch.empty(c["K"], off[-1], dtype=dt, device=DEV)
    g = torch.empty(c["K"], off[-1], dtype=dt, device=DEV)
    for k in range(c["K"]):
        x[k] = (x0 + torch.randn(off[-1], generator=gen, device=DEV) * 1e-3) * gap
        g[k] = torch.randn(off[-1], generator=gen, device=DEV) * (1e-3 * math.exp(scale.uniform(-1.0, 1.0))) * gap
    if "bad" in c:                                                     # an overflow somewhere in one replica's backward pass
        t = random.Random(int(seed) + 1).randrange(len(numels))
        g[c["bad"], off[t] + numels[t] // 2] = math.inf
    return x, g


class _State:
    pass


def prepare(case, seed):
    c, st = case, _State()
    st.c, st.K, st.lr, st.max_norm = c, c["K"], _lr(c), _max_norm(c)
    st.skip = bool(c.get("skip", False))
    st.x, st.g = _inputs(c, seed)
    st.members = _members(c)
    st.mask, st.full = _mask(st.members), (1 << st.K) - 1
    st.norms = torch.zeros(1 if c["op"] == "sgd_ar" else st.K, device=DEV)
    if c["op"] == "clip":
        st.fresh = st.g.clone()                                        # what the backward passes of a step leave behind
    if not own:                                                        # the optimizer's state, which the framework keeps in its context
        st.part = torch.tensor(st.members, device=DEV)
        if c["op"] in ("step", "cycle", "sgd_ar"):
            st.master = st.x.float() if c["storage"] == "bf16" else st.x
            st.v = torch.zeros(st.x.shape, device=DEV)
        if c["op"] == "cycle":
            st.s = st.master.clone()
        return st
    from paper_2203_13085_amd import binding as B
    st.main = torch.cuda.Stream(device=DEV)
    st.side = torch.cuda.Stream(device=DEV) if c["op"] == "cycle" else st.main
    bf16 = c["storage"] == "bf16"
    off, esize = _offsets(c), 2 if bf16 else 4
    torch.cuda.synchronize()
    st.ctx = B.Context(st.K, _numels(c), storage=B.BF16 if bf16 else B.F32, momentum=MU, nesterov=True, wd_scalar=WD,
                       main_stream=st.main.cuda_stream, side_stream=st.side.cuda_stream)
    for k in range(st.K):
        st.ctx.bind(k, [st.x[k].data_ptr() + o * esize for o in off[:-1]], [st.g[k].data_ptr() + o * esize for o in off[:-1]])
    if bf16:
        st.ctx.init_master()
    if c["op"] == "cycle":
        st.ctx.snapshot()
    return st


# ---- one pass ----------------------------------------------------------------------------------------------------------
def run(state):
    return _calls(state) if own else _plain(state)


def _calls(st):
    c, ctx, norms = st.c, st.ctx, st.norms.data_ptr()
    op = c["op"]
    if op == "norms":
        ctx.grad_norms(norms, st.mask)
        return {"norms": st.norms}
    if op == "clip":
        with torch.cuda.stream(st.main):
            st.g.copy_(st.fresh)
        ctx.clip_grads(st.max_norm, st.mask, skip_nonfinite=st.skip, norms=norms)
        return {"grad": st.g, "norms": st.norms}
    if op == "step":
        ctx.local_step_clip(st.lr, st.max_norm, st.mask, skip_nonfinite=st.skip, norms=norms)
    elif op == "cycle":
        ctx.average()
        for _ in range(c["m"] - 1):
            ctx.local_step_clip(st.lr, st.max_norm, skip_nonfinite=st.skip, norms=norms)
        ctx.step_merge_clip(st.lr, st.max_norm, st.mask, st.full, True, skip_nonfinite=st.skip, norms=norms)
    else:
        ctx.sgd_ar_step_clip(st.lr, st.max_norm, skip_nonfinite=st.skip, norms=norms)
    return {"x": st.x, "norms": st.norms}


def _coefficient(st, norm):
    c = st.max_norm / (norm + EPS)
    return torch.where(c >= 1.0, torch.ones_like(c), c)               # a NaN stays one


def _plain_step(st, g, norm, part):
    """g [K or 1, total] in 32 bits, scaled; rows of part that are to sit the step out keep what they have."""
    g1 = g * _coefficient(st, norm)[:, None] + WD * st.master
    vn = MU * st.v + g1
    xn = st.master - st.lr * (g1 + MU * vn)
    live = part & torch.isfinite(norm) if st.skip else part
    st.v = torch.where(live[:, None], vn, st.v)
    st.master.copy_(torch.where(live[:, None], xn, st.master))


def _plain(st):
    c, op = st.c, st.c["op"]
    if op == "clip":
        st.g.copy_(st.fresh)
    if op == "cycle":
        z = st.s.mean(0)
    g = st.g.float()
    if op == "sgd_ar":
        g = g.mean(0, keepdim=True)
    norm = (g * g).sum(1).sqrt()
    if op == "sgd_ar":
        st.norms.copy_(norm)
        _plain_step(st, g, norm, st.part)
    elif op == "norms":
        st.norms.copy_(torch.where(st.part, norm, st.norms))
        return {"norms": st.norms}
    elif op == "clip":
        live = st.part & torch.isfinite(norm) if st.skip else st.part
        st.norms.copy_(torch.where(st.part, norm, st.norms))
        st.g.copy_(torch.where(live[:, None], g * _coefficient(st, norm)[:, None], g))
        return {"grad": st.g, "norms": st.norms}
    elif op == "step":
        st.norms.copy_(torch.where(st.part, norm, st.norms))
        _plain_step(st, g, norm, st.part)
    else:
        st.norms.copy_(norm if c["m"] > 1 else torch.where(st.part, norm, st.norms))
        for i in range(c["m"]):                                       # the gradients stand in for those of m backward passes
            if i:
                norm = (g * g).sum(1).sqrt()
            _plain_step(st, g, norm, st.part if i == c["m"] - 1 else torch.ones_like(st.part))
        st.master.copy_(z + (st.master - st.s))
        st.s.copy_(st.master)
    if st.master is not st.x:
        st.x.copy_(st.master)
    return {"x": st.x, "norms": st.norms}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------
def work(case):
    """Each call's inputs read once and its outputs written once. A step moves 20 bytes a replica-parameter in either storage type
    (f32: g, x, v in, x, v out; bf16: 2 + 4 + 4 in, 4 + 4 + 2 out) and does 11 operations with the norm's two and the scaling; a global update adds s in
    and out and z once; a mean reads K sent models and writes z. Clipping in place reads the new gradients and writes the scaled ones."""
    c = case
    K, n, e = c["K"], float(sum(_numels(c))), 2.0 if c["storage"] == "bf16" else 4.0
    P = sum(_members(c))
    if c["op"] == "norms":
        return {"bytes": e * P * n + 4.0 * P, "flops": 2.0 * P * n}
    if c["op"] == "clip":
        return {"bytes": 2.0 * e * K * n, "flops": 3.0 * P * n}
    if c["op"] == "step":
        return {"bytes": 20.0 * P * n, "flops": 11.0 * P * n}
    if c["op"] == "cycle":
        m = c["m"]
        steps = (m - 1) * K + P
        return {"bytes": 20.0 * steps * n + 8.0 * (K - P) * n + 8.0 * K * n + 4.0 * n + 4.0 * (K + 1) * n,
                "flops": 11.0 * steps * n + 3.0 * K * n}
    return {"bytes": 20.0 * K * n, "flops": 10.0 * K * n + 3.0 * n}


# ---- the same in 64 bits ------------------------------------------------------------------------------------------------------
def exact(case, seed):
    """One pass, replica by replica, from the definition."""
    c, f = case, lambda a: float(np.float32(a))  # noqa: E731  (the entry points take 32-bit coefficients)
    x, g = _inputs(c, seed)
    K, most, lr, mu, wd = c["K"], _max_norm(c), f(_lr(c)), f(MU), f(WD)
    members, skip = _members(c), bool(c.get("skip", False))

    def clipped(a):
        n = float(torch.linalg.vector_norm(a.double()))
        if skip and not math.isfinite(n):
            return None, n
        return a.double() * min(1.0, most / (n + EPS)), n

    if c["op"] in ("norms", "clip"):
        norms = [clipped(g[k])[1] if members[k] else 0.0 for k in range(K)]
        if c["op"] == "norms":
            return {"norms": torch.tensor(norms, dtype=torch.float64)}
        rows = [clipped(g[k])[0] if members[k] else None for k in range(K)]
        return {"grad": torch.stack([g[k].double() if r is None else r for k, r in enumerate(rows)]), "norms": torch.tensor(norms, dtype=torch.float64)}
    if c["op"] == "sgd_ar":
        total = torch.zeros(g.shape[1], dtype=torch.float64, device=DEV)
        for k in range(K):
            total += g[k]
        shared, norm = clipped(total / K)
    z = None
    if c["op"] == "cycle":
        z = torch.zeros(x.shape[1], dtype=torch.float64, device=DEV)
        for k in range(K):
            z += x[k]
        z /= K
    out, norms = [], []
    for k in range(K):
        w0 = x[k].double()
        if c["op"] == "sgd_ar":
            a, n, steps = shared, norm, 1
        else:
            steps = (c["m"] - 1 if c["op"] == "cycle" else 0) + int(members[k])
            a, n = clipped(g[k])
        w, v = w0.clone(), torch.zeros_like(w0)
        for _ in range(steps if a is not None else 0):
            d = a + wd * w
            v = mu * v + d
            w = w - lr * (d + mu * v)
        if z is not None:
            w = z + (w - w0)
        out.append(w)
        norms.append(n if c["op"] == "sgd_ar" or c["op"] == "cycle" and c["m"] > 1 or members[k] else 0.0)
    return {"x": torch.stack(out), "norms": torch.tensor(norms[:1] if c["op"] == "sgd_ar" else norms, dtype=torch.float64)}
