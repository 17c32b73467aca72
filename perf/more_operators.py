"""The feed-forward half of a language model's layer for K replicas at once, as timed cases: the operators in plain torch, and the
framework's calls, which read each replica's bound weights and leave gradients in its bound buffers.

  dropout      y = residual + drop(x), and the backward pass dx = drop(dy) with the same mask, which is never stored
  norm         h = residual + x, y = gain * h / rms(h), in the storage type or (out8) in 8 bits with a scale for each row
  norm_train   h = residual + drop(x), y as above, then the backward pass with the gain's gradient
  gated        a = act(x Wg^T) * (x Wu^T)
  gated_train  the same and its backward pass with both weights' gradients
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False
DEV = "cuda:0"
EPS = 1e-6                              # under the root of a norm
E4M3_MAX = 448.0
ACTS = ("silu", "gelu", "gelu_tanh", "relu")


# ---- the cases -------------------------------------------------------------------------------------------------------
# A case: K replicas, up to `rows` rows (tokens) each, `cols` columns (the model's width), `wide` the hidden width of a gated block.
# ragged: a seed for unlike numbers of rows, none among them. layout: "dense" [K, rows, cols], "padded" (rows a little apart),
# "turned" [rows, K, cols].
def listed():
    return [
        # the smallest call: a few odd rows of a head or an adapter being tuned; latency is all
        dict(name="dropout-small-k3", op="dropout", K=3, rows=7, cols=260, p=0.1, storage="f32", layout="dense"),
        # the end of a sublayer in training: its output dropped out and added to the residual stream, and back
        dict(name="dropout-residual-bf16-k8", op="dropout", K=8, rows=4096, cols=2048, p=0.1, storage="bf16", layout="dense"),
        # one token a replica: an ensemble of the replicas that answers
        dict(name="norm-token-bf16-k4", op="norm", K=4, rows=1, cols=2048, storage="bf16", layout="dense"),
        # prompts for a product in 8 bits
        dict(name="norm-out8-bf16-k8", op="norm", K=8, rows=2048, cols=4096, storage="bf16", layout="dense", out8=True),
        # odd widths, unlike mini-batches, rows apart
        dict(name="norm-train-odd-k5", op="norm_train", K=5, rows=1531, cols=1023, p=0.0, storage="f32", layout="padded", ragged=11),
        # the largest of the norms
        dict(name="norm-train-bf16-k8", op="norm_train", K=8, rows=4096, cols=2048, p=0.1, storage="bf16", layout="dense"),
        # one token a replica
        dict(name="gated-token-bf16-k4", op="gated", K=4, rows=1, cols=2048, wide=5504, act="silu", storage="bf16", layout="dense"),
        # evaluation of small replicas with odd sizes and unlike prompts
        dict(name="gated-odd-k3", op="gated", K=3, rows=333, cols=515, wide=1030, act="gelu", storage="f32", layout="turned", ragged=3),
        # micro-batches of a few tokens: the weights and their gradients are all there is to move
        dict(name="gated-train-few-bf16-k8", op="gated_train", K=8, rows=4, cols=2048, wide=5504, act="silu", storage="bf16", layout="dense"),
        # small replicas, unlike mini-batches: too little for one replica to fill the chip
        dict(name="gated-train-small-bf16-k16", op="gated_train", K=16, rows=192, cols=512, wide=1408, act="gelu_tanh", storage="bf16", layout="dense", ragged=5),
        # the ordinary size in 32 bits
        dict(name="gated-train-f32-k4", op="gated_train", K=4, rows=1024, cols=1024, wide=2816, act="silu", storage="f32", layout="dense"),
        # the largest
        dict(name="gated-train-bf16-k8", op="gated_train", K=8, rows=2048, cols=2048, wide=5504, act="silu", storage="bf16", layout="dense"),
    ]


_MOST = {"elements": 8 * 4096 * 2048, "products": 8 * 2048 * 2048 * 5504}        # the largest listed cases'


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _size(rng, lo, hi):
    """Half of them any number, half a multiple of 64, or 8."""
    n = _log(rng, lo, hi)
    if rng.random() < 0.5:
        m = 64 if n >= 64 else 8
        n = max(m, n // m * m)
    return n


def draw(rng):
    op = rng.choice(["dropout", "norm", "norm_train", "gated", "gated_train", "gated_train"])
    c = dict(op=op, K=_log(rng, 1, 16), storage=rng.choice(["f32", "bf16", "bf16"]), layout=rng.choice(["dense", "dense", "padded", "turned"]))
    if op in ("gated", "gated_train"):
        c["act"] = rng.choice(ACTS)
        c["cols"], c["wide"] = _size(rng, 16, 4096), _size(rng, 16, 8192)
        c["rows"] = _size(rng, 1, 4096) if rng.random() < 0.7 else rng.randint(1, 16)
        most = _MOST["products"] // (1 if c["storage"] == "bf16" else 8)
        while c["K"] * c["rows"] * c["cols"] * c["wide"] > most:
            c["rows"], c["K"] = max(1, c["rows"] * 2 // 3), max(1, c["K"] - 1)
    else:
        c["cols"] = _size(rng, 8, 16384)
        c["rows"] = _size(rng, 1, 8192) if rng.random() < 0.8 else rng.randint(1, 8)
        while c["K"] * c["rows"] * c["cols"] > _MOST["elements"]:
            c["rows"], c["K"] = max(1, c["rows"] * 2 // 3), max(1, c["K"] - 1)
        if op != "norm":
            c["p"] = rng.choice([0.0, 0.1, 0.1, 0.5, round(rng.uniform(0.01, 0.9), 3)]) if op == "norm_train" else rng.choice([0.1, 0.2, 0.5])
        else:
            c["out8"] = rng.random() < 0.4
    if rng.random() < 0.4:
        c["ragged"] = rng.randrange(1 << 20)
    return c


def _rows(c):
    if "ragged" not in c:
        return [c["rows"]] * c["K"]
    r = random.Random(int(c["ragged"]))
    rows = [r.randint(0, c["rows"]) for _ in range(c["K"])]
    rows[r.randrange(c["K"])] = c["rows"]
    return rows


def _dtype(c):
    return torch.bfloat16 if c["storage"] == "bf16" else torch.float32


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _empty(c, cols, dtype):
    """[K, rows, cols], zeros, in the case's layout."""
    K, R = c["K"], c["rows"]
    if c["layout"] == "turned":
        return torch.zeros(R, K, cols, dtype=dtype, device=DEV).transpose(0, 1)
    if c["layout"] == "padded":
        return torch.zeros(K, R, cols + 24, dtype=dtype, device=DEV)[:, :, :cols]
    return torch.zeros(K, R, cols, dtype=dtype, device=DEV)


def _grads(c, *shape):
    """A bound gradient of every replica: a tensor of its own that starts on 16 bytes."""
    n = math.prod(shape)
    return torch.zeros(c["K"], (n + 7) // 8 * 8, dtype=_dtype(c), device=DEV)[:, :n].view(c["K"], *shape)


def _inputs(c, seed):
    """Activations with a few columns of far larger values, as trained models have them; weights of unit gain; small gradients."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    dt, K, R, D = _dtype(c), c["K"], c["rows"], c["cols"]
    out = {}

    def rows(name, cols, scale, loud=False):
        v = torch.randn(K, R, cols, generator=gen, device=DEV) * scale
        if loud:
            v[:, :, :: max(1, cols // 6)] *= 12.0
        out[name] = _empty(c, cols, dt)
        out[name].copy_(v)

    def weight(name, *shape, scale, plus=0.0):
        n = math.prod(shape)
        out[name] = _grads(c, *shape)                                      # where a bound tensor may start, its gradient may
        out[name].copy_((torch.randn(K, n, generator=gen, device=DEV) * scale + plus).view(K, *shape))

    if c["op"] in ("gated", "gated_train"):
        H = c["wide"]
        rows("x", D, 1.0)
        weight("gate", H, D, scale=D ** -0.5)
        weight("up", H, D, scale=D ** -0.5)
        if c["op"] == "gated_train":
            rows("da", H, 0.02)
        return out
    rows("x", D, 1.0)
    rows("residual", D, 2.0, loud=True)
    if c["op"] != "norm":
        rows("dy", D, 0.02)
    if c["op"] != "dropout":
        weight("gain", D, scale=0.2, plus=1.0)
    if c["op"] == "norm_train":
        rows("dsum", D, 0.02)
    return out


def _lots(seed):
    """(key, call number) of a pass's masks."""
    r = random.Random(int(seed) * 2 + 1)
    return r.getrandbits(64), r.getrandbits(40)


class _State:
    pass


def prepare(case, seed):
    c, st = case, _State()
    st.c, st.rows = c, _rows(case)
    st.t = _inputs(c, seed)
    st.key, st.call = _lots(seed)
    dt, D, op = _dtype(c), c["cols"], c["op"]
    st.out = {}
    if op == "dropout":
        st.out.update(y=_empty(c, D, dt), dx=_empty(c, D, dt))
    elif op in ("norm", "norm_train"):
        st.out.update(sum=_empty(c, D, dt))
        if not c.get("out8"):
            st.out.update(y=_empty(c, D, dt))
        if op == "norm_train":
            st.out.update(dx=_empty(c, D, dt), dresidual=_empty(c, D, dt), dgain=_grads(c, D))
    else:
        st.out.update(a=_empty(c, c["wide"], dt))
        if op == "gated_train":
            st.out.update(dx=_empty(c, D, dt))
            st.out.update(dgate=_grads(c, c["wide"], D), dup=_grads(c, c["wide"], D))
    if c.get("out8"):
        st.q = torch.zeros(c["K"], c["rows"], D, dtype=torch.uint8, device=DEV)
        st.scales = torch.zeros(c["K"], c["rows"], device=DEV)
    if not own:
        return st
    from paper_2203_13085_amd import binding as B
    st.B = B
    names = ("gate", "up") if op.startswith("gated") else ("gain",) if op.startswith("norm") else ()
    esize = 2 if c["storage"] == "bf16" else 4
    torch.cuda.synchronize()
    st.ctx = B.Context(c["K"], [st.t[n][0].numel() for n in names] or [8], storage=B.BF16 if esize == 2 else B.F32,
                       main_stream=torch.cuda.current_stream().cuda_stream)
    st.spare = torch.zeros(16, dtype=dt, device=DEV)
    grads = [st.out["d" + n] if "d" + n in st.out else st.t[n] for n in names]              # no gradients: nothing writes there
    for k in range(c["K"]):
        if names:
            st.ctx.bind(k, [st.t[n][k].data_ptr() for n in names], [g[k].data_ptr() for g in grads])
        else:
            st.ctx.bind(k, [st.spare.data_ptr()], [st.spare.data_ptr()])
    if op == "norm_train":
        st.bytes = st.ctx.rms_norm_backward_bytes(0, st.rows)
    if op == "gated_train":
        st.g, st.u = _empty(c, c["wide"], dt), _empty(c, c["wide"], dt)
        st.bytes = st.ctx.gated_backward_bytes(0, 1, st.rows, D)
    if op.endswith("_train"):
        st.work = torch.zeros(max(16, st.bytes), dtype=torch.uint8, device=DEV)
    return st


# ---- one pass ----------------------------------------------------------------------------------------------------------
def run(state):
    return _calls(state) if own else _plain(state)


def _at(t):
    return t.data_ptr(), t.stride(0), t.stride(1)


def _calls(st):
    c, ctx, t, o, rows = st.c, st.ctx, st.t, st.out, st.rows
    op, s = c["op"], torch.cuda.current_stream().cuda_stream
    if op == "dropout":
        ctx.dropout(rows, c["cols"], _at(t["x"]), _at(o["y"]), c["p"], residual=_at(t["residual"]), seed=st.key, call=st.call, stream=s)
        ctx.dropout(rows, c["cols"], _at(t["dy"]), _at(o["dx"]), c["p"], seed=st.key, call=st.call, stream=s)
        return dict(o)
    if op == "norm":
        if not c.get("out8"):
            ctx.rms_norm(0, rows, _at(t["x"]), _at(o["y"]), residual=_at(t["residual"]), sum=_at(o["sum"]), eps=EPS, stream=s)
            return dict(o)
        ctx.rms_norm(0, rows, _at(t["x"]), _at(st.q), residual=_at(t["residual"]), sum=_at(o["sum"]),
                     scales=(st.scales.data_ptr(), st.scales.stride(0), 1), eps=EPS, stream=s)
        return {"sum": o["sum"], "y": st.q.view(torch.float8_e4m3fn).float() * st.scales[:, :, None]}
    if op == "norm_train":
        drop = dict(p=c["p"], seed=st.key, call=st.call)
        ctx.rms_norm(0, rows, _at(t["x"]), _at(o["y"]), residual=_at(t["residual"]), sum=_at(o["sum"]), eps=EPS, stream=s, **drop)
        ctx.rms_norm_backward(0, rows, _at(o["sum"]), _at(t["dy"]), _at(o["dx"]), dsum=_at(t["dsum"]), dresidual=_at(o["dresidual"]),
                              eps=EPS, accumulate=False, workspace=st.work.data_ptr(), workspace_bytes=st.bytes, stream=s, **drop)
        return dict(o)
    act = getattr(st.B, c["act"].upper())
    if op == "gated":
        ctx.gated(0, 1, rows, c["cols"], _at(t["x"]), _at(o["a"]), activation=act, stream=s)
        return dict(o)
    ctx.gated(0, 1, rows, c["cols"], _at(t["x"]), _at(o["a"]), g=_at(st.g), u=_at(st.u), activation=act, stream=s)
    ctx.gated_backward(0, 1, rows, c["cols"], _at(t["x"]), _at(st.g), _at(st.u), _at(t["da"]), _at(o["dx"]), activation=act,
                       accumulate=False, workspace=st.work.data_ptr(), workspace_bytes=st.bytes, stream=s)
    return dict(o)


def _low_high(a, m):
    """The two halves of 32-bit a times 32-bit m, held in 64."""
    p = a * m
    return p & 0xFFFFFFFF, (p >> 32) & 0xFFFFFFFF


def _kept(st, k, rows, cols, p):
    """[rows, cols]: true where the mask leaves an element. Eight columns share a draw of Philox 4x32 (ten rounds; Salmon et al.,
    SC 2011): counter (group, replica, call number), key; each takes 16 bits and stays if they are not below p 2^16."""
    groups = (cols + 7) // 8
    i = torch.arange(rows * groups, dtype=torch.int64, device=DEV)
    c0, c1 = i & 0xFFFFFFFF, (i >> 32) | (k << 16)
    c2, c3 = torch.full_like(i, st.call & 0xFFFFFFFF), torch.full_like(i, st.call >> 32)
    k0, k1 = st.key & 0xFFFFFFFF, st.key >> 32
    for _ in range(10):
        l0, h0 = _low_high(c0, 0xD2511F53)
        l1, h1 = _low_high(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    lots = torch.stack([v for w in (c0, c1, c2, c3) for v in (w & 0xFFFF, w >> 16)], dim=1)
    return (lots >= round(p * 65536)).view(rows, groups * 8)[:, :cols]


def _dropped(st, k, rows, v):
    p = st.c.get("p", 0.0)
    if not p:
        return v
    return torch.where(_kept(st, k, rows, v.shape[1], p), v * (1.0 / (1.0 - round(p * 65536) / 65536)), 0.0)


def _act(name, v):
    """The activation and its slope."""
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-v))
        return v * s, s * (1.0 + v * (1.0 - s))
    if name == "relu":
        return torch.where(v > 0, v, 0.0), (v > 0).to(v.dtype)
    if name == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(v * math.sqrt(0.5)))
        return v * cdf, cdf + v * torch.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi)
    b = math.sqrt(2.0 / math.pi)
    t = torch.tanh(b * (v + 0.044715 * v * v * v))
    return 0.5 * v * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * v * (1.0 - t * t) * b * (1.0 + 3 * 0.044715 * v * v)


def _plain(st):
    c, t, o = st.c, st.t, dict(st.out)
    op = c["op"]
    if c.get("out8"):
        o["y"] = torch.zeros(c["K"], c["rows"], c["cols"], device=DEV)
    for k, n in enumerate(st.rows):
        if op == "dropout":
            o["y"][k, :n] = (t["residual"][k, :n].float() + _dropped(st, k, n, t["x"][k, :n].float())).to(_dtype(c))
            o["dx"][k, :n] = _dropped(st, k, n, t["dy"][k, :n].float()).to(_dtype(c))
        elif op in ("norm", "norm_train"):
            h = t["residual"][k, :n].float() + _dropped(st, k, n, t["x"][k, :n].float())
            gain = t["gain"][k].float()
            r = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
            y = gain * (h * r)
            o["sum"][k, :n] = h.to(_dtype(c))
            if c.get("out8"):
                y = gain.double() * (h.double() / torch.sqrt((h.double() ** 2).mean(1, keepdim=True) + EPS))
                scale = y.abs().amax(1, keepdim=True) / E4M3_MAX
                q = torch.where(scale > 0, y / scale, 0.0).float().to(torch.float8_e4m3fn)
                o["y"][k, :n] = q.float() * scale.float()
                continue
            o["y"][k, :n] = y.to(_dtype(c))
            if op == "norm_train":
                dy, hat = t["dy"][k, :n].float(), h * r
                wdy = gain * dy
                dh = r * (wdy - hat * (hat * wdy).mean(1, keepdim=True)) + t["dsum"][k, :n].float()
                o["dresidual"][k, :n] = dh.to(_dtype(c))
                o["dx"][k, :n] = _dropped(st, k, n, dh).to(_dtype(c))
                o["dgain"][k] = (dy * hat).sum(0).to(_dtype(c))
        else:
            x, gate, up = t["x"][k, :n].float(), t["gate"][k].float(), t["up"][k].float()
            g, u = x @ gate.T, x @ up.T
            f, slope = _act(c["act"], g)
            o["a"][k, :n] = (f * u).to(_dtype(c))
            if op == "gated_train":
                da = t["da"][k, :n].float()
                dg, du = da * u * slope, da * f
                o["dx"][k, :n] = (dg @ gate + du @ up).to(_dtype(c))
                o["dgate"][k] = (dg.T @ x).to(_dtype(c))
                o["dup"][k] = (du.T @ x).to(_dtype(c))
    return o


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------
def work(case):
    """Inputs once and outputs once. A norm with an 8-bit output writes a byte an element and four a row (and, read as the values
    that stand for, no more than that); g and u of a gated block are the framework's own to keep or to make again."""
    c, e, D = case, 2.0 if case["storage"] == "bf16" else 4.0, float(case["cols"])
    n = float(sum(_rows(c)))
    if c["op"] == "dropout":
        return {"bytes": 5.0 * e * n * D, "flops": 5.0 * n * D}
    if c["op"] == "norm":
        return {"bytes": 3.0 * e * n * D + (1.0 * n * D + 4.0 * n if c.get("out8") else e * n * D) + e * c["K"] * D, "flops": 5.0 * n * D}
    if c["op"] == "norm_train":
        return {"bytes": 8.0 * e * n * D + 2.0 * e * c["K"] * D, "flops": 17.0 * n * D}
    H, K = float(c["wide"]), c["K"]
    if c["op"] == "gated":
        return {"bytes": e * (n * (D + H) + 2.0 * K * H * D), "flops": 4.0 * n * H * D}
    return {"bytes": e * (n * (2.0 * D + 2.0 * H) + 4.0 * K * H * D), "flops": 12.0 * n * H * D}


# ---- the same in 64 bits ------------------------------------------------------------------------------------------------------
def _philox(i, k, call, key):
    """Philox 4x32 with ten rounds on whole arrays of counters: words [n, 4]."""
    w = [(i & np.uint64(0xFFFFFFFF)), (i >> np.uint64(32)) | np.uint64(k << 16), np.full_like(i, call & 0xFFFFFFFF), np.full_like(i, call >> 32)]
    a, b = key & 0xFFFFFFFF, key >> 32
    for turn in range(10):
        p, q = w[0] * np.uint64(0xD2511F53), w[2] * np.uint64(0xCD9E8D57)
        ka, kb = (a + turn * 0x9E3779B9) & 0xFFFFFFFF, (b + turn * 0xBB67AE85) & 0xFFFFFFFF
        w = [(q >> np.uint64(32)) ^ w[1] ^ np.uint64(ka), q & np.uint64(0xFFFFFFFF), (p >> np.uint64(32)) ^ w[3] ^ np.uint64(kb), p & np.uint64(0xFFFFFFFF)]
    return np.stack(w, axis=1)


def exact(case, seed):
    """One pass, replica by replica, from the definition. (8-bit values: the ones next to the exact quotient in the same row scale.)"""
    c, D, op = case, case["cols"], case["op"]
    t, rows = _inputs(c, seed), _rows(c)
    key, call = _lots(seed)
    zeros = lambda cols: torch.zeros(c["K"], c["rows"], cols, dtype=torch.float64, device=DEV)  # noqa: E731

    def factor(k, n):
        """What a row's elements count times: 0 or 1 / (1 - p)."""
        below = round(c.get("p", 0.0) * 65536)
        if not below or not n:
            return torch.ones(n, D, dtype=torch.float64, device=DEV)
        groups = -(-D // 8)
        words = _philox(np.arange(n * groups, dtype=np.uint64), k, call, key).astype(np.uint32)
        lots = words.view(np.uint16).reshape(n, groups * 8)[:, :D]                       # little end first
        return torch.from_numpy(lots >= below).to(DEV).double() * (65536.0 / (65536 - below))

    if op == "dropout":
        y, dx = zeros(D), zeros(D)
        for k, n in enumerate(rows):
            m = factor(k, n)
            y[k, :n] = t["residual"][k, :n].double() + m * t["x"][k, :n].double()
            dx[k, :n] = m * t["dy"][k, :n].double()
        return {"y": y, "dx": dx}
    if op in ("norm", "norm_train"):
        out = {n: zeros(D) for n in (("sum", "y", "dx", "dresidual") if op == "norm_train" else ("sum", "y"))}
        if op == "norm_train":
            out["dgain"] = torch.zeros(c["K"], D, dtype=torch.float64, device=DEV)
        for k, n in enumerate(rows):
            m, w = factor(k, n), t["gain"][k].double()
            h = t["residual"][k, :n].double() + m * t["x"][k, :n].double()
            length = torch.sqrt(h.pow(2).sum(1) / D + EPS)[:, None]
            y = h / length * w
            out["sum"][k, :n] = h
            out["y"][k, :n] = y
            if c.get("out8") and n:
                step = y.abs().max(dim=1, keepdim=True).values / E4M3_MAX
                out["y"][k, :n] = (y / step).float().to(torch.float8_e4m3fn).double() * step
            if op == "norm_train":
                dy = t["dy"][k, :n].double()
                along = (dy * w * h).sum(1, keepdim=True) / (D * length.pow(3))
                dh = dy * w / length - h * along + t["dsum"][k, :n].double()
                out["dresidual"][k, :n] = dh
                out["dx"][k, :n] = dh * m
                out["dgain"][k] = (dy * h / length).sum(0)
        return out
    if 12.0 * sum(rows) * D * c["wide"] > 1.0e14:
        return None
    out = {"a": zeros(c["wide"])}
    if op == "gated_train":
        out.update(dx=zeros(D), dgate=torch.zeros(t["gate"].shape, dtype=torch.float64, device=DEV), dup=torch.zeros(t["up"].shape, dtype=torch.float64, device=DEV))
    for k, n in enumerate(rows):
        x, gate, up = t["x"][k, :n].double(), t["gate"][k].double(), t["up"][k].double()
        g, u = torch.mm(x, gate.t()), torch.mm(x, up.t())
        if c["act"] == "silu":
            s = torch.sigmoid(g)
            f, slope = g * s, s + g * s * torch.sigmoid(-g)
        elif c["act"] == "relu":
            f, slope = g.clamp(min=0.0), (g > 0.0).double()
        elif c["act"] == "gelu":
            f = g * torch.special.ndtr(g)
            slope = torch.special.ndtr(g) + g * torch.exp(-g * g / 2) * 0.3989422804014327
        else:
            e = torch.exp(-2.0 * 0.7978845608028654 * (g + 0.044715 * g ** 3))           # tanh(v) + 1 = 2 / (1 + exp(-2 v))
            s = 1.0 / (1.0 + e)
            f, slope = g * s, s + 2.0 * g * s * (1.0 - s) * 0.7978845608028654 * (1.0 + 0.134145 * g ** 2)
        out["a"][k, :n] = f * u
        if op == "gated_train":
            da = t["da"][k, :n].double()
            dg, du = da * u * slope, da * f
            out["dx"][k, :n] = torch.mm(dg, gate) + torch.mm(du, up)
            out["dgate"][k] = torch.mm(dg.t(), x)
            out["dup"][k] = torch.mm(du.t(), x)
    return out
