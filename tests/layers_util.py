"""What the tests of the layers' operators share: contexts with bound weights, activations in every layout with canaries around
them, the mask from its definition, and the operators in 64 bits."""
import math

import numpy as np
import torch

from paper_2203_13085_amd import binding as B

DEV = "cuda:0"
U = 2.0 ** -24                                      # half a step of fp32, relative
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # torch.finfo(t).eps / 2
CANARY = 77.0


def dtype_of(storage):
    return torch.bfloat16 if storage == "bf16" else torch.float32


# ---- the mask, in Python's integers -----------------------------------------------------------------------------------
def philox(counter, key):
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def mask_of(k, rows, cols, p, seed, n):
    """bool [rows, cols]: true where an element stays."""
    groups, below = (cols + 7) // 8, round(p * 65536)
    i = np.arange(rows * groups, dtype=object)
    c = [i & 0xFFFFFFFF, (i >> 32) | (k << 16), i * 0 + (n & 0xFFFFFFFF), i * 0 + (n >> 32)]
    w = philox(c, [seed & 0xFFFFFFFF, seed >> 32])
    lots = np.stack([h for a in w for h in (a & 0xFFFF, a >> 16)], axis=1).astype(np.int64)
    return torch.from_numpy((lots >= below).reshape(rows, groups * 8)[:, :cols].copy())


def scale_of(p):
    below = round(p * 65536)
    return 65536.0 / (65536 - below) if below < 65536 else 0.0


# ---- activations --------------------------------------------------------------------------------------------------------
class Act:
    """[K, most, cols] in a layout, in a buffer full of canaries; rows beyond rows[k] hold them too."""

    def __init__(self, rows, cols, dtype, layout="dense", gen=None, scale=1.0):
        K, R = len(rows), max(max(rows), 1)
        self.rows, self.cols = rows, cols
        lead = {"dense": 0, "padded": 16, "turned": 0, "odd": 1}[layout]
        pitch = {"dense": cols, "padded": cols + 24, "turned": cols, "odd": cols + 3}[layout]
        self.buf = torch.full((lead + K * R * pitch + 64,), CANARY, device=DEV, dtype=torch.float32).to(dtype)
        if layout == "turned":
            self.t = self.buf[: R * K * cols].view(R, K, cols).transpose(0, 1)
        else:
            self.t = self.buf[lead: lead + K * R * pitch].view(K, R, pitch)[:, :, :cols]
        if gen is not None:
            for k, n in enumerate(rows):
                self.t[k, :n] = (torch.randn(n, cols, generator=gen, device=DEV) * scale).to(dtype)

    @property
    def at(self):
        return self.t.data_ptr(), self.t.stride(0), self.t.stride(1)

    def __getitem__(self, k):
        return self.t[k, : self.rows[k]]

    def d(self, k):
        return self[k].double()

    def untouched_outside(self):
        """Everything but the replicas' rows still holds canaries."""
        mine = torch.zeros_like(self.buf, dtype=torch.bool)
        v = mine.as_strided(self.t.shape, self.t.stride(), self.t.storage_offset())
        for k, n in enumerate(self.rows):
            v[k, :n] = True
        return bool((self.buf.float()[~mine] == CANARY).all())


class Model:
    """A context with weights and gradients of given shapes bound, each replica's its own."""

    def __init__(self, K, shapes, storage, gen, scales=None, plus=0.0, bind=True):
        self.K, self.dt = K, dtype_of(storage)
        self.numels = [math.prod(s) for s in shapes]
        self.ctx = B.Context(K, self.numels, storage=B.BF16 if storage == "bf16" else B.F32, main_stream=torch.cuda.current_stream().cuda_stream)
        self.w, self.g = [], []
        for i, s in enumerate(shapes):
            n = math.prod(s)
            pad = (n + 7) // 8 * 8 + 8
            w = torch.full((K, pad), CANARY, device=DEV).to(self.dt)
            w[:, :n] = (torch.randn(K, n, generator=gen, device=DEV) * (scales[i] if scales else 1.0) + plus).to(self.dt)
            g = torch.full((K, pad), CANARY, device=DEV).to(self.dt)
            g[:, :n] = (torch.randn(K, n, generator=gen, device=DEV) * 0.1).to(self.dt)
            self.w.append((w, w[:, :n].view(K, *s)))
            self.g.append((g, g[:, :n].view(K, *s)))
        if bind:
            for k in range(K):
                self.ctx.bind(k, [w[k].data_ptr() for w, _ in self.w], [g[k].data_ptr() for g, _ in self.g])

    def weight(self, i, k):
        return self.w[i][1][k]

    def grad(self, i, k):
        return self.g[i][1][k]

    def gaps_untouched(self):
        return all(bool((b.float()[:, n:] == CANARY).all()) for (b, _), n in zip(self.w + self.g, self.numels * 2))

    def close(self):
        torch.cuda.synchronize()
        self.ctx.close()


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def workspace(nbytes):
    """A workspace with canaries behind it."""
    w = torch.full((nbytes + 256,), 0xA5, dtype=torch.uint8, device=DEV)
    return w


def workspace_kept(w, nbytes):
    return bool((w[nbytes:] == 0xA5).all())


def within(got, want, bound, what=""):
    """|got - want| <= bound, element by element, all of them numbers."""
    got = got.double()
    bad = ~((got - want).abs() <= bound)
    if bool(bad.any()):
        i = int(bad.flatten().nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside, first at {i}: got {float(got.flatten()[i])!r}, "
                             f"want {float(want.flatten()[i])!r}, bound {float(bound.flatten()[i]):.3g}")


# ---- activations' functions, 64 bits ------------------------------------------------------------------------------------
ACTS = {"silu": B.SILU, "gelu": B.GELU, "gelu_tanh": B.GELU_TANH, "relu": B.RELU}


def act64(name, v):
    if name == "silu":
        s = torch.sigmoid(v)
        return v * s, s * (1 + v * (1 - s))
    if name == "relu":
        return v.clamp(min=0), (v > 0).double()
    if name == "gelu":
        cdf = 0.5 * torch.special.erfc(-v / math.sqrt(2.0))
        return v * cdf, cdf + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    b = math.sqrt(2 / math.pi)
    t = torch.tanh(b * (v + 0.044715 * v ** 3))
    return 0.5 * v * (1 + t), 0.5 * (1 + t) + 0.5 * v * (1 - t * t) * b * (1 + 3 * 0.044715 * v * v)
