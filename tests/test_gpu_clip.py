"""Gradient norms and clipping against 64-bit sums and, for the clipped updates, the oracle fed with gradients that were scaled on the host.

Tolerances, all from the roundings: a norm is one rounding to fp32 of a 64-bit sum (2^-24, and the sums' own 1e-12), a gradient
scaled in place two more (c and the product; bf16 storage, whose 8 bits round by up to 2^-8).  Everything else is compared to the bit: c is the 64-bit quotient rounded
once, and the updates have the oracle's order of operations."""
import copy
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import lasgd_oracle as O32                     # noqa: E402
from paper_2203_13085_amd import binding as B              # noqa: E402
from paper_2203_13085_amd import workloads as W            # noqa: E402
from tests.parity_util import assert_close                 # noqa: E402

pytestmark = pytest.mark.gpu

EPS = 1e-6
INF = float("inf")


def norm64(g):
    a = g.astype(np.float64)
    return float(np.sqrt(np.dot(a, a)))


def coefficient(n, max_norm):
    """(c as the library holds it)"""
    with np.errstate(invalid="ignore"):
        q = np.float64(np.float32(max_norm)) / (np.float64(n) + EPS)
    return np.float32(1.0) if q >= 1.0 else np.float32(q)


def check_norms(got, want):
    for k, (a, b) in enumerate(zip(got, want)):
        if not np.isfinite(b):
            assert np.isnan(a) == np.isnan(b) and (np.isnan(a) or a == b), (k, a, b)
        else:
            with np.errstate(over="ignore"):
                lim = float(np.float32(b))
            assert a == lim or abs(a - b) <= b * (2.0 ** -24 + 1e-12) + 1e-45, (k, a, b)


class Rig:
    """A context of K replicas, its f32 oracle (bf16 storage is fp32 arithmetic on widened gradients), and gradients in hand."""

    def __init__(self, K, numels, storage="f32", side_stream=True, lead=4096, seed=7, **kw):
        from paper_2203_13085_amd.driver import DeviceReplicas
        self.w = W.small(K=K, numels=numels, storage=storage, seed=seed, **kw)
        self.bf16 = storage == "bf16"
        self.K, self.N = K, self.w.N
        wd = [1e-3 * (t % 3) for t in range(len(numels))]
        x0 = np.concatenate([W.initial_tensor(self.w, t) for t in range(len(numels))])
        bits = W.to_bf16_bits(x0) if self.bf16 else x0
        self.orc = O32.Oracle(K, list(numels), self.w.momentum, self.w.nesterov, wd)
        self.dev = DeviceReplicas(self.w, weight_decay=wd, side_stream=side_stream, grad_lead_bytes=lead)
        self.orc.set_model(W.bf16_bits_to_f32(bits) if self.bf16 else x0)
        self.dev.load_model(bits)
        self.ctx = self.dev.ctx
        self.norms = torch.full((K,), -1.0, device="cuda")
        torch.cuda.synchronize()

    def grads(self, step, scales=None):
        """Replica k's gradients are `scales[k]` times N(0, 1e-3^2); as fp32, exactly what the device gets."""
        scales = scales if scales is not None else [np.exp(np.sin(1.0 + 2.0 * k + step)) for k in range(self.K)]
        out = []
        for k in range(self.K):
            g = np.concatenate([W.gradient_tensor(self.w, step, k, t) for t in range(len(self.w.numels))]) * np.float32(scales[k])
            out.append(W.bf16_bits_to_f32(W.to_bf16_bits(g)) if self.bf16 else g.astype(np.float32))
        return out

    def load(self, g):
        self.dev.load_grads([W.to_bf16_bits(a) for a in g] if self.bf16 else g)

    def device_grads(self, k):
        self.ctx.sync()
        a = self.dev._get(self.dev.g[k])
        return W.bf16_bits_to_f32(a) if self.bf16 else a

    def read_norms(self):
        self.ctx.sync()
        return self.norms.cpu().numpy().astype(np.float64)

    def same(self, what, send=True):
        for k in range(self.K):
            assert_close(self.ctx.read_state(B.STATE_X, k), self.orc.x[k], f"x replica {k} {what}")
            assert_close(self.ctx.read_state(B.STATE_V, k), self.orc.v[k], f"v replica {k} {what}")
            if send:
                assert_close(self.ctx.read_state(B.STATE_S, k), self.orc.s[k], f"s replica {k} {what}")
            if self.bf16:
                np.testing.assert_array_equal(self.dev.params(k), W.to_bf16_bits(self.orc.x[k]), err_msg=f"x16 replica {k} {what}")

    def clipped(self, g, max_norm, members=None):
        """Gradients as a clipped update sees them."""
        return [coefficient(norm64(a), max_norm) * a if members is None or members[k] else a for k, a in enumerate(g)]

    def max_norm(self, g):
        """Between the replicas' norms: some are clipped and some are not (one replica: it is)."""
        n = sorted(norm64(a) for a in g)
        return float(np.float32(0.5 * (n[(len(n) - 1) // 2] + n[len(n) // 2]) if len(n) > 1 else 0.7 * n[0]))

    def close(self):
        self.dev.close()


LISTS = {
    "one": (1,),
    "three": (3,),
    "odd": (5, 1024, 1, 4099, 260, 64),
    "rows": (255, 256, 257, 511, 512, 513, 1, 2, 3, 4),
    "many": tuple(1 + (37 * i) % 300 for i in range(150)),              # several tensors in every block of tiles, more than sixteen in some
    "blocks": (64 * 256, 64 * 256 - 1, 64 * 256 + 1, 5, 3 * 64 * 256 + 77),
    "long": (1_300_001, 3, 70_000),
    "48 tiles": (12_288,),
    "48 of many": (3, 700, 256) + (1,) * 43,
    "49 tiles": (12_289,),
    "64 tiles": (16_384,),
    "64 of one": (1,) * 64,
    "63 and 300": (1,) * 62 + (300,),
    "65 tiles": (16_385,),
    "65 of one": (1,) * 65,
    "128 tiles": (32_768,),
    "127 of many": (300, 1, 20_000, 700) + (1,) * 40 + (257,) + (3,) * 1,
    "129 tiles": (32_769,),
}


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("K", [1, 3, 17, 64])
@pytest.mark.parametrize("name", list(LISTS))
def test_norms(name, K, storage):
    if name == "long" and K > 3:
        pytest.skip("covered by fewer replicas")
    r = Rig(K, LISTS[name], storage)
    try:
        g = r.grads(0)
        r.load(g)
        want = [norm64(a) for a in g]
        r.ctx.grad_norms(r.norms.data_ptr())
        first = r.read_norms()
        check_norms(first, want)
        # a second time: the same bits; and into part of the array only
        part = sum(1 << k for k in range(0, K, 3))
        r.norms.fill_(-1.0)
        torch.cuda.synchronize()
        r.ctx.grad_norms(r.norms.data_ptr(), part)
        again = r.read_norms()
        for k in range(K):
            assert again[k] == (first[k] if (part >> k) & 1 else -1.0)
    finally:
        r.close()


def test_norms_of_a_long_list_over_many_replicas():
    """More tiles than workgroups, and the last replica of sixty-four."""
    r = Rig(64, (200_003, 1, 33), "bf16")
    try:
        g = r.grads(1)
        r.load(g)
        r.ctx.grad_norms(r.norms.data_ptr())
        check_norms(r.read_norms(), [norm64(a) for a in g])
    finally:
        r.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("value", [0.0, 1e-30, 1e-42, 1e30, 3e38])
def test_norms_of_values_whose_squares_leave_fp32(value, storage):
    r = Rig(2, LISTS["odd"], storage)
    try:
        n = r.N
        g = [np.full(n, value, dtype=np.float32), np.zeros(n, dtype=np.float32)]
        g[1][n // 2] = -value
        g = [W.bf16_bits_to_f32(W.to_bf16_bits(a)) for a in g]           # the same values in both storages
        r.load(g)
        want = [norm64(a) for a in g]
        r.ctx.grad_norms(r.norms.data_ptr())
        check_norms(r.read_norms(), want)
        # a norm beyond fp32 is not an infinity among the gradients: it is clipped, not skipped
        r.ctx.clip_grads(1.0, skip_nonfinite=True)
        for k in range(2):
            scaled = coefficient(want[k], 1.0) * g[k]
            np.testing.assert_array_equal(r.device_grads(k), W.bf16_bits_to_f32(W.to_bf16_bits(scaled)) if r.bf16 else scaled)
    finally:
        r.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("name,K", [("one", 1), ("odd", 3), ("rows", 5), ("many", 4), ("blocks", 3), ("long", 2), ("odd", 64),
                                    ("64 tiles", 5), ("64 of one", 3), ("63 and 300", 9), ("65 tiles", 4), ("65 of one", 3), ("65 of one", 64)])
def test_clip_in_place(name, K, storage):
    r = Rig(K, LISTS[name], storage)
    try:
        for step in range(2):
            g = r.grads(step)
            r.load(g)
            members = [k % 4 != 1 or K == 1 for k in range(K)]
            mask = sum(1 << k for k in range(K) if members[k])
            most = r.max_norm(g)
            whole = [t.clone() for t in r.dev._g_alloc]
            r.norms.fill_(-1.0)
            torch.cuda.synchronize()
            r.ctx.clip_grads(most, mask, norms=r.norms.data_ptr())
            norms = r.read_norms()
            for k in range(K):
                if not members[k]:
                    assert norms[k] == -1.0
                    np.testing.assert_array_equal(r.device_grads(k), g[k])
                    continue
                n = norm64(g[k])
                check_norms(norms[k:k + 1], [n])
                scaled = coefficient(n, most) * g[k]
                if r.bf16:
                    scaled = W.bf16_bits_to_f32(W.to_bf16_bits(scaled))
                np.testing.assert_array_equal(r.device_grads(k), scaled)
                exact = min(1.0, most / (n + EPS)) * g[k].astype(np.float64)
                assert np.all(np.abs(scaled - exact) <= np.abs(exact) * ((2.0 ** -8 if r.bf16 else 0.0) + 2.0 ** -22) + 1e-40)
                # the gaps between the tensors and what lies around them stay as they were
                lead = r.dev._g_alloc[k].numel() - r.dev.g[k].numel()
                touched = torch.zeros(whole[k].numel(), dtype=torch.bool, device="cuda")
                touched[lead + r.dev._idx] = True
                assert torch.equal(r.dev._g_alloc[k][~touched], whole[k][~touched])
    finally:
        r.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_gradients_that_need_no_clipping_keep_every_bit(storage):
    """c = 1: also minus zeros and denormals; the model and the state are not touched by either call."""
    r = Rig(3, LISTS["odd"], storage)
    try:
        g = r.grads(0)
        g[0][:3] = [-0.0, 1e-40, -1e-40]
        g[2][:] = 0.0                                           # a norm of zero
        r.load(g)
        before = [t.clone() for t in r.dev.g]
        r.ctx.clip_grads(1e3)
        r.ctx.clip_grads(INF, norms=r.norms.data_ptr())
        r.ctx.sync()
        view = torch.int16 if r.bf16 else torch.int32
        assert all(torch.equal(a.view(view), b.view(view)) for a, b in zip(before, r.dev.g))
        assert r.read_norms()[2] == 0.0
        r.same("")
    finally:
        r.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [INF, -INF, float("nan")])
@pytest.mark.parametrize("place", [0, -1, 1030])
def test_what_is_not_finite(bad, place, storage):
    """In the first element, in the last one of an odd tail, inside a tensor."""
    r = Rig(3, LISTS["odd"], storage)
    try:
        g = r.grads(0)
        g[1][place] = bad
        most = r.max_norm([g[0], g[2]])
        r.load(g)
        r.ctx.clip_grads(most, skip_nonfinite=True, norms=r.norms.data_ptr())
        norms = r.read_norms()
        check_norms(norms, [norm64(g[0]), abs(bad), norm64(g[2])])
        np.testing.assert_array_equal(r.device_grads(1), g[1])                         # left as they are
        for k in (0, 2):
            want = coefficient(norm64(g[k]), most) * g[k]
            np.testing.assert_array_equal(r.device_grads(k), W.bf16_bits_to_f32(W.to_bf16_bits(want)) if r.bf16 else want)
        # a step: replica 1 sits out
        r.load(g)
        r.ctx.local_step_clip(r.w.lr, most, skip_nonfinite=True)
        r.orc.local_step(r.clipped(g, most, [True, False, True]), [r.w.lr] * 3, mask=0b101)
        r.same("after a step that one replica sits out", send=False)
        # without skip_nonfinite: the formula as it stands
        r.ctx.clip_grads(most)
        with np.errstate(invalid="ignore"):
            want = coefficient(INF if np.isinf(bad) else np.nan, most) * g[1]
        np.testing.assert_array_equal(r.device_grads(1), want)
    finally:
        r.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("name,K,tuning", [("one", 1, {}), ("odd", 3, {}), ("rows", 5, dict(nontemporal=3)), ("many", 4, {}), ("blocks", 3, dict(nontemporal=3)),
                                           ("long", 2, dict(nontemporal=3)), ("odd", 64, {}), ("odd", 64, dict(nontemporal=3)),
                                           ("odd", 6, dict(vec=4, kper_step=2, waves_per_block=4, max_blocks=3)), ("odd", 6, dict(vec=2, waves_per_block=2)),
                                           ("long", 3, {}), ("64 tiles", 5, {}), ("64 tiles", 64, dict(vec=4)), ("64 of one", 3, {}),
                                           ("63 and 300", 9, dict(nontemporal=3)), ("128 tiles", 5, {}), ("128 tiles", 64, {}), ("128 tiles", 62, dict(vec=2)), ("127 of many", 9, {}), ("129 tiles", 5, {}), ("48 tiles", 6, dict(vec=4)), ("48 of many", 64, {}), ("49 tiles", 4, dict(vec=2)), ("65 tiles", 4, dict(vec=2)), ("65 of one", 7, {}), ("65 of one", 64, dict(kper_step=5))])
def test_local_steps(name, K, tuning, storage):
    r = Rig(K, LISTS[name], storage)
    try:
        if tuning:
            r.ctx.set_tuning(**tuning)
        for step in range(3):
            g = r.grads(step)
            r.load(g)
            most = r.max_norm(g)
            members = [(k + step) % 3 != 1 or K == 1 for k in range(K)]
            mask = sum(1 << k for k in range(K) if members[k])
            lrs = [r.w.lr * (1.0 - 0.01 * k) for k in range(K)]
            if step == 2:                                       # all of them, one step size
                mask, members, lrs = None, [True] * K, r.w.lr
            r.ctx.local_step_clip(lrs, most, mask, norms=r.norms.data_ptr())
            r.orc.local_step(r.clipped(g, most), lrs if step < 2 else [lrs] * K, mask=mask)
            r.same(f"step {step}", send=False)
            norms = r.read_norms()
            check_norms([norms[k] for k in range(K) if members[k]], [norm64(g[k]) for k in range(K) if members[k]])
            for k in range(K):                                  # only read
                np.testing.assert_array_equal(r.device_grads(k), g[k])
        r.ctx.local_step_clip(r.w.lr, most, 0)                  # nobody steps
        r.same("after an empty call", send=False)
    finally:
        r.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("K,numels,tuning,side", [(3, LISTS["odd"], {}, True), (5, LISTS["rows"], dict(nontemporal=3), True), (2, LISTS["long"], {}, True),
                                                  (4, LISTS["many"], {}, False), (4, (700_001, 3, 256), {}, True), (4, (700_001, 3, 256), dict(nontemporal=3), True),
                                                  (6, LISTS["odd"], dict(kper_merge=6, waves_per_block=2, vec=2), True), (5, LISTS["63 and 300"], {}, True),
                                                  (64, LISTS["128 tiles"], {}, True), (62, LISTS["128 tiles"], {}, False), (64, LISTS["64 tiles"], {}, True), (9, LISTS["127 of many"], {}, True), (7, LISTS["48 tiles"], dict(vec=4), True), (6, LISTS["48 of many"], {}, True), (7, LISTS["64 tiles"], dict(vec=4), True), (7, LISTS["65 of one"], dict(vec=4, kper_merge=3), True), (4, LISTS["65 tiles"], {}, False)])
def test_global_updates(K, numels, tuning, side, storage):
    """Steps and updates in turn; masks of the step, of the update, and a replica that is not finite and takes the update all the same.
    The lists with 700,001 elements hold a bf16 model in one place after an update."""
    r = Rig(K, numels, storage, side_stream=side)
    full = (1 << K) - 1
    try:
        if tuning:
            r.ctx.set_tuning(**tuning)
        for o in (r.orc, r.ctx):
            o.snapshot()
        for step in range(6):
            for o in (r.orc, r.ctx):
                o.average()
            g = r.grads(step)
            bad = step % K if step in (2, 3) else None
            most = r.max_norm(g)
            use = r.clipped(g, most)
            if bad is not None:
                g[bad][step] = INF
            r.load(g)
            steppers = full if step in (0, 2, 5) else full & 0x2D
            live = steppers & ~(1 << bad) if bad is not None else steppers
            lrs = [r.w.lr * (1.0 + 0.02 * k) for k in range(K)]
            if step % 2:                                         # a clipped local step in between
                r.ctx.local_step_clip(lrs, most, steppers, skip_nonfinite=True)
                r.orc.local_step(use, lrs, mask=live)
            resnap = step != 4
            r.ctx.step_merge_clip(lrs, most, steppers, full, resnap, skip_nonfinite=True, norms=r.norms.data_ptr())
            r.orc.local_step(use, lrs, mask=live)
            r.orc.merge(resnap)
            r.same(f"update {step}")
            if not resnap:
                for o in (r.orc, r.ctx):
                    o.snapshot()
        # a partial mean, its participants' update, nobody steps
        half = full & 0x35
        for o in (r.orc, r.ctx):
            o.average_ex(half) if o is r.ctx else o.average(mask=half)
        r.ctx.step_merge_clip(r.w.lr, 1.0, 0, half)
        r.orc.merge(True, mask=half)
        r.same("a partial update without a step")
    finally:
        r.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("K,numels", [(4, LISTS["odd"]), (5, (700_001, 3, 256)), (13, (161_515, 64))])
def test_no_limit_is_the_unclipped_call_to_the_bit(K, numels, storage):
    """max_norm = infinity next to the plain calls, on a context of its own; elastic coefficients among them."""
    a, b = Rig(K, numels, storage), Rig(K, numels, storage)
    full = (1 << K) - 1
    try:
        for c in (a.ctx, b.ctx):
            c.snapshot()
        for step in range(4):
            g = a.grads(step)
            for r in (a, b):
                r.load(g)
                r.ctx.average()
                if step == 2:
                    r.ctx.set_elastic(0.5, 0.75)
            lrs = [0.05 * (1.0 + 0.1 * k) for k in range(K)]
            a.ctx.local_step_clip(lrs, INF)
            b.ctx.local_step_ex(lrs, full)
            a.ctx.step_merge_clip(lrs, INF, full, full, True)
            b.ctx.step_merge_ex(lrs, full, full, True)
            for which in (B.STATE_X, B.STATE_V, B.STATE_S):
                for k in range(K):
                    np.testing.assert_array_equal(a.ctx.read_state(which, k).view(np.uint32), b.ctx.read_state(which, k).view(np.uint32))
        a.ctx.sgd_ar_step_clip(0.05, INF)
        b.ctx.sgd_ar_step(0.05)
        for k in range(K):
            np.testing.assert_array_equal(a.ctx.read_state(B.STATE_X, k).view(np.uint32), b.ctx.read_state(B.STATE_X, k).view(np.uint32))
    finally:
        a.close()
        b.close()


@pytest.mark.parametrize("storage,K,n", [("f32", 9, 3_100_003), ("bf16", 20, 2_800_003)])
def test_more_gradients_than_a_cache_holds(storage, K, n):
    """Plain and masked steps, after updates that leave a bf16 model in one place, and recorded."""
    r = Rig(K, (n, 33, 256), storage, side_stream=False)
    full, part = (1 << K) - 1, ((1 << K) - 1) & 0xFFEB7
    try:
        g = r.grads(0)
        r.load(g)
        most = r.max_norm(g)
        use = r.clipped(g, most)
        lrs = [r.w.lr * (1.0 - 0.01 * k) for k in range(K)]
        for o in (r.orc, r.ctx):
            o.snapshot()
            o.average()
        r.ctx.step_merge_clip(r.w.lr, most, norms=r.norms.data_ptr())
        r.orc.local_step(use, r.w.lr)
        r.orc.merge(True)
        graph = torch.cuda.CUDAGraph()
        r.ctx.sync()
        with torch.cuda.graph(graph, stream=r.dev.main):
            r.ctx.local_step_clip(r.w.lr, most)
        for rep in range(2):
            with torch.cuda.stream(r.dev.main):
                graph.replay()
            r.orc.local_step(use, r.w.lr)
        r.ctx.local_step_clip(lrs, most, part, norms=r.norms.data_ptr())
        r.orc.local_step(use, lrs, mask=part)
        r.same("at the end")
        check_norms(r.read_norms(), [norm64(a) for a in g])
        r.ctx.clip_grads(most, part)
        for k in range(K):
            want = use[k] if (part >> k) & 1 else g[k]
            np.testing.assert_array_equal(r.device_grads(k), W.bf16_bits_to_f32(W.to_bf16_bits(want)) if r.bf16 else want)
    finally:
        r.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_batches(dtype):
    """From 400 MiB of bf16 gradients on steps, and clipping in place, take some replicas at a time; another context takes them one by one,
    in calls too small for that.  Recorded too, with the models in s alone before."""
    bf16 = dtype == torch.bfloat16
    K, n = (7, 36_000_003) if bf16 else (3, 50_000_003)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    st = torch.cuda.Stream()
    x0 = torch.randn(n, generator=gen, device="cuda").to(dtype)
    rows = (n + 255) // 256 * 256
    g = torch.zeros(K, rows, device="cuda", dtype=dtype)
    for k in range(K):
        g[k, :n] = torch.randn(n, generator=gen, device="cuda") * (0.3 + 0.3 * k)
    want = [float(torch.linalg.vector_norm(g[k, :n].double())) for k in range(K)]
    most = float(np.float32(0.5 * (want[0] + want[-1])))
    sides = []
    for _ in range(2):
        x = torch.zeros(K, rows, device="cuda", dtype=dtype)
        x[:, :n] = x0
        c = B.Context(K, [n], storage=B.BF16 if bf16 else B.F32, main_stream=st.cuda_stream, side_stream=st.cuda_stream, wd_scalar=1e-4)
        for k in range(K):
            c.bind(k, [x[k].data_ptr()], [g[k].data_ptr()])
        torch.cuda.synchronize()
        if bf16:
            c.init_master()
        c.snapshot()
        c.average()
        c.step_merge(0.1, True)                          # a bf16 model is in s alone now
        sides.append((x, c))
    (xa, a), (xb, b) = sides
    norms = torch.zeros(K, device="cuda")
    try:
        graph = torch.cuda.CUDAGraph()
        a.sync()
        with torch.cuda.graph(graph, stream=st):
            a.local_step_clip(0.1, most, norms=norms.data_ptr())
        with torch.cuda.stream(st):
            graph.replay()
        a.local_step_clip(0.1, most, (1 << K) - 2)
        a.local_step_clip(0.1, most)
        for mask in ((1 << K) - 1, (1 << K) - 2, (1 << K) - 1):
            for k in range(K):
                if (mask >> k) & 1:
                    b.local_step_clip(0.1, most, 1 << k)
        a.sync()
        assert torch.equal(xa, xb)
        check_norms(norms.cpu().numpy().astype(np.float64), want)
        before = g[:, :n].clone()
        torch.cuda.synchronize()                         # the copy reads what the call is about to write, on another stream
        a.clip_grads(most, (1 << K) - 2)
        a.sync()
        assert torch.equal(g[0, :n], before[0])
        for k in range(1, K):
            assert torch.equal(g[k, :n], (before[k].float() * float(coefficient(want[k], most))).to(dtype)), k
    finally:
        a.close()
        b.close()
        del xa, xb, g, sides
        torch.cuda.empty_cache()


def mean_gradient(g):
    acc = np.zeros(g[0].size)
    for a in g:
        acc += a.astype(np.float64)
    return (acc / len(g)).astype(np.float32)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("K,name,tuning", [(1, "one", {}), (3, "odd", {}), (4, "rows", {}), (7, "many", dict(nontemporal=3)), (16, "odd", dict(nontemporal=3)), (2, "long", {}),
                                           (31, "blocks", {}), (64, "odd", {}), (6, "odd", dict(vec=4, waves_per_block=4, max_blocks=2, kper_merge=3)),
                                           (9, "blocks", dict(nontemporal=3, max_blocks=2))])
def test_sgd_all_reduce(K, name, tuning, storage):
    r = Rig(K, LISTS[name], storage)
    try:
        if tuning:
            r.ctx.set_tuning(**tuning)
        for step in range(4):
            g = r.grads(step)
            mean = mean_gradient(g)
            n = norm64(mean)
            most = float(np.float32(n * (0.4 if step % 2 == 0 else 1.5)))
            skips = step == 3
            if skips:
                g[K // 2][0] = -INF
            r.load(g)
            r.norms.fill_(-1.0)
            torch.cuda.synchronize()
            r.ctx.sgd_ar_step_clip(r.w.lr, most, skip_nonfinite=True, norms=r.norms.data_ptr())
            if not skips:
                r.orc.local_step([coefficient(n, most) * mean] * K, r.w.lr)
            r.same(f"step {step}", send=False)
            norms = r.read_norms()
            check_norms(norms[:1], [INF if skips else n])
            assert np.all(norms[1:] == -1.0)
        r.ctx.sgd_ar_step(r.w.lr)                                # and the plain call after it, on the same context
    finally:
        r.close()


def test_unclipped_sgd_all_reduce_after_a_clipped_one():
    """The clipped call brings the mean gradient's array; the plain call goes by its own rule and gives its own bits."""
    r = Rig(18, (1030, 257, 3))
    try:
        r.ctx.set_tuning(nontemporal=3)
        for step in range(3):
            g = r.grads(step)
            r.load(g)
            mean = mean_gradient(g)
            most = float(np.float32(0.5 * norm64(mean)))
            r.ctx.sgd_ar_step_clip(r.w.lr, most)
            r.orc.local_step([coefficient(norm64(mean), most) * mean] * r.K, r.w.lr)
            r.ctx.sgd_ar_step(r.w.lr)
            r.orc.sgd_ar_step(g, r.w.lr)
            r.same(f"step {step}", send=False)
    finally:
        r.close()


@pytest.mark.parametrize("storage,n", [("f32", 5000), ("f32", 50_000), ("bf16", 5000), ("bf16", 700_001)])
def test_graphs(storage, n):
    """The first clipped calls of a context are recorded: a cycle, clipping in place and an All-Reduce step; replays with new gradients, with
    eager calls and other work between them."""
    r = Rig(4, (n, 3, 257), storage, side_stream=False)
    K, lr = r.K, r.w.lr
    try:
        for o in (r.orc, r.ctx):
            o.snapshot()
        g = r.grads(0)
        r.load(g)
        most = r.max_norm(g)
        graph = torch.cuda.CUDAGraph()
        r.ctx.sync()
        with torch.cuda.graph(graph, stream=r.dev.main):
            r.ctx.average()
            r.ctx.local_step_clip(lr, most, skip_nonfinite=True)
            r.ctx.step_merge_clip(lr, most, norms=r.norms.data_ptr())
            r.ctx.sgd_ar_step_clip(lr, most)
            r.ctx.snapshot()
            r.ctx.clip_grads(most)

        def oracle(g):
            r.orc.average()
            use = r.clipped(g, most)
            r.orc.local_step(use, lr)
            r.orc.local_step(use, lr)
            r.orc.merge(True)
            mean = mean_gradient(g)
            r.orc.local_step([coefficient(norm64(mean), most) * mean] * K, lr)
            r.orc.snapshot()

        for rep in range(4):
            g = r.grads(10 + rep)
            r.load(g)
            if rep == 2:                                         # an eager call between two replays, on other gradients
                r.ctx.local_step_clip(lr, most)
                r.orc.local_step(r.clipped(g, most), lr)
                torch.zeros(1 << 16, device="cuda").add_(1.0)
            with torch.cuda.stream(r.dev.main):
                graph.replay()
            oracle(g)
            r.same(f"replay {rep}")
            check_norms(r.read_norms(), [norm64(a) for a in g])
            for k in range(K):
                want = coefficient(norm64(g[k]), most) * g[k]
                np.testing.assert_array_equal(r.device_grads(k), W.bf16_bits_to_f32(W.to_bf16_bits(want)) if r.bf16 else want)
    finally:
        r.close()


@pytest.mark.parametrize("name", ["odd", "blocks"])
def test_eager_calls_come_before_the_first_replay(name):
    """Recorded first, replayed late: eager calls in between find what they need."""
    r = Rig(3, LISTS[name], side_stream=False)
    try:
        graph = torch.cuda.CUDAGraph()
        r.ctx.sync()
        with torch.cuda.graph(graph, stream=r.dev.main):
            r.ctx.local_step_clip(r.w.lr, 0.05, norms=r.norms.data_ptr())
        for step in range(3):
            g = r.grads(step)
            r.load(g)
            r.ctx.local_step_clip(r.w.lr, 0.02)
            r.orc.local_step(r.clipped(g, 0.02), r.w.lr)
            with torch.cuda.stream(r.dev.main):
                graph.replay()
            r.orc.local_step(r.clipped(g, 0.05), r.w.lr)
            r.same(f"step {step}", send=False)
            check_norms(r.read_norms(), [norm64(a) for a in g])
    finally:
        r.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tensors_on_16_bytes(dtype):
    """Tensors packed as closely as the interface allows, so that rows start anywhere in a KiB; NaN in the gaps and behind the end."""
    numels = [5, 256, 1, 1030, 3, 70_001, 64]
    off = [0]
    for n in numels:
        off.append(off[-1] + (n + 7) // 8 * 8)
    K = 3
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    g = torch.full((K, off[-1] + 8), float("nan"), device="cuda", dtype=dtype)
    x = torch.zeros(K, off[-1] + 8, device="cuda", dtype=dtype)
    for k in range(K):
        for n, o in zip(numels, off):
            g[k, o:o + n] = (torch.randn(n, generator=gen, device="cuda") * (k + 1)).to(dtype)
    inside = torch.zeros(off[-1] + 8, dtype=torch.bool, device="cuda")
    for n, o in zip(numels, off):
        inside[o:o + n] = True
    g0 = g.clone()
    norms = torch.zeros(K, device="cuda")
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    c = B.Context(K, numels, storage=B.BF16 if dtype == torch.bfloat16 else B.F32, main_stream=st.cuda_stream, side_stream=st.cuda_stream)
    try:
        es = g.element_size()
        for k in range(K):
            c.bind(k, [x[k].data_ptr() + o * es for o in off[:-1]], [g[k].data_ptr() + o * es for o in off[:-1]])
        c.clip_grads(300.0, norms=norms.data_ptr())
        c.sync()
        for k in range(K):
            v = g0[k][inside].float().cpu().numpy()
            n = norm64(v)
            check_norms([float(norms[k])], [n])
            want = torch.from_numpy(coefficient(n, 300.0) * v).to(dtype)
            assert torch.equal(g[k][inside].cpu(), want)
            assert bool(torch.isnan(g[k][~inside]).all())
    finally:
        c.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_tensor_beyond_four_gigabytes(dtype):
    """2^31 - 2^21 elements, so that offsets pass 32 bits, with values at the beginning, around 2^31 bytes, 2^30 elements and at the odd end."""
    n = (1 << 31) - (1 << 21) - 3 if dtype == torch.bfloat16 else (1 << 30) + 1027
    x, g = torch.zeros(n, device="cuda", dtype=dtype), torch.zeros(n, device="cuda", dtype=dtype)
    at = sorted({0, 1, (1 << 29) - 1, 1 << 29, (1 << 30) - 1, (1 << 30) + 5, n - 2, n - 1})
    for i, j in enumerate(at):
        g[j] = float(i + 1)
    want = float(sum((i + 1) ** 2 for i in range(len(at)))) ** 0.5
    norms = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    c = B.Context(1, [n], storage=B.BF16 if dtype == torch.bfloat16 else B.F32, momentum=0.0, nesterov=False, main_stream=st.cuda_stream, side_stream=st.cuda_stream)
    try:
        c.bind(0, [x.data_ptr()], [g.data_ptr()])
        if dtype == torch.bfloat16:
            c.init_master()
        c.grad_norms(norms.data_ptr())
        c.sync()
        check_norms([float(norms)], [want])
        c.local_step_clip(1.0, 1.0)
        c.clip_grads(1.0)
        c.sync()
        cl = coefficient(want, 1.0)
        for i, j in enumerate(at):
            scaled = torch.tensor(float(cl * np.float32(i + 1)))
            assert float(g[j]) == float(scaled.to(dtype)) and float(x[j]) == float((-scaled).to(dtype)), j
        assert int(torch.count_nonzero(g)) == len(at) and int(torch.count_nonzero(x)) == len(at)
    finally:
        c.close()
        del x, g
        torch.cuda.empty_cache()


def test_refusals():
    """Every one leaves the context and the caller's buffers as they are."""
    r = Rig(3, LISTS["odd"])
    L, h = r.ctx._L, r.ctx._h
    p = r.norms.data_ptr()
    lrs = (ctypes.c_float * 3)(0.1, 0.1, 0.1)
    nan = float("nan")
    try:
        r.load(r.grads(0))

        def refused(status, what, st):
            assert st == status and L.lasgd_last_error(h), (what, st)

        for bad in (B.Clip(-1.0, 0, None), B.Clip(nan, 0, None), B.Clip(-INF, 0, None), B.Clip(1.0, 0, p + 2)):
            b = ctypes.byref(bad)
            refused(B.ERR_INVALID, "clip_grads", L.lasgd_clip_grads(h, 7, b))
            refused(B.ERR_INVALID, "local_step_clip", L.lasgd_local_step_clip(h, lrs, 7, b))
            refused(B.ERR_INVALID, "step_merge_clip", L.lasgd_step_merge_clip(h, lrs, 7, 7, 1, b))
            refused(B.ERR_INVALID, "sgd_ar_step_clip", L.lasgd_sgd_ar_step_clip(h, 0.1, b))
        ok = ctypes.byref(B.Clip(1.0, 0, p))
        for st in (L.lasgd_grad_norms(h, 7, None), L.lasgd_grad_norms(h, 0, p), L.lasgd_grad_norms(h, 8, p), L.lasgd_grad_norms(h, 7, p + 1),
                   L.lasgd_clip_grads(h, 0, ok), L.lasgd_clip_grads(h, 15, ok), L.lasgd_clip_grads(h, 7, None),
                   L.lasgd_local_step_clip(h, None, 7, ok), L.lasgd_local_step_clip(h, lrs, 8, ok), L.lasgd_local_step_clip(h, lrs, 7, None),
                   L.lasgd_local_step_clip(h, (ctypes.c_float * 3)(0.1, nan, 0.1), 7, ok),
                   L.lasgd_step_merge_clip(h, None, 7, 7, 1, ok), L.lasgd_step_merge_clip(h, lrs, 7, 0, 1, ok), L.lasgd_step_merge_clip(h, lrs, 9, 7, 1, ok),
                   L.lasgd_step_merge_clip(h, lrs, 7, 7, 1, None), L.lasgd_sgd_ar_step_clip(h, nan, ok), L.lasgd_sgd_ar_step_clip(h, 0.1, None)):
            refused(B.ERR_INVALID, "argument", st)
        refused(B.ERR_STATE, "no mean", L.lasgd_step_merge_clip(h, lrs, 7, 7, 1, ok))
        for f, args in ((L.lasgd_grad_norms, (7, p)), (L.lasgd_clip_grads, (7, ok)), (L.lasgd_local_step_clip, (lrs, 7, ok)),
                        (L.lasgd_step_merge_clip, (lrs, 7, 7, 1, ok)), (L.lasgd_sgd_ar_step_clip, (0.1, ok))):
            assert f(None, *args) == B.ERR_INVALID
        r.ctx.sync()
        assert bool((r.norms == -1.0).all())
        r.same("after refusals")
        # nothing is bound; a bf16 master that is not there
        c = B.Context(2, [16])
        n = torch.zeros(2, device="cuda")
        d = torch.zeros(2, 16, device="cuda", dtype=torch.bfloat16)
        e = B.Context(2, [16], storage=B.BF16)
        for k in range(2):
            e.bind(k, [d[k].data_ptr()], [d[k].data_ptr()])
        for f in (lambda: c.grad_norms(n.data_ptr()), lambda: c.clip_grads(1.0), lambda: c.local_step_clip(0.1, 1.0),
                  lambda: c.sgd_ar_step_clip(0.1, 1.0), lambda: e.local_step_clip(0.1, 1.0), lambda: e.sgd_ar_step_clip(0.1, 1.0)):
            with pytest.raises(B.LasgdError) as err:
                f()
            assert err.value.status == B.ERR_STATE
        e.clip_grads(1.0)                                       # needs no master
        e.close()
        c.close()
    finally:
        r.close()


# ---- the torch class ------------------------------------------------------------------------------------------------
def _modules(K, dtype=torch.float32):
    torch.manual_seed(0)
    base = torch.nn.Sequential(torch.nn.Linear(20, 33), torch.nn.ReLU(), torch.nn.Linear(33, 5)).to("cuda:0", dtype)
    return base, [copy.deepcopy(base) for _ in range(K)]


def _flat(tensors):
    return np.concatenate([t.detach().float().cpu().numpy().ravel() for t in tensors])


def _backward(replicas, step, dtype=torch.float32):
    for k, model in enumerate(replicas):
        g = torch.Generator(device="cuda:0")
        g.manual_seed(1000 * step + k)
        x = torch.randn(16, 20, generator=g, device="cuda:0").to(dtype)
        y = torch.randn(16, 5, generator=g, device="cuda:0").to(dtype)
        torch.nn.functional.mse_loss(model(x), y).mul((1.0, 20.0, 0.05)[k % 3]).backward()


@pytest.mark.parametrize("m", [1, 3])
@pytest.mark.parametrize("skip", [False, True])
def test_modules_train_with_clipped_gradients(m, skip):
    """The whole use: backward, clipped step, now and then an overflow in one replica's backward pass."""
    from paper_2203_13085_amd.torch_api import LASGD
    K, lr, mu, wd, most = 3, 0.05, 0.9, 1e-3, 0.5
    base, replicas = _modules(K)
    opt = LASGD(replicas, lr=lr, momentum=mu, nesterov=True, weight_decay=wd, m=m, max_grad_norm=most, skip_nonfinite=skip)
    ps = list(base.parameters())
    orc = O32.Oracle(K, [p.numel() for p in ps], mu, True, [wd] * len(ps))
    orc.set_model(_flat(ps))
    clipped = 0
    try:
        tau, started = 0, False
        for step in range(8):
            opt.zero_grad()
            _backward(replicas, step)
            if skip and step in (2, 5):
                list(replicas[step % K].parameters())[1].grad[4] = INF
            torch.cuda.synchronize()
            grads = [_flat([p.grad for p in r.parameters()]) for r in replicas]
            norms = [norm64(g) for g in grads]
            live = sum(1 << k for k in range(K) if np.isfinite(norms[k]))
            clipped += sum(n > most for n in norms)
            opt.step()
            check_norms(opt.grad_norms.cpu().numpy().astype(np.float64), norms)
            with np.errstate(invalid="ignore"):
                orc.local_step([coefficient(n, most) * g for n, g in zip(norms, grads)], [lr] * K, mask=live)
            tau += 1
            if not started:
                orc.snapshot(); orc.average(); started, tau = True, 0
            elif tau == m:
                orc.merge(True); orc.average(); tau = 0
            torch.cuda.synchronize()
            for k, r in enumerate(replicas):
                assert_close(_flat(list(r.parameters())), orc.x[k], f"step {step} replica {k}")
        assert 0 < clipped < 8 * K
    finally:
        opt.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_clip_grad_norm_in_place(dtype):
    """Against torch's own, replica by replica; the version counters notice; the caller's stream need not be waited for by hand."""
    from paper_2203_13085_amd.torch_api import LASGD
    K, most = 3, 0.5
    _, replicas = _modules(K, dtype)
    opt = LASGD(replicas, lr=0.1)
    try:
        opt.zero_grad()
        _backward(replicas, 0, dtype)
        torch.cuda.synchronize()
        before = [[p.grad.detach().clone() for p in r.parameters()] for r in replicas]
        versions = [p.grad._version for p in opt._flat]
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            norms = opt.clip_grad_norm_(most)
            after = [[p.grad.clone() for p in r.parameters()] for r in replicas]        # on s, right behind it
        s.synchronize()
        for k in range(K):
            n = norm64(_flat(before[k]))
            check_norms([float(norms[k])], [n])
            for a, b in zip(after[k], before[k]):
                want = torch.from_numpy(coefficient(n, most) * b.float().cpu().numpy()).to(dtype)
                assert torch.equal(a.cpu(), want)
        assert all(p.grad._version > v for p, v in zip(opt._flat, versions))
        # another tensor in a gradient's place is not what the library is bound to
        keep = opt._flat[1].grad
        opt._flat[1].grad = keep.clone()
        with pytest.raises(AssertionError, match="not the buffer"):
            opt.clip_grad_norm_(most)
        opt._flat[1].grad = None
        with pytest.raises(AssertionError, match="dropped"):
            opt.clip_grad_norm_(most)
        opt._flat[1].grad = keep
        opt.clip_grad_norm_(most)
    finally:
        opt.close()
    with pytest.raises(AssertionError, match="closed"):
        opt.clip_grad_norm_(most)


def test_class_arguments():
    from paper_2203_13085_amd.torch_api import LASGD
    _, replicas = _modules(1)
    for kw in (dict(max_grad_norm=-1.0), dict(max_grad_norm=float("nan")), dict(skip_nonfinite=True)):
        with pytest.raises(AssertionError):
            LASGD(replicas, lr=0.1, **kw)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_driver_loop(storage):
    """The fixed-cadence loop of the driver, clipped, fused and in two calls, against the oracle."""
    r = Rig(4, (70_000, 5, 1024), storage)
    try:
        g = r.grads(0)
        r.load(g)
        most = r.max_norm(g)
        r.dev.prologue(r.w.lr, most)
        r.orc.local_step(r.clipped(g, most), r.w.lr)
        r.orc.snapshot()
        r.orc.average()
        tau = 0
        for step in range(1, 5):
            g = r.grads(step)
            r.load(g)
            tau = r.dev.iteration(r.w.lr, tau, 2, fused=step < 3, max_norm=most)
            r.orc.local_step(r.clipped(g, most), r.w.lr)
            if tau == 0:
                r.orc.merge(True)
                r.orc.average()
            r.same(f"step {step}")
    finally:
        r.close()
