"""Gradient norms and clipping where a promise is easily broken: no limit next to what is not finite, one norm for calls that are to give the
same bits, and torch watching its operations.

No tolerances: everything here is the other call's result, bit by bit, or a value that is rounded once."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2203_13085_amd import binding as B              # noqa: E402
from tests.test_gpu_clip import LISTS, Rig, check_norms, coefficient, norm64, _backward, _flat, _modules      # noqa: E402

pytestmark = pytest.mark.gpu

INF = float("inf")
BAD = {"inf": INF, "-inf": -INF, "nan": float("nan")}


def same_state(a, b, K, what):
    """NaN where the other has one, and everything else to the bit."""
    for which in (B.STATE_X, B.STATE_V, B.STATE_S):
        for k in range(K):
            p, q = a.ctx.read_state(which, k), b.ctx.read_state(which, k)
            nan = np.isnan(p)
            np.testing.assert_array_equal(nan, np.isnan(q), err_msg=f"{what}: NaN, array {which}, replica {k}")
            np.testing.assert_array_equal(p[~nan].view(np.uint32), q[~nan].view(np.uint32), err_msg=f"{what}: array {which}, replica {k}")


def with_a_bad_element(r, step, bad):
    g = r.grads(step)
    g[1][r.N // 2] = BAD[bad]
    return g


# ---- no limit ------------------------------------------------------------------------------------------------------------
NO_LIMIT = [("odd", 3), ("blocks", 3), ("128 tiles", 4)]           # one launch; norms and then the rest; one launch for steps alone


@pytest.mark.parametrize("skip", [False, True])
@pytest.mark.parametrize("bad", list(BAD))
@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("name,K", NO_LIMIT)
def test_no_limit_scales_nothing_in_place(name, K, storage, bad, skip):
    """max_norm = infinity: whatever the gradients hold, clipping in place leaves every bit, and the norms say what is not finite."""
    r = Rig(K, LISTS[name], storage)
    try:
        g = with_a_bad_element(r, 0, bad)
        r.load(g)
        view = torch.int16 if r.bf16 else torch.int32
        before = [t.clone().view(view) for t in r.dev.g]
        torch.cuda.synchronize()
        r.ctx.clip_grads(INF, skip_nonfinite=skip, norms=r.norms.data_ptr())
        check_norms(r.read_norms(), [norm64(a) for a in g])
        assert all(torch.equal(a.view(view), b) for a, b in zip(r.dev.g, before))
    finally:
        r.close()


@pytest.mark.parametrize("skip", [False, True])
@pytest.mark.parametrize("bad", ["inf", "nan"])
@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("name,K", NO_LIMIT)
def test_no_limit_steps_as_the_unclipped_calls(name, K, storage, bad, skip):
    """max_norm = infinity: an infinity or a NaN does to the model what it does in the unclipped calls, to its own element; with skip_nonfinite the replica
    that holds it takes no step, as in a masked call."""
    a, b = Rig(K, LISTS[name], storage), Rig(K, LISTS[name], storage)
    full = (1 << K) - 1
    live = full & ~2 if skip else full
    lrs = [0.05 * (1.0 + 0.1 * k) for k in range(K)]
    try:
        g = a.grads(0)
        for r in (a, b):                                             # a step of finite gradients first: there is a momentum to keep
            r.load(g)
            r.ctx.snapshot()
            r.ctx.average()
        a.ctx.local_step_clip(lrs, INF, skip_nonfinite=skip)
        b.ctx.local_step_ex(lrs, full)
        g = with_a_bad_element(a, 1, bad)
        for r in (a, b):
            r.load(g)
        a.ctx.local_step_clip(lrs, INF, skip_nonfinite=skip)
        b.ctx.local_step_ex(lrs, live)
        same_state(a, b, K, "step")
        a.ctx.step_merge_clip(lrs, INF, full, full, True, skip_nonfinite=skip)
        b.ctx.step_merge_ex(lrs, live, full, True)
        same_state(a, b, K, "step and update")
        for k in range(K):
            assert np.isfinite(a.ctx.read_state(B.STATE_X, k)).sum() >= a.N - 1
    finally:
        a.close()
        b.close()


@pytest.mark.parametrize("bad", ["inf", "nan"])
@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("name,K", NO_LIMIT[:2])
def test_no_limit_all_reduce_as_the_unclipped_call(name, K, storage, bad):
    a, b = Rig(K, LISTS[name], storage), Rig(K, LISTS[name], storage)
    try:
        g = with_a_bad_element(a, 0, bad)
        for r in (a, b):
            r.load(g)
        a.ctx.sgd_ar_step_clip(0.05, INF)
        b.ctx.sgd_ar_step(0.05)
        same_state(a, b, K, "step")
        for k in range(K):
            assert np.isfinite(a.ctx.read_state(B.STATE_X, k)).sum() == a.N - 1
        a.ctx.sgd_ar_step_clip(0.05, INF, skip_nonfinite=True)       # all sit out
        same_state(a, b, K, "a step that all sit out")
    finally:
        a.close()
        b.close()


def test_class_without_a_limit_takes_the_norms_only():
    """LASGD(max_grad_norm=infinity) next to LASGD(): an infinity in one replica's gradients spoils its own element and no other."""
    from paper_2203_13085_amd.torch_api import LASGD
    K = 3
    _, plain = _modules(K)
    _, taken = _modules(K)
    p, q = LASGD(plain, lr=0.05, m=2), LASGD(taken, lr=0.05, m=2, max_grad_norm=INF)
    try:
        for step in range(4):
            p.zero_grad()
            _backward(plain, step)
            if step == 1:
                list(plain[1].parameters())[0].grad[2, 3] = INF
            for u, v in zip(p._flat, q._flat):
                v.grad.copy_(u.grad)
            p.step()
            q.step()
            torch.cuda.synchronize()
            for u, v in zip(plain, taken):
                x, y = _flat(list(u.parameters())), _flat(list(v.parameters()))
                np.testing.assert_array_equal(x, y)                  # a NaN equals a NaN here
                assert step > 1 or np.isfinite(y).sum() >= y.size - 1
            if step < 2:
                assert np.isinf(q.grad_norms.cpu().numpy()).tolist() == [False, step == 1, False]
    finally:
        p.close()
        q.close()


# ---- one norm ------------------------------------------------------------------------------------------------------------
def straddling(numels, big, tiny):
    """`big` in the first of a lane's four elements in the first sixteen tiles, `tiny` elsewhere: tiny^2 is just under half an ulp of big^2's binade, so it is
    lost where it is added to big^2 and counts where it meets its like first, and the 64-bit sum tells the order it was made in."""
    out, tile = [], 0
    for n in numels:
        i = np.arange(n)
        out.append(np.where((i % 4 == 0) & (tile + i // 256 < 16), np.float32(big), np.float32(tiny)).astype(np.float32))
        tile += (n + 255) // 256
    return np.concatenate(out)


@pytest.mark.parametrize("numels,big,most", [((32_768,), "0x1.2ca558p+0", "0x1.8f7026p+4"),                # whole runs of one tensor
                                             ((3, 20_000, 12_000), "0x1.624e48p+0", "0x1.4cac20p+5")])     # several tensors in a run
def test_a_clipped_step_is_clipping_and_a_step(numels, big, most):
    """fp32, lists of two blocks of tiles: the step takes one launch and clipping in place two, and both have to come to one coefficient.  The limits were
    found by search: sums that differ by a few ulps on either side of where the coefficient rounds to its neighbour."""
    tiny, most = float.fromhex("0x1.69db8cp-27"), float.fromhex(most)
    a, b = Rig(1, numels), Rig(1, numels)
    g = straddling(numels, float.fromhex(big), tiny)
    try:
        for r in (a, b):
            r.load([g])
        a.ctx.local_step_clip(0.05, most, norms=a.norms.data_ptr())
        b.ctx.clip_grads(most, norms=b.norms.data_ptr())
        b.ctx.local_step_ex([0.05], 1)
        same_state(a, b, 1, "step")
        assert a.read_norms().tolist() == b.read_norms().tolist()
    finally:
        a.close()
        b.close()


@pytest.mark.parametrize("K", [1, 5, 64])
@pytest.mark.parametrize("name", ["odd", "64 tiles", "65 tiles", "128 tiles", "127 of many", "129 tiles", "blocks"])
def test_a_clipped_step_is_clipping_and_a_step_on_every_route(name, K):
    if K == 64:
        name = {"blocks": "rows"}.get(name, name)
    a, b = Rig(K, LISTS[name]), Rig(K, LISTS[name])
    full, part = (1 << K) - 1, ((1 << K) - 1) & 0x5555555555555555
    lrs = [0.05 * (1.0 + 0.01 * k) for k in range(K)]
    try:
        for r in (a, b):
            r.ctx.snapshot()
        for step, mask in enumerate((full, part, full)):
            g = a.grads(step)
            most = a.max_norm(g)
            for r in (a, b):
                r.load(g)
                r.ctx.average()
            a.ctx.local_step_clip(lrs, most, mask)
            a.ctx.step_merge_clip(lrs, most, mask, full, True)
            b.ctx.clip_grads(most, mask)
            b.ctx.local_step_ex(lrs, mask)
            b.ctx.step_merge_ex(lrs, mask, full, True)
            same_state(a, b, K, f"step {step}")
    finally:
        a.close()
        b.close()


# ---- torch watching ------------------------------------------------------------------------------------------------------
def _watch(kind, seen):
    """A mode that notes which memory torch's operations write in place."""
    from torch.overrides import TorchFunctionMode
    from torch.utils._python_dispatch import TorchDispatchMode

    def note(func, args):
        name = getattr(func, "__name__", str(func)).split(".")[0]
        if name.endswith("_") and not name.endswith("__"):
            for t in args[0] if isinstance(args[0], (list, tuple)) else [args[0]]:
                seen.add(t.data_ptr())

    class Dispatch(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            note(func, args)
            return func(*args, **(kwargs or {}))

    class Function(TorchFunctionMode):
        def __torch_function__(self, func, types, args=(), kwargs=None):
            note(func, args)
            return func(*args, **(kwargs or {}))

    return Dispatch() if kind == "dispatch" else Function()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["dispatch", "function"])
@pytest.mark.parametrize("most,skip", [(0.5, False), (0.5, True), (INF, False), (1e9, True), (0.0, False)])
def test_clip_grad_norm_is_seen_by_modes(kind, dtype, most, skip):
    """While a mode watches torch's operations it sees every gradient written; the result is that of a call nobody watches."""
    from paper_2203_13085_amd.torch_api import LASGD
    K = 3
    _, replicas = _modules(K, dtype)
    opt = LASGD(replicas, lr=0.1)
    view = torch.int16 if dtype == torch.bfloat16 else torch.int32
    try:
        opt.zero_grad()
        _backward(replicas, 0, dtype)
        list(replicas[2].parameters())[1].grad[4] = INF
        torch.cuda.synchronize()
        fresh = [p.grad.detach().clone() for p in opt._flat]
        seen = set()
        with _watch(kind, seen):
            norms = opt.clip_grad_norm_(most, skip_nonfinite=skip)
        assert {p.grad.data_ptr() for p in opt._flat} <= seen
        watched = [p.grad.detach().clone() for p in opt._flat]
        for p, g in zip(opt._flat, fresh):
            p.grad.copy_(g)
        plain = opt.clip_grad_norm_(most, skip_nonfinite=skip)
        assert norms.dtype == plain.dtype and norms.tolist() == plain.tolist()
        for w, p in zip(watched, opt._flat):
            nan = torch.isnan(w)
            assert torch.equal(nan, torch.isnan(p.grad))
            assert torch.equal(w.view(view)[~nan], p.grad.view(view)[~nan])
        with _watch(kind, seen), pytest.raises(B.LasgdError) as err:
            opt.clip_grad_norm_(-1.0)
        assert err.value.status == B.ERR_INVALID
    finally:
        opt.close()


def test_clip_grad_norm_recorded():
    """Inside a graph the library's own kernels are recorded; replays on new gradients, with eager work between them."""
    from paper_2203_13085_amd.torch_api import LASGD
    K, most = 3, 0.5
    _, replicas = _modules(K)
    opt = LASGD(replicas, lr=0.1)
    try:
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            norms = opt.clip_grad_norm_(most)
        for step in range(3):
            opt.zero_grad()
            _backward(replicas, step)
            torch.cuda.synchronize()
            before = [[p.grad.detach().clone() for p in r.parameters()] for r in replicas]
            graph.replay()
            torch.cuda.synchronize()
            for k, r in enumerate(replicas):
                n = norm64(_flat(before[k]))
                check_norms([float(norms[k])], [n])
                for p, b in zip(r.parameters(), before[k]):
                    assert torch.equal(p.grad.cpu(), torch.from_numpy(coefficient(n, most) * b.cpu().numpy()))
    finally:
        torch.cuda.synchronize()
        opt.close()


# ---- what the calls' routes leave out elsewhere ----------------------------------------------------------------------------
def test_streamed_norms_recorded_and_masked():
    """More than 256 MiB of fp32 gradients, whose norms an update reads with the streaming hint: recorded, with masks, and next to the same calls in
    pieces that are too small for that."""
    K, n, st = 3, 25_000_003, torch.cuda.Stream()
    rows = (n + 255) // 256 * 256
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    g = torch.zeros(K, rows, device="cuda")
    for k in range(K):
        g[k, :n] = torch.randn(n, generator=gen, device="cuda") * (1e-3 * (k + 1))
    x0 = torch.randn(n, generator=gen, device="cuda") * 0.05
    want = [float(torch.linalg.vector_norm(g[k, :n].double())) for k in range(K)]
    most, full = float(np.float32(want[1])) * 0.75, (1 << K) - 1
    sides, norms = [], torch.zeros(2, K, device="cuda")
    for _ in range(2):
        x = torch.zeros(K, rows, device="cuda")
        x[:, :n] = x0
        c = B.Context(K, [n], main_stream=st.cuda_stream, side_stream=st.cuda_stream, wd_scalar=1e-4)
        for k in range(K):
            c.bind(k, [x[k].data_ptr()], [g[k].data_ptr()])
        sides.append((x, c))
    torch.cuda.synchronize()
    (xa, a), (xb, b) = sides
    try:
        assert 4 * K * rows > 256 << 20 > 4 * rows
        a.snapshot()
        b.snapshot()
        graph = torch.cuda.CUDAGraph()
        a.sync()
        with torch.cuda.graph(graph, stream=st):
            a.average()
            a.local_step_clip(0.1, most)
            a.step_merge_clip(0.1, most, full, full, True, norms=norms[0].data_ptr())
        for rep in range(3):
            with torch.cuda.stream(st):
                graph.replay()
            b.average()
            for k in range(K):
                b.local_step_clip(0.1, most, 1 << k)
            for k in range(K):
                b.local_step_clip(0.1, most, 1 << k, norms=norms[1].data_ptr())
            b.merge(True)
            a.sync()
            assert torch.equal(xa, xb), rep
            check_norms(norms[0].cpu().numpy().astype(np.float64), want)
            check_norms(norms[1].cpu().numpy().astype(np.float64), want)
        a.local_step_clip(0.1, most, full)
        a.local_step_clip(0.1, most, 0b101)
        for k in (0, 1, 2, 0, 2):
            b.local_step_clip(0.1, most, 1 << k)
        a.sync()
        assert torch.equal(xa, xb)
    finally:
        a.close()
        b.close()
        del xa, xb, g, sides
        torch.cuda.empty_cache()


@pytest.mark.parametrize("skip", [False, True])
def test_bf16_modules_train_with_clipped_gradients(skip):
    """bf16 modules with fp32 master copies: backward, clipped step, now and then an overflow, against the oracle on the widened gradients."""
    from oracle import lasgd_oracle as O32
    from paper_2203_13085_amd import workloads as W
    from paper_2203_13085_amd.torch_api import LASGD
    K, m, lr, mu, wd, most = 3, 2, 0.05, 0.9, 1e-3, 0.5
    base, replicas = _modules(K, torch.bfloat16)
    opt = LASGD(replicas, lr=lr, momentum=mu, nesterov=True, weight_decay=wd, m=m, max_grad_norm=most, skip_nonfinite=skip)
    ps = list(base.parameters())
    orc = O32.Oracle(K, [p.numel() for p in ps], mu, True, [wd] * len(ps))
    orc.set_model(_flat(ps))
    clipped = 0
    try:
        tau, started = 0, False
        for step in range(7):
            opt.zero_grad()
            _backward(replicas, step, torch.bfloat16)
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
                orc.snapshot()
                orc.average()
                started, tau = True, 0
            elif tau == m:
                orc.merge(True)
                orc.average()
                tau = 0
            torch.cuda.synchronize()
            for k, r in enumerate(replicas):
                got = np.concatenate([p.detach().view(torch.int16).cpu().numpy().ravel() for p in r.parameters()]).view(np.uint16)
                np.testing.assert_array_equal(got, W.to_bf16_bits(orc.x[k]), err_msg=f"step {step} replica {k}")
        assert 0 < clipped < 7 * K
    finally:
        opt.close()
