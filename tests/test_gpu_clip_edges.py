"""Gradient norms and clipping where a promise is easily broken: no limit next to what is not finite.

No tolerances: everything here is the other call's result, bit by bit, or a value that is rounded once."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2203_13085_amd import binding as B              # noqa: E402
from tests.test_gpu_clip import LISTS, Rig, check_norms, norm64, _backward, _flat, _modules      # noqa: E402

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
