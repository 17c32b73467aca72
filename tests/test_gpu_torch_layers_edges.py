"""The layers through the torch class, where a program can go wrong without a word."""
import gc

import pytest
import torch

from paper_2203_13085_amd import torch_api
from tests.layers_util import DEV
from tests.test_gpu_torch_layers import close, forward64, make

pytestmark = pytest.mark.gpu


# ---- weights that are no longer where they were bound --------------------------------------------------------------------
def _other_data(opt, m):
    m.gate.weight.data = m.gate.weight.data.clone()


def _other_parameter(opt, m):
    m.gate.weight = torch.nn.Parameter(m.gate.weight.detach().clone())


def _assigned(opt, m):
    m.load_state_dict({n: q.clone() for n, q in m.state_dict().items()}, assign=True)


def _other_type(opt, m):
    m.to(torch.bfloat16)


def _other_layout(opt, m):
    m.gate.weight.data = m.gate.weight.data.t()             # the same address


def _fewer(opt, m):
    m.gate.weight.data = m.gate.weight.data[:4]             # the same address


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("replica", [0, 1])
@pytest.mark.parametrize("change", [_other_data, _other_parameter, _assigned, _other_type, _other_layout, _fewer])
def test_a_weight_that_moved_is_refused(change, replica, native, monkeypatch):
    """Forward passes, with and without gradients, and the backward pass of a call that was made before. What was bound stays alive here, so that
    a call that goes wrong reads old weights and nothing worse."""
    K, D, H = 2, 32, 32
    replicas, opt = make(K, D, H)
    if not native:
        monkeypatch.setattr(torch_api, "_walk", None)       # the class does without it where it is not built
    alive = [t for m in replicas for q in m.parameters() for t in (q.detach(), q.grad.detach())]
    old = [(m, dict(m._parameters), {n: dict(c._parameters) for n, c in m.named_children()}, [q.data for q in m.parameters()]) for m in replicas]
    x = torch.randn(K, 4, D, device=DEV)
    a, y = opt.gated("gate.weight", "up.weight", x), opt.rms_norm("norm", x)
    change(opt, replicas[replica])
    with pytest.raises(RuntimeError, match="bound"):
        opt.gated("gate.weight", "up.weight", x)
    with torch.no_grad(), pytest.raises(RuntimeError, match="bound"):
        opt.gated("gate.weight", "up.weight", x)
    with pytest.raises(RuntimeError, match="bound"):
        a.sum().backward()
    if change in (_assigned, _other_type):
        for call in (opt.rms_norm, opt.rms_norm_8bit):
            with pytest.raises(RuntimeError, match="bound"):
                call("norm", x)
        with pytest.raises(RuntimeError, match="bound"):
            y.sum().backward()
    else:
        opt.rms_norm("norm", x)                             # the norm's is where it was
    # back where it was bound
    for m, own, children, data in old:
        m._parameters.update(own)
        for n, ps in children.items():
            getattr(m, n)._parameters.update(ps)
        for q, d in zip(m.parameters(), data):
            q.data = d
    assert torch.equal(opt.gated("gate.weight", "up.weight", x), a.detach()) and len(alive) == 16
    opt.close()


class Renamed(torch.nn.Linear):
    """A module that names its parameters in its own way."""

    def named_parameters(self, *args, **kwargs):
        for n, q in super().named_parameters(*args, **kwargs):
            yield "shard.0." + n, q


def test_modules_that_name_their_parameters_in_their_own_way():
    """The submodule that the name speaks of is not there: the parameter's own place is compared all the same."""
    replicas = [Renamed(16, 16, bias=False).to(DEV) for _ in range(2)]
    opt = torch_api.LASGD(replicas, lr=0.1)
    x = torch.randn(2, 3, 16, device=DEV)
    opt.zero_grad()
    assert opt.gated("shard.0.weight", "shard.0.weight", x).shape == (2, 3, 8)          # both weights in one
    alive = replicas[1].weight.data
    replicas[1].weight.data = alive.clone()
    with pytest.raises(RuntimeError, match="bound"):
        opt.gated("shard.0.weight", "shard.0.weight", x)
    replicas[1].weight.data = alive
    opt.step()
    opt.close()


# ---- call numbers of recorded masks ----------------------------------------------------------------------------------------
def test_masks_of_eager_calls_and_of_two_graphs_never_meet():
    """Two graphs with two and three dropouts, replayed in turn, a third one recorded in between, and eager calls before, between and after: no mask comes twice."""
    K, rows, cols = 2, 8, 64
    replicas, opt = make(K, cols, 8, seed=5)
    x = torch.ones(K, rows, cols, device=DEV)
    masks = []

    def keep(*outs):
        torch.cuda.synchronize()
        masks.extend((o[k] != 0).cpu() for o in outs for k in range(K))
    side = torch.cuda.Stream()

    def record(n):
        graph = torch.cuda.CUDAGraph()
        gc.collect()                                        # a graph that is freed while another one is recorded ends the process
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            outs = [opt.dropout(x, 0.5) for _ in range(n - 1)]
            outs.append(opt.rms_norm("norm", x, torch.zeros_like(x), p=0.5)[1])
        return graph, outs
    with torch.no_grad():
        for _ in range(4):
            keep(opt.dropout(x, 0.5))
        graphs = [record(2), record(3)]
        for turn in range(6):
            if turn == 4:
                graphs.append(record(4))
            for graph, outs in graphs:
                opt.next_masks()
                graph.replay()
                keep(*outs)
            for _ in range(5):
                keep(opt.dropout(x, 0.5))
    seen = {m.numpy().tobytes() for m in masks}
    assert len(seen) == len(masks) == K * (4 + 6 * 5 + 6 * 5 + 2 * 4)
    opt.close()


def test_a_replay_without_moving_on_repeats_its_masks_and_its_backward_pass_has_the_same():
    K, cols = 2, 64
    replicas, opt = make(K, cols, 8, seed=6)
    x = torch.ones(K, 5, cols, device=DEV, requires_grad=True)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    warm = torch.ones(3, device=DEV, requires_grad=True)
    torch.autograd.grad(warm.sum(), warm)                   # what torch loads at its first gradient
    gc.collect()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        y = opt.dropout(x, 0.5)
        dx, = torch.autograd.grad(y, x, torch.ones_like(y))
    seen = []
    for turn in range(3):
        opt.next_masks()
        for _ in range(2):
            graph.replay()
            torch.cuda.synchronize()
            seen.append(y.detach().clone())
            assert torch.equal(y.detach(), dx)
        assert torch.equal(seen[-1], seen[-2])
    assert not torch.equal(seen[0], seen[2]) and not torch.equal(seen[2], seen[4])
    with pytest.raises(RuntimeError, match="record"):
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=side):
            opt.dropout(x.detach(), 0.5)
            opt.next_masks()
    torch.cuda.synchronize()
    opt.close()


# ---- forward passes that are run again in the backward pass ---------------------------------------------------------------------
@pytest.mark.parametrize("reentrant", [False, True])
def test_a_repeated_forward_pass_needs_its_call_numbers(reentrant):
    """torch.utils.checkpoint runs a forward pass again: without numbers of its own a dropout would draw another mask there."""
    from torch.utils.checkpoint import checkpoint
    K, D, H, p = 2, 48, 32, 0.5
    replicas, opt = make(K, D, H, seed=8)
    x, res = torch.randn(K, 6, D, device=DEV, requires_grad=True), torch.randn(K, 6, D, device=DEV)

    def block(x, *calls):
        y, h = opt.rms_norm("norm", x, res, p=p, call=calls[0] if calls else None)
        return opt.dropout(opt.gated("gate.weight", "up.weight", y), p, call=calls[1] if calls else None).square().sum() + h.sum()

    def grads():
        return [x.grad.clone(), *(q.grad.clone() for m in replicas for q in m.parameters())]
    opt.zero_grad()
    block(x, 1, 2).backward()
    want = grads()
    x.grad = None
    opt.zero_grad()
    checkpoint(lambda x: block(x, 1, 2), x, use_reentrant=reentrant).backward()
    for a, b in zip(grads(), want):
        assert torch.equal(a, b)
    loss = checkpoint(block, x, use_reentrant=reentrant)
    with pytest.raises(RuntimeError, match="call"):
        loss.backward()
    loss = checkpoint(lambda x: opt.dropout(x, 0.0).sum(), x, use_reentrant=reentrant)         # no mask, no number
    loss.backward()
    torch.cuda.synchronize()
    opt.close()


# ---- batches without rows -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows", [None, [0, 0]])
def test_a_batch_without_rows_has_a_backward_pass(rows):
    K, D, H = 2, 32, 24
    replicas, opt = make(K, D, H)
    x, res = (torch.randn(K, 0, D, device=DEV, requires_grad=True) for _ in range(2))
    opt.zero_grad()
    y, h = opt.rms_norm("norm", x, res, p=0.5, rows=rows)
    a = opt.gated("gate.weight", "up.weight", y, rows=rows)
    d = opt.dropout(h, 0.5, res, rows=rows)
    (a.sum() + d.sum()).backward()
    assert x.grad.shape == res.grad.shape == (K, 0, D) and a.shape == (K, 0, H)
    assert all(bool(q.grad.eq(0).all()) for m in replicas for q in m.parameters())
    opt.close()


# ---- unlike numbers of rows -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D,H,R,rows", [(40, 24, 12, [12, 0, 5]), (64, 88, 70, [1, 70, 33]), (33, 17, 9, [0, 2, 9])])
def test_ragged_rows_against_64_bits(D, H, R, rows, dtype):
    """Outputs and all gradients of every replica's rows, as if it were alone with them."""
    K, p, calls = 3, 0.25, (11, 12)
    replicas, opt = make(K, D, H, dtype, seed=31)
    x, res, dy = (torch.randn(K, R, D, device=DEV).to(dtype) for _ in range(3))
    for k, n in enumerate(rows):
        x[k, n:], res[k, n:], dy[k, n:] = float("nan"), float("inf"), float("nan")       # counts for nothing
    downs = [m.down.weight for m in replicas]

    x.requires_grad_(), res.requires_grad_()
    opt.zero_grad()
    y, h = opt.rms_norm("norm", x, res, p=p, rows=rows, call=calls[0], eps=1e-5)
    a = opt.gated("gate.weight", "up.weight", y, rows=rows)
    out = opt.dropout(torch.stack([a[k] @ downs[k].T for k in range(K)]), p, h, rows=rows, call=calls[1])
    out.backward(dy)
    out = out.detach()
    for k, (n, m) in enumerate(zip(rows, replicas)):
        assert all(bool((t[k, n:] == 0).all()) for t in (out, x.grad, res.grad))
        if not n:
            assert all(bool(q.grad.eq(0).all()) for q in m.parameters())
            continue
        W = {name: q.detach().double().requires_grad_() for name, q in m.named_parameters()}
        xk, rk = x[k, :n].detach().double().requires_grad_(), res[k, :n].detach().double().requires_grad_()
        want = forward64(W, k, xk, rk, p, calls, 31)
        want.backward(dy[k, :n].double())
        close(out[k, :n], want, dtype, D + H, "out")
        for name, q in m.named_parameters():
            close(q.grad, W[name].grad, dtype, D + H + 2 * n, name)
        close(x.grad[k, :n], xk.grad, dtype, 2 * (D + H), "dx")
        close(res.grad[k, :n], rk.grad, dtype, 2 * (D + H), "dres")
    opt.close()
