"""The layers through the torch class, where a program can go wrong without a word."""
import pytest
import torch

from tests.layers_util import DEV
from tests.test_gpu_torch_layers import make

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


@pytest.mark.parametrize("replica", [0, 1])
@pytest.mark.parametrize("change", [_other_data, _other_parameter, _assigned, _other_type, _other_layout, _fewer])
def test_a_weight_that_moved_is_refused(change, replica):
    """Forward passes, with and without gradients, and the backward pass of a call that was made before. What was bound stays alive here, so that
    a call that goes wrong reads old weights and nothing worse."""
    K, D, H = 2, 32, 32
    replicas, opt = make(K, D, H)
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
