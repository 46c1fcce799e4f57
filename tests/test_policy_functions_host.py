"""What the Functions of ssm_policy do with inputs that carry a forward-mode tangent, around stand-ins for the handles (plain
torch on the CPU); without a GPU.  The handles read tensors by address, so that a tangent has nowhere to go: the call has to
raise, as the Functions' own forward-mode rule does, and not to return a result that looks constant."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2603_12145_b200 import gated_recurrence, ssm_policy


class StandIn:
    """A result of plain torch operations on the detached values: what reading by address sees."""

    def saved(self, *sizes):
        return (torch.zeros(1), torch.zeros(1)) if len(sizes) == 1 and self.pair else torch.zeros(1)

    def __init__(self, pair=False):
        self.pair = pair

    def forward(self, x, *args, residual=None, saved=None):
        y = x.detach() * 2.0
        return y if residual is None else (y, x.detach() + residual.detach())

    def sequence(self, x, *args, **kw):
        return x.detach() * 2.0

    scan = sequence


def call(name, v):
    """A Function's call with v its tensors by name; what is not there is a constant."""
    x = torch.ones(1, 3, 2) if name in ("scan", "recurrence") else torch.ones(3, 2)
    w = torch.ones(2)
    at = lambda key, other: v.get(key, other)                                              # noqa: E731
    if name == "norm":
        return ssm_policy.NormFunction.apply(StandIn(), at("x", x), None, at("w", w), at("b", w))
    if name == "added":
        return ssm_policy.NormFunction.apply(StandIn(), at("x", x), at("residual", x), at("w", w), at("b", w))[0]
    if name == "recurrence":
        return ssm_policy.RecurrenceFunction.apply(StandIn(), at("x", x), at("r", x), at("i", x), at("a", -w), None,
                                                   at("state", torch.ones(1, 2)), None)
    if name == "scan":
        return ssm_policy.ScanFunction.apply(StandIn(), at("x", x), at("dt", x), at("a", -torch.ones(2, 4)), at("b", torch.ones(1, 3, 4)),
                                             torch.ones(1, 3, 4), w, x, w, None, None, None)
    return ssm_policy.FfnFunction.apply(StandIn(pair=True), at("x", x), at("w_in", torch.ones(4, 2)), torch.ones(2, 2))


TENSORS = {"norm": {"x": (3, 2), "w": (2,), "b": (2,)}, "added": {"x": (3, 2), "residual": (3, 2), "w": (2,)},
           "recurrence": {"x": (1, 3, 2), "r": (1, 3, 2), "a": (2,), "state": (1, 2)},
           "scan": {"x": (1, 3, 2), "dt": (1, 3, 2), "b": (1, 3, 4)}, "ffn": {"x": (3, 2), "w_in": (4, 2)}}


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("name,key", [(n, k) for n, keys in TENSORS.items() for k in keys])
def test_a_tangent_is_refused(name, key, grad):
    with forward_ad.dual_level(), torch.set_grad_enabled(grad):
        v = torch.full(TENSORS[name][key], -1.0 if key == "a" else 1.0)
        with pytest.raises(NotImplementedError):
            call(name, {key: forward_ad.make_dual(v, torch.ones_like(v))})


@pytest.mark.parametrize("name", list(TENSORS))
def test_without_one_the_call_goes_through(name):
    want = call(name, {})
    with forward_ad.dual_level():                    # nobody carries one
        assert torch.equal(call(name, {}), want)
        with torch.no_grad():
            assert torch.equal(call(name, {}), want)


class Recurrence(StandIn):
    """y_t = x_t + state (where no episode starts at the first step), and its gradients."""

    def sequence(self, x, r, i, a, reset=None, state=None, state_out=None, saved=None):
        return x.detach() + (0.0 if state is None else self.kept(reset) * state.detach().unsqueeze(1))

    def kept(self, reset):
        return 1.0 if reset is None else (reset[:, :1] == 0).unsqueeze(-1).float()

    def backward(self, dy, x, r, i, a, saved, reset=None, dstate_out=None, want_dstate=False):
        self.wanted = want_dstate
        zero = torch.zeros_like(x)
        return {"dx": dy.clone(), "dr": zero, "di": zero, "da": torch.zeros_like(a),
                "dstate": (self.kept(reset) * dy).sum(1) if want_dstate else None}


@pytest.mark.parametrize("alone", [False, True])
@pytest.mark.parametrize("reset", [None, 0, 1])
def test_the_state_at_the_start_has_its_gradient(alone, reset):
    """With or without another input that requires one; none is formed where none is wanted."""
    op, x, a = Recurrence(), torch.ones(2, 3, 4, requires_grad=not alone), -torch.ones(4)
    state = torch.ones(2, 4, requires_grad=True)
    mask = None if reset is None else torch.tensor([[reset, 0, 0], [0, 1, 0]], dtype=torch.uint8)
    weight = torch.arange(24.0).view(2, 3, 4)
    (weight * ssm_policy.RecurrenceFunction.apply(op, x, x, x, a, mask, state, None)).sum().backward()
    want = weight.sum(1)
    if reset:
        want[0] = 0.0
    assert torch.equal(state.grad, want)
    if not alone:
        ssm_policy.RecurrenceFunction.apply(op, x, x, x, a, mask, state.detach(), None).sum().backward()
        assert op.wanted is False


def test_a_second_derivative_by_the_state_is_refused():
    op, x = Recurrence(), torch.ones(2, 3, 4, requires_grad=True)
    state = torch.ones(2, 4, requires_grad=True)
    (g,) = torch.autograd.grad(ssm_policy.RecurrenceFunction.apply(op, x, x, x, -torch.ones(4), None, state, None).sum(), x,
                               create_graph=True)
    with pytest.raises(RuntimeError, match="first derivatives only"):
        torch.autograd.grad(g.sum(), state)


# ---- the recurrence's outputs ---------------------------------------------------------------


@pytest.mark.parametrize("strides", [(40, 8, 1), (8, 32, 1), (0, 8, 1), (8, 0, 1), (0, 0, 1), (5, 1, 1), (1, 5, 1), (1, 1, 1), (100, 3, 1),
                                     (3, 100, 1)], ids=str)
def test_outputs_have_contiguous_rows_that_lie_apart(strides):
    """Whatever the strides of the input: expanded ones and overlapping windows among them."""
    op = object.__new__(gated_recurrence.GatedRecurrence)
    op.torch, op.dtype, op.channels, op.device, op.h = torch, torch.float32, 8, torch.device("cpu"), None
    v = torch.zeros(1000).as_strided((4, 5, 8), strides)
    out = op._like(v)
    assert out.shape == v.shape and out.stride(2) == 1 and out.is_contiguous() == (strides[0] >= strides[1])
    assert out.is_contiguous() or out.transpose(0, 1).is_contiguous()
