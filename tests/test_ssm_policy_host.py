"""What autograd sees of the sequence operators: the Functions of ssm_policy around stand-ins for the
handles (plain torch on the CPU), without a GPU."""
import pytest
import torch

from paper_2603_12145_b200 import ssm_policy


class StandIn:
    """Element-wise operators with the handles' interfaces: y = x^2, and what a gradient needs beyond the
    inputs is read back from the buffers that the forward call filled."""

    def __init__(self):
        self.asked = 0           # buffers for a backward pass

    # ssm.Ssm
    def conv(self, x, w, bias=None, reset=None, history=None, history_out=None):
        return x * x + 0 * w.sum()

    def conv_backward(self, dy, x, w, bias=None, reset=None, history=None):
        scale = 1.0 if history is None else history.sum()
        return (2 * x * dy * scale * (1.0 if reset is None else (reset == 0).unsqueeze(-1)), torch.zeros_like(w),
                None if bias is None else torch.zeros_like(bias))

    def saved(self, *sizes):
        self.asked += 1
        return (torch.zeros(1), torch.zeros(1)) if len(sizes) == 1 else torch.zeros(1)

    def scan(self, x, dt, a, b, c, d=None, z=None, dt_bias=None, reset=None, state=None, state_out=None, saved=None):
        if saved is not None:
            saved.fill_(2.0)
        return x * x

    def scan_backward(self, dy, x, dt, a, b, c, saved, d=None, z=None, dt_bias=None, reset=None):
        grads = {"d" + k: (None if v is None else torch.zeros_like(v))
                 for k, v in (("x", x), ("dt", dt), ("a", a), ("b", b), ("c", c), ("d", d), ("z", z), ("dt_bias", dt_bias))}
        grads["dx"] = saved * x * dy * (1.0 if reset is None else (reset == 0).unsqueeze(-1))
        return grads

    # gated_ffn.GatedFfn
    def forward(self, x, w_in, w_out, saved=None):
        if saved is not None:
            saved[0].fill_(2.0)
        return x * x

    def backward(self, dy, x, w_in, w_out, saved, want_dx=True):
        return saved[0] * x * dy, torch.zeros_like(w_in), torch.zeros_like(w_out)


def through(name, op, x, reset=None, history=None):
    """One of the Functions on x [batch, time, features] (the block: rows)."""
    w = torch.zeros(1)
    if name == "conv":
        return ssm_policy.ConvFunction.apply(op, x, w, None, reset, history, None)
    if name == "scan":
        return ssm_policy.ScanFunction.apply(op, x, torch.zeros_like(x), w, w, w, None, None, None, reset, None, None)
    return ssm_policy.FfnFunction.apply(op, x, w, w)


def inputs():
    return torch.tensor([[[1.0], [2.0], [3.0]]], requires_grad=True)


@pytest.mark.parametrize("name", ["conv", "scan", "ffn"])
def test_first_derivatives_pass_and_second_ones_are_refused(name):
    """The backward calls are kernels, which autograd cannot differentiate: with a residual connection a second
    derivative would come out as that of the residual alone."""
    x = inputs()
    y = x * x + through(name, StandIn(), x)
    (g,) = torch.autograd.grad(y.sum(), x, create_graph=True)
    assert torch.equal(g, 4 * x)
    with pytest.raises(RuntimeError, match="first derivatives only"):
        torch.autograd.grad(g.sum(), x)
    scale = torch.tensor(3.0, requires_grad=True)      # the incoming gradient has a graph, the input has none behind it
    (g,) = torch.autograd.grad((scale * through(name, StandIn(), x)).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="first derivatives only"):
        torch.autograd.grad(g.sum(), scale)
