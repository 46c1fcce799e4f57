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

    def conv_step(self, x, history, w, bias=None, done=None):
        return x

    def scan_step(self, x, dt, a, b, c, state, d=None, z=None, dt_bias=None, done=None):
        return x

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


@pytest.mark.parametrize("name,which", [("conv", "reset"), ("conv", "history"), ("scan", "reset")])
def test_a_mask_or_history_changed_before_the_backward_pass_is_noticed(name, which):
    x, reset, history = inputs(), torch.tensor([[0, 1, 0]], dtype=torch.uint8), torch.ones(1, 3, 1)
    more = {"reset": reset}
    if name == "conv":
        more["history"] = history
    y = through(name, StandIn(), x, **more)
    y.sum().backward(retain_graph=True)                # as it was
    more[which].zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


@pytest.mark.parametrize("name", ["conv", "scan", "ffn"])
def test_saved_tensor_hooks_see_all_that_the_backward_pass_reads(name):
    """Under hooks that replace what is kept (to move it elsewhere, say), the gradients come from the replacements."""
    x, reset, history, kept = inputs(), torch.tensor([[0, 1, 0]], dtype=torch.uint8), torch.full((1, 1, 1), 3.0), []

    def pack(v):
        kept.append(v.detach().clone())
        return len(kept) - 1

    with torch.autograd.graph.saved_tensors_hooks(pack, lambda i: kept[i]):
        y = through(name, StandIn(), x, *([] if name == "ffn" else [reset] + ([history] if name == "conv" else [])))
    with torch.no_grad():
        reset.fill_(1)
        history.zero_()
    y.sum().backward()
    scale, mask = (3.0 if name == "conv" else 1.0), torch.tensor([1.0, 1.0 if name == "ffn" else 0.0, 1.0]).view(1, 3, 1)
    assert torch.equal(x.grad, 2 * x.detach() * scale * mask)
    assert len(kept) >= (5 if name == "ffn" else 4)     # inputs, mask and history, the forward call's buffers


def test_an_agent_step_between_forward_and_backward_is_noticed(monkeypatch):
    """The step writes the history by address, which autograd does not see by itself."""
    op = StandIn()
    monkeypatch.setattr(ssm_policy.ssm, "Ssm", lambda *args, **kw: op)
    monkeypatch.setattr(ssm_policy.gated_ffn, "GatedFfn", lambda *args, **kw: op)
    layer = ssm_policy.Layer(8, 4, 4, 4, 16, "cpu", 0)
    state, history = torch.zeros((1, 16, 4)), torch.ones((1, 3, 16), dtype=torch.bfloat16)
    y = layer.sequence(torch.ones((1, 5, 8), dtype=torch.bfloat16, requires_grad=True), None, state, history)
    with torch.no_grad():
        layer.step(layer.weights(), torch.ones((1, 8), dtype=torch.bfloat16), None, state, history)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.float().sum().backward()


@pytest.mark.parametrize("name", ["scan", "ffn"])
def test_nothing_is_kept_where_no_gradient_is_wanted(name):
    op, x = StandIn(), inputs()
    want = through(name, op, x)
    assert want.requires_grad and op.asked == 1
    with torch.no_grad():
        assert torch.equal(through(name, op, x), want)
    assert torch.equal(through(name, op, x.detach()), want) and op.asked == 1
