"""What autograd sees of the training operators: the Functions of ssm_policy around stand-ins for the handles (plain torch on
the CPU), and the optimiser around one for the products; without a GPU."""
import copy
import pickle
import warnings

import pytest
import torch

from paper_2603_12145_b200 import optimizers, ssm_policy


class StandIn:
    """Element-wise operators with the handles' interfaces: y = x^2 (with a residual, of the sum)."""

    def __init__(self):
        self.asked = 0

    def saved(self, *sizes):
        self.asked += 1
        return torch.zeros(1)

    # layer_norm.LayerNorm
    def forward(self, x, w=None, b=None, residual=None, saved=None):
        if saved is not None:
            saved.fill_(2.0)
        s = x if residual is None else x + residual
        return s * s if residual is None else (s * s, s)

    def backward(self, dy, s, w, saved, dsum=None, want_params=True):
        dx = saved * s * dy + (0.0 if dsum is None else dsum)
        return dx, torch.ones_like(w) if want_params else None, torch.ones_like(w) if want_params else None


class RecurrenceStandIn(StandIn):
    def sequence(self, x, r, i, a, reset=None, state=None, state_out=None, saved=None):
        if saved is not None:
            saved.fill_(2.0)
        return x * x

    def backward(self, dy, x, r, i, a, saved, reset=None, dstate_out=None, want_dstate=False):
        mask = 1.0 if reset is None else (reset == 0).unsqueeze(-1)
        return {"dx": saved * x * dy * mask, "dr": torch.zeros_like(r), "di": torch.zeros_like(i), "da": torch.zeros_like(a), "dstate": None}


def through(name, x, op=None, reset=None):
    w = torch.zeros(1)
    if name == "norm":
        return ssm_policy.NormFunction.apply(op or StandIn(), x, None, w, w)
    if name == "added":
        return ssm_policy.NormFunction.apply(op or StandIn(), x, torch.zeros_like(x), w, w)[0]
    return ssm_policy.RecurrenceFunction.apply(op or RecurrenceStandIn(), x, x.detach(), x.detach(), w, reset, None, None)


def inputs():
    return torch.tensor([[[1.0], [2.0], [3.0]]], requires_grad=True)


@pytest.mark.parametrize("name", ["norm", "added", "recurrence"])
def test_first_derivatives_pass_and_second_ones_are_refused(name):
    x = inputs()
    (g,) = torch.autograd.grad((x * x + through(name, x)).sum(), x, create_graph=True)
    assert torch.equal(g, 4 * x)
    with pytest.raises(RuntimeError, match="first derivatives only"):
        torch.autograd.grad(g.sum(), x)
    scale = torch.tensor(3.0, requires_grad=True)
    (g,) = torch.autograd.grad((scale * through(name, x)).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="first derivatives only"):
        torch.autograd.grad(g.sum(), scale)


def test_both_results_of_the_norm_bring_their_gradients():
    """The rows alone, the stream alone, both; what needs no gradient gets none."""
    for use in ((1.0, 0.0), (0.0, 1.0), (1.0, 1.0)):
        x, r = inputs(), inputs()
        w, b = torch.zeros(1, requires_grad=True), torch.zeros(1)
        y, s = ssm_policy.NormFunction.apply(StandIn(), x, r, w, b)
        loss = sum(k * v.sum() for k, v in zip(use, (y, s)) if k)
        loss.backward()
        want = use[0] * 4 * x.detach() + use[1]                                # of (x + r)^2 and of x + r, with r = x
        assert torch.equal(x.grad, want) and torch.equal(r.grad, want)
        assert (w.grad is None) == (use[0] == 0.0) and b.grad is None


@pytest.mark.parametrize("name", ["norm", "added", "recurrence"])
def test_saved_tensor_hooks_see_all_that_the_backward_pass_reads(name):
    x, reset, kept = inputs(), torch.tensor([[0, 1, 0]], dtype=torch.uint8), []

    def pack(v):
        kept.append(v.detach().clone())
        return len(kept) - 1

    with torch.autograd.graph.saved_tensors_hooks(pack, lambda i: kept[i]):
        y = through(name, x, reset=reset)
    with torch.no_grad():
        reset.fill_(1)
    y.sum().backward()
    mask = torch.tensor([1.0, 0.0 if name == "recurrence" else 1.0, 1.0]).view(1, 3, 1)
    assert torch.equal(x.grad, 2 * x.detach() * mask)


def test_a_mask_changed_before_the_backward_pass_is_noticed():
    x, reset = inputs(), torch.tensor([[0, 1, 0]], dtype=torch.uint8)
    y = through("recurrence", x, reset=reset)
    reset.zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


@pytest.mark.parametrize("name", ["norm", "recurrence"])
def test_nothing_is_kept_where_no_gradient_is_wanted(name):
    op, x = (StandIn if name == "norm" else RecurrenceStandIn)(), inputs()
    want = through(name, x, op)
    assert want.requires_grad and op.asked == 1
    with torch.no_grad():
        assert torch.equal(through(name, x, op), want)
    assert torch.equal(through(name, x.detach(), op), want) and op.asked == 1


# ---- the optimiser ------------------------------------------------------------------------

def test_orthogonal_momentum_is_its_formula(monkeypatch):
    """Against the formula with a stand-in for the products; two shapes, one parameter without a gradient, a group of
    its own settings, state that survives saving."""
    class Halves:
        def __init__(self, rows, cols, dtype=None, steps=5, device=None):
            assert dtype is torch.float32

        def update(self, g):
            assert g.dim() == 3
            return (0.5 * g).to(torch.bfloat16)

        def status(self):
            pass

    monkeypatch.setattr(optimizers.orthogonal, "Orthogonal", Halves)
    gen = torch.Generator().manual_seed(0)
    p = [torch.nn.Parameter(torch.randn(s, generator=gen)) for s in ((8, 2), (8, 2), (3, 5), (2, 2))]
    opt = optimizers.OrthogonalMomentum([{"params": p[:2]}, {"params": p[2:], "nesterov": False, "weight_decay": 0.1}], lr=0.1, momentum=0.9)
    want, m = [v.detach().clone() for v in p], [torch.zeros_like(v) for v in p]
    for step in range(3):
        for j in range(3):
            g = torch.randn(p[j].shape, generator=gen)
            p[j].grad = g
            m[j] = 0.9 * m[j] + g
            u = g + 0.9 * m[j] if j < 2 else m[j]
            decay = 1.0 - 0.1 * 0.1 if j == 2 else 1.0
            want[j] = decay * want[j] - 0.1 * max(1.0, p[j].shape[0] / p[j].shape[1]) ** 0.5 * (0.5 * u).to(torch.bfloat16).float()
        opt.step()
        if step == 0:
            saved = opt.state_dict()
            opt.load_state_dict(saved)
    for a, b in zip(p, want):
        assert torch.allclose(a, b, rtol=1e-6, atol=1e-6)
    opt.check()
    for bad in ([torch.nn.Parameter(torch.zeros(3))], [torch.nn.Parameter(torch.zeros(2, 2, dtype=torch.float64))]):
        with pytest.raises(ValueError):
            optimizers.OrthogonalMomentum(bad)
    with pytest.raises(ValueError):
        optimizers.OrthogonalMomentum(p, momentum=1.0)


def test_orthogonal_momentum_is_copied_and_takes_no_parameter_twice(monkeypatch):
    class Whole:
        def __init__(self, *args, **kw):
            pass

        def update(self, g):
            return g.to(torch.bfloat16)

    monkeypatch.setattr(optimizers.orthogonal, "Orthogonal", Whole)
    p = torch.nn.Parameter(torch.ones(4, 4))
    opt = optimizers.OrthogonalMomentum([p], lr=0.5, momentum=0.0)
    for o in (opt, copy.deepcopy(opt), pickle.loads(pickle.dumps(opt))):
        q = o.param_groups[0]["params"][0]
        q.grad = torch.ones(4, 4)
        o.step()
        assert (q == 0.5).all()
    with warnings.catch_warnings():
        warnings.simplefilter("ignore")                # the base class warns
        with pytest.raises(ValueError):
            optimizers.OrthogonalMomentum([p, p])
