"""The policy of ssm_policy.py with its further parts: the gated recurrence as mixer, normalised branches, orthogonalised
momentum; and the training operators together as such a policy uses them, against autograd in binary64."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

VARIANTS = [("recurrence", False), ("recurrence", True), ("scan", True)]


@pytest.fixture(scope="module")
def torch():
    import torch
    from paper_2603_12145_b200 import build
    build.build()
    return torch


@pytest.mark.parametrize("mixer,norm", VARIANTS)
def test_rollout_and_sequence_form_give_the_same_logits(torch, mixer, norm):
    """The rollout takes tokens one by one, the training pass takes them in one piece.  Both round each layer's activations to
    bfloat16, at places whose binary32 inputs differ in the last bits: a value near a rounding boundary may go the
    other way (2^-8 relative), a handful of times per layer.  A logit is a product of 64 normalised (unnormalised: of about
    unit size) activations with weights of 0.1 / 8, so that one of them going the other way moves it by 0.1 / 8 * 2^-8; with
    four roundings per layer and unit all the other way it would move by 64 * 8 * 0.1 / 8 * 2^-8 = 0.025."""
    from paper_2603_12145_b200 import ssm_policy
    policy = ssm_policy.StateSpacePolicy(model=64, layers=2, ffn_hidden=72, mixer=mixer, norm=norm)
    trainer = ssm_policy.Trainer(policy, 40, 50, seed=3)
    for _ in range(2):          # the second starts from a carried state
        before = trainer.rollout()
    reset = (torch.rand((50, 40), device="cuda", generator=torch.Generator("cuda").manual_seed(1)) < 0.1).to(torch.uint8)
    carry, weights = [(s.clone(), h.clone()) for s, h in before], policy.weights()
    stepped = torch.stack([policy.step(trainer.obs[t], reset[t], carry, weights) for t in range(50)])
    with torch.no_grad():
        logits = policy.sequence(trainer.obs.transpose(0, 1), reset.t(), before).transpose(0, 1)
        same = policy.sequence(trainer.obs.transpose(0, 1), trainer.done[:-1].t(), before).transpose(0, 1)
    trainer.check()
    assert (logits - stepped).abs().max().item() < 0.025
    assert (same - trainer.logits).abs().max().item() < 0.025
    assert trainer.logits.std().item() > 0.02        # the bound means something


@pytest.mark.parametrize("mixer,norm", VARIANTS)
def test_a_reset_cuts_all_influence(torch, mixer, norm):
    """Logits and gradients after a reset do not see what came before it."""
    from paper_2603_12145_b200 import ssm_policy
    policy = ssm_policy.StateSpacePolicy(model=64, layers=2, ffn_hidden=72, mixer=mixer, norm=norm)
    obs = torch.randn((3, 20, 6), device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    reset = torch.zeros((3, 20), dtype=torch.uint8, device="cuda")
    reset[:, 9] = 1
    other = obs.clone()
    other[:, :9] = 5.0
    carry = policy.start(3)
    obs.requires_grad_(True)
    a = policy.sequence(obs, reset, carry)
    b = policy.sequence(other, reset, carry)
    assert torch.equal(a[:, 9:], b[:, 9:]) and not torch.equal(a[:, :9], b[:, :9])
    a[:, 9:].square().sum().backward()
    assert bool((obs.grad[:, :9] == 0).all()) and bool((obs.grad[:, 9:] != 0).any())


@pytest.mark.parametrize("mixer,norm,optimizer", [("recurrence", True, "orthogonal"), ("scan", False, "orthogonal"), ("recurrence", False, "adam")])
def test_a_training_step_runs_and_moves_every_parameter(torch, mixer, norm, optimizer):
    from paper_2603_12145_b200 import ssm_policy
    policy = ssm_policy.StateSpacePolicy(model=64, layers=2, ffn_hidden=128, mixer=mixer, norm=norm)
    trainer = ssm_policy.Trainer(policy, 32, 24, seed=5, optimizer=optimizer)
    before = {k: v.detach().clone() for k, v in policy.named_parameters()}
    start = trainer.rollout()
    # no point is won or lost in so few steps: every reward is zero, and so would be every gradient
    assert (trainer.reward == 0).all()
    trainer.reward.copy_(torch.randn((24, 32), device="cuda", generator=torch.Generator("cuda").manual_seed(9)))
    loss = trainer.update(start)
    trainer.check()
    assert np.isfinite(loss.item())
    for k, v in policy.named_parameters():
        assert torch.isfinite(v).all() and not torch.equal(v, before[k]), k
    if trainer.matrix_optimizer is not None:
        # a first step is the gradient's own update: momentum and its look ahead are multiples of it
        from oracle import training as tr
        w = policy.layers[0].w_in
        change = (before["layers.0.w_in"] - w.detach()).double() / (0.02 * max(1.0, w.shape[0] / w.shape[1]) ** 0.5)
        want = tr.orthogonal(w.grad.double().cpu().numpy())
        # (the update's bound for a gradient of few directions, see test_gpu_orthogonal.py, and 2^-24 of weights up to 1 in the change)
        assert np.linalg.norm(change.cpu().numpy() - want) <= 2 * (5.3e-3 + 2.0 ** -8) * np.linalg.norm(want) + 2.0 ** -24 * 50 * w.numel() ** 0.5


def test_default_policy_is_what_it_was(torch):
    """Without the new choices the same parameters in the same order with the same values."""
    from paper_2603_12145_b200 import ssm_policy
    policy = ssm_policy.StateSpacePolicy(model=64, layers=1)
    names = [k for k, _ in policy.named_parameters()]
    assert names == ["embed", "head"] + ["layers.0." + k for k in ("w_xz", "w_p", "w_dt", "w_y", "w_in", "w_out", "conv_w", "conv_b", "log_rate",
                                                                   "skip", "dt_bias")]
    gen = torch.Generator().manual_seed(1)
    assert torch.equal(policy.layers[0].w_xz.cpu(), torch.randn(256, 64, generator=gen) * 64 ** -0.5)


def plain_norm(torch, x, w, b):
    m = x.mean(-1, keepdim=True)
    return (x - m) / ((x - m).square().mean(-1, keepdim=True) + 1e-5).sqrt() * w + b


def plain_recurrence(torch, x, r, i, a, reset, state):
    h, out = state, []
    for t in range(x.shape[1]):
        h = h * (reset[:, t, None] == 0)
        L = a * torch.sigmoid(r[:, t])
        h = torch.exp(L) * h + torch.sqrt(-torch.expm1(2 * L)) * torch.sigmoid(i[:, t]) * x[:, t]
        out.append(h)
    return torch.stack(out, 1)


def test_the_operators_together_against_autograd(torch):
    """norm -> recurrence -> added norm -> loss in binary32, gradients of everything against autograd of the formulas in
    binary64; then the gradient of a weight through the orthogonalised update.  Each operator keeps its outputs within some 2^-18 of
    their size (the bounds of their own tests, with 24 steps); three in a row and back stay within 2^-14."""
    from oracle import training as tr
    from paper_2603_12145_b200 import gated_recurrence, layer_norm, orthogonal, ssm_policy
    g = torch.Generator("cuda").manual_seed(4)
    batch, time, ch = 5, 24, 96
    mk = lambda *s: torch.randn(s, generator=g, device="cuda")                             # noqa: E731
    leaves = {"h": mk(time, batch, ch), "w1": 1 + 0.1 * mk(ch), "b1": 0.1 * mk(ch), "wr": mk(ch, ch) / 10, "wi": mk(ch, ch) / 10,
              "log_rate": 0.5 * mk(ch) - 2, "w2": 1 + 0.1 * mk(ch), "b2": 0.1 * mk(ch)}
    reset = (torch.rand((batch, time), generator=g, device="cuda") < 0.1).to(torch.uint8)
    state, k1, k2 = mk(batch, ch), mk(time * batch, ch), mk(time * batch, ch)
    norm, rec = layer_norm.LayerNorm(ch, dtype=torch.float32), gated_recurrence.GatedRecurrence(ch, dtype=torch.float32)

    def run(v, plain):
        rows = v["h"].reshape(time * batch, ch)
        y = plain_norm(torch, rows, v["w1"], v["b1"]) if plain else ssm_policy.NormFunction.apply(norm, rows, None, v["w1"], v["b1"])
        x = y.view(time, batch, ch).transpose(0, 1)
        args = (x, x @ v["wr"].t(), x @ v["wi"].t(), -torch.exp(v["log_rate"]))
        m = (plain_recurrence(torch, *args, reset, state.double()) if plain
             else ssm_policy.RecurrenceFunction.apply(rec, *args, reset, state, None))
        m = m.transpose(0, 1).reshape(time * batch, ch)
        if plain:
            s = rows + m
            z = plain_norm(torch, s, v["w2"], v["b2"])
        else:
            z, s = ssm_policy.NormFunction.apply(norm, rows, m, v["w2"], v["b2"])
        return (z * k1.to(z.dtype)).sum() + (s * k2.to(s.dtype)).sin().sum()

    torch.backends.cuda.matmul.allow_tf32 = False
    own = {k: v.clone().requires_grad_(True) for k, v in leaves.items()}
    ref = {k: v.double().requires_grad_(True) for k, v in leaves.items()}
    a, b = run(own, False), run(ref, True)
    assert abs(a.item() - b.item()) <= 2.0 ** -14 * (k1.abs().sum() + k2.abs().sum()).item()
    a.backward()
    b.backward()
    for k in leaves:
        err = (own[k].grad.double() - ref[k].grad).norm() / ref[k].grad.norm()
        assert err.item() <= 2.0 ** -14, (k, err.item())
    op = orthogonal.Orthogonal(ch, ch, dtype=torch.float32)
    want = tr.orthogonal(own["wr"].grad.double().cpu().numpy())
    err = np.linalg.norm(op.update(own["wr"].grad).double().cpu().numpy() - want) / np.linalg.norm(want)
    assert err <= 5.3e-3 + 2.0 ** -8


def test_gradients_against_differences(torch):
    """Central differences of the policy's own forward pass, in binary32 handles, along random directions.  With a step of 2^-6 the
    difference quotient's third-order term is about 2^-12 of the slope; the outputs' roundings, 2^-20 of a loss of the slope's
    size, come to 2^-14: 2^-9 is allowed."""
    from paper_2603_12145_b200 import gated_recurrence, layer_norm, ssm_policy
    g = torch.Generator("cuda").manual_seed(7)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda")                             # noqa: E731
    rec, norm = gated_recurrence.GatedRecurrence(40, dtype=torch.float32), layer_norm.LayerNorm(40, dtype=torch.float32)
    x, r, i, dy = mk(3, 17, 40), mk(3, 17, 40), mk(3, 17, 40), mk(3, 17, 40)
    a, w, b = -torch.exp(0.5 * mk(40) - 1), 1 + 0.2 * mk(40), mk(40)
    reset = (torch.rand((3, 17), generator=g, device="cuda") < 0.2).to(torch.uint8)

    def f(x, r, i, a, w, b):
        y = ssm_policy.RecurrenceFunction.apply(rec, x, r, i, a, reset, None, None)
        return (ssm_policy.NormFunction.apply(norm, y.reshape(51, 40), None, w, b).view(3, 17, 40) * dy).double().sum()

    leaves = [v.clone().requires_grad_(True) for v in (x, r, i, a, w, b)]
    grads = torch.autograd.grad(f(*leaves), leaves)
    for k, gr in enumerate(grads):
        d = gr / gr.norm()                       # the steepest direction: the largest slope against the same roundings
        h = 2.0 ** -6 * (leaves[k].detach().norm().item() / leaves[k].numel() ** 0.5 + 0.1)
        up, down = [v.detach() for v in leaves], [v.detach() for v in leaves]
        up[k], down[k] = up[k] + h * d, down[k] - h * d
        slope = ((f(*up) - f(*down)) / (2 * h)).item()
        assert abs(slope - gr.norm().item()) <= 2.0 ** -9 * gr.norm().item() + 2.0 ** -9, (k, slope, gr.norm().item())
