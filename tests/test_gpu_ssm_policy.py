"""The state-space policy on Pong: its two forms agree, gradients move it, episodes stay apart."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    from paper_2603_12145_b200 import build
    build.build()
    return torch


def test_rollout_and_sequence_form_give_the_same_logits(torch):
    """The rollout takes tokens one by one, the training pass takes them in one piece.  Both round each
    layer's activations to bfloat16, at places whose binary32 inputs differ in the last bits: a value near
    a rounding boundary may go the other way (2^-8 relative), a handful of times per layer; the logits (head
    weights 0.1) then differ by far less than 0.02."""
    from paper_2603_12145_b200 import ssm_policy
    policy = ssm_policy.StateSpacePolicy(model=64, layers=2, ffn_hidden=72)
    trainer = ssm_policy.Trainer(policy, 40, 50, seed=3)
    for _ in range(3):          # the second and third start from a carried state
        before = trainer.rollout()
    # episodes that end inside the rollout: Pong's are long, so mark some by hand and roll out again
    with torch.no_grad():
        logits = policy.sequence(trainer.obs.transpose(0, 1), trainer.done[:-1].t(), before).transpose(0, 1)
    trainer.check()
    assert (logits - trainer.logits).abs().max().item() < 0.02
    assert trainer.logits.std().item() > 0.02        # the bound means something

    reset = (torch.rand((50, 40), device="cuda", generator=torch.Generator("cuda").manual_seed(1)) < 0.1).to(torch.uint8)
    carry, weights = [(s.clone(), h.clone()) for s, h in before], policy.weights()
    stepped = torch.stack([policy.step(trainer.obs[t], reset[t], carry, weights) for t in range(50)])
    with torch.no_grad():
        logits = policy.sequence(trainer.obs.transpose(0, 1), reset.t(), before).transpose(0, 1)
    assert (logits - stepped).abs().max().item() < 0.02


def test_a_reset_cuts_all_influence(torch):
    """Logits and gradients after a reset do not see what came before it."""
    from paper_2603_12145_b200 import ssm_policy
    policy = ssm_policy.StateSpacePolicy(model=64, layers=1, ffn_hidden=72)
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


def test_training_on_a_fixed_batch_lowers_its_loss(torch):
    from paper_2603_12145_b200 import ssm_policy
    torch.manual_seed(0)
    policy = ssm_policy.StateSpacePolicy(model=64, layers=2, ffn_hidden=128)
    trainer = ssm_policy.Trainer(policy, 64, 32, seed=5, learning_rate=1e-3)
    before = trainer.rollout()
    # a task for the memory: the action is the sign of an observation three steps ago
    target = (torch.roll(trainer.obs[..., 1], 3, dims=0) > 0.5).long()
    target[:3] = 0
    losses = []
    for _ in range(60):
        logits = policy.sequence(trainer.obs.transpose(0, 1), trainer.done[:-1].t(), before).transpose(0, 1)
        loss = torch.nn.functional.cross_entropy(logits.reshape(-1, 3), target.reshape(-1))
        trainer.optimizer.zero_grad(set_to_none=True)
        loss.backward()
        assert all(torch.isfinite(p.grad).all() for p in policy.parameters())
        trainer.optimizer.step()
        losses.append(loss.item())
    trainer.check()
    assert losses[-1] < 0.5 * losses[0], losses[::10]
    before = trainer.rollout()
    loss = trainer.update(before)
    assert np.isfinite(loss.item())
